"""ctypes binding of include/rnnt_greedy.h.  Argument marshalling only.

Tensors are anything with .data_ptr() (torch tensors on the GPU, fp32 / int32,
contiguous); torch is used for device memory and streams, nothing else.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))

RNNT_OK, RNNT_ERR_UNSUPPORTED = 0, -5
RNNT_DEV_LEN_CLAMPED, RNNT_DEV_OVERFLOW, RNNT_DEV_ABORTED = 1, 2, 4

EXPORTS = (
    "rnnt_engine_create", "rnnt_engine_destroy", "rnnt_greedy_decode",
    "rnnt_label_looping_decode", "tdt_label_looping_decode", "rnnt_encoder_projection",
    "rnnt_engine_status", "rnnt_engine_stats", "rnnt_engine_configure", "rnnt_status_string",
    "rnnt_engine_set_logp_output",
    "rnnt_engine_set_done_flags", "rnnt_engine_set_wait_limit",
    "rnnt_label_looping_decode_noalloc",
    "rnnt_engine_phase_timers",
    "rnnt_probe_stream", "rnnt_probe_exchange", "rnnt_probe_mfma", "rnnt_probe_e4m3_widening",
    "rnnt_quantize_rows_e4m3", "rnnt_quantize_blocks_e2m1", "rnnt_probe_e2m1_widening",
    "rnnt_probe_gate",
    "rnnt_mx4_sizes", "rnnt_mx4_quantize", "rnnt_mx4_product_workspace", "rnnt_mx4_product",
    "rnnt_beam_select_workspace", "rnnt_beam_select", "rnnt_beam_reorder",
)


RNNT_FLAG_BF16_WEIGHTS = 1
RNNT_FLAG_FP8_WEIGHTS = 2
RNNT_FLAG_PLAIN_LAUNCH = 4
RNNT_FLAG_BF16_ARITHMETIC = 8
RNNT_FLAG_MULTI_BLANK = 16
RNNT_FLAG_FP4_WEIGHTS = 32
RNNT_FLAG_COOPERATIVE_LAUNCH = 128
RNNT_FP4_BLOCK = 128
RNNT_MX4_BLOCK = 32
RNNT_BEAM_STATES = 16
RNNT_TYPE_F32, RNNT_TYPE_BF16, RNNT_TYPE_F16, RNNT_TYPE_MX4 = 0, 1, 2, 3
RNNT_TYPES = {"f32": RNNT_TYPE_F32, "bf16": RNNT_TYPE_BF16, "f16": RNNT_TYPE_F16, "mx4": RNNT_TYPE_MX4}


class RnntError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"rnnt_greedy error {code}: {text}")
        self.code = code


class _ModelDesc(C.Structure):
    _fields_ = [
        ("F", C.c_int32), ("E", C.c_int32), ("H", C.c_int32), ("L", C.c_int32),
        ("J", C.c_int32), ("V1", C.c_int32), ("blank", C.c_int32), ("D", C.c_int32),
        ("durations", C.POINTER(C.c_int32)),
        ("emb", C.c_void_p),
        ("w_ih", C.POINTER(C.c_void_p)), ("w_hh", C.POINTER(C.c_void_p)),
        ("b_ih", C.POINTER(C.c_void_p)), ("b_hh", C.POINTER(C.c_void_p)),
        ("w_enc", C.c_void_p), ("b_enc", C.c_void_p),
        ("w_pred", C.c_void_p), ("b_pred", C.c_void_p),
        ("w_out", C.c_void_p), ("b_out", C.c_void_p),
    ]


class _BeamState(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p)] + [(name, C.c_int64) for name in (
        "outer", "row_bytes", "src_outer", "src_batch", "src_beam", "dst_outer", "dst_batch", "dst_beam")]


class RnntStats(C.Structure):
    _fields_ = [
        ("pred_steps", C.c_int64), ("joint_steps", C.c_int64),
        ("max_pred_steps", C.c_int64), ("max_joint_steps", C.c_int64),
        ("joint_samples", C.c_int64), ("barrier_polls", C.c_int64),
        ("n_teams", C.c_int32), ("team_size", C.c_int32),
        ("lookahead", C.c_int32), ("xcd_mismatch", C.c_int32),
        ("joint_groups", C.c_int32), ("search_steps", C.c_int32),
        ("projection_ms", C.c_float), ("decode_ms", C.c_float),
    ]

    def as_dict(self) -> dict:
        return {name: (float(getattr(self, name)) if name.endswith("_ms")
                       else int(getattr(self, name))) for name, _ in self._fields_}


def lib_path() -> str:
    return os.path.join(HERE, "librnnt_greedy.so")


_LIB = None


def load_library():
    """Load librnnt_greedy.so; raise if it has not been built."""
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError(
                f"{path} is missing: build it with `python -m paper_2406_03791_amd.build` "
                "(there is no fallback path)")
        # PyTorch ships its own HIP runtime; it has to be in the process before this library
        # pulls in the system one, or the two runtimes disagree about the device.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        lib = C.CDLL(path)
        dec_args = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                    C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        lib.rnnt_engine_create.argtypes = [C.POINTER(_ModelDesc), C.c_int32, C.c_int32, C.c_int32,
                                           C.POINTER(C.c_void_p)]
        lib.rnnt_engine_destroy.argtypes = [C.c_void_p]
        lib.rnnt_greedy_decode.argtypes = dec_args + [C.c_void_p]
        lib.rnnt_label_looping_decode.argtypes = dec_args + [C.c_void_p]
        lib.rnnt_label_looping_decode_noalloc.argtypes = dec_args + [C.c_void_p]
        lib.tdt_label_looping_decode.argtypes = dec_args + [C.c_void_p, C.c_void_p]
        lib.rnnt_encoder_projection.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                                C.c_int32, C.c_void_p, C.c_void_p]
        lib.rnnt_engine_status.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        lib.rnnt_engine_stats.argtypes = [C.c_void_p, C.POINTER(RnntStats)]
        lib.rnnt_engine_configure.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        lib.rnnt_engine_set_logp_output.argtypes = [C.c_void_p, C.c_void_p]
        lib.rnnt_engine_set_done_flags.argtypes = [C.c_void_p, C.c_void_p]
        lib.rnnt_engine_set_wait_limit.argtypes = [C.c_void_p, C.c_int64]
        lib.rnnt_engine_phase_timers.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_double), C.c_int32]
        lib.rnnt_probe_stream.argtypes = [C.c_int32, C.POINTER(C.c_double), C.POINTER(C.c_double)]
        lib.rnnt_probe_exchange.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_double)]
        lib.rnnt_probe_mfma.argtypes = [C.c_int32, C.POINTER(C.c_double)]
        lib.rnnt_probe_e4m3_widening.argtypes = [C.c_float, C.POINTER(C.c_uint16)]
        for name in ("rnnt_quantize_rows_e4m3", "rnnt_quantize_blocks_e2m1"):
            getattr(lib, name).argtypes = [C.POINTER(C.c_float), C.c_int64, C.c_int64,
                                           C.POINTER(C.c_float), C.POINTER(C.c_float)]
        lib.rnnt_probe_e2m1_widening.argtypes = [C.c_float, C.POINTER(C.c_uint16)]
        lib.rnnt_probe_gate.argtypes = [C.c_int32, C.POINTER(C.c_float), C.c_int64, C.POINTER(C.c_float)]
        i32, i64, ptr, out64 = C.c_int32, C.c_int64, C.c_void_p, C.POINTER(C.c_int64)
        lib.rnnt_mx4_sizes.argtypes = [i64, i64, out64, out64]
        lib.rnnt_mx4_quantize.argtypes = [ptr, i32, i64, i64, i64, ptr, ptr, ptr, ptr]
        lib.rnnt_mx4_product_workspace.argtypes = [i32, i64, i64, i64, out64]
        lib.rnnt_mx4_product.argtypes = [ptr, ptr, i32, i64, ptr, ptr, ptr, ptr, i32, i64, i64, i64, i64, ptr, i64, ptr]
        lib.rnnt_beam_select_workspace.argtypes = [i32, i32, i32, i32, out64]
        lib.rnnt_beam_select.argtypes = [ptr, i32, i64, i64, ptr, ptr, i32, i32, i32, i32, i32, ptr, ptr, ptr, ptr, i64, ptr]
        lib.rnnt_beam_reorder.argtypes = [C.POINTER(_BeamState), i32, ptr, i32, i32, i32, ptr]
        lib.rnnt_status_string.argtypes = [C.c_int]
        lib.rnnt_status_string.restype = C.c_char_p
        for name in EXPORTS:
            if name != "rnnt_status_string":
                getattr(lib, name).restype = C.c_int
        _LIB = lib
    return _LIB


def rnnt_status_string(code: int) -> str:
    return load_library().rnnt_status_string(int(code)).decode()


def _check(code: int) -> None:
    if code != RNNT_OK:
        raise RnntError(code, rnnt_status_string(code))


def _p(t) -> Optional[int]:
    return None if t is None else C.c_void_p(t.data_ptr())


def rnnt_engine_create(dims, weights: dict, max_B: int, max_T: int, flags: int = 0):
    """dims: object with F, E, H, L, J, V1, blank, durations; weights: name ->
    device tensor (emb, w_ih0.., w_hh0.., b_ih0.., b_hh0.., w_enc, b_enc, w_pred,
    b_pred, w_out, b_out).  Returns the engine handle."""
    L = int(dims.L)
    dur = list(dims.durations)
    # a multi-blank model's extra output columns are its big blanks: their spans travel in the
    # descriptor's durations and the flag says what they are
    spans = list(getattr(dims, "big_blanks", ()))
    if spans:
        assert not dur, "a model has durations or big blanks, not both"
        dur, flags = spans, flags | RNNT_FLAG_MULTI_BLANK
    d = _ModelDesc()
    d.F, d.E, d.H, d.L, d.J, d.V1 = int(dims.F), int(dims.E), int(dims.H), L, int(dims.J), int(dims.V1)
    d.blank, d.D = int(dims.blank), len(dur)
    dur_arr = (C.c_int32 * max(1, len(dur)))(*dur)
    d.durations = C.cast(dur_arr, C.POINTER(C.c_int32))
    arrs = {}
    for key in ("w_ih", "w_hh", "b_ih", "b_hh"):
        arrs[key] = (C.c_void_p * L)(*[weights[f"{key}{l}"].data_ptr() for l in range(L)])
        setattr(d, key, C.cast(arrs[key], C.POINTER(C.c_void_p)))
    for key in ("emb", "w_enc", "b_enc", "w_pred", "b_pred", "w_out", "b_out"):
        setattr(d, key, weights[key].data_ptr())
    out = C.c_void_p()
    _check(load_library().rnnt_engine_create(C.byref(d), int(max_B), int(max_T), int(flags),
                                             C.byref(out)))
    return out


def rnnt_engine_destroy(eng) -> None:
    _check(load_library().rnnt_engine_destroy(eng))


def rnnt_engine_set_logp_output(eng, logp_out) -> None:
    _check(load_library().rnnt_engine_set_logp_output(eng, _p(logp_out)))


def rnnt_engine_set_done_flags(eng, done) -> None:
    _check(load_library().rnnt_engine_set_done_flags(eng, _p(done)))


def rnnt_engine_set_wait_limit(eng, polls: int = -1) -> None:
    _check(load_library().rnnt_engine_set_wait_limit(eng, int(polls)))


def rnnt_engine_configure(eng, n_teams: int = 0, joint_groups: int = 0, lookahead: int = 0,
                          search_steps: int = 0) -> None:
    _check(load_library().rnnt_engine_configure(eng, int(n_teams), int(joint_groups),
                                                int(lookahead), int(search_steps)))


def _decode(fn, eng, enc_out, enc_len, B, T, max_symbols, tokens_out, tok_len_out, cap,
            frames_out, logit_out, extra, stream):
    args = [eng, _p(enc_out), _p(enc_len), int(B), int(T), int(max_symbols), _p(tokens_out),
            _p(tok_len_out), int(cap), _p(frames_out), _p(logit_out)]
    args += extra
    args.append(C.c_void_p(stream) if stream else None)
    _check(fn(*args))


def rnnt_greedy_decode(eng, enc_out, enc_len, B, T, max_symbols, tokens_out, tok_len_out, cap,
                       frames_out=None, logit_out=None, stream: int = 0) -> None:
    _decode(load_library().rnnt_greedy_decode, eng, enc_out, enc_len, B, T, max_symbols,
            tokens_out, tok_len_out, cap, frames_out, logit_out, [], stream)


def rnnt_label_looping_decode(eng, enc_out, enc_len, B, T, max_symbols, tokens_out, tok_len_out,
                              cap, frames_out=None, logit_out=None, stream: int = 0) -> None:
    _decode(load_library().rnnt_label_looping_decode, eng, enc_out, enc_len, B, T, max_symbols,
            tokens_out, tok_len_out, cap, frames_out, logit_out, [], stream)


def rnnt_label_looping_decode_noalloc(eng, enc_out, enc_len, B, T, max_symbols, tokens_out,
                                      tok_len_out, cap, frames_out=None, logit_out=None,
                                      stream: int = 0) -> None:
    _decode(load_library().rnnt_label_looping_decode_noalloc, eng, enc_out, enc_len, B, T,
            max_symbols, tokens_out, tok_len_out, cap, frames_out, logit_out, [], stream)


def tdt_label_looping_decode(eng, enc_out, enc_len, B, T, max_symbols, tokens_out, tok_len_out,
                             cap, frames_out=None, logit_out=None, durations_out=None,
                             stream: int = 0) -> None:
    _decode(load_library().tdt_label_looping_decode, eng, enc_out, enc_len, B, T, max_symbols,
            tokens_out, tok_len_out, cap, frames_out, logit_out, [_p(durations_out)], stream)


def rnnt_encoder_projection(eng, enc_out, enc_len, B, T, proj_out, stream: int = 0) -> None:
    _check(load_library().rnnt_encoder_projection(eng, _p(enc_out), _p(enc_len), int(B), int(T),
                                                  _p(proj_out),
                                                  C.c_void_p(stream) if stream else None))


def rnnt_engine_status(eng) -> int:
    out = C.c_int32(0)
    _check(load_library().rnnt_engine_status(eng, C.byref(out)))
    return int(out.value)


def rnnt_engine_phase_timers(eng, team: int, n: int = 24):
    """Microseconds per phase for rank 0 of `team` (profile builds only)."""
    out = (C.c_double * n)()
    _check(load_library().rnnt_engine_phase_timers(eng, int(team), out, int(n)))
    return [float(v) for v in out]


def rnnt_probe_stream(from_l2: bool):
    """(GB/s over the device, GB/s per compute unit)"""
    a, b = C.c_double(0), C.c_double(0)
    _check(load_library().rnnt_probe_stream(int(bool(from_l2)), C.byref(a), C.byref(b)))
    return float(a.value), float(b.value)


def rnnt_probe_exchange(team_size: int, length: int, tagged: bool) -> float:
    out = C.c_double(0)
    _check(load_library().rnnt_probe_exchange(int(team_size), int(length), int(bool(tagged)), C.byref(out)))
    return float(out.value)


def rnnt_probe_e4m3_widening(scale: float = 1.0):
    """[4][256] uint16 array: the bf16 code each e4m3 code becomes under the scale operand,
    per byte position."""
    import numpy as np
    out = np.zeros((4, 256), dtype=np.uint16)
    _check(load_library().rnnt_probe_e4m3_widening(C.c_float(scale), out.ctypes.data_as(C.POINTER(C.c_uint16))))
    return out


def rnnt_quantize_rows_e4m3(w):
    """(quantised copy, row scales) of a 2-D float32 numpy array: every row as e4m3 values
    times a power of two (host-side helper of the library, no device work)."""
    import numpy as np
    w = np.ascontiguousarray(w, dtype=np.float32)
    assert w.ndim == 2
    out = np.empty_like(w)
    scales = np.empty(w.shape[0], dtype=np.float32)
    fp = C.POINTER(C.c_float)
    _check(load_library().rnnt_quantize_rows_e4m3(w.ctypes.data_as(fp), w.shape[0], w.shape[1],
                                                  out.ctypes.data_as(fp), scales.ctypes.data_as(fp)))
    return out, scales


def rnnt_quantize_blocks_e2m1(w):
    """(quantised copy, block scales [rows, ceil(cols / 128)]) of a 2-D float32 numpy array:
    every block of 128 consecutive weights of a row as e2m1 values times a power of two."""
    import numpy as np
    w = np.ascontiguousarray(w, dtype=np.float32)
    assert w.ndim == 2
    out = np.empty_like(w)
    scales = np.empty((w.shape[0], (w.shape[1] + RNNT_FP4_BLOCK - 1) // RNNT_FP4_BLOCK), dtype=np.float32)
    fp = C.POINTER(C.c_float)
    _check(load_library().rnnt_quantize_blocks_e2m1(w.ctypes.data_as(fp), w.shape[0], w.shape[1],
                                                    out.ctypes.data_as(fp), scales.ctypes.data_as(fp)))
    return out, scales


def rnnt_probe_e2m1_widening(scale: float = 1.0):
    """[4][256][2] uint16 array: the two bf16 codes a byte of two e2m1 codes becomes under the
    scale operand, per byte position (low nibble first)."""
    import numpy as np
    out = np.zeros((4, 256, 2), dtype=np.uint16)
    _check(load_library().rnnt_probe_e2m1_widening(C.c_float(scale), out.ctypes.data_as(C.POINTER(C.c_uint16))))
    return out


def rnnt_probe_gate(is_tanh: bool, x):
    """sigmoid or tanh of a float32 numpy array as the resident decode kernel computes them."""
    import numpy as np
    x = np.ascontiguousarray(x, dtype=np.float32)
    out = np.empty_like(x)
    fp = C.POINTER(C.c_float)
    _check(load_library().rnnt_probe_gate(int(bool(is_tanh)), x.ctypes.data_as(fp), x.size, out.ctypes.data_as(fp)))
    return out


def rnnt_mx4_sizes(rows: int, cols: int):
    """(bytes of the codes, bytes of the scales) of a microscaled 4-bit matrix."""
    a, b = C.c_int64(0), C.c_int64(0)
    _check(load_library().rnnt_mx4_sizes(rows, cols, C.byref(a), C.byref(b)))
    return a.value, b.value


def _a(t):
    """A tensor's address as ctypes takes it."""
    return None if t is None else t.data_ptr()


def rnnt_mx4_quantize(x, type, rows, cols, x_stride, codes, scales, values=None, stream: int = 0) -> None:
    _check(load_library().rnnt_mx4_quantize(_a(x), type, rows, cols, x_stride, _a(codes), _a(scales), _a(values),
                                            stream or None))


def rnnt_mx4_product_workspace(a_type: int, M: int, N: int, K: int) -> int:
    out = C.c_int64(0)
    _check(load_library().rnnt_mx4_product_workspace(a_type, M, N, K, C.byref(out)))
    return out.value


def rnnt_mx4_product(a, a_scales, a_type, a_stride, w_codes, w_scales, bias, y, y_type, y_stride, M, N, K,
                     workspace=None, workspace_bytes=0, stream: int = 0) -> None:
    _check(load_library().rnnt_mx4_product(_a(a), _a(a_scales), a_type, a_stride, _a(w_codes), _a(w_scales), _a(bias),
                                           _a(y), y_type, y_stride, M, N, K, _a(workspace), workspace_bytes,
                                           stream or None))


def _counts(*counts) -> None:
    """Refuses what an int32 argument does not hold: ctypes would cut it off."""
    if any(not -0x80000000 <= n <= 0x7fffffff for n in counts):
        raise RnntError(RNNT_ERR_UNSUPPORTED, f"a count of {counts} is beyond 32 bits")


def rnnt_beam_select_workspace(B: int, beams: int, V: int, n_out: int) -> int:
    if (B | beams | V | n_out) >> 31:
        _counts(B, beams, V, n_out)
    out = C.c_int64(0)
    _check(load_library().rnnt_beam_select_workspace(B, beams, V, n_out, C.byref(out)))
    return out.value


def rnnt_beam_select(logits, type, batch_stride, beam_stride, scores, finished, B, beams, V, n_out, end_token,
                     scores_out, tokens_out, parents_out, workspace=None, workspace_bytes=0, stream: int = 0) -> None:
    if (B | beams | V | n_out | end_token) >> 31:
        _counts(B, beams, V, n_out, end_token)
    _check(load_library().rnnt_beam_select(_a(logits), type, batch_stride, beam_stride, _a(scores), _a(finished),
                                           B, beams, V, n_out, end_token, _a(scores_out), _a(tokens_out),
                                           _a(parents_out), _a(workspace), workspace_bytes, stream or None))


class BeamStates:
    """What rnnt_beam_reorder moves: the C descriptors of pairs of tensors, and the tensors, kept alive."""

    def __init__(self, pairs):
        self.pairs = [(s, d) for s, d in pairs]
        self.array = (_BeamState * max(1, len(self.pairs)))(*[_beam_state(s, d) for s, d in self.pairs])


def _outer(t):
    """(number, stride) of the rows of a tensor [..., B, beams, row] along its leading axes, which have to be as one."""
    n, stride = 1, 0
    for size, st in reversed(list(zip(t.shape[:-3], t.stride()[:-3]))):
        if size == 1:
            continue
        if n > 1 and st != n * stride:
            raise ValueError("the leading axes of a state have to have one stride between them")
        n, stride = n * size, stride if n > 1 else st
    return n, stride


def _beam_state(src, dst):
    if src.dim() < 3 or dst.dim() != src.dim() or src.dtype != dst.dtype or src.device != dst.device:
        raise ValueError("states are pairs of tensors [..., B, beams, row] of one type on one device")
    if src.shape[:-2] != dst.shape[:-2] or src.shape[-1] != dst.shape[-1]:
        raise ValueError(f"states differ in more than the beams: {tuple(src.shape)} and {tuple(dst.shape)}")
    if src.shape[-1] > 1 and (src.stride(-1) != 1 or dst.stride(-1) != 1):
        raise ValueError("rows of a state have to be contiguous")
    e, (n, so), (_, do) = src.element_size(), _outer(src), _outer(dst)
    return _BeamState(src.data_ptr(), dst.data_ptr(), n if src.numel() or dst.numel() else 0, e * src.shape[-1],
                      e * so, e * src.stride(-3), e * src.stride(-2), e * do, e * dst.stride(-3), e * dst.stride(-2))


def rnnt_beam_states(pairs) -> BeamStates:
    """Descriptors for rnnt_beam_reorder of (source, destination) tensors [..., B, beams, row]; a
    destination may be its source."""
    return BeamStates(pairs)


def rnnt_beam_reorder(states, parents, B, beams_in, beams_out, stream: int = 0) -> None:
    """states: of rnnt_beam_states, to be used again as long as the tensors stay where they are."""
    if (B | beams_in | beams_out) >> 31:
        _counts(B, beams_in, beams_out)
    _check(load_library().rnnt_beam_reorder(states.array, len(states.pairs), _a(parents), B, beams_in, beams_out,
                                            stream or None))


def rnnt_probe_mfma(shape: int) -> float:
    out = C.c_double(0)
    _check(load_library().rnnt_probe_mfma(int(shape), C.byref(out)))
    return float(out.value)


def rnnt_engine_stats(eng) -> RnntStats:
    out = RnntStats()
    _check(load_library().rnnt_engine_stats(eng, C.byref(out)))
    return out


class Engine:
    """Convenience owner of an engine handle plus output allocation with torch.
    Holds no decode logic: each method forwards to the C entry point of the
    same name."""

    def __init__(self, model, max_B: int, max_T: int, device: str = "cuda:0", flags: int = 0):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.dims = model.dims
        self.weights = {k: torch.from_numpy(v).to(self.device).contiguous()
                        for k, v in model.arrays().items()}
        torch.cuda.synchronize(self.device)
        self.handle = rnnt_engine_create(self.dims, self.weights, max_B, max_T, flags)

    def close(self) -> None:
        if getattr(self, "handle", None):
            rnnt_engine_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def configure(self, n_teams: int = 0, joint_groups: int = 0, lookahead: int = 0,
                  search_steps: int = 0) -> None:
        rnnt_engine_configure(self.handle, n_teams, joint_groups, lookahead, search_steps)

    def set_wait_limit(self, polls: int = -1) -> None:
        """Polls a device-side wait may repeat before the call gives up (-1 = default)."""
        rnnt_engine_set_wait_limit(self.handle, polls)

    def alloc_outputs(self, B: int, cap: int, pinned: bool = False):
        """Output tensors on the device, or (pinned=True) in pinned host memory,
        which a host thread can read while a decode call runs."""
        t = self.torch
        kw = dict(pin_memory=True) if pinned else dict(device=self.device)
        out = dict(tokens=t.empty((B, cap), dtype=t.int32, **kw),
                   tok_len=t.empty((B,), dtype=t.int32, **kw),
                   frames=t.empty((B, cap), dtype=t.int32, **kw),
                   logits=t.empty((B, cap), dtype=t.float32, **kw))
        if self.dims.D:
            out["durs"] = t.empty((B, cap), dtype=t.int32, **kw)
        return out

    def decode(self, variant: str, enc_out, enc_len, max_symbols: int, out=None,
               cap: Optional[int] = None, logp: bool = False, done=None):
        """enc_out [B,T,F] fp32 and enc_len [B] int32 device tensors.  Queues the
        decode on the current stream and returns the output tensors (device).
        logp=True also asks for the log-probabilities (out["logps"]); done is an
        int32 [B] tensor of completion flags the caller has zeroed."""
        B, T = int(enc_out.shape[0]), int(enc_out.shape[1])
        if cap is None:
            cap = T * max_symbols
        if out is None:
            out = self.alloc_outputs(B, cap)
        if logp and "logps" not in out:
            out["logps"] = self.torch.empty((B, cap), dtype=self.torch.float32, device=self.device)
        rnnt_engine_set_logp_output(self.handle, out["logps"] if logp else None)
        rnnt_engine_set_done_flags(self.handle, done)
        stream = self.torch.cuda.current_stream(self.device).cuda_stream
        common = (self.handle, enc_out, enc_len, B, T, max_symbols, out["tokens"], out["tok_len"],
                  cap, out["frames"], out["logits"])
        if variant == "frame":
            rnnt_greedy_decode(*common, stream=stream)
        elif variant == "label":
            rnnt_label_looping_decode(*common, stream=stream)
        elif variant == "label_noalloc":
            rnnt_label_looping_decode_noalloc(*common, stream=stream)
        elif variant == "tdt":
            tdt_label_looping_decode(*common, durations_out=out.get("durs"), stream=stream)
        else:
            raise ValueError(variant)
        return out

    def encoder_projection(self, enc_out, enc_len):
        B, T = int(enc_out.shape[0]), int(enc_out.shape[1])
        proj = self.torch.zeros((B, T, self.dims.J), dtype=self.torch.float32, device=self.device)
        stream = self.torch.cuda.current_stream(self.device).cuda_stream
        rnnt_encoder_projection(self.handle, enc_out, enc_len, B, T, proj, stream)
        return proj

    def status(self) -> int:
        return rnnt_engine_status(self.handle)

    def stats(self) -> dict:
        return rnnt_engine_stats(self.handle).as_dict()

    def phase_timers(self, team: int, n: int = 24):
        return rnnt_engine_phase_timers(self.handle, team, n)


def _type_of(t) -> int:
    name = {"torch.float32": "f32", "torch.bfloat16": "bf16", "torch.float16": "f16"}.get(str(t.dtype))
    if name is None:
        raise TypeError(f"float32, bfloat16 or float16 is wanted, not {t.dtype}")
    return RNNT_TYPES[name]


def _on_device(first, *others):
    """The device of tensors that have to share one."""
    if first.device.type != "cuda":
        raise ValueError(f"tensors on the GPU are wanted, not on {first.device}")
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError(f"tensors on one device are wanted, not on {first.device} and {t.device}")
    return first.device


def _no_gradients(*tensors) -> None:
    """Refuses operands that a gradient is to be recorded for: the operators have no backward pass."""
    import torch
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError("an operand requires a gradient, and this operator has none: call it under torch.no_grad() or on detached tensors")


def _workspace(given, need: int, device):
    """A workspace of at least `need` bytes and its size: the given one, or a new one."""
    import torch
    if given is None:
        return (torch.empty(need, dtype=torch.uint8, device=device), need) if need else (None, 0)
    if given.dtype != torch.uint8 or not given.is_contiguous():
        raise ValueError("workspace: a contiguous uint8 tensor is wanted")
    return given, given.numel()


def _rows_of(t, what: str):
    """The row stride of a matrix whose rows are contiguous."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: a matrix with contiguous rows is wanted")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


class Mx4Matrix:
    """Owner of a microscaled 4-bit matrix [rows, cols]: codes and scales as rnnt_mx4_quantize lays them out.
    Like Engine it holds no arithmetic: the methods allocate with torch, run on the current stream of the
    tensors' device and forward to the C entry points."""

    def __init__(self, rows: int, cols: int, device):
        import torch
        self.rows, self.cols = int(rows), int(cols)
        codes, scales = rnnt_mx4_sizes(self.rows, self.cols)
        self.codes = torch.empty(codes, dtype=torch.uint8, device=device)
        self.scales = torch.empty(scales, dtype=torch.uint8, device=device)

    @property
    def device(self):
        return self.codes.device

    def quantize(self, x, values=None) -> "Mx4Matrix":
        """Quantise x [rows, cols] (float32, bfloat16 or float16, contiguous rows) into this matrix; values: a
        contiguous float32 tensor [rows, cols] for what the codes stand for."""
        import torch
        stride = _rows_of(x, "x")
        if tuple(x.shape) != (self.rows, self.cols):
            raise ValueError(f"x is {tuple(x.shape)}, the matrix {(self.rows, self.cols)}")
        if values is not None and (values.dtype != torch.float32 or values.shape != x.shape or not values.is_contiguous()):
            raise ValueError("values: a contiguous float32 tensor of the matrix' size is wanted")
        if values is not None:                             # (codes alone are integers)
            _no_gradients(x, values)
        with torch.cuda.device(_on_device(x, self.codes, values)):
            rnnt_mx4_quantize(x, _type_of(x), self.rows, self.cols, stride, self.codes, self.scales, values,
                              torch.cuda.current_stream().cuda_stream)
        return self

    def product(self, a, bias=None, out=None, dtype=None, workspace=None):
        """Q(a) of this matrix transposed, plus bias [rows]: [M, rows] of `dtype` (float32 if not given) or in
        `out`.  a: a tensor [M, cols] or an Mx4Matrix.  workspace: a uint8 tensor to be used instead of a new one."""
        import torch
        quantised = isinstance(a, Mx4Matrix)
        stride, a_type = (a.cols, RNNT_TYPE_MX4) if quantised else (_rows_of(a, "a"), _type_of(a))
        M, cols = (a.rows, a.cols) if quantised else a.shape
        codes, scales = (a.codes, a.scales) if quantised else (a, None)
        if cols != self.cols:
            raise ValueError(f"a has {cols} columns, the matrix {self.cols}")
        if bias is not None and (bias.dtype != torch.float32 or tuple(bias.shape) != (self.rows,) or not bias.is_contiguous()):
            raise ValueError("bias: a contiguous float32 vector of the matrix' rows is wanted")
        _no_gradients(codes, bias, out)
        device = _on_device(codes, scales, self.codes, bias, out, workspace)
        if out is None:
            out = torch.empty((M, self.rows), dtype=dtype or torch.float32, device=device)
        elif tuple(out.shape) != (M, self.rows) or (dtype is not None and out.dtype != dtype):
            raise ValueError(f"out: a {dtype or 'float'} matrix {(M, self.rows)} is wanted")
        out_stride, out_type = _rows_of(out, "out"), _type_of(out)
        workspace, space = _workspace(workspace, rnnt_mx4_product_workspace(a_type, M, self.rows, self.cols), device)
        with torch.cuda.device(device):
            rnnt_mx4_product(codes, scales, a_type, stride, self.codes, self.scales, bias, out, out_type, out_stride,
                             M, self.rows, self.cols, workspace, space, torch.cuda.current_stream().cuda_stream)
        return out


def mx4_quantize(x) -> Mx4Matrix:
    """A new microscaled 4-bit copy of a matrix."""
    _rows_of(x, "x")
    return Mx4Matrix(x.shape[0], x.shape[1], x.device).quantize(x)


def beam_select(logits, scores, n_out: Optional[int] = None, finished=None, end_token: int = 0, workspace=None):
    """The n_out (by default as many as there are beams) best continuations of every utterance:
    (scores, tokens, parents), tensors [B, n_out].  logits [B, beams, V], float32, bfloat16 or float16, contiguous
    rows; scores [B, beams] float32; finished [B, beams] uint8 or bool (rnnt_beam_select)."""
    import torch
    if logits.dim() != 3 or (logits.shape[2] > 1 and logits.stride(2) != 1):
        raise ValueError("logits: a tensor [B, beams, V] with contiguous rows is wanted")
    B, beams, V = logits.shape
    n_out = beams if n_out is None else int(n_out)
    if scores.dtype != torch.float32 or tuple(scores.shape) != (B, beams) or not scores.is_contiguous():
        raise ValueError("scores: a contiguous float32 tensor [B, beams] is wanted")
    if finished is not None and (finished.dtype not in (torch.uint8, torch.bool) or tuple(finished.shape) != (B, beams)
                                 or not finished.is_contiguous()):
        raise ValueError("finished: a contiguous uint8 or bool tensor [B, beams] is wanted")
    _no_gradients(logits, scores)
    device = _on_device(logits, scores, finished, workspace)
    workspace, space = _workspace(workspace, rnnt_beam_select_workspace(B, beams, V, n_out), device)
    best = torch.empty((B, n_out), dtype=torch.float32, device=device)
    tokens, parents = torch.empty((2, B, n_out), dtype=torch.int32, device=device)
    with torch.cuda.device(device):
        rnnt_beam_select(logits, _type_of(logits), logits.stride(0), logits.stride(1), scores, finished, B, beams, V,
                         n_out, int(end_token), best, tokens, parents, workspace, space,
                         torch.cuda.current_stream().cuda_stream)
    return best, tokens, parents


def beam_reorder(pairs, parents) -> None:
    """States follow the hypotheses: for every (source, destination) of `pairs` (or of a kept
    rnnt_beam_states), tensors [..., B, beams, row], the destination's row of hypothesis j becomes the source's row of
    hypothesis parents[b, j], zeros where there is none.  A destination may be its source."""
    import torch
    states = pairs if isinstance(pairs, BeamStates) else rnnt_beam_states(pairs)
    if not states.pairs:
        return
    if parents.dtype != torch.int32 or parents.dim() != 2 or not parents.is_contiguous():
        raise ValueError("parents: a contiguous int32 tensor [B, beams] is wanted")
    (B, beams_out), beams_in = parents.shape, states.pairs[0][0].shape[-2]
    moved = [t for pair in states.pairs for t in pair]
    _no_gradients(*moved)
    device = _on_device(parents, *moved)
    for src, dst in states.pairs:
        if tuple(src.shape[-3:-1]) != (B, beams_in) or tuple(dst.shape[-3:-1]) != (B, beams_out):
            raise ValueError(f"states of {B} utterances, {beams_in} and {beams_out} beams are wanted, not "
                             f"{tuple(src.shape)} and {tuple(dst.shape)}")
    with torch.cuda.device(device):
        rnnt_beam_reorder(states, parents, B, beams_in, beams_out, torch.cuda.current_stream().cuda_stream)

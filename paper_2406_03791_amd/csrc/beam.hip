// A beam search's step over hypotheses: selection over beams and vocabulary, and states that follow it.
#include "../../include/rnnt_greedy.h"

#include <hip/hip_runtime.h>

#include <math.h>

#include "engine.h"

namespace rnnt {

constexpr int kMaxBeams = 64;

struct SelectArgs {
    const void *logits;
    const float *scores;
    const unsigned char *finished;
    float *scores_out;
    int *tokens_out, *parents_out;
    long long batch_stride, beam_stride;
    int beams, V, n_out, end_token;
};

template <int TYPE>
__device__ __forceinline__ float logit(const void *p, long long at)
{
    if constexpr (TYPE == RNNT_TYPE_F32) return static_cast<const float *>(p)[at];
    else if constexpr (TYPE == RNNT_TYPE_BF16) return (float)static_cast<const __bf16 *>(p)[at];
    else return (float)static_cast<const _Float16 *>(p)[at];
}

// A work-group an utterance.  The largest logit and the sum of a hypothesis first, then winner by winner the best of
// what comes behind the last one.
template <int TYPE>
__global__ void __launch_bounds__(256)
beam_select_kernel(const SelectArgs a)
{
    __shared__ double base[kMaxBeams];                 // of a hypothesis: its score less the logarithm of the sum
    __shared__ float top[kMaxBeams];
    __shared__ double s_best[256];
    __shared__ float s_logit[256];
    __shared__ int s_at[256];
    const int b = blockIdx.x, tid = threadIdx.x;
    const float *scores = a.scores + (long long)b * a.beams;
    for (int k = 0; k < a.beams; ++k) {
        const long long row = b * a.batch_stride + k * a.beam_stride;
        float m = -INFINITY;
        bool nan = false;
        for (int v = tid; v < a.V; v += 256) { const float x = logit<TYPE>(a.logits, row + v); nan = nan || x != x; m = fmaxf(m, x); }
        s_logit[tid] = nan ? INFINITY : m;
        __syncthreads();
        for (int h = 128; h > 0; h >>= 1) { if (tid < h) s_logit[tid] = fmaxf(s_logit[tid], s_logit[tid + h]); __syncthreads(); }
        m = s_logit[0];
        double sum = 0;
        if (m < INFINITY && m > -INFINITY)
            for (int v = tid; v < a.V; v += 256) sum += exp((double)logit<TYPE>(a.logits, row + v) - (double)m);
        s_best[tid] = sum;
        __syncthreads();
        for (int h = 128; h > 0; h >>= 1) { if (tid < h) s_best[tid] += s_best[tid + h]; __syncthreads(); }
        // (no candidates: the score becomes -inf)
        if (tid == 0) { top[k] = m; base[k] = m < INFINITY && m > -INFINITY ? (double)scores[k] - log(s_best[0]) : -INFINITY; }
        __syncthreads();
    }
    double last = INFINITY;
    float last_x = INFINITY;
    int last_at = -1;
    for (int i = 0; i < a.n_out; ++i) {
        double best = -INFINITY;
        float best_x = -INFINITY;
        int best_at = -1;
        auto offer = [&](double t, float x, int at) {
            if (!(t > -INFINITY)) return;
            auto before = [&](double t0, float x0, int at0, double t1, float x1, int at1) {
                if (at0 / a.V == at1 / a.V) return x0 > x1 || (x0 == x1 && at0 < at1);
                return t0 > t1 || (t0 == t1 && at0 < at1);
            };
            if (last_at >= 0 && !before(last, last_x, last_at, t, x, at)) return;
            if (best_at < 0 || before(t, x, at, best, best_x, best_at)) { best = t; best_x = x; best_at = at; }
        };
        for (int k = 0; k < a.beams; ++k) {
            if (a.finished && a.finished[(long long)b * a.beams + k]) {
                if (tid == 0) offer((double)scores[k], 0.f, k * a.V + a.end_token);
                continue;
            }
            const long long row = b * a.batch_stride + k * a.beam_stride;
            for (int v = tid; v < a.V; v += 256) {
                const float x = logit<TYPE>(a.logits, row + v);
                if (x > -INFINITY) offer(base[k] + ((double)x - (double)top[k]), x, k * a.V + v);
            }
        }
        s_best[tid] = best; s_logit[tid] = best_x; s_at[tid] = best_at;
        __syncthreads();
        for (int t = 0; t < 256; ++t) if (s_at[t] >= 0) offer(s_best[t], s_logit[t], s_at[t]);
        __syncthreads();
        if (tid == 0) {
            const long long o = (long long)b * a.n_out + i;
            a.scores_out[o] = best_at < 0 ? -INFINITY : (float)best;
            a.tokens_out[o] = best_at < 0 ? -1 : best_at % a.V;
            a.parents_out[o] = best_at < 0 ? -1 : best_at / a.V;
        }
        if (best_at < 0) { last = -INFINITY; last_x = -INFINITY; last_at = 0x7fffffff; }
        else { last = best; last_x = best_x; last_at = best_at; }
    }
}

struct ReorderState {
    const char *src;
    char *dst;
    long long src_outer, src_batch, src_beam, dst_outer, dst_batch, dst_beam;
    unsigned columns;       // a row in pieces of `width` bytes
    unsigned width, first;  // first: its first work-group
    unsigned chunks;        // work-groups a row set
};
struct ReorderArgs {
    ReorderState s[RNNT_BEAM_STATES];
    const int *parents;
    int n, B, beams_in, beams_out;
};

// A thread moves one column of all hypotheses of an utterance: every source is read before the first
// destination is written, so that a state may be moved within itself.
template <class T, int BEAMS>
__device__ __forceinline__ void reorder_columns(const ReorderState &s, const int *parents, unsigned c, long long o, long long b, int beams_in, int beams_out)
{
    const char *from = s.src + o * s.src_outer + b * s.src_batch + (long long)c * sizeof(T);
    char *to = s.dst + o * s.dst_outer + b * s.dst_batch + (long long)c * sizeof(T);
    T v[BEAMS];
#pragma unroll
    for (int j = 0; j < BEAMS; ++j) {
        v[j] = T{};
        if (j >= beams_out) continue;
        const int p = parents[j];
        if (p >= 0 && p < beams_in) v[j] = *reinterpret_cast<const T *>(from + p * s.src_beam);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < BEAMS; ++j)
        if (j < beams_out) *reinterpret_cast<T *>(to + j * s.dst_beam) = v[j];
}

template <int BEAMS>
__global__ void __launch_bounds__(256)
beam_reorder_kernel(const ReorderArgs a)
{
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    int i = 0;
    while (i + 1 < a.n && blockIdx.x >= a.s[i + 1].first) ++i;
    const ReorderState &s = a.s[i];
    const unsigned at = blockIdx.x - s.first, set = at / s.chunks, c = (at - set * s.chunks) * 256 + threadIdx.x;
    const long long o = set / a.B, b = set - o * a.B;
    if (c >= s.columns) return;
    const int *parents = a.parents + b * a.beams_out;
    switch (s.width) {
    case 8: reorder_columns<v2u, BEAMS>(s, parents, c, o, b, a.beams_in, a.beams_out); break;
    case 4: reorder_columns<unsigned, BEAMS>(s, parents, c, o, b, a.beams_in, a.beams_out); break;
    case 2: reorder_columns<unsigned short, BEAMS>(s, parents, c, o, b, a.beams_in, a.beams_out); break;
    default: reorder_columns<unsigned char, BEAMS>(s, parents, c, o, b, a.beams_in, a.beams_out); break;
    }
}

}  // namespace rnnt

using namespace rnnt;

namespace {

#define BEAM_TRY(expr)                                          \
    do {                                                        \
        hipError_t e_ = (expr);                                 \
        if (e_ != hipSuccess) return hip_fail(e_, #expr);       \
    } while (0)

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

extern "C" {

int rnnt_beam_select_workspace(int32_t B, int32_t beams, int32_t V, int32_t n_out, int64_t *bytes_out)
{
    if (!bytes_out) return RNNT_ERR_NULL;
    if (B < 0 || beams < 1 || beams > kMaxBeams || V < 1 || n_out < 1 || n_out > kMaxBeams) return RNNT_ERR_SHAPE;
    if ((int64_t)beams * V > 0x7fffffff) return RNNT_ERR_UNSUPPORTED;
    *bytes_out = 0;
    return RNNT_OK;
}

int rnnt_beam_select(const void *logits, int32_t type, int64_t batch_stride, int64_t beam_stride,
                     const float *scores, const uint8_t *finished, int32_t B, int32_t beams, int32_t V,
                     int32_t n_out, int32_t end_token, float *scores_out, int32_t *tokens_out,
                     int32_t *parents_out, void *workspace, int64_t workspace_bytes, rnnt_stream_t stream)
{
    int64_t need = 0;
    if (const int rc = rnnt_beam_select_workspace(B, beams, V, n_out, &need)) return rc;
    if (type != RNNT_TYPE_F32 && type != RNNT_TYPE_BF16 && type != RNNT_TYPE_F16) return RNNT_ERR_SHAPE;
    if (batch_stride < 0 || beam_stride < 0 || workspace_bytes < 0) return RNNT_ERR_SHAPE;
    if (finished && (end_token < 0 || end_token >= V)) return RNNT_ERR_SHAPE;
    if (B == 0) return RNNT_OK;
    if (!logits || !scores || !scores_out || !tokens_out || !parents_out) return RNNT_ERR_NULL;
    if (!aligned(logits, type == RNNT_TYPE_F32 ? 4 : 2) || !aligned(scores, 4) || !aligned(scores_out, 4) || !aligned(tokens_out, 4) ||
        !aligned(parents_out, 4)) return RNNT_ERR_SHAPE;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return RNNT_ERR_SCRATCH;
    const SelectArgs args{logits, scores, finished, scores_out, tokens_out, parents_out, batch_stride, beam_stride, beams, V, n_out, end_token};
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(B), dim3(256), 0, static_cast<hipStream_t>(stream), args); };
    if (type == RNNT_TYPE_F32) run(beam_select_kernel<RNNT_TYPE_F32>);
    else if (type == RNNT_TYPE_BF16) run(beam_select_kernel<RNNT_TYPE_BF16>);
    else run(beam_select_kernel<RNNT_TYPE_F16>);
    BEAM_TRY(hipGetLastError());
    return RNNT_OK;
}

int rnnt_beam_reorder(const rnnt_beam_state *states, int32_t n_states, const int32_t *parents,
                      int32_t B, int32_t beams_in, int32_t beams_out, rnnt_stream_t stream)
{
    if (!states) return RNNT_ERR_NULL;
    if (n_states < 1 || n_states > RNNT_BEAM_STATES || B < 0 || beams_in < 1 || beams_in > kMaxBeams || beams_out < 1 || beams_out > kMaxBeams)
        return RNNT_ERR_SHAPE;
    if (!aligned(parents, 4)) return RNNT_ERR_SHAPE;
    ReorderArgs args{};
    args.parents = parents;
    args.B = B; args.beams_in = beams_in; args.beams_out = beams_out;
    int64_t groups = 0;
    for (int i = 0; i < n_states; ++i) {
        const rnnt_beam_state &s = states[i];
        if (s.outer < 0 || s.row_bytes < 0 || s.src_outer < 0 || s.src_batch < 0 || s.src_beam < 0 || s.dst_outer < 0 || s.dst_batch < 0 || s.dst_beam < 0)
            return RNNT_ERR_SHAPE;
        if (beams_out > 1 && s.dst_beam < s.row_bytes) return RNNT_ERR_SHAPE;
        if (s.src == s.dst && s.src && (beams_in != beams_out || s.src_outer != s.dst_outer || s.src_batch != s.dst_batch || s.src_beam != s.dst_beam))
            return RNNT_ERR_SHAPE;
        if (B == 0 || s.outer == 0 || s.row_bytes == 0) continue;
        if (!s.src || !s.dst || !parents) return RNNT_ERR_NULL;
        // the widest piece that divides addresses, strides and rows
        const uint64_t all = reinterpret_cast<uintptr_t>(s.src) | reinterpret_cast<uintptr_t>(s.dst) | (uint64_t)s.row_bytes | (uint64_t)s.src_outer |
                             (uint64_t)s.src_batch | (uint64_t)s.src_beam | (uint64_t)s.dst_outer | (uint64_t)s.dst_batch | (uint64_t)s.dst_beam | 8u;
        const unsigned width = (unsigned)(all & (~all + 1));
        const int64_t columns = s.row_bytes / width, chunks = (columns + 255) / 256;
        if (s.outer > 0x7fffffff / B || chunks > 0x7fffffff / (s.outer * B)) return RNNT_ERR_UNSUPPORTED;
        args.s[args.n++] = ReorderState{static_cast<const char *>(s.src), static_cast<char *>(s.dst), s.src_outer, s.src_batch, s.src_beam, s.dst_outer,
                                        s.dst_batch, s.dst_beam, (unsigned)columns, width, (unsigned)groups, (unsigned)chunks};
        groups += chunks * s.outer * B;
        if (groups > 0x7fffffff) return RNNT_ERR_UNSUPPORTED;
    }
    if (args.n == 0) return RNNT_OK;
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, static_cast<hipStream_t>(stream), args); };
    if (beams_out <= 8) run(beam_reorder_kernel<8>);
    else if (beams_out <= 16) run(beam_reorder_kernel<16>);
    else if (beams_out <= 32) run(beam_reorder_kernel<32>);
    else run(beam_reorder_kernel<64>);
    BEAM_TRY(hipGetLastError());
    return RNNT_OK;
}

}  // extern "C"

// Microscaled 4-bit matrices: quantisation, and products on the scaled matrix instructions.
#include "../../include/rnnt_greedy.h"

#include <hip/hip_runtime.h>

#include "engine.h"
#include "parts.h"

namespace rnnt {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr int kTileRows = 16, kTileCols = 128, kTileBytes = 1024;     // a tile of codes
constexpr int kScaleCols = 512, kScaleBytes = 256;                    // its scales, with those of three more

__host__ __device__ __forceinline__ long long tiles(long long n, int by) { return (n + by - 1) / by; }

// An element of a type, widened
template <int TYPE> struct Element;
template <> struct Element<RNNT_TYPE_F32> { typedef float T; };
template <> struct Element<RNNT_TYPE_BF16> { typedef __bf16 T; };
template <> struct Element<RNNT_TYPE_F16> { typedef _Float16 T; };

// The biased exponent k + 127 of a block whose largest magnitude has these bits: the smallest k with top <= 1.5 * 2^(k + 2).
// (Adding 0x3fffff carries into the exponent where the mantissa is above 1.5; below 2^-126 there is only -127.)
__device__ __forceinline__ unsigned block_scale(unsigned top)
{
    if (top == 0u) return 127u;
    if (top >= 0x7f800000u) return 255u;
    const int e = (int)((top + 0x3fffffu) >> 23) - 2;
    return (unsigned)max(e, 0);
}

// Quantises a block that one lane holds: 32 values into 16 bytes, the earlier value in the low half of a byte.
__device__ __forceinline__ v4u quantize_block(const float (&v)[32], unsigned &scale)
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    scale = block_scale(top);
    v4u c = {0u, 0u, 0u, 0u};
    if (scale == 255u) return c;
    // (the instruction takes the exponent field of its scale operand alone: 0 is 2^-127)
    const float s = __uint_as_float(scale << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[i * 8 + 0], v[i * 8 + 1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[i * 8 + 2], v[i * 8 + 3], s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[i * 8 + 4], v[i * 8 + 5], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[i * 8 + 6], v[i * 8 + 7], s, 3);
        c[i] = w;
    }
    return c;
}

// N neighbours of a row, at any address that is a multiple of an element's size; zeros beyond the first `left`.
template <class T, int N> struct Piece { T e[N]; };
template <class T, int N>
__device__ __forceinline__ Piece<T, N> load_piece(const T *p, long long left)
{
    struct __attribute__((packed, aligned(sizeof(T)))) At { T e[N]; };
    Piece<T, N> v;
    if (left >= N) {
        const At a = *reinterpret_cast<const At *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) v.e[i] = a.e[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v.e[i] = i < left ? p[i] : (T)0.f;
    }
    return v;
}
template <class T, int N>
__device__ __forceinline__ void store_piece(T *p, const Piece<T, N> &v, long long left)
{
    struct __attribute__((packed, aligned(sizeof(T)))) At { T e[N]; };
    if (left >= N) {
        At a;
#pragma unroll
        for (int i = 0; i < N; ++i) a.e[i] = v.e[i];
        *reinterpret_cast<At *>(p) = a;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) if (i < left) p[i] = v.e[i];
    }
}

// The block of 32 values at p of a row that goes on for `left` values from there
template <class T>
__device__ __forceinline__ void load_block(float (&v)[32], const T *p, long long left)
{
    constexpr int PER = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 32 / PER; ++i) {
        const Piece<T, PER> a = load_piece<T, PER>(p + i * PER, left - i * PER);
#pragma unroll
        for (int e = 0; e < PER; ++e) v[i * PER + e] = (float)a.e[e];
    }
}

// The largest of the lanes that hold a block: 8 or 4 neighbours.
template <int LANES>
__device__ __forceinline__ unsigned block_top(unsigned m)
{
    m = max(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));                       // quad_perm [1,0,3,2]
    m = max(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));                       // quad_perm [2,3,0,1]
    if (LANES == 8) m = max(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, true));      // row_half_mirror
    return m;
}

// Memory bound: a work-group takes 16 rows by 512 columns, four rows a wave, and reads and writes whole lines: a lane
// holds 16 bytes of a row, so that 8 lanes (16-bit types: 4) share a block and find its largest value in three (two) steps
// between lanes.  Codes and scales are put in order in LDS and leave in one piece.
template <int TYPE>
__global__ void __launch_bounds__(256)
mx4_quantize_kernel(const void *x, long long rows, long long cols, long long stride, unsigned char *codes, unsigned char *scales, float *values,
                    int col_tiles, int scale_tiles)
{
    typedef typename Element<TYPE>::T T;
    constexpr int PER = 16 / sizeof(T), PARTS = kScaleCols / (64 * PER), LANES = RNNT_MX4_BLOCK / PER, ROWS = kTileRows / 4;
    __shared__ __align__(16) unsigned char tile[4 * kTileBytes + kScaleBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int rt = blockIdx.x / scale_tiles, st = blockIdx.x - rt * scale_tiles;
    const bool whole = (long long)(st + 1) * kScaleCols <= cols;
    Piece<T, PER> v[ROWS][PARTS];
    // (the same for all lanes: whether there is the row, and whether all its columns are inside)
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const long long row = (long long)rt * kTileRows + wave * ROWS + i;
        const T *p = static_cast<const T *>(x) + row * stride + (long long)st * kScaleCols + lane * PER;
        const long long left = row < rows ? cols - (long long)st * kScaleCols - lane * PER : 0;
        if (whole && row < rows) {
#pragma unroll
            for (int h = 0; h < PARTS; ++h) v[i][h] = load_piece<T, PER>(p + h * 64 * PER, PER);
        } else {
#pragma unroll
            for (int h = 0; h < PARTS; ++h) v[i][h] = load_piece<T, PER>(p + h * 64 * PER, left - h * 64 * PER);
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = wave * ROWS + i;
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
            float f[PER];
            unsigned top = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) { f[e] = (float)v[i][h].e[e]; top = max(top, __float_as_uint(f[e]) & 0x7fffffffu); }
            const unsigned scale = block_scale(block_top<LANES>(top));
            const float unit = __uint_as_float(scale << 23);
            unsigned c = 0;
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], unit, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], unit, 1);
            if constexpr (PER == 8) {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], unit, 2);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], unit, 3);
            }
            if (scale == 255u) c = 0;
            const int in = (h * 64 + lane) * PER, t = in / kTileCols, b = in % kTileCols / RNNT_MX4_BLOCK;
            unsigned char *to = tile + t * kTileBytes + (b * 16 + r) * 16 + in % RNNT_MX4_BLOCK / 2;
            if constexpr (PER == 8) *reinterpret_cast<unsigned *>(to) = c;
            else *reinterpret_cast<unsigned short *>(to) = (unsigned short)c;
            if (lane % LANES == 0) tile[4 * kTileBytes + (b * 16 + r) * 4 + t] = (unsigned char)scale;
            if (values) {
                const long long row = (long long)rt * kTileRows + r, col = (long long)st * kScaleCols + in;
                if (row >= rows || col >= cols) continue;
                Piece<float, PER> o;
#pragma unroll
                for (int e = 0; e < PER; e += 2) {
                    typedef float v2f __attribute__((ext_vector_type(2)));
                    const unsigned pair = c >> (e * 4);
                    const v2f two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(pair, unit, 0);
                    o.e[e] = scale == 255u ? __uint_as_float(0x7fc00000u) : two.x;
                    o.e[e + 1] = scale == 255u ? __uint_as_float(0x7fc00000u) : two.y;
                }
                store_piece<float, PER>(values + row * cols + col, o, whole ? PER : cols - col);
            }
        }
    }
    __syncthreads();
    const int ct = st * 4 + wave;
    if (ct < col_tiles)
        *reinterpret_cast<v4u *>(codes + ((long long)rt * col_tiles + ct) * kTileBytes + lane * 16) = *reinterpret_cast<const v4u *>(tile + wave * kTileBytes + lane * 16);
    if (wave == 0)
        *reinterpret_cast<unsigned *>(scales + ((long long)rt * scale_tiles + st) * kScaleBytes + lane * 4) = *reinterpret_cast<const unsigned *>(tile + 4 * kTileBytes + lane * 4);
}

__device__ __forceinline__ void store(void *y, int type, long long at, float v)
{
    if (type == RNNT_TYPE_F32) static_cast<float *>(y)[at] = v;
    else if (type == RNNT_TYPE_BF16) static_cast<__bf16 *>(y)[at] = (__bf16)v;
    else static_cast<_Float16 *>(y)[at] = (_Float16)v;
}

// A wave computes 16 x 16 outputs: rows of w are the instruction's rows, rows of a its columns.
template <int A>
__global__ void __launch_bounds__(256)
mx4_product_kernel(const void *a, const unsigned char *a_scales, long long a_stride, const unsigned char *w, const unsigned char *w_scales,
                   const float *bias, void *y, int y_type, long long y_stride, long long M, long long N, long long K)
{
    const int lane = threadIdx.x & 63, r = lane & 15, b = lane >> 4;
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long mts = tiles(M, kTileRows), nt = i / mts, mt = i - nt * mts;
    if (nt >= tiles(N, kTileRows)) return;
    const int steps = (int)tiles(K, kTileCols), scale_tiles = (int)tiles(K, kScaleCols);
    v4f sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < steps; ++s) {
        const v4u wc = *reinterpret_cast<const v4u *>(w + (nt * steps + s) * kTileBytes + lane * 16);
        const unsigned ws = w_scales[(nt * scale_tiles + s / 4) * kScaleBytes + lane * 4 + (s & 3)];
        v4u ac;
        unsigned as;
        if constexpr (A == RNNT_TYPE_MX4) {
            ac = *reinterpret_cast<const v4u *>(static_cast<const unsigned char *>(a) + (mt * steps + s) * kTileBytes + lane * 16);
            as = a_scales[(mt * scale_tiles + s / 4) * kScaleBytes + lane * 4 + (s & 3)];
        } else {
            float v[32];
            typedef typename Element<A>::T T;
            const long long row = mt * kTileRows + r, col = (long long)s * kTileCols + b * RNNT_MX4_BLOCK;
            load_block<T>(v, static_cast<const T *>(a) + row * a_stride + col, row < M ? K - col : 0);
            ac = quantize_block(v, as);
        }
        const v8i wv = {(int)wc.x, (int)wc.y, (int)wc.z, (int)wc.w, 0, 0, 0, 0}, av = {(int)ac.x, (int)ac.y, (int)ac.z, (int)ac.w, 0, 0, 0, 0};
        sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, sum, 4, 4, 0, (int)ws, 0, (int)as);
    }
    const long long m = mt * kTileRows + r;
    if (m >= M) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const long long n = nt * kTileRows + b * 4 + e;
        if (n < N) store(y, y_type, m * y_stride + n, sum[e] + (bias ? bias[n] : 0.f));
    }
}

}  // namespace rnnt

using namespace rnnt;

namespace {

#define MX4_TRY(expr)                                           \
    do {                                                        \
        hipError_t e_ = (expr);                                 \
        if (e_ != hipSuccess) return hip_fail(e_, #expr);       \
    } while (0)

constexpr int64_t kMost = 0x7fffffff;

bool is_number(int32_t type) { return type == RNNT_TYPE_F32 || type == RNNT_TYPE_BF16 || type == RNNT_TYPE_F16; }
bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
uintptr_t size_of(int32_t type) { return type == RNNT_TYPE_F32 ? 4 : 2; }

}  // namespace

extern "C" {

int rnnt_mx4_sizes(int64_t rows, int64_t cols, int64_t *codes_bytes_out, int64_t *scales_bytes_out)
{
    if (!codes_bytes_out || !scales_bytes_out) return RNNT_ERR_NULL;
    if (rows < 0 || cols < 0) return RNNT_ERR_SHAPE;
    if (rows > kMost || cols > kMost) return RNNT_ERR_UNSUPPORTED;
    *codes_bytes_out = tiles(rows, kTileRows) * tiles(cols, kTileCols) * kTileBytes;
    *scales_bytes_out = tiles(rows, kTileRows) * tiles(cols, kScaleCols) * kScaleBytes;
    return RNNT_OK;
}

int rnnt_mx4_quantize(const void *x, int32_t type, int64_t rows, int64_t cols, int64_t x_stride,
                      void *codes_out, void *scales_out, float *values_out, rnnt_stream_t stream)
{
    if (!is_number(type) || rows < 0 || cols < 0 || x_stride < cols) return RNNT_ERR_SHAPE;
    if (rows > kMost || cols > kMost) return RNNT_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return RNNT_OK;
    if (!x || !codes_out || !scales_out) return RNNT_ERR_NULL;
    if (!aligned(x, size_of(type)) || !aligned(codes_out, 16) || !aligned(scales_out, 4) || !aligned(values_out, 4)) return RNNT_ERR_SHAPE;
    const int ct = (int)tiles(cols, kTileCols), st = (int)tiles(cols, kScaleCols);
    const long long blocks = tiles(rows, kTileRows) * st;
    if (blocks > kMost) return RNNT_ERR_UNSUPPORTED;
    auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), x, (long long)rows, (long long)cols,
                           (long long)x_stride, static_cast<unsigned char *>(codes_out), static_cast<unsigned char *>(scales_out), values_out, ct, st);
    };
    if (type == RNNT_TYPE_F32) run(mx4_quantize_kernel<RNNT_TYPE_F32>);
    else if (type == RNNT_TYPE_BF16) run(mx4_quantize_kernel<RNNT_TYPE_BF16>);
    else run(mx4_quantize_kernel<RNNT_TYPE_F16>);
    MX4_TRY(hipGetLastError());
    return RNNT_OK;
}

int rnnt_mx4_product_workspace(int32_t a_type, int64_t M, int64_t N, int64_t K, int64_t *bytes_out)
{
    if (!bytes_out) return RNNT_ERR_NULL;
    if ((!is_number(a_type) && a_type != RNNT_TYPE_MX4) || M < 0 || N < 0 || K < 0) return RNNT_ERR_SHAPE;
    if (M > kMost || N > kMost || K > kMost) return RNNT_ERR_UNSUPPORTED;
    *bytes_out = 0;
    return RNNT_OK;
}

int rnnt_mx4_product(const void *a, const void *a_scales, int32_t a_type, int64_t a_stride,
                     const void *w_codes, const void *w_scales, const float *bias,
                     void *y, int32_t y_type, int64_t y_stride, int64_t M, int64_t N, int64_t K,
                     void *workspace, int64_t workspace_bytes, rnnt_stream_t stream)
{
    int64_t need = 0;
    if (const int rc = rnnt_mx4_product_workspace(a_type, M, N, K, &need)) return rc;
    const bool codes = a_type == RNNT_TYPE_MX4;
    if (!is_number(y_type) || y_stride < N || (!codes && a_stride < K) || workspace_bytes < 0) return RNNT_ERR_SHAPE;
    if (M == 0 || N == 0) return RNNT_OK;
    if (!y || (K > 0 && (!a || (codes && !a_scales) || !w_codes || !w_scales))) return RNNT_ERR_NULL;
    if (!aligned(y, size_of(y_type)) || !aligned(bias, 4) || !aligned(w_codes, 16) || !aligned(w_scales, 4) ||
        !aligned(a, codes ? 16 : size_of(a_type)) || (codes && !aligned(a_scales, 4))) return RNNT_ERR_SHAPE;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return RNNT_ERR_SCRATCH;
    const long long blocks = tiles(tiles(M, kTileRows) * tiles(N, kTileRows), 4);
    if (blocks > kMost) return RNNT_ERR_UNSUPPORTED;
    auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), a, static_cast<const unsigned char *>(a_scales),
                           (long long)a_stride, static_cast<const unsigned char *>(w_codes), static_cast<const unsigned char *>(w_scales), bias, y,
                           (int)y_type, (long long)y_stride, (long long)M, (long long)N, (long long)K);
    };
    if (a_type == RNNT_TYPE_F32) run(mx4_product_kernel<RNNT_TYPE_F32>);
    else if (a_type == RNNT_TYPE_BF16) run(mx4_product_kernel<RNNT_TYPE_BF16>);
    else if (a_type == RNNT_TYPE_F16) run(mx4_product_kernel<RNNT_TYPE_F16>);
    else run(mx4_product_kernel<RNNT_TYPE_MX4>);
    MX4_TRY(hipGetLastError());
    return RNNT_OK;
}

}  // extern "C"

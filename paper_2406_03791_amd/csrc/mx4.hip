// Microscaled 4-bit matrices: quantisation, and products on the scaled matrix instructions.
#include "../../include/rnnt_greedy.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "engine.h"
#include "wave.h"

namespace rnnt {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
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
template <> struct Element<RNNT_TYPE_MX4> { typedef unsigned char T; };

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
// between lanes.  Codes and scales are put in order in LDS and leave in one piece.  With the values asked for, a lane holds four of whatever
// type, 16 bytes of values; where there are more of them than the L2s hold, their stores are marked as not to be kept there.
// With the values, 8192 x 8192 fp32: 101.6 us, 5.6 TB/s (107.5 without the mark); 11309 x 1024 bf16: 12.5 (14.5).
enum { kNoValues, kValues, kStreamedValues };
template <int TYPE, int OUT>
__global__ void __launch_bounds__(256)
mx4_quantize_kernel(const void *x, long long rows, long long cols, long long stride, unsigned char *codes, unsigned char *scales, float *values,
                    int col_tiles, int scale_tiles)
{
    typedef typename Element<TYPE>::T T;
    constexpr int PER = OUT == kNoValues ? 16 / (int)sizeof(T) : 4, PARTS = kScaleCols / (64 * PER), LANES = RNNT_MX4_BLOCK / PER, ROWS = kTileRows / 4;
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
            if constexpr (OUT != kNoValues) {
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
                if (OUT == kStreamedValues && whole) {
#pragma unroll
                    for (int e = 0; e < PER; e += 4) {
                        typedef v4f At __attribute__((aligned(4)));
                        __builtin_nontemporal_store(v4f{o.e[e], o.e[e + 1], o.e[e + 2], o.e[e + 3]}, reinterpret_cast<At *>(values + row * cols + col + e));
                    }
                } else store_piece<float, PER>(values + row * cols + col, o, whole ? PER : cols - col);
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

// Four neighbours of a row of y, rounded to its type; the first `left` of them
__device__ __forceinline__ void store_four(void *y, int type, long long at, const float (&v)[4], long long left)
{
    if (type == RNNT_TYPE_F32) store_piece<float, 4>(static_cast<float *>(y) + at, Piece<float, 4>{{v[0], v[1], v[2], v[3]}}, left);
    else if (type == RNNT_TYPE_BF16) store_piece<__bf16, 4>(static_cast<__bf16 *>(y) + at, Piece<__bf16, 4>{{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]}}, left);
    else store_piece<_Float16, 4>(static_cast<_Float16 *>(y) + at, Piece<_Float16, 4>{{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]}}, left);
}

struct ProductArgs {
    const void *a;
    const unsigned char *a_scales, *w, *w_scales;
    const float *bias;
    void *y;
    long long a_stride, y_stride;
    int y_type, M, N, K;
};

__device__ __forceinline__ v8i operand(const v4u &c) { return v8i{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}; }

// Few rows: bound by latency, and for large w by reading it.  A work-group computes 16 rows of a by 16 NT rows of w; its WAVES waves
// take the tiles of K in turn and add up at the end.  Operands go from memory to registers: a lane's part of a tile is a row's
// block, 32 values, which it quantises by itself.  Two shapes: eight waves by 32 rows of w, and, from 256 work-groups of it on, four by 64, with
// half as many readers of a.  us, bf16, first shape and second: 16 x 8192 x 8192 12.3 and 15.6, 128 x 4096 x 1024 8.2 and 5.8.
// (Tiles asked for ahead, two to four: 4.4 to 4.8 in place of 4.0 for small ones, nothing gained for large ones.)
template <int A, int NT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64)
mx4_product_kernel(const ProductArgs g)
{
    typedef typename Element<A>::T T;                      // (of codes: bytes, 16 of them)
    constexpr int PITCH = NT * 16 + 4, PER = 16 / (int)sizeof(T), PIECES = A == RNNT_TYPE_MX4 ? 1 : RNNT_MX4_BLOCK / PER;
    __shared__ __align__(16) float sums[WAVES][16 * PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r = lane & 15, b = lane >> 4;
    const int steps = (int)tiles(g.K, kTileCols), groups = (int)tiles(g.K, kScaleCols), n_tiles = (int)tiles(g.N, kTileRows);
    const int across = (int)tiles(n_tiles, NT), mt = blockIdx.x / across, nt = (blockIdx.x - mt * across) * NT;
    // (a row beyond the last one repeats it and is not stored)
    const T *row = static_cast<const T *>(g.a) + (A == RNNT_TYPE_MX4 ? (long long)mt * steps * kTileBytes + lane * 16
                                                                   : min((long long)mt * kTileRows + r, (long long)g.M - 1) * g.a_stride + b * RNNT_MX4_BLOCK);
    struct Tile { v4u w[NT]; Piece<T, PER> a[PIECES]; unsigned ws[NT], as; };
    auto load = [&](Tile &o, int s) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const long long t = min(nt + i, n_tiles - 1);
            o.w[i] = *reinterpret_cast<const v4u *>(g.w + (t * steps + s) * kTileBytes + lane * 16);
            o.ws[i] = g.w_scales[(t * groups + s / 4) * kScaleBytes + lane * 4 + (s & 3)];
        }
        if constexpr (A == RNNT_TYPE_MX4) {
            o.a[0] = load_piece<T, PER>(row + (long long)s * kTileBytes, PER);
            o.as = g.a_scales[((long long)mt * groups + s / 4) * kScaleBytes + lane * 4 + (s & 3)];
        } else if ((long long)(s + 1) * kTileCols <= g.K) {        // (the same for all lanes)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) o.a[i] = load_piece<T, PER>(row + s * kTileCols + i * PER, PER);
        } else {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) o.a[i] = load_piece<T, PER>(row + s * kTileCols + i * PER, g.K - s * kTileCols - b * RNNT_MX4_BLOCK - i * PER);
        }
    };
    v4f sum[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) sum[i] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int s = wave; s < steps; s += WAVES) {
        Tile t;
        load(t, s);
        v4u c;
        unsigned scale;
        if constexpr (A == RNNT_TYPE_MX4) { c = __builtin_bit_cast(v4u, t.a[0]); scale = t.as; }
        else {
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = (float)t.a[i / PER].e[i % PER];
            c = quantize_block(v, scale);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
            sum[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(t.w[i]), operand(c), sum[i], 4, 4, 0, (int)t.ws[i], 0, (int)scale);
    }
    // (a lane holds four neighbours of w's rows for one of a's)
#pragma unroll
    for (int i = 0; i < NT; ++i) *reinterpret_cast<v4f *>(&sums[wave][r * PITCH + i * 16 + b * 4]) = sum[i];
    __syncthreads();
    const int m = threadIdx.x / (NT * 4), c = threadIdx.x % (NT * 4) * 4;
    if (m >= 16 || (long long)mt * kTileRows + m >= g.M) return;
    const long long n = (long long)nt * kTileRows + c;
    if (n >= g.N) return;
    float o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int at = m * PITCH + c + e;
        float all[WAVES];
#pragma unroll
        for (int i = 0; i < WAVES; ++i) all[i] = sums[i][at];
#pragma unroll
        for (int half = WAVES / 2; half > 0; half /= 2)
#pragma unroll
            for (int i = 0; i < half; ++i) all[i] += all[i + half];
        o[e] = all[0] + (g.bias && n + e < g.N ? g.bias[n + e] : 0.f);
    }
    store_four(g.y, g.y_type, ((long long)mt * kTileRows + m) * g.y_stride + n, o, g.N - n);
}

// Many rows: bound by the matrix instructions, 32 cycles for 32 x 32 x 64, and by the schedule around them: they fill 51 % of the 515 000 cycles of a
// product of 8192^3, whatever the codes.  (In long products the clock falls, too, to 1.75 - 1.95 GHz on random codes, 2.3 - 2.4 on
// zeros: 258 - 287 us and 216 - 227; those instructions alone reach 6.6 PFLOP/s on random codes, on zeros 9.5.)  A block of y, BM x BN outputs, is that of 2 x 2 waves
// with TM x TN tiles of 32 x 32 each.  Tiles of codes lie in memory as the lanes take them: they go to LDS in pieces of 1 KB, STAGES
// tiles of K in turn, and from there to registers without bank conflicts.
//
// A work-group has a block after the other, and asks for pieces of the next one while it is still at this one: the
// pipeline does not run dry between blocks, and results are on their way to memory while the next block is multiplied.
// In a step (a tile of K, two instructions deep) the operands of the second half are read while the first half is
// multiplied; then the wave waits for the next step's pieces, meets the others, asks for the pieces STAGES - 1 steps
// ahead (their place was last read a step ago), and reads the next step's first half while the second is multiplied.
// Between matrix instructions there is room for others: one thing is asked for or read behind each.  Scales: four steps' in a word,
// asked for with the first step's codes.
// CHAIN: a work-group has several blocks, and the results a place of their own in LDS; else it has one, and they take that of the codes.
template <int TM_, int TN_, int STAGES_, bool CHAIN_>
struct TileShape {
    static constexpr int TM = TM_, TN = TN_, STAGES = STAGES_;
    static constexpr bool CHAIN = CHAIN_;
    static constexpr int BM = TM * 64, BN = TN * 64, TILES = (BM + BN) / kTileRows;
    static constexpr int CODES = TILES * kTileBytes, SCALES = TILES * kScaleBytes, OUT = CHAIN ? 4 * 4096 : 0;
    static constexpr int LDS = STAGES * CODES + 2 * SCALES + OUT, GROUPS = 160 * 1024 / LDS;      // work-groups of a compute unit
};

template <class S, int Y>
__global__ void __launch_bounds__(256, S::GROUPS)
mx4_tile_kernel(const ProductArgs g, int m_blocks, int n_blocks)
{
    typedef typename Element<Y>::T YT;
    constexpr int TM = S::TM, TN = S::TN, STAGES = S::STAGES;
    constexpr int LOADS = S::TILES / 4, SCALE_LOADS = S::TILES / 16;       // of a wave: a tile of codes a load, four tiles' scales a load
    static_assert(S::TILES % 16 == 0 && S::BM % 64 == 0, "whole loads, of one operand each");
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int steps = (int)tiles(g.K, kTileCols), groups = (int)tiles(g.K, kScaleCols);
    const int m_last = (int)tiles(g.M, kTileRows) - 1, n_last = (int)tiles(g.N, kTileRows) - 1;
    // An XCD has blocks that follow each other, in bands of eight blocks of rows of a, so that its L2 serves each operand to several
    // work-groups; those of it take them in turn.
    const int n_all = m_blocks * n_blocks, xcd = blockIdx.x & 7, here = n_all / 8 + (xcd < n_all % 8), peers = ((int)gridDim.x - xcd + 7) / 8;
    struct Block { int mb, nb; };
    auto block = [&](int i) {
        const int at = xcd * (n_all / 8) + min(xcd, n_all % 8) + i;
        const int band = at / (8 * n_blocks), in = at - band * 8 * n_blocks, high = min(8, m_blocks - band * 8);
        return Block{band * 8 + in % high, in / high};
    };
    // What is asked for: pieces of step ask_step of block ask_block, from `code` and `scale` on
    int ask_block = blockIdx.x >> 3, ask_step = 0, ask_group = 0;
    if (ask_block >= here) return;
    const unsigned char *code[LOADS], *scale[SCALE_LOADS];
    unsigned scale_off[SCALE_LOADS];
    auto aim = [&]() {
        const Block k = block(ask_block);
        // row of tiles number i of the block: first those of a, then those of w; what is beyond the end repeats the last one and is not stored
        auto tile_row = [&](int i) { return i < S::BM / 16 ? min(k.mb * (S::BM / 16) + i, m_last) : min(k.nb * (S::BN / 16) + i - S::BM / 16, n_last); };
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int t = wave * LOADS + i;
            code[i] = uniform((t < S::BM / 16 ? static_cast<const unsigned char *>(g.a) : g.w) + (long long)tile_row(t) * steps * kTileBytes);
        }
#pragma unroll
        for (int i = 0; i < SCALE_LOADS; ++i) {
            // (four rows of tiles of one operand: their first one's address, and a lane's distance from it)
            const int t = (wave * SCALE_LOADS + i) * 4, first = tile_row(t);
            scale[i] = uniform((t < S::BM / 16 ? g.a_scales : g.w_scales) + (long long)first * groups * kScaleBytes);
            scale_off[i] = (unsigned)(tile_row(t + (lane >> 4)) - first) * (unsigned)groups * kScaleBytes + (lane & 15) * 16;
        }
    };
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds;
    auto to_lds = [&](const unsigned char *from, unsigned off, unsigned to) {
        const unsigned m = (unsigned)__builtin_amdgcn_readfirstlane((int)(lds0 + to));
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" :: "v"(off), "s"(m), "s"(from) : "memory");
    };
    auto ask_scales = [&]() {
        if (ask_step % 4 != 0) return;
#pragma unroll
        for (int i = 0; i < SCALE_LOADS; ++i)
            to_lds(uniform(scale[i] + (long long)(ask_step / 4) * kScaleBytes), scale_off[i],
                   (unsigned)(STAGES * S::CODES + (ask_group & 1) * S::SCALES + (wave * SCALE_LOADS + i) * 1024));
        ++ask_group;
    };
    auto ask_code = [&](int stage, int i) {
        to_lds(uniform(code[i] + (long long)ask_step * kTileBytes), (unsigned)lane * 16u, (unsigned)(stage * S::CODES + (wave * LOADS + i) * kTileBytes));
    };
    // the step behind; behind the last block's last one its first again, which nobody reads
    auto advance = [&]() {
        if (++ask_step < steps) return;
        ask_step = 0;
        if constexpr (S::CHAIN) {
            if (ask_block + peers < here) ask_block += peers;
            aim();
        }
    };
    const int wm = wave & 1, wn = wave >> 1;
    // a lane's operand of 32 rows and half h of a tile: rows lane % 32, block 2 h + lane / 32
    const unsigned char *mine = lds + (lane >> 4 & 1) * kTileBytes + (lane >> 5) * 256 + (lane & 15) * 16;
    const unsigned char *mine_s = lds + STAGES * S::CODES + (lane >> 4 & 1) * kScaleBytes + (lane >> 5) * 64 + (lane & 15) * 4;
    struct Half { v4u a[TM], w[TN]; };
    struct Scales { int a[2][TM], w[2][TN]; };             // of four steps, the step's own in the lowest byte
    auto tile_of = [&](int i) { return i < TM ? wm * TM * 2 + i * 2 : S::BM / 16 + wn * TN * 2 + (i - TM) * 2; };
    auto read_one = [&](Half &o, int stage, int h, int i) {
        const v4u v = *reinterpret_cast<const v4u *>(mine + stage * S::CODES + tile_of(i) * kTileBytes + h * 512);
        if (i < TM) o.a[i] = v; else o.w[i - TM] = v;
    };
    auto read_scales = [&](Scales &o, int group) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < TM + TN; ++i) {
                const int v = *reinterpret_cast<const int *>(mine_s + (group & 1) * S::SCALES + tile_of(i) * kScaleBytes + h * 128);
                if (i < TM) o.a[h][i] = v; else o.w[h][i - TM] = v;
            }
    };
    auto shift = [&](Scales &o) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < TM; ++i) o.a[h][i] = (int)((unsigned)o.a[h][i] >> 8);
#pragma unroll
            for (int i = 0; i < TN; ++i) o.w[h][i] = (int)((unsigned)o.w[h][i] >> 8);
        }
    };
    // in the order in which they are needed: w's first tile, a's, the others of w
    auto in_order = [](int r) { return r == 0 ? TM : r <= TM ? r - 1 : r; };
    // Keeps a matrix instruction where it is written: the branches of a step would otherwise have the compiler move all of them to its end.
    auto stay = [](v16f &v) { asm volatile("" : "+a"(v)); };
    constexpr int ALL = TM * TN, READS = TM + TN;
    // Stores of a whole block by a wave.  Waits count what was issued behind what they wait for; vmcnt holds 63 at most.
    constexpr int STORES = TM * TN * (Y == RNNT_TYPE_F32 ? 4 : 2), AHEAD = (STAGES - 3) * LOADS, AFTER = AHEAD + STORES < 63 ? AHEAD + STORES : 63;
    static_assert(AHEAD < 63, "waits are counted");
    Half half[2];
    Scales now, next;
    aim();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        ask_scales();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) ask_code(s, i);
        advance();
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"((STAGES - 2) * LOADS) : "memory");
    int stage = 0, group = 0;                              // of the step that comes; of the scales in `now`
    read_scales(now, 0);
#pragma unroll
    for (int i = 0; i < READS; ++i) read_one(half[0], 0, 0, i);
    // Of the first steps of a block: whether there was none before it; whether STORES stores of the one before follow their pieces.
    bool first = true, counted = false;
#pragma clang loop unroll(disable)
    for (int i_block = blockIdx.x >> 3; i_block < here; i_block += peers) {
        v16f sum[TN][TM];
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[i][j][e] = 0.f;
#pragma clang loop unroll(disable)
        for (int t = 0; t < steps; ++t) {
            const int stage1 = stage + 1 == STAGES ? 0 : stage + 1, before = stage == 0 ? STAGES - 1 : stage - 1;
            const bool rare = S::CHAIN && t < STAGES - 2 && !first, turn = t % 4 == 3 || t + 1 == steps;       // turn: the next step has other scales
#pragma unroll
            for (int e = 0; e < ALL; ++e) {
                const int i = e / TM, j = e % TM;
                sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(half[0].w[i]), operand(half[0].a[j]), sum[i][j], 4, 4, 0, now.w[0][i], 0, now.a[0][j]);
                stay(sum[i][j]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < READS; ++r) if (r * ALL / READS == e) read_one(half[1], stage, 1, in_order(r));
                __builtin_amdgcn_sched_barrier(0);
            }
            // What step t + 1 needs is there; what was asked for later, and stores behind it, may still be on their way.
            // (Stores of a block that is not whole are not counted: all of them are waited for.)
            if (!rare) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(AHEAD) : "memory");
            else if (counted) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(AFTER) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            asm volatile("s_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < ALL; ++e) {
                const int i = e / TM, j = e % TM;
                sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(half[1].w[i]), operand(half[1].a[j]), sum[i][j], 4, 4, 0, now.w[1][i], 0, now.a[1][j]);
                stay(sum[i][j]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < READS; ++r) if (r * ALL / READS == e) read_one(half[0], stage1, 0, in_order(r));
                if (e == 0) ask_scales();
#pragma unroll
                for (int r = 0; r < LOADS; ++r) if (1 + r * (ALL - 2) / LOADS == e) ask_code(before, r);
                if (e == ALL / 2 && turn) read_scales(next, group + 1);
                if (e == ALL - 1) advance();
                __builtin_amdgcn_sched_barrier(0);
            }
            stage = stage1;
            if (turn) { now = next; ++group; }
            else shift(now);
        }
        // Results leave by way of a wave's own part of LDS, 32 rows of 128 bytes of y at a time, so that lines are stored whole; 16-byte pieces are
        // xored with the row.  Register v of lane l holds row 8 (v / 4) + 4 (l / 32) + v % 4 of w's 32, row l % 32 of a's.
        // (Straight from the registers, sixteen bytes a row and store, this took 80 of 290 us of a product of 8192^3.)
        constexpr int ACROSS = 128 / (32 * (int)sizeof(YT)), PIECE = 16 / (int)sizeof(YT);     // tiles of 32 columns, elements of 16 bytes
        const Block k = block(i_block);
        const int m0 = k.mb * S::BM + wm * TM * 32, n0 = k.nb * S::BN + wn * TN * 32;
        const bool whole = (long long)m0 + TM * 32 <= g.M && (long long)n0 + TN * 32 <= g.N;
        unsigned char *part = lds + (S::CHAIN ? STAGES * S::CODES + 2 * S::SCALES : 0) + wave * 4096;
        // (without a place of their own: nothing is on its way to it or read there)
        if constexpr (!S::CHAIN) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        int l = lane;
        asm volatile("" : "+v"(l));                        // (places in y are worked out here, not before the steps, whose registers they would take)
        const int row = l & 31, high = l >> 5, out_row = l >> 3, out_piece = l & 7;
#pragma unroll
        for (int i0 = 0; i0 < TN; i0 += ACROSS) {
            // (the same for all lanes of a half: by way of the scalar cache, beside the loads that are counted)
            float bias[ACROSS][4][4] = {};
            const float *from_bias = g.bias + n0 + i0 * 32;
            if (g.bias && whole) {
#pragma unroll
                for (int i = 0; i < ACROSS * 16; ++i) {
                    const float low = from_bias[i / 4 * 8 + i % 4], up = from_bias[i / 4 * 8 + 4 + i % 4];
                    bias[i / 16][i / 4 % 4][i % 4] = high ? up : low;
                }
            } else if (g.bias) {
#pragma unroll
                for (int i = 0; i < ACROSS * 16; ++i) bias[i / 16][i / 4 % 4][i % 4] = g.bias[min(n0 + i0 * 32 + i / 4 * 8 + high * 4 + i % 4, g.N - 1)];
            }
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                wave_sync();
#pragma unroll
                for (int i = 0; i < ACROSS; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const v16f &from = sum[i0 + i][j];
                        Piece<YT, 4> o;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o.e[e] = (YT)(from[q * 4 + e] + bias[i][q][e]);
                        if constexpr (sizeof(YT) == 4) *reinterpret_cast<v4u *>(part + row * 128 + ((q * 2 + high) ^ (row & 7)) * 16) = __builtin_bit_cast(v4u, o);
                        else *reinterpret_cast<unsigned long long *>(part + row * 128 + ((i * 4 + q) ^ (row & 7)) * 16 + high * 8) = __builtin_bit_cast(unsigned long long, o);
                    }
                wave_sync();
                const int n = n0 + i0 * 32 + out_piece * PIECE;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int m = m0 + j * 32 + r * 8 + out_row;
                    const unsigned char *piece = part + (r * 8 + out_row) * 128 + (out_piece ^ out_row) * 16;
                    YT *to = static_cast<YT *>(g.y) + (long long)m * g.y_stride + n;
                    if (whole) store_piece<YT, PIECE>(to, __builtin_bit_cast(Piece<YT, PIECE>, *reinterpret_cast<const v4u *>(piece)), PIECE);
                    else if (m < g.M) {
                        const int some = min(PIECE, g.N - n);
#pragma unroll 1
                        for (int e = 0; e < some; ++e) to[e] = reinterpret_cast<const YT *>(piece)[e];
                    }
                }
            }
        }
        first = false;
        counted = whole;
    }
    // (nothing is on its way to LDS that is given up)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

}  // namespace rnnt

using namespace rnnt;

namespace {

#define MX4_TRY(expr)                                           \
    do {                                                        \
        hipError_t e_ = (expr);                                 \
        if (e_ != hipSuccess) return hip_fail(e_, #expr);       \
    } while (0)

constexpr int64_t kMost = 0x7fffffff, kMostThreads = 0xffffffff;          // rows or columns; threads of a launch
constexpr int64_t kStreamValues = 8 << 20;    // floats that the L2s of the eight XCDs hold together

bool is_number(int32_t type) { return type == RNNT_TYPE_F32 || type == RNNT_TYPE_BF16 || type == RNNT_TYPE_F16; }
bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
uintptr_t size_of(int32_t type) { return type == RNNT_TYPE_F32 ? 4 : 2; }

// Which kernel computes a product.  The one for few rows takes 3.5 us and one more for every 2 * 10^8 of M N K (of codes twice
// that); tiles (and the quantisation before them) take 10 us, up to K = 8192 25, before their size shows (of codes 7 and 20).
// us, few rows and tiles, of bf16: 256 x 4096 x 1024 9.2 and 10.8, 2048 x 1030 x 640 13.3 and 11.7, 128 x 4096 x 4096 13.6 and 17.5,
// 256 x 4096 x 4096 25.6 and 18.2, 64 x 8192 x 8192 24.9 and 28.4, 128 x 8192 x 8192 45.4 and 28.8; of codes: 256 x 4096 x 4096 12.2 and 13.8,
// 128 x 8192 x 8192 21.1 and 23.9.  Blocks of 256 x 256 where there is one for every compute unit (and two steps of K, which their
// pipeline is made for): 8192 x 8192 x 1024 62 us, by 128 x 128 71; 4096^3 42, by 128 x 128 45.
enum Plan { kDirect, kTiles128, kTiles256 };
constexpr int64_t kDirectGroups = 256;
constexpr double kDirectWork = 1 << 28;
constexpr int kComputeUnits = 256;     // of MI355X
int64_t direct_groups(int64_t M, int64_t N, int nt) { return tiles(M, kTileRows) * tiles(tiles(N, kTileRows), nt); }
Plan plan_of(int32_t a_type, int64_t M, int64_t N, int64_t K)
{
    if ((double)M * (double)N * (double)K <= kDirectWork * (3 + K / kScaleCols) * (a_type == RNNT_TYPE_MX4 ? 1.5 : 1.0)) return kDirect;
    return tiles(M, 256) * tiles(N, 256) >= kComputeUnits && K > kTileCols ? kTiles256 : kTiles128;
}

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
    if (!aligned(x, size_of(type)) || !aligned(codes_out, 16) || !aligned(scales_out, 16) || !aligned(values_out, 4)) return RNNT_ERR_SHAPE;
    const int ct = (int)tiles(cols, kTileCols), st = (int)tiles(cols, kScaleCols);
    const long long blocks = tiles(rows, kTileRows) * st;
    if (blocks * 256 > kMostThreads) return RNNT_ERR_UNSUPPORTED;
    auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), x, (long long)rows, (long long)cols,
                           (long long)x_stride, static_cast<unsigned char *>(codes_out), static_cast<unsigned char *>(scales_out), values_out, ct, st);
    };
    auto with = [&](auto t) {
        if (!values_out) run(mx4_quantize_kernel<t(), kNoValues>);
        else if (rows * cols <= kStreamValues) run(mx4_quantize_kernel<t(), kValues>);
        else run(mx4_quantize_kernel<t(), kStreamedValues>);
    };
    if (type == RNNT_TYPE_F32) with(std::integral_constant<int, RNNT_TYPE_F32>());
    else if (type == RNNT_TYPE_BF16) with(std::integral_constant<int, RNNT_TYPE_BF16>());
    else with(std::integral_constant<int, RNNT_TYPE_F16>());
    MX4_TRY(hipGetLastError());
    return RNNT_OK;
}

int rnnt_mx4_product_workspace(int32_t a_type, int64_t M, int64_t N, int64_t K, int64_t *bytes_out)
{
    if (!bytes_out) return RNNT_ERR_NULL;
    if ((!is_number(a_type) && a_type != RNNT_TYPE_MX4) || M < 0 || N < 0 || K < 0) return RNNT_ERR_SHAPE;
    if (M > kMost || N > kMost || K > kMost) return RNNT_ERR_UNSUPPORTED;
    int64_t codes = 0, scales = 0;
    if (a_type != RNNT_TYPE_MX4 && plan_of(a_type, M, N, K) != kDirect) (void)rnnt_mx4_sizes(M, K, &codes, &scales);
    *bytes_out = codes + scales;
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
    if (!aligned(y, size_of(y_type)) || !aligned(bias, 4) || !aligned(w_codes, 16) || !aligned(w_scales, 16) ||
        !aligned(a, codes ? 16 : size_of(a_type)) || (codes && !aligned(a_scales, 16))) return RNNT_ERR_SHAPE;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return RNNT_ERR_SCRATCH;
    const hipStream_t on = static_cast<hipStream_t>(stream);
    ProductArgs args{a, static_cast<const unsigned char *>(a_scales), static_cast<const unsigned char *>(w_codes), static_cast<const unsigned char *>(w_scales),
                     bias, y, a_stride, y_stride, y_type, (int)M, (int)N, (int)K};
    const Plan plan = plan_of(a_type, M, N, K);
    if (plan == kDirect) {
        const int nt = direct_groups(M, N, 4) >= kDirectGroups ? 4 : 2;
        const int64_t blocks = direct_groups(M, N, nt);
        if (blocks > kMostThreads / 512) return RNNT_ERR_UNSUPPORTED;
        auto run = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(waves * 64), 0, on, args); };
        auto with = [&](auto t) {
            if (nt == 4) run(mx4_product_kernel<t(), 4, 4>, 4);
            else run(mx4_product_kernel<t(), 2, 8>, 8);
        };
        if (a_type == RNNT_TYPE_F32) with(std::integral_constant<int, RNNT_TYPE_F32>());
        else if (a_type == RNNT_TYPE_BF16) with(std::integral_constant<int, RNNT_TYPE_BF16>());
        else if (a_type == RNNT_TYPE_F16) with(std::integral_constant<int, RNNT_TYPE_F16>());
        else with(std::integral_constant<int, RNNT_TYPE_MX4>());
        MX4_TRY(hipGetLastError());
        return RNNT_OK;
    }
    auto run = [&](auto shape, auto y) -> int {
        typedef decltype(shape) S;
        const auto kernel = mx4_tile_kernel<S, decltype(y)::value>;
        const int64_t mb = tiles(M, S::BM), nb = tiles(N, S::BN);
        if (mb * nb > kMostThreads / 256) return RNNT_ERR_UNSUPPORTED;
        MX4_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS));
        if (!codes) {                                      // (the first that is queued, behind everything that may be refused)
            int64_t cb = 0, sb = 0;
            (void)rnnt_mx4_sizes(M, K, &cb, &sb);
            unsigned char *to = static_cast<unsigned char *>(workspace);
            if (const int rc = rnnt_mx4_quantize(a, a_type, M, K, a_stride, to, to + cb, nullptr, stream)) return rc;
            args.a = to;
            args.a_scales = to + cb;
        }
        const int64_t groups = S::CHAIN ? std::min<int64_t>(mb * nb, kComputeUnits * S::GROUPS) : mb * nb;
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), S::LDS, on, args, (int)mb, (int)nb);
        MX4_TRY(hipGetLastError());
        return RNNT_OK;
    };
    auto with = [&](auto shape) -> int {
        if (y_type == RNNT_TYPE_F32) return run(shape, std::integral_constant<int, RNNT_TYPE_F32>());
        if (y_type == RNNT_TYPE_BF16) return run(shape, std::integral_constant<int, RNNT_TYPE_BF16>());
        return run(shape, std::integral_constant<int, RNNT_TYPE_F16>());
    };
    return plan == kTiles256 ? with(TileShape<4, 4, 4, true>()) : with(TileShape<2, 2, 4, false>());
}

}  // extern "C"

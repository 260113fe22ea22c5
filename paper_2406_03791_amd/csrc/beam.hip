// A beam search's step over hypotheses: selection over beams and vocabulary, and states that follow it.
#include "../../include/rnnt_greedy.h"

#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "engine.h"
#include "wave.h"

namespace rnnt {

constexpr int kMaxBeams = 64;
constexpr int kTile = 1024;             // logits of a row that a wave looks at together, 16 a lane
constexpr int kBuffer = 128;            // candidates of a wave that wait to be sorted in
constexpr int kJoinWaves = 16;          // waves of a work-group that joins lists, at most

typedef unsigned long long u64;
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

struct SelectArgs {
    const void *logits;
    const float *scores;
    const unsigned char *finished;
    float *scores_out;
    int *tokens_out, *parents_out;
    long long batch_stride, beam_stride;
    int B, beams, V, n_out, end_token;
    // Of two launches: a row is cut into so many pieces for a work-group each, whose waves have so many tiles each
    int pieces, piece_tiles;
    u64 *lists;                         // [B][beams][pieces][n_out]: the pieces' best
    double *sums, *refs;                // [B][beams][pieces][kScanWaves]: sums of exp(x - ref)
};

// The value of lane ^ M
template <int M> __device__ __forceinline__ unsigned from_lane(unsigned v)
{
#define RNNT_DPP(x, c) ((unsigned)__builtin_amdgcn_mov_dpp((int)(x), c, 0xf, 0xf, true))
    if constexpr (M == 1) return RNNT_DPP(v, 0xb1);                           // quad_perm [1,0,3,2]
    else if constexpr (M == 2) return RNNT_DPP(v, 0x4e);                      // quad_perm [2,3,0,1]
    else if constexpr (M == 4) return RNNT_DPP(RNNT_DPP(v, 0x141), 0x1b);     // row_half_mirror, then quad_perm [3,2,1,0]
    else if constexpr (M == 8) return RNNT_DPP(v, 0x128);                     // row_ror:8
    else if constexpr (M == 15) return RNNT_DPP(v, 0x140);                    // row_mirror
    else if constexpr (M == 16) {
        const auto both = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return threadIdx.x & 16 ? both[0] : both[1];
    } else {
        static_assert(M == 32, "a power of two below 64, or 15");
        const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? both[0] : both[1];
    }
#undef RNNT_DPP
}
template <int M> __device__ __forceinline__ float from_lane(float v) { return __uint_as_float(from_lane<M>(__float_as_uint(v))); }
template <int M> __device__ __forceinline__ u64 from_lane(u64 v) { return (u64)from_lane<M>((unsigned)(v >> 32)) << 32 | from_lane<M>((unsigned)v); }
template <int M> __device__ __forceinline__ double from_lane(double v) { return __builtin_bit_cast(double, from_lane<M>(__builtin_bit_cast(u64, v))); }

// An item of a list of a row, best first: the logit's place in the order of floats, and below it the token's complement, so that
// of equal logits the lower token is the larger number.  0: nothing.
struct InRow {
    u64 key;
    __device__ __forceinline__ bool above(const InRow &o) const { return key > o.key; }
    template <int M> __device__ __forceinline__ InRow lane() const { return {from_lane<M>(key)}; }
};
// An item of a list of an utterance: the score's place in the order of doubles (0: nothing), and the complement of where it
// comes from, hypothesis * 64 + rank in its list.
struct InAll {
    u64 key;
    unsigned from;
    __device__ __forceinline__ bool above(const InAll &o) const { return key > o.key || (key == o.key && from > o.from); }
    template <int M> __device__ __forceinline__ InAll lane() const { return {from_lane<M>(key), from_lane<M>(from)}; }
};

__device__ __forceinline__ u64 row_key(float x, int token)
{
    const unsigned u = __float_as_uint(x + 0.f);                       // (-0 becomes 0)
    return (u64)(u ^ ((unsigned)((int)u >> 31) | 0x80000000u)) << 32 | ~(unsigned)token;
}
__device__ __forceinline__ float key_logit(u64 key)
{
    const unsigned o = (unsigned)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// A step of a sorting network: of lanes M apart the one keeps the better item, which has its bit of M clear or, if not
// `first_up`, set.
template <int M, class Item> __device__ __forceinline__ void exchange(Item &mine, bool better)
{
    const Item other = mine.template lane<M>();
    const bool take = other.above(mine) == better;
    if (take) mine = other;
}
// Lists are 64 items long, or 16 (WIDTH; lanes 0 .. 15, what the others hold does not matter) where no more are wanted.
// The items of a wave or of the 16 lanes of a row of it, worst first
template <int WIDTH, class Item> __device__ __forceinline__ void sort_lanes(Item &v)
{
    const int lane = threadIdx.x & 63;
#define RNNT_STEP(K, M) exchange<M>(v, ((lane & M) == 0) != ((lane & K) == 0 || K == WIDTH))
    RNNT_STEP(2, 1);
    RNNT_STEP(4, 2); RNNT_STEP(4, 1);
    RNNT_STEP(8, 4); RNNT_STEP(8, 2); RNNT_STEP(8, 1);
    RNNT_STEP(16, 8); RNNT_STEP(16, 4); RNNT_STEP(16, 2); RNNT_STEP(16, 1);
    if constexpr (WIDTH == 64) {
        RNNT_STEP(32, 16); RNNT_STEP(32, 8); RNNT_STEP(32, 4); RNNT_STEP(32, 2); RNNT_STEP(32, 1);
        RNNT_STEP(64, 32); RNNT_STEP(64, 16); RNNT_STEP(64, 8); RNNT_STEP(64, 4); RNNT_STEP(64, 2); RNNT_STEP(64, 1);
    }
#undef RNNT_STEP
}
// The best of a list and of another one that is given worst first, as a list
template <int WIDTH, class Item> __device__ __forceinline__ void join(Item &list, const Item &reversed)
{
    const int lane = threadIdx.x & 63;
    if (reversed.above(list)) list = reversed;
    if constexpr (WIDTH == 64) { exchange<32>(list, (lane & 32) == 0); exchange<16>(list, (lane & 16) == 0); }
    exchange<8>(list, (lane & 8) == 0); exchange<4>(list, (lane & 4) == 0); exchange<2>(list, (lane & 2) == 0); exchange<1>(list, (lane & 1) == 0);
}
template <int WIDTH, class Item> __device__ __forceinline__ Item reverse(const Item &v)
{
    const Item r = v.template lane<15>();
    if constexpr (WIDTH == 16) return r;
    else return r.template lane<16>().template lane<32>();
}

template <int TYPE> struct Logit;
template <> struct Logit<RNNT_TYPE_F32> { typedef float T; };
template <> struct Logit<RNNT_TYPE_BF16> { typedef __bf16 T; };
template <> struct Logit<RNNT_TYPE_F16> { typedef _Float16 T; };

// Wave-wide maximum and sum
template <class F> __device__ __forceinline__ F wave_max(F v)
{
    auto larger = [](F a, F b) { if constexpr (sizeof(F) == 4) return fmaxf(a, b); else return fmax(a, b); };
    v = larger(v, from_lane<1>(v)); v = larger(v, from_lane<2>(v)); v = larger(v, from_lane<4>(v));
    v = larger(v, from_lane<8>(v)); v = larger(v, from_lane<16>(v)); return larger(v, from_lane<32>(v));
}
// (The first lane's sum for all of them: where v is a product that the compiler fuses with the first addition, the lanes' differ in their last
// bit, and equal logits would no longer have equal scores.)
__device__ __forceinline__ double wave_sum(double v)
{
    v += from_lane<1>(v); v += from_lane<2>(v); v += from_lane<4>(v);
    v += from_lane<8>(v); v += from_lane<16>(v); v += from_lane<32>(v);
    const u64 u = __builtin_bit_cast(u64, v);
    return __builtin_bit_cast(double, (u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u));
}

constexpr float kLog2E = 1.44269504f, kLowest = -3.402823466e38f;
// Differences of x log2(e) to a rounded shift are off by half a step of the shift, a power of two at 2^24 and beyond all floats at 2^31: where the largest
// logit of all is as far out as kFar, differences of logits are taken, and a lane with lower ones only has the shift kLeast and adds nothing.
constexpr float kFar = 0x1p23f, kLeast = -0x1p24f;
// A running sum is of 2^(x log2(e) - shift) with a whole shift, so that it is rescaled without a rounding, however often: a row that rises
// all along does so in every tile.  (By the hardware's exponential of a difference of shifts, off by up to a unit each time, 5.5e-6
// of a logarithm were lost over 512 tiles, 26e-6 over 2048.)  This is the shift for logits up to `top`, and a sum with shift `from` as one with `to`.
__device__ __forceinline__ float shift_of(float top) { return __builtin_rintf(fmaxf(top * kLog2E, kLeast)); }
__device__ __forceinline__ double rescaled(double sum, float from, float to) { return ldexp(sum, (int)fmaxf(from - to, -2048.f)); }

// One pass over a piece of a row by a wave: the running maximum and sum of a softmax, a lane's own, and the best n of its
// logits.  A tile is 16 logits a lane (and 64 more where the row ends with them: vocabularies are a power of two and a blank).
// A tile none of whose logits is above the n-th best so far goes by at the price of one comparison; of the others a lane
// notes which of its own are, and one a lane at a time they go into a buffer, which is sorted and joined with the list 64 at a time.
// (LONG: for many tiles a wave; where the buffer has room they go there from the registers, 17 places in the code that are mostly skipped.
// For a tile or two that costs more in instructions fetched than it saves: 4 rows of 1025 logits take 6.1 us with it and 5.6 without.)
// Before there is a list, the maxima of n or more groups of lanes bound the n-th best from below.
template <class T, int WIDTH, bool LONG> struct Scan {
    static constexpr int PER = 16 / sizeof(T), LOADS = kTile / 64 / PER, ALL = kTile / 64 + 1;
    struct __attribute__((packed, aligned(sizeof(T)))) At { T e[PER]; };
    const T *row;
    u64 *buffer;
    int n, lane;
    int count = 0;                 // in the buffer
    bool started = false;          // there is a list
    float bar = -INFINITY;         // logits above it are looked at
    // A lane's sum has the shift of its largest logit.  In the end the sum is the wave's, of exp(x - ref): what shift was
    // rounded by is in ref.
    float top = kLowest, shift = kLeast;       // (never -inf: no differences of infinities)
    double sum = 0, ref = 0;
    InRow list{0};

    __device__ __forceinline__ void flush()
    {
        wave_sync();
        const u64 raw = buffer[lane], rest = buffer[lane + 64];
        InRow v{lane < count ? row_key(__uint_as_float((unsigned)(raw >> 32)), (int)(unsigned)raw) : 0};
        wave_sync();
        buffer[lane] = rest;
        if (WIDTH == 16 && count <= 16) sort_lanes<16>(v);
        else {
            sort_lanes<64>(v);
            if constexpr (WIDTH == 16) v = v.template lane<16>().template lane<32>();      // the best 16, worst first, to lanes 0 .. 15
        }
        count = max(count - 64, 0);
        if (started) join<WIDTH>(list, v);
        else list = reverse<WIDTH>(v);
        started = true;
        const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(list.key >> 32), n - 1);
        if (hi != 0u) bar = key_logit((u64)hi << 32);
    }
    __device__ __forceinline__ void first_bar(float m)
    {
        float t = m;
        if (n <= 8) t = fmaxf(t, from_lane<4>(t));
        if (n <= 16) t = fmaxf(t, from_lane<2>(t));
        if (n <= 32) t = fmaxf(t, from_lane<1>(t));
        t = fminf(t, from_lane<32>(t)); t = fminf(t, from_lane<16>(t)); t = fminf(t, from_lane<8>(t));
        if (n > 8) t = fminf(t, from_lane<4>(t));
        if (n > 16) t = fminf(t, from_lane<2>(t));
        if (n > 32) t = fminf(t, from_lane<1>(t));
        // the next lower number: it is among the best itself
        const unsigned u = __float_as_uint(t);
        bar = t == -INFINITY ? t : __uint_as_float(t == 0.f ? 0x80000001u : t > 0.f ? u - 1u : u + 1u);
    }
    At next[LOADS];
    T more;
    __device__ __forceinline__ void load(int base, int to)
    {
#pragma unroll
        for (int q = 0; q < LOADS; ++q) next[q] = *reinterpret_cast<const At *>(row + base + (q * 64 + lane) * PER);
        more = row[base + min(kTile + lane, to - 1 - base)];
    }
    __device__ __forceinline__ void begin(int from, int to) { if (to - from >= kTile) load(from, to); }
    // (tokens may go on to the largest int)
    __device__ __forceinline__ void run(int from, int to)
    {
        for (int base = from; base < to;) {
            const int rest = to - base, size = rest <= kTile + 64 ? rest : kTile;
            const bool full = rest >= kTile;
            float f[ALL];
            if (full) {
#pragma unroll
                for (int i = 0; i < ALL - 1; ++i) f[i] = (float)next[i / PER].e[i % PER];
                f[ALL - 1] = kTile + lane < size ? (float)more : -INFINITY;
                // (of many tiles without a branch, which would wait for the loads at its end: with nothing more to load this tile again)
                if constexpr (LONG) load(rest - size >= kTile ? base + size : base, to);
                else if (rest - size >= kTile) load(base + size, to);
            } else {
                T v[ALL - 1];
#pragma unroll
                for (int i = 0; i < ALL - 1; ++i) v[i] = row[base + min(i * 64 + lane, rest - 1)];
#pragma unroll
                for (int i = 0; i < ALL - 1; ++i) f[i] = i * 64 + lane < rest ? (float)v[i] : -INFINITY;
                f[ALL - 1] = -INFINITY;
            }
            float m = f[0];
#pragma unroll
            for (int i = 1; i < ALL; ++i) m = fmaxf(m, f[i]);
            top = fmaxf(top, m);
            const float now = shift_of(top);
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < ALL; ++i) part[i % 4] += __builtin_amdgcn_exp2f(__builtin_fmaf(f[i], kLog2E, -now));
            sum = rescaled(sum, shift, now) + (double)((part[0] + part[1]) + (part[2] + part[3]));
            shift = now;
            if (base == from) first_bar(m);
            const bool last = size == rest, sort = last || base == from;
            auto place = [&](int i) { return !full ? i * 64 + lane : i < ALL - 1 ? (i / PER * 64 + lane) * PER + i % PER : kTile + lane; };
            auto append = [&](bool in, u64 all, float x, int at) {
                if (in) buffer[count + __builtin_amdgcn_mbcnt_hi((unsigned)(all >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)all, 0u))] = (u64)__float_as_uint(x) << 32 | (unsigned)(base + at);
                count += __popcll(all);
            };
            unsigned mine = 0;                             // a lane's logits above the bar that are to be appended one by one
            if (__ballot(m > bar) != 0ull) {
                u64 above[ALL];
                int found = 0;
                if constexpr (LONG) {
#pragma unroll
                    for (int i = 0; i < ALL; ++i) { above[i] = __ballot(f[i] > bar); found += __popcll(above[i]); }
                }
                if (LONG && count + found <= kBuffer) {
#pragma unroll
                    for (int i = 0; i < ALL; ++i) if (above[i] != 0ull) append(f[i] > bar, above[i], f[i], place(i));
                } else {
#pragma unroll
                    for (int i = ALL - 1; i >= 0; --i) mine = mine + mine + (f[i] > bar ? 1u : 0u);
                }
            }
            for (;;) {
                const bool more_of_it = __ballot(mine != 0u) != 0ull;
                if (more_of_it) {
                    const int at = place(__builtin_ctz(mine | 0x80000000u));
                    const float x = mine != 0u ? (float)row[base + at] : -INFINITY;
                    // (the bar may have risen to a logit with a higher token)
                    const bool in = mine != 0u && x >= bar;
                    append(in, __ballot(in), x, at);
                    mine &= mine - 1u;
                }
                if (count >= 64 || (!more_of_it && sort && count > 0)) flush();
                if (!more_of_it && count < (sort ? 1 : 64)) break;
            }
            base += size;
        }
        top = wave_max(top);
        if (!(fabsf(top) < kFar)) { far(from, to); return; }
        const float all = wave_max(shift);
        sum = wave_sum(rescaled(sum, shift, all));
        ref = (double)all / (double)kLog2E;
    }
    // A row whose largest logit is far out (a mask in all of it; an infinity): the terms are made of differences to it.
    __device__ __forceinline__ void far(int from, int to)
    {
        sum = 0;
        for (int j = lane; j < to - from; j += 64) sum += (double)__builtin_amdgcn_exp2f(((float)row[from + j] - top) * kLog2E);
        sum = wave_sum(sum);
        ref = (double)top;
    }
};

// A hypothesis' row or a piece of it
template <class T, int WIDTH, bool LONG> __device__ __forceinline__ Scan<T, WIDTH, LONG> scan_of(const SelectArgs &a, int b, int k, u64 *buffer)
{
    Scan<T, WIDTH, LONG> s;
    s.row = static_cast<const T *>(a.logits) + b * a.batch_stride + k * a.beam_stride;
    s.buffer = buffer; s.n = a.n_out; s.lane = threadIdx.x & 63;
    return s;
}

// The waves of a work-group make one list of an utterance's rows: hypothesis by hypothesis with its score, then wave by wave.
template <int WIDTH> struct Joined {
    const SelectArgs &a;
    int *tokens;           // [beams][n_out], in LDS
    int lane;
    InAll best{0, 0};
    bool first = true;
    // the best of hypothesis k; ended: its only candidate is the end token
    __device__ __forceinline__ void add(int k, float score, bool ended, InRow list, double ref, double sum)
    {
        double base = (double)score - log(sum);            // (NaN where the row holds a NaN or an infinity)
        if (ended) { base = (double)score; ref = 0; list.key = lane == 0 ? row_key(0.f, a.end_token) : 0; }
        InAll item{0, ~(unsigned)(k * 64 + lane)};
        const double t = base + ((double)key_logit(list.key) - ref) + 0.0;
        const u64 u = __builtin_bit_cast(u64, t);
        if (list.key != 0 && t > -INFINITY) item.key = u >> 63 ? ~u : u | 0x8000000000000000ull;
        if (lane < a.n_out) tokens[k * a.n_out + lane] = (int)~(unsigned)list.key;
        if (first) best = item;
        else join<WIDTH>(best, reverse<WIDTH>(item));
        first = false;
    }
    // tree: [waves][WIDTH] keys and as many words, in LDS
    __device__ __forceinline__ void finish(int b, int wave, int waves, u64 *tree_keys, unsigned *tree_from)
    {
        for (int half = waves / 2; half > 0; half /= 2) {
            if (wave >= half && wave < 2 * half && lane < WIDTH) { tree_keys[wave * WIDTH + lane] = best.key; tree_from[wave * WIDTH + lane] = best.from; }
            __syncthreads();
            const int at = (wave + half) * WIDTH + WIDTH - 1 - lane % WIDTH;
            if (wave < half) join<WIDTH>(best, InAll{tree_keys[at], tree_from[at]});
        }
        if (waves == 1) __syncthreads();                   // (a single wave reads its own tokens)
        if (wave == 0 && lane < a.n_out) {
            const long long o = (long long)b * a.n_out + lane;
            const int from = (int)~best.from, k = from >> 6;
            const u64 u = best.key >> 63 ? best.key ^ 0x8000000000000000ull : ~best.key;
            a.scores_out[o] = best.key ? (float)__builtin_bit_cast(double, u) : -INFINITY;
            a.tokens_out[o] = best.key ? tokens[k * a.n_out + (from & 63)] : -1;
            a.parents_out[o] = best.key ? k : -1;
        }
    }
};

// LDS of a work-group that joins: the waves' buffers or their lists, which take turns, and the tokens
__host__ __device__ constexpr size_t join_lds(int waves, int beams, int n) { return (size_t)waves * kBuffer * 8 + (size_t)beams * n * 4; }

// The hypotheses of an utterance by a work-group, whose waves take them in turn
template <int TYPE, int WIDTH>
__device__ __forceinline__ void select_rows(const SelectArgs &a, unsigned char *lds)
{
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), b = blockIdx.x;
    u64 *buffers = reinterpret_cast<u64 *>(lds);
    Joined<WIDTH> all{a, reinterpret_cast<int *>(buffers + waves * kBuffer), (int)threadIdx.x & 63};
    for (int k = wave; k < a.beams; k += waves) {
        auto s = scan_of<typename Logit<TYPE>::T, WIDTH, false>(a, b, k, buffers + wave * kBuffer);
        s.begin(0, a.V);                                   // (on their way while the score is read)
        const float score = a.scores[(long long)b * a.beams + k];
        const bool ended = a.finished && a.finished[(long long)b * a.beams + k];
        // nothing of a hypothesis that has ended, or that there is not, is looked at
        if (!ended && score > -INFINITY) s.run(0, a.V);
        all.add(k, score, ended, s.list, s.ref, s.sum);
    }
    __syncthreads();
    all.finish(b, wave, waves, buffers, reinterpret_cast<unsigned *>(buffers + waves * 64));
}
template <int TYPE, int WIDTH>
__global__ void __launch_bounds__(kJoinWaves * 64)
beam_select_kernel(const SelectArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    select_rows<TYPE, WIDTH>(a, lds);
}

// Short rows (a tile and a last lane each), a wave for one or two of them, few winners: no lists.  The lanes' largest candidates over all rows are 64
// different ones; the n-th of those bounds the n-th best of the utterance from below, and what is not below the bound, for n = 16 about
// 18 candidates of independent logits, for 32 about 44, is put together in LDS and ranked by counting.  Where ties make more than
// kShort of them, the utterance is done by lists.  bf16, with lists in brackets: 128 utterances of 16 rows of 1025 for 16 winners
// 8.6 us (12.0), of 4 rows for 4 5.3 (6.5); 2048 of 8 rows for 8 25 (33); 2048 of 16 rows of 128 for 16 53 (76).  Every wave counts for itself where
// the bound is, which one or two rows do not repay: 4096 of one row of 1025 for 16 15.2 (11.5), 128 of two 7.5 (7.4).
constexpr int kShort = 128, kShortWinners = 32, kShortLeast = 3, kShortMost = 2 * kJoinWaves, kShortRow = kTile + 64;
struct Candidate {
    u64 key, sub;          // the score's place in the order of doubles; hypothesis (complement), logit's place, token (complement)
    __device__ __forceinline__ bool above(const Candidate &o) const { return key > o.key || (key == o.key && sub > o.sub); }
};
struct ShortLds { unsigned group[64]; Candidate found[kShort]; int count; };

__device__ __forceinline__ unsigned float_key(float f)      // (more than 0, which is nothing)
{
    const unsigned u = __float_as_uint(f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_float(unsigned u) { return u >> 31 ? __uint_as_float(u ^ 0x80000000u) : u ? __uint_as_float(~u) : -INFINITY; }

__device__ __forceinline__ u64 score_key(double t)
{
    const u64 u = __builtin_bit_cast(u64, t + 0.0);
    return t > -INFINITY ? (u >> 63 ? ~u : u | 0x8000000000000000ull) : 0;
}

// The n-th of the lanes' largest scores, rounded down
__device__ __forceinline__ float score_bar(const ShortLds &s, int lane, int n)
{
    const unsigned best = s.group[lane];
    unsigned nth = 0;
#pragma unroll
    for (int bit = 31; bit >= 8; --bit) {
        const unsigned with = nth | 1u << bit;
        if (__popcll(__ballot(best >= with)) >= n) nth = with;
    }
    return key_float(nth);
}
// It in the logits of a row whose scores are base + (logit - ref), and lower by more than all these roundings are off: logits from there on are candidates.
__device__ __forceinline__ float logit_bar(float bar, double base, double ref)
{
    const double at = (double)bar - base + ref;
    return at == at ? fmaxf((float)(at - (fabs(at) + fabs((double)bar) + fabs(ref)) * 1e-6 - 1e-5), kLowest) : kLowest;
}
__device__ __forceinline__ void put_candidate(ShortLds &s, int to, int k, float x, int token, double score)
{
    if (to < kShort) s.found[to] = Candidate{score_key(score), (u64)(63 - k) << 58 | (row_key(x, 0) >> 32) << 26 | (u64)(0x3ffffff - token)};
}
// What the waves have put together, or, where that is too much, the utterance by lists
template <int TYPE, int WIDTH>
__device__ __forceinline__ void rank_candidates(const SelectArgs &a, ShortLds &s, unsigned char *lds)
{
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, b = blockIdx.x, n = a.n_out;
    __syncthreads();
    const int count = s.count;
    if (count > kShort) {                                  // (the whole work-group)
        __syncthreads();
        select_rows<TYPE, WIDTH>(a, lds);
        return;
    }
    // a wave ranks every waves-th candidate: how many are above it
    const Candidate own[2] = {lane < count ? s.found[lane] : Candidate{0, 0}, lane + 64 < count ? s.found[lane + 64] : Candidate{0, 0}};
    for (int c = wave; c < count; c += waves) {
        const Candidate it = s.found[c];
        const int rank = __popcll(__ballot(own[0].above(it))) + __popcll(__ballot(own[1].above(it)));
        if (lane == 0 && rank < n && it.key != 0) {
            const long long o = (long long)b * n + rank;
            const u64 u = it.key >> 63 ? it.key ^ 0x8000000000000000ull : ~it.key;
            a.scores_out[o] = (float)__builtin_bit_cast(double, u);
            a.tokens_out[o] = 0x3ffffff - (int)(it.sub & 0x3ffffff);
            a.parents_out[o] = 63 - (int)(it.sub >> 58);
        }
    }
    const int there = __popcll(__ballot(own[0].key != 0)) + __popcll(__ballot(own[1].key != 0));
    if (wave == 0 && lane >= there && lane < n) {
        const long long o = (long long)b * n + lane;
        a.scores_out[o] = -INFINITY; a.tokens_out[o] = -1; a.parents_out[o] = -1;
    }
}

// WIDTH: of the lists, where they are needed; ROWS: of a wave
template <int TYPE, int WIDTH, int ROWS>
__global__ void __launch_bounds__(kJoinWaves * 64)
beam_short_kernel(const SelectArgs a)
{
    typedef typename Logit<TYPE>::T T;
    constexpr int PER = 16 / (int)sizeof(T), LOADS = kTile / 64 / PER, ALL = kTile / 64 + 1;
    struct __attribute__((packed, aligned(sizeof(T)))) At { T e[PER]; };
    extern __shared__ __align__(16) unsigned char lds[];
    ShortLds &s = *reinterpret_cast<ShortLds *>(lds);
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, b = blockIdx.x, n = a.n_out;
    const bool full = a.V >= kTile;
    // the rows' logits, 17 a lane; `place`: where in the row
    float f[ROWS][ALL], scores[ROWS];
    bool ended[ROWS], live[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int k = wave + r * waves;
        const bool has_row = k < a.beams;
        const long long hyp = (long long)b * a.beams + (has_row ? k : 0);
        const T *row = static_cast<const T *>(a.logits) + b * a.batch_stride + (has_row ? k : 0) * a.beam_stride;
        if (full) {
            At v[LOADS];
#pragma unroll
            for (int q = 0; q < LOADS; ++q) v[q] = *reinterpret_cast<const At *>(row + (q * 64 + lane) * PER);
            const T more = row[min(kTile + lane, a.V - 1)];
#pragma unroll
            for (int i = 0; i < ALL - 1; ++i) f[r][i] = (float)v[i / PER].e[i % PER];
            f[r][ALL - 1] = kTile + lane < a.V ? (float)more : -INFINITY;
        } else {
            T v[ALL - 1];
#pragma unroll
            for (int i = 0; i < ALL - 1; ++i) v[i] = row[min(i * 64 + lane, a.V - 1)];
#pragma unroll
            for (int i = 0; i < ALL - 1; ++i) f[r][i] = i * 64 + lane < a.V ? (float)v[i] : -INFINITY;
            f[r][ALL - 1] = -INFINITY;
        }
        scores[r] = a.scores[hyp];
        ended[r] = has_row && a.finished && a.finished[hyp];
        live[r] = has_row && !ended[r] && scores[r] > -INFINITY;
    }
    auto place = [&](int i) { return !full ? i * 64 + lane : i < ALL - 1 ? (i / PER * 64 + lane) * PER + i % PER : kTile + lane; };
    if (wave == 0) { s.group[lane] = 0; if (lane == 0) s.count = 0; }
    float m[ROWS], top[ROWS];
    double base[ROWS];
    auto total = [&](int r, float x) { return base[r] + ((double)x - (double)top[r]); };
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        m[r] = f[r][0];
#pragma unroll
        for (int i = 1; i < ALL; ++i) m[r] = fmaxf(m[r], f[r][i]);
        top[r] = fmaxf(wave_max(m[r]), kLowest);
        // (differences to the largest logit: at the ends of the type, too)
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ALL; ++i) part[i % 4] += __builtin_amdgcn_exp2f((f[r][i] - top[r]) * kLog2E);
        base[r] = (double)scores[r] - log(wave_sum((double)((part[0] + part[1]) + (part[2] + part[3]))));      // (NaN where the row holds a NaN or an infinity)
    }
    __syncthreads();                                       // (the cleared LDS)
    double t = -INFINITY;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) if (live[r] && m[r] > -INFINITY && base[r] == base[r]) t = fmax(t, total(r, m[r]));
    if (t > -INFINITY) atomicMax(&s.group[lane], float_key((float)t));
    __syncthreads();
    const float bar = score_bar(s, lane, n);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const float low = logit_bar(bar, base[r], (double)top[r]);
        const int k = wave + r * waves;
        u64 in[ALL];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < ALL; ++i) { in[i] = live[r] && base[r] == base[r] ? __ballot(f[r][i] >= low) : 0; mine += __popcll(in[i]); }
        if (ended[r]) mine = 1;
        if (mine == 0) continue;
        int from = 0;
        if (lane == 0) from = atomicAdd(&s.count, mine);
        from = __builtin_amdgcn_readfirstlane(from);
        if (ended[r]) { if (lane == 0) put_candidate(s, from, k, 0.f, a.end_token, (double)scores[r]); continue; }
#pragma unroll
        for (int i = 0; i < ALL; ++i) {
            if (in[i] == 0ull) continue;
            if (in[i] >> lane & 1)
                put_candidate(s, from + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(in[i] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)in[i], 0u)), k, f[r][i], place(i), total(r, f[r][i]));
            from += __popcll(in[i]);
        }
    }
    rank_candidates<TYPE, WIDTH>(a, s, lds);
}

// A row or a piece of one that a wave holds as a whole, kHeld loads a lane
constexpr int kHeld = 16, kHeldWinners = 32;
template <class T> constexpr int held_size() { return kHeld * 64 * 16 / (int)sizeof(T); }
template <class T> struct Held {
    static constexpr int PER = 16 / (int)sizeof(T);
    struct __attribute__((packed, aligned(sizeof(T)))) At { T e[PER]; };
    const T *row;
    int rest, lane;
    At held[kHeld];
    float most[kHeld], m;          // the lane's largest of each load, and of all
    double sum, ref;               // the wave's, of exp(x - ref)
    // A load that would go on behind the end is the last one before it (a row has PER logits or more); `twice`
    // of its logits are another load's, or another wave's.
    __device__ __forceinline__ int off(int q) const { return min((q * 64 + lane) * PER, rest - PER); }
    __device__ __forceinline__ void load()
    {
#pragma unroll
        for (int q = 0; q < kHeld; ++q) held[q] = *reinterpret_cast<const At *>(row + off(q));
    }
    // (a lane's running maximum and sum, as in Scan, sixteen logits at a time: made while others are on their way)
    __device__ __forceinline__ void add_up()
    {
        constexpr int LOADS = 16 / PER;
        float shift = kLeast;
        m = -INFINITY;
        sum = 0;
#pragma unroll
        for (int q0 = 0; q0 < kHeld; q0 += LOADS) {
#pragma unroll
            for (int q = q0; q < q0 + LOADS; ++q) {
                most[q] = -INFINITY;
                if (q * 64 * PER >= rest) continue;
                if ((q + 1) * 64 * PER > rest) {
                    const int twice = (q * 64 + lane) * PER - off(q);
#pragma unroll
                    for (int e = 0; e < PER; ++e) if (e < twice) held[q].e[e] = (T)-INFINITY;
                }
#pragma unroll
                for (int e = 0; e < PER; ++e) most[q] = fmaxf(most[q], (float)held[q].e[e]);
                m = fmaxf(m, most[q]);
            }
            if (q0 * 64 * PER >= rest) continue;
            const float now = shift_of(m);
            float part[2] = {0.f, 0.f};
#pragma unroll
            for (int q = q0; q < q0 + LOADS; ++q) {
                if (q * 64 * PER >= rest) continue;
#pragma unroll
                for (int e = 0; e < PER; ++e) part[e % 2] += __builtin_amdgcn_exp2f(__builtin_fmaf((float)held[q].e[e], kLog2E, -now));
            }
            sum = rescaled(sum, shift, now) + (double)(part[0] + part[1]);
            shift = now;
        }
        const float top = wave_max(fmaxf(m, kLowest));
        if (!(fabsf(top) < kFar)) {
            sum = 0;
#pragma unroll 1
            for (int j = lane; j < rest; j += 64) sum += (double)__builtin_amdgcn_exp2f(((float)row[j] - top) * kLog2E);
            sum = wave_sum(sum);
            ref = (double)top;
            return;
        }
        const float all = wave_max(shift);
        sum = wave_sum(rescaled(sum, shift, all));
        ref = (double)all / (double)kLog2E;
    }
    // put(logit, place) for each logit from `low` on
    template <class Put> __device__ __forceinline__ void each(float low, Put &&put)
    {
        // (widened anew: kept, they would take twice the registers)
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            v4u raw = __builtin_bit_cast(v4u, held[q]);
            asm volatile("" : "+v"(raw));
            held[q] = __builtin_bit_cast(At, raw);
        }
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            if (__ballot(most[q] >= low) == 0ull) continue;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const float x = (float)held[q].e[e];
                if (x >= low) put(x, off(q) + e);
            }
        }
    }
};

// Rows of a few tiles, one for each wave, the way of the short ones
template <int TYPE, int WIDTH>
__global__ void __launch_bounds__(kJoinWaves * 64)
beam_row_kernel(const SelectArgs a)
{
    typedef typename Logit<TYPE>::T T;
    extern __shared__ __align__(16) unsigned char lds[];
    ShortLds &s = *reinterpret_cast<ShortLds *>(lds);
    const int k = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, b = blockIdx.x;
    const bool has_row = k < a.beams;
    const long long hyp = (long long)b * a.beams + (has_row ? k : 0);
    Held<T> h;
    h.row = static_cast<const T *>(a.logits) + b * a.batch_stride + (has_row ? k : 0) * a.beam_stride;
    h.rest = a.V;
    h.lane = lane;
    h.load();
    const float score = a.scores[hyp];
    const bool ended = has_row && a.finished && a.finished[hyp], live = has_row && !ended && score > -INFINITY;
    if (k == 0) { s.group[lane] = 0; if (lane == 0) s.count = 0; }
    double base = 0;
    h.ref = 0;
    if (live) {
        h.add_up();
        base = (double)score - log(h.sum);                 // (NaN where the row holds a NaN or an infinity)
    }
    auto total = [&](float x) { return base + ((double)x - h.ref); };
    const bool good = live && base == base;
    __syncthreads();                                       // (the cleared LDS)
    if (good && h.m > -INFINITY) {
        const double t = total(h.m);
        if (t > -INFINITY) atomicMax(&s.group[lane], float_key((float)t));
    }
    __syncthreads();
    const float low = logit_bar(score_bar(s, lane, a.n_out), base, h.ref);
    if (good) h.each(low, [&](float x, int token) { put_candidate(s, atomicAdd(&s.count, 1), k, x, token, total(x)); });
    if (ended && lane == 0) put_candidate(s, atomicAdd(&s.count, 1), k, 0.f, a.end_token, (double)score);
    rank_candidates<TYPE, WIDTH>(a, s, lds);
}

// Long rows: pieces over the whole device, joined by a second launch.  A work-group's waves have four pieces
// of a row and join their lists, two by two.
constexpr int kScanWaves = 4;
struct ScanLds { u64 buffers[kScanWaves][kBuffer]; double sums[kScanWaves], refs[kScanWaves]; };
struct ScanPiece { unsigned hyp, b; int from, to; };
__device__ __forceinline__ ScanPiece piece_of(const SelectArgs &a, int wave)
{
    const unsigned hyp = blockIdx.x / a.pieces;
    const long long piece = (long long)(blockIdx.x - hyp * a.pieces) * kScanWaves + wave;
    return {hyp, hyp / a.beams, (int)min(piece * a.piece_tiles * kTile, (long long)a.V), (int)min((piece + 1) * a.piece_tiles * kTile, (long long)a.V)};
}
__device__ __forceinline__ void store_list(const SelectArgs &a, const ScanLds &lds, int lane, u64 key)
{
    if (lane < a.n_out) a.lists[(long long)blockIdx.x * a.n_out + lane] = key;
    if (lane < kScanWaves) { a.sums[(long long)blockIdx.x * kScanWaves + lane] = lds.sums[lane]; a.refs[(long long)blockIdx.x * kScanWaves + lane] = lds.refs[lane]; }
}
template <int TYPE, int WIDTH>
__device__ __forceinline__ void scan_pieces(const SelectArgs &a, ScanLds &lds)
{
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const ScanPiece p = piece_of(a, wave);
    auto s = scan_of<typename Logit<TYPE>::T, WIDTH, true>(a, (int)p.b, (int)(p.hyp - p.b * a.beams), lds.buffers[wave]);
    s.begin(p.from, p.to);
    if ((a.finished && a.finished[p.hyp]) || !(a.scores[p.hyp] > -INFINITY)) return;       // (the whole work-group)
    s.run(p.from, p.to);
    if (lane == 0) { lds.sums[wave] = s.sum; lds.refs[wave] = s.ref; }
    for (int half = kScanWaves / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half && lane < WIDTH) lds.buffers[wave][lane] = s.list.key;
        __syncthreads();
        if (wave < half) join<WIDTH>(s.list, InRow{lds.buffers[wave + half][WIDTH - 1 - lane % WIDTH]});
    }
    if (wave == 0) store_list(a, lds, lane, s.list.key);
}
template <int TYPE, int WIDTH>
__global__ void __launch_bounds__(kScanWaves * 64)
beam_scan_kernel(const SelectArgs a)
{
    __shared__ ScanLds lds;
    scan_pieces<TYPE, WIDTH>(a, lds);
}

// The same for few winners and pieces that a wave holds as a whole, kHeld loads a lane.  The lanes' largest logits in the four pieces are 64
// different ones; the n-th of them bounds the n-th best from below, and what is not below it, for n = 8 about nine logits of four pieces, is the
// list.  Where ties make more than 64 of them, the work-group does its pieces the other way.  Bound by memory, and by the exponentials behind it: 67 MB
// of f16 logits (64 x 8 rows of 65535) 18 us (lists: 24), 14 without the sums and the list.
template <int TYPE, int WIDTH>
__global__ void __launch_bounds__(kScanWaves * 64, 4)
beam_held_kernel(const SelectArgs a)
{
    typedef typename Logit<TYPE>::T T;
    __shared__ ScanLds lds;
    __shared__ u64 found[64];
    __shared__ unsigned group[64];
    __shared__ int found_count;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const ScanPiece p = piece_of(a, wave);
    Held<T> h;
    h.row = static_cast<const T *>(a.logits) + p.b * a.batch_stride + (p.hyp - p.b * a.beams) * a.beam_stride + p.from;
    h.rest = p.to - p.from;
    h.lane = lane;
    h.load();
    if ((a.finished && a.finished[p.hyp]) || !(a.scores[p.hyp] > -INFINITY)) return;       // (the whole work-group)
    if (wave == 0) { group[lane] = 0; if (lane == 0) found_count = 0; }
    h.add_up();
    if (lane == 0) { lds.sums[wave] = h.sum; lds.refs[wave] = h.ref; }
    __syncthreads();                                       // (the cleared LDS)
    if (h.m > -INFINITY) atomicMax(&group[lane], (unsigned)(row_key(h.m, 0) >> 32));
    __syncthreads();
    const unsigned best = group[lane];
    unsigned nth = 0;                                      // (its highest 20 bits: from a little lower on)
#pragma unroll
    for (int bit = 31; bit >= 12; --bit) if (__popcll(__ballot(best >= (nth | 1u << bit))) >= a.n_out) nth |= 1u << bit;
    h.each(fmaxf(key_logit((u64)nth << 32), kLowest), [&](float x, int token) {
        const int at = atomicAdd(&found_count, 1);
        if (at < 64) found[at] = row_key(x, p.from + token);
    });
    __syncthreads();
    const int count = found_count;
    if (count > 64) {                                      // (the whole work-group)
        scan_pieces<TYPE, WIDTH>(a, lds);
        return;
    }
    if (wave != 0) return;
    InRow v{lane < count ? found[lane] : 0};
    if (WIDTH == 16 && count <= 16) sort_lanes<16>(v);
    else {
        sort_lanes<64>(v);
        if constexpr (WIDTH == 16) v = v.template lane<16>().template lane<32>();     // the best 16, worst first, to lanes 0 .. 15
    }
    store_list(a, lds, lane, reverse<WIDTH>(v).key);
}
template <int WIDTH>
__global__ void __launch_bounds__(kJoinWaves * 64)
beam_join_kernel(const SelectArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, b = blockIdx.x, n = a.n_out;
    u64 *tree = reinterpret_cast<u64 *>(lds);
    Joined<WIDTH> all{a, reinterpret_cast<int *>(tree + waves * kBuffer), lane};
    for (int k = wave; k < a.beams; k += waves) {
        const long long hyp = (long long)b * a.beams + k;
        // (asked for together, whether they are there or not: the tables are)
        const u64 *mine = a.lists + hyp * a.pieces * n;
        const u64 first = mine[min(lane, n - 1)];
        const bool mine_too = lane < a.pieces * kScanWaves;
        const long long sum_at = hyp * a.pieces * kScanWaves + (mine_too ? lane : 0);
        const double piece_ref = a.refs[sum_at], piece_sum = a.sums[sum_at];
        const float score = a.scores[hyp];
        const bool ended = a.finished && a.finished[hyp];
        InRow list{0};
        double ref = 0, sum = 0;
        if (!ended && score > -INFINITY) {
            list.key = lane < n ? first : 0;
            for (int s = 1; s < a.pieces; ++s) {
                const int at = WIDTH - 1 - lane % WIDTH;
                join<WIDTH>(list, InRow{at < n ? mine[s * n + at] : 0});
            }
            // (a wave without logits has a sum of 0)
            ref = wave_max(mine_too && piece_sum != 0.0 ? piece_ref : -(double)INFINITY);
            sum = wave_sum(mine_too && piece_sum != 0.0 ? piece_sum * exp(piece_ref - ref) : 0.0);
        }
        all.add(k, score, ended, list, ref, sum);
    }
    __syncthreads();
    all.finish(b, wave, waves, tree, reinterpret_cast<unsigned *>(tree + waves * 64));
}

// A state as the reorder kernel moves it: rows in columns of `width` bytes.  Out of place a work-group takes kItems
// columns of all rows of an utterance (of one o), row behind row; in place the same 256 columns of every row.
constexpr int kUnroll = 8, kItems = 256 * kUnroll;
constexpr double kStreamBytes = 32 << 20;                             // the L2s of the eight XCDs together
struct ReorderState {
    const char *src;
    char *dst;
    long long src_outer, src_batch, src_beam, dst_outer, dst_batch, dst_beam;
    unsigned columns, width;
    unsigned chunks;        // work-groups of an utterance
    unsigned inverse;       // 2^32 / columns, rounded up, where there are fewer columns than kItems
    unsigned in_place;
};
struct ReorderArgs {
    unsigned first[RNNT_BEAM_STATES];   // the states' first work-groups, side by side: one load finds a work-group's state
    ReorderState s[RNNT_BEAM_STATES];
    const int *parents;
    int n, B, beams_in, beams_out;
};


// Memory bound.  Eight loads of a thread are on their way together, whatever rows they are of.  STREAM: the stores are marked as not
// to be kept in the L2s, for calls that write more than those hold (kStreamBytes).  128 utterances of 16 beams, 67 MB of
// states: 30.4 us without the mark, 20.8 with it (6.4 TB/s); what a small call writes, the next kernel reads there.
template <bool STREAM, class T>
__device__ __forceinline__ void move_items(const ReorderState &s, const int *parents, unsigned chunk, long long o, long long b, int beams_in, int beams_out)
{
    const char *from = s.src + o * s.src_outer + b * s.src_batch;
    char *to = s.dst + o * s.dst_outer + b * s.dst_batch;
    const unsigned long long start = (unsigned long long)chunk * kItems;
    unsigned row0 = 0;                                     // start / columns, bit by bit
#pragma unroll
    for (unsigned bit = kMaxBeams / 2; bit > 0; bit /= 2) if ((unsigned long long)(row0 + bit) * s.columns <= start) row0 += bit;
    const unsigned col0 = (unsigned)(start - (unsigned long long)row0 * s.columns);
    // row and column of the thread's i-th item.  (With fewer than kItems columns the number below is under 2 kItems, and the
    // quotient by the inverse exact; with more it is under two rows.)
    auto item = [&](int i, unsigned &j, unsigned &c) {
        const unsigned at = col0 + i * 256 + threadIdx.x;
        const unsigned down = s.columns >= (unsigned)kItems ? (at >= s.columns ? 1u : 0u) : s.columns > 1 ? __umulhi(at, s.inverse) : at;
        j = row0 + down;
        c = at - down * s.columns;
    };
    T v[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        unsigned j, c;
        item(i, j, c);
        // (where there is no source, the first row's column stands in: no branch around a load)
        const bool in = j < (unsigned)beams_out;
        const int p = parents[in ? j : 0u];
        const bool there = in && p >= 0 && p < beams_in;
        v[i] = *reinterpret_cast<const T *>(from + (there ? p * s.src_beam : 0ll) + (unsigned long long)(in ? c : 0u) * sizeof(T));
        if (!there) v[i] = T{};
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        unsigned j, c;
        item(i, j, c);
        if (j >= (unsigned)beams_out) continue;
        T *at = reinterpret_cast<T *>(to + j * s.dst_beam + (unsigned long long)c * sizeof(T));
        if constexpr (STREAM) __builtin_nontemporal_store(v[i], at);
        else *at = v[i];
    }
}

// Within itself: a thread has one column of all rows, and has read every source before it writes.  A row that stays where it
// is, is left alone.
template <class T, int BEAMS>
__device__ __forceinline__ void move_within(const ReorderState &s, const int *parents, unsigned c, long long o, long long b, int beams)
{
    if (c >= s.columns) return;
    char *at = s.dst + o * s.dst_outer + b * s.dst_batch + (unsigned long long)c * sizeof(T);
    // (no branch around a load: where there is no source, or no such row, a row that there is stands in)
    T v[BEAMS];
#pragma unroll
    for (int j = 0; j < BEAMS; ++j) {
        const int row = min(j, beams - 1), p = parents[row];
        const bool there = p >= 0 && p < beams;
        v[j] = *reinterpret_cast<const T *>(at + (there ? p : row) * s.dst_beam);
        if (!there) v[j] = T{};
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < BEAMS; ++j)
        if (j < beams && parents[j] != j) *reinterpret_cast<T *>(at + j * s.dst_beam) = v[j];
}

// BEAMS: room for the rows of an utterance that is moved within itself (0: no state is)
template <int BEAMS, bool STREAM>
__global__ void __launch_bounds__(256)
beam_reorder_kernel(const ReorderArgs a)
{
    unsigned i = 0, at = blockIdx.x;
#pragma unroll
    for (int k = 1; k < RNNT_BEAM_STATES; ++k) if (blockIdx.x >= a.first[k]) { i = k; at = blockIdx.x - a.first[k]; }
    const ReorderState &s = a.s[i];
    const unsigned set = at / s.chunks, chunk = at - set * s.chunks;
    const long long o = set / a.B, b = set - o * a.B;
    const int *parents = a.parents + b * a.beams_out;
    if constexpr (BEAMS > 0) {
        if (s.in_place) {
            const unsigned c = chunk * 256 + threadIdx.x;
            switch (s.width) {
            case 16: if constexpr (BEAMS <= 16) move_within<v4u, BEAMS>(s, parents, c, o, b, a.beams_out); break;
            case 8: move_within<v2u, BEAMS>(s, parents, c, o, b, a.beams_out); break;
            case 4: move_within<unsigned, BEAMS>(s, parents, c, o, b, a.beams_out); break;
            case 2: move_within<unsigned short, BEAMS>(s, parents, c, o, b, a.beams_out); break;
            default: move_within<unsigned char, BEAMS>(s, parents, c, o, b, a.beams_out); break;
            }
            return;
        }
    }
    switch (s.width) {
    case 16: move_items<STREAM, v4u>(s, parents, chunk, o, b, a.beams_in, a.beams_out); break;
    case 8: move_items<STREAM, v2u>(s, parents, chunk, o, b, a.beams_in, a.beams_out); break;
    case 4: move_items<STREAM, unsigned>(s, parents, chunk, o, b, a.beams_in, a.beams_out); break;
    case 2: move_items<STREAM, unsigned short>(s, parents, chunk, o, b, a.beams_in, a.beams_out); break;
    default: move_items<STREAM, unsigned char>(s, parents, chunk, o, b, a.beams_in, a.beams_out); break;
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

constexpr int64_t kMostThreads = 0xffffffff;                                // of a launch, at most
bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// How a selection is cut up.  One launch, a work-group an utterance: short rows; rows that a wave holds as a whole, where there are few winners
// for each of its waves to rank, and no more than kOneRowTiles tiles a work-group or kOneRowUtterances of them; and by lists, where a wave has no
// more than kOneLaunchTiles tiles, of fewer than kWavesWanted rows that could be held in pieces kFewTiles: the second launch costs what a wave takes
// for several tiles.  Else pieces of two tiles or more, towards sixteen waves on every compute unit; lists in pieces of fewer than kWavesWanted rows only.
// us of the kernels, bf16, rows held whole and the other way (pieces, or lists where rows are two tiles or 4096).  Tiles: 16 x 16 rows of 4097
// for 16 12.2 and 12.9, 64 x 16 12.5 and 16.5, 16 x 16 of 6000 12.4 and 12.2, 512 x 16 28.9 and 52.9; beyond kOneRowTiles 16 x 16 of 8000 13.8 and 12.1,
// 48 x 16 of 8192 14.5 and 14.4, 64 x 16 of 8000 14.5 and 15.4, 256 x 16 18.0 and 30.6.  Winners a wave, kRowWinners = 4: one row of 4097 for 4 6.9 and 7.5,
// for 8 9.1 and 8.1; 64 x 2 of 4097 for 8 8.8 and 9.7, for 16 11.3 and 10.5; 4096 x 2 of 8000 for 8 33.5 and 53.9, for 16 40.3 and 58.8; 64 x 4 of 4097
// for 16 10.4 and 11.1, for 24 12.6 and 11.8; 64 x 8 of 8192 for 32 14.6 and 13.0, 300 x 8 21.0 and 29.6.  Of one or two rows that are short, where lists are one tile's,
// as many winners a wave as there are waves: one of 1025 for one 4.6 and 4.8, for 2 5.3 and 4.8; 128 x 2 for 4 6.3 and 6.4, for 8 7.3 and 6.4.
// By lists and in pieces: 128 x 20 of 4000 for 20 28.6 and 22.6, 8 x 32 of 2000 for 32 32 and 14.7, 512 x 4 of 65537 for 4 69 and 54, but
// 128 x 32 of 2000 for 32 32 and 34.
constexpr int kOneLaunchTiles = 8, kOneRowTiles = 96, kOneRowUtterances = 48, kRowWinners = 4, kFewTiles = 2, kWavesWanted = 4096, kMostPieces = 64 / kScanWaves;

struct SelectPlan {
    bool two = false, is_short = false, one_row = false, held = false;
    int pieces = 1, piece_tiles = 1, waves = 1;
    size_t lds = 0;
    int64_t bytes = 0;
    SelectPlan(int type, int64_t B, int beams, int V, int n)
    {
        const int row = (V - 1) / kTile + 1;
        while (waves < kJoinWaves && waves < beams) waves *= 2;
        is_short = V <= kShortRow && beams >= kShortLeast && beams <= kShortMost && n <= kShortWinners;
        lds = std::max(join_lds(waves, beams, n), sizeof(ShortLds));
        // (rows that waves hold as a whole: in no more pieces than the join takes)
        const int most = (type == RNNT_TYPE_F32 ? held_size<float>() : held_size<__bf16>()) / kTile;
        held = n <= kHeldWinners && V >= 8 && (row + most * kScanWaves - 1) / (most * kScanWaves) <= kMostPieces;
        one_row = !is_short && held && row <= most && beams <= kJoinWaves && n <= waves * (V > kShortRow ? kRowWinners : waves) &&
                  (row * waves <= kOneRowTiles || B >= kOneRowUtterances);
        if (is_short || one_row || (beams + waves - 1) / waves * row <= (held && B * beams < kWavesWanted ? kFewTiles : kOneLaunchTiles) || (!held && B * beams >= kWavesWanted)) return;
        two = true;
        const int64_t into = std::min<int64_t>(std::max<int64_t>(kWavesWanted / (B * beams * kScanWaves), 1), std::min(kMostPieces, (row + 2 * kScanWaves - 1) / (2 * kScanWaves)));
        piece_tiles = (int)((row + into * kScanWaves - 1) / (into * kScanWaves));
        if (held) piece_tiles = std::min(piece_tiles, most);
        pieces = (row + piece_tiles * kScanWaves - 1) / (piece_tiles * kScanWaves);
        bytes = B * beams * pieces * (n * 8 + kScanWaves * 16);
    }
};

}  // namespace

extern "C" {

int rnnt_beam_select_workspace(int32_t B, int32_t beams, int32_t V, int32_t n_out, int64_t *bytes_out)
{
    if (!bytes_out) return RNNT_ERR_NULL;
    if (B < 0 || beams < 1 || beams > kMaxBeams || V < 1 || n_out < 1 || n_out > kMaxBeams) return RNNT_ERR_SHAPE;
    if ((int64_t)beams * V > 0x7fffffff) return RNNT_ERR_UNSUPPORTED;
    // (enough for logits of any type)
    *bytes_out = B > 0 ? std::max(SelectPlan(RNNT_TYPE_F32, B, beams, V, n_out).bytes, SelectPlan(RNNT_TYPE_BF16, B, beams, V, n_out).bytes) : 0;
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
    const SelectPlan p(type, B, beams, V, n_out);
    if ((int64_t)B * p.waves * 64 > kMostThreads) return RNNT_ERR_UNSUPPORTED;
    SelectArgs args{logits, scores, finished, scores_out, tokens_out, parents_out, batch_stride, beam_stride, B, beams, V, n_out, end_token,
                    p.pieces, p.piece_tiles, nullptr, nullptr, nullptr};
    const hipStream_t on = static_cast<hipStream_t>(stream);
    if (!p.two) {
        auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(B), dim3(p.waves * 64), (unsigned)p.lds, on, args); };
        auto with = [&](auto t) {
            if (p.one_row && n_out <= 16) run(beam_row_kernel<t(), 16>);
            else if (p.one_row) run(beam_row_kernel<t(), 64>);
            else if (p.is_short && p.waves < beams) run(beam_short_kernel<t(), 64, 2>);
            else if (p.is_short && n_out <= 16) run(beam_short_kernel<t(), 16, 1>);
            else if (p.is_short) run(beam_short_kernel<t(), 64, 1>);
            else if (n_out <= 16) run(beam_select_kernel<t(), 16>);
            else run(beam_select_kernel<t(), 64>);
        };
        if (type == RNNT_TYPE_F32) with(std::integral_constant<int, RNNT_TYPE_F32>());
        else if (type == RNNT_TYPE_BF16) with(std::integral_constant<int, RNNT_TYPE_BF16>());
        else with(std::integral_constant<int, RNNT_TYPE_F16>());
        BEAM_TRY(hipGetLastError());
        return RNNT_OK;
    }
    const int64_t n = (int64_t)B * beams * p.pieces;
    if (n * kScanWaves * 64 > kMostThreads) return RNNT_ERR_UNSUPPORTED;
    args.lists = static_cast<u64 *>(workspace);
    args.sums = reinterpret_cast<double *>(args.lists + n * n_out);
    args.refs = args.sums + n * kScanWaves;
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(kScanWaves * 64), 0, on, args); };
    auto with = [&](auto t) {
        if (p.held && n_out <= 16) run(beam_held_kernel<t(), 16>);
        else if (p.held) run(beam_held_kernel<t(), 64>);
        else if (n_out <= 16) run(beam_scan_kernel<t(), 16>);
        else run(beam_scan_kernel<t(), 64>);
    };
    if (type == RNNT_TYPE_F32) with(std::integral_constant<int, RNNT_TYPE_F32>());
    else if (type == RNNT_TYPE_BF16) with(std::integral_constant<int, RNNT_TYPE_BF16>());
    else with(std::integral_constant<int, RNNT_TYPE_F16>());
    BEAM_TRY(hipGetLastError());
    auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(B), dim3(p.waves * 64), (unsigned)p.lds, on, args); };
    if (n_out <= 16) join(beam_join_kernel<16>); else join(beam_join_kernel<64>);
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
    for (unsigned &f : args.first) f = 0xffffffffu;
    args.parents = parents;
    args.B = B; args.beams_in = beams_in; args.beams_out = beams_out;
    int64_t groups = 0;
    bool any_within = false;
    double bytes = 0;
    for (int i = 0; i < n_states; ++i) {
        const rnnt_beam_state &s = states[i];
        if (s.outer < 0 || s.row_bytes < 0 || s.src_outer < 0 || s.src_batch < 0 || s.src_beam < 0 || s.dst_outer < 0 || s.dst_batch < 0 || s.dst_beam < 0)
            return RNNT_ERR_SHAPE;
        if ((beams_out > 1 && s.dst_beam < s.row_bytes) || (B > 1 && s.dst_batch < s.row_bytes) || (s.outer > 1 && s.dst_outer < s.row_bytes)) return RNNT_ERR_SHAPE;
        if (s.src == s.dst && s.src && (beams_in != beams_out || s.src_outer != s.dst_outer || s.src_batch != s.dst_batch || s.src_beam != s.dst_beam))
            return RNNT_ERR_SHAPE;
        if (B == 0 || s.outer == 0 || s.row_bytes == 0) continue;
        if (!s.src || !s.dst || !parents) return RNNT_ERR_NULL;
        // the widest piece that divides addresses, strides and rows (in place, where a thread holds a column
        // of all rows, with more than 16 rows 8 bytes)
        const bool within = s.src == s.dst;
        const uint64_t all = reinterpret_cast<uintptr_t>(s.src) | reinterpret_cast<uintptr_t>(s.dst) | (uint64_t)s.row_bytes | (uint64_t)s.src_outer |
                             (uint64_t)s.src_batch | (uint64_t)s.src_beam | (uint64_t)s.dst_outer | (uint64_t)s.dst_batch | (uint64_t)s.dst_beam | (within && beams_out > 16 ? 8u : 16u);
        const unsigned width = (unsigned)(all & (~all + 1));
        const int64_t columns = s.row_bytes / width, chunks = within ? (columns + 255) / 256 : (columns * beams_out + kItems - 1) / kItems;
        if (columns > 0x7fffffff - kItems || s.outer > 0x7fffffff / B || chunks > 0x7fffffff / (s.outer * B)) return RNNT_ERR_UNSUPPORTED;
        args.first[args.n] = (unsigned)groups;
        args.s[args.n++] = ReorderState{static_cast<const char *>(s.src), static_cast<char *>(s.dst), s.src_outer, s.src_batch, s.src_beam, s.dst_outer,
                                        s.dst_batch, s.dst_beam, (unsigned)columns, width, (unsigned)chunks,
                                        columns > 1 && columns < kItems ? (unsigned)(0x100000000ull / columns + 1) : 0u, within ? 1u : 0u};
        any_within = any_within || within;
        bytes += (double)s.row_bytes * beams_out * s.outer * B;
        groups += chunks * s.outer * B;
        if (groups * 256 > kMostThreads) return RNNT_ERR_UNSUPPORTED;
    }
    if (args.n == 0) return RNNT_OK;
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, static_cast<hipStream_t>(stream), args); };
    if (!any_within && bytes > kStreamBytes) run(beam_reorder_kernel<0, true>);
    else if (!any_within) run(beam_reorder_kernel<0, false>);
    else if (beams_out <= 8) run(beam_reorder_kernel<8, false>);
    else if (beams_out <= 16) run(beam_reorder_kernel<16, false>);
    else if (beams_out <= 32) run(beam_reorder_kernel<32, false>);
    else run(beam_reorder_kernel<64, false>);
    BEAM_TRY(hipGetLastError());
    return RNNT_OK;
}

}  // extern "C"

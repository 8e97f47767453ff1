// Attention of the new rows of speculation windows over the paged cache (aj_cache_attend).
//
// A window's R rows and the G query heads that share a head of keys and values are R*G query vectors against the same tokens: vector x = r * G + g.
// A workgroup takes up to QB of them and walks over tiles of ST tokens with the running maximum and sum of a softmax; scores and weights
// never leave its registers.
//
// Products.  v_mfma 32x32: scores S^T = K Q^T (A = 32 tokens, B = 32 vectors), so that a lane owns one vector and 16 of 32 tokens: maximum and sum run in
// the lane, with one exchange between the wave's halves.  Then O^T = V^T P^T: the weights are needed as the B operand, where lane (column, half h) holds
// 8 consecutive places of the contraction; which token stands at which place is free as long as V^T agrees, so the weights stay where the scores were
// made (a half's registers 8s .. 8s+7 are tokens 16s + 4h + {0..3} and 16s + 8 + 4h + {0..3}) and V^T's fragments are gathered in that order: bf16 and
// FP8 by the transposing LDS reads (ds_read_b64_tr_b16 / _b8: 16 lanes read 4 or 8 rows and each gets a column), fp32 by plain ones.
// The maximum that weights refer to moves only when a score exceeds it by 2^8 (any reference gives the same quotients): otherwise every
// tile would rescale the whole of O.
//
// Tiles travel global -> LDS by direct 16-byte loads, NST stages; a lane asks for its own token's address, so pages may end anywhere in a tile.
// 16-byte chunks are permuted within a row (f_k, f_v) so that the fragment reads of 8 or 16 rows fall on different banks.
//
// Work.  Lengths are known on the device only.  All (window, head of keys and values) items' tiles form one line, which is cut into equal pieces for
// `clusters` clusters of NB workgroups (one per block of QB vectors; a cluster's workgroups run on one XCD and read the same tokens at the same
// time).  Every workgroup finds its piece by a prefix sum over the windows.  Items cut by a piece's border leave partial results (maximum, sum,
// unscaled O in fp32), which the last workgroup to arrive adds in the order of the pieces, so that the same call gives the same bits.
#pragma once
#include <float.h>
#include <math.h>

#include "cache.h"
#include "lds_pipeline.h"

#define ALWAYS_INLINE __attribute__((always_inline))

namespace aj {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;

// DP: head size, padded; WQ x WK x WD waves: WQ blocks of 32 vectors, WK parts of KT tokens of a tile, WD parts of the head size: those waves make the same
// scores, each for its own part of O.  At DP = 256 all of O for 32 vectors leaves a wave too few registers for its loads' addresses, which then come back
// from memory between the loads: with WD = 2, 21 windows x 1 row x 8 heads over 5000 tokens of 4 heads take 86 us (5.0 TB/s) instead of 215.  Smaller heads gain by more waves to issue loads
template <CacheType TYPE_, int DP_, int WQ_, int WK_, int KT_, int NST_, int PER_CU_, int WD_ = 1>
struct Form {
    static constexpr CacheType TYPE = TYPE_;
    static constexpr int DP = DP_, WQ = WQ_, WK = WK_, WD = WD_, KT = KT_, NST = NST_, PER_CU = PER_CU_;
    static constexpr int KES = TYPE == CACHE_FP8 ? 1 : TYPE == CACHE_F32 ? 4 : 2;
    static constexpr int WAVES = WQ * WK * WD, THREADS = 64 * WAVES, QB = 32 * WQ, ST = WK * KT;
    static constexpr int RB = DP * KES, CPR = RB / 16, RPI = 64 / CPR;        // bytes and chunks of a row, rows of a load instruction
    static constexpr int TILE = ST * RB, STAGE = 2 * TILE;                    // keys, then values
    static constexpr int NI = TILE / 1024 / WAVES;                            // load instructions of a wave for the keys of a tile (values: the same)
    static constexpr int NKB = KT / 32, DB = DP / 32 / WD, QREGS = TYPE == CACHE_F32 ? DP / 8 : DP / 16;
    static constexpr int SEG = 1024;                                          // pages in LDS
    static constexpr bool ZEROS = TYPE == CACHE_BF16 && DP == 256 && WQ > 1;
    static constexpr int MERGE = WK > 1 ? WQ * WK * DP * 32 * 4 : 0;            // bytes to add up the waves' parts
    static constexpr int LDS = NST * STAGE > MERGE ? NST * STAGE : MERGE;
    static_assert(TILE % (1024 * WAVES) == 0 && CPR <= 64 && 2 * NI * (NST - 1) < 64, "whole load instructions, vmcnt");
};

// chunk permutation of a row of keys / values
template <class F>
__device__ __forceinline__ int f_k(int row)
{
    return F::RB >= 256 ? row & 15 : F::RB == 128 ? row >> 1 & 7 : row >> 2 & 3;
}
template <class F>
__device__ __forceinline__ int f_v(int row)
{
    if (F::TYPE == CACHE_F32) return (row >> 2 & 1) << 3;                                      // tokens 4 apart are read together
    // The transposing reads of 32 lanes go together: bf16 64 bytes of 4 rows, FP8 32 bytes of 8 rows, 4 and 4 that are 8 apart.  Rows that begin on the same bank
    // (all of 256 bytes, every second of 128, ..) move by whole pieces, and the other half's rows to the gaps: no
    // conflicts, which were a third of the LDS cycles when rows moved by single pieces (the time is the same within 0.5 %)
    if (F::TYPE == CACHE_FP8) {
        if (F::RB >= 256) return (row & 3) << 1 | (row >> 3 & 1) << 3 | (row >> 2 & 1);
        if (F::RB == 128) return (row >> 1 & 1) << 1 | (row >> 3 & 1) << 2 | (row >> 2 & 1);
        return (row >> 3 & 1) << 1 | (row >> 2 & 1);
    }
    return F::RB >= 256 ? (row & 3) << 2 | (row >> 2 & 1) << 1 : (row >> 1 & 1) << 2 | (row >> 2 & 1) << 1;
}

// (s_nop: the wait state between the write of M0 and a load into LDS)
__device__ __forceinline__ void load_to_lds_16_at(const char *at, uint32_t lds_dst)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(at), "s"(lds_dst) : "memory");
}

__device__ __forceinline__ void load_to_lds_16_at_nt(const char *at, uint32_t lds_dst)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(at), "s"(lds_dst) : "memory");
}

// maximum and sum of the lane's value and that of the lane 32 away (swapping the halves of two copies leaves each half's values in both)
__device__ __forceinline__ float max_halves(float x)
{
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float sum_halves(float x)
{
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// V^T as the A operand of a product over 16 tokens: element d = 32 db + lane % 32 of the tokens 16 ks + 4 h + {0..3} and 16 ks + 8 + 4 h + {0..3}.
// Sixteen lanes give the addresses of 4 (8) rows of 16 elements, in pieces of 8 bytes, and lane i of them gets column i
template <class T>
__device__ __forceinline__ T from_lds(uint32_t at)
{
    return *(const __attribute__((address_space(3))) T *)at;
}

template <class F>
__device__ __forceinline__ uint32_t values_base(int lane)      // of ks = db = 0, from the first row of the wave's values
{
    const int h = lane >> 5, part = lane >> 4 & 1, i = lane & 15;
    if constexpr (F::TYPE == CACHE_BF16) {
        const int row = 4 * h + (i >> 2);
        return row * F::RB + ((2 * part + (i >> 1 & 1)) ^ f_v<F>(row)) * 16 + (i & 1) * 8;
    } else {
        const int j = i >> 1, row = 4 * h + (j & 3) + 8 * (j >> 2);
        return row * F::RB + (part ^ f_v<F>(row)) * 16 + (i & 1) * 8;
    }
}

template <class F>
__device__ __forceinline__ bf16x8 values(uint32_t base, int ks, int db)
{
    // the chunk's number is changed by exclusive or, so that is how 32 db elements are added
    const uint32_t at = (base ^ (32 * db * F::KES)) + 16 * ks * F::RB;
    if constexpr (F::TYPE == CACHE_BF16) {
        typedef __attribute__((address_space(3))) i16x4 *p;
        const i16x4 y0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p)at), y1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p)(at + 8 * F::RB));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        typedef __attribute__((address_space(3))) i32x2 *p;
        const i32x2 y = __builtin_amdgcn_ds_read_tr8_b64_v2i32((p)at);
        return widen(y[0], y[1]);
    }
}

// Partial results go from one workgroup to another that may run on another XCD, behind another L2: stores and loads of the device's scope pass them by,
// so that neither side has to write back or invalidate a cache (fences of that scope do both: 243 us instead of 198 for 64 windows of 17 .. 8192 tokens and 8 heads)
struct Part {
    static constexpr int DEVICE = 16;      // cache policy: sc1
    __amdgpu_buffer_rsrc_t o, ml;

    __device__ __forceinline__ Part(const AttendArgs &a, int64_t unit, int vectors, int size)
        : o(__builtin_amdgcn_make_buffer_rsrc(a.part_o + unit * vectors * size, 0, vectors * size * 4, 0x00020000)),
          ml(__builtin_amdgcn_make_buffer_rsrc(a.part_ml + unit * vectors, 0, vectors * 8, 0x00020000))
    {
    }
    __device__ __forceinline__ void store(int at, f32x4 y) const { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, y), o, at * 16, 0, DEVICE); }
    __device__ __forceinline__ void store(int x, float m, float l) const
    {
        typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(m), __float_as_uint(l)}, ml, x * 8, 0, DEVICE);
    }
    __device__ __forceinline__ f32x4 load(int at) const { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(o, at * 16, 0, DEVICE)); }
    __device__ __forceinline__ float2 load_ml(int x) const
    {
        const auto y = __builtin_amdgcn_raw_buffer_load_b64(ml, x * 8, 0, DEVICE);
        return float2{__uint_as_float(y[0]), __uint_as_float(y[1])};
    }
};

// Keeps what is computed from x where it is written: what is needed once per tile or per item would otherwise be computed ahead of the loops and take
// registers throughout
__device__ __forceinline__ int here(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Values that are the same in all lanes but are computed in vector registers (divisions, fp64).  (The compiler drops a readfirstlane of what it knows to
// be the same in all lanes, and then has no scalar register for an operand that needs one)
__device__ __forceinline__ int uniform(int x)
{
    asm("" : "+v"(x));
    return __builtin_amdgcn_readfirstlane(x);
}

__device__ __forceinline__ const char *uniform(const char *p)
{
    const uint64_t x = (uint64_t)p;
    return (const char *)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// What a window's tokens look like to its rows
struct Span {
    int L, R;         // cached tokens, live rows
    int hi;           // tokens are t < hi
    int lo;           // sinks <= t < lo: seen by no row
    int ns, first, n; // tiles that are visited: 0 .. ns-1, first .. ; n of them in all
};

template <int ST>
__device__ __forceinline__ Span span_of(const AttendArgs &a, int L, int R)
{
    Span s;
    s.L = L;
    s.R = R;
    s.lo = s.ns = s.first = 0;
    const int cap = a.pages.width << a.pages.log_page;
    s.hi = s.L + s.R < cap ? s.L + s.R : cap;
    const int end = (s.hi - 1) / ST + 1;
    s.n = end;
    if (a.window) {
        const int lo = s.L - a.window + 1, sk = a.sinks < s.hi ? a.sinks : s.hi;
        s.lo = lo > 0 ? lo : 0;
        s.ns = (sk + ST - 1) / ST;
        s.first = s.lo / ST > s.ns ? s.lo / ST : s.ns;
        if (s.first > end) s.first = end;
        s.n = s.ns + end - s.first;
        if (s.n == 0) s.n = 1, s.first = 0;      // nothing is seen: the rows' zeros have to be written all the same
    }
    if (s.R == 0) s.n = 0;
    return s;
}

template <int ST>
__device__ __forceinline__ Span span_of(const AttendArgs &a, int b)
{
    return span_of<ST>(a, cached_tokens(a.pages, b), live_rows(a.pages, b));
}

// The line's `total` places are cut into `cuts` pieces that differ by one place at most: the first place of a piece, and the piece of a place.
// (Products are below 2^46 and quotients below 2^15: in fp64 no quotient is rounded to a whole number that it does not reach.)
__device__ __forceinline__ int cut(int piece, int total, int cuts) { return uniform((int)((double)piece * total / cuts)); }
__device__ __forceinline__ int piece_of(int place, int total, int cuts) { return uniform((int)((((double)place + 1.0) * cuts - 1.0) / total)); }

// A workgroup's piece of the line of all items' tiles, and the window where it begins
template <int ST, int THREADS>
struct Line {
    int total, cuts, w, w_end;   // places of the line, pieces, the piece
    int b, start, L, R;          // the window, its first place, its cached tokens and live rows

    // sum of the values of the threads before this one and of all threads
    static __device__ __forceinline__ void scan(int mine, int *sums, int &before, int &all)
    {
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int y = __shfl_up(incl, o);
            if ((int)threadIdx.x % 64 >= o) incl += y;
        }
        if (threadIdx.x % 64 == 63) sums[threadIdx.x / 64] = incl;
        __syncthreads();
        before = incl - mine;
        all = 0;
#pragma unroll
        for (int v = 0; v < THREADS / 64; ++v) {
            if (v < (int)threadIdx.x / 64) before += sums[v];
            all += sums[v];
        }
    }

    __device__ __forceinline__ bool begin(const AttendArgs &a, int cluster, int clusters, int *sums, int *found)
    {
        const int B = a.pages.B, tid = threadIdx.x;
        int mine = 0, before = 0, all = 0, my_L = 0, my_R = 0;      // (what differs between lanes stays out of the members)
        if (B <= THREADS) {      // every thread has a window, and looks it up once
            if (tid < B) {
                my_L = cached_tokens(a.pages, tid);
                my_R = live_rows(a.pages, tid);
                mine = span_of<ST>(a, my_L, my_R).n * a.groups;
            }
        } else {
            for (int i = tid; i < B; i += THREADS) mine += span_of<ST>(a, i).n * a.groups;
        }
        scan(mine, sums, before, all);
        total = uniform(all);
        // A piece of an item of n tiles that is cut into pieces of x tiles takes x tiles' time, and its join n / x parts' time: together least at
        // x = sqrt(n * a part's time / a tile's).  Items of a few tiles stay whole
        const int items = B * a.groups;
        const float n = (float)total / items;
        const int least = uniform((int)(n <= a.whole ? ceilf(n) : sqrtf(n * a.part_cost))), most = uniform(total / (least < 1 ? 1 : least));
        cuts = most < 1 ? 1 : most < clusters ? most : clusters;
        // As many pieces to every item of a batch of equal ones, where that makes the pieces longer by less than a second item's start and join take, about four
        // tiles: 44 x 38 rows x 4 heads over 1000 tokens 45 -> 33 us.  (One tile: 100 x 38 rows over 700 44 instead of 39.5; sixteen: 33 x 1 row x 32 heads over 700 33 instead of
        // 29.5)
        const int even = cuts > items ? cuts - cuts % items : cuts;
        if (uniform((int)((float)total * (cuts - even) <= 4.f * even * cuts))) cuts = even;
        if (cluster >= cuts) return false;
        w = cut(cluster, total, cuts);
        w_end = cut(cluster + 1, total, cuts);
        if (w >= w_end) return false;
        if (B <= THREADS) {
            if (w >= before && w < before + mine) found[0] = tid, found[1] = before, found[2] = my_L, found[3] = my_R;
            __syncthreads();
        } else {
            for (int base = 0, carry = 0;; base += THREADS, carry += all) {      // (w is somewhere)
                const int i = base + tid;
                my_L = i < B ? cached_tokens(a.pages, i) : 0;
                my_R = i < B ? live_rows(a.pages, i) : 0;
                mine = span_of<ST>(a, my_L, my_R).n * a.groups;
                __syncthreads();
                scan(mine, sums, before, all);
                before += carry;
                if (w >= before && w < before + mine) found[0] = i, found[1] = before, found[2] = my_L, found[3] = my_R;
                if (w < carry + all) break;
            }
            __syncthreads();
        }
        b = uniform(found[0]);
        start = uniform(found[1]);
        L = uniform(found[2]);
        R = uniform(found[3]);
        return true;
    }
};

// four consecutive elements of a row of values
template <class F>
__device__ __forceinline__ f32x4 four(const char *at)
{
    if constexpr (F::TYPE == CACHE_F32) return *(const f32x4 *)at;
    else if constexpr (F::TYPE == CACHE_BF16) {
        const bf16x4 y = *(const bf16x4 *)at;
        return f32x4{(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
    } else {
        const bf16x8 y = widen(*(const uint32_t *)at, 0);
        return f32x4{(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
    }
}

// row of vector x: x / G.  (x < 2^20 and G <= 1024: x + 1/2 is further from the next multiple of G than the two roundings can carry it)
__device__ __forceinline__ int row_of(const AttendArgs &a, int x) { return (int)(((float)x + 0.5f) * a.inv_G); }
// ... and its number among all rows' query heads
__device__ __forceinline__ int64_t vector_of(const AttendArgs &a, int b, int kvh, int x)
{
    const int r = row_of(a, x);
    return ((int64_t)b * a.pages.rows + r) * a.n_q + kvh * a.G + x - r * a.G;
}

__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// out and lse of one vector from its unscaled sums
template <CacheType TYPE>
__device__ __forceinline__ void finish(const AttendArgs &a, int64_t vec, int d4, f32x4 o, float l)
{
    if (4 * d4 >= a.D) return;
    const float f = a.v_scale / l;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = l == 0.f ? 0.f : o[i] * f;      // (a sum of zeros times values that are not finite is no number)
    if constexpr (TYPE == CACHE_F32) {
        *(f32x4 *)((float *)a.out + vec * a.D + 4 * d4) = o;
    } else {
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (__bf16)o[i];
        *(bf16x4 *)((__bf16 *)a.out + vec * a.D + 4 * d4) = y;
    }
}

__device__ __forceinline__ void finish_lse(const AttendArgs &a, int64_t vec, float m, float l)
{
    // m: the reference of the weights as a power of two
    if (a.lse) a.lse[vec] = l > 0.f || l != l ? (m + __builtin_amdgcn_logf(l)) * 0.69314718f : -INFINITY;
}

// Parts of one vector, pieces d0, d0 + step, .. of them.  These are round trips to memory, and count by the number of loads in flight: PARTS x PIECES
template <class F, int PARTS, int PIECES, class P>
__device__ __forceinline__ void join(const AttendArgs &a, const P &part, int c0, int c1, int xl, int64_t vec, int d0, int step)
{
    float m = -INFINITY, l = 0.f;
    f32x4 o[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) o[p] = f32x4{0, 0, 0, 0};
    for (int cl = c0; cl <= c1; cl += PARTS) {
        float2 ml[PARTS];
        f32x4 y[PARTS][PIECES];
#pragma unroll
        for (int j = 0; j < PARTS; ++j) {
            const Part one = part(cl + j < c1 ? cl + j : c1);      // (the last part once more, which is then left out)
            ml[j] = one.load_ml(xl);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) y[j][p] = one.load((d0 + p * step < F::DP / 4 ? d0 + p * step : 0) * F::QB + xl);
        }
        float top = m;
#pragma unroll
        for (int j = 0; j < PARTS; ++j)
            top = fmaxf(top, ml[j].x);
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= keep;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) o[p] *= keep;
#pragma unroll
        for (int j = 0; j < PARTS; ++j) {
            const float f = ml[j].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[j].x - m);
            if (cl + j <= c1) {      // (no product with zero: the part may be infinite)
                l += ml[j].y * f;
#pragma unroll
                for (int p = 0; p < PIECES; ++p) o[p] += y[j][p] * f;
            }
        }
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
        if (d0 + p * step < a.D / 4) finish<F::TYPE>(a, vec, d0 + p * step, o[p], l);
    if (d0 == 0) finish_lse(a, vec, m, l);
}

// Pages of a segment of an item's tiles, in LDS: byte offsets into a pool (page 0's for a page that is nowhere) and whether they are somewhere
template <class F>
struct Segment {
    int64_t at[F::SEG];
    uint8_t gone[F::SEG];
};

// PADDED: the head size is below DP.  What the loads put behind a key are copies of its first elements, which must not count: an infinity among them times the
// query's zero is no number.  Steps of the scores that lie there are left out, or (ZEROS) take zeros for the keys: 32 windows x 1 row over 4000 tokens in fp32, heads of
// 208: 690 us, with all steps 756; 16 windows x 64 rows over 1000 tokens in bf16, heads of 240: 72 us with zeros, 76 with steps left out, whose branches make that
// form spill.  (FP8 has no infinities, and its heads may end inside a step)
template <class F, bool PADDED>
__global__ __launch_bounds__(F::THREADS, F::PER_CU *F::WAVES / 4 < 1 ? 1 : F::PER_CU *F::WAVES / 4) void attend_kernel(AttendArgs a)
{
    constexpr int ST = F::ST, RB = F::RB, KT = F::KT, DB = F::DB, NKB = F::NKB, NI = F::NI, QB = F::QB, NST = F::NST;
    constexpr bool F32 = F::TYPE == CACHE_F32;
    __shared__ __attribute__((aligned(1024))) char lds[F::LDS];
    __shared__ Segment<F> pages;
    __shared__ int sums[F::WAVES], found[4];
    __shared__ int wflag[2][F::WAVES];
    __shared__ float mls[2][F::WK][QB];
    __shared__ u32x4 zero;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, col = lane & 31;
    const int wq = wave % F::WQ, wk = wave / F::WQ % F::WK, wd = wave / (F::WQ * F::WK), db0 = wd * DB;      // db0: the wave's first 32 elements of O
    const int G = a.G, words = (a.pages.rows + 31) / 32;
    const int cap = a.pages.width << a.pages.log_page, page = 1 << a.pages.log_page;

    // this workgroup's piece of the line of tiles; its block of vectors
    const int xcd = blockIdx.x & 7, place = blockIdx.x >> 3, per_xcd = a.clusters / 8;
    const int members = a.heads * a.blocks, cluster = uniform(xcd * per_xcd + place / members), member = uniform(place % members);
    const int block = uniform(member % a.blocks), head_of_group = uniform(member / a.blocks);
    if (PADDED && F::ZEROS && tid == 0) zero = u32x4{0, 0, 0, 0};      // (there are barriers before it is read)
    Line<ST, F::THREADS> line;
    if (!line.begin(a, cluster, a.clusters, sums, found)) return;
    const int total = line.total, cuts = line.cuts, w_end = line.w_end;
    int w = line.w, b = line.b, start = line.start;
    Span sp = span_of<ST>(a, line.L, line.R);

    const uint32_t lds0 = lds_offset_of(lds);
    const float c = a.score_scale, threshold = __int_as_float(uniform(__float_as_int(fminf(8.f / c, FLT_MAX))));      // (infinite, nothing would exceed -infinity by it)
    const int per_tile = page < ST ? ST >> a.pages.log_page : 1, seg_tiles = F::SEG / per_tile;
    const bool once = a.blocks == 1;
    const uint32_t slot_stride = (uint32_t)a.pages.slot_stride;
    // what a lane asks for in the n-th load instruction of a tile, behind the address of its page
    uint32_t k_off[NI], v_off[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int row = (wave * NI + n) * F::RPI + lane / F::CPR, pc = lane % F::CPR;
        int ck = pc ^ f_k<F>(row), cv = pc ^ f_v<F>(row);
        if (ck * 16 >= a.D * F::KES) ck = 0;      // padding: the scores leave it out, and what comes of the values is not written
        if (cv * 16 >= a.D * F::KES) cv = 0;
        k_off[n] = (uint32_t)(row & (page - 1)) * slot_stride + ck * 16;
        v_off[n] = (uint32_t)(row & (page - 1)) * slot_stride + cv * 16;
    }

    while (w < w_end) {
        while (w >= start + sp.n * a.groups) {      // (windows without rows have no places)
            start += sp.n * a.groups;
            ++b;
            sp = span_of<ST>(a, b);
        }
        const int group = uniform((w - start) / sp.n), kvh = group * a.heads + head_of_group, i_first = w - start - group * sp.n;
        const int i_last = sp.n - i_first < w_end - w ? sp.n : i_first + (w_end - w);     // end of the visits
        const int item = start + group * sp.n;                                            // first place of the item
        const bool whole = i_first == 0 && i_last == sp.n;
        w += i_last - i_first;
        const int nvec = sp.R * G;
        if (block * QB >= nvec) continue;
        const int x_last = (block + 1) * QB < nvec ? (block + 1) * QB - 1 : nvec - 1;
        const int r_first = uniform(row_of(a, block * QB)), r_last = uniform(row_of(a, x_last));

        // the visits that this block needs: not those behind its last row, nor those before its first row's window; among them, from i_full to i_part, the
        // tiles of which every row of the block sees everything
        int i_begin = i_first, i_end = i_last, i_full, i_part;
        {
            const int hi = sp.L + r_last + 1 < cap ? sp.L + r_last + 1 : cap;
            const int tile = (hi - 1) / ST, last = tile >= sp.first ? sp.ns + tile - sp.first : tile < sp.ns ? tile : sp.ns - 1;
            if (i_end > last + 1) i_end = last + 1 > i_begin ? last + 1 : i_begin;
            i_full = i_begin;
            if (a.window) {
                const int lo = sp.L + r_first - a.window + 1, i = sp.ns + lo / ST - sp.first;
                if (!a.pages.depth && i_begin >= sp.ns && lo > 0 && i > i_begin) i_begin = i < i_end ? i : i_end;
                const int near = sp.L + r_last - a.window + 1, f = near > 0 ? sp.ns + (near + ST - 1) / ST - sp.first : 0;
                i_full = i_begin > sp.ns ? i_begin : sp.ns;
                i_full = f > i_full ? f : i_full;
            }
            const int seen = a.mask || a.pages.depth ? sp.L : sp.L + r_first + 1, until = sp.ns + (seen < sp.hi ? seen : sp.hi) / ST - sp.first;
            i_full = i_full < i_end ? i_full : i_end;
            i_part = until < i_end ? until : i_end;
            i_part = i_part > i_full ? i_part : i_full;
        }

        // queries as the B operand: column = vector
        const int x = block * QB + wq * 32 + col, xc = x < nvec ? x : nvec - 1, r = row_of(a, xc), head = kvh * G + xc - r * G;
        const bool active = block * QB + wq * 32 < nvec;
        const int64_t vec = ((int64_t)b * a.pages.rows + r) * a.n_q + head;
        u32x4 q[F::QREGS];
        {
            const char *row = (const char *)a.q + (((int64_t)b * a.pages.rows + r) * a.q_stride + head * a.D) * (F32 ? 4 : 2);
            const int h = here(lane) >> 5;
#pragma unroll
            for (int s = 0; s < F::QREGS; ++s) {
                const int d = F32 ? 4 * (2 * s + h) : F::TYPE == CACHE_FP8 ? 16 * (2 * (s / 2) + h) + 8 * (s & 1) : 16 * s + 8 * h;
                q[s] = d < a.D ? *(const u32x4 *)(row + d * (F32 ? 4 : 2)) : u32x4{0, 0, 0, 0};
            }
        }
        int my_depth = depth_of(a.pages, b, r);
        f32x16 acc[DB];
#pragma unroll
        for (int i = 0; i < DB; ++i) acc[i] = f32x16{0};
        float m = -INFINITY, l = 0.f, over = 0.f;      // over: what l holds too much

        const char *k_head = uniform((const char *)a.k_pool + kvh * a.pages.head_stride), *v_head = uniform((const char *)a.v_pool + kvh * a.pages.head_stride);
        const auto tile_of_visit = [&](int i) ALWAYS_INLINE { return i < sp.ns ? i : sp.first + i - sp.ns; };

        for (int seg = i_begin; seg < i_end; seg += seg_tiles) {
            const int seg_end = seg + seg_tiles < i_end ? seg + seg_tiles : i_end;
            __syncthreads();
            int bad = 0;
            for (int e = tid; e < (seg_end - seg) * per_tile; e += F::THREADS) {
                const int t = tile_of_visit(seg + e / per_tile) * ST + (e % per_tile << a.pages.log_page);   // (its first token, or one on its page)
                int p = -1;
                if (t < cap) {
                    p = a.pages.table[(int64_t)b * a.pages.width + (t >> a.pages.log_page)];
                    if ((uint32_t)p >= (uint32_t)a.pages.n_pages) p = -1;
                }
                pages.at[e] = p < 0 ? 0 : p * a.pages.page_stride;
                pages.gone[e] = p < 0;
                const int until = page < ST ? t + page : t + ST;
                if (p < 0 && t < sp.hi && !(t >= a.sinks && until <= sp.lo)) bad = 1;
            }
            bad = __any(bad);
            if (lane == 0) wflag[1][wave] = bad;
            // what was loaded so far has to be there before the tiles' loads begin: a wait for it later would wait for them too
#pragma unroll
            for (int s = 0; s < F::QREGS; ++s) asm volatile("" : "+v"(q[s]));
            asm volatile("" : "+v"(my_depth));
            __syncthreads();
            bad = 0;
#pragma unroll
            for (int v = 0; v < F::WAVES; ++v) bad |= wflag[1][v];
            bad = uniform(bad);

            const auto page_of = [&](int i, int row) ALWAYS_INLINE { return (i - seg) * per_tile + (page < ST ? row >> a.pages.log_page : 0); };
            // Loads of tile i.  (A token that is nowhere reads a slot of page 0, and one behind the last the slot where it would be.)
            const auto issue = [&](int i, int stage) ALWAYS_INLINE {
                const int t0 = tile_of_visit(i) * ST;
                const uint32_t dst = (uint32_t)uniform(lds0 + stage * F::STAGE + wave * NI * 1024);
                if (page >= F::RPI) {
                    // the rows of a load instruction lie on one page, whose address is the same for all lanes: lane n looks up that of the n-th instruction
                    const int64_t mine = pages.at[page_of(i, (wave * NI + (lane < NI ? lane : 0)) * F::RPI)] +
                                         (page > ST ? (uint64_t)(uint32_t)(t0 & (page - 1)) * slot_stride : 0);
                    const int lo = (int)mine, hi = (int)(mine >> 32);
#pragma unroll
                    for (int n = 0; n < NI; ++n) {
                        const int64_t at = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, n) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, n));
                        if (once) {
                            lds_dma_16_nt(k_head + at, k_off[n], dst + n * 1024);
                            lds_dma_16_nt(v_head + at, v_off[n], dst + n * 1024 + F::TILE);
                        } else {
                            lds_dma_16(k_head + at, k_off[n], dst + n * 1024);
                            lds_dma_16(v_head + at, v_off[n], dst + n * 1024 + F::TILE);
                        }
                    }
                } else {
                    const int row0 = wave * NI * F::RPI + here(lane) / F::CPR;
                    constexpr int BATCH = NI < 4 ? NI : 4;
#pragma unroll
                    for (int n0 = 0; n0 < NI; n0 += BATCH) {
                        int64_t at[BATCH];
#pragma unroll
                        for (int n = 0; n < BATCH; ++n) at[n] = pages.at[page_of(i, row0 + (n0 + n) * F::RPI)];
#pragma unroll
                        for (int n = 0; n < BATCH; ++n) {
                            const char *k = k_head + (at[n] + (uint32_t)here(k_off[n0 + n])), *v = v_head + (at[n] + (uint32_t)here(v_off[n0 + n]));
                            if (once) {
                                load_to_lds_16_at_nt(k, dst + (n0 + n) * 1024);
                                load_to_lds_16_at_nt(v, dst + (n0 + n) * 1024 + F::TILE);
                            } else {
                                load_to_lds_16_at(k, dst + (n0 + n) * 1024);
                                load_to_lds_16_at(v, dst + (n0 + n) * 1024 + F::TILE);
                            }
                        }
                    }
                }
            };

            // scores of the wave's tokens
            f32x16 s[NKB];
            const auto score = [&](uint32_t kt) ALWAYS_INLINE {
                const uint32_t base = kt + here(col * RB + (h ^ f_k<F>(col)) * 16);
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb) s[kb] = f32x16{0};
                // fragments are asked for two steps ahead; the barriers keep the compiler from asking for all of them at once, which
                // would take more registers than there are
                constexpr int KS = RB / 32, AHEAD = 2;
                u32x4 y[AHEAD + 1][NKB];
                // whether step ks lies behind the head (which is longer than half of DP, or the smaller form has it, and comes in steps of 16 elements)
                const auto behind = [&](int ks) ALWAYS_INLINE {
                    return PADDED && (F::DP == 64 || 2 * ks >= KS) && 32 * ks % (16 * F::KES) == 0 && 32 * ks >= a.D * F::KES;
                };
                const auto ask = [&](int ks) ALWAYS_INLINE {
#pragma unroll
                    for (int kb = 0; kb < NKB; ++kb) {
                        const uint32_t at = (base ^ (32 * ks)) + kb * 32 * RB;
                        y[ks % (AHEAD + 1)][kb] = from_lds<u32x4>(F::ZEROS && behind(ks) ? lds_offset_of(&zero) : at);
                    }
                };
#pragma unroll
                for (int ks = 0; ks < AHEAD && ks < KS; ++ks) ask(ks);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if (!F::ZEROS && behind(ks)) break;
                    if (ks + AHEAD < KS) ask(ks + AHEAD);
#pragma unroll
                    for (int kb = 0; kb < NKB; ++kb) {
                        const u32x4 z = y[ks % (AHEAD + 1)][kb];
                        if constexpr (F32) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(z[e]), __uint_as_float(q[ks][e]), s[kb], 0, 0, 0);
                        } else if constexpr (F::TYPE == CACHE_BF16) {
                            s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, z), __builtin_bit_cast(bf16x8, q[ks]), s[kb], 0, 0, 0);
                        } else {
                            s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(z[0], z[1]), __builtin_bit_cast(bf16x8, q[2 * ks]), s[kb], 0, 0, 0);
                            s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(z[2], z[3]), __builtin_bit_cast(bf16x8, q[2 * ks + 1]), s[kb], 0, 0, 0);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            // scores to weights
            const auto weigh = [&]() ALWAYS_INLINE {
                float mx = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
                mx = max_halves(mx);
                if (__any(mx > m + threshold)) {
                    const float mn = fmaxf(m, mx), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * c);
#pragma unroll
                    for (int i = 0; i < DB; ++i)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[i][e] *= f;
                    l *= f;
                    if (F32) over *= f;
                    m = mn;
                }
                const float base = m == -INFINITY ? 0.f : m * c;
                float sum = 0.f;
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        s[kb][e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], c, -base));
                        sum += s[kb][e];
                    }
                }
                // Additions of nearly equal terms to a long sum round the same way until its exponent changes: over 131072 tokens of weight 0.7 or 0.9, one after another, sums
                // are 6 10^-4 off.  So a tile's weights are added up by themselves; and in fp32 what adding them to l rounds away goes into the next addition: 10^-6.  (Results of
                // 16 bits need no more than the former, some 10^-5, and the latter takes up to 6 % there, heads of 256 and 64 rows)
                if constexpr (F32) {
                    const float more = sum - over, to = l + more;
                    over = to - l - more;
                    l = to;
                } else {
                    l += sum;
                }
            };
            // O^T += V^T P^T
            const auto add = [&](uint32_t vt) ALWAYS_INLINE {
                if constexpr (F32) {
                    const uint32_t base = (vt + here(4 * h * RB + ((col >> 2) ^ (h << 3)) * 16 + (col & 3) * 4)) ^ (128 * db0);
                    // DG blocks of 32 elements at a time.  A tile's products are added up by themselves too, since one takes two tokens: 4 10^-5 for a value that all those
                    // tokens share, 10^-3 otherwise (in the other types one takes 16, and the result is rounded to 2^-8)
                    constexpr int DG = F::WQ > 1 && DB > 2 ? 2 : DB;
#pragma unroll
                    for (int d0 = 0; d0 < DB; d0 += DG) {
                        f32x16 o[DG];
#pragma unroll
                        for (int j = 0; j < DG; ++j) o[j] = f32x16{0};
#pragma unroll
                        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                            for (int e = 0; e < 16; ++e)
#pragma unroll
                                for (int j = 0; j < DG; ++j) {
                                    const float y = from_lds<float>((base ^ (128 * (d0 + j))) + (kb * 32 + e % 4 + 8 * (e / 4)) * RB);
                                    o[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(y, s[kb][e], o[j], 0, 0, 0);
                                }
#pragma unroll
                        for (int j = 0; j < DG; ++j)
#pragma unroll
                            for (int e = 0; e < 16; ++e) acc[d0 + j][e] += o[j][e];
                    }
                } else {
                    // DG blocks of 32 elements at a time: their fragments are asked for while the products before them run
                    constexpr int KS = KT / 16, DG = DB < 4 ? DB : 4, STEPS = KS * DB / DG;
                    const uint32_t base = (vt + values_base<F>(here(lane))) ^ (32 * db0 * F::KES);
                    bf16x8 y[2][DG], p;
                    const auto ask = [&](int n) ALWAYS_INLINE {
#pragma unroll
                        for (int j = 0; j < DG; ++j) y[n & 1][j] = values<F>(base, n / (DB / DG), n % (DB / DG) * DG + j);
                    };
                    ask(0);
#pragma unroll
                    for (int n = 0; n < STEPS; ++n) {
                        const int ks = n / (DB / DG), d0 = n % (DB / DG) * DG;
                        if (d0 == 0) {
                            // weights lose at most half a step of bf16, 2^-8 of each: as the products' operand they have to
#pragma unroll
                            for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[ks / 2][8 * (ks & 1) + e];
                        }
                        if (n + 1 < STEPS) ask(n + 1);
#pragma unroll
                        for (int j = 0; j < DG; ++j) acc[d0 + j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[n & 1][j], p, acc[d0 + j], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };

            // first the tiles that are seen whole, then the others: their loads form one sequence
            int f0 = i_full > seg ? i_full : seg, f1 = i_part < seg_end ? i_part : seg_end;
            if (f0 > seg_end) f0 = seg_end;
            if (f1 < f0 || bad) f1 = f0;
            const int nf = f1 - f0, n_all = seg_end - seg;
            const auto visit = [&](int n) ALWAYS_INLINE { return n < nf ? f0 + n : n - nf < f0 - seg ? seg + n - nf : n - nf + seg + nf; };
#pragma unroll
            for (int n = 0; n < NST - 1; ++n)
                if (n < n_all) issue(visit(n), n);
            int stage = 0;
            const auto next = [&](int n) ALWAYS_INLINE {
                // tile n has landed, for every wave, and nobody reads the stage before it any more
                if (NST > 3 && n + 2 < n_all) wait_vm_lgkm_and_barrier<(NST > 3 ? 4 * NI : 0)>();
                else if (NST > 2 && n + 1 < n_all) wait_vm_lgkm_and_barrier<(NST > 2 ? 2 * NI : 0)>();
                else wait_vm_lgkm_and_barrier<0>();
                if (n + NST - 1 < n_all) issue(visit(n + NST - 1), stage == 0 ? NST - 1 : stage - 1);
            };
            for (int n = 0; n < nf; ++n) {
                next(n);
                if (active) {
                    const uint32_t tile = lds0 + stage * F::STAGE + wk * KT * RB;
                    // a wave that has products to issue goes before one that weighs: the matrix pipe works while the other wave of the SIMD is at its
                    // exponentials (128 windows x 64 rows x 64 heads over 2048 tokens: 762 -> 707 us)
                    __builtin_amdgcn_s_setprio(1);
                    score(tile);
                    __builtin_amdgcn_s_setprio(0);
                    weigh();
                    __builtin_amdgcn_s_setprio(1);
                    add(tile + F::TILE);
                    __builtin_amdgcn_s_setprio(0);
                }
                stage = stage + 1 == NST ? 0 : stage + 1;
            }

            for (int n = nf; n < n_all; ++n) {
                next(n);
                const int i = visit(n), t_tile = tile_of_visit(i) * ST;
                char *tile = lds + stage * F::STAGE;
                stage = stage + 1 == NST ? 0 : stage + 1;
                // values of tokens that nobody sees count as zero whatever they are; and look for values that are not finite
                int odd = 0;
                for (int e = here(tid); e < ST * F::CPR; e += F::THREADS) {
                    const int row = e / F::CPR, t = t_tile + row;
                    const bool dead = t >= sp.hi || (a.window && t >= a.sinks && t < sp.lo) || pages.gone[page_of(i, row)];
                    u32x4 *at = (u32x4 *)(tile + F::TILE + e * 16);
                    if (dead) *at = u32x4{0, 0, 0, 0};
                    else if (sp.R > 1 || a.mask) {      // (a lone row sees what is not dead, unless its mask says otherwise)
                        const u32x4 y = *at;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if constexpr (F32) odd |= (y[j] & 0x7f800000u) == 0x7f800000u;
                            else if constexpr (F::TYPE == CACHE_BF16) odd |= (y[j] & 0x7f80u) == 0x7f80u || (y[j] & 0x7f800000u) == 0x7f800000u;
                            else odd |= (((y[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
                        }
                    }
                }
                odd = __any(odd);
                if (lane == 0) wflag[0][wave] = odd;
                __syncthreads();
                odd = 0;
#pragma unroll
                for (int v = 0; v < F::WAVES; ++v) odd |= wflag[0][v];
                if (!active) continue;

                const char *vt = tile + F::TILE + wk * KT * RB;
                score(lds_offset_of(tile) + wk * KT * RB);
                uint32_t vis[NKB];      // bit e: the lane's row sees token e of the 32
                const int xm = block * QB + wq * 32 + (here(lane) & 31), r = row_of(a, xm < nvec ? xm : nvec - 1);
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb) {
                    const int t = t_tile + wk * KT + 32 * kb;
                    uint32_t y = below(sp.hi - t) & below(sp.L + r + 1 - t);
                    const uint32_t old = below(sp.L - t);
                    if (a.mask && old != ~0u) {
                        const uint32_t *mw = a.mask + ((int64_t)b * a.pages.rows + r) * words;
                        const int at = t - sp.L, wd = at >> 5, sh = at & 31;      // (at > -32)
                        const uint32_t m0 = wd >= 0 && wd < words ? mw[wd] : 0u, m1 = wd + 1 < words ? mw[wd + 1] : 0u;
                        y &= old | (sh ? m0 >> sh | m1 << (32 - sh) : m0);
                    }
                    if (a.window) {
                        const uint32_t sunk = below(a.sinks - t), near = ~below(sp.L + my_depth - a.window + 1 - t);
                        if (!a.pages.depth) {
                            y &= sunk | near;
                        } else {
                            y &= ~old | sunk | near;
                            if (my_depth >= a.window)      // new rows further away than the window
                                for (uint32_t left = y & ~old; left; left &= left - 1) {
                                    const int e = __ffs(left) - 1, d = depth_of(a.pages, b, t + e - sp.L);
                                    if (my_depth - d >= a.window && sp.L + d >= a.sinks) y &= ~(1u << e);
                                }
                        }
                    }
                    if (bad)
                        for (int e = 0; e < 32; ++e)
                            if (pages.gone[page_of(i, wk * KT + kb * 32 + e)]) y &= ~(1u << e);
                    vis[kb] = y;
                    y >>= 4 * (here(lane) >> 5);
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[kb][e] = y >> (e % 4 + 8 * (e / 4)) & 1 ? s[kb][e] : -INFINITY;
                }
                weigh();
                if (!odd) {
                    add(lds_offset_of(vt));
                    continue;
                }
                // some values are not finite: a token at a time, and only for the vectors that see it
                for (int e = 0; e < KT; ++e) {
                    const int h = here(lane) >> 5, from = e % 32 % 4 + 4 * (e % 32 / 8);      // the register and (below) the half that have its weight
                    float p = 0.f;
                    uint32_t seen = 0;
#pragma unroll
                    for (int kb = 0; kb < NKB; ++kb) {
                        if (kb == e / 32) seen = vis[kb] >> (e % 32) & 1;
#pragma unroll
                        for (int j = 0; j < 16; ++j) p = kb == e / 32 && j == from ? s[kb][j] : p;
                    }
                    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(p), __float_as_uint(p), false, false);
                    p = __uint_as_float(e >> 2 & 1 ? both[1] : both[0]);
                    const char *row = vt + e * RB;
                    const int f = f_v<F>(wk * KT + e);
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const int at = (32 * (db0 + db) + 8 * g + 4 * h) * F::KES;
                            const f32x4 y = four<F>(row + ((at / 16) ^ f) * 16 + at % 16);
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[db][4 * g + j] = seen ? fmaf(p, y[j], acc[db][4 * g + j]) : acc[db][4 * g + j];
                        }
                }
            }
        }

        // the halves' sums; the waves that shared the block's tokens
        l = sum_halves(l);
        // (of a cluster's items, the first may have begun in an earlier one and the last may end in a later one)
        const int c0 = piece_of(item, total, cuts), c1 = piece_of(item + sp.n - 1, total, cuts), later = item > cut(c0, total, cuts);
        const auto unit = [&](int cl) ALWAYS_INLINE { return ((int64_t)cl * 2 + (cl == c0 ? later : 0)) * members + member; };
        const Part mine_part(a, unit(cluster), QB, F::DP);
        if constexpr (F::WK == 1) {
            const int col = here(lane) & 31, h = here(lane) >> 5;
            if (x < nvec) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x4 o = {acc[db][4 * e], acc[db][4 * e + 1], acc[db][4 * e + 2], acc[db][4 * e + 3]};
                        const int d4 = 8 * (db0 + db) + 2 * e + h;
                        if (whole) finish<F::TYPE>(a, vec, d4, o, l);
                        else mine_part.store(d4 * QB + wq * 32 + col, o);
                    }
                if (h == 0 && wd == 0) {
                    if (whole) finish_lse(a, vec, m * c, l);
                    else mine_part.store(wq * 32 + col, m * c, l);
                }
            }
        } else {
            __syncthreads();      // the stages are free
            if (h == 0 && wd == 0) mls[0][wk][wq * 32 + col] = m, mls[1][wk][wq * 32 + col] = l;
            __syncthreads();
            float top = -INFINITY;
#pragma unroll
            for (int v = 0; v < F::WK; ++v) top = fmaxf(top, mls[0][v][wq * 32 + col]);
            const float mine = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * c);
            float *merge = (float *)lds + ((wk * (F::DP / 4) + 8 * db0 + (here(lane) >> 5)) * QB + wq * 32 + (here(lane) & 31)) * 4;      // [WK][DP/4][QB][4]
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *(f32x4 *)(merge + (8 * db + 2 * e) * QB * 4) =
                        f32x4{acc[db][4 * e] * mine, acc[db][4 * e + 1] * mine, acc[db][4 * e + 2] * mine, acc[db][4 * e + 3] * mine};
            __syncthreads();
            // (as many vectors as there are, rounded up to a power of two)
            const int nv = x_last + 1 - block * QB, log_nv = nv > 1 ? 32 - __builtin_clz(nv - 1) : 0;
            for (int e = here(tid); e < (a.D / 4) << log_nv; e += F::THREADS) {
                const int d4 = e >> log_nv, xl = e & ((1 << log_nv) - 1), xx = block * QB + xl;
                if (xl >= nv) continue;
                float tm = -INFINITY, tl = 0.f;
#pragma unroll
                for (int v = 0; v < F::WK; ++v) tm = fmaxf(tm, mls[0][v][xl]);
                f32x4 o = {0, 0, 0, 0};
#pragma unroll
                for (int v = 0; v < F::WK; ++v) {
                    const float mv = mls[0][v][xl];
                    tl += mls[1][v][xl] * (mv == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mv - tm) * c));
                    o += *(const f32x4 *)((float *)lds + ((v * (F::DP / 4) + d4) * QB + xl) * 4);
                }
                const int64_t vx = vector_of(a, b, kvh, xx);
                if (whole) finish<F::TYPE>(a, vx, d4, o, tl);
                else mine_part.store(d4 * QB + xl, o);
                if (d4 == 0) {
                    if (whole) finish_lse(a, vx, tm * c, tl);
                    else mine_part.store(xl, tm * c, tl);
                }
            }
            // (the barrier before the next item's page numbers keeps its loads out of `merge`)
        }
        if (whole) continue;

        // The workgroup that is the last of the item's to arrive adds the parts, in the order of the clusters whoever it is, and leaves the
        // count at zero for the next call.  The border behind cluster c cuts one item at most
        int *arrived = a.arrived + c0 * members + member;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the part is there
        __syncthreads();
        if (tid == 0) sums[0] = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (uniform(sums[0]) != c1 - c0) continue;      // (`sums` is next written behind another barrier)
        if (tid == 0) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // a thread adds for one vector, as many pieces of 4 elements as it has to
        const int nv = x_last + 1 - block * QB, log_nv = nv > 1 ? 32 - __builtin_clz(nv - 1) : 0;
        const int xl = here(tid) & ((1 << log_nv) - 1), first = here(tid) >> log_nv, step = F::THREADS >> log_nv;
        if (xl >= nv) continue;
        const int xx = block * QB + xl;
        const int64_t vx = vector_of(a, b, kvh, xx);
        const auto part = [&](int cl) ALWAYS_INLINE { return Part(a, unit(cl), QB, F::DP); };
        if (step >= a.D / 4) {
            if (first < a.D / 4) join<F, 8, 1>(a, part, c0, c1, xl, vx, first, step);
        } else if (c1 - c0 < 2) {
            for (int d0 = first; d0 < a.D / 4; d0 += 8 * step) join<F, 2, 8>(a, part, c0, c1, xl, vx, d0, step);
        } else {
            for (int d0 = first; d0 < a.D / 4; d0 += 8 * step) join<F, 4, 8>(a, part, c0, c1, xl, vx, d0, step);
        }
    }
}

template <class F>
hipError_t launch_attend(const AttendArgs &a, hipStream_t s)
{
    constexpr bool CAN_PAD = F::TYPE != CACHE_FP8;
    if (CAN_PAD && a.D < F::DP) attend_kernel<F, CAN_PAD><<<a.clusters * a.heads * a.blocks, F::THREADS, 0, s>>>(a);
    else attend_kernel<F, false><<<a.clusters * a.heads * a.blocks, F::THREADS, 0, s>>>(a);
    return hipGetLastError();
}

template <class F>
AttendPlan plan_attend(int vectors, int n_kv, int num_cus)
{
    AttendPlan p;
    p.blocks = (vectors + F::QB - 1) / F::QB;
    const int places = num_cus / 8 * F::PER_CU;      // of an XCD
    // as many heads of a window as leave a tenth of the places unused at most: 128 windows x 65 rows x 64 heads over 1000 tokens take 480 us, one head at a time 486, with up to
    // half of the places unused 655; one row at a time within 1.5 % either way
    p.heads = 1;
    for (int h = 2; h <= n_kv; ++h)
        if (n_kv % h == 0 && places / (h * p.blocks) * h * p.blocks * 10 >= places * 9) p.heads = h;
    const int per_xcd = places / (p.heads * p.blocks);
    p.clusters = 8 * (per_xcd < 1 ? 1 : per_xcd);
    p.parts = (size_t)p.clusters * 2 * p.heads * p.blocks * F::QB;
    p.part_size = F::DP;
    return p;
}

}  // namespace aj

// The paged cache around its attention: new rows in (aj_cache_append), masks of draft trees (aj_tree_mask), the accepted path kept
// (aj_cache_commit).  All three move bytes: few launches, 16 bytes per lane, many loads in flight.
#include "cache.h"

namespace aj {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// ---- new rows ------------------------------------------------------------------------------------------------------------
// A head is D/8 lanes of 8 elements (LG of them, a power of two, so that sums and partners of the rotation are shuffles); a workgroup takes
// 256/LG heads of one row at a time, queries first, then keys, then values, which are only stored.  Cosines and sines are made once per
// workgroup, in LDS: an fp64 product and its remainder, so that a position of 10^6 turns as exactly as a position of 10.

template <bool F32>
__device__ __forceinline__ void load8(const void *base, int64_t at, float *x)
{
    if constexpr (F32) {
        const float4 a = *(const float4 *)((const float *)base + at), b = *(const float4 *)((const float *)base + at + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const bf16x8 a = *(const bf16x8 *)((const __bf16 *)base + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
    }
}

template <bool F32>
__device__ __forceinline__ void store8(void *base, int64_t at, const float *x)
{
    if constexpr (F32) {
        *(float4 *)((float *)base + at) = float4{x[0], x[1], x[2], x[3]};
        *(float4 *)((float *)base + at + 4) = float4{x[4], x[5], x[6], x[7]};
    } else {
        bf16x8 a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];      // to nearest even
        *(bf16x8 *)((__bf16 *)base + at) = a;
    }
}

// x / scale as FP8 E4M3, to nearest even; beyond the largest value as that value, NaN as NaN
__device__ __forceinline__ void store8_fp8(char *at, const float *x, float scale)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = x[i] / scale;
        y[i] = q > 448.f ? 448.f : q < -448.f ? -448.f : q;
    }
    uint2 w = {0, 0};
    w.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w.x, false);
    w.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w.x, true);
    w.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], w.y, false);
    w.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], w.y, true);
    *(uint2 *)at = w;
}

template <CacheType TYPE, int LG>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    constexpr bool F32 = TYPE == CACHE_F32;
    constexpr int KV_ES = TYPE == CACHE_FP8 ? 1 : F32 ? 4 : 2;
    __shared__ float2 turn[128];      // cosine, sine per pair
    const int row = blockIdx.x, b = row / a.pages.rows, r = row % a.pages.rows;
    if (r >= live_rows(a.pages, b)) return;
    const int L = cached_tokens(a.pages, b), half = a.rot / 2;
    if ((int)threadIdx.x < half) {
        const double angle = ((double)L + depth_of(a.pages, b, r)) * (double)a.inv_freq[threadIdx.x];
        const double turns = angle * 0.15915494309189535;                  // of 2 pi
        const float part = (float)(turns - rint(turns));                   // -0.5 .. 0.5
        float2 t;
        sincospif(2.f * part, &t.y, &t.x);
        turn[threadIdx.x] = t;
    }
    __syncthreads();
    const int64_t slot = slot_offset(a.pages, b, L + r);
    const int group = threadIdx.x / LG, lane = threadIdx.x % LG, e0 = 8 * lane;
    const bool in = e0 < a.D;
    const int heads = a.n_q + 2 * a.n_kv;
    for (int h = blockIdx.y * (256 / LG) + group; h < heads; h += gridDim.y * (256 / LG)) {
        const int kind = h < a.n_q ? 0 : h < a.n_q + a.n_kv ? 1 : 2;       // queries, keys, values
        const int hh = kind == 0 ? h : kind == 1 ? h - a.n_q : h - a.n_q - a.n_kv;
        const void *src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
        const void *norm = kind == 0 ? a.q_norm : kind == 1 ? a.k_norm : nullptr;
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (in) load8<F32>(src, row * (kind == 0 ? a.q_in_stride : a.kv_in_stride) + hh * a.D + e0, x);
        if (norm) {
            float w[8] = {0, 0, 0, 0, 0, 0, 0, 0}, ss = 0.f;
            if (in) load8<F32>(norm, e0, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
            for (int o = LG / 2; o; o /= 2) ss += __shfl_xor(ss, o);
            const float inv = 1.f / sqrtf(ss / a.D + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * w[i];
        }
        if (kind < 2 && a.rot) {
            if (a.interleaved) {
                if (e0 < a.rot)
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const float2 t = turn[(e0 + i) / 2];
                        const float x0 = x[i], x1 = x[i + 1];
                        x[i] = x0 * t.x - x1 * t.y;
                        x[i + 1] = x1 * t.x + x0 * t.y;
                    }
            } else {
                // half of the rotated elements is a multiple of 8: the partner's lane is half / 8 away
                const bool low = e0 < half, turned = e0 < a.rot;
                const int partner = (threadIdx.x & 63 & ~(LG - 1)) + (turned ? (low ? lane + half / 8 : lane - half / 8) : lane);
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner);
                if (turned)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 t = turn[low ? e0 + i : e0 + i - half];
                        x[i] = x[i] * t.x + (low ? -y[i] : y[i]) * t.y;
                    }
            }
        }
        if (!in) continue;
        if (kind == 0) {
            store8<F32>(a.q_out, row * a.q_stride + hh * a.D + e0, x);
        } else if (slot >= 0) {
            char *to = (char *)(kind == 1 ? a.k_pool : a.v_pool) + slot + hh * a.pages.head_stride + e0 * KV_ES;
            if constexpr (TYPE == CACHE_FP8) store8_fp8(to, x, kind == 1 ? a.k_scale : a.v_scale);
            else store8<F32>(to, 0, x);
        }
    }
}

template <CacheType TYPE>
static hipError_t launch_append(const AppendArgs &a, hipStream_t s)
{
    const int LG = a.D <= 64 ? 8 : a.D <= 128 ? 16 : 32, per = 256 / LG, passes = (a.n_q + 2 * a.n_kv + per - 1) / per;
    const int rows = a.pages.B * a.pages.rows;
    // a few rows: one pass per workgroup, for latency; many: one workgroup per row, which makes its cosines once (64 + 16 heads of 128: 264 rows 7.6 us in five passes and 9.0
    // in one workgroup, 1024 rows 13.4 and 14.0, 2048 rows 22.3 and 21.2, 8320 rows 95 and 79)
    const dim3 grid(rows, rows > 1024 ? 1 : passes);
    if (LG == 8) append_kernel<TYPE, 8><<<grid, 256, 0, s>>>(a);
    else if (LG == 16) append_kernel<TYPE, 16><<<grid, 256, 0, s>>>(a);
    else append_kernel<TYPE, 32><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t cache_append(CacheType type, const AppendArgs &a, hipStream_t s)
{
    return type == CACHE_F32 ? launch_append<CACHE_F32>(a, s) : type == CACHE_FP8 ? launch_append<CACHE_FP8>(a, s) : launch_append<CACHE_BF16>(a, s);
}

// ---- masks of draft trees ------------------------------------------------------------------------------------------------
// One workgroup per window.  In round i a row knows its ancestors up to distance 2^i - 1 and the one at distance 2^i (`up`, -1 if there is
// none): it takes over that one's bits and that one's `up`.  ceil(log2(K + 1)) rounds whatever the shape of the tree.  The bits are updated in
// place: a reader that finds another row's word updated in the same round already finds more of its ancestors there, never anything else,
// and what a round has to bring is there in either case.  `up` is not like that and has two copies.
// Row r has no ancestors behind itself, so it keeps r / 32 + 1 words: 1024 rows are 67 KB.
__device__ __forceinline__ int tree_word(int r, int w) { return (16 * (r / 32) + r % 32) * (r / 32 + 1) + w; }

template <int ROWS, int THREADS>
__global__ __launch_bounds__(THREADS) void tree_mask_kernel(int rows, const int32_t *parent, int32_t *depth, uint32_t *mask)
{
    __shared__ uint32_t bits[16 * (ROWS / 32) * (ROWS / 32 + 1)];
    __shared__ int16_t up[2][ROWS];
    // a thread has one word of every STEP-th row
    constexpr int WORDS = ROWS / 32, STEP = THREADS / WORDS, MINE = ROWS / STEP;
    const int words = (rows + 31) / 32, tid = threadIdx.x, w = tid % WORDS, first = tid / WORDS;
    const int32_t *mine = parent + (int64_t)blockIdx.x * (rows - 1);
    for (int r = tid; r < rows; r += THREADS) {
        int p = -1;
        if (r) {
            p = mine[r - 1];
            p = (p < -1 ? -1 : p > r - 2 ? r - 2 : p) + 1;      // node j = r - 1 hangs under one of -1 .. j - 1; rows count from the root
        }
        up[0][r] = (int16_t)p;
    }
    // it keeps its words in registers, so that a round's reads do not wait for its writes
    uint32_t own[MINE];
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
        const int r = first + k * STEP;
        own[k] = w == r / 32 ? 1u << (r & 31) : 0u;
        if (r < rows && w <= r / 32) bits[tree_word(r, w)] = own[k];
    }
    __syncthreads();
    int from = 0;
    for (int reach = 1; reach < rows; reach *= 2, from ^= 1) {
        int p[MINE];
        uint32_t y[MINE];
#pragma unroll
        for (int k = 0; k < MINE; ++k) p[k] = first + k * STEP < rows ? up[from][first + k * STEP] : -1;
#pragma unroll
        for (int k = 0; k < MINE; ++k) y[k] = p[k] >= 0 && w <= p[k] / 32 ? bits[tree_word(p[k], w)] : 0u;
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            own[k] |= y[k];
            if (p[k] >= 0 && w <= p[k] / 32) bits[tree_word(first + k * STEP, w)] = own[k];
        }
        for (int r = tid; r < rows; r += THREADS) {
            const int p = up[from][r];
            up[from ^ 1][r] = p >= 0 ? up[from][p] : (int16_t)-1;
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < MINE; ++k)
        if (first + k * STEP < rows && w < words) mask[((int64_t)blockIdx.x * rows + first + k * STEP) * words + w] = own[k];
    for (int r = tid; r < rows; r += THREADS) {
        int count = -1;
        for (int v = 0; v <= r / 32; ++v) count += __popc(bits[tree_word(r, v)]);
        depth[(int64_t)blockIdx.x * rows + r] = count;
    }
}

hipError_t tree_mask(int B, int K, const int32_t *parent, int32_t *depth, uint32_t *mask, hipStream_t s)
{
    const int rows = K + 1;
    // words and rows of a thread are known at compile time, and a workgroup is no larger than the tree: the largest form for all would take 24 us instead of 5.5 for 128 trees of 60 nodes, 34
    // instead of 11.5 for 500
    if (rows <= 64) tree_mask_kernel<64, 64><<<B, 64, 0, s>>>(rows, parent, depth, mask);
    else if (rows <= 128) tree_mask_kernel<128, 256><<<B, 256, 0, s>>>(rows, parent, depth, mask);
    else if (rows <= 256) tree_mask_kernel<256, 512><<<B, 512, 0, s>>>(rows, parent, depth, mask);
    else if (rows <= 512) tree_mask_kernel<512, 1024><<<B, 1024, 0, s>>>(rows, parent, depth, mask);
    else tree_mask_kernel<1024, 1024><<<B, 1024, 0, s>>>(rows, parent, depth, mask);
    return hipGetLastError();
}

// ---- the accepted path ---------------------------------------------------------------------------------------------------
// One workgroup per window and layer.  The path's rows come from the mask of the accepted node's row in ascending order: the i-th of them moves to
// token L + i.  A row's destination is never behind its source, and no source behind it is a destination of an earlier row that has not
// been read yet, so a thread that keeps to one 16-byte column may move the rows in order, a batch of loads before the batch's stores.
__global__ __launch_bounds__(256) void commit_kernel(CommitArgs a)
{
    constexpr int BATCH = 8;
    __shared__ int64_t to[1024], of[1024];
    const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x, rows = a.pages.rows, words = (rows + 31) / 32;
    const int L = cached_tokens(a.pages, b);
    int node = a.out_node[b];
    node = (node < -1 ? -1 : node > rows - 2 ? rows - 2 : node) + 1;      // its row
    const uint32_t *m = a.mask + ((int64_t)b * rows + node) * words;
    int n = 0, first = rows;                                              // rows of the path; the first of them that moves
    for (int w = 0; w <= node / 32; ++w) {
        uint32_t x = m[w] & (w < node / 32 ? ~0u : ~0u >> (31 - node % 32));
        if (w == 0) x |= 1u;
        const int gap = x == ~0u ? 32 : __ffs(~x) - 1;                    // rows below it are in their places
        if (first == rows && gap < 32) first = 32 * w + gap;
        const int r = 32 * w + tid;
        if (tid < 32 && x >> tid & 1) {
            const int i = n + __popc(x & ((1u << tid) - 1u));
            to[i] = slot_offset(a.pages, b, L + i);      // (the path's rows reach no further than K behind L)
            of[i] = slot_offset(a.pages, b, L + r);
        }
        n += __popc(x);
    }
    __syncthreads();
    if (layer == 0 && tid == 0) a.new_len[b] = L + n;
    if (a.n_layers == 0) return;
    const int per_head = a.row_bytes / 16, columns = 2 * a.n_kv * per_head;
    for (int c = tid; c < columns; c += 256) {
        const int h = c / per_head;
        char *pool = (h < a.n_kv ? a.k_pool : a.v_pool) + layer * a.layer_stride + (h < a.n_kv ? h : h - a.n_kv) * a.pages.head_stride +
                     c % per_head * 16;
        for (int i0 = first; i0 < n; i0 += BATCH) {
            u32x4 x[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i0 + i < n && of[i0 + i] >= 0 && to[i0 + i] >= 0) x[i] = *(const u32x4 *)(pool + of[i0 + i]);
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i0 + i < n && of[i0 + i] >= 0 && to[i0 + i] >= 0) *(u32x4 *)(pool + to[i0 + i]) = x[i];
        }
    }
}

hipError_t cache_commit(const CommitArgs &a, hipStream_t s)
{
    // gridDim.y holds 65535 layers at a time
    for (int done = 0; done == 0 || done < a.n_layers; done += 65535) {
        CommitArgs part = a;
        part.k_pool += done * a.layer_stride;
        part.v_pool += done * a.layer_stride;
        part.n_layers = a.n_layers - done < 65535 ? a.n_layers - done : 65535;
        commit_kernel<<<dim3(a.pages.B, part.n_layers ? part.n_layers : 1), 256, 0, s>>>(part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace aj

// Internal declarations of the paged cache's operators (aj_cache_*, aj_tree_mask).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aj {

enum CacheType { CACHE_BF16 = 0, CACHE_FP8 = 1, CACHE_F32 = 2 };   // queries / pools: bf16 / bf16, bf16 / FP8 E4M3, f32 / f32

// Where the tokens of the windows are.  Strides in bytes
struct Pages {
    const int32_t *table, *cache_len, *n_rows, *depth;   // n_rows, depth may be nullptr
    int B, rows;            // windows, rows of a window (K + 1)
    int log_page, n_pages, width;
    int64_t page_stride, slot_stride, head_stride;
};

__device__ __forceinline__ int cached_tokens(const Pages &p, int b)
{
    // below 2^31 with all rows behind it
    const int n = p.cache_len[b];
    return n < 0 ? 0 : n > 0x7fff0000 ? 0x7fff0000 : n;
}

__device__ __forceinline__ int live_rows(const Pages &p, int b)
{
    if (!p.n_rows) return p.rows;
    const int n = p.n_rows[b];
    return n < 0 ? 0 : n > p.rows ? p.rows : n;
}

__device__ __forceinline__ int depth_of(const Pages &p, int b, int r)
{
    if (!p.depth) return r;
    const int d = p.depth[(int64_t)b * p.rows + r];
    return d < 0 ? 0 : d > r ? r : d;
}

// byte offset of a token's slot in a pool, or -1 if the token is nowhere
__device__ __forceinline__ int64_t slot_offset(const Pages &p, int b, int t)
{
    const int e = t >> p.log_page;
    if (e >= p.width) return -1;
    const int page = p.table[(int64_t)b * p.width + e];
    if ((uint32_t)page >= (uint32_t)p.n_pages) return -1;
    return page * p.page_stride + (t & ((1 << p.log_page) - 1)) * p.slot_stride;
}

struct AppendArgs {
    Pages pages;
    const void *q, *k, *v, *q_norm, *k_norm;
    const float *inv_freq;
    void *q_out, *k_pool, *v_pool;
    int n_q, n_kv, D, rot, interleaved;
    int64_t q_in_stride, kv_in_stride, q_stride;   // elements
    float eps, k_scale, v_scale;
};
hipError_t cache_append(CacheType type, const AppendArgs &a, hipStream_t s);

struct AttendArgs {
    Pages pages;
    const void *q, *k_pool, *v_pool;
    const uint32_t *mask;
    void *out;
    float *lse;
    int n_q, n_kv, G, D, window, sinks;   // G = n_q / n_kv
    int64_t q_stride;      // elements
    float score_scale;     // scale * k_scale * log2(e): weights are powers of two
    float v_scale, inv_G;
    // the line of tiles is cut into `clusters` pieces; a cluster has a workgroup for each of `heads` heads of keys and values and `blocks` blocks of
    // vectors; groups = n_kv / heads.  Partial results of two items per piece
    int clusters, heads, groups, blocks;
    float part_cost;       // what adding a part of an item takes, in tiles
    float whole;           // items of as many tiles or fewer are not cut
    float *part_o;         // [clusters][2][heads][blocks][head size / 4][vectors of a block][4]
    float2 *part_ml;       // [clusters][2][heads][blocks][vectors of a block]
    int *arrived;          // [clusters][heads][blocks], zero between calls
};
struct AttendPlan {
    int blocks, heads, clusters;
    size_t parts, part_size;   // partial results, one per vector, and their floats
};
AttendPlan cache_attend_plan_bf16(int D, int vectors, int n_kv, int num_cus);
AttendPlan cache_attend_plan_fp8(int D, int vectors, int n_kv, int num_cus);
AttendPlan cache_attend_plan_f32(int D, int vectors, int n_kv, int num_cus);
// few: up to 32 vectors, which the waves of a workgroup share, each with tokens of its own; otherwise a wave has vectors of its own.  (64 windows over 2000 tokens, heads of 128: 4 .. 32
// vectors 96 .. 101 us, as many 111; 40 and 64 vectors 110 as many, 149 as two blocks of few)
hipError_t cache_attend_bf16(bool few, const AttendArgs &a, hipStream_t s);
hipError_t cache_attend_fp8(bool few, const AttendArgs &a, hipStream_t s);
hipError_t cache_attend_f32(bool few, const AttendArgs &a, hipStream_t s);

struct CommitArgs {
    Pages pages;
    const uint32_t *mask;
    const int32_t *out_node;
    char *k_pool, *v_pool;
    int n_layers, n_kv, row_bytes;   // bytes of one head of a token
    int64_t layer_stride;            // bytes
    int32_t *new_len;
};
hipError_t cache_commit(const CommitArgs &a, hipStream_t s);

hipError_t tree_mask(int B, int K, const int32_t *parent, int32_t *depth, uint32_t *mask, hipStream_t s);

}  // namespace aj

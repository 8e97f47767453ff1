// C ABI of the paged cache's operators (declared in include/aj.h): argument checks and workspace.
#include <math.h>
#include <new>

#include "../../include/aj.h"
#include "aj_internal.h"
#include "cache.h"

using namespace aj;

struct aj_cache {
    aj_cache_config cfg;   // strides filled in
    CacheType type;
    int es, kv_es;         // bytes of an element of q, k, v, out; of the pools
    int log_page;
    int device;
    AttendPlan plan;
    float *part_o;         // partial results of aj_cache_attend
    float2 *part_ml;
    int *arrived;
};

static bool aligned(const void *p, unsigned n) { return (((uintptr_t)p) & (n - 1)) == 0; }

static bool plan_cache(const aj_cache_config &cfg, aj_cache *h)
{
    h->cfg = cfg;
    aj_cache_config &c = h->cfg;
    if (c.B < 0 || c.K < 0 || c.K > 1023 || (int64_t)c.B * (c.K + 1) >= (1 << 24)) return false;
    if (c.n_kv < 1 || c.n_q < 1 || c.n_q > 1024 || c.n_q % c.n_kv) return false;
    if (c.head_dim < 16 || c.head_dim > 256 || c.head_dim % 16) return false;
    if (c.dtype != AJ_F32 && c.dtype != AJ_BF16) return false;
    if (c.kv_dtype != AJ_KV_SAME && !(c.kv_dtype == AJ_KV_FP8_E4M3 && c.dtype == AJ_BF16)) return false;
    if (c.page_size < 1 || c.page_size > 65536 || (c.page_size & (c.page_size - 1))) return false;
    if (c.n_pages < 1 || c.table_width < 1 || (int64_t)c.table_width * c.page_size > (1 << 30)) return false;
    if (c.window < 0 || c.sinks < 0 || (c.window == 0 && c.sinks)) return false;
    if (c.rot_dim < 0 || c.rot_dim > c.head_dim || c.rot_dim % 16) return false;
    if (c.rope != AJ_ROPE_HALF && c.rope != AJ_ROPE_INTERLEAVED) return false;
    if (c.flags) return false;
    h->type = c.dtype == AJ_F32 ? CACHE_F32 : c.kv_dtype == AJ_KV_FP8_E4M3 ? CACHE_FP8 : CACHE_BF16;
    h->es = c.dtype == AJ_F32 ? 4 : 2;
    h->kv_es = h->type == CACHE_FP8 ? 1 : h->es;
    for (h->log_page = 0; (1 << h->log_page) < c.page_size;) ++h->log_page;
    const int64_t row_q = (int64_t)c.n_q * c.head_dim, row_kv = (int64_t)c.n_kv * c.head_dim;
    if (!c.page_stride && !c.slot_stride && !c.head_stride) {
        c.head_stride = c.head_dim;
        c.slot_stride = row_kv;
        c.page_stride = c.page_size * row_kv;
    }
    const int64_t most = (int64_t)1 << 46;      // elements; offsets stay within 64 bits
    for (const int64_t s : {c.page_stride, c.slot_stride, c.head_stride})
        if (s < c.head_dim || s > most || s * h->kv_es % 16) return false;
    if (c.slot_stride * h->kv_es * c.page_size >= (1LL << 32)) return false;
    if ((double)c.n_pages * c.page_stride + (double)c.page_size * c.slot_stride + (double)c.n_kv * c.head_stride > 1e18) return false;
    if (c.qkv_stride && (c.qkv_stride < row_q || c.qkv_stride > most || c.qkv_stride * h->es % 16)) return false;
    if (!c.q_stride) c.q_stride = row_q;
    if (c.q_stride < row_q || c.q_stride > most || c.q_stride * h->es % 16) return false;
    return true;
}

static void free_cache(aj_cache *h)
{
    if (h->part_o) (void)hipFree(h->part_o);
    if (h->part_ml) (void)hipFree(h->part_ml);
    if (h->arrived) (void)hipFree(h->arrived);
    delete h;
}

extern "C" int aj_cache_create(const aj_cache_config *cfg, aj_cache **out)
{
    if (out) *out = nullptr;
    if (!cfg || !out) return AJ_EINVAL;
    aj_cache *h = new (std::nothrow) aj_cache();
    if (!h) return AJ_ENOMEM;
    if (!plan_cache(*cfg, h)) {
        delete h;
        return AJ_EINVAL;
    }
    const aj_cache_config &c = h->cfg;
    // places of the line of tiles are counted in 32 bits (tiles have 32 tokens or more)
    if ((double)c.B * c.n_kv * ((double)c.table_width * c.page_size / 32 + 2) > 2e9) {
        delete h;
        return AJ_EINVAL;
    }
    int cus = 0;
    hipError_t e = hipGetDevice(&h->device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, h->device);
    if (e != hipSuccess) {
        delete h;
        return hip_fail(e);
    }
    if (c.B > 0) {
        const int vectors = (c.K + 1) * (c.n_q / c.n_kv);
        h->plan = h->type == CACHE_F32   ? cache_attend_plan_f32(c.head_dim, vectors, c.n_kv, cus)
                  : h->type == CACHE_FP8 ? cache_attend_plan_fp8(c.head_dim, vectors, c.n_kv, cus)
                                         : cache_attend_plan_bf16(c.head_dim, vectors, c.n_kv, cus);
        const AttendPlan &p = h->plan;
        const size_t counts = (size_t)p.clusters * p.heads * p.blocks * sizeof(int);
        if (hipMalloc(&h->part_o, p.parts * p.part_size * sizeof(float)) != hipSuccess || hipMalloc(&h->part_ml, p.parts * sizeof(float2)) != hipSuccess ||
            hipMalloc(&h->arrived, counts) != hipSuccess) {
            (void)hipGetLastError();
            free_cache(h);
            return AJ_ENOMEM;
        }
        e = hipMemset(h->arrived, 0, counts);
        if (e == hipSuccess) e = hipDeviceSynchronize();
        if (e != hipSuccess) {
            free_cache(h);
            return hip_fail(e);
        }
    }
    *out = h;
    return AJ_OK;
}

extern "C" int aj_cache_destroy(aj_cache *h)
{
    if (!h) return AJ_EINVAL;
    free_cache(h);
    return AJ_OK;
}

// The workspace and the pools belong to the device that was current at aj_cache_create
static int on_its_device(const aj_cache *h)
{
    int device = -1;
    const hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return hip_fail(e);
    return device == h->device ? AJ_OK : AJ_ESTATE;
}

static bool scales_fit(const aj_cache *h, float k_scale, float v_scale)
{
    if (h->type != CACHE_FP8) return k_scale == 1.f && v_scale == 1.f;
    return k_scale > 0.f && v_scale > 0.f && isfinite(k_scale) && isfinite(v_scale);
}

static Pages pages_of(const aj_cache *h, const int32_t *table, const int32_t *cache_len, const int32_t *n_rows, const int32_t *depth)
{
    const aj_cache_config &c = h->cfg;
    Pages p;
    p.table = table;
    p.cache_len = cache_len;
    p.n_rows = n_rows;
    p.depth = depth;
    p.B = c.B;
    p.rows = c.K + 1;
    p.log_page = h->log_page;
    p.n_pages = c.n_pages;
    p.width = c.table_width;
    p.page_stride = c.page_stride * h->kv_es;
    p.slot_stride = c.slot_stride * h->kv_es;
    p.head_stride = c.head_stride * h->kv_es;
    return p;
}

extern "C" int aj_cache_append(aj_cache *h, const void *q, const void *k, const void *v, const void *q_norm, const void *k_norm, float eps,
                               const float *inv_freq, const int32_t *page_table, const int32_t *cache_len, const int32_t *n_rows,
                               const int32_t *depth, float k_scale, float v_scale, void *q_out, void *k_pool, void *v_pool, void *stream)
{
    if (!h) return AJ_EINVAL;
    if (!(eps >= 0.f) || !isfinite(eps) || !scales_fit(h, k_scale, v_scale)) return AJ_EINVAL;
    const aj_cache_config &c = h->cfg;
    if (c.B == 0) return AJ_OK;
    if (!q || !k || !v || !page_table || !cache_len || !q_out || !k_pool || !v_pool || (c.rot_dim && !inv_freq)) return AJ_EINVAL;
    for (const void *p : {q, k, v, q_norm, k_norm, (const void *)q_out, (const void *)k_pool, (const void *)v_pool})
        if (!aligned(p, 16)) return AJ_EINVAL;
    for (const void *p : {(const void *)inv_freq, (const void *)page_table, (const void *)cache_len, (const void *)n_rows, (const void *)depth})
        if (!aligned(p, 4)) return AJ_EINVAL;
    const int rc = on_its_device(h);
    if (rc != AJ_OK) return rc;
    AppendArgs a;
    a.pages = pages_of(h, page_table, cache_len, n_rows, depth);
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_norm = q_norm;
    a.k_norm = k_norm;
    a.inv_freq = inv_freq;
    a.q_out = q_out;
    a.k_pool = k_pool;
    a.v_pool = v_pool;
    a.n_q = c.n_q;
    a.n_kv = c.n_kv;
    a.D = c.head_dim;
    a.rot = c.rot_dim;
    a.interleaved = c.rope == AJ_ROPE_INTERLEAVED;
    a.q_in_stride = c.qkv_stride ? c.qkv_stride : (int64_t)c.n_q * c.head_dim;
    a.kv_in_stride = c.qkv_stride ? c.qkv_stride : (int64_t)c.n_kv * c.head_dim;
    a.q_stride = c.q_stride;
    a.eps = eps;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    const hipError_t e = cache_append(h->type, a, (hipStream_t)stream);
    return e == hipSuccess ? AJ_OK : hip_fail(e);
}

extern "C" int aj_cache_attend(aj_cache *h, const void *q, const void *k_pool, const void *v_pool, const int32_t *page_table,
                               const int32_t *cache_len, const int32_t *n_rows, const int32_t *depth, const uint32_t *mask, float scale,
                               float k_scale, float v_scale, void *out, float *lse, void *stream)
{
    if (!h) return AJ_EINVAL;
    if (!scales_fit(h, k_scale, v_scale)) return AJ_EINVAL;
    const float score_scale = (float)((double)scale * k_scale * 1.4426950408889634);
    if (!(scale > 0.f) || !isnormal(score_scale)) return AJ_EINVAL;
    const aj_cache_config &c = h->cfg;
    if (c.B == 0) return AJ_OK;
    if (!q || !k_pool || !v_pool || !page_table || !cache_len || !out) return AJ_EINVAL;
    for (const void *p : {q, k_pool, v_pool, (const void *)out})
        if (!aligned(p, 16)) return AJ_EINVAL;
    for (const void *p : {(const void *)page_table, (const void *)cache_len, (const void *)n_rows, (const void *)depth, (const void *)mask,
                          (const void *)lse})
        if (!aligned(p, 4)) return AJ_EINVAL;
    const int rc = on_its_device(h);
    if (rc != AJ_OK) return rc;
    AttendArgs a;
    a.pages = pages_of(h, page_table, cache_len, n_rows, depth);
    a.q = q;
    a.k_pool = k_pool;
    a.v_pool = v_pool;
    a.mask = mask;
    a.out = out;
    a.lse = lse;
    a.n_q = c.n_q;
    a.n_kv = c.n_kv;
    a.G = c.n_q / c.n_kv;
    a.inv_G = 1.f / (float)a.G;
    a.D = c.head_dim;
    a.window = c.window < 0x7fff0400 ? c.window : 0x7fff0400;      // beyond every position, and differences stay within 32 bits
    a.sinks = c.sinks;
    a.q_stride = c.q_stride;
    a.score_scale = score_scale;
    a.v_scale = v_scale;
    const bool few = (c.K + 1) * (c.n_q / c.n_kv) <= 32;
    a.clusters = h->plan.clusters;
    a.heads = h->plan.heads;
    a.groups = c.n_kv / h->plan.heads;
    a.blocks = h->plan.blocks;
    // Measured over one to four windows of 500 .. 30000 tokens (heads of 128 elements): few vectors 0.1 .. 0.2 (2 x 8 rows over 2500 tokens 30 us without, 26;
    // 0.4: 27), many in bf16 0.8 (32 rows over 2500 tokens 60, 35), in FP8 up to 0.4 (65 rows over 4000 tokens 40.6, 40.4; 0.8: 44), fp32, whose tiles take long, none
    a.part_cost = few ? 0.15f : h->type == CACHE_BF16 ? 0.8f : h->type == CACHE_FP8 ? 0.3f : 0.05f;
    // Many vectors in 16 or 8 bits: an item of one or two tiles takes 17 us whole, 26 in two pieces, of four 23 and 28 (44 windows x 38 rows x 4 heads), of nine
    // 35 and 28.  Few vectors take 13 in eight pieces and 19 whole (one row over 500 tokens)
    a.whole = few || h->type == CACHE_F32 ? 1.f : 4.f;
    a.part_o = h->part_o;
    a.part_ml = h->part_ml;
    a.arrived = h->arrived;
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = h->type == CACHE_F32 ? cache_attend_f32(few, a, s) : h->type == CACHE_FP8 ? cache_attend_fp8(few, a, s) : cache_attend_bf16(few, a, s);
    return e == hipSuccess ? AJ_OK : hip_fail(e);
}

extern "C" int aj_tree_mask(int32_t B, int32_t K, const int32_t *parent, int32_t *depth, uint32_t *mask, void *stream)
{
    if (B < 0 || K < 1 || K > 1023 || (int64_t)B * (K + 1) >= (1 << 24)) return AJ_EINVAL;
    if (B == 0) return AJ_OK;
    if (!parent || !depth || !mask) return AJ_EINVAL;
    if (!aligned(parent, 4) || !aligned(depth, 4) || !aligned(mask, 4)) return AJ_EINVAL;
    const hipError_t e = tree_mask(B, K, parent, depth, mask, (hipStream_t)stream);
    return e == hipSuccess ? AJ_OK : hip_fail(e);
}

extern "C" int aj_cache_commit(aj_cache *h, const uint32_t *mask, const int32_t *out_node, const int32_t *page_table, const int32_t *cache_len,
                               int32_t n_layers, int64_t layer_stride, void *k_pool, void *v_pool, int32_t *new_len, void *stream)
{
    if (!h || n_layers < 0) return AJ_EINVAL;
    const aj_cache_config &c = h->cfg;
    if (n_layers > 1 && (layer_stride < c.head_dim || layer_stride > ((int64_t)1 << 46) || layer_stride * h->kv_es % 16 ||
                         (double)layer_stride * n_layers > 1e18))
        return AJ_EINVAL;
    if (c.B == 0) return AJ_OK;
    if (!mask || !out_node || !page_table || !cache_len || !new_len || (n_layers && (!k_pool || !v_pool))) return AJ_EINVAL;
    if (new_len == cache_len) return AJ_EINVAL;
    if (!aligned(k_pool, 16) || !aligned(v_pool, 16)) return AJ_EINVAL;
    for (const void *p : {(const void *)mask, (const void *)out_node, (const void *)page_table, (const void *)cache_len, (const void *)new_len})
        if (!aligned(p, 4)) return AJ_EINVAL;
    const int rc = on_its_device(h);
    if (rc != AJ_OK) return rc;
    CommitArgs a;
    a.pages = pages_of(h, page_table, cache_len, nullptr, nullptr);
    a.mask = mask;
    a.out_node = out_node;
    a.k_pool = (char *)k_pool;
    a.v_pool = (char *)v_pool;
    a.n_layers = n_layers;
    a.n_kv = c.n_kv;
    a.row_bytes = c.head_dim * h->kv_es;
    a.layer_stride = n_layers > 1 ? layer_stride * h->kv_es : 0;
    a.new_len = new_len;
    const hipError_t e = cache_commit(a, (hipStream_t)stream);
    return e == hipSuccess ? AJ_OK : hip_fail(e);
}

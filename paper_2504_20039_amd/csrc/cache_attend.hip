// Attention of the new rows of speculation windows over the paged cache (aj_cache_attend), the plain way: one wave per row and query head,
// a token at a time with the running maximum and sum of its softmax.
#include <math.h>
#include <type_traits>

#include "cache.h"

namespace aj {

template <CacheType TYPE>
__device__ __forceinline__ float element(const char *row, int d)
{
    if constexpr (TYPE == CACHE_F32) return ((const float *)row)[d];
    else if constexpr (TYPE == CACHE_BF16) return (float)((const __bf16 *)row)[d];
    else return __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)row)[d], 0);
}

template <CacheType TYPE>
__global__ __launch_bounds__(64) void attend_kernel(AttendArgs a)
{
    typedef typename std::conditional<TYPE == CACHE_F32, float, __bf16>::type T;
    const int row = blockIdx.x, b = row / a.pages.rows, r = row % a.pages.rows, h = blockIdx.y, lane = threadIdx.x;
    if (r >= live_rows(a.pages, b)) return;
    const int L = cached_tokens(a.pages, b), hk = h / (a.n_q / a.n_kv), d = depth_of(a.pages, b, r), words = (a.pages.rows + 31) / 32;
    float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = lane + 64 * i < a.D ? (float)((const T *)a.q)[row * a.q_stride + h * a.D + lane + 64 * i] : 0.f;
    const int64_t cap = (int64_t)a.pages.width << a.pages.log_page, end = L + r + 1 < cap ? L + r + 1 : cap;
    for (int t = 0; t < end; ++t) {
        const int j = t - L;
        if (j >= 0 && a.mask && !(a.mask[(int64_t)row * words + j / 32] >> (j & 31) & 1)) continue;
        const int pos = j < 0 ? t : L + depth_of(a.pages, b, j);
        if (a.window && L + d - pos >= a.window && pos >= a.sinks) continue;
        const int64_t slot = slot_offset(a.pages, b, t);
        if (slot < 0) continue;
        const char *k = (const char *)a.k_pool + slot + hk * a.pages.head_stride, *v = (const char *)a.v_pool + slot + hk * a.pages.head_stride;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < a.D) s = fmaf(q[i], element<TYPE>(k, lane + 64 * i), s);
#pragma unroll
        for (int x = 32; x; x /= 2) s += __shfl_xor(s, x);
        s *= a.score_scale;
        const float mn = fmaxf(m, s), keep = m == -INFINITY ? 0.f : exp2f(m - mn), p = mn == -INFINITY ? 0.f : exp2f(s - mn);
        l = l * keep + p;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < a.D) o[i] = o[i] * keep + p * element<TYPE>(v, lane + 64 * i);
        m = mn;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < a.D)
            ((T *)a.out)[((int64_t)row * a.n_q + h) * a.D + lane + 64 * i] = (T)(m == -INFINITY ? 0.f : o[i] / l * a.v_scale);
    if (lane == 0 && a.lse) a.lse[(int64_t)row * a.n_q + h] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * 0.69314718f;
}

hipError_t cache_attend(CacheType type, const AttendArgs &a, hipStream_t s)
{
    const dim3 grid(a.pages.B * a.pages.rows, a.n_q);
    if (type == CACHE_F32) attend_kernel<CACHE_F32><<<grid, 64, 0, s>>>(a);
    else if (type == CACHE_FP8) attend_kernel<CACHE_FP8><<<grid, 64, 0, s>>>(a);
    else attend_kernel<CACHE_BF16><<<grid, 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace aj

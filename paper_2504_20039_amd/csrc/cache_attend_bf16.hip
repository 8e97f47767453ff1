// Attention over the paged cache, bf16 storage: the forms that are built (cache_attend.h)
#include "cache_attend.h"

namespace aj {

// Few vectors: tiles of 64 tokens, so that two workgroups' stages fit a compute unit up to heads of 128, and waves enough for the issue of their loads.  32 windows x 1 row x
// 32 heads over 4000 tokens of 8: heads of 64 take 53 us (4 waves over 128 tokens 58), of 128 95 (2 waves with all of O 98, 4 with a quarter of O each over tiles of 32 tokens 102), of 256 166 (4 waves 180)
// Many: a wave has 32 vectors, two workgroups per compute unit up to heads of 128; 16 windows x 64 rows x 32 heads over 2000 tokens of 8: heads of 128 61 us (tiles of 32 tokens 60, but 840 and 860 for 128 windows
// x 65 rows with two and four stages of them, no less than 840), of 256 116 (tiles of 64 149)
template <int DP, bool FEW> struct Choice;
template <> struct Choice<64, true> { typedef Form<CACHE_BF16, 64, 1, 2, 32, 2, 2, 2> F; };
template <> struct Choice<128, true> { typedef Form<CACHE_BF16, 128, 1, 2, 32, 2, 2, 2> F; };
template <> struct Choice<256, true> { typedef Form<CACHE_BF16, 256, 1, 2, 32, 2, 1, 4> F; };
template <> struct Choice<64, false> { typedef Form<CACHE_BF16, 64, 4, 1, 64, 2, 2> F; };
template <> struct Choice<128, false> { typedef Form<CACHE_BF16, 128, 4, 1, 64, 2, 2> F; };
template <> struct Choice<256, false> { typedef Form<CACHE_BF16, 256, 4, 1, 32, 4, 1> F; };

template <int DP>
static hipError_t launch(bool few, const AttendArgs &a, hipStream_t s)
{
    return few ? launch_attend<typename Choice<DP, true>::F>(a, s) : launch_attend<typename Choice<DP, false>::F>(a, s);
}

hipError_t cache_attend_bf16(bool few, const AttendArgs &a, hipStream_t s)
{
    return a.D <= 64 ? launch<64>(few, a, s) : a.D <= 128 ? launch<128>(few, a, s) : launch<256>(few, a, s);
}

template <int DP>
static AttendPlan plan(int vectors, int n_kv, int num_cus)
{
    return vectors <= 32 ? plan_attend<typename Choice<DP, true>::F>(vectors, n_kv, num_cus) : plan_attend<typename Choice<DP, false>::F>(vectors, n_kv, num_cus);
}

AttendPlan cache_attend_plan_bf16(int D, int vectors, int n_kv, int num_cus)
{
    return D <= 64 ? plan<64>(vectors, n_kv, num_cus) : D <= 128 ? plan<128>(vectors, n_kv, num_cus) : plan<256>(vectors, n_kv, num_cus);
}

}  // namespace aj

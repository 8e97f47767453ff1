// Attention over the paged cache, FP8 storage: the forms that are built (cache_attend.h)
#include "cache_attend.h"

namespace aj {

// Few vectors, 32 windows x 1 row x 32 heads over 4000 tokens of 8: heads of 64 take 35.5 us (2 waves 41), of 128 55 (4 waves over 128 tokens 59), of 256 98.  Many, 16 windows x 64 rows x 32 heads over 2000 tokens of 8:
// heads of 256 107 us (tiles of 32 tokens 114), of 128 57 with two stages and with three
template <int DP, bool FEW> struct Choice;
template <> struct Choice<64, true> { typedef Form<CACHE_FP8, 64, 1, 4, 32, 2, 2> F; };
template <> struct Choice<128, true> { typedef Form<CACHE_FP8, 128, 1, 2, 32, 2, 2, 2> F; };
template <> struct Choice<256, true> { typedef Form<CACHE_FP8, 256, 1, 2, 32, 2, 2, 2> F; };
template <> struct Choice<64, false> { typedef Form<CACHE_FP8, 64, 4, 1, 64, 2, 2> F; };
template <> struct Choice<128, false> { typedef Form<CACHE_FP8, 128, 4, 1, 64, 2, 2> F; };
template <> struct Choice<256, false> { typedef Form<CACHE_FP8, 256, 4, 1, 64, 4, 1> F; };

template <int DP>
static hipError_t launch(bool few, const AttendArgs &a, hipStream_t s)
{
    return few ? launch_attend<typename Choice<DP, true>::F>(a, s) : launch_attend<typename Choice<DP, false>::F>(a, s);
}

hipError_t cache_attend_fp8(bool few, const AttendArgs &a, hipStream_t s)
{
    return a.D <= 64 ? launch<64>(few, a, s) : a.D <= 128 ? launch<128>(few, a, s) : launch<256>(few, a, s);
}

template <int DP>
static AttendPlan plan(int vectors, int n_kv, int num_cus)
{
    return vectors <= 32 ? plan_attend<typename Choice<DP, true>::F>(vectors, n_kv, num_cus) : plan_attend<typename Choice<DP, false>::F>(vectors, n_kv, num_cus);
}

AttendPlan cache_attend_plan_fp8(int D, int vectors, int n_kv, int num_cus)
{
    return D <= 64 ? plan<64>(vectors, n_kv, num_cus) : D <= 128 ? plan<128>(vectors, n_kv, num_cus) : plan<256>(vectors, n_kv, num_cus);
}

}  // namespace aj

// Launch of the cache's attention: how many workgroups share a call, which
// kernel takes it, and the join of their partial results.
#include "cache_attend.h"

namespace bscache {

template <> hipError_t launch_attend_dp<64>(const Attend&, hipStream_t);
template <> hipError_t launch_attend_dp<128>(const Attend&, hipStream_t);
template <> hipError_t launch_attend_dp<256>(const Attend&, hipStream_t);

int attend_blocks(const Attend& a, int64_t max_units) {
    // as many workgroups as run at once
    const int dp = a.c.dim > 128 ? 256 : a.c.dim > 64 ? 128 : 64;
    const int64_t most =
        (int64_t)device_cus() * attend_waves(dp, a.dtype);
    const int64_t n = max_units < most ? max_units : most;
    return (int)(n < 1 ? 1 : n);
}

hipError_t launch_attend(const Attend& a, bool join, hipStream_t st) {
    const hipError_t e = a.c.dim > 128  ? launch_attend_dp<256>(a, st)
                         : a.c.dim > 64 ? launch_attend_dp<128>(a, st)
                                        : launch_attend_dp<64>(a, st);
    if (e != hipSuccess || !join) return e;
    hipLaunchKernelGGL((join_kernel<0>), dim3(a.heads * a.batch),
                       dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace bscache

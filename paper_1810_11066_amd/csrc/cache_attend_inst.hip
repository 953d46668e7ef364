// The attention kernels for BS_DP padded channels: key and value widths, and
// float32 (two float16 terms) or 16-bit calls.
#include "cache_attend.h"

namespace bscache {
namespace {

template <int DP, int KB, int VB>
hipError_t go(const Attend& a, hipStream_t st) {
    if (a.dtype == kF32)
        hipLaunchKernelGGL((attend_kernel<DP, KB, VB, true>), dim3(a.blocks),
                           dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((attend_kernel<DP, KB, VB, false>), dim3(a.blocks),
                           dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace

template <>
hipError_t launch_attend_dp<BS_DP>(const Attend& a, hipStream_t st) {
    if (a.c.bits[0] == 8)
        return a.c.bits[1] == 8 ? go<BS_DP, 8, 8>(a, st)
                                : go<BS_DP, 8, 4>(a, st);
    return a.c.bits[1] == 8 ? go<BS_DP, 4, 8>(a, st) : go<BS_DP, 4, 4>(a, st);
}

}  // namespace bscache

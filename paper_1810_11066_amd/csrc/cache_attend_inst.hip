// The attention kernels for BS_DP padded channels: every pair of key and value
// widths, every type.
#include "cache_attend.h"

namespace bscache {
namespace {

template <int DP, int KB, int VB, int T>
hipError_t go(const Attend& a, hipStream_t st) {
    if constexpr (attend_waves(DP, T) > 1)
        if (a.wide)
            return launch(attend_kernel<DP, KB, VB, T, true>, a.blocks,
                          64 * group_waves(DP, T, true), st, a);
    return launch(attend_kernel<DP, KB, VB, T, false>, a.blocks,
                  64 * group_waves(DP, T, false), st, a);
}

template <int DP, int KB, int VB>
hipError_t go(const Attend& a, hipStream_t st) {
    return a.dtype == kF32   ? go<DP, KB, VB, kF32>(a, st)
           : a.dtype == kF16 ? go<DP, KB, VB, kF16>(a, st)
                             : go<DP, KB, VB, kBF16>(a, st);
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

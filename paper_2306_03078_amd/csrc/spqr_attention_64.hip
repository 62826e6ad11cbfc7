// The attention kernels for heads of 64 elements.
#include "spqr_attention.h"

namespace spqr_srv {
template hipError_t launch_attend<_Float16, 64>(const Attend& a, const AttendPlan& p, hipStream_t st);
template hipError_t launch_attend<__bf16, 64>(const Attend& a, const AttendPlan& p, hipStream_t st);
}  // namespace spqr_srv

// The attention kernels (ivf_attend.h) over quantised caches.
#include "ivf_attend.h"

namespace ivf {

hipError_t launch_attend_quant(const AttendArgs& a, const AttendPlan& p, int row_dtype, int d, hipStream_t s) {
    return row_dtype == IVF_F16 ? launch_attend<_Float16, true>(a, p, d, s) : launch_attend<__bf16, true>(a, p, d, s);
}

}  // namespace ivf

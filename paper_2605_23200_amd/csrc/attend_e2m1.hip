// Attention over a cache of 4 bits (ams_attend): the kernels of attend_kernel.h for its codes.
#include "attend_kernel.h"

namespace ams {

hipError_t launch_attend_e2m1(const AttendArgs& a, const AttendLayout& lay, bool bf16, hipStream_t s) {
  return bf16 ? launch_dim<EL_E2M1, true>(a, lay, s) : launch_dim<EL_E2M1, false>(a, lay, s);
}

}  // namespace ams

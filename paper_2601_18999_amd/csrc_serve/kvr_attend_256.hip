// kvr_attend_256.hip - the attention kernel for heads of 256 elements.
#include "kvr_attend.h"

namespace kvr {
hipError_t launch_attend_256(const AttendArgs& a, bool fp16, bool fp8, hipStream_t st) {
  return launch_attend<256>(a, fp16, fp8, st);
}
}  // namespace kvr

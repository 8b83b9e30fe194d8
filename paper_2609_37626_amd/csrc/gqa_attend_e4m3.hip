// gqa_attend_kernel over E4M3 codes, and the choice between the code types.
#include "gqa_attend.hpp"

namespace splash {

hipError_t launch_gqa_attend_int8(const GqaAttendLaunch& a, hipStream_t s);

hipError_t launch_gqa_attend(const GqaAttendLaunch& a, hipStream_t s) {
  return a.code_type == 0 ? gqa::launch_code<0>(a, s) : launch_gqa_attend_int8(a, s);
}

}  // namespace splash

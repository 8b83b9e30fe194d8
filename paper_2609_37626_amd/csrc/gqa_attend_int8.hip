// gqa_attend_kernel over signed 8-bit codes.
#include "gqa_attend.hpp"

namespace splash {

hipError_t launch_gqa_attend_int8(const GqaAttendLaunch& a, hipStream_t s) { return gqa::launch_code<1>(a, s); }

}  // namespace splash

// ls_attend_fp8_f16.hip - attention over keys and values held in 8 bits, of float16 queries.
#include "ls_attend_codes.h"

namespace ls {

hipError_t launch_attend_fp8_f16(const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws, hipStream_t st) {
    return attend_codes_dim<_Float16, Fp8>(c, LS_F16, a, plan, ws, st);
}

}  // namespace ls

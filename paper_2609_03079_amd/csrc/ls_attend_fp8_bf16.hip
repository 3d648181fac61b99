// ls_attend_fp8_bf16.hip - attention over keys and values held in 8 bits, of bfloat16 queries.
#include "ls_attend_codes.h"

namespace ls {

hipError_t launch_attend_fp8_bf16(const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws, hipStream_t st) {
    return attend_codes_dim<__bf16, Fp8>(c, LS_BF16, a, plan, ws, st);
}

}  // namespace ls

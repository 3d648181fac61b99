// ls_attend_fp8.hip - attention over keys and values held in 8 bits.
#include "ls_attend_codes.h"

namespace ls {

hipError_t launch_attend_fp8(const ls_kvq_cache& c, ls_dtype type, const ls_attend_args& a, const AttendPlan& plan, void* ws,
                             hipStream_t st) {
    return type == LS_F16 ? attend_codes_dim<_Float16, Fp8>(c, type, a, plan, ws, st) : attend_codes_dim<__bf16, Fp8>(c, type, a, plan, ws, st);
}

}  // namespace ls

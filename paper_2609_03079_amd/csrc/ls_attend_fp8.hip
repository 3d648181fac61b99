// ls_attend_fp8.hip - attention over keys and values held in 8 bits.
#include "ls_attend.h"

namespace ls {

hipError_t launch_attend_fp8(const ls_kvq_cache& c, ls_dtype type, const ls_attend_args& a, const AttendPlan& plan, void* ws,
                             hipStream_t st) {
    const ls_kv_cache shape = shape_of(c, type);
    return type == LS_F16 ? attend_dim<_Float16, Fp8>(shape, &c, a, plan, ws, st) : attend_dim<__bf16, Fp8>(shape, &c, a, plan, ws, st);
}

}  // namespace ls

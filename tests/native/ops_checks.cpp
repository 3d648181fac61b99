// The C entry points of the decoder-layer operators with a host that has no GPU: the runtime's calls answer as one device would, and a
// launch counts itself and reads nothing, so that a test can ask for every refusal with pointers that lead nowhere.
#include <cstdlib>
#include <cstring>

#include "../../paper_2609_03079_amd/csrc/ls_ops_api.hip"

static int launches = 0;

extern "C" {
int ops_launches() { return launches; }

hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipMalloc(void** p, size_t) { return *p = std::malloc(16), hipSuccess; }
hipError_t hipFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
}

namespace ls {
static hipError_t counted() { return ++launches, hipSuccess; }
hipError_t launch_norm(const ls_norm_args&, hipStream_t) { return counted(); }
hipError_t launch_append(const ls_kv_cache&, const ls_append_args&, hipStream_t) { return counted(); }
size_t linear_workspace(const ls_linear_i8_args&) { return 0; }
hipError_t launch_linear(const ls_linear_i8_args&, void*, size_t, int, hipStream_t) { return counted(); }
bool plan_attend(const ls_kv_cache&, const ls_attend_args&, size_t, int, AttendPlan*) { return true; }
hipError_t launch_attend(const ls_kv_cache&, const ls_attend_args&, const AttendPlan&, void*, hipStream_t) { return counted(); }
hipError_t launch_kvq_append(const ls_kvq_cache&, ls_dtype, const ls_append_args&, hipStream_t) { return counted(); }
hipError_t launch_kvq_read(const ls_kvq_cache&, const ls_kvq_read_args&, hipStream_t) { return counted(); }
// What a plan may be: parts that the join and the workspace hold, chunks that cover the keys, fewer threads than a launch has.
static hipError_t planned(const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& p) {
    const int64_t parts = p.pre_parts + p.suf_parts, G = a.n_heads / c.n_kv_heads;
    const int64_t rows_pre = (int64_t)a.n_seqs * a.n_q * G, rows_suf = (int64_t)a.n_q * G;
    const bool good = parts >= 1 && parts <= kMaxParts && p.pre_chunk >= 64 && p.suf_chunk >= 64 && p.pre_chunk % 64 == 0 && p.suf_chunk % 64 == 0 &&
                      (int64_t)p.pre_parts * p.pre_chunk >= a.prefix_len && (int64_t)p.suf_parts * p.suf_chunk >= a.max_len &&
                      (int64_t)p.pre_tiles * (p.pre_wide ? 128 : 16) >= rows_pre && (int64_t)p.suf_tiles * (p.suf_wide ? 128 : 16) >= rows_suf;
    return good ? counted() : hipErrorInvalidValue;
}
hipError_t launch_attend_fp4_f16(const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& p, void*, hipStream_t) { return planned(c, a, p); }
hipError_t launch_attend_fp4_bf16(const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& p, void*, hipStream_t) { return planned(c, a, p); }
hipError_t launch_attend_fp8_f16(const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& p, void*, hipStream_t) { return planned(c, a, p); }
hipError_t launch_attend_fp8_bf16(const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& p, void*, hipStream_t) { return planned(c, a, p); }
hipError_t launch_verify(const ls_verify_args&, void*, size_t, int, hipStream_t) { return counted(); }
}  // namespace ls

#include "../../paper_2609_03079_amd/csrc/ls_attend_plan.hip"

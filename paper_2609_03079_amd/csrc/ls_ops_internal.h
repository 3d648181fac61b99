// ls_ops_internal.h - shared declarations of the decoder-layer operators (include/ls_ops.h).
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/ls_ops.h"

namespace ls {

// ---- norms around a block (ls_rows.hip) ----------------------------------------------------
hipError_t launch_norm(const ls_norm_args& a, hipStream_t st);

// ---- append to the paged cache (ls_rows.hip) -----------------------------------------------
hipError_t launch_append(const ls_kv_cache& c, const ls_append_args& a, hipStream_t st);

// ---- 8-bit products (ls_linear.hip) --------------------------------------------------------
// Workspace that the call needs: the quantised tokens and their scales, where they go through memory.
size_t linear_workspace(const ls_linear_i8_args& a);
// ws_bytes: what there is; what is left of it may hold sums of a k that is split.
hipError_t launch_linear(const ls_linear_i8_args& a, void* ws, size_t ws_bytes, int n_cu, hipStream_t st);

// ---- attention (ls_attend.hip) -------------------------------------------------------------
constexpr int kMaxParts = 128;  // partial results of one row, at most
struct AttendPlan {
    int pre_chunk, pre_parts, pre_tiles;  // keys per part of the prefix, parts, row tiles
    int suf_chunk, suf_parts, suf_tiles;
    bool pre_wide, suf_wide;              // 128-row tiles instead of 32-row tiles
    bool alike;                           // prefix and sequences by the same kernel, in one launch
    bool together;                        // a wide prefix and narrow sequences in one launch
};
// For at most 2^20 rows n_seqs n_q n_heads, or one sequence.  False where no split fits the workspace.
bool plan_attend(const ls_kv_cache& c, const ls_attend_args& a, size_t ws_bytes, int n_cu, AttendPlan* plan);
hipError_t launch_attend(const ls_kv_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws,
                         hipStream_t st);

// ---- elements ------------------------------------------------------------------------------
// V elements moved as one access of up to 16 bytes.
template <typename T, int V>
struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Pack {
    T e[V];
};

template <typename T, int V>
__device__ inline Pack<T, V> load_pack(const void* p, int64_t elem) {
    return *reinterpret_cast<const Pack<T, V>*>(static_cast<const T*>(p) + elem);
}
template <typename T, int V>
__device__ inline void store_pack(void* p, int64_t elem, const Pack<T, V>& v) {
    *reinterpret_cast<Pack<T, V>*>(static_cast<T*>(p) + elem) = v;
}

inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int64_t ceil_div(int64_t x, int64_t y) { return (x + y - 1) / y; }
inline size_t type_size(ls_dtype t) { return t == LS_F32 ? 4 : t == LS_I8 ? 1 : 2; }

}  // namespace ls

// ls_attend.h - what the attention's kernels share: their parameters, the work of a workgroup, the join of the parts, the launches of
// a plan.  ls_attend.hip holds keys and values of 16 bits, ls_attend_codes.h those of 4 and 8.
#pragma once

#include <algorithm>
#include <type_traits>

#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <typename T>
using vec8 = std::conditional_t<std::is_same_v<T, _Float16>, f16x8, bf16x8>;

__device__ inline f32x16 mma(const f16x8& a, const f16x8& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Quotients of 0 <= n < 2^31 by a number the host knows: a product and a shift.
struct Div {
    uint32_t m;
    int shift, d;
    Div() = default;
    explicit Div(int d_) : d(d_) {
        int log = 0;
        while ((int64_t)1 << log < d_) ++log;
        shift = 31 + log;
        m = (uint32_t)((((uint64_t)1 << shift) + (uint32_t)d_ - 1) / (uint32_t)d_);
    }
    __host__ __device__ inline int of(int n) const { return (int)(((uint64_t)(uint32_t)n * m) >> shift); }
};

struct AttendP {
    const void* q;
    int64_t q_token, q_head;
    void* out;
    int64_t o_token, o_head;
    const void* k;
    const void* v;
    int64_t page_stride, head_stride, token_stride;  // elements; bytes where the cache holds codes
    const uint8_t* k_scale;                          // codes only
    const uint8_t* v_scale;
    int64_t s_page, s_head, s_token;
    int n_pages, page_shift;
    const int32_t* prefix_pages;
    const int32_t* pages;
    int64_t pages_stride;
    const int32_t* lens;
    int prefix_len, max_len;
    int S, n_q, H, KV, G, D;
    Div by_S, by_n_q, by_H, by_KV, by_G, by_pre_tiles, by_suf_tiles, by_suf_chunk;
    float c;                 // scale log2(e): the softmax runs in powers of two
    AttendPlan plan;
    int pre_items, suf_items;  // workgroups of this launch
    int near_units;          // sequences times parts whose heads are near each other (codes only); 0: heads are apart
    Div by_near;             // eight units' workgroups, over eight
    int parts;               // partial results per row
    bool direct;             // a row has one part, which is the result
    float* part;             // [rows][parts][D]
    float* ml;               // [rows][parts][2]
};

// The largest weight is 2^kLift.  Weights enter the second product in 16 bits (in 32 the product
// would run at a sixteenth of the rate), and with a largest of one float16 would drop those below 2^-25,
// which the sum counts: 30000 keys that far below one that dominates are a thousandth of the
// result.  With 2^7 those below 2^-32 are dropped, a part's 65536 at most a 2^-16th; what is left
// of the type's range is for a maximum that was rounded (by 2^8 at most while |m| < 2^28).
template <typename T>
constexpr float kLift = std::is_same_v<T, _Float16> ? 7.f : 0.f;

// The value of lane ^ 32.
__device__ inline float other_half(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// What a workgroup works on.
struct Item {
    const int32_t* table;  // page ids
    int begin, end;        // keys
    int kv;                // key/value head
    int row0, rows;        // first row of its tile, rows of all tiles
    int seq;               // -1: the prefix
    int part;              // its place among a row's parts
    int len;               // the sequence's keys
};

// Share `b` of the prefix's or of the sequences' work; a sequence's length is not looked up yet.
template <int R>
__device__ inline bool item_of(const AttendP& p, bool prefix, int b, Item* it) {
    if (prefix) {
        // workgroups that follow each other run on different XCDs: the row tiles of the same keys
        // take every eighth workgroup, so that they share an L2
        const int eighth = b >> 3, turn = p.by_pre_tiles.of(eighth), group = turn * 8 + (b & 7);
        if (group >= p.plan.pre_parts * p.KV) return false;
        it->row0 = (eighth - turn * p.plan.pre_tiles) * R;
        it->part = p.by_KV.of(group);
        it->kv = group - it->part * p.KV;
        it->seq = -1;
        it->table = p.prefix_pages;
        it->begin = it->part * p.plan.pre_chunk;
        it->end = min(p.prefix_len, it->begin + p.plan.pre_chunk);
        it->rows = p.S * p.n_q * p.G;
        return true;
    }
    const int tile = b, rest = p.by_suf_tiles.of(b), of_kv = p.by_KV.of(rest), j = p.by_S.of(of_kv);
    it->row0 = (tile - rest * p.plan.suf_tiles) * R;
    it->kv = rest - of_kv * p.KV;
    it->seq = of_kv - j * p.S;
    it->table = p.pages + it->seq * p.pages_stride;
    it->begin = j * p.plan.suf_chunk;
    it->end = min(p.max_len, it->begin + p.plan.suf_chunk);
    it->rows = p.n_q * p.G;
    it->part = p.plan.pre_parts + j;
    return true;
}

template <int CTRL, int ROWS>
__device__ inline float max_dpp(float v) {
    const int x = __float_as_int(v);
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xf, false)));
}
__device__ inline float wave_max(float v) {
    v = max_dpp<0xb1, 0xf>(v);   // quad_perm [1,0,3,2]
    v = max_dpp<0x4e, 0xf>(v);   // quad_perm [2,3,0,1]
    v = max_dpp<0x141, 0xf>(v);  // row_half_mirror
    v = max_dpp<0x140, 0xf>(v);  // row_mirror
    v = max_dpp<0x142, 0xa>(v);  // row_bcast:15
    v = max_dpp<0x143, 0xc>(v);  // row_bcast:31
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Joins the parts of a row: a wave for 64 of its elements, 16 lanes across them and the other lanes on
// other parts (a wave for a whole row took 9.2 us, not 4.0, for 48 rows of 65 parts of 256 elements).
// Bound by latency: the sequence's length, the maxima and sums and the first parts are all asked for
// at once, parts that turn out never to have been written among them (their weight is zero, and they
// are not looked at).
template <typename T, int DP>
__global__ __launch_bounds__(64) void join_kernel(const AttendP p) {
    constexpr int L = 16, GR = 64 / L, U = 16 / GR;  // 16 parts at a time
    const int lane = threadIdx.x & 63, r = blockIdx.x;
    const int token = p.by_H.of(r), seq = p.by_n_q.of(token);
    const float* ml = p.ml + (int64_t)r * p.parts * 2;
    const float* part = p.part + (int64_t)r * p.parts * p.D;
    const int d = blockIdx.y * 64 + (lane % L) * 4, g = lane / L, dd = min(d, p.D - 4);
    float m[2], l[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int j = min(i * 64 + lane, p.parts - 1);
        m[i] = ml[j * 2];
        l[i] = ml[j * 2 + 1];
    }
    f32x4 v[U];
    auto ask = [&](int j0) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const f32x4*>(part + (int64_t)min(j0 + u * GR + g, p.parts - 1) * p.D + dd);
    };
    ask(0);
    const int len = min(p.lens[seq], p.max_len);
    // parts that were written: the prefix's unless the slot is idle, and the sequence's that hold keys
    const int first = len < 0 ? p.plan.pre_parts : 0;
    const int last = p.plan.pre_parts + (len > 0 ? p.by_suf_chunk.of(len + p.plan.suf_chunk - 1) : 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int j = i * 64 + lane;
        const bool in = j >= first && j < last;
        m[i] = in ? m[i] : -INFINITY;
        l[i] = in ? l[i] : 0.f;
    }
    const float top = wave_max(fmaxf(m[0], m[1])), base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = l[i] == 0.f ? 0.f : __builtin_amdgcn_exp2f(m[i] - base);  // now its weight
    const float sum = wave_sum_dpp(l[0] * m[0] + l[1] * m[1]);
    // parts without a key must not count, whatever lies in their place; the others must, even with a weight
    // that is zero in fp32: a value that is no number makes the row none
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = l[i] == 0.f ? -1.f : m[i];
    f32x4 acc{};
    for (int j0 = 0; j0 < last; j0 += U * GR) {
        if (j0) ask(j0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * GR + g;
            const float w = __shfl(j < 64 ? m[0] : m[1], j & 63, 64);
            if (j < last && !(w < 0.f)) acc += v[u] * w;
        }
    }
#pragma unroll
    for (int off = L; off < 64; off <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], off, 64);
    if (g == 0 && d < p.D) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        Pack<T, 4> o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o.e[e] = (T)(acc[e] * inv);
        store_pack<T, 4>(p.out, token * p.o_token + (r - token * p.H) * p.o_head + d, o);
    }
}

// The parameters of a plan; c: the cache (of codes: its shape, and strides in bytes).
inline AttendP attend_params(const ls_kv_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws) {
    AttendP p{};
    p.q = a.q, p.q_token = a.q_token_stride, p.q_head = a.q_head_stride;
    p.out = a.out, p.o_token = a.out_token_stride, p.o_head = a.out_head_stride;
    p.k = c.k, p.v = c.v;
    p.page_stride = c.page_stride, p.head_stride = c.head_stride, p.token_stride = c.token_stride;
    p.n_pages = c.n_pages, p.page_shift = __builtin_ctz(c.page_size);
    p.prefix_pages = a.prefix_pages, p.pages = a.pages, p.pages_stride = a.pages_stride, p.lens = a.lens;
    p.prefix_len = a.prefix_len, p.max_len = a.max_len;
    p.S = a.n_seqs, p.n_q = a.n_q, p.H = a.n_heads, p.KV = c.n_kv_heads, p.G = a.n_heads / c.n_kv_heads, p.D = c.head_dim;
    p.c = a.scale * 1.44269504f;
    p.plan = plan;
    p.by_S = Div(p.S), p.by_n_q = Div(p.n_q), p.by_H = Div(p.H), p.by_KV = Div(p.KV), p.by_G = Div(p.G);
    p.by_pre_tiles = Div(plan.pre_tiles), p.by_suf_tiles = Div(plan.suf_tiles), p.by_suf_chunk = Div(plan.suf_chunk);
    p.parts = plan.pre_parts + plan.suf_parts;
    p.direct = plan.pre_parts == 0 && plan.suf_parts == 1;
    const int64_t rows = (int64_t)p.S * p.n_q * p.H;
    p.part = static_cast<float*>(ws);
    p.ml = p.part + rows * p.parts * p.D;
    return p;
}

// Launches what a plan asks for: `go` takes a shape (of the prefix, of the sequences, or of a wide prefix beside narrow sequences) and
// the workgroups of each.
template <typename T, int DP, typename Role, typename Go>
hipError_t launch_plan(const AttendP& p, Role pre_role, Role suf_role, Role both_role, hipStream_t st, Go go) {
    const AttendPlan& plan = p.plan;
    const int pre = (int)round_up(plan.pre_parts * p.KV, 8) * plan.pre_tiles, suf = plan.suf_parts * p.S * p.KV * plan.suf_tiles;
    hipError_t e;
    if (pre == 0 || suf == 0 || plan.alike) {
        e = go(pre ? pre_role : suf_role, pre, suf);
    } else if (plan.together) {
        e = go(both_role, pre, suf);
    } else {
        e = go(pre_role, pre, 0);
        if (e == hipSuccess) e = go(suf_role, 0, suf);
    }
    if (e != hipSuccess || p.direct) return e;
    const int64_t rows = (int64_t)p.S * p.n_q * p.H;
    hipLaunchKernelGGL((join_kernel<T, DP>), dim3((unsigned)rows, (unsigned)ceil_div(p.D, 64)), dim3(64), 0, st, p);
    return hipGetLastError();
}

}  // namespace
}  // namespace ls

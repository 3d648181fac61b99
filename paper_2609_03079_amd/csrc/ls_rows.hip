// ls_rows.hip - operators that touch every element of a token's rows once: the norms around a
// block with its gated residual update, and the append of rotated keys and values to a paged cache.
//
// Both are bound by HBM (or, for a handful of tokens, by the latency of one pass of loads): a
// row is read once, everything is computed in fp32, and the result is written once.
#include <algorithm>

#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {
namespace {

// A store that leaves no trace in the caches, where the output is larger than they are.
template <typename T, int V>
__device__ inline void put_pack(void* p, int64_t elem, const Pack<T, V>& v, bool past_caches) {
    constexpr int kBytes = sizeof(T) * V;
    if constexpr (kBytes % 16 == 0) {
        if (past_caches) {
            u32x4 w[kBytes / 16];
            __builtin_memcpy(w, &v, kBytes);
            u32x4* to = reinterpret_cast<u32x4*>(static_cast<T*>(p) + elem);
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) __builtin_nontemporal_store(w[i], to + i);
            return;
        }
    }
    store_pack<T, V>(p, elem, v);
}

// ---- norms ---------------------------------------------------------------------------------
// Sum over NT threads in a fixed order: lanes of a wave, then the waves in order.
template <int NT>
__device__ inline float row_sum(float v, float* part) {
    v = wave_sum_dpp(v);
    if (NT == 64) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) s += part[w];
    return s;
}

// One workgroup per token; thread t holds the V-element vectors t, t + NT, ... (C of them) of the
// row.  All loads are issued before the first sum, so a single token costs one memory round trip
// and two sums.  Rows of up to 8192 elements have a thread for every vector: 8191 x 8192 bfloat16
// with a gate for each token 171 us, with four vectors a thread 230; outputs larger than the caches
// are stored past them: 163 to 173 us (939 MB at 5.4 to 5.7 TB/s; a copy of 1 GiB moves 5.2).
// The row stays in registers up to 16384 elements in whole vectors, up to 8192 otherwise; longer ones do not
// fit the 128 that 1024 threads leave a lane (55 to 168 spilled) and go partly through scratch memory: 4096 rows
// of bfloat16 with a gate for each token take 193 us at 16384 elements, 458 at 20480, 549 at 12289.
// Rows of odd lengths or addresses move an element an access: 8191 elements 166 us, 8192 94.
template <typename T, int V, int C, int NT>
__global__ __launch_bounds__(NT) void norm_kernel(const ls_norm_args p, bool past_caches) {
    __shared__ float part[2][NT / 64];
    const int64_t row = blockIdx.x;
    float x[C][V];
    Pack<T, V> y[C], g[C], wp[C], wh[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = ((int)threadIdx.x + NT * c) * V;
        if (e >= p.d) continue;
        if (p.y) y[c] = load_pack<T, V>(p.y, row * p.y_stride + e);
        const auto xv = load_pack<float, V>(p.x, row * p.x_stride + e);
#pragma unroll
        for (int i = 0; i < V; ++i) x[c][i] = xv.e[i];
        if (p.y && p.gate) g[c] = load_pack<T, V>(p.gate, row * p.gate_stride + e);
        if (p.y && p.post_weight) wp[c] = load_pack<T, V>(p.post_weight, e);
        if (p.h && p.pre_weight) wh[c] = load_pack<T, V>(p.pre_weight, e);
    }
    float post = 1.f;
    if (p.y && p.post_norm) {
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (((int)threadIdx.x + NT * c) * V >= p.d) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) ss = fmaf((float)y[c].e[i], (float)y[c].e[i], ss);
        }
        post = 1.f / sqrtf(row_sum<NT>(ss, part[0]) / (float)p.d + p.eps);
    }
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = ((int)threadIdx.x + NT * c) * V;
        if (e >= p.d) continue;
        Pack<float, V> o;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v = p.x_scale * x[c][i];
            if (p.y) {
                float t = (float)y[c].e[i] * post;
                if (p.post_weight) t *= (float)wp[c].e[i];
                if (p.gate) t *= (float)g[c].e[i];
                v = fmaf(p.y_scale, t, v);
            }
            x[c][i] = o.e[i] = v;
            ss = fmaf(v, v, ss);
        }
        if (p.x_out) put_pack<float, V>(p.x_out, row * p.x_out_stride + e, o, past_caches);
    }
    if (!p.h) return;
    const float pre = p.pre_norm ? 1.f / sqrtf(row_sum<NT>(ss, part[1]) / (float)p.d + p.eps) : 1.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = ((int)threadIdx.x + NT * c) * V;
        if (e >= p.d) continue;
        Pack<T, V> o;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v = x[c][i] * pre;
            if (p.pre_weight) v *= (float)wh[c].e[i];
            o.e[i] = (T)v;
        }
        put_pack<T, V>(p.h, row * p.h_stride + e, o, past_caches);
    }
}

// Outputs of a call that the 32 MB of the L2s cannot hold are not kept there.
bool past_caches(double bytes) { return bytes > 32e6; }

template <typename T, int V, int C, int NT>
hipError_t norm_launch(const ls_norm_args& a, hipStream_t st) {
    const double bytes = (double)a.n_tokens * a.d * ((a.x_out ? 4 : 0) + (a.h ? sizeof(T) : 0));
    hipLaunchKernelGGL((norm_kernel<T, V, C, NT>), dim3(a.n_tokens), dim3(NT), 0, st, a, past_caches(bytes));
    return hipGetLastError();
}

template <typename T>
hipError_t norm_type(const ls_norm_args& a, hipStream_t st) {
    const size_t es = sizeof(T);
    auto row_ok = [&](const void* p, int64_t stride, size_t size) {
        return !p || (aligned(p, 16) && stride * size % 16 == 0);
    };
    const bool vec = a.d % 8 == 0 && row_ok(a.x, a.x_stride, 4) && row_ok(a.x_out, a.x_out_stride, 4) &&
                     row_ok(a.y, a.y_stride, es) && row_ok(a.gate, a.gate_stride, es) &&
                     row_ok(a.h, a.h_stride, es) && row_ok(a.post_weight, 0, es) && row_ok(a.pre_weight, 0, es);
    if (!vec) {  // odd lengths or alignments: one element per access
        if (a.d <= 1024) return norm_launch<T, 1, 4, 256>(a, st);
        if (a.d <= 8192) return norm_launch<T, 1, 8, 1024>(a, st);
        return norm_launch<T, 1, 32, 1024>(a, st);
    }
    const int units = a.d / 8;
    if (units <= 64) return norm_launch<T, 8, 1, 64>(a, st);
    if (units <= 128) return norm_launch<T, 8, 1, 128>(a, st);
    if (units <= 256) return norm_launch<T, 8, 1, 256>(a, st);
    if (units <= 512) return norm_launch<T, 8, 1, 512>(a, st);
    if (units <= 1024) return norm_launch<T, 8, 1, 1024>(a, st);
    if (units <= 2048) return norm_launch<T, 8, 2, 1024>(a, st);
    return norm_launch<T, 8, 4, 1024>(a, st);
}

// ---- append --------------------------------------------------------------------------------
struct AppendP {
    ls_kv_cache c;
    ls_append_args a;
    int rot_units, units, v_units;  // vectors of a key or query head that turn, all of them, of a value head
};

// A thread moves one vector of one head at a time: V pairs that turn (or V / 2 of neighbours), or
// V elements that are copied.  The vectors of a token's query, key and value heads follow each
// other; blockIdx.x is the token, blockIdx.y 256 of its vectors.  8192 tokens of 64 query and 8 key
// heads of 128 bfloat16: 58 to 65 us (340 MB at 5.2 to 5.8 TB/s), 73 with the stores kept in the caches, 78 with
// one workgroup for all of a token's vectors.
template <typename T, int V, bool PAIR>
__global__ __launch_bounds__(256) void append_kernel(const AppendP p, bool past_caches) {
    const ls_append_args& a = p.a;
    const ls_kv_cache& c = p.c;
    const int64_t t = blockIdx.x;
    int pos = 0;
    if (a.rot_dim) {
        pos = a.positions[t];
        if (pos < 0 || pos >= a.n_pos) return;
    }
    const int slot = a.slots[t];
    const bool keep = slot >= 0 && slot < c.n_pages * c.page_size;
    const int64_t to = keep ? (int64_t)(slot / c.page_size) * c.page_stride + (int64_t)(slot % c.page_size) * c.token_stride : 0;
    const int qk_heads = a.n_heads + c.n_kv_heads, half = a.rot_dim / 2;
    const int qk_total = qk_heads * p.units, total = qk_total + (keep ? c.n_kv_heads * p.v_units : 0);
    const float* cs = a.cos_sin + (int64_t)pos * a.rot_dim;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < total; i += 256 * gridDim.y) {
        if (i >= qk_total) {
            const int j = i - qk_total, h = j / p.v_units, e = (j - h * p.v_units) * V;
            put_pack<T, V>(c.v, to + h * c.head_stride + e,
                             load_pack<T, V>(a.v, t * a.v_token_stride + h * a.v_head_stride + e), past_caches);
            continue;
        }
        const int r = i / p.units, u = i - r * p.units;
        const bool is_q = r < a.n_heads;
        if (!is_q && !keep) continue;
        const int h = is_q ? r : r - a.n_heads;
        const void* src = is_q ? a.q : a.k;
        void* dst = is_q ? a.q_out : c.k;
        const int64_t from = is_q ? t * a.q_token_stride + h * a.q_head_stride : t * a.k_token_stride + h * a.k_head_stride;
        const int64_t at = is_q ? t * a.q_out_token_stride + h * a.q_out_head_stride : to + h * c.head_stride;
        if (u >= p.rot_units) {
            const int e = a.rot_dim + (u - p.rot_units) * V;
            put_pack<T, V>(dst, at + e, load_pack<T, V>(src, from + e), past_caches);
        } else if (!PAIR) {
            const int e = u * V;
            auto x = load_pack<T, V>(src, from + e), y = load_pack<T, V>(src, from + half + e);
            const auto co = load_pack<float, V>(cs, e), si = load_pack<float, V>(cs, half + e);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float l = (float)x.e[k], m = (float)y.e[k];
                x.e[k] = (T)(l * co.e[k] - m * si.e[k]);
                y.e[k] = (T)(m * co.e[k] + l * si.e[k]);
            }
            put_pack<T, V>(dst, at + e, x, past_caches);
            put_pack<T, V>(dst, at + half + e, y, past_caches);
        } else {
            constexpr int W = V < 2 ? 2 : V;  // elements of a unit; single ones go one by one
            const int e = u * W;
            T x[W];
            if (V < 2) {
                x[0] = static_cast<const T*>(src)[from + e];
                x[1] = static_cast<const T*>(src)[from + e + 1];
            } else {
                const auto v = load_pack<T, W>(src, from + e);
#pragma unroll
                for (int k = 0; k < W; ++k) x[k] = v.e[k];
            }
            const auto co = load_pack<float, W / 2>(cs, e / 2), si = load_pack<float, W / 2>(cs, half + e / 2);
            Pack<T, W> o;
#pragma unroll
            for (int k = 0; k < W / 2; ++k) {
                const float l = (float)x[2 * k], m = (float)x[2 * k + 1];
                o.e[2 * k] = (T)(l * co.e[k] - m * si.e[k]);
                o.e[2 * k + 1] = (T)(m * co.e[k] + l * si.e[k]);
            }
            if (V < 2) {
                static_cast<T*>(dst)[at + e] = o.e[0];
                static_cast<T*>(dst)[at + e + 1] = o.e[1];
            } else {
                put_pack<T, W>(dst, at + e, o, past_caches);
            }
        }
    }
}

template <typename T, int V>
hipError_t append_launch(const ls_kv_cache& c, const ls_append_args& a, hipStream_t st) {
    AppendP p{c, a, 0, 0, 0};
    const bool pair = a.style == LS_ROPE_PAIR;
    p.rot_units = pair ? a.rot_dim / (V < 2 ? 2 : V) : a.rot_dim / 2 / V;
    p.units = p.rot_units + (c.head_dim - a.rot_dim) / V;
    p.v_units = c.head_dim / V;
    const int64_t total = (int64_t)(a.n_heads + c.n_kv_heads) * p.units + (int64_t)c.n_kv_heads * p.v_units;
    const dim3 grid(a.n_tokens, (unsigned)std::min<int64_t>(ceil_div(total, 256), 65535));
    const bool past = past_caches((double)a.n_tokens * (a.n_heads + 2 * c.n_kv_heads) * c.head_dim * sizeof(T));
    if (pair)
        hipLaunchKernelGGL((append_kernel<T, V, true>), grid, dim3(256), 0, st, p, past);
    else
        hipLaunchKernelGGL((append_kernel<T, V, false>), grid, dim3(256), 0, st, p, past);
    return hipGetLastError();
}

template <typename T>
hipError_t append_type(const ls_kv_cache& c, const ls_append_args& a, hipStream_t st) {
    // vectors of v elements: every address and offset that the kernel forms is a multiple of them
    auto fits = [&](int v) {
        const int64_t by = std::min<int64_t>(16, (int64_t)v * sizeof(T)), el = by / (int64_t)sizeof(T);
        const int fl = a.style == LS_ROPE_PAIR ? v / 2 : v;  // cosines of one access
        for (int64_t s : {c.page_stride, c.head_stride, c.token_stride, a.k_token_stride, a.k_head_stride, a.v_token_stride,
                          a.v_head_stride, a.q_token_stride, a.q_head_stride, a.q_out_token_stride, a.q_out_head_stride})
            if (s % el) return false;
        for (const void* q : {(const void*)c.k, (const void*)c.v, a.k, a.v, a.q, (const void*)a.q_out})
            if (q && !aligned(q, by)) return false;
        if (a.rot_dim && !aligned(a.cos_sin, std::min(16, 4 * fl))) return false;
        return c.head_dim % v == 0 && (a.rot_dim / 2) % fl == 0 && a.rot_dim % v == 0;
    };
    if (fits(8)) return append_launch<T, 8>(c, a, st);
    if (fits(4)) return append_launch<T, 4>(c, a, st);
    return append_launch<T, 1>(c, a, st);
}

}  // namespace

// A launch holds fewer than 2^32 threads along x: calls with a workgroup of up to 1024 for each of
// more tokens than this are cut.
constexpr int kTokensPerLaunch = 1 << 21;

hipError_t launch_norm(const ls_norm_args& a, hipStream_t st) {
    for (int64_t t = 0; t < a.n_tokens; t += kTokensPerLaunch) {
        ls_norm_args b = a;
        const int64_t es = (int64_t)type_size(a.dtype);
        auto skip = [&](const void* p, int64_t stride) { return p ? static_cast<const char*>(p) + t * stride * es : nullptr; };
        b.n_tokens = (int32_t)std::min<int64_t>(kTokensPerLaunch, a.n_tokens - t);
        b.x += t * a.x_stride;
        if (b.x_out) b.x_out += t * a.x_out_stride;
        b.y = skip(a.y, a.y_stride);
        b.gate = skip(a.gate, a.gate_stride);
        b.h = const_cast<char*>(skip(a.h, a.h_stride));
        const hipError_t e = a.dtype == LS_F32   ? norm_type<float>(b, st)
                             : a.dtype == LS_F16 ? norm_type<_Float16>(b, st)
                                                 : norm_type<__bf16>(b, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_append(const ls_kv_cache& c, const ls_append_args& a, hipStream_t st) {
    for (int64_t t = 0; t < a.n_tokens; t += kTokensPerLaunch) {
        ls_append_args b = a;
        const int64_t es = (int64_t)type_size(c.dtype);
        auto skip = [&](const void* p, int64_t stride) { return p ? static_cast<const char*>(p) + t * stride * es : nullptr; };
        b.n_tokens = (int32_t)std::min<int64_t>(kTokensPerLaunch, a.n_tokens - t);
        b.k = skip(a.k, a.k_token_stride);
        b.v = skip(a.v, a.v_token_stride);
        b.q = skip(a.q, a.q_token_stride);
        b.q_out = const_cast<char*>(skip(a.q_out, a.q_out_token_stride));
        if (b.positions) b.positions += t;
        b.slots += t;
        const hipError_t e = c.dtype == LS_F32   ? append_type<float>(c, b, st)
                             : c.dtype == LS_F16 ? append_type<_Float16>(c, b, st)
                                                 : append_type<__bf16>(c, b, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ls

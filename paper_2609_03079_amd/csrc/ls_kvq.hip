// ls_kvq.hip - a paged cache of keys and values in 4 or 8 bits: written (the keys, and queries beside them,
// turned to their positions on the way) and read back.
#include <algorithm>

#include "ls_codes.h"
#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {
namespace {

// Elements e .. e + 7 of a row in fp32.  VEC: the row's start and e are aligned to 16 bytes.
template <typename T, bool VEC>
__device__ inline void load8(const void* row, int64_t at, float* x) {
    if (VEC) {
        constexpr int V = sizeof(T) == 4 ? 4 : 8;
#pragma unroll
        for (int i = 0; i < 8; i += V) {
            const auto v = load_pack<T, V>(row, at + i);
#pragma unroll
            for (int k = 0; k < V; ++k) x[i + k] = (float)v.e[k];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)static_cast<const T*>(row)[at + i];
    }
}

template <typename T, bool VEC>
__device__ inline void store8(void* row, int64_t at, const float* x) {
    if (VEC) {
        constexpr int V = sizeof(T) == 4 ? 4 : 8;
#pragma unroll
        for (int i = 0; i < 8; i += V) {
            Pack<T, V> v;
#pragma unroll
            for (int k = 0; k < V; ++k) v.e[k] = (T)x[i + k];
            store_pack<T, V>(row, at + i, v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) static_cast<T*>(row)[at + i] = (T)x[i];
    }
}

// ---- append --------------------------------------------------------------------------------
struct KvqAppendP {
    ls_kvq_cache c;
    ls_append_args a;
    int q_pairs;  // units of a query head that turn, 1 or (vectors) 8 pairs each, 4 of neighbours
    int q_units;  // those and what is copied, an element or eight
    int quads;    // lanes of a head in the cache: four to a group of 32
    int q_total;  // lanes for the queries, a multiple of four
    int total;
    int most;     // largest scale byte
};

// Elements e .. e + 7 of a head turned to their position.  VEC: whole vectors of them turn or do not, with partners
// in one vector; otherwise element by element.
template <typename T, bool VEC, bool PAIR>
__device__ inline void turned8(const ls_append_args& a, const float* cs, const void* src, int64_t from, int e, float* x) {
    load8<T, VEC>(src, from + e, x);
    const int half = a.rot_dim / 2;
    if (e >= a.rot_dim) return;
    if (PAIR) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            if (!VEC && e + i >= a.rot_dim) break;
            const float co = cs[(e + i) / 2], si = cs[half + (e + i) / 2], l = x[i], m = x[i + 1];
            x[i] = l * co - m * si;
            x[i + 1] = m * co + l * si;
        }
    } else if (VEC) {
        const bool second = e >= half;
        float y[8], co[8], si[8];
        load8<T, true>(src, from + (second ? e - half : e + half), y);
        load8<float, true>(cs, second ? e - half : e, co);
        load8<float, true>(cs, second ? e : e + half, si);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = second ? x[i] * co[i] + y[i] * si[i] : x[i] * co[i] - y[i] * si[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = e + i;
            if (k >= a.rot_dim) break;
            const bool second = k >= half;
            const float y = (float)static_cast<const T*>(src)[from + (second ? k - half : k + half)];
            const float co = cs[second ? k - half : k], si = cs[second ? k : k + half];
            x[i] = second ? x[i] * co + y * si : x[i] * co - y * si;
        }
    }
}

// Unit u of a query head: both elements of its pairs, as the output may lie where the input does.
template <typename T, bool VEC, bool PAIR>
__device__ inline void turn_query(const KvqAppendP& p, const float* cs, int64_t from, int64_t to, int u) {
    const ls_append_args& a = p.a;
    const int half = a.rot_dim / 2;
    float x[8], y[8], co[8], si[8];
    if (u >= p.q_pairs) {
        const int e = a.rot_dim + (u - p.q_pairs) * (VEC ? 8 : 1);
        if (VEC) {
            load8<T, true>(a.q, from + e, x);
            store8<T, true>(a.q_out, to + e, x);
        } else {
            static_cast<T*>(a.q_out)[to + e] = static_cast<const T*>(a.q)[from + e];
        }
    } else if (VEC && PAIR) {
        turned8<T, true, true>(a, cs, a.q, from, u * 8, x);
        store8<T, true>(a.q_out, to + u * 8, x);
    } else if (VEC) {
        const int e = u * 8;
        load8<T, true>(a.q, from + e, x);
        load8<T, true>(a.q, from + half + e, y);
        load8<float, true>(cs, e, co);
        load8<float, true>(cs, half + e, si);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float l = x[i], m = y[i];
            x[i] = l * co[i] - m * si[i];
            y[i] = m * co[i] + l * si[i];
        }
        store8<T, true>(a.q_out, to + e, x);
        store8<T, true>(a.q_out, to + half + e, y);
    } else {
        const int i = PAIR ? 2 * u : u, j = PAIR ? 2 * u + 1 : u + half;
        const float l = (float)static_cast<const T*>(a.q)[from + i], m = (float)static_cast<const T*>(a.q)[from + j];
        const float c = cs[u], s = cs[half + u];
        static_cast<T*>(a.q_out)[to + i] = (T)(l * c - m * s);
        static_cast<T*>(a.q_out)[to + j] = (T)(m * c + l * s);
    }
}

template <int CTRL>
__device__ inline uint32_t max_quad(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return v > o ? v : o;
}

// A lane takes eight pairs of a query head, or eight elements of a key or value, which it
// quantises with the other three lanes of their group: one read of the data, the largest magnitude over four
// lanes, one conversion.  blockIdx.x is the token, blockIdx.y 256 of its lanes.
template <typename T, class C, bool VEC, bool PAIR>
__global__ __launch_bounds__(256) void kvq_append_kernel(const KvqAppendP p) {
    const ls_append_args& a = p.a;
    const ls_kvq_cache& c = p.c;
    const int64_t t = blockIdx.x;
    int pos = 0;
    if (a.rot_dim) {
        pos = a.positions[t];
        if (pos < 0 || pos >= a.n_pos) return;
    }
    const int slot = a.slots[t];
    const bool keep = slot >= 0 && slot < c.n_pages * c.page_size;
    const int64_t page = keep ? slot / c.page_size : 0, place = keep ? slot % c.page_size : 0;
    const float* cs = a.cos_sin + (int64_t)pos * a.rot_dim;
    const int total = keep ? p.total : p.q_total;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < total; i += 256 * gridDim.y) {
        if (i < p.q_total) {
            const int h = i / p.q_units;
            if (h < a.n_heads)
                turn_query<T, VEC, PAIR>(p, cs, t * a.q_token_stride + h * a.q_head_stride,
                                         t * a.q_out_token_stride + h * a.q_out_head_stride, i - h * p.q_units);
            continue;
        }
        const int j = i - p.q_total, row = j / p.quads, e = (j - row * p.quads) * 8;
        const bool value = row >= c.n_kv_heads;
        const int h = value ? row - c.n_kv_heads : row;
        float x[8] = {};
        if (e < c.head_dim) {
            if (value)
                load8<T, VEC>(a.v, t * a.v_token_stride + h * a.v_head_stride + e, x);
            else
                turned8<T, VEC, PAIR>(a, cs, a.k, t * a.k_token_stride + h * a.k_head_stride, e, x);
        }
        // magnitudes compare as their bits do, infinities and NaN above every number
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
        top = max_quad<0xb1>(top);  // quad_perm [1,0,3,2]
        top = max_quad<0x4e>(top);  // quad_perm [2,3,0,1]
        const bool fine = top < 0x7f800000u;
        const uint32_t byte = fine ? (uint32_t)min(max((int)((top + C::kCarry) >> 23) - C::kBelow, 1), p.most) : 255u;
        uint32_t w[C::kBits / 4] = {};
        if (fine) narrow8<C>(x, scale_of(byte), w);
        if (e < c.head_dim) {
            uint8_t* to = static_cast<uint8_t*>(value ? c.v : c.k) + page * c.page_stride + place * c.token_stride + h * c.head_stride +
                          e * C::kBits / 8;
            if constexpr (C::kBits == 4)
                *reinterpret_cast<uint32_t*>(to) = w[0];
            else
                *reinterpret_cast<u32x2a*>(to) = u32x2a{w[0], w[1]};
            if (e % kGroup == 0)
                (value ? c.v_scale : c.k_scale)[page * c.scale_page_stride + place * c.scale_token_stride + h * c.scale_head_stride + e / kGroup] =
                    (uint8_t)byte;
        }
    }
}

template <typename T, class C>
hipError_t kvq_append_type(const ls_kvq_cache& c, const ls_append_args& a, hipStream_t st) {
    KvqAppendP p{c, a, 0, 0, 0, 0, 0, 0};
    p.quads = (int)ceil_div(c.head_dim, kGroup) * 4;
    p.most = 127 + (std::is_same_v<T, _Float16> ? C::kMostExp16 : C::kMostExp);
    const bool pair = a.style == LS_ROPE_PAIR;
    const int64_t el = 16 / (int64_t)sizeof(T);
    bool vec = a.rot_dim % (pair ? 8 : 16) == 0 && (!a.rot_dim || aligned(a.cos_sin, 16));
    for (int64_t s : {a.k_token_stride, a.k_head_stride, a.v_token_stride, a.v_head_stride, a.q_token_stride, a.q_head_stride,
                      a.q_out_token_stride, a.q_out_head_stride})
        vec = vec && s % el == 0;
    for (const void* q : {a.k, a.v, a.q, (const void*)a.q_out}) vec = vec && aligned(q, 16);
    p.q_pairs = vec ? a.rot_dim / (pair ? 8 : 16) : a.rot_dim / 2;
    p.q_units = p.q_pairs + (c.head_dim - a.rot_dim) / (vec ? 8 : 1);
    p.q_total = (int)round_up((size_t)a.n_heads * p.q_units, 4);
    p.total = p.q_total + 2 * c.n_kv_heads * p.quads;
    const dim3 grid(a.n_tokens, (unsigned)std::min<int64_t>(ceil_div(p.total, 256), 65535));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, p);
        return hipGetLastError();
    };
    if (pair) return vec ? go(kvq_append_kernel<T, C, true, true>) : go(kvq_append_kernel<T, C, false, true>);
    return vec ? go(kvq_append_kernel<T, C, true, false>) : go(kvq_append_kernel<T, C, false, false>);
}

// ---- read ----------------------------------------------------------------------------------
struct KvqReadP {
    ls_kvq_cache c;
    ls_kvq_read_args a;
    int units;  // eights of a head
};

// A lane widens eight elements; blockIdx.x is the token, blockIdx.y 256 of its eights, keys before values.
template <typename T, class C, bool VEC>
__global__ __launch_bounds__(256) void kvq_read_kernel(const KvqReadP p) {
    const ls_kvq_read_args& a = p.a;
    const ls_kvq_cache& c = p.c;
    const int64_t t = blockIdx.x;
    const int slot = a.slots[t];
    if (slot < 0 || slot >= c.n_pages * c.page_size) return;
    const int64_t page = slot / c.page_size, place = slot % c.page_size;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < 2 * c.n_kv_heads * p.units; i += 256 * gridDim.y) {
        const int row = i / p.units, e = (i - row * p.units) * 8;
        const bool value = row >= c.n_kv_heads;
        const int h = value ? row - c.n_kv_heads : row;
        const uint8_t* from = static_cast<const uint8_t*>(value ? c.v : c.k) + page * c.page_stride + place * c.token_stride +
                              h * c.head_stride + e * C::kBits / 8;
        const uint32_t byte = (value ? c.v_scale : c.k_scale)[page * c.scale_page_stride + place * c.scale_token_stride +
                                                              h * c.scale_head_stride + e / kGroup];
        uint32_t w[2];
        if constexpr (C::kBits == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(from);
        } else {
            const u32x2a v = *reinterpret_cast<const u32x2a*>(from);
            w[0] = v[0], w[1] = v[1];
        }
        float x[1][8];
        widen8<C, float>(w, scale_of(byte), x);
        store8<T, VEC>(value ? a.v : a.k, value ? t * a.v_token_stride + h * a.v_head_stride + e : t * a.k_token_stride + h * a.k_head_stride + e,
                       x[0]);
    }
}

template <typename T, class C>
hipError_t kvq_read_type(const ls_kvq_cache& c, const ls_kvq_read_args& a, hipStream_t st) {
    const KvqReadP p{c, a, c.head_dim / 8};
    const int64_t el = 16 / (int64_t)sizeof(T);
    bool vec = aligned(a.k, 16) && aligned(a.v, 16);
    for (int64_t s : {a.k_token_stride, a.k_head_stride, a.v_token_stride, a.v_head_stride}) vec = vec && s % el == 0;
    const dim3 grid(a.n_tokens, (unsigned)std::min<int64_t>(ceil_div(2 * c.n_kv_heads * p.units, 256), 65535));
    if (vec)
        hipLaunchKernelGGL((kvq_read_kernel<T, C, true>), grid, dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((kvq_read_kernel<T, C, false>), grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

template <class C>
hipError_t kvq_append_code(const ls_kvq_cache& c, ls_dtype type, const ls_append_args& a, hipStream_t st) {
    return type == LS_F32   ? kvq_append_type<float, C>(c, a, st)
           : type == LS_F16 ? kvq_append_type<_Float16, C>(c, a, st)
                            : kvq_append_type<__bf16, C>(c, a, st);
}
template <class C>
hipError_t kvq_read_code(const ls_kvq_cache& c, const ls_kvq_read_args& a, hipStream_t st) {
    return a.type == LS_F32   ? kvq_read_type<float, C>(c, a, st)
           : a.type == LS_F16 ? kvq_read_type<_Float16, C>(c, a, st)
                              : kvq_read_type<__bf16, C>(c, a, st);
}

// A launch holds fewer than 2^32 threads along x: calls of more tokens than this, a workgroup of 256 for each, are cut.
constexpr int kTokensPerLaunch = 1 << 21;

}  // namespace

hipError_t launch_kvq_append(const ls_kvq_cache& c, ls_dtype type, const ls_append_args& a, hipStream_t st) {
    for (int64_t t = 0; t < a.n_tokens; t += kTokensPerLaunch) {
        ls_append_args b = a;
        const int64_t es = (int64_t)type_size(type);
        auto skip = [&](const void* p, int64_t stride) { return p ? static_cast<const char*>(p) + t * stride * es : nullptr; };
        b.n_tokens = (int32_t)std::min<int64_t>(kTokensPerLaunch, a.n_tokens - t);
        b.k = skip(a.k, a.k_token_stride);
        b.v = skip(a.v, a.v_token_stride);
        b.q = skip(a.q, a.q_token_stride);
        b.q_out = const_cast<char*>(skip(a.q_out, a.q_out_token_stride));
        if (b.positions) b.positions += t;
        b.slots += t;
        const hipError_t e = c.code == LS_FP4 ? kvq_append_code<Fp4>(c, type, b, st) : kvq_append_code<Fp8>(c, type, b, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_kvq_read(const ls_kvq_cache& c, const ls_kvq_read_args& a, hipStream_t st) {
    for (int64_t t = 0; t < a.n_tokens; t += kTokensPerLaunch) {
        ls_kvq_read_args b = a;
        const int64_t es = (int64_t)type_size(a.type);
        b.n_tokens = (int32_t)std::min<int64_t>(kTokensPerLaunch, a.n_tokens - t);
        b.k = static_cast<char*>(a.k) + t * a.k_token_stride * es;
        b.v = static_cast<char*>(a.v) + t * a.v_token_stride * es;
        b.slots += t;
        const hipError_t e = c.code == LS_FP4 ? kvq_read_code<Fp4>(c, b, st) : kvq_read_code<Fp8>(c, b, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ls

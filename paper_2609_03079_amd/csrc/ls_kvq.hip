// ls_kvq.hip - a paged cache of keys and values in 4 or 8 bits: written (the keys, and queries beside them,
// turned to their positions on the way) and read back.
//
//   top = max |x_i| of 32;  2^e the smallest power of two with top < 7 * 2^e (4 bits) or 464 * 2^e (8);  code_i = x_i / 2^e, rounded
//
// Bound by memory: every element is read and written once.  8192 tokens of 64 + 2 x 8 heads of 128 are written in 49 us (bf16 to FP4,
// 6.3 TB/s), 32768 of 8 heads read in 29 (FP8 to bf16, 6.9 TB/s).  Single tokens take 3.7 and 2.1 us, three dependent loads and one.  (Medians
// of 30 launches.)  Where not all of a call comes in vectors of 16 bytes whose partners do too (a half-style turn of 40 of 80
// elements, of 56 of 112) it goes element by element: 4096 tokens of 10 + 2 x 5 heads of 80 written and read take 31 us, not 18, of
// 16 + 2 x 16 heads of 112 60, not 29.
#include <algorithm>

#include "ls_codes.h"
#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {
namespace {

// Calls with more data than this pass the caches by and leave a page's tokens to one die: writing 8192 tokens (64 query
// heads, 8 key heads of 128, FP4) took 73 us and takes 48, of which 15 by loads and stores that are not kept, 5 by lanes of four
// heads; reading 32768 tokens of 8 heads (FP8) 51 and 30 (tokens by two 4, stores 15, one die for a page 3).  At the border 512
// tokens written and read, 20 buffers in turn, take 12.9 and 10.7, 1024 read 8.8 and 6.1, and 512 read from one buffer 5.1 and 4.7.
// What a die's L2 kept would be no nearer to the next kernel, which runs on all eight.
constexpr int64_t kStreamBytes = 4 << 20;

// Block b of n, such that runs of 64 are on one die (they take blocks in turn): tokens of a page share cache lines.
__device__ inline int64_t in_runs(uint32_t b, uint32_t n) {
    const uint32_t first = b / 512 * 512, k = b - first;
    return first + 512 <= n ? first + k % 8 * 64 + k / 8 : b;
}

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

// 16 bytes that the caches need not keep.
typedef uint32_t u32x4n __attribute__((ext_vector_type(4)));
template <typename T, int V>
__device__ inline Pack<T, V> load_nt(const void* p, int64_t elem) {
    return __builtin_bit_cast(Pack<T, V>, __builtin_nontemporal_load(reinterpret_cast<const u32x4n*>(static_cast<const T*>(p) + elem)));
}
template <typename T, int V>
__device__ inline void store_nt(void* p, int64_t elem, const Pack<T, V>& v) {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4n, v), reinterpret_cast<u32x4n*>(static_cast<T*>(p) + elem));
}

// STREAM: past the caches.
template <typename T, bool VEC, bool STREAM = false>
__device__ inline void store8(void* row, int64_t at, const float* x) {
    if (VEC) {
        constexpr int V = sizeof(T) == 4 ? 4 : 8;
#pragma unroll
        for (int i = 0; i < 8; i += V) {
            Pack<T, V> v;
#pragma unroll
            for (int k = 0; k < V; ++k) v.e[k] = (T)x[i + k];
            if (STREAM)
                store_nt<T, V>(row, at + i, v);
            else
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
    int q_by;     // query heads, or a fourth of them: those that one lane takes are so far apart
    int q_total;  // lanes for the queries, a multiple of four
    int total;
    int most;     // largest scale byte
};

// x turned by its partner y, c and s cosine and sine (minus it for a pair's first half).  One product is rounded, the sum is in
// fp32 and then in T, in every kernel, so that no bit depends on how many tokens or what strides a call has: without the empty
// asm some kernels would round the sum to float16 at once.
__device__ inline float turn(float x, float y, float c, float s) {
    float r = __builtin_fmaf(y, s, x * c);
    asm("" : "+v"(r));
    return r;
}

// The same for a key, which is rounded but once, to its code: the products are exact in 64 bits, their sum is off by 2^-53, and
// what is inexact in fp32 is rounded to odd there, so that it lies on the side of every border between two codes or
// scales that it was on.  (In fp32 a few of 8 million elements fall to the other side; time: nothing, the data's reading hides it.)
// A finite key beyond fp32 becomes its largest number, which is odd, and with it the largest code of the largest scale.
__device__ inline float turn_key(float x, float y, float c, float s) {
    const double d = __builtin_fma((double)y, (double)s, (double)x * (double)c);
    const float f = (float)d;
    const uint32_t toward_zero = __float_as_uint(f) - (__builtin_fabs((double)f) > __builtin_fabs(d) ? 1u : 0u);
    return (double)f == d || d != d ? f : __uint_as_float(toward_zero | 1u);
}

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
            x[i] = turn_key(l, m, co, -si);
            x[i + 1] = turn_key(m, l, co, si);
        }
    } else if (VEC) {
        const bool second = e >= half;
        float y[8], co[8], si[8];
        load8<T, true>(src, from + (second ? e - half : e + half), y);
        load8<float, true>(cs, second ? e - half : e, co);
        load8<float, true>(cs, second ? e : e + half, si);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = turn_key(x[i], y[i], co[i], second ? si[i] : -si[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = e + i;
            if (k >= a.rot_dim) break;
            const bool second = k >= half;
            const float y = (float)static_cast<const T*>(src)[from + (second ? k - half : k + half)];
            const float co = cs[second ? k - half : k], si = cs[second ? k : k + half];
            x[i] = turn_key(x[i], y, co, second ? si : -si);
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
        const auto c4 = load_pack<float, 4>(cs, u * 4), s4 = load_pack<float, 4>(cs, half + u * 4);
        load8<T, true>(a.q, from + u * 8, x);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float l = x[i], m = x[i + 1];
            x[i] = turn(l, m, c4.e[i / 2], -s4.e[i / 2]);
            x[i + 1] = turn(m, l, c4.e[i / 2], s4.e[i / 2]);
        }
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
            x[i] = turn(l, m, co[i], -si[i]);
            y[i] = turn(m, l, co[i], si[i]);
        }
        store8<T, true>(a.q_out, to + e, x);
        store8<T, true>(a.q_out, to + half + e, y);
    } else {
        const int i = PAIR ? 2 * u : u, j = PAIR ? 2 * u + 1 : u + half;
        const float l = (float)static_cast<const T*>(a.q)[from + i], m = (float)static_cast<const T*>(a.q)[from + j];
        const float c = cs[u], s = cs[half + u];
        static_cast<T*>(a.q_out)[to + i] = (T)turn(l, m, c, -s);
        static_cast<T*>(a.q_out)[to + j] = (T)turn(m, l, c, s);
    }
}

// The same of heads h, h + by, h + 2 by and h + 3 by, in vectors: all loads first, and one of the table.
constexpr int kHeads = 4;
template <typename T, bool PAIR>
__device__ inline void turn_queries(const KvqAppendP& p, const float* cs, int64_t from, int64_t to, int h, int u) {
    const ls_append_args& a = p.a;
    constexpr int V = sizeof(T) == 4 ? 4 : 8, N = 8 / V;
    const int half = a.rot_dim / 2;
    const bool turns = u < p.q_pairs, second = !PAIR && turns;
    const int e = turns ? u * 8 : a.rot_dim + (u - p.q_pairs) * 8;
    Pack<T, V> x[kHeads][N], y[kHeads][N];
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
        if (h + g * p.q_by >= a.n_heads) break;
        const int64_t at = from + (h + g * p.q_by) * a.q_head_stride + e;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            x[g][n] = load_nt<T, V>(a.q, at + n * V);
            if (second) y[g][n] = load_nt<T, V>(a.q, at + half + n * V);
        }
    }
    float co[8], si[8];
    if (turns && PAIR) {
        const auto c4 = load_pack<float, 4>(cs, u * 4), s4 = load_pack<float, 4>(cs, half + u * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) co[i] = c4.e[i], si[i] = s4.e[i];
    } else if (turns) {
        load8<float, true>(cs, e, co);
        load8<float, true>(cs, half + e, si);
    }
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
        if (h + g * p.q_by >= a.n_heads) break;
        const int64_t at = to + (h + g * p.q_by) * a.q_out_head_stride + e;
        if (turns) {
#pragma unroll
            for (int i = 0; i < (PAIR ? 4 : 8); ++i) {
                T& l = PAIR ? x[g][2 * i / V].e[2 * i % V] : x[g][i / V].e[i % V];
                T& m = PAIR ? x[g][2 * i / V].e[2 * i % V + 1] : y[g][i / V].e[i % V];
                const float lf = (float)l, mf = (float)m;
                l = (T)turn(lf, mf, co[i], -si[i]);
                m = (T)turn(mf, lf, co[i], si[i]);
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            store_nt<T, V>(a.q_out, at + n * V, x[g][n]);
            if (second) store_nt<T, V>(a.q_out, at + half + n * V, y[g][n]);
        }
    }
}

template <int CTRL>
__device__ inline uint32_t max_quad(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return v > o ? v : o;
}

// Eight elements from e of a key or value are quantised with those of the other three lanes of their group and written.
template <class C>
__device__ inline void put8(const KvqAppendP& p, bool value, int64_t page, int64_t place, int h, int e, const float* x) {
    const ls_kvq_cache& c = p.c;
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
    if (e >= c.head_dim) return;
    uint8_t* to = static_cast<uint8_t*>(value ? c.v : c.k) + page * c.page_stride + place * c.token_stride + h * c.head_stride + e * C::kBits / 8;
    if constexpr (C::kBits == 4)
        *reinterpret_cast<uint32_t*>(to) = w[0];
    else
        *reinterpret_cast<u32x2a*>(to) = u32x2a{w[0], w[1]};
    if (e % kGroup == 0)
        (value ? c.v_scale : c.k_scale)[page * c.scale_page_stride + place * c.scale_token_stride + h * c.scale_head_stride + e / kGroup] =
            (uint8_t)byte;
}

// A lane takes eight pairs of a query head, or eight elements of a key or value.  STREAM: of four query heads, or
// of a key and its value.  blockIdx.x is the token, blockIdx.y 256 of its lanes.
template <typename T, class C, bool VEC, bool PAIR, bool STREAM>
__global__ __launch_bounds__(256) void kvq_append_kernel(const KvqAppendP p) {
    const ls_append_args& a = p.a;
    const ls_kvq_cache& c = p.c;
    const int64_t t = STREAM ? in_runs(blockIdx.x, gridDim.x) : blockIdx.x;
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
            const int h = i / p.q_units, u = i - h * p.q_units;
            if (h >= p.q_by) continue;
            if constexpr (STREAM)
                turn_queries<T, PAIR>(p, cs, t * a.q_token_stride, t * a.q_out_token_stride, h, u);
            else
                turn_query<T, VEC, PAIR>(p, cs, t * a.q_token_stride + h * a.q_head_stride, t * a.q_out_token_stride + h * a.q_out_head_stride, u);
            continue;
        }
        const int j = i - p.q_total, row = j / p.quads, e = (j - row * p.quads) * 8;
        const bool value = !STREAM && row >= c.n_kv_heads;
        const int h = value ? row - c.n_kv_heads : row;
        float x[8] = {}, y[8] = {};
        if (e < c.head_dim) {
            if (value || STREAM) load8<T, VEC>(a.v, t * a.v_token_stride + h * a.v_head_stride + e, value ? x : y);
            if (!value) turned8<T, VEC, PAIR>(a, cs, a.k, t * a.k_token_stride + h * a.k_head_stride, e, x);
        }
        put8<C>(p, value, page, place, h, e, x);
        if (STREAM) put8<C>(p, true, page, place, h, e, y);
    }
}

template <typename T, class C>
hipError_t kvq_append_type(const ls_kvq_cache& c, const ls_append_args& a, hipStream_t st) {
    KvqAppendP p{c, a, 0, 0, 0, 0, 0, 0, 0};
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
    const int64_t bytes = (int64_t)a.n_tokens * c.head_dim * (a.n_heads + 2 * c.n_kv_heads) * (int64_t)sizeof(T);
    const bool stream = vec && bytes > kStreamBytes;
    p.q_by = stream ? (int)ceil_div(a.n_heads, kHeads) : a.n_heads;
    p.q_total = (int)round_up((size_t)p.q_by * p.q_units, 4);
    p.total = p.q_total + (stream ? 1 : 2) * c.n_kv_heads * p.quads;
    const dim3 grid(a.n_tokens, (unsigned)std::min<int64_t>(ceil_div(p.total, 256), 65535));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, p);
        return hipGetLastError();
    };
    if (stream) return pair ? go(kvq_append_kernel<T, C, true, true, true>) : go(kvq_append_kernel<T, C, true, false, true>);
    if (pair) return vec ? go(kvq_append_kernel<T, C, true, true, false>) : go(kvq_append_kernel<T, C, false, true, false>);
    return vec ? go(kvq_append_kernel<T, C, true, false, false>) : go(kvq_append_kernel<T, C, false, false, false>);
}

// ---- read ----------------------------------------------------------------------------------
struct KvqReadP {
    ls_kvq_cache c;
    ls_kvq_read_args a;
    int units;  // eights of a head
};

// A lane widens eight elements, STREAM: of two tokens, with their loads in flight together.  blockIdx.x is the token or two,
// blockIdx.y 256 of a token's eights, keys before values.
template <typename T, class C, bool VEC, bool STREAM>
__global__ __launch_bounds__(256) void kvq_read_kernel(const KvqReadP p) {
    const ls_kvq_read_args& a = p.a;
    const ls_kvq_cache& c = p.c;
    constexpr int TOKENS = STREAM ? 2 : 1;
    const int64_t t0 = (STREAM ? in_runs(blockIdx.x, gridDim.x) : blockIdx.x) * TOKENS;
    int slot[TOKENS];
#pragma unroll
    for (int n = 0; n < TOKENS; ++n) slot[n] = t0 + n < a.n_tokens ? a.slots[t0 + n] : -1;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < 2 * c.n_kv_heads * p.units; i += 256 * gridDim.y) {
        const int row = i / p.units, e = (i - row * p.units) * 8;
        const bool value = row >= c.n_kv_heads;
        const int h = value ? row - c.n_kv_heads : row;
        const uint8_t* codes = static_cast<const uint8_t*>(value ? c.v : c.k) + h * c.head_stride + e * C::kBits / 8;
        const uint8_t* scales = (value ? c.v_scale : c.k_scale) + h * c.scale_head_stride + e / kGroup;
        void* to = value ? a.v : a.k;
        const int64_t at = value ? h * a.v_head_stride + e : h * a.k_head_stride + e, by = value ? a.v_token_stride : a.k_token_stride;
        uint32_t w[TOKENS][2];
        uint8_t byte[TOKENS];
#pragma unroll
        for (int n = 0; n < TOKENS; ++n) {
            if (slot[n] < 0 || slot[n] >= c.n_pages * c.page_size) continue;
            const int64_t page = slot[n] / c.page_size, place = slot[n] % c.page_size;
            const uint8_t* from = codes + page * c.page_stride + place * c.token_stride;
            byte[n] = scales[page * c.scale_page_stride + place * c.scale_token_stride];
            if constexpr (C::kBits == 4) {
                w[n][0] = *reinterpret_cast<const uint32_t*>(from);
            } else {
                const u32x2a v = *reinterpret_cast<const u32x2a*>(from);
                w[n][0] = v[0], w[n][1] = v[1];
            }
        }
#pragma unroll
        for (int n = 0; n < TOKENS; ++n) {
            if (slot[n] < 0 || slot[n] >= c.n_pages * c.page_size) continue;
            float x[1][8];
            widen8<C, float>(w[n], scale_of(byte[n]), x);
            store8<T, VEC, STREAM>(to, at + (t0 + n) * by, x[0]);
        }
    }
}

template <typename T, class C>
hipError_t kvq_read_type(const ls_kvq_cache& c, const ls_kvq_read_args& a, hipStream_t st) {
    const KvqReadP p{c, a, c.head_dim / 8};
    const int64_t el = 16 / (int64_t)sizeof(T);
    bool vec = aligned(a.k, 16) && aligned(a.v, 16);
    for (int64_t s : {a.k_token_stride, a.k_head_stride, a.v_token_stride, a.v_head_stride}) vec = vec && s % el == 0;
    const unsigned y = (unsigned)std::min<int64_t>(ceil_div(2 * c.n_kv_heads * p.units, 256), 65535);
    const int64_t bytes = (int64_t)a.n_tokens * 2 * c.n_kv_heads * c.head_dim * (int64_t)sizeof(T);
    auto go = [&](auto kernel, int tokens) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(a.n_tokens, tokens), y), dim3(256), 0, st, p);
        return hipGetLastError();
    };
    if (vec && bytes > kStreamBytes) return go(kvq_read_kernel<T, C, true, true>, 2);
    return vec ? go(kvq_read_kernel<T, C, true, false>, 1) : go(kvq_read_kernel<T, C, false, false>, 1);
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

// ls_linear.hip - matrix products in 8-bit integers with a scale for each token and channel:
// out[t, n] = s_t w_scale[n] sum_k q[t, k] w[n, k] + bias[n].
//
// Both operands are contiguous in k, which is what the integer matrix instructions take: a lane
// holds 16 consecutive bytes of a row of w and of a row of q.  Sums are exact (32-bit integers,
// |sum| < 2^31 for k < 2^17), so neither the order of the sum nor the kernel chosen changes a bit
// of the result; the two scales and the bias are applied once, in fp32.
#include <algorithm>

#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(1))) void* gptr;
typedef __attribute__((address_space(3))) void* lptr;

// What a chunk past the end of a row is read from.
__device__ const uint32_t g_zero_chunk[4] = {0, 0, 0, 0};

struct LinearP {
    const int8_t* q;  // [T, k] quantised tokens
    int64_t q_stride;
    const float* s;   // [T]
    const int8_t* w;
    int64_t w_stride;
    const float* w_scale;
    const float* bias;
    void* out;
    int64_t out_stride;
    int T, k, n;
};

template <typename O>
__device__ inline void put(const LinearP& p, int t, int n, int acc, float s) {
    float v = (float)acc * s * p.w_scale[n];
    if (p.bias) v += p.bias[n];
    static_cast<O*>(p.out)[(int64_t)t * p.out_stride + n] = (O)v;
}

// ---- quantisation --------------------------------------------------------------------------
// |x| as ordered integers: an infinity is 0x7f800000, a NaN above it.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ inline uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int off = 32; off; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off, 64));
    return m;
}

// The scale of a token from its largest magnitude, and what its elements are divided by (0: all zero).
__device__ inline float token_scale(uint32_t m, float* top) {
    if (m >= 0x7f800000u) {
        *top = 0.f;
        return __uint_as_float(0x7fc00000u);
    }
    const float s = __uint_as_float(m) / 127.f;
    const bool none = s < 1.17549435e-38f;
    *top = none ? 0.f : __uint_as_float(m);
    return none ? 0.f : s;
}

// 127 x / max with one rounding of the quotient: for 16-bit x the product is exact, so this is
// the definition's value (multiplying by a rounded 127 / max could move a tie).
__device__ inline int quantise(float x, float top) {
    return top > 0.f ? (int)rintf(x * 127.f / top) : 0;
}

// One workgroup per token; 16 elements per thread and step.
template <typename T>
__global__ __launch_bounds__(256) void quantise_kernel(const void* x, int64_t x_stride, int k, int8_t* q, float* s) {
    __shared__ uint32_t part[4];
    const int64_t t = blockIdx.x;
    const T* row = static_cast<const T*>(x) + t * x_stride;
    constexpr int kHeld = 4;  // vectors a thread keeps in registers (rows of up to 16384 elements)
    Pack<T, 16> v[kHeld];
    uint32_t m = 0;
    const int step = 256 * 16;
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
        const int e = (int)threadIdx.x * 16 + c * step;
        if (e < k) {
            v[c] = load_pack<T, 16>(row, e);
#pragma unroll
            for (int i = 0; i < 16; ++i) m = max(m, magnitude((float)v[c].e[i]));
        }
    }
    for (int e = (int)threadIdx.x * 16 + kHeld * step; e < k; e += step) {
        const auto u = load_pack<T, 16>(row, e);
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, magnitude((float)u.e[i]));
    }
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(part[0], part[1]), max(part[2], part[3]));
    float top;
    const float scale = token_scale(m, &top);
    if (threadIdx.x == 0) s[t] = scale;
    auto write = [&](int e, const Pack<T, 16>& u) {
        Pack<int8_t, 16> o;
#pragma unroll
        for (int i = 0; i < 16; ++i) o.e[i] = (int8_t)quantise((float)u.e[i], top);
        store_pack<int8_t, 16>(q, t * k + e, o);
    };
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
        const int e = (int)threadIdx.x * 16 + c * step;
        if (e < k) write(e, v[c]);
    }
    for (int e = (int)threadIdx.x * 16 + kHeld * step; e < k; e += step) write(e, load_pack<T, 16>(row, e));
}

// ---- tiles through shared memory -----------------------------------------------------------
// out tile of BM tokens by BN channels; WM x WN waves, each with a (BM / WM) x (BN / WN) part in
// 32 x 32 matrix tiles.  Both operands come in 128-byte slices of k, copied straight to shared
// memory two slices deep: slice i + 1 arrives while slice i is multiplied.  A row's eight 16-byte
// chunks lie at places permuted by its number, so that the 16 rows a read touches together lie in
// different banks.
constexpr int kSlice = 128;

__device__ inline int place(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

template <int ROWS, int WAVES>
__device__ inline void fetch(const int8_t* base, int64_t stride, int row0, int rows, int k, int k0, int8_t* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    static_assert(ROWS % (8 * WAVES) == 0, "whole instructions");
#pragma unroll
    for (int i = 0; i < ROWS / (8 * WAVES); ++i) {
        const int r0 = (i * WAVES + wave) * 8, r = r0 + (lane >> 3);
        const int at = k0 + place(r, lane & 7) * 16;
        const int8_t* src = base + (int64_t)min(row0 + r, rows - 1) * stride + at;
        if (at >= k) src = reinterpret_cast<const int8_t*>(g_zero_chunk);
        __builtin_amdgcn_global_load_lds((gptr)src, (lptr)(lds + r0 * kSlice), 16, 0, 0);
    }
}

template <int BM, int BN, int WM, int WN>
struct Tile {
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32, kWaves = WM * WN;
    i32x16 acc[TM][TN];

    __device__ inline void multiply(const int8_t* a, const int8_t* b) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
        const int m0 = (wave / WN) * (BM / WM), n0 = (wave % WN) * (BN / WN);
#pragma unroll
        for (int kk = 0; kk < kSlice / 32; ++kk) {
            i32x4 x[TM], y[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i)
                x[i] = *reinterpret_cast<const i32x4*>(a + (m0 + i * 32 + r) * kSlice + place(r, kk * 2 + h) * 16);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                y[j] = *reinterpret_cast<const i32x4*>(b + (n0 + j * 32 + r) * kSlice + place(r, kk * 2 + h) * 16);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[i], y[j], acc[i][j], 0, 0, 0);
        }
    }
};

__device__ inline void arrive() {
    __builtin_amdgcn_s_waitcnt(0x0070);  // this wave's copies have landed, its reads are done
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

template <typename O, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void tile_kernel(const LinearP p, int tiles_n) {
    // four arrays, not one: a read of one slice must not wait for the copy into the other
    __shared__ __attribute__((aligned(16))) int8_t a0[BM * kSlice];
    __shared__ __attribute__((aligned(16))) int8_t a1[BM * kSlice];
    __shared__ __attribute__((aligned(16))) int8_t b0[BN * kSlice];
    __shared__ __attribute__((aligned(16))) int8_t b1[BN * kSlice];
    const int t0 = (blockIdx.x / tiles_n) * BM, n0 = (blockIdx.x % tiles_n) * BN;
    Tile<BM, BN, WM, WN> tile;
#pragma unroll
    for (auto& r : tile.acc)
        for (auto& v : r) v = i32x16{};
    constexpr int W = WM * WN;
    auto copy = [&](int k0, int8_t* a, int8_t* b) {
        fetch<BM, W>(p.q, p.q_stride, t0, p.T, p.k, k0, a);
        fetch<BN, W>(p.w, p.w_stride, n0, p.n, p.k, k0, b);
    };
    copy(0, a0, b0);
    for (int k0 = 0; k0 < p.k; k0 += 2 * kSlice) {
        arrive();
        if (k0 + kSlice < p.k) copy(k0 + kSlice, a1, b1);
        tile.multiply(a0, b0);
        if (k0 + kSlice >= p.k) break;
        arrive();
        if (k0 + 2 * kSlice < p.k) copy(k0 + 2 * kSlice, a0, b0);
        tile.multiply(a1, b1);
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int m0 = t0 + (wave / WN) * (BM / WM), c0 = n0 + (wave % WN) * (BN / WN) + (lane & 31);
#pragma unroll
    for (int i = 0; i < tile.TM; ++i)
#pragma unroll
        for (int g = 0; g < 16; ++g) {
            const int t = m0 + i * 32 + 8 * (g / 4) + 4 * (lane >> 5) + g % 4;
            if (t >= p.T) continue;
            const float s = p.s[t];
#pragma unroll
            for (int j = 0; j < tile.TN; ++j) {
                const int n = c0 + j * 32;
                if (n < p.n) put<O>(p, t, n, tile.acc[i][j][g], s);
            }
        }
}

// ---- few tokens ----------------------------------------------------------------------------
// Bound by reading w once: each wave takes 16 rows of w and a slice of k, its weights going from
// memory straight into matrix operands (16 rows x 64 bytes per instruction), and the eight
// waves of a workgroup add their sums through shared memory.  MT groups of 16 tokens share each
// weight operand.
template <typename O, int MT>
__global__ __launch_bounds__(512) void skinny_kernel(const LinearP p) {
    constexpr int W = 8;
    __shared__ int sums[W][MT][64][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const int steps = (p.k + 63) / 64, s0 = steps * wave / W, s1 = steps * (wave + 1) / W;
    const int8_t* wr = p.w + (int64_t)min(n0 + r, p.n - 1) * p.w_stride + g * 16;
    const int8_t* qr[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) qr[m] = p.q + (int64_t)min(m * 16 + r, p.T - 1) * p.q_stride + g * 16;
    i32x4 acc[MT] = {};
    constexpr int U = 4;  // steps in flight
    for (int s = s0; s < s1; s += U) {
        i32x4 a[U], b[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (s + u) * 64;
            const bool in = s + u < s1 && at + g * 16 < p.k;
            a[u] = in ? __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(wr + at)) : i32x4{};
#pragma unroll
            for (int m = 0; m < MT; ++m) b[u][m] = in ? *reinterpret_cast<const i32x4*>(qr[m] + at) : i32x4{};
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u], b[u][m], acc[m], 0, 0, 0);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) *reinterpret_cast<i32x4*>(sums[wave][m][lane]) = acc[m];
    __syncthreads();
    // lane l of the matrix layout: token l % 16, channels 4 (l / 16) .. + 3
    for (int i = threadIdx.x; i < MT * 256; i += W * 64) {
        const int m = i >> 8, l = (i >> 2) & 63, c = i & 3;
        int v = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) v += sums[w][m][l][c];
        const int t = m * 16 + (l & 15), n = n0 + 4 * (l >> 4) + c;
        if (t < p.T && n < p.n) put<O>(p, t, n, v, p.s[t]);
    }
}

template <typename O>
hipError_t product(const LinearP& p, int n_cu, hipStream_t st) {
    if (p.T <= 64) {
        const dim3 grid((unsigned)ceil_div(p.n, 16));
        switch ((p.T + 15) / 16) {
            case 1: hipLaunchKernelGGL((skinny_kernel<O, 1>), grid, dim3(512), 0, st, p); break;
            case 2: hipLaunchKernelGGL((skinny_kernel<O, 2>), grid, dim3(512), 0, st, p); break;
            case 3: hipLaunchKernelGGL((skinny_kernel<O, 3>), grid, dim3(512), 0, st, p); break;
            default: hipLaunchKernelGGL((skinny_kernel<O, 4>), grid, dim3(512), 0, st, p);
        }
        return hipGetLastError();
    }
    const int tn = (int)ceil_div(p.n, 128);
    const int64_t tiles = ceil_div(p.T, 128) * tn;
    hipLaunchKernelGGL((tile_kernel<O, 128, 128, 2, 2>), dim3((unsigned)tiles), dim3(256), 0, st, p, tn);
    return hipGetLastError();
}

}  // namespace

size_t linear_workspace(const ls_linear_i8_args& a) {
    if (a.x_type == LS_I8) return 0;
    return round_up((size_t)a.n_tokens * a.k, 256) + round_up((size_t)a.n_tokens * 4, 256);
}

hipError_t launch_linear(const ls_linear_i8_args& a, void* ws, int n_cu, hipStream_t st) {
    LinearP p{static_cast<const int8_t*>(a.x), a.x_stride, a.x_scale, a.w, a.w_stride, a.w_scale, a.bias, a.out,
              a.out_stride, a.n_tokens, a.k, a.n};
    if (a.x_type != LS_I8) {
        int8_t* q = static_cast<int8_t*>(ws);
        float* s = reinterpret_cast<float*>(q + round_up((size_t)a.n_tokens * a.k, 256));
        const dim3 grid(a.n_tokens), block(256);
        if (a.x_type == LS_F32)
            hipLaunchKernelGGL(quantise_kernel<float>, grid, block, 0, st, a.x, a.x_stride, a.k, q, s);
        else if (a.x_type == LS_F16)
            hipLaunchKernelGGL(quantise_kernel<_Float16>, grid, block, 0, st, a.x, a.x_stride, a.k, q, s);
        else
            hipLaunchKernelGGL(quantise_kernel<__bf16>, grid, block, 0, st, a.x, a.x_stride, a.k, q, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        p.q = q;
        p.q_stride = a.k;
        p.s = s;
    }
    switch (a.out_type) {
        case LS_F32: return product<float>(p, n_cu, st);
        case LS_F16: return product<_Float16>(p, n_cu, st);
        default: return product<__bf16>(p, n_cu, st);
    }
}

}  // namespace ls

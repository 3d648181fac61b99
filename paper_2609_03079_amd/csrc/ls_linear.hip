// ls_linear.hip - matrix products in 8-bit integers with a scale for each token and channel:
// out[t, n] = s_t w_scale[n] sum_k q[t, k] w[n, k] + bias[n].
//
// Both operands are contiguous in k, which is what the integer matrix instructions take: a lane
// holds 16 consecutive bytes of a row of w and of a row of q.  Sums are exact (32-bit integers,
// |sum| < 2^31 for k < 2^17), so neither the order of the sum nor the kernel chosen changes a bit
// of the result; the two scales and the bias are applied once, in fp32 and in the same order everywhere.
#include <algorithm>
#include <type_traits>

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
    int slices, splits;  // tiles: 128-byte slices of k per split; splits of k
    int32_t* part;       // [splits][T][n] sums of the splits
};

// A sum with its scales and bias, the same three roundings in every kernel: left to the compiler, some
// added the bias in one step with the product and some after it, and some rounded to float16 in that step
// too, which the empty statement keeps apart.  Without a bias: adds -0, which changes nothing.
__device__ inline float scaled(int acc, float s, float w_scale, float bias) {
    float v = fmaf((float)acc * s, w_scale, bias);
    asm("" : "+v"(v));
    return v;
}
__device__ inline float bias_of(const LinearP& p, int n) { return p.bias ? p.bias[n] : -0.f; }

template <typename O>
__device__ inline void put(const LinearP& p, int t, int n, int acc, float s) {
    static_cast<O*>(p.out)[(int64_t)t * p.out_stride + n] = (O)scaled(acc, s, p.w_scale[n], bias_of(p, n));
}

// Channels n0 .. n0 + n - 1 of the product, and tokens t0 .. t0 + T - 1.
template <typename O>
LinearP channels(LinearP p, int64_t n0, int64_t n) {
    p.n = (int)n;
    p.w += n0 * p.w_stride;
    p.w_scale += n0;
    if (p.bias) p.bias += n0;
    p.out = static_cast<O*>(p.out) + n0;
    return p;
}
template <typename O>
LinearP tokens(LinearP p, int64_t t0, int64_t T) {
    p.T = (int)T;
    p.q += t0 * p.q_stride;
    p.s += t0;
    p.out = static_cast<O*>(p.out) + t0 * p.out_stride;
    return p;
}

// A launch holds fewer than 2^32 threads along x, and the kernels count channels and tokens in 31 bits
// with room for a grid's stride: larger products are cut into pieces of at most this (2^23 of the smallest tiles).
constexpr int64_t kChannelsPerLaunch = 1 << 20, kTokensPerLaunch = 1 << 16;

template <typename O, typename F>
hipError_t by_channels(const LinearP& p, F&& launch) {
    for (int64_t n = 0; n < p.n; n += kChannelsPerLaunch) {
        const hipError_t e = launch(channels<O>(p, n, std::min(kChannelsPerLaunch, p.n - n)));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- quantisation --------------------------------------------------------------------------
// |x| as ordered integers: an infinity is 0x7f800000, a NaN above it.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Over the 64 lanes by lane exchanges within the registers; the result is in every lane.
template <int CTRL, int ROWS>
__device__ inline int dpp(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ inline uint32_t wave_max(uint32_t m) {
    m = max(m, (uint32_t)dpp<0xb1, 0xf>((int)m));   // quad_perm [1,0,3,2]
    m = max(m, (uint32_t)dpp<0x4e, 0xf>((int)m));   // quad_perm [2,3,0,1]
    m = max(m, (uint32_t)dpp<0x141, 0xf>((int)m));  // row_half_mirror
    m = max(m, (uint32_t)dpp<0x140, 0xf>((int)m));  // row_mirror
    m = max(m, (uint32_t)dpp<0x142, 0xa>((int)m));  // row_bcast:15
    m = max(m, (uint32_t)dpp<0x143, 0xc>((int)m));  // row_bcast:31
    return (uint32_t)__builtin_amdgcn_readlane((int)m, 63);
}
__device__ inline int wave_add(int v) {
    v += dpp<0xb1, 0xf>(v);
    v += dpp<0x4e, 0xf>(v);
    v += dpp<0x141, 0xf>(v);
    v += dpp<0x140, 0xf>(v);
    v += dpp<0x142, 0xa>(v);
    v += dpp<0x143, 0xc>(v);
    return __builtin_amdgcn_readlane(v, 63);
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

// round(127 x / max), ties to even.  The product with the rounded inverse is off by less than 1e-4,
// so away from a tie it rounds to the same integer; near one the quotient decides (for 16-bit x
// 127/128 x is exact, and cannot overflow as 127 x can, and the quotient rounded once, so a tie is
// seen as one).  A division for every element made the kernel twice as slow.
__device__ inline int quantise(float x, float top, float inv) {
    const float p = x * inv;
    float r = rintf(p);
    if (fabsf(p - r) > 0.4999f) r = rintf(x * 0.9921875f / top * 128.f);
    return (int)r;
}

// One workgroup of NT threads per token; 8 elements per thread and step, the first kHeld of them kept in
// registers between the maximum and the division.  2048 x 8192 bfloat16: 16 us; with a thread for every
// vector 22.2, a workgroup's chain of loads, maximum and barrier being longer than its work.
template <typename T, int NT, int kHeld>
__global__ __launch_bounds__(NT) void quantise_kernel(const void* x, int64_t x_stride, int k, int8_t* q, float* s) {
    __shared__ uint32_t part[NT / 64];
    const int64_t t = blockIdx.x;
    const T* row = static_cast<const T*>(x) + t * x_stride;
    constexpr int kStep = NT * 8;
    Pack<T, 8> v[kHeld];
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
        const int e = (int)threadIdx.x * 8 + c * kStep;
        if (e < k) v[c] = load_pack<T, 8>(row, e);
    }
    auto look = [&](const Pack<T, 8>& u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, magnitude((float)u.e[i]));
    };
#pragma unroll
    for (int c = 0; c < kHeld; ++c)
        if ((int)threadIdx.x * 8 + c * kStep < k) look(v[c]);
    for (int e = (int)threadIdx.x * 8 + kHeld * kStep; e < k; e += kStep) look(load_pack<T, 8>(row, e));
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) m = max(m, part[w]);
    float top;
    const float scale = token_scale(m, &top), inv = top > 0.f ? 127.f / top : 0.f;
    if (threadIdx.x == 0) s[t] = scale;
    auto write = [&](int e, const Pack<T, 8>& u) {
        Pack<int8_t, 8> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.e[i] = top > 0.f ? (int8_t)quantise((float)u.e[i], top, inv) : (int8_t)0;
        store_pack<int8_t, 8>(q, t * k + e, o);
    };
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
        const int e = (int)threadIdx.x * 8 + c * kStep;
        if (e < k) write(e, v[c]);
    }
    for (int e = (int)threadIdx.x * 8 + kHeld * kStep; e < k; e += kStep) write(e, load_pack<T, 8>(row, e));
}

template <typename T>
hipError_t quantise_rows(const ls_linear_i8_args& a, int8_t* q, float* s, hipStream_t st) {
    const dim3 grid(a.n_tokens);
    if (a.k <= 2048)
        hipLaunchKernelGGL((quantise_kernel<T, 256, 1>), grid, dim3(256), 0, st, a.x, a.x_stride, a.k, q, s);
    else if (a.k <= 4096)
        hipLaunchKernelGGL((quantise_kernel<T, 256, 2>), grid, dim3(256), 0, st, a.x, a.x_stride, a.k, q, s);
    else if (a.k <= 8192)
        hipLaunchKernelGGL((quantise_kernel<T, 256, 4>), grid, dim3(256), 0, st, a.x, a.x_stride, a.k, q, s);
    else
        hipLaunchKernelGGL((quantise_kernel<T, 512, 4>), grid, dim3(512), 0, st, a.x, a.x_stride, a.k, q, s);
    return hipGetLastError();
}

// ---- tiles through shared memory -----------------------------------------------------------
// out tile of BM tokens by BN channels; WM x WN waves, each with a (BM / WM) x (BN / WN) part in
// 32 x 32 matrix tiles.  Both operands come in 128-byte slices of k, copied straight to a ring of S
// slices in shared memory, S - 1 of them under way while one is used.  (A whole line of memory a row:
// with slices of 64 bytes, each line asked for twice, the largest tiles' copies alone took 82 us of
// 2048 x 8192 x 8192 in place of 71, and the product 143 in place of 125.)  A slice is multiplied in
// four steps; a step's operands are read from shared memory while the products of the step before
// run.  What is left is the products themselves: without any copies they take 102 us with random
// operands, 73 with zeros, the clock falling under their load.
// A row's eight 16-byte chunks lie at places permuted by its number, so that the 16 rows a read
// touches together lie in different banks.
constexpr int kSlice = 128;

__device__ inline int place(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

// A workgroup's copies of ROWS rows, slice by slice: 8 rows an instruction.
template <int ROWS, int WAVES>
struct Fetch {
    static constexpr int N = ROWS / (8 * WAVES);
    static_assert(ROWS % (8 * WAVES) == 0, "whole instructions");
    const int8_t* src[N];  // this lane's chunk of a slice at 0

    __device__ inline void start(const int8_t* base, int64_t stride, int row0, int rows) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = (i * WAVES + wave) * 8 + (lane >> 3);
            src[i] = base + (int64_t)min(row0 + r, rows - 1) * stride + place(r, lane & 7) * 16;
        }
    }
    // The slice at k0, of which bytes below `last` count.
    __device__ inline void copy(int k0, int last, int8_t* lds) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r0 = (i * WAVES + wave) * 8;
            const int8_t* from = src[i] + k0;
            if (k0 + kSlice > last && k0 + place(r0 + (lane >> 3), lane & 7) * 16 >= last) from = reinterpret_cast<const int8_t*>(g_zero_chunk);
            __builtin_amdgcn_global_load_lds((gptr)from, (lptr)(lds + r0 * kSlice), 16, 0, 0);
        }
    }
};

template <int BM, int BN, int WM, int WN>
struct Tile {
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32, kAll = TM * TN;
    i32x16 acc[TM][TN];
    i32x4 x[2][TM], y[2][TN];  // the operands of the present step and of the next

    // Operands R: step kk (32 bytes of k) of a slice.
    template <int R>
    __device__ inline void read(const int8_t* a, const int8_t* b, int kk) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
        const int m0 = (wave / WN) * (BM / WM), n0 = (wave % WN) * (BN / WN);
#pragma unroll
        for (int i = 0; i < TM; ++i)
            x[R][i] = *reinterpret_cast<const i32x4*>(a + (m0 + i * 32 + r) * kSlice + place(r, kk * 2 + h) * 16);
#pragma unroll
        for (int j = 0; j < TN; ++j)
            y[R][j] = *reinterpret_cast<const i32x4*>(b + (n0 + j * 32 + r) * kSlice + place(r, kk * 2 + h) * 16);
    }
    // The products of operands R from the FROM-th on, below the TO-th.
    template <int R, int FROM, int TO>
    __device__ inline void multiply() {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                if (i * TN + j >= FROM && i * TN + j < TO)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[R][i], y[R][j], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
    // The products of operands R; once the first has them (the wait for a read is for all reads), `next`
    // asks for those of the next step.
    template <int R, typename F>
    __device__ inline void step(F&& next) {
        multiply<R, 0, 1>();
        next();
        __builtin_amdgcn_sched_barrier(0);
        multiply<R, 1, kAll>();
    }
};

// All but this wave's newest N copies have landed, its reads of shared memory are done, and so for
// the other waves.
template <int N>
__device__ inline void arrive() {
    static_assert(N < 64, "the counter");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// k in p.splits parts, one workgroup each (blockIdx.y): where the tiles alone would leave compute
// units idle.  Their sums meet in finish_kernel.
template <typename O, int BM, int BN, int WM, int WN, int S>
__global__ __launch_bounds__(WM * WN * 64, WM * WN / 4) void tile_kernel(const LinearP p, int tiles_n) {
    static_assert(S >= 2 && S <= 4, "the ring");
    // an array for each slice, not one: a read of one must not wait for the copies into the others
    constexpr int kA = BM * kSlice, kB = BN * kSlice;
    __shared__ __attribute__((aligned(16))) int8_t a0[kA], a1[kA], a2[S > 2 ? kA : 16], a3[S > 3 ? kA : 16];
    __shared__ __attribute__((aligned(16))) int8_t b0[kB], b1[kB], b2[S > 2 ? kB : 16], b3[S > 3 ? kB : 16];
    __shared__ __attribute__((aligned(16))) float scale[BM];  // of the tokens
    const int t0 = (blockIdx.x / tiles_n) * BM, n0 = (blockIdx.x % tiles_n) * BN;
    const int first = blockIdx.y * p.slices * kSlice, last = min(p.k, first + p.slices * kSlice);
    Tile<BM, BN, WM, WN> tile;
#pragma unroll
    for (auto& r : tile.acc)
        for (auto& v : r) v = i32x16{};
    constexpr int W = WM * WN;
    Fetch<BM, W> fa;
    Fetch<BN, W> fb;
    fa.start(p.q, p.q_stride, t0, p.T);
    fb.start(p.w, p.w_stride, n0, p.n);
    constexpr int kCopies = fa.N + fb.N;  // of a slice, by each wave
    // Slices are taken in turn from one that depends on the workgroup (rows a power of two apart would
    // all ask the same memory channel at once: with slices of 64 bytes 2048 x 8192 x 10240 took 241 us
    // without, 223 with it), and past the end
    // slices of zeros: the count under way stays the same, and the ring's S steps are one loop
    // without exits (whose copies of the sums cost more than the products).
    const int n_slices = (last - first + kSlice - 1) / kSlice;
    const int turn = (int)(blockIdx.x % tiles_n / 8 % 4) * 2 % n_slices;
    auto copy = [&](int i, int8_t* a, int8_t* b) {
        int at = i + turn;
        at -= at >= n_slices ? n_slices : 0;
        const int k0 = i < n_slices ? first + at * kSlice : last;
        fa.copy(k0, last, a);
        fb.copy(k0, last, b);
    };
    const float own = p.s[min(t0 + (int)threadIdx.x % BM, p.T - 1)];
    copy(0, a0, b0);
    copy(1, a1, b1);
    if constexpr (S > 2) copy(2, a2, b2);
    if constexpr (S > 3) copy(3, a3, b3);
    scale[threadIdx.x % BM] = own;
    arrive<(S - 1) * kCopies>();
    tile.template read<0>(a0, b0, 0);
    // Slice i, the operands of whose first step are on their way.  Before its last step everything of it
    // has been read, so its place is free for slice i + S, and slice i + 1 has landed.
    auto slice = [&](int i, int8_t* a, int8_t* b, const int8_t* a_next, const int8_t* b_next) {
        tile.template step<0>([&] { tile.template read<1>(a, b, 1); });
        tile.template step<1>([&] { tile.template read<0>(a, b, 2); });
        tile.template step<0>([&] { tile.template read<1>(a, b, 3); });
        arrive<(S - 2) * kCopies>();
        tile.template step<1>([&] {
            tile.template read<0>(a_next, b_next, 0);
            copy(i + S, a, b);
        });
    };
    for (int i = 0; i < n_slices; i += S) {
        slice(i, a0, b0, a1, b1);
        if constexpr (S == 2) slice(i + 1, a1, b1, a0, b0);
        if constexpr (S > 2) slice(i + 1, a1, b1, a2, b2);
        if constexpr (S == 3) slice(i + 2, a2, b2, a0, b0);
        if constexpr (S > 3) {
            slice(i + 2, a2, b2, a3, b3);
            slice(i + 3, a3, b3, a0, b0);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0070);  // no copy into shared memory outlives the workgroup
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // Element g of a lane's sums belongs to row 8 (g / 4) + g % 4 of its rows, which begin at r0 of the tile.
    const int r0 = (wave / WN) * (BM / WM) + 4 * (lane >> 5), c0 = n0 + (wave % WN) * (BN / WN) + (lane & 31);
    if (p.splits > 1) {
        int32_t* to = p.part + ((int64_t)blockIdx.y * p.T + t0 + r0) * p.n + c0;
#pragma unroll
        for (int i = 0; i < tile.TM; ++i)
#pragma unroll
            for (int g = 0; g < 16; ++g)
#pragma unroll
                for (int j = 0; j < tile.TN; ++j) {
                    const int row = i * 32 + 8 * (g / 4) + g % 4;
                    if (t0 + r0 + row < p.T && c0 + j * 32 < p.n) to[(int64_t)row * p.n + j * 32] = tile.acc[i][j][g];
                }
        return;
    }
    // The scales before the first store (a load after a store waits for it), those of the tokens from
    // shared memory: with loads in between, the 256 x 256 tiles of 2048 x 8192 x 8192 took 152 us, not 137.
    float ws[tile.TN], bias[tile.TN];
#pragma unroll
    for (int j = 0; j < tile.TN; ++j) {
        const int n = min(c0 + j * 32, p.n - 1);
        ws[j] = p.w_scale[n], bias[j] = bias_of(p, n);
    }
    O* to = static_cast<O*>(p.out) + (int64_t)(t0 + r0) * p.out_stride + c0;
    auto write = [&](auto whole) {  // whole: nothing of the tile lies outside the product
#pragma unroll
        for (int i = 0; i < tile.TM; ++i)
#pragma unroll
            for (int g = 0; g < 16; g += 4) {
                const f32x4 s = *reinterpret_cast<const f32x4*>(scale + r0 + i * 32 + 2 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < tile.TN; ++j) {
                        const int row = i * 32 + 2 * g + e;
                        if (whole.value || (t0 + r0 + row < p.T && c0 + j * 32 < p.n))
                            to[row * p.out_stride + j * 32] = (O)scaled(tile.acc[i][j][g + e], s[e], ws[j], bias[j]);
                    }
            }
    };
    if (t0 + BM <= p.T && n0 + BN <= p.n)
        write(std::true_type{});
    else
        write(std::false_type{});
}

template <typename O>
__global__ __launch_bounds__(256) void finish_kernel(const LinearP p) {
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= p.n) return;
    for (int t = blockIdx.y; t < p.T; t += gridDim.y) {
        int v = 0;
        for (int i = 0; i < p.splits; ++i) v += p.part[((int64_t)i * p.T + t) * p.n + n];
        put<O>(p, t, n, v, p.s[t]);
    }
}

// ---- up to four tokens ---------------------------------------------------------------------
// Bound by reading w once.  One workgroup of 16 waves per compute unit; a wave takes whole rows of
// w, one after the other, four kilobytes at a time, a kilobyte of consecutive bytes an instruction,
// the next four under way while these are multiplied on the vector ALU (four products an
// instruction).  The tokens lie in shared memory; floating ones are quantised on the way there, by
// every workgroup, while its first weights are under way: one token x 4096 x 12288 takes 9.6 us
// a pass, 7.4 of them reading (50 MB at 6.8 TB/s), 8.4 from 8-bit inputs; 13.2 with small workgroups, each
// of which quantised the token again.
constexpr int kVecWaves = 16, kVecBlock = 4096;

inline size_t vec_shared(int T, int k) { return (size_t)T * round_up(k, kVecBlock); }
inline bool vec_takes(int T, int k) { return T <= 4 && vec_shared(T == 3 ? 4 : T, k) <= 65536; }

template <typename O, typename X, int TT>
__global__ __launch_bounds__(kVecWaves * 64) void vec_kernel(const LinearP p, const void* x, int64_t x_stride) {
    constexpr int C = kVecBlock / 1024;
    extern __shared__ __attribute__((aligned(16))) int8_t xs[];  // [TT][padded]
    __shared__ uint32_t part[TT][kVecWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = threadIdx.x;
    const int blocks = (p.k + kVecBlock - 1) / kVecBlock, padded = blocks * kVecBlock;
    const int rows = gridDim.x * kVecWaves;  // at a time
    int n = blockIdx.x + gridDim.x * wave, block = 0;
    i32x4 a[2][C];
    auto load = [&](i32x4 (&to)[C], int row, int b) {
#pragma unroll
        for (int c = 0; c < C; ++c)  // (past the row its last bytes: they meet zeros)
            to[c] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(
                p.w + (int64_t)row * p.w_stride + min(b * kVecBlock + c * 1024 + lane * 16, p.k - 16)));
    };
    if (n < p.n) load(a[0], n, 0);
    float scale[TT];
    if constexpr (std::is_same_v<X, int8_t>) {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int tt = min(t, p.T - 1);
            scale[t] = p.s[tt];
            for (int e = tid * 16; e < padded; e += kVecWaves * 1024)
                *reinterpret_cast<i32x4*>(xs + t * padded + e) = e < p.k ? *reinterpret_cast<const i32x4*>(p.q + tt * p.q_stride + e) : i32x4{};
        }
    } else {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            uint32_t m = 0;
            for (int e = tid * 4; e < p.k; e += kVecWaves * 256) {
                const auto u = load_pack<X, 4>(x, min(t, p.T - 1) * x_stride + e);
#pragma unroll
                for (int i = 0; i < 4; ++i) m = max(m, magnitude((float)u.e[i]));
            }
            m = wave_max(m);
            if (lane == 0) part[t][wave] = m;
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < kVecWaves; ++w) m = max(m, part[t][w]);
            float top;
            scale[t] = token_scale(m, &top);
            const float inv = top > 0.f ? 127.f / top : 0.f;
            for (int e = tid * 4; e < padded; e += kVecWaves * 256) {
                Pack<int8_t, 4> o{};
                if (e < p.k && top > 0.f) {
                    const auto u = load_pack<X, 4>(x, min(t, p.T - 1) * x_stride + e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o.e[i] = (int8_t)quantise((float)u.e[i], top, inv);
                }
                store_pack<int8_t, 4>(xs, t * padded + e, o);
            }
        }
    }
    __syncthreads();
    if (n >= p.n) return;
    int acc[TT] = {};
    // this block of the row, its sum if it is the row's last; the next one loaded meanwhile.  False: that was all.
    auto step = [&](const i32x4 (&now)[C], i32x4 (&next)[C]) {
        int row = n, b = block + 1;
        if (b == blocks) b = 0, row += rows;
        if (row < p.n) load(next, row, b);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const i32x4 q = *reinterpret_cast<const i32x4*>(xs + t * padded + block * kVecBlock + c * 1024 + lane * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t] = __builtin_amdgcn_sdot4(now[c][e], q[e], acc[t], false);
            }
        if (b == 0) {
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const int v = wave_add(acc[t]);
                acc[t] = 0;
                if (lane == 0 && t < p.T) put<O>(p, t, n, v, scale[t]);
            }
        }
        n = row, block = b;
        return n < p.n;
    };
    while (step(a[0], a[1]) && step(a[1], a[0])) {
    }
}

template <typename O, typename X>
hipError_t vec(const LinearP& p, const void* x, int64_t x_stride, int n_cu, hipStream_t st) {
    const dim3 grid((unsigned)std::min<int64_t>(n_cu, ceil_div(p.n, kVecWaves))), block(kVecWaves * 64);
    const size_t shared = vec_shared(p.T == 3 ? 4 : p.T, p.k);
    if (p.T == 1)
        hipLaunchKernelGGL((vec_kernel<O, X, 1>), grid, block, shared, st, p, x, x_stride);
    else if (p.T == 2)
        hipLaunchKernelGGL((vec_kernel<O, X, 2>), grid, block, shared, st, p, x, x_stride);
    else
        hipLaunchKernelGGL((vec_kernel<O, X, 4>), grid, block, shared, st, p, x, x_stride);
    return hipGetLastError();
}

// ---- up to 48 tokens -----------------------------------------------------------------------
// Few enough that reading w sets the pace, too many for the vector ALU: each wave copies 256-byte
// slices of 16 NR rows of w and of the tokens to shared memory of its own, every W-th slice, without
// barriers, one slice ahead, and the waves' sums are added at the end.  8 tokens x 5120 x 5120 6.4 us,
// x 8192 x 28672 46 us (with both operands read straight into the matrix operands, 16 rows x 64 bytes
// an instruction, 14.3 and 53.7).  From 17 tokens on only while each workgroup has a compute unit at
// once: 48 tokens x 5120 x 5120 10.2 us (in tiles with k split 14.4), but x 8192 x 10240 36.4 (22.8).
template <typename O, int MT, int NR, int W>
__global__ __launch_bounds__(W * 64) void slice_kernel(const LinearP p) {
    constexpr int RW = 16 * NR, RX = 16 * MT, kBytes = 256;
    __shared__ __attribute__((aligned(16))) int8_t buf0[W * (RW + RX) * kBytes];
    __shared__ __attribute__((aligned(16))) int8_t buf1[W * (RW + RX) * kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * RW;
    i32x4 acc[NR][MT] = {};
    // four rows an instruction; a row's 16 chunks permuted by its number (banks)
    auto copy = [&](int k0, int8_t* buf) {
        int8_t* dst = buf + wave * (RW + RX) * kBytes;
#pragma unroll
        for (int i = 0; i < (RW + RX) / 4; ++i) {
            const int r4 = i * 4 + (lane >> 4), at = k0 + ((lane & 15) ^ (r4 & 15)) * 16;
            const int8_t* src = i < RW / 4 ? p.w + (int64_t)min(n0 + r4, p.n - 1) * p.w_stride
                                           : p.q + (int64_t)min(r4 - RW, p.T - 1) * p.q_stride;
            if (i >= RW / 4 && i * 4 - RW >= p.T) continue;  // rows of no token: their sums are dropped
            __builtin_amdgcn_global_load_lds((gptr)(at < p.k ? src + at : reinterpret_cast<const int8_t*>(g_zero_chunk)),
                                             (lptr)(dst + i * 1024), 16, 0, 0);
        }
    };
    auto use = [&](const int8_t* buf) {
        const int8_t* src = buf + wave * (RW + RX) * kBytes;
#pragma unroll
        for (int kk = 0; kk < kBytes / 64; ++kk) {
            const int chunk = ((kk * 4 + g) ^ r) * 16;
            i32x4 a[NR], b[MT];
#pragma unroll
            for (int i = 0; i < NR; ++i) a[i] = *reinterpret_cast<const i32x4*>(src + (i * 16 + r) * kBytes + chunk);
#pragma unroll
            for (int m = 0; m < MT; ++m) b[m] = *reinterpret_cast<const i32x4*>(src + (RW + m * 16 + r) * kBytes + chunk);
#pragma unroll
            for (int i = 0; i < NR; ++i)
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[i][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[m], acc[i][m], 0, 0, 0);
        }
    };
    auto landed = [] {  // the wave's copies are in shared memory, its reads done
        __builtin_amdgcn_s_waitcnt(0x0070);
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    };
    int k0 = wave * kBytes;
    if (k0 < p.k) {
        copy(k0, buf0);
        for (;;) {
            landed();
            if (k0 + W * kBytes < p.k) copy(k0 + W * kBytes, buf1);
            use(buf0);
            if ((k0 += W * kBytes) >= p.k) break;
            landed();
            if (k0 + W * kBytes < p.k) copy(k0 + W * kBytes, buf0);
            use(buf1);
            if ((k0 += W * kBytes) >= p.k) break;
        }
    }
    __syncthreads();
    int* sums = reinterpret_cast<int*>(buf0);  // [wave][NR][MT][64][4]
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int m = 0; m < MT; ++m) *reinterpret_cast<i32x4*>(sums + (((wave * NR + i) * MT + m) * 64 + lane) * 4) = acc[i][m];
    __syncthreads();
    for (int e = threadIdx.x; e < NR * MT * 256; e += W * 64) {
        const int i = e / (MT * 256), m = (e >> 8) % MT, l = (e >> 2) & 63, c = e & 3;
        int v = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) v += sums[w * NR * MT * 256 + e];
        const int t = m * 16 + (l & 15), n = n0 + i * 16 + 4 * (l >> 4) + c;
        if (t < p.T && n < p.n) put<O>(p, t, n, v, p.s[t]);
    }
}

template <typename O, int MT, int NR, int W>
hipError_t slices(const LinearP& p, hipStream_t st) {
    hipLaunchKernelGGL((slice_kernel<O, MT, NR, W>), dim3((unsigned)ceil_div(p.n, 16 * NR)), dim3(W * 64), 0, st, p);
    return hipGetLastError();
}

// ---- choice of tiles -----------------------------------------------------------------------
// The tile shapes, by tokens and channels: slices in the ring, workgroups that run at once on a
// compute unit, and the time of a 128-byte slice of k with all of them running, as measured on 64 to
// 2048 tokens of k = 8192 (us).  Where a workgroup has its compute unit to itself, a longer ring
// hides the copies' way (2048 x 8192 x 2048 in 128 x 128 tiles: 47 us with two slices, 40 with four).
struct TileShape {
    int bm, bn, ring, per_cu;
    double slice_us;
};
constexpr TileShape kTiles[] = {{64, 128, 4, 1, 0.48}, {64, 128, 3, 2, 0.67}, {128, 128, 4, 1, 0.62}, {128, 128, 2, 2, 1.17}, {256, 256, 2, 1, 1.95}};
constexpr int kShapes = 5, kLargest = 4, kMaxSplits = 8;

// Shape and splits of k with the least estimated time for T x n: rounds of workgroups x (slices +
// start), and for a split the traffic of its sums.
struct TilePlan {
    int shape, splits, slices;
    double us;
};
TilePlan plan_tiles(int64_t T, int64_t k, int64_t n, int n_cu, size_t room) {
    const int64_t slices = ceil_div(k, kSlice);
    TilePlan best{0, 1, (int)slices, 0};
    for (int i = 0; i < kShapes; ++i)
        for (int s = 1; s <= kMaxSplits; ++s) {
            const TileShape& t = kTiles[i];
            const int64_t per = round_up(ceil_div(slices, s), t.ring);
            if (s > 1 && ((uint64_t)s * T * n * 4 > room || ceil_div(slices, per) != s)) continue;
            const int64_t wgs = ceil_div(T, t.bm) * ceil_div(n, t.bn) * s, slots = (int64_t)n_cu * t.per_cu;
            const double us = ceil_div(wgs, slots) * (per * t.slice_us + 3.0) + (s > 1 ? 4.0 + (double)s * T * n * 8 / 4e6 : 0.0);
            if (best.us == 0 || us < best.us) best = {i, s, (int)per, us};
        }
    return best;
}

template <typename O, int SHAPE, int WM, int WN>
hipError_t tiles(const LinearP& p, hipStream_t st) {
    constexpr TileShape t = kTiles[SHAPE];
    const int tn = (int)ceil_div(p.n, t.bn);
    hipLaunchKernelGGL((tile_kernel<O, t.bm, t.bn, WM, WN, t.ring>), dim3((unsigned)(ceil_div(p.T, t.bm) * tn), p.splits),
                       dim3(WM * WN * 64), 0, st, p, tn);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL(finish_kernel<O>, dim3((unsigned)ceil_div(p.n, 256), (unsigned)std::min(p.T, 65535)), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <typename O>
hipError_t tiles_of(LinearP p, const TilePlan& plan, int32_t* part, hipStream_t st) {
    p.splits = plan.splits, p.slices = plan.slices, p.part = part;
    switch (plan.shape) {
        case 0: return tiles<O, 0, 2, 2>(p, st);
        case 1: return tiles<O, 1, 2, 2>(p, st);
        case 2: return tiles<O, 2, 2, 2>(p, st);
        case 3: return tiles<O, 3, 2, 2>(p, st);
        default: return tiles<O, kLargest, 2, 4>(p, st);
    }
}

template <typename O>
hipError_t product(const LinearP& p, int32_t* part, size_t room, int n_cu, hipStream_t st) {
    if (vec_takes(p.T, p.k)) return vec<O, int8_t>(p, nullptr, 0, n_cu, st);
    if (p.T <= 16) return slices<O, 1, 1, 4>(p, st);
    if (p.T <= 48 && ceil_div(p.n, 32) <= n_cu)
        return p.T <= 32 ? slices<O, 2, 2, 4>(p, st) : slices<O, 3, 2, 4>(p, st);
    const TilePlan whole = plan_tiles(p.T, p.k, p.n, n_cu, room);
    // The largest tiles in whole rounds, the channels left over by the best shape for them, where
    // that is faster: 2048 x 8192 x 10240 is 1.25 rounds of 256 x 256 tiles.
    const int64_t rows = ceil_div(p.T, 256), columns = ceil_div(p.n, 256), rounds = rows * columns / n_cu;
    const int64_t first = rounds * n_cu / rows;  // columns of tiles in those rounds
    if (first > 0 && first < columns) {
        const int64_t slices = ceil_div(p.k, kSlice), n1 = first * 256;
        const TilePlan rest = plan_tiles(p.T, p.k, p.n - n1, n_cu, room);
        if (rounds * (round_up(slices, 2) * kTiles[kLargest].slice_us + 3.0) + rest.us + 2.0 < whole.us) {
            hipError_t e = tiles_of<O>(channels<O>(p, 0, n1), {kLargest, 1, (int)round_up(slices, 2), 0}, part, st);
            if (e != hipSuccess) return e;
            return tiles_of<O>(channels<O>(p, n1, p.n - n1), rest, part, st);
        }
    }
    return tiles_of<O>(p, whole, part, st);
}

template <typename O>
hipError_t linear(const ls_linear_i8_args& a, LinearP p, uint8_t* ws, size_t ws_bytes, int n_cu, hipStream_t st) {
    const size_t used = linear_workspace(a);
    if (a.x_type != LS_I8) {
        if (vec_takes(p.T, p.k)) {
            return by_channels<O>(p, [&](const LinearP& b) {
                return a.x_type == LS_F32   ? vec<O, float>(b, a.x, a.x_stride, n_cu, st)
                       : a.x_type == LS_F16 ? vec<O, _Float16>(b, a.x, a.x_stride, n_cu, st)
                                            : vec<O, __bf16>(b, a.x, a.x_stride, n_cu, st);
            });
        }
        int8_t* q = reinterpret_cast<int8_t*>(ws);
        float* s = reinterpret_cast<float*>(ws + round_up((size_t)a.n_tokens * a.k, 256));
        const hipError_t e = a.x_type == LS_F32   ? quantise_rows<float>(a, q, s, st)
                             : a.x_type == LS_F16 ? quantise_rows<_Float16>(a, q, s, st)
                                                  : quantise_rows<__bf16>(a, q, s, st);
        if (e != hipSuccess) return e;
        p.q = q, p.q_stride = a.k, p.s = s;
    }
    for (int64_t t = 0; t < p.T; t += kTokensPerLaunch) {
        const hipError_t e = by_channels<O>(tokens<O>(p, t, std::min(kTokensPerLaunch, p.T - t)), [&](const LinearP& b) {
            return product<O>(b, reinterpret_cast<int32_t*>(ws + used), ws_bytes - used, n_cu, st);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t linear_workspace(const ls_linear_i8_args& a) {
    if (a.x_type == LS_I8 || vec_takes(a.n_tokens, a.k)) return 0;
    return round_up((size_t)a.n_tokens * a.k, 256) + round_up((size_t)a.n_tokens * 4, 256);
}

hipError_t launch_linear(const ls_linear_i8_args& a, void* ws, size_t ws_bytes, int n_cu, hipStream_t st) {
    const LinearP p{static_cast<const int8_t*>(a.x), a.x_stride, a.x_scale, a.w, a.w_stride, a.w_scale, a.bias, a.out, a.out_stride,
                    a.n_tokens, a.k, a.n, 0, 1, nullptr};
    uint8_t* at = static_cast<uint8_t*>(ws);
    switch (a.out_type) {
        case LS_F32: return linear<float>(a, p, at, ws_bytes, n_cu, st);
        case LS_F16: return linear<_Float16>(a, p, at, ws_bytes, n_cu, st);
        default: return linear<__bf16>(a, p, at, ws_bytes, n_cu, st);
    }
}

}  // namespace ls

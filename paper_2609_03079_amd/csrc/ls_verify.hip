// ls_verify.hip - drafted tokens against the target's probabilities.
//
//   draft i is accepted while u_i q_i(x_i) < p_i(x_i); the token after the last accepted one comes from
//   w = max(p_r - q_r, 0) where draft r was refused, from w = p_r behind the last draft:
//   the first token whose running sum of w exceeds u sum(w).
//
// Everything that decides is computed in 64 bits: the products of the comparison are exact there, and running sums of
// 131072 terms are off by 2^-36 of their total at most, so a token does not depend on the order they are summed in
// (in 32 bits one number in forty would fall on another token).  Bound by reading the one row, or the two, that
// the token comes from.
#include <algorithm>

#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {
namespace {

struct VerifyP {
    ls_verify_args a;
};

__device__ inline double wave_sum64(double v) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// What row r of a sequence gives its tokens: no number and what is below zero give none, infinities as the largest number.
template <typename T>
struct Weights {
    const T* p;
    const T* q;   // NULL: nothing is taken off, but for `token`
    int token;    // -1: none
    __device__ inline double of(int t) const {
        const double x = (double)(float)p[t] - (q ? (double)(float)q[t] : t == token ? 1.0 : 0.0);
        return x > 0.0 ? fmin(x, 3.4028234663852886e38) : 0.0;
    }
};

constexpr int kVerifyThreads = 1024, kWaves = kVerifyThreads / 64;

// One workgroup a sequence.  Each wave takes a run of the vocabulary, each lane every 64th token of it.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(const VerifyP P) {
    const ls_verify_args& a = P.a;
    __shared__ double sums[kWaves];
    __shared__ int first;
    const int s = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = a.counts ? min(a.counts[s], a.n_drafts) : a.n_drafts;
    int32_t* tokens = a.tokens + s * a.tokens_stride;
    if (n < 0) {  // an idle slot
        if ((int)threadIdx.x <= a.n_drafts) tokens[threadIdx.x] = -1;
        if (threadIdx.x == 0) a.n_accepted[s] = -1;
        return;
    }
    const T* target = static_cast<const T*>(a.target) + s * a.target_seq_stride;
    const T* draft = a.draft ? static_cast<const T*>(a.draft) + s * a.draft_seq_stride : nullptr;
    // lane i decides about draft i
    bool accepted = false;
    int x = -1;
    if (lane < n) {
        x = a.drafts[s * a.drafts_stride + lane];
        if (x >= 0 && x < a.vocab) {
            const double p = (float)target[lane * a.target_token_stride + x];
            const double q = draft ? (double)(float)draft[lane * a.draft_token_stride + x] : 1.0;
            accepted = (double)a.accept[s * a.accept_stride + lane] * q < p;
        }
    }
    const uint64_t refused = ~__ballot(accepted);
    const int r = min(n, refused ? (int)__builtin_ctzll(refused) : 64);
    const int x_r = __shfl(x, r & 63, 64);
    Weights<T> w{target + r * a.target_token_stride, r < n && draft ? draft + r * a.draft_token_stride : nullptr, r < n && !draft ? x_r : -1};
    const int per = ((a.vocab + kWaves - 1) / kWaves + 63) / 64 * 64, begin = min(a.vocab, wave * per), end = min(a.vocab, begin + per);
    double total = 0.0;
    for (int pass = 0; pass < 2; ++pass) {
        double sum = 0.0;
        for (int t = begin + lane; t < end; t += 64) sum += w.of(t);
        sum = wave_sum64(sum);
        __syncthreads();
        if (lane == 0) sums[wave] = sum;
        if (threadIdx.x == 0) first = 0x7fffffff;
        __syncthreads();
        total = 0.0;
        for (int i = 0; i < kWaves; ++i) total += sums[i];
        if (total > 0.0 || pass) break;
        w.q = nullptr, w.token = -1;  // nothing is left over: the target's own
    }
    // the wave whose run crosses u sum(w) looks for the token in it; behind the last crossing, the last token that has a weight
    const float u = a.sample[s];
    const double want = (u > 0.f ? (double)u : u == u ? 0.0 : 2.0) * total;
    double before = 0.0;
    int mine = -1, last = -1;
    for (int i = 0; i < kWaves; ++i) {
        if (sums[i] > 0.0) last = i;
        if (mine < 0 && before + sums[i] > want) mine = i;
        if (mine < 0) before += sums[i];
    }
    const bool past = mine < 0;
    if (past) mine = last;
    if (wave == mine) {
        int found = -1, positive = -1;
        double run = before;
        for (int t0 = begin; t0 < end && found < 0; t0 += 64) {
            const int t = t0 + lane;
            const double v = t < end ? w.of(t) : 0.0;
            double upto = v;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const double o = __shfl_up(upto, off, 64);
                if (lane >= off) upto += o;
            }
            const uint64_t over = __ballot(run + upto > want && v > 0.0), some = __ballot(v > 0.0);
            if (over && !past) found = t0 + (int)__builtin_ctzll(over);
            if (some) positive = t0 + 63 - (int)__builtin_clzll(some);
            run += __shfl(upto, 63, 64);
        }
        if (lane == 0) first = found >= 0 ? found : positive;
    }
    __syncthreads();
    if (threadIdx.x <= a.n_drafts && threadIdx.x < 64) {
        const int i = threadIdx.x;
        tokens[i] = i < r ? x : i > r ? -1 : mine < 0 ? -1 : first;
    }
    if (threadIdx.x == 0) a.n_accepted[s] = r;
}

}  // namespace

hipError_t launch_verify(const ls_verify_args& a, void* ws, size_t ws_bytes, int n_cu, hipStream_t st) {
    (void)ws, (void)ws_bytes, (void)n_cu;
    const VerifyP p{a};
    const dim3 grid(a.n_seqs), wg(kVerifyThreads);
    if (a.type == LS_F32)
        hipLaunchKernelGGL((verify_kernel<float>), grid, wg, 0, st, p);
    else if (a.type == LS_F16)
        hipLaunchKernelGGL((verify_kernel<_Float16>), grid, wg, 0, st, p);
    else
        hipLaunchKernelGGL((verify_kernel<__bf16>), grid, wg, 0, st, p);
    return hipGetLastError();
}

}  // namespace ls

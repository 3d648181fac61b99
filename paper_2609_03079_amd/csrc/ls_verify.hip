// ls_verify.hip - drafted tokens against the target's probabilities.
//
//   draft i is accepted while u_i q_i(x_i) < p_i(x_i); the token after the last accepted one comes from
//   w = max(p_r - q_r, 0) where draft r was refused, from w = p_n behind the last draft:
//   the first token whose running sum of w exceeds u sum(w).
//
// Everything that decides is computed in 64 bits: the products of the comparison are exact there, and running sums of
// 131072 terms are off by 2^-36 of their total at most, so a token does not depend on the order they are summed in
// (in 32 bits one number in forty would fall on another token).
//
// Only the row that the token comes from is read, or the two.  They are cut into parts, so that the few sequences of a step fill
// the card: a first launch adds the parts (bound by reading them), a second finds the part that u sum(w) falls into and the
// token in it.  With as many sequences as fill the card by themselves, or rows of up to 8192 tokens, a workgroup does both: a launch
// less (4000 tokens 9.5 -> 7.5 us, where 16000 would go from 9.1 to 10.1).  Measured: 1 x 4 drafts of 32000 (fp32) 9.5 us, most of it
// the two launches; 64 x 7 of 131072 20.3 us, of which the sums 14 (4.7 TB/s of the rows that they read).  Rows that do not all begin at
// multiples of 16 bytes (an odd vocabulary) are read an element a lane, eight in flight: 64 x 7 of 131071 23.7 us, in bfloat16 18.6
// against 17.2 of 131072.
#include <algorithm>

#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {
namespace {

struct VerifyP {
    ls_verify_args a;
    int chunk, chunks;   // tokens of a part, parts of a row
    bool vec;            // rows begin at multiples of 16 bytes
    double* sums;        // [n_seqs][chunks]
    int32_t* accepted;   // [n_seqs]: drafts accepted
    int32_t* refused;    // [n_seqs]: the draft that was refused, -1 where its id is none or none was
};

// Sum over the lanes of a wave, the same in every lane.
__device__ inline double wave_sum64(double v) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// What a row gives its tokens: no number and what is below zero give none, infinities as the largest number.
template <typename T>
struct Weights {
    const T* p;
    const T* q;   // NULL: nothing is taken off, but for `token`
    int token;    // -1: none
    __device__ inline double weight(float x, float y, int t) const {
        const double d = (double)x - (q ? (double)y : t == token ? 1.0 : 0.0);
        return d > 0.0 ? fmin(d, 3.4028234663852886e38) : 0.0;
    }
    __device__ inline double of(int t) const { return weight((float)p[t], q ? (float)q[t] : 0.f, t); }

    // This thread's share of the sum over [begin, end): every N-th token, or every N-th 16 bytes of them (vec; begin is a multiple).
    template <int N>
    __device__ inline double sum(int thread, int begin, int end, bool vec) const {
        constexpr int V = 16 / sizeof(T), U = 16 / V;  // a wave's 1024 tokens at a time
        double s = 0.0;
        int t = begin;
        if (vec) {
            for (; end - t >= N * V * U; t += N * V * U) {
                Pack<T, V> x[U], y[U] = {};
#pragma unroll
                for (int k = 0; k < U; ++k) x[k] = load_pack<T, V>(p, t + (k * N + thread) * V);
                if (q) {
#pragma unroll
                    for (int k = 0; k < U; ++k) y[k] = load_pack<T, V>(q, t + (k * N + thread) * V);
                }
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) s += weight((float)x[k].e[i], (float)y[k].e[i], t + (k * N + thread) * V + i);
            }
            for (; t + (thread + 1) * V <= end; t += N * V) {
                const auto x = load_pack<T, V>(p, t + thread * V);
                Pack<T, V> y{};
                if (q) y = load_pack<T, V>(q, t + thread * V);
#pragma unroll
                for (int i = 0; i < V; ++i) s += weight((float)x.e[i], (float)y.e[i], t + thread * V + i);
            }
            t = end - (end - begin) % V;  // fewer than V are left
            if (thread < end - t) s += of(t + thread);
            return s;
        }
        for (; end - t >= N * 8; t += N * 8) {
            float x[8], y[8] = {};
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = (float)p[t + k * N + thread];
            if (q) {
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = (float)q[t + k * N + thread];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) s += weight(x[k], y[k], t + k * N + thread);
        }
        for (; t + thread < end; t += N) s += of(t + thread);
        return s;
    }
};

// Of a wave's lanes: r of sequence s, and the id that was refused.
__device__ inline int drafts_of(const ls_verify_args& a, int s) { return a.counts ? min(a.counts[s], a.n_drafts) : a.n_drafts; }

template <typename T>
__device__ inline int decide(const ls_verify_args& a, int64_t s, int n, int* id) {
    const int lane = threadIdx.x & 63;
    bool accepted = false;
    int x = -1;
    if (lane < n) {  // lane i decides about draft i
        x = a.drafts[s * a.drafts_stride + lane];
        const float u = a.accept[s * a.accept_stride + lane];
        if (x >= 0 && x < a.vocab) {
            const T* p = static_cast<const T*>(a.target) + s * a.target_seq_stride + lane * a.target_token_stride;
            double q = 1.0;
            if (a.draft) q = (float)static_cast<const T*>(a.draft)[s * a.draft_seq_stride + lane * a.draft_token_stride + x];
            accepted = (double)u * q < (double)(float)p[x];
        }
    }
    const uint64_t not_taken = ~__ballot(accepted);  // n <= 63: never zero
    const int r = min(n, (int)__builtin_ctzll(not_taken));
    *id = r < n ? __shfl(x, r, 64) : -1;
    return r;
}

template <typename T>
__device__ inline Weights<T> weights_of(const ls_verify_args& a, int64_t s, int n, int r, int id) {
    const T* p = static_cast<const T*>(a.target) + s * a.target_seq_stride + r * a.target_token_stride;
    if (r == n) return {p, nullptr, -1};
    if (!a.draft) return {p, nullptr, id};
    return {p, static_cast<const T*>(a.draft) + s * a.draft_seq_stride + r * a.draft_token_stride, -1};
}

// What a sampled number stands for among weights of a total; past: the last token with a weight.
__device__ inline double wanted(float u, double total, bool* past) {
    *past = !(u < 1.f);
    return (u > 0.f ? (double)u : 0.0) * total;
}

// Among N threads with a sum each, in order: the first that has one and takes the running sum (which starts at `before`) over
// `want`, or the last that has one, if none does or `past`.  -1: no thread has one.  *upto: the running sum before it.
template <int N>
__device__ inline int pick(double sum, double before, double want, bool past, double* upto) {
    __shared__ double waves[N / 64];
    __shared__ double run_before;
    __shared__ int over, some;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double run = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    __syncthreads();  // whoever read these last is done
    if (lane == 63) waves[wave] = run;
    if (threadIdx.x == 0) over = N, some = -1;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before += waves[w];
    const double first = __shfl_up(run, 1, 64);
    const double mine = lane ? before + first : before;
    const uint64_t crossed = past ? 0 : __ballot(sum > 0.0 && before + run > want), any = __ballot(sum > 0.0);
    if (lane == 0) {
        if (crossed) atomicMin(&over, wave * 64 + (int)__builtin_ctzll(crossed));
        if (any) atomicMax(&some, wave * 64 + 63 - (int)__builtin_clzll(any));
    }
    __syncthreads();
    const int at = over < N ? over : some;
    if ((int)threadIdx.x == at) run_before = mine;
    __syncthreads();
    *upto = at >= 0 ? run_before : before;
    return at;
}

// The token of [begin, end) by N threads, each a run of it; -1 where nothing there has a weight.
template <int N, typename T>
__device__ inline int token_in(const Weights<T>& w, int begin, int end, double before, double want, bool past) {
    __shared__ int found;
    const int per = (int)(((int64_t)end - begin + N - 1) / N);
    const int b = (int)min((int64_t)end, (int64_t)begin + (int64_t)per * threadIdx.x), e = min(end, b + per);
    double sum = 0.0, run;
    for (int t = b; t < e; t += 4) {  // four at a time: their reads do not wait for each other
        double v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = w.of(min(t + i, e - 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += t + i < e ? v[i] : 0.0;
    }
    const int at = pick<N>(sum, before, want, past, &run);
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    if ((int)threadIdx.x == at) {
        int last = -1, hit = -1;
        for (int t = b; t < e && hit < 0; t += 4) {
            double v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = w.of(min(t + i, e - 1));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (t + i >= e || !(v[i] > 0.0) || hit >= 0) continue;
                run += v[i];
                last = t + i;
                if (!past && run > want) hit = t + i;
            }
        }
        found = hit >= 0 ? hit : last;
    }
    __syncthreads();
    return found;
}

// tokens and n_accepted of a sequence, by the first wave or more
__device__ inline void write_out(const ls_verify_args& a, int64_t s, int r, int token) {
    const int i = threadIdx.x;
    if (i <= a.n_drafts) a.tokens[s * a.tokens_stride + i] = i < r ? a.drafts[s * a.drafts_stride + i] : i == r ? token : -1;
    if (i == 0) a.n_accepted[s] = r;
}

// One workgroup a sequence.  Each wave adds a run of the vocabulary; the workgroup looks through the run that the token is in.
constexpr int kWhole = 1024, kWaves = kWhole / 64;

template <typename T>
__global__ __launch_bounds__(kWhole) void verify_kernel(const VerifyP p, int first_seq) {
    const ls_verify_args& a = p.a;
    __shared__ double sums[kWaves];
    const int s = first_seq + blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = drafts_of(a, s);
    if (n < 0) return write_out(a, s, -1, -1);  // an idle slot
    int id;
    const int r = decide<T>(a, s, n, &id);
    Weights<T> w = weights_of<T>(a, s, n, r, id);
    const int64_t per = ((int64_t)a.vocab + kWhole * 8 - 1) / (kWhole * 8) * 512;  // whole vectors of 64 lanes
    auto begin_of = [&](int i) { return (int)min((int64_t)a.vocab, i * per); };
    double total = 0.0;
    for (int pass = 0;; ++pass) {
        const double sum = wave_sum64(w.template sum<64>(lane, begin_of(wave), begin_of(wave + 1), p.vec));
        __syncthreads();
        if (lane == 0) sums[wave] = sum;
        __syncthreads();
        total = 0.0;
        for (int i = 0; i < kWaves; ++i) total += sums[i];
        if (total > 0.0 || pass) break;
        w.q = nullptr, w.token = -1;  // nothing is left over: the target's own
    }
    bool past;
    const double want = wanted(a.sample[s], total, &past);
    double before = 0.0, last_before = 0.0;
    int at = -1, last = -1;
    for (int i = 0; i < kWaves && at < 0; ++i) {
        if (sums[i] > 0.0) last = i, last_before = before;
        if (!past && sums[i] > 0.0 && before + sums[i] > want) at = i;
        if (at < 0) before += sums[i];
    }
    if (at < 0) at = last, before = last_before;
    const int token = at < 0 ? -1 : token_in<kWhole>(w, begin_of(at), begin_of(at + 1), before, want, past);
    write_out(a, s, r, token);
}

// A wave adds a part: four of them are a workgroup, blockIdx.y is the sequence.
constexpr int kPart = 256;

template <typename T>
__global__ __launch_bounds__(kPart) void verify_sum_kernel(const VerifyP p) {
    const ls_verify_args& a = p.a;
    const int s = blockIdx.y, n = drafts_of(a, s);
    if (n < 0) return;
    int id;
    const int r = decide<T>(a, s, n, &id);
    const int part = blockIdx.x * (kPart / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (part == 0 && lane == 0) p.accepted[s] = r, p.refused[s] = id;
    if (part >= p.chunks) return;
    const Weights<T> w = weights_of<T>(a, s, n, r, id);
    const int begin = part * p.chunk, end = (int)min((int64_t)a.vocab, (int64_t)begin + p.chunk);
    const double sum = wave_sum64(w.template sum<64>(lane, begin, end, p.vec));
    if (lane == 0) p.sums[(int64_t)s * p.chunks + part] = sum;
}

template <typename T>
__global__ __launch_bounds__(kPart) void verify_token_kernel(const VerifyP p) {
    const ls_verify_args& a = p.a;
    __shared__ double waves[kPart / 64];
    const int s = blockIdx.x, n = drafts_of(a, s);
    if (n < 0) return write_out(a, s, -1, -1);
    const int r = p.accepted[s], id = p.refused[s];
    Weights<T> w = weights_of<T>(a, s, n, r, id);
    const double* sums = p.sums + (int64_t)s * p.chunks;
    // a thread has a few parts that follow each other
    const int per = (p.chunks + kPart - 1) / kPart, b = min(p.chunks, per * (int)threadIdx.x), e = min(p.chunks, b + per);
    double mine = 0.0;
    for (int i = b; i < e; ++i) mine += sums[i];
    double total = wave_sum64(mine);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = total;
    __syncthreads();
    total = (waves[0] + waves[1]) + (waves[2] + waves[3]);
    bool past;
    int token = -1;
    if (!(total > 0.0)) {  // nothing is left over: the target's own, once more from the start
        if (r < n) {
            w.q = nullptr, w.token = -1;
            const double sum = wave_sum64(w.template sum<kPart>(threadIdx.x, 0, a.vocab, p.vec));
            __syncthreads();
            if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
            __syncthreads();
            total = (waves[0] + waves[1]) + (waves[2] + waves[3]);
            const double want = wanted(a.sample[s], total, &past);
            if (total > 0.0) token = token_in<kPart>(w, 0, a.vocab, 0.0, want, past);
        }
        return write_out(a, s, r, token);
    }
    const double want = wanted(a.sample[s], total, &past);
    double before;
    __shared__ int part;
    __shared__ double part_before;
    const int at = pick<kPart>(mine, 0.0, want, past, &before);
    if ((int)threadIdx.x == at) {  // of its parts the one
        int last = -1;
        double last_before = before, run = before;
        for (int i = b; i < e; ++i) {
            if (sums[i] > 0.0) {
                last = i, last_before = run;
                if (!past && run + sums[i] > want) break;
            }
            run += sums[i];
        }
        part = last, part_before = last_before;
    }
    __syncthreads();
    const int begin = part * p.chunk;
    token = token_in<kPart>(w, begin, (int)min((int64_t)a.vocab, (int64_t)begin + p.chunk), part_before, want, past);
    write_out(a, s, r, token);
}

template <typename T>
hipError_t verify_type(VerifyP p, void* ws, size_t ws_bytes, int n_cu, hipStream_t st) {
    const ls_verify_args& a = p.a;
    const int64_t el = 16 / (int64_t)sizeof(T);
    p.vec = aligned(a.target, 16) && a.target_seq_stride % el == 0 && a.target_token_stride % el == 0 &&
            (!a.draft || (aligned(a.draft, 16) && a.draft_seq_stride % el == 0 && a.draft_token_stride % el == 0));
    // Parts of 1024 tokens, larger where they are more waves than run in two rounds (256 rows of 128256 in bf16:
    // 52 -> 33 us), or the workspace or a thread's share of them (8) would not do.
    const int64_t bytes = (int64_t)a.n_seqs * 8;  // what a part of each row takes; the decisions as much once
    const int64_t at_once = std::max<int64_t>(1, 64 * n_cu / a.n_seqs);
    const int64_t chunks = std::min({ceil_div(a.vocab, 1024), at_once, (int64_t)ws_bytes / bytes - 1, (int64_t)(8 * kPart)});
    if (a.n_seqs < 2 * n_cu && a.vocab > 8192 && chunks > 1) {
        p.chunk = (int)round_up((size_t)ceil_div(a.vocab, chunks), 1024);
        p.chunks = (int)ceil_div(a.vocab, p.chunk);
        p.sums = static_cast<double*>(ws);
        p.accepted = reinterpret_cast<int32_t*>(p.sums + (int64_t)a.n_seqs * p.chunks);
        p.refused = p.accepted + a.n_seqs;
        hipLaunchKernelGGL((verify_sum_kernel<T>), dim3((unsigned)ceil_div(p.chunks, kPart / 64), a.n_seqs), dim3(kPart), 0, st, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((verify_token_kernel<T>), dim3(a.n_seqs), dim3(kPart), 0, st, p);
        return hipGetLastError();
    }
    constexpr int kSeqs = 1 << 21;  // a launch holds fewer than 2^32 threads
    for (int64_t s = 0; s < a.n_seqs; s += kSeqs) {
        hipLaunchKernelGGL((verify_kernel<T>), dim3((unsigned)std::min<int64_t>(kSeqs, a.n_seqs - s)), dim3(kWhole), 0, st, p, (int)s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_verify(const ls_verify_args& a, void* ws, size_t ws_bytes, int n_cu, hipStream_t st) {
    const VerifyP p{a, 0, 0, false, nullptr, nullptr, nullptr};
    return a.type == LS_F32   ? verify_type<float>(p, ws, ws_bytes, n_cu, st)
           : a.type == LS_F16 ? verify_type<_Float16>(p, ws, ws_bytes, n_cu, st)
                              : verify_type<__bf16>(p, ws, ws_bytes, n_cu, st);
}

}  // namespace ls

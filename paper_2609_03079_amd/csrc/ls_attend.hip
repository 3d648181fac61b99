// ls_attend.hip - attention of a batch that shares a prefix, over a paged cache.
//
//   o_r = sum_j p_rj v_j,   p_rj = exp(scale q_r k_j - m_r) / l_r,   r a query row of one key/value head
//
// The prefix's keys serve the rows of every sequence at once (n_seqs n_q G rows per key/value head,
// G query heads sharing it), a sequence's own keys its n_q G rows.  Both are cut along the keys
// into parts; each part keeps the running maximum, sum l and sum of weighted values of its rows
// (one pass over the keys), and a second kernel joins the parts of a row.  What is kept of the
// maximum is m = max scale log2(e) q k - kLift, rounded: the number that the weights are taken relative
// to, so that a maximum that stays rescales by exactly one, whatever the rows beside it do.
//
// The products run transposed, S^T = K Q^T and O^T = V^T P^T, on the 32 x 32 x 16 matrix
// instructions: a lane then holds one query row's scores, 16 of each 32 keys, so the softmax
// needs one exchange with the lane that holds the other 16, and the scores become the second
// product's operand in place: both products may take the keys in any order as long as it is the
// same, and the values are read from shared memory (transposed on the way) in the order in which
// the scores lie.
//
// Two shapes of workgroup:
//  - wide: four waves of 32 rows share 64 keys in shared memory, the scores of the next 64 computed
//    while the exponentials of these are: bound by the vector and matrix units together (64
//    sequences, 64 query and 8 key heads of 128 bfloat16, 32768 prefix keys: 93 to 107 us, 68.7
//    GFLOP, the matrix units busy for two fifths of it; 79 without any copies);
//  - narrow (up to 32 rows): two waves, each taking every second 32 keys through its own share of
//    shared memory, without barriers, the waves' results joined at the end: bound by each wave's
//    chain of copy, products, exponentials and products (the same 64 sequences' own keys, 512 to
//    1024 each: 44 us, 200 MB at 4.6 TB/s) and, for few keys, by its start: table, page, keys and
//    the first products wait for each other, about 5.5 us.  Asking for keys and values two tiles
//    ahead in place of one changed nothing there.
// In both the next keys are copied straight to shared memory while the present ones are used.
//
// Registers, with 512 a lane for one wave a SIMD and 256 for two: the kernels of one token spill 5 to 7 at
// heads of 128, held to two; a path that takes a sequence's tokens one by one (for values that
// are no numbers) costs the kernels of several tokens more, 62 to 65 spilled where a wide prefix
// runs beside narrow sequences at heads of 128, 110 to 127 at heads of 256, and its own
// launch of wide workgroups runs one of them a compute unit at heads of up to 128, where the others run two.
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
typedef __attribute__((address_space(1))) void* gptr;
typedef __attribute__((address_space(3))) void* lptr;

// What masked keys and the padding of a head are read from: a row of zeros.
__device__ const uint32_t g_zero_row[128] = {};

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
    int64_t page_stride, head_stride, token_stride;
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
    int parts;               // partial results per row
    bool direct;             // a row has one part, which is the result
    float* part;             // [rows][parts][D]
    float* ml;               // [rows][parts][2]
};

// Chunks (8 elements, 16 bytes) of a row lie at places permuted by its number, so that neither
// 16 rows at one chunk (keys) nor 4 rows at 4 chunks (values) meet in a bank.
template <int CPR>
__device__ inline int swz(int row) {
    return CPR == 8 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
}

template <typename T, int DP, bool WIDE>
struct Shape {
    // The largest weight is 2^kLift.  Weights enter the second product in 16 bits (in 32 the product
    // would run at a sixteenth of the rate), and with a largest of one float16 would drop those below 2^-25,
    // which the sum counts: 30000 keys that far below one that dominates are a thousandth of the
    // result.  With 2^7 those below 2^-32 are dropped, a part's 65536 at most a 2^-16th; what is left
    // of the type's range is for a maximum that was rounded (by 2^8 at most while |m| < 2^28).
    static constexpr float kLift = std::is_same_v<T, _Float16> ? 7.f : 0.f;
    static constexpr int NW = WIDE ? 4 : 2;                     // waves
    static constexpr int KT = WIDE && DP < 256 ? 64 : 32;       // keys at a time
    static constexpr int CPR = DP / 8;                          // chunks per row
    static constexpr int RPI = 64 / CPR;                        // rows per copy instruction
    static constexpr int kRows = WIDE ? KT / NW : KT;           // rows a wave copies
    static constexpr int kBuf = (WIDE ? 1 : NW) * KT * DP;      // elements of a buffer, of keys or of values
    static constexpr int kTileRows = WIDE ? 128 : 32;
};

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

// MULTI: sequences with several query tokens each, whose last keys only some of them see.
// The four arrays are four, not one: a read of one must not wait for the copy into another.
template <typename T, int DP, bool WIDE, bool MULTI>
__device__ __forceinline__ void attend(const AttendP& p, bool prefix, int b, T* k0, T* k1, T* v0, T* v1, float (*wave_ml)[2][32],
                                       float* row_sum) {
    using Sh = Shape<T, DP, WIDE>;
    constexpr bool PIPE = WIDE && !MULTI;  // scores one tile ahead (MULTI's rare path leaves no registers)
    constexpr int NW = Sh::NW, KT = Sh::KT, CPR = Sh::CPR, NF = DP / 16, ND = DP / 32, SUB = KT / 32;
    Item it;
    if (!item_of<Sh::kTileRows>(p, prefix, b, &it)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, h = lane >> 5;

    // The first page ids are on their way before the sequence's length is known: the table holds
    // max_len keys.  Each lane looks up one key of a tile; -1 where there is none.
    constexpr int kStep = WIDE ? KT : NW * KT;
    int key = it.begin + (WIDE ? 0 : wave * KT);
    auto page_id = [&](int key0) {
        const int at = key0 + (lane & (KT - 1));
        return at < it.end ? it.table[at >> p.page_shift] : -1;
    };
    const int first0 = page_id(key), first1 = page_id(key + kStep);
    int id2 = page_id(key + 2 * kStep);
    it.len = it.seq < 0 ? p.prefix_len : min(p.lens[it.seq], p.max_len);
    it.end = min(it.end, it.len);
    if (it.begin >= it.end && !p.direct) return;

    // this lane's query row: token and head of it, keys it sees
    const int row = it.row0 + (WIDE ? wave * 32 : 0) + n;
    const bool row_ok = row < it.rows;
    const int rr = row_ok ? row : it.rows - 1;
    const int tk = p.by_G.of(rr), g = rr - tk * p.G;  // token of the batch (prefix) or of the sequence
    const int64_t token = it.seq < 0 ? tk : (int64_t)it.seq * p.n_q + tk;
    const int head = it.kv * p.G + g;
    const int limit = it.seq < 0 ? it.end : min(it.end, it.len - p.n_q + 1 + tk);
    // keys below are seen by every row (of a sequence; of its part)
    const int full_len = it.seq < 0 ? it.end : it.len - p.n_q + 1, full = min(it.end, full_len);

    vec8<T> q[NF];
    {
        const T* src = static_cast<const T*>(p.q) + token * p.q_token + head * p.q_head;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int d = f * 16 + h * 8;
            q[f] = row_ok && d < p.D ? *reinterpret_cast<const vec8<T>*>(src + d) : vec8<T>{};
        }
    }
    f32x16 o[ND];
#pragma unroll
    for (auto& x : o) x = f32x16{};
    float m = -INFINITY, l = 0.f;

    const T* kbase = static_cast<const T*>(p.k) + it.kv * p.head_stride;
    const T* vbase = static_cast<const T*>(p.v) + it.kv * p.head_stride;
    const T* zero = reinterpret_cast<const T*>(g_zero_row);
    const int page_mask = (1 << p.page_shift) - 1;

    // A key's place in the cache, in elements, -1 where it is masked.
    auto place = [&](int key0, int id) {
        const int key = key0 + (lane & (KT - 1));
        const int64_t at = (int64_t)id * p.page_stride + (int64_t)(key & page_mask) * p.token_stride;
        return (unsigned)id < (unsigned)p.n_pages && key < it.end ? at : (int64_t)-1;
    };
    // Copies a tile's rows, RPI of them an instruction: lane -> row lane / CPR, chunk lane % CPR permuted.
    // 16 rows that are all there lie in one page (of 16 keys or more): one address for the wave and
    // fixed places for the lanes.  Otherwise each lane asks the row's lane for its address.
    const int c_row = lane / CPR;
    const bool regular = page_mask >= 15 && p.D == DP && p.token_stride < 1 << 24;
    uint32_t c_at[16 / Sh::RPI];  // bytes
#pragma unroll
    for (int i = 0; i < 16 / Sh::RPI; ++i) {
        const int r = i * Sh::RPI + c_row;
        c_at[i] = ((uint32_t)r * (uint32_t)p.token_stride + ((lane % CPR) ^ swz<CPR>(r)) * 8) * sizeof(T);
    }
    auto copy = [&](const T* base, int64_t at, T* buf) {
        T* dst = buf + wave * Sh::kRows * DP;
        const int first = WIDE ? wave * Sh::kRows : 0;
        const uint32_t all = Sh::kRows == 32 ? ~0u : (1u << Sh::kRows % 32) - 1;
        if (Sh::kRows % 16 == 0 && regular && ((uint32_t)(__ballot(at >= 0) >> first) & all) == all) {
#pragma unroll
            for (int g = 0; g < Sh::kRows / 16; ++g) {
                const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)at, first + g * 16);
                const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(at >> 32), first + g * 16);
                const char* rows = reinterpret_cast<const char*>(base + (int64_t)(((uint64_t)hi << 32) | lo));
#pragma unroll
                for (int i = 0; i < 16 / Sh::RPI; ++i)
                    __builtin_amdgcn_global_load_lds((gptr)(rows + c_at[i]), (lptr)(dst + g * 16 * DP + i * 512), 16, 0, 0);
            }
            return;
        }
        const uint64_t from = (uint64_t)(at < 0 ? zero : base + at);
#pragma unroll
        for (int i = 0; i < Sh::kRows / Sh::RPI; ++i) {
            const int r0 = first + i * Sh::RPI;
            const int chunk = (lane % CPR) ^ swz<CPR>(c_row) ^ swz<CPR>(r0);  // the bits of the two do not mix
            const uint32_t lo = __shfl((uint32_t)from, r0 + c_row, 64), hi = __shfl((uint32_t)(from >> 32), r0 + c_row, 64);
            const T* row = reinterpret_cast<const T*>(((uint64_t)hi << 32) | lo);
            __builtin_amdgcn_global_load_lds((gptr)(chunk * 8 < p.D ? row + chunk * 8 : zero), (lptr)(dst + i * 512), 16, 0, 0);
        }
    };
    // Where this lane finds its operands in a tile, in elements: key u * 32 + n, chunk 2 f + h; and for
    // the values element d = 32 t + n of keys 16 kk + 4 h + 0 .. 3 and + 8 (read by fours, transposed).
    const int k_at = n * DP + (h ^ swz<CPR>(n)) * 8;  // chunk bits of f are flipped in
    const int r4 = (lane & 15) >> 2, col = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const int v_at = (4 * h + r4) * DP + (col ^ swz<CPR>(4 * h + r4)) * 8 + (lane & 1) * 4;
    const int v_at8 = (4 * h + r4 + 8) * DP + (col ^ swz<CPR>(4 * h + r4 + 8)) * 8 + (lane & 1) * 4;
    const bool idle_wave = WIDE && it.row0 + wave * 32 >= it.rows;  // no rows: it only copies
    struct Scores {
        f32x16 u[SUB];
        float top;  // the largest of the lane's
    };
    auto largest = [](Scores& s) {
        float top = s.u[0][0];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s.u[u][i]);
        s.top = top;
    };
    auto scores = [&](const T* buf) {
        const T* kt = buf + (WIDE ? 0 : wave * KT * DP);
        Scores s;
#pragma unroll
        for (int u = 0; u < SUB; ++u) s.u[u] = f32x16{};
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int u = 0; u < SUB; ++u)
                s.u[u] = mma(*reinterpret_cast<const vec8<T>*>(kt + (k_at ^ (f * 16)) + u * 32 * DP), q[f], s.u[u]);
        return s;
    };
    // One tile.  PIPE: its scores are in s already, and those of the next tile (keys in kbuf) are
    // computed while its exponentials are: matrix and vector instructions of one wave run side by
    // side, so the next maximum is part of the same stretch of code.
    auto use = [&](Scores& s, int key0, int64_t at, const T* vbuf, const T* kbuf) {
        if (!PIPE) {
            s = scores(kbuf);
            largest(s);
        }
        const T* vt = vbuf + (WIDE ? 0 : wave * KT * DP);
        // score i of a lane belongs to key 8 (i / 4) + 4 h + i % 4 of its 32
        const uint64_t valid = __ballot(at >= 0);
        if (key0 + KT > full || (KT == 64 ? ~valid != 0 : (uint32_t)~valid != 0)) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const int left = limit - key0 - u * 32;  // keys of these 32 that the row sees
                const uint32_t below = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1;
                const uint32_t seen = (below & (uint32_t)(valid >> (u * 32))) >> (4 * h);
#pragma unroll
                for (int i = 0; i < 16; ++i) s.u[u][i] = (seen >> (8 * (i / 4) + i % 4)) & 1 ? s.u[u][i] : -INFINITY;
            }
            largest(s);
        }
        const float top = fmaxf(s.top, other_half(s.top));
        const float next = fmaxf(m, top * p.c - Sh::kLift), base = next == -INFINITY ? 0.f : next;
        if (__any(next > m)) {
            const float scale = __builtin_amdgcn_exp2f(m - base);  // m = -inf: 0
            l *= scale;
#pragma unroll
            for (auto& x : o) x *= scale;
            m = next;
        }
        Scores after;
        if (PIPE) after = scores(kbuf);
        vec8<T> pr[2 * SUB];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(s.u[u][i], p.c, -base));
                l += e;
                pr[2 * u + i / 8][i % 8] = (T)e;
            }
        auto value = [&](int kk, int t) {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const T* at = vt + kk * 16 * DP;
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + (v_at ^ (t * 32))));
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + (v_at8 ^ (t * 32))));
            struct { s16x4 a, b; } both{x, y};
            return __builtin_bit_cast(vec8<T>, both);
        };
        bool odd = false;
        // Where later tokens of a sequence see keys that earlier ones do not, a weight of zero must
        // also keep out a value that is no number: only then are the tokens taken one by one.
        if (MULTI && it.seq >= 0 && key0 + KT > full) {
#pragma unroll 1
            for (int kk = max(0, full - key0) / 16; kk < 2 * SUB && key0 + 16 * kk < it.end; ++kk)
#pragma unroll
                for (int t = 0; t < ND; ++t) {
                    const auto v = value(kk, t);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        odd |= key0 + 16 * kk + 8 * (j / 4) + 4 * h + j % 4 >= full && !(fabsf((float)v[j]) < INFINITY);
                }
        }
        if (MULTI && __any(odd)) {
#pragma unroll 1
            for (int i = 0; i < p.n_q; ++i) {
                const int seen = full_len + i;
#pragma unroll
                for (int t = 0; t < ND; ++t) {
                    __builtin_amdgcn_sched_barrier(0);  // one tile's operands at a time: registers
                    f32x16 x = o[t];
#pragma unroll
                    for (int kk = 0; kk < 2 * SUB; ++kk) {
                        auto v = value(kk, t);
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (key0 + 16 * kk + 8 * (j / 4) + 4 * h + j % 4 >= seen) v[j] = (T)0.f;
                        x = mma(v, pr[kk], x);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[t][e] = tk == i ? x[e] : o[t][e];
                }
            }
        } else {
#pragma unroll
            for (int kk = 0; kk < 2 * SUB; ++kk)
#pragma unroll
                for (int t = 0; t < ND; ++t) o[t] = mma(value(kk, t), pr[kk], o[t]);
        }
        if (PIPE) {
            s = after;
            largest(s);
        }
    };
    auto landed = [&] {
        __builtin_amdgcn_s_waitcnt(0x0070);  // this wave's copies are in shared memory, its reads done
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        if (WIDE) __builtin_amdgcn_s_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    };

    // While tile j is used, V of j + 1 and K of j + 1 (PIPE: j + 2) arrive.  Past the end PIPE
    // copies and multiplies tiles of zeros; nothing uses their scores.
    if (key < it.end) {
        int64_t at0 = place(key, first0), at1 = place(key + kStep, first1);
        copy(kbase, at0, k0);
        copy(vbase, at0, v0);
        Scores s;
        if (PIPE) {
            copy(kbase, at1, k1);
            landed();
            s = scores(k0);
            largest(s);
        }
        auto tile = [&](T* ka, T* kb, T* va, T* vb) {  // K of j + 1 in kb (else of j in ka), V of j in va
            const int64_t at2 = place(key + 2 * kStep, id2);
            landed();
            id2 = page_id(key + 3 * kStep);
            if (PIPE || key + kStep < it.end) {
                copy(kbase, PIPE ? at2 : at1, PIPE ? ka : kb);
                copy(vbase, at1, vb);
            }
            if (!idle_wave) use(s, key, at0, va, PIPE ? kb : ka);
            key += kStep;
            at0 = at1, at1 = at2;
        };
        for (;;) {
            tile(k0, k1, v0, v1);
            if (key >= it.end) break;
            tile(k1, k0, v1, v0);
            if (key >= it.end) break;
        }
        landed();  // nothing is under way when the arrays are used again
    }
    l += other_half(l);

    const int64_t out_row = token * p.H + head;
    // four elements of a row: the part's sums, or with a single part the result
    auto put = [&](int64_t token_, int head_, int d, f32x4 x, float row_l) {
        if (d >= p.D) return;
        if (p.direct) {
            const float inv = row_l == 0.f ? 0.f : 1.f / row_l;
            Pack<T, 4> v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v.e[i] = (T)(x[i] * inv);
            store_pack<T, 4>(p.out, token_ * p.o_token + head_ * p.o_head + d, v);
        } else {
            *reinterpret_cast<f32x4*>(p.part + ((token_ * p.H + head_) * p.parts + it.part) * p.D + d) = x;
        }
    };
    auto put_ml = [&](float row_m, float row_l) {
        if (p.direct) return;
        float* at = p.ml + (out_row * p.parts + it.part) * 2;
        at[0] = row_m;
        at[1] = row_l;
    };
    if (WIDE) {
        if (!row_ok) return;
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : o[t][i + e];
                put(token, head, t * 32 + 2 * i + 4 * h, x, l);
            }
        if (h == 0) put_ml(m, l);
        return;
    }
    // narrow: join the waves
    if (h == 0) {
        wave_ml[wave][0][n] = m;
        wave_ml[wave][1][n] = l;
    }
    __syncthreads();  // also: every wave is done with its buffers
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, wave_ml[w][0][n]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float wl = wave_ml[w][1][n];
        if (wl != 0.f) sum += wl * __builtin_amdgcn_exp2f(wave_ml[w][0][n] - base);
    }
    // [wave][row][DP], 16-byte chunks permuted by the row: half of each row in the keys' array, half in the values'
    static_assert(WIDE || Sh::kBuf * sizeof(T) >= NW * 32 * DP / 2 * 4, "room for the waves' sums");
    auto joined = [&](int w, int r, int chunk) {
        const int c = chunk ^ (r & (DP / 4 - 1)), half = DP / 8;
        return reinterpret_cast<f32x4*>(c < half ? k0 : v0) + (w * 32 + r) * half + c % half;
    };
    if (row_ok) {
        const float scale = __builtin_amdgcn_exp2f(m - base);
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int chunk = t * 8 + i / 2 + h;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : o[t][i + e] * scale;
                *joined(wave, n, chunk) = v;
            }
        if (wave == 0 && h == 0) {
            row_sum[n] = sum;
            put_ml(top, sum);
        }
    }
    __syncthreads();
    const int here = min(32, it.rows - it.row0);
    for (int i = threadIdx.x; i < here * (DP / 4); i += NW * 64) {
        const int r = i / (DP / 4), chunk = i % (DP / 4);
        f32x4 v{};
#pragma unroll
        for (int w = 0; w < NW; ++w) v += *joined(w, r, chunk);
        const int tr = p.by_G.of(it.row0 + r);
        put(it.seq < 0 ? tr : (int64_t)it.seq * p.n_q + tr, it.kv * p.G + it.row0 + r - tr * p.G, chunk * 4, v, row_sum[r]);
    }
}

// Which shapes a launch holds.  BOTH: a wide prefix beside narrow sequences, eight workgroups of one after
// eight of the other (one for each XCD).
enum Roles { NARROW, WIDE_ROWS, BOTH };

template <typename T, int DP, Roles ROLES, bool MULTI>
__global__ __launch_bounds__((Shape<T, DP, ROLES != NARROW>::NW * 64), (ROLES != NARROW && DP <= 128 && (ROLES == BOTH || !MULTI) ? 2 : 1)) void attend_kernel(const AttendP p) {
    constexpr int kBuf = ROLES == WIDE_ROWS ? Shape<T, DP, true>::kBuf : Shape<T, DP, false>::kBuf;
    static_assert(Shape<T, DP, false>::kBuf >= Shape<T, DP, true>::kBuf, "room for either shape");
    __shared__ __attribute__((aligned(16))) T k0[kBuf], k1[kBuf], v0[kBuf], v1[kBuf];
    __shared__ float wave_ml[Shape<T, DP, false>::NW][2][32], row_sum[32];
    int b = blockIdx.x;
    if constexpr (ROLES == BOTH) {
        const int both = 2 * min(p.pre_items, p.suf_items / 8 * 8);  // pre_items is a multiple of 8
        bool prefix;
        if (b < both) {
            prefix = !((b >> 3) & 1);
            b = (b >> 4) * 8 + (b & 7);
        } else {
            prefix = b - both / 2 < p.pre_items;
            b -= both / 2;
            if (!prefix) b -= p.pre_items - both / 2;
        }
        if (prefix) {
            attend<T, DP, true, false>(p, true, b, k0, k1, v0, v1, wave_ml, row_sum);
        } else if (threadIdx.x < Shape<T, DP, false>::NW * 64) {
            attend<T, DP, false, MULTI>(p, false, b, k0, k1, v0, v1, wave_ml, row_sum);
        }
    } else {
        const bool prefix = b < p.pre_items;
        attend<T, DP, ROLES == WIDE_ROWS, MULTI>(p, prefix, prefix ? b : b - p.pre_items, k0, k1, v0, v1, wave_ml, row_sum);
    }
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

template <typename T, int DP>
hipError_t attend_type(const ls_kv_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws, hipStream_t st) {
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
    const int pre = (int)round_up(plan.pre_parts * p.KV, 8) * plan.pre_tiles, suf = plan.suf_parts * p.S * p.KV * plan.suf_tiles;
    auto go = [&](Roles roles, int pre_items, int suf_items) {
        p.pre_items = pre_items;
        p.suf_items = suf_items;
        const dim3 grid((unsigned)(pre_items + suf_items)), narrow_wg(Shape<T, DP, false>::NW * 64), wide_wg(256);
        const bool multi = p.n_q > 1 && suf_items;
        if (roles == NARROW) {
            if (multi)
                hipLaunchKernelGGL((attend_kernel<T, DP, NARROW, true>), grid, narrow_wg, 0, st, p);
            else
                hipLaunchKernelGGL((attend_kernel<T, DP, NARROW, false>), grid, narrow_wg, 0, st, p);
        } else if (roles == WIDE_ROWS) {
            if (multi)
                hipLaunchKernelGGL((attend_kernel<T, DP, WIDE_ROWS, true>), grid, wide_wg, 0, st, p);
            else
                hipLaunchKernelGGL((attend_kernel<T, DP, WIDE_ROWS, false>), grid, wide_wg, 0, st, p);
        } else {
            if (multi)
                hipLaunchKernelGGL((attend_kernel<T, DP, BOTH, true>), grid, wide_wg, 0, st, p);
            else
                hipLaunchKernelGGL((attend_kernel<T, DP, BOTH, false>), grid, wide_wg, 0, st, p);
        }
        return hipGetLastError();
    };
    const Roles pre_role = plan.pre_wide ? WIDE_ROWS : NARROW, suf_role = plan.suf_wide ? WIDE_ROWS : NARROW;
    hipError_t e;
    if (pre == 0 || suf == 0 || plan.alike) {
        e = go(pre ? pre_role : suf_role, pre, suf);
    } else if (plan.together) {
        e = go(BOTH, pre, suf);
    } else {
        e = go(pre_role, pre, 0);
        if (e == hipSuccess) e = go(suf_role, 0, suf);
    }
    if (e != hipSuccess || p.direct) return e;
    hipLaunchKernelGGL((join_kernel<T, DP>), dim3((unsigned)rows, (unsigned)ceil_div(p.D, 64)), dim3(64), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t attend_dim(const ls_kv_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws, hipStream_t st) {
    if (c.head_dim <= 64) return attend_type<T, 64>(c, a, plan, ws, st);
    if (c.head_dim <= 128) return attend_type<T, 128>(c, a, plan, ws, st);
    return attend_type<T, 256>(c, a, plan, ws, st);
}

}  // namespace

bool plan_attend(const ls_kv_cache& c, const ls_attend_args& a, size_t ws_bytes, int n_cu, AttendPlan* plan) {
    const int G = a.n_heads / c.n_kv_heads;
    const int64_t pre_rows = (int64_t)a.n_seqs * a.n_q * G, suf_rows = (int64_t)a.n_q * G;
    const int64_t part_bytes = (int64_t)a.n_seqs * a.n_q * a.n_heads * (c.head_dim + 2) * 4;
    plan->pre_wide = pre_rows > 32;
    plan->suf_wide = suf_rows > 32;
    plan->pre_tiles = (int)ceil_div(pre_rows, plan->pre_wide ? 128 : 32);
    plan->suf_tiles = (int)ceil_div(suf_rows, plan->suf_wide ? 128 : 32);
    plan->alike = plan->pre_wide == plan->suf_wide;
    // Workgroups that run at once on a compute unit (by shared memory and registers: wide ones of several tokens
    // take more than half of those); the time of a key and of a start and end, as measured with the unit full (us).
    enum Kind { NARROW_ITEM, WIDE_ITEM, TOKENS_ITEM };
    const Kind pre_kind = plan->pre_wide ? WIDE_ITEM : NARROW_ITEM;
    const Kind suf_kind = !plan->suf_wide ? NARROW_ITEM : a.n_q > 1 && a.max_len ? TOKENS_ITEM : WIDE_ITEM;
    const int wide_cu = c.head_dim <= 128 ? 2 : 1, narrow_cu = c.head_dim <= 64 ? 4 : c.head_dim <= 128 ? 2 : 1;
    const double by_dim = (c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256) / 128.0;
    const double tokens_key = c.head_dim <= 64 ? 0.024 : c.head_dim <= 128 ? 0.038 : 0.139;
    auto item_us = [&](Kind kind, int64_t chunk) {
        return kind == TOKENS_ITEM ? chunk * tokens_key + 4.0 : kind == WIDE_ITEM ? chunk * by_dim * 0.050 + 4.0 : chunk * by_dim * 0.038 + 5.5;
    };
    const double part_us = 2.0 * part_bytes / 5e6;  // written, and read by the join
    // The chunk (a multiple of 128 keys) with the least estimated time, at most half of kMaxParts parts
    // and half of the workspace for each of prefix and sequences: rounds of workgroups, and the parts.
    double least = 0;
    auto choose = [&](Kind kind, int64_t n_pre, int64_t pre_keys, int64_t n_suf, int64_t suf_keys) {
        int64_t best = 0;
        const int64_t slots = (int64_t)n_cu * (kind == TOKENS_ITEM ? 1 : kind == WIDE_ITEM ? wide_cu : narrow_cu);
        const int64_t most = round_up((size_t)std::max<int64_t>(std::max(pre_keys, suf_keys), 1), 128);
        for (int64_t chunk = 128;; chunk = std::min(most, chunk + std::max<int64_t>(128, chunk / 8 / 128 * 128))) {
            const int64_t pp = ceil_div(pre_keys, chunk), sp = ceil_div(suf_keys, chunk), items = n_pre * pp + n_suf * sp;
            const bool fits = pp <= kMaxParts / 2 && sp <= kMaxParts / 2 && std::max(pp, sp) * part_bytes <= (int64_t)ws_bytes / 2 &&
                              (n_pre + 8) * (pp + 8) + n_suf * sp < (int64_t)1 << 24;  // 2^32 threads of a launch
            if (fits) {
                const double t = item_us(kind, chunk) * ceil_div(items, slots) + (pp + sp) * part_us;
                if (!best || t < least) best = chunk, least = t;
            }
            if (chunk >= most) break;
        }
        return (int)best;
    };
    const int64_t n_pre = a.prefix_len ? (int64_t)c.n_kv_heads * plan->pre_tiles : 0;
    const int64_t n_suf = (int64_t)a.n_seqs * c.n_kv_heads * plan->suf_tiles;
    auto at_once = [&](int64_t pre_chunk, int64_t suf_chunk) {  // all workgroups, the prefix's filled up to eights
        return n_pre * ceil_div(a.prefix_len, pre_chunk) + 8 * plan->pre_tiles + n_suf * ceil_div(a.max_len, suf_chunk) <= (int64_t)wide_cu * n_cu;
    };
    if (plan->alike || !a.prefix_len) {
        plan->pre_chunk = plan->suf_chunk = choose(suf_kind, n_pre, a.prefix_len, n_suf, a.max_len);
        // In one launch the prefix, too, goes by the kernel of several tokens; apart where that costs less: 16 sequences
        // of 8 tokens behind 8192 keys, 64 / 8 heads of 128 127 -> 79 us, while 2 behind 500 keys take 24 apart, 15 at once.
        if (suf_kind == TOKENS_ITEM && a.prefix_len) {
            const double one_us = least;
            const int pre_chunk = choose(pre_kind, n_pre, a.prefix_len, 0, 0);
            double apart = least + 2.0;
            const int suf_chunk = choose(suf_kind, 0, 0, n_suf, a.max_len);
            apart += least;
            if (pre_chunk && suf_chunk && (!plan->pre_chunk || apart < one_us)) {
                plan->pre_chunk = pre_chunk, plan->suf_chunk = suf_chunk;
                plan->alike = false;
            }
        }
    } else {
        plan->pre_chunk = choose(pre_kind, n_pre, a.prefix_len, 0, 0);
        double apart = least + 2.0;
        plan->suf_chunk = choose(suf_kind, 0, 0, n_suf, a.max_len);
        apart += least;
        // Longer parts that let both run at once, in one launch, if that costs less than one after the other
        // (33 x 2 tokens behind 5456 keys, 8 heads of 256: 51.5 -> 35.7 us; 18 behind 4417, 16 heads of 64: 24.0 -> 17.8).
        if (plan->pre_wide && plan->pre_chunk && plan->suf_chunk && a.max_len && !at_once(plan->pre_chunk, plan->suf_chunk)) {
            int64_t chunk = round_up((size_t)((n_pre * a.prefix_len + n_suf * a.max_len) / ((int64_t)n_cu * wide_cu) + 1), 128);
            for (int i = 0; i < 8 && !at_once(chunk, chunk); ++i) chunk += 128;
            const int64_t parts = ceil_div(a.prefix_len, chunk) + ceil_div(a.max_len, chunk);
            if (at_once(chunk, chunk) && parts <= kMaxParts && parts * part_bytes <= (int64_t)ws_bytes &&
                std::max(item_us(WIDE_ITEM, chunk), item_us(NARROW_ITEM, chunk)) + parts * part_us < apart)
                plan->pre_chunk = plan->suf_chunk = (int)chunk;
        }
    }
    if (!plan->pre_chunk || !plan->suf_chunk) return false;
    plan->pre_parts = (int)ceil_div(a.prefix_len, plan->pre_chunk);
    plan->suf_parts = (int)ceil_div(a.max_len, plan->suf_chunk);
    if (plan->pre_parts + plan->suf_parts == 0) plan->suf_parts = 1;  // no key anywhere: rows of zeros
    // A wide prefix and narrow sequences in one launch where all their workgroups run at once (5 x 4 tokens
    // behind 333 keys 20.4 -> 16.3 us).  Larger ones apart: the sequences' stream through the caches takes
    // from the prefix more than running beside it gives (64 sequences behind 32768 keys 149 -> 184 us).
    plan->together = plan->pre_parts && plan->suf_parts && plan->pre_wide && !plan->suf_wide && at_once(plan->pre_chunk, plan->suf_chunk);
    return true;
}

hipError_t launch_attend(const ls_kv_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws, hipStream_t st) {
    return c.dtype == LS_F16 ? attend_dim<_Float16>(c, a, plan, ws, st) : attend_dim<__bf16>(c, a, plan, ws, st);
}

}  // namespace ls

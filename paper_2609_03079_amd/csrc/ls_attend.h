// ls_attend.h - attention of a batch that shares a prefix, over a paged cache: the kernels, for keys and values
// of the queries' type (ls_attend.hip) and for codes of 4 or 8 bits (ls_attend_fp4.hip, ls_attend_fp8.hip).
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
#pragma once

#include <algorithm>
#include <type_traits>

#include "ls_codes.h"
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
__device__ inline f32x4 mma16(const f16x8& a, const f16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
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
    const uint8_t* k_scale;  // codes only
    const uint8_t* v_scale;
    int64_t s_page, s_head, s_token;
    bool rows16;             // rows of codes are whole chunks of 16 bytes, and aligned to them
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

// Keys and values of the queries' type.
struct Whole {
    static constexpr int kBits = 16;
};

// Codes on their way through shared memory (wide workgroups): rows of kRowBytes, in chunks of 16 bytes.
template <class C, typename T, int DP>
struct Raw {
    static constexpr int kRows = Shape<T, DP, true>::kRows;      // rows a wave copies
    static constexpr int kRowBytes = DP * C::kBits / 8, CR = kRowBytes / 16;
    static constexpr int kElems = 128 / C::kBits;                // elements of a chunk
    static constexpr int RPI = 64 / CR;                          // rows per copy instruction
    static constexpr int kInstr = kRows > RPI ? kRows / RPI : 1;
    static constexpr int kOf8 = C::kBits / 4;                    // words of eight elements
};
// Scale bytes of a tile, as they are loaded: a lane waits for them where it uses them.
template <int N>
struct Scales {
    uint8_t b[N];
    bool there[N];  // false: a masked row's, nothing
};

// The value of lane ^ 32.
__device__ inline float other_half(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// Of this lane's value and that of lane ^ D (16 or 32): the same in both.
template <int D>
__device__ inline void both_of(float v, float* a, float* b) {
    const uint32_t x = __float_as_uint(v);
    if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        *a = __uint_as_float(r[0]), *b = __uint_as_float(r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        *a = __uint_as_float(r[0]), *b = __uint_as_float(r[1]);
    }
}
template <int D>
__device__ inline float pair_max(float v) {
    float a, b;
    both_of<D>(v, &a, &b);
    return fmaxf(a, b);
}
template <int D>
__device__ inline float pair_sum(float v) {
    float a, b;
    both_of<D>(v, &a, &b);
    return a + b;
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
template <typename T, int DP, bool WIDE, bool MULTI, class C>
__device__ __forceinline__ void attend(const AttendP& p, bool prefix, int b, T* k0, T* k1, T* v0, T* v1, float (*wave_ml)[2][32],
                                       float* row_sum) {
    using Sh = Shape<T, DP, WIDE>;
    constexpr bool PIPE = WIDE && !MULTI;  // scores one tile ahead (MULTI's rare path leaves no registers)
    constexpr int NW = Sh::NW, KT = Sh::KT, CPR = Sh::CPR, NF = DP / 16, ND = DP / 32, SUB = KT / 32;
    constexpr bool CODES = C::kBits < 16;
    static_assert(WIDE || !CODES, "few rows of codes are thin");
    using R = Raw<C, T, DP>;
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

    using Elem = std::conditional_t<CODES, uint8_t, T>;
    const Elem* kbase = static_cast<const Elem*>(p.k) + it.kv * p.head_stride;
    const Elem* vbase = static_cast<const Elem*>(p.v) + it.kv * p.head_stride;
    const T* zero = reinterpret_cast<const T*>(g_zero_row);
    const int page_mask = (1 << p.page_shift) - 1;

    // A key's place in the cache, in elements, -1 where it is masked.
    auto place = [&](int key0, int id) {
        const int key = key0 + (lane & (KT - 1));
        const int64_t at = (int64_t)id * p.page_stride + (int64_t)(key & page_mask) * p.token_stride;
        return (unsigned)id < (unsigned)p.n_pages && key < it.end ? at : (int64_t)-1;
    };
    // The place of its scales, where it is not masked.
    auto scale_place = [&](int key0, int id) {
        return CODES ? (int64_t)id * p.s_page + (int64_t)((key0 + (lane & (KT - 1))) & page_mask) * p.s_token + it.kv * p.s_head : 0;
    };
    // Copies the codes of this wave's rows of a tile to shared memory, RPI rows an instruction (or, where rows are no
    // multiple of 16 bytes, a word a lane): lane -> row lane / CR, chunk lane % CR.  What is
    // masked or past a row's end comes from the row of zeros.
    // The value at lane r of a 64-bit number.
    auto of_lane = [&](int64_t x, int r) {
        return (int64_t)(((uint64_t)__shfl((uint32_t)(x >> 32), r, 64) << 32) | __shfl((uint32_t)x, r, 64));
    };
    auto copy_codes = [&](const Elem* base, int64_t at, uint8_t* to) {
        const uint8_t* codes = reinterpret_cast<const uint8_t*>(base);
        const uint8_t* none = reinterpret_cast<const uint8_t*>(g_zero_row);
        const int first = wave * R::kRows;
        if (p.rows16) {
#pragma unroll
            for (int i = 0; i < R::kInstr; ++i) {
                const int r = i * R::RPI + lane / R::CR, chunk = lane % R::CR;
                const int64_t row = of_lane(at, (first + r) & (KT - 1));
                const bool there = row >= 0 && chunk * R::kElems < p.D;
                if (R::kRows >= R::RPI || r < R::kRows)
                    __builtin_amdgcn_global_load_lds((gptr)(there ? codes + row + chunk * 16 : none), (lptr)(to + i * 1024), 16, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < R::kRows * R::CR / 16; ++i) {
                const int g = i * 64 + lane, r = g / (R::CR * 4);
                const int word = g % (R::CR * 4);
                const int64_t row = of_lane(at, first + r);
                const bool there = row >= 0 && word * (32 / C::kBits) < p.D;
                __builtin_amdgcn_global_load_lds((gptr)(there ? codes + row + word * 4 : none), (lptr)(to + i * 256), 4, 0, 0);
            }
        }
    };
    // Eight elements of a lane's codes.
    auto widen = [&](const uint32_t* w, uint8_t scale, bool there) {
        vec8<T> v;
        widen8<C, T>(w, scale_of(there ? scale : 0), &v);
        return v;
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
    auto copy = [&](const Elem* base_, int64_t at, T* buf) {
        const T* base = reinterpret_cast<const T*>(base_);
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
    // The scales of what this lane copied; the codes in the last part of the wave's rows of a tile, all of them read, then
    // widened into these rows.
    using Copied = Scales<R::kInstr>;
    auto copied_scales = [&](const uint8_t* scales, int64_t at, int64_t s_at, Copied& x) {
#pragma unroll
        for (int i = 0; i < R::kInstr; ++i) {
            const int r = (wave * R::kRows + i * R::RPI + lane / R::CR) & (KT - 1), e = lane % R::CR * R::kElems;
            const int64_t row = of_lane(at, r), s = of_lane(s_at, r);
            x.b[i] = scales[(row >= 0 ? s : 0) + (e < p.D ? e / kGroup : 0)];
            x.there[i] = row >= 0;
        }
    };
    constexpr int kRawAt = R::kRows * DP * (int)sizeof(T) - R::kRows * R::kRowBytes;  // bytes into the wave's rows
    auto raw_of = [&](T* buf) { return reinterpret_cast<uint8_t*>(buf + wave * R::kRows * DP) + kRawAt; };
    auto spread = [&](T* buf, const Copied& x) {
        if (R::kRows < R::RPI && lane / R::CR >= R::kRows) return;
        u32x4 c[R::kInstr];
#pragma unroll
        for (int i = 0; i < R::kInstr; ++i) c[i] = *reinterpret_cast<const u32x4*>(raw_of(buf) + i * 1024 + lane * 16);
        __builtin_amdgcn_s_waitcnt(0xc07f);  // read by every lane before one of them writes there (vmcnt and expcnt untouched)
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
#pragma unroll
        for (int i = 0; i < R::kInstr; ++i) {
            const int r = wave * R::kRows + i * R::RPI + lane / R::CR;
            const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
            for (int j = 0; j < R::kElems / 8; ++j) {
                const int chunk = lane % R::CR * (R::kElems / 8) + j;
                *reinterpret_cast<vec8<T>*>(buf + r * DP + (chunk ^ swz<CPR>(r)) * 8) = widen(w + j * R::kOf8, x.b[i], x.there[i]);
            }
        }
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

    if constexpr (CODES) {
        // As below; the codes are copied to the end of the rows that they become while a tile is used, and spread after it.
        if (key < it.end) {
            int64_t at0 = place(key, first0), at1 = place(key + kStep, first1), s_at1 = scale_place(key + kStep, first1);
            Copied kx, vx;
            Scores s;
            auto ask = [&](const Elem* base, const uint8_t* scales, int64_t at, int64_t s_at, T* buf, Copied& x) {
                copied_scales(scales, at, s_at, x);
                copy_codes(base, at, raw_of(buf));
            };
            auto arrived = [&] {
                __builtin_amdgcn_s_waitcnt(0x0f70);
                __atomic_signal_fence(__ATOMIC_SEQ_CST);
            };
            ask(kbase, p.k_scale, at0, scale_place(key, first0), k0, kx);
            ask(vbase, p.v_scale, at0, scale_place(key, first0), v0, vx);
            arrived();
            spread(k0, kx);
            spread(v0, vx);
            if (PIPE) {
                ask(kbase, p.k_scale, at1, s_at1, k1, kx);
                arrived();
                spread(k1, kx);
                landed();
                s = scores(k0);
                largest(s);
            }
            auto tile = [&](T* ka, T* kb, T* va, T* vb) {  // as below
                const int64_t at2 = place(key + 2 * kStep, id2), s_at2 = scale_place(key + 2 * kStep, id2);
                landed();
                id2 = page_id(key + 3 * kStep);
                const bool more = PIPE || key + kStep < it.end;
                if (more) {
                    ask(kbase, p.k_scale, PIPE ? at2 : at1, PIPE ? s_at2 : s_at1, PIPE ? ka : kb, kx);
                    ask(vbase, p.v_scale, at1, s_at1, vb, vx);
                }
                if (!idle_wave) use(s, key, at0, va, PIPE ? kb : ka);
                if (more) {
                    arrived();
                    spread(PIPE ? ka : kb, kx);
                    spread(vb, vx);
                }
                key += kStep;
                at0 = at1, at1 = at2, s_at1 = s_at2;
            };
            for (;;) {
                tile(k0, k1, v0, v1);
                if (key >= it.end) break;
                tile(k1, k0, v1, v0);
                if (key >= it.end) break;
            }
            landed();
        }
    } else if (key < it.end) {
        // While tile j is used, V of j + 1 and K of j + 1 (PIPE: j + 2) arrive.  Past the end PIPE
        // copies and multiplies tiles of zeros; nothing uses their scores.
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

typedef const __attribute__((address_space(1))) uint8_t* gbyte;
typedef const __attribute__((address_space(1))) uint32_t* gword;
typedef const __attribute__((address_space(1))) u32x2a* gwords2;
typedef const __attribute__((address_space(1))) u32x4a* gwords4;

// An address that is the same in every lane, in scalar registers.
__device__ inline const uint8_t* wave_address(const uint8_t* p) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uint64_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)p >> 32));
    return reinterpret_cast<const uint8_t*>(((uint64_t)hi << 32) | lo);
}

constexpr int kThinPad = 8;  // elements

// Up to 16 rows over codes.  The products run on the 16 x 16 x 32 instructions: half the scores, sums and
// query operands a lane of the narrow shape, which leaves registers for three waves a SIMD (and the codes need no shared memory on
// their way).  A lane takes a quarter of a key's row, straight from the cache: key n of the first 16 of a tile and of the
// second, elements g DP / 4 and on; its scores are those of keys 16 t + 4 g + i and query row n.
template <typename T, int DP, bool MULTI, class C>
__device__ __forceinline__ void attend_thin(const AttendP& p, bool prefix, int b, T* v0, float (*wave_ml)[2][32]) {
    using Sh = Shape<T, DP, false>;
    constexpr int NW = Sh::NW, KT = 32, kStep = NW * KT, NF = DP / 32, ND = DP / 16;
    constexpr int kOwn = DP / 4, kWords = kOwn * C::kBits / 32, kOf8 = C::kBits / 4, kScales = kOwn > kGroup ? kOwn / kGroup : 1;
    Item it;
    if (!item_of<16>(p, prefix, b, &it)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;

    int key = it.begin + wave * KT;
    auto page_id = [&](int key0, int t) {
        const int at = key0 + t * 16 + n;
        return at < it.end ? it.table[at >> p.page_shift] : -1;
    };
    int ids0[2] = {page_id(key, 0), page_id(key, 1)}, ids1[2] = {page_id(key + kStep, 0), page_id(key + kStep, 1)};
    it.len = it.seq < 0 ? p.prefix_len : min(p.lens[it.seq], p.max_len);
    it.end = min(it.end, it.len);
    if (it.begin >= it.end && !p.direct) return;

    const int row = it.row0 + n;
    const bool row_ok = row < it.rows;
    const int rr = row_ok ? row : it.rows - 1;
    const int tk = p.by_G.of(rr), head = it.kv * p.G + rr - tk * p.G;
    const int64_t token = it.seq < 0 ? tk : (int64_t)it.seq * p.n_q + tk;
    const int limit = it.seq < 0 ? it.end : min(it.end, it.len - p.n_q + 1 + tk);
    const int full_len = it.seq < 0 ? it.end : it.len - p.n_q + 1, full = min(it.end, full_len);

    vec8<T> q[NF];
    {
        const T* src = static_cast<const T*>(p.q) + token * p.q_token + head * p.q_head;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int d = g * kOwn + f * 8;
            q[f] = row_ok && d < p.D ? *reinterpret_cast<const vec8<T>*>(src + d) : vec8<T>{};
        }
    }
    f32x4 o[ND];
#pragma unroll
    for (auto& x : o) x = f32x4{};
    float m = -INFINITY, l = 0.f;

    const uint8_t* kbase = static_cast<const uint8_t*>(p.k) + it.kv * p.head_stride;
    const uint8_t* vbase = static_cast<const uint8_t*>(p.v) + it.kv * p.head_stride;
    const uint8_t* ksbase = p.k_scale + it.kv * p.s_head;
    const uint8_t* vsbase = p.v_scale + it.kv * p.s_head;
    const int page_mask = (1 << p.page_shift) - 1;
    struct Codes {
        uint32_t k[2][kWords], v[2][kWords];
        uint8_t ks[2][kScales], vs[2][kScales];  // bytes as they are loaded: a lane waits for them where it uses them
        uint32_t valid;                          // bit j: key j of the tile is not masked
    };
    // A lane's codes and scales of a tile.  A masked key's are those of the cache's first rows (`use` makes zeros of them), so that
    // there is nothing but loads here: a choice between these and zeros becomes branches that wait for what they have loaded.
    // What is past a row's end is its start once more: it meets zeros of the query, or becomes columns that are not written.
    // GRAIN: elements that are there or past a row's end together, the lane's whole share or 16 or 8.  PAGED: the 16 keys of a half lie in one page, at an address that the wave
    // shares and places that the lanes keep; otherwise each lane works out its own.
    const int e = g * kOwn;
    int s_of[kScales], w_of[kWords];
#pragma unroll
    for (int i = 0; i < kScales; ++i) s_of[i] = e + i * kGroup < p.D ? (e + i * kGroup) / kGroup : 0;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        const int w = e + j * (32 / C::kBits);
        w_of[j] = w < p.D ? w * C::kBits / 8 : 0;
    }
    auto load = [&](auto GRAIN, auto PAGED, const uint8_t* codes, const uint8_t* scales, int64_t c_at, int64_t s_at, uint32_t (&w)[kWords],
                    uint8_t (&s)[kScales]) {
        constexpr int kTake = decltype(GRAIN)::value * C::kBits / 32;  // words together
        const int c_n = decltype(PAGED)::value ? n * (int)p.token_stride : 0, s_n = decltype(PAGED)::value ? n * (int)p.s_token : 0;
        const uint8_t* from = decltype(PAGED)::value ? wave_address(codes + c_at) : codes + c_at;
        const uint8_t* s_from = decltype(PAGED)::value ? wave_address(scales + s_at) : scales + s_at;
#pragma unroll
        for (int i = 0; i < kScales; ++i) s[i] = *(gbyte)(s_from + (uint32_t)(s_n + s_of[i]));
#pragma unroll
        for (int i = 0; i < kWords; i += kTake) {
            const uint8_t* at = from + (uint32_t)(c_n + w_of[i]);
            if constexpr (kTake == 1) {
                w[i] = *(gword)at;
            } else if constexpr (kTake == 2) {
                const u32x2a v = *(gwords2)at;
                w[i] = v[0], w[i + 1] = v[1];
            } else {
#pragma unroll
                for (int k = 0; k < kTake; k += 4) {
                    const u32x4a v = *(gwords4)(at + k * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[i + k + j] = v[j];
                }
            }
        }
    };
    auto fetch = [&](auto GRAIN, auto PAGED, int key0, const int (&ids)[2], Codes& x) {
        x.valid = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int at = key0 + t * 16 + (decltype(PAGED)::value ? 0 : n);
            int id = decltype(PAGED)::value ? __builtin_amdgcn_readfirstlane(ids[t]) : ids[t];
            const bool there = (unsigned)id < (unsigned)p.n_pages && at < it.end;
            if (decltype(PAGED)::value)
                x.valid |= there ? (it.end - at >= 16 ? 0xffffu : (1u << (it.end - at)) - 1) << (16 * t) : 0u;
            else
                x.valid |= ((uint32_t)__ballot(there) & 0xffff) << (16 * t);
            id = there ? id : 0;
            const int64_t place = at & page_mask;
            const int64_t c_at = id * p.page_stride + place * p.token_stride, s_at = id * p.s_page + place * p.s_token;
            load(GRAIN, PAGED, kbase, ksbase, c_at, s_at, x.k[t], x.ks[t]);
            load(GRAIN, PAGED, vbase, vsbase, c_at, s_at, x.v[t], x.vs[t]);
        }
    };
    auto widen = [&](const uint32_t* w, uint8_t scale) {
        vec8<T> v;
        widen8<C, T>(w, scale_of(scale), &v);
        return v;
    };
    // The wave's values: rows 16 bytes longer than they are, so that neither eight rows at one place (written) nor 16 rows at 32
    // bytes (read) meet in a bank more often than their number asks, and one address serves with fixed offsets.
    constexpr int kPitch = DP + kThinPad;
    T* vt = v0 + wave * KT * kPitch;
    T* v_put = vt + n * kPitch + g * kOwn;
    const T* v_get = vt + (4 * g + ((lane & 15) >> 2)) * kPitch + (lane & 3) * 4;

    auto use = [&](Codes& x, int key0) {
        const uint32_t valid = x.valid;
        const bool some = key0 + KT > full || ~valid != 0;  // keys that not every row sees
        if (~valid != 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bool there = (valid >> (16 * t + n)) & 1;
#pragma unroll
                for (int j = 0; j < kWords; ++j) x.k[t][j] = there ? x.k[t][j] : 0, x.v[t][j] = there ? x.v[t][j] : 0;
#pragma unroll
                for (int i = 0; i < kScales; ++i) x.ks[t][i] = there ? x.ks[t][i] : 0, x.vs[t][i] = there ? x.vs[t][i] : 0;
            }
        }
        f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mma16(widen(&x.k[t][f * kOf8], x.ks[t][f * 8 / kGroup]), q[f], s[t]);
        if (some) {
            const int left = limit - key0;
            const uint32_t below = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1, seen = (below & valid) >> (4 * g);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][i] = (seen >> (16 * t + i)) & 1 ? s[t][i] : -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int f = 0; f < NF; ++f)
                *reinterpret_cast<vec8<T>*>(v_put + t * 16 * kPitch + f * 8) = widen(&x.v[t][f * kOf8], x.vs[t][f * 8 / kGroup]);
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        top = pair_max<16>(top);
        top = pair_max<32>(top);
        const float next = fmaxf(m, top * p.c - Sh::kLift), base = next == -INFINITY ? 0.f : next;
        if (__any(next > m)) {
            const float scale = __builtin_amdgcn_exp2f(m - base);  // m = -inf: 0
            l *= scale;
#pragma unroll
            for (auto& y : o) y *= scale;
            m = next;
        }
        vec8<T> pr;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(s[t][i], p.c, -base));
                l += e;
                pr[4 * t + i] = (T)e;
            }
        auto value = [&](int d) {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(v_get + d * 16));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(v_get + 16 * kPitch + d * 16));
            struct { s16x4 a, b; } both{a, b};
            return __builtin_bit_cast(vec8<T>, both);
        };
        bool odd = false;
        if (MULTI && it.seq >= 0 && key0 + KT > full) {  // as above: a weight of zero must keep out a value that is no number
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const auto v = value(d);
#pragma unroll
                for (int j = 0; j < 8; ++j) odd |= key0 + 16 * (j / 4) + 4 * g + j % 4 >= full && !(fabsf((float)v[j]) < INFINITY);
            }
        }
        if (MULTI && __any(odd)) {
#pragma unroll 1
            for (int i = 0; i < p.n_q; ++i) {
                const int seen = full_len + i;
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    auto v = value(d);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (key0 + 16 * (j / 4) + 4 * g + j % 4 >= seen) v[j] = (T)0.f;
                    const f32x4 y = mma16(v, pr, o[d]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[d][e] = tk == i ? y[e] : o[d][e];
                }
            }
        } else {
#pragma unroll
            for (int d = 0; d < ND; ++d) o[d] = mma16(value(d), pr, o[d]);
        }
    };
    // While a tile is used, the codes of the next are on their way, and the page ids of the one behind it.
    // (A loop for each way to load: a branch inside would wait for the loads that each side has under way.)
    auto run = [&](auto GRAIN, auto PAGED) {
        Codes a, b;
        fetch(GRAIN, PAGED, key, ids0, a);
        auto tile = [&](Codes& now, Codes& next) {
            const int ids2[2] = {page_id(key + 2 * kStep, 0), page_id(key + 2 * kStep, 1)};
            fetch(GRAIN, PAGED, key + kStep, ids1, next);  // (past the end: the cache's first rows)
            use(now, key);
            key += kStep;
            ids1[0] = ids2[0], ids1[1] = ids2[1];
        };
        for (;;) {
            tile(a, b);
            if (key >= it.end) break;
            tile(b, a);
            if (key >= it.end) break;
        }
    };
    if (key < it.end) {
        const bool paged = page_mask >= 15 && p.token_stride < 1 << 26 && p.s_token < 1 << 26;
        auto by_page = [&](auto GRAIN) {
            if (paged)
                run(GRAIN, std::true_type{});
            else
                run(GRAIN, std::false_type{});
        };
        if (p.D % kOwn == 0)
            by_page(std::integral_constant<int, kOwn>{});
        else if (kOwn > 16 && p.D % 16 == 0)
            by_page(std::integral_constant<int, 16>{});
        else
            by_page(std::integral_constant<int, 8>{});
    }
    l = pair_sum<32>(pair_sum<16>(l));

    // the waves' results joined: the second's sums through the values' array, to be added by the first, lane by lane
    if (g == 0) {
        wave_ml[wave][0][n] = m;
        wave_ml[wave][1][n] = l;
    }
    __syncthreads();
    const float top = fmaxf(wave_ml[0][0][n], wave_ml[1][0][n]), base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float wl = wave_ml[w][1][n];
        if (wl != 0.f) sum += wl * __builtin_amdgcn_exp2f(wave_ml[w][0][n] - base);
    }
    static_assert(NW == 2 && NW * KT * kPitch * sizeof(T) >= ND * 64 * 16, "room for a wave's sums");
    const float scale = __builtin_amdgcn_exp2f(m - base);
    f32x4* sums = reinterpret_cast<f32x4*>(v0) + lane;
    if (wave == 1) {
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : o[d][e] * scale;
            sums[d * 64] = v;
        }
    }
    __syncthreads();
    if (wave == 1 || !row_ok) return;
    const int64_t out_row = token * p.H + head;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
        const int e0 = d * 16 + 4 * g;
        f32x4 v = sums[d * 64];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += l == 0.f ? 0.f : o[d][e] * scale;
        if (e0 >= p.D) continue;
        if (p.direct) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            Pack<T, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y.e[e] = (T)(v[e] * inv);
            store_pack<T, 4>(p.out, token * p.o_token + head * p.o_head + e0, y);
        } else {
            *reinterpret_cast<f32x4*>(p.part + (out_row * p.parts + it.part) * p.D + e0) = v;
        }
    }
    if (g == 0 && !p.direct) {
        float* at = p.ml + (out_row * p.parts + it.part) * 2;
        at[0] = top;
        at[1] = sum;
    }
}

// Which shapes a launch holds.  BOTH: a wide prefix beside narrow (of codes: thin) sequences, eight workgroups of one after
// eight of the other (one for each XCD).  NARROW: elements of 16 bits only, THIN: codes only.
enum Roles { NARROW, WIDE_ROWS, BOTH, THIN };

// Waves a SIMD that the registers are shared out for.
template <int DP, Roles ROLES, bool MULTI, class C>
constexpr int waves_of() {
    if (ROLES == THIN) return DP <= 64 ? (C::kBits == 4 && !MULTI ? 4 : 3) : DP <= 128 ? (C::kBits == 4 && !MULTI ? 3 : 2) : 1;
    if (ROLES == NARROW) return 1;
    return DP <= 128 && (ROLES == BOTH || !MULTI) ? 2 : 1;
}
template <typename T, int DP, Roles ROLES>
constexpr int threads_of = Shape<T, DP, ROLES == WIDE_ROWS || ROLES == BOTH>::NW * 64;

template <typename T, int DP, Roles ROLES, bool MULTI, class C>
__global__ __launch_bounds__((threads_of<T, DP, ROLES>), (waves_of<DP, ROLES, MULTI, C>())) void attend_kernel(const AttendP p) {
    constexpr bool kCodes = C::kBits < 16;
    constexpr int kBuf = ROLES == WIDE_ROWS ? Shape<T, DP, true>::kBuf : Shape<T, DP, false>::kBuf;
    static_assert(Shape<T, DP, false>::kBuf >= Shape<T, DP, true>::kBuf, "room for either shape");
    // thin workgroups: a tile of values for each wave
    constexpr int kKeys = ROLES == THIN ? 1 : kBuf;
    constexpr int kValues = kCodes && (ROLES == THIN || ROLES == BOTH) ? Shape<T, DP, false>::NW * 32 * (DP + kThinPad) : kBuf;
    static_assert(kValues >= kBuf || ROLES == THIN, "room for a wide tile");
    __shared__ __attribute__((aligned(16))) T k0[kKeys], k1[kKeys], v0[kValues], v1[kKeys];
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
            attend<T, DP, true, false, C>(p, true, b, k0, k1, v0, v1, wave_ml, row_sum);
        } else if (threadIdx.x < Shape<T, DP, false>::NW * 64) {
            if constexpr (kCodes)
                attend_thin<T, DP, MULTI, C>(p, false, b, v0, wave_ml);
            else
                attend<T, DP, false, MULTI, C>(p, false, b, k0, k1, v0, v1, wave_ml, row_sum);
        }
    } else {
        const bool prefix = b < p.pre_items;
        if constexpr (ROLES == THIN)
            attend_thin<T, DP, MULTI, C>(p, prefix, prefix ? b : b - p.pre_items, v0, wave_ml);
        else
            attend<T, DP, ROLES == WIDE_ROWS, MULTI, C>(p, prefix, prefix ? b : b - p.pre_items, k0, k1, v0, v1, wave_ml, row_sum);
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

// c: the cache's shape, and what Whole keys and values are read from; `codes`: what is read otherwise.
template <typename T, int DP, class C>
hipError_t attend_type(const ls_kv_cache& c, const ls_kvq_cache* codes, const ls_attend_args& a, const AttendPlan& plan, void* ws,
                       hipStream_t st) {
    AttendP p{};
    p.q = a.q, p.q_token = a.q_token_stride, p.q_head = a.q_head_stride;
    p.out = a.out, p.o_token = a.out_token_stride, p.o_head = a.out_head_stride;
    p.k = c.k, p.v = c.v;
    p.page_stride = c.page_stride, p.head_stride = c.head_stride, p.token_stride = c.token_stride;
    if (codes) {
        p.k_scale = codes->k_scale, p.v_scale = codes->v_scale;
        const int64_t row = (int64_t)c.head_dim * C::kBits / 8;
        p.rows16 = row % 16 == 0 && aligned(c.k, 16) && aligned(c.v, 16) && c.page_stride % 16 == 0 && c.head_stride % 16 == 0 &&
                   c.token_stride % 16 == 0;
        p.s_page = codes->scale_page_stride, p.s_head = codes->scale_head_stride, p.s_token = codes->scale_token_stride;
    }
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
            if constexpr (C::kBits < 16)
                return hipErrorInvalidValue;  // (never: codes are thin)
            else if (multi)
                hipLaunchKernelGGL((attend_kernel<T, DP, NARROW, true, C>), grid, narrow_wg, 0, st, p);
            else
                hipLaunchKernelGGL((attend_kernel<T, DP, NARROW, false, C>), grid, narrow_wg, 0, st, p);
        } else if (roles == WIDE_ROWS) {
            if (multi)
                hipLaunchKernelGGL((attend_kernel<T, DP, WIDE_ROWS, true, C>), grid, wide_wg, 0, st, p);
            else
                hipLaunchKernelGGL((attend_kernel<T, DP, WIDE_ROWS, false, C>), grid, wide_wg, 0, st, p);
        } else if (roles == THIN) {
            if constexpr (C::kBits < 16) {
                if (multi)
                    hipLaunchKernelGGL((attend_kernel<T, DP, THIN, true, C>), grid, narrow_wg, 0, st, p);
                else
                    hipLaunchKernelGGL((attend_kernel<T, DP, THIN, false, C>), grid, narrow_wg, 0, st, p);
            }
        } else {
            if (multi)
                hipLaunchKernelGGL((attend_kernel<T, DP, BOTH, true, C>), grid, wide_wg, 0, st, p);
            else
                hipLaunchKernelGGL((attend_kernel<T, DP, BOTH, false, C>), grid, wide_wg, 0, st, p);
        }
        return hipGetLastError();
    };
    const Roles pre_role = plan.pre_thin ? THIN : plan.pre_wide ? WIDE_ROWS : NARROW;
    const Roles suf_role = plan.suf_thin ? THIN : plan.suf_wide ? WIDE_ROWS : NARROW;
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

template <typename T, class C>
hipError_t attend_dim(const ls_kv_cache& c, const ls_kvq_cache* codes, const ls_attend_args& a, const AttendPlan& plan, void* ws,
                      hipStream_t st) {
    if (c.head_dim <= 64) return attend_type<T, 64, C>(c, codes, a, plan, ws, st);
    if (c.head_dim <= 128) return attend_type<T, 128, C>(c, codes, a, plan, ws, st);
    return attend_type<T, 256, C>(c, codes, a, plan, ws, st);
}

}  // namespace
}  // namespace ls

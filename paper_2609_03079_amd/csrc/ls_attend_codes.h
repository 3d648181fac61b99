// ls_attend_codes.h - attention over keys and values held in 4 or 8 bits (ls_attend_fp4_f16.hip and so on,
// a file for each code and type: they take minutes to compile).
//
// The mathematics and the parts are those of ls_attend.hip; the products run transposed on 16-bit operands, into which the codes are widened
// (two by one instruction, exactly, their group's power of two among its operands).  What differs is where that happens.  A key's
// codes go from the cache to the registers of the lanes that multiply them, as both products may take a head's elements
// in any order: a lane takes a part of the row that follows itself in memory.  A value's elements are needed key
// by key, so they are widened into shared memory and read from there transposed.
//
// Two shapes of workgroup: thin, tiles of 16 query rows (up to 32 rows), and broad, tiles of 128.
#pragma once

#include <type_traits>

#include "ls_attend.h"
#include "ls_codes.h"

namespace ls {
namespace {

typedef const __attribute__((address_space(1))) uint8_t* gbyte;
typedef const __attribute__((address_space(1))) uint32_t* gword;
typedef const __attribute__((address_space(1))) u32x2a* gwords2;
typedef const __attribute__((address_space(1))) u32x4a* gwords4;

__device__ inline f32x4 mma16(const f16x8& a, const f16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
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

// An address that is the same in every lane, in scalar registers.
__device__ inline const uint8_t* wave_address(const uint8_t* p) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uint64_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)p >> 32));
    return reinterpret_cast<const uint8_t*>(((uint64_t)hi << 32) | lo);
}

// The place of a page's token where 32 bits hold both strides, in two scalar products.
__device__ inline int64_t place_of(int id, int64_t page_stride, int place, int64_t token_stride) {
    return (int64_t)((uint64_t)(uint32_t)id * (uint32_t)page_stride + (uint32_t)place * (uint32_t)token_stride);
}

// A row's sums are rescaled where its maximum has grown by more than this since they last were (in powers of two): while it creeps up, by
// a little in most steps, its largest weight is above 2^kLift instead.  float16 has room for one more power (ls_attend.h).
template <typename T>
constexpr float kSlack = std::is_same_v<T, _Float16> ? 1.f : 8.f;

// The sums of weighted values are divided by the weights' sum when all keys have been seen.  bfloat16 has values of up to 2^127.8: weights
// of up to 2^8 (kSlack) of some of them, or those of many keys, are beyond fp32 though the row is not.  A wave (thin) or workgroup (broad) one of
// whose sums came near that (kFar: 128 parts of less can be joined) goes over its keys a second time, those rows' weights smaller by
// 2^32: 2^22 keys of weights of 2^-24 stay below the largest value.  (Smaller from the start, the products with small values would be
// lost: fp32 ends at 2^-126.)  Rows are told apart, so that a row's bits do not depend on those beside it.  Others pay for looking at
// the sums, one instruction for two: 8 sequences behind 7901 keys 16.4 -> 16.6 us, 64 behind 32768 116.5 -> 116.8.
template <typename T>
constexpr bool kTwice = !std::is_same_v<T, _Float16>;
constexpr float kFar = 0x1p118f, kLower = 32.f;

// The lanes among whose sums one is far, or no number.
template <typename V, int N>
__device__ __forceinline__ uint64_t far_rows(const V (&o)[N]) {
    float most = 0.f;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int e = 0; e < (int)(sizeof(V) / 4); ++e) most = __builtin_elementwise_maximum(most, fabsf(o[d][e]));  // NaN, if one is
    return __ballot(!(most < kFar));
}

// A pass of a workgroup over its keys: the first, or the SECOND, which is seldom asked for and looks every key's place up by itself.
// What follows from the call, the thread and the workgroup is worked out anew in it: kept, it would take registers that the first
// one needs (as one loop over both, calls of a few keys took 7 to 10 in a hundred more).
template <bool SECOND>
struct Pass {
    const AttendP& p;
    int thread, b;
};
__device__ __forceinline__ Pass<false> first_pass(const AttendP& p, int b) { return {p, (int)threadIdx.x, b}; }
__device__ __forceinline__ Pass<true> second_pass(int b) {
    typedef const __attribute__((address_space(4))) AttendP* Argument;
    Argument p = (Argument)__builtin_amdgcn_kernarg_segment_ptr();  // the kernel's only one
    int thread = threadIdx.x;
    asm volatile("" : "+s"(p), "+v"(thread), "+s"(b));
    return {*(const AttendP*)p, thread, b};
}

// Eight elements of a lane's codes.
template <class C, typename T>
__device__ inline vec8<T> widened(const uint32_t* w, uint8_t scale) {
    vec8<T> v;
    widen8<C, T>(w, scale_of(scale), &v);
    return v;
}

// A lane's share of a row: OWN elements from e on.  What is past a row's end (PAD: heads of fewer elements than the lanes have shares
// of) is loaded from its start once more.  Of a value it becomes columns that are not written.  Of a key it meets zeros of the query, which
// cancel no infinity (the start's own, or of its codes under another group's scale), so `clear` makes its codes zeros.  Its scale is
// that of a group of the row, no number only where an element of the row is none.
template <class C, int OWN>
struct Share {
    static constexpr int kWords = OWN * C::kBits / 32, kScales = OWN > kGroup ? OWN / kGroup : 1;
    int s_of[kScales], w_of[kWords];
    uint32_t in = 0;  // bit j: word j is of the row
    __device__ inline Share(int e, int D) {
#pragma unroll
        for (int i = 0; i < kScales; ++i) s_of[i] = e + i * kGroup < D ? (e + i * kGroup) / kGroup : 0;
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            const int w = e + j * (32 / C::kBits);
            in |= (uint32_t)(w < D) << j;
            w_of[j] = w < D ? w * C::kBits / 8 : 0;
        }
    }
    // Of N keys, and only where one has a scale under which a code may be infinite: asking is three instructions of the hundreds that
    // a tile takes, the zeros 16 to 48 (52 x 5 tokens in heads of 96, FP8: 28.4 us without either, 28.6 asked, 29.3 always cleared).
    template <typename T, int N>
    __device__ __forceinline__ void clear(uint32_t (&w)[N][kWords], const uint8_t (&s)[N][kScales]) const {
        uint32_t top = 0;
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int i = 0; i < kScales; ++i) top = max(top, (uint32_t)s[t][i]);
        if (!__any(top > 127 + (std::is_same_v<T, _Float16> ? C::kMostExp16 : C::kMostExp))) return;
        uint32_t bits = in;
        asm volatile("" : "+v"(bits));  // the masks are worked out here, not kept in registers over the loop
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int j = 0; j < kWords; ++j) w[t][j] &= (uint32_t)__builtin_amdgcn_sbfe((int)bits, j, 1);
    }
    // GRAIN: elements that are there or past the row's end together, the whole share or 16 or 8 (and loaded together).
    // SHARED: the addresses are the wave's, the offsets its lanes'.
    // ONCE: codes that the caches need not keep.
    template <typename G, typename S, typename O>
    __device__ __forceinline__ void load(G, S, O, const uint8_t* codes, const uint8_t* scales, uint32_t c_n, uint32_t s_n, uint32_t (&w)[kWords],
                                uint8_t (&s)[kScales]) const {
        constexpr int kTake = G::value * C::kBits / 32;  // words together
        const uint8_t* from = S::value ? wave_address(codes) : codes;
        const uint8_t* s_from = S::value ? wave_address(scales) : scales;
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
                    const u32x4a v = O::value ? __builtin_nontemporal_load((gwords4)(at + k * 4)) : *(gwords4)(at + k * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[i + k + j] = v[j];
                }
            }
        }
    }
};

// Pages of 16 tokens or more whose offsets 32 bits hold, and a page's.
__device__ inline bool whole_pages(const AttendP& p, bool paged) {
    return paged && (p.token_stride << p.page_shift) < (int64_t)1 << 31 && (p.s_token << p.page_shift) < (int64_t)1 << 31 &&
           p.page_stride < (int64_t)1 << 32 && p.s_page < (int64_t)1 << 32;
}

// Calls run(GRAIN, PAGED) with the grain of shares of OWN elements.  (A loop for each: a branch inside a loop would wait for the
// loads that either side has under way.)
template <int OWN, bool PAD, bool SECOND, typename Run>
__device__ __forceinline__ void by_grain(const AttendP& p, bool paged, Run run) {
    if constexpr (SECOND) {
        run(std::integral_constant<int, 8>{}, std::false_type{});
    } else {
        paged = whole_pages(p, paged);
        auto by_page = [&](auto GRAIN) __attribute__((always_inline)) {
            if (paged)
                run(GRAIN, std::true_type{});
            else
                run(GRAIN, std::false_type{});
        };
        if constexpr (!PAD) {
            by_page(std::integral_constant<int, OWN>{});
        } else {
            if (p.D % OWN == 0)
                by_page(std::integral_constant<int, OWN>{});
            else if (OWN > 16 && p.D % 16 == 0)
                by_page(std::integral_constant<int, 16>{});
            else
                by_page(std::integral_constant<int, 8>{});
        }
    }
}

// Where a token's heads follow each other in a page, rows of codes and scales are smaller than the cache lines that they share: the
// heads of a part then run on one die (workgroups take the eight in turn) and read the lines once.  Of the prefix a die has
// an eighth of the parts and heads; of the sequences every eighth part of each, another one of the next.
__device__ inline int near(const AttendP& p, bool prefix, int b) {
    if (!p.near_units) return b;
    const int eighth = b >> 3, die = b & 7;
    if (prefix) {
        const int tiles = p.plan.pre_tiles, turn = p.by_pre_tiles.of(eighth), group = die * p.by_pre_tiles.of(p.pre_items >> 3) + turn;
        return ((group >> 3) * tiles + eighth - turn * tiles) * 8 + (group & 7);
    }
    const int round = p.by_near.of(eighth);
    if (round * 8 + 8 > p.near_units) return b;
    return (round * 8 + ((die - round) & 7)) * p.by_near.d + eighth - round * p.by_near.d;
}

// Several query tokens: the last keys are not seen by all of them, and a weight of zero does not keep a value out that is no
// number.  So such values of these keys are made zeros as they are widened, in shared memory (take_odd: a lane's N elements,
// where its key is one of them; true in every lane if any lane had one), and added behind the loop, which they happen seldom to need, to the
// sums of the rows that see them (add_odd: `add(key, d0, v)` with eight elements of each key from `from` that is `mine`).
template <typename T, int N>
__device__ __forceinline__ bool take_odd(T* at, bool late) {
    // exponents of ones: infinities and NaN
    constexpr uint32_t kOnes = std::is_same_v<T, _Float16> ? 0x7c00 : 0x7f80;
    bool some = false;
#pragma unroll
    for (int j = 0; j < N; j += 8) {
        const auto v = __builtin_bit_cast(u32x4a, *reinterpret_cast<const vec8<T>*>(at + j));
#pragma unroll
        for (int i = 0; i < 4; ++i) some |= (v[i] & kOnes) == kOnes || (v[i] >> 16 & kOnes) == kOnes;
    }
    if (!__any(late && some)) return false;
#pragma unroll 1
    for (int j = 0; j < N; ++j)
        if (late && !(fabsf((float)at[j]) < INFINITY)) at[j] = (T)0.f;
    return true;
}

template <typename T, class C, typename Mine, typename Add>
__device__ __forceinline__ void add_odd(const AttendP& p, const Item& it, int from, const uint8_t* v, const uint8_t* scales, Mine mine, Add add) {
#pragma unroll 1
    for (int key = from; key < it.end; ++key) {
        const int id = it.table[key >> p.page_shift], place = key & ((1 << p.page_shift) - 1);
        if (!mine(key) || (unsigned)id >= (unsigned)p.n_pages) continue;
        const uint8_t* row = v + id * p.page_stride + place * p.token_stride;
        const uint8_t* of_row = scales + id * p.s_page + place * p.s_token;
#pragma unroll 1
        for (int d0 = 0; d0 < p.D; d0 += 8) {
            uint32_t w[C::kBits / 4];
#pragma unroll
            for (int i = 0; i < C::kBits / 4; ++i) w[i] = *reinterpret_cast<const uint32_t*>(row + d0 * C::kBits / 8 + i * 4);
            add(key, d0, widened<C, T>(w, of_row[d0 / kGroup]));
        }
    }
}

// Those of four of the elements, the first or second, that are no numbers, zeros beside them and for a row that does not see them.
template <typename T>
__device__ __forceinline__ f32x4 odd_of(const vec8<T>& v, bool second, bool seen) {
    f32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = second ? (float)v[4 + e] : (float)v[e];
        if (!seen || fabsf(x[e]) < INFINITY) x[e] = 0.f;
    }
    return x;
}

constexpr int kThinPad = 8;  // elements

// Up to 16 rows over codes.  Bound by memory where there are waves enough, by a wave's chain of loads, products and exponentials
// (12 ns a key of 128) where there are few: 4 sequences of 100001 keys (32 / 8 heads of 128, FP4) take 80 us with their join, 5.4 TB/s (alone,
// 77 in the best of 30 launches and 88 in the median), 1000 keys of 32 heads 6.1 and 6.9.  Two waves take 32 keys each in turn.  The
// products run on the 16 x 16 x 32 instructions, which need half the scores, sums and query operands a lane that tiles of 32 rows do:
// 168 registers, three waves a SIMD, and in place of those tiles 8 sequences behind 7901 keys 19.4 -> 17.0 us, 16 x 8 tokens of 2000 keys
// 35.6 -> 23.9.  A lane takes a quarter of a key's row, straight from the cache: key n of the first 16 of a tile and of the second,
// elements g DP / 4 and on; its scores are those of keys 16 t + 4 g + i and query row n.
// True: the pass has to be taken again (kTwice), lift_of_row then says with what weights this lane's row.
template <typename T, int DP, bool MULTI, class C, bool PAD, bool SECOND>
__device__ __forceinline__ bool attend_thin(const Pass<SECOND>& pass, bool prefix, float* lift_of_row, T* v0, float (*wave_ml)[2][32]) {
    constexpr int NW = 2, KT = 32, kStep = NW * KT, NF = DP / 32, ND = DP / 16;
    constexpr int kOwn = DP / 4, kWords = kOwn * C::kBits / 32, kOf8 = C::kBits / 4, kScales = kOwn > kGroup ? kOwn / kGroup : 1;
    const AttendP& p = pass.p;
    Item it;
    if (!item_of<16>(p, prefix, near(p, prefix, pass.b), &it)) return false;
    const int lane = pass.thread & 63, wave = __builtin_amdgcn_readfirstlane(pass.thread >> 6);
    const int n = lane & 15, g = lane >> 4;

    int key = it.begin + wave * KT;
    auto page_id = [&](int key0, int t) {
        const int at = key0 + t * 16 + n;
        return at < it.end ? it.table[at >> p.page_shift] : -1;
    };
    int ids0[2] = {page_id(key, 0), page_id(key, 1)}, ids1[2] = {page_id(key + kStep, 0), page_id(key + kStep, 1)};
    it.len = it.seq < 0 ? p.prefix_len : min(p.lens[it.seq], p.max_len);
    it.end = min(it.end, it.len);
    if (it.begin >= it.end && !p.direct) return false;

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
    const float lift = SECOND ? *lift_of_row : kLift<T>;

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
    // PAGED: the 16 keys of a half lie in one page, at an address that the wave shares and places that the lanes keep;
    // otherwise each lane works out its own.
    const Share<C, kOwn> share(g * kOwn, p.D);
    auto fetch = [&](auto GRAIN, auto PAGED, auto ONCE, int key0, const int (&ids)[2], Codes& x) __attribute__((always_inline)) {
        const uint32_t c_n = decltype(PAGED)::value ? n * (uint32_t)p.token_stride : 0, s_n = decltype(PAGED)::value ? n * (uint32_t)p.s_token : 0;
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
            const int place = at & page_mask;
            int64_t c_at, s_at;
            if (decltype(PAGED)::value) {
                c_at = place_of(id, p.page_stride, place, p.token_stride);
                s_at = place_of(id, p.s_page, place, p.s_token);
            } else {
                c_at = id * p.page_stride + place * p.token_stride;
                s_at = id * p.s_page + place * p.s_token;
            }
            share.load(GRAIN, PAGED, ONCE, kbase + c_at, ksbase + s_at, c_n, s_n, x.k[t], x.ks[t]);
            share.load(GRAIN, PAGED, ONCE, vbase + c_at, vsbase + s_at, c_n, s_n, x.v[t], x.vs[t]);
        }
    };
    // The wave's values: rows 16 bytes longer than they are, so that neither eight rows at one place (written) nor 16 rows at 32
    // bytes (read) meet in a bank more often than their number asks, and one address serves with fixed offsets.
    constexpr int kPitch = DP + kThinPad;
    T* vt = v0 + wave * KT * kPitch;
    T* v_put = vt + n * kPitch + g * kOwn;
    const T* v_get = vt + (4 * g + ((lane & 15) >> 2)) * kPitch + (lane & 3) * 4;

    bool odd = false;  // MULTI: this wave took out values that are no numbers, of keys that not all tokens see
    auto use = [&](Codes& x, int key0) __attribute__((always_inline)) {
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
        if (PAD) share.template clear<T>(x.k, x.ks);
        f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mma16(widened<C, T>(&x.k[t][f * kOf8], x.ks[t][f * 8 / kGroup]), q[f], s[t]);
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
                *reinterpret_cast<vec8<T>*>(v_put + t * 16 * kPitch + f * 8) = widened<C, T>(&x.v[t][f * kOf8], x.vs[t][f * 8 / kGroup]);
        if (MULTI && it.seq >= 0 && key0 + KT > full)
            odd |= take_odd<T, kOwn>(v_put, key0 + n >= full) | take_odd<T, kOwn>(v_put + 16 * kPitch, key0 + 16 + n >= full);
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        top = pair_max<16>(top);
        top = pair_max<32>(top);
        const float next = top * p.c - lift;
        const bool grown = next > m + kSlack<T>;
        if (__any(grown)) {
            const float to = grown ? next : m, scale = grown ? __builtin_amdgcn_exp2f(m - next) : 1.f;  // m = -inf: 0
            l *= scale;
#pragma unroll
            for (auto& y : o) y *= scale;
            m = to;
        }
        const float base = m == -INFINITY ? 0.f : m;
        vec8<T> pr;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(s[t][i], p.c, -base));
                l += e;
                pr[4 * t + i] = (T)e;
            }
        auto value = [&](int d) __attribute__((always_inline)) {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(v_get + d * 16));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(v_get + 16 * kPitch + d * 16));
            struct { s16x4 a, b; } both{a, b};
            return __builtin_bit_cast(vec8<T>, both);
        };
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = mma16(value(d), pr, o[d]);
    };
    // While a tile is used, the codes of the next are on their way, and the page ids of the one behind it.
    // (A loop for each way to load: a branch inside would wait for the loads that each side has under way.)
    auto run_once = [&](auto GRAIN, auto PAGED, auto ONCE) __attribute__((always_inline)) {
        Codes a, b;
        fetch(GRAIN, PAGED, ONCE, key, ids0, a);
        auto tile = [&](Codes& now, Codes& next) __attribute__((always_inline)) {
            const int ids2[2] = {page_id(key + 2 * kStep, 0), page_id(key + 2 * kStep, 1)};
            fetch(GRAIN, PAGED, ONCE, key + kStep, ids1, next);  // (past the end: the cache's first rows)
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
    auto run = [&](auto GRAIN, auto PAGED) __attribute__((always_inline)) { run_once(GRAIN, PAGED, std::false_type{}); };
    // A sequence's own keys, heads apart, are read by this workgroup alone: past the caches (4 sequences of 100001 keys 87.5 -> 79.9 us;
    // a prefix read so, which several workgroups share: 8 sequences behind 7901 keys 15.7 -> 16.0).
    const bool once = it.seq >= 0 && p.plan.suf_tiles == 1 && !p.near_units;
    if (key < it.end) {
        if (!SECOND && kOwn * C::kBits >= 128 && once && (!PAD || p.D % kOwn == 0) && whole_pages(p, page_mask >= 15))
            run_once(std::integral_constant<int, kOwn>{}, std::true_type{}, std::true_type{});
        else
            by_grain<kOwn, PAD, SECOND>(p, page_mask >= 15, run);
    }
    if (kTwice<T> && !SECOND) {
        uint64_t rows = far_rows(o);
        if (__builtin_expect(rows != 0, false)) {
            rows |= rows >> 32;
            rows |= rows >> 16;
            *lift_of_row = (rows >> n) & 1 ? kLift<T> - kLower : kLift<T>;
            return true;
        }
    }
    if (MULTI && odd) {
        auto own = [&](int key) { return ((key - it.begin) / KT & 1) == wave; };
        add_odd<T, C>(p, it, max(it.begin, full), vbase, vsbase, own, [&](int key, int d0, const vec8<T>& v) __attribute__((always_inline)) {
            const f32x4 x = odd_of<T>(v, g & 1, key < limit && (d0 >> 3 & 1) == g >> 1);
#pragma unroll
            for (int d = 0; d < ND; ++d)
                if (d0 / 16 == d) o[d] += x;
        });
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
    static_assert(NW * KT * kPitch * sizeof(T) >= ND * 64 * 16, "room for a wave's sums");
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
    if (wave == 1 || !row_ok) return false;
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
    return false;
}


constexpr int kBroadPad = 16;  // elements

// Tiles of 128 query rows, 32 a wave, on the 32 x 32 x 16 instructions.  Bound by vector and matrix instructions: 64 sequences behind
// 32768 keys (64 / 8 heads of 128, FP4) take 108 us in the median of 30 launches, 640 TFLOP/s (102 in the best; FP8 115 and 111).  Of
// 181 thousand clocks the matrix units are busy for 66 thousand and the vector units, which widen codes and take 134 million exponentials, for
// about 100; the two seldom at once, as a wave's parts depend on each other and two waves a SIMD are all that the registers hold.  Each
// wave widens the keys it multiplies by itself: 32 at a time, a half of their row a lane, the scores of the next 32 computed while the
// exponentials of these are.  The values of 64 keys are widened by the four waves together, 16 rows each, for all of them.
template <typename T, int DP, bool MULTI, class C, bool PAD, bool SECOND>
__device__ __forceinline__ bool attend_broad(const Pass<SECOND>& pass, bool prefix, float* lift_of_row, T* v0, T* v1) {
    constexpr int KT = 64, NF = DP / 16, ND = DP / 32, kPitch = DP + kBroadPad, kOf8 = C::kBits / 4;
    using KeyShare = Share<C, DP / 2>;
    using ValueShare = Share<C, DP / 4>;
    const AttendP& p = pass.p;
    Item it;
    if (!item_of<128>(p, prefix, near(p, prefix, pass.b), &it)) return false;
    const int lane = pass.thread & 63, wave = __builtin_amdgcn_readfirstlane(pass.thread >> 6);
    const int n = lane & 31, h = lane >> 5;    // of keys, and of scores: row n of 32
    const int vn = lane & 15, vg = lane >> 4;  // of values, as they are widened

    // Each lane looks up the page of its key of the two halves of a tile, and of its value.
    struct Ids {
        int k[2], v;
    };
    auto page_ids = [&](int key0) {
        auto look = [&](int key) { return key < it.end ? it.table[key >> p.page_shift] : -1; };
        return Ids{{look(key0 + n), look(key0 + 32 + n)}, look(key0 + wave * 16 + vn)};
    };
    int key = it.begin;
    Ids ids0 = page_ids(key), ids1 = page_ids(key + KT);
    it.len = it.seq < 0 ? p.prefix_len : min(p.lens[it.seq], p.max_len);
    it.end = min(it.end, it.len);
    if (it.begin >= it.end && !p.direct) return false;

    const int row = it.row0 + wave * 32 + n;
    const bool row_ok = row < it.rows, idle_wave = it.row0 + wave * 32 >= it.rows;  // (which only widens values)
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
            const int d = h * (DP / 2) + f * 8;
            q[f] = row_ok && d < p.D ? *reinterpret_cast<const vec8<T>*>(src + d) : vec8<T>{};
        }
    }
    f32x16 o[ND];
#pragma unroll
    for (auto& x : o) x = f32x16{};
    float m = -INFINITY, l = 0.f;
    const float lift = SECOND ? *lift_of_row : kLift<T>;

    const uint8_t* kbase = static_cast<const uint8_t*>(p.k) + it.kv * p.head_stride;
    const uint8_t* vbase = static_cast<const uint8_t*>(p.v) + it.kv * p.head_stride;
    const uint8_t* ksbase = p.k_scale + it.kv * p.s_head;
    const uint8_t* vsbase = p.v_scale + it.kv * p.s_head;
    const int page_mask = (1 << p.page_shift) - 1;
    const KeyShare key_share(h * (DP / 2), p.D);
    const ValueShare value_share(vg * (DP / 4), p.D);

    // As of thin workgroups: only loads, of a masked key those of the cache's first rows, made zeros where they are used.
    struct Keys {
        uint32_t w[1][KeyShare::kWords];
        uint8_t s[1][KeyShare::kScales];
        uint32_t valid;  // bit j: key j of the 32 is not masked
    };
    struct Values {
        uint32_t w[ValueShare::kWords];
        uint8_t s[ValueShare::kScales];
        bool there;
    };
    auto fetch_keys = [&](auto GRAIN, auto PAGED, int key0, int id, Keys& x) __attribute__((always_inline)) {
        if constexpr (decltype(PAGED)::value) {  // each 16 keys in one page
            int64_t c_at[2], s_at[2];
            x.valid = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int at = key0 + t * 16, its = __builtin_amdgcn_readlane(id, t * 16);
                const bool there = (unsigned)its < (unsigned)p.n_pages && at < it.end;
                x.valid |= there ? (it.end - at >= 16 ? 0xffffu : (1u << (it.end - at)) - 1) << (16 * t) : 0u;
                const int pg = there ? its : 0, place = at & page_mask;
                c_at[t] = place_of(pg, p.page_stride, place, p.token_stride);
                s_at[t] = place_of(pg, p.s_page, place, p.s_token);
            }
            const bool second = n >= 16;
            const uint32_t in = n & 15;
            key_share.load(GRAIN, std::false_type{}, std::false_type{}, kbase + (second ? c_at[1] : c_at[0]), ksbase + (second ? s_at[1] : s_at[0]),
                           in * (uint32_t)p.token_stride, in * (uint32_t)p.s_token, x.w[0], x.s[0]);
        } else {
            const int at = key0 + n;
            const bool there = (unsigned)id < (unsigned)p.n_pages && at < it.end;
            x.valid = (uint32_t)__ballot(there);
            const int64_t pg = there ? id : 0, place = at & page_mask;
            key_share.load(GRAIN, std::false_type{}, std::false_type{}, kbase + pg * p.page_stride + place * p.token_stride,
                           ksbase + pg * p.s_page + place * p.s_token, 0, 0, x.w[0], x.s[0]);
        }
    };
    auto fetch_values = [&](auto GRAIN, auto PAGED, int key0, int id, Values& x) __attribute__((always_inline)) {
        const int first = key0 + wave * 16;
        x.there = (unsigned)id < (unsigned)p.n_pages && first + vn < it.end;
        if constexpr (decltype(PAGED)::value) {
            const int its = __builtin_amdgcn_readfirstlane(id);
            const int pg = (unsigned)its < (unsigned)p.n_pages ? its : 0, place = first & page_mask;
            value_share.load(GRAIN, PAGED, std::false_type{}, vbase + place_of(pg, p.page_stride, place, p.token_stride),
                             vsbase + place_of(pg, p.s_page, place, p.s_token), vn * (uint32_t)p.token_stride, vn * (uint32_t)p.s_token, x.w, x.s);
        } else {
            const int64_t pg = x.there ? id : 0, place = (first + vn) & page_mask;
            value_share.load(GRAIN, PAGED, std::false_type{}, vbase + pg * p.page_stride + place * p.token_stride, vsbase + pg * p.s_page + place * p.s_token, 0, 0,
                             x.w, x.s);
        }
    };
    bool odd = false;  // MULTI: this wave took out values that are no numbers, of keys that not all tokens see
    auto put_values = [&](Values& x, int key0, T* buf) __attribute__((always_inline)) {
        if (!__all(x.there)) {
#pragma unroll
            for (int j = 0; j < ValueShare::kWords; ++j) x.w[j] = x.there ? x.w[j] : 0;
#pragma unroll
            for (int i = 0; i < ValueShare::kScales; ++i) x.s[i] = x.there ? x.s[i] : 0;
        }
        T* to = buf + (wave * 16 + vn) * kPitch + vg * (DP / 4);
#pragma unroll
        for (int f = 0; f < DP / 32; ++f) *reinterpret_cast<vec8<T>*>(to + f * 8) = widened<C, T>(&x.w[f * kOf8], x.s[f * 8 / kGroup]);
        if (MULTI && it.seq >= 0 && key0 + wave * 16 + 16 > full) odd |= take_odd<T, DP / 4>(to, key0 + wave * 16 + vn >= full);
    };
    auto clear = [&](Keys& x) __attribute__((always_inline)) {
        if (~x.valid != 0) {
            const bool there = (x.valid >> n) & 1;
#pragma unroll
            for (int j = 0; j < KeyShare::kWords; ++j) x.w[0][j] = there ? x.w[0][j] : 0;
#pragma unroll
            for (int i = 0; i < KeyShare::kScales; ++i) x.s[0][i] = there ? x.s[0][i] : 0;
        }
        if (PAD) key_share.template clear<T>(x.w, x.s);
    };
    auto score = [&](const Keys& x, int f, f32x16& s) __attribute__((always_inline)) {  // the f-th product of NF
        s = mma(widened<C, T>(&x.w[0][f * kOf8], x.s[0][f * 8 / kGroup]), q[f], s);
    };
    // where this lane finds element 32 t + n of keys 4 h + 0 .. 3 and + 8, by fours, transposed (rows 32 bytes apart in their banks)
    const int v_get = (4 * h + ((lane & 15) >> 2)) * kPitch + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;

    // 32 keys: their scores are in s; those of the next 32 are computed ahead.  Matrix and vector instructions of a wave run side
    // by side where they are asked for in turn, so the order is written down: a product of the scores ahead, each of which waits for
    // the one before, beside two exponentials; then the values' products, their operands read three products early.
    auto use = [&](f32x16& s, uint32_t valid, int key0, const T* vt, Keys& ahead) __attribute__((always_inline)) {
        // score i of a lane belongs to key 8 (i / 4) + 4 h + i % 4
        if (key0 + 32 > full || ~valid != 0) {
            const int left = limit - key0;
            const uint32_t below = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1, seen = (below & valid) >> (4 * h);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = (seen >> (8 * (i / 4) + i % 4)) & 1 ? s[i] : -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = pair_max<32>(top);
        const float next = top * p.c - lift;
        const bool grown = next > m + kSlack<T>;
        if (__any(grown)) {
            const float to = grown ? next : m, scale = grown ? __builtin_amdgcn_exp2f(m - next) : 1.f;  // m = -inf: 0
            l *= scale;
#pragma unroll
            for (auto& x : o) x *= scale;
            m = to;
        }
        const float base = m == -INFINITY ? 0.f : m;
        auto value = [&](int kk, int t) __attribute__((always_inline)) {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const T* at = vt + v_get + kk * 16 * kPitch + t * 32;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 8 * kPitch));
            struct { s16x4 a, b; } both{a, b};
            return __builtin_bit_cast(vec8<T>, both);
        };
        __builtin_amdgcn_s_setprio(1);  // before waves that work out addresses or wait (114.3 -> 112.5 us)
        clear(ahead);
        constexpr int kEarly = 3;
        vec8<T> pr[2], val[2 * ND];
        f32x16 after{};
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            score(ahead, f, after);
#pragma unroll
            for (int i = f * 16 / NF; i < (f + 1) * 16 / NF; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(s[i], p.c, -base));
                l += e;
                pr[i / 8][i % 8] = (T)e;
            }
            if (f >= NF - kEarly) val[f - (NF - kEarly)] = value((f - (NF - kEarly)) / ND, (f - (NF - kEarly)) % ND);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 2 * ND; ++i) {
            if (i + kEarly < 2 * ND) val[i + kEarly] = value((i + kEarly) / ND, (i + kEarly) % ND);
            o[i % ND] = mma(val[i], pr[i / ND], o[i % ND]);
            __builtin_amdgcn_sched_barrier(0);
        }
        s = after;
        __builtin_amdgcn_s_setprio(0);
    };
    // The values of a tile are in shared memory; what this wave wrote there is seen by the others.
    auto landed = [&] {
        __builtin_amdgcn_s_waitcnt(0xc07f);  // (loads that are under way stay so)
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        __builtin_amdgcn_s_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    };
    auto run = [&](auto GRAIN, auto PAGED) __attribute__((always_inline)) {
        Keys ka, kb;
        Values x;
        fetch_values(GRAIN, PAGED, key, ids0.v, x);
        fetch_keys(GRAIN, PAGED, key, ids0.k[0], ka);
        fetch_keys(GRAIN, PAGED, key + 32, ids0.k[1], kb);
        put_values(x, key, v0);
        f32x16 s{};
        clear(ka);
#pragma unroll
        for (int f = 0; f < NF; ++f) score(ka, f, s);
        uint32_t valid_a = ka.valid;
        // While a tile is used, the next one's values are on their way, and 32 keys behind those whose scores are computed.
        auto tile = [&](const T* now, T* next) __attribute__((always_inline)) {
            landed();
            const Ids ids2 = page_ids(key + 2 * KT);
            fetch_values(GRAIN, PAGED, key + KT, ids1.v, x);
            fetch_keys(GRAIN, PAGED, key + KT, ids1.k[0], ka);
            if (!idle_wave) use(s, valid_a, key, now, kb);
            const uint32_t valid_b = kb.valid;
            valid_a = ka.valid;
            fetch_keys(GRAIN, PAGED, key + KT + 32, ids1.k[1], kb);
            if (!idle_wave) use(s, valid_b, key + 32, now + 32 * kPitch, ka);
            put_values(x, key + KT, next);
            key += KT;
            ids1 = ids2;
        };
        T *now = v0, *next = v1;
        while (key < it.end) {
            tile(now, next);
            T* const used = now;
            now = next, next = used;
        }
    };
    if (key < it.end) by_grain<DP / 4, PAD, SECOND>(p, page_mask >= 15, run);
    if (kTwice<T> && !SECOND) {
        __shared__ int waves_far[4];
        uint64_t rows = far_rows(o);
        if (lane == 0) waves_far[wave] = rows != 0;
        landed();
        if (__builtin_expect(waves_far[0] | waves_far[1] | waves_far[2] | waves_far[3], 0)) {
            rows |= rows >> 32;
            *lift_of_row = (rows >> n) & 1 ? kLift<T> - kLower : kLift<T>;
            return true;
        }
    }
    if (MULTI && it.seq >= 0) {
        __shared__ int waves_odd[4];
        if (lane == 0) waves_odd[wave] = odd;
        landed();
        if (waves_odd[0] | waves_odd[1] | waves_odd[2] | waves_odd[3]) {
            auto all = [](int) { return true; };
            add_odd<T, C>(p, it, max(it.begin, full), vbase, vsbase, all, [&](int key, int d0, const vec8<T>& v) __attribute__((always_inline)) {
                const f32x4 x = odd_of<T>(v, h, key < limit);
#pragma unroll
                for (int t = 0; t < ND; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (d0 != t * 32 + i * 8) continue;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][i * 4 + e] += x[e];
                    }
            });
        }
    }
    l += other_half(l);
    if (!row_ok) return false;
    const int64_t out_row = token * p.H + head;
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = t * 32 + 2 * i + 4 * h;
            if (d >= p.D) continue;
            if (p.direct) {
                Pack<T, 4> y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y.e[e] = (T)(l == 0.f ? 0.f : o[t][i + e] * inv);
                store_pack<T, 4>(p.out, token * p.o_token + head * p.o_head + d, y);
            } else {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : o[t][i + e];
                *reinterpret_cast<f32x4*>(p.part + (out_row * p.parts + it.part) * p.D + d) = v;
            }
        }
    if (h == 0 && !p.direct) {
        float* at = p.ml + (out_row * p.parts + it.part) * 2;
        at[0] = m;
        at[1] = l;
    }
    return false;
}

// Which shapes a launch holds (rows of up to 32 are thin: broad ones at 32 rows would leave three waves of four without work).  BOTH: a broad prefix beside thin sequences, eight workgroups of one after eight of the other (one
// for each XCD).
enum Shapes { THIN, BROAD, BOTH };

// Waves a SIMD that the registers are shared out for.
template <int DP, Shapes S, bool MULTI, class C>
constexpr int waves_of() {
    if (S == THIN) return DP <= 64 ? (C::kBits == 4 ? 4 : 3) : DP <= 128 ? (C::kBits == 4 ? 3 : 2) : 1;
    return DP <= 64 && C::kBits == 4 ? 3 : DP <= 128 ? 2 : 1;
}

template <typename T, int DP, Shapes S, bool MULTI, class C, bool PAD>
__global__ __launch_bounds__((S == THIN ? 128 : 256), (waves_of<DP, S, MULTI, C>())) void attend_codes_kernel(const AttendP p) {
    constexpr int kThin = 2 * 32 * (DP + kThinPad), kBroad = 64 * (DP + kBroadPad);
    static_assert(kBroad >= kThin, "room for either shape");
    __shared__ __attribute__((aligned(16))) T v0[S == THIN ? kThin : kBroad], v1[S == THIN ? 1 : kBroad];
    __shared__ float wave_ml[2][2][32];
    auto thin = [&](int b, bool prefix) __attribute__((always_inline)) {
        float lift;
        const bool again = attend_thin<T, DP, MULTI, C, PAD>(first_pass(p, b), prefix, &lift, v0, wave_ml);
        if constexpr (kTwice<T>)
            if (__builtin_expect(again, false)) attend_thin<T, DP, MULTI, C, PAD>(second_pass(b), prefix, &lift, v0, wave_ml);
    };
    auto broad = [&](auto SEVERAL, int b, bool prefix) __attribute__((always_inline)) {
        constexpr bool several = decltype(SEVERAL)::value;
        float lift;
        const bool again = attend_broad<T, DP, several, C, PAD>(first_pass(p, b), prefix, &lift, v0, v1);
        if constexpr (kTwice<T>)
            if (__builtin_expect(again, false)) attend_broad<T, DP, several, C, PAD>(second_pass(b), prefix, &lift, v0, v1);
    };
    int b = blockIdx.x;
    if constexpr (S == BOTH) {
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
        if (prefix)
            broad(std::false_type{}, b, true);
        else if (threadIdx.x < 128)
            thin(b, false);
    } else {
        const bool prefix = b < p.pre_items;
        if (!prefix) b -= p.pre_items;
        if constexpr (S == THIN)
            thin(b, prefix);
        else
            broad(std::bool_constant<MULTI>{}, b, prefix);
    }
}

template <typename T, int DP, bool PAD, class C>
hipError_t attend_codes(const ls_kv_cache& shape, const ls_kvq_cache& c, const ls_attend_args& a, const AttendPlan& plan, void* ws,
                        hipStream_t st) {
    AttendP p = attend_params(shape, a, plan, ws);
    p.k_scale = c.k_scale, p.v_scale = c.v_scale;
    p.by_near = Div(p.KV * plan.suf_tiles);
    p.near_units = c.n_kv_heads > 1 && c.head_stride < c.token_stride ? p.S * std::max(plan.suf_parts, 1) : 0;
    p.s_page = c.scale_page_stride, p.s_head = c.scale_head_stride, p.s_token = c.scale_token_stride;
    auto go = [&](Shapes s, int pre_items, int suf_items) {
        p.pre_items = pre_items;
        p.suf_items = suf_items;
        const dim3 grid((unsigned)(pre_items + suf_items)), wg(s == THIN ? 128 : 256);
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, wg, 0, st, p);
            return hipGetLastError();
        };
        const bool multi = p.n_q > 1 && suf_items;
        if (s == THIN) return multi ? launch(attend_codes_kernel<T, DP, THIN, true, C, PAD>) : launch(attend_codes_kernel<T, DP, THIN, false, C, PAD>);
        if (s == BROAD) return multi ? launch(attend_codes_kernel<T, DP, BROAD, true, C, PAD>) : launch(attend_codes_kernel<T, DP, BROAD, false, C, PAD>);
        return multi ? launch(attend_codes_kernel<T, DP, BOTH, true, C, PAD>) : launch(attend_codes_kernel<T, DP, BOTH, false, C, PAD>);
    };
    return launch_plan<T, DP>(p, plan.pre_wide ? BROAD : THIN, plan.suf_wide ? BROAD : THIN, BOTH, st, go);
}

template <typename T, class C>
hipError_t attend_codes_dim(const ls_kvq_cache& c, ls_dtype type, const ls_attend_args& a, const AttendPlan& plan, void* ws, hipStream_t st) {
    const ls_kv_cache shape = shape_of(c, type);
    const int d = c.head_dim;
    if (d <= 64) return (d == 64 ? attend_codes<T, 64, false, C> : attend_codes<T, 64, true, C>)(shape, c, a, plan, ws, st);
    if (d <= 128) return (d == 128 ? attend_codes<T, 128, false, C> : attend_codes<T, 128, true, C>)(shape, c, a, plan, ws, st);
    return (d == 256 ? attend_codes<T, 256, false, C> : attend_codes<T, 256, true, C>)(shape, c, a, plan, ws, st);
}

}  // namespace
}  // namespace ls

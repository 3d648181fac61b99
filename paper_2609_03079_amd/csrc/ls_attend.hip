// ls_attend.hip - attention over keys and values of 16 bits, and the plan of every attention.
#include "ls_attend.h"

namespace ls {

bool plan_attend(const ls_kv_cache& c, int bits, const ls_attend_args& a, size_t ws_bytes, int n_cu, AttendPlan* plan) {
    const int G = a.n_heads / c.n_kv_heads;
    const int64_t pre_rows = (int64_t)a.n_seqs * a.n_q * G, suf_rows = (int64_t)a.n_q * G;
    const int64_t part_bytes = (int64_t)a.n_seqs * a.n_q * a.n_heads * (c.head_dim + 2) * 4;
    plan->pre_wide = pre_rows > 32;
    plan->suf_wide = suf_rows > 32;
    plan->pre_thin = bits < 16 && !plan->pre_wide;
    plan->suf_thin = bits < 16 && !plan->suf_wide;
    plan->pre_tiles = (int)ceil_div(pre_rows, plan->pre_wide ? 128 : plan->pre_thin ? 16 : 32);
    plan->suf_tiles = (int)ceil_div(suf_rows, plan->suf_wide ? 128 : plan->suf_thin ? 16 : 32);
    plan->alike = plan->pre_wide == plan->suf_wide;
    // Workgroups that run at once on a compute unit (by shared memory and registers: wide ones of several tokens
    // take more than half of those); the time of a key and of a start and end, as measured with the unit full (us).
    enum Kind { NARROW_ITEM, WIDE_ITEM, TOKENS_ITEM };
    const Kind pre_kind = plan->pre_wide ? WIDE_ITEM : NARROW_ITEM;
    const Kind suf_kind = !plan->suf_wide ? NARROW_ITEM : a.n_q > 1 && a.max_len ? TOKENS_ITEM : WIDE_ITEM;
    const int wide_cu = c.head_dim <= 128 ? 2 : 1, narrow_cu = plan->suf_thin ? (c.head_dim <= 64 ? 6 : c.head_dim <= 128 ? (bits == 4 && a.n_q == 1 ? 6 : 4) : 2) : bits < 16 ? (c.head_dim <= 128 ? 4 : 2) : c.head_dim <= 64 ? 4 : c.head_dim <= 128 ? 2 : 1;
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
    return c.dtype == LS_F16 ? attend_dim<_Float16, Whole>(c, nullptr, a, plan, ws, st) : attend_dim<__bf16, Whole>(c, nullptr, a, plan, ws, st);
}

}  // namespace ls

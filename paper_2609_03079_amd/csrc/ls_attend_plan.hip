// ls_attend_plan.hip - how an attention over codes is cut into parts (host code).
#include <algorithm>
#include <cmath>

#include "ls_ops_internal.h"

namespace ls {

// As plan_attend: the chunks of keys with the least estimated time.  Rows of up to 32 are thin (tiles of 16), more of them broad (tiles
// of 128); prefix and sequences of one shape go in one launch.  Against the plan of the 16-bit kernels, whose tiles of 32 rows and
// chunks from 128 keys cost otherwise: 1000 keys x 32 heads 9.7 -> 8.7 us, 8 sequences behind 7901 keys 17.0 -> 15.7, 5 x 4 tokens
// 12.1 -> 10.3, 4 sequences of 100001 keys 89.8 -> 87.3.
bool plan_attend_codes(const ls_kvq_cache& c, const ls_attend_args& a, size_t ws_bytes, int n_cu, AttendPlan* plan) {
    const int G = a.n_heads / c.n_kv_heads, bits = c.code == LS_FP4 ? 4 : 8, dp = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
    const int64_t pre_rows = (int64_t)a.n_seqs * a.n_q * G, suf_rows = (int64_t)a.n_q * G;
    const int64_t part_bytes = (int64_t)a.n_seqs * a.n_q * a.n_heads * (c.head_dim + 2) * 4;
    plan->pre_wide = pre_rows > 32;
    plan->suf_wide = suf_rows > 32;
    plan->pre_tiles = (int)ceil_div(pre_rows, plan->pre_wide ? 128 : 16);
    plan->suf_tiles = (int)ceil_div(suf_rows, plan->suf_wide ? 128 : 16);
    plan->alike = plan->pre_wide == plan->suf_wide;
    plan->together = false;
    enum Kind { THIN, BROAD };
    const Kind pre_kind = plan->pre_wide ? BROAD : THIN;
    const Kind suf_kind = plan->suf_wide ? BROAD : THIN;
    // workgroups that run at once on a compute unit, by registers
    const int thin_cu = dp == 64 ? (bits == 4 ? 8 : 6) : dp == 128 ? (bits == 4 ? 6 : 4) : 2;
    const int broad_cu = dp == 64 ? 3 : dp == 128 ? 2 : 1;
    // Time of a workgroup among others on its compute unit (us): a start and an end, and the keys.  Thin: the wave's own chain and
    // the unit's share of the memory (5.3 TB/s), which overlap but for the loads that a lone wave has not in flight.  Broad: as
    // measured with the unit full, of FP4 (FP8 takes 115 us where FP4 takes 108, a part of any length as much more).
    const double key_bytes = 2.0 * ((double)c.head_dim * bits / 8 + (double)ceil_div(c.head_dim, 32));
    auto item_us = [&](Kind kind, int64_t chunk, int64_t at_once) {
        if (kind == THIN) return 4.5 + chunk * std::hypot(0.0118 * (dp + 128) / 256, at_once * key_bytes / (5.3e6 / n_cu));
        return 4.0 + chunk * (dp == 64 ? 0.056 : dp == 128 ? 0.044 : 0.088);
    };
    auto run_us = [&](Kind kind, int64_t chunk, int64_t items) {
        const int64_t per_cu = kind == THIN ? thin_cu : broad_cu, slots = per_cu * n_cu, rest = items % slots;
        return (items / slots) * item_us(kind, chunk, per_cu) + (rest ? item_us(kind, chunk, ceil_div(rest, n_cu)) : 0.0);
    };
    // parts are written, and read by the join, 16 of a row at a time
    auto join_us = [&](int64_t parts) { return parts * 2.0 * part_bytes / 5e6 + 0.6 * ceil_div(parts, 16); };
    // Chunks of whole tiles; prefix and sequences, where there are both, have half of kMaxParts and of the workspace each.
    const int shares = a.prefix_len && a.max_len ? 2 : 1;
    double least = 0;
    auto choose = [&](Kind kind, int64_t n_pre, int64_t pre_keys, int64_t n_suf, int64_t suf_keys) {
        int64_t best = 0;
        const int64_t most = round_up((size_t)std::max<int64_t>(std::max(pre_keys, suf_keys), 1), 64);
        for (int64_t chunk = 64;; chunk = std::min(most, chunk + std::max<int64_t>(64, chunk / 16 / 64 * 64))) {
            const int64_t pp = ceil_div(pre_keys, chunk), sp = ceil_div(suf_keys, chunk), items = n_pre * pp + n_suf * sp;
            const bool fits = std::max(pp, sp) <= kMaxParts / shares && std::max(pp, sp) * part_bytes <= (int64_t)ws_bytes / shares &&
                              (n_pre + 8) * (pp + 8) + n_suf * sp < (int64_t)1 << 24;  // 2^32 threads of a launch
            if (fits) {
                const double t = run_us(kind, chunk, items) + join_us(pp + sp);
                if (!best || t < least) best = chunk, least = t;
            }
            if (chunk >= most) break;
        }
        return (int)best;
    };
    const int64_t n_pre = a.prefix_len ? (int64_t)c.n_kv_heads * plan->pre_tiles : 0;
    const int64_t n_suf = (int64_t)a.n_seqs * c.n_kv_heads * plan->suf_tiles;
    auto at_once = [&](int64_t pre_chunk, int64_t suf_chunk) {  // all workgroups, the prefix's filled up to eights
        return n_pre * ceil_div(a.prefix_len, pre_chunk) + 8 * plan->pre_tiles + n_suf * ceil_div(a.max_len, suf_chunk) <= (int64_t)broad_cu * n_cu;
    };
    if (!a.prefix_len) {
        plan->pre_chunk = plan->suf_chunk = choose(suf_kind, 0, 0, n_suf, a.max_len);
    } else {
        // one after the other, or in one launch of one shape
        plan->pre_chunk = choose(pre_kind, n_pre, a.prefix_len, 0, 0);
        double apart = least + 2.0;
        plan->suf_chunk = choose(suf_kind, 0, 0, n_suf, a.max_len);
        apart += least;
        const bool found = plan->pre_chunk && plan->suf_chunk;
        if (plan->alike) {
            const int both = choose(suf_kind, n_pre, a.prefix_len, n_suf, a.max_len);
            if (both && (!found || least <= apart))
                plan->pre_chunk = plan->suf_chunk = both;
            else
                plan->alike = false;
        } else if (plan->pre_wide && found && a.max_len && !at_once(plan->pre_chunk, plan->suf_chunk)) {
            // longer parts that let a broad prefix and thin sequences run at once, if that costs less
            int64_t chunk = round_up((size_t)((n_pre * a.prefix_len + n_suf * a.max_len) / ((int64_t)n_cu * broad_cu) + 1), 64);
            for (int i = 0; i < 8 && !at_once(chunk, chunk); ++i) chunk += 64;
            const int64_t parts = ceil_div(a.prefix_len, chunk) + ceil_div(a.max_len, chunk);
            if (at_once(chunk, chunk) && parts <= kMaxParts && parts * part_bytes <= (int64_t)ws_bytes &&
                std::max(item_us(BROAD, chunk, 2), item_us(THIN, chunk, 2)) + join_us(parts) < apart)
                plan->pre_chunk = plan->suf_chunk = (int)chunk;
        }
    }
    if (!plan->pre_chunk || !plan->suf_chunk) return false;
    plan->pre_parts = (int)ceil_div(a.prefix_len, plan->pre_chunk);
    plan->suf_parts = (int)ceil_div(a.max_len, plan->suf_chunk);
    if (plan->pre_parts + plan->suf_parts == 0) plan->suf_parts = 1;  // no key anywhere: rows of zeros
    plan->together = plan->pre_parts && plan->suf_parts && plan->pre_wide && !plan->suf_wide && at_once(plan->pre_chunk, plan->suf_chunk);
    return true;
}

}  // namespace ls

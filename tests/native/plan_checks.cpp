// The plans of the attention over codes as a host function: what a launch would do, in numbers.
#include "../../paper_2609_03079_amd/csrc/ls_attend_plan.hip"

extern "C" {
// False where no split fits.  out: parts of the prefix and of the sequences, bytes of partial results that the launches write in the workspace,
// workgroups of the launches before the join (two where prefix and sequences go apart; the second may be 0), keys of a part of each.
int plan_of(const ls_kvq_cache* c, const ls_attend_args* a, uint64_t ws_bytes, int n_cu, int64_t* out) {
    ls::AttendPlan p;
    if (!ls::plan_attend_codes(*c, *a, ws_bytes, n_cu, &p)) return 0;
    const int64_t rows = (int64_t)a->n_seqs * a->n_q * a->n_heads, parts = p.pre_parts + p.suf_parts;
    const bool direct = p.pre_parts == 0 && p.suf_parts == 1;
    const int64_t pre = (int64_t)ls::round_up((size_t)p.pre_parts * c->n_kv_heads, 8) * p.pre_tiles;
    const int64_t suf = (int64_t)p.suf_parts * a->n_seqs * c->n_kv_heads * p.suf_tiles;
    const bool once = pre == 0 || suf == 0 || p.alike || p.together;
    const int64_t numbers[] = {p.pre_parts, p.suf_parts, direct ? 0 : rows * parts * (c->head_dim + 2) * 4, once ? pre + suf : pre, once ? 0 : suf,
                               p.pre_chunk, p.suf_chunk, p.pre_wide, p.suf_wide, p.alike, p.together};
    for (int i = 0; i < 11; ++i) out[i] = numbers[i];
    return 1;
}
}

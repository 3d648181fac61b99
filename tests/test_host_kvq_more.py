"""Rows that ls_kvq_read takes and refuses, without a GPU (the C entry points built for the host, tests/native/ops_checks.cpp)."""
import itertools

import paper_2609_03079_amd as lsffn
from test_host_kvq import cache, call, ctx, lib, read  # noqa: F401


def apart(strides, counts, n):
    """No two rows of n elements overlap, every row looked at."""
    seen = set()
    for at in itertools.product(*(range(c) for c in counts)):
        start = sum(i * s for i, s in zip(at, strides))
        row = range(start, start + n)
        if not seen.isdisjoint(row):
            return False
        seen.update(row)
    return True


def test_rows_that_overlap_are_refused_and_no_others(lib, ctx):
    """Tokens and heads at any strides, nested in each other or not."""
    answers = {True: 0, False: 0}
    for tokens, heads in ((1, 1), (1, 3), (2, 1), (2, 2), (3, 2), (2, 3), (5, 4)):
        for by_token, by_head in itertools.product((0, 4, 8, 12, 16, 20, 24, 40, 48, 56, 64, 72, 160), repeat=2):
            ok = apart((by_token, by_head), (tokens, heads), 8)
            c = cache(n_kv_heads=heads, head_dim=8, token_stride=4, head_stride=64, page_stride=64 * heads)
            for which in ("k", "v"):
                far = dict(k_token_stride=8, k_head_stride=8 * tokens, v_token_stride=8, v_head_stride=8 * tokens)
                st = call(lib, ctx, "read", c, read(n_tokens=tokens, **{**far, which + "_token_stride": by_token, which + "_head_stride": by_head}))
                assert st == (lsffn.LS_OK if ok else lsffn.LS_E_INVAL), (tokens, heads, by_token, by_head, which)
                assert ok or "overlap" in lib.ls_ops_last_error(ctx).decode()
            answers[ok] += 1
    assert min(answers.values()) > 100


def test_rows_far_apart(lib, ctx):
    """Strides up to the largest, whose products pass 64 bits."""
    c = cache(n_kv_heads=4096, head_dim=8, token_stride=4, head_stride=64, page_stride=64 * 4096)
    big = 2 ** 63 - 8
    assert call(lib, ctx, "read", c, read(n_tokens=2 ** 31 - 1, k_token_stride=8, k_head_stride=big, v_token_stride=2 ** 15, v_head_stride=8)) == lsffn.LS_OK
    assert call(lib, ctx, "read", c, read(n_tokens=2 ** 31 - 1, k_token_stride=big, k_head_stride=8, v_token_stride=2 ** 15, v_head_stride=8)) == lsffn.LS_OK
    assert call(lib, ctx, "read", c, read(n_tokens=2 ** 31 - 1, k_token_stride=8, k_head_stride=8 * (2 ** 31 - 2), v_token_stride=2 ** 15,
                                          v_head_stride=8)) == lsffn.LS_E_INVAL
    assert call(lib, ctx, "read", c, read(n_tokens=2 ** 31 - 1, k_token_stride=8, k_head_stride=8 * (2 ** 31 - 1), v_token_stride=2 ** 15,
                                          v_head_stride=8)) == lsffn.LS_OK

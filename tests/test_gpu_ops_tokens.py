"""Attention of several query tokens a sequence, for every head size and type: wide and narrow workgroups, and keys and
values that are no numbers where only the later tokens see them."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_ops import BOTH, check_attend, ops  # noqa: E402, F401

DIMS = [64, 80, 128, 136, 256]


@pytest.mark.parametrize("dt", BOTH, ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("heads,kv,n_q", [(24, 1, 5), (64, 8, 8), (2, 1, 16), (8, 2, 3)])
def test_attend_tokens(ops, dt, dim, heads, kv, n_q):
    # 120, 64, 32 and 12 rows a sequence and key/value head; lengths that leave rows which see nothing or the prefix alone
    lens = [n_q, 90, n_q - 1, 0, -1, 1, 64, 65, 333]
    check_attend(ops, lens=lens, heads=heads, kv=kv, n_q=n_q, dim=dim, dt=dt, seed=dim)
    check_attend(ops, lens=lens, prefix=150, heads=heads, kv=kv, n_q=n_q, dim=dim, dt=dt, layout="token", bad_pages=True, seed=dim + 1)


@pytest.mark.parametrize("dt", BOTH, ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("heads,n_q", [(24, 5), (2, 16)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_later_tokens_key_or_value_stays_out(ops, dt, dim, heads, n_q, bad):
    """Seen by the last token alone, or by all but the first (in the tile before the last where there are 16): the
    others keep the bits that they have without it."""
    args = dict(lens=[70, 30], prefix=50, heads=heads, kv=1, n_q=n_q, dim=dim, dt=dt, seed=dim)
    clean = check_attend(ops, **args).clone()
    for back in (1, n_q - 1):
        for which in ("k", "v"):
            def touch(kc, vc, pages, prefix_pages):
                at = 70 - back
                (kc if which == "k" else vc)[pages[0, at // 16], :, at % 16, 3] = bad
            out = check_attend(ops, touch=touch, **args)
            first = n_q - back
            assert torch.equal(out[:first], clean[:first]) and torch.equal(out[n_q:], clean[n_q:]), (back, which)
            if which == "v":
                assert not torch.any(torch.isfinite(out[first:n_q, :, 3]))
            elif math.isnan(bad):
                assert torch.all(torch.isnan(out[first:n_q]))

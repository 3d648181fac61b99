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


def attend_us(ops, S, n_q, heads, kv, dim, own, prefix):
    """Microseconds of a call among others, the least of several rounds."""
    page, dt, dev = 64, torch.bfloat16, "cuda:0"
    n, pre = -(-own // page), -(-prefix // page)
    g = torch.Generator(dev).manual_seed(1)
    kc, vc = (torch.randn((n * S + pre, kv, page, dim), device=dev, generator=g).to(dt) for _ in range(2))
    pages = torch.arange(n * S, dtype=torch.int32, device=dev).view(S, n)
    prefix_pages = torch.arange(n * S, n * S + pre, dtype=torch.int32, device=dev)
    lens = torch.full((S,), own, dtype=torch.int32, device=dev)
    q = torch.randn((S * n_q, heads, dim), device=dev, generator=g).to(dt)
    out, best = torch.empty_like(q), math.inf
    for _ in range(8):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        torch.cuda.synchronize()
        a.record()
        for _ in range(10):
            ops.ls_attend(q, kc, vc, pages, lens, out, max_len=own, n_q=n_q, scale=dim ** -0.5, prefix_pages=prefix_pages, prefix_len=prefix)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 100)
    return best


@pytest.mark.parametrize("S,n_q,heads,kv,dim,own,prefix", [(16, 8, 64, 8, 128, 512, 8192), (64, 16, 32, 8, 128, 200, 16384),
                                                           (16, 8, 64, 8, 64, 512, 8192)])
def test_tokens_cost_little_more_than_as_many_heads(ops, S, n_q, heads, kv, dim, own, prefix):
    """The same rows and keys, once as tokens of a sequence and once as heads of one token: what the masks of a
    sequence's last keys cost must not be paid along the prefix, nor a second round of workgroups by a
    plan that counts more of them at once than run."""
    tokens = attend_us(ops, S, n_q, heads, kv, dim, own, prefix)
    one = attend_us(ops, S, 1, heads * n_q, kv, dim, own, prefix)
    print(f"{tokens:.1f} us, as heads {one:.1f}")
    assert tokens <= 1.6 * one

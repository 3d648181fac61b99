"""Attention rows that share a wave with others, and weights far below their row's largest."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_ops import BOTH, DEV, ops  # noqa: E402, F401


@pytest.mark.parametrize("dt", BOTH, ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("shared", [False, True], ids=["own", "prefix"])
def test_a_row_does_not_depend_on_the_rows_of_its_wave(ops, dt, dim, shared):
    """Heads 0 to 3 see the same score everywhere: their maximum stays.  That of heads 4 to 7, in the same
    wave, rises with every tile in one call and not at all in the other; heads 0 to 3 keep their bits."""
    S, kv, G, page, n = 8, 64, 8, 64, 16384
    kc, vc = (torch.zeros((n // page, kv, page, dim), dtype=dt, device=DEV) for _ in range(2))
    kc[..., 0] = 1
    kc[..., 1] = (torch.arange(n, device=DEV).view(-1, 1, page) * (4 / n)).to(dt)
    vc.normal_(generator=torch.Generator(DEV).manual_seed(dim))
    pages = torch.arange(n // page, dtype=torch.int32, device=DEV)
    q = torch.zeros((S, kv, G, dim), dtype=dt, device=DEV)
    q[:, :, :4, 0] = torch.tensor([301.0, 517.0, 911.0, 1511.0], dtype=dt, device=DEV)
    outs = []
    for loud in (0.0, 100.0):
        q[:, :, 4:, 1] = loud
        out = torch.empty((S, kv * G, dim), dtype=dt, device=DEV)
        if shared:
            args = dict(max_len=0, prefix_pages=pages, prefix_len=n)
        else:
            args = dict(max_len=n)
        lens = torch.full((S,), 0 if shared else n, dtype=torch.int32, device=DEV)
        ops.ls_attend(q.view(S, kv * G, dim), kc, vc, None if shared else pages.repeat(S, 1), lens, out, scale=1.0, **args)
        outs.append(out.view(S, kv, G, dim))
    assert torch.equal(outs[0][:, :, :4], outs[1][:, :, :4])
    # equal weights: the mean of the values.  Weights and the result are rounded once each, a sum of n terms
    # in fp32 is off by far less
    u = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dt]
    mean, size = (f(vc.double()).transpose(1, 2).flatten(0, 1).mean(0)[:, None] for f in (lambda v: v, torch.abs))
    assert torch.all((outs[1][:, :, :4].double() - mean).abs() <= u * mean.abs() + 2 * u * size)
    assert math.isfinite(float(outs[1].double().sum()))


@pytest.mark.parametrize("dt", BOTH, ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 80, 256])
@pytest.mark.parametrize("form", ["own", "prefix", "tokens"])
@pytest.mark.parametrize("gap", [14.0, 17.5, 19.0])
def test_many_keys_far_below_the_largest_count(ops, dt, dim, form, gap):
    """One key's score is `gap` above all others' and its value is zero: the result is what the others add."""
    S, G, page, n_q, n = 12, 4, 16, 3 if form == "tokens" else 1, 640
    kc, vc = (torch.zeros((n // page, 1, page, dim), dtype=dt, device=DEV) for _ in range(2))
    kc[0, 0, 5, 0] = 1
    vc.uniform_(500, 1500, generator=torch.Generator(DEV).manual_seed(int(gap)))
    vc[0, 0, 5] = 0
    pages = torch.arange(n // page, dtype=torch.int32, device=DEV)
    q = torch.zeros((S * n_q, G, dim), dtype=dt, device=DEV)
    q[..., 0] = gap
    out = torch.empty_like(q)
    if form == "prefix":
        args = dict(max_len=0, prefix_pages=pages, prefix_len=n)
    else:
        args = dict(max_len=n)
    lens = torch.full((S,), 0 if form == "prefix" else n, dtype=torch.int32, device=DEV)
    ops.ls_attend(q, kc, vc, None if form == "prefix" else pages.repeat(S, 1), lens, out, n_q=n_q, scale=1.0, **args)
    v = vc.double().view(n, dim)
    u = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dt]
    # a weight is rounded to u of itself or half a step of 2^-31 of the largest, its exponent (below 64, rounded twice)
    # to 2^-18 and the exponential to a few of fp32's; so is the sum; the result is rounded once, to u or half a subnormal step
    for i in range(n_q):
        seen = v[:n - n_q + 1 + i]
        w = math.exp(-gap)
        total = 1 + (len(seen) - 1) * w
        ref, size = w * seen.sum(0) / total, seen.sum(0) / total
        tol = (2 * u + 2.0 ** -17) * ref + (2.0 ** -32 * size if dt == torch.float16 else 0) + 2.0 ** -25
        assert torch.all((out[i::n_q].double() - ref).abs() <= tol)


@pytest.mark.parametrize("dt", BOTH, ids=["f16", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("shared", [False, True], ids=["own", "prefix"])
@pytest.mark.parametrize("at", [0, 77, 2000, 4095])
def test_a_visible_value_that_is_no_number_counts_at_any_weight(ops, dt, bad, shared, at):
    """A key 200 below the largest, the value of whose element 3 is no number: so is the row's element 3, and no other."""
    n, G, page, dim = 4096, 4, 64, 64
    kc, vc = (torch.zeros((n // page, 1, page, dim), dtype=dt, device=DEV) for _ in range(2))
    vc.normal_(generator=torch.Generator(DEV).manual_seed(at))
    top = 1000
    kc[top // page, 0, top % page, 0] = 1
    vc[at // page, 0, at % page, 3] = bad
    pages = torch.arange(n // page, dtype=torch.int32, device=DEV)
    q = torch.zeros((1, G, dim), dtype=dt, device=DEV)
    q[..., 0] = 200
    out = torch.empty_like(q)
    args = dict(max_len=0, prefix_pages=pages, prefix_len=n) if shared else dict(max_len=n)
    lens = torch.full((1,), 0 if shared else n, dtype=torch.int32, device=DEV)
    ops.ls_attend(q, kc, vc, None if shared else pages[None], lens, out, scale=1.0, **args)
    fine = torch.isfinite(out)
    assert not fine[..., 3].any() and fine[..., :3].all() and fine[..., 4:].all()

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

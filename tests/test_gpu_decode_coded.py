"""The example's decoder stack on a cache of codes and with drafted tokens: a step's attention against 64 bits on the values that the
cache holds, drafted tokens against the definition of their acceptance, and steps of several tokens against steps of one."""
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_decode_batch import _example, _rel  # noqa: E402
from test_gpu_kvq import decoded  # noqa: E402
from test_gpu_verify import reference  # noqa: E402


@pytest.mark.parametrize("cache", ["fp4", "fp8"])
def test_attention_of_a_step(cache):
    """What attention gives against 64 bits on the rows that the cache holds (bfloat16 queries and outputs: 2^-7 of relative L2), and
    those rows against the values that were appended: an FP4 step is at most half of the code below it, uniform errors of half a
    step are a tenth of the values in the root mean square, 1/8 bounds a row's; an FP8 code is within 2^-4 of each."""
    ex = _example()
    shape = ex.Shape(layers=1)
    m = ex.Decoder(shape, 5, cache=cache)
    g = torch.Generator().manual_seed(3)
    m.prompt(torch.randn((77, shape.d), generator=g).cuda())
    b, lens = m.buffers(5), torch.zeros(5, dtype=torch.int32, device="cuda")
    for _ in range(20):
        m.step(torch.randn((5, shape.d), generator=g).cuda(), b, lens)
    kc, ks, vc, vs = m.layers[0][-4:]
    s, n = shape, int(lens[0])
    keys, values = decoded(kc, ks, s.dim), decoded(vc, vs, s.dim)
    v = b["qkv"].split([s.heads * s.dim, s.kv * s.dim, s.kv * s.dim], 1)[2].view(5, -1, s.dim)
    take = torch.cat([torch.arange(77), 80 + torch.arange(n)]).cuda()
    for i in range(5):
        page, at = int(m.pages[i, (n - 1) // ex.PAGE]), (n - 1) % ex.PAGE
        assert _rel(values[page, :, at], v[i]) < (1 / 8 if cache == "fp4" else 2 ** -4)
        rows = torch.cat([m.prompt_pages[:5], m.pages[i, :2]]).long()
        kk, vv = (t[rows].transpose(0, 1).flatten(1, 2)[:, take] for t in (keys, values))
        p = torch.softmax(b["q"][i].double().view(s.kv, -1, s.dim) @ kk.transpose(1, 2).contiguous() * s.dim ** -0.5, -1)
        assert _rel(b["o"][i].view(s.kv, -1, s.dim), p @ vv) < 2 ** -7
    m.close()


@pytest.mark.parametrize("cache", ["16", "fp4", "fp8"])
def test_drafted_tokens(cache):
    """Each step's tokens by the definition from the probabilities and numbers that it used, and the cache behind them: the next step
    overwrites what refused tokens left, so that a sequence's keys are those of its tokens alone."""
    ex = _example()
    m = ex.Decoder(ex.Shape(layers=1), 2, cache=cache)
    m.prompt(torch.randn((21, m.shape.d), generator=torch.Generator().manual_seed(4)).cuda())
    d = ex.Drafts(m, 3)
    said = [[int(t)] for t in d.last]
    for _ in range(12):
        lens = d.lens.tolist()
        d.step()
        assert d.ids[:, 0].tolist() == [x[-1] for x in said]
        ref = reference(d.p, d.ids[:, 1:], d.chance[:, 1:], d.chance[:, 0], torch.stack(d.q, 1))
        assert np.array_equal(d.tokens.cpu().numpy(), ref[0]) and np.array_equal(d.n_accepted.cpu().numpy(), ref[1])
        for i, x in enumerate(said):
            x += d.tokens[i, :ref[1][i] + 1].tolist()
            assert int(d.lens[i]) == lens[i] + ref[1][i] + 1 == len(x) - 1
    # the same tokens, one a step, in a stack of their own; layer 0's keys depend on the tokens alone
    one = ex.Decoder(m.shape, 2, cache=cache)
    one.prompt(torch.randn((21, m.shape.d), generator=torch.Generator().manual_seed(4)).cuda())
    b, lens = one.buffers(2), torch.zeros(2, dtype=torch.int32, device="cuda")
    n = min(len(x) for x in said) - 1
    for t in range(n):
        one.step(d.rows[torch.tensor([x[t] for x in said], device="cuda")], b, lens)
    for x, y in zip(m.layers[0][6:], one.layers[0][6:]):
        for i in range(2):
            rows = [t[m.pages[i].long()].transpose(1, 2).flatten(0, 1)[:n].view(torch.uint8) for t in (x, y)]
            assert torch.equal(*rows)
    m.close()
    one.close()


def test_example_runs(capsys, monkeypatch):
    ex = _example()
    for more in (["--cache", "fp8"], ["--cache", "fp4", "--drafts", "1"]):
        monkeypatch.setattr(sys, "argv", ["decode_batch.py", "--batch", "3", "--prompt", "21", "--steps", "4", *more])
        ex.main()
        assert "behind 21 shared tokens" in capsys.readouterr().out
    monkeypatch.setattr(sys, "argv", ["decode_batch.py", "--batch", "3", "--drafts", "2"])
    with pytest.raises(SystemExit):
        ex.main()

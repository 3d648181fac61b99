"""The example's decoder stack (examples/decode_batch.py): every layer of a step against 64 bits on the values
that the operators themselves produced, and the shared prompt against a copy of it in every sequence's own pages."""
import importlib.util
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("decode_batch", os.path.join(ROOT, "examples", "decode_batch.py"))
    m = importlib.util.module_from_spec(spec)
    sys.modules["decode_batch"] = m
    spec.loader.exec_module(m)
    return m


def _rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


def _rms(v):
    return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt()


def _product(x, w, s):
    x = x.double()
    top = x.abs().amax(1, keepdim=True)
    return (torch.round(x * 127 / top) @ w.double().T.contiguous()) * (top / 127) * s.double()


def test_attention_block_of_a_step():
    """One layer's attention half, teacher-forced: each stage in 64 bits from the stage before as the operators wrote it
    (bfloat16: half a unit of 2^-8 a rounding, and a bound of 2^-7 on each relative L2; the residual, in fp32,
    carries its input's rounding alone)."""
    ex = _example()
    shape = ex.Shape(layers=1)
    m = ex.Decoder(shape, 5)
    g = torch.Generator().manual_seed(3)
    m.prompt(torch.randn((77, shape.d), generator=g).cuda())
    b, lens = m.buffers(5), torch.zeros(5, dtype=torch.int32, device="cuda")
    for _ in range(20):
        x = torch.randn((5, shape.d), generator=g).cuda()
        m.step(x, b, lens)
    w_qkv, s_qkv, w_o, s_o, w1, w2, kc, vc = m.layers[0]
    s, n = shape, int(lens[0])
    assert _rel(b["h"], _rms(x.double()) * w1.double()) < 2 ** -7
    assert _rel(b["qkv"], _product(b["h"], w_qkv, s_qkv)) < 2 ** -7
    q, k, v = (t.view(5, -1, s.dim).double() for t in b["qkv"].split([s.heads * s.dim, s.kv * s.dim, s.kv * s.dim], 1))
    cs = m.table[77 + n - 1].double()
    c, si, half = cs[:64], cs[64:], 64

    def turn(t):
        return torch.cat([t[..., :half] * c - t[..., half:] * si, t[..., half:] * c + t[..., :half] * si], -1)
    assert _rel(b["q"], turn(q)) < 2 ** -7
    for i in range(5):
        page, at = int(m.pages[i, (n - 1) // ex.PAGE]), (n - 1) % ex.PAGE
        assert _rel(kc[page, :, at], turn(k)[i]) < 2 ** -7 and torch.equal(vc[page, :, at].double(), v[i])
        rows = torch.cat([m.prompt_pages[:5], m.pages[i, :2]]).long()
        take = torch.cat([torch.arange(77), 80 + torch.arange(n)]).cuda()
        keys, values = (t[rows].transpose(0, 1).flatten(1, 2)[:, take].double() for t in (kc, vc))  # [kv, keys, dim]
        qq = b["q"][i].double().view(s.kv, -1, s.dim)
        p = torch.softmax(qq @ keys.transpose(1, 2).contiguous() * s.dim ** -0.5, -1)
        assert _rel(b["o"][i].view(s.kv, -1, s.dim), p @ values) < 2 ** -7
    assert _rel(b["y"], _product(b["o"].view(5, -1), w_o, s_o)) < 2 ** -7
    assert _rel(b["x"][0], x.double() + _rms(b["y"].double()) * w2.double()) < 1e-6
    m.close()


def test_shared_prompt_equals_a_copy_for_each_sequence():
    """The prompt's keys copied into every sequence's own pages: the same attention but for the order of its sums."""
    ex = _example()
    shape = ex.Shape(layers=1)
    m = ex.Decoder(shape, 4)
    g = torch.Generator().manual_seed(4)
    n = 3 * ex.PAGE
    m.prompt(torch.randn((n, shape.d), generator=g).cuda())
    x, b = torch.randn((4, shape.d), generator=g).cuda(), m.buffers(4)
    m.step(x, b, torch.zeros(4, dtype=torch.int32, device="cuda"))
    shared = b["o"].clone()
    kc, vc = m.layers[0][-2:]
    for t in (kc, vc):
        own = t[m.pages[:, 0].long()].clone()
        t[m.pages[:, :3].long()] = t[m.prompt_pages[:3].long()][None]
        t[m.pages[:, 3].long()] = own
    alone = torch.empty_like(shared)
    m.ops.ls_attend(b["q"], kc, vc, m.pages, torch.full((4,), n + 1, dtype=torch.int32, device="cuda"), alone, max_len=shape.max_len,
                    scale=shape.dim ** -0.5)
    assert _rel(shared, alone) < 2 ** -7
    m.close()


def test_example_runs(capsys, monkeypatch):
    ex = _example()
    monkeypatch.setattr(sys, "argv", ["decode_batch.py", "--batch", "3", "--prompt", "21", "--steps", "4"])
    ex.main()
    assert "3 sequences behind 21 shared tokens" in capsys.readouterr().out

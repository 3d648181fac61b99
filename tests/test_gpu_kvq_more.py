"""The quantised cache's calls and ls_verify as programs call them: tensors of another GPU, two captured graphs of one context, heads near each other
in a page over many parts, calls larger than one launch."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_03079_amd as lsffn  # noqa: E402
from test_gpu_kvq import CODES, OUT, check_attend, empty_cache, packed, same, step, step_tensors  # noqa: E402
from test_gpu_ops import DEV, ints, ops, rand, refused, table  # noqa: E402, F401
from test_gpu_ops_devices import Elsewhere  # noqa: E402


def calls(ops):
    cache = dict(zip(("kc", "ks", "vc", "vs"), empty_cache(4, 2, 16, 64, "fp8")))
    for t in cache.values():
        t.view(torch.uint8).fill_(56)
    all4 = lambda t: [t[n] for n in ("kc", "ks", "vc", "vs")]  # noqa: E731
    k, q = rand((2, 2, 64), 1, torch.float16), rand((2, 4, 64), 2, torch.float16)
    yield lambda t: ops.ls_kvq_append(*all4(t), t["k"], t["v"], t["positions"], t["slots"], t["cs"], q=t["q"], q_out=t["q_out"]), \
        {**cache, "k": k, "v": k, "positions": ints([0, 1]), "slots": ints([0, 1]), "cs": table(8, 64), "q": q, "q_out": torch.empty_like(q)}
    yield lambda t: ops.ls_kvq_read(*all4(t), t["slots"], t["k"], t["v"]), \
        {**cache, "slots": ints([0, 1]), "k": torch.empty_like(k), "v": torch.empty_like(k)}
    yield lambda t: ops.ls_kvq_attend(t["q"], *all4(t), t["pages"], t["lens"], t["out"], max_len=16, scale=0.1, prefix_pages=t["prefix"], prefix_len=4), \
        {**cache, "q": q, "pages": ints([[0], [1]]), "lens": ints([3, 9]), "out": torch.empty_like(q), "prefix": ints([2])}
    p = torch.full((2, 3, 50), 0.02, device=DEV)
    yield lambda t: ops.ls_verify(t["target"], t["drafts"], t["accept"], t["sample"], t["tokens"], t["n"], draft=t["draft"], n_drafts=t["counts"]), \
        {"target": p, "drafts": ints([[1, 2], [3, 4]]), "accept": torch.full((2, 2), 0.5, device=DEV), "sample": torch.full((2,), 0.5, device=DEV),
         "tokens": ints([[0] * 3] * 2), "n": ints([0, 0]), "draft": p[:, :2].contiguous(), "counts": ints([2, 1])}


def test_tensors_of_another_gpu_are_refused(ops):
    for call, tensors in calls(ops):
        call(tensors)
        for which, t in tensors.items():
            with pytest.raises(ValueError, match="another GPU"):
                call({**tensors, which: Elsewhere(t)})
        call(tensors)
    ops.ls_ops_sync()


@pytest.mark.parametrize("code", CODES)
def test_two_graphs_of_one_context(code):
    """Two captured steps and one of drafted tokens share the context's workspace: replayed in any order on its stream they give what eager
    calls give."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        sets = [step_tensors(code), step_tensors(code)]
        sets[1]["qkv"].mul_(0.7)
        p = torch.softmax(rand((4, 3, 20000), 5), -1)
        q = torch.softmax(rand((4, 2, 20000), 6), -1)
        drafts, accept, sample = q.argmax(-1).to(torch.int32), torch.rand((4, 2), device=DEV), torch.rand(4, device=DEV)
        tokens, n = torch.zeros((4, 3), dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
        s.synchronize()
        o = lsffn.Ops(stream=s)
        runs = [lambda: step(o, sets[0]), lambda: step(o, sets[1]), lambda: o.ls_verify(p, drafts, accept, sample, tokens, n, draft=q)]
        outs = [lambda t=t: [t[k] for k in OUT] for t in sets] + [lambda: [tokens, n]]
        graphs, want = [], []
        for run, out in zip(runs, outs):
            run()
            s.synchronize()
            want.append([x.clone() for x in out()])
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=s):
                run()
        for i in (0, 2, 1, 1, 0, 2, 0, 1, 2):
            for x in outs[i]():
                x.zero_()
            graphs[i].replay()
            runs[(i + 1) % 3]()   # an eager call right behind it
            s.synchronize()
            assert all(same(x, y) for x, y in zip(outs[i](), want[i])), i
        o.close()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("lens,heads,kv,dim,n_q,prefix,page", [
    ([700, 3, 0, 450, 1300, 64, -1, 900, 1, 77, 640], 6, 3, 80, 1, 333, 16),     # thin, units no multiple of eight
    ([900] * 8, 16, 8, 64, 2, 0, 8), ([40, 2000, 128], 40, 5, 128, 7, 0, 64),   # thin and broad, several tokens
    ([33] * 9, 8, 4, 128, 3, 2100, 16), ([500, 20] * 20, 4, 2, 256, 1, 900, 4),   # a broad prefix beside thin sequences
    ([5000], 4, 4, 40, 16, 0, 16), ([300] * 17, 24, 8, 112, 5, 70, 32)])
def test_heads_near_each_other(ops, code, lens, heads, kv, dim, n_q, prefix, page):
    check_attend(ops, lens=lens, code=code, heads=heads, kv=kv, dim=dim, dt=torch.bfloat16, prefix=prefix, n_q=n_q, page=page, layout="token",
                 max_len=max(lens) + 5, spare=8)


@pytest.mark.parametrize("heads,n_q,dim", [(2, 1, 64), (40, 1, 128), (3, 16, 80), (20, 16, 256)])
@pytest.mark.parametrize("code", CODES)
def test_late_values_that_are_no_numbers(ops, code, heads, n_q, dim):
    """Each of the last tokens' values holds none in a group of its own: a token's row has none where the values it sees have, in its own
    and earlier ones, and nowhere else, whatever page and part those keys are in."""
    groups = -(-dim // 32)

    def touch(k, v, pages, prefix_pages):
        for s, n in ((0, 141), (2, 8)):
            for i in range(n_q):
                at = n - n_q + i
                if at >= 0:
                    v[1][pages[s, at // 8], :, at % 8, i % groups] = 255
    out = check_attend(ops, lens=[141, 60, 8], prefix=20, heads=heads, kv=1, n_q=n_q, dim=dim, page=8, touch=touch, code=code)
    bad = ~torch.isfinite(out.double()).view(3, n_q, heads, dim).all(2)
    for s, n in ((0, 141), (2, 8)):
        for i in range(n_q):
            hit = {j % groups for j in range(i + 1) if n - n_q + j >= 0}
            assert {g for g in range(groups) if bad[s, i, g * 32:g * 32 + 32].all()} == hit
            assert {g for g in range(groups) if bad[s, i, g * 32:g * 32 + 32].any()} == hit
    assert not bad[1].any()


def test_more_rows_than_a_launch():
    # 2^20 rows and some: sequences of one key each; of one weight, so the value itself.  By the header, what a split of 2^20 rows
    # takes is 2 (dim + 2) floats of each, 528 MiB: more than the default workspace, which is refused.
    S, heads, dim = 40000, 32, 64
    assert 2 ** 20 * 2 * (dim + 2) * 4 > 256 << 20
    ops = lsffn.Ops(workspace_bytes=544 << 20)
    k, v = (packed(rand((1, 2, 16, dim), i).double(), "fp4", torch.float16) for i in (1, 2))
    q = rand((S, heads, dim), 3, torch.float16)
    pages, lens = torch.zeros((S, 1), dtype=torch.int32, device=DEV), torch.ones(S, dtype=torch.int32, device=DEV)
    lens[::7] = -1
    o = torch.full_like(q, math.nan)
    ops.ls_kvq_attend(q, *k, *v, pages, lens, o, max_len=1, scale=0.1)
    one = torch.empty((1, 2, dim), dtype=torch.float16, device=DEV)
    ops.ls_kvq_read(*k, *v, ints([0]), torch.empty_like(one), one)
    want = one[0].repeat_interleave(heads // 2, 0)[None].expand(S, -1, -1) * (lens > 0)[:, None, None]
    assert same(o, want.to(torch.float16))
    ops.close()
    ops = lsffn.Ops()
    refused(lambda: ops.ls_kvq_attend(q, *k, *v, pages, lens, o, max_len=1, scale=0.1), status=lsffn.LS_E_CAPACITY)
    ops.close()

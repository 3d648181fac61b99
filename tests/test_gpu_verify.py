"""Verification of drafted tokens (ls_verify) against the definition, in 64 bits and in whole fractions."""
import math
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_03079_amd as lsffn  # noqa: E402
from test_gpu_ops import DEV, TYPES, ints, ops, refused  # noqa: E402, F401


def token_of(w, u):
    """The first index whose running sum of w exceeds u sum(w), exactly; -1 where w is zero everywhere."""
    w = [Fraction(float(x)) if x > 0 else Fraction(0) for x in w]
    total = sum(w)
    if total == 0:
        return -1
    if not u < 1:
        return max(i for i, x in enumerate(w) if x)
    want, run = Fraction(max(float(u), 0.0)) * total, Fraction(0)
    for i, x in enumerate(w):
        run += x
        if run > want:
            return i
    raise AssertionError


def reference(target, drafts, accept, sample, draft=None, counts=None):
    """Row by row in exact fractions: (tokens, n_accepted, how far each sampled number lay from a border of the running sum)."""
    target = target.double().cpu().numpy()
    draft = None if draft is None else draft.double().cpu().numpy()
    drafts, accept, sample = drafts.cpu().numpy(), accept.cpu().numpy(), sample.cpu().numpy()
    S, K1, V = target.shape
    tokens, n_accepted = np.full((S, K1), -1, np.int64), np.zeros(S, np.int64)
    for s in range(S):
        n = K1 - 1 if counts is None else min(int(counts[s]), K1 - 1)
        if n < 0:
            n_accepted[s] = -1
            continue
        r = 0
        while r < n:
            x = int(drafts[s, r])
            if not 0 <= x < V:
                break
            q = 1.0 if draft is None else float(draft[s, r, x])
            u, p = float(accept[s, r]), float(target[s, r, x])
            if not (math.isfinite(q) and math.isfinite(u) and math.isfinite(p)) or not Fraction(u) * Fraction(q) < Fraction(p):
                break
            r += 1
        p = target[s, r]
        w = p
        if r < n:
            if draft is not None:
                w = p - draft[s, r]
            else:
                w = p.copy()
                if 0 <= drafts[s, r] < V:
                    w[drafts[s, r]] -= 1.0
            if not np.any(w > 0):
                w = p
        tokens[s, :r] = drafts[s, :r]
        tokens[s, r] = token_of(w, float(sample[s]))
        n_accepted[s] = r
    return tokens, n_accepted


def case(S, K, V, dt, seed, greedy=False, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn((S, K + 1, V), generator=g) * spread
    target = torch.softmax(logits, -1).to(dt)
    q = torch.softmax(logits[:, :K] + torch.randn((S, K, V), generator=g) * 0.8, -1).to(dt)
    drafts = torch.zeros((S, K), dtype=torch.int32)
    if K:
        drafts = (q.float().argmax(-1) if greedy else torch.multinomial(q.float().reshape(S * K, V), 1, generator=g).view(S, K)).to(torch.int32)
    accept, sample = torch.rand((S, K), generator=g), torch.rand((S,), generator=g)
    return [x.to(DEV) for x in (target, drafts, accept, sample)] + [None if greedy or K == 0 else q.to(DEV)]


def run(ops, target, drafts, accept, sample, draft, counts=None):
    S, K1, _ = target.shape
    tokens = torch.full((S, K1 + 2), 77, dtype=torch.int32, device=DEV)
    n = torch.full((S,), 77, dtype=torch.int32, device=DEV)
    ops.ls_verify(target, drafts, accept, sample, tokens[:, :K1], n, draft=draft, n_drafts=None if counts is None else ints(counts))
    assert torch.all(tokens[:, K1:] == 77)
    return tokens[:, :K1].cpu().numpy(), n.cpu().numpy()


def check(ops, *args, counts=None):
    got = run(ops, *args, counts=counts)
    ref = reference(*args, counts=counts)
    assert np.array_equal(got[1], ref[1]), (got[1], ref[1])
    assert np.array_equal(got[0], ref[0]), (got[0], ref[0])
    return got


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("S,K,V", [(1, 0, 1), (1, 1, 1), (3, 2, 2), (5, 4, 7), (2, 3, 63), (2, 3, 64), (2, 3, 65), (4, 1, 1000), (3, 15, 1025),
                                   (2, 63, 333), (7, 0, 2049), (2, 4, 32000), (9, 5, 4097), (1, 7, 65537)])
def test_against_the_definition(ops, dtype, greedy, S, K, V):
    check(ops, *case(S, K, V, TYPES[dtype], S * 100 + K, greedy))


@pytest.mark.parametrize("V", [3, 100, 5000, 50001])
def test_every_number_of_accepted_tokens_and_ragged_batches(ops, V):
    S, K = 12, 5
    target, drafts, accept, sample, draft = case(S, K, V, torch.float32, V)
    accept[:] = 0.0 if V > 3 else accept
    accept[torch.arange(S), torch.arange(S).clamp(max=K - 1)] = 1e30   # sequence s is refused at draft s
    got = check(ops, target, drafts, accept, sample, draft)
    assert V == 3 or got[1].tolist()[:K] == list(range(K))
    accept[:] = 0.0
    got = check(ops, target, drafts, accept, sample, draft, counts=[0, 1, 2, 3, 4, 5, 6, 100, -1, -100, 5, 2])
    assert got[1][8] == got[1][9] == -1 and np.all(got[0][8:10] == -1)


@pytest.mark.parametrize("V", [3000, 11000])
def test_sampled_numbers_at_the_ends(ops, V):
    S = 8
    target, drafts, accept, sample, _ = case(S, 0, V, torch.float32, 3)
    target[:, :, 0], target[:, :, -1], target[:, :, 1500] = 0.0, 0.0, 0.0
    sample[:] = torch.tensor([0.0, -1.0, 1.0, 2.0, math.nan, math.inf, 1 - 2.0 ** -24, 1e-30])
    tokens, _ = check(ops, target, drafts, accept, sample, None)
    assert tokens[0, 0] == tokens[1, 0] == 1 and tokens[2, 0] == tokens[4, 0] == tokens[5, 0] == V - 2


@pytest.mark.parametrize("V", [700, 9700])
def test_weights_that_are_none(ops, V):
    target, drafts, accept, sample, draft = case(6, 2, V, torch.float32, 4)
    accept[:] = 1e30
    draft[0, 0] = target[0, 0]                     # nothing is left over: the target's own
    target[1, 0] = 0.0                             # nothing at all
    draft[2, 0] = 2.0                              # less than nothing everywhere: the target's own
    target[3, 0, 100:] = math.nan                  # no numbers do not count
    target[4, 0, 5] = -1.0
    drafts[5, 0] = V                               # outside the vocabulary: refused
    tokens, n = check(ops, target, drafts, accept, sample, draft)
    assert tokens[1, 0] == -1 and np.all(n == 0)
    drafts[5, 0] = -3
    accept[:] = 0.0
    check(ops, target, drafts, accept, sample, draft)
    check(ops, target, drafts, accept, sample, None)
    # an infinity counts as the largest number: every other weight vanishes beside it
    target[0, 0, 123] = math.inf
    accept[0] = 1e30
    assert run(ops, target, drafts, accept, sample, draft)[0][0, 0] == 123


@pytest.mark.parametrize("V", [4096, 16384])
def test_borders_are_decided_exactly(ops, V):
    # u q = p exactly is a refusal, one step less of u an acceptance; equal weights: token floor(u V), in 64 bits
    S = 64
    p = torch.full((S, 2, V), 0.25, device=DEV)
    q = torch.full((S, 1, V), 0.5, device=DEV)
    drafts, sample = torch.zeros((S, 1), dtype=torch.int32, device=DEV), torch.arange(S, device=DEV) / S
    accept = torch.full((S, 1), 0.5, device=DEV)
    accept[1::2] = 0.5 - 2.0 ** -25
    tokens, n = run(ops, p, drafts, accept, sample, q)
    assert n.tolist() == [s % 2 for s in range(S)]
    # refused: p - q is below zero everywhere, so p itself; accepted: p
    want = [s * V // S for s in range(S)]
    assert [int(tokens[s, s % 2]) for s in range(S)] == want


@pytest.mark.parametrize("V", [500, 9100])
def test_strides_and_shared_rows(ops, V):
    target, drafts, accept, sample, draft = case(4, 3, V, torch.bfloat16, 9)
    t = torch.zeros((4, 5, V + 20), dtype=torch.bfloat16, device=DEV)
    t[:, 1:, 3:V + 3] = target
    d = torch.zeros((4, 3, V + 1), dtype=torch.bfloat16, device=DEV)
    d[..., 1:] = draft
    check(ops, t[:, 1:, 3:V + 3], drafts, accept, sample, d[..., 1:])
    check(ops, target[:1].expand(4, 4, V), drafts, accept, sample, draft[:1].expand(4, 3, V))   # one row for all


@pytest.mark.parametrize("S,V", [(5, 1 << 20), (600, 9001), (300, 20000), (40, 60001)])
def test_large_vocabulary(ops, S, V):
    # against running sums in 64 bits: a number within 2^-40 of a border is not asked for
    K = 2
    target, drafts, accept, sample, draft = case(S, K, V, torch.float32, 11, spread=1.0)
    accept[:3], accept[3:] = 1e30, 0.0
    tokens, n = run(ops, target, drafts, accept, sample, draft)
    for s in range(S):
        r = int(n[s])
        w = target[s, r].double() - (draft[s, r].double() if r < K else 0.0)
        run_sum = w.clamp(min=0).cumsum(0)
        want = float(sample[s]) * float(run_sum[-1])
        i = int(torch.searchsorted(run_sum, torch.tensor(want, dtype=torch.float64, device=DEV), right=True))
        assert float((run_sum - want).abs().min()) > 2.0 ** -40 * float(run_sum[-1])
        assert tokens[s, r] == i and r == (0 if s < 3 else K)


def test_the_tokens_follow_the_targets_distribution(ops):
    """Drafts from q, then verified: the first token is distributed as p.  20000 trials of 6 tokens: within 5 standard deviations."""
    N, V = 20000, 6
    g = torch.Generator(DEV).manual_seed(1)
    p = torch.tensor([0.30, 0.05, 0.25, 0.15, 0.20, 0.05], device=DEV)
    q = torch.tensor([0.10, 0.40, 0.10, 0.15, 0.05, 0.20], device=DEV)
    drafts = torch.multinomial(q, N, replacement=True, generator=g)[:, None].to(torch.int32)
    tokens, n = torch.empty((N, 2), dtype=torch.int32, device=DEV), torch.empty(N, dtype=torch.int32, device=DEV)
    ops.ls_verify(p.expand(N, 2, V), drafts, torch.rand((N, 1), device=DEV, generator=g), torch.rand(N, device=DEV, generator=g), tokens, n,
                  draft=q.expand(N, 1, V))
    share = torch.bincount(tokens[:, 0].long(), minlength=V).double() / N
    assert torch.all((share - p.double()).abs() <= 5 * (p.double() * (1 - p.double()) / N).sqrt())
    took = float((n == 1).double().mean())
    assert abs(took - float(torch.minimum(p, q).double().sum())) <= 5 * 0.5 / math.sqrt(N)


def test_many_sequences(ops):
    N = 2 ** 18 + 3
    p = torch.rand((1, 1, 4), device=DEV).expand(N, 1, 4)
    sample = torch.rand(N, device=DEV)
    tokens, n = torch.empty((N, 1), dtype=torch.int32, device=DEV), torch.empty(N, dtype=torch.int32, device=DEV)
    none = torch.empty((N, 0), device=DEV)
    ops.ls_verify(p, none.to(torch.int32), none, sample, tokens, n)
    runs = p[0, 0].double().cumsum(0)
    assert torch.equal(tokens[:, 0].long(), (runs[None] <= sample.double()[:, None] * runs[-1]).sum(1)) and not n.any()


@pytest.mark.parametrize("V", [5000, 12000])
def test_graph_replays_read_their_arguments_anew(V):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        target, drafts, accept, sample, draft = case(6, 3, V, torch.float32, 5)
        counts = ints([3, 2, 1, 0, 3, -1])
        tokens, n = torch.zeros((6, 4), dtype=torch.int32, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
        s.synchronize()
        o = lsffn.Ops(stream=s)

        def call():
            o.ls_verify(target, drafts, accept, sample, tokens, n, draft=draft, n_drafts=counts)

        call()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call()
        for i in range(4):
            sample.copy_(torch.rand(6, generator=torch.Generator().manual_seed(i)))
            accept.copy_(torch.rand((6, 3), generator=torch.Generator().manual_seed(i + 9)))
            counts.copy_(counts.roll(1))
            s.synchronize()
            graph.replay()
            s.synchronize()
            got = tokens.clone(), n.clone()
            tokens.fill_(-9), n.fill_(-9)
            call()
            s.synchronize()
            assert torch.equal(got[0], tokens) and torch.equal(got[1], n)
            ref = reference(target, drafts, accept, sample, draft, counts.tolist())
            assert np.array_equal(tokens.cpu().numpy(), ref[0]) and np.array_equal(n.cpu().numpy(), ref[1])
        o.close()


def test_refusals(ops):
    target, drafts, accept, sample, draft = case(2, 3, 100, torch.float16, 1)
    tokens, n = torch.empty((2, 4), dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    ops.ls_verify(target, drafts, accept, sample, tokens, n, draft=draft)
    refused(lambda: ops.ls_verify(target, drafts, accept, sample, tokens[0].expand(2, 4), n, draft=draft), text="tokens_stride")
    many = torch.zeros((2, 65, 8), device=DEV)
    refused(lambda: ops.ls_verify(many, torch.zeros((2, 64), dtype=torch.int32, device=DEV), torch.zeros((2, 64), device=DEV), sample,
                                  torch.zeros((2, 65), dtype=torch.int32, device=DEV), n), text="n_drafts")
    refused(lambda: ops.ls_verify(target[..., :0], drafts, accept, sample, tokens, n), text="vocab")
    for bad in (lambda: ops.ls_verify(target, drafts, accept, sample, tokens, n, draft=draft.float()),
                lambda: ops.ls_verify(target, drafts.long(), accept, sample, tokens, n, draft=draft),
                lambda: ops.ls_verify(target, drafts, accept.half(), sample, tokens, n, draft=draft),
                lambda: ops.ls_verify(target, drafts, accept, sample[:1], tokens, n, draft=draft),
                lambda: ops.ls_verify(target, drafts, accept, sample, tokens[:, :3], n, draft=draft),
                lambda: ops.ls_verify(target, drafts, accept, sample, tokens, n.long(), draft=draft),
                lambda: ops.ls_verify(target, drafts, accept, sample, tokens, n, draft=draft[:, :2]),
                lambda: ops.ls_verify(target.transpose(1, 2), drafts, accept, sample, tokens, n),
                lambda: ops.ls_verify(target[:, 0], drafts, accept, sample, tokens, n),
                lambda: ops.ls_verify(target, drafts, accept, sample, tokens, n, n_drafts=n[:1])):
        with pytest.raises(ValueError):
            bad()
    assert lsffn.load().ls_verify(ops.ctx, None) == lsffn.LS_E_INVAL
    ops.ls_verify(target[:0], drafts[:0], accept[:0], sample[:0], tokens[:0], n[:0])   # no sequences: nothing
    ops.ls_ops_sync()

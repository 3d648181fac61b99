"""Operator calls larger than one launch: cut, and the same results."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_ops import DEV, E, TINY, TYPES, U, check_linear, ops, quantised  # noqa: E402, F401


def uniform(shape, seed, lo, hi, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV).uniform_(lo, hi, generator=torch.Generator(DEV).manual_seed(seed))


def close(got, ref, dt, roundings=4):
    """Within the roundings of fp32 that made it and the one of its type."""
    tol = (roundings + 1) * E * ref.abs() + U[dt] * ref.abs() * (1 + 8 * E) + TINY[dt]
    return bool(torch.all((got.double() - ref).abs() <= tol))


@pytest.mark.parametrize("T,k,n", [(1, 16, 2 ** 20 + 5), (7, 32, 2 ** 21 + 1), (40, 16, 2 ** 20 + 1), (70, 48, 2 ** 20 + 37),
                                   (2 ** 16 + 3, 32, 130), (2 ** 17 + 1, 16, 1)])
def test_linear_in_pieces(ops, T, k, n):
    check_linear(ops, T, k, n, "i8", "f32", bias=True, seed=n)
    check_linear(ops, T, k, n, "f16", "f16", pad=1, seed=T)


@pytest.mark.parametrize("T", [5, 16])
def test_linear_of_2_28_channels(ops, T):
    n, k = 2 ** 28 + 37, 16
    w = torch.randint(-128, 128, (n, k), dtype=torch.int8, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    x, xs = torch.randint(-128, 128, (T, k), dtype=torch.int8, device=DEV), uniform((T,), 2, 0.1, 1.0)
    ws, out = uniform((n,), 3, 0.001, 0.002), torch.empty((T, n), dtype=torch.float16, device=DEV)
    ops.ls_linear_i8(x, w, ws, out, x_scale=xs)
    for i in range(0, n, 2 ** 24):
        s = slice(i, i + 2 ** 24)
        ref = (x.double() @ w[s].double().T.contiguous()) * xs.double()[:, None] * ws[s].double()
        assert close(out[:, s], ref, torch.float16), i
    ops.ls_ops_sync()


@pytest.mark.parametrize("x_type", ["i8", "f32"])
def test_linear_of_all_channels_that_32_bits_count(ops, x_type):
    # one row of w for every channel, each with its own scale
    n, k = 2 ** 31 - 1, 16
    w = torch.randint(-128, 128, (1, k), dtype=torch.int8, device=DEV).expand(n, k)
    ws, out = uniform((n,), 3, 0.5, 1.0), torch.empty((1, n), device=DEV)
    x = torch.arange(-127, 129, 17, device=DEV)[None, :k].float()   # (the last, 128, is -128 in 8 bits)
    if x_type == "i8":
        q, s = x.to(torch.int8), torch.ones(1, device=DEV)
        ops.ls_linear_i8(q, w, ws, out, x_scale=s)
    else:
        q, s = quantised(x)
        ops.ls_linear_i8(x, w, ws, out)
    acc = float((q.double() * w[0].double()).sum()) * float(s[0])
    for i in range(0, n, 2 ** 27):
        assert close(out[0, i:i + 2 ** 27], ws[i:i + 2 ** 27].double() * acc, torch.float32), i


def test_linear_of_all_tokens_that_32_bits_count(ops):
    # one row of x for every token, each with its own scale
    T, k = 2 ** 31 - 1, 16
    x, w = (torch.randint(-128, 128, (1, k), dtype=torch.int8, device=DEV) for _ in range(2))
    xs, out = uniform((T,), 3, 0.5, 1.0), torch.empty((T, 1), device=DEV)
    ops.ls_linear_i8(x.expand(T, k), w, torch.ones(1, device=DEV), out, x_scale=xs)
    acc = float((x.double() * w.double()).sum())
    for i in range(0, T, 2 ** 27):
        assert close(out[i:i + 2 ** 27, 0], xs[i:i + 2 ** 27].double() * acc, torch.float32), i


def test_attend_of_more_sequences_than_a_launch_holds_with_no_key(ops):
    S, dim = 2 ** 25 + 3, 8
    kc, vc = (torch.ones((1, 1, 1, dim), dtype=torch.float16, device=DEV) for _ in range(2))
    q = torch.ones((1, 1, dim), dtype=torch.float16, device=DEV).expand(S, 1, dim)
    lens = torch.zeros(S, dtype=torch.int32, device=DEV)
    out = torch.full((S, 1, dim), 5.0, dtype=torch.float16, device=DEV)
    ops.ls_attend(q, kc, vc, None, lens, out, max_len=0, scale=1.0)
    assert not out.any()
    ops.ls_ops_sync()


@pytest.mark.parametrize("prefix,n_q", [(0, 1), (5, 1), (5, 2)])
def test_attend_of_millions_of_sequences(ops, prefix, n_q):
    """2^24 rows and more, sequences of up to 3 keys behind a prefix or none, against 64 bits."""
    S, kv, page, dim, most = 2 ** 21 + 5, 8, 4, 8, 3
    g = torch.Generator(DEV).manual_seed(prefix)
    kc, vc = (torch.randn((64, kv, page, dim), device=DEV, generator=g).half() for _ in range(2))
    pages = torch.randint(2, 64, (S, 1), dtype=torch.int32, device=DEV, generator=g)
    pre = torch.arange(2, dtype=torch.int32, device=DEV)
    lens = torch.randint(-1, most + 1, (S,), dtype=torch.int32, device=DEV, generator=g)
    q = torch.randn((S * n_q, kv, dim), device=DEV, generator=g).half()
    out = torch.full_like(q, 7.0)
    ops.ls_attend(q, kc, vc, pages, lens, out, max_len=most, n_q=n_q, scale=0.5, prefix_pages=pre, prefix_len=prefix)
    pk, pv = (t[:2].transpose(1, 2).flatten(0, 1)[:prefix].transpose(0, 1).double() for t in (kc, vc))   # [kv, prefix, dim]
    for s in range(0, S, 2 ** 18):
        e = min(S, s + 2 ** 18)
        at = pages[s:e, 0].long()
        k, v = (torch.cat([p.expand(e - s, -1, -1, -1), t[at, :, :most].double()], 2) for p, t in ((pk, kc), (pv, vc)))
        for i in range(n_q):
            qq = q[s * n_q + i:e * n_q:n_q].double()
            size = 0.5 * (qq.abs()[:, :, None] * k.abs()).sum(-1).amax(-1, keepdim=True)[..., None]
            sc = 0.5 * (qq[:, :, None] * k).sum(-1)
            last = torch.where(lens[s:e] < 0, -prefix - 1, lens[s:e] - n_q + i)[:, None]
            seen = torch.arange(-prefix, most, device=DEV) <= last
            seen[:, :prefix] = (lens[s:e] >= 0)[:, None]
            p = torch.exp(sc.masked_fill(~seen[:, None], -torch.inf))
            total = p.sum(-1, keepdim=True)
            p = p / torch.where(total > 0, total, 1.0)
            ref, pv_size = (p[..., None] * v).sum(2), (p[..., None] * v.abs()).sum(2)
            # weights rounded once, scores and their exponentials in fp32, the result rounded once
            tol = (2.0 ** -11 + (2 * (dim + 8) * size[..., 0] + 64) * E) * pv_size + 2.0 ** -11 * ref.abs() + 2.0 ** -24
            assert torch.all((out[s * n_q + i:e * n_q:n_q].double() - ref).abs() <= tol), (s, i)

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

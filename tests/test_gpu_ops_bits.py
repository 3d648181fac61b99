"""8-bit products: a token's row has the same bits whichever kernel computes it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_ops import DEV, TYPES, ops  # noqa: E402, F401


@pytest.mark.parametrize("out_type", list(TYPES))
@pytest.mark.parametrize("x_type", ["i8", "f32", "f16"])
@pytest.mark.parametrize("k,n", [(1040, 515), (1040, 8301), (5120, 4096), (256, 32900)])
def test_a_tokens_row_does_not_depend_on_the_tokens_beside_it(ops, out_type, x_type, k, n):
    # 1 to 4 tokens by rows, to 48 by slices, tiles of every shape, k whole and split
    g = torch.Generator(DEV).manual_seed(k + n)
    x, xs = torch.randint(-128, 128, (2100, k), dtype=torch.int8, device=DEV, generator=g), None
    if x_type == "i8":
        xs = torch.rand(2100, device=DEV, generator=g) + 0.1
    else:
        x = (x * (torch.rand((2100, 1), device=DEV, generator=g) + 0.1)).to(TYPES[x_type])
    w = torch.randint(-128, 128, (n, k), dtype=torch.int8, device=DEV, generator=g)
    ws, bias = (torch.rand(n, device=DEV, generator=g) + 0.1) * 1e-3, torch.randn(n, device=DEV, generator=g)
    for b in (bias, None):
        want = None
        for T in (2100, 300, 130, 64, 49, 40, 20, 16, 5, 4, 2, 1):
            out = torch.empty((T, n), dtype=TYPES[out_type], device=DEV)
            ops.ls_linear_i8(x[:T], w, ws, out, x_scale=None if xs is None else xs[:T], bias=b)
            want = out if want is None else want
            assert torch.equal(out, want[:T]), (T, b is None)

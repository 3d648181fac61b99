"""Codes and scales of appended keys and values by their definition, bit for bit, in every kernel of ls_kvq_append."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_kvq import CODES, decoded, empty_cache, packed, same  # noqa: E402
from test_gpu_ops import DEV, TYPES, ops, rand, rope_ref, table  # noqa: E402, F401


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,dim,rot,style,shift", [
    (200, 128, 128, 0, 0), (200, 128, 128, 1, 0), (1, 128, 128, 0, 0), (130, 80, 40, 1, 0),     # vectors
    (200, 80, 40, 0, 0), (200, 112, 56, 0, 0), (200, 24, 6, 0, 0), (200, 24, 10, 1, 0),         # element by element: few pairs
    (200, 128, 128, 0, 1), (200, 128, 128, 1, 1), (1500, 80, 40, 0, 0), (1500, 112, 56, 0, 0),  # or a row that begins anywhere
    (1500, 80, 40, 1, 0), (1500, 112, 64, 0, 0)])                                                # past the caches
def test_turned_keys_are_rounded_once_in_every_kernel(ops, code, dtype, T, dim, rot, style, shift):
    """As test_turned_keys_are_rounded_once, which has vectors and many tokens: codes and scales by the definition, bit for bit, and
    what is not turned from what it is."""
    dt, kv, page = TYPES[dtype], 8, 16
    k = torch.empty((T, kv, dim + shift), dtype=dt, device=DEV)[..., shift:]
    k.copy_(rand((T, kv, dim), 5, dt))
    some = min(T, 40)
    k[:some] = (torch.randint(-24, 25, (some, kv, dim), generator=torch.Generator().manual_seed(1)) / 4).to(dt).to(DEV)
    cs = table(70, rot)
    cs[60:], cs[62, :rot // 2], cs[63, rot // 2:] = 0.0, 1.0, -1.0   # quarter turns put ties among the numbers between codes
    at = torch.arange(T, dtype=torch.int32, device=DEV)
    positions = (at * 7 + 62) % 70
    cache = empty_cache(T // page + 1, kv, page, dim, code)
    ops.ls_kvq_append(*cache, k, k, positions, at, cs, style=style)
    ref, _ = rope_ref(k, cs[positions.long()], rot, style)
    pg, pl = at.long() // page, at.long() % page
    for c, s, x in ((*cache[:2], ref), (*cache[2:], k.double())):
        rows, scales = packed(x, code, dt)
        assert same(s[pg, :, pl], scales)
        assert same(decoded(c.view(torch.uint8)[pg, :, pl].view(c.dtype), scales, dim), decoded(rows, scales, dim))

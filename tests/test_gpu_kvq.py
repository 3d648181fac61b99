"""The cache in 4 or 8 bits (ls_kvq_append, ls_kvq_read, ls_kvq_attend) against its definition in 64 bits.

Tolerances follow from the arithmetic: E = 2^-24 is the unit roundoff of fp32, U that of the output's type."""
import ctypes
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_03079_amd as lsffn  # noqa: E402
from test_gpu_ops import BOTH, DEV, E, TINY, TYPES, U, attend_ref, ints, ops, rand, refused, rope_ref, table, within  # noqa: E402, F401

CODES = ["fp4", "fp8"]
MOST = {"fp4": 6.0, "fp8": 448.0}
BORDER = {"fp4": 7.0, "fp8": 464.0}


def most_exp(code, dt):
    """The largest exponent of a scale: the largest code times it is a number of the type."""
    return {"fp4": 13, "fp8": 7}[code] if dt == torch.float16 else {"fp4": 125, "fp8": 119}[code]


def two_to(e):
    """2^e in 64 bits, by its bits (the GPU's power function may miss by a rounding, and a tie with it)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def same(a, b):
    return bool(torch.equal(a, b))


def levels(code):
    """What the codes 0, 1, .. stand for, in 64 bits."""
    if code == "fp4":
        up = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    else:
        i = torch.arange(128)
        e, m = i // 8, (i % 8).double()
        up = torch.where(e > 0, torch.ldexp(1 + m / 8, e - 7), torch.ldexp(m / 8, torch.tensor(-6)))
        up[127] = math.nan
    return torch.cat([up, -up]).to(DEV)


def grouped(x, dim):
    n = -(-dim // 32)
    return torch.nn.functional.pad(x, (0, 32 * n - dim)).unflatten(-1, (n, 32))


def exponents(x, code, dt):
    """Exponents of the groups' scales of rows x (64 bits), [..., groups]."""
    top = grouped(x, x.shape[-1]).abs().amax(-1)
    e = torch.full(top.shape, -126, dtype=torch.int64, device=x.device)
    for k in range(-125, most_exp(code, dt) + 1):
        e += (top >= BORDER[code] * 2.0 ** (k - 1)).long()
    return e


def nearest(x, e, code):
    """Rows x (64 bits) on the numbers of their groups' scales 2^e: to nearest, ties to the even code."""
    s = two_to(e).repeat_interleave(32, -1)[..., :x.shape[-1]]
    lv = levels(code)[:8 if code == "fp4" else 127]
    y = (x / s).abs()
    hi = torch.bucketize(y.contiguous(), lv).clamp(1, len(lv) - 1)   # lv[hi - 1] < y <= lv[hi]
    lo = hi - 1
    up = (lv[hi] - y < y - lv[lo]) | ((lv[hi] - y == y - lv[lo]) & (hi % 2 == 0))
    return torch.sign(x) * lv[torch.where(up, hi, lo)] * s


def decoded(codes, scales, dim):
    """Rows of the cache in 64 bits."""
    code = "fp4" if codes.dtype == torch.uint8 else "fp8"
    c = codes.view(torch.uint8).long()
    if code == "fp4":
        c = torch.stack([c & 15, c >> 4], -1).flatten(-2)
    s = two_to(scales.long() - 127)
    s = torch.where(scales == 255, math.nan, s)
    return levels(code)[c] * s.repeat_interleave(32, -1)[..., :dim]


def packed(x, code, dt):
    """(codes, scales) of rows x (64 bits, finite), by the definition."""
    e = exponents(x, code, dt)
    s = two_to(e).repeat_interleave(32, -1)[..., :x.shape[-1]]
    v = nearest(x, e, code) / s
    lv = levels(code)[:8 if code == "fp4" else 127]
    c = torch.bucketize(v.abs().contiguous(), lv) + torch.signbit(x).long() * (8 if code == "fp4" else 128)
    if code == "fp4":
        return (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8), (e + 127).to(torch.uint8)
    return c.to(torch.uint8).view(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def in_pages(x, layout, spare=0):
    """[pages, kv, page, n] of the same values with heads or tokens outermost within a page, rows `spare` elements apart."""
    x8 = x.view(torch.uint8)
    shape = list(x8.shape) if layout == "head" else [x8.shape[0], x8.shape[2], x8.shape[1], x8.shape[3]]
    out = torch.full((*shape[:3], shape[3] + spare), 0xAB, dtype=torch.uint8, device=DEV)[..., :shape[3]]
    out = out if layout == "head" else out.transpose(1, 2)
    out.copy_(x8)
    return out.view(x.dtype) if x.dtype != torch.uint8 else out


def empty_cache(pages, kv, page, dim, code, layout="head", spare=0):
    """k codes, k scales, v codes, v scales, filled with what no call writes by chance."""
    def one(n, dt, more):
        return in_pages(torch.full((pages, kv, page, n), 0x5A, dtype=torch.uint8, device=DEV).view(dt), layout, more)
    n, dt = (dim // 2, torch.uint8) if code == "fp4" else (dim, torch.float8_e4m3fn)
    return [one(n, dt, spare), one(-(-dim // 32), torch.uint8, spare // 4), one(n, dt, spare), one(-(-dim // 32), torch.uint8, spare // 4)]


def raw(cache):
    return [x.view(torch.uint8).clone() for x in cache]


# ---- append ----------------------------------------------------------------------------------------
def check_rows(codes, scales, x, tol, code, dt):
    """Quantised rows against rows x (64 bits) known to `tol`: the scale of a number within it, and each code that of one."""
    dim = x.shape[-1]
    e = scales.long() - 127
    low = exponents((x.abs() - tol).clamp(min=0), code, dt)
    high = exponents(x.abs() + tol, code, dt)
    assert torch.all((low <= e) & (e <= high))
    got = decoded(codes, scales, dim)
    assert torch.all((nearest(x - tol, e, code) <= got) & (got <= nearest(x + tol, e, code)))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,heads,kv,dim,rot,style,page,layout,in_place", [
    (1, 32, 32, 128, 128, 0, 16, "head", False), (1, 8, 1, 256, 256, 0, 64, "token", True), (37, 10, 5, 80, 40, 1, 16, "token", False),
    (37, 10, 5, 80, 40, 0, 16, "head", True), (9, 4, 2, 8, 6, 0, 1, "head", True), (9, 4, 2, 24, 10, 1, 2, "token", True),
    (130, 6, 3, 112, 56, 0, 128, "head", False), (130, 6, 3, 112, 112, 1, 8, "token", True), (5, 0, 3, 64, 64, 0, 4, "head", False),
    (300, 3, 1, 40, 0, 0, 4096, "head", False), (700, 2, 2, 64, 32, 1, 32, "head", True), (3, 5, 5, 1024, 1024, 0, 2, "head", True)])
def test_append(ops, code, dtype, T, heads, kv, dim, rot, style, page, layout, in_place):
    dt = TYPES[dtype]
    pages = T // page + 3
    cache = empty_cache(pages, kv, page, dim, code, layout, spare=8)
    qkv = rand((T, (heads + 2 * kv) * dim), 3, dt)
    q, k, v = (x.view(T, -1, dim) for x in qkv.split([heads * dim, kv * dim, kv * dim], 1))
    g = torch.Generator().manual_seed(T)
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    positions = torch.randint(0, 50, (T,), generator=g).to(torch.int32)
    if T > 4:  # padding, a slot past the cache, positions outside the table
        slots[1], slots[2], positions[3], positions[4] = -1, pages * page, -1, 50
    cs = table(50, rot) if rot else None
    q0, before = qkv.clone(), raw(cache)
    q_out = None if heads == 0 else q if in_place else torch.full((T, heads, dim), 7.0, device=DEV, dtype=dt)
    q_before = None if heads == 0 else q_out.clone()
    ops.ls_kvq_append(*cache, k, v, positions.to(DEV) if rot else None, slots.to(DEV), cs, q=q if heads else None, q_out=q_out, style=style)
    placed = torch.tensor([rot == 0 or 0 <= int(p) < 50 for p in positions])
    kept = (placed & (slots >= 0) & (slots < pages * page))
    at = cs[positions.clamp(0, 49).long().to(DEV)] if rot else torch.zeros((T, 0), device=DEV)
    src = [x.view(T, -1, dim) for x in q0.split([heads * dim, kv * dim, kv * dim], 1)]
    sl = slots[kept].long().to(DEV)
    pg, pl, kept = sl // page, sl % page, kept.to(DEV)
    rk, mk = rope_ref(src[1], at, rot, style)
    # two products and a sum in fp32
    check_rows(cache[0].view(torch.uint8)[pg, :, pl].view(cache[0].dtype), cache[1][pg, :, pl], rk[kept], 3 * E * mk[kept], code, dt)
    rows, scales = packed(src[2][kept].double(), code, dt)
    got = cache[2].view(torch.uint8)[pg, :, pl]
    # a negative number that rounds to zero keeps its sign here, which a value does not show
    assert same(decoded(got.view(cache[2].dtype), cache[3][pg, :, pl], dim), decoded(rows, scales, dim))
    assert same(cache[3][pg, :, pl], scales)
    after = raw(cache)
    for x, y in zip(before, after):  # nothing else was written
        y[pg, :, pl] = x[pg, :, pl]
        assert same(x, y)
    if heads:
        rq, mq = rope_ref(src[0], at, rot, style)
        placed = placed.to(DEV)
        within(q_out[placed], rq[placed], 4 * E * mq[placed] + U[dt] * rq[placed].abs() * (1 + 8 * E) + TINY[dt])
        assert same(q_out[~placed], q_before[~placed])


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_append_at_the_borders(ops, code, dtype):
    """Every code, every tie between two, largest magnitudes at the border between two scales and one number either side of it, zeros,
    the type's smallest and largest numbers, by the definition, bit for bit; groups that hold no numbers."""
    dt = TYPES[dtype]
    lv = levels(code)[:8 if code == "fp4" else 127].cpu()
    ties = (lv[1:] + lv[:-1]) / 2
    points = torch.cat([lv, ties, ties * (1 + 2.0 ** -6), ties * (1 - 2.0 ** -6)])
    rows = []
    for start in range(0, len(points), 31):   # a group each, whose scale is one
        x = torch.zeros(32, dtype=torch.float64)
        some = points[start:start + 31]
        x[:len(some)] = some * torch.tensor([1, -1]).repeat(16)[:len(some)]
        x[31] = MOST[code]
        rows += [x, -x * 2.0 ** -7]
    step = torch.finfo(dt).eps
    for b in (BORDER[code], BORDER[code] * 2.0 ** -9):
        for y in (b, b * (1 - step / 2), b * (1 + step)):
            x = torch.linspace(-1, 1, 32, dtype=torch.float64) * b
            x[7] = y
            rows.append(x)
    big, tiny = torch.finfo(dt).max, torch.finfo(dt).tiny
    for top in (big, big / 1.1, big / 1.5, big / 2, tiny, tiny * 64, tiny * 2.0 ** -5, 0.0):
        rows.append(torch.linspace(-1, 1, 32, dtype=torch.float64) * top)
    x = torch.stack(rows).to(dt)
    x = x[: len(rows) // 4 * 4].view(-1, 2, 64).to(DEV)
    T = x.shape[0]
    cache = empty_cache(T // 16 + 1, 2, 16, 64, code)
    ops.ls_kvq_append(*cache, x, x, None, torch.arange(T, dtype=torch.int32, device=DEV), None)
    rows, scales = packed(x.double(), code, dt)
    at = torch.arange(T, device=DEV)
    for i in (0, 2):
        got, sc = cache[i].view(torch.uint8)[at // 16, :, at % 16].view(cache[i].dtype), cache[i + 1][at // 16, :, at % 16]
        assert same(sc, scales)
        assert same(decoded(got, sc, 64), decoded(rows, scales, 64))
    # one infinity or NaN: its group alone
    y = rand((3, 2, 64), 5, dt)
    y[0, 0, 3], y[1, 1, 40], y[2, 0, 63] = math.nan, math.inf, -math.inf
    ops.ls_kvq_append(*cache, y, y, None, ints([0, 1, 2]), None)
    out = [torch.zeros_like(y) for _ in range(2)]
    ops.ls_kvq_read(*cache, ints([0, 1, 2]), *out)
    bad = torch.zeros((3, 2, 2), dtype=torch.bool, device=DEV)
    bad[0, 0, 0] = bad[1, 1, 1] = bad[2, 0, 1] = True
    for o, s in zip(out, (cache[1], cache[3])):
        assert same(torch.isnan(o), bad.repeat_interleave(32, -1)) and same(s[0, :, :3].transpose(0, 1) == 255, bad)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("style", [0, 1])
def test_turned_keys_are_rounded_once(ops, code, dtype, style):
    """Codes and scales of turned keys by the definition from the angle's product in 64 bits, whose products of fp32 numbers are exact;
    quarter turns of numbers between two codes put exact ties among them."""
    dt, T, kv, dim, page = TYPES[dtype], 3001, 8, 128, 16
    k = rand((T, kv, dim), 5, dt)
    k[:64] = (torch.randint(-24, 25, (64, kv, dim), generator=torch.Generator().manual_seed(1)) / 4).to(dt).to(DEV)
    cs = table(70, dim)
    cs[60:], cs[62, :64], cs[63, 64:] = 0.0, 1.0, -1.0
    at = torch.arange(T, dtype=torch.int32, device=DEV)
    positions = at % 70
    cache = empty_cache(T // page + 1, kv, page, dim, code)
    ops.ls_kvq_append(*cache, k, k, positions, at, cs, style=style)
    ref, _ = rope_ref(k, cs[positions.long()], dim, style)
    rows, scales = packed(ref, code, dt)
    pg, pl = at.long() // page, at.long() % page
    assert same(cache[1][pg, :, pl], scales)
    assert same(decoded(cache[0].view(torch.uint8)[pg, :, pl].view(cache[0].dtype), scales, dim), decoded(rows, scales, dim))


def test_append_keeps_turned_keys_that_overflow_apart(ops):
    # keys near the end of float16 that grow beyond it when they turn are held as the largest number of their group's largest scale
    k = torch.full((1, 1, 64), 65504.0, dtype=torch.float16, device=DEV)
    cs = torch.full((1, 64), math.sqrt(0.5), device=DEV)   # (a c - b s, b c + a s) = (0, 92637)
    for code in CODES:
        cache = empty_cache(1, 1, 1, 64, code)
        ops.ls_kvq_append(*cache, k, k, ints([0]), ints([0]), cs)
        got = decoded(cache[0], cache[1], 64)[0, 0, 0]
        # the difference of two products in fp32: what one of them was rounded by, E * 46319, held to within an eighth
        assert torch.all(got[:32].abs() <= 2 * E * 46320) and torch.all(got[32:] == MOST[code] * 2.0 ** most_exp(code, torch.float16))


# ---- read ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kv,dim,page,layout,pad", [(2, 64, 16, "head", 0), (3, 80, 8, "token", 0), (1, 8, 1, "head", 3), (5, 1024, 4, "token", 8),
                                                    (40, 112, 32, "head", 1), (8, 256, 128, "token", 0)])
def test_read(ops, code, dtype, kv, dim, page, layout, pad):
    """Every code under many scales, exactly where the type holds the value; slots in any order, twice, outside the cache."""
    dt = TYPES[dtype]
    pages = 40 // page + 2
    cache = empty_cache(pages, kv, page, dim, code, layout)
    g = torch.Generator().manual_seed(dim)
    for i, x in enumerate(cache):
        u = x.view(torch.uint8)
        u.copy_(torch.randint(0, 256, u.shape, generator=g).to(torch.uint8) if i % 2 == 0 else torch.randint(1, 256, u.shape, generator=g).to(torch.uint8))
        if i % 2:
            near = torch.rand(u.shape, generator=g).to(DEV) < 0.7   # most of them in every type's range
            u[near] = u[near] % 32 + 110
    slots = torch.randint(0, pages * page, (40,), generator=g).to(torch.int32)
    slots[3], slots[11], slots[12], slots[7] = -1, pages * page, 2 ** 31 - 1, slots[8]
    out = [torch.full((40, kv, dim + pad), 9.0, dtype=dt, device=DEV)[..., :dim] for _ in range(2)]
    ops.ls_kvq_read(*cache, slots.to(DEV), *out)
    there = ((slots >= 0) & (slots < pages * page)).to(DEV)
    at = slots.clamp(0, pages * page - 1).long().to(DEV)
    for i, o in ((0, out[0]), (2, out[1])):
        ref = decoded(cache[i].view(torch.uint8)[at // page, :, at % page].view(cache[i].dtype), cache[i + 1][at // page, :, at % page], dim)
        ref = ref.float().to(dt)   # exact in fp32, then one rounding
        ref[~there] = 9.0
        assert same(torch.isnan(o), torch.isnan(ref))
        assert same(o.nan_to_num(0, 1e30, -1e30), ref.nan_to_num(0, 1e30, -1e30))


def test_offsets_past_32_bits(ops):
    # pages of 64 KiB, 70000 of them: the last ones lie over 4 GiB from the start of the codes
    pages, kv, page, dim = 70000, 8, 128, 128
    cache = [torch.empty((pages, kv, page, n), dtype=torch.uint8, device=DEV) for n in (64, 4, 64, 4)]
    k, v = rand((3, kv, dim), 1, torch.float16), rand((3, kv, dim), 2, torch.float16)
    slots = ints([pages * page - 1, 66000 * page + 5, 3])
    ops.ls_kvq_append(*cache, k, v, None, slots, None)
    out = [torch.empty_like(k) for _ in range(2)]
    ops.ls_kvq_read(*cache, slots, *out)
    for x, o, i in ((k, out[0], 0), (v, out[1], 2)):
        rows, scales = packed(x.double(), "fp4", torch.float16)
        assert same(o.double(), decoded(rows, scales, dim))
        for j, s in enumerate(slots.tolist()):
            assert same(cache[i + 1][s // page, :, s % page], scales[j])
    q = rand((1, 16, dim), 3, torch.float16)
    o, small = torch.empty_like(q), torch.empty_like(q)
    last = [packed(rand((kv, page, dim), 4 + i, torch.float16).double(), "fp4", torch.float16) for i in range(2)]
    for i, (c, s) in enumerate(last):
        cache[2 * i][pages - 1], cache[2 * i + 1][pages - 1] = c, s
    ops.ls_kvq_attend(q, *cache, ints([[pages - 1]]), ints([page]), o, max_len=page, scale=0.1)
    ops.ls_kvq_attend(q, *[x[pages - 1:].clone() for x in cache], ints([[0]]), ints([page]), small, max_len=page, scale=0.1)
    assert same(o, small) and torch.any(o != 0)


def test_tokens_of_more_than_one_launch(ops):
    T, dim = 2 ** 21 + 3, 8
    cache = empty_cache(T // 4096 + 1, 1, 4096, dim, "fp8")
    x = rand((T, 1, dim), 1, torch.bfloat16)
    at = torch.arange(T, dtype=torch.int32, device=DEV)
    slots = T - 1 - at
    ops.ls_kvq_append(*cache, x, x, None, slots, None)
    out = [torch.zeros_like(x) for _ in range(2)]
    ops.ls_kvq_read(*cache, slots, *out)
    rows, scales = packed(x.double(), "fp8", torch.bfloat16)
    ref = decoded(rows, scales, dim)
    assert same(out[0].double(), ref) and same(out[1].double(), ref)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("heads,kv,dim,rot,style,in_place", [(37, 3, 80, 64, 0, True), (37, 3, 80, 40, 1, False), (0, 21, 128, 128, 0, False),
                                                             (64, 8, 64, 0, 0, False), (5, 33, 72, 32, 0, True)])
def test_calls_of_many_bytes_equal_those_of_few(ops, code, dtype, heads, kv, dim, rot, style, in_place):
    """Calls that pass the caches by (more than 4 MiB of data) write what the same tokens give at most 190 at a time."""
    dt, page = TYPES[dtype], 16
    T = (36 << 20) // (dim * (heads + 2 * kv) * dt.itemsize) + 3
    assert 190 * dim * (heads + 2 * kv) * dt.itemsize <= 4 << 20
    qkv = rand((T, (heads + 2 * kv) * dim), 3, dt)
    g = torch.Generator().manual_seed(T)
    pages = T // page + 3
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    positions = torch.randint(0, 50, (T,), generator=g).to(torch.int32)
    slots[1], slots[T - 1], positions[3], positions[700] = -1, pages * page, -1, 50
    slots, positions, cs = slots.to(DEV), positions.to(DEV), table(50, rot) if rot else None

    def run(step):
        cache, data = empty_cache(pages, kv, page, dim, code), qkv.clone()
        q, k, v = (x.view(T, -1, dim) for x in data.split([heads * dim, kv * dim, kv * dim], 1))
        o = None if not heads else q if in_place else torch.full((T, heads, dim), 7.0, device=DEV, dtype=dt)
        for t in range(0, T, step):
            c = slice(t, t + step)
            ops.ls_kvq_append(*cache, k[c], v[c], positions[c] if rot else None, slots[c], cs, q=q[c] if heads else None,
                              q_out=o[c] if heads else None, style=style)
        return cache, o

    (large, q_large), (small, q_small) = run(T), run(190)
    for x, y in zip(raw(large), raw(small)):
        assert same(x, y)
    if heads:
        assert same(q_large, q_small)
    # read, the slots twice over so that there is enough of it
    n = (36 << 20) // (2 * kv * dim * dt.itemsize) + 1
    at = slots.repeat(n // T + 1)[:n].contiguous()
    outs = []
    for step in (n, 190):
        out = [torch.full((n, kv, dim), 9.0, dtype=dt, device=DEV) for _ in range(2)]
        for t in range(0, n, step):
            ops.ls_kvq_read(*large, at[t:t + step], out[0][t:t + step], out[1][t:t + step])
        outs.append(out)
    for x, y in zip(*outs):
        assert same(x, y)   # the rows written are finite


# ---- attention -------------------------------------------------------------------------------------
def check_attend(ops, *, lens, code="fp4", heads=4, kv=2, dim=64, dt=torch.float16, prefix=0, n_q=1, page=16, layout="head", max_len=None,
                 bad_pages=False, seed=0, std=1.0, poison=True, stride_pad=0, spare=0, touch=None, key_std=1.0):
    S = len(lens)
    most = max([0, *lens])
    max_len = most if max_len is None else max_len
    n, pre = -(-max_len // page), -(-prefix // page)
    total = pre + n * S + 2
    shape = (total, kv, page, dim)
    k, v = (packed((rand(shape, seed + i) * (key_std if i == 0 else 1.0)).double(), code, dt) for i in (0, 1))
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(total, generator=g).to(torch.int32)
    prefix_pages, pages = order[:pre].clone(), order[pre:pre + n * S].view(S, n).clone()
    if bad_pages:
        if n > 1:
            pages[0, 0], pages[S - 1, n // 2] = -1, total
        if pre > 2:
            prefix_pages[1], prefix_pages[pre - 1] = -5, 2 ** 31 - 1
    if poison:  # whatever no row may see is no number
        seen = torch.zeros((total, page), dtype=torch.bool)
        for row, m in [(prefix_pages, prefix)] + [(pages[s], min(max(0, lens[s]), max_len)) for s in range(S)]:
            for j in range(m):
                if 0 <= row[j // page] < total:
                    seen[row[j // page], j % page] = True
        hide = (~seen)[:, None, :, None].to(DEV)
        for x in (k, v):
            x[0].view(torch.uint8).masked_fill_(hide, 0x7F)
            x[1].masked_fill_(hide, 255)
    if touch:
        touch(k, v, pages, prefix_pages)
    cache = [in_pages(x, layout, spare * (8 if i % 2 == 0 else 1)) for i, x in enumerate((*k, *v))]
    kd, vd = decoded(*k, dim), decoded(*v, dim)
    q = rand((S * n_q, heads + stride_pad, dim), seed + 7, dt, std)[:, :heads]
    out = torch.full((S * n_q, heads + stride_pad, dim), 5.0, device=DEV, dtype=dt)
    scale = 1 / math.sqrt(dim)
    wide = torch.full((S, n + spare), 2 ** 30, dtype=torch.int32)
    wide[:, :n] = pages
    args = dict(n_q=n_q, max_len=max_len, prefix_pages=prefix_pages.to(DEV), prefix_len=prefix, scale=scale)
    ops.ls_kvq_attend(q, *cache, wide.to(DEV), ints(lens), out[:, :heads], **args)
    ref, tol = attend_ref(q, kd, vd, pages, lens, n_q, max_len, prefix_pages, prefix, scale)
    within(out[:, :heads], ref, tol)
    assert stride_pad == 0 or torch.all(out[:, heads:] == 5.0)
    again = torch.empty_like(out)[:, :heads]
    ops.ls_kvq_attend(q, *cache, wide.to(DEV), ints(lens), again, **args)
    assert same(out[:, :heads].nan_to_num(9), again.nan_to_num(9))  # the same bits
    return out[:, :heads]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dt", BOTH, ids=["f16", "bf16"])
@pytest.mark.parametrize("length", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1300])
def test_attend_lengths(ops, code, dt, length):
    check_attend(ops, lens=[length], code=code, dt=dt, seed=length)
    check_attend(ops, lens=[length, 3, 0, length // 2], prefix=length, code=code, dt=dt, seed=length + 1)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 112, 128, 136, 160, 192, 248, 256])
@pytest.mark.parametrize("prefix,lens,heads,kv", [(0, [70], 3, 3), (77, [5, 200], 8, 2), (150, [40, 1, 90], 40, 1)])
def test_attend_head_sizes(ops, code, dim, prefix, lens, heads, kv):
    for dt in BOTH:
        check_attend(ops, lens=lens, prefix=prefix, heads=heads, kv=kv, dim=dim, code=code, dt=dt, seed=dim)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("page", [1, 2, 8, 16, 32, 64, 128, 1024])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_attend_pages(ops, code, page, layout):
    check_attend(ops, lens=[300, 17], prefix=131, page=page, layout=layout, spare=3, code=code, seed=page)
    check_attend(ops, lens=[300, 17, 64, 65, 128, 2, 9, 40, 77], prefix=131, heads=16, page=page, layout=layout, bad_pages=True, code=code,
                 dim=128, seed=page)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("n_q", [1, 2, 3, 5, 8, 16])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (8, 2), (12, 2), (32, 1)])
def test_attend_query_tokens(ops, code, n_q, heads, kv):
    # lengths shorter than n_q leave rows that see nothing, or the prefix alone
    lens = [n_q, 90, n_q - 1, 0, -1, 1, 64, 65]
    check_attend(ops, lens=lens, prefix=0, heads=heads, kv=kv, n_q=n_q, code=code, dt=torch.bfloat16, seed=n_q)
    check_attend(ops, lens=lens, prefix=45, heads=heads, kv=kv, n_q=n_q, code=code, seed=n_q + 1)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("rows", [1, 31, 32, 33, 64, 127, 128, 129, 260])
def test_attend_row_tiles(ops, code, rows):
    check_attend(ops, lens=[(7 * s) % 40 for s in range(rows)], prefix=200, heads=2, kv=2, dim=32, code=code, dt=torch.bfloat16, seed=rows)


@pytest.mark.parametrize("code", CODES)
def test_attend_nothing_to_see(ops, code):
    out = check_attend(ops, lens=[0, -1, -7], prefix=0, max_len=40, code=code)
    assert torch.all(out == 0)
    out = check_attend(ops, lens=[0, -1, 0], prefix=0, max_len=0, code=code)
    assert torch.all(out == 0)
    out = check_attend(ops, lens=[-1, 4, -1], prefix=100, code=code)
    assert torch.all(out[[0, 2]] == 0) and torch.any(out[1] != 0)
    out = check_attend(ops, lens=[0, -1], prefix=100, max_len=0, code=code)  # the prefix alone
    assert torch.any(out[0] != 0) and torch.all(out[1] == 0)

    def all_bad(k, v, pages, prefix_pages):
        pages.fill_(-1)
        prefix_pages.fill_(10 ** 6)
    out = check_attend(ops, lens=[30, 60], prefix=70, touch=all_bad, poison=False, code=code)
    assert torch.all(out == 0)
    check_attend(ops, lens=[500, 20], max_len=100, prefix=10, poison=False, code=code)
    check_attend(ops, lens=[2 ** 31 - 1, 3], max_len=64, poison=False, code=code)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,n_q", [(2, 4), (2, 16), (24, 5)])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_attend_a_later_tokens_value_stays_out(ops, code, heads, n_q, dim):
    # the last token's first group of values holds no numbers: the tokens before it must not see it, it must itself
    def touch(k, v, pages, prefix_pages):
        v[1][pages[0, 69 // 16], :, 69 % 16, 0] = 255
    out = check_attend(ops, lens=[70, 30], prefix=50, heads=heads, kv=1, n_q=n_q, dim=dim, touch=touch, code=code)
    finite = torch.isfinite(out)
    assert torch.all(finite[:n_q - 1]) and not torch.any(finite[n_q - 1, :, :32]) and torch.all(finite[n_q - 1, :, 32:])
    assert torch.all(finite[n_q:])


@pytest.mark.parametrize("code", CODES)
def test_attend_no_numbers_in_sight(ops, code):
    def touch(k, v, pages, prefix_pages):
        k[1][pages[0, 0], 0, 1, 1] = 255   # a key of sequence 0, head 0 of 2: its rows alone
    out = check_attend(ops, lens=[40, 40], touch=touch, code=code)
    assert torch.all(torch.isnan(out[0, :2])) and torch.all(torch.isfinite(out[0, 2:])) and torch.all(torch.isfinite(out[1]))
    check_attend(ops, lens=[200, 33], prefix=100, key_std=60.0, dt=torch.bfloat16, std=30.0, poison=False, code=code)  # weights of 0 and 1
    check_attend(ops, lens=[200, 33], prefix=100, key_std=60.0, dt=torch.float16, std=30.0, poison=False, code=code, heads=64, dim=128)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dim", [40, 64, 80, 128, 136, 192, 256])
@pytest.mark.parametrize("n_q", [1, 3, 4])
def test_attend_wide_prefix_beside_narrow_sequences(ops, code, dim, n_q):
    # more than 32 rows share the prefix, at most 32 a sequence
    for dt in BOTH:
        check_attend(ops, lens=[0, 1, 33, 300, -1, 64, 517], prefix=333, heads=8, kv=1, n_q=n_q, dim=dim, code=code, dt=dt, page=16,
                     seed=dim + n_q)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dim", [64, 80, 136, 256])
def test_attend_many_parts(ops, code, dim):
    check_attend(ops, lens=[7000, 20], prefix=9000, heads=4, kv=1, dim=dim, page=64, code=code, seed=dim, poison=False)
    check_attend(ops, lens=[2000] * 5, prefix=9000, heads=8, kv=1, n_q=2, dim=dim, page=64, code=code, seed=dim, poison=False)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("lens,prefix,heads,kv,n_q", [([3000] * 2, 9000, 8, 8, 1), ([200 * s for s in range(20)], 5000, 32, 4, 2),
                                                      ([1000] * 6, 700, 64, 2, 2)])
def test_attend_longer(ops, code, lens, prefix, heads, kv, n_q):
    check_attend(ops, lens=lens, prefix=prefix, heads=heads, kv=kv, n_q=n_q, dim=128, code=code, dt=torch.bfloat16, page=64, poison=False,
                 layout="token", stride_pad=3)


def test_attend_small_workspace():
    o = lsffn.Ops(workspace_bytes=1 << 20)
    check_attend(o, lens=[4000] * 8, prefix=6000, heads=32, kv=32, dim=128, page=64, poison=False)
    q = torch.zeros((64, 64, 128), dtype=torch.float16, device=DEV)
    cache = empty_cache(4, 64, 16, 128, "fp4")
    refused(lambda: o.ls_kvq_attend(q, *cache, ints([[0]] * 64), ints([4] * 64), torch.empty_like(q), max_len=4, scale=1.0,
                                    prefix_pages=ints([1]), prefix_len=3), status=lsffn.LS_E_CAPACITY)
    o.close()


def test_attend_of_millions_of_sequences(ops):
    S, dim = 2 ** 20 + 5, 8
    cache = [x.clone() for x in packed(rand((64, 1, 4, dim), 1).double(), "fp4", torch.float16) for _ in (0, 1)]
    cache = [cache[0], cache[2], cache[1], cache[3]]
    g = torch.Generator(DEV).manual_seed(3)
    pages = torch.randint(0, 64, (S, 1), dtype=torch.int32, device=DEV, generator=g)
    q = rand((S, 1, dim), 2, torch.float16)
    out = torch.full_like(q, 7.0)
    # one key: its value, whatever the query (the weight is one)
    ops.ls_kvq_attend(q, *cache, pages, torch.ones(S, dtype=torch.int32, device=DEV), out, max_len=3, scale=0.5)
    assert same(out[:, 0].double(), decoded(cache[2], cache[3], dim)[pages[:, 0].long(), 0, 0])


# ---- streams, graphs, refusals ---------------------------------------------------------------------
def step(o, t):
    """A step's calls on a quantised cache, in their order."""
    q, k, v = (a.view(8, -1, 64) for a in t["qkv"].split([512, 128, 128], 1))
    o.ls_kvq_append(*t["cache"], k, v, t["positions"], t["slots"], t["table"], q=q, q_out=t["q"])
    o.ls_kvq_attend(t["q"], *t["cache"], t["pages"], t["lens"], t["o"], n_q=2, max_len=64, prefix_pages=t["prefix"], prefix_len=40, scale=0.125)
    o.ls_kvq_read(*t["cache"], t["slots"], t["k"], t["v"])


def step_tensors(code):
    k, v = (packed(rand((24, 2, 16, 64), i).double(), code, torch.bfloat16) for i in (1, 2))
    at = torch.tensor([0, 1, 64 + 4, 64 + 5, 128 + 16, 128 + 17, 192 + 28, 192 + 29], dtype=torch.int32, device=DEV)
    return {"qkv": rand((8, 768), 3, torch.bfloat16), "q": torch.empty((8, 8, 64), dtype=torch.bfloat16, device=DEV),
            "o": torch.empty((8, 8, 64), dtype=torch.bfloat16, device=DEV), "table": table(200, 64), "prefix": ints([20, 21, 22]),
            "pages": torch.arange(16, dtype=torch.int32, device=DEV).view(4, 4), "lens": ints([2, 6, 18, 30]), "slots": at,
            "positions": at % 64 + 40, "cache": [x.clone() for x in (*k, *v)],
            "k": torch.zeros((8, 2, 64), dtype=torch.bfloat16, device=DEV), "v": torch.zeros((8, 2, 64), dtype=torch.bfloat16, device=DEV)}


OUT = ("q", "o", "k", "v")


@pytest.mark.parametrize("code", CODES)
def test_graph_replays_read_their_arguments_anew(code):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        t = step_tensors(code)
        s.synchronize()
        o = lsffn.Ops(stream=s)
        step(o, t)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(o, t)
        for _ in range(4):
            for n in ("lens", "positions", "slots"):
                t[n].add_(1)
            t["qkv"].mul_(1.1)
            graph.replay()
            s.synchronize()
            got = {n: t[n].clone() for n in OUT}
            for n in OUT:
                t[n].fill_(math.nan)
            step(o, t)  # eager, on the same state: the same bits
            s.synchronize()
            for n in OUT:
                assert same(got[n], t[n]) and torch.all(torch.isfinite(got[n])), n
        o.close()


def test_another_stream_gives_the_same_bits(ops):
    t = step_tensors("fp4")
    step(ops, t)
    ops.ls_ops_sync()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o = lsffn.Ops(stream=s)
    u = step_tensors("fp4")
    torch.cuda.synchronize()
    step(o, u)
    o.ls_ops_sync()
    for n in OUT:
        assert same(t[n], u[n])
    o.close()


@pytest.mark.parametrize("code", CODES)
def test_step_reads_what_it_wrote(ops, code):
    """Append, attention and read of one step against 64 bits."""
    t = step_tensors(code)
    before = [x.clone() for x in t["cache"]]
    step(ops, t)
    q, k, v = (a.view(8, -1, 64) for a in t["qkv"].split([512, 128, 128], 1))
    at, sl = t["table"][t["positions"].long()], t["slots"].long()
    rk, mk = rope_ref(k, at, 64, lsffn.LS_ROPE_HALF)
    codes, scales = (t["cache"][i].view(torch.uint8)[sl // 16, :, sl % 16] for i in (0, 1))
    check_rows(codes.view(before[0].dtype), scales, rk, 3 * E * mk, code, torch.bfloat16)
    kd, vd = decoded(*t["cache"][:2], 64), decoded(*t["cache"][2:], 64)
    assert same(t["k"].double(), kd[sl // 16, :, sl % 16]) and same(t["v"].double(), vd[sl // 16, :, sl % 16])
    ref, tol = attend_ref(t["q"], kd, vd, t["pages"].cpu(), t["lens"].tolist(), 2, 64, t["prefix"].cpu(), 40, 0.125)
    within(t["o"], ref, tol)


def test_refusals(ops):
    k, cs, one = rand((2, 2, 64), 1, torch.float16), table(8, 64), ints([0, 1])
    cache = empty_cache(4, 2, 16, 64, "fp4")
    ops.ls_kvq_append(*cache, k, k, one, one, cs)
    refused(lambda: ops.ls_kvq_append(*cache, k, k, None, one, cs), text="positions")
    refused(lambda: ops.ls_kvq_append(*cache, k, k, one, one, cs, q=k), text="q_out")
    refused(lambda: ops.ls_kvq_append(*cache, k, k, one, one, cs, style=2), text="style")
    refused(lambda: ops.ls_kvq_append(*empty_cache(4, 2, 12, 64, "fp4"), k, k, one, one, cs), text="power of two")
    odd = rand((2, 2, 60), 1, torch.float16)
    refused(lambda: ops.ls_kvq_append(*empty_cache(4, 2, 16, 60, "fp4"), odd, odd, None, one, None), text="multiple of 8")
    base = torch.zeros(4 * 2 * 16 * 32 + 8, dtype=torch.uint8, device=DEV)
    crooked = base[2:2 + 4 * 2 * 16 * 32].view(4, 2, 16, 32)
    refused(lambda: ops.ls_kvq_append(crooked, cache[1], crooked, cache[3], k, k, one, one, cs), text="multiples of 4 bytes")
    for bad in (lambda: ops.ls_kvq_append(cache[0].view(torch.int8), *cache[1:], k, k, one, one, cs),
                lambda: ops.ls_kvq_append(cache[0], cache[1][..., :1], *cache[2:], k, k, one, one, cs),
                lambda: ops.ls_kvq_append(*cache, k, k.float(), one, one, cs),
                lambda: ops.ls_kvq_append(*cache[:3], cache[3].to(torch.int32), k, k, one, one, cs),
                lambda: ops.ls_kvq_append(cache[0], cache[1], cache[2].transpose(1, 2).contiguous().transpose(1, 2), cache[3], k, k, one, one, cs),
                lambda: ops.ls_kvq_append(*cache, k, k, one, one.long(), cs),
                lambda: ops.ls_kvq_read(*cache, one, k, k[:1]),
                lambda: ops.ls_kvq_read(*cache, one, k.double(), k.double()),
                lambda: ops.ls_kvq_read(*cache, one, k.cpu(), k)):
        with pytest.raises(ValueError):
            bad()
    refused(lambda: ops.ls_kvq_read(*cache, one, k[:, :1].expand(2, 2, 64), k), text="overlap")
    q, pages, lens = rand((2, 4, 64), 1, torch.float16), ints([[0, 1], [2, 3]]), ints([20, 3])
    o = torch.empty_like(q)
    ok = dict(max_len=32, scale=0.1)
    ops.ls_kvq_attend(q, *cache, pages, lens, o, **ok)
    refused(lambda: ops.ls_kvq_attend(q, *cache, pages, lens, o, max_len=32, scale=0.0), text="scale")
    refused(lambda: ops.ls_kvq_attend(q, *cache, pages, lens, o, max_len=-1, scale=0.1), text="max_len")
    refused(lambda: ops.ls_kvq_attend(q[:, :3], *cache, pages, lens, o[:, :3], **ok), text="multiple of n_kv_heads")
    refused(lambda: ops.ls_kvq_attend(q.float(), *cache, pages, lens, o.float(), **ok), status=lsffn.LS_E_UNSUPPORTED)
    big = empty_cache(4, 2, 16, 264, "fp8")
    q264 = rand((2, 4, 264), 1, torch.float16)
    refused(lambda: ops.ls_kvq_attend(q264, *big, pages, lens, torch.empty_like(q264), **ok), text="at most 256")
    refused(lambda: ops.ls_kvq_attend(rand((2, 4, 68), 1, torch.float16)[..., :64], *cache, pages, lens, o, **ok), text="multiples of 8")
    for bad in (lambda: ops.ls_kvq_attend(q, *cache, pages, lens, o, max_len=33, scale=0.1),
                lambda: ops.ls_kvq_attend(q, *cache, pages, lens, o, prefix_pages=ints([0]), prefix_len=17, **ok),
                lambda: ops.ls_kvq_attend(q, *cache, pages, lens, o.bfloat16(), **ok)):
        with pytest.raises(ValueError):
            bad()
    lib = lsffn.load()
    assert lib.ls_kvq_append(ops.ctx, None, lsffn.LS_F16, None) == lsffn.LS_E_INVAL
    assert lib.ls_kvq_read(ops.ctx, None, None) == lsffn.LS_E_INVAL and lib.ls_kvq_attend(ops.ctx, None, lsffn.LS_F16, None) == lsffn.LS_E_INVAL
    ops.ls_kvq_attend(q, *cache, pages, lens, o, **ok)
    # no tokens, no sequences: nothing
    ops.ls_kvq_append(*cache, k[:0], k[:0], one[:0], one[:0], cs)
    ops.ls_kvq_read(*cache, one[:0], k[:0], k[:0])
    ops.ls_kvq_attend(q[:0], *cache, pages[:0], lens[:0], o[:0], **ok)
    ops.ls_ops_sync()
    assert ctypes.c_void_p(ops.ctx).value

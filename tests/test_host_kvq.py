"""What the quantised cache's calls and ls_verify refuse, and how attention over codes is cut into parts, without a GPU: the C entry points
built for the host, over a runtime whose launches count themselves (tests/native/ops_checks.cpp)."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2609_03079_amd as lsffn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F16, BF16, I8, FP4, FP8 = lsffn.LS_F32, lsffn.LS_F16, lsffn.LS_BF16, lsffn.LS_I8, lsffn.LS_FP4, lsffn.LS_FP8
I32, I64, P = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
A = 1 << 20   # an aligned address that nothing reads


def struct(name, *fields):
    return type(name, (ctypes.Structure,), {"_fields_": [(n, t) for names, t in fields for n in names.split()]})


Cache = struct("Cache", ("k v k_scale v_scale", P), ("code n_pages page_size n_kv_heads head_dim", I32),
               ("page_stride head_stride token_stride scale_page_stride scale_head_stride scale_token_stride", I64))
Append = struct("Append", ("n_tokens n_heads rot_dim n_pos style", I32), ("k", P), ("k_token_stride k_head_stride", I64), ("v", P),
                ("v_token_stride v_head_stride", I64), ("q", P), ("q_token_stride q_head_stride", I64), ("q_out", P),
                ("q_out_token_stride q_out_head_stride", I64), ("positions slots cos_sin", P))
Read = struct("Read", ("n_tokens type", I32), ("slots k", P), ("k_token_stride k_head_stride", I64), ("v", P), ("v_token_stride v_head_stride", I64))
Attend = struct("Attend", ("n_seqs n_q n_heads prefix_len max_len", I32), ("scale", ctypes.c_float), ("q", P), ("q_token_stride q_head_stride", I64),
                ("out", P), ("out_token_stride out_head_stride", I64), ("prefix_pages pages", P), ("pages_stride", I64), ("lens", P))
Verify = struct("Verify", ("n_seqs n_drafts vocab type", I32), ("target", P), ("target_seq_stride target_token_stride", I64), ("draft", P),
                ("draft_seq_stride draft_token_stride", I64), ("drafts", P), ("drafts_stride", I64), ("counts accept", P), ("accept_stride", I64),
                ("sample tokens", P), ("tokens_stride", I64), ("n_accepted", P))


def cache(**more):
    v = dict(k=A, v=A, k_scale=A + 1, v_scale=A + 3, code=FP4, n_pages=9, page_size=16, n_kv_heads=2, head_dim=80, page_stride=1280, head_stride=640,
             token_stride=40, scale_page_stride=96, scale_head_stride=48, scale_token_stride=3)
    return Cache(**{**v, **more})


def append(**more):
    v = dict(n_tokens=5, n_heads=4, rot_dim=80, n_pos=7, style=0, k=A, k_token_stride=160, k_head_stride=80, v=A, v_token_stride=160, v_head_stride=80,
             q=A, q_token_stride=320, q_head_stride=80, q_out=A, q_out_token_stride=320, q_out_head_stride=80, positions=A, slots=A, cos_sin=A)
    return Append(**{**v, **more})


def read(**more):
    v = dict(n_tokens=5, type=F16, slots=A, k=A, k_token_stride=160, k_head_stride=80, v=A, v_token_stride=160, v_head_stride=80)
    return Read(**{**v, **more})


def attend(**more):
    v = dict(n_seqs=3, n_q=2, n_heads=4, prefix_len=20, max_len=100, scale=0.1, q=A, q_token_stride=320, q_head_stride=80, out=A, out_token_stride=320,
             out_head_stride=80, prefix_pages=A, pages=A, pages_stride=7, lens=A)
    return Attend(**{**v, **more})


def verify(**more):
    v = dict(n_seqs=3, n_drafts=2, vocab=100, type=F32, target=A, target_seq_stride=300, target_token_stride=100, draft=A, draft_seq_stride=200,
             draft_token_stride=100, drafts=A, drafts_stride=2, counts=None, accept=A, accept_stride=2, sample=A, tokens=A, tokens_stride=3,
             n_accepted=A)
    return Verify(**{**v, **more})


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("native") / "ops_checks.so")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-x", "c++", "-D__HIP_PLATFORM_AMD__", f"-I{rocm}/include",
                        f"-I{ROOT}/include", os.path.join(ROOT, "tests", "native", "ops_checks.cpp"), "-o", so], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lib = ctypes.CDLL(so)
    lib.ls_ops_last_error.restype = ctypes.c_char_p
    lib.ls_ops_last_error.argtypes = lib.ls_ops_destroy.argtypes = [P]
    return lib


@pytest.fixture
def ctx(lib):
    h, desc = P(), lsffn.LsOpsDesc(0, None, 0)
    assert lib.ls_ops_create(ctypes.byref(desc), ctypes.byref(h)) == lsffn.LS_OK
    yield h
    assert lib.ls_ops_destroy(h) == lsffn.LS_OK


def call(lib, ctx, what, c, args, typ=F16):
    r = ctypes.byref
    if what == "append":
        return lib.ls_kvq_append(ctx, r(c) if c else None, typ, r(args))
    if what == "read":
        return lib.ls_kvq_read(ctx, r(c) if c else None, r(args))
    if what == "attend":
        return lib.ls_kvq_attend(ctx, r(c) if c else None, typ, r(args))
    return lib.ls_verify(ctx, r(args))


MAKE = {"append": append, "read": read, "attend": attend, "verify": verify}

BAD_CACHES = [(dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(k_scale=None), "NULL"), (dict(v_scale=None), "NULL"), (dict(code=I8), "code"),
              (dict(code=F16), "code"), (dict(n_pages=0), "n_pages"), (dict(page_size=0), "page_size"), (dict(page_size=12), "power of two"),
              (dict(page_size=8192), "page_size"), (dict(n_pages=1 << 27, page_size=16), "2^31"), (dict(n_kv_heads=0), "n_kv_heads"),
              (dict(n_kv_heads=4097), "n_kv_heads"), (dict(head_dim=0), "head_dim"), (dict(head_dim=1032), "head_dim"), (dict(head_dim=76), "multiple of 8"),
              (dict(page_stride=-4), "negative"), (dict(scale_page_stride=-1), "negative"), (dict(scale_token_stride=-1), "negative"),
              (dict(k=A + 2), "4 bytes"), (dict(token_stride=42), "4 bytes"), (dict(code=FP8, token_stride=84), "8 bytes"), (dict(code=FP8, v=A + 4), "8 bytes")]


@pytest.mark.parametrize("what", ["append", "read", "attend"])
@pytest.mark.parametrize("bad,word", BAD_CACHES, ids=lambda x: x if isinstance(x, str) else "-".join(x))
def test_bad_caches(lib, ctx, what, bad, word):
    before = lib.ops_launches()
    assert call(lib, ctx, what, cache(**bad), MAKE[what]()) == lsffn.LS_E_INVAL
    assert word in lib.ls_ops_last_error(ctx).decode() and lib.ops_launches() == before
    assert call(lib, ctx, what, cache(), MAKE[what]()) == lsffn.LS_OK and lib.ops_launches() == before + 1


BAD = [("append", dict(n_tokens=-1), "n_tokens"), ("append", dict(n_heads=-1), "n_heads"), ("append", dict(rot_dim=41), "rot_dim"),
       ("append", dict(rot_dim=82), "rot_dim"), ("append", dict(style=2), "style"), ("append", dict(q=None), "q and q_out"),
       ("append", dict(q_out=None), "q and q_out"), ("append", dict(n_heads=0), "q and q_out"), ("append", dict(k=None), "NULL"),
       ("append", dict(slots=None), "NULL"), ("append", dict(positions=None), "rotation"), ("append", dict(cos_sin=None), "rotation"),
       ("append", dict(n_pos=0), "rotation"), ("append", dict(k_head_stride=-1), "negative"), ("append", dict(q_out=A + 1), "aligned"),
       ("append", dict(slots=A + 2), "aligned"), ("append", dict(cos_sin=A + 2), "aligned"),
       ("read", dict(n_tokens=-1), "n_tokens"), ("read", dict(type=I8), "type"), ("read", dict(type=FP4), "type"), ("read", dict(k=None), "NULL"),
       ("read", dict(slots=None), "NULL"), ("read", dict(v_head_stride=-1), "negative"), ("read", dict(k_head_stride=40), "overlap"),
       ("read", dict(k_token_stride=80), "overlap"), ("read", dict(v_token_stride=0), "overlap"), ("read", dict(v_head_stride=0), "overlap"),
       ("read", dict(k_token_stride=152), "overlap"), ("read", dict(k_token_stride=80, k_head_stride=392), "overlap"),
       ("read", dict(k=A + 1), "aligned"), ("read", dict(slots=A + 1), "aligned"),
       ("attend", dict(n_seqs=-1), "n_seqs"), ("attend", dict(n_q=0), "n_q"), ("attend", dict(n_q=17), "n_q"), ("attend", dict(n_heads=3), "multiple"),
       ("attend", dict(n_heads=0), "multiple"), ("attend", dict(prefix_len=-1), "prefix_len"), ("attend", dict(max_len=1 << 22), "max_len"),
       ("attend", dict(scale=0.0), "scale"), ("attend", dict(scale=float("nan")), "scale"), ("attend", dict(scale=float("inf")), "scale"),
       ("attend", dict(q=None), "NULL"), ("attend", dict(lens=None), "NULL"), ("attend", dict(prefix_pages=None), "prefix_pages"),
       ("attend", dict(pages=None), "pages"), ("attend", dict(pages_stride=6), "pages_stride"), ("attend", dict(q_head_stride=84), "multiples of 8"),
       ("attend", dict(out_token_stride=-8), "multiples of 8"), ("attend", dict(out=A + 8), "16-byte"), ("attend", dict(lens=A + 2), "aligned"),
       ("verify", dict(type=FP8), "type"), ("verify", dict(n_seqs=-1), "n_seqs"), ("verify", dict(n_drafts=64), "n_drafts"),
       ("verify", dict(n_drafts=-1), "n_drafts"), ("verify", dict(vocab=0), "vocab"), ("verify", dict(vocab=(1 << 30) + 1), "vocab"),
       ("verify", dict(target=None), "NULL"), ("verify", dict(sample=None), "NULL"), ("verify", dict(drafts=None), "NULL"),
       ("verify", dict(accept=None), "NULL"), ("verify", dict(n_accepted=None), "NULL"), ("verify", dict(target_seq_stride=-1), "negative"),
       ("verify", dict(tokens_stride=2), "tokens_stride"), ("verify", dict(target=A + 2), "aligned"), ("verify", dict(counts=A + 1), "aligned")]


@pytest.mark.parametrize("what,bad,word", BAD, ids=lambda x: x if isinstance(x, str) else "-".join(x))
def test_bad_arguments(lib, ctx, what, bad, word):
    before = lib.ops_launches()
    assert call(lib, ctx, what, cache(), MAKE[what](**bad)) == lsffn.LS_E_INVAL
    assert word in lib.ls_ops_last_error(ctx).decode() and lib.ops_launches() == before


def test_other_answers(lib, ctx):
    before = lib.ops_launches()
    for what in ("append", "read", "attend"):
        assert call(lib, ctx, what, None, MAKE[what]()) == lsffn.LS_E_INVAL
        assert call(lib, None, what, cache(), MAKE[what]()) == lsffn.LS_E_INVAL
    for what, none in (("append", dict(n_tokens=0)), ("read", dict(n_tokens=0)), ("attend", dict(n_seqs=0)), ("verify", dict(n_seqs=0))):
        assert call(lib, ctx, what, cache(), MAKE[what](**none)) == lsffn.LS_OK
    assert call(lib, ctx, "attend", cache(), attend(), F32) == lsffn.LS_E_UNSUPPORTED
    assert call(lib, ctx, "append", cache(), append(), I8) == lsffn.LS_E_INVAL
    assert call(lib, ctx, "attend", cache(head_dim=264, token_stride=132, head_stride=2112, page_stride=4224), attend()) == lsffn.LS_E_INVAL
    assert lib.ops_launches() == before
    assert call(lib, ctx, "verify", None, verify(n_drafts=0, drafts=None, accept=None, draft=None, tokens_stride=1)) == lsffn.LS_OK
    assert call(lib, ctx, "append", cache(), append(n_heads=0, q=None, q_out=None, rot_dim=0, positions=None, cos_sin=None)) == lsffn.LS_OK
    # heads outermost, one head, one token
    assert call(lib, ctx, "read", cache(), read(k_token_stride=80, k_head_stride=400)) == lsffn.LS_OK
    assert call(lib, ctx, "read", cache(n_kv_heads=1), read(k_token_stride=80, k_head_stride=0, v_token_stride=80, v_head_stride=0)) == lsffn.LS_OK
    assert call(lib, ctx, "read", cache(), read(n_tokens=1, k_token_stride=0, v_token_stride=0)) == lsffn.LS_OK
    assert lib.ops_launches() == before + 5


def test_plans(lib, ctx):
    """Whatever the shapes, the parts cover the keys and fit the join, the workspace and a launch (the stub looks at each plan); where no split
    fits the workspace, which is where the header says so alone, the call says so."""
    rng = random.Random(1)
    h, desc = P(), lsffn.LsOpsDesc(1 << 20, None, 0)
    assert lib.ls_ops_create(ctypes.byref(desc), ctypes.byref(h)) == lsffn.LS_OK
    small = 0
    for _ in range(600):
        kv, G, dim, code = rng.choice([1, 2, 5, 8, 32, 128]), rng.choice([1, 2, 7, 8, 16]), rng.choice([8, 64, 80, 128, 256]), rng.choice([FP4, FP8])
        pages, page = 1 << 15, rng.choice([1, 16, 64, 4096])
        row = dim // 2 if code == FP4 else dim
        c = cache(code=code, n_kv_heads=kv, head_dim=dim, n_pages=pages, page_size=page, token_stride=row, head_stride=row * page,
                  page_stride=row * page * kv)
        n = int(10 ** rng.uniform(0, 3.5))
        top = rng.choice([0, 1, 63, 64, 65, int(10 ** rng.uniform(1, 6.5))])
        a = attend(n_seqs=n, n_q=rng.choice([1, 1, 2, 8, 16]), n_heads=kv * G, prefix_len=rng.choice([0, 1, 100, int(10 ** rng.uniform(1, 6.5))]), max_len=top,
                   pages_stride=max(1, -(-top // page)), q_token_stride=kv * G * dim, q_head_stride=dim, out_token_stride=kv * G * dim, out_head_stride=dim)
        rows = a.n_q * a.n_heads
        need = 2 * 4 * (dim + 2) * rows * min(n, max(1, (1 << 20) // rows))   # what a split takes, by the header
        for x, ws in ((ctx, 256 << 20), (h, 1 << 20)):
            st = call(lib, x, "attend", c, a)
            assert st == lsffn.LS_OK or (st == lsffn.LS_E_CAPACITY and need > ws), lib.ls_ops_last_error(x)
            small += st == lsffn.LS_E_CAPACITY
    assert 0 < small < 1200
    assert lib.ls_ops_destroy(h) == lsffn.LS_OK


def test_native_module_has_the_calls():
    if not os.path.exists(lsffn.LIB_PATH):
        from paper_2609_03079_amd import build
        build.build()
    for name in ("ls_kvq_append", "ls_kvq_read", "ls_kvq_attend", "ls_verify"):
        assert name in lsffn.OPS_EXPORTS and hasattr(lsffn._load_native().Ops, name)

"""Every plan of the attention over codes writes inside the workspace and launches what a launch may hold, without a GPU (the plans built for the
host, tests/native/plan_checks.cpp)."""
import ctypes
import os
import random
import subprocess

import pytest

from test_host_kvq import FP4, FP8, attend, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PARTS = 128   # that a row's join takes


@pytest.fixture(scope="module")
def plan_of(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("native") / "plan_checks.so")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-x", "c++", "-D__HIP_PLATFORM_AMD__", f"-I{rocm}/include",
                        os.path.join(ROOT, "tests", "native", "plan_checks.cpp"), "-o", so], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    f = ctypes.CDLL(so).plan_of
    f.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int, ctypes.c_void_p]

    def run(c, a, ws, n_cu=256):
        out = (ctypes.c_int64 * 11)()
        names = "pre_parts suf_parts bytes first second pre_chunk suf_chunk pre_wide suf_wide alike together".split()
        return dict(zip(names, out)) if f(ctypes.byref(c), ctypes.byref(a), ws, n_cu, out) else None
    return run


def shape(rng):
    kv, G, dim, code = rng.choice([1, 2, 5, 8, 32, 128, 4096]), rng.choice([1, 1, 2, 7, 8, 16]), rng.choice([8, 64, 80, 128, 136, 256]), rng.choice([FP4, FP8])
    heads, n_q = min(kv * G, 4096 // kv * kv), rng.choice([1, 1, 2, 3, 8, 16])
    length = lambda: rng.choice([0, 1, 64, int(10 ** rng.uniform(0, 6.62)), 2 ** 22 - 1])  # noqa: E731
    a = attend(n_heads=heads, n_q=n_q, prefix_len=length(), max_len=length())
    # as many rows as a plan is made for: 2^20, or one sequence
    a.n_seqs = max(1, min(int(10 ** rng.uniform(0, 6.1)), 2 ** 20 // (n_q * heads)))
    if rng.random() < 0.6:   # a prefix of more than 32 rows beside sequences of at most 32, which may run at once
        kv, G, a.n_q = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3])
        a.n_heads, a.n_seqs = kv * G, 33 // (a.n_q * G) + int(10 ** rng.uniform(0, 3))
        a.prefix_len, a.max_len = (int(10 ** rng.uniform(1, 6.6)) for _ in range(2))
    return cache(code=code, n_kv_heads=kv, head_dim=dim, page_size=rng.choice([1, 16, 4096])), a


@pytest.mark.parametrize("n_cu", [8, 256, 304])
def test_plans_fit(plan_of, n_cu):
    rng, kinds = random.Random(n_cu), set()
    for _ in range(20000):
        c, a = shape(rng)
        ws = int(2 ** rng.uniform(20, 31))
        p = plan_of(c, a, ws, n_cu)
        row_parts = a.n_seqs * a.n_q * a.n_heads * (c.head_dim + 2) * 4
        if p is None:
            assert 2 * row_parts > ws   # as the header says: what a split takes does not fit
            kinds.add("refused")
            continue
        assert p["bytes"] <= ws
        assert 1 <= p["pre_parts"] + p["suf_parts"] <= PARTS
        assert p["pre_parts"] * p["pre_chunk"] >= a.prefix_len and p["suf_parts"] * p["suf_chunk"] >= a.max_len
        for n in (p["first"], p["second"]):
            assert n * 256 < 2 ** 32
        assert p["first"] > 0
        for what in ("pre_wide", "suf_wide", "alike", "together", "second"):
            kinds.add((what, bool(p[what])))
        kinds.add(("direct", p["bytes"] == 0))
    if n_cu == 256:
        assert len(kinds) == 13, kinds   # every kind of plan was there


@pytest.mark.parametrize("extra", [-1, 0])
def test_where_the_workspace_ends(plan_of, extra):
    """One part of prefix and sequences each is what has to fit, to the byte."""
    for c, a in ((cache(), attend(n_seqs=40, n_q=16, n_heads=64, prefix_len=2000, max_len=100)),
                 (cache(n_kv_heads=1), attend(n_seqs=1000, n_q=1, n_heads=8, prefix_len=30, max_len=70))):
        ws = 2 * a.n_seqs * a.n_q * a.n_heads * (c.head_dim + 2) * 4
        assert (plan_of(c, a, ws + extra) is not None) == (extra == 0)

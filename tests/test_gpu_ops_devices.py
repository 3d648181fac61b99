"""Tensors of another GPU than the context's are refused before any call (stand-ins without memory: one GPU is enough)."""
from types import SimpleNamespace

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_03079_amd as lsffn  # noqa: E402
from test_gpu_ops import DEV, ints, make_cache, ops, rand, table  # noqa: E402, F401


class Elsewhere(torch.Tensor):
    """A tensor of t's shape, strides and type on another GPU, without memory."""

    @staticmethod
    def __new__(cls, t):
        return torch.Tensor._make_wrapper_subclass(cls, t.shape, strides=t.stride(), dtype=t.dtype, device="cuda:1")

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise RuntimeError("a stand-in computes nothing")


def calls(ops):
    f16 = dict(dtype=torch.float16, device=DEV)
    x, y, w = rand((2, 64), 1), rand((2, 64), 2, torch.float16), rand((64,), 3, torch.float16)
    yield "norm", lambda t: ops.ls_norm_residual(t["x"], y=t["y"], gate=t["gate"], post_norm=True, post_weight=t["post"], pre_norm=True,
                                                 pre_weight=t["pre"], x_out=t["x_out"], h=t["h"]), \
        {"x": x, "y": y, "gate": w, "post": w, "pre": w, "x_out": torch.empty_like(x), "h": torch.empty_like(y)}
    yield "linear", lambda t: ops.ls_linear_i8(t["x"], t["w"], t["ws"], t["out"], x_scale=t["xs"], bias=t["bias"]), \
        {"x": torch.ones((2, 64), dtype=torch.int8, device=DEV), "w": torch.ones((8, 64), dtype=torch.int8, device=DEV),
         "ws": torch.ones(8, device=DEV), "out": torch.empty((2, 8), device=DEV), "xs": torch.ones(2, device=DEV), "bias": torch.ones(8, device=DEV)}
    kc, vc = make_cache(4, 2, 16, 64, torch.float16, 0)
    k, q = rand((2, 2, 64), 1, torch.float16), rand((2, 4, 64), 2, torch.float16)
    yield "append", lambda t: ops.ls_kv_append(t["kc"], t["vc"], t["k"], t["v"], t["positions"], t["slots"], t["cs"], q=t["q"], q_out=t["q_out"]), \
        {"kc": kc, "vc": vc, "k": k, "v": k, "positions": ints([0, 1]), "slots": ints([0, 1]), "cs": table(8, 64), "q": q,
         "q_out": torch.empty((2, 4, 64), **f16)}
    yield "attend", lambda t: ops.ls_attend(t["q"], t["kc"], t["vc"], t["pages"], t["lens"], t["out"], max_len=16, scale=0.1,
                                            prefix_pages=t["prefix"], prefix_len=4), \
        {"q": q, "kc": kc, "vc": vc, "pages": ints([[0], [1]]), "lens": ints([3, 9]), "out": torch.empty((2, 4, 64), **f16), "prefix": ints([2])}


def test_tensors_of_another_gpu_are_refused(ops):
    for name, call, tensors in calls(ops):
        call(tensors)
        for which, t in tensors.items():
            with pytest.raises(ValueError, match="another GPU"):
                call({**tensors, which: Elsewhere(t)})
        call(tensors)
    ops.ls_ops_sync()


def test_a_stream_of_another_device_is_refused():
    # what the constructor asks a stream: its device and its address
    with pytest.raises(ValueError, match="device 1"):
        lsffn.Ops(stream=SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))

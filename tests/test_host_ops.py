"""Host-side checks of the decoder-layer operators that need no GPU: the library exports every entry
point that their header declares and refuses bad descriptors."""
import ctypes
import os
import re

import paper_2609_03079_amd as lsffn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _lib():
    if not os.path.exists(lsffn.LIB_PATH):
        from paper_2609_03079_amd import build
        build.build()
    return lsffn.load()


def test_library_exports_every_declared_operator():
    text = open(os.path.join(ROOT, "include", "ls_ops.h")).read()
    declared = set(re.findall(r"^\s*(?:ls_status|const char\*)\s+(ls_\w+)\s*\(", text, re.M))
    assert declared == set(lsffn.OPS_EXPORTS)
    lib = ctypes.CDLL(_lib()._name)
    for name in declared:
        assert hasattr(lib, name), name


def test_native_module_is_of_these_sources():
    _lib()
    native = lsffn._load_native()
    from paper_2609_03079_amd import build
    assert native.digest == build.source_digest()
    for name in ("ls_norm_residual", "ls_linear_i8", "ls_kv_append", "ls_attend", "ls_ops_sync", "close"):
        assert hasattr(native.Ops, name)


def test_create_refuses_bad_arguments():
    lib = _lib()
    h = ctypes.c_void_p()
    assert lib.ls_ops_create(None, ctypes.byref(h)) == lsffn.LS_E_INVAL and not h.value
    assert b"desc" in lib.ls_ops_last_error(None)
    for desc, word in ((lsffn.LsOpsDesc(0, None, 7), b"debug_flags"), (lsffn.LsOpsDesc(1000, None, 0), b"workspace_bytes")):
        assert lib.ls_ops_create(ctypes.byref(desc), ctypes.byref(h)) == lsffn.LS_E_INVAL and not h.value
        assert word in lib.ls_ops_last_error(None)
    assert lib.ls_ops_destroy(None) == lsffn.LS_E_INVAL
    assert lib.ls_attend(None, None, None) == lsffn.LS_E_INVAL

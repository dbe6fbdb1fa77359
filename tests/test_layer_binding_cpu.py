"""Host side of the layer operators' torch functions (no GPU needed)."""
import ctypes
import os
import types

import paper_2609_14706_amd as ff
from paper_2609_14706_amd import layer


def test_another_thread_during_the_first_call(monkeypatch):
    """The table of functions is empty or whole at every moment: a thread that
    finds it empty makes its own, one that finds it filled can use all of it."""
    seen = []

    class Library:
        def __getattr__(self, name):
            seen.append(len(layer._FN))
            return types.SimpleNamespace(name=name)
    monkeypatch.setattr(layer, "_FN", {})
    monkeypatch.setattr(layer, "load_library", Library)
    made = layer._library()
    assert len(seen) == len(made) == 10 and not any(seen)
    assert layer._library() is layer._FN and len(layer._FN) == 10


def test_a_scale_beyond_fp32():
    """Refused before a device is touched (the addresses are never read)."""
    if not os.path.exists(ff.LIB_PATH):
        from paper_2609_14706_amd.build import build
        build()
    p = 1 << 40
    a = ff.ff_ortho_args(1, 8, 8, 0, p, 8, 64, 2 * p, 8, 64, 5, 3.4445, -4.775, 2.0315, 1e-7, 1e39)
    assert layer._library()["ff_orthogonalize"](ctypes.byref(a)) == ff.FF_ERR_INVALID_ARG
    assert "scale" in ff.ff_last_error()

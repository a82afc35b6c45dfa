"""Host-side checks of the decoder operators' entry points that need no GPU."""
import ctypes

import paper_2609_00224_gb300 as qt
from paper_2609_00224_gb300 import decoder as d

P = ctypes.c_void_p(256)
BAD = qt.QTEA_ERR_INVALID_ARG


def test_kv_create_refuses_before_it_looks_for_a_device():
    lib = qt.load()
    h = ctypes.c_void_p(5)
    make = lib.qtea_kv_create
    assert make(None, P, None, None, 1, 16, 1, 64, 0, ctypes.byref(h)) == BAD and not h.value
    assert make(P, P, None, None, 1, 16, 1, 64, 1, ctypes.byref(h)) == BAD  # FP8 without scales
    assert make(P, P, None, None, 1, 16, 1, 64, 5, ctypes.byref(h)) == BAD  # no such format
    assert make(ctypes.c_void_p(24), P, None, None, 1, 16, 1, 64, 0, ctypes.byref(h)) == BAD  # alignment
    assert make(P, P, None, None, 0, 16, 1, 64, 0, ctypes.byref(h)) == BAD
    assert make(P, P, None, None, 1 << 28, 16, 1, 64, 0, ctypes.byref(h)) == BAD  # 2^32 rows
    for page, dim in ((8, 64), (24, 64), (512, 64), (16, 32), (16, 96), (16, 256)):
        assert make(P, P, None, None, 1, page, 1, dim, 0, ctypes.byref(h)) == qt.QTEA_ERR_UNSUPPORTED
    assert make(P, P, None, None, 1, 16, 1, 64, 0, None) == BAD
    lib.qtea_kv_free(None)


def test_calls_without_a_cache_are_refused():
    lib = qt.load()
    b = ctypes.byref(d._Batch(P, P, P, 1, 1, 1, 1))
    assert lib.qtea_kv_append(None, b, bytes(d._APPEND.size), None) == BAD
    assert lib.qtea_kv_read(None, b, P, 1, P, P, None) == BAD
    assert lib.qtea_attention(None, b, P, 64, 1, 1.0, 0, P, 64, None, P, 1 << 30, None) == BAD
    assert lib.qtea_attention_workspace(None) == BAD
    assert lib.qtea_attention_status(None, 1 << 20, None) == BAD
    assert lib.qtea_attention_status(P, 16, None) == BAD


def norm(**kw):
    a = dict(h=256, y=256, post_weight=256, gate=256, weight=256, h_out=256, x=256, h_ld=64, y_ld=64, gate_ld=64,
             h_out_ld=64, x_ld=64, h_type=0, y_type=0, n_rows=2, n_cols=64, res_scale=1.0, eps=1e-6)
    a.update(kw)
    return qt.load().qtea_norm(d._NORM.pack(*(v or 0 for v in a.values())), None)


def test_norm_refusals():
    assert qt.load().qtea_norm(None, None) == BAD
    assert norm(n_rows=0) == qt.QTEA_OK  # nothing to do
    for kw in (dict(n_rows=-1), dict(n_cols=0), dict(n_cols=(1 << 20) + 1), dict(h=None), dict(h=258), dict(h_ld=63),
               dict(y_ld=63), dict(y=258), dict(h_out=None), dict(h_out_ld=60), dict(weight=None), dict(x_ld=63),
               dict(gate_ld=63), dict(gate=257), dict(post_weight=257), dict(h_type=2), dict(y_type=-1),
               dict(y=None), dict(y=None, post_weight=None, gate=None, x=None)):
        assert norm(**kw) == BAD, kw


def test_workspace_header_is_the_kernels():
    import pathlib
    import re
    text = (pathlib.Path(qt.__file__).parent / "csrc" / "qtea_attn.h").read_text()
    assert int(re.search(r"kAttnHeaderBytes = (\d+);", text).group(1)) == d._WORKSPACE_HEADER

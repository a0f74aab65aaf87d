"""Arguments that attention over shared prefixes refuses, on the host and before anything is launched (no GPU is touched here;
addresses are made up and never followed), and the workspace sizes it states."""
import ctypes

import numpy as np
import pytest

import paper_2509_10798_amd as jq
from paper_2509_10798_amd.binding import _CPages, _CPrefixes

M = 1 << 30
Q, K, V, KP, VP, OUT, LSE, LENS, PLENS, WS, TABLE, PTABLE = (M * (1024 + 8 * i) for i in range(12))
NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIAS = -1, -2, -4, -5, -6
I32P = ctypes.POINTER(ctypes.c_int32)


def shape(**kw):
    base = dict(n_layers=2, seq_lens=[100, 64, 30], n_q=4, h_q=8, h_kv=2)
    base.update(kw)
    return jq.Shape(**base)


def prefixes(members=(0, 2, 3), rows=(0, 500, 533), n=2, lens=PLENS, per=16, table=PTABLE):
    keep = [np.array(x, dtype=np.int32) if x is not None else None for x in (members, rows)]
    ptr = [ctypes.cast(None, I32P) if x is None else x.ctypes.data_as(I32P) for x in keep]
    p = _CPrefixes(n, ptr[0], ptr[1], lens, per, table)
    p.keep = keep
    return p


def pages(size=32, n=64, per=4, table=TABLE):
    return _CPages(size, n, per, table)


def call(sh=None, pre=None, pg=None, none=False, **kw):
    sh, pre = sh or shape(), pre or prefixes()
    a = dict(lens=LENS, q=Q, kp=KP, vp=VP, k=K, v=V, out=OUT, lse=LSE, ws=WS, ws_bytes=1 << 29)
    a.update(kw)
    pp = None if none else ctypes.byref(pre)
    if pg is not None:
        return jq.lib().jq_attend_shared_paged(ctypes.byref(sh.c_struct()), ctypes.byref(pg), pp, a["lens"], a["q"], a["k"], a["v"], a["out"], a["lse"], a["ws"],
                                               a["ws_bytes"], None)
    return jq.lib().jq_attend_shared(ctypes.byref(sh.c_struct()), pp, a["lens"], a["q"], a["kp"], a["vp"], a["k"], a["v"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


def size(sh, pre):
    n = ctypes.c_size_t()
    rc = jq.lib().jq_attend_shared_workspace_bytes(ctypes.byref(sh.c_struct()), ctypes.byref(pre), ctypes.byref(n))
    return rc if rc else n.value


@pytest.mark.parametrize("pg", [None, pages()])
def test_prefixes(pg):
    assert call(none=True, pg=pg) == NULL
    assert call(pre=prefixes(members=None), pg=pg) == NULL and call(pre=prefixes(rows=None), pg=pg) == NULL
    for bad in ((0, 2, 2), (0, 3, 3), (1, 2, 3), (0, 2, 4), (0, 0, 3)):
        assert call(pre=prefixes(members=bad), pg=pg) == SHAPE
    for bad in ((0, 500, 500), (1, 500, 533), (0, -5, 533)):
        assert call(pre=prefixes(rows=bad), pg=pg) == SHAPE
    assert call(pre=prefixes(n=0), pg=pg) == SHAPE and call(pre=prefixes(n=-1), pg=pg) == SHAPE
    assert call(pre=prefixes(members=(0, 1, 2, 3, 3), rows=(0, 5, 6, 7, 8), n=4), pg=pg) == SHAPE
    assert call(pre=prefixes(lens=PLENS + 2), pg=pg) == UNSUPPORTED
    assert call(pre=prefixes(rows=(0, 500, 500 + (1 << 23)))) == UNSUPPORTED   # 4 GiB of a prefix's keys


def test_pointers():
    for field in ("q", "kp", "vp", "k", "v", "out", "ws"):
        assert call(**{field: None}) == NULL
    for field, at in (("q", Q), ("kp", KP), ("vp", VP), ("k", K), ("v", V), ("out", OUT)):
        assert call(**{field: at + 8}) == UNSUPPORTED
    assert call(lse=LSE + 2) == UNSUPPORTED and call(lens=LENS + 1) == UNSUPPORTED
    assert call(ws=WS + 8) == WORKSPACE
    need = size(shape(), prefixes())
    assert call(ws_bytes=need - 1) == WORKSPACE
    assert call(sh=shape(d=64)) == UNSUPPORTED and call(sh=shape(h_q=7)) == SHAPE and call(sh=shape(n_q=31, window=True)) == SHAPE


def test_pages():
    assert call(pg=pages(size=48)) == SHAPE and call(pg=pages(per=3)) == SHAPE and call(pg=pages(table=None)) == NULL
    assert call(pg=pages(), pre=prefixes(per=15)) == SHAPE and call(pg=pages(), pre=prefixes(table=None)) == NULL
    assert call(pg=pages(), pre=prefixes(table=PTABLE + 1)) == UNSUPPORTED


def test_nothing_may_overlap_what_is_written():
    q, own, pre = 2 * 3 * 4 * 8 * 256, 2 * 194 * 2 * 256, 2 * 533 * 2 * 256
    for at, n in ((Q, q), (K, own), (V, own), (KP, pre), (VP, pre), (LENS, 24), (PLENS, 16)):
        last = (at + n - 1) & ~15
        assert call(out=last) == ALIAS and call(lse=last) == ALIAS and call(ws=last) == ALIAS
    assert call(out=WS) == ALIAS and call(lse=OUT + q - 16) == ALIAS
    for at, n in ((TABLE, 3 * 4 * 4), (PTABLE, 2 * 16 * 4)):
        assert call(pg=pages(), out=(at + n - 1) & ~15) == ALIAS


def test_workspace_sizes():
    """Parts of both sweeps: 520 bytes a query row, head and share, of the prefixes and of the sequences."""
    one = size(shape(n_layers=1, seq_lens=[10], n_q=1, h_q=2, h_kv=1), prefixes(members=(0, 1), rows=(0, 10), n=1))
    assert 2 * 2 * 520 <= one <= 2 * 2 * 520 + 4 * 256
    assert size(shape(), prefixes(members=(0, 3, 3))) == SHAPE
    assert jq.lib().jq_attend_shared_workspace_bytes(ctypes.byref(shape().c_struct()), ctypes.byref(prefixes()), None) == NULL
    many = jq.Shape(n_layers=1, seq_lens=[1] * 128, n_q=1 << 14, h_q=1, h_kv=1)
    assert size(many, prefixes(members=(0, 128), rows=(0, 10), n=1)) == UNSUPPORTED   # 2^21 query rows of one prefix


def test_the_binding_checks_tensors():
    import torch
    sh, bf = shape(), torch.bfloat16
    pre = jq.Prefixes([500, 33], [2, 1])
    assert pre.T == 533 and jq.attend_shared_workspace_bytes(sh, pre) == size(sh, prefixes())
    with pytest.raises(ValueError, match="2 prefixes"):
        jq.Prefixes([500, 33], [3]).c_struct()
    x = torch.zeros((2, 194, 2, 128), dtype=bf)
    with pytest.raises(ValueError, match="not on a GPU"):
        jq.attend_shared(sh, pre, x, x, x, x, x)
    with pytest.raises(jq.JQError):
        jq.attend_shared_workspace_bytes(sh, jq.Prefixes([500, 33], [1, 1]))

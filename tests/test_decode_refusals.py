"""Arguments that the decoding calls refuse, on the host and before anything is launched (no GPU is touched here; addresses are
made up and never followed), and the workspace sizes they state."""
import ctypes

import pytest

import paper_2509_10798_amd as jq
from paper_2509_10798_amd.binding import _CPages

M = 1 << 30
Q, K, V, OUT, LSE, W, LENS, SEEN, WS, POS, KO, VO, WO, PO, IDX, TABLE, NEW_K, NEW_V, TOKEN, SLOT = (M * (1024 + 8 * i) for i in range(20))
NULL, SHAPE, BUDGET, UNSUPPORTED, WORKSPACE, ALIAS = -1, -2, -3, -4, -5, -6


def shape(**kw):
    base = dict(n_layers=2, seq_lens=[100, 64], n_q=4, h_q=8, h_kv=2, pool_k=1, budgets=[32, 16])
    base.update(kw)
    return jq.Shape(**base)


def pages(size=32, n=16, per=4, table=TABLE):
    return _CPages(size, n, per, table)


def attend(sh=None, pg=None, ws=WS, ws_bytes=None, weights=None, **kw):
    sh = sh or shape()
    a = dict(lens=LENS, q=Q, k=K, v=V, out=OUT, lse=LSE)
    a.update(kw)
    if ws_bytes is None:
        try:
            ws_bytes = jq.attend_workspace_bytes(sh, weights is not None)
        except jq.JQError:
            ws_bytes = 1 << 20
    front = (ctypes.byref(sh.c_struct()),) + (() if pg is None else (ctypes.byref(pg),))
    call = jq.lib().jq_attend if pg is None else jq.lib().jq_attend_paged
    return call(*front, a["lens"], a["q"], a["k"], a["v"], a["out"], a["lse"], weights, ws, ws_bytes, None)


def tree(sh=None, pg=None, seen=SEEN, ws=WS, **kw):
    sh = sh or shape()
    a = dict(lens=LENS, q=Q, k=K, v=V, out=OUT, lse=LSE)
    a.update(kw)
    front = (ctypes.byref(sh.c_struct()),) + (() if pg is None else (ctypes.byref(pg),))
    call = jq.lib().jq_attend_tree if pg is None else jq.lib().jq_attend_tree_paged
    return call(*front, a["lens"], seen, a["q"], a["k"], a["v"], a["out"], a["lse"], ws, 1 << 30, None)


def evict(sh=None, pg=None, ws=WS, ws_bytes=1 << 20, **kw):
    sh = sh or shape()
    a = dict(lens=LENS, k=K, v=V, w=W, pos=POS, ko=KO, vo=VO, wo=WO, po=PO, idx=IDX)
    a.update(kw)
    front = (ctypes.byref(sh.c_struct()),) + (() if pg is None else (ctypes.byref(pg),))
    call = jq.lib().jq_evict_weight if pg is None else jq.lib().jq_evict_weight_paged
    return call(*front, a["lens"], a["k"], a["v"], a["w"], a["pos"], a["ko"], a["vo"], a["wo"], a["po"], a["idx"], ws, ws_bytes, None)


def replace(sh=None, pg=None, **kw):
    sh = sh or shape()
    a = dict(lens=LENS, nk=NEW_K, nv=NEW_V, token=TOKEN, k=K, v=V, w=W, pos=POS, slot=SLOT)
    a.update(kw)
    front = (ctypes.byref(sh.c_struct()),) + (() if pg is None else (ctypes.byref(pg),))
    call = jq.lib().jq_replace_lightest if pg is None else jq.lib().jq_replace_lightest_paged
    return call(*front, a["lens"], a["nk"], a["nv"], a["token"], a["k"], a["v"], a["w"], a["pos"], a["slot"], None)


@pytest.mark.parametrize("call", [attend, tree, evict, replace])
@pytest.mark.parametrize("kw,code", [
    (dict(h_q=9), SHAPE), (dict(n_q=0), SHAPE), (dict(seq_lens=[100, 0]), SHAPE), (dict(d=64), UNSUPPORTED), (dict(n_layers=70000), UNSUPPORTED),
    (dict(scale=float("nan")), SHAPE), (dict(seq_lens=[2200000], h_q=8, h_kv=8, budgets=[4]), UNSUPPORTED), (dict(keep_last=-1), SHAPE)])
def test_malformed_shapes(call, kw, code):
    assert call(shape(**kw)) == code


@pytest.mark.parametrize("call", [attend, tree, evict, replace])
@pytest.mark.parametrize("pg,code", [
    (pages(size=16), SHAPE), (pages(size=48), SHAPE), (pages(per=3), SHAPE), (pages(n=0), SHAPE), (pages(table=None), NULL),
    (pages(table=TABLE + 2), UNSUPPORTED), (pages(size=65536, n=1 << 17), UNSUPPORTED)])
def test_malformed_pages(call, pg, code):
    assert call(pg=pg) == code


@pytest.mark.parametrize("call,names", [(attend, "q k v out ws"), (tree, "q k v out seen ws"), (evict, "k v w ko vo wo po ws"),
                                        (replace, "nk nv token k v w pos")])
def test_null_pointers(call, names):
    for name in names.split():
        assert call(**{name: None}) == NULL, name
        if name != "ws":
            assert call(pg=pages(), **{name: None}) == NULL, name


@pytest.mark.parametrize("call,names", [(attend, "q k v out"), (tree, "q k v out"), (evict, "k v ko vo"), (replace, "nk nv k v")])
def test_tensors_of_rows_lie_at_multiples_of_16(call, names):
    where = dict(q=Q, k=K, v=V, out=OUT, ko=KO, vo=VO, nk=NEW_K, nv=NEW_V)
    for name in names.split():
        assert call(**{name: where[name] + 8}) == UNSUPPORTED, name


@pytest.mark.parametrize("call,names", [(attend, "lens lse"), (tree, "lens lse seen"), (evict, "lens w pos wo po idx"), (replace, "lens token w pos slot")])
def test_words_lie_at_multiples_of_4(call, names):
    where = dict(lens=LENS, lse=LSE, seen=SEEN, w=W, pos=POS, wo=WO, po=PO, idx=IDX, token=TOKEN, slot=SLOT)
    for name in names.split():
        assert call(**{name: where[name] + 2}) == UNSUPPORTED, name
    assert attend(weights=W + 1) == UNSUPPORTED


def test_workspaces():
    sh = shape()
    need = jq.attend_workspace_bytes(sh)
    more = jq.attend_workspace_bytes(sh, weights=True)
    assert 0 < need < more and need % 256 == 0 and more % 256 == 0
    assert attend(ws=WS + 8) == WORKSPACE and attend(ws_bytes=need - 1) == WORKSPACE
    assert attend(weights=W, ws_bytes=need) == WORKSPACE         # sized for a call without weights
    assert evict(ws_bytes=jq.evict_weight_workspace_bytes(sh) - 1) == WORKSPACE and evict(ws=WS + 4) == WORKSPACE


def test_overlaps():
    assert attend(out=Q) == ALIAS and attend(out=K) == ALIAS and attend(lse=V + 512) == ALIAS and attend(lse=OUT) == ALIAS
    assert attend(weights=K + 4096) == ALIAS and attend(ws=OUT) == ALIAS and attend(weights=LENS) == ALIAS
    assert attend(pg=pages(), out=TABLE) == ALIAS
    assert tree(out=SEEN - 256) == ALIAS and tree(lse=SEEN) == ALIAS and tree(ws=K) == ALIAS
    same = dict(ko=K, vo=V, wo=W, po=POS)                        # within the cache: all outputs are their inputs ...
    for name, other in (("ko", KO), ("vo", VO), ("wo", WO), ("po", PO)):
        assert evict(**dict(same, **{name: other})) == ALIAS, name  # ... or none is
    assert evict(ko=V) == ALIAS and evict(ko=K + 256) == ALIAS and evict(idx=W) == ALIAS and evict(**dict(same, ws=K)) == ALIAS
    assert evict(**dict(same, idx=POS)) == ALIAS and evict(**dict(same, vo=K, v=K)) == ALIAS
    assert replace(k=V) == ALIAS and replace(nk=K + 4096) == ALIAS and replace(slot=POS) == ALIAS and replace(w=POS) == ALIAS
    assert replace(token=W) == ALIAS and replace(lens=POS) == ALIAS


def test_masks_and_room():
    assert attend(shape(window=True, seq_lens=[100, 3], budgets=[32, 3])) == SHAPE   # fewer rows than the window's tokens
    assert tree(shape(window=True)) == SHAPE                                          # a tree says itself what is seen
    assert tree(shape(n_q=65)) == SHAPE                                               # 64 rows cannot hold 65 drafted tokens
    assert tree(shape(n_q=1025, seq_lens=[2000, 1100])) == UNSUPPORTED
    assert attend(shape(n_q=33), weights=W) == UNSUPPORTED                            # 132 query rows a KV head
    with pytest.raises(jq.JQError):
        jq.attend_workspace_bytes(shape(n_q=33), weights=True)
    assert jq.attend_workspace_bytes(shape(n_q=33)) > 0


def test_budgets():
    assert evict(shape(budgets=[101, 1])) == BUDGET and evict(shape(budgets=[0, 1])) == BUDGET
    assert evict(shape(budgets=None)) == NULL
    assert evict(shape(keep_first=10, keep_last=7)) == BUDGET                         # more protected rows than 16
    assert evict(shape(window=True)) == SHAPE and replace(shape(window=True)) == SHAPE
    assert replace(shape(keep_first=60, keep_last=5)) == BUDGET                       # of 64 rows none may go
    assert replace(shape(keep_first=64)) == BUDGET


def test_python_checks_come_first():
    import torch
    sh = shape()
    with pytest.raises(jq.JQError):
        jq.attend_tree(sh, None, None, None, None)
    k = torch.zeros((2, 164, 2, 128), dtype=torch.bfloat16)
    for call in (lambda: jq.attend(sh, k, k, k), lambda: jq.evict_weight(sh, k, k, None), lambda: jq.replace_lightest(sh, k, k, k, k, k, k, k)):
        with pytest.raises(ValueError, match="lies on cpu"):
            call()


def test_tensor_checks():
    """What every tensor of these calls is looked at for, on tensors of the host (GPU number -1)."""
    import torch
    from paper_2509_10798_amd.binding import _cache_size, _tensor
    t = torch.zeros((4, 6), dtype=torch.int32)
    assert _tensor("t", t, torch.int32, (4, 6), -1) == t.data_ptr() and _tensor("t", None, torch.int32, (4, 6), -1) is None
    with pytest.raises(ValueError, match="t: .*float32.*is wanted"):
        _tensor("t", t, torch.float32, (4, 6), -1)
    with pytest.raises(ValueError, match=r"t: .*\(6, 4\) is wanted"):
        _tensor("t", t, torch.int32, (6, 4), -1)
    with pytest.raises(ValueError, match="not contiguous"):
        _tensor("t", t.T, torch.int32, (6, 4), -1)
    with pytest.raises(ValueError, match="lies on cpu, the call runs on GPU 0"):
        _tensor("t", t, torch.int32, (4, 6), 0)
    pg = jq.Pages(32, 6, None)
    assert _cache_size(shape(), pg, torch.zeros(1, 1, 1, 1, 1)) == (2, 6, 32, 2, 128)
    assert _cache_size(shape(), pg, torch.zeros(1, 1, 1, 1)) == (2, 192, 2, 128)      # rows numbered through
    assert _cache_size(shape(), None, t) == (2, 164, 2, 128)

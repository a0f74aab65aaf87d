"""Arguments that the calls on a cache of codes refuse, on the host and before anything is launched (no GPU is touched here; addresses
are made up and never followed)."""
import ctypes

import pytest

import paper_2509_10798_amd as jq
from paper_2509_10798_amd.binding import _CCodes, _CPages

M = 1 << 30
Q, K, V, OUT, LSE, W, FIRST, SEEN, WS, CK, CV, KS, VS, TABLE, LB = (M * (1024 + 8 * i) for i in range(15))
NULL, SHAPE, BUDGET, UNSUPPORTED, WORKSPACE, ALIAS = -1, -2, -3, -4, -5, -6


def shape(**kw):
    base = dict(n_layers=2, seq_lens=[100, 64], n_q=4, h_q=8, h_kv=2, pool_k=1, budgets=[32, 16])
    base.update(kw)
    return jq.Shape(**base)


def pages(size=32, n=16, per=4, table=TABLE):
    return _CPages(size, n, per, table)


def codes(**kw):
    a = dict(kb=8, vb=8, k=CK, v=CV, ks=KS, vs=VS)
    a.update(kw)
    return _CCodes(a["kb"], a["vb"], a["k"], a["v"], a["ks"], a["vs"])


def call(name, sh=None, pg=None, c=None, none=False, **kw):
    sh, c = sh or shape(), c or codes()
    a = dict(first=FIRST, k=K, v=V, q=Q, out=OUT, lse=LSE, w=W, ws=WS, ws_bytes=1 << 30, seen=SEEN)
    a.update(kw)
    front = (ctypes.byref(sh.c_struct()),) + (() if pg is None else (ctypes.byref(pg),))
    cp = None if none else ctypes.byref(c)
    f = getattr(jq.lib(), "jq_" + name + ("" if pg is None else "_paged"))
    if name == "quantize":
        return f(*front, a["first"], a["k"], a["v"], cp, None)
    if name == "dequantize":
        return f(*front, a["first"], cp, a["k"], a["v"], None)
    if name == "attend_quantized":
        return f(*front, a["first"], a["q"], cp, a["out"], a["lse"], a["w"], a["ws"], a["ws_bytes"], None)
    return f(*front, a["first"], a["seen"], a["q"], cp, a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


ALL = ["quantize", "dequantize", "attend_quantized", "attend_tree_quantized"]


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("pg", [None, pages()])
def test_codes(name, pg):
    assert call(name, pg=pg, none=True) == NULL
    for bad in (0, 2, 16, -8):
        assert call(name, pg=pg, c=codes(kb=bad)) == SHAPE and call(name, pg=pg, c=codes(vb=bad)) == SHAPE
    assert call(name, pg=pg, c=codes(kb=4, vb=8)) == UNSUPPORTED
    for field in ("k", "v", "ks", "vs"):
        assert call(name, pg=pg, c=codes(**{field: None})) == NULL
    for field, at in (("k", CK), ("v", CV)):
        assert call(name, pg=pg, c=codes(**{field: at + 8})) == UNSUPPORTED
    for field, at in (("ks", KS), ("vs", VS)):
        assert call(name, pg=pg, c=codes(**{field: at + 2})) == UNSUPPORTED


@pytest.mark.parametrize("name", ["quantize", "dequantize"])
def test_rows(name):
    assert call(name, k=None) == NULL and call(name, v=None) == NULL
    assert call(name, k=K + 8) == UNSUPPORTED and call(name, v=V + 2) == UNSUPPORTED and call(name, first=FIRST + 1) == UNSUPPORTED
    assert call(name, sh=shape(budgets=None)) == NULL
    assert call(name, sh=shape(budgets=[0, 16])) == BUDGET and call(name, sh=shape(budgets=[32, 65])) == BUDGET
    assert call(name, sh=shape(window=True)) == SHAPE
    assert call(name, sh=shape(d=64)) == UNSUPPORTED
    assert call(name, pg=pages(size=48)) == SHAPE and call(name, pg=pages(per=3)) == SHAPE and call(name, pg=pages(table=None)) == NULL
    # 2^32 threads: 64 rows of a head a workgroup of 256
    assert call(name, sh=shape(n_layers=1, n_q=1, h_q=256, h_kv=256, seq_lens=[60000] * 128, budgets=[60000] * 128)) == UNSUPPORTED


def test_what_a_selection_keeps_does_not_limit_rows():
    """One new token a sequence with the shape of an eviction: refused for the address that is misaligned, not for its budgets."""
    for name in ("quantize", "dequantize"):
        assert call(name, sh=shape(budgets=[1, 1], keep_first=4, keep_last=32), k=K + 8) == UNSUPPORTED


def test_a_workspace_serves_either_kind_of_cache():
    """Sized by jq_attend_workspace_bytes: the call over codes, which shares the work out in its own way, goes on to the address that is
    misaligned."""
    import random
    rng = random.Random(5)
    for _ in range(400):
        h_kv = rng.choice([1, 2, 3, 8, 16, 64])
        sh = jq.Shape(n_layers=rng.choice([1, 1, 2, 7]), seq_lens=[int(2 ** rng.uniform(0, 14)) for _ in range(rng.choice([1, 1, 2, 7, 30, 128]))],
                      n_q=rng.choice([1, 1, 2, 4, 9, 30]), h_q=h_kv * rng.choice([1, 2, 4, 5]), h_kv=h_kv)
        for weights in (False, True):
            if weights and sh.n_q * (sh.h_q // h_kv) > 128:
                continue
            need = jq.attend_workspace_bytes(sh, weights)
            assert call("attend_quantized", sh=sh, q=Q + 8, w=W if weights else None, ws_bytes=need) == UNSUPPORTED, sh


@pytest.mark.parametrize("bits", [(8, 8), (8, 4), (4, 4)])
def test_nothing_may_overlap_what_is_written(bits):
    kb, vb = bits
    rows = 2 * 2 * 164
    sizes = {"k": rows * 16 * kb, "v": rows * 16 * vb, "ks": rows * 4, "vs": rows * 4}
    own = {"k": CK, "v": CV, "ks": KS, "vs": VS}
    for field, n in sizes.items():
        c = codes(kb=kb, vb=vb)
        last = (own[field] + n - 16) & ~15
        assert call("quantize", c=c, k=last) == ALIAS and call("quantize", c=c, v=last) == ALIAS and call("quantize", c=c, first=last) == ALIAS
        assert call("dequantize", c=c, k=last) == ALIAS and call("dequantize", c=c, v=last) == ALIAS
        assert call("attend_quantized", c=c, out=last) == ALIAS and call("attend_quantized", c=c, ws=last) == ALIAS
        assert call("attend_quantized", c=c, lse=last) == ALIAS and call("attend_quantized", c=c, w=last) == ALIAS
        assert call("attend_tree_quantized", c=c, out=last) == ALIAS
    for other in ("v", "ks", "vs"):
        assert call("quantize", c=codes(kb=kb, vb=vb, **{other: CK + 16})) == ALIAS
    assert call("dequantize", k=K, v=K + 2 * 48 * 2 * 256 - 16) == ALIAS
    assert call("quantize", sh=shape(layer_budgets=type("T", (), {"data_ptr": lambda self: CK})())) == ALIAS
    assert call("dequantize", sh=shape(layer_budgets=type("T", (), {"data_ptr": lambda self: K})())) == ALIAS
    assert call("quantize", pg=pages(), first=CK) == ALIAS and call("quantize", pg=pages(table=CV), first=None) == ALIAS


def test_attention():
    assert call("attend_quantized", q=None) == NULL and call("attend_quantized", out=None) == NULL and call("attend_quantized", ws=None) == NULL
    assert call("attend_quantized", ws_bytes=64) == WORKSPACE and call("attend_quantized", ws=WS + 8) == WORKSPACE
    assert call("attend_quantized", sh=shape(n_q=33)) == UNSUPPORTED   # weights of 132 query rows a KV head
    assert call("attend_tree_quantized", seen=None) == NULL and call("attend_tree_quantized", sh=shape(window=True)) == SHAPE
    assert call("attend_tree_quantized", sh=shape(n_q=65)) == SHAPE    # no room for the drafted tokens' rows


def test_the_binding_checks_tensors():
    import torch
    sh = shape()
    c = jq.alloc_codes(sh, 8, 4, device="cpu")
    assert c.K.shape == (2, 2, 164, 128) and c.V.shape == (2, 2, 164, 64) and c.K_scale.shape == c.V_scale.shape == (2, 2, 164, 4)
    assert (c.k_bits, c.v_bits) == (8, 4)
    p = jq.Pages(32, 16, torch.zeros((2, 4), dtype=torch.int32))
    assert jq.alloc_codes(sh, 4, 4, pages=p, device="cpu").K.shape == (2, 16, 2, 32, 64)
    for bad in ((16, 8), (8, 3), (0, 0)):
        with pytest.raises(ValueError):
            jq.alloc_codes(sh, *bad, device="cpu")
    rows = torch.zeros((2, 48, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="not on a GPU"):
        jq.quantize(sh, rows, rows, c)
    with pytest.raises(ValueError, match="not on a GPU"):
        jq.attend_quantized(sh, torch.zeros((2, 2, 4, 8, 128), dtype=torch.bfloat16), c)
    for field, t in (("K", torch.zeros((2, 2, 164, 32), dtype=torch.uint8)), ("V", torch.zeros((2, 2, 163, 128), dtype=torch.uint8)),
                     ("K_scale", torch.zeros((2, 2, 164, 8), dtype=torch.uint8)), ("V_scale", torch.zeros((2, 2, 164, 4), dtype=torch.int8)),
                     ("K", torch.zeros((2, 164, 2, 128), dtype=torch.uint8).transpose(1, 2))):
        d = jq.Codes(c.K, c.V, c.K_scale, c.V_scale)
        setattr(d, field, t)
        with pytest.raises(ValueError, match=field):
            d.c_struct(sh, None, -1)
    for f in (jq.attend_tree_quantized,):
        with pytest.raises(jq.JQError):
            f(sh, None, rows, c)


def _parts(sh, coded):
    """Shares times sequences that a call plans for, out of the bytes of workspace that it asks for: 520 a query row, head and share."""
    lo, hi = 0, 1 << 40
    while lo < hi:
        mid = (lo + hi) // 2
        if coded:
            rc = call("attend_quantized", sh=sh, q=Q + 8, w=None, ws_bytes=mid)
        else:
            rc = jq.lib().jq_attend(ctypes.byref(sh.c_struct()), FIRST, Q + 8, K, V, OUT, LSE, None, WS, mid, None)
        assert rc in (WORKSPACE, UNSUPPORTED)   # (too small, or gone on to the address that is misaligned)
        lo, hi = (mid + 1, hi) if rc == WORKSPACE else (lo, mid)
    return lo // (520 * sh.n_layers * sh.n_q * sh.h_q)


@pytest.mark.parametrize("rows", [33, 36, 48, 64])
@pytest.mark.parametrize("L", [129, 1000, 4096, 9000, 40000])
def test_shares_of_a_wide_sweep_do_not_depend_on_the_cache(rows, L):
    """33 to 64 query rows a KV head take the keys 128 at a time, out of codes as out of bf16: as many workgroups as there are such stages, up
    to one a CU."""
    sh = jq.Shape(n_layers=1, seq_lens=[L], n_q=rows, h_q=8, h_kv=8)
    assert _parts(sh, True) == _parts(sh, False) == -(-L // (128 * max(1, -(-L // (128 * 32)))))

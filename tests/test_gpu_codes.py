"""Rows written into a cache of 8- or 4-bit codes (jq.quantize), read back (jq.dequantize) and attended to (jq.attend_quantized,
jq.attend_tree_quantized), in dense and paged caches, against forms written from the definitions in 64 bits.  Codes, scales and
values read back are exact; attention is held to the bounds of decode_ref over the values that the codes stand for."""
import numpy as np
import pytest

import paper_2509_10798_amd as jq
from codes_ref import bf16_bits, by_head, decode, encode, pages_by_head, random_codes
from decode_ref import attend_ref, bf16, dev_f32, dev_i32, f64, random_tree, to_pages, visible
from parity import from_dev_bf16, to_dev_bf16
from test_gpu_attend import check

pytestmark = pytest.mark.gpu
FORMATS = [(8, 8), (8, 4), (4, 4)]
OLD = 0xA5  # what a cache holds where nothing has been written


def dev_u8(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.uint8)).cuda()


def filled(sh, bits, pages=None):
    c = jq.alloc_codes(sh, *bits, pages=pages)
    for t in (c.K, c.V, c.K_scale, c.V_scale):
        t.fill_(OLD)
    return c


def host(c):
    return [t.cpu().numpy() for t in (c.K, c.V, c.K_scale, c.V_scale)]


def room(seed, caps, page, spare=2):
    """(pages, block table on the host, number of pages) for sequences of these rooms; unused entries -1."""
    rng = np.random.default_rng(seed)
    per = [-(-c // page) for c in caps]
    n = sum(per) + spare
    order = rng.permutation(n)
    table = np.full((len(caps), max(per) + 1), -1, np.int32)
    used = 0
    for s, m in enumerate(per):
        table[s, :m] = order[used:used + m]
        used += m
    return jq.Pages(page, n, dev_i32(table)), table, n


# ---- writing and reading back ---------------------------------------------------------------------------------------
def written(K, V, caps, buds, first, bits, page=0, table=None, n_pages=0, layer_budgets=None):
    """The cache that jq.quantize has to leave: OLD wherever no row goes."""
    nl, _, h, _ = K.shape
    cu, cb = np.concatenate([[0], np.cumsum(caps)]), np.concatenate([[0], np.cumsum(buds)])
    out = []
    for rows, b in ((K, bits[0]), (V, bits[1])):
        codes, scales = encode(rows, b)
        for x in (codes, scales):
            lead = (nl, n_pages, h, page) if page else (nl, h, sum(caps))
            to = np.full(lead + x.shape[-1:], OLD, np.uint8)
            for l in range(nl):
                for s in range(len(caps)):
                    n = buds[s] if layer_budgets is None else max(0, min(buds[s], int(layer_budgets[l, s])))
                    for i in range(n):
                        at = (0 if first is None else int(first[l, s])) + i
                        if not 0 <= at < caps[s]:
                            continue
                        if page:
                            to[l, table[s, at // page], :, at % page] = x[l, cb[s] + i]
                        else:
                            to[l, :, cu[s] + at] = x[l, cb[s] + i]
            out.append(to)
    return out[0], out[2], out[1], out[3]


def keep(seed, nl, caps, buds, h, bits, first=None, page=0, layer_budgets=None, rows=None):
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    print("keep", seed, nl, caps[:8], buds[:8], h, bits, page, flush=True)
    rng = np.random.default_rng(seed)
    if rows is None:
        scale = 2.0 ** rng.integers(-20, 20, (1, 1, h, 128)).astype(np.float64)
        rows = [bf16(rng, nl, sum(buds), h, 128, scale=scale) for _ in range(2)]
    K, V = rows
    lb = None if layer_budgets is None else dev_i32(layer_budgets)
    sh = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h, h_kv=h, pool_k=1, budgets=buds, layer_budgets=lb)
    pages, table, n = room(seed, caps, page) if page else (None, None, 0)
    codes = filled(sh, bits, pages)
    f = None if first is None else dev_i32(first)
    Ko, Vo = (torch.full((nl, sum(buds), h, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if page:
        jq.quantize_paged(sh, pages, to_dev_bf16(K), to_dev_bf16(V), codes, first=f)
        jq.dequantize_paged(sh, pages, codes, first=f, K_out=Ko, V_out=Vo)
    else:
        jq.quantize(sh, to_dev_bf16(K), to_dev_bf16(V), codes, first=f)
        jq.dequantize(sh, codes, first=f, K_out=Ko, V_out=Vo)
    torch.cuda.synchronize()
    got, want = host(codes), written(K, V, caps, buds, first, bits, page, table, n, layer_budgets)
    for name, g, w in zip(("K_scale", "V_scale", "K", "V"), (got[2], got[3], got[0], got[1]), (want[2], want[3], want[0], want[1])):
        bad = np.argwhere(g != w)
        assert not len(bad), "%s: %d bytes, first at %s: %x for %x" % (name, len(bad), bad[0].tolist(), g[tuple(bad[0])], w[tuple(bad[0])])
    cb = np.concatenate([[0], np.cumsum(buds)])
    for x, out, b in ((K, Ko, bits[0]), (V, Vo, bits[1])):
        ref, out = decode(*encode(x, b), b), f64(from_dev_bf16(out))
        for l in range(nl):
            for s in range(len(caps)):
                for i in range(buds[s]):
                    at = (0 if first is None else int(first[l, s])) + i
                    there = 0 <= at < caps[s] and (layer_budgets is None or i < layer_budgets[l, s])
                    np.testing.assert_array_equal(out[l, cb[s] + i], ref[l, cb[s] + i] if there else 7.0)
    return codes


@pytest.mark.parametrize("bits", FORMATS)
def test_every_bf16_value(bits):
    """Each of the 65536 patterns beside values of its own size, beside much larger and smaller ones, and beside what is not finite."""
    p = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    rng = np.random.default_rng(1)
    near = p.reshape(-1, 32)                    # neighbours in size
    far = rng.permutation(p).reshape(-1, 32)    # anything; most groups hold something that is not finite
    finite = rng.permutation(p[(p & 0x7F80) != 0x7F80])
    finite = finite[:len(finite) // 32 * 32].reshape(-1, 32)
    spread = np.stack([np.where(np.arange(32) % 3 == 0, near[i], (near[i] & 0x807F) | np.clip((near[i] >> 7 & 0xFF).astype(int) - np.arange(32), 0, 254).astype(np.uint16) << 7)
                       for i in range(2048)]).astype(np.uint16)
    rows = np.concatenate([near, far, finite, spread])
    rows = rows[:len(rows) // 4 * 4].reshape(1, -1, 1, 128)
    keep(1, 1, [rows.shape[1]], [rows.shape[1]], 1, bits, rows=[rows, rows[:, ::-1].copy()])


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 130])
def test_numbers_of_rows(bits, n):
    keep(n, 2, [n + 3], [n], 2, bits, first=np.array([[0], [3]], np.int32))


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("page", [0, 32, 64])
def test_ragged_rows_behind_those_that_are_there(bits, page):
    caps, buds = [130, 40, 1, 500, 32, 64], [100, 7, 1, 333, 32, 1]
    first = np.array([[30, 33, 0, 0, 0, 63], [0, 0, 0, 167, 0, 5]], np.int32)
    keep(5, 2, caps, buds, 3, bits, first, page)


@pytest.mark.parametrize("page", [0, 32])
def test_rows_for_which_there_is_no_room(page):
    caps, buds = [50, 60, 70, 33, 40], [20, 60, 1, 33, 10]
    first = np.array([[40, -5, 70, -40, 2 ** 31 - 1]], np.int32)
    keep(6, 1, caps, buds, 2, (8, 4), first, page)
    keep(7, 1, caps, buds, 2, (4, 4), np.array([[-2 ** 31, 59, -1, 32, 39]], np.int32), page)


@pytest.mark.parametrize("page", [0, 64])
def test_numbers_that_differ_from_layer_to_layer(page):
    lb = np.array([[20, 0, 5], [-3, 60, 100], [7, 1, 0]], np.int32)
    keep(8, 3, [50, 60, 70], [20, 60, 5], 2, (8, 8), np.array([[1, 0, 2], [0, 0, 65], [30, 59, 0]], np.int32), page, lb)


def test_one_token_of_as_many_sequences_as_a_call_takes():
    caps = [3 + i % 5 for i in range(128)]
    keep(9, 3, caps, [1] * 128, 8, (8, 8), np.array([[(i + l) % 4 for i in range(128)] for l in range(3)], np.int32), 32)
    keep(10, 1, [70 - i % 3 for i in range(128)], [1 + (7 * i) % 60 for i in range(128)], 1, (8, 4))


def test_many_heads():
    keep(11, 1, [40, 9], [33, 2], 256, (8, 4))
    keep(12, 1, [9], [9], 1, (4, 4), page=32)


@pytest.mark.parametrize("bits", FORMATS)
def test_tokens_one_after_the_other_leave_what_one_call_leaves(bits):
    import torch
    rng = np.random.default_rng(13)
    nl, caps, h, n = 2, [40, 33], 2, 20
    K, V = (bf16(rng, nl, 2 * n, h, 128) for _ in range(2))
    bulk = filled(jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h, h_kv=h, budgets=[n, n]), bits)
    jq.quantize(jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h, h_kv=h, budgets=[n, n]), to_dev_bf16(K), to_dev_bf16(V), bulk)
    one = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h, h_kv=h, budgets=[1, 1])
    codes, lens = filled(one, bits), dev_i32(np.zeros((nl, 2)))
    k, v = to_dev_bf16(K), to_dev_bf16(V)
    for i in range(n):
        jq.quantize(one, k[:, [i, n + i]].contiguous(), v[:, [i, n + i]].contiguous(), codes, first=lens)
        lens += 1
    torch.cuda.synchronize()
    for a, b in zip(host(codes), host(bulk)):
        np.testing.assert_array_equal(a, b)


def test_rows_past_31_bits_of_offset():
    """Nine layers of 1.2 million rows of two heads: 2.7 GB of codes each of K and V, of which the last rows of the last layer are written."""
    import torch
    nl, L, h = 9, 1_200_003, 2
    sh = jq.Shape(n_layers=nl, seq_lens=[L], n_q=1, h_q=h, h_kv=h, budgets=[3])
    codes = jq.alloc_codes(sh, 8, 8)
    for t in (codes.K, codes.V, codes.K_scale, codes.V_scale):
        t.zero_()
    rng = np.random.default_rng(14)
    K, V = (bf16(rng, nl, 3, h, 128) for _ in range(2))
    first = dev_i32(np.full((nl, 1), L - 2))
    jq.quantize(sh, to_dev_bf16(K), to_dev_bf16(V), codes, first=first)
    Ko, Vo = jq.dequantize(sh, codes, first=first)
    torch.cuda.synchronize()
    for x, o, c, s in ((K, Ko, codes.K, codes.K_scale), (V, Vo, codes.V, codes.V_scale)):
        want, scales = encode(x, 8)
        np.testing.assert_array_equal(f64(from_dev_bf16(o))[:, :2], decode(want, scales, 8)[:, :2])
        np.testing.assert_array_equal(c[:, :, L - 2:].cpu().numpy(), by_head(want[:, :2]))
        np.testing.assert_array_equal(s[:, :, L - 2:].cpu().numpy(), by_head(scales[:, :2]))
        assert int(c.count_nonzero(dim=-1).count_nonzero()) <= nl * h * 2


# ---- attention ------------------------------------------------------------------------------------------------------
def make(seed, nl, caps, h_q, h_kv, n_q, lens, bits, peak=1.0, dead=True):
    """Random codes; rows that are not live are NaN.  Codes by row [nl, T, h, ..] and the bf16 rows that they stand for."""
    rng = np.random.default_rng(seed)
    T = sum(caps)
    Q = bf16(rng, nl, len(caps), n_q, h_q, 128, scale=peak)
    codes = [random_codes(rng, b, nl, T, h_kv) for b in bits]
    cu = np.concatenate([[0], np.cumsum(caps)])
    live = np.broadcast_to(np.asarray(caps)[None], (nl, len(caps))) if lens is None else np.clip(lens, 0, np.asarray(caps)[None])
    if dead:
        for l in range(nl):
            for s in range(len(caps)):
                for c, sc in codes:
                    sc[l, cu[s] + live[l, s]:cu[s + 1]] = 255
    rows = [bf16_bits(np.nan_to_num(decode(c, s, b), nan=0.0)) for (c, s), b in zip(codes, bits)]
    return rng, Q, codes, rows, cu, live


def on_device(codes, caps, page, seed):
    """(Codes, pages) of codes by row."""
    (ck, sk), (cv, sv) = codes
    if not page:
        return jq.Codes(*(dev_u8(by_head(x)) for x in (ck, cv, sk, sv))), None
    out = []
    for x, fill in ((ck, 0x3C), (cv, 0x3C), (sk, 255), (sv, 255)):
        pool, table = to_pages(np.random.default_rng(seed + 1), x.astype(np.uint16), caps, page, fill=fill)
        out.append(dev_u8(pages_by_head(pool.astype(np.uint8))))
    return jq.Codes(*out), jq.Pages(page, pool.shape[1], dev_i32(table))


def attend(seed, nl, caps, h_q, h_kv, n_q, lens=None, mode="all", page=0, weigh=False, peak=1.0, bits=(8, 8), seen=None):
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    print("attend codes", seed, nl, caps[:8], h_q, h_kv, n_q, mode, page, bits, flush=True)
    rng, Q, codes, (K, V), cu, live = make(seed, nl, caps, h_q, h_kv, n_q, lens, bits, peak)
    sh = jq.Shape(n_layers=nl, seq_lens=caps, n_q=n_q, h_q=h_q, h_kv=h_kv, window=mode == "causal")
    c, pages = on_device(codes, caps, page, seed)
    kw = {"lens": None if lens is None else dev_i32(lens)}
    start = weights = None
    if weigh:
        start = rng.random((nl, h_kv, sum(caps))).astype(np.float32)
        weights = kw["weights"] = dev_f32(start)
    args = (sh,) if pages is None else (sh, pages)
    if mode == "tree":
        seen = np.stack([random_tree(rng, n_q) for _ in caps]) if seen is None else seen
        args += (dev_i32(seen.view(np.int32)),)
        call = jq.attend_tree_quantized if pages is None else jq.attend_tree_quantized_paged
    else:
        call = jq.attend_quantized if pages is None else jq.attend_quantized_paged
    kw["ws"] = jq.alloc_attend_workspace(sh, weights=weigh)
    kw["ws"].fill_(0xFF)
    out, lse = call(*args, to_dev_bf16(Q), c, **kw)
    torch.cuda.synchronize()
    check(Q, K, V, cu, live, out, lse, mode, seen, None, weights, start)


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("L", [1, 2, 16, 31, 32, 33, 64, 127, 128, 129, 255, 257, 1000, 4097])
def test_lengths(bits, L):
    attend(L, 1, [L], 8, 2, 1, weigh=True, bits=bits)


@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (4, 4), (6, 2), (24, 3), (16, 1), (20, 1), (33, 1), (40, 8)])
def test_head_layouts(h_q, h_kv):
    attend(h_q, 1, [333], h_q, h_kv, 1, weigh=True, bits=(8, 4))


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("n_q", [3, 5, 9, 16, 32, 33, 100])   # 12 to 400 query rows a KV head: each way of sharing rows and keys out
@pytest.mark.parametrize("mode", ["all", "causal", "tree"])
def test_several_tokens(bits, n_q, mode):
    attend(n_q, 1, [1200 + n_q, 70 + n_q, 33 + n_q], 8, 2, n_q, mode=mode, weigh=mode != "tree" and n_q <= 32, bits=bits)


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("page", [0, 32, 64, 256])
def test_ragged_batch_partly_filled(bits, page):
    lens = np.array([[0, 1, 77, 500, 31, 64], [130, 0, 100, 499, 32, 1]], np.int32)
    attend(5, 2, [130, 40, 100, 500, 32, 64], 8, 2, 1, lens=lens, page=page, weigh=True, bits=bits)
    attend(6, 2, [130, 40, 100, 500, 32, 64], 8, 2, 17, lens=lens, page=page, mode="causal" if page else "all", bits=bits)


@pytest.mark.parametrize("page", [0, 32])
def test_causal_rows_without_any_key(page):
    attend(7, 1, [40, 64, 33], 8, 2, 9, lens=np.array([[3, 0, 8]], np.int32), mode="causal", page=page, weigh=True, bits=(8, 4))
    attend(8, 2, [50, 64], 8, 2, 20, lens=np.zeros((2, 2), np.int32), bits=(4, 4))


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("n_q", [2, 7, 25, 64])
def test_trees_in_pages(bits, n_q):
    attend(n_q, 1, [300 + n_q, n_q, n_q + 1, 97 + n_q], 8, 2, n_q, mode="tree", page=64, bits=bits)


@pytest.mark.parametrize("peak", [0.0, 8.0, 40.0])
def test_flat_and_peaked(peak):
    attend(15, 1, [2000, 313], 8, 2, 1, peak=peak, weigh=True, bits=(8, 4))


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("n_q", [1, 16])
def test_many_tiles_a_wave(bits, n_q):
    """As many heads as there are CUs: a wave sweeps all of its keys, requested ahead, of lengths that end within them."""
    for L in (700, 769, 991):
        attend(L, 1, [L], 512, 256, n_q // 2 + 1, bits=bits, weigh=True)


@pytest.mark.parametrize("n_q", [1, 16])
def test_ragged_sequences_in_shares_of_several_rounds(n_q):
    """248 (sequence, head) pairs, one of them far longer than the others."""
    caps = [40 + (53 * i) % 400 for i in range(30)] + [6000]
    attend(70, 1, caps, 8, 8, n_q, weigh=True, bits=(8, 8), lens=np.array([[max(c - i, n_q) for i, c in enumerate(caps)]], np.int32), mode="causal" if n_q > 1 else "all")
    attend(71, 1, [c + 3 * n_q for c in caps], 8, 8, 3 * n_q, bits=(4, 4), page=64, mode="tree")  # (room for the drafted tokens' rows)


def test_more_sequences_than_the_chip_takes_at_a_time():
    caps = [5, 2000, 37, 700, 1, 333] * 15
    attend(24, 1, caps, 3, 3, 1, weigh=True, bits=(8, 4), page=32)
    attend(26, 1, [c + 20 for c in caps], 12, 3, 20, mode="tree", bits=(8, 8))


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("n_q", [1, 4, 16, 32, 64])
@pytest.mark.parametrize("mode", ["all", "causal", "tree"])
def test_groups_of_v_that_are_not_finite(bits, n_q, mode):
    """They make NaN of their own dimensions, of the queries that see their row, and of nothing else: all the rest is the bits of a call
    with finite values there."""
    import torch
    n, h_q, h_kv, G = 1003 + n_q, 8, 2, 4
    rng, Q, codes, rows, cu, live = make(100 + n_q, 1, [n], h_q, h_kv, n_q, None, bits)
    sh = jq.Shape(n_layers=1, seq_lens=[n], n_q=n_q, h_q=h_q, h_kv=h_kv, window=mode == "causal")
    seen = random_tree(rng, n_q)
    weigh = mode != "tree" and n_q <= 32

    def call(c):
        if mode == "tree":
            return jq.attend_tree_quantized(sh, dev_i32(seen[None].view(np.int32)), to_dev_bf16(Q), c) + (None,)
        w = torch.ones((1, h_kv, n), device="cuda") if weigh else None
        return jq.attend_quantized(sh, to_dev_bf16(Q), c, weights=w) + (w,)
    clean, _ = on_device(codes, [n], 0, 0)
    ref = call(clean)
    for keys in ((n - 1, 5), (n - 2, n - 1), (77, 300)):
        dirty = jq.Codes(clean.K, clean.V, clean.K_scale, clean.V_scale.clone())
        for key, group in zip(keys, (1, 3)):
            dirty.V_scale[0, 1, key, group] = 255
        got = call(dirty)
        torch.cuda.synchronize()
        assert torch.equal(got[1], ref[1]) and (not weigh or torch.equal(got[2], ref[2]))
        out, was = (f64(from_dev_bf16(x[0]))[0, 0] for x in (got, ref))
        see = visible(mode, n, n_q, G, seen)
        nan = np.zeros((n_q * G, 128), bool)
        for key, group in zip(keys, (1, 3)):
            nan[:, 32 * group:32 * group + 32] |= see[:, key][:, None]
        want = was.copy()
        want[:, G:2 * G] = np.where(nan.reshape(n_q, G, 128), np.nan, want[:, G:2 * G])
        np.testing.assert_array_equal(out, want)


def test_the_same_call_twice_gives_the_same_bits():
    import torch
    rng, Q, codes, rows, cu, live = make(19, 1, [9000, 511], 32, 8, 1, None, (8, 4))
    sh = jq.Shape(n_layers=1, seq_lens=[9000, 511], n_q=1, h_q=32, h_kv=8)
    c, _ = on_device(codes, [9000, 511], 0, 0)
    res = []
    for _ in range(3):
        w = torch.zeros((1, 8, 9511), device="cuda")
        res.append(jq.attend_quantized(sh, to_dev_bf16(Q), c, weights=w) + (w,))
    torch.cuda.synchronize()
    for r in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, res[0]))


def test_long_cache_offsets_past_31_bits():
    """Nine layers of 1.2 million rows of two heads, 2.7 GB of codes each of K and V, whose last row stands out."""
    import torch
    nl, L, h = 9, 1_200_003, 2
    gen = torch.Generator(device="cuda").manual_seed(3)
    sh = jq.Shape(n_layers=nl, seq_lens=[L], n_q=1, h_q=h, h_kv=h)
    c = jq.alloc_codes(sh, 8, 8)
    for t in (c.K, c.V):
        t.random_(0, 0x70, generator=gen)
    for t in (c.K_scale, c.V_scale):
        t.fill_(127 - 5)
    Q = torch.randn((nl, 1, 1, h, 128), generator=gen, device="cuda").to(torch.bfloat16)
    table = torch.tensor(np.concatenate([[(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)]]), device="cuda")
    c.K[-1, :, -1] = torch.where(Q[-1, 0, 0].float() > 0, 0x70, 0xF0).to(torch.uint8)
    out, lse = jq.attend_quantized(sh, Q, c)
    torch.cuda.synchronize()
    for g in range(h):
        code = c.K[-1, g].int()
        k = torch.empty((L, 128), dtype=torch.float64, device="cuda")
        k = table[code & 0x7F] * torch.where(code > 0x7F, -1.0, 1.0) * 2.0 ** -5
        x = (k @ Q[-1, 0, 0, g].double()) / 128 ** 0.5
        p = torch.softmax(x, 0)
        v = table[c.V[-1, g].int()] * 2.0 ** -5
        ref = p @ v
        # (300 roundings of 2^-24 in a row, as for a bf16 cache)
        assert (out[-1, 0, 0, g].double() - ref).abs().max() <= 2.0 ** -8 * ref.abs().max() + 1e-3 * (p @ v.abs()).max()
        assert abs(float(lse[-1, 0, 0, g]) - float(torch.logsumexp(x, 0))) < 1e-4 * max(1.0, float(x.abs().max()))


# ---- together -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("page", [0, 32])
def test_a_prompt_is_pruned_kept_in_codes_and_decoded_on(bits, page):
    """Eviction at the end of a prompt, its pruned cache written into codes, then tokens: each appended as codes, attended to, its
    attention accumulated; at the end the cache is read back and attended to in bf16.  Written and read in captured calls that follow
    lens on the device, with eager work between the replays."""
    import torch
    rng = np.random.default_rng(50)
    nl, prompt, B, h_q, h_kv, steps = 2, [300, 190], [96, 64], 8, 2, 12
    caps = [b + steps for b in B]
    Q, K, V = bf16(rng, nl, 2, 8, h_q, 128), bf16(rng, nl, sum(prompt), h_kv, 128), bf16(rng, nl, sum(prompt), h_kv, 128)
    prune = jq.Shape(n_layers=nl, seq_lens=prompt, n_q=8, h_q=h_q, h_kv=h_kv, budgets=B)
    Ko, Vo, _, _ = jq.evict(prune, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    bulk = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h_q, h_kv=h_kv, budgets=B)
    one = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h_q, h_kv=h_kv, budgets=[1, 1])
    pages = room(3, caps, page)[0] if page else None
    codes = filled(bulk, bits, pages)
    at = lambda sh: (sh,) if pages is None else (sh, pages)
    put = jq.quantize if pages is None else jq.quantize_paged
    look = jq.attend_quantized if pages is None else jq.attend_quantized_paged
    put(*at(bulk), Ko, Vo, codes)
    lens = dev_i32(np.broadcast_to(B, (nl, 2)))
    weights = torch.zeros((nl, h_kv, sum(caps)), device="cuda")
    ws = jq.alloc_attend_workspace(one, weights=True)
    k, v = (torch.zeros((nl, 2, h_kv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((nl, 2, 1, h_q, 128), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((nl, 2, 1, h_q), device="cuda")

    def step():
        put(*at(one), k, v, codes, first=lens)
        lens.add_(1)
        look(*at(one), q, codes, lens=lens, weights=weights, out=out, lse=lse, ws=ws)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                       # warm-up: its row is written again below
    side.synchronize()
    lens.sub_(1)
    weights.zero_()
    with torch.cuda.graph(graph, stream=side):
        step()
    rows = [[from_dev_bf16(x)[:, sum(B[:s]):sum(B[:s]) + B[s]] for s in range(2)] for x in (Ko, Vo)]
    want_w = np.zeros((nl, h_kv, sum(caps)))
    tol_w = np.zeros_like(want_w)
    cu = np.concatenate([[0], np.cumsum(caps)])
    for i in range(steps):
        new = [bf16(rng, nl, 2, n, 128) for n in (h_kv, h_kv, h_q)]
        for t, x in zip((k, v, q), (new[0], new[1], new[2][:, :, None])):
            t.copy_(to_dev_bf16(x))
        graph.replay()
        torch.cuda.synchronize()
        for kv in range(2):
            for s in range(2):
                rows[kv][s] = np.concatenate([rows[kv][s], new[kv][:, s][:, None]], axis=1)
        held = [np.concatenate([np.concatenate([bf16_bits(decode(*encode(r, b), b)), np.zeros((nl, caps[s] - r.shape[1], h_kv, 128), np.uint16)], 1)
                                for s, r in enumerate(rr)], 1) for rr, b in zip(rows, bits)]
        live = np.array([[r.shape[1] for r in rows[0]]] * nl)
        assert lens.cpu().numpy().tolist() == live.tolist()
        check(new[2][:, :, None], held[0], held[1], cu, live, out, lse)
        for l in range(nl):
            for s in range(2):
                for g in range(h_kv):
                    n = live[l, s]
                    _, _, w, _, _, t = attend_ref(f64(new[2][l, s, 4 * g:4 * g + 4]), f64(held[0][l, cu[s]:cu[s] + n, g]), f64(held[1][l, cu[s]:cu[s] + n, g]),
                                                  np.ones((4, n), bool), 128 ** -0.5)
                    want_w[l, g, cu[s]:cu[s] + n] += w
                    tol_w[l, g, cu[s]:cu[s] + n] += t + 2.0 ** -23 * want_w[l, g, cu[s]:cu[s] + n]
    assert (np.abs(weights.cpu().numpy() - want_w) <= tol_w).all()
    whole = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h_q, h_kv=h_kv, budgets=caps)
    Kb, Vb = jq.dequantize(whole, codes) if pages is None else jq.dequantize_paged(whole, pages, codes)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(f64(from_dev_bf16(Kb)), f64(held[0]))
    np.testing.assert_array_equal(f64(from_dev_bf16(Vb)), f64(held[1]))
    out2, lse2 = jq.attend(one, q, Kb, Vb, lens=lens)
    torch.cuda.synchronize()
    check(new[2][:, :, None], held[0], held[1], cu, live, out2, lse2)


def test_two_captured_calls_share_a_workspace():
    import torch
    rng, Q, codes, (K, V), cu, _ = make(20, 1, [700, 300], 8, 2, 1, None, (8, 4))
    sh = jq.Shape(n_layers=1, seq_lens=[700, 300], n_q=1, h_q=8, h_kv=2)
    c, _ = on_device(codes, [700, 300], 0, 0)
    q, lens, ws = to_dev_bf16(Q), dev_i32([[1, 0]]), jq.alloc_attend_workspace(sh, weights=True)
    outs = [(torch.empty_like(q), torch.empty((1, 2, 1, 8), device="cuda"), torch.zeros((1, 2, 1000), device="cuda")) for _ in range(2)]
    graphs, side = [], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o, e, w in outs:
        with torch.cuda.stream(side):
            jq.attend_quantized(sh, q, c, lens=lens, weights=w, out=o, lse=e, ws=ws)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            jq.attend_quantized(sh, q, c, lens=lens, weights=w, out=o, lse=e, ws=ws)
        graphs.append(g)
        w.zero_()
    for n0, n1 in ((1, 0), (5, 300), (333, 31), (700, 1), (0, 299)):
        lens.copy_(dev_i32([[n0, n1]]))
        for g, (o, e, w) in zip(graphs, outs):
            start = w.cpu().numpy()
            g.replay()
            torch.cuda.synchronize()
            check(Q, K, V, cu, np.array([[n0, n1]]), o, e, weights=w, start=start)
            eager = jq.attend_quantized(sh, q, c, lens=lens, ws=ws)
            torch.cuda.synchronize()
            assert torch.equal(eager[0], o) and torch.equal(eager[1], e)


def test_calls_on_another_stream():
    """Temporaries belong to the stream of the call, while the current stream overwrites memory of the same sizes."""
    import torch
    rng, Q, codes, rows, cu, live = make(29, 1, [3000], 16, 4, 1, None, (8, 8))
    sh = jq.Shape(n_layers=1, seq_lens=[3000], n_q=1, h_q=16, h_kv=4, budgets=[500])
    c, _ = on_device(codes, [3000], 0, 0)
    q = to_dev_bf16(Q)
    ref, back = jq.attend_quantized(sh, q, c), jq.dequantize(sh, c)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    for _ in range(20):
        got.append(jq.attend_quantized(sh, q, c, stream=side) + jq.dequantize(sh, c, stream=side))
        torch.empty(jq.attend_workspace_bytes(sh), dtype=torch.uint8, device="cuda").fill_(0xFF)
        torch.full((500 * 4 * 128,), 9.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    for r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, ref + back))


def test_calls_of_several_host_threads():
    import threading
    import torch
    rng, Q, codes, rows, cu, live = make(43, 1, [5000, 77], 16, 4, 1, None, (8, 4))
    shapes = [jq.Shape(n_layers=1, seq_lens=[5000, 77], n_q=1, h_q=16, h_kv=4, budgets=[600, 70]) for _ in range(4)]
    c, _ = on_device(codes, [5000, 77], 0, 0)
    q = to_dev_bf16(Q)
    ref = jq.attend_quantized(shapes[0], q, c) + jq.dequantize(shapes[0], c)
    torch.cuda.synchronize()
    got = [[] for _ in shapes]

    def work(i):
        side = torch.cuda.Stream()
        for _ in range(10):
            got[i].append(jq.attend_quantized(shapes[i], q, c, stream=side) + jq.dequantize(shapes[i], c, stream=side))
        side.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(shapes))]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for r in g for a, b in zip(r, ref)) and all(len(g) == 10 for g in got)


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("n_q", [1, 5])
def test_shares_from_one_tile_a_wave_to_many(bits, n_q):
    """Workgroups of four and of eight waves, one launch and two, lengths that end inside a tile, inside a turn and at its end."""
    for L in (255, 1279, 3000, 8191, 8192 + 257, 20011):
        attend(L, 1, [L], 8, 2, n_q, bits=bits, mode="causal" if n_q > 1 else "all", weigh=True)
    attend(7, 1, [9000, 300, 5000], 4, 1, n_q, bits=bits, lens=np.array([[8997, 0, 31]], np.int32), weigh=True, page=32)


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("below,beyond", [(-1, 9), (-2 ** 31, 2 ** 31 - 1)])
def test_rows_whose_page_is_not_handed_out(bits, below, beyond):
    """Rows within a sequence's room whose page the block table does not name yet: neither written, over whoever has the first or the last
    page of the pool, nor read."""
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    nl, h, page, n, caps, buds, first = 2, 3, 32, 9, [96, 64, 96], [40, 10, 30], [[20, 0, 60], [30, 3, 64]]
    table = np.array([[3, below, 8], [5, 0, -1], [6, 4, beyond]], np.int32)   # (rows of pages 0 and 8 are nobody's to write in this call)
    rng = np.random.default_rng(70)
    rows = [bf16(rng, nl, sum(buds), h, 128) for _ in range(2)]
    sh = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h, h_kv=h, pool_k=1, budgets=buds)
    pages, f = jq.Pages(page, n, dev_i32(table)), dev_i32(first)
    codes = filled(sh, bits, pages)
    outs = [torch.full((nl, sum(buds), h, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    print("not handed out", bits, below, beyond, flush=True)
    jq.quantize_paged(sh, pages, *(to_dev_bf16(x) for x in rows), codes, first=f)
    jq.dequantize_paged(sh, pages, codes, first=f, K_out=outs[0], V_out=outs[1])
    torch.cuda.synchronize()
    got = host(codes)
    for x, out, b, g, gs in zip(rows, outs, bits, got[:2], got[2:]):
        c, scales = encode(x, b)
        ref = decode(c, scales, b)
        want, want_s, want_out = (np.full(y.shape, v, y.dtype) for y, v in ((g, OLD), (gs, OLD), (ref, 7.0)))
        for l in range(nl):
            i = 0
            for s in range(3):
                for at in range(first[l][s], first[l][s] + buds[s]):
                    if at < caps[s] and 0 <= table[s, at // page] < n:
                        want[l, table[s, at // page], :, at % page], want_s[l, table[s, at // page], :, at % page] = c[l, i], scales[l, i]
                        want_out[l, i] = ref[l, i]
                    i += 1
        np.testing.assert_array_equal(gs, want_s)
        np.testing.assert_array_equal(g, want)
        np.testing.assert_array_equal(f64(from_dev_bf16(out)), want_out)


@pytest.mark.parametrize("caps,h,n_q", [([4000, 90, 1500, 700, 2500, 33], 2, 2), ([900], 2, 1), ([40, 300], 4, 1), ([700, 5000, 260], 2, 12)])
def test_calls_over_either_kind_of_cache_in_turn_on_one_workspace(caps, h, n_q):
    """Eager and captured, with weights and without: the two kinds lay the workspace out in their own ways, and neither leaves there what
    misleads the other."""
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    print("in turn", caps, h, n_q, flush=True)
    rng = np.random.default_rng(80)
    K, V = (to_dev_bf16(bf16(rng, 1, sum(caps), h, 128)) for _ in range(2))
    sh = jq.Shape(n_layers=1, seq_lens=caps, n_q=n_q, h_q=4 * h, h_kv=h, pool_k=1, budgets=caps)
    codes = jq.quantize(sh, K, V, jq.alloc_codes(sh))
    Q = to_dev_bf16(bf16(rng, 1, len(caps), n_q, 4 * h, 128))

    def call(kind, weigh, ws):
        w = torch.zeros((1, h, sum(caps)), device="cuda") if weigh else None
        o = jq.attend(sh, Q, K, V, weights=w, ws=ws) if kind == "rows" else jq.attend_quantized(sh, Q, codes, weights=w, ws=ws)
        return o if w is None else o + (w,)
    kinds = [(k, w) for k in ("rows", "codes") for w in (False, True)]
    want = [call(*x, jq.alloc_attend_workspace(sh, weights=x[1]).fill_(0xFF)) for x in kinds]
    ws = jq.alloc_attend_workspace(sh, weights=True).fill_(0xFF)
    torch.cuda.synchronize()
    same = lambda got, ref: all(torch.equal(a, b) for a, b in zip(got, ref))
    for _ in range(3):
        got = [call(*x, ws) for x in kinds]
        torch.cuda.synchronize()
        assert all(map(same, got, want))
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    for x in kinds:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = call(*x, ws)
        graphs.append((g, got))
    torch.cuda.synchronize()
    for _ in range(4):
        for (g, got), ref, x in zip(graphs, want, kinds):
            g.replay()
            torch.cuda.synchronize()
            assert same(got, ref), x
            eager = [call(*y, ws) for y in reversed(kinds)]
            torch.cuda.synchronize()
            assert all(map(same, eager, reversed(want))), x

"""Eviction by accumulated attention weight (jq.evict_weight, jq.replace_lightest and their paged forms) against plain Python:
exact, whatever the weights, ties included; and the calls together as a decoding loop uses them."""
import numpy as np
import pytest

import paper_2509_10798_amd as jq
from decode_ref import attend_ref, bf16, dev_f32, dev_i32, evict_order, f64, from_pages, lightest, to_pages
from parity import from_dev_bf16, to_dev_bf16

pytestmark = pytest.mark.gpu


def cache(seed, nl, caps, h_kv, ties=False, order="ascending"):
    rng = np.random.default_rng(seed)
    T = sum(caps)
    K, V = bf16(rng, nl, T, h_kv, 128), bf16(rng, nl, T, h_kv, 128)
    w = rng.exponential(size=(nl, h_kv, T)).astype(np.float32)
    if ties:
        w = np.floor(w * 4).astype(np.float32)
        w[w == 0] = np.where(rng.random((w == 0).sum()) < 0.5, -0.0, 0.0)
    pos = np.cumsum(rng.integers(1, 4, (nl, h_kv, T)), axis=2).astype(np.int32)
    if order == "scrambled":
        pos = np.take_along_axis(pos, rng.random(pos.shape).argsort(-1), -1)
    return rng, K, V, w, pos


def evict(seed, nl, caps, budgets, h_kv, lens=None, page=0, inplace=False, first=0, last=0, ties=False, order="ascending", with_pos=True,
          layer_budgets=None):
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    print("evict", seed, nl, caps, budgets, page, inplace, flush=True)
    rng, K, V, w, pos = cache(seed, nl, caps, h_kv, ties, order)
    cu, cb = np.concatenate([[0], np.cumsum(caps)]), np.concatenate([[0], np.cumsum(budgets)])
    live = np.broadcast_to(np.asarray(caps)[None], (nl, len(caps))) if lens is None else np.clip(lens, 0, np.asarray(caps)[None])
    sh = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h_kv, h_kv=h_kv, budgets=budgets, keep_first=first, keep_last=last,
                  layer_budgets=None if layer_budgets is None else dev_i32(layer_budgets))
    k, v = K, V
    at = (sh,)
    if page:
        k, table = to_pages(np.random.default_rng(seed + 1), K, caps, page)
        v, _ = to_pages(np.random.default_rng(seed + 1), V, caps, page)
        at = (sh, jq.Pages(page, k.shape[1], dev_i32(table)))
    kd, vd, wd, pd = to_dev_bf16(k), to_dev_bf16(v), dev_f32(w), dev_i32(pos) if with_pos else None
    idx = torch.full((nl, h_kv, sum(budgets)), -7, dtype=torch.int32, device="cuda")
    kw = {"lens": None if lens is None else dev_i32(lens), "idx_out": idx}
    marked = rng.integers(0, 2 ** 15, k.shape).astype(np.uint16)  # what a second cache held before
    if not inplace:
        kw.update(K_out=to_dev_bf16(marked), V_out=to_dev_bf16(marked), weights_out=torch.full_like(wd, -5), pos_out=torch.full_like(dev_i32(pos), -9))
    Ko, Vo, wo, po, idx = (jq.evict_weight_paged if page else jq.evict_weight)(*at, kd, vd, wd, pd, **kw)
    torch.cuda.synchronize()
    for got, src in ((Ko, K), (Vo, V)):
        got = from_dev_bf16(got)
        if page:
            pool_before = (marked if not inplace else (k if src is K else v))
            owned = np.zeros(got.shape[1:3], bool)
            for s, c in enumerate(caps):
                j = np.arange(c)
                owned[table[s, j // page], j % page] = True
            np.testing.assert_array_equal(got[:, ~owned], pool_before[:, ~owned])  # nobody's rows are left alone
            got, was = from_pages(got, table, caps, page), from_pages(pool_before, table, caps, page)
        else:
            was = src if inplace else marked
        want = was.copy()
        for l in range(nl):
            for s in range(len(caps)):
                for g in range(h_kv):
                    n = int(live[l, s])
                    B = budgets[s] if layer_budgets is None else int(np.clip(layer_budgets[l, s], max(1, first + last), budgets[s]))
                    p = pos[l, g, cu[s]:cu[s + 1]] if with_pos else np.arange(caps[s])
                    kept = evict_order(w[l, g, cu[s]:cu[s + 1]], p, n, B, first, last)
                    m = kept.size
                    want[l, cu[s]:cu[s] + m, g] = src[l, cu[s] + kept, g]
                    if got is not None and src is K:
                        i = idx[l, g, cb[s]:cb[s + 1]].cpu().numpy()
                        np.testing.assert_array_equal(i[:m], kept)
                        assert (i[m:] == -7).all()
                        x = wo[l, g, cu[s]:cu[s + 1]].cpu().numpy()
                        np.testing.assert_array_equal(x[:m], w[l, g, cu[s] + kept])
                        rest = w[l, g, cu[s] + m:cu[s + 1]] if inplace else np.full(caps[s] - m, -5, np.float32)
                        np.testing.assert_array_equal(x[m:], rest)
                        if with_pos:
                            x = po[l, g, cu[s]:cu[s + 1]].cpu().numpy()
                            np.testing.assert_array_equal(x[:m], p[kept])
                            np.testing.assert_array_equal(x[m:], p[m:] if inplace else np.full(caps[s] - m, -9))
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("L,B", [(1, 1), (2, 1), (63, 62), (64, 64), (1023, 7), (1024, 1000), (1025, 1024), (2500, 2048), (5000, 300)])
def test_lengths_and_budgets(L, B, inplace):
    evict(L, 1, [L], [B], 2, inplace=inplace)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("page", [0, 32, 64])
def test_ragged_partly_filled(page, inplace):
    lens = np.array([[300, 0, 17, 1000, 1], [128, 50, 40, 333, 64]], np.int32)
    evict(3, 2, [300, 50, 40, 1000, 64], [100, 50, 16, 700, 1], 3, lens=lens, page=page, inplace=inplace)


@pytest.mark.parametrize("inplace", [False, True])
def test_ties_go_to_lower_rows(inplace):
    evict(4, 2, [1500, 700], [600, 350], 2, ties=True, inplace=inplace)


@pytest.mark.parametrize("order", ["ascending", "scrambled"])
@pytest.mark.parametrize("with_pos", [True, False])
def test_sinks_and_newest_stay(order, with_pos):
    evict(5, 1, [900, 400], [100, 40], 2, first=4, last=32, order=order, with_pos=with_pos, inplace=True)


def test_budget_of_protected_rows_alone():
    evict(6, 1, [500], [36], 2, first=4, last=32, with_pos=False)


def test_budgets_per_layer_are_clamped():
    lb = np.array([[10, 300], [-4, 100000]], np.int32)
    evict(7, 2, [300, 400], [128, 256], 2, layer_budgets=lb, first=2, last=3, inplace=True)


def test_all_positions_protected_by_mistake():
    """Positions that repeat, so that more rows are protected than the budget holds: exactly the budget's rows stay, the lowest."""
    import torch
    rng, K, V, w, _ = cache(8, 1, [300], 1)
    pos = np.full((1, 1, 300), 5, np.int32)
    sh = jq.Shape(n_layers=1, seq_lens=[300], n_q=1, h_q=1, h_kv=1, budgets=[64], keep_last=2)
    *_, idx = jq.evict_weight(sh, to_dev_bf16(K), to_dev_bf16(V), dev_f32(w), dev_i32(pos))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(idx[0, 0].cpu().numpy(), np.arange(64))


@pytest.mark.parametrize("kind", ["inf", "negative", "denormal"])
def test_extreme_weights(kind):
    import torch
    rng, K, V, w, pos = cache(9, 1, [800], 2)
    if kind == "inf":
        w[rng.random(w.shape) < 0.1] = np.inf
    elif kind == "negative":
        w -= 1
    else:
        w = (w * 1e-42).astype(np.float32)
    sh = jq.Shape(n_layers=1, seq_lens=[800], n_q=1, h_q=2, h_kv=2, budgets=[333])
    *_, idx = jq.evict_weight(sh, to_dev_bf16(K), to_dev_bf16(V), dev_f32(w), dev_i32(pos))
    torch.cuda.synchronize()
    for g in range(2):
        np.testing.assert_array_equal(idx[0, g].cpu().numpy(), evict_order(w[0, g], pos[0, g], 800, 333, 0, 0))


def test_long_sequence_keeps_the_same_rows_as_the_plain_selection():
    import torch
    L, B = 200_001, 2048
    rng = np.random.default_rng(10)
    w = rng.exponential(size=(1, 2, L)).astype(np.float32)
    K, V = bf16(rng, 1, L, 2, 128), bf16(rng, 1, L, 2, 128)
    sh = jq.Shape(n_layers=1, seq_lens=[L], n_q=1, h_q=2, h_kv=2, budgets=[B])
    kd, vd, wd = to_dev_bf16(K), to_dev_bf16(V), dev_f32(w)
    plain = jq.select_topk(sh, wd)
    Ko, Vo, wo, _, idx = jq.evict_weight(sh, kd, vd, wd, K_out=torch.empty_like(kd), V_out=torch.empty_like(vd), weights_out=torch.empty_like(wd))
    torch.cuda.synchronize()
    assert torch.equal(plain, idx)
    for g in range(2):
        i = idx[0, g].cpu().numpy()
        np.testing.assert_array_equal(from_dev_bf16(Ko)[0, :B, g], K[0, i, g])
        np.testing.assert_array_equal(from_dev_bf16(Vo)[0, :B, g], V[0, i, g])
        np.testing.assert_array_equal(wo[0, g, :B].cpu().numpy(), w[0, g, i])


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("with_pos", [True, False])
def test_sequences_selected_in_pieces(inplace, with_pos):
    """Long sequences beside short ones, ties, protected rows of either end; live counts at the pieces' edges."""
    caps, budgets = [40000, 300, 33000, 70001], [900, 200, 64, 1500]
    lens = np.array([[40000, 300, 16384, 70001], [16385, 10, 32768, 65537]], np.int32)
    evict(13, 2, caps, budgets, 1, lens=lens, inplace=inplace, first=3, last=20, ties=True, order="scrambled" if with_pos else "ascending",
          with_pos=with_pos)


def test_a_sequence_of_many_pieces():
    evict(16, 1, [150_001, 16_385], [700, 90], 1, inplace=True, first=3, last=70, order="scrambled")


@pytest.mark.parametrize("first,last", [(0, 0), (3, 0), (0, 5), (3, 5)])
@pytest.mark.parametrize("L", [700, 40_000])
def test_positions_at_the_ends_of_their_type(L, first, last):
    import torch
    rng, K, V, w, pos = cache(17, 1, [L], 1, order="scrambled")
    at = rng.permutation(L)
    pos[0, 0, at[:6]] = np.array([2 ** 31 - 1, 2 ** 31 - 2, -1, -2 ** 31, -2 ** 31 + 1, 2 ** 31 - 7], np.int64).astype(np.int32)
    for p in (pos, np.minimum(pos, 9), np.where(pos < 0, pos, -2 ** 31).astype(np.int32)):  # of the last, more are protected than stay
        sh = jq.Shape(n_layers=1, seq_lens=[L], n_q=1, h_q=1, h_kv=1, budgets=[100], keep_first=first, keep_last=last)
        *_, idx = jq.evict_weight(sh, to_dev_bf16(K), to_dev_bf16(V), dev_f32(w), dev_i32(p))
        torch.cuda.synchronize()
        q = p[0, 0].astype(np.int64)
        stay = np.flatnonzero((q < first) | (q > q.max() - last))
        want = stay[:100] if stay.size > 100 else evict_order(w[0, 0], q, L, 100, first, last)
        np.testing.assert_array_equal(idx[0, 0].cpu().numpy(), want)


def test_long_sequence_that_keeps_most_of_its_rows():
    evict(14, 1, [40000], [30000], 1, inplace=True, first=2, last=5)
    evict(15, 1, [40000], [30000], 1, ties=True, page=64, lens=np.array([[33333]], np.int32))


@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("first,last", [(0, 0), (4, 16)])
def test_replace(page, first, last):
    import torch
    nl, caps, h_kv = 2, [64, 300, 33, 1025], 3
    rng, K, V, w, pos = cache(11, nl, caps, h_kv, ties=True, order="scrambled")
    cu = np.concatenate([[0], np.cumsum(caps)])
    lens = np.array([[64, 299, 33, 1025], [0, 300, 5, 1025]], np.int32)
    token = np.array([500, 1500, 400, 4000], np.int32)
    kn, vn = bf16(rng, nl, 4, h_kv, 128), bf16(rng, nl, 4, h_kv, 128)
    sh = jq.Shape(n_layers=nl, seq_lens=caps, n_q=1, h_q=h_kv, h_kv=h_kv, keep_first=first, keep_last=last)
    k, v, at = K, V, (sh,)
    if page:
        k, table = to_pages(np.random.default_rng(1), K, caps, page, fill=0)
        v, _ = to_pages(np.random.default_rng(1), V, caps, page, fill=0)
        at = (sh, jq.Pages(page, k.shape[1], dev_i32(table)))
    kd, vd, wd, pd = to_dev_bf16(k), to_dev_bf16(v), dev_f32(w), dev_i32(pos)
    slot = (jq.replace_lightest_paged if page else jq.replace_lightest)(*at, to_dev_bf16(kn), to_dev_bf16(vn), dev_i32(token), kd, vd, wd, pd,
                                                                          lens=dev_i32(lens))
    torch.cuda.synchronize()
    slot = slot.cpu().numpy()
    for l in range(nl):
        for s, c in enumerate(caps):
            for g in range(h_kv):
                n = int(lens[l, s])
                j = n if n < c else lightest(w[l, g, cu[s]:cu[s + 1]], pos[l, g, cu[s]:cu[s + 1]], n, token[s], first, last)
                assert slot[l, s, g] == j
                K[l, cu[s] + j, g], V[l, cu[s] + j, g] = kn[l, s, g], vn[l, s, g]
                w[l, g, cu[s] + j], pos[l, g, cu[s] + j] = 0, token[s]
    got_k, got_v = from_dev_bf16(kd), from_dev_bf16(vd)
    if page:
        got_k, got_v = from_pages(got_k, table, caps, page), from_pages(got_v, table, caps, page)
    np.testing.assert_array_equal(got_k, K)
    np.testing.assert_array_equal(got_v, V)
    np.testing.assert_array_equal(wd.cpu().numpy(), w)
    np.testing.assert_array_equal(pd.cpu().numpy(), pos)


@pytest.mark.parametrize("page", [0, 32])
def test_a_decoding_loop(page):
    """A prompt evicted to its budget by its soft tokens, then tokens decoded one by one: each takes the place of the row that
    has received least attention, attends over the cache and adds to the weights; at last the cache is evicted to fewer rows.
    Every step is compared with 64-bit arithmetic on the state as it stands on the device."""
    import torch
    h_q, h_kv, d, L, B, cap, n_soft = 8, 2, 128, 700, 96, 100, 8
    G = h_q // h_kv
    rng = np.random.default_rng(12)
    K, V = bf16(rng, 1, L + n_soft, h_kv, d), bf16(rng, 1, L + n_soft, h_kv, d)
    Q = bf16(rng, 1, 1, n_soft, h_q, d)
    kd, vd, qd = to_dev_bf16(K), to_dev_bf16(V), to_dev_bf16(Q)
    # the soft tokens' own attention, which leaves the normalisers of a one-pass eviction
    soft = jq.Shape(n_layers=1, seq_lens=[L + n_soft], n_q=n_soft, h_q=h_q, h_kv=h_kv, window=True)
    _, lse = jq.attend(soft, qd, kd, vd)
    prompt = jq.Shape(n_layers=1, seq_lens=[L], n_q=n_soft, h_q=h_q, h_kv=h_kv, budgets=[B], keep_first=2, keep_last=4)
    pk, pv = kd[:, :L].contiguous(), vd[:, :L].contiguous()
    Ko, Vo, idx, pooled = jq.evict(prompt, qd, pk, pv, lse=lse)
    _, _, idx2, pooled2 = jq.evict(prompt, qd, pk, pv, k_tail=kd[:, L:].view(1, 1, n_soft, h_kv, d).contiguous())
    torch.cuda.synchronize()
    # the same normalisers either way, each within the bounds of a sum over 708 keys
    assert (pooled - pooled2).abs().max() <= 1e-5 * pooled2.abs().max()
    sh = jq.Shape(n_layers=1, seq_lens=[cap], n_q=1, h_q=h_q, h_kv=h_kv, keep_first=2, keep_last=4)
    at = (sh,)
    table = None
    kc, vc = torch.zeros((1, cap, h_kv, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, cap, h_kv, d), dtype=torch.bfloat16, device="cuda")
    kc[:, :B], vc[:, :B] = Ko, Vo
    if page:
        kp, table = to_pages(np.random.default_rng(2), from_dev_bf16(kc), [cap], page, fill=0)
        vp, _ = to_pages(np.random.default_rng(2), from_dev_bf16(vc), [cap], page, fill=0)
        kc, vc = to_dev_bf16(kp), to_dev_bf16(vp)
        at = (sh, jq.Pages(page, kp.shape[1], dev_i32(table)))
    pos = torch.zeros((1, h_kv, cap), dtype=torch.int32, device="cuda")
    pos[:, :, :B] = idx
    w = torch.zeros((1, h_kv, cap), device="cuda")
    w[:, :, :B] = torch.gather(pooled, 2, idx.long())
    lens, token = dev_i32([[B]]), dev_i32([L])
    taken = []

    def rows(x):
        x = from_dev_bf16(x)
        return f64(from_pages(x, table, [cap], page) if page else x)[0]
    for step in range(12):
        kn, vn, q = (to_dev_bf16(bf16(rng, 1, 1, h, d)) for h in (h_kv, h_kv, h_q))
        slot = (jq.replace_lightest_paged if page else jq.replace_lightest)(*at, kn, vn, token, kc, vc, w, pos, lens=lens)
        lens.add_(1).clamp_(max=cap)
        before = w.clone()
        out, e = (jq.attend_paged if page else jq.attend)(*at, q.view(1, 1, 1, h_q, d), kc, vc, lens=lens, weights=w)
        torch.cuda.synchronize()
        n = int(lens[0, 0])
        assert n == min(B + step + 1, cap)
        k, v = rows(kc), rows(vc)
        for g in range(h_kv):
            ro, rl, rw, to, tl, tw = attend_ref(f64(from_dev_bf16(q))[0, 0, g * G:(g + 1) * G], k[:n, g], v[:n, g], np.ones((G, n), bool), d ** -0.5)
            assert (np.abs(f64(from_dev_bf16(out))[0, 0, 0, g * G:(g + 1) * G] - ro) <= to).all()
            assert (np.abs(e[0, 0, 0, g * G:(g + 1) * G].cpu().numpy() - rl) <= tl).all()
            grown = w[0, g, :n].cpu().numpy().astype(np.float64) - before[0, g, :n].cpu().numpy()
            assert (np.abs(grown - rw) <= tw + 2.0 ** -22 * w[0, g, :n].cpu().numpy()).all()
            assert int(pos[0, g, int(slot[0, 0, g])]) == L + step
        taken.append(slot.cpu().numpy().ravel())
        token.add_(1)
    assert (np.stack(taken)[:4] == np.arange(B, cap)[:, None]).all()   # first the room that is left
    newest = pos.amax(-1)
    assert (newest == L + 11).all()
    few = jq.Shape(n_layers=1, seq_lens=[cap], n_q=1, h_q=h_q, h_kv=h_kv, budgets=[40], keep_first=2, keep_last=4)
    wh, ph, kh = w.cpu().numpy().copy(), pos.cpu().numpy().copy(), rows(kc)
    at = (few,) + at[1:]
    (jq.evict_weight_paged if page else jq.evict_weight)(*at, kc, vc, w, pos, lens=lens)
    torch.cuda.synchronize()
    for g in range(h_kv):
        kept = evict_order(wh[0, g], ph[0, g], cap, 40, 2, 4)
        np.testing.assert_array_equal(rows(kc)[:40, g], kh[kept, g])
        np.testing.assert_array_equal(pos[0, g, :40].cpu().numpy(), ph[0, g, kept])
        assert set(range(L + 8, L + 12)) <= set(pos[0, g, :40].tolist())


@pytest.mark.parametrize("page", [0, 64])
def test_a_captured_decoding_step_replayed(page):
    """Replacement, attention of the token and of a drafted tree, then eviction, as two captured graphs that share their workspaces:
    every replay leaves the bits that the same calls leave eagerly on a copy of the state."""
    import torch
    h_q, h_kv, cap, n_draft = 8, 2, 300, 6
    rng = np.random.default_rng(50)
    K, V = bf16(rng, 1, cap, h_kv, 128), bf16(rng, 1, cap, h_kv, 128)
    pages = ()
    if page:
        K, table = to_pages(np.random.default_rng(3), K, [cap], page, fill=0)
        V, _ = to_pages(np.random.default_rng(3), V, [cap], page, fill=0)
        pages = (jq.Pages(page, K.shape[1], dev_i32(table)),)
    step = jq.Shape(n_layers=1, seq_lens=[cap], n_q=1, h_q=h_q, h_kv=h_kv, keep_first=2, keep_last=8)
    tree = jq.Shape(n_layers=1, seq_lens=[cap], n_q=n_draft, h_q=h_q, h_kv=h_kv)
    few = jq.Shape(n_layers=1, seq_lens=[cap], n_q=1, h_q=h_q, h_kv=h_kv, budgets=[200], keep_first=2, keep_last=8)
    kn, vn, q = (to_dev_bf16(bf16(rng, 1, 1, h, 128)) for h in (h_kv, h_kv, h_q))
    qt = to_dev_bf16(bf16(rng, 1, 1, n_draft, h_q, 128))
    from decode_ref import random_tree
    seen = dev_i32(random_tree(rng, n_draft)[None].view(np.int32))
    ws = jq.alloc_attend_workspace(step, weights=True), jq.alloc_attend_workspace(tree), jq.alloc_evict_weight_workspace(few)
    rep, att, atree, ev = ((jq.replace_lightest_paged, jq.attend_paged, jq.attend_tree_paged, jq.evict_weight_paged) if page else
                           (jq.replace_lightest, jq.attend, jq.attend_tree, jq.evict_weight))

    def state():
        s = {"K": to_dev_bf16(K), "V": to_dev_bf16(V), "w": torch.linspace(0.1, 3, h_kv * cap, device="cuda").view(1, h_kv, cap).flip(-1).contiguous(),
             "pos": torch.arange(cap, dtype=torch.int32, device="cuda").expand(1, h_kv, cap).contiguous(), "lens": dev_i32([[cap - 3]]),
             "token": dev_i32([cap]), "slot": torch.zeros((1, 1, h_kv), dtype=torch.int32, device="cuda"), "out": torch.zeros_like(q.view(1, 1, 1, h_q, 128)),
             "lse": torch.zeros((1, 1, 1, h_q), device="cuda"), "tout": torch.zeros_like(qt), "tlse": torch.zeros((1, 1, n_draft, h_q), device="cuda"),
             "idx": torch.zeros((1, h_kv, 200), dtype=torch.int32, device="cuda")}
        return s

    def decode(s):
        rep(step, *pages, kn, vn, s["token"], s["K"], s["V"], s["w"], s["pos"], lens=s["lens"], slot_out=s["slot"])
        s["lens"].add_(1).clamp_(max=cap)
        att(step, *pages, q.view(1, 1, 1, h_q, 128), s["K"], s["V"], lens=s["lens"], weights=s["w"], out=s["out"], lse=s["lse"], ws=ws[0])
        atree(tree, *pages, seen, qt, s["K"], s["V"], lens=s["lens"], out=s["tout"], lse=s["tlse"], ws=ws[1])
        s["token"].add_(1)

    def prune(s):
        ev(few, *pages, s["K"], s["V"], s["w"], s["pos"], lens=s["lens"], idx_out=s["idx"], ws=ws[2])
        s["lens"].clamp_(max=200)
    side = torch.cuda.Stream()
    warm = state()
    with torch.cuda.stream(side):
        decode(warm), prune(warm)
    side.synchronize()
    a, b = state(), state()
    graphs = []
    for f in (decode, prune):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            f(a)
        graphs.append(g)
    torch.cuda.synchronize()
    for i, which in enumerate((0, 0, 0, 0, 0, 0, 1, 0, 0, 1, 0)):
        graphs[which].replay()
        torch.cuda.synchronize()
        (decode, prune)[which](b)
        torch.cuda.synchronize()
        for name in a:
            x, y = a[name], b[name]
            assert torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x, y.view(torch.int16) if y.dtype == torch.bfloat16 else y), (i, name)


def test_offsets_past_32_bits():
    """Two sequences of more than 2 GiB of keys each: their last rows are attended to by many query rows, appended and kept."""
    import torch
    caps, h_kv, h_q, n_q, B = [1_200_003, 1_100_001], 8, 32, 10, 8
    T = sum(caps)
    K = torch.zeros((1, T, h_kv, 128), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    w, pos = torch.zeros((1, h_kv, T), device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda").expand(1, h_kv, T).contiguous()
    gen = torch.Generator(device="cuda").manual_seed(18)
    new = [torch.randn((1, 2, h_kv, 128), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    new[0].fill_(4.0)
    cu = [0, caps[0], T]
    lens = torch.tensor([[c - 1 for c in caps]], dtype=torch.int32, device="cuda")
    token = torch.tensor([2 ** 30, 2 ** 30 + 1], dtype=torch.int32, device="cuda")
    sh = jq.Shape(n_layers=1, seq_lens=caps, n_q=n_q, h_q=h_q, h_kv=h_kv, budgets=[B, B])
    slot = jq.replace_lightest(sh, *new, token, K, V, w, pos, lens=lens)
    # scores: 45 for the new row, 0 for the others, which together weigh 4e-14 of it
    Q = torch.ones((1, 2, n_q, h_q, 128), dtype=torch.bfloat16, device="cuda")
    out, lse = jq.attend(sh, Q, K, V, weights=w)
    torch.cuda.synchronize()
    for s in range(2):
        assert (slot[0, s] == caps[s] - 1).all()
        assert torch.equal(K[0, cu[s + 1] - 1], new[0][0, s]) and torch.equal(V[0, cu[s + 1] - 1], new[1][0, s])
        assert (pos[0, :, cu[s + 1] - 1] == 2 ** 30 + s).all()
        want = new[1][0, s].repeat_interleave(h_q // h_kv, 0).expand(n_q, h_q, 128)
        assert torch.equal(out[0, s], want)
        assert (lse[0, s] - 4 * 128 / 128 ** 0.5).abs().max() < 1e-4
        assert (w[0, :, cu[s + 1] - 1] - n_q * h_q // h_kv).abs().max() < 1e-3
    last = torch.arange(B, device="cuda")
    for s in range(2):  # the last rows stand out, and stay
        K[0, cu[s + 1] - B:cu[s + 1]] = (1 + last + 100 * s).to(torch.bfloat16)[:, None, None]
        V[0, cu[s + 1] - B:cu[s + 1]] = -(1 + last + 100 * s).to(torch.bfloat16)[:, None, None]
        w[0, :, cu[s + 1] - B:cu[s + 1]] = 50.0 + last
    *_, idx = jq.evict_weight(sh, K, V, w, pos)
    torch.cuda.synchronize()
    for s in range(2):
        assert torch.equal(idx[0, :, s * B:(s + 1) * B], (caps[s] - B + last).to(torch.int32).expand(h_kv, B))
        rows = (1 + last + 100 * s).to(torch.bfloat16)[:, None, None].expand(B, h_kv, 128)
        assert torch.equal(K[0, cu[s]:cu[s] + B], rows) and torch.equal(V[0, cu[s]:cu[s] + B], -rows)
        assert not K[0, cu[s] + B:cu[s + 1] - B].any()

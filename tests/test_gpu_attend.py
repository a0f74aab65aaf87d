"""Attention over a pruned cache (jq.attend, jq.attend_tree and their paged forms) against a 64-bit form written from the
definition, at the lengths, head layouts and masks where it can go wrong.  Everything that must not be read holds NaN."""
import numpy as np
import pytest

import paper_2509_10798_amd as jq
from decode_ref import attend_ref, dev_f32, dev_i32, f64, bf16, random_tree, to_pages, visible
from parity import from_dev_bf16, to_dev_bf16

pytestmark = pytest.mark.gpu
NAN = 0x7FC0


def make(seed, nl, caps, h_q, h_kv, n_q, lens, dead=NAN, peak=1.0):
    rng = np.random.default_rng(seed)
    T = sum(caps)
    Q = bf16(rng, nl, len(caps), n_q, h_q, 128, scale=peak)
    K, V = bf16(rng, nl, T, h_kv, 128), bf16(rng, nl, T, h_kv, 128)
    cu = np.concatenate([[0], np.cumsum(caps)])
    live = np.broadcast_to(np.asarray(caps)[None], (nl, len(caps))) if lens is None else np.clip(lens, 0, np.asarray(caps)[None])
    if dead is not None:
        for l in range(nl):
            for s in range(len(caps)):
                K[l, cu[s] + live[l, s]:cu[s + 1]] = dead
                V[l, cu[s] + live[l, s]:cu[s + 1]] = dead
    return rng, Q, K, V, cu, live


def check(Q, K, V, cu, live, out, lse, mode="all", seen=None, scale=None, weights=None, start=None):
    nl, S, n_q, h_q, d = Q.shape
    h_kv = K.shape[2]
    G = h_q // h_kv
    scale = 1 / np.sqrt(d) if scale is None else scale
    out, lse = f64(from_dev_bf16(out)), lse.cpu().numpy().astype(np.float64)
    for l in range(nl):
        for s in range(S):
            n = int(live[l, s])
            see = visible(mode, n, n_q, G, None if seen is None else seen[s])
            for g in range(h_kv):
                q = f64(Q[l, s, :, g * G:(g + 1) * G]).reshape(n_q * G, d)
                k, v = f64(K[l, cu[s]:cu[s] + n, g]), f64(V[l, cu[s]:cu[s] + n, g])
                # what a row does not see is not part of its sums, whatever it holds
                ro, rl, rw, to, tl, tw = attend_ref(q, k, v, see, scale)
                o = out[l, s, :, g * G:(g + 1) * G].reshape(n_q * G, d)
                e = lse[l, s, :, g * G:(g + 1) * G].reshape(n_q * G)
                what = "layer %d sequence %d (%d rows) head %d" % (l, s, n, g)
                bad = ~(np.abs(o - ro) <= to)
                assert not bad.any(), "%s: out off by %g at %s" % (what, np.nanmax(np.abs(o - ro)), np.argwhere(bad)[:3].tolist())
                empty = np.isneginf(rl)
                assert np.array_equal(np.isneginf(e), empty), what
                off = np.abs(e[~empty] - rl[~empty])
                assert (off <= tl[~empty]).all(), "%s: lse off by %g" % (what, off.max())
                if weights is not None:
                    got = weights[l, g, cu[s]:cu[s + 1]].cpu().numpy().astype(np.float64)
                    was = start[l, g, cu[s]:cu[s + 1]].astype(np.float64)
                    want = was.copy()
                    want[:n] += rw
                    tol = np.zeros(was.size)
                    tol[:n] = tw + 2.0 ** -23 * np.abs(want[:n])
                    assert (np.abs(got - want) <= tol).all(), "%s: weights off by %g" % (what, np.abs(got - want).max())


def run(seed, nl, caps, h_q, h_kv, n_q, lens=None, mode="all", page=0, weigh=False, peak=1.0, scale=0.0, seen=None, dead=NAN):
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    print("attend", seed, nl, caps, h_q, h_kv, n_q, mode, page, flush=True)
    rng, Q, K, V, cu, live = make(seed, nl, caps, h_q, h_kv, n_q, lens, dead, peak)
    sh = jq.Shape(n_layers=nl, seq_lens=caps, n_q=n_q, h_q=h_q, h_kv=h_kv, window=mode == "causal", scale=scale)
    kw = {"lens": None if lens is None else dev_i32(lens)}
    start = weights = None
    if weigh:
        start = rng.random((nl, h_kv, sum(caps))).astype(np.float32)
        weights = kw["weights"] = dev_f32(start)
    args = (to_dev_bf16(Q),)
    if mode == "tree":
        seen = np.stack([random_tree(rng, n_q) for _ in caps]) if seen is None else seen
        args = (dev_i32(seen.view(np.int32)),) + args
    ws = jq.alloc_attend_workspace(sh, weights=weigh)
    ws.fill_(0xFF)  # NaN wherever something not yet written is read
    kw["ws"] = ws
    if page:
        kp, table = to_pages(np.random.default_rng(seed + 1), K, caps, page)
        vp, _ = to_pages(np.random.default_rng(seed + 1), V, caps, page)
        pages = jq.Pages(page, kp.shape[1], dev_i32(table))
        call = jq.attend_tree_paged if mode == "tree" else jq.attend_paged
        out, lse = call(sh, pages, *args, to_dev_bf16(kp), to_dev_bf16(vp), **kw)
    else:
        call = jq.attend_tree if mode == "tree" else jq.attend
        out, lse = call(sh, *args, to_dev_bf16(K), to_dev_bf16(V), **kw)
    torch.cuda.synchronize()
    check(Q, K, V, cu, live, out, lse, mode, seen, scale or None, weights, start)


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 1000, 4097])
def test_lengths(L):
    run(L, 1, [L], 8, 2, 1, weigh=True)


@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (4, 4), (4, 2), (6, 2), (8, 1), (24, 3), (16, 1), (20, 1), (32, 1), (33, 1), (40, 8)])
def test_head_layouts(h_q, h_kv):
    run(h_q, 1, [333], h_q, h_kv, 1, weigh=True)


@pytest.mark.parametrize("n_q", [2, 3, 5, 8, 9, 16, 17, 32])
@pytest.mark.parametrize("mode", ["all", "causal"])
def test_several_tokens(n_q, mode):
    run(n_q, 1, [200 + n_q, 70, 33 + n_q], 8, 2, n_q, mode=mode, weigh=True)


@pytest.mark.parametrize("page", [0, 32, 64, 256])
def test_ragged_batch_partly_filled(page):
    lens = np.array([[0, 1, 77, 500, 31, 64], [130, 0, 100, 499, 32, 1]], np.int32)
    run(5, 2, [130, 40, 100, 500, 32, 64], 8, 2, 1, lens=lens, page=page, weigh=True)


def test_live_counts_are_clamped():
    run(6, 1, [50, 60, 70], 4, 2, 1, lens=np.array([[-3, 1000, 2 ** 31 - 1]], np.int32), weigh=True)


@pytest.mark.parametrize("page", [0, 32])
def test_causal_rows_without_any_key(page):
    """Fewer live rows than queries: the first queries see nothing."""
    run(7, 1, [40, 64, 33], 8, 2, 9, lens=np.array([[3, 0, 8]], np.int32), mode="causal", page=page, weigh=True)


@pytest.mark.parametrize("n_q", [1, 2, 7, 16, 31, 32, 33, 64, 100])
@pytest.mark.parametrize("page", [0, 64])
def test_trees(n_q, page):
    caps = [300 + n_q, n_q, n_q + 1, 97 + n_q]
    run(n_q, 1, caps, 8, 2, n_q, mode="tree", page=page)


def test_tree_of_two_layers_partly_filled():
    n_q = 12
    lens = np.array([[100, 12, 5, 0], [13, 200, 12, 11]], np.int32)
    run(11, 2, [120, 200, 20, 12], 8, 4, n_q, lens=lens, mode="tree")


def test_tree_whose_rows_see_nothing():
    """No bit set and nothing cached before the drafted tokens: zeros and -infinity, beside rows that do see something."""
    n_q = 6
    seen = np.zeros((2, n_q, 1), np.uint32)
    seen[0, 2, 0], seen[0, 4, 0], seen[1, 5, 0] = 0b101, 0b10000, 0xFFFFFFFF
    run(12, 1, [n_q, n_q + 40], 4, 2, n_q, mode="tree", seen=seen)


@pytest.mark.parametrize("where", ["k", "v", "both"])
@pytest.mark.parametrize("value", [0x7FC0, 0x7F80, 0xFF80])  # NaN, infinities
def test_what_a_drafted_token_does_not_see_may_hold_anything(where, value):
    import torch
    n_q, caps, h_q, h_kv = 8, [57 + 8], 8, 2
    rng, Q, K, V, cu, live = make(13, 1, caps, h_q, h_kv, n_q, None)
    seen = np.zeros((1, n_q, 1), np.uint32)
    for i in range(n_q):
        seen[0, i, 0] = 1 << i if i % 2 else (1 << i) | 1   # odd tokens see themselves, even ones token 0 too
    clean_k, clean_v = K.copy(), V.copy()
    for j in (2, 4):                                        # tokens 2 and 4 see rows that are not finite, the others do not
        if where != "v": K[0, 57 + j] = value
        if where != "k": V[0, 57 + j, :, 5] = value
    sh = jq.Shape(n_layers=1, seq_lens=caps, n_q=n_q, h_q=h_q, h_kv=h_kv)
    out, lse = jq.attend_tree(sh, dev_i32(seen.view(np.int32)), to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    ref, rlse = jq.attend_tree(sh, dev_i32(seen.view(np.int32)), to_dev_bf16(Q), to_dev_bf16(clean_k), to_dev_bf16(clean_v))
    torch.cuda.synchronize()
    others = [i for i in range(n_q) if i not in (2, 4)]
    assert torch.equal(out[:, :, others], ref[:, :, others]) and torch.equal(lse[:, :, others], rlse[:, :, others])
    if value == 0x7FC0:
        assert torch.isnan(out[:, :, [2, 4]].float()).any()  # who sees it gets it


def test_causal_rows_do_not_see_later_nan():
    import torch
    n_q, caps = 4, [40]
    rng, Q, K, V, cu, live = make(14, 1, caps, 4, 2, n_q, None)
    sh = jq.Shape(n_layers=1, seq_lens=caps, n_q=n_q, h_q=4, h_kv=2, window=True)
    ref, rlse = jq.attend(sh, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    V[0, 39] = K[0, 39] = NAN
    out, lse = jq.attend(sh, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    torch.cuda.synchronize()
    assert torch.equal(out[:, :, :3], ref[:, :, :3]) and torch.equal(lse[:, :, :3], rlse[:, :, :3])
    assert torch.isnan(lse[:, :, 3]).all()


@pytest.mark.parametrize("peak", [0.0, 8.0, 40.0])
def test_flat_and_peaked(peak):
    """Queries of zeros (every row alike) up to scores hundreds of powers of two apart."""
    run(15, 1, [2000, 313], 8, 2, 1, peak=peak, weigh=True)


@pytest.mark.parametrize("scale", [1e-30, 0.5, 3.0])
def test_scales(scale):
    run(16, 1, [500], 4, 2, 2, scale=scale)


def test_rising_scores():
    """Keys whose scores rise along the cache, so that the running maximum keeps moving."""
    import torch
    from workloads import f32_to_bf16_bits
    rng, Q, K, V, cu, live = make(17, 1, [3000], 4, 2, 1, None)
    ramp = np.linspace(-2, 2, 3000)[:, None, None]
    K = f32_to_bf16_bits((f64(K[0]) * 0.1 + ramp).astype(np.float32))[None]
    Q = f32_to_bf16_bits((np.ones(Q.shape) * 8 + 0.1 * f64(Q)).astype(np.float32))
    sh = jq.Shape(n_layers=1, seq_lens=[3000], n_q=1, h_q=4, h_kv=2)
    out, lse = jq.attend(sh, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    torch.cuda.synchronize()
    check(Q, K, V, cu, live, out, lse)


@pytest.mark.parametrize("n_q", [4, 16, 32, 64])  # each way of sharing query rows and keys out
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("value", [0x7FC0, 0xFF80])
def test_rows_unseen_by_any_number_of_tokens_may_hold_anything(n_q, where, value):
    import torch
    base, h_q, h_kv = 200, 8, 2
    rng, Q, K, V, cu, live = make(30 + n_q, 1, [base + n_q], h_q, h_kv, n_q, None)
    seen = np.zeros((1, n_q, -(-n_q // 32)), np.uint32)
    for i in range(n_q):
        seen[0, i, i // 32] |= np.uint32(1 << (i % 32))
        seen[0, i, 0] |= np.uint32(1)
    clean = K.copy(), V.copy()
    dirty = [j for j in (1, n_q // 2, n_q - 1)]
    for j in dirty:
        (K if where == "k" else V)[0, base + j, :, j % 128] = value
    sh = jq.Shape(n_layers=1, seq_lens=[base + n_q], n_q=n_q, h_q=h_q, h_kv=h_kv)
    mask = dev_i32(seen.view(np.int32))
    out, lse = jq.attend_tree(sh, mask, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    ref, rlse = jq.attend_tree(sh, mask, to_dev_bf16(Q), to_dev_bf16(clean[0]), to_dev_bf16(clean[1]))
    torch.cuda.synchronize()
    others = [i for i in range(n_q) if i not in dirty]
    assert torch.equal(out[:, :, others], ref[:, :, others]) and torch.equal(lse[:, :, others], rlse[:, :, others])
    check(Q, *clean, cu, live, ref, rlse, "tree", seen)
    # the same of causal queries: those before the first dirty row do not see it
    causal = jq.Shape(n_layers=1, seq_lens=[base + n_q], n_q=n_q, h_q=h_q, h_kv=h_kv, window=True)
    out, lse = jq.attend(causal, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    ref, rlse = jq.attend(causal, to_dev_bf16(Q), to_dev_bf16(clean[0]), to_dev_bf16(clean[1]))
    torch.cuda.synchronize()
    assert torch.equal(out[:, :, :1], ref[:, :, :1]) and torch.equal(lse[:, :, :1], rlse[:, :, :1])


@pytest.mark.parametrize("n_q", [2, 16, 32, 64])
@pytest.mark.parametrize("way", ["rising", "falling", "sawtooth", "one_late"])
def test_scores_hundreds_of_octaves_apart(n_q, way):
    """The running maximum has to follow, sums must neither overflow nor vanish: scores between -600 and 600."""
    import torch
    from workloads import f32_to_bf16_bits
    n = 3000
    rng, Q, K, V, cu, live = make(40, 1, [n], 8, 2, n_q, None)
    x = np.linspace(-1, 1, n)
    ramp = {"rising": x, "falling": -x, "sawtooth": np.where(np.arange(n) % 97 < 50, x, -x), "one_late": np.where(np.arange(n) == n - 70, 1.0, -1.0)}[way]
    K = f32_to_bf16_bits((0.05 * f64(K[0]) + ramp[:, None, None]).astype(np.float32))[None]
    Q = f32_to_bf16_bits((np.ones(Q.shape) * 53 + 0.2 * f64(Q)).astype(np.float32))
    sh = jq.Shape(n_layers=1, seq_lens=[n], n_q=n_q, h_q=8, h_kv=2)
    out, lse = jq.attend(sh, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    torch.cuda.synchronize()
    check(Q, K, V, cu, live, out, lse)


@pytest.mark.parametrize("n_q", [1, 9, 20, 40])
def test_nothing_live_anywhere(n_q):
    run(41, 2, [50, 64], 8, 2, n_q, lens=np.zeros((2, 2), np.int32), weigh=n_q < 20)
    run(42, 1, [n_q, n_q], 8, 2, n_q, mode="causal", weigh=n_q < 20)


def test_calls_of_several_host_threads():
    import threading
    import torch
    rng, Q, K, V, cu, live = make(43, 1, [5000, 77], 16, 4, 1, None)
    sh = [jq.Shape(n_layers=1, seq_lens=[5000, 77], n_q=1, h_q=16, h_kv=4) for _ in range(4)]
    q, k, v = to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V)
    ref = jq.attend(sh[0], q, k, v)
    torch.cuda.synchronize()
    got = [[] for _ in sh]

    def work(i):
        side = torch.cuda.Stream()
        for _ in range(10):
            got[i].append(jq.attend(sh[i], q, k, v, stream=side))
        side.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sh))]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref[0]) and torch.equal(e, ref[1]) for g in got for o, e in g) and all(len(g) == 10 for g in got)


def test_many_layers_sequences_and_heads():
    run(18, 3, list(range(20, 20 + 40)), 32, 8, 1, weigh=True)


def test_as_many_sequences_as_a_call_takes():
    lens = np.array([[(37 * i) % 70 for i in range(128)]], np.int32)
    run(22, 1, [70 - (i % 3) for i in range(128)], 4, 2, 1, lens=lens, page=32, weigh=True)
    run(23, 1, [70 - (i % 3) for i in range(128)], 4, 2, 9, mode="tree")


def test_more_sequences_than_the_chip_takes_at_a_time():
    """300 (sequence, head) pairs of very different lengths, cut into shares of several rounds, with and without weights to hold."""
    caps = [5, 2000, 37, 700, 1, 333] * 25
    run(24, 1, caps[:100], 3, 3, 1, weigh=True)
    run(25, 1, [c + 20 for c in caps[:100]], 12, 3, 20, mode="causal", lens=np.array([[c + i % 23 for i, c in enumerate(caps[:100])]], np.int32))
    run(26, 1, [c + 20 for c in caps[:100]], 12, 3, 20, mode="tree")


def test_more_query_rows_than_a_workgroup_takes():
    run(27, 1, [700, 400], 8, 2, 300, mode="causal")
    run(28, 1, [333], 40, 2, 40, mode="tree", page=32)


def test_the_same_call_twice_gives_the_same_bits():
    import torch
    rng, Q, K, V, cu, live = make(19, 1, [9000, 511], 32, 8, 1, None)
    sh = jq.Shape(n_layers=1, seq_lens=[9000, 511], n_q=1, h_q=32, h_kv=8)
    q, k, v = to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V)
    res = []
    for _ in range(3):
        w = torch.zeros((1, 8, 9511), device="cuda")
        out, lse = jq.attend(sh, q, k, v, weights=w)
        res.append((out, lse, w))
    torch.cuda.synchronize()
    for r in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, res[0]))


def test_captured_calls_follow_the_live_rows():
    """Two captured calls that share a workspace, replayed in turn with eager calls between, while lens grows on the device."""
    import torch
    rng, Q, K, V, cu, _ = make(20, 1, [700, 300], 8, 2, 1, None)
    sh = jq.Shape(n_layers=1, seq_lens=[700, 300], n_q=1, h_q=8, h_kv=2)
    q, k, v = to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V)
    lens = dev_i32([[1, 0]])
    ws = jq.alloc_attend_workspace(sh, weights=True)
    outs = [(torch.empty_like(q), torch.empty((1, 1 * 2, 1, 8), device="cuda").view(1, 2, 1, 8), torch.zeros((1, 2, 1000), device="cuda")) for _ in range(2)]
    graphs = []
    side = torch.cuda.Stream()
    for o, e, w in outs:
        with torch.cuda.stream(side):
            jq.attend(sh, q, k, v, lens=lens, weights=w, out=o, lse=e, ws=ws)  # warm-up
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            jq.attend(sh, q, k, v, lens=lens, weights=w, out=o, lse=e, ws=ws)
        graphs.append(g)
        w.zero_()
    for n0, n1 in ((1, 0), (5, 300), (333, 31), (700, 1), (0, 299)):
        lens.copy_(dev_i32([[n0, n1]]))
        for g, (o, e, w) in zip(graphs, outs):
            start = w.cpu().numpy()
            g.replay()
            torch.cuda.synchronize()
            check(Q, K, V, cu, np.array([[n0, n1]]), o, e, weights=w, start=start)
            eager = jq.attend(sh, q, k, v, lens=lens, ws=ws)
            torch.cuda.synchronize()
            assert torch.equal(eager[0], o) and torch.equal(eager[1], e)


def test_calls_on_two_streams():
    import torch
    rng, Q, K, V, cu, live = make(21, 1, [6000], 32, 8, 1, None)
    sh = jq.Shape(n_layers=1, seq_lens=[6000], n_q=1, h_q=32, h_kv=8)
    q, k, v = to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V)
    ref = jq.attend(sh, q, k, v)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    wss = [jq.alloc_attend_workspace(sh) for _ in streams]
    torch.cuda.synchronize()
    for i in range(6):
        o, e = torch.empty_like(q), torch.empty((1, 1, 1, 32), device="cuda")
        torch.cuda.synchronize()
        got.append((o, e))
    for i, (o, e) in enumerate(got):
        jq.attend(sh, q, k, v, out=o, lse=e, ws=wss[i % 2], stream=streams[i % 2])
    torch.cuda.synchronize()
    for o, e in got:
        assert torch.equal(o, ref[0]) and torch.equal(e, ref[1])


def test_temporaries_belong_to_the_stream_of_the_call():
    """Calls on a side stream whose workspace and outputs are allocated inside, while the current stream allocates and overwrites
    memory of the same sizes."""
    import torch
    rng, Q, K, V, cu, live = make(29, 1, [3000], 16, 4, 1, None)
    sh = jq.Shape(n_layers=1, seq_lens=[3000], n_q=1, h_q=16, h_kv=4)
    q, k, v = to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V)
    ref = jq.attend(sh, q, k, v)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    for _ in range(20):
        got.append(jq.attend(sh, q, k, v, stream=side))
        torch.empty(jq.attend_workspace_bytes(sh), dtype=torch.uint8, device="cuda").fill_(0xFF)
    torch.cuda.synchronize()
    for o, e in got:
        assert torch.equal(o, ref[0]) and torch.equal(e, ref[1])


def test_long_cache_offsets_past_31_bits():
    """1.2 million rows of 8 heads, 2.3 GiB each of K and V, whose last row stands out."""
    import torch
    L, h_kv, h_q = 1_200_003, 8, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    K = torch.empty((1, L, h_kv, 128), dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    for a in range(0, L, 100_000):
        b = min(L, a + 100_000)
        K[0, a:b] = torch.randn((b - a, h_kv, 128), generator=gen, device="cuda").to(torch.bfloat16)
        V[0, a:b] = torch.randn((b - a, h_kv, 128), generator=gen, device="cuda").to(torch.bfloat16)
    Q = torch.randn((1, 1, 1, h_q, 128), generator=gen, device="cuda").to(torch.bfloat16)
    K[0, -1] = 0.5 * Q[0, 0, 0]  # the last row stands out
    sh = jq.Shape(n_layers=1, seq_lens=[L], n_q=1, h_q=h_q, h_kv=h_kv)
    w = torch.zeros((1, h_kv, L), device="cuda")
    out, lse = jq.attend(sh, Q, K, V, weights=w)
    torch.cuda.synchronize()
    for g in (0, 7):
        x = (K[0, :, g].double() @ Q[0, 0, 0, g].double()) / 128 ** 0.5
        p = torch.softmax(x, 0)
        ref = p @ V[0, :, g].double()
        # a wave adds some 100 tiles one after the other, the join some 100 workgroups: 300 roundings of 2^-24 in a row are 2e-5
        assert (out[0, 0, 0, g].double() - ref).abs().max() <= 2.0 ** -8 * ref.abs().max() + 1e-3 * (p @ V[0, :, g].double().abs()).max()
        assert abs(float(lse[0, 0, 0, g]) - float(torch.logsumexp(x, 0))) < 1e-4
        assert (w[0, g].double() - p).abs().max() <= 1e-4 * p.max()

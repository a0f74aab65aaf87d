"""Attention of sequences that continue shared prefixes (jq.attend_shared, jq.attend_shared_paged) against a 64-bit form over the
prefix's and the sequence's rows one after the other.  Everything that must not be read holds NaN.  Bounds: decode_ref's, where
probabilities are one bf16 part for the rows of a prefix when that of the call's prefixes with most has more than 64 query rows a KV
head (one kernel sweeps them all, the one for the largest).  A part is off by at most half a step of bf16, 2^-8 p, so out, the sum of
p v, by at most 2^-8 sum p |v| more than with the second part, which is what check() adds."""
import numpy as np
import pytest

import paper_2509_10798_amd as jq
from decode_ref import attend_ref, bf16, dev_i32, f64, to_pages, visible
from parity import from_dev_bf16, to_dev_bf16

pytestmark = pytest.mark.gpu
NAN, INF = 0x7FC0, 0x7F80


def spoil(nl, cu, live, *caches):
    """NaN in rows that are not live."""
    for l in range(nl):
        for s in range(len(cu) - 1):
            for x in caches:
                x[l, cu[s] + live[l, s]:cu[s + 1]] = NAN


class Case:
    def __init__(self, seed, nl, prefix, members, caps, h_q, h_kv, n_q=1, lens=None, prefix_lens=None, causal=False, peak=1.0):
        rng = self.rng = np.random.default_rng(seed)
        assert sum(members) == len(caps)
        self.nl, self.prefix, self.members, self.caps, self.h_q, self.h_kv, self.n_q, self.causal = nl, prefix, members, caps, h_q, h_kv, n_q, causal
        self.Q = bf16(rng, nl, len(caps), n_q, h_q, 128, scale=peak)
        self.K, self.V = (bf16(rng, nl, sum(caps), h_kv, 128) for _ in range(2))
        self.Kp, self.Vp = (bf16(rng, nl, sum(prefix), h_kv, 128) for _ in range(2))
        self.cu, self.cp = (np.concatenate([[0], np.cumsum(x)]) for x in (caps, prefix))
        self.lens, self.prefix_lens = lens, prefix_lens
        self.live = np.broadcast_to(np.asarray(caps)[None], (nl, len(caps))) if lens is None else np.clip(lens, 0, np.asarray(caps)[None])
        self.plive = np.broadcast_to(np.asarray(prefix)[None], (nl, len(prefix))) if prefix_lens is None else np.clip(prefix_lens, 0, np.asarray(prefix)[None])
        spoil(nl, self.cu, self.live, self.K, self.V)
        spoil(nl, self.cp, self.plive, self.Kp, self.Vp)
        self.of = [p for p, m in enumerate(members) for _ in range(m)]
        self.shape = jq.Shape(n_layers=nl, seq_lens=caps, n_q=n_q, h_q=h_q, h_kv=h_kv, window=causal)

    def call(self, page=0, **kw):
        import torch
        assert torch.cuda.is_available(), "this test needs the GPU"
        print("shared", self.nl, self.prefix[:6], self.members[:6], self.caps[:6], self.h_q, self.h_kv, self.n_q, page, flush=True)
        pre = jq.Prefixes(self.prefix, self.members, None if self.prefix_lens is None else dev_i32(self.prefix_lens))
        kw["lens"] = None if self.lens is None else dev_i32(self.lens)
        if "ws" not in kw:
            kw["ws"] = jq.alloc_attend_shared_workspace(self.shape, pre)
            kw["ws"].fill_(0xFF)  # NaN wherever something not yet written is read
        q = to_dev_bf16(self.Q)
        if not page:
            return jq.attend_shared(self.shape, pre, q, *(to_dev_bf16(x) for x in (self.Kp, self.Vp, self.K, self.V)), **kw)
        pools = []
        for own, shared in ((self.K, self.Kp), (self.V, self.Vp)):   # prefixes and sequences in one pool
            pool, table = to_pages(np.random.default_rng(3), np.concatenate([shared, own], 1), list(self.prefix) + list(self.caps), page)
            pools.append(to_dev_bf16(pool))
        n = len(self.prefix)
        pre.block_table = dev_i32(table[:n])
        pages = jq.Pages(page, pool.shape[1], dev_i32(table[n:]))
        return jq.attend_shared_paged(self.shape, pages, pre, q, *pools, **kw)

    def rows_of(self, l, s, g):
        p, n, m = self.of[s], int(self.live[l, s]), int(self.plive[l, self.of[s]])
        k, v = (np.concatenate([f64(a[l, self.cp[p]:self.cp[p] + m, g]), f64(b[l, self.cu[s]:self.cu[s] + n, g])]) for a, b in ((self.Kp, self.K), (self.Vp, self.V)))
        see = visible("causal" if self.causal else "all", n, self.n_q, self.h_q // self.h_kv)
        return k, v, np.concatenate([np.ones((see.shape[0], m), bool), see], 1)

    def check(self, out, lse):
        G = self.h_q // self.h_kv
        out, lse = f64(from_dev_bf16(out)), lse.cpu().numpy().astype(np.float64)
        for l in range(self.nl):
            for s in range(len(self.caps)):
                many = max(self.members) * self.n_q * G > 64 >= self.n_q * G
                for g in range(self.h_kv):
                    k, v, see = self.rows_of(l, s, g)
                    q = f64(self.Q[l, s, :, g * G:(g + 1) * G]).reshape(self.n_q * G, 128)
                    ro, rl, _, to, tl, _ = attend_ref(q, k, v, see, 128 ** -0.5)
                    if many:
                        to = to + 2.0 ** -8 * attend_ref(q, k, np.abs(v), see, 128 ** -0.5)[0]
                    o, e = out[l, s, :, g * G:(g + 1) * G].reshape(ro.shape), lse[l, s, :, g * G:(g + 1) * G].reshape(rl.shape)
                    what = "layer %d sequence %d (%d rows, prefix %d) head %d" % (l, s, self.live[l, s], self.plive[l, self.of[s]], g)
                    bad = ~(np.abs(o - ro) <= to)
                    assert not bad.any(), "%s: out off by %g at %s" % (what, np.nanmax(np.abs(o - ro)), np.argwhere(bad)[:3].tolist())
                    empty = np.isneginf(rl)
                    assert np.array_equal(np.isneginf(e), empty), what
                    assert (np.abs(e[~empty] - rl[~empty]) <= tl[~empty]).all(), "%s: lse off by %g" % (what, np.abs(e[~empty] - rl[~empty]).max())


def run(*args, page=0, **kw):
    import torch
    c = Case(*args, **kw)
    out, lse = c.call(page)
    torch.cuda.synchronize()
    c.check(out, lse)


@pytest.mark.parametrize("P", [1, 2, 31, 32, 33, 127, 128, 255, 256, 257, 1000, 4097])
@pytest.mark.parametrize("page", [0, 32])
def test_prefix_lengths(P, page):
    run(P, 1, [P], [3], [1, 40, 300], 8, 2, page=page)


@pytest.mark.parametrize("L", [1, 2, 31, 32, 33, 255, 256, 257, 1000, 2500])
def test_lengths_of_the_sequences(L):
    run(L, 1, [700], [2], [L, 7], 8, 2)


@pytest.mark.parametrize("members", [1, 3, 4, 5, 8, 9, 16, 17, 32, 33, 64, 70])   # 4 to 280 query rows a KV head: every way of sharing rows and keys out
@pytest.mark.parametrize("page", [0, 64])
def test_numbers_of_sequences(members, page):
    run(members, 1, [1100], [members], [1 + (37 * i) % 90 for i in range(members)], 8, 2, page=page)


@pytest.mark.parametrize("n_q", [2, 4, 5, 8, 9, 16, 20])   # of one sequence 8 to 80 query rows
@pytest.mark.parametrize("members", [1, 3, 9])
@pytest.mark.parametrize("causal", [False, True])
def test_several_tokens(n_q, members, causal):
    run(n_q, 1, [500], [members], [n_q + (37 * i) % 90 for i in range(members)], 8, 2, n_q=n_q, causal=causal)


@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (4, 4), (6, 2), (24, 3), (16, 1), (33, 1), (40, 8)])
def test_head_layouts(h_q, h_kv):
    run(h_q, 1, [333, 90], [3, 2], [40, 5, 64, 100, 1], h_q, h_kv)


@pytest.mark.parametrize("page", [0, 32, 256])
def test_prefixes_of_different_lengths_and_numbers(page):
    """Partly filled prefixes and sequences, some of them empty, other numbers in each layer; a sequence alone with an empty prefix, one
    with nothing at all."""
    caps = [300, 77, 129, 511, 40, 50, 33, 64, 80, 95]
    lens = np.array([[300, 0, 100, 500, 1, 0, 33, 50, 0, 95], [1, 77, 0, 511, 40, 50, 0, 64, 80, 0]], np.int32)
    plens = np.array([[1203, 0, 30, 1, 0], [0, 300, 8, 2000, 0]], np.int32)
    run(5, 2, [1203, 300, 43, 2071, 20], [4, 2, 1, 2, 1], caps, 8, 2, lens=lens, prefix_lens=plens, page=page)


def test_live_counts_are_clamped():
    run(6, 1, [50, 60, 70], [2, 1, 1], [40, 30, 20, 10], 4, 2, lens=np.array([[-3, 1000, 2 ** 31 - 1, 5]], np.int32),
        prefix_lens=np.array([[-1, 2 ** 31 - 1, 99]], np.int32))


@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("n_q", [9, 20])
def test_causal_tokens_with_fewer_rows_of_their_own(page, n_q):
    """Tokens in front of the first live row see the prefix alone, or nothing."""
    run(7, 1, [100, 64], [2, 2], [40, 64, 33, 40], 8, 2, n_q=n_q, lens=np.array([[3, 0, 8, n_q]], np.int32), prefix_lens=np.array([[90, 0]], np.int32), causal=True, page=page)


@pytest.mark.parametrize("members", [1, 5, 12, 40])
def test_nothing_live_anywhere(members):
    run(8, 2, [50], [members], [9] * members, 8, 2, lens=np.zeros((2, members), np.int32), prefix_lens=np.zeros((2, 1), np.int32))


def test_as_many_sequences_and_prefixes_as_a_call_takes():
    run(9, 1, [70 - i % 3 for i in range(128)], [1] * 128, [20 + i % 7 for i in range(128)], 4, 2, page=32)
    run(10, 1, [900], [128], [1 + i % 50 for i in range(128)], 8, 2)
    run(11, 1, [100 + 9 * i for i in range(40)], [1 + i % 5 for i in range(40)], [5 + (11 * i) % 70 for i in range(sum(1 + i % 5 for i in range(40)))], 6, 3)


def test_many_layers_and_heads():
    run(12, 5, [600, 200], [7, 3], [30 + i for i in range(10)], 64, 16)
    run(13, 1, [300], [2], [70, 300], 512, 256)


def test_more_work_than_the_chip_takes_at_a_time():
    """Long prefixes and many long sequences: shares of several rounds, more parts than a wave has lanes."""
    run(14, 1, [20000], [3], [300, 7000, 50], 2, 1)
    run(15, 2, [3000, 2000], [20, 10], [1500 + 10 * i for i in range(30)], 8, 4, n_q=2, causal=True)


@pytest.mark.parametrize("peak", [0.0, 8.0, 40.0])
@pytest.mark.parametrize("members", [2, 20])
def test_flat_and_peaked(peak, members):
    run(16, 1, [1500], [members], [100] * members, 8, 2, peak=peak)


@pytest.mark.parametrize("members", [2, 8, 16, 32, 64])
@pytest.mark.parametrize("way", ["prefix", "own"])
def test_one_part_outweighs_the_other_by_hundreds_of_octaves(members, way):
    import torch
    from workloads import f32_to_bf16_bits
    c = Case(17, 1, [900], [members], [60] * members, 8, 2)
    sign = 1 if way == "prefix" else -1
    c.Kp = f32_to_bf16_bits((0.05 * f64(c.Kp[0]) + sign).astype(np.float32))[None]
    c.K = f32_to_bf16_bits((0.05 * f64(c.K[0]) - sign).astype(np.float32))[None]
    c.Q = f32_to_bf16_bits((np.ones(c.Q.shape) * 53 + 0.2 * f64(c.Q)).astype(np.float32))
    out, lse = c.call()
    torch.cuda.synchronize()
    c.check(out, lse)


@pytest.mark.parametrize("members", [2, 8, 16, 32, 64])
def test_values_that_are_not_finite(members):
    """They reach their own dimension of the queries that see their row -- all of a prefix's sequences, or one -- and nothing else."""
    import torch
    c = Case(18, 1, [700, 300], [members, 1], [60] * (members + 1), 8, 2, n_q=2, causal=True)
    ref = c.call()
    c.Vp[0, 333, 1, 7], c.Vp[0, 0, 1, 100], c.V[0, 60 * (members - 1) + 59, 1, 64] = NAN, INF, INF
    out, lse = c.call()
    torch.cuda.synchronize()
    assert torch.equal(lse, ref[1])
    want = f64(from_dev_bf16(ref[0]))
    want[0, :members, :, 4:, 7] = np.nan
    want[0, :members, :, 4:, 100] = np.inf
    want[0, members - 1, 1, 4:, 64] = np.inf   # the last row is seen by the last token alone
    np.testing.assert_array_equal(f64(from_dev_bf16(out)), want)


def test_the_same_call_twice_gives_the_same_bits():
    import torch
    c = Case(19, 1, [9000, 511], [12, 3], [200 + i for i in range(15)], 32, 8)
    res = [c.call() for _ in range(3)]
    torch.cuda.synchronize()
    for r in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, res[0]))


def test_two_captured_calls_share_a_workspace():
    """Replayed in turn with eager calls between, while both live counts change on the device."""
    import torch
    c = Case(20, 1, [600, 100], [3, 1], [50, 60, 70, 80], 8, 2)
    args = [to_dev_bf16(x) for x in (c.Q, c.Kp, c.Vp, c.K, c.V)]
    lens, plens = dev_i32([c.caps]), dev_i32([c.prefix])
    pre = jq.Prefixes(c.prefix, c.members, plens)
    ws = jq.alloc_attend_shared_workspace(c.shape, pre)
    outs = [(torch.empty_like(args[0]), torch.empty((1, 4, 1, 8), device="cuda")) for _ in range(2)]
    graphs, side = [], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o, e in outs:
        with torch.cuda.stream(side):
            jq.attend_shared(c.shape, pre, *args, lens=lens, out=o, lse=e, ws=ws)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            jq.attend_shared(c.shape, pre, *args, lens=lens, out=o, lse=e, ws=ws)
        graphs.append(g)
    for n, m in (([50, 60, 70, 80], [600, 100]), ([1, 0, 33, 80], [0, 100]), ([0, 0, 0, 0], [333, 0]), ([49, 2, 70, 5], [600, 1])):
        lens.copy_(dev_i32([n]))
        plens.copy_(dev_i32([m]))
        c.live, c.plive = np.array([n]), np.array([m])
        for g, (o, e) in zip(graphs, outs):
            o.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            c.check(o, e)
            eager = jq.attend_shared(c.shape, pre, *args, lens=lens, ws=ws)
            torch.cuda.synchronize()
            assert torch.equal(eager[0], o) and torch.equal(eager[1], e)


def test_calls_on_another_stream():
    import torch
    c = Case(21, 1, [3000], [6], [100] * 6, 16, 4)
    args = [to_dev_bf16(x) for x in (c.Q, c.Kp, c.Vp, c.K, c.V)]
    pre = jq.Prefixes(c.prefix, c.members)
    ref = jq.attend_shared(c.shape, pre, *args)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    for _ in range(20):
        got.append(jq.attend_shared(c.shape, pre, *args, stream=side))
        torch.empty(jq.attend_shared_workspace_bytes(c.shape, pre), dtype=torch.uint8, device="cuda").fill_(0xFF)
    torch.cuda.synchronize()
    for o, e in got:
        assert torch.equal(o, ref[0]) and torch.equal(e, ref[1])


def test_prefix_offsets_past_31_bits():
    """Three layers of a prefix of 500 000 rows of 8 heads, 3 GB each of K and V, whose last row stands out."""
    import torch
    nl, P, h = 3, 500_003, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    K, V = (torch.empty((nl, P, h, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for x in (K, V):
        for a in range(0, P, 100_000):
            b = min(P, a + 100_000)
            x[:, a:b] = torch.randn((nl, b - a, h, 128), generator=gen, device="cuda").to(torch.bfloat16)
    Q = torch.randn((nl, 3, 1, h, 128), generator=gen, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((nl, 30, h, 128), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    K[-1, -1] = 0.5 * Q[-1, 1, 0]
    sh = jq.Shape(n_layers=nl, seq_lens=[10] * 3, n_q=1, h_q=h, h_kv=h)
    out, lse = jq.attend_shared(sh, jq.Prefixes([P], [3]), Q, K, V, k, v)
    torch.cuda.synchronize()
    for s in range(3):
        for g in (0, 7):
            kk, vv = (torch.cat((a[-1, :, g], b[-1, 10 * s:10 * s + 10, g])).double() for a, b in ((K, k), (V, v)))
            x = (kk @ Q[-1, s, 0, g].double()) / 128 ** 0.5
            p = torch.softmax(x, 0)
            ref = p @ vv
            # (some 100 tiles a wave and 100 parts one after the other: 300 roundings of 2^-24 are 2e-5 of a term)
            assert (out[-1, s, 0, g].double() - ref).abs().max() <= 2.0 ** -8 * ref.abs().max() + 1e-3 * (p @ vv.abs()).max()
            assert abs(float(lse[-1, s, 0, g]) - float(torch.logsumexp(x, 0))) < 1e-4


def test_answers_to_one_pruned_prompt():
    """A prompt is pruned once; five answers are decoded from it side by side, each appending its rows to a cache of its own, and agree with
    answers decoded one by one on caches of their own with the prompt's rows in front."""
    import torch
    rng = np.random.default_rng(50)
    nl, prompt, B, n, h_q, h_kv, steps = 2, 700, 200, 5, 8, 2, 6
    Q, K, V = bf16(rng, nl, 1, 8, h_q, 128), bf16(rng, nl, prompt, h_kv, 128), bf16(rng, nl, prompt, h_kv, 128)
    prune = jq.Shape(n_layers=nl, seq_lens=[prompt], n_q=8, h_q=h_q, h_kv=h_kv, budgets=[B])
    Kp, Vp, _, _ = jq.evict(prune, to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V))
    c = Case(51, nl, [B], [n], [steps] * n, h_q, h_kv)
    c.Kp, c.Vp = from_dev_bf16(Kp), from_dev_bf16(Vp)
    own = [torch.full((nl, n * steps, h_kv, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    alone = [torch.cat([torch.cat((p, torch.zeros((nl, steps, h_kv, 128), dtype=torch.bfloat16, device="cuda")), 1) for _ in range(n)], 1) for p in (Kp, Vp)]
    one = jq.Shape(n_layers=nl, seq_lens=[B + steps] * n, n_q=1, h_q=h_q, h_kv=h_kv)
    pre = jq.Prefixes([B], [n])
    lens = torch.zeros((nl, n), dtype=torch.int32, device="cuda")
    for i in range(steps):
        new = [bf16(rng, nl, n, h, 128) for h in (h_kv, h_kv, h_q)]
        for t, x, y, z in zip(own, new, (c.K, c.V), alone):
            t.view(nl, n, steps, h_kv, 128)[:, :, i] = to_dev_bf16(x)
            z.view(nl, n, B + steps, h_kv, 128)[:, :, B + i] = to_dev_bf16(x)
            y.reshape(nl, n, steps, h_kv, 128)[:, :, i] = x
        lens += 1
        c.Q, c.live = new[2][:, :, None], np.full((nl, n), i + 1)
        out, lse = jq.attend_shared(c.shape, pre, to_dev_bf16(c.Q), Kp, Vp, *own, lens=lens)
        ref, rlse = jq.attend(one, to_dev_bf16(c.Q), *alone, lens=lens + B)
        torch.cuda.synchronize()
        c.check(out, lse)
        assert (lse - rlse).abs().max() < 1e-5 and (out.float() - ref.float()).abs().max() <= 2.0 ** -7 * ref.float().abs().max()


def test_calls_of_several_host_threads():
    import threading
    import torch
    c = Case(60, 1, [2000, 77], [5, 2], [90] * 7, 16, 4)
    args = [to_dev_bf16(x) for x in (c.Q, c.Kp, c.Vp, c.K, c.V)]
    shapes = [(jq.Shape(n_layers=1, seq_lens=c.caps, n_q=1, h_q=16, h_kv=4), jq.Prefixes(c.prefix, c.members)) for _ in range(4)]
    ref = jq.attend_shared(*shapes[0], *args)
    torch.cuda.synchronize()
    got = [[] for _ in shapes]

    def work(i):
        side = torch.cuda.Stream()
        for _ in range(10):
            got[i].append(jq.attend_shared(*shapes[i], *args, stream=side))
        side.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(shapes))]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref[0]) and torch.equal(e, ref[1]) for g in got for o, e in g) and all(len(g) == 10 for g in got)


@pytest.mark.parametrize("h_kv", [1, 3, 5])
@pytest.mark.parametrize("page", [0, 32])
def test_several_groups_of_query_rows_beside_few(h_kv, page):
    """Prefixes with 600, 20 and 4 query rows a KV head, heads that do not fill an eighth of the chip's dies, several layers."""
    caps = [3 + (13 * i) % 60 for i in range(156)][:128]
    members = [120, 5, 3]
    run(61, 2, [1300, 40, 900], members, caps, 4 * h_kv, h_kv, n_q=1, page=page)
    run(62, 1, [500, 1300], [9, 1], [30 + i for i in range(10)], 4 * h_kv, h_kv, n_q=17, causal=True, page=page)


@pytest.mark.parametrize("room", [16, 2048, 30000])    # (how rows and keys are shared out goes by the room, not by what is live)
@pytest.mark.parametrize("members,n_q", [([17], 1), ([32], 1), ([33], 1), ([64], 1), ([12, 5, 1], 4), ([40, 1], 1), ([1], 20), ([2, 1], 17)])
def test_probabilities_are_two_parts_whatever_the_number_of_query_rows(members, n_q, room):
    """Sixteen rows of a prefix, so that what a second bf16 part adds to out (2^-8 p without it) stands out against the other roundings: bounds of
    two parts, 2^-16 p, for every sequence, those alone on a prefix beside a crowded one among them."""
    import torch
    n, G = sum(members), 4
    c = Case(70 + n_q, 1, [room] * len(members), members, [n_q + 2] * n, 8, 2, n_q=n_q, lens=np.array([[i % 3 for i in range(n)]], np.int32),
             prefix_lens=np.full((1, len(members)), 16, np.int32), peak=0.5)
    out, lse = (x.cpu() for x in c.call())
    out = f64(from_dev_bf16(out))
    for s in range(n):
        for g in range(2):
            k, v, see = c.rows_of(0, s, g)
            q = f64(c.Q[0, s, :, g * G:(g + 1) * G]).reshape(n_q * G, 128)
            o, e = out[0, s, :, g * G:(g + 1) * G].reshape(-1, 128), lse[0, s, :, g * G:(g + 1) * G].reshape(-1).double().numpy()
            for r in range(0, n_q * G, 64):
                ro, rl, _, to, tl, _ = attend_ref(q[r:r + 64], k, v, see[r:r + 64], 128 ** -0.5)   # (its bounds for up to 64 rows)
                assert (np.abs(o[r:r + 64] - ro) <= to).all(), "sequence %d: out off by %g of its bound" % (s, (np.abs(o[r:r + 64] - ro) / to).max())
                assert (np.abs(e[r:r + 64] - rl) <= tl).all(), s


def test_the_last_row_of_a_prefix_past_31_bits_of_offset():
    """Three layers of a prefix of 500 000 rows of 8 heads, 3 GB each of K and V.  The last row's score is ahead of all others together by more than
    2^24 for every sequence, so that its values are the outputs, to the bit: parts of p (2^-16) and fp32 sums stay far within half a step of bf16."""
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    nl, P, h = 3, 500_003, 8
    gen = torch.Generator(device="cuda").manual_seed(4)
    K, V = (torch.empty((nl, P, h, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for x in (K, V):
        for a in range(0, P, 100_000):
            b = min(P, a + 100_000)
            x[:, a:b] = torch.randn((nl, b - a, h, 128), generator=gen, device="cuda").to(torch.bfloat16)
    one = torch.randn((nl, 1, 1, h, 128), generator=gen, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((nl, 30, h, 128), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    K[:, -1] = 4 * one[:, 0, 0]
    V[:, -1] = 8 * torch.randn((nl, h, 128), generator=gen, device="cuda").to(torch.bfloat16)
    sh = jq.Shape(n_layers=nl, seq_lens=[10] * 3, n_q=1, h_q=h, h_kv=h)
    out, lse = jq.attend_shared(sh, jq.Prefixes([P], [3]), one.expand(nl, 3, 1, h, 128).contiguous(), K, V, k, v)
    torch.cuda.synchronize()
    top = 4 * (one[:, :, 0].double() ** 2).sum(-1) / 128 ** 0.5       # [nl, 1, h], some 45
    for g in range(h):                                                # (what the inputs are meant to be, before what comes of them)
        for l in range(nl):
            x = (K[l, :-1, g].float() @ one[l, 0, 0, g].float()).double() / 128 ** 0.5
            assert float(torch.logsumexp(x, 0)) + 24 * np.log(2) < float(top[l, 0, g])
    assert torch.equal(out, V[:, -1][:, None, None].expand(nl, 3, 1, h, 128))
    u = 2.0 ** -24
    assert ((lse[:, :, 0].double() - top).abs() <= 132 * u * top + 4 * u * (top + 16) + 404 * u * (1 + top)).all()   # (a score, and its log-sum-exp)

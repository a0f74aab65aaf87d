"""What a value of V that is not finite does to attention (jq.attend, jq.attend_tree): by the definition out = sum_j p_j V[j] it reaches
the outputs of its own dimension, of the queries that see its row, and nothing else -- log-sum-exps and accumulated weights are
functions of Q and K.  Everything else has to be the bits that the same call leaves with finite values in those places."""
import numpy as np
import pytest

import paper_2509_10798_amd as jq
from decode_ref import bf16, dev_f32, dev_i32, f64, random_tree, to_pages, visible
from parity import from_dev_bf16, to_dev_bf16

pytestmark = pytest.mark.gpu
NAN, INF, MINUS_INF = 0x7FC0, 0x7F80, 0xFF80
# one dimension each: a NaN, an infinity of either sign, both signs of two rows, a NaN beside an infinity
PLACES = ((3, (NAN, None)), (70, (INF, None)), (127, (None, MINUS_INF)), (40, (INF, MINUS_INF)), (41, (NAN, INF)), (42, (INF, INF)))


def expected(see, first, second):
    """What the rows of out hold in a dimension where keys `first` and `second` hold those values: finite ones are left to the clean call."""
    got = np.zeros(see.shape[0])
    with np.errstate(invalid="ignore"):
        for key, value in (first, second):
            if value is not None:
                got += np.where(see[:, key], {NAN: np.nan, INF: np.inf, MINUS_INF: -np.inf}[value], 0.0)
    return got


def compare(n, n_q, mode, keys, h_q=8, h_kv=2, page=0, weigh=False, lens=None, K_of=None, scale=0.0):
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    print("values seen", n, n_q, mode, keys, h_q, h_kv, page, flush=True)
    rng = np.random.default_rng(100 + n_q)
    G, cap = h_q // h_kv, n if lens is None else n + 9
    Q, K, V = bf16(rng, 1, 1, n_q, h_q, 128), bf16(rng, 1, cap, h_kv, 128), bf16(rng, 1, cap, h_kv, 128)
    if K_of is not None:
        Q, K = K_of(Q, K)
    dirty = V.copy()
    for dim, values in PLACES:
        for key, value in zip(keys, values):
            if value is not None:
                dirty[0, key, 1, dim] = value     # head 1 only: head 0 is as it was
    sh = jq.Shape(n_layers=1, seq_lens=[cap], n_q=n_q, h_q=h_q, h_kv=h_kv, window=mode == "causal", scale=scale)
    front = (sh,)
    pools = [K, V, dirty]
    if page:
        pools = [to_pages(np.random.default_rng(1), x, [cap], page) for x in pools]
        front += (jq.Pages(page, pools[0][0].shape[1], dev_i32(pools[0][1])),)
        pools = [x[0] for x in pools]
    k, v, d = (to_dev_bf16(x) for x in pools)
    seen, args = None, (to_dev_bf16(Q),)
    if mode == "tree":
        seen = random_tree(rng, n_q)
        args = (dev_i32(seen[None].view(np.int32)),) + args
    call = {(False, False): jq.attend, (False, True): jq.attend_paged, (True, False): jq.attend_tree, (True, True): jq.attend_tree_paged}[mode == "tree", bool(page)]

    def attend(values):
        kw = {"lens": None if lens is None else dev_i32([[lens]])}
        if weigh:
            kw["weights"] = torch.ones((1, h_kv, cap), device="cuda")
        out, lse = call(*front, *args, k, values, **kw)
        torch.cuda.synchronize()
        return out.view(torch.int16).cpu().numpy().view(np.uint16)[0, 0], lse.cpu().numpy(), kw["weights"].cpu().numpy() if weigh else None
    (out, lse, w), (ref, rlse, rw) = attend(d), attend(v)
    assert np.isfinite(f64(ref)).all()
    np.testing.assert_array_equal(lse, rlse)
    if weigh:
        np.testing.assert_array_equal(w, rw)
    others = [h for h in range(h_q) if h // G != 1]
    np.testing.assert_array_equal(out[:, others], ref[:, others])
    see = visible(mode, n, n_q, G, seen)
    out, ref = (x[:, G:2 * G].reshape(n_q * G, 128) for x in (out, ref))
    dims = [dim for dim, _ in PLACES]
    rest = [i for i in range(128) if i not in dims]
    np.testing.assert_array_equal(out[:, rest], ref[:, rest])
    for dim, values in PLACES:
        want = expected(see, *zip(keys, values))
        clean = want == 0
        np.testing.assert_array_equal(out[clean, dim], ref[clean, dim])
        np.testing.assert_array_equal(f64(out[~clean, dim]), want[~clean])


@pytest.mark.parametrize("n_q", [1, 4, 8, 16, 32, 64])   # 4 to 256 query rows a KV head: each way of sharing rows and keys out
@pytest.mark.parametrize("mode", ["all", "causal", "tree"])
@pytest.mark.parametrize("where", ["front", "end", "either"])
def test_values_reach_their_dimension_of_who_sees_them(n_q, mode, where):
    n = 1003 + n_q
    keys = {"front": (5, 77), "end": (n - 1, n - 2), "either": (n - 1, 300)}[where]
    compare(n, n_q, mode, keys, weigh=mode != "tree" and n_q <= 32)


@pytest.mark.parametrize("n_q", [1, 8, 16, 64])
@pytest.mark.parametrize("page", [0, 32])
def test_values_of_short_and_partly_filled_caches(n_q, page):
    compare(n_q + 20, n_q, "causal", (n_q + 10, 2), page=page, weigh=n_q <= 32, lens=n_q + 20)
    compare(64, n_q, "all", (0, 63), page=page, weigh=n_q <= 32)


@pytest.mark.parametrize("n_q", [1, 16, 32])
def test_values_in_a_cache_swept_by_one_workgroup_a_sequence(n_q):
    """As many heads as there are CUs: no sequence is shared, and one wave has many tiles."""
    compare(700, n_q, "all", (699, 31), h_q=512, h_kv=256, weigh=True)


@pytest.mark.parametrize("n_q", [1, 8, 16])
@pytest.mark.parametrize("keys", [(7, 128 * 127 + 5), (17_999, 9_000)])
def test_values_among_more_shares_than_a_wave_has_lanes(n_q, keys):
    compare(18_000, n_q, "all", keys, weigh=True)


@pytest.mark.parametrize("n_q", [1, 8, 16, 32, 64])
@pytest.mark.parametrize("keys", [(3, 9), (2990, 2999), (3, 2999)])
def test_values_of_rows_that_hardly_weigh_anything(n_q, keys):
    """Scores from -600 to 600: a share of 1e-500 of an infinity is one, wherever its row lies and whoever has the larger scores."""
    from workloads import f32_to_bf16_bits

    def steep(Q, K):
        ramp = np.linspace(-1, 1, K.shape[1])[:, None, None]
        return (f32_to_bf16_bits((np.ones(Q.shape) * 53 + 0.2 * f64(Q)).astype(np.float32)),
                f32_to_bf16_bits((0.05 * f64(K[0]) + ramp).astype(np.float32))[None])
    compare(3000, n_q, "all", keys, K_of=steep, weigh=n_q <= 32)


def test_a_call_captured_with_finite_values_meets_others():
    import torch
    rng = np.random.default_rng(7)
    Q, K, V = bf16(rng, 1, 1, 1, 8, 128), bf16(rng, 1, 500, 2, 128), bf16(rng, 1, 500, 2, 128)
    sh = jq.Shape(n_layers=1, seq_lens=[500], n_q=1, h_q=8, h_kv=2)
    q, k, v, ws = to_dev_bf16(Q), to_dev_bf16(K), to_dev_bf16(V), jq.alloc_attend_workspace(sh)
    out, lse = jq.attend(sh, q, k, v, ws=ws)
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        jq.attend(sh, q, k, v, out=out, lse=lse, ws=ws)
    for value in (1.0, float("inf"), 2.0, float("nan"), 0.0):
        v[0, 100, 0, 17] = value
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        eager = jq.attend(sh, q, k, v, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(got[0].view(torch.int16), eager[0].view(torch.int16)) and torch.equal(got[1], eager[1])
        spoilt = ~torch.isfinite(got[0][0, 0, 0].float())
        assert spoilt.sum() == (0 if np.isfinite(value) else 4) and spoilt[:4, 17].all() == (not np.isfinite(value))

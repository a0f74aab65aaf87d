"""Rows that eviction by weight never takes (jq.evict_weight, jq.replace_lightest) stay whatever the others weigh, also beside weights
that are not numbers: a NaN of all ones ranks above infinity, and below the rows that stay."""
import numpy as np
import pytest

import paper_2509_10798_amd as jq
from decode_ref import bf16, dev_f32, dev_i32
from parity import from_dev_bf16, to_dev_bf16

pytestmark = pytest.mark.gpu
ONES = np.array([0x7FFFFFFF], np.uint32).view(np.float32)[0]


def order(w, pos, n, first, newest_from):
    """Rows by rank: those that stay, NaNs of positive sign, then by weight; lower rows first."""
    stays = (pos[:n] < first) | (pos[:n] > newest_from)
    return sorted(range(n), key=lambda j: (not stays[j], not np.isnan(w[j]), 0.0 if np.isnan(w[j]) else -float(w[j]), j))


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("L,B,nans", [(700, 64, 400), (700, 600, 690), (5000, 100, 4000), (20000, 100, 18000), (40000, 30000, 35000)])
def test_protected_rows_stay_beside_weights_of_all_ones(L, B, nans, inplace):
    """Each length takes another way through the selection; the NaNs stand in front, the newest rows at the end."""
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    rng = np.random.default_rng(L + B)
    K, V = bf16(rng, 1, L, 1, 128), bf16(rng, 1, L, 1, 128)
    w = rng.exponential(size=(1, 1, L)).astype(np.float32)
    w[0, 0, :nans] = ONES
    w[0, 0, 5] = np.inf
    pos = 3 * np.arange(L, dtype=np.int32)[None, None]
    pos[0, 0, -40:] = 3 * L + np.arange(40)
    sh = jq.Shape(n_layers=1, seq_lens=[L], n_q=1, h_q=1, h_kv=1, budgets=[B], keep_first=2, keep_last=32)
    k, v, wd, pd = to_dev_bf16(K), to_dev_bf16(V), dev_f32(w), dev_i32(pos)
    kw = {} if inplace else dict(K_out=torch.zeros_like(k), V_out=torch.zeros_like(v), weights_out=torch.zeros_like(wd), pos_out=torch.zeros_like(pd))
    Ko, Vo, wo, po, idx = jq.evict_weight(sh, k, v, wd, pd, **kw)
    torch.cuda.synchronize()
    newest = int(pos.max())
    kept = np.array(sorted(order(w[0, 0], pos[0, 0], L, 2, newest - 32)[:B]))
    assert set(range(L - 32, L)) <= set(kept.tolist())
    np.testing.assert_array_equal(idx[0, 0].cpu().numpy(), kept)
    np.testing.assert_array_equal(po[0, 0, :B].cpu().numpy(), pos[0, 0, kept])
    np.testing.assert_array_equal(wo[0, 0, :B].cpu().numpy().view(np.uint32), w[0, 0, kept].view(np.uint32))
    np.testing.assert_array_equal(from_dev_bf16(Ko)[0, :B, 0], K[0, kept, 0])
    np.testing.assert_array_equal(from_dev_bf16(Vo)[0, :B, 0], V[0, kept, 0])


@pytest.mark.parametrize("L", [40, 3000])
def test_a_new_token_takes_no_protected_row_beside_weights_of_all_ones(L):
    import torch
    rng = np.random.default_rng(L)
    k, v = (to_dev_bf16(bf16(rng, 1, L, 1, 128)) for _ in range(2))
    kn, vn = (to_dev_bf16(bf16(rng, 1, 1, 1, 128)) for _ in range(2))
    w = dev_f32(np.full((1, 1, L), ONES))
    pos = dev_i32(np.arange(L)[None, None])
    sh = jq.Shape(n_layers=1, seq_lens=[L], n_q=1, h_q=1, h_kv=1, keep_first=7, keep_last=5)
    slot = jq.replace_lightest(sh, kn, vn, dev_i32([L]), k, v, w, pos)
    torch.cuda.synchronize()
    assert int(slot) == 7 and int(pos[0, 0, 7]) == L and float(w[0, 0, 7]) == 0.0


def test_where_every_row_is_protected_the_lowest_goes():
    """Positions that repeat, or lie beyond the new token's, can leave no row to take: the lowest row is taken."""
    import torch
    rng = np.random.default_rng(3)
    k, v = (to_dev_bf16(bf16(rng, 1, 50, 1, 128)) for _ in range(2))
    kn, vn = (to_dev_bf16(bf16(rng, 1, 1, 1, 128)) for _ in range(2))
    w = dev_f32(rng.random((1, 1, 50)))
    pos = dev_i32(np.full((1, 1, 50), 99))
    sh = jq.Shape(n_layers=1, seq_lens=[50], n_q=1, h_q=1, h_kv=1, keep_first=7, keep_last=5)
    slot = jq.replace_lightest(sh, kn, vn, dev_i32([60]), k, v, w, pos)
    torch.cuda.synchronize()
    assert int(slot) == 0 and torch.equal(k[0, 0], kn[0, 0]) and torch.equal(v[0, 0], vn[0, 0]) and int(pos[0, 0, 0]) == 60


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("with_pos", [True, False])
def test_kept_rows_beyond_what_a_workgroup_holds(inplace, with_pos):
    """Pieces that leave more than 16384 rows to choose from, beside a short and a long sequence that are not cut; live counts at the
    edges of pieces, protected rows at both ends, ties."""
    from test_gpu_weight_eviction import evict
    caps, budgets = [150_001, 300, 16_384], [1800, 120, 9000]
    lens = np.array([[150_001, 300, 16_384], [131_073, 17, 16_383], [16_384, 0, 9001]], np.int32)
    evict(31, 3, caps, budgets, 1, lens=lens, inplace=inplace, first=3, last=40, ties=True, order="scrambled" if with_pos else "ascending", with_pos=with_pos)


@pytest.mark.parametrize("inplace", [False, True])
def test_pieces_with_budgets_of_each_layer(inplace):
    """Pieces have room for the largest budget of a sequence; a layer's own may be smaller, down to the protected rows."""
    from test_gpu_weight_eviction import evict
    evict(33, 3, [50_000, 700], [1200, 300], 2, layer_budgets=np.array([[1200, 300], [333, 1], [-5, 2 ** 31 - 1]], np.int32), inplace=inplace, first=3, last=12,
          ties=True, order="scrambled", lens=np.array([[50_000, 700], [32_769, 650], [49_151, 2]], np.int32))

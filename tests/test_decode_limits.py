"""Sizes up to which the decoding calls go: what fits the device is not refused, what no launch could hold is."""
import pytest

import paper_2509_10798_amd as jq
from test_decode_refusals import NULL, evict, pages


def bytes_of(weights=False, **kw):
    return jq.attend_workspace_bytes(jq.Shape(**dict(dict(n_layers=1, n_q=1, h_q=32, h_kv=8), **kw)), weights)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("h_q,h_kv", [(32, 8), (8, 8), (64, 4)])
def test_as_many_long_sequences_as_a_call_takes(h_q, h_kv, weights):
    """128 sequences of 131072 rows: 64 GiB of K and V a layer."""
    assert bytes_of(weights, seq_lens=[131072] * 128, h_q=h_q, h_kv=h_kv) > 0
    assert bytes_of(weights, seq_lens=[131072] * 127 + [7], h_q=h_q, h_kv=h_kv, n_layers=4) > 0


def test_query_rows_that_no_launch_holds():
    with pytest.raises(jq.JQError):
        bytes_of(seq_lens=[64] * 128, n_q=1 << 18, h_q=1024, h_kv=256)
    assert bytes_of(seq_lens=[4096], n_q=1 << 15) > 0


@pytest.mark.parametrize("layers", [65, 70, 1000])
def test_kept_rows_have_no_limit_of_their_own(layers):
    """2^28 kept (layer, row, head) rows and more, 128 GiB of K and V: the shape passes, the missing tensor is what is refused."""
    sh = jq.Shape(n_layers=layers, seq_lens=[4096] * 128, n_q=1, h_q=8, h_kv=8, pool_k=1, budgets=[4096] * 128)
    assert evict(sh, v=None) == NULL
    assert evict(sh, pg=pages(size=32, n=1 << 14, per=128), v=None) == NULL
    assert jq.evict_weight_workspace_bytes(sh) >= layers * 8 * 4096 * 128 * 4


@pytest.mark.gpu
def test_attention_over_as_many_long_sequences_as_a_call_takes():
    """64 GiB of K and V: keys of zeros, so that every row weighs the same, and one value a sequence."""
    import torch
    assert torch.cuda.is_available(), "this test needs the GPU"
    L, S, h_kv, h_q = 131072, 128, 8, 32
    K = torch.zeros((1, L * S, h_kv, 128), dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    for s in range(S):
        V[0, s * L:(s + 1) * L] = s + 1
    sh = jq.Shape(n_layers=1, seq_lens=[L] * S, n_q=1, h_q=h_q, h_kv=h_kv)
    w = torch.zeros((1, h_kv, L * S), device="cuda")
    Q = torch.ones((1, S, 1, h_q, 128), dtype=torch.bfloat16, device="cuda")
    out, lse = jq.attend(sh, Q, K, V, weights=w)
    torch.cuda.synchronize()
    # terms of 1 and sums of whole numbers below 2^24: out is off by its division and rounding, lse by a few roundings of 11.8
    assert torch.equal(out[0, :, 0].float(), torch.arange(1.0, S + 1, device="cuda")[:, None, None].expand(S, h_q, 128))
    assert (lse - 11.783502069519).abs().max() < 1e-5
    assert (w * L / 4 - 1).abs().max() < 1e-5

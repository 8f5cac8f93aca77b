"""Rows that hold a NaN, in the calls for k experts per token: they come out as NaN, and their neighbours' bits are those of a batch without them."""
import pytest
import torch

from paper_2308_15030_amd import binding as b
from test_ffn_mx_gpu import DEV, make, slots_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,d,f,T,k", [(3, 96, 160, 20, 1), (2, 416, 1696, 25, 2), (3, 96, 160, 700, 1), (2, 160, 2144, 900, 1), (2, 768, 768, 1024, 2)])
def test_nan_row_of_the_8_bit_products(K, d, f, T, k):
    """One NaN among a row's 8-bit values, in the streamed products and in tiles: all its features are NaN in front of the ReLU, and stay so."""
    L, w1, w2, held = make(K, K, d, f, T * k, K + d)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(DEV).bfloat16()
    L.slot.copy_(torch.from_numpy(slots_of(T * k, K, T, skew=0.5)))
    L.permute_topk(None, T, k)
    q, qs = L.mx_buffers(T)
    L.add_norm(x, T, torch.ones(d, device=DEV), 1e-6, q=q, q_scale=qs)
    clean = L.expert_ffn_mx(q, qs, T, k).clone().view(torch.bfloat16)
    bad = T // 2
    q[bad, 37] = 0x7F
    got = L.expert_ffn_mx(q, qs, T, k).view(torch.bfloat16)
    torch.cuda.synchronize()
    hit = L.perm // k == bad
    assert int(hit.sum()) == k and got[hit].isnan().all()
    assert torch.equal(got[~hit], clean[~hit]) and not clean.isnan().any()
    L.close()

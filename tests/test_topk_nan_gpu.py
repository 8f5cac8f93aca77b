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


@pytest.mark.parametrize("dtype,T", [(b.SMOE_F32, 20), (b.SMOE_F32, 700), (b.SMOE_BF16, 20), (b.SMOE_BF16, 700), (b.SMOE_MXFP8, 20), (b.SMOE_MXFP8, 700)])
@pytest.mark.parametrize("score,groups,best", [(b.SMOE_SCORE_SOFTMAX, 1, 1), (b.SMOE_SCORE_SIGMOID, 4, 2)])
@pytest.mark.parametrize("biased", [False, True])
def test_nan_token_of_a_pass(dtype, T, score, groups, best, biased):
    """As for one expert per token: the token's choices lie in range, each expert at most once, it has its places in the order, its row of the
    output is NaN; the other tokens' results are those of a batch without it."""
    E, K, d, f, k = 16, 16, 96, 160, 3
    act = torch.float32 if dtype == b.SMOE_F32 else torch.bfloat16
    g = torch.Generator().manual_seed(3)
    L = b.Layer(E, K, d, f, T * k, dtype, router_w=0.2 * torch.randn(E, d, generator=g))
    for s in range(K):
        L.set_resident(s, s, *(torch.randn(n, generator=g).to(act).to(DEV) / 10 for n in (d * f, d * f)))
    x = torch.randn(T, d, generator=g).to(act).to(DEV)
    bias = (0.1 * torch.randn(E, generator=g)).to(DEV) if biased else None
    rule = b.smoe_topk_rule(k, score, groups, max(1, groups // 2), best)
    q, qs = L.mx_buffers(T) if dtype == b.SMOE_MXFP8 else (None, None)
    bad, y, runs = T // 2, torch.empty_like(x), []
    for with_nan in (False, True):
        if with_nan:
            x[bad, 5] = float("nan")
        out = L.block_topk(x, T, torch.ones(d, device=DEV), 1e-6, rule, y, bias=bias, accumulate=0, q=q, q_scale=qs)
        torch.cuda.synchronize()
        runs.append([t.clone().view(T, -1) for t in (L.orig_expert, L.orig_gate, L.slot, L.gate)] + [L.out[:T].view(act).clone(), L.perm.clone(), L.inv_perm.clone()])
    clean, got = runs
    for ids, gates in ((got[0], got[1]), (got[2], got[3])):
        assert (ids >= 0).all() and (ids < E).all() and len(set(ids[bad].tolist())) == k and gates[bad].isnan().all()
    assert torch.equal(got[5].sort().values, torch.arange(T * k, dtype=torch.int32, device=DEV))
    assert torch.equal(got[5][got[6].long()], torch.arange(T * k, dtype=torch.int32, device=DEV))
    assert got[4][bad].isnan().all()
    rest = torch.arange(T, device=DEV) != bad
    for a, c in zip(got[:5], clean[:5]):
        assert torch.equal(a[rest], c[rest])
    L.close()


@pytest.mark.parametrize("dtype,T", [(b.SMOE_F32, 600), (b.SMOE_BF16, 300), (b.SMOE_F32, 40)])
def test_nan_expert(dtype, T):
    """A router row with a NaN: by their sigmoids its expert is chosen only where there is no other, last, and other weights do not see it."""
    E, d, k = 8, 64, 7
    g = torch.Generator().manual_seed(5)
    router = 0.2 * torch.randn(E, d, generator=g)
    router[2, 7] = float("nan")
    act = torch.float32 if dtype == b.SMOE_F32 else torch.bfloat16
    x = torch.randn(T, d, generator=g).to(act).to(DEV)
    L = b.Layer(E, E, d, 32, T * (k + 1), dtype, router_w=router)
    w = torch.zeros(d * 32, dtype=act, device=DEV)
    for s in range(E):
        L.set_resident(s, s, w, w)
    for bias in (None, torch.zeros(E, device=DEV)):
        L.route_topk(x, T, b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID), bias)
        seven = L.slot[:T * k].view(T, k).clone()
        assert torch.equal(seven.sort(1).values, torch.tensor([0, 1, 3, 4, 5, 6, 7], dtype=torch.int32, device=DEV).expand(T, k))
        gate = L.gate[:T * k].view(T, k)
        assert (gate.sum(1) - 1).abs().max() < 1e-5 and torch.equal(gate, L.orig_gate[:T * k].view(T, k))
        L.route_topk(x, T, b.smoe_topk_rule(k + 1, b.SMOE_SCORE_SIGMOID, renorm=0), bias)
        eight, gate = L.slot.view(T, k + 1), L.gate.view(T, k + 1)
        assert torch.equal(eight[:, :k], seven) and (eight[:, k] == 2).all() and gate[:, k].isnan().all() and not gate[:, :k].isnan().any()
    L.close()

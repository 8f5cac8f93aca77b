"""Batches that take smoe_route_topk's one launch, in every instance of it, with tokens whose choices are nearer than an fp32 logit can tell: fp32 beyond the
sizes of the launches for few tokens, and workgroups with none, one, some and all of their tokens to be repeated."""
import numpy as np
import pytest
import torch

from paper_2308_15030_amd import binding as b
from test_topk_gpu import DEV, _check_route, _route_case, act, layer

pytestmark = pytest.mark.gpu
SIG, SOFT = b.SMOE_SCORE_SIGMOID, b.SMOE_SCORE_SOFTMAX


@pytest.mark.parametrize("E,d,T,k", [(8, 36, 520, 2), (20, 100, 513, 4), (33, 260, 545, 3), (64, 768, 600, 6), (100, 516, 600, 6), (128, 1024, 1024, 8), (256, 288, 530, 16)])
@pytest.mark.parametrize("score", [SOFT, SIG])
def test_fp32_batches(E, d, T, k, score):
    router, x, resident, g = _route_case(E, max(2, E // 3), d, T, b.SMOE_F32, E + d + k, 0.05)
    L = layer(E, len(resident), d, T * k + 3, b.SMOE_F32, router, resident)
    bias = (0.05 * torch.randn(E, generator=g)).to(DEV)
    for rule, bb in ((b.smoe_topk_rule(k, score), None), (b.smoe_topk_rule(k, score, renorm=0, scale=2.5), bias)):
        _check_route(L, x.to(DEV), T, rule, bb, router, resident, b.SMOE_F32)
    L.close()


@pytest.mark.parametrize("E,groups,kept,k", [(20, 4, 2, 5), (64, 8, 4, 8), (64, 16, 3, 6), (96, 3, 2, 4), (66, 11, 5, 7), (256, 8, 3, 16)])
@pytest.mark.parametrize("best", [1, 2])
def test_fp32_groups(E, groups, kept, k, best):
    d, T = 132, 540
    for K in (1, E // 6):
        router, x, resident, g = _route_case(E, K, d, T, b.SMOE_F32, E * groups + K, 0.08)
        L = layer(E, K, d, T * k, b.SMOE_F32, router, resident)
        bias = (0.1 * torch.randn(E, generator=g)).to(DEV)
        for score, bb in ((SIG, None), (SIG, bias), (SOFT, bias)):
            _check_route(L, x.to(DEV), T, b.smoe_topk_rule(k, score, groups, kept, best, 1, 1.5), bb, router, resident, b.SMOE_F32)
        L.close()


def _pairs(E, d, g, apart=0.5):
    """A router whose rows 2 i and 2 i + 1 differ by one unit in the last place in column 0, and by `apart` in column 1: a token whose column 1 is zero
    has them nearer than fp32 can tell, one with a 1 there has not."""
    router = 0.1 * torch.randn(E, d, generator=g)
    router[1::2] = router[::2][:E // 2]
    router[:, 0] = 0.25
    router[1::2, 0] = torch.nextafter(router[1::2, 0], torch.tensor(1.0))
    router[:, 1] = 0
    router[1::2, 1] = apart
    return router


@pytest.mark.parametrize("dtype,E,d,T", [(b.SMOE_BF16, 20, 96, 96), (b.SMOE_BF16, 64, 352, 96), (b.SMOE_BF16, 64, 96, 8300), (b.SMOE_BF16, 100, 288, 96), (b.SMOE_MXFP8, 128, 64, 8300),
                                         (b.SMOE_BF16, 200, 64, 96), (b.SMOE_BF16, 256, 224, 96), (b.SMOE_F32, 20, 100, 520), (b.SMOE_F32, 64, 36, 520),
                                         (b.SMOE_F32, 100, 132, 520), (b.SMOE_F32, 256, 100, 520)])
@pytest.mark.parametrize("how", ["softmax-bias", "softmax", "sigmoid-bias", "sigmoid-groups", "equal"])
def test_workgroups_with_some_tokens_to_repeat(dtype, E, d, T, how):
    """0, 1, 2, 5, 6, 7, 8, 9 and all tokens of a block of 32 (two of them make a workgroup of long batches).  Where all logits of a token are repeated,
    the whole workgroup takes up to 6 tokens one after the other, and from 7 on a wave each."""
    K, k = E // 2, 5
    g = torch.Generator().manual_seed(E + T)
    router = _pairs(E, d, g)
    if how == "equal":
        router[1::2, 0] = 0.25
    x = torch.randn(T, d, generator=g)
    x[:, 0], x[:, 1] = 1, 1
    counts = [1, 0, 2, 5, 6, 7, 8, 9, 32, 6, 0, 1, 32, 7]
    for i, at in enumerate(range(0, T, 32)):
        n = min(counts[(i + E) % len(counts)], T - at)
        x[at + torch.randperm(min(32, T - at), generator=g)[:n], 1] = 0
    x = x.to(act(dtype))
    resident = torch.randperm(E, generator=g)[:K].tolist()
    L = layer(E, K, d, T * k, dtype, router, resident)
    bias = (0.003 * torch.randn((E + 1) // 2, generator=g)).repeat_interleave(2)[:E].to(DEV)
    rule, bb = {"softmax-bias": (b.smoe_topk_rule(k, SOFT), bias), "softmax": (b.smoe_topk_rule(k, SOFT, renorm=0), None),
                "sigmoid-bias": (b.smoe_topk_rule(k, SIG), bias), "sigmoid-groups": (b.smoe_topk_rule(k, SIG, 4, 2, 2), bias),
                "equal": (b.smoe_topk_rule(k, SOFT), bias)}[how]
    _check_route(L, x.to(DEV), T, rule, bb, router, resident, dtype)
    L.close()


@pytest.mark.parametrize("E,groups", [(20, 4), (64, 8), (100, 4), (256, 8)])
@pytest.mark.parametrize("how", ["near", "near-bias", "near-groups", "softmax-bias"])
def test_fp32_near_ties(E, groups, how):
    """Every token near a tie, fp32."""
    K, d, T, k = E // 3, 196, 530, 4
    g = torch.Generator().manual_seed(E)
    router = _pairs(E, d, g, 0.0)
    x = torch.randn(T, d, generator=g)
    resident = torch.randperm(E, generator=g)[:K].tolist()
    L = layer(E, K, d, T * k, b.SMOE_F32, router, resident)
    bias = (0.01 * torch.arange(E // 2).repeat_interleave(2)).float().to(DEV)
    rule, bb = {"near": (b.smoe_topk_rule(k, SOFT), None), "near-bias": (b.smoe_topk_rule(k, SIG), bias),
                "near-groups": (b.smoe_topk_rule(k, SIG, groups, 3, 2), None), "softmax-bias": (b.smoe_topk_rule(k, SOFT, groups, 3, 2), bias)}[how]
    _check_route(L, x.to(DEV), T, rule, bb, router, resident, b.SMOE_F32)
    L.close()

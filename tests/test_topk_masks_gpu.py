"""Biases that keep experts out with large finite numbers, -infinity or the lowest float: the choices are those of float64, down to where masked experts
have to be taken, and a batch costs what it costs without masked experts."""
import numpy as np
import pytest
import torch

from paper_2308_15030_amd import binding as b
from test_topk_gpu import DEV, _check_route, _route_case, act, layer

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(torch.float32).min


def time_us(call, n=10):
    for _ in range(3):
        call()
    best = float("inf")
    for _ in range(5):
        a, e = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(n):
            call()
        e.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(e) / n * 1e3)
    return best


@pytest.mark.parametrize("mask", [-1e9, -30000.0, LOWEST, 1e9])
@pytest.mark.parametrize("dtype,E,d,T", [(b.SMOE_BF16, 64, 1024, 30), (b.SMOE_BF16, 64, 256, 200), (b.SMOE_MXFP8, 24, 64, 50), (b.SMOE_F32, 24, 100, 600),
                                         (b.SMOE_BF16, 200, 64, 700)])
@pytest.mark.parametrize("score,groups,kept,best", [("softmax", 1, 1, 1), ("sigmoid", 1, 1, 1), ("sigmoid", 4, 2, 2), ("softmax", 4, 3, 2), ("sigmoid", 8, 7, 2)])
@pytest.mark.parametrize("left", [2, 0.25, 0.75])
def test_masked_experts(mask, dtype, E, d, T, score, groups, kept, best, left):
    """`left` experts, or that share of them, are not masked.  Where fewer than k are left, masked ones are chosen by what float64 keeps of their
    scores: of -1e9 steps of 2^-23, of the lowest float nothing (the lowest id)."""
    K, k = E // 2, 4
    router, x, resident, g = _route_case(E, K, d, T, dtype, E + T, 0.05)
    L = layer(E, K, d, T * k + 3, dtype, router, resident)
    bias = torch.full((E,), mask)
    on = torch.randperm(E, generator=g)[:left if left == 2 else int(left * E)]
    bias[on] = 0.1 * torch.randn(len(on), generator=g)
    rule = b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX, groups, kept, best, 1, 1.5)
    _check_route(L, x.to(DEV), T, rule, bias.to(DEV), router, resident, dtype)
    L.close()


@pytest.mark.parametrize("mask", [-np.inf, -1e9, LOWEST])
@pytest.mark.parametrize("score,groups,kept,best", [("sigmoid", 8, 4, 2), ("softmax", 1, 1, 1)])
@pytest.mark.parametrize("dtype", [b.SMOE_BF16, b.SMOE_F32])
def test_masked_experts_take_no_longer(dtype, mask, score, groups, kept, best):
    """A quarter of the experts masked: at most twice the time of the same batch with none (it was 10 to 25 times, every token being repeated in 64
    bits; 30 us are allowed for a few more or fewer tokens that are)."""
    E, d, T, k = 128, 1024, 16384, 8
    router, x, resident, g = _route_case(E, 32, d, T, dtype, 1)
    L = layer(E, 32, d, T * k, dtype, router, resident)
    x = x.to(DEV)
    rule = b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX, groups, kept, best)
    bias = 0.05 * torch.randn(E, generator=g)
    masked = bias.clone()
    masked[::4] = mask
    plain, with_mask = (time_us(lambda v=v: L.route_topk(x, T, rule, v)) for v in (bias.to(DEV), masked.to(DEV)))
    assert with_mask <= 2 * plain + 30, (plain, with_mask)
    L.close()

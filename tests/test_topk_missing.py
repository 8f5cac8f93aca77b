"""Experts switched off by a bias of -infinity, down to fewer than k of them and none: what cannot be had is expert -1 among all and slot -1 among the
resident ones, weight 0, and nothing behind the router takes it for a choice."""
import numpy as np
import pytest
import torch

import topk_reference as ref
from paper_2308_15030_amd import binding as b


def test_a_missing_choice_asks_for_no_load():
    h = b.smoe_create(7, 3, 64, 64, 16, b.SMOE_F32)
    cs, ce = np.empty(3, np.int32), np.empty(3, np.int32)
    assert b.smoe_on_demand_plan(h, np.array([-1, 5, -1, -1, 2, 5], np.int32), 6, cs, ce) == 2
    assert cs[:2].tolist() == [0, 1] and ce[:2].tolist() == [5, 2]
    assert b.smoe_on_demand_plan(h, np.array([-1, -1], np.int32), 2, cs, ce) == 0
    with pytest.raises(b.SmoeError) as e:
        b.smoe_on_demand_plan(h, np.array([-2], np.int32), 1, cs, ce)
    assert e.value.status == b.SMOE_EINVAL
    b.smoe_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,E,d,T", [(b.SMOE_BF16, 64, 1024, 30), (b.SMOE_BF16, 64, 1024, 200), (b.SMOE_MXFP8, 24, 64, 50), (b.SMOE_F32, 24, 100, 30),
                                         (b.SMOE_F32, 24, 100, 600), (b.SMOE_BF16, 200, 64, 9000)])
@pytest.mark.parametrize("left", [0, 1, 3, 9])
@pytest.mark.parametrize("score,groups,kept,best", [("softmax", 1, 1, 1), ("sigmoid", 1, 1, 1), ("sigmoid", 4, 2, 2), ("softmax", 4, 3, 2), ("sigmoid", 4, 3, 1)])
def test_experts_switched_off(dtype, E, d, T, left, score, groups, kept, best):
    from test_topk_gpu import DEV, _check_route, _route_case, f64, layer
    K, k = E // 2, 5
    router, x, resident, g = _route_case(E, K, d, T, dtype, E + T, 0.05)
    L = layer(E, K, d, T * k + 3, dtype, router, resident)
    bias = torch.full((E,), -np.inf)
    on = torch.randperm(E, generator=g)[:left]
    bias[on] = 0.1 * torch.randn(left, generator=g)
    rule = b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX, groups, kept, best, 1, 1.5)
    _check_route(L, x.to(DEV), T, rule, bias.to(DEV), router, resident, dtype)
    want = L.orig_expert[:T * k].cpu().numpy()
    assert (want == -1).any() == (left < k or groups > 1 and (want == -1).any())
    L.importance(T * k, 0)
    torch.cuda.synchronize()
    assert np.array_equal(L.count.cpu().numpy(), np.bincount(want[want >= 0], minlength=E))
    gate, xn = f64(L.orig_gate[:T * k]), f64(L.xnorm[:T * k])
    score_of = np.zeros(E)
    np.add.at(score_of, want[want >= 0], (gate * xn)[want >= 0])
    assert np.allclose(f64(L.score), score_of, rtol=1e-4)
    plan = L.on_demand_plan(T * k)
    assert sorted(e for _, e in plan) == sorted(set(want[want >= 0].tolist()) - set(resident))[:len(plan)] or len(plan) == K
    L.close()

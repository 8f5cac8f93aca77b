"""Rows of zeros, as a padded batch has them, among others: all their logits are equal, the biases or the lowest ids decide, and the batch takes no longer
for them.  And rows so small that their squares underflow."""
import numpy as np
import pytest
import torch

import topk_reference as ref
from paper_2308_15030_amd import binding as b
from test_topk_gpu import DEV, _check_route, _route_case, act, f64, layer
from test_topk_masks_gpu import time_us

pytestmark = pytest.mark.gpu
RULES = [("softmax", 1, 1, 1, None), ("sigmoid", 1, 1, 1, None), ("sigmoid", 4, 2, 2, None), ("softmax", 4, 2, 2, None), ("sigmoid", 8, 3, 2, "some"),
         ("softmax", 8, 3, 2, "some"), ("sigmoid", 1, 1, 1, "some"), ("softmax", 1, 1, 1, "zero"), ("sigmoid", 4, 3, 2, "zero"), ("sigmoid", 1, 1, 1, "signed"), ("softmax", 4, 2, 2, "signed"), ("sigmoid", 4, 2, 1, "steps"),
         ("sigmoid", 4, 2, 2, "steps"), ("sigmoid", 1, 1, 1, "inf")]


def _bias(how, E, g):
    if how is None:
        return None
    v = 0.1 * torch.randn(E, generator=g) if how != "zero" else torch.zeros(E)
    if how == "inf":
        v[::3] = -np.inf
    if how == "signed":                                    # zeros of either sign, which are equal
        v = torch.where(torch.rand(E, generator=g) < 0.5, -0.0, 0.0)
    if how == "steps":                                     # many equal ones
        v = 0.125 * torch.randint(-1, 2, (E,), generator=g)
    return v.to(DEV)


@pytest.mark.parametrize("dtype,E,d,T", [(b.SMOE_BF16, 64, 1024, 30), (b.SMOE_BF16, 64, 1056, 333), (b.SMOE_MXFP8, 24, 64, 50), (b.SMOE_F32, 24, 100, 601),
                                         (b.SMOE_BF16, 200, 64, 700), (b.SMOE_BF16, 40, 32, 8300)])
@pytest.mark.parametrize("score,groups,kept,best,bias", RULES)
def test_rows_of_zeros(dtype, E, d, T, score, groups, kept, best, bias):
    K, k = E // 2, 4
    router, x, resident, g = _route_case(E, K, d, T, dtype, E + T, 0.05)
    x[T // 2:] = 0                                         # padding at the end
    x[T // 2 + 1::3] = -0.0
    x[5:T // 2:4] = 0                                      # and between
    L = layer(E, K, d, T * k + 3, dtype, router, resident)
    rule = b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX, groups, kept, best, 1, 1.5)
    _check_route(L, x.to(DEV), T, rule, _bias(bias, E, g), router, resident, dtype)
    L.close()


@pytest.mark.parametrize("dtype,E,d,T", [(b.SMOE_BF16, 64, 256, 200), (b.SMOE_F32, 24, 100, 601), (b.SMOE_BF16, 200, 64, 300)])
@pytest.mark.parametrize("size", [1e-12, 1e-16, 1e-22, 1e-36])
def test_rows_whose_squares_underflow(dtype, E, d, T, size):
    """Choices among logits of that size, near ties (router rows in pairs that differ in the last places) included."""
    K, k = E // 2, 4
    router, x, resident, g = _route_case(E, K, d, T, dtype, E + T, 0.5)
    router[1::2] = router[::2]
    router[1::2, :3] = torch.nextafter(router[1::2, :3], torch.tensor(9.0))
    x[::2] = (x[::2].float() * size).to(act(dtype))
    L = layer(E, K, d, T * k, dtype, router, resident)
    L.route_topk(x.to(DEV), T, b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID))
    torch.cuda.synchronize()
    z = f64(x) @ f64(router).T                             # (a sigmoid near 1/2 keeps less of such logits than they do)
    for name, held in (("orig_expert", np.arange(E)), ("slot", np.array(resident))):
        order = np.lexsort((held[None].repeat(T, 0), -z[:, held]), axis=1)[:, :k]
        want = held[order] if name == "orig_expert" else order
        assert np.array_equal(getattr(L, name).cpu().numpy().reshape(T, k), want), name
    L.close()


@pytest.mark.parametrize("score,groups,kept,best,bias", [("sigmoid", 8, 4, 2, None), ("sigmoid", 8, 4, 2, "zero"), ("softmax", 1, 1, 1, None), ("softmax", 1, 1, 1, "zero")])
@pytest.mark.parametrize("dtype", [b.SMOE_BF16, b.SMOE_F32])
def test_padding_takes_no_longer(dtype, score, groups, kept, best, bias):
    """Half of the rows zeros: at most twice the time of a batch without (it was 5 to 25 times; 30 us are allowed for a few more tokens that are
    repeated in 64 bits)."""
    E, d, T, k = 128, 1024, 16384, 8
    router, x, resident, g = _route_case(E, 32, d, T, dtype, 1)
    L = layer(E, 32, d, T * k, dtype, router, resident)
    x = x.to(DEV)
    padded = x.clone()
    padded[T // 2:] = 0
    rule = b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX, groups, kept, best)
    bv = _bias(bias, E, g)
    plain, half = (time_us(lambda v=v: L.route_topk(v, T, rule, bv)) for v in (x, padded))
    assert half <= 2 * plain + 30, (plain, half)
    L.close()

"""Weights of served experts whose logits lie far below the best expert's, and of sigmoids far below 0: divided by their sum they do not depend on how
small each is by itself, on either side of the batch sizes where the launches change."""
import numpy as np
import pytest
import torch

import topk_reference as ref
from paper_2308_15030_amd import binding as b
from test_topk_gpu import DEV, U, act, f64, layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,E,d,T", [(b.SMOE_BF16, 64, 1024, 128), (b.SMOE_BF16, 64, 1024, 129), (b.SMOE_BF16, 20, 64, 40), (b.SMOE_MXFP8, 128, 64, 70),
                                         (b.SMOE_BF16, 200, 64, 9000), (b.SMOE_F32, 20, 64, 512), (b.SMOE_F32, 20, 64, 513), (b.SMOE_F32, 200, 64, 520)])
@pytest.mark.parametrize("gap", [50, 90, 104, 120, 800])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_weights_far_below_the_best(dtype, E, d, T, gap, score):
    """Logits are multiples of 1/32 below 2^11, exact in fp32, and the chosen ones are at least 1/32 apart: a weight's relative error is that of two
    exponentials (2 units of 2^-23 each), the sum 1 + e^-|l|, two quotients and a sum of k weights, less than 16 roundings of 2^-24 each way.  Below
    2^-126 numbers are multiples of 2^-149: an exponential is off by 2 of these units at most, a quotient by half of one, the product with the scale, 1.5 times that, by
    half of one more: 1.5 (2 + 1/2 + 1/2) + 1/2 = 5 units."""
    k, K = 4, 7
    g = torch.Generator().manual_seed(gap + E)
    resident = (3 + torch.randperm(E - 3, generator=g)[:K]).tolist()
    router = torch.zeros(E, d)
    router[3:, 0] = -gap                                   # all but the first three, which nobody holds
    if score == "sigmoid":
        router[:3, 0] = -gap
    router[:, 1] = torch.randperm(E, generator=g) / 8
    x = torch.zeros(T, d)
    x[:, 0] = 1
    x[:, 1] = torch.tensor([0.25, 0.5, 1.0])[torch.randint(0, 3, (T,), generator=g)]
    L = layer(E, K, d, T * k, dtype, router, resident)
    L.route_topk(x.to(act(dtype)).to(DEV), T, b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX, scale=1.5))
    torch.cuda.synchronize()
    logits = f64(x) @ f64(router).T
    for name, held in (("orig", np.arange(E)), ("served", np.array(resident))):
        l = logits[:, held]
        order = np.argsort(-l, axis=1, kind="stable")[:, :k]
        l = np.take_along_axis(l, order, 1)
        p = np.minimum(l, 0) if score == "sigmoid" else l  # a common factor e^m left out
        w = np.exp(p - p.max(1, keepdims=True)) / (1 + np.exp(-np.abs(l)) if score == "sigmoid" else 1)
        w *= 1.5 / w.sum(1, keepdims=True)
        got = f64(L.orig_gate if name == "orig" else L.gate).reshape(T, k)
        ids = (L.orig_expert if name == "orig" else L.slot).cpu().numpy().reshape(T, k)
        assert np.array_equal(ids, held[order] if name == "orig" else order), name
        assert (np.abs(got - w) <= 32 * U * w + 5 * 2.0 ** -149).all(), (name, np.abs(got / w - 1).max())
    L.close()


def test_reference_agrees_where_nothing_underflows():
    """The weights above are those of the tests' oracle wherever its scores are numbers."""
    l = np.array([[-50.0, -51.5, -49.25]])
    s = 1 / (1 + np.exp(-l))
    ids, w = ref.choose(s[0], s[0], 3, 1, 1, 1, True, 1.0)
    p = np.exp(np.minimum(l, 0) + 49.25) / (1 + np.exp(-np.abs(l)))
    assert ids == [2, 0, 1] and np.allclose(sorted(w), np.sort(p / p.sum())[0], rtol=1e-12)

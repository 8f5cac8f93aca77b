"""Rows that follow a router row for part of the columns and its negative for the rest, so that the sums of a logit grow and vanish again and their
roundings are large beside it, with pairs of experts nearer than these: the choices are those of 64-bit sums."""
import numpy as np
import pytest
import torch

from paper_2308_15030_amd import binding as b
from test_topk_gpu import DEV, act, layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,E,d,period", [(b.SMOE_BF16, 64, 1024, 256), (b.SMOE_BF16, 64, 4096, 4096), (b.SMOE_BF16, 64, 16384, 16384), (b.SMOE_BF16, 128, 2048, 2048),
                                              (b.SMOE_BF16, 16, 16384, 16384), (b.SMOE_MXFP8, 8, 128, 0), (b.SMOE_F32, 64, 1024, 256), (b.SMOE_F32, 64, 4096, 1024),
                                              (b.SMOE_F32, 16, 16384, 2048), (b.SMOE_F32, 128, 768, 0)])
@pytest.mark.parametrize("apart", [1.5, 3, 8])
def test_sums_that_grow_and_vanish(dtype, E, d, period, apart):
    """Experts 2 i and 2 i + 1 of the first eight are `apart` 2^-24 |x| |w| apart on average, the others' rows small; period 0: rows that follow all of a
    router row.  float64 tells them apart: it is off by 10^-8 of that.  The batches are beyond those of the launches for few tokens."""
    T, k, wrong = 16384, 2, 0
    for seed in range(12):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def rand(*shape):
            return torch.randn(*shape, device=DEV, generator=g, dtype=torch.float64)
        base = rand(E // 2, d) / d ** 0.5
        base[4:] *= 0.02
        router = torch.stack([base, base], 1).reshape(E, d).float()
        near = apart * 2.0 ** -24 * d ** 0.5
        router[1::2] = (router[::2].double() * (1 + near * rand(E // 2, d))).float()
        sign = 1.0 if period == 0 else torch.where(torch.arange(d, device=DEV) % period < period // 2, 1.0, -1.0)
        x = (sign * base[torch.randint(0, 4, (T,), device=DEV, generator=g)] * d ** 0.5 + 0.02 * rand(T, d)).to(act(dtype))
        L = layer(E, E, d, T * k, dtype, router, range(E))
        L.route_topk(x, T, b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID))
        torch.cuda.synchronize()
        z = (x.double() @ router.double().T).cpu().numpy()
        want = np.argsort(-z, axis=1, kind="stable")[:, :k]
        wrong += int((L.orig_expert.cpu().numpy().reshape(T, k) != want).any(1).sum())
        L.close()
    assert wrong == 0

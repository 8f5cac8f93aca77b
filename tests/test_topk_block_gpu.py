"""What block_topk and forward_topk refuse, before anything is launched, and the buffers that may lie over each other."""
import pytest
import torch

from paper_2308_15030_amd import binding as b
from test_ffn_mx_gpu import DEV, _pass_case

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.mark.parametrize("dtype", [b.SMOE_F32, b.SMOE_BF16, b.SMOE_MXFP8])
def test_the_norm_may_not_lie_over_the_stream(dtype):
    """Without a buffer for the sum x itself is added to the layer's result, so y over x would add y."""
    T, k = 30, 2
    L, w1, w2, router, resident, x, r, nw, act = _pass_case(dtype, T, k)
    rule = b.smoe_topk_rule(k)
    q, qs = L.mx_buffers(T) if dtype == b.SMOE_MXFP8 else (None, None)
    kept = x.clone()
    for bad in (dict(y=x), dict(y=r, residual=r, total=r), dict(y=x, residual=r, total=x)):
        with pytest.raises(ValueError):
            L.block_topk(x, T, nw, EPS, rule, q=q, q_scale=qs, **bad)
    assert torch.equal(x, kept)
    want = L.block_topk(x, T, nw, EPS, rule, torch.empty_like(x), out=torch.empty_like(x), q=q, q_scale=qs).clone()
    assert torch.equal(x, kept)                            # the stream is only read
    inplace = L.block_topk(x, T, nw, EPS, rule, torch.empty_like(x), out=x, q=q, q_scale=qs)
    torch.cuda.synchronize()
    assert inplace is x and torch.equal(x, want)
    # with a buffer for the sum y may lie over x or the residual, and the result over y
    total = torch.empty_like(x)
    want = L.block_topk(kept, T, nw, EPS, rule, torch.empty_like(x), residual=r, total=total, out=torch.empty_like(x), q=q, q_scale=qs).clone()
    for over in ("x", "residual"):
        a, c = kept.clone(), r.clone()
        y = a if over == "x" else c
        got = L.block_topk(a, T, nw, EPS, rule, y, residual=c, total=torch.empty_like(x), out=y, q=q, q_scale=qs)
        torch.cuda.synchronize()
        assert torch.equal(got, want), over
    L.close()


def test_8_bit_layers_need_the_rows_in_8_bits():
    T, k = 12, 2
    L, w1, w2, router, resident, x, r, nw, act = _pass_case(b.SMOE_MXFP8, T, k)
    L.count.fill_(5)
    q, qs = L.mx_buffers(T)
    for kw in (dict(), dict(q=q), dict(q_scale=qs)):
        with pytest.raises(ValueError):
            L.forward_topk(x, T, b.smoe_topk_rule(k), **kw)
        with pytest.raises(ValueError):
            L.block_topk(x, T, nw, EPS, b.smoe_topk_rule(k), torch.empty_like(x), **kw)
    torch.cuda.synchronize()
    assert (L.count == 5).all()                            # nothing has been counted
    L.close()

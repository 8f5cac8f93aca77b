"""k experts per token at the edges of what the calls allow: arrays past 2^31 elements and 2^32 bytes, the first call after one that was only
captured, and timing events."""
import numpy as np
import pytest
import torch

import topk_reference as ref
from paper_2308_15030_amd import binding as b
from test_ffn_mx_gpu import DEV, bank, expected, f64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("d,f", [(16384, 32), (512, 16384)])
def test_offsets_past_32_bits(d, f):
    """A block of 140000 tokens, 2 experts each: rows (d = 16384) or hidden activations (f = 16384) past 2^32 bytes.  The first, the last
    and some tokens between, against float64 from the rows in 8 bits on."""
    T, k, E, K = 140000, 2, 8, 3
    w1, w2 = bank(E, d, f, 5)
    L = b.Layer(E, K, d, f, T * k, b.SMOE_MXFP8, router_w=0.02 * torch.randn(E, d, generator=torch.Generator().manual_seed(5)))
    held = [1, 4, 6]
    for s, e in enumerate(held):
        L.set_resident(s, e, w1[e], w2[e])
    x = torch.randn(T, d, device=DEV, dtype=torch.bfloat16, generator=torch.Generator(device=DEV).manual_seed(1))
    nw = torch.rand(d, device=DEV) + 0.5
    y = torch.empty_like(x)
    q, qs = L.mx_buffers(T)
    rule = b.smoe_topk_rule(k)
    L.block_topk(x, T, nw, 1e-6, rule, y, q=q, q_scale=qs)
    torch.cuda.synchronize()
    assert int(L.offsets[-1]) == T * k and int(L.inv_perm[:T * k].long().sum()) == T * k * (T * k - 1) // 2
    at = torch.tensor([0, 1, 65535, 65536, 131071, 131072, T - 2, T - 1], device=DEV)
    xd = f64(x[at])
    h = xd / np.sqrt((xd ** 2).mean(1, keepdims=True) + 1e-6) * f64(nw)
    # a lane adds at most 64 squares, then 6 + 16 sums of lanes and waves: half of it through the root; two products; one rounding to bf16
    assert (np.abs(f64(y[at]) - h) <= np.abs(h) * (2.0 ** -8 + 64 * U)).all()
    xv = ref.from_blocks(ref.e4m3_values(q[at].cpu().numpy()), qs[at].cpu().numpy().astype(int)[:, :d // 32] - 127)
    # half a step of e4m3 of normal values, half a step at the block's bottom below
    s = np.repeat(2.0 ** (qs[at].cpu().numpy().astype(float)[:, :d // 32] - 127), 32, axis=1)
    assert (np.abs(xv - h) <= np.maximum(np.abs(h) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 64 * U) + np.abs(h) * 64 * U).all()
    slot, gate = (v[:T * k].view(T, k)[at].cpu().numpy() for v in (L.slot, L.gate))
    want, far, size = xd.copy(), np.zeros_like(xd), np.abs(xd)
    for sl, e in enumerate(held):
        ys, fs = expected(xv, f64(w1[e]), f64(w2[e]))
        g = np.where(slot == sl, gate.astype(np.float64), 0).sum(1)[:, None]
        want, far, size = want + g * ys, far + g * fs, size + g * np.abs(ys)
    assert (np.abs(f64(L.out[:T].view(torch.bfloat16)[at]) - want) <= far + 2.0 ** -8 * (np.abs(want) + far) + (k + 1) * U * size).all()
    # as it would be used with rows of the layer's type: sorted rows past 2^32 bytes
    L.permute_topk(y, T, k)
    torch.cuda.synchronize()
    pos = L.inv_perm[:T * k].view(T, k)[at].long()
    for j in range(k):
        assert torch.equal(L.x_perm[pos[:, j]].view(torch.bfloat16), y[at])
    L.close()


@pytest.mark.parametrize("dtype", [b.SMOE_BF16, b.SMOE_MXFP8])
@pytest.mark.parametrize("first", ["route", "route_topk"])
def test_first_call_after_a_capture(first, dtype):
    """What a captured call prepares is not there before a replay: the next eager call prepares its own."""
    E, K, d, T, k = 16, 8, 256, 200, 2
    router = torch.randn(E, d, generator=torch.Generator().manual_seed(3))
    w1, w2 = bank(E, d, 64, 3)
    x = torch.randn(T, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).bfloat16()
    layers = [b.Layer(E, K, d, 64, T * k, dtype, router_w=router) for _ in range(2)]
    for L in layers:
        for s in range(K):
            L.set_resident(s, s, w1[s], w2[s])
    rule = b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID)
    late, plain = layers
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        late.route(x, T) if first == "route" else late.route_topk(x, T, rule)
    for L in layers:
        L.route_topk(x, T, rule)
    torch.cuda.synchronize()
    for name in ("orig_expert", "orig_gate", "slot", "gate", "xnorm"):
        assert torch.equal(getattr(late, name)[:T * k], getattr(plain, name)[:T * k]), name
    late.close(), plain.close()


@pytest.mark.parametrize("T", [5, 700])
def test_events_take_the_products_times(T):
    """As for smoe_expert_ffn: four events for the next call, used once."""
    E, d, f, k = 4, 128, 256, 2
    w1, w2 = bank(E, d, f, 7)
    L = b.Layer(E, E, d, f, T * k, b.SMOE_MXFP8)
    for s in range(E):
        L.set_resident(s, s, w1[s], w2[s])
    x = torch.randn(T, d, device=DEV).bfloat16()
    q, qs = L.mx_buffers(T)
    L.add_norm(x, T, torch.ones(d, device=DEV), 1e-6, q=q, q_scale=qs)
    L.route_topk(x, T, b.smoe_topk_rule(k))
    L.permute_topk(None, T, k)
    plain = L.expert_ffn_mx(q, qs, T, k).clone()
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
    for e in ev:
        e.record()
    torch.cuda.synchronize()
    b.smoe_set_profile_events(L.handle, *ev)
    for _ in range(2):                                     # the second call has none
        L.y_perm.zero_()
        L.expert_ffn_mx(q, qs, T, k)
        torch.cuda.synchronize()
        assert torch.equal(L.y_perm, plain)
        assert 0 < ev[0].elapsed_time(ev[1]) < 100 and 0 < ev[2].elapsed_time(ev[3]) < 100
    L.close()


@pytest.mark.parametrize("E,d,T,dtype", [(33, 100, 511, b.SMOE_F32), (33, 100, 512, b.SMOE_F32), (33, 100, 513, b.SMOE_F32), (64, 1024, 128, b.SMOE_BF16),
                                         (64, 1024, 129, b.SMOE_BF16), (64, 992, 128, b.SMOE_BF16), (129, 512, 127, b.SMOE_MXFP8)])
def test_route_where_the_launches_change(E, d, T, dtype):
    """Few tokens take two launches, more of them one: both sides of the borders, against float64."""
    from test_topk_gpu import _check_route, _route_case, layer
    K, k = E // 3, 4
    router, x, resident, g = _route_case(E, K, d, T, dtype, E + T, 0.05)
    L = layer(E, K, d, T * k + 3, dtype, router, resident)
    bias = (0.05 * torch.randn(E, generator=g)).to(DEV)
    _check_route(L, x.to(DEV), T, b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID, renorm=0), bias, router, resident, dtype)
    _check_route(L, x.to(DEV), T, b.smoe_topk_rule(k), None, router, resident, dtype)
    L.close()

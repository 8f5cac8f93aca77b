"""Experts' products on 8-bit values (smoe_expert_ffn_mx), loads into 8-bit slots, and whole passes with k experts per token, against
plain float64 on weights and rows rounded to blocks of 32.

Tolerance of a product.  The matrix unit adds 8 consecutive products at a time, each rounded to a unit of at most 2^-13 of the largest
of the 8; the roundings are independent, a third of a unit squared each in the mean at most, so a sum of g such groups is off by less
than six standard deviations, dh = 6 sqrt(8/3 sum_g unit_g^2), and by the roundings of the fp32 accumulator, one a step and some, 2^-24 of
the sum of magnitudes each.  Where a hidden value h is further than dh from every border of its rounding, the 8-bit value is the
reference's; elsewhere it is off by at most a whole step, 2^-3 |h| or 2^-9 units, and where the block's largest magnitude is within dh of a
border of the scale, that holds for its 32 values, with the larger unit.  The second product adds those, again independent, through w2, and
has its own sums and one rounding to bf16, 2^-8."""
import numpy as np
import pytest
import torch

import topk_reference as ref
from paper_2308_15030_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f64(t):
    return t.detach().double().cpu().numpy()


def bank(n, d, f, seed, spread=False):
    """n experts in bank layout, bf16; spread: columns of very different size."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = [torch.randn(n, r, c, device=DEV, generator=g) * (torch.exp(3 * torch.randn(n, 1, c, device=DEV, generator=g)) if spread else 1) / r ** 0.5
         for r, c in ((d, f), (f, d))]
    return [v.bfloat16() for v in w]


def rows8(L, x):
    """8-bit rows of x by the oracle, in the library's layout, and the values they stand for."""
    q, e = ref.to_blocks(f64(x))
    by = np.searchsorted(ref.E4M3, np.abs(q)).astype(np.uint8) | np.where(np.signbit(q), 128, 0).astype(np.uint8)
    T, d = x.shape
    dq, ds = L.mx_buffers(T)
    dq.copy_(torch.from_numpy(by))
    ds.fill_(0xFF)                                         # bytes behind the last block are not used, NaN scales though they are
    ds[:, :d // 32].copy_(torch.from_numpy((e + 127).astype(np.uint8)))
    return dq, ds, ref.from_blocks(q, e)


def sums_off(a, m):
    """How far the matrix unit's a @ m may be off (above)."""
    pad = -a.shape[1] % 64
    a, m = np.pad(np.abs(a), ((0, 0), (0, pad))), np.pad(np.abs(m), ((0, pad), (0, 0)))
    units = np.zeros((a.shape[0], m.shape[1]))
    for g in range(0, a.shape[1], 8):
        big = np.zeros_like(units)
        for i in range(g, g + 8):
            big = np.maximum(big, a[:, i:i + 1] * m[i])
        units += (2.0 ** -13 * big) ** 2
    return 6 * np.sqrt(8 / 3 * units) + (a.shape[1] // 64 + 12) * 2.0 ** -24 * (a @ m)


def expected(xv, w1, w2):
    """(y, how far it may be off) of rows of one slot."""
    w1, w2 = ref.round_columns(w1), ref.round_columns(w2)
    y, h = ref.expert_ffn(xv, w1, w2)
    dh = sums_off(xv, w1)
    n = h.shape[0]
    hb, db = h.reshape(n, -1, 32), dh.reshape(n, -1, 32)
    amax = np.abs(hb).max(-1, keepdims=True)
    e = ref.scale_exponent(amax[..., 0])[..., None]
    s = 2.0 ** e.astype(np.float64)
    reach = db.max(-1, keepdims=True)
    moved = (ref.scale_exponent((amax + reach)[..., 0]) != e[..., 0]) | (ref.scale_exponent(np.maximum(amax - reach, 0)[..., 0]) != e[..., 0])
    lo, hi = (ref.to_blocks((hb + sign * db).reshape(n, -1)) for sign in (-1, 1))
    near = (ref.from_blocks(*lo) != ref.from_blocks(*hi)).reshape(hb.shape) | moved[..., None]
    step = np.where(near, np.maximum(2.0 ** -3 * np.abs(hb), 2.0 ** -9 * 2 * s) + db, 0).reshape(n, -1)
    hq = ref.from_blocks(*ref.to_blocks(h))
    return y, 6 * np.sqrt(step ** 2 @ w2 ** 2) + sums_off(hq, w2) + 2.0 ** -8 * np.abs(y) + 1e-30


def check(L, x, slot, k, w1, w2, held):
    """held: expert of each slot."""
    T, n = x.shape[0], x.shape[0] * k
    dq, ds, xv = rows8(L, x)
    L.slot[:n].copy_(torch.from_numpy(slot.astype(np.int32)))
    L.permute_topk(None, T, k)
    L.y_perm.fill_(77)
    L.expert_ffn_mx(dq, ds, T, k)
    torch.cuda.synchronize()
    perm, inv, off = ref.sort_pairs(slot, L.K)
    got = f64(L.y_perm[:n].view(torch.bfloat16))
    assert (L.y_perm[off[-1]:] == 77).all()                # rows behind the last segment
    for s in range(L.K):
        rows = perm[off[s]:off[s + 1]]
        if len(rows):
            y, far = expected(xv[rows // k], f64(w1[held[s]]), f64(w2[held[s]]))
            bad = np.abs(got[off[s]:off[s + 1]] - y) > far
            assert not bad.any(), (s, np.argwhere(bad)[:4], np.abs(got[off[s]:off[s + 1]] - y).max())


def make(E, K, d, f, pairs, seed=0, spread=False, spare=0):
    w1, w2 = bank(E, d, f, seed, spread)
    L = b.Layer(E, K, d, f, pairs, b.SMOE_MXFP8, router_w=0.1 * torch.randn(E, d, generator=torch.Generator().manual_seed(seed)), spare_slots=spare)
    for s in range(K):
        L.set_resident(s, (s * 5 + 1) % E if K * 5 % E else s, w1[(s * 5 + 1) % E if K * 5 % E else s], w2[(s * 5 + 1) % E if K * 5 % E else s])
    return L, w1, w2, L.maps()[0]


def slots_of(n, K, seed, skew=1.0, lost=0.0):
    rng = np.random.default_rng(seed)
    p = np.arange(1, K + 1.0) ** -skew
    if K > 2:
        p[K // 2] = 0
    s = rng.choice(K, size=n, p=p / p.sum())
    s[rng.random(n) < lost] = -1
    return s


@pytest.mark.parametrize("K,d,f,T,k,lost", [(1, 32, 32, 1, 1, 0), (2, 64, 64, 3, 2, 0), (3, 96, 160, 7, 2, .2), (4, 32, 288, 40, 1, 0), (5, 288, 32, 33, 3, .1),
                                            (3, 416, 1696, 50, 2, 0), (16, 768, 1024, 13, 2, 0), (70, 64, 96, 60, 4, 0), (2, 1024, 512, 31, 1, 1.0)])
def test_few_rows_a_slot(K, d, f, T, k, lost):
    E = K + 3
    L, w1, w2, held = make(E, K, d, f, T * k + 4, K + d)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(DEV)
    check(L, x, slots_of(T * k, K, T, lost=lost), k, w1, w2, held)
    L.close()


@pytest.mark.parametrize("K,d,f,T,k,lost", [(1, 32, 32, 200, 1, 0), (1, 96, 288, 129, 1, 0), (2, 160, 544, 300, 2, .1), (3, 416, 1696, 400, 2, 0), (3, 256, 256, 999, 1, 0),
                                            (70, 64, 96, 2500, 2, .02), (2, 64, 2080, 65, 8, 0), (4, 1056, 96, 700, 1, 0), (2, 768, 768, 1024, 2, 0)])
def test_many_rows_a_slot(K, d, f, T, k, lost):
    E = K + 3
    L, w1, w2, held = make(E, K, d, f, T * k + 4, K + d)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(DEV)
    check(L, x, slots_of(T * k, K, T, skew=0.5, lost=lost), k, w1, w2, held)
    L.close()


@pytest.mark.parametrize("T,form", [(300, 2), (900, 4), (2600, 8)])
@pytest.mark.parametrize("d,f,which", [(96, 2080, 0), (2080, 96, 1), (160, 2144, 0), (2144, 224, 1)])
def test_every_width_of_tiles(d, f, which, T, form):
    """Either product on tiles of 2, 4 and 8 feature blocks, with odd numbers of blocks, steps and half steps, and ragged slots."""
    K = 3
    L, w1, w2, held = make(K, K, d, f, T)
    name = b.smoe_describe_ffn(L.handle, T).split(" | ")[which]
    assert name.startswith(f"tile_mx_kernel<{'false' if which else 'true'}, {form},"), name
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(DEV)
    check(L, x, slots_of(T, K, T, skew=0.7, lost=0.05), 1, w1, w2, held)
    L.close()


@pytest.mark.parametrize("T", [9, 600])
def test_scales_that_spread(T):
    """Columns of the matrices and of the rows of sizes from 2^-12 to 2^12, zero rows, zero columns."""
    K, d, f = 2, 192, 224
    w1, w2 = bank(K, d, f, 3, spread=True)
    w1[0, :, :40] = 0
    w2[1, :64] = 0
    L = b.Layer(K, K, d, f, T, b.SMOE_MXFP8)
    for s in range(K):
        L.set_resident(s, s, w1[s], w2[s])
    g = torch.Generator().manual_seed(1)
    x = torch.randn(T, d, generator=g) * torch.exp(3 * torch.randn(T, d // 32, 1, generator=g)).expand(-1, -1, 32).reshape(T, d)
    x[0] = 0
    check(L, x.to(DEV), np.arange(T) % K, 1, w1, w2, [0, 1])
    L.close()


def test_without_perm_rows_are_tokens():
    K, d, f, T = 2, 64, 128, 20
    L, w1, w2, held = make(K, K, d, f, T)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(1)).to(DEV)
    dq, ds, xv = rows8(L, x)
    off = torch.tensor([0, 12, 20], dtype=torch.int32, device=DEV)
    y = torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    b.smoe_expert_ffn_mx(L.handle, dq, ds, None, 1, off, T, y)
    torch.cuda.synchronize()
    for s, (lo, hi) in enumerate(((0, 12), (12, 20))):
        want, far = expected(xv[lo:hi], f64(w1[held[s]]), f64(w2[held[s]]))
        assert (np.abs(f64(y)[lo:hi] - want) <= far).all()
    with pytest.raises(b.SmoeError) as e:
        b.smoe_expert_ffn_mx(L.handle, dq, ds, None, 2, off, T // 2, y)
    assert e.value.status == b.SMOE_EINVAL
    with pytest.raises(b.SmoeError) as e:
        L.expert_ffn(T)
    assert "smoe_expert_ffn_mx" in str(e.value)
    with pytest.raises(b.SmoeError):
        L.forward_fused(x.bfloat16(), T)
    L.close()


def test_loads_from_pinned_memory_and_updates():
    """A slot filled from pinned host memory and one filled by an asynchronous update hold the same bytes as one filled from the device."""
    E, K, d, f = 6, 2, 96, 160
    w1, w2 = bank(E, d, f, 4)
    h1, h2 = (torch.empty(w.shape, dtype=w.dtype, pin_memory=True).copy_(w) for w in (w1, w2))
    torch.cuda.synchronize()
    want = b.Layer(E, K, d, f, 8, b.SMOE_MXFP8)
    for s, e in enumerate((4, 5)):
        want.set_resident(s, e, w1[e], w2[e])
    torch.cuda.synchronize()
    one = want.slot_w1.numel() // K

    def bytes_of(L, phys):
        return torch.cat([w[p * one:(p + 1) * one] for w in (L.slot_w1, L.slot_w2) for p in phys])
    pinned = b.Layer(E, K, d, f, 8, b.SMOE_MXFP8)
    for t in (want, pinned):                              # the larger of two matrices sets the stride: the rest of the smaller is never written
        assert t.slot_w1.numel() == K * one
    n1, n2 = (-(-r // 64) * 2048 + -(-r // 256) * 256 for r in (d, f))
    n1, n2 = n1 * f // 32, n2 * d // 32
    for s, e in enumerate((4, 5)):
        pinned.set_resident(s, e, h1[e], h2[e])
    for banks in ((w1, w2), (h1, h2)):
        L = b.Layer(E, K, d, f, 8, b.SMOE_MXFP8, spare_slots=1)
        for s in range(K):
            L.set_resident(s, s, w1[s], w2[s])
        side = torch.cuda.Stream()
        assert L.update_begin(np.array([0, 0, 0, 0, 2, 1], np.float32)) == 2
        for _ in range(200):
            L.update_tick(*banks, side)
            if not L.update_pending():
                break
            torch.cuda.synchronize()
        assert sorted(L.maps()[0].tolist()) == [4, 5]
        phys = [None, None]
        x = torch.randn(8, d, generator=torch.Generator().manual_seed(1)).to(DEV)
        check(L, x, np.arange(8) % K, 1, w1, w2, L.maps()[0])
        L.close()
    torch.cuda.synchronize()
    for s in range(K):
        assert torch.equal(want.slot_w1[s * one:s * one + n1], pinned.slot_w1[s * one:s * one + n1])
        assert torch.equal(want.slot_w2[s * one:s * one + n2], pinned.slot_w2[s * one:s * one + n2])
    want.close(), pinned.close()


# ------------------------------------------------------------------ whole passes
def _pass_case(dtype, T, k, d=96, f=160, E=12, K=6, seed=0):
    act = torch.float32 if dtype == b.SMOE_F32 else torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(seed)
    w1, w2 = (v.to(act) for v in bank(E, d, f, seed))
    router = 0.2 * torch.randn(E, d, generator=torch.Generator().manual_seed(seed))
    L = b.Layer(E, K, d, f, max(T * k, 1), dtype, router_w=router)
    resident = list(range(1, 2 * K, 2))
    for s, e in enumerate(resident):
        L.set_resident(s, e, w1[e], w2[e])
    L.expert_norm.copy_(L.expert_norm_of(w1, w2))
    x, r = (torch.randn(T, d, device=DEV, generator=g).to(act) for _ in range(2))
    nw = 1 + 0.1 * torch.randn(d, device=DEV, generator=g)
    return L, w1, w2, router, resident, x, r, nw, act


@pytest.mark.parametrize("dtype", [b.SMOE_F32, b.SMOE_BF16, b.SMOE_MXFP8])
@pytest.mark.parametrize("T,k", [(1, 1), (1, 2), (19, 2), (300, 3)])
def test_block(T, k, dtype):
    """norm -> route -> importance -> sort -> FFN -> weighted sum, from the library's own intermediate results step by step: each step has
    its own tests, here the steps hand each other the right things."""
    L, w1, w2, router, resident, x, r, nw, act = _pass_case(dtype, T, k)
    rule = b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID, 4, 3, 2, 1, 1.5)
    bias = (0.1 * torch.randn(L.E, generator=torch.Generator().manual_seed(3))).to(DEV)
    total, y, out = (torch.empty_like(x) for _ in range(3))
    q, qs = L.mx_buffers(T) if dtype == b.SMOE_MXFP8 else (None, None)
    got = L.block_topk(x, T, nw, 1e-6, rule, y, residual=r, total=total, bias=bias, accumulate=0, out=out, q=q, q_scale=qs)
    assert got is out
    torch.cuda.synchronize()
    e2s = np.full(L.E, -1)
    e2s[resident] = np.arange(L.K)
    want = ref.route(f64(y), router.double().numpy(), e2s, k, True, f64(bias), 4, 3, 2, True, 1.5)
    n = T * k
    slot, gate = L.slot.cpu().numpy()[:n].reshape(T, k), f64(L.gate)[:n].reshape(T, k)
    assert np.array_equal(slot, want["slot"]) and np.allclose(gate, want["gate"], rtol=2e-5)
    # importance over the pairs, by the choices among all experts
    oe = want["orig_expert"].reshape(-1)
    assert np.array_equal(L.count.cpu().numpy(), np.bincount(oe, minlength=L.E))
    eq1 = np.zeros(L.E)
    np.add.at(eq1, oe, np.repeat(want["xnorm"], k) * want["orig_gate"].reshape(-1))
    assert np.allclose(f64(L.score), eq1 * f64(L.expert_norm), rtol=1e-4)
    acc, far = f64(total), np.zeros((T, L.d_model))
    tv = f64(total)
    if dtype == b.SMOE_MXFP8:
        yv = ref.from_blocks(ref.e4m3_values(q.cpu().numpy()), qs.cpu().numpy().astype(int)[:, :L.d_model // 32] - 127)
    else:
        yv = f64(y)
    for t in range(T):
        for j in range(k):
            s = slot[t, j]
            if s < 0:
                continue
            a, c = f64(w1[resident[s]]), f64(w2[resident[s]])
            if dtype == b.SMOE_MXFP8:
                e, d = expected(yv[t:t + 1], a, c)
            else:
                h = np.maximum(yv[t:t + 1] @ a, 0)
                e = h @ c
                step = 2.0 ** -8 if dtype == b.SMOE_BF16 else 2.0 ** -18
                d = step * (np.abs(h) @ np.abs(c)) + step * np.abs(e)    # the hidden values and the result, each rounded once
            acc[t] += gate[t, j] * e[0]
            far[t] += gate[t, j] * d[0]
    last = 2.0 ** -8 if dtype != b.SMOE_F32 else 2.0 ** -20
    assert (np.abs(f64(out) - acc) <= 1.01 * far + last * np.abs(acc) + 2.0 ** -18 * (np.abs(tv) + np.abs(acc))).all()
    L.close()


@pytest.mark.parametrize("dtype", [b.SMOE_BF16, b.SMOE_MXFP8])
@pytest.mark.parametrize("T", [3, 400])
def test_block_replays_from_a_graph_and_on_another_stream(T, dtype):
    """A pass captured into a graph, replayed with other inputs and eager work in between, gives the eager bits; so does the same pass
    on another stream; two layers do not disturb each other."""
    k = 2
    L, w1, w2, router, resident, x, r, nw, act = _pass_case(dtype, T, k)
    other = _pass_case(dtype, T, k, seed=9)[0]
    rule = b.smoe_topk_rule(k)
    total, y, out = (torch.empty_like(x) for _ in range(3))
    q, qs = L.mx_buffers(T) if dtype == b.SMOE_MXFP8 else (None, None)
    x_in = torch.empty_like(x)

    def go():
        L.block_topk(x_in, T, nw, 1e-6, rule, y, residual=r, total=total, accumulate=0, out=out, q=q, q_scale=qs)
    inputs = [x, x.flip(0) * 2, torch.zeros_like(x)]
    names = ("slot", "perm", "offsets", "count", "score", "gate")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    x_in.copy_(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):         # the first pass of all: what a bind leaves to do is captured too
            go()
    torch.cuda.current_stream().wait_stream(side)
    want = []
    for v in inputs:
        x_in.copy_(v)
        go()
        torch.cuda.synchronize()
        want.append([getattr(L, n).clone() for n in names] + [out.clone(), total.clone()])
    for rep in range(3):
        for v, w in zip(inputs, want):
            x_in.copy_(v)
            out.zero_()
            L.slot.fill_(-3)
            torch.cuda.synchronize()
            graph.replay()
            o2 = torch.empty_like(out)
            other.route_topk(x, T, rule)                   # another layer's work
            torch.cuda.synchronize()
            n = T * k
            served = int(w[2][-1])
            for name, a, c in zip(names, [getattr(L, m) for m in names], w):
                lim = served if name == "perm" else n if name in ("slot", "gate") else len(a)
                assert torch.equal(a[:lim], c[:lim]), (rep, name)
            assert torch.equal(out, w[-2]) and torch.equal(total, w[-1])
    x_in.copy_(inputs[0])
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0][-2])
    L.close(), other.close()


def test_describe_names_the_kernels():
    L = b.Layer(4, 4, 64, 64, 4096, b.SMOE_MXFP8)
    few, many = b.smoe_describe_ffn(L.handle, 8), b.smoe_describe_ffn(L.handle, 4096)
    assert "stream_mx_kernel" in few and "tile_mx_kernel" in many
    with pytest.raises(ValueError):
        L.block_topk(None, 1, None, 1e-6, b.smoe_topk_rule(1), None, residual=torch.zeros(1, 64))
    L.close()

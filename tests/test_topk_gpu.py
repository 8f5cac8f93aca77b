"""smoe_add_norm, smoe_route_topk, smoe_permute_topk and smoe_combine_topk through the C ABI against plain float64.

Roundings counted in the tolerances: a result rounded to bf16 is off by at most 2^-8 of itself, an fp32 one by 2^-24, an e4m3 one by 2^-4
(or half the smallest step, 2^-10 units).  Whole numbers are equal: choices nearer than an fp32 logit can tell are decided in 64 bits."""
import numpy as np
import pytest
import torch

import topk_reference as ref
from paper_2308_15030_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ROUND = {b.SMOE_F32: U, b.SMOE_BF16: 2.0 ** -8, b.SMOE_MXFP8: 2.0 ** -8}


def act(dtype):
    return torch.float32 if dtype == b.SMOE_F32 else torch.bfloat16


def f64(t):
    return t.detach().double().cpu().numpy()


def layer(E, K, d, pairs, dtype, router=None, resident=None, f=32):
    L = b.Layer(E, K, d, f, pairs, dtype, router_w=router)
    if resident is not None:
        w = torch.zeros(d * f, dtype=act(dtype), device=DEV)
        for s, e in enumerate(resident):
            L.set_resident(s, int(e), w, w)
    return L


# ------------------------------------------------------------------ norm
@pytest.mark.parametrize("dtype", [b.SMOE_F32, b.SMOE_BF16])
@pytest.mark.parametrize("T,d", [(1, 32), (3, 96), (2, 512), (33, 544), (1, 768), (257, 1024), (5, 1056), (4, 2048), (3, 4160), (2, 8192),
                                 (2, 8224), (1, 65536)])
def test_add_norm(T, d, dtype):
    g = torch.Generator().manual_seed(T * d)
    col = torch.exp(torch.randn(d, generator=g))
    x, r = (torch.randn(T, d, generator=g).to(act(dtype)).to(DEV), (torch.randn(T, d, generator=g) * col).to(act(dtype)).to(DEV))
    x[:, :32] = -r[:, :32]                                # a block that cancels to zero
    w = (1 + 0.1 * torch.randn(d, generator=g)).to(DEV)
    L = layer(1, 1, d, T, dtype)
    for res in (r, None):
        total, y = (torch.full((T, d), 7.0, dtype=act(dtype), device=DEV) for _ in range(2))
        q, qs = L.mx_buffers(T)
        qs.fill_(0xEE)
        L.add_norm(x, T, w, 1e-6, res, total, y, q, qs)
        torch.cuda.synchronize()
        h, want = ref.add_norm(f64(x), None if res is None else f64(res), f64(w), 1e-6)
        # h: one fp32 rounding; y: the sum of squares (64 lanes x at most 64 terms and a tree) by half, the scale, two products
        assert (np.abs(f64(total) - h) <= np.abs(h) * (ROUND[dtype] + U)).all()
        near = 64 * U
        assert (np.abs(f64(y) - want) <= np.abs(want) * (ROUND[dtype] + near)).all()
        e = qs.cpu().numpy().astype(int)[:, :d // 32] - 127
        assert (qs.cpu().numpy()[:, d // 32:] == 0).all()
        amax = np.abs(want).reshape(T, -1, 32).max(-1)
        s = 2.0 ** e.astype(float)
        assert (amax * (1 - near) <= 448 * s).all() and ((amax * (1 + near) > 224 * s) | (e == -126)).all()
        got = ref.from_blocks(ref.e4m3_values(q.cpu().numpy()), e)
        half = np.maximum(np.abs(want) * 2.0 ** -4, np.repeat(s, 32, 1) * 2.0 ** -10)
        assert (np.abs(got - want) <= half * (1 + 2.0 ** -10)).all()
    L.close()


def test_add_norm_odd_width_in_place_and_parts():
    """fp32 rows of 4 mod 8 values; outputs over the inputs; every output alone gives the same bits; rows behind T stay."""
    T, d = 7, 1036
    g = torch.Generator().manual_seed(3)
    x, r, w = (torch.randn(*s, generator=g).to(DEV) for s in ((T + 2, d), (T + 2, d), (d,)))
    L = layer(1, 1, d, T + 2, b.SMOE_F32)
    total, y = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    L.add_norm(x, T, w, 1e-5, r, total, y)
    torch.cuda.synchronize()
    h, want = ref.add_norm(f64(x)[:T], f64(r)[:T], f64(w), 1e-5)
    assert (np.abs(f64(total)[:T] - h) <= np.abs(h) * 2 * U).all() and (np.abs(f64(y)[:T] - want) <= np.abs(want) * 64 * U).all()
    assert (total[T:] == 9).all() and (y[T:] == 9).all()
    y2, t2 = torch.empty_like(x), torch.empty_like(x)
    L.add_norm(x, T, w, 1e-5, r, None, y2)
    L.add_norm(x, T, w, 1e-5, r, t2)
    assert torch.equal(y2[:T], y[:T]) and torch.equal(t2[:T], total[:T])
    x2, r2 = x.clone(), r.clone()
    L.add_norm(x2, T, w, 1e-5, r2, r2, x2)                # the stream in place, the result over x
    assert torch.equal(r2[:T], total[:T]) and torch.equal(x2[:T], y[:T])
    L.close()


def test_add_norm_of_zeros_and_extremes():
    L = layer(1, 1, 64, 4, b.SMOE_F32)
    x = torch.zeros(4, 64, device=DEV)
    x[1] = 1e-20
    x[2] = 1e18
    x[3, 0] = 1.0
    w, y = torch.ones(64, device=DEV), torch.empty_like(x)
    q, qs = L.mx_buffers(4)
    L.add_norm(x, 4, w, 1e-6, None, None, y, q, qs)
    torch.cuda.synchronize()
    got = ref.from_blocks(ref.e4m3_values(q.cpu().numpy()), qs.cpu().numpy().astype(int)[:, :2] - 127)
    assert (y[0] == 0).all() and (got[0] == 0).all()
    assert np.allclose(f64(y)[1], 1e-17, rtol=1e-6) and np.allclose(f64(y)[2], 1.0, rtol=1e-6)
    assert np.allclose(f64(y)[3, 0], 8.0, rtol=1e-4) and (f64(y)[3, 1:] == 0).all() and (got[3, 1:] == 0).all()
    L.close()


# ------------------------------------------------------------------ router
def _route_case(E, K, d, T, dtype, seed, scale=0.02):
    g = torch.Generator().manual_seed(seed)
    router = scale * torch.randn(E, d, generator=g)
    x = (torch.randn(8, d, generator=g)[torch.randint(0, 8, (T,), generator=g)] + 0.5 * torch.randn(T, d, generator=g)).to(act(dtype))
    resident = torch.randperm(E, generator=g)[:K].tolist()
    return router, x, resident, g


def _check_route(L, x, T, rule, bias, router, resident, dtype):
    E, k = L.E, rule.k
    e2s = np.full(E, -1)
    e2s[resident] = np.arange(len(resident))
    for t in (L.orig_expert, L.slot):
        t.fill_(-9)
    L.route_topk(x, T, rule, bias)
    torch.cuda.synchronize()
    xd, wd = f64(x), f64(router)
    want = ref.route(xd, wd, e2s, k, rule.score == b.SMOE_SCORE_SIGMOID, None if bias is None else f64(bias), rule.groups,
                     rule.groups_kept, rule.group_best, bool(rule.renorm), rule.scale)
    n = T * k
    for name in ("orig_expert", "slot"):
        got = getattr(L, name).cpu().numpy()
        assert np.array_equal(got[:n].reshape(T, k), want[name]), name
        assert (got[n:] == -9).all()
    # a logit is off by at most (2.5 + n / 10) 2^-24 |x| |w| (n roundings of partial sums); a weight by four times that and some roundings
    steps = 3 * d_steps(L.d_model) if dtype != b.SMOE_F32 else L.d_model // 2
    far = (2.5 + 0.1 * steps) * U * want["xnorm"].max() * np.linalg.norm(wd, axis=1).max()
    for name in ("orig_gate", "gate"):
        got = f64(getattr(L, name))[:n].reshape(T, k)
        assert (np.abs(got - want[name]) <= np.abs(want[name]) * (4 * far + 32 * U)).all(), name
    got = f64(L.xnorm)[:n].reshape(T, k)
    assert (np.abs(got - want["xnorm"][:, None]) <= want["xnorm"][:, None] * L.d_model / 16 * U).all()


def d_steps(d):
    return d // 16


@pytest.mark.parametrize("dtype", [b.SMOE_F32, b.SMOE_BF16, b.SMOE_MXFP8])
@pytest.mark.parametrize("E,K,d,T,k", [(8, 2, 64, 1, 1), (8, 8, 64, 5, 8), (33, 11, 96, 70, 3), (64, 16, 768, 31, 2), (100, 30, 512, 130, 6),
                                       (128, 32, 1056, 65, 8), (256, 40, 288, 40, 16), (20, 16, 32, 257, 16)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_topk(E, K, d, T, k, score, dtype):
    router, x, resident, g = _route_case(E, K, d, T, dtype, E + d + k, 0.05)
    L = layer(E, K, d, T * k + 3, dtype, router, resident)
    code = b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX
    bias = (0.05 * torch.randn(E, generator=g)).to(DEV)
    for rule, bb in ((b.smoe_topk_rule(k, code), None), (b.smoe_topk_rule(k, code, renorm=0, scale=2.5), bias),
                     (b.smoe_topk_rule(k, code), bias)):
        _check_route(L, x.to(DEV), T, rule, bb, router, resident, dtype)
    L.close()


@pytest.mark.parametrize("E,groups,kept,k", [(64, 8, 4, 8), (64, 16, 3, 6), (60, 4, 2, 5), (24, 2, 1, 4), (96, 3, 2, 4), (256, 4, 2, 16),
                                             (16, 16, 4, 4), (8, 2, 2, 8), (128, 2, 1, 3), (66, 11, 5, 7)])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_groups(E, groups, kept, k, best, score):
    """Groups of every kind: sizes that are powers of two and not, one expert a group, across the chunks of 64; few residents, so that
    groups are left without any and tokens get fewer than k choices."""
    d, T = 128, 90
    code = b.SMOE_SCORE_SIGMOID if score == "sigmoid" else b.SMOE_SCORE_SOFTMAX
    for K in (1, max(2, E // 6)):
        router, x, resident, g = _route_case(E, K, d, T, b.SMOE_BF16, E * groups + K, 0.08)
        L = layer(E, K, d, T * k, b.SMOE_BF16, router, resident)
        bias = (0.1 * torch.randn(E, generator=g)).to(DEV)
        for bb in (None, bias):
            _check_route(L, x.to(DEV), T, b.smoe_topk_rule(k, code, groups, kept, best, 1, 1.5), bb, router, resident, b.SMOE_BF16)
        L.close()


@pytest.mark.parametrize("dtype", [b.SMOE_F32, b.SMOE_BF16])
@pytest.mark.parametrize("how", ["equal", "near", "near-bias", "near-groups", "softmax-bias"])
def test_route_ties_and_near_ties(how, dtype):
    """Rows of the router in pairs: equal (the lowest id wins) or apart by single units in the last place of a few weights, which an fp32
    logit cannot tell: the choice is that of 64-bit arithmetic."""
    E, K, d, T, k = 32, 12, 192, 150, 4
    g = torch.Generator().manual_seed(5)
    base = 0.1 * torch.randn(E // 2, d, generator=g)
    router = torch.stack([base, base], 1).reshape(E, d).clone()
    if how != "equal":
        flip = torch.randint(0, d, (E // 2, 3), generator=g)
        for i in range(E // 2):
            router[2 * i + 1, flip[i]] = torch.nextafter(router[2 * i + 1, flip[i]], torch.tensor(1.0))
    x = torch.randn(T, d, generator=g).to(act(dtype))
    resident = torch.randperm(E, generator=g)[:K].tolist()
    L = layer(E, K, d, T * k, dtype, router, resident)
    sig, soft = b.SMOE_SCORE_SIGMOID, b.SMOE_SCORE_SOFTMAX
    rule, bias = {"equal": (b.smoe_topk_rule(k, soft), None), "near": (b.smoe_topk_rule(k, soft), None),
                  "near-bias": (b.smoe_topk_rule(k, sig), (0.01 * torch.arange(E // 2).repeat_interleave(2)).float()),
                  "near-groups": (b.smoe_topk_rule(k, sig, 8, 3, 2), None),
                  "softmax-bias": (b.smoe_topk_rule(k, soft, 8, 5, 2), (0.01 * torch.arange(E // 2).repeat_interleave(2)).float())}[how]
    _check_route(L, x.to(DEV), T, rule, None if bias is None else bias.to(DEV), router, resident, dtype)
    L.close()


def test_route_equal_groups_and_long_batch():
    """All group ranks equal (the router repeats): the lowest groups are kept.  And a batch of the kernels' two-block form."""
    E, d, T, k = 64, 64, 80, 4
    g = torch.Generator().manual_seed(8)
    router = (0.1 * torch.randn(8, d, generator=g)).repeat(8, 1)
    x = torch.randn(T, d, generator=g).bfloat16()
    L = layer(E, E, d, T * k, b.SMOE_BF16, router, range(E))
    _check_route(L, x.to(DEV), T, b.smoe_topk_rule(k, b.SMOE_SCORE_SIGMOID, 8, 2, 2), None, router, list(range(E)), b.SMOE_BF16)
    L.close()
    for E, d in ((32, 64), (32, 1088), (128, 64)):
        router, x, resident, g = _route_case(E, 8, d, 8300, b.SMOE_BF16, E + d, 0.1)
        L = layer(E, 8, d, 8300 * 2, b.SMOE_BF16, router, resident)
        _check_route(L, x.to(DEV), 8300, b.smoe_topk_rule(2), None, router, resident, b.SMOE_BF16)
        L.close()


def test_route_topk_of_one_is_the_top_one_route():
    """k = 1 with softmax over all: the choices, slots and gates of smoe_route (without renormalisation, gate over all experts)."""
    E, K, d, T = 64, 16, 256, 333
    router, x, resident, g = _route_case(E, K, d, T, b.SMOE_BF16, 2, 0.1)
    L = layer(E, K, d, T, b.SMOE_BF16, router, resident)
    L.route(x.to(DEV), T)
    torch.cuda.synchronize()
    want = [getattr(L, n).clone() for n in ("orig_expert", "slot", "orig_gate", "gate", "xnorm")]
    L.route_topk(x.to(DEV), T, b.smoe_topk_rule(1, renorm=0))
    torch.cuda.synchronize()
    got = [getattr(L, n) for n in ("orig_expert", "slot", "orig_gate", "gate", "xnorm")]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for a, c in zip(got[2:], want[2:]):
        assert torch.allclose(a, c, rtol=1e-6, atol=0)
    L.close()


def test_route_nan_rows_stay_in_range():
    E, K, d, T, k = 16, 6, 64, 40, 3
    router, x, resident, g = _route_case(E, K, d, T, b.SMOE_BF16, 4, 0.1)
    x[7] = float("nan")
    L = layer(E, K, d, T * k, b.SMOE_BF16, router, resident)
    clean = x.clone()
    clean[7] = 0
    for score, groups in ((b.SMOE_SCORE_SOFTMAX, 1), (b.SMOE_SCORE_SIGMOID, 4)):
        rule = b.smoe_topk_rule(k, score, groups, max(1, groups // 2), 1)
        L.route_topk(clean.to(DEV), T, rule)
        want = [getattr(L, n).clone().view(T, k) for n in ("orig_expert", "slot", "gate")]
        L.route_topk(x.to(DEV), T, rule)
        torch.cuda.synchronize()
        got = [getattr(L, n).view(T, k) for n in ("orig_expert", "slot", "gate")]
        keep = torch.arange(T, device=DEV) != 7
        for a, c in zip(got, want):
            assert torch.equal(a[keep], c[keep])
        assert (got[0] >= 0).all() and (got[0] < E).all() and (got[1] >= -1).all() and (got[1] < K).all()
    L.close()


def test_route_topk_refuses_bad_rules():
    router, x, resident, g = _route_case(12, 4, 64, 8, b.SMOE_BF16, 1)
    L = layer(12, 4, 64, 64, b.SMOE_BF16, router, resident)
    for kw in (dict(score=2), dict(groups=0), dict(groups=5), dict(groups=3, groups_kept=0), dict(groups=3, groups_kept=4), dict(group_best=0),
               dict(group_best=3), dict(renorm=2), dict(scale=float("inf")), dict(scale=float("nan")), dict(k=5, groups=3, groups_kept=1)):
        with pytest.raises(b.SmoeError) as e:
            L.route_topk(x.to(DEV), 8, b.smoe_topk_rule(**{**dict(k=2), **kw}))
        assert e.value.status == b.SMOE_EINVAL, kw
    L.route_topk(x.to(DEV), 0, b.smoe_topk_rule(2))       # an empty batch is legal
    L.close()


# ------------------------------------------------------------------ sorting and weighted sum
@pytest.mark.parametrize("T,k,K,d", [(0, 2, 4, 64), (1, 1, 1, 32), (1, 16, 20, 64), (5, 3, 2, 96), (64, 2, 16, 768), (333, 3, 11, 416), (1024, 2, 256, 64),
                                     (700, 6, 70, 128), (9000, 4, 8, 32), (600, 8, 16, 4096), (5000, 8, 3, 64)])
@pytest.mark.parametrize("dtype", [b.SMOE_F32, b.SMOE_BF16])
def test_permute_and_combine(T, k, K, d, dtype):
    rng = np.random.default_rng(T * k + K)
    p = np.arange(1, K + 1.0) ** -1.1
    if K > 2:
        p[K // 2] = 0                                     # an empty slot
    slot = rng.choice(K, size=T * k, p=p / p.sum()).astype(np.int32)
    slot[rng.random(T * k) < 0.1] = -1
    slot[rng.random(T * k) < 0.02] = K + 5                # out of range: not served either
    n, at = T * k, act(dtype)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(K)).to(at).to(DEV)
    L = layer(K, K, d, n + 5, dtype)
    L.slot[:n].copy_(torch.from_numpy(slot))
    perm, inv, off = ref.sort_pairs(slot, K)
    for rows in (True, False):
        for t in (L.perm, L.inv_perm, L.offsets):
            t.fill_(-7)
        L.x_perm.fill_(3)
        L.permute_topk(x if rows else None, T, k)
        torch.cuda.synchronize()
        m = len(perm)
        assert np.array_equal(L.offsets.cpu().numpy(), off)
        assert np.array_equal(L.perm.cpu().numpy()[:m], perm) and (L.perm.cpu().numpy()[m:] == -7).all()
        assert np.array_equal(L.inv_perm.cpu().numpy()[:n], inv) and (L.inv_perm.cpu().numpy()[n:] == -7).all()
        assert (L.x_perm[m if rows else 0:] == 3).all()
        if rows and m:
            want = x[torch.from_numpy(perm // k).to(DEV)]
            assert torch.equal(L.x_perm[:m].view(at), want)
    if T == 0:
        return
    y = torch.randn(n + 5, d, generator=torch.Generator().manual_seed(1)).to(at).to(DEV)
    y[len(perm):] = float("nan")                          # rows that nobody reads
    L.y_perm.copy_(y.view(L.y_perm.dtype))
    gate = torch.rand(n, generator=torch.Generator().manual_seed(2)).to(DEV)
    L.gate[:n].copy_(gate)
    L.gate[:n][torch.from_numpy(inv).to(DEV) < 0] = float("nan")   # and weights
    res = torch.randn(T, d, generator=torch.Generator().manual_seed(3)).to(at).to(DEV)
    yd, gd = f64(y), f64(gate)
    parts = np.where((inv >= 0)[:, None], gd[:, None] * yd[np.maximum(inv, 0)], 0).reshape(T, k, d)
    parts[np.isnan(parts)] = 0                            # row 0 stands in for no row
    for r in (None, res):
        want = parts.sum(1) + (0 if r is None else f64(r))
        size = np.abs(parts).sum(1) + (0 if r is None else np.abs(f64(r)))
        out = torch.full((T + 1, d), 5.0, dtype=at, device=DEV)
        L.combine_topk(T, k, r, out)
        torch.cuda.synchronize()
        assert (np.abs(f64(out)[:T] - want) <= np.abs(want) * ROUND[dtype] + (k + 1) * U * size).all()
        assert (out[T] == 5).all()
    same = res.clone()
    L.combine_topk(T, k, same, same)                      # in place over the residual
    torch.cuda.synchronize()
    assert torch.equal(same, out[:T])
    L.close()

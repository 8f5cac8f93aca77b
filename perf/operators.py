"""The operators around a mixture-of-experts layer that serves several experts per token, as cases that can be timed.

Five operators, in the order in which a block calls them:

  norm     residual addition and root-mean-square norm in front of the layer, its result in bf16 (or fp32) and in 8 bits
           with a scale for every 32 values                                       binding.Layer.add_norm
  route    scores, bias for balance, groups, k experts per token, among all experts and among the resident ones
                                                                                  binding.Layer.route_topk
  permute  the T * k (token, choice) pairs sorted by resident slot, rows copied   binding.Layer.permute_topk
  ffn      the experts' two products on 8-bit values, matrices resident in 8 bits binding.Layer.expert_ffn_mx
  combine  a token's k results weighted and added                                 binding.Layer.combine_topk

`run` computes each in elementary torch operations, or, where `own` is true, through the calls above.  8-bit values are
e4m3 numbers in blocks of 32 with a power of two for each block, the smallest with which no value of the block exceeds
448; they are returned as float8_e4m3fn tensors and their scales as float8_e8m0fnu tensors.

Shapes are those of the repository's workloads (workloads.CONFIGS) and between them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_EPS = 1e-6
_W_STD = 0.02


def _norm(**kw):
    return dict(kind="norm", T=1, d=768, dtype="bf16", residual=True, eight=True, **kw)


def _route(**kw):
    return dict(dict(kind="route", E=64, K=16, T=1, d=768, k=2, dtype="bf16", score="softmax", bias=False, groups=1, kept=1,
                     best=1, renorm=True, scale=1.0), **kw)


def _permute(**kw):
    return dict(dict(kind="permute", K=16, T=32, d=768, k=2, dtype="bf16", unserved=0.0), **kw)


def _combine(**kw):
    return dict(dict(kind="combine", T=32, d=768, k=2, dtype="bf16", residual=True, unserved=0.0), **kw)


def _ffn(**kw):
    return dict(dict(kind="ffn", K=16, T=32, d=768, f=3072, k=2, unserved=0.0), **kw)


def listed():
    return [
        # one sequence decoding: all latency
        dict(_norm(), name="norm-1"),
        # Switch-large-128 prefill: the whole batch's residual stream, with 8-bit values for the experts
        dict(_norm(), name="norm-16384", T=16384, d=1024),
        # one sequence decoding through a 64-expert layer with two experts per token
        dict(_route(), name="route-1"),
        # Switch-base-64 prefill, four experts per token
        dict(_route(), name="route-4096", T=4096, k=4),
        # Switch-large-128 prefill, eight of 128 experts out of four of eight groups, balanced by a bias
        dict(_route(), name="route-16384-groups", E=128, K=32, T=16384, d=1024, k=8, score="sigmoid", bias=True, groups=8,
             kept=4, best=2, scale=2.5),
        # a decode batch, two experts per token
        dict(_permute(), name="permute-32"),
        # Switch-large-128 prefill, four experts per token, some choices with no resident expert
        dict(_permute(), name="permute-16384", K=32, T=16384, d=1024, k=4, unserved=0.05),
        # a prefill chunk of odd length
        dict(_combine(), name="combine-777", T=777),
        # Switch-large-128 prefill, four experts per token
        dict(_combine(), name="combine-16384", T=16384, d=1024, k=4, unserved=0.05),
        # a half-filled decode batch
        dict(_ffn(), name="ffn-13", K=10, T=13),
        # widths and counts that fit no tile
        dict(_ffn(), name="ffn-1213", K=11, T=1213, d=416, f=1696, unserved=0.03),
        # Switch-large-128 prefill of 8192 tokens, two experts per token
        dict(_ffn(), name="ffn-8192", K=32, T=8192, d=1024, f=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "route", "route", "permute", "combine", "ffn", "ffn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([768, 1024, 512, 32 * rng.randint(8, 32)])
    if kind == "norm":
        return dict(_norm(), T=_log_int(rng, 1, 16384), d=d, dtype=dtype, residual=rng.random() < 0.7, eight=rng.random() < 0.7)
    k = rng.choice([1, 2, 2, 3, 4, 6, 8])
    if kind == "route":
        E = rng.choice([8, 16, 24, 32, 33, 60, 64, 100, 128])
        K = max(k, _log_int(rng, max(2, E // 8), E))
        groups = rng.choice([g for g in (1, 1, 2, 4, 8) if E % g == 0])
        kept = rng.randint(-(-groups // 2), groups)
        k = min(k, E // groups * kept, K)
        return _route(E=E, K=min(K, E), T=_log_int(rng, 1, 16384), d=d, k=k, dtype=dtype, score=rng.choice(["softmax", "sigmoid"]),
                      bias=rng.random() < 0.5, groups=groups, kept=kept, best=rng.choice([1, 2]), renorm=rng.random() < 0.6,
                      scale=rng.choice([1.0, 1.0, 2.5]))
    K = max(k, _log_int(rng, 2, 32))
    T = _log_int(rng, 1, 65536 // (max(k, 4)))
    unserved = rng.choice([0.0, 0.0, rng.uniform(0.0, 0.2)])
    if kind == "permute":
        return _permute(K=K, T=T, d=d, k=k, dtype=dtype, unserved=unserved)
    if kind == "combine":
        return _combine(T=T, d=d, k=k, dtype=dtype, residual=rng.random() < 0.7, unserved=unserved)
    d, f = rng.choice([(768, 3072), (1024, 4096), (768, 2048), (512, 2048), (32 * rng.randint(8, 32), 32 * rng.randint(24, 128))])
    return _ffn(K=K, T=_log_int(rng, 1, 16384 // k), d=d, f=f, k=k, unserved=unserved)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _act(c):
    return torch.float32 if c.get("dtype") == "f32" else torch.bfloat16


def _blocks(v):
    """v [..., n] fp32 or wider -> (e4m3 values in units of their block's scale, exponents of the scales [..., n / 32])."""
    b = v.unflatten(-1, (-1, 32))
    m, p = torch.frexp(b.abs().amax(-1))
    e = torch.where(m > 0.875, p - 8, p - 9).clamp(-126, 127)           # 448 = 0.875 * 2^9
    return torch.ldexp(b, -e.unsqueeze(-1)).flatten(-2).to(torch.float8_e4m3fn), e


def _widen(q, e):
    return torch.ldexp(q.float().unflatten(-1, (-1, 32)), e.unsqueeze(-1)).flatten(-2)


def _choices(c, g, dev):
    """Slots of T tokens' k choices: distinct slots of skewed popularity, a share of them unserved (-1)."""
    p = torch.arange(1, c["K"] + 1, device=dev, dtype=torch.float32).pow(-0.7).log()
    u = torch.rand(c["T"], c["K"], device=dev, generator=g).clamp_(1e-9, 1 - 1e-7)
    slot = (p - (-u.log()).log()).topk(c["k"], dim=1).indices.to(torch.int32)
    return torch.where(torch.rand(slot.shape, device=dev, generator=g) < c["unserved"], -1, slot).to(torch.int32).contiguous()


def _sorted_pairs(slot, K):
    """Pairs sorted by slot, the unserved ones last: (perm, inverse with -1 for the unserved, offsets [K + 1])."""
    key = torch.where(slot.view(-1) < 0, K, slot.view(-1))
    order = torch.sort(key, stable=True).indices
    inv = torch.empty_like(order)
    inv[order] = torch.arange(order.numel(), device=order.device)
    offsets = torch.searchsorted(key[order].contiguous(), torch.arange(K + 1, device=key.device, dtype=key.dtype))
    return order, torch.where(slot.view(-1) < 0, -1, inv), offsets


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    act, T, d = _act(c), c["T"], c["d"]
    s = {"case": c}

    def rand(*shape):
        return torch.randn(*shape, device=dev, generator=g)

    def layer(E, K, f, pairs, dtype=None, router=None):
        from paper_2308_15030_amd import binding as b
        code = b.SMOE_F32 if act == torch.float32 else b.SMOE_BF16
        return b.Layer(E, K, d, f, pairs, code if dtype is None else getattr(b, dtype), router_w=router, device=dev)

    if c["kind"] == "norm":
        # the residual stream has columns of very different size
        col = torch.exp(rand(d))
        s.update(x=rand(T, d).to(act), residual=(rand(T, d) * col).to(act) if c["residual"] else None, weight=1 + 0.1 * rand(d))
        if own:
            lay = layer(1, 1, 32, T)
            s.update(layer=lay, total=torch.empty(T, d, dtype=act, device=dev) if c["residual"] else None,
                     y=torch.empty(T, d, dtype=act, device=dev))
            s["q"], s["q_scale"] = lay.mx_buffers(T) if c["eight"] else (None, None)
    elif c["kind"] == "route":
        E, K, k = c["E"], c["K"], c["k"]
        x = (rand(16, d)[torch.randint(0, 16, (T,), device=dev, generator=g)] + 0.5 * rand(T, d)).to(act)   # clusters of tokens
        router = _W_STD * rand(E, d)
        resident = torch.randperm(E, device=dev, generator=g)[:K]
        e2s = torch.full((E,), -1, dtype=torch.int32, device=dev)
        e2s[resident] = torch.arange(K, dtype=torch.int32, device=dev)
        spread = 0.05 if c["score"] == "sigmoid" else 0.3 / E
        s.update(x=x, router=router, e2s=e2s, bias=spread * rand(E) if c["bias"] else None)
        if own:
            from paper_2308_15030_amd import binding as b
            lay = layer(E, K, 32, T * k, router=router)
            w = torch.zeros(d * 32, dtype=act, device=dev)
            for slot, e in enumerate(resident.tolist()):
                lay.set_resident(slot, e, w, w)
            score = {"softmax": b.SMOE_SCORE_SOFTMAX, "sigmoid": b.SMOE_SCORE_SIGMOID}[c["score"]]
            s.update(layer=lay, rule=b.smoe_topk_rule(k, score, c["groups"], c["kept"], c["best"], int(c["renorm"]), c["scale"]))
    elif c["kind"] == "permute":
        s.update(x=rand(T, d).to(act), slot=_choices(c, g, dev))
        n = T * c["k"]
        s.update(x_perm=torch.zeros(n, d, dtype=act, device=dev), perm=torch.zeros(n, dtype=torch.int32, device=dev))
        if own:
            s["layer"] = lay = layer(c["K"], c["K"], 32, n)
            lay.x_perm, lay.perm = s["x_perm"], s["perm"]
            lay.slot.copy_(s["slot"].view(-1))
    elif c["kind"] == "combine":
        k = c["k"]
        order, inv, _ = _sorted_pairs(_choices(dict(c, K=max(k, 16)), g, dev), max(k, 16))
        s.update(y_perm=rand(T * k, d).to(act), inv_perm=inv.to(torch.int32), gate=torch.rand(T, k, device=dev, generator=g),
                 residual=rand(T, d).to(act) if c["residual"] else None)
        if own:
            s["layer"] = lay = layer(1, 1, 32, T * k)
            lay.y_perm, lay.inv_perm = s["y_perm"], s["inv_perm"]
            lay.gate.copy_(s["gate"].view(-1))
            s["out"] = torch.empty(T, d, dtype=act, device=dev)
    else:
        K, k, f = c["K"], c["k"], c["f"]
        slot = _choices(c, g, dev)
        perm, _, offsets = _sorted_pairs(slot, K)
        # the experts as an 8-bit checkpoint gives them: numbers with a scale per 32 of a column, widened to bf16
        w = [torch.cat([_widen(*_blocks((_W_STD * rand(n, r)))).T[None].to(torch.bfloat16) for _ in range(K)])
             for r, n in ((d, f), (f, d))]
        q, e = _blocks(rand(T, d))
        s.update(q=q, exponent=e, w1=w[0], w2=w[1], perm=perm.to(torch.int32), offsets=offsets.to(torch.int32),
                 y_perm=torch.zeros(T * k, d, dtype=torch.bfloat16, device=dev), longest=int((offsets[1:] - offsets[:-1]).max()))
        if own:
            s["layer"] = lay = layer(K, K, f, T * k, "SMOE_MXFP8")
            for i in range(K):
                lay.set_resident(i, i, w[0][i].contiguous(), w[1][i].contiguous())
            s["q"], s["q_scale"] = lay.mx_buffers(T)
            s["q"].copy_(q.view(torch.uint8))
            s["q_scale"].zero_()
            s["q_scale"][:, :d // 32].copy_((e + 127).to(torch.uint8))
            lay.perm, lay.offsets, lay.y_perm = s["perm"], s["offsets"], s["y_perm"]
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def _plain_norm(s, c):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + _EPS) * s["weight"]
    out = {"y": y.to(s["x"].dtype)}
    if s["residual"] is not None:
        out["total"] = h.to(s["x"].dtype)
    if c["eight"]:
        q, e = _blocks(y)
        out.update(q=q, q_scale=(e + 127).to(torch.uint8).view(torch.float8_e8m0fnu))
    return out


def _pick(scores, biased, c):
    """The k best experts of each row by `biased` (-inf: not to be had), best first, the lowest id among equals; -1 where there is
    none, and their weights."""
    grouped = biased.unflatten(-1, (c["groups"], -1))
    top = torch.sort(grouped, dim=-1, descending=True).values[..., :c["best"]]
    rank = torch.where(top > -math.inf, top, 0).sum(-1).where(top[..., 0] > -math.inf, torch.tensor(-math.inf, device=top.device, dtype=top.dtype))
    keep = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:, :c["kept"]]
    kept = torch.zeros_like(rank, dtype=torch.bool).scatter_(1, keep, True)
    biased = torch.where(kept.unsqueeze(-1), grouped, -math.inf).flatten(-2)
    best = torch.sort(biased, dim=-1, descending=True, stable=True)
    idx, there = best.indices[:, :c["k"]], best.values[:, :c["k"]] > -math.inf
    w = torch.where(there, scores.gather(1, idx), 0)
    if c["renorm"]:
        w = w / w.sum(-1, keepdim=True).clamp_min(torch.finfo(torch.float64).tiny)
    return torch.where(there, idx, -1), w * c["scale"]


def _plain_route(s, c):
    # in 64 bits: which of two near scores is larger decides the expert
    x = s["x"].double()
    logits = x @ s["router"].double().T
    p = torch.softmax(logits, -1) if c["score"] == "softmax" else torch.sigmoid(logits)
    biased = p if s["bias"] is None else p + s["bias"].double()
    expert, orig_gate = _pick(p, biased, c)
    served, gate = _pick(p, torch.where(s["e2s"] >= 0, biased, -math.inf), c)
    slot = torch.where(served >= 0, s["e2s"][served.clamp_min(0)], -1)
    xnorm = x.square().sum(-1, keepdim=True).sqrt().expand(-1, c["k"])
    return {"expert": expert.to(torch.int32), "orig_gate": orig_gate.float(), "slot": slot.to(torch.int32), "gate": gate.float(),
            "xnorm": xnorm.float()}


def _plain_permute(s, c):
    order, inv, offsets = _sorted_pairs(s["slot"], c["K"])
    at = torch.arange(order.numel(), device=order.device) < offsets[-1]
    perm = torch.where(at, order, 0)
    x_perm = torch.where(at[:, None], s["x"][perm // c["k"]], 0)
    return {"x_perm": x_perm, "perm": perm.to(torch.int32), "inv_perm": inv.to(torch.int32), "offsets": offsets.to(torch.int32)}


def _plain_combine(s, c):
    inv = s["inv_perm"].view(c["T"], c["k"]).long()
    g = torch.where(inv < 0, 0, s["gate"]).unsqueeze(-1)
    out = (g * s["y_perm"].float()[inv.clamp_min(0)]).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(s["y_perm"].dtype)}


def _plain_ffn(s, c):
    lo, hi = s["offsets"][:-1].long(), s["offsets"][1:].long()
    at = lo[:, None] + torch.arange(s["longest"], device=lo.device)      # [K, longest] rows of each slot
    live = at < hi[:, None]
    row = torch.where(live, at, 0)
    x = _widen(s["q"], s["exponent"])[s["perm"].long()[row] // c["k"]]
    h = torch.bmm(x, s["w1"].float()).relu()
    y = torch.bmm(_widen(*_blocks(h)), s["w2"].float()).to(torch.bfloat16)
    out = torch.zeros(c["T"] * c["k"] + 1, c["d"], dtype=torch.bfloat16, device=y.device)
    out[torch.where(live, at, c["T"] * c["k"])] = y                      # what is past a slot's end goes to the row behind
    return {"y_perm": out[:-1]}


def run(state):
    s, c = state, state["case"]
    T, kind = c["T"], c["kind"]
    if not own:
        return {"norm": _plain_norm, "route": _plain_route, "permute": _plain_permute, "combine": _plain_combine,
                "ffn": _plain_ffn}[kind](s, c)
    lay = s["layer"]
    if kind == "norm":
        lay.add_norm(s["x"], T, s["weight"], _EPS, residual=s["residual"], total=s["total"], y=s["y"], q=s["q"], q_scale=s["q_scale"])
        out = {"y": s["y"]}
        if c["residual"]:
            out["total"] = s["total"]
        if c["eight"]:
            out.update(q=s["q"].view(torch.float8_e4m3fn), q_scale=s["q_scale"][:, :c["d"] // 32].view(torch.float8_e8m0fnu))
        return out
    k = c["k"]
    if kind == "route":
        lay.route_topk(s["x"], T, s["rule"], bias=s["bias"])
        return {"expert": lay.orig_expert.view(T, k), "orig_gate": lay.orig_gate.view(T, k), "slot": lay.slot.view(T, k),
                "gate": lay.gate.view(T, k), "xnorm": lay.xnorm.view(T, k)}
    if kind == "permute":
        lay.permute_topk(s["x"], T, k)
        return {"x_perm": lay.x_perm, "perm": lay.perm, "inv_perm": lay.inv_perm, "offsets": lay.offsets}
    if kind == "combine":
        return {"out": lay.combine_topk(T, k, residual=s["residual"], out=s["out"])}
    return {"y_perm": lay.expert_ffn_mx(s["q"], s["q_scale"], T, k)}


def work(case):
    """Inputs once, outputs once; of the experts' matrices those of the slots that get a row, if rows are spread evenly, one byte
    a weight and one for 32."""
    c = case
    T, d, size = c["T"], c["d"], 4 if c.get("dtype") == "f32" else 2
    if c["kind"] == "norm":
        return {"bytes": T * d * size * (4 if c["residual"] else 2) + T * d * (33 / 32 if c["eight"] else 0) + 4 * d, "flops": 6.0 * T * d}
    n = T * c["k"]
    if c["kind"] == "route":
        return {"bytes": T * d * size + 4 * c["E"] * d + 20 * n, "flops": 2.0 * T * d * c["E"]}
    served = n * (1 - c["unserved"])
    if c["kind"] == "permute":
        return {"bytes": (T + served) * d * size + 12 * n + 4 * c["K"], "flops": float(n)}
    if c["kind"] == "combine":
        return {"bytes": (served + T * (2 if c["residual"] else 1)) * d * size + 8 * n, "flops": 2.0 * served * d}
    K, f = c["K"], c["f"]
    active = K * (1 - (1 - 1 / K) ** served)
    return {"bytes": active * 2 * d * f * 33 / 32 + T * d * 33 / 32 + served * d * 2 + 4 * n, "flops": 4.0 * served * d * f}


# --------------------------------------------------------------------------
# the definitions in 64 bits, apart from the plain forms
# --------------------------------------------------------------------------

def _exact_blocks(v):
    """v [..., n] float64 -> (values in units of the scale, scale): rounded to a multiple of the spacing of e4m3 numbers of that size."""
    b = v.reshape(*v.shape[:-1], -1, 32)
    big = b.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(big.clamp_min(1e-300) / 448)).clamp(-126, 127))
    u = b / scale
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(u / step) * step).reshape(v.shape), scale.squeeze(-1)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c, kind, T = case, case["kind"], case["T"]
    if kind == "norm":
        total = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
        y = total / ((total * total).sum(-1, keepdim=True) / c["d"] + _EPS).sqrt() * s["weight"].double()
        out = {"y": y}
        if c["residual"]:
            out["total"] = total
        if c["eight"]:
            out["q"], out["q_scale"] = _exact_blocks(y)
        return out
    k = c["k"]
    if kind == "route":
        x, w = s["x"].double().cpu().numpy(), s["router"].double().cpu().numpy()
        z = x @ w.T
        if c["score"] == "softmax":
            p = np.exp(z - z.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
        else:
            p = 1 / (1 + np.exp(-z))
        e2s = s["e2s"].cpu().numpy()
        b = p + (0 if s["bias"] is None else s["bias"].double().cpu().numpy())
        rows, per, out = np.arange(T), c["E"] // c["groups"], {}
        for name, ok in (("orig", np.ones(c["E"], bool)), ("served", e2s >= 0)):
            m = np.where(ok, b, -np.inf)
            rank = np.full((T, c["groups"]), -np.inf)
            for j in range(c["groups"]):
                part = np.sort(m[:, j * per:(j + 1) * per], 1)[:, ::-1][:, :c["best"]]
                rank[:, j] = np.where(np.isinf(part[:, 0]), -np.inf, np.where(np.isinf(part), 0, part).sum(1))
            keep = np.zeros((T, c["E"]), bool)
            for _ in range(c["kept"]):
                j = rank.argmax(1)
                for t in range(per):
                    keep[rows, j * per + t] = True
                rank[rows, j] = -np.inf
            m = np.where(keep, m, -np.inf)
            e, g = np.full((T, k), -1), np.zeros((T, k))
            for i in range(k):
                j = m.argmax(1)
                there = m[rows, j] > -np.inf
                e[:, i], g[:, i] = np.where(there, j, -1), np.where(there, p[rows, j], 0)
                m[rows, j] = -np.inf
            if c["renorm"]:
                g = g / np.maximum(g.sum(1, keepdims=True), 1e-300)
            out[name] = (e, g * c["scale"])
        slot = np.where(out["served"][0] >= 0, e2s[np.maximum(out["served"][0], 0)], -1)
        return {"expert": out["orig"][0].astype(np.int32), "orig_gate": out["orig"][1], "slot": slot.astype(np.int32),
                "gate": out["served"][1], "xnorm": np.repeat(np.sqrt((x * x).sum(1))[:, None], k, 1)}
    if kind == "permute":
        return None                                        # whole numbers and copies
    if kind == "combine":
        inv = s["inv_perm"].view(T, k).long()
        out = torch.zeros(T, c["d"], dtype=torch.float64, device=inv.device) if s["residual"] is None else s["residual"].double()
        for j in range(k):
            row = s["y_perm"].double()[inv[:, j].clamp_min(0)] * s["gate"][:, j:j + 1].double()
            out = out + torch.where(inv[:, j:j + 1] < 0, 0, row)
        return {"out": out}
    q = s["q"].double()
    x = (q.reshape(T, -1, 32) * torch.exp2(s["exponent"].double())[..., None]).reshape(T, c["d"])
    out = torch.zeros(T * k, c["d"], dtype=torch.float64, device=x.device)
    bounds, token = s["offsets"].tolist(), torch.div(s["perm"].long(), k, rounding_mode="floor")
    for i in range(c["K"]):
        lo, hi = bounds[i], bounds[i + 1]
        if hi > lo:
            h, scale = _exact_blocks((x[token[lo:hi]] @ s["w1"][i].double()).clamp_min(0))
            h = (h.reshape(hi - lo, -1, 32) * scale[..., None]).reshape(hi - lo, -1)
            out[lo:hi] = h @ s["w2"][i].double()
    return {"y_perm": out}

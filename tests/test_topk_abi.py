"""Refusals of the calls around a layer that serves k experts per token, before any launch (no GPU), and the sizes of layers with
8-bit slots.  The oracle's helpers are checked here too."""
import ctypes as C

import numpy as np
import pytest
import torch

import topk_reference as ref
from paper_2308_15030_amd import binding as b

FAKE = 0x10000
SHAPE = dict(E=12, K=4, d_model=64, d_ff=96, max_tokens=64)


@pytest.fixture(params=[b.SMOE_F32, b.SMOE_BF16, b.SMOE_MXFP8])
def bound(request):
    h = b.smoe_create(dtype=request.param, **SHAPE)
    assert b._lib.smoe_bind(h, FAKE, FAKE, FAKE, FAKE, FAKE) == b.SMOE_OK
    yield h, request.param
    b.smoe_destroy(h)


def refused(status, fn, *args, text=None):
    assert fn(*args) == status
    if text:
        assert text in b.smoe_last_error()


def test_add_norm_refusals(bound):
    h, dtype = bound
    f = b._lib.smoe_add_norm

    def call(x=FAKE, res=FAKE, w=FAKE, eps=1e-6, T=4, total=FAKE, y=FAKE, q=FAKE, qs=FAKE, layer=h):
        return f(layer, x, res, w, eps, T, total, y, q, qs, None)
    E = b.SMOE_EINVAL
    for kw in (dict(layer=None), dict(T=-1), dict(T=65), dict(x=None), dict(w=None), dict(total=None, y=None, q=None, qs=None),
               dict(q=None), dict(qs=None), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=FAKE + 8),
               dict(res=FAKE + 4), dict(w=FAKE + 4), dict(y=FAKE + 8), dict(total=FAKE + 8), dict(q=FAKE + 8), dict(qs=FAKE + 4)):
        assert call(**kw) == E, kw
        assert b.smoe_last_error() != ""
    assert call(T=0, x=None, w=None) == b.SMOE_OK
    odd = b.smoe_create(4, 2, 36, 36, 8, b.SMOE_F32)
    refused(E, f, odd, FAKE, None, FAKE, 1e-6, 4, None, None, FAKE, FAKE, None, text="multiple of 32")
    b.smoe_destroy(odd)


def test_route_topk_refusals(bound):
    h, dtype = bound
    f = b._lib.smoe_route_topk

    def call(T=4, bias=None, bufs=(FAKE,) * 5, x=FAKE, layer=h, rule=True, **kw):
        r = b.smoe_topk_rule(**{**dict(k=2), **kw})
        return f(layer, C.byref(r) if rule else None, bias, x, T, *bufs, None)
    assert call(rule=False) == call(layer=None) == b.SMOE_EINVAL
    assert call(T=33) == call(T=-1) == call(k=0) == call(k=17, T=1) == b.SMOE_EINVAL          # 33 * 2 pairs of 64
    for kw in (dict(score=2), dict(groups=0), dict(groups=5), dict(groups=3, groups_kept=0), dict(groups=3, groups_kept=4), dict(group_best=0),
               dict(group_best=3), dict(renorm=2), dict(scale=float("inf")), dict(scale=float("nan")), dict(k=5, groups=3, groups_kept=1)):
        assert call(**kw) == b.SMOE_EINVAL and "smoe_route_topk" in b.smoe_last_error(), kw
    assert call() == b.SMOE_ESTATE                                                            # empty slots
    full = b.smoe_create(12, 4, 64, 96, 64, dtype)
    refused(b.SMOE_ESTATE, f, full, C.byref(b.smoe_topk_rule(2)), None, FAKE, 4, *(FAKE,) * 5, None, text="smoe_bind")
    b.smoe_destroy(full)


def test_pairs_refusals(bound):
    h, dtype = bound
    p, c, m, E = b._lib.smoe_permute_topk, b._lib.smoe_combine_topk, b._lib.smoe_expert_ffn_mx, b.SMOE_EINVAL
    B = (FAKE,) * 4
    for bad in ((None, FAKE, FAKE, 4, 2, *B), (h, FAKE, FAKE, -1, 2, *B), (h, FAKE, FAKE, 33, 2, *B), (h, FAKE, FAKE, 4, 0, *B),
                (h, FAKE, FAKE, 2, 17, *B), (h, FAKE, None, 4, 2, *B), (h, None, FAKE, 4, 2, *B), (h, FAKE + 8, FAKE, 4, 2, *B),
                (h, FAKE, FAKE, 4, 2, FAKE + 8, FAKE, FAKE, FAKE), (h, FAKE, FAKE, 4, 2, FAKE, None, FAKE, FAKE),
                (h, FAKE, FAKE, 4, 2, FAKE, FAKE, None, FAKE), (h, FAKE, FAKE, 4, 2, FAKE, FAKE, FAKE, None)):
        assert p(*bad, None) == E, bad
    for bad in ((None, FAKE, FAKE, FAKE, None, 4, 2, FAKE), (h, None, FAKE, FAKE, None, 4, 2, FAKE), (h, FAKE, None, FAKE, None, 4, 2, FAKE),
                (h, FAKE, FAKE, None, None, 4, 2, FAKE), (h, FAKE, FAKE, FAKE, None, 4, 2, None), (h, FAKE, FAKE, FAKE, FAKE + 8, 4, 2, FAKE),
                (h, FAKE + 8, FAKE, FAKE, None, 4, 2, FAKE), (h, FAKE, FAKE, FAKE, None, 33, 2, FAKE), (h, FAKE, FAKE, FAKE, None, 4, 0, FAKE)):
        assert c(*bad, None) == E, bad
    assert c(h, None, None, None, None, 0, 2, None, None) == b.SMOE_OK
    assert m(None, FAKE, FAKE, FAKE, 2, FAKE, 4, FAKE, None) == E
    assert m(h, FAKE, FAKE, FAKE, 2, FAKE, 33, FAKE, None) == E
    # empty slots; a layer of another type is refused before that
    assert m(h, FAKE, FAKE, FAKE, 2, FAKE, 4, FAKE, None) == (b.SMOE_ESTATE if dtype == b.SMOE_MXFP8 else E)
    assert b._lib.smoe_expert_ffn(h, FAKE, FAKE, 4, FAKE, None) == b.SMOE_ESTATE


def test_sizes_of_8_bit_layers():
    """Operand order: steps of 64 reduction elements, one scale for 32, scales in groups of four steps; both arrays the larger matrix."""
    def matrix(r, n):
        return n // 32 * (-(-r // 64) * 2048 + -(-r // 256) * 256)
    for d, f in ((64, 96), (416, 1696), (768, 2048), (1024, 4096)):
        h = b.smoe_create(8, 3, d, f, 100, b.SMOE_MXFP8, spare_slots=2)
        one = max(matrix(d, f), matrix(f, d))
        assert b.smoe_slot_weight_bytes(h) == 5 * one
        m = b.smoe_profile_memory(8, 3, d, f, 100, b.SMOE_MXFP8, spare_slots=2)
        assert m["expert_bytes"] == 2 * one and m["resident_bytes"] == 10 * one and m["bank_bytes"] == 8 * 2 * d * f * 2
        assert b.smoe_workspace_bytes(h) > (100 + 32 * 3) * f
        b.smoe_destroy(h)
    assert [b.smoe_mx_scale_pitch(d) for d in (32, 256, 288, 768, 1024)] == [8, 8, 16, 24, 32]
    assert b.smoe_mx_scale_pitch(0) == b.smoe_mx_scale_pitch(-32) == b.smoe_mx_scale_pitch(40) == 0
    with pytest.raises(b.SmoeError):
        b.smoe_create(8, 3, 48, 64, 100, b.SMOE_MXFP8)


def test_8_bit_layers_refuse_what_they_lack():
    h = b.smoe_create(8, 2, 64, 64, 32, b.SMOE_MXFP8)
    assert b._lib.smoe_bind(h, FAKE, FAKE, FAKE, FAKE, FAKE) == b.SMOE_OK
    refused(b.SMOE_EINVAL, b._lib.smoe_update_on_device, h, FAKE, FAKE, FAKE, None, text="bf16 layers only")
    b.smoe_destroy(h)


def test_rule_defaults():
    r = b.smoe_topk_rule(3)
    assert (r.k, r.score, r.groups, r.groups_kept, r.group_best, r.renorm, r.scale) == (3, b.SMOE_SCORE_SOFTMAX, 1, 1, 1, 1, 1.0)


# ------------------------------------------------------------------ the oracle's helpers
def test_reference_e4m3_is_torchs():
    x = torch.cat([torch.linspace(-448, 448, 20001), torch.randn(5000) * 0.02])
    q, e = ref.to_blocks(np.pad(x.double().numpy(), (0, -len(x) % 32)))
    got = ref.from_blocks(q, e)[:len(x)]
    scale = np.repeat(2.0 ** e.astype(float), 32)[:len(x)]
    want = (x.double() / torch.from_numpy(scale)).to(torch.float8_e4m3fn).double().numpy() * scale
    assert np.array_equal(np.abs(got), np.abs(want))
    by = np.arange(127, dtype=np.uint8)
    assert np.array_equal(ref.e4m3_values(by), torch.from_numpy(by).view(torch.float8_e4m3fn).double().numpy())


def test_reference_scale_is_the_smallest():
    for a, e in ((448.0, 0), (448.1, 1), (224.0, -1), (0.0, -126), (1.0, -8), (1.75, -8), (1.76, -7), (2.0 ** -140, -126)):
        assert ref.scale_exponent(np.array([a]))[0] == e


def test_reference_choice_by_hand():
    s = np.array([.1, .4, .2, .3, .0, .25, .25, .1])
    assert ref.choose(s, s, 3, 1, 1, 1, True, 1.0)[0] == [1, 3, 5]
    assert ref.choose(s, s, 3, 4, 2, 1, False, 2.0) == ([1, 3, 2], [.8, .6, .4])
    assert ref.choose(s, s, 2, 4, 1, 2, False, 1.0)[0] == [1, 0]            # pairs (.5, .5, .25, .35): the lower group on a tie
    m = np.where(np.arange(8) == 5, s, -np.inf)
    assert ref.choose(s, m, 2, 4, 2, 2, True, 1.0) == ([5, -1], [1.0, 0.0])


def test_host_code_under_asan_ubsan(tmp_path):
    """The argument checks of these calls under the address and undefined-behaviour sanitizers, host code only, launchers stubbed."""
    import os
    import test_sanitizers_cpu as san
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    exe = str(tmp_path / "topk_san")
    csrc = os.path.join(san.ROOT, "paper_2308_15030_amd", "csrc")
    san._run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
              "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-omit-frame-pointer",
              "-I", os.path.join(san.ROOT, "include"), "-I", csrc,
              *(os.path.join(csrc, n) for n in ("api.hip", "api_topk.hip", "policy.hip")),
              "-x", "hip", os.path.join(san.SAN, "topk_driver.cpp"), "-o", exe], exe, tmp_path)

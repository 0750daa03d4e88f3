"""The 64-bit references of the gated delta rule and the group norm against automatic differentiation, differences and special
cases with known answers, and what their entry points refuse (CPU only: every call returns before a launch)."""
import ctypes
import os
import re

import pytest
import torch

import delta_norm_ref as ref
from paper_2405_18425_amd import binding as vb

PTR = 0x10000  # a non-NULL, 16-byte aligned dummy: validation must reject before dereferencing
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "vig_bigla.h")


def _inputs(B=2, H=4, Hk=2, L=9, dk=3, dv=5, layout="bhld", seed=0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)
    heads = lambda h, *d: (B, h, L, *d) if layout == "bhld" else (B, L, h, *d)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    return (n(*heads(Hk, dk)), unit(n(*heads(Hk, dk))), n(*heads(H, dv)), -n(*heads(H)).abs() * 0.3, torch.sigmoid(n(*heads(H))),
            n(B, H, dk, dv), n(*heads(H, dv)), n(B, H, dk, dv))


@pytest.mark.parametrize("layout", ("bhld", "blhd"))
@pytest.mark.parametrize("direction", ("forward", "backward"))
def test_delta_adjoint_against_differences(layout, direction):
    q, k, v, g, beta, s0, d_out, d_fin = _inputs(layout=layout)
    grads = ref.delta_bwd(q, k, v, g, beta, d_out, s0, d_fin, layout, direction)

    def loss(*a):
        out, fin = ref.delta_fwd(*a, layout=layout, direction=direction)
        return (out * d_out).sum() + (fin * d_fin).sum()

    tensors = [q, k, v, g, beta, s0]
    gen = torch.Generator().manual_seed(5)
    for i, got in enumerate(grads):
        assert got.shape == tensors[i].shape
        step = torch.randn(tensors[i].shape, generator=gen, dtype=torch.float64)
        h = 1e-5
        up, down = list(tensors), list(tensors)
        up[i], down[i] = tensors[i] + h * step, tensors[i] - h * step
        slope = (loss(*up) - loss(*down)) / (2 * h)
        # central differences: h^2 times a third derivative of order 100, and 1e-16 / h of rounding on a loss of order 100
        assert abs(slope - (got * step).sum()) < 1e-6 * (1 + abs(slope)), i


def test_delta_known_answers():
    q, k, v, g, beta, s0, _, _ = _inputs(H=2, Hk=2, L=6)
    # beta 0 and gate 0: the state stays, every output reads it
    out, fin = ref.delta_fwd(q, k, v, g * 0, beta * 0, s0)
    assert torch.allclose(fin, s0) and torch.allclose(out, torch.einsum("bhlk,bhkv->bhlv", q, s0))
    # a closed gate forgets everything; with beta 1 and unit keys the state answers v_t for k_t
    out, fin = ref.delta_fwd(q, k, v, torch.full_like(g, -float("inf")), beta * 0 + 1, s0)
    assert torch.allclose(torch.einsum("bhk,bhkv->bhv", k[:, :, -1], fin), v[:, :, -1])
    # gate 0, beta 1: after a write the state answers v_t for k_t, whatever it held
    _, fin = ref.delta_fwd(q, k, v, g * 0, beta * 0 + 1, s0)
    assert torch.allclose(torch.einsum("bhk,bhkv->bhv", k[:, :, -1], fin), v[:, :, -1])
    # the two scan directions mirror each other
    rev = [x.flip(2) for x in (q, k, v, g, beta)]
    a, fa = ref.delta_fwd(q, k, v, g, beta, s0, direction="backward")
    b, fb = ref.delta_fwd(*rev, s0)
    assert torch.allclose(a, b.flip(2)) and torch.allclose(fa, fb)


@pytest.mark.parametrize("act", ("silu", "none"))
@pytest.mark.parametrize("affine", (True, False))
def test_norm_reference_against_the_library(act, affine):
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(2, 7, 12, generator=gen, dtype=torch.float64, requires_grad=True)
    w = torch.randn(12, generator=gen, dtype=torch.float64, requires_grad=True) if affine else None
    b = torch.randn(12, generator=gen, dtype=torch.float64, requires_grad=True) if affine else None
    d = torch.randn(2, 7, 12, generator=gen, dtype=torch.float64)
    z = torch.nn.functional.group_norm(x.transpose(1, 2), 3, w, b, 1e-5).transpose(1, 2)
    y = torch.nn.functional.silu(z) if act == "silu" else z
    assert torch.allclose(ref.norm_fwd(x, 3, w, b, act=act)[0], y.detach())
    want = torch.autograd.grad((y * d).sum(), [x, w, b] if affine else [x])
    got = ref.norm_bwd(x, d, 3, w, b, act=act)
    for g, e in zip(got, want):
        assert torch.allclose(g, e)


# ---- refusals --------------------------------------------------------------------------------------

DELTA_SIZES = dict(B=1, H=2, Hk=1, L=8, dk=16, dv=16, dtype=vb.VIG_BF16)


def _fwd(layout=0, direction=0, ws=PTR, ws_bytes=1 << 40, **kw):
    p = {n: kw.pop(n, PTR) for n in ("q", "k", "v", "g", "beta", "initial", "out", "final")}
    z = {**DELTA_SIZES, **kw}
    return vb.lib().gated_delta_fwd(*p.values(), *z.values(), layout, direction, ws, ws_bytes, None)


def _bwd(layout=0, direction=0, ws=PTR, ws_bytes=1 << 40, **kw):
    p = {n: kw.pop(n, PTR) for n in ("q", "k", "v", "g", "beta", "initial", "d_out", "d_final", "dq", "dk_", "dv_", "dg", "dbeta", "d_initial")}
    z = {**DELTA_SIZES, **kw}
    return vb.lib().gated_delta_bwd(*p.values(), *z.values(), layout, direction, ws, ws_bytes, None)


def _step(**kw):
    p = {n: kw.pop(n, PTR) for n in ("q", "k", "v", "g", "beta", "state", "slots", "out")}
    z = {**dict(B=3, H=2, Hk=1, dk=16, dv=16, n_slots=4, dtype=vb.VIG_BF16), **kw}
    return vb.lib().gated_delta_step(*p.values(), *z.values(), None)


@pytest.mark.parametrize("call,pointers", ((_fwd, ("q", "k", "v", "g", "beta", "out")),
                                           (_bwd, ("q", "k", "v", "g", "beta", "d_out", "dq", "dk_", "dv_", "dg", "dbeta"))))
def test_delta_refusals(call, pointers):
    optional = ("initial", "final") if call is _fwd else ("initial", "d_final", "d_initial")
    for name in pointers:
        assert call(**{name: None}) == vb.VIG_ERR_NULL
    for name in pointers + optional:
        assert call(**{name: PTR + 8}) == vb.VIG_ERR_ALIGN
    assert call(ws=PTR + 4) == vb.VIG_ERR_ALIGN
    for name in ("B", "H", "Hk", "L", "dk", "dv"):
        assert call(**{name: 0}) == vb.VIG_ERR_SHAPE
        assert call(**{name: -1}) == vb.VIG_ERR_SHAPE
    assert call(dtype=2) == vb.VIG_ERR_DTYPE
    assert call(layout=2) == vb.VIG_ERR_LAYOUT
    assert call(direction=2) == vb.VIG_ERR_UNSUPPORTED
    for name in ("dk", "dv"):
        assert call(**{name: 48}) == vb.VIG_ERR_UNSUPPORTED
        assert call(**{name: 256}) == vb.VIG_ERR_UNSUPPORTED
    assert call(H=3, Hk=2) == vb.VIG_ERR_UNSUPPORTED  # heads that do not share evenly
    assert call(H=2, Hk=4) == vb.VIG_ERR_UNSUPPORTED
    assert call(B=1 << 20, L=1 << 30) == vb.VIG_ERR_SHAPE
    assert call(H=1 << 15, Hk=1) == vb.VIG_ERR_SHAPE
    query = vb.lib().gated_delta_workspace_bytes if call is _fwd else vb.lib().gated_delta_bwd_workspace_bytes
    need = query(*DELTA_SIZES.values())
    assert need > 0
    assert call(ws=None, ws_bytes=0) == vb.VIG_ERR_WORKSPACE
    assert call(ws_bytes=need - 1) == vb.VIG_ERR_WORKSPACE


def test_delta_workspace_queries():
    for query in (vb.lib().gated_delta_workspace_bytes, vb.lib().gated_delta_bwd_workspace_bytes):
        small = query(1, 2, 1, 64, 64, 64, vb.VIG_BF16)
        assert 0 < small < query(1, 2, 1, 65, 64, 64, vb.VIG_BF16) and small % 16 == 0
        for bad in ((0, 2, 1, 64, 64, 64, 1), (1, 2, 1, 64, 48, 64, 1), (1, 3, 2, 64, 64, 64, 1), (1, 2, 1, 64, 64, 64, 7)):
            assert query(*bad) == 0
    # a workspace beyond 32 bits is counted in 64
    assert vb.lib().gated_delta_workspace_bytes(8, 64, 64, 1 << 16, 64, 64, vb.VIG_BF16) > 1 << 33


def test_step_refusals():
    for name in ("q", "k", "v", "g", "beta", "state", "out"):
        assert _step(**{name: None}) == vb.VIG_ERR_NULL
    for name in ("q", "k", "v", "g", "beta", "state", "slots", "out"):
        assert _step(**{name: PTR + 4}) == vb.VIG_ERR_ALIGN
    for name in ("B", "H", "Hk", "dk", "dv", "n_slots"):
        assert _step(**{name: 0}) == vb.VIG_ERR_SHAPE
    assert _step(slots=None, n_slots=2) == vb.VIG_ERR_SHAPE  # fewer states than sequences
    assert _step(dtype=-1) == vb.VIG_ERR_DTYPE
    assert _step(dk=24) == vb.VIG_ERR_UNSUPPORTED
    assert _step(H=3, Hk=2) == vb.VIG_ERR_UNSUPPORTED


def test_norm_refusals():
    L = vb.lib()

    def fwd(x=PTR, w=PTR, b=PTR, out=PTR, stats=PTR, B=2, Ln=4, C=64, G=4, eps=1e-5, act=1, dtype=vb.VIG_BF16, ws=PTR, ws_bytes=1 << 30):
        return L.group_norm_act_fwd(x, w, b, out, stats, B, Ln, C, G, eps, act, dtype, ws, ws_bytes, None)

    def bwd(x=PTR, w=PTR, b=PTR, stats=PTR, d=PTR, dx=PTR, dw=PTR, db=PTR, B=2, Ln=4, C=64, G=4, act=1, dtype=vb.VIG_BF16, ws=PTR,
            ws_bytes=1 << 30):
        return L.group_norm_act_bwd(x, w, b, stats, d, dx, dw, db, B, Ln, C, G, act, dtype, ws, ws_bytes, None)

    for call, names in ((fwd, ("x", "out", "stats")), (bwd, ("x", "stats", "d", "dx"))):
        for name in names:
            assert call(**{name: None}) == vb.VIG_ERR_NULL
        assert call(w=None) == vb.VIG_ERR_NULL and call(b=None) == vb.VIG_ERR_NULL  # one of the two alone
        for name in names + ("w", "b", "ws"):
            assert call(**{name: PTR + 8}) == vb.VIG_ERR_ALIGN
        for name in ("B", "Ln", "C", "G"):
            assert call(**{name: 0}) == vb.VIG_ERR_SHAPE
        assert call(dtype=4) == vb.VIG_ERR_DTYPE
        assert call(act=2) == vb.VIG_ERR_UNSUPPORTED
        assert call(C=60, G=4) == vb.VIG_ERR_UNSUPPORTED   # not a multiple of 8
        assert call(C=64, G=5) == vb.VIG_ERR_UNSUPPORTED
        assert call(C=16384, G=4) == vb.VIG_ERR_UNSUPPORTED
        assert call(B=1 << 16, Ln=1 << 30) == vb.VIG_ERR_SHAPE
    assert bwd(dw=None) == vb.VIG_ERR_NULL and bwd(db=None) == vb.VIG_ERR_NULL
    for eps in (0.0, -1.0, float("nan")):
        assert fwd(eps=eps) == vb.VIG_ERR_SHAPE
    need = L.group_norm_workspace_bytes(2, 5000, 64, 4, vb.VIG_BF16)
    assert need > 0 and fwd(Ln=5000, ws_bytes=need - 1) == vb.VIG_ERR_WORKSPACE and fwd(Ln=5000, ws=None, ws_bytes=0) == vb.VIG_ERR_WORKSPACE
    need = L.group_norm_bwd_workspace_bytes(2, 4, 64, 4, vb.VIG_BF16)
    assert need > 0 and bwd(ws_bytes=need - 1) == vb.VIG_ERR_WORKSPACE
    assert L.group_norm_workspace_bytes(2, 16, 64, 4, vb.VIG_BF16) == 0  # a group in registers
    assert L.group_norm_workspace_bytes(2, 16, 60, 4, vb.VIG_BF16) == 0
    assert f"#define VIG_GROUP_NORM_MAX_CHANNELS 8192" in open(HEADER).read()


def test_binding_refuses_cpu_tensors_and_names():
    t = torch.zeros(1, 1, 4, 16)
    s = torch.zeros(1, 1, 4)
    for call in (lambda: vb.gated_delta_fwd(t, t, t, s, s), lambda: vb.gated_delta_bwd(t, t, t, s, s, t),
                 lambda: vb.gated_delta_step(t[0], t[0], t[0], s[0], s[0], t), lambda: vb.group_norm_act_fwd(t, 1),
                 lambda: vb.gated_delta_fwd(t, t, t, s, s, direction="sideways"), lambda: vb.gated_delta_fwd(t, t, t, s, s, layout="hlbd"),
                 lambda: vb.group_norm_act_fwd(t, 1, act="tanh")):
        with pytest.raises(vb.VigError):
            call()


def test_header_names_the_new_constants():
    text = open(HEADER).read()
    for name, value in (("VIG_SCAN_FORWARD", vb.SCANS["forward"]), ("VIG_SCAN_BACKWARD", vb.SCANS["backward"]),
                        ("VIG_ACT_NONE", vb.ACTS["none"]), ("VIG_ACT_SILU", vb.ACTS["silu"]),
                        ("VIG_KERNEL_GATED_DELTA", vb.KERNELS["gated_delta"]),
                        ("VIG_KERNEL_GROUP_NORM_BACKWARD", vb.KERNELS["group_norm_backward"])):
        assert re.search(rf"\b{name} = {value}\b", text), name
    ms, n = ctypes.c_double(0.0), ctypes.c_long(0)
    assert vb.lib().vig_timing_collect(vb.KERNELS["group_norm_backward"], ctypes.byref(ms), ctypes.byref(n)) == vb.VIG_OK
    assert vb.lib().vig_timing_collect(vb.KERNELS["group_norm_backward"] + 1, ctypes.byref(ms), ctypes.byref(n)) == vb.VIG_ERR_SHAPE

"""GPU tests of what the binding of the gated delta rule and the group norm refuses: GPU tensors of another type, shape, order or place.  Every call raises
before a launch."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _wrong(t):
    """(what, tensor) like t but for one thing."""
    yield "type", t.to(torch.float16)
    yield "other type", t.to(F32 if t.dtype == BF16 else BF16)
    yield "order", torch.empty(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype, device=t.device)[..., ::2].copy_(t)
    yield "shape", torch.cat([t, t[:1]])
    yield "dimensions", t[None]
    yield "last axis", t[..., :-1].contiguous()
    yield "place", t.cpu()
    yield "kind", t.tolist()


def _refused(call, tensors, where):
    from paper_2405_18425_amd import binding as vb

    call(**tensors)
    for name in where:
        for what, bad in _wrong(tensors[name]):
            with pytest.raises(vb.VigError):
                call(**{**tensors, name: bad})
                pytest.fail(f"{name} of another {what} was taken")
    torch.cuda.synchronize()


def test_step():
    from paper_2405_18425_amd import binding as vb

    B, H, Hk, dk, dv = 5, 4, 2, 32, 64
    n = lambda *s: torch.randn(s, device="cuda").to(BF16)
    t = {"q": n(B, Hk, dk), "k": n(B, Hk, dk) * 0.1, "v": n(B, H, dv), "g": -n(B, H).abs(), "beta": n(B, H).sigmoid(),
         "state": torch.randn(7, H, dk, dv, device="cuda"), "out": torch.empty(B, H, dv, device="cuda", dtype=BF16)}
    # (a state of another number of slots and a wider last axis are sizes of their own: the first is a call like any other, see below)
    names = ("q", "k", "v", "g", "beta", "out")
    _refused(vb.gated_delta_step, t, names)
    once = t["state"].clone()
    for what, bad in _wrong(t["state"]):
        if what != "shape":
            with pytest.raises(vb.VigError):
                vb.gated_delta_step(**{**t, "state": bad})
    slots = torch.arange(B, device="cuda", dtype=torch.int32)
    for bad in (slots.long(), slots.float(), slots[:-1].contiguous(), torch.arange(2 * B, device="cuda", dtype=torch.int32)[::2], slots.cpu(), slots[None], slots.tolist()):
        with pytest.raises(vb.VigError):
            vb.gated_delta_step(**t, slots=bad)
    with pytest.raises(vb.VigError):
        vb.gated_delta_step(**{**t, "state": t["state"][:B - 1].contiguous()})  # fewer states than sequences
    torch.cuda.synchronize()
    assert torch.equal(t["state"], once)
    vb.gated_delta_step(**{**t, "state": torch.cat([t["state"], t["state"][:1]])})


@pytest.mark.parametrize("layout", ("bhld", "blhd"))
def test_sequences(layout):
    from paper_2405_18425_amd import binding as vb

    B, H, Hk, L, dk, dv = 2, 4, 2, 9, 32, 64
    heads = lambda h, *d: torch.randn((B, h, L, *d) if layout == "bhld" else (B, L, h, *d), device="cuda").to(BF16)
    t = {"q": heads(Hk, dk), "k": heads(Hk, dk) * 0.1, "v": heads(H, dv), "g": -heads(H).abs(), "beta": heads(H).sigmoid(),
         "initial_state": torch.randn(B, H, dk, dv, device="cuda")}
    forward = lambda **a: vb.gated_delta_fwd(**a, layout=layout)
    _refused(forward, {**t, "final_state": torch.empty_like(t["initial_state"]), "out": torch.empty_like(t["v"])},
             (*t, "final_state", "out"))
    _refused(lambda **a: vb.gated_delta_bwd(**a, layout=layout), {**t, "d_out": heads(H, dv), "d_final_state": t["initial_state"].clone()},
             (*t, "d_out", "d_final_state"))
    need = vb.gated_delta_workspace_bytes(B, H, Hk, L, dk, dv, vb.VIG_BF16)
    for bad in (torch.empty(need - 1, device="cuda", dtype=torch.uint8), torch.empty(need, dtype=torch.uint8)):
        with pytest.raises(vb.VigError):
            forward(**t, workspace=bad)


def test_norm():
    from paper_2405_18425_amd import binding as vb

    n = lambda *s: torch.randn(s, device="cuda").to(BF16)
    x = n(3, 50, 48)
    t = {"x": x, "weight": n(48), "bias": n(48), "out": torch.empty_like(x), "stats": torch.empty(3, 6, 2, device="cuda")}
    vb.group_norm_act_fwd(groups=6, **t)
    for call, tensors in ((vb.group_norm_act_fwd, t), (vb.group_norm_act_bwd, {**{k: t[k] for k in ("x", "weight", "bias", "stats")}, "d_out": n(3, 50, 48)})):
        _refused(lambda **a: call(groups=6, **a), tensors, tuple(tensors))
        for one in ("weight", "bias"):
            with pytest.raises(vb.VigError):
                call(groups=6, **{**tensors, one: None})
        for groups in (0, -1, 5, 7, 49):
            with pytest.raises(vb.VigError):
                call(groups=groups, **tensors)
    for bad in (x[:0], x[..., :0], x[0, 0], torch.randn(2, 3, 12, device="cuda")):
        with pytest.raises(vb.VigError):
            vb.group_norm_act_fwd(bad, 1)
    assert vb.group_norm_act_fwd(x[0], 6)[1].shape == (50, 6, 2)  # rows of channels: a group of one position each

"""GPU tests of calls of more than 2^24 workgroups of 256 threads, whose launch would pass 2^32 work-items.  References in 64 bits on the GPU,
a slice of the batch at a time.

Tolerances (bf16 results): half a step of their own rounding, 2^-8, and 2^-12 of the tensor's root mean square for the 32-bit
arithmetic before it, six of them since single values lie beyond it.  (The longest sums, over 2^24 rows in sixteen parts, are off by 2^-16 of the rms: 2^20
roundings of either sign, 2^-24 of a partial sum of up to 2^-2 of the whole's.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _close(got, want, rms, what):
    worst = ((got.double() - want).abs() / (2.0 ** -8 * want.abs() + 6 * 2.0 ** -12 * rms)).max().item()
    assert worst <= 1.0, f"{what}: {worst:.2f} of the bound"


# groups of 8 channels in one workgroup's registers, and of 4, which are strips' (one row each)
@pytest.mark.parametrize("B,C,groups", (((1 << 21) + 3, 64, 8), ((1 << 24) + 3, 8, 2)))
def test_norm_of_more_groups_than_a_launch_has_workgroups(B, C, groups):
    from paper_2405_18425_amd import binding as vb

    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(B, 1, C, device="cuda", generator=gen, dtype=BF16)
    d = torch.randn(B, 1, C, device="cuda", generator=gen, dtype=BF16)
    w, b = (torch.randn(C, device="cuda", generator=gen, dtype=BF16) for _ in range(2))
    y, stats = (torch.full_like(x, 77.0), torch.full((B, groups, 2), 77.0, device="cuda"))
    vb.group_norm_act_fwd(x, groups, w, b, act="none", out=y, stats=stats)
    dx, dw, db = vb.group_norm_act_bwd(x, d, stats, groups, w, b, act="none")
    torch.cuda.synchronize()
    want_dw, want_db = torch.zeros(C, dtype=torch.float64, device="cuda"), torch.zeros(C, dtype=torch.float64, device="cuda")
    step = 1 << 20
    for at in range(0, B, step):
        part = slice(at, min(B, at + step))
        xs, ds = x[part, 0].double(), d[part, 0].double()
        xg = xs.view(-1, groups, C // groups)
        mean, var = xg.mean(-1, keepdim=True), xg.var(-1, unbiased=False, keepdim=True)
        rstd = (var + 1e-5).rsqrt()
        xn = (xg - mean) * rstd
        _close(y[part, 0], xn.view(-1, C) * w.double() + b.double(), 1.0, f"out from {at}")
        assert ((stats[part, :, :1] - mean).abs() <= 2.0 ** -18).all() and ((stats[part, :, 1:] / rstd - 1).abs() <= 2.0 ** -18).all(), at
        dn = (ds * w.double()).view_as(xg)
        # (values of a group are few: a rounding of its own scale, 1 / sqrt(var), rather than the tensor's)
        want = rstd * (dn - dn.mean(-1, keepdim=True) - xn * (dn * xn).mean(-1, keepdim=True))
        _close(dx[part, 0].view_as(xg), want, rstd, f"dx from {at}")
        want_dw += (ds * xn.view(-1, C)).sum(0)
        want_db += ds.sum(0)
    rms = B ** 0.5
    _close(dw, want_dw, rms, "dw")
    _close(db, want_db, rms, "db")


def test_steps_of_more_heads_than_a_launch_has_workgroups():
    """2^20 sequences of 66 heads are 2^26 workgroups of 64 threads; but for some of the first and the last sequences they are padded rows."""
    from paper_2405_18425_amd import binding as vb

    B, H, Hk, d = 1 << 20, 66, 1, 16
    gen = torch.Generator(device="cuda").manual_seed(0)
    n = lambda *s: torch.randn(s, device="cuda", generator=gen, dtype=BF16)
    q, k, v, g, beta = n(B, Hk, d) * 0.25, n(B, Hk, d) * 0.25, n(B, H, d), -n(B, H).abs(), n(B, H).sigmoid()
    state = torch.randn(8, H, d, d, device="cuda", generator=gen)
    before = state.double()
    slots = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    live = torch.tensor([0, 5, B // 2, B - 40000, B - 5, B - 1], device="cuda")
    slots[live] = torch.tensor([3, 0, 7, 1, 6, 2], dtype=torch.int32, device="cuda")
    out = torch.full_like(v, 77.0)
    vb.gated_delta_step(q, k, v, g, beta, state, slots=slots, out=out)
    torch.cuda.synchronize()
    at = slots[live].long()
    S = before[at] * g[live].double().exp()[..., None, None]
    ks = k[live].double().expand(-1, H, -1)
    u = beta[live].double()[..., None] * (v[live].double() - (ks[..., None] * S).sum(-2))
    S = S + ks[..., None] * u[..., None, :]
    _close(out[live], (q[live].double().expand(-1, H, -1)[..., None] * S).sum(-2), 1.0, "out")
    assert ((state[at].double() - S).abs() <= 2.0 ** -18 * (1 + S.abs())).all()
    assert torch.equal(state[[4, 5]].double(), before[[4, 5]])  # of no sequence
    out[live] = 0
    assert not out.any()  # padded rows

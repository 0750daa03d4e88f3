"""GPU tests of the gated delta rule and the group norm on large problems: matrices that are written around the caches, workspaces beyond 4 GB, tensors
beyond 2^31 elements or 2^32 bytes.  Some heads or groups are compared, with the 64-bit references and the tolerances of the small ones."""
import pytest
import torch

import delta_norm_ref as ref
from test_delta_norm_gpu import BF16, F32, _close, _delta

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "g", "beta")


@pytest.mark.parametrize("direction", ("forward", "backward"))
def test_gradient_with_matrices_around_the_caches(direction):
    """48 heads of 64 chunks of 64 x 64: 163 MB of matrices, over the 128 MB from which they are streamed."""
    from paper_2405_18425_amd import binding as vb

    t = _delta(8, 6, 6, 4096, 64, 64, BF16, states=False, seed=1)
    got = vb.gated_delta_bwd(*(t[n] for n in NAMES), t["d_out"], direction=direction)
    for b, h in ((0, 0), (7, 5)):
        head = lambda x: x[b:b + 1, h:h + 1]
        want = ref.delta_bwd(*(head(t[n]) for n in NAMES), head(t["d_out"]), direction=direction)
        for name, a, e in zip(("dq", "dk", "dv", "dg", "dbeta"), got, want):
            _close(head(a), e, BF16, f"{b} {h} {name}")


@pytest.mark.parametrize("dtype,H,Hk,L,dk,dv", ((BF16, 6, 6, 8192, 64, 64), (F32, 8, 4, 3300, 128, 64)))
def test_forward_with_matrices_around_the_caches(dtype, H, Hk, L, dk, dv):
    from paper_2405_18425_amd import binding as vb

    B = 8
    t = _delta(B, H, Hk, L, dk, dv, dtype, "blhd", states=True, seed=2)
    args = [t[n] for n in NAMES]
    assert vb.gated_delta_workspace_bytes(B, H, Hk, L, dk, dv, vb.VIG_BF16 if dtype == BF16 else vb.VIG_F32) > 128 << 20
    out, fin = vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=True, layout="blhd")
    share = H // Hk
    for b, h in ((0, 0), (B - 1, H - 1)):
        key, head = (lambda x: x[b:b + 1, :, h // share:h // share + 1]), (lambda x: x[b:b + 1, :, h:h + 1])
        want, want_fin = ref.delta_fwd(key(args[0]), key(args[1]), *(head(x) for x in args[2:]), t["s0"][b:b + 1, h:h + 1], "blhd")
        _close(head(out), want, dtype, f"{b} {h} out")
        _close(fin[b:b + 1, h:h + 1], want_fin, F32, f"{b} {h} state")


@pytest.mark.parametrize("direction", ("forward", "backward"))
def test_gradient_beyond_32_bits(direction):
    """Token-major values of 4.3 GB and a workspace of 40 GB: the last tokens of the first and the last head."""
    from paper_2405_18425_amd import binding as vb

    B, H, L, dk, dv = 1, 128, (1 << 17) + 70, 16, 128
    gen = torch.Generator(device="cuda").manual_seed(0)
    n = lambda *s: torch.randn(s, device="cuda", dtype=BF16, generator=gen)
    q, v, d_out = n(B, L, H, dk) * 0.25, n(B, L, H, dv), n(B, L, H, dv)
    k = torch.nn.functional.normalize(n(B, L, H, dk).float(), dim=-1).to(BF16)
    g = torch.full((B, L, H), -0.25, device="cuda", dtype=BF16)
    beta = torch.full((B, L, H), 0.5, device="cuda", dtype=BF16)
    assert v.numel() * 2 > 1 << 32
    got = vb.gated_delta_bwd(q, k, v, g, beta, d_out, layout="blhd", direction=direction)
    torch.cuda.synchronize()
    tail = slice(L - 330, L)  # what is 200 tokens before the last 130 has decayed to exp(-50) of itself, in either scan direction
    for h in (0, H - 1):
        cut = lambda x: x[:, tail, h:h + 1]
        want = ref.delta_bwd(*(cut(x) for x in (q, k, v, g, beta)), cut(d_out), layout="blhd", direction=direction)
        for name, a, e in zip(("dq", "dk", "dv", "dg", "dbeta"), got, want):
            _close(a[:, L - 130:, h:h + 1], e[:, -130:], BF16, f"head {h} {name}")


def test_norm_beyond_31_bits():
    """Two elements of 2^30 values and more: the second one's last group, and the channels of that group."""
    from paper_2405_18425_amd import binding as vb

    B, L, C, G = 2, (1 << 18) + 5, 4096, 32
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, d = (torch.randn(B, L, C, device="cuda", dtype=BF16, generator=gen) for _ in range(2))
    w, b = (torch.randn(C, device="cuda", dtype=BF16, generator=gen) for _ in range(2))
    assert x.numel() > 1 << 31
    y, stats = vb.group_norm_act_fwd(x, G, w, b)
    dx, dw, db = vb.group_norm_act_bwd(x, d, stats, G, w, b)
    torch.cuda.synchronize()
    at = slice(C - C // G, C)
    want_dw, want_db = 0, 0
    for e in range(B):
        xs, ds, ws, bs = (t.double() for t in (x[e, :, at], d[e, :, at], w[at], b[at]))
        mean, rstd = xs.mean(), (xs.var(unbiased=False) + 1e-5).rsqrt()
        assert abs(stats[e, -1, 0].item() - mean.item()) <= 2 ** -16 and abs(stats[e, -1, 1].item() / rstd.item() - 1) <= 2 ** -16
        xn = (xs - mean) * rstd
        z = xn * ws + bs
        sig = torch.sigmoid(z)
        da = ds * sig * (1 + z * (1 - sig))
        dn = da * ws
        want_dw, want_db = want_dw + (da * xn).sum(0), want_db + da.sum(0)
        if e == B - 1:
            rows = slice(L - 1000, L)
            _close(y[e, rows, at], (z * sig)[rows].cpu(), BF16, "out")
            _close(dx[e, rows, at], (rstd * (dn - dn.mean() - xn * (dn * xn).mean()))[rows].cpu(), BF16, "dx")
    _close(dw[at], want_dw.cpu(), BF16, "dw")
    _close(db[at], want_db.cpu(), BF16, "db")

"""Plain 64-bit implementations of the gated delta rule and the channels-last group norm, on the CPU: the recurrence token by
token and its adjoint, the norm from its formulas.  Test infrastructure."""
from __future__ import annotations

import torch

F64 = torch.float64


def scan_order(x, layout, direction, share=1):
    """[L, B, H, ...] in scan order, in 64 bits; `share`: value heads per key head."""
    x = x.detach().cpu().to(F64)
    x = x.permute(2, 0, 1, *range(3, x.dim())) if layout == "bhld" else x.transpose(0, 1)
    if direction == "backward":
        x = x.flip(0)
    return x.repeat_interleave(share, 2)


def back(x, layout, direction, share=1):
    if share > 1:
        x = x.unflatten(2, (-1, share)).sum(3)
    if direction == "backward":
        x = x.flip(0)
    return x.permute(1, 2, 0, *range(3, x.dim())) if layout == "bhld" else x.transpose(0, 1)


def _heads(q, v, layout):
    return (q.shape[1], v.shape[1]) if layout == "bhld" else (q.shape[2], v.shape[2])


def delta_fwd(q, k, v, g, beta, initial=None, layout="bhld", direction="forward"):
    """(out, final state) in 64 bits."""
    Hk, H = _heads(q, v, layout)
    qs, ks = (scan_order(x, layout, direction, H // Hk) for x in (q, k))
    vs, gs, bs = (scan_order(x, layout, direction) for x in (v, g, beta))
    L, B = vs.shape[:2]
    S = torch.zeros(B, H, q.shape[-1], v.shape[-1], dtype=F64) if initial is None else initial.detach().cpu().to(F64)
    out = []
    for t in range(L):
        S = gs[t].exp()[..., None, None] * S
        e = vs[t] - torch.einsum("bhk,bhkv->bhv", ks[t], S)
        S = S + ks[t][..., None] * (bs[t][..., None] * e)[..., None, :]
        out.append(torch.einsum("bhk,bhkv->bhv", qs[t], S))
    return back(torch.stack(out), layout, direction), S


def delta_bwd(q, k, v, g, beta, d_out, initial=None, d_final=None, layout="bhld", direction="forward"):
    """(dq, dk, dv, dg, dbeta, d_initial) in 64 bits, from the adjoint of the recurrence."""
    Hk, H = _heads(q, v, layout)
    share = H // Hk
    qs, ks = (scan_order(x, layout, direction, share) for x in (q, k))
    vs, gs, bs, dos = (scan_order(x, layout, direction) for x in (v, g, beta, d_out))
    L, B = vs.shape[:2]
    zero = torch.zeros(B, H, q.shape[-1], v.shape[-1], dtype=F64)
    S = zero if initial is None else initial.detach().cpu().to(F64)
    decayed, wrong = [], []
    for t in range(L):
        S = gs[t].exp()[..., None, None] * S
        e = vs[t] - torch.einsum("bhk,bhkv->bhv", ks[t], S)
        decayed.append(S)
        wrong.append(e)
        S = S + ks[t][..., None] * (bs[t][..., None] * e)[..., None, :]
    D = zero.clone() if d_final is None else d_final.detach().cpu().to(F64)
    dq, dk, dv, dg, db = [], [], [], [], []
    for t in range(L - 1, -1, -1):
        b = bs[t][..., None]
        S = decayed[t] + ks[t][..., None] * (b * wrong[t])[..., None, :]
        dq.append(torch.einsum("bhkv,bhv->bhk", S, dos[t]))
        D = D + qs[t][..., None] * dos[t][..., None, :]
        r = torch.einsum("bhk,bhkv->bhv", ks[t], D)
        dv.append(b * r)
        db.append((r * wrong[t]).sum(-1))
        dk.append(torch.einsum("bhkv,bhv->bhk", D, b * wrong[t]) - torch.einsum("bhkv,bhv->bhk", decayed[t], b * r))
        D = D - ks[t][..., None] * (b * r)[..., None, :]
        dg.append((D * decayed[t]).sum((-1, -2)))
        D = gs[t].exp()[..., None, None] * D
    stack = lambda x: torch.stack(x[::-1])
    return (back(stack(dq), layout, direction, share), back(stack(dk), layout, direction, share),
            *(back(stack(x), layout, direction) for x in (dv, dg, db)), D)


def norm_fwd(x, groups, weight=None, bias=None, eps=1e-5, act="silu"):
    """(out, stats [B, groups, 2]) in 64 bits; x: [B, L, C]."""
    x = x.detach().cpu().to(F64)
    B, L, C = x.shape
    xg = x.reshape(B, L, groups, C // groups)
    mean = xg.mean((1, 3))
    rstd = ((xg - mean[:, None, :, None]) ** 2).mean((1, 3)).add(eps).rsqrt()
    z = ((xg - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(B, L, C)
    if weight is not None:
        z = z * weight.detach().cpu().to(F64) + bias.detach().cpu().to(F64)
    return (z * torch.sigmoid(z) if act == "silu" else z), torch.stack((mean, rstd), -1)


def norm_bwd(x, d_out, groups, weight=None, bias=None, eps=1e-5, act="silu"):
    """(dx, d_weight, d_bias) in 64 bits."""
    _, stats = norm_fwd(x, groups, eps=eps, act="none")
    x, d = (t.detach().cpu().to(F64) for t in (x, d_out))
    B, L, C = x.shape
    mean, rstd = (stats[..., i][:, None, :, None] for i in (0, 1))
    xn = ((x.reshape(B, L, groups, -1) - mean) * rstd).reshape(B, L, C)
    w = torch.ones(C, dtype=F64) if weight is None else weight.detach().cpu().to(F64)
    b = torch.zeros(C, dtype=F64) if bias is None else bias.detach().cpu().to(F64)
    if act == "silu":
        s = torch.sigmoid(xn * w + b)
        d = d * (s + (xn * w + b) * s * (1 - s))
    dn, xg = (d * w).reshape(B, L, groups, -1), xn.reshape(B, L, groups, -1)
    dx = rstd * (dn - dn.mean((1, 3), keepdim=True) - xg * (dn * xg).mean((1, 3), keepdim=True))
    return dx.reshape(B, L, C), (d * xn).sum((0, 1)), d.sum((0, 1))

"""The gated delta rule (chunked forward, gradient, single-token step) and the channels-last group norm with an
activation, as cases that can be timed and compared.

With `own` false, `run` computes an operator in elementary torch operations in 32 bits (the chunk form of the delta rule,
its gradient by differentiating that form); with `own` true it calls paper_2405_18425_amd.binding.  `exact` evaluates the
definitions in 64 bits: the recurrence and its adjoint token by token, the norm by its formulas.
"""
import math

import torch

own = False

TAU = 4.0    # gates: log sigmoid(z) / TAU, 0.02 to 0.5 nats a token
CHUNK = 64   # of the plain form
EPS = 1e-5   # of the group norm


def _delta(name, op, B, H, L, dk=64, dv=64, Hk=None, dtype="bf16", layout="bhld", direction="forward", states=False, mu=1.0):
    return {"name": name, "op": op, "B": B, "H": H, "Hk": Hk or H, "L": L, "dk": dk, "dv": dv, "dtype": dtype, "layout": layout,
            "direction": direction, "states": states, "mu": mu}


def _step(name, B, H, dk, dv, Hk=None, dtype="bf16", slots=0, padded=0, mu=1.0):
    return {"name": name, "op": "step", "B": B, "H": H, "Hk": Hk or H, "dk": dk, "dv": dv, "dtype": dtype, "slots": slots,
            "padded": padded, "mu": mu}


def _norm(name, op, B, L, C, groups, dtype="bf16", act="silu", affine=True, mean=0.5):
    return {"name": name, "op": op, "B": B, "L": L, "C": C, "groups": groups, "dtype": dtype, "act": act, "affine": affine,
            "mean": mean}


def listed():
    return [
        # one 224-pixel image through a mixer of the small model, token-major as projections emit it: latency
        _delta("one_image_224", "fwd", 1, 6, 196, layout="blhd"),
        # 1024-pixel images, small model, the direction that scans from the last token on: few long sequences
        _delta("vig_s_1024", "fwd", 8, 6, 4096, direction="backward", mu=-1.0),
        # two long prompts, wide heads of which two share keys, state in and state out: a server's prefill
        _delta("prompts_shared_keys", "fwd", 2, 16, 8191, 128, 128, Hk=8, layout="blhd", states=True, mu=2.0),
        # the ImageNet training shape of the small model: many short sequences
        _delta("vig_s_224_train", "bwd", 64, 6, 196),
        # training at 1024 pixels
        _delta("vig_s_1024_train", "bwd", 8, 6, 4096, mu=-1.0),
        # full precision on a grid that is a multiple of nothing, shared narrow keys, states: validating a training run
        _delta("ragged_37x53_f32_train", "bwd", 3, 6, 37 * 53, 32, 64, Hk=3, dtype="f32", layout="blhd", direction="backward",
               states=True),
        # one stream's next token: latency
        _step("one_stream_step", 1, 6, 64, 64),
        # a server's batch, padded to the size that its graph was captured for, states in a pool
        _step("many_streams_step", 128, 16, 128, 128, Hk=8, slots=150, padded=11),
        # last stage of a hierarchical model at 224 pixels, a group a head
        _norm("stage4_7x7_norm", "norm", 64, 49, 1024, 16),
        # the small model's grid at 1024 pixels
        _norm("vig_s_1024_norm", "norm", 8, 4096, 384, 6),
        # first stage at 224 pixels, training
        _norm("stage1_56x56_norm_train", "norm_bwd", 16, 3136, 128, 2),
        # full precision, groups of six channels, no activation: validating a training run
        _norm("f32_224_norm_train", "norm_bwd", 4, 196, 192, 32, dtype="f32", act="none"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("fwd", "fwd", "bwd", "bwd", "step", "norm", "norm_bwd"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if op in ("norm", "norm_bwd"):
        most = 8 * 4096 * 384 if op == "norm" else 16 * 3136 * 128
        while True:
            B, L = _log_int(rng, 1, 64), _log_int(rng, 1, 4096)
            groups = rng.choice((1, 2, 3, 4, 6, 8, 16, 32))
            C = groups * rng.choice((8, 16, 24, 32, 64))
            if B * L * C <= most:
                break
        case = _norm("", op, B, L, C, groups, dtype, rng.choice(("silu", "silu", "none")), rng.random() < 0.8,
                     round(rng.uniform(-2.0, 2.0), 1))
    else:
        Hk, share = rng.choice((1, 2, 3, 4, 6, 8)), rng.choice((1, 1, 2, 4))
        dk, dv = rng.choice(((64, 64), (64, 64), (128, 128), (32, 64), (16, 16), (64, 128)))
        mu = round(rng.uniform(-2.0, 3.0), 1)
        if op == "step":
            while True:
                B = _log_int(rng, 1, 128)
                if B * Hk * share * dk * dv <= 128 * 16 * 128 * 128:
                    break
            padded = rng.randrange(0, B // 4 + 1)
            case = _step("", B, Hk * share, dk, dv, Hk, dtype, rng.choice((0, B + rng.randrange(0, 20))), padded, mu)
            case["padded"] = padded if case["slots"] else 0
        else:
            most = (2 * 16 * 8191 * 128 * 128 if op == "fwd" else 8 * 6 * 4096 * 64 * 64) // (8 if dtype == "f32" else 1)
            while True:
                B, L = _log_int(rng, 1, 64), _log_int(rng, 1, 8191 if op == "fwd" else 4096)
                if B * Hk * share * L * dk * dv <= most:
                    break
            case = _delta("", op, B, Hk * share, L, dk, dv, Hk, dtype, rng.choice(("bhld", "blhd")),
                          rng.choice(("forward", "backward")), rng.random() < 0.4, mu)
    del case["name"]
    return case


def _unit(x):
    return x / x.square().sum(-1, keepdim=True).sqrt().clamp_min(1e-6)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = {"case": case}
    B = case["B"]
    if case["op"] in ("norm", "norm_bwd"):
        L, C, G = case["L"], case["C"], case["groups"]
        s["x"] = (normal(B, L, C) * (0.5 + normal(C).abs()) + case["mean"] * normal(C)).to(dtype)
        s["weight"] = (1.0 + 0.2 * normal(C)).to(dtype) if case["affine"] else None
        s["bias"] = (0.2 * normal(C)).to(dtype) if case["affine"] else None
        if case["op"] == "norm_bwd":
            s["d_out"] = normal(B, L, C).to(dtype)
            x = s["x"].double().view(B, L, G, C // G)  # the forward's statistics
            mean = x.mean((1, 3))
            var = (x - mean[:, None, :, None]).square().mean((1, 3))
            s["stats"] = torch.stack((mean, (var + EPS).rsqrt()), -1).float().contiguous()
        return s
    H, Hk, dk, dv = case["H"], case["Hk"], case["dk"], case["dv"]
    if case["op"] == "step":
        s["q"] = (_unit(normal(B, Hk, dk)) * dk ** -0.5).to(dtype)
        s["k"] = _unit(normal(B, Hk, dk)).to(dtype)
        s["v"] = normal(B, H, dv).to(dtype)
        s["g"] = (torch.nn.functional.logsigmoid(normal(B, H) + case["mu"]) / TAU).to(dtype)
        s["beta"] = torch.sigmoid(normal(B, H)).to(dtype)
        pool = case["slots"] or B
        s["state"] = normal(pool, H, dk, dv)
        s["slots"] = None
        if case["slots"]:
            order = torch.randperm(pool, generator=gen, device="cuda")[:B].to(torch.int32)
            if case["padded"]:
                order[B - case["padded"]:] = -1
            s["slots"] = order
        return s
    L = case["L"]

    def heads(h, *d):
        return (B, h, L, *d) if case["layout"] == "bhld" else (B, L, h, *d)

    s["q"] = (_unit(normal(*heads(Hk, dk))) * dk ** -0.5).to(dtype)
    s["k"] = _unit(normal(*heads(Hk, dk))).to(dtype)
    s["v"] = normal(*heads(H, dv)).to(dtype)
    s["g"] = (torch.nn.functional.logsigmoid(normal(*heads(H)) + case["mu"]) / TAU).to(dtype)
    s["beta"] = torch.sigmoid(normal(*heads(H))).to(dtype)
    s["initial"] = normal(B, H, dk, dv) if case["states"] else None
    if case["op"] == "bwd":
        s["d_out"] = normal(*heads(H, dv)).to(dtype)
        s["d_final"] = 0.1 * normal(B, H, dk, dv) if case["states"] else None
    return s


# ---- plain forms ---------------------------------------------------------------------------------

def _plain_delta(q, k, v, g, beta, state):
    """Chunk form in 32 bits; [B, H, L, d] in, output and final state out."""
    B, H, L, dk = q.shape
    n = -(-L // CHUNK)
    pad = n * CHUNK - L
    q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, pad)).view(B, H, n, CHUNK, x.shape[-1]) for x in (q, k, v))
    g, beta = (torch.nn.functional.pad(x, (0, pad)).view(B, H, n, CHUNK) for x in (g, beta))
    b = g.double().cumsum(-1)  # differences of long sums: 64 bits
    at = torch.arange(CHUNK, device=q.device)
    later = at[:, None] < at[None, :]
    decay = (b[..., :, None] - b[..., None, :]).masked_fill(later, -math.inf).exp().float()
    gamma, rest = b.exp().float()[..., None], (b[..., -1:] - b).exp().float()[..., None]
    a = beta[..., None] * decay * (k @ k.transpose(-1, -2))
    a = a.masked_fill(at[:, None] <= at[None, :], 0.0)
    t = torch.eye(CHUNK, device=q.device)
    for level in range(6):  # inverse of 1 + a: blocks of 2^level are joined to blocks twice as large
        block = at >> level
        below = (block[:, None] == block[None, :] + 1) & (block[:, None] % 2 == 1)
        t = t - t @ (a * below) @ t
    u_own, u_state = t @ (beta[..., None] * v), t @ (beta[..., None] * gamma * k)
    scores, keys, reads = decay * (q @ k.transpose(-1, -2)), (rest * k).transpose(-1, -2), gamma * q
    out = []
    for c in range(n):
        u = u_own[:, :, c] - u_state[:, :, c] @ state
        out.append(reads[:, :, c] @ state + scores[:, :, c] @ u)
        state = gamma[:, :, c, -1:] * state + keys[:, :, c] @ u
    return torch.stack(out, 2).reshape(B, H, n * CHUNK, -1)[:, :, :L], state


def _sequences(s, names):
    """32-bit [B, heads, L, ...] in scan order, every tensor with the value heads."""
    c = s["case"]
    got = []
    for name in names:
        x = s[name].float()
        x = x.transpose(1, 2) if c["layout"] == "blhd" else x
        got.append(x.flip(2) if c["direction"] == "backward" else x)
    return got


def _back(x, c, dtype):
    x = x.flip(2) if c["direction"] == "backward" else x
    return (x.transpose(1, 2) if c["layout"] == "blhd" else x).to(dtype).contiguous()


def _plain_fwd(s):
    c, dtype = s["case"], s["v"].dtype
    q, k, v, g, beta = _sequences(s, ("q", "k", "v", "g", "beta"))
    share = c["H"] // c["Hk"]
    q, k = q.repeat_interleave(share, 1), k.repeat_interleave(share, 1)
    state = s["initial"] if c["states"] else v.new_zeros(c["B"], c["H"], c["dk"], c["dv"])
    out, final = _plain_delta(q, k, v, g, beta, state)
    out = _back(out, c, dtype)
    return (out, final) if c["states"] else out


def _plain_bwd(s):
    c, dtype = s["case"], s["v"].dtype
    leaves = [x.detach().requires_grad_() for x in _sequences(s, ("q", "k", "v", "g", "beta"))]
    state = s["initial"] if c["states"] else leaves[2].new_zeros(c["B"], c["H"], c["dk"], c["dv"])
    state = state.detach().requires_grad_()
    share = c["H"] // c["Hk"]
    with torch.enable_grad():
        out, final = _plain_delta(leaves[0].repeat_interleave(share, 1), leaves[1].repeat_interleave(share, 1), *leaves[2:], state)
        d_out = _sequences(s, ("d_out",))[0]
        loss = (out * d_out).sum()
        if c["states"]:
            loss = loss + (final * s["d_final"]).sum()
    grads = torch.autograd.grad(loss, leaves + [state])
    got = tuple(_back(x, c, dtype) for x in grads[:5])
    return got + (grads[5],) if c["states"] else got


def _plain_step(s):
    c, dtype = s["case"], s["v"].dtype
    share = c["H"] // c["Hk"]
    q, k = (s[n].float().repeat_interleave(share, 1) for n in ("q", "k"))
    v, g, beta = (s[n].float() for n in ("v", "g", "beta"))
    live = slice(0, c["B"] - c["padded"])
    at = s["slots"][live].long() if s["slots"] is not None else torch.arange(c["B"], device=v.device)
    q, k, v, g, beta = (x[live] for x in (q, k, v, g, beta))
    state = s["state"][at] * g.exp()[..., None, None]
    u = beta[..., None] * (v - (k[..., None] * state).sum(-2))
    state = state + k[..., None] * u[..., None, :]
    out = torch.zeros_like(s["v"])
    out[live] = (q[..., None] * state).sum(-2).to(dtype)
    s["state"][at] = state
    return out, s["state"]


def _plain_norm(s):
    c = s["case"]
    B, L, C, G = c["B"], c["L"], c["C"], c["groups"]
    x = s["x"].float().view(B, L, G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    rstd = ((x - mean).square().mean((1, 3), keepdim=True) + EPS).rsqrt()
    y = ((x - mean) * rstd).view(B, L, C)
    if c["affine"]:
        y = y * s["weight"].float() + s["bias"].float()
    y = y * torch.sigmoid(y) if c["act"] == "silu" else y
    return y.to(s["x"].dtype), torch.stack((mean.view(B, G), rstd.view(B, G)), -1)


def _plain_norm_bwd(s):
    c, dtype = s["case"], s["x"].dtype
    B, L, C, G = c["B"], c["L"], c["C"], c["groups"]
    mean, rstd = (s["stats"][..., i].view(B, 1, G, 1) for i in (0, 1))
    xn = ((s["x"].float().view(B, L, G, C // G) - mean) * rstd).view(B, L, C)
    w = s["weight"].float() if c["affine"] else torch.ones(C, device=xn.device)
    d = s["d_out"].float()
    if c["act"] == "silu":
        z = xn * w + s["bias"].float() if c["affine"] else xn
        sig = torch.sigmoid(z)
        d = d * sig * (1 + z * (1 - sig))
    dn = (d * w).view(B, L, G, C // G)
    xg = xn.view(B, L, G, C // G)
    dx = rstd * (dn - dn.mean((1, 3), keepdim=True) - xg * (dn * xg).mean((1, 3), keepdim=True))
    dx = dx.view(B, L, C).to(dtype)
    return (dx, (d * xn).sum((0, 1)).to(dtype), d.sum((0, 1)).to(dtype)) if c["affine"] else dx


# ---- one pass ------------------------------------------------------------------------------------

def _own(s):
    from paper_2405_18425_amd import binding as vb

    c, op = s["case"], s["case"]["op"]
    if op == "fwd":
        return vb.gated_delta_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], initial_state=s["initial"],
                                  return_final_state=c["states"], layout=c["layout"], direction=c["direction"])
    if op == "bwd":
        return vb.gated_delta_bwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["d_out"], initial_state=s["initial"],
                                  d_final_state=s["d_final"], layout=c["layout"], direction=c["direction"])
    if op == "step":
        return vb.gated_delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state"], slots=s["slots"]), s["state"]
    if op == "norm":
        return vb.group_norm_act_fwd(s["x"], c["groups"], s["weight"], s["bias"], eps=EPS, act=c["act"])
    got = vb.group_norm_act_bwd(s["x"], s["d_out"], s["stats"], c["groups"], s["weight"], s["bias"], act=c["act"])
    return got if c["affine"] else got[0]


def run(s):
    if own:
        return _own(s)
    return {"fwd": _plain_fwd, "bwd": _plain_bwd, "step": _plain_step, "norm": _plain_norm,
            "norm_bwd": _plain_norm_bwd}[s["case"]["op"]](s)


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    B, op = case["B"], case["op"]
    if op in ("norm", "norm_bwd"):
        values = B * case["L"] * case["C"]
        vectors = case["C"] * (2 if op == "norm" else 4) if case["affine"] else 0
        return {"bytes": (values * (2 if op == "norm" else 3) + vectors) * size + B * case["groups"] * 8,
                "flops": values * (15 if op == "norm" else 30)}
    H, Hk, dk, dv = case["H"], case["Hk"], case["dk"], case["dv"]
    state = dk * dv * 4
    if op == "step":
        live = B - case["padded"]
        return {"bytes": live * H * 2 * state + B * (2 * Hk * dk + 2 * H * dv + 2 * H) * size + (4 * B if case["slots"] else 0),
                "flops": live * H * 7 * dk * dv}
    tokens = B * case["L"]
    if op == "fwd":  # read, correct, write and read out a state per token: three products of a row with the state
        return {"bytes": tokens * (2 * Hk * dk + 2 * H * dv + 2 * H) * size + (2 * B * H * state if case["states"] else 0),
                "flops": tokens * H * 6 * dk * dv}
    # the states again (two products), their adjoints (three), and dq, dk (two of them)
    return {"bytes": tokens * (4 * Hk * dk + 3 * H * dv + 4 * H) * size + (3 * B * H * state if case["states"] else 0),
            "flops": tokens * H * 16 * dk * dv}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _scan_order(s, name):
    c, x = s["case"], s[name].double()
    if c["layout"] == "bhld":
        x = x.movedim(2, 0)
    else:
        x = x.movedim(1, 0)
    if c["direction"] == "backward":
        x = x.flip(0)
    if name in ("q", "k"):
        x = x.repeat_interleave(c["H"] // c["Hk"], 2)
    return x.contiguous()  # [L, B, H, ...]


def _leave_order(x, c, shared=False):
    if shared and c["H"] != c["Hk"]:
        x = x.unflatten(2, (c["Hk"], c["H"] // c["Hk"])).sum(3)
    if c["direction"] == "backward":
        x = x.flip(0)
    return x.movedim(0, 2 if c["layout"] == "bhld" else 1)


def _exact_delta(s):
    """S_t = a_t (1 - b_t k_t^T k_t) S_{t-1} + b_t k_t^T v_t and o_t = q_t S_t, token by token, and the adjoint of that."""
    c = s["case"]
    q, k, v, g, beta = (_scan_order(s, n) for n in ("q", "k", "v", "g", "beta"))
    alpha = g.exp()
    state = s["initial"].double() if c["states"] else torch.zeros(c["B"], c["H"], c["dk"], c["dv"], dtype=torch.float64, device=q.device)
    train, before, out = c["op"] == "bwd", [], []
    for t in range(c["L"]):
        if train:
            before.append(state)
        kt = k[t][..., None]
        state = alpha[t][..., None, None] * state
        wrong = v[t] - (kt * state).sum(-2)
        state = state + kt * (beta[t][..., None] * wrong)[..., None, :]
        if not train:
            out.append((q[t][..., None] * state).sum(-2))
    if not train:
        o = _leave_order(torch.stack(out), c)
        return (o, state) if c["states"] else o
    d_out = _scan_order(s, "d_out")
    ds = s["d_final"].double() if c["states"] else torch.zeros_like(state)
    dq, dk, dv, dg, db = [], [], [], [], []
    for t in range(c["L"] - 1, -1, -1):
        kt, bt, dot = k[t][..., None], beta[t][..., None], d_out[t][..., None, :]
        decayed = alpha[t][..., None, None] * before[t]
        wrong = v[t] - (kt * decayed).sum(-2)
        after = decayed + kt * (bt * wrong)[..., None, :]
        dq.append((after * dot).sum(-1))
        ds = ds + q[t][..., None] * dot
        du = (kt * ds).sum(-2)                       # of u = beta * wrong
        dwrong = bt * du
        dv.append(dwrong)
        db.append((du * wrong).sum(-1))
        dk.append((ds * (bt * wrong)[..., None, :]).sum(-1) - (decayed * dwrong[..., None, :]).sum(-1))
        ds = ds - kt * dwrong[..., None, :]          # of the decayed state
        dg.append((ds * decayed).sum((-1, -2)))
        ds = alpha[t][..., None, None] * ds
    dq, dk, dv, dg, db = (torch.stack(x[::-1]) for x in (dq, dk, dv, dg, db))
    got = (_leave_order(dq, c, True), _leave_order(dk, c, True), *(_leave_order(x, c) for x in (dv, dg, db)))
    return got + (ds,) if c["states"] else got


def exact(case, seed):
    if case["op"] == "bwd" and case["B"] * case["H"] * case["L"] * case["dk"] * case["dv"] * 8 > 60e9:
        return None  # the states of all tokens would not fit beside the inputs
    s = prepare(case, seed)
    if case["op"] in ("fwd", "bwd"):
        return _exact_delta(s)
    if case["op"] == "step":
        share, state = case["H"] // case["Hk"], s["state"].double()
        out = torch.zeros(s["v"].shape, dtype=torch.float64, device=state.device)
        rows = s["slots"].tolist() if s["slots"] is not None else range(case["B"])
        for i, at in enumerate(rows):
            if at < 0:
                continue
            q, k = (s[n][i].double().repeat_interleave(share, 0) for n in ("q", "k"))
            now = state[at] * s["g"][i].double().exp()[:, None, None]
            wrong = s["v"][i].double() - torch.matmul(k[:, None, :], now)[:, 0]
            now = now + k[:, :, None] * (s["beta"][i].double()[:, None] * wrong)[:, None, :]
            out[i] = torch.matmul(q[:, None, :], now)[:, 0]
            state[at] = now
        return out, state
    B, L, C, G = case["B"], case["L"], case["C"], case["groups"]
    x = s["x"].double().view(B, L, G, -1)
    mean = x.mean((1, 3), keepdim=True)
    std = (x.var((1, 3), unbiased=False, keepdim=True) + EPS).sqrt()
    xn = ((x - mean) / std).view(B, L, C)
    w, b = (s[n].double() if case["affine"] else torch.full((C,), f, dtype=torch.float64, device=x.device) for n, f in (("weight", 1.0), ("bias", 0.0)))
    z = xn * w + b
    if case["op"] == "norm":
        return (z / (1 + (-z).exp()) if case["act"] == "silu" else z), torch.stack((mean.view(B, G), 1 / std.view(B, G)), -1)
    dz = s["d_out"].double()
    if case["act"] == "silu":
        e = (-z).exp()
        dz = dz * (1 / (1 + e) + z * e / (1 + e) ** 2)
    dn, xn4 = (dz * w).view(B, L, G, -1), xn.view(B, L, G, -1)
    dx = ((dn - dn.mean((1, 3), keepdim=True) - xn4 * (dn * xn4).mean((1, 3), keepdim=True)) / std).view(B, L, C)
    return (dx, (dz * xn).sum((0, 1)), dz.sum((0, 1))) if case["affine"] else dx

"""GPU tests of the gated delta rule and the channels-last group norm, through the binding, against the 64-bit references.

Tolerances, as a share of the reference's size plus a share of its root mean square over the tensor:
  bf16 results: half a step of their own rounding, 2^-8, plus 2^-11 for the arithmetic before it.  Operands that are not inputs are
  held to 2^-17 (two bf16 parts); at most four of them stand between an input and a result of a chunk, each in sums of up to 128
  terms of either sign, and a chunk's errors reach later ones through decays of at most one: 4 * 2^-17 * 16 = 2^-11.
  32-bit results (fp32 calls, states, statistics): sums of up to 128 channels and 64 tokens in 32 bits, three parts (2^-25) where
  the inputs are bf16: 256 * 2^-24 = 2^-16."""
import pytest
import torch

import delta_norm_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _close(got, want, dtype, what):
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    rms = want.square().mean().sqrt()
    rel, absolute = (2.0 ** -8, 2.0 ** -11) if dtype == BF16 else (2.0 ** -16, 2.0 ** -16)
    # (the rounding of a value that is itself off by `absolute` of the rms; 6 covers the values beyond the rms)
    bound = rel * want.abs() + 6 * absolute * rms + 1e-30
    worst = ((got - want).abs() / bound).max().item()
    assert worst <= 1.0, f"{what}: {worst:.2f} of the bound"


def _delta(B, H, Hk, L, dk, dv, dtype, layout="bhld", states=True, seed=0, mu=1.0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen)
    heads = lambda h, *d: (B, h, L, *d) if layout == "bhld" else (B, L, h, *d)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    t = {"q": unit(n(*heads(Hk, dk))) * dk ** -0.5, "k": unit(n(*heads(Hk, dk))), "v": n(*heads(H, dv)),
         "g": torch.nn.functional.logsigmoid(n(*heads(H)) + mu) / 4, "beta": torch.sigmoid(n(*heads(H))), "d_out": n(*heads(H, dv))}
    t = {k: x.to(dtype).cuda() for k, x in t.items()}
    t["s0"], t["d_fin"] = (n(B, H, dk, dv).cuda(), 0.3 * n(B, H, dk, dv).cuda()) if states else (None, None)
    return t


def _check_delta(t, dtype, layout, direction, what):
    from paper_2405_18425_amd import binding as vb

    states = t["s0"] is not None
    args = (t["q"], t["k"], t["v"], t["g"], t["beta"])
    got = vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=states, layout=layout, direction=direction)
    out, fin = got if states else (got, None)
    want, want_fin = ref.delta_fwd(*args, t["s0"], layout, direction)
    _close(out, want, dtype, f"{what} out")
    if states:
        _close(fin, want_fin, F32, f"{what} final state")
    grads = vb.gated_delta_bwd(*args, t["d_out"], initial_state=t["s0"], d_final_state=t["d_fin"], layout=layout, direction=direction)
    wants = ref.delta_bwd(*args, t["d_out"], t["s0"], t["d_fin"], layout, direction)
    assert len(grads) == (6 if states else 5)
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "d_initial"), grads, wants):
        _close(a, b, F32 if name == "d_initial" else dtype, f"{what} {name}")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("dk,dv", ((16, 16), (16, 128), (32, 64), (64, 64), (64, 128), (128, 16), (128, 128)))
@pytest.mark.parametrize("L", (1, 63, 64, 65, 130))
def test_delta_shapes(dtype, dk, dv, L):
    layout, direction = ("bhld", "forward") if L % 2 else ("blhd", "backward")
    print(f"delta {dtype} {dk} {dv} {L}", flush=True)
    t = _delta(2, 4, 2, L, dk, dv, dtype, layout, states=L != 64, seed=L + dk)
    _check_delta(t, dtype, layout, direction, f"L={L}")


@pytest.mark.parametrize("layout", ("bhld", "blhd"))
@pytest.mark.parametrize("direction", ("forward", "backward"))
@pytest.mark.parametrize("H,Hk", ((1, 1), (3, 3), (6, 2), (4, 1)))
def test_delta_layouts_and_shared_heads(layout, direction, H, Hk):
    t = _delta(3, H, Hk, 100, 64, 64, BF16, layout, seed=H)
    _check_delta(t, BF16, layout, direction, f"{layout} {direction} {H}/{Hk}")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("kind", ("closed", "some closed", "strong", "no decay", "beta 0", "some beta 0", "beta 2", "same key", "zero keys",
                                  "padded"))
def test_delta_special_inputs(dtype, kind):
    L = 150
    t = _delta(2, 2, 2, L, 64, 64, dtype, seed=3)
    if kind == "closed":
        t["g"].fill_(-float("inf"))
    elif kind == "some closed":
        t["g"][:, :, ::7] = -float("inf")
        t["g"][:, 1, 70:75] = -3e4
    elif kind == "strong":
        t["g"][:, :, ::2] = -30.0
    elif kind == "no decay":
        t["g"].zero_()
    elif kind == "beta 0":
        t["beta"].zero_()
    elif kind == "some beta 0":
        t["beta"][:, :, ::3] = 0
    elif kind == "beta 2":
        t["beta"].fill_(2.0)
        t["g"].fill_(-0.25)
    elif kind == "same key":
        t["k"][:] = t["k"][:, :, :1]
        t["beta"].fill_(1.0)
    elif kind == "zero keys":
        t["k"].zero_()
    elif kind == "padded":
        t["g"][:, :, 60:] = 0
        t["beta"][:, :, 60:] = 0
    _check_delta(t, dtype, "bhld", "forward", kind)
    if kind == "padded":  # the state is what it was before the padding, bit for bit
        from paper_2405_18425_amd import binding as vb

        args = [t[n] for n in ("q", "k", "v", "g", "beta")]
        _, whole = vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=True)
        _, part = vb.gated_delta_fwd(*(x[:, :, :60].contiguous() for x in args), initial_state=t["s0"], return_final_state=True)
        assert torch.equal(whole, part)


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,H,Hk,L", ((1, 4, 4, 700), (2, 2, 1, 129), (5, 8, 4, 330)))
def test_delta_wide_heads_few_and_many(dtype, B, H, Hk, L):
    """128 channels, 32 to 320 workgroups of 16 columns: a chain is two waves' or one wave's"""
    print(f"delta {dtype} {B} {H} {Hk} {L}", flush=True)
    t = _delta(B, H, Hk, L, 128, 128, dtype, states=B != 2, seed=L)
    _check_delta(t, dtype, "bhld", "forward" if B == 1 else "backward", f"{B} x {H} heads of {L}")


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_delta_nan_gate_reaches_its_head_only(dtype):
    from paper_2405_18425_amd import binding as vb

    t = _delta(2, 3, 3, 200, 64, 64, dtype)
    args = [t[x] for x in ("q", "k", "v", "g", "beta")]
    clean, fin = vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=True)
    t["g"][1, 1, 70] = float("nan")
    out, nan_fin = vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=True)
    others = [(b, h) for b in range(2) for h in range(3) if (b, h) != (1, 1)]
    for b, h in others:
        assert torch.equal(out[b, h], clean[b, h]) and torch.equal(nan_fin[b, h], fin[b, h])
    assert torch.equal(out[1, 1, :64], clean[1, 1, :64])
    assert torch.isnan(out[1, 1, 70:]).all() and torch.isnan(nan_fin[1, 1]).all()
    grads = vb.gated_delta_bwd(*args, t["d_out"], initial_state=t["s0"])
    for g in grads[:5]:
        assert all(torch.isfinite(g[b, h]).all() for b, h in others)
    assert torch.isnan(grads[0][1, 1]).any()


def test_delta_continues_from_a_state_in_place():
    from paper_2405_18425_amd import binding as vb

    t = _delta(2, 4, 2, 200, 64, 64, BF16, seed=9)
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    out, fin = vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=True)
    state, parts = t["s0"].clone(), []
    for a, b in ((0, 64), (64, 67), (67, 200)):
        o, same = vb.gated_delta_fwd(*(x[:, :, a:b].contiguous() for x in args), initial_state=state, final_state=state)
        assert same is state
        parts.append(o)
    want, want_fin = ref.delta_fwd(*args, t["s0"])
    _close(torch.cat(parts, 2), want, BF16, "in parts")
    _close(state, want_fin, F32, "state")
    _close(fin, want_fin, F32, "whole")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("dk", (16, 32, 64, 128))
@pytest.mark.parametrize("dv", (16, 32, 64, 128))
def test_step_shapes_and_slots(dtype, dk, dv):
    from paper_2405_18425_amd import binding as vb

    B, H, Hk, pool = 6, 4, 2, 9
    t = _delta(B, H, Hk, 1, dk, dv, dtype, "blhd", states=False, seed=dk + dv)
    q, k, v, g, beta = (t[n][:, 0].contiguous() for n in ("q", "k", "v", "g", "beta"))
    gen = torch.Generator().manual_seed(1)
    state = torch.randn(pool, H, dk, dv, generator=gen).cuda()
    slots = torch.tensor([7, -1, 0, pool, 3, -(2 ** 31)], dtype=torch.int32).cuda()
    before = state.clone()
    out = vb.gated_delta_step(q, k, v, g, beta, state, slots=slots)
    torch.cuda.synchronize()
    live = [0, 2, 4]
    want, fin = ref.delta_fwd(*(t[n][live] for n in ("q", "k", "v", "g", "beta")), before[slots[live].long()], "blhd")
    _close(out[live], want[:, 0], dtype, "out")
    _close(state[slots[live].long()], fin, F32, "state")
    assert torch.equal(out[[1, 3, 5]], torch.zeros_like(out[[1, 3, 5]]))  # padded rows
    others = [i for i in range(pool) if i not in (7, 0, 3)]
    assert torch.equal(state[others], before[others])
    state2 = before.clone()
    out2 = vb.gated_delta_step(q, k, v, g, beta, state2)  # sequence b has state b
    want, fin = ref.delta_fwd(*(t[n] for n in ("q", "k", "v", "g", "beta")), before[:B], "blhd")
    _close(out2, want[:, 0], dtype, "out without slots")
    _close(state2[:B], fin, F32, "state without slots")
    assert torch.equal(state2[B:], before[B:])


def test_prefill_steps_and_norm_together():
    """A server's run: a prompt chunkwise, then tokens one at a time from the state it left, each output normed a group a head."""
    from paper_2405_18425_amd import binding as vb

    B, H, Hk, L, d, steps = 3, 4, 2, 77, 64, 5
    t = _delta(B, H, Hk, L + steps, d, d, BF16, "blhd", seed=21)
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    w, b = torch.linspace(0.5, 1.5, H * d).to(BF16).cuda(), torch.linspace(-0.3, 0.3, H * d).to(BF16).cuda()
    out, state = vb.gated_delta_fwd(*(x[:, :L].contiguous() for x in args), initial_state=t["s0"], return_final_state=True, layout="blhd")
    outs = [out]
    for i in range(L, L + steps):
        outs.append(vb.gated_delta_step(*(x[:, i].contiguous() for x in args), state)[:, None])
    mixed = torch.cat(outs, 1).reshape(B, L + steps, H * d)
    want, want_fin = ref.delta_fwd(*args, t["s0"], "blhd")
    _close(mixed.view(B, L + steps, H, d), want, BF16, "mixer")
    _close(state, want_fin, F32, "state")
    y, stats = vb.group_norm_act_fwd(mixed, H, w, b)
    want_y, want_stats = ref.norm_fwd(mixed, H, w, b)
    _close(y, want_y, BF16, "norm")
    _close(stats, want_stats, F32, "stats")
    # and back: the norm's gradient into the mixer's, on the prompt
    dy = torch.ones_like(y[:, :L].contiguous())
    ys, st = vb.group_norm_act_fwd(out.reshape(B, L, H * d), H, w, b)
    dx, dw, db = vb.group_norm_act_bwd(out.reshape(B, L, H * d), dy, st, H, w, b)
    want_dx, want_dw, want_db = ref.norm_bwd(out.reshape(B, L, H * d), dy, H, w, b)
    for name, a, e in (("dx", dx, want_dx), ("dw", dw, want_dw), ("db", db, want_db)):
        _close(a, e, BF16, name)
    prompt = [x[:, :L].contiguous() for x in args]
    grads = vb.gated_delta_bwd(*prompt, dx.view(B, L, H, d), initial_state=t["s0"], layout="blhd")
    wants = ref.delta_bwd(*prompt, dx.view(B, L, H, d), t["s0"], None, "blhd")
    for name, a, e in zip(("dq", "dk", "dv", "dg", "dbeta", "d_initial"), grads, wants):
        _close(a, e, F32 if name == "d_initial" else BF16, name)


def _guarded(shape, dtype, fill):
    """A tensor inside a larger one whose ends hold `fill`: (tensor, check)."""
    n = 1
    for s in shape:
        n *= s
    pad = 4096
    whole = torch.full((n + 2 * pad,), fill, dtype=dtype, device="cuda")

    def check():
        assert (whole[:pad] == fill).all() and (whole[pad + n:] == fill).all()

    return whole[pad:pad + n].view(shape), check


@pytest.mark.parametrize("layout,direction", (("bhld", "forward"), ("blhd", "backward")))
def test_delta_writes_nothing_around_its_tensors(layout, direction):
    from paper_2405_18425_amd import binding as vb

    t = _delta(2, 6, 3, 70, 32, 64, BF16, layout, seed=4)
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    out, c1 = _guarded(t["v"].shape, BF16, 7.0)
    fin, c2 = _guarded(t["s0"].shape, F32, 7.0)
    ws, c3 = _guarded((vb.gated_delta_workspace_bytes(2, 6, 3, 70, 32, 64, vb.VIG_BF16),), torch.uint8, 77)
    vb.gated_delta_fwd(*args, initial_state=t["s0"], out=out, final_state=fin, workspace=ws, layout=layout, direction=direction)
    _close(out, ref.delta_fwd(*args, t["s0"], layout, direction)[0], BF16, "out")
    for c in (c1, c2, c3):
        c()
    ws, c4 = _guarded((int(vb.lib().gated_delta_bwd_workspace_bytes(2, 6, 3, 70, 32, 64, vb.VIG_BF16)),), torch.uint8, 77)
    first = vb.gated_delta_bwd(*args, t["d_out"], initial_state=t["s0"], workspace=ws, layout=layout, direction=direction)
    c4()
    # raw call into guarded outputs
    outs = [_guarded(x.shape, x.dtype, 7.0) for x in (*args, t["s0"])]
    ptr = lambda x: x.data_ptr()
    st = vb.lib().gated_delta_bwd(*map(ptr, args), ptr(t["s0"]), ptr(t["d_out"]), None, *(ptr(o) for o, _ in outs), 2, 6, 3, 70, 32, 64,
                                  vb.VIG_BF16, vb.LAYOUTS[layout], vb.SCANS[direction], ptr(ws), ws.numel(),
                                  torch.cuda.current_stream().cuda_stream)
    assert st == vb.VIG_OK
    torch.cuda.synchronize()
    for (o, check), same in zip(outs, first):
        check()
        assert torch.equal(o, same)


def test_delta_is_deterministic_and_ignores_old_workspaces():
    from paper_2405_18425_amd import binding as vb

    t = _delta(2, 8, 4, 190, 64, 64, BF16, seed=6)
    args = [t[n] for n in ("q", "k", "v", "g", "beta")]
    need = int(vb.lib().gated_delta_bwd_workspace_bytes(2, 8, 4, 190, 64, 64, vb.VIG_BF16))
    runs = []
    for fill in (0, 255, 127):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        runs.append(vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=True, workspace=ws)
                    + vb.gated_delta_bwd(*args, t["d_out"], initial_state=t["s0"], d_final_state=t["d_fin"], workspace=ws))
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


def test_captured_graph_replays_with_new_inputs():
    """Prefill, a step, the norm and both gradients in one graph on a side stream, replayed three times on new values."""
    from paper_2405_18425_amd import binding as vb

    B, H, L, d = 2, 4, 100, 64

    def run(t, state, slots, x):
        args = [t[n] for n in ("q", "k", "v", "g", "beta")]
        out, fin = vb.gated_delta_fwd(*args, initial_state=t["s0"], return_final_state=True, layout="blhd")
        grads = vb.gated_delta_bwd(*args, t["d_out"], initial_state=t["s0"], layout="blhd")
        step = vb.gated_delta_step(*(a[:, 0].contiguous() for a in args), state, slots=slots)
        y, stats = vb.group_norm_act_fwd(x, 4)
        dx, _, _ = vb.group_norm_act_bwd(x, y, stats, 4)
        return [out, fin, step, state, y, stats, dx, *grads]

    t = _delta(B, H, H, L, d, d, BF16, "blhd", seed=0)
    state = torch.zeros(B, H, d, d, device="cuda")
    slots = torch.tensor([1, -1], dtype=torch.int32, device="cuda")
    x = torch.zeros(2, 3000, 64, device="cuda", dtype=BF16)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        run(t, state, slots, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = run(t, state, slots, x)
    for seed in (1, 2, 3):
        new = _delta(B, H, H, L, d, d, BF16, "blhd", seed=seed)
        for n in t:
            t[n].copy_(new[n])
        gen = torch.Generator().manual_seed(seed)
        s_new, x_new = torch.randn(state.shape, generator=gen).cuda(), torch.randn(x.shape, generator=gen).to(BF16).cuda()
        state.copy_(s_new)
        x.copy_(x_new)
        graph.replay()
        torch.cuda.synchronize()
        got = [c.clone() for c in captured]
        eager = run(new, s_new, slots, x_new)
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    from paper_2405_18425_amd import binding as vb

    jobs = [_delta(2, 6, 6, 300, 64, 64, BF16, seed=s) for s in (1, 2)]
    args = [[t[n] for n in ("q", "k", "v", "g", "beta")] for t in jobs]
    alone = [(*vb.gated_delta_fwd(*a, initial_state=t["s0"], return_final_state=True), *vb.gated_delta_bwd(*a, t["d_out"])) for a, t in zip(args, jobs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    both = []
    for s, a, t in zip(streams, args, jobs):
        with torch.cuda.stream(s):
            both.append((*vb.gated_delta_fwd(*a, initial_state=t["s0"], return_final_state=True), *vb.gated_delta_bwd(*a, t["d_out"])))
    torch.cuda.synchronize()
    for x, y in zip(alone, both):
        for a, b in zip(x, y):
            assert torch.equal(a, b)


def test_delta_many_heads_and_few():
    """More slabs than the chip has places for, a number that is no multiple of eight, and a long single one."""
    for B, H, L in ((37, 9, 65), (1, 1, 1500)):
        t = _delta(B, H, H, L, 64, 64, BF16, states=False, seed=B)
        _check_delta(t, BF16, "bhld", "forward", f"{B}x{H}x{L}")


def test_delta_beyond_32_bits():
    """Token-major values of 4.3 GB: the last head's last tokens."""
    from paper_2405_18425_amd import binding as vb

    B, H, L, dk, dv = 1, 128, (1 << 17) + 70, 16, 128
    gen = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randn(B, L, 1, dk, device="cuda", dtype=BF16, generator=gen) * 0.25
    k = torch.nn.functional.normalize(torch.randn(B, L, 1, dk, device="cuda", generator=gen), dim=-1).to(BF16)
    v = torch.randn(B, L, H, dv, device="cuda", dtype=BF16, generator=gen)
    g = torch.full((B, L, H), -0.25, device="cuda", dtype=BF16)
    beta = torch.full((B, L, H), 0.5, device="cuda", dtype=BF16)
    assert v.numel() * 2 > 1 << 32
    out = vb.gated_delta_fwd(q, k, v, g, beta, layout="blhd")
    torch.cuda.synchronize()
    tail = slice(L - 330, L)  # what came before has decayed to exp(-50) of itself at the last 130
    for h in (0, H - 1):
        want, _ = ref.delta_fwd(q[:, tail], k[:, tail], v[:, tail, h:h + 1], g[:, tail, h:h + 1], beta[:, tail, h:h + 1], layout="blhd")
        _close(out[:, L - 130:, h:h + 1], want[:, -130:], BF16, f"head {h}")


# ---- group norm --------------------------------------------------------------------------------------

def _norm(B, L, C, dtype, affine=True, mean=0.0, std=1.0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen)
    x = (mean + std * n(B, L, C)).to(dtype).cuda()
    w = (1 + 0.3 * n(C)).to(dtype).cuda() if affine else None
    b = (0.3 * n(C)).to(dtype).cuda() if affine else None
    return x, w, b, n(B, L, C).to(dtype).cuda()


def _check_norm(x, w, b, d, groups, act, dtype, what):
    from paper_2405_18425_amd import binding as vb

    y, stats = vb.group_norm_act_fwd(x, groups, w, b, act=act)
    want, want_stats = ref.norm_fwd(x, groups, w, b, act=act)
    _close(y, want, dtype, f"{what} out")
    _close(stats[..., 0], want_stats[..., 0], F32, f"{what} mean")
    _close(stats[..., 1], want_stats[..., 1], F32, f"{what} rstd")
    dx, dw, db = vb.group_norm_act_bwd(x, d, stats, groups, w, b, act=act)
    wants = ref.norm_bwd(x, d, groups, w, b, act=act)
    _close(dx, wants[0], dtype, f"{what} dx")
    if w is None:
        assert dw is None and db is None
    else:
        _close(dw, wants[1], dtype, f"{what} dw")
        _close(db, wants[2], dtype, f"{what} db")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,L,C,groups", ((1, 2, 8, 1), (2, 49, 64, 8), (3, 7, 96, 96), (2, 300, 2304, 9), (1, 5000, 32, 2),
                                          (2, 1000, 4096, 4), (2, 33, 8192, 1), (5, 17, 40, 5), (2, 260, 64, 4), (70, 40, 24, 3)))
def test_norm_shapes(dtype, B, L, C, groups):
    print(f"norm {dtype} {B} {L} {C} {groups}", flush=True)
    x, w, b, d = _norm(B, L, C, dtype, affine=L % 2 == 0 or B == 1, seed=L)
    _check_norm(x, w, b, d, groups, "silu" if C % 64 == 0 else "none", dtype, f"{B}x{L}x{C}/{groups}")


@pytest.mark.parametrize("L", (40, 3000))
def test_norm_mean_far_from_zero(L):
    """Values around 1000 with a spread of 1: a variance from a difference of sums of squares would be off by a tenth."""
    x, w, b, d = _norm(2, L, 64, F32, mean=1000.0, seed=2)
    from paper_2405_18425_amd import binding as vb

    _, stats = vb.group_norm_act_fwd(x, 4, w, b)
    _, want = ref.norm_fwd(x, 4, w, b)
    _close(stats[..., 0], want[..., 0], F32, "mean")
    # a mean rounded to 2^-24 of 1000 shifts the squared distances by its square, 4e-9
    _close(stats[..., 1], want[..., 1], F32, "rstd")


@pytest.mark.parametrize("L", (40, 3000))
def test_norm_constant_input_and_single_values(L):
    from paper_2405_18425_amd import binding as vb

    x = torch.full((2, L, 64), 3.0, device="cuda")
    w, b = torch.ones(64, device="cuda"), torch.full((64,), 0.5, device="cuda")
    y, stats = vb.group_norm_act_fwd(x, 4, w, b, act="none")
    assert torch.equal(y, torch.full_like(y, 0.5))  # no spread: the bias
    assert torch.allclose(stats[..., 1], torch.full_like(stats[..., 1], (1e-5) ** -0.5))
    one = torch.randn(3, 1, 8, device="cuda")
    y, stats = vb.group_norm_act_fwd(one, 8, act="none")  # a group of a single value
    assert torch.equal(y, torch.zeros_like(y)) and torch.equal(stats[..., 0], one[:, 0])
    dx, _, _ = vb.group_norm_act_bwd(one, torch.ones_like(one), stats, 8, act="none")
    assert torch.equal(dx, torch.zeros_like(dx))


def test_norm_large_values_and_extreme_activations():
    x, w, b, d = _norm(2, 500, 64, F32, seed=3)
    w, b = w * 60, b * 60  # z in the hundreds: exp(-z) overflows on one side
    _check_norm(x, w, b, d, 4, "silu", F32, "steep")


def test_norm_takes_grids_and_writes_nothing_around():
    from paper_2405_18425_amd import binding as vb

    x, w, b, d = _norm(2, 35 * 31, 48, BF16, seed=8)
    grid = x.view(2, 35, 31, 48)
    out, c1 = _guarded(grid.shape, BF16, 7.0)
    stats, c2 = _guarded((2, 3, 2), F32, 7.0)
    ws, c3 = _guarded((int(vb.lib().group_norm_workspace_bytes(2, 35 * 31, 48, 3, vb.VIG_BF16)),), torch.uint8, 77)
    vb.group_norm_act_fwd(grid, 3, w, b, out=out, stats=stats, workspace=ws)
    _close(out.view(x.shape), ref.norm_fwd(x, 3, w, b)[0], BF16, "grid")
    for c in (c1, c2, c3):
        c()
    ws, c4 = _guarded((int(vb.lib().group_norm_bwd_workspace_bytes(2, 35 * 31, 48, 3, vb.VIG_BF16)),), torch.uint8, 77)
    got = vb.group_norm_act_bwd(grid, d.view(grid.shape), stats, 3, w, b, workspace=ws)
    again = vb.group_norm_act_bwd(grid, d.view(grid.shape), stats, 3, w, b)
    c4()
    for a, e in zip(got, again):
        assert torch.equal(a, e)

"""GPU tests of the gated delta rule with its states given, asked for and differentiated one at a time, against the 64-bit reference."""
import pytest
import torch

import delta_norm_ref as ref
from test_delta_norm_gpu import BF16, F32, _close, _delta

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "g", "beta")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("d", (32, 64, 128))
@pytest.mark.parametrize("given,asked", ((True, False), (False, True), (True, True)))
def test_forward(dtype, d, given, asked):
    from paper_2405_18425_amd import binding as vb

    t = _delta(2, 4, 2, 75, d, d, dtype, seed=d)
    args = [t[n] for n in NAMES]
    initial = t["s0"] if given else None
    got = vb.gated_delta_fwd(*args, initial_state=initial, return_final_state=asked, direction="backward")
    want, want_fin = ref.delta_fwd(*args, initial, direction="backward")
    out, fin = got if asked else (got, None)
    _close(out, want, dtype, "out")
    if asked:
        _close(fin, want_fin, F32, "state")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("d", (32, 64, 128))
@pytest.mark.parametrize("given,later", ((True, False), (False, True)))
def test_gradient(dtype, d, given, later):
    from paper_2405_18425_amd import binding as vb

    t = _delta(2, 4, 2, 75, d, d, dtype, seed=d)
    args = [t[n] for n in NAMES]
    initial, d_final = t["s0"] if given else None, t["d_fin"] if later else None
    got = vb.gated_delta_bwd(*args, t["d_out"], initial_state=initial, d_final_state=d_final, layout="bhld", direction="backward")
    want = ref.delta_bwd(*args, t["d_out"], initial, d_final, direction="backward")
    assert len(got) == (6 if given else 5)
    for name, a, e in zip(("dq", "dk", "dv", "dg", "dbeta", "d_initial"), got, want):
        _close(a, e, F32 if name == "d_initial" else dtype, name)


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_gradient_of_a_state_that_is_zero(dtype):
    """Through the C entry point d_initial_state may be asked for without an initial state."""
    from paper_2405_18425_amd import binding as vb

    B, H, L, d = 2, 3, 100, 64
    t = _delta(B, H, H, L, d, d, dtype, seed=5)
    args = [t[n] for n in NAMES]
    code = vb.VIG_BF16 if dtype == BF16 else vb.VIG_F32
    grads = [torch.full_like(x, 7.0) for x in (*args, t["s0"])]
    ws = torch.empty(int(vb.lib().gated_delta_bwd_workspace_bytes(B, H, H, L, d, d, code)), dtype=torch.uint8, device="cuda")
    ptr = lambda x: x.data_ptr()
    assert vb.lib().gated_delta_bwd(*map(ptr, args), None, ptr(t["d_out"]), ptr(t["d_fin"]), *map(ptr, grads), B, H, H, L, d, d, code, 0, 0, ptr(ws),
                                    ws.numel(), torch.cuda.current_stream().cuda_stream) == vb.VIG_OK
    torch.cuda.synchronize()
    want = ref.delta_bwd(*args, t["d_out"], None, t["d_fin"])
    for name, a, e in zip(("dq", "dk", "dv", "dg", "dbeta", "d_initial"), grads, want):
        _close(a, e, F32 if name == "d_initial" else dtype, name)

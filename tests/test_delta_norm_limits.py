"""How large the gated delta rule's calls may be (CPU only: every call returns before a launch)."""
import pytest

from paper_2405_18425_amd import binding as vb

PTR = 0x10000  # a non-NULL, 16-byte aligned dummy: validation must reject before dereferencing


def _fwd(*sizes):
    return vb.lib().gated_delta_fwd(*[PTR] * 8, *sizes, 0, 0, PTR, 1, None)


def _bwd(*sizes):
    return vb.lib().gated_delta_bwd(*[PTR] * 14, *sizes, 0, 0, PTR, 1, None)


# The largest B, H, Hk, L, dk, dv that a launch of fewer than 2^32 work-items holds, and the next ones: 256 work-items a chunk of a head; 128 a chain of 16 columns
# (two of them in the gradient, heads in eights)
@pytest.mark.parametrize("call,query,fits,beyond", (
    (_fwd, "gated_delta_workspace_bytes", ((1 << 24) - 1, 1, 1, 1, 16, 16), (1 << 24, 1, 1, 1, 16, 16)),
    (_fwd, "gated_delta_workspace_bytes", ((1 << 22) - 8, 1, 1, 1, 16, 128), ((1 << 22) - 7, 1, 1, 1, 16, 128)),
    (_fwd, "gated_delta_workspace_bytes", ((1 << 20) - 2, 4, 2, 9, 128, 128), ((1 << 20) - 1, 4, 2, 9, 128, 128)),
    (_bwd, "gated_delta_bwd_workspace_bytes", ((1 << 21) - 8, 1, 1, 1, 16, 128), ((1 << 21) - 7, 1, 1, 1, 16, 128)),
    (_bwd, "gated_delta_bwd_workspace_bytes", ((1 << 24) - 8, 1, 1, 1, 64, 16), ((1 << 24) - 7, 1, 1, 1, 64, 16))))
def test_sequences_beyond_a_launch_are_refused(call, query, fits, beyond):
    for code in (vb.VIG_BF16, vb.VIG_F32):
        assert getattr(vb.lib(), query)(*fits, code) > 0
        assert call(*fits, code) == vb.VIG_ERR_WORKSPACE  # (of one byte: the sizes have passed)
        assert getattr(vb.lib(), query)(*beyond, code) == 0
        assert call(*beyond, code) == vb.VIG_ERR_SHAPE


def test_a_step_has_no_such_limit():
    """Its workgroups are shared out over launches."""
    call = lambda B: vb.lib().gated_delta_step(*[PTR] * 7, PTR + 8, B, 1, 1, 16, 16, 1 << 27, vb.VIG_BF16, None)
    assert call(1 << 27) == vb.VIG_ERR_ALIGN  # (of the output: the sizes have passed)
    assert call(1 << 28) == vb.VIG_ERR_SHAPE

"""GPU tests of the channels-last group norm's statistics: values that are not finite."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")


# 40 tokens: a group in one workgroup's registers, one launch; 3000: partial sums of strips, two launches
@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("L", (40, 3000))
@pytest.mark.parametrize("bad", (INF, -INF, float("nan")))
@pytest.mark.parametrize("at", ((0, 16), (17, 20)))
def test_values_that_are_not_finite_reach_their_group_only(dtype, L, bad, at):
    from paper_2405_18425_amd import binding as vb

    gen = torch.Generator().manual_seed(L)
    x, d = (torch.randn(3, L, 64, generator=gen).to(dtype).cuda() for _ in range(2))
    w, b = (torch.randn(64, generator=gen).to(dtype).cuda() for _ in range(2))
    clean, clean_stats = vb.group_norm_act_fwd(x, 4, w, b, act="none")
    clean_grads = vb.group_norm_act_bwd(x, d, clean_stats, 4, w, b, act="none")
    x[1, at[0], at[1]] = bad  # channels 16 to 31 are group 1
    y, stats = vb.group_norm_act_fwd(x, 4, w, b, act="none")
    assert torch.isnan(stats[1, 1, 1]) and not torch.isfinite(stats[1, 1, 0])
    assert torch.isnan(y[1, :, 16:32]).all()
    dx, dw, db = vb.group_norm_act_bwd(x, d, stats, 4, w, b, act="none")
    assert torch.isnan(dx[1, :, 16:32]).all() and torch.isnan(dw[16:32]).all()
    others = torch.ones(3, 64, dtype=torch.bool, device="cuda")
    others[1, 16:32] = False
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[16:32] = False
    assert torch.equal(y.transpose(1, 2)[others], clean.transpose(1, 2)[others])
    assert torch.equal(stats.flatten(0, 1)[[i for i in range(12) if i != 5]], clean_stats.flatten(0, 1)[[i for i in range(12) if i != 5]])
    assert torch.equal(dx.transpose(1, 2)[others], clean_grads[0].transpose(1, 2)[others])
    assert torch.equal(dw[rest], clean_grads[1][rest]) and torch.equal(db, clean_grads[2])

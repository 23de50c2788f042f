"""Rows with a NaN leave the positions that they do not see alone: the step's own positions behind them."""
import pytest
import torch

from test_gpu_kv_weights_not_finite import EVERY, run, setup

pytestmark = pytest.mark.gpu


@EVERY
@pytest.mark.parametrize("slot", [0, 2])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_row_in_the_middle_of_a_step(path, slot, bad):
    s = setup(path, 4, [200, 193, 4], 4)
    clean = run(s, 0.5)
    s["q"][:, slot, 0, 5] = bad
    w = run(s, 0.5)
    for b, n in enumerate((200, 193, 4)):
        seen = n - 4 + slot + 1                              # positions that the row sees
        at = torch.arange(seen, device="cuda")
        keys = s["k"][s["table"][b, at // s["k"].shape[2]].long(), 0, at % s["k"].shape[2], 5].float()
        if bad == float("inf") and (keys < 0).all():         # (few positions, all keys negative: every score of the row is -inf, it adds nothing)
            assert seen <= 3 and torch.isfinite(w[b, 0, :n]).all()
        else:
            assert torch.isnan(w[b, 0, :seen]).all()
        assert torch.equal(w[b, 0, seen:], clean[b, 0, seen:]), (b, w[b, 0, seen:n], clean[b, 0, seen:n])
    assert torch.equal(w[:, 1:], clean[:, 1:])
    # the same slots by an accepted path
    s["alen"] = torch.full((3,), 3, dtype=torch.int32, device="cuda")
    s["path"] = torch.arange(4, dtype=torch.int32, device="cuda").repeat(3, 1).contiguous()
    assert torch.equal(torch.nan_to_num(run(s, 0.5), nan=-1.0), torch.nan_to_num(w, nan=-1.0))


@EVERY
def test_rows_without_weight_and_rows_with_a_nan_together(path):
    """A row whose scores are all -inf adds nothing; a row with a NaN shows only in what it sees."""
    s = setup(path, 3, [100, 70], 5)
    s["k"].abs_()
    s["q"].abs_()
    s["q"][0, 0, 1] = 0.0
    s["q"][0, 0, 1, 3] = -float("inf")
    before = run(s)
    assert torch.isfinite(before).all()
    s["q"][0, 1, 0, 3] = float("nan")                        # sees positions up to 98
    w = run(s)
    assert torch.isnan(w[0, 0, :99]).all() and torch.equal(w[0, 0, 99:], before[0, 0, 99:])
    assert torch.equal(w[0, 1:], before[0, 1:]) and torch.equal(w[1], before[1])

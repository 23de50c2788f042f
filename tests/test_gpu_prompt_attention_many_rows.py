"""seer_prompt_attention where it takes 256 query rows a workgroup: heads of 128, 131 072 query rows or more, 8192 or more for a request on
average.  Padding counts among them, so short requests reach this form too.  Tolerance: as in the test of the call's other forms."""
import pytest
import torch

from test_gpu_prompt_attention import call, check, compare, make, plain, spoil

pytestmark = pytest.mark.gpu


def padded(new, Hq, Hkv):
    """Padding that is just enough."""
    wanted = max(-(-131072 // Hq), -(-8192 * len(new) // (Hq // Hkv)))
    return max(0, wanted - sum(new))


@pytest.mark.parametrize("heads", [(8, 1, 128, 128, 16), (8, 2, 128, 128, 48), (128, 1, 128, 128, 64), (20, 4, 128, 128, 16)])
def test_lengths_around_every_border(heads):
    new = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 16, 15, 255, 256, 257, 3, 0]
    past = [5, 0, 1, 0, 0, 0, 1, 64, 31, 0, 128, 1, 0, 1000, 15, 17, 333, 700, 0, 0]
    check(31, new, past, *heads, pad=padded(new, *heads[:2]))


@pytest.mark.parametrize("heads,new,past", [((64, 8, 128, 128, 16), [1500, 610], [0, 700]), ((16, 16, 128, 128, 32), [8200], [100]), ((8, 1, 128, 128, 16), [16000, 500, 1], [0, 20000, 3])])
def test_long_ones(heads, new, past):
    check(32, new, past, *heads, rows=40, pad=padded(new, *heads[:2]))


def test_many_requests():
    new = [1 if b % 3 else 0 for b in range(700)]
    check(33, new, [(b * 37) % 900 for b in range(700)], 64, 1, 128, 128, 16, rows=4, pad=padded(new, 64, 1))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_a_token_does_not_see_does_not_reach_it(value):
    heads, new, past = (8, 1, 128, 128, 16), [200, 70, 33], [0, 300, 0]
    c = make(34, new, past, *heads, pad=padded(new, 8, 1))
    good, _ = call(c)
    for b, j in enumerate((100, 340, 20)):
        spoil(c["k"], b, j, c, value)
        spoil(c["v"], b, j, c, value, slice(0, 2))
    out, status = call(c)
    assert status == 0
    for first, before in ((0, 100), (200, 240), (270, 290)):
        assert torch.equal(out[first:before], good[first:before])


def test_values_that_are_not_finite_stay_in_their_component():
    new = [150, 40]
    c = make(35, new, [0, 200], 8, 2, 128, 128, 16, std=0.5, pad=padded(new, 8, 2))
    want = plain(c)
    for b, j in ((0, 70), (1, 215)):
        spoil(c["v"], b, j, c, float("inf"), 5)
    out, _ = call(c)
    keep = torch.tensor([d for d in range(128) if d != 5], device="cuda")
    compare(out[..., keep], [(t, hq, ref[:, keep], weight[:, keep]) for t, hq, ref, weight in want])
    assert torch.isinf(out[70:150, :, 5].float()).all() and torch.isinf(out[165:190, :, 5].float()).all()
    assert torch.isfinite(out[:70, :, 5].float()).all() and torch.isfinite(out[150:165, :, 5].float()).all()


def test_wrong_numbers_are_reported_and_kept_in_bounds():
    new = [20, 30, 40, 50]
    c = make(36, new, [10, 0, 5, 9], 8, 2, 128, 128, 16, pad=padded(new, 8, 2))
    want = plain(c)
    bad = dict(c, ctx=c["ctx"].clone(), table=c["table"].clone())
    bad["ctx"][1], bad["ctx"][2] = 29, c["table"].shape[1] * 16 + 1
    bad["table"][0, 0] = -5
    out, status = call(bad)
    assert status == 3 and (out[20:90] == 0).all()
    compare(out, [w for w in want if int(w[0][0]) == 90])
    assert (out[140:] == 7.0).all()


def test_captured_and_replayed():
    from paper_2511_14617_amd import binding as b
    new = [300, 90]
    c = make(37, new, [700, 0], 8, 1, 128, 128, 16, pad=padded(new, 8, 1))
    dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    run = lambda out: b.seer_prompt_attention(dev["q"], dev["k"], dev["v"], dev["table"], dev["ctx"], dev["first"], c["scale"], out=out)
    want, out = run(None), torch.zeros(c["q"].shape[0], 8, 128, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:390], want[:390])

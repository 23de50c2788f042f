"""Forms of the log probability calls: several slots per request without a path, and outputs that are not asked for."""
import pytest
import torch

from test_gpu_token_logprobs import check, make, run_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T,V,pad", [(3, 5, 1003, 0), (2, 7, 4099, 13), (70, 33, 130, 6)])
def test_all_slots_without_a_path(B, T, V, pad, dtype):
    """[B,T,V] with T > 1: every slot is its own row, forward, gradient and in place."""
    x, tok = make(B, V, dtype, B + V, pad=pad, T=T)
    tok[0, T - 1], tok[B - 1, 0] = -1, V
    out = check(x, tok, 0.9, 3)
    flat = check(x.reshape(B * T, V), tok.reshape(-1), 0.9, 3)
    assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(out, flat))
    want = run_grad(x, tok, 0.9)
    same = x.clone().contiguous()
    assert torch.equal(run_grad(same, tok, 0.9, out=same), want)
    room = torch.full((B, T, V + 11), 5.0, device="cuda", dtype=dtype)
    run_grad(x, tok, 0.9, out=room[:, :, :V])
    assert torch.equal(room[:, :, :V], want) and (room[:, :, V:] == 5).all()


def test_outputs_that_are_not_asked_for():
    from paper_2511_14617_amd import binding
    x, tok = make(9, 5003, torch.float32, 7)
    want = binding.seer_token_logprobs(x, tok, top_n=2)
    empty = lambda *shape: torch.full((9, *shape), -7.0, device="cuda")
    for keep in ((0,), (0, 1), (0, 2)):
        out = tuple(empty() if i in keep else None for i in range(3)) + (empty(2), torch.zeros((9, 2), dtype=torch.int32, device="cuda"))
        assert binding.seer_token_logprobs(x, tok, top_n=2, out=out) is out
        assert all(a is None or torch.equal(a, b) for a, b in zip(out, want))
    only = (empty(), None, None)
    binding.seer_token_logprobs(x, tok, out=only)
    assert torch.equal(only[0], binding.seer_token_logprobs(x, tok)[0])     # (chunks have other lengths where alternatives are asked for)
    for out in ((None, empty(), empty()), (empty(), empty()[:3], None)):
        with pytest.raises(ValueError):
            binding.seer_token_logprobs(x, tok, out=out)
    with pytest.raises(ValueError):
        binding.seer_token_logprobs(x, tok, top_n=2, out=(empty(), None, None, None, None))

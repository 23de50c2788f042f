"""Rows with a NaN or +inf among their logits: log probability, entropy, logsumexp and the alternatives' log probabilities are NaN whatever the token's logit is,
and the other rows do not notice."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("V", [5, 300, 20000])
def test_a_masked_token_in_a_broken_row(V, bad, dtype):
    from paper_2511_14617_amd import binding
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((7, V), device="cuda", generator=g).to(dtype)
    tok = torch.zeros(7, dtype=torch.int32, device="cuda")
    x[:, 0] = -float("inf")                                  # every token is masked
    x[1, 3] = bad
    x[2, 1:] = -float("inf")                                 # one finite logit at most beside the bad one
    x[2, V - 1] = bad
    x[4, :] = -float("inf")                                  # nothing left: no NaN
    x[5, :] = -float("inf")
    x[5, 2] = bad                                            # the bad one alone
    x[6, :] = bad
    n = min(V, 9)
    lp, h, lse, alt, at = binding.seer_token_logprobs(x, tok, top_n=n)
    for r in (1, 2, 5, 6):
        assert torch.isnan(lp[r]) and torch.isnan(h[r]) and torch.isnan(lse[r]), r
        assert torch.isnan(alt[r]).all(), (r, alt[r])
    assert (at >= 0).all() and (at < V).all()
    assert (lp[[0, 3, 4]] == -float("inf")).all() and torch.isfinite(h[[0, 3, 4]]).all() and torch.isfinite(lse[[0, 3]]).all()
    assert lse[4] == -float("inf") and (alt[4] == -float("inf")).all() and at[4].tolist() == list(range(n))
    ok = [0, 3, 4]
    want = binding.seer_token_logprobs(x[ok].contiguous(), tok[ok].contiguous(), top_n=n)
    assert all(torch.equal(a[ok], b) for a, b in zip((lp, h, lse, alt, at), want))

"""Log probabilities where finite mask values fill whole ranges of a vocabulary, and where all logits are far from zero, against the definitions in 64 bits.

Tolerances (u = 2^-24, half a step of fp32), as in test_gpu_token_logprobs.py: ln l and the entropy's sums are good to 128 u.  A log probability (x - m) / tau - ln l
takes three roundings of its first part and one of the result: 4 u of the larger of the two, element by element.  A row's logsumexp takes 4 u of itself."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def reference(x, tau):
    """x [N,V] on the device: z, row maximum, log probabilities, probabilities, entropy, logsumexp in 64 bits."""
    z = x.double() / float(np.float32(tau))
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    l = e.sum(1, keepdim=True)
    logp, p = z - m - torch.log(l), e / l
    h = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    return z, m, logp, p, h, (m + torch.log(l))[:, 0]


def rows_with_masks(V, dtype, mask, rows, seed):
    """Normal logits in a stretch of some rows, everywhere in others, nowhere in the rest, and a token of each kind."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((rows, V), device="cuda", generator=g) * 2).to(dtype)
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    live = [(V // 2, V // 2 + 100), (0, 0), (0, 5), (V - 3, V), (0, V), (V // 3, V // 3 + 1), (0, V // 2)]
    for r in range(rows):
        lo, hi = live[r % len(live)]
        x[r, :lo], x[r, hi:] = mask, mask
        tok[r] = lo if r % 2 == 0 or hi == 0 else (hi + 7) % V       # (every second one is masked, as far as anything is)
    return x, tok


def check_forward(x, tok, tau, top_n):
    from paper_2511_14617_amd import binding
    lp, h, lse, alt, alt_token = binding.seer_token_logprobs(x, tok, temperature=tau, top_n=top_n)
    z, m, logp, p, h64, lse64 = reference(x, tau)
    off = lambda z_, logp_: 128 * U + 4 * U * torch.maximum((z_ - m).abs(), logp_.abs())
    pick = tok.long()[:, None]
    want, tol = logp.gather(1, pick)[:, 0], off(z.gather(1, pick), logp.gather(1, pick))[:, 0]
    assert ((lp.double() - want).abs() <= tol).all(), (lp, want)
    assert ((h.double() - h64).abs() <= 128 * U * (2 + h64)).all(), (h, h64)
    assert ((lse.double() - lse64).abs() <= 128 * U + 4 * U * lse64.abs()).all(), (lse, lse64)
    order = torch.sort(x.double(), dim=1, descending=True, stable=True)[1][:, :top_n]
    assert torch.equal(alt_token.long(), order)
    assert ((alt.double() - logp.gather(1, order)).abs() <= off(z.gather(1, order), logp.gather(1, order))).all()
    return lp, h, lse


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tau", [0.6, 1.0, 2.0])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -2e9, -1e10, -1e12, -1e20, -1e29, -1e30, -1e38])
def test_mask_values_in_whole_chunks(mask, tau, dtype):
    check_forward(*rows_with_masks(33000, dtype, mask, 14, 1), tau, 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e20])
def test_mask_values_in_whole_long_chunks(mask, dtype):
    check_forward(*rows_with_masks(33000, dtype, mask, 700, 2), 0.8, 3)


@pytest.mark.parametrize("base", [3e6, -3e6, 1e9, -1e9, 1e15, -1e15])
def test_all_logits_far_from_zero(base):
    """Rows of a few values, steps of the type apart, around a base whose quotient by the temperature is beyond 2^22."""
    step = abs(base) * 2.0 ** -22
    g = torch.Generator(device="cuda").manual_seed(3)
    x = (base + step * torch.randint(-3, 4, (6, 9001), device="cuda", generator=g, dtype=torch.float64)).float()
    for tau in (1.0, step, 0.7 * step):
        check_forward(x, torch.arange(6, device="cuda", dtype=torch.int32), tau, 4)

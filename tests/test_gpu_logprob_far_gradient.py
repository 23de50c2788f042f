"""The gradient of rows whose logits are far from zero (masked throughout, or divided by a small temperature): fp32 holds their logsumexp to
steps that are no longer small, so the kernel takes the row's own maximum and sum.  Against the formula in 64 bits.

Tolerances (u = 2^-24): p = exp(z - lse) takes the roundings of z, of lse (2 u of it) and of their difference into its exponent where |lse| is below 4096, and those of
(x - m) / tau (3 u) and of its difference to ln l beyond; the exponent's product with log2 e, the forward call's 128 u for ln l (twice: logsumexp and entropy) and the element's own
products are below 300 u more.  The result is rounded to the logits' type once."""
import pytest
import torch

from test_gpu_logprob_masked_ranges import U, reference, rows_with_masks

pytestmark = pytest.mark.gpu
FAR = 4096.0


def check_gradient(x, tok, tau, seed=0, in_place=False, entropy=True):
    from paper_2511_14617_amd import binding
    g = torch.Generator(device="cuda").manual_seed(seed)
    g_lp = torch.randn(len(x), device="cuda", generator=g)
    g_h = torch.randn(len(x), device="cuda", generator=g) if entropy else torch.zeros(len(x), device="cuda")
    _, h, lse, _, _ = binding.seer_token_logprobs(x, tok, temperature=tau)
    z, m, logp, p, h64, lse64 = reference(x, tau)
    hot = torch.zeros_like(z)
    hot.scatter_(1, tok.clamp(min=0).long()[:, None], (tok >= 0).double()[:, None])
    a, b = g_lp.double()[:, None], g_h.double()[:, None]
    logp = torch.where(p > 0, logp, torch.zeros_like(logp))
    live = (tok >= 0)[:, None]
    want = torch.where(live, (a * (hot - p) - b * p * (logp + h64[:, None])) / tau, torch.zeros_like(z))
    far = lse64.abs()[:, None] >= FAR * 1.001
    exponent = torch.where(far, 3 * (z - m).abs(), z.abs() + 2 * lse64.abs()[:, None]) + 4 * logp.abs() + 300
    size = (p * (a.abs() + b.abs() * (logp.abs() + h64[:, None] + 1)) + hot * a.abs()) / tau
    to = x.clone() if in_place else None
    got = binding.seer_token_logprobs_grad(to if in_place else x, tok, lse, g_lp, entropy=h if entropy else None, grad_entropy=g_h if entropy else None,
                                           temperature=tau, out=to)
    half = 2.0 ** -8 if x.dtype == torch.bfloat16 else U
    lost = 2.0 ** -126 * (a.abs() + b.abs() * (100 + h64[:, None])) / tau                   # (a p below the normal numbers may be 0)
    token = 2 * U * hot * a.abs() / tau                      # (1 / tau and its product with the incoming gradient are rounded, u each: also where p is 0)
    bound = torch.where(live & (p > 0), size * exponent * U + lost, torch.zeros_like(z)) + 1.01 * (half * want.abs() + token) + 1e-37
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (err <= bound).all(), (float((err - bound).max()), (err > bound).nonzero()[:4])
    return got


DT = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


@DT
@pytest.mark.parametrize("tau", [0.6, 1.0, 2.0])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e20, -1e30, -1e38])
def test_rows_with_masks_and_rows_of_masks(mask, tau, dtype):
    x, tok = rows_with_masks(33000, dtype, mask, 14, 4)
    tok[8] = -1                                              # (a row of masks without a token)
    got = check_gradient(x, tok, tau)
    assert (got[8] == 0).all()
    assert torch.equal(check_gradient(x, tok, tau, in_place=True), got)
    check_gradient(x, tok, tau, entropy=False)


@DT
def test_rows_of_masks_among_many(dtype):
    check_gradient(*rows_with_masks(33000, dtype, -1e9, 700, 5), 1.0, in_place=True)


@DT
@pytest.mark.parametrize("V", [1, 7, 255, 4096, 5003])
def test_the_type_s_lowest_value_everywhere(V, dtype):
    """Also where the quotient by the temperature leaves the floats."""
    x = torch.full((4, V), torch.finfo(dtype).min, device="cuda", dtype=dtype)
    x[1, V // 2:] = torch.finfo(dtype).max
    x[2] = torch.finfo(dtype).max
    for tau in (0.5, 1.0, 1.5):
        check_gradient(x, torch.zeros(4, dtype=torch.int32, device="cuda") + V - 1, tau)


@pytest.mark.parametrize("tau", [1e-3, 3e-3, 1e-5])
def test_small_temperatures(tau):
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((5, 20001), device="cuda", generator=g) * 2 + 20
    x[:, 77] = x.amax(1) + tau                               # (another one of weight)
    x[4] -= 60
    check_gradient(x, torch.tensor([77, 0, 5, 20000, 77], dtype=torch.int32, device="cuda"), tau)


def test_captured_rows_on_both_sides_of_the_limit():
    from paper_2511_14617_amd import binding
    x, tok = rows_with_masks(9000, torch.float32, -1e9, 14, 7)
    own, g, out = x.clone(), torch.ones(14, device="cuda"), torch.empty_like(x)
    ws = torch.empty(binding.seer_token_logprobs_workspace(binding.logprob_params(x)), dtype=torch.uint8, device="cuda")

    def step(logits, to):
        f = binding.seer_token_logprobs(logits, tok, workspace=ws)
        binding.seer_token_logprobs_grad(logits, tok, f[2], g, entropy=f[1], grad_entropy=g, out=to)

    eager = torch.empty_like(x)
    step(x, eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(own, out)
    for replay in range(4):
        now = torch.roll(x, replay, 0)
        step(now, eager)
        own.copy_(now)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), replay

"""The log probability, weights and eviction calls at sizes beyond the other tests': the widest vocabulary, many rows, many heads, contexts of millions of positions."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_widest_vocabulary(dtype):
    """2^24 logits: 4096 chunks, whose lists of 32 are merged one by one.  Tolerance: ln l as in test_gpu_token_logprobs.py, its sums of chunks 64 terms a lane: 192 u."""
    from paper_2511_14617_amd import binding
    V = 1 << 24
    g = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.randn((2, V), device="cuda", generator=g) * 3).to(dtype)
    x[1, : V // 2] = -float("inf")
    tok = torch.tensor([V - 1, 5], dtype=torch.int32, device="cuda")
    lp, h, lse, alt, at = binding.seer_token_logprobs(x, tok, top_n=32)
    z = x.double()
    m = z.amax(1, keepdim=True)
    l = torch.exp(z - m).sum(1, keepdim=True)
    logp = z - m - torch.log(l)
    order = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :32]
    assert torch.equal(at.long(), order)
    reach = (z.gather(1, order) - m).abs()
    assert ((alt.double() - logp.gather(1, order)).abs() <= 192 * U + 4 * U * (reach + 20)).all()
    assert abs(lp[0].double() - logp[0, V - 1]) <= 192 * U + 4 * U * (logp[0, V - 1].abs() + 20) and lp[1] == -float("inf")
    p = torch.exp(logp)
    want = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    assert ((h.double() - want).abs() <= 192 * U * (2 + want)).all()
    grad = binding.seer_token_logprobs_grad(x, tok, lse, torch.ones(2, device="cuda"))
    hot = torch.zeros_like(p).scatter_(1, tok.long()[:, None], 1.0)
    half = U if dtype == torch.float32 else 2.0 ** -8
    assert ((grad.double() - (hot - p)).abs() <= (half + 400 * U) * (hot + p) + 1e-37).all()


def test_many_short_rows():
    from test_gpu_token_logprobs import check, make, run_grad
    x, tok = make(70001, 41, torch.float32, 2)
    tok[::7] = -1
    check(x, tok, 0.9, 3)
    run_grad(x, tok, 0.9)


@pytest.mark.parametrize("T,G", [(1, 1), (3, 7)])
def test_more_heads_than_workgroups(T, G):
    """1201 KV heads: one stretch for each, with kept scores and in two sweeps; on a short table, a workgroup for each."""
    from test_gpu_kv_weights import build, check
    check(build(3, T, 1201 * G, 1201, 64, 16, [T, 40, 530], 3, T > 1), 0.5)
    check(build(3, T, 1201 * G, 1201, 64, 16, [T, 40, 100], 4, T > 1), 0.5)


def select(w, first, n, end, last, budget):
    """Where each slot's position comes from, by the documented rule, on arrays."""
    key = torch.where(torch.isnan(w[first:n - last]), torch.full((), -float("inf"), device=w.device), w[first:n - last])
    order = torch.sort(key, descending=True, stable=True)[1][:end - first] + first
    chosen = torch.sort(order)[0]
    slot = torch.arange(budget, device=w.device)
    free = torch.ones(budget, dtype=torch.bool, device=w.device)
    free[:first], free[end:] = False, False
    free[chosen[chosen < end]] = False
    slot[free] = chosen[chosen >= end]
    slot[end:] = torch.arange(n - last, n, device=w.device)
    return slot


@pytest.mark.parametrize("n,budget", [(400_000, 100_000), (400_000, 399_900), (2_300_000, 1_000_000), (2_300_000, 70_000)])
@pytest.mark.parametrize("ties", [False, True])
def test_contexts_of_millions_of_positions(n, budget, ties):
    """More keys between the sampled bounds than LDS holds, and more segments than it has ranks for."""
    from paper_2511_14617_amd import binding
    P, D, first, last = 64, 8, 37, 5000
    g = torch.Generator(device="cuda").manual_seed(5)
    lengths = [n, n // 3, n - 777]
    pages = -(-n // P)
    table = torch.randperm(3 * pages, device="cuda", generator=g).int().view(3, pages)
    k = torch.randint(-32768, 32767, (3 * pages, 1, P, D), device="cuda", generator=g, dtype=torch.int16).view(torch.bfloat16)
    w = torch.randn((3, 1, pages * P), device="cuda", generator=g).exp_()
    if ties:
        w = torch.round(w * 2) / 2                           # (a few values, most positions at three of them)
    before = k.clone()
    to = w.clone()
    ctx = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    new, kept = binding.seer_kv_evict(k, None, table, ctx, to, limit=budget, budget=budget, keep_first=first, keep_last=last, new_weights=to)
    for b, m in enumerate(lengths):
        if m <= budget:
            assert new[b] == m and (kept[b] == -1).all() and torch.equal(to[b], w[b])
            continue
        slot = select(w[b, 0], first, m, budget - last, last, budget)
        assert new[b] == budget and torch.equal(kept[b, 0].long(), slot)
        assert torch.equal(to[b, 0, :budget], w[b, 0, slot]) and torch.equal(to[b, 0, budget:], w[b, 0, budget:])
        at = torch.arange(budget, device="cuda")
        got = k.view(torch.int16)[table[b, at // P].long(), 0, at % P]
        assert torch.equal(got, before.view(torch.int16)[table[b, slot // P].long(), 0, slot % P])


def test_a_context_of_a_million_positions():
    """Tolerance as in test_gpu_kv_weights.py, with the denominators' sums: 32 pieces of up to 1100 tiles a lane, 2048 u."""
    from paper_2511_14617_amd import binding
    n, D, P = 1_000_003, 64, 128
    g = torch.Generator(device="cuda").manual_seed(6)
    for Hq, T in ((2, 2), (20, 1)):                          # (kept scores, two sweeps)
        pages = -(-n // P)
        table = torch.randperm(pages, device="cuda", generator=g).int()[None].contiguous()
        k = torch.randn((pages, 1, P, D), device="cuda", generator=g).to(torch.bfloat16)
        q = torch.randn((1, T, Hq, D), device="cuda", generator=g).to(torch.bfloat16)
        w = torch.rand((1, 1, pages * P), device="cuda", generator=g)
        ctx = torch.full((1,), n, dtype=torch.int32, device="cuda")
        got = w.clone()
        binding.seer_kv_weights(got, q, k, table, ctx, None, None, D ** -0.5, decay=0.5)
        keys = k[table[0].long(), 0].reshape(-1, D)[:n].double()
        want, tol = 0.5 * w[0, 0, :n].double(), torch.zeros(n, dtype=torch.float64, device="cuda")
        want[n - T:] = 0
        for i in range(T):
            see = n - T + i + 1
            s = (keys[:see] @ q[0, i].double().t().contiguous()) * D ** -0.5
            mag = (keys[:see].abs() @ q[0, i].double().abs().t().contiguous()).amax() * D ** -0.5
            p = torch.softmax(s, 0)
            want[:see] += p.sum(1)
            tol[:see] += (p * (2 * D * U * mag + 8 * U * s.abs().amax() + 2048 * U)).sum(1)
        assert ((got[0, 0, :n].double() - want).abs() <= tol + 3 * U * want.abs()).all()
        assert torch.equal(got[0, 0, n:], w[0, 0, n:])

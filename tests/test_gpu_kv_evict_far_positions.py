"""Eviction where positions, a segment or a stride further on, pass 2^31: a table of 2.1e9 positions, nearly all of them always kept."""
import numpy as np
import pytest
import torch

from test_gpu_kv_evict import rule

pytestmark = pytest.mark.gpu


def test_positions_near_two_to_the_31():
    from paper_2511_14617_amd import binding
    P, pages, D = 1 << 20, 2047, 8                           # (the last page that a table may have: its positions end 2^20 below 2^31)
    first, n = 2_100_000_000, 2_100_030_000
    page, at = first // P, first % P
    assert (n - 1) // P == page
    last, limit, budget = 100, first + 20000, first + 15000
    g = torch.Generator(device="cuda").manual_seed(1)
    table = torch.full((1, pages), 1 << 29, dtype=torch.int32, device="cuda")           # (pages of always-kept positions are not looked at)
    table[0, page] = 1
    pool = lambda: torch.randint(-32768, 32767, (2, 1, P, D), device="cuda", generator=g, dtype=torch.int16).view(torch.bfloat16)
    k, v = pool(), pool()
    w = torch.zeros((1, 1, pages * P), device="cuda")
    w[0, 0, first:n] = torch.randn(n - first, device="cuda", generator=g).exp_()
    # the same request without its always-kept positions
    short = dict(k=k[1:, :, at:at + n - first].contiguous(), v=v[1:, :, at:at + n - first].contiguous(), w=w[:, :, first:n].contiguous(),
                 table=torch.zeros((1, 1), dtype=torch.int32, device="cuda"), ctx=torch.full((1,), n - first, dtype=torch.int32, device="cuda"))
    _, kept, sums, pools = rule(short, limit - first, budget - first, [0], last)
    before = [t[:, :, :at].clone() for t in (k, v)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx = torch.full((1,), n, dtype=torch.int32, device="cuda")
    new, got = binding.seer_kv_evict(k, v, table, ctx, w, limit=limit, budget=budget, keep_first=first, keep_last=last, new_weights=w, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0 and new.item() == budget
    assert np.array_equal(got[0, 0, first:].cpu().numpy(), kept[0, 0] + first)
    step = 1 << 28
    for j in range(0, first, step):
        assert torch.equal(got[0, 0, j:min(first, j + step)], torch.arange(j, min(first, j + step), dtype=torch.int32, device="cuda")), j
    assert np.array_equal(w[0, 0, first:budget].cpu().numpy(), sums[0, 0, :budget - first])
    for t, want, old in zip((k, v), pools, before):
        assert np.array_equal(t.view(torch.int16)[1, 0, at:at + n - first].cpu().numpy(), want[0, 0])
        assert torch.equal(t[:, :, :at].view(torch.int16), old.view(torch.int16))
    # a request that is not cut: kept is -1 up to the end
    del got
    ctx.fill_(limit)
    new, got = binding.seer_kv_evict(k, v, table, ctx, w, limit=limit, budget=budget, keep_first=first, keep_last=last, status=status)
    torch.cuda.synchronize()
    assert new.item() == limit and all((got[0, 0, j:j + step] == -1).all() for j in range(0, budget, step))
    del w, got, k, v
    torch.cuda.empty_cache()

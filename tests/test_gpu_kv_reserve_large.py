"""seer_kv_reserve beyond the sizes of a server's step, exactly: more rows than first_token's copy in LDS holds, more pieces of the pool than a workgroup has
threads, pieces of more than one pass; free pages in the last pieces and far apart."""
import random

import pytest

from test_gpu_kv_reserve import Server, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,pages,width,page,longest", [(4096, 9000, 6, 16, 30), (4097, 9000, 6, 16, 30), (16384, 30000, 5, 8, 20), (16384, 33000, 4, 1, 3)])
def test_many_rows(B, pages, width, page, longest):
    server = Server(B, B, pages, width, page)
    for k in range(4):
        server.step(longest, pad=(0, 7, 300, 1)[k])


# (a pool is looked at in pieces of 4096 pages, 256 of them a pass; beyond 2048 pieces in pieces of twice as many and more)
@pytest.mark.parametrize("pages", [256 * 4096, 256 * 4096 + 1, 1_100_000, 2048 * 4096, 2048 * 4096 + 1, 9_000_001])
@pytest.mark.parametrize("where", ["last", "apart"])
def test_large_pools(pages, where):
    """Nearly all pages are taken; the rows ask for more than there are free, then for somewhat fewer, then one row for what all give back."""
    rng, page, width, B = random.Random(pages), 4, 100, 70
    free = range(pages - 2800, pages) if where == "last" else sorted({0, pages - 1} | set(rng.sample(range(pages), 2798)))
    refs = [1] * pages
    for p in free:
        refs[p] = 0
    table, held, ctx = [[0] * width for _ in range(B)], [0] * B, [0] * B
    taken = iter(rng.sample([p for p in range(0, pages, pages // 5000) if refs[p]], 600))
    for b in range(0, B, 3):                                          # (every third row holds pages, some of them more than it needs)
        held[b] = rng.randint(1, 20)
        table[b][:held[b]] = [next(taken) for _ in range(held[b])]
        ctx[b] = rng.randint(0, held[b] * page)
    for longest, status, left in ((width, 8, 100), (35, 0, 1200)):   # (rows are served until one needs more than there is)
        new = [longest * page - rng.randint(0, 9) - c for c in ctx]
        new[3], new[9] = -1, 0
        out = check(table, held, refs, ctx, new, None, None, sum(max(n, 0) for n in new) + 5, page)
        assert out[7] == status and sum(r == 0 for r in out[2]) < left
    out = check(table, held, refs, [0] * B, [-1] * (B - 1) + [width * page], None, None, width * page, page)
    assert out[7] == 0 and out[1] == [0] * (B - 1) + [width]

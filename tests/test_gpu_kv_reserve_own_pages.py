"""seer_kv_reserve with SEER_RESERVE_OWN_PAGES, exactly: no slot in a page that another row holds as well, whatever brought the row there; and the same
results otherwise as without the flag."""
import random

import pytest
import torch

from reserve_reference import reserve
from test_gpu_kv_reserve import Server, dev, signed

pytestmark = pytest.mark.gpu


def both(table, held, refs, ctx, new, share, mask, n_tokens, page):
    """The call with the flag against the plain implementation, whose slots in pages of a count above 1 are taken back."""
    from paper_2511_14617_amd import binding as b
    want = list(reserve(table, held, refs, ctx, new, share, mask, n_tokens, page))
    want[5], want[6] = want[5][:], want[6][:]
    for i, s in enumerate(want[5]):
        if s >= 0 and want[2][s // page] > 1:
            want[5][i] = want[6][i] = -1
            want[7] |= 32
    t, h, r, status = dev(table), dev(held), dev(refs), dev([0])
    got = b.seer_kv_reserve(t, h, r, dev(ctx), dev(new), n_tokens, page, share_from=dev(share), tree_mask=dev(signed(mask), torch.int64), status=status,
                            own_pages=True)
    torch.cuda.synchronize()
    for name, x, y in zip(("block_table", "pages_held", "page_refs", "step_len", "first_token", "slot", "position"), (t, h, r, *got), want):
        assert x.tolist() == y, name
    assert status.item() == want[7]
    return want


@pytest.mark.parametrize("pages", [64, 40000])
def test_every_way_into_a_shared_page(pages):
    page, width = 4, 6
    table = [[1, 2, 3, 0, 0, 0], [1, 2, 4, 0, 0, 0], [5, 6, 0, 0, 0, 0], [0] * 6, [7, 8, 0, 0, 0, 0], [0] * 6]
    held, refs = [3, 3, 2, 0, 2, 0], [0] * pages
    for row, h in zip(table, held):
        for p in row[:h]:
            refs[p] += 1
    go = [12, 11, 8, 0, 8, 0]

    def run(status, slots, new, **ctx):
        c, share = go[:], [-1] * 6
        for b, (x, s) in ctx.items():
            c[int(b[1:])], share[int(b[1:])] = x, s
        out = both(table, held, refs, c, new, share, None, sum(max(n, 0) for n in new) + 1, page)
        assert out[7] == status and [i for i, s in enumerate(out[5]) if s < 0] == slots, (out[5], out[7])

    run(0, [9], [1, 5, 1, 0, 2, 0])                                   # (nobody in a shared page: the rows' own tails and new pages)
    run(32, [0, 1, 6], [6, 0, 0, 0, 0, 0], r0=(6, -1))                # cut into the second page, which row 1 holds too: two slots there
    run(32, [0, 1, 2, 3, 4, 5, 6, 9], [0, 9, 0, 0, 0, 0], r1=(1, -1))                     # ... into the first: both shared pages, not the row's own
    run(0, [6], [6, -1, 0, 0, 0, 0], r0=(6, -1))                      # the other row is over: the page is the row's own from now on
    run(32, [0, 3], [0, 0, 2, 1, 0, 0], r2=(7, -1), r3=(8, 2))        # row 3 takes over the page in which row 2 goes on
    run(0, [2], [0, 0, 1, 1, 0, 0], r2=(8, -1), r3=(8, 2))            # ... which row 2 has filled
    run(32, [0, 1, 4], [0, 0, 0, 0, 2, 2], r4=(6, -1), r5=(8, 4))
    run(0, [2], [0, 0, 0, 0, 2, 0], r4=(6, -1))
    refs[8] += 1                                                      # (the caller keeps a page)
    run(32, [0, 1, 2], [0, 0, 0, 0, 2, 0], r4=(6, -1))


def test_a_row_that_gets_nothing_shares_nothing():
    """Row 1 would take over row 0's half full page, but there is no page for its new tokens: row 0 goes on."""
    for pages in (4, 33000):
        refs = [1] * pages
        out = both([[2, 0, 0], [0, 0, 0]], [1, 0], refs, [3, 4], [1, 5], [-1, 0], None, 6, 4)
        assert out[7] == 8 and out[5][0] == 2 * 4 + 3


@pytest.mark.parametrize("seed,B,pages,width,page,longest", [(4, 64, 5000, 60, 16, 700), (5, 5, 64, 30, 7, 150), (7, 65, 32769, 40, 16, 300), (8, 40, 70000, 300, 3, 700)])
def test_steps_of_a_server(seed, B, pages, width, page, longest):
    server, seen = Server(seed, B, pages, width, page), 0
    for k in range(6):
        ctx, new, share, mask, tokens = server.ask(longest, (0, 5, 0, 300, 1, 0)[k])
        out = both(server.table, server.held, server.refs, ctx, new, share, mask, tokens, page)
        server.table, server.held, server.refs, step = out[:4]
        seen |= out[7]
        for b in range(B):
            if new[b] == -1:
                server.len[b] = 0
            elif step[b]:
                server.len[b] = step[b]
    assert B == 5 or seen & 32                                       # (the servers' requests come to it)


def test_the_other_row_keeps_its_cache():
    """A group on one prompt, one response cut into it: its new rows do not reach the pages of the others."""
    from paper_2511_14617_amd import binding as b
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, held, refs = i32([[0] * 8] * 3), i32([0] * 3), i32([0] * 40)
    pool = torch.zeros((40, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    rows = lambda n, value: torch.full((n, 1, 64), value, dtype=torch.bfloat16, device="cuda")
    for ctx, new, share, value, n in (([0, 0, 0], [64, 0, 0], None, 1.0, 64), ([64, 64, 48], [5, 5, 21], [-1, 0, 0], 2.0, 31)):
        made = b.seer_kv_reserve(table, held, refs, i32(ctx), i32(new), n, 16, share_from=None if share is None else i32(share), own_pages=True)
        b.seer_kv_append(None, rows(n, value), None, made[2], None, pool, None)
    before, status = pool.clone(), i32([0])
    made = b.seer_kv_reserve(table, held, refs, i32([69, 40, 69]), i32([1, 30, 1]), 32, 16, own_pages=True, status=status)
    b.seer_kv_append(None, rows(32, 9.0), None, made[2], None, pool, None)
    assert status.item() == 32
    for row in (0, 2):
        pages = table[row, :5].long()
        flat = lambda x: x[pages].transpose(1, 2).reshape(-1, 64)[:69]
        assert torch.equal(flat(pool), flat(before))


def test_refused_and_captured():
    from paper_2511_14617_amd import binding as b
    import ctypes
    p = b.SeerReserveParams(2, 4, 40000, 6, 7, 2)
    assert b.seer_kv_reserve_workspace(p) == 0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for pages in (64, 40000):
        state = i32([[1, 2, 0, 0, 0, 0], [1, 3, 0, 0, 0, 0]]), i32([2, 2]), i32([0, 2, 1, 1] + [0] * (pages - 4))
        keep = [x.clone() for x in state]
        ctx, new = i32([2, 8]), i32([3, 4])
        out, status = (i32([0] * 2), i32([0] * 3), i32([0] * 7), i32([0] * 7)), i32([0])
        ws = torch.empty(max(256, b.seer_kv_reserve_workspace(b.SeerReserveParams(2, 4, pages, 6, 7, 1))), dtype=torch.uint8, device="cuda")
        call = lambda: b.seer_kv_reserve(*state, ctx, new, 7, 4, out=out, status=status, workspace=ws, own_pages=True)
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(3):
            for x, y in zip(state, keep):
                x.copy_(y)
            status.zero_()
            graph.replay()
            torch.cuda.synchronize()
            first = state[0][1, 2].item()
            assert status.item() == 32 and out[2].tolist() == [-1, -1, 8, first * 4, first * 4 + 1, first * 4 + 2, first * 4 + 3]
            assert out[3].tolist() == [-1, -1, 4, 8, 9, 10, 11]

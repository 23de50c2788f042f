"""The calls of a server's step one behind the other, as a program makes them: pages for a group's prompt, its rows into the cache, attention over
it; the group's other responses on the prompt's pages; a verify step of drafts over that cache (attention, acceptance, commit, pages
of the next step); a cut cache and finished requests whose pages come back.  Checked against a dense cache of every request in 64
bits, kept from the unrotated keys and the positions."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

PAGE, HQ, HKV, D, WIDTH, POOL = 16, 8, 2, 128, 24, 90
SCALE = D ** -0.5


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Dense:
    """What every request's cache should hold: rotated keys (64 bits) and values, position by position."""

    def __init__(self, B, inv):
        self.k, self.v, self.inv = [[] for _ in range(B)], [[] for _ in range(B)], inv

    def rotate(self, x, position):
        angle = position * self.inv
        c, s = torch.cos(angle), torch.sin(angle)
        a, b = x[..., :D // 2].double(), x[..., D // 2:].double()
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    def attend(self, b, q, position, seen):
        """Attention of q [HQ,D] at `position` over the entries `seen` of request b; (output, sum p |v|)."""
        k, v = torch.stack([self.k[b][j] for j in seen]), torch.stack([self.v[b][j] for j in seen]).double()
        q = self.rotate(q, position).bfloat16().double().view(HKV, HQ // HKV, D)          # (what the call writes to q_out)
        p = torch.softmax(torch.einsum("hgd,jhd->hgj", q, k.bfloat16().double()) * SCALE, -1)
        return torch.einsum("hgj,jhd->hgd", p, v).reshape(HQ, D), torch.einsum("hgj,jhd->hgd", p, v.abs()).reshape(HQ, D)


def close(out, want, what):
    """Output and weights as for the attention call, and the rotation: q and k are off by half a bf16 step (2^-8) where the reference's rounding of the same
    value goes the other way, by fp32's error in it; a flipped rounding of a component changes a score by 2^-8 |q k| scale of one of 128 terms: no more
    than 2^-8 of the sum of |q_d k_d| scale, of which a flip touches one.  2^-6 A holds all of it."""
    ref, weight = want
    error, bound = (out.double() - ref).abs(), 2.0 ** -8 * ref.abs() + 2.0 ** -6 * weight
    assert (error <= bound).all(), "%s: %.2f of the bound" % (what, (error / bound).max())


def test_group_of_responses_from_prompt_to_cut_cache():
    from paper_2511_14617_amd import binding as b
    g = torch.Generator(device="cuda").manual_seed(5)
    bf = lambda *s: torch.randn(s, dtype=torch.bfloat16, device="cuda", generator=g)
    inv32 = (10000.0 ** (-torch.arange(0, D, 2, device="cuda").double() / D)).float()
    B = 4
    dense = Dense(B, inv32.double())
    table, held, refs = i32([[0] * WIDTH] * B), i32([0] * B), i32([0] * POOL)
    kp, vp = bf(POOL, HKV, PAGE, D), bf(POOL, HKV, PAGE, D)
    status = i32([0])

    def tokens_in(step, first, slot, position, mask=None):
        """Rows for all packed tokens: through the cache, and into the dense one."""
        n = slot.numel()
        row = bf(n, (HQ + 2 * HKV) * D)
        q, k, v = row.split([HQ * D, HKV * D, HKV * D], 1)
        q, k, v = q.view(n, HQ, D), k.view(n, HKV, D), v.view(n, HKV, D)
        q_out = b.seer_kv_append(q, k, v, slot, position, kp, vp, inv_freq=inv32, status=status)
        return q, k, v, q_out

    def check_rows(out, q, first, ctx, position, seen_of, what):
        f, c, p = first.tolist(), ctx.tolist(), position.tolist()
        for r in range(B):
            for i in range(f[r], f[r + 1]):
                close(out[i], dense.attend(r, q[i], p[i], seen_of(r, i - f[r], c[r], f[r + 1] - f[r])), (what, r, i - f[r]))

    # 1 the prompt of 71 tokens, in request 0, in two pieces; the others have nothing yet
    prompt = 71
    ctx = i32([0] * B)
    for piece in (40, 31):
        new = i32([piece, 0, 0, 0])
        step, first, slot, position = b.seer_kv_reserve(table, held, refs, ctx, new, 64, PAGE, status=status)
        q, k, v, q_out = tokens_in(step, first, slot, position)
        for i in range(piece):
            dense.k[0].append(dense.rotate(k[i], float(position[i]))), dense.v[0].append(v[i])
        out = b.seer_prompt_attention(q_out, kp, vp, table, step, first, SCALE, status=status)
        check_rows(out, q, first, step, position, lambda r, i, c, n: range(c - n + i + 1), "prompt")
        ctx = step
    # 2 the group's other responses: the prompt's whole pages, the rest of the prompt among their own tokens; request 0 decodes a token beside them
    ctx = i32([prompt, 64, 64, 64])
    new, share = i32([1, 7, 7, 7]), i32([-1, 0, 0, 0])
    before = refs.clone()
    step, first, slot, position = b.seer_kv_reserve(table, held, refs, ctx, new, 25, PAGE, share_from=share, status=status)
    assert refs[table[0, :4].long()].tolist() == [4] * 4 and (refs - before).sum().item() == 3 * 5
    q, k, v, q_out = tokens_in(step, first, slot, position)
    for r in range(B):
        if r:
            dense.k[r], dense.v[r] = dense.k[0][:64], dense.v[0][:64]
    for r in range(B):
        for i in range(int(first[r]), int(first[r + 1])):
            dense.k[r].append(dense.rotate(k[i], float(position[i]))), dense.v[r].append(v[i])
    out = b.seer_prompt_attention(q_out, kp, vp, table, step, first, SCALE, status=status)
    check_rows(out, q, first, step, position, lambda r, i, c, n: range(c - n + i + 1), "responses")
    ctx = step
    # 3 three verify steps with draft trees: positions by depth, slots by node
    T = 5
    parent = [-1, 0, 0, 1, 2]
    words = [1]
    for t in range(1, T):
        words.append(words[parent[t]] | 1 << t)
    mask = torch.tensor(words * B, dtype=torch.int64, device="cuda")
    rng = np.random.default_rng(1)
    for step_no in range(3):
        step, first, slot, position = b.seer_kv_reserve(table, held, refs, ctx, i32([T] * B), B * T, PAGE, tree_mask=mask, status=status)
        assert (position.view(B, T) - ctx[:, None]).tolist() == [[0, 1, 1, 2, 2]] * B
        q, k, v, q_out = tokens_in(step, first, slot, position)
        for r in range(B):
            for i in range(T):
                dense.k[r].append(dense.rotate(k[r * T + i], float(position[r * T + i]))), dense.v[r].append(v[r * T + i])
        out = b.seer_verify_attention(q_out.view(B, T, HQ, D), kp, vp, table, step, mask.view(B, T), SCALE)
        n0 = ctx.tolist()
        sees = lambda r, i, c, n: list(range(n0[r])) + [n0[r] + s for s in range(T) if words[i] >> s & 1]
        check_rows(out.view(B * T, HQ, D), q, first, step, position, sees, "verify")
        # the target's tokens: some paths are accepted as far as they go, some not
        logits = torch.randn((B, T, 50), device="cuda", generator=g)
        best = logits.argmax(-1).tolist()
        draft = [[0] * T for _ in range(B)]
        for r in range(B):
            for t in range(1, T):
                draft[r][t] = best[r][parent[t]] if rng.random() < 0.7 else 49 - best[r][parent[t]]
        parents = i32([parent] * B)
        alen, path, bonus, _ = b.seer_accept(logits, i32(draft), parents)
        b.seer_kv_commit(kp, vp, table, step, alen, path, draft_tokens=i32(draft), bonus_token=bonus, status=status)
        for r, (n, slots) in enumerate(zip(alen.tolist(), path.tolist())):
            kept = [n0[r] + s for s in slots[:n + 1]]
            dense.k[r] = dense.k[r][:n0[r]] + [dense.k[r][j] for j in kept]
            dense.v[r] = dense.v[r][:n0[r]] + [dense.v[r][j] for j in kept]
        ctx = step
        assert ctx.tolist() == [len(x) for x in dense.k]
    # 4 one token each, by the packed call, on what the commits left; then request 2 is over and request 0 is cut to 70 positions
    step, first, slot, position = b.seer_kv_reserve(table, held, refs, ctx, i32([1] * B), B, PAGE, status=status)
    q, k, v, q_out = tokens_in(step, first, slot, position)
    for r in range(B):
        dense.k[r].append(dense.rotate(k[r], float(position[r]))), dense.v[r].append(v[r])
    out = b.seer_prompt_attention(q_out, kp, vp, table, step, first, SCALE, status=status)
    check_rows(out, q, first, step, position, lambda r, i, c, n: range(c), "decode")
    weights = torch.rand((B, HKV, WIDTH * PAGE), device="cuda", generator=g)
    only = i32([0] * B)
    only[0] = step[0]
    cut, _ = b.seer_kv_evict(kp, vp, table, only, weights, limit=70, budget=70, keep_first=64, status=status)
    ctx = torch.where(only > 0, cut, step)
    new = i32([0, 1, -1, 1])
    held_before = held.clone()
    step, first, slot, position = b.seer_kv_reserve(table, held, refs, ctx, new, 4, PAGE, status=status)
    assert held.tolist()[0] == 5 and held.tolist()[2] == 0 and step.tolist()[2] == 0 and held_before[0] >= 5
    assert refs.sum().item() == held.sum().item() and refs[table[0, :4].long()].tolist() == [3] * 4
    assert status.item() == 0
    # 5 everything is over: all pages are free
    b.seer_kv_reserve(table, held, refs, step, i32([-1] * B), 0, PAGE, status=status)
    assert refs.sum().item() == 0 and held.sum().item() == 0 and status.item() == 0


def test_captured_step():
    """Reserve, append and attention of a step in one graph, with lengths that change between replays, against eager calls."""
    from paper_2511_14617_amd import binding as b
    g = torch.Generator(device="cuda").manual_seed(6)
    bf = lambda *s: torch.randn(s, dtype=torch.bfloat16, device="cuda", generator=g)
    inv = (10000.0 ** (-torch.arange(0, D, 2, device="cuda").double() / D)).float()
    B, N = 4, 96
    state = lambda: [i32([[0] * WIDTH] * B), i32([0] * B), i32([0] * POOL)]
    kp0, vp0 = bf(POOL, HKV, PAGE, D), bf(POOL, HKV, PAGE, D)
    ctx, new = i32([0] * B), i32([0] * B)
    row = bf(N, (HQ + 2 * HKV) * D)

    def step(st, kp, vp, out):
        q, k, v = row.split([HQ * D, HKV * D, HKV * D], 1)
        made = b.seer_kv_reserve(*st, ctx, new, N, PAGE)
        q_out = b.seer_kv_append(q.view(N, HQ, D), k.view(N, HKV, D), v.view(N, HKV, D), made[2], made[3], kp, vp, inv_freq=inv,
                                 q_out=torch.zeros((N, HQ, D), dtype=torch.bfloat16, device="cuda"))
        b.seer_prompt_attention(q_out, kp, vp, st[0], made[0], made[1], SCALE, out=out)
        return made

    st, kp, vp, out = state(), kp0.clone(), vp0.clone(), torch.zeros((N, HQ, D), dtype=torch.bfloat16, device="cuda")
    new.fill_(3)
    step(state(), kp0.clone(), vp0.clone(), out.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = step(st, kp, vp, out)
    st2, kp2, vp2, out2 = state(), kp0.clone(), vp0.clone(), torch.zeros_like(out)
    at = torch.zeros(B, dtype=torch.int32, device="cuda")
    for lengths in ([20, 30, 40, 6], [1, 1, 1, 1], [30, 0, 5, 60], [-1, 17, 1, -1], [50, 2, 2, 30]):
        ctx.copy_(at), new.copy_(i32(lengths))
        row.copy_(bf(*row.shape))
        out.zero_(), out2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        made2 = step(st2, kp2, vp2, out2)
        torch.cuda.synchronize()
        for x, y in zip((*st, kp, vp, out, *made), (*st2, kp2, vp2, out2, *made2)):
            assert torch.equal(x, y)
        at = made2[0].clone()

"""seer_prompt_attention against the softmax in 64 bits, row by row.

Tolerance, per output with A = sum_j p_j |v_j|:
  the output is rounded once to bf16: half a step, 2^-8 |out| at most (2^-9 to 2^-8 of it);
  every probability enters the product with V as bf16, off by 2^-8 of it at most and by no more than 2^-9 of it and a half on average
  over the mantissas; the denominator is the sum of the same rounded values, so what is common to all cancels: |error| <= 2 * 2^-8 A at the very
  most (one position up, the others down), which needs all probabilities at the worst mantissa; 2^-8 A is held here;
  scores are fp32 sums of Dqk exact products: off by at most Dqk 2^-24 sum |q k| scale, below 2^-12 for the sizes here, which a
  probability takes over as a relative error: below 2^-11 A with the sum's and the exponential's own.
Together 2^-8 |out| + (2^-8 + 2^-11) A."""
import itertools

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LATENT = (576, 512)


def make(seed, new, past, Hq, Hkv, D, Dv, page, pad=0, std=2.0, spare=2):
    """Random caches with pages in random order; requests of new[b] tokens behind past[b] positions."""
    rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    new, past = np.asarray(new), np.asarray(past)
    ctx = new + past
    need = -(-ctx // page)
    pages = int(need.sum()) + spare
    ids, at = rng.permutation(pages), 0
    table = np.full((len(new), max(1, int(need.max()) + 1)), 2 ** 31 - 1)             # (entries behind the end are not looked at)
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    N = int(new.sum()) + pad
    bf = lambda *shape: torch.randn(shape, generator=g).bfloat16()
    return dict(q=(bf(N, Hq, D).float() * std).bfloat16(), k=bf(pages, Hkv, page, D), v=None if (D, Dv) == LATENT else bf(pages, Hkv, page, Dv),
                table=torch.from_numpy(table).int(), ctx=torch.from_numpy(ctx).int(), first=torch.from_numpy(np.concatenate([[0], np.cumsum(new)])).int(),
                Dv=Dv, page=page, scale=D ** -0.5)


def plain(c, rows=None):
    """(outputs, A) in 64 bits on the device, by request; None for padding.  rows: of each request, at most so many tokens are computed."""
    out = []
    dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    first, ctx = c["first"].tolist(), c["ctx"].tolist()
    Hkv, Hq = c["k"].shape[1], c["q"].shape[1]
    G = Hq // Hkv
    for b, L in enumerate(ctx):
        n = first[b + 1] - first[b]
        if n == 0:
            continue
        j = torch.arange(L, device="cuda")
        pages, inside = dev["table"][b, j // c["page"]].long(), j % c["page"]
        tokens = np.arange(n) if rows is None or n <= rows else np.unique(np.concatenate([[0, n - 1], np.random.default_rng(b).integers(0, n, rows - 2)]))
        t = torch.from_numpy(tokens).cuda()
        for h in range(Hkv):
            k = dev["k"][pages, h, inside].double()
            v = k[:, :c["Dv"]] if c["v"] is None else dev["v"][pages, h, inside].double()
            for hq in range(h * G, h * G + G):
                z = dev["q"][first[b] + t, hq].double() @ k.t() * c["scale"]
                p = torch.softmax(z.masked_fill(j[None] > (L - n + t)[:, None], -float("inf")), -1)
                out.append((first[b] + t, hq, p @ v, p @ v.abs()))
    return out


def call(c, **kw):
    from paper_2511_14617_amd import binding as b
    dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    out = kw.pop("out", None)
    if out is None:
        out = torch.full((c["q"].shape[0], c["q"].shape[1], c["Dv"]), 7.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    got = b.seer_prompt_attention(dev["q"], dev["k"], dev["v"], dev["table"], dev["ctx"], dev["first"], c["scale"], Dv=c["Dv"], out=out, status=status, **kw)
    torch.cuda.synchronize()
    assert got is out
    return out, status.item()


def compare(out, want, what=""):
    worst = 0.0
    for t, hq, ref, weight in want:
        error = (out[t, hq].double() - ref).abs()
        bound = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -11) * weight
        assert torch.isfinite(out[t, hq].float()).all(), what
        worst = max(worst, float((error / bound.clamp(min=1e-30)).max()))
    assert worst <= 1.0, "%s: %.3f of the bound" % (what, worst)


def check(seed, new, past, Hq, Hkv, D, Dv, page, rows=None, **kw):
    c = make(seed, new, past, Hq, Hkv, D, Dv, page, **kw)
    out, status = call(c)
    assert status == 0
    compare(out, plain(c, rows), (new, past, Hq, Hkv, D, page))
    assert (out[int(c["first"][-1]):] == 7.0).all()          # padding
    return c, out


HEADS = [(8, 2, 128, 128, 16), (4, 4, 64, 64, 16), (8, 1, 256, 256, 32), (16, 2, 192, 128, 64), (5, 1, 128, 128, 20), (6, 2, 64, 64, 1), (14, 2, 128, 128, 128),
         (3, 3, 256, 256, 7), (2, 2, 192, 128, 48), (16, 1, 576, 512, 64), (128, 1, 576, 512, 32), (6, 2, 576, 512, 16), (5, 1, 576, 512, 20)]


@pytest.mark.parametrize("heads", HEADS)
def test_lengths_around_every_border(heads):
    """Lengths of zero, one, around tiles, pages and row tiles, whole prompts and behind cached positions, in one batch."""
    new = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 16, 15, 17, 200, 1, 3, 0]
    past = [5, 0, 1, 0, 0, 0, 1, 64, 31, 0, 128, 1, 0, 1000, 15, 17, 333, 700, 0, 0]
    check(1, new, past, *heads, pad=3)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("new,past", [([1], [0]), ([1], [5000]), ([2500], [0]), ([700], [3001]), ([1] * 17, list(range(0, 1700, 100)))])
def test_one_request_and_single_tokens(heads, new, past):
    check(2, new, past, *heads, rows=300)


@pytest.mark.parametrize("seed", range(8))
def test_random_batches(seed):
    rng = np.random.default_rng(seed)
    B = int(rng.integers(1, 40))
    new = [int(rng.choice([0, 1, 1, rng.integers(1, 50), rng.integers(1, 900)])) for _ in range(B)]
    past = [int(rng.choice([0, 0, rng.integers(0, 100), rng.integers(0, 6000)])) for _ in range(B)]
    heads = [(8, 2, 128, 128, 16), (8, 8, 128, 128, 64), (16, 1, 64, 64, 16), (10, 2, 128, 128, 16), (32, 4, 192, 128, 16), (8, 1, 256, 256, 16), (16, 1, 576, 512, 64), (128, 1, 576, 512, 32)][seed]
    check(seed, new, past, *heads, rows=60, pad=int(rng.integers(0, 9)))


def test_more_requests_than_threads():
    """Requests of which most have nothing to do, more of them than a workgroup has threads."""
    rng = np.random.default_rng(0)
    new = np.where(rng.random(1500) < 0.9, 0, rng.integers(1, 40, 1500))
    new[:300] = 0
    check(3, new, rng.integers(0, 60, 1500), 4, 2, 128, 128, 16)


@pytest.mark.parametrize("heads,new,past", [((8, 1, 128, 128, 16), [9000], [0]), ((8, 1, 128, 128, 16), [300, 1, 40], [50000, 60000, 3]), ((64, 8, 128, 128, 16), [4000, 10, 900], [0, 3000, 100]),
                                            ((8, 1, 64, 64, 32), [12000, 5], [0, 30000]), ((16, 2, 256, 256, 16), [3000], [2000]), ((128, 1, 128, 128, 16), [700], [900]),
                                            ((128, 1, 576, 512, 64), [300, 2], [900, 9000]), ((16, 1, 576, 512, 64), [1500, 4], [20000, 3])])
def test_long_ones(heads, new, past):
    check(4, new, past, *heads, rows=40)


def test_results_do_not_depend_on_what_is_beside():
    """The same request alone, with others, and twice: equal bits twice; alone and with others within the tolerance (the cuts differ)."""
    c = make(5, [700, 1, 90], [100, 4000, 0], 8, 2, 128, 128, 16)
    a, _ = call(c)
    b, _ = call(c)
    assert torch.equal(a, b)


def test_equal_scores_and_far_ones():
    """Rows whose scores are all equal (a running mean of V), and scores of several hundred (one position takes all)."""
    for std, zero in ((1.0, True), (200.0, False)):
        c = make(6, [300, 50], [0, 700], 8, 2, 128, 128, 16, std=std)
        if zero:
            c["q"].zero_()
        out, _ = call(c)
        compare(out, plain(c))


@pytest.mark.parametrize("heads", [(8, 2, 128, 128, 16), (16, 1, 576, 512, 64)])
def test_scores_far_below_zero(heads):
    """All scores of a row equal and as low as -10^37 (exactly equal: no rounding is between them): still a running mean of V."""
    c = make(15, [150, 3], [0, 90], *heads)
    c["q"].fill_(1e18)
    if c["v"] is not None:
        c["k"].fill_(-1e18)
    else:                                                            # (the latent's value components stay as they are and meet queries of zero)
        c["q"][..., :512] = 0
        c["k"][..., 512:] = -1e18
    out, _ = call(c)
    compare(out, plain(c))


@pytest.mark.parametrize("base", [2.0 ** 23, -2.0 ** 23, 2.0 ** 11])
@pytest.mark.parametrize("heads", [(8, 1, 128, 128, 16), (4, 1, 64, 64, 20), (16, 1, 576, 512, 64)])
def test_small_differences_of_scores_far_from_zero(heads, base):
    """Scores of base + 0 .. 11, rising with the position and exact in fp32, values of 1 and -1 in turn: what is rounded on the way to the exponential may not be
    rounded at the size of the scores, and pieces of one row, whose references differ, have to agree on it."""
    c = make(27, [40, 3], [4000, 2500], *heads)
    D, Dv = heads[2], heads[3]
    c["scale"] = 1.0
    c["q"].zero_()
    c["q"][..., D - 2], c["q"][..., D - 1] = 2.0 ** 11, 1.0
    c["k"][..., D - 2:] = 0
    for b, L in enumerate(c["ctx"].tolist()):
        j = torch.arange(L)
        at = c["table"][b, j // c["page"]].long(), 0, j % c["page"]
        k = c["k"][at]
        k[:, D - 2], k[:, D - 1] = base / 2 ** 11, (j * 12 // L).bfloat16()
        c["k"][at] = k
        value = (1.0 - 2.0 * (j * 12 // L % 2)).bfloat16()[:, None].expand(L, Dv)
        if c["v"] is None:
            k[:, :Dv] = value
            c["k"][at] = k
        else:
            c["v"][at] = value
    out, _ = call(c)
    compare(out, plain(c))


def spoil(x, b, j, c, value, dims=slice(None)):
    x[c["table"][b, j // c["page"]].long(), :, j % c["page"], dims] = value


@pytest.mark.parametrize("heads", [(8, 2, 128, 128, 16), (4, 4, 64, 64, 20), (8, 1, 256, 256, 32), (16, 2, 192, 128, 64), (16, 1, 576, 512, 64), (5, 1, 576, 512, 20)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_a_token_does_not_see_does_not_reach_it(heads, value):
    """NaN and infinities in keys and values of the second half of a prompt, and in the page behind its end: the first half is what it is without
    them, bit for bit; tokens that see them in a value get them in that component."""
    c = make(7, [200, 70, 33], [0, 300, 0], *heads)
    good, _ = call(c)
    at = [100, 340, 20]
    for b, j in enumerate(at):
        spoil(c["k"], b, j, c, value)
        if c["v"] is not None:
            spoil(c["v"], b, j, c, value, slice(0, 2))
    for b, L in enumerate(c["ctx"].tolist()):                        # slots behind the last position
        for j in range(L, -(-L // c["page"]) * c["page"]):
            spoil(c["k"], b, j, c, value)
            if c["v"] is not None:
                spoil(c["v"], b, j, c, value)
    out, status = call(c)
    assert status == 0
    first, ctx = c["first"].tolist(), c["ctx"].tolist()
    for b, j in enumerate(at):
        before = first[b] + j - (ctx[b] - (first[b + 1] - first[b]))        # the token at position j
        assert torch.equal(out[first[b]:before], good[first[b]:before])


@pytest.mark.parametrize("heads", [(8, 2, 128, 128, 16), (4, 4, 64, 64, 20), (8, 1, 256, 256, 32), (16, 2, 192, 128, 64)])
def test_values_that_are_not_finite_stay_in_their_component(heads):
    """The other components are held to the outputs without the infinity, within the tolerance above: where a tile has masked positions, a value row
    that is not finite enters the sums by itself, in another order than by the matrix product (bits may differ where a sum lies by a border of bf16)."""
    c = make(8, [150, 40], [0, 200], *heads, std=0.5)
    good, _ = call(c)
    want = plain(c)
    for b, j in ((0, 70), (1, 215)):
        spoil(c["v"], b, j, c, float("inf"), 5)
    out, _ = call(c)
    keep = torch.tensor([d for d in range(c["Dv"]) if d != 5], device="cuda")
    compare(out[..., keep], [(t, hq, ref[:, keep], weight[:, keep]) for t, hq, ref, weight in want])
    assert torch.isinf(out[70:150, :, 5].float()).all() and torch.isinf(out[150 + 15:190, :, 5].float()).all()
    assert torch.equal(out[:70, :, 5], good[:70, :, 5])


@pytest.mark.parametrize("page", [64, 20])
def test_a_latent_that_is_not_finite_in_one_component(page):
    """An infinite component of a latent whose score is -inf: rows that see it are what they are without that position, but for the component."""
    c = make(14, [60], [10], 16, 1, 576, 512, page, std=0.5)
    c["q"][..., 7] = c["q"][..., 7].abs() + 0.01
    good, _ = call(c)
    spoil(c["k"], 0, 40, c, -float("inf"), 7)                        # score -inf: probability 0, and 0 * inf in component 7
    out, _ = call(c)
    without = dict(c, k=c["k"].clone())
    spoil(without["k"], 0, 40, c, -1e30, 7)                          # (a score that no probability is left of)
    spoil(without["k"], 0, 40, c, 0.0, slice(0, 7))
    ref, _ = call(without)
    keep = [d for d in range(512) if d > 7]
    assert torch.equal(out[:30], good[:30])
    assert torch.equal(out[30:, :, keep], ref[30:, :, keep])


@pytest.mark.parametrize("page", [64, 20])
@pytest.mark.parametrize("past", [10, 5000])
def test_zero_times_an_infinite_latent(page, past):
    """The same position in a tile that all rows see and in one that some see, for whole row tiles and cut ones: 0 * inf in the component, as in the formula."""
    c = make(15, [160], [past], 16, 1, 576, 512, page, std=0.5)
    c["q"][..., 7] = c["q"][..., 7].abs() + 0.01
    c["q"][..., 300] = c["q"][..., 300].abs() + 0.01
    good, _ = call(c)
    spoil(c["k"], 0, past + 70, c, -float("inf"), 7)
    spoil(c["k"], 0, past + 73, c, -float("inf"), 300)
    out, _ = call(c)
    for component, first in ((7, 70), (300, 73)):
        assert torch.equal(out[:70, :, component], good[:70, :, component])      # (behind it the weights are without position 70)
        assert torch.isfinite(out[:first, :, component]).all() and torch.isnan(out[first:, :, component]).all()
    keep = [d for d in range(512) if d not in (7, 300)]
    assert torch.isfinite(out[..., keep]).all()


def test_scores_of_nothing_but_minus_infinity_give_zeros():
    c = make(9, [40], [0], 4, 2, 128, 128, 16)
    c["q"][:, 1] = 0
    c["q"][:, 1, 0] = 1.0
    c["k"][..., 0] = -float("inf")
    c["q"][:, [0, 2, 3], 0] = 0
    out, _ = call(c)
    assert (out[:, 1] == 0).all()                                    # (0 * inf in the others' scores is NaN)
    assert torch.isnan(out[:, [0, 2, 3]].float()).all()


def test_wrong_numbers_are_reported_and_kept_in_bounds():
    c = make(10, [20, 30, 40, 50], [10, 0, 5, 9], 8, 2, 128, 128, 16)
    want = plain(c)
    ok = lambda out, rows: compare(out, [w for w in want if int(w[0][0]) in rows])
    bad = dict(c, ctx=c["ctx"].clone())
    bad["ctx"][1] = 29
    bad["ctx"][2] = c["table"].shape[1] * 16 + 1
    out, status = call(bad)
    assert status == 1 and (out[20:90] == 0).all()
    ok(out, (0, 90))
    bad = dict(c, table=c["table"].clone())
    bad["table"][0, 0], bad["table"][3, 1] = -5, 2 ** 31 - 1
    out, status = call(bad)
    assert status == 2
    ok(out, (20, 50))
    for first, left in (([0, 20, 50, 90, 141], (90, 140)), ([0, 20, 15, 90, 140], (20, 15)), ([-1, 20, 50, 90, 140], (0, 20)), ([0, 20, 50, 2 ** 31 - 1, 2 ** 31 - 1], (50, 140))):
        out, status = call(dict(c, first=torch.tensor(first, dtype=torch.int32)))
        assert status & 4
        if left[0] < left[1]:
            assert (out[left[0]:left[1]] == 7.0).all()
    # intervals that lie over one another again and again
    B = 300
    big = dict(c, table=c["table"][:1].repeat(B, 1), ctx=torch.full((B,), 140, dtype=torch.int32), first=torch.tensor([0, 140] * (B // 2) + [0], dtype=torch.int32))
    _, status = call(big)
    assert status & 4


def test_nothing_to_do():
    c = make(11, [0, 0, 0], [5, 0, 9], 8, 2, 128, 128, 16, pad=4)
    out, status = call(c)
    assert status == 0 and (out == 7.0).all()
    c = make(11, [0, 3], [5, 0], 8, 2, 128, 128, 16)
    from paper_2511_14617_amd import binding as b
    empty = b.seer_prompt_attention(c["q"][:0].cuda(), c["k"].cuda(), c["v"].cuda(), c["table"].cuda(), c["ctx"].cuda(), c["first"].cuda(), c["scale"])
    assert tuple(empty.shape) == (0, 8, 128)


def test_a_pool_behind_32_bits():
    """Pages at both ends of pools of 5 GiB each."""
    c = make(12, [50, 3], [100, 20], 8, 1, 128, 128, 16, spare=0)
    pages = 5 * 2 ** 30 // (16 * 128 * 2)
    big = lambda x: torch.zeros((pages, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
    want = plain(c)
    k, v = big(0), big(0)
    move = torch.randperm(len(c["k"]), generator=torch.Generator().manual_seed(1)) * ((pages - 1) // (len(c["k"]) - 1))
    k[move.cuda()], v[move.cuda()] = c["k"].cuda(), c["v"].cuda()
    table = torch.where(c["table"] < len(c["k"]), move[c["table"].clamp(max=len(c["k"]) - 1).long()].int(), c["table"])
    from paper_2511_14617_amd import binding as b
    out = b.seer_prompt_attention(c["q"].cuda(), k, v, table.cuda(), c["ctx"].cuda(), c["first"].cuda(), c["scale"])
    compare(out, want)


def test_stream_workspace_and_graph():
    """Captured with lengths that change from replay to replay, against eager calls; on a stream and a workspace of its own."""
    from paper_2511_14617_amd import binding as b
    make_n = lambda seed: make(seed, np.random.default_rng(seed).multinomial(300, [0.25] * 4), [100 * seed, 0, 700, 5], 8, 2, 128, 128, 16)
    width, pages = 80, 200
    pad = lambda c: dict(c, table=torch.nn.functional.pad(c["table"], (0, width - c["table"].shape[1]))) | {
        "k": torch.cat([c["k"], torch.zeros(pages - len(c["k"]), 2, 16, 128).bfloat16()]), "v": torch.cat([c["v"], torch.zeros(pages - len(c["v"]), 2, 16, 128).bfloat16()])}
    cases = [pad(make_n(s)) for s in (1, 2, 3, 4)]
    buf = {k: v.cuda() for k, v in cases[0].items() if isinstance(v, torch.Tensor)}
    p = b.attn_params(buf["q"].unsqueeze(1), buf["k"], buf["v"], buf["table"], cases[0]["scale"])
    p.B = 4
    ws = torch.empty(b.seer_prompt_attention_workspace(p, 300), dtype=torch.uint8, device="cuda")
    out = torch.zeros((300, 8, 128), dtype=torch.bfloat16, device="cuda")
    run = lambda: b.seer_prompt_attention(buf["q"], buf["k"], buf["v"], buf["table"], buf["ctx"], buf["first"], cases[0]["scale"], out=out, workspace=ws)
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    stream = torch.cuda.Stream()
    for c in cases[1:] + cases[:1]:
        for k in buf:
            buf[k].copy_(c[k])
        graph.replay()
        torch.cuda.synchronize()
        eager, _ = call(c, stream=stream)
        assert torch.equal(out, eager)
        compare(out, plain(c))


@pytest.mark.parametrize("T", [1, 4, 9])
def test_agrees_with_the_verify_call(T):
    """Requests of T tokens each: what seer_verify_attention computes for a chain, within both calls' roundings."""
    from paper_2511_14617_amd import binding as b
    c = make(13, [T] * 6, [0, 5, 100, 1000, 3000, 64], 8, 2, 128, 128, 16)
    out, _ = call(c)
    table = torch.where(c["table"] == 2 ** 31 - 1, 0, c["table"]).cuda()
    verify = b.seer_verify_attention(c["q"].cuda().view(6, T, 8, 128), c["k"].cuda(), c["v"].cuda(), table, c["ctx"].cuda(), None, c["scale"])
    want = plain(c)
    compare(out, want)
    compare(verify.view(6 * T, 8, 128), want)

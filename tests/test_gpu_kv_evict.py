"""Eviction from the paged cache, against the rule written out on lists: every output is a copy of an input or a whole number, so all comparisons are
for equality."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def build(B, Hkv, D, Dv, P, ctx, seed, ties=0.1, extra_pages=1):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    ctx = np.asarray(ctx, dtype=np.int32)
    need = -(-ctx // P)
    total = int(need.sum()) + 2
    ids, at = rng.permutation(total), 0
    table = np.full((B, int(max(1, need.max())) + extra_pages), 1 << 29, dtype=np.int32)     # (behind a request's end: anything)
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    pool = lambda d: torch.randint(-32768, 32767, (total, Hkv, P, d), device="cuda", generator=g, dtype=torch.int16).view(torch.bfloat16)
    w = torch.randn((B, Hkv, table.shape[1] * P), device="cuda", generator=g).exp_()
    pick = torch.rand(w.shape, device="cuda", generator=g)
    w[pick < ties] = 0.0
    w[pick > 1 - ties] = 0.75
    dev = lambda a: torch.from_numpy(a).cuda()
    return dict(k=pool(D), v=pool(Dv) if Dv else None, table=dev(table), ctx=dev(ctx), w=w)


def rule(s, limit, budget, first, last):
    """(new lengths, kept, moved sums, pools) by the documented rule."""
    table, ctx, w = s["table"].cpu().numpy(), s["ctx"].cpu().numpy(), s["w"].cpu().numpy()
    pools = [None if t is None else t.view(torch.int16).cpu().numpy() for t in (s["k"], s["v"])]
    B, Hkv, _ = w.shape
    P, E = pools[0].shape[2], budget - last
    new, kept, sums, out = ctx.copy(), np.full((B, Hkv, budget), -1, dtype=np.int32), w.copy(), [None if t is None else t.copy() for t in pools]
    for b in range(B):
        n, f = int(ctx[b]), int(first[b])
        if n <= limit:
            continue
        new[b] = budget
        for h in range(Hkv):
            key = np.where(np.isnan(w[b, h]), -np.inf, w[b, h].astype(np.float64))
            nan = np.isnan(w[b, h])
            order = sorted(range(f, n - last), key=lambda j: (nan[j], -key[j], j))[:E - f]
            chosen = np.sort(np.asarray(order, dtype=np.int64))
            stay = chosen[chosen < E]
            free = np.setdiff1d(np.arange(f, E), stay)
            slot = np.arange(budget)
            slot[free] = chosen[chosen >= E]
            slot[E:] = np.arange(n - last, n)
            kept[b, h] = slot
            sums[b, h, :budget] = w[b, h, slot]
            to = np.arange(budget)
            for old, o in zip(pools, out):
                if o is not None:
                    o[table[b, to // P], h, to % P] = old[table[b, slot // P], h, slot % P]
    return new, kept, sums, out


def check(s, limit, budget, first, last, in_place=True, tensor_first=True, **kw):
    from paper_2511_14617_amd import binding
    B = s["ctx"].shape[0]
    firsts = np.asarray(first if np.ndim(first) else [first] * B, dtype=np.int32)
    new, kept, sums, pools = rule(s, limit, budget, firsts, last)
    k, v = s["k"].clone(), None if s["v"] is None else s["v"].clone()
    w, ctx = s["w"].clone(), s["ctx"].clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    to = w if in_place else torch.full_like(w, -7.0)
    got_len, got_kept = binding.seer_kv_evict(k, v, s["table"], ctx, w, limit=limit, budget=budget, keep_last=last,
                                              keep_first=torch.from_numpy(firsts).cuda() if tensor_first else int(firsts[0]), new_weights=to,
                                              new_ctx_len=ctx if in_place else None, status=status, **kw)
    torch.cuda.synchronize()
    assert status.item() == 0
    assert np.array_equal(got_len.cpu().numpy(), new)
    assert np.array_equal(got_kept.cpu().numpy(), kept)
    for got, want in zip((k, v), pools):
        if got is not None:
            assert np.array_equal(got.view(torch.int16).cpu().numpy(), want)
    got = to.cpu().numpy()
    old = s["w"].cpu().numpy()
    for b in range(B):
        m = int(new[b])
        assert np.array_equal(got[b, :, :m], sums[b, :, :m], equal_nan=True)
        assert np.array_equal(got[b, :, m:], old[b, :, m:] if in_place else np.full_like(old[b, :, m:], -7.0), equal_nan=True)
    if not in_place:
        assert torch.equal(w.view(torch.int32), s["w"].view(torch.int32)) and torch.equal(ctx, s["ctx"])
    return k, v, to


@pytest.mark.parametrize("D,Dv,Hkv,P", [(128, 128, 2, 16), (64, 64, 3, 20), (256, 256, 1, 32), (192, 128, 2, 1), (576, 0, 1, 64), (128, 128, 1, 7), (8, 24, 2, 16)])
@pytest.mark.parametrize("in_place", [True, False])
def test_head_sizes_and_pages(D, Dv, Hkv, P, in_place):
    s = build(5, Hkv, D, Dv, P, [300, 200, 1000, 257, 256], D + P)
    check(s, 256, 200, [16, 0, 33, 100, 7], 40, in_place)


@pytest.mark.parametrize("limit,budget,first,last", [(64, 64, 0, 0), (64, 64, 16, 48), (100, 64, 0, 64), (64, 63, 63, 0), (99, 1, 0, 0), (99, 1, 1, 0), (99, 1, 0, 1),
                                                     (500, 500, 3, 2), (98, 90, 10, 80), (64, 2, 1, 1), (5000, 5000, 0, 0)])
def test_budgets_from_one_on(limit, budget, first, last):
    """Also: windows longer than what is dropped (they overlap their destination), nothing between the two kept ends, a limit nobody reaches."""
    s = build(7, 2, 128, 128, 16, [65, 99, 100, 101, 150, 500, 501], budget)
    check(s, limit, budget, first, last, True, tensor_first=False)
    check(s, limit, budget, first, last, False)


def test_empty_requests_and_one_position():
    s = build(4, 2, 64, 64, 16, [0, 1, 2, 40], 3)
    check(s, 1, 1, 0, 0)
    check(s, 1, 1, 0, 1, False)


WIDE = 700       # pages of 16 beyond the longest request: a table of more than 8192 positions, whose rows are cut into segments


@pytest.mark.parametrize("limit,budget,first,last", [(64, 64, 0, 0), (64, 64, 16, 48), (100, 64, 0, 64), (99, 1, 0, 1), (64, 2, 1, 1), (4096, 4096, 0, 0),
                                                     (4095, 4000, 3, 1), (8000, 7000, 300, 500), (4200, 4100, 4, 4096)])
@pytest.mark.parametrize("in_place", [True, False])
def test_rows_of_segments(limit, budget, first, last, in_place):
    """Lengths around one, two and three segments of candidates."""
    s = build(8, 1, 64, 64, 16, [65, 4096, 4097, 4100 + last, 8192 + first + last, 8193 + first + last, 9000, 12345], budget, extra_pages=WIDE)
    check(s, limit, budget, first, last, in_place)


def test_rows_of_segments_with_equal_negative_infinite_and_nan_sums():
    s = build(8, 1, 64, 64, 16, [9000] * 8, 9, extra_pages=WIDE)
    w = s["w"]
    w[0] = 1.0                                               # all equal: the lowest positions stay
    w[1] = -w[1]
    w[2, :, ::3] = float("inf")
    w[3, :, ::2] = float("nan")
    w[4] = 0.0
    w[4, :, ::2] = -0.0
    w[5] = float("nan")
    w[5, :, 5000] = -float("inf")
    w[6] = torch.arange(w.shape[2], device="cuda", dtype=torch.float32)
    w[7] = -w[6]
    check(s, 8999, 2000, 3, 20)
    check(s, 8999, 8990, 3, 20, False)


@pytest.mark.parametrize("seen", ["low", "high"])
def test_rows_whose_sampled_sums_mislead(seen):
    """The search looks at 512 sums, spread evenly, to know where to look closer: here these are the smallest (largest) of all."""
    n, first, last = 40000, 100, 50
    s = build(2, 1, 64, 64, 16, [n, n], 12)
    total = n - first - last
    at = first + (2 * torch.arange(512, device="cuda") + 1) * total // 1024
    s["w"].add_(1.0)
    s["w"][:, :, at] = 0.5 if seen == "low" else 1e6
    check(s, 20000, 15000, first, last)
    check(s, 20000, 400, first, last, False)
    check(s, 20000, 700, first, last, False)
    check(s, 39990, 39980, first, last)


@pytest.mark.parametrize("n", [70000, 131072])
def test_long_caches(n):
    s = build(2, 1, 64, 64, 16, [n, n // 3], 5)
    check(s, 20000, 12345, 512, 1500)
    check(s, n - 1, n - 40, 512, 3000, False)


def test_many_requests():
    rng = np.random.default_rng(8)
    s = build(300, 1, 64, 64, 16, rng.integers(0, 200, 300), 8)
    check(s, 100, 64, rng.integers(0, 20, 300), 16)


def test_equal_negative_infinite_and_nan_sums():
    s = build(6, 1, 64, 64, 16, [400] * 6, 9)
    s["w"][0] = 1.0                                          # all equal: the lowest positions stay
    s["w"][1] = -s["w"][1]
    s["w"][2, :, ::3] = float("inf")
    s["w"][3, :, ::2] = float("nan")
    s["w"][4] = 0.0
    s["w"][4, :, ::2] = -0.0                                 # (equal to +0)
    s["w"][5] = float("nan")
    s["w"][5, :, 5] = -float("inf")
    check(s, 399, 200, 3, 20)
    check(s, 399, 390, 3, 20, False)


def test_sums_that_differ_in_their_last_bits_only():
    s = build(2, 2, 64, 64, 16, [3000, 2000], 10)
    bits = torch.randint(0, 700, s["w"].shape, device="cuda", dtype=torch.int32)
    s["w"] = (bits + 0x3F800000).view(torch.float32)
    check(s, 1999, 1024, 100, 64)


def test_without_optional_outputs():
    from paper_2511_14617_amd import binding
    s = build(3, 2, 128, 128, 16, [300, 100, 222], 11)
    want = rule(s, 200, 150, [5] * 3, 20)
    k, v, w = s["k"].clone(), s["v"].clone(), s["w"].clone()
    lib = binding.load_library()
    import ctypes
    p = binding.SeerAttnParams(3, 1, 2, 2, 128, 128, 16, k.shape[0], s["table"].shape[1], 0, 0, 0, 1.0)
    e = binding.SeerEvictParams(200, 150, 5, 20)
    ws = torch.full((binding.seer_kv_evict_workspace(p, e),), 0xEE, dtype=torch.uint8, device="cuda")
    new = torch.empty(3, dtype=torch.int32, device="cuda")
    rc = lib.seer_kv_evict(ctypes.byref(p), ctypes.byref(e), k.data_ptr(), v.data_ptr(), s["table"].data_ptr(), s["ctx"].data_ptr(), None, w.data_ptr(),
                           new.data_ptr(), None, None, None, ws.data_ptr(), ws.numel(), None)
    torch.cuda.synchronize()
    assert rc == 0 and np.array_equal(new.cpu().numpy(), want[0]) and torch.equal(w, s["w"])
    assert np.array_equal(k.view(torch.int16).cpu().numpy(), want[3][0]) and np.array_equal(v.view(torch.int16).cpu().numpy(), want[3][1])


@pytest.mark.parametrize("extra", [1, WIDE])
def test_unusable_requests_are_left_alone_and_reported(extra):
    from paper_2511_14617_amd import binding
    s = build(4, 2, 128, 128, 16, [300, 300, 300, 250], 12, extra_pages=extra)
    firsts = np.asarray([5, 5, 5, 5], dtype=np.int32)
    for what, at, value, bit in (("ctx", 1, -1, 1), ("ctx", 1, 16 * s["table"].shape[1] + 1, 1), ("first", 1, -1, 4), ("first", 1, 181, 4), ("table", (1, 0), -1, 2),
                                 ("table", (1, 18), 1 << 29, 2)):
        t = dict(s, ctx=s["ctx"].clone(), table=s["table"].clone(), first=torch.from_numpy(firsts).cuda())
        t[what][at] = value
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        k, v, w = s["k"].clone(), s["v"].clone(), s["w"].clone()
        new, kept = binding.seer_kv_evict(k, v, t["table"], t["ctx"], w, limit=250, budget=200, keep_first=t["first"], keep_last=20, new_weights=w, status=status)
        assert status.item() == bit, what
        ref = dict(s, ctx=s["ctx"].clone())
        ref["ctx"][1] = 100                                  # (as if it were short)
        want = rule(ref, 250, 200, firsts, 20)
        assert new[1] == t["ctx"][1] and (kept[1] == -1).all()
        assert np.array_equal(kept.cpu().numpy(), want[1])
        assert np.array_equal(k.view(torch.int16).cpu().numpy(), want[3][0]) and np.array_equal(v.view(torch.int16).cpu().numpy(), want[3][1])
        assert np.array_equal(w.cpu().numpy(), want[2])
    # a bad keep_first or page of a request that is not cut is nobody's business
    t = dict(s, table=s["table"].clone(), first=torch.from_numpy(firsts).cuda())
    t["first"][3], t["table"][3, 2] = 10 ** 6, -5
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    new, _ = binding.seer_kv_evict(s["k"].clone(), s["v"].clone(), t["table"], t["ctx"] if "ctx" in t else s["ctx"], s["w"].clone(), limit=250, budget=200,
                                   keep_first=t["first"], keep_last=20, status=status)
    assert status.item() == 0 and new.tolist() == [200, 200, 200, 250]


def test_a_page_of_the_common_prefix_may_be_shared():
    s = build(4, 2, 128, 128, 16, [300, 310, 290, 320], 13)
    s["table"][1:, :4] = s["table"][0, :4].clone()
    k, v, _ = check(s, 200, 180, 64, 16)
    shared = s["table"][0, :4].long()
    assert torch.equal(k[shared].view(torch.int16), s["k"][shared].view(torch.int16)) and torch.equal(v[shared].view(torch.int16), s["v"][shared].view(torch.int16))


@pytest.mark.parametrize("extra", [1, WIDE])
def test_other_stream_and_graph(extra):
    from paper_2511_14617_amd import binding
    s = build(6, 2, 128, 128, 16, [300, 500, 260, 100, 777, 1000], 14, extra_pages=extra)
    p = binding.SeerAttnParams(6, 1, 2, 2, 128, 128, 16, s["k"].shape[0], s["table"].shape[1], 0, 0, 0, 1.0)
    ws = torch.full((binding.seer_kv_evict_workspace(p, binding.SeerEvictParams(256, 200, 8, 33)),), 0x77, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    k, v, w = s["k"].clone(), s["v"].clone(), s["w"].clone()
    ctx, new, kept = s["ctx"].clone(), torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros((6, 2, 200), dtype=torch.int32, device="cuda")
    call = lambda k, v, w, ctx, **kw: binding.seer_kv_evict(k, v, s["table"], ctx, w, limit=256, budget=200, keep_first=8, keep_last=33, new_weights=w, workspace=ws, **kw)
    torch.cuda.synchronize()
    call(k, v, w, ctx, stream=side)
    side.synchronize()
    want = rule(s, 256, 200, [8] * 6, 33)
    assert np.array_equal(k.view(torch.int16).cpu().numpy(), want[3][0]) and np.array_equal(w.cpu().numpy()[4, :, :200], want[2][4, :, :200])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(k, v, w, ctx, new_ctx_len=new, kept=kept)
    for replay in range(4):
        now = torch.roll(s["w"], replay * 11, 2)
        k.copy_(s["k"]), v.copy_(s["v"]), w.copy_(now)
        want = rule(dict(s, w=now), 256, 200, [8] * 6, 33)
        new.zero_(), kept.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(new.cpu().numpy(), want[0]) and np.array_equal(kept.cpu().numpy(), want[1]), replay
        assert np.array_equal(k.view(torch.int16).cpu().numpy(), want[3][0]) and np.array_equal(v.view(torch.int16).cpu().numpy(), want[3][1]), replay


def test_binding_refuses_what_it_cannot_marshal():
    from paper_2511_14617_amd import binding
    s = build(2, 2, 128, 128, 16, [300, 200], 15)
    good = dict(limit=250, budget=200)
    for bad in (dict(k=s["k"].float()), dict(v=s["v"][:-1]), dict(w=s["w"][:, :, :-1]), dict(ctx=s["ctx"].long()), dict(k=s["k"].transpose(1, 2)),
                dict(table=s["table"][0])):
        t = dict(s, **bad)
        with pytest.raises(ValueError):
            binding.seer_kv_evict(t["k"], t["v"], t["table"], t["ctx"], t["w"], **good)
    with pytest.raises(ValueError):
        binding.seer_kv_evict(s["k"], s["v"], s["table"], s["ctx"], s["w"], keep_first=torch.zeros(2, device="cuda"), **good)
    for kw in (dict(limit=100, budget=101), dict(limit=100, budget=0), dict(limit=100, budget=50, keep_last=51), dict(limit=100, budget=50, keep_first=-1)):
        with pytest.raises(binding.SeerError):
            binding.seer_kv_evict(s["k"], s["v"], s["table"], s["ctx"], s["w"], **kw)

"""seer_kv_append against the rotation in 64 bits.

Tolerance.  An output a cos - b sin is rounded once to bf16 (half a step: 2^-8 of it, and denormals do not occur).  Before that, in fp32: the
angle, exact to 2^-24 of half a turn once it is reduced (64 bits: a product of up to 10^6 turns leaves 10^-10), gives sine and cosine
an error of at most pi 2^-24 each; their evaluation and the two roundings of the products and the sum add a few 2^-24.  Together below
2^-20 (|a| + |b|), which matters where a cos and b sin cancel.  What is copied has to be equal."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu


def make(seed, N, Hq, Hkv, D, Dv, page, pages, R, at, interleaved, far=40000, empty=0.1, fused=False, pad=0):
    g = torch.Generator().manual_seed(seed)
    bf = lambda *shape: torch.randn(shape, generator=g).bfloat16()
    if fused:                                            # slices of one projection, with a few components between
        row = bf(N, (Hq + Hkv) * D + Hkv * Dv + 8 * 3)
        q, k = row[:, :Hq * D].view(N, Hq, D), row[:, Hq * D + 8:(Hq + Hkv) * D + 8].view(N, Hkv, D)
        v = row[:, (Hq + Hkv) * D + 16:(Hq + Hkv) * D + 16 + Hkv * Dv].view(N, Hkv, Dv) if Dv else None
    else:
        q, k, v = bf(N, Hq, D), bf(N, Hkv, D), bf(N, Hkv, Dv) if Dv else None
    slot = torch.randperm(pages * page, generator=g)[:N].int()
    slot[torch.rand(N, generator=g) < empty] = -1
    position = torch.randint(0, far, (N,), generator=g).int()
    inv = (10000.0 ** (-torch.arange(0, R, 2).double() / max(R, 1))).float()
    return dict(q=q if Hq else None, k=k, v=v, slot=slot, position=position, inv=inv, at=at, interleaved=interleaved,
                kp=bf(pages, Hkv, page, D), vp=bf(pages, Hkv, page, Dv) if Dv else None)


def turned(x, position, inv, at, interleaved):
    """(the rotation in 64 bits, |a| + |b| of each component's pair; zero where nothing is rotated)"""
    y, weight = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    R = 2 * len(inv)
    for j in range(len(inv)):
        i0, i1 = (at + 2 * j, at + 2 * j + 1) if interleaved else (at + j, at + j + R // 2)
        angle = position.double() * inv[j].double()
        a, b = x[..., i0].double(), x[..., i1].double()
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        y[..., i0], y[..., i1] = a * c - b * s, b * c + a * s
        weight[..., i0] = weight[..., i1] = a.abs() + b.abs()
    return y, weight


def close(got, want, weight, what):
    error = (got.double() - want).abs()
    bound = torch.where(weight > 0, 2.0 ** -8 * want.abs() + 2.0 ** -20 * weight, 0.0)
    assert (error <= bound).all(), "%s: %g of the bound" % (what, (error / bound.clamp(min=1e-30)).max())


def run(c, page, q_out="new", **kw):
    from paper_2511_14617_amd import binding as b
    up = lambda x: None if x is None else x.cuda()
    if c["q"] is not None and not c["q"].is_contiguous():                       # (a copy to the device keeps no distance between rows)
        base = c["q"]._base.cuda()
        like = lambda x: base.as_strided(x.shape, x.stride(), x.storage_offset())
        q, k, v = like(c["q"]), like(c["k"]), None if c["v"] is None else like(c["v"])
    else:
        q, k, v = up(c["q"]), up(c["k"]), up(c["v"])
    kp, vp, status = up(c["kp"]), up(c["vp"]), torch.zeros(1, dtype=torch.int32, device="cuda")
    before = None if q is None else torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
    out = {"new": before, "itself": q}[q_out] if q is not None else None
    got = b.seer_kv_append(q, k, v, up(c["slot"]), up(c["position"]), kp, vp, inv_freq=up(c["inv"]) if len(c["inv"]) else None, rotary_at=c["at"],
                           interleaved=c["interleaved"], q_out=out, status=status, **kw)
    torch.cuda.synchronize()
    live = (c["slot"] >= 0) & (c["slot"] < kp.shape[0] * page)
    assert status.item() == int(((c["slot"] < -1) | (c["slot"] >= kp.shape[0] * page)).any())
    slot = c["slot"][live].long()
    if q is not None:
        assert got is out
        want, weight = turned(c["q"], c["position"], c["inv"], c["at"], c["interleaved"])
        close(got.cpu()[live], want[live], weight[live], "q")
        stays = torch.full_like(c["q"], 3.0) if q_out == "new" else c["q"]
        assert torch.equal(got.cpu()[~live], stays[~live])
    want, weight = turned(c["k"], c["position"], c["inv"], c["at"], c["interleaved"])
    wk, wv = c["kp"].double(), None if vp is None else c["vp"].clone()
    heavy = torch.zeros(wk.shape, dtype=torch.float64)
    wk[slot // page, :, slot % page], heavy[slot // page, :, slot % page] = want[live], weight[live]
    close(kp.cpu(), wk, heavy, "k")
    if vp is not None:
        wv[slot // page, :, slot % page] = c["v"][live]
        assert torch.equal(vp.cpu(), wv)
    return got, kp, vp


SHAPES = [  # Hq, Hkv, D, Dv, page, R, at
    (8, 2, 128, 128, 16, 128, 0), (64, 8, 128, 128, 16, 64, 0), (5, 5, 64, 64, 20, 32, 16), (1, 1, 8, 8, 1, 0, 0), (3, 1, 16, 24, 7, 16, 0),
    (8, 1, 256, 256, 32, 256, 0), (16, 16, 192, 128, 64, 64, 128), (128, 1, 576, 0, 64, 64, 512), (16, 1, 576, 0, 64, 64, 512), (0, 2, 128, 128, 16, 128, 0),
    (2, 1, 4096, 4096, 3, 512, 8)]


@pytest.mark.parametrize("shape,N,interleaved", [(s, n, i) for (s, n), i in itertools.product(zip(SHAPES, (37, 9, 130, 1, 23, 6, 40, 5, 21, 64, 3)), (False, True))])
def test_shapes(shape, N, interleaved):
    Hq, Hkv, D, Dv, page, R, at = shape
    run(make(N, N, Hq, Hkv, D, Dv, page, N // page + 3, R, at, interleaved, fused=Hq > 0 and N % 2 == 1), page)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 255, 1024, 1027])
def test_lengths_and_in_place(N):
    for place in ("new", "itself"):
        run(make(N, N, 8, 2, 128, 128, 16, N // 16 + 2, 128, 0, False, empty=0.0 if N == 1 else 0.2), 16, place)


@pytest.mark.parametrize("far", [1, 2 ** 20, 2 ** 31 - 1])
def test_far_positions(far):
    c = make(3, 200, 4, 2, 128, 128, 16, 20, 128, 0, False, far=far)
    c["position"][:3] = torch.tensor([0, far - 1, far // 2], dtype=torch.int32)
    if far > 2 ** 24:
        c["inv"][0] = 0.5                                # (2^31 radians in fp64: 10^-7 of a turn are left, as the reference leaves itself)
        c["inv"][1:] *= 1e-3
    run(c, 16)


def test_slots_beyond_the_pool_are_left_out():
    c = make(5, 40, 4, 2, 64, 64, 16, 5, 64, 0, False)
    c["slot"][3:7] = torch.tensor([80, -2, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    run(c, 16)


def test_copies_keep_every_bit():
    """Without a rotation, and beside the rotated components: all bit patterns, NaN among them."""
    from paper_2511_14617_amd import binding as b
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(64, 8, 128)
    x = bits.view(torch.bfloat16).cuda()
    slot = torch.arange(64, dtype=torch.int32, device="cuda")
    kp, vp = (torch.zeros((4, 8, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = b.seer_kv_append(x, x, x, slot, None, kp, vp)
    for got in (q, kp.transpose(1, 2).reshape(64, 8, 128), vp.transpose(1, 2).reshape(64, 8, 128)):
        assert torch.equal(got.contiguous().view(torch.int16).cpu(), bits)


def test_a_pool_behind_32_bits():
    """Rows whose byte offsets do not fit 32 bits, at both ends of a pool of 6 GiB."""
    from paper_2511_14617_amd import binding as b
    pages, page, H, D = 3 * 2 ** 30 // (16 * 8 * 128) * 1, 16, 8, 128
    kp = torch.zeros((pages, H, page, D), dtype=torch.bfloat16, device="cuda")
    k = torch.randn((3, H, D), dtype=torch.bfloat16, device="cuda")
    slot = torch.tensor([pages * page - 1, 0, pages * page // 2 + 5], dtype=torch.int32, device="cuda")
    b.seer_kv_append(None, k, None, slot, None, kp, None)
    for i, s in enumerate(slot.tolist()):
        assert torch.equal(kp[s // page, :, s % page], k[i])
    assert int((kp.view(torch.int16) != 0).sum()) == int((k.view(torch.int16) != 0).sum())


def test_stream_and_graph():
    from paper_2511_14617_amd import binding as b
    c = make(8, 100, 8, 2, 128, 128, 16, 9, 128, 0, False)
    stream = torch.cuda.Stream()
    got = run(c, 16, stream=stream)
    up = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    out = torch.zeros_like(up["q"])
    call = lambda: b.seer_kv_append(up["q"], up["k"], up["v"], up["slot"], up["position"], up["kp"], up["vp"], inv_freq=up["inv"], q_out=out)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (1, 2, 3):
        n = make(seed, 100, 8, 2, 128, 128, 16, 9, 128, 0, False)
        for name in ("q", "k", "v", "slot", "position", "kp", "vp"):
            up[name].copy_(n[name])
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = run(n, 16)
        assert all(torch.equal(x, y) for x, y in zip((out, up["kp"], up["vp"]), eager))

"""Log probabilities of given tokens, entropies, alternatives and their gradient against the definitions in 64 bits.

Tolerances (u = 2^-24, half a step of fp32).  A term exp2(d) of the sum has the roundings of d (two, so 2 u |d| of its value) and of the
exponential (2 u); the sum adds at most 65 terms per thread, 8 levels across the workgroup and one per chunk and lane: 80 u.  Terms with large |d| are
small (|d| exp2(d) < 1), so l is good to 96 u relative and ln l to 96 u plus its own rounding.  128 u covers both; what
multiplies z or a result is added where it is used."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def reference(x, tokens, tau, top_n):
    """x [N,V] float64, tokens [N]: the outputs in 64 bits (rows of -inf included)."""
    with np.errstate(all="ignore"):
        z = x / tau
        m = z.max(1, keepdims=True)
        safe = np.where(np.isneginf(m), 0.0, m)
        e = np.exp(z - safe)
        l = e.sum(1, keepdims=True)
        lse = (safe + np.log(l))[:, 0]
        logp = np.where(np.isneginf(z), -np.inf, z - safe - np.log(l))      # (z - lse would lose ln l in rows of the type's lowest value)
        p = np.where(np.isneginf(z), 0.0, e / l)
        h = -np.where(p > 0, p * logp, 0.0).sum(1)
    order = np.argsort(-x, axis=1, kind="stable")[:, :top_n]
    ok = (tokens >= 0) & (tokens < x.shape[1])
    pick = logp[np.arange(len(x)), np.where(ok, tokens, 0)]
    return dict(ok=ok, lse=lse, logp=logp, p=p, h=np.where(np.isneginf(lse), 0.0, h), pick=pick, order=order,
                alt=np.take_along_axis(logp, order, 1), reach=np.abs(np.where(np.isfinite(z), z - safe, 0.0)).max(1))


def close(got, ref, tol, what):
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), what
    assert np.all(np.abs(got - np.where(inf, 0, ref))[~inf] <= np.broadcast_to(tol, got.shape)[~inf]), (
        what, float(np.max(np.abs(got - np.where(inf, 0, ref))[~inf] - np.broadcast_to(tol, got.shape)[~inf])))


def check(logits, tokens, tau=1.0, top_n=0, path=None, **kw):
    from paper_2511_14617_amd import binding
    out = binding.seer_token_logprobs(logits, tokens, path, temperature=tau, top_n=top_n, **kw)
    torch.cuda.synchronize()
    V = logits.shape[-1]
    x = logits.double().cpu().numpy().reshape(-1, logits.shape[-2], V) if logits.dim() == 3 else logits.double().cpu().numpy()[:, None]
    tok = tokens.cpu().numpy().reshape(x.shape[:2])
    if path is not None:
        at = path.cpu().numpy()
        tok = np.where((at >= 0) & (at < x.shape[1]), tok, -1)
        x = np.take_along_axis(x, np.clip(at, 0, x.shape[1] - 1)[:, :, None], 1)
    r = reference(x.reshape(-1, V), tok.reshape(-1), float(np.float32(tau)), top_n)
    got = [None if t is None else t.double().cpu().numpy().reshape(len(r["ok"]), -1) for t in out]
    ok = r["ok"]
    zero = [g[~ok] for g in got[:4] if g is not None]
    assert all((z == 0).all() for z in zero)
    base = 128 * U + 4 * U * r["reach"]
    close(got[0][ok, 0], r["pick"][ok], base[ok], "logprob")
    close(got[1][ok, 0], r["h"][ok], (128 * U * (2 + r["h"]))[ok], "entropy")
    close(got[2][ok, 0], r["lse"][ok], (base + 4 * U * np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0)))[ok], "logsumexp")
    if top_n:
        assert (out[4].cpu().numpy().reshape(len(ok), top_n)[~ok] == -1).all()
        assert np.array_equal(out[4].cpu().numpy().reshape(len(ok), top_n)[ok], r["order"][ok]), "alternatives"
        close(got[3][ok], r["alt"][ok], base[ok, None], "their log probabilities")
    return out


def make(N, V, dtype, seed, pad=0, T=None, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (N, V + pad) if T is None else (N, T, V + pad)
    x = (torch.randn(shape, device="cuda", generator=g) * spread).to(dtype)
    tok = torch.randint(0, V, shape[:-1], device="cuda", generator=g, dtype=torch.int32)
    return x[..., :V], tok


DT = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
@pytest.mark.parametrize("N,V,top_n", [(1, 1, 1), (1, 2, 2), (3, 3, 0), (5, 40, 32), (7, 255, 5), (2, 257, 32), (33, 1027, 20), (1, 4096, 8),
                                       (1, 4097, 20), (2, 50257, 20), (3, 152064, 5), (1, 152067, 32), (2, 262144 + 5, 32), (2100, 300, 7),
                                       (2049, 17, 0), (300, 130001, 3)])
def test_sizes(N, V, top_n, dtype):
    check(*make(N, V, dtype, N + V), 0.8 if V % 2 else 1.0, top_n)


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
def test_rows_apart_and_at_any_alignment(dtype):
    x, tok = make(37, 1001, dtype, 3, pad=6)
    check(x, tok, 1.3, 4)
    flat = torch.randn(3 + 40 * 515, device="cuda").to(dtype)
    for off in (1, 2, 3):
        rows = flat[off:off + 40 * 515].view(40, 515)[:, :513]
        check(rows, torch.arange(40, device="cuda", dtype=torch.int32), 1.0, 3)


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
def test_entries_without_a_token_are_zero_and_what_lies_behind_stays(dtype):
    from paper_2511_14617_amd import binding
    x, tok = make(6, 700, dtype, 4)
    tok[1], tok[3], tok[4] = -1, -100, 700
    check(x, tok, 1.0, 3)
    out = tuple(torch.full((9,), 7.0, device="cuda") for _ in range(3)) + (torch.full((9, 3), 7.0, device="cuda"),
                                                                         torch.full((9, 3), 7, dtype=torch.int32, device="cuda"))
    binding.seer_token_logprobs(x, tok, top_n=3, out=tuple(t[:6] for t in out))
    assert all((t[6:] == 7).all() for t in out)


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T,V", [(3, 5, 1024), (9, 33, 3001), (64, 9, 4099), (1, 2, 152064)])
def test_emitted_tokens_of_an_accepted_path(B, T, V, dtype):
    x, tok = make(B, V, dtype, B + T, T=T)
    rng = np.random.default_rng(B)
    path = np.full((B, T), -1, dtype=np.int32)
    for b in range(B):
        a = int(rng.integers(0, T))
        path[b, 0] = 0
        path[b, 1:a + 1] = 1 + np.sort(rng.permutation(T - 1)[:a])
    path[0, T - 1] = T + 3                                   # (outside the slots: no entry)
    check(x, tok, 0.8, 5, torch.from_numpy(path).cuda())
    # the same slot twice is two entries
    check(x, tok, 0.8, 2, torch.full((B, T), T - 1, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(4, 5003), (2100, 97), (2, 40000)])
def test_masked_and_equal_logits(N, V, dtype):
    x, tok = make(N, V, dtype, 11)
    x = x.clone()
    x[0] = -float("inf")                                     # nothing left
    x[1, :] = -float("inf")
    x[1, [V - 1, 5, V // 2]] = torch.tensor([1.0, -3.0, 1.0], device="cuda", dtype=dtype)   # three left, two of them equal
    x[2 % N] = 0.25                                          # flat
    x[3 % N, ::2] = -0.0                                     # (equal to +0)
    x[3 % N, 1::2] = 0.0
    tok[1] = 5
    check(x, tok, 0.7, 20)
    lowest = torch.finfo(dtype).min
    x[0, 3:] = lowest                                        # masks of the type's lowest value
    check(x, tok, 1.0, 9)


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 3, 1001, 4099, 16391])
def test_masked_logits_behind_the_last_whole_vector(V, dtype):
    x, tok = make(6, V, dtype, V)
    x = x.clone()
    x[0, -1] = -float("inf")
    x[1, V // 4 * 4:] = -float("inf")
    x[2, V // 8 * 8:] = -float("inf")
    x[3, :V // 8 * 8] = -float("inf")
    x[4, -1] = torch.finfo(dtype).min
    tok[:] = 0
    check(x, tok, 1.25, min(3, V))                          # (below 1 the lowest value over the temperature leaves the floats)


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
def test_few_distinct_values_give_the_lowest_indices(dtype):
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randint(0, 4, (3, 70001), device="cuda", generator=g).to(dtype)
    x[1] = torch.randint(0, 2, (70001,), device="cuda", generator=g).to(dtype) * 1e-3
    x[2, 69000:] = 9.0
    check(x, torch.tensor([0, 69999, 70000], dtype=torch.int32, device="cuda"), 1.0, 32)


def test_rising_and_falling_rows_reach_every_candidate():
    x = torch.arange(50001, device="cuda", dtype=torch.float32)[None] / 5000
    x = torch.cat([x, x.flip(1), x.abs().roll(20000, 1)])
    check(x, torch.zeros(3, dtype=torch.int32, device="cuda"), 1.0, 32)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_not_finite_values_show_in_their_row_only(bad):
    from paper_2511_14617_amd import binding
    x, tok = make(3, 20000, torch.float32, 8)
    x[1, 12345] = bad
    out = binding.seer_token_logprobs(x, tok, top_n=4)
    assert all(torch.isnan(t[1]) for t in out[:3])
    assert (out[4] >= 0).all() and (out[4] < 20000).all()
    assert torch.isfinite(torch.stack([t[[0, 2]] for t in out[:3]])).all()
    want = binding.seer_token_logprobs(x[[0, 2]].contiguous(), tok[[0, 2]].contiguous(), top_n=4)
    assert torch.equal(out[4][[0, 2]], want[4])


def test_far_apart_and_extreme_temperatures():
    x, tok = make(4, 3001, torch.float32, 9, spread=200.0)
    check(x, tok, 1.0, 5)
    check(x, tok, 0.01, 5)
    check(x, tok, 50.0, 5)


# ------------------------------------------------------------------------------------------------
# gradient
# ------------------------------------------------------------------------------------------------
def grad_reference(x, tok, tau, g_lp, g_h):
    r = reference(x, tok, tau, 1)
    hot = np.zeros_like(x)
    hot[np.arange(len(x))[r["ok"]], tok[r["ok"]]] = 1.0
    logp = np.where(r["p"] > 0, r["logp"], 0.0)
    g = g_lp[:, None] * (hot - r["p"]) - g_h[:, None] * r["p"] * (logp + r["h"][:, None])
    live = r["ok"] & np.isfinite(r["lse"])
    g = np.where(live[:, None], g / tau, 0.0)
    # what each step of the kernel may round: the exponent of p, then a handful of products and sums
    size = (r["p"] * (np.abs(g_lp)[:, None] + np.abs(g_h)[:, None] * (np.abs(logp) + r["h"][:, None])) + hot * np.abs(g_lp)[:, None]) / tau
    expo = np.abs(np.where(np.isfinite(x), x, 0) / tau) + 2 * np.abs(logp) + np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0))[:, None] + 16
    return np.where(live[:, None], g, 0.0), size * expo * U


def run_grad(x, tok, tau, entropy=True, out=None, seed=0):
    from paper_2511_14617_amd import binding
    g = torch.Generator(device="cuda").manual_seed(seed)
    lead = tuple(x.shape[:-1])
    g_lp = torch.randn(lead, device="cuda", generator=g)
    g_h = torch.randn(lead, device="cuda", generator=g) if entropy else None
    xs = x.double().cpu().numpy().reshape(-1, x.shape[-1])
    toks = tok.cpu().numpy().reshape(-1)
    f = binding.seer_token_logprobs(x, tok, temperature=tau)
    want, tol = grad_reference(xs, toks, float(np.float32(tau)), g_lp.double().cpu().numpy().reshape(-1),
                               g_h.double().cpu().numpy().reshape(-1) if entropy else np.zeros(len(xs)))
    got = binding.seer_token_logprobs_grad(x, tok, f[2], g_lp, entropy=f[1] if entropy else None, grad_entropy=g_h, temperature=tau, out=out)
    torch.cuda.synchronize()
    half = 2.0 ** -8 if x.dtype == torch.bfloat16 else U
    # (logsumexp and entropy come from the forward call: 128 u, as derived above, times p's share)
    err = np.abs(got.double().cpu().numpy().reshape(want.shape) - want)
    bound = tol + 160 * tol / 16 + half * (np.abs(want) + tol) + 1e-38 + (2.0 ** -134 if half > U else 0)
    assert (err <= bound).all(), float((err - bound).max())
    return got


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(1, 1), (3, 2), (5, 41), (2, 4096), (3, 4099), (2, 50257), (2100, 130), (1, 152067)])
@pytest.mark.parametrize("entropy", [True, False])
def test_gradient(N, V, entropy, dtype):
    x, tok = make(N, V, dtype, N * 7 + V, pad=3)
    if N > 2:
        tok[1] = -1
    run_grad(x, tok, 0.8, entropy)


@pytest.mark.parametrize("dtype", DT, ids=["f32", "bf16"])
def test_gradient_of_masked_rows_strided_outputs_and_in_place(dtype):
    x, tok = make(7, 1003, dtype, 5, pad=9)
    x[0] = -float("inf")
    x[1, 4:] = -float("inf")
    x[2, :] = -float("inf")
    x[2, 77] = 1.0
    tok[1], tok[2] = 2, 77
    want = run_grad(x, tok, 1.0)
    room = torch.full((7, 1100), 3.0, device="cuda", dtype=dtype)
    run_grad(x, tok, 1.0, out=room[:, 20:1023])
    assert torch.equal(room[:, 20:1023], want) and (room[:, :20] == 3).all() and (room[:, 1023:] == 3).all()
    x3 = x.clone().contiguous().view(7, 1, 1003)
    assert torch.equal(run_grad(x3, tok.view(7, 1), 1.0)[:, 0], want)
    same = x.clone()
    assert torch.equal(run_grad(same, tok, 1.0, out=same), want)


def test_gradient_against_differences_of_the_definition():
    """Central differences of the 64-bit definition at step h: they differ from the derivative by at most h^2 times a bound on the third
    derivative (here below 8 of any coefficient) plus rounding of the sums, 1e-16 * 10 / h."""
    x, tok = make(3, 29, torch.float32, 13)
    got = run_grad(x, tok, 0.8, True, seed=4).double().cpu().numpy()
    g = torch.Generator(device="cuda").manual_seed(4)
    g_lp, g_h = (torch.randn(3, device="cuda", generator=g).double().cpu().numpy() for _ in range(2))
    xs, toks, h = x.double().cpu().numpy(), tok.cpu().numpy(), 1e-4

    def loss(v):
        r = reference(v, toks, float(np.float32(0.8)), 1)
        return (g_lp * r["pick"] + g_h * r["h"]).sum()

    for r in range(3):
        for v in range(29):
            up, down = xs.copy(), xs.copy()
            up[r, v] += h
            down[r, v] -= h
            assert abs((loss(up) - loss(down)) / (2 * h) - got[r, v]) < 8 * 2 * h * h * 10 + 1e-11 + 400 * U * (abs(g_lp[r]) + 4 * abs(g_h[r]))


def test_gradient_of_one_of_the_two_alone_is_the_sum_s_part():
    from paper_2511_14617_amd import binding
    x, tok = make(4, 999, torch.float32, 2)
    lp, h, lse, _, _ = binding.seer_token_logprobs(x, tok)
    g = torch.ones(4, device="cuda")
    zero = torch.zeros(4, device="cuda")
    a = binding.seer_token_logprobs_grad(x, tok, lse, None, entropy=h, grad_entropy=g)
    b = binding.seer_token_logprobs_grad(x, tok, lse, zero, entropy=h, grad_entropy=g)
    assert torch.equal(a, b)
    assert (binding.seer_token_logprobs_grad(x, tok, lse, None) == 0).all()


# ------------------------------------------------------------------------------------------------
# streams, graphs, refusals of the binding
# ------------------------------------------------------------------------------------------------
def test_other_stream_and_dirty_workspace():
    from paper_2511_14617_amd import binding
    x, tok = make(12, 9001, torch.float32, 21)
    want = binding.seer_token_logprobs(x, tok, top_n=8)
    ws = torch.full((binding.seer_token_logprobs_workspace(binding.logprob_params(x, 1.0, 8)),), 0xA5, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.seer_token_logprobs(x, tok, top_n=8, workspace=ws, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_recorded_in_a_graph_and_replayed_with_other_logits():
    from paper_2511_14617_amd import binding
    x, tok = make(20, 5003, torch.bfloat16, 22)
    own = x.clone()
    p = binding.logprob_params(x, 1.0, 6)
    ws = torch.empty(binding.seer_token_logprobs_workspace(p), dtype=torch.uint8, device="cuda")
    grad = torch.empty_like(x)
    g = torch.ones(20, device="cuda")

    def step(logits, out):
        f = binding.seer_token_logprobs(logits, tok, top_n=6, workspace=ws, out=out)
        binding.seer_token_logprobs_grad(logits, tok, f[2], g, entropy=f[1], grad_entropy=g, out=grad)

    def buffers():
        return tuple(torch.zeros(20, device="cuda") for _ in range(3)) + (torch.zeros((20, 6), device="cuda"), torch.zeros((20, 6), dtype=torch.int32, device="cuda"))

    eager, graphed = buffers(), buffers()
    step(x, eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(own, graphed)
    for replay in range(4):
        now = torch.roll(x, replay, 1)
        step(now, eager)
        want = grad.clone()
        own.copy_(now)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(graphed, eager)), replay
        assert torch.equal(grad, want), replay


def test_the_same_call_twice_gives_the_same_bits():
    from paper_2511_14617_amd import binding
    x, tok = make(40, 30011, torch.float32, 23)
    a, b = (binding.seer_token_logprobs(x, tok, top_n=32) for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_binding_refuses_what_it_cannot_marshal():
    from paper_2511_14617_amd import binding
    x, tok = make(4, 64, torch.float32, 1)
    for bad in (x.half(), x.cpu(), x.t(), x[:, ::2], x[0]):
        with pytest.raises(ValueError):
            binding.seer_token_logprobs(bad, tok)
    with pytest.raises(ValueError):
        binding.seer_token_logprobs(x, tok.long())
    with pytest.raises(ValueError):
        binding.seer_token_logprobs(x, tok, tok[:3])
    with pytest.raises(ValueError):
        binding.seer_token_logprobs_grad(x, tok, torch.zeros(4, device="cuda"), None, out=x.bfloat16())
    for kw in (dict(top_n=33), dict(temperature=0.0), dict(top_n=-1)):
        with pytest.raises(binding.SeerError):
            binding.seer_token_logprobs(x, tok, **kw)
    with pytest.raises(binding.SeerError):
        binding.seer_token_logprobs_grad(x, tok, torch.zeros(4, device="cuda"), None, grad_entropy=torch.zeros(4, device="cuda"))

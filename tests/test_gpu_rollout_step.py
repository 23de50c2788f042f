"""The calls of a decoding step in the order in which a rollout makes them, on two layers: attention, acceptance, commit, log probabilities of the emitted
tokens, attention weights, eviction, and the next step on the cache that is left.

Beside the pools a plain list of K and V rows per layer, request and head goes along; the attention of every accepted row is held against it (to the bar of
the attention tests), the pools exactly.  Log probabilities and weights are held against their definitions in 64 bits, eviction against its rule, and the
step's own outputs have the same bits as those checked calls.  A captured step gives the same bits as an eager one."""
import numpy as np
import pytest
import torch

from gpu_util import check_attention_values
from test_gpu_kv_evict import check as check_evict
from test_gpu_kv_weights import check as check_weights
from test_gpu_token_logprobs import check as check_logprobs

pytestmark = pytest.mark.gpu
LAYERS, TOP_N = 2, 4


class Rollout:
    def __init__(self, B, T, Hq, Hkv, D, P, V, start, seed, parent=None, latent_Dv=0, tau=None, limit=96, budget=64, first=5, last=20):
        self.rng, self.g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
        self.B, self.T, self.Hq, self.Hkv, self.D, self.P, self.V = B, T, Hq, Hkv, D, P, V
        self.Dv, self.latent, self.tau, self.scale = latent_Dv or D, latent_Dv > 0, tau, D ** -0.5
        self.limit, self.budget, self.last = limit, budget, last
        pages = -(-(max(limit, max(start)) + T) // P)
        total = B * pages + 3
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.table = dev(self.rng.permutation(total)[:B * pages].reshape(B, pages).astype(np.int32))
        self.first = dev(np.minimum(np.arange(B) + first, budget - last).astype(np.int32))
        self.ctx = dev(np.asarray(start, np.int32))
        self.k = [self.random(total, Hkv, P, D) for _ in range(LAYERS)]
        self.v = [None if self.latent else self.random(total, Hkv, P, self.Dv) for _ in range(LAYERS)]
        self.w = [torch.rand((B, Hkv, pages * P), device="cuda", generator=self.g) for _ in range(LAYERS)]
        self.parent, self.mask = None, None
        if parent is not None:
            bits = [1]
            for t in range(1, T):
                bits.append(bits[parent[t]] | 1 << t)
            self.parent = dev(np.tile(np.asarray(parent, np.int32), (B, 1)))
            self.mask = dev(np.tile(np.asarray(bits, np.int64), (B, 1)))
        self.up = parent if parent is not None else list(range(-1, T - 1))
        self.seed = 1234
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        # what the model gives a step
        self.q = [self.random(B, T, Hq, D) for _ in range(LAYERS)]
        self.nk = [self.random(B, T, Hkv, D) for _ in range(LAYERS)]
        self.nv = [None if self.latent else self.random(B, T, Hkv, self.Dv) for _ in range(LAYERS)]
        self.logits = torch.empty((B, T, V), device="cuda")
        self.draft = torch.empty((B, T), dtype=torch.int32, device="cuda")

    def random(self, *shape):
        return torch.randn(shape, device="cuda", generator=self.g).to(torch.bfloat16)

    def model(self):
        """New queries, K/V rows, logits and drafts, a part of which agrees with the logits."""
        for x in self.q + self.nk + [t for t in self.nv if t is not None]:
            x.copy_(self.random(*x.shape))
        x = torch.randn(self.logits.shape, device="cuda", generator=self.g) * 2
        best = torch.randint(0, self.V, (self.B, self.T), device="cuda", generator=self.g)
        x.scatter_(2, best[..., None], 30.0)
        self.logits.copy_(x)
        draft, target = self.rng.integers(0, self.V, (self.B, self.T)).astype(np.int32), best.cpu().numpy()
        for b in range(self.B):
            for t in range(1, self.T):
                if self.rng.random() < 0.8:
                    draft[b, t] = target[b, self.up[t]]
        self.draft.copy_(torch.from_numpy(draft))

    def step(self, seen=None):
        from paper_2511_14617_amd import binding as sv
        at = self.ctx[:, None].long() + torch.arange(self.T, device="cuda")
        page, row = torch.gather(self.table.long(), 1, at // self.P), at % self.P
        for i in range(LAYERS):
            self.k[i][page, :, row] = self.nk[i]
            if not self.latent:
                self.v[i][page, :, row] = self.nv[i]
        self.ctx.add_(self.T)
        out = [sv.seer_verify_attention(self.q[i], self.k[i], self.v[i], self.table, self.ctx, self.mask, self.scale, Dv=self.Dv if self.latent else None)
               for i in range(LAYERS)]
        if self.tau is None:
            alen, path, bonus, _ = sv.seer_accept(self.logits, self.draft, self.parent)
        else:
            alen, path, bonus, _ = sv.seer_accept_sampled(self.logits, self.draft, self.parent, self.tau, self.seed)
        for i in range(LAYERS):                             # (each commit moves the length it is given: the last one keeps it)
            n = self.ctx if i == LAYERS - 1 else self.ctx.clone()
            emitted, count = sv.seer_kv_commit(self.k[i], self.v[i], self.table, n, alen, path, draft_tokens=self.draft, bonus_token=bonus, status=self.status)
        lp = sv.seer_token_logprobs(self.logits, emitted, path, temperature=self.tau or 1.0, top_n=TOP_N)
        before = [w.clone() for w in self.w]
        for i in range(LAYERS):
            sv.seer_kv_weights(self.w[i], self.q[i], self.k[i], self.table, self.ctx, alen, path, self.scale, decay=0.75, status=self.status)
        if seen is not None:
            seen.update(n=self.ctx.clone(), k=[t.clone() for t in self.k], v=[None if t is None else t.clone() for t in self.v], w=[t.clone() for t in self.w],
                        before=before)
        kept = []
        for i in range(LAYERS):                             # (the lengths are the same for all layers: the last one moves them)
            n = self.ctx if i == LAYERS - 1 else torch.empty_like(self.ctx)
            kept.append(sv.seer_kv_evict(self.k[i], self.v[i], self.table, self.ctx, self.w[i], limit=self.limit, budget=self.budget, keep_first=self.first,
                                         keep_last=self.last, new_weights=self.w[i], new_ctx_len=n, status=self.status)[1])
        return dict(out=out, alen=alen, path=path, emitted=emitted, count=count, lp=lp, kept=kept)

    def rows(self, i, b, n):
        """The first n K and V rows of a request in layer i, [Hkv, n, D] float64."""
        at = np.arange(n)
        page, row = self.table[b].cpu().long()[at // self.P], torch.from_numpy(at % self.P)
        pick = lambda t: t.cpu()[page, :, row].double().transpose(0, 1).numpy()
        k = pick(self.k[i])
        return k, k[..., :self.Dv] if self.latent else pick(self.v[i])


TREE = [-1, 0, 1, 2, 0, 4, 5]
SETUPS = {
    "chain": dict(B=5, T=5, Hq=8, Hkv=2, D=128, P=16, V=1003, start=[1, 40, 90, 96, 77], seed=1),
    "tree_sampled": dict(B=4, T=7, Hq=8, Hkv=2, D=128, P=20, V=5003, start=[30, 95, 96, 60], seed=2, parent=TREE, tau=0.8),
    "latent": dict(B=3, T=4, Hq=16, Hkv=1, D=576, P=64, V=257, start=[100, 1, 96], seed=3, latent_Dv=512),
    "long": dict(B=3, T=4, Hq=6, Hkv=2, D=64, P=16, V=4099, start=[700, 600, 590], seed=4, limit=600, budget=560, first=16, last=64),
}


@pytest.mark.parametrize("name", sorted(SETUPS))
def test_a_rollout_on_the_cache_that_is_left(name):
    r = Rollout(**SETUPS[name])
    B, G = r.B, r.Hq // r.Hkv
    plain = [[r.rows(i, b, int(r.ctx[b])) for b in range(B)] for i in range(LAYERS)]
    dropped = accepted = 0
    for _ in range(5):
        r.model()
        seen = {}
        got = r.step(seen)
        torch.cuda.synchronize()
        assert r.status.item() == 0
        alen, path, emitted, count = (got[x].cpu().numpy() for x in ("alen", "path", "emitted", "count"))
        accepted += int(alen.sum())
        assert np.array_equal(count, alen + 1) and all((emitted[b, :count[b]] >= 0).all() for b in range(B))
        want, have, size = [], [], []
        for i in range(LAYERS):
            q, out = r.q[i].double().cpu().numpy(), got["out"][i].double().cpu().numpy()
            nk = r.nk[i].double().cpu().numpy()
            nv = nk[..., :r.Dv] if r.latent else r.nv[i].double().cpu().numpy()
            for b in range(B):
                slots = path[b, :alen[b] + 1]
                k, v = (np.concatenate([old, new[b, slots].transpose(1, 0, 2)], 1) for old, new in zip(plain[i][b], (nk, nv)))
                for x, slot in enumerate(slots):
                    see = k.shape[1] - len(slots) + x + 1
                    s = q[b, slot].reshape(r.Hkv, G, r.D) @ k[:, :see].transpose(0, 2, 1) * r.scale
                    p = np.exp(s - s.max(2, keepdims=True))
                    p /= p.sum(2, keepdims=True)
                    want.append((p @ v[:, :see]).reshape(r.Hq, r.Dv))
                    size.append((p @ np.abs(v[:, :see])).reshape(r.Hq, r.Dv))
                    have.append(out[b, slot])
                plain[i][b] = (k, v)
                assert int(seen["n"][b]) == k.shape[1]
        # (Values of |v| = 3 where one of a few tokens has the weight: the rounding of the probabilities to bf16, 2^-8 of each at most, is worth up to
        # 2^-8 sum p |v| = 0.012 there, six times the constant of the plain bar.  The sum of magnitudes goes along, as for the other inputs with outputs of that size.)
        check_attention_values(np.stack(have), np.stack(want), name, ref_abs=np.stack(size))
        again = check_logprobs(r.logits, got["emitted"], r.tau or 1.0, TOP_N, got["path"])
        assert all(torch.equal(x, y) for x, y in zip(got["lp"], again))
        for i in range(LAYERS):
            s = dict(w=seen["before"][i], q=r.q[i], k=seen["k"][i], table=r.table, ctx=seen["n"], alen=got["alen"], path=got["path"], scale=r.scale)
            assert torch.equal(check_weights(s, 0.75), seen["w"][i])
            s = dict(k=seen["k"][i], v=seen["v"][i], table=r.table, ctx=seen["n"], w=seen["w"][i])
            k, v, w = check_evict(s, r.limit, r.budget, r.first.cpu().numpy(), r.last)
            assert torch.equal(k, r.k[i]) and torch.equal(w, r.w[i]) and (r.latent or torch.equal(v, r.v[i]))
            kept = got["kept"][i].cpu().numpy()
            for b in range(B):
                n = int(r.ctx[b])
                if int(seen["n"][b]) > r.limit:
                    dropped += 1
                    assert n == r.budget
                    plain[i][b] = tuple(np.stack([x[h, kept[b, h]] for h in range(r.Hkv)]) for x in plain[i][b])
                assert all(np.array_equal(x, y) for x, y in zip(plain[i][b], r.rows(i, b, n)))
    # (a step adds a position at least, so that every request that starts within 4 of the limit is cut in each layer: one of them in every setup)
    assert dropped >= LAYERS and accepted > 8


@pytest.mark.parametrize("name", ["tree_sampled", "latent", "long"])
def test_a_captured_step_gives_the_bits_of_an_eager_one(name):
    a, b = Rollout(**SETUPS[name]), Rollout(**SETUPS[name])
    for r in (a, b):
        r.model()
        r.step()                                            # (before the capture: loads the kernels)
    torch.cuda.synchronize()
    held = [t.clone() for t in b.k + [x for x in b.v if x is not None] + b.w + [b.ctx]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = b.step()
    assert all(torch.equal(x, y) for x, y in zip(held, b.k + [x for x in b.v if x is not None] + b.w + [b.ctx]))       # (captured, not run)
    for _ in range(4):
        a.model()
        b.model()
        want = a.step()
        graph.replay()
        torch.cuda.synchronize()
        flat = lambda d: [t for x in ("out", "lp", "kept") for t in d[x]] + [d[x] for x in ("alen", "path", "emitted", "count")]
        assert all(torch.equal(x, y) for x, y in zip(flat(want), flat(res)))
        for x, y in zip(a.k + a.v + a.w + [a.ctx, a.status], b.k + b.v + b.w + [b.ctx, b.status]):
            assert x is None or torch.equal(x, y)
    assert a.status.item() == 0


def test_memory_of_a_call_on_another_stream_is_that_stream_s():
    """A call on a busy stream, then work of the current stream on memory that the allocator hands out there: neither finds the other's data in its own."""
    from paper_2511_14617_amd import binding as sv
    logits = torch.randn((6, 70000), device="cuda")
    tokens = torch.arange(6, device="cuda", dtype=torch.int32)
    r = Rollout(**SETUPS["long"])
    r.model()

    held = []

    def calls(stream):
        lp = sv.seer_token_logprobs(logits, tokens, top_n=20, stream=stream)
        w, k, v = [t.clone() for t in r.w], r.k[1].clone(), r.v[1].clone()
        held.extend([*w, k, v])                             # (the caller's own memory is the caller's to keep)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        sv.seer_kv_weights(w[0], r.q[0], r.k[0], r.table, r.ctx, None, None, r.scale, stream=stream)
        n, kept = sv.seer_kv_evict(k, v, r.table, r.ctx, w[1], limit=550, budget=500, stream=stream)
        return [*lp, w[0], n, kept]

    want = calls(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = calls(side)
    junk = [torch.full((size,), 0x7FC07FC0, dtype=torch.int32, device="cuda") for size in (64, 1 << 10, 1 << 12, 1 << 14, 1 << 16, 1 << 18) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and all((t == 0x7FC07FC0).all() for t in junk)

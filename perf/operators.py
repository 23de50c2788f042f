"""The operators around a verification step that record what was sampled and keep the cache small, as cases that can be
timed and compared.

Kinds of case
  logprob  log probability of given tokens under the target's logits, entropy and the most probable alternatives of each row:
           what a rollout stores beside its tokens, what scoring a batch of responses computes
  grad     the gradient of those log probabilities and entropies with respect to the logits
  weights  attention weight that the accepted tokens of a step gave to every cached position, added to the running sums
  evict    the cached positions with the smallest sums leave the cache, the others are kept in `budget` slots

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` computes the operator with
elementary torch operations, or with the framework's calls where `own` is set.  Context lengths, accepted lengths and lengths of
common prefixes are quantiles of a stated distribution, so a case has the same work whatever the seed; which request has
which, the page order and all values come from the seed.
"""
from __future__ import annotations

import math
from statistics import NormalDist

import numpy as np
import torch

own = False

SCORE_STD = 1.5      # standard deviation of scaled scores: some hundred tokens of a context carry the weight


def _logprob(name, B, T, V, dtype, top_n, temperature=1.0, path=False, pad=0):
    return {"name": name, "kind": "logprob", "B": B, "T": T, "V": V, "pad": pad, "dtype": dtype, "top_n": top_n,
            "temperature": temperature, "path": path}


def _grad(name, B, V, dtype, temperature=1.0, entropy=True, pad=0):
    return {"name": name, "kind": "grad", "B": B, "T": 1, "V": V, "pad": pad, "dtype": dtype, "temperature": temperature,
            "entropy": entropy}


def _weights(name, B, T, Hq, Hkv, D, page, lo, mid, hi, decay=1.0, path=True):
    return {"name": name, "kind": "weights", "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "lo": lo, "mid": mid,
            "hi": hi, "decay": decay, "path": path}


def _evict(name, B, Hkv, D, Dv, page, lo, mid, hi, limit, budget, first, last):
    return {"name": name, "kind": "evict", "B": B, "Hkv": Hkv, "D": D, "Dv": Dv, "page": page, "lo": lo, "mid": mid, "hi": hi,
            "limit": limit, "budget": budget, "first": first, "last": last}


def listed():
    return [
        # one request that decodes by itself and reports its 20 most probable tokens: launches and latency
        _logprob("logprob_one_token", 1, 1, 152064, "float32", 20),
        # the emitted tokens of a grouped rollout's verify step, with five alternatives each, at the sampling temperature
        _logprob("logprob_verify_step", 64, 9, 152064, "float32", 5, 0.8, path=True),
        # a small model's odd vocabulary, rows that begin at any alignment, the most probable token beside each
        _logprob("logprob_odd_vocabulary", 1023, 1, 50257, "bfloat16", 1, 1.0),
        # responses scored for a training step: log probabilities and entropies of 4096 tokens
        _logprob("logprob_training", 4096, 1, 151936, "bfloat16", 0, 1.0, pad=128),
        # the gradient of a short response on a small vocabulary, with the entropy's
        _grad("grad_short", 16, 32003, "float32", 0.8),
        # the gradient of 4096 tokens of a training step
        _grad("grad_training", 4096, 152064, "bfloat16", 1.0),
        # a handful of short requests after a verify step
        _weights("weights_tiny", 4, 5, 8, 2, 128, 16, 64, 256, 512),
        # plain decoding of a grouped rollout, one token a step, sums that fade
        _weights("weights_decode", 64, 1, 32, 8, 128, 16, 512, 4096, 32768, decay=0.98, path=False),
        # the accepted tokens of a verify step, one GPU's share of a dense 72B-class model under 8-way tensor parallelism
        _weights("weights_verify", 64, 9, 8, 1, 128, 16, 512, 4096, 32768),
        # all heads of a large MoE model over the shared latent, the accepted tokens of a verify step
        _weights("weights_latent", 16, 5, 128, 1, 576, 64, 8192, 14000, 24576),
        # every request a few tokens over its limit: the step that rollouts of bounded memory make again and again
        _evict("evict_each_step", 64, 8, 128, 128, 16, 4160, 4224, 4352, 4128, 4096, 512, 64),
        # the long tail of a rollout, cut to an eighth
        _evict("evict_long_tail", 8, 8, 128, 128, 16, 65536, 98304, 131072, 32768, 12288, 512, 256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprob", "logprob", "grad", "weights", "weights", "weights", "evict", "evict"])
    while True:
        if kind in ("logprob", "grad"):
            V = rng.choice([1024, 32000, 50257, 128256, 151936, 152064, 163840, _log_int(rng, 40, 163840)]) + rng.choice([0, 0, 3])
            dtype, temperature, pad = rng.choice(["float32", "bfloat16"]), rng.choice([0.6, 0.8, 1.0, 1.0, 1.3]), rng.choice([0, 0, 64, 7])
            if kind == "grad":
                c = _grad("", _log_int(rng, 1, 4096), V, dtype, temperature, rng.random() < 0.6, pad)
            else:
                path = rng.random() < 0.5
                T = rng.randint(2, 33) if path else 1
                c = _logprob("", _log_int(rng, 1, 256 if path else 4096), T, V, dtype, min(V, rng.choice([0, 0, 1, 5, 8, 20, 32])), temperature, path, pad)
            # (the plain form's indices and sorted keys take eight bytes a logit)
            fits = c["B"] * c["T"] * V * (4 if c.get("top_n") else 1) <= 4096 * 152064
        elif kind == "weights":
            D, Hkv, G = rng.choice([(128, 8, 4), (128, 1, 8), (128, 2, 4), (128, 4, 5), (128, 8, 1), (64, 4, 4), (256, 1, 8), (192, 2, 8),
                                    (576, 1, 16), (576, 1, 128)])
            mid = _log_int(rng, 64, 32768)
            T = rng.choice([1, 1, 2, 5, 9, 17])
            c = _weights("", _log_int(rng, 1, 128), T, Hkv * G, Hkv, D, rng.choice([16, 16, 20, 32, 64, 128]), max(T, mid // 8), mid, mid * 4,
                         rng.choice([1.0, 1.0, 0.95]), T > 1 and rng.random() < 0.8)
            # (the plain form lays all requests out to the longest one's length)
            slots = c["B"] * Hkv * mid * 4
            fits = slots * D <= 64 * 8 * 32768 * 128 and slots * T * G <= 5e8 and work(c)["flops"] <= 8.4e10
        else:
            D, Dv = rng.choice([(128, 128), (128, 128), (64, 64), (256, 256), (192, 128), (576, 0)])
            mid = _log_int(rng, 128, 65536)
            budget = max(64, int(mid * rng.uniform(0.1, 0.98)))
            last = rng.randint(0, budget // 4)
            c = _evict("", _log_int(rng, 1, 64), 1 if D == 576 else rng.choice([1, 2, 4, 8]), D, Dv, rng.choice([16, 16, 20, 32, 64, 128]), max(1, mid // 3), mid, mid * 2,
                       budget + rng.choice([0, 0, 32, budget // 8]), budget, rng.randint(0, budget // 3), last)
            fits = c["B"] * c["Hkv"] * mid * 2 * (D + Dv) <= 8 * 8 * 131072 * 256
        if fits:
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------
# what a case's numbers stand for
# ------------------------------------------------------------------------------------------------
def _lengths(c):
    """Context lengths, ascending: B quantiles of a lognormal distribution (sigma 0.8) between lo and hi."""
    n = [min(max(c["mid"] * math.exp(0.8 * NormalDist().inv_cdf((i + 0.5) / c["B"])), c["lo"]), c["hi"]) for i in range(c["B"])]
    return np.maximum(np.rint(np.asarray(n)), c.get("T", 1)).astype(np.int64)


def _accepted(c):
    """Accepted draft tokens of a step, ascending: a third of them on average."""
    return np.asarray([min(c["T"] - 1, int(c["T"] * ((b + 0.5) / c["B"]) ** 2)) for b in range(c["B"])], dtype=np.int64)


def _rows(c):
    """Query rows (accepted tokens and the root) of each request, ascending; all slots without a path."""
    return _accepted(c) + 1 if c["path"] else np.full(c["B"], c["T"], dtype=np.int64)


def _first(c):
    """Lengths of the common prefix that stays whatever its sums: between half of `first` and `first`."""
    return np.asarray([c["first"] - (b % 4) * (c["first"] // 8) for b in range(c["B"])], dtype=np.int64)


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _paths(c, rng):
    """(accepted_len, accepted_path): ascending slots of the accepted path from the root, then -1."""
    alen = rng.permutation(_accepted(c))
    path = np.full((c["B"], c["T"]), -1, dtype=np.int64)
    for b, a in enumerate(alen):
        path[b, 0] = 0
        path[b, 1:a + 1] = 1 + np.sort(rng.permutation(c["T"] - 1)[:a])
    return _i32(alen), _i32(path)


def _pool(c, rng, gen, widths):
    """Block table of random pages and one pool [pages, Hkv, page, D] per width."""
    ctx = rng.permutation(_lengths(c))
    need = -(-ctx // c["page"])
    table = np.zeros((c["B"], int(need.max())), dtype=np.int64)
    total = int(need.sum()) + 3
    ids, at = rng.permutation(total), 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    pools = [torch.randn((total, c["Hkv"], c["page"], d), dtype=torch.bfloat16, device="cuda", generator=gen) if d else None for d in widths]
    return _i32(ctx), _i32(table), pools


def prepare(case, seed):
    c, rng, gen = case, np.random.default_rng([seed, 9]), _generator(seed)
    s = {"case": c}
    if c["kind"] in ("logprob", "grad"):
        B, T, V, dtype = c["B"], c["T"], c["V"], getattr(torch, c["dtype"])
        store = torch.randn((B, T, V + c["pad"]), dtype=dtype, device="cuda", generator=gen).mul_(2.0)
        s["logits"] = store[:, :, :V]
        # the sampled tokens are mostly among the probable ones; a few rows have none (padding)
        s["tokens"] = torch.randint(0, V, (B, T), device="cuda", generator=gen, dtype=torch.int32)
        at = torch.randint(0, V, (B, T, 1), device="cuda", generator=gen)
        s["logits"].scatter_(2, at, (9.0 + 3.0 * torch.rand((B, T, 1), device="cuda", generator=gen)).to(dtype))
        likely = torch.rand((B, T), device="cuda", generator=gen) < 0.7
        s["tokens"] = torch.where(likely, at[:, :, 0].int(), s["tokens"])
        if B * T >= 16:
            s["tokens"].view(-1)[:: 16] = -1
        if c["kind"] == "grad":
            s["logits"], s["tokens"] = s["logits"].reshape(B, -1) if not c["pad"] else s["logits"][:, 0], s["tokens"][:, 0].contiguous()
            z = s["logits"].float() / c["temperature"]
            m = z.amax(1)
            e = torch.exp(z - m[:, None])
            total = e.sum(1)
            s["logsumexp"] = m + torch.log(total)
            s["entropy"] = torch.log(total) - (e * (z - m[:, None])).sum(1) / total
            del z, e
            # policy-gradient coefficients: advantages over the number of tokens, and a small entropy bonus
            s["grad_logprob"] = torch.randn(B, device="cuda", generator=gen) / B
            s["grad_entropy"] = torch.full((B,), 0.01 / B, device="cuda") if c["entropy"] else None
        elif c["path"]:
            _, s["path"] = _paths(c, rng)
            s["tokens"] = torch.where(s["path"] >= 0, s["tokens"].clamp(min=0), -1)
        else:
            s["path"] = None
            s["logits"], s["tokens"] = (s["logits"][:, 0], s["tokens"][:, 0].contiguous())
    elif c["kind"] == "weights":
        s["ctx"], s["table"], (s["k"],) = _pool(c, rng, gen, (c["D"],))
        s["q"] = torch.randn((c["B"], c["T"], c["Hq"], c["D"]), dtype=torch.bfloat16, device="cuda", generator=gen).mul_(SCORE_STD)
        s["alen"], s["path"] = _paths(c, rng) if c["path"] else (None, None)
        s["scale"] = c["D"] ** -0.5
        s["weights"] = torch.rand((c["B"], c["Hkv"], s["table"].shape[1] * c["page"]), device="cuda", generator=gen)
    else:
        s["ctx"], s["table"], (s["k"], s["v"]) = _pool(c, rng, gen, (c["D"], c["Dv"]))
        # sums of attention weights: heavy-tailed, with positions that nothing ever looked at
        w = torch.randn((c["B"], c["Hkv"], s["table"].shape[1] * c["page"]), device="cuda", generator=gen).mul_(2.0).exp_()
        w[torch.rand(w.shape, device="cuda", generator=gen) < 0.05] = 0.0
        s["weights"], s["new_weights"] = w, torch.zeros_like(w)
        s["first"] = _i32(rng.permutation(_first(c)))
    return s


# ------------------------------------------------------------------------------------------------
# the calls
# ------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2511_14617_amd import binding
    c, kind = s["case"], s["case"]["kind"]
    if kind == "logprob":
        return binding.seer_token_logprobs(s["logits"], s["tokens"], s["path"], temperature=c["temperature"], top_n=c["top_n"])
    if kind == "grad":
        return binding.seer_token_logprobs_grad(s["logits"], s["tokens"], s["logsumexp"], s["grad_logprob"], entropy=s["entropy"],
                                                grad_entropy=s["grad_entropy"], temperature=c["temperature"])
    if kind == "weights":
        return binding.seer_kv_weights(s["weights"], s["q"], s["k"], s["table"], s["ctx"], s["alen"], s["path"], s["scale"],
                                       decay=c["decay"])
    lens, kept = binding.seer_kv_evict(s["k"], s["v"], s["table"], s["ctx"], s["weights"], limit=c["limit"], budget=c["budget"],
                                       keep_first=s["first"], keep_last=c["last"], new_weights=s["new_weights"])
    return [lens, kept, s["new_weights"], s["k"], s["v"]]


def _keys(x):
    """Whole numbers ordered as the values of the last dimension, equal ones by their index, the lowest first."""
    i = x.contiguous().view(torch.int32).long()
    i = torch.where(i < 0, -(i & 0x7FFFFFFF), i)
    low = torch.arange(x.shape[-1] - 1, -1, -1, device=x.device)
    return i * 2 ** 32 + low


def _plain_logprob(s):
    c, tokens = s["case"], s["tokens"]
    logits = s["logits"]
    if s["path"] is not None:
        logits = torch.gather(logits, 1, s["path"].clamp(min=0).long()[:, :, None].expand(-1, -1, c["V"]))
    valid = tokens >= 0
    z = logits.float() / c["temperature"]
    m = z.amax(-1)
    d = z - m[..., None]
    e = torch.exp(d)
    total = e.sum(-1)
    lse = m + torch.log(total)
    entropy = torch.log(total) - (e * d).sum(-1) / total
    logp = torch.gather(d, -1, tokens.clamp(min=0).long()[..., None])[..., 0] - torch.log(total)
    zero = torch.zeros_like(lse)
    out = [torch.where(valid, x, zero) for x in (logp, entropy, lse)]
    if not c["top_n"]:
        return out + [None, None]
    top = c["V"] - 1 - (torch.topk(_keys(logits.float()), c["top_n"], dim=-1).values & 0xFFFFFFFF)
    value = torch.gather(d, -1, top) - torch.log(total)[..., None]
    return out + [torch.where(valid[..., None], value, 0.0), torch.where(valid[..., None], top, -1).int()]


def _plain_grad(s):
    c = s["case"]
    logp = s["logits"].float() / c["temperature"] - s["logsumexp"][:, None]
    p = torch.exp(logp)
    g = -s["grad_logprob"][:, None] * p
    if s["grad_entropy"] is not None:
        g = g - s["grad_entropy"][:, None] * p * (logp + s["entropy"][:, None])
    g.scatter_add_(1, s["tokens"].clamp(min=0).long()[:, None], s["grad_logprob"][:, None])
    return torch.where((s["tokens"] >= 0)[:, None], g / c["temperature"], 0.0).to(s["logits"].dtype)


def _plain_weights(s):
    c, ctx = s["case"], s["ctx"].long()
    B, T, Hkv, D = c["B"], c["T"], c["Hkv"], c["D"]
    k = s["k"][s["table"].long()].permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D).float()
    if s["path"] is None:
        q, rows = s["q"].float(), torch.full_like(ctx, T)
    else:
        q = torch.gather(s["q"], 1, s["path"].clamp(min=0).long()[:, :, None, None].expand(-1, -1, c["Hq"], D)).float()
        rows = s["alen"].long() + 1
    q = q.reshape(B, T, Hkv, -1, D).permute(0, 2, 4, 1, 3).reshape(B, Hkv, D, -1)
    scores = torch.matmul(k, q).view(B, Hkv, k.shape[2], T, -1) * s["scale"]
    j, i = torch.arange(k.shape[2], device=k.device)[None, :, None], torch.arange(T, device=k.device)[None, None, :]
    seen = (j <= (ctx - rows)[:, None, None] + i) & (i < rows[:, None, None])
    scores = torch.where(seen[:, None, :, :, None], scores, -math.inf)
    m = scores.amax(2, keepdim=True)
    e = torch.exp(scores - torch.where(torch.isinf(m), 0.0, m))
    total = e.sum(2, keepdim=True)
    got = (e / torch.where(total > 0, total, 1.0)).sum((3, 4))
    j = j[:, :, 0][:, None]
    old = torch.where(j < (ctx - rows)[:, None, None], s["weights"] * c["decay"], 0.0)
    s["weights"].copy_(torch.where(j < ctx[:, None, None], old + got, s["weights"]))
    return s["weights"]


def _plain_evict(s):
    c, w, L = s["case"], s["weights"], s["weights"].shape[2]
    n, first = s["ctx"].long()[:, None, None], s["first"].long()[:, None, None]
    budget, last, end = c["budget"], c["last"], c["budget"] - c["last"]
    j = torch.arange(L, device=w.device).expand_as(w)
    cut = (n > c["limit"]).expand_as(w)
    middle = (j >= first) & (j < n - last)
    order = torch.argsort(torch.where(middle, _keys(w), -2 ** 63), dim=2, descending=True)
    rank = torch.empty_like(order).scatter_(2, order, j)
    keep = middle & (rank < end - first)
    hole, mover = (j >= first) & (j < end) & ~keep & cut, keep & (j >= end) & cut
    at = torch.where(mover, torch.cumsum(mover, 2) - 1, L)
    source = torch.zeros((*w.shape[:2], L + 1), dtype=torch.long, device=w.device).scatter_(2, at, j)
    moved = torch.gather(source, 2, (torch.cumsum(hole, 2) - 1).clamp(min=0))
    kept = torch.where(hole, moved, torch.where((j >= end) & cut, j + n - budget, j)).clamp(max=L - 1)
    inside = j < torch.where(cut, budget, n)
    s["new_weights"].copy_(torch.where(inside, torch.gather(w, 2, kept), s["new_weights"]))
    b, h, to = torch.nonzero(cut & inside & (kept != j), as_tuple=True)
    table, P = s["table"].long(), c["page"]
    at, to = kept[b, h, to], to
    for pool in (s["k"], s["v"]):
        if pool is not None:
            pool[table[b, to // P], h, to % P] = pool[table[b, at // P], h, at % P]
    short = torch.full((*w.shape[:2], budget), -1, dtype=torch.int32, device=w.device)
    width = min(budget, L)
    short[:, :, :width] = torch.where(cut, kept, -1)[:, :, :width].int()
    return [torch.where(s["ctx"] > c["limit"], budget, s["ctx"]).int(), short, s["new_weights"], s["k"], s["v"]]


def run(state):
    if own:
        return _own(state)
    return {"logprob": _plain_logprob, "grad": _plain_grad, "weights": _plain_weights, "evict": _plain_evict}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without, and what its outputs are in 64 bits
# ------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] in ("logprob", "grad"):
        size = 4 if c["dtype"] == "float32" else 2
        rows = c["B"] * c["T"]
        if c["kind"] == "grad":
            return {"bytes": (2 * size * c["V"] + 20) * rows, "flops": 8 * rows * c["V"]}
        read = int(_rows(c).sum()) if c["path"] else rows
        return {"bytes": read * c["V"] * size + rows * (16 + 8 * c["top_n"]), "flops": 5 * read * c["V"]}
    n = _lengths(c)
    if c["kind"] == "weights":
        r = np.sort(_rows(c))
        return {"bytes": int(n.sum()) * c["Hkv"] * (2 * c["D"] + 8) + int(r.sum()) * c["Hq"] * c["D"] * 2,
                "flops": 2 * c["D"] * c["Hq"] * int(round(float(n.mean()) * float(r.sum())))}
    total = 4 * int(n.sum()) * c["Hkv"]
    for length, first in zip(n, np.sort(_first(c))):
        total += 4 * c["Hkv"] * min(int(length), c["budget"])
        if length > c["limit"]:
            slots, middle = c["budget"] - c["last"] - first, length - c["last"] - first
            rows = slots * (middle - slots) / middle + c["last"]      # (every position as likely to stay as the next)
            total += c["Hkv"] * (4 * c["budget"] + rows * 4 * (c["D"] + c["Dv"]))
    return {"bytes": int(total), "flops": 4 * int(n.sum()) * c["Hkv"]}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "logprob":
        T, V, n = c["T"], c["V"], c["top_n"]
        flat, toks = s["logits"].reshape(-1, T, V), s["tokens"].reshape(-1, T)
        outs = [torch.zeros(toks.shape, dtype=torch.float64, device="cuda") for _ in range(3)]
        tops = [torch.zeros((*toks.shape, n), dtype=torch.float64, device="cuda"), torch.full((*toks.shape, n), -1, dtype=torch.int32, device="cuda")]
        step = max(1, (1 << 27) // (T * V))
        for b in range(0, flat.shape[0], step):
            slot = torch.arange(T, device="cuda").expand(toks[b:b + step].shape) if s["path"] is None else s["path"][b:b + step].long()
            bb, tt = torch.nonzero(toks[b:b + step] >= 0, as_tuple=True)
            z = flat[b + bb, slot[bb, tt]].double() / c["temperature"]
            lse = torch.logsumexp(z, 1)
            logp = z - lse[:, None]
            p = torch.exp(logp)
            outs[0][b + bb, tt] = logp[torch.arange(len(bb), device="cuda"), toks[b + bb, tt].long()]
            outs[1][b + bb, tt] = -(p * logp).sum(1)
            outs[2][b + bb, tt] = lse
            if n:
                index = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :n]
                tops[0][b + bb, tt] = torch.gather(logp, 1, index)
                tops[1][b + bb, tt] = index.int()
        shape = s["tokens"].shape
        return [x.reshape(shape) for x in outs] + ([x.reshape(*shape, n) for x in tops] if n else [None, None])
    if c["kind"] == "grad":
        out = torch.zeros((c["B"], c["V"]), dtype=torch.float64, device="cuda")
        for b in range(0, c["B"], 512):
            rows = torch.nonzero(s["tokens"][b:b + 512] >= 0)[:, 0] + b
            z = s["logits"][rows].double() / c["temperature"]
            logp = z - torch.logsumexp(z, 1, keepdim=True)
            p = torch.exp(logp)
            hot = torch.zeros_like(p)
            hot[torch.arange(len(rows), device="cuda"), s["tokens"][rows].long()] = 1.0
            g = s["grad_logprob"][rows].double()[:, None] * (hot - p)
            if s["grad_entropy"] is not None:
                h = -(p * logp).sum(1, keepdim=True)
                g -= s["grad_entropy"][rows].double()[:, None] * p * (logp + h)
            out[rows] = g / c["temperature"]
        return out
    P, table, ctx = c["page"], s["table"].long(), s["ctx"].tolist()
    if c["kind"] == "weights":
        out = s["weights"].double()
        for b in range(c["B"]):
            n = ctx[b]
            slots = list(range(c["T"])) if s["path"] is None else s["path"][b, :int(s["alen"][b]) + 1].tolist()
            k = s["k"][table[b, : -(-n // P)]].double().transpose(0, 1).reshape(c["Hkv"], -1, c["D"])[:, :n]
            got = torch.zeros((c["Hkv"], n), dtype=torch.float64, device="cuda")
            for i, slot in enumerate(slots):
                see = n - len(slots) + i + 1
                q = s["q"][b, slot].double().reshape(c["Hkv"], -1, c["D"])
                got[:, :see] += torch.softmax(torch.matmul(q, k[:, :see].transpose(1, 2).contiguous()) * s["scale"], -1).sum(1)
            old = n - len(slots)
            out[b, :, :old] = out[b, :, :old] * c["decay"] + got[:, :old]
            out[b, :, old:n] = got[:, old:]
        return out
    # evict: request by request and head by head, on lists of positions
    lens, kept = list(ctx), torch.full((c["B"], c["Hkv"], c["budget"]), -1, dtype=torch.int32, device="cuda")
    end, new, k, v = c["budget"] - c["last"], s["new_weights"], s["k"].clone(), None if s["v"] is None else s["v"].clone()
    for b, n in enumerate(ctx):
        if n <= c["limit"]:
            new[b, :, :n] = s["weights"][b, :, :n]
            continue
        first, lens[b] = int(s["first"][b]), c["budget"]
        for h in range(c["Hkv"]):
            w = s["weights"][b, h, first:n - c["last"]].double()
            chosen = torch.sort(torch.sort(w, descending=True, stable=True).indices[: end - first]).values + first
            stay, move = chosen[chosen < end], chosen[chosen >= end]
            slot = torch.arange(c["budget"], device="cuda")
            free = torch.ones(end, dtype=torch.bool, device="cuda")
            free[:first] = False
            free[stay] = False
            slot[:end][free] = move
            slot[end:] = torch.arange(n - c["last"], n, device="cuda")
            kept[b, h] = slot.int()
            new[b, h, : c["budget"]] = s["weights"][b, h, slot]
            to = torch.arange(c["budget"], device="cuda")
            k[table[b, to // P], h, to % P] = s["k"][table[b, slot // P], h, slot % P]
            if v is not None:
                v[table[b, to // P], h, to % P] = s["v"][table[b, slot // P], h, slot % P]
    return [torch.tensor(lens, dtype=torch.int32), kept, new, k, v]

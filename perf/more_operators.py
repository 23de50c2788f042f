"""The operators in front of the first verification step, which give requests their pages, write the rows of new tokens into
them and attend over whole prompts, as cases that can be timed and compared.

Kinds of case
  reserve    pages for the tokens that each request adds in a step (none, a few draft slots, a whole prompt), pages of finished
             requests back, leading pages of a prompt shared by its group, and for every new token its slot and its position
  append     rotation of the new tokens' queries and keys by their positions, keys and values into the slots of the paged cache
  attention  causal attention of the new tokens, packed sequence behind sequence, over each request's cache: whole prompts,
             pieces of prompts behind a cached beginning, single tokens among them

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` computes the operator with
elementary torch operations, or with the framework's calls where `own` is set.  Lengths are quantiles of a stated
distribution, so a case has the same work whatever the seed; which request has which, the page order and all values come from
the seed.
"""
from __future__ import annotations

import math
from statistics import NormalDist

import numpy as np
import torch

own = False

SCORE_STD = 1.5      # standard deviation of scaled scores: some hundred tokens of a context carry the weight
CHUNK = 1 << 28      # scores that the plain form holds at a time


def _reserve(name, B, page, pages, T, lo, mid, hi, group, turnover, tree=False, pad=0):
    return {"name": name, "kind": "reserve", "B": B, "page": page, "pages": pages, "T": T, "lo": lo, "mid": mid, "hi": hi,
            "group": group, "turnover": turnover, "tree": tree, "pad": pad}


def _append(name, N, Hq, Hkv, D, Dv, page, rotary, at, interleaved, far=32768, pad=0, fused=True):
    return {"name": name, "kind": "append", "N": N, "Hq": Hq, "Hkv": Hkv, "D": D, "Dv": Dv, "page": page, "rotary": rotary,
            "at": at, "interleaved": interleaved, "far": far, "pad": pad, "fused": fused}


def _attention(name, B, Hq, Hkv, D, Dv, page, lo, mid, hi, past=0, singles=0, pad=0):
    return {"name": name, "kind": "attention", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "Dv": Dv, "page": page, "lo": lo, "mid": mid,
            "hi": hi, "past": past, "singles": singles, "pad": pad}


def listed():
    return [
        # a verify step of a grouped rollout, nine slots of a draft tree a request: a third of the rows need a page; latency
        _reserve("reserve_verify_step", 64, 16, 16384, 9, 512, 2048, 8192, 8, 0.0, tree=True),
        # continuous batching of groups: an eighth of the responses is over, another eighth starts on its group's prompt
        _reserve("reserve_groups", 512, 16, 327680, 5, 256, 2048, 32768, 16, 0.25, pad=100),
        # whole prompts come and go, a pool of a million pages
        _reserve("reserve_prompts", 64, 16, 1048576, 1, 1024, 8192, 32768, 1, 1.0),
        # the rows of a verify step, all heads of a dense 72B-class model
        _append("append_verify_step", 576, 64, 8, 128, 128, 16, 128, 0, False, far=98304),
        # prompts of a group step, the same heads, out of one fused projection
        _append("append_prompts", 16384, 64, 8, 128, 128, 16, 128, 0, False, pad=37),
        # a piece of a prompt over the shared latent, whose last 64 components are rotated in pairs
        _append("append_latent", 4096, 128, 1, 576, 0, 64, 64, 512, True, fused=False),
        # short questions on one GPU's share of the heads: launches and latency
        _attention("attention_short_prompts", 8, 8, 2, 128, 128, 16, 17, 90, 300, pad=5),
        # prompts of mixed lengths, all heads of a dense 72B-class model
        _attention("attention_prompts", 16, 64, 8, 128, 128, 16, 256, 2048, 8192),
        # one very long prompt on one GPU's share under 8-way tensor parallelism
        _attention("attention_long_prompt", 1, 8, 1, 128, 128, 16, 32768, 32768, 32768),
        # a piece of a long prompt behind its cached beginning, in one batch with 63 requests that decode
        _attention("attention_piece_and_decodes", 64, 32, 8, 128, 128, 16, 2048, 2048, 2048, past=16384, singles=63),
        # prompts on a small model's heads, pages that are no power of two
        _attention("attention_small_heads", 12, 16, 4, 64, 64, 20, 100, 1500, 6000),
        # pieces of prompts over the shared latent, all heads of a large MoE model
        _attention("attention_latent", 4, 128, 1, 576, 512, 64, 256, 1024, 2048, past=512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["reserve", "reserve", "append", "append", "attention", "attention", "attention", "attention"])
    while True:
        if kind == "reserve":
            mid = _log_int(rng, 32, 8192)
            c = _reserve("", _log_int(rng, 1, 768), rng.choice([16, 16, 16, 20, 32, 64, 128]), _log_int(rng, 256, 1048576), rng.randint(1, 17),
                         max(1, mid // 8), mid, mid * 8, rng.choice([1, 4, 8, 16, 33]), rng.choice([0.0, 0.1, 0.25, 0.5, 1.0]),
                         rng.random() < 0.3, rng.choice([0, 0, 3, 100]))
            fits = c["B"] * min(mid * 3, c["hi"]) / c["page"] <= 400000 and c["B"] * c["hi"] / c["page"] <= 8e6 and work(c)["bytes"] <= 7.2e6
        elif kind == "append":
            D, Dv, rotary, at, Hkv, G = rng.choice([(128, 128, 128, 0, 8, 8), (128, 128, 128, 0, 1, 8), (128, 128, 64, 0, 2, 4), (64, 64, 64, 0, 4, 4),
                                                    (256, 256, 128, 0, 1, 8), (192, 128, 64, 128, 16, 1), (576, 0, 64, 512, 1, 16), (576, 0, 64, 512, 1, 128)])
            c = _append("", _log_int(rng, 1, 16384), Hkv * G, Hkv, D, Dv, rng.choice([16, 16, 20, 32, 64, 128]), rotary, at, rng.random() < 0.4,
                        _log_int(rng, 64, 1000000), rng.choice([0, 0, 37]), rng.random() < 0.5)
            fits = work(c)["bytes"] <= 1.2e9
        else:
            D, Dv, Hkv, G = rng.choice([(128, 128, 8, 8), (128, 128, 8, 4), (128, 128, 1, 8), (128, 128, 2, 4), (128, 128, 4, 5), (128, 128, 8, 1),
                                        (64, 64, 4, 4), (256, 256, 1, 8), (192, 128, 2, 8), (576, 512, 1, 16), (576, 512, 1, 128)])
            B, mid = _log_int(rng, 1, 64), _log_int(rng, 8, 16384)
            c = _attention("", B, Hkv * G, Hkv, D, Dv, rng.choice([16, 16, 16, 32, 64, 20, 128]) if D != 576 else rng.choice([64, 64, 32]),
                           max(1, mid // 8), mid, mid * 4, rng.choice([0, 0, 0, 500, 4096, 16384]), rng.choice([0, 0, 0, B // 2, B]), rng.choice([0, 0, 13]))
            w = work(c)
            fits = w["flops"] <= 2.9e12 and w["bytes"] <= 4e9
        if fits:
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------
# what a case's numbers stand for
# ------------------------------------------------------------------------------------------------
def _quantiles(count, lo, mid, hi):
    """`count` quantiles of a lognormal distribution (sigma 0.8) between lo and hi, ascending."""
    n = [min(max(mid * math.exp(0.8 * NormalDist().inv_cdf((i + 0.5) / count)), lo), hi) for i in range(count)]
    return np.rint(np.asarray(n)).astype(np.int64)


def _new_lengths(c):
    """New tokens of each request, ascending; the first `singles` requests add one token."""
    n = np.ones(c["B"], dtype=np.int64)
    if c["B"] > c["singles"]:
        n[c["singles"]:] = _quantiles(c["B"] - c["singles"], c["lo"], c["mid"], c["hi"])
    return n


def _past_lengths(c):
    """Cached positions of each request before the call: around `past`, the longer ones not beside the longer pieces."""
    if not c["past"]:
        return np.zeros(c["B"], dtype=np.int64)
    n = _quantiles(c["B"], c["past"] // 8, c["past"], c["past"] * 2)
    return n[(np.arange(c["B"]) * 7 + 3) % c["B"]] if math.gcd(7, c["B"]) == 1 else n[::-1].copy()


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _reserve_rows(c):
    """Rows of a reserve case, without their order: (prompt length of the row's group, response length, role), role 0 = goes on,
    1 = over in even passes and starts in odd ones, 2 = the other way round.  The first row of a group goes on."""
    B, group = c["B"], c["group"]
    groups = -(-B // group)
    prompt = np.repeat(_quantiles(groups, c["lo"], c["mid"], c["hi"]), group)[:B]
    response = np.tile(_quantiles(group, c["lo"], c["mid"], c["hi"]), groups)[:B]
    role = np.zeros(B, dtype=np.int64)
    turn = [b for b in range(B) if (b % group or group == 1) and (b * 0.618034) % 1.0 < c["turnover"]]
    role[turn] = 1 + np.arange(len(turn)) % 2
    return prompt, response, role


def _turns(c):
    """The two steps that a reserve case alternates between: (ctx_len, n_new, share_from) of each."""
    prompt, response, role = _reserve_rows(c)
    B, page, group = c["B"], c["page"], c["group"]
    leader = np.arange(B) // group * group
    turns = []
    for turn in range(2):
        ctx, new, share = prompt + response + min(5, c["T"]) * turn, np.full(B, c["T"], dtype=np.int64), np.full(B, -1, dtype=np.int64)
        over, starts = role == 1 + turn, role == 2 - turn
        ctx[over], new[over] = 0, -1
        if group > 1:
            ctx[starts] = prompt[starts] // page * page
            share[starts] = leader[starts]
            new[starts] = prompt[starts] % page + c["T"]
        else:
            ctx[starts], new[starts] = 0, prompt[starts]
        turns.append((ctx, new, share))
    return turns


def _reserve_sizes(c):
    """(table width, pages of the pool, tokens of a call, padding included)."""
    prompt, response, _ = _reserve_rows(c)
    need = (prompt + response + 5 + c["T"] + c["page"] - 1) // c["page"] + 1
    tokens = max(int(np.maximum(new, 0).sum()) for _, new, _ in _turns(c))
    return int(need.max()), max(c["pages"], int(need.sum() * 1.1) + 64), tokens + c["pad"]


def _prepare_reserve(c, rng):
    width, pages, tokens = _reserve_sizes(c)
    prompt, response, role = _reserve_rows(c)
    B, page, order = c["B"], c["page"], rng.permutation(c["B"])        # order[i]: the row that stands at place i
    place = np.argsort(order)
    table, held, refs = np.zeros((B, width), dtype=np.int64), np.zeros(B, dtype=np.int64), np.zeros(pages, dtype=np.int64)
    ids, at = rng.permutation(pages), 0
    for b in range(B):
        if role[b] == 2:
            continue                                                   # (starts in the first step)
        leader, n = b // c["group"] * c["group"], int(-(-(prompt[b] + response[b]) // page))
        shared = int(prompt[b] // page) if b != leader else 0
        row = place[b]
        table[row, :shared] = table[place[leader], :shared]
        table[row, shared:n] = ids[at:at + n - shared]
        at += n - shared
        held[row] = n
        refs[table[row, :n]] += 1
    turns = []
    for ctx, new, share in _turns(c):
        share = np.where(share >= 0, place[np.maximum(share, 0)], -1)
        mask = None
        if c["tree"]:
            # ancestor bits of a random tree for the rows of a verify step, none for other tokens
            mask = np.zeros(tokens, dtype=np.int64)
            first = np.concatenate([[0], np.cumsum(np.maximum(new[order], 0))])
            for i in range(B):
                if new[order][i] == c["T"]:
                    words = [1]
                    for t in range(1, c["T"]):
                        words.append(words[int(rng.integers(0, t))] | 1 << t)
                    mask[first[i]:first[i] + c["T"]] = words
            mask = torch.from_numpy(mask).cuda()
        turns.append((_i32(ctx[order]), _i32(new[order]), _i32(share[order]) if c["group"] > 1 else None, mask))
    return {"case": c, "table": _i32(table), "held": _i32(held), "refs": _i32(refs), "turns": turns, "turn": 0, "tokens": tokens}


def _prepare_append(c, rng, gen):
    N, Hq, Hkv, D, Dv = c["N"], c["Hq"], c["Hkv"], c["D"], c["Dv"]
    widths = [Hq * D, Hkv * D, Hkv * Dv]
    total = N + c["pad"]
    if c["fused"]:
        parts = torch.randn((total, sum(widths)), dtype=torch.bfloat16, device="cuda", generator=gen).split(widths, 1)
    else:
        parts = [torch.randn((total, w), dtype=torch.bfloat16, device="cuda", generator=gen) for w in widths]
    s = {"case": c, "q": parts[0].view(total, Hq, D), "k": parts[1].view(total, Hkv, D), "v": parts[2].view(total, Hkv, Dv) if Dv else None}
    # tokens of a few sequences, one behind the other in their pages, at positions up to `far`
    page, length = c["page"], min(max(1, N // 8), c["far"])
    slots, positions, pages = [], [], rng.permutation(-(-N // page) + 2 * -(-N // length) + 2)
    at = 0
    for first in range(0, N, length):
        n = min(length, N - first)
        begin = int(rng.integers(0, c["far"] - n + 1))
        inside = begin % page + np.arange(n)
        own_pages = pages[at:at + -(-int(inside[-1] + 1) // page)]
        at += len(own_pages)
        slots.append(own_pages[inside // page] * page + inside % page)
        positions.append(begin + np.arange(n))
    s["slot"] = _i32(np.concatenate(slots + [np.full(c["pad"], -1)]))
    s["position"] = _i32(np.concatenate(positions + [np.full(c["pad"], -1)]))
    s["inv_freq"] = torch.from_numpy(500000.0 ** (-np.arange(0, c["rotary"], 2) / c["rotary"])).float().cuda()
    s["q_out"] = torch.zeros((total, Hq, D), dtype=torch.bfloat16, device="cuda")
    s["k_pages"] = torch.randn((len(pages), Hkv, page, D), dtype=torch.bfloat16, device="cuda", generator=gen)
    s["v_pages"] = torch.randn((len(pages), Hkv, page, Dv), dtype=torch.bfloat16, device="cuda", generator=gen) if Dv else None
    return s


def _prepare_attention(c, rng, gen):
    new, past, order = _new_lengths(c), _past_lengths(c), rng.permutation(c["B"])
    new, ctx = new[order], (new + past)[order]
    need = -(-ctx // c["page"])
    pages = int(need.sum()) + 3
    ids, table, at = rng.permutation(pages), np.zeros((c["B"], int(need.max())), dtype=np.int64), 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    first = np.concatenate([[0], np.cumsum(new)])
    N = int(first[-1]) + c["pad"]
    shared = c["D"] == 576
    s = {"case": c, "new": new.tolist(), "ctx_host": ctx.tolist(), "ctx": _i32(ctx), "first": _i32(first), "table": _i32(table), "scale": c["D"] ** -0.5}
    s["q"] = torch.randn((N, c["Hq"], c["D"]), dtype=torch.bfloat16, device="cuda", generator=gen).mul_(SCORE_STD)
    s["k"] = torch.randn((pages, c["Hkv"], c["page"], c["D"]), dtype=torch.bfloat16, device="cuda", generator=gen)
    s["v"] = None if shared else torch.randn((pages, c["Hkv"], c["page"], c["Dv"]), dtype=torch.bfloat16, device="cuda", generator=gen)
    s["out"] = torch.zeros((N, c["Hq"], c["Dv"]), dtype=torch.bfloat16, device="cuda")
    return s


def prepare(case, seed):
    rng, gen = np.random.default_rng([seed, 11]), _generator(seed)
    if case["kind"] == "reserve":
        return _prepare_reserve(case, rng)
    return (_prepare_append if case["kind"] == "append" else _prepare_attention)(case, rng, gen)


# ------------------------------------------------------------------------------------------------
# the calls
# ------------------------------------------------------------------------------------------------
def _next_turn(s):
    """The step of this pass: the two alternate, so that every pass finds work, and the next but one the same again."""
    turn = s["turns"][s["turn"]]
    s["turn"] ^= 1
    return turn


def _own(s):
    from paper_2511_14617_amd import binding
    c, kind = s["case"], s["case"]["kind"]
    if kind == "reserve":
        ctx, new, share, mask = _next_turn(s)
        made = binding.seer_kv_reserve(s["table"], s["held"], s["refs"], ctx, new, s["tokens"], c["page"], share_from=share, tree_mask=mask)
        return [s["table"], s["held"], s["refs"], *made]
    if kind == "append":
        binding.seer_kv_append(s["q"], s["k"], s["v"], s["slot"], s["position"], s["k_pages"], s["v_pages"], inv_freq=s["inv_freq"],
                               rotary_at=c["at"], interleaved=c["interleaved"], q_out=s["q_out"])
        return [s["q_out"], s["k_pages"], s["v_pages"]]
    return binding.seer_prompt_attention(s["q"], s["k"], s["v"], s["table"], s["ctx"], s["first"], s["scale"], Dv=c["Dv"], out=s["out"])


def _plain_reserve(s):
    c, page = s["case"], s["case"]["page"]
    ctx, new, share, mask = _next_turn(s)
    ctx, new, table, held = ctx.long(), new.long(), s["table"].long(), s["held"].long()
    share = torch.full_like(ctx, -1) if share is None else share.long()
    B, pages, dev = len(ctx), s["refs"].numel(), ctx.device
    j, shares = torch.arange(table.shape[1], device=dev), share >= 0
    need = torch.where(new < 0, 0, (ctx + new + page - 1) // page)
    base = torch.where(shares, ctx // page, held)
    grow = (need - base).clamp(min=0)
    parent = table[share.clamp(min=0)]
    take = shares[:, None] & (j < base[:, None])
    drop = ~shares[:, None] & (j >= need[:, None]) & (j < held[:, None])
    # (entries behind the pool take what is not meant, each its own)
    spare = pages + torch.arange(table.numel(), device=dev).view_as(table)
    refs = torch.cat([s["refs"].long(), torch.zeros(table.numel(), dtype=torch.long, device=dev)])
    refs.index_add_(0, torch.where(take, parent, spare).view(-1), take.view(-1).long())
    refs.index_add_(0, torch.where(drop, table, spare).view(-1), -drop.view(-1).long())
    free = refs[:pages] == 0
    ids = torch.arange(pages, device=dev)
    source = torch.zeros(2 * pages, dtype=torch.long, device=dev).scatter_(0, torch.where(free, torch.cumsum(free, 0) - 1, pages + ids), ids)
    end = torch.cumsum(grow, 0)
    ok = (grow == 0) | (end <= free.sum())
    undo = take & ~ok[:, None]
    refs.index_add_(0, torch.where(undo, parent, spare).view(-1), -undo.view(-1).long())
    given = ok[:, None] & (j >= base[:, None]) & (j < (base + grow)[:, None])
    page_id = source[((end - grow - base)[:, None] + j).clamp(0, pages - 1)]
    table = torch.where(given, page_id, torch.where(take & ok[:, None], parent, table))
    refs.scatter_(0, torch.where(given, page_id, spare).view(-1), 1)
    s["table"].copy_(table)
    s["held"].copy_(torch.where(ok, need, held))
    s["refs"].copy_(refs[:pages])
    first = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), torch.cumsum(new.clamp(min=0), 0)])
    i = torch.arange(s["tokens"], device=dev)
    b = torch.searchsorted(first[1:], i, right=True)
    real = b < B
    b = b.clamp(max=B - 1)
    real = real & ok[b]
    at = ctx[b] + i - first[b]
    slot = table[b, (at // page).clamp(max=table.shape[1] - 1)] * page + at % page
    if mask is not None:
        depth = ((mask[:, None] >> torch.arange(64, device=dev)) & 1).sum(1) - 1
        at = torch.where(mask != 0, ctx[b] + depth, at)
    step = torch.where(ok & (new >= 0), ctx + new, 0)
    return [s["table"], s["held"], s["refs"], step.int(), first.int(), torch.where(real, slot, -1).int(), torch.where(real, at, -1).int()]


def _turned(x, angle, at, interleaved):
    """x [N,H,D] float32 with the components from `at` on rotated by angle [N,R/2] (64 bits)."""
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    R = 2 * angle.shape[1]
    part = x[..., at:at + R]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., : R // 2], part[..., R // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    part = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([x[..., :at], part, x[..., at + R:]], -1)


def _plain_append(s):
    c, n, page = s["case"], s["case"]["N"], s["case"]["page"]
    angle = s["position"][:n].double()[:, None] * s["inv_freq"].double()
    s["q_out"][:n] = _turned(s["q"][:n].float(), angle, c["at"], c["interleaved"]).bfloat16()
    slot = s["slot"][:n].long()
    s["k_pages"][slot // page, :, slot % page] = _turned(s["k"][:n].float(), angle, c["at"], c["interleaved"]).bfloat16()
    if s["v"] is not None:
        s["v_pages"][slot // page, :, slot % page] = s["v"][:n]
    return [s["q_out"], s["k_pages"], s["v_pages"]]


def _plain_attention(s):
    c, Hkv, D, Dv = s["case"], s["case"]["Hkv"], s["case"]["D"], s["case"]["Dv"]
    out, first = torch.zeros_like(s["out"]), 0
    for b, (n, ctx) in enumerate(zip(s["new"], s["ctx_host"])):
        rows = s["table"][b, : -(-ctx // c["page"])].long()
        k = s["k"][rows].transpose(0, 1).reshape(Hkv, -1, D)[:, :ctx].float()
        v = k[:, :, :Dv] if s["v"] is None else s["v"][rows].transpose(0, 1).reshape(Hkv, -1, Dv)[:, :ctx].float()
        step = max(1, CHUNK // (c["Hq"] * ctx))
        for i in range(0, n, step):
            m = min(step, n - i)
            end = ctx - n + i + m                                     # what the last of these tokens sees
            q = s["q"][first + i:first + i + m].float().view(m, Hkv, -1, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
            scores = torch.matmul(q, k[:, :end].transpose(1, 2).contiguous()).view(Hkv, -1, m, end) * s["scale"]
            seen = torch.arange(end, device=q.device)[None, :] <= (end - m + torch.arange(m, device=q.device))[:, None]
            scores = torch.where(seen, scores, -math.inf)
            e = torch.exp(scores - scores.amax(-1, keepdim=True))
            o = torch.matmul(e.view(Hkv, -1, end), v[:, :end]).view(Hkv, -1, m, Dv) / e.sum(-1, keepdim=True)
            out[first + i:first + i + m] = o.permute(2, 0, 1, 3).reshape(m, -1, Dv).bfloat16()
        first += n
    return out


def run(state):
    if own:
        return _own(state)
    return {"reserve": _plain_reserve, "append": _plain_append, "attention": _plain_attention}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without, and what its outputs are in 64 bits
# ------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "reserve":
        _, pages, tokens = _reserve_sizes(c)
        prompt, response, role = _reserve_rows(c)
        moved = 0
        for turn in (0, 1):                                           # page ids given, shared or taken back, of the two steps
            shared = (prompt // c["page"]) if c["group"] > 1 else 0 * prompt
            starts, over = role == 2 - turn, role == 1 + turn
            moved += 12 * int(((prompt + c["T"]) // c["page"])[starts].sum()) + 8 * int(shared[over].sum()) + 12 * int(over.sum())
        return {"bytes": 4 * pages + 8 * tokens + c["B"] * 24 + moved // 2 + (8 * tokens if c["tree"] else 0), "flops": pages + 8 * tokens}
    if c["kind"] == "append":
        row = c["Hq"] * c["D"] + c["Hkv"] * (c["D"] + c["Dv"])
        return {"bytes": c["N"] * (4 * row + 8), "flops": 3 * c["N"] * (c["Hq"] + c["Hkv"]) * c["rotary"]}
    new, past = _new_lengths(c), _past_lengths(c)
    pairs = int((new * past + new * (new + 1) // 2).sum())
    cached = 2 * (c["D"] if c["D"] == 576 else c["D"] + c["Dv"])
    return {"bytes": int(new.sum()) * c["Hq"] * 2 * (c["D"] + c["Dv"]) + int((new + past).sum()) * c["Hkv"] * cached,
            "flops": 2 * (c["D"] + c["Dv"]) * c["Hq"] * pairs}


def _exact_reserve(c, s):
    """Request by request, on lists."""
    page = c["page"]
    table, held, refs = s["table"].tolist(), s["held"].tolist(), s["refs"].tolist()
    ctx, new, share, mask = (None if x is None else x.tolist() for x in s["turns"][s["turn"]])
    B = len(ctx)
    before, start = [row[:] for row in table], [0] * B
    for b in range(B):
        if share is not None and share[b] >= 0:
            start[b] = ctx[b] // page
            for x in range(start[b]):
                table[b][x] = before[share[b]][x]
                refs[table[b][x]] += 1
        else:
            start[b] = held[b]
    for b in range(B):
        keep = 0 if new[b] < 0 else -(-(ctx[b] + new[b]) // page)
        for x in range(keep, start[b]):
            refs[before[b][x]] -= 1
        held[b] = min(start[b], keep)
    free = iter([x for x, r in enumerate(refs) if r == 0])
    step, first, slots, positions = [], [0], [], []
    for b in range(B):
        n = max(new[b], 0)
        while new[b] >= 0 and held[b] * page < ctx[b] + n:
            table[b][held[b]] = next(free)
            refs[table[b][held[b]]] = 1
            held[b] += 1
        for i in range(n):
            at = ctx[b] + i
            slots.append(table[b][at // page] * page + at % page)
            word = mask[first[b] + i] if mask is not None else 0
            positions.append(ctx[b] + bin(word & (2 ** 64 - 1)).count("1") - 1 if word else at)
        step.append(ctx[b] + n if new[b] >= 0 else 0)
        first.append(first[b] + n)
    padding = [-1] * (s["tokens"] - first[-1])
    return [torch.tensor(x, dtype=torch.int32) for x in (table, held, refs, step, first, slots + padding, positions + padding)]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "reserve":
        return _exact_reserve(c, s)
    if c["kind"] == "append":
        page, R, at = c["page"], c["rotary"], c["at"]
        angle = s["position"].double()[:, None] * s["inv_freq"].double()[None]
        turn = torch.complex(torch.cos(angle), torch.sin(angle))[:, None]
        outs = [s["q_out"].double(), s["k_pages"].double(), None if s["v"] is None else s["v_pages"].double()]
        live = torch.nonzero(s["slot"] >= 0)[:, 0]
        slot = s["slot"][live].long()
        for x, name in ((s["q"], 0), (s["k"], 1), (s["v"], 2)):
            if x is None:
                continue
            y = x[live].double()
            if name < 2:
                part = y[..., at:at + R]
                pairs = part.unflatten(-1, (R // 2, 2)) if c["interleaved"] else part.unflatten(-1, (2, R // 2)).transpose(-1, -2)
                z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[live])
                y[..., at:at + R] = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
            if name == 0:
                outs[0][live] = y
            else:
                outs[name].transpose(1, 2)[slot // page, slot % page] = y
        return outs
    out, first = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), s["first"].tolist()
    for b, ctx in enumerate(s["ctx"].tolist()):
        n = first[b + 1] - first[b]
        place = torch.arange(ctx, device="cuda")
        rows, inside = s["table"][b].long()[place // c["page"]], place % c["page"]
        step = max(1, (1 << 26) // ctx)
        for h in range(c["Hkv"]):
            k = s["k"][rows, h, inside].double()
            v = k[:, :c["Dv"]] if s["v"] is None else s["v"][rows, h, inside].double()
            G = c["Hq"] // c["Hkv"]
            for hq in range(h * G, h * G + G):
                for i in range(0, n, step):
                    q = s["q"][first[b] + i:min(first[b] + i + step, first[b + 1]), hq].double()
                    seen = place[None, :] <= (ctx - n + i + torch.arange(len(q), device="cuda"))[:, None]
                    z = torch.matmul(q, k.t()) * s["scale"]
                    p = torch.softmax(z.masked_fill_(~seen, -math.inf), -1)
                    out[first[b] + i:first[b] + i + len(q), hq] = torch.matmul(p, v)
    return out

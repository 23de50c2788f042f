"""Plain implementation of seer_kv_reserve for the tests: one row after the other, on lists, from the documented rules."""


def reserve(table, held, refs, ctx, new, share, mask, n_tokens, page):
    """The arrays after the call and what it writes: (table, held, refs, step_len, first_token, slot, position, status); the inputs are left
    alone.  table: list of lists; share, mask: lists or None."""
    table0, held0 = table, held
    table, held, refs = [row[:] for row in table], held[:], refs[:]
    B, width, pages = len(table), len(table[0]), len(refs)
    status = 0
    first, total = [0], 0
    for b in range(B):
        total += max(new[b], 0)
        first.append(min(total, 2 ** 31 - 1))
    before = [0]
    for b in range(B):
        before.append(before[-1] + max(new[b], 0))
    good, base, need, shared = [False] * B, held[:], [0] * B, [-1] * B
    for b in range(B):
        if new[b] < -1 or not 0 <= held0[b] <= width:
            status |= 1
            continue
        if new[b] == -1:
            good[b] = True
            continue
        if ctx[b] < 0 or ctx[b] + new[b] > width * page:
            status |= 1
            continue
        r = share[b] if share is not None else -1
        if r >= 0:
            if r >= B or r == b or held0[b] != 0 or ctx[b] % page or not 0 <= held0[r] <= width or ctx[b] // page > held0[r]:
                status |= 1
                continue
        elif ctx[b] > held0[b] * page:
            status |= 1
            continue
        if before[b] + new[b] > n_tokens:
            status |= 4
            continue
        if r >= 0:
            shared[b], base[b] = r, ctx[b] // page
        good[b], need[b] = True, -(-(ctx[b] + new[b]) // page)
    for b in range(B):
        if good[b] and shared[b] >= 0:
            for p in table0[shared[b]][:base[b]]:
                if not 0 <= p < pages:
                    status |= 2
                else:
                    refs[p] += 1
    for b in range(B):
        if good[b] and shared[b] < 0:
            for p in table0[b][need[b]:base[b]]:
                if not 0 <= p < pages:
                    status |= 2
                else:
                    refs[p] -= 1
    if min(refs) < 0:
        status |= 16
    free = [p for p in range(pages) if refs[p] == 0]
    asked = 0
    granted = [False] * B
    at = 0
    for b in range(B):
        if not good[b]:
            continue
        grow = max(0, need[b] - base[b])
        asked += grow
        granted[b] = grow == 0 or asked <= len(free)
        if not granted[b]:
            status |= 8
            if shared[b] >= 0:
                for p in table0[shared[b]][:base[b]]:
                    if 0 <= p < pages:
                        refs[p] -= 1
            continue
        if shared[b] >= 0:
            table[b][:base[b]] = table0[shared[b]][:base[b]]
        for j in range(base[b], need[b]):
            at = asked - grow + j - base[b]
            table[b][j] = free[at]
            refs[free[at]] = 1
        held[b] = need[b]
    step = [ctx[b] + new[b] if granted[b] and new[b] >= 0 else 0 for b in range(B)]
    slot, position = [-1] * n_tokens, [-1] * n_tokens
    for b in range(B):
        if not granted[b] or new[b] < 1:
            continue
        for i in range(new[b]):
            t, pos = before[b] + i, ctx[b] + i
            p = table[b][pos // page]
            if 0 <= p < pages:
                slot[t] = p * page + pos % page
            else:
                status |= 2
            word = mask[t] & (2 ** 64 - 1) if mask is not None else 0
            position[t] = ctx[b] + bin(word).count("1") - 1 if word else pos
    return table, held, refs, step, first, slot, position, status

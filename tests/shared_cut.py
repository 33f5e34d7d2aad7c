"""How tetra_kv_attend_shared cuts the tokens that groups share into parts, restated: which part a CTA has after which."""

STEP, BLOCK, COLUMNS, LEAST, COST = 64, 16, 128, 8, 8  # tokens of a step and a block, columns of a slot, blocks that are shared at least, steps a part costs


def tile(D):
    return COLUMNS * (1 if D == 256 else 2)


def ceil(a, b):
    return -(-a // b)


def cut(D, kv_heads, group, prompts, ctas):
    """prompts: (rows of a group's sequences together, tokens that they share).  Returns for each CTA its parts in order: (steps, whether
    both slots share its columns)."""
    live = [(rows * group, tokens // BLOCK * BLOCK) for rows, tokens in prompts if tokens // BLOCK >= LEAST]
    work = [(ceil(cols, tile(D)) * kv_heads, ceil(tokens, STEP)) for cols, tokens in live]
    rows, groups = sum(r for r, _ in prompts), len(prompts)
    most = max((rows * group // tile(D) + min(groups, rows)) * kv_heads, 2 * 160)
    items, total, longest = sum(i for i, _ in work), sum(i * s for i, s in work), max([s for _, s in work] + [1])
    share, cost = longest, None
    for k in (1, 2):
        may = min(k * ctas, most)
        if items > may or (k > 1 and (2 * items <= ctas or (cost is not None and k * (1 + COST) >= cost))):
            continue
        at = max(1, ceil(total, may))
        while True:
            by = max(1, at >> 4)
            tried = [min(at + lane * by, longest) for lane in range(32)]
            fits = [t for t in tried if sum(i * ceil(s, t) for i, s in work) <= may]
            if fits:
                break
            at += 32 * by
        if cost is None or k * (fits[0] + COST) < cost:
            cost, share = k * (fits[0] + COST), fits[0]
    parts = []
    for (cols, _), (items, steps) in zip(live, work):
        each = steps if steps <= share else ceil(steps, ceil(steps, share))
        for item in range(items):
            both = D != 256 and min(tile(D), cols - item % ceil(cols, tile(D)) * tile(D)) <= COLUMNS
            parts += [(min(each, steps - at), both) for at in range(0, steps, each)]
    return [parts[c::ctas] for c in range(ctas)]


def one_step_ahead_of_another(parts):
    """CTAs in which a part of one step, whose columns the slots share, comes before another such part."""
    return [c for c, mine in enumerate(parts) if any(a == (1, True) and b[1] for a, b in zip(mine, mine[1:]))]


# Prompts of two answers each: four that share 1344 tokens, then sixteen that share 128.
TWENTY = [(2, 1344)] * 4 + [(2, 128)] * 16

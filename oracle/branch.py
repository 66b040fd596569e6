"""Definitions of the pages of a batch (forking, reserving, compacting) and of the judging of drafted tokens, request by
request, in Python integers and 64 bits.

Test infrastructure: shares no code with the library.  Arrays are numpy, changed in place where the calls do.
"""
import numpy as np


def pages_select(table, lens, pages, rows_from, new_table, refs, page):
    """Returns (new lengths, new pages); changes new_table and refs."""
    n, most = table.shape
    new_lens, new_pages = np.zeros(len(rows_from), np.int32), np.zeros(len(rows_from), np.int32)
    for i, s in enumerate(rows_from):
        if not 0 <= s < n:
            continue
        new_lens[i] = min(max(int(lens[s]), 0), most * page)
        new_pages[i] = min(-(-int(new_lens[i]) // page), min(max(int(pages[s]), 0), most))
        for j in range(new_pages[i]):
            b = table[s, j]
            new_table[i, j] = b
            if 0 <= b < len(refs):
                refs[b] += 1
    for s in range(n):
        for j in range(min(max(int(pages[s]), 0), most)):
            if 0 <= table[s, j] < len(refs):
                refs[table[s, j]] -= 1
    return new_lens, new_pages


def pages_reserve(table, lens, pages, grow, refs, page):
    """Returns (served, copy_src, copy_dst); changes table, pages and refs."""
    n, most = table.shape
    held = refs.copy()
    served, src, dst = np.zeros(n, np.int32), np.full(n, -1, np.int32), np.full(n, -1, np.int32)

    def wants(i):
        """(page of the next token, pages held (less those that are given up), pages wanted, whether a shared page would be written)"""
        length, g = min(max(int(lens[i]), 0), most * page), max(int(grow[i]), 0)
        has = min(max(int(pages[i]), 0), most)
        at = length // page
        wanted = min(-(-(length + g) // page), most) if g else 0
        for j in range(-(-length // page), min(has, wanted)):      # a shared page without a token of the request, where tokens are to go: it is given up, with what is behind it
            if 0 <= table[i, j] < len(refs) and held[table[i, j]] > 1:
                has = j
                break
        end = max(has, wanted)
        b = table[i, at] if g and length % page and at < has else -1
        return at, has, end, 0 <= b < len(refs) and held[b] > 1

    writers = {}
    for i in range(n):
        at, _, _, shared = wants(i)
        if shared:
            writers.setdefault(int(table[i, at]), []).append(i)
    keepers = {w[-1] for b, w in writers.items() if len(w) == held[b]}
    free = [b for b in range(len(refs)) if refs[b] == 0]
    short = False
    for i in range(n):
        at, has, end, shared = wants(i)
        copies = shared and i not in keepers
        need = end - has + int(copies)
        short = short or need > len(free)
        if short and (need or i in keepers):
            continue
        served[i] = 1
        for b in table[i, has:min(max(int(pages[i]), 0), most)]:
            if 0 <= b < len(refs):
                refs[b] -= 1
        if copies:
            src[i], dst[i] = table[i, at], free.pop(0)
            refs[src[i]] -= 1
            refs[dst[i]] = 1
            table[i, at] = dst[i]
        for j in range(has, end):
            table[i, j] = free.pop(0)
            refs[table[i, j]] = 1
        pages[i] = end
    return served, src, dst


def pages_compact(table, pages, refs, max_moves):
    """Returns (new table, new refs, copy_src, copy_dst)."""
    used = int((refs > 0).sum())
    src = [b for b in range(used, len(refs)) if refs[b] > 0][:max_moves]
    dst = [b for b in range(used) if refs[b] <= 0][:len(src)]
    to = dict(zip(src, dst))
    new_table, new_refs = table.copy(), refs.copy()
    for i in range(len(table)):
        for j in range(min(max(int(pages[i]), 0), table.shape[1])):
            new_table[i, j] = to.get(int(table[i, j]), table[i, j])
    for a, b in to.items():
        new_refs[b], new_refs[a] = refs[a], 0
    pad = [-1] * (max_moves - len(src))
    return new_table, new_refs, np.array(src + pad, np.int32), np.array(dst + pad, np.int32)


def probabilities(logits, temperature):
    """softmax(logits / temperature); NaN counts as -inf, inf as the largest fp32 number.  Zeros where nothing can be drawn."""
    x = np.asarray(logits, np.float64)
    x = np.minimum(np.where(np.isnan(x), -np.inf, x), float(np.finfo(np.float32).max))
    if (x == -np.inf).all():
        return np.zeros_like(x)
    with np.errstate(over="ignore", under="ignore"):
        w = np.where(x == -np.inf, 0.0, np.exp(np.where(x == -np.inf, 0.0, x - x.max()) / temperature))
    return w / w.sum()


def first_largest(logits):
    """Number of the first of the largest logits, -1 where there is none above -inf."""
    x = np.asarray(logits, np.float64)
    x = np.minimum(np.where(np.isnan(x), -np.inf, x), float(np.finfo(np.float32).max))
    return int(x.argmax()) if x.max() > -np.inf else -1


def draft_verify(target, draft, tokens, mask, temperature, accept_u, sample_u, max_keep):
    """One request.  target, draft: [T, V] (draft None: the tokens were not drawn); mask: a word for each token, None: a
    chain.  Returns (tokens that stay, the token behind them), with the textbook's residuals, normalised anew after every refusal."""
    T = len(tokens)
    if T == 0:
        return [], -1
    V = target.shape[1]
    ancestors = [(int(mask[t]) if mask is not None else (1 << t) - 1) & ((1 << t) - 1) for t in range(T)]
    parent = [a.bit_length() - 1 for a in ancestors]
    greedy = not temperature > 0
    at, kept, left = 0, [0], None
    for t in range(1, T):
        if len(kept) == max_keep:
            break
        x = int(tokens[t])
        if parent[t] != at or not 0 <= x < V:
            continue
        if greedy:
            if first_largest(target[at]) == x:
                at = t
                kept.append(t)
            continue
        if left is None:
            left = probabilities(target[at], temperature)
        q = None if draft is None else probabilities(draft[at], temperature)
        if left[x] > float(accept_u[t]) * (1.0 if q is None else q[x]):
            at, left = t, None
            kept.append(t)
            continue
        if q is None:
            left = left.copy()
            left[x] = 0
        else:
            left = np.maximum(left - q, 0)
        if left.sum() > 0:
            left = left / left.sum()
    if greedy:
        return kept, first_largest(target[at])
    p = probabilities(target[at], temperature)
    left = p if left is None or not left.sum() > 0 else left
    if not left.sum() > 0:
        return kept, -1
    upto = left.cumsum()
    over = np.nonzero((upto > min(max(float(sample_u), 0.0), 1.0) * upto[-1]) & (left > 0))[0]
    return kept, int(over[0] if len(over) else np.nonzero(left > 0)[0][-1])

"""A cache in pages, position by position on the host, and attention over it in 64 bits from the formulas with the bounds of attention_plain."""
import numpy as np
import torch

from tests import attention_plain as plain


def step(lengths, added, tables, stack, count, page, pages, tokens):
    """What paged_tables makes of lists of numbers: (lengths, row_ptr, rows, seen, slots, counts), and tables and stack as they are then."""
    width, room = len(tables[0]) if tables else 0, len(stack)
    tables, stack = [list(t) for t in tables], list(stack)
    count = min(max(count, 0), room)
    ok = lambda p: p if 0 <= p < pages else -1  # noqa: E731
    most = min(width * page, 2 ** 31 - 1)
    lengths = [min(max(n, 0), most) for n in lengths]
    popped = list(stack[:count])
    for r, more in enumerate(added):
        if more < 0:
            popped += tables[r][:-(-lengths[r] // page)]
    popped = popped[:room]
    stack[count:len(popped)] = popped[count:]
    top, taken, row_ptr, totals, rows, seen, slots, fit, none = len(popped), 0, [0], [], [], [], [], 0, set()
    for r, more in enumerate(added):
        total = 0 if more < 0 else min(lengths[r] + more, most)
        for p in range(-(-lengths[r] // page), -(-total // page)):
            top, taken = top - 1, taken + 1
            tables[r][p] = ok(popped[top]) if top >= 0 else -1
            if top < 0:
                none.add((r, p))
        for at in range(lengths[r], lengths[r] + max(more, 0)):
            if len(rows) == tokens:
                break
            held = ok(tables[r][at // page]) if at < total else -1
            rows.append(r)
            seen.append(at + 1 if held >= 0 else 0)
            slots.append(held * page + at % page if held >= 0 else -1)
            fit += at < total and (r, at // page) not in none       # (a page that is no page is not missing)
        totals.append(total)
        row_ptr.append(min(row_ptr[-1] + max(more, 0), 2 ** 31 - 1))
    pad = tokens - len(rows)
    return [totals, row_ptr, rows + [-1] * pad, seen + [0] * pad, slots + [-1] * pad, [top, row_ptr[-1], min(sum(max(x, 0) for x in added) - fit, 2 ** 31 - 1), taken]], tables, stack


def positions(tables, row, seen, page, pages, listed=None):
    """(page, row in it) of what a token sees, in order; listed: pages of its list, each entry a term of its own."""
    if not 0 <= row < len(tables):
        return []
    seen = min(max(seen, 0), len(tables[row]) * page)
    # of a list the first entries count, as many as there are pages
    at = range(seen) if listed is None else [c * page + i for c in listed[:-(-seen // page)] if c >= 0 for i in range(page)]
    return [(tables[row][p // page], p % page) for p in at if p < seen and 0 <= tables[row][p // page] < pages]


def attention(q, k_pages, v_pages, tables, seen, rows=None, lists=None, scale=None):
    """For each token (O [H, d], lse [H], bounds of both), float64 on the CPU; each key head its own list."""
    M, H, d = q.shape
    pages, Hkv, page = k_pages.shape[:3]
    group, scale = H // Hkv, d ** -0.5 if scale is None else scale
    q, k_pages, v_pages = q.cpu(), k_pages.cpu(), v_pages.cpu()
    tables, seen = tables.tolist(), seen.tolist()
    rows = list(range(M)) if rows is None else rows.tolist()
    for i in range(M):
        parts = []
        for g in range(Hkv):
            at = positions(tables, rows[i], seen[i], page, pages, None if lists is None else lists[i, g].tolist())
            c, r = (torch.tensor(x, dtype=torch.long) for x in zip(*at)) if at else (torch.zeros(0, dtype=torch.long),) * 2
            mask = torch.ones((1, group, 1, len(at)), dtype=torch.bool)
            parts.append(plain.forward(mask, q[i, g * group:(g + 1) * group].view(1, group, 1, d), k_pages[c, g, r].view(1, 1, -1, d),
                                       v_pages[c, g, r].view(1, 1, -1, d), scale))
        yield [torch.cat([p[j].view(group, -1) for p in parts]).squeeze(1) if j % 2 else torch.cat([p[j].view(group, d) for p in parts])
               for j in range(4)]


def select(q, means, tables, seen, page, keep, first, last, rows=None):
    """Lists of pages in 64 bits, ties to the lower page, NaN last."""
    M, H, d = q.shape
    pages, Hkv = means.shape[:2]
    q, means, tables, seen = q.cpu().double(), means.cpu().double(), tables.tolist(), seen.tolist()
    rows = list(range(M)) if rows is None else rows.tolist()
    out = torch.full((M, Hkv, keep), -1, dtype=torch.int32)
    for i in range(M):
        if not 0 <= rows[i] < len(tables):
            continue
        table = tables[rows[i]]
        n = -(-min(max(seen[i], 0), len(table) * page) // page)
        for g in range(Hkv):
            total = q[i].view(Hkv, H // Hkv, d)[g].sum(0)
            score = [float(total @ means[c, g]) if 0 <= c < pages else -np.inf for c in table[:n]]
            order = sorted(range(n), key=lambda p: (not (p < first or p >= n - last), np.isnan(score[p]), -score[p] if not np.isnan(score[p]) else 0, p))
            best = sorted(order[:keep])
            out[i, g, :len(best)] = torch.tensor(best, dtype=torch.int32)
    return out

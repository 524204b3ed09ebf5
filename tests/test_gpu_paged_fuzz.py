"""Seeded random steps of a server through all calls on a cache in pages: sizes, types, layouts, strides, sharing of heads, missing pages and empty
rows at random, each result against the plain forms of paged_plain."""
import numpy as np
import pytest
import torch

from tests import attention_plain as plain
from tests import paged_plain as pp

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def _room(rng, gen, shape, dtype, by_row):
    """A [pages, heads, page, d] cache inside something larger, with numbers in it."""
    pages, heads, page, d = shape
    step = 16 // dtype.itemsize
    wide = -(-d // step) * step + step * int(rng.integers(0, 2))
    more = int(rng.integers(0, 2))
    if by_row:
        t = torch.randn((pages + 1, page, heads + more, wide), generator=gen).to(dtype).cuda()[1:, :, more:].transpose(1, 2)
    else:
        t = torch.randn((pages + 1, heads + more, page, wide), generator=gen).to(dtype).cuda()[1:, more:]
    return t[..., :d]


def _tokens(rng, gen, n, heads, d, dtype):
    """[n, heads, d] inside something larger, at any alignment."""
    a, b = int(rng.integers(0, 3)), int(rng.integers(0, 3))
    return torch.randn((n, heads + a, d + b), generator=gen).to(dtype).cuda()[:, a:, b:]


@pytest.mark.parametrize("seed", range(40))
def test_random_steps(seed):
    from paper_2311_00368_b200 import binding as b
    rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    dtype = (torch.float32, torch.bfloat16)[int(rng.integers(0, 2))]
    R, page = int(rng.integers(1, 12)), int(rng.choice([1, 3, 8, 16, 16, 24, 32, 64, 100]))
    Hkv = int(rng.choice([1, 2, 3, 8]))
    H = Hkv * int(rng.choice([1, 2, 3, 4, 7, 8, 12, 20]))
    d = int(rng.choice([1, 8, 33, 64, 64, 80, 128, 128, 200, 256]))
    longest = int(rng.choice([1, 5, 40, 300, 2500]))
    lengths = rng.integers(0, longest + 1, R)
    added = rng.choice([-1, 0, 1, 1, 1, 4, 30], R)
    owned = -(-lengths // page)
    width = int((lengths + np.maximum(added, 0)).max() // page) + int(rng.integers(0, 2))    # (sometimes too narrow)
    width = max(width, int(owned.max()), 1)
    spare = int(rng.integers(0, 2 * R + 40 // page + 1))
    pages = int(owned.sum()) + spare + 1
    order = rng.permutation(pages)
    tables, at = np.full((R, width), -1), 0
    for r in range(R):
        tables[r, :owned[r]] = order[at:at + owned[r]]
        at += owned[r]
    stack = np.concatenate((order[at:at + spare], np.full(int(owned.sum()), -5)))
    if rng.random() < 0.2 and owned.sum():
        r = int(rng.choice(np.nonzero(owned)[0]))
        tables[r, int(rng.integers(0, owned[r]))] = int(rng.choice([-1, pages, 1 << 30]))     # a page that is missing
    tokens = max(0, int(np.maximum(added, 0).sum()) + int(rng.integers(-2, 4)))

    t, s = _int(tables), _int(stack)
    got = b.paged_tables(_int(lengths), _int(added), t, s, _int([spare]), page, pages, tokens)
    want, want_t, want_s = pp.step(lengths.tolist(), added.tolist(), tables.tolist(), stack.tolist(), spare, page, pages, tokens)
    assert [x.tolist() for x in got] == want and t.tolist() == want_t and s.tolist() == want_s
    after, row_ptr, rows, seen, slots, _ = got

    by_row = rng.random() < 0.4
    kp, vp = (_room(rng, gen, (pages, Hkv, page, d), dtype, by_row) for _ in range(2))
    means = _room(rng, gen, (pages, Hkv, 1, d), dtype, False)[:, :, 0]
    k, v, q = (_tokens(rng, gen, tokens, h, d, dtype) for h in (Hkv, Hkv, H))
    want_k, want_v, want_m = (x.cpu().clone() for x in (kp, vp, means))
    b.paged_write(k, v, row_ptr, _int(lengths), t, kp, vp, means, dtype=dtype)
    touched = {}
    for i, slot in enumerate(want[4]):
        if slot >= 0:
            c, r = divmod(slot, page)
            want_k[c, :, r], want_v[c, :, r] = k[i].cpu(), v[i].cpu()
            touched[c] = max(touched.get(c, 0), r + 1)
    assert torch.equal(kp.cpu(), want_k) and torch.equal(vp.cpu(), want_v)
    half = plain.U if dtype == torch.float32 else 2.0 ** -8
    for c in range(pages):
        if c in touched:
            x = want_k[c, :, :touched[c]].double()
            off = (touched[c] + 2) * plain.U * x.abs().mean(1) + half * x.mean(1).abs()
            assert ((means[c].cpu().double() - x.mean(1)).abs() <= off + 1e-40).all()
        else:
            assert torch.equal(means[c].cpu(), want_m[c])

    ptr, col = b.paged_lists(t, seen, page, pages, sum(want[3]) + 5, rows=rows)
    flat, ends = [], [0]
    for i in range(tokens):
        at = want[2][i]
        flat += [want_t[at][p // page] * page + p % page if 0 <= want_t[at][p // page] < pages else -1 for p in range(want[3][i])]
        ends.append(len(flat))
    assert ptr.tolist() == ends and col.tolist() == flat + [-1] * 5

    first, last = int(rng.integers(0, 2)), int(rng.integers(0, 3))
    keep = max(1, first + last) + int(rng.integers(0, 6))
    lists = b.paged_select(q, means, t, seen, page, keep, first, last, rows=rows, dtype=dtype)
    assert torch.equal(lists.cpu(), pp.select(q, means, t, seen, page, keep, first, last, rows))
    scale = float(rng.choice([d ** -0.5, 0.3, -0.1]))
    for what in (None, lists):
        o, lse = b.attention_paged(q, kp, vp, t, seen, rows=rows, lists=what, scale=scale, dtype=dtype)
        for i, (wo, wl, bo, bl) in enumerate(pp.attention(q, kp, vp, t, seen, rows, what, scale)):
            assert plain.inside(lse[i].cpu(), wl, bl) <= 1, i
            assert plain.inside(o[i].cpu(), wo, bo) <= 1, i

"""Attention over pages where values are not finite: rows that a token does not see stay out of what it gets, whatever they hold and whichever tokens share
them, and what is not finite in one column takes nothing from the others; and that weights keep their bits."""
import numpy as np
import pytest
import torch

from tests import attention_plain as plain
from tests import paged_plain as pp

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _caches(seed, requests, longest, Hkv, d, page, dtype):
    from paper_2311_00368_b200 import binding as b
    gen = torch.Generator().manual_seed(seed)
    width = -(-longest // page)
    tables = torch.randperm(requests * width, generator=gen).view(requests, width).to(torch.int32).cuda()
    caches = [b.paged_cache(requests * width, Hkv, page, d, dtype) for _ in range(2)]
    for c in caches:
        c.copy_(torch.randn(c.shape, generator=gen).to(dtype))
    return tables, *caches, gen


def _check(q, k, v, tables, seen, rows, dtype, lists=None):
    """O and lse of the call: infinities and NaN where a value that a token sees is one, and everything else as without them."""
    from paper_2311_00368_b200 import binding as b
    o, lse = b.attention_paged(q, k, v, tables, seen, rows=rows, lists=lists, dtype=dtype)
    again = b.attention_paged(q, k, v, tables, seen, rows=rows, lists=lists, dtype=dtype)
    assert torch.equal(o.nan_to_num(7.0), again[0].nan_to_num(7.0)) and torch.equal(lse, again[1])
    page, group = v.shape[2], q.shape[1] // v.shape[1]
    of = list(range(q.shape[0])) if rows is None else rows.tolist()
    seen_of = seen.tolist()
    v_host, table = v.cpu().float(), tables.tolist()
    for i, (want, want_lse, bound, bound_lse) in enumerate(pp.attention(q, k, v, tables, seen, rows, lists)):
        for g in range(v.shape[1]):
            at = pp.positions(table, of[i], seen_of[i], page, v.shape[0], None if lists is None else lists[i, g].tolist())
            if at:
                c, r = (torch.tensor(x) for x in zip(*at))
                odd = v_host[c, g, r].double()
                odd = torch.where(odd.isfinite(), 0.0, odd).sum(0)        # inf - inf and NaN: NaN
                want[g * group:(g + 1) * group, odd != 0] = odd[odd != 0]  # (NaN != 0)
        assert plain.inside(lse[i].cpu(), want_lse, bound_lse) <= 1, i
        assert plain.inside(o[i].cpu(), want, bound) <= 1, i


# heads, key heads, width, rows of a page: groups that several tokens share a unit with, each width class, pages that are whole tiles and such that are not
SHAPES = [(4, 1, 64, 16), (2, 2, 64, 32), (4, 2, 128, 16), (6, 2, 80, 24), (1, 1, 128, 7), (8, 1, 256, 16), (2, 1, 200, 5), (3, 1, 256, 64)]


@pytest.mark.parametrize("H,Hkv,d,page", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_token_gets_nothing_of_rows_that_only_later_ones_see(H, Hkv, d, page, dtype):
    """Guessed tokens of which later ones' values are not finite: whole units, and rows so long that they are cut into parts."""
    for longest, requests in ((50, 3), (5000, 1)):
        tables, k, v, gen = _caches(d + page, requests, longest, Hkv, d, page, dtype)
        rows = [r for r in range(requests) for _ in range(7)]
        seen = [longest - 6 + i % 7 - 3 * r for i, r in enumerate(rows)]
        q = torch.randn((len(rows), H, d), generator=gen).to(dtype).cuda()
        at = lambda r, p: (int(tables[r, p // page]), slice(None), p % page)  # noqa: E731
        for r in range(requests):
            last = longest - 1 - 3 * r
            v[at(r, last)] = float("nan")                                 # seen by the last token alone
            v[at(r, last - 2)][:, d // 2] = float("inf")                  # by the last three
            v[at(r, last - 3)][:, d - 1] = -float("inf")
            k[at(r, last)][:, 0] = float("nan")
        want_last = slice(6, None, 7)
        k_seen = k.clone()
        for r in range(requests):
            k_seen[at(r, longest - 1 - 3 * r)] = 0
        # (a key that is NaN makes all that the last token gets NaN; the others' are checked as if it were any number)
        from paper_2311_00368_b200 import binding as b
        o, lse = b.attention_paged(q, k, v, tables, _int(seen), rows=_int(rows), dtype=dtype)
        assert torch.isnan(o[want_last]).all() and torch.isnan(lse[want_last]).all()
        o2, lse2 = b.attention_paged(q, k_seen, v, tables, _int(seen), rows=_int(rows), dtype=dtype)
        others = [i for i in range(len(rows)) if i % 7 != 6]
        assert torch.equal(lse[others], lse2[others]) and torch.equal(o[others].nan_to_num(7.0), o2[others].nan_to_num(7.0))
        _check(q, k_seen, v, tables, _int(seen), _int(rows), dtype)


@pytest.mark.parametrize("H,Hkv,d,page", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_of_one_request_in_any_order(H, Hkv, d, page, dtype):
    """Neighbours of which the first sees most, some see nothing, and some are of no request; values that are not finite all over the rows."""
    tables, k, v, gen = _caches(d, 2, 300, Hkv, d, page, dtype)
    rows = [0, 0, 0, 0, 0, 0, 0, 0, 1, 1, -1, -1, 1, 0, 0, 1, 1, 1, 1]
    seen = [300, 20, 0, 7, 299, 100, 33, 1, 0, 50, 9, 9, 290, 64, 65, 16, 300, 2, 15]
    q = torch.randn((len(rows), H, d), generator=gen).to(dtype).cuda()
    for n, (r, p) in enumerate([(0, 298), (0, 90), (0, 63), (0, 5), (1, 299), (1, 288), (1, 14), (1, 15)]):
        v[int(tables[r, p // page]), n % Hkv, p % page, (n * 37) % d] = (float("inf"), float("nan"), -float("inf"))[n % 3]
    _check(q, k, v, tables, _int(seen), _int(rows), dtype)
    _check(q[:8], k, v, tables, _int(seen[:8]), _int(rows[:8]), dtype)
    lists = torch.stack([torch.randperm(tables.shape[1], generator=gen)[:5] for _ in range(len(rows) * Hkv)]).view(len(rows), Hkv, 5).to(torch.int32).cuda()
    _check(q, k, v, tables, _int(seen), _int(rows), dtype, lists)

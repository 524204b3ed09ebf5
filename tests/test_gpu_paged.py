"""A cache in pages: tables and lists number by number, rows and means that are written, the choice of pages, and attention over it against the
formula in 64 bits (bounds of attention_plain; nothing in these kernels rounds but the results, so r is their half step alone)."""
import numpy as np
import pytest
import torch

from tests import attention_plain as plain
from tests import paged_plain as pp

pytestmark = pytest.mark.gpu
U = plain.U


def _binding():
    from paper_2311_00368_b200 import binding
    return binding


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- tables ----------------------------------------------------------------------------------------------------------------------
def _check_step(lengths, added, tables, stack, count, page, pages, tokens):
    b = _binding()
    t, s = _int(tables), _int(stack)
    keep = [x.clone() for x in (_int(lengths), _int(added), _int([count]))]
    got = b.paged_tables(*keep[:2], t, s, keep[2], page, pages, tokens)
    want, want_t, want_s = pp.step(lengths, added, tables, stack, count, page, pages, tokens)
    for name, x, y in zip(("lengths", "row_ptr", "rows", "seen", "slots", "counts"), got, want):
        assert x.tolist() == y, name
    assert t.tolist() == want_t and s.tolist() == want_s
    again = b.paged_tables(*keep[:2], t, s, keep[2], page, pages, tokens)      # the same step once more: the same
    assert all(torch.equal(x, y) for x, y in zip(got, again)) and t.tolist() == want_t and s.tolist() == want_s
    return got


def _requests(seed, R, longest, page, width, spare, kinds):
    rng = np.random.default_rng(seed)
    lengths = [int(rng.integers(0, longest + 1)) for _ in range(R)]
    added = [int(rng.choice(kinds)) for _ in range(R)]
    owned = [-(-n // page) for n in lengths]
    order = rng.permutation(sum(owned) + spare).tolist()
    tables, at = [], 0
    for n in owned:
        tables.append(order[at:at + n] + [-7] * (width - n))
        at += n
    room = order[at:] + [-9] * (sum(owned))
    return lengths, added, tables, room, spare, page, len(order)


@pytest.mark.parametrize("seed,R,longest,page,width,spare,kinds,tokens", [
    (0, 1, 0, 1, 4, 4, [1], 1),
    (1, 1, 17, 16, 2, 1, [1], 3),
    (2, 64, 300, 64, 8, 64, [1], 64),
    (3, 37, 100, 7, 40, 300, [-1, 0, 1, 5, 60], 2000),
    (4, 300, 50, 16, 9, 900, [-1, 1, 33], 4000),
    (5, 513, 40, 5, 30, 4000, [-1, 0, 1, 70], 20000),
    (6, 1025, 9, 4, 6, 3000, [-1, 1, 2], 1500),           # fewer places than tokens
    (7, 8192, 6, 3, 4, 9000, [-1, 0, 1], 6000),           # the most requests
    (8, 50, 90, 10, 9, 20, [-1, 1, 30], 600),             # tables too narrow, and not enough pages
    (9, 20, 60, 8, 12, 0, [-1, 9], 300),                  # pages of requests that end are all there is
    (10, 12, 30, 1, 40, 100, [3], 0),                     # no room at all
])
def test_tables(seed, R, longest, page, width, spare, kinds, tokens):
    _check_step(*_requests(seed, R, longest, page, width, spare, kinds), tokens)


def test_tables_of_nothing():
    b = _binding()
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    got = b.paged_tables(none, none, none.view(0, 4), _int([5, 6]), _int([2]), 16, 8, 3)
    assert [x.tolist() for x in got] == [[], [0], [-1] * 3, [0] * 3, [-1] * 3, [2, 0, 0, 0]]


def test_tables_with_numbers_that_make_no_sense():
    """Entries and free pages outside the cache, lengths below 0 and beyond the tables, a count beyond the array, huge numbers of new tokens."""
    _check_step([5, -3, 100, 4], [1, 2, 1, -1], [[0, 99, -1], [-1] * 3, [3, -5, 1 << 30], [7, 2, 1]], [6, 77, -2, 4], 9, 2, 8, 6)
    _check_step([0, 3], [2 ** 31 - 1, 2 ** 31 - 1], [[-1] * 4, [1, 0, -1, -1]], [2, 3, 4], 3, 2, 8, 9)


def test_tables_layouts_and_outputs():
    """Tables that are a slice of wider ones; results into the caller's tensors; the next step's count is the last one's."""
    b = _binding()
    room = torch.full((3, 10), -3, dtype=torch.int32, device="cuda")
    free, count = _int([0, 1, 2, 3, 4, 5]), _int([6])
    out = tuple(torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (3, 4, 5, 5, 5, 4))
    got = b.paged_tables(_int([0, 0, 0]), _int([3, 1, 0]), room[:, 2:6], free, count, 2, 6, 5, out=out)
    assert all(x is y for x, y in zip(got, out))
    assert room.tolist() == [[-3, -3, 5, 4] + [-3] * 6, [-3, -3, 3] + [-3] * 7, [-3] * 10]
    assert [x.tolist() for x in out] == [[3, 1, 0], [0, 3, 4, 4], [0, 0, 0, 1, -1], [1, 2, 3, 1, 0], [10, 11, 8, 6, -1], [3, 4, 0, 3]]
    after = b.paged_tables(out[0], _int([1, -1, 2]), room[:, 2:6], free, out[5][:1], 2, 6, 5)
    assert after[0].tolist() == [4, 0, 2] and after[5].tolist() == [3, 3, 0, 1] and room[2, 2] == 3 and free.tolist() == [0, 1, 2, 3, 4, 5]
    with pytest.raises(b.B2spError):
        b.paged_tables(out[0], _int([1, 1, 1]), room[:, 2:6], free, count, 2, 6, 5, out=out)


@pytest.mark.parametrize("seen,page,rows", [
    ([0], 4, None), ([1], 1, None), ([5, 0, 0, 9], 4, [3, 1, 2, 0]), ([40] * 33 + [0] * 70 + [2], 16, None), ([1] * 3000, 8, None),
    ([0] * 2000 + [1, 0, 3], 5, None), ([2000, 1, 3000], 24, [2, -1, 0]), ([100, 7000], 150, [1, 1]), ([3] * 1100 + [1500], 64, None), ([2, 0, 5] * 3000 + [40], 4, None),
])
@pytest.mark.parametrize("slack", [0, 37, -1])
def test_lists(seen, page, rows, slack):
    b = _binding()
    rng = np.random.default_rng(len(seen))
    width, M = max(seen) // page + 1, len(seen)
    R = M if rows is None else max(rows) + 1
    pages = R * width + 3
    tables = rng.permutation(pages)[:R * width].reshape(R, width).astype(np.int32)
    tables[rng.random((R, width)) < 0.05] = pages + 1
    at = list(range(M)) if rows is None else rows
    lists = [[int(c) * page + p % page if 0 <= (c := tables[at[i]][p // page]) < pages else -1 for p in range(n)] if 0 <= at[i] < R else []
             for i, n in enumerate(seen)]
    flat = sum(lists, [])
    entries = len(flat) + slack if slack >= 0 else len(flat) // 2
    ends = np.minimum(np.cumsum([0] + [len(x) for x in lists]), entries).tolist()
    ptr, col = b.paged_lists(_int(tables.tolist()), _int(seen), page, pages, entries, rows=None if rows is None else _int(rows))
    assert ptr.tolist() == ends and col.tolist() == (flat + [-1] * max(0, slack))[:entries]


# ---- writing ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("lengths,added,H,d,page,layout", [
    ([0], [1], 1, 1, 1, "head"), ([3, 0, 15], [1, 1, 1], 2, 64, 16, "head"), ([0, 70, 5], [130, 0, 59], 3, 128, 64, "row"),
    ([9, 0, 2], [40, 1, 0], 2, 33, 7, "head"), ([100] * 40, [1] * 40, 8, 80, 24, "row"), ([5, 6], [1000, 3], 1, 256, 150, "head"), ([1], [9], 2, 1000, 4, "row"),
])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("wide", [True, False])
def test_write(lengths, added, H, d, page, layout, dtype, wide):
    b = _binding()
    gen = torch.Generator().manual_seed(d)
    R, T = len(lengths), sum(added)
    width = max(n + m for n, m in zip(lengths, added)) // page + 1
    pages = R * width + 2
    order = torch.randperm(pages, generator=gen).tolist()
    tables = [order[r * width:(r + 1) * width] for r in range(R)]
    shape = (pages, H, page, d) if layout == "head" else (pages, page, H, d)
    step = 16 // dtype.itemsize
    room = torch.randn(shape[:3] + (-(-d // step) * step + step,), generator=gen).to(dtype)   # (what lies behind d stays)
    kr, vr = room.cuda(), (-room).cuda()
    mr = torch.randn((pages, H, -(-d // step) * step), generator=gen).to(dtype).cuda()
    view = (lambda t: t[..., :d]) if layout == "head" else (lambda t: t.transpose(1, 2)[..., :d])
    kv = torch.randn((T + 1, 2, H, d + (0 if wide else 1)), generator=gen).to(dtype)[..., :d]
    k, v = kv[:T, 0].cuda() if wide else kv.cuda()[:T, 0], kv.cuda()[:T, 1]
    ptr = np.cumsum([0] + added).tolist()
    want_k, want_v, want_m, off = view(kr).cpu().clone(), view(vr).cpu().clone(), mr.cpu().double(), torch.zeros((pages, H, mr.shape[2]), dtype=torch.float64)
    for r in range(R):
        touched = set()
        for j in range(added[r]):
            c, i = divmod(lengths[r] + j, page)
            want_k[tables[r][c], :, i], want_v[tables[r][c], :, i] = k[ptr[r] + j].cpu(), v[ptr[r] + j].cpu()
            touched.add(c)
        for c in touched:
            n = min(page, lengths[r] + added[r] - c * page)
            x = want_k[tables[r][c], :, :n].double()
            want_m[tables[r][c], :, :d] = x.mean(1)
            # sums of n terms in fp32 and the division: (n + 2) u sum|x| / n; the result's half step
            off[tables[r][c], :, :d] = (n + 2) * U * x.abs().mean(1) + (U if dtype == torch.float32 else 2.0 ** -8) * x.mean(1).abs()
    before = [t.clone() for t in (kr, vr)]
    b.paged_write(k, v, _int(ptr), _int(lengths), _int(tables), view(kr), view(vr), mr[..., :d], dtype=dtype)
    assert torch.equal(view(kr).cpu(), want_k) and torch.equal(view(vr).cpu(), want_v)
    assert torch.equal(kr[..., d:], before[0][..., d:]) and torch.equal(vr[..., d:], before[1][..., d:])
    assert ((mr.cpu().double() - want_m).abs() <= off).all()
    kr2, vr2 = before
    b.paged_write(k, v, _int(ptr), _int(lengths), _int(tables), view(kr2), view(vr2), dtype=dtype)      # without means
    assert torch.equal(kr2, kr) and torch.equal(vr2, vr)


def test_write_leaves_out_what_has_no_page():
    """Pages outside the cache, positions beyond the table, tokens beyond those there are, requests without new tokens."""
    b = _binding()
    kp, vp, m = b.paged_cache(4, 1, 2, 8), b.paged_cache(4, 1, 2, 8), b.paged_means(4, 1, 8)
    x = torch.arange(1, 8, device="cuda").float().view(7, 1, 1).repeat(1, 1, 8)
    tables = _int([[1, 9], [3, -1], [2, 0], [0, 2]])
    b.paged_write(x, 10 * x, _int([0, 3, 9, 9, 8]), _int([1, 0, 1, -5]), tables, kp, vp, m)
    # request 0: position 1 (page 1), 2 and 3 (no page); request 1: tokens 3 to 6, positions 0 and 1 (page 3), the others have no page
    assert kp[:, 0, :, 0].tolist() == [[0, 0], [0, 1], [0, 0], [4, 5]] and vp[:, 0, :, 3].tolist() == [[0, 0], [0, 10], [0, 0], [40, 50]]
    assert m[:, 0, 0].tolist() == [0, 0.5, 0, 4.5]


# ---- the choice of pages ---------------------------------------------------------------------------------------------------------
class Cache:
    """A cache with something in it: M tokens of R requests."""
    def __init__(self, seed, seen, H, Hkv, d, page, dtype=torch.bfloat16, rows=None, layout="head", spread=1.0, width=None):
        b = _binding()
        gen = torch.Generator().manual_seed(seed)
        M = len(seen)
        R = M if rows is None else max(rows) + 1
        self.page, width = page, max(1, -(-max(seen) // page)) if width is None else width
        pages = R * width + 2
        self.tables = torch.randperm(pages, generator=gen)[:R * width].view(R, width).to(torch.int32).cuda()
        self.seen, self.rows = _int(seen), None if rows is None else _int(rows)
        step = 16 // dtype.itemsize
        shape = ((pages, Hkv, page) if layout == "head" else (pages, page, Hkv)) + (-(-d // step) * step,)
        view = (lambda t: t[..., :d]) if layout == "head" else (lambda t: t.transpose(1, 2)[..., :d])
        self.k = view(torch.randn(shape, generator=gen).to(dtype).cuda())
        self.v = view((torch.randn(shape, generator=gen) * torch.exp(torch.randn(shape[:3] + (1,), generator=gen))).to(dtype).cuda())
        self.q = (torch.randn((M, H, d), generator=gen) * spread).to(dtype).cuda()
        self.means = b.paged_means(pages, Hkv, d, dtype)
        self.means.copy_(self.k.float().mean(2))
        self.dtype = dtype

    def select(self, keep, first=1, last=1, **more):
        return _binding().paged_select(self.q, self.means, self.tables, self.seen, self.page, keep, first, last, rows=self.rows, dtype=self.dtype, **more)

    def attend(self, lists=None, **more):
        return _binding().attention_paged(self.q, self.k, self.v, self.tables, self.seen, rows=self.rows, lists=lists, dtype=self.dtype, **more)

    def check_select(self, keep, first=1, last=1):
        got = self.select(keep, first, last)
        want = pp.select(self.q, self.means, self.tables, self.seen, self.page, keep, first, last, self.rows)
        assert torch.equal(got.cpu(), want)
        return got

    def check(self, lists=None, scale=None):
        o, lse = self.attend(lists, scale=scale)
        for i, (want, want_lse, bound, bound_lse) in enumerate(pp.attention(self.q, self.k, self.v, self.tables, self.seen, self.rows, lists, scale)):
            worst = plain.inside(lse[i].cpu(), want_lse, bound_lse)
            assert worst <= 1, (i, worst)
            worst = plain.inside(o[i].cpu(), want, bound)
            assert worst <= 1, (i, worst)
        again = self.attend(lists, scale=scale)
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
        return o, lse


@pytest.mark.parametrize("seen,H,Hkv,d,page,keep,first,last", [
    ([1], 1, 1, 64, 16, 1, 0, 0), ([200], 4, 1, 64, 1, 7, 2, 3), ([0, 16, 17, 160, 161], 8, 2, 128, 16, 4, 1, 2), ([700, 64, 650], 6, 3, 50, 24, 13, 1, 2),
    ([5000], 8, 8, 80, 2, 100, 0, 5), ([900], 2, 1, 256, 3, 299, 1, 1), ([9000, 8193], 2, 2, 17, 1, 33, 1, 1), ([300] * 70, 4, 4, 96, 5, 8, 3, 0),
    ([40, 3], 4, 2, 33, 8, 2, 0, 2), ([20000, 16385], 2, 1, 64, 1, 50, 1, 1), ([2049, 2048, 1025, 257, 256], 2, 1, 64, 1, 20, 0, 0),
])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select(seen, H, Hkv, d, page, keep, first, last, dtype):
    Cache(d + page, seen, H, Hkv, d, page, dtype).check_select(keep, first, last)


def test_select_ties_infinities_and_nan():
    c = Cache(1, [640, 630], 4, 2, 64, 16)
    c.means[:, :, :] = c.means[:1]                                        # all the same: the lower pages
    c.check_select(9)
    c.means[c.tables[0, 5].long(), 0, 3] = float("nan")
    c.means[c.tables[0, 6].long(), 1, 3] = float("inf")
    c.means[c.tables[1, 7].long(), 1, 3] = -float("inf")
    c.means[c.tables[1, 9].long(), 0] = 0.0
    c.means[c.tables[1, 12].long(), 0] = -0.0
    for keep in (2, 3, 20, 38, 39):
        c.check_select(keep)
    c.tables[0, 4], c.tables[0, 11] = -1, 1 << 20                        # no page: below all but NaN
    c.check_select(5)
    c.check_select(38)
    c.means.fill_(float("nan"))
    c.check_select(12)
    c.q.zero_()
    c.means.copy_(c.k.float().mean(2))
    c.check_select(7, 0, 0)


@pytest.mark.parametrize("n", [40, 600, 1500, 2300])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_between_close_scores(n, dtype):
    """Scores that sums in 32 bits cannot tell apart: means that differ in the last place of one element, in elements that weigh next to nothing,
    and not at all; some that are 0; scores that underflow or overflow in 32 bits."""
    c = Cache(3, [n * 4, n * 4 - 5], 4, 2, 64, 4, dtype)
    gen = torch.Generator().manual_seed(n)
    base = torch.randn((1, 2, 64), generator=gen).to(dtype).cuda()
    order = torch.randperm(n, generator=gen)
    for i in range(2):
        at = c.tables[i].long()
        c.means[at] = base
        step = torch.finfo(dtype).eps * base[0, :, 5].float().abs() * 2.0 ** -14     # far below the last place of a score
        c.means[at[order], :, 63] = ((torch.arange(n).cuda()[:, None] // 2 - n // 4) * step).to(dtype)
    for keep in (3, 17, n // 2, n - 1):
        c.check_select(keep)
    c.means[c.tables[0, ::3].long()] = 0
    c.means[c.tables[1, 1::2].long(), 1] = -0.0
    for keep in (5, n // 3, n - 2):
        c.check_select(keep)
    keep_q = c.q.clone()
    for f in (2.0 ** -100, 2.0 ** 100):
        c.q, means = (keep_q.float() * f).to(dtype), c.means.clone()
        c.means.copy_((means.float() * f).to(dtype))
        c.check_select(n // 2)
        c.means.copy_(means)


@pytest.mark.parametrize("n", [33, 256, 257, 1500, 2048, 3000, 9000, 17000])
def test_select_scores_of_any_spread(n):
    """Scores that are far apart, far out, all alike, tiny, or of pages that are not there: one query of a one, so that a score is a number of the mean."""
    c = Cache(5, [n] * 8, 2, 2, 8, 1, torch.float32)
    gen = torch.Generator().manual_seed(n)
    c.q[:] = 0
    c.q[:, :, 0] = 1
    x = torch.randn((8, n, 2), generator=gen)
    x[0] = torch.exp(x[0] * 8)                                            # over 20 decades
    x[1, n // 2] = 1e4                                                    # far out, to either side
    x[1, n // 3] = -1e4
    x[2] = 3.25                                                           # all alike
    x[3] = torch.exp(x[3] * 3) * 1e-44                                    # multiples of the smallest number
    x[4] = (x[4] * 2).round()                                             # many alike
    x[5] = -torch.exp(x[5])                                               # below zero, a page above it
    x[5, n - 2] = 1.5
    x[6] = 1 + (torch.arange(n).flip(0)[:, None] % 4096) * 2.0 ** -23     # neighbouring numbers
    for i in range(8):
        c.means[c.tables[i].long(), :, 0] = x[i].cuda()
    gone = torch.randperm(n, generator=gen)[:n - 5]
    c.tables[7, gone.cuda()] = -1                                         # hardly a page is there
    x[7, gone] = -float("inf")
    score = x.double().numpy()
    for keep, first, last in ((2, 1, 1), (3, 1, 1), (32, 0, 0), (32, 5, 20), (n // 2 + 10, 1, 1), (n - 1, 0, 1)):
        got = c.select(keep, first, last).cpu().numpy()
        for i in range(8):
            for g in range(2):
                y = score[i, :, g].copy()
                y[:first] = y[n - last:] = np.inf
                assert (got[i, g] == np.sort(np.lexsort((np.arange(n), -y))[:keep])).all(), (i, g, keep)


def test_select_rows_and_layout():
    c = Cache(2, [300, 299, 298, 0, 120, 500], 4, 2, 64, 16, rows=[1, 1, 1, 0, -1, 2])
    c.check_select(6)
    wide = torch.randn((6, 3, 4, 64), device="cuda").to(torch.bfloat16)
    c.q = wide[:, 1]                                                      # a slice of a projection
    both = torch.randn((c.means.shape[0], 2, 2, 72), device="cuda").to(torch.bfloat16)
    c.means = both[:, 1, :, :64]
    c.check_select(6)
    c.rows[0] = 7
    assert (c.check_select(6)[0] == -1).all()


# ---- attention -------------------------------------------------------------------------------------------------------------------
CASES = [
    ([1], 1, 1, 64, 1), ([15, 16, 17, 0, 1], 4, 2, 128, 16), ([70, 0, 64, 65, 3, 500], 8, 1, 64, 64), ([129, 1000], 16, 1, 32, 24),
    ([300, 20, 7], 20, 1, 96, 7), ([200, 31], 6, 2, 17, 150), ([5000], 8, 2, 128, 64), ([40] * 33, 32, 8, 80, 16), ([3000, 10, 0, 800], 40, 1, 128, 128),
    ([2, 0, 4, 1] * 30, 4, 4, 128, 5), ([1, 3] * 100 + [3000], 8, 2, 64, 16), ([500, 90], 4, 2, 256, 32), ([77, 260], 9, 3, 200, 11), ([33], 2, 2, 1, 4),
    ([700] * 3, 64, 1, 64, 64), ([900, 3, 0, 2000], 16, 1, 256, 64), ([300, 70], 48, 1, 200, 24), ([5, 1500], 100, 2, 128, 32), ([40], 1000, 1, 64, 16),
]


@pytest.mark.parametrize("seen,H,Hkv,d,page", CASES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_paged(seen, H, Hkv, d, page, dtype):
    Cache(len(seen) + d, seen, H, Hkv, d, page, dtype, layout="row" if d % 3 else "head").check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,d,page", [(4, 1, 64, 16), (2, 2, 128, 16), (6, 2, 80, 24), (16, 2, 64, 64), (3, 1, 256, 7)])
def test_attention_tokens_of_one_request(H, Hkv, d, page, dtype):
    """Neighbouring tokens of a request read its rows together, whatever each sees; rows in any order, tokens of no request among them."""
    rows = [0] * 4 + [1] * 4 + [2] * 3 + [3] * 7 + [1, 2, -1, -1, 3, 3, 0, 0, 0, 2] + [4] * 17
    rng = np.random.default_rng(H)
    seen = [int(x) for x in np.concatenate([np.arange(97, 101), rng.integers(0, 300, len(rows) - 4)])]
    seen[7] = seen[12] = 0
    Cache(H + d, seen, H, Hkv, d, page, dtype, rows=rows).check()
    Cache(H + d, [5 + i for i in range(16)], H, Hkv, d, page, dtype, rows=[0] * 16).check()
    # every token of one long row, cut into many parts
    Cache(H + d, [3000 + i for i in range(9)], H, Hkv, d, page, dtype, rows=[0] * 9).check()


def test_attention_logits_far_below_zero():
    for dtype in (torch.float32, torch.bfloat16):
        c = Cache(16, [300, 40], 4, 2, 64, 16, dtype)
        c.k.copy_(-c.k.abs() - 20)
        c.q.copy_(c.q.abs() + 20)
        c.check(scale=1.0)                                               # products of about -28000


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_paged_large_logits_and_scales(dtype):
    Cache(5, [2000, 300], 8, 2, 64, 16, dtype, spread=6.0).check()
    Cache(6, [200, 100], 8, 2, 64, 16, dtype).check(scale=-0.3)
    Cache(7, [200, 100], 8, 2, 64, 16, dtype).check(scale=0.0)
    c = Cache(8, [900], 4, 1, 64, 16, dtype)
    # logits that grow along the row: the reference of the exponentials moves all the time
    grow = torch.linspace(0, 40, 912, device="cuda").view(57, 16)
    c.k[c.tables[0].long(), 0] = (grow[..., None] * c.q[0, 0].float() / c.q[0, 0].float().square().sum()).to(dtype)
    c.check(scale=1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("seen,H,Hkv,d,page,keep", [
    ([640, 600, 3, 0], 8, 2, 128, 16, 5), ([700, 64, 650], 6, 3, 50, 24, 13), ([333], 16, 1, 96, 7, 20), ([8000], 8, 8, 64, 64, 32),
])
def test_attention_over_selected_pages(seen, H, Hkv, d, page, keep, dtype):
    c = Cache(keep, seen, H, Hkv, d, page, dtype)
    c.check(c.check_select(keep, 1, 2))


def test_attention_lists_of_any_kind():
    """Pages twice, out of order, not seen, outside the table, and gaps in between."""
    c = Cache(9, [100, 50, 33], 4, 2, 64, 16)
    c.check(_int([[[3, 3, 0, -1, 6, 9], [-1, -1, -1, -1, 2, 1]], [[3, 4, 0, 1, 2, 100000], [-1] * 6], [[2, 1, 0, 2, 2, 2], [6, 5, 4, 3, -9, 2]]]))


def test_attention_sees_nothing_of_what_is_not_there():
    """NaN in rows behind the last position, in other pages and heads' padding; missing pages; requests that are none; lengths out of range."""
    for dtype in (torch.float32, torch.bfloat16):
        for d, page in ((64, 16), (40, 7), (33, 24)):
            c = Cache(10, [100, 37, 16, 5, 9], 4, 2, d, page, dtype, rows=[0, 1, 2, -1, 3], width=20)
            used = torch.zeros(c.k.shape[0], page, dtype=torch.bool)
            for i, n in ((0, 100), (1, 37), (2, 16), (4, 9)):
                row = 3 if i == 4 else i
                for p in range(n):
                    used[c.tables[row, p // page], p % page] = True
            for t in (c.k, c.v):
                base = t._base if t._base is not None else t
                base[..., d:] = float("nan")
                t.masked_fill_(~used.cuda()[:, None, :, None], float("nan"))
            o, _ = c.check()
            assert torch.isfinite(o.float()).all() and (o[3] == 0).all()
            c.tables[0, 1], c.tables[1, 0] = -1, 1 << 20
            c.check()
            c.seen[2], c.seen[4] = -4, 0
            o, lse = c.check()
            assert (o[2:] == 0).all() and (lse[2:] == -np.inf).all()
            c.tables.fill_(-1)
            assert (c.attend()[0] == 0).all()


def test_attention_nan_and_infinities_that_are_seen():
    for dtype in (torch.float32, torch.bfloat16):
        c = Cache(11, [50, 50, 50, 50], 2, 1, 64, 16, dtype)
        at = lambda i, p: (int(c.tables[i, p // 16]), 0, p % 16)  # noqa: E731
        c.k[at(0, 7)][3] = float("nan")
        c.v[at(1, 20)][5] = float("inf")
        c.q[2, 0] = float("nan")
        c.k[int(c.tables[3, 0]):int(c.tables[3, 0]) + 1, 0, 4, :] = 0
        c.q[3] = 0
        c.q[3, :, 0] = 1
        c.k[at(3, 9)][0] = -float("inf")                                  # a weight of zero
        o, lse = c.attend()
        assert torch.isnan(o[0]).all() and torch.isnan(lse[0]).all()
        assert (o[1, :, 5] == np.inf).all() and torch.isfinite(o[1, :, :5]).all() and torch.isfinite(lse[1]).all()
        assert torch.isnan(o[2, 0]).all() and torch.isfinite(o[2, 1].float()).all()
        assert torch.isfinite(o[3].float()).all() and torch.isfinite(lse[3]).all()
        c.k[:] = 0
        c.k[..., 0] = -float("inf")
        o, lse = c.attend()
        assert (o[3] == 0).all() and (lse[3] == -np.inf).all()            # all products -inf


def test_attention_other_layouts():
    """Q a slice of a projection at odd addresses, O inside a larger tensor, keys and values side by side in one tensor, tables shared by stride 0."""
    for dtype in (torch.float32, torch.bfloat16):
        c = Cache(12, [90, 80, 70], 4, 2, 40, 16, dtype, rows=[0, 1, 2])
        wide = torch.randn((3, 4 * 43 + 1), device="cuda").to(dtype)
        c.q = wide[:, 1:].view(3, 4, 43)[..., 1:41]
        both = torch.randn((20, 16, 2, 2, 40), device="cuda").to(dtype)
        c.k, c.v = both[:, :, :, 0].transpose(1, 2), both[:, :, :, 1].transpose(1, 2)
        c.tables = torch.randperm(20, device="cuda")[:6].to(torch.int32).expand(3, 6)
        o, lse = c.check()
        room = torch.full((3, 5, 47), 9.0, device="cuda").to(dtype)
        o2, lse2 = c.attend(out=room[:, 1:, 3:43], lse=torch.empty_like(lse))
        assert torch.equal(o2, o) and torch.equal(lse2, lse)
        room[:, 1:, 3:43] = 9
        assert (room == 9).all()
        c.q = c.q[:1].expand(3, 4, 40)                                   # one query for all
        c.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("seen,H,Hkv,d,rows", [([20000, 0, 5], 8, 2, 128, None), ([7] * 3000, 4, 2, 64, None), ([900, 3, 40, 40, 41] * 60, 20, 1, 50, None),
                                               ([300, 301, 302, 303] * 50, 2, 1, 64, [i // 4 for i in range(200)])])
def test_the_output_in_place_of_the_queries(seen, H, Hkv, d, rows, dtype):
    c = Cache(31, seen, H, Hkv, d, 16, dtype, rows=rows)
    o, lse = c.attend()
    room = torch.randn((len(seen), H + 3, d), device="cuda").to(dtype)     # queries among other heads
    room[:, 1:H + 1] = c.q
    before, c.q = room.clone(), room[:, 1:H + 1]
    got, got_lse = c.attend(out=c.q)
    assert got.data_ptr() == c.q.data_ptr() and torch.equal(got, o) and torch.equal(got_lse, lse)
    assert torch.equal(room[:, :1], before[:, :1]) and torch.equal(room[:, H + 1:], before[:, H + 1:])


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes and elements apart: pages near its end."""
    b = _binding()
    pages, page, d = (1 << 32) // (64 * 64) + 40, 64, 64
    k = torch.zeros((pages, 1, page, d), dtype=torch.bfloat16, device="cuda")
    small = Cache(13, [600, 128], 4, 1, d, page)
    n = small.k.shape[0]
    k[-n:].copy_(small.k)
    want = small.attend()
    big = b.attention_paged(small.q, k, k, small.tables + (pages - n), small.seen, dtype=torch.bfloat16)
    v = small.k
    small.v = v
    want = small.attend()
    assert torch.equal(big[0], want[0]) and torch.equal(big[1], want[1])
    new = torch.randn((2, 1, d), device="cuda").to(torch.bfloat16)
    b.paged_write(new, -new, _int([0, 1, 2]), _int([600, 128]), small.tables + (pages - n), k, k.clone(), dtype=torch.bfloat16)
    assert torch.equal(k[int(small.tables[0, 9]) + pages - n, 0, 600 % 64], new[0, 0])
    assert torch.equal(k[int(small.tables[1, 2]) + pages - n, 0, 0], new[1, 0])


# ---- calls beside each other -----------------------------------------------------------------------------------------------------
def test_captured_beside_another_graph():
    cs = [Cache(20 + i, [4000, 100], 8, 2, 128, 16) for i in range(2)]
    run = lambda c: (lists := c.select(20), *c.attend(lists), *c.attend())  # noqa: E731
    want = [run(c) for c in cs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in cs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(c))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(got, ref))


def test_given_workspaces():
    """Workspaces of just the size asked for, whatever they hold; nothing behind them is written, and their status word is in order."""
    b = _binding()
    for dtype in (torch.float32, torch.bfloat16):
        c = Cache(31, [3000, 40, 0, 700], 8, 2, 64, 16, dtype)
        lists, want = c.select(9), c.attend()
        for need, call in ((b.lib.b2sp_paged_select_workspace_bytes(4, 2, c.tables.shape[1]), lambda ws: (c.select(9, workspace=ws),)),
                           (b.lib.b2sp_attention_paged_workspace_bytes(4, 8, 2, 64), lambda ws: c.attend(workspace=ws))):
            room = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
            got = call(room[:need])
            assert all(torch.equal(x, y) for x, y in zip(got, (lists,) if len(got) == 1 else want))
            assert (room[need:] == 0xAB).all() and b.device_status(room) == 0
            with pytest.raises(b.B2spError):
                call(room[:need - 1])


def test_on_another_stream():
    c = Cache(30, [900, 30], 8, 2, 64, 16)
    want = c.attend()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = [c.attend() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(st)
    for o, lse in got:
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_server(dtype):
    """Steps of a server, prompts, new tokens, requests that end: tables, writing, attention over all pages and over selected ones; each step
    agrees with attention over the keys and values as the test kept them.  The graph of a step is replayed on new lengths."""
    b = _binding()
    gen = torch.Generator().manual_seed(40)
    R, H, Hkv, d, page, pages, room, width = 5, 4, 2, 64, 8, 64, 96, 16
    tables = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    free, count = torch.arange(pages, dtype=torch.int32, device="cuda"), _int([pages])
    kp, vp, means = b.paged_cache(pages, Hkv, page, d, dtype), b.paged_cache(pages, Hkv, page, d, dtype), b.paged_means(pages, Hkv, d, dtype)
    lengths, added = _int([0] * R), _int([0] * R)
    q, k, v = (torch.zeros((room, h, d), dtype=dtype, device="cuda") for h in (H, Hkv, Hkv))

    def step():
        after, row_ptr, rows, seen, slots, counts = b.paged_tables(lengths, added, tables, free, count, page, pages, room)
        b.paged_write(k, v, row_ptr, lengths, tables, kp, vp, means, dtype=dtype)
        o, lse = b.attention_paged(q, kp, vp, tables, seen, rows=rows, dtype=dtype)
        lists = b.paged_select(q, means, tables, seen, page, 4, rows=rows, dtype=dtype)
        few = b.attention_paged(q, kp, vp, tables, seen, rows=rows, lists=lists, dtype=dtype)
        return after, row_ptr, rows, seen, counts, o, lse, lists, few[0], few[1], slots

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    held = [[torch.zeros((0, Hkv, d), dtype=dtype)] * 2 for _ in range(R)]
    taken = 0
    for new in ([20, 0, 7, 1, 33], [1, 30, 1, 1, 1], [1, 1, -1, 1, -1], [1, 1, 40, 1, 25], [-1, 1, 1, 1, 1]):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen))
        added.copy_(torch.tensor(new, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        after, row_ptr, rows, seen, counts, o, lse, lists, few, few_lse, slots = out
        at = 0
        for r, n in enumerate(new):
            held[r] = [torch.zeros((0, Hkv, d), dtype=dtype)] * 2 if n < 0 else [torch.cat((x, y[at:at + n].cpu())) for x, y in zip(held[r], (k, v))]
            for j in range(max(n, 0)):
                see = held[r][0].shape[0] - n + j + 1
                assert int(seen[at + j]) == see and int(rows[at + j]) == r
                K, V = (x[:see].transpose(0, 1)[None] for x in held[r])
                for lst, got, got_lse in ((None, o, lse), (lists[at + j].tolist(), few, few_lse)):
                    mask = torch.ones((1, H, 1, see), dtype=torch.bool)
                    if lst is not None:
                        for h in range(H):
                            mask[0, h, 0] = torch.tensor([p // page in lst[h // (H // Hkv)] for p in range(see)])
                    want, want_lse, bound, bound_lse = plain.forward(mask, q[at + j].cpu().view(1, H, 1, d), K, V, d ** -0.5)
                    assert plain.inside(got[at + j].cpu().view(1, H, 1, d), want, bound) <= 1
                    assert plain.inside(got_lse[at + j].cpu().view(1, H, 1), want_lse, bound_lse) <= 1
            at += max(n, 0)
        assert after.tolist() == [x[0].shape[0] for x in held] and int(counts[1]) == at and int(counts[2]) == 0
        assert (o[at:] == 0).all() and (lse[at:] == -np.inf).all() and (lists[at:] == -1).all() and (slots[at:] == -1).all()
        taken = sum(-(-x[0].shape[0] // page) for x in held)
        assert int(counts[0]) == pages - taken
        assert sorted(free[:pages - taken].tolist() + [p for r in range(R) for p in tables[r, :-(-held[r][0].shape[0] // page)].tolist()]) == list(range(pages))
        lengths.copy_(after)
        count.copy_(counts[:1])


def test_the_4_bit_cache_by_pages():
    """Tables and lists in front of the 4-bit cache's calls: what kv4_write and attention_kv4 make of them is attention over the values held."""
    b = _binding()
    gen = torch.Generator().manual_seed(41)
    R, H, Hkv, d, page, pages = 3, 4, 2, 64, 16, 40
    tables = torch.full((R, 10), -1, dtype=torch.int32, device="cuda")
    free, count = torch.randperm(pages, generator=gen).to(torch.int32).cuda(), _int([pages])
    lengths, row_ptr, rows, seen, slots, counts = b.paged_tables(_int([0] * R), _int([50, 1, 100]), tables, free, count, page, pages, 160)
    assert counts.tolist() == [pages - 12, 151, 0, 12]
    x = torch.randn((2, 160, Hkv, d), generator=gen).cuda()
    caches = b.kv4_cache(Hkv, pages * page, d) + b.kv4_cache(Hkv, pages * page, d)
    b.kv4_write(x[0], slots, *caches[:2])
    b.kv4_write(x[1], slots, *caches[2:])
    q = torch.randn((R, H, d), generator=gen).to(torch.bfloat16).cuda()
    ptr, col = b.paged_lists(tables, lengths, page, pages, 200)
    assert torch.equal(ptr, row_ptr) and torch.equal(col[:151], slots[:151])
    o, lse = b.attention_kv4(ptr, col, q, *caches)
    held = [b.kv4_read(slots[:151], *c, d).to(torch.bfloat16) for c in (caches[:2], caches[2:])]
    kp, vp = b.paged_cache(pages, Hkv, page, d, torch.bfloat16), b.paged_cache(pages, Hkv, page, d, torch.bfloat16)
    b.paged_write(*held, row_ptr, _int([0] * R), tables, kp, vp, dtype=torch.bfloat16)
    want, want_lse = b.attention_paged(q, kp, vp, tables, lengths, dtype=torch.bfloat16)
    # the values held have up to 11 bits and are rounded to 8 here: K moves logits by at most 2^-9 sum|q k| scale (below 0.1 for these), V
    # and the results by 2 x 2^-8 of the largest |v|, the weights by the logits' e^0.2
    assert (lse - want_lse).abs().max() <= 0.1
    assert (o.float() - want.float()).abs().max() <= (0.25 + 2 * 2.0 ** -8) * held[1].float().abs().max()

"""Steps that find too few pages: a step on top of one does nothing and says so, no entry that is no page gets among the free ones, and the short step can be
made again from what it read, however many steps were queued behind it."""
import numpy as np
import pytest
import torch

from tests import paged_plain as pp

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server:
    def __init__(self, requests, width, page, pages):
        self.tables, self.free = _int([[-1] * width] * requests), _int(list(range(pages)))
        self.lengths, self.count, self.page, self.pages = _int([0] * requests), _int([pages]), page, pages

    def step(self, added, tokens, lengths=None, count=None):
        from paper_2311_00368_b200 import binding as b
        return b.paged_tables(self.lengths if lengths is None else lengths, _int(added), self.tables, self.free, self.count if count is None else count,
                              self.page, self.pages, tokens)

    def keep(self, out):
        self.lengths, self.count = out[0].clone(), out[5][:1].clone()

    def check(self):
        """Every page once, in a table or on the stack."""
        held = [p for t, n in zip(self.tables.tolist(), self.lengths.tolist()) for p in t[:-(-n // self.page)]]
        assert sorted(held + self.free[:int(self.count)].tolist()) == list(range(self.pages))


def test_a_token_behind_one_that_found_no_page():
    s = Server(1, 4, 16, 1)
    s.keep(s.step([16], 16))
    short = s.step([1], 1)
    assert short[0].tolist() == [17] and short[4].tolist() == [-1] and short[5].tolist() == [-1, 1, 1, 1]
    before = s.tables.clone(), s.free.clone()
    then = s.step([1], 2, short[0], short[5][:1])
    assert [x.tolist() for x in then] == [[17], [0, 0], [-1, -1], [0, 0], [-1, -1], [-1, 0, 1, 0]]
    assert torch.equal(s.tables, before[0]) and torch.equal(s.free, before[1])


def test_what_no_page_holds_does_not_become_a_free_page():
    """Two requests that fill the cache; one more token for one of them; then that one ends and another one wants twenty tokens."""
    s = Server(3, 4, 16, 2)
    s.keep(s.step([16, 16, 0], 32))
    short = s.step([1, 0, 0], 1)
    assert short[5].tolist() == [-1, 1, 1, 1]
    then = s.step([-1, 0, 20], 20, short[0], short[5][:1])
    assert then[0].tolist() == [17, 16, 0] and then[1].tolist() == [0] * 4 and then[4].tolist() == [-1] * 20 and then[5].tolist() == [-1, 0, 20, 0]
    again = s.step([-1, 0, 16], 20)                                        # the short step, made again
    assert again[5].tolist() == [0, 16, 0, 1] and (again[4][:16] >= 0).all()
    s.keep(again)
    s.check()


@pytest.mark.parametrize("R,pages,tokens", [(7, 12, 40), (300, 600, 3000), (8192, 2 * 8192, 9000)])
def test_steps_queued_behind_a_short_one(R, pages, tokens):
    """A captured step that reads its lengths and count from the step before: all behind a short one leave lengths, tables and stack as they are, write
    nothing and see nothing."""
    from paper_2311_00368_b200 import binding as b
    rng = np.random.default_rng(R)
    s = Server(R, 6, 4, pages)
    s.keep(s.step(rng.integers(0, 5, R).tolist(), 5 * R))
    s.check()
    added = rng.integers(-1, 12, R)
    want = pp.step(s.lengths.tolist(), added.tolist(), s.tables.tolist(), s.free.tolist(), int(s.count), 4, pages, tokens)
    assert want[0][5][0] < 0
    short = s.step(added.tolist(), tokens)
    assert [x.tolist() for x in short] == want[0] and s.tables.tolist() == want[1] and s.free.tolist() == want[2]
    kp, vp = b.paged_cache(pages, 1, 4, 8), b.paged_cache(pages, 1, 4, 8)
    x = torch.randn((tokens, 1, 8), device="cuda")
    lengths, count, new = short[0].clone(), short[5][:1].clone(), _int(added.tolist())
    run = lambda: (lambda out: (b.paged_write(x, x, out[1], lengths, s.tables, kp, vp),  # noqa: E731
                                *b.attention_paged(x, kp, vp, s.tables, out[3], rows=out[2]), *out))(
        b.paged_tables(lengths, new, s.tables, s.free, count, 4, pages, tokens))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for n in range(3):
        new.copy_(torch.from_numpy(rng.integers(-1, 3, R).astype(np.int32)))
        graph.replay()
        asked = int(new.clamp(min=0).sum())
        _, o, lse, after, ptr, rows, seen, slots, counts = out
        assert torch.equal(after, short[0]) and not ptr.any() and (rows == -1).all() and not seen.any() and (slots == -1).all()
        assert counts.tolist() == [want[0][5][0], 0, asked, 0]
        assert s.tables.tolist() == want[1] and s.free.tolist() == want[2]
        assert not kp.any() and not vp.any() and not o.any() and (lse == -np.inf).all()
        lengths.copy_(after)
        count.copy_(counts[:1])
    fewer = np.where(rng.random(R) < 0.6, -1, np.minimum(added, 1))        # made again, with fewer tokens and more room
    got = s.step(fewer.tolist(), tokens)
    want = pp.step(s.lengths.tolist(), fewer.tolist(), want[1], want[2], int(s.count), 4, pages, tokens)
    assert [x.tolist() for x in got] == want[0] and got[5][0] >= 0 and s.tables.tolist() == want[1] and s.free.tolist() == want[2]
    s.keep(got)
    s.check()

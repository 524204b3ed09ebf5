"""Refusals of the calls on a cache in pages: argument checks run before any CUDA call, so no GPU is needed."""
import pytest
import torch

from paper_2311_00368_b200 import build as b2sp_build

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 5


@pytest.fixture(scope="module")
def b():
    b2sp_build.build()
    from paper_2311_00368_b200 import binding
    return binding


def _tab(b, **other):
    base = dict(entries=4096, ld=16, requests=3, width=16)
    base.update(other)
    return b._PAGE_TABLES(*base.values())


def _cache(b, **other):   # 32 pages of 2 heads, 16 rows, d = 64
    base = dict(data=1 << 20, ld=64, stride_head=1024, stride_page=2048, pages=32, page=16)
    base.update(other)
    return b._PAGES(*base.values())


BAD_TABLES = (dict(entries=0), dict(requests=-1), dict(width=-1), dict(ld=-1))
BAD_CACHES = (dict(data=0), dict(data=(1 << 20) + 8), dict(ld=60), dict(ld=66), dict(stride_head=1026), dict(stride_page=2050), dict(pages=-1),
              dict(page=0), dict(stride_page=-16))


def test_tables(b):
    f = lambda t=None, pages=32, page=16, lengths=4096, added=8192, free=1 << 14, room=32, count=1 << 15, tokens=8, out=1 << 16, ptr=1 << 17,\
        rows=1 << 18, seen=1 << 19, slots=1 << 20, counts=1 << 21: b.lib.b2sp_paged_tables(  # noqa: E731
            t or _tab(b, entries=1 << 22), pages, page, lengths, added, free, room, count, tokens, out, ptr, rows, seen, slots, counts, None)
    for bad in BAD_TABLES + (dict(ld=15),):
        assert f(_tab(b, **bad)) == INVALID, bad
    assert b.lib.b2sp_paged_tables(None, 32, 16, *[4096] * 3, 32, 4096, 8, *[4096] * 6, None) == INVALID
    assert f(pages=-1) == f(page=0) == f(room=-1) == f(tokens=-1) == INVALID
    assert f(lengths=None) == f(added=None) == f(free=None) == f(count=None) == f(out=None) == f(ptr=None) == INVALID
    assert f(rows=None) == f(seen=None) == f(slots=None) == f(counts=None) == INVALID
    # read by one CTA, written by another
    assert f(out=4096) == f(out=4096 + 8) == f(counts=1 << 15) == f(counts=(1 << 15) - 12) == f(seen=8192) == f(ptr=(1 << 14) + 124) == INVALID
    assert f(slots=(1 << 22) + 4 * 47) == INVALID
    assert f(_tab(b, requests=8193)) == f(pages=1 << 27, page=16) == UNSUPPORTED


def test_lists(b):
    f = lambda M=3, t=None, pages=32, page=16, seen=4096, entries=9, ptr=1 << 16, col=1 << 17: b.lib.b2sp_paged_lists(  # noqa: E731
        M, t or _tab(b), pages, page, None, seen, entries, ptr, col, None)
    for bad in BAD_TABLES:
        assert f(t=_tab(b, **bad)) == INVALID, bad
    assert f(M=-1) == f(pages=-1) == f(page=0) == f(seen=None) == f(entries=-1) == f(ptr=None) == f(col=None) == INVALID
    assert f(ptr=4096 + 8) == f(col=4096 + 4) == f(t=_tab(b, entries=1 << 20), ptr=(1 << 20) + 8) == INVALID     # outputs in inputs
    assert f(entries=2 ** 31, seen=1 << 40) == f(pages=1 << 27, seen=1 << 40, t=_tab(b, entries=1 << 41)) == UNSUPPORTED
    assert f(M=(1 << 30) + 1, seen=1 << 40, t=_tab(b, entries=1 << 41)) == UNSUPPORTED


def test_write(b):
    def f(tokens=4, heads=2, d=64, k=4096, ldk=128, shk=64, v=4096, t=None, kp=None, vp=None, means=None, ptr=4096, lengths=4096, fn="b2sp_paged_write"):
        return getattr(b.lib, fn)(tokens, heads, d, k, ldk, shk, v, 128, 64, ptr, lengths, t or _tab(b), kp or _cache(b), vp or _cache(b, data=1 << 24), means, None)
    for bad in BAD_TABLES:
        assert f(t=_tab(b, **bad)) == INVALID, bad
    for bad in BAD_CACHES:
        assert f(kp=_cache(b, **bad)) == f(vp=_cache(b, **bad)) == INVALID, bad
        if "ld" not in bad and "page" not in bad:
            assert f(means=_cache(b, **bad)) == INVALID, bad
    assert f(kp=_cache(b, ld=68), fn="b2sp_paged_write_bf16") == INVALID                       # 16 bytes are eight of them
    assert f(tokens=-1) == f(heads=0) == f(d=0) == f(k=None) == f(v=None) == f(ldk=-1) == f(ptr=None) == f(lengths=None) == INVALID
    assert f(kp=_cache(b, pages=31)) == f(kp=_cache(b, page=8)) == f(means=_cache(b, pages=31)) == f(vp=_cache(b)) == INVALID
    for over in (dict(stride_head=960), dict(stride_page=1024), dict(ld=128)):
        assert f(kp=_cache(b, **over)) == f(vp=_cache(b, **over)) == INVALID, over             # rows that are written overlap
    assert f(means=_cache(b, stride_head=32)) == INVALID
    assert f(t=_tab(b, requests=8193)) == UNSUPPORTED
    wide = _cache(b, ld=1028, stride_head=1 << 16, stride_page=1 << 17)
    assert f(d=1025, kp=wide, vp=wide) == UNSUPPORTED
    assert f(tokens=0) == f(t=_tab(b, requests=0)) == OK


def test_select(b):
    need = b.lib.b2sp_paged_select_workspace_bytes
    def f(M=3, H=4, Hkv=2, d=64, q=4096, ldq=256, means=None, t=None, seen=4096, keep=4, first=1, last=1, out=4096, ws=1 << 20, wsb=1 << 30):
        return b.lib.b2sp_paged_select(M, H, Hkv, d, q, ldq, 64, means or _cache(b, stride_head=64, stride_page=128), t or _tab(b), None, seen, keep,
                                       first, last, out, ws, wsb, None)
    for bad in BAD_TABLES:
        assert f(t=_tab(b, **bad)) == INVALID, bad
    for bad in (dict(data=0), dict(data=(1 << 20) + 8), dict(stride_head=66), dict(stride_page=-16), dict(pages=-1), dict(page=0)):
        assert f(means=_cache(b, **{**dict(stride_head=64, stride_page=128), **bad})) == INVALID, bad
    assert f(M=-1) == f(H=3) == f(Hkv=0) == f(d=0) == f(q=None) == f(ldq=-1) == f(seen=None) == f(out=None) == INVALID
    assert f(keep=0) == f(first=-1) == f(last=-1) == f(first=3, last=2) == INVALID
    assert f(d=257) == UNSUPPORTED
    assert need(3, 2, 16) >= 3 * 2 * 16 * 8 and need(3, 2, 16) % 256 == 0 and need(-1, 2, 16) == need(3, 0, 16) == need(3, 2, -1) == 0
    assert f(ws=None) == f(ws=(1 << 20) + 16) == f(wsb=need(3, 2, 16) - 1) == WORKSPACE
    assert f(M=0) == OK


def test_select_lists_in_what_is_read(b):
    f = lambda out: b.lib.b2sp_paged_select(3, 4, 2, 64, 4096, 256, 64, _cache(b, stride_head=64, stride_page=128),  # noqa: E731
                                            _tab(b, entries=1 << 21), 1 << 22, 1 << 23, 4, 1, 1, out, 1 << 30, 1 << 20, None)
    for at in (1 << 21, 1 << 22, 1 << 23):                                                     # tables (48 entries), rows, seen (3 of each); 24 are written
        n = 48 if at == 1 << 21 else 3
        assert f(at) == f(at + 4 * n - 4) == f(at - 4 * 23) == INVALID


def test_attention(b):
    need = b.lib.b2sp_attention_paged_workspace_bytes
    def f(M=3, H=4, Hkv=2, d=64, q=4096, ldq=256, kp=None, vp=None, t=None, seen=4096, lists=None, keep=0, scale=0.1, o=4096, ldo=256, sho=64, lse=4096,
          ws=1 << 20, wsb=1 << 40):
        return b.lib.b2sp_attention_paged(M, H, Hkv, d, q, ldq, 64, kp or _cache(b), vp or _cache(b), t or _tab(b), None, seen, lists, keep, scale, o, ldo,
                                          sho, lse, ws, wsb, None)
    for bad in BAD_TABLES:
        assert f(t=_tab(b, **bad)) == INVALID, bad
    for bad in BAD_CACHES:
        assert f(kp=_cache(b, **bad)) == f(vp=_cache(b, **bad)) == INVALID, bad
    assert f(vp=_cache(b, pages=31)) == f(vp=_cache(b, page=8)) == INVALID
    assert f(M=-1) == f(H=3) == f(Hkv=0) == f(d=0) == f(q=None) == f(ldq=-1) == f(seen=None) == f(o=None) == f(lse=None) == INVALID
    assert f(scale=float("nan")) == f(lists=4096, keep=0) == f(lists=4096, keep=-1) == INVALID
    assert f(ldo=192) == f(sho=32) == f(ldo=64, sho=128) == INVALID                            # rows of O overlap
    wide = _cache(b, ld=260, stride_head=1 << 13, stride_page=1 << 14)
    assert f(d=257, kp=wide, vp=wide, ldo=2048, sho=260) == UNSUPPORTED
    assert f(lists=4096, keep=1 << 27) == UNSUPPORTED
    assert need(3, 4, 2, 64) >= 256 and need(3, 4, 2, 64) % 256 == 0 and need(3, 3, 2, 64) == need(-1, 4, 2, 64) == need(3, 4, 2, 257) == 0
    assert f(ws=None) == f(ws=(1 << 20) + 16) == f(wsb=need(3, 4, 2, 64) - 1) == WORKSPACE
    assert f(M=0) == OK


def test_binding_checks_types_and_shapes(b):
    i = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    c, m, x = b.paged_cache(4, 2, 8, 33, device="cpu"), b.paged_means(4, 2, 33, device="cpu"), torch.zeros(3, 4, 33)
    assert c.shape == (4, 2, 8, 33) and c.stride(2) == 36 and m.shape == (4, 2, 33)
    assert b.paged_cache(4, 2, 8, 33, torch.bfloat16, "cpu").stride(2) == 40
    with pytest.raises(ValueError):
        b.paged_tables(i(3), i(3), i(3, 4), i(4), i(1), 8, 4, 3)                               # not on a GPU
    for bad in ((i(3).long(), i(3), i(3, 4), i(4), i(1)), (i(3), i(3), i(3, 4).long(), i(4), i(1)), (i(3), i(3), i(3, 4), i(4), i(1).float())):
        with pytest.raises(TypeError):
            b.paged_tables(*bad, 8, 4, 3)
    for bad in ((i(2), i(3), i(3, 4), i(4), i(1)), (i(3), i(3), i(3, 4), i(2, 2), i(1)), (i(3), i(3), i(4, 3).t(), i(4), i(1)),
                (i(3), i(3), i(3, 4), i(4), i(0))):
        with pytest.raises(ValueError):
            b.paged_tables(*bad, 8, 4, 3)
    with pytest.raises(ValueError):
        b.paged_lists(i(3, 4), i(3), 8, 4, -1)
    with pytest.raises(ValueError):
        b.paged_lists(i(3, 4), i(3), 8, 4, 10, rows=i(2))
    kv = torch.zeros(3, 2, 33)
    with pytest.raises(TypeError):
        b.paged_write(kv, kv, i(4), i(3), i(3, 4), c, c, dtype=torch.bfloat16)
    for bad in ((kv, kv[:2], i(4), i(3), i(3, 4), c, c), (kv, kv, i(3), i(3), i(3, 4), c, c), (kv, kv, i(4), i(3), i(3, 4), c, c[:2]),
                (kv, kv, i(4), i(3), i(3, 4), c, c, m[:2]), (kv[..., :32], kv[..., :32], i(4), i(3), i(3, 4), c, c)):
        with pytest.raises(ValueError):
            b.paged_write(*bad)
    for bad in ((x, m[..., :32], i(3, 4), i(3), 8, 2), (x, m, i(3, 4), i(2), 8, 2), (x[:, :3], m, i(3, 4), i(3), 8, 2), (x, m, i(3, 4), i(3), 8, 0)):
        with pytest.raises(ValueError):
            b.paged_select(*bad)
    for bad in (dict(tables=i(12)), dict(seen=i(2)), dict(rows=i(2)), dict(lists=i(3, 1, 4)), dict(k_pages=c[:2]), dict(q=x[:, :3]), dict(out=x[..., :32])):
        with pytest.raises(ValueError):
            b.attention_paged(**{**dict(q=x, k_pages=c, v_pages=c, tables=i(3, 4), seen=i(3)), **bad})
    for bad in (torch.float64, torch.float16):
        with pytest.raises(TypeError):
            b.attention_paged(x.to(bad), c.to(bad), c.to(bad), i(3, 4), i(3), dtype=bad)

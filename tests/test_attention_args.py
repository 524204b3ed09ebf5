"""Refusals of the attention and 4-bit cache entry points: argument checks run before any CUDA call, so no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2311_00368_b200 import build as b2sp_build

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 5


@pytest.fixture(scope="module")
def b():
    b2sp_build.build()
    from paper_2311_00368_b200 import binding
    return binding


def _problem(b, **other):
    base = dict(batch=2, heads=4, kv_heads=2, M=8, K=16, d=64, patterns=1, scale=0.125, row_ptr=4096, row_ptr_stride=9, col_idx=8192,
                nnz_stride=32, plan=0, plan_tiles=0)
    base.update({k: v or 0 if k in ("row_ptr", "col_idx", "plan") else v for k, v in other.items()})
    return b._PROBLEM(*base.values())


def _heads(b, data, *strides):
    return b._HEADS(data or 0, *strides)


def _forward(b, p, q=None, o=None, lse=4096, ws=1 << 20, ws_bytes=1 << 40, algo=0, fn="b2sp_attention"):
    rows, kv = _heads(b, 1 << 20, 64, 64 * 64, 64 * 64 * 8), _heads(b, 1 << 20, 64, 64 * 64, 64 * 64 * 8)
    return getattr(b.lib, fn)(p, q or rows, kv, kv, o or rows, lse, ws, ws_bytes, algo, None)


def test_problem_sizes(b):
    for bad in (dict(batch=0), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(M=-1), dict(K=-1), dict(d=0), dict(nnz_stride=-1),
                dict(nnz_stride=2 ** 31), dict(patterns=3), dict(patterns=0), dict(row_ptr=None), dict(col_idx=None), dict(scale=float("nan")),
                dict(patterns=2, row_ptr_stride=8), dict(plan=1 << 20, plan_tiles=-1), dict(plan=(1 << 20) + 8)):
        p = _problem(b, **bad)
        assert _forward(b, p) == INVALID, bad
        assert b.lib.b2sp_attention_workspace_bytes(p, 0) == 0, bad
    assert _forward(b, None) == INVALID
    assert _forward(b, _problem(b, d=257)) == UNSUPPORTED


def test_operands_workspace_and_algo(b):
    p = _problem(b)
    need = b.lib.b2sp_attention_workspace_bytes(p, 0)
    assert need >= 512 and need % 256 == 0
    assert _forward(b, p, q=_heads(b, None, 64, 1, 1)) == INVALID
    assert _forward(b, p, lse=None) == INVALID
    for over in (_heads(b, 1 << 20, 63, 64 * 64, 64 * 64 * 8), _heads(b, 1 << 20, 64, 0, 64 * 64), _heads(b, 1 << 20, 64, 64 * 7, 64 * 64),
                 _heads(b, 1 << 20, 64, 64 * 8, 64 * 31)):
        assert _forward(b, p, o=over) == INVALID
    assert _forward(b, p, ws=None) == WORKSPACE
    assert _forward(b, p, ws=(1 << 20) + 128) == WORKSPACE
    assert _forward(b, p, ws_bytes=need - 1) == WORKSPACE
    assert _forward(b, p, algo=4) == INVALID and _forward(b, p, algo=-1) == INVALID
    assert _forward(b, p, algo=b.ALGO_TILE) == UNSUPPORTED                                       # no plan
    assert _forward(b, _problem(b, d=129, plan=1 << 20, plan_tiles=1), o=_heads(b, 1 << 20, 129, 129 * 64, 129 * 64 * 8), algo=b.ALGO_TILE) == UNSUPPORTED   # fp32
    assert _forward(b, p, algo=b.ALGO_TILE, fn="b2sp_attention_bf16") == UNSUPPORTED             # no plan
    for bad in (dict(d=130), dict(d=136)):
        assert _forward(b, _problem(b, plan=1 << 20, plan_tiles=1, **bad), o=_heads(b, 1 << 20, 136, 136 * 64, 136 * 64 * 8), algo=b.ALGO_TILE,
                        fn="b2sp_attention_bf16") == UNSUPPORTED
    odd = _heads(b, (1 << 20) + 2, 64, 64 * 64, 64 * 64 * 8)
    assert _forward(b, _problem(b, plan=1 << 20, plan_tiles=1), q=odd, algo=b.ALGO_TILE, fn="b2sp_attention_bf16") == UNSUPPORTED
    # fp32, d > 64: 64 KB a tile and problem, 2 GB at most
    wide = dict(d=80, plan=1 << 20, heads=4, kv_heads=4)
    assert b.lib.b2sp_attention_workspace_bytes(_problem(b, plan_tiles=4096, **wide), 0) > 1 << 31
    assert b.lib.b2sp_attention_workspace_bytes(_problem(b, plan_tiles=4097, **wide), 0) < 1 << 31
    assert b.lib.b2sp_attention_workspace_bytes_bf16(_problem(b, plan_tiles=4096, **wide), 0) < 1 << 28
    assert _forward(b, _problem(b, plan_tiles=4097, **wide), o=_heads(b, 1 << 20, 80, 80 * 64, 80 * 64 * 8), algo=b.ALGO_TILE) == UNSUPPORTED
    # nothing to do: no launch, so this passes without a device
    assert _forward(b, _problem(b, M=0)) == OK


def test_backward_needs_a_plan(b):
    p, x = _problem(b), _heads(b, 1 << 20, 64, 64 * 64, 64 * 64 * 8)
    assert b.lib.b2sp_attention_backward(p, x, x, x, x, 4096, x, x, x, x, 1 << 20, 1 << 40, 0, None) == INVALID


def test_plan_sizes(b):
    f = b.lib.b2sp_attention_plan_bytes
    assert f(0, 8, 8, 4, 1) == f(1, -1, 8, 4, 1) == f(1, 8, 8, -1, 1) == f(1, 8, 8, 4, -1) == 0
    assert f(1, 8, 128 * 32768 + 1, 4, 1) == 0
    assert f(1, 4096, 4096, 100, 8) - f(1, 4096, 4096, 100, 0) >= 8 * 4096
    n = ctypes.c_longlong(0)
    g = b.lib.b2sp_attention_count_tiles
    assert g(1, 8, 128 * 32768 + 1, 4, 4096, 9, 4096, 1 << 20, 256, ctypes.byref(n), None) == UNSUPPORTED
    assert g(1, 8, 8, 4, 4096, 9, 4096, None, 256, ctypes.byref(n), None) == WORKSPACE
    assert g(1, 8, 8, 4, 4096, 9, 4096, 1 << 20, 256, None, None) == INVALID
    assert g(1, 0, 8, 0, None, 1, None, 1 << 20, 256, ctypes.byref(n), None) == OK and n.value == 0


def _cache(b, G=2, **other):
    base = dict(codes=1 << 20, code_ld=16 * G, code_stride_head=1 << 12, scales=1 << 16, scale_ld=G, scale_stride_head=1 << 8, slots=32)
    base.update({k: v or 0 for k, v in other.items()})
    return b._KV4(*base.values())


def test_kv4_refusals(b):
    write, read, att = b.lib.b2sp_kv4_write, b.lib.b2sp_kv4_read, b.lib.b2sp_attention_kv4
    w = lambda c, tokens=4, heads=2, d=64, x=1 << 20, ws=None, wsb=0: write(tokens, heads, d, x, 128, 64, 4096, c, ws, wsb, None)  # noqa: E731
    r = lambda c, tokens=4, heads=2, d=64, ld=128, sh=64: read(tokens, heads, d, 4096, c, 1 << 20, ld, sh, None)  # noqa: E731
    for bad in (dict(codes=(1 << 20) + 8), dict(code_ld=40), dict(code_ld=16), dict(scale_ld=1), dict(scales=(1 << 16) + 2), dict(slots=-1),
                dict(codes=None), dict(scale_stride_head=255)):
        c = _cache(b, **bad)
        assert w(c) == r(c) == INVALID, bad
        assert att(1, 4, 2, 64, 8, 4096, 4096, 4096, 256, 64, _cache(b), c, 0.1, 4096, 256, 64, 4096, 1 << 20, 1 << 30, None) == INVALID, bad
    assert w(None) == r(None) == INVALID
    assert w(_cache(b, code_stride_head=64)) == INVALID               # heads of the cache overlap
    assert w(_cache(b), tokens=-1) == w(_cache(b), heads=0) == w(_cache(b), d=0) == w(_cache(b), x=None) == INVALID
    assert r(_cache(b), ld=64) == r(_cache(b), sh=32) == r(_cache(b), ld=100) == INVALID
    assert w(_cache(b), tokens=1025) == w(_cache(b), tokens=1025, ws=4096 + 8, wsb=1 << 20) == w(_cache(b), tokens=1025, ws=4096, wsb=127) == WORKSPACE
    assert w(_cache(b), tokens=0) == r(_cache(b), tokens=0) == OK
    a = lambda M=1, H=4, Hkv=2, d=64, nnz=8, q=4096, ldo=256, sho=64, lse=4096, ws=1 << 20, wsb=1 << 30: att(  # noqa: E731
        M, H, Hkv, d, nnz, 4096, 4096, q, 256, 64, _cache(b, (d + 31) // 32 if d <= 64 else 4), _cache(b, (d + 31) // 32 if d <= 64 else 4), 0.1,
        4096, ldo, sho, lse, ws, wsb, None)
    assert a(M=-1) == a(H=3) == a(Hkv=0) == a(nnz=-1) == a(q=None) == a(lse=None) == a(sho=32) == a(M=2, ldo=100) == INVALID
    assert a(d=129) == UNSUPPORTED
    assert a(ws=None) == a(ws=(1 << 20) + 16) == a(wsb=511) == WORKSPACE
    assert a(M=0) == OK
    assert b.lib.b2sp_attention_kv4_workspace_bytes(1, 32, 8, 128, 32768) > 32 * 128 * 4
    assert b.lib.b2sp_attention_kv4_workspace_bytes(1, 3, 2, 128, 8) == 0


def test_binding_checks_types_and_shapes(b):
    """The binding refuses what it can see before it asks the library."""
    i32 = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        b.attention_plan(i32, i32, 4)                      # not on a GPU
    with pytest.raises(TypeError):
        b.attention_plan(i32.long(), i32, 4)
    with pytest.raises(ValueError):
        b.kv4_write(torch.zeros(2, 1, 32), i32[:2], torch.zeros((1, 4, 16), dtype=torch.uint8), torch.zeros((1, 4, 1), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        b.attention_backward(i32, i32, None, None, None, None, None, None, None)

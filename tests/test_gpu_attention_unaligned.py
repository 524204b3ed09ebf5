"""Attention on fp32 views of any alignment: rows that the tile kernels give up are taken again entry by entry, from operands that need
not be groups of four beside outputs that are."""
import numpy as np
import pytest
import torch

from tests import attention_plain as plain
from tests.test_gpu_attention import Problem

pytestmark = pytest.mark.gpu

TILE = 3


def _moved(t, by, pad):
    """The same values `by` elements behind the beginning of rows that are `pad` elements longer."""
    room = torch.full((*t.shape[:-1], t.shape[-1] + pad), 7.0, dtype=t.dtype, device=t.device)
    view = room[..., by:by + t.shape[-1]]
    view.copy_(t)
    return view


def _with_rows_to_take_again(K, d, **more):
    """NaN and infinities in rows that no entry names, in tiles that hold entries: every row of those tiles is taken again."""
    p = Problem(800 + d, H=2, M=300, K=K, d=d, **more)
    m = p.mask[0, 0].clone()
    m[:, 40:44] = False
    m[200:204] = False
    p.row_ptr, p.col_idx = (t.cuda() for t in plain.csr(m.cpu().numpy()))
    p.mask = m.expand(1, 2, 300, K)
    p.k[:, :, 40:42] = float("nan")
    p.v[:, :, 40:42] = float("inf")
    p.v[:, :, 42:44] = float("nan")
    p.q[:, :, 200:202] = float("nan")
    p.do[:, :, 202:204] = float("nan")
    return p


@pytest.mark.parametrize("which", ["q", "k", "v", "do", "qkv do"])
@pytest.mark.parametrize("K, d", [(300, 64), (300, 100), (4000, 64), (2500, 128), (300, 36)])
def test_rows_taken_again_from_unaligned_operands(K, d, which):
    p = _with_rows_to_take_again(K, d)
    for name in ("q", "k", "v", "do"):
        if name in which.replace("qkv", "q k v").split():
            setattr(p, name, _moved(getattr(p, name), 1, 4))
    p.check(TILE)


@pytest.mark.parametrize("by, pad", [(0, 1), (2, 2), (3, 5)])
def test_rows_of_odd_strides(by, pad):
    p = _with_rows_to_take_again(300, 64)
    for name in ("q", "k", "v", "do"):
        setattr(p, name, _moved(getattr(p, name), by, pad))
    p.check(TILE)


def test_weights_lost_to_a_masked_product_of_unaligned_operands():
    """A key that few rows name is so large that the others' weights vanish beside it: those rows are taken again."""
    p = Problem(810, M=300, K=300, d=64)
    p.q[..., 0] = 4.0
    p.k[:, :, 17] = 0.0
    p.k[:, :, 17, 0] = 400.0
    p.q, p.k, p.v, p.do = (_moved(t, 1, 4) for t in (p.q, p.k, p.v, p.do))
    p.check(TILE)


@pytest.mark.parametrize("inputs", [0, 1])
def test_unaligned_outputs(inputs):
    p = _with_rows_to_take_again(300, 64)
    plan = p.plan()
    ref = p.forward(TILE, plan)
    grads = p.backward(*ref, plan, TILE)
    for name in ("q", "k", "v", "do"):
        if inputs:
            setattr(p, name, _moved(getattr(p, name), 1, 4))
    o, lse = p.forward(TILE, plan, out=_moved(torch.zeros_like(ref[0]), 1, 4))
    assert torch.equal(torch.nan_to_num(o, 3.0), torch.nan_to_num(ref[0], 3.0)) and torch.equal(lse, ref[1])
    like = [_moved(torch.zeros_like(t), 3, 4) for t in grads]
    got = p.backward(*ref, plan, TILE, dq=like[0], dk=like[1], dv=like[2])
    for g, w in zip(got, grads):
        assert torch.equal(torch.nan_to_num(g, 3.0), torch.nan_to_num(w, 3.0))
    assert np.isfinite(float(ref[0][0, 0, 0, 0]))

"""What rows that no entry names hold: fp32 results by tiles do not depend on it, to the bit, while it is finite, bfloat16 ones no further than
their rounding."""
import pytest
import torch

from tests import attention_plain as plain
from tests.test_gpu_attention import Problem

pytestmark = pytest.mark.gpu

TILE = 3


def _problem(dtype, d, K=700):
    """Every seventh column and the last row block's first rows are in tiles with entries, but have none."""
    p = Problem(1100 + d, H=2, Hkv=1, M=300, K=K, d=d, dtype=dtype)
    m = p.mask[0, 0].clone()
    m[:, ::7] = False
    m[256:260] = False
    p.row_ptr, p.col_idx = (t.cuda() for t in plain.csr(m.cpu().numpy()))
    p.mask = m.expand(1, 2, 300, K)
    return p


def _results(p, plan):
    o, lse = p.forward(TILE, plan)
    return (o, lse, *p.backward(o, lse, plan, TILE))


@pytest.mark.parametrize("size", [0.0, 30.0, 1e4, 1e18])
@pytest.mark.parametrize("d", [4, 64, 100])
def test_fp32_results_do_not_depend_on_rows_that_no_entry_names(d, size):
    """Products of up to a few, of some hundred (weights beside them vanish) and beyond what an exponential holds."""
    p = _problem(torch.float32, d)
    plan = p.plan()
    want = _results(p, plan)
    p.k[:, :, ::7] *= size
    p.v[:, :, ::7] = 5.0
    p.q[:, :, 256:260] *= size
    got = _results(p, plan)
    for name, x, y in zip(("O", "lse", "dQ", "dK", "dV"), got, want):
        assert torch.equal(x, y), f"{name} differs by {float((x - y).abs().max()):.3g}"


@pytest.mark.parametrize("size", [0.0, 30.0, 1e4, 1e18])
@pytest.mark.parametrize("dtype, d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 33), (torch.float32, 64), (torch.float32, 128)])
def test_results_stay_within_their_bounds(dtype, d, size):
    p = _problem(dtype, d)
    p.k[:, :, ::7] *= size
    p.q[:, :, 256:260] *= size
    p.check(TILE)


def test_the_first_entries_come_late_and_low():
    """Rows whose first tiles hold entries of other rows only, and whose own products lie far below zero; parts of rows among them."""
    for K in (1000, 5000):
        p = Problem(1120, M=200, K=K, d=16)
        m = p.mask[0, 0].clone()
        m[::2, :K - 100] = False
        p.q[..., 0] = 30.0
        p.k[..., 0] = torch.where(torch.arange(K, device="cuda") < K - 100, 20.0, -20.0)
        p.row_ptr, p.col_idx = (t.cuda() for t in plain.csr(m.cpu().numpy()))
        p.mask = m.expand(1, 1, 200, K)
        p.check(TILE)
        p.k[..., K - 50:, 0] = -1e30    # products of -infinity are none: the row is taken entry by entry
        p.q[..., 0] = 1e10
        o, lse = p.forward(TILE, p.plan())
        want, want_lse, _, _ = plain.forward(p.mask, p.q, p.k, p.v, p.scale)
        assert torch.isfinite(o).all() and torch.equal(torch.isinf(lse), ~p.mask.any(3))

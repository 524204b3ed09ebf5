"""The far end of what lengths can be."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_neighbours_that_see_all_positions_there_can_be(dtype):
    """2^31 - 1 positions, all of whose pages are one.  A weight of one in a page's last row but one, nothing in the others: the token that sees the last
    position counts 2048 of them, the one before it 2047.  (lse: half a step of a number below 8, some of log2: 1e-5 is ten times that, and 1/50 of what is
    between the two)"""
    from paper_2311_00368_b200 import binding as b
    page = 1 << 20
    k, v = (b.paged_cache(1, 1, page, 8, dtype) for _ in range(2))
    k.fill_(-100)
    k[:, :, page - 2] = 0
    v[:, :, page - 2] = 3
    tables = torch.zeros((1, 2048), dtype=torch.int32, device="cuda")
    o, lse = b.attention_paged(torch.ones((2, 1, 8), device="cuda").to(dtype), k, v, tables, _int([2 ** 31 - 2, 2 ** 31 - 1]), rows=_int([0, 0]), scale=1.0, dtype=dtype)
    assert (lse.cpu().view(2).double() - torch.tensor([math.log(2047), math.log(2048)])).abs().max() <= 1e-5
    assert (o == 3).all()

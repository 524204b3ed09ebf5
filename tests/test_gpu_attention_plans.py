"""Plans of patterns without a single tile: what is wrong with them is reported as for any other pattern."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BAD_CSR = 3


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("row_ptr, col_idx, K", [
    ((0, 2, 3), (2, 3, 2), 2),                  # every column is out of range
    ((0, 1), (-1,), 5),
    ((0, 2, 3), (1 << 30, -7, 300), 300),
    ((0, 1, 2), (0, 0), 0),                     # no columns at all
    ((0, 1, 1), (), 4),                         # row pointers beyond the entries
    ((0, -1, 0), (), 4),
    ((1, 1, 1), (), 4),
    ((0, 0, 1), (), 0),
])
def test_patterns_without_tiles_that_a_plan_refuses(row_ptr, col_idx, K):
    from paper_2311_00368_b200 import binding as b
    with pytest.raises(b.B2spError) as e:
        b.attention_plan(_i32(*row_ptr), _i32(*col_idx), K)
    assert e.value.status == BAD_CSR


def test_one_bad_pattern_among_several():
    from paper_2311_00368_b200 import binding as b
    rp = _i32(0, 0, 0, 0, 0, 1).view(2, 3)
    with pytest.raises(b.B2spError) as e:
        b.attention_plan(rp, _i32(0, 9).view(2, 1), 3)
    assert e.value.status == BAD_CSR


@pytest.mark.parametrize("row_ptr, K", [((0, 0, 0), 4), ((0,), 4), ((0, 0), 0)])
def test_patterns_without_entries_are_plans(row_ptr, K):
    from paper_2311_00368_b200 import binding as b
    assert b.attention_plan(_i32(*row_ptr), _i32(), K).tiles == 0

"""The far end of what lengths can be, and calls behind one whose launch failed."""
import ctypes
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


def test_a_launch_that_fails_leaves_nothing_behind():
    """A call on the legacy stream while another stream is being captured is an error of that call, and not of the next one."""
    from paper_2311_00368_b200 import binding as b
    runtime = ctypes.CDLL("libcudart.so.12")
    tables, seen = _int([[0, 1]]), _int([9])
    ptr, col = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(9, dtype=torch.int32, device="cuda")
    b.paged_lists(tables, seen, 8, 2, 9, out=(ptr, col))
    torch.cuda.synchronize()
    call = lambda stream: b.lib.b2sp_paged_lists(1, b._page_tables(tables), 2, 8, None, seen.data_ptr(), 9, ptr.data_ptr(), col.data_ptr(), stream)  # noqa: E731
    stream, graph = ctypes.c_void_p(), ctypes.c_void_p()
    assert runtime.cudaStreamCreate(ctypes.byref(stream)) == 0            # (one that the legacy stream waits for)
    try:
        assert runtime.cudaStreamBeginCapture(stream, 0) == 0
        failed = call(None)
        runtime.cudaStreamEndCapture(stream, ctypes.byref(graph))
        runtime.cudaGetLastError()
        assert failed == 4
        col.fill_(-5)
        assert call(stream) == 0
        assert runtime.cudaStreamSynchronize(stream) == 0
        assert col.tolist() == list(range(9))
    finally:
        runtime.cudaStreamDestroy(stream)

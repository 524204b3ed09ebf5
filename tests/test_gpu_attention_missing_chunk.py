"""Attention's tile kernels when a load never arrives.  b2sp_debug_inject_wait_timeout makes the loading warp of every CTA leave one load out and
shortens the limit of the bounded waits to 2 ms: the CTAs leave through their teardown (loads and products in flight awaited, tensor
memory freed), the call reports B2SP_ERR_TIMEOUT (6) through the status word, and the next call gives the bits of the one before."""
import pytest
import torch

from tests.test_gpu_attention import Problem

pytestmark = pytest.mark.gpu

TILE, TIMEOUT, LIMIT_NS = 3, 6, 2_000_000

CASES = {   # (512 tiles: three or four for each CTA of the gradients, seven loads or more)
    "bf16-64": dict(H=2, Hkv=1, M=2000, K=2000, d=64, dtype=torch.bfloat16),
    "bf16-128": dict(H=2, Hkv=2, M=2000, K=2000, d=128, dtype=torch.bfloat16),
    "bf16-83": dict(H=2, Hkv=2, M=2000, K=2000, d=83, dtype=torch.bfloat16),
    "bf16-parts": dict(H=2, Hkv=1, M=100, K=5000, d=64, dtype=torch.bfloat16),
    "fp32-64": dict(H=2, Hkv=1, M=2000, K=2000, d=64),
    "fp32-100": dict(H=2, Hkv=1, M=2000, K=2000, d=100),
}


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("name", CASES)
def test_a_load_that_never_arrives_is_reported(name, backward):
    from paper_2311_00368_b200 import binding as b
    p = Problem(900, **CASES[name])
    plan, ws = p.plan(), torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    o, lse = p.forward(TILE, plan)

    def call():
        out = p.backward(o, lse, plan, TILE, workspace=ws) if backward else p.forward(TILE, plan, workspace=ws)
        assert b.attention_last_algo(backward) == TILE
        return out, b.device_status(ws)

    before, status = call()
    assert status == 0
    # load 0 is a block's own rows, the others are those of steps (in the forward pass of bfloat16 K and V each have theirs)
    for chunk in (0, 1, 2) if name == "bf16-parts" else (0, 1, 2, 3, 6):
        b.debug_inject_wait_timeout(chunk, LIMIT_NS)
        try:
            _, status = call()
        finally:
            b.debug_inject_wait_timeout(-1)
        assert status == TIMEOUT, (chunk, status)
        after, status = call()
        assert status == 0
        for x, y in zip(after, before):
            assert torch.equal(x, y), f"the call after a missing load {chunk} differs"

"""Attention over pages in bfloat16: the weights that V is multiplied by keep sixteen bits, also beside a value that is not finite.

The bounds of attention_plain allow for a weight of eight bits; here logits are sums of eight products of small numbers, so that their own roundings are
small, and values cancel, so that the result's rounding is.  Per element, u = 2^-24:
  |O - want| <= sum p |v| (2 e + 2 (n + 8) u + 2^-16) + 2^-8 |O|
with e as in attention_plain for eight terms; 2^-16: a weight as two bfloat16, each off by at most 2^-8 of what it stands for."""
import pytest
import torch

from tests import attention_plain as plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,H,Hkv,each,page", [(64, 4, 1, 1, 16), (64, 8, 2, 4, 24), (128, 4, 1, 4, 16), (128, 16, 1, 1, 16), (256, 4, 1, 2, 16), (256, 16, 1, 1, 32)])
@pytest.mark.parametrize("odd", [None, float("inf"), float("nan")])
def test_weights_of_sixteen_bits(d, H, Hkv, each, page, odd):
    from paper_2311_00368_b200 import binding as b
    dtype, gen = torch.bfloat16, torch.Generator().manual_seed(d + H)
    n, M = 60, 4 * each
    width = -(-n // page)
    tables = torch.randperm(4 * width, generator=gen).view(4, width).to(torch.int32)
    kp, vp = (b.paged_cache(4 * width, Hkv, page, d, dtype) for _ in range(2))
    q = torch.zeros((M, H, d))
    q[..., :8] = torch.randint(-3, 4, (M, H, 8), generator=gen)
    k = torch.zeros((4, Hkv, width * page, d))
    k[..., :8] = torch.randint(-3, 4, (4, Hkv, width * page, 8), generator=gen)
    v = torch.randn((4, Hkv, width * page, d), generator=gen).to(dtype)
    if odd is not None:
        v[:, :, n // 2, 11] = odd
        v[1:, :, 3, d - 1] = odd
    for r in range(4):
        for c in range(width):
            kp[tables[r, c]] = k[r, :, c * page:(c + 1) * page].to(dtype).cuda()
            vp[tables[r, c]] = v[r, :, c * page:(c + 1) * page].cuda()
    rows = torch.arange(M) // each
    seen = n - (each - 1 - torch.arange(M) % each)
    o, _ = b.attention_paged(q.to(dtype).cuda(), kp, vp, tables.cuda(), seen.int().cuda(), rows=rows.int().cuda(), scale=2.0 ** -5, dtype=dtype)
    tight = 0
    for i in range(M):
        r, m = int(rows[i]), int(seen[i])
        mask = torch.ones((1, H, 1, m), dtype=torch.bool)
        K, V = k[r:r + 1, :, :m, :8], v[r:r + 1, :, :m].float()
        want, _, bound, _ = plain.forward(mask, q[i].view(1, H, 1, d)[..., :8], K, V, 2.0 ** -5)
        size = plain.forward(mask, q[i].view(1, H, 1, d)[..., :8], K, V.abs(), 2.0 ** -5)[0]
        bound += 2.0 ** -16 * size + 2.0 ** -8 * want.abs()
        there = torch.isfinite(V).all(2).repeat_interleave(H // Hkv, 1)   # columns of numbers
        got = o[i].cpu().double().view(1, H, 1, d)[:, :, 0]
        assert (torch.isfinite(got) == there).all()
        off = ((got - want[:, :, 0]).abs() / bound[:, :, 0])[there]
        assert off.max() <= 1, (i, off.max())
        tight += int((bound[:, :, 0] < 2.0 ** -12 * size[:, :, 0])[there].sum())
    assert tight > 20                                                     # elements that a weight of eight bits would be seen in

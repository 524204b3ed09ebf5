"""Attention over a 4-bit cache, per head, within what its arithmetic allows, over any range of scales in the values.

Bounds of one token and head over n slots; k, v the values that the cache holds, u = 2^-24, g_jc = 7 s_jc the largest magnitude of group c in
slot j's row of V.  A code is exact in f16, an element of q too unless it is below 2^-14 of the largest one (2^-25 of that one then); products are exact,
their sums in the tensor core are truncated (2 u of the partial sum an addition).  With S_j = scale sum_e |q_e k_je| and
F_j = scale 2^-25 max|q| sum_e |k_je| the weight's relative error is at most e = max_j 4 (d + 6) u S_j + 2 F_j + 8 u (|lse| + 8).
  lse:  e + 8 u (|lse| + 8)
  O:    sum_j p_j |v_j| (2 e + 2 (n + 8) u + 2^-11)       2^-11: weight times scale to f16
        + sum_j min(p_j, 2^-25) min(g_jc, 2^15 g_c)       products below f16's smallest normal number, where scales lie close together
                                                          (within 2^7 of each other, and 2^8 to the step; g_c: the smallest g_jc that is not 0)
        + n 2^-25 max_j p_j g_jc                          the same where they do not: in parts of the largest product
        + 2^-8 |O|                                        the result to bfloat16
"""
import numpy as np
import pytest
import torch

from tests import attention_plain as plain
from tests.test_gpu_kv4 import Served

pytestmark = pytest.mark.gpu

U = plain.U


def expected(q, k, v, scale):
    """q [H, d]; k, v [n, Hkv, d]: (O, lse, their bounds) in 64 bits."""
    H, d = q.shape
    n, Hkv = k.shape[:2]
    if n == 0:
        zero = torch.zeros((H, d), dtype=torch.float64, device=q.device)
        return zero, torch.full((H,), -np.inf, dtype=torch.float64, device=q.device), zero + 1e-300, zero[:, 0] + 1e-300
    rep = lambda t: t.double().repeat_interleave(H // Hkv, 1).transpose(0, 1)  # noqa: E731
    q, k, v = q.double().unsqueeze(1), rep(k), rep(v)
    s = (q @ k.transpose(1, 2)).squeeze(1) * scale
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse.unsqueeze(1))
    o = (p.unsqueeze(1) @ v).squeeze(1)
    S = (q.abs() @ k.abs().transpose(1, 2)).squeeze(1) * scale
    F = scale * 2.0 ** -25 * q.abs().amax((1, 2)).unsqueeze(1) * k.abs().sum(2)
    e = (4 * (d + 6) * U * S + 2 * F).amax(1) + 8 * U * (lse.abs() + 8)
    bound = (p.unsqueeze(1) @ v.abs()).squeeze(1) * (2 * e + 2 * (n + 8) * U + 2.0 ** -11).unsqueeze(1) + 2.0 ** -8 * o.abs()
    for c in range(0, d, 32):
        g = v[:, :, c:c + 32].abs().amax(2)
        least = torch.where(g > 0, g, np.inf).amin(1, keepdim=True)
        least = torch.where(torch.isinf(least), 0.0, least)
        small = (p.clamp(max=2.0 ** -25) * torch.minimum(g, 2.0 ** 15 * least)).sum(1) + n * 2.0 ** -25 * (p * g).amax(1)
        bound[:, c:c + 32] += small.unsqueeze(1)
    return o, lse, bound + 1e-300, e + 8 * U * (lse.abs() + 8)


def check(s):
    from paper_2311_00368_b200 import binding as b
    Hkv, slots = s.caches[0].shape[:2]
    M, H, d = s.q.shape
    everything = torch.arange(slots, dtype=torch.int32, device="cuda")
    k, v = (b.kv4_read(everything, *s.caches[i:i + 2], d) for i in (0, 2))
    o, lse = s.run()
    ends = s.row_ptr.tolist()
    for i in range(M):
        at = s.col_idx[ends[i]:ends[i + 1]].long()
        at = at[(at >= 0) & (at < slots)]
        want, want_lse, bound, bound_lse = expected(s.q[i], k[at], v[at], d ** -0.5)
        worst = plain.inside(lse[i], want_lse, bound_lse)
        assert worst <= 1, f"token {i}, lse: {worst:.3g} x the bound"
        worst = plain.inside(o[i], want, bound)
        assert worst <= 1, f"token {i}, O: {worst:.3g} x the bound"
    again = s.run()
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("lengths,H,Hkv,d,slots,spread", [
    ([1], 1, 1, 64, 1, 1.0),
    ([15, 16, 17, 0, 1], 4, 2, 128, 100, 1.0),
    ([70, 0, 64, 65, 3, 500], 8, 1, 64, 333, 3.0),
    ([129, 1000], 16, 1, 32, 2000, 1.0),
    ([300, 20, 7], 20, 1, 96, 400, 2.0),
    ([200, 31], 6, 2, 17, 250, 1.0),
    ([5000], 8, 2, 128, 6000, 6.0),
    ([40] * 33, 32, 8, 80, 900, 1.0),
    ([3000, 10, 0, 800], 40, 1, 128, 3000, 1.0),
    ([2, 0, 4, 1] * 30, 4, 4, 128, 1024, 1.0),
    ([1, 3] * 100 + [3000], 8, 2, 64, 3000, 2.0),
    ([20000, 5], 8, 1, 128, 20000, 0.1),
])
def test_within_the_kernels_arithmetic(lengths, H, Hkv, d, slots, spread):
    check(Served(900 + len(lengths) + d, lengths, H, Hkv, d, slots, spread))


class Uneven(Served):
    """All tokens see all slots in order.  Slots `large` hold values `factor` times the others'; their logits are lower by `below` (in powers of
    e), for the heads in `seen` higher by 3."""
    def __init__(self, slots, H, Hkv, d, large, factor, below, seen=(), M=1):
        from paper_2311_00368_b200 import binding as b
        super().__init__(950 + d, [slots] * M, H, Hkv, d, slots)
        self.col_idx = torch.arange(slots, dtype=torch.int32, device="cuda").repeat(M)
        k, v = self.k.clone(), self.v.clone()
        k[:, :, 0], v[large] = 0.0, v[large] * factor
        k[large] = 0.0
        k[large, :, 0] = 1.0
        q = self.q.float()
        q[:, :, 0] = -below * d ** 0.5
        for h in seen:
            q[:, h, 0] = 3 * d ** 0.5
        self.q = q.to(torch.bfloat16)
        everything = torch.arange(slots, dtype=torch.int32, device="cuda")
        b.kv4_write(k.cuda(), everything, *self.caches[:2])
        b.kv4_write(v.cuda(), everything, *self.caches[2:])


@pytest.mark.parametrize("H, Hkv, d", [(8, 2, 128), (16, 1, 64), (5, 1, 96), (2, 2, 17), (444, 444, 32)])   # (the last: a CTA per head)
@pytest.mark.parametrize("large", ["first", "middle", "last", "tile", "half"])
@pytest.mark.parametrize("power, below", [(10, 60), (22, 60), (32, 60), (60, 80), (40, 24), (22, 12)])
def test_a_large_value_that_weighs_little(H, Hkv, d, large, power, below):
    slots = 700
    at = {"first": [0], "middle": [333], "last": [699], "tile": list(range(256, 288)), "half": list(range(1, 700, 2))}[large]
    check(Uneven(slots, H, Hkv, d, at, 2.0 ** power, below, M=2))


@pytest.mark.parametrize("power", [10, 24, 40])
def test_a_large_value_that_some_heads_see(power):
    check(Uneven(1500, 8, 1, 128, [40, 41, 900], 2.0 ** power, 60, seen=(1, 2, 7)))


@pytest.mark.parametrize("power", [-10, -30, -80])
def test_a_small_value_that_weighs_most(power):
    """It has most of the weight, and the others, with little, are nearly all of the result."""
    check(Uneven(600, 8, 2, 64, [3], 2.0 ** power, -9))


def test_scales_that_grow_along_the_list():
    """A CTA per head goes through the whole list: every 128 slots twice the scale of those before, with less and less weight."""
    from paper_2311_00368_b200 import binding as b
    slots, H, d = 5200, 444, 32
    s = Served(970, [slots], H, H, d, slots)
    s.col_idx = torch.arange(slots, dtype=torch.int32, device="cuda")
    step = (torch.arange(slots) // 128).float()
    k = torch.zeros_like(s.k)
    k[:, :, 1] = -step.unsqueeze(1)
    q = torch.zeros(s.q.shape)
    q[:, :, 1] = torch.tensor([0.3, 0.45, 0.6, 0.9]).repeat(111) * d ** 0.5
    s.q = q.to(torch.bfloat16).cuda()
    everything = torch.arange(slots, dtype=torch.int32, device="cuda")
    b.kv4_write(k.cuda(), everything, *s.caches[:2])
    b.kv4_write((s.v * 2.0 ** step.view(-1, 1, 1)).cuda(), everything, *s.caches[2:])
    check(s)


def test_row_pointers_beyond_the_entries():
    """Entries that are not there are left out, of the token they would belong to and of those behind."""
    s = Served(980, [40, 20, 0], 8, 2, 64, 100)
    want = s.run()
    for beyond in ([0, 40, 100, 130], [0, 40, 60, 2 ** 31 - 1]):
        s.row_ptr = torch.tensor(beyond, dtype=torch.int32, device="cuda")
        got = s.run()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

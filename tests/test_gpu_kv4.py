"""A cache in 4 bits: its format bit by bit, and attention over it against the formula in 64 bits on the values that it holds."""
import numpy as np
import pytest
import torch

from tests import attention_plain as plain

pytestmark = pytest.mark.gpu


def _binding():
    from paper_2311_00368_b200 import binding
    return binding


def quantised(x):
    """codes [.., 16 G], scales [.., G] and values [.., d] of rows x, element by element of the format's definition (CPU)."""
    d = x.shape[-1]
    G = (d + 31) // 32
    rows = x.reshape(-1, d).float().numpy()
    codes = np.zeros((rows.shape[0], 16 * G), np.uint8)
    scales = torch.zeros((rows.shape[0], G), dtype=torch.bfloat16)
    values = np.zeros(rows.shape, np.float32)
    for c in range(G):
        part = rows[:, 32 * c:32 * c + 32]
        top = np.abs(part).max(1).astype(np.float32)
        s = torch.from_numpy(top / np.float32(7)).to(torch.bfloat16)
        scales[:, c] = s
        s = s.float().numpy()[:, None]
        with np.errstate(divide="ignore", invalid="ignore"):
            n = np.where(s > 0, np.clip(np.rint(part / s), -7, 7), 0)
        values[:, 32 * c:32 * c + 32] = n * s
        for e in range(32):
            g, i = e // 4, e % 4
            code = (n[:, e].astype(np.int64) + 8 if e < part.shape[1] else np.full(len(rows), 8)).astype(np.uint8)
            codes[:, 2 * (g * G + c) + i // 2] |= code << (4 * (i % 2))
    lead = x.shape[:-1]
    return torch.from_numpy(codes).view(*lead, -1), scales.view(*lead, G), torch.from_numpy(values).view(*lead, d)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,d", [(1, 1, 1), (3, 2, 17), (64, 8, 128), (9, 3, 96), (130, 1, 33), (5, 2, 256), (4100, 1, 64)])
def test_write_and_read(T, H, d, dtype):
    b = _binding()
    gen = torch.Generator().manual_seed(T + d)
    x = (torch.randn((T, H, d), generator=gen) * torch.exp(2 * torch.randn((T, H, 1), generator=gen))).to(dtype)
    x[0, 0] = 0                                          # a row of zeros
    slots = torch.randperm(T + 7, generator=gen)[:T].to(torch.int32)
    codes, scales = b.kv4_cache(H, T + 7, d)
    codes.fill_(0xAB)
    scales.fill_(3.0)
    b.kv4_write(x.cuda(), slots.cuda(), codes, scales, dtype=dtype)
    want_c, want_s, want_v = quantised(x)
    at = slots.long()
    assert torch.equal(codes.cpu()[:, at], want_c.transpose(0, 1))
    assert torch.equal(scales.cpu()[:, at], want_s.transpose(0, 1))
    left = torch.ones(T + 7, dtype=torch.bool)
    left[at] = False
    assert (codes.cpu()[:, left] == 0xAB).all() and (scales.cpu()[:, left] == 3).all()
    for out in (torch.float32, torch.bfloat16):
        got = b.kv4_read(slots.cuda(), codes, scales, d, dtype=out)
        assert torch.equal(got.cpu(), want_v.to(out))


def test_values_at_the_edges_of_the_format():
    b = _binding()
    x = torch.zeros((6, 1, 64))
    x[0, 0, :4] = torch.tensor([7.0, 0.5, 1.5, -2.5])     # scale 1: halves go to even
    x[1, 0, 5] = 3.3e38
    x[2, 0, 6] = 1e-45                                    # the scale rounds to 0
    x[3, 0, 7] = float("nan")
    x[4, 0, 40] = float("inf")
    x[5, 0, 1] = -1e-38
    codes, scales = b.kv4_cache(1, 6, 64)
    b.kv4_write(x.cuda(), torch.arange(6, dtype=torch.int32, device="cuda"), codes, scales)
    got = b.kv4_read(torch.arange(6, dtype=torch.int32, device="cuda"), codes, scales, 64).cpu()
    assert got[0, 0, :4].tolist() == [7.0, 0.0, 2.0, -2.0]
    want = quantised(x[[1, 2, 5]])[2]
    assert torch.equal(got[[1, 2, 5]], want)
    assert torch.isnan(got[3, 0, :32]).all() and (got[3, 0, 32:] == 0).all()
    assert torch.isnan(got[4, 0, 32:]).all() and (got[4, 0, :32] == 0).all()


def test_every_quotient_of_two_bfloat16():
    """Rows whose largest element has each eight-bit significand in turn, with elements at and beside every half step of its scale."""
    b = _binding()
    tops = (torch.arange(128, 256).float() / 128 * 2.0 ** torch.arange(-3, 5).repeat(16).float()).to(torch.bfloat16)
    x = torch.zeros((128, 1, 64), dtype=torch.bfloat16)
    x[:, 0, 0] = tops
    x[:, 0, 32] = -tops
    s = (tops.float() / 7).to(torch.bfloat16).float()
    for i in range(1, 16):
        half = (s * (i - 0.5) / 2).clamp(max=tops.float())
        x[:, 0, i] = half.to(torch.bfloat16)
        x[:, 0, 15 + i] = -((s * (i // 2 + 0.5)).clamp(max=tops.float())).to(torch.bfloat16)
        x[:, 0, 32 + i] = torch.nextafter((s * (i % 7 + 0.5)).to(torch.bfloat16), torch.tensor(0.0, dtype=torch.bfloat16)).clamp(max=tops)
        x[:, 0, 47 + i] = (s * (i % 7 + 0.5)).to(torch.bfloat16).clamp(max=tops)
    codes, scales = b.kv4_cache(1, 128, 64)
    b.kv4_write(x.cuda(), torch.arange(128, dtype=torch.int32, device="cuda"), codes, scales, dtype=torch.bfloat16)
    want_c, want_s, _ = quantised(x)
    assert torch.equal(codes.cpu()[0], want_c[:, 0]) and torch.equal(scales.cpu()[0], want_s[:, 0])


def test_slots_outside_and_slots_twice():
    """Slots outside the cache are skipped and read as zeros; of several tokens with one slot the last one stays, across launches too."""
    b = _binding()
    T = 9000
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((T, 2, 32), generator=gen)
    slots = torch.randint(-3, 50, (T,), generator=gen).to(torch.int32)
    slots[-1] = 1 << 30
    codes, scales = b.kv4_cache(2, 40, 32)
    b.kv4_write(x.cuda(), slots.cuda(), codes, scales)
    last = {int(s): t for t, s in enumerate(slots.tolist()) if 0 <= s < 40}
    got = b.kv4_read(torch.arange(-1, 41, dtype=torch.int32, device="cuda"), codes, scales, 32).cpu()
    want = quantised(x)[2]
    assert (got[0] == 0).all() and (got[41] == 0).all()
    for s in range(40):
        assert torch.equal(got[s + 1], want[last[s]] if s in last else torch.zeros(2, 32)), s


def test_other_layouts():
    """A cache laid out slot by slot, written from a slice of a wider projection, read into a slice."""
    b = _binding()
    gen = torch.Generator().manual_seed(4)
    qkv = torch.randn((20, 3 * 2 * 64), generator=gen).cuda()
    x = qkv[:, 128:256].view(20, 2, 64)
    codes = torch.zeros((30, 2, 32), dtype=torch.uint8, device="cuda").transpose(0, 1)
    scales = torch.zeros((30, 2, 2), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    slots = torch.arange(5, 25, dtype=torch.int32, device="cuda")
    b.kv4_write(x, slots, codes, scales)
    room = torch.full((20, 2, 70), 9.0, device="cuda")
    b.kv4_read(slots, codes, scales, 64, out=room[..., :64])
    assert torch.equal(room[..., :64].cpu(), quantised(x.cpu())[2]) and (room[..., 64:] == 9).all()


class Served:
    def __init__(self, seed, lengths, H, Hkv, d, slots, spread=1.0, by_slot=False):
        b = _binding()
        gen = torch.Generator().manual_seed(seed)
        self.k = torch.randn((slots, Hkv, d), generator=gen)
        self.v = torch.randn((slots, Hkv, d), generator=gen) * torch.exp(torch.randn((slots, Hkv, 1), generator=gen))
        everything = torch.arange(slots, dtype=torch.int32, device="cuda")
        self.caches = []
        for x in (self.k, self.v):
            c, s = b.kv4_cache(Hkv, slots, d)
            if by_slot:
                c, s = c.transpose(0, 1).contiguous().transpose(0, 1), s.transpose(0, 1).contiguous().transpose(0, 1)
            b.kv4_write(x.cuda(), everything, c, s)
            self.caches += [c, s]
        self.row_ptr = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, device="cuda")
        self.col_idx = torch.randint(0, slots, (int(sum(lengths)),), generator=gen).to(torch.int32).cuda()
        self.q = (torch.randn((len(lengths), H, d), generator=gen) * spread).to(torch.bfloat16).cuda()

    def run(self, **more):
        return _binding().attention_kv4(self.row_ptr, self.col_idx, self.q, *self.caches, **more)

    def check(self):
        b = _binding()
        slots = self.caches[0].shape[1]
        M, H, d = self.q.shape
        Hkv = self.caches[0].shape[0]
        everything = torch.arange(slots, dtype=torch.int32, device="cuda")
        k, v = (b.kv4_read(everything, *self.caches[i:i + 2], d).transpose(0, 1) for i in (0, 2))
        o, lse = self.run()
        ends = self.row_ptr.tolist()
        for i in range(M):
            at = self.col_idx[ends[i]:ends[i + 1]].long()
            at = at[(at >= 0) & (at < slots)]
            mask = torch.ones((1, H, 1, at.numel()), dtype=torch.bool, device="cuda")
            # (bfloat16's half step enters the bound through q's type)
            want, want_lse, bound, bound_lse = plain.forward(mask, self.q[i].view(1, H, 1, d), k[None, :, at], v[None, :, at], d ** -0.5)
            # K's products carry 136 too much per code, which is taken off again: 136 sum|q| s instead of sum|q k|, at most 136 times over in
            # the dot product's own error (d + 2) u sum|terms|
            extra = 2 * 136 * (d + 6) * plain.U * (self.q[i].double().abs().sum(1) * k[:, at].abs().amax().double()).max() * d ** -0.5 if at.numel() else 0.0
            worst = plain.inside(lse[i].view(1, H, 1), want_lse, bound_lse + extra)
            assert worst <= 1, (i, worst)
            weight = 2 * extra * v[:, at].abs().amax().double() if at.numel() else 0.0
            worst = plain.inside(o[i].view(1, H, 1, d), want, bound + weight)
            assert worst <= 1, (i, worst)
        o2, lse2 = self.run()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


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
    ([2, 0, 4, 1] * 30, 4, 4, 128, 1024, 1.0),      # shares of a few entries
    ([1, 3] * 100 + [3000], 8, 2, 64, 3000, 2.0),
])
def test_attention_kv4(lengths, H, Hkv, d, slots, spread):
    Served(len(lengths) + d, lengths, H, Hkv, d, slots, spread).check()


@pytest.mark.parametrize("d", [64, 96, 33])
def test_attention_kv4_slot_by_slot_layout(d):
    Served(11, [100, 37], 6, 3, d, 150, by_slot=True).check()


def test_attention_kv4_leaves_out_what_is_outside():
    s = Served(12, [50, 60], 4, 2, 64, 200)
    s.col_idx[3], s.col_idx[70], s.col_idx[71] = -1, 200, 1 << 30
    s.check()
    s.col_idx[:50] = -1
    o, lse = s.run()
    assert (o[0] == 0).all() and (lse[0] == -np.inf).all()


def test_nan_in_slots_that_nobody_names():
    s = Served(13, [90], 4, 2, 64, 100)
    s.col_idx.clamp_(max=98)
    s.caches[1][:, 99] = float("nan")
    s.caches[3][:, 99] = float("nan")
    s.check()


def test_captured_beside_another_graph():
    ss = [Served(20 + i, [4000, 100], 8, 2, 128, 4000) for i in range(2)]
    want = [s.run() for s in ss]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in ss:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in ss]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_a_decoder_step():
    """Prompt through attention, its keys and values into the cache, one more token through the cache: the run of them together agrees with
    attention over the values that the cache holds."""
    b = _binding()
    gen = torch.Generator().manual_seed(30)
    B, H, Hkv, L, d = 2, 4, 2, 200, 64
    t = lambda h, n: torch.randn((B, h, n, d), generator=gen).to(torch.bfloat16).cuda()  # noqa: E731
    q, k, v = t(H, L), t(Hkv, L), t(Hkv, L)
    mask = np.tril(np.ones((L, L), bool))
    rp, ci = (x.cuda() for x in plain.csr(mask))
    plan = b.attention_plan(rp, ci, L)
    o, _ = b.attention(rp, ci, q, k, v, plan=plan, dtype=torch.bfloat16)
    kc, ks = b.kv4_cache(Hkv, B * L, d)
    vc, vs = b.kv4_cache(Hkv, B * L, d)
    slots = torch.randperm(B * L, generator=gen).to(torch.int32).cuda()
    tokens = lambda x: x.transpose(1, 2).reshape(B * L, Hkv, d)  # noqa: E731
    b.kv4_write(tokens(k), slots, kc, ks, dtype=torch.bfloat16)
    b.kv4_write(tokens(v), slots, vc, vs, dtype=torch.bfloat16)
    row_ptr = torch.tensor([0, L, 2 * L], dtype=torch.int32, device="cuda")
    new = torch.randn((B, H, d), generator=gen).to(torch.bfloat16).cuda()
    got, lse = b.attention_kv4(row_ptr, slots, new, kc, ks, vc, vs)
    held = [b.kv4_read(slots, c, s, d).view(B, L, Hkv, d).transpose(1, 2) for c, s in ((kc, ks), (vc, vs))]
    one = torch.tensor([0, L], dtype=torch.int32, device="cuda")
    want, want_lse = b.attention(one, torch.arange(L, dtype=torch.int32, device="cuda"), new.float().view(B, H, 1, d), *held)
    # weights and result each rounded to bfloat16: 2 x 2^-8 of sum p |v|, which is at most the largest |v|
    assert (got.float() - want.view(B, H, d)).abs().max() <= 2 * 2.0 ** -8 * held[1].abs().max()
    assert (lse - want_lse.view(B, H)).abs().max() < 1e-4
    assert o.shape == q.shape and torch.isfinite(o.float()).all()

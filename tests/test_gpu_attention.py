"""Attention over a CSR pattern, forward and backward, against the formulas in 64 bits (tests/attention_plain.py has the bounds)."""
import numpy as np
import pytest
import torch

from tests import attention_plain as plain

pytestmark = pytest.mark.gpu


def _binding():
    from paper_2311_00368_b200 import binding
    return binding


def _mask(rng, kind, M, K):
    if kind == "random":
        m = rng.random((M, K)) < 0.15
        m[rng.random(M) < 0.1] = False           # rows that see nothing
    elif kind == "sparse":
        m = rng.random((M, K)) < 3.0 / max(3, K)
    elif kind == "window":
        i, j = np.arange(M)[:, None] + K - M, np.arange(K)[None, :]
        m = (j <= i) & (j > i - 200)
    elif kind == "full":
        m = np.ones((M, K), bool)
    else:
        m = np.zeros((M, K), bool)
    return m


class Problem:
    def __init__(self, seed, B=1, H=1, Hkv=1, M=64, K=64, d=64, kind="random", per="all", dtype=torch.float32, strided=False, spread=1.0):
        rng = np.random.default_rng(seed)
        n = {"all": 1, "sequence": B, "problem": B * H}[per]
        masks = [_mask(rng, kind, M, K) for _ in range(n)]
        lead = {"all": (1, 1), "sequence": (B, 1), "problem": (B, H)}[per]
        self.mask = torch.from_numpy(np.stack(masks)).view(*lead, M, K).expand(B, H, M, K).cuda()
        if per == "all":
            self.row_ptr, self.col_idx = (t.cuda() for t in plain.csr(masks[0]))
        else:
            self.row_ptr, self.col_idx = (t.cuda() for t in plain.stacked(masks, (B,) if per == "sequence" else (B, H)))
        gen = torch.Generator().manual_seed(seed)

        def operand(h, rows, f=1.0):
            t = (torch.randn((B, rows, h, d), generator=gen) * f).to(dtype).cuda()
            return t.transpose(1, 2) if strided else t.transpose(1, 2).contiguous()
        self.q, self.k, self.v, self.do = operand(H, M, spread), operand(Hkv, K), operand(Hkv, K), operand(H, M)
        self.dtype, self.K, self.scale = dtype, K, d ** -0.5

    def plan(self):
        return _binding().attention_plan(self.row_ptr, self.col_idx, self.K)

    def forward(self, algo=0, plan=None, **more):
        return _binding().attention(self.row_ptr, self.col_idx, self.q, self.k, self.v, plan=plan, algo=algo, dtype=self.dtype, **more)

    def backward(self, o, lse, plan, algo=0, **more):
        return _binding().attention_backward(self.row_ptr, self.col_idx, self.q, self.k, self.v, o, lse, self.do, plan, algo=algo, dtype=self.dtype, **more)

    def check(self, algo, with_plan=True):
        plan = self.plan()
        o, lse = self.forward(algo, plan if with_plan else None)
        want_o, want_lse, bound_o, bound_lse = plain.forward(self.mask, self.q, self.k, self.v, self.scale)
        worst = plain.inside(lse, want_lse, bound_lse)
        assert worst <= 1, f"lse: {worst:.3g} x the bound"
        worst = plain.inside(o, want_o, bound_o)
        assert worst <= 1, f"O: {worst:.3g} x the bound"
        if algo:
            assert _binding().attention_last_algo() == algo
        got = self.backward(o, lse, plan, algo)
        want, bound = plain.backward(self.mask, self.q, self.k, self.v, o, lse, self.do, self.scale)
        for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bound):
            worst = plain.inside(g, w, b)
            assert worst <= 1, f"{name}: {worst:.3g} x the bound"
        again = (*self.forward(algo, plan if with_plan else None), *self.backward(o, lse, plan, algo))
        for a, b in zip(again, (o, lse, *got)):
            assert torch.equal(a, b), "the same call gave other bits"


SHAPES = [
    dict(M=1, K=1, d=1, kind="full"),
    dict(M=1, K=300, d=64, kind="full"),
    dict(M=3, K=5, d=7),
    dict(B=2, H=3, Hkv=3, M=150, K=290, d=50, per="sequence"),
    dict(H=4, Hkv=2, M=257, K=130, d=33, strided=True),
    dict(H=6, Hkv=2, M=130, K=129, d=128, per="problem", strided=True),
    dict(M=100, K=700, d=256, kind="sparse"),
    dict(M=70, K=90, d=200),
    dict(B=2, H=2, Hkv=1, M=128, K=256, d=64, kind="window"),
    dict(M=64, K=64, d=64, kind="nothing"),
    dict(M=300, K=100, d=96, kind="full"),
]


@pytest.mark.parametrize("i", range(len(SHAPES)))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_row_kernels(i, dtype):
    Problem(100 + i, dtype=dtype, **SHAPES[i]).check(_binding().ALGO_ROW)


@pytest.mark.parametrize("i", [1, 3, 8])
def test_row_kernels_without_a_plan(i):
    Problem(200 + i, **SHAPES[i]).check(_binding().ALGO_ROW, with_plan=False)


TILE_SHAPES = [
    dict(M=1, K=300, d=64, kind="full"),
    dict(M=128, K=128, d=64),
    dict(M=128, K=128, d=128, kind="full"),
    dict(B=2, H=3, Hkv=3, M=150, K=290, d=56, per="sequence"),
    dict(H=6, Hkv=2, M=513, K=513, d=128, kind="window", strided=True),
    dict(B=2, H=4, Hkv=1, M=1100, K=1300, d=64, per="problem", strided=True),
    dict(H=2, Hkv=1, M=900, K=640, d=80, kind="sparse"),
    dict(M=640, K=1100, d=8),
    dict(M=200, K=200, d=64, kind="nothing"),
    dict(M=1000, K=1000, d=96, kind="full", spread=4.0),
    dict(M=700, K=2100, d=128, spread=8.0),
    dict(M=1, K=1, d=1, kind="full"),                                       # widths that are staged
    dict(B=2, H=4, Hkv=2, M=300, K=410, d=83, per="sequence", strided=True),
    dict(H=3, Hkv=3, M=513, K=513, d=121, kind="window"),
    dict(B=3, H=2, Hkv=1, M=140, K=700, d=50, per="problem", spread=4.0),
    dict(M=1, K=8192, d=64, kind="full"),                                   # few blocks with many tiles: cut into parts
    dict(H=4, Hkv=2, M=130, K=5000, d=128, spread=8.0, strided=True),
    dict(B=2, H=2, Hkv=1, M=300, K=3001, d=72, kind="window", per="sequence"),
    dict(H=2, Hkv=2, M=100, K=2500, d=43),
]


@pytest.mark.parametrize("i", range(len(TILE_SHAPES)))
def test_tile_kernels(i):
    Problem(300 + i, dtype=torch.bfloat16, **TILE_SHAPES[i]).check(_binding().ALGO_TILE)


TILE32_SHAPES = [
    dict(M=1, K=1, d=1, kind="full"),
    dict(M=1, K=300, d=64, kind="full"),
    dict(M=128, K=128, d=64),
    dict(B=2, H=3, Hkv=3, M=150, K=290, d=50, per="sequence"),
    dict(H=6, Hkv=2, M=513, K=513, d=33, kind="window", strided=True),
    dict(B=2, H=4, Hkv=1, M=1100, K=1300, d=64, per="problem", strided=True),
    dict(H=2, Hkv=1, M=900, K=640, d=16, kind="sparse"),
    dict(M=200, K=200, d=64, kind="nothing"),
    dict(M=1000, K=1000, d=48, kind="full", spread=4.0),
    dict(B=3, H=2, Hkv=2, M=260, K=2100, d=64, spread=8.0),
    dict(M=1, K=1, d=65, kind="full"),                                     # widths whose products go through memory
    dict(H=4, Hkv=2, M=300, K=410, d=128, strided=True),
    dict(B=2, H=4, Hkv=2, M=513, K=513, d=97, kind="window", per="sequence"),
    dict(B=3, H=2, Hkv=1, M=260, K=900, d=80, per="problem", spread=4.0),
    dict(M=200, K=200, d=100, kind="nothing"),
    dict(H=2, Hkv=1, M=900, K=640, d=128, kind="sparse"),
]


@pytest.mark.parametrize("i", range(len(TILE32_SHAPES)))
def test_tile_kernels_on_fp32(i):
    """fp32 operands on the tensor cores: what is left out of a product of planes is below 2^-23 of each term, and 24 truncated additions
    are off by 24 u at most; the bound of the dot products, 2 (d + 6) u sum|terms| with one product of six planes per 16 elements, holds them."""
    Problem(350 + i, **TILE32_SHAPES[i]).check(_binding().ALGO_TILE)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_choice_of_the_library(dtype):
    Problem(400, B=2, H=4, Hkv=2, M=300, K=400, d=64, dtype=dtype).check(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_few_entries_go_row_by_row_and_many_by_tiles(dtype):
    b = _binding()
    for more, algo in ((dict(M=4000, K=300, kind="sparse"), b.ALGO_ROW), (dict(M=1000, K=1000, kind="sparse"), b.ALGO_ROW),
                       (dict(H=8, Hkv=2, M=2000, K=2000, kind="full"), b.ALGO_TILE)):
        p = Problem(401, d=64, dtype=dtype, **more)
        p.forward(0, p.plan())
        assert b.attention_last_algo() == algo, more


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("algo", [1, 3])
@pytest.mark.parametrize("K, d", [(300, 64), (300, 100), (4000, 100)])
def test_what_no_entry_names_does_not_matter(algo, dtype, K, d):
    """NaN and infinities in rows of Q, K, V and dO that no entry names, next to ones that entries do name."""
    p = Problem(500, H=2, M=300, K=K, d=d, dtype=dtype)
    m = p.mask[0, 0].clone()
    m[:, 40:50] = False
    m[200:210] = False
    p.row_ptr, p.col_idx = (t.cuda() for t in plain.csr(m.cpu().numpy()))
    p.mask = m.expand(1, 2, 300, K)
    p.k[:, :, 40:45] = float("nan")
    p.v[:, :, 40:45] = float("nan")
    p.k[:, :, 45:50] = float("inf")
    p.v[:, :, 45:50] = float("-inf")
    p.q[:, :, 200:205] = float("nan")
    p.do[:, :, 200:205] = float("inf")
    p.q[:, :, 205:210] = float("inf")
    p.do[:, :, 205:210] = float("nan")
    p.check(algo)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("algo", [1, 3])
@pytest.mark.parametrize("K, d", [(256, 64), (2500, 90)])
def test_nan_reaches_the_rows_that_name_it(algo, dtype, K, d):
    p = Problem(501, M=256, K=K, d=d, dtype=dtype)
    p.v[0, 0, 7, 3] = float("nan")
    o, lse = p.forward(algo, p.plan())
    rows = p.mask[0, 0, :, 7]
    assert torch.equal(torch.isnan(o[0, 0, :, 3]), rows)
    assert not torch.isnan(o[0, 0, ~rows]).any() and not torch.isnan(lse).any()


def test_columns_in_any_order():
    p = Problem(502, M=200, K=300, d=64, dtype=torch.bfloat16)
    ends, g = p.row_ptr.tolist(), torch.Generator().manual_seed(1)
    for a, e in zip(ends, ends[1:]):
        p.col_idx[a:e] = p.col_idx[a:e][torch.randperm(e - a, generator=g).cuda()]
    for algo in (1, 3):
        p.check(algo)


def test_patterns_that_a_plan_refuses():
    b = _binding()
    rp = torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda")
    ok = torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda")
    b.attention_plan(rp, ok, 2)
    for bad in ([1, 1, 0], [0, 2, 1], [0, -1, 1]):
        with pytest.raises(b.B2spError) as e:
            b.attention_plan(rp, torch.tensor(bad, dtype=torch.int32, device="cuda"), 2)
        assert e.value.status == 3
    for bad in ([0, 3, 2], [1, 2, 3], [0, 2, 4]):
        with pytest.raises(b.B2spError) as e:
            b.attention_plan(torch.tensor(bad, dtype=torch.int32, device="cuda"), ok, 2)
        assert e.value.status == 3


def test_without_a_plan_each_entry_is_a_term():
    b = _binding()
    rp = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    ci = torch.tensor([1, 1, 0], dtype=torch.int32, device="cuda")
    q, k = torch.zeros((1, 1, 1, 4), device="cuda"), torch.zeros((1, 1, 2, 4), device="cuda")
    v = torch.tensor([[0.0] * 4, [3.0] * 4], device="cuda").view(1, 1, 2, 4)
    o, lse = b.attention(rp, ci, q, k, v)
    assert torch.allclose(o, torch.full_like(o, 2.0)) and abs(float(lse) - np.log(3)) < 1e-6


def test_gradients_against_differences():
    """Directional derivatives of sum(O * dO) by central differences of the formula in 64 bits.  h = 1e-4: the differences' own error
    (h^2 times a third derivative of order 10, and 2^-53 / h) is below 1e-6; the kernels' is the bound's, below 1e-4 here."""
    p = Problem(503, H=2, Hkv=1, M=40, K=50, d=16)
    plan = p.plan()
    o, lse = p.forward(plan=plan)
    grads = p.backward(o, lse, plan)
    gen = torch.Generator().manual_seed(9)
    base = [t.double() for t in (p.q, p.k, p.v)]
    for which in range(3):
        way = torch.randn(base[which].shape, generator=gen).double().cuda()
        ends = []
        for h in (1e-4, -1e-4):
            at = list(base)
            at[which] = at[which] + h * way
            group = p.q.shape[1]
            s = (at[0] @ at[1].repeat_interleave(group, 1).transpose(2, 3) * p.scale).masked_fill(~p.mask, -np.inf)
            w = torch.where(p.mask, torch.exp(s - s.amax(3, keepdim=True).clamp(min=-1e30)), 0.0)
            out = (w / w.sum(3, keepdim=True).clamp(min=1e-300)) @ at[2].repeat_interleave(group, 1)
            ends.append(float((out * p.do.double()).sum()))
        slope = (ends[0] - ends[1]) / 2e-4
        got = float((grads[which].double() * way).sum())
        size = float((grads[which].double() * way).abs().sum())
        assert abs(got - slope) <= 1e-5 * size + 1e-5, (which, got, slope)


@pytest.mark.parametrize("algo", [1, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [dict(M=600, K=700, d=64), dict(M=100, K=2600, d=100)])   # (and: products in memory, copies, parts)
def test_captured_and_replayed_beside_another_graph(algo, dtype, sizes):
    """Two graphs of forward and backward, captured on one stream, replayed at once on two: neither disturbs the other."""
    ps = [Problem(600 + i, H=2, dtype=dtype, **sizes) for i in range(2)]
    plans = [p.plan() for p in ps]
    want = []
    for p, plan in zip(ps, plans):
        o, lse = p.forward(algo, plan)
        want.append((o, lse, *p.backward(o, lse, plan, algo)))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for p, plan in zip(ps, plans):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o, lse = p.forward(algo, plan)
            outs.append((o, lse, *p.backward(o, lse, plan, algo)))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        for a, b in zip(got, ref):
            assert torch.equal(a, b)


def test_outputs_that_the_caller_gives():
    """Views with room between rows: what lies there stays as it was."""
    p = Problem(700, H=2, Hkv=2, M=130, K=140, d=64, dtype=torch.bfloat16)
    plan = p.plan()
    for algo in (1, 3):
        o, lse = p.forward(algo, plan)
        room = torch.full((1, 2, 135, 72), 5.0, dtype=torch.bfloat16, device="cuda")
        view = room[:, :, :130, :64]
        got, _ = p.forward(algo, plan, out=view)
        assert got.data_ptr() == room.data_ptr() and torch.equal(view, o)
        assert (room[:, :, 130:] == 5).all() and (room[..., 64:] == 5).all()
        rooms = [torch.full((1, 2, 150, 72), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        rows = (130, 140, 140)
        views = [r[:, :, :n, :64] for r, n in zip(rooms, rows)]
        ref = p.backward(o, lse, plan, algo)
        p.backward(o, lse, plan, algo, dq=views[0], dk=views[1], dv=views[2])
        for r, n, w, a in zip(rooms, rows, views, ref):
            assert torch.equal(w, a) and (r[:, :, n:] == 5).all() and (r[..., 64:] == 5).all()


def test_another_stream():
    p = Problem(701, H=2, M=500, K=500, d=64, dtype=torch.bfloat16)
    plan = p.plan()
    o, lse = p.forward(plan=plan)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        o2, lse2 = p.forward(plan=plan)
        grads = p.backward(o2, lse2, plan)
    s.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, b in zip(grads, p.backward(o, lse, plan)):
        assert torch.equal(a, b)


def test_no_rows_or_no_columns():
    b = _binding()
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    plan = b.attention_plan(i32(0), i32(), 5)
    o, lse = b.attention(i32(0), i32(), z(1, 1, 0, 8), z(1, 1, 5, 8), z(1, 1, 5, 8))
    assert o.shape == (1, 1, 0, 8)
    rp, ci = plan.row_ptr, plan.col_idx
    dq, dk, dv = b.attention_backward(rp, ci, z(1, 1, 0, 8), z(1, 1, 5, 8) + 1, z(1, 1, 5, 8), o, lse, z(1, 1, 0, 8), plan)
    assert (dk == 0).all() and (dv == 0).all()
    rp, ci = i32(0, 0, 0), i32()
    plan = b.attention_plan(rp, ci, 0)
    o, lse = b.attention(rp, ci, z(1, 1, 2, 8) + 1, z(1, 1, 0, 8), z(1, 1, 0, 8), plan=plan)
    assert (o == 0).all() and (lse == -np.inf).all()
    dq, dk, dv = b.attention_backward(rp, ci, z(1, 1, 2, 8), z(1, 1, 0, 8), z(1, 1, 0, 8), o, lse, z(1, 1, 2, 8), plan)
    assert (dq == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("more", [dict(H=8, Hkv=2, M=1200, K=1200, kind="window"), dict(B=2, H=3, Hkv=3, M=513, K=300, per="problem"),
                                  dict(H=2, Hkv=1, M=150, K=4000), dict(B=4, M=4000, K=140), dict(H=2, Hkv=1, M=1000, K=900, d=111)])
def test_no_wait_runs_out(more, dtype):
    """The tile kernels' waits are bounded and a row that one of them gives up is taken otherwise: the status word tells."""
    b, p = _binding(), Problem(700, **{"d": 64, "dtype": dtype, **more})
    plan, ws = p.plan(), torch.empty(1 << 29, dtype=torch.uint8, device="cuda")
    for _ in range(5):
        o, lse = p.forward(b.ALGO_TILE, plan, workspace=ws)
        assert b.device_status(ws) == 0
        p.backward(o, lse, plan, b.ALGO_TILE, workspace=ws)
        assert b.device_status(ws) == 0


def test_a_workspace_of_the_wrong_kind():
    p = Problem(701)
    for ws in (torch.empty(1 << 20, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            p.forward(0, p.plan(), workspace=ws)

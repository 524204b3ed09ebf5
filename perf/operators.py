"""Attention over a CSR pattern, for training and for serving from a cache held in 4 bits: the calls whose speed is looked at.

The library's FusedMM is attention without its softmax.  The operators here are what a model around it calls:

  attention           O_i = sum_j softmax_j(scale q_i . k_j) v_j over the stored positions of row i, and the row's log-sum
  attention_backward  dQ, dK, dV from Q, K, V, O, the log-sums and dO; the probabilities are computed again
  kv4_write           new rows of a cache are quantised to 4 bits as they are written, and read back
  kv4_read            rows of such a cache, in any order
  attention_kv4       query tokens over the rows of such a cache that their CSR rows name

An attention case holds: batch, heads, kv_heads (heads / kv_heads query heads share one K and V), M, K (the pattern is M x K),
d (head width), density, pattern ("random"; "band": a 128-wide diagonal band and random extras; "window": each query sees the
last density * K keys up to its own, and the first 64), per (the pattern belongs to "all" problems, to a "sequence" or to each
"problem"), empty (share of rows that see nothing, as rows of padding do), dtype.
A cache case holds: tokens, kv_heads, d, slots, dtype (of what is written and of what is read).
An attention_kv4 case holds: M query tokens, heads, kv_heads, d, slots, longest (row lengths are spread over 1 to longest;
a single row has that length).
"""
import math

import torch

own = False

_BAND = 128
_SINKS = 64
_CELLS_MOST = 16 * 8192 * 8192   # batch * heads * M * K of the largest listed attention


def _attention(name, op, batch, heads, kv_heads, M, K, d, density, pattern="random", per="all", empty=0.0, dtype="bf16"):
    c = dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, M=M, K=K, d=d, density=density, pattern=pattern, per=per,
             empty=empty, dtype=dtype)
    return c if name is None else dict(c, name=name)


def _cache(name, op, tokens, kv_heads, d, slots, dtype="bf16"):
    c = dict(op=op, tokens=tokens, kv_heads=kv_heads, d=d, slots=slots, dtype=dtype)
    return c if name is None else dict(c, name=name)


def _serve(name, M, heads, kv_heads, d, slots, longest):
    c = dict(op="attention_kv4", M=M, heads=heads, kv_heads=kv_heads, d=d, slots=slots, longest=longest)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a short prompt in a small model, on the smallest workload's pattern: what a call costs when there is little to do
        _attention("fwd_small", "attention", 1, 4, 4, 256, 256, 64, 0.10),
        # the eight attention problems of the named workloads, each with a pattern of its own
        _attention("fwd_8x4096", "attention", 8, 1, 1, 4096, 4096, 64, 0.20, "band", "problem"),
        # a long prompt under a sliding window with a few keys that all queries see; four query heads share keys and values
        _attention("fwd_window_8k", "attention", 1, 16, 4, 8192, 8192, 128, 0.125, "window"),
        # sizes that are a multiple of nothing, in fp32, with rows of padding
        _attention("fwd_ragged_fp32", "attention", 2, 3, 3, 1501, 2903, 50, 0.12, "random", "sequence", 0.05, "fp32"),
        # the backward passes of the last three
        _attention("bwd_8x4096", "attention_backward", 8, 1, 1, 4096, 4096, 64, 0.20, "band", "problem"),
        _attention("bwd_window_8k", "attention_backward", 1, 16, 4, 8192, 8192, 128, 0.125, "window"),
        _attention("bwd_ragged_fp32", "attention_backward", 2, 3, 3, 1501, 2903, 50, 0.12, "random", "sequence", 0.05, "fp32"),
        # one new token for each of 64 sequences: written to the cache, and read back
        _cache("kv4_write_64", "kv4_write", 64, 8, 128, 65536),
        # prompts of 16384 tokens in all
        _cache("kv4_write_16k", "kv4_write", 16384, 8, 128, 131072),
        # rows of a cache moved elsewhere, in 16 bits
        _cache("kv4_read_64k", "kv4_read", 65536, 8, 64, 262144),
        # one sequence, its next token
        _serve("kv4_one_token", 1, 32, 8, 128, 65536, 32768),
        # 64 sequences of all lengths, one token each
        _serve("kv4_batch_64", 64, 32, 8, 128, 786432, 16384),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: each operator, sizes over the whole range, odd ones among them, each pattern, type and sharing of heads."""
    op = rng.choice(["attention", "attention", "attention_backward", "attention_backward", "kv4_write", "kv4_read",
                     "attention_kv4", "attention_kv4"])
    if op in ("attention", "attention_backward"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        pattern = rng.choice(["random", "band", "window"])
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        heads = kv_heads * rng.choice([1, 1, 2, 4, 5])
        batch = rng.choice([1, 1, 2, 3, 8])
        K = _log_uniform(rng, 64, 8192)
        M = K if pattern != "random" or rng.random() < 0.5 else _log_uniform(rng, 1, 8192)
        if rng.random() < 0.4:
            K = max(128, K // 128 * 128)
            M = K if pattern != "random" else M
        density = round(math.exp(rng.uniform(math.log(0.02), math.log(0.30))), 3)
        most = _CELLS_MOST if dtype == "bf16" else _CELLS_MOST // 8
        while batch * heads * M * K > most:
            if batch > 1:
                batch -= 1
            elif heads > kv_heads:
                heads -= kv_heads
            elif kv_heads > 1:
                heads = kv_heads = kv_heads - 1
            else:
                M = K = M // 2
        d = rng.choice([64, 64, 128, 128, 32, 80, 96, rng.randint(9, 128)])
        return _attention(None, op, batch, heads, kv_heads, M, K, d, density, pattern, rng.choice(["all", "sequence", "problem"]),
                          rng.choice([0.0, 0.0, 0.05]), dtype)
    d = rng.choice([64, 64, 128, 128, 96, 80, rng.randint(17, 128)])
    kv_heads = rng.choice([1, 2, 4, 8])
    if op == "attention_kv4":
        longest, M = _log_uniform(rng, 1, 32768), _log_uniform(rng, 1, 256)
        while M * longest > 64 * 16384:
            M = max(1, M // 2)
        return _serve(None, M, kv_heads * rng.choice([1, 2, 4, 6, 8, 16]), kv_heads, d, max(1024, M * longest * 3 // 4), longest)
    tokens = _log_uniform(rng, 1, 16384 if op == "kv4_write" else 65536)
    return _cache(None, op, tokens, kv_heads, d, max(1024, 4 * tokens), rng.choice(["bf16", "bf16", "fp32"]))


_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _patterns(case):
    return {"all": 1, "sequence": case["batch"], "problem": case["batch"] * case["heads"]}[case["per"]]


def _mask(case, gen):
    """[patterns, M, K] truth values."""
    P, M, K = _patterns(case), case["M"], case["K"]
    i = torch.arange(M, device="cuda")[:, None] + (K - M)
    j = torch.arange(K, device="cuda")[None, :]
    masks = []
    for _ in range(P):
        if case["pattern"] == "window":
            seen = max(1, int(case["density"] * K))
            m = (j <= i) & ((j > i - seen) | (j < _SINKS))
        else:
            extra = case["density"]
            if case["pattern"] == "band":
                extra = max(0.0, extra - _BAND / K) / max(1e-9, 1 - _BAND / K)
            m = torch.rand((M, K), generator=gen, device="cuda") < extra
            if case["pattern"] == "band":
                m |= (j >= i - _BAND // 2) & (j < i + _BAND // 2)
        if case["empty"]:
            m = m & (torch.rand((M, 1), generator=gen, device="cuda") >= case["empty"])
        masks.append(m)
    return torch.stack(masks)


def _csr(mask):
    """row_ptr [P, M + 1], col_idx [P, longest] (one pattern: without the first dimension)."""
    P, M, K = mask.shape
    row_ptr = torch.zeros((P, M + 1), dtype=torch.int32, device="cuda")
    row_ptr[:, 1:] = mask.sum(2).cumsum(1)
    at = mask.view(P, -1)
    cols = [(at[p].nonzero().view(-1) % K).to(torch.int32) for p in range(P)]
    col_idx = torch.zeros((P, max(1, max(c.numel() for c in cols))), dtype=torch.int32, device="cuda")
    for p in range(P):
        col_idx[p, :cols[p].numel()] = cols[p]
    return (row_ptr[0], col_idx[0]) if P == 1 else (row_ptr, col_idx)


def _per_problem(case, t):
    """A pattern's tensor with the dimensions [batch, heads] or what broadcasts to them in front."""
    P = _patterns(case)
    if P == 1:
        return t.view((1, 1) + t.shape[1:])
    if case["per"] == "sequence":
        return t.view((case["batch"], 1) + t.shape[1:])
    return t.view((case["batch"], case["heads"]) + t.shape[1:])


def _prepare_attention(case, gen):
    B, H, Hkv, M, K, d = (case[n] for n in ("batch", "heads", "kv_heads", "M", "K", "d"))
    dtype = _DTYPE[case["dtype"]]
    # as a projection leaves them: [batch, tokens, heads, d], seen as [batch, heads, tokens, d]
    rows = lambda n, h: torch.randn((B, n, h, d), generator=gen, device="cuda").to(dtype).transpose(1, 2)  # noqa: E731
    state = {"case": case, "scale": d ** -0.5, "q": rows(M, H), "k": rows(K, Hkv), "v": rows(K, Hkv)}
    mask = _mask(case, gen)
    row_ptr, col_idx = _csr(mask)
    if case["per"] == "problem" and mask.shape[0] > 1:
        row_ptr, col_idx = row_ptr.view(B, H, -1), col_idx.view(B, H, -1)
    # the fixed mask that a program keeps, in the form that each side's calls take
    state.update(row_ptr=row_ptr, col_idx=col_idx, mask=_per_problem(case, mask))
    if case["op"] == "attention_backward":
        state["out"], state["lse"] = _plain_attention(state)
        state["dout"] = rows(M, H)
    if own:
        from paper_2311_00368_b200 import binding
        state["plan"] = binding.attention_plan(row_ptr, col_idx, K)
    return state


def _groups(d):
    return (d + 31) // 32


def _quantise(x):
    """x [..., d] -> codes [..., 16 * groups] (uint8), scales [..., groups] (bf16).

    A group of 32 neighbours along d has the scale s = bf16(largest |x| / 7), and x is held as the whole number
    clamp(round(x / s), -7, 7) + 8, in 4 bits.  Elements 4 g to 4 g + 3 of group c are the 16 bits at place g * groups + c."""
    d, G = x.shape[-1], _groups(x.shape[-1])
    x = torch.nn.functional.pad(x.float(), (0, 32 * G - d)).unflatten(-1, (G, 32))
    seven = torch.full((), 7.0, device=x.device)
    s = (x.abs().amax(-1) / seven).to(torch.bfloat16)
    c = torch.where(s[..., None] > 0, (x / s[..., None].float()).round().clamp(-7, 7), 0).to(torch.int32) + 8
    c = c.unflatten(-1, (8, 4)).transpose(-3, -2)                       # [..., 8, G, 4]
    word = c[..., 0] | c[..., 1] << 4 | c[..., 2] << 8 | c[..., 3] << 12
    return torch.stack((word & 255, word >> 8), -1).to(torch.uint8).flatten(-3), s


def _values(codes, scales, d):
    """The fp32 values that codes [..., 16 * groups] and scales [..., groups] stand for: [..., d]."""
    G = scales.shape[-1]
    byte = codes.unflatten(-1, (8, G, 2)).to(torch.int32)
    c = torch.stack((byte & 15, byte >> 4), -1).flatten(-2) - 8         # [..., 8, G, 4]
    return (c.transpose(-3, -2).flatten(-2) * scales[..., None].float()).flatten(-2)[..., :d]


def _cache_of(gen, kv_heads, slots, d, filled):
    """codes [kv_heads, slots, 16 * groups], scales [kv_heads, slots, groups] of a cache with something in it, or nothing."""
    G = _groups(d)
    codes = torch.full((kv_heads, slots, 16 * G), 0x88, dtype=torch.uint8, device="cuda")
    scales = torch.zeros((kv_heads, slots, G), dtype=torch.bfloat16, device="cuda")
    if filled:
        for h in range(kv_heads):
            for a in range(0, slots, 1 << 17):
                x = torch.randn((min(slots, a + (1 << 17)) - a, d), generator=gen, device="cuda")
                codes[h, a:a + x.shape[0]], scales[h, a:a + x.shape[0]] = _quantise(x.to(torch.bfloat16))
    return codes, scales


def _prepare_cache(case, gen):
    T, H, d, slots = case["tokens"], case["kv_heads"], case["d"], case["slots"]
    dtype = _DTYPE[case["dtype"]]
    write = case["op"] == "kv4_write"
    codes, scales = _cache_of(gen, H, slots, d, not write)
    state = {"case": case, "dtype": dtype, "codes": codes, "scales": scales,
             "slots": torch.randperm(slots, generator=gen, device="cuda")[:T].to(torch.int32)}
    if write:
        state["x"] = torch.randn((T, H, d), generator=gen, device="cuda").to(dtype)
    return state


def _prepare_serve(case, gen):
    M, H, Hkv, d, slots, longest = (case[n] for n in ("M", "heads", "kv_heads", "d", "slots", "longest"))
    lengths = torch.randint(1, longest + 1, (M,), generator=gen, device="cuda")
    if M == 1:
        lengths[0] = longest
    row_ptr = torch.zeros(M + 1, dtype=torch.int32, device="cuda")
    row_ptr[1:] = lengths.cumsum(0)
    n = int(row_ptr[-1])
    # sequences own runs of 64 rows of the cache, which lie in any order
    runs = torch.randperm((slots + 63) // 64, generator=gen, device="cuda")
    at = torch.arange(n, device="cuda")
    col_idx = ((runs[(at // 64) % runs.numel()] * 64 + at % 64) % slots).to(torch.int32)
    state = {"case": case, "scale": d ** -0.5, "row_ptr": row_ptr, "col_idx": col_idx, "longest": int(lengths.max()),
             "q": torch.randn((M, H, d), generator=gen, device="cuda").to(torch.bfloat16)}
    state["k_codes"], state["k_scales"] = _cache_of(gen, Hkv, slots, d, True)
    state["v_codes"], state["v_scales"] = _cache_of(gen, Hkv, slots, d, True)
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "attention_kv4":
        return _prepare_serve(case, gen)
    return (_prepare_cache if case["op"].startswith("kv4") else _prepare_attention)(case, gen)


def _shared(state, t):
    """K or V [batch, kv_heads, K, d] in fp32, each as often as query heads share it."""
    t, H = t.float(), state["case"]["heads"]
    B, Hkv, K, d = t.shape
    return t[:, :, None].expand(B, Hkv, H // Hkv, K, d).reshape(B, H, K, d)


def _plain_attention(state):
    q, k, v = state["q"].float(), _shared(state, state["k"]), _shared(state, state["v"])
    s = (q @ k.transpose(2, 3)).mul_(state["scale"]).masked_fill_(~state["mask"], -math.inf)
    top = s.amax(3, keepdim=True)
    p = s.sub_(top.clamp(min=-1e30)).exp_()                             # a row that sees nothing: exp(-inf) = 0 throughout
    total = p.sum(3, keepdim=True)
    out = (p @ v) / total.clamp(min=1e-30)
    return out.to(state["q"].dtype), (top + total.log()).squeeze(3)


def _plain_backward(state):
    q, k, v = state["q"].float(), _shared(state, state["k"]), _shared(state, state["v"])
    dout, scale = state["dout"].float(), state["scale"]
    s = (q @ k.transpose(2, 3)).mul_(scale).masked_fill_(~state["mask"], -math.inf)
    p = s.sub_(state["lse"].unsqueeze(3).clamp(min=-1e30)).exp_()
    delta = (dout * state["out"].float()).sum(3, keepdim=True)
    dv = p.transpose(2, 3) @ dout
    ds = (dout @ v.transpose(2, 3)).sub_(delta).mul_(p)
    dq = (ds @ k) * scale
    dk = (ds.transpose(2, 3) @ q) * scale
    B, Hkv, K, d = state["k"].shape
    fold = lambda t: t.view(B, Hkv, -1, K, d).sum(2)  # noqa: E731
    return [t.to(state["q"].dtype) for t in (dq, fold(dk), fold(dv))]


def _plain_write(state):
    codes, scales = _quantise(state["x"])
    at = state["slots"].long()
    state["codes"][:, at], state["scales"][:, at] = codes.transpose(0, 1), scales.transpose(0, 1)


def _plain_read(state):
    at = state["slots"].long()
    x = _values(state["codes"][:, at], state["scales"][:, at], state["case"]["d"])
    return x.transpose(0, 1).to(state["dtype"]).contiguous()


def _plain_serve(state):
    c = state["case"]
    M, H, Hkv, d, L = c["M"], c["heads"], c["kv_heads"], c["d"], state["longest"]
    first, last = state["row_ptr"][:-1, None].long(), state["row_ptr"][1:, None].long()
    at = first + torch.arange(L, device="cuda")[None, :]
    inside = at < last                                                  # [M, L]
    at = state["col_idx"][at.clamp(max=state["col_idx"].numel() - 1)].long()
    k = _values(state["k_codes"][:, at], state["k_scales"][:, at], d)   # [Hkv, M, L, d]
    q = state["q"].float().view(M, Hkv, H // Hkv, d).transpose(0, 1)    # [Hkv, M, H / Hkv, d]
    s = (q @ k.transpose(2, 3)).mul_(state["scale"]).masked_fill_(~inside[None, :, None, :], -math.inf)
    del k
    top = s.amax(3, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    out = (p @ _values(state["v_codes"][:, at], state["v_scales"][:, at], d)) / total
    lse = (top + total.log()).squeeze(3)
    return out.transpose(0, 1).reshape(M, H, d).to(torch.bfloat16), lse.transpose(0, 1).reshape(M, H)


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        if op == "attention":
            return _plain_attention(state)
        if op == "attention_backward":
            return _plain_backward(state)
        if op == "attention_kv4":
            return _plain_serve(state)
        if op == "kv4_write":
            _plain_write(state)
        return _plain_read(state)
    from paper_2311_00368_b200 import binding as b
    if op == "attention":
        return b.attention(state["row_ptr"], state["col_idx"], state["q"], state["k"], state["v"], scale=state["scale"],
                           plan=state["plan"], dtype=_DTYPE[case["dtype"]])
    if op == "attention_backward":
        return b.attention_backward(state["row_ptr"], state["col_idx"], state["q"], state["k"], state["v"], state["out"],
                                    state["lse"], state["dout"], state["plan"], scale=state["scale"], dtype=_DTYPE[case["dtype"]])
    if op == "attention_kv4":
        return b.attention_kv4(state["row_ptr"], state["col_idx"], state["q"], state["k_codes"], state["k_scales"],
                               state["v_codes"], state["v_scales"], scale=state["scale"])
    if op == "kv4_write":
        b.kv4_write(state["x"], state["slots"], state["codes"], state["scales"], dtype=state["dtype"])
    return b.kv4_read(state["slots"], state["codes"], state["scales"], case["d"], dtype=state["dtype"])


def _entries(case):
    """About how many positions a pattern stores."""
    M, K = case["M"], case["K"]
    if case["pattern"] == "window":
        seen = max(1, int(case["density"] * K))
        full = sum(min(max(0, i + K - M + 1), seen + min(_SINKS, max(0, i + K - M + 1 - seen))) for i in range(M))
    elif case["pattern"] == "band":
        full = M * K * max(case["density"], min(1.0, _BAND / K))
    else:
        full = M * K * case["density"]
    return full * (1 - case["empty"])


def work(case):
    if case["op"] == "attention_kv4":
        M, H, Hkv, d = case["M"], case["heads"], case["kv_heads"], case["d"]
        n = case["longest"] if M == 1 else M * (case["longest"] + 1) / 2
        rows = min(n, case["slots"])
        return {"bytes": rows * Hkv * 2 * 18 * _groups(d) + 4 * n + 4 * M * H * (d + 1), "flops": 4 * n * H * d}
    if case["op"].startswith("kv4"):
        n, wide = case["tokens"] * case["kv_heads"], 2 if case["dtype"] == "bf16" else 4
        held = n * 18 * _groups(case["d"])
        full = n * case["d"] * wide
        # read: what is held in, values out; write: values in, held out, and that read again
        return {"bytes": (held + full) * (2 if case["op"] == "kv4_write" else 1) + 4 * case["tokens"], "flops": 2 * n * case["d"]}
    B, H, Hkv, M, K, d = (case[n] for n in ("batch", "heads", "kv_heads", "M", "K", "d"))
    wide = 2 if case["dtype"] == "bf16" else 4
    entries = _entries(case)
    pattern = _patterns(case) * min(4 * entries, M * K / 8)
    q, kv = B * H * M * d * wide, 2 * B * Hkv * K * d * wide
    if case["op"] == "attention":
        return {"bytes": 2 * q + kv + 4 * B * H * M + pattern, "flops": 4 * entries * B * H * d}
    return {"bytes": 4 * q + 2 * kv + 4 * B * H * M + pattern, "flops": 10 * entries * B * H * d}


def exact(case, seed):
    """The definitions in 64 bits, row by row of the batch and head by head."""
    state = prepare(case, seed)
    if case["op"] == "attention_kv4":
        return _exact_serve(state)
    if case["op"].startswith("kv4"):
        return _exact_cache(state)
    B, H, Hkv = case["batch"], case["heads"], case["kv_heads"]
    scale, q, k, v = state["scale"], state["q"], state["k"], state["v"]
    back = case["op"] == "attention_backward"
    if back:
        dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (q, k, v))
    else:
        out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(q.shape[:3], dtype=torch.float64, device="cuda")
    masks = state["mask"].expand(B, H, -1, -1)
    for b in range(B):
        for h in range(H):
            g = h // (H // Hkv)
            Q, Kh, Vh = q[b, h].double(), k[b, g].double(), v[b, g].double()
            logits = torch.einsum("id,jd->ij", Q, Kh) * scale
            logits[~masks[b, h]] = -math.inf
            if not back:
                total = torch.logsumexp(logits, 1)
                weights = torch.softmax(logits, 1)
                weights[total == -math.inf] = 0
                out[b, h], lse[b, h] = weights @ Vh, total
                continue
            sees = masks[b, h].any(1)
            weights = torch.exp(logits - torch.where(sees, state["lse"][b, h].double(), 0.0)[:, None])
            dO = state["dout"][b, h].double()
            dv[b, g] += weights.T @ dO
            dS = weights * (dO @ Vh.T - (dO * state["out"][b, h].double()).sum(1)[:, None])
            dq[b, h] = dS @ Kh * scale
            dk[b, g] += dS.T @ Q * scale
    return [dq, dk, dv] if back else (out, lse)


def _exact_rows(codes, scales, at, d):
    """[rows, kv_heads, d] of a cache, element by element of the definition."""
    G = scales.shape[-1]
    e = torch.arange(d, device="cuda")
    c, r = e // 32, e % 32
    half = (r // 4) * G + c
    nibble = r % 4
    byte = codes[:, at][..., 2 * half + nibble // 2].to(torch.int64)
    whole = torch.where(nibble % 2 == 0, byte % 16, byte // 16) - 8
    return (whole.double() * scales[:, at][..., c].double()).transpose(0, 1)


def _exact_cache(state):
    at, d = state["slots"].long(), state["case"]["d"]
    if state["case"]["op"] == "kv4_read":
        return _exact_rows(state["codes"], state["scales"], at, d)
    x = state["x"].double()
    for a in range(0, d, 32):
        part = x[..., a:a + 32]
        s = (part.abs().amax(-1, keepdim=True) / 7).to(torch.bfloat16).double()
        x[..., a:a + 32] = torch.where(s > 0, (part / s).round().clamp(-7, 7) * s, 0.0)
    return x


def _exact_serve(state):
    c = state["case"]
    M, H, Hkv, d = c["M"], c["heads"], c["kv_heads"], c["d"]
    out = torch.zeros((M, H, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((M, H), dtype=torch.float64, device="cuda")
    ends = state["row_ptr"].tolist()
    for i in range(M):
        at = state["col_idx"][ends[i]:ends[i + 1]].long()
        K = _exact_rows(state["k_codes"], state["k_scales"], at, d).repeat_interleave(H // Hkv, 1)
        V = _exact_rows(state["v_codes"], state["v_scales"], at, d).repeat_interleave(H // Hkv, 1)
        logits = torch.einsum("hd,lhd->hl", state["q"][i].double(), K) * state["scale"]
        lse[i] = torch.logsumexp(logits, 1)
        out[i] = torch.einsum("hl,lhd->hd", torch.softmax(logits, 1), V)
    return out, lse

"""Serving from a cache in pages: the calls whose speed is looked at.

A cache of keys or values is [pages, kv_heads, page, d]: pages of `page` rows in any order, and request r's position p lies in row
p % page of page tables[r, p // page].  A server's step makes the tables, writes the new rows, and lets the new tokens look:

  paged_tables      lengths and new tokens of each request -> pages taken from (and given back to) the stack of free ones, where each
                    token goes, how much it sees; with lists: also the lists of slots that attention over the 4-bit cache takes
  paged_write       the new rows of K and V into their pages; with means: the mean key of every page that was touched
  attention_paged   softmax(scale q . k) v of each new token over the positions that it sees, and the log-sum
  paged_select      for each token and key head the pages whose mean key scores best, then attention_paged over these alone

A paged_tables case holds: requests, longest (lengths are spread over 0 to longest), kind ("decode": one new token each; "mixed":
prompts, single tokens and requests that end), tokens (room in the step), page, lists.
A paged_write case holds: requests, longest, tokens in all (spread over the requests), kv_heads, d, page, means, dtype, layout (of the
cache in memory: "head", a page holds one head's rows after the other's; "row", one row's heads after the other's).
The two attention cases hold: requests, each (new tokens of a request), longest, heads, kv_heads, d, page, padding (tokens behind the
last, which see nothing), dtype, layout, and for paged_select keep (pages of a list).
"""
import math

import torch

own = False

_ROWS_MOST = 64 * 32768          # requests * longest of the largest listed case
_FIRST, _LAST = 1, 2             # pages that paged_select always takes


def _tables(name, requests, longest, kind, tokens, page, lists=False):
    c = dict(op="paged_tables", requests=requests, longest=longest, kind=kind, tokens=tokens, page=page, lists=lists)
    return c if name is None else dict(c, name=name)


def _write(name, requests, longest, tokens, kv_heads, d, page, means=True, dtype="bf16", layout="head"):
    c = dict(op="paged_write", requests=requests, longest=longest, tokens=tokens, kv_heads=kv_heads, d=d, page=page, means=means,
             dtype=dtype, layout=layout)
    return c if name is None else dict(c, name=name)


def _attend(name, op, requests, each, longest, heads, kv_heads, d, page, padding=0, dtype="bf16", layout="head", keep=0):
    c = dict(op=op, requests=requests, each=each, longest=longest, heads=heads, kv_heads=kv_heads, d=d, page=page, padding=padding,
             dtype=dtype, layout=layout)
    if op == "paged_select":
        c["keep"] = keep
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one new token for each of 64 sequences: what a decoding step costs before its first layer
        _tables("tables_decode_64", 64, 4096, "decode", 64, 64),
        # a step of a busy server: prompts, single tokens and requests that end
        _tables("tables_mixed_512", 512, 2048, "mixed", 16384, 16),
        # the lists of slots of 64 sequences for attention over the 4-bit cache
        _tables("tables_lists_64", 64, 16384, "decode", 64, 64, True),
        # the new rows of a decoding step, and the mean keys of the pages that they lie in
        _write("write_decode_64", 64, 1000, 64, 8, 128, 64),
        # prompts of 16384 tokens in all
        _write("write_prompts_16k", 24, 500, 16384, 8, 128, 64),
        # one sequence, its next token
        _attend("paged_one_token", "attention_paged", 1, 1, 32768, 32, 8, 128, 64),
        # 64 sequences of all lengths, one token each
        _attend("paged_batch_64", "attention_paged", 64, 1, 16384, 32, 8, 128, 64),
        # many short sequences with four guessed tokens each to be checked, small pages with the heads of a row together
        _attend("paged_guessed_4", "attention_paged", 128, 4, 700, 16, 4, 64, 16, 0, "bf16", "row"),
        # sizes that are a multiple of nothing, in fp32, with rows of padding
        _attend("paged_ragged_fp32", "attention_paged", 37, 1, 2903, 6, 3, 50, 24, 3, "fp32"),
        # one long sequence of which a token reads 32 pages
        _attend("selected_one_token", "paged_select", 1, 1, 131072, 32, 8, 128, 64, 0, "bf16", "head", 32),
        # 64 sequences of all lengths
        _attend("selected_batch_64", "paged_select", 64, 1, 32768, 32, 8, 128, 64, 0, "bf16", "head", 32),
        # ragged, in fp32
        _attend("selected_ragged_fp32", "paged_select", 21, 2, 2903, 6, 3, 50, 24, 3, "fp32", "row", 13),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: each operator, sizes over the whole range, odd ones among them, each type, layout and sharing of heads."""
    op = rng.choice(["paged_tables", "paged_write", "attention_paged", "attention_paged", "attention_paged", "paged_select",
                     "paged_select"])
    page = rng.choice([16, 16, 32, 64, 64, 128, rng.randint(5, 150)])
    if op == "paged_tables":
        requests = _log_uniform(rng, 1, 512)
        kind = rng.choice(["decode", "mixed"])
        lists = rng.random() < 0.4
        longest = max(8, min(_log_uniform(rng, 16, 16384), 64 * 16384 // requests))
        return _tables(None, requests, longest, kind, requests if kind == "decode" else _log_uniform(rng, requests, 16384), page, lists)
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    layout = rng.choice(["head", "head", "row"])
    d = rng.choice([64, 64, 128, 128, 128, 96, 80, 256, rng.randint(17, 128)])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    if op == "paged_write":
        requests = _log_uniform(rng, 1, 256)
        tokens = max(requests, _log_uniform(rng, 1, 16384 if d <= 128 and dtype == "bf16" else 4096))
        return _write(None, requests, _log_uniform(rng, 16, 1000), tokens, kv_heads, d, page, rng.random() < 0.7, dtype, layout)
    group = rng.choice([1, 2, 4, 4, 6, 8, 16])
    longest = _log_uniform(rng, 1, 32768 if op == "attention_paged" else 131072)
    most = _ROWS_MOST // 2 if op == "attention_paged" else _ROWS_MOST
    if dtype == "fp32" or d > 128:
        most //= 4
    requests = max(1, min(_log_uniform(rng, 1, 512), most // longest))
    each = rng.choice([1, 1, 1, 2, 4]) if requests * longest * 4 <= most else 1
    return _attend(None, op, requests, each, longest, kv_heads * group, kv_heads, d, page, rng.choice([0, 0, 3]), dtype, layout,
                   rng.randint(_FIRST + _LAST, max(8, min(64, 4096 // page))))


_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _pages_of(gen, case, lengths, spare, width):
    """(tables [requests, width] filled as the lengths need, -1 behind; pages in all; the order in which the others are free)."""
    page = case["page"]
    owned = (lengths + page - 1) // page
    used = int(owned.sum())
    pages = used + spare
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    column = torch.arange(width, device="cuda")
    tables = torch.full((lengths.numel(), width), -1, dtype=torch.int32, device="cuda")
    tables[column[None, :] < owned[:, None]] = order[:used]
    return tables, pages, order[used:]


def _added(case, gen):
    """New tokens of each request; -1 where a request ends."""
    R, tokens = case["requests"], case["tokens"]
    if case.get("kind") == "decode" or tokens == R:
        return torch.ones(R, dtype=torch.int32, device="cuda")
    fate = torch.rand(R, generator=gen, device="cuda")
    if case["op"] == "paged_write":
        fate.fill_(1.0)
    prompts = fate >= (0.75 if R > 4 else 0.0)
    if not bool(prompts.any()):
        prompts[0] = True
    ends = (fate < 0.1) & ~prompts
    added = torch.where(ends, -1, 1)
    # what the single tokens leave is spread over the prompts
    left = max(0, tokens - int((added == 1).sum()))
    share = torch.rand(R, generator=gen, device="cuda").add_(0.05) * prompts
    added += (share / share.sum() * left * prompts).long()
    added[prompts.long().argmax()] += max(0, tokens - int(added.clamp(min=0).sum()))
    return added.to(torch.int32)


def _spread(gen, requests, longest):
    """Lengths from 0 to longest, the same ones in another order for another seed."""
    lengths = torch.arange(requests, device="cuda") * (longest + 1) // requests
    return lengths[torch.randperm(requests, generator=gen, device="cuda")].to(torch.int32)


def _prepare_tables(case, gen):
    R, page = case["requests"], case["page"]
    lengths = _spread(gen, R, case["longest"])
    added = _added(case, gen)
    most = 1 if case["kind"] == "decode" else max(R, case["tokens"])
    width = (case["longest"] + most) // page + 1
    tables, pages, free = _pages_of(gen, case, lengths, max(R, case["tokens"]) // page + R + 8, width)
    room = torch.zeros(pages, dtype=torch.int32, device="cuda")
    room[:free.numel()] = free
    state = {"case": case, "lengths": lengths, "added": added, "tables": tables, "pages": pages, "free": room,
             "count": torch.tensor([free.numel()], dtype=torch.int32, device="cuda"), "width": width}
    if case["lists"]:
        state["entries"] = int(lengths.sum()) + max(R, case["tokens"])   # (all that the step could come to)
    return state


def _cache(gen, case, pages, filled):
    """[pages, kv_heads, page, d], rows of a multiple of 16 bytes, laid out as the case says."""
    H, P, d, dtype = case["kv_heads"], case["page"], case["d"], _DTYPE[case["dtype"]]
    wide = -(-d * dtype.itemsize // 16) * 16 // dtype.itemsize
    shape = (pages, H, P, wide) if case["layout"] == "head" else (pages, P, H, wide)
    data = torch.zeros(shape, dtype=dtype, device="cuda")
    if filled:
        step = max(1, (1 << 26) // max(1, H * P * wide))
        for a in range(0, pages, step):
            part = data[a:a + step]
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    return (data if case["layout"] == "head" else data.transpose(1, 2))[..., :d]


def _means_room(case, pages):
    d, dtype = case["d"], _DTYPE[case["dtype"]]
    wide = -(-d * dtype.itemsize // 16) * 16 // dtype.itemsize
    return torch.zeros((pages, case["kv_heads"], wide), dtype=dtype, device="cuda")[..., :d]


def _prepare_write(case, gen):
    R, H, d, page, dtype = case["requests"], case["kv_heads"], case["d"], case["page"], _DTYPE[case["dtype"]]
    lengths = _spread(gen, R, case["longest"])
    added = _added(case, gen)
    row_ptr = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    row_ptr[1:] = added.cumsum(0)
    T = int(row_ptr[-1])
    total = lengths + added
    used = int(((total + page - 1) // page).sum())
    spare = int(((lengths + page - 1) // page).sum()) + T // page + R + 4 - used
    tables, pages, _ = _pages_of(gen, case, total, spare, int((total.max() + page - 1) // page) + 2)
    # as a projection leaves them: rows of K next to rows of V
    kv = torch.randn((T, 2, H, d), generator=gen, device="cuda").to(dtype)
    state = {"case": case, "k": kv[:, 0], "v": kv[:, 1], "row_ptr": row_ptr, "lengths": lengths, "tables": tables,
             "k_pages": _cache(gen, case, pages, True), "v_pages": _cache(gen, case, pages, True)}
    if case["means"]:
        state["means"] = _means_room(case, pages)
    return state


def _prepare_attend(case, gen):
    R, each, H, d, page, dtype = (case["requests"], case["each"], case["heads"], case["d"], case["page"], _DTYPE[case["dtype"]])
    lengths = torch.randint(1, case["longest"] + 1, (R,), generator=gen, device="cuda", dtype=torch.int32)
    if R == 1:
        lengths[0] = case["longest"]
    tables, pages, _ = _pages_of(gen, case, lengths, 4, int((lengths.max() + page - 1) // page) + 1)
    M = R * each + case["padding"]
    rows = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    seen = torch.zeros(M, dtype=torch.int32, device="cuda")
    token = torch.arange(R * each, device="cuda")
    rows[:R * each] = (token // each).to(torch.int32)
    # the last of a request's new tokens sees all of it, the ones before that each one less
    seen[:R * each] = (lengths[token // each] - (each - 1 - token % each)).clamp(min=0).to(torch.int32)
    state = {"case": case, "scale": d ** -0.5, "tables": tables, "rows": rows, "seen": seen, "longest": int(lengths.max()),
             "q": torch.randn((M, H, d), generator=gen, device="cuda").to(dtype),
             "k_pages": _cache(gen, case, pages, True), "v_pages": _cache(gen, case, pages, True)}
    if case["op"] == "paged_select":
        # mean keys, as the writing of the rows left them
        state["means"] = _means_room(case, pages)
        for a in range(0, pages, 4096):
            state["means"][a:a + 4096] = state["k_pages"][a:a + 4096].float().mean(2).to(dtype)
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "paged_tables":
        return _prepare_tables(case, gen)
    return (_prepare_write if case["op"] == "paged_write" else _prepare_attend)(case, gen)


def _prefix(x):
    return torch.cat((torch.zeros(1, dtype=torch.int64, device=x.device), x.long().cumsum(0)))


def _plain_tables(state):
    case, tables, free = state["case"], state["tables"], state["free"]
    page, tokens, width = case["page"], case["tokens"], state["width"]
    lengths, added = state["lengths"].long(), state["added"].long()
    ends, new, count = added < 0, added.clamp(min=0), state["count"].long()[0]
    owned = (lengths + page - 1) // page
    total = torch.where(ends, 0, (lengths + new).clamp(max=width * page))
    need = torch.where(ends, 0, (total + page - 1) // page - owned)
    back = _prefix(torch.where(ends, owned, 0))
    take, row_ptr = _prefix(need), _prefix(new)
    column = torch.arange(width, device="cuda")[None, :]
    given = ends[:, None] & (column < owned[:, None])
    free[(count + back[:-1, None] + column)[given]] = tables[given]
    fresh = (column >= owned[:, None]) & (column < (owned + need)[:, None])
    at = (count + back[-1] - 1 - take[:-1, None] - column + owned[:, None])[fresh]
    tables[fresh] = torch.where(at >= 0, free[at.clamp(min=0)], -1)
    t = torch.arange(tokens, device="cuda")
    r = torch.searchsorted(row_ptr[1:], t, right=True)
    there = r < lengths.numel()
    r = r.clamp(max=lengths.numel() - 1)
    position = lengths[r] + t - row_ptr[r]
    held = tables[r, (position // page).clamp(max=width - 1)].long()
    fits = there & (position < width * page) & (held >= 0)
    slots = torch.where(fits, held * page + position % page, -1)
    counts = torch.stack((count + back[-1] - take[-1], row_ptr[-1], row_ptr[-1] - fits.sum(), take[-1]))
    whole = lambda *x: [y.to(torch.int32) for y in x]  # noqa: E731
    out = whole(total, row_ptr, torch.where(there, r, -1), torch.where(fits, position + 1, 0), slots, counts)
    if case["lists"]:
        ptr = _prefix(total)
        e = torch.arange(state["entries"], device="cuda")
        i = torch.searchsorted(ptr[1:], e, right=True)
        p = e - ptr[i]
        i = i.clamp(max=lengths.numel() - 1)
        held = tables[i, (p // page).clamp(max=width - 1)].long()
        out += whole(ptr.clamp(max=e.numel()), torch.where((e < ptr[-1]) & (held >= 0), held * page + p % page, -1))
    return out + [tables, free]


def _plain_write(state):
    case, k_pages = state["case"], state["k_pages"]
    page, row_ptr, lengths = case["page"], state["row_ptr"].long(), state["lengths"].long()
    t = torch.arange(state["k"].shape[0], device="cuda")
    r = torch.searchsorted(row_ptr[1:], t, right=True)
    position = lengths[r] + t - row_ptr[r]
    at, row = state["tables"][r, position // page].long(), position % page
    k_pages[at, :, row] = state["k"]
    state["v_pages"][at, :, row] = state["v"]
    if not case["means"]:
        return [k_pages, state["v_pages"]]
    filled = torch.zeros(k_pages.shape[0], dtype=torch.int64, device="cuda").scatter_reduce_(0, at, row + 1, "amax")
    touched = filled.nonzero().view(-1)
    n = filled[touched].view(-1, 1, 1, 1)
    inside = torch.arange(page, device="cuda").view(1, 1, page, 1) < n
    state["means"][touched] = (k_pages[touched].float().masked_fill(~inside, 0).sum(2) / n[..., 0]).to(state["means"].dtype)
    return [k_pages, state["v_pages"], state["means"]]


def _plain_over(state, position, inside):
    """Attention of every token over positions [M, kv_heads, L] of its request, those that `inside` names."""
    c = state["case"]
    H, Hkv, d, page = c["heads"], c["kv_heads"], c["d"], c["page"]
    M = position.shape[0]
    rows = state["rows"].long().clamp(min=0).view(M, 1, 1)
    width = state["tables"].shape[1]
    held = state["tables"][rows, (position // page).clamp(0, width - 1)].long().clamp(min=0)
    head = torch.arange(Hkv, device="cuda").view(1, Hkv, 1)
    out = torch.zeros((M, H, d), device="cuda")
    lse = torch.zeros((M, H), device="cuda")
    step = max(1, (1 << 32) // max(1, position.shape[1] * position.shape[2] * d * 4))
    for a in range(0, M, step):
        at, row, keep = held[a:a + step], position[a:a + step] % page, inside[a:a + step]
        at, row, h = torch.broadcast_tensors(at, row, head)
        q = state["q"][a:a + step].float().view(-1, Hkv, H // Hkv, d)
        s = (q @ state["k_pages"][at, h, row].float().transpose(2, 3)).mul_(state["scale"]).masked_fill_(~keep[:, :, None, :], -math.inf)
        top = s.amax(3, keepdim=True)
        p = s.sub_(top.clamp(min=-1e30)).exp_()                         # a token that sees nothing: exp(-inf) = 0 throughout
        total = p.sum(3, keepdim=True)
        v = state["v_pages"][at, h, row].float().masked_fill_(~keep[..., None], 0)
        out[a:a + step] = ((p @ v) / total.clamp(min=1e-30)).reshape(-1, H, d)
        lse[a:a + step] = (top + total.log()).reshape(-1, H)
    return out.to(state["q"].dtype), lse


def _plain_attend(state):
    position = torch.arange(max(1, state["longest"]), device="cuda").view(1, 1, -1).expand(state["q"].shape[0], -1, -1)
    return _plain_over(state, position, position < state["seen"].view(-1, 1, 1))


def _plain_select(state):
    c = state["case"]
    H, Hkv, page, keep = c["heads"], c["kv_heads"], c["page"], c["keep"]
    M, width = state["q"].shape[0], state["tables"].shape[1]
    n = ((state["seen"].long() + page - 1) // page).view(M, 1, 1)
    q = state["q"].double().view(M, Hkv, H // Hkv, -1).sum(2)           # (64 bits: a choice must not hang on the order of a sum)
    held = state["tables"].long().clamp(min=0)[state["rows"].long().clamp(min=0)]
    score = torch.empty((M, Hkv, width), dtype=torch.float64, device="cuda")
    for i in range(M):
        score[i] = torch.matmul(state["means"][held[i]].double().transpose(0, 1), q[i].unsqueeze(2)).squeeze(2)
    p = torch.arange(width, device="cuda").view(1, 1, width)
    score.masked_fill_((p < _FIRST) | (p >= n - _LAST), math.inf).masked_fill_(p >= n, -math.inf)
    best = torch.sort(score, dim=2, descending=True, stable=True).indices[..., :keep]
    if best.shape[2] < keep:
        best = torch.nn.functional.pad(best, (0, keep - best.shape[2]), value=width)
    best = torch.where(best < n, best, 1 << 30).sort(2).values
    return torch.where(best < 1 << 30, best, -1).to(torch.int32)


def _plain_selected(state):
    page = state["case"]["page"]
    lists = _plain_select(state)
    position = (lists.long()[..., None] * page + torch.arange(page, device="cuda")).flatten(2)
    inside = (position >= 0) & (position < state["seen"].view(-1, 1, 1))
    return (lists,) + _plain_over(state, position.clamp(min=0), inside)


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        if op == "paged_tables":
            return _plain_tables(state)
        if op == "paged_write":
            return _plain_write(state)
        return _plain_attend(state) if op == "attention_paged" else _plain_selected(state)
    from paper_2311_00368_b200 import binding as b
    page = case["page"]
    if op == "paged_tables":
        out = list(b.paged_tables(state["lengths"], state["added"], state["tables"], state["free"], state["count"], page,
                                  state["pages"], case["tokens"]))
        if case["lists"]:
            out += b.paged_lists(state["tables"], out[0], page, state["pages"], state["entries"])
        return out + [state["tables"], state["free"]]
    dtype = _DTYPE[case["dtype"]]
    if op == "paged_write":
        out = [state["k_pages"], state["v_pages"]] + ([state["means"]] if case["means"] else [])
        b.paged_write(state["k"], state["v"], state["row_ptr"], state["lengths"], state["tables"], *out, dtype=dtype)
        return out
    lists = None
    if op == "paged_select":
        lists = b.paged_select(state["q"], state["means"], state["tables"], state["seen"], page, case["keep"], first=_FIRST, last=_LAST,
                               rows=state["rows"], dtype=dtype)
    out = b.attention_paged(state["q"], state["k_pages"], state["v_pages"], state["tables"], state["seen"], rows=state["rows"],
                            lists=lists, scale=state["scale"], dtype=dtype)
    return out if lists is None else (lists,) + tuple(out)


def work(case):
    R, page = case["requests"], case["page"]
    if case["op"] == "paged_tables":
        held = R * case["longest"] / 2 + case["tokens"]
        # lengths, new tokens and what they become; three numbers for each token; pages that are new or given back
        n = 4 * (4 * R + 3 * case["tokens"] + 3 * case["tokens"] / page)
        if case["lists"]:
            n += 4 * (held + held / page)
        return {"bytes": n, "flops": 0}
    wide = 2 if case["dtype"] == "bf16" else 4
    H, d = case["kv_heads"], case["d"]
    if case["op"] == "paged_write":
        T = case["tokens"]
        n = 4 * T * H * d * wide
        if case["means"]:
            n += (T / page + R) * H * d * wide + R * page / 2 * H * d * wide
        return {"bytes": n, "flops": T * H * d if case["means"] else 0}
    M, L = R * case["each"], case["longest"]
    seen = L if R == 1 else (L + 1) / 2
    ends = 2 * M * case["heads"] * d * wide
    if case["op"] == "attention_paged":
        return {"bytes": 2 * R * seen * H * d * wide + ends, "flops": 4 * M * seen * case["heads"] * d}
    pages = seen / page + 0.5
    read = min(seen, case["keep"] * page)
    return {"bytes": R * pages * H * d * wide + 2 * M * read * H * d * wide + ends,
            "flops": 2 * M * pages * H * d + 4 * M * read * case["heads"] * d}


def exact(case, seed):
    """The definitions, request by request and token by token."""
    state = prepare(case, seed)
    if case["op"] == "paged_tables":
        return _exact_tables(state)
    return (_exact_write if case["op"] == "paged_write" else _exact_attend)(state)


def _exact_tables(state):
    case = state["case"]
    page, width, tokens = case["page"], state["width"], case["tokens"]
    lengths, added, tables = state["lengths"].tolist(), state["added"].tolist(), state["tables"].tolist()
    stack = state["free"].tolist()
    top = int(state["count"][0])
    for r, more in enumerate(added):
        if more < 0:
            for p in range(-(-lengths[r] // page)):
                stack[top] = tables[r][p]
                top += 1
    row_ptr, totals, rows, seen, slots, taken, lost = [0], [], [], [], [], 0, 0
    for r, more in enumerate(added):
        has = -(-lengths[r] // page)
        total = 0 if more < 0 else min(lengths[r] + more, width * page)
        if more >= 0:
            for p in range(has, -(-total // page)):
                top -= 1
                taken += 1
                tables[r][p] = stack[top] if top >= 0 else -1
        for position in range(lengths[r], lengths[r] + max(more, 0)):
            held = tables[r][position // page] if position < width * page else -1
            if len(rows) == tokens or held < 0:
                lost += 1
            if len(rows) < tokens:
                rows.append(r)
                seen.append(position + 1 if held >= 0 else 0)
                slots.append(held * page + position % page if held >= 0 else -1)
        totals.append(total)
        row_ptr.append(row_ptr[-1] + max(more, 0))
    pad = tokens - len(rows)
    out = [totals, row_ptr, rows + [-1] * pad, seen + [0] * pad, slots + [-1] * pad, [top, row_ptr[-1], lost, taken]]
    if case["lists"]:
        ptr, cols = [0], []
        for r, total in enumerate(totals):
            ptr.append(ptr[-1] + total)
            cols += [tables[r][p // page] * page + p % page if tables[r][p // page] >= 0 else -1 for p in range(total)]
        out += [ptr, cols + [-1] * (state["entries"] - len(cols))]
    return [torch.tensor(x, dtype=torch.int32, device="cuda") for x in out + [tables, stack]]


def _exact_write(state):
    case, k_pages, v_pages = state["case"], state["k_pages"].clone(), state["v_pages"].clone()
    page, ptr, lengths, tables = case["page"], state["row_ptr"].tolist(), state["lengths"].tolist(), state["tables"].tolist()
    means = state["means"].double() if case["means"] else None
    for r, start in enumerate(lengths):
        at, end = start, start + ptr[r + 1] - ptr[r]
        while at < end:
            p, row = tables[r][at // page], at % page
            n = min(page - row, end - at)
            t = ptr[r] + at - start
            k_pages[p, :, row:row + n] = state["k"][t:t + n].transpose(0, 1)
            v_pages[p, :, row:row + n] = state["v"][t:t + n].transpose(0, 1)
            if means is not None:
                means[p] = k_pages[p, :, :row + n].double().mean(1)
            at += n
    return [k_pages, v_pages] + ([means] if case["means"] else [])


def _exact_attend(state):
    c = state["case"]
    H, Hkv, d, page = c["heads"], c["kv_heads"], c["d"], c["page"]
    group, M = H // Hkv, state["q"].shape[0]
    if M * Hkv > 4096:
        return None
    out = torch.zeros((M, H, d), dtype=torch.float64, device="cuda")
    lse = torch.full((M, H), -math.inf, dtype=torch.float64, device="cuda")
    lists = torch.full((M, Hkv, c["keep"]), -1, dtype=torch.int32, device="cuda") if "keep" in c else None
    rows, seen = state["rows"].tolist(), state["seen"].tolist()
    for i in range(M):
        n = -(-seen[i] // page)
        if n == 0:
            continue
        held = state["tables"][rows[i], :n].long()
        for g in range(Hkv):
            q = state["q"][i, g * group:(g + 1) * group].double()
            mine = torch.arange(n, device="cuda")
            if lists is not None:
                if n > c["keep"]:
                    score = torch.mv(state["means"][held, g].double(), q.sum(0))
                    middle = score[_FIRST:n - _LAST].cpu()
                    left = c["keep"] - _FIRST - _LAST
                    order = torch.argsort(-middle, stable=True)[:left].sort().values.cuda() + _FIRST
                    mine = torch.cat((mine[:_FIRST], order, mine[n - _LAST:]))
                lists[i, g, :mine.numel()] = mine.to(torch.int32)
            K = state["k_pages"][held[mine], g].double()
            V = state["v_pages"][held[mine], g].double()
            see = (mine[:, None] * page + torch.arange(page, device="cuda")).flatten() < seen[i]
            K, V = K.flatten(0, 1)[see], V.flatten(0, 1)[see]
            logits = torch.einsum("hd,ld->hl", q, K) * state["scale"]
            lse[i, g * group:(g + 1) * group] = torch.logsumexp(logits, 1)
            out[i, g * group:(g + 1) * group] = torch.softmax(logits, 1) @ V
    return (out, lse) if lists is None else (lists, out, lse)

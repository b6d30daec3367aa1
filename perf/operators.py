"""The paged 4-bit cache and the decode over it, as a serving program calls them.

Kinds of case:
  assign  dma_cache_assign: pages, block tables and slots for a step's new tokens, then the step taken back
  append  dma_cache_append: rows of K and V into the cache (scores, 4-bit codes), then dma_cache_read of the same slots
  decode  dma_cache_decode: new rows of every request against its cache
  serve   a whole step: assign, append, decode, and the step taken back (the last draft tokens rejected)

The cache is one uint8 tensor [n_pages, page bytes].  A page of `ps` tokens holds, in this order, per kv-head and token d / 2
bytes of K codes and d / 2 of V codes; per kv-head and token d / 32 scale bytes of K and d / 32 of V; per q-head `ps` scores
(fp32); and zeros up to a multiple of 256 bytes.  A code is an OCP e2m1 value (low nibble first), a scale byte b stands for
2^(b - 127) over 32 channels (255: not a number).  The free list is int32: [0] the number of free pages, [4 ...] a stack of them.
"""
import math
import random

import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
FREE_HEADER = 4


def _case(kind, reqs, tokens, cut, H_q, H_kv, d, k, ps, rows=1, dtype="bf16", given=False):
    return dict(kind=kind, reqs=reqs, tokens=tokens, cut=cut, H_q=H_q, H_kv=H_kv, d=d, k=k, ps=ps, rows=rows,
                dtype=dtype, given=given)


def listed():
    """reqs requests hold `tokens` cached tokens in all, cut as `cut` says (-1: equal).  rows: new rows a request, or, for
    assign, 0 = a mixed step (prompts, single tokens, requests that end); for append the rows of the call."""
    cases = {
        # a decoding step of a full batch: one token each, pages of 64
        "assign_step": _case("assign", 256, 256 * 1500, 3, 32, 8, 128, 2048, 64),
        # a mixed step of a large batch with small pages: prompts arrive, requests end
        "assign_mixed": _case("assign", 777, 900001, 5, 32, 8, 128, 2048, 16, rows=0),
        # one user's newest token into the cache
        "append_token": _case("append", 1, 1, -1, 32, 8, 128, 2048, 64),
        # a step of a batch with narrow heads and scores from elsewhere (the cross-head ones)
        "append_batch_given": _case("append", 333, 333, -1, 16, 16, 64, 512, 16, given=True),
        # the headline prompt, and wide heads in fp32
        "append_prompt_64k": _case("append", 1, 65536, -1, 32, 8, 128, 2048, 64),
        "append_d256_f32": _case("append", 1, 5003, -1, 16, 4, 256, 2048, 128, dtype="f32"),
        # the next token of a prompt shorter than the window
        "decode_prompt_1k": _case("decode", 1, 1019, -1, 32, 8, 128, 2048, 64),
        # one user's next token against a long cache
        "decode_64k": _case("decode", 1, 65536, -1, 32, 8, 128, 2048, 64),
        # a serving batch of mixed lengths
        "decode_batch": _case("decode", 24, 131072, 11, 32, 8, 128, 2048, 64),
        # drafts of five rows a request, narrow heads, small window and pages
        "decode_draft_d64": _case("decode", 9, 30011, 7, 16, 16, 64, 512, 16, rows=5),
        # wide heads, fp32 queries
        "decode_d256_f32": _case("decode", 3, 16384, 2, 16, 4, 256, 2048, 128, dtype="f32"),
        # a whole step of a batch, two rows a request
        "serve_batch": _case("serve", 16, 65537, 9, 32, 8, 128, 1024, 32, rows=2),
    }
    return [dict(name=name, **case) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["assign", "append", "append", "decode", "decode", "decode", "serve"])
        d = rng.choice([64, 128, 128, 256])
        H_q, H_kv = rng.choice([(2, 2), (8, 2), (8, 1), (16, 4), (16, 16), (32, 8)])
        ps, k = rng.choice([16, 32, 64, 128, 256]), _log_int(rng, 64, 4096)
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        cut, rows, given = rng.randint(0, 9999), 1, False
        if kind == "assign":
            reqs = _log_int(rng, 1, 1500)
            tokens, rows = reqs * _log_int(rng, 8, 1200), rng.choice([0, 1, 4])
        elif kind == "append":
            reqs, tokens, given = 1, _log_int(rng, 1, 65536), rng.random() < 0.25
        else:
            reqs, rows = _log_int(rng, 1, 24), rng.choice([1, 1, 2, 5])
            tokens = reqs * _log_int(rng, 300, 65536)
        case = _case(kind, reqs, tokens, cut, H_q, H_kv, d, k, ps, rows, dtype, given)
        if _most(case) <= 1.0:
            return case


def _most(case):
    """The case's cost relative to what the largest listed ones cost (gathered values, ranked scores, cached bytes)."""
    if case["kind"] == "assign":
        return case["tokens"] / 900001
    if case["kind"] == "append":
        return case["tokens"] * case["H_kv"] * case["d"] * (2 if case["dtype"] == "f32" else 1) / (65536 * 1024)
    longest = max(_lengths(case))
    n_rows = case["reqs"] * case["rows"]
    gathered = n_rows * case["H_q"] * min(case["k"], longest) * case["d"] / (24 * 32 * 2048 * 128)
    return max(gathered, n_rows * case["H_q"] * longest / (24 * 32 * 10240), case["tokens"] / 131072)


def _lengths(case):
    n, total = case["reqs"], case["tokens"]
    if case["cut"] < 0:
        weights = [1.0] * n
    else:
        state, weights = case["cut"] * 2 + 1, []
        for _ in range(n):  # a small congruential generator: the cut belongs to the case, not to the inputs' seed
            state = (state * 1103515245 + 12345) % (1 << 31)
            weights.append(0.12 + 1.76 * state / (1 << 31))
    whole, ends, run = sum(weights), [], 0.0
    for w in weights:
        run += w
        ends.append(int(round(total * run / whole)))
    ends[-1] = total
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def _changes(case):
    """New tokens of every request (below 0: given back) in the step of an assign or serve case."""
    lengths = _lengths(case)
    if case["rows"]:
        return [case["rows"]] * len(lengths)
    rng, out = random.Random(case["cut"]), []
    for n in lengths:
        what = rng.random()
        if what < 0.15:
            out.append(-n)                       # the request ends
        elif what < 0.2:
            out.append(-min(n, rng.randint(1, 4)))  # rejected drafts
        elif what < 0.3:
            out.append(_log_int(rng, 1, 2000))   # a prompt, or a piece of one
        elif what < 0.9:
            out.append(1)
        else:
            out.append(0)
    return out


def _sizes(case):
    """(rows of a call, pages of a request at most, pages of the pool)"""
    lengths, ps = _lengths(case), case["ps"]
    if case["kind"] == "append":
        pages = case["tokens"] // ps + 2
        return case["tokens"], pages, pages + 3
    if case["kind"] == "decode":
        return case["reqs"] * case["rows"], -(-max(lengths) // ps), sum(-(-n // ps) for n in lengths) + 5
    changes = _changes(case)
    rows = max(sum(c for c in changes if c > 0), sum(-c for c in changes if c < 0))
    after = [n + max(c, 0) for n, c in zip(lengths, changes)]
    return rows, -(-max(after) // ps) + 1, sum(-(-n // ps) for n in after) + 7


def _offsets(case):
    """Byte offsets in a page: of the scales, of the scores, and its size."""
    scales = case["H_kv"] * case["ps"] * case["d"]
    scores = scales + case["H_kv"] * case["ps"] * case["d"] // 16
    return scales, scores, -(-(scores + 4 * case["H_q"] * case["ps"]) // 256) * 256


def _views(case, pages):
    """codes [pages, H_kv, ps, K / V, d / 2], scale bytes [pages, H_kv, ps, K / V, d / 32], scores [pages, H_q, ps]"""
    n, ps, d, H_q, H_kv = pages.shape[0], case["ps"], case["d"], case["H_q"], case["H_kv"]
    at_scales, at_scores, _ = _offsets(case)
    codes = pages[:, :at_scales].unflatten(1, (H_kv, ps, 2, d // 2))
    scales = pages[:, at_scales:at_scores].unflatten(1, (H_kv, ps, 2, d // 32))
    return codes, scales, pages[:, at_scores:at_scores + 4 * H_q * ps].view(torch.float32).view(n, H_q, ps)


def work(case):
    T, H_q, H_kv, d = (case[x] for x in ("tokens", "H_q", "H_kv", "d"))
    size = 4 if case["dtype"] == "f32" else 2
    cached = H_kv * (d + d // 16) + 4 * H_q          # bytes of a token in the cache
    n_rows = _sizes(case)[0]

    def assign():
        # in: changes and lengths; out: lengths, row offsets, status; a slot, request and length a row; a table entry and a list entry a page
        changed = sum(-(-abs(c) // case["ps"]) for c in _changes(case))
        return 20 * case["reqs"] + 12 * n_rows + 8 * changed

    def append(rows):
        return rows * (2 * H_kv * d * size + cached + 4) + 4 * H_q * (d + 1), 2.0 * rows * H_q * d

    def decode():
        total, flops = 0.0, 0.0
        for n in _lengths(case):
            kept, G = min(case["k"], n), H_q // H_kv
            rows_read = n * (1.0 - (1.0 - kept / n) ** G) if n else 0.0  # union of the group's kept sets, expected
            total += rows_read * H_kv * (d + d // 16) + 4 * H_q * n + case["rows"] * H_q * (2 * d * size + 4 * kept + 4)
            flops += 4.0 * case["rows"] * H_q * kept * d
        return total, flops

    if case["kind"] == "assign":
        return {"bytes": 2 * assign(), "flops": 0}
    if case["kind"] == "append":
        b, f = append(T)
        if case["given"]:
            b, f = b + 4 * H_q * T, 0
        return {"bytes": b + T * (cached + 2 * H_kv * d * size + 4 * H_q), "flops": f}
    b, f = decode()
    if case["kind"] == "decode":
        return {"bytes": b, "flops": f}
    more = append(n_rows)
    return {"bytes": 2 * assign() + more[0] + b, "flops": more[1] + f}


# ---------------------------------------------------------------- the plain forms
def _quantise(x):
    """x [..., d] -> (codes [..., d / 2], scale bytes [..., d / 32]): every 32 channels share the power of two at which the
    largest of them rounds to at most 6."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    byte = (((top.view(torch.int32) + 0x200000) >> 23) - 2).clamp(2, 252)  # (a mantissa of 1.75 or more carries)
    byte = torch.where(torch.isfinite(top), byte, torch.full_like(byte, 255))
    a = x.abs() * ((254 - byte.clamp(max=252)) << 23).view(torch.float32)[..., None]
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code | (torch.signbit(x).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte.to(torch.uint8)


def _values(codes, scales):
    """Codes [..., d / 2] and scale bytes [..., d / 32] -> fp32 [..., d]."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    nibbles = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    step = (scales.int() << 23).view(torch.float32)
    step = torch.where(scales == 255, torch.full_like(step, float("nan")), step)
    return (table[nibbles.int()].unflatten(-1, (-1, 32)) * step[..., None]).flatten(-2)


def _assign(state, changes):
    case, lens, table, free = state["case"], state["lens"], state["table"], state["free"]
    ps, n_rows, max_pages = case["ps"], state["n_rows"], table.shape[1]
    old, change = lens.long(), changes.long()
    grow, shrink = change.clamp(min=0), torch.minimum((-change).clamp(min=0), old)
    ends = grow.cumsum(0)
    pages, less = (old + ps - 1) // ps, (old - shrink + ps - 1) // ps
    # the pages given back go on top of the stack, request by request
    place = torch.arange(max_pages, device=lens.device)
    back = (place >= less[:, None]) & (place < pages[:, None])
    freed = pages - less
    to = free[0] + (freed.cumsum(0) - freed)[:, None] + place - less[:, None]
    stack = torch.cat((free[FREE_HEADER:], free[:1]))
    stack[torch.where(back, to, stack.numel() - 1)] = table
    table = torch.where(back, -1, table)
    have = free[0] + freed.sum()
    # new pages are taken from its top, request by request
    want = (old + grow + ps - 1) // ps
    need = torch.where(change > 0, want - pages, 0)
    status = torch.where(want > max_pages, 2, torch.where((ends > n_rows) & (grow > 0), 3, 0))
    need = torch.where(status == 0, need, 0)
    upto = need.cumsum(0)
    status = torch.where((need > 0) & (upto > have), 1, status)
    served = status == 0
    need = torch.where(served, need, 0)
    new = (place >= pages[:, None]) & (place < (pages + need)[:, None])
    at = have - 1 - ((upto - need)[:, None] + place - pages[:, None])
    table = torch.where(new, stack[at.clamp(0, stack.numel() - 1)], table).int()
    lens.copy_(torch.where(served, old - shrink + grow, old))
    state["table"].copy_(table)
    free[FREE_HEADER:] = stack[:-1]
    free[0] = have - need.sum()
    row = torch.arange(n_rows, device=lens.device)
    req = torch.searchsorted(ends, row, right=True)
    inside = req < case["reqs"]
    req = req.clamp(max=case["reqs"] - 1)
    inside &= served[req]
    pos = old[req] + row - (ends - grow)[req]
    slot = table[req, (pos // ps).clamp(0, max_pages - 1)] * ps + pos % ps
    cu = torch.cat((ends.new_zeros(1), ends)).clamp(max=n_rows).int()
    return (cu, torch.where(inside, req, -1).int(), torch.where(inside, pos + 1, 0).int(),
            torch.where(inside, slot, -1).int(), status.int())


def _append(state, K, V, slots):
    case, ps = state["case"], state["case"]["ps"]
    codes, scales, scores = _views(case, state["pages"])
    if state["z"] is None:
        G = case["H_q"] // case["H_kv"]
        x = (V.float().repeat_interleave(G, 1) * state["W"]).sum(-1)
        z = torch.exp(state["A"] * torch.nn.functional.softplus(x, threshold=80))
    else:
        z = state["z"].t()
    page, off = slots.long() // ps, slots.long() % ps
    c, s = _quantise(torch.stack((K, V), 2))
    codes[page, :, off] = c
    scales[page, :, off] = s
    scores[page, :, off] = z


def _read(state, slots):
    case, ps = state["case"], state["case"]["ps"]
    codes, scales, scores = _views(case, state["pages"])
    page, off = slots.long() // ps, slots.long() % ps
    both = _values(codes[page, :, off], scales[page, :, off]).to(state["type"])
    return both[:, :, 0].contiguous(), both[:, :, 1].contiguous(), scores[page, :, off].t().contiguous()


def _decode(state, q, row_req, row_len):
    case, ps, d = state["case"], state["case"]["ps"], state["case"]["d"]
    codes, scales, scores = _views(case, state["pages"])
    n, H_q, G = state["longest"], case["H_q"], case["H_q"] // case["H_kv"]
    kcap = state["kept"].shape[2]
    place = torch.arange(n, device=q.device)
    page, off = state["table"][row_req.long()][:, place // ps].long().clamp(min=0), place % ps
    inside = place < row_len[:, None]
    z = torch.where(inside[..., None], scores[page, :, off], float("-inf")).transpose(1, 2)
    # the window's best keys, ties to the earlier one, in order of position
    take = min(kcap, n)
    rank = torch.sort(z, dim=-1, descending=True, stable=True).indices[..., :take]
    kept = torch.where(torch.arange(take, device=q.device) < row_len[:, None, None], rank, n).sort(-1).values
    inside, kept = kept < n, kept.clamp(max=n - 1)
    row = torch.arange(q.shape[0], device=q.device)[:, None, None]
    page, off, head = page[row, kept], kept % ps, torch.arange(H_q, device=q.device)[:, None]
    both = _values(codes[page, head // G, off], scales[page, head // G, off])  # [rows, H_q, window, K / V, d]
    s = (both[..., 0, :] * q.float()[:, :, None]).sum(-1) / math.sqrt(d) + z.gather(2, kept)
    s = torch.where(inside, s, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - top)
    total = p.sum(-1)
    o = (p[..., None] * both[..., 1, :]).sum(2) / total[..., None]
    slots = torch.where(inside, page * ps + off, -1).int()
    full = torch.full((q.shape[0], H_q, kcap), -1, dtype=torch.int32, device=q.device)
    full[..., :take] = slots
    return o.to(state["type"]), (top[..., 0] + total.log()).t().contiguous(), full


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    H_q, H_kv, d, ps, reqs = (case[x] for x in ("H_q", "H_kv", "d", "ps", "reqs"))
    lengths, (n_rows, max_pages, n_pages) = _lengths(case), _sizes(case)
    kind, real = case["kind"], torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    order = torch.randperm(n_pages, generator=gen, device=dev).int()   # a pool long in use: pages in no order
    state = dict(case=case, n_rows=n_rows, type=real, longest=max(lengths), order=order)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=dev)
    if kind != "append":
        # the requests' tables, the stack of the pages that are left
        lens = torch.tensor(lengths, device=dev)
        pages = (lens + ps - 1) // ps
        before, place = pages.cumsum(0) - pages, torch.arange(max_pages, device=dev)
        table = torch.where(place < pages[:, None], order[(before[:, None] + place).clamp(max=n_pages - 1)], -1)
        taken = sum(-(-n // ps) for n in lengths)
        free = torch.zeros(FREE_HEADER + n_pages, dtype=torch.int32, device=dev)
        free[0] = n_pages - taken
        free[FREE_HEADER:FREE_HEADER + n_pages - taken] = order[taken:]
        state.update(lens=lens.int(), table=table.int(), free=free)
    if kind in ("assign", "serve"):
        changes = torch.tensor(_changes(case), dtype=torch.int32, device=dev)
        state.update(changes=changes, undo=-changes,
                     rows=[dict(cu=ints(reqs + 1), req=ints(n_rows), len=ints(n_rows), slots=ints(n_rows), status=ints(reqs))
                           for _ in range(2)])
    if kind == "assign":
        return state
    state["pages"] = torch.zeros((n_pages, _offsets(case)[2]), dtype=torch.uint8, device=dev)
    if kind != "decode":
        # q, K and V of the new rows, side by side as a projection leaves them
        state["qkv"] = torch.randn((n_rows, H_q + 2 * H_kv, d), generator=gen, device=dev, dtype=real)
        state["W"] = torch.randn((H_q, d), generator=gen, device=dev) / math.sqrt(d)
        state["A"] = -(0.5 + 1.5 * torch.rand(H_q, generator=gen, device=dev))
        state["z"] = torch.rand((H_q, n_rows), generator=gen, device=dev) if case["given"] else None
    if kind == "append":
        at = torch.arange(n_rows, device=dev) + (0 if n_rows == 1 else 5)   # the call starts inside a page
        state["slots"] = order[at // ps] * ps + (at % ps).int()
        state["out"] = (torch.zeros((n_rows, H_kv, d), dtype=real, device=dev), torch.zeros((n_rows, H_kv, d), dtype=real, device=dev),
                        torch.zeros((H_q, n_rows), device=dev))
        return state
    # the cached tokens: K, V ~ N(0, 1) in 4 bits, scores as exp(A softplus(x)) with x ~ N(0, 1)
    codes, scales, scores = _views(case, state["pages"])
    gate = -(0.5 + 1.5 * torch.rand((H_q, 1), generator=gen, device=dev))
    step = max(1, (1 << 25) // (H_kv * ps * 2 * d))
    for i in range(0, n_pages, step):
        m = min(step, n_pages - i)
        codes[i:i + m], scales[i:i + m] = _quantise(torch.randn((m, H_kv, ps, 2, d), generator=gen, device=dev))
        scores[i:i + m] = torch.exp(gate * torch.nn.functional.softplus(torch.randn((m, H_q, ps), generator=gen, device=dev)))
    if kind == "decode":
        state["qkv"] = torch.randn((n_rows, H_q + 2 * H_kv, d), generator=gen, device=dev, dtype=real)
        r = case["rows"]
        req = torch.arange(reqs, device=dev).repeat_interleave(r)
        back = torch.arange(r - 1, -1, -1, device=dev).repeat(reqs)
        state["rows"] = [dict(req=req.int(), len=(state["lens"][req] - back).clamp(min=1).int())]
    else:
        state["longest"] = max(n + c for n, c in zip(lengths, _changes(case)))
    state["kept"] = ints(n_rows, H_q, min(case["k"], max_pages * ps))
    state["o"] = torch.zeros((n_rows, H_q, d), dtype=real, device=dev)
    state["lse"] = torch.zeros((H_q, n_rows), device=dev)
    return state


# ---------------------------------------------------------------- one pass
def _setup(state):
    """What a serving program makes once: the binding, the cache's shape and the workspace of a decode."""
    from paper_2508_02124_amd import binding as B
    case, (n_rows, max_pages, n_pages) = state["case"], _sizes(state["case"])
    shape = B.make_cache_shape(case["reqs"], n_pages, max_pages, case["ps"], case["H_q"], case["H_kv"], case["d"],
                               dtype=B.DMA_F32 if case["dtype"] == "f32" else B.DMA_BF16)
    ws_bytes = 0 if "kept" not in state else B.dma_cache_decode_bytes(shape, n_rows, case["k"])
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device="cuda")
    state["own"] = (B, shape, ws, ws_bytes)
    return state["own"]


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    H_q, H_kv = case["H_q"], case["H_kv"]
    if kind != "assign":
        q, K, V = state["qkv"].split((H_q, H_kv, H_kv), 1)
    if not own:
        if kind == "append":
            _append(state, K, V, state["slots"])
            return _read(state, state["slots"])
        if kind == "decode":
            return _decode(state, q, state["rows"][0]["req"], state["rows"][0]["len"])
        first = _assign(state, state["changes"])
        if kind == "serve":
            _append(state, K, V, first[3])
            out = _decode(state, q, first[1], first[2])
        second = _assign(state, state["undo"])
        return (first, second, state["lens"], state["table"], state["free"]) if kind == "assign" else (*out, *first)
    B, shape, ws, ws_bytes = state.get("own") or _setup(state)
    n_rows, pitch = state["n_rows"], (H_q + 2 * H_kv) * case["d"]

    def assign(changes, rows):
        B.dma_cache_assign(shape, n_rows, changes, state["lens"], state["table"], state["free"], rows["cu"], rows["req"],
                           rows["len"], rows["slots"], rows["status"])
        return tuple(rows.values())

    def append(slots):
        scores = (state["W"], state["A"], None) if state["z"] is None else (None, None, state["z"])
        B.dma_cache_append(shape, n_rows, K, pitch, V, pitch, *scores, slots, state["pages"])

    def decode(rows):
        B.dma_cache_decode(shape, n_rows, case["k"], 0.0, q, pitch, state["pages"], state["table"], rows["req"],
                           rows["len"], state["o"], state["lse"], state["kept"], ws, ws_bytes)
        return state["o"], state["lse"], state["kept"]

    if kind == "append":
        append(state["slots"])
        B.dma_cache_read(shape, n_rows, state["slots"], state["pages"], *state["out"])
        return state["out"]
    if kind == "decode":
        return decode(state["rows"][0])
    first = assign(state["changes"], state["rows"][0])
    if kind == "serve":
        append(first[3])
        out = decode(state["rows"][0])
    second = assign(state["undo"], state["rows"][1])
    return (first, second, state["lens"], state["table"], state["free"]) if kind == "assign" else (*out, *first)


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _nearest(x):
    """The values in 4 bits that stand for x [..., 32] float64: the nearest of the sixteen, ties to the even code."""
    grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    top = x.abs().amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(top)                       # top = mantissa 2^exponent, mantissa in [0.5, 1)
    e = (exponent - 3 + (mantissa >= 0.875)).clamp(-125, 125).double()
    a = x.abs() / torch.exp2(e)
    hi = torch.searchsorted(grid, a.contiguous()).clamp(1, 7)
    down, up = a - grid[hi - 1], grid[hi] - a
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return torch.copysign(grid[code], x) * torch.exp2(e)


def _rounded(x):
    return torch.cat([_nearest(part.double().unflatten(-1, (-1, 32))).flatten(-2) for part in x.split(8192)])


def _scores(V, W, A):
    G, out = W.shape[0] // V.shape[1], []
    for h in range(W.shape[0]):
        x = V[:, h // G].double() @ W[h].double()
        out.append(torch.exp(A[h].double() * (torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs())))))
    return torch.stack(out)


def exact(case, seed):
    state = prepare(case, seed)
    kind, H_q, H_kv, d, ps = case["kind"], case["H_q"], case["H_kv"], case["d"], case["ps"]
    if kind == "assign":
        return None
    if kind != "decode":
        q, K, V = state["qkv"].split((H_q, H_kv, H_kv), 1)
        z = state["z"].double() if case["given"] else _scores(V, state["W"], state["A"])
        K, V = _rounded(K), _rounded(V)
        if kind == "append":
            return K, V, z
    q, lengths, r = state["qkv"][:, :H_q].double(), _lengths(case), case["rows"]
    codes, scales, scores = _views(case, state["pages"])
    sign = torch.tensor([1.0] * 8 + [-1.0] * 8, dtype=torch.float64, device=q.device)
    grid = torch.tensor(E2M1 * 2, dtype=torch.float64, device=q.device) * sign
    o = torch.zeros((state["n_rows"], H_q, d), dtype=torch.float64, device=q.device)
    lse = torch.zeros((H_q, state["n_rows"]), dtype=torch.float64, device=q.device)
    for b, n in enumerate(lengths):
        pages = state["table"][b, :-(-n // ps)].long()
        zb = scores[pages].transpose(0, 1).reshape(H_q, -1)[:, :n].double()
        cached = codes[pages].transpose(0, 1).reshape(H_kv, -1, 2, d // 2)[:, :n]
        power = torch.exp2(scales[pages].transpose(0, 1).reshape(H_kv, -1, 2, d // 32)[:, :n].double() - 127)
        for row in range(b * r, b * r + r):
            m = max(1, n - r + 1 + row - b * r) if kind == "decode" else n + 1 + row - b * r
            zr = zb
            if kind == "serve":
                zr = torch.cat((zb, z[:, b * r:row + 1].float().double()), 1)
            for h in range(H_q):
                g = h // (H_q // H_kv)
                best = torch.argsort(-zr[h, :m], stable=True)[:case["k"]]
                old = best[best < n]
                both = torch.stack((cached[g, old] & 15, cached[g, old] >> 4), -1).flatten(-2).long()
                both = (grid[both].unflatten(-1, (-1, 32)) * power[g, old][..., None]).flatten(-2)
                if kind == "serve":
                    new = best[best >= n] - n + b * r
                    both = torch.cat((both, torch.stack((K[new, g], V[new, g]), 1)))
                    best = torch.cat((old, best[best >= n]))
                s = both[:, 0] @ q[row, h] / math.sqrt(d) + zr[h, best]
                lse[h, row] = torch.logsumexp(s, 0)
                o[row, h] = torch.softmax(s, 0) @ both[:, 1]
    return (o, lse, None) if kind == "decode" else (o, lse, None, None, None, None, None, None)

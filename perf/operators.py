"""Performance cases of the operators on a paged key-value cache: what a serving program calls between and inside decode steps.

    listed(), draw(rng)   the cases, and more of the same ranges
    prepare(case, seed)   inputs, page pools and page tables on the GPU, as a program has them before the call
    run(state)            one pass through an operator; its outputs, and the pools it wrote
    work(case)            bytes and flops a pass cannot do without
    exact(case, seed)     the same outputs in float64, one sequence or token after the other

With `own` false, run() computes the operators by elementary torch operations, in 32 bits; with `own` true it calls
`binding.PagedCache`.

The pools: a page holds `page_rows` rows of every key-value head.  Keys [layer][page][head][row][dim]; values
[layer][page][head][row / R][dim][row % R] with R rows in 16 bytes (8 of fp16, 4 of fp32).  A slot is page * page_rows + row.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
ROPE_BASE = 10000.0
HALF_MAX = 65504.0        # an fp16 cache holds values clamped to this


def _reserve(name, mix, B, tokens, page_rows):
    return {"name": name, "op": "reserve", "mix": mix, "B": B, "tokens": tokens, "page_rows": page_rows}


def _append(name, layers, tokens, heads, hd, src, kv, page_rows, rope):
    return {"name": name, "op": "append", "layers": layers, "tokens": tokens, "heads": heads, "hd": hd, "src": src, "kv": kv,
            "page_rows": page_rows, "rope": rope}


def _fill(name, layers, dropped, B, heads, hd, kv, page_rows):
    return {"name": name, "op": "fill", "layers": layers, "dropped": dropped, "B": B, "heads": heads, "hd": hd, "kv": kv, "page_rows": page_rows}


def _attend(name, B, rows, spread, heads, group, hd, act, kv, page_rows, new):
    return {"name": name, "op": "attend", "B": B, "rows": rows, "spread": spread, "heads": heads, "group": group, "hd": hd, "act": act,
            "kv": kv, "page_rows": page_rows, "new": new}


def listed():
    return [
        # a step of a few users: one new row each, now and then a new page
        _reserve("reserve_step_b8", "step", 8, 8, 16),
        # a busy server: most requests decode, some end, new prompts come in, some places are idle
        _reserve("reserve_mixed_b256", "mixed", 256, 20000, 16),
        # a batch of long prompts (the batch-32 configuration)
        _reserve("reserve_prompts_b32", "prompts", 32, 65536, 32),
        # a prompt's keys and values of one block, rotated and rounded on their way into pages (7B widths)
        _append("append_prompt_7b", 1, 512, 32, 128, "f32", "f16", 16, True),
        # a piece of a prompt of odd length from a bf16 model, head_dim 64
        _append("append_piece_odd", 1, 77, 8, 64, "bf16", "f16", 16, True),
        # the rows of a whole prompt pass moved into pages, several blocks in one call (70B widths, fp32 cache)
        _append("append_blocks_70b", 8, 1024, 8, 128, "f32", "f32", 64, False),
        # the blocks that a step dropped get the row of the last block that ran: one user
        _fill("fill_7b_b1", 32, 15, 1, 32, 128, "f16", 16),
        # the same of a batch, deep model, fp32 cache
        _fill("fill_70b_b8", 80, 40, 8, 8, 128, "f32", 64),
        # one user's step, nothing but latency (7B widths)
        _attend("attend_7b_b1", 1, 640, "equal", 32, 1, 128, "f32", "f16", 16, True),
        # grouped queries over an fp32 cache (70B widths, batch 8)
        _attend("attend_70b_b8", 8, 1152, "equal", 8, 8, 128, "f32", "f32", 64, True),
        # requests of all ages, one to 32768 rows, some places empty; a bf16 model's queries, rows written before
        _attend("attend_ragged_b48", 48, 32768, "log", 8, 4, 128, "bf16", "f16", 16, False),
        # the full batch with long contexts: the largest stream of cache rows (7B widths, batch 32)
        _attend("attend_7b_b32", 32, 2304, "equal", 32, 1, 128, "f32", "f16", 32, True),
    ]


def _between(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    case = _drawn(rng)
    del case["name"]
    return case


def _drawn(rng):
    op = rng.choice(["reserve", "append", "fill", "attend", "attend"])
    page_rows = rng.choice([16, 16, 32, 64, 128])
    hd = rng.choice([64, 128, 128])
    kv = rng.choice(["f16", "f16", "f32"])
    if op == "reserve":
        mix = rng.choice(["step", "mixed", "prompts"])
        B = _between(rng, 1, 512 if mix != "prompts" else 48)
        return _reserve("", mix, B, B if mix == "step" else _between(rng, B, 60000), page_rows)
    if op == "append":
        heads, layers = rng.choice([1, 2, 4, 5, 8, 32]), rng.choice([1, 1, 2, 5])
        most = min(6000, (1 << 26) // (heads * hd * layers))
        return _append("", layers, _between(rng, 1, most), heads, hd, rng.choice(["f32", "bf16", "f16"]), kv, page_rows, rng.random() < 0.5)
    if op == "fill":
        layers = rng.choice([4, 32, 40, 80])
        heads = rng.choice([2, 4, 8, 40 if layers == 40 else 32])
        most = min(32, max(1, (1 << 29) // (layers * heads * page_rows * hd)))
        return _fill("", layers, rng.randint(1, layers - 1), _between(rng, 1, most), heads, hd, kv, page_rows)
    B = _between(rng, 1, 96)
    group = rng.choice([1, 1, 2, 3, 4, 5, 7, 8, 16, 20])
    heads = rng.choice([1, 2, 4, 8, 32] if group <= 4 else [1, 2, 8])
    most = max(16, min(32768, (1 << 30) // (B * heads * hd * 2 * BYTES[kv] * max(1, group // 4))))
    return _attend("", B, _between(rng, 1, most), rng.choice(["equal", "log"]), heads, group, hd, rng.choice(["f32", "bf16", "f16"]), kv,
                   page_rows, rng.random() < 0.5)


def _unit_rows(kv):
    return 16 // BYTES[kv]


def _lengths(case):
    """Rows of every sequence: all alike, or from 1 to case["rows"] evenly over the logarithm in a fixed mixed order, every 16th of 16 or more none."""
    B, rows = case["B"], case["rows"]
    if case["spread"] == "equal":
        return [rows] * B
    n = [max(1, round(rows ** ((i + 1) / B))) for i in range(B)]
    step = next(s for s in (37, 41, 43, 47, 53, 59, 61, 67) if math.gcd(s, B) == 1)
    return [0 if B >= 16 and b % 16 == 5 else n[b * step % B] for b in range(B)]


def _pages(rows, page_rows):
    return -(-rows // page_rows)


def _requests(case):
    """(rows, added) of every sequence of a reserve case, from the case alone."""
    B, tokens, pr = case["B"], case["tokens"], case["page_rows"]
    rng = np.random.RandomState(B * 131 + tokens)
    if case["mix"] == "step":
        return rng.randint(1, 2000, B), np.ones(B, np.int64)
    if case["mix"] == "prompts":
        cut = np.sort(rng.choice(np.arange(1, tokens), B - 1, replace=False)) if tokens > B else np.arange(1, B)
        return np.zeros(B, np.int64), np.diff(np.concatenate([[0], cut, [max(tokens, B)]]))
    rows, added = rng.randint(1, 2000, B), np.ones(B, np.int64)
    kind = rng.randint(0, 16, B)
    added[kind == 0] = -1                                  # ended
    added[kind == 1] = 0                                   # idle
    rows[kind == 2] = 0                                    # a new prompt
    n_new = int((kind == 2).sum())
    if n_new:
        added[kind == 2] = max(1, (tokens - B) // n_new) if tokens > B else 1
    return rows, added


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _pools(g, layers, n_pages, heads, page_rows, hd, kv):
    R = _unit_rows(kv)
    k = torch.empty(layers, n_pages, heads, page_rows, hd, dtype=TYPES[kv], device=DEVICE).normal_(generator=g)
    v = torch.empty(layers, n_pages, heads, page_rows // R, hd, R, dtype=TYPES[kv], device=DEVICE).normal_(generator=g)
    return k, v


def _angles(positions, hd):
    """(cos, sin) of the rotary angles of the given positions: [n][hd / 2][2], from 64 bits."""
    inv = ROPE_BASE ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64, device=DEVICE) / hd)
    a = positions.double()[:, None] * inv
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def prepare(case, seed):
    g = _generator(seed)
    s = SimpleNamespace(case=case)
    pr, op = case["page_rows"], case["op"]
    ints = dict(dtype=torch.int32, device=DEVICE)
    if op == "reserve":
        rows, added = _requests(case)
        B = case["B"]
        held, asked = int(_pages(rows, pr).sum()), int(_pages(rows + np.maximum(added, 0), pr).sum())
        s.n_pages = asked + 16
        s.max_pages = int(_pages(rows + np.maximum(added, 0), pr).max()) + 4
        order = torch.randperm(s.n_pages, generator=g, device=DEVICE).int()
        s.rows, s.added = torch.tensor(rows, **ints), torch.tensor(added, **ints)
        s.tables = torch.full((B, s.max_pages), -1, **ints)
        at = torch.arange(s.max_pages, device=DEVICE)[None] < ((s.rows + pr - 1) // pr)[:, None]
        s.tables[at] = order[:held]
        s.free_pages = torch.full((s.n_pages,), -1, **ints)
        s.free_pages[: s.n_pages - held] = order[held:]
        s.n_free = torch.tensor([s.n_pages - held, 0], **ints)
        s.rows_out, s.n_free_out = torch.zeros_like(s.rows), torch.zeros_like(s.n_free)
        s.max_tokens = max(1, int(np.maximum(added, 0).sum()))
        s.starts, s.slots = torch.empty(B + 1, **ints), torch.empty(s.max_tokens, **ints)
        s.positions = torch.empty(s.max_tokens, **ints)
        if own:
            from paper_2503_08524_amd import binding
            # the pools hold no rows here: this operator reads and writes page numbers only
            s.cache = binding.PagedCache(1, 1, 64, s.n_pages, pr, max_batch=B, max_pages=s.max_pages, tables=s.tables, rows=s.rows,
                                         free_pages=s.free_pages, n_free=s.n_free, device=DEVICE)
        return s
    kv, hd, heads = case["kv"], case["hd"], case["heads"]
    layers, group = case.get("layers", 1), case.get("group", 1)
    if op == "attend":
        B = case["B"]
        n = _lengths(case)
        s.max_pages = max(1, _pages(max(n), pr))
        s.n_pages = sum(_pages(x, pr) for x in n) + 8
        s.rows = torch.tensor(n, **ints)
        s.tables = torch.full((B, s.max_pages), -1, **ints)
        at = torch.arange(s.max_pages, device=DEVICE)[None] < ((s.rows + pr - 1) // pr)[:, None]
        s.tables[at] = torch.randperm(s.n_pages, generator=g, device=DEVICE).int()[: int(at.sum())]
        s.k_pages, s.v_pages = _pools(g, 1, s.n_pages, heads, pr, hd, kv)
        act = dict(dtype=TYPES[case["act"]], device=DEVICE)
        s.q = torch.empty(B, heads * group, hd, **act).normal_(generator=g)
        s.k = s.v = s.rope_cs = None
        if case["new"]:
            s.k = torch.empty(B, heads, hd, **act).normal_(generator=g)
            s.v = torch.empty(B, heads, hd, **act).normal_(generator=g)
            s.rope_cs = _angles((s.rows - 1).clamp(min=0), hd)
        s.out = torch.empty_like(s.q)
    else:
        n = case["tokens"] if op == "append" else case["B"]
        s.n_pages = _pages(n + 5, pr) + 2 if op == "append" else n + 2
        order = torch.randperm(s.n_pages, generator=g, device=DEVICE).int()
        if op == "append":                                 # consecutive rows of one sequence that holds 5 already
            p = torch.arange(5, n + 5, device=DEVICE)
            s.slots = order[p // pr] * pr + (p % pr).int()
            s.k = torch.empty(layers, n, heads, hd, dtype=TYPES[case["src"]], device=DEVICE).normal_(generator=g)
            s.v = torch.empty(layers, n, heads, hd, dtype=TYPES[case["src"]], device=DEVICE).normal_(generator=g)
            s.rope_cs = _angles(p, hd) if case["rope"] else None
        else:                                              # the newest row of every sequence
            s.slots = order[:n] * pr + torch.randint(0, pr, (n,), generator=g, device=DEVICE).int()
        s.k_pages, s.v_pages = _pools(g, layers, s.n_pages, heads, pr, hd, kv)
    if own:
        from paper_2503_08524_amd import binding
        more = dict(tables=s.tables, rows=s.rows, max_batch=case["B"], max_pages=s.max_pages) if op == "attend" else dict(max_batch=1, max_pages=1)
        s.cache = binding.PagedCache(heads * group, heads, hd, s.n_pages, pr, kv_dtype=kv, n_layers=layers, k_pages=s.k_pages,
                                     v_pages=s.v_pages, device=DEVICE, **more)
    return s


def _window(case):
    """(source block, first dropped block) of a fill: the window begins at 0.6 of the depth, or where it still fits."""
    first = min(int(0.6 * case["layers"]), case["layers"] - case["dropped"])
    return (first - 1 if first > 0 else case["dropped"]), first


def run(s):
    case, op = s.case, s.case["op"]
    if own:
        if op == "reserve":
            s.cache.reserve(s.added, s.max_tokens, starts=s.starts, slots=s.slots, positions=s.positions, rows_out=s.rows_out, n_free_out=s.n_free_out)
            return {"starts": s.starts, "slots": s.slots, "positions": s.positions, "rows": s.rows_out, "n_free": s.n_free_out, "tables": s.tables}
        if op == "append":
            s.cache.append(0, s.slots, s.k, s.v, rope_cs=s.rope_cs)
            return {"k": s.k_pages, "v": s.v_pages}
        if op == "fill":
            src, first = _window(case)
            s.cache.fill(s.slots, src, first, case["dropped"])
            return {"k": s.k_pages, "v": s.v_pages}
        s.cache.attend(0, s.q, s.k, s.v, rope_cs=s.rope_cs, out=s.out)
        return {"out": s.out, "k": s.k_pages, "v": s.v_pages} if case["new"] else {"out": s.out}
    return _plain[op](s)


# ---------------- the plain forms ----------------

def _plain_reserve(s):
    pr = s.case["page_rows"]
    cap = s.max_pages * pr
    ended = s.added < 0
    held = ((s.rows + pr - 1) // pr).long()
    rows = torch.where(ended, 0, s.rows).long()
    # pages of ended sequences go on top of the stack, in order
    cols = torch.arange(s.max_pages, device=DEVICE)
    back = s.tables[ended[:, None] & (cols[None] < held[:, None])]
    n_free = int(s.n_free[0])
    s.free_pages[n_free: n_free + back.numel()] = back
    avail = n_free + back.numel()
    # what is asked, and what of it is granted
    asked = s.added.clamp(min=0).long()
    asked = torch.where(rows + asked <= cap, asked, 0)
    fits = asked.cumsum(0) <= s.max_tokens
    asked = torch.where(fits, asked, 0)
    need = (rows + asked + pr - 1) // pr - (rows + pr - 1) // pr
    upto = need.cumsum(0)
    granted = torch.where((need == 0) | (upto <= avail), asked, 0)
    need_granted = torch.where(granted > 0, need, 0)
    s.rows_out.copy_(rows + granted)
    s.n_free_out[0] = avail - need_granted.sum()
    s.n_free_out[1] = (need.sum() - avail).clamp(min=0)
    s.starts[0] = 0
    s.starts[1:] = granted.cumsum(0)
    # the k-th granted page is the k-th from the top
    first = (rows + pr - 1) // pr
    new = (cols[None] >= first[:, None]) & (cols[None] < (first + need_granted)[:, None])
    taken = int(need_granted.sum())
    s.tables[new] = s.free_pages[avail - taken: avail].flip(0)
    t = torch.arange(s.max_tokens, device=DEVICE)
    b = torch.searchsorted(s.starts[1:].contiguous().long(), t, right=True)
    live = b < s.added.numel()
    b = b.clamp(max=s.added.numel() - 1)
    p = rows[b] + t - s.starts[b]
    page = s.tables[b, (p // pr).clamp(max=s.max_pages - 1)]
    s.slots.copy_(torch.where(live, page * pr + p % pr, -1))
    s.positions.copy_(torch.where(live, p, -1))
    return {"starts": s.starts, "slots": s.slots, "positions": s.positions, "rows": s.rows_out, "n_free": s.n_free_out, "tables": s.tables}


def _rotated(x, cs):
    """x [..., n, heads, hd] turned by cs [n][hd / 2][2]: dims j and j + hd / 2 together."""
    half = x.shape[-1] // 2
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * n, a * n + b * c], -1)


def _held(x, kv):
    """As the cache holds it."""
    return x.clamp(-HALF_MAX, HALF_MAX).half() if kv == "f16" else x


def _put(s, slots, k, v):
    """k, v [layers][n][heads][hd] into the rows `slots` of the pools."""
    pr, R = s.case["page_rows"], _unit_rows(s.case["kv"])
    page, row = (slots // pr).long(), (slots % pr).long()
    s.k_pages[:, page, :, row] = _held(k, s.case["kv"]).transpose(0, 1)
    s.v_pages[:, page, :, row // R, :, row % R] = _held(v, s.case["kv"]).transpose(0, 1)


def _plain_append(s):
    k, v = s.k.float(), s.v.float()
    _put(s, s.slots, _rotated(k, s.rope_cs) if s.rope_cs is not None else k, v)
    return {"k": s.k_pages, "v": s.v_pages}


def _plain_fill(s):
    pr, R = s.case["page_rows"], _unit_rows(s.case["kv"])
    src, first = _window(s.case)
    last = first + s.case["dropped"]
    page, row = (s.slots // pr).long(), (s.slots % pr).long()
    s.k_pages[first:last, page, :, row] = s.k_pages[src, page, :, row][:, None]
    s.v_pages[first:last, page, :, row // R, :, row % R] = s.v_pages[src, page, :, row // R, :, row % R][:, None]
    return {"k": s.k_pages, "v": s.v_pages}


def _plain_attend(s):
    case = s.case
    B, pr, R, hd, heads, group = case["B"], case["page_rows"], _unit_rows(case["kv"]), case["hd"], case["heads"], case["group"]
    q = s.q.float()
    rows = s.rows.long()
    if case["new"]:
        q = _rotated(q, s.rope_cs)
        last = (rows - 1).clamp(min=0)
        slots = s.tables.gather(1, (last // pr)[:, None])[:, 0].long() * pr + last % pr
        live = rows > 0
        _put(s, slots[live], _rotated(s.k.float(), s.rope_cs)[live][None], s.v.float()[live][None])
    t = torch.arange(case["rows"], device=DEVICE)
    page = s.tables[:, t // pr].clamp(min=0).long()        # [B][rows]
    k = s.k_pages[0][page, :, t % pr].float()              # [B][rows][heads][hd]
    v = s.v_pages[0][page, :, (t % pr) // R, :, t % R].float()
    score = torch.matmul(q.view(B, heads, group, hd), k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(hd)
    dead = (t[None] >= rows[:, None])[:, None, None]
    score = score.masked_fill(dead, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()) / torch.where(total > 0, total, 1)
    s.out.copy_(out.view(B, heads * group, hd))
    return {"out": s.out, "k": s.k_pages, "v": s.v_pages} if case["new"] else {"out": s.out}


_plain = {"reserve": _plain_reserve, "append": _plain_append, "fill": _plain_fill, "attend": _plain_attend}


# ---------------- 64 bits ----------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"reserve": _exact_reserve, "append": _exact_append, "fill": _exact_fill, "attend": _exact_attend}[case["op"]](s)


def _exact_reserve(s):
    pr = s.case["page_rows"]
    rows, added, tables = s.rows.cpu().numpy().copy(), s.added.cpu().numpy(), s.tables.cpu().numpy().copy()
    stack = s.free_pages.cpu().numpy()[: int(s.n_free[0])].tolist()
    for b in range(len(rows)):
        if added[b] < 0:
            stack += tables[b, : -(-rows[b] // pr)].tolist()
            rows[b] = 0
    avail, asked_tokens, asked_pages = len(stack), 0, 0
    starts, slots, positions = [0], [], []
    for b in range(len(rows)):
        n = max(0, int(added[b]))
        if n and rows[b] + n <= s.max_pages * pr:
            asked_tokens += n
            if asked_tokens <= s.max_tokens:
                first, end = -(-rows[b] // pr), -(-(rows[b] + n) // pr)
                asked_pages += end - first
                if end == first or asked_pages <= avail:
                    for j in range(first, end):
                        tables[b, j] = stack.pop()
                    p = np.arange(rows[b], rows[b] + n)
                    positions += p.tolist()
                    slots += (tables[b, p // pr] * pr + p % pr).tolist()
                    rows[b] += n
        starts.append(len(slots))
    short = s.max_tokens - len(slots)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32)
    return {"starts": ints(starts), "slots": ints(slots + [-1] * short), "positions": ints(positions + [-1] * short), "rows": ints(rows),
            "n_free": ints([len(stack), max(0, asked_pages - avail)]), "tables": ints(tables)}


def _turn(x, positions):
    """The rotation by its definition: x [n][heads][hd] double, angles from the positions."""
    hd = x.shape[-1]
    j = torch.arange(hd // 2, dtype=torch.float64, device=x.device)
    z = torch.complex(x[..., : hd // 2], x[..., hd // 2:]) * torch.polar(torch.ones_like(j), positions.double()[:, None] / ROPE_BASE ** (2 * j / hd))[:, None]
    return torch.cat([z.real, z.imag], -1)


def _exact_append(s):
    pr, R = s.case["page_rows"], _unit_rows(s.case["kv"])
    most = HALF_MAX if s.case["kv"] == "f16" else math.inf
    k, v = s.k_pages.double(), s.v_pages.double()
    at = torch.arange(5, 5 + s.slots.numel(), device=DEVICE)
    slots = s.slots.long()
    for l in range(k.shape[0]):
        new = s.k[l].double()
        k[l][slots // pr, :, slots % pr] = (_turn(new, at) if s.case["rope"] else new).clamp(-most, most)
        v[l][slots // pr, :, slots % pr // R, :, slots % R] = s.v[l].double().clamp(-most, most)
    return {"k": k, "v": v}


def _exact_fill(s):
    pr, R = s.case["page_rows"], _unit_rows(s.case["kv"])
    src, first = _window(s.case)
    for l in range(first, first + s.case["dropped"]):
        for slot in s.slots.tolist():
            page, row = divmod(slot, pr)
            s.k_pages[l, page, :, row] = s.k_pages[src, page, :, row]
            s.v_pages[l, page, :, row // R, :, row % R] = s.v_pages[src, page, :, row // R, :, row % R]
    return {"k": s.k_pages.double(), "v": s.v_pages.double()}


def _exact_attend(s):
    case = s.case
    pr, hd, heads, group, kv = case["page_rows"], case["hd"], case["heads"], case["group"], case["kv"]
    R = _unit_rows(kv)
    most = HALF_MAX if kv == "f16" else math.inf
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=DEVICE)
    whole_k, whole_v = (s.k_pages.double(), s.v_pages.double()) if case["new"] else (None, None)
    for b, n in enumerate(s.rows.tolist()):
        if n == 0:
            continue
        pages = s.tables[b, : _pages(n, pr)].long()
        k = s.k_pages[0][pages].permute(0, 2, 1, 3).reshape(-1, heads, hd)[:n].double()
        v = s.v_pages[0][pages].permute(0, 2, 4, 1, 3).reshape(-1, heads, hd)[:n].double()
        q = s.q[b].double()
        if case["new"]:
            at = torch.tensor([n - 1], device=DEVICE)
            q = _turn(q[None], at)[0]
            new_k, new_v = _turn(s.k[b:b + 1].double(), at)[0].clamp(-most, most), s.v[b].double().clamp(-most, most)
            k[-1], v[-1] = new_k.to(TYPES[kv]).double(), new_v.to(TYPES[kv]).double()      # rows are used as the cache holds them
            page, row = int(pages[-1]), (n - 1) % pr
            whole_k[0, page, :, row] = new_k
            whole_v[0, page, :, row // R, :, row % R] = new_v
        score = torch.bmm(q.view(heads, group, hd), k.permute(1, 2, 0).contiguous()) / math.sqrt(hd)
        out[b] = torch.bmm(torch.softmax(score, -1), v.permute(1, 0, 2).contiguous()).view(heads * group, hd)
    return {"out": out, "k": whole_k, "v": whole_v} if case["new"] else {"out": out}


def work(case):
    op = case["op"]
    if op == "reserve":
        rows, added = _requests(case)
        asked = np.maximum(added, 0)
        tokens = int(asked.sum())
        pages = int((_pages(rows + asked, case["page_rows"]) - _pages(rows, case["page_rows"])).sum())
        back = int(_pages(rows[added < 0], case["page_rows"]).sum())
        # rows and requests in, rows and starts out, pages from and to the stack and the tables, a slot and a position a token
        return {"bytes": 4 * (4 * case["B"] + 2 * pages + 2 * back + 2 * tokens), "flops": 0}
    row = case["heads"] * case["hd"] * 2
    if op == "append":
        n = case["tokens"] * case["layers"]
        angles = case["tokens"] * (case["hd"] * 4 if case["rope"] else 0)
        return {"bytes": n * row * (BYTES[case["src"]] + BYTES[case["kv"]]) + angles + 4 * case["tokens"], "flops": n * row * 3 // 2 if case["rope"] else 0}
    if op == "fill":
        return {"bytes": case["B"] * row * BYTES[case["kv"]] * (1 + case["dropped"]), "flops": 0}
    n, heads = sum(_lengths(case)), case["heads"] * case["group"]
    act = case["B"] * BYTES[case["act"]] * (2 * heads * case["hd"] + (row if case["new"] else 0))
    return {"bytes": n * row * BYTES[case["kv"]] + act, "flops": 4 * n * heads * case["hd"]}

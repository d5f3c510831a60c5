"""A paged cache held in 8 bits, and rows read back from pages of every type, against plain implementations: codes and scales bit by bit, attention in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MOST_CODE = {"i8": 127.0, "e4m3": 448.0}


def _types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def _bits(x):
    import torch
    return x.view(torch.uint8)


def _generator(seed):
    import torch
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _quantised(x, kv):
    """(codes, scales) of rows x [..., hd] (fp32) by the definition, operation by operation on the CPU: every one of them rounds once."""
    import torch
    x = x.float().cpu()
    a = x.abs().amax(-1).clamp(max=3e38)
    q = torch.full_like(a, MOST_CODE[kv])
    zeros = a < 2.0 ** -100
    scale, inv = torch.where(zeros, 0, a / q), torch.where(zeros, 0, q / a)
    y = (x * inv[..., None]).clamp(-MOST_CODE[kv], MOST_CODE[kv])
    y = torch.where(a.isnan()[..., None], 0, y)             # (codes of a row with a NaN say nothing)
    return (y.round() if kv == "i8" else y).to(_types()[kv]), scale


def _turned32(x, cs):
    """The rotation in fp32, products and sums rounded each."""
    import torch
    half = x.shape[-1] // 2
    x, cs = x.float().cpu(), cs.cpu()
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _turned64(x, cs):
    import torch
    half = x.shape[-1] // 2
    c, s = cs.double()[:, None, :, 0], cs.double()[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, a * s + b * c], -1)


def _angles(positions, hd):
    import torch
    p = torch.as_tensor(positions, dtype=torch.float64, device=DEV)
    a = p[:, None] * 10000.0 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64, device=DEV) / hd)
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _as_rows(pool, values=None):
    """A pool of keys or values as [layer][slot][head][dim], scales as [layer][slot][head] (copies; codes as bytes)."""
    import torch
    if values is None:
        L, n, h, pr = pool.shape
        return pool.permute(0, 1, 3, 2).reshape(L, n * pr, h).clone(memory_format=torch.contiguous_format)
    pool = _bits(pool) if pool.element_size() == 1 else pool
    if values:
        L, n, h, blocks, hd, R = pool.shape
        return pool.permute(0, 1, 3, 5, 2, 4).reshape(L, n * blocks * R, h, hd).clone(memory_format=torch.contiguous_format)
    L, n, h, pr, hd = pool.shape
    return pool.permute(0, 1, 3, 2, 4).reshape(L, n * pr, h, hd).clone(memory_format=torch.contiguous_format)


def _state(cache):
    """(key codes, value codes, key scales, value scales) as rows."""
    return [_as_rows(cache.k_pages, False), _as_rows(cache.v_pages, True), _as_rows(cache.k_scales), _as_rows(cache.v_scales)]


def _set_rows(cache, codes_k, codes_v, ks, vs):
    """The other way round, of one cache."""
    pr, hd, h, n, L = cache.page_rows, cache.head_dim, cache.n_kv_heads, cache.n_pages, cache.n_layers
    _bits(cache.k_pages).copy_(codes_k.view(L, n, pr, h, hd).permute(0, 1, 3, 2, 4))
    R = cache.v_pages.shape[-1]
    _bits(cache.v_pages).copy_(codes_v.view(L, n, pr // R, R, h, hd).permute(0, 1, 4, 2, 5, 3))
    cache.k_scales.copy_(ks.view(L, n, pr, h).permute(0, 1, 3, 2))
    cache.v_scales.copy_(vs.view(L, n, pr, h).permute(0, 1, 3, 2))


def _values(codes, scales, kv):
    """64-bit values of codes given as bytes."""
    return codes.contiguous().view(_types()[kv]).double() * scales.double()[..., None]


def _slots(cache, b, rows):
    import torch
    p = torch.as_tensor(list(rows), dtype=torch.long, device=DEV)
    return cache.tables[b].long()[p // cache.page_rows] * cache.page_rows + p % cache.page_rows


def _fill_random(cache, g):
    """Codes of rows of normal values, scales of the size these have."""
    import torch
    Q = MOST_CODE[cache.kv_dtype]
    for pool in (cache.k_pages, cache.v_pages):
        x = torch.empty(pool.shape, device=DEV).normal_(0, Q / 3.5, generator=g).clamp_(-Q, Q)
        pool.copy_((x.round() if cache.kv_dtype == "i8" else x).to(pool.dtype))
    for s in (cache.k_scales, cache.v_scales):
        s.uniform_(2 / Q, 4 / Q, generator=g)


def _cache(lens, heads, group, hd, kv, page_rows, layers=1, spare=3, seed=0, room=0, garbage=False):
    """A cache whose sequences have the given rows on pages in random order; garbage: wherever no sequence has a row, codes and scales of any bits, NaN among them."""
    import torch
    from paper_2503_08524_amd import PagedCache
    g = _generator(seed)
    held = [-(-(n + room) // page_rows) for n in lens]
    cache = PagedCache(heads * group, heads, hd, sum(held) + spare, page_rows, len(lens), max(max(held), 1), kv_dtype=kv, n_layers=layers, device=DEV)
    order = torch.randperm(cache.n_pages, generator=g, device=DEV).int()
    at = 0
    for b, n in enumerate(held):
        cache.tables[b, :n] = order[at: at + n]
        at += n
    cache.rows.copy_(torch.tensor(lens, dtype=torch.int32))
    _fill_random(cache, g)
    if garbage:
        state = _state(cache)
        none = torch.ones(cache.n_pages * page_rows, dtype=torch.bool, device=DEV)
        for b, n in enumerate(lens):
            none[_slots(cache, b, range(n))] = False
        for x in state[:2]:
            x[:, none] = torch.randint(0, 256, x[:, none].shape, generator=g, device=DEV).to(torch.uint8)
            x[:, none, :, ::7] = 0x7f
        state[2][:, none], state[3][:, none] = math.nan, math.inf
        _set_rows(cache, *state)
    return cache, g


# ---------------- rows into pages ----------------

APPENDS = [  # tokens, heads, hd, src, kv, page_rows, layers, rotated
    (1, 1, 64, "f32", "i8", 16, 1, True), (77, 8, 64, "bf16", "i8", 16, 1, True), (64, 2, 128, "f16", "e4m3", 16, 2, False), (65, 5, 128, "f32", "e4m3", 64, 1, True),
    (200, 2, 128, "f32", "i8", 128, 3, False), (130, 1, 128, "bf16", "e4m3", 32, 1, False), (300, 3, 64, "f16", "i8", 16, 1, True), (97, 2, 64, "f32", "e4m3", 32, 1, True),
    (31, 1, 128, "f16", "i8", 16, 2, True), (16, 2, 128, "bf16", "i8", 1024, 1, True)]


def _some_slots(order, n, page_rows, n_pages, g):
    """Slots of n rows: consecutive ones, from the 6th of a sequence on, pieces with gaps, any order, some that are none."""
    import torch
    total = n_pages * page_rows
    pages = torch.randperm(n_pages, generator=g, device=DEV)
    p = torch.arange(n, device=DEV) + (5 if order == "late" else 0)
    slots = pages[p // page_rows] * page_rows + p % page_rows
    if order == "runs" and n + n // 23 * 3 + 30 <= total:
        slots = torch.cat([torch.arange(23, device=DEV) + 26 * j for j in range(n // 23 + 1)])[:n]
    if order == "mixed":
        slots = torch.randperm(total, generator=g, device=DEV)[:n]
    if order == "backwards":
        slots = slots.flip(0)
    slots = slots.int()
    if order in ("none", "runs"):
        slots[::7] = torch.tensor([-1, total, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV).repeat(n)[: slots[::7].numel()]
    return slots


@pytest.mark.parametrize("case", range(len(APPENDS)))
@pytest.mark.parametrize("order", ["run", "late", "runs", "mixed", "backwards", "none"])
def test_append_holds_the_codes_of_the_definition(case, order):
    import torch
    from paper_2503_08524_amd import PagedCache
    n, heads, hd, src, kv, page_rows, layers, rope = APPENDS[case]
    g = _generator(case)
    n_pages = (n + 60) // page_rows + 4
    cache = PagedCache(heads, heads, hd, n_pages, page_rows, 1, 1, kv_dtype=kv, n_layers=layers + 1, device=DEV)
    _fill_random(cache, g)
    total = n_pages * page_rows
    slots = _some_slots(order, n, page_rows, n_pages, g)
    t = _types()[src]
    k, v = (torch.empty(layers, n, heads, hd, dtype=t, device=DEV).normal_(generator=g) for _ in range(2))
    k[0, 0], v[0, -1] = 0, k[0, -1] * 1000
    cs = _angles(list(range(3, n + 3)), hd) if rope else None
    before = _state(cache)
    cache.append(1, slots, k, v, rope_cs=cs)
    live = ((slots >= 0) & (slots < total)).nonzero()[:, 0]
    at, kept = slots[live].long(), torch.ones(total, dtype=torch.bool, device=DEV)
    kept[at] = False
    after = _state(cache)
    for was, now in zip(before, after):
        assert torch.equal(was[0].view(torch.uint8), now[0].view(torch.uint8)) and torch.equal(was[:, kept].view(torch.uint8), now[:, kept].view(torch.uint8))
    x64 = [(_turned64(k.double(), cs) if rope else k.double())[:, live], v.double()[:, live]]
    for i, x in enumerate([torch.stack([_turned32(y, cs) for y in k]) if rope else k, v]):
        codes, scales = _quantised(x[:, live.to(x.device)], kv)
        assert torch.equal(after[2 + i][1:, at].cpu(), scales)
        assert torch.equal(after[i][1:, at].cpu(), _bits(codes))
        # half a step, and what the rotation's three roundings and those of the scale and its inverse (2 of 2^-24 a code) move
        got, a = _values(after[i][1:, at], after[2 + i][1:, at], kv), x64[i].abs().amax(-1, keepdim=True)
        half = a / 254 if kv == "i8" else torch.maximum(2.0 ** -4 * x64[i].abs(), a * 2.0 ** -10 / 448)
        assert ((got - x64[i]).abs() <= half * (1 + 2.0 ** -20) + a * (6 + 3) * 2.0 ** -24).all()


@pytest.mark.parametrize("kv", ["i8", "e4m3"])
@pytest.mark.parametrize("hd", [64, 128])
def test_append_of_zeros_tiny_and_huge_rows_infinities_and_nan(kv, hd):
    import torch
    from paper_2503_08524_amd import PagedCache
    g = _generator(hd)
    n = 40
    x = torch.empty(n, 2, hd, device=DEV).normal_(generator=g)
    x[0] = 0
    x[1] = -0.0
    x[2] *= 1e-38
    x[3], x[3, :, 5] = 0, 2.0 ** -100
    x[4], x[4, :, 5] = 0, float(np.nextafter(np.float32(2.0 ** -100), np.float32(0)))
    x[5] *= 1e37
    x[6, :, 7] = 3.4e38
    x[7, :, 3], x[7, :, 9] = math.inf, -math.inf
    x[8, 1, 11] = math.nan
    x[9], x[9, :, hd - 1] = 1e-45, 1.0
    x[10] = 2.5
    x[11] = torch.linspace(-127, 127, hd, device=DEV)
    x[12, :, 0] = 1e6
    for first in (0, 3):                                   # rows 0 .. 31 and 32 .. fill units; from slot 3 on rows 13 .. 28 do
        cache = PagedCache(2, 2, hd, 5, 16, 1, 1, kv_dtype=kv, device=DEV)
        slots = torch.arange(first, first + n, dtype=torch.int32, device=DEV)
        cache.append(0, slots, x, x.flip(0).contiguous().flip(0))
        codes, scales = _quantised(x, kv)
        for got, s in zip(_state(cache)[:2], _state(cache)[2:]):
            got, s = got[0, first: first + n].cpu(), s[0, first: first + n].cpu()
            assert torch.equal(s.isnan(), scales.isnan()) and torch.equal(torch.nan_to_num(s), torch.nan_to_num(scales))
            fine = ~scales.isnan()
            assert torch.equal(got[fine], _bits(codes)[fine])
        back = cache.read(0, slots)[0]
        assert back[8, 1].isnan().all() and back.isnan().sum() == hd                   # a row with a NaN is NaN, its neighbours are not
        assert (back[:2] == 0).all() and (back[2] == 0).all() and (back[4] == 0).all() and back[3, 0, 5] > 0
        assert back[7, 0, 3] > 2.99e38 and back[7, 0, 9] < -2.99e38 and back[6, 0, 7] > 2.99e38


def test_append_strides_and_no_rows():
    import torch
    from paper_2503_08524_amd import PagedCache
    cache = PagedCache(2, 2, 64, 4, 16, 1, 1, kv_dtype="i8", device=DEV)
    buf = torch.randn(20, 2, 2, 3, 64, device=DEV)          # token, head, other things
    k, v = buf[:, :, 0, 0], buf[:, :, 1, 2]
    slots = torch.arange(7, 27, dtype=torch.int32, device=DEV)
    cache.append(0, slots, k, v)
    state = _state(cache)
    for i, x in enumerate((k, v)):
        codes, scales = _quantised(x, "i8")
        assert torch.equal(state[i][0, 7:27].cpu(), _bits(codes)) and torch.equal(state[2 + i][0, 7:27].cpu(), scales)
        assert not state[i][0, :7].any() and not state[i][0, 27:].any() and not state[2 + i][0, 27:].any()
    cache.append(0, slots[:0], k[:0], v[:0])
    # out again into places with gaps, and rows of slots that are none stay as they are
    out = torch.full((20, 2, 2, 3, 64), 7.0, device=DEV)
    slots[4], slots[9] = -1, 64
    ko, vo = cache.read(0, slots, out[:, :, 0, 0], out[:, :, 1, 2])
    keep = torch.ones(20, dtype=torch.bool, device=DEV)
    keep[4] = keep[9] = False
    for i, x in enumerate((ko, vo)):
        want = _values(state[i][0, 7:27], state[2 + i][0, 7:27], "i8")
        assert torch.equal(x[keep].double(), want[keep].float().double()) and (x[~keep] == 7).all()
    out[:, :, 0, 0], out[:, :, 1, 2] = 7, 7
    assert (out == 7).all()
    cache.read(0, slots[:0], ko[:0], vo[:0])
    made = cache.read(0, slots)
    assert torch.equal(made[0][keep], cache.read(0, slots[keep].contiguous())[0]) and not made[0][4].any() and not made[1][9].any()


# ---------------- rows out of pages ----------------

@pytest.mark.parametrize("kv", ["i8", "e4m3", "f16", "f32"])
@pytest.mark.parametrize("to", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,heads,hd,page_rows,layers,order", [
    (1, 1, 64, 16, 1, "run"), (16, 2, 128, 16, 2, "run"), (333, 8, 64, 16, 1, "late"), (100, 3, 128, 64, 3, "runs"), (70, 2, 64, 32, 1, "mixed"), (128, 1, 128, 1024, 1, "backwards"),
    (95, 5, 128, 16, 1, "none")])
def test_read_gives_what_the_pools_hold(kv, to, n, heads, hd, page_rows, layers, order):
    import torch
    from paper_2503_08524_amd import PagedCache
    g = _generator(n)
    n_pages = (n + 60) // page_rows + 4
    cache = PagedCache(heads, heads, hd, n_pages, page_rows, 1, 1, kv_dtype=kv, n_layers=layers + 1, device=DEV)
    if kv in MOST_CODE:
        _fill_random(cache, g)
    else:
        for p in (cache.k_pages, cache.v_pages):
            p.normal_(generator=g)
    slots = _some_slots(order, n, page_rows, n_pages, g)
    if order == "mixed":
        slots[1:9] = slots[0]                              # a row as often as one likes
    k, v = cache.read(1, slots, dtype=_types()[to], n_layers=layers)
    assert k.shape == (layers, n, heads, hd) and k.dtype == _types()[to]
    live = (slots >= 0) & (slots < n_pages * page_rows)
    at = slots[live].long()
    for got, pool, scales, values in ((k, cache.k_pages, cache.k_scales, False), (v, cache.v_pages, cache.v_scales, True)):
        rows = _as_rows(pool, values)[1:, at]
        # a code times its scale is rounded to fp32 and from there to the output's type
        want = rows.contiguous().view(pool.dtype).float() * _as_rows(scales)[1:, at][..., None] if kv in MOST_CODE else rows.float()
        assert torch.equal(got[:, live], want.to(got.dtype)) and not got[:, ~live].any()
    one = cache.read(layers, slots)
    assert one[0].dtype == torch.float32 and one[0].shape == (n, heads, hd)
    assert torch.equal(one[1].to(v.dtype), v[-1])


def test_read_then_append_to_another_cache_keeps_the_codes():
    """Out of one cache and into another: the largest code of a row is 127 (or 448) again and the scale the same but for its rounding, so the codes come back."""
    import torch
    from paper_2503_08524_amd import PagedCache
    for kv in ("i8", "e4m3"):
        caches = [PagedCache(3, 3, 128, 20, 16, 1, 1, kv_dtype=kv, n_layers=2, device=DEV) for _ in range(2)]
        x = torch.randn(2, 300, 3, 128, device=DEV), torch.randn(2, 300, 3, 128, device=DEV)
        slots = [torch.arange(2, 302, dtype=torch.int32, device=DEV), torch.randperm(320, device=DEV)[:300].int()]
        caches[0].append(0, slots[0], *x)
        caches[1].append(0, slots[1], *caches[0].read(0, slots[0], n_layers=2))
        a, b = _state(caches[0]), _state(caches[1])
        for i in range(4):
            p, q = a[i][:, slots[0].long()], b[i][:, slots[1].long()]
            assert torch.equal(p, q) if i < 2 else ((p - q).abs() <= 2.0 ** -23 * p).all()


# ---------------- the missing-state fill ----------------

@pytest.mark.parametrize("kv,heads,hd,page_rows", [("i8", 3, 128, 16), ("e4m3", 2, 64, 32), ("i8", 1, 64, 16), ("e4m3", 32, 128, 16)])
def test_fill_copies_codes_and_scales_into_the_dropped_layers(kv, heads, hd, page_rows):
    import torch
    cache, g = _cache([40, 33], heads, 1, hd, kv, page_rows, layers=20, seed=3, garbage=True)
    slots = torch.cat([_slots(cache, 0, [39, 0, 17]), _slots(cache, 1, [32])]).int()
    slots = torch.cat([slots, slots[:1], torch.tensor([-1, cache.n_pages * page_rows], dtype=torch.int32, device=DEV)])      # one row twice, two that are none
    at = slots[:4].long()
    for src, first, n in ((4, 5, 15), (19, 0, 3), (7, 8, 1), (-1, 2, 9)):
        before = _state(cache)
        cache.fill(slots, src, first, n)
        for was, now in zip(before, _state(cache)):
            want = was.clone()
            for l in range(first, first + n):
                want[l, at] = was[src, at] if src >= 0 else 0
            assert torch.equal(_bits(now), _bits(want))
    cache.fill(slots[:0], 0, 1, 1)
    cache.fill(slots, 0, 1, 0)


@pytest.mark.parametrize("n,heads,layers", [(16, 2, 64), (16, 2, 65), (64, 8, 9), (512, 8, 3), (511, 8, 11), (2048, 1, 1)])
def test_fill_on_either_side_of_its_shares(n, heads, layers):
    import torch
    from paper_2503_08524_amd import PagedCache
    g = _generator(n + layers)
    cache = PagedCache(heads, heads, 64, n // 16 + 2, 16, 1, 1, kv_dtype="i8", n_layers=layers + 2, device=DEV)
    _fill_random(cache, g)
    slots = torch.randperm(cache.n_pages * 16, generator=g, device=DEV)[:n]
    want = _state(cache)
    for rows in want:
        rows[1:layers + 1, slots] = rows[layers + 1, slots][None]
    cache.fill(slots.int(), layers + 1, 1, layers)
    for rows, now in zip(want, _state(cache)):
        assert torch.equal(rows, now)


# ---------------- attention ----------------

def _reference(cache, q, lens, layer=0, scale=None, gone=()):
    """(out, allowed error) in 64 bits from what the pools hold; `gone`: (sequence, page index) whose rows do not count.

    The error, relative to sum_j p_j |v_j| of a dim: codes are exact in the products.  A score has the roundings of q (rotation: 3 of 2^-24; as two fp16 halves 2^-22), of hd products summed in fp32 (hd
    of 2^-24) and of three factors (3 of 2^-24), all relative to sum |q k|, and moves a weight by that, once for itself and once for the maximum.  A weight has the exponential and rescalings
    (2^-22), its row's scale and the unit's factor (2^-22 together) and two halves (2^-22); the sums over n rows n / 8 + 64 roundings at most in a row.  Halves count in steps of 2^-24 where the largest
    weight times scale is 2^15, so every row may be 2^-40 of that times its largest code off."""
    import torch
    B, H, hd = q.shape
    group = H // cache.n_kv_heads
    scale = 1 / math.sqrt(hd) if scale is None else scale
    state = _state(cache)
    K, V = (_values(state[i][layer], state[2 + i][layer], cache.kv_dtype) for i in range(2))
    out, most = (torch.zeros(B, H, hd, dtype=torch.float64, device=DEV) for _ in range(2))
    for b, n in enumerate(lens):
        rows = [j for j in range(n) if (b, j // cache.page_rows) not in gone]
        if not rows:
            continue
        at = _slots(cache, b, rows)
        k, v = K[at].repeat_interleave(group, 1), V[at].repeat_interleave(group, 1)
        s = torch.einsum("hd,nhd->hn", q[b], k) * scale
        p = torch.softmax(s, -1)
        out[b] = torch.einsum("hn,nhd->hd", p, v)
        size = torch.einsum("hd,nhd->hn", q[b].abs(), k.abs()).amax(-1) * abs(scale)
        each = 2.0 ** -22 + (hd + 6) * 2.0 ** -24
        step = (p * state[3][layer][at].double().T.repeat_interleave(group, 0)).amax(-1) * MOST_CODE[cache.kv_dtype]
        most[b] = (torch.einsum("hn,nhd->hd", p, v.abs()) * (2 * each * size + 3 * 2.0 ** -22 + (n / 8 + 64) * 2.0 ** -24)[:, None] + (n * 2.0 ** -40 * step)[:, None])
    return out, most


def _check(got, want, most):
    import torch
    step = torch.finfo(got.dtype).eps / 2
    bad = (got.double() - want).abs() > most * 1.01 + step * want.abs() + 1e-30
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((got.double() - want).abs().max()):.3e}, allowed {float(most.max()):.3e}"


def _check_newest(cache, before, k, v, lens, kv, layer=0):
    """The newest rows are held by the definition (k as it was turned, fp32), every other row as before."""
    import torch
    after = _state(cache)
    live = [b for b, n in enumerate(lens) if n > 0]
    at = torch.cat([_slots(cache, b, [lens[b] - 1]) for b in live]) if live else torch.zeros(0, dtype=torch.long, device=DEV)
    rest = torch.ones(after[0].shape[1], dtype=torch.bool, device=DEV)
    rest[at] = False
    for i, x in enumerate((k, v)):
        for j in (i, 2 + i):
            assert torch.equal(_bits(before[j][:, rest].contiguous()), _bits(after[j][:, rest].contiguous()))
        if live:
            codes, scales = _quantised(x[live], kv)
            assert torch.equal(after[2 + i][layer, at].cpu(), scales) and torch.equal(after[i][layer, at].cpu(), _bits(codes))


EDGES = [0, 1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000]
CASES = [  # lens, heads, group, hd, kv, act, page_rows, new rows, rotated
    (EDGES, 2, 1, 128, "i8", "f32", 16, False, False),
    (EDGES, 2, 2, 64, "i8", "bf16", 16, True, True),
    (EDGES, 2, 4, 128, "e4m3", "f32", 16, True, True),
    (EDGES, 1, 8, 64, "e4m3", "f16", 32, True, False),
    (EDGES, 3, 3, 128, "e4m3", "f16", 64, False, True),
    (EDGES, 1, 16, 128, "i8", "bf16", 128, True, True),
    (EDGES, 1, 17, 128, "i8", "f32", 16, True, True),
    ([300, 0, 77], 2, 40, 64, "i8", "f32", 32, True, True),
    ([300, 1, 77], 1, 33, 128, "e4m3", "bf16", 16, True, True),
    ([640], 32, 1, 128, "e4m3", "f32", 16, True, True),
    ([1], 4, 1, 64, "i8", "f32", 16, True, True),
    ([0, 0, 0], 4, 2, 128, "i8", "f32", 16, True, True),
    ([20000], 1, 4, 128, "i8", "f32", 16, True, True),
    ([9000, 3, 0, 4001], 2, 5, 64, "e4m3", "f32", 1024, True, True),
    ([(37 * b) % 91 if b % 5 else 0 for b in range(200)], 2, 2, 128, "i8", "f32", 16, True, True),
    ([0] * 130 + [5] + [0] * 69 + [700], 2, 1, 64, "i8", "f16", 16, True, False),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_against_64_bits(case):
    import torch
    lens, heads, group, hd, kv, act, page_rows, new, rope = CASES[case]
    cache, g = _cache(lens, heads, group, hd, kv, page_rows, seed=case, garbage=True)
    B, H, t = len(lens), heads * group, _types()[act]
    q = torch.empty(B, H, hd, dtype=t, device=DEV).normal_(generator=g)
    k, v = (torch.empty(B, heads, hd, dtype=t, device=DEV).normal_(generator=g) for _ in range(2))
    cs = _angles([max(n - 1, 0) for n in lens], hd) if rope else None
    before = _state(cache)
    out = cache.attend(0, q, k if new else None, v if new else None, rope_cs=cs)
    _check_newest(cache, before, _turned32(k, cs) if rope else k, v, lens if new else [0] * B, kv)
    _check(out, *_reference(cache, _turned64(q.double(), cs) if rope else q.double(), lens))
    assert torch.equal(out, cache.attend(0, q, k if new else None, v if new else None, rope_cs=cs))       # the same bits again


@pytest.mark.parametrize("heads,group,hd,kv,act,page_rows", [(8, 1, 128, "i8", "f32", 32), (8, 4, 128, "e4m3", "f32", 16), (16, 2, 64, "i8", "bf16", 64), (8, 3, 64, "e4m3", "f16", 16)])
def test_attention_runs_of_many_chunks(heads, group, hd, kv, act, page_rows):
    """More rows than a chunk for every workgroup: runs of many turns that begin anywhere in their circle, end inside sequences and hold several."""
    import torch
    rng = np.random.RandomState(hd + heads)
    lens = [4096] * 12 + [4097, 4095, 0, 1] + rng.randint(3000, 5200, 20).tolist() + rng.randint(1, 200, 12).tolist()
    cache, g = _cache(lens, heads, group, hd, kv, page_rows, seed=21, garbage=True, spare=0)
    t = _types()[act]
    q = torch.empty(len(lens), heads * group, hd, dtype=t, device=DEV).normal_(generator=g)
    k, v = (torch.empty(len(lens), heads, hd, dtype=t, device=DEV).normal_(generator=g) for _ in range(2))
    before = _state(cache)
    out = cache.attend(0, q, k, v)
    _check_newest(cache, before, k, v, lens, kv)
    del before
    _check(out, *_reference(cache, q.double(), lens))


@pytest.mark.parametrize("B,heads,group,hd,kv,act,page_rows,longest,long", [
    (300, 8, 4, 128, "i8", "bf16", 16, 70, 4000), (70, 32, 1, 128, "e4m3", "f32", 16, 100, 0), (260, 4, 17, 128, "i8", "f32", 32, 100, 1000),
    (150, 16, 3, 64, "e4m3", "f16", 16, 200, 6000), (520, 4, 16, 64, "i8", "bf16", 64, 90, 3000)])
def test_attention_of_many_short_sequences(B, heads, group, hd, kv, act, page_rows, longest, long):
    """As many (sequence, heads) as waves, and few rows of each: every wave takes a run of its own.  Also with sequences that many waves share, and with the same tables when half of
    the sequences have no rows, or all have more of them."""
    import torch
    turn = 1024 * 8 // hd                                   # rows of a wave's turn
    rng = np.random.RandomState(B)
    few = rng.randint(1, longest, B)
    few[:6] = 1, turn, turn + 1, 2 * turn, turn - 1, 0
    few[B // 2] = long or 1
    few[B // 3] = 0
    many = np.maximum(few, 4 * turn + rng.randint(-3, 4, B))
    half = np.where(np.arange(B) % 2 == 0, few, 0)
    cache, g = _cache(many.tolist(), heads, group, hd, kv, page_rows, seed=B)
    q = torch.empty(B, heads * group, hd, dtype=_types()[act], device=DEV).normal_(generator=g)
    k, v = (torch.empty(B, heads, hd, dtype=_types()[act], device=DEV).normal_(generator=g) for _ in range(2))
    cs = _angles(list(range(B)), hd)
    k32 = _turned32(k, cs)
    for lens in (few, half, many, few):
        lens = lens.tolist()
        cache.rows.copy_(torch.tensor(lens, dtype=torch.int32))
        before = _state(cache)
        out = cache.attend(0, q, k, v, rope_cs=cs)
        _check_newest(cache, before, k32, v, lens, kv)
        _check(out, *_reference(cache, _turned64(q.double(), cs), lens))
        assert torch.equal(out, cache.attend(0, q, k, v, rope_cs=cs))


@pytest.mark.parametrize("heads,group,hd,kv", [(8, 2, 128, "i8"), (4, 5, 64, "e4m3"), (2, 17, 128, "e4m3")])
def test_attention_of_every_number_of_parts(heads, group, hd, kv):
    """One sequence of one to twenty chunks: as many partial results a head, joined in rounds of every width, and in two rounds."""
    import torch
    chunk = 4 * 1024 * 8 // hd
    for parts in range(1, 21):
        lens = [parts * chunk - parts % 3]
        cache, g = _cache(lens, heads, group, hd, kv, 16, seed=parts)
        q = torch.empty(1, heads * group, hd, device=DEV).normal_(generator=g)
        out = cache.attend(0, q)
        _check(out, *_reference(cache, q.double(), lens))
        assert torch.equal(out, cache.attend(0, q))


@pytest.mark.parametrize("kv", ["i8", "e4m3"])
@pytest.mark.parametrize("how", ["values", "keys", "zeros", "one"])
def test_attention_of_scales_far_apart(kv, how):
    """Scales of rows from 2^-60 to 2^60 (values), 2^-40 to 4 (keys); values that are zeros where the scores are largest; a single row with a large value among small ones."""
    import torch
    lens = [1, 64, 65, 700, 5000, 130]
    cache, g = _cache(lens, 2, 3, 128, kv, 16, seed=17, garbage=True)
    state = _state(cache)
    far = torch.rand(state[2].shape, generator=g, device=DEV)
    held = ~state[2].isnan()
    if how == "values":
        state[3] = torch.where(held, state[3] * torch.exp2(far * 120 - 60), state[3])
    elif how == "keys":
        state[2] = torch.where(held, state[2] * torch.exp2(far * 42 - 40), state[2])
    elif how == "zeros":
        state[3] = torch.where(held & (far < 0.7), 0, state[3])
        state[2] = torch.where(held & (far < 0.7), state[2] * 10, state[2])
        state[3][0, _slots(cache, 1, range(64))] = 0            # nothing but zeros
        state[1][0, _slots(cache, 2, range(65))] = 0
    else:
        state[3] = torch.where(held, state[3] * 2.0 ** -100, state[3])
        state[3][0, _slots(cache, 4, [2500])] = 1e30
    _set_rows(cache, *state)
    q = torch.empty(6, 6, 128, device=DEV).normal_(generator=g)
    out = cache.attend(0, q)
    _check(out, *_reference(cache, q.double(), lens))
    if how == "zeros":
        assert not out[1].any() and not out[2].any()


def test_attention_of_a_nan_scale_stays_with_its_sequence_and_head():
    import torch
    for kv in ("i8", "e4m3"):
        cache, g = _cache([50, 50, 50], 2, 2, 128, kv, 16, seed=8)
        q = torch.empty(3, 4, 128, device=DEV).normal_(generator=g)
        clean = cache.attend(0, q)
        state = _state(cache)
        for at in (2, 3):
            bad = [x.clone() for x in state]
            bad[at][0, _slots(cache, 1, [20]), 1] = math.nan
            _set_rows(cache, *bad)
            out = cache.attend(0, q)
            assert out[1, 2:].isnan().all()
            out[1, 2:] = clean[1, 2:]
            assert torch.equal(out, clean)
        _set_rows(cache, *state)
        k, v = (torch.empty(3, 2, 128, device=DEV).normal_(generator=g) for _ in range(2))
        want = cache.attend(0, q, k, v)
        v[0, 1, 77] = math.nan                             # the newest value
        out = cache.attend(0, q, k, v)
        assert out[0, 2:].isnan().all()
        out[0, 2:] = want[0, 2:]
        assert torch.equal(out, want)


def test_attention_large_scores():
    """One row ahead of all others by more than fp32 exponents reach, and queries far from one."""
    import torch
    for kv in ("i8", "e4m3"):
        cache, g = _cache([70, 300], 1, 2, 64, kv, 16, seed=9)
        for size in (1e-6, 1e4):
            q = torch.empty(2, 2, 64, device=DEV).normal_(generator=g) * size
            out = cache.attend(0, q)
            want, most = _reference(cache, q.double(), [70, 300])
            if size < 1:
                _check(out, want, most)
            else:                                           # scores thousands apart: the weights are 0 and 1 wherever no two scores are within the error
                assert out.isfinite().all()
                assert ((out.double() - want).abs() <= 1e-5 * want.abs() + 1e-6).double().mean() > 0.9


@pytest.mark.parametrize("kv", ["i8", "e4m3"])
@pytest.mark.parametrize("keys,queries", [(1e-25, 1.0), (1e-25, 1e25), (1e20, 1e-20), (1e30, 1e-30), (1e33, 1.0), (1e36, 1.0), (3e36, 1e-36)])
def test_attention_of_keys_and_queries_of_any_size(kv, keys, queries):
    """Keys far from one: where the queries make up for them the outputs are those of ordinary ones, and where they do not the weights are all alike or 0 and 1; nothing but a score that is too large for
    fp32 (sum |q k| is 1e38 at most here) would overflow."""
    import torch
    lens = [70, 300, 1000]
    cache, g = _cache(lens, 2, 2, 128, kv, 16, seed=19, garbage=True)
    cache.k_scales.mul_(keys)
    q = torch.empty(3, 4, 128, device=DEV).normal_(generator=g) * queries
    out = cache.attend(0, q)
    want, most = _reference(cache, q.double(), lens)
    if keys * queries < 100:
        _check(out, want, most)
    else:                                                   # rows whose scores are apart by more than fp32's error of the largest: all heads but those with a tie to that
        assert out.isfinite().all()
        assert ((out.double() - want).abs() <= 1e-5 * want.abs() + 1e-6).double().mean() > 0.9


def test_attention_scale_layers_strides_and_an_output_with_gaps():
    import torch
    heads, group, hd, lens = 2, 2, 128, [40, 300, 0, 9]
    for kv in ("i8", "e4m3"):
        cache, g = _cache(lens, heads, group, hd, kv, 16, layers=3, seed=5)
        H = heads * group
        buf = torch.empty(4, (H + 2 * heads) * hd + 32, device=DEV).normal_(generator=g)          # a projection's rows: q, k, v and something else
        q, k, v = buf[:, : H * hd].view(4, H, hd), buf[:, H * hd: (H + heads) * hd].view(4, heads, hd), buf[:, (H + heads) * hd: (H + 2 * heads) * hd].view(4, heads, hd)
        wide = torch.full((4, H * hd + 3), 7.0, device=DEV)
        before = _state(cache)
        got = cache.attend(1, q, k, v, scale=-0.3, out=wide[:, 1: 1 + H * hd].view(4, H, hd))
        _check_newest(cache, before, k, v, lens, kv, layer=1)
        _check(got, *_reference(cache, q.double(), lens, layer=1, scale=-0.3))
        assert (wide[:, 0] == 7).all() and (wide[:, 1 + H * hd:] == 7).all()


def test_attention_leaves_out_pages_that_are_none():
    import torch
    lens, gone = [100, 33, 16, 64], {(0, 1), (0, 6), (1, 2), (2, 0), (3, 0), (3, 1)}
    for kv in ("i8", "e4m3"):
        cache, g = _cache(lens, 2, 4, 128, kv, 16, seed=6, spare=1, garbage=True)
        good = cache.tables.clone()
        state = _state(cache)
        for bad in (-1, cache.n_pages, 2 ** 31 - 1, -2 ** 31):
            for b, j in gone:
                cache.tables[b, j] = bad
            q = torch.empty(4, 8, 128, device=DEV).normal_(generator=g)
            k, v = (torch.empty(4, 2, 128, device=DEV).normal_(generator=g) for _ in range(2))
            out = cache.attend(0, q, k, v)
            cache.tables.copy_(good)
            _check(out, *_reference(cache, q.double(), lens, gone=gone))
            assert (out[2] == 0).all()
            for was, now in zip(state, _state(cache)):             # sequence 1's and 2's newest rows have no page, 0's has none either
                changed = (_bits(was.contiguous()).view(was.shape[1], -1) != _bits(now.contiguous()).view(was.shape[1], -1)).any(1).nonzero()[:, 0]
                assert set(changed.tolist()) <= set(_slots(cache, 3, [63]).tolist())
            _set_rows(cache, *state)


def test_attention_leaves_out_sequences_without_a_granted_row():
    """attend with the starts of a reserve that refused some: their rows stay as they are, bit by bit, and their outputs are 0."""
    import torch
    from paper_2503_08524_amd import PagedCache
    cache = PagedCache(4, 2, 64, 6, 16, 4, 3, kv_dtype="i8", device=DEV)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    _, slots, _ = cache.reserve(ints(16, 5, 32, 16), 69)
    cache.append(0, slots, torch.randn(69, 2, 64, device=DEV), torch.randn(69, 2, 64, device=DEV))
    starts, _, _ = cache.reserve(ints(1, 1, 0, 1), 4)              # one page is left: the last one is refused
    assert starts.tolist() == [0, 1, 2, 2, 2] and cache.rows.tolist() == [17, 6, 32, 16]
    before = _state(cache)
    q, k, v = torch.randn(4, 4, 64, device=DEV), torch.randn(4, 2, 64, device=DEV), torch.randn(4, 2, 64, device=DEV)
    out = cache.attend(0, q, k, v, starts=starts)
    _check_newest(cache, before, k, v, [17, 6, 0, 0], "i8")
    _check(out, *_reference(cache, q.double(), [17, 6, 0, 0]))


def test_offsets_past_32_bits():
    import torch
    from paper_2503_08524_amd import PagedCache
    # 18000 pages of 2 heads x 1024 rows x 128: 4.7e9 bytes a pool; the rows used are in the last pages
    cache = PagedCache(4, 2, 128, 18000, 1024, 2, 2, kv_dtype="i8", n_layers=2, device=DEV)
    cache.tables.copy_(torch.tensor([[17999, 17997], [17998, -1]], dtype=torch.int32))
    lens = [1500, 800]
    cache.rows.copy_(torch.tensor(lens, dtype=torch.int32))
    slots = torch.cat([_slots(cache, b, range(n)) for b, n in enumerate(lens)]).int()
    g = _generator(1)
    k, v = (torch.empty(2300, 2, 128, device=DEV).normal_(generator=g) for _ in range(2))
    cache.append(0, slots, k, v)
    cache.fill(slots, 0, 1, 1)
    q = torch.empty(2, 4, 128, device=DEV).normal_(generator=g)
    held = [codes.to(torch.float64) * scales.double()[..., None] for codes, scales in (_quantised(k, "i8"), _quantised(v, "i8"))]
    for layer in (0, 1):
        back = cache.read(layer, slots)
        assert all(torch.equal(x.double().cpu(), y.float().double()) for x, y in zip(back, held))
        out = cache.attend(layer, q)
        for b, (lo, hi) in enumerate(((0, 1500), (1500, 2300))):
            kk, vv = (x[lo:hi].to(DEV).repeat_interleave(2, 1) for x in held)
            s = torch.einsum("hd,nhd->hn", q[b].double(), kk) / math.sqrt(128)
            want = torch.einsum("hn,nhd->hd", torch.softmax(s, -1), vv)
            # as in _reference, with sum |q k| / sqrt(hd) below 16 and sum p |v| below 2
            assert (out[b].double() - want).abs().max() < 2 * (2 * 139 * 2.0 ** -24 * 16 + 260 * 2.0 ** -24)
    for pool in (cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales):
        assert not pool[:, :17997].any()


# ---------------- used together ----------------

def test_operators_together_as_a_server_uses_them():
    """Requests of unequal length come in, decode, end and make room: reserve, append, attend with a new row, fill and read on three layers, against lists of held rows in 64 bits."""
    import torch
    from paper_2503_08524_amd import PagedCache
    heads, group, hd, B, layers = 2, 4, 64, 5, 3
    for kv in ("i8", "e4m3"):
        cache = PagedCache(heads * group, heads, hd, 14, 16, B, 6, kv_dtype=kv, n_layers=layers, device=DEV)
        g = _generator(2)
        normal = lambda *dims: torch.empty(dims, device=DEV).normal_(generator=g)
        held = [[[torch.zeros(0, heads, hd, dtype=torch.float64) for _ in range(B)] for _ in range(layers)] for _ in range(2)]
        value = lambda x: (lambda c, s: c.double() * s.double()[..., None])(*_quantised(x, kv))
        for added in [[17, 40, 0, 0, 3], [1, 1, 70, 0, 1], [1, -1, 1, 20, 1], [1, 30, 1, 1, 1], [-1, 1, -1, 1, 1], [60, 1, 0, 1, 1], [1, 1, 9, 1, 1], [1, 1, 1, 1, 1]]:
            starts, slots, positions = cache.reserve(torch.tensor(added, dtype=torch.int32, device=DEV), 100)
            st = starts.tolist()
            one = all(a == 1 for a in added)                        # a decode step: the rows come with the attention
            total = st[-1]
            cs = torch.zeros(100, hd // 2, 2, device=DEV)
            cs[:total] = _angles(positions[:total].tolist(), hd)
            for b in range(B):
                if added[b] < 0:
                    for x in held:
                        for l in range(layers):
                            x[l][b] = x[l][b][:0]
            outs = []
            for l in range(layers - 1):                            # the last layer is dropped in every step and filled
                k, v = normal(100, heads, hd), normal(100, heads, hd)
                q = normal(B, heads * group, hd)
                if one:
                    mine = torch.tensor([min(st[b], 99) for b in range(B)], device=DEV)
                    outs.append((q, cs[mine], cache.attend(l, q, k[mine], v[mine], rope_cs=cs[mine].contiguous(), starts=starts)))
                else:
                    cache.append(l, slots, k, v, rope_cs=cs)
                for x, y in zip(held, (value(_turned32(k, cs)), value(v))):
                    for b in range(B):
                        x[l][b] = torch.cat([x[l][b], y[st[b]: st[b + 1]]])
            cache.fill(slots, layers - 2, layers - 1, 1)
            for x in held:
                x[-1] = list(x[-2])
            assert cache.rows.tolist() == [x.shape[0] for x in held[0][0]]
            for l in range(layers):
                for b in range(B):
                    n = held[0][l][b].shape[0]
                    if n:
                        back = cache.read(l, _slots(cache, b, range(n)).int())
                        assert all(torch.equal(x.cpu().double(), y[l][b].float().double()) for x, y in zip(back, held))
            for l, (q, turn, out) in enumerate(outs):
                lens = [n if st[b + 1] > st[b] else 0 for b, n in enumerate(cache.rows.tolist())]
                _check(out, *_reference(cache, _turned64(q.double(), turn), lens, layer=l))


def test_a_captured_step_replayed_while_sequences_grow():
    """reserve, attend with a new row, fill and read captured once; every replay is checked against eager calls on a second cache, with eager work on a third between them."""
    import torch
    from paper_2503_08524_amd import PagedCache
    heads, group, hd, B = 4, 2, 128, 3
    for kv in ("i8", "e4m3"):
        caches = [PagedCache(heads * group, heads, hd, 60, 16, B, 20, kv_dtype=kv, n_layers=3, device=DEV) for _ in range(3)]
        g = _generator(4)
        first = torch.tensor([30, 1, 200], dtype=torch.int32, device=DEV)
        k, v = (torch.empty(231, heads, hd, device=DEV).normal_(generator=g) for _ in range(2))
        for c in caches:
            _, slots, _ = c.reserve(first, 231)
            c.append(0, slots, k, v)
        ones = torch.ones(B, dtype=torch.int32, device=DEV)
        q, nk, nv = torch.empty(B, heads * group, hd, device=DEV), torch.empty(B, heads, hd, device=DEV), torch.empty(B, heads, hd, device=DEV)
        starts, slots, positions = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, B))
        out, rk, rv = torch.empty_like(q), torch.empty(3, B, heads, hd, device=DEV), torch.empty(3, B, heads, hd, device=DEV)
        ak = torch.empty(B, heads, hd, device=DEV)
        torch.cuda.synchronize()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            caches[0].reserve(ones, B, starts=starts, slots=slots, positions=positions)
            caches[0].attend(0, q, nk, nv, out=out)
            caches[0].append(2, slots, ak, nv)
            caches[0].fill(slots, 0, 1, 1)
            caches[0].read(0, slots, rk, rv)
        for step in range(12):
            for x in (q, nk, nv, ak):
                x.normal_(generator=g)
            graph.replay()
            caches[2].attend(0, q)                                  # a cache of its own, its own workspace
            torch.cuda.synchronize()
            s2, m2, _ = caches[1].reserve(ones, B)
            want = caches[1].attend(0, q, nk, nv)
            caches[1].append(2, m2, ak, nv)
            caches[1].fill(m2, 0, 1, 1)
            assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip((rk, rv), caches[1].read(0, m2, n_layers=3)))
            assert all(torch.equal(x, y) for x, y in zip(_state(caches[0]), _state(caches[1])))
        assert caches[0].rows.tolist() == [42, 13, 212]


def test_calls_on_another_stream_and_two_handles_at_once():
    import torch
    from paper_2503_08524_amd import PagedCache
    lens = [700, 90, 0, 4000]
    cache, g = _cache(lens, 2, 4, 128, "i8", 16, seed=12)
    shared = dict(k_pages=cache.k_pages, v_pages=cache.v_pages, k_scales=cache.k_scales, v_scales=cache.v_scales, tables=cache.tables, rows=cache.rows, free_pages=cache.free_pages,
                  n_free=cache.n_free)
    other = PagedCache(8, 2, 128, cache.n_pages, 16, 4, cache.max_pages, kv_dtype="i8", device="cuda", **shared)
    q = torch.empty(4, 8, 128, device=DEV).normal_(generator=g)
    slots = _slots(cache, 3, range(1000)).int()
    want, rows = cache.attend(0, q), cache.read(0, slots)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs, reads = ([[None] * 30 for _ in streams] for _ in range(2))
    for i in range(30):
        for c, s, o, r in zip((cache, other), streams, outs, reads):
            with torch.cuda.stream(s):
                o[i], r[i] = c.attend(0, q), c.read(0, slots)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for o in outs for x in o)
    assert all(torch.equal(x, y) for r in reads for z in r for x, y in zip(z, rows))


def test_attention_writes_over_its_queries():
    import torch
    for act, lens in (("f32", [700, 90, 0, 4000]), ("bf16", [2000] * 40)):
        cache, g = _cache(lens, 2, 20, 64, "i8", 16, seed=13)
        q = torch.empty(len(lens), 40, 64, dtype=_types()[act], device=DEV).normal_(generator=g)
        want = cache.attend(0, q)
        assert cache.attend(0, q, out=q) is q and torch.equal(q, want)


def test_refusals():
    import torch
    from paper_2503_08524_amd import D3Error, PagedCache
    cache = PagedCache(4, 2, 64, 8, 16, 3, 4, kv_dtype="i8", n_layers=2, device=DEV)
    half = PagedCache(4, 2, 64, 8, 16, 3, 4, device=DEV)
    assert half.k_scales is None and half.v_scales is None and cache.k_pages.dtype == torch.int8 and tuple(cache.v_pages.shape) == (2, 8, 2, 1, 64, 16)
    slots = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    k = torch.zeros(3, 2, 64, device=DEV)
    scales, codes = torch.zeros(1, 8, 2, 16, device=DEV), torch.zeros(1, 8, 2, 16, 64, dtype=torch.int8, device=DEV)
    for call in (lambda: PagedCache(4, 2, 64, 8, 16, 3, 4, k_scales=scales, device=DEV), lambda: PagedCache(4, 2, 64, 8, 16, 3, 4, kv_dtype="f32", v_scales=scales, device=DEV),
                 lambda: PagedCache(4, 2, 64, 8, 16, 3, 4, kv_dtype="i8", k_scales=scales.half(), device=DEV), lambda: PagedCache(4, 2, 64, 8, 16, 3, 4, kv_dtype="i8", k_scales=scales[:, :7], device=DEV),
                 lambda: PagedCache(4, 2, 64, 8, 16, 3, 4, kv_dtype="e4m3", k_pages=codes, device=DEV), lambda: PagedCache(4, 2, 64, 8, 16, 3, 4, kv_dtype="i8", k_scales=scales.cpu(), device=DEV),
                 lambda: cache.append(0, slots, codes[0, 0, :, :3].transpose(0, 1).contiguous(), codes[0, 0, :, :3].transpose(0, 1).contiguous()),
                 lambda: cache.read(0, slots, k), lambda: cache.read(0, slots, None, k), lambda: cache.read(0, slots, k, k[:2]), lambda: cache.read(0, slots, k, k.half()),
                 lambda: cache.read(0, slots.long()), lambda: cache.read(0, slots, k.double(), k.double()), lambda: cache.read(0, slots, k, k, dtype=torch.float32),
                 lambda: cache.read(0, slots, k, k, n_layers=1), lambda: cache.read(0, slots, dtype=torch.int8), lambda: cache.read(0, slots.cpu(), k, k),
                 lambda: cache.read(0, slots, k.transpose(1, 2).contiguous().transpose(1, 2), k.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros(3 * 128 + 8, device=DEV)
    for call, status, word in ((lambda: cache.read(2, slots), -3, "layers"), (lambda: cache.read(-1, slots), -3, "layers"), (lambda: cache.read(1, slots, n_layers=2), -3, "layers"),
                               (lambda: cache.read(0, slots, wide[1: 385].view(3, 2, 64), wide[1: 385].view(3, 2, 64)), -1, "16 bytes"),
                               (lambda: cache.read(0, slots, n_layers=0), -3, "layers")):
        with pytest.raises(D3Error) as e:
            call()
        assert e.value.status == status and word in str(e.value)
    for n, status, word in (((1 << 28) + 1, -2, "more than one launch"), ((1 << 30) + 1, -1, "2^30"), (-1, -1, "2^30")):
        assert cache.lib.d3_pages_read(cache.handle, 0, 1, n, slots.data_ptr(), k.data_ptr(), k.data_ptr(), 0, 0, 64, 0, None) == status
        assert word in cache.lib.d3_last_error().decode()
    assert cache.lib.d3_pages_read(cache.handle, 0, 1, 3, slots.data_ptr(), k.data_ptr(), k.data_ptr(), 3, 128, 64, 0, None) == -1        # a type of pools only
    torch.cuda.synchronize()
    assert not cache.k_pages.any() and not cache.k_scales.any() and not k.any()

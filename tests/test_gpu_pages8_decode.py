"""Decode steps of the depth schedule on pages of 8 bits: prompts stored, steps, fills and reads, against the decoder in 64 bits that attends over the rows that the pages hold."""
import numpy as np
import pytest

import d3_inputs
from d3_inputs import ModelShape
from tests.test_gpu_pages8 import MOST_CODE, _as_rows, _bits, _quantised, _slots, _state, _values

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
GQA32 = ModelShape("pages8-gqa", L=4, d=512, H=8, H_kv=2, hd=128, F=1376, V=2000, dtype="f32")
GQA = ModelShape("pages8-gqa-bf16", L=4, d=512, H=8, H_kv=2, hd=128, F=1376, V=2000)


def _setup(shape, kv, lengths, G, max_batch=None, cache_kv="f32", extra_pages=2):
    import torch
    from paper_2503_08524_amd import PagedCache, binding
    B, P = len(lengths), max(lengths)
    w = d3_inputs.make_weights(shape, 0)
    dec = binding.Decoder(shape, binding.weights_to_device(shape, w, DEV), max_batch or B, P + G, kv_dtype=cache_kv, device=DEV)
    cache = PagedCache(shape.H, shape.H_kv, shape.hd, sum(-(-(n + G) // 16) for n in lengths) + extra_pages, 16, B, -(-(P + G) // 16), kv_dtype=kv, n_layers=shape.L, device=DEV)
    prompts = d3_inputs.make_prompt(B, P, shape.V, seed=1)
    tok = torch.from_numpy(prompts).to(DEV)
    dec.set_plan(0.8, 1, 0, G)
    dec.prefill_ragged(tok, lengths)
    starts, slots, _ = cache.reserve(torch.tensor(lengths, dtype=torch.int32, device=DEV), sum(lengths))
    at = starts.tolist()
    for b in range(B):
        dec.store_pages(cache, b, slots[at[b]: at[b + 1]])
    return w, dec, cache, slots, at


def _rms(x, gain, eps):
    import torch
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain


def _step64(shape, w, cache, b, token, n, blocks):
    """(logits, {block: (k, v) of the newest row}) of sequence b's token at row n - 1, through `blocks`, over the rows that the pages hold."""
    import torch
    s = shape
    t = {k: torch.from_numpy(v).to(DEV) for k, v in w.items() if k != "layers"}
    x = t["tok_emb"][token]
    j = torch.arange(s.hd // 2, dtype=torch.float64, device=DEV)
    angle = torch.polar(torch.ones_like(j), (n - 1) * s.rope_base ** (-2 * j / s.hd))

    def turn(y):
        z = torch.complex(y[:, : s.hd // 2], y[:, s.hd // 2:]) * angle
        return torch.cat([z.real, z.imag], -1)
    state, at, newest = _state(cache), _slots(cache, b, range(n)), {}
    for l in blocks:
        lw = {k: torch.from_numpy(v).to(DEV) for k, v in w["layers"][l].items()}
        a = _rms(x, lw["attn_norm"], s.eps)
        q, k, v = turn((lw["wq"] @ a).view(s.H, s.hd)), turn((lw["wk"] @ a).view(s.H_kv, s.hd)), (lw["wv"] @ a).view(s.H_kv, s.hd)
        newest[l] = (k, v)
        K, V = (_values(state[i][l, at], state[2 + i][l, at], cache.kv_dtype).repeat_interleave(s.H // s.H_kv, 1) for i in range(2))
        p = torch.softmax(torch.einsum("hd,nhd->hn", q, K) / s.hd ** 0.5, -1)
        x = x + lw["wo"] @ torch.einsum("hn,nhd->hd", p, V).reshape(-1)
        a = _rms(x, lw["mlp_norm"], s.eps)
        x = x + lw["w_down"] @ (torch.nn.functional.silu(lw["w_gate"] @ a) * (lw["w_up"] @ a))
    return t["lm_head"] @ _rms(x, t["final_norm"], s.eps), newest


@pytest.mark.parametrize("kv", ["i8", "e4m3"])
@pytest.mark.parametrize("shape,cache_kv,lengths,logit_atol,row_tol", [(d3_inputs.TINY, "f32", [20, 4, 11], 1e-4, 2e-5), (GQA32, "f32", [37], 1e-4, 2e-5),
                                                                       (GQA, "f16", [150, 20, 1, 77], 2e-2, 1e-2)])
def test_steps_over_held_rows(kv, shape, cache_kv, lengths, logit_atol, row_tol):
    """After every step the logits are those of the rows that the pages hold (the bounds that the suite has for hidden states and logits of fp32 and bf16 models), and the newest rows of the blocks that
    ran are the keys and values of the step, half a step of their codes off at most; the dropped blocks hold the source block's codes."""
    import torch
    G, B = 6, len(lengths)
    w, dec, cache, slots, at = _setup(shape, kv, lengths, G, cache_kv=cache_kv)
    w64 = d3_inputs.weights_as_f64(shape, w)
    # the prompt's rows are the codes of the rows in the context's cache
    for b, n in enumerate(lengths):
        own = slots[at[b]: at[b + 1]].long()
        for i, rows in enumerate((dec.k_cache, dec.v_cache)):
            x = rows[:, b, :, max(lengths) - n: max(lengths)].transpose(1, 2)           # [L][n][H_kv][hd]
            codes, scales = _quantised(x, kv)
            state = _state(cache)
            assert torch.equal(state[i][:, own].cpu(), _bits(codes)) and torch.equal(state[2 + i][:, own].cpu(), scales)
    from paper_2503_08524_amd import binding
    ids = binding.d3_plan_depth(shape.L, 0.8, 1, 0, G)
    forced = d3_inputs.make_prompt(B, G, shape.V, seed=2)
    ones, nxt, logits = torch.ones(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, shape.V, device=DEV)
    for i in range(1, G):
        starts, new, _ = cache.reserve(ones, B)
        dec.decode_step_paged(cache, torch.from_numpy(np.ascontiguousarray(forced[:, i])).to(DEV), i, nxt, logits=logits, starts=starts)
        dec.fill_missing_paged(cache, new, i)
        blocks = [int(x) for x in ids[2][i] if x >= 0]
        state = _state(cache)
        for b, n in enumerate(lengths):
            want, newest = _step64(shape, w64, cache, b, int(forced[b, i]), n + i, blocks)
            assert (logits[b].double() - want).abs().max() <= logit_atol
            row = _slots(cache, b, [n + i - 1])
            for l, kv64 in newest.items():
                for j, x in enumerate(kv64):
                    got, a = _values(state[j][l, row], state[2 + j][l, row], kv)[0], x.abs().amax(-1, keepdim=True)
                    half = a / 254 if kv == "i8" else torch.maximum(2.0 ** -4 * x.abs(), a * 2.0 ** -10 / 448)
                    assert ((got - x).abs() <= half * (1 + 2 * row_tol) + row_tol * a).all()
            first, dropped = int(ids[1][i]), shape.L - len(blocks)
            src = first - 1 if first > 0 else first + dropped
            for x in state:
                for l in range(first, first + dropped):
                    assert torch.equal(x[l, row], x[src, row])


def test_a_captured_step_on_pages_of_8_bits():
    """Reserve, step and fill captured once, replayed with eager steps of another cache between the replays: tokens and pages are those of eager calls."""
    import torch
    shape, lengths, G = d3_inputs.TINY, [18, 5], 6
    _, dec, cache, _, _ = _setup(shape, "i8", lengths, G)
    _, dec2, cache2, _, _ = _setup(shape, "i8", lengths, G)
    ones, tok = torch.ones(2, dtype=torch.int32, device=DEV), torch.tensor([3, 7], dtype=torch.int32, device=DEV)
    out, slots, starts = torch.zeros_like(tok), torch.empty(2, dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        cache.reserve(ones, 2, starts=starts, slots=slots)
        dec.decode_step_paged(cache, tok, 3, out, starts=starts)
        dec.fill_missing_paged(cache, slots, 3)
    want = torch.zeros_like(tok)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        s2, m2, _ = cache2.reserve(ones, 2)
        dec2.decode_step_paged(cache2, tok, 3, want, starts=s2)
        dec2.fill_missing_paged(cache2, m2, 3)
        assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip(_state(cache), _state(cache2)))
        tok.copy_(out)


def test_rows_leave_the_pages_and_come_back():
    """A sequence's rows read out, its pages given back and taken by others, its rows appended again elsewhere: the next step is the one it would have made."""
    import torch
    shape, lengths, G = GQA32, [40, 25], 4
    _, dec, cache, _, _ = _setup(shape, "e4m3", lengths, G, extra_pages=6)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    before = [x.clone() for x in _state(cache)]
    old = _slots(cache, 0, range(40))
    k, v = cache.read(0, old.int(), n_layers=shape.L)
    cache.reserve(ints(-1, 0), 1)
    cache.reserve(ints(0, 20), 20)                                  # sequence 1 takes some of the pages
    cache.rows[1:].fill_(25)                                        # (and forgets what it did with them)
    _, slots, _ = cache.reserve(ints(40, 0), 40)
    cache.append(0, slots[:40], k, v)
    new = _slots(cache, 0, range(40))
    for was, now in zip(before[:2], _state(cache)[:2]):
        assert torch.equal(was[:, old], now[:, new])
    for was, now in zip(before[2:], _state(cache)[2:]):            # a scale is rounded once more
        assert ((was[:, old] - now[:, new]).abs() <= 2.0 ** -23 * was[:, old]).all()
    tok, nxt, logits = ints(11, 12), torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, shape.V, device=DEV)
    starts, _, _ = cache.reserve(ints(1, 0), 1)
    dec.decode_step_paged(cache, tok, 1, nxt, logits=logits, starts=starts)
    _, dec2, cache2, _, _ = _setup(shape, "e4m3", lengths, G)
    want, nxt2 = torch.zeros_like(logits), torch.zeros_like(nxt)
    starts, _, _ = cache2.reserve(ints(1, 0), 1)
    dec2.decode_step_paged(cache2, tok, 1, nxt2, logits=want, starts=starts)
    # scales off by 2^-23 and their sums: far inside what two sums of fp32 products over these widths differ by
    assert (logits[0] - want[0]).abs().max() <= 1e-4 and int(nxt[1]) == 12 and int(nxt2[1]) == 12


def test_refusals():
    import torch
    from paper_2503_08524_amd import D3Error, PagedCache, binding
    shape = d3_inputs.TINY
    dec = binding.Decoder(shape, binding.weights_to_device(shape, d3_inputs.make_weights(shape, 0), DEV), 2, 32, kv_dtype="f32", device=DEV)
    dec.set_plan(0.9, 1, 0, 4)
    tok, out = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    for change in (dict(kv_dtype="f16"), dict(kv_dtype="i8", n_layers=3), dict(kv_dtype="i8", head_dim=128), dict(kv_dtype="e4m3", n_heads=8)):
        args = {**dict(n_heads=shape.H, n_kv_heads=shape.H_kv, head_dim=shape.hd, n_pages=4, page_rows=16, max_batch=2, max_pages=2, n_layers=shape.L, device=DEV), **change}
        with pytest.raises(D3Error) as e:
            dec.decode_step_paged(PagedCache(**args), tok, 1, out)
        assert e.value.status == -2
    for kv in MOST_CODE:                                            # a context's own cache is never of 8 bits
        with pytest.raises((D3Error, KeyError)):
            binding.Decoder(shape, dec.weights, 1, 32, kv_dtype=kv, device=DEV)
    assert _as_rows(PagedCache(4, 4, 64, 4, 16, 2, 2, kv_dtype="i8", device=DEV).k_scales).sum() == 0

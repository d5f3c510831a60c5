"""Sequences that got no row: refused, paused or ended ones beside those that go on, in the attention on pages and in decode steps; sequences of different ages."""
import math

import numpy as np
import pytest

import d3_inputs
from tests import test_gpu_paged_decode as steps
from tests import test_gpu_pages as pages

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _ints(*x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("lens,heads,group,hd,kv,act,page_rows", [
    ([40, 1, 300, 16, 700, 33], 2, 4, 128, "f16", "f32", 16), ([17, 200, 64, 5], 2, 20, 64, "f32", "bf16", 32), ([640, 640], 32, 1, 128, "f16", "f16", 16),
    ([(37 * b) % 91 for b in range(200)], 2, 2, 128, "f16", "f32", 16), ([1 + (31 * b) % 60 for b in range(300)], 8, 2, 64, "f32", "f32", 16)])
def test_attention_of_the_sequences_that_got_a_row(lens, heads, group, hd, kv, act, page_rows):
    """All, every other one, one and none of them; the others' rows stay as they were and their outputs are 0, also in a captured launch whose starts change."""
    import torch
    B = len(lens)
    cache, g = pages._cache(lens, heads, group, hd, kv, page_rows, seed=B)
    t = pages._types()[act]
    q = torch.empty(B, heads * group, hd, dtype=t, device=DEV).normal_(generator=g)
    k, v = (torch.empty(B, heads, hd, dtype=t, device=DEV).normal_(generator=g) for _ in range(2))
    cs = pages._angles([max(n - 1, 0) for n in lens], hd)
    b = np.arange(B)
    starts, out = torch.zeros(B + 1, dtype=torch.int32, device=DEV), torch.empty_like(q)
    pools = cache.k_pages, cache.v_pages
    first = [p.clone() for p in pools]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.attend(0, q, k, v, rope_cs=cs, out=out, starts=starts)
    for got in (b % 2 == 0, b == B - 1, b < 0, b >= 0, b % 2 == 1):
        starts[1:] = torch.from_numpy(np.cumsum(got)).to(DEV)
        n = [x if y else 0 for x, y in zip(lens, got)]
        for pool, was in zip(pools, first):
            pool.copy_(was)
        graph.replay()
        torch.cuda.synchronize()
        want = [pages._as_rows(cache, p) for p in (cache.k_pages, cache.v_pages)]
        live = [x for x in range(B) if n[x]]
        written = torch.zeros(cache.n_pages * page_rows, dtype=torch.bool, device=DEV)
        if live:
            at = torch.cat([pages._slots(cache, x, [n[x] - 1]) for x in live])
            written[at] = True
            for rows, x in zip(want, (pages._turned(k.double(), cs), v.double())):
                err = (rows[0, at].double() - x[live]).abs()
                assert (err <= torch.finfo(rows.dtype).eps / 2 * x[live].abs() + 3 * 2.0 ** -24 * x[live].abs().amax() * 2 + 2.0 ** -25).all()
        for rows, pool, was in zip(want, pools, first):
            pool.copy_(was)
            assert torch.equal(rows[:, ~written], pages._as_rows(cache, pool)[:, ~written])
        eager = cache.attend(0, q, k, v, rope_cs=cs, starts=starts)
        assert torch.equal(out, eager)
        pages._check(out, *pages._reference(cache, pages._turned(q.double(), cs), n))
        assert not out[torch.from_numpy(~got).to(DEV)].any()
    # without new rows: those of the others are still not read
    got = b % 2 == 0
    starts[1:] = torch.from_numpy(np.cumsum(got)).to(DEV)
    pages._check(cache.attend(0, q, starts=starts), *pages._reference(cache, q.double(), [x if y else 0 for x, y in zip(lens, got)]))


def _own_logits(dec, prompts, lengths, forced, fill):
    """Logits [step][sequence] of the context's own cache, all sequences in step; step 0 the prompt's."""
    import torch
    B, n = prompts.shape[0], forced.shape[0]
    logits, nxt = torch.zeros(B, dec.shape.V, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    dec.prefill_ragged(prompts, lengths, logits=logits)
    out = [logits.clone()]
    for i in range(1, n):
        dec.decode_step(forced[i], i, nxt, logits=logits)
        if fill:
            dec.fill_missing_kv(dec.n_ctx - 1, dec.n_ctx)
        out.append(logits.clone())
    dec.prefill_ragged(prompts, lengths)                             # as it was, for the rows of the prompts
    return out


@pytest.mark.parametrize("captured", [False, True])
def test_a_refused_sequence_keeps_its_rows_and_its_token_and_goes_on(captured):
    """A pool that runs out: of three sequences one goes on, the others are refused for pages until that one ends; then they continue as if nothing had been."""
    import torch
    lengths, G = [16, 16, 15], 8
    w = d3_inputs.make_weights(steps.GQA, 0)
    dec = steps._decoder(steps.GQA, w, 3, 40, "f32")
    dec.set_plan(1.0, 0, 0, G)
    prompts = torch.from_numpy(d3_inputs.make_prompt(3, 16, steps.GQA.V, seed=11)).to(DEV)
    forced = torch.from_numpy(d3_inputs.make_prompt(G, 3, steps.GQA.V, seed=12)).to(DEV)
    want = _own_logits(dec, prompts, lengths, forced, fill=False)
    cache = steps._pages(dec, 4, 3, 40)
    steps._admit(dec, cache, lengths)
    added, tok, logits = _ints(1, 1, 1), torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, steps.GQA.V, device=DEV)
    starts, slots, positions = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (4, 3, 3))

    def step():
        cache.reserve(added, 3, starts=starts, slots=slots, positions=positions)
        dec.decode_step_paged(cache, tok, 1, tok, logits=logits, starts=starts)
    if captured:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step()
        step = graph.replay
    done = [0, 0, 0]                                                # steps that each sequence has taken
    for turn, (ask, granted) in enumerate([((1, 1, 1), (1, 0, 1)), ((1, 1, 1), (1, 0, 0)), ((1, 1, 1), (1, 0, 0)), ((-1, 1, 1), (0, 1, 1)), ((0, 1, 1), (0, 1, 1)),
                                           ((0, 0, 1), (0, 0, 1)), ((0, 1, 1), (0, 1, 1))]):
        added.copy_(_ints(*ask))
        tok.copy_(torch.stack([forced[done[b] + 1, b] for b in range(3)]))
        fed, held, before = tok.tolist(), cache.rows.tolist(), [pages._as_rows(cache, p) for p in (cache.k_pages, cache.v_pages)]
        step()
        torch.cuda.synchronize()
        assert np.diff(starts.tolist()).tolist() == list(granted), turn
        for b in range(3):
            if granted[b]:
                done[b] += 1
                assert (logits[b] - want[done[b]][b]).abs().max() < 1e-4, (turn, b)
                assert cache.rows[b] == held[b] + 1 == lengths[b] + done[b]
            else:
                assert int(tok[b]) == fed[b]
                if ask[b] >= 0 and held[b]:
                    at = pages._slots(cache, b, range(held[b]))
                    assert cache.rows[b] == held[b] and all(torch.equal(x[:, at], pages._as_rows(cache, p)[:, at]) for x, p in zip(before, (cache.k_pages, cache.v_pages)))
    assert done == [3, 3, 5]


def test_a_sequence_at_the_end_of_its_table_sits_out_and_its_token_is_handed_on():
    """Refused for its table's room, which the count of lacking pages does not show; and the tokens of idle sequences in a tok_out that is not tok_in."""
    import torch
    w = d3_inputs.make_weights(steps.GQA, 0)
    dec = steps._decoder(steps.GQA, w, 2, 40, "f16")
    dec.set_plan(1.0, 0, 0, 6)
    dec.prefill_ragged(torch.from_numpy(d3_inputs.make_prompt(2, 32, steps.GQA.V, seed=13)).to(DEV), [32, 20])
    cache = steps._pages(dec, 10, 2, 32)
    steps._admit(dec, cache, [32, 20])
    rows = [pages._as_rows(cache, p)[:, pages._slots(cache, 0, range(32))] for p in (cache.k_pages, cache.v_pages)]
    tok, nxt = _ints(77, 78), _ints(-1, -1)
    for i in range(3):
        starts, _, _ = cache.reserve(_ints(1, 1), 2)
        assert starts.tolist() == [0, 0, 1] and cache.n_free[1] == 0
        dec.decode_step_paged(cache, tok, 1, nxt, starts=starts)
        assert nxt[0] == 77 and 0 <= nxt[1] < steps.GQA.V
    assert cache.rows.tolist() == [32, 23]
    for was, p in zip(rows, (cache.k_pages, cache.v_pages)):
        assert torch.equal(was, pages._as_rows(cache, p)[:, pages._slots(cache, 0, range(32))])


def test_sequences_of_different_ages_step_in_groups():
    """A shrinking depth, two sequences three steps ahead of the other two: a reserve, a step and a fill for each group.  Logits are those of the context's own cache, where all are in step."""
    import torch
    lengths, G = [30, 9, 16, 22], 9
    w = d3_inputs.make_weights(steps.GQA, 0)
    dec = steps._decoder(steps.GQA, w, 4, 50, "f32")
    dec.set_plan(0.8, 1, 0, G)
    kept = steps.dec_keep(steps.GQA.L, 0.8, 1, G).tolist()
    assert kept[1] > kept[4] > kept[8]
    prompts = torch.from_numpy(d3_inputs.make_prompt(4, 30, steps.GQA.V, seed=14)).to(DEV)
    forced = torch.from_numpy(d3_inputs.make_prompt(G, 4, steps.GQA.V, seed=15)).to(DEV)
    want = _own_logits(dec, prompts, lengths, forced, fill=True)
    cache = steps._pages(dec, 20, 4, 50)
    steps._admit(dec, cache, lengths)
    tok, logits = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(4, steps.GQA.V, device=DEV)
    age = [0, 0, 0, 0]
    for turn in range(1, G + 3):
        for group in ((0, 1), (2, 3)):
            step = turn if group == (0, 1) else turn - 3
            if not 1 <= step < G:
                continue
            starts, slots, _ = cache.reserve(_ints(*(int(b in group) for b in range(4))), 2)
            for b in group:
                tok[b] = forced[step, b]
            others = tok.clone()
            dec.decode_step_paged(cache, tok, step, tok, logits=logits, starts=starts)
            dec.fill_missing_paged(cache, slots, step)
            for b in range(4):
                if b in group:
                    age[b] += 1
                    assert (logits[b] - want[step][b]).abs().max() < 1e-4, (turn, b)
                else:
                    assert tok[b] == others[b]
    assert age == [G - 1] * 4 and cache.rows.tolist() == [n + G - 1 for n in lengths]


def test_starts_that_are_refused():
    import torch
    w = d3_inputs.make_weights(steps.GQA, 0)
    dec = steps._decoder(steps.GQA, w, 2, 32, "f16")
    dec.set_plan(1.0, 0, 0, 4)
    cache = steps._pages(dec, 10, 4, 32)
    tok, q = _ints(1, 2), torch.zeros(2, 8, 128, device=DEV)
    for starts in (_ints(0, 1), _ints(0, 1, 2).long(), torch.zeros(3, dtype=torch.int32), _ints(0, 0, 1, 1, 2, 2)[::2]):
        for call in (lambda: dec.decode_step_paged(cache, tok, 1, tok, starts=starts), lambda: cache.attend(0, q, starts=starts)):
            with pytest.raises(ValueError):
                call()
    assert cache.attend(0, q, scale=1.0, starts=_ints(0, 1, 2, 2)).abs().max() == 0 and not math.isnan(float(q.sum()))

"""The decode path on a paged cache (d3_store_pages, d3_decode_step_paged, d3_fill_missing_paged) against the path on the context's own cache and the oracle."""
import numpy as np
import pytest

import d3_inputs
from d3_inputs import ModelShape
from tests import helpers

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
GQA = ModelShape("paged-gqa", L=4, d=512, H=8, H_kv=2, hd=128, F=1376, V=2000)
MHA64 = ModelShape("paged-mha64", L=4, d=256, H=4, H_kv=4, hd=64, F=704, V=1024)


def _decoder(shape, w_np, B, max_seq, kv):
    from paper_2503_08524_amd import binding
    return binding.Decoder(shape, binding.weights_to_device(shape, w_np, DEV), B, max_seq, kv_dtype=kv, device=DEV)


def _pages(dec, n_pages, max_batch, max_rows, page_rows=16):
    from paper_2503_08524_amd import PagedCache
    s = dec.shape
    return PagedCache(s.H, s.H_kv, s.hd, n_pages, page_rows, max_batch, -(-max_rows // page_rows), kv_dtype=dec.kv_dtype, n_layers=s.L, device=DEV)


def _admit(dec, cache, lengths):
    """The prompts that dec holds, into pages of sequences 0 .. B - 1."""
    import torch
    starts, slots, _ = cache.reserve(torch.tensor(lengths, dtype=torch.int32, device=DEV), sum(lengths))
    at = starts.tolist()
    for b in range(len(lengths)):
        dec.store_pages(cache, b, slots[at[b]: at[b + 1]])


@pytest.mark.parametrize("shape,kv,B,lengths", [(d3_inputs.TINY, "f32", 1, None), (d3_inputs.TINY, "f32", 3, [20, 4, 11]), (GQA, "f16", 1, None), (GQA, "f32", 5, None),
                                                (GQA, "f16", 4, [150, 20, 1, 77]), (MHA64, "f16", 3, [33, 32, 5])])
def test_paged_steps_agree_with_the_oracle(shape, kv, B, lengths):
    """Prompts through the context's cache, their rows stored into pages, decode steps with a shrinking depth and the fill on pages; each sequence has its own length."""
    import torch
    P, G, alpha, start = (max(lengths) if lengths else 40), 8, 0.8, 1
    w = d3_inputs.make_weights(shape, 0)
    prompts = d3_inputs.make_prompt(B, P, shape.V, seed=1)
    forced = d3_inputs.make_prompt(B, G, shape.V, seed=2)[:, : G - 1]
    _, gens = helpers.oracle_generate(shape, w, prompts, G, alpha, start, forced=forced, lengths=lengths)
    dec = _decoder(shape, w, B, P + G, kv)
    dec.set_plan(alpha, start, 0, G)
    own = lengths or [P] * B
    cache = _pages(dec, sum(-(-(n + G) // 16) for n in own) + 2, B, P + G)
    tok = torch.from_numpy(prompts).to(DEV)
    logits, hid = torch.zeros(B, shape.V, device=DEV), torch.zeros(shape.L + 1, B, shape.d, device=DEV)
    cur = dec.prefill_ragged(tok, lengths, logits=logits, hidden_dump=hid) if lengths else dec.prefill(tok, logits=logits, hidden_dump=hid)
    got = {"tokens": [cur.cpu().numpy().copy()], "logits": [logits.cpu().numpy()], "hidden": [hid.cpu().numpy()]}
    _admit(dec, cache, own)
    was = dec.n_ctx
    ones, nxt = torch.ones(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    for i in range(1, G):
        _, slots, positions = cache.reserve(ones, B)
        assert positions.tolist() == [n + i - 1 for n in own]
        kept = int(dec_keep(shape.L, alpha, start, G)[i])
        hid = torch.zeros(kept + 1, B, shape.d, device=DEV)
        dec.decode_step_paged(cache, torch.from_numpy(np.ascontiguousarray(forced[:, i - 1])).to(DEV), i, nxt, logits=logits, hidden_dump=hid)
        dec.fill_missing_paged(cache, slots, i)
        got["tokens"].append(nxt.cpu().numpy().copy()); got["logits"].append(logits.cpu().numpy().copy()); got["hidden"].append(hid.cpu().numpy())
    assert dec.n_ctx == was
    tight = dict(check_tokens="all", logit_atol=1e-4, hidden_tol=1e-5) if shape.dtype == "f32" else {}
    helpers.compare(got, gens, G, **tight)


def dec_keep(L, alpha, start, G):
    from paper_2503_08524_amd import binding
    return binding.d3_plan_depth(L, alpha, start, 0, G)[0]


def test_paged_rows_and_fill_are_those_of_the_contexts_own_cache():
    """Same steps on both caches: every row of every layer, the dropped ones' among them, up to the attention's rounding."""
    import torch
    B, P, G = 4, 50, 6
    w = d3_inputs.make_weights(GQA, 0)
    dec = _decoder(GQA, w, B, P + G, "f32")
    dec.set_plan(0.7, 1, 0, G)
    cache = _pages(dec, 40, B, P + G)
    dec.prefill(torch.from_numpy(d3_inputs.make_prompt(B, P, GQA.V, seed=3)).to(DEV))
    _admit(dec, cache, [P] * B)
    forced = torch.from_numpy(d3_inputs.make_prompt(G, B, GQA.V, seed=4)).to(DEV)
    ones = torch.ones(B, dtype=torch.int32, device=DEV)
    a, b = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    la, lb = torch.zeros(B, GQA.V, device=DEV), torch.zeros(B, GQA.V, device=DEV)
    for i in range(1, G):
        dec.decode_step(forced[i], i, a, logits=la)
        dec.fill_missing_kv(dec.n_ctx - 1, dec.n_ctx)
        _, slots, _ = cache.reserve(ones, B)
        dec.decode_step_paged(cache, forced[i], i, b, logits=lb)
        dec.fill_missing_paged(cache, slots, i)
        assert torch.equal(a, b) and (la - lb).abs().max() < 1e-4
    n = P + G - 1
    p = torch.arange(n, device=DEV)
    for s in range(B):
        page = cache.tables[s].long()[p // 16]
        k = cache.k_pages[:, page, :, p % 16]                     # [n][L][H_kv][hd]
        v = cache.v_pages[:, page, :, p % 16 // 4, :, p % 4]
        for got, own in ((k, dec.k_cache), (v, dec.v_cache)):
            want = own[:, s, :, :n].permute(2, 0, 1, 3)
            assert torch.equal(got[:P], want[:P])                 # the prompt's are copies
            assert (got - want).abs().max() <= 1e-4


def test_sequences_come_and_go_and_idle_ones_do_not_matter():
    """A batch with an idle place, and one whose request ends and is followed by another: the others' tokens are those of a batch without them."""
    import torch
    w = d3_inputs.make_weights(GQA, 0)
    dec = _decoder(GQA, w, 4, 64, "f16")
    dec.set_plan(1.0, 0, 0, 40)
    lengths = [40, 17, 30]
    prompts = torch.from_numpy(d3_inputs.make_prompt(3, 40, GQA.V, seed=5)).to(DEV)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)

    def run(alone):
        cache = _pages(dec, 12 if not alone else 40, 4, 64)
        first = dec.prefill_ragged(prompts, lengths).clone()
        starts, slots, _ = cache.reserve(ints(40, 17, 0, 0), 57)
        dec.store_pages(cache, 0, slots[:40]); dec.store_pages(cache, 1, slots[40:])
        tok, out = torch.zeros(4, dtype=torch.int32, device=DEV), []
        tok[:2] = first[:2]
        for i in range(1, 12):
            if i == 4 and not alone:                              # sequence 1 ends; sequence 2's prompt takes place 3
                starts, slots, _ = cache.reserve(ints(0, -1, 0, 30), 30)
                assert starts.tolist() == [0, 0, 0, 0, 30]
                dec.store_pages(cache, 2, slots)
                tok[3] = first[2]
            live = ints(1, 1 if i < 4 or alone else 0, 0, 1 if i >= 4 and not alone else 0)
            cache.reserve(live, 4)
            nxt = torch.zeros_like(tok)
            dec.decode_step_paged(cache, tok, i, nxt)
            tok = nxt
            out.append(tok.tolist())
        assert cache.n_free[1].item() == 0
        return [o[0] for o in out], [o[1] for o in out[:3]], [o[3] for o in out[3:]]
    with_others, alone = run(False), run(True)
    assert with_others[0] == alone[0] and with_others[1] == alone[1]
    # the newcomer's tokens are those it gets on the context's own cache
    cur = dec.prefill(prompts[2:, 10:].contiguous())
    want = []
    for i in range(1, 9):
        nxt = torch.zeros_like(cur)
        dec.decode_step(cur, i, nxt)
        cur = nxt
        want.append(int(cur))
    agree = sum(x == y for x, y in zip(with_others[2], want))
    assert agree >= 1 and (agree == 8 or with_others[2][:agree] == want[:agree])


def test_a_whole_captured_step_equals_eager_ones():
    import torch
    B, P, G = 3, 30, 14
    w = d3_inputs.make_weights(GQA, 0)
    dec = _decoder(GQA, w, B, P + G, "f16")
    dec.set_plan(1.0, 0, 0, G)
    prompts = torch.from_numpy(d3_inputs.make_prompt(B, P, GQA.V, seed=6)).to(DEV)
    ones = torch.ones(B, dtype=torch.int32, device=DEV)
    first = dec.prefill(prompts).clone()
    caches = [_pages(dec, 20, B, P + G) for _ in range(2)]
    for c in caches:
        _admit(dec, c, [P] * B)
    tok, logits = first.clone(), torch.zeros(B, GQA.V, device=DEV)
    starts, slots, positions = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, B))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        caches[0].reserve(ones, B, starts=starts, slots=slots, positions=positions)
        dec.decode_step_paged(caches[0], tok, 1, tok, logits=logits)          # the next token takes the place of this one
    eager, elog, nxt = first.clone(), torch.zeros_like(logits), torch.zeros_like(first)
    for i in range(1, G):
        graph.replay()
        torch.cuda.synchronize()
        caches[1].reserve(ones, B)
        dec.decode_step_paged(caches[1], eager, 1, nxt, logits=elog)
        eager = nxt.clone()
        assert torch.equal(tok, eager) and torch.equal(logits, elog)
        assert torch.equal(caches[0].k_pages, caches[1].k_pages) and torch.equal(caches[0].v_pages, caches[1].v_pages)


def test_refusals():
    import torch
    from paper_2503_08524_amd import D3Error, PagedCache
    from paper_2503_08524_amd.binding import D3_FILL_RECOMPUTE
    w = d3_inputs.make_weights(GQA, 0)
    dec = _decoder(GQA, w, 2, 32, "f16")
    cache = _pages(dec, 10, 4, 32)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    tok = ints(1, 2)

    def refused(status, word, call):
        with pytest.raises(D3Error) as e:
            call()
        assert e.value.status == status and word in str(e.value), str(e.value)
    refused(-4, "no plan", lambda: dec.decode_step_paged(cache, tok, 1, tok.clone()))
    refused(-4, "no plan", lambda: dec.fill_missing_paged(cache, tok, 1))
    refused(-4, "no prompt", lambda: dec.store_pages(cache, 0, tok))
    dec.set_plan(0.5, 1, 0, 4)
    dec.prefill_ragged(torch.zeros(2, 9, dtype=torch.int32, device=DEV), [9, 4])
    for step in (-1, 4):
        refused(-3, "outside the plan", lambda: dec.decode_step_paged(cache, tok, step, tok.clone()))
        refused(-3, "outside the plan", lambda: dec.fill_missing_paged(cache, tok, step))
    refused(-2, "B must be", lambda: dec.decode_step_paged(cache, ints(1, 2, 3), 1, ints(0, 0, 0)))
    refused(-3, "sequence 2", lambda: dec.store_pages(cache, 2, tok))
    refused(-3, "rows", lambda: dec.store_pages(cache, 1, tok, row_begin=3))
    refused(-3, "rows", lambda: dec.store_pages(cache, 1, tok, row_begin=-1))
    for other in (PagedCache(8, 2, 128, 4, 16, 2, 2, n_layers=3, device=DEV), PagedCache(8, 4, 128, 4, 16, 2, 2, n_layers=4, device=DEV), PagedCache(8, 2, 64, 4, 16, 2, 2, n_layers=4, device=DEV)):
        refused(-2, "the context's", lambda: dec.decode_step_paged(other, tok, 1, tok.clone()))
        refused(-2, "the context's", lambda: dec.store_pages(other, 0, tok))
    f32 = PagedCache(8, 2, 128, 4, 16, 2, 2, n_layers=4, kv_dtype="f32", device=DEV)
    refused(-2, "type", lambda: dec.decode_step_paged(f32, tok, 1, tok.clone()))
    dec.store_pages(f32, 1, ints(0, 1, 2, 3))                      # rows may be stored into a wider type
    assert torch.equal(f32.k_pages[:, 0, :, :4], dec.k_cache[:, 1, :, 5:9].float())
    dec.set_fill_mode(D3_FILL_RECOMPUTE)
    refused(-4, "RECOMPUTE", lambda: dec.decode_step_paged(cache, tok, 1, tok.clone()))
    with pytest.raises(ValueError):
        dec.decode_step_paged(cache, tok, 1, tok[:1])
    with pytest.raises(ValueError):
        dec.store_pages(cache, 0, tok.long())


@pytest.mark.parametrize("order", [[5, 4, 3, 2, 1, 0], [3, 5, 0, 4, 1, 2]])
@pytest.mark.parametrize("kv", ["f16", "f32"])
def test_steps_in_any_order_on_pages_that_held_other_rows(order, kv):
    """Each step followed by the fill of its rows: a block that an earlier step dropped finds the rows it attends over.  Pools of NaN (what another request left may be anything) against
    the context's own cache with a plan of the same depths in that order."""
    import math
    import torch
    from paper_2503_08524_amd import binding
    B, P, lengths = 3, 21, [21, 16, 6]
    w = d3_inputs.make_weights(GQA, 0)
    dec = _decoder(GQA, w, B, P + 8, kv)
    keep, drop, _ = binding.d3_plan_depth(GQA.L, 0.75, 1, 0, 6)
    assert len(set(keep.tolist())) >= 3
    prompts = torch.from_numpy(d3_inputs.make_prompt(B, P, GQA.V, seed=31)).to(DEV)
    forced = torch.from_numpy(d3_inputs.make_prompt(6, B, GQA.V, seed=32)).to(DEV)
    dec.set_plan_table(np.concatenate([[GQA.L], keep[order]]), np.concatenate([[0], drop[order]]))
    logits, nxt, want = torch.zeros(B, GQA.V, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV), []
    dec.prefill_ragged(prompts, lengths)
    for n in range(6):
        dec.decode_step(forced[n], n + 1, nxt, logits=logits)
        dec.fill_missing_kv(dec.n_ctx - 1, dec.n_ctx)
        want.append(logits.clone())
    dec.set_plan(0.75, 1, 0, 6)
    dec.prefill_ragged(prompts, lengths)
    cache = _pages(dec, 9, B, P + 8)
    cache.k_pages.fill_(math.nan)
    cache.v_pages.fill_(math.nan)
    _admit(dec, cache, lengths)
    for n, step in enumerate(order):
        starts, slots, _ = cache.reserve(torch.ones(B, dtype=torch.int32, device=DEV), B)
        dec.decode_step_paged(cache, forced[n], step, nxt, logits=logits, starts=starts)
        dec.fill_missing_paged(cache, slots, step)
        # fp32 rows differ by the order of sums; an fp16 row that is rounded the other way for that is 2^-11 of itself off
        assert (logits - want[n]).abs().max() < (1e-4 if kv == "f32" else helpers.LOGIT_ATOL), (n, step)


def test_rows_go_into_pages_of_a_handle_with_other_query_heads():
    """Rows know KV heads only: storing and filling need the context's layers, KV heads and head_dim, as documented; a step needs its query heads too."""
    import torch
    from paper_2503_08524_amd import D3Error, PagedCache
    dec = _decoder(GQA, d3_inputs.make_weights(GQA, 0), 1, 32, "f16")
    dec.set_plan(0.5, 1, 0, 4)
    tok = dec.prefill(torch.from_numpy(d3_inputs.make_prompt(1, 9, GQA.V, seed=8)).to(DEV))
    caches = [PagedCache(heads, GQA.H_kv, GQA.hd, 3, 16, 1, 2, n_layers=GQA.L, device=DEV) for heads in (GQA.H, GQA.H_kv)]
    for cache in caches:
        _admit(dec, cache, [9])
        dec.fill_missing_paged(cache, torch.arange(3, 5, dtype=torch.int32, device=DEV), 2)
    assert torch.equal(caches[0].k_pages, caches[1].k_pages) and torch.equal(caches[0].v_pages, caches[1].v_pages) and caches[0].k_pages.any()
    with pytest.raises(D3Error) as e:
        dec.decode_step_paged(caches[1], tok, 1, tok)
    assert e.value.status == -2 and "heads" in str(e.value)


@pytest.mark.parametrize("kv,tight", [("f32", 1e-4), ("f16", helpers.LOGIT_ATOL)])
def test_a_newcomer_on_recycled_pages_has_the_logits_of_its_own_run(kv, tight):
    """A sequence takes the place and the pages of one that ended; forced tokens, and its logits in every step are those of the context's own cache, which it has to itself there."""
    import torch
    w = d3_inputs.make_weights(GQA, 0)
    dec = _decoder(GQA, w, 3, 64, kv)
    dec.set_plan(1.0, 0, 0, 12)
    lengths = [40, 37, 30]
    prompts = torch.from_numpy(d3_inputs.make_prompt(3, 40, GQA.V, seed=41)).to(DEV)
    forced = torch.from_numpy(d3_inputs.make_prompt(12, 3, GQA.V, seed=42)).to(DEV)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    logits, nxt = torch.zeros(2, GQA.V, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    cache = _pages(dec, 7, 2, 64)                                  # seven pages for 40 + 8 and 37 + 3 rows: the newcomer's are the ended one's
    dec.prefill_ragged(prompts, lengths)
    starts, slots, _ = cache.reserve(ints(40, 37), 77)
    dec.store_pages(cache, 0, slots[:40])
    dec.store_pages(cache, 1, slots[40:])
    former, got = set(cache.tables[1, :3].tolist()), []
    for i in range(11):
        if i == 3:
            starts, slots, _ = cache.reserve(ints(0, -1), 1)
            starts, slots, _ = cache.reserve(ints(0, 30), 30)
            assert starts.tolist() == [0, 0, 30] and set(cache.tables[1, :2].tolist()) <= former
            dec.store_pages(cache, 2, slots)
        starts, slots, positions = cache.reserve(ints(1, 1), 2)
        assert positions.tolist() == [40 + i, 37 + i if i < 3 else 30 + i - 3]
        tok = torch.stack([forced[i, 0], forced[i, 1] if i < 3 else forced[i - 3, 2]])
        dec.decode_step_paged(cache, tok, 1, nxt, logits=logits, starts=starts)
        got.append(logits.clone())
    own = torch.zeros(1, GQA.V, device=DEV)
    for b, mine in ((0, [x[0] for x in got]), (1, [x[1] for x in got[:3]]), (2, [x[1] for x in got[3:]])):
        dec.prefill(prompts[b:b + 1, 40 - lengths[b]:].contiguous())
        for i, x in enumerate(mine):
            dec.decode_step(forced[i, b:b + 1].contiguous(), i + 1, nxt[:1], logits=own)
            assert (x - own[0]).abs().max() < tight, (b, i)

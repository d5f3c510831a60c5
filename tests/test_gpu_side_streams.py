"""Handles made on a stream that is not the null stream, from memory that work queued on it still writes: torch's allocator hands a freed block on to the same stream at once."""
import numpy as np
import pytest

import d3_inputs
from tests import test_gpu_paged_decode as steps
from tests import test_gpu_pages as pages

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _busy_block(n_bytes):
    """Work of some milliseconds queued on the current stream that ends by writing ones to a block of n_bytes, which is then free for the stream's next allocation."""
    import torch
    a = torch.ones(4096, 4096, device=DEV)
    for _ in range(20):
        a = (a @ a) * 2.0 ** -12
    block = torch.empty(n_bytes, dtype=torch.uint8, device=DEV)
    block.fill_(1)
    return block.data_ptr()


def test_a_paged_cache_whose_workspace_is_still_written():
    import torch
    from paper_2503_08524_amd import PagedCache
    lens = [700, 90, 0, 4000]
    cache, g = pages._cache(lens, 2, 4, 128, "f16", 16, seed=12)
    q = torch.empty(4, 8, 128, device=DEV).normal_(generator=g)
    want = cache.attend(0, q)
    shared = dict(k_pages=cache.k_pages, v_pages=cache.v_pages, tables=cache.tables, rows=cache.rows, free_pages=cache.free_pages, n_free=cache.n_free)
    torch.cuda.synchronize()
    reused = False
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(3):
            at = _busy_block(cache.workspace.numel())
            other = PagedCache(8, 2, 128, cache.n_pages, 16, 4, cache.max_pages, device=DEV, **shared)
            reused = reused or other.workspace.data_ptr() == at
            out = [other.attend(0, q) for _ in range(3)]
            torch.cuda.current_stream().synchronize()
            assert all(torch.equal(x, want) for x in out)
    assert reused


def test_a_decoder_whose_workspace_is_still_written():
    """Frequencies and counters lie in the workspace: a decoder made on a busy side stream gives the logits of one made in quiet."""
    import torch
    from paper_2503_08524_amd import binding
    w = binding.weights_to_device(steps.GQA, d3_inputs.make_weights(steps.GQA, 0), DEV)
    tok = torch.from_numpy(d3_inputs.make_prompt(2, 20, steps.GQA.V, seed=7)).to(DEV)

    def run():
        dec = binding.Decoder(steps.GQA, w, 2, 32, kv_dtype="f16", device=DEV)
        dec.set_plan(1.0, 0, 0, 3)
        logits = [torch.zeros(2, steps.GQA.V, device=DEV) for _ in range(3)]
        nxt = dec.prefill(tok, logits=logits[0])
        for i in (1, 2):
            dec.decode_step(nxt, i, nxt, logits=logits[i])
        torch.cuda.current_stream().synchronize()
        return dec, logits
    dec, want = run()
    size = dec.workspace.numel()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(3):
            _busy_block(size)
            got = run()[1]
            assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(np.isfinite(x.cpu().numpy()).all() for x in got)

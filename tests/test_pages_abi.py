"""Host-side checks of the paged cache's entry points (no GPU): descriptions, workspaces and NULL arguments."""
import ctypes as C

import numpy as np
import pytest

import paper_2503_08524_amd as d3
from paper_2503_08524_amd import binding
from paper_2503_08524_amd import build as d3_build

GOOD = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=128, kv_dtype=binding.D3_F16, n_pages=100, page_rows=16, max_batch=4, max_pages=10)


@pytest.fixture(scope="module")
def lib():
    if d3_build.is_stale():
        d3_build.build()
    return d3.load_library()


def desc(**change):
    return binding._PagesDesc(**{**GOOD, **change})


def size(lib, **change):
    return lib.d3_pages_workspace_size(C.byref(desc(**change)))


def test_workspace_holds_two_partials_and_counters_a_run_and_a_counter_per_sequence_and_heads(lib):
    n = size(lib)
    assert n % 256 == 0 and 2 * 2048 * (4 * 130 * 4 + 4) <= n <= 2 * 2048 * (4 * 130 * 4 + 4) + 1024
    assert size(lib, n_heads=64, n_kv_heads=2) == size(lib, n_heads=32, n_kv_heads=2)      # 32 heads of a KV head are taken 16 at a time
    assert size(lib, max_batch=4096) - n == (4096 - 4) * 2 * 4 // 256 * 256
    assert size(lib, n_pages=100000) == n


@pytest.mark.parametrize("change,word", [
    (dict(n_layers=0), "n_layers"), (dict(n_heads=0), "n_heads"), (dict(n_kv_heads=0), "n_heads"), (dict(n_kv_heads=3), "multiple"),
    (dict(n_heads=70000, n_kv_heads=1), "n_heads"), (dict(head_dim=96), "head_dim"), (dict(kv_dtype=binding.D3_BF16), "D3_BF16"), (dict(kv_dtype=7), "kv_dtype"),
    (dict(page_rows=8), "page_rows"), (dict(page_rows=48), "page_rows"), (dict(page_rows=2048), "page_rows"), (dict(n_pages=0), "n_pages"),
    (dict(n_pages=1 << 28), "n_pages"), (dict(max_batch=0), "max_batch"), (dict(max_batch=4097), "max_batch"), (dict(max_pages=0), "max_pages"),
    (dict(max_pages=1 << 27), "max_pages"), (dict(max_batch=4096, max_pages=1 << 20), "max_pages"),
    (dict(max_batch=4096, max_pages=500000, n_heads=4096, n_kv_heads=4096), "more rows")])
def test_descriptions_that_are_refused(lib, change, word):
    assert size(lib, **change) == 0
    assert word in lib.d3_last_error().decode()


def test_create_checks_its_pointers_before_the_device(lib):
    room = np.zeros(4096, np.uint8)
    at = (room.ctypes.data + 255) // 256 * 256
    out, d = C.c_void_p(), desc()
    need = lib.d3_pages_workspace_size(C.byref(d))
    call = lambda o, dd, k, v, w, n: (lib.d3_pages_create(o, dd, k, v, w, n), lib.d3_last_error().decode())
    assert call(None, C.byref(d), at, at, at, need) == (-1, "d3_pages_create: out is NULL")
    for args, word in [((C.byref(out), None, at, at, at, need), "desc"), ((C.byref(out), C.byref(d), None, at, at, need), "NULL"), ((C.byref(out), C.byref(d), at, None, at, need), "NULL"),
                       ((C.byref(out), C.byref(d), at, at, None, need), "NULL"), ((C.byref(out), C.byref(d), at + 8, at, at, need), "16-byte"),
                       ((C.byref(out), C.byref(d), at, at, at + 128, need), "256-byte"), ((C.byref(out), C.byref(d), at, at, at, need - 1), "workspace has")]:
        status, message = call(*args)
        assert status == -1 and word in message and out.value is None


def test_null_handles_are_errors(lib):
    for status in (lib.d3_pages_reserve(None, 1, None, None, None, None, None, None, None, 1, None, None, None, None),
                   lib.d3_pages_append(None, 0, 1, 1, None, None, None, 0, 0, 0, 0, None, None),
                   lib.d3_pages_attention(None, 0, 1, None, None, None, 0, 0, 0, None, None, None, 0.0, None, 0, None),
                   lib.d3_pages_fill(None, 1, None, 0, 1, 1, None), lib.d3_store_pages(None, None, 0, 0, 1, None, None),
                   lib.d3_decode_step_paged(None, None, None, 1, 1, None, None, None, None, None, None), lib.d3_fill_missing_paged(None, None, 1, 1, None, None)):
        assert status == -1
    assert lib.d3_pages_destroy(None) == 0


def test_attention_keeps_its_rows_in_registers(tmp_path):
    """Two workgroups of four waves a compute unit have 256 registers a lane; with spills in the loop over rows the attention takes twice as long, and nothing else shows it."""
    import os
    import re
    import subprocess
    out = str(tmp_path / "attention_paged.s")
    flags = [f for f in d3_build.FLAGS if f != "-fPIC"]
    subprocess.run([d3_build.HIPCC] + flags + ["-x", "hip", "-S", "--offload-device-only", os.path.join(d3_build.CSRC, "attention_paged.hip"), "-o", out], check=True, capture_output=True)
    text = open(out).read()
    kernels = re.findall(r"\.name:\s+(\S*attn_paged_kernel\S*)", text)
    assert len(set(kernels)) == 16
    for field, most in ((".private_segment_fixed_size", 0), (".vgpr_spill_count", 0), (".vgpr_count", 256)):
        found = [int(x) for x in re.findall(re.escape(field) + r":\s+(\d+)", text)]
        assert len(found) == 16 and max(found) <= most, (field, found)


def test_null_handles_are_errors_of_the_calls_with_starts(lib):
    for call, args in ((lib.d3_pages_live, (None, 1, None, None, None, None)),
                       (lib.d3_decode_step_granted, (None, None, None, 1, 1, None, None, None, None, None, None, None))):
        assert call(*args) == -1 and "NULL" in lib.d3_last_error().decode()

"""Host-side checks of the paged cache of 8 bits (no GPU): descriptions, handles, NULL arguments, and that its kernels keep to their registers."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

import paper_2503_08524_amd as d3
from paper_2503_08524_amd import binding
from paper_2503_08524_amd import build as d3_build

GOOD = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=128, kv_dtype=binding.D3_I8, n_pages=100, page_rows=16, max_batch=4, max_pages=10)


@pytest.fixture(scope="module")
def lib():
    if d3_build.is_stale():
        d3_build.build()
    return d3.load_library()


def desc(**change):
    return binding._PagesDesc(**{**GOOD, **change})


@pytest.mark.parametrize("kv", [binding.D3_I8, binding.D3_E4M3])
def test_descriptions(lib, kv):
    n = lib.d3_pages_workspace_size(C.byref(desc(kv_dtype=kv)))
    assert n > 0 and n == lib.d3_pages_workspace_size(C.byref(desc(kv_dtype=binding.D3_F16)))       # partial results are fp32 whatever the pools hold
    for change, word in ((dict(kv_dtype=5), "D3_E4M3"), (dict(kv_dtype=-1), "kv_dtype"), (dict(head_dim=96), "head_dim"), (dict(page_rows=8), "page_rows"),
                         (dict(max_batch=4096, max_pages=500000, n_heads=8192, n_kv_heads=8192), "more rows")):
        assert lib.d3_pages_workspace_size(C.byref(desc(**{"kv_dtype": kv, **change}))) == 0
        assert word in lib.d3_last_error().decode()


def test_create_checks_its_pointers_before_the_device(lib):
    room = np.zeros(4096, np.uint8)
    at = (room.ctypes.data + 255) // 256 * 256
    out, d, half = C.c_void_p(), desc(), desc(kv_dtype=binding.D3_F16)
    need = lib.d3_pages_workspace_size(C.byref(d))
    assert lib.d3_pages_create(C.byref(out), C.byref(d), at, at, at, need) == -1 and "d3_pages_create_scaled" in lib.d3_last_error().decode()
    for args, word in (((None, C.byref(d), at, at, at, at, at, need), "out is NULL"), ((C.byref(out), None, at, at, at, at, at, need), "desc"),
                       ((C.byref(out), C.byref(half), at, at, at, at, at, need), "8 bits"), ((C.byref(out), C.byref(d), None, at, at, at, at, need), "NULL"),
                       ((C.byref(out), C.byref(d), at, at, None, at, at, need), "scales"), ((C.byref(out), C.byref(d), at, at, at, None, at, need), "scales"),
                       ((C.byref(out), C.byref(d), at, at, at + 4, at, at, need), "16-byte"), ((C.byref(out), C.byref(d), at, at, at, at + 8, at, need), "16-byte"),
                       ((C.byref(out), C.byref(d), at + 8, at, at, at, at, need), "16-byte"), ((C.byref(out), C.byref(d), at, at, at, at, at + 128, need), "256-byte"),
                       ((C.byref(out), C.byref(d), at, at, at, at, at, need - 1), "workspace has")):
        assert lib.d3_pages_create_scaled(*args) == -1 and word in lib.d3_last_error().decode() and out.value is None


def test_a_null_handle_is_an_error(lib):
    assert lib.d3_pages_read(None, 0, 1, 1, None, None, None, 0, 0, 0, 0, None) == -1 and "NULL" in lib.d3_last_error().decode()


def test_a_context_has_no_cache_of_8_bits(lib):
    for kv in (binding.D3_I8, binding.D3_E4M3):
        d = binding._ModelDesc(2, 256, 4, 4, 64, 512, 1000, 1e-6, 10000.0, binding.D3_F32, kv, 1, 64)
        assert lib.d3_workspace_size(C.byref(d)) == 0


@pytest.mark.parametrize("source,kernel,count", [("attention_paged8.hip", "attn_paged_kernel", 16), ("pages8.hip", "pages_", 36)])
def test_kernels_use_no_scratch(tmp_path, source, kernel, count):
    """A kernel with any scratch at all starts 1 us later, and the attention's loop over rows takes up to twice as long with spills in it; nothing else shows either."""
    out = str(tmp_path / "k.s")
    flags = [f for f in d3_build.FLAGS if f != "-fPIC"]
    subprocess.run([d3_build.HIPCC] + flags + ["-x", "hip", "-S", "--offload-device-only", os.path.join(d3_build.CSRC, source), "-o", out], check=True, capture_output=True)
    text = open(out).read()
    assert len(set(re.findall(r"\.name:\s+(\S*" + kernel + r"\S*)", text))) == count
    for field, most in ((".private_segment_fixed_size", 0), (".vgpr_spill_count", 0), (".vgpr_count", 256)):
        found = [int(x) for x in re.findall(re.escape(field) + r":\s+(\d+)", text)]
        assert len(found) == count and max(found) <= most, (field, found)

"""What a caller is told who hands a wrong pointer to a handle of pages (host checks, no GPU)."""
import ctypes as C

import numpy as np
import pytest

import paper_2503_08524_amd as d3
from paper_2503_08524_amd import binding
from paper_2503_08524_amd import build as d3_build


@pytest.fixture(scope="module")
def lib():
    if d3_build.is_stale():
        d3_build.build()
    return d3.load_library()


@pytest.mark.parametrize("entry,kind", [("d3_pages_create", binding.D3_F16), ("d3_pages_create_scaled", binding.D3_I8)])
def test_messages_of_create_name_the_call(lib, entry, kind):
    room = np.zeros(4096, np.uint8)
    at = (room.ctypes.data + 255) // 256 * 256
    out, d = C.c_void_p(), binding._PagesDesc(2, 8, 2, 128, kind, 100, 16, 4, 10)
    need = lib.d3_pages_workspace_size(C.byref(d))
    scales = [at, at] if entry.endswith("scaled") else []
    call = getattr(lib, entry)
    for k, v, ws, size, word in ((None, at, at, need, "NULL"), (at, None, at, need, "NULL"), (at, at, None, need, "NULL"), (at + 8, at, at, need, "16-byte"), (at, at, at + 128, need, "256-byte"),
                                 (at, at, at, need - 1, "needed")):
        assert call(C.byref(out), C.byref(d), k, v, *scales, ws, size) == -1
        message = lib.d3_last_error().decode()
        assert message.startswith(entry + ": ") and word in message and out.value is None

"""What a caller is told who asks for a cache type that is not offered, or hands a wrong pointer to a pool of 8 bits (host checks, no GPU)."""
import ctypes as C

import numpy as np
import pytest

import d3_inputs
import paper_2503_08524_amd as d3
from paper_2503_08524_amd import binding
from paper_2503_08524_amd import build as d3_build


@pytest.fixture(scope="module")
def lib():
    if d3_build.is_stale():
        d3_build.build()
    return d3.load_library()


@pytest.mark.parametrize("kv,code", [("i8", binding.D3_I8), ("e4m3", binding.D3_E4M3)])
def test_a_context_with_a_cache_of_8_bits_is_refused_by_name(lib, kv, code):
    with pytest.raises(d3.D3Error) as e:
        binding.Decoder(d3_inputs.TINY, {}, 1, 64, kv_dtype=kv)
    assert "kv_dtype must be D3_F32 or D3_F16" in str(e.value)
    assert binding.d3_workspace_size(d3_inputs.TINY, kv, 1, 64) == 0
    desc, out = binding._desc(d3_inputs.TINY, kv, 1, 64), C.c_void_p()
    assert desc.kv_dtype == code
    room = np.zeros(4096, np.uint8).ctypes.data
    assert lib.d3_create(C.byref(out), C.byref(desc), C.byref(binding._Weights()), room, room, room, 1 << 20) == -1
    assert "kv_dtype must be D3_F32 or D3_F16" in lib.d3_last_error().decode() and out.value is None


def test_a_type_that_is_none_is_a_value_error_that_names_them(lib):
    for kv in ("fp16", "int8", "F32"):
        for make in (lambda: binding.Decoder(d3_inputs.TINY, {}, 1, 64, kv_dtype=kv), lambda: binding.d3_workspace_size(d3_inputs.TINY, kv, 1, 64)):
            with pytest.raises(ValueError) as e:
                make()
            assert "kv_dtype" in str(e.value) and "'f16'" in str(e.value)


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

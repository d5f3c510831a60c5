"""ctypes binding of libd3.so: the same entry points as include/d3.h, argument
marshalling only.  PyTorch supplies device memory and streams; every step of the
path runs in the library's kernels.  There is no fallback: if the library is not
built, loading fails."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB: Optional[C.CDLL] = None

D3_F32, D3_BF16, D3_F16 = 0, 1, 2
D3_FILL_COPY = 0
D3_FILL_RECOMPUTE = 1
D3_K_NONE, D3_K_QKV, D3_K_ATTN, D3_K_OPROJ, D3_K_GATE_UP, D3_K_DOWN, D3_K_LM_HEAD, D3_K_EMPTY = range(8)


class D3Error(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"d3 status {status}: {message}")
        self.status = status


class _ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab")] + [
        ("rms_eps", C.c_float), ("rope_base", C.c_float)] + [
        (n, C.c_int32) for n in ("weight_dtype", "kv_dtype", "max_batch", "max_seq")]


class _LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")]


class _Weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("layers", C.POINTER(_LayerWeights)), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)]


class _PagesDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_heads", "n_kv_heads", "head_dim", "kv_dtype", "n_pages", "page_rows", "max_batch", "max_pages")]


def library_path() -> str:
    return os.environ.get("D3_LIBRARY", os.path.join(_HERE, "libd3.so"))


def load_library() -> C.CDLL:
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise OSError(f"{path} is not built: run `python -m paper_2503_08524_amd.build` (there is no fallback path)")
        # PyTorch ships its own HIP runtime and owns the device memory and streams handed to the library, so it is
        # loaded first: libd3.so then binds to that runtime.  Loaded the other way round the process holds two
        # runtimes and the second one to initialise finds no device.
        import torch  # noqa: F401
        lib = C.CDLL(path)
        i32, vp, dbl = C.c_int32, C.c_void_p, C.c_double
        lib.d3_last_error.restype = C.c_char_p
        lib.d3_plan_depth.argtypes = [i32, dbl, i32, i32, i32, vp, vp, vp]
        lib.d3_plan_depth_linear.argtypes = [i32, i32, i32, i32, i32, vp, vp, vp]
        lib.d3_plan_from_table.argtypes = [i32, i32, vp, vp, vp]
        lib.d3_workspace_size.argtypes = [C.POINTER(_ModelDesc)]
        lib.d3_workspace_size.restype = C.c_size_t
        lib.d3_create.argtypes = [C.POINTER(vp), C.POINTER(_ModelDesc), C.POINTER(_Weights), vp, vp, vp, C.c_size_t]
        lib.d3_destroy.argtypes = [vp]
        lib.d3_set_plan.argtypes = [vp, dbl, i32, i32, i32]
        lib.d3_set_plan_table.argtypes = [vp, vp, vp, i32]
        lib.d3_prefill.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, vp]
        lib.d3_prefill_ragged.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp]
        lib.d3_decode_step.argtypes = [vp, vp, i32, vp, vp, vp, vp]
        lib.d3_decode_step_static.argtypes = [vp, vp, i32, vp, vp, vp, vp]
        lib.d3_static_scratch_bytes.restype = C.c_size_t
        lib.d3_fill_missing_kv.argtypes = [vp, i32, i32, i32, vp]
        lib.d3_set_fill_mode.argtypes = [vp, i32]
        lib.d3_n_ctx.argtypes = [vp]
        lib.d3_n_ctx.restype = i32
        lib.d3_truncate.argtypes = [vp, i32]
        lib.d3_stream_read.argtypes = [vp, vp, C.c_size_t, vp]
        i64 = C.c_int64
        lib.d3_pages_workspace_size.argtypes = [C.POINTER(_PagesDesc)]
        lib.d3_pages_workspace_size.restype = C.c_size_t
        lib.d3_pages_create.argtypes = [C.POINTER(vp), C.POINTER(_PagesDesc), vp, vp, vp, C.c_size_t]
        lib.d3_pages_destroy.argtypes = [vp]
        lib.d3_pages_reserve.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
        lib.d3_pages_append.argtypes = [vp, i32, i32, i32, vp, vp, vp, i32, i64, i64, i64, vp, vp]
        lib.d3_pages_attention.argtypes = [vp, i32, i32, vp, vp, vp, i32, i64, i64, vp, vp, vp, C.c_float, vp, i64, vp]
        lib.d3_pages_live.argtypes = [vp, i32, vp, vp, vp, vp]
        lib.d3_pages_fill.argtypes = [vp, i32, vp, i32, i32, i32, vp]
        lib.d3_store_pages.argtypes = [vp, vp, i32, i32, i32, vp, vp]
        lib.d3_decode_step_paged.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp]
        lib.d3_decode_step_granted.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.d3_fill_missing_paged.argtypes = [vp, vp, i32, i32, vp, vp]
        lib.d3_mfma_yardstick.argtypes = [vp, i32, i32, vp]
        lib.d3_profile_select.argtypes = [vp, i32]
        lib.d3_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        _LIB = lib
    return _LIB


def _check(rc: int) -> None:
    if rc != 0:
        raise D3Error(rc, load_library().d3_last_error().decode())


def d3_plan_depth(L: int, alpha: float, start_layer: int, min_keep: int, n_steps: int):
    """(keep[n_steps], drop_begin[n_steps], layer_ids[n_steps][L]) int32 arrays (host only)."""
    keep = np.zeros(max(n_steps, 0), np.int32)
    drop = np.zeros(max(n_steps, 0), np.int32)
    ids = np.zeros((max(n_steps, 0), max(L, 0)), np.int32)
    _check(load_library().d3_plan_depth(L, float(alpha), start_layer, min_keep, n_steps,
                                        keep.ctypes.data, drop.ctypes.data, ids.ctypes.data))
    return keep, drop, ids


def d3_plan_depth_linear(L: int, keep_first: int, keep_last: int, start_layer: int, n_steps: int):
    """Linear decay from keep_first to keep_last; same three arrays as d3_plan_depth (host only)."""
    keep = np.zeros(max(n_steps, 0), np.int32)
    drop = np.zeros(max(n_steps, 0), np.int32)
    ids = np.zeros((max(n_steps, 0), max(L, 0)), np.int32)
    _check(load_library().d3_plan_depth_linear(L, keep_first, keep_last, start_layer, n_steps,
                                               keep.ctypes.data, drop.ctypes.data, ids.ctypes.data))
    return keep, drop, ids


def d3_plan_from_table(L: int, keep, drop_begin):
    """layer_ids[n_steps][L] of a caller-made schedule (host only); raises D3Error on a step that does not fit."""
    keep = np.ascontiguousarray(keep, np.int32); drop = np.ascontiguousarray(drop_begin, np.int32)
    if keep.shape != drop.shape or keep.ndim != 1:
        raise ValueError("keep and drop_begin must be 1-d arrays of one length")
    ids = np.zeros((keep.size, max(L, 0)), np.int32)
    _check(load_library().d3_plan_from_table(L, keep.size, keep.ctypes.data, drop.ctypes.data, ids.ctypes.data))
    return ids


def _desc(shape, kv_dtype: str, max_batch: int, max_seq: int) -> _ModelDesc:
    dt = {"f32": D3_F32, "bf16": D3_BF16, "f16": D3_F16}
    return _ModelDesc(shape.L, shape.d, shape.H, shape.H_kv, shape.hd, shape.F, shape.V, float(shape.eps),
                      float(shape.rope_base), dt[shape.dtype], dt[kv_dtype], max_batch, max_seq)


def d3_workspace_size(shape, kv_dtype: str, max_batch: int, max_seq: int) -> int:
    d = _desc(shape, kv_dtype, max_batch, max_seq)
    return int(load_library().d3_workspace_size(C.byref(d)))


def default_kv_dtype(shape) -> str:
    """Cache precision that keeps logits within 2e-2 of full precision at the model's depth: the rounding of the cache
    rows moves the hidden state by about 4.5e-4 (relative) per block with fp16 rows and grows like sqrt(L), which is
    inside the bound for the 32 and 40 blocks of the 7B and 13B shapes and outside it for the 80 blocks of the 70B shape
    (measured 1.1e-2, 1.7e-2 and 3.3e-2); fp32 rows stay at 4e-4 of logit error at 80 blocks."""
    if shape.dtype == "f32" or shape.L > 48:
        return "f32"
    return "f16"


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class Decoder:
    """One d3_ctx plus the device buffers it borrows (all torch tensors on one GPU).

    weights: dict like d3_inputs.make_weights but of torch CUDA tensors
    (float32, or bfloat16 for bf16 models; gains float32).  kv_dtype: "f32" or "f16"; default: default_kv_dtype(shape)."""

    def __init__(self, shape, weights: Dict[str, object], max_batch: int, max_seq: int, kv_dtype: Optional[str] = None,
                 device: str = "cuda:0"):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.shape = shape
        self.device = torch.device(device)
        self.kv_dtype = kv_dtype or default_kv_dtype(shape)
        self.max_batch, self.max_seq = max_batch, max_seq
        self.weights = weights                       # keep the tensors alive
        desc = _desc(shape, self.kv_dtype, max_batch, max_seq)
        ws_bytes = int(self.lib.d3_workspace_size(C.byref(desc)))
        if ws_bytes == 0:
            _check(-2)
        tdt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[self.kv_dtype]
        kv_shape = (shape.L, max_batch, shape.H_kv, max_seq, shape.hd)
        with torch.cuda.device(self.device):
            self.k_cache = torch.zeros(kv_shape, dtype=tdt, device=self.device)
            self.v_cache = torch.zeros(kv_shape, dtype=tdt, device=self.device)
            self.workspace = torch.zeros(ws_bytes, dtype=torch.uint8, device=self.device)
            layers = (_LayerWeights * shape.L)()
            for l, lw in enumerate(weights["layers"]):
                for name, _ in _LayerWeights._fields_:
                    t = lw[name]
                    assert t.is_cuda and t.is_contiguous(), name
                    setattr(layers[l], name, t.data_ptr())
            self._layers = layers
            w = _Weights(weights["tok_emb"].data_ptr(), layers, weights["final_norm"].data_ptr(), weights["lm_head"].data_ptr())
            # d3_create writes to the workspace on the null stream, which does not wait for this one, where the zeros are still to be written.
            torch.cuda.current_stream(self.device).synchronize()
            ctx = C.c_void_p()
            _check(self.lib.d3_create(C.byref(ctx), C.byref(desc), C.byref(w), self.k_cache.data_ptr(), self.v_cache.data_ptr(),
                                      self.workspace.data_ptr(), ws_bytes))
        self.ctx = ctx

    def close(self) -> None:
        if getattr(self, "ctx", None):
            self.lib.d3_destroy(self.ctx)
            self.ctx = None

    __del__ = close

    def _stream(self) -> int:
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def set_plan(self, alpha: float, start_layer: int, min_keep: int, n_steps: int) -> None:
        _check(self.lib.d3_set_plan(self.ctx, float(alpha), start_layer, min_keep, n_steps))

    def set_plan_table(self, keep, drop_begin) -> None:
        keep = np.ascontiguousarray(keep, np.int32); drop = np.ascontiguousarray(drop_begin, np.int32)
        if keep.shape != drop.shape or keep.ndim != 1:
            raise ValueError("keep and drop_begin must be 1-d arrays of one length")
        _check(self.lib.d3_set_plan_table(self.ctx, keep.ctypes.data, drop.ctypes.data, keep.size))

    def prefill(self, tokens, pos_begin: int = 0, next_tok=None, logits=None, hidden_dump=None):
        """tokens: int32 CUDA tensor [B, P].  Returns next_tok (int32 CUDA tensor [B])."""
        B, P = tokens.shape
        if next_tok is None:
            next_tok = self.torch.empty(B, dtype=self.torch.int32, device=self.device)
        _check(self.lib.d3_prefill(self.ctx, tokens.data_ptr(), B, P, pos_begin, next_tok.data_ptr(), _ptr(logits),
                                   _ptr(hidden_dump), self._stream()))
        return next_tok

    def prefill_ragged(self, tokens, lengths, next_tok=None, logits=None, hidden_dump=None):
        """tokens: int32 CUDA tensor [B, P], left-padded; lengths: B host ints (the longest equals P)."""
        B, P = tokens.shape
        lens = np.ascontiguousarray(lengths, np.int32)
        if lens.shape != (B,):
            raise ValueError("lengths must hold one entry per sequence")
        if next_tok is None:
            next_tok = self.torch.empty(B, dtype=self.torch.int32, device=self.device)
        _check(self.lib.d3_prefill_ragged(self.ctx, tokens.data_ptr(), lens.ctypes.data, B, P, next_tok.data_ptr(),
                                          _ptr(logits), _ptr(hidden_dump), self._stream()))
        return next_tok

    def decode_step(self, tok_in, step_i: int, tok_out, logits=None, hidden_dump=None) -> None:
        _check(self.lib.d3_decode_step(self.ctx, tok_in.data_ptr(), step_i, tok_out.data_ptr(), _ptr(logits),
                                       _ptr(hidden_dump), self._stream()))

    def decode_step_static(self, tok_in, step_i: int, tok_out, logits=None, hidden_dump=None) -> None:
        """decode_step with its intermediates in the library's static scratch array (no workspace use, no allocation)."""
        _check(self.lib.d3_decode_step_static(self.ctx, tok_in.data_ptr(), step_i, tok_out.data_ptr(), _ptr(logits),
                                              _ptr(hidden_dump), self._stream()))

    def fill_missing_kv(self, pos_begin: int, pos_end: int, mode: int = D3_FILL_COPY) -> None:
        _check(self.lib.d3_fill_missing_kv(self.ctx, pos_begin, pos_end, mode, self._stream()))

    def set_fill_mode(self, mode: int) -> None:
        _check(self.lib.d3_set_fill_mode(self.ctx, mode))

    def store_pages(self, cache: "PagedCache", seq: int, slots, row_begin: int = 0) -> None:
        """Rows row_begin .. of sequence seq, as a prompt pass wrote them, into the slots (int32 CUDA tensor) of every layer of `cache`."""
        cache._ints(slots=slots)
        _check(self.lib.d3_store_pages(self.ctx, cache.handle, seq, row_begin, slots.numel(), slots.data_ptr(), self._stream()))

    def decode_step_paged(self, cache: "PagedCache", tok_in, step_i: int, tok_out, logits=None, hidden_dump=None, starts=None) -> None:
        """One step of the cache's first tok_in.numel() sequences, whose newest rows cache.reserve has made room for.  starts: what that reserve returned; the sequences
        that it gave no row (refused, paused, ended) are idle: their rows stay, tok_out is tok_in.  Without it every sequence that has rows must have got one, or
        the step overwrites its newest row.  fill_missing_paged of that reserve's slots comes next, before any step that runs a block this one drops."""
        cache._ints(tok_in=tok_in, tok_out=tok_out)
        B = tok_in.numel()
        if tok_out.numel() < B:
            raise ValueError("tok_out is shorter than tok_in")
        at = (self.ctx, cache.handle, tok_in.data_ptr(), B, step_i, cache.tables.data_ptr(), cache.rows.data_ptr())
        out = (tok_out.data_ptr(), _ptr(logits), _ptr(hidden_dump), self._stream())
        if starts is None:
            _check(self.lib.d3_decode_step_paged(*at, *out))
        else:
            _check(self.lib.d3_decode_step_granted(*at, cache._starts(starts, B), *out))

    def fill_missing_paged(self, cache: "PagedCache", slots, step_i: int) -> None:
        """COPY fill of the rows `slots`, which a reserve returned, in the blocks that step step_i of the plan drops, after that step: the pages hold there what their last owner left."""
        cache._ints(slots=slots)
        _check(self.lib.d3_fill_missing_paged(self.ctx, cache.handle, step_i, slots.numel(), slots.data_ptr(), self._stream()))

    def synchronize(self) -> None:
        self.torch.cuda.current_stream(self.device).synchronize()

    def truncate(self, n_rows: int) -> None:
        _check(self.lib.d3_truncate(self.ctx, n_rows))

    def stream_read(self, tensor) -> None:
        """Read-only streaming yardstick over a CUDA tensor (one launch, asynchronous)."""
        _check(self.lib.d3_stream_read(self.ctx, tensor.data_ptr(), tensor.numel() * tensor.element_size(), self._stream()))

    def mfma_yardstick(self, mode: int, stages: int) -> None:
        """Matrix-core yardstick of the prompt pass (one launch, asynchronous): mode 0 MFMAs alone, 1 with LDS
        fragment reads, 2 with a barrier per stage too; n_cu workgroups x 8 waves x stages x 32 instructions of 16384 flops."""
        _check(self.lib.d3_mfma_yardstick(self.ctx, mode, stages, self._stream()))

    def profile_select(self, kernel_class: int) -> None:
        _check(self.lib.d3_profile_select(self.ctx, kernel_class))

    def profile_read(self):
        """(summed milliseconds, launches) of the selected kernel class since the last read."""
        ms, n = C.c_double(), C.c_int64()
        _check(self.lib.d3_profile_read(self.ctx, C.byref(ms), C.byref(n)))
        return ms.value, n.value

    @property
    def n_ctx(self) -> int:
        return int(self.lib.d3_n_ctx(self.ctx))


class PagedCache:
    """A paged key-value cache (the d3_pages_* entry points) and the operators on it: one handle, the page pools and the
    state of the sequences, all torch tensors on one GPU.  Every call is asynchronous on the current stream, allocates nothing on the
    device unless an output is left out, and can be captured into a graph.  Making one waits for the current stream and cannot be captured; before one that other
    streams have used goes away, these have to be waited for.

    k_pages [n_layers][n_pages][n_kv_heads][page_rows][head_dim] and v_pages [n_layers][n_pages][n_kv_heads][page_rows / R][head_dim][R]
    (R = 8 for "f16", 4 for "f32"); tables int32 [max_batch][max_pages]; rows int32 [max_batch]; free_pages int32 [n_pages], a stack of which
    the first n_free[0] entries count.  Buffers that are not given are made: pools of zeros, no sequences, all pages free."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, page_rows: int, max_batch: int, max_pages: int,
                 kv_dtype: str = "f16", n_layers: int = 1, k_pages=None, v_pages=None, tables=None, rows=None, free_pages=None, n_free=None,
                 device: str = "cuda:0"):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.handle = None
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.n_layers, self.n_heads, self.n_kv_heads, self.head_dim = n_layers, n_heads, n_kv_heads, head_dim
        self.n_pages, self.page_rows, self.max_batch, self.max_pages, self.kv_dtype = n_pages, page_rows, max_batch, max_pages, kv_dtype
        kinds = {"f32": D3_F32, "bf16": D3_BF16, "f16": D3_F16}
        if kv_dtype not in kinds:
            raise ValueError(f"kv_dtype must be one of {sorted(kinds)} (got {kv_dtype!r})")
        desc = _PagesDesc(n_layers, n_heads, n_kv_heads, head_dim, kinds[kv_dtype], n_pages, page_rows, max_batch, max_pages)
        ws_bytes = int(self.lib.d3_pages_workspace_size(C.byref(desc)))
        if ws_bytes == 0:
            raise D3Error(-2, self.lib.d3_last_error().decode())
        self._kinds = {torch.float32: D3_F32, torch.bfloat16: D3_BF16, torch.float16: D3_F16}
        self._int32, self._float32 = torch.int32, torch.float32
        self._index = self.device.index
        # the current stream's handle without the object around it (2 us a call), where torch offers that
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
        tdt = {"f32": torch.float32, "f16": torch.float16}[kv_dtype]
        unit = 16 // tdt.itemsize
        with torch.cuda.device(self.device):
            def buffer(name, given, dims, dtype, make):
                if given is None:
                    return make(dims, dtype=dtype, device=self.device)
                if tuple(given.shape) != tuple(dims) or given.dtype != dtype or given.device != self.device or not given.is_contiguous():
                    raise ValueError(f"{name} must be a contiguous {dtype} tensor {tuple(dims)} on {self.device}")
                return given
            self.k_pages = buffer("k_pages", k_pages, (n_layers, n_pages, n_kv_heads, page_rows, head_dim), tdt, torch.zeros)
            self.v_pages = buffer("v_pages", v_pages, (n_layers, n_pages, n_kv_heads, page_rows // unit, head_dim, unit), tdt, torch.zeros)
            none = lambda dims, **kw: torch.full(dims, -1, **kw)
            self.tables = buffer("tables", tables, (max_batch, max_pages), torch.int32, none)
            self.rows = buffer("rows", rows, (max_batch,), torch.int32, torch.zeros)
            self.free_pages = buffer("free_pages", free_pages, (n_pages,), torch.int32, lambda dims, **kw: torch.arange(n_pages - 1, -1, -1, **kw))
            self.n_free = buffer("n_free", n_free, (2,), torch.int32, torch.zeros)
            if n_free is None:
                self.n_free[:1].fill_(n_pages)
            self._live = torch.empty(max_batch, dtype=torch.int32, device=self.device)      # rows that an attend with starts counts
            self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)
            # The counters are cleared on the null stream, which does not wait for this one, where work on memory that the workspace was made from may still be queued.
            torch.cuda.current_stream(self.device).synchronize()
            handle = C.c_void_p()
            _check(self.lib.d3_pages_create(C.byref(handle), C.byref(desc), self.k_pages.data_ptr(), self.v_pages.data_ptr(),
                                            self.workspace.data_ptr(), ws_bytes))
        self.handle = handle

    def close(self) -> None:
        if getattr(self, "handle", None):
            self.lib.d3_pages_destroy(self.handle)
            self.handle = None

    __del__ = close

    # (A decode step makes a few of these calls per block, so their checks look at each tensor once.)
    def _stream(self) -> int:
        return self._raw_stream(self._index)

    def _ints(self, **tensors) -> None:
        for name, t in tensors.items():
            if t.dtype is not self._int32 or t.get_device() != self._index or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 tensor on {self.device}")

    def _starts(self, starts, B: int) -> int:
        self._ints(starts=starts)
        if starts.numel() < B + 1:
            raise ValueError(f"starts must have {B + 1} entries, as reserve returns it for these sequences")
        return starts.data_ptr()

    def _angles(self, rope_cs, n: int) -> Optional[int]:
        if rope_cs is None:
            return None
        if rope_cs.shape != (n, self.head_dim // 2, 2) or rope_cs.dtype is not self._float32 or rope_cs.get_device() != self._index or not rope_cs.is_contiguous():
            raise ValueError(f"rope_cs must be a contiguous float32 tensor ({n}, {self.head_dim // 2}, 2) on {self.device}")
        return rope_cs.data_ptr()

    def _heads(self, name: str, t, dims, dtype, strides=None):
        """The tensor's strides; it must have these dims, this dtype, a dense last dim (and these strides, where a dim has more than one entry)."""
        own = t.stride()
        if (t.shape != dims or t.dtype is not dtype or t.get_device() != self._index or own[-1] != 1
                or (strides is not None and own != strides and any(x != y and n > 1 for x, y, n in zip(own, strides, dims)))):
            raise ValueError(f"{name} must be a {dtype} tensor {tuple(dims)} on {self.device}, its last dim dense{'' if strides is None else f', with strides {strides}'}")
        return own

    def _kind(self, t) -> int:
        kind = self._kinds.get(t.dtype)
        if kind is None:
            raise ValueError(f"keys, values and queries must be float32, bfloat16 or float16 (got {t.dtype})")
        return kind

    def reserve(self, added, max_tokens: int, starts=None, slots=None, positions=None, rows_out=None, n_free_out=None):
        """Room for added[b] more rows of sequence b (int32 CUDA tensor [B]; 0: none, negative: the sequence has ended), B <= max_batch, at most max_tokens rows in all.
        Updates tables, rows and the stack of free pages (rows_out [B] and n_free_out [2]: elsewhere than in place) and returns (starts [B + 1], slots [max_tokens],
        positions [max_tokens]): sequence b's new rows are entries starts[b] .. starts[b + 1] - 1 of the other two, none where the request was refused."""
        torch, B = self.torch, added.numel()
        new = lambda n: torch.empty(n, dtype=torch.int32, device=self.device)
        if B > self.max_batch or max_tokens < 0:
            raise ValueError(f"added must have at most {self.max_batch} entries and max_tokens must not be negative")
        starts = new(B + 1) if starts is None else starts
        slots = new(max_tokens) if slots is None else slots
        positions = new(max_tokens) if positions is None else positions
        rows_out = self.rows if rows_out is None else rows_out
        n_free_out = self.n_free if n_free_out is None else n_free_out
        self._ints(added=added, starts=starts, slots=slots, positions=positions, rows_out=rows_out, n_free_out=n_free_out)
        if starts.numel() < B + 1 or slots.numel() < max_tokens or positions.numel() < max_tokens or rows_out.numel() < B or n_free_out.numel() < 2:
            raise ValueError("an output is shorter than what reserve writes")
        _check(self.lib.d3_pages_reserve(self.handle, B, added.data_ptr(), self.rows.data_ptr(), rows_out.data_ptr(), self.tables.data_ptr(),
                                         self.free_pages.data_ptr(), self.n_free.data_ptr(), n_free_out.data_ptr(), max_tokens, starts.data_ptr(),
                                         slots.data_ptr(), positions.data_ptr(), self._stream()))
        return starts, slots, positions

    def append(self, layer: int, slots, k, v, rope_cs=None) -> None:
        """k, v [n][n_kv_heads][head_dim], or [m][n][n_kv_heads][head_dim] for the m layers from `layer` on, into the rows `slots` (int32 CUDA tensor [n]) of the pools.  k and v have
        the same strides, the last dim dense.
        rope_cs [n][head_dim / 2][2]: (cos, sin) by which the keys turn first."""
        self._ints(slots=slots)
        n, kind = slots.numel(), self._kind(k)
        layers = k.shape[0] if k.dim() == 4 else 1
        dims = (layers, n, self.n_kv_heads, self.head_dim) if k.dim() == 4 else (n, self.n_kv_heads, self.head_dim)
        strides = self._heads("k", k, dims, k.dtype)
        self._heads("v", v, dims, k.dtype, strides)
        # (the stride of a dim with one entry says nothing)
        _check(self.lib.d3_pages_append(self.handle, layer, layers, n, slots.data_ptr(), k.data_ptr(), v.data_ptr(), kind, strides[-3] if n > 1 else 0,
                                        strides[-2] if self.n_kv_heads > 1 else 0, strides[0] if layers > 1 else 0, self._angles(rope_cs, n), self._stream()))

    def attend(self, layer: int, q, k=None, v=None, rope_cs=None, scale: float = 0.0, out=None, starts=None):
        """Attention of one token of each of the first B sequences, q [B][n_heads][head_dim], over their rows; returns out [B][n_heads][head_dim] of q's dtype.
        k, v [B][n_kv_heads][head_dim]: the newest rows (row rows[b] - 1), which the call also writes to their pages; without them they are there already.  The heads of a
        sequence lie side by side in all of them, and k and v have the same strides.
        rope_cs [B][head_dim / 2][2]: q and k turn by it.  scale 0: 1 / sqrt(head_dim).
        starts: what the reserve before it returned; of the sequences that it gave no row nothing is read or written, and out is 0.  Without it, and with k and v, every sequence
        that has rows must have got one."""
        B, dtype, kind = q.shape[0], q.dtype, self._kind(q)
        dims = (B, self.n_heads, self.head_dim)
        if out is None:
            out = self.torch.empty(dims, dtype=dtype, device=self.device)
        q_strides, out_strides = self._heads("q", q, dims, dtype), self._heads("out", out, dims, dtype)
        if self.n_heads > 1 and (q_strides[1] != self.head_dim or out_strides[1] != self.head_dim):
            raise ValueError("q and out must have the heads of a sequence side by side")
        k_at = v_at = None
        kv_strides = (0,)
        if k is not None and v is not None:
            dims = (B, self.n_kv_heads, self.head_dim)
            kv_strides = self._heads("k", k, dims, dtype)
            self._heads("v", v, dims, dtype, kv_strides)
            if self.n_kv_heads > 1 and kv_strides[1] != self.head_dim:
                raise ValueError("k and v must have the heads of a sequence side by side")
            k_at, v_at = k.data_ptr(), v.data_ptr()
        elif k is not None or v is not None:
            raise ValueError("k and v come together or not at all")
        if B == 1:                                                  # (the stride of a dim with one entry says nothing)
            q_strides = kv_strides = out_strides = (0,)
        angles, rows, stream = self._angles(rope_cs, B), self.rows, self._stream()
        if starts is not None:
            rows = self._live
            _check(self.lib.d3_pages_live(self.handle, B, self.rows.data_ptr(), self._starts(starts, B), rows.data_ptr(), stream))
        _check(self.lib.d3_pages_attention(self.handle, layer, B, q.data_ptr(), k_at, v_at, kind, q_strides[0], kv_strides[0], angles,
                                           self.tables.data_ptr(), rows.data_ptr(), scale, out.data_ptr(), out_strides[0], stream))
        return out

    def fill(self, slots, src: int, first: int, n_layers: int) -> None:
        """Rows `slots` of layer src (zeros if negative) copied into layers first .. first + n_layers - 1."""
        self._ints(slots=slots)
        _check(self.lib.d3_pages_fill(self.handle, slots.numel(), slots.data_ptr(), src, first, n_layers, self._stream()))


def weights_to_device(shape, weights_np: Dict[str, object], device: str = "cuda:0") -> Dict[str, object]:
    """numpy weights (float32, or uint16 bf16 bit patterns) -> torch CUDA tensors, bit-exact."""
    import torch

    def conv(a: np.ndarray):
        if a.dtype == np.uint16:
            return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
        return torch.from_numpy(a).to(device)

    out = {k: conv(v) for k, v in weights_np.items() if k != "layers"}
    out["layers"] = [{k: conv(v) for k, v in lw.items()} for lw in weights_np["layers"]]
    return out


def random_weights_on_device(shape, seed: int = 0, device: str = "cuda:0") -> Dict[str, object]:
    """N(0, 0.02) weights drawn on the GPU (performance runs only: not bit-reproducible on the host)."""
    import torch
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    tdt = torch.float32 if shape.dtype == "f32" else torch.bfloat16

    def normal(*dims):
        t = torch.empty(dims, dtype=torch.float32, device=device)
        t.normal_(0.0, 0.02, generator=g)
        return t.to(tdt)

    s = shape
    layers = []
    for _ in range(s.L):
        layers.append({
            "attn_norm": torch.ones(s.d, dtype=torch.float32, device=device),
            "wq": normal(s.H * s.hd, s.d), "wk": normal(s.H_kv * s.hd, s.d), "wv": normal(s.H_kv * s.hd, s.d),
            "wo": normal(s.d, s.H * s.hd), "mlp_norm": torch.ones(s.d, dtype=torch.float32, device=device),
            "w_gate": normal(s.F, s.d), "w_up": normal(s.F, s.d), "w_down": normal(s.d, s.F)})
    return {"tok_emb": normal(s.V, s.d), "lm_head": normal(s.V, s.d),
            "final_norm": torch.ones(s.d, dtype=torch.float32, device=device), "layers": layers}

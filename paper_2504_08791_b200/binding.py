"""Thin ctypes binding of ``libprima.so`` (argument marshalling only; every step runs in the library).

Function names mirror ``include/prima.h``.  Device buffers are torch CUDA tensors (torch is used
for device memory and streams only); host buffers are numpy arrays.  Loading fails loudly when
the library has not been built: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# PRIMA_LIB=bounds selects the range-checked build of the same sources (tests)
LIB_PATH = os.path.join(_HERE, "libprima_bounds.so" if os.environ.get("PRIMA_LIB") == "bounds" else "libprima.so")

OK, ERR_ARG, ERR_STATE, ERR_CUDA, ERR_NOMEM, ERR_DEVICE = 0, -1, -2, -3, -4, -5
ATTN_NORM, WQ, WK, WV, WO, FFN_NORM, W_GATE, W_UP, W_DOWN, OUT_NORM, W_HEAD, TOK_EMBD = range(12)
MAX_N_TOK = 8      # tokens of one sequence per step
MAX_N_SEQ = 16     # requests per step / columns of a product
PROF_GEMV, PROF_ATTENTION = 0, 1
PROF_GEMV_QKV, PROF_GEMV_O, PROF_GEMV_GATE_UP, PROF_GEMV_DOWN, PROF_GEMV_HEAD = 16, 17, 18, 19, 20
OPT_FIRST_WAIT_POLLS = 1
OPT_FAIL_AFTER_LAUNCHES = 2
OPT_RESIDENT_LAYERS = 3
OPT_STREAM_SLOTS = 4
OPT_L2_AHEAD_BYTES = 5
OPT_L2_AHEAD_O_BYTES = 6

EXPORTS = [
    "prima_ctx_create", "prima_ctx_destroy", "prima_load_q4k_weights", "prima_forward_window", "prima_logits",
    "prima_embed", "prima_argmax", "prima_kv_load", "prima_kv_read", "prima_sync", "prima_last_error",
    "prima_launch_count", "prima_profile_enable", "prima_profile_read", "prima_dequant_q4k", "prima_gemv_q4k", "prima_gemv_plan_create", "prima_gemv_plan_run",
    "prima_gemv_plan_destroy", "prima_gemv_q4k_noalloc", "prima_gemv_q4k_noalloc_error",
    "prima_forward_window_seqs", "prima_kv_load_seq", "prima_kv_read_seq", "prima_ctx_set_option", "prima_stream_stats",
    "prima_fmt_block_weights", "prima_fmt_block_bytes", "prima_dequant_fmt", "prima_gemv_fmt", "prima_fmt_last_error",
    "prima_paged_create", "prima_paged_destroy", "prima_paged_sync", "prima_paged_append", "prima_paged_accept", "prima_paged_reorder",
    "prima_tree_attention", "prima_tree_attention_workspace", "prima_beam_select", "prima_beam_select_workspace", "prima_forward_window_paged",
]


class ModelConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab",
                                         "kv_capacity", "max_n_tok")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float), ("rope_mode", C.c_int32), ("device", C.c_int32)]


class PagedConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")] + \
               [("rope_theta", C.c_float), ("rope_mode", C.c_int32), ("device", C.c_int32)]


class PagedBatchDesc(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("n_tok", C.c_int32), ("row_begin", C.c_void_p), ("ctx_len", C.c_void_p), ("table", C.c_void_p),
                ("table_stride", C.c_int64), ("pos", C.c_void_p), ("mask", C.c_void_p), ("mask_words", C.c_int32)]


class PrimaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"prima error {code}: {msg}")
        self.code = code


_lib = None


def lib():
    """Load the C-ABI library; raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_08791_b200.build` (`--bounds` for the range-checked one) "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
        L.prima_ctx_create.argtypes = [C.POINTER(ModelConfig), vp, C.POINTER(vp)]
        L.prima_ctx_destroy.argtypes = [vp]
        L.prima_load_q4k_weights.argtypes = [vp, i32, i32, vp, i64, i64, i64]
        L.prima_forward_window.argtypes = [vp, i32, i32, vp, vp, i32, i32]
        L.prima_logits.argtypes = [vp, vp, i32, vp]
        L.prima_embed.argtypes = [vp, vp, i32, vp]
        L.prima_argmax.argtypes = [vp, vp, i32, vp]
        L.prima_kv_load.argtypes = [vp, i32, i32, i32, vp, vp]
        L.prima_kv_read.argtypes = [vp, i32, i32, i32, vp, vp]
        L.prima_forward_window_seqs.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32]
        L.prima_kv_load_seq.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.prima_kv_read_seq.argtypes = [vp, i32, i32, i32, i32, vp, vp]
        L.prima_sync.argtypes = [vp]
        L.prima_ctx_set_option.argtypes = [vp, i32, i64]
        L.prima_stream_stats.argtypes = [vp, C.POINTER(i64), C.POINTER(C.c_double)]
        L.prima_last_error.argtypes = [vp]
        L.prima_last_error.restype = C.c_char_p
        L.prima_launch_count.argtypes = [vp]
        L.prima_launch_count.restype = i64
        L.prima_profile_enable.argtypes = [vp, i32]
        L.prima_profile_read.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(i64), C.POINTER(i64)]
        L.prima_dequant_q4k.argtypes = [vp, i64, vp, vp]
        L.prima_gemv_q4k.argtypes = [vp, i64, i64, vp, i32, vp, vp]
        L.prima_gemv_plan_create.argtypes = [vp, i64, i64, i32, C.POINTER(vp)]
        L.prima_gemv_plan_run.argtypes = [vp, vp, i32, vp, vp]
        L.prima_gemv_plan_destroy.argtypes = [vp]
        L.prima_fmt_block_weights.argtypes = [i32]
        L.prima_fmt_block_bytes.argtypes = [i32]
        L.prima_dequant_fmt.argtypes = [i32, vp, i64, vp, vp]
        L.prima_gemv_fmt.argtypes = [i32, vp, i64, i64, vp, i32, vp, vp]
        L.prima_fmt_last_error.argtypes = []
        L.prima_fmt_last_error.restype = C.c_char_p
        L.prima_gemv_q4k_noalloc.argtypes = [vp, i64, i64, vp, i32, vp, vp]
        L.prima_gemv_q4k_noalloc_error.argtypes = []
        L.prima_gemv_q4k_noalloc_error.restype = C.c_char_p
        L.prima_paged_create.argtypes = [C.POINTER(PagedConfig), vp, vp, C.POINTER(vp)]
        L.prima_paged_destroy.argtypes = [vp]
        L.prima_paged_sync.argtypes = [vp, vp]
        L.prima_paged_append.argtypes = [vp, i32, vp, vp, vp, vp, i32, i32, i64, i64, i64, vp, vp]
        L.prima_paged_accept.argtypes = [vp, vp, vp, vp, i32, vp]
        L.prima_paged_reorder.argtypes = [vp, i32, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp]
        L.prima_tree_attention.argtypes = [vp, i32, vp, vp, i32, C.c_float, vp, i32, vp, vp, i64, vp]
        L.prima_tree_attention_workspace.argtypes = [vp, i32, i32, i32]
        L.prima_tree_attention_workspace.restype = i64
        L.prima_beam_select.argtypes = [vp, i32, i32, i32, i32, i64, vp, vp, i32, i32, vp, vp, vp, vp, i64, vp]
        L.prima_forward_window_paged.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.prima_beam_select_workspace.argtypes = [i32, i32, i32, i32]
        L.prima_beam_select_workspace.restype = i64
        for name in EXPORTS:
            if name not in ("prima_last_error", "prima_launch_count", "prima_gemv_q4k_noalloc_error", "prima_fmt_last_error",
                            "prima_tree_attention_workspace", "prima_beam_select_workspace"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(rc: int, ctx=None):
    if rc != OK:
        msg = lib().prima_last_error(ctx)
        raise PrimaError(rc, msg.decode() if msg else "")


def _dev_ptr(t):
    """Raw device pointer of a contiguous torch CUDA tensor."""
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    return C.c_void_p(t.data_ptr())


def _stream_ptr(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _host_ptr(a: np.ndarray):
    return C.c_void_p(a.ctypes.data)


# -------------------------------------------------------------------------------------------------
def prima_dequant_q4k(dev_blocks, n_superblocks: int, dev_out, stream=None):
    _check(lib().prima_dequant_q4k(_dev_ptr(dev_blocks), n_superblocks, _dev_ptr(dev_out), _stream_ptr(stream)))


def prima_gemv_q4k(dev_w, rows: int, cols: int, dev_x, n_cols: int, dev_y, stream=None):
    _check(lib().prima_gemv_q4k(_dev_ptr(dev_w), rows, cols, _dev_ptr(dev_x), n_cols, _dev_ptr(dev_y), _stream_ptr(stream)))


FMT_Q4_K, FMT_Q6_K, FMT_Q8_0, FMT_F16 = 0, 1, 2, 3


def _check_fmt(rc: int):
    if rc != OK:
        msg = lib().prima_fmt_last_error() or lib().prima_last_error(None)
        raise PrimaError(rc, msg.decode() if msg else "")


def prima_dequant_fmt(fmt: int, dev_blocks, n_blocks: int, dev_out, stream=None):
    _check_fmt(lib().prima_dequant_fmt(fmt, _dev_ptr(dev_blocks), n_blocks, _dev_ptr(dev_out), _stream_ptr(stream)))


def prima_gemv_fmt(fmt: int, dev_w, rows: int, cols: int, dev_x, n_cols: int, dev_y, stream=None):
    _check_fmt(lib().prima_gemv_fmt(fmt, _dev_ptr(dev_w), rows, cols, _dev_ptr(dev_x), n_cols, _dev_ptr(dev_y), _stream_ptr(stream)))


def prima_gemv_q4k_noalloc(dev_w, rows: int, cols: int, dev_x, n_cols: int, dev_y, stream=None):
    """Matrix-vector product that allocates nothing (for callers that own all device memory themselves).

    Same arguments as ``prima_gemv_q4k``; limited to rows*(cols/256)*n_cols <= 4,194,304; queues its
    kernels on the stream and returns without waiting.  Calls on one device must not overlap."""
    rc = lib().prima_gemv_q4k_noalloc(_dev_ptr(dev_w), rows, cols, _dev_ptr(dev_x), n_cols, _dev_ptr(dev_y), _stream_ptr(stream))
    if rc != OK:
        raise PrimaError(rc, lib().prima_gemv_q4k_noalloc_error().decode())


class GemvPlan:
    """prima_gemv_plan_create / _run / _destroy."""

    def __init__(self, dev_w, rows: int, cols: int, max_n_cols: int = 1):
        self._h = C.c_void_p()
        self.rows, self.cols = rows, cols
        _check(lib().prima_gemv_plan_create(_dev_ptr(dev_w), rows, cols, max_n_cols, C.byref(self._h)))

    def run(self, dev_x, n_cols: int, dev_y, stream=None):
        _check(lib().prima_gemv_plan_run(self._h, _dev_ptr(dev_x), n_cols, _dev_ptr(dev_y), _stream_ptr(stream)))

    def close(self):
        if self._h:
            lib().prima_gemv_plan_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Context:
    """prima_ctx_* : one model (or one window's worth of layers) resident on one GPU."""

    def __init__(self, cfg: dict, device: int = 0, stream=None):
        self.cfg = dict(cfg)
        mc = ModelConfig(cfg["n_layers"], cfg["hidden"], cfg["n_q_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["ffn"],
                         cfg["vocab"], cfg["kv_capacity"], cfg.get("max_n_tok", MAX_N_TOK), cfg["rms_eps"], cfg["rope_theta"],
                         cfg.get("rope_mode", 0), device)
        self._h = C.c_void_p()
        if stream is None:
            import torch
            stream = torch.cuda.current_stream()
        self._stream = stream      # what follows the context's steps has to run on it, whatever is current by then
        _check(lib().prima_ctx_create(C.byref(mc), _stream_ptr(stream), C.byref(self._h)))

    def close(self):
        if self._h:
            lib().prima_ctx_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def load(self, layer: int, tensor_id: int, data, rows: int, cols: int):
        """prima_load_q4k_weights; ``data`` is a numpy array (host) or a torch CUDA tensor."""
        if isinstance(data, np.ndarray):
            data = np.ascontiguousarray(data)
            ptr, nbytes = _host_ptr(data), data.nbytes
        else:
            ptr, nbytes = _dev_ptr(data), data.numel() * data.element_size()
        _check(lib().prima_load_q4k_weights(self._h, layer, tensor_id, ptr, rows, cols, nbytes), self._h)

    def forward_window(self, layer_begin: int, layer_end: int, hidden_in, hidden_out, pos: int, n_tok: int):
        _check(lib().prima_forward_window(self._h, layer_begin, layer_end, _dev_ptr(hidden_in), _dev_ptr(hidden_out), pos, n_tok),
               self._h)

    def logits(self, hidden, n_tok: int, logits_out):
        _check(lib().prima_logits(self._h, _dev_ptr(hidden), n_tok, _dev_ptr(logits_out)), self._h)

    def embed(self, tokens, hidden_out):
        tokens = np.ascontiguousarray(tokens, dtype=np.int32).reshape(-1)
        _check(lib().prima_embed(self._h, _host_ptr(tokens), tokens.size, _dev_ptr(hidden_out)), self._h)

    def argmax(self, logits, n_tok: int) -> np.ndarray:
        out = np.zeros(n_tok, np.int32)
        _check(lib().prima_argmax(self._h, _dev_ptr(logits), n_tok, _host_ptr(out)), self._h)
        return out

    def kv_load(self, layer: int, pos_begin: int, k_bits: np.ndarray, v_bits: np.ndarray, seq: int = 0):
        k_bits = np.ascontiguousarray(k_bits, dtype=np.uint16)
        v_bits = np.ascontiguousarray(v_bits, dtype=np.uint16)
        _check(lib().prima_kv_load_seq(self._h, seq, layer, pos_begin, k_bits.shape[0], _host_ptr(k_bits), _host_ptr(v_bits)), self._h)

    def kv_read(self, layer: int, pos_begin: int, n_pos: int, seq: int = 0):
        shape = (n_pos, self.cfg["n_kv_heads"], self.cfg["head_dim"])
        k, v = np.empty(shape, np.uint16), np.empty(shape, np.uint16)
        _check(lib().prima_kv_read_seq(self._h, seq, layer, pos_begin, n_pos, _host_ptr(k), _host_ptr(v)), self._h)
        return k, v

    def forward_window_seqs(self, layer_begin: int, layer_end: int, hidden_in, hidden_out, seqs, positions):
        """prima_forward_window_seqs: one token of each of several independent requests."""
        seqs = np.ascontiguousarray(seqs, dtype=np.int32).reshape(-1)
        positions = np.ascontiguousarray(positions, dtype=np.int32).reshape(-1)
        if seqs.size != positions.size:
            raise ValueError("one position per sequence")
        _check(lib().prima_forward_window_seqs(self._h, layer_begin, layer_end, _dev_ptr(hidden_in), _dev_ptr(hidden_out),
                                               _host_ptr(seqs), _host_ptr(positions), seqs.size), self._h)

    def forward_window_paged(self, pool: "PagedCache", layer_begin: int, layer_end: int, hidden_in, hidden_out, batch: "PagedBatch"):
        """prima_forward_window_paged: the rows of a batch of sequences over a paged cache."""
        for name, t in (("hidden_in", hidden_in), ("hidden_out", hidden_out)):
            if t.dim() != 2 or t.shape[0] < batch.n_tok or t.shape[1] != self.cfg["hidden"]:
                raise ValueError(f"{name}: expected [{batch.n_tok}, {self.cfg['hidden']}], got {tuple(t.shape)}")
        _check(lib().prima_forward_window_paged(self._h, pool._h, layer_begin, layer_end, _dev_ptr(hidden_in), _dev_ptr(hidden_out), pool._batch(batch)), self._h)

    def sync(self):
        _check(lib().prima_sync(self._h), self._h)

    def set_option(self, option: int, value: int):
        _check(lib().prima_ctx_set_option(self._h, option, value), self._h)

    def stream_stats(self):
        """(bytes copied host-to-device for streamed layers, summed copy time in ms)."""
        b, ms = C.c_int64(), C.c_double()
        _check(lib().prima_stream_stats(self._h, C.byref(b), C.byref(ms)), self._h)
        return b.value, ms.value

    def profile_enable(self, mode):
        """0 / False: off; 1 / True: events around every launch (isolated kernels); 2: in-situ stamps."""
        _check(lib().prima_profile_enable(self._h, int(mode)), self._h)

    def profile_read(self, klass: int):
        """(milliseconds, launches, algorithmic bytes) recorded for one kernel class."""
        ms, n, b = C.c_double(), C.c_int64(), C.c_int64()
        _check(lib().prima_profile_read(self._h, klass, C.byref(ms), C.byref(n), C.byref(b)), self._h)
        return ms.value, n.value, b.value

    def launch_count(self) -> int:
        return int(lib().prima_launch_count(self._h))

    def last_error(self) -> str:
        return lib().prima_last_error(self._h).decode()


# ---- several candidate continuations over one paged cache ------------------------------------------------
DT_F32, DT_F16, DT_BF16 = 0, 1, 2


_DTYPES: dict = {}      # torch type -> code, filled at the first use (torch is imported late)


def _dtype_code(t) -> int:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: DT_F32, torch.float16: DT_F16, torch.bfloat16: DT_BF16})
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"expected float32, float16 or bfloat16, got {t.dtype}")
    return code


def _need(t, name: str, dtype, shape, device):
    """Checks a contiguous CUDA tensor of a plain argument; returns its address."""
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _stream_of(stream, device):
    """The raw stream: torch's current one on the device unless one is given."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index)


def _scratch(n_bytes: int, device, stream):
    """A workspace for one call.  It comes from torch's allocator on the stream that the call runs on, so that it is
    reused only behind the call (and lies in the graph's own pool under capture)."""
    import torch
    if stream is None:
        return torch.empty(n_bytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(n_bytes, dtype=torch.uint8, device=device)


class PagedBatch:
    """prima_paged_batch: the sequences of a step, their page tables and the rows that belong to them.

    ``table`` int32 [n_seq, pages], ``row_begin`` int32 [n_seq + 1], ``ctx_len`` int32 [n_seq], ``pos`` int32 [n_tok]
    or None, ``mask`` int64 [n_tok, words] (bits) or None: contiguous CUDA tensors, read when the kernels run.  One
    batch serves every layer of a step."""

    def __init__(self, table, row_begin, ctx_len, n_tok: int, pos=None, mask=None):
        import torch
        i32, n_seq, dev = torch.int32, ctx_len.numel(), ctx_len.device
        if table.dim() != 2 or not table.is_cuda:
            raise ValueError("table: expected a CUDA tensor [n_seq, pages]")
        self.device, self.n_seq, self.n_tok = dev, n_seq, int(n_tok)
        self._keep = (table, row_begin, ctx_len, pos, mask)
        words = 0
        if mask is not None:
            if mask.dim() != 2 or mask.shape[1] < 1:      # without words it has no address, which would read as no mask
                raise ValueError("mask: expected [n_tok, words]")
            words = mask.shape[1]
        self.desc = PagedBatchDesc(n_seq, self.n_tok, _need(row_begin, "row_begin", i32, (n_seq + 1,), dev), _need(ctx_len, "ctx_len", i32, (n_seq,), dev),
                                   _need(table, "table", i32, (n_seq, table.shape[1]), dev), table.shape[1],
                                   _need(pos, "pos", i32, (self.n_tok,), dev) if pos is not None else None,
                                   _need(mask, "mask", torch.int64, (self.n_tok, words), dev) if mask is not None else None, words)
        self._ref = C.byref(self.desc)


class PagedCache:
    """prima_paged_*: a paged cache over two caller-owned tensors [n_layers, n_pages, n_kv_heads, page_size, head_dim]."""

    def __init__(self, k_pages, v_pages, rope_theta: float = 1e4, rope_mode: int = 0):
        if k_pages.dim() != 5 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype or k_pages.device != v_pages.device:
            raise ValueError("k_pages and v_pages: two tensors [n_layers, n_pages, n_kv_heads, page_size, head_dim] of one type on one device")
        kp, vp = _dev_ptr(k_pages), _dev_ptr(v_pages)
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k_pages.shape
        self.dtype, self.device = k_pages.dtype, k_pages.device
        self._keep = (k_pages, v_pages)
        import torch
        self._i32, self._f32 = torch.int32, torch.float32
        self._code = _dtype_code(k_pages)
        self._h = C.c_void_p()
        cfg = PagedConfig(*k_pages.shape[:2], self.page_size, self.n_kv_heads, self.head_dim, self._code, rope_theta, rope_mode, self.device.index)
        self._lib = lib()
        _check(self._lib.prima_paged_create(C.byref(cfg), kp, vp, C.byref(self._h)))

    def close(self):
        if self._h:
            lib().prima_paged_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t, name: str, n_tok: int, heads: int, dtype):
        """(address, elements from token to token) of [n_tok, heads, head_dim] with adjacent heads."""
        stride = t.stride()
        if t.shape != (n_tok, heads, self.head_dim) or t.dtype != dtype or t.device != self.device or stride[2] != 1 or (heads > 1 and stride[1] != self.head_dim):
            raise ValueError(f"{name}: expected {dtype} [{n_tok}, {heads}, {self.head_dim}] on {self.device} with adjacent heads, got {t.dtype} {tuple(t.shape)} on {t.device}, strides {stride}")
        return t.data_ptr(), (stride[0] if n_tok > 1 else heads * self.head_dim)

    def _batch(self, batch: PagedBatch):
        if batch.device != self.device:
            raise ValueError("the batch is on another device than the cache")
        return batch._ref

    def append(self, layer: int, batch: PagedBatch, q, k, v, q_out=None, stream=None):
        """prima_paged_append: rotate q (or None) and k, write q_out, append k and v to ``layer``."""
        n, dt = batch.n_tok, k.dtype
        kp, ks = self._rows(k, "k", n, self.n_kv_heads, dt)
        vp, vs = self._rows(v, "v", n, self.n_kv_heads, dt)
        qp = qo = None
        qs = heads = 0
        if q is not None:
            heads = q.shape[1]
            qp, qs = self._rows(q, "q", n, heads, dt)
            if q_out is None:
                raise ValueError("q_out: expected a tensor")
            qo = _need(q_out, "q_out", self.dtype, (n, heads, self.head_dim), self.device)
        rc = self._lib.prima_paged_append(self._h, layer, self._batch(batch), qp, kp, vp, _dtype_code(k), heads, qs, ks, vs, qo, _stream_of(stream, self.device))
        if rc:
            _check(rc)

    def tree_attention_workspace(self, batch: PagedBatch, n_q_heads: int = 0, stream=None):
        """A workspace for ``tree_attention`` (for any number of query heads if none is named); calls that may overlap need one each."""
        n = lib().prima_tree_attention_workspace(self._h, batch.n_seq, batch.n_tok, n_q_heads or 64 * self.n_kv_heads)
        if n < 0:
            raise PrimaError(n, "prima_tree_attention_workspace")
        return _scratch(n, self.device, stream)

    def tree_attention(self, layer: int, batch: PagedBatch, q, out, scale=None, lse=None, workspace=None, stream=None):
        """prima_tree_attention; ``scale`` defaults to head_dim ** -0.5."""
        heads = q.shape[1] if q.dim() == 3 else 0
        shape = (batch.n_tok, heads, self.head_dim)
        qp = _need(q, "q", self.dtype, shape, self.device)
        op = _need(out, "out", out.dtype, shape, self.device)
        lp = _need(lse, "lse", self._f32, shape[:2], self.device) if lse is not None else None
        if workspace is None:
            workspace = self.tree_attention_workspace(batch, heads, stream)
        elif workspace.device != self.device or not workspace.is_contiguous():
            raise ValueError(f"workspace: expected a contiguous tensor on {self.device}")
        rc = self._lib.prima_tree_attention(self._h, layer, self._batch(batch), qp, heads, self.head_dim ** -0.5 if scale is None else scale, op, _dtype_code(out), lp,
                                            workspace.data_ptr(), workspace.nbytes, _stream_of(stream, self.device))
        if rc:
            _check(rc)

    def accept(self, batch: PagedBatch, path, path_len, stream=None):
        """prima_paged_accept: ``path`` int32 [n_seq, longest], ``path_len`` int32 [n_seq]."""
        if path.dim() != 2:
            raise ValueError("path: expected [n_seq, longest path]")
        pp = _need(path, "path", self._i32, (batch.n_seq, path.shape[1]), self.device)
        pl = _need(path_len, "path_len", self._i32, (batch.n_seq,), self.device)
        _check(self._lib.prima_paged_accept(self._h, self._batch(batch), pp, pl, path.shape[1], _stream_of(stream, self.device)))

    def reorder(self, table, length, parent, fresh, table_out, length_out, stream=None):
        """prima_paged_reorder: ``parent`` int32 [n_req, keep]; ``table`` int32 [n_req * n_beams, pages]; ``fresh`` int32 [n_req * keep]."""
        n_req, keep = parent.shape
        rows, pages = table.shape
        if rows % n_req:
            raise ValueError("table: expected a row for every beam of every request")
        dev, i32, new = self.device, self._i32, n_req * keep
        _check(self._lib.prima_paged_reorder(self._h, n_req, rows // n_req, keep, _need(table, "table", i32, (rows, pages), dev), pages,
                                             _need(length, "length", i32, (rows,), dev), _need(parent, "parent", i32, (n_req, keep), dev),
                                             _need(fresh, "fresh", i32, (new,), dev), _need(table_out, "table_out", i32, (new, pages), dev),
                                             _need(length_out, "length_out", i32, (new,), dev), _stream_of(stream, dev)))

    def sync(self, stream=None):
        """Waits; raises if a kernel met a bad page, slot, row or path since the last call."""
        _check(lib().prima_paged_sync(self._h, _stream_of(stream, self.device)))


def prima_beam_select_workspace(n_req: int, n_beams: int, vocab: int, keep: int, device=None, stream=None):
    """A workspace for ``prima_beam_select``; calls that may overlap need one each."""
    n = lib().prima_beam_select_workspace(n_req, n_beams, vocab, keep)
    if n < 0:
        raise PrimaError(n, "prima_beam_select_workspace: sizes out of range")
    return _scratch(n, device if device is not None else "cuda", stream)


def prima_beam_select(logits, cum, score, parent, token, finished=None, end_token: int = -1, workspace=None, stream=None):
    """prima_beam_select: ``logits`` [n_req, n_beams, vocab] (rows may be padded), ``cum`` fp32 [n_req, n_beams],
    outputs ``score`` fp32, ``parent`` and ``token`` int32 [n_req, keep]."""
    import torch
    shape, step = logits.shape, logits.stride()
    if len(shape) != 3 or not logits.is_cuda or step[2] != 1 or (shape[0] > 1 and shape[1] > 1 and step[0] != shape[1] * step[1]):
        raise ValueError("logits: expected a CUDA tensor [n_req, n_beams, vocab] with evenly spaced rows")
    n_req, n_beams, vocab = shape
    dev, keep = logits.device, score.shape[-1]
    beams, kept, f32, i32 = (n_req, n_beams), (n_req, keep), torch.float32, torch.int32
    if workspace is None:
        workspace = prima_beam_select_workspace(n_req, n_beams, vocab, keep, dev, stream)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on {dev}")
    stride = step[1] if n_beams > 1 else step[0] if n_req > 1 else vocab
    args = (logits.data_ptr(), _dtype_code(logits), n_req, n_beams, vocab, stride, _need(cum, "cum", f32, beams, dev),
            _need(finished, "finished", torch.uint8, beams, dev) if finished is not None else None, end_token, keep, _need(score, "score", f32, kept, dev),
            _need(parent, "parent", i32, kept, dev), _need(token, "token", i32, kept, dev), workspace.data_ptr(), workspace.nbytes, _stream_of(stream, dev))
    if torch._C._cuda_getDevice() == dev.index:
        rc = lib().prima_beam_select(*args)
    else:
        with torch.cuda.device(dev):
            rc = lib().prima_beam_select(*args)
    if rc:
        _check(rc)

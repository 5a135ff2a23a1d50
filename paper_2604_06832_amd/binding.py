"""Thin ctypes binding of libbd.so (include/bd.h, include/bd_kernels.h).

Argument marshalling only: every step of the decode path runs inside the library's HIP kernels.
PyTorch tensors are used as device buffers; their data pointers are handed over as plain pointers.
There is no fallback: if the shared library is missing, importing `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbd.so")

BD_OK, BD_E_ARG, BD_E_STATE, BD_E_CAPACITY, BD_E_DTYPE, BD_E_HIP = 0, -1, -2, -3, -4, -5
BD_F32, BD_BF16, BD_FP8_E4M3 = 0, 1, 2
BD_MODE_BIDIR, BD_MODE_CAUSAL = 0, 1
BD_FLAG_CHIP_WIDE_HANDOVER, BD_FLAG_REGISTER_RING, BD_FLAG_PREFILL_DECODE, BD_FLAG_PREFILL_STAGED = 1, 2, 4, 8
BD_FLAG_ATTENTION_KEY_SPLIT = 16
BD_FLAG_MEASURE_NO_WEIGHTS = 32
BD_KV8_PAGE, BD_KV8_BAD_ROWS, BD_KV8_BAD_PAGE = 32, 1, 2
BD_ROPE_HALF, BD_ROPE_INTERLEAVED = 0, 1
BD_ROPE_PLAIN, BD_ROPE_LINEAR, BD_ROPE_BASE, BD_ROPE_PARTS = 0, 1, 2, 3

# every symbol the two headers declare
EXPORTS = [
    "bd_create", "bd_destroy", "bd_load_weight", "bd_prefill", "bd_denoise_step", "bd_commit_block",
    "bd_verify_block", "bd_decode_block", "bd_speculative_step", "bd_quad_draft", "bd_quad_step", "bd_crop", "bd_cache_len", "bd_status", "bd_debug_logits", "bd_read_logits", "bd_read_kv",
    "bd_read_carry", "bd_read_rows", "bd_forward_bytes", "bd_strerror", "bd_last_error",
    "bd_k_attention", "bd_k_attention_static", "bd_k_profile", "bd_k_profile_read", "bd_k_class_count", "bd_k_class_name",
    "bd_k_class_bytes", "bd_k_trace", "bd_k_trace_read", "bd_k_stream_floor", "bd_kv_page_order", "bd_kv_pages", "bd_k_raise_device_error",
    "bd_k_kv8_write", "bd_k_kv8_read", "bd_k_kv8_attention", "bd_k_kv8_attention_workspace", "bd_k_rope", "bd_k_rope_plan",
]


class bd_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab")] + \
               [("rope_theta", C.c_float), ("rms_eps", C.c_float)] + \
               [(n, C.c_int32) for n in ("max_seq", "max_block", "mask_token_id", "weight_dtype", "flags")]


class bd_kv8(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dev_codes", "dev_scales", "dev_pages", "dev_len", "dev_status")] + \
               [(n, C.c_int32) for n in ("n_pages", "n_kv", "D", "n_seq", "max_blocks")]


class bd_rope(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("D", "rotary_dim", "layout")] + [("amplitude", C.c_float), ("inv_freq", C.c_double * 64)]


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    L = C.CDLL(LIB_PATH)
    vp, i32, f32 = C.c_void_p, C.c_int, C.c_float
    L.bd_create.argtypes = [C.POINTER(bd_config), vp, C.POINTER(vp)]
    L.bd_destroy.argtypes = [vp]
    L.bd_destroy.restype = None
    L.bd_load_weight.argtypes = [vp, C.c_char_p, vp, C.c_size_t, i32, vp]
    L.bd_prefill.argtypes = [vp, vp, i32, vp, i32]
    L.bd_denoise_step.argtypes = [vp, vp, vp, i32, f32, i32, vp, vp]
    L.bd_commit_block.argtypes = [vp, vp, i32]
    L.bd_verify_block.argtypes = [vp, vp, i32, i32, vp, vp]
    L.bd_decode_block.argtypes = [vp, i32, f32, i32, vp, vp]
    L.bd_quad_draft.argtypes = [vp, i32, vp]
    L.bd_quad_step.argtypes = [vp, i32, vp, vp, C.POINTER(C.c_int32)]
    L.bd_speculative_step.argtypes = [vp, i32, vp, C.POINTER(C.c_int32)]
    L.bd_crop.argtypes = [vp, i32]
    L.bd_cache_len.argtypes = [vp]
    L.bd_status.argtypes = [vp]
    L.bd_debug_logits.argtypes = [vp, i32]
    L.bd_read_logits.argtypes = [vp, vp, i32]
    L.bd_read_kv.argtypes = [vp, i32, i32, i32, vp, vp]
    L.bd_read_carry.argtypes = [vp, vp, vp]
    L.bd_read_rows.argtypes = [vp, vp, vp, i32]
    L.bd_forward_bytes.argtypes = [vp]
    L.bd_forward_bytes.restype = C.c_int64
    L.bd_strerror.argtypes = [i32]
    L.bd_strerror.restype = C.c_char_p
    L.bd_last_error.argtypes = []
    L.bd_last_error.restype = C.c_char_p
    L.bd_k_attention.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, i32, C.POINTER(f32)]
    L.bd_k_attention_static.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp]
    L.bd_k_profile.argtypes = [vp, i32]
    L.bd_k_profile_read.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(i32)]
    L.bd_k_class_count.argtypes = []
    L.bd_k_class_name.argtypes = [i32]
    L.bd_k_class_name.restype = C.c_char_p
    L.bd_k_class_bytes.argtypes = [vp, i32]
    L.bd_k_class_bytes.restype = C.c_int64
    L.bd_k_trace.argtypes = [vp, i32]
    L.bd_kv_page_order.argtypes = [vp, vp, i32]
    L.bd_kv_pages.argtypes = [vp, vp, i32]
    L.bd_k_raise_device_error.argtypes = [vp]
    L.bd_k_stream_floor.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    L.bd_k_trace_read.argtypes = [vp, vp, i32, C.POINTER(i32), C.POINTER(i32)]
    i64 = C.c_int64
    L.bd_k_kv8_write.argtypes = [vp, vp, vp, i64, i64, vp, i64, i64, i32, i32, vp]
    L.bd_k_kv8_read.argtypes = [vp, vp, vp, i32, vp, i32, vp, i64, i64, vp, i64, i64]
    L.bd_k_kv8_attention.argtypes = [vp, vp, vp, i64, i64, i32, i32, vp, i32, i32, i32, f32, vp, i64, i64, vp, i64]
    L.bd_k_kv8_attention_workspace.argtypes = [vp, i32, i32, i32, i32]
    L.bd_k_kv8_attention_workspace.restype = i64
    L.bd_k_rope_plan.argtypes = [vp, i32, i32, i32, C.c_double, i32, C.c_double, i32]
    L.bd_k_rope.argtypes = [vp, vp, vp, i64, i64, vp, i64, i64, i32, i32, i32, i32, vp, vp]
    _lib = L
    return L


class BdError(RuntimeError):
    """workspace: BD_E_CAPACITY of a call that has no cache of its own to exceed, whose text says what it needs."""

    def __init__(self, code: int, workspace: bool = False):
        L = lib()
        msg = L.bd_strerror(code).decode()
        if code == BD_E_HIP:
            msg += ": " + L.bd_last_error().decode()
        elif code == BD_E_CAPACITY and workspace:
            msg = L.bd_last_error().decode()
        super().__init__(f"bd error {code}: {msg}")
        self.code = code


def _check(code: int) -> int:
    if code < 0:
        raise BdError(code)
    return code


def _ptr(t) -> Optional[int]:
    """Device pointer of a torch tensor (None passes NULL)."""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    return t.data_ptr()


class Context:
    """One decode context = one bd_ctx.  Methods carry the names of the C calls they wrap."""

    def __init__(self, shape, max_seq: int, max_block: int, weight_dtype: int = BD_BF16, stream=None, flags: int = 0):
        import torch
        self.shape = shape
        cfg = bd_config(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn,
                        shape.vocab, shape.rope_theta, shape.rms_eps, max_seq, max_block, shape.mask_token_id,
                        weight_dtype, flags)
        self._stream = stream if stream is not None else torch.cuda.current_stream()
        h = C.c_void_p()
        _check(lib().bd_create(C.byref(cfg), C.c_void_p(self._stream.cuda_stream), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().bd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:       # interpreter shutdown: the module globals may already be gone
            pass

    # -- weights ------------------------------------------------------------------------------------------
    def bd_load_weight(self, name: str, arr: np.ndarray, scales: Optional[np.ndarray] = None):
        arr = np.ascontiguousarray(arr)
        dt = {np.dtype(np.float32): BD_F32, np.dtype(np.uint16): BD_BF16, np.dtype(np.uint8): BD_FP8_E4M3}[arr.dtype]
        sp = None
        if scales is not None:
            scales = np.ascontiguousarray(scales, dtype=np.float32)
            sp = scales.ctypes.data
        _check(lib().bd_load_weight(self._h, name.encode(), arr.ctypes.data, arr.nbytes, dt, sp))

    def load_model(self, weights: Dict[str, np.ndarray], as_bf16_bits: bool = True):
        """Upload every tensor of an inputs.make_weights() dict (matrices as bf16 bit patterns when they are
        already bf16-representable, else as fp32, which the library rounds)."""
        from . import inputs
        # gain vectors first: the library folds each into the matrices it feeds
        order = sorted(weights.items(), key=lambda kv: kv[1].ndim != 1)
        for name, w in order:
            if name.endswith(".scale"):
                continue
            if w.dtype == np.uint8:
                self.bd_load_weight(name, w, weights[name + ".scale"])
            elif w.ndim == 1 or not as_bf16_bits:
                self.bd_load_weight(name, w.astype(np.float32, copy=False))
            else:
                self.bd_load_weight(name, inputs.bf16_bits(w))

    # -- decode calls --------------------------------------------------------------------------------------
    def bd_prefill(self, embeds, ids):
        n_e = 0 if embeds is None else embeds.shape[0]
        n_i = 0 if ids is None else ids.shape[0]
        _check(lib().bd_prefill(self._h, _ptr(embeds), n_e, _ptr(ids), n_i))

    def bd_denoise_step(self, tokens, mask, threshold: float, fixed_k: int = 0, n_unmasked=None, conf_out=None):
        _check(lib().bd_denoise_step(self._h, _ptr(tokens), _ptr(mask), tokens.shape[0], threshold, fixed_k,
                                     _ptr(n_unmasked), _ptr(conf_out)))

    def bd_commit_block(self, tokens):
        _check(lib().bd_commit_block(self._h, _ptr(tokens), tokens.shape[0]))

    def bd_verify_block(self, draft, commit: bool, ar_pred=None, n_accept=None):
        _check(lib().bd_verify_block(self._h, _ptr(draft), draft.shape[0], int(commit), _ptr(ar_pred), _ptr(n_accept)))

    def bd_decode_block(self, B: int, threshold: float, fixed_k: int, tokens_out, steps_out=None):
        _check(lib().bd_decode_block(self._h, B, threshold, fixed_k, _ptr(tokens_out), _ptr(steps_out)))

    def bd_quad_draft(self, B: int, draft_out):
        _check(lib().bd_quad_draft(self._h, B, _ptr(draft_out)))

    def bd_quad_step(self, B: int, draft, next_draft) -> int:
        k = C.c_int32(0)
        _check(lib().bd_quad_step(self._h, B, _ptr(draft), _ptr(next_draft), C.byref(k)))
        return int(k.value)

    def bd_speculative_step(self, B: int, tokens_out) -> int:
        k = C.c_int32(0)
        _check(lib().bd_speculative_step(self._h, B, _ptr(tokens_out), C.byref(k)))
        return int(k.value)

    def bd_crop(self, new_len: int):
        _check(lib().bd_crop(self._h, new_len))

    def bd_cache_len(self) -> int:
        return _check(lib().bd_cache_len(self._h))

    def bd_status(self):
        _check(lib().bd_status(self._h))

    # -- inspection ----------------------------------------------------------------------------------------
    def bd_debug_logits(self, enable: bool):
        _check(lib().bd_debug_logits(self._h, int(enable)))

    def bd_read_logits(self, rows: int):
        import torch
        out = torch.empty((rows, self.shape.vocab), dtype=torch.float32, device="cuda")
        _check(lib().bd_read_logits(self._h, _ptr(out), rows))
        return out

    def bd_read_kv(self, layer: int, pos0: int, count: int):
        import torch
        k = torch.empty((count, self.shape.n_kv_heads, self.shape.head_dim), dtype=torch.float32, device="cuda")
        v = torch.empty_like(k)
        _check(lib().bd_read_kv(self._h, layer, pos0, count, _ptr(k), _ptr(v)))
        return k, v

    def bd_read_carry(self):
        import torch
        cand = torch.empty(1, dtype=torch.int32, device="cuda")
        conf = torch.empty(1, dtype=torch.float32, device="cuda")
        _check(lib().bd_read_carry(self._h, _ptr(cand), _ptr(conf)))
        return int(cand.item()), float(conf.item())

    def bd_read_rows(self, rows: int):
        import torch
        cand = torch.empty(rows, dtype=torch.int32, device="cuda")
        conf = torch.empty(rows, dtype=torch.float32, device="cuda")
        _check(lib().bd_read_rows(self._h, _ptr(cand), _ptr(conf), rows))
        return cand, conf

    def bd_forward_bytes(self) -> int:
        return _check(lib().bd_forward_bytes(self._h))

    # -- per-kernel timing ---------------------------------------------------------------------------------
    def bd_k_profile(self, enable: bool):
        _check(lib().bd_k_profile(self._h, int(enable)))

    def bd_k_profile_read(self):
        """{class name: (total ms, launches, algorithmic bytes per launch)}"""
        L = lib()
        out = {}
        for k in range(L.bd_k_class_count()):
            ms, cnt = C.c_double(), C.c_int()
            _check(L.bd_k_profile_read(self._h, k, C.byref(ms), C.byref(cnt)))
            out[L.bd_k_class_name(k).decode()] = (ms.value, cnt.value, int(L.bd_k_class_bytes(self._h, k)))
        return out


def _trace_methods():
    def bd_k_trace(self, enable: bool):
        _check(lib().bd_k_trace(self._h, int(enable)))

    def bd_kv_page_order(self, order):
        """Order in which free cache pages are handed out: a permutation of range(ceil(max_seq / 32))."""
        o = np.ascontiguousarray(order, dtype=np.int32)
        _check(lib().bd_kv_page_order(self._h, o.ctypes.data, int(o.size)))

    def bd_kv_pages(self):
        """Pages of the blocks in use, in sequence order."""
        n = lib().bd_kv_pages(self._h, None, 0)
        _check(min(n, 0))
        out = np.zeros(max(n, 1), dtype=np.int32)
        lib().bd_kv_pages(self._h, out.ctypes.data, n)
        return out[:n]

    def bd_k_raise_device_error(self):
        _check(lib().bd_k_raise_device_error(self._h))

    def bd_k_stream_floor(self, repeats: int = 10):
        """(milliseconds, bytes) of reading one forward's layer weights with no consumer, hand-over or barrier."""
        ms, nb = C.c_double(0), C.c_int64(0)
        _check(lib().bd_k_stream_floor(self._h, repeats, C.byref(ms), C.byref(nb)))
        return ms.value, nb.value

    def bd_k_trace_read(self):
        """Timestamps (100 MHz ticks) of the last forward, array [n_wg, per_wg]."""
        n_layers = self.shape.n_layers
        cap = 4096 * (10 * n_layers + 4 + 64)
        buf = np.zeros(cap, dtype=np.uint64)
        n_wg, per = C.c_int(), C.c_int()
        _check(lib().bd_k_trace_read(self._h, buf.ctypes.data, cap, C.byref(n_wg), C.byref(per)))
        n1 = n_wg.value * per.value
        self.last_subtrace = buf[n1:n1 + n_wg.value * 64].reshape(n_wg.value, 64)
        return buf[:n1].reshape(n_wg.value, per.value)

    Context.bd_k_trace = bd_k_trace
    Context.bd_k_stream_floor = bd_k_stream_floor
    Context.bd_k_raise_device_error = bd_k_raise_device_error
    Context.bd_kv_page_order = bd_kv_page_order
    Context.bd_kv_pages = bd_kv_pages
    Context.bd_k_trace_read = bd_k_trace_read


_trace_methods()


def bd_k_attention(q, k, v, n_prefix: int, mode: int, iters: int = 1):
    """Block-causal GQA attention on explicit fp32 cuda operands (see include/bd_kernels.h)."""
    import torch
    M, n_q, D = q.shape
    n_kv = k.shape[1]
    out = torch.empty((M, n_q * D), dtype=torch.float32, device="cuda")
    ms = C.c_float(0)
    _check(lib().bd_k_attention(C.c_void_p(torch.cuda.current_stream().cuda_stream), _ptr(q), _ptr(k), _ptr(v), n_prefix,
                                M, n_q, n_kv, D, mode, _ptr(out), iters, C.byref(ms)))
    return out, ms.value


def bd_k_attention_static(q, k, v, n_prefix: int, mode: int, out=None):
    """The same operation through the entry point that allocates nothing (its working buffers are a static device
    array).  `out` (fp32 [M, n_q*D], cuda) is allocated here when not given; the call only enqueues."""
    import torch
    M, n_q, D = q.shape
    n_kv = k.shape[1]
    if out is None:
        out = torch.empty((M, n_q * D), dtype=torch.float32, device="cuda")
    _check(lib().bd_k_attention_static(C.c_void_p(torch.cuda.current_stream().cuda_stream), _ptr(q), _ptr(k), _ptr(v),
                                       n_prefix, M, n_q, n_kv, D, mode, _ptr(out)))
    return out


# -- attention on a key/value cache in 8 bits (include/bd_kernels.h) --------------------------------------------------------
# (A step makes these calls once a layer: what the checks and the call cost on the host counts, 5 to 6 us in all, 2.5 of them the launch.)

_torch = _int32 = _bf16 = _dtypes = _current_device = _current_stream = None


def _with_torch():
    """torch, imported on first use, and what of it every call needs."""
    global _torch, _int32, _bf16, _dtypes, _current_device, _current_stream
    if _torch is None:
        import torch
        _int32, _bf16, _dtypes = torch.int32, torch.bfloat16, {torch.bfloat16: BD_BF16, torch.float32: BD_F32}
        _current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        _torch = torch
    return _torch


# (a number past 32 bits would arrive as another one: ctypes cuts it without a word)
_LEAST, _MOST = -0x80000000, 0x7FFFFFFF


def _check_ints(**numbers):
    for name, x in numbers.items():
        if not _LEAST <= x <= _MOST:
            raise ValueError(f"{name}: {x} is no 32-bit number")


def _check_rows(shape, name, heads, D):
    if len(shape) != 4 or shape[2] != heads or shape[3] != D or shape[1] > _MOST:
        raise ValueError(f"{name}: expected [n_seq, M, {heads}, {D}], got {list(shape)}")


def _rows_of(t, name, heads, D, index):
    """(pointer, stride between sequences, stride between rows) of a tensor of rows [n_seq, M, heads, D] (checked) on device `index`."""
    s0, s1, s2, s3 = t.stride()
    if s3 != 1 or (s2 != D and heads > 1) or t.get_device() != index:
        raise ValueError(f"{name}: heads and dimensions have to be contiguous, on cuda:{index}")
    return t.data_ptr(), s0, s1


def _ints_of(t, name, n_seq, index):
    """Pointer of an int32 tensor with one number for each sequence; None passes NULL."""
    if t is None:
        return None
    if t.dtype is not _int32 or t.numel() != n_seq or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: expected {n_seq} int32 numbers on cuda:{index}")
    return t.data_ptr()


def _dtype_of(t, name):
    dtype = _dtypes.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{name}: bfloat16 or float32, got {t.dtype}")
    return dtype


def _enqueue(index, call, args):
    """call(stream, *args) on the current stream of device `index`."""
    if _current_device() == index:
        code = call(_current_stream(index), *args)
    else:
        with _torch.cuda.device(index):
            code = call(_current_stream(index), *args)
    if code < 0:
        raise BdError(code, workspace=True)


class Kv8Cache:
    """A key/value cache in 8 bits: caller's tensors behind one bd_kv8.  Methods carry the names of the C calls they wrap.

    codes uint8 [n_pages, n_kv, 64 D], scales int32 [n_pages, n_kv], pages int32 [n_seq, max_blocks], lens int32 [n_seq]
    (positions held; moved on by the caller), status None or one int32.  The tensors are kept alive, and looked at when the kernels run: change
    them in place (lens += rows, pages.copy_(...)).  The kernels and captured graphs hold their addresses, so another tensor in the place of one is refused;
    for other tensors make another Kv8Cache."""

    def __setattr__(self, name, value):
        if self.__dict__.get(name, value) is not value:
            raise AttributeError(f"Kv8Cache.{name} is fixed: change the tensor in place, or make another Kv8Cache")
        object.__setattr__(self, name, value)

    def __init__(self, codes, scales, pages, lens, status=None):
        torch = _with_torch()
        if codes.dtype != torch.uint8 or codes.dim() != 3 or not codes.is_cuda or not codes.is_contiguous():
            raise ValueError("codes: expected a contiguous uint8 tensor [n_pages, n_kv, 64 D] on the GPU")
        n_pages, n_kv, size = codes.shape
        index = codes.get_device()
        if scales.dtype != torch.int32 or list(scales.shape) != [n_pages, n_kv] or not scales.is_contiguous() or scales.get_device() != index:
            raise ValueError(f"scales: expected a contiguous int32 tensor [{n_pages}, {n_kv}] on cuda:{index}")
        if pages.dtype != torch.int32 or pages.dim() != 2 or not pages.is_contiguous() or pages.get_device() != index:
            raise ValueError(f"pages: expected a contiguous int32 tensor [n_seq, max_blocks] on cuda:{index}")
        _check_ints(n_seq=pages.shape[0], max_blocks=pages.shape[1])
        self.index, self.n_seq, self.n_kv, self.D = index, pages.shape[0], n_kv, size // 64
        if lens is None:
            raise ValueError("lens: expected one int32 for each sequence")
        self.codes, self.scales, self.pages, self.lens, self.status = codes, scales, pages, lens, status
        self._c = bd_kv8(codes.data_ptr(), scales.data_ptr(), pages.data_ptr(), _ints_of(lens, "lens", self.n_seq, index),
                         _ints_of(status, "status", 1, index), n_pages, n_kv, self.D if size % 64 == 0 else 0, self.n_seq, pages.shape[1])
        self._p = C.addressof(self._c)
        L = lib()
        self._write, self._read, self._attention, self._workspace = (L.bd_k_kv8_write, L.bd_k_kv8_read, L.bd_k_kv8_attention,
                                                                     L.bd_k_kv8_attention_workspace)

    @staticmethod
    def empty(n_pages, n_kv, D, pages, lens, status=None):
        """A cache of n_pages pages that hold nothing yet."""
        torch = _with_torch()
        return Kv8Cache(torch.zeros((n_pages, n_kv, 64 * D), dtype=torch.uint8, device=pages.device),
                        torch.zeros((n_pages, n_kv), dtype=torch.int32, device=pages.device), pages, lens, status)

    def _pair(self, k, v, what):
        """Pointers and strides of keys and values, their type and M."""
        index, heads, D, shape = self.index, self.n_kv, self.D, k.shape
        _check_rows(shape, "keys", heads, D)
        if shape[0] != self.n_seq or v.shape != shape or v.dtype is not k.dtype:
            raise ValueError(f"{what}: keys and values have the same shape, with {self.n_seq} sequences, and type")
        return _rows_of(k, "keys", heads, D, index), _rows_of(v, "values", heads, D, index), _dtype_of(k, "keys"), shape[1]

    def bd_k_kv8_write(self, k, v, rows=None):
        """Keys and values [n_seq, M, n_kv, D] (bfloat16 or float32) to positions lens ..."""
        kp, vp, dtype, M = self._pair(k, v, "bd_k_kv8_write")
        _enqueue(self.index, self._write, (self._p, *kp, *vp, dtype, M, _ints_of(rows, "rows", self.n_seq, self.index)))

    def bd_k_kv8_read(self, start, k_out, v_out, rows=None):
        """Positions start .. (None: from 0) as values, to k_out and v_out [n_seq, M, n_kv, D]."""
        kp, vp, dtype, M = self._pair(k_out, v_out, "bd_k_kv8_read")
        _enqueue(self.index, self._read, (self._p, _ints_of(start, "start", self.n_seq, self.index), M,
                                          _ints_of(rows, "rows", self.n_seq, self.index), dtype, *kp, *vp))

    def bd_k_kv8_attention_workspace(self, n_q, M, window=0, sinks=0) -> int:
        _check_ints(n_q=n_q, M=M, window=window, sinks=sinks)
        return _check(self._workspace(self._p, n_q, M, window, sinks))

    def bd_k_kv8_attention(self, q, out, mode, window=0, sinks=0, scale=0.0, rows=None, workspace=None):
        """Attention of q [n_seq, M, n_q, D] (bfloat16) on the cache, to out (same shape).  workspace: a uint8 tensor of
        bd_k_kv8_attention_workspace bytes that nothing else uses while the call runs; None takes one from torch for this call."""
        shape, index, bf16 = q.shape, self.index, _bf16
        if not (_LEAST <= window <= _MOST and _LEAST <= sinks <= _MOST and _LEAST <= mode <= _MOST):
            _check_ints(window=window, sinks=sinks, mode=mode)
        if len(shape) != 4 or shape[0] != self.n_seq or q.dtype is not bf16 or out.dtype is not bf16 or out.shape != shape:
            raise ValueError(f"q and out: bfloat16 [{self.n_seq}, M, n_q, {self.D}], same shape")
        _, M, n_q, D = shape
        if D != self.D or M > _MOST:
            raise ValueError(f"q: expected [{self.n_seq}, M, n_q, {self.D}], got {list(shape)}")
        qp, op = _rows_of(q, "q", n_q, self.D, index), _rows_of(out, "out", n_q, self.D, index)
        if workspace is None:
            wn = self._workspace(self._p, n_q, M, window, sinks)
            if wn > 0:
                workspace = _torch.empty(wn, dtype=_torch.uint8, device=q.device)
        elif workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError(f"workspace: expected a contiguous tensor on cuda:{index}")
        wp, wn = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
        _enqueue(index, self._attention, (self._p, *qp, n_q, M, _ints_of(rows, "rows", self.n_seq, index), mode, window, sinks, scale, *op, wp, wn))
        return out


def bd_k_rope_plan(D, rotary_dim=None, layout=BD_ROPE_HALF, theta=1.0e6, scaling=BD_ROPE_PLAIN, factor=1.0, trained=1) -> bd_rope:
    """Plan of rotary positions (see include/bd_kernels.h); rotary_dim None: the whole head."""
    plan = bd_rope()
    rotary_dim = D if rotary_dim is None else rotary_dim
    _check_ints(D=D, rotary_dim=rotary_dim, layout=layout, scaling=scaling, trained=trained)
    _check(lib().bd_k_rope_plan(C.addressof(plan), D, rotary_dim, layout, theta, scaling, factor, trained))
    return plan


def bd_k_rope(plan, x, pos, out=None, rows=None):
    """The rows x [n_seq, M, heads, D] turned by their positions pos[s] + row, to out (None: a new tensor; x itself: in place)."""
    if _torch is None:
        _with_torch()
    shape, index = x.shape, x.get_device()
    if len(shape) != 4 or index < 0 or shape[0] > _MOST or shape[1] > _MOST:
        raise ValueError(f"x: expected [n_seq, M, heads, D] on the GPU, got {list(shape)}")
    n, M, heads, D = shape
    if out is None:
        out = (_torch.empty if rows is None else _torch.zeros)(shape, dtype=x.dtype, device=x.device)
    elif out.shape != shape or out.dtype is not x.dtype:
        raise ValueError("x and out: same shape and type")
    if D != plan.D:
        raise ValueError(f"x: heads of {D}, the plan is for {plan.D}")
    _enqueue(index, (_lib or lib()).bd_k_rope, (C.addressof(plan), *_rows_of(x, "x", heads, D, index), *_rows_of(out, "out", heads, D, index),
                                                _dtype_of(x, "x"), heads, n, M, _ints_of(pos, "pos", n, index), _ints_of(rows, "rows", n, index)))
    return out

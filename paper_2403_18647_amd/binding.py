"""ctypes binding of ``libsdsat.so`` (C-ABI in include/sdsat.h).

Argument marshalling only: every step of the decode path runs in the HIP
library.  PyTorch provides device memory (tensors) and the HIP stream.  The
functions carry the C names; ``Context`` bundles a context with the
workspace and weight tensors it must keep alive.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsdsat.so")

SDSAT_OK = 0
ERRORS = {-1: "EINVAL", -2: "ENOMEM", -3: "EDEVICE", -4: "ECAPACITY", -5: "EUNSUPPORTED", -6: "EDATA"}
DTYPE_FP32, DTYPE_BF16 = 0, 1
MODE_GREEDY, MODE_NUCLEUS = 0, 1
PROFILE_KINDS = {"off": 0, "gateup": 1, "qkv": 2, "attention": 3, "down": 4, "o": 5, "lm_head": 6, "block": 7,
                 "prefill": 8}


class sdsat_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("n_adaptive", ctypes.c_int32), ("rms_eps", ctypes.c_float), ("rope_base", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("max_batch", ctypes.c_int32), ("max_ctx", ctypes.c_int32),
                ("max_block", ctypes.c_int32)]


class sdsat_stats(ctypes.Structure):
    _fields_ = [("loops", ctypes.c_int64), ("blocks", ctypes.c_int64), ("prefill_blocks", ctypes.c_int64),
                ("tokens", ctypes.c_int64), ("accepted", ctypes.c_int64),
                ("accept_hist", ctypes.c_int64 * 65), ("prefill_ms", ctypes.c_double),
                ("decode_ms", ctypes.c_double)]


class sdsat_logit_rules(ctypes.Structure):
    _fields_ = [("d_history", ctypes.c_void_p), ("d_history_len", ctypes.c_void_p), ("d_prompt_len", ctypes.c_void_p),
                ("history_ld", ctypes.c_int32), ("d_tokens", ctypes.c_void_p), ("d_mask", ctypes.c_void_p),
                ("d_penalties", ctypes.c_void_p), ("d_bias", ctypes.c_void_p), ("bias_ld", ctypes.c_int64),
                ("d_allowed", ctypes.c_void_p), ("allowed_ld", ctypes.c_int32)]


class sdsat_paged_config(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_rows", ctypes.c_int32),
                ("max_batch", ctypes.c_int32), ("max_ctx", ctypes.c_int32)]


class sdsat_paged_batch(ctypes.Structure):
    _fields_ = [("d_start", ctypes.c_void_p), ("d_len", ctypes.c_void_p), ("d_pages", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("pages_ld", ctypes.c_int32), ("rows", ctypes.c_int32),
                ("max_q", ctypes.c_int32), ("max_len", ctypes.c_int32)]
    device = None   # index of its tensors', where paged_batch() made it


class sdsat_rope(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rot_dims", ctypes.c_int32), ("mscale", ctypes.c_float),
                ("turns", ctypes.c_double * 64)]


PAGE = 32
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}

_VP, _I32, _I64, _F32, _U64, _SZ = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                   ctypes.c_uint64, ctypes.c_size_t)
_F64 = ctypes.c_double
_SIGNATURES = {
    "sdsat_query_sizes": ([ctypes.POINTER(sdsat_config), ctypes.POINTER(_SZ)], _I32),
    "sdsat_init": ([ctypes.POINTER(sdsat_config), ctypes.POINTER(_VP), _I32, _VP, _SZ, _VP, ctypes.POINTER(_VP)], _I32),
    "sdsat_reset": ([_VP, _I32], _I32),
    "sdsat_set_cache_len": ([_VP, _I32, ctypes.POINTER(_I32)], _I32),
    "sdsat_cache_len_ptr": ([_VP], _VP),
    "sdsat_forward_block": ([_VP, _I32, _I32, _VP, _VP, _VP], _I32),
    "sdsat_verify_greedy": ([_VP, _I32, _I32, _VP, _VP, _VP, _VP], _I32),
    "sdsat_verify_nucleus": ([_VP, _I32, _I32, _VP, _VP, _F32, _F32, _I32, _U64, _VP, _VP, _VP], _I32),
    "sdsat_forward_block_shared": ([_VP, _I32, _I32, _I32, ctypes.POINTER(_I32), _VP, _VP, _VP], _I32),
    "sdsat_token_logprobs": ([_VP, _I32, _I32, _VP, _VP, _F32, _I32, _VP, _VP, _VP, _VP], _I32),
    "sdsat_adjust_logits": ([_VP, _I32, _I32, _VP, ctypes.POINTER(sdsat_logit_rules), _VP], _I32),
    "sdsat_rope_init": ([_I32, _I32, _F64, _I32, _F64, _F64, _F64, _F64, _F32, ctypes.POINTER(sdsat_rope)], _I32),
    "sdsat_paged_query_sizes": ([ctypes.POINTER(sdsat_paged_config), ctypes.POINTER(_SZ)], _I32),
    "sdsat_paged_init": ([ctypes.POINTER(sdsat_paged_config), _VP, _SZ, _VP, ctypes.POINTER(_VP)], _I32),
    "sdsat_paged_append": ([_VP, ctypes.POINTER(sdsat_paged_batch), _VP, _VP, _VP, _I32, _I64, ctypes.POINTER(sdsat_rope),
                            _VP, _VP, _VP, _F32, _VP, _I64], _I32),
    "sdsat_paged_attention": ([_VP, ctypes.POINTER(sdsat_paged_batch), _VP, _VP, _VP, _I64, _VP, _I32, _F32, _VP, _I32,
                               _I64], _I32),
    "sdsat_paged_status": ([_VP], _I32),
    "sdsat_paged_destroy": ([_VP], _I32),
    "sdsat_paged_last_error": ([_VP], ctypes.c_char_p),
    "sdsat_commit_kv": ([_VP, _I32, _I32, _VP, _VP], _I32),
    "sdsat_kv_reorder": ([_VP, _I32, _VP, _I32], _I32),
    "sdsat_cache_ptr": ([_VP, _I32, ctypes.POINTER(_VP), ctypes.POINTER(_VP)], _I32),
    "sdsat_generate": ([_VP, _I32, ctypes.POINTER(_I32), _I32, _I32, _I32, ctypes.POINTER(_I32), _I32, _F32, _F32,
                        _I32, _U64, ctypes.POINTER(_I32), ctypes.POINTER(sdsat_stats)], _I32),
    "sdsat_generate_tree": ([_VP, _I32, ctypes.POINTER(_I32), _I32, _I32, _I32, _I32, ctypes.POINTER(_I32), _I32,
                             _F32, _F32, _I32, _U64, ctypes.POINTER(_I32), ctypes.POINTER(sdsat_stats)], _I32),
    "sdsat_generate_forced": ([_VP, _I32, ctypes.POINTER(_I32), _I32, _I32, _I32, ctypes.POINTER(_I32), _I32, _F32,
                               _F32, _I32, _U64, ctypes.POINTER(_I32), _I32, ctypes.POINTER(_I32),
                               ctypes.POINTER(sdsat_stats)], _I32),
    "sdsat_kv_write": ([_VP, _I32, _I32, _I32, _VP, _VP, _VP], _I32),
    "sdsat_attention": ([_VP, _I32, _I32, _I32, _VP, _VP, _VP], _I32),
    "sdsat_attention_shared": ([_VP, _I32, _I32, _I32, _I32, ctypes.POINTER(_I32), _VP, _VP, _VP], _I32),
    "sdsat_linear_packed_bytes": ([_I32, _I32, _I32], _SZ),
    "sdsat_linear_pack": ([_I32, _I32, _I32, _VP, _VP, _VP], _I32),
    "sdsat_linear_scratch_bytes": ([_I32, _I32, _I32], _SZ),
    "sdsat_linear": ([_I32, _I32, _I32, _I32, _VP, _VP, _VP, _VP, _VP], _I32),
    "sdsat_linear_noalloc": ([_I32, _I32, _I32, _I32, _VP, _VP, _VP, _VP], _I32),
    "sdsat_profile_kernel": ([_VP, _I32, _I32], _I32),
    "sdsat_kernel_time": ([_VP, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_I64)], _I32),
    "sdsat_kernel_samples": ([_VP, ctypes.POINTER(ctypes.c_float), _I64, ctypes.POINTER(_I64)], _I32),
    "sdsat_stream_read": ([_VP, _SZ, _VP], _I32),
    "sdsat_destroy": ([_VP], _I32),
    "sdsat_last_error": ([_VP], ctypes.c_char_p),
}
EXPORTS = tuple(_SIGNATURES)

_lib = None


def lib():
    """Load libsdsat.so (raises if it has not been built: there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


class SdsatError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"sdsat error {ERRORS.get(code, code)}: {msg}")
        self.code = code


def _check(rc: int, ctx=None) -> None:
    if rc != SDSAT_OK:
        msg = lib().sdsat_last_error(ctx)
        raise SdsatError(rc, msg.decode() if msg else "")


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def make_config(shape, max_batch: int, max_ctx: int, max_block: int) -> sdsat_config:
    """Config from any object with the shape fields of ``synth.ModelShape``."""
    return sdsat_config(shape.n_layers, shape.d_model, shape.n_heads, shape.head_dim, shape.d_ffn, shape.vocab,
                        shape.n_adaptive, shape.rms_eps, shape.rope_base,
                        DTYPE_BF16 if shape.dtype == "bf16" else DTYPE_FP32, max_batch, max_ctx, max_block)


# ------------------------------------------------------------------ C names
def sdsat_query_sizes(cfg: sdsat_config) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().sdsat_query_sizes(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def sdsat_init(cfg, weights, workspace, stream=None):
    arr = (ctypes.c_void_p * len(weights))(*[_ptr(w) for w in weights])
    out = ctypes.c_void_p()
    _check(lib().sdsat_init(ctypes.byref(cfg), arr, len(weights), _ptr(workspace), workspace.numel(),
                            _stream(stream), ctypes.byref(out)))
    return out


def sdsat_reset(ctx, batch):
    _check(lib().sdsat_reset(ctx, batch), ctx)


def sdsat_set_cache_len(ctx, lengths):
    a = np.ascontiguousarray(lengths, np.int32)
    _check(lib().sdsat_set_cache_len(ctx, a.size, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))), ctx)


def sdsat_cache_len_ptr(ctx) -> int:
    return lib().sdsat_cache_len_ptr(ctx)


def sdsat_forward_block(ctx, batch, q, tokens, mask=None, logits=None):
    _check(lib().sdsat_forward_block(ctx, batch, q, _ptr(tokens), _ptr(mask), _ptr(logits)), ctx)


def sdsat_verify_greedy(ctx, batch, q, logits, drafts, tokens_out, n_accept):
    _check(lib().sdsat_verify_greedy(ctx, batch, q, _ptr(logits), _ptr(drafts), _ptr(tokens_out),
                                     _ptr(n_accept)), ctx)


def sdsat_verify_nucleus(ctx, batch, q, logits, drafts, temperature, top_p, top_k, seed, pos0, tokens_out,
                         n_accept):
    _check(lib().sdsat_verify_nucleus(ctx, batch, q, _ptr(logits), _ptr(drafts), temperature, top_p, top_k,
                                      seed, _ptr(pos0), _ptr(tokens_out), _ptr(n_accept)), ctx)


def _prefix_lens(batch, group, prefix_len):
    """Host lengths of the groups' prefixes as a C array (one per group)."""
    n = batch // group if group > 0 else 0
    if len(prefix_len) != n:
        raise ValueError("prefix_len must hold one length per group")
    return (ctypes.c_int32 * max(1, n))(*prefix_len)


def sdsat_forward_block_shared(ctx, batch, q, group, prefix_len, tokens, mask=None, logits=None):
    """prefix_len: host lengths, one per group of `group` sequences."""
    _check(lib().sdsat_forward_block_shared(ctx, batch, q, group, _prefix_lens(batch, group, prefix_len), _ptr(tokens),
                                            _ptr(mask), _ptr(logits)), ctx)


def sdsat_token_logprobs(ctx, batch, q, logits, tokens, temperature, n_top, logprob, entropy, top_ids=None,
                         top_logprobs=None):
    _check(lib().sdsat_token_logprobs(ctx, batch, q, _ptr(logits), _ptr(tokens), temperature, n_top, _ptr(logprob),
                                      _ptr(entropy), _ptr(top_ids), _ptr(top_logprobs)), ctx)


def logit_rules(history=None, history_len=None, prompt_len=None, tokens=None, mask=None, penalties=None, bias=None,
                allowed=None) -> sdsat_logit_rules:
    """Rules for sdsat_adjust_logits from device tensors (kept alive by the result): int32 history [batch, n], history_len
    and prompt_len [batch], tokens [batch, q]; int64 mask [batch * q]; float32 penalties [3, batch] (repetition, frequency,
    presence) and bias [V], [1, V] or [batch, V]; int32 allowed [batch * q, words], a bit for each id."""
    _dense(history, history_len, prompt_len, tokens, mask, penalties, bias, allowed)
    _elements("int32", history=history, history_len=history_len, prompt_len=prompt_len, tokens=tokens, allowed=allowed)
    _elements("int64", mask=mask)
    _elements("float32", penalties=penalties, bias=bias)
    shared = bias is None or bias.dim() == 1 or bias.shape[0] == 1
    r = sdsat_logit_rules(_ptr(history), _ptr(history_len), _ptr(prompt_len), 0 if history is None else history.shape[-1],
                          _ptr(tokens), _ptr(mask), _ptr(penalties), _ptr(bias), 0 if shared else bias.shape[-1],
                          _ptr(allowed), 0 if allowed is None else allowed.shape[-1])
    r.tensors = (history, history_len, prompt_len, tokens, mask, penalties, bias, allowed)
    return r


def sdsat_adjust_logits(ctx, batch, q, logits, rules, out):
    for t in (logits, out):
        if not isinstance(t, int) and (str(t.dtype) != "torch.float32" or not t.is_contiguous()):
            raise ValueError("logits and out must be float32 and contiguous")
    _check(lib().sdsat_adjust_logits(ctx, batch, q, _ptr(logits), ctypes.byref(rules), _ptr(out)), ctx)


def _dense(*tensors):
    for t in tensors:
        if t is not None and not isinstance(t, int) and not t.is_contiguous():
            raise ValueError("tensor must be contiguous")


def _elements(kind, **tensors):
    """Tensors (None, addresses: not looked at) hold elements of this type; for int32 and int64 the unsigned one does too."""
    import torch
    allowed = [getattr(torch, n) for n in (kind, "u" + kind) if hasattr(torch, n)]
    for name, t in tensors.items():
        if t is not None and not isinstance(t, int) and t.dtype not in allowed:
            raise ValueError(f"{name} must be {kind}, not {t.dtype}")


def _dtype_codes():
    import torch
    return {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16}


def _dtype_code(t):
    codes = _dtype_codes()
    if t.dtype not in codes:
        raise ValueError("tensor must be float32 or bfloat16")
    return codes[t.dtype]


def _row_stride(t, rows=0, columns=0):
    """Elements between rows of a 2-D tensor whose rows are contiguous, at least `rows` of at least `columns`."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("tensor must be 2-D with contiguous rows")
    n, width = shape
    if n < rows or width < columns:
        raise ValueError(f"tensor of {n} rows of {width} elements, fewer than the call's {rows} rows of {columns}")
    return stride[0] if n > 1 else max(stride[0], width)


class _PagedLimits:
    """What a handle's tensors have to be like, kept beside it: looked at in every call, for a microsecond of the host's
    time (the library sees addresses only)."""

    def __init__(self, cfg, workspace):
        import torch
        self.dtype = torch.bfloat16 if cfg.dtype == DTYPE_BF16 else torch.float32
        self.k_shape = torch.Size((cfg.n_pages, cfg.n_kv_heads, PAGE, cfg.head_dim))
        self.v_shape = torch.Size((cfg.n_pages, cfg.n_kv_heads, cfg.head_dim, PAGE))
        self.q_columns = cfg.n_heads * cfg.head_dim
        self.x_columns = (cfg.n_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
        self.head_dim, self.max_rows = cfg.head_dim, cfg.max_rows
        self.device = workspace.get_device()
        self.codes = _dtype_codes()
        self.pool_codes = {self.dtype: cfg.dtype}
        self.float32, self.int32, self.int64 = ((d,) for d in (torch.float32, torch.int32, torch.int64))
        if hasattr(torch, "uint32"):
            self.int32, self.int64 = (torch.int32, torch.uint32), (torch.int64, torch.uint64)

    def elsewhere(self, t, what):
        if t.is_cuda or not t.is_pinned():
            raise ValueError(f"{what} is on another device than the handle")

    def rows(self, batch):
        """A call's rows, as far as tensors must have them: the library refuses calls of more than it takes."""
        if batch.device != self.device and batch.device is not None:
            raise ValueError("the batch's tensors are on another device than the handle")
        return batch.rows if batch.rows <= self.max_rows else 0

    def pools(self, k, v):
        """Addresses of K and V."""
        try:
            if (k.shape == self.k_shape and v.shape == self.v_shape and k.dtype is self.dtype and v.dtype is self.dtype and
                    k.get_device() == self.device and v.get_device() == self.device and k.is_contiguous() and v.is_contiguous()):
                return k.data_ptr(), v.data_ptr()
        except AttributeError:   # addresses
            pass
        return self.pool(k, self.k_shape, "k"), self.pool(v, self.v_shape, "v")

    def pool(self, t, shape, what):
        if t is None or isinstance(t, int):
            return t
        if t.shape != shape and (t.dim() != 4 or t.shape[1:] != shape[1:] or t.shape[0] < shape[0]):
            raise ValueError(f"{what} must be {list(shape)}, not {list(t.shape)}")
        if t.dtype is not self.dtype or not t.is_contiguous():
            raise ValueError(f"{what} must be {self.dtype} and contiguous")
        if t.get_device() != self.device:
            self.elsewhere(t, what)
        return t.data_ptr()

    def rows_of(self, t, rows, columns, codes, what):
        """Address, type and row stride of a call's rows."""
        if t is None:
            raise ValueError(f"{what} is missing")
        code = codes.get(t.dtype)
        if code is None:
            raise ValueError(f"{what} must be {' or '.join(map(str, codes))}")
        shape = t.shape
        if len(shape) == 2 and t.is_contiguous() and shape[0] >= rows and shape[1] >= columns:
            ld = shape[1]
        else:
            ld = _row_stride(t, rows, columns)
        if t.get_device() != self.device:
            self.elsewhere(t, what)
        return t.data_ptr(), code, ld

    def vector(self, t, kinds, n, what):
        if isinstance(t, int):
            return t
        if t.dtype not in kinds or t.numel() < n or not t.is_contiguous():
            raise ValueError(f"{what} must be at least {n} elements of {kinds[0]}, contiguous")
        if t.get_device() != self.device:
            self.elsewhere(t, what)
        return t.data_ptr()


def paged_batch(start, length, pages, rows, max_q, max_len) -> sdsat_paged_batch:
    """The sequences of a call on a paged cache from int32 device tensors (kept alive by the result): start [batch + 1],
    length [batch], pages [batch, width]; rows of the call's arrays; host bounds of the new tokens of a sequence and of
    its slots with them."""
    _dense(start, length)
    _elements("int32", start=start, length=length, pages=pages)
    if start.numel() != length.numel() + 1 or pages.dim() != 2 or pages.shape[0] != length.numel():
        raise ValueError("start must be [batch + 1], length [batch] and pages [batch, width]")
    b = sdsat_paged_batch(_ptr(start), _ptr(length), _ptr(pages), length.numel(), _row_stride(pages), rows, max_q, max_len)
    if b.pages_ld > pages.shape[1] and max_len > PAGE * pages.shape[1]:
        raise ValueError(f"max_len of {max_len} slots, {pages.shape[1]} pages of 32 in a row of the view")
    b.tensors = (start, length, pages)
    b.device = start.get_device()
    if length.get_device() != b.device or pages.get_device() != b.device:
        raise ValueError("start, length and pages must be on one device")
    return b


def sdsat_rope_init(layout="half", rot_dims=128, base=10000.0, scaling="none", factor=1.0, ctx=0.0, low=1.0, high=4.0,
                    mscale=1.0) -> sdsat_rope:
    """Rotary positions (see include/sdsat.h): layout "half" or "interleaved", scaling "none", "linear", "ntk" or
    "parts"."""
    r = sdsat_rope()
    _check(lib().sdsat_rope_init(ROPE_LAYOUTS[layout], rot_dims, base, ROPE_SCALINGS[scaling], factor, ctx, low, high,
                                 mscale, ctypes.byref(r)))
    return r


def _check_paged(rc, paged):
    if rc != SDSAT_OK:
        msg = lib().sdsat_paged_last_error(paged)
        raise SdsatError(rc, msg.decode() if msg else "")


def sdsat_paged_query_sizes(cfg: sdsat_paged_config) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().sdsat_paged_query_sizes(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def sdsat_paged_init(cfg, workspace, stream=None):
    out = ctypes.c_void_p()
    _check(lib().sdsat_paged_init(ctypes.byref(cfg), _ptr(workspace), workspace.numel(), _stream(stream), ctypes.byref(out)))
    out.limits = _PagedLimits(cfg, workspace)
    return out


def sdsat_paged_append(paged, batch, k, v, x, rope=None, pos=None, q_gain=None, k_gain=None, eps=0.0, q_out=None):
    """x [rows, (heads + 2 kv_heads) * head_dim] float32 or bfloat16, q_out [rows, heads * head_dim] in the pool's type; rows
    may be strided.  k and v as Paged.pool() makes them, pos int32 [rows], gains float32 [head_dim]."""
    t = paged.limits
    rows = t.rows(batch)
    k_at, v_at = t.pools(k, v)
    x_at, x_code, x_ld = t.rows_of(x, rows, t.x_columns, t.codes, "x")
    q_at, _, q_ld = t.rows_of(q_out, rows, t.q_columns, t.pool_codes, "q_out")
    _check_paged(lib().sdsat_paged_append(paged, ctypes.byref(batch), k_at, v_at, x_at, x_code, x_ld,
                                          None if rope is None else ctypes.byref(rope),
                                          None if pos is None else t.vector(pos, t.int32, rows, "pos"),
                                          None if q_gain is None else t.vector(q_gain, t.float32, t.head_dim, "q_gain"),
                                          None if k_gain is None else t.vector(k_gain, t.float32, t.head_dim, "k_gain"),
                                          eps, q_at, q_ld), paged)


def sdsat_paged_attention(paged, batch, k, v, q, mask=None, window=0, scale=0.0, out=None):
    """q [rows, heads * head_dim] in the pool's type, out the same or float32; rows may be strided.  k and v as Paged.pool()
    makes them, mask int64 [rows]."""
    t = paged.limits
    rows = t.rows(batch)
    k_at, v_at = t.pools(k, v)
    q_at, _, q_ld = t.rows_of(q, rows, t.q_columns, t.pool_codes, "q")
    out_at, out_code, out_ld = t.rows_of(out, rows, t.q_columns, t.codes, "out")
    _check_paged(lib().sdsat_paged_attention(paged, ctypes.byref(batch), k_at, v_at, q_at, q_ld,
                                             None if mask is None else t.vector(mask, t.int64, rows, "mask"), window, scale,
                                             out_at, out_code, out_ld), paged)


def sdsat_paged_status(paged):
    _check_paged(lib().sdsat_paged_status(paged), paged)


def sdsat_paged_destroy(paged):
    _check(lib().sdsat_paged_destroy(paged))


def sdsat_kv_reorder(ctx, batch, src, first_slot=0):
    _check(lib().sdsat_kv_reorder(ctx, batch, _ptr(src), first_slot), ctx)


def sdsat_cache_ptr(ctx, layer):
    k, v = ctypes.c_void_p(), ctypes.c_void_p()
    _check(lib().sdsat_cache_ptr(ctx, layer, ctypes.byref(k), ctypes.byref(v)), ctx)
    return k.value, v.value


def sdsat_commit_kv(ctx, batch, q, n_commit, rows=None):
    _check(lib().sdsat_commit_kv(ctx, batch, q, _ptr(n_commit), _ptr(rows)), ctx)


def sdsat_generate(ctx, prompts, max_new, k, adaptive_ids, mode=MODE_GREEDY, temperature=0.0, top_p=1.0,
                   top_k=0, seed=0, ref=None, width=1):
    """prompts: host int32 [batch, P].  Returns (tokens int32 [batch, max_new], stats dict).  With ref
    (host int32 [batch, ref_len]) calls sdsat_generate_forced: draft step 2 takes its drafts from ref.
    With width > 1 calls sdsat_generate_tree (draft tree of that width)."""
    p = np.ascontiguousarray(prompts, np.int32)
    batch, P = p.shape
    ad = np.ascontiguousarray(adaptive_ids if k else np.zeros(1), np.int32)
    out = np.zeros((batch, max_new), np.int32)
    st = sdsat_stats()
    ip = ctypes.POINTER(ctypes.c_int32)
    if width > 1:
        if ref is not None:
            raise ValueError("ref and width > 1 cannot be combined")
        _check(lib().sdsat_generate_tree(ctx, batch, p.ctypes.data_as(ip), P, max_new, k, width,
                                         ad.ctypes.data_as(ip), mode, temperature, top_p, top_k, seed,
                                         out.ctypes.data_as(ip), ctypes.byref(st)), ctx)
    elif ref is None:
        _check(lib().sdsat_generate(ctx, batch, p.ctypes.data_as(ip), P, max_new, k, ad.ctypes.data_as(ip), mode,
                                    temperature, top_p, top_k, seed, out.ctypes.data_as(ip), ctypes.byref(st)), ctx)
    else:
        r = np.ascontiguousarray(ref, np.int32)
        if r.ndim != 2 or r.shape[0] != batch:
            raise ValueError("ref must be [batch, ref_len]")
        _check(lib().sdsat_generate_forced(ctx, batch, p.ctypes.data_as(ip), P, max_new, k, ad.ctypes.data_as(ip),
                                           mode, temperature, top_p, top_k, seed, r.ctypes.data_as(ip), r.shape[1],
                                           out.ctypes.data_as(ip), ctypes.byref(st)), ctx)
    stats = {"loops": st.loops, "blocks": st.blocks, "prefill_blocks": st.prefill_blocks, "tokens": st.tokens,
             "accepted": st.accepted, "accept_hist": list(st.accept_hist)[: k + 1],
             "prefill_ms": st.prefill_ms, "decode_ms": st.decode_ms}
    return out, stats


def sdsat_kv_write(ctx, layer, batch, n, k, v, pos):
    _check(lib().sdsat_kv_write(ctx, layer, batch, n, _ptr(k), _ptr(v), _ptr(pos)), ctx)


def sdsat_attention(ctx, layer, batch, q, qin, mask, out):
    _check(lib().sdsat_attention(ctx, layer, batch, q, _ptr(qin), _ptr(mask), _ptr(out)), ctx)


def sdsat_attention_shared(ctx, layer, batch, q, group, prefix_len, qin, mask, out):
    """prefix_len: host lengths, one per group of `group` sequences."""
    _check(lib().sdsat_attention_shared(ctx, layer, batch, q, group, _prefix_lens(batch, group, prefix_len), _ptr(qin),
                                        _ptr(mask), _ptr(out)), ctx)


def sdsat_linear_packed_bytes(dtype, N, K) -> int:
    return lib().sdsat_linear_packed_bytes(dtype, N, K)


def sdsat_linear_pack(dtype, N, K, w, packed, stream=None):
    _check(lib().sdsat_linear_pack(dtype, N, K, _ptr(w), _ptr(packed), _stream(stream)))


def sdsat_linear_scratch_bytes(M, N, K) -> int:
    return lib().sdsat_linear_scratch_bytes(M, N, K)


def sdsat_linear(dtype, M, N, K, x, packed, y, scratch, stream=None):
    _check(lib().sdsat_linear(dtype, M, N, K, _ptr(x), _ptr(packed), _ptr(y), _ptr(scratch), _stream(stream)))


def sdsat_linear_noalloc(dtype, M, N, K, x, packed, y, stream=None):
    _check(lib().sdsat_linear_noalloc(dtype, M, N, K, _ptr(x), _ptr(packed), _ptr(y), _stream(stream)))


def sdsat_profile_kernel(ctx, kind, period=1):
    _check(lib().sdsat_profile_kernel(ctx, PROFILE_KINDS.get(kind, kind), period), ctx)


def sdsat_kernel_time(ctx):
    ms = ctypes.c_double(0)
    n = ctypes.c_int64(0)
    _check(lib().sdsat_kernel_time(ctx, ctypes.byref(ms), ctypes.byref(n)), ctx)
    return ms.value, n.value


def sdsat_kernel_samples(ctx, cap=1 << 16):
    """Milliseconds of each timed launch since the last call (a list, launch order)."""
    buf = (ctypes.c_float * cap)()
    n = ctypes.c_int64(0)
    _check(lib().sdsat_kernel_samples(ctx, buf, cap, ctypes.byref(n)), ctx)
    return [buf[i] for i in range(min(cap, n.value))]


def sdsat_stream_read(src, nbytes=None, stream=None):
    """Stream nbytes (default: all) of the device tensor src with the library's read-only kernel."""
    nbytes = src.numel() * src.element_size() if nbytes is None else nbytes
    _check(lib().sdsat_stream_read(_ptr(src), nbytes, _stream(stream)))


def sdsat_destroy(ctx):
    _check(lib().sdsat_destroy(ctx))


# ------------------------------------------------------------------ convenience
class Context:
    """A library context plus the device tensors it needs kept alive."""

    def __init__(self, cfg: sdsat_config, weights, device="cuda"):
        import torch
        self.cfg = cfg
        self.weights = list(weights)
        self.workspace = torch.empty(sdsat_query_sizes(cfg), dtype=torch.uint8, device=device)
        self.stream = torch.cuda.current_stream(device)
        self.handle = sdsat_init(cfg, self.weights, self.workspace, self.stream)

    def close(self):
        if getattr(self, "handle", None):
            sdsat_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def cache_len(self) -> np.ndarray:
        """Current cache_len[max_batch] (synchronises the stream)."""
        self.stream.synchronize()
        out = np.zeros(self.cfg.max_batch, np.int32)
        _hip_memcpy_d2h(out, sdsat_cache_len_ptr(self.handle))
        return out

    def cache(self):
        """The cache in place, as device views of the workspace: K [layers, max_batch, heads, slots, head_dim],
        V [layers, max_batch, heads, slots / 32, 2, 4, 4, head_dim] (the key 16a + 4g + r of a page at [a, g, r]) and
        the committed lengths [max_batch] (to be read: sdsat_set_cache_len writes them)."""
        import torch
        c = self.cfg
        dt = torch.bfloat16 if c.dtype == DTYPE_BF16 else torch.float32
        pages = (c.max_ctx + 31) // 32
        dh, bh = c.head_dim, c.max_batch * c.n_heads

        def view(ptr, dtype, shape, strides):
            at = (ptr - self.workspace.data_ptr()) // dtype.itemsize
            whole = self.workspace[: self.workspace.numel() // 4 * 4].view(dtype)
            return whole.as_strided(shape, strides, whole.storage_offset() + at)

        k, v = sdsat_cache_ptr(self.handle, 0)
        page, row, layer = 32 * dh, 32 * dh * pages, 32 * dh * pages * bh
        lead, lead_strides = (c.n_layers, c.max_batch, c.n_heads), (layer, row * c.n_heads, row)
        return (view(k, dt, lead + (32 * pages, dh), lead_strides + (dh, 1)),
                view(v, dt, lead + (pages, 2, 4, 4, dh), lead_strides + (page, 4, 8, 1, 32)),
                view(sdsat_cache_len_ptr(self.handle), torch.int32, (c.max_batch,), (1,)))


class Paged:
    """A paged-cache handle with its workspace, on the current stream; pool(): tensors for one layer's K and V."""

    def __init__(self, cfg: sdsat_paged_config, device="cuda"):
        import torch
        self.cfg = cfg
        self.workspace = torch.empty(sdsat_paged_query_sizes(cfg), dtype=torch.uint8, device=device)
        self.stream = torch.cuda.current_stream(device)
        with torch.cuda.device(self.workspace.device):   # the handle's device is the one that is current here
            self.handle = sdsat_paged_init(cfg, self.workspace, self.stream)

    def pool(self):
        """K [pages, kv_heads, 32, head_dim] and V [pages, kv_heads, head_dim, 32], uninitialised."""
        import torch
        c = self.cfg
        dt = torch.bfloat16 if c.dtype == DTYPE_BF16 else torch.float32
        dev = self.workspace.device
        return (torch.empty((c.n_pages, c.n_kv_heads, PAGE, c.head_dim), dtype=dt, device=dev),
                torch.empty((c.n_pages, c.n_kv_heads, c.head_dim, PAGE), dtype=dt, device=dev))

    def close(self):
        if getattr(self, "handle", None):
            sdsat_paged_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_hip = None


def _hip_memcpy_d2h(dst: np.ndarray, src_ptr: int) -> None:
    """Blocking device-to-host copy through the HIP runtime that torch already loaded."""
    global _hip
    if _hip is None:
        _hip = ctypes.CDLL("libamdhip64.so")
        _hip.hipMemcpy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
        _hip.hipMemcpy.restype = ctypes.c_int
    rc = _hip.hipMemcpy(dst.ctypes.data, src_ptr, dst.nbytes, 2)   # hipMemcpyDeviceToHost
    if rc != 0:
        raise RuntimeError(f"hipMemcpy failed ({rc})")

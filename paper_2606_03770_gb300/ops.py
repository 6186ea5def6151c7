"""Binding of the block operators' C ABI (include/e2ops.h) for torch tensors.

What one served decoder block and its output layer are made of, with 4-bit
weights and a 4-bit cache:

* ``quant_matmul``: products with 4-bit weights and group scales, with the
  residual add or the gated (SwiGLU) form;
* ``cache_append`` / ``cache_read`` / ``cache_attend``: a paged 4-bit cache of
  keys and values, written with the position rotation on the way, read back,
  and attended to by decode batches and prompts;
* ``cache_attend_tree`` / ``verify_drafts`` / ``cache_keep``: a decode step with a tree
  of drafted tokens for each request: attention in which a node sees its own way
  only, which of the drafted tokens the target's probabilities accept, and the
  accepted way's keys and values moved to where they belong;
* ``token_logprobs``: log probabilities of given tokens, entropy and top
  alternatives.

Each function checks its tensors, allocates outputs that are not given, and
enqueues on the current stream of the tensors' device.  Formulas, layouts and what
happens to values out of range are in include/e2ops.h.  There is no CPU
fallback: without the library, or with tensors off the GPU, the calls raise.  Nor are
there gradients: a tensor that requires one is refused while gradients are recorded.
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import warnings

import torch

from . import build, e2ga
from .e2ga import E2_OK

E2_F16, E2_BF16, E2_F32 = 0, 1, 2
E2_CACHE_GROUP, E2_MAX_TOP, E2_MAX_COLS, E2_MAX_DRAFT = 64, 32, 1 << 20, 64
DTYPES = {torch.float16: E2_F16, torch.bfloat16: E2_BF16, torch.float32: E2_F32}
_P, _I, _L = C.c_void_p, C.c_int32, C.c_int64
_MOST = 2 ** 31 - 1                        # of a c_int32, which takes larger numbers without their high bits


class e2_quant_weight(C.Structure):
    _fields_ = [("rows", _I), ("cols", _I), ("group", _I), ("codes", _P), ("scales", _P), ("mins", _P)]


class e2_matmul_args(C.Structure):
    _fields_ = [("tokens", _I), ("dtype", _I), ("gated", _I), ("x", _P), ("x_stride", _L), ("residual", _P),
                ("residual_stride", _L), ("y", _P), ("y_stride", _L)]


class e2_cache(C.Structure):
    _fields_ = [("pages", _I), ("page_size", _I), ("kv_heads", _I), ("head_dim", _I), ("k_codes", _P),
                ("k_scales", _P), ("v_codes", _P), ("v_scales", _P)]


class e2_append_args(C.Structure):
    _fields_ = [("tokens", _I), ("dtype", _I), ("q_heads", _I), ("rot", _I), ("interleaved", _I),
                ("table_rows", _I), ("slots", _P), ("positions", _P), ("cos", _P), ("sin", _P), ("k", _P),
                ("k_stride", _L), ("v", _P), ("v_stride", _L), ("q", _P), ("q_stride", _L), ("q_out", _P),
                ("q_out_stride", _L)]


class e2_attend_args(C.Structure):
    _fields_ = [("tokens", _I), ("dtype", _I), ("q_heads", _I), ("batch", _I), ("table", _P), ("table_cols", _I),
                ("table_stride", _L),
                ("lens", _P), ("starts", _P), ("max_new", _I), ("max_len", _I), ("scale", C.c_float),
                ("window", _I), ("q", _P), ("q_stride", _L), ("out", _P), ("out_stride", _L)]


class e2_logprobs_args(C.Structure):
    _fields_ = [("rows", _I), ("vocab", _I), ("dtype", _I), ("top", _I), ("logits", _P), ("stride", _L),
                ("tokens", _P), ("logprob", _P), ("entropy", _P), ("values", _P), ("ids", _P)]


class e2_verify_args(C.Structure):
    _fields_ = [("tokens", _I), ("vocab", _I), ("dtype", _I), ("batch", _I), ("max_new", _I), ("logits", _P),
                ("logits_stride", _L), ("draft", _P), ("draft_stride", _L), ("ids", _P), ("parents", _P),
                ("starts", _P), ("uniforms", _P), ("temperature", _P), ("kept", _P), ("nodes", _P), ("answer", _P)]


class e2_keep_args(C.Structure):
    _fields_ = [("layers", _I), ("batch", _I), ("cols", _I), ("arrays", _P), ("table", _P), ("table_cols", _I),
                ("table_stride", _L), ("lens", _P), ("starts", _P), ("nodes", _P), ("nodes_stride", _L), ("kept", _P),
                ("lens_out", _P)]


# name -> (restype, argtypes); the exported surface of include/e2ops.h
SIGNATURES = {
    "e2_ops_error": (C.c_char_p, []),
    "e2_quant_matmul_workspace": (C.c_size_t, [_I] * 3),
    "e2_quant_matmul": (C.c_int, [_P, _P, _P, C.c_size_t, _P]),
    "e2_cache_append": (C.c_int, [_P, _P, _P]),
    "e2_cache_read": (C.c_int, [_P, _P, _I, _I, _P, _L, _P, _L, _P]),
    "e2_cache_attend_workspace": (C.c_size_t, [_P, _P]),
    "e2_cache_attend": (C.c_int, [_P, _P, _P, C.c_size_t, _P]),
    "e2_cache_attend_tree_workspace": (C.c_size_t, [_P, _P]),
    "e2_cache_attend_tree": (C.c_int, [_P, _P, _P, _P, C.c_size_t, _P]),
    "e2_verify_drafts": (C.c_int, [_P, _P]),
    "e2_cache_layers": (C.c_int, [_P, _I, _P]),
    "e2_cache_keep": (C.c_int, [_P, _P, _P]),
    "e2_token_logprobs": (C.c_int, [_P, _P]),
}
_lib = None


def load():
    """The library with the operators' signatures; raises if it is not built."""
    global _lib
    if _lib is None:
        lib = e2ga.load()
        for name, (res, args) in SIGNATURES.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args
        _lib = lib
    return _lib


_binding = None


class _NoBinding:
    """In the module's place where it is not built: every call goes the whole way here."""
    attend_tree = verify = keep = staticmethod(lambda *a: None)


def binding():
    """The module of the calls whose time is the host's: None from one of its functions says that the
    call is to go the whole way here.  Where there is none for this Python and torch, all do."""
    global _binding
    if _binding is None:
        load()
        if build.binding_built_for() is not None and build.binding_built_for() == build.binding_for():
            spec = importlib.util.spec_from_loader("e2binding", importlib.machinery.ExtensionFileLoader("e2binding", build.BINDING))
            _binding = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(_binding)
        else:
            warnings.warn("e2binding.so is not built for this Python and torch: calls take some 15 us longer")
            _binding = _NoBinding
    return _binding


def _need(cond, text):
    if not cond:
        raise ValueError(text)


def _tensor(x, name, dtypes, shape, device=None):
    """x is a tensor on the GPU with one of these types, this shape (None: any
    size) and contiguous rows; returns its shape."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda):
        raise ValueError(f"{name} must be a tensor on the GPU")
    if device is not None and x.device != device:
        raise ValueError(f"{name} must be on {device}")
    if x.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {x.dtype}")
    s = x.shape
    ok = len(s) == len(shape)
    if ok:
        for a, b in zip(s, shape):
            ok = ok and (b is None or a == b)
    if not ok:
        raise ValueError(f"{name} has shape {tuple(s)}, not {tuple('any' if b is None else b for b in shape)}")
    if s[-1] > 1 and x.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous in its last axis")
    if x.numel() > _MOST and max(s) > _MOST:
        raise ValueError(f"{name} has shape {tuple(s)}: sizes are below 2^31")
    return s


def _like(x, name, dtype, shape, device):
    """_tensor for one type and a whole shape: a few comparisons where all is
    well (these run on every call of an operator)."""
    if not (isinstance(x, torch.Tensor) and x.dtype is dtype and x.shape == shape and x.device == device
            and x.stride(-1) == 1):
        _tensor(x, name, (dtype,), shape, device)


def _no_gradient(handle, **tensors):
    """The operators have no gradients: what requires one is refused, not left without."""
    if handle is not None and handle.requires_grad:
        raise ValueError(f"{type(handle).__name__} was made of tensors that require gradients; there are none here "
                         "(torch.no_grad(), or detach them)")
    for name, x in tensors.items():
        if x is not None and x.requires_grad:
            raise ValueError(f"{name} requires a gradient; there are none here (torch.no_grad(), or detach it)")


_HALF = (torch.float16, torch.bfloat16)
_FLOAT = (torch.float16, torch.bfloat16, torch.float32)


def _stride(x):
    """Row stride (a single row's does not matter)."""
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def _heads(x, name, dtype, shape, device):
    """Token stride of x [tokens, heads, dim], of one type and this shape, whose
    heads lie side by side (a single token's does not matter)."""
    if not (isinstance(x, torch.Tensor) and x.dtype is dtype and x.shape == shape and x.device == device):
        _tensor(x, name, (dtype,), shape, device)
    _, heads, dim = shape
    token, head, element = x.stride()
    if element != 1 and dim > 1:
        _tensor(x, name, (dtype,), shape, device)
    if head != dim and heads > 1:
        raise ValueError(f"{name}: a token's heads must lie side by side")
    return token if shape[0] > 1 else heads * dim


def _stream(device):
    """The device's current stream, as a number."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _call(name, device, *args):
    """Calls a function of the library on the device's current stream, with
    the device as the current one."""
    f = getattr(_lib or load(), name)
    if torch._C._cuda_getDevice() == device.index:
        status = f(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            status = f(*args, _stream(device))
    if status != E2_OK:
        raise e2ga.E2Error(status, name, load().e2_ops_error().decode())


class _Handle:
    """What holds tensors and the struct that the library takes of them.  The struct has
    their addresses and sizes, so none of what it is made of is assigned later."""

    _made = frozenset()                    # names that are not assigned any more

    def _hold(self, *tensors):
        """Views of its own, and the memory whatever becomes of any view."""
        self.requires_grad = any(x.requires_grad for x in tensors if x is not None)
        self._memory = [x.untyped_storage() for x in tensors if x is not None]
        return [x.detach() if x is not None else None for x in tensors]

    def __setattr__(self, name, value):
        if name in self._made:
            raise AttributeError(f"{type(self).__name__}.{name} cannot be changed: make another {type(self).__name__}")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in self._made:
            raise AttributeError(f"{type(self).__name__}.{name} cannot be deleted")
        object.__delattr__(self, name)


def _workspace(name, device, *args):
    """A workspace of the size that a function of the library says for `device`, None for 0."""
    f = getattr(_lib or load(), name)
    if torch._C._cuda_getDevice() == device.index:
        need = f(*args)
    else:
        with torch.cuda.device(device):
            need = f(*args)
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None


# ---- products with 4-bit weights --------------------------------------------------
class QuantWeight(_Handle):
    """4-bit weights [rows][cols]: ``codes`` uint8 [rows, cols / 2] (column 2j
    in the low four bits), ``scales`` float16 [rows, cols / group] and, for
    scale * code + min instead of scale * (code - 8), ``mins`` like scales.
    Holds views of the tensors, no copies: what is written into them counts, other
    tensors need another QuantWeight."""

    def __init__(self, codes, scales, mins=None):
        _tensor(codes, "codes", (torch.uint8,), (None, None))
        rows, cols = codes.shape[0], 2 * codes.shape[1]
        _tensor(scales, "scales", (torch.float16,), (rows, None), codes.device)
        groups = scales.shape[1]
        _need(groups > 0 and cols % groups == 0 and cols // groups in (32, 64, 128),
              "scales must have one column per 32, 64 or 128 columns of weights")
        for x, n in ((codes, "codes"), (scales, "scales")) + (((mins, "mins"),) if mins is not None else ()):
            _need(x.is_contiguous(), f"{n} must be contiguous")
        if mins is not None:
            _tensor(mins, "mins", (torch.float16,), (rows, groups), codes.device)
        self.rows, self.cols, self.group, self.device = rows, cols, cols // groups, codes.device
        self.codes, self.scales, self.mins = self._hold(codes, scales, mins)
        self.struct = e2_quant_weight(rows, cols, self.group, codes.data_ptr(), scales.data_ptr(),
                                      mins.data_ptr() if mins is not None else None)
        self.ref = C.byref(self.struct)
        self._made = frozenset(vars(self)) | {"_made"}

    def dequantize(self):
        """The weights in float32 (plain torch; for checks and inspection)."""
        c = torch.stack([self.codes & 15, self.codes >> 4], -1).flatten(1).float()
        s = self.scales.float().repeat_interleave(self.group, 1)
        if self.mins is None:
            return (c - 8) * s
        return c * s + self.mins.float().repeat_interleave(self.group, 1)


def quantize_weight(w, group=64, symmetric=True):
    """Round a float weight [rows, cols] to 4 bits with group scales (plain
    torch; done once, when a model is loaded).  Scales and minima end at fp16's
    largest, so weights beyond 7 (symmetric), 15 times that do too."""
    _need(w.dim() == 2 and group in (32, 64, 128) and w.shape[1] % group == 0,
          "w must be [rows, cols], cols a multiple of the group (32, 64 or 128)")
    x = w.float().unflatten(1, (-1, group))
    if symmetric:
        scales = (x.abs().amax(-1) / 7).clamp(max=65504).half()
        s = scales.float()[..., None]
        q = torch.where(s > 0, torch.round(x / s) + 8, 8.0)
        mins = None
    else:
        lo = x.amin(-1).clamp(-65504, 65504)
        mins, scales = lo.half(), ((x.amax(-1) - lo) / 15).clamp(max=65504).half()
        s = scales.float()[..., None]
        q = torch.where(s > 0, torch.round((x - mins.float()[..., None]) / s), 0.0)
    q = q.clamp(0, 15).to(torch.uint8).flatten(1)
    return QuantWeight((q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), scales.contiguous(),
                       mins.contiguous() if mins is not None else None)


def quant_matmul(x, w, residual=None, gated=False, out=None, workspace=None):
    """x [tokens, cols] times the weights' rows (+ residual): [tokens, rows],
    or, ``gated``, silu(x W_gate) * (x W_up) [tokens, rows / 2]."""
    dev = w.device
    tokens = _tensor(x, "x", _HALF, (None, w.cols), dev)[0] if not (
        isinstance(x, torch.Tensor) and x.dtype in _HALF and x.dim() == 2 and x.shape[1] == w.cols
        and x.device == dev and x.stride(1) == 1) else x.shape[0]
    outs = w.rows // 2 if gated else w.rows
    dtype, shape = x.dtype, (tokens, outs)
    if residual is not None:
        _like(residual, "residual", dtype, shape, dev)
    if out is None:
        out, out_stride = torch.empty(shape, dtype=dtype, device=dev), outs
    else:
        _like(out, "out", dtype, shape, dev)
        out_stride = _stride(out)
    if torch.is_grad_enabled() and (w.requires_grad or x.requires_grad or out.requires_grad
                                    or residual is not None and residual.requires_grad):
        _no_gradient(w, x=x, residual=residual, out=out)
    a = e2_matmul_args(tokens, DTYPES[dtype], bool(gated), x.data_ptr(), _stride(x),
                       residual.data_ptr() if residual is not None else None,
                       _stride(residual) if residual is not None else 0, out.data_ptr(), out_stride)
    if workspace is None:
        workspace = _workspace("e2_quant_matmul_workspace", dev, w.rows, w.cols, tokens)
    else:
        _need(workspace.is_contiguous(), "workspace must be contiguous")
    _call("e2_quant_matmul", dev, w.ref, C.byref(a), workspace.data_ptr() if workspace is not None else None,
          workspace.nbytes if workspace is not None else 0)
    return out


# ---- the cache ------------------------------------------------------------------------
class Cache(_Handle):
    """A paged 4-bit cache over four tensors: codes uint8
    [pages, kv_heads, page_size, head_dim / 2] and scales float16
    [pages, kv_heads, page_size, head_dim / 64, 2] of keys and of values.  Holds
    views of them: what is written into them counts, others need another Cache."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        _tensor(k_codes, "k_codes", (torch.uint8,), (None,) * 4)
        pages, heads, page, half = k_codes.shape
        _need(half in (32, 64), "head_dim must be 64 or 128")
        _need(page in (16, 32, 64, 128, 256), "page_size must be 16, 32, 64, 128 or 256")
        _tensor(v_codes, "v_codes", (torch.uint8,), k_codes.shape, k_codes.device)
        for x, n in ((k_scales, "k_scales"), (v_scales, "v_scales")):
            _tensor(x, n, (torch.float16,), (pages, heads, page, 2 * half // E2_CACHE_GROUP, 2), k_codes.device)
        for x in (k_codes, k_scales, v_codes, v_scales):
            _need(x.is_contiguous(), "cache tensors must be contiguous")
        self.pages, self.kv_heads, self.page_size, self.head_dim = pages, heads, page, 2 * half
        self.device = k_codes.device
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = self._hold(k_codes, k_scales, v_codes, v_scales)
        self.struct = e2_cache(pages, page, heads, 2 * half, k_codes.data_ptr(), k_scales.data_ptr(),
                               v_codes.data_ptr(), v_scales.data_ptr())
        self.ref = C.byref(self.struct)
        self.fast = (C.addressof(self.struct), self.device.index, self.requires_grad)
        self._made = frozenset(vars(self)) | {"_made"}

    @classmethod
    def empty(cls, pages, page_size, kv_heads, head_dim, device="cuda"):
        """A cache of zeros (every token reads as zeros)."""
        shape = (pages, kv_heads, page_size)
        codes = [torch.zeros(*shape, head_dim // 2, dtype=torch.uint8, device=device) for _ in range(2)]
        scales = [torch.zeros(*shape, head_dim // E2_CACHE_GROUP, 2, dtype=torch.float16, device=device)
                  for _ in range(2)]
        return cls(codes[0], scales[0], codes[1], scales[1])


def cache_append(cache, k, v, slots, positions, cos, sin, q=None, q_out=None, interleaved=False):
    """Append keys (turned by their positions) and values [tokens, kv_heads,
    head_dim] at ``slots`` (int64; page * page_size + token in page; -1: none).
    Returns the turned queries (``q_out``, allocated unless given), or None."""
    dev, D, H = cache.device, cache.head_dim, cache.kv_heads
    if not (isinstance(k, torch.Tensor) and k.dtype in _HALF and k.dim() == 3):
        _tensor(k, "k", _HALF, (None, H, D), dev)
    dtype, tokens = k.dtype, k.shape[0]
    ks, vs = (_heads(x, n, dtype, (tokens, H, D), dev) for x, n in ((k, "k"), (v, "v")))
    _like(slots, "slots", torch.int64, (tokens,), dev)
    _like(positions, "positions", torch.int32, (tokens,), dev)
    table_rows, half = _tensor(cos, "cos", (torch.float32,), (None, None), dev)
    _like(sin, "sin", torch.float32, (table_rows, half), dev)
    _need(cos.is_contiguous() and sin.is_contiguous(), "cos and sin must be contiguous")
    heads = qs = qos = 0
    if q is not None:
        if not (isinstance(q, torch.Tensor) and q.dim() == 3):
            _tensor(q, "q", (dtype,), (tokens, None, D), dev)
        heads = q.shape[1]
        qs = _heads(q, "q", dtype, (tokens, heads, D), dev)
        if q_out is None:
            q_out = torch.empty((tokens, heads, D), dtype=dtype, device=dev)
            qos = heads * D
        else:
            qos = _heads(q_out, "q_out", dtype, (tokens, heads, D), dev)
    else:
        _need(q_out is None, "q_out without q")
    if torch.is_grad_enabled() and (cache.requires_grad or k.requires_grad or v.requires_grad or cos.requires_grad
                                    or sin.requires_grad or heads and (q.requires_grad or q_out.requires_grad)):
        _no_gradient(cache, k=k, v=v, q=q, q_out=q_out, cos=cos, sin=sin)
    a = e2_append_args(tokens, DTYPES[dtype], heads, 2 * half, bool(interleaved), table_rows, slots.data_ptr(),
                       positions.data_ptr(), cos.data_ptr(), sin.data_ptr(), k.data_ptr(), ks, v.data_ptr(), vs,
                       q.data_ptr() if heads else None, qs, q_out.data_ptr() if heads else None, qos)
    _call("e2_cache_append", dev, cache.ref, C.byref(a))
    return q_out


def cache_read(cache, slots, dtype=torch.bfloat16):
    """The keys and values at ``slots``, as the values their codes stand for."""
    dev = cache.device
    tokens = _tensor(slots, "slots", (torch.int64,), (None,), dev)[0]
    _need(dtype in DTYPES, "dtype must be float16, bfloat16 or float32")
    shape = (tokens, cache.kv_heads, cache.head_dim)
    k = torch.empty(shape, dtype=dtype, device=dev)
    v = torch.empty(shape, dtype=dtype, device=dev)
    if torch.is_grad_enabled() and cache.requires_grad:
        _no_gradient(cache)
    row = shape[1] * shape[2]
    _call("e2_cache_read", dev, cache.ref, slots.data_ptr(), tokens, DTYPES[dtype], k.data_ptr(), row, v.data_ptr(),
          row)
    return k, v


def cache_attend(cache, q, table, lens, starts, max_new=None, max_len=None, scale=None, window=0, out=None,
                 workspace=None):
    """Attention of the queries q [tokens, q_heads, head_dim] of a batch of
    requests over the cache (their own keys already appended): ``table`` int32
    [batch, pages], ``lens`` int32 [batch] cached tokens, ``starts`` int32
    [batch + 1] first query of each request.  ``max_new`` and ``max_len``, the
    largest counts of queries and of cached tokens, are read from the device
    (a synchronisation) unless given.  scale: 1/sqrt(head_dim) unless given."""
    return _attend("e2_cache_attend", (), cache, q, table, lens, starts, max_new, max_len, scale, window, out, workspace)


def _attend(name, more, cache, q, table, lens, starts, max_new, max_len, scale, window, out, workspace):
    """A function of the library that takes e2_attend_args, and `more` tensors after them."""
    dev = cache.device
    if not (isinstance(q, torch.Tensor) and q.dtype in _HALF and q.dim() == 3):
        _tensor(q, "q", _HALF, (None, None, cache.head_dim), dev)
    tokens, heads, _ = shape = (q.shape[0], q.shape[1], cache.head_dim)
    q_stride = _heads(q, "q", q.dtype, shape, dev)
    batch, cols = _tensor(table, "table", (torch.int32,), (None, None), dev)
    _like(lens, "lens", torch.int32, (batch,), dev)
    _like(starts, "starts", torch.int32, (batch + 1,), dev)
    if max_new is None:
        max_new = max(0, int((starts[1:].long() - starts[:-1].long()).max())) if batch else 0
    if max_len is None:
        max_len = max(0, int(lens.max())) if batch else 0
    if out is None:
        # (tokens outside every request are not written)
        out = (torch.empty if batch else torch.zeros)(shape, dtype=q.dtype, device=dev)
        out_stride = heads * cache.head_dim
    else:
        out_stride = _heads(out, "out", q.dtype, shape, dev)
    if torch.is_grad_enabled() and (cache.requires_grad or q.requires_grad or out.requires_grad):
        _no_gradient(cache, q=q, out=out)
    if max_new > _MOST or max_len > _MOST or not -1 <= window <= _MOST:
        max_new, max_len, window = min(max_new, _MOST), min(max_len, _MOST), max(-1, min(window, _MOST))
    a = e2_attend_args(tokens, DTYPES[q.dtype], heads, batch, table.data_ptr(), cols, _stride(table),
                       lens.data_ptr(), starts.data_ptr(), max_new, max_len,
                       cache.head_dim ** -0.5 if scale is None else scale, window, q.data_ptr(), q_stride,
                       out.data_ptr(), out_stride)
    if workspace is None:
        workspace = _workspace(name + "_workspace", dev, cache.ref, C.byref(a))
    else:
        _need(workspace.is_contiguous(), "workspace must be contiguous")
    _call(name, dev, cache.ref, C.byref(a), *(x.data_ptr() for x in more),
          workspace.data_ptr() if workspace is not None else None, workspace.nbytes if workspace is not None else 0)
    return out


# ---- a decode step with drafted tokens ----------------------------------------------------
def cache_attend_tree(cache, q, parents, table, lens, starts, max_new=None, max_len=None, scale=None, window=0,
                      out=None, workspace=None):
    """``cache_attend`` where each request's new tokens are the nodes of a tree:
    ``parents`` int32 [tokens], a node's parent by its number in its request, -1 for
    none.  A node sees the tokens before the tree, itself and the nodes on its way up.
    Up to E2_MAX_DRAFT nodes a request (more are refused where ``max_new`` says so).  Which rows'
    keys and values are rounded to fp16 on the way goes by the sizes (include/e2ops.h)."""
    done = (_binding or binding()).attend_tree(cache.fast, q, parents, table, lens, starts, max_new, max_len, scale, window, out,
                                               workspace)
    if done is not None:
        return done
    _like(parents, "parents", torch.int32, (q.shape[0] if isinstance(q, torch.Tensor) and q.dim() else 0,), cache.device)
    return _attend("e2_cache_attend_tree", (parents,), cache, q, table, lens, starts, max_new, max_len, scale, window, out,
                   workspace)


def verify_drafts(logits, ids, parents, starts, uniforms, draft=None, temperature=None, max_new=None):
    """(kept, nodes, answer): which tokens of each request's tree the target's
    probabilities accept.  ``logits`` [tokens, vocab] of what follows each node, ``draft``
    those that the tokens were drawn from, siblings each by itself and at the same temperature
    (None: they were chosen in any other way, such as without putting back), ``ids`` int32
    and ``uniforms`` float32 [tokens], ``parents`` and ``starts`` as for
    ``cache_attend_tree``, ``temperature`` float32 [batch] (None: 1; 0: the largest
    logit).  ``kept`` int32 [batch] counts the accepted nodes, node 0 among them; ``nodes`` and
    ``answer`` int32 [batch, max_new] have them and the token after each, -1 behind.  ``max_new``,
    at most E2_MAX_DRAFT, is read from the device (a synchronisation) unless given; nodes of a
    request beyond it are not looked at."""
    done = (_binding or binding()).verify(logits, ids, parents, starts, uniforms, draft, temperature, max_new)
    if done is not None:
        return done
    tokens, vocab = _tensor(logits, "logits", _FLOAT, (None, None))
    dev = logits.device
    if draft is not None:
        _like(draft, "draft", logits.dtype, (tokens, vocab), dev)
    for x, name, dtype in ((ids, "ids", torch.int32), (parents, "parents", torch.int32), (uniforms, "uniforms", torch.float32)):
        _like(x, name, dtype, (tokens,), dev)
    if not (isinstance(starts, torch.Tensor) and starts.dim() == 1 and starts.shape[0] > 0):
        _tensor(starts, "starts", (torch.int32,), (None,), dev)
        raise ValueError("starts has one entry more than there are requests")
    batch = starts.shape[0] - 1
    _like(starts, "starts", torch.int32, (batch + 1,), dev)
    if temperature is not None:
        _like(temperature, "temperature", torch.float32, (batch,), dev)
    if torch.is_grad_enabled() and (logits.requires_grad or uniforms.requires_grad or draft is not None and draft.requires_grad
                                    or temperature is not None and temperature.requires_grad):
        _no_gradient(None, logits=logits, draft=draft, uniforms=uniforms, temperature=temperature)
    if max_new is None:
        max_new = max(0, int((starts[1:].long() - starts[:-1].long()).max())) if batch else 0
    _need(0 <= max_new <= E2_MAX_DRAFT, f"max_new must be in 0..{E2_MAX_DRAFT}")
    i32 = dict(dtype=torch.int32, device=dev)
    kept = torch.empty(batch, **i32)
    nodes, answer = torch.empty((batch, max_new), **i32), torch.empty((batch, max_new), **i32)
    a = e2_verify_args(tokens, vocab, DTYPES[logits.dtype], batch, max_new, logits.data_ptr(), _stride(logits),
                       draft.data_ptr() if draft is not None else None, _stride(draft) if draft is not None else 0,
                       ids.data_ptr(), parents.data_ptr(), starts.data_ptr(), uniforms.data_ptr(),
                       temperature.data_ptr() if temperature is not None else None, kept.data_ptr(), nodes.data_ptr(),
                       answer.data_ptr())
    _call("e2_verify_drafts", dev, C.byref(a))
    return kept, nodes, answer


class CacheLayers(_Handle):
    """The caches of a model's layers, all of one shape and of different memory, for calls that
    treat them at once.  Their addresses go to the device here, some 0.2 ms for 80 layers with a
    synchronisation, so it is made once and kept."""

    def __init__(self, caches):
        self.caches = tuple(caches)
        _need(self.caches and all(isinstance(c, Cache) for c in self.caches), "caches must be Cache objects, one at least")
        first = self.caches[0]
        self.device, self.requires_grad = first.device, any(c.requires_grad for c in self.caches)
        for c in self.caches:
            _need(c.device == first.device, f"every cache must be on {first.device}")
        n = len(self.caches)
        structs, arrays = (e2_cache * n)(*(c.struct for c in self.caches)), (C.c_uint64 * (4 * n))()
        with torch.cuda.device(self.device):
            status = load().e2_cache_layers(structs, n, arrays)
        if status != E2_OK:
            raise ValueError(load().e2_ops_error().decode())
        self.arrays = torch.tensor(list(arrays), dtype=torch.int64, device=self.device)
        torch.cuda.current_stream(self.device).synchronize()         # (whatever stream they are used on)
        self.fast = first.fast[:2] + (self.requires_grad, n, self.arrays.data_ptr())
        self._made = frozenset(vars(self)) | {"_made"}

    def __len__(self):
        return len(self.caches)


def cache_keep(layers, table, lens, starts, nodes, kept, lens_out=None):
    """Move the accepted nodes' keys and values, in every layer (``CacheLayers``), to where the
    tokens after the tree's first belong: node ``nodes[r, k]`` of request r to token
    k of its tree, for k < ``kept[r]``.  Returns the cached tokens of each request after
    that, int32 [batch] (``lens_out``, allocated unless given; of memory of its own)."""
    _need(isinstance(layers, CacheLayers), "layers must be a CacheLayers")
    done = (_binding or binding()).keep(layers.fast, table, lens, starts, nodes, kept, lens_out)
    if done is not None:
        return done
    dev = layers.device
    batch, cols = _tensor(table, "table", (torch.int32,), (None, None), dev)
    for x, name, n in ((lens, "lens", batch), (starts, "starts", batch + 1), (kept, "kept", batch)):
        _like(x, name, torch.int32, (n,), dev)
    if not (isinstance(nodes, torch.Tensor) and nodes.dim() == 2 and nodes.shape[0] == batch):
        _tensor(nodes, "nodes", (torch.int32,), (batch, None), dev)
    most = nodes.shape[1]
    if most:
        _like(nodes, "nodes", torch.int32, (batch, most), dev)
    else:
        _need(nodes.dtype is torch.int32 and nodes.device == dev, f"nodes must be torch.int32 on {dev}")
    _need(most <= E2_MAX_DRAFT, f"nodes has more than {E2_MAX_DRAFT} columns")
    if lens_out is None:
        lens_out = torch.empty(batch, dtype=torch.int32, device=dev)
    else:
        _like(lens_out, "lens_out", torch.int32, (batch,), dev)
    if torch.is_grad_enabled() and layers.requires_grad:
        _no_gradient(layers)
    first = layers.caches[0]
    a = e2_keep_args(len(layers), batch, most, layers.arrays.data_ptr(), table.data_ptr(), cols, _stride(table),
                     lens.data_ptr(), starts.data_ptr(), nodes.data_ptr(), _stride(nodes), kept.data_ptr(),
                     lens_out.data_ptr())
    _call("e2_cache_keep", dev, first.ref, C.byref(a))
    return lens_out


# ---- the output layer --------------------------------------------------------------------
def token_logprobs(logits, tokens=None, top=0, entropy=True):
    """(logprob, entropy, values, ids) of logits [rows, vocab]: the log
    probability of tokens[row] (int32; None without tokens), the entropy (None
    unless asked for), and the ``top`` largest log probabilities with their indices
    [rows, top], equal ones by their index.  All float32 / int32."""
    rows, vocab = _tensor(logits, "logits", _FLOAT, (None, None))
    dev = logits.device
    _need(0 <= top <= E2_MAX_TOP, f"top must be in 0..{E2_MAX_TOP}")
    if tokens is not None:
        _like(tokens, "tokens", torch.int32, (rows,), dev)
    if torch.is_grad_enabled() and logits.requires_grad:
        _no_gradient(None, logits=logits)
    f32 = dict(dtype=torch.float32, device=dev)
    logprob = torch.empty(rows, **f32) if tokens is not None else None
    ent = torch.empty(rows, **f32) if entropy else None
    values, ids = torch.empty((rows, top), **f32), torch.empty((rows, top), dtype=torch.int32, device=dev)
    a = e2_logprobs_args(rows, vocab, DTYPES[logits.dtype], top, logits.data_ptr(), _stride(logits),
                         tokens.data_ptr() if tokens is not None else None,
                         logprob.data_ptr() if tokens is not None else None, ent.data_ptr() if entropy else None,
                         values.data_ptr(), ids.data_ptr())
    _call("e2_token_logprobs", dev, C.byref(a))
    return logprob, ent, values, ids

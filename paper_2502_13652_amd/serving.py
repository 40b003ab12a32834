"""What goes around a draft phase: a paged K/V cache with its attention, adjusted logits, and a layer's norm, rotation and attention over
prompts (the second part of include/c2t.h).  Argument marshalling and checks only; like the binding it needs a GPU and has no fallback."""
import ctypes
import dataclasses
import fractions
import struct
import threading
from typing import Optional

import torch

from . import binding
from .binding import BF16, E4M3, F16, F32, _check, load_library

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
ATTENTION_COUNTERS = 8192                                   # C2T_ATTENTION_COUNTERS


class _Adjustments(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("n_tokens", ctypes.c_void_p), ("n_prompt", ctypes.c_void_p),
                ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("bias_tokens", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("n_bias", ctypes.c_void_p), ("bias_stride", ctypes.c_int32),
                ("allowed", ctypes.c_void_p), ("allowed_row_stride", ctypes.c_int64), ("allowed_batch_stride", ctypes.c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "layers", "pages", "page_size", "kv_heads", "head_dim", "max_pages", "dtype")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "page_table", "length", "refcount", "status")]


class _Attention(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_batch_stride", ctypes.c_int64), ("q_token_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("out_batch_stride", ctypes.c_int64), ("out_token_stride", ctypes.c_int64),
                ("lse", ctypes.c_void_p), ("n_new", ctypes.c_void_p), ("tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("layer", ctypes.c_int32), ("nodes", ctypes.c_int32), ("mask", ctypes.c_void_p), ("scale", ctypes.c_float)]


class _Norm(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "weight", "residual", "residual_out", "out", "scales")] + \
               [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "residual_out_stride", "out_stride", "scales_stride")] + \
               [(n, ctypes.c_int32) for n in ("rows", "width", "dtype", "weight_dtype", "residual_dtype", "out_dtype", "scale_block")] + [("eps", ctypes.c_float)]


class _Append(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v", "q_out", "k_out")] + \
               [(n, ctypes.c_int64) for n in ("q_batch_stride", "q_token_stride", "kv_batch_stride", "kv_token_stride",
                                              "q_out_batch_stride", "q_out_token_stride", "k_out_batch_stride", "k_out_token_stride")] + \
               [(n, ctypes.c_void_p) for n in ("n_new", "starts", "position", "turns")] + [("magnitude", ctypes.c_float)] + \
               [(n, ctypes.c_int32) for n in ("tokens", "q_heads", "layer", "nodes", "pairs", "neighbours")]


class _Prompt(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v", "out", "lse")] + [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride", "out_stride")] + \
               [("starts", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("rows", "sequences", "q_heads", "kv_heads", "head_dim", "dtype")] + [("scale", ctypes.c_float)]


def _packer(fields):
    """A call's structure as bytes: a third of the time that ctypes takes to fill one.  The layout is the structure's."""
    code = {ctypes.c_void_p: "P", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f"}
    p = struct.Struct("@" + "".join(code[t] for _, t in fields._fields_) + "0P")
    assert p.size == ctypes.sizeof(fields)
    return p.pack


_pack_adjustments, _pack_attention = _packer(_Adjustments), _packer(_Attention)
_pack_norm, _pack_append, _pack_prompt = _packer(_Norm), _packer(_Append), _packer(_Prompt)


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _whole(t, device, dtype, shape, name):
    """The address of a contiguous device tensor of that type and shape; -1 in the shape: any size."""
    try:
        if t.dtype is dtype and t.get_device() == device.index and t.is_contiguous():
            have = t.shape
            if have == shape or (-1 in shape and len(have) == len(shape) and all(s in (-1, n) for s, n in zip(shape, have))):
                return t.data_ptr()
    except AttributeError:                                   # no tensor
        pass
    raise ValueError("%s: a contiguous %s tensor %s on %s" % (name, dtype, list(shape), device))


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_current_stream = binding._current_raw_stream or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(device, stream, fn, *args):
    """fn(*args, stream handle) with the tensors' device current."""
    index = device.index
    if stream is None and _current_device() == index:
        return fn(*args, _current_stream(index))
    _need(stream is None or stream.device == device, "stream: of another device than the tensors")
    with torch.cuda.device(device):
        return fn(*args, binding._stream_ptr(stream))


def _empty_like_on(stream, make):
    """An output made by the call: by the allocator of the stream that writes it."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


@dataclasses.dataclass
class LogitAdjustments:
    """What is done to logits (c2t_adjustments): device tensors, None leaves a term out.

    tokens int32 [B][L], n_tokens and n_prompt int32 [B]; repetition, frequency, presence float32 [B];
    bias_tokens int32 and bias float32 [B][M], n_bias int32 [B];
    allowed int32 [B][rows][ceil(V / 32)], rows the logits' or 1: bit v % 32 of word v // 32 set where token v may follow."""
    tokens: Optional[torch.Tensor] = None
    n_tokens: Optional[torch.Tensor] = None
    n_prompt: Optional[torch.Tensor] = None
    repetition: Optional[torch.Tensor] = None
    frequency: Optional[torch.Tensor] = None
    presence: Optional[torch.Tensor] = None
    bias_tokens: Optional[torch.Tensor] = None
    bias: Optional[torch.Tensor] = None
    n_bias: Optional[torch.Tensor] = None
    allowed: Optional[torch.Tensor] = None

    def _packed(self, B, rows, V, device):
        i32, f32 = torch.int32, torch.float32
        tokens, n_tokens, n_prompt, bias, bias_tokens, n_bias, allowed = \
            self.tokens, self.n_tokens, self.n_prompt, self.bias, self.bias_tokens, self.n_bias, self.allowed
        _need((tokens is None) == (n_tokens is None), "tokens and n_tokens come together")
        _need((bias is None) == (bias_tokens is None), "bias and bias_tokens come together")
        one = (B,)

        def each(t, dtype, name):
            return 0 if t is None else _whole(t, device, dtype, one, name)
        p_tokens = p_n = p_bias = p_bias_tokens = L = M = p_allowed = row = batch = 0
        if tokens is not None:
            p_tokens, p_n = _whole(tokens, device, i32, (B, -1), "tokens"), each(n_tokens, i32, "n_tokens")
            L = tokens.shape[1]
        p_prompt = each(n_prompt, i32, "n_prompt")
        if L == 0:                                         # a list without a place holds nothing; its address would be none
            p_tokens = p_n = p_prompt = 0
        if bias is not None:
            p_bias = _whole(bias, device, f32, (B, -1), "bias")
            M = bias.shape[1]
            p_bias_tokens = _whole(bias_tokens, device, i32, (B, M), "bias_tokens")
            if M == 0:
                p_bias = p_bias_tokens = 0
        if allowed is not None:
            words = (V + 31) // 32
            p_allowed = _whole(allowed, device, i32, (B, -1, words), "allowed")
            masks = allowed.shape[1]
            _need(masks in (1, rows), "allowed: a mask a row, or one a sequence")
            row, batch = (words if masks == rows else 0), masks * words
        return _pack_adjustments(p_tokens, L, p_n, p_prompt, each(self.repetition, f32, "repetition"), each(self.frequency, f32, "frequency"),
                                 each(self.presence, f32, "presence"), p_bias_tokens, p_bias, each(n_bias, i32, "n_bias"), M, p_allowed, row, batch)


def _rows(x, B, rows, V, name):
    """The distance of a logits tensor's rows, in elements."""
    shape, strides = x.shape, x.stride()
    _need(x.is_cuda and len(shape) == 3 and shape[0] == B and shape[1] == rows and shape[2] >= V and strides[2] == 1 and
          (B == 1 or strides[0] == rows * strides[1] or rows == 1 and strides[0] >= V), "%s: [%d][%d][at least %d], rows evenly spaced" % (name, B, rows, V))
    # (a sequence's one row is as far from the next one's as the sequences are; one row alone may be anywhere)
    return strides[1] if rows > 1 else strides[0] if B > 1 else max(strides[1], V + (-V) % (16 // x.element_size()))


def adjust_tree_logits(logits, tree, adjustments, vocab=None, out=None, stream=None):
    """The target model's logits [B][1 + N][stride >= vocab] (float32 or bfloat16) of a tree's root and nodes with `adjustments` (a
    LogitAdjustments) made, into `out` (a new tensor; may be `logits`).  tree: a finalize_tree output (tokens, parent, n_nodes), or None for one
    row a sequence.  Rows behind a sequence's nodes, and what is behind `vocab` (default: all), are left as they are; in a new tensor they are not filled in."""
    L = load_library()
    B, rows, width = logits.shape
    V = width if vocab is None else int(vocab)
    dev, dtype = logits.device, logits.dtype
    _need(dtype is torch.float32 or dtype is torch.bfloat16, "logits: float32 or bfloat16")
    stride = _rows(logits, B, rows, V, "logits")
    tokens = parent = 0
    if tree is None:
        _need(rows == 1, "logits: one row a sequence without a tree")
        none = _empty_like_on(stream, lambda: torch.zeros(B, dtype=torch.int32, device=dev))
        n_nodes = none.data_ptr()
    else:
        nodes = (B, rows - 1)
        tokens, parent = _whole(tree["tokens"], dev, torch.int32, nodes, "tree tokens"), _whole(tree["parent"], dev, torch.int32, nodes, "tree parent")
        n_nodes = _whole(tree["n_nodes"], dev, torch.int32, (B,), "tree n_nodes")
    if out is None:
        out = _empty_like_on(stream, lambda: torch.empty((B, rows, stride), dtype=dtype, device=dev)[:, :, :width])
    _need(out.dtype is dtype and out.device == dev, "out: of the logits' type and device")
    _check(_launch(dev, stream, L.c2t_adjust_tree_logits, adjustments._packed(B, rows, V, dev), B, V, rows - 1, _DTYPES[dtype], tokens, parent, n_nodes,
                   logits.data_ptr(), stride, out.data_ptr(), _rows(out, B, rows, V, "out")), "c2t_adjust_tree_logits")
    return out


def adjust_frontier_logits(ctx, logits, adjustments, out=None, stream=None):
    """C2TContext.adjust_logits."""
    B, F, V = ctx.B, ctx.F, ctx.V
    dev = logits.device
    _need(logits.dtype is ctx._logits_dtype and dev == ctx._ws.device, "logits: of the context's type and device")
    out = logits if out is None else out
    _need(out.dtype is logits.dtype and out.device == dev, "out: of the logits' type and device")
    _check(_launch(dev, stream, ctx.L.c2t_adjust_logits, ctx.ctx, adjustments._packed(B, F, V, dev), logits.data_ptr(), _rows(logits, B, F, V, "logits"),
                   out.data_ptr(), _rows(out, B, F, V, "out")), "c2t_adjust_logits")
    return out


def _even_rows(t, shape, index, name):
    """The distance, in elements, of the rows of a tensor of that shape on that device: its last dimension whole, the others as if they were one."""
    if t.shape != shape or t.get_device() != index:
        raise ValueError("%s: %s on the same device" % (name, list(shape)))
    width = shape[-1]
    if t.is_contiguous():
        return width
    strides = t.stride()
    at = [(n, s) for n, s in zip(shape[:-1], strides[:-1]) if n > 1]       # (a stride over one element is of no use and may be any number)
    if (strides[-1] != 1 and width != 1) or any(a[1] != b[0] * b[1] for a, b in zip(at, at[1:])):
        raise ValueError("%s: rows evenly spaced, elements next to each other" % name)
    return at[-1][1] if at else width


def rms_norm(x, weight, eps=1e-5, residual=None, residual_out=None, out=None, scale_block=None, scales=None, stream=None):
    """Root-mean-square norm of x + residual: h = x + residual, h / sqrt(mean(h^2) + eps) * weight over the last dimension, of h in fp32.

    x [...][width] float32, bfloat16 or float16, its rows evenly spaced, as those of the other arrays (some heads of a fused projection, [:, :heads], are not, and are refused);
    weight [width] of that type or float32; residual, of x's shape, of that type or float32: h goes to
    residual_out (default: residual itself), rounded to its type.  out: of x's shape and type (default: a new tensor; may be x).  With scale_block (32, 64, 128
    or the width), out is float8_e4m3fn and stands for out * scale, with a scale for each scale_block elements of a row (the last may be fewer): scales float32
    [...][ceil(width / scale_block)] (default: new), max |y| / 448 of the block; returns (out, scales), without it out."""
    dtype, shape, index = x.dtype, x.shape, x.get_device()
    code = out_code = residual_code = _DTYPES.get(dtype)
    if code is None or index < 0 or not shape or shape[-1] < 1:
        raise ValueError("x: [...][width] of float32, bfloat16 or float16 on the GPU")
    dev, width, out_dtype = x.device, shape[-1], dtype
    x_stride = _even_rows(x, shape, index, "x")
    p_residual = p_residual_out = residual_stride = residual_out_stride = p_scales = scales_stride = 0
    if residual is not None:
        kind = residual.dtype
        if kind is not dtype:
            _need(kind is torch.float32, "residual: of x's type or float32")
            residual_code = F32
        residual_stride = residual_out_stride = _even_rows(residual, shape, index, "residual")
        p_residual = p_residual_out = residual.data_ptr()
        if residual_out is not None and residual_out is not residual:
            _need(residual_out.dtype is kind, "residual_out: of the residual's type")
            residual_out_stride = _even_rows(residual_out, shape, index, "residual_out")
            p_residual_out = residual_out.data_ptr()
    else:
        _need(residual_out is None, "residual_out: with a residual")
    weight_code = code if weight.dtype is dtype else F32
    p_weight = _whole(weight, dev, dtype if weight_code == code else torch.float32, (width,), "weight")
    if scale_block is not None:
        _need(scale_block == width or scale_block in (32, 64, 128), "scale_block: 32, 64, 128 or the width")
        out_code, out_dtype = E4M3, torch.float8_e4m3fn
        wanted = shape[:-1] + (-(-width // scale_block),)
        if scales is None:
            scales = _empty_like_on(stream, lambda: torch.empty(wanted, dtype=torch.float32, device=dev))
        _need(scales.dtype is torch.float32, "scales: float32")
        scales_stride, p_scales = _even_rows(scales, wanted, index, "scales"), scales.data_ptr()
    else:
        _need(scales is None, "scales: with a scale_block")
    if out is None:
        out = _empty_like_on(stream, lambda: torch.empty(shape, dtype=out_dtype, device=dev))
    elif out.dtype is not out_dtype:
        raise ValueError("out: %s" % out_dtype)
    rows = x.numel() // width
    _need(rows < 1 << 31, "x: fewer than 2^31 rows")
    if rows > 0:
        a = _pack_norm(x.data_ptr(), p_weight, p_residual, p_residual_out, out.data_ptr(), p_scales, x_stride, residual_stride, residual_out_stride,
                       _even_rows(out, shape, index, "out"), scales_stride, rows, width, code, weight_code, residual_code, out_code, scale_block or 0, eps)
        _check(_launch(dev, stream, load_library().c2t_rms_norm, a), "c2t_rms_norm")
    return out if scale_block is None else (out, scales)


def _packed_rows(x, rows, heads, head_dim, dtype, index, name):
    """The distance, in elements, of the rows of [rows][heads][head_dim]."""
    strides = x.stride()
    if not (x.shape == (rows, heads, head_dim) and x.dtype is dtype and strides[2] == 1 and (heads == 1 or strides[1] == head_dim) and x.get_device() == index):
        raise ValueError("%s: %s [%d][%d][%d] on the same device, heads next to each other" % (name, dtype, rows, heads, head_dim))
    return strides[0] if rows > 1 else heads * head_dim


def prompt_attention(q, k, v, starts, scale=None, out=None, lse=None, stream=None):
    """Causal attention over whole prompts packed one behind the other: rows starts[b] .. starts[b + 1] - 1 are sequence b's, and each sees those of its
    sequence up to itself.

    q [rows][q_heads][head_dim], k and v [rows][kv_heads][head_dim], bfloat16 or float16, e.g. slices of one projection's output; starts int32 [sequences + 1].
    scale: of the scores, default head_dim ** -0.5.  out: as q (default: a new tensor), lse: float32 [rows][q_heads] for the log of the softmax's sums; rows in no
    sequence are left as they are (in a new tensor they are not filled in)."""
    shape, dtype, index = q.shape, q.dtype, q.get_device()
    if len(shape) != 3 or k.dim() != 3 or index < 0 or not (dtype is torch.bfloat16 or dtype is torch.float16):
        raise ValueError("q: [rows][q_heads][head_dim] of bfloat16 or float16 on the GPU")
    dev = q.device
    rows, heads, D = shape
    kv_heads = k.shape[1]
    sq, sk = _packed_rows(q, rows, heads, D, dtype, index, "q"), _packed_rows(k, rows, kv_heads, D, dtype, index, "k")
    sv = _packed_rows(v, rows, kv_heads, D, dtype, index, "v")
    if out is None:
        out = _empty_like_on(stream, lambda: torch.empty((rows, heads, D), dtype=dtype, device=dev))
    so = _packed_rows(out, rows, heads, D, dtype, index, "out")
    p_lse = 0 if lse is None else _whole(lse, dev, torch.float32, (rows, heads), "lse")
    p_starts = _whole(starts, dev, torch.int32, (-1,), "starts")
    sequences = starts.shape[0] - 1
    _need(sequences >= 0, "starts: int32 [sequences + 1]")
    if rows > 0 and sequences > 0:
        a = _pack_prompt(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), p_lse, sq, sk, sv, so, p_starts, rows, sequences, heads, kv_heads, D, _DTYPES[dtype],
                         D ** -0.5 if scale is None else scale)
        _check(_launch(dev, stream, load_library().c2t_prompt_attention, a), "c2t_prompt_attention")
    return out


_PI = fractions.Fraction("3.14159265358979323846264338327950288419716939937510582097")


class Rotation:
    """How queries and keys are turned by their positions (PagedCache.append): the first dim elements of each head's row in pairs, elements j and dim / 2 + j, or, with
    `neighbours`, 2j and 2j + 1; pair j by position * base ** (-2j / dim), or by position * frequencies[j] (radians, dim / 2 of them), and times magnitude.
    dim: a multiple of 16.  Held on the device as 64-bit fractions of a turn, so that far positions are as exact as near ones."""

    def __init__(self, dim, base=10000.0, neighbours=False, frequencies=None, magnitude=1.0, device="cuda:0"):
        _need(dim > 0 and dim % 16 == 0, "dim: a multiple of 16")
        f = [float(base) ** (-2.0 * j / dim) for j in range(dim // 2)] if frequencies is None else [float(x) for x in frequencies]
        _need(len(f) == dim // 2 and all(abs(x) < float("inf") for x in f), "frequencies: dim / 2 finite numbers")
        turns = [round(fractions.Fraction(x) / (2 * _PI) * (1 << 64)) % (1 << 64) for x in f]
        self.dim, self.neighbours, self.magnitude = dim, bool(neighbours), float(magnitude)
        self.turns = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns], dtype=torch.int64, device=device)


class PagedCache:
    """A paged K/V cache (c2t_cache): tensors k, v [layers][pages][kv_heads][page_size][head_dim], page_table int32 [B][max_pages] (-1: no
    page), length int32 [B], refcount int32 [pages], status uint32 [B] (POOL_EMPTY, ROW_FULL, INVALID, SHARED; set by calls, cleared by the
    user).  All calls are enqueued on torch's current stream (or `stream`) and answer on the device alone.  Calls on one cache belong on one
    stream; attention alone may run on several (each stream has a workspace of its own).  Several threads may make them: each is enqueued whole."""
    POOL_EMPTY, ROW_FULL, INVALID, SHARED = 1, 2, 4, 8

    def __init__(self, batch, layers, pages, page_size, kv_heads, head_dim, max_pages, dtype=torch.bfloat16, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("the C2T HIP path needs a GPU; there is no CPU fallback")
        shape = (layers, pages, kv_heads, page_size, head_dim)
        i32 = dict(dtype=torch.int32, device=device)
        self._take(torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device),
                   torch.full((batch, max_pages), -1, **i32), torch.zeros(batch, **i32), torch.zeros(pages, **i32))

    @classmethod
    def of_tensors(cls, k, v, page_table, length, refcount):
        """A cache over tensors that are there already; they are used, not copied."""
        self = cls.__new__(cls)
        self._take(k, v, page_table, length, refcount)
        return self

    def _take(self, k, v, page_table, length, refcount):
        self.L = load_library()
        _need(k.is_cuda and k.dim() == 5 and k.dtype in _DTYPES, "k: [layers][pages][kv_heads][page_size][head_dim] on the GPU")
        self.device, self.dtype = k.device, k.dtype
        layers, pages, kv_heads, page_size, head_dim = k.shape
        dev = k.device
        p_k, p_v = _whole(k, dev, k.dtype, k.shape, "k"), _whole(v, dev, k.dtype, k.shape, "v")
        p_table = _whole(page_table, dev, torch.int32, (-1, -1), "page_table")
        batch, max_pages = page_table.shape
        p_length, p_refs = _whole(length, dev, torch.int32, (batch,), "length"), _whole(refcount, dev, torch.int32, (pages,), "refcount")
        self.k, self.v, self.page_table, self.length, self.refcount = k, v, page_table, length, refcount
        self.status = torch.zeros(batch, dtype=torch.int32, device=k.device).view(torch.uint32)
        self.batch, self.layers, self.pages, self.page_size, self.kv_heads, self.head_dim, self.max_pages = batch, layers, pages, page_size, kv_heads, head_dim, max_pages
        self._c = _Cache(batch, layers, pages, page_size, kv_heads, head_dim, max_pages, _DTYPES[k.dtype], p_k, p_v, p_table, p_length, p_refs,
                         self.status.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._each, self._scale = (batch,), head_dim ** -0.5
        self._launching = threading.Lock()                   # a call's launches share a workspace: no other call's come between them on the stream
        need = ctypes.c_size_t()
        _check(self.L.c2t_cache_workspace_bytes(self._ref, ctypes.byref(need)), "c2t_cache_workspace_bytes")
        self._ws = self._workspace(need.value)
        self._attention_ws = {}                            # (stream, in a capture) -> capture, {bytes: workspace}
        self._attention_bytes = {}

    def _workspace(self, nbytes):
        w = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        pad = (-w.data_ptr()) % 256
        return w[pad:pad + nbytes]

    def _run(self, what, stream, *args):
        with self._launching:
            rc = _launch(self.device, stream, getattr(self.L, what), self._ref, *args)
        if rc != 0:
            raise binding.C2TError(rc, what)

    def _per_sequence(self, t, name):
        return _whole(t, self.device, torch.int32, self._each, name)

    def reserve(self, n_new, stream=None):
        """Pages for n_new (int32 [B]) tokens behind each sequence's length, its own to write."""
        self._run("c2t_cache_reserve", stream, self._per_sequence(n_new, "n_new"), self._ws.data_ptr(), self._ws.numel())

    def _tokens(self, x, heads, name):
        """Batch and token stride of [B][tokens][heads][head_dim]."""
        shape, strides = x.shape, x.stride()
        D = self.head_dim
        if not (x.dtype is self.dtype and len(shape) == 4 and shape[0] == self.batch and shape[1] > 0 and shape[2] == heads and shape[3] == D and
                strides[3] == 1 and (heads == 1 or strides[2] == D) and x.device == self.device):
            raise ValueError("%s: %s [%d][tokens][%d][%d] on %s, heads next to each other" % (name, self.dtype, self.batch, heads, D, self.device))
        # (a stride over one element is of no use and may be any number)
        return (strides[0] if self.batch > 1 else heads * D), (strides[1] if shape[1] > 1 else heads * D)

    def write(self, layer, k, v, n_new=None, stream=None):
        """K and V [B][tokens][kv_heads][head_dim] of new tokens, n_new (int32 [B], default all) of them, to positions length + t of `layer`."""
        sk = self._tokens(k, self.kv_heads, "k")
        _need(self._tokens(v, self.kv_heads, "v") == sk and k.shape == v.shape, "k and v: of one shape and strides")
        self._run("c2t_cache_write", stream, int(layer), k.data_ptr(), v.data_ptr(), sk[0], sk[1], k.shape[1],
                  None if n_new is None else self._per_sequence(n_new, "n_new"))

    def append(self, layer, q, k, v, rotation, n_new=None, position=None, starts=None, q_out=None, k_out=None, stream=None):
        """Queries and keys of new tokens turned by their positions (a Rotation), keys and values to places length + t of `layer`, as write does; returns q_out.

        q [B][T][q_heads][head_dim], k and v [B][T][kv_heads][head_dim], n_new (int32 [B], default all) of them.  A token's position is its place, but for a
        tree's nodes, the last N of the T slots: position int32 [B][N] as finalize_tree writes it, from the slot ahead of them (the root) on.
        Or packed, with starts (int32 [B + 1]): [rows][heads][head_dim], rows starts[b] .. starts[b + 1] - 1 are sequence b's.
        q_out: as q (default: a new tensor; may be q); k_out: as k, for the turned keys (may be k); rows of no token are left as they are.  What the cache has no room
        or page for is left out of it alone, and its status says so."""
        packed = starts is not None
        shape, D, H, index = q.shape, self.head_dim, self.kv_heads, self.device.index
        if len(shape) != (3 if packed else 4):
            raise ValueError("q: [rows][q_heads][head_dim] with starts, [B][T][q_heads][head_dim] without")
        T, heads = shape[-3], shape[-2]
        if packed:
            _need(n_new is None and position is None, "n_new and position: without starts")
            rows = lambda x, n, name: (0, _packed_rows(x, T, n, D, self.dtype, index, name))
        else:
            rows = self._tokens
        sq, sk = rows(q, heads, "q"), rows(k, H, "k")
        if not (v.shape == k.shape and (v.stride() == k.stride() or rows(v, H, "v") == sk) and v.dtype is k.dtype and v.get_device() == index and k.shape[-3] == T):
            raise ValueError("k and v: of one shape, type and strides, as many tokens as q")
        if q_out is None:
            q_out = _empty_like_on(stream, lambda: torch.empty(q.shape, dtype=self.dtype, device=self.device))
        so = sq if q_out is q else rows(q_out, heads, "q_out")
        _need(q_out.shape == shape and (k_out is None or k_out.shape == k.shape), "q_out and k_out: of q's and k's shape")
        ko = (0, 0) if k_out is None else rows(k_out, H, "k_out")
        nodes = p_position = 0
        if position is not None:
            nodes = position.shape[-1]
            p_position = _whole(position, self.device, torch.int32, (self.batch, nodes), "position") if nodes else 0
        turns = rotation.turns
        p_turns = _whole(turns, self.device, torch.int64, (rotation.dim // 2,), "rotation")
        if T == 0:
            return q_out
        a = _pack_append(q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), 0 if k_out is None else k_out.data_ptr(), sq[0], sq[1], sk[0], sk[1],
                         so[0], so[1], ko[0], ko[1], 0 if n_new is None else self._per_sequence(n_new, "n_new"),
                         _whole(starts, self.device, torch.int32, (self.batch + 1,), "starts") if packed else 0, p_position, p_turns, rotation.magnitude,
                         T, heads, layer, nodes, rotation.dim // 2, rotation.neighbours)
        self._run("c2t_cache_append", stream, a)
        return q_out

    def commit(self, path, n_path, stream=None):
        """The tokens in slots path[b][i] (int32 [B][P], rising) behind the length move to slots i < n_path[b]; the length grows by n_path."""
        p = _whole(path, self.device, torch.int32, (self.batch, -1), "path")
        self._run("c2t_cache_commit", stream, p, path.shape[1], self._per_sequence(n_path, "n_path"))

    def truncate(self, new_length=None, keep=0, stream=None):
        """Lengths cut to new_length (int32 [B], default as they are); pages behind length + keep tokens let go."""
        self._run("c2t_cache_truncate", stream, None if new_length is None else self._per_sequence(new_length, "new_length"), int(keep))

    def fork(self, src, dst, stream=None):
        """Sequences dst[i] become copies of src[i] (int32 [n] each); the pages are shared until they are written."""
        s = _whole(src, self.device, torch.int32, (-1,), "src")
        n = src.shape[0]
        self._run("c2t_cache_fork", stream, s, _whole(dst, self.device, torch.int32, (n,), "dst"), n)

    def attention(self, layer, q, n_new=None, mask=None, scale=None, out=None, lse=None, workspace=None, stream=None):
        """Attention of the last n_new (int32 [B], default all) tokens, which have been written behind the length, over the cache.

        q [B][T][q_heads][head_dim]; mask uint8 [B][N][N] as finalize_tree writes it: the last N of the T slots are the tree's nodes, those
        before them (the root) a causal chain; no mask: all of them are.  Keys on no page are left out and set INVALID in the sequence's status, new
        tokens that its row of page_table has no room for are left out and set ROW_FULL.  scale: of the scores, default head_dim ** -0.5.  lse: float32
        [B][T][q_heads] for the log of the softmax's sums.  out: [B][T][q_heads][head_dim], rows behind n_new left as
        they are (default: a new tensor, in which they are not filled in: they hold whatever the memory held).  workspace: uint8, zeros, of attention_workspace_bytes and 256-byte aligned, for calls that run at once otherwise than by stream.
        Without one the cache keeps one a stream, and in a graph's capture one that is the graph's: from its pool, counters cleared at each replay."""
        _need(q.dim() == 4, "q: [B][T][q_heads][head_dim]")
        _, T, heads, _ = q.shape
        sq = self._tokens(q, heads, "q")
        if out is None:
            out = _empty_like_on(stream, lambda: torch.empty((self.batch, T, heads, self.head_dim), dtype=self.dtype, device=self.device))
        so = self._tokens(out, heads, "out")
        _need(out.shape[1] == T, "out: of q's shape")
        nodes = p_mask = p_lse = 0
        if mask is not None:
            nodes = mask.shape[-1]
            p_mask = _whole(mask, self.device, torch.uint8, (self.batch, nodes, nodes), "mask") if nodes else 0
        _need(workspace is None or (workspace.dtype is torch.uint8 and workspace.device == self.device and workspace.is_contiguous()),
              "workspace: contiguous uint8 on %s" % self.device)
        if lse is not None:
            p_lse = _whole(lse, self.device, torch.float32, (self.batch, T, heads), "lse")
        a = _pack_attention(q.data_ptr(), sq[0], sq[1], out.data_ptr(), so[0], so[1], p_lse, 0 if n_new is None else self._per_sequence(n_new, "n_new"),
                            T, heads, layer, nodes, p_mask, self._scale if scale is None else scale)
        need = self._attention_bytes.get((T, heads, nodes))
        if need is None:
            need = self._attention_bytes[(T, heads, nodes)] = self.attention_workspace_bytes(T, heads, nodes)
        with self._launching:
            rc = _launch(self.device, stream, self._attend, a, workspace, need)
        if rc != 0:
            raise binding.C2TError(rc, "c2t_cache_attention")
        return out

    def _attend(self, a, workspace, need, s):
        w = self._attention_workspace(s, need) if workspace is None else workspace
        return self.L.c2t_cache_attention(self._ref, a, w.data_ptr(), w.numel(), s)

    def _attention_workspace(self, s, need):
        """One a stream, and one a captured graph: graphs may be replayed at once, and an eager call beside them."""
        capture = 0
        if s:
            number = ctypes.c_uint64()
            _check(self.L.c2t_stream_capture_id(s, ctypes.byref(number)), "c2t_stream_capture_id")
            capture = number.value
        entry = self._attention_ws.get((s, capture != 0))
        if entry is None or entry[0] != capture:             # of a capture that has ended: its graph's pool holds the memory
            entry = self._attention_ws[(s, capture != 0)] = (capture, {})
        w = entry[1].get(need)
        if w is None:
            here = torch.cuda.current_stream(self.device)
            with torch.cuda.stream(here if here.cuda_stream == s else torch.cuda.ExternalStream(s, self.device)):
                w = entry[1][need] = self._workspace(need)
                w[:ATTENTION_COUNTERS].zero_()               # on the stream that is going to use them
        return w

    def attention_workspace_bytes(self, tokens, q_heads, nodes=0):
        a = _Attention(tokens=tokens, q_heads=q_heads, nodes=nodes)
        n = ctypes.c_size_t()
        _check(self.L.c2t_attention_workspace_bytes(self._ref, ctypes.byref(a), ctypes.byref(n)), "c2t_attention_workspace_bytes")
        return n.value

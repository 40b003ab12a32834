"""What goes around a draft phase: a paged K/V cache with its attention, and adjusted logits (the second part of
include/c2t.h).  Argument marshalling and checks only; like the binding it needs a GPU and has no fallback."""
import ctypes
import dataclasses
from typing import Optional

import torch

from . import binding
from .binding import BF16, F16, F32, _check, load_library

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


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


def _ptr(t):
    return None if t is None else t.data_ptr()


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _whole(t, device, dtype, shape, name):
    """A contiguous device tensor of that type; -1 in `shape`: any size."""
    _need(torch.is_tensor(t) and t.device == device and t.dtype == dtype and t.is_contiguous() and t.dim() == len(shape) and
          all(s in (-1, n) for s, n in zip(shape, t.shape)),
          "%s: a contiguous %s tensor %s on %s" % (name, dtype, list(shape), device))
    return t


def _launch(device, stream, call):
    """call(stream handle) with the tensors' device current."""
    if stream is not None:
        _need(stream.device == device, "stream: of another device than the tensors")
    if torch._C._cuda_getDevice() == device.index:
        return call(binding._stream_ptr(stream))
    with torch.cuda.device(device):
        return call(binding._stream_ptr(stream))


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

    def _struct(self, B, rows, V, device):
        i32, f32 = torch.int32, torch.float32
        _need((self.tokens is None) == (self.n_tokens is None), "tokens and n_tokens come together")
        _need((self.bias is None) == (self.bias_tokens is None), "bias and bias_tokens come together")
        if self.tokens is not None:
            _whole(self.tokens, device, i32, (B, -1), "tokens")
        for name, dtype in (("n_tokens", i32), ("n_prompt", i32), ("n_bias", i32), ("repetition", f32), ("frequency", f32), ("presence", f32)):
            if getattr(self, name) is not None:
                _whole(getattr(self, name), device, dtype, (B,), name)
        if self.bias is not None:
            _whole(self.bias, device, f32, (B, -1), "bias")
            _whole(self.bias_tokens, device, i32, tuple(self.bias.shape), "bias_tokens")
        row = batch = 0
        if self.allowed is not None:
            words = (V + 31) // 32
            _whole(self.allowed, device, i32, (B, -1, words), "allowed")
            _need(self.allowed.shape[1] in (1, rows), "allowed: a mask a row, or one a sequence")
            row, batch = (words if self.allowed.shape[1] == rows else 0), self.allowed.shape[1] * words
        # a list without a place holds nothing; its address would be none
        tokens = self.tokens if self.tokens is not None and self.tokens.shape[1] else None
        bias = self.bias if self.bias is not None and self.bias.shape[1] else None
        return _Adjustments(_ptr(tokens), tokens.shape[1] if tokens is not None else 0, _ptr(self.n_tokens) if tokens is not None else None,
                            _ptr(self.n_prompt) if tokens is not None else None,
                            _ptr(self.repetition), _ptr(self.frequency), _ptr(self.presence), _ptr(self.bias_tokens) if bias is not None else None, _ptr(bias),
                            _ptr(self.n_bias), bias.shape[1] if bias is not None else 0, _ptr(self.allowed), row, batch)


def _rows(x, B, rows, V, name):
    _need(x.is_cuda and x.dim() == 3 and x.shape[0] == B and x.shape[1] == rows and x.shape[2] >= V and x.stride(2) == 1 and
          (B == 1 or x.stride(0) == rows * x.stride(1) or rows == 1 and x.stride(0) >= V), "%s: [%d][%d][at least %d], rows evenly spaced" % (name, B, rows, V))
    # (a sequence's one row is as far from the next one's as the sequences are; one row alone may be anywhere)
    return x.stride(1) if rows > 1 else x.stride(0) if B > 1 else max(x.stride(1), V + (-V) % (16 // x.element_size()))


def adjust_tree_logits(logits, tree, adjustments, vocab=None, out=None, stream=None):
    """The target model's logits [B][1 + N][stride >= vocab] (float32 or bfloat16) of a tree's root and nodes with `adjustments` (a
    LogitAdjustments) made, into `out` (a new tensor; may be `logits`).  tree: a finalize_tree output (tokens, parent, n_nodes), or None for one
    row a sequence.  Rows behind a sequence's nodes, and what is behind `vocab` (default: all), are left as they are."""
    L = load_library()
    B, rows = logits.shape[0], logits.shape[1]
    V = logits.shape[2] if vocab is None else int(vocab)
    dev = logits.device
    _need(logits.dtype in (torch.float32, torch.bfloat16), "logits: float32 or bfloat16")
    stride = _rows(logits, B, rows, V, "logits")
    if tree is None:
        _need(rows == 1, "logits: one row a sequence without a tree")
        tokens = parent = None
        n_nodes = torch.zeros(B, dtype=torch.int32, device=dev)
    else:
        tokens, parent, n_nodes = (_whole(tree[k], dev, torch.int32, s, "tree " + k) for k, s in
                                   (("tokens", (B, rows - 1)), ("parent", (B, rows - 1)), ("n_nodes", (B,))))
    if out is None:
        out = _empty_like_on(stream, lambda: torch.empty((B, rows, stride), dtype=logits.dtype, device=dev)[:, :, :logits.shape[2]])
    _need(out.dtype == logits.dtype and out.device == dev, "out: of the logits' type and device")
    a = adjustments._struct(B, rows, V, dev)
    out_stride = _rows(out, B, rows, V, "out")
    _check(_launch(dev, stream, lambda s: L.c2t_adjust_tree_logits(ctypes.byref(a), B, V, rows - 1, _DTYPES[logits.dtype], _ptr(tokens), _ptr(parent), n_nodes.data_ptr(),
                                                                    logits.data_ptr(), stride, out.data_ptr(), out_stride, s)), "c2t_adjust_tree_logits")
    return out


def adjust_frontier_logits(ctx, logits, adjustments, out=None, stream=None):
    """C2TContext.adjust_logits."""
    B, F, V = ctx.B, ctx.F, ctx.V
    _need(logits.dtype == ctx._logits_dtype and logits.device == ctx._ws.device, "logits: of the context's type and device")
    stride = _rows(logits, B, F, V, "logits")
    out = logits if out is None else out
    _need(out.dtype == logits.dtype and out.device == logits.device, "out: of the logits' type and device")
    a = adjustments._struct(B, F, V, logits.device)
    out_stride = _rows(out, B, F, V, "out")
    _check(_launch(logits.device, stream, lambda s: ctx.L.c2t_adjust_logits(ctx.ctx, ctypes.byref(a), logits.data_ptr(), stride, out.data_ptr(), out_stride, s)),
           "c2t_adjust_logits")
    return out


class PagedCache:
    """A paged K/V cache (c2t_cache): tensors k, v [layers][pages][kv_heads][page_size][head_dim], page_table int32 [B][max_pages] (-1: no
    page), length int32 [B], refcount int32 [pages], status uint32 [B] (POOL_EMPTY, ROW_FULL, INVALID, SHARED; set by calls, cleared by the
    user).  All calls are enqueued on torch's current stream (or `stream`) and answer on the device alone.  Calls on one cache belong on one
    stream; attention alone may run on several (each stream has a workspace of its own)."""
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
        _whole(k, k.device, k.dtype, tuple(k.shape), "k")
        self.k, self.v = k, _whole(v, k.device, k.dtype, tuple(k.shape), "v")
        self.page_table = _whole(page_table, k.device, torch.int32, (-1, -1), "page_table")
        batch, max_pages = page_table.shape
        self.length = _whole(length, k.device, torch.int32, (batch,), "length")
        self.refcount = _whole(refcount, k.device, torch.int32, (pages,), "refcount")
        self.status = torch.zeros(batch, dtype=torch.int32, device=k.device).view(torch.uint32)
        self.batch, self.layers, self.pages, self.page_size, self.kv_heads, self.head_dim, self.max_pages = batch, layers, pages, page_size, kv_heads, head_dim, max_pages
        self._c = _Cache(batch, layers, pages, page_size, kv_heads, head_dim, max_pages, _DTYPES[k.dtype], k.data_ptr(), v.data_ptr(), page_table.data_ptr(),
                         length.data_ptr(), refcount.data_ptr(), self.status.data_ptr())
        self._ref = ctypes.byref(self._c)
        need = ctypes.c_size_t()
        _check(self.L.c2t_cache_workspace_bytes(self._ref, ctypes.byref(need)), "c2t_cache_workspace_bytes")
        self._ws = self._workspace(need.value)
        self._attention_ws = {}                            # (stream, capture, bytes) -> workspace; kept: a captured graph refers to it
        self._capture = ctypes.c_uint64()
        self._capture_ref = ctypes.byref(self._capture)
        self._attention_bytes = {}

    def _workspace(self, nbytes):
        w = torch.zeros(nbytes + 256, dtype=torch.uint8, device=self.device)
        pad = (-w.data_ptr()) % 256
        return w[pad:pad + nbytes]

    def _run(self, what, stream, *args):
        fn = getattr(self.L, what)
        rc = _launch(self.device, stream, lambda s: fn(self._ref, *args, s))
        if rc != 0:
            raise binding.C2TError(rc, what)

    def _per_sequence(self, t, name):
        return _whole(t, self.device, torch.int32, (self.batch,), name).data_ptr()

    def reserve(self, n_new, stream=None):
        """Pages for n_new (int32 [B]) tokens behind each sequence's length, its own to write."""
        self._run("c2t_cache_reserve", stream, self._per_sequence(n_new, "n_new"), self._ws.data_ptr(), self._ws.numel())

    def _tokens(self, x, heads, name):
        _need(x.device == self.device and x.dtype == self.dtype and x.dim() == 4 and x.shape[0] == self.batch and x.shape[1] > 0 and
              x.shape[2] == heads and x.shape[3] == self.head_dim and x.stride(3) == 1 and (heads == 1 or x.stride(2) == self.head_dim),
              "%s: %s [%d][tokens][%d][%d] on %s, heads next to each other" % (name, self.dtype, self.batch, heads, self.head_dim, self.device))
        # (a stride over one element is of no use and may be any number)
        row = heads * self.head_dim
        token = x.stride(1) if x.shape[1] > 1 else row
        return (x.stride(0) if self.batch > 1 else row), token

    def write(self, layer, k, v, n_new=None, stream=None):
        """K and V [B][tokens][kv_heads][head_dim] of new tokens, n_new (int32 [B], default all) of them, to positions length + t of `layer`."""
        sk, sv = self._tokens(k, self.kv_heads, "k"), self._tokens(v, self.kv_heads, "v")
        _need(k.shape == v.shape and sk == sv, "k and v: of one shape and strides")
        self._run("c2t_cache_write", stream, int(layer), k.data_ptr(), v.data_ptr(), sk[0], sk[1], k.shape[1],
                  None if n_new is None else self._per_sequence(n_new, "n_new"))

    def commit(self, path, n_path, stream=None):
        """The tokens in slots path[b][i] (int32 [B][P], rising) behind the length move to slots i < n_path[b]; the length grows by n_path."""
        _whole(path, self.device, torch.int32, (self.batch, -1), "path")
        self._run("c2t_cache_commit", stream, path.data_ptr(), path.shape[1], self._per_sequence(n_path, "n_path"))

    def truncate(self, new_length=None, keep=0, stream=None):
        """Lengths cut to new_length (int32 [B], default as they are); pages behind length + keep tokens let go."""
        self._run("c2t_cache_truncate", stream, None if new_length is None else self._per_sequence(new_length, "new_length"), int(keep))

    def fork(self, src, dst, stream=None):
        """Sequences dst[i] become copies of src[i] (int32 [n] each); the pages are shared until they are written."""
        n = _whole(src, self.device, torch.int32, (-1,), "src").shape[0]
        _whole(dst, self.device, torch.int32, (n,), "dst")
        self._run("c2t_cache_fork", stream, src.data_ptr(), dst.data_ptr(), n)

    def attention(self, layer, q, n_new=None, mask=None, scale=None, out=None, lse=None, workspace=None, stream=None):
        """Attention of the last n_new (int32 [B], default all) tokens, which have been written behind the length, over the cache.

        q [B][T][q_heads][head_dim]; mask uint8 [B][N][N] as finalize_tree writes it: the last N of the T slots are the tree's nodes, those
        before them (the root) a causal chain; no mask: all of them are.  scale: of the scores, default head_dim ** -0.5.  lse: float32
        [B][T][q_heads] for the log of the softmax's sums.  out: [B][T][q_heads][head_dim] (default: a new tensor), rows behind n_new left as
        they are.  workspace: uint8, zeros, of attention_workspace_bytes and 256-byte aligned, for calls that run at once otherwise than by stream."""
        _need(q.dim() == 4, "q: [B][T][q_heads][head_dim]")
        heads, T = q.shape[2], q.shape[1]
        sq = self._tokens(q, heads, "q")
        if out is None:
            out = _empty_like_on(stream, lambda: torch.empty((self.batch, T, heads, self.head_dim), dtype=self.dtype, device=self.device))
        _need(out.shape == q.shape, "out: of q's shape")
        so = self._tokens(out, heads, "out")
        nodes = 0
        if mask is not None:
            nodes = mask.shape[-1]
            _whole(mask, self.device, torch.uint8, (self.batch, nodes, nodes), "mask")
        if lse is not None:
            _whole(lse, self.device, torch.float32, (self.batch, T, heads), "lse")
        a = _Attention(q.data_ptr(), sq[0], sq[1], out.data_ptr(), so[0], so[1], _ptr(lse), None if n_new is None else self._per_sequence(n_new, "n_new"),
                       T, heads, int(layer), nodes, _ptr(mask) if nodes else None, self.head_dim ** -0.5 if scale is None else float(scale))
        ref = ctypes.byref(a)
        need = self._attention_bytes.get((T, heads, nodes))
        if need is None:
            n = ctypes.c_size_t()
            _check(self.L.c2t_attention_workspace_bytes(self._ref, ref, ctypes.byref(n)), "c2t_attention_workspace_bytes")
            need = self._attention_bytes[(T, heads, nodes)] = n.value

        def call(s):
            w = workspace
            if w is None:
                w = self._attention_workspace(s, need)
            return self.L.c2t_cache_attention(self._ref, ref, w.data_ptr(), w.numel(), s)
        rc = _launch(self.device, stream, call)
        if rc != 0:
            raise binding.C2TError(rc, "c2t_cache_attention")
        return out

    def _attention_workspace(self, s, need):
        """One a stream, and one a captured graph: graphs may be replayed at once, and an eager call beside them."""
        capture = 0
        if s:
            _check(self.L.c2t_stream_capture_id(s, self._capture_ref), "c2t_stream_capture_id")
            capture = self._capture.value
        key = (s, capture, need)
        w = self._attention_ws.get(key)
        if w is None:
            w = self._attention_ws[key] = self._workspace(need)
        return w

    def attention_workspace_bytes(self, tokens, q_heads, nodes=0):
        a = _Attention(tokens=tokens, q_heads=q_heads, nodes=nodes)
        n = ctypes.c_size_t()
        _check(self.L.c2t_attention_workspace_bytes(self._ref, ctypes.byref(a), ctypes.byref(n)), "c2t_attention_workspace_bytes")
        return n.value

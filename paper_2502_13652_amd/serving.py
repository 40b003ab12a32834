"""What goes around a draft phase: a paged K/V cache with its attention, and adjusted logits (the second part of
include/c2t.h).  Argument marshalling and checks only; like the binding it needs a GPU and has no fallback."""
import ctypes
import dataclasses
import struct
import threading
from typing import Optional

import torch

from . import binding
from .binding import BF16, F16, F32, _check, load_library

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


def _packer(fields):
    """A call's structure as bytes: a third of the time that ctypes takes to fill one.  The layout is the structure's."""
    code = {ctypes.c_void_p: "P", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f"}
    p = struct.Struct("@" + "".join(code[t] for _, t in fields._fields_) + "0P")
    assert p.size == ctypes.sizeof(fields)
    return p.pack


_pack_adjustments, _pack_attention = _packer(_Adjustments), _packer(_Attention)


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


def _launch(device, stream, fn, *args):
    """fn(*args, stream handle) with the tensors' device current."""
    if stream is None and _current_device() == device.index:
        return fn(*args, binding._stream_ptr(None))
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

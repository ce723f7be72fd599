"""The attention half of a serving iteration's layer: keys and values in pages,
the attention of each slot's new token over them, and the norms around a block
with their gradient (fm_kv_*, fm_attn_*, fm_block_norm* of
include/finemoe_map.h).

Argument marshalling only, under the conventions of model.py.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import _DTYPES, _TORCH, _aligned_bytes, _lib, _need, _ptr, _raw_stream
from .model import _CODE, _call, _flags, _float_rows, _new, _on

_GRADS = "dx", "dy", "dpost", "dgate", "dpre"


def _int32(n: int, name: str) -> int:
    """n, which ctypes would cut to 32 bits."""
    if not -2 ** 31 <= n < 2 ** 31:
        raise ValueError(f"{name}={n} does not fit 32 bits")
    return n


def kv_page_bytes(layers: int, heads: int, head_dim: int, page: int = 64, dtype: str = "bf16") -> int:
    return int(_lib.load().fm_kv_page_bytes(_int32(layers, "layers"), _int32(heads, "heads"),
                                            _int32(head_dim, "head_dim"), _int32(page, "page"), _DTYPES[dtype]))


class KvCache:
    """Keys and values of a batch's requests on the GPU, in pages that all layers of ``page`` tokens share.

    ``pages`` [n_pages][elements of a page], ``table`` [slots][max_pages] int32, ``length`` [slots] int32 (tokens of a
    slot) and ``refs`` [n_pages] int32 (slots that hold a page) are plain tensors that the owner may also fill itself, in
    place and in agreement with each other: calls read the memory that they had at first.  Calls that change the cache
    must be ordered with every other call on it."""

    def __init__(self, slots: int, max_tokens: int, pages: int, layers: int, heads: int, head_dim: int,
                 dtype: str = "bf16", page: int = 64, device="cuda"):
        self.slots, self.n_pages, self.page = _int32(int(slots), "slots"), _int32(int(pages), "pages"), int(page)
        self.layers, self.heads, self.head_dim = int(layers), int(heads), int(head_dim)
        self.dtype = _TORCH[_DTYPES[dtype]]
        self.page_bytes = kv_page_bytes(self.layers, self.heads, self.head_dim, self.page, dtype)
        if self.page_bytes == 0:
            raise ValueError(f"invalid cache page={page} layers={layers} heads={heads} head_dim={head_dim}")
        self.max_pages = _int32((int(max_tokens) + self.page - 1) // self.page, "max_pages")
        self._desc = _lib.KvCacheDesc(self.slots, self.max_pages, self.n_pages, self.page, self.layers, self.heads,
                                      self.head_dim, _DTYPES[dtype], None, None, None, None)
        self.desc = C.byref(self._desc)
        scratch = int(_lib.load().fm_kv_scratch_bytes(self.desc))
        if scratch == 0:
            raise ValueError(f"invalid cache slots={slots} max_tokens={max_tokens} pages={pages}")
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._pages = _aligned_bytes(self.n_pages * self.page_bytes, self.device).view(self.dtype).view(self.n_pages, -1)
        self._table = torch.full((self.slots, self.max_pages), -1, dtype=torch.int32, device=self.device)
        self._length = torch.zeros(self.slots, dtype=torch.int32, device=self.device)
        self._refs = torch.zeros(self.n_pages, dtype=torch.int32, device=self.device)
        self.flags = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._scratch = _aligned_bytes(scratch, self.device)
        for name in ("pages", "table", "length", "refs"):
            setattr(self._desc, name, getattr(self, name).data_ptr())
        self._workspaces = {}    # stream handle -> the workspace of its calls
        self._replaced = []      # workspaces that calls of more query heads outgrew

    @property
    def pages(self) -> torch.Tensor:
        return self._pages

    @pages.setter
    def pages(self, t):
        self._same(t, self._pages, "pages")

    @property
    def table(self) -> torch.Tensor:
        return self._table

    @table.setter
    def table(self, t):
        self._same(t, self._table, "table")

    @property
    def length(self) -> torch.Tensor:
        return self._length

    @length.setter
    def length(self, t):
        self._same(t, self._length, "length")

    @property
    def refs(self) -> torch.Tensor:
        return self._refs

    @refs.setter
    def refs(self, t):
        self._same(t, self._refs, "refs")

    @staticmethod
    def _same(t, own, name: str) -> None:
        if t is not own:   # (cache.length += 1 ends in such an assignment)
            raise AttributeError(f"{name} cannot be replaced: write into it")

    def check(self, stream=None) -> int:
        """Synchronise the stream and return the sticky FM_FLAG_* bits of the calls that it has seen, cleared.  Calls on
        other streams must have ended: a bit that one sets in the meantime may be cleared unseen."""
        with _on(stream):
            f = int(self.flags.item())
            self.flags.zero_()
        return f

    def ensure_workspace(self, q_heads: int, stream=None) -> "AttnWorkspace":
        """The cache's own workspace of the stream, made or enlarged for attn_decode calls of q_heads query heads.  Each
        stream has one; one that is replaced stays allocated as long as the cache: a captured graph may hold its
        address."""
        handle = self._handle(stream)
        own = self._workspaces.get(handle)
        if own is None or attn_workspace_bytes(self, q_heads) > own.nbytes:
            with _on(stream):
                made = AttnWorkspace(self, q_heads)
            if own is not None:
                self._replaced.append(own)
            own = self._workspaces[handle] = made
        return own

    def _handle(self, stream) -> int:
        """The hipStream_t of ``stream``, or of the current stream of the cache's device (0 for one that is no GPU)."""
        if stream is not None:
            return stream.cuda_stream
        if self.device.type != "cuda":
            return 0
        if _raw_stream is None:
            return torch.cuda.current_stream(self.device).cuda_stream
        return _raw_stream(self.device.index)


def attn_workspace_bytes(cache: KvCache, q_heads: int) -> int:
    return int(_lib.load().fm_attn_workspace_bytes(cache.desc, _int32(q_heads, "q_heads")))


def _capturing(device: torch.device) -> bool:
    """Whether the current stream of the device, which need not be the current one, records a graph."""
    if device.type != "cuda":
        return False
    with torch.cuda.device(device):
        return torch.cuda.is_current_stream_capturing()


class AttnWorkspace:
    """Device scratch for attn_decode calls of q_heads query heads on a cache.  Calls sharing one must be ordered; all
    layers may share one.  Its first bytes count parts of split sequences: zeros between calls.  The zeros of one that is
    made during a graph's capture come with that graph's replays only, so every call with it brings its own."""

    def __init__(self, cache: KvCache, q_heads: int):
        self.nbytes = attn_workspace_bytes(cache, q_heads)
        if self.nbytes == 0:
            raise ValueError(f"invalid workspace request q_heads={q_heads} for {cache.heads} heads")
        self.buf = _aligned_bytes(self.nbytes, cache.device)
        self.in_capture = _capturing(cache.device)
        self.clear()

    def clear(self) -> None:
        self.buf[:_lib.FM_ATTN_TICKET_BYTES].zero_()


def _change(name: str, cache: KvCache, stream, *args) -> None:
    _call(name, cache.device, stream, cache.desc, *args, _flags(cache.flags, cache.device), cache._scratch.data_ptr(),
          cache._scratch.numel())


def kv_resize(cache: KvCache, delta: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Room for delta[s] more tokens behind slot s (> 0), or its last -delta[s] dropped (< 0; -2^31 ends any request):
    delta [slots] int32 -> granted [slots] uint8, 1 where tokens were added: the ``active`` of the calls that follow.
    Slots that find no free page are refused and flagged (cache.check())."""
    _need(delta, "delta", torch.int32, (cache.slots,), cache.device)
    if out is None:
        out = _new((cache.slots,), torch.uint8, cache.device, stream)
    else:
        _need(out, "out", torch.uint8, (cache.slots,), cache.device)
    _change("fm_kv_resize", cache, stream, delta.data_ptr(), out.data_ptr())
    return out


def kv_fork(cache: KvCache, parent: torch.Tensor, stream=None) -> None:
    """Slot s becomes what slot parent[s] was, sharing its pages; -1 leaves it alone.  parent [slots] int32."""
    _need(parent, "parent", torch.int32, (cache.slots,), cache.device)
    _change("fm_kv_fork", cache, stream, parent.data_ptr())


def kv_compact(cache: KvCache, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Move the live pages to the lowest numbers -> how many there are, [1] int32: cache.pages from there on is free."""
    if out is None:
        out = _new((1,), torch.int32, cache.device, stream)
    else:
        _need(out, "out", torch.int32, (1,), cache.device)
    _change("fm_kv_compact", cache, stream, out.data_ptr())
    return out


def kv_copy(cache: KvCache, src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
    """Contents of the pages src [n] int32 to the pages dst [n]; tables and counts stay.  Pairs whose destination is
    named twice, or that name no page, are left out and flagged."""
    _need(src, "src", torch.int32, (None,), cache.device)
    _need(dst, "dst", torch.int32, (src.shape[0],), cache.device)
    _change("fm_kv_copy", cache, stream, src.data_ptr(), dst.data_ptr(), _int32(src.shape[0], "n"))


def _rows(t, name: str, dtype, T: Optional[int], heads: Optional[int], head_dim: int, device) -> Tuple[int, int, int, int]:
    """Address, row stride, T and heads of a [T][heads][head_dim] tensor whose rows need not follow each other (None:
    any)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 3 or shape[2] != head_dim or (heads is not None and shape[1] != heads) \
            or (T is not None and shape[0] != T) or t.device != device:
        want = "x".join("*" if w is None else str(w) for w in (T, heads, head_dim))
        raise ValueError(f"{name} must be a {dtype} [{want}] tensor on {device}, got {t.dtype} {list(shape)} on "
                         f"{t.device}")
    T, H, D = shape
    row, head, one = t.stride()
    if (one != 1 and D > 1) or (head != D and H > 1) or (row < H * D and T > 1):
        raise ValueError(f"{name} must have contiguous rows, got strides {t.stride()}")
    return t.data_ptr(), row if T > 1 else H * D, T, H


def _token_rows(name: str, cache: KvCache, layer: int, k, v, offsets, active, stream) -> None:
    dev = cache.device
    slots = cache.slots if offsets is None else None
    k_ptr, k_stride, T, _ = _rows(k, "k", cache.dtype, slots, cache.heads, cache.head_dim, dev)
    v_ptr, v_stride, rows, _ = _rows(v, "v", cache.dtype, slots, cache.heads, cache.head_dim, dev)
    if T != rows:
        raise ValueError(f"k and v must have as many rows, got {T} and {rows}")
    if offsets is not None:
        _need(offsets, "offsets", torch.int32, (cache.slots + 1,), dev)
    if active is not None:
        _need(active, "active", torch.uint8, (cache.slots,), dev)
    _call(name, dev, stream, cache.desc, _int32(layer, "layer"), k_ptr, k_stride, v_ptr, v_stride, _ptr(offsets),
          _int32(T, "T"), _ptr(active), _flags(cache.flags, dev))


def kv_write(cache: KvCache, layer: int, k: torch.Tensor, v: torch.Tensor, offsets: Optional[torch.Tensor] = None,
             active: Optional[torch.Tensor] = None, stream=None) -> None:
    """Keys and values of new tokens into a layer's pages: k, v [T][heads][head_dim], whose rows may be parts of longer
    ones.  Without ``offsets`` row s is slot s's last token; otherwise rows offsets[s] .. offsets[s + 1] - 1 are its last
    ones (offsets [slots + 1] int32).  Slots where active [slots] uint8 is 0 write nothing."""
    _token_rows("fm_kv_write", cache, layer, k, v, offsets, active, stream)


def kv_read(cache: KvCache, layer: int, T: Optional[int] = None, offsets: Optional[torch.Tensor] = None,
            active: Optional[torch.Tensor] = None, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream=None):
    """The reverse of kv_write: -> (k, v), rows that belong to no slot left as they are (zeros without ``out``).  With
    ``offsets`` and without ``out``, T says how many rows there are."""
    if out is None:
        if T is None:
            if offsets is not None:
                raise ValueError("offsets need T or out")
            T = cache.slots
        with _on(stream):
            out = tuple(torch.zeros((T, cache.heads, cache.head_dim), dtype=cache.dtype, device=cache.device)
                        for _ in range(2))
    elif T is not None and any(t.shape[0] != T for t in out):
        raise ValueError(f"out must have T={T} rows")
    _token_rows("fm_kv_read", cache, layer, out[0], out[1], offsets, active, stream)
    return out


def attn_decode(cache: KvCache, layer: int, q: torch.Tensor, scale: Optional[float] = None, window: int = 0,
                first: Optional[torch.Tensor] = None, active: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                workspace: Optional[AttnWorkspace] = None, stream=None) -> torch.Tensor:
    """Attention of every slot's last token over the slot's tokens of a layer: q [slots][q_heads][head_dim] (rows may be
    parts of longer ones) -> [slots][q_heads][head_dim].  scale defaults to head_dim ** -0.5; the last ``window`` tokens
    are seen (0: all), from place first[s] on (int32 [slots]); slots where active [slots] uint8 is 0, and queries that
    see no token, give zeros.  ``lse`` [slots][q_heads] float32 takes the log of each query's sum of weights.  Without
    ``workspace`` the cache's own of the stream serves the call (cache.ensure_workspace before a capture saves it a fill
    per call); replays of all graphs that captured such calls on one stream must be ordered with each other and with the
    later calls on that stream."""
    dev = cache.device
    q_ptr, q_stride, _, q_heads = _rows(q, "q", cache.dtype, cache.slots, None, cache.head_dim, dev)
    if out is None:
        out = _new((cache.slots, q_heads, cache.head_dim), cache.dtype, dev, stream)
    else:
        _need(out, "out", cache.dtype, (cache.slots, q_heads, cache.head_dim), dev)
        if out.data_ptr() == q_ptr:
            raise ValueError("out must not be q")
    if first is not None:
        _need(first, "first", torch.int32, (cache.slots,), dev)
    if active is not None:
        _need(active, "active", torch.uint8, (cache.slots,), dev)
    if lse is not None:
        _need(lse, "lse", torch.float32, (cache.slots, q_heads), dev)
    if workspace is None:
        if q_heads < 1 or q_heads % cache.heads != 0:
            raise ValueError(f"q has {q_heads} heads, not a multiple of the cache's {cache.heads}")
        workspace = cache.ensure_workspace(q_heads, stream)
    _need(workspace.buf, "workspace", torch.uint8, (workspace.nbytes,), dev)
    if workspace.in_capture:
        with _on(stream):
            workspace.clear()
    _call("fm_attn_decode", dev, stream, cache.desc, _int32(layer, "layer"), q_ptr, q_stride,
          _int32(q_heads, "q_heads"), cache.head_dim ** -0.5 if scale is None else scale, _int32(window, "window"),
          _ptr(first), _ptr(active), out.data_ptr(), _ptr(lse), _flags(cache.flags, dev), workspace.buf.data_ptr(), workspace.nbytes)
    return out


def _usual(t, dtype, shape, device) -> bool:
    """Whether _need has nothing to say about t."""
    return type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous()


def _norm_inputs(x, y, post, gate, pre):
    """Check the inputs that a norm and its gradient share -> the gate's kind, x's shape, type and device."""
    _float_rows(x, "x")
    shape, dtype, dev = x.shape, x.dtype, x.device
    T, d = shape
    row = (d,)
    if y is not None and not _usual(y, dtype, shape, dev):
        _need(y, "y", dtype, (T, d), dev)
    if post is not None and not _usual(post, dtype, row, dev):
        _need(post, "post", dtype, row, dev)
    if pre is not None and not _usual(pre, dtype, row, dev):
        _need(pre, "pre", dtype, row, dev)
    if gate is None:
        return 0, shape, dtype, dev
    if not isinstance(gate, torch.Tensor):
        raise TypeError(f"gate must be a torch.Tensor, got {type(gate).__name__}")
    g = gate.shape
    kind = 1 if g == row else 3 if g == shape else 2 if g == (T, 1) else 0
    if kind == 0:
        raise ValueError(f"gate must have shape [{d}], [{T}x1] or [{T}x{d}], got {list(g)}")
    _need(gate, "gate", dtype, g, dev)
    return kind, shape, dtype, dev


def block_norm(x: torch.Tensor, y: Optional[torch.Tensor] = None, post: Optional[torch.Tensor] = None,
               gate: Optional[torch.Tensor] = None, scale: float = 1.0, pre: Optional[torch.Tensor] = None,
               eps: float = 1e-6, out=None, stream=None):
    """A block's output into the residual stream, and the norm before the next block, in one pass:
    r = x + scale * gate * norm(y) * post, h = norm(r) * pre, norm(z) = z / sqrt(mean(z^2) + eps) -> (r, h).
    x, y [T][d], post and pre [d], gate [d], [T][1] or [T][d].  Without post y is not normed, without pre h is None,
    without y (the norm before a first block) r is x itself.  ``out`` gives (r, h): r may be x or y, h may be y."""
    kind, shape, dtype, dev = _norm_inputs(x, y, post, gate, pre)
    r, h = (None, None) if out is None else out
    if y is None:
        if r is not None and r is not x:
            raise ValueError("out[0] (r) must be None or x without y")
        if pre is None or post is not None or kind:
            raise ValueError("without y there is only the norm by pre")
        r = None
    elif r is None:
        r = _new(shape, dtype, dev, stream)
    elif not _usual(r, dtype, shape, dev):
        _need(r, "out[0] (r)", dtype, shape, dev)
    if pre is None:
        if h is not None:
            raise ValueError("out[1] (h) must be None without pre")
    elif h is None:
        h = _new(shape, dtype, dev, stream)
    elif not _usual(h, dtype, shape, dev):
        _need(h, "out[1] (h)", dtype, shape, dev)
    _call("fm_block_norm", dev, stream, x.data_ptr(), _ptr(y), _ptr(post), _ptr(gate), kind, scale, _ptr(pre), eps,
          _int32(shape[0], "T"), _int32(shape[1], "d"), _CODE[dtype], _ptr(r), _ptr(h))
    return (x if r is None else r), h


def block_norm_scratch_bytes(T_max: int, d: int) -> int:
    return int(_lib.load().fm_block_norm_scratch_bytes(_int32(T_max, "T_max"), _int32(d, "d")))


class BlockNormScratch:
    """Device scratch for block_norm_grad calls of up to T_max tokens (every call rewrites what it reads).  Calls
    sharing one must be ordered."""

    def __init__(self, T_max: int, d: int, device="cuda"):
        self.nbytes = block_norm_scratch_bytes(T_max, d)
        if self.nbytes == 0:
            raise ValueError(f"invalid scratch request T_max={T_max} d={d}")
        self.buf = _aligned_bytes(self.nbytes, device)


def block_norm_grad(dr: Optional[torch.Tensor], dh: Optional[torch.Tensor], x: torch.Tensor,
                    y: Optional[torch.Tensor] = None, post: Optional[torch.Tensor] = None,
                    gate: Optional[torch.Tensor] = None, scale: float = 1.0, pre: Optional[torch.Tensor] = None,
                    eps: float = 1e-6, accumulate: bool = False, out=None, scratch: Optional[BlockNormScratch] = None,
                    stream=None):
    """Gradient of block_norm, whose inputs come again: dr and dh are the gradients of r and h (dr may be None, dh is
    given exactly where pre is) -> (dx, dy, dpost, dgate, dpre), None where the input is.  dx and dy are of x's type; dpost,
    dpre and the gradient of a gate per channel or token float32, of a full gate x's type.  accumulate adds the sums
    over tokens (dpost, dpre, a channel gate's) to what ``out`` holds.  dx may be dr, dy may be y or dh."""
    kind, shape, dtype, dev = _norm_inputs(x, y, post, gate, pre)
    T, d = shape
    if dr is not None and not _usual(dr, dtype, shape, dev):
        _need(dr, "dr", dtype, shape, dev)
    if dh is not None and not _usual(dh, dtype, shape, dev):
        _need(dh, "dh", dtype, shape, dev)
    if y is None and (post is not None or kind):
        raise ValueError("post and gate need y")
    if (dh is None) != (pre is None):
        raise ValueError("dh must be given exactly where pre is")
    if dr is None and dh is None:
        raise ValueError("dr or dh is required")
    # what each gradient is like, where its input is
    row = (d,)
    want = (shape, dtype), None if y is None else (shape, dtype), None if post is None else (row, torch.float32), \
        None if kind == 0 else (gate.shape, dtype if kind == 3 else torch.float32), \
        None if pre is None else (row, torch.float32)
    if out is None:
        if accumulate and (post is not None or pre is not None or kind == 1):
            raise ValueError("accumulate needs out")
        out = tuple(None if w is None else _new(*w, dev, stream) for w in want)
    else:
        if len(out) != 5:
            raise ValueError(f"out must hold dx, dy, dpost, dgate and dpre, got {len(out)}")
        for i, (t, w) in enumerate(zip(out, want)):
            if w is None:
                if t is not None:
                    raise ValueError(f"out[{i}] ({_GRADS[i]}) must be None: its input is")
            elif not _usual(t, w[1], w[0], dev):
                _need(t, f"out[{i}] ({_GRADS[i]})", w[1], w[0], dev)
    if scratch is None:
        with _on(stream):
            scratch = BlockNormScratch(T, d, dev)
    _need(scratch.buf, "scratch", torch.uint8, (scratch.nbytes,), dev)
    dx, dy, dpost, dgate, dpre = out
    _call("fm_block_norm_grad", dev, stream, _ptr(dr), _ptr(dh), x.data_ptr(), _ptr(y), _ptr(post), _ptr(gate), kind,
          scale, _ptr(pre), eps, _int32(T, "T"), _int32(d, "d"), _CODE[dtype], 1 if accumulate else 0, dx.data_ptr(),
          _ptr(dy), _ptr(dpost), _ptr(dgate), _ptr(dpre), scratch.buf.data_ptr(), scratch.nbytes)
    return out

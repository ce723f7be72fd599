"""The model operators around the expert-map search: token embeddings and their
gradient, the gate of an MoE layer, and the chosen experts' products on experts
that a cache holds (fm_embed_*, fm_moe_* of include/finemoe_map.h).

Argument marshalling only, as the rest of the binding: every step runs in the
library's HIP kernels.  Tensors must be contiguous, on one GPU and of the stated
type; outputs are created unless ``out`` gives them.  Work goes to the current
stream, or to ``stream``, and memory that a call creates (outputs, scratch,
workspaces) belongs to the same stream.  The calls stand outside torch's
autograd: no output requires a gradient, whatever the inputs do, and embed_grad
is the lookup's.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Tuple

import torch

from . import _DTYPES, _TORCH, _aligned_bytes, _lib, _need, _ptr, _raw_stream, _stream

_CODE = {torch.float32: _lib.FM_F32, torch.bfloat16: _lib.FM_BF16}
_LIBRARY = _lib.load()


def _call(name: str, device: torch.device, stream, *args) -> None:
    """Call the library, which enqueues on the current device, with the tensors' device current."""
    if device.type != "cuda":
        raise ValueError(f"tensors are on {device}, not on a GPU")
    if device.index == torch.cuda.current_device():
        status = getattr(_LIBRARY, name)(*args, _stream(stream))
    else:
        with torch.cuda.device(device):
            status = getattr(_LIBRARY, name)(*args, _stream(stream))
    if status != _lib.FM_OK:
        _lib.check(status, name)


def _on(stream):
    """The allocator's context for memory that work on ``stream`` uses: a block that another stream owns could be in
    use there still, or be given out there again while this work runs."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _new(shape, dtype: torch.dtype, device: torch.device, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _on(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _float_rows(t, name: str) -> torch.Tensor:
    """A float32 or bfloat16 matrix; later tensors are checked against its device."""
    if type(t) is torch.Tensor and t.dtype in _CODE and t.dim() == 2 and t.is_contiguous():
        return t   # the usual case
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in _CODE:
        raise ValueError(f"{name} must be torch.float32 or torch.bfloat16, got {t.dtype}")
    return _need(t, name, t.dtype, (None, None), t.device)


def _vector(t, name: str, device: torch.device) -> int:
    """The length of an int32 vector."""
    if not (type(t) is torch.Tensor and t.dtype is torch.int32 and t.dim() == 1 and t.device == device
            and t.is_contiguous()):
        _need(t, name, torch.int32, (None,), device)
    return t.shape[0]


def _flags(flags, dev):
    return None if flags is None else _need(flags, "flags", torch.int32, (1,), dev).data_ptr()


def embed_lookup(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                 flags: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """scale * table[tokens]: table [V][d], tokens [T] int32 (negative: padding, a row of zeros) -> [T][d]."""
    _float_rows(table, "table")
    V, d = table.shape
    dev = table.device
    T = _vector(tokens, "tokens", dev)
    if out is None:
        out = _new((T, d), table.dtype, dev, stream)
    else:
        _need(out, "out", table.dtype, (T, d), dev)
    _call("fm_embed_lookup", dev, stream, table.data_ptr(), V, d, _CODE[table.dtype], tokens.data_ptr(), T, scale,
          out.data_ptr(), _flags(flags, dev))
    return out


def embed_pool(table: torch.Tensor, tokens: torch.Tensor, offsets: torch.Tensor, scale: float = 1.0,
               out: Optional[torch.Tensor] = None, flags: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Mean embedding of each request, times scale: offsets [B + 1] int32 into tokens -> [B][d] bfloat16, the
    queries of match_semantic."""
    _float_rows(table, "table")
    V, d = table.shape
    dev = table.device
    T = _vector(tokens, "tokens", dev)
    B = _vector(offsets, "offsets", dev) - 1
    if B < 0:
        raise ValueError("offsets must hold at least one element")
    if out is None:
        out = _new((B, d), torch.bfloat16, dev, stream)
    else:
        _need(out, "out", torch.bfloat16, (B, d), dev)
    _call("fm_embed_pool", dev, stream, table.data_ptr(), V, d, _CODE[table.dtype], tokens.data_ptr(), T,
          offsets.data_ptr(), B, scale, out.data_ptr(), _flags(flags, dev))
    return out


def embed_grad_scratch_bytes(T_max: int, V: int) -> int:
    return int(_lib.load().fm_embed_grad_scratch_bytes(T_max, V))


class EmbedGradScratch:
    """Device scratch for embed_grad calls of up to T_max tokens on a table of V
    rows (every call rewrites what it reads).  Calls sharing one must be ordered."""

    def __init__(self, T_max: int, V: int, device="cuda"):
        self.nbytes = embed_grad_scratch_bytes(T_max, V)
        if self.nbytes == 0:
            raise ValueError(f"invalid scratch request T_max={T_max} V={V}")
        self.buf = _aligned_bytes(self.nbytes, device)


def embed_grad(dout: torch.Tensor, tokens: torch.Tensor, V: int, scale: float = 1.0,
               grad_dtype: Optional[torch.dtype] = None, accumulate: bool = False, out: Optional[torch.Tensor] = None,
               scratch: Optional[EmbedGradScratch] = None, flags: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """Gradient of embed_lookup with respect to the table: dout [T][d], tokens [T] int32 -> [V][d] of grad_dtype
    (float32 by default, or out's).  accumulate adds to the rows of ``out`` that tokens select."""
    _float_rows(dout, "dout")
    T, d = dout.shape
    dev = dout.device
    _need(tokens, "tokens", torch.int32, (T,), dev)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = _new((V, d), torch.float32 if grad_dtype is None else grad_dtype, dev, stream)
    if grad_dtype is not None and out.dtype != grad_dtype:
        raise ValueError(f"out must be {grad_dtype}, got {out.dtype}")
    _float_rows(out, "out")
    _need(out, "out", out.dtype, (V, d), dev)
    if scratch is None:
        with _on(stream):
            scratch = EmbedGradScratch(T, V, dev)
    _need(scratch.buf, "scratch", torch.uint8, (scratch.nbytes,), dev)
    _call("fm_embed_grad", dev, stream, dout.data_ptr(), _CODE[dout.dtype], tokens.data_ptr(), T, V, d, scale,
          1 if accumulate else 0, out.data_ptr(), _CODE[out.dtype], scratch.buf.data_ptr(), scratch.nbytes,
          _flags(flags, dev))
    return out


def moe_route(x: torch.Tensor, gate: torch.Tensor, k: int, renorm: bool = False,
              active: Optional[torch.Tensor] = None, probs_dtype: torch.dtype = torch.float32,
              out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, Optional[torch.Tensor]]] = None,
              stream=None):
    """The gate of one MoE layer: x [T][d], gate [E][d], active [T] uint8 or None -> (probs [T][E], ids [T][k] int32,
    weight [T][k] float32, mask [T] int64 holding uint64 bits).  ``out`` may give probs as a layer's rows of a batch of
    maps or trajectory queries (q[:, layer]): its rows need not follow each other; mask may be None there."""
    _float_rows(x, "x")
    T, d = x.shape
    dev = x.device
    _float_rows(gate, "gate")
    E = gate.shape[0]
    _need(gate, "gate", x.dtype, (E, d), dev)
    if active is not None:
        _need(active, "active", torch.uint8, (T,), dev)
    if out is None:
        out = (_new((T, E), probs_dtype, dev, stream), _new((T, k), torch.int32, dev, stream),
               _new((T, k), torch.float32, dev, stream), _new((T,), torch.int64, dev, stream))
    probs, ids, weight, mask = out
    if not isinstance(probs, torch.Tensor) or probs.dtype not in _CODE or probs.shape != (T, E) or probs.device != dev \
            or (E > 1 and probs.stride(1) != 1) or (T > 1 and probs.stride(0) < E):
        raise ValueError(f"out[0] (probs) must be a float32 or bfloat16 [{T}x{E}] tensor on {dev} with contiguous rows")
    _need(ids, "out[1] (ids)", torch.int32, (T, k), dev)
    _need(weight, "out[2] (weight)", torch.float32, (T, k), dev)
    if mask is not None:
        _need(mask, "out[3] (mask)", torch.int64, (T,), dev)
    _call("fm_moe_route", dev, stream, x.data_ptr(), gate.data_ptr(), _CODE[x.dtype], T, d, E, k, 1 if renorm else 0,
          _ptr(active), probs.data_ptr(), _CODE[probs.dtype], probs.stride(0) if T > 1 else E, ids.data_ptr(),
          weight.data_ptr(), _ptr(mask))
    return out


class ExpertCache:
    """Experts of one MoE layer held on the GPU: ``weights`` [slots][3 d f] (a slot is one expert's gate and up
    projections [f][d], then its down projection [d][f], one block), ``slot_of`` [E] int32 (-1: not held).  Both are
    plain tensors that the owner may also fill itself, in place: calls read the memory that they had at first."""

    def __init__(self, slots: int, E: int, d: int, f: int, dtype: str = "bf16", device="cuda"):
        self.slots, self.E, self.d, self.f = int(slots), int(E), int(d), int(f)
        self.dtype = _TORCH[_DTYPES[dtype]]
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        if not (1 <= self.E <= 64 and self.slots >= 1) or moe_workspace_bytes(self.d, self.f, dtype, 1, 1) == 0:
            raise ValueError(f"invalid expert cache slots={slots} E={E} d={d} f={f}")
        self._weights = torch.empty((self.slots, 3 * self.d * self.f), dtype=self.dtype, device=self.device)
        self._slot_of = torch.full((self.E,), -1, dtype=torch.int32, device=self.device)
        self.flags = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._desc = _lib.ExpertCacheDesc(self.E, self.slots, self.d, self.f, _DTYPES[dtype], self._weights.data_ptr(),
                                          self._slot_of.data_ptr())
        self.desc = C.byref(self._desc)
        self.workspace = None    # of the last call without one of its own
        self._workspaces = {}    # stream handle -> the workspace of its calls
        self._replaced = []      # workspaces that calls of more tokens outgrew

    @property
    def weights(self) -> torch.Tensor:
        return self._weights

    @weights.setter
    def weights(self, t):
        self._same(t, self._weights, "weights")

    @property
    def slot_of(self) -> torch.Tensor:
        return self._slot_of

    @slot_of.setter
    def slot_of(self, t):
        self._same(t, self._slot_of, "slot_of")

    @staticmethod
    def _same(t, own, name: str) -> None:
        if t is not own:   # (cache.weights *= 2 ends in such an assignment)
            raise AttributeError(f"{name} cannot be replaced: write into it")

    def load(self, expert: int, slot: int, gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor) -> None:
        """Put an expert (gate, up [f][d], down [d][f]) into a slot, on the current stream; an expert that the slot
        held before is no longer held."""
        if not (0 <= expert < self.E and 0 <= slot < self.slots):
            raise ValueError(f"expert {expert} or slot {slot} out of range")
        n = self.d * self.f
        for t, name, shape in ((gate, "gate", (self.f, self.d)), (up, "up", (self.f, self.d)),
                               (down, "down", (self.d, self.f))):
            if tuple(t.shape) != shape or t.dtype != self.dtype:
                raise ValueError(f"{name} must be {self.dtype} of shape {list(shape)}")
        for i, t in enumerate((gate, up, down)):
            self.weights[slot, i * n:(i + 1) * n].view(t.shape).copy_(t, non_blocking=True)
        self.slot_of.masked_fill_(self.slot_of == slot, -1)
        self.slot_of[expert] = slot

    def evict(self, expert: int) -> None:
        """The expert is no longer held (its slot may be loaded again)."""
        self.slot_of[expert] = -1

    def check(self, stream=None) -> int:
        """Synchronise the stream and return the sticky FM_FLAG_* bits of the calls that it has seen, cleared.  Calls on
        other streams must have ended: a bit that one sets in the meantime may be cleared unseen."""
        with _on(stream):
            f = int(self.flags.item())
            self.flags.zero_()
        return f

    def ensure_workspace(self, T: int, K: int, stream=None) -> "MoeWorkspace":
        """The cache's own workspace of the stream, made or enlarged for calls of T tokens of K experts each.  Each
        stream has one, in memory of its own, so that calls on different streams need no order.  One that is replaced
        stays allocated as long as the cache: a captured graph may hold its address.  Sizes are of powers of two of
        tokens, so that few are."""
        handle = self._handle(stream)
        own = self._workspaces.get(handle)
        if own is None or moe_workspace_bytes(self.d, self.f, self._name(), max(T, 1), K) > own.nbytes:
            with _on(stream):
                made = MoeWorkspace(self, max(16, 1 << (T - 1).bit_length()), K)
            if own is not None:
                self._replaced.append(own)
            own = self._workspaces[handle] = made
        self.workspace = own
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

    def _name(self) -> str:
        return "bf16" if self.dtype is torch.bfloat16 else "f32"


def moe_workspace_bytes(d: int, f: int, dtype: str = "bf16", T_max: int = 256, K: int = 8) -> int:
    return int(_lib.load().fm_moe_workspace_bytes(d, f, _DTYPES[dtype], T_max, K))


class MoeWorkspace:
    """Device scratch for moe_experts calls of up to T_max tokens of K experts each (every call rewrites what it
    reads); above 128 tokens one size, of about half a GB at most, serves all.  Calls sharing one workspace must be
    ordered; the caches of all layers of a model may share one, where each would otherwise make its own."""

    def __init__(self, cache: ExpertCache, T_max: int = 256, K: int = 8):
        self.nbytes = moe_workspace_bytes(cache.d, cache.f, cache._name(), T_max, K)
        if self.nbytes == 0:
            raise ValueError(f"invalid workspace request T_max={T_max} K={K}")
        self.buf = _aligned_bytes(self.nbytes, cache.device)


def moe_experts(cache: ExpertCache, x: torch.Tensor, ids: torch.Tensor, weight: torch.Tensor,
                residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                workspace: Optional[MoeWorkspace] = None, stream=None) -> torch.Tensor:
    """residual + the weighted products of each token's experts: x [T][d], ids [T][K] int32, weight [T][K] float32 as
    moe_route gives them -> [T][d]; T from a decode iteration's few to a prompt's thousands.  Experts that the cache
    does not hold are left out and flagged (cache.check()).  Without ``workspace`` the cache's own of the stream serves
    the call; replays of a graph that captured such a call must be ordered with each other and with the later calls on
    the stream of the capture, as with any workspace that they share."""
    dev = cache.device
    _float_rows(x, "x")
    T = x.shape[0]
    _need(x, "x", cache.dtype, (T, cache.d), dev)
    if not (isinstance(ids, torch.Tensor) and ids.dim() == 2):
        _need(ids, "ids", torch.int32, (T, None), dev)
    K = ids.shape[1]
    _need(ids, "ids", torch.int32, (T, K), dev)
    _need(weight, "weight", torch.float32, (T, K), dev)
    if residual is not None:
        _need(residual, "residual", cache.dtype, (T, cache.d), dev)
    if out is None:
        out = _new((T, cache.d), cache.dtype, dev, stream)
    else:
        _need(out, "out", cache.dtype, (T, cache.d), dev)
    ws = workspace if workspace is not None else cache.ensure_workspace(T, K, stream)
    _need(ws.buf, "workspace", torch.uint8, (ws.nbytes,), dev)
    _call("fm_moe_experts", dev, stream, cache.desc, x.data_ptr(), ids.data_ptr(), weight.data_ptr(), T, K,
          _ptr(residual), out.data_ptr(), _flags(cache.flags, dev), ws.buf.data_ptr(), ws.nbytes)
    return out

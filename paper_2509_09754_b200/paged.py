"""The paged cache: ctypes binding of its C functions, and `PagedCache`, which owns the buffers.

The functions carry the names of the C ABI in include/lava.h, which describes the arguments.  Beside
marshalling they refuse tensors that the C side cannot look into: a wrong type, shape, layout or device.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from .binding import (LAVA_BF16, LAVA_F32, EvictionPlan, LavaError, LayerDesc, _CCache, _check, _CRotary, _ptr,
                      _raw_stream, evict_scores, lava_last_error, lava_poll_status, load_library)

LAVA_ROTARY_PLAIN, LAVA_ROTARY_LINEAR, LAVA_ROTARY_BASE, LAVA_ROTARY_BANDS, LAVA_ROTARY_RAMP = 0, 1, 2, 3, 4
LAVA_DEV_PAGES_EXHAUSTED, LAVA_DEV_BAD_ROWS = 16, 32

_I32, _I64, _F32, _U8, _TWO = torch.int32, torch.int64, torch.float32, torch.uint8, (2,)
_TORCH = {LAVA_F32: torch.float32, LAVA_BF16: torch.bfloat16}


# The checks are most of a call's time on the host, so they are few and cheap: the current device is asked for once a
# call, and a tensor on the host has device -1.
_current = getattr(torch._C, "_cuda_getDevice", None)  # absent in builds without CUDA


def _device() -> int:
    try:
        return _current()
    except (TypeError, RuntimeError):  # no CUDA, or none to be had
        return -2


def _on(dev, stream):
    """The stream's handle: the current one of the device unless given."""
    return _raw_stream(dev) if stream is None else stream.cuda_stream


def _arg(dev, name, t, dtype, shape):
    """The address of a contiguous tensor of this type and shape on this device."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    raise LavaError(1, "%s must be a %s tensor of shape %s, contiguous, on the current device (got %s %s)" % (
        name, str(dtype).replace("torch.", ""), tuple(shape), str(t.dtype).replace("torch.", ""), tuple(t.shape)))


def _vectors(dev, name, t, dtype, shape):
    """Address and strides of [tokens, heads, dim] vectors whose elements are contiguous."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev:
        st, sh, one = t.stride()
        if one == 1:
            return t.data_ptr(), st, sh
    raise LavaError(1, "%s must be a %s tensor of shape %s with contiguous vectors, on the current device (got %s %s)" % (
        name, str(dtype).replace("torch.", ""), shape, str(t.dtype).replace("torch.", ""), tuple(t.shape)))


@dataclass(frozen=True)
class CacheDesc:
    """Geometry of a paged cache (lava_cache_desc of the C ABI)."""
    n_layers: int
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    max_pages: int
    n_pages: int
    dtype: int = LAVA_BF16
    page_rows: int = 64
    sm_scale: float = 0.0
    softcap: float = 0.0

    def __post_init__(self):
        c = _CCache(self.n_layers, self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype,
                    self.page_rows, self.max_pages, self.n_pages, self.sm_scale, self.softcap)
        # what every call hands over and checks against; the fields are frozen, so it holds
        object.__setattr__(self, "_c", c)
        object.__setattr__(self, "_ref", ctypes.byref(c))
        object.__setattr__(self, "_type", _TORCH.get(self.dtype))
        heads = (self.n_layers, self.batch, self.n_kv_heads)
        object.__setattr__(self, "_heads", heads)
        object.__setattr__(self, "_table", heads + (self.max_pages,))
        object.__setattr__(self, "_pool", (self.n_pages, self.page_rows, self.head_dim))
        object.__setattr__(self, "_ring", (self.n_pages,))
        object.__setattr__(self, "_queries", (self.batch, self.n_q_heads, self.head_dim))

    def __reduce__(self):  # copies and pickles make their own structure
        return type(self), tuple(getattr(self, f) for f in self.__dataclass_fields__)


@dataclass(frozen=True)
class RotaryDesc:
    """Rotary positions of one geometry (lava_rotary_desc of the C ABI)."""
    head_dim: int
    rotary_dim: int
    dtype: int = LAVA_BF16
    interleaved: bool = False
    backward: bool = False
    scale: float = 1.0

    def __post_init__(self):
        c = _CRotary(self.head_dim, self.rotary_dim, int(self.interleaved), int(self.backward), self.dtype,
                     self.scale)
        object.__setattr__(self, "_c", c)
        object.__setattr__(self, "_ref", ctypes.byref(c))
        object.__setattr__(self, "_type", _TORCH.get(self.dtype))
        object.__setattr__(self, "_half", (self.rotary_dim // 2,))

    def __reduce__(self):
        return type(self), tuple(getattr(self, f) for f in self.__dataclass_fields__)


def _status(dev, word):
    """The address of a status word: the first bytes of a workspace, or an int32 of its own."""
    if word is None:
        return None
    if word.numel() * word.element_size() < 4 or word.get_device() != dev or not word.is_contiguous():
        raise LavaError(1, "status_word must have 4 bytes on the current device")
    return word.data_ptr()


def _freqs_of(dev, rotary, freqs):
    if freqs is None and rotary.rotary_dim == 0:
        return None
    return _arg(dev, "freqs", freqs, torch.float64, rotary._half)


# ----------------------------------------------------------------------------- page tables
def lava_cache_workspace_bytes(cache: CacheDesc) -> int:
    n = int(load_library().lava_cache_workspace_bytes(cache._ref))
    if n == 0:
        raise LavaError(1, lava_last_error())
    return n


def lava_page_admit(cache: CacheDesc, first_seq, head_offsets, head_rows, page_table, free_pages, counters,
                    first_row, status_word=None, head_rows_out=None, counters_out=None, stream=None) -> None:
    """Pages for the selection of head_offsets.shape[1] new prompts; without *_out the counts are updated in place."""
    dev, (L, _, H) = _device(), cache._heads
    n_seqs = head_offsets.shape[1] if head_offsets.dim() == 3 else 0
    rows, cnt = _arg(dev, "head_rows", head_rows, _I32, cache._heads), _arg(dev, "counters", counters, _I64, _TWO)
    _check(load_library().lava_page_admit(
        cache._ref, first_seq, n_seqs, _arg(dev, "head_offsets", head_offsets, _I32, (L, n_seqs, H + 1)), rows,
        rows if head_rows_out is None else _arg(dev, "head_rows_out", head_rows_out, _I32, cache._heads),
        _arg(dev, "page_table", page_table, _I32, cache._table),
        _arg(dev, "free_pages", free_pages, _I32, cache._ring), cnt,
        cnt if counters_out is None else _arg(dev, "counters_out", counters_out, _I64, _TWO),
        _arg(dev, "first_row", first_row, _I32, (L, n_seqs, H)), _status(dev, status_word), _on(dev, stream)))


def lava_page_extend(cache: CacheDesc, add, head_rows, page_table, free_pages, counters, slots, status_word=None,
                     head_rows_out=None, counters_out=None, stream=None) -> None:
    """Pages and places for add[b] new rows of every head of sequence b (slots.shape[2] at most)."""
    dev, (L, B, H) = _device(), cache._heads
    max_add = slots.shape[2] if slots.dim() == 4 else 0
    rows, cnt = _arg(dev, "head_rows", head_rows, _I32, cache._heads), _arg(dev, "counters", counters, _I64, _TWO)
    _check(load_library().lava_page_extend(
        cache._ref, _arg(dev, "add", add, _I32, (B,)), max_add, rows,
        rows if head_rows_out is None else _arg(dev, "head_rows_out", head_rows_out, _I32, cache._heads),
        _arg(dev, "page_table", page_table, _I32, cache._table),
        _arg(dev, "free_pages", free_pages, _I32, cache._ring), cnt,
        cnt if counters_out is None else _arg(dev, "counters_out", counters_out, _I64, _TWO),
        _arg(dev, "slots", slots, _I32, (L, B, max_add, H)), _status(dev, status_word), _on(dev, stream)))


def lava_compact_kv_pages(desc: LayerDesc, cache: CacheDesc, first_seq, k, v, k_layer_stride, v_layer_stride,
                          keep_idx, head_offsets, first_row, page_table, k_pages, v_pages, stream=None) -> None:
    """lava_compact_kv_layers into the pages of a cache."""
    dev, (L, _, H) = _device(), cache._heads
    shape = (L, H, desc.total_tokens, cache.head_dim)
    for name, x in (("k", k), ("v", v)):
        if x.dtype is not cache._type or x.shape != shape or x.stride(3) != 1 or x.get_device() != dev:
            raise LavaError(1, "%s must be a %s tensor of shape %s with contiguous rows, on the current device" % (
                name, str(cache._type).replace("torch.", ""), shape))
    _check(load_library().lava_compact_kv_pages(
        ctypes.byref(desc._for_call()), cache._ref, first_seq, k.data_ptr(), v.data_ptr(), k_layer_stride,
        v_layer_stride, _arg(dev, "keep_idx", keep_idx, _I32, (L, desc.total_scores)),
        _arg(dev, "head_offsets", head_offsets, _I32, (L, desc.batch, H + 1)),
        _arg(dev, "first_row", first_row, _I32, (L, desc.batch, H)),
        _arg(dev, "page_table", page_table, _I32, cache._table),
        _arg(dev, "k_pages", k_pages, cache._type, cache._pool),
        _arg(dev, "v_pages", v_pages, cache._type, cache._pool), _on(dev, stream)))


# ----------------------------------------------------------------------------- rotary positions
def lava_rotary_freqs(rotary_dim: int, base: float = 10000.0, kind: int = LAVA_ROTARY_PLAIN, factor: float = 1.0,
                      original_length: float = 8192.0, low: float = 1.0, high: float = 4.0):
    """(frequencies as a HOST float64 tensor [rotary_dim / 2], scale of the rotated vectors)."""
    # (up to 128 is what the C side can accept: it refuses the rest before it writes)
    freqs = torch.empty(max(0, min(int(rotary_dim), 128)) // 2, dtype=torch.float64)
    scale = ctypes.c_float(1.0)
    _check(load_library().lava_rotary_freqs(kind, rotary_dim, base, factor, original_length, low, high, _ptr(freqs),
                                            ctypes.byref(scale)))
    return freqs, float(scale.value)


def lava_rotary(rotary: RotaryDesc, freqs, positions, q, k, q_out, k_out, stream=None) -> None:
    """Queries and keys [n_tokens, heads, head_dim] (any strides of tokens and heads) turned into q_out and k_out."""
    dev = _device()
    n = positions.shape[0] if positions.dim() == 1 else -1
    args = []
    for name, x, y in (("q", q, q_out), ("k", k, k_out)):
        if x is None and y is None:
            args += (None, 0, 0, 0, None, 0, 0)
            continue
        if x is None or y is None:
            raise LavaError(1, "%s and %s_out are both given or both None" % (name, name))
        heads = x.shape[1] if x.dim() == 3 else 0
        shape = (n, heads, rotary.head_dim)
        xp, st, sh = _vectors(dev, name, x, rotary._type, shape)
        yp, ot, oh = _vectors(dev, name + "_out", y, rotary._type, shape)
        args += (xp, heads, st, sh, yp, ot, oh)
    _check(load_library().lava_rotary(rotary._ref, _freqs_of(dev, rotary, freqs), n,
                                      _arg(dev, "positions", positions, _I32, (n,)), *args, _on(dev, stream)))


def lava_rotary_append(rotary: RotaryDesc, freqs, cache: CacheDesc, layer, positions, q, k, v, q_out, slots,
                       k_pages, v_pages, stream=None) -> None:
    """New tokens of layer `layer`: queries turned into q_out, keys turned and values into the rows that `slots`
    (of lava_page_extend, all layers) names.  q, k, v [batch * max_add, heads, head_dim]."""
    dev, (L, B, H) = _device(), cache._heads
    max_add = slots.shape[2] if slots.dim() == 4 else 0
    n, dt, d, Hq = B * max_add, cache._type, cache.head_dim, cache.n_q_heads
    sp = _arg(dev, "slots", slots, _I32, (L, B, max_add, H))
    if not 0 <= layer < L:
        raise LavaError(1, "layer %d is not in a cache of %d" % (layer, L))
    qp, qt, qh = _vectors(dev, "q", q, dt, (n, Hq, d))
    kp, kt, kh = _vectors(dev, "k", k, dt, (n, H, d))
    vp, vt, vh = _vectors(dev, "v", v, dt, (n, H, d))
    _check(load_library().lava_rotary_append(
        rotary._ref, _freqs_of(dev, rotary, freqs), cache._ref, n, _arg(dev, "positions", positions, _I32, (n,)),
        qp, qt, qh, _arg(dev, "q_out", q_out, dt, (n, Hq, d)), kp, kt, kh, vp, vt, vh, sp + layer * 4 * n * H,
        _arg(dev, "k_pages", k_pages, dt, cache._pool), _arg(dev, "v_pages", v_pages, dt, cache._pool),
        _on(dev, stream)))


# ----------------------------------------------------------------------------- attention
def lava_decode_attention_pages(cache: CacheDesc, first_layer, q, k_pages, v_pages, page_table, head_rows, out,
                                lse, workspace, stream=None) -> None:
    """Attention of one new token per sequence for q.shape[0] layers from first_layer on; lse may be None."""
    dev, dt, shape = _device(), cache._type, q.shape
    if len(shape) != 4 or shape[1:] != cache._queries:
        raise LavaError(1, "q must have the shape (n_layers, %d, %d, %d) (got %s)" % (*cache._queries, tuple(shape)))
    _check(load_library().lava_decode_attention_pages(
        cache._ref, first_layer, shape[0], _arg(dev, "q", q, dt, shape),
        _arg(dev, "k_pages", k_pages, dt, cache._pool), _arg(dev, "v_pages", v_pages, dt, cache._pool),
        _arg(dev, "page_table", page_table, _I32, cache._table),
        _arg(dev, "head_rows", head_rows, _I32, cache._heads), _arg(dev, "out", out, dt, shape),
        None if lse is None else _arg(dev, "lse", lse, _F32, shape[:3]),
        _arg(dev, "workspace", workspace, _U8, workspace.shape), workspace.numel(), _on(dev, stream)))


class PagedCache:
    """A paged cache and its buffers.  A prompt enters with `admit` after its selection (or with `evict`, which
    scores and selects as well); then, for every token, `extend` once and `append` and `attend` layer by layer.

        cache = PagedCache(lava.CacheDesc(n_layers=32, batch=8, n_q_heads=32, n_kv_heads=8, head_dim=128,
                                          max_pages=512, n_pages=65536))
        cache.evict(plan, q_win, k, v, first_seq=0)
        cache.extend(add)
        for layer in range(32):
            q = cache.append(rotary, freqs, layer, positions, q, k, v)
            out, lse = cache.attend(layer, q)
    """

    def __init__(self, desc: CacheDesc, device="cuda"):
        need = lava_cache_workspace_bytes(desc)  # refuses a bad geometry
        i32 = dict(dtype=torch.int32, device=device)
        self.desc = desc
        self.k_pages = torch.empty(desc._pool, dtype=desc._type, device=device)
        self.v_pages = torch.empty(desc._pool, dtype=desc._type, device=device)
        self.head_rows = torch.zeros(desc._heads, **i32)
        self.page_table = torch.full(desc._table, -1, **i32)
        self.free_pages = torch.arange(desc.n_pages, **i32)
        self.counters = torch.tensor([0, desc.n_pages], dtype=torch.int64, device=device)
        self.workspace = torch.zeros(need, dtype=torch.uint8, device=device)
        self.slots = None  # of the last extend

    def free_page_count(self) -> int:
        """Pages that are free; waits for the device."""
        taken, given = self.counters.tolist()
        return given - taken

    def poll_status(self, stream=None) -> int:
        """LAVA_DEV_* bits since the last poll; waits for the stream."""
        return lava_poll_status(self.workspace, stream)

    def admit(self, plan: EvictionPlan, k, v, first_seq: int = 0, stream=None) -> None:
        """The selection of a plan (its keep_idx and head_offsets) as sequences first_seq ... of the cache: pages, and
        the kept rows of k and v [n_layers, H_kv, total_tokens, d] in them, behind what the sequences hold."""
        d = self.desc
        first_row = torch.empty((d.n_layers, plan.desc.batch, d.n_kv_heads), dtype=torch.int32,
                                device=self.head_rows.device)
        lava_page_admit(d, first_seq, plan.head_offsets, self.head_rows, self.page_table, self.free_pages,
                        self.counters, first_row, self.workspace, stream=stream)
        lava_compact_kv_pages(plan.desc, d, first_seq, k, v, k.stride(0), v.stride(0), plan.keep_idx,
                              plan.head_offsets, first_row, self.page_table, self.k_pages, self.v_pages, stream)

    def evict(self, plan: EvictionPlan, q_win, k, v, first_seq: int = 0, mode: int = 0, stream=None) -> None:
        """evict_model with the kept rows in the pages of this cache instead of the plan's packed cache."""
        evict_scores(plan, q_win, k, v, mode, stream)
        self.admit(plan, k, v, first_seq, stream)

    def extend(self, add, max_add: int = 1, stream=None) -> torch.Tensor:
        """Room for add[b] new rows in every head of sequence b, -1 releases it; the rows' places."""
        d = self.desc
        shape = (d.n_layers, d.batch, max_add, d.n_kv_heads)
        if self.slots is None or self.slots.shape != shape:
            self.slots = torch.empty(shape, dtype=torch.int32, device=self.head_rows.device)
        lava_page_extend(d, add, self.head_rows, self.page_table, self.free_pages, self.counters, self.slots,
                         self.workspace, stream=stream)
        return self.slots

    def append(self, rotary: RotaryDesc, freqs, layer: int, positions, q, k, v, q_out=None, stream=None):
        """Turned queries of the new tokens; their turned keys and their values go where `extend` made room."""
        if self.slots is None:
            raise LavaError(1, "append without extend")
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lava_rotary_append(rotary, freqs, self.desc, layer, positions, q, k, v, q_out, self.slots, self.k_pages,
                           self.v_pages, stream)
        return q_out

    def attend(self, first_layer: int, q, out=None, lse=None, stream=None):
        """(out, lse) of q [batch, H_q, d] or [n_layers, batch, H_q, d] over the rows that the heads hold."""
        one = q.dim() == 3
        q = q.unsqueeze(0) if one else q
        out = torch.empty_like(q) if out is None else out.view(q.shape)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if lse is None else lse.view(q.shape[:3])
        lava_decode_attention_pages(self.desc, first_layer, q, self.k_pages, self.v_pages, self.page_table,
                                    self.head_rows, out, lse, self.workspace, stream)
        return (out[0], lse[0]) if one else (out, lse)

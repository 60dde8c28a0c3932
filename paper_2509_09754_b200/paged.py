"""The paged cache: binding of its C functions, and `PagedCache`, which owns the buffers.

The functions carry the names of the C ABI in include/lava.h, which describes the arguments.  They go through a small
native module (csrc/paged_calls.cpp) that looks into the tensors and refuses a wrong type, shape, layout or device with
a LavaError before the C function sees them.  What they write carries no gradient.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
from dataclasses import dataclass

import torch

from .binding import (LAVA_BF16, LAVA_F32, EvictionPlan, LavaError, LayerDesc, _CCache, _check, _CRotary, _ptr,
                      evict_scores, lava_last_error, lava_poll_status, library_path, load_library)

LAVA_ROTARY_PLAIN, LAVA_ROTARY_LINEAR, LAVA_ROTARY_BASE, LAVA_ROTARY_BANDS, LAVA_ROTARY_RAMP = 0, 1, 2, 3, 4
LAVA_DEV_PAGES_EXHAUSTED, LAVA_DEV_BAD_ROWS = 16, 32

_TORCH = {LAVA_F32: torch.float32, LAVA_BF16: torch.bfloat16}
_CALLS = None


def load_paged_calls():
    """Load the native module; raises if it has not been built, or for another torch (there is no fallback path)."""
    global _CALLS
    if _CALLS is None:
        load_library()
        path = os.path.join(os.path.dirname(library_path()), "_paged_calls.so")
        if not os.path.exists(path):
            raise RuntimeError("%s is missing: build it with `python -m paper_2509_09754_b200.build`" % path)
        loader = importlib.machinery.ExtensionFileLoader("_paged_calls", path)
        try:
            module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_paged_calls", loader))
            loader.exec_module(module)
            built = "torch " + module.torch_version
        except (ImportError, AttributeError) as e:
            built = "another torch (%s)" % e
        if built != "torch %s" % torch.__version__:
            raise RuntimeError("%s was built for %s, this is torch %s: build it again with "
                               "`python -m paper_2509_09754_b200.build --force`" % (path, built, torch.__version__))
        module.set_error(LavaError)
        _CALLS = module
    return _CALLS


def _handle(stream):
    return None if stream is None else stream.cuda_stream


def _empty(shape, dtype, device, stream):
    """Memory for work on this stream: torch hands it out, and takes it back, in the order of the stream's work."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


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
        # what every call hands over; the fields are frozen, so it holds
        object.__setattr__(self, "_c", c)
        object.__setattr__(self, "_ref", ctypes.byref(c))
        object.__setattr__(self, "_at", ctypes.addressof(c))

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
        object.__setattr__(self, "_at", ctypes.addressof(c))

    def __reduce__(self):
        return type(self), tuple(getattr(self, f) for f in self.__dataclass_fields__)


# ----------------------------------------------------------------------------- page tables
def lava_cache_workspace_bytes(cache: CacheDesc) -> int:
    n = int(load_library().lava_cache_workspace_bytes(cache._ref))
    if n == 0:
        raise LavaError(1, lava_last_error())
    return n


def lava_page_admit(cache: CacheDesc, first_seq, head_offsets, head_rows, page_table, free_pages, counters,
                    first_row, status_word=None, head_rows_out=None, counters_out=None, stream=None) -> None:
    """Pages for the selection of head_offsets.shape[1] new prompts; without *_out the counts are updated in place."""
    (_CALLS or load_paged_calls()).page_admit(
        cache._at, first_seq, head_offsets, head_rows, page_table, free_pages, counters, first_row, status_word,
        head_rows_out, counters_out, _handle(stream))


def lava_page_extend(cache: CacheDesc, add, head_rows, page_table, free_pages, counters, slots, status_word=None,
                     head_rows_out=None, counters_out=None, stream=None) -> None:
    """Pages and places for add[b] new rows of every head of sequence b (slots.shape[2] at most)."""
    (_CALLS or load_paged_calls()).page_extend(
        cache._at, add, head_rows, page_table, free_pages, counters, slots, status_word, head_rows_out, counters_out,
        _handle(stream))


def lava_compact_kv_pages(desc: LayerDesc, cache: CacheDesc, first_seq, k, v, k_layer_stride, v_layer_stride,
                          keep_idx, head_offsets, first_row, page_table, k_pages, v_pages, stream=None) -> None:
    """lava_compact_kv_layers into the pages of a cache."""
    layer = desc._for_call()
    (_CALLS or load_paged_calls()).compact_kv_pages(
        ctypes.addressof(layer), cache._at, first_seq, k, v, k_layer_stride, v_layer_stride, keep_idx, head_offsets,
        first_row, page_table, k_pages, v_pages, _handle(stream))


def lava_check_compact_kv_pages(desc: LayerDesc, cache: CacheDesc, first_seq, k, v, k_layer_stride, v_layer_stride,
                                keep_idx, head_offsets, first_row, page_table, k_pages, v_pages) -> None:
    """Raises what lava_compact_kv_pages would, and does nothing."""
    layer = desc._for_call()
    (_CALLS or load_paged_calls()).check_compact_kv_pages(
        ctypes.addressof(layer), cache._at, first_seq, k, v, k_layer_stride, v_layer_stride, keep_idx, head_offsets,
        first_row, page_table, k_pages, v_pages, None)


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
    """Queries and keys [n_tokens, heads, head_dim] (any strides of tokens and heads) turned into q_out and k_out.
    Autograd does not follow the call, so tensors that require a gradient are refused where it records: a
    torch.autograd.Function turns in its forward, and the gradients with RotaryDesc(backward=True) in its backward."""
    (_CALLS or load_paged_calls()).rotary(rotary._at, freqs, positions, q, q_out, k, k_out, _handle(stream))


def lava_rotary_append(rotary: RotaryDesc, freqs, cache: CacheDesc, layer, positions, q, k, v, q_out, slots,
                       k_pages, v_pages, stream=None) -> None:
    """New tokens of layer `layer`: queries turned into q_out, keys turned and values into the rows that `slots`
    (of lava_page_extend, all layers) names.  q, k, v [batch * max_add, heads, head_dim]."""
    (_CALLS or load_paged_calls()).rotary_append(
        rotary._at, freqs, cache._at, layer, slots, positions, q, k, v, q_out, k_pages, v_pages, _handle(stream))


# ----------------------------------------------------------------------------- attention
def lava_decode_attention_pages(cache: CacheDesc, first_layer, q, k_pages, v_pages, page_table, head_rows, out,
                                lse, workspace, stream=None) -> None:
    """Attention of one new token per sequence for q.shape[0] layers from first_layer on; lse may be None."""
    (_CALLS or load_paged_calls()).decode_attention_pages(
        cache._at, first_layer, q, k_pages, v_pages, page_table, head_rows, out, lse, workspace, _handle(stream))


class PagedCache:
    """A paged cache and its buffers.  A prompt enters with `admit` after its selection (or with `evict`, which
    scores and selects as well); then, for every token, `extend` once and `append` and `attend` layer by layer.
    Its calls share tables and a workspace: they follow one another, on one stream or on streams that wait.

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
        heads = (desc.n_layers, desc.batch, desc.n_kv_heads)
        pool = (desc.n_pages, desc.page_rows, desc.head_dim)
        self.k_pages = torch.empty(pool, dtype=_TORCH[desc.dtype], device=device)
        self.v_pages = torch.empty(pool, dtype=_TORCH[desc.dtype], device=device)
        self.head_rows = torch.zeros(heads, **i32)
        self.page_table = torch.full(heads + (desc.max_pages,), -1, **i32)
        self.free_pages = torch.arange(desc.n_pages, **i32)
        self.workspace = torch.zeros(need, dtype=torch.uint8, device=device)
        # (last: this copy from the host waits for what the stream had before it, so any stream may use the cache now)
        self.counters = torch.tensor([0, desc.n_pages], dtype=torch.int64, device=device)
        self.slots = None  # of the last extend
        # by number of rows: a captured extend keeps their address, and a stream may be behind the one that calls next, so
        # none is given up while the cache lives
        self._slots = {}

    def free_page_count(self) -> int:
        """Pages that are free; waits for the device, whatever streams the calls before were on."""
        if self.counters.is_cuda:
            torch.cuda.synchronize(self.counters.device)
        taken, given = self.counters.tolist()
        return given - taken

    def poll_status(self, stream=None) -> int:
        """LAVA_DEV_* bits since the last poll; waits for the stream."""
        return lava_poll_status(self.workspace, stream)

    def admit(self, plan: EvictionPlan, k, v, first_seq: int = 0, stream=None) -> None:
        """The selection of a plan (its keep_idx and head_offsets, after evict_scores or evict_model) as sequences
        first_seq ... of the cache: pages, and the kept rows of k and v [n_layers, H_kv, total_tokens, d] in them, behind
        what the sequences hold.  Of a batch with a sequence shorter than the window nothing is selected (the plan's status
        word says so), and nothing enters."""
        d = self.desc
        first_row = _empty((d.n_layers, plan.desc.batch, d.n_kv_heads), torch.int32, self.head_rows.device, stream)
        rows = (plan.desc, d, first_seq, k, v, k.stride(0), v.stride(0), plan.keep_idx, plan.head_offsets, first_row,
                self.page_table, self.k_pages, self.v_pages)
        lava_check_compact_kv_pages(*rows)  # (a refusal after the next call would leave pages without their rows)
        lava_page_admit(d, first_seq, plan.head_offsets, self.head_rows, self.page_table, self.free_pages,
                        self.counters, first_row, self.workspace, stream=stream)
        lava_compact_kv_pages(*rows, stream)

    def evict(self, plan: EvictionPlan, q_win, k, v, first_seq: int = 0, mode: int = 0, stream=None) -> None:
        """evict_model with the kept rows in the pages of this cache instead of the plan's packed cache."""
        evict_scores(plan, q_win, k, v, mode, stream)
        self.admit(plan, k, v, first_seq, stream)

    def extend(self, add, max_add: int = 1, stream=None) -> torch.Tensor:
        """Room for add[b] new rows in every head of sequence b, -1 releases it; the rows' places (in memory of the
        cache's own, which `append` reads and the next call with the same max_add writes)."""
        d = self.desc
        slots = self._slots.get(max_add)
        if slots is None:
            slots = _empty((d.n_layers, d.batch, max_add, d.n_kv_heads), torch.int32, self.head_rows.device, stream)
        lava_page_extend(d, add, self.head_rows, self.page_table, self.free_pages, self.counters, slots,
                         self.workspace, stream=stream)
        self.slots = self._slots[max_add] = slots
        return slots

    def append(self, rotary: RotaryDesc, freqs, layer: int, positions, q, k, v, q_out=None, stream=None):
        """Turned queries of the new tokens; their turned keys and their values go where `extend` made room."""
        if self.slots is None:
            raise LavaError(1, "append without extend")
        if q_out is None:
            q_out = _empty(q.shape, q.dtype, q.device, stream)
        lava_rotary_append(rotary, freqs, self.desc, layer, positions, q, k, v, q_out, self.slots, self.k_pages,
                           self.v_pages, stream)
        return q_out

    def attend(self, first_layer: int, q, out=None, lse=None, stream=None):
        """(out, lse) of q [batch, H_q, d] or [n_layers, batch, H_q, d] over all the rows that the heads hold: one query
        per sequence, its last token's where `extend` made room for several."""
        one = q.dim() == 3
        q = q.unsqueeze(0) if one else q
        out = _empty(q.shape, q.dtype, q.device, stream) if out is None else out.view(q.shape)
        lse = _empty(q.shape[:3], torch.float32, q.device, stream) if lse is None else lse.view(q.shape[:3])
        lava_decode_attention_pages(self.desc, first_layer, q, self.k_pages, self.v_pages, self.page_table,
                                    self.head_rows, out, lse, self.workspace, stream)
        return (out[0], lse[0]) if one else (out, lse)

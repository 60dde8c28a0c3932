"""Paged cache and rotary positions on the host: refusals before any launch, and the frequencies."""
import copy
import ctypes
import math
import pickle

import numpy as np
import pytest
import torch

import paper_2509_09754_b200 as lava
from oracle import paged_oracle as PO
from paper_2509_09754_b200 import binding
from paper_2509_09754_b200 import paged as P

GOOD = dict(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64, max_pages=4, n_pages=64, page_rows=16)


def _cache(**kw):
    return lava.CacheDesc(**dict(GOOD, **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(n_layers=0), 1), (dict(batch=0), 1), (dict(n_q_heads=7), 1), (dict(n_kv_heads=0), 1), (dict(head_dim=96), 2),
    (dict(n_q_heads=258, n_kv_heads=129), 2), (dict(dtype=2), 1), (dict(page_rows=8), 2), (dict(page_rows=48), 2),
    (dict(page_rows=512), 2), (dict(max_pages=0), 1), (dict(n_pages=0), 1), (dict(n_pages=1 << 27), 2),
    (dict(max_pages=1 << 27), 2), (dict(sm_scale=-1.0), 1), (dict(sm_scale=float("nan")), 1),
    (dict(softcap=float("inf")), 1), (dict(softcap=-2.0), 1), (dict(n_layers=1 << 20, batch=1 << 10), 2),
])
def test_bad_caches_are_refused(kw, status):
    lib = lava.load_library()
    c = _cache(**kw)
    assert lib.lava_cache_workspace_bytes(c._ref) == 0
    with pytest.raises(lava.LavaError):
        lava.lava_cache_workspace_bytes(c)
    p = 256
    assert lib.lava_page_extend(c._ref, p, 1, p, p, p, p, p, p, p, None, None) == status
    assert lib.lava_page_admit(c._ref, 0, 1, p, p, p, p, p, p, p, p, None, None) == status
    assert lib.lava_decode_attention_pages(c._ref, 0, 1, p, p, p, p, p, p, None, p, 1 << 40, None) == status


def test_bad_arguments_of_page_tables_are_refused():
    lib = lava.load_library()
    c, p = _cache(), 256
    good = [p, 1, p, p, p, p, p, p, p]
    for i in (0, 2, 3, 4, 5, 6, 7, 8):
        bad = list(good)
        bad[i] = None
        assert lib.lava_page_extend(c._ref, *bad, None, None) == 1
    assert lib.lava_page_extend(c._ref, p, 0, p, p, p, p, p, p, p, None, None) == 1
    for first, n in ((-1, 1), (0, 0), (0, 4), (3, 1), (2, 2), (2147483647, 2)):
        assert lib.lava_page_admit(c._ref, first, n, p, p, p, p, p, p, p, p, None, None) == 1
    assert "cache of 3" in lava.lava_last_error()
    for i in range(8):
        ptrs = [p] * 8
        ptrs[i] = None
        assert lib.lava_page_admit(c._ref, 0, 1, *ptrs, None, None) == 1


def test_a_status_word_that_is_not_aligned_is_refused():
    """(It may be a view of a buffer of bytes.)"""
    lib = lava.load_library()
    c, p = _cache(), 256
    for off in (1, 2, 3):
        assert lib.lava_page_extend(c._ref, p, 1, p, p, p, p, p, p, p, p + off, None) == 1
        assert lib.lava_page_admit(c._ref, 0, 1, p, p, p, p, p, p, p, p, p + off, None) == 1
        assert "aligned" in lava.lava_last_error()


def test_outputs_of_the_attention_that_overlap_its_queries_are_refused():
    lib = lava.load_library()
    c, p, q = _cache(), 256, 1 << 20
    need, size = lava.lava_cache_workspace_bytes(c), 2 * 3 * 8 * 64 * 2  # of 2 layers, 3 sequences, 8 heads
    for out in (q, q + 16, q - 16, q + size - 16, q - size + 16):
        assert lib.lava_decode_attention_pages(c._ref, 0, 2, q, p, p, p, p, out, None, p, need, None) == 1
        assert "overlaps" in lava.lava_last_error()


def _layer_desc(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, window=16, total_tokens=512, k_stride_head=512 * 64,
                k_stride_tok=64, v_stride_head=512 * 64, v_stride_tok=64)
    base.update(kw)
    return lava.LayerDesc(**base)


def test_bad_arguments_of_the_compaction_are_refused():
    lib = lava.load_library()
    c, p = _cache(), 256

    def call(desc, cache, first=0, ptrs=(p,) * 8, strides=(0, 0)):
        k, v, keep, hoff, first_row, table, kp, vp = ptrs
        return lib.lava_compact_kv_pages(ctypes.byref(desc.to_c()), cache._ref, first, k, v, *strides, keep, hoff,
                                         first_row, table, kp, vp, None)

    assert call(_layer_desc(head_dim=96), c) == 2
    assert call(_layer_desc(n_kv_heads=4), c) == 1
    assert call(_layer_desc(dtype=lava.LAVA_F32), c) == 1
    assert call(_layer_desc(), _cache(head_dim=128)) == 1
    assert call(_layer_desc(), c, first=3) == 1
    assert call(_layer_desc(), c, first=-1) == 1
    assert call(_layer_desc(), c, strides=(4, 0)) == 1
    assert call(_layer_desc(), c, strides=(0, -8)) == 1
    for i in range(8):
        ptrs = [p] * 8
        ptrs[i] = None
        assert call(_layer_desc(), c, ptrs=ptrs) == 1
    for i in (0, 1, 6, 7):
        ptrs = [p] * 8
        ptrs[i] = p + 8
        assert call(_layer_desc(), c, ptrs=ptrs) == 1


def test_bad_arguments_of_the_attention_are_refused():
    lib = lava.load_library()
    c, p = _cache(), 256
    need = lava.lava_cache_workspace_bytes(c)
    args = [p] * 6
    assert lib.lava_decode_attention_pages(c._ref, 0, 0, *args, None, p, need, None) == 1
    assert lib.lava_decode_attention_pages(c._ref, 1, 2, *args, None, p, need, None) == 1
    assert lib.lava_decode_attention_pages(c._ref, -1, 1, *args, None, p, need, None) == 1
    assert lib.lava_decode_attention_pages(c._ref, 0, 2, *args, None, None, need, None) == 3
    assert lib.lava_decode_attention_pages(c._ref, 0, 2, *args, None, p, need - 1, None) == 3
    assert lib.lava_decode_attention_pages(c._ref, 0, 2, *args, None, p + 4, need, None) == 1
    for i in range(6):
        bad = list(args)
        bad[i] = None
        assert lib.lava_decode_attention_pages(c._ref, 0, 2, *bad, None, p, need, None) == 1
    for i in (0, 1, 2, 5):
        bad = list(args)
        bad[i] = p + 8
        assert lib.lava_decode_attention_pages(c._ref, 0, 2, *bad, None, p, need, None) == 1


def _rotary(lib, desc, n=4, q=(1 << 20, 8, 512, 64, 1 << 21, 512, 64), k=(None, 0, 0, 0, None, 0, 0), freqs=256,
            positions=256):
    return lib.lava_rotary(desc._ref, freqs, n, positions, *q, *k, None)


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), 2), (dict(rotary_dim=24), 2), (dict(rotary_dim=80), 1), (dict(rotary_dim=-16), 1),
    (dict(dtype=5), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(interleaved=2), 1),
    (dict(backward=-1), 1),
])
def test_bad_rotary_geometries_are_refused(kw, status):
    lib = lava.load_library()
    desc = lava.RotaryDesc(**dict(dict(head_dim=64, rotary_dim=64), **kw))
    assert _rotary(lib, desc) == status
    if kw.get("dtype", 1) != 5:
        assert lib.lava_rotary_append(desc._ref, 256, _cache()._ref, 3, 256, 256, 512, 64, 256, 256, 512, 64, 256, 512,
                                      64, 256, 256, 256, None) == status


def test_bad_rotary_arguments_are_refused():
    lib = lava.load_library()
    desc = lava.RotaryDesc(head_dim=64, rotary_dim=64)
    a, b = 1 << 20, 1 << 21
    assert _rotary(lib, desc, n=-1) == 1
    assert _rotary(lib, desc, freqs=None) == 1
    assert _rotary(lib, desc, positions=None) == 1
    assert _rotary(lib, desc, q=(None, 0, 0, 0, None, 0, 0)) == 1                  # nothing to do
    assert _rotary(lib, desc, q=(a, 8, 512, 64, None, 512, 64)) == 1               # one of a pair
    assert _rotary(lib, desc, q=(a + 8, 8, 512, 64, b, 512, 64)) == 1              # alignment
    assert _rotary(lib, desc, q=(a, 8, 512, 64, b + 4, 512, 64)) == 1
    assert _rotary(lib, desc, q=(a, 0, 512, 64, b, 512, 64)) == 1                  # heads
    assert _rotary(lib, desc, q=(a, 8, 516, 64, b, 512, 64)) == 1                  # strides
    assert _rotary(lib, desc, q=(a, 8, -512, 64, b, 512, 64)) == 1
    assert _rotary(lib, desc, q=(a, 8, 512, 64, b, 512, 32)) == 1                  # output vectors overlap
    assert _rotary(lib, desc, q=(a, 8, 512, 64, b, 0, 64)) == 1
    assert _rotary(lib, desc, q=(a, 8, 512, 64, b, 256, 64)) == 1
    assert _rotary(lib, desc, q=(a, 8, 0, 0, a, 512, 64)) == 1                     # over its own broadcast input
    assert _rotary(lib, desc, q=(a, 8, 512, 64, a + 128, 512, 64)) == 1            # partly over its input
    assert _rotary(lib, desc, q=(a, 8, 512, 64, a, 64, 256)) == 1                  # in place in another order
    assert _rotary(lib, desc, n=0) == 0                                            # no tokens: nothing is launched
    cache = _cache()

    def append(cache=cache, desc=desc, n=3, slots=256, q=(a, 512, 64, b), k=(a, 128, 64), v=(a, 128, 64), kp=b, vp=b):
        return lib.lava_rotary_append(desc._ref, 256, cache._ref, n, 256, *q, *k, *v, slots, kp, vp, None)

    assert append(cache=_cache(head_dim=128)) == 1
    assert append(cache=_cache(dtype=lava.LAVA_F32)) == 1
    assert append(slots=None) == 1
    assert append(kp=None) == 1
    assert append(vp=b + 8) == 1
    assert append(k=(a, 4, 64)) == 1
    assert append(q=(a, 512, 64, a + 64)) == 1
    assert append(n=0) == 0


def test_bad_frequencies_are_refused():
    for kw in (dict(rotary_dim=24), dict(rotary_dim=0), dict(rotary_dim=256), dict(rotary_dim=-16), dict(kind=5),
               dict(kind=-1), dict(base=1.0), dict(base=float("nan")), dict(kind=1, factor=0.5),
               dict(kind=2, factor=float("inf")), dict(kind=3, factor=8.0, original_length=0.0),
               dict(kind=3, factor=8.0, low=4.0, high=1.0), dict(kind=4, factor=8.0, low=0.0, high=32.0)):
        with pytest.raises(lava.LavaError):
            lava.lava_rotary_freqs(**dict(dict(rotary_dim=64), **kw))


@pytest.mark.parametrize("r", [16, 48, 64, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies_follow_their_formulas(r, base):
    i = np.arange(r // 2)
    plain = base ** (-2.0 * i / r)
    tol = dict(rtol=1e-14, atol=0)
    f, s = lava.lava_rotary_freqs(r, base)
    assert s == 1.0 and f.dtype == torch.float64 and np.allclose(f, plain, **tol)
    f, s = lava.lava_rotary_freqs(r, base, lava.LAVA_ROTARY_LINEAR, factor=4.0)
    assert s == 1.0 and np.allclose(f, plain / 4, **tol)
    f, s = lava.lava_rotary_freqs(r, base, lava.LAVA_ROTARY_BASE, factor=4.0)
    # the slowest pair turns `factor` times slower, the fastest as before
    assert s == 1.0 and np.allclose(f[-1], plain[-1] / 4, rtol=1e-12) and f[0] == 1.0
    f, s = lava.lava_rotary_freqs(r, base, lava.LAVA_ROTARY_BANDS, factor=8.0, original_length=8192.0, low=1.0, high=4.0)
    wave = 2 * math.pi / plain
    for x, p, w in zip(f.tolist(), plain, wave):
        if w < 8192.0 / 4.0:
            want = p
        elif w > 8192.0:
            want = p / 8.0
        else:
            share = (8192.0 / w - 1.0) / 3.0
            want = (1 - share) * p / 8.0 + share * p
        assert abs(x - want) <= 1e-13 * want
    f, s = lava.lava_rotary_freqs(r, base, lava.LAVA_ROTARY_RAMP, factor=8.0, original_length=4096.0, low=1.0, high=32.0)
    assert abs(s - (0.1 * math.log(8.0) + 1.0)) < 1e-6
    turns = 4096.0 * plain / (2 * math.pi)
    lo, hi = (r * math.log(4096.0 / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (32.0, 1.0))
    ratio = plain / f.numpy()
    assert np.all(ratio >= 1 - 1e-12) and np.all(ratio <= 8 + 1e-12) and np.all(np.diff(ratio) >= -1e-12)
    assert np.allclose(ratio[i <= math.floor(lo)], 1.0) and np.allclose(ratio[i >= math.ceil(hi)], 8.0)
    assert np.all(turns[i <= math.floor(lo)] >= 32.0 * (1 - 1e-9))


def test_descriptors_are_frozen_and_can_be_copied():
    c = _cache(softcap=30.0)
    r = lava.RotaryDesc(head_dim=64, rotary_dim=32, interleaved=True)
    for x in (c, r):
        with pytest.raises(AttributeError):
            x.head_dim = 128
        for y in (copy.copy(x), copy.deepcopy(x), pickle.loads(pickle.dumps(x))):
            assert y == x and y._c is not x._c and bytes(y._c) == bytes(x._c)
    assert ctypes.sizeof(binding._CCache) == 48 and ctypes.sizeof(binding._CRotary) == 24


def test_tensors_that_do_not_fit_are_refused_before_the_library_sees_them():
    c = _cache()
    L, B, H = 2, 3, 2
    i32 = torch.int32
    rows, table = torch.zeros((L, B, H), dtype=i32), torch.zeros((L, B, H, 4), dtype=i32)
    free, counters = torch.arange(64, dtype=i32), torch.tensor([0, 64])
    add, slots = torch.ones(B, dtype=i32), torch.empty((L, B, 1, H), dtype=i32)

    def refused(f, *a):
        with pytest.raises(lava.LavaError) as e:
            f(*a)
        assert e.value.status == 1

    good = dict(add=add, rows=rows, table=table, free=free, counters=counters, slots=slots)
    wrong = dict(add=[torch.ones(2, dtype=i32), torch.ones(B)], rows=[rows[0], rows.long(), rows.transpose(0, 2)],
                 table=[table[..., :3]], free=[free[:-1]], counters=[counters.int()], slots=[slots[:, :, 0], slots[:1]])
    for name, xs in wrong.items():
        for x in xs:
            refused(lava.lava_page_extend, c, *dict(good, **{name: x}).values())
    refused(lava.lava_page_extend, c, *good.values())            # on the host
    refused(lava.lava_page_admit, c, 0, torch.zeros((L, 1, H), dtype=i32), rows, table, free, counters,
            torch.zeros((L, 1, H), dtype=i32))
    pool = torch.zeros((64, 16, 64), dtype=torch.bfloat16)
    q = torch.zeros((1, B, 8, 64), dtype=torch.bfloat16)
    ws = torch.zeros(lava.lava_cache_workspace_bytes(c), dtype=torch.uint8)
    for x in (q[0], q.float(), q[..., :32], q[:, :2]):
        refused(lava.lava_decode_attention_pages, c, 0, x, pool, pool, table, rows, torch.empty_like(x), None, ws)
    refused(lava.lava_decode_attention_pages, c, 0, q, pool, pool, table, rows, q.clone(), None, ws)
    rot, f = lava.RotaryDesc(head_dim=64, rotary_dim=64), torch.zeros(32, dtype=torch.float64)
    pos = torch.zeros(3, dtype=i32)
    x = torch.zeros((3, 8, 64), dtype=torch.bfloat16)
    refused(lava.lava_rotary, rot, f, pos, x, None, None, None)
    refused(lava.lava_rotary, rot, f, pos, x[:2], None, x[:2], None)
    refused(lava.lava_rotary, rot, f, pos, x, None, x.transpose(1, 2), None)
    refused(lava.lava_rotary, rot, f.float(), pos, x, None, x, None)
    refused(lava.lava_rotary_append, rot, f, c, 2, pos, x, x[:, :2], x[:, :2], x.clone(), slots, pool, pool)


def test_arguments_of_another_kind_are_refused():
    """What is no tensor, no number in range or no stream is an exception, whatever comes after it."""
    c = _cache()
    rot = lava.RotaryDesc(head_dim=64, rotary_dim=64)
    L, B, H = 2, 3, 2
    table = torch.zeros((L, B, H, 4), dtype=torch.int32)
    rows = torch.zeros((L, B, H), dtype=torch.int32)
    pool = torch.zeros((64, 16, 64), dtype=torch.bfloat16)
    q = torch.zeros((1, B, 8, 64), dtype=torch.bfloat16)
    ws = torch.zeros(lava.lava_cache_workspace_bytes(c), dtype=torch.uint8)
    for x in (None, 7, "q", [1.0], object()):
        with pytest.raises(lava.LavaError) as e:
            lava.lava_decode_attention_pages(c, 0, x, pool, pool, table, rows, q, None, ws)
        assert e.value.status == 1 and "q must be a tensor" in str(e.value)
        with pytest.raises(lava.LavaError):
            lava.lava_rotary(rot, x, None, None, None, None, None)
        with pytest.raises(lava.LavaError):
            lava.lava_page_extend(c, x, rows, table, x, x, x)
    for n in (1 << 31, -(1 << 31) - 1, 1 << 63, -(1 << 70)):
        with pytest.raises(lava.LavaError) as e:
            lava.lava_decode_attention_pages(c, n, q, pool, pool, table, rows, q, None, ws)
        assert "first_layer is out of range" in str(e.value)
    with pytest.raises(TypeError):
        lava.lava_decode_attention_pages(c, 0.5, q, pool, pool, table, rows, q, None, ws)
    with pytest.raises(TypeError):
        P.load_paged_calls().rotary(1, 2, 3)
    with pytest.raises(lava.LavaError):
        P.load_paged_calls().rotary(*[0] * 8)          # a descriptor that is NULL
    with pytest.raises(lava.LavaError):                # a tensor without memory
        lava.lava_decode_attention_pages(c, 0, q.to("meta"), pool, pool, table, rows, q, None, ws)


def test_a_missing_module_of_calls_is_an_error(monkeypatch, tmp_path):
    lib = tmp_path / "liblava.so"
    monkeypatch.setattr(P, "library_path", lambda: str(lib))
    monkeypatch.setattr(P, "_CALLS", None)
    with pytest.raises(RuntimeError, match="_paged_calls.so is missing"):
        P.load_paged_calls()


def test_oracle_tables():
    t = PO.Tables(2, 16, 3, [5, 3, 9, 1])
    assert t.change([17, 1]) == [[80 + r for r in range(16)] + [48], [144]]
    assert t.pages == [[5, 3], [9]] and t.free == [1]
    assert t.change([0, 32]) is None and t.rows == [17, 1]      # two pages are wanted, one is free
    assert t.change([None, 2]) == [[], [145, 146]] and t.free == [1, 5, 3]
    assert t.change([0, 46]) is None                            # 49 rows, the table holds 48
    assert t.change([0, 45])[1][-1] == 5 * 16 + 15


def test_oracle_rotation_undoes_itself_and_keeps_lengths():
    g = np.random.default_rng(0)
    x = g.standard_normal((5, 3, 64))
    f, _ = lava.lava_rotary_freqs(32)
    pos = np.array([0, 1, 77, 131071, 2000000])
    for inter in (False, True):
        y = PO.rotate(x, pos, f.numpy(), inter)
        assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
        assert np.allclose(PO.rotate(y, pos, f.numpy(), inter, backward=True), x)
        assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
        # the product of two turned vectors depends on the distance of their positions alone
        a, b = PO.rotate(x[:1], [10], f.numpy(), inter), PO.rotate(x[1:2], [3], f.numpy(), inter)
        c, d = PO.rotate(x[:1], [110], f.numpy(), inter), PO.rotate(x[1:2], [103], f.numpy(), inter)
        assert np.allclose((a * b).sum(-1), (c * d).sum(-1))

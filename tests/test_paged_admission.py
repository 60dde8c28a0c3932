"""An admission that is refused leaves the cache as it was: no pages are taken for rows that will not come."""
import ctypes

import pytest
import torch

import paper_2509_09754_b200 as lava
from paper_2509_09754_b200 import paged as P


def _plan(device, H=2, d=64, w=16, n=200, L=2):
    k = torch.randn((L, H, n, d)).bfloat16().to(device)
    desc = lava.LayerDesc.for_tensors(torch.empty((1, 4 * H, w, d)), k[0], k[0], w, max_seqlen=n)
    return lava.EvictionPlan.create(desc, L, [L * H * 64], [n], device=device), k


def _bad(k):
    wide = torch.zeros((*k.shape[:3], 2 * k.shape[3]), dtype=k.dtype, device=k.device)[..., : k.shape[3]]
    return [k.float(), k[:, :, :-1], k[:1], k.transpose(1, 2), wide, k.cpu() if k.is_cuda else k.to("meta")]


def test_nothing_is_admitted_when_the_compaction_would_be_refused(monkeypatch):
    """On the CPU, where every compaction is refused: the page tables' call must not come first."""
    plan, k = _plan("cpu")
    cache = lava.PagedCache(lava.CacheDesc(n_layers=2, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, max_pages=4,
                                           n_pages=64), device="cpu")
    calls = []
    monkeypatch.setattr(P, "lava_page_admit", lambda *a, **kw: calls.append(a))
    with pytest.raises(lava.LavaError):
        cache.admit(plan, k, k)
    assert not calls


def test_the_check_refuses_what_the_compaction_refuses():
    lib = lava.load_library()
    c = lava.CacheDesc(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64, max_pages=4, n_pages=64, page_rows=16)
    layer = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, window=16, total_tokens=512, k_stride_head=512 * 64,
                 k_stride_tok=64, v_stride_head=512 * 64, v_stride_tok=64)

    def both(cache=c, first=0, ptrs=(256,) * 8, strides=(0, 0), **kw):
        k, v, keep, hoff, first_row, table, kp, vp = ptrs
        args = (ctypes.byref(lava.LayerDesc(**dict(layer, **kw)).to_c()), cache._ref, first, k, v, *strides, keep, hoff,
                first_row, table, kp, vp)
        status = lib.lava_check_compact_kv_pages(*args)
        assert status == 0 or lib.lava_compact_kv_pages(*args, None) == status
        return status

    assert both() == 0                                                       # nothing is launched or read
    assert both(head_dim=96) == 2 and both(n_kv_heads=4) == 1 and both(dtype=lava.LAVA_F32) == 1
    assert both(first=3) == 1 and both(first=-1) == 1 and both(strides=(4, 0)) == 1 and both(strides=(0, -8)) == 1
    for i in range(8):
        assert both(ptrs=[None if j == i else 256 for j in range(8)]) == 1
    for i in (0, 1, 6, 7):
        assert both(ptrs=[264 if j == i else 256 for j in range(8)]) == 1


@pytest.mark.gpu
def test_refused_admissions_leave_the_cache_as_it_was():
    plan, k = _plan("cuda")
    q = torch.randn((2, 1, 8, 16, 64), device="cuda").bfloat16()
    cache = lava.PagedCache(lava.CacheDesc(n_layers=2, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, max_pages=4,
                                           n_pages=64))
    lava.evict_scores(plan, q, k, k)
    for bad in _bad(k):
        for kk, vv in ((bad, k), (k, bad)):
            with pytest.raises(lava.LavaError):
                cache.admit(plan, kk, vv)
    with pytest.raises(lava.LavaError):
        cache.admit(plan, k, k, first_seq=2)
    assert int(cache.head_rows.sum()) == 0 and cache.free_page_count() == 64
    cache.admit(plan, k, k, first_seq=1)
    assert cache.poll_status() == 0 and int(cache.head_rows[:, 1].sum()) == 2 * 2 * 64

"""The slots of `PagedCache.extend` stay where they are: a captured step keeps their address, so a call that makes room for
another number of rows must neither free nor move them.  On the CPU with the library's call replaced; then on the GPU."""
import pytest
import torch

import paper_2509_09754_b200 as lava
from paper_2509_09754_b200 import paged as P


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(P, "lava_page_extend", lambda desc, add, rows, table, free, counters, slots, *a, **kw:
                        slots.fill_(int(add[0])))
    return lava.PagedCache(lava.CacheDesc(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64, max_pages=4,
                                          n_pages=64, page_rows=16), device="cpu")


def test_slots_keep_their_place_when_another_number_of_rows_comes_between(cache):
    ones, fives = torch.full((3,), 1, dtype=torch.int32), torch.full((3,), 5, dtype=torch.int32)
    first = cache.extend(ones)
    at = first.data_ptr()
    five = cache.extend(fives, max_add=5)
    del first
    # memory of the first call's size, as a program that goes on allocating has it: none of it is the slots'
    others = [torch.zeros((2, 3, 1, 2), dtype=torch.int32) for _ in range(64)]
    assert at not in [x.data_ptr() for x in others]
    assert cache.extend(ones).data_ptr() == at
    assert cache.extend(fives, max_add=5).data_ptr() == five.data_ptr()


def test_append_reads_the_slots_of_the_last_extend(cache):
    for n in (1, 5, 1, 2):
        slots = cache.extend(torch.full((3,), n, dtype=torch.int32), max_add=n)
        assert cache.slots is slots and slots.shape == (2, 3, n, 2) and bool((slots == n).all())


def test_the_copy_that_waits_is_the_last_of_a_new_cache(monkeypatch):
    """Every other buffer is filled on the current stream without waiting for it."""
    calls = []
    for name in ("empty", "zeros", "full", "arange", "tensor"):
        f = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, _f=f, _n=name, **kw: (calls.append(_n), _f(*a, **kw))[1])
    lava.PagedCache(lava.CacheDesc(n_layers=1, batch=1, n_q_heads=2, n_kv_heads=1, head_dim=64, max_pages=1, n_pages=1),
                    device="cpu")
    assert "tensor" not in calls[:-1] and calls[-1] == "tensor"


@pytest.mark.gpu
def test_a_captured_step_keeps_its_slots():
    """A step of one token in a graph; five rows eagerly; memory of the slots' size filled; the step replayed."""
    L, B, Hq, H, d = 2, 3, 4, 2, 64
    cache = lava.PagedCache(lava.CacheDesc(n_layers=L, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, page_rows=16,
                                           max_pages=4, n_pages=64))
    cache.k_pages.zero_(), cache.v_pages.zero_()
    add, fives = torch.ones(B, dtype=torch.int32, device="cuda"), torch.full((B,), 5, dtype=torch.int32, device="cuda")
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    rotary, freqs = lava.RotaryDesc(head_dim=d, rotary_dim=d), lava.lava_rotary_freqs(d)[0].cuda()
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((B, h, d), generator=g).bfloat16().cuda() for h in (Hq, H, H))

    def step():
        slots = cache.extend(add)
        for l in range(L):
            cache.append(rotary, freqs, l, pos, q, k, v)
        return slots

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slots = step()
    cache.extend(fives, max_add=5)
    fill = [torch.full((L, B, 1, H), 7, dtype=torch.int32, device="cuda") for _ in range(64)]
    before = cache.head_rows.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert cache.poll_status() == 0 and all(bool((x == 7).all()) for x in fill)
    assert torch.equal(cache.head_rows, before + 1)
    # the slots are those of the row that the replay made room for, and hold its values
    j = before.long()
    page = cache.page_table.gather(3, (j // 16).unsqueeze(-1)).squeeze(-1).long()
    assert torch.equal(slots[:, :, 0].long(), page * 16 + j % 16)
    rows = cache.v_pages.view(-1, d)[slots[:, :, 0].long()]
    assert torch.equal(rows, v.expand(L, B, H, d))

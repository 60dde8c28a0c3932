"""Page tables and compaction into pages against lists and plain indexing; everything is compared bit for bit."""
import numpy as np
import pytest
import torch

import paper_2509_09754_b200 as lava
from oracle import paged_oracle as PO

pytestmark = pytest.mark.gpu


class Device:
    """A cache's tables on the device beside the oracle's lists."""

    def __init__(self, L, B, H, page_rows, max_pages, n_pages, seed=0, taken=0):
        g = np.random.default_rng(seed)
        order = g.permutation(n_pages)
        self.shape, self.n_pages = (L, B, H), n_pages
        self.desc = lava.CacheDesc(n_layers=L, batch=B, n_q_heads=H, n_kv_heads=H, head_dim=64, page_rows=page_rows,
                                   max_pages=max_pages, n_pages=n_pages)
        self.lists = PO.Tables(L * B * H, page_rows, max_pages, order.tolist())
        i32 = dict(dtype=torch.int32, device="cuda")
        self.rows = torch.zeros((L, B, H), **i32)
        self.table = torch.full((L, B, H, max_pages), -7, **i32)
        self.free = torch.tensor(np.roll(order, taken % n_pages), **i32)
        self.counters = torch.tensor([taken, taken + n_pages], dtype=torch.int64, device="cuda")
        self.status = torch.zeros(64, **i32)

    def poll(self):
        word = int(self.status[0])
        self.status.zero_()
        return word

    def check(self):
        L, B, H = self.shape
        assert self.rows.view(-1).tolist() == self.lists.rows
        table = self.table.view(L * B * H, -1).cpu().numpy()
        for h, pages in enumerate(self.lists.pages):
            assert table[h, : len(pages)].tolist() == pages
        taken, given = self.counters.tolist()
        ring = self.free.cpu().numpy()
        assert [int(ring[i % self.n_pages]) for i in range(taken, given)] == self.lists.free

    def admit(self, counts, first=0):
        """counts [L, n_seqs, H]; the places where the new rows start."""
        L, n, H = counts.shape
        hoff = np.zeros((L, n, H + 1), dtype=np.int32)
        hoff[:, :, 1:] = counts.cumsum(2)
        out = torch.full((L, n, H), -9, dtype=torch.int32, device="cuda")
        before = self.rows.cpu().numpy()
        add = np.zeros(self.shape, dtype=np.int64)
        add[:, first: first + n] = counts
        places = self.lists.change(add.reshape(-1).tolist())
        lava.lava_page_admit(self.desc, first, torch.tensor(hoff).cuda(), self.rows, self.table, self.free,
                             self.counters, out, self.status)
        want = before[:, first: first + n] if places is not None else np.full(out.shape, -1)
        assert np.array_equal(out.cpu().numpy(), want)
        self.check()
        return places is not None

    def extend(self, add, most, slots=None):
        L, B, H = self.shape
        slots = torch.full((L, B, most, H), -9, dtype=torch.int32, device="cuda") if slots is None else slots
        per_head = [None if a < 0 else a for _ in range(L) for a in add for _ in range(H)]
        places = self.lists.change(per_head) if max(add) <= most else None
        lava.lava_page_extend(self.desc, torch.tensor(add, dtype=torch.int32).cuda(), self.rows, self.table, self.free,
                              self.counters, slots, self.status)
        want = np.full((L, B, most, H), -1)
        for h, p in enumerate(places or []):
            want[h // (B * H), h // H % B, : len(p), h % H] = p
        assert np.array_equal(slots.cpu().numpy(), want)
        self.check()
        return places is not None


@pytest.mark.parametrize("L,B,H,page_rows,taken", [
    (1, 1, 1, 16, 0), (1, 3, 2, 16, 5), (3, 5, 7, 32, 10**12), (4, 8, 8, 64, 3), (2, 2, 8, 256, 0),
    (32, 4, 8, 16, 77),      # exactly one block's heads
    (32, 8, 8, 16, 1),       # two blocks
    (28, 37, 4, 16, 9),      # several blocks, an odd share each
    (33, 40, 8, 16, 2),      # more than eight blocks' heads: some take two rounds
])
def test_tables_follow_admissions_tokens_and_releases(L, B, H, page_rows, taken):
    g = np.random.default_rng(L * 1000 + B)
    heads = L * B * H
    d = Device(L, B, H, page_rows, 6, 5 * heads + 3, seed=B, taken=taken)
    first = B // 3
    counts = g.integers(0, 3 * page_rows, (L, B - first, H))
    counts[0, 0, 0] = 0
    assert d.admit(counts, first)
    for step in range(4):
        add = g.integers(0, 3, B)
        if step == 2:
            add[g.integers(0, B)] = -1
        assert d.extend(add.tolist(), 2)
    # a released sequence comes back beside the running ones
    assert d.extend([-1] + [1] * (B - 1), 1)
    assert d.admit(g.integers(0, 2 * page_rows, (L, 1, H)), 0)
    assert d.poll() == 0


@pytest.mark.parametrize("L,B,H", [(1, 1, 3), (2, 6, 8), (33, 40, 8)])
def test_heads_of_many_pages(L, B, H):
    """Heads that take and give back up to 70 pages beside others that take one or none."""
    g = np.random.default_rng(L)
    heads = L * B * H
    d = Device(L, B, H, 16, 75, 80 * min(heads, 60) + 6 * heads, seed=1, taken=heads)
    counts = np.where(g.random((L, B, H)) < min(1.0, 40 / heads), g.integers(0, 70 * 16, (L, B, H)), g.integers(0, 20, (L, B, H)))
    assert d.admit(counts)
    for step in range(3):
        add = g.integers(0, 40, B)
        add[g.integers(0, B)] = -1
        assert d.extend(add.tolist(), 40)
    assert d.extend([-1] * B, 1)
    assert d.counters[1] - d.counters[0] == d.n_pages and d.poll() == 0


def test_what_does_not_fit_changes_nothing():
    d = Device(1, 2, 2, 16, 3, 6)
    assert d.admit(np.array([[[16, 17], [1, 0]]]))               # 1 + 2 + 1 + 0 pages of 6
    assert not d.extend([33, 16], 40)                            # 49 and 50 rows in a table of 48
    assert d.poll() == lava.LAVA_DEV_BAD_ROWS
    assert not d.extend([16, 17], 40)                            # 1 + 1 + 1 + 2 pages, 2 are free
    assert d.poll() == lava.LAVA_DEV_PAGES_EXHAUSTED
    assert not d.extend([3, 1], 2)                               # more than the slots have room for
    assert d.poll() == lava.LAVA_DEV_BAD_ROWS
    assert not d.admit(np.array([[[49, 0]]]), 1)
    assert d.poll() == lava.LAVA_DEV_BAD_ROWS
    assert not d.admit(np.array([[[5, -3]]]), 1)
    assert d.poll() == lava.LAVA_DEV_BAD_ROWS
    assert not d.extend([-1, 40], 40)                            # what is given back is there for the next call
    assert d.poll() == lava.LAVA_DEV_PAGES_EXHAUSTED
    assert d.extend([-1, 0], 1)
    assert d.extend([0, 40], 40)
    assert d.extend([-1, -1], 1) and len(d.lists.free) == 6
    assert d.poll() == 0


def test_counters_that_make_no_sense_are_refused():
    for taken, given in ((-1, 3), (5, 4), (0, 9)):
        d = Device(1, 1, 1, 16, 3, 8)
        d.counters.copy_(torch.tensor([taken, given]))
        slots = torch.zeros((1, 1, 1, 1), dtype=torch.int32, device="cuda")
        lava.lava_page_extend(d.desc, torch.ones(1, dtype=torch.int32, device="cuda"), d.rows, d.table, d.free,
                              d.counters, slots, d.status)
        assert d.poll() == lava.LAVA_DEV_PAGES_EXHAUSTED
        assert d.counters.tolist() == [taken, given] and int(slots) == -1 and int(d.rows) == 0
    d = Device(1, 1, 1, 16, 3, 8)                                # rows that no page was taken for
    d.rows.fill_(40)
    slots = torch.zeros((1, 1, 1, 1), dtype=torch.int32, device="cuda")
    lava.lava_page_extend(d.desc, torch.full((1,), -1, dtype=torch.int32, device="cuda"), d.rows, d.table, d.free,
                          d.counters, slots, d.status)
    assert d.poll() == lava.LAVA_DEV_BAD_ROWS and int(d.rows) == 40


def test_counts_can_go_to_other_buffers():
    d = Device(2, 2, 2, 16, 4, 40)
    d.admit(np.full((2, 2, 2), 20))
    rows, counters = d.rows.clone(), d.counters.clone()
    rows_out, counters_out = torch.full_like(rows, -3), torch.full_like(counters, -3)
    table = d.table.clone()
    slots = torch.empty((2, 2, 3, 2), dtype=torch.int32, device="cuda")
    add = torch.tensor([3, -1], dtype=torch.int32, device="cuda")
    lava.lava_page_extend(d.desc, add, d.rows, d.table, d.free, d.counters, slots, d.status, rows_out, counters_out)
    assert torch.equal(d.rows, rows) and torch.equal(d.counters, counters)
    d.table.copy_(table)
    assert d.extend([3, -1], 3)
    assert torch.equal(d.rows, rows_out) and torch.equal(d.counters, counters_out)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64), (torch.bfloat16, 64), (torch.float32, 128)])
@pytest.mark.parametrize("page_rows", [16, 64, 256])
def test_kept_rows_go_to_their_pages(dtype, d, page_rows):
    L, H, w, lens, B, first = 2, 3, 16, (150, 16, 61), 5, 1
    g = torch.Generator().manual_seed(5)
    T = sum(lens)
    k, v = (torch.randn((L, H, T, d), generator=g).to(dtype).cuda() for _ in range(2))
    # a view with other strides: tokens first
    v = v.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    cu = torch.tensor([0, 150, 166, 227], dtype=torch.int32, device="cuda")
    desc = lava.LayerDesc.for_tensors(torch.empty((3, H, w, d), dtype=dtype), k[0], v[0], w, cu_seqlens=cu, max_seqlen=150)
    rng = np.random.default_rng(6)
    counts = np.zeros((L, 3, H), dtype=np.int64)
    keep = np.full((L, desc.total_scores), -1, dtype=np.int32)
    chosen = {}
    for l in range(L):
        for b, n in enumerate(lens):
            at = H * (int(cu[b]) - b * w)
            for h in range(H):
                kept = np.sort(rng.choice(n - w, rng.integers(0, n - w + 1), replace=False)) if n > w else np.zeros(0, int)
                keep[l, at: at + len(kept)] = kept
                at += len(kept)
                chosen[l, b, h] = int(cu[b]) + np.concatenate([kept, np.arange(n - w, n)])
                counts[l, b, h] = len(kept) + w
    dev = Device(L, B, H, page_rows, 12 if page_rows == 16 else 4, 2 + 14 * L * B * H)
    dev.desc = lava.CacheDesc(n_layers=L, batch=B, n_q_heads=H, n_kv_heads=H, head_dim=d, page_rows=page_rows,
                              max_pages=dev.desc.max_pages, n_pages=dev.n_pages,
                              dtype=lava.LAVA_BF16 if dtype == torch.bfloat16 else lava.LAVA_F32)
    dev.admit(rng.integers(0, 2 * 16, (L, 1, H)), 1)             # rows that are there already: the new ones follow
    held = dev.rows.cpu().numpy()
    hoff = np.zeros((L, 3, H + 1), dtype=np.int32)
    hoff[:, :, 1:] = counts.cumsum(2)
    hoff, first_row = torch.tensor(hoff).cuda(), torch.empty((L, 3, H), dtype=torch.int32, device="cuda")
    lava.lava_page_admit(dev.desc, first, hoff, dev.rows, dev.table, dev.free, dev.counters, first_row, dev.status)
    assert dev.poll() == 0
    first_row[1, 2, 1] = -1                                      # a head without places is left out
    pools = [torch.full((dev.n_pages, page_rows, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    lava.lava_compact_kv_pages(desc, dev.desc, first, k, v, k.stride(0), v.stride(0), torch.tensor(keep).cuda(), hoff,
                               first_row, dev.table, *pools)
    table = dev.table.cpu().numpy()
    for pool, x in zip(pools, (k, v)):
        want = torch.full((dev.n_pages * page_rows, d), float("nan"), dtype=dtype)
        for (l, b, h), tok in chosen.items():
            if (l, b, h) != (1, 2, 1):
                row = held[l, first + b, h] + np.arange(len(tok))
                at = table[l, first + b, h, row // page_rows].astype(np.int64) * page_rows + row % page_rows
                want[torch.tensor(at)] = x[l, h].cpu()[torch.tensor(tok)]
        assert torch.equal(pool.view(-1, d).cpu().view(torch.uint8), want.view(torch.uint8))


def test_pages_outside_the_pool_are_not_written():
    k = torch.randn((1, 1, 40, 64), device="cuda")
    desc = lava.LayerDesc.for_tensors(torch.empty((1, 1, 8, 64)), k[0], k[0], 8)
    cache = lava.CacheDesc(n_layers=1, batch=1, n_q_heads=1, n_kv_heads=1, head_dim=64, page_rows=16, max_pages=2,
                           n_pages=2, dtype=lava.LAVA_F32)
    hoff = torch.tensor([[[0, 40]]], dtype=torch.int32, device="cuda")     # eight rows more than the table holds
    keep = torch.arange(32, dtype=torch.int32, device="cuda").view(1, 32)
    table = torch.tensor([[[[2, 1]]]], dtype=torch.int32, device="cuda")   # page 2 of 2
    room = torch.zeros((4, 16, 64), device="cuda")
    pool = room[1:3]
    lava.lava_compact_kv_pages(desc, cache, 0, k, k, 0, 0, keep, hoff, torch.zeros((1, 1, 1), dtype=torch.int32, device="cuda"),
                               table, pool, pool.clone())
    assert torch.equal(room[2], k[0, 0, 16:32]) and int((room[[0, 1, 3]] != 0).sum()) == 0

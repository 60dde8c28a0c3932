"""Paged decode attention against 64-bit attention head by head.

Tolerance per output, relative to sum_i p_i |V[i][c]|.  A logit is off by at most E = d 2^-24 sum |q_j k_j| scale (fp32
products and sums, also where a sum is cut off instead of rounded: 2^-23) + 2^-21 (|x| + cap) (scaling, the cap's tanh,
the change of base, the difference to the maximum), so a probability and its sum are off by 2 E + 2^-21 (exponential);
the sums over n rows add n 2^-23; with bf16 the probabilities enter as two terms, 2^-16, and the output is rounded by
2^-8 of itself.  The log-sum-exp is off by E + 2^-21 + n 2^-23 + 2^-22 |lse|.
"""
import math

import numpy as np
import pytest
import torch

import paper_2509_09754_b200 as lava
from oracle import paged_oracle as PO

pytestmark = pytest.mark.gpu

CODE = {torch.bfloat16: lava.LAVA_BF16, torch.float32: lava.LAVA_F32}


class Case:
    """A cache with these rows per head [L, B, H], pages in random order, and queries of layers first ... first + n - 1."""

    def __init__(self, rows, group=4, d=128, dtype=torch.bfloat16, page_rows=64, softcap=0.0, sm_scale=0.0, first=0,
                 n=None, seed=0, behind=float("nan"), q_scale=1.5, spare=3):
        g = torch.Generator().manual_seed(seed)
        rows = torch.tensor(rows)
        L, B, H = rows.shape
        n = L - first if n is None else n
        ps, Hq = page_rows, H * group
        held = -(-rows // ps)
        n_pages, most = int(held.sum()) + spare, max(1, int(held.max()) + 1)
        order = torch.randperm(n_pages, generator=g)
        table = torch.full((L, B, H, most), 2**30, dtype=torch.int64)       # behind the last page: anything
        at = 0
        self.flat = []
        k, v = torch.full((n_pages, ps, d), behind), torch.full((n_pages, ps, d), behind)
        for h in range(L * B * H):
            r, p = int(rows.view(-1)[h]), int(held.view(-1)[h])
            table.view(-1, most)[h, :p] = order[at: at + p]
            kh = torch.randn((r, d), generator=g) * torch.where(torch.rand((r, 1), generator=g) < 0.05, 3.0, 1.0)
            vh = torch.randn((r, d), generator=g)
            kh, vh = kh.to(dtype), vh.to(dtype)
            j = torch.arange(r)
            slot = order[at: at + p][j // ps] * ps + j % ps
            k.view(-1, d)[slot], v.view(-1, d)[slot] = kh.float(), vh.float()
            self.flat.append((kh.double().numpy(), vh.double().numpy()))
            at += p
        self.cache = lava.CacheDesc(n_layers=L, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, page_rows=ps,
                                    max_pages=most, n_pages=n_pages, dtype=CODE[dtype], softcap=softcap,
                                    sm_scale=sm_scale)
        self.k, self.v = k.to(dtype).cuda(), v.to(dtype).cuda()
        self.table, self.rows = table.int().cuda(), rows.int().cuda()
        self.q = (q_scale * torch.randn((n, B, Hq, d), generator=g)).to(dtype).cuda()
        self.ws = torch.zeros(lava.lava_cache_workspace_bytes(self.cache), dtype=torch.uint8, device="cuda")
        self.first, self.group, self.softcap, self.scale = first, group, softcap, sm_scale or 1 / math.sqrt(d)

    def run(self, q=None, first=None, ws=None):
        q = self.q if q is None else q
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        lse = torch.full(q.shape[:3], float("nan"), device="cuda")
        lava.lava_decode_attention_pages(self.cache, self.first if first is None else first, q, self.k, self.v, self.table,
                                         self.rows, out, lse, self.ws if ws is None else ws)
        return out, lse

    def check(self, out, lse):
        n, B, Hq, d = self.q.shape
        H, g, bf16 = Hq // self.group, self.group, self.q.dtype == torch.bfloat16
        q = self.q.double().cpu().numpy().reshape(n * B * H, g, d)
        out, lse = out.double().cpu().numpy().reshape(q.shape), lse.double().cpu().numpy().reshape(n * B * H, g)
        for h in range(n * B * H):
            k, v = self.flat[self.first * B * H + h]
            want, want_lse = PO.attend(q[h], k, v, self.scale, self.softcap)
            if len(k) == 0:
                assert np.all(out[h] == 0) and np.all(lse[h] == -np.inf), h
                continue
            mag, _ = PO.attend(q[h], k, np.abs(v), self.scale, self.softcap)
            size = np.abs(q[h]) @ np.abs(k).T * self.scale                       # sum |q_j k_j| scale of every logit
            e = (d * 2.0 ** -23 * size + 2.0 ** -21 * (size + self.softcap)).max(axis=1, keepdims=True)
            rel = 2 * e + 2.0 ** -21 + len(k) * 2.0 ** -23 + (2.0 ** -16 if bf16 else 0.0)
            tol = rel * mag
            tol += 2.0 ** -8 * (np.abs(want) + tol) if bf16 else 0.0
            err = np.abs(out[h] - want)
            assert np.all(err <= tol), (h, len(k), err.max(), (err / tol).max())
            tol = e[:, 0] + 2.0 ** -21 + len(k) * 2.0 ** -23 + 2.0 ** -22 * np.abs(want_lse)
            assert np.all(np.abs(lse[h] - want_lse) <= tol), (h, len(k), np.abs(lse[h] - want_lse).max())


def _check(*a, **kw):
    c = Case(*a, **kw)
    out, lse = c.run()
    c.check(out, lse)
    return c, out, lse


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257, 500, 1030]


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64)])
@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 256])
def test_every_length_and_page_size(dtype, d, page_rows):
    _check([[LENGTHS[i: i + 2]] for i in range(0, len(LENGTHS), 2)], d=d, dtype=dtype, page_rows=page_rows)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64)])
@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 32, 33])
def test_every_group(dtype, d, group):
    _check([[[100, 0, 37]], [[700, 1, 64]]], group=group, d=d, dtype=dtype, page_rows=32, seed=group)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("softcap,sm_scale,q_scale", [(30.0, 0.0, 1.5), (50.0, 0.2, 8.0), (0.0, 0.5, 4.0), (2.0, 0.0, 20.0),
                                                      (1e4, 0.0, 1.5)])
def test_caps_and_scales(dtype, softcap, sm_scale, q_scale):
    _check([[[300, 90]], [[5, 1000]]], dtype=dtype, softcap=softcap, sm_scale=sm_scale, q_scale=q_scale)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_one_long_head_is_split_and_joined(dtype, d):
    _check([[[40000]]], dtype=dtype, d=d, group=4)
    _check([[[20011, 3]]], dtype=dtype, d=d, group=7, page_rows=16, seed=1)


def test_many_heads_of_uneven_length():
    g = np.random.default_rng(3)
    rows = np.minimum(3000, (60 * np.exp(1.5 * g.standard_normal((3, 40, 8)))).astype(int))
    rows[1, 7] = 0
    _check(rows.tolist(), group=4)
    rows = np.minimum(700, (20 * np.exp(1.5 * g.standard_normal((2, 9, 3)))).astype(int))
    _check(rows.tolist(), group=3, dtype=torch.float32)


def test_more_heads_than_a_block_has_threads():
    g = np.random.default_rng(4)
    rows = g.integers(0, 40, (8, 70, 8))
    _check(rows.tolist(), group=1, d=64, page_rows=16)


@pytest.mark.parametrize("dtype,d,group", [(torch.bfloat16, 128, 4), (torch.bfloat16, 128, 8), (torch.bfloat16, 128, 12),
                                           (torch.bfloat16, 64, 16), (torch.bfloat16, 64, 20), (torch.float32, 64, 2),
                                           (torch.float32, 64, 8), (torch.float32, 64, 9), (torch.float32, 128, 3)])
def test_many_short_heads(dtype, d, group):
    """Thousands of heads of a few boxes of 16 rows, some without rows: whole heads per warp where the type allows it."""
    g = np.random.default_rng(d + group)
    rows = np.where(g.random((5, 90, 8)) < 0.2, 0, g.integers(1, 50, (5, 90, 8)))
    rows[0, 0], rows[4, 89] = 0, 0                                   # at both ends too
    rows[2, 45, 3] = 64
    _check(rows.tolist(), group=group, d=d, dtype=dtype, page_rows=16)


@pytest.mark.parametrize("rows,group", [([[[9000, 100]]], 20), ([[[3000, 1700, 0, 2500]]] * 5, 40), ([[[2600] * 8]] * 9, 2)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_heads_and_large_groups(rows, group, dtype):
    """Pieces of both sizes and equal parts of the line, one and several portions of a group's queries."""
    _check(rows, group=group, d=64, dtype=dtype)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 128), (torch.bfloat16, 64)])
@pytest.mark.parametrize("n_heads", [1, 3, 40, 1024, 1030, 2100])
def test_heads_of_odd_numbers_of_boxes(dtype, d, n_heads):
    """Heads whose last tile is not full, one after the other on the line: every cut falls elsewhere in a tile."""
    g = np.random.default_rng(n_heads)
    rows = g.choice([1, 17, 33, 49, 65, 79, 161, 300], (n_heads, 1, 1))
    if n_heads > 1000:
        rows[n_heads // 3] = 9001                                    # too long for whole heads per warp
    _check(rows.tolist(), group=2, d=d, dtype=dtype, page_rows=16)


def test_first_rows_at_minus_infinity_over_many_tiles():
    """-inf logits fill whole tiles, pieces and parts before the first finite one."""
    c = Case([[[3000, 40]]], group=2, dtype=torch.float32, d=64)
    c.q.copy_(c.q.abs() + 0.1)
    table = c.table[0, 0, 0].cpu()
    c.k.view(-1, 64)[[int(table[j // 64]) * 64 + j % 64 for j in range(2900)]] = -float("inf")
    out, lse = c.run()
    k, v = c.flat[0]
    c.flat[0] = (k[2900:], v[2900:])
    c.check(out, lse)


@pytest.mark.parametrize("L,rows", [(1, 2048), (32, 64)])
def test_an_expired_wait_is_reported_and_a_zeroed_workspace_serves_again(L, rows):
    """With a limit of one cycle a wait gives up at its second look: those for the first rows do (512 long heads by all
    warps, 16384 short ones by a warp each).  The kernel returns, and the status word says so."""
    B, H, d, ps = 64, 8, 128, 64
    held = rows // ps
    cache = lava.CacheDesc(n_layers=L, batch=B, n_q_heads=4 * H, n_kv_heads=H, head_dim=d, page_rows=ps, max_pages=held,
                           n_pages=L * B * H * held)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((cache.n_pages, ps, d), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.randperm(cache.n_pages, generator=g, device="cuda").int().view(L, B, H, held)
    counts = torch.full((L, B, H), rows, dtype=torch.int32, device="cuda")
    q = torch.randn((L, B, 4 * H, d), generator=g, device="cuda", dtype=torch.bfloat16)
    ws = torch.zeros(lava.lava_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")

    def run():
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
        lava.lava_decode_attention_pages(cache, 0, q, k, v, table, counts, out, lse, ws)
        return out, lse

    want = run()
    normal = lava.lava_get_option("wait_limit_cycles")
    try:
        lava.lava_set_option("wait_limit_cycles", 1)
        run()
        with pytest.raises(lava.LavaError) as err:
            lava.lava_poll_status(ws)
        assert err.value.status == 5                                   # LAVA_ERR_TIMEOUT
    finally:
        lava.lava_set_option("wait_limit_cycles", normal)
    ws.zero_()
    got = run()
    assert lava.lava_poll_status(ws) == 0
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_cache_without_any_rows():
    _, out, lse = _check([[[0, 0], [0, 0]]], behind=1.0)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("behind", [float("inf"), -float("inf"), float("nan"), 3e38])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_behind_the_last_are_never_read_into_a_result(behind, dtype):
    c, out, lse = _check([[[1, 17], [70, 0]], [[200, 63], [64, 130]]], behind=behind, dtype=dtype)
    d = Case([[[1, 17], [70, 0]], [[200, 63], [64, 130]]], behind=0.0, dtype=dtype)
    out0, lse0 = d.run()
    assert torch.equal(out, out0) and torch.equal(lse, lse0)


def test_single_layers_and_ranges_of_layers():
    rows = np.random.default_rng(5).integers(0, 300, (5, 3, 2)).tolist()
    for first, n in ((0, 1), (4, 1), (1, 3), (0, 5)):
        _check(rows, first=first, n=n, seed=2)


def test_infinite_and_missing_values_among_the_rows_follow_the_formula():
    """A row whose logit is -inf has probability 0 (its V must be finite), one of +inf or NaN makes the head NaN."""
    c = Case([[[80, 80, 80]]], group=2, dtype=torch.float32, d=64)
    table = c.table[0, 0].cpu()
    c.q.copy_(c.q.abs())
    flat = c.k.view(-1, 64)
    rows = [int(table[h, 40 // 64]) * 64 + 40 for h in range(3)]
    flat[rows[0]] = -float("inf")
    flat[rows[1]] = float("inf")
    flat[rows[2], 5] = float("nan")
    out, lse = c.run()
    assert bool(torch.isfinite(out[0, 0, :2]).all()) and bool(torch.isfinite(lse[0, 0, :2]).all())
    k, v = c.flat[0]
    keep = np.arange(80) != 40
    want, _ = PO.attend(c.q[0, 0, :2].double().cpu().numpy(), k[keep], v[keep])
    # (as above, with logits of at most 64 * 2^-23 * sum |q k| scale < 2^-12)
    assert np.all(np.abs(out[0, 0, :2].double().cpu().numpy() - want) <= 2.0 ** -10 * np.abs(v).max())
    assert bool(torch.isnan(out[0, 0, 2:]).all())
    # all of a head's first rows at -inf: what follows counts
    c.k.view(-1, 64)[[int(table[0, j // 64]) * 64 + j % 64 for j in range(70)]] = -float("inf")
    out, _ = c.run()
    k, v = c.flat[0]
    want, _ = PO.attend(c.q[0, 0, :2].double().cpu().numpy(), k[70:], v[70:])
    assert np.all(np.abs(out[0, 0, :2].double().cpu().numpy() - want) <= 2.0 ** -10 * np.abs(v).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pages_outside_the_pool_read_as_zeros(dtype):
    c = Case([[[40, 40]]], group=1, page_rows=16, dtype=dtype, behind=0.0)
    for bad in (-1, c.cache.n_pages, 2**31 - 1, -2**31):
        c.table[0, 0, 0, 1] = bad
        out, lse = c.run()
        k, v = (x.copy() for x in c.flat[0])
        k[16:32], v[16:32] = 0, 0
        keep, c.flat[0] = c.flat[0], (k, v)
        c.check(out, lse)
        c.flat[0] = keep


def test_row_counts_outside_the_table_are_held_inside():
    c = Case([[[64, 20]]], group=2)
    c.rows[0, 0, 0], c.rows[0, 0, 1] = 2**31 - 1, -5
    c.table[0, 0, 0, 1] = int(c.table[0, 0, 0, 0])                # both pages of the table: the same rows twice
    out, lse = c.run()
    k, v = c.flat[0]
    c.flat[0] = (np.concatenate([k, k]), np.concatenate([v, v]))
    c.flat[1] = (k[:0], v[:0])
    c.check(out, lse)


def test_heads_may_share_pages():
    c = Case([[[100, 100]]], group=4)
    c.table[0, 0, 1] = c.table[0, 0, 0]
    c.flat[1] = c.flat[0]
    c.check(*c.run())


def test_the_same_call_gives_the_same_bits_and_leaves_its_workspace_ready():
    g = np.random.default_rng(6)
    big = Case((g.integers(0, 900, (2, 9, 8))).tolist(), group=4)
    small = Case([[[1500, 3]]], group=4, seed=9)
    ws = torch.zeros(max(big.ws.numel(), small.ws.numel()), dtype=torch.uint8, device="cuda")
    first_b, first_s = big.run(ws=ws), small.run(ws=ws)
    for _ in range(20):
        for c, first in ((small, first_s), (big, first_b)):
            again = c.run(ws=ws)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    big.check(*first_b)
    small.check(*first_s)


def test_a_captured_call_follows_the_row_counts_of_its_replay():
    c = Case([[[700, 20, 300], [5, 1000, 64]]], group=4)
    full = c.rows.clone()
    out, lse = torch.empty_like(c.q), torch.empty(c.q.shape[:3], device="cuda")
    c.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lava.lava_decode_attention_pages(c.cache, 0, c.q, c.k, c.v, c.table, c.rows, out, lse, c.ws)
    keep = list(c.flat)
    for cut in (0, 1, 650, 63, 0):
        c.rows.copy_((full - cut).clamp(min=0))
        c.flat = [(k[: max(0, len(k) - cut)], v[: max(0, len(v) - cut)]) for k, v in keep]
        graph.replay()
        torch.cuda.synchronize()
        c.check(out, lse)


def test_two_streams_with_a_workspace_each():
    a, b = Case([[[2000, 500]]], seed=1), Case([[[30, 900, 1]]], seed=2, group=8)
    want = [x.run() for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(10):
        for c, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                got.append(c.run())
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


def test_rows_far_into_a_large_pool():
    """Byte offsets past 32 bits: a pool of 5 GB, the head's pages at its end."""
    ps, d, n_pages = 256, 128, 80000
    cache = lava.CacheDesc(n_layers=1, batch=1, n_q_heads=4, n_kv_heads=1, head_dim=d, page_rows=ps, max_pages=3,
                           n_pages=n_pages)
    k = torch.empty((n_pages, ps, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    g = torch.Generator().manual_seed(3)
    pages, n = [79999, 40000, 79998], 600
    kh, vh = torch.randn((3 * ps, d), generator=g).bfloat16(), torch.randn((3 * ps, d), generator=g).bfloat16()
    k[pages], v[pages] = kh.view(3, ps, d).cuda(), vh.view(3, ps, d).cuda()
    c = Case.__new__(Case)
    c.cache, c.k, c.v = cache, k, v
    c.table = torch.tensor([[[pages]]], dtype=torch.int32, device="cuda")
    c.rows = torch.full((1, 1, 1), n, dtype=torch.int32, device="cuda")
    c.q = torch.randn((1, 1, 4, d), generator=g).bfloat16().cuda()
    c.ws = torch.zeros(lava.lava_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    c.first, c.group, c.softcap, c.scale = 0, 4, 0.0, d ** -0.5
    c.flat = [(kh[:n].double().numpy(), vh[:n].double().numpy())]
    c.check(*c.run())


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("rows", [130, 600, 2500, 9000, 17000, 36000, 80001, 170000])
def test_few_heads_in_pieces_of_every_size(rows, dtype, d):
    """Few heads are cut into pieces of 64 KB to 2 MB, as long as there are CTAs for them, or into equal parts.  The heads
    are long by naming the pages of a small pool again and again; the wanted values come from the rows' multiplicity."""
    g = torch.Generator().manual_seed(rows)
    lens = torch.tensor([rows, rows // 2, 1, rows - 7, 0, rows, rows // 3, rows - 64])
    ps, n_pages, group = 64, 48, 3
    most = -(-rows // ps)
    table = torch.randint(0, n_pages, (1, 1, 8, most), generator=g)
    k, v = (torch.randn((n_pages, ps, d), generator=g).to(dtype).cuda() for _ in range(2))
    q = torch.randn((1, 1, 8 * group, d), generator=g).to(dtype).cuda()
    cache = lava.CacheDesc(n_layers=1, batch=1, n_q_heads=8 * group, n_kv_heads=8, head_dim=d, page_rows=ps,
                           max_pages=most, n_pages=n_pages, dtype=CODE[dtype])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    ws = torch.zeros(lava.lava_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        lava.lava_decode_attention_pages(cache, 0, q, k, v, table.int().cuda(), lens.int().view(1, 1, 8).cuda(), out, lse, ws)
    assert lava.lava_poll_status(ws) == 0
    kd, vd = k.double().view(-1, d), v.double().view(-1, d)
    for h in range(8):
        n = int(lens[h])
        got, got_lse = out[0, 0, h * group: (h + 1) * group].double(), lse[0, 0, h * group: (h + 1) * group].double()
        if n == 0:
            assert bool((got == 0).all()) and bool((got_lse == -math.inf).all())
            continue
        times = torch.zeros(n_pages * ps, dtype=torch.float64)
        j = torch.arange(n)
        times.index_add_(0, table[0, 0, h][j // ps] * ps + j % ps, torch.ones(n, dtype=torch.float64))
        times = times.cuda()
        qh = q[0, 0, h * group: (h + 1) * group].double()
        x = qh @ kd.T / math.sqrt(d)
        x = torch.where(times > 0, x, -math.inf)
        p = times * torch.exp(x - x.max(dim=1, keepdim=True).values)
        want, mag = p @ vd / p.sum(1, keepdim=True), p @ vd.abs() / p.sum(1, keepdim=True)
        want_lse = x.max(dim=1).values + p.sum(1).log()
        size = qh.abs() @ kd.abs().T / math.sqrt(d)
        e = (d * 2.0 ** -23 * size + 2.0 ** -21 * size).max(dim=1, keepdim=True).values
        # (a warp sums at most a tile's share in one go and adds a sum per tile: no more than n terms in all)
        tol = (2 * e + 2.0 ** -21 + n * 2.0 ** -23 + (2.0 ** -16 if dtype == torch.bfloat16 else 0.0)) * mag
        tol += 2.0 ** -8 * (want.abs() + tol) if dtype == torch.bfloat16 else 0.0
        assert bool(((got - want).abs() <= tol).all()), (h, float(((got - want).abs() / tol).max()))
        tol = e[:, 0] + 2.0 ** -21 + n * 2.0 ** -23 + 2.0 ** -22 * want_lse.abs()
        assert bool(((got_lse - want_lse).abs() <= tol).all()), h

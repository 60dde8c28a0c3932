"""Paged decode attention over more than 64 x 512 heads, whose segments are counted in several rounds of 512.  Against batched attention in 64 bits on the device, every head.

Tolerances as for single heads (tests/test_gpu_paged_attention.py): a logit is off by E = d 2^-23 sum |q_j k_j| scale +
2^-21 of that sum, a probability by 2 E + 2^-21, the sums over n rows by n 2^-23, bf16 terms of probabilities by 2^-16, a
bf16 output by 2^-8 of itself."""
import math

import pytest
import torch

import paper_2509_09754_b200 as lava

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L,B,H,group,d,dtype,rows,long", [
    (64, 80, 8, 1, 64, torch.bfloat16, (0, 40), 0),        # whole heads by a warp each
    (64, 80, 8, 1, 64, torch.bfloat16, (0, 40), 5000),     # a few long ones: equal parts of the line
    (33, 125, 8, 2, 64, torch.float32, (0, 40), 3000),     # one head over 32768 and not a multiple of 512
    (64, 80, 8, 1, 128, torch.float32, (0, 40), 0),        # tiles of 32 rows: no whole heads
    (70, 130, 8, 1, 64, torch.bfloat16, (1, 3), 0),        # 72800 heads: segments of 2048
    (32, 64, 8, 4, 128, torch.bfloat16, (64, 64), 0),      # 16384 heads of one length
])
def test_more_than_32768_heads(L, B, H, group, d, dtype, rows, long):
    heads, ps = L * B * H, 16
    g = torch.Generator(device="cuda").manual_seed(heads + d)
    n = torch.randint(rows[0], rows[1] + 1, (heads,), generator=g, device="cuda")
    longs = [0, 1, heads // 3, 32767, heads - 1] if long else []
    for i, h in enumerate(longs):
        n[h] = long + 17 * i
    n_pages, most = 3000, -(-int(n.max()) // ps)
    # pages of a small pool, each in many heads
    table = torch.randint(0, n_pages, (L, B, H, most), generator=g, device="cuda", dtype=torch.int32)
    k, v = (torch.randn((n_pages, ps, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = (1.5 * torch.randn((L, B, H * group, d), generator=g, device="cuda")).to(dtype)
    cache = lava.CacheDesc(n_layers=L, batch=B, n_q_heads=H * group, n_kv_heads=H, head_dim=d, page_rows=ps, max_pages=most,
                           n_pages=n_pages, dtype=lava.LAVA_F32 if dtype == torch.float32 else lava.LAVA_BF16)
    out = torch.full(q.shape, float("nan"), dtype=dtype, device="cuda")
    lse = torch.full(q.shape[:3], float("nan"), device="cuda")
    ws = torch.zeros(lava.lava_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    lava.lava_decode_attention_pages(cache, 0, q, k, v, table, n.int().view(L, B, H), out, lse, ws)
    assert lava.lava_poll_status(ws) == 0

    def check(at):  # heads of about one length
        top = max(1, int(n[at].max()))
        j = torch.arange(top, device="cuda")
        row = table.view(heads, most)[at][:, j // ps].long() * ps + j % ps
        there = (j < n[at].unsqueeze(1)).unsqueeze(1)
        kk, vv = k.view(-1, d)[row].double(), v.view(-1, d)[row].double()
        qq = q.view(heads, group, d)[at].double()
        x = torch.where(there, qq @ kk.transpose(1, 2) / math.sqrt(d), -math.inf)
        p = torch.where(there.any(-1, keepdim=True), torch.softmax(x, -1), 0.0)
        want, mag, want_lse = p @ vv, p @ vv.abs(), torch.logsumexp(x, -1)
        size = torch.where(there, qq.abs() @ kk.abs().transpose(1, 2) / math.sqrt(d), 0.0).amax(-1, keepdim=True)
        e = (d * 2.0 ** -23 + 2.0 ** -21) * size
        bf16 = dtype == torch.bfloat16
        tol = (2 * e + 2.0 ** -21 + top * 2.0 ** -23 + (2.0 ** -16 if bf16 else 0.0)) * mag
        tol = tol + (2.0 ** -8 * (want.abs() + tol) if bf16 else 0.0)
        got, got_lse = out.view(heads, group, d)[at].double(), lse.view(heads, group)[at].double()
        err = (got - want).abs()
        assert bool((err <= tol).all()), (float(err.max()), at[(err > tol).flatten(1).any(1)][:8].tolist())
        empty = n[at] == 0
        assert bool((got[empty] == 0).all()) and bool((got_lse[empty] == -math.inf).all())
        tol = e[..., 0] + 2.0 ** -21 + top * 2.0 ** -23 + 2.0 ** -22 * want_lse.abs()
        assert bool(((got_lse - want_lse).abs() <= tol)[~empty].all())

    short = torch.ones(heads, dtype=torch.bool, device="cuda")
    short[longs] = False
    for at in short.nonzero().view(-1).split(8192):
        check(at)
    for h in longs:
        check(torch.tensor([h], device="cuda"))

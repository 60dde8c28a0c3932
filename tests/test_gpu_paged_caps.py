"""The cap of the paged attention's logits, by itself: heads of one row, whose log-sum-exp is the capped logit.

Keys are a unit vector and the scale is 1, so a logit is an element of the query, exactly.  With u = 2^-24, relative to the
result: the factor 1 / cap and its product 2 u (tanh passes on no more of it); tanhf within 2 ulp, 4 u; cap * log2(e) and its
product 3 u; the change of base 2 u; second order terms 1 u."""
import numpy as np
import pytest
import torch

import paper_2509_09754_b200 as lava

pytestmark = pytest.mark.gpu


def _capped(z, dtype, d, cap, seed):
    """Queries that ask for logits cap * z, and the log-sum-exp of heads of one row."""
    H, group, ps = 4, 8, 16
    B = len(z) // (H * group)
    g = torch.Generator().manual_seed(seed)
    q = torch.zeros((1, B, H * group, d))
    q[..., 3] = (cap * z).view(1, B, H * group)
    q = q.to(dtype).cuda()
    k = torch.zeros((B * H, ps, d), dtype=dtype, device="cuda")
    k[:, :, 3] = 1.0
    v = torch.randn((B * H, ps, d), generator=g).to(dtype).cuda()
    cache = lava.CacheDesc(n_layers=1, batch=B, n_q_heads=H * group, n_kv_heads=H, head_dim=d, page_rows=ps, max_pages=1,
                           n_pages=B * H, sm_scale=1.0, softcap=cap,
                           dtype=lava.LAVA_F32 if dtype == torch.float32 else lava.LAVA_BF16)
    table = torch.arange(B * H, dtype=torch.int32, device="cuda").view(1, B, H, 1)
    rows = torch.ones((1, B, H), dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, B, H * group), device="cuda")
    ws = torch.zeros(lava.lava_cache_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    lava.lava_decode_attention_pages(cache, 0, q, k, v, table, rows, out, lse, ws)
    assert torch.equal(out.view(B, H, group, d), v.view(B, H, ps, d)[:, :, :1].expand(B, H, group, d))
    return q[..., 3].double().cpu().numpy(), lse.double().cpu().numpy()


@pytest.mark.parametrize("dtype,d", [(torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 128), (torch.bfloat16, 64)])
@pytest.mark.parametrize("cap", [50.0, 30.0, 3.0])
def test_capped_logits_of_single_rows(dtype, d, cap):
    n = 2048
    g = torch.Generator().manual_seed(int(cap))
    z = torch.cat([0.2 + 0.4 * torch.rand(n // 2, generator=g),                        # around a quarter of the cap
                   10.0 ** (4 * torch.rand(n // 2, generator=g) - 3)])                 # 0.001 ... 10 of it
    z = z * torch.where(torch.rand(z.shape, generator=g) < 0.5, -1.0, 1.0)
    x, lse = _capped(z, dtype, d, cap, 1)
    want = cap * np.tanh(x / cap)
    err = np.abs(lse - want)
    assert np.all(err <= 12 * 2.0 ** -24 * np.abs(want)), float((err / np.abs(want)).max() * 2 ** 24)


@pytest.mark.parametrize("d", [64, 128])
def test_the_cap_keeps_the_bits_of_a_tanh(d):
    """A cap of 4: its factors are exact, and of the terms above are left tanhf 4 u, the bases' constants 0.3 u, the product
    with each 1 u, and 0.2 u of second order."""
    for low, high in ((0.05, 0.25), (0.25, 0.26), (0.26, 0.27), (0.27, 0.3), (0.3, 0.4), (0.4, 0.6), (0.6, 2.0), (2.0, 12.0)):
        x, lse = _capped(torch.linspace(low, high, 8192), torch.float32, d, 4.0, 2)
        want = 4.0 * np.tanh(x / 4.0)
        err = np.abs(lse - want) / want
        assert err.max() <= 6.5 * 2.0 ** -24, (low, high, err.max() * 2 ** 24)

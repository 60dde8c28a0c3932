"""Rotary positions and the append of new tokens against complex products in 64 bits.

Tolerance, relative to |a| + |b| of a pair times the scale: the angle in turns is reduced in 64 bits and rounded to
fp32 (2^-25 turns at most, 1.9e-7 rad), sincospif is within 2 ulp (1.2e-7), the factor, the two products and their
sum round once each (4 * 2^-24): 5.5e-7 < 2^-20.  For positions p and frequency 1 both sides' 64-bit products carry
p * 2^-52 more.  The output's rounding adds half a step: 2^-8 of the value with bf16.
"""
import numpy as np
import pytest
import torch

import paper_2509_09754_b200 as lava
from oracle import paged_oracle as PO

pytestmark = pytest.mark.gpu

CODE = {torch.bfloat16: lava.LAVA_BF16, torch.float32: lava.LAVA_F32}


def _check(got, x, positions, freqs, interleaved, backward, scale):
    x, got, r = x.double().cpu().numpy(), got.double().cpu(), 2 * len(freqs)
    dtype_round = 2.0 ** -8 if _check.dtype == torch.bfloat16 else 0.0
    want = PO.rotate(x, positions, freqs, interleaved, backward, scale)
    size = np.zeros_like(x)
    if r:
        lead = np.abs(x[..., :r])
        both = lead[..., 0::2] + lead[..., 1::2] if interleaved else lead[..., : r // 2] + lead[..., r // 2:]
        size[..., :r] = np.repeat(both, 2, -1) if interleaved else np.concatenate([both, both], -1)
    far = 2.0 ** -20 + 2.0 ** -51 * np.abs(np.asarray(positions, dtype=np.float64)).max(initial=0)
    err = np.abs(got.numpy() - want)
    tol = far * scale * size
    tol = tol + dtype_round * (np.abs(want) + tol) * (size > 0)
    assert np.all(err <= tol), (err.max(), (err - tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,r", [(64, 64), (128, 128), (128, 64), (128, 16), (64, 48), (128, 112), (64, 0)])
@pytest.mark.parametrize("interleaved,backward,scale", [(False, False, 1.0), (True, False, 1.2), (False, True, 1.2),
                                                        (True, True, 1.0)])
def test_rotation_matches_complex_products(dtype, d, r, interleaved, backward, scale):
    _check.dtype = dtype
    g = torch.Generator().manual_seed(d + r)
    N, Hq, H = 37, 6, 2
    x = torch.randn((N, (Hq + H) * d), generator=g).to(dtype).cuda()
    q, k = x[:, : Hq * d].view(N, Hq, d), x[:, Hq * d:].view(N, H, d)
    pos = torch.randint(0, 200000, (N,), generator=g).int()
    pos[:3] = torch.tensor([0, 1, 2**31 - 1])
    pos[3] = -5                                                    # before the first token: turns the other way
    freqs = lava.lava_rotary_freqs(r)[0] if r else torch.zeros(0, dtype=torch.float64)
    desc = lava.RotaryDesc(head_dim=d, rotary_dim=r, dtype=CODE[dtype], interleaved=interleaved, backward=backward,
                           scale=scale)
    q_out = torch.full((N, Hq, d), float("nan"), dtype=dtype, device="cuda")
    k_out = torch.full((H, N, d), float("nan"), dtype=dtype, device="cuda").permute(1, 0, 2)
    lava.lava_rotary(desc, freqs.cuda(), pos.cuda(), q, k, q_out, k_out)
    _check(q_out, q, pos.numpy(), freqs.numpy(), interleaved, backward, scale)
    _check(k_out, k, pos.numpy(), freqs.numpy(), interleaved, backward, scale)
    assert torch.equal(q_out[..., r:], q[..., r:]) and torch.equal(k_out[..., r:], k[..., r:])
    # in place, and one array alone: the same bits
    both = x.clone()
    lava.lava_rotary(desc, freqs.cuda(), pos.cuda(), both[:, : Hq * d].view(N, Hq, d), both[:, Hq * d:].view(N, H, d),
                     both[:, : Hq * d].view(N, Hq, d), both[:, Hq * d:].view(N, H, d))
    assert torch.equal(both[:, : Hq * d].view(N, Hq, d), q_out) and torch.equal(both[:, Hq * d:].view(N, H, d), k_out)
    alone = torch.empty_like(k_out)
    lava.lava_rotary(desc, freqs.cuda(), pos.cuda(), None, k, None, alone)
    assert torch.equal(alone, k_out)


@pytest.mark.parametrize("N", [0, 1, 2, 31, 33, 300, 5000])
@pytest.mark.parametrize("Hq,H,dtype", [(32, 8, torch.bfloat16), (28, 4, torch.bfloat16), (1, 1, torch.float32), (5, 5, torch.float32)])
def test_any_number_of_tokens_and_heads(N, Hq, H, dtype):
    _check.dtype = dtype
    d = 128
    g = torch.Generator().manual_seed(N)
    q, k = torch.randn((N, Hq, d), generator=g).to(dtype).cuda(), torch.randn((N, H, d), generator=g).to(dtype).cuda()
    pos = (1000003 + torch.arange(N)).int()
    freqs, scale = lava.lava_rotary_freqs(d, 500000.0, lava.LAVA_ROTARY_RAMP, 8.0, 8192.0, 1.0, 32.0)
    desc = lava.RotaryDesc(head_dim=d, rotary_dim=d, dtype=CODE[dtype], scale=scale)
    # rows in front and behind stay as they are
    room = torch.full((N + 2, Hq, d), 7.0, dtype=dtype, device="cuda")
    k_out = torch.empty_like(k)
    lava.lava_rotary(desc, freqs.cuda(), pos.cuda(), q, k, room[1: N + 1], k_out)
    if N:
        _check(room[1: N + 1], q, pos.numpy(), freqs.numpy(), False, False, scale)
        _check(k_out, k, pos.numpy(), freqs.numpy(), False, False, scale)
    assert bool((room[[0, N + 1]] == 7.0).all())


def test_inputs_shared_by_all_heads_and_tokens():
    _check.dtype = torch.float32
    x = torch.randn((1, 1, 64), device="cuda").expand(9, 4, 64)
    freqs = lava.lava_rotary_freqs(64)[0]
    out = torch.empty((9, 4, 64), device="cuda")
    desc = lava.RotaryDesc(head_dim=64, rotary_dim=64, dtype=lava.LAVA_F32)
    lava.lava_rotary(desc, freqs.cuda(), torch.arange(9, dtype=torch.int32, device="cuda"), x, None, out, None)
    _check(out, x, np.arange(9), freqs.numpy(), False, False, 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_backward_is_the_gradient(interleaved):
    """Against the formula: <R x, g> = <x, R^T g>; and against differences of the forward pass, which is linear, so
    that the difference of two outputs is the output of the difference up to the roundings of fp32."""
    d, r, N, H = 64, 48, 11, 3
    g = torch.Generator().manual_seed(1)
    x, grad, step = (torch.randn((N, H, d), generator=g).cuda() for _ in range(3))
    pos = (torch.arange(N) * 997).int().cuda()
    freqs, scale = lava.lava_rotary_freqs(r, kind=lava.LAVA_ROTARY_RAMP, factor=4.0, low=1.0, high=32.0)
    make = dict(head_dim=d, rotary_dim=r, dtype=lava.LAVA_F32, interleaved=interleaved, scale=scale)
    ahead, back = lava.RotaryDesc(**make), lava.RotaryDesc(backward=True, **make)

    def turn(desc, t):
        out = torch.empty_like(t)
        lava.lava_rotary(desc, freqs.cuda(), pos, t, None, out, None)
        return out.double()

    dx = turn(back, grad)
    # each of N*H*d products is off by 2^-20 (|a| + |b|) s |g| at most; |a| + |b| sums to 2 |x|
    tol = 2.0 ** -20 * scale * 2 * float((x.abs().max() * grad.abs().max()) * x.numel())
    assert abs(float((turn(ahead, x) * grad.double()).sum() - (x.double() * dx).sum())) <= 2 * tol
    eps = 2.0 ** -6
    diff = (turn(ahead, x + eps * step) - turn(ahead, x - eps * step)) / (2 * eps)
    slope, along = float((diff * grad.double()).sum()), float((step.double() * dx).sum())
    # the outputs' errors over 2 eps, two of them, and the rounding of x + eps step (2^-24 of |x| + eps |step|)
    size = float((x.abs().max() + eps * step.abs().max()) * grad.abs().max() * x.numel())
    assert abs(slope - along) <= (2 * 2.0 ** -20 + 2 * 2.0 ** -23) * scale * 2 * size / (2 * eps) + tol


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 128), (torch.bfloat16, 64), (torch.float32, 64)])
@pytest.mark.parametrize("B,T,Hq,H,r", [(1, 1, 32, 8, 64), (3, 1, 4, 4, 64), (7, 5, 28, 4, 16), (70, 1, 8, 1, 0)])
def test_append_writes_the_places_and_nothing_else(dtype, d, B, T, Hq, H, r):
    _check.dtype = dtype
    g = torch.Generator().manual_seed(B)
    L, layer, ps, N = 3, 1, 16, B * T
    n_pages = L * B * H * 2
    qkv = torch.randn((N, (Hq + 2 * H) * d), generator=g).to(dtype).cuda()
    q, k, v = (qkv[:, a * d: b * d].view(N, b - a, d) for a, b in ((0, Hq), (Hq, Hq + H), (Hq + H, Hq + 2 * H)))
    cache = lava.CacheDesc(n_layers=L, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, page_rows=ps, max_pages=4,
                           n_pages=n_pages, dtype=CODE[dtype])
    slots = torch.randperm(n_pages * ps, generator=g)[: L * N * H].view(L, B, T, H).int()
    slots[layer].view(-1)[:: 5] = -1
    slots[layer, B - 1, 0, H - 1] = n_pages * ps                  # behind the pool: not written
    pos = torch.randint(0, 100000, (N,), generator=g).int()
    freqs = lava.lava_rotary_freqs(r)[0] if r else torch.zeros(0, dtype=torch.float64)
    desc = lava.RotaryDesc(head_dim=d, rotary_dim=r, dtype=CODE[dtype])
    q_out = torch.empty((N, Hq, d), dtype=dtype, device="cuda")
    room = [torch.full((n_pages + 2, ps, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    pools = [x[1: n_pages + 1] for x in room]
    lava.lava_rotary_append(desc, freqs.cuda(), cache, layer, pos.cuda(), q, k, v, q_out, slots.cuda(), *pools)
    _check(q_out, q, pos.numpy(), freqs.numpy(), False, False, 1.0)
    turned = torch.empty((N, H, d), dtype=dtype, device="cuda")
    lava.lava_rotary(desc, freqs.cuda(), pos.cuda(), None, k, None, turned)
    at = slots[layer].view(-1).long()
    there = (at >= 0) & (at < n_pages * ps)
    for pool, rows in zip(room, (turned, v)):
        want = torch.full(((n_pages + 2) * ps, d), 7.0, dtype=dtype)
        want[at[there] + ps] = rows.reshape(-1, d).cpu()[there]
        assert torch.equal(pool.cpu().view(-1, d), want)

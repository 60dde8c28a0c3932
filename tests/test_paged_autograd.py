"""The paged calls write through addresses, outside autograd: what it follows is refused, and what it saved counts as
written to."""
import pytest
import torch

import paper_2509_09754_b200 as lava

ROT = lava.RotaryDesc(head_dim=64, rotary_dim=64, dtype=lava.LAVA_F32)


def _inputs(device):
    freqs = lava.lava_rotary_freqs(64)[0].to(device)
    return freqs, torch.arange(3, dtype=torch.int32, device=device), torch.randn((3, 8, 64), device=device)


@pytest.mark.gpu
def test_tensors_that_require_a_gradient_are_refused():
    freqs, pos, x = _inputs("cuda")
    w = x.clone().requires_grad_()
    for q, out in ((w, torch.empty_like(x)), (x, w), (w, w), (w * 2, x), (x, w * 2)):
        for args in ((q, None, out, None), (None, q, None, out)):
            with pytest.raises(lava.LavaError, match="requires a gradient") as e:
                lava.lava_rotary(ROT, freqs, pos, *args)
            assert e.value.status == 1
            with torch.no_grad():
                lava.lava_rotary(ROT, freqs, pos, *args)


class _Turn(torch.autograd.Function):
    """How a model in training turns: forward, and the gradient with the transpose."""

    @staticmethod
    def forward(ctx, x, freqs, pos):
        ctx.freqs, ctx.pos = freqs, pos
        out = torch.empty_like(x)
        lava.lava_rotary(ROT, freqs, pos, x, None, out, None)
        return out

    @staticmethod
    def backward(ctx, g):
        back = lava.RotaryDesc(head_dim=64, rotary_dim=64, dtype=lava.LAVA_F32, backward=True)
        out = torch.empty_like(g)
        lava.lava_rotary(back, ctx.freqs, ctx.pos, g.contiguous(), None, out, None)
        return out, None, None


@pytest.mark.gpu
def test_a_function_of_its_own_follows_the_gradient():
    freqs, pos, x = _inputs("cuda")
    w = x.clone().requires_grad_()
    r = torch.randn_like(x)
    (_Turn.apply(w, freqs, pos) * r).sum().backward()
    angle = pos.double()[:, None] * freqs[None]
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = r.double()[..., :32], r.double()[..., 32:]
    want = torch.cat([a * c + b * s, b * c - a * s], -1)
    # (cosines and sines within 1.5 * 2^-24, two products and a sum: 4 * 2^-24 of |a| + |b|)
    size = (a.abs() + b.abs()).repeat(1, 1, 2)
    assert bool(((w.grad.double() - want).abs() <= 4 * 2.0 ** -24 * size).all())


@pytest.mark.gpu
def test_what_autograd_saved_counts_as_written_to():
    freqs, pos, x = _inputs("cuda")
    w = x.clone().requires_grad_()
    y = w.exp()                                              # its backward reads y
    with torch.no_grad():
        lava.lava_rotary(ROT, freqs, pos, y, None, y, None)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    before = x._version
    lava.lava_rotary(ROT, freqs, pos, x, None, x, None)
    assert x._version == before + 1
    with torch.inference_mode():                             # tensors that have no versions
        z = torch.randn_like(x)
        lava.lava_rotary(ROT, freqs, pos, z, None, z, None)
    lava.lava_rotary(ROT, freqs, pos, z, None, z, None)


@pytest.mark.gpu
def test_a_step_of_the_cache_marks_what_it_writes():
    cache = lava.PagedCache(lava.CacheDesc(n_layers=1, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64, max_pages=4, n_pages=16,
                                           page_rows=16, dtype=lava.LAVA_F32))
    freqs, pos, x = _inputs("cuda")
    cache.extend(torch.ones(3, dtype=torch.int32, device="cuda"))
    k, v = cache.k_pages._version, cache.v_pages._version
    w = x.clone().requires_grad_()                           # (inputs of a model that was not told no_grad are taken)
    q = cache.append(ROT, freqs, 0, pos, w, w[:, :2], w[:, :2])
    assert (cache.k_pages._version, cache.v_pages._version, q._version) == (k + 1, v + 1, 1)
    out, lse = torch.empty_like(q), torch.empty((3, 8), device="cuda")
    cache.attend(0, q, out, lse)
    assert not q.requires_grad and out._version == 1 and lse._version == 1
    with pytest.raises(lava.LavaError, match="out requires a gradient"):
        cache.attend(0, q, out.requires_grad_(), lse)
    with torch.no_grad():
        cache.attend(0, q, out, lse)


@pytest.mark.gpu
def test_an_admission_marks_the_pages_once():
    k = torch.randn((1, 2, 200, 64), device="cuda")
    q = torch.randn((1, 1, 8, 16, 64), device="cuda")
    plan = lava.EvictionPlan.create(lava.LayerDesc.for_tensors(q[0], k[0], k[0], 16, max_seqlen=200), 1, [128], [200],
                                    kv_dtype=torch.float32)
    cache = lava.PagedCache(lava.CacheDesc(n_layers=1, batch=1, n_q_heads=8, n_kv_heads=2, head_dim=64, max_pages=16, n_pages=16,
                                           page_rows=16, dtype=lava.LAVA_F32))
    before = cache.k_pages._version, cache.v_pages._version
    cache.evict(plan, q, k, k)
    assert (cache.k_pages._version, cache.v_pages._version) == (before[0] + 1, before[1] + 1)
    assert cache.poll_status() == 0 and int(cache.head_rows.sum()) == 128

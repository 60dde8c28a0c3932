"""The paged cache as a model uses it: prompts are evicted into pages, tokens are appended and attended, sequences
leave and others come, eagerly and in a captured step."""
import numpy as np
import pytest
import torch

import paper_2509_09754_b200 as lava
from lava_workloads import get_config
from oracle import paged_oracle as PO
from tests.parity_harness import make_plan, upload_model

pytestmark = pytest.mark.gpu


def _rows_of(cache, layer, b, g):
    """Keys and values that a head holds, read through its page table."""
    d = cache.desc
    n = int(cache.head_rows[layer, b, g])
    pages = cache.page_table[layer, b, g, : -(-n // d.page_rows)].long()
    return [x[pages].reshape(-1, d.head_dim)[:n].double().cpu().numpy() for x in (cache.k_pages, cache.v_pages)]


def _attended(cache, layer, q, out, lse):
    """out against attention over the rows that the pages hold.  bf16: 2^-8 of the output (its rounding) and 2^-11 of
    sum p |V|: logits are within 2^-14 (128 products of at most 5 x 5 in fp32, scaled), probabilities 2^-16; fp32: 2^-11."""
    d = cache.desc
    group = d.n_q_heads // d.n_kv_heads
    for b in range(d.batch):
        for g in range(d.n_kv_heads):
            k, v = _rows_of(cache, layer, b, g)
            qh = q[b, g * group: (g + 1) * group].double().cpu().numpy()
            want, want_lse = PO.attend(qh, k, v)
            mag = PO.attend(qh, k, np.abs(v))[0]
            got = out[b, g * group: (g + 1) * group].double().cpu().numpy()
            tol = 2.0 ** -11 * mag + (2.0 ** -8 * (np.abs(want) + mag * 2.0 ** -11) if q.dtype == torch.bfloat16 else 0.0)
            assert np.all(np.abs(got - want) <= tol), (layer, b, g)
            if len(k):
                assert np.all(np.abs(lse[b, g * group: (g + 1) * group].cpu().numpy() - want_lse) <= 2.0 ** -10)


@pytest.mark.parametrize("name,kw", [
    ("mistral7b_ragged", dict(seq_lens=(640, 901, 333), n_layers=2, budget_per_head=96)),
    ("gqa7_128k", dict(seq_lens=(700,), n_layers=2, budget_per_head=100)),
    ("tiny", dict(seq_lens=(300,), n_layers=2, budget_per_head=40)),
])
def test_prompts_tokens_and_releases(name, kw):
    cfg = get_config(name).scaled(**kw)
    q, k, v, cu = upload_model(cfg)
    plan = make_plan(cfg, q, k, v, cu)
    L, H, Hq, d, B = cfg.n_layers, cfg.n_kv_heads, cfg.n_q_heads, cfg.head_dim, cfg.batch + 2
    dt = k.dtype
    code = lava.LAVA_BF16 if dt == torch.bfloat16 else lava.LAVA_F32
    cache = lava.PagedCache(lava.CacheDesc(n_layers=L, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, dtype=code,
                                           page_rows=32, max_pages=40, n_pages=4000))
    lava.evict_model(plan, q, k, v)                              # the packed cache, to compare with
    cache.evict(plan, q, k, v, first_seq=1)
    assert cache.poll_status() == 0 and lava.lava_poll_status(plan.workspace) == 0
    hoff, roff = plan.head_offsets.cpu().numpy(), plan.layer_row_offset.cpu().numpy()
    for l in range(L):
        for b in range(cfg.batch):
            for g in range(H):
                r0 = int(roff[l * cfg.batch + b])
                lo, hi = r0 + int(hoff[l, b, g]), r0 + int(hoff[l, b, g + 1])
                kk, vv = _rows_of(cache, l, 1 + b, g)
                assert np.array_equal(kk, plan.k_out[lo:hi].double().cpu().numpy())
                assert np.array_equal(vv, plan.v_out[lo:hi].double().cpu().numpy())
    freqs = lava.lava_rotary_freqs(d, 500000.0)[0].cuda()
    rotary = lava.RotaryDesc(head_dim=d, rotary_dim=d, dtype=code)
    gen = torch.Generator().manual_seed(8)
    at = torch.tensor([0] + list(cfg.seq_lens) + [0])
    live = torch.tensor([0] + [1] * cfg.batch + [0])
    for step in range(5):
        add = live.clone()
        if step == 3:
            add[1] = -1                                          # the first prompt is done
            live[1] = 0
            live[0] = 1                                          # and a sequence without a prompt begins
        before = cache.head_rows.clone()
        cache.extend(add.int().cuda())
        assert cache.poll_status() == 0
        pos = at.int().cuda()
        for l in range(L):
            qkv = torch.randn((B, (Hq + 2 * H) * d), generator=gen).to(dt).cuda()
            qn, kn, vn = (qkv[:, a * d: b * d].view(B, b - a, d) for a, b in ((0, Hq), (Hq, Hq + H), (Hq + H, Hq + 2 * H)))
            turned = cache.append(rotary, freqs, l, pos, qn, kn, vn)
            out, lse = cache.attend(l, turned)
            _attended(cache, l, turned, out, lse)
            k_turned = PO.rotate(kn.double().cpu().numpy(), at.numpy(), freqs.cpu().numpy())
            for b in range(B):
                for g in range(H):
                    n = int(cache.head_rows[l, b, g])
                    assert n == (0 if add[b] < 0 else int(before[l, b, g]) + int(add[b]))
                    if add[b] > 0:                               # the last row is the new one
                        kk, vv = _rows_of(cache, l, b, g)
                        assert np.array_equal(vv[-1], vn[b, g].double().cpu().numpy())
                        assert np.all(np.abs(kk[-1] - k_turned[b, g]) <= 2.0 ** -8 * np.abs(k_turned[b, g]) + 2.0 ** -16)
        at += add.clamp(min=0)
    used = int((-(-cache.head_rows // 32)).sum())
    assert cache.free_page_count() == 4000 - used


def test_a_captured_step_serves_every_token():
    """extend, append and attend of all layers in one graph, replayed; the same steps eagerly give the same bits."""
    L, B, Hq, H, d = 3, 4, 8, 2, 64
    desc = lava.CacheDesc(n_layers=L, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, page_rows=16, max_pages=8, n_pages=150)
    rotary, freqs = lava.RotaryDesc(head_dim=d, rotary_dim=32), lava.lava_rotary_freqs(32)[0].cuda()
    gen = torch.Generator().manual_seed(9)
    steps = 40
    qkv = torch.randn((steps, L, B, (Hq + 2 * H) * d), generator=gen).bfloat16().cuda()
    adds = torch.randint(0, 2, (steps, B), generator=gen).int()
    adds[25, 1] = -1
    adds = adds.cuda()
    qkv_in, add_in, pos_in = torch.empty_like(qkv[0]), torch.empty_like(adds[0]), torch.zeros(B, dtype=torch.int32, device="cuda")

    def step(cache, outs):
        cache.extend(add_in)
        for l in range(L):
            x = qkv_in[l]
            qn, kn, vn = (x[:, a * d: b * d].view(B, b - a, d) for a, b in ((0, Hq), (Hq, Hq + H), (Hq + H, Hq + 2 * H)))
            turned = cache.append(rotary, freqs, l, pos_in, qn, kn, vn)
            out, _ = cache.attend(l, turned)
            outs[l].copy_(out)

    results = []
    for captured in (False, True):
        cache = lava.PagedCache(desc)
        outs = torch.zeros((L, B, Hq, d), dtype=torch.bfloat16, device="cuda")
        add_in.zero_()
        pos_in.zero_()
        qkv_in.copy_(qkv[0])
        step(cache, outs)                                        # a step that adds nothing
        graph = None
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(cache, outs)
        got = []
        for i in range(steps):
            qkv_in.copy_(qkv[i])
            add_in.copy_(adds[i])
            graph.replay() if captured else step(cache, outs)
            got.append(outs.clone())
            pos_in.add_(add_in.clamp(min=0))
        assert cache.poll_status() == 0
        turned = qkv[0, 0][:, : Hq * d].view(B, Hq, d).contiguous()
        _attended(cache, L - 1, turned, *cache.attend(L - 1, turned))
        results.append(torch.stack(got))
    assert torch.equal(results[0], results[1])


def test_a_prompt_that_finds_no_pages_leaves_the_cache_as_it_was():
    cfg = get_config("tiny").scaled(seq_lens=(200,), n_layers=1, budget_per_head=64)
    q, k, v, cu = upload_model(cfg)
    plan = make_plan(cfg, q, k, v, cu)
    H, d = cfg.n_kv_heads, cfg.head_dim
    cache = lava.PagedCache(lava.CacheDesc(n_layers=1, batch=2, n_q_heads=cfg.n_q_heads, n_kv_heads=H, head_dim=d,
                                           dtype=lava.LAVA_F32, page_rows=16, max_pages=20, n_pages=10))
    cache.evict(plan, q, k, v, first_seq=0)                      # 128 rows, 9 pages or so
    assert cache.poll_status() == 0
    rows, k0 = cache.head_rows.clone(), cache.k_pages.clone()
    cache.evict(plan, q, k, v, first_seq=1)
    assert cache.poll_status() == lava.LAVA_DEV_PAGES_EXHAUSTED
    assert torch.equal(cache.head_rows, rows) and torch.equal(cache.k_pages.view(torch.int32), k0.view(torch.int32))
    cache.extend(torch.tensor([-1, 0], dtype=torch.int32, device="cuda"))
    cache.evict(plan, q, k, v, first_seq=1)
    assert cache.poll_status() == 0 and int(cache.head_rows[0, 1].sum()) == 128


def _cache_of(cfg, batch, dt, **kw):
    return lava.PagedCache(lava.CacheDesc(n_layers=cfg.n_layers, batch=batch, n_q_heads=cfg.n_q_heads,
                                          n_kv_heads=cfg.n_kv_heads, head_dim=cfg.head_dim,
                                          dtype=lava.LAVA_BF16 if dt == torch.bfloat16 else lava.LAVA_F32,
                                          **dict(dict(page_rows=32, max_pages=40, n_pages=4000), **kw)))


@pytest.mark.parametrize("name", ["mistral7b_ragged", "tiny"])
def test_a_batch_with_a_prompt_shorter_than_the_window_does_not_enter(name):
    """Nothing of such a batch is scored or selected, and the plan still has the offsets of the batch before."""
    cfg = get_config(name).scaled(seq_lens=(300, 333), n_layers=2, budget_per_head=40)
    q, k, v, cu = upload_model(cfg)
    plan = make_plan(cfg, q, k, v, cu)
    cache = _cache_of(cfg, 4, k.dtype)
    cache.evict(plan, q, k, v)
    # (40 entries per head are less than the one window: LAVA_DEV_BUDGET_INFEASIBLE says that they were clamped)
    assert lava.lava_poll_status(plan.workspace) & ~2 == 0 and int(cache.head_rows[:, :2].min()) > 0
    rows, free, table = cache.head_rows.clone(), cache.free_page_count(), cache.page_table.clone()
    pages = cache.k_pages.clone()
    short = cfg.window // 2
    cu.copy_(torch.tensor([0, short, 333], dtype=torch.int32))
    cache.evict(plan, q, k, v, first_seq=2)
    assert lava.lava_poll_status(plan.workspace) & 1    # LAVA_DEV_SHORT_SEQUENCE
    assert torch.equal(cache.head_rows, rows) and cache.free_page_count() == free
    assert torch.equal(cache.page_table, table)
    # (untouched memory may hold NaN: compared as bits)
    assert torch.equal(cache.k_pages.view(torch.uint8), pages.view(torch.uint8))


def test_a_stream_of_its_own():
    """All of a cache's work on a stream that is not the current one, which allocates and writes meanwhile: what the
    calls allocate belongs to their stream."""
    cfg = get_config("mistral7b_ragged").scaled(seq_lens=(640, 901), n_layers=2, budget_per_head=96)
    q, k, v, cu = upload_model(cfg)
    freqs = lava.lava_rotary_freqs(cfg.head_dim, 10000.0)[0].cuda()
    rotary = lava.RotaryDesc(head_dim=cfg.head_dim, rotary_dim=cfg.head_dim)
    gen = torch.Generator().manual_seed(5)
    new = {n: torch.randn((2, h, cfg.head_dim), generator=gen).bfloat16().cuda()
           for n, h in (("q", cfg.n_q_heads), ("k", cfg.n_kv_heads), ("v", cfg.n_kv_heads))}
    at, add = torch.tensor([640, 901], dtype=torch.int32).cuda(), torch.ones(2, dtype=torch.int32).cuda()
    got = []
    for own in (False, True):
        plan = make_plan(cfg, q, k, v, cu)
        cache = _cache_of(cfg, 2, k.dtype)
        cache.k_pages.zero_()
        stream = torch.cuda.Stream() if own else None
        torch.cuda.synchronize()
        cache.evict(plan, q, k, v, stream=stream)
        junk = [torch.full((2, 2, cfg.n_kv_heads), 1 << 30, dtype=torch.int32, device="cuda") for _ in range(8)]
        cache.extend(add, stream=stream)
        outs = []
        for l in range(2):
            turned = cache.append(rotary, freqs, l, at, new["q"], new["k"], new["v"], stream=stream)
            outs.append((turned, *cache.attend(l, turned, stream=stream)))
            junk.append(torch.full_like(new["q"], 7.0))
        torch.cuda.synchronize()
        assert cache.poll_status() == 0 and len(junk) == 10
        got.append([x.clone() for o in outs for x in o] + [cache.head_rows, cache.page_table, cache.k_pages])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_strides_that_desc_does_not_name_are_refused():
    cfg = get_config("tiny").scaled(seq_lens=(300,), n_layers=2, budget_per_head=40)
    q, k, v, cu = upload_model(cfg)
    plan = make_plan(cfg, q, k, v, cu)
    cache = _cache_of(cfg, 1, k.dtype)
    cache.evict(plan, q, k, v)
    first_row = torch.zeros((2, 1, cfg.n_kv_heads), dtype=torch.int32, device="cuda")
    wide = torch.zeros((*k.shape[:3], 2 * k.shape[3]), dtype=k.dtype, device="cuda")[..., : k.shape[3]]
    for kk, vv in ((wide, v), (k, wide), (k[:, :, :1].expand(k.shape), v), (k[:1].expand(k.shape), v),
                   (k, v[:, :1].expand(v.shape))):
        with pytest.raises(lava.LavaError) as e:
            lava.lava_compact_kv_pages(plan.desc, cache.desc, 0, kk, vv, k.stride(0), v.stride(0), plan.keep_idx,
                                       plan.head_offsets, first_row, cache.page_table, cache.k_pages, cache.v_pages)
        assert e.value.status == 1 and "strides" in str(e.value)

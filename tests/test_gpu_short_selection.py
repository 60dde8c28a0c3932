"""A batch with a sequence shorter than the window: nothing is selected, and head_offsets say so whatever a batch before
left in them, so that neither the paged cache nor anything else takes those rows for this batch's."""
import pytest
import torch

import paper_2509_09754_b200 as lava
from lava_workloads import get_config
from tests.parity_harness import make_plan, upload_model

pytestmark = pytest.mark.gpu


def _model(name, flags=0):
    cfg = get_config(name).scaled(seq_lens=(300, 333), n_layers=2, budget_per_head=40)
    q, k, v, cu = upload_model(cfg)
    plan = make_plan(cfg, q, k, v, cu)
    plan.desc.flags |= flags
    return cfg, q, k, v, cu, plan


@pytest.mark.parametrize("name", ["mistral7b_ragged", "tiny"])
@pytest.mark.parametrize("evict", [lava.evict_model, lava.evict_scores])
def test_an_admission_after_a_short_batch_takes_no_rows(name, evict):
    cfg, q, k, v, cu, plan = _model(name)
    cache = lava.PagedCache(lava.CacheDesc(
        n_layers=2, batch=4, n_q_heads=cfg.n_q_heads, n_kv_heads=cfg.n_kv_heads, head_dim=cfg.head_dim, page_rows=32,
        max_pages=40, n_pages=4000, dtype=lava.LAVA_BF16 if k.dtype == torch.bfloat16 else lava.LAVA_F32))
    evict(plan, q, k, v)
    cache.admit(plan, k, v)
    assert lava.lava_poll_status(plan.workspace) & 1 == 0 and int(cache.head_rows[:, :2].min()) > 0
    rows, free, table = cache.head_rows.clone(), cache.free_page_count(), cache.page_table.clone()
    cu.copy_(torch.tensor([0, cfg.window // 2, 333], dtype=torch.int32))
    evict(plan, q, k, v)
    cache.admit(plan, k, v, first_seq=2)
    assert lava.lava_poll_status(plan.workspace) & 1                 # LAVA_DEV_SHORT_SEQUENCE
    assert cache.poll_status() == 0
    assert torch.equal(cache.head_rows, rows) and cache.free_page_count() == free
    assert torch.equal(cache.page_table, table)


@pytest.mark.parametrize("flags", [0, lava.LAVA_FLAG_PER_HEAD_TOPK])
def test_head_offsets_of_a_short_batch_are_zeros(flags):
    cfg, q, k, v, cu, plan = _model("mistral7b_ragged", flags)
    lava.evict_scores(plan, q, k, v)
    assert lava.lava_poll_status(plan.workspace) & 1 == 0 and int(plan.head_offsets[..., -1].min()) > 0
    cu.copy_(torch.tensor([0, cfg.window // 2, 333], dtype=torch.int32))
    keep = plan.keep_idx.clone()
    lava.evict_scores(plan, q, k, v)
    assert lava.lava_poll_status(plan.workspace) & 1
    assert bool((plan.head_offsets == 0).all()) and torch.equal(plan.keep_idx, keep)


def test_head_offsets_of_a_short_batch_over_shards_are_zeros():
    H, w, L, lens = 2, 32, 2, (300, 333)
    cu = torch.tensor([0, w // 2, 633], dtype=torch.int32, device="cuda")
    desc = lava.LayerDesc(n_q_heads=H, n_kv_heads=H, head_dim=128, window=w, batch=2, max_seqlen=333, cu_seqlens=cu,
                          total_tokens=sum(lens), k_stride_head=633 * 128, k_stride_tok=128, v_stride_head=633 * 128,
                          v_stride_tok=128)
    scores = torch.rand((L, desc.total_scores), device="cuda")
    state = torch.zeros(lava.lava_select_shard_bytes(desc, L), dtype=torch.uint8, device="cuda")
    keep = torch.full((L, desc.total_scores), -7, dtype=torch.int32, device="cuda")
    hoff = torch.full((L, 2, H + 1), 50, dtype=torch.int32, device="cuda")
    roff = torch.full((2 * L + 1,), 50, dtype=torch.int64, device="cuda")
    before = torch.zeros(2 * L, dtype=torch.int64, device="cuda")
    lava.lava_select_shard_begin(desc, L, H, torch.full((L, 2), 100, dtype=torch.int64, device="cuda"), state)
    for p in range(3):
        lava.lava_select_shard_hist(desc, L, scores, p, state)
        lava.lava_select_shard_step(desc, L, p, state)
    lava.lava_select_shard_count(desc, L, scores, state)
    lava.lava_select_shard_emit(desc, L, scores, before, keep, hoff, roff, state)
    assert bool((hoff == 0).all()) and bool((roff == 0).all()) and bool((keep == -7).all())

"""A plan's packed cache holds what the budgets make of its totals: a total below one window per head and layer is
raised to that (LAVA_DEV_BUDGET_INFEASIBLE), and so many rows are written."""
import pytest
import torch

import paper_2509_09754_b200 as lava


@pytest.mark.parametrize("budgets", [[0, 0], [640, 640], [2 * 8 * 64, 5000], [100, 10 ** 5], [2 * 8 * 64 + 1, 1]])
def test_a_plan_has_room_for_the_least_budget(budgets):
    L, H, w, lens = 2, 8, 64, (300, 333)
    total = sum(lens)
    cu = torch.tensor([0, 300, 633], dtype=torch.int32)
    desc = lava.LayerDesc(n_q_heads=4 * H, n_kv_heads=H, head_dim=128, window=w, batch=2, max_seqlen=333,
                          cu_seqlens=cu, total_tokens=total, k_stride_head=total * 128, k_stride_tok=128, v_stride_head=total * 128,
                          v_stride_tok=128)
    plan = lava.EvictionPlan.create(desc, L, budgets, lens, device="cpu")
    least = L * H * w
    in_force = [min(max(b, least), L * H * n) for b, n in zip(budgets, lens)]   # what the budgets' kernel clamps to
    assert plan.k_out.shape == plan.v_out.shape and plan.k_out.shape[0] >= sum(in_force)
    if all(b >= least for b in budgets):
        assert plan.k_out.shape[0] == sum(budgets)                              # as it was
    assert plan.total_budget.tolist() == budgets

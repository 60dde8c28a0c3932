"""Scales and caps whose products leave fp32 are refused: a logit of 0 would be 0 * infinity."""
import pytest

import paper_2509_09754_b200 as lava


def _bytes(**kw):
    c = lava.CacheDesc(n_layers=1, batch=1, n_q_heads=4, n_kv_heads=1, head_dim=64, max_pages=4, n_pages=4, **kw)
    return lava.load_library().lava_cache_workspace_bytes(c._ref)


@pytest.mark.parametrize("kw", [
    dict(sm_scale=3e38),                          # * log2(e)
    dict(softcap=3e38), dict(sm_scale=1e5, softcap=3e38),
    dict(softcap=1e-40), dict(sm_scale=1e20, softcap=1e-20),   # scale / cap
    dict(softcap=2e37), dict(sm_scale=1e-30, softcap=1e10),    # a quotient with few bits, or none
])
def test_scales_whose_products_leave_fp32_are_refused(kw):
    assert _bytes(**kw) == 0 and "fp32" in lava.lava_last_error()


@pytest.mark.parametrize("kw", [
    dict(), dict(sm_scale=1e-30), dict(sm_scale=2e38), dict(softcap=1e4), dict(softcap=1e36), dict(softcap=1e-30),
    dict(sm_scale=1e20, softcap=1e38), dict(sm_scale=0.2, softcap=50.0),
])
def test_others_are_taken(kw):
    assert _bytes(**kw) > 0

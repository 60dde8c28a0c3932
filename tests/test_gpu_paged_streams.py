"""What PagedCache says of itself while its work is on another stream than the current one."""
import pytest
import torch

import paper_2509_09754_b200 as lava

pytestmark = pytest.mark.gpu

DESC = lava.CacheDesc(n_layers=1, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, max_pages=4, n_pages=64, page_rows=16)
LONG = 200_000_000                                            # cycles, about a tenth of a second


def test_free_pages_are_counted_after_what_other_streams_do():
    cache = lava.PagedCache(DESC)
    add = torch.ones(2, dtype=torch.int32, device="cuda")
    cache.extend(add)
    assert cache.free_page_count() == 60
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        torch.cuda._sleep(LONG)
    cache.extend(torch.full((2,), 16, dtype=torch.int32, device="cuda"), max_add=16, stream=stream)
    assert cache.free_page_count() == 56
    torch.cuda.synchronize()


def test_a_cache_is_ready_for_any_stream_when_it_is_made():
    lava.PagedCache(DESC)                                     # (what the first one loads)
    torch.cuda._sleep(LONG)
    cache = lava.PagedCache(DESC)
    assert torch.cuda.current_stream().query()
    stream = torch.cuda.Stream()
    add = torch.ones(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    cache.extend(add, stream=stream)
    q = torch.randn((2, 4, 64), device="cuda").bfloat16()
    torch.cuda.synchronize()
    cache.attend(0, q, stream=stream)
    assert cache.poll_status(stream) == 0 and cache.free_page_count() == 60

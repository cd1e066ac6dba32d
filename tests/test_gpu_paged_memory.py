"""Memory that a paged cache makes for itself, used by calls on other streams than the one that it was made on."""
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import build, queries

pytestmark = pytest.mark.gpu

BUSY = 200_000_000                                                   # cycles: a tenth of a second


@pytest.mark.parametrize("how", ["argument", "raw", "current"])
def test_memory_of_a_cache_is_not_given_away_while_another_stream_uses_it(how):
    cache, gen = build([300, 40], H=2, G=4, page_size=16)
    q = queries(cache, gen)
    own = Bn.PagedKV(cache.k_pages, cache.v_pages, cache.page_table, n_q_heads=8, weights=cache.weights)
    side = torch.cuda.Stream()
    cache.laser_kv_paged_attention(q)                                # the first call of a process loads the kernel, for longer than BUSY
    torch.cuda.synchronize()
    size, at = own.workspace.numel(), own.workspace.data_ptr()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        if how == "current":
            own.laser_kv_paged_attention(q)
    if how != "current":
        own.laser_kv_paged_attention(q, stream=side if how == "argument" else side.cuda_stream)
    own.close()
    del own
    taken = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not side.query()                                          # the call is still to run
    assert all(t.data_ptr() != at for t in taken)
    torch.cuda.synchronize()

"""Tables far wider than what their sequences hold: a server's are as wide as the longest context that it takes."""
import pytest
import torch

from paged_util import append_plain, build, check_attention, evict_plain, queries, same, snapshot

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,page_size,table,lens", [
    (8, 16, 131072, [2049, 2049, 100, 3000]),                         # clusters of several CTAs, most of them without an entry
    (2, 64, 400000, [2049, 0, 50]),
    (1, 64, 786432, [300, 5000]),                                     # clusters of sixteen
    (3, 8, 50000, [257] * 30),                                        # more clusters than the device holds at once
])
def test_eviction_goes_by_lengths(H, page_size, table, lens):
    cache, gen = build(lens, H=H, G=2, D=64, page_size=page_size, max_pages=table // page_size)
    for keep, anchors, recent in ((250, 4, 100), (200, 0, 0), (33, 33, 0)):
        want = evict_plain(snapshot(cache), page_size, keep, anchors, recent)
        cache.laser_kv_paged_evict(keep, anchors=anchors, recent=recent)
        cache.laser_kv_paged_poll_status()
        same(snapshot(cache), want)
    check_attention(cache, queries(cache, gen), accumulate=True)


def test_a_decoding_step():
    cache, gen = build([300, 7, 0, 260], H=4, G=4, page_size=16, max_pages=131072 // 16, spare=20)
    free = torch.arange(cache.cfg.n_pages, device="cuda")
    used = torch.zeros(cache.cfg.n_pages, dtype=torch.bool, device="cuda")
    used[cache.page_table[cache.page_table < cache.cfg.n_pages].long()] = True
    free = free[~used]
    for b, n in enumerate([300, 7, 0, 260]):                          # a page more for every sequence
        cache.page_table[b, -(-n // 16)] = free[b]
    for _ in range(3):
        k, v = (torch.randn(4, 4, 1, 128, generator=gen, device="cuda").bfloat16() for _ in range(2))
        want = append_plain(snapshot(cache), 16, *(x.view(torch.int16).cpu().numpy() for x in (k, v)), [1] * 4)
        cache.laser_kv_paged_append(k, v)
        same(snapshot(cache), want)
        check_attention(cache, queries(cache, gen), accumulate=True)
        want = evict_plain(snapshot(cache), 16, 256, 4, 50)
        cache.laser_kv_paged_evict(256, anchors=4, recent=50)
        cache.laser_kv_paged_poll_status()
        same(snapshot(cache), want)

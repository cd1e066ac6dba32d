"""Positions of a paged cache that its owner has not given: entries are protected by positions alone, and -1 is none."""
import numpy as np
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import evict_plain, rows, same, snapshot

pytestmark = pytest.mark.gpu


def _cache(held, seen, H=2, page_size=16, max_pages=13, seed=4):
    """A cache made around a filled pool, without positions."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = len(held)
    k, v = (torch.randn(n * max_pages, H, page_size, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(n * max_pages, generator=gen, device="cuda").to(torch.int32).view(n, max_pages)
    table[0, -1] = -1                                                # a page that is yet to come
    w = torch.rand(n * max_pages, H, page_size, generator=gen, device="cuda")
    state = torch.tensor([held, seen], dtype=torch.int32, device="cuda")
    return Bn.PagedKV(k, v, table, n_q_heads=H, weights=w, state=state), gen


def test_entries_of_a_cache_made_with_a_state_have_their_places_as_positions():
    cache, gen = _cache([190, 100, 0, 40], [190, 100, 0, 40])
    for b, n in enumerate([190, 100, 0, 40]):
        page, off = rows(cache, b, n)
        assert torch.equal(cache.pos[page, :, off], torch.arange(n, dtype=torch.int32, device="cuda")[:, None].expand(-1, 2))
    for keep, anchors, recent in ((90, 0, 0), (80, 4, 30), (30, 30, 0), (20, 0, 20)):
        want = evict_plain(snapshot(cache), 16, keep, anchors, recent)
        cache.laser_kv_paged_evict(keep, anchors=anchors, recent=recent)
        cache.laser_kv_paged_poll_status()
        same(snapshot(cache), want)


def test_a_length_set_by_hand_finds_positions_too():
    cache, gen = _cache([0, 0], [0, 0])
    cache.state.copy_(torch.tensor([[120, 60], [120, 60]], dtype=torch.int32))
    want = evict_plain(snapshot(cache), 16, 50, 3, 20)
    page, off = rows(cache, 0, 50)
    cache.laser_kv_paged_evict(50, anchors=3, recent=20)
    cache.laser_kv_paged_poll_status()
    same(snapshot(cache), want)
    assert (cache.pos[page, :, off] >= 100).any(0).all()             # the newest ones are there


def test_entries_without_a_position_go_by_their_weight_alone():
    """More tokens seen than entries held: nobody knows which ones these are. With tokens seen fewer than `recent`, as after an append
    that brings its positions, -1 is not one of the last ones either."""
    for seen in (500, 10):
        cache, gen = _cache([150, 100], [seen, 100])
        page, off = rows(cache, 0, 150)
        assert (cache.pos[page, :, off] == -1).all()
        before = snapshot(cache)
        cache.laser_kv_paged_evict(60, anchors=4, recent=40)
        cache.laser_kv_paged_poll_status()
        after = snapshot(cache)
        by_weight = dict(before, state=before["state"][:, [0]], table=before["table"][[0]])
        by_weight["pos"] = np.where(by_weight["pos"] == -1, 1 << 20, by_weight["pos"])       # neither first nor last
        by_weight["state"] = np.array([[150], [1 << 30]], dtype=np.int32)
        want = evict_plain({x: by_weight[x].copy() for x in by_weight}, 16, 60, 4, 40)
        p, o = (x[:60].cpu().numpy() for x in (page, off))
        for x in ("k", "v", "w"):
            assert np.array_equal(after[x][p, :, o].view(np.int16), want[x][p, :, o].view(np.int16)), x
        assert after["state"][0].tolist() == [60, 60]


def test_given_positions_are_left_alone():
    cache, gen = _cache([50, 20], [50, 20])
    pos = torch.randint(0, 1000, cache.pos.shape, generator=gen, device="cuda").to(torch.int32)
    kept = pos.clone()
    again = Bn.PagedKV(cache.k_pages, cache.v_pages, cache.page_table, n_q_heads=2, weights=cache.weights, pos=pos, state=cache.state)
    assert again.pos is pos and torch.equal(pos, kept)

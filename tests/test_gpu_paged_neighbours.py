"""A sequence of a paged cache whose length is wrong takes nothing from the others: not their entries, not their weights."""
import math

import numpy as np
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import attention64, build, evict_plain, queries, rows, same, snapshot

pytestmark = pytest.mark.gpu


def _status(cache):
    with pytest.raises(Bn.LaserKVError) as e:
        cache.laser_kv_paged_poll_status()
    return e.value.status


def _evicted(before, seqs, page_size, keep, anchors=0, recent=0):
    """The snapshot after an eviction of the sequences `seqs` alone."""
    want = dict(before, **{x: before[x].copy() for x in ("k", "v", "w", "pos", "state")})
    state = want["state"][:, seqs].copy()
    evict_plain(dict(want, state=state, table=before["table"][seqs]), page_size, keep, anchors, recent)
    want["state"][:, seqs] = state
    return want


@pytest.mark.parametrize("where", [0, 1, 2])
@pytest.mark.parametrize("length", [1 << 30, (1 << 31) - 1, 161, -1, -(1 << 31)])
def test_eviction_beside_a_length_out_of_range(length, where):
    """The pool is full, so that the list of moves has room for what its sequences can need and no more."""
    lens = [150, 150, 150]
    lens[where] = 80
    cache, gen = build(lens, H=2, G=1, page_size=16, max_pages=10, spare=0)
    cache.lens[where] = length
    before = snapshot(cache)
    cache.laser_kv_paged_evict(75, anchors=3, recent=20)
    assert _status(cache) == Bn.ERR_INVALID_ARG
    same(snapshot(cache), _evicted(before, [b for b in range(3) if b != where], 16, 75, 3, 20))


def test_a_sequence_whose_moves_find_no_room_keeps_its_entries():
    """A length that the table could hold, but the pool does not: sequences behind it may have to wait, and lose nothing."""
    cache, gen = build([80, 150, 150], H=2, G=1, page_size=16, max_pages=10, spare=0)
    cache.lens[0] = 160
    cache.seen[0] = 160
    before = snapshot(cache)
    cache.laser_kv_paged_evict(75, anchors=3, recent=20)
    _status(cache)
    after = snapshot(cache)
    assert after["state"][0].tolist() == [75, 75, 150]
    want = _evicted(before, [1], 16, 75, 3, 20)
    for b in (1, 2):
        page = rows(cache, b, 150)[0].unique().cpu().numpy()
        for x in ("k", "v", "pos"):
            assert np.array_equal(after[x][page], want[x][page])
        assert np.array_equal(after["w"][page].view(np.int32), want["w"][page].view(np.int32))
    cache.lens[0] = 75
    cache.laser_kv_paged_evict(75, anchors=3, recent=20)
    cache.laser_kv_paged_poll_status()
    same(snapshot(cache), _evicted(after, [2], 16, 75, 3, 20))


@pytest.mark.parametrize("where", [0, 1, 2])
@pytest.mark.parametrize("length", [1 << 30, 6401, -1])
def test_weights_grow_beside_a_length_out_of_range(length, where):
    lens = [600, 600, 600]
    lens[where] = 64
    cache, gen = build(lens, H=2, G=4, page_size=16, max_pages=400, spare=0)
    q = queries(cache, gen)
    want, lse64, grow, t_out, t_lse, t_grow = attention64(cache, q)
    before, others = cache.weights.clone(), [b for b in range(3) if b != where]
    mine = rows(cache, where, 64)[0]
    cache.lens[where] = length
    lse = torch.empty(3, 8, device="cuda")
    out = cache.laser_kv_paged_attention(q, accumulate=True, lse=lse)
    assert _status(cache) == Bn.ERR_INVALID_ARG
    assert ((out.double() - want).abs() <= t_out)[others].all() and ((lse.double() - lse64).abs() <= t_lse)[others].all()
    for x in (grow, t_grow):
        x[mine] = 0.0
    w = before.double() + grow
    assert ((cache.weights.double() - w).abs() <= t_grow + 2.0 ** -24 * w.abs()).all()
    # entries of no sequence: nobody's
    assert bool((out[where] == 0).all()) and bool((lse[where] == -math.inf).all())

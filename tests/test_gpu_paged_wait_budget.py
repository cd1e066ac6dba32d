"""The give-up path of the paged attention's waits, reached on purpose, as in test_gpu_wait_budget: a budget of a poll runs out although
nothing is wrong. Tiles on their way are still waited for with the full budget; the host sees LASER_KV_ERR_TIMEOUT, no weight has
grown, and the next ordinary call gives what it gives on a cache that never saw a timeout."""
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import attention64, build, check_attention, evict_plain, queries, same, snapshot

pytestmark = pytest.mark.gpu


def _timed_out(cache):
    with pytest.raises(Bn.LaserKVError) as e:
        cache.laser_kv_paged_poll_status()
    assert e.value.status == Bn.ERR_TIMEOUT
    cache.laser_kv_paged_poll_status()                                # cleared by the read


def _soil(cache):
    """Scores, normalisers and lists of a workspace that no call has used yet hold anything; the counters at its start are zero."""
    c = cache.cfg
    wide = 8 if c.n_q_heads // c.n_kv_heads <= 8 else 16
    up = lambda x: -(-x // 256) * 256
    counters = 256 + up(4 * c.n_seqs) + up(4 * c.n_seqs * c.n_kv_heads * -(-(c.n_q_heads // c.n_kv_heads) // wide))
    rest = cache.workspace[counters:]
    rest.random_(0, 256)


@pytest.mark.parametrize("dtype,D,G,H,page_size,lens", [
    ("bf16", 128, 4, 4, 16, [20000, 70, 0, 9000]),                    # rings that go round, parts read directly
    ("fp16", 64, 20, 1, 64, [70000]),                                 # a join of many parts, two blocks of heads
    ("bf16", 256, 9, 2, 8, [5, 3000, 129]),
    ("fp16", 128, 2, 8, 32, [200] * 40),                              # nothing is split
])
def test_waits_that_run_out_are_reported_and_add_no_weight(dtype, D, G, H, page_size, lens):
    cache, gen = build(lens, H=H, G=G, D=D, page_size=page_size, dtype=dtype, seed=6)
    fresh, _ = build(lens, H=H, G=G, D=D, page_size=page_size, dtype=dtype, seed=6)
    q = queries(cache, gen)
    before = snapshot(cache)
    _soil(cache)
    cache.laser_kv_paged_set_wait_budget(1)
    for accumulate in (True, False, True):                            # the first call of all, and later ones
        cache.laser_kv_paged_attention(q, accumulate=accumulate)
        _timed_out(cache)
        same(snapshot(cache), before)
    cache.laser_kv_paged_set_wait_budget(0)
    for _ in range(2):
        lse = [torch.empty(len(lens), H * G, device="cuda") for _ in range(2)]
        a, b = (c.laser_kv_paged_attention(q, accumulate=True, lse=z) for c, z in zip((cache, fresh), lse))
        assert torch.equal(a, b) and torch.equal(*lse) and torch.equal(cache.weights, fresh.weights)
    cache.laser_kv_paged_poll_status()
    # stale scores of good calls lie in the workspace now
    cache.laser_kv_paged_set_wait_budget(1)
    before = snapshot(cache)
    cache.laser_kv_paged_attention(q, accumulate=True)
    _timed_out(cache)
    same(snapshot(cache), before)
    cache.laser_kv_paged_set_wait_budget(0)
    check_attention(cache, q, accumulate=True)


def test_no_weight_grows_until_the_timeout_is_reported():
    """What the sums of a call that gave up would add is not known; a bad page that was recorded first hides the code, not this."""
    cache, gen = build([500, 300], H=2, G=4, page_size=16, max_pages=40)
    q = queries(cache, gen)
    cache.laser_kv_paged_attention(q, accumulate=True)
    page, before = int(cache.page_table[0, 5]), snapshot(cache)
    for number in (page, -1):
        cache.laser_kv_paged_set_wait_budget(1)
        cache.page_table[0, 5] = number
        cache.laser_kv_paged_attention(q, accumulate=True)
        cache.page_table[0, 5] = page
        cache.laser_kv_paged_set_wait_budget(0)
        cache.laser_kv_paged_attention(q, accumulate=True)
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_poll_status()
        assert e.value.status in ((Bn.ERR_TIMEOUT,) if number == page else (Bn.ERR_TIMEOUT, Bn.ERR_INVALID_ARG))
        same(snapshot(cache), before)
    want, _, grow, t_out, _, t_grow = attention64(cache, q)
    out = cache.laser_kv_paged_attention(q, accumulate=True)
    cache.laser_kv_paged_poll_status()
    assert ((out.double() - want).abs() <= t_out).all()
    w = torch.from_numpy(before["w"]).cuda().double() + grow
    assert ((cache.weights.double() - w).abs() <= t_grow + 2.0 ** -24 * w.abs()).all()


def test_a_workspace_that_holds_anything():
    """Only its counters have to be zero between calls."""
    for dtype, G in (("bf16", 4), ("fp16", 17)):
        cache, gen = build([700, 64, 0, 3000], H=2, G=G, page_size=16, dtype=dtype)
        for _ in range(3):
            _soil(cache)
            check_attention(cache, queries(cache, gen), accumulate=True)
        _soil(cache)
        want = evict_plain(snapshot(cache), 16, 200, 4, 100)
        cache.laser_kv_paged_evict(200, anchors=4, recent=100)
        cache.laser_kv_paged_poll_status()
        same(snapshot(cache), want)


def test_a_budget_needs_a_cache():
    assert Bn.load().laser_kv_paged_set_wait_budget(None, 1) == Bn.ERR_INVALID_ARG

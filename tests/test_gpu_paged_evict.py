"""Eviction from a paged cache on the GPU: every byte of the pool against the definition."""
import math

import numpy as np
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import build, evict_plain, rows, same, snapshot

pytestmark = pytest.mark.gpu


def _evict(cache, keep, anchors=0, recent=0):
    want = evict_plain(snapshot(cache), cache.cfg.page_size, keep, anchors, recent)
    cache.laser_kv_paged_evict(keep, anchors=anchors, recent=recent)
    cache.laser_kv_paged_poll_status()
    same(snapshot(cache), want)


@pytest.mark.parametrize("lens,H,D,page_size,dtype,token_major,keep,anchors,recent", [
    ([2049] * 16, 8, 128, 16, "bf16", False, 2048, 4, 256),           # one entry out
    ([100, 64, 65, 0, 1, 63, 128], 2, 64, 8, "fp16", True, 64, 4, 16),
    ([5000], 1, 128, 64, "bf16", False, 1200, 10, 100),               # one cluster of several CTAs
    ([5000, 3000, 1100], 2, 256, 32, "fp16", True, 1024, 0, 512),
    ([777, 333], 3, 128, 16, "bf16", True, 1, 0, 0),
    ([777, 333], 3, 128, 16, "bf16", False, 0, 0, 0),                 # all of them
    ([777, 333], 3, 64, 16, "bf16", False, 332, 100, 232),            # nothing but protected entries stays
    ([600, 50], 1, 256, 128, "bf16", False, 599, 1, 1),
    ([40000, 39999], 8, 64, 64, "fp16", False, 20000, 1000, 5000),
    ([300] * 600, 1, 64, 16, "bf16", False, 200, 3, 50),              # more clusters than SMs
    ([5000, 4097], 2, 64, 4096, "fp16", True, 4096, 10, 100),
    ([1087, 1088, 3, 1024, 1025, 0], 5, 256, 32, "bf16", True, 1024, 16, 64),
    ([1089], 5, 256, 32, "bf16", True, 1024, 16, 64),
    ([500, 64, 70, 1000], 1, 64, 8, "fp16", False, 64, 3, 5),
])
def test_evict_against_the_definition(lens, H, D, page_size, dtype, token_major, keep, anchors, recent):
    cache, gen = build(lens, H=H, G=1, D=D, page_size=page_size, dtype=dtype, token_major=token_major)
    _evict(cache, keep, anchors, recent)
    _evict(cache, keep, anchors, recent)                              # nothing more to do
    if keep > 10:
        _evict(cache, keep - 7, anchors // 2, recent // 2)


@pytest.mark.parametrize("values", [
    [0.0], [0.0, -0.0], [1.0, 2.0], [math.nan, 0.0], [math.nan, -math.inf, -1.0], [math.inf, 1.0, -math.inf], [math.nan], [math.inf],
    [1.0, 1.0 + 2.0 ** -23], [1e-45, 2e-45, 0.0, -1e-45], [3.4e38, 1e-38, -3.4e38, 0.5]])
def test_ties_and_special_weights(values):
    """Few different weights: equal ones go by index, across warps and CTAs."""
    for lens, H, keep in (([3001, 2000], 2, 1500), ([130] * 40, 4, 100)):
        cache, gen = build(lens, H=H, G=1, D=64, page_size=8)
        pick = torch.randint(0, len(values), cache.weights.shape, generator=gen, device="cuda")
        cache.weights.copy_(torch.tensor(values, dtype=torch.float32, device="cuda")[pick])
        _evict(cache, keep, 5, 20)
        _evict(cache, keep // 2, 0, 0)
        _evict(cache, 1, 0, 0)
        _evict(cache, 0, 0, 0)


@pytest.mark.parametrize("lens,H", [([60000], 1), ([60000, 30000], 8), ([400000], 2), ([786432], 1)])   # the last is as long as a table may be
def test_heavy_tailed_weights(lens, H):
    """Weights over many octaves, some never attended to; clusters of up to sixteen CTAs."""
    cache, gen = build(lens, H=H, G=1, D=64, page_size=64, stale=None)
    w = torch.exp(3.0 * torch.randn(cache.weights.shape, generator=gen, device="cuda") - 6.0)
    w[torch.rand(w.shape, generator=gen, device="cuda") < 0.3] = 0.0
    cache.weights.copy_(w)
    _evict(cache, lens[0] // 3, 64, lens[0] // 10)


def test_positions_decide_what_is_protected():
    """Positions in no order, repeated ones (more protected entries than places), and tokens seen far ahead."""
    cache, gen = build([900, 500], H=3, G=1, D=64, page_size=16, seen=[5000, 1 << 30])
    pos = torch.randint(0, 5000, cache.pos.shape, generator=gen, device="cuda").to(torch.int32)
    cache.pos.copy_(pos)
    _evict(cache, 400, 200, 200)
    cache.pos.fill_(4999)
    cache.pos[:, 1] = 3
    cache.state[0, 0] = 400
    _evict(cache, 300, 100, 200)
    _evict(cache, 50, 4, 1)


@pytest.mark.parametrize("n_new,recent", [(1, 64), (13, 64), (64, 64)])
def test_steady_state_at_a_budget(n_new, recent):
    """Tokens in, as many entries out, many times over: the cache stays what the definition makes it, in one captured graph."""
    keep, H = 300, 2
    cache, gen = build([keep, 10, keep], H=H, G=1, D=128, page_size=16, max_pages=(keep + n_new + 15) // 16 + 1, whole_table=True,
                       seen=[1000, 10, keep])
    k, v = (torch.randn(3, H, n_new, 128, generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(3, H, n_new, generator=gen, device="cuda")

    def step():
        cache.laser_kv_paged_append(k, v, weights=w)
        cache.laser_kv_paged_evict(keep, anchors=4, recent=recent)

    from paged_util import append_plain
    want = snapshot(cache)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(30):
        k.normal_(generator=gen), v.normal_(generator=gen), w.uniform_(generator=gen)
        bits = [x.view(torch.int16).cpu().numpy() for x in (k, v)]
        want = evict_plain(append_plain(want, 16, *bits, [n_new] * 3, w.cpu().numpy()), 16, keep, 4, recent)
        graph.replay() if i % 2 else step()
    cache.laser_kv_paged_poll_status()
    same(snapshot(cache), want)


def test_bad_pages_and_lengths_are_reported_and_go_no_further():
    cache, gen = build([200, 150, 90], H=2, G=1, page_size=16, max_pages=16)
    for number in (-1, cache.cfg.n_pages, 1 << 30, -(1 << 31)):
        before = snapshot(cache)
        page = int(cache.page_table[1, 3])
        cache.page_table[1, 3] = number
        cache.laser_kv_paged_evict(100, anchors=4, recent=30)
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_poll_status()
        assert e.value.status == Bn.ERR_INVALID_ARG
        after = snapshot(cache)
        used = {b: rows(cache, b, n)[0].unique().cpu().numpy() for b, n in ((0, 200), (2, 90))}
        want = evict_plain(dict(before, state=before["state"][:, [0]], table=before["table"][[0]]), 16, 100, 4, 30)
        for x in ("k", "v", "w", "pos"):
            for b in used:
                a, c = (s[x][used[b]].view(np.int32) if s[x].dtype == np.float32 else s[x][used[b]] for s in (after, want))
                assert np.array_equal(a, c)
        assert after["state"][0].tolist() == [100, 100, 90]
        cache.page_table[1, 3] = page
        cache.lens.copy_(torch.tensor([200, 150, 90], dtype=torch.int32))
    cache.lens[1] = -1
    before = snapshot(cache)
    cache.laser_kv_paged_evict(250)
    with pytest.raises(Bn.LaserKVError) as e:
        cache.laser_kv_paged_poll_status()
    same(snapshot(cache), before)


def test_refusals():
    cache, gen = build([100], H=1, G=1, page_size=16)
    plain, _ = build([100], H=1, G=1, page_size=16, weights=False)
    before = snapshot(cache)
    for c, status, a in ((cache, Bn.ERR_INVALID_ARG, (-1,)), (cache, Bn.ERR_INVALID_ARG, (10, -1, 0)), (cache, Bn.ERR_INVALID_ARG, (10, 0, -1)),
                         (cache, Bn.ERR_INVALID_ARG, (10, 6, 5)), (cache, Bn.ERR_INVALID_ARG, (10, (1 << 31) - 1, (1 << 31) - 1)),
                         (plain, Bn.ERR_STATE, (10,))):
        with pytest.raises(Bn.LaserKVError) as e:
            c.laser_kv_paged_evict(*a)
        assert e.value.status == status
    cache.laser_kv_paged_evict(1 << 30)                               # more than the table holds
    same(snapshot(cache), before)
    pool = torch.zeros(1, 1, 8, 64, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(1, 786440 // 8, dtype=torch.int32, device="cuda")
    long = Bn.PagedKV(pool, pool.clone(), table, n_q_heads=1, weights=torch.zeros(1, 1, 8, device="cuda"))
    with pytest.raises(Bn.LaserKVError) as e:
        long.laser_kv_paged_evict(5)
    assert e.value.status == Bn.ERR_UNSUPPORTED

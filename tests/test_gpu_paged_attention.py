"""Attention of one token over a paged cache on the GPU, and the weights it accumulates, against the definition in 64 bits (the
bounds of the errors are derived in paged_util.attention64)."""
import math

import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import attention64, build, check_attention, queries, same, snapshot

pytestmark = pytest.mark.gpu

EDGES = [0, 1, 2, 7, 8, 9, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 1000]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,G,H,page_size,token_major,lens", [
    (128, 4, 8, 16, False, [1637]),                       # one sequence over all CTAs
    (128, 4, 2, 16, True, EDGES),
    (64, 8, 3, 8, False, EDGES),
    (256, 7, 2, 32, True, EDGES),
    (128, 16, 1, 64, False, EDGES),                       # two sets of eight heads
    (64, 12, 2, 128, True, EDGES),
    (128, 20, 1, 256, False, [0, 300, 1]),                # two readings of the cache
    (256, 9, 1, 8, False, [129, 5, 0]),
    (128, 1, 5, 32, False, [0, 0, 0]),                    # nothing at all
    (128, 3, 1, 16, True, [5000, 0, 1, 64]),
    (128, 4, 3, 16, False, [256, 255, 0, 193, 1]),        # no item is split: up to four tiles
    (64, 9, 2, 8, True, [257, 100, 256]),
    (64, 70, 1, 16, False, [100, 3000]),                  # five readings, more heads than a warp has lanes
    (128, 4, 1, 4096, False, [5000, 4096, 4095, 1]),
    (64, 2, 2, 1024, True, [1025, 2048, 70]),
])
def test_attention_against_64_bits(dtype, D, G, H, page_size, token_major, lens):
    cache, gen = build(lens, H=H, G=G, D=D, page_size=page_size, dtype=dtype, token_major=token_major)
    check_attention(cache, queries(cache, gen, 2.0, strided=token_major))
    check_attention(cache, queries(cache, gen, 2.0), out_dtype=cache.k_pages.dtype)
    for _ in range(2):                                    # weights on top of weights
        check_attention(cache, queries(cache, gen, 2.0), accumulate=True, out_dtype=cache.k_pages.dtype if G % 2 else None)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [31, 32, 33, 70, 1023, 1024, 1025, 2500])
def test_many_sequences(dtype, n):
    for most in (190, 257, 500):
        lens = [(i * 37) % most if i % 5 else 0 for i in range(n)]
        cache, gen = build(lens, H=2, G=2, D=64, page_size=16, dtype=dtype)
        check_attention(cache, queries(cache, gen), accumulate=True)


@pytest.mark.parametrize("D,H,lens", [(64, 1, [200001]), (128, 1, [70000, 3, 33333]), (256, 2, [20011])])
def test_long_caches_are_split_and_joined(D, H, lens):
    for dtype in ("bf16", "fp16"):
        for G in (4, 13):
            cache, gen = build(lens, H=H, G=G, D=D, page_size=64, dtype=dtype)
            check_attention(cache, queries(cache, gen, 3.0), accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("scale", [0.0, 0.01, 30.0])
def test_flat_and_steep_scores(dtype, scale):
    """Scores that hardly differ, and scores hundreds apart, the largest of them anywhere."""
    cache, gen = build([700, 65, 16], H=2, G=8, page_size=16, dtype=dtype)
    check_attention(cache, queries(cache, gen), softmax_scale=scale, scale=scale or None, accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_sink_beside_many_small_weights(dtype):
    """One entry of weight 1 whose value is zero, 60000 others of 2^-22: their share of the result is not lost."""
    cache, gen = build([60001], H=1, G=2, page_size=64, dtype=dtype, stale=None)
    page, off = int(cache.page_table[0, 3]), 5
    q = torch.zeros(1, 2, 128, device="cuda", dtype=cache.k_pages.dtype)
    q[..., 0] = 16.0
    cache.k_pages[..., 0] = 0.0
    cache.k_pages[page, 0, off, 0] = 15.25 * 128 ** 0.5 / 16          # 15.25 natural units above the others: 2^-22
    cache.v_pages[page, 0, off] = 0.0
    check_attention(cache, q, accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("stale", [math.nan, math.inf, -math.inf, None])
def test_rows_that_no_sequence_holds_do_not_matter(dtype, stale):
    """Tails of last pages hold NaN, infinities or other sequences' rows; stages of the ring hold earlier tiles."""
    for page_size in (8, 16, 64, 128):
        cache, gen = build([1, 70, 0, 129, 640, 33], H=2, G=4, page_size=page_size, dtype=dtype, stale=stale)
        check_attention(cache, queries(cache, gen), accumulate=True)


def test_infinities_and_nan_in_held_rows_stay_in_their_sequence():
    for bad in (math.nan, math.inf, -math.inf):
        cache, gen = build([100, 100, 40], H=2, G=2, page_size=16)
        q = queries(cache, gen)
        good = cache.laser_kv_paged_attention(q).clone()
        page = int(cache.page_table[1, 2])
        cache.v_pages[page, 1, 3] = bad
        out = cache.laser_kv_paged_attention(q)
        assert torch.equal(out[[0, 2]], good[[0, 2]]) and torch.equal(out[1, :2], good[1, :2])
        assert not torch.isfinite(out[1, 2:]).any()
        # a key whose scores are -inf or NaN: weight 0, or NaN for all of that sequence's head
        cache.v_pages[page, 1, 3] = 1.0
        cache.k_pages[page, 1, 3] = 0.0
        cache.k_pages[page, 1, 3, 0] = bad
        q[1, 2:, 0] = 1.0
        out = cache.laser_kv_paged_attention(q)
        assert torch.equal(out[[0, 2]], good[[0, 2]]) and torch.equal(out[1, :2], good[1, :2])
        if bad == -math.inf:
            assert torch.isfinite(out).all()
            keep = torch.tensor([i for i in range(100) if i != 35], device="cuda")
            p, off = cache.page_table[1, keep // 16].long(), keep % 16
            k, v = cache.k_pages[p, 1, off].double(), cache.v_pages[p, 1, off].double()
            want = torch.softmax(q[1, 2:].double() @ k.T * 128 ** -0.5, -1) @ v
            assert (out[1, 2:].double() - want).abs().max() < 1e-5
        else:
            assert torch.isnan(out[1, 2:]).all()
        cache.laser_kv_paged_poll_status()


def test_a_block_of_rows_at_minus_infinity():
    """Sixteen rows, a whole tile and all rows of a head at -inf: the others decide, or the result is NaN as the formula's is."""
    cache, gen = build([256], H=1, G=1, page_size=64)
    q = queries(cache, gen)
    q[..., 0] = 1.0
    for rows in (range(16, 32), range(64, 128), range(0, 250)):
        j = torch.tensor(list(rows), device="cuda")
        cache.k_pages[cache.page_table[0, j // 64].long(), 0, j % 64, 0] = -math.inf
        keep = [i for i in range(256) if bool(torch.isfinite(cache.k_pages[cache.page_table[0, i // 64].long(), 0, i % 64, 0]))]
        keep = torch.tensor(keep, device="cuda")
        p, off = cache.page_table[0, keep // 64].long(), keep % 64
        want = torch.softmax(q[0].double() @ cache.k_pages[p, 0, off].double().T * 128 ** -0.5, -1) @ cache.v_pages[p, 0, off].double()
        assert (cache.laser_kv_paged_attention(q)[0].double() - want).abs().max() < 1e-5
    cache.k_pages[..., 0] = -math.inf
    assert torch.isnan(cache.laser_kv_paged_attention(q)).all()


def test_results_repeat_and_weights_do_not_depend_on_timing():
    cache, gen = build([3000, 17, 0, 900, 4097], H=4, G=4, page_size=16)
    q, w0 = queries(cache, gen), cache.weights.clone()
    lse = torch.empty(5, 16, device="cuda")
    first = cache.laser_kv_paged_attention(q, accumulate=True, lse=lse).clone(), lse.clone(), cache.weights.clone()
    for _ in range(20):
        cache.weights.copy_(w0)
        out = cache.laser_kv_paged_attention(q, accumulate=True, lse=lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]) and torch.equal(cache.weights, first[2])


def test_a_captured_call_follows_lengths_tables_and_contents():
    cache, gen = build([900, 64, 5], H=2, G=4, page_size=16, max_pages=200, whole_table=True, stale=None)
    q = queries(cache, gen)
    out, lse = torch.empty(3, 8, 128, device="cuda"), torch.empty(3, 8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.laser_kv_paged_attention(q, accumulate=True, out=out, lse=lse)
    for lens in ([900, 64, 5], [0, 3200, 1], [0, 0, 0], [3199, 0, 700]):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        cache.page_table.copy_(cache.page_table.roll(1, 1))
        q.copy_(queries(cache, gen))
        want, lse64, grow, t_out, t_lse, t_grow = attention64(cache, q)
        w = cache.weights.double() + grow
        graph.replay()
        cache.laser_kv_paged_poll_status()
        assert ((out.double() - want).abs() <= t_out + 1e-30).all()
        assert ((cache.weights.double() - w).abs() <= t_grow + 2.0 ** -24 * w).all()


def test_two_caches_on_two_streams():
    pairs = []
    for seed in (1, 2):
        cache, gen = build([5000, 300, 2000], H=4, G=4, page_size=16, seed=seed)
        q = queries(cache, gen)
        pairs.append((cache, q, attention64(cache, q), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i, (cache, q, _, stream) in enumerate(pairs):
            with torch.cuda.stream(stream):
                outs[i].append(cache.laser_kv_paged_attention(q, accumulate=True))
    torch.cuda.synchronize()
    for i, (cache, q, (want, _, _, t_out, _, _), _) in enumerate(pairs):
        for out in outs[i]:
            assert ((out.double() - want).abs() <= t_out).all() and torch.equal(out, outs[i][0])


def test_keys_and_values_in_one_allocation():
    """[n_pages][2][H][page_size][d], one page's keys beside its values, at an offset into a larger buffer."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    both = torch.randn(40 * 2 * 3 * 16 * 128 + 8, generator=gen, device="cuda").half()[8:].view(40, 2, 3, 16, 128)
    table = torch.randperm(40, generator=gen, device="cuda").to(torch.int32).view(4, 10)
    state = torch.tensor([[160, 3, 0, 77]] * 2, dtype=torch.int32, device="cuda")
    cache = Bn.PagedKV(both[:, 0], both[:, 1], table, n_q_heads=15, weights=torch.zeros(40, 3, 16, device="cuda"), state=state)
    check_attention(cache, queries(cache, gen), accumulate=True)
    k, v = (torch.randn(4, 3, 1, 128, generator=gen, device="cuda").half() for _ in range(2))
    cache.lens[0] = 159
    cache.laser_kv_paged_append(k, v)
    check_attention(cache, queries(cache, gen), accumulate=True)
    cache.laser_kv_paged_evict(60)
    check_attention(cache, queries(cache, gen), out_dtype=torch.float16)


def test_queries_that_are_not_numbers_stay_in_their_head():
    for G, bad in ((4, math.nan), (16, math.inf), (7, -math.inf)):
        cache, gen = build([300, 70], H=2, G=G, page_size=16)
        q = queries(cache, gen)
        good = cache.laser_kv_paged_attention(q).clone()
        q[0, 1, 5] = bad
        out = cache.laser_kv_paged_attention(q)
        keep = torch.ones(2, 2 * G, dtype=torch.bool, device="cuda")
        keep[0, 1] = False
        assert torch.equal(out[keep], good[keep]) and torch.isnan(out[0, 1]).all()


def test_pages_that_sequences_share():
    """A common prefix, read-only: allowed without weights."""
    cache, gen = build([64, 100, 90], H=2, G=4, page_size=16, weights=False)
    cache.page_table[1, :4] = cache.page_table[0, :4]
    cache.page_table[2, :2] = cache.page_table[0, :2]
    check_attention(cache, queries(cache, gen), out_dtype=torch.bfloat16)


def test_bad_pages_and_lengths_are_reported_and_go_no_further():
    cache, gen = build([100, 70, 33], H=2, G=4, page_size=16, max_pages=8)
    q = queries(cache, gen)
    good = cache.laser_kv_paged_attention(q, accumulate=True).clone()
    bound = attention64(cache, q)[3]
    table, state = cache.page_table.clone(), cache.state.clone()

    def bad():
        out = cache.laser_kv_paged_attention(q, accumulate=True)
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_poll_status()
        assert e.value.status == Bn.ERR_INVALID_ARG
        assert ((out - good).abs() <= 2 * bound)[[0, 2]].all()       # the split may go by the other sequence's length
        cache.page_table.copy_(table)
        cache.state.copy_(state)
        assert torch.equal(cache.laser_kv_paged_attention(q), good)
        cache.laser_kv_paged_poll_status()

    for number in (-1, cache.cfg.n_pages, 1 << 30, -(1 << 31)):
        cache.page_table[1, 2] = number
        bad()
    cache.lens[1] = -5
    bad()
    cache.page_table[1] = torch.arange(8, device="cuda")
    cache.lens[1] = 129                                              # the table has room for 128
    bad()


def test_weights_of_shared_pages_are_refused_where_they_do_not_fit():
    """Sequences of a cache with weights that share pages can hold more entries than the pool: reported, nothing is written past the room."""
    cache, gen = build([1024] + [0] * 39, H=1, G=2, page_size=64, spare=0)
    cache.page_table[:] = cache.page_table[0]
    cache.lens[:] = 1024
    out = cache.laser_kv_paged_attention(queries(cache, gen), accumulate=True)
    assert torch.isfinite(out).all()
    with pytest.raises(Bn.LaserKVError) as e:
        cache.laser_kv_paged_poll_status()
    assert e.value.status == Bn.ERR_CAPACITY


def test_refusals():
    cache, gen = build([10, 3], H=2, G=2, page_size=8, weights=False)
    q = queries(cache, gen)

    def refused(status, *a, **kw):
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_attention(*a, **kw)
        assert e.value.status == status, e.value

    before = snapshot(cache)
    refused(Bn.ERR_STATE, q, accumulate=True)
    refused(Bn.ERR_INVALID_ARG, q.half())
    refused(Bn.ERR_INVALID_ARG, q[:1])
    refused(Bn.ERR_INVALID_ARG, q.cpu())
    refused(Bn.ERR_INVALID_ARG, q, softmax_scale=-1.0)
    refused(Bn.ERR_INVALID_ARG, q, softmax_scale=math.nan)
    refused(Bn.ERR_INVALID_ARG, q, softmax_scale=math.inf)
    refused(Bn.ERR_INVALID_ARG, q, out=torch.empty(2, 4, 128, dtype=torch.float16, device="cuda"))
    refused(Bn.ERR_INVALID_ARG, q, out=torch.empty(2, 128, 4, device="cuda").transpose(1, 2))
    refused(Bn.ERR_INVALID_ARG, q, lse=torch.empty(2, 4, dtype=torch.float64, device="cuda"))
    refused(Bn.ERR_ALIGNMENT, torch.zeros(2, 4, 132, dtype=torch.bfloat16, device="cuda")[..., :128])
    refused(Bn.ERR_ALIGNMENT, torch.zeros(1032, dtype=torch.bfloat16, device="cuda")[4:1028].view(2, 4, 128))
    refused(Bn.ERR_ALIGNMENT, q, out=torch.zeros(1026, device="cuda")[2:].view(2, 4, 128))
    same(snapshot(cache), before)

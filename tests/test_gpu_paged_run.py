"""The paged cache's calls together, and with the rest of the library: as a server would decode."""
import math

import numpy as np
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn
from paper_2602_02199_b200 import synth

from paged_util import append_plain, attention64, build, check_attention, evict_plain, queries, rows, same, snapshot
from parity_util import run_workload_layer

pytestmark = pytest.mark.gpu


def test_a_compacted_prompt_goes_to_pages_and_is_decoded_from_there():
    """Selected entries with their positions move from the compacted cache to pages: the same attention, then tokens on top."""
    w = synth.workload("tiny").with_(block_size=512, context_len=2048, batch=2, n_layers=1, lsh_tables=16)
    run = run_workload_layer(w, 0, n_blocks=4, debug=0)
    eng = run["engine"]
    k, v, pos, length = eng.laser_kv_cache_view(0)
    k, v, pos = k[:, :, :length], v[:, :, :length], pos[:, :, :length]
    H, G, page_size = w.n_kv_heads, w.group, 16
    max_pages = -(-(length + 40) // page_size)
    pool = [torch.empty(2 * max_pages, H, page_size, 128, dtype=torch.bfloat16, device="cuda").fill_(math.nan) for _ in range(2)]
    table = torch.randperm(2 * max_pages, device="cuda").to(torch.int32).view(2, max_pages)
    cache = Bn.PagedKV(*pool, table, n_q_heads=H * G, weights=torch.zeros(2 * max_pages, H, page_size, device="cuda"))
    cache.laser_kv_paged_append(k, v, pos=pos)
    cache.seen.fill_(2048)
    q = torch.from_numpy(run["Q"][:, :, 3].copy().view(np.int16)).cuda()
    want = eng.laser_kv_decode_attention(0, q)
    bound = attention64(cache, q.view(torch.bfloat16))[3]
    out = cache.laser_kv_paged_attention(q, accumulate=True)
    # both are rounded in fp32 alone: twice the bound that is derived for one of them
    assert ((out - want).abs() <= 2 * bound).all()
    cache.laser_kv_paged_poll_status()
    assert cache.lens.tolist() == [length] * 2 and cache.seen.tolist() == [2048] * 2
    for b in range(2):
        page, off = rows(cache, b, length)
        assert torch.equal(cache.pos[page, :, off].T, pos[b])
        assert ((cache.weights[page, :, off].sum(0) - G).abs() < 1e-3 * G).all()       # every query head gives 1
    gen = torch.Generator(device="cuda").manual_seed(1)
    for step in range(36):
        kn, vn = (torch.randn(2, H, 1, 128, generator=gen, device="cuda").bfloat16() for _ in range(2))
        cache.laser_kv_paged_append(kn, vn)
        q = queries(cache, gen)
        check_attention(cache, q, accumulate=True)
    page, off = rows(cache, 0, length + 36)
    assert cache.pos[page, 0, off][-36:].tolist() == list(range(2048, 2084))
    cache.laser_kv_paged_evict(length, anchors=4, recent=36)
    cache.laser_kv_paged_poll_status()
    assert cache.lens.tolist() == [length] * 2
    check_attention(cache, queries(cache, gen))


def test_greedy_prefill_from_window_scores():
    """Block by block: the window's scores are the new entries' weights, then the cache goes back to its budget."""
    w = synth.workload("tiny").with_(block_size=256, context_len=1024, batch=1, n_layers=1)
    S, H, keep, page_size = 256, w.n_kv_heads, 300, 32
    K, V = synth.kv_blocks(w, 0, 0, 0, 4)
    Q = torch.from_numpy(synth.q_window(w, 0, 0).view(np.int16)).cuda()[None]
    max_pages = -(-(keep + S) // page_size)
    pool = [torch.zeros(max_pages, H, page_size, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = Bn.PagedKV(*pool, torch.arange(max_pages, dtype=torch.int32, device="cuda")[None], n_q_heads=w.n_q_heads,
                       weights=torch.zeros(max_pages, H, page_size, device="cuda"))
    want = snapshot(cache)
    for t in range(4):
        k, v = (torch.from_numpy(x[:, t * S:(t + 1) * S].copy().view(np.int16)).cuda()[None] for x in (K, V))
        scores = Bn.laser_kv_window_scores(k, Q, S, 1)                # [1][H][1][S]
        cache.laser_kv_paged_append(k, v, weights=scores[:, :, 0])
        cache.laser_kv_paged_evict(keep, anchors=8, recent=64)
        want = evict_plain(append_plain(want, page_size, k.cpu().numpy(), v.cpu().numpy(), [S], scores[:, :, 0].cpu().numpy()), page_size, keep, 8, 64)
    cache.laser_kv_paged_poll_status()
    same(snapshot(cache), want)
    assert cache.lens.tolist() == [keep] and cache.seen.tolist() == [4 * S]


@pytest.mark.parametrize("dtype,D,G,captured", [("bf16", 128, 4, False), ("fp16", 64, 12, True), ("bf16", 256, 2, True)])
def test_decoding_at_a_budget(dtype, D, G, captured):
    """Append, attention with weights, eviction, over and over, without a synchronisation in between; then every step again with one,
    each call against its definition. The two runs end with the same bytes."""
    H, page_size, keep, steps = 2, 16, 200, 24
    lens = [200, 3, 0, 150]

    def make():
        return build(lens, H=H, G=G, D=D, page_size=page_size, dtype=dtype, max_pages=14, whole_table=True, seen=[900, 3, 0, 150], seed=5)

    ends = []
    for checked in (False, True):
        cache, gen = make()
        k, v = (torch.empty(4, H, 1, D, dtype=cache.k_pages.dtype, device="cuda") for _ in range(2))
        q, out = queries(cache, gen), torch.empty(4, H * G, D, device="cuda")

        def step():
            cache.laser_kv_paged_append(k, v)
            cache.laser_kv_paged_attention(q, accumulate=True, out=out)
            cache.laser_kv_paged_evict(keep, anchors=2, recent=50)

        graph = torch.cuda.CUDAGraph() if captured and not checked else None
        if graph:
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step()
        gen = torch.Generator(device="cuda").manual_seed(77)
        outs = []
        for i in range(steps):
            k.normal_(generator=gen), v.normal_(generator=gen), q.normal_(generator=gen)
            if graph:
                graph.replay()
            elif not checked:
                step()
            else:
                want = append_plain(snapshot(cache), page_size, *(x.view(torch.int16).cpu().numpy() for x in (k, v)), [1] * 4)
                cache.laser_kv_paged_append(k, v)
                same(snapshot(cache), want)
                out = check_attention(cache, q, accumulate=True)
                want = evict_plain(snapshot(cache), page_size, keep, 2, 50)
                cache.laser_kv_paged_evict(keep, anchors=2, recent=50)
                same(snapshot(cache), want)
            outs.append(out.clone())
        cache.laser_kv_paged_poll_status()
        ends.append((snapshot(cache), outs))
    same(ends[0][0], ends[1][0])
    assert all(torch.equal(a, b) for a, b in zip(ends[0][1], ends[1][1]))
    assert ends[0][0]["state"][0].tolist() == [200, 27, 24, 174]


def test_calls_right_behind_one_another_on_one_stream():
    """Queries, lengths and tables that the kernel just ahead writes; results that the next kernel reads."""
    cache, gen = build([400, 0, 37, 100], H=2, G=4, page_size=16, max_pages=30, whole_table=True, stale=None)
    stream = torch.cuda.Stream()
    big = torch.empty(64 << 20, device="cuda")
    lens = [[400, 0, 37, 100], [1, 480, 0, 250], [479, 16, 17, 0]]
    qs = [queries(cache, gen) for _ in lens]
    tables = [cache.page_table[torch.randperm(4, device="cuda")].contiguous() for _ in lens]
    dev_lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in lens]
    want = []
    for i in range(3):
        cache.lens.copy_(dev_lens[i]), cache.page_table.copy_(tables[i])
        want.append(attention64(cache, qs[i]))
    q, out = torch.empty_like(qs[0]), []
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for i in (0, 1, 2, 1, 0):
            big.fill_(i)                                             # the kernels ahead are still at work when the call is made
            cache.lens.copy_(dev_lens[i]), cache.page_table.copy_(tables[i]), q.copy_(qs[i])
            out.append((i, cache.laser_kv_paged_attention(q) * 1.0))
    stream.synchronize()
    for i, o in out:
        assert ((o.double() - want[i][0]).abs() <= want[i][3] + 1e-30).all()


def test_calls_take_no_device_memory():
    cache, gen = build([300, 200], H=2, G=4, page_size=16, max_pages=30, whole_table=True)
    q, out = queries(cache, gen), torch.empty(2, 8, 128, device="cuda")
    k, v = (torch.randn(2, 2, 1, 128, generator=gen, device="cuda").bfloat16() for _ in range(2))
    for i in range(3):
        cache.laser_kv_paged_append(k, v)
        cache.laser_kv_paged_attention(q, accumulate=True, out=out)
        cache.laser_kv_paged_evict(250, anchors=1, recent=5)
        torch.cuda.synchronize()
        if i == 0:
            count = lambda: torch.cuda.memory_stats().get("allocation.all.allocated", 0)
            before, free = count(), torch.cuda.mem_get_info()[0]
    assert count() == before and torch.cuda.mem_get_info()[0] >= free
    before = Bn.laser_kv_launch_count()
    cache.laser_kv_paged_append(k, v)
    cache.laser_kv_paged_attention(q, out=out)
    cache.laser_kv_paged_attention(q, accumulate=True, out=out)
    cache.laser_kv_paged_evict(250)
    assert Bn.laser_kv_launch_count() - before == 1 + 1 + 2 + 2


def test_a_pool_of_more_than_2_to_the_31_elements():
    """Pages at the end of a pool whose offsets need more than 32 bits, in bytes and in elements."""
    n_pages, H, page_size, D = 34000, 8, 64, 128                      # 2.2e9 elements, 4.5 GB a side
    pool = [torch.zeros(n_pages, H, page_size, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    weights = torch.zeros(n_pages, H, page_size, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(9)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2, n_pages - 4], [n_pages - 3, n_pages - 5, 0, 7]], dtype=torch.int32, device="cuda")
    cache = Bn.PagedKV(*pool, table, n_q_heads=4 * H, weights=weights)
    k, v = (torch.randn(2, H, 250, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(2, H, 250, generator=gen, device="cuda")
    cache.laser_kv_paged_append(k, v, weights=w)
    for b in range(2):
        page, off = rows(cache, b, 250)
        assert torch.equal(cache.k_pages[page, :, off].transpose(0, 1), k[b]) and torch.equal(cache.v_pages[page, :, off].transpose(0, 1), v[b])
        assert torch.equal(cache.weights[page, :, off].T, w[b])
    check_attention(cache, queries(cache, gen), accumulate=True)
    before = [x[table.long()].clone() for x in (cache.k_pages, cache.v_pages, cache.weights, cache.pos)]     # [2][4][H][page_size]...
    cache.laser_kv_paged_evict(100, anchors=4, recent=20)
    cache.laser_kv_paged_poll_status()
    s = dict(table=np.arange(8).reshape(2, 4), state=np.array([[250, 250], [250, 250]], dtype=np.int32))
    for name, x in zip(("k", "v", "w", "pos"), before):
        x = x.flatten(0, 1)
        s[name] = (x.view(torch.int16) if x.dtype == torch.bfloat16 else x).cpu().numpy().copy()
    want = evict_plain(s, page_size, 100, 4, 20)
    for name, x in zip(("k", "v", "w", "pos"), (cache.k_pages, cache.v_pages, cache.weights, cache.pos)):
        x = x[table.long()].flatten(0, 1)
        assert np.array_equal((x.view(torch.int16) if x.dtype == torch.bfloat16 else x).cpu().numpy(), want[name]), name
    check_attention(cache, queries(cache, gen))

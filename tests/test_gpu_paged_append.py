"""Appending to a paged cache on the GPU: every byte of the pool against plain copies."""
import numpy as np
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import append_plain, build, same, snapshot

pytestmark = pytest.mark.gpu


def _new(gen, n, H, m, D, dtype, token_major):
    shape = (n, m, H, D) if token_major else (n, H, m, D)
    k, v = (torch.randn(shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
    return (k.transpose(1, 2), v.transpose(1, 2)) if token_major else (k, v)


def _bits(x):
    return x.contiguous().view(torch.int16).cpu().numpy()


@pytest.mark.parametrize("lens,m,counts,H,D,page_size,dtype,token_major,weights,given", [
    ([0, 1, 15, 16, 17], 1, None, 8, 128, 16, "bf16", False, True, False),
    ([0, 5, 63, 64], 1, [1, 0, 1, 1], 2, 64, 8, "fp16", True, True, False),
    ([3, 200], 70, [70, 1], 3, 128, 32, "bf16", True, True, True),                # several CTAs per sequence, odd heads
    ([0], 1001, None, 1, 256, 64, "fp16", False, False, False),
    ([0, 7, 31], 33, [0, 33, 20], 5, 256, 8, "bf16", True, False, True),
    ([100, 0, 40], 515, [515, 0, 77], 4, 64, 128, "bf16", False, True, True),
    ([5] * 40, 700, [(37 * i) % 90 for i in range(40)], 7, 128, 16, "bf16", False, True, False),   # padded far beyond the tables
    ([0, 9000], 9001, [9001, 1], 2, 64, 4096, "fp16", True, True, False),
])
def test_append_against_plain_copies(lens, m, counts, H, D, page_size, dtype, token_major, weights, given):
    n = len(lens)
    most = max(x + c for x, c in zip(lens, counts or [m] * n))
    cache, gen = build(lens, H=H, G=1, D=D, page_size=page_size, dtype=dtype, token_major=token_major, weights=weights,
                       max_pages=-(-most // page_size), whole_table=True, seen=[x + 10 for x in lens])
    k, v = _new(gen, n, H, m, D, cache.k_pages.dtype, not token_major)
    w = torch.rand(n, H, m + 3, generator=gen, device="cuda")[:, :, :m] if weights and given else None
    pos = torch.randint(0, 1 << 30, (n, H, m + 1), generator=gen, device="cuda").to(torch.int32)[:, :, :m] if given else None
    dev_counts = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    before = snapshot(cache)
    cache.laser_kv_paged_append(k, v, counts=dev_counts, weights=w, pos=pos)
    cache.laser_kv_paged_poll_status()
    want = append_plain(before, page_size, _bits(k), _bits(v), counts or [m] * n, None if w is None else w.cpu().numpy(),
                        None if pos is None else pos.cpu().numpy())
    same(snapshot(cache), want)


def test_token_by_token_and_empty_calls():
    cache, gen = build([0, 9], H=2, G=2, page_size=8, max_pages=4, whole_table=True)
    want = snapshot(cache)
    for step in range(20):
        k, v = _new(gen, 2, 2, 1, 128, torch.bfloat16, False)
        cache.laser_kv_paged_append(k, v)
        want = append_plain(want, 8, _bits(k), _bits(v), [1, 1])
    cache.laser_kv_paged_append(k[:, :, :0], v[:, :, :0])
    cache.laser_kv_paged_append(k, v, counts=torch.zeros(2, dtype=torch.int32, device="cuda"))
    cache.laser_kv_paged_poll_status()
    same(snapshot(cache), want)


def test_what_does_not_fit_is_not_written():
    """A sequence without room or with a bad count stays as it is, the others get their entries; a bad page loses its rows alone."""
    cache, gen = build([0, 30, 31, 5], H=2, G=1, page_size=8, max_pages=4, whole_table=True)
    k, v = _new(gen, 4, 2, 2, 128, torch.bfloat16, False)
    before = snapshot(cache)
    cache.laser_kv_paged_append(k, v)                                # 31 + 2 > 32
    with pytest.raises(Bn.LaserKVError) as e:
        cache.laser_kv_paged_poll_status()
    assert e.value.status == Bn.ERR_CAPACITY
    want = append_plain(before, 8, _bits(k), _bits(v), [2, 2, 0, 2])
    same(snapshot(cache), want)
    for counts in ([1, 0, -1, 3], [0, 0, 1, 1 << 30]):
        cache.laser_kv_paged_append(k, v, counts=torch.tensor(counts, dtype=torch.int32, device="cuda"))
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_poll_status()
        assert e.value.status == Bn.ERR_INVALID_ARG
        want = append_plain(want, 8, _bits(k), _bits(v), [c if 0 <= c <= 2 else 0 for c in counts])
        same(snapshot(cache), want)
    cache.laser_kv_paged_poll_status()                               # cleared
    # entries 2 of sequence 0 and on lie in page 0 of its table, entry 8 and on in page 1
    cache.state.copy_(torch.tensor([[7, 0, 0, 0], [7, 0, 0, 0]], dtype=torch.int32))
    for bad in (-1, cache.cfg.n_pages, 1 << 30, -(1 << 31)):
        page = int(cache.page_table[0, 1])
        cache.page_table[0, 1] = bad
        before = snapshot(cache)
        cache.laser_kv_paged_append(k, v, counts=torch.tensor([2, 0, 0, 0], dtype=torch.int32, device="cuda"))
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_poll_status()
        assert e.value.status == Bn.ERR_INVALID_ARG
        after = snapshot(cache)
        p0 = before["table"][0, 0]
        before["k"][p0, :, 7], before["v"][p0, :, 7] = _bits(k)[0, :, 0], _bits(v)[0, :, 0]
        before["pos"][p0, :, 7], before["w"][p0, :, 7] = 7, 0
        before["state"][:, 0] = 9
        same(after, before)
        cache.page_table[0, 1] = page
        cache.state[:, 0] = 7


def test_refusals():
    cache, gen = build([0, 3], H=2, G=1, page_size=8, max_pages=2, whole_table=True, weights=False)
    k, v = _new(gen, 2, 2, 1, 128, torch.bfloat16, False)

    def refused(status, *a, **kw):
        before = snapshot(cache)
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_append(*a, **kw)
        assert e.value.status == status, e.value
        same(snapshot(cache), before)

    refused(Bn.ERR_STATE, k, v, weights=torch.zeros(2, 2, 1, device="cuda"))
    refused(Bn.ERR_INVALID_ARG, k, v.half())
    refused(Bn.ERR_INVALID_ARG, k[:1], v[:1])
    refused(Bn.ERR_INVALID_ARG, k.cpu(), v.cpu())
    refused(Bn.ERR_INVALID_ARG, k, v, counts=torch.zeros(2, dtype=torch.int64, device="cuda"))
    refused(Bn.ERR_INVALID_ARG, k, v, pos=torch.zeros(2, 2, 2, dtype=torch.int32, device="cuda"))
    refused(Bn.ERR_INVALID_ARG, k[:, :, :, :64], v[:, :, :, :64])
    wide = torch.zeros(2, 2, 1, 129, dtype=torch.bfloat16, device="cuda")
    refused(Bn.ERR_ALIGNMENT, wide[..., :128], wide[..., :128])
    refused(Bn.ERR_ALIGNMENT, wide.flatten()[4:4 + 512].view(2, 2, 1, 128), v)
    refused(Bn.ERR_CAPACITY, k.expand(2, 2, 17, 128), v.expand(2, 2, 17, 128))
    with pytest.raises(Bn.LaserKVError):
        Bn.PagedKV(cache.k_pages, cache.v_pages.half(), cache.page_table, n_q_heads=2)
    with pytest.raises(Bn.LaserKVError):
        Bn.PagedKV(cache.k_pages, cache.v_pages, cache.page_table.long(), n_q_heads=2)
    with pytest.raises(Bn.LaserKVError):
        Bn.PagedKV(cache.k_pages.cpu(), cache.v_pages.cpu(), cache.page_table, n_q_heads=2)
    cache.close()
    refused(Bn.ERR_INVALID_ARG, k, v)

"""Dimensions of one entry have no stride: whatever a view says there, calls on a paged cache take it."""
import pytest
import torch

from paper_2602_02199_b200 import binding as Bn

from paged_util import append_plain, build, check_attention, queries, same, snapshot

pytestmark = pytest.mark.gpu


def _odd(x, dims, stride):
    """The same tensor with another stride in dimensions of one entry."""
    st = list(x.stride())
    for d in dims:
        assert x.shape[d] == 1
        st[d] = stride
    y = x.as_strided(x.shape, st, x.storage_offset())
    assert torch.equal(*(z.contiguous().view(torch.int16) for z in (x, y)))       # bits: unused rows are NaN
    return y


@pytest.mark.parametrize("stride", [1, 4, 3000001])
@pytest.mark.parametrize("n,H,m,dims", [(2, 3, 1, [2]), (1, 3, 5, [0]), (4, 1, 3, [1]), (1, 1, 1, [0, 1, 2])])
def test_append(n, H, m, dims, stride):
    cache, gen = build([7] * n, H=H, G=1, D=64, page_size=8, max_pages=3, whole_table=True)
    k, v = (torch.randn(n, H, m, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    want = append_plain(snapshot(cache), 8, *(x.view(torch.int16).cpu().numpy() for x in (k, v)), [m] * n)
    cache.laser_kv_paged_append(_odd(k, dims, stride), _odd(v, dims, stride + 1))
    cache.laser_kv_paged_poll_status()
    same(snapshot(cache), want)


def test_one_token_out_of_a_transposed_projection():
    cache, gen = build([3, 0], H=2, G=1, D=128, page_size=8, max_pages=2, whole_table=True)
    x = torch.randn(2, 2, 128, 1, generator=gen, device="cuda").bfloat16().permute(0, 1, 3, 2)
    assert x.stride(2) == 1
    want = append_plain(snapshot(cache), 8, *[x.contiguous().view(torch.int16).cpu().numpy()] * 2, [1, 1])
    cache.laser_kv_paged_append(x, x)
    same(snapshot(cache), want)


@pytest.mark.parametrize("stride", [1, 4, 3000001])
@pytest.mark.parametrize("n,H,G,dims", [(1, 2, 2, [0]), (3, 1, 1, [1]), (1, 1, 1, [0, 1])])
def test_attention(n, H, G, dims, stride):
    cache, gen = build([70] * n, H=H, G=G, D=64, page_size=16)
    check_attention(cache, _odd(queries(cache, gen), dims, stride), accumulate=True)


def test_pools_of_one_page_or_head():
    cache, gen = build([70, 9], H=1, G=4, D=64, page_size=16)
    k, v = cache.k_pages, cache.v_pages
    for a, b in ((k, _odd(v, [1], 8)), (_odd(k, [1], 24), v), (_odd(k, [1], 3), _odd(v, [1], 5))):
        again = Bn.PagedKV(a, b, cache.page_table, n_q_heads=4, weights=cache.weights, pos=cache.pos, state=cache.state)
        check_attention(again, queries(cache, gen))
    with pytest.raises(Bn.LaserKVError):
        Bn.PagedKV(k, v[..., :32].repeat(1, 1, 1, 4)[..., :64], cache.page_table, n_q_heads=4)


def test_strides_of_more_than_one_entry_are_still_looked_at():
    cache, gen = build([7, 7], H=2, G=1, D=64, page_size=8, max_pages=3, whole_table=True)
    wide = torch.zeros(2, 2, 1, 68, dtype=torch.bfloat16, device="cuda")[..., :64]
    for x in (wide, torch.zeros(2, 2, 3, 68, dtype=torch.bfloat16, device="cuda")[..., :64]):
        with pytest.raises(Bn.LaserKVError) as e:
            cache.laser_kv_paged_append(x, x)
        assert e.value.status == Bn.ERR_ALIGNMENT
    with pytest.raises(Bn.LaserKVError) as e:
        cache.laser_kv_paged_attention(wide[:, :, 0])
    assert e.value.status == Bn.ERR_ALIGNMENT

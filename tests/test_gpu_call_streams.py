"""Results of calls on a stream that is not the current one: what the binding allocates for them belongs to that stream."""
import math

import pytest
import torch

from paper_2602_02199_b200 import binding as Bn
from paper_2602_02199_b200 import synth

from paged_util import attention64, build, queries
from parity_util import run_workload_layer

pytestmark = pytest.mark.gpu

BUSY = 200_000_000                                                   # cycles: a tenth of a second


def _beside_a_busy_stream(shape, call):
    """The result of call(stream) while work on the current stream that was queued before it has yet to write a tensor of `shape`,
    which is free again by then."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    old = torch.empty(shape, device="cuda")
    old.fill_(math.nan)
    del old
    out = call(side)
    side.synchronize()
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("raw", [False, True])
def test_results_are_not_written_over_by_the_current_stream(raw):
    cache, gen = build([300, 40], H=2, G=4, page_size=16)
    q = queries(cache, gen)
    want, _, _, t_out, _, _ = attention64(cache, q)
    for _ in range(3):
        out = _beside_a_busy_stream(q.shape, lambda s: cache.laser_kv_paged_attention(q, stream=s.cuda_stream if raw else s))
        assert ((out.double() - want).abs() <= t_out).all()


class Wrapped:
    def __init__(self, handle):
        self.cuda_stream = handle


def test_whatever_names_a_stream():
    import numpy as np
    cache, gen = build([300, 40], H=2, G=4, page_size=16)
    q, side = queries(cache, gen), torch.cuda.Stream()
    want = cache.laser_kv_paged_attention(q)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream, np.int64(side.cuda_stream), Wrapped(side.cuda_stream), 0, torch.cuda.default_stream(), torch.cuda.ExternalStream(side.cuda_stream)):
        out = cache.laser_kv_paged_attention(q, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_results_of_the_compacted_cache_are_not_written_over():
    w = synth.workload("tiny").with_(block_size=512, context_len=2048, batch=2, n_layers=1, lsh_tables=16)
    run = run_workload_layer(w, 0, n_blocks=4, debug=0)
    eng = run["engine"]
    q = torch.from_numpy(run["Q"][:, :, 3].copy().view("int16")).cuda()
    want = eng.laser_kv_decode_attention(0, q)
    for _ in range(3):
        out = _beside_a_busy_stream(want.shape, lambda s: eng.laser_kv_decode_attention(0, q, stream=s))
        assert torch.equal(out, want)


def test_window_scores_are_not_written_over():
    w = synth.workload("tiny").with_(block_size=256, context_len=1024, batch=1, n_layers=1)
    k = torch.from_numpy(synth.kv_blocks(w, 0, 0, 0, 4)[0].view("int16")).cuda()[None]
    q = torch.from_numpy(synth.q_window(w, 0, 0).view("int16")).cuda()[None]
    want = Bn.laser_kv_window_scores(k, q, 256, 4)
    for _ in range(3):
        out = _beside_a_busy_stream(want.shape, lambda s: Bn.laser_kv_window_scores(k, q, 256, 4, stream=s))
        assert torch.equal(out, want)

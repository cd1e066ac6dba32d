"""The paged cache on the CPU: configurations, refusals of the C ABI and of the native call path, and the rules that cut calls."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2602_02199_b200 import binding as Bn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _cfg(**kw):
    base = dict(n_seqs=4, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, n_pages=64, max_pages=32, dtype=Bn.BF16, track_weights=1,
                device=0)
    base.update(kw)
    return Bn.PagedConfig(**base)


def _message():
    return (Bn.load().laser_kv_last_error(None) or b"").decode()


@pytest.mark.parametrize("change,status", [
    (dict(n_seqs=0), Bn.ERR_INVALID_ARG), (dict(n_pages=0), Bn.ERR_INVALID_ARG), (dict(max_pages=0), Bn.ERR_INVALID_ARG),
    (dict(n_kv_heads=0), Bn.ERR_INVALID_ARG), (dict(n_q_heads=30), Bn.ERR_INVALID_ARG), (dict(n_q_heads=0), Bn.ERR_INVALID_ARG),
    (dict(head_dim=96), Bn.ERR_UNSUPPORTED), (dict(head_dim=512), Bn.ERR_UNSUPPORTED), (dict(page_size=4), Bn.ERR_UNSUPPORTED),
    (dict(page_size=24), Bn.ERR_UNSUPPORTED), (dict(page_size=8192), Bn.ERR_UNSUPPORTED), (dict(dtype=2), Bn.ERR_INVALID_ARG),
    (dict(track_weights=2), Bn.ERR_INVALID_ARG), (dict(n_seqs=65536), Bn.ERR_UNSUPPORTED), (dict(max_pages=1 << 27), Bn.ERR_UNSUPPORTED),
    (dict(n_pages=1 << 28), Bn.ERR_UNSUPPORTED), (dict(n_q_heads=8 * 129), Bn.ERR_UNSUPPORTED), (dict(n_seqs=60000, max_pages=1 << 17), Bn.ERR_UNSUPPORTED)])
def test_configurations_out_of_range_are_refused(change, status):
    with pytest.raises(Bn.LaserKVError) as e:
        Bn.laser_kv_paged_query_sizes(_cfg(**change))
    assert e.value.status == status
    out = C.c_void_p(1)
    st = (C.c_int64 * 3)(8 * 16 * 128, 16 * 128, 128)
    assert Bn.load().laser_kv_paged_init(C.byref(_cfg(**change)), 256, 256, st, 256, 256, 256, 256, 256, 1 << 40, C.byref(out)) == status
    assert not out.value


@pytest.mark.parametrize("group,track", [(1, 0), (4, 1), (7, 1), (16, 0), (20, 1)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_workspace_sizes(group, track, d):
    cfg = _cfg(n_q_heads=8 * group, head_dim=d, track_weights=track)
    size = Bn.laser_kv_paged_query_sizes(cfg)
    assert size % 256 == 0
    # parts of the CTAs, and with weights a score per query head (a power of two of them) and entry, a pair of indices per two
    wide, ctas = 1 if group <= 8 else 2, {64: 480, 128: 320, 256: 160}[d]
    least = ctas * 2 * wide * 8 * (d + 2) * 4
    if track:
        heads = max(4, 1 << (group - 1).bit_length())
        units = (64 * 16 // 64 + 6 * 4) * 8
        least += units * (64 * heads * 4 + 8) + 64 * 16 * 8 // 2 * 8
    assert least <= size <= least + 20000


def test_init_refuses_what_it_can_see():
    lib, out = Bn.load(), C.c_void_p()
    need = Bn.laser_kv_paged_query_sizes(_cfg())
    good = dict(k=256, v=256, st=(8 * 16 * 128, 16 * 128, 128), w=256, pos=256, table=256, state=256, ws=256, bytes=need)

    def init(cfg=None, **kw):
        a = dict(good, **kw)
        return lib.laser_kv_paged_init(C.byref(cfg or _cfg()), a["k"], a["v"], (C.c_int64 * 3)(*a["st"]), a["w"], a["pos"], a["table"], a["state"],
                                       a["ws"], a["bytes"], C.byref(out))

    for name in ("k", "v", "pos", "table", "state", "ws"):
        assert init(**{name: 0}) == Bn.ERR_INVALID_ARG and "NULL" in _message()
        assert init(**{name: 264 if name != "ws" else 384}) == Bn.ERR_ALIGNMENT
    assert init(w=0) == Bn.ERR_INVALID_ARG and "track_weights" in _message()
    assert init(cfg=_cfg(track_weights=0)) == Bn.ERR_INVALID_ARG
    assert init(bytes=need - 1) == Bn.ERR_CAPACITY and f"needs {need} bytes" in _message()
    for st in ((8 * 16 * 128, 16 * 128, 64), (8 * 16 * 128, 16 * 128, 132), (8 * 16 * 128, 16 * 128, -128), (0, 16 * 128, 128)):
        assert init(st=st) == Bn.ERR_ALIGNMENT
    for st in ((8 * 16 * 128, 8 * 128, 128), (7 * 16 * 128, 16 * 128, 128), (128, 128, 128), (8 * 16 * 128 - 8, 128, 8 * 128)):
        assert init(st=st) == Bn.ERR_INVALID_ARG and "overlap" in _message()
    assert init(st=(1 << 38, 16 * 128, 128)) == Bn.ERR_UNSUPPORTED
    assert init(cfg=_cfg(n_pages=1 << 16), bytes=1 << 50, st=(1 << 37, 16 * 128, 128)) == Bn.ERR_UNSUPPORTED
    # rows that lie beside one another in any order of the strides; a dimension of one entry has no stride
    for st, kw in (((8 * 16 * 128, 128, 8 * 128), {}), ((128, 64 * 128, 8 * 64 * 128), {}), ((16 * 128, 8, 128), dict(n_kv_heads=1, n_q_heads=4)),
                   ((3 * 8 * 16 * 128, 16 * 136, 136), {})):
        s = init(cfg=_cfg(**kw), st=st, ws=256, bytes=1 << 40, table=0)
        assert s == Bn.ERR_INVALID_ARG and "NULL" in _message()
    if not _have_gpu():
        assert init() == Bn.ERR_CUDA and "no CPU path" in _message()


def _have_gpu():
    import torch
    return torch.cuda.is_available()


def test_calls_refuse_a_null_handle():
    lib = Bn.load()
    Bn.load()
    st = (128, 128, 128, 1)
    n = Bn._pycall
    assert n.paged_append(0, 16, 16, st, st, 1, 0, 0, (0, 0), 0, (0, 0), 0) == Bn.ERR_INVALID_ARG and "NULL handle" in _message()
    assert n.paged_attention(0, 16, st, 0.0, 0, 16, 1, 0, 0) == Bn.ERR_INVALID_ARG and "NULL handle" in _message()
    assert n.paged_evict(0, 1, 0, 0, 0) == Bn.ERR_INVALID_ARG and "NULL handle" in _message()
    assert lib.laser_kv_paged_poll_status(None, None) == Bn.ERR_INVALID_ARG
    lib.laser_kv_paged_destroy(None)
    c = Bn._CtypesCalls(lib)
    assert c.paged_append(0, 16, 16, st, st, 1, 0, 0, (0, 0), 0, (0, 0), 0) == Bn.ERR_INVALID_ARG
    assert c.paged_attention(0, 16, st, 0.0, 0, 16, 1, 0, 0) == Bn.ERR_INVALID_ARG
    assert c.paged_evict(0, 1, 0, 0, 0) == Bn.ERR_INVALID_ARG
    with pytest.raises(TypeError):
        n.paged_evict(0, 1, 0, 0)
    with pytest.raises(ValueError):
        n.paged_attention(0, 16, (128,), 0.0, 0, 16, 1, 0, 0)


RULES = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "launch_rules.h"
using namespace lkv;
static void need(bool ok, const char* what, long long a, long long b) { if (!ok) { printf("%s %lld %lld\n", what, a, b); exit(1); } }
int main() {
  const int totals[] = {1, 2, 3, 7, 147, 148, 149, 295, 296, 297, 1000, 4097, 123457, 2147483647};
  for (int total : totals)
    for (int grid : {1, 2, 3, 148, 296, 444, 480}) {
      const PagedShares s(total, grid, false);
      const int n = s.n;
      need(n >= 1 && n <= grid && n <= total, "shares", total, grid);
      need(s.begin(0) == 0 && s.begin(n) == total, "ends", total, n);
      for (int c = 0; c < n; ++c) {
        const int lo = s.begin(c), hi = s.begin(c + 1);
        need(lo == (long long)total * c / n && hi > lo, "empty share", total, c);
        need(s.owner(lo) == c && s.owner(hi - 1) == c && s.owner(lo + (hi - lo) / 2) == c, "owner", total, c);
      }
    }
  need(PagedShares(0, 296, false).n == 0 && PagedShares(0, 296, true).n == 0, "no tiles", 0, 0);
  for (int items : {1, 2, 7, 295, 296, 297, 5000, 268435455})        // none is split
    for (int grid : {1, 3, 148, 296, 480}) {
      const PagedShares s(items * kPagedWholeUnits, grid, true);
      need(s.n >= 1 && s.n <= grid && s.n <= items && s.begin(0) == 0 && s.begin(s.n) == items * kPagedWholeUnits, "whole", items, grid);
      for (int c = 0; c < s.n; ++c) need(s.begin(c) % kPagedWholeUnits == 0 && s.begin(c + 1) > s.begin(c), "item", items, c);
    }
  for (long long heads : {1ll, 2ll, 8ll, 30ll, 64ll, 100ll, 512ll, 100000ll})
    for (long long cap : {8ll, 64ll, 1024ll, 1025ll, 2056ll, 40960ll, 49152ll, 49153ll, 400000ll, 786432ll, 786433ll})
      for (int most : {8, 16}) {
        // a device of 148 SMs with a CTA each, in parts of 18
        auto room = [most](int n, long long) { return n > most ? 0 : 8 * (18 / n); };
        const int n = evict_cluster(heads, cap, room);
        need((n == 0) == (cap > 49152ll * most), "limit", heads, cap);
        if (!n) continue;
        need(n <= most && (n & (n - 1)) == 0 && (long long)n * kEvictKeys >= cap, "cluster", heads, cap);
        need(n == 1 || room(n, cap) >= heads || (long long)n / 2 * kEvictKeys < cap, "more than the device holds", heads, cap);
        const int m = move_ctas(148, heads, cap);
        need(m >= 1 && (m == 1 || (m * heads <= 4 * 148 && (m - 1) * 32ll < cap)), "movers", heads, cap);
      }
  for (unsigned d = 1; d <= 65536; d = d < 300 ? d + 1 : d * 5 / 4) {
    const Quotient q(d);
    for (long long r : {0ll, 1ll, (long long)d - 1, (long long)d, 2ll * d - 1, 12345ll, 1000003ll, (1ll << 30) / d * d - 1, (1ll << 30) / d * d, 2147483647ll / d * d - 1,
                        2147483647ll / d * d, 2147483647ll, 2147483646ll})
      if (r >= 0 && r <= 2147483647ll) need(q.of((int)r) == r / d, "quotient", r, d);
  }
  for (long long rows : {1ll, 8ll, 128000ll, 1ll << 30})
    for (long long n : {1ll, 6ll, 64ll, 65535ll}) need(append_times(148, n, rows, 32) >= 1 && append_times(148, n, rows, 32) <= kAppendTimes, "times", rows, n);
  return 0;
}
"""


def test_rules_that_cut_paged_calls(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "rules.cpp", tmp_path / "rules"
    src.write_text(RULES)
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "paper_2602_02199_b200", "csrc"), str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout

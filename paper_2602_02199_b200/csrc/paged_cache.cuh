// The kernels that change a paged cache:
//   paged_append_kernel  new entries behind each sequence's last one
//   paged_evict_kernel   every (sequence, KV head) back to `keep` entries by accumulated attention weight
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "aux_kernels.cuh"
#include "decode_attn.cuh"
#include "launch_rules.h"
#include "paged_attn.cuh"

namespace lkv {

struct PagedRows {                                         // where the rows of the pool lie
  uint16_t* K;
  uint16_t* V;
  long long s_page, s_head, s_row;                         // strides (elements)
  float* weights;                                          // [n_pages][H][page_size]; NULL: not kept
  int* pos;                                                // [n_pages][H][page_size]
  int vecs;                                                // 16-byte vectors of a row: 8, 16 or 32
};

// ------------------------------------------------------------------------------------------------
// Append. Rows (token, head) of a sequence, head by head within a token, are dealt to CTAs of kPagedAppendRows; a thread has a
// vector of the key and of the value of up to four rows under way. Bound by HBM for prompts, by round trips (length, page,
// row) for single tokens. The last CTA of a sequence to have read its length advances it.
// ------------------------------------------------------------------------------------------------
struct PagedAppendArgs {
  PagedPool pool;
  PagedRows rows;
  const uint16_t* K;
  const uint16_t* V;
  long long ks[3], vs[3];                                  // strides (elements): sequence, head, token
  const float* w;                                          // weights of the new entries or NULL (0)
  const int* at;                                           // their positions or NULL (counted on)
  long long ws[2], as[2];                                  // strides: sequence, head
  const int* counts;                                       // [n_seqs] or NULL (n_new)
  int n_new;
  int* tickets;                                            // [n_seqs] CTAs that have read the length; zero between calls
};

constexpr int kPagedAppendThreads = 256;

template <int VECS>
__global__ void __launch_bounds__(kPagedAppendThreads, 4) paged_append_kernel(const PagedAppendArgs a) {
  constexpr int kPer = kPagedAppendThreads / VECS, N = 4;  // rows side by side, rows of a thread
  allow_dependents();
  const PagedPool& p = a.pool;
  const int b = blockIdx.y, part = threadIdx.x % VECS;
  grid_dependency_wait();
  const int held = p.lens[b], seen = p.seen[b];
  int count = a.counts ? a.counts[b] : a.n_new, bad = 0;
  if (count < 0 || count > a.n_new || held < 0 || held > p.max_pages << p.page_shift) bad = kPagedBadPage;
  else if (count > (p.max_pages << p.page_shift) - held) bad = kStatusCapacity;
  if (bad) {
    if (threadIdx.x == 0) record_status(p.status, bad);
    count = 0;                                             // nothing of this sequence
  }
  const int n_rows = count * p.H, r0 = (int)blockIdx.x * (kPer * N) + threadIdx.x / VECS;   // below 2^31: the host looks
  uint4 kv[N], vv[N];
  long long to[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int r = r0 + j * kPer;
    to[j] = -1;
    if (r >= n_rows) continue;
    const int i = r / p.H, h = r - i * p.H;
    const int page = p.page(b, held + i), row = (held + i) & (p.page_size() - 1);
    if ((unsigned)page >= (unsigned)p.n_pages) {           // never written outside the pool
      if (part == 0) record_status(p.status, kPagedBadPage);
      continue;
    }
    kv[j] = ld_nc_v4(a.K + b * a.ks[0] + h * a.ks[1] + i * a.ks[2] + part * 8);
    vv[j] = ld_nc_v4(a.V + b * a.vs[0] + h * a.vs[1] + i * a.vs[2] + part * 8);
    to[j] = page * a.rows.s_page + h * a.rows.s_head + row * a.rows.s_row;
    if (part == 0) {
      const long long slot = (((long long)page * p.H + h) << p.page_shift) + row;
      a.rows.pos[slot] = a.at ? a.at[b * a.as[0] + h * a.as[1] + i] : seen + i;
      if (a.rows.weights) a.rows.weights[slot] = a.w ? a.w[b * a.ws[0] + h * a.ws[1] + i] : 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (to[j] < 0) continue;
    *reinterpret_cast<uint4*>(a.rows.K + to[j] + part * 8) = kv[j];
    *reinterpret_cast<uint4*>(a.rows.V + to[j] + part * 8) = vv[j];
  }
  __syncthreads();                                         // the whole CTA has read the length
  if (threadIdx.x == 0 && !bad) {
    bool last = gridDim.x == 1;
    if (!last) {
      __threadfence();
      last = atomicAdd(a.tickets + b, 1) == (int)gridDim.x - 1;
      if (last) a.tickets[b] = 0;
    }
    if (last) {
      p.lens[b] = held + count;
      if (!a.at) p.seen[b] = seen + count;
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Eviction. One cluster per (sequence, KV head); every CTA holds the sort keys of a slice of the entries in shared memory.
//   1. keys: the weight as an ordered integer, the largest for protected entries (the first positions and the last ones),
//      -inf for NaN, which therefore leaves first.
//   2. the keep-th largest key, by radix rounds over the eleven highest bits in which undecided keys can differ (as in
//      take_topk), the histograms summed across the cluster; protected keys, often the most, are counted apart, so that they
//      do not pile up in one bin.
//   3. a sweep in index order with two counts (keys above, keys equal to it) gives every entry its rank among the kept ones.
//      An evicted entry before `keep` is a hole, a kept one behind it a mover; holes are counted from the start, movers from the end,
//      and the pairs go to a list.
//   4. the cluster's warps move rows by the list. All sources lie behind `keep`, all destinations before it: no move
//      waits for another, and only rows that have to move are touched. (Closing the gaps in order would move nearly every row.)
// Reads 8 bytes per entry and moves two rows per hole: bound by HBM for large calls, by barriers and round trips for small ones.
// ------------------------------------------------------------------------------------------------
struct PagedEvictArgs {
  PagedPool pool;
  PagedRows rows;
  int keep, anchors, recent;
  int2* moves;                                             // lists of (hole, mover): per sequence, per KV head
  long long n_moves;                                       // pairs that `moves` holds
  int* ticket;                                             // clusters that are done; zero between calls
};

constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;

struct EvictShared {
  int hist[kSelBins];                                      // this CTA's; zero between rounds
  int sums[kSelBins];                                      // its share of the cluster's bins, summed over the CTAs
  int share;                                               // sum of its share
  int chunk[kEvictWarps];
  int found[3];
  uint32_t lo[kEvictWarps], hi[kEvictWarps];
  int prot[kEvictWarps];
  uint32_t range[2];                                       // smallest and largest unprotected key of the CTA
  int n_prot;
  int above[kEvictWarps], equal[kEvictWarps], holes[kEvictWarps];
  int totals[3];                                           // CTA: keys above, keys equal, holes
  int offset_lo;                                           // (sequence, head)'s place in the list
  int last;
};

__host__ __device__ constexpr uint32_t evict_smem_bytes(int slice) { return (uint32_t)slice * 4u + (uint32_t)sizeof(EvictShared) + 16u; }
// Entries of a CTA's slice: whole warps' worths.
LKV_HOST_DEVICE inline int evict_slice(long long len, int n) { return (int)((len + n - 1) / n + kEvictThreads - 1) / kEvictThreads * kEvictThreads; }

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

constexpr uint32_t kEvictProtected = 0xFFFFFFFFu;

__global__ void __launch_bounds__(kEvictThreads, 2) paged_evict_kernel(const PagedEvictArgs a) {
  extern __shared__ __align__(16) uint8_t esm_raw[];
  EvictShared& sh = *reinterpret_cast<EvictShared*>(esm_raw);
  uint32_t* const keys = reinterpret_cast<uint32_t*>(esm_raw + (sizeof(EvictShared) + 15) / 16 * 16);
  const PagedPool& p = a.pool;
  const int C = gridDim.x, rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto remote = [&](const void* at, int r) { return ld_cluster_u32(cluster_addr(smem_u32(at), r)); };
  for (int i = tid; i < kSelBins; i += kEvictThreads) sh.hist[i] = 0;
  grid_dependency_wait();
  allow_dependents();

  const int len = p.length(b), keep = a.keep;
  // Lengths change only when every cluster has read all that it needs of them: the last one does it.
  auto done = [&]() {
    if (rank == 0 && tid == 0) {
      __threadfence();
      const int all = (int)(gridDim.y * gridDim.z);
      sh.last = atomicAdd(a.ticket, 1) == all - 1;
      if (sh.last) *a.ticket = 0;
    }
    __syncthreads();
    if (rank == 0 && sh.last)
      for (int i = tid; i < p.n_seqs; i += kEvictThreads)
        if (p.lens[i] > keep) p.lens[i] = keep;
  };
  if (len != p.lens[b] && tid == 0) record_status(p.status, kPagedBadPage);
  if (len <= keep) {                                       // the same in all of the cluster
    if (C > 1) cluster_sync(); else __syncthreads();       // all of it has read the length
    done();
    return;
  }

  // ---- 1. keys ----------------------------------------------------------------------------------
  const int slice = evict_slice(len, C), lo_i = min(len, rank * slice), n = min(len - lo_i, slice);
  const int newest = p.seen[b] - a.recent;
  uint32_t lo = 0xFFFFFFFFu, hi = 0u;
  int prot = 0;
  for (int i0 = tid; i0 < n; i0 += 4 * kEvictThreads) {
    int page[4], at[4];
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) page[j] = i0 + j * kEvictThreads < n ? p.page(b, lo_i + i0 + j * kEvictThreads) : -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + j * kEvictThreads;
      const bool ok = (unsigned)page[j] < (unsigned)p.n_pages;
      const long long slot = (((long long)page[j] * p.H + h) << p.page_shift) + ((lo_i + i) & (p.page_size() - 1));
      x[j] = ok ? a.rows.weights[slot] : -INFINITY;
      at[j] = ok ? a.rows.pos[slot] : a.anchors;
      if (i < n && !ok) record_status(p.status, kPagedBadPage);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + j * kEvictThreads;
      if (i >= n) continue;
      const bool safe = at[j] < a.anchors || at[j] >= newest || x[j] == INFINITY;
      const uint32_t key = safe ? kEvictProtected : orderable_f32(x[j] != x[j] ? -INFINITY : x[j] + 0.f);   // + 0: -0 is 0
      keys[i] = key;
      prot += safe;
      if (!safe) { lo = min(lo, key); hi = max(hi, key); }
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  prot = __reduce_add_sync(0xffffffffu, prot);
  if (lane == 0) { sh.lo[warp] = lo; sh.hi[warp] = hi; sh.prot[warp] = prot; }
  __syncthreads();
  if (warp == 0) {
    lo = __reduce_min_sync(0xffffffffu, sh.lo[lane % kEvictWarps]);
    hi = __reduce_max_sync(0xffffffffu, sh.hi[lane % kEvictWarps]);
    prot = __reduce_add_sync(0xffffffffu, lane < kEvictWarps ? sh.prot[lane] : 0);
    if (lane == 0) { sh.range[0] = lo; sh.range[1] = hi; sh.n_prot = prot; }
  }
  if (C > 1) cluster_sync(); else __syncthreads();
  {
    const int r = lane < C ? lane : 0;
    lo = __reduce_min_sync(0xffffffffu, remote(&sh.range[0], r));
    hi = __reduce_max_sync(0xffffffffu, remote(&sh.range[1], r));
    prot = __reduce_add_sync(0xffffffffu, lane < C ? (int)remote(&sh.n_prot, r) : 0);
  }

  // ---- 2. the keep-th largest key ----------------------------------------------------------------
  // kept: keys from `from` on, and of those equal to `tie` the first `ties` in index order
  uint32_t from = kEvictProtected, tie = kEvictProtected;
  long long ties = 0;
  bool with_ties = false;
  if (prot >= keep) {
    from = 0;                                              // none by being above
    with_ties = true;
    ties = keep;
  } else {
    int need = keep - prot;                                // of len - prot > need unprotected ones
    uint32_t base = lo;
    uint64_t span_hi = hi;                                 // undecided: keys in [base, span_hi]
    int shift = 32 - __clz(hi - lo) - kSelBinBits;
    if (shift < 0) shift = 0;
    const int per = kSelBins / C;                          // bins of a CTA's share
    for (;;) {
      for (int i = tid; i < n; i += kEvictThreads) {
        const uint32_t key = keys[i];
        if (key != kEvictProtected && key >= base && key <= span_hi) atomicAdd(&sh.hist[(key - base) >> shift], 1);
      }
      const int* bins = sh.hist;
      int share = 0, before = 0;
      if (C > 1) {
        cluster_sync();
        // this CTA's share: bins [rank * per, (rank + 1) * per)
        int mine = 0;
        for (int i = tid; i < per; i += kEvictThreads) {
          int v = 0;
          for (int r = 0; r < C; ++r) v += (int)remote(&sh.hist[rank * per + i], r);
          sh.sums[i] = v;
          mine += v;
        }
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) sh.chunk[warp] = mine;
        __syncthreads();
        if (tid == 0) {
          int s = 0;
          for (int i = 0; i < kEvictWarps; ++i) s += sh.chunk[i];
          sh.share = s;
        }
        cluster_sync();                                    // sums are written, histograms read
        // the share that holds the need-th from the top
        const int v = lane < C ? (int)remote(&sh.share, C - 1 - lane) : 0;
        const int incl = warp_inclusive(v, lane);
        const int who = __ffs(__ballot_sync(0xffffffffu, lane < C && incl >= need)) - 1;
        share = C - 1 - who;
        before = __shfl_sync(0xffffffffu, incl - v, who);
        bins = nullptr;
      } else {
        __syncthreads();
      }
      // bins of the share from high to low; a warp takes a run of them
      constexpr int kMost = kSelBins / kEvictThreads;
      const int mine_n = (per + kEvictThreads - 1) / kEvictThreads;
      int c[kMost], sum = 0;
#pragma unroll
      for (int k = 0; k < kMost; ++k) {
        const int i = per - 1 - (tid * mine_n + k);
        c[k] = k < mine_n && i >= 0 ? (bins ? bins[i] : (int)remote(&sh.sums[i], share)) : 0;
        sum += c[k];
      }
      const int wsum = __reduce_add_sync(0xffffffffu, sum);
      __syncthreads();                                     // sh.chunk is read (share sums), the bins too
      if (lane == 0) sh.chunk[warp] = wsum;
      for (int i = tid; i < kSelBins; i += kEvictThreads) sh.hist[i] = 0;
      __syncthreads();
      {
        const int x = lane < kEvictWarps ? sh.chunk[lane] : 0;
        const int incl = warp_inclusive(x, lane);
        int run = before + __shfl_sync(0xffffffffu, incl - x, warp);
        run += warp_inclusive(sum, lane) - sum;            // keys in higher bins than this thread's
#pragma unroll
        for (int k = 0; k < kMost; ++k) {
          if (run < need && need <= run + c[k]) {
            sh.found[0] = share * per + per - 1 - (tid * mine_n + k);
            sh.found[1] = need - run;
            sh.found[2] = c[k];
          }
          run += c[k];
        }
      }
      __syncthreads();
      const uint32_t bin = (uint32_t)sh.found[0];
      need = sh.found[1];
      const int held = sh.found[2];
      base += bin << shift;
      if (need == held) {                                  // the whole bin
        from = base;
        break;
      }
      if (shift == 0) {                                    // equal keys: the ones of lowest index
        from = base + 1;                                   // base < kEvictProtected
        tie = base;
        ties = need;
        with_ties = true;
        break;
      }
      span_hi = (uint64_t)base + (1ull << shift) - 1;
      shift = shift > kSelBinBits ? shift - kSelBinBits : 0;
    }
  }
  const bool none_above = with_ties && tie == kEvictProtected;

  // ---- 3. ranks and the list of moves -------------------------------------------------------------
  const int run_n = slice / kEvictWarps, w_lo = min(n, warp * run_n), w_hi = min(n, w_lo + run_n);
  {
    int above = 0, equal = 0;
    for (int i = w_lo + lane; i < w_hi; i += 32) {
      const uint32_t key = keys[i];
      above += !none_above && key >= from;
      equal += with_ties && key == tie;
    }
    above = __reduce_add_sync(0xffffffffu, above);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane == 0) { sh.above[warp] = above; sh.equal[warp] = equal; }
  }
  // the place of this (sequence, head)'s pairs: at most min(keep, len - keep) per head
  if (warp == 1) {
    long long sum = 0;
    for (int i = lane; i < b; i += 32) sum += max(0, min(keep, p.length(i) - keep));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    const long long most = min(keep, len - keep), at = sum * p.H + (long long)h * most;
    // the list is as large as a pool whose pages are not shared can need
    if (lane == 0) sh.offset_lo = at + most <= a.n_moves ? (int)at : -1;
  }
  __syncthreads();
  int above0 = 0, equal0 = 0;                              // before this warp's run
  {
    const int va = lane < kEvictWarps ? sh.above[lane] : 0, ve = lane < kEvictWarps ? sh.equal[lane] : 0;
    const int ia = warp_inclusive(va, lane), ie = warp_inclusive(ve, lane);
    above0 = __shfl_sync(0xffffffffu, ia - va, warp);
    equal0 = __shfl_sync(0xffffffffu, ie - ve, warp);
    if (C > 1) {
      if (warp == 0 && lane == 31) { sh.totals[0] = ia; sh.totals[1] = ie; }
      cluster_sync();
      const int ra = lane < rank ? (int)remote(&sh.totals[0], lane) : 0, re = lane < rank ? (int)remote(&sh.totals[1], lane) : 0;
      above0 += __reduce_add_sync(0xffffffffu, ra);
      equal0 += __reduce_add_sync(0xffffffffu, re);
    }
  }
  const bool room = sh.offset_lo >= 0;
  int2* const list = a.moves + (room ? sh.offset_lo : 0);
  int holes = 0;
  for (int i0 = w_lo; i0 < w_hi; i0 += 32) {
    const int i = i0 + lane, e = lo_i + i;                 // entry
    const bool in = i < w_hi;
    const uint32_t key = in ? keys[i] : 0u;
    const bool is_above = in && !none_above && key >= from, is_equal = in && with_ties && key == tie;
    const uint32_t ma = __ballot_sync(0xffffffffu, is_above), me = __ballot_sync(0xffffffffu, is_equal);
    const uint32_t below = (1u << lane) - 1u;
    const long long eq = (long long)equal0 + __popc(me & below);
    const bool kept = is_above || (is_equal && eq < ties);
    const int kept_before = above0 + __popc(ma & below) + (int)(eq < ties ? eq : ties);
    if (in && room) {
      if (e < keep && !kept) list[e - kept_before].x = e;
      if (e >= keep && kept) list[keep - 1 - kept_before].y = e;
    }
    holes += in && e < keep && !kept;
    above0 += __popc(ma);
    equal0 += __popc(me);
  }
  holes = __reduce_add_sync(0xffffffffu, holes);
  if (lane == 0) sh.holes[warp] = holes;
  __syncthreads();
  if (warp == 0) {
    holes = __reduce_add_sync(0xffffffffu, lane < kEvictWarps ? sh.holes[lane] : 0);
    if (lane == 0) sh.totals[2] = holes;
  }
  // ---- 4. moves ---------------------------------------------------------------------------------
  if (C > 1) cluster_sync(); else __syncthreads();         // the list is written, by all of the cluster
  const int total = __reduce_add_sync(0xffffffffu, lane < C ? (int)remote(&sh.totals[2], lane) : 0);
  if (!room) {
    if (tid == 0) record_status(p.status, kStatusCapacity);
  } else {
    const int vecs = a.rows.vecs, lanes = min(2 * vecs, 32), per_warp = 32 / lanes;   // lanes of a move: half on the key, half on the value
    const int sub = lane / lanes, l = lane % lanes, half = lanes / 2;
    const int step = C * kEvictWarps * per_warp;
    constexpr int N = 4;                                   // moves of a thread under way together
    for (int r0 = (rank * kEvictWarps + warp) * per_warp + sub; r0 < total; r0 += N * step) {
      long long fr[N], to[N], sf[N], sd[N];
      bool ok[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int r = r0 + j * step;
        ok[j] = r < total;
        const int2 mv = ok[j] ? __ldcg(list + r) : make_int2(0, 0);
        const int pd = ok[j] ? p.page(b, mv.x) : -1, ps = ok[j] ? p.page(b, mv.y) : -1;
        ok[j] = (unsigned)pd < (unsigned)p.n_pages && (unsigned)ps < (unsigned)p.n_pages;   // others were recorded above
        const int rd = mv.x & (p.page_size() - 1), rs = mv.y & (p.page_size() - 1);
        to[j] = pd * a.rows.s_page + h * a.rows.s_head + rd * a.rows.s_row;
        fr[j] = ps * a.rows.s_page + h * a.rows.s_head + rs * a.rows.s_row;
        sd[j] = (((long long)pd * p.H + h) << p.page_shift) + rd;
        sf[j] = (((long long)ps * p.H + h) << p.page_shift) + rs;
      }
      uint16_t* const side = l < half ? a.rows.K : a.rows.V;
      const int v0 = l < half ? l : l - half;
      for (int v = v0; v < vecs; v += half) {
        uint4 x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) if (ok[j]) x[j] = *reinterpret_cast<const uint4*>(side + fr[j] + v * 8);
#pragma unroll
        for (int j = 0; j < N; ++j) if (ok[j]) *reinterpret_cast<uint4*>(side + to[j] + v * 8) = x[j];
      }
      if (l == 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) if (ok[j]) a.rows.weights[sd[j]] = a.rows.weights[sf[j]];
      } else if (l == half) {
#pragma unroll
        for (int j = 0; j < N; ++j) if (ok[j]) a.rows.pos[sd[j]] = a.rows.pos[sf[j]];
      }
    }
  }
  if (C > 1) cluster_sync();                               // no CTA leaves while another may read its shared memory
  done();
}

}  // namespace lkv

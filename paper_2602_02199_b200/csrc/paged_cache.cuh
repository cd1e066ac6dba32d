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
// Append. Rows (token, head) of a sequence, head by head within a token, are dealt to CTAs; a thread has a vector of the key and of
// the value of two rows under way, several times over. Bound by HBM for prompts, by round trips (length, page, row) for
// single tokens. The last CTA of a sequence to have read its length advances it.
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
  int n_new, times;                                        // entries at most; how often a CTA takes kPagedAppendRows rows per thread
  Quotient by_heads;                                       // rows of a token
  int* tickets;                                            // [n_seqs] CTAs that have read the length; zero between calls
};

constexpr int kPagedAppendThreads = 256, kPagedAppendCtas = 5;   // per SM
constexpr int kPagedAppendRows = 2;                        // of a thread

template <int VECS>
__global__ void __launch_bounds__(kPagedAppendThreads, kPagedAppendCtas) paged_append_kernel(const PagedAppendArgs a) {
  constexpr int kPer = kPagedAppendThreads / VECS, N = kPagedAppendRows;   // rows side by side; of a thread
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
  const int n_rows = count * p.H, first = (int)blockIdx.x * (kPer * N * a.times), last = min(n_rows, first + kPer * N * a.times);   // below 2^31: the host looks
  // Nothing is loaded under a condition, so that the rows of a thread are under way together; rows past the end repeat the last.
  const uint16_t *src_k = a.K + b * a.ks[0] + part * 8, *src_v = a.V + b * a.vs[0] + part * 8;
  for (int r0 = first + threadIdx.x / VECS; r0 < last; r0 += kPer * N) {
    uint4 kv[N], vv[N];
    int page[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int r = min(r0 + j * kPer, n_rows - 1), i = a.by_heads.of(r), h = r - i * p.H;
      page[j] = p.page(b, held + i);
      kv[j] = ld_nc_v4(src_k + h * a.ks[1] + i * a.ks[2]);
      vv[j] = ld_nc_v4(src_v + h * a.vs[1] + i * a.vs[2]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int r = r0 + j * kPer, i = a.by_heads.of(r), h = r - i * p.H;
      if (r >= n_rows) continue;
      if ((unsigned)page[j] >= (unsigned)p.n_pages) {      // never written outside the pool
        if (part == 0) record_status(p.status, kPagedBadPage);
        continue;
      }
      const long long to = page[j] * a.rows.s_page + h * a.rows.s_head + ((held + i) & (p.page_size() - 1)) * a.rows.s_row + part * 8;
      *reinterpret_cast<uint4*>(a.rows.K + to) = kv[j];
      *reinterpret_cast<uint4*>(a.rows.V + to) = vv[j];
    }
  }
  // positions and weights, a row per thread
  for (int r = first + threadIdx.x; r < last; r += kPagedAppendThreads) {
    const int i = a.by_heads.of(r), h = r - i * p.H, page = p.page(b, held + i);
    const int at = a.at ? a.at[b * a.as[0] + h * a.as[1] + i] : seen + i;
    const float w = a.w ? a.w[b * a.ws[0] + h * a.ws[1] + i] : 0.f;
    if ((unsigned)page >= (unsigned)p.n_pages) continue;
    const long long slot = (((long long)page * p.H + h) << p.page_shift) + ((held + i) & (p.page_size() - 1));
    a.rows.pos[slot] = at;
    if (a.rows.weights) a.rows.weights[slot] = w;
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
// Eviction. paged_evict_kernel: one cluster per (sequence, KV head); every CTA holds the sort keys of a slice of the entries in
// shared memory.
//   1. keys: the weight as an ordered integer, the largest for protected entries (the first positions and the last ones; a negative
//      position is neither), -inf for NaN, which therefore leaves first.
//   2. the keep-th largest key, by radix rounds over 11, 11 and 10 bits, the histograms summed across the cluster; protected
//      keys, often the most, are counted apart, so that they do not pile up in one bin. (Starting from the smallest and the largest key, as
//      take_topk does, takes one more barrier and gains nothing where some entries never received any weight.) A lone CTA ranks
//      the last few undecided keys against one another instead of further rounds.
//   3. a sweep in index order with two counts (keys above, keys equal to it) gives every entry its rank among the kept ones.
//      An evicted entry before `keep` is a hole, a kept one behind it a mover; holes are counted from the start, movers from the end,
//      and the pairs go to a list, as slots of the pool.
// paged_move_kernel moves rows by the lists, with all SMs, and sets the lengths; a sequence whose pairs found no room stays as it is. All sources lie behind `keep`, all destinations
// before it: no move waits for another, and only rows that have to move are touched. (Closing the gaps in order would move
// nearly every row.) The first kernel reads 8 bytes per entry and is bound by barriers and round trips, the second by HBM.
// ------------------------------------------------------------------------------------------------
struct PagedEvictArgs {
  PagedPool pool;
  PagedRows rows;
  int keep, anchors, recent;
  int2* moves;                                             // lists of (hole, mover): per sequence, per KV head
  long long n_moves;                                       // pairs that `moves` holds
  int2* lists;                                             // [n_seqs][H] where each list starts (-1: no room for the sequence's) and how long it is
};

constexpr int kEvictThreads = 1024;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictFew = 256;                             // undecided keys that a lone CTA ranks directly

struct EvictShared {
  int hist[2][kSelBins];                                   // this CTA's, of alternate rounds; the next round's is zero
  int sums[kSelBins];                                      // large clusters: its share of the cluster's bins, summed over the CTAs
  int share;                                               // sum of its share
  int chunk[kEvictWarps];
  int found[3];
  int n_prot, n_few;                                       // protected entries of the CTA; keys in `few`
  uint32_t few[kEvictFew];
  int above[kEvictWarps], equal[kEvictWarps];
  int totals[2];                                           // CTA: keys above, keys equal
  int offset;                                              // (sequence, head)'s place in the list
};

__host__ __device__ constexpr uint32_t evict_smem_bytes(int slice) { return (uint32_t)slice * 4u + (uint32_t)sizeof(EvictShared) + 16u; }
// Entries of a CTA's slice.
LKV_HOST_DEVICE inline int evict_slice(long long len, int n) { return (int)((len + n - 1) / n + 31) / 32 * 32; }

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

constexpr uint32_t kEvictProtected = 0xFFFFFFFFu;

__global__ void __launch_bounds__(kEvictThreads, 1) paged_evict_kernel(const PagedEvictArgs a) {
  extern __shared__ __align__(16) uint8_t esm_raw[];
  EvictShared& sh = *reinterpret_cast<EvictShared*>(esm_raw);
  uint32_t* const keys = reinterpret_cast<uint32_t*>(esm_raw + (sizeof(EvictShared) + 15) / 16 * 16);
  const PagedPool& p = a.pool;
  const int C = gridDim.x, rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto remote = [&](const void* at, int r) { return ld_cluster_u32(cluster_addr(smem_u32(at), r)); };
  for (int i = tid; i < 2 * kSelBins; i += kEvictThreads) sh.hist[0][i] = 0;
  if (tid == 0) sh.n_prot = sh.n_few = 0;
  __syncthreads();
  grid_dependency_wait();
  allow_dependents();

  const int len = p.length(b), keep = a.keep;
  const int held = p.lens[b], newest = p.seen[b] - a.recent;
  if (warp == 1) {
    // the place of this (sequence, head)'s pairs in the list: at most min(keep, len - keep) per head of the sequences before
    long long pairs = 0;
    for (int i = lane; i < b; i += 32) pairs += max(0, min(keep, p.length(i) - keep));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) pairs += __shfl_xor_sync(0xffffffffu, pairs, off);
    const long long most = max(0, min(keep, len - keep)), at = pairs * p.H + (long long)h * most;
    // the list is as large as a pool whose pages are not shared can need; a sequence goes by all of its heads, in each of them
    if (lane == 0) sh.offset = (pairs + most) * p.H <= a.n_moves ? (int)at : -1;
  }
  if (len != held && tid == 0) record_status(p.status, kPagedBadPage);
  if (len <= keep) {                                       // the same in all of the cluster
    if (rank == 0 && tid == 0) a.lists[b * p.H + h] = make_int2(0, 0);
    return;
  }

  // ---- 1. keys ----------------------------------------------------------------------------------
  const int slice = evict_slice(len, C), lo_i = min(len, rank * slice), n = min(len - lo_i, slice);
  constexpr int kFirst = 32 - kSelBinBits;                 // the first round's bins: the highest bits
  int prot = 0;
  constexpr int kAtOnce = 4;                               // keys of a thread under way together: nothing is loaded under a condition
  for (int i0 = tid; i0 < n; i0 += kAtOnce * kEvictThreads) {
    int page[kAtOnce], at[kAtOnce];
    float x[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) page[j] = p.page(b, lo_i + min(i0 + j * kEvictThreads, n - 1));
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int i = lo_i + min(i0 + j * kEvictThreads, n - 1);
      const bool ok = (unsigned)page[j] < (unsigned)p.n_pages;
      const long long slot = (((long long)(ok ? page[j] : 0) * p.H + h) << p.page_shift) + (i & (p.page_size() - 1));
      x[j] = a.rows.weights[slot];
      at[j] = a.rows.pos[slot];
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int i = i0 + j * kEvictThreads;
      if (i >= n) continue;
      const bool bad = (unsigned)page[j] >= (unsigned)p.n_pages;     // counts as -inf
      if (bad) record_status(p.status, kPagedBadPage);
      const bool safe = !bad && ((at[j] >= 0 && (at[j] < a.anchors || at[j] >= newest)) || x[j] == INFINITY);
      const uint32_t key = safe ? kEvictProtected : orderable_f32(bad || x[j] != x[j] ? -INFINITY : x[j] + 0.f);   // + 0: -0 is 0
      keys[i] = key;
      prot += safe;
      if (!safe) atomicAdd(&sh.hist[0][key >> kFirst], 1);
    }
  }
  prot = __reduce_add_sync(0xffffffffu, prot);
  if (lane == 0 && prot) atomicAdd(&sh.n_prot, prot);
  if (C > 1) cluster_sync(); else __syncthreads();         // the first histograms and the numbers of protected entries are there
  prot = __reduce_add_sync(0xffffffffu, lane < C ? (int)remote(&sh.n_prot, lane) : 0);

  // ---- 2. the keep-th largest key ----------------------------------------------------------------
  // kept: keys from `from` on, and of those equal to `tie` the first `ties` in index order
  uint32_t from = kEvictProtected, tie = kEvictProtected;
  int ties = 0;                                            // 0: none goes by its index
  const bool any_above = prot < keep;
  if (!any_above) {
    ties = keep;                                           // of the protected ones themselves
  } else {
    int need = keep - prot;                                // of len - prot > need unprotected ones
    uint32_t base = 0, last = kEvictProtected - 1u;        // undecided: keys in [base, last]
    int shift = kFirst;                                    // a bin has 2^shift of them
    const int per = kSelBins / C;                          // large clusters: bins of a CTA's share
    for (int round = 0;; ++round) {
      int* const hist = sh.hist[round & 1];
      if (round > 0) {
        for (int i = tid; i < n; i += kEvictThreads) {
          const uint32_t key = keys[i];
          if (key >= base && key <= last) atomicAdd(&hist[(key - base) >> shift], 1);
        }
        if (C > 1) cluster_sync(); else __syncthreads();
      }
      // bins from high to low, a warp takes a run of them: of the whole histogram, which every CTA of a small cluster adds up for
      // itself, or of the share that holds the need-th from the top
      constexpr int kMost = kSelBins / kEvictThreads;
      int c[kMost], bins = kSelBins, share = 0, before = 0;
      if (C <= 4) {
#pragma unroll
        for (int k = 0; k < kMost; ++k) {
          const int i = kSelBins - 1 - (tid * kMost + k);
          c[k] = C == 1 ? hist[i] : 0;
          if (C > 1) {
            int x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = (int)remote(&hist[i], min(r, C - 1));   // together
#pragma unroll
            for (int r = 0; r < 4; ++r) if (r < C) c[k] += x[r];
          }
        }
      } else {
        // this CTA's share: bins [rank * per, (rank + 1) * per)
        int mine = 0;
        for (int i = tid; i < per; i += kEvictThreads) {
          int v = 0;
          for (int r0 = 0; r0 < C; r0 += 4) {              // four reads under way together
            int x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = (int)remote(&hist[rank * per + i], min(r0 + r, C - 1));
#pragma unroll
            for (int r = 0; r < 4; ++r) if (r0 + r < C) v += x[r];
          }
          sh.sums[i] = v;
          mine += v;
        }
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) sh.chunk[warp] = mine;
        __syncthreads();
        if (warp == 0) {
          const int s = __reduce_add_sync(0xffffffffu, lane < kEvictWarps ? sh.chunk[lane] : 0);
          if (lane == 0) sh.share = s;
        }
        cluster_sync();                                    // sums are written
        const int v = lane < C ? (int)remote(&sh.share, C - 1 - lane) : 0;
        const int incl = warp_inclusive(v, lane);
        const int who = (__ffs(__ballot_sync(0xffffffffu, lane < C && incl >= need)) - 1) & 31;
        share = C - 1 - who;
        before = __shfl_sync(0xffffffffu, incl - v, who);
        bins = per;
#pragma unroll
        for (int k = 0; k < kMost; ++k) c[k] = 0;
        if (tid < per) c[0] = (int)remote(&sh.sums[per - 1 - tid], share);   // per <= kEvictThreads
      }
      int sum = 0;
#pragma unroll
      for (int k = 0; k < kMost; ++k) sum += c[k];
      const int wsum = __reduce_add_sync(0xffffffffu, sum);
      // the other histogram: all of the cluster have read it, in the round before this one's barrier
      for (int i = tid; i < kSelBins; i += kEvictThreads) sh.hist[(round + 1) & 1][i] = 0;
      __syncthreads();                                     // sh.chunk is read
      if (lane == 0) sh.chunk[warp] = wsum;
      __syncthreads();
      {
        const int x = lane < kEvictWarps ? sh.chunk[lane] : 0;
        const int incl = warp_inclusive(x, lane);
        int run = before + __shfl_sync(0xffffffffu, incl - x, warp);
        run += warp_inclusive(sum, lane) - sum;            // keys in higher bins than this thread's
#pragma unroll
        for (int k = 0; k < kMost; ++k) {
          if (run < need && need <= run + c[k]) {
            sh.found[0] = C <= 4 ? kSelBins - 1 - (tid * kMost + k) : share * per + bins - 1 - tid;
            sh.found[1] = need - run;
            sh.found[2] = c[k];
          }
          run += c[k];
        }
      }
      __syncthreads();
      const uint32_t bin = (uint32_t)sh.found[0];
      need = sh.found[1];
      const int held_in = sh.found[2];
      base += bin << shift;
      if (need == held_in) {                               // the whole bin
        from = base;
        break;
      }
      if (shift == 0) {                                    // equal keys: the ones of lowest index
        from = base + 1;                                   // base < kEvictProtected
        tie = base;
        ties = need;
        break;
      }
      last = base + (1u << shift) - 1u;                    // below kEvictProtected
      if (C == 1 && held_in <= kEvictFew) {
        for (int i0 = warp * 32; i0 < n; i0 += kEvictThreads) {
          const int i = i0 + lane;
          const uint32_t key = i < n ? keys[i] : kEvictProtected;
          const bool in = key >= base && key <= last;
          const uint32_t mask = __ballot_sync(0xffffffffu, in);
          int at = 0;
          if (lane == 0 && mask) at = atomicAdd(&sh.n_few, __popc(mask));
          at = __shfl_sync(0xffffffffu, at, 0) + __popc(mask & ((1u << lane) - 1u));
          if (in) sh.few[at] = key;                        // in any order
        }
        __syncthreads();
        if (tid < held_in) {
          const uint32_t key = sh.few[tid];
          int over = 0, same = 0;
#pragma unroll 4
          for (int i = 0; i < held_in; ++i) {
            over += sh.few[i] > key;
            same += sh.few[i] == key;
          }
          if (over < need && need <= over + same) {        // the threads that hold the need-th agree
            sh.found[0] = (int)key;
            sh.found[1] = need - over;
          }
        }
        __syncthreads();
        tie = (uint32_t)sh.found[0];
        ties = sh.found[1];
        from = tie + 1;
        break;
      }
      shift -= shift > kSelBinBits ? kSelBinBits : shift;  // 21, 10, 0
    }
  }

  // ---- 3. ranks and the list of moves -------------------------------------------------------------
  const int run_n = (slice / 32 + kEvictWarps - 1) / kEvictWarps * 32, w_lo = min(n, warp * run_n), w_hi = min(n, w_lo + run_n);
  {
    int above = 0, equal = 0;
    for (int i = w_lo + lane; i < w_hi; i += 32) {
      const uint32_t key = keys[i];
      above += any_above && key >= from;
      equal += ties > 0 && key == tie;
    }
    above = __reduce_add_sync(0xffffffffu, above);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane == 0) { sh.above[warp] = above; sh.equal[warp] = equal; }
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
      cluster_arrive();                                    // the last look at another CTA's shared memory
    }
  }
  const bool room = sh.offset >= 0;
  int2* const list = a.moves + (room ? sh.offset : 0);
  for (int i0 = w_lo; i0 < w_hi; i0 += 32) {
    const int i = i0 + lane, e = lo_i + i;                 // entry
    const bool in = i < w_hi;
    const uint32_t key = in ? keys[i] : 0u;
    const bool is_above = in && any_above && key >= from, is_equal = in && ties > 0 && key == tie;
    const uint32_t ma = __ballot_sync(0xffffffffu, is_above), me = __ballot_sync(0xffffffffu, is_equal);
    const uint32_t below = (1u << lane) - 1u;
    const int eq = equal0 + __popc(me & below);
    const bool kept = is_above || (is_equal && eq < ties);
    const int kept_before = above0 + __popc(ma & below) + min(eq, ties);
    const bool hole = in && e < keep && !kept, mover = in && e >= keep && kept;
    if (room && (hole || mover)) {
      const int page = p.page(b, e);                       // of a page out of range, recorded above: no slot
      const int slot = (unsigned)page < (unsigned)p.n_pages ? (page << p.page_shift) + (e & (p.page_size() - 1)) : -1;
      if (hole) list[e - kept_before].x = slot;
      else list[keep - 1 - kept_before].y = slot;
    }
    if (in && e == keep) {                                 // entry `keep` knows how many holes are before it
      a.lists[b * p.H + h] = make_int2(sh.offset, room ? keep - kept_before : 0);
      if (!room) record_status(p.status, kStatusCapacity);
    }
    above0 += __popc(ma);
    equal0 += __popc(me);
  }
  __syncwarp();
  if (C > 1) cluster_wait();                               // no CTA leaves while another may read its shared memory
}

constexpr int kMoveThreads = 256;

// Moves the rows of the lists, one (sequence, KV head) per blockIdx (z, y), dealt to the warps of its gridDim.x CTAs.
template <int VECS>
__global__ void __launch_bounds__(kMoveThreads, 4) paged_move_kernel(const PagedEvictArgs a) {
  constexpr int kLanes = VECS == 8 ? 16 : 32, kPerWarp = 32 / kLanes;   // lanes of a move: half on the key, half on the value
  constexpr int kHalf = kLanes / 2, kTimes = VECS / kHalf, N = kTimes == 2 ? 2 : 4;   // 16-byte vectors of a lane; moves of a thread under way together
  const PagedPool& p = a.pool;
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, l = lane % kLanes;
  grid_dependency_wait();
  allow_dependents();
  const int2 of = a.lists[b * p.H + h];
  if (blockIdx.x == 0 && h == 0 && tid == 0 && of.x >= 0 && p.length(b) > a.keep) p.lens[b] = a.keep;   // nothing else here goes by lengths
  const int2* const list = a.moves + of.x;
  uint16_t* const side = l < kHalf ? a.rows.K : a.rows.V;
  int* const word = l < kHalf ? reinterpret_cast<int*>(a.rows.weights) : a.rows.pos;     // moved by lanes 0 and kHalf
  const int v0 = (l % kHalf) * 8;
  auto row = [&](int slot) {
    return (slot >> p.page_shift) * a.rows.s_page + h * a.rows.s_head + (slot & (p.page_size() - 1)) * a.rows.s_row + v0;
  };
  auto entry = [&](int slot) { return (((long long)(slot >> p.page_shift) * p.H + h) << p.page_shift) + (slot & (p.page_size() - 1)); };
  const int step = gridDim.x * (kMoveThreads / 32) * kPerWarp;
  for (int r0 = (blockIdx.x * (kMoveThreads / 32) + (tid >> 5)) * kPerWarp + lane / kLanes; r0 < of.y; r0 += N * step) {
    int2 mv[N];
    uint4 x[N][kTimes];
    int y[N];
#pragma unroll
    for (int j = 0; j < N; ++j) mv[j] = __ldcg(list + min(r0 + j * step, of.y - 1));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int from = max(mv[j].y, 0);
#pragma unroll
      for (int k = 0; k < kTimes; ++k) x[j][k] = *reinterpret_cast<const uint4*>(side + row(from) + k * kHalf * 8);
      y[j] = word[entry(from)];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (r0 + j * step >= of.y || mv[j].x < 0 || mv[j].y < 0) continue;
#pragma unroll
      for (int k = 0; k < kTimes; ++k) *reinterpret_cast<uint4*>(side + row(mv[j].x) + k * kHalf * 8) = x[j][k];
      if (l % kHalf == 0) word[entry(mv[j].x)] = y[j];
    }
  }
}

}  // namespace lkv

// Attention of one new token per sequence over a paged cache. For every sequence b with len_b entries, entry i in row
// i mod P of page table[b][i / P], and every query head g of KV head h:
//   x_i = <q_g, k_i> * scale,   lse = log sum_i exp(x_i),   out = sum_i exp(x_i - lse) v_i      (len_b = 0: 0, -inf)
// and, where the cache accumulates weights, w_i += sum over the group's heads of exp(x_i - lse).
//
//   paged_attn_kernel     every key and value row is read once: bound by HBM. The tiles (64 entries of one KV head) of all
//                         sequences are one list, cut into equal shares, one per CTA: the lengths lie on the device, so no
//                         host-side plan is needed, ragged batches balance and a captured graph follows the lengths. A
//                         producer warp reads page numbers and brings tiles into a ring of stages with TMA, one box per page
//                         and 64 columns (128-byte swizzle); a page that is shorter than a tile takes as many boxes as the
//                         tile has pages. Four consumer warps own 16 rows of every tile each: scores S^T = K Q^T,
//                         O^T += V^T P^T as m16n8k16 MMAs with the heads on the 8-wide side. A (sequence, head) that
//                         crosses CTAs leaves partials; the CTA that finishes last joins them in a fixed order, so
//                         results depend on lengths and shapes alone. 64 sequences of 4000 to 24000 entries, 8 heads of
//                         four queries (2.94 GB): 442 us, 6.6 TB/s; one of 131,071 87.2 us, 6.2 TB/s (a plain reduction over 2 GB reads at
//                         6.85, a copy moves 6.52). About 7 us are not
//                         streaming: the chain of length, page and first tile (3.5), merge, partial and join (3.5), each a
//                         few trips to L2 of 0.5 to 0.9 us; small calls are made of them (1637 entries 9.6 us).
//   paged_weights_kernel  exp(x_i - lse) from the scores that the first kernel left (4 bytes per query head and entry
//                         against the 512 of its key and value), added to the entries' weights.
//
// Numerators are taken relative to the maximum of their own 16 (or 32) rows, where they are at most 1, and the rows' sums are
// added to the running ones in fp32, rounded to nearest, with the factor between the two maxima. The MMAs' accumulators do not
// round to nearest: over the few rows of a block that does not matter, over thousands it would be a drift. bf16: a numerator
// is split into three terms, which hold all 24 bits. fp16: two terms of the numerator times 2^15 hold 22 bits down to
// 2^-18 of the block's largest, 2^-40 of it below that.
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "decode_attn.cuh"
#include "launch_rules.h"
#include "ptx.cuh"
#include "stream_gemm.cuh"

namespace lkv {

constexpr int kPagedWarps = 4;                             // consumer warps, 16 rows of every tile each
constexpr int kPagedThreads = (kPagedWarps + 1) * 32;
constexpr float kPagedLeast = -3.4e38f;                    // stands for a maximum of -inf where it is subtracted: all powers are 0
constexpr int kPagedBadPage = 1;                           // status of a page number or length out of range: LASER_KV_ERR_INVALID_ARG

struct PagedPool {                                         // what all kernels of a paged cache are told about it
  const int* table;                                        // [n_seqs][max_pages]
  int* lens;                                               // [n_seqs]
  int* seen;                                               // [n_seqs]
  int n_seqs, H, n_pages, max_pages, page_shift;
  int* status;
  __device__ __forceinline__ int page_size() const { return 1 << page_shift; }
  // Entries of a sequence. A length that the table cannot hold counts as none: it takes no part of what sequences share, the list
  // of tiles, the room for scores and the list of moves.
  __device__ __forceinline__ int length(int b) const {
    const int held = lens[b];
    return (unsigned)held <= (unsigned)(max_pages << page_shift) ? held : 0;
  }
  __device__ __forceinline__ int page(int b, int i) const { return table[(long long)b * max_pages + (i >> page_shift)]; }
};

struct PagedAttnArgs {
  PagedPool pool;
  const uint16_t* Q;                                       // [n_seqs][H_q][D] via strides
  long long qs_b, qs_h;
  void* out;                                               // [n_seqs][H_q][D], fp32 or the queries' type
  float* lse;                                              // [n_seqs][H_q] or NULL
  float* lse2;                                             // the same in log2 units, for paged_weights_kernel; NULL without
  float* scores;                                           // [tile of all heads][64][Gs]; NULL without weights
  float* weights;                                          // [n_pages][H][page_size]
  int2* score_at;                                          // [units of all heads] sequence and KV head of a tile of `scores`, tile of the sequence
  int* score_units;                                        // units in use; behind it, nonzero: a wait of an attention ran out (8-byte aligned)
  int score_tiles;                                         // units that `scores` and `score_at` hold
  float* part;                                             // [2][grid] partials
  int* tickets;                                            // [n_seqs][H][head blocks] parts that are done; zero between calls
  int G, Gs, head_blocks;                                  // query heads per KV head, up to a power of two from 4 on; blocks of NG * 8 of them
  int out16;
  float scale_log2e;
  uint32_t polls, poll_ns;                                 // budget of the waits for tiles, as of mbar_wait
};

template <int D>
__host__ __device__ constexpr int paged_stage_bytes() { return kDecTile * D * 4; }
// 192 KB of tiles in flight per SM, of three, two or one CTAs.
template <int D>
__host__ __device__ constexpr int paged_stages() { return D == 64 ? 4 : 3; }
template <int D>
__host__ __device__ constexpr int paged_ctas_per_sm() { return D == 64 ? 3 : 256 / D; }
template <int D, int NG>
__host__ __device__ constexpr int paged_part_floats() { return NG * 8 * (D + 2); }
template <int D, int NG>
__host__ __device__ constexpr uint32_t paged_smem_bytes() {
  return 1024u + paged_stages<D>() * paged_stage_bytes<D>() + 2u * D / 16 * 512u + 2u * kPagedWarps * 8u * 4u + (2u * paged_stages<D>() + 2u) * 8u + 16u;
}

// D (16x8, fp32) += A (16x16, row) * B (16x8, col). Not volatile: the compiler may interleave independent ones.
template <bool HALF>
__device__ __forceinline__ void paged_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if constexpr (HALF)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t paged_trans(uint32_t x) {       // as movmatrix_trans
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool HALF>
__device__ __forceinline__ uint32_t paged_pack(float lo, float hi) {
  if constexpr (HALF) {
    uint32_t y;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
  } else {
    return pack_bf16x2(lo, hi);
  }
}
template <bool HALF>
__device__ __forceinline__ float2 paged_unpack(uint32_t x) {
  if constexpr (HALF) return __half22float2(*reinterpret_cast<const __half2*>(&x));
  else return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
}
__device__ __forceinline__ void paged_consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kPagedWarps * 32) : "memory"); }

// Where a warp is in the list: sequences one after the other, in each `heads` items, in each kPagedItemUnits units for the
// item itself and one for each of the sequence's tiles.
struct PagedWalk {
  int b, head;                                             // sequence, item in it
  int len, n_tiles;                                        // of the sequence
  int before;                                              // units per item of the sequences before this one
  int unit0;                                               // the item's first unit
  bool whole;                                              // all items count alike
  __device__ __forceinline__ int units() const { return whole ? kPagedWholeUnits : n_tiles + kPagedItemUnits; }
  // The item's tiles in the units [begin, stop) are [first, last); none where first >= last.
  __device__ __forceinline__ int first(int begin) const { return max(0, begin - unit0 - kPagedItemUnits); }
  __device__ __forceinline__ int last(int stop) const { return min(n_tiles, stop - unit0 - kPagedItemUnits); }
  // The next item starts before `stop`, or there is none to go on with.
  __device__ __forceinline__ bool next(const PagedPool& p, int heads, int stop) {
    unit0 += units();
    if (unit0 >= stop) return false;
    if (++head < heads) return true;
    head = 0;
    before += units();
    do {
      ++b;
      len = p.length(b);                                   // the list goes on: there is a sequence with entries
      n_tiles = (len + kDecTile - 1) / kDecTile;
    } while (n_tiles == 0);
    return true;
  }
};

__device__ __forceinline__ int paged_units(int len, bool whole) {
  return len <= 0 ? 0 : whole ? kPagedWholeUnits : (len + kDecTile - 1) / kDecTile + kPagedItemUnits;
}

__device__ __forceinline__ int warp_inclusive(int x, int lane) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int n = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += n;
  }
  return x;
}
// Units per item over all sequences, and up to and with this lane's; called by whole warps. A lane has `per` sequences in a row: one,
// or, of more than 32, as many blocks of 32 as it takes.
struct PagedSum {
  int per, incl, mine, total, len;                         // len: the lane's only sequence's, where per is 1
  bool whole;                                              // no sequence has more than kPagedWhole tiles
  __device__ __forceinline__ PagedSum(const PagedPool& p, int lane) {
    int longest = 0;
    len = 0;
    if (p.n_seqs <= 32) {
      per = 1;
      len = longest = lane < p.n_seqs ? p.length(lane) : 0;
      whole = __reduce_max_sync(0xffffffffu, longest) <= kPagedWhole * kDecTile;
      mine = paged_units(len, whole);
    } else {
      const int blocks = (p.n_seqs + 1023) >> 10;          // of a lane
      per = 32 * blocks;
      int all = 0, alike = 0;
      const int n = (p.n_seqs + 31) >> 5;
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const int x = p.length(min(32 * k + lane, p.n_seqs - 1)), here = 32 * k + lane < p.n_seqs ? x : 0;
        longest = max(longest, here);
        const int s = __reduce_add_sync(0xffffffffu, paged_units(here, false)), w = kPagedWholeUnits * __popc(__ballot_sync(0xffffffffu, here > 0));
        if (k / blocks == lane) { all += s; alike += w; }
      }
      whole = __reduce_max_sync(0xffffffffu, longest) <= kPagedWhole * kDecTile;
      mine = whole ? alike : all;
    }
    incl = warp_inclusive(mine, lane);
    total = __shfl_sync(0xffffffffu, incl, 31);
  }
};
// The place of unit `at` (below total * heads) of the list.
__device__ __forceinline__ PagedWalk paged_seek(const PagedPool& p, int lane, const PagedSum& sum, int heads, int at) {
  const int q = at / heads;                                // the sequence: the first with more than q units per item up to its end
  const int who = (__ffs(__ballot_sync(0xffffffffu, sum.incl > q)) - 1) & 31;
  PagedWalk w;
  w.before = __shfl_sync(0xffffffffu, sum.incl - sum.mine, who);
  w.b = who * sum.per;
  w.len = __shfl_sync(0xffffffffu, sum.len, who);
  w.whole = sum.whole;
  if (sum.per > 1) {
    for (;;) {
      const int i = w.b + lane;
      const int len = i < p.n_seqs ? p.length(i) : 0, u = paged_units(len, sum.whole);
      const int incl = w.before + warp_inclusive(u, lane);
      const uint32_t found = __ballot_sync(0xffffffffu, incl > q);
      if (found || w.b + 32 >= p.n_seqs) {                 // `at` is in the list: found
        const int l = (__ffs(found) - 1) & 31;
        w.b += l;
        w.before = __shfl_sync(0xffffffffu, incl - u, l);
        w.len = __shfl_sync(0xffffffffu, len, l);
        break;
      }
      w.before = __shfl_sync(0xffffffffu, incl, 31);
      w.b += 32;
    }
  }
  w.n_tiles = (w.len + kDecTile - 1) / kDecTile;
  w.head = (at - w.before * heads) / w.units();
  w.unit0 = w.before * heads + w.head * w.units();
  return w;
}

// TMA load of what is read once: its lines leave the L2 cache before the others, scores and old weights among them.
__device__ __forceinline__ uint64_t l2_evict_first() {
  uint64_t policy;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ void tma_load_4d_once(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2, int c3,
                                                 uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%3, %4, %5, %6}], [%2], %7;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void st_shared_zero(uint32_t addr) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0) : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ int atom_add_acq_rel(int* p, int v) {
  int old;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
  return old;
}

template <bool HALF, int D, int NG>
__global__ void __launch_bounds__(kPagedThreads, paged_ctas_per_sm<D>())
paged_attn_kernel(const __grid_constant__ CUtensorMap map_k,      // keys: (D, page_size, H, n_pages), box (64, min(page_size, 64), 1, 1)
                  const __grid_constant__ CUtensorMap map_v, const PagedAttnArgs a) {
  constexpr int kStages = paged_stages<D>(), kBox = kDecBoxBytes, kHalf = kDecTile * D * 2, MT = D / 16;
  extern __shared__ uint8_t psm_raw[];
  const uint32_t base = (smem_u32(psm_raw) + 1023u) & ~1023u;
  uint8_t* const gen = psm_raw + (base - smem_u32(psm_raw));
  float4* const red = reinterpret_cast<float4*>(gen + kStages * paged_stage_bytes<D>());   // [2][MT][32]: merge of the warps
  float* const wm = reinterpret_cast<float*>(red + 2 * MT * 32);                           // [warps][8] maxima
  float* const wl = wm + kPagedWarps * 8;                                                  // sums
  int* const s_last = reinterpret_cast<int*>(wl + kPagedWarps * 8);
  const uint32_t bars = smem_u32(s_last) + 16u;
  auto bar_full = [&](int s) { return bars + 8u * s; };
  auto bar_empty = [&](int s) { return bars + 8u * (kStages + s); };
  auto bar_join = [&](int s) { return bars + 8u * (2 * kStages + s); };
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const PagedPool& p = a.pool;
  const int heads = p.H * a.head_blocks;
  auto give_up = [&]() {                                           // one thread: a wait ran out, the call's results are incomplete
    record_status(p.status, kStatusTimeout);
    if (a.scores) a.score_units[1] = 1;                            // no weight grows by them
  };

  if (tid == kPagedWarps * 32) {
    for (int s = 0; s < kStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), kPagedWarps); }
    for (int s = 0; s < 2; ++s) mbar_init(bar_join(s), 1);
    fence_mbar_init();
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  // Lengths, page numbers and queries are asked for one after the other: the L2 cache gets them together and ahead.
  {
    const long long at = ((long long)blockIdx.x * kPagedThreads + tid) * 128, table = (long long)p.n_seqs * p.max_pages * 4;
    if (at < table) prefetch_l2(reinterpret_cast<const char*>(p.table) + at);
    if (at < p.n_seqs * 4) prefetch_l2(reinterpret_cast<const char*>(p.lens) + at);
  }
  __syncthreads();                                                 // the barriers are set up
  // launched beside the kernel ahead in the stream: nothing is read or written before that is complete
  grid_dependency_wait();
  allow_dependents();

  const PagedSum sum(p, lane);
  const PagedShares shares(sum.total * heads, (int)gridDim.x, sum.whole);
  const int cta = blockIdx.x;
  const int begin = cta < shares.n ? shares.begin(cta) : 0, stop = cta < shares.n ? shares.begin(cta + 1) : 0;
  bool more = begin < stop;
  PagedWalk w{};
  if (more) w = paged_seek(p, lane, sum, heads, begin);
  if (a.scores && cta == 0 && tid == 0) *a.score_units = sum.total * p.H;

  if (warp == kPagedWarps) {
    // ---- producer ---------------------------------------------------------------------------------
    const int rows_shift = min(p.page_shift, 6);                   // rows of a box
    const int per_shift = 6 - rows_shift;                          // pages of a tile
    const uint64_t once = l2_evict_first();
    int st = 0, round = 0;
    for (bool ok = true; ok && more; more = w.next(p, heads, stop)) {
      const int first = w.first(begin), end = w.last(stop), h = w.head / a.head_blocks;
      const int last_page = (w.len - 1) >> p.page_shift;
      int ids = 0;
      for (int t = first; t < end; ++t) {
        const int chunk = 32 >> per_shift, k = (t - first) & (chunk - 1);   // tiles whose page numbers the lanes hold
        if (k == 0) {
          const int at = per_shift ? (t << per_shift) + lane : ((t + lane) << 6) >> p.page_shift;
          ids = at <= last_page ? p.table[(long long)w.b * p.max_pages + at] : 0;
          if ((unsigned)ids >= (unsigned)p.n_pages) {              // a box of that page is read as zeros
            record_status(p.status, kPagedBadPage);
            ids = p.n_pages;
          }
        }
        const int rows = min(kDecTile, w.len - t * kDecTile), pages = (rows + (1 << rows_shift) - 1) >> rows_shift;
        const int id = __shfl_sync(0xffffffffu, ids, (k << per_shift) + (lane & ((1 << per_shift) - 1)));
        if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(bar_empty(st), (uint32_t)(round - 1) & 1u))) {
          if (lane == 0) give_up();
          ok = false;                                              // the consumers' waits run out, too
          break;
        }
        if (lane == 0) mbar_expect_tx(bar_full(st), (uint32_t)pages << (rows_shift + 7 + (D == 64 ? 1 : D == 128 ? 2 : 3)));
        __syncwarp();
        if (a.scores) {                                            // for paged_weights_kernel: the old weights, eight to a sector
          const int e = (lane & 7) << 3, pg = per_shift ? e >> rows_shift : 0;
          const int wid = __shfl_sync(0xffffffffu, ids, (k << per_shift) + pg);
          if (lane < 8 && e < rows && wid < p.n_pages)
            prefetch_l2(a.weights + (((long long)wid * p.H + h) << p.page_shift) + (((t << 6) + e) & (p.page_size() - 1)));
        }
        if (lane < pages) {
          const uint32_t dst = base + st * paged_stage_bytes<D>() + ((uint32_t)lane << (rows_shift + 7));
          const int row = per_shift ? 0 : (t << 6) & (p.page_size() - 1);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) tma_load_4d_once(dst + c * kBox, &map_k, bar_full(st), 64 * c, row, h, id, once);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) tma_load_4d_once(dst + kHalf + c * kBox, &map_v, bar_full(st), 64 * c, row, h, id, once);
        }
        __syncwarp();
        if (++st == kStages) { st = 0; ++round; }
      }
    }
    // no tile is still on its way here when the CTA ends, also where a consumer has given up
    for (int n = round * kStages + st - 1, k = 0; n >= 0 && k < kStages; --n, ++k) mbar_wait(bar_full(n % kStages), (uint32_t)(n / kStages) & 1u);
    return;
  }

  // ---- consumers ------------------------------------------------------------------------------------
  // With one set of eight heads a warp has 16 rows of every tile; with two, a pair of warps has a set, a warp of it 32 rows: a
  // warp's registers hold eight heads either way.
  constexpr int kTeam = kPagedWarps / NG;                          // warps of a set
  const int g = lane >> 2, c = lane & 3;                           // fragment coordinates, as in decode_split_kernel
  const int team = warp / kTeam, mate = warp % kTeam;
  auto first_head = [&](int head, int h) { return ((head - h * a.head_blocks) * NG + team) * 8; };   // of the warp's set, in the group

  uint32_t qb[MT][2];                                              // B fragments of Q^T, heads past G are zero
  auto load_q = [&]() {                                            // without a condition, so that all loads are under way together
    const int h = w.head / a.head_blocks, hg = first_head(w.head, h) + g;
    const uint32_t keep = hg < a.G ? 0xFFFFFFFFu : 0u;
    const uint16_t* q = a.Q + w.b * a.qs_b + ((long long)h * a.G + min(hg, a.G - 1)) * a.qs_h + 2 * c;
#pragma unroll
    for (int ks = 0; ks < MT; ++ks) {
      qb[ks][0] = *reinterpret_cast<const uint32_t*>(q + 16 * ks);
      qb[ks][1] = *reinterpret_cast<const uint32_t*>(q + 16 * ks + 8);
    }
#pragma unroll
    for (int ks = 0; ks < MT; ++ks) { qb[ks][0] &= keep; qb[ks][1] &= keep; }
  };
  if (more) load_q();

  // rows without entries
  for (int b = cta; b < p.n_seqs; b += gridDim.x) {
    if (p.length(b) != p.lens[b] && tid == 0) record_status(p.status, kPagedBadPage);
    if (p.length(b) > 0) continue;
    const int n = p.H * a.G * D;
    if (a.out16) {
      uint32_t* o = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + (long long)b * n);
      for (int i = tid; i < n / 2; i += kPagedWarps * 32) o[i] = 0u;
    } else {
      float* o = static_cast<float*>(a.out) + (long long)b * n;
      for (int i = tid; i < n; i += kPagedWarps * 32) o[i] = 0.f;
    }
    if (a.lse) for (int i = tid; i < p.H * a.G; i += kPagedWarps * 32) a.lse[(long long)b * p.H * a.G + i] = -INFINITY;
  }

  float o[MT][4], m[2], l[2];
  auto clear = [&]() {
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[mt][i] = 0.f;
  };
  // the results of a team's warps are combined in its first one: sums in a fixed order
  auto merge_warps = [&]() {
    if (g == 0) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        wm[warp * 8 + 2 * c + x] = m[x];
        wl[warp * 8 + 2 * c + x] = l[x];
      }
    }
    paged_consumers_sync();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int at = team * kTeam * 8 + 2 * c + x;
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int wi = 0; wi < kTeam; ++wi) top = fmaxf(top, wm[wi * 8 + at]);
      const float ref = fmaxf(top, kPagedLeast);
#pragma unroll
      for (int wi = 0; wi < kTeam; ++wi) sum = fmaf(wl[wi * 8 + at], ex2_approx(wm[wi * 8 + at] - ref), sum);
      const float f = ex2_approx(m[x] - ref);
      m[x] = top;
      l[x] = sum;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) { o[mt][x] *= f; o[mt][x + 2] *= f; }
    }
    auto put = [&](int slot) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) red[(slot * MT + mt) * 32 + lane] = make_float4(o[mt][0], o[mt][1], o[mt][2], o[mt][3]);
    };
    auto add = [&](int slot) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const float4 v = red[(slot * MT + mt) * 32 + lane];
        o[mt][0] += v.x; o[mt][1] += v.y; o[mt][2] += v.z; o[mt][3] += v.w;
      }
    };
    if constexpr (NG == 1) {
      if (warp >= 2) put(warp - 2);
      paged_consumers_sync();
      if (warp < 2) add(warp);
      if (warp == 1) put(1);
      paged_consumers_sync();
      if (warp == 0) add(1);
    } else {
      if (mate == 1) put(team);
      paged_consumers_sync();
      if (mate == 0) add(team);
    }
  };
  auto finish = [&](int b, int head) {                             // a team's first warp: its heads' results
    const int h = head / a.head_blocks;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int hg = first_head(head, h) + 2 * c + x;
      if (hg >= a.G) continue;
      const long long row = ((long long)b * p.H + h) * a.G + hg;
      const float inv = 1.f / l[x];
      if (a.out16) {
        uint16_t* dst = static_cast<uint16_t*>(a.out) + row * D + g;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const uint32_t y = paged_pack<HALF>(o[mt][x] * inv, o[mt][x + 2] * inv);
          dst[16 * mt] = (uint16_t)y;
          dst[16 * mt + 8] = (uint16_t)(y >> 16);
        }
      } else {
        float* dst = static_cast<float*>(a.out) + row * D + g;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          dst[16 * mt] = o[mt][x] * inv;
          dst[16 * mt + 8] = o[mt][x + 2] * inv;
        }
      }
      if (g == 0) {
        const float z = m[x] + log2f(l[x]);
        if (a.lse) a.lse[row] = z * 0.6931471805599453f;
        if (a.lse2) a.lse2[row] = z;
      }
    }
  };

  int st = 0, round = 0;
  int gone = 0;                                                    // 1: a wait ran out, the list is walked, nothing is computed; 2: and no tile comes
  while (more) {
    const int t0 = w.first(begin), t1 = w.last(stop);
    if (t0 >= t1) break;                                           // the share ends with units of the item itself
    const int h = w.head / a.head_blocks;
    clear();
    const int score_unit = w.before * p.H + h * w.units();           // of the item
    if (a.scores && t0 == 0 && tid < kPagedWholeUnits && (tid < kPagedItemUnits || (w.whole && tid >= kPagedItemUnits + w.n_tiles)) &&
        score_unit + tid < a.score_tiles)
      a.score_at[score_unit + tid] = make_int2(0, -1);               // units that are no tiles
    for (int t = t0; t < t1; ++t) {
      // Every warp waits for every tile, in order, also for one that it has no rows of and where it has given up: a wait tells
      // rounds of a stage apart by their parity alone, and a stage that is freed before its tile has landed is filled twice at once.
      if (!gone && !__all_sync(0xffffffffu, mbar_wait(bar_full(st), (uint32_t)round & 1u, a.polls, a.poll_ns))) {
        if (lane == 0) give_up();
        gone = 1;
      }
      if (gone == 1 && !__all_sync(0xffffffffu, mbar_wait(bar_full(st), (uint32_t)round & 1u))) gone = 2;
      const int row0 = mate * (16 * NG), rows = w.len - t * kDecTile - row0;   // the warp's first row, how many the sequence has from there on
      if (!gone && rows > 0) {
        const uint32_t k_tile = base + st * paged_stage_bytes<D>(), v_tile = k_tile + kHalf;
        float x[NG][4];                                            // scores, then numerators, of 16 rows each
#pragma unroll
        for (int r = 0; r < NG; ++r) {
          float x1[4] = {0.f, 0.f, 0.f, 0.f};                      // two chains
#pragma unroll
          for (int i = 0; i < 4; ++i) x[r][i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < MT; ks += 2) {
            uint32_t k0[4], k1[4];
            ldsm_x4(k_tile + dec_swz(row0 + 16 * r + (lane & 15), 2 * ks + (lane >> 4)), k0);
            ldsm_x4(k_tile + dec_swz(row0 + 16 * r + (lane & 15), 2 * ks + 2 + (lane >> 4)), k1);
            paged_mma<HALF>(x[r], k0, qb[ks][0], qb[ks][1]);
            paged_mma<HALF>(x1, k1, qb[ks + 1][0], qb[ks + 1][1]);
          }
          // rows past the sequence's end hold whatever the page or an earlier tile left there
#pragma unroll
          for (int i = 0; i < 4; ++i) x[r][i] = 16 * r + g + (i & 2) * 4 < rows ? (x[r][i] + x1[i]) * a.scale_log2e : -INFINITY;
        }
        const int unit = score_unit + kPagedItemUnits + t;
        if (a.scores && unit < a.score_tiles) {
          const int hg = first_head(w.head, h) + 2 * c;
          if (tid == 0) a.score_at[unit] = make_int2((int)((unsigned)w.b | (unsigned)h << 16), t);
          float* dst = a.scores + ((long long)unit * kDecTile + row0 + g) * a.Gs + hg;
          if (hg < a.G) {
#pragma unroll
            for (int r = 0; r < 2 * NG; ++r)
              if (8 * r + g < rows) *reinterpret_cast<float2*>(dst + 8 * r * a.Gs) = make_float2(x[r / 2][2 * (r & 1)], x[r / 2][2 * (r & 1) + 1]);
          }
        }
        float alpha[2], beta[2];
        bool raise = false;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          float top = fmaxf(x[0][y], x[0][y + 2]);
#pragma unroll
          for (int r = 1; r < NG; ++r) top = fmaxf(top, fmaxf(x[r][y], x[r][y + 2]));
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
          const float ref = fmaxf(top, kPagedLeast), old = m[y], now = fmaxf(old, top), run = fmaxf(now, kPagedLeast);
          alpha[y] = ex2_approx(old - run);
          beta[y] = ex2_approx(top - run);
          raise |= now > old;
          m[y] = now;
          float part = 0.f;
#pragma unroll
          for (int r = 0; r < NG; ++r) {
            x[r][y] = ex2_approx(x[r][y] - ref);
            x[r][y + 2] = ex2_approx(x[r][y + 2] - ref);
            part += x[r][y] + x[r][y + 2];
            if constexpr (HALF) {                                  // exact: powers of two
              x[r][y] *= 32768.f;
              x[r][y + 2] *= 32768.f;
            }
          }
          l[y] = fmaf(part, beta[y], l[y] * alpha[y]);
          if constexpr (HALF) beta[y] *= 1.f / 32768.f;
        }
        constexpr int kTerms = HALF ? 2 : 3;
        uint32_t pb[NG][kTerms][2];                                // B fragments of P^T, term by term
#pragma unroll
        for (int r = 0; r < NG; ++r)
#pragma unroll
          for (int term = 0; term < kTerms; ++term) {
            const uint32_t lo = paged_pack<HALF>(x[r][0], x[r][1]), hi = paged_pack<HALF>(x[r][2], x[r][3]);
            pb[r][term][0] = paged_trans(lo);
            pb[r][term][1] = paged_trans(hi);
            const float2 f0 = paged_unpack<HALF>(lo), f1 = paged_unpack<HALF>(hi);
            x[r][0] -= f0.x; x[r][1] -= f0.y; x[r][2] -= f1.x; x[r][3] -= f1.y;
          }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[mt][i] *= alpha[i & 1];
        }
        if (rows < 16 * NG) {                                      // values of rows past the end: 0 times what lies there could be NaN
          for (int i = rows * (D / 8) + lane; i < 16 * NG * (D / 8); i += 32) st_shared_zero(v_tile + dec_swz(row0 + i / (D / 8), i % (D / 8)));
          fence_proxy_async_smem();                                // before a later tile is brought here
          __syncwarp();
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < NG; ++r) {
            uint32_t vt[4];
            ldsm_x4_trans(v_tile + dec_swz(row0 + 16 * r + (lane & 7) + 8 * (lane >> 4), 2 * mt + ((lane >> 3) & 1)), vt);
#pragma unroll
            for (int term = 0; term < kTerms; ++term) paged_mma<HALF>(sum, vt, pb[r][term][0], pb[r][term][1]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) o[mt][i] = fmaf(sum[i], beta[i & 1], o[mt][i]);
        }
      }
      __syncwarp();
      if (lane == 0 && gone < 2) mbar_arrive(bar_empty(st));       // 2: the stage may yet be written, the producer gives up as well
      if (++st == kStages) { st = 0; ++round; }
    }
    // lanes with equal c hold different rows
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], off);
    // the next item's queries are on their way while this one's results are merged
    const int b = w.b, head = w.head, item = b * heads + head, n_tiles = w.n_tiles, unit0 = w.unit0;
    more = w.next(p, heads, stop) && w.last(stop) > 0;             // not just units of the next item itself
    if (more) load_q();
    merge_warps();
    if (t1 - t0 == n_tiles) {
      if (mate == 0) finish(b, head);
      continue;
    }
    // the item's parts lie in consecutive CTAs: its start in the first one's second slot, the others in their first
    constexpr int kPart = paged_part_floats<D, NG>();              // per set of heads: accumulators, then maxima and sums
    const int from = shares.owner(unit0 + kPagedItemUnits), to = shares.owner(unit0 + kPagedItemUnits + n_tiles - 1);
    // Many parts come by bulk copies, all at once, into the ring, which is free when nothing is left to do (another SM's part is
    // 0.9 us away); rounds of half the ring in turn. `from`'s part lies apart from the others.
    const bool bulk = !more && to - from >= kTeam;
    constexpr int kRound = kStages * paged_stage_bytes<D>() / 2 / (kPart * 4);
    auto fetch = [&](int r) {                                      // one thread: round r, if there is one
      const int q0 = r * kRound, n = min(kRound, to - from + 1 - q0);
      if (n <= 0) return;
      const uint32_t dst = base + (r & 1) * kRound * kPart * 4;
      mbar_expect_tx(bar_join(r & 1), (uint32_t)n * kPart * 4);
      if (q0 == 0) bulk_load(dst, a.part + ((long long)gridDim.x + from) * kPart, kPart * 4, bar_join(0));
      const int skip = q0 == 0 ? 1 : 0;
      if (n > skip) bulk_load(dst + skip * kPart * 4, a.part + (long long)(from + q0 + skip) * kPart, (uint32_t)(n - skip) * kPart * 4, bar_join(r & 1));
    };
    const int acc_at = team * MT * 32 + lane, ml_at = NG * MT * 32 + team * 4 + c;   // in units of four floats
    if (mate == 0) {
      float4* dst = reinterpret_cast<float4*>(a.part + ((t0 == 0 ? (long long)gridDim.x : 0) + cta) * kPart);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) dst[acc_at + mt * 32] = make_float4(o[mt][0], o[mt][1], o[mt][2], o[mt][3]);
      if (g == 0) dst[ml_at] = make_float4(m[0], m[1], l[0], l[1]);
    }
    if constexpr (NG == 1) __syncwarp(); else paged_consumers_sync();
    if (tid == 0) {
      // the part is visible before the count goes up, and who counts last sees the others'
      const int last = atom_add_acq_rel(a.tickets + item, 1) == to - from;
      *s_last = last;
      if (last) {
        a.tickets[item] = 0;                                       // ready for the next call
        if (bulk) {
          fence_proxy_async_global();                              // the parts are read by bulk copies, which
          fence_proxy_async_smem();                                // overwrite tiles that all warps have done with
          fetch(0);
          fetch(1);
        }
      }
    }
    paged_consumers_sync();
    if (*s_last) {
      clear();
      auto join = [&](const float4 ml, auto v_of) {                // adds one part
        float f[2], e[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float top = x ? ml.y : ml.x, now = fmaxf(m[x], top), ref = fmaxf(now, kPagedLeast);
          f[x] = ex2_approx(m[x] - ref);
          e[x] = ex2_approx(top - ref);
          l[x] = fmaf(x ? ml.w : ml.z, e[x], l[x] * f[x]);
          m[x] = now;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const float4 v = v_of(mt);
          o[mt][0] = fmaf(v.x, e[0], o[mt][0] * f[0]);
          o[mt][1] = fmaf(v.y, e[1], o[mt][1] * f[1]);
          o[mt][2] = fmaf(v.z, e[0], o[mt][2] * f[0]);
          o[mt][3] = fmaf(v.w, e[1], o[mt][3] * f[1]);
        }
      };
      if (bulk) {
        bool landed = true;
        for (int r = 0; r * kRound <= to - from; ++r) {
          const int n = min(kRound, to - from + 1 - r * kRound);
          if (landed && !__all_sync(0xffffffffu, mbar_wait(bar_join(r & 1), (uint32_t)(r >> 1) & 1u))) {
            landed = false;
            if (lane == 0) give_up();
            mbar_wait(bar_join(r & 1), (uint32_t)(r >> 1) & 1u);   // what is in flight, before the CTA ends
            if ((r + 1) * kRound <= to - from) mbar_wait(bar_join((r + 1) & 1), (uint32_t)((r + 1) >> 1) & 1u);
          }
          if (landed) {
            for (int q = mate; q < n; q += kTeam) {
              const float4* src = reinterpret_cast<const float4*>(gen + (r & 1) * kRound * kPart * 4) + q * (kPart / 4);
              join(src[ml_at], [&](int mt) { return src[acc_at + mt * 32]; });
            }
          }
          paged_consumers_sync();                                  // the half is read
          if (tid == 0 && landed) {
            fence_proxy_async_smem();
            fetch(r + 2);
          }
        }
      } else {
        for (int q = from + mate; q <= to; q += kTeam) {
          const float4* src = reinterpret_cast<const float4*>(a.part + ((q == from ? (long long)gridDim.x : 0) + q) * kPart);
          join(__ldcg(src + ml_at), [&](int mt) { return __ldcg(src + acc_at + mt * 32); });
        }
      }
      merge_warps();
      if (mate == 0) finish(b, head);
    }
    paged_consumers_sync();                                        // s_last is read
  }
}

// Adds the group's attention to the entries' weights, from the scores and normalisers of paged_attn_kernel, which also wrote down
// whose each tile of scores is. A lane reads four heads' scores of an entry at a time, a warp 512 bytes in a row; Gs / 4 lanes
// share an entry and add up. A warp has two such reads, a Gs / 4th of a tile. The rest is a chain of round trips: what a tile is, with its
// scores; the entries' pages and the normalisers; the old weights, which the attention kernel's producers have asked the L2 cache
// for. An entry per lane, head after head, fetched every sector four times over, and normalisers past L1, asked for by
// thousands of warps at once, waited for one another: 131,000 entries of four KV heads took 25 us behind the attention, now 12.
constexpr int kPagedWeightsCtas = 4;                       // per SM
__global__ void __launch_bounds__(256, kPagedWeightsCtas) paged_weights_kernel(const PagedAttnArgs a) {
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 31, share = a.Gs / 4, share_shift = 31 - __clz(share);   // lanes of an entry, parts of a tile
  const int quad = lane & (share - 1);                     // heads 4 quad .. 4 quad + 3
  grid_dependency_wait();
  allow_dependents();
  const int2 units = *reinterpret_cast<const int2*>(a.score_units);
  const int total = units.x;
  const int parts = a.score_tiles << share_shift;          // of a kilobyte each
  auto load = [&](int part, int2& at, float4 (&x)[2]) {    // behind the units in use lies what an earlier call left
    part = min(part, parts - 1);
    at = __ldcg(a.score_at + (part >> share_shift));
    const float4* src = reinterpret_cast<const float4*>(a.scores) + (long long)part * 64 + lane;
    x[0] = __ldcg(src);
    x[1] = __ldcg(src + 32);
  };
  int part = blockIdx.x * 8 + (threadIdx.x >> 5);
  int2 at_next;
  float4 x_next[2];
  load(part, at_next, x_next);
  // An attention that gave up leaves scores and normalisers of an earlier call, or of none: no weight grows until that is reported.
  const int n_parts = units.y ? 0 : min(total, a.score_tiles) << share_shift;
  const int most_tiles = ((p.max_pages << p.page_shift) + kDecTile - 1) / kDecTile;
  for (; part < n_parts; part += gridDim.x * 8) {
    const int2 at = at_next;
    const float4 x[2] = {x_next[0], x_next[1]};
    load(part + gridDim.x * 8, at_next, x_next);
    const int b = at.x & 0xFFFF, h = (int)((unsigned)at.x >> 16);
    if ((unsigned)at.y >= (unsigned)most_tiles || b >= p.n_seqs || h >= p.H) continue;   // a unit of an item itself
    const float* z = a.lse2 + ((long long)b * p.H + h) * a.G;
    const int len = p.length(b), first = at.y * kDecTile + (((part & (share - 1)) * 64 + lane) >> share_shift);
    int page[2];
    float zz[4], *dst[2], old[2];
    bool ok[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) page[k] = p.page(b, min(first + (k * 32 >> share_shift), (p.max_pages << p.page_shift) - 1));
#pragma unroll
    for (int j = 0; j < 4; ++j) zz[j] = z[min(4 * quad + j, a.G - 1)];   // through L1: thousands of warps ask for the same few
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = first + (k * 32 >> share_shift);
      ok[k] = i < len && (unsigned)page[k] < (unsigned)p.n_pages && quad == 0;   // bad pages were recorded by the attention
      dst[k] = a.weights + (ok[k] ? (((long long)page[k] * p.H + h) << p.page_shift) + (i & (p.page_size() - 1)) : 0);
      old[k] = *dst[k];
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float e[4] = {ex2_approx(x[k].x - zz[0]), ex2_approx(x[k].y - zz[1]), ex2_approx(x[k].z - zz[2]), ex2_approx(x[k].w - zz[3])};
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) if (4 * quad + j < a.G) sum += e[j];
      for (int off = 1; off < share; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      if (ok[k]) *dst[k] = old[k] + sum;
    }
  }
  if (total > a.score_tiles && blockIdx.x == 0 && threadIdx.x == 0) record_status(p.status, kStatusCapacity);   // sequences share pages: not for caches with weights
}

}  // namespace lkv

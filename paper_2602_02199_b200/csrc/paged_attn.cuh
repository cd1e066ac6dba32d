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
//                         crosses CTAs leaves partials; the CTA that finishes last joins them in order of the CTAs, so
//                         results depend on lengths and shapes alone.
//   paged_weights_kernel  exp(x_i - lse) from the scores that the first kernel left (4 bytes per query head and entry
//                         against the 512 of its key and value), added to the entries' weights.
//
// Numerators are taken relative to the maximum of their own 16 rows, where they are at most 1, and the 16 rows' sums are
// added to the running ones in fp32, rounded to nearest, with the factor between the two maxima. The MMAs' accumulators do not
// round to nearest: over the 16 rows of a block that does not matter, over thousands it would be a drift. bf16: a numerator
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
constexpr int kPagedBadPage = 1;                           // status of a page number or length out of range: LASER_KV_ERR_INVALID_ARG

struct PagedPool {                                         // what all kernels of a paged cache are told about it
  const int* table;                                        // [n_seqs][max_pages]
  int* lens;                                               // [n_seqs]
  int* seen;                                               // [n_seqs]
  int n_seqs, H, n_pages, max_pages, page_shift;
  int* status;
  __device__ __forceinline__ int page_size() const { return 1 << page_shift; }
  // Entries of a sequence: a length that the table cannot hold is cut.
  __device__ __forceinline__ int length(int b) const {
    return min(max(lens[b], 0), max_pages << page_shift);
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
  int score_tiles;                                         // tiles that `scores` holds
  float* part;                                             // [CTA][2] partials
  int* tickets;                                            // [n_seqs][H][head blocks] parts that are done; zero between calls
  int G, Gs, head_blocks;                                  // query heads per KV head, rounded up to even; blocks of NG * 8 of them
  int out16;
  float scale_log2e;
};

template <int D>
__host__ __device__ constexpr int paged_stage_bytes() { return kDecTile * D * 4; }
// Stages: 96 KB of tiles in flight per CTA, two CTAs per SM; heads of 256 have 192 KB and the SM to themselves.
template <int D>
__host__ __device__ constexpr int paged_stages() { return D == 64 ? 6 : 3; }
template <int D>
__host__ __device__ constexpr int paged_ctas_per_sm() { return D == 256 ? 1 : 2; }
template <int D, int NG>
__host__ __device__ constexpr int paged_part_floats() { return NG * 8 * (D + 2); }
template <int D, int NG>
__host__ __device__ constexpr uint32_t paged_smem_bytes() {
  return 1024u + paged_stages<D>() * paged_stage_bytes<D>() + 2u * D / 16 * 512u + 2u * kPagedWarps * NG * 8u * 4u + 2u * paged_stages<D>() * 8u + 16u;
}

// D (16x8, fp32) += A (16x16, row) * B (16x8, col)
template <bool HALF>
__device__ __forceinline__ void paged_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if constexpr (HALF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    mma_bf16(d, a, b0, b1);
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

// Where a warp is in the list of tiles: sequences one after the other, in each `heads` items, in each the sequence's tiles.
struct PagedWalk {
  int b, head, tile, n_tiles;                              // sequence, item in it, tile of the item, the sequence's tiles per item
  int len;
  int before;                                              // tiles per item of the sequences before this one
  __device__ __forceinline__ void next_item(const PagedPool& p, int heads) {
    tile = 0;
    if (++head < heads) return;
    head = 0;
    do {
      before += n_tiles;
      ++b;
      len = b < p.n_seqs ? p.length(b) : 1;                // past the end: not asked for any more
      n_tiles = (len + kDecTile - 1) / kDecTile;
    } while (n_tiles == 0);
  }
};

// Tiles per item over all sequences; called by whole warps. `mine`: this lane's part, see paged_seek.
__device__ __forceinline__ int paged_total(const PagedPool& p, int lane, int& mine) {
  const int per = (p.n_seqs + 31) / 32;
  mine = 0;
  for (int i = lane * per; i < min((lane + 1) * per, p.n_seqs); ++i) mine += (p.length(i) + kDecTile - 1) / kDecTile;
  return __reduce_add_sync(0xffffffffu, mine);
}
__device__ __forceinline__ int warp_inclusive(int x, int lane) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int n = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += n;
  }
  return x;
}
// The place of tile `at` (below total * heads) of the list.
__device__ __forceinline__ PagedWalk paged_seek(const PagedPool& p, int lane, int mine, int heads, int at) {
  const int per = (p.n_seqs + 31) / 32, q = at / heads;    // the sequence: the first with more than q tiles per item up to its end
  int incl = warp_inclusive(mine, lane);
  const int who = __ffs(__ballot_sync(0xffffffffu, incl > q)) - 1;
  PagedWalk w;
  w.before = __shfl_sync(0xffffffffu, incl - mine, who);
  w.b = who * per;
  for (;;) {
    const int i = w.b + lane;
    const int len = i < p.n_seqs ? p.length(i) : 0, t = (len + kDecTile - 1) / kDecTile;
    incl = w.before + warp_inclusive(t, lane);
    const uint32_t found = __ballot_sync(0xffffffffu, incl > q);
    const int l = found ? __ffs(found) - 1 : 31;
    if (found) {
      w.b += l;
      w.before = __shfl_sync(0xffffffffu, incl - t, l);
      w.len = __shfl_sync(0xffffffffu, len, l);
      w.n_tiles = __shfl_sync(0xffffffffu, t, l);
      break;
    }
    w.before = __shfl_sync(0xffffffffu, incl, 31);
    w.b += 32;
    if (w.b >= p.n_seqs) {                                 // cannot be: `at` is in the list
      w.len = w.n_tiles = 1;
      break;
    }
  }
  const int r = at - w.before * heads;
  w.head = r / w.n_tiles;
  w.tile = r - w.head * w.n_tiles;
  return w;
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
  float* const wm = reinterpret_cast<float*>(red + 2 * MT * 32);                           // [warps][NG * 8] maxima
  float* const wl = wm + kPagedWarps * NG * 8;                                             // sums
  int* const s_last = reinterpret_cast<int*>(wl + kPagedWarps * NG * 8);
  const uint32_t bars = smem_u32(s_last) + 16u;
  auto bar_full = [&](int s) { return bars + 8u * s; };
  auto bar_empty = [&](int s) { return bars + 8u * (kStages + s); };
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const PagedPool& p = a.pool;
  const int heads = p.H * a.head_blocks;

  if (tid == kPagedWarps * 32) {
    for (int s = 0; s < kStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), kPagedWarps); }
    fence_mbar_init();
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  // launched beside the kernel ahead in the stream: nothing is read or written before that is complete
  grid_dependency_wait();
  allow_dependents();

  int mine;
  const int total = paged_total(p, lane, mine) * heads;
  const int n_act = paged_shares(total, (int)gridDim.x);
  const int cta = blockIdx.x;
  const int begin = cta < n_act ? paged_share_begin(total, n_act, cta) : 0;
  int left = cta < n_act ? paged_share_begin(total, n_act, cta + 1) - begin : 0;
  PagedWalk w{};
  if (left > 0) w = paged_seek(p, lane, mine, heads, begin);
  __syncthreads();                                                 // the barriers are set up

  if (warp == kPagedWarps) {
    // ---- producer ---------------------------------------------------------------------------------
    const int rows_shift = min(p.page_shift, 6);                   // rows of a box
    const int per_shift = 6 - rows_shift;                          // pages of a tile
    int st = 0, round = 0;
    while (left > 0) {
      const int n = min(left, w.n_tiles - w.tile), end = w.tile + n, h = w.head / a.head_blocks;
      const int last_page = (w.len - 1) >> p.page_shift;
      int ids = 0;
      for (int t = w.tile; t < end; ++t) {
        const int chunk = 32 >> per_shift, k = (t - w.tile) & (chunk - 1);   // tiles whose page numbers the lanes hold
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
          if (lane == 0) record_status(p.status, kStatusTimeout);
          left = n;                                                // the consumers give up, too
          break;
        }
        if (lane == 0) mbar_expect_tx(bar_full(st), (uint32_t)pages << (rows_shift + 7 + (D == 64 ? 1 : D == 128 ? 2 : 3)));
        __syncwarp();
        if (lane < pages) {
          const uint32_t dst = base + st * paged_stage_bytes<D>() + ((uint32_t)lane << (rows_shift + 7));
          const int row = per_shift ? 0 : (t << 6) & (p.page_size() - 1);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) tma_load_4d(dst + c * kBox, &map_k, bar_full(st), 64 * c, row, h, id);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) tma_load_4d(dst + kHalf + c * kBox, &map_v, bar_full(st), 64 * c, row, h, id);
        }
        __syncwarp();
        if (++st == kStages) { st = 0; ++round; }
      }
      left -= n;
      if (left > 0) w.next_item(p, heads);
    }
    return;
  }

  // ---- consumers ------------------------------------------------------------------------------------
  const int g = lane >> 2, c = lane & 3;                           // fragment coordinates, as in decode_split_kernel
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

  float o[NG][MT][4], m[NG][2], l[NG][2];
  // the warps' results are combined in warp 0: sums in a fixed order
  auto merge_warps = [&]() {
    if (g == 0) {
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          wm[warp * NG * 8 + ng * 8 + 2 * c + x] = m[ng][x];
          wl[warp * NG * 8 + ng * 8 + 2 * c + x] = l[ng][x];
        }
    }
    paged_consumers_sync();
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int at = ng * 8 + 2 * c + x;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int wi = 0; wi < kPagedWarps; ++wi) top = fmaxf(top, wm[wi * NG * 8 + at]);
        const float ref = top == -INFINITY ? 0.f : top;            // nothing above -inf: all factors are 0
#pragma unroll
        for (int wi = 0; wi < kPagedWarps; ++wi) sum = fmaf(wl[wi * NG * 8 + at], exp2f(wm[wi * NG * 8 + at] - ref), sum);
        const float f = exp2f(m[ng][x] - ref);
        m[ng][x] = top;
        l[ng][x] = sum;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) { o[ng][mt][x] *= f; o[ng][mt][x + 2] *= f; }
      }
    // through a buffer that holds 8 heads of two warps at a time
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      auto put = [&](int slot) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          red[(slot * MT + mt) * 32 + lane] = make_float4(o[ng][mt][0], o[ng][mt][1], o[ng][mt][2], o[ng][mt][3]);
      };
      auto add = [&](int slot) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const float4 v = red[(slot * MT + mt) * 32 + lane];
          o[ng][mt][0] += v.x; o[ng][mt][1] += v.y; o[ng][mt][2] += v.z; o[ng][mt][3] += v.w;
        }
      };
      if (ng > 0) paged_consumers_sync();
      if (warp >= 2) put(warp - 2);
      paged_consumers_sync();
      if (warp < 2) add(warp);
      if (warp == 1) put(1);
      paged_consumers_sync();
      if (warp == 0) add(1);
    }
  };
  auto finish = [&](int b, int head) {                             // warp 0: the item's results
    const int h = head / a.head_blocks, first = (head - h * a.head_blocks) * NG * 8;
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int hg = first + ng * 8 + 2 * c + x;
        if (hg >= a.G) continue;
        const long long row = ((long long)b * p.H + h) * a.G + hg;
        const float inv = 1.f / l[ng][x];
        if (a.out16) {
          uint16_t* dst = static_cast<uint16_t*>(a.out) + row * D + g;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const uint32_t y = paged_pack<HALF>(o[ng][mt][x] * inv, o[ng][mt][x + 2] * inv);
            dst[16 * mt] = (uint16_t)y;
            dst[16 * mt + 8] = (uint16_t)(y >> 16);
          }
        } else {
          float* dst = static_cast<float*>(a.out) + row * D + g;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            dst[16 * mt] = o[ng][mt][x] * inv;
            dst[16 * mt + 8] = o[ng][mt][x + 2] * inv;
          }
        }
        if (g == 0) {
          const float z = m[ng][x] + log2f(l[ng][x]);
          if (a.lse) a.lse[row] = z * 0.6931471805599453f;
          if (a.lse2) a.lse2[row] = z;
        }
      }
  };
  auto clear = [&]() {
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      m[ng][0] = m[ng][1] = -INFINITY;
      l[ng][0] = l[ng][1] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[ng][mt][i] = 0.f;
    }
  };

  int st = 0, round = 0;
  bool gone = false;                                               // a wait ran out: the list is walked, nothing is computed
  while (left > 0) {
    const int n = min(left, w.n_tiles - w.tile), h = w.head / a.head_blocks, first = (w.head - h * a.head_blocks) * NG * 8;
    uint32_t qb[NG][MT][2];                                        // B fragments of Q^T, heads past G are zero
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      const int hg = first + ng * 8 + g;
      const uint16_t* q = a.Q + w.b * a.qs_b + ((long long)h * a.G + hg) * a.qs_h;
#pragma unroll
      for (int ks = 0; ks < MT; ++ks) {
        qb[ng][ks][0] = hg < a.G ? *reinterpret_cast<const uint32_t*>(q + 16 * ks + 2 * c) : 0u;
        qb[ng][ks][1] = hg < a.G ? *reinterpret_cast<const uint32_t*>(q + 16 * ks + 8 + 2 * c) : 0u;
      }
    }
    clear();
    const int score_tile = w.before * p.H + h * w.n_tiles;
    for (int t = w.tile; t < w.tile + n; ++t) {
      if (!gone && !__all_sync(0xffffffffu, mbar_wait(bar_full(st), (uint32_t)round & 1u))) {
        if (lane == 0) record_status(p.status, kStatusTimeout);
        gone = true;
      }
      const int rows = w.len - t * kDecTile - warp * 16;           // of the warp's 16 in this tile
      if (!gone && rows > 0) {
        const uint32_t k_tile = base + st * paged_stage_bytes<D>(), v_tile = k_tile + kHalf;
        float s[NG][4], s1[NG][4];
#pragma unroll
        for (int ng = 0; ng < NG; ++ng)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[ng][i] = s1[ng][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < MT; ks += 2) {
          uint32_t k0[4], k1[4];
          ldsm_x4(k_tile + dec_swz(warp * 16 + (lane & 15), 2 * ks + (lane >> 4)), k0);
          ldsm_x4(k_tile + dec_swz(warp * 16 + (lane & 15), 2 * ks + 2 + (lane >> 4)), k1);
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) {
            paged_mma<HALF>(s[ng], k0, qb[ng][ks][0], qb[ng][ks][1]);
            paged_mma<HALF>(s1[ng], k1, qb[ng][ks + 1][0], qb[ng][ks + 1][1]);
          }
        }
        // rows past the sequence's end hold whatever the page or an earlier tile left there
        const bool v_lo = g < rows, v_hi = g + 8 < rows;
        uint32_t pb[NG][HALF ? 2 : 3][2];                          // B fragments of P^T, term by term
        float beta[NG][2];
        bool raise = false;
        float alpha[NG][2];
#pragma unroll
        for (int ng = 0; ng < NG; ++ng) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = (i < 2 ? v_lo : v_hi) ? (s[ng][i] + s1[ng][i]) * a.scale_log2e : -INFINITY;
          if (a.scores && score_tile + t < a.score_tiles) {
            const int hg = first + ng * 8 + 2 * c;
            float* dst = a.scores + ((long long)(score_tile + t) * kDecTile + warp * 16 + g) * a.Gs + hg;
            if (hg < a.G) {
              if (v_lo) *reinterpret_cast<float2*>(dst) = make_float2(x[0], x[1]);
              if (v_hi) *reinterpret_cast<float2*>(dst + 8 * a.Gs) = make_float2(x[2], x[3]);
            }
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float top = fmaxf(x[y], x[y + 2]);
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float ref = top == -INFINITY ? 0.f : top;
            const float old = m[ng][y], now = fmaxf(old, top), run = now == -INFINITY ? 0.f : now;
            alpha[ng][y] = exp2f(old - run);
            beta[ng][y] = exp2f(top - run);
            raise |= now > old;
            m[ng][y] = now;
            x[y] = exp2f(x[y] - ref);
            x[y + 2] = exp2f(x[y + 2] - ref);
            l[ng][y] = fmaf(x[y] + x[y + 2], beta[ng][y], l[ng][y] * alpha[ng][y]);
            if constexpr (HALF) {                                  // exact: powers of two
              x[y] *= 32768.f;
              x[y + 2] *= 32768.f;
              beta[ng][y] *= 1.f / 32768.f;
            }
          }
#pragma unroll
          for (int term = 0; term < (HALF ? 2 : 3); ++term) {
            const uint32_t lo = paged_pack<HALF>(x[0], x[1]), hi = paged_pack<HALF>(x[2], x[3]);
            pb[ng][term][0] = movmatrix_trans(lo);
            pb[ng][term][1] = movmatrix_trans(hi);
            const float2 f0 = paged_unpack<HALF>(lo), f1 = paged_unpack<HALF>(hi);
            x[0] -= f0.x; x[1] -= f0.y; x[2] -= f1.x; x[3] -= f1.y;
          }
        }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
          for (int ng = 0; ng < NG; ++ng)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[ng][mt][i] *= alpha[ng][i & 1];
        }
        // values of rows past the end are taken as zeros: 0 times what lies there could be NaN
        const bool cut = rows < 16;
        const uint32_t keep_lo = (2 * c < rows ? 0xFFFFu : 0u) | (2 * c + 1 < rows ? 0xFFFF0000u : 0u);
        const uint32_t keep_hi = (2 * c + 8 < rows ? 0xFFFFu : 0u) | (2 * c + 9 < rows ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t vt[4];
          ldsm_x4_trans(v_tile + dec_swz(warp * 16 + (lane & 7) + 8 * (lane >> 4), 2 * mt + ((lane >> 3) & 1)), vt);
          if (cut) { vt[0] &= keep_lo; vt[1] &= keep_lo; vt[2] &= keep_hi; vt[3] &= keep_hi; }
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) {
            float blk[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int term = 0; term < (HALF ? 2 : 3); ++term) paged_mma<HALF>(blk, vt, pb[ng][term][0], pb[ng][term][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[ng][mt][i] = fmaf(blk[i], beta[ng][i & 1], o[ng][mt][i]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty(st));
      if (++st == kStages) { st = 0; ++round; }
    }
    // lanes with equal c hold different rows
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l[ng][x] += __shfl_xor_sync(0xffffffffu, l[ng][x], off);
    merge_warps();
    const bool whole = n == w.n_tiles;
    if (whole) {
      if (warp == 0) finish(w.b, w.head);
    } else {
      // the item's parts lie in consecutive CTAs: its start in the first one's second slot, the others in their first
      constexpr int kPart = paged_part_floats<D, NG>();
      const int t0 = (w.before * heads) + w.head * w.n_tiles, item = w.b * heads + w.head;
      const int from = paged_share_owner(total, n_act, t0), to = paged_share_owner(total, n_act, t0 + w.n_tiles - 1);
      if (warp == 0) {
        float* dst = a.part + ((long long)cta * 2 + (w.tile == 0 ? 1 : 0)) * kPart;
#pragma unroll
        for (int i = 0; i < NG * MT; ++i) {
          const float* v = o[i / MT][i % MT];
          reinterpret_cast<float4*>(dst)[i * 32 + lane] = make_float4(v[0], v[1], v[2], v[3]);
        }
        if (g == 0) {
#pragma unroll
          for (int ng = 0; ng < NG; ++ng)
            reinterpret_cast<float4*>(dst + NG * 8 * D)[ng * 4 + c] = make_float4(m[ng][0], m[ng][1], l[ng][0], l[ng][1]);
        }
        __syncwarp();
        if (lane == 0) {
          __threadfence();                                         // the part is visible before the count goes up
          const int last = atomicAdd(a.tickets + item, 1) == to - from;
          if (last) {
            a.tickets[item] = 0;                                   // ready for the next call
            __threadfence();                                       // the other CTAs' parts are visible from here on
          }
          *s_last = last;
        }
      }
      paged_consumers_sync();
      if (*s_last) {
        clear();
        for (int q = from + warp; q <= to; q += kPagedWarps) {
          const float* src = a.part + ((long long)q * 2 + (q == from ? 1 : 0)) * kPart;
          float4 ml[NG], v[NG * MT];
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) ml[ng] = __ldcg(reinterpret_cast<const float4*>(src + NG * 8 * D) + ng * 4 + c);
#pragma unroll
          for (int i = 0; i < NG * MT; ++i) v[i] = __ldcg(reinterpret_cast<const float4*>(src) + i * 32 + lane);
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) {
            const float now_a = fmaxf(m[ng][0], ml[ng].x), now_b = fmaxf(m[ng][1], ml[ng].y);
            const float ref_a = now_a == -INFINITY ? 0.f : now_a, ref_b = now_b == -INFINITY ? 0.f : now_b;
            const float fa = exp2f(m[ng][0] - ref_a), fb = exp2f(m[ng][1] - ref_b);
            const float ga = exp2f(ml[ng].x - ref_a), gb = exp2f(ml[ng].y - ref_b);
            l[ng][0] = fmaf(ml[ng].z, ga, l[ng][0] * fa);
            l[ng][1] = fmaf(ml[ng].w, gb, l[ng][1] * fb);
            m[ng][0] = now_a;
            m[ng][1] = now_b;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              const float4 x = v[ng * MT + mt];
              o[ng][mt][0] = fmaf(x.x, ga, o[ng][mt][0] * fa);
              o[ng][mt][1] = fmaf(x.y, gb, o[ng][mt][1] * fb);
              o[ng][mt][2] = fmaf(x.z, ga, o[ng][mt][2] * fa);
              o[ng][mt][3] = fmaf(x.w, gb, o[ng][mt][3] * fb);
            }
          }
        }
        merge_warps();
        if (warp == 0) finish(w.b, w.head);
      }
      paged_consumers_sync();                                      // s_last is read
    }
    left -= n;
    if (left > 0) w.next_item(p, heads);
  }
}

// Adds the group's attention to the entries' weights, from the scores and normalisers of paged_attn_kernel. The tiles of all
// KV heads are cut into equal shares, one per warp; a lane has two entries of a tile.
__global__ void __launch_bounds__(256) paged_weights_kernel(const PagedAttnArgs a) {
  grid_dependency_wait();
  allow_dependents();
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 31;
  int mine;
  const int total = paged_total(p, lane, mine) * p.H;
  const int n_warps = (int)gridDim.x * 8, n_act = min(total, n_warps), me = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (me >= n_act) return;
  const int begin = paged_share_begin(total, n_act, me);
  int left = paged_share_begin(total, n_act, me + 1) - begin;
  PagedWalk w = paged_seek(p, lane, mine, p.H, begin);
  while (left > 0) {
    const int n = min(left, w.n_tiles - w.tile);
    const float* z = a.lse2 + ((long long)w.b * p.H + w.head) * a.G;
    for (int t = w.tile; t < w.tile + n; ++t) {
      const int tile = w.before * p.H + w.head * w.n_tiles + t;
      if (tile >= a.score_tiles) {                                 // pages that several sequences share: not for accumulating caches
        if (lane == 0) record_status(p.status, kStatusCapacity);
        return;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = t * kDecTile + k * 32 + lane;
        if (i >= w.len) continue;
        const int page = p.page(w.b, i);
        if ((unsigned)page >= (unsigned)p.n_pages) continue;       // recorded by the attention
        float* dst = a.weights + (((long long)page * p.H + w.head) << p.page_shift) + (i & (p.page_size() - 1));
        const float* x = a.scores + ((long long)tile * kDecTile + k * 32 + lane) * a.Gs;
        float sum = 0.f;
        for (int hg = 0; hg < a.G; hg += 2) {                      // heads in order: the same sums every time
          const float2 y = *reinterpret_cast<const float2*>(x + hg);
          sum += exp2f(y.x - z[hg]);
          if (hg + 1 < a.G) sum += exp2f(y.y - z[hg + 1]);
        }
        *dst += sum;
      }
    }
    left -= n;
    if (left > 0) w.next_item(p, p.H);
  }
}

}  // namespace lkv

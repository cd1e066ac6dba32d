// Host side of the paged cache: configuration checks, workspace carving, tensor maps and launches. Included by api.cu, whose
// error, launch and encoding helpers it uses.
#pragma once

struct laser_kv_paged_ctx {
  laser_kv_paged_config_t cfg;
  lkv::PagedPool pool;
  lkv::PagedRows rows;
  CUtensorMap map_k, map_v;
  uint8_t* ws = nullptr;
  size_t zeroed = 0;             // bytes of the workspace, from its start, that are zero between calls
  int* attn_tickets = nullptr;
  int* append_tickets = nullptr;
  float* part = nullptr;
  float* lse2 = nullptr;
  float* scores = nullptr;
  int2* score_at = nullptr;
  int2* moves = nullptr;
  int2* lists = nullptr;
  int group, head_blocks, n_wide;           // query heads per KV head; blocks of 8 * n_wide of them
  int score_heads = 0;                      // scores of an entry
  int score_tiles = 0;
  long long n_moves = 0, cap = 0;
  int num_sms = 1;
  int evict_ctas = 1;                       // cluster of an eviction; 0: too many entries
  uint32_t polls = 0;                       // 0: built-in wait budget (laser_kv_paged_set_wait_budget)
};

namespace {

constexpr int paged_max_ctas(int d) { return d == 64 ? 480 : d == 128 ? 320 : 160; }   // upper bounds of the attention's persistent grid

struct PagedDerived {
  int group, n_wide, head_blocks, page_shift, score_tiles, score_heads;
  long long cap, n_moves;
  size_t append_tickets, attn_tickets, part, lse2, scores, score_at, moves, lists, zeroed, total;
};

laser_kv_status_t paged_derive(const laser_kv_paged_config_t* c, PagedDerived* d) {
  if (!c) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged config is NULL");
  if (c->n_seqs < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_pages < 1 || c->max_pages < 1)
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged config: counts must be positive");
  if (c->n_q_heads % c->n_kv_heads)
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged config: n_q_heads must be a multiple of n_kv_heads");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged config: head_dim must be 64, 128 or 256");
  if (c->page_size < 8 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged config: page_size must be a power of two from 8 to 4096");
  if (c->dtype != LASER_KV_BF16 && c->dtype != LASER_KV_FP16)
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged config: dtype must be LASER_KV_BF16 or LASER_KV_FP16");
  if (c->track_weights != 0 && c->track_weights != 1)
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged config: track_weights must be 0 or 1");
  d->cap = (long long)c->max_pages * c->page_size;
  const long long rows = (long long)c->n_pages * c->page_size * c->n_kv_heads;
  d->group = c->n_q_heads / c->n_kv_heads;
  d->n_wide = d->group <= 8 ? 1 : 2;
  d->head_blocks = (d->group + 8 * d->n_wide - 1) / (8 * d->n_wide);
  const long long seq_tiles = (d->cap + kDecTile - 1) / kDecTile + kPagedWholeUnits;   // units at most
  if (c->n_seqs > 65535 || c->n_kv_heads > 65535 || d->cap > (1ll << 30) || rows > 0x7fffffffLL ||
      (double)c->n_seqs * c->n_kv_heads * d->head_blocks * (double)seq_tiles > 2147483647.0 ||
      (double)c->n_seqs * c->n_q_heads > 2147483647.0)
    return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged config: more than 65535 sequences or KV heads, 2^30 entries per sequence or 2^31 rows or tiles");
  for (d->page_shift = 3; (1 << d->page_shift) < c->page_size;) ++d->page_shift;
  // Pages that no two sequences share bound the entries of all sequences together.
  const long long all = (long long)c->n_seqs * seq_tiles, pooled = (long long)c->n_pages * c->page_size / kDecTile + kPagedWholeUnits * (long long)c->n_seqs;
  const long long tiles = (all < pooled ? all : pooled) * c->n_kv_heads;
  if (tiles * (c->n_q_heads / c->n_kv_heads + 3) > 0x3fffffffLL && c->track_weights) return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged config: too many entries");
  d->score_tiles = c->track_weights ? (int)tiles : 0;
  d->n_moves = c->track_weights ? rows / 2 + 1 : 0;
  for (d->score_heads = 4; d->score_heads < d->group;) d->score_heads *= 2;
  if (c->track_weights && d->group > 128)
    return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged config: weights for at most 128 query heads per KV head");
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes); return o; };
  take(256);                                                   // status word; two words on, units of the last accumulating call and whether one gave up
  d->append_tickets = take((size_t)c->n_seqs * 4);
  d->attn_tickets = take((size_t)c->n_seqs * c->n_kv_heads * d->head_blocks * 4);
  d->zeroed = off;
  d->part = take((size_t)paged_max_ctas(c->head_dim) * 2 * d->n_wide * 8 * (c->head_dim + 2) * sizeof(float));
  d->lse2 = take(c->track_weights ? (size_t)c->n_seqs * c->n_q_heads * 4 : 0);
  d->scores = take((size_t)d->score_tiles * kDecTile * d->score_heads * sizeof(float));
  d->score_at = take((size_t)d->score_tiles * sizeof(int2));
  d->moves = take((size_t)d->n_moves * sizeof(int2));
  d->lists = take(c->track_weights ? (size_t)c->n_seqs * c->n_kv_heads * sizeof(int2) : 0);
  d->total = off;
  return LASER_KV_OK;
}

// Whether rows of `row` elements, `n` of each kind `stride` apart, lie beside one another.
bool paged_disjoint(long long row, int64_t (&stride)[3], long long (&n)[3]) {
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[order[j]] < stride[order[i]]) { const int t = order[i]; order[i] = order[j]; order[j] = t; }
  long long extent = row;
  for (int k : order) {
    if (n[k] == 1) continue;
    if (stride[k] < extent) return false;
    extent = stride[k] * (n[k] - 1) + extent;
  }
  return true;
}

bool paged_map(EncodeTiledFn enc, CUtensorMap* m, const laser_kv_paged_config_t& c, const void* ptr, const int64_t* strides) {
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t bytes[3] = {(cuuint64_t)strides[2] * 2, (cuuint64_t)strides[1] * 2, (cuuint64_t)strides[0] * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)(c.page_size < kDecTile ? c.page_size : kDecTile), 1, 1}, ones[4] = {1, 1, 1, 1};
  return enc(m, c.dtype == LASER_KV_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims,
             bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             // rows of 128 bytes that lie apart: no more than a row is fetched, what is beside it belongs to another head
             c.head_dim == 64 && strides[2] != 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

laser_kv_status_t paged_device(laser_kv_paged_ctx* h, const char* who) {
  int dev = -1;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "%s: cudaGetDevice: %s", who, cudaGetErrorString(e));
  if (dev != h->cfg.device)
    return fail(nullptr, LASER_KV_ERR_STATE, "%s: the current device is %d, the cache was created on device %d", who, dev, h->cfg.device);
  return LASER_KV_OK;
}

cudaError_t evict_limits() {                  // set for the largest slice there is
  static std::atomic<unsigned long long> limit_set{0};
  return ensure_smem_limit(limit_set, paged_evict_kernel, (int)evict_smem_bytes(kEvictKeys), true);
}

// How many clusters of n eviction CTAs, of a slice of `cap` entries each, the current device holds at once; 0 also where it cannot say.
int evict_room(int n, long long cap) {
  if (cap > (long long)kEvictKeys * n) return 1;      // a slice that no CTA has: asked for on the way to a larger cluster
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n);
  cfg.blockDim = dim3(kEvictThreads);
  cfg.dynamicSmemBytes = evict_smem_bytes(evict_slice(cap, n));
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = n;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int room = 0;
  if (evict_limits() != cudaSuccess || cudaOccupancyMaxActiveClusters(&room, paged_evict_kernel, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  return room;
}

template <bool HALF, int D, int NG>
cudaError_t launch_paged_attn(const laser_kv_paged_ctx* h, const PagedAttnArgs& a, cudaStream_t st) {
  static std::atomic<unsigned long long> limit_set{0};
  const cudaError_t e = ensure_smem_limit(limit_set, paged_attn_kernel<HALF, D, NG>, (int)paged_smem_bytes<D, NG>());
  if (e != cudaSuccess) return e;
  const long long most = (long long)h->cfg.n_seqs * h->cfg.n_kv_heads * h->head_blocks * ((h->cap + kDecTile - 1) / kDecTile);
  long long grid = (long long)h->num_sms * paged_ctas_per_sm<D>();
  if (grid > paged_max_ctas(D)) grid = paged_max_ctas(D);
  if (grid > most) grid = most;
  return launch(paged_attn_kernel<HALF, D, NG>, dim3((unsigned)grid), kPagedThreads, paged_smem_bytes<D, NG>(), st, true, h->map_k, h->map_v, a);
}
template <bool HALF>
cudaError_t launch_paged_attn_t(const laser_kv_paged_ctx* h, const PagedAttnArgs& a, cudaStream_t st) {
  switch (h->cfg.head_dim) {
    case 64: return h->n_wide == 1 ? launch_paged_attn<HALF, 64, 1>(h, a, st) : launch_paged_attn<HALF, 64, 2>(h, a, st);
    case 128: return h->n_wide == 1 ? launch_paged_attn<HALF, 128, 1>(h, a, st) : launch_paged_attn<HALF, 128, 2>(h, a, st);
    default: return h->n_wide == 1 ? launch_paged_attn<HALF, 256, 1>(h, a, st) : launch_paged_attn<HALF, 256, 2>(h, a, st);
  }
}

template <int VECS>
cudaError_t launch_paged_append(PagedAppendArgs a, int num_sms, cudaStream_t st) {
  const long long rows = (long long)a.n_new * a.pool.H;
  a.by_heads = Quotient((unsigned)a.pool.H);
  a.times = append_times(num_sms, a.pool.n_seqs, rows, kPagedAppendThreads / VECS * kPagedAppendRows);
  const long long per = (long long)kPagedAppendThreads / VECS * kPagedAppendRows * a.times;
  return launch(paged_append_kernel<VECS>, dim3((unsigned)((rows + per - 1) / per), (unsigned)a.pool.n_seqs), kPagedAppendThreads, 0, st, true, a);
}

}  // namespace

extern "C" {

laser_kv_status_t laser_kv_paged_query_sizes(const laser_kv_paged_config_t* cfg, size_t* workspace_bytes) {
  PagedDerived d;
  const laser_kv_status_t s = paged_derive(cfg, &d);
  if (s == LASER_KV_OK && workspace_bytes) *workspace_bytes = d.total;
  return s;
}

laser_kv_status_t laser_kv_paged_init(const laser_kv_paged_config_t* cfg, void* k_pages, void* v_pages, const int64_t kv_strides[3],
                                      float* weights, int32_t* pos, const int32_t* page_table, int32_t* state, void* workspace,
                                      size_t workspace_bytes, laser_kv_paged_handle_t* out) {
  if (!out) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_init: out is NULL");
  *out = nullptr;
  PagedDerived d;
  const laser_kv_status_t s = paged_derive(cfg, &d);
  if (s != LASER_KV_OK) return s;
  if (!k_pages || !v_pages || !kv_strides || !pos || !page_table || !state || !workspace)
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_init: NULL argument");
  if (cfg->track_weights != (weights ? 1 : 0))
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_init: weights must be given exactly when track_weights is 1");
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(weights) || !aligned16(pos) || !aligned16(page_table) || !aligned16(state))
    return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_init: device pointers must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(workspace) & (kAlign - 1))
    return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_init: the workspace must be 256-byte aligned");
  int64_t strides[3] = {kv_strides[0], kv_strides[1], kv_strides[2]};
  long long counts[3] = {cfg->n_pages, cfg->n_kv_heads, cfg->page_size};
  for (int i = 0; i < 3; ++i) {
    if (counts[i] == 1) strides[i] = cfg->head_dim;              // never stepped over
    if (strides[i] < cfg->head_dim || (strides[i] % 8))
      return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_init: strides must be multiples of 8 elements, a row at least");
    if (strides[i] >= (1ll << 38) || (double)strides[i] * (double)counts[i] > 1e15)
      return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged_init: stride of 2^38 elements or more, or a pool of 1e15");
  }
  if (!paged_disjoint(cfg->head_dim, strides, counts)) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_init: the strides make rows overlap");
  if (workspace_bytes < d.total) return fail(nullptr, LASER_KV_ERR_CAPACITY, "paged_init: workspace needs %zu bytes, got %zu", d.total, workspace_bytes);
  int ndev = 0;
  cudaError_t e = cudaGetDeviceCount(&ndev);
  if (e != cudaSuccess || cfg->device < 0 || ndev <= cfg->device)
    return fail(nullptr, LASER_KV_ERR_CUDA, "paged_init: no usable CUDA device %d (%s); this library has no CPU path", cfg->device, cudaGetErrorString(e));
  if ((e = cudaSetDevice(cfg->device)) != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_init: cudaSetDevice: %s", cudaGetErrorString(e));
  int major = 0, sms = 0;
  if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, cfg->device)) != cudaSuccess ||
      (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, cfg->device)) != cudaSuccess)
    return fail(nullptr, LASER_KV_ERR_CUDA, "paged_init: device query: %s", cudaGetErrorString(e));
  if (major != 10) return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged_init: the kernels are built for sm_100a only");
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
  if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn)
    return fail(nullptr, LASER_KV_ERR_CUDA, "paged_init: cuTensorMapEncodeTiled not available from the driver");
  laser_kv_paged_ctx* h = new (std::nothrow) laser_kv_paged_ctx();
  if (!h) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_init: out of host memory");
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  h->cfg = *cfg;
  h->ws = ws;
  h->zeroed = d.zeroed;
  h->pool = PagedPool{page_table, state, state + cfg->n_seqs, cfg->n_seqs, cfg->n_kv_heads, cfg->n_pages, cfg->max_pages, d.page_shift,
                      reinterpret_cast<int*>(ws)};
  h->rows = PagedRows{static_cast<uint16_t*>(k_pages), static_cast<uint16_t*>(v_pages), strides[0], strides[1], strides[2], weights, pos,
                      cfg->head_dim / 8};
  h->append_tickets = reinterpret_cast<int*>(ws + d.append_tickets);
  h->attn_tickets = reinterpret_cast<int*>(ws + d.attn_tickets);
  h->part = reinterpret_cast<float*>(ws + d.part);
  if (weights) {
    h->lse2 = reinterpret_cast<float*>(ws + d.lse2);
    h->scores = reinterpret_cast<float*>(ws + d.scores);
    h->score_at = reinterpret_cast<int2*>(ws + d.score_at);
    h->moves = reinterpret_cast<int2*>(ws + d.moves);
    h->lists = reinterpret_cast<int2*>(ws + d.lists);
  }
  h->group = d.group;
  h->head_blocks = d.head_blocks;
  h->n_wide = d.n_wide;
  h->score_tiles = d.score_tiles;
  h->score_heads = d.score_heads;
  h->n_moves = d.n_moves;
  h->cap = d.cap;
  h->num_sms = sms;
  const EncodeTiledFn enc = reinterpret_cast<EncodeTiledFn>(fn);
  laser_kv_status_t bad = LASER_KV_OK;
  if (!paged_map(enc, &h->map_k, *cfg, k_pages, strides) || !paged_map(enc, &h->map_v, *cfg, v_pages, strides))
    bad = fail(nullptr, LASER_KV_ERR_CUDA, "paged_init: cuTensorMapEncodeTiled failed");
  else if ((e = cudaDeviceSynchronize()) != cudaSuccess ||     // whatever used this memory before is done with it, on any stream
           (e = cudaMemset(ws, 0, d.zeroed)) != cudaSuccess ||
           (e = cudaDeviceSynchronize()) != cudaSuccess)         // the first call may come on a stream that does not wait for this one
    bad = fail(nullptr, LASER_KV_ERR_CUDA, "paged_init: clearing the counters: %s", cudaGetErrorString(e));
  if (bad != LASER_KV_OK) {
    delete h;
    return bad;
  }
  if (weights) {
    const long long heads = (long long)cfg->n_seqs * cfg->n_kv_heads;
    h->evict_ctas = evict_cluster(heads, d.cap, evict_room);
  }
  *out = h;
  return LASER_KV_OK;
}

laser_kv_status_t laser_kv_paged_append(laser_kv_paged_handle_t h, const void* K_new, const void* V_new, const int64_t k_strides[3],
                                        const int64_t v_strides[3], int32_t n_new, const int32_t* counts, const float* weights,
                                        const int64_t w_strides[2], const int32_t* pos, const int64_t pos_strides[2], void* stream) {
  if (!h) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_append: NULL handle");
  if (n_new < 0) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_append: n_new is negative");
  if (n_new == 0) return paged_device(h, "paged_append");          // tensors without elements have no address
  if (!K_new || !V_new || !k_strides || !v_strides || (weights && !w_strides) || (pos && !pos_strides))
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_append: NULL argument");
  if (weights && !h->rows.weights) return fail(nullptr, LASER_KV_ERR_STATE, "paged_append: the cache keeps no weights");
  if (!aligned16(K_new) || !aligned16(V_new)) return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_append: K_new and V_new must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(counts) | reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(pos)) & 3u)
    return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_append: counts, weights and pos must be 4-byte aligned");
  PagedAppendArgs a{};
  const int extents[3] = {h->cfg.n_seqs, h->cfg.n_kv_heads, n_new};
  for (int i = 0; i < 3; ++i) {
    if (extents[i] == 1) continue;                                 // never stepped over
    if (k_strides[i] < 0 || v_strides[i] < 0 || (k_strides[i] % 8) || (v_strides[i] % 8))
      return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_append: strides must be non-negative multiples of 8 elements");
    a.ks[i] = k_strides[i];
    a.vs[i] = v_strides[i];
  }
  for (int i = 0; i < 2; ++i) {
    if (extents[i] == 1) continue;
    a.ws[i] = weights ? w_strides[i] : 0;
    a.as[i] = pos ? pos_strides[i] : 0;
    if (a.ws[i] < 0 || a.as[i] < 0) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_append: negative stride");
  }
  if ((long long)n_new * h->cfg.n_kv_heads > (1ll << 30)) return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged_append: more than 2^30 rows per sequence");
  if (n_new > h->cap && !counts)
    return fail(nullptr, LASER_KV_ERR_CAPACITY, "paged_append: %d entries do not fit a table of %lld", n_new, h->cap);
  if (const laser_kv_status_t ds = paged_device(h, "paged_append")) return ds;
  a.pool = h->pool;
  a.rows = h->rows;
  a.K = static_cast<const uint16_t*>(K_new);
  a.V = static_cast<const uint16_t*>(V_new);
  a.w = weights;
  a.at = pos;
  a.counts = counts;
  a.n_new = n_new;
  a.tickets = h->append_tickets;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = h->rows.vecs == 8 ? launch_paged_append<8>(a, h->num_sms, st)
                        : h->rows.vecs == 16 ? launch_paged_append<16>(a, h->num_sms, st) : launch_paged_append<32>(a, h->num_sms, st);
  if (e != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_append_kernel launch: %s", cudaGetErrorString(e));
  return LASER_KV_OK;
}

laser_kv_status_t laser_kv_paged_attention(laser_kv_paged_handle_t h, const void* Q, const int64_t q_strides[2], float softmax_scale,
                                           int32_t accumulate, void* out, int32_t out_fp32, float* lse, void* stream) {
  if (!h) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_attention: NULL handle");
  if (!Q || !q_strides || !out) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_attention: NULL argument");
  if (!aligned16(Q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u))
    return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_attention: Q and out must be 16-byte aligned, lse 4-byte aligned");
  const int64_t qs_b = h->cfg.n_seqs == 1 ? 0 : q_strides[0], qs_h = h->cfg.n_q_heads == 1 ? 0 : q_strides[1];   // of one entry: never stepped over
  if (qs_b < 0 || qs_h < 0 || (qs_b % 8) || (qs_h % 8))
    return fail(nullptr, LASER_KV_ERR_ALIGNMENT, "paged_attention: strides must be non-negative multiples of 8 elements");
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale))
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_attention: softmax_scale must be positive (0 selects 1/sqrt(head_dim))");
  if (accumulate && !h->rows.weights) return fail(nullptr, LASER_KV_ERR_STATE, "paged_attention: the cache keeps no weights");
  if (const laser_kv_status_t ds = paged_device(h, "paged_attention")) return ds;
  PagedAttnArgs a{};
  a.pool = h->pool;
  a.Q = static_cast<const uint16_t*>(Q);
  a.qs_b = qs_b;
  a.qs_h = qs_h;
  a.out = out;
  a.out16 = out_fp32 ? 0 : 1;
  a.lse = lse;
  a.part = h->part;
  a.tickets = h->attn_tickets;
  a.G = h->group;
  a.Gs = h->score_heads;
  a.head_blocks = h->head_blocks;
  a.polls = h->polls ? h->polls : kMaxPolls;
  a.poll_ns = h->polls ? 0u : kPollHintNs;
  a.scale_log2e = (softmax_scale == 0.f ? 1.0f / std::sqrt((float)h->cfg.head_dim) : softmax_scale) * 1.4426950408889634f;
  if (accumulate) {
    a.lse2 = h->lse2;
    a.scores = h->scores;
    a.score_at = h->score_at;
    a.score_units = reinterpret_cast<int*>(h->ws) + 2;
    a.score_tiles = h->score_tiles;
    a.weights = h->rows.weights;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = h->cfg.dtype == LASER_KV_FP16 ? launch_paged_attn_t<true>(h, a, st) : launch_paged_attn_t<false>(h, a, st);
  if (e != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_attn_kernel launch: %s", cudaGetErrorString(e));
  if (accumulate) {
    long long grid = ((long long)h->score_tiles * (a.Gs / 4) + 7) / 8;   // a warp a part
    if (grid > (long long)kPagedWeightsCtas * h->num_sms) grid = (long long)kPagedWeightsCtas * h->num_sms;
    e = launch(paged_weights_kernel, dim3((unsigned)grid), 256, 0, st, true, a);
    if (e != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_weights_kernel launch: %s", cudaGetErrorString(e));
  }
  return LASER_KV_OK;
}

laser_kv_status_t laser_kv_paged_evict(laser_kv_paged_handle_t h, int32_t keep, int32_t anchors, int32_t recent, void* stream) {
  if (!h) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_evict: NULL handle");
  if (keep < 0 || anchors < 0 || recent < 0) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_evict: negative count");
  if ((long long)anchors + recent > keep)
    return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_evict: %d first and %d last positions do not fit %d entries", anchors, recent, keep);
  if (!h->rows.weights) return fail(nullptr, LASER_KV_ERR_STATE, "paged_evict: the cache keeps no weights");
  if (const laser_kv_status_t ds = paged_device(h, "paged_evict")) return ds;
  if (keep >= h->cap) return LASER_KV_OK;
  if (!h->evict_ctas)
    return fail(nullptr, LASER_KV_ERR_UNSUPPORTED, "paged_evict: a table of %lld entries is longer than a cluster's shared memory sorts", h->cap);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const PagedEvictArgs a{h->pool, h->rows, keep, anchors, recent, h->moves, h->n_moves, h->lists};
  const int heads = h->cfg.n_kv_heads, seqs = h->cfg.n_seqs;
  cudaError_t e = evict_limits();
  if (e == cudaSuccess)
    e = launch_clusters(paged_evict_kernel, dim3((unsigned)h->evict_ctas, (unsigned)heads, (unsigned)seqs), kEvictThreads,
                        evict_smem_bytes(evict_slice(h->cap, h->evict_ctas)), st, true, h->evict_ctas, a);
  if (e != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_evict_kernel launch: %s", cudaGetErrorString(e));
  const unsigned ctas = (unsigned)move_ctas(h->num_sms, (long long)seqs * heads, keep < h->cap - keep ? keep : h->cap - keep);
  const dim3 grid(ctas, (unsigned)heads, (unsigned)seqs);
  e = h->rows.vecs == 8    ? launch(paged_move_kernel<8>, grid, kMoveThreads, 0, st, true, a)
      : h->rows.vecs == 16 ? launch(paged_move_kernel<16>, grid, kMoveThreads, 0, st, true, a)
                           : launch(paged_move_kernel<32>, grid, kMoveThreads, 0, st, true, a);
  if (e != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_move_kernel launch: %s", cudaGetErrorString(e));
  return LASER_KV_OK;
}

laser_kv_status_t laser_kv_paged_poll_status(laser_kv_paged_handle_t h, void* stream) {
  if (!h) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_poll_status: NULL handle");
  if (const laser_kv_status_t ds = paged_device(h, "paged_poll_status")) return ds;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, h->ws, sizeof word, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && word != 0) {
    e = cudaMemsetAsync(h->ws, 0, h->zeroed, st);                // a call that gave up may leave counts
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  }
  if (e != cudaSuccess) return fail(nullptr, LASER_KV_ERR_CUDA, "paged_poll_status: %s", cudaGetErrorString(e));
  if (word == LASER_KV_ERR_TIMEOUT) return fail(nullptr, LASER_KV_ERR_TIMEOUT, "a bounded device-side wait gave up");
  if (word == LASER_KV_ERR_CAPACITY)
    return fail(nullptr, LASER_KV_ERR_CAPACITY, "new entries did not fit their sequence's table, or sequences of a cache with weights share pages");
  if (word == kPagedBadPage) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "a page number, a length or a count was out of range");
  if (word != 0) return fail(nullptr, (laser_kv_status_t)word, "device status word %d", word);
  return LASER_KV_OK;
}

laser_kv_status_t laser_kv_paged_set_wait_budget(laser_kv_paged_handle_t h, uint32_t max_polls) {
  if (!h) return fail(nullptr, LASER_KV_ERR_INVALID_ARG, "paged_set_wait_budget: NULL handle");
  h->polls = max_polls;
  return LASER_KV_OK;
}

void laser_kv_paged_destroy(laser_kv_paged_handle_t h) { delete h; }

}  // extern "C"

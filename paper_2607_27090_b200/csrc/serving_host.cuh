// Host side of the serving calls (memstore_grow_blocks, memstore_release_blocks, memstore_append, memstore_attend); included by
// memstore.cu inside extern "C".  None of them uses scratch of the store
// (memstore_attend sets one word of it when a wait ran out).

static_assert(kReqTableShort == MS_REQ_BLOCK_TABLE_SHORT && kReqBadBlock == MS_REQ_BAD_BLOCK_ID && kReqPosOverflow == MS_REQ_POSITION_OVERFLOW &&
                  kReqTimeout == MS_REQ_KERNEL_TIMEOUT && kReqBadStart == MS_REQ_BAD_START && kReqNoBlocks == MS_REQ_NO_BLOCKS &&
                  kReqBadLength == MS_REQ_BAD_LENGTH,
              "status bits of the kernels and the header");

// Counts are at most 2^30, so that the kernels' 32-bit loops end before they wrap.
constexpr int32_t kMaxCount = 1 << 30;
// Requests of an attention call: passing that many over takes the chunk kernel's describing warp 0.3 s (4 ns each), well inside the bound of
// the other roles' waits.
constexpr int32_t kMaxAttendReqs = 1 << 26;
static ms_status check_counts(memstore* s, int32_t a, int32_t b, int32_t c) {
  const int32_t most = std::max(a, std::max(b, c));
  return most <= kMaxCount ? MS_OK : fail(s, MS_ERR_UNSUPPORTED, "a count of %d is more than 2^30", most);
}

static ms_status check_geometry(memstore* s, const ms_paged_cache* c) {
  if (!c || c->block_size <= 0 || c->num_blocks <= 0) return fail(s, MS_ERR_INVALID_ARG, "bad cache description");
  return MS_OK;
}

// The cache as the append and attention kernels need it: 16-byte loads and stores of bf16 rows, 8-byte stores (append) and
// 16-byte loads (attention) of e4m3 rows.
static ms_status check_cache(memstore* s, const ms_paged_cache* c, int32_t layer, bool reads) {
  const ms_status rc = check_geometry(s, c);
  if (rc != MS_OK) return rc;
  if (!c->k_base || !c->v_base) return fail(s, MS_ERR_INVALID_ARG, "bad cache description");
  if (layer < 0 || layer >= s->cfg.n_layers) return fail(s, MS_ERR_INVALID_ARG, "layer %d of %d", layer, s->cfg.n_layers);
  if (((uintptr_t)c->k_base & 15) || ((uintptr_t)c->v_base & 15) || (c->layer_stride % 8) || (c->block_stride % 8) || (c->token_stride % 8) ||
      (c->head_stride % 8) || c->layer_stride < 0 || c->block_stride < 0 || c->token_stride < 0 || c->head_stride < 0)
    return fail(s, MS_ERR_INVALID_ARG, "cache bases must be 16-byte aligned and strides non-negative multiples of 8");
  if (c->dtype != MS_CACHE_BF16 && c->dtype != MS_CACHE_FP8_E4M3) return fail(s, MS_ERR_INVALID_ARG, "unknown cache dtype %d", c->dtype);
  if (c->dtype == MS_CACHE_FP8_E4M3) {
    if (!(c->k_scale > 0.f && c->v_scale > 0.f && std::isfinite(c->k_scale) && std::isfinite(c->v_scale)))
      return fail(s, MS_ERR_INVALID_ARG, "an 8-bit cache needs finite positive k_scale and v_scale");
    if (reads && ((c->layer_stride | c->block_stride | c->token_stride | c->head_stride) % 16))
      return fail(s, MS_ERR_UNSUPPORTED, "memstore_attend reads an 8-bit cache whose strides are multiples of 16");
  }
  return MS_OK;
}

// written: two of its rows must not be the same memory
static ms_status check_heads(memstore* s, const ms_heads* h, int64_t n_tokens, int32_t n_heads, bool written, const char* name) {
  if (!h) return fail(s, MS_ERR_INVALID_ARG, "%s is NULL", name);
  if ((!h->base && n_tokens > 0) || ((uintptr_t)h->base & 15) || h->token_stride < 0 || h->head_stride < 0 || (h->token_stride % 8) || (h->head_stride % 8))
    return fail(s, MS_ERR_INVALID_ARG, "%s needs a 16-byte aligned base and strides that are non-negative multiples of 8", name);
  if (written && ((n_tokens > 1 && h->token_stride < s->cfg.head_dim) || (n_heads > 1 && h->head_stride < s->cfg.head_dim)))
    return fail(s, MS_ERR_INVALID_ARG, "%s is written: its strides must be head_dim or more", name);
  return MS_OK;
}

ms_status memstore_grow_blocks(memstore_t* s, const int32_t* start_lens, const int32_t* new_lens, int32_t nreq, int32_t* block_tables,
                               int32_t max_blocks, const ms_paged_cache* cache, const int32_t* free_blocks, int32_t n_free,
                               const int32_t* n_taken, int32_t token_capacity, int32_t* out_q_start, int32_t* out_seq_lens,
                               int32_t* out_positions, int64_t* out_slots, int32_t* out_n_taken, int32_t* out_status, ms_stream stream) {
  Range range("memstore_grow_blocks");
  if (!s) return MS_ERR_INVALID_ARG;
  std::lock_guard<std::recursive_mutex> lock(s->mu);
  ms_status rc = check_geometry(s, cache);
  if (rc != MS_OK) return rc;
  if (nreq < 0 || max_blocks < 0 || n_free < 0 || token_capacity < 0)
    return fail(s, MS_ERR_INVALID_ARG, "nreq=%d max_blocks=%d n_free=%d token_capacity=%d", nreq, max_blocks, n_free, token_capacity);
  if ((rc = check_counts(s, nreq, max_blocks, token_capacity)) != MS_OK) return rc;
  if (!n_taken || !out_q_start || !out_n_taken || (n_free > 0 && !free_blocks) ||
      (nreq > 0 && (!start_lens || !new_lens || !out_seq_lens || !out_status || (max_blocks > 0 && !block_tables))))
    return fail(s, MS_ERR_INVALID_ARG, "null request arrays");
  DeviceGuard g(s->cfg.device);
  GrowParams p{};
  p.start_lens = start_lens;
  p.new_lens = new_lens;
  p.nreq = nreq;
  p.tables = block_tables;
  p.max_blocks = max_blocks;
  p.block_size = cache->block_size;
  p.num_blocks = cache->num_blocks;
  p.max_position = (int32_t)s->cfg.max_position;
  p.free_blocks = free_blocks;
  p.n_free = n_free;
  p.n_taken = n_taken;
  p.token_capacity = token_capacity;
  p.q_start = out_q_start;
  p.seq_lens = out_seq_lens;
  p.positions = out_positions;
  p.slots = out_slots;
  p.out_n_taken = out_n_taken;
  p.status = out_status;
  cudaStream_t st = (cudaStream_t)stream;
  const bool one = token_capacity <= kGrowOneLaunch;
  MS_CUDA(s, launch_dependent(grow_plan_kernel, dim3(1), dim3(kGrowThreads), 0, st, p, one ? 1 : 0));
  s->kernels_launched++;
  if (!one) {
    MS_CUDA(s, launch_dependent(grow_map_kernel, dim3((unsigned)((token_capacity + kGrowMapTokens - 1) / kGrowMapTokens)), dim3(kGrowMapThreads), 0, st, p));
    s->kernels_launched++;
  }
  return MS_OK;
}

ms_status memstore_release_blocks(memstore_t* s, const int32_t* release, int32_t* seq_lens, int32_t nreq, int32_t* block_tables, int32_t max_blocks,
                                  const ms_paged_cache* cache, int32_t* free_blocks, int32_t n_free, int32_t* n_taken, int32_t* out_status,
                                  ms_stream stream) {
  Range range("memstore_release_blocks");
  if (!s) return MS_ERR_INVALID_ARG;
  std::lock_guard<std::recursive_mutex> lock(s->mu);
  ms_status rc = check_geometry(s, cache);
  if (rc != MS_OK) return rc;
  if (nreq < 0 || max_blocks < 0 || n_free < 0) return fail(s, MS_ERR_INVALID_ARG, "nreq=%d max_blocks=%d n_free=%d", nreq, max_blocks, n_free);
  if ((rc = check_counts(s, nreq, max_blocks, 0)) != MS_OK) return rc;
  if (nreq == 0) return MS_OK;
  if (!seq_lens || !n_taken || (n_free > 0 && !free_blocks) || (max_blocks > 0 && !block_tables)) return fail(s, MS_ERR_INVALID_ARG, "null request arrays");
  DeviceGuard g(s->cfg.device);
  const ReleaseParams p{release, seq_lens, nreq, block_tables, max_blocks, cache->block_size, cache->num_blocks, free_blocks, n_free, n_taken, out_status};
  MS_CUDA(s, launch_dependent(release_kernel, dim3(1), dim3(kGrowThreads), 0, (cudaStream_t)stream, p));
  s->kernels_launched++;
  return MS_OK;
}

ms_status memstore_append(memstore_t* s, int32_t layer, const ms_heads* q, int32_t n_q_heads, const ms_heads* k, const ms_heads* v,
                          const int32_t* positions, const int64_t* slots, int32_t n_tokens, const ms_paged_cache* cache, const ms_heads* q_out,
                          int32_t* out_status, ms_stream stream) {
  Range range("memstore_append");
  if (!s) return MS_ERR_INVALID_ARG;
  std::lock_guard<std::recursive_mutex> lock(s->mu);
  const memstore_config& c = s->cfg;
  if (n_tokens < 0 || n_q_heads < 0 || n_q_heads > (1 << 16)) return fail(s, MS_ERR_INVALID_ARG, "n_tokens=%d n_q_heads=%d", n_tokens, n_q_heads);
  ms_status rc = check_cache(s, cache, layer, false);
  if (rc == MS_OK) rc = check_counts(s, n_tokens, 0, 0);
  if (rc == MS_OK) rc = check_heads(s, k, n_tokens, c.n_kv_heads, false, "k");
  if (rc == MS_OK) rc = check_heads(s, v, n_tokens, c.n_kv_heads, false, "v");
  if (rc == MS_OK && n_q_heads > 0) rc = check_heads(s, q, n_tokens, n_q_heads, false, "q");
  if (rc == MS_OK && n_q_heads > 0) rc = check_heads(s, q_out, n_tokens, n_q_heads, true, "q_out");
  if (rc != MS_OK) return rc;
  if (n_tokens == 0) return MS_OK;
  if (!positions || !slots) return fail(s, MS_ERR_INVALID_ARG, "positions and slots are needed");
  DeviceGuard g(c.device);
  AppendParams p{};
  if (n_q_heads > 0) {
    p.q = (const __nv_bfloat16*)q->base;
    p.q_ts = q->token_stride;
    p.q_hs = q->head_stride;
    p.q_out = (__nv_bfloat16*)q_out->base;
    p.o_ts = q_out->token_stride;
    p.o_hs = q_out->head_stride;
  }
  p.k = (const __nv_bfloat16*)k->base;
  p.k_ts = k->token_stride;
  p.k_hs = k->head_stride;
  p.v = (const __nv_bfloat16*)v->base;
  p.v_ts = v->token_stride;
  p.v_hs = v->head_stride;
  p.n_q = n_q_heads;
  p.n_kv = c.n_kv_heads;
  p.head_dim = c.head_dim;
  p.rotary_dim = c.rotary_dim;
  p.max_position = (int32_t)c.max_position;
  p.inv_freq = s->inv_freq_d;
  p.positions = positions;
  p.slots = slots;
  p.n_tokens = n_tokens;
  const bool fp8 = cache->dtype == MS_CACHE_FP8_E4M3;
  const int64_t esz = fp8 ? 1 : 2;
  p.k_cache = (__nv_bfloat16*)((char*)cache->k_base + layer * cache->layer_stride * esz);
  p.v_cache = (__nv_bfloat16*)((char*)cache->v_base + layer * cache->layer_stride * esz);
  p.block_stride = cache->block_stride;
  p.token_stride = cache->token_stride;
  p.head_stride = cache->head_stride;
  p.num_blocks = cache->num_blocks;
  p.block_size = cache->block_size;
  p.k_scale = fp8 ? cache->k_scale : 1.f;
  p.v_scale = fp8 ? cache->v_scale : 1.f;
  p.k_recip = (float)(1.0 / (double)p.k_scale);
  p.v_recip = (float)(1.0 / (double)p.v_scale);
  p.status = out_status;
  // threads per token: a power of two that gives a thread about kAppendBatch heads
  const int G = c.head_dim / 16;
  const int64_t units = (int64_t)(n_q_heads + 2 * c.n_kv_heads) * G;
  int tpt = G;
  while (tpt < kAppendThreads && (int64_t)tpt * kAppendBatch < units) tpt *= 2;
  p.threads_per_token = tpt;
  const int per_cta = kAppendThreads / tpt;
  const dim3 grid((unsigned)((n_tokens + per_cta - 1) / per_cta));
  auto awkward = [](float sc, float rc2) {
    uint32_t u;
    memcpy(&u, &sc, 4);
    return (u & 0x7fffffu) == 0x7fffffu || !std::isnormal(rc2) || !std::isnormal(sc);
  };
  const int mode = !fp8 ? 0 : (awkward(p.k_scale, p.k_recip) || awkward(p.v_scale, p.v_recip)) ? 2 : 1;  // (see div_by_scale)
  cudaStream_t st = (cudaStream_t)stream;
  const bool half = c.rope_style == MS_ROPE_HALF_SPLIT;
  auto kernel = half ? (mode == 0 ? append_kernel<0, 0> : mode == 1 ? append_kernel<0, 1> : append_kernel<0, 2>)
                     : (mode == 0 ? append_kernel<1, 0> : mode == 1 ? append_kernel<1, 1> : append_kernel<1, 2>);
  MS_CUDA(s, launch_dependent(kernel, grid, dim3(kAppendThreads), 0, st, p));
  s->kernels_launched++;
  return MS_OK;
}

// ---- attention --------------------------------------------------------------------------------------------------------
// Requests with more rows (new tokens x query heads per K/V head) than this go to the tensor-core kernel, when head_dim allows it: than
// two units of the rows kernel where the batch leaves half of the SMs without a unit of their own, else than one.  Rows kernel against
// chunk kernel (32/8 heads of 128, bf16): 20 or 32 rows, one request of 4,096 tokens 17 against 22 us, two 22 against 26, eight of 2,000
// 31 against 36 (of 8,000 90 against 82); 64 of 2,000 170 against 159, 32 of 8,000 318 against 238.  64 rows: one request 23.4 against
// 22.8 us, 64 of 2,000 321 against 165.
static int chunk_min_rows(int64_t units, int sm_count) { return units <= sm_count / 2 ? 2 * kAttnRows : kAttnRows; }

// The workspace: unfinished rows of the rows kernel (kAttnMaxCtasPerSm CTAs per SM at most) and their statistics, then those of the chunk kernel
// (one CTA per SM), its error words and the gate between the two.  It depends on the GPU and head_dim alone.
struct AttendLayout {
  size_t rows_o, rows_ml, rows_cuts, chunk_o, chunk_ml, chunk_cuts, errors, gate, bytes;
};
static bool attend_has_chunks(int head_dim) { return head_dim == 64 || head_dim == 128; }
static AttendLayout attend_layout(const memstore* s) {
  const size_t d = (size_t)s->cfg.head_dim, sms = (size_t)s->sm_count;
  AttendLayout w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
  };
  w.rows_o = take(sms * kAttnMaxCtasPerSm * 2 * kAttnRows * d * 4);
  w.rows_ml = take(sms * kAttnMaxCtasPerSm * 2 * kAttnRows * 8);
  w.rows_cuts = take(sms * kAttnMaxCtasPerSm * sizeof(AttnCut));
  if (attend_has_chunks(s->cfg.head_dim)) {
    w.chunk_o = take(sms * 2 * kChunkRows * d * 4);
    w.chunk_ml = take(sms * 2 * kChunkRows * 8);
    w.chunk_cuts = take(sms * sizeof(AttnCut));
    w.errors = take(sms * 4);
    w.gate = take(8);
  }
  w.bytes = at;
  return w;
}

extern "C++" {
// Shared-memory limits of the attention kernels, raised once per device.
template <int D, bool FP8>
static cudaError_t attend_prepare(int device) {
  static std::mutex mu;
  static bool done[64] = {false};
  std::lock_guard<std::mutex> lock(mu);
  if (done[device & 63]) return cudaSuccess;
  cudaError_t e = cudaFuncSetAttribute(attend_rows_kernel<D, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, AttnCfg<D, FP8>::kSmemBytes);
  if constexpr (D == 64 || D == 128)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attend_chunk_kernel<D, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (ChunkCfg<D, FP8>::kSmemBytes));
  if (e == cudaSuccess) done[device & 63] = true;
  return e;
}

template <int D, bool FP8>
static ms_status attend_launch(memstore* s, ChunkParams& c, int64_t max_rows, cudaStream_t st) {
  MS_CUDA(s, (attend_prepare<D, FP8>(s->cfg.device)));
  AttendParams& p = c.a;
  // Which kernels: the chunk kernel when a request may have more rows than the rows kernel serves well, the rows kernel when a
  // request may have fewer.  A single request whose rows are probably many goes to the chunk kernel whatever it turns out to be,
  // and one kernel is saved.
  const int min_rows = chunk_min_rows((int64_t)p.n_kv * p.nreq, s->sm_count);
  bool chunks = (D == 64 || D == 128) && max_rows > min_rows;
  const bool rows = !chunks || p.nreq > 1;
  c.min_rows = rows ? min_rows : 0;
  p.max_rows = chunks ? c.min_rows : 0x7fffffff;
  if (!chunks || !rows) p.gate = nullptr;  // (with both kernels there is a unit, so a join kernel too, which clears the word)
  c.step_tok = kChunkRows / p.group;
  c.step_sub = kChunkRows % p.group;
  const int64_t all_rows = (int64_t)p.n_tokens * p.group;
  p.tile_shift = __builtin_ctz((unsigned)AttnCfg<D, FP8>::kTileKeys);
  int chunk_ctas = 0, rows_ctas = 0;
  if constexpr (D == 64 || D == 128) {
    if (chunks) {
      chunk_ctas = s->sm_count;
      MS_CUDA(s, launch_dependent(attend_chunk_kernel<D, FP8>, dim3((unsigned)chunk_ctas), dim3(kChunkThreads), (ChunkCfg<D, FP8>::kSmemBytes), st, c));
      s->kernels_launched++;
      s->attn_chunks = true;
    }
  }
  if (rows) {
    rows_ctas = s->sm_count * AttnCfg<D, FP8>::kCtasPerSm;
    MS_CUDA(s, launch_dependent(attend_rows_kernel<D, FP8>, dim3((unsigned)rows_ctas), dim3(kAttnThreads), AttnCfg<D, FP8>::kSmemBytes, st, p));
    s->kernels_launched++;
  }
  const int checks = p.status ? (p.nreq + kCombineThreads / 32 - 1) / (kCombineThreads / 32) : 0;
  // units that the call can have at most, whatever the lengths on the device say, and so cuts to join (each unit has one first border)
  const int64_t units = (int64_t)p.n_kv * p.nreq;
  const int chunk_joins = (int)std::max<int64_t>(0, std::min<int64_t>(chunk_ctas - 1, units * (all_rows / kChunkRows + 1)));
  const int rows_joins = (int)std::max<int64_t>(0, std::min<int64_t>(rows_ctas - 1, units * (all_rows / kAttnRows + 1)));
  // Few cuts are spread over more blocks: 61 tokens of one request (8 cuts) 25 us with 16 pieces a cut, 39 with 4; a batch with 147 cuts
  // 57 us with 4, 60 with 16.
  const int pieces = chunk_joins <= 32 ? kChunkRows / kChunkJoinRows : 4;
  const int blocks = chunk_joins * pieces + rows_joins + checks;
  if (blocks > 0) {
    MS_CUDA(s, launch_dependent(attend_join_kernel<D>, dim3((unsigned)blocks), dim3(kCombineThreads), 0, st, c, chunk_ctas, chunk_joins, pieces, rows_ctas, rows_joins));
    s->kernels_launched++;
  }
  return MS_OK;
}
}  // extern "C++"

size_t memstore_attend_workspace(memstore_t* s) { return s ? attend_layout(s).bytes : 0; }

ms_status memstore_attend(memstore_t* s, int32_t layer, const ms_heads* q, int32_t n_q_heads, int32_t n_tokens, const int32_t* q_start,
                          const int32_t* seq_lens, int32_t nreq, const int32_t* block_tables, int32_t max_blocks, const ms_paged_cache* cache,
                          float scale, int32_t max_q_len, const ms_heads* out, float* out_lse, int32_t* out_status, void* workspace,
                          size_t workspace_bytes, ms_stream stream) {
  Range range("memstore_attend");
  if (!s) return MS_ERR_INVALID_ARG;
  std::lock_guard<std::recursive_mutex> lock(s->mu);
  const memstore_config& c = s->cfg;
  if (n_tokens < 0 || nreq < 0 || max_blocks < 0 || max_q_len < 0)
    return fail(s, MS_ERR_INVALID_ARG, "n_tokens=%d nreq=%d max_blocks=%d max_q_len=%d", n_tokens, nreq, max_blocks, max_q_len);
  if (n_q_heads <= 0 || n_q_heads % c.n_kv_heads)
    return fail(s, MS_ERR_INVALID_ARG, "%d query heads for %d K/V heads", n_q_heads, c.n_kv_heads);
  const int32_t group = n_q_heads / c.n_kv_heads;
  if (group > kAttnMaxGroup) return fail(s, MS_ERR_UNSUPPORTED, "%d query heads per K/V head (at most %d)", group, kAttnMaxGroup);
  if ((int64_t)n_tokens * group > kMaxCount) return fail(s, MS_ERR_UNSUPPORTED, "%d tokens of %d heads", n_tokens, n_q_heads);
  if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(s, MS_ERR_INVALID_ARG, "scale must be positive and finite, or 0 for the default");
  ms_status rc = check_cache(s, cache, layer, true);
  if (rc == MS_OK) rc = check_counts(s, nreq, max_blocks, 0);
  if (rc == MS_OK && nreq > kMaxAttendReqs) rc = fail(s, MS_ERR_UNSUPPORTED, "%d requests in one attention call (at most 2^26)", nreq);
  if (rc == MS_OK) rc = check_heads(s, q, n_tokens, n_q_heads, false, "q");
  if (rc == MS_OK) rc = check_heads(s, out, n_tokens, n_q_heads, true, "out");
  if (rc != MS_OK) return rc;
  if (nreq == 0) return MS_OK;
  if (!q_start || !seq_lens || (max_blocks > 0 && !block_tables)) return fail(s, MS_ERR_INVALID_ARG, "null request arrays");
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < memstore_attend_workspace(s))
    return fail(s, MS_ERR_INVALID_ARG, "a 256-byte aligned workspace of %zu bytes is needed", memstore_attend_workspace(s));
  DeviceGuard g(c.device);
  const bool fp8 = cache->dtype == MS_CACHE_FP8_E4M3;
  const int64_t esz = fp8 ? 1 : 2;
  ChunkParams cp{};
  AttendParams& p = cp.a;
  p.q = (const __nv_bfloat16*)q->base;
  p.q_ts = q->token_stride;
  p.q_hs = q->head_stride;
  p.out = (__nv_bfloat16*)out->base;
  p.o_ts = out->token_stride;
  p.o_hs = out->head_stride;
  p.n_q = n_q_heads;
  p.n_kv = c.n_kv_heads;
  p.group = group;
  p.group_magic = group == 1 ? 0u : (uint32_t)((1ull << 32) / (uint32_t)group + 1);
  p.n_tokens = n_tokens;
  p.q_start = q_start;
  p.seq_lens = seq_lens;
  p.nreq = nreq;
  p.tables = block_tables;
  p.max_blocks = max_blocks;
  p.k_cache = (const uint8_t*)cache->k_base + layer * cache->layer_stride * esz;
  p.v_cache = (const uint8_t*)cache->v_base + layer * cache->layer_stride * esz;
  p.block_stride = cache->block_stride * esz;
  p.token_stride = cache->token_stride * esz;
  p.head_stride = cache->head_stride * esz;
  p.num_blocks = cache->num_blocks;
  p.block_size = cache->block_size;
  p.block_shift = (p.block_size & (p.block_size - 1)) ? -1 : __builtin_ctz((unsigned)p.block_size);
  const double sc = scale > 0.f ? (double)scale : 1.0 / std::sqrt((double)c.head_dim);
  // (a scale of zero would turn the minus infinity of a masked score into NaN, an infinite one a score of zero)
  p.scale_log2 = (float)std::min(std::max(sc * 1.4426950408889634 * (fp8 ? (double)cache->k_scale : 1.0), (double)FLT_MIN), (double)FLT_MAX);
  p.v_scale = fp8 ? cache->v_scale : 1.f;
  p.lse = out_lse;
  p.status = out_status;
  p.min_share = 2;  // (one decode request of 2,033 tokens: 1 tile per CTA at least 12.6 us, 2 11.2, 4 10.9; long batches do not care)
  const AttendLayout w = attend_layout(s);
  char* base = (char*)workspace;
  p.part_o = (float*)(base + w.rows_o);
  p.part_ml = (float2*)(base + w.rows_ml);
  p.cuts = (AttnCut*)(base + w.rows_cuts);
  cp.min_share = 1;  // (61 tokens of one request: 24 us, with two or three tiles 32)
  cp.part_o = (float*)(base + w.chunk_o);
  cp.part_ml = (float2*)(base + w.chunk_ml);
  cp.cuts = (AttnCut*)(base + w.chunk_cuts);
  cp.errors = (int32_t*)(base + w.errors);
  p.gate = (unsigned long long*)(base + w.gate);
  cp.timed_out = s->attn_timed_out;
  cp.spin_limit = s->test_spin_limit;
  cp.mute_producer = s->test_mute_producers;
  const int64_t max_rows = (int64_t)(max_q_len > 0 && max_q_len < n_tokens ? max_q_len : n_tokens) * group;
  cudaStream_t st = (cudaStream_t)stream;
  switch (c.head_dim) {
    case 16: return fp8 ? attend_launch<16, true>(s, cp, max_rows, st) : attend_launch<16, false>(s, cp, max_rows, st);
    case 32: return fp8 ? attend_launch<32, true>(s, cp, max_rows, st) : attend_launch<32, false>(s, cp, max_rows, st);
    case 64: return fp8 ? attend_launch<64, true>(s, cp, max_rows, st) : attend_launch<64, false>(s, cp, max_rows, st);
    case 128: return fp8 ? attend_launch<128, true>(s, cp, max_rows, st) : attend_launch<128, false>(s, cp, max_rows, st);
    default: return fp8 ? attend_launch<256, true>(s, cp, max_rows, st) : attend_launch<256, false>(s, cp, max_rows, st);
  }
}

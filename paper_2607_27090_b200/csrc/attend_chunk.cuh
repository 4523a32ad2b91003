// Attention of new tokens over the paged cache (memstore_attend): the tensor-core kernel for chunks of tokens (tcgen05 + TMEM).
//
// Mathematics as in attend.cuh (one pass, running maximum and sum).  Bound: the tensor cores - 4 * head_dim operations per (query row,
// key) - with the exponentials close behind: a tile of 128 x 128 scores takes 2 x 512 tensor cycles (head_dim 128) and 1024 cycles
// of the SM's 16 exponentials per cycle.
//
// A unit is (request, K/V head, 256 rows): rows are (token, query head of the group) pairs, so K and V are read once for all heads
// of a group.  Two halves of 128 rows work in turn: while the tensor cores multiply for one half, the other half's warps form its
// weights.  Scores go to TMEM, a thread owns one row (no shuffles), the weights return to TMEM in the type of V over the scores'
// columns and are the A operand of the second product, whose accumulator stays in TMEM for the whole unit.
//   warps 0-3, 4-7  weights of rows 0-127, 128-255, and the epilogue
//   warps 8-11      loads: queries (scaled to fp16 for an 8-bit cache), then K and V tiles of 128 keys through a ring of 5 buffers,
//                   gathered through the block table with cp.async (8-bit: loaded, converted to fp16 exactly, stored)
//   warp 12         TMEM allocation, tcgen05.mma issue
// Work split: as in attend.cuh, the tiles of all units (causal: only as many as a unit's last row sees) form one line of which every
// CTA takes an equal share, so 64 units on 148 SMs balance as well as 6400.
// Running maximum: the weights are formed with the maximum of the tiles before, and formed again only when a tile's maximum exceeds it
// by more than 2^8 (then the accumulator is rescaled too): fp32 sums and weights of up to 256 lose nothing.
// Every wait is bounded; when one runs out the CTA reports it, frees its tensor memory and leaves.
#pragma once
#include "attend.cuh"
#include "score_gemm.cuh"

namespace ms {

constexpr int kChunkRows = 256;
constexpr int kChunkKeys = 128;
constexpr int kChunkStages = 5;
constexpr int kChunkLag = 2;          // tiles that a loading thread keeps in flight behind the one it issues
constexpr int kChunkThreads = 13 * 32;
constexpr int kChunkMaskRing = 8;     // (a tile's masks are read at most three tiles after the loader wrote them)
constexpr float kChunkSlack = 8.f;    // log2 of the growth of the maximum that is tolerated without rescaling

template <int D>
struct ChunkCfg {
  static constexpr int kHalves = D / 64;                             // 128-byte column blocks of a 16-bit row
  static constexpr int kTileBytes = kChunkKeys * D * 2;              // K or V tile, 16 bits per element
  static constexpr int kQBytes = kChunkRows * D * 2;
  static constexpr int kRingBytes = kChunkStages * kTileBytes;
  static constexpr int kSmemBytes = 1024 + kQBytes + kRingBytes + 1536;  // + alignment, barriers, masks
  static constexpr int kColO = 2 * kChunkKeys;                       // TMEM: S0, S1 (128 columns each), O0, O1 (D columns each)
  static constexpr int kTmemCols = 512;
};

struct ChunkParams {
  AttendParams a;
  int32_t min_rows;   // requests with more rows than this are served here
  int32_t min_share;
  float* part_o;      // [CTAs][2][D / 4][kChunkRows][4]
  float2* part_ml;    // [CTAs][2][kChunkRows]
  int32_t* errors;    // [CTAs]: 1 when a wait ran out
  uint32_t spin_limit;
  int mute_producer;
};

// Tiles of a unit: up to the last key that its last row sees (one at least: rows without keys are written too).
__device__ __forceinline__ int chunk_tiles(const AttendParams& p, const AttnReq& q, int rt) {
  const int last_row = min((rt + 1) * kChunkRows, q.rows) - 1;
  const int end = min(q.keys, q.len - q.n + last_row / p.group + 1);
  return max(1, (end + kChunkKeys - 1) / kChunkKeys);
}
__device__ __forceinline__ int chunk_row_tiles(const AttnReq& q) { return (q.rows + kChunkRows - 1) / kChunkRows; }
__device__ __forceinline__ int64_t chunk_head_tiles(const AttendParams& p, const AttnReq& q) {
  int64_t s = 0;
  for (int rt = 0; rt < chunk_row_tiles(q); ++rt) s += chunk_tiles(p, q, rt);
  return s;
}
__device__ __forceinline__ int64_t chunk_cost(const ChunkParams& c, const AttnReq& q) {
  if (q.n == 0 || q.rows <= c.min_rows) return 0;
  return chunk_head_tiles(c.a, q) * c.a.n_kv;
}

template <int THREADS>
__device__ __forceinline__ int64_t chunk_total(const ChunkParams& c, int64_t* s_warp) {
  int64_t sum = 0;
  for (int r = threadIdx.x; r < c.a.nreq; r += THREADS) sum += chunk_cost(c, attn_request(c.a, r));
  int64_t total;
  block_scan<THREADS>(sum, s_warp, &total);
  return total;
}

// A piece of a unit that one CTA works on: tiles t0 .. t1 - 1 of it.
struct ChunkSeg {
  int r, kvh, rt, t0, t1, tiles;
  AttnReq q;
};

// The unit that tile `off` of the line lies in, by the whole block; false when off lies behind the line.
template <int THREADS>
__device__ __forceinline__ bool chunk_locate(const ChunkParams& c, int64_t off, int64_t* s_warp, int64_t* s_found, ChunkSeg* seg) {
  int64_t before = 0;
  for (int r0 = 0; r0 < c.a.nreq; r0 += THREADS) {
    const int r = r0 + threadIdx.x;
    const int64_t cost = r < c.a.nreq ? chunk_cost(c, attn_request(c.a, r)) : 0;
    int64_t total;
    const int64_t end = before + block_scan<THREADS>(cost, s_warp, &total);
    if (off < before + total) {  // uniform
      if (cost > 0 && off >= end - cost && off < end) {
        s_found[0] = r;
        s_found[1] = off - (end - cost);
      }
      __syncthreads();
      seg->r = (int)s_found[0];
      seg->q = attn_request(c.a, seg->r);
      const int64_t per_head = chunk_head_tiles(c.a, seg->q);
      seg->kvh = (int)(s_found[1] / per_head);
      int64_t rem = s_found[1] % per_head;
      seg->rt = 0;
      for (;;) {
        seg->tiles = chunk_tiles(c.a, seg->q, seg->rt);
        if (rem < seg->tiles) break;
        rem -= seg->tiles;
        ++seg->rt;
      }
      seg->t0 = (int)rem;
      return true;
    }
    before += total;
  }
  return false;
}
// The unit after seg (t0 = 0); false behind the last request.
__device__ __forceinline__ bool chunk_next(const ChunkParams& c, ChunkSeg* seg) {
  seg->t0 = 0;
  if (++seg->rt == chunk_row_tiles(seg->q)) {
    seg->rt = 0;
    if (++seg->kvh == c.a.n_kv) {
      seg->kvh = 0;
      do {
        if (++seg->r >= c.a.nreq) return false;
        seg->q = attn_request(c.a, seg->r);
      } while (seg->q.n == 0 || seg->q.rows <= c.min_rows);
    }
  }
  seg->tiles = chunk_tiles(c.a, seg->q, seg->rt);
  return true;
}

// ---- tcgen05 forms that the scoring kernel does not use
// Shared-memory descriptor of V as the B operand whose N dimension (head_dim) is contiguous: rows of 128 bytes (64 elements of one
// key), 128-byte swizzled; 8-key groups are 1 KiB apart (stride offset), blocks of 64 elements one tile column apart (leading offset).
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t smem_addr, uint32_t block_bytes) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(block_bytes >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// A from tensor memory (lane = row, two 16-bit elements per column).
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %6, %7, %8}, p;\n\t"
      "}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u), "r"(0u), "r"(0u), "r"(0u)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// byte offset of 16-byte chunk c of row r in a [rows][64 elements] block with 128-byte swizzle
__device__ __forceinline__ int chunk_swz(int r, int c) { return r * 128 + ((c ^ (r & 7)) << 4); }

// The 32 columns of a row that the bits of `see` keep; the others become minus infinity.
__device__ __forceinline__ void chunk_mask(float* s, uint32_t see) {
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (!((see >> e) & 1u)) s[e] = -INFINITY;
}
// Bits of 32 keys from key k0 on that a row with last key lim may see, out of those that exist.
__device__ __forceinline__ uint32_t chunk_see(uint32_t there, int k0, int lim) {
  const int n = lim - k0;  // keys k0 .. k0 + n are seen
  return n >= 31 ? there : n < 0 ? 0u : there & ((2u << n) - 1u);
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kChunkThreads, 1) attend_chunk_kernel(const ChunkParams c) {
  using C = ChunkCfg<D>;
  const AttendParams& p = c.a;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* q_smem = smem;                    // [2 halves of rows][D / 64 column blocks][128 rows][128 B]
  uint8_t* ring = smem + C::kQBytes;         // kChunkStages tiles of [D / 64][128 keys][128 B]
  uint64_t* bars = reinterpret_cast<uint64_t*>(ring + C::kRingBytes);
  uint64_t* q_full = bars;
  uint64_t* q_empty = bars + 1;
  uint64_t* kv_full = bars + 2;
  uint64_t* kv_empty = kv_full + kChunkStages;
  uint64_t* s_full = kv_empty + kChunkStages;  // [2]
  uint64_t* p_full = s_full + 2;               // [2]
  uint64_t* o_full = p_full + 2;               // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_full + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* s_masks = tmem_slot + 4;           // [kChunkMaskRing][4]: keys of the tile that the table names
  uint32_t* s_bad = s_masks + 4 * kChunkMaskRing;  // [kChunkMaskRing][4]: a loading warp's part of the V tile holds values that are not
                                                   // finite (looked for in causal tiles only)
  float* s_qscale = reinterpret_cast<float*>(s_bad + 4 * kChunkMaskRing);  // [256], 8-bit cache: the rows' powers of two, inverted
  __shared__ int64_t s_warp[32], s_found[2];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(q_full, 4);
    mbar_init(q_empty, 1);
    for (int s = 0; s < kChunkStages; ++s) {
      mbar_init(&kv_full[s], 4);
      mbar_init(&kv_empty[s], 1);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(&s_full[h], 1);
      mbar_init(&p_full[h], 4);
      mbar_init(&o_full[h], 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  grid_dependency_wait();  // (before tensor memory is taken: a kernel before this one may still hold it)
  grid_launch_dependents();
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t limit = c.spin_limit ? c.spin_limit : kSpinLimit;

  const int64_t total = chunk_total<kChunkThreads>(c, s_warp);
  const int64_t share = attn_share(total, gridDim.x, c.min_share);
  int64_t off = blockIdx.x * share;
  const int64_t off_end = min(total, off + share);
  ChunkSeg seg;
  bool more = off < off_end && chunk_locate<kChunkThreads>(c, off, s_warp, s_found, &seg);
  // every role walks the same segments
  auto set_end = [&] { seg.t1 = (int)min((int64_t)seg.tiles, seg.t0 + (off_end - off)); };
  auto next = [&] {
    off += seg.t1 - seg.t0;
    more = off < off_end && chunk_next(c, &seg);
  };
  // tiles of a segment that hold keys (a unit without keys counts one tile on the line)
  auto n_tiles = [&] {
    const int last_row = min((seg.rt + 1) * kChunkRows, seg.q.rows) - 1;
    const int end = min(seg.q.keys, seg.q.len - seg.q.n + last_row / p.group + 1);
    return end <= 0 ? 0 : seg.t1 - seg.t0;
  };

  if (warp >= 8 && warp < 12) {
    // ------------------------------------------------------------------ loads
    const int w = warp - 8, lt = tid - 8 * 32;
    bool ok = !c.mute_producer;
    uint32_t q_ph = 1;
    int stage = 0, unpublished = 0, pub = 0, mask_at = 0;
    uint32_t ph = 1;
    auto publish = [&] {
      // this thread's copies into the stage have landed: make them visible to the tensor cores, then count the warp in
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&kv_full[pub]);
      if (++pub == kChunkStages) pub = 0;
      --unpublished;
    };
    for (; more && ok; next()) {
      set_end();
      const int nt = n_tiles();
      if (nt == 0) continue;
      const AttnReq& q = seg.q;
      const int row0 = seg.rt * kChunkRows, rows = min(kChunkRows, q.rows - row0);
      const int pos0 = q.len - q.n;
      const int key_end = min(q.keys, pos0 + (row0 + rows - 1) / p.group + 1), lim_min = pos0 + row0 / p.group;
      // everything in flight becomes visible before this warp waits for the unit before to end
      if (!FP8) cp_async_wait<0>();
      while (unpublished > 0) publish();
      ok = mbar_wait(q_empty, q_ph, abort_flag, limit);
      q_ph ^= 1u;
      if (!ok) break;
      // ---- queries: a warp takes 64 rows, 32 lanes a row (D / 32 elements each)
      {
        constexpr int kE = D / 32;  // 2 or 4 elements per lane
#pragma unroll 4
        for (int i = 0; i < kChunkRows / 4; ++i) {
          const int row = w * (kChunkRows / 4) + i;
          uint32_t x[kE / 2];
#pragma unroll
          for (int e = 0; e < kE / 2; ++e) x[e] = 0u;
          if (row < rows) {
            const int R = row0 + row;
            const __nv_bfloat16* src = p.q + (int64_t)(q.q0 + R / p.group) * p.q_ts + (int64_t)(seg.kvh * p.group + R % p.group) * p.q_hs + lane * kE;
            if constexpr (kE == 4) {
              const uint2 y = *reinterpret_cast<const uint2*>(src);
              x[0] = y.x, x[1] = y.y;
            } else {
              x[0] = *reinterpret_cast<const uint32_t*>(src);
            }
          }
          if constexpr (FP8) {  // to fp16 by a power of two per row (see attend.cuh)
            float m = 0.f;
#pragma unroll
            for (int e = 0; e < kE / 2; ++e) m = fmaxf(m, fmaxf(fabsf(bf16lo(x[e])), fabsf(bf16hi(x[e]))));
#pragma unroll
            for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const int ex = min(max(268 - (int)(__float_as_uint(m) >> 23), 13), 227);
            const float f = __uint_as_float((uint32_t)ex << 23);
            if (lane == 0) s_qscale[row] = __uint_as_float((uint32_t)(254 - ex) << 23);
#pragma unroll
            for (int e = 0; e < kE / 2; ++e) x[e] = pack_half(bf16lo(x[e]) * f, bf16hi(x[e]) * f);
          }
          const int byte = lane * kE * 2, blk = byte >> 7, in = byte & 127;
          uint8_t* dst = q_smem + (row >> 7) * (C::kQBytes / 2) + blk * 16384 + chunk_swz(row & 127, in >> 4) + (in & 15);
          if constexpr (kE == 4)
            *reinterpret_cast<uint2*>(dst) = make_uint2(x[0], x[1]);
          else
            *reinterpret_cast<uint32_t*>(dst) = x[0];
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
      }
      // ---- tiles: K, V, K, V ...; a thread looks up key lt of the tile, a warp copies its own 32 keys
      const int32_t* table = p.tables + (int64_t)seg.r * p.max_blocks;
      auto entry_of = [&](int t) {
        const int key = t * kChunkKeys + lt;
        return key < key_end ? __ldg(table + key / p.block_size) : -1;
      };
      int32_t nxt = entry_of(seg.t0);
      for (int t = seg.t0; ok && t < seg.t1; ++t) {
        const int32_t blk = nxt;
        if (t + 1 < seg.t1) nxt = entry_of(t + 1);
        const int key = t * kChunkKeys + lt;
        const bool live = blk >= 0 && blk < p.num_blocks;
        const int64_t at = live ? blk * p.block_stride + (key % p.block_size) * p.token_stride + seg.kvh * p.head_stride : 0;
        const uint32_t mask = __ballot_sync(0xffffffffu, live);
        const bool causal = t * kChunkKeys + kChunkKeys - 1 > lim_min;
        if (lane == 0) s_masks[mask_at * 4 + w] = mask;
        bool bad = false;
        for (int kv = 0; kv < 2; ++kv) {
          ok = mbar_wait(&kv_empty[stage], ph, abort_flag, limit);
          if (!ok) break;
          uint8_t* dst = ring + stage * C::kTileBytes;
          const uint8_t* base = kv ? p.v_cache : p.k_cache;
          if constexpr (!FP8) {
            const uint32_t du = smem_u32(dst);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int rl = i * 4 + (lane >> 3), row = w * 32 + rl, ch = lane & 7;
              const int64_t ro = __shfl_sync(0xffffffffu, at, rl);
              const bool there = (mask >> rl) & 1u;
#pragma unroll
              for (int b = 0; b < C::kHalves; ++b) cp_async16(du + b * 16384 + chunk_swz(row, ch), base + ro + b * 128 + ch * 16, there);
            }
            cp_async_commit();
          } else {
            constexpr int kLoads = 32 * D / 512;  // 16-byte loads per lane: the warp's 32 rows of D bytes
            uint4 x[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
              const int idx = i * 32 + lane, rl = idx / (D / 16), ch = idx % (D / 16);
              const int64_t ro = __shfl_sync(0xffffffffu, at, rl);
              x[i] = ((mask >> rl) & 1u) ? *reinterpret_cast<const uint4*>(base + ro + ch * 16) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
              const int idx = i * 32 + lane, row = w * 32 + idx / (D / 16), ch = idx % (D / 16);
              uint32_t y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
              if (kv && causal) {  // NaN codes become zeros here; the epilogue adds them to the rows that see them
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t m = __vcmpeq4(y[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                  bad = bad || m;
                  y[e] &= ~m;
                }
              }
              uint4 lo, hi;
              lo = make_uint4(e4m3x2_half2(y[0]), e4m3x2_half2(y[0] >> 16), e4m3x2_half2(y[1]), e4m3x2_half2(y[1] >> 16));
              hi = make_uint4(e4m3x2_half2(y[2]), e4m3x2_half2(y[2] >> 16), e4m3x2_half2(y[3]), e4m3x2_half2(y[3] >> 16));
              uint8_t* d = dst + (ch >> 2) * 16384;
              *reinterpret_cast<uint4*>(d + chunk_swz(row, 2 * (ch & 3))) = lo;
              *reinterpret_cast<uint4*>(d + chunk_swz(row, 2 * (ch & 3) + 1)) = hi;
            }
          }
          ++unpublished;
          const int here = stage;
          if (++stage == kChunkStages) {
            stage = 0;
            ph ^= 1u;
          }
          if constexpr (FP8) {
            if (kv) {
              const bool any = __any_sync(0xffffffffu, bad);
              if (lane == 0) s_bad[mask_at * 4 + w] = any;
            }
            publish();
          } else {
            if (kv && !causal && lane == 0) s_bad[mask_at * 4 + w] = 0u;
            if (kv && causal) {
              // (the last tiles of a unit) wait for the copies and look at the values: one that is not finite would reach rows that
              // must not see it as 0 * inf.  It becomes zero here, and the epilogue adds it to the rows that see it.
              cp_async_wait<0>();
#pragma unroll 1
              for (int i = 0; i < 8; ++i) {
                const int row = w * 32 + i * 4 + (lane >> 3), ch = lane & 7;
                for (int b = 0; b < C::kHalves; ++b) {
                  uint32_t* z = reinterpret_cast<uint32_t*>(ring + here * C::kTileBytes + b * 16384 + chunk_swz(row, ch));
                  for (int e = 0; e < 4; ++e) {
                    uint32_t m = 0u;
                    if ((z[e] & 0x7f80u) == 0x7f80u) m |= 0xffffu;
                    if ((z[e] & 0x7f800000u) == 0x7f800000u) m |= 0xffff0000u;
                    if (m) {
                      z[e] &= ~m;
                      bad = true;
                    }
                  }
                }
              }
              const bool any = __any_sync(0xffffffffu, bad);
              if (lane == 0) s_bad[mask_at * 4 + w] = any;
              while (unpublished > 0) publish();
            } else if (unpublished > kChunkLag) {
              cp_async_wait<kChunkLag>();
              publish();
            }
          }
        }
        if (++mask_at == kChunkMaskRing) mask_at = 0;
      }
    }
    if (!FP8) cp_async_wait<0>();
    while (unpublished > 0) publish();
  } else if (warp == 12) {
    // ------------------------------------------------------------------ tensor-core issue
    if (lane == 0) {
      constexpr uint32_t kTypes = FP8 ? 0u : (1u << 7) | (1u << 10);  // fp16 or bf16 operands
      constexpr uint32_t kIdescS = (1u << 4) | kTypes | ((uint32_t)(kChunkKeys >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      constexpr uint32_t kIdescO = (1u << 4) | kTypes | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      bool ok = true;
      uint32_t q_ph = 0, p_ph[2] = {0, 0};
      int stage = 0;
      uint32_t ph = 0;
      const uint32_t q_u = smem_u32(q_smem), ring_u = smem_u32(ring);
      for (; more && ok; next()) {
        set_end();
        const int nt = n_tiles();
        if (nt == 0) continue;
        const int halves = min(kChunkRows, seg.q.rows - seg.rt * kChunkRows) > 128 ? 2 : 1;
        ok = mbar_wait(q_full, q_ph, abort_flag, limit);
        q_ph ^= 1u;
        int v_stage = 0;
        uint32_t v_ph = 0;
        for (int j = 0; ok && j <= nt; ++j) {
          int k_stage = stage;
          if (j < nt) {
            ok = mbar_wait(&kv_full[stage], ph, abort_flag, limit);
            if (!ok) break;
          }
          for (int h = 0; ok && h < halves; ++h) {
            if (j > 0) {  // O += P V of the tile before
              if (h == 0) ok = mbar_wait(&kv_full[v_stage], v_ph, abort_flag, limit);
              if (ok) ok = mbar_wait(&p_full[h], p_ph[h], abort_flag, limit);
              if (!ok) break;
              p_ph[h] ^= 1u;
              tc_fence_after();
              const uint64_t vd = umma_desc_mn_sw128(ring_u + v_stage * C::kTileBytes, 16384);
#pragma unroll
              for (int k = 0; k < kChunkKeys / 16; ++k)  // 16 keys are two 1 KiB groups
                umma_f16_ts(tmem + C::kColO + h * D, tmem + h * kChunkKeys + k * 8, vd + (uint64_t)(k * 128), kIdescO, (j > 1 || k > 0) ? 1u : 0u);
              if (h == halves - 1) umma_commit(&kv_empty[v_stage]);
              if (j == nt) umma_commit(&o_full[h]);
            }
            if (j < nt) {  // S = Q K^T
              tc_fence_after();
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint64_t qd = umma_desc_k_sw128(q_u + h * (C::kQBytes / 2) + (k >> 2) * 16384) + (uint64_t)(2 * (k & 3));
                const uint64_t kd = umma_desc_k_sw128(ring_u + k_stage * C::kTileBytes + (k >> 2) * 16384) + (uint64_t)(2 * (k & 3));
                umma_f16(tmem + h * kChunkKeys, qd, kd, kIdescS, k > 0 ? 1u : 0u);
              }
              umma_commit(&s_full[h]);
            }
          }
          if (!ok) break;
          if (j < nt) {
            umma_commit(&kv_empty[k_stage]);
            if (j == nt - 1) umma_commit(q_empty);
            if (++stage == kChunkStages) {
              stage = 0;
              ph ^= 1u;
            }
            v_stage = stage;
            v_ph = ph;
            if (++stage == kChunkStages) {
              stage = 0;
              ph ^= 1u;
            }
          }
        }
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ weights, epilogue
    const int h = warp >> 2, row = tid;  // row of the unit (0 .. 255)
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + h * kChunkKeys, to = tmem + lanes + C::kColO + h * D;
    bool ok = true;
    uint32_t s_ph = 0, o_ph = 0;
    int mask_at = 0;
    for (; more && ok; next()) {
      set_end();
      const int nt = n_tiles();
      const AttnReq& q = seg.q;
      const int row0 = seg.rt * kChunkRows, rows = min(kChunkRows, q.rows - row0);
      const bool active = h == 0 || rows > 128;
      const int pos0 = q.len - q.n;
      const int lim = pos0 + (row0 + min(row, rows - 1)) / p.group, lim_min = pos0 + row0 / p.group;
      if (!active) {
        mask_at = (mask_at + nt) % kChunkMaskRing;
        continue;
      }
      float m = -INFINITY, l = 0.f, sc = p.scale_log2;
      bool any_bad = false;
      int v_at = 0;
      auto look_at_v = [&] {
        const uint4 b = *reinterpret_cast<const uint4*>(s_bad + v_at * 4);
        any_bad = any_bad || (b.x | b.y | b.z | b.w) != 0u;
      };
      for (int j = 0; j < nt; ++j) {
        ok = mbar_wait(&s_full[h], s_ph, abort_flag, limit);
        s_ph ^= 1u;
        if (!ok) break;
        tc_fence_after();
        if (FP8 && j == 0) sc = p.scale_log2 * s_qscale[row];
        const int k0 = (seg.t0 + j) * kChunkKeys;
        const uint4 there = *reinterpret_cast<const uint4*>(s_masks + mask_at * 4);
        if (j > 0) look_at_v();  // (of the tile before: its product with V was issued before these scores)
        v_at = mask_at;
        if (++mask_at == kChunkMaskRing) mask_at = 0;
        const uint32_t tw[4] = {there.x, there.y, there.z, there.w};
        const bool masked = k0 + kChunkKeys - 1 > lim_min || (there.x & there.y & there.z & there.w) != 0xffffffffu;
        uint32_t pk[kChunkKeys / 2];
        float sum = 0.f, mx = -INFINITY;
        // weights with maximum `mm` of the 128 scores, packed; their sum and the scores' maximum
        auto form = [&](float mm) {
          const float sub = mm == -INFINITY ? 0.f : mm;
          float s0 = 0.f, s1 = 0.f, x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            float s[32];
            tmem_ld32(ts + b * 32, s);
            tmem_ld_wait();
            if (masked) chunk_mask(s, chunk_see(tw[b], k0 + b * 32, lim));
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              x0 = fmaxf(x0, s[e]);
              x1 = fmaxf(x1, s[e + 1]);
              const float w0 = ex2(fmaf(s[e], sc, -sub)), w1 = ex2(fmaf(s[e + 1], sc, -sub));
              s0 += w0;
              s1 += w1;
              pk[b * 16 + e / 2] = FP8 ? pack_half(w0, w1) : pack_bf16(w0, w1);
            }
          }
          sum = s0 + s1;
          mx = fmaxf(x0, x1);
        };
        form(m);
        const float top = mx * sc;
        if (__any_sync(0xffffffffu, top > m + kChunkSlack)) {  // (always in a unit's first tile)
          const float n = top > m + kChunkSlack ? top : m;
          const float f = n == -INFINITY || m == n ? 1.f : ex2(m - n);
          if (j > 0) {
            // the accumulator holds the tiles before this one (the commit that signalled these scores follows their product)
#pragma unroll 1
            for (int b = 0; b < D / 32; ++b) {
              float o[32];
              tmem_ld32(to + b * 32, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= f;
              tmem_st16(to + b * 32, reinterpret_cast<const uint32_t*>(o));
              tmem_st16(to + b * 32 + 16, reinterpret_cast<const uint32_t*>(o) + 16);
            }
          }
          l *= f;
          m = n;
          form(m);
        }
        l += sum;
#pragma unroll
        for (int b = 0; b < 4; ++b) tmem_st16(ts + b * 16, pk + b * 16);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[h]);
      }
      if (ok && nt > 0) {
        ok = mbar_wait(&o_full[h], o_ph, abort_flag, limit);
        o_ph ^= 1u;
        tc_fence_after();
        look_at_v();
      }
      if (!ok) break;
      // ---- epilogue: this thread's row
      const bool whole = seg.t0 == 0 && seg.t1 == seg.tiles;
      const bool mine = row < rows;
      const int R = row0 + min(row, rows - 1), tok = q.q0 + R / p.group, head = seg.kvh * p.group + R % p.group;
      const float inv = l == 0.f ? 0.f : p.v_scale / l;
      const int64_t slot = (int64_t)blockIdx.x * 2 + (seg.t0 == 0 ? 1 : 0);
      if (mine) {
        if (whole) {
          if (p.lse) p.lse[(int64_t)tok * p.n_q + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        } else {
          c.part_ml[slot * kChunkRows + row] = make_float2(m, l);
        }
      }
#pragma unroll 1
      for (int b = 0; b < D / 32; ++b) {
        float o[32];
        if (nt > 0) {
          tmem_ld32(to + b * 32, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (any_bad) {
          // values that are not finite, at the keys of this segment's causal tiles that the row sees: their weight is positive, so
          // they decide the sum
          const int32_t* table = p.tables + (int64_t)seg.r * p.max_blocks;
          const int from = max(seg.t0, (lim_min + 1) / kChunkKeys) * kChunkKeys;
          const int to_key = min(min(lim, q.keys - 1), seg.t1 * kChunkKeys - 1);
          for (int key = from; key <= to_key; ++key) {
            const int32_t blk = __ldg(table + key / p.block_size);
            if (blk < 0 || blk >= p.num_blocks) continue;
            const uint8_t* v = p.v_cache + blk * p.block_stride + (key % p.block_size) * p.token_stride + seg.kvh * p.head_stride;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              if (FP8) {
                if ((v[b * 32 + e] & 0x7f) == 0x7f) o[e] = NAN;
              } else {
                const uint32_t x = (uint32_t)reinterpret_cast<const uint16_t*>(v)[b * 32 + e] << 16;
                if ((x & 0x7f800000u) == 0x7f800000u) o[e] += __uint_as_float(x);
              }
            }
          }
        }
        if (mine) {
          if (whole) {
            __nv_bfloat16* dst = p.out + tok * p.o_ts + head * p.o_hs + b * 32;
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              *reinterpret_cast<uint4*>(dst + e) = make_uint4(pack_bf16(o[e] * inv, o[e + 1] * inv), pack_bf16(o[e + 2] * inv, o[e + 3] * inv),
                                                              pack_bf16(o[e + 4] * inv, o[e + 5] * inv), pack_bf16(o[e + 6] * inv, o[e + 7] * inv));
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(c.part_o + ((slot * (D / 4) + b * 8 + e / 4) * kChunkRows + row) * 4) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
      }
      tc_fence_before();  // (the accumulator is read; the next unit's first product follows this warp's next arrival)
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    for (int w = 0; w < 4096; ++w) __nanosleep(256);  // let products and copies that may still be in flight end
  }
  if (tid == 0) c.errors[blockIdx.x] = *abort_flag;
  if (warp == 12) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
  }
}

// Joins the parts of a chunk unit that CTA borders cut: block (b - 1, y) looks at the border in front of CTA b's share and serves 16 rows
// of the unit there when that border is the unit's first.
constexpr int kChunkJoinRows = 16;
template <int D>
__device__ __forceinline__ void chunk_join(const ChunkParams& c, int b, int y, int ctas, int64_t* s_warp, int64_t* s_found) {
  const AttendParams& p = c.a;
  const int64_t total = chunk_total<kCombineThreads>(c, s_warp);
  const int64_t share = attn_share(total, ctas, c.min_share);
  const int64_t off = b * share;
  ChunkSeg seg;
  const bool found = off < total && chunk_locate<kCombineThreads>(c, off, s_warp, s_found, &seg);
  grid_dependency_wait();
  if (!found || seg.t0 == 0 || share < seg.t0) return;  // no unit is cut here, or an earlier border is the unit's first
  const int c_last = (int)((off - seg.t0 + seg.tiles - 1) / share);
  const int row0 = seg.rt * kChunkRows, rows = min(kChunkRows, seg.q.rows - row0);
  const int row = y * kChunkJoinRows + threadIdx.x % kChunkJoinRows;
  if (row >= rows) return;
  const int R = row0 + row, tok = seg.q.q0 + R / p.group, head = seg.kvh * p.group + R % p.group;
  for (int d4 = threadIdx.x / kChunkJoinRows; d4 < D / 4; d4 += kCombineThreads / kChunkJoinRows) {
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = b - 1; i <= c_last; ++i) {
      const int64_t slot = (int64_t)i * 2 + (i == b - 1 ? 1 : 0);
      const float2 ml = c.part_ml[slot * kChunkRows + row];
      const float4 x = *reinterpret_cast<const float4*>(c.part_o + ((slot * (D / 4) + d4) * kChunkRows + row) * 4);
      const float n = fmaxf(m, ml.x);
      const float fa = m == -INFINITY ? 1.f : ex2(m - n), fb = ml.x == -INFINITY ? 1.f : ex2(ml.x - n);
      l = l * fa + ml.y * fb;
      o = make_float4(o.x * fa + x.x * fb, o.y * fa + x.y * fb, o.z * fa + x.z * fb, o.w * fa + x.w * fb);
      m = n;
    }
    const float inv = l == 0.f ? 0.f : p.v_scale / l;
    *reinterpret_cast<uint2*>(p.out + tok * p.o_ts + head * p.o_hs + d4 * 4) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (p.lse && d4 == 0) p.lse[(int64_t)tok * p.n_q + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  }
}

// Joins what CTA borders cut and reports on the requests; the last kernel of a call.  Blocks: 16 rows of a border of the chunk kernel
// each, borders of the rows kernel, then four requests each.
template <int D>
__global__ void __launch_bounds__(kCombineThreads) attend_join_kernel(const ChunkParams c, const int chunk_ctas, const int rows_ctas) {
  __shared__ int64_t s_warp[32], s_found[2];
  grid_launch_dependents();
  // (every path waits for the kernels before this one, so that whatever waits for this kernel has waited for them)
  constexpr int kPieces = kChunkRows / kChunkJoinRows;
  int b = blockIdx.x;
  const int chunk_blocks = chunk_ctas > 1 ? (chunk_ctas - 1) * kPieces : 0, row_blocks = rows_ctas > 1 ? rows_ctas - 1 : 0;
  if (b < chunk_blocks) {
    chunk_join<D>(c, b / kPieces + 1, b % kPieces, chunk_ctas, s_warp, s_found);
  } else if (b < chunk_blocks + row_blocks) {
    rows_join<D>(c.a, b - chunk_blocks + 1, rows_ctas, s_warp, s_found);
  } else {
    grid_dependency_wait();
    attend_report(c.a, b - chunk_blocks - row_blocks, chunk_ctas > 0 ? c.errors : nullptr, chunk_ctas, c.min_rows);
  }
}

}  // namespace ms

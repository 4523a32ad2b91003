// Attention of new tokens over the paged cache (memstore_attend): the tensor-core kernel for chunks of tokens (tcgen05 + TMEM).
//
// Mathematics as in attend.cuh (one pass, running maximum and sum).  Bound: the tensor cores - 4 * head_dim operations per (query row,
// key) - with the exponentials close behind: a tile of 128 x 128 scores takes 2 x 512 tensor cycles (head_dim 128) and 1024 cycles
// of the SM's 16 exponentials per cycle.  (With head_dim 64 the products take half of that and the exponentials are the bound.)
// Measured: 2,047 tokens behind 11,653 with 40/8 heads of 128 490 us in short runs at 1,965 MHz (1.08 PFLOP/s, 0.63 of the measured
// product rate), 562 us (0.95) call after call, when the power limit holds the clock at 1,690 MHz; 512 tokens of 4,096 with 32/8 heads
// 57 us (head_dim 64: 46, 8-bit cache: 67).  A tile of 256 rows takes about 3,500 cycles against 2,048 of products: what is left is the
// chain of a half - scores out of TMEM, weights, their store over the scores, which the two warps of a row group do together (a barrier),
// second product, next scores - with one score tile per half in flight.  (At head_dim 128 the accumulators and two score tiles fill
// TMEM; at 64 a quarter is unused.)
//
// A unit is (request, K/V head, 256 rows): rows are (token, query head of the group) pairs, so K and V are read once for all heads
// of a group.  Two halves of 128 rows work in turn: while the tensor cores multiply for one half, the other half's warps form its
// weights.  Scores go to TMEM, two threads share a row (no shuffles), the weights return to TMEM in the type of V over the scores'
// columns and are the A operand of the second product, whose accumulator stays in TMEM for the whole unit.
//   warps 0-7, 8-15  queries (scaled to fp16 for an 8-bit cache), weights and epilogue of rows 0-127, 128-255: two threads share a row,
//                    64 of the tile's keys each (16 warps: a single warp per scheduler cannot keep the exponentials' unit busy)
//   warps 16-19      loads: K and V tiles of 128 keys through a ring of 5 buffers, gathered through the block table with cp.async
//                    (8-bit: the codes go to a place of the loading thread's own, a tile ahead, and are converted to fp16, exactly, from there)
//   warp 20          TMEM allocation, tcgen05.mma issue by one elected lane
//   warp 21          walks the CTA's share of the line and describes its units to the other roles (warps 22, 23 complete the warpgroup)
// Work split: as in attend.cuh, the tiles of all units (causal: only as many as a unit's last row sees) form one line of which every
// CTA takes an equal share, so 64 units on 148 SMs balance as well as 6400.  Starting and ending a unit costs as much as a few of its
// tiles, so each unit takes kChunkUnitCost places more on the line.  Places for that, and the time of a call (32/8 heads of 128,
// bf16): none: 2,048 tokens of 2,048 131 us, 512 of 512 39 us, 512 of 4,096 64 us, 64 of 32,000 70 us; three: 83, 30, 60, 65;
// four: 82, 30, 59, 63; five: 76, 33, 58, 61 (and an 8-bit cache 69 instead of 67).
// Running maximum: the weights are formed with the maximum of the tiles before; no maximum is looked for unless the sum of a thread's 64
// weights passes 2^14 (8-bit cache: 61,440), when the row takes a new maximum, its weights are formed again and its accumulator is
// rescaled.  fp32 sums, and weights of that size in bf16 or fp16, lose nothing by that.
// Every wait is bounded; when one runs out the CTA reports it, frees its tensor memory and leaves.
#pragma once
#include "attend.cuh"
#include "score_gemm.cuh"

namespace ms {

constexpr int kChunkRows = 256;
constexpr int kChunkKeys = 128;
constexpr int kChunkStages = 5;
constexpr int kChunkThreads = 24 * 32;
constexpr int kChunkRegsWeights = 88, kChunkRegsLoads = 72, kChunkRegsIssue = 56;
static_assert(4 * kChunkRegsWeights + kChunkRegsLoads + kChunkRegsIssue <= 6 * 80, "six warpgroups share the 80 registers a thread of the launch");
constexpr int kChunkUnitCost = 4;    // places on the line of tiles that stand for the set-up and the end of a unit
constexpr int kChunkMaskRing = 8;     // (a tile's masks are read at most three tiles after the loader wrote them)
constexpr uint32_t kChunkSpinLimit = 1u << 26;  // polls (a second or more)

template <int D, bool FP8>
struct ChunkCfg {
  static constexpr int kStages = FP8 ? 4 : kChunkStages;             // an 8-bit cache gives one tile's place to codes on their way
  static constexpr int kHalves = D / 64;                             // 128-byte column blocks of a 16-bit row
  static constexpr int kTileBytes = kChunkKeys * D * 2;              // K or V tile, 16 bits per element
  static constexpr int kQBytes = kChunkRows * D * 2;
  static constexpr int kRawBytes = FP8 ? kTileBytes : 0;             // two tiles of codes
  static constexpr int kRingBytes = kStages * kTileBytes + kRawBytes;
  static constexpr int kSmemBytes = 1024 + kQBytes + kRingBytes + 2048;  // alignment, tiles, barriers and small arrays
  static_assert(kSmemBytes <= 232448, "shared memory of a CTA");
  static constexpr int kColO = 2 * kChunkKeys;                       // TMEM: S0, S1 (128 columns each), O0, O1 (D columns each)
  static constexpr int kTmemCols = 512;
  // Sum of 64 weights (and so a weight) that is tolerated without taking a new maximum, and what the exponents are lifted by when one is
  // taken (see AttnCfg::kLift).  fp16 weights stay below 65,504; what the lift takes from the room above it is paid in new maxima where
  // scores spread: 512 tokens of 4,096 in an 8-bit cache (32/8 heads of 128, scores of standard deviation 1.5 / 3 / 4.5 / 7.5) take 66.7 / 66.7 /
  // 67.8 / 80.5 us without a lift, 66.6 / 66.8 / 71.6 / 82.8 with 4, 66.6 / 67.4 / 77.0 / 84.1 with 6, 66.6 / 71.7 / 82.0 / 85.0 with 8.
  static constexpr float kMaxSum = FP8 ? 61440.f : 16384.f;
  static constexpr float kLift = FP8 ? 4.f : 0.f;
};

struct ChunkParams {
  AttendParams a;
  int32_t min_rows;   // requests with more rows than this are served here
  int32_t min_share;
  int32_t step_tok, step_sub;  // kChunkRows / group and kChunkRows % group
  float* part_o;      // [CTAs][2][D / 4][kChunkRows][4]
  float2* part_ml;    // [CTAs][2][kChunkRows]
  AttnCut* cuts;      // [CTAs]
  int32_t* errors;    // [CTAs]: 1 when a wait ran out
  int32_t* timed_out; // of the store: set to 1 when one did, for whoever asks for no status
  uint32_t spin_limit;
  int mute_producer;
};

// The row tiles of a request one after another: token and query head of the group of the tile's first row.
struct ChunkWalk {
  int tok = 0, sub = 0;
  __device__ __forceinline__ void step(const ChunkParams& c) {
    tok += c.step_tok;
    sub += c.step_sub;
    if (sub >= c.a.group) {
      sub -= c.a.group;
      ++tok;
    }
  }
};
// Tiles of a unit: up to the last key that its last row sees (one at least: rows without keys are written too).
__device__ __forceinline__ int chunk_tiles(const AttendParams& p, const AttnReq& q, const ChunkWalk& w) {
  const int last = min(q.n - 1, w.tok + group_div(p, w.sub + kChunkRows - 1));
  return max(1, (min(q.keys, q.len - q.n + last + 1) + kChunkKeys - 1) / kChunkKeys);
}
__device__ __forceinline__ int chunk_row_tiles(const AttnReq& q) { return (q.rows + kChunkRows - 1) / kChunkRows; }
__device__ __forceinline__ int64_t chunk_head_cost(const ChunkParams& c, const AttnReq& q) {
  int64_t s = 0;
  ChunkWalk w;
  const int n = chunk_row_tiles(q);
  for (int rt = 0; rt < n; ++rt, w.step(c)) s += chunk_tiles(c.a, q, w) + kChunkUnitCost;
  return s;
}
__device__ __forceinline__ int64_t chunk_cost(const ChunkParams& c, const AttnReq& q) {
  if (q.n == 0 || q.rows <= c.min_rows) return 0;
  return chunk_head_cost(c, q) * c.a.n_kv;
}

// What the roles need to know of a unit, in a small ring of shared memory: worked out once, ahead of its use.
constexpr int kChunkUnits = 4;
struct __align__(16) ChunkUnit {
  int32_t nt;               // tiles with keys in this CTA's part, -1: no more units
  int32_t t0, t1;           // first tile, and one behind the last on the line (t1 - t0 = nt unless the unit has no keys)
  int32_t rows;             // rows of the unit
  int32_t req, kvh;         // request and K/V head
  int32_t tok0, sub0;       // token (row of q) and query head of the group of the unit's row 0
  int32_t lim_min;          // position of that token: last key that every row sees
  int32_t key_end;          // one behind the last key that any row sees
  int32_t keys;             // keys of the request that the table can name
  int32_t whole;            // all tiles of the unit are here
};

// A unit, and the place on it where a CTA's share begins (the first kChunkUnitCost places stand for its set-up, then come its tiles).
struct ChunkSeg {
  int r, kvh, rt, tiles, pos;
  ChunkWalk w;
  AttnReq q;
};

// The unit that place `off` of the line lies in; false when off lies behind the line.
template <int THREADS>
__device__ __forceinline__ bool chunk_locate(const ChunkParams& c, const AttnLine<THREADS>& line, int64_t off, int64_t* s_warp, int64_t* s_found,
                                             ChunkSeg* seg) {
  int64_t start, rem;
  seg->r = line.locate(c.a.nreq, [&](int i) { return chunk_cost(c, attn_request(c.a, i)); }, off, s_warp, s_found, &start);
  if (seg->r < 0) return false;
  seg->q = attn_request(c.a, seg->r);
  seg->kvh = (int)attn_div(off - start, chunk_head_cost(c, seg->q), &rem);
  seg->rt = 0;
  seg->w = ChunkWalk();
  for (;;) {
    seg->tiles = chunk_tiles(c.a, seg->q, seg->w);
    if (rem < seg->tiles + kChunkUnitCost) break;
    rem -= seg->tiles + kChunkUnitCost;
    ++seg->rt;
    seg->w.step(c);
  }
  seg->pos = (int)rem;
  return true;
}
// The unit after seg; false behind the last request.  By a whole warp: the other roles of the CTA wait while requests of the other kernel
// are passed over, 32 at a time (a million of them between two chunks: 4 ms).
__device__ __forceinline__ bool chunk_next(const ChunkParams& c, ChunkSeg* seg) {
  seg->pos = 0;
  seg->w.step(c);
  if (++seg->rt == chunk_row_tiles(seg->q)) {
    seg->rt = 0;
    seg->w = ChunkWalk();
    if (++seg->kvh == c.a.n_kv) {
      seg->kvh = 0;
      unsigned here = 0u;
      for (++seg->r; seg->r < c.a.nreq; seg->r += 32) {
        const int r = seg->r + (int)(threadIdx.x & 31);
        bool chunk = false;
        if (r < c.a.nreq) {
          const AttnReq q = attn_request(c.a, r);
          chunk = q.n != 0 && q.rows > c.min_rows;
        }
        here = __ballot_sync(0xffffffffu, chunk);
        if (here) break;
      }
      if (!here) return false;
      seg->r += __ffs(here) - 1;
      seg->q = attn_request(c.a, seg->r);
    }
  }
  seg->tiles = chunk_tiles(c.a, seg->q, seg->w);
  return true;
}

// ---- tcgen05 forms that the scoring kernel does not use
// Shared-memory descriptors, low and high words.  All tiles have rows of 128 bytes (64 elements), 128-byte swizzled, in groups of 8
// rows 1 KiB apart (the stride offset).  Q and K are K-major.  V as the B operand has its N dimension (head_dim) contiguous: blocks of
// 64 elements are one column block (16 KiB) apart, the leading offset.  Shared addresses fit the 14 bits of the address field (units of
// 16 bytes), so an advance is an addition to the low word.
constexpr uint32_t kDescHi = (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29);  // stride offset, version, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_lo_k(uint32_t smem_addr) { return (smem_addr >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_lo_mn(uint32_t smem_addr) { return (smem_addr >> 4) | ((uint32_t)(16384 >> 4) << 16); }
// (the whole warp comes here, so that operands stay in uniform registers; the lane with `lead` issues)
__device__ __forceinline__ void umma_ss(bool lead, uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p, e;\n\t"
      ".reg .b64 a, b;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 e, %6, 0;\n\t"
      "mov.b64 a, {%1, %5};\n\t"
      "mov.b64 b, {%2, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t"
      "}\n" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"((uint32_t)lead)
      : "memory");
}
// A from tensor memory (lane = row, two 16-bit elements per column)
__device__ __forceinline__ void umma_ts(bool lead, uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p, e;\n\t"
      ".reg .b64 b;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 e, %6, 0;\n\t"
      "mov.b64 b, {%2, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t"
      "}\n" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"((uint32_t)lead)
      : "memory");
}
__device__ __forceinline__ void umma_commit_if(bool lead, uint64_t* bar) {
  asm volatile("{ .reg .pred e; setp.ne.b32 e, %1, 0; @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(smem_u32(bar)), "r"((uint32_t)lead) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
        "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Bounded wait without pauses between the polls (a hundred nanoseconds between a barrier and its waiter would show in every tile).
__device__ __forceinline__ bool chunk_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  const uint32_t addr = smem_u32(bar);
  for (uint32_t spin = 0; spin < limit; ++spin) {
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
        : "=r"(ok)
        : "r"(addr), "r"(parity)
        : "memory");
    if (ok) return true;
    if ((spin & 63u) == 63u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{ .reg .pred q; elect.sync _|q, 0xffffffff; selp.u32 %0, 1, 0, q; }" : "=r"(p));
  return p != 0u;
}
// Barrier of the two warps that share 32 rows, and the same with the disjunction of a predicate.
__device__ __forceinline__ void pair_sync(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool pair_any(int id, bool v) {
  uint32_t r;
  asm volatile("{ .reg .pred p, q; setp.ne.u32 p, %2, 0; barrier.cta.red.or.pred q, %1, 64, p; selp.u32 %0, 1, 0, q; }" : "=r"(r) : "r"(id), "r"((uint32_t)v) : "memory");
  return r != 0u;
}

// ---- pairs of fp32 (the packed instructions round each half as the scalar ones do)
typedef unsigned long long f2;
__device__ __forceinline__ f2 f2_make(float a, float b) { return pack_f32x2(a, b); }
__device__ __forceinline__ void f2_split(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 f2_fma(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f2 f2_add(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// byte offset of 16-byte chunk c of row r in a [rows][64 elements] block with 128-byte swizzle
__device__ __forceinline__ int chunk_swz(int r, int c) { return r * 128 + ((c ^ (r & 7)) << 4); }

// The 16 scores that the low bits of `see` keep; the others become minus infinity.
__device__ __forceinline__ void chunk_mask(float* s, uint32_t see) {
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (!((see >> e) & 1u)) s[e] = -INFINITY;
}
// Bits of 32 keys from key k0 on that a row with last key lim may see, out of those that exist.
__device__ __forceinline__ uint32_t chunk_see(uint32_t there, int k0, int lim) {
  const int n = lim - k0;  // keys k0 .. k0 + n are seen
  return n >= 31 ? there : n < 0 ? 0u : there & ((2u << n) - 1u);
}

struct ChunkYes {
  static constexpr bool value = true;
};
struct ChunkNo {
  static constexpr bool value = false;
};

template <int D, bool FP8>
__global__ void __launch_bounds__(kChunkThreads, 1) attend_chunk_kernel(const ChunkParams c) {
  using C = ChunkCfg<D, FP8>;
  const AttendParams& p = c.a;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* q_smem = smem;                    // [2 halves of rows][D / 64 column blocks][128 rows][128 B]
  uint8_t* ring = smem + C::kQBytes;         // kChunkStages tiles of [D / 64][128 keys][128 B]
  uint64_t* bars = reinterpret_cast<uint64_t*>(ring + C::kRingBytes);
  uint64_t* q_full = bars;  // [2 halves]
  uint64_t* kv_full = bars + 2;
  uint64_t* kv_empty = kv_full + kChunkStages;
  uint64_t* s_full = kv_empty + kChunkStages;  // [2]
  uint64_t* p_full = s_full + 2;               // [2]
  uint64_t* o_full = p_full + 2;               // [2]
  uint64_t* u_full = o_full + 2;               // [kChunkUnits]
  uint64_t* u_empty = u_full + kChunkUnits;    // [kChunkUnits]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(u_empty + kChunkUnits);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* s_masks = tmem_slot + 4;           // [kChunkMaskRing][4]: keys of the tile that the table names
  // [kChunkMaskRing][4]: a loading warp's part of the V tile holds values that are not finite.  Looked for in causal tiles alone (0 for
  // the others); may be read once the next tile's scores, or the unit's last accumulator, are there.
  uint32_t* s_bad = s_masks + 4 * kChunkMaskRing;
  float* s_pair = reinterpret_cast<float*>(s_bad + 4 * kChunkMaskRing);  // [256]: exchange between the two threads of a row
  uint8_t* s_qexp = reinterpret_cast<uint8_t*>(s_pair + kChunkRows);  // [256], 8-bit cache: exponent fields of the rows' inverse powers of two
  int64_t* s_warp = reinterpret_cast<int64_t*>(s_qexp + kChunkRows);  // [32]
  int64_t* s_found = s_warp + 32;                                      // [2]
  ChunkUnit* units = reinterpret_cast<ChunkUnit*>(s_warp);             // [kChunkUnits], once the first unit has been found
  static_assert(sizeof(ChunkUnit) * kChunkUnits <= 32 * sizeof(int64_t), "the units' ring takes the place of the scan's");

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&kv_full[s], 4);
      mbar_init(&kv_empty[s], 1);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(&q_full[h], 8);
      mbar_init(&s_full[h], 1);
      mbar_init(&p_full[h], 8);
      mbar_init(&o_full[h], 1);
    }
    for (int i = 0; i < kChunkUnits; ++i) {
      mbar_init(&u_full[i], 1);
      mbar_init(&u_empty[i], 21);  // every warp of the other roles
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    if (p.gate && blockIdx.x == 0) {
      grid_dependency_wait();
      open_gate(p.gate);
    }
  }
  grid_dependency_wait();  // (before tensor memory is taken: a kernel before this one may still hold it)
  grid_launch_dependents();
  if (warp == 20) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  const uint32_t limit = c.spin_limit ? c.spin_limit : kChunkSpinLimit;

  auto cost_of = [&](int i) { return chunk_cost(c, attn_request(p, i)); };
  int64_t off = 0, off_end = 0, share = 1;
  ChunkSeg seg;
  bool more = false;
  auto find = [&] {
    AttnLine<kChunkThreads> line;
    line.init(p.nreq, cost_of, s_warp);
    share = attn_share(line.total, gridDim.x, c.min_share);
    off = blockIdx.x * share;
    off_end = min(line.total, off + share);
    more = off < off_end && chunk_locate<kChunkThreads>(c, line, off, s_warp, s_found, &seg);
  };
  if (p.nreq > 32 * kLinePerLane) {
    find();           // (by the whole block; few requests are looked through by the describing warp alone)
    __syncthreads();  // the scan's memory becomes the units' ring
  }
  // unit n of this CTA, once it has been described
  auto unit_ready = [&](int n) { return chunk_wait(&u_full[n % kChunkUnits], (uint32_t)(n / kChunkUnits) & 1u, abort_flag, limit); };
  auto unit_done = [&](int n) {
    if (lane == 0) mbar_arrive(&u_empty[n % kChunkUnits]);
  };

  if (warp >= 16 && warp < 20) {
    // ------------------------------------------------------------------ loads
    regs_down<kChunkRegsLoads>();
    const int w = warp - 16, lt = tid - 16 * 32;
    bool ok = !c.mute_producer;
    int stage = 0, pub = 0, unpublished = 0, mask_at = 0;
    uint32_t ph = 1;
    // the oldest tile's copies have landed: make them visible to the tensor cores, then count the warp in
    auto publish = [&] {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&kv_full[pub]);
      if (++pub == C::kStages) pub = 0;
      --unpublished;
    };
    // 8-bit cache: this thread's 16-byte pieces of its warp's 32 rows, into a place that only it reads
    constexpr int kLoads = 32 * D / 512;
    uint8_t* raw = ring + C::kStages * C::kTileBytes + lt * 16;
    int raw_in = 0, raw_out = 0;
    auto raw_issue = [&](const uint8_t* base, int64_t at, uint32_t mask) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int idx = i * 32 + lane, rl = idx / (D / 16), ch = idx % (D / 16);
        const int64_t ro = __shfl_sync(0xffffffffu, at, rl);
        cp_async16(smem_u32(raw + (raw_in * kLoads + i) * 2048), base + ro + ch * 16, (mask >> rl) & 1u);
      }
      cp_async_commit();
      raw_in ^= 1;
    };
    for (int n = 0; ok; ++n) {
      ok = unit_ready(n);
      if (!ok) break;
      const ChunkUnit u = units[n % kChunkUnits];
      __syncwarp();
      if (u.nt < 0) break;
      unit_done(n);
      if (u.nt == 0) {
        // A tile that has been held back (see below) goes out now: after a few units without keys the next description waits for the
        // weights of the last unit that had some, and those wait for this tile.
        cp_async_wait<0>();
        while (unpublished > 0) publish();
        continue;
      }
      const int t_end = u.t0 + u.nt;
      // ---- tiles: K, V, K, V ...; a thread looks up key lt of the tile, a warp copies its own 32 keys
      const int32_t* table = p.tables + (int64_t)u.req * p.max_blocks;
      auto entry_of = [&](int t) {
        const int key = t * kChunkKeys + lt;
        return key < u.key_end ? __ldg(table + attn_page(p, key)) : -1;
      };
      // where the row of this thread's key starts (bytes from the base of K or V), and which of the warp's keys there are
      auto row_of = [&](int32_t blk, int t, uint32_t* there) -> int64_t {
        const bool live = blk >= 0 && blk < p.num_blocks;
        *there = __ballot_sync(0xffffffffu, live);
        return live ? blk * p.block_stride + attn_in_page(p, t * kChunkKeys + lt) * p.token_stride + u.kvh * p.head_stride : 0;
      };
      uint32_t mask;
      int64_t at = row_of(entry_of(u.t0), u.t0, &mask);
      int32_t nxt = u.t0 + 1 < t_end ? entry_of(u.t0 + 1) : -1;
      if constexpr (FP8) raw_issue(p.k_cache, at, mask);
      for (int t = u.t0; ok && t < t_end; ++t) {
        uint32_t next_mask = 0u;
        int64_t next_at = 0;
        if (t + 1 < t_end) {
          next_at = row_of(nxt, t + 1, &next_mask);
          nxt = t + 2 < t_end ? entry_of(t + 2) : -1;
        }
        const bool causal = t * kChunkKeys + kChunkKeys - 1 > u.lim_min;
        if (lane == 0) s_masks[mask_at * 4 + w] = mask;
        bool bad = false;
        for (int kv = 0; kv < 2; ++kv) {
          if constexpr (FP8) {  // the next tile's codes, then wait for this one's
            if (kv == 0)
              raw_issue(p.v_cache, at, mask);
            else if (t + 1 < t_end)
              raw_issue(p.k_cache, next_at, next_mask);
            else
              cp_async_commit();
            cp_async_wait<1>();
          }
          ok = chunk_wait(&kv_empty[stage], ph, abort_flag, limit);
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
          } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
              const int idx = i * 32 + lane, row = w * 32 + idx / (D / 16), ch = idx % (D / 16);
              const uint4 x = *reinterpret_cast<const uint4*>(raw + (raw_out * kLoads + i) * 2048);
              uint32_t y[4] = {x.x, x.y, x.z, x.w};
              if (kv && causal) {  // NaN codes become zeros here; the epilogue adds them to the rows that see them
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t m = __vcmpeq4(y[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                  bad = bad || m;
                  y[e] &= ~m;
                }
              }
              uint4 lo, hi;
              e4m3x4_half2(y[0], lo.x, lo.y);
              e4m3x4_half2(y[1], lo.z, lo.w);
              e4m3x4_half2(y[2], hi.x, hi.y);
              e4m3x4_half2(y[3], hi.z, hi.w);
              uint8_t* d = dst + (ch >> 2) * 16384;
              *reinterpret_cast<uint4*>(d + chunk_swz(row, 2 * (ch & 3))) = lo;
              *reinterpret_cast<uint4*>(d + chunk_swz(row, 2 * (ch & 3) + 1)) = hi;
            }
            raw_out ^= 1;
          }
          if (!FP8) cp_async_commit();
          ++unpublished;
          if (kv && causal) {
            if constexpr (!FP8) {
              // (the last tiles of a unit) wait for the copies and look at the values: one that is not finite would reach rows that
              // must not see it as 0 * inf.  It becomes zero here, and the epilogue adds it to the rows that see it.
              asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int row = w * 32 + i * 4 + (lane >> 3), ch = lane & 7;
#pragma unroll
                for (int b = 0; b < C::kHalves; ++b) {
                  uint4* at16 = reinterpret_cast<uint4*>(dst + b * 16384 + chunk_swz(row, ch));
                  const uint4 z = *at16;
                  const uint32_t y[4] = {z.x, z.y, z.z, z.w};
                  uint32_t keep[4];
                  bool some = false;
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    keep[e] = ((y[e] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((y[e] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
                    some = some || keep[e] != 0xffffffffu;
                  }
                  if (some) {
                    *at16 = make_uint4(y[0] & keep[0], y[1] & keep[1], y[2] & keep[2], y[3] & keep[3]);
                    bad = true;
                  }
                }
              }
            }
            bad = __any_sync(0xffffffffu, bad);
          }
          if (kv && lane == 0) s_bad[mask_at * 4 + w] = bad;
          if (FP8 || (kv && causal)) {
            while (unpublished > 0) publish();
          } else if (unpublished > 1) {  // (this one is on its way, the one before has had the time of a tile)
            cp_async_wait<1>();
            publish();
          }
          if (++stage == C::kStages) {
            stage = 0;
            ph ^= 1u;
          }
        }
        if (++mask_at == kChunkMaskRing) mask_at = 0;
        at = next_at;
        mask = next_mask;
      }
    }
    cp_async_wait<0>();
    while (unpublished > 0) publish();
  } else if (warp >= 20) {
    // ------------------------------------------------------------------ tensor-core issue
    regs_down<kChunkRegsIssue>();
    if (warp == 21) {
      // ---------------------------------------------------------------- units
      if (p.nreq <= 32 * kLinePerLane) find();
      bool ok = true;
      for (int n = 0; ok; ++n) {
        ChunkUnit u{};
        u.nt = -1;
        int64_t begin = off;
        int pos = 0, tiles = 0;
        while (more && u.nt < 0) {
          begin = off;
          pos = seg.pos;
          tiles = seg.tiles;
          const int here = (int)min((int64_t)(tiles + kChunkUnitCost - pos), off_end - off);  // places of this CTA on the unit
          u.t0 = max(0, pos - kChunkUnitCost);
          u.t1 = max(0, pos + here - kChunkUnitCost);
          if (u.t1 > u.t0) {
            u.rows = min(kChunkRows, seg.q.rows - seg.rt * kChunkRows);
            u.req = seg.r;
            u.kvh = seg.kvh;
            u.tok0 = seg.q.q0 + seg.w.tok;
            u.sub0 = seg.w.sub;
            u.lim_min = seg.q.len - seg.q.n + seg.w.tok;
            u.key_end = min(seg.q.keys, u.lim_min + group_div(p, u.sub0 + u.rows - 1) + 1);
            u.keys = seg.q.keys;
            u.nt = u.key_end <= 0 ? 0 : u.t1 - u.t0;
            u.whole = u.t0 == 0 && u.t1 == tiles;
          }
          off += here;
          more = off < off_end && chunk_next(c, &seg);
        }
        if (n == 0 && lane == 0) {
          AttnCut cut{};
          cut.c_last = -1;
          if (u.nt >= 0 && u.t0 != 0 && share >= u.t0) {  // the border before this CTA cuts the unit, and is the first that does
            int64_t rem;
            cut.c_last = (int)attn_div(begin - pos + tiles + kChunkUnitCost - 1, share, &rem);
            cut.rows = u.rows;
            cut.tok0 = u.tok0;
            cut.sub0 = u.sub0;
            cut.head0 = u.kvh * p.group;
          }
          c.cuts[blockIdx.x] = cut;
        }
        ok = chunk_wait(&u_empty[n % kChunkUnits], ((uint32_t)(n / kChunkUnits) & 1u) ^ 1u, abort_flag, limit);
        if (!ok) break;
        if (lane == 0) {
          units[n % kChunkUnits] = u;
          mbar_arrive(&u_full[n % kChunkUnits]);
        }
        if (u.nt < 0) break;
      }
    } else if (warp == 20) {
      const bool lead = elect_one();
      constexpr uint32_t kTypes = FP8 ? 0u : (1u << 7) | (1u << 10);  // fp16 or bf16 operands
      constexpr uint32_t kIdescS = (1u << 4) | kTypes | ((uint32_t)(kChunkKeys >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      constexpr uint32_t kIdescO = (1u << 4) | kTypes | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      bool ok = true;
      uint32_t q_ph = 0, p_ph[2] = {0, 0};
      int stage = 0;
      uint32_t ph = 0;
      const uint32_t q_u = smem_u32(q_smem), ring_u = smem_u32(ring);
      for (int n = 0; ok; ++n) {
        ok = unit_ready(n);
        if (!ok) break;
        const int nt = units[n % kChunkUnits].nt, halves = units[n % kChunkUnits].rows > 128 ? 2 : 1;
        __syncwarp();
        if (nt < 0) break;
        unit_done(n);
        if (nt == 0) continue;
        int v_stage = 0;
        uint32_t v_ph = 0;
        for (int j = 0; ok && j <= nt; ++j) {
          int k_stage = stage;
          if (j < nt) {
            ok = chunk_wait(&kv_full[stage], ph, abort_flag, limit);
            if (!ok) break;
          }
          for (int h = 0; ok && h < halves; ++h) {
            if (j > 0) {  // O += P V of the tile before
              if (h == 0) ok = chunk_wait(&kv_full[v_stage], v_ph, abort_flag, limit);
              if (ok) ok = chunk_wait(&p_full[h], p_ph[h], abort_flag, limit);
              if (!ok) break;
              p_ph[h] ^= 1u;
              tc_fence_after();
              const uint32_t vd = desc_lo_mn(ring_u + v_stage * C::kTileBytes);
#pragma unroll
              for (int k = 0; k < kChunkKeys / 16; ++k)  // 16 keys are two 1 KiB groups
                umma_ts(lead, tmem + C::kColO + h * D, tmem + h * kChunkKeys + k * 8, vd + k * 128, kIdescO, (j > 1 || k > 0) ? 1u : 0u);
              if (h == halves - 1) umma_commit_if(lead, &kv_empty[v_stage]);
              if (j == nt) umma_commit_if(lead, &o_full[h]);
            }
            if (j < nt) {  // S = Q K^T
              if (j == 0) {
                ok = chunk_wait(&q_full[h], (q_ph >> h) & 1u, abort_flag, limit);
                if (!ok) break;
                q_ph ^= 1u << h;
              }
              tc_fence_after();
              const uint32_t qd = desc_lo_k(q_u + h * (C::kQBytes / 2)), kd = desc_lo_k(ring_u + k_stage * C::kTileBytes);
#pragma unroll
              for (int k = 0; k < D / 16; ++k)  // 16 elements are 32 bytes of a row, 64 a column block
                umma_ss(lead, tmem + h * kChunkKeys, qd + (k >> 2) * 1024 + 2 * (k & 3), kd + (k >> 2) * 1024 + 2 * (k & 3), kIdescS, k > 0 ? 1u : 0u);
              umma_commit_if(lead, &s_full[h]);
            }
          }
          if (!ok) break;
          if (j < nt) {
            umma_commit_if(lead, &kv_empty[k_stage]);
            if (++stage == C::kStages) {
              stage = 0;
              ph ^= 1u;
            }
            v_stage = stage;
            v_ph = ph;
            if (++stage == C::kStages) {
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
    regs_up<kChunkRegsWeights>();
    const int h = warp >> 3, part = (warp >> 2) & 1;     // half of the rows; half of a tile's keys and of the accumulator's columns
    const int row = h * 128 + (warp & 3) * 32 + lane;    // of the unit
    const int pair = 1 + h * 4 + (warp & 3);             // barrier of the two warps that share these rows
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + h * kChunkKeys, to = tmem + lanes + C::kColO + h * D + part * (D / 2);
    // both threads of a row get what `join` makes of their values
    auto pair_join = [&](float v, auto join) {
      if (part) s_pair[row] = v;
      pair_sync(pair);
      if (!part) {
        v = join(v, s_pair[row]);
        s_pair[row] = v;
      }
      pair_sync(pair);
      if (part) v = s_pair[row];
      return v;
    };
    bool ok = true;
    uint32_t s_ph = 0, o_ph = 0;
    int mask_at = 0;
    // queries of this warp's 16 rows of a unit, 16 bytes a lane; the products of the unit before have read theirs
    auto load_queries = [&](const ChunkUnit& g) {
      constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes, kLoads = 16 / kPerWarp;  // lanes of a row, rows of a load
      const int ql = lane % kLanes, first = h * 128 + (warp & 3) * 32 + part * 16 + lane / kLanes;
      const int rows = g.rows, sub0 = g.sub0, head0 = g.kvh * p.group;
      const __nv_bfloat16* q0 = p.q + g.tok0 * p.q_ts + ql * 8;
      auto place = [&](int r) { return q_smem + h * (C::kQBytes / 2) + (ql >> 3) * 16384 + chunk_swz(r & 127, ql & 7); };
      auto source = [&](int r) {
        const int dt = group_div(p, sub0 + r);
        return q0 + dt * p.q_ts + (int64_t)(head0 + sub0 + r - dt * p.group) * p.q_hs;
      };
      if constexpr (!FP8) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int r = first + i * kPerWarp;
          cp_async16(smem_u32(place(r)), r < rows ? source(r) : p.q, r < rows);
        }
        cp_async_commit();
        cp_async_wait<0>();
      } else {
        uint4 x[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int r = first + i * kPerWarp;
          x[i] = make_uint4(0u, 0u, 0u, 0u);
          if (r < rows) x[i] = *reinterpret_cast<const uint4*>(source(r));
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          // to fp16 by a power of two per row (see attend.cuh)
          const int r = first + i * kPerWarp;
          uint32_t y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          float top = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(bf16lo(y[e])), fabsf(bf16hi(y[e]))));
#pragma unroll
          for (int o = kLanes / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          const int ex = min(max(268 - (int)(__float_as_uint(top) >> 23), 13), 227);
          const float f = __uint_as_float((uint32_t)ex << 23);
          if (ql == 0) s_qexp[r] = (uint8_t)(254 - ex);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = pack_half(bf16lo(y[e]) * f, bf16hi(y[e]) * f);
          *reinterpret_cast<uint4*>(place(r)) = make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[h]);
    };
    // (the two warps of a pair always learn the same of a wait: neither is left at a barrier)
    bool ready = false, loaded = false;  // the unit has been waited for already, and its queries loaded
    for (int n = 0; ok; ++n) {
      if (!ready) ok = !pair_any(pair, !unit_ready(n));
      if (!ok) break;
      ready = false;
      const ChunkUnit& un = units[n % kChunkUnits];
      const int nt = un.nt;
      if (nt < 0) break;
      const int rows = un.rows;
      if (h == 1 && rows <= 128) {
        mask_at = (mask_at + nt) % kChunkMaskRing;
        __syncwarp();
        unit_done(n);
        continue;
      }
      if (!loaded && nt > 0) load_queries(un);
      loaded = false;
      const int lim_min = un.lim_min, lim = lim_min + group_div(p, un.sub0 + min(row, rows - 1)), t0 = un.t0;
      float m = -INFINITY, l = 0.f, sc = p.scale_log2;
      bool any_bad = false;
      int v_at = 0;
      bool v_causal = false;  // the tile before was a causal one
      auto look_at_v = [&] {
        const uint4 b = *reinterpret_cast<const uint4*>(s_bad + v_at * 4);
        any_bad = any_bad || (b.x | b.y | b.z | b.w) != 0u;
      };
      for (int j = 0; j < nt; ++j) {
        ok = chunk_wait(&s_full[h], s_ph, abort_flag, limit);
        s_ph ^= 1u;
        tc_fence_after();
        if (FP8 && j == 0) sc = attn_scale(p.scale_log2, s_qexp[row]);
        const int k0 = (t0 + j) * kChunkKeys + part * 64;
        const uint2 there = *reinterpret_cast<const uint2*>(s_masks + mask_at * 4 + part * 2);
        if (v_causal) look_at_v();  // (of the tile before: its product with V was issued before these scores)
        v_at = mask_at;
        v_causal = (t0 + j) * kChunkKeys + kChunkKeys - 1 > lim_min;
        if (++mask_at == kChunkMaskRing) mask_at = 0;
        const bool masked = k0 + 63 > lim_min || (there.x & there.y) != 0xffffffffu;
        uint32_t pk[32];
        float sum = 0.f;
        // weights of the 64 scores with maximum `mm`, rounded to the 16 bits that the product takes (V has no more; half a step is
        // 2^-9 of a bf16 weight, 2^-12 of an fp16 one) and packed, and the fp32 sum of the unrounded ones
        auto form = [&](float mm, auto with_mask) {
          const float sub = mm == -INFINITY ? 0.f : -mm;
          const f2 sc2 = f2_make(sc, sc), sub2 = f2_make(sub, sub);
          f2 total2 = 0ull;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            float s[16];
            tmem_ld16(ts + part * 64 + b * 16, s);
            tmem_ld_wait();
            if (with_mask.value) chunk_mask(s, chunk_see(b >= 2 ? there.y : there.x, k0 + (b >> 1) * 32, lim) >> ((b & 1) * 16));
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              float w0, w1;
              f2_split(f2_fma(f2_make(s[e], s[e + 1]), sc2, sub2), w0, w1);
              w0 = ex2(w0);
              w1 = ex2(w1);
              total2 = f2_add(total2, f2_make(w0, w1));
              pk[b * 8 + e / 2] = FP8 ? pack_half(w0, w1) : pack_bf16(w0, w1);
            }
          }
          float a, b;
          f2_split(total2, a, b);
          sum = a + b;
        };
        auto form_any = [&](float mm) {
          if (masked)
            form(mm, ChunkYes{});
          else
            form(mm, ChunkNo{});
        };
        // A new maximum is taken first in a segment's first tile, and later when the sum asks for one.  (The vote is also the point
        // from which both warps have read their scores, over which the weights are stored.)
        bool renew = j == 0, again = renew, stop = false;  // stop: a wait ran out, and both warps leave together
        if (again) stop = pair_any(pair, !ok);
#pragma unroll 1
        while (!stop) {
          if (again) {
            float mx = -INFINITY;
#pragma unroll 1
            for (int b = 0; b < 2; ++b) {
              float s[32];
              tmem_ld32(ts + part * 64 + b * 32, s);
              tmem_ld_wait();
              if (masked) {
                const uint32_t see = chunk_see(b ? there.y : there.x, k0 + b * 32, lim);
                chunk_mask(s, see);
                chunk_mask(s + 16, see >> 16);
              }
#pragma unroll
              for (int e = 0; e < 32; e += 2) mx = max3(mx, s[e], s[e + 1]);
            }
            // (a row's maximum changes by its own scores alone, so that a row does not depend on its neighbours)
            mx = pair_join(mx, [](float a, float b) { return fmaxf(a, b); });
            const bool own = j == 0 || pair_join(renew ? 1.f : 0.f, [](float a, float b) { return fmaxf(a, b); }) != 0.f;
            const float n = own ? fmaxf(m, fmaf(mx, sc, -C::kLift)) : m;
            const float f = n == -INFINITY || m == n ? 1.f : ex2(m - n);
            if (j > 0) {
              // the accumulator holds the tiles before this one (the commit that signalled these scores follows their product)
#pragma unroll 1
              for (int b = 0; b < D / 2; b += 16) {
                float o[16];
                tmem_ld16(to + b, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] *= f;
                tmem_st16(to + b, reinterpret_cast<const uint32_t*>(o));
              }
            }
            l *= f;
            m = n;
          }
          if (ok) form_any(m);
          if (again) {
            pair_sync(pair);
            break;
          }
          renew = sum > C::kMaxSum || m == -INFINITY;
          again = pair_any(pair, !ok || renew);
          if (!again) break;
          stop = pair_any(pair, !ok);
        }
        if (stop) {
          ok = false;
          break;
        }
        l += sum;
        tmem_st16(ts + part * 32, pk);
        tmem_st16(ts + part * 32 + 16, pk + 16);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[h]);
      }
      // all scores of this half have been taken, so its queries' place is free: the next unit's come while the last product runs
      if (ok) {
        ok = !pair_any(pair, !unit_ready(n + 1));
        const ChunkUnit& next = units[(n + 1) % kChunkUnits];
        ready = ok;
        if (ok && next.nt > 0 && (h == 0 || next.rows > 128)) {
          load_queries(next);
          loaded = true;
        }
      }
      if (ok && nt > 0) {
        ok = chunk_wait(&o_full[h], o_ph, abort_flag, limit);
        o_ph ^= 1u;
        tc_fence_after();
        if (v_causal) look_at_v();
        ok = !pair_any(pair, !ok);
      }
      if (!ok) break;
      // ---- epilogue: this thread's half of its row
      if (nt > 0) l = pair_join(l, [](float a, float b) { return a + b; });
      const bool whole = un.whole != 0;
      const bool mine = row < rows;
      const int sr = un.sub0 + min(row, rows - 1), dt = group_div(p, sr), tok = un.tok0 + dt, head = un.kvh * p.group + sr - dt * p.group;
      const float inv = l == 0.f ? 0.f : p.v_scale / l;
      const int64_t slot = (int64_t)blockIdx.x * 2 + (t0 == 0 ? 1 : 0);
      if (mine && part == 0) {
        if (whole) {
          if (p.lse) p.lse[(int64_t)tok * p.n_q + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        } else {
          c.part_ml[slot * kChunkRows + row] = make_float2(m, l);
        }
      }
#pragma unroll 1
      for (int b = 0; b < D / 2; b += 32) {
        const int col = part * (D / 2) + b;
        float o[32];
        if (nt > 0) {
          tmem_ld32(to + b, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (any_bad) {
          // values that are not finite, at the keys of this segment's causal tiles that the row sees: their weight is positive, so
          // they decide the sum
          const int32_t* table = p.tables + (int64_t)un.req * p.max_blocks;
          const int from = max(t0, (lim_min + 1) / kChunkKeys) * kChunkKeys;
          const int to_key = min(min(lim, un.keys - 1), un.t1 * kChunkKeys - 1);
          for (int key = from; key <= to_key; ++key) {
            const int32_t blk = __ldg(table + key / p.block_size);
            if (blk < 0 || blk >= p.num_blocks) continue;
            const uint8_t* v = p.v_cache + blk * p.block_stride + (key % p.block_size) * p.token_stride + un.kvh * p.head_stride;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              if (FP8) {
                if ((v[col + e] & 0x7f) == 0x7f) o[e] = NAN;
              } else {
                const uint32_t x = (uint32_t)reinterpret_cast<const uint16_t*>(v)[col + e] << 16;
                if ((x & 0x7f800000u) == 0x7f800000u) o[e] += __uint_as_float(x);
              }
            }
          }
        }
        if (mine) {
          if (whole) {
            __nv_bfloat16* dst = p.out + tok * p.o_ts + head * p.o_hs + col;
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              *reinterpret_cast<uint4*>(dst + e) = make_uint4(pack_bf16(o[e] * inv, o[e + 1] * inv), pack_bf16(o[e + 2] * inv, o[e + 3] * inv),
                                                              pack_bf16(o[e + 4] * inv, o[e + 5] * inv), pack_bf16(o[e + 6] * inv, o[e + 7] * inv));
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(c.part_o + ((slot * (D / 4) + (col + e) / 4) * kChunkRows + row) * 4) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
      }
      __syncwarp();
      unit_done(n);
      tc_fence_before();  // (the accumulator is read; the next unit's first product follows this warp's next arrival)
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    for (int w = 0; w < 4096; ++w) __nanosleep(256);  // let products and copies that may still be in flight end
  }
  if (tid == 0) {
    c.errors[blockIdx.x] = *abort_flag;
    if (*abort_flag) *c.timed_out = 1;
  }
  if (warp == 20) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
  }
}

// Joins 16 rows of the chunk unit that the border in front of CTA b's share cuts, if it is the unit's first border.
constexpr int kChunkJoinRows = 16;
template <int D>
__device__ __forceinline__ void chunk_join(const ChunkParams& c, int b, int row0) {
  const AttendParams& p = c.a;
  const AttnCut cut = c.cuts[b];
  const int row = row0 + threadIdx.x % kChunkJoinRows;
  if (row >= cut.rows) return;
  const int c_last = cut.c_last, dt = group_div(p, cut.sub0 + row), tok = cut.tok0 + dt, head = cut.head0 + cut.sub0 + row - dt * p.group;
  for (int d4 = threadIdx.x / kChunkJoinRows; d4 < D / 4; d4 += kCombineThreads / kChunkJoinRows) {
    JoinSum sum;
    for (int i0 = b - 1; i0 <= c_last; i0 += kJoinBatch) {
      float2 ml[kJoinBatch];
      float4 x[kJoinBatch];
#pragma unroll
      for (int k = 0; k < kJoinBatch; ++k) {
        const int i = i0 + k;
        if (i > c_last) break;  // uniform
        const int64_t slot = (int64_t)i * 2 + (i == b - 1 ? 1 : 0);
        ml[k] = c.part_ml[slot * kChunkRows + row];
        x[k] = *reinterpret_cast<const float4*>(c.part_o + ((slot * (D / 4) + d4) * kChunkRows + row) * 4);
      }
      sum.add(ml, x, c_last - i0 + 1);
    }
    sum.write(p, tok, head, d4 * 4);
  }
}

// Joins what CTA borders cut and reports on the requests; the last kernel of a call.  Blocks: `pieces` for each cut unit of the chunk
// kernel (16 rows at a time), cut units of the rows kernel, then sixteen requests each.  There are as many blocks as units could be
// cut - no more than there are units or borders - and block n looks for the n-th cut among those that the CTAs recorded.
// Bound: L2 (147 cuts of 256 rows x 128 elements, two or three fp32 parts each: 40 MB, 20 us alone) and the latency of a block's few
// dependent loads, so two blocks share an SM (one block an SM: 28 us) and only parts that exist are loaded.
template <int D>
__global__ void __launch_bounds__(kCombineThreads, 2) attend_join_kernel(const ChunkParams c, const int chunk_ctas, const int chunk_joins, const int pieces,
                                                                      const int rows_ctas, const int rows_joins) {
  grid_launch_dependents();
  grid_dependency_wait();
  if (c.a.gate && blockIdx.x == 0 && threadIdx.x == 0) *c.a.gate = 0;
  int b = blockIdx.x;
  if (b < chunk_joins * pieces) {
    const int cta = nth_cut(c.cuts, chunk_ctas, chunk_joins, b / pieces);
    if (cta >= 0)
      for (int row0 = (b % pieces) * kChunkJoinRows; row0 < kChunkRows; row0 += pieces * kChunkJoinRows) chunk_join<D>(c, cta, row0);
  } else if ((b -= chunk_joins * pieces) < rows_joins) {
    const int cta = nth_cut(c.a.cuts, rows_ctas, rows_joins, b);
    if (cta >= 0) rows_join<D>(c.a, cta);
  } else {
    attend_report(c.a, b - rows_joins, chunk_ctas > 0 ? c.errors : nullptr, chunk_ctas, c.min_rows);
  }
}

}  // namespace ms

// Attention of new tokens over the paged cache (memstore_attend): the kernel for few query rows per request.
//
// Mathematics: one pass over a row's keys with a running maximum m and sum l: for a group of keys with scores s_j (log2 units)
//   m' = max(m, max_j s_j),  O <- O 2^(m - m') + sum_j 2^(s_j - m') V_j,  l <- l 2^(m - m') + sum_j 2^(s_j - m'),
// and parts of a row's keys join by the same rule: O = sum_i O_i 2^(m_i - m), l = sum_i l_i 2^(m_i - m).  out = O / l.
//
// Bound: HBM (a decode step reads every key and value once and does 4 operations per element and query head).  The 16 rows of
// an m16n8k16 product are (token, query head) pairs that share a K/V head, so a cache row is read once for all heads of its
// group; the legacy matrix instructions are far from their limit here.  Measured (GPU time, 32/8 heads of 128): 16 requests of
// 16,384 tokens 160 us (6.7 TB/s), 100 of 900 67 us (5.5 TB/s), 100 of 500 - 1,300 71 us (5.2 TB/s); an 8-bit cache is held back by the
// instructions that convert it: 16 of 32,768 185 us (5.8 TB/s), 16 of 7,000 - 32,700 116 - 135 us on
// different GPUs (4.8 - 5.6 TB/s).
//
// Work split: a unit is (request, K/V head, 16 rows) x all its tiles of 64 keys (128 where cache rows are at most 128 bytes: an
// 8-bit cache with 64 keys a tile takes 168 us where 128 take 121).  The tiles of all units are numbered one after another and
// every CTA of one resident wave takes an equal share of that line, wherever unit borders fall: ragged lengths balance exactly, and a
// CTA leaves at most two unfinished units (its first and its last), which attend_join_kernel joins. The workspace therefore depends on
// the number of CTAs alone.  Every order of summation follows from the lengths: results are the same on every run.
// Inside a CTA each warp streams its own quarter of a tile's keys through a private ring (cp.async), with running statistics of its
// own: no barrier inside a unit; the four warps join at its end.
#pragma once
#include "blocks.cuh"
#include "inject.cuh"

namespace ms {

constexpr int kAttnRows = 16;      // query rows of a unit
constexpr int kAttnWarps = 4;
constexpr int kAttnThreads = kAttnWarps * 32;
constexpr int kAttnMaxGroup = 1024;
constexpr int kAttnMaxCtasPerSm = 2;
constexpr int32_t kAttnMaxLen = 1 << 30;  // (key numbers stay inside 32 bits)

// Which keys a row sees:
//   kSeeCausal  all at positions up to its own                                                              (memstore_attend)
//   kSeeTree    all in front of the request's new tokens, and of those the ones that the row's bits name    (memstore_attend_tree)
//   kSeeBlocks  those at positions up to its own in the blocks that the token's list for the K/V head names (memstore_attend_blocks).
//               The keys of a unit are then numbered along its list: key v is place v % block_size of listed block v / block_size, and a
//               unit has rows of one token alone, so that all its rows see the same keys and what they do not see is not loaded.
enum { kSeeCausal = 0, kSeeTree = 1, kSeeBlocks = 2 };
constexpr int kTreeMaxWords = 128;  // 32-bit words of a row's bits

// What the border in front of a CTA's share cuts, written by that CTA: the unit to join when the border is the unit's first one.
struct __align__(16) AttnCut {
  int32_t c_last;          // last CTA with a part of the unit, -1: nothing to join
  int32_t rows;            // rows of the unit
  int32_t tok0, sub0;      // token and query head of the group of row 0
  int32_t head0;           // first query head of the K/V head
  int32_t pad[3];
};

struct AttendParams {
  const __nv_bfloat16* q;
  int64_t q_ts, q_hs;
  __nv_bfloat16* out;
  int64_t o_ts, o_hs;
  int32_t n_q, n_kv, group;  // heads, and query heads per K/V head (at most kAttnMaxGroup)
  uint32_t group_magic;      // floor(2^32 / group) + 1, 0 for group == 1
  int32_t n_tokens;
  const int32_t* q_start;
  const int32_t* seq_lens;
  int32_t nreq;
  const int32_t* tables;
  int32_t max_blocks;
  const uint8_t *k_cache, *v_cache;                    // of the layer
  int64_t block_stride, token_stride, head_stride;     // bytes
  int64_t num_blocks;
  int32_t block_size, block_shift;  // block_shift: log2 of the block size, or -1
  float scale_log2;  // scale * log2(e) (* k_scale)
  float v_scale;     // 1 for a bf16 cache
  float* lse;        // [n_tokens][n_q] or nullptr
  int32_t* status;
  int32_t max_rows;  // requests with more rows per K/V head are served by the kernel for chunks
  int32_t min_share; // fewest tiles a CTA takes
  int32_t tile_shift; // log2 of the keys of a tile
  unsigned long long* gate;  // not nullptr: the kernel before this one is the same call's chunk kernel (see gate_open)
  float* part_o;     // [CTAs][2][kAttnRows][head_dim]
  float2* part_ml;   // [CTAs][2][kAttnRows]
  AttnCut* cuts;     // [CTAs]
  const uint32_t* tree;  // kSeeTree: [n_tokens][tree_words], bit j of row i: new token i of a request sees the request's new token j
  int32_t tree_words;    // (0 otherwise)
  const int32_t* lists;  // kSeeBlocks: [n_tokens][n_kv][list_len] blocks of the token's request, counted from its first
  int32_t list_len;
  int32_t token_tiles;   // kSeeBlocks: row tiles of a token
};

// One request as the kernels see it.
struct AttnReq {
  int32_t q0, n;    // rows of q; n = 0: left out
  int32_t len;      // tokens in the cache
  int32_t keys;     // keys the table can name (kSeeBlocks: that a list can)
  int32_t rows;     // n * group
};
template <int SEE = kSeeCausal>
__device__ __forceinline__ AttnReq attn_request(const AttendParams& p, int r) {
  AttnReq a;
  const int32_t q0 = __ldg(p.q_start + r), q1 = __ldg(p.q_start + r + 1);
  a.len = __ldg(p.seq_lens + r);
  bool ok = q0 >= 0 && q1 >= q0 && q1 <= p.n_tokens && a.len >= 0 && a.len <= kAttnMaxLen;
  if (SEE == kSeeTree) ok = ok && q1 - q0 <= 32 * p.tree_words;
  a.q0 = q0;
  a.n = ok ? q1 - q0 : 0;
  if (SEE == kSeeBlocks)  // (a list has no more entries than the request has blocks; list_len * block_size is at most 2^30)
    a.keys = ok ? min(p.list_len, (int32_t)(((int64_t)a.len + p.block_size - 1) / p.block_size)) * p.block_size : 0;
  else
    a.keys = (int32_t)min((int64_t)a.len, (int64_t)p.max_blocks * p.block_size);
  a.rows = a.n * p.group;
  return a;
}
// Tiles of one unit of the request (one at least, so that rows without keys are written too), and of all its units.
__device__ __forceinline__ int attn_tiles(const AttendParams& p, const AttnReq& a) { return max(1, (a.keys + (1 << p.tile_shift) - 1) >> p.tile_shift); }
// row tiles of a K/V head
template <int SEE = kSeeCausal>
__device__ __forceinline__ int attn_row_tiles(const AttendParams& p, const AttnReq& a) {
  return SEE == kSeeBlocks ? a.n * p.token_tiles : (a.rows + kAttnRows - 1) / kAttnRows;
}
template <int SEE = kSeeCausal>
__device__ __forceinline__ int64_t attn_cost(const AttendParams& p, const AttnReq& a) {
  if (a.n == 0 || a.rows > p.max_rows) return 0;
  return (int64_t)attn_row_tiles<SEE>(p, a) * p.n_kv * attn_tiles(p, a);
}

// Which of the 32 keys from k0 on a row of a tree sees, out of those in `there`: the row's bits, with ones for everything in front of the
// new tokens (the first of which is at position pos0).
__device__ __forceinline__ uint32_t tree_see(uint32_t there, int k0, int pos0, const uint32_t* row, int words) {
  const int rel = k0 - pos0;
  if (rel <= -32) return there;
  const int w = rel >> 5;
  const uint32_t lo = w < 0 ? 0xffffffffu : w < words ? __ldg(row + w) : 0u, hi = w + 1 < words ? __ldg(row + w + 1) : 0u;
  return there & __funnelshift_r(lo, hi, rel & 31);
}

// a / b and a % b; 64-bit division only where it is needed
__device__ __forceinline__ int64_t attn_div(int64_t a, int64_t b, int64_t* rem) {
  if (((a | b) >> 32) == 0) {
    const uint32_t q = (uint32_t)a / (uint32_t)b;
    *rem = (uint32_t)a - q * (uint32_t)b;
    return q;
  }
  const int64_t q = a / b;
  *rem = a - q * b;
  return q;
}
// x / group for x < 2^20 (exact: the product's error x * group / 2^32 stays below 1 / group)
__device__ __forceinline__ int group_div(const AttendParams& p, int x) { return p.group_magic ? (int)__umulhi((uint32_t)x, p.group_magic) : x; }

// The line of all tiles of a call.  Up to 128 requests every warp holds the line by itself, request 32 i + l in lane l (no barrier);
// more requests are scanned by the block, a pass per THREADS requests.
constexpr int kLinePerLane = 4;
template <int THREADS>
struct AttnLine {
  int64_t cost[kLinePerLane] = {}, end[kLinePerLane] = {};  // of this lane's requests: tiles, and place behind the last on the line
  int64_t total = 0;

  template <typename F>
  __device__ __forceinline__ void init(int nreq, F cost_of, int64_t* s_warp) {
    if (nreq <= 32 * kLinePerLane) {
      const int lane = threadIdx.x & 31;
#pragma unroll
      for (int i = 0; i < kLinePerLane; ++i) {
        if (32 * i >= nreq) break;  // uniform
        const int r = 32 * i + lane;
        cost[i] = r < nreq ? cost_of(r) : 0;
        int64_t v = cost[i];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
          if (lane >= o) v += u;
        }
        end[i] = total + v;
        total = __shfl_sync(0xffffffffu, end[i], 31);
      }
    } else {
      int64_t sum = 0;
      for (int r = threadIdx.x; r < nreq; r += THREADS) sum += cost_of(r);
      block_scan<THREADS>(sum, s_warp, &total);
    }
  }
  // Request that tile `off` belongs to, and the offset of the request's first tile; -1 when off lies behind the line.  All threads
  // of the block come here with the same off.
  template <typename F>
  __device__ __forceinline__ int locate(int nreq, F cost_of, int64_t off, int64_t* s_warp, int64_t* s_found, int64_t* start) const {
    if (off >= total) return -1;
    if (nreq <= 32 * kLinePerLane) {
      int found = -1;
      int64_t found_at = 0;
#pragma unroll
      for (int i = 0; i < kLinePerLane; ++i)
        if (off < end[i] && off >= end[i] - cost[i]) {
          found = 32 * i + (int)(threadIdx.x & 31);
          found_at = end[i] - cost[i];
        }
      const int src = __ffs(__ballot_sync(0xffffffffu, found >= 0)) - 1;
      *start = __shfl_sync(0xffffffffu, found_at, src);
      return __shfl_sync(0xffffffffu, found, src);
    }
    int64_t before_pass = 0;
    for (int r0 = 0; r0 < nreq; r0 += THREADS) {
      const int r = r0 + threadIdx.x;
      const int64_t c = r < nreq ? cost_of(r) : 0;
      int64_t pass;
      const int64_t end = before_pass + block_scan<THREADS>(c, s_warp, &pass);
      if (off < before_pass + pass) {  // uniform
        if (c > 0 && off >= end - c && off < end) {
          s_found[0] = r;
          s_found[1] = end - c;
        }
        __syncthreads();
        *start = s_found[1];
        return (int)s_found[0];
      }
      before_pass += pass;
    }
    return -1;
  }
};
__device__ __forceinline__ int64_t attn_share(int64_t total, int ctas, int min_share) {
  int64_t rem;
  const int64_t s = attn_div(total + ctas - 1, ctas, &rem);
  return s > min_share ? s : min_share;
}

// block of the table that a key lies in, and its place there
__device__ __forceinline__ int attn_page(const AttendParams& p, int key) { return p.block_shift >= 0 ? key >> p.block_shift : key / p.block_size; }
__device__ __forceinline__ int attn_in_page(const AttendParams& p, int key) {
  return p.block_shift >= 0 ? key & (p.block_size - 1) : key % p.block_size;
}

__device__ __forceinline__ uint32_t attn_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
  // a dead lane's 16 bytes are zero-filled; nothing is read for it
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
template <bool HALF>
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if (HALF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The factor of a row's scores when the row was scaled by the inverse of the power of two with this exponent field; never zero or infinite
// (minus infinity, a masked score, times zero and zero times infinity would be NaN).
__device__ __forceinline__ float attn_scale(float scale_log2, int field) {
  return fminf(fmaxf(scale_log2 * __uint_as_float((uint32_t)field << 23), 1.17549435e-38f), 3.40282347e+38f);
}
// four e4m3 codes as four fp16 (exact), two to a word
__device__ __forceinline__ void e4m3x4_half2(uint32_t u, uint32_t& lo, uint32_t& hi) {
  asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b; }" : "=r"(lo), "=r"(hi) : "r"(u));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The rows kernel of a call starts beside the call's chunk kernel. Everything before the call has completed by then, since every CTA of
// the chunk kernel has waited for it before it lets this grid start - but what those kernels wrote is visible here only through a wait of
// this grid's own, which would last until the chunk kernel ends, or through a chain from a thread that has waited: CTA 0 of the chunk
// kernel stores kGateOpen with release semantics behind its wait and before its trigger, a thread of each CTA here loads it with acquire
// semantics, and the block's barrier passes it on.  The word is in the workspace and is cleared by the call's join kernel.  Where it is
// not found open (it always should be), the CTA waits for the chunk kernel to end, which is always right.
constexpr unsigned long long kGateOpen = 0x6761746520697321ull;
constexpr int kGatePolls = 256;
__device__ __forceinline__ void open_gate(unsigned long long* gate) {
  asm volatile("st.release.gpu.global.u64 [%0], %1;" ::"l"(gate), "l"(kGateOpen) : "memory");
}
__device__ __forceinline__ bool gate_open(const unsigned long long* gate) {
  for (int i = 0; i < kGatePolls; ++i) {
    unsigned long long v;
    asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(gate) : "memory");
    if (v == kGateOpen) return true;
  }
  return false;
}

template <int D, bool FP8>
struct AttnCfg {
  // Keys of a warp in a tile: 32 while rows are at most 128 bytes.  The work around the products (maximum, waits, table look-ups) is per
  // group of keys and the products of two groups of 16 overlap: an 8-bit cache with head_dim 128 reads 5.3 TB/s instead of 3.8.
  static constexpr int kKeys = D * (FP8 ? 1 : 2) <= 128 ? 32 : 16;
  static constexpr int kTileKeys = kAttnWarps * kKeys;
  static constexpr int kGroups = kKeys / 16, kST = 2 * kGroups;       // products of 16 keys, score fragments of 8 keys
  static constexpr int kRowBytes = D * (FP8 ? 1 : 2);
  static constexpr int kChunks = kRowBytes / 16;                      // 16-byte chunks of a cache row
  static constexpr int kTileBytes = kKeys * kRowBytes;                // K or V of a warp's keys of a tile
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kWant = 96 * 1024 / (kAttnWarps * kStageBytes);
  static constexpr int kStages = kWant < 3 ? 3 : kWant > 8 ? 8 : kWant;
  static constexpr int kRingBytes = kAttnWarps * kStages * kStageBytes;
  static constexpr int kMergeBytes = kAttnWarps * kAttnRows * D * 4;  // the warps' O at the end of a unit, over the ring
  static constexpr int kSmemBytes = kRingBytes > kMergeBytes ? kRingBytes : kMergeBytes;
  static constexpr int kCtasPerSm = kSmemBytes > 110 * 1024 ? 1 : 2;
  // fp8: bytes that a thread takes of a key row at once, and the 16-element steps they hold (the order of the elements in a
  // product's inner dimension is free as long as q follows it)
  static constexpr int kKB = D >= 64 ? 16 : D / 4;
  static constexpr int kSPB = kKB / 4;
  // Weights are formed as 2^(score - maximum + kLift) (the statistics keep maximum - kLift).  fp16 weights of at most 1 would
  // use half of the type's range: one below 2^-14 would lose bits and one below 2^-25 would vanish, and the many small weights of a long
  // context behind one large score would be gone while the sum counts them.  Lifted by 14 the largest is 2^14 (65,504 is the limit) and
  // the step of the smallest 2^-38 of it.  bf16 has the range of fp32.
  static constexpr float kLift = FP8 ? 14.f : 0.f;
};

// Byte offset of chunk c of row r in a warp's K or V tile; the chunks are permuted so that the lanes of a matrix load hit
// different banks.
template <int CHUNKS, bool FP8, bool IS_V>
__device__ __forceinline__ int attn_swz(int r, int c) {
  int x;
  if (!FP8)
    x = CHUNKS >= 8 ? (r & 7) : (r / (8 / CHUNKS)) & (CHUNKS - 1);
  else
    x = (IS_V ? ((r >> 1) & 3) << 1 : (r & 1) << 2) & (CHUNKS - 1);
  return (r * CHUNKS + (c ^ x)) * 16;
}

template <int D, bool FP8, int SEE>
__global__ void __launch_bounds__(kAttnThreads, AttnCfg<D, FP8>::kCtasPerSm) attend_rows_kernel(const AttendParams p) {
  using C = AttnCfg<D, FP8>;
  constexpr int kSteps = D / 16, kNT = D / 8;
  constexpr uint32_t kAllKeys = C::kKeys == 32 ? 0xffffffffu : (1u << (C::kKeys & 31)) - 1u;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t s_warp[32], s_found[2];
  __shared__ float s_m[kAttnWarps][kAttnRows], s_l[kAttnWarps][kAttnRows];
  __shared__ uint32_t s_mask[kAttnWarps][C::kStages];
  // (beside the chunk kernel of its call this one need not wait for that kernel to begin, only to end: the two touch different rows, and
  // whatever waits for this grid has then waited for both)
  if (!p.gate || !__syncthreads_and(threadIdx.x != 0 || gate_open(p.gate))) grid_dependency_wait();
  grid_launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;

  auto cost_of = [&](int i) { return attn_cost<SEE>(p, attn_request<SEE>(p, i)); };
  AttnLine<kAttnThreads> line;
  line.init(p.nreq, cost_of, s_warp);
  const int64_t total = line.total;
  const int64_t share = attn_share(total, gridDim.x, p.min_share);
  int64_t off = blockIdx.x * share;
  const int64_t off_end = min(total, off + share);
  if (tid == 0) p.cuts[blockIdx.x].c_last = -1;  // (until the first unit says otherwise)
  int64_t req_start = 0;
  int r = off < off_end ? line.locate(p.nreq, cost_of, off, s_warp, s_found, &req_start) : -1;
  AttnReq rq{};
  if (r >= 0) rq = attn_request<SEE>(p, r);
  bool first = true;

  uint8_t* ring = smem + warp * (C::kStages * C::kStageBytes);
  const uint32_t ring_u = attn_smem(ring);

  while (r >= 0 && off < off_end) {
    // ---- the unit that tile `off` belongs to
    const int tiles = attn_tiles(p, rq), n_rt = attn_row_tiles<SEE>(p, rq);
    int64_t rem;
    const int64_t u = attn_div(off - req_start, tiles, &rem);  // row tile fastest, so that the row tiles of a K/V head follow one another
    const int t0 = (int)rem;
    const int kvh = (int)attn_div(u, n_rt, &rem), rt = (int)rem;
    const int t1 = (int)min((int64_t)tiles, t0 + (off_end - off));
    const bool whole = t0 == 0 && t1 == tiles;
    int rows, tok0, sub0;  // rows, and new token and query head of the group of row 0
    if constexpr (SEE == kSeeBlocks) {
      tok0 = rt / p.token_tiles;
      sub0 = (rt - tok0 * p.token_tiles) * kAttnRows;
      rows = min(kAttnRows, p.group - sub0);
    } else {
      const int row0 = rt * kAttnRows;
      rows = min(kAttnRows, rq.rows - row0);
      tok0 = row0 / p.group;
      sub0 = row0 - tok0 * p.group;
    }
    if (first && tid == 0 && t0 != 0 && share >= t0) {
      AttnCut cut{};
      cut.c_last = (int)attn_div(off - t0 + tiles - 1, share, &rem);
      cut.rows = rows;
      cut.tok0 = rq.q0 + tok0;
      cut.sub0 = sub0;
      cut.head0 = kvh * p.group;
      p.cuts[blockIdx.x] = cut;
    }
    first = false;
    const int pos0 = rq.len - rq.n;  // position of the request's first new token
    const int last_pos = pos0 + tok0 + group_div(p, sub0 + rows - 1);
    // keys that any row of the unit may see
    const int key_end = SEE == kSeeBlocks ? (last_pos < 0 ? 0 : rq.keys) : SEE == kSeeTree ? rq.keys : min(rq.keys, last_pos + 1);
    const int n_it = min(t1, (key_end + C::kTileKeys - 1) / C::kTileKeys) - t0;  // <= 0: nothing to read
    // last key of this thread's two rows (rows behind the unit's last follow the last one)
    const int dt0 = group_div(p, sub0 + min(g, rows - 1)), dt1 = group_div(p, sub0 + min(g + 8, rows - 1));
    const int lim0 = pos0 + tok0 + dt0, lim1 = pos0 + tok0 + dt1;
    // last key that every row sees (of those that are loaded)
    const int lim_min = SEE == kSeeBlocks ? 0x7fffffff - C::kTileKeys : SEE == kSeeTree ? pos0 - 1 : pos0 + tok0;
    const uint32_t *tree0 = nullptr, *tree1 = nullptr;  // this thread's rows' bits
    if constexpr (SEE == kSeeTree) {
      tree0 = p.tree + (int64_t)(rq.q0 + tok0 + dt0) * p.tree_words;
      tree1 = p.tree + (int64_t)(rq.q0 + tok0 + dt1) * p.tree_words;
    }

    const int32_t* table = p.tables + (int64_t)r * p.max_blocks;
    const uint8_t* kh = p.k_cache + kvh * p.head_stride;
    const uint8_t* vh = p.v_cache + kvh * p.head_stride;
    // lane's key of iteration i, and its table entry (fetched one iteration before it is needed)
    auto key_of = [&](int i) { return (t0 + i) * C::kTileKeys + warp * C::kKeys + (lane & (C::kKeys - 1)); };
    const int32_t* list = nullptr;
    int last_block = -1;  // kSeeBlocks: of those that hold keys the token may see and that the table has
    if constexpr (SEE == kSeeBlocks) {
      list = p.lists + ((int64_t)(rq.q0 + tok0) * p.n_kv + kvh) * p.list_len;
      if (last_pos >= 0) last_block = min(attn_page(p, last_pos), p.max_blocks - 1);
    }
    auto listed = [&](int i) {  // kSeeBlocks: the entry of the list
      const int key = key_of(i);
      return i < n_it && key < key_end ? __ldg(list + attn_page(p, key)) : -1;
    };
    auto entry_of = [&](int i, int32_t block) {
      const int key = key_of(i);
      if constexpr (SEE == kSeeBlocks) {
        const bool there = block >= 0 && block <= last_block && block * p.block_size + attn_in_page(p, key) <= last_pos;
        return there ? __ldg(table + block) : -1;
      }
      return i < n_it && key < key_end ? __ldg(table + attn_page(p, key)) : -1;
    };
    auto issue = [&](int i, int32_t blk) {
      if (i < n_it) {
        const int key = key_of(i);
        const bool live = blk >= 0 && blk < p.num_blocks;
        const int64_t at = live ? blk * p.block_stride + attn_in_page(p, key) * p.token_stride : 0;
        const uint32_t mask = __ballot_sync(0xffffffffu, live) & kAllKeys;
        const int st = i % C::kStages;
        if (lane == 0) s_mask[warp][st] = mask;
        const uint32_t dst = ring_u + st * C::kStageBytes;
        constexpr int kPer = C::kKeys * C::kChunks / 32 > 0 ? C::kKeys * C::kChunks / 32 : 1;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const int idx = j * 32 + lane, row = (idx / C::kChunks) & (C::kKeys - 1), ch = idx % C::kChunks;
          const int64_t ro = __shfl_sync(0xffffffffu, at, row);
          const bool ok = (mask >> row) & 1u;
          if (C::kKeys * C::kChunks >= 32 || idx < C::kKeys * C::kChunks) {
            cp_async16(dst + attn_swz<C::kChunks, FP8, false>(row, ch), kh + ro + ch * 16, ok);
            cp_async16(dst + C::kTileBytes + attn_swz<C::kChunks, FP8, true>(row, ch), vh + ro + ch * 16, ok);
          }
        }
      }
      cp_async_commit();
    };

    // kSeeBlocks looks up twice, list and table: each look-up has the time of a tile
    int32_t nxt_block = -1;
    if constexpr (SEE == kSeeBlocks) nxt_block = listed(0);
    int32_t nxt = entry_of(0, nxt_block);
    if constexpr (SEE == kSeeBlocks) nxt_block = listed(1);
#pragma unroll 1
    for (int i = 0; i < C::kStages - 1; ++i) {
      const int32_t blk = nxt;
      nxt = entry_of(i + 1, nxt_block);
      if constexpr (SEE == kSeeBlocks) nxt_block = listed(i + 2);
      issue(i, blk);
    }
    // ---- queries: A fragments of the 16 rows, zero behind the last
    uint32_t qf[kSteps][4];
    float sc0 = p.scale_log2, sc1 = p.scale_log2;
    {
      const int ta = group_div(p, sub0 + g), tb = group_div(p, sub0 + g + 8);
      const __nv_bfloat16* qa = p.q + (int64_t)(rq.q0 + tok0 + ta) * p.q_ts + (int64_t)(kvh * p.group + sub0 + g - ta * p.group) * p.q_hs;
      const __nv_bfloat16* qb = p.q + (int64_t)(rq.q0 + tok0 + tb) * p.q_ts + (int64_t)(kvh * p.group + sub0 + g + 8 - tb * p.group) * p.q_hs;
      const bool la = g < rows, lb = g + 8 < rows;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const int d0 = FP8 ? (k / C::kSPB) * 64 + C::kKB * t4 + 4 * (k % C::kSPB) : 16 * k + 2 * t4;
        const int d1 = FP8 ? d0 + 2 : d0 + 8;
        qf[k][0] = la ? *reinterpret_cast<const uint32_t*>(qa + d0) : 0u;
        qf[k][1] = lb ? *reinterpret_cast<const uint32_t*>(qb + d0) : 0u;
        qf[k][2] = la ? *reinterpret_cast<const uint32_t*>(qa + d1) : 0u;
        qf[k][3] = lb ? *reinterpret_cast<const uint32_t*>(qb + d1) : 0u;
      }
      if (FP8) {
        // e4m3 is exact in fp16, bf16 is not: each row of q is scaled by the power of two that brings its largest element to
        // [2^14, 2^15), which keeps every element above 2^-28 of it exact; the scores are scaled back in fp32
        float ma = 0.f, mb = 0.f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          ma = fmaxf(ma, fmaxf(fmaxf(fabsf(bf16lo(qf[k][0])), fabsf(bf16hi(qf[k][0]))), fmaxf(fabsf(bf16lo(qf[k][2])), fabsf(bf16hi(qf[k][2])))));
          mb = fmaxf(mb, fmaxf(fmaxf(fabsf(bf16lo(qf[k][1])), fabsf(bf16hi(qf[k][1]))), fmaxf(fabsf(bf16lo(qf[k][3])), fabsf(bf16hi(qf[k][3])))));
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
          ma = fmaxf(ma, __shfl_xor_sync(0xffffffffu, ma, o));
          mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, o));
        }
        // exponent field of the maximum -> the fields of the power of two, 127 + 14 - (field - 127), and of its inverse
        const int ea = min(max(268 - (int)(__float_as_uint(ma) >> 23), 13), 227), eb = min(max(268 - (int)(__float_as_uint(mb) >> 23), 13), 227);
        const float fa = __uint_as_float((uint32_t)ea << 23), fb = __uint_as_float((uint32_t)eb << 23);
        sc0 = attn_scale(sc0, 254 - ea);
        sc1 = attn_scale(sc1, 254 - eb);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          qf[k][0] = pack_half(bf16lo(qf[k][0]) * fa, bf16hi(qf[k][0]) * fa);
          qf[k][2] = pack_half(bf16lo(qf[k][2]) * fa, bf16hi(qf[k][2]) * fa);
          qf[k][1] = pack_half(bf16lo(qf[k][1]) * fb, bf16hi(qf[k][1]) * fb);
          qf[k][3] = pack_half(bf16lo(qf[k][3]) * fb, bf16hi(qf[k][3]) * fb);
        }
      }
    }

    float o[kNT][4];
#pragma unroll
    for (int n = 0; n < kNT; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;

#pragma unroll 1
    for (int i = 0; i < n_it; ++i) {
      cp_async_wait<C::kStages - 2>();
      __syncwarp();
      {
        const int32_t blk = nxt;
        nxt = entry_of(i + C::kStages, nxt_block);
        if constexpr (SEE == kSeeBlocks) nxt_block = listed(i + C::kStages + 1);
        issue(i + C::kStages - 1, blk);
      }
      const int st = i % C::kStages;
      const int k0 = (t0 + i) * C::kTileKeys + warp * C::kKeys;
      const uint32_t mask = s_mask[warp][st];
      if (k0 >= key_end) continue;  // (uniform in the warp)
      const uint32_t kt = ring_u + st * C::kStageBytes, vt = kt + C::kTileBytes;

      // ---- scores of the warp's keys
      float s[C::kST][4];
#pragma unroll
      for (int nt = 0; nt < C::kST; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
      if constexpr (!FP8) {
        const int kr = (lane & 7) + ((lane >> 4) << 3), kc = (lane >> 3) & 1;
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
          for (int gr = 0; gr < C::kGroups; ++gr) {
            uint32_t b[4];
            ldsm4(kt + attn_swz<C::kChunks, false, false>(gr * 16 + kr, 2 * k + kc), b);
            mma16816<false>(s[2 * gr], qf[k], b[0], b[1]);
            mma16816<false>(s[2 * gr + 1], qf[k], b[2], b[3]);
          }
      } else {
        const uint8_t* kp = ring + st * C::kStageBytes;
#pragma unroll
        for (int kb = 0; kb < kSteps / C::kSPB; ++kb)
#pragma unroll
          for (int nt = 0; nt < C::kST; ++nt) {
            const int row = nt * 8 + g, byte = kb * 64 + C::kKB * t4;
            const uint8_t* src = kp + attn_swz<C::kChunks, true, false>(row, byte >> 4) + (byte & 15);
            uint32_t w[4];
            if constexpr (C::kKB == 16) {
              const uint4 x = *reinterpret_cast<const uint4*>(src);
              w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
            } else if constexpr (C::kKB == 8) {
              const uint2 x = *reinterpret_cast<const uint2*>(src);
              w[0] = x.x, w[1] = x.y;
            } else {
              w[0] = *reinterpret_cast<const uint32_t*>(src);
            }
#pragma unroll
            for (int q = 0; q < C::kSPB; ++q) {
              uint32_t b0, b1;
              e4m3x4_half2(w[q], b0, b1);
              mma16816<true>(s[nt], qf[kb * C::kSPB + q], b0, b1);
            }
          }
      }
      // ---- mask, running maximum and sum
      const bool causal = k0 + C::kKeys - 1 > lim_min;  // some row ends inside or before these keys, or may leave some of them out
      uint32_t tsee0 = mask, tsee1 = mask;
      if (SEE == kSeeTree && causal) {
        tsee0 = tree_see(mask, k0, pos0, tree0, p.tree_words);
        tsee1 = tree_see(mask, k0, pos0, tree1, p.tree_words);
      }
      if (causal || mask != kAllKeys) {
#pragma unroll
        for (int nt = 0; nt < C::kST; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int c = nt * 8 + 2 * t4 + e;
            if constexpr (SEE == kSeeTree) {
              if (!((tsee0 >> c) & 1u)) s[nt][e] = -INFINITY;
              if (!((tsee1 >> c) & 1u)) s[nt][2 + e] = -INFINITY;
            } else {
              const bool there = (mask >> c) & 1u;
              if (!there || (SEE == kSeeCausal && k0 + c > lim0)) s[nt][e] = -INFINITY;
              if (!there || (SEE == kSeeCausal && k0 + c > lim1)) s[nt][2 + e] = -INFINITY;
            }
          }
      }
      float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
      for (int nt = 0; nt < C::kST; ++nt) {
        x0 = fmaxf(x0, fmaxf(s[nt][0], s[nt][1]));
        x1 = fmaxf(x1, fmaxf(s[nt][2], s[nt][3]));
      }
      x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1));
      x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
      x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2));
      x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
      const float n0 = fmaxf(m0, fmaf(x0, sc0, -C::kLift)), n1 = fmaxf(m1, fmaf(x1, sc1, -C::kLift));
      if (__any_sync(0xffffffffu, n0 != m0 || n1 != m1)) {
        // (a maximum of minus infinity: nothing has been summed yet, any finite stand-in gives weights of zero)
        const float a0 = n0 == -INFINITY ? 1.f : ex2(m0 - n0), a1 = n1 == -INFINITY ? 1.f : ex2(m1 - n1);
        l0 *= a0;
        l1 *= a1;
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
          o[n][0] *= a0;
          o[n][1] *= a0;
          o[n][2] *= a1;
          o[n][3] *= a1;
        }
        m0 = n0;
        m1 = n1;
      }
      const float b0 = m0 == -INFINITY ? 0.f : m0, b1 = m1 == -INFINITY ? 0.f : m1;
#pragma unroll
      for (int nt = 0; nt < C::kST; ++nt) {  // the scores become weights
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          s[nt][e] = ex2(fmaf(s[nt][e], sc0, -b0));
          s[nt][2 + e] = ex2(fmaf(s[nt][2 + e], sc1, -b1));
        }
        l0 += s[nt][0] + s[nt][1];
        l1 += s[nt][2] + s[nt][3];
      }

      // ---- a value that is not finite at a key that some row must not see would reach that row as 0 * inf: such keys (only a chunk's
      // last ones can be) are summed one by one
      bool by_key = false;
      if (SEE != kSeeBlocks && causal) {
        const uint4* vp = reinterpret_cast<const uint4*>(ring + st * C::kStageBytes + C::kTileBytes);
        bool bad = false;
        for (int j = lane; j < C::kTileBytes / 16; j += 32) {
          const uint4 x = vp[j];
          const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (FP8)
              bad = bad || __vcmpeq4(y[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0u;
            else
              bad = bad || (y[e] & 0x7f80u) == 0x7f80u || (y[e] & 0x7f800000u) == 0x7f800000u;
          }
        }
        by_key = __any_sync(0xffffffffu, bad);
      }
      if (by_key) {
        const uint8_t* vp = ring + st * C::kStageBytes + C::kTileBytes;
#pragma unroll
        for (int nt = 0; nt < C::kST; ++nt)
#pragma unroll 1
          for (int c8 = 0; c8 < 8; ++c8) {
            const int c = nt * 8 + c8, from = (lane & 28) | (c8 >> 1);
            const float e0 = __shfl_sync(0xffffffffu, s[nt][0], from), e1 = __shfl_sync(0xffffffffu, s[nt][1], from);
            const float e2 = __shfl_sync(0xffffffffu, s[nt][2], from), e3 = __shfl_sync(0xffffffffu, s[nt][3], from);
            const float w0 = c & 1 ? e1 : e0, w1 = c & 1 ? e3 : e2;
            const bool there = (mask >> c) & 1u;
            const bool see0 = SEE == kSeeTree ? (tsee0 >> c) & 1u : there && k0 + c <= lim0, see1 = SEE == kSeeTree ? (tsee1 >> c) & 1u : there && k0 + c <= lim1;
#pragma unroll
            for (int n = 0; n < kNT; ++n) {
              float v0, v1;
              if constexpr (!FP8) {
                const int d = 8 * n + 2 * t4;
                const uint32_t x = *reinterpret_cast<const uint32_t*>(vp + attn_swz<C::kChunks, false, true>(c, d >> 3) + (d & 7) * 2);
                v0 = bf16lo(x), v1 = bf16hi(x);
              } else {
                constexpr int kVB = D >= 32 ? 4 : D / 8;
                const int d = (n / kVB) * (8 * kVB) + 2 * t4 * kVB + n % kVB;
                const uint32_t x0b = vp[attn_swz<C::kChunks, true, true>(c, d >> 4) + (d & 15)];
                const uint32_t x1b = vp[attn_swz<C::kChunks, true, true>(c, (d + kVB) >> 4) + ((d + kVB) & 15)];
                uint32_t h, unused;
                e4m3x4_half2(x0b | (x1b << 8), h, unused);
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
                v0 = f.x, v1 = f.y;
              }
              if (see0) o[n][0] = fmaf(w0, v0, o[n][0]), o[n][1] = fmaf(w0, v1, o[n][1]);
              if (see1) o[n][2] = fmaf(w1, v0, o[n][2]), o[n][3] = fmaf(w1, v1, o[n][3]);
            }
          }
        continue;
      }

      // ---- O += P V.  P is rounded to the type of the product (half a step is 2^-9 of a bf16 weight, 2^-12 of an fp16 one): the matrix
      // instructions take 16-bit operands, and V has no more bits than that itself.  l holds the unrounded weights.
#pragma unroll
      for (int gr = 0; gr < C::kGroups; ++gr) {
        const float* wa = s[2 * gr];
        const float* wb = s[2 * gr + 1];
        if constexpr (!FP8) {
          const uint32_t pa[4] = {pack_bf16(wa[0], wa[1]), pack_bf16(wa[2], wa[3]), pack_bf16(wb[0], wb[1]), pack_bf16(wb[2], wb[3])};
          const int vr = gr * 16 + (lane & 15), vc = lane >> 4;
#pragma unroll
          for (int n = 0; n < kNT; n += 2) {
            uint32_t b[4];
            ldsm4t(vt + attn_swz<C::kChunks, false, true>(vr, n + vc), b);
            mma16816<false>(o[n], pa, b[0], b[1]);
            mma16816<false>(o[n + 1], pa, b[2], b[3]);
          }
        } else {
          const uint32_t pa[4] = {pack_half(wa[0], wa[1]), pack_half(wa[2], wa[3]), pack_half(wb[0], wb[1]), pack_half(wb[2], wb[3])};
          const uint8_t* vp = ring + st * C::kStageBytes + C::kTileBytes;
          // a thread takes kVB neighbouring elements of four key rows: column c of product n holds element (n / kVB) * 8 kVB + c kVB + n % kVB
          constexpr int kVB = D >= 32 ? 4 : D / 8;
#pragma unroll
          for (int jj = 0; jj < kNT / kVB; ++jj) {
            const int d = jj * 8 * kVB + g * kVB;
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int row = gr * 16 + 2 * t4 + (e & 1) + (e >> 1) * 8;
              const uint8_t* src = vp + attn_swz<C::kChunks, true, true>(row, d >> 4) + (d & 15);
              if constexpr (kVB == 4) x[e] = *reinterpret_cast<const uint32_t*>(src);
              else x[e] = *reinterpret_cast<const uint16_t*>(src);
            }
#pragma unroll
            for (int h = 0; h < kVB / 2; ++h) {  // bytes 2h, 2h + 1 of the rows, paired by key
              const uint32_t lo = __byte_perm(x[0], x[1], h ? 0x7362 : 0x5140), hi = __byte_perm(x[2], x[3], h ? 0x7362 : 0x5140);
              uint32_t l0h, l1h, h0h, h1h;
              e4m3x4_half2(lo, l0h, l1h);
              e4m3x4_half2(hi, h0h, h1h);
              mma16816<true>(o[jj * kVB + 2 * h], pa, l0h, h0h);
              mma16816<true>(o[jj * kVB + 2 * h + 1], pa, l1h, h1h);
            }
          }
        }
      }
    }
    cp_async_wait<0>();

    // ---- join the four warps
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
    l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    if (t4 == 0) {
      s_m[warp][g] = m0;
      s_m[warp][g + 8] = m1;
      s_l[warp][g] = l0;
      s_l[warp][g + 8] = l1;
    }
    __syncthreads();  // nobody reads the ring any more
    float* s_o = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      int d0, d1;
      if constexpr (!FP8) {
        d0 = 8 * n + 2 * t4;
        d1 = d0 + 1;
      } else {
        constexpr int kVB = D >= 32 ? 4 : D / 8;
        d0 = (n / kVB) * (8 * kVB) + 2 * t4 * kVB + n % kVB;
        d1 = d0 + kVB;
      }
      float* a = s_o + (warp * kAttnRows + g) * D;
      float* b = a + 8 * D;
      a[d0] = o[n][0];
      a[d1] = o[n][1];
      b[d0] = o[n][2];
      b[d1] = o[n][3];
    }
    __syncthreads();
    const int slot = t0 == 0 ? 1 : 0;
    for (int e = tid; e < rows * (D / 2); e += kAttnThreads) {
      const int row = e / (D / 2), d = 2 * (e % (D / 2));
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kAttnWarps; ++w) m = fmaxf(m, s_m[w][row]);
      float l = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
      for (int w = 0; w < kAttnWarps; ++w) {
        const float mw = s_m[w][row];
        const float f = mw == -INFINITY ? 1.f : ex2(mw - m);  // (sums without a maximum: zeros, or NaN that has to stay)
        l = fmaf(f, s_l[w][row], l);
        const float2 x = *reinterpret_cast<const float2*>(s_o + (w * kAttnRows + row) * D + d);
        y0 = fmaf(f, x.x, y0);
        y1 = fmaf(f, x.y, y1);
      }
      if (whole) {
        const int dt = group_div(p, sub0 + row), tok = rq.q0 + tok0 + dt, head = kvh * p.group + sub0 + row - dt * p.group;
        const float inv = l == 0.f ? 0.f : p.v_scale / l;
        *reinterpret_cast<uint32_t*>(p.out + tok * p.o_ts + head * p.o_hs + d) = pack_bf16(y0 * inv, y1 * inv);
        if (p.lse && d == 0) p.lse[(int64_t)tok * p.n_q + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      } else {
        const int64_t at = ((int64_t)blockIdx.x * 2 + slot) * kAttnRows + row;
        *reinterpret_cast<float2*>(p.part_o + at * D + d) = make_float2(y0, y1);
        if (d == 0) p.part_ml[at] = make_float2(m, l);
      }
    }
    __syncthreads();  // the ring is filled again

    // ---- next
    off += t1 - t0;
    if (off < off_end && off - req_start >= attn_cost<SEE>(p, rq)) {
      req_start = off;
      do {
        if (++r >= p.nreq) r = -1;  // (cannot be: off lies before the end of the line)
        else rq = attn_request<SEE>(p, r);
      } while (r >= 0 && attn_cost<SEE>(p, rq) == 0);
    }
  }
  if (p.gate) grid_dependency_wait();
}

// Joins the parts of the unit that the border in front of CTA b's share cuts, if it is the unit's first border.
constexpr int kCombineThreads = 512;
constexpr int kJoinBatch = 5;  // parts whose loads fly together (as many as two blocks on an SM have registers for)
// CTA whose border makes the n-th cut, or -1; by the whole block.
__device__ __forceinline__ int nth_cut(const AttnCut* cuts, int ctas, int cuts_at_most, int n) {
  if (cuts_at_most >= ctas - 1) return cuts[n + 1].c_last >= 0 ? n + 1 : -1;  // a block per border
  __shared__ int s_count[kCombineThreads / 32], s_cta;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) s_cta = -1;
  int before = 0;
  for (int c0 = 0; c0 < ctas; c0 += kCombineThreads) {
    const int cta = c0 + threadIdx.x;
    const bool cut = cta < ctas && cuts[cta].c_last >= 0;
    const unsigned m = __ballot_sync(0xffffffffu, cut);
    if (lane == 0) s_count[warp] = __popc(m);
    __syncthreads();
    int at = before;
#pragma unroll
    for (int w = 0; w < kCombineThreads / 32; ++w) {
      if (w < warp) at += s_count[w];
      before += s_count[w];
    }
    if (cut && at + __popc(m & ((1u << lane) - 1u)) == n) s_cta = cta;
    __syncthreads();
  }
  return s_cta;
}

// Four elements of a row, summed over parts.
struct JoinSum {
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void add(const float2* ml, const float4* x, int n) {  // the first min(n, kJoinBatch) parts
    float top = m;
#pragma unroll
    for (int i = 0; i < kJoinBatch; ++i)
      if (i < n) top = fmaxf(top, ml[i].x);
    const float f = m == -INFINITY ? 1.f : ex2(m - top);  // (sums without a maximum: zeros, or NaN that has to stay)
    l *= f;
    o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
#pragma unroll
    for (int i = 0; i < kJoinBatch; ++i)
      if (i < n) {
        const float w = ml[i].x == -INFINITY ? 1.f : ex2(ml[i].x - top);
        l = fmaf(ml[i].y, w, l);
        o = make_float4(fmaf(x[i].x, w, o.x), fmaf(x[i].y, w, o.y), fmaf(x[i].z, w, o.z), fmaf(x[i].w, w, o.w));
      }
    m = top;
  }
  __device__ __forceinline__ void write(const AttendParams& p, int tok, int head, int d) const {
    const float inv = l == 0.f ? 0.f : p.v_scale / l;
    *reinterpret_cast<uint2*>(p.out + tok * p.o_ts + head * p.o_hs + d) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (p.lse && d == 0) p.lse[(int64_t)tok * p.n_q + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  }
};
template <int D>
__device__ __forceinline__ void rows_join(const AttendParams& p, int b) {
  const AttnCut cut = p.cuts[b];
  if (cut.c_last < 0) return;
  const int c_last = cut.c_last;
  for (int e = threadIdx.x; e < cut.rows * (D / 4); e += kCombineThreads) {
    const int row = e / (D / 4), d = 4 * (e % (D / 4));
    JoinSum sum;
    for (int c0 = b - 1; c0 <= c_last; c0 += kJoinBatch) {
      float2 ml[kJoinBatch];
      float4 x[kJoinBatch];
#pragma unroll
      for (int i = 0; i < kJoinBatch; ++i) {  // (the loads of several parts fly together)
        const int c = c0 + i;
        if (c > c_last) break;  // uniform
        const int64_t at = ((int64_t)c * 2 + (c == b - 1 ? 1 : 0)) * kAttnRows + row;
        ml[i] = p.part_ml[at];
        x[i] = *reinterpret_cast<const float4*>(p.part_o + at * D + d);
      }
      sum.add(ml, x, c_last - c0 + 1);
    }
    const int dt = group_div(p, cut.sub0 + row);
    sum.write(p, cut.tok0 + dt, cut.head0 + cut.sub0 + row - dt * p.group, d);
  }
}

// The status words of sixteen requests, a warp each; errors: time-outs of the chunk kernel's CTAs (it serves requests of more than
// min_rows rows), or nullptr.
__device__ __forceinline__ void attend_report(const AttendParams& p, int block, const int32_t* errors, int n_errors, int min_rows) {
  const int r = block * (kCombineThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (!p.status || r >= p.nreq) return;
  const int32_t q0 = p.q_start[r], q1 = p.q_start[r + 1], len = p.seq_lens[r];
  int st = 0;
  if (q0 < 0 || q1 < q0 || q1 > p.n_tokens || len < 0 || len > kAttnMaxLen || (p.tree_words > 0 && q1 - q0 > 32 * p.tree_words)) {
    st = kReqBadLength;
  } else {
    const int64_t blocks = ((int64_t)len + p.block_size - 1) / p.block_size;
    if (blocks > p.max_blocks) st = kReqTableShort;
    const int n = (int)min(blocks, (int64_t)p.max_blocks);
    bool bad = false;
    for (int b = lane; b < n; b += 32) {
      const int32_t x = p.tables[(int64_t)r * p.max_blocks + b];
      bad = bad || x < 0 || x >= p.num_blocks;
    }
    if (__any_sync(0xffffffffu, bad)) st |= kReqBadBlock;
    if (errors && (q1 - q0) * p.group > min_rows) {
      bool late = false;
      for (int i = lane; i < n_errors; i += 32) late = late || errors[i] != 0;
      if (__any_sync(0xffffffffu, late)) st |= kReqTimeout;
    }
  }
  if (lane == 0) p.status[r] = st;
}

}  // namespace ms

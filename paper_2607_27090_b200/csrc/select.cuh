// Summaries of cache blocks (memstore_summarize_blocks) and the choice of the blocks that a token reads (memstore_select_blocks).
//
// The summary of a block and K/V head is the smallest and the largest value of each coordinate over the block's keys.  For a query q the sum over
// coordinates of max(q lo, q hi) is no less than q . k for any key k of the block; its sum over the query heads of a group is
//   score = sum_d P_d hi_d + N_d lo_d,   P = sum over the group of max(q, 0),  N = sum over the group of min(q, 0),
// so a group costs as much as one head: a product of 2 head_dim numbers per block.
#pragma once
#include <cooperative_groups.h>

#include "attend.cuh"

namespace ms {

// ---- summaries
struct SummaryParams {
  const int32_t* q_start;   // nullptr: every block of a request
  int32_t n_tokens;
  const int32_t* seq_lens;
  int32_t nreq;
  const int32_t* tables;
  int32_t max_blocks, block_size;
  int64_t num_blocks;
  const uint8_t* k_cache;                           // of the layer
  int64_t block_stride, token_stride, head_stride;  // bytes
  int32_t n_kv;
  uint4* summaries;         // [num_blocks][n_kv][2][head_dim] bf16
};

// The blocks of request r that hold its new tokens: [first, end).
struct SummarySpan {
  int32_t first, end, len;
};
__device__ __forceinline__ SummarySpan summary_span(const SummaryParams& p, int r) {
  const int32_t len = __ldg(p.seq_lens + r);
  int32_t start = 0;
  bool ok = len >= 0 && len <= kAttnMaxLen;
  if (p.q_start) {
    const int32_t q0 = __ldg(p.q_start + r), q1 = __ldg(p.q_start + r + 1);
    ok = ok && q0 >= 0 && q1 >= q0 && q1 <= p.n_tokens;
    start = ok ? max(0, len - (q1 - q0)) : 0;
    ok = ok && q1 > q0;
  }
  SummarySpan s;
  s.len = len;
  s.first = min(start / p.block_size, p.max_blocks);
  s.end = ok ? max(s.first, (int32_t)min(((int64_t)len + p.block_size - 1) / p.block_size, (int64_t)p.max_blocks)) : s.first;
  return s;
}

// (the forms that return NaN where an operand is one: a key that is not a number must not vanish from its block's summary)
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b, bool half) {
  uint32_t r;
  if (half)
    asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b, bool half) {
  uint32_t r;
  if (half)
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// e4m3 has few enough bits that fp16 and bf16 hold its values exactly
__device__ __forceinline__ uint32_t half2_to_bf16(uint32_t h) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return pack_bf16(f.x, f.y);
}

constexpr int kSummaryThreads = 256;
constexpr int kSummaryCtasPerSm = 6;
constexpr int kSummaryFlight = 4;  // loads of a thread that fly together

// A warp per (block, K/V head); heads of a block follow one another, so that a CTA reads whole rows of a token-major cache.  The items of
// all requests form a line of which every CTA takes an equal share.  Bound: HBM where there are many blocks (each key is read once), else latency.
template <int D, bool FP8>
__global__ void __launch_bounds__(kSummaryThreads) summarize_kernel(const SummaryParams p) {
  constexpr int kLanes = D * (FP8 ? 1 : 2) / 16;  // lanes of a key's row
  constexpr int kRows = 32 / kLanes;              // rows of a load
  constexpr int kWords = FP8 ? 8 : 4;
  __shared__ int64_t s_warp[32], s_found[2];
  grid_dependency_wait();
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto cost_of = [&](int i) {
    const SummarySpan s = summary_span(p, i);
    return (int64_t)(s.end - s.first) * p.n_kv;
  };
  AttnLine<kSummaryThreads> line;
  line.init(p.nreq, cost_of, s_warp);
  const int64_t share = attn_share(line.total, gridDim.x, kSummaryThreads / 32);
  const int64_t off = blockIdx.x * share, off_end = min(line.total, off + share);
  if (off >= off_end) return;
  int64_t req_start;
  int r = line.locate(p.nreq, cost_of, off, s_warp, s_found, &req_start);
  if (r < 0) return;
  SummarySpan span = summary_span(p, r);
  int64_t req_end = req_start + (int64_t)(span.end - span.first) * p.n_kv;
  for (int64_t item = off + warp; item < off_end; item += kSummaryThreads / 32) {
    while (item >= req_end && r + 1 < p.nreq) {
      // the next request with blocks (requests without are passed over 32 at a time)
      unsigned some = 0u;
      for (++r; r < p.nreq; r += 32) {
        some = __ballot_sync(0xffffffffu, r + lane < p.nreq && cost_of(r + lane) > 0);
        if (some) break;
      }
      if (!some) return;  // (cannot be: the item lies before the end of the line)
      r += __ffs(some) - 1;
      span = summary_span(p, r);
      req_start = req_end;
      req_end += (int64_t)(span.end - span.first) * p.n_kv;
    }
    int64_t rem;
    const int b = span.first + (int)attn_div(item - req_start, p.n_kv, &rem), head = (int)rem;
    const int32_t blk = __ldg(p.tables + (int64_t)r * p.max_blocks + b);
    if (blk < 0 || blk >= p.num_blocks) continue;
    const int last = min(p.block_size, span.len - b * p.block_size) - 1;  // the block's last key
    const uint8_t* base = p.k_cache + blk * p.block_stride + head * p.head_stride + (lane % kLanes) * 16;
    uint32_t lo[kWords], hi[kWords];
    for (int k0 = 0; k0 <= last; k0 += kRows * kSummaryFlight) {
      uint4 x[kSummaryFlight];
#pragma unroll
      for (int i = 0; i < kSummaryFlight; ++i)  // (behind the last key the last key again, which changes nothing)
        x[i] = ld_stream(reinterpret_cast<const uint4*>(base + (int64_t)min(last, k0 + i * kRows + lane / kLanes) * p.token_stride));
#pragma unroll
      for (int i = 0; i < kSummaryFlight; ++i) {
        uint32_t y[kWords];
        if constexpr (FP8) {
          e4m3x4_half2(x[i].x, y[0], y[1]);
          e4m3x4_half2(x[i].y, y[2], y[3]);
          e4m3x4_half2(x[i].z, y[4], y[5]);
          e4m3x4_half2(x[i].w, y[6], y[7]);
        } else {
          y[0] = x[i].x, y[1] = x[i].y, y[2] = x[i].z, y[3] = x[i].w;
        }
#pragma unroll
        for (int e = 0; e < kWords; ++e) {
          lo[e] = k0 == 0 && i == 0 ? y[e] : min_pair(lo[e], y[e], FP8);
          hi[e] = k0 == 0 && i == 0 ? y[e] : max_pair(hi[e], y[e], FP8);
        }
      }
    }
#pragma unroll
    for (int o = kLanes; o < 32; o <<= 1)
#pragma unroll
      for (int e = 0; e < kWords; ++e) {
        lo[e] = min_pair(lo[e], __shfl_xor_sync(0xffffffffu, lo[e], o), FP8);
        hi[e] = max_pair(hi[e], __shfl_xor_sync(0xffffffffu, hi[e], o), FP8);
      }
    if (lane < kLanes) {
      uint4* out = p.summaries + ((int64_t)blk * p.n_kv + head) * (D / 4) + lane * (kWords / 4);  // 2 * D * 2 / 16 pieces of a summary
      if constexpr (FP8) {
#pragma unroll
        for (int e = 0; e < kWords; ++e) lo[e] = half2_to_bf16(lo[e]), hi[e] = half2_to_bf16(hi[e]);
      }
#pragma unroll
      for (int e = 0; e < kWords; e += 4) {
        out[e / 4] = make_uint4(lo[e], lo[e + 1], lo[e + 2], lo[e + 3]);
        out[D / 8 + e / 4] = make_uint4(hi[e], hi[e + 1], hi[e + 2], hi[e + 3]);
      }
    }
  }
}

// ---- selection
struct SelectParams {
  const __nv_bfloat16* q;
  int64_t q_ts, q_hs;
  int32_t n_q, n_kv, group;
  int32_t n_tokens;
  const int32_t* q_start;
  const int32_t* seq_lens;
  int32_t nreq;
  const uint4* summaries;  // [num_blocks][n_kv][2][head_dim] bf16
  const int32_t* tables;
  int32_t max_blocks, block_size;
  int64_t num_blocks;
  int32_t n_select, n_first, n_last;
  int32_t* blocks;         // [n_tokens][n_kv][n_select]
  float* scores;           // [n_tokens][n_kv][max_blocks] or nullptr
};

constexpr int kSelectThreads = 256;
constexpr int kSelectMaxBlocks = 49152;  // keys of a token that fit the shared memory of a CTA
constexpr int kSelectBins = 2048;
constexpr uint32_t kKeyForced = 0xffffffffu;  // above every score's, which end at plus infinity (NaN counts as that)
// Order-preserving map of fp32 to integers; 0 is left for blocks that cannot be chosen.
__device__ __forceinline__ uint32_t select_key(float s) {
  const uint32_t u = s != s ? 0x7f800000u : __float_as_uint(s + 0.f);  // (-0 and +0 are equal)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The request of token t, -1: none; by a whole warp, 32 borders at a time.
__device__ __forceinline__ int request_of_token(const int32_t* q_start, int nreq, int t) {
  // (a decode step has one token per request)
  if (t < nreq && __ldg(q_start + t) == t && __ldg(q_start + t + 1) == t + 1) return t;
  const int lane = threadIdx.x & 31;
  int lo = 0, n = nreq + 1;  // borders lo .. lo + n - 1: find the last one that is <= t
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int i = lane * step;
    const bool below = i < n && __ldg(q_start + lo + i) <= t;
    const unsigned m = __ballot_sync(0xffffffffu, below);
    const int k = m ? 31 - __clz(m) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo < nreq && __ldg(q_start + lo) <= t && __ldg(q_start + lo + 1) > t ? lo : -1;
}

// A cluster per (token, K/V head): its CTAs score a part of the blocks each and put the scores' keys into the shared memory of the first one,
// which finds the border of the n_select best by three passes of counting (11, 11 and 10 bits) and writes the chosen blocks in order.  The sums are
// formed in 64 bits and rounded to fp32 once: near the border a list depends on the last bits of the scores, which must therefore not depend on the
// order of summation.  Bound: HBM where many long contexts are scored (a summary is read once per token).
template <int D>
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const SelectParams p) {
  namespace cg = cooperative_groups;
  constexpr int kLanes = D / 4 < 16 ? D / 4 : 16;  // lanes of a summary
  constexpr int kPieces = D / 4 / kLanes;          // 16-byte pieces that a lane takes of it
  constexpr int kPerWarp = 32 / kLanes;
  constexpr int kFlight = kPieces >= 4 ? 2 : 4;    // summaries of a lane that fly together
  extern __shared__ uint32_t s_keys[];             // [max_blocks], of the cluster's first CTA
  __shared__ double s_q[2][D];                     // N, P
  __shared__ uint32_t s_hist[kSelectBins];
  __shared__ int64_t s_scan[32];
  __shared__ int32_t s_req;
  __shared__ uint32_t s_border[3];
  __shared__ uint32_t s_counts[2 * kSelectThreads / 32];
  grid_dependency_wait();
  grid_launch_dependents();
  cg::cluster_group cluster = cg::this_cluster();
  const unsigned rank = cluster.block_rank(), parts = cluster.num_blocks();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t unit = blockIdx.x / parts;
  const int t = (int)(unit / p.n_kv), head = (int)(unit - (int64_t)t * p.n_kv);
  if (warp == 0) {
    const int r = request_of_token(p.q_start, p.nreq, t);
    if (lane == 0) s_req = r;
  }
  for (int d = tid; d < D; d += kSelectThreads) {
    double lo = 0., hi = 0.;
    for (int g = 0; g < p.group; ++g) {
      const float x = __bfloat162float(p.q[t * p.q_ts + (head * p.group + g) * p.q_hs + d]);
      if (x >= 0.f) hi += x;
      else lo += x;  // (NaN too)
    }
    s_q[0][d] = lo;
    s_q[1][d] = hi;
  }
  cluster.sync();  // (shared memory is there, and the first CTA's may be written)
  const int r = s_req;
  if (r < 0) return;  // (the whole cluster)
  const int32_t q0 = __ldg(p.q_start + r), q1 = __ldg(p.q_start + r + 1), len = __ldg(p.seq_lens + r);
  if (q0 < 0 || q1 > p.n_tokens || len < 0 || len > kAttnMaxLen) return;
  const int64_t pos = (int64_t)len - (q1 - q0) + (t - q0);
  const int all = pos < 0 ? 0 : (int)(pos / p.block_size) + 1;  // blocks with keys that the token may see
  const int nb = min(all, p.max_blocks);
  const int32_t* table = p.tables + (int64_t)r * p.max_blocks;
  float* scores = p.scores ? p.scores + unit * p.max_blocks : nullptr;

  // ---- scores
  const int sub = lane % kLanes;
  double q[kPieces][8];
#pragma unroll
  for (int i = 0; i < kPieces; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) q[i][e] = (&s_q[0][0])[(sub + i * kLanes) * 8 + e];
  uint32_t* keys = cluster.map_shared_rank(s_keys, 0);
  const int step = kPerWarp * kFlight, warps = (int)parts * (kSelectThreads / 32);
  for (int b0 = ((int)rank * (kSelectThreads / 32) + warp) * step; b0 < nb; b0 += warps * step) {
    uint4 x[kFlight][kPieces];
    int32_t blk[kFlight];
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const int b = b0 + f * kPerWarp + lane / kLanes;
      blk[f] = b < nb ? __ldg(table + b) : -1;
      if (blk[f] >= p.num_blocks) blk[f] = -1;
    }
#pragma unroll
    for (int f = 0; f < kFlight; ++f)
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        x[f][i] = blk[f] >= 0 ? ld_stream(p.summaries + ((int64_t)blk[f] * p.n_kv + head) * (D / 4) + sub + i * kLanes) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      double s = 0.;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const uint32_t y[4] = {x[f][i].x, x[f][i].y, x[f][i].z, x[f][i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s = fma(q[i][2 * e], (double)bf16lo(y[e]), s);
          s = fma(q[i][2 * e + 1], (double)bf16hi(y[e]), s);
        }
      }
#pragma unroll
      for (int o = kLanes / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      const int b = b0 + f * kPerWarp + lane / kLanes;
      if (sub == 0 && b < nb) {
        const float v = blk[f] >= 0 ? (float)s : -INFINITY;
        if (scores) scores[b] = v;
        keys[b] = blk[f] < 0 ? 0u : b < p.n_first || b >= all - p.n_last ? kKeyForced : select_key(v);
      }
    }
  }
  cluster.sync();
  if (rank != 0) return;

  // ---- the border: the key of the n_select-th best, and how many blocks with that key are taken
  int can = 0;
  for (int b = tid; b < nb; b += kSelectThreads) can += s_keys[b] != 0u;
  int64_t total;
  block_scan<kSelectThreads>(can, s_scan, &total);
  uint32_t border = 0u;
  int ties = 0;
  if (total > p.n_select) {
    uint32_t prefix = 0u, prefix_mask = 0u;
    int want = p.n_select;
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
      for (int i = tid; i < kSelectBins; i += kSelectThreads) s_hist[i] = 0u;
      __syncthreads();
      for (int b = tid; b < nb; b += kSelectThreads) {
        const uint32_t k = s_keys[b];
        if (k != 0u && (k & prefix_mask) == prefix) atomicAdd(&s_hist[(k >> shift) & (bins - 1)], 1u);
      }
      __syncthreads();
      // thread i has the bins from the top: 8 i .. 8 i + 7
      constexpr int kBins = kSelectBins / kSelectThreads;
      uint32_t mine = 0u;
#pragma unroll
      for (int i = 0; i < kBins; ++i) mine += s_hist[kSelectBins - 1 - (tid * kBins + i)];
      const int64_t upto = block_scan<kSelectThreads>((int64_t)mine, s_scan, &total);
      if (upto >= want && upto - mine < want) {
        int before = (int)(upto - mine);
        for (int i = 0; i < kBins; ++i) {
          const int bin = kSelectBins - 1 - (tid * kBins + i);
          if (before + (int)s_hist[bin] >= want) {
            s_border[0] = (uint32_t)bin;
            s_border[1] = (uint32_t)(want - before);
            break;
          }
          before += s_hist[bin];
        }
      }
      __syncthreads();
      prefix |= s_border[0] << shift;
      prefix_mask |= (uint32_t)(bins - 1) << shift;
      want = (int)s_border[1];
    }
    border = prefix;
    ties = want;
  }
  // ---- the chosen blocks in rising order: a warp has a run of blocks
  const int run = ((nb + kSelectThreads - 1) / kSelectThreads) * 32, from = warp * run, to = min(nb, from + run);
  uint32_t above = 0u, equal = 0u;
  for (int b0 = from; b0 < to; b0 += 32) {
    const int b = b0 + lane;
    const uint32_t k = b < to ? s_keys[b] : 0u;
    above += __popc(__ballot_sync(0xffffffffu, k > border));
    equal += __popc(__ballot_sync(0xffffffffu, k == border && k != 0u));
  }
  if (lane == 0) {
    s_counts[warp] = above;
    s_counts[kSelectThreads / 32 + warp] = equal;
  }
  __syncthreads();
  uint32_t above_before = 0u, equal_before = 0u, above_all = 0u, equal_all = 0u;
  for (int w = 0; w < kSelectThreads / 32; ++w) {
    if (w < warp) above_before += s_counts[w], equal_before += s_counts[kSelectThreads / 32 + w];
    above_all += s_counts[w], equal_all += s_counts[kSelectThreads / 32 + w];
  }
  int32_t* out = p.blocks + unit * p.n_select;
  const unsigned lower = (1u << lane) - 1u;
  for (int b0 = from; b0 < to; b0 += 32) {
    const int b = b0 + lane;
    const uint32_t k = b < to ? s_keys[b] : 0u;
    const unsigned ma = __ballot_sync(0xffffffffu, k > border), me = __ballot_sync(0xffffffffu, k == border && k != 0u);
    const uint32_t eq = equal_before + __popc(me & lower);  // blocks with the border's key before this one
    if (k > border || (k != 0u && k == border && eq < (uint32_t)ties)) out[above_before + __popc(ma & lower) + min(eq, (uint32_t)ties)] = b;
    above_before += __popc(ma);
    equal_before += __popc(me);
  }
  const int taken = (int)(above_all + min(equal_all, (uint32_t)ties));
  for (int i = taken + tid; i < p.n_select; i += kSelectThreads) out[i] = -1;
}

}  // namespace ms

// memstore_append: rotate the queries and keys of new tokens at their positions and write keys and values into one layer of
// the paged cache.
//
// Mathematics: (a, b) -> (a cos - b sin, b cos + a sin) for every pair at angle pos * inv_freq, with the angle, the fp32
// arithmetic and the single rounding of the injection kernel (rope_sincos, rotate_unit); an 8-bit cache takes
// e4m3(bf16 value / scale), as there.  So a token appended here has the bytes that injecting it would have written.
// Bound: HBM (every value is read once and written once).
#pragma once
#include "inject.cuh"

namespace ms {

struct AppendParams {
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* q_out;
  int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;  // token and head strides in elements
  int32_t n_q, n_kv;  // heads
  int32_t head_dim, rotary_dim, max_position;
  const float* inv_freq;
  const int32_t* positions;
  const int64_t* slots;
  int32_t n_tokens;
  int32_t threads_per_token;  // a power of two and a multiple of head_dim / 16, at most kAppendThreads
  __nv_bfloat16 *k_cache, *v_cache;  // of the layer
  int64_t block_stride, token_stride, head_stride, num_blocks;
  int32_t block_size;
  float k_scale, v_scale, k_recip, v_recip;
  int32_t* status;
};

constexpr int kAppendThreads = 256;
constexpr int kAppendBatch = 4;  // units a thread loads before it works on the first

// A read that leaves nothing behind in L1 (plain, not through the read-only path: q_out may be q).
__device__ __forceinline__ uint4 ld_once(const __nv_bfloat16* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

// A unit is (head, octet of frequencies): two 16-byte vectors.  threads_per_token threads serve a token; all units of a thread
// have one octet, so that it forms its eight sines and cosines once.  The heads are numbered q, k, v.
// What limits it is how many loads are in flight: three CTAs per SM with four units per thread take 21.4 us for 4,097 tokens of 56 heads
// (5.5 TB/s); two CTAs (no limit on registers) 24.5, four 24.6, two units 25.6, 27 without the streaming forms of loads and stores, and 23.1
// when the CTA shares its sines and cosines through shared memory (the barrier costs more than the arithmetic).  An 8-bit cache is held
// back by instructions: 8,191 tokens of 32 query and 16 other heads execute 25 % more of them than with a bf16 cache at the same issue rate
// (58 - 60 % of the slots) and take 43.6 us instead of 35.4, although they write less.
template <int STYLE, int FP8>
__global__ void __launch_bounds__(kAppendThreads, 3) append_kernel(const AppendParams p) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int tpt = p.threads_per_token;
  const int64_t t = (int64_t)blockIdx.x * (kAppendThreads / tpt) + threadIdx.x / tpt;
  if (t >= p.n_tokens) return;
  const int l = threadIdx.x & (tpt - 1);
  const int D = p.head_dim, G = D >> 4, g_shift = 31 - __clz(G);
  const int j = l & (G - 1);
  const int R = p.rotary_dim;
  const bool rotates = 16 * j < R;
  const int offA = (STYLE == 0 && rotates) ? 8 * j : 16 * j;
  const int offB = (STYLE == 0 && rotates) ? R / 2 + 8 * j : 16 * j + 8;

  const int32_t pos = p.positions[t];
  const int64_t slot = p.slots[t];
  const bool pos_ok = pos >= 0 && pos < p.max_position;
  // (slots below 2^32 are divided in 32 bits)
  const int64_t blk = slot < 0 ? -1 : (slot >> 32) == 0 ? (int64_t)((uint32_t)slot / (uint32_t)p.block_size) : slot / p.block_size;
  const bool slot_ok = blk >= 0 && blk < p.num_blocks;
  if (p.status && l == 0) p.status[t] = pos < 0 ? 64 : pos >= p.max_position ? 16 : slot_ok ? 0 : 8;
  if (!pos_ok) return;
  const int64_t dst = slot_ok ? blk * p.block_stride + (slot - blk * p.block_size) * p.token_stride : 0;

  const int h_step = tpt >> g_shift;
  const int h_end = slot_ok ? p.n_q + 2 * p.n_kv : p.n_q;
  float sn[8], cs[8];
  bool have = false;
  for (int h0 = l >> g_shift; h0 < h_end; h0 += kAppendBatch * h_step) {
    uint4 a[kAppendBatch], b[kAppendBatch];
#pragma unroll
    for (int u = 0; u < kAppendBatch; ++u) {
      const int h = h0 + u * h_step;
      if (h < h_end) {
        const int hk = h - p.n_q, hv = hk - p.n_kv;
        const __nv_bfloat16* x = hk < 0 ? p.q + t * p.q_ts + h * p.q_hs : hv < 0 ? p.k + t * p.k_ts + hk * p.k_hs : p.v + t * p.v_ts + hv * p.v_hs;
        a[u] = ld_once(x + offA);
        b[u] = ld_once(x + offB);
      }
    }
    if (!have && rotates) {  // formed while the first loads fly
      const float posf = (float)pos;
#pragma unroll
      for (int i = 0; i < 8; ++i) rope_sincos(posf, __ldg(p.inv_freq + 8 * j + i), sn[i], cs[i]);
    }
    have = true;
#pragma unroll
    for (int u = 0; u < kAppendBatch; ++u) {
      const int h = h0 + u * h_step;
      if (h < h_end) {
        const int hk = h - p.n_q, hv = hk - p.n_kv;
        if (hv < 0 && rotates) rotate_unit<STYLE>(a[u], b[u], sn, cs);
        if (hk < 0) {
          __nv_bfloat16* o = p.q_out + t * p.o_ts + h * p.o_hs;
          st_stream(reinterpret_cast<uint4*>(o + offA), a[u]);
          st_stream(reinterpret_cast<uint4*>(o + offB), b[u]);
        } else if (!FP8) {
          __nv_bfloat16* o = (hv < 0 ? p.k_cache + hk * p.head_stride : p.v_cache + hv * p.head_stride) + dst;
          st_stream(reinterpret_cast<uint4*>(o + offA), a[u]);
          st_stream(reinterpret_cast<uint4*>(o + offB), b[u]);
        } else {
          float fa[8], fb[8];
          const float scale = hv < 0 ? p.k_scale : p.v_scale, recip = hv < 0 ? p.k_recip : p.v_recip;
          scaled_floats<FP8 == 2>(a[u], scale, recip, fa);
          scaled_floats<FP8 == 2>(b[u], scale, recip, fb);
          uint8_t* o = (hv < 0 ? reinterpret_cast<uint8_t*>(p.k_cache) + hk * p.head_stride : reinterpret_cast<uint8_t*>(p.v_cache) + hv * p.head_stride) + dst;
          st_stream8(reinterpret_cast<uint2*>(o + offA), pack_e4m3x8(fa));
          st_stream8(reinterpret_cast<uint2*>(o + offB), pack_e4m3x8(fb));
        }
      }
    }
  }
}

}  // namespace ms

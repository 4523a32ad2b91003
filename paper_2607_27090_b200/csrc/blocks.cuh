// Block tables and slot maps from request lengths (memstore_grow_blocks) and the return of blocks
// (memstore_release_blocks).  The free list is a stack in an array: entries [n_taken, n_free) are free.
#pragma once
#include "common.cuh"

namespace ms {

// request status bits (the MS_REQ_* of the header; static_asserts in memstore.cu compare them)
constexpr int32_t kReqTableShort = 4, kReqBadBlock = 8, kReqPosOverflow = 16, kReqTimeout = 32, kReqBadStart = 64, kReqNoBlocks = 128,
                  kReqBadLength = 256;
constexpr int32_t kReqRefused = kReqTableShort | kReqPosOverflow | kReqBadStart | kReqNoBlocks | kReqBadLength;

constexpr int kGrowThreads = 1024;      // one thread per request of a pass over the requests
// Tokens up to which the planning CTA maps them itself; above, a second kernel does (whose CTAs scan the requests).  4,096 / 8,192 /
// 16,384 tokens in one launch and in two: 1 request 6.6 / 9.5 / 15.4 us against 10.0 / 10.2 / 10.0, 24 requests 7.8 / 11.8 / 19.4 against 12.4 /
// 12.2 / 12.3, 256 requests 8.6 / 13.4 / 23.1 against 14.1 / 13.9 / 14.2; 2,048 requests cross later (17.7 against 26.8 at 8,192, 28.5 against
// 26.5 at 16,384).
constexpr int kGrowOneLaunch = 8192;
constexpr int kGrowMapThreads = 256;
constexpr int kGrowMapTokens = 2048;    // tokens of one CTA of the mapping kernel

struct GrowParams {
  const int32_t* start_lens;
  const int32_t* new_lens;
  int32_t nreq;
  int32_t* tables;
  int32_t max_blocks;
  int32_t block_size;
  int64_t num_blocks;
  int32_t max_position;
  const int32_t* free_blocks;
  int32_t n_free;
  const int32_t* n_taken;
  int32_t token_capacity;
  int32_t* q_start;
  int32_t* seq_lens;
  int32_t* positions;
  int64_t* slots;
  int32_t* out_n_taken;
  int32_t* status;
};

// Inclusive scan over the block's threads (THREADS a multiple of 32, at most 1024); *total receives the sum.
template <int THREADS>
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* s_warp, int64_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();  // the previous scan's readers are done with s_warp
  if (lane == 31) s_warp[warp] = v;
  __syncthreads();
  // every warp scans the warp totals for itself
  int64_t w = lane < THREADS / 32 ? s_warp[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += u;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const int64_t before = __shfl_sync(0xffffffffu, w, warp == 0 ? 0 : warp - 1);
  return warp == 0 ? v : v + before;
}

// What the mapping of a token needs to know of its request.
struct GrowReq {
  int32_t q_end;  // exclusive end of the request's tokens in the packed arrays
  int32_t n;      // its tokens
  int32_t start;  // position of the first one, -1: refused
  int32_t first;  // index in the free list of its first new block
};

// Positions and slots of the packed tokens [tok0, tok1) whose requests are r0 .. r0 + n_reqs - 1 of this pass; the token that
// opens a new block writes the block's table entry.
__device__ __forceinline__ void grow_map_tokens(const GrowParams& p, const GrowReq* s_req, int r0, int n_reqs, int tok0, int tok1, int tid,
                                                int threads) {
  const int bs = p.block_size;
  for (int i = tok0 + tid; i < tok1; i += threads) {
    int lo = 0, hi = n_reqs - 1;  // the first request whose end lies behind token i
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_req[mid].q_end > i) hi = mid; else lo = mid + 1;
    }
    const GrowReq q = s_req[lo];
    int32_t pos = -1;
    int64_t slot = -1;
    if (q.start >= 0) {
      pos = q.start + (i - (q.q_end - q.n));
      const int32_t held = (int32_t)(((int64_t)q.start + bs - 1) / bs);
      const int32_t b = pos / bs;
      int32_t* entry = p.tables + (int64_t)(r0 + lo) * p.max_blocks + b;
      int32_t blk = b < held ? *entry : p.free_blocks[q.first + (b - held)];
      const bool good = blk >= 0 && blk < p.num_blocks;
      if (!good) {
        atomicOr(p.status + r0 + lo, kReqBadBlock);
        blk = -1;
      }
      if (b >= held && pos == b * bs) *entry = blk;
      if (good) slot = (int64_t)blk * bs + (pos - b * bs);
    }
    if (p.positions) p.positions[i] = pos;
    if (p.slots) p.slots[i] = slot;
  }
}

// One CTA decides every request: two scans (tokens, then blocks) per 1024 requests.  With map_tokens it also writes positions,
// slots and table entries itself (few tokens: one launch); otherwise grow_map_kernel follows.  All inputs of a pass are read
// before its outputs are written, so the lengths and the counter may be updated in place.
__global__ void __launch_bounds__(kGrowThreads) grow_plan_kernel(const GrowParams p, const int map_tokens) {
  __shared__ int64_t s_warp[32];
  __shared__ GrowReq s_req[kGrowThreads];
  grid_dependency_wait();
  grid_launch_dependents();
  const int tid = threadIdx.x;
  const int bs = p.block_size;
  const int64_t taken = *p.n_taken;
  const bool list_ok = taken >= 0 && taken <= p.n_free;
  int64_t tokens = 0, asked = 0;    // of the requests before this pass
  int64_t given_end = taken;        // free-list index behind the last block given out
  if (tid == 0) p.q_start[0] = 0;
  for (int r0 = 0; r0 < p.nreq; r0 += kGrowThreads) {
    const int r = r0 + tid;
    const bool live = r < p.nreq;
    const int32_t s = live ? p.start_lens[r] : 0, n_in = live ? p.new_lens[r] : 0;
    const int32_t n = max(n_in, 0);
    int32_t st = (s < 0 ? kReqBadStart : 0) | (n_in < 0 ? kReqBadLength : 0);
    int64_t total;
    const int64_t end = tokens + block_scan<kGrowThreads>(n, s_warp, &total);  // (contains a barrier: the pass's inputs are read)
    tokens += total;
    if (end > p.token_capacity && n > 0) st |= kReqBadLength;
    const int64_t last = (int64_t)s + n;
    if (last > p.max_position) st |= kReqPosOverflow;
    const int64_t held = s > 0 ? ((int64_t)s + bs - 1) / bs : 0, want = last > 0 ? (last + bs - 1) / bs : 0;
    if (want > p.max_blocks) st |= kReqTableShort;
    const int64_t need = st == 0 ? want - held : 0;
    const int64_t upto = asked + block_scan<kGrowThreads>(need, s_warp, &total);
    asked += total;
    const bool fits = list_ok && taken + upto <= p.n_free;
    if (need > 0 && !fits) st |= kReqNoBlocks;
    const bool served = st == 0;
    // the blocks given out are those of the served requests: a prefix of the ones asked for
    int64_t dummy;
    const int64_t mine = served && need > 0 ? need : 0;
    block_scan<kGrowThreads>(mine, s_warp, &dummy);
    given_end += dummy;
    if (live) {
      const int32_t q_end = (int32_t)min(end, (int64_t)p.token_capacity);
      p.q_start[r + 1] = q_end;
      p.seq_lens[r] = served ? (int32_t)last : s;
      p.status[r] = st;
      s_req[tid] = GrowReq{q_end, (int32_t)(q_end - min(end - n, (int64_t)p.token_capacity)), served ? s : -1, (int32_t)(taken + upto - need)};
    }
    if (map_tokens) {
      __syncthreads();
      const int n_reqs = min(kGrowThreads, p.nreq - r0);
      const int tok0 = s_req[0].q_end - s_req[0].n, tok1 = s_req[n_reqs - 1].q_end;
      grow_map_tokens(p, s_req, r0, n_reqs, tok0, tok1, tid, kGrowThreads);
      __syncthreads();  // s_req is reused
    }
  }
  if (map_tokens) {
    for (int64_t i = min(tokens, (int64_t)p.token_capacity) + tid; i < p.token_capacity; i += kGrowThreads) {
      if (p.positions) p.positions[i] = -1;
      if (p.slots) p.slots[i] = -1;
    }
  }
  if (tid == 0) *p.out_n_taken = (int32_t)given_end;
}

// Positions, slots and table entries of many tokens: every CTA serves kGrowMapTokens of them and scans the requests for itself,
// from what grow_plan_kernel wrote (so that updates in place are safe): a served request's blocks follow those of the served
// requests before it.
__global__ void __launch_bounds__(kGrowMapThreads) grow_map_kernel(const GrowParams p) {
  __shared__ int64_t s_warp[32];
  __shared__ GrowReq s_req[kGrowMapThreads];
  grid_dependency_wait();
  grid_launch_dependents();
  const int tid = threadIdx.x;
  const int bs = p.block_size;
  const int tok0 = blockIdx.x * kGrowMapTokens;
  const int tok1 = (int)min((int64_t)p.token_capacity, (int64_t)tok0 + kGrowMapTokens);
  // the free-list index of the first block given out by this call = the counter now - all blocks given out
  int64_t all = 0;
  for (int r = tid; r < p.nreq; r += kGrowMapThreads) {
    if (p.status[r] & kReqRefused) continue;
    const int64_t last = p.seq_lens[r], n = p.q_start[r + 1] - p.q_start[r], s = last - n;
    all += (last + bs - 1) / bs - (s + bs - 1) / bs;
  }
  int64_t total;
  block_scan<kGrowMapThreads>(all, s_warp, &total);
  int64_t first = *p.out_n_taken - total;
  for (int r0 = 0; r0 < p.nreq; r0 += kGrowMapThreads) {
    const int r = r0 + tid;
    int64_t need = 0;
    GrowReq q{0, 0, -1, 0};
    if (r < p.nreq) {
      const int32_t a = p.q_start[r], b = p.q_start[r + 1];
      q.q_end = b;
      q.n = b - a;
      if (!(p.status[r] & kReqRefused)) {
        const int64_t last = p.seq_lens[r], s = last - q.n;
        need = (last + bs - 1) / bs - (s + bs - 1) / bs;
        q.start = (int32_t)s;
      }
    }
    const int64_t upto = block_scan<kGrowMapThreads>(need, s_warp, &total);
    q.first = (int32_t)(first + upto - need);
    first += total;
    s_req[tid] = q;
    __syncthreads();
    const int n_reqs = min(kGrowMapThreads, p.nreq - r0);
    const int p0 = s_req[0].q_end - s_req[0].n, p1 = s_req[n_reqs - 1].q_end;
    grow_map_tokens(p, s_req, r0, n_reqs, max(tok0, p0), min(tok1, p1), tid, kGrowMapThreads);
    __syncthreads();
    if (p1 >= tok1) return;  // (uniform) the requests that follow have no tokens here
  }
  for (int i = max(tok0, p.q_start[p.nreq]) + tid; i < tok1; i += kGrowMapThreads) {
    if (p.positions) p.positions[i] = -1;
    if (p.slots) p.slots[i] = -1;
  }
}

struct ReleaseParams {
  const int32_t* release;
  int32_t* seq_lens;
  int32_t nreq;
  int32_t* tables;
  int32_t max_blocks;
  int32_t block_size;
  int64_t num_blocks;
  int32_t* free_blocks;
  int32_t n_free;
  int32_t* n_taken;
  int32_t* status;
};

// One CTA, a warp per request: count the blocks to return, scan the counts, write them back in front of the free part.  Latency: 24
// requests of 250 blocks 5 us, 100 of 80 9 us, 512 of 1,000 179 us (32 requests at a time, 32 entries a step; finished requests are few at a
// time in a serving loop).
__global__ void __launch_bounds__(kGrowThreads) release_kernel(const ReleaseParams p) {
  __shared__ int64_t s_warp[32];
  __shared__ int32_t s_count[kGrowThreads];
  __shared__ int64_t s_at[kGrowThreads];  // free-list index of the request's first block, -1: it keeps its blocks
  grid_dependency_wait();
  grid_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int bs = p.block_size;
  const int64_t taken = *p.n_taken;
  const bool list_ok = taken >= 0 && taken <= p.n_free;
  auto held_of = [&](int r) -> int {
    if (p.release && p.release[r] == 0) return 0;
    const int64_t len = p.seq_lens[r];
    return (int)min(len > 0 ? (len + bs - 1) / bs : (int64_t)0, (int64_t)p.max_blocks);
  };
  // Requests are served in order as long as their blocks fit, so the blocks of request r go below those of earlier ones:
  // the list grows downwards from n_taken, request 0's blocks ending at n_taken.
  int64_t asked = 0, returned = 0;
  for (int r0 = 0; r0 < p.nreq; r0 += kGrowThreads) {
    const int n_reqs = min(kGrowThreads, p.nreq - r0);
    s_count[tid] = 0;
    __syncthreads();
    for (int i = warp; i < n_reqs; i += kGrowThreads / 32) {
      const int held = held_of(r0 + i);
      const int32_t* t = p.tables + (int64_t)(r0 + i) * p.max_blocks;
      int count = 0;
      for (int b = lane; b < held; b += 32) count += t[b] >= 0 && t[b] < p.num_blocks;
      count = __reduce_add_sync(0xffffffffu, count);
      if (lane == 0) s_count[i] = count;
    }
    __syncthreads();
    const int64_t c = s_count[tid];
    int64_t total, given;
    const int64_t upto = asked + block_scan<kGrowThreads>(c, s_warp, &total);
    asked += total;
    const bool fits = c == 0 || (list_ok && upto <= taken);
    s_at[tid] = fits ? taken - upto : -1;
    block_scan<kGrowThreads>(fits ? c : 0, s_warp, &given);
    returned += given;
    __syncthreads();
    for (int i = warp; i < n_reqs; i += kGrowThreads / 32) {
      const int r = r0 + i;
      const int held = held_of(r);
      const int64_t at = s_at[i];
      int32_t st = 0;
      if (held > 0 && at < 0 && s_count[i] > 0) {
        st = kReqNoBlocks;
      } else if (held > 0) {
        int32_t* t = p.tables + (int64_t)r * p.max_blocks;
        int done = 0;
        for (int b0 = 0; b0 < held; b0 += 32) {
          const int b = b0 + lane;
          const int32_t blk = b < held ? t[b] : -1;
          const bool good = blk >= 0 && blk < p.num_blocks;
          const unsigned m = __ballot_sync(0xffffffffu, good);
          if (good) p.free_blocks[at + done + __popc(m & ((1u << lane) - 1u))] = blk;
          done += __popc(m);
          if (b < held) t[b] = -1;
        }
        if (done < held) st = kReqBadBlock;
        __syncwarp();  // every lane has read the length
        if (lane == 0) p.seq_lens[r] = 0;
      } else if (lane == 0 && (!p.release || p.release[r] != 0)) {
        p.seq_lens[r] = 0;
      }
      if (p.status && lane == 0) p.status[r] = st;
    }
    __syncthreads();
  }
  if (tid == 0) *p.n_taken = (int32_t)(taken - returned);
}

}  // namespace ms

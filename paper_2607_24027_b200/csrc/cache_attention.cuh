// What the two attention kernels over the 4-bit cache (cache_attention.cu, cache_attention_chunk.cu) share: parameters, the
// division of the work among blocks, and where partial results go.
#pragma once

#include "cache.cuh"

namespace sol {
namespace cache {

// An item of which a block had the last piece and others the rest: the first of them (-1: there is no such item), and where its rows
// belong.
struct alignas(32) Record { int from, head, tile, queries, first, pad0, pad1, pad2; };

struct AttnParams {
  const void* q;
  void* out;
  float* lse;
  long long q_s[2], o_s[2], table_stride;
  const int32_t *cu_q, *kv_lens, *tables;
  const unsigned char* data;
  int tokens, requests, max_blocks, Hq, Hk, group, causal, pages, page_shift;
  long long rows_from, rows_to;                  // requests with other numbers of rows are another kernel's
  float sl2;                                     // logit scale * log2(e) * 2^k_exp
  float v_scale;                                 // 2^v_exp
  int32_t* status;
  long long wait_limit;                          // SM clocks after which a bounded wait gives up
  int withhold;                                  // test hook: >= 0: the arrival for this step of each block is left out
  Record* records;                               // per block: what it leaves to be joined
  float* parts;                                  // two partial results per block
};

// Queries and keys of a request, within what the caller's buffers hold.
struct Request { int first, queries, keys; };
__device__ __forceinline__ Request request_at(const AttnParams& p, int b) {
  Request r;
  r.first = max(0, min(p.cu_q[b], p.tokens));
  r.queries = max(0, min(p.cu_q[b + 1], p.tokens) - r.first);
  r.keys = (int)max(0LL, min((long long)p.kv_lens[b], (long long)p.max_blocks << p.page_shift));
  return r;
}

// Work is counted in steps of so many keys of one item: a tile of rows of one request and key / value head, a row being one query
// of one of the head's `group` query heads.  Items lie one after the other (request, head, tile), and the blocks take equal
// shares of the steps, the first ones one more where they do not come out even: every block has the same to do, however ragged the
// batch, and an item is cut into as many pieces as there are blocks on it.  A piece that is not a whole item is left in `parts`
// and joined by a second kernel, in order.
struct Work {
  int tiles, steps;                              // of a request: row tiles per head, steps per item (at least one)
  __device__ Work(const AttnParams& p, const Request& r, int rows, int step) {
    const long long all = (long long)r.queries * p.group;
    tiles = all < p.rows_from || all > p.rows_to ? 0 : (int)(((uint32_t)all + rows - 1) / rows);     // (not this kernel's request: none)
    steps = max(1, (r.keys + step - 1) / step);
  }
  __device__ long long total(int heads) const { return (long long)tiles * heads * steps; }
};

// a / b for a >= 0, b > 0; 32 bits do it nearly always, and are several times as fast.
__device__ __forceinline__ long long quotient(long long a, long long b) {
  return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}
struct Shares {
  long long work, blocks, each, extra;           // blocks with work; steps of a block, and how many have one more
  __device__ Shares(long long work_, long long grid) : work(work_), blocks(min(grid, work_)) {
    each = blocks ? quotient(work, blocks) : 0;
    extra = work - each * blocks;
  }
  __device__ long long begin(long long c) const { return c * each + min(c, extra); }
  __device__ long long owner(long long w) const {
    return w < extra * (each + 1) ? quotient(w, each + 1) : extra + quotient(w - extra * (each + 1), each);
  }
};

struct Start {                                   // where a block begins
  Request request;
  int index;                                     // of the request
  long long base;                                // its first step
};

// The sum of the requests' work, and, where `c` has a share of it, where that begins (in `start`, shared memory).  The whole block
// calls it; `sums`: shared memory, a word per warp.
template <int kThreads>
__device__ Shares find_share(const AttnParams& p, int rows, int step, long long c, long long* sums, Start* start) {
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  long long all = 0, x = 0, n = 0;
  Request r{0, 0, 0};
  auto scan = [&](int b0) {                      // of requests b0 ...: x the sum up to this thread's, n its own; returns that of all
    r = Request{0, 0, 0};
    n = 0;
    if (b0 + tid < p.requests) { r = request_at(p, b0 + tid); n = Work(p, r, rows, step).total(p.Hk); }
    x = n;
    for (int o = 1; o < 32; o *= 2) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    long long s = 0;
    for (int w = 0; w < kThreads / 32; ++w) { if (w == warp) x += s; s += sums[w]; }
    return s;
  };
  for (int b0 = 0; b0 < p.requests; b0 += kThreads) all += scan(b0);
  const Shares sh(all, gridDim.x);
  if (c < sh.blocks) {
    const long long w = sh.begin(c);
    long long base = 0;
    for (int b0 = 0; b0 < p.requests; b0 += kThreads) {
      const long long s = p.requests > kThreads ? scan(b0) : all;              // (a single round is still at hand)
      const long long lo = base + x - n;
      if (n > 0 && lo <= w && w < lo + n) *start = Start{r, b0 + tid, lo};
      base += s;
      if (w < base) break;                       // (the whole block)
    }
    __syncthreads();
  }
  return sh;
}

}  // namespace cache
}  // namespace sol

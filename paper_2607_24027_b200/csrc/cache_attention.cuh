// What the two attention kernels over the 4-bit cache (cache_attention.cu, cache_attention_chunk.cu) share: parameters, the
// division of the work among blocks, and where partial results go.
#pragma once

#include "cache.cuh"

namespace sol {
namespace cache {

// Weights are 2^(x - m + kShift) with x the logit times log2(e) and m a maximum of earlier keys, which is replaced once a weight would
// pass 2^kMost: fp16 holds them to 2^-11 down to 2^-25 of the largest, and is off by 2^-36 of it at most below.
// fp16 because the values are exact in it, and one kind of operand is all that a product takes; bf16 would hold weights to 2^-8.  A row's sum is that
// of the weights before rounding: it is lse as well as the denominator.  With the sum of the rounded ones out is as far from 64 bits (2.80e-4 against 2.82e-4,
// fp16, of which 2.1e-4 is its own rounding) and lse ten to a hundred times as far (1.5e-4 against 2e-6), and many queries take 12 to 18 % longer.
constexpr float kShift = 11.f, kMost = 15.f;
constexpr float kLn2 = 0.6931471805599453f;

constexpr int kMostBlocks = 4 * 160, kMostChunkBlocks = 160;   // of the kernel for few queries, of the other
constexpr int kChunkRows = 256;                  // rows of a block of the other

// An item of which a block had the last piece and others the rest: the first of them (-1: there is no such item), and where its rows
// belong.
struct alignas(16) Record {
  int from_head, tile, queries, first;           // from | head << 16
  __host__ __device__ bool is() const { return from_head >= 0; }
  __host__ __device__ int from() const { return from_head & 0xffff; }
  __host__ __device__ int head() const { return from_head >> 16; }
  __host__ __device__ static Record none() { return Record{-1, 0, 0, 0}; }
};

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

// Queries and keys of a request, within what the caller's buffers hold.  What they do not hold still has its place: query i lies `ahead` + i
// behind the request's first key also where the last queries are not in q, or the last keys not in the table.
struct Request {
  int first, queries, keys, ahead;
  // Keys that query i sees, causal.
  __device__ int sees(int i) const { return (int)max(0LL, min((long long)keys, (long long)ahead + i + 1)); }
};
__device__ __forceinline__ Request request_at(const AttnParams& p, int b) {
  const int end = p.cu_q[b + 1];
  const long long kv = max(0, p.kv_lens[b]);
  Request r;
  r.first = max(0, min(p.cu_q[b], p.tokens));
  r.queries = max(0, min(end, p.tokens) - r.first);
  // (0x7fff0000: sums with a step stay within 32 bits; a cache has fewer tokens than 2^31)
  r.keys = (int)min(min(kv, (long long)p.max_blocks << p.page_shift), 0x7fff0000LL);
  r.ahead = (int)max(-0x7fffffffLL, min(kv - end + r.first, (long long)r.keys));
  return r;
}

// Work is counted in steps of so many keys of one item: a tile of rows of one request and key / value head, a row being one query
// of one of the head's `group` query heads.  Items lie one after the other (request, head, tile), and the blocks take equal
// shares of the steps, the first ones one more where they do not come out even: every block has the same to do, however ragged the
// batch, and an item is cut into as many pieces as there are blocks on it.  A piece that is not a whole item is left in `parts`
// and joined by a second kernel, in order.
template <int kRows, int kStep>
struct Tiles {
  // Row tiles of a request, per head; none if the request is another kernel's.
  __device__ static int count(const AttnParams& p, const Request& r) {
    const long long all = (long long)r.queries * p.group;
    return all < p.rows_from || all > p.rows_to ? 0 : (int)(((uint32_t)all + kRows - 1) / kRows);
  }
  // Steps of a tile (at least one): up to the last key that its last row sees.
  __device__ static int steps(const AttnParams& p, const Request& r, int tile) {
    int sees = r.keys;
    if (p.causal) {
      const int last = min((tile + 1) * kRows, r.queries * p.group) - 1;
      sees = r.sees(last / p.group);
    }
    return max(1, (sees + kStep - 1) / kStep);
  }
  // Steps of all tiles of a head.
  __device__ static long long per_head(const AttnParams& p, const Request& r) {
    const int n = count(p, r);
    if (!p.causal || n <= 1) return n ? (long long)n * steps(p, r, n - 1) : 0;
    long long s = 0;
    for (int i = 0; i < n; ++i) s += steps(p, r, i);
    return s;
  }
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

// The pieces of a block's share, one after the other.
template <class Tiling>
struct Pieces {
  Request r;
  int b, head, tile, s_begin, s_end, steps;      // the piece: steps [s_begin, s_end) of `steps`
  int more;                                      // there is one
  long long w, w_end, base, per_head, item_begin;
  __device__ void start(const AttnParams& p, const Start& at, long long begin, long long end) {
    r = at.request; b = at.index; base = at.base; w = begin; w_end = end;
    per_head = Tiling::per_head(p, r);
    head = tile = s_begin = s_end = steps = 0;
    item_begin = 0;
  }
  __device__ bool next(const AttnParams& p) {
    if (w >= w_end) return false;
    if (s_end != 0 && s_end == steps && w < base + per_head * (head + 1)) {    // the head's next tile
      ++tile;
      item_begin = w;
    } else {
      while (w >= base + per_head * p.Hk) {      // the next request with work
        base += per_head * p.Hk;
        r = request_at(p, ++b);
        per_head = Tiling::per_head(p, r);
      }
      head = (int)quotient(w - base, per_head);
      item_begin = base + per_head * head;
      tile = 0;
      for (int n; w >= item_begin + (n = Tiling::steps(p, r, tile)); ++tile) item_begin += n;
    }
    steps = Tiling::steps(p, r, tile);
    s_begin = (int)(w - item_begin);
    s_end = (int)min((long long)steps, w_end - item_begin);
    w = item_begin + s_end;
    return true;
  }
  __device__ bool begins() const { return s_begin == 0; }
  __device__ bool ends() const { return s_end == steps; }
};

// The sum of the requests' work, and, where `c` has a share of it, where that begins (in `start`, shared memory).  The whole block
// calls it; `sums`: shared memory, a word per warp.
template <int kThreads, class Tiling>
__device__ Shares find_share(const AttnParams& p, long long c, long long* sums, Start* start) {
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  long long all = 0, x = 0, n = 0;
  Request r{0, 0, 0, 0};
  auto scan = [&](int b0) {                      // of requests b0 ...: x the sum up to this thread's, n its own; returns that of all
    r = Request{0, 0, 0, 0};
    n = 0;
    if (b0 + tid < p.requests) { r = request_at(p, b0 + tid); n = Tiling::per_head(p, r) * p.Hk; }
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

// The kernel for many queries (cache_attention_chunk.cu); `grid` gets its blocks.
cudaError_t launch_chunk(const AttnParams& p, int d, int type, int sms, cudaStream_t stream, int* grid);

}  // namespace cache
}  // namespace sol

// What the two attention kernels over the 4-bit cache (cache_attention.cu, cache_attention_chunk.cu) share: parameters, the
// division of the work among blocks, and where partial results go.
#pragma once

#include "cache.cuh"

namespace sol {
namespace cache {

struct AttnParams {
  const void* q;
  void* out;
  float* lse;
  long long q_s[2], o_s[2], table_stride;
  const int32_t *cu_q, *kv_lens, *tables;
  const unsigned char* data;
  int tokens, requests, max_blocks, Hq, Hk, group, causal, pages, page_shift;
  float sl2;                                     // logit scale * log2(e) * 2^k_exp
  float v_scale;                                 // 2^v_exp
  int32_t* status;
  long long wait_limit;                          // SM clocks after which a bounded wait gives up
  int withhold;                                  // test hook: >= 0: the arrival for this step of each block is left out
  int4* records;                                 // per block: what it leaves to be combined
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

// Work is counted in steps of kStep keys of one item: kRows rows of one request and key / value head, a row being one query of
// one of the head's `group` query heads.  Items lie one after the other (request, head, rows), and block c of G takes the steps
// [c W / G, (c + 1) W / G): every block has the same share, however ragged the batch, and an item is cut into as many pieces as
// there are blocks on it.  A piece that is not a whole item is left in `parts` and combined by a second kernel, in order.
struct Work {
  int tiles, steps;                              // of a request: row tiles per head, steps per item (at least one)
  __device__ Work(const Request& r, int group, int rows, int step) {
    tiles = (int)(((long long)r.queries * group + rows - 1) / rows);
    steps = max(1, (int)(((long long)r.keys + step - 1) / step));
  }
  __device__ long long items(int heads) const { return (long long)tiles * heads; }
  __device__ long long total(int heads) const { return items(heads) * steps; }
};

__device__ __forceinline__ long long share_begin(long long work, long long blocks, long long c) { return c * work / blocks; }
__device__ __forceinline__ long long owner_of(long long work, long long blocks, long long w) { return ((w + 1) * blocks - 1) / work; }

}  // namespace cache
}  // namespace sol

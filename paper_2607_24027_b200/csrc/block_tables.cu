// Block tables, slots and positions of a step's tokens (sol_attn_block_tables).
//
// Everything follows from two running sums over the requests, of new tokens and of new pages.  Requests are few beside
// tokens, so every block forms both sums for itself and fills the tokens that it owns: one launch, no block waits for
// another.  A page is entered in its request's table by the thread of the first token that it holds; those of tokens behind max_tokens, which
// have no thread, by the first block.
// Bound by latency: lengths, two barriers, the free list.  64 requests with a token each 3.1 us in a graph, 192 with 196 000 tokens 6.2
// (2.8 and 5.5 without the look at the pages that are taken).
#include "cache.cuh"

namespace sol {
namespace {

constexpr int kThreads = 256;
constexpr int kTokensPerBlock = 1024;

struct TablesParams {
  const int32_t *old_lens, *new_lens, *free_pages, *free_count;
  int32_t *tables, *cu_q, *kv_lens, *slots, *positions, *result;
  long long table_stride;
  int requests, max_blocks, max_tokens, free_capacity, page_shift;
};

struct Sum { long long tokens, pages; };
__device__ __forceinline__ Sum operator+(Sum a, Sum b) { return {a.tokens + b.tokens, a.pages + b.pages}; }

// Inclusive sum over the block's threads; `total` gets the block's.
__device__ Sum block_scan(Sum x, Sum* warps, Sum* total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  for (int o = 1; o < 32; o *= 2) {
    const Sum y{__shfl_up_sync(0xffffffffu, x.tokens, o), __shfl_up_sync(0xffffffffu, x.pages, o)};
    if (lane >= o) x = x + y;
  }
  __syncthreads();                               // (the last call's readers)
  if (lane == 31) warps[warp] = x;
  __syncthreads();
  Sum before{0, 0}, all{0, 0};
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before = before + warps[w];
    all = all + warps[w];
  }
  *total = all;
  return before + x;
}

__device__ __forceinline__ int clamp_int(long long x) { return x > 0x7fffffffLL ? 0x7fffffff : (int)x; }

__global__ void __launch_bounds__(kThreads) block_tables_kernel(const TablesParams p) {
  __shared__ Sum warps[kThreads / 32];
  __shared__ long long first[kThreads + 1];      // first token of each request of this round, and one behind
  __shared__ long long page0[kThreads];          // pages taken before it
  __shared__ int old_of[kThreads];
  __shared__ unsigned long long without;
  kernel_wait();
  const int mask = (1 << p.page_shift) - 1;
  const long long lo = (long long)blockIdx.x * kTokensPerBlock;
  const long long hi = min((long long)p.max_tokens, lo + kTokensPerBlock);
  const int count = max(0, min(*p.free_count, p.free_capacity));
  const bool writer = blockIdx.x == 0;           // of what there is one of a request
  if (threadIdx.x == 0) without = 0;
  auto pages_of = [&](long long tokens) { return min((tokens + mask) >> p.page_shift, (long long)p.max_blocks); };
  auto is_page = [&](long long page) { return page >= 0 && page <= 0x7fffffff >> p.page_shift; };      // its slots are of 32 bits
  // The last request of the round whose entry is at most x (one without tokens, or pages, has that of the next).
  auto last_upto = [&](const long long* of, long long x) {
    int a = 0, z = kThreads;
    while (z - a > 1) {
      const int m = (a + z) / 2;
      if (of[m] <= x) a = m; else z = m;
    }
    return a;
  };
  Sum base{0, 0};
  for (int r = 0; r < p.requests; r += kThreads) {
    const int b = r + threadIdx.x;
    const bool on = b < p.requests;
    const int o = on ? max(0, p.old_lens[b]) : 0, n = on ? max(0, p.new_lens[b]) : 0;
    const long long have = pages_of(o), need = pages_of((long long)o + n);
    Sum total;
    const Sum end = base + block_scan(Sum{n, need - have}, warps, &total);
    const long long t0 = end.tokens - n, p0 = end.pages - (need - have);
    first[threadIdx.x] = t0;
    if (threadIdx.x == kThreads - 1) first[kThreads] = end.tokens;
    page0[threadIdx.x] = p0;
    old_of[threadIdx.x] = o;
    if (writer && on) {
      p.cu_q[b] = clamp_int(t0);
      if (b == p.requests - 1) p.cu_q[p.requests] = clamp_int(end.tokens);
      p.kv_lens[b] = clamp_int((long long)o + n);
      // tokens without a slot: those behind max_tokens; of the others those of the page that was begun, if it is no page, and those behind
      // the pages that there were (those of pages taken that are none: below)
      const long long got = max(0LL, min(need - have, (long long)count - p0));
      const long long kept = max(0LL, min((long long)p.max_tokens - t0, (long long)n));
      const long long begun = min(kept, min((have << p.page_shift), (long long)o + n) - o);   // < 0: its table is too short
      long long miss = n - kept + max(0LL, o + kept - max((have + got) << p.page_shift, (long long)o));
      if (begun > 0 && !is_page(p.tables[b * p.table_stride + (o >> p.page_shift)])) miss += begun;
      // Pages of tokens behind max_tokens are taken like any others, and no thread has their first token.
      if (kept < n)
        for (long long j = max(have, (o + kept + mask) >> p.page_shift); j < need; ++j) {
          const long long rank = p0 + j - have;
          p.tables[b * p.table_stride + j] = rank < count ? p.free_pages[count - 1 - rank] : -1;
        }
      if (miss) atomicAdd(&without, (unsigned long long)miss);
    }
    __syncthreads();
    const long long from = max(lo, base.tokens), to = min(hi, base.tokens + total.tokens);
    for (long long t = from + threadIdx.x; t < to; t += kThreads) {
      const int a = last_upto(first, t);
      const long long pos = old_of[a] + (t - first[a]);
      const long long j = pos >> p.page_shift, had = pages_of(old_of[a]);
      long long page = -1;
      if (j < p.max_blocks) {
        int32_t* entry = p.tables + (r + a) * p.table_stride + j;
        if (j < had) {
          page = *entry;
        } else {
          const long long rank = page0[a] + j - had;
          page = rank < count ? p.free_pages[count - 1 - rank] : -1;
          if (!(pos & mask)) *entry = (int32_t)page;
        }
      }
      const long long slot = (page << p.page_shift) + (pos & mask);
      p.slots[t] = is_page(page) ? (int32_t)slot : -1;
      if (p.positions) p.positions[t] = clamp_int(pos);
    }
    if (writer) {                                // pages taken that are none: their tokens have no slot
      const long long pages_end = min((long long)count, base.pages + total.pages);
      constexpr int kAtOnce = 8;
      for (long long rank0 = base.pages + threadIdx.x; rank0 < pages_end; rank0 += kThreads * kAtOnce) {
        int id[kAtOnce];
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) id[x] = rank0 + x * kThreads < pages_end ? p.free_pages[count - 1 - rank0 - x * kThreads] : 0;
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
          if (is_page(id[x])) continue;
          const long long rank = rank0 + x * kThreads;
          const int a = last_upto(page0, rank);
          const long long kept = min((long long)p.max_tokens, first[a + 1]) - first[a];    // (< 0: none of the request's)
          const long long at = ((pages_of(old_of[a]) + rank - page0[a]) << p.page_shift) - old_of[a];
          const long long miss = min(kept, at + mask + 1) - at;
          if (miss > 0) atomicAdd(&without, (unsigned long long)miss);
        }
      }
    }
    base = base + total;
    if (!writer && base.tokens >= hi) break;
    __syncthreads();
  }
  if (writer) {
    __syncthreads();
    if (threadIdx.x == 0) {
      if (p.requests == 0) p.cu_q[0] = 0;
      p.result[0] = (int32_t)max(0LL, count - base.pages);
      p.result[1] = clamp_int((long long)without);
    }
  }
}

int shift_of(int page_size) {
  for (int s = 4; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

}  // namespace
}  // namespace sol

extern "C" sol_status_t sol_attn_block_tables(const sol_attn_tables_args* a) {
  if (!a) return SOL_ERR_INVALID_ARG;
  if (a->requests < 0 || a->max_tokens < 0 || a->max_blocks <= 0 || a->free_capacity < 0) return SOL_ERR_INVALID_ARG;
  if (!a->cu_q || !a->result || !a->free_count || a->result == a->free_count || a->result + 1 == a->free_count) return SOL_ERR_INVALID_ARG;
  // every block reads the inputs for itself, whenever it gets to run: no output may be one of them
  for (const void* out : {(const void*)a->cu_q, (const void*)a->kv_lens, (const void*)a->slots, (const void*)a->positions, (const void*)a->result,
                          (const void*)a->block_tables})
    for (const void* in : {(const void*)a->old_lens, (const void*)a->new_lens, (const void*)a->free_pages, (const void*)a->free_count})
      if (out && out == in) return SOL_ERR_INVALID_ARG;
  if (a->requests > 0 && (!a->old_lens || !a->new_lens || !a->block_tables || !a->kv_lens)) return SOL_ERR_INVALID_ARG;
  if ((a->max_tokens > 0 && !a->slots) || (a->free_capacity > 0 && !a->free_pages)) return SOL_ERR_INVALID_ARG;
  if (a->table_stride < a->max_blocks) return SOL_ERR_INVALID_ARG;
  const int shift = sol::shift_of(a->page_size);
  if (shift < 0) return SOL_ERR_UNSUPPORTED_SHAPE;
  for (const void* p : {(const void*)a->old_lens, (const void*)a->new_lens, (const void*)a->free_pages, (const void*)a->free_count,
                        (const void*)a->block_tables, (const void*)a->cu_q, (const void*)a->kv_lens, (const void*)a->slots,
                        (const void*)a->positions, (const void*)a->result})
    if (!sol::cache::aligned(p, 4)) return SOL_ERR_INVALID_ARG;
  const sol_status_t s = sol::check_device_arch();
  if (s != SOL_OK) return s;
  sol::TablesParams p{a->old_lens, a->new_lens, a->free_pages, a->free_count, a->block_tables, a->cu_q, a->kv_lens, a->slots,
                      a->positions, a->result, a->table_stride, a->requests, a->max_blocks, a->max_tokens, a->free_capacity, shift};
  const int grid = a->max_tokens > 0 ? sol::ceil_div(a->max_tokens, sol::kTokensPerBlock) : 1;
  const cudaError_t e = sol::launch_after(sol::block_tables_kernel, dim3(grid), sol::kThreads, 0, 0, 0,
                                          static_cast<cudaStream_t>(a->stream), p);
  sol::count_launches(1);
  return e == cudaSuccess ? SOL_OK : SOL_ERR_CUDA;
}

// Attention of few queries over the 4-bit cache (sol_attn_cache_attention): single tokens, drafts, short chunks.
//
// Per key and head 9 d / 8 bytes are read for 4 d flops a row, so with few rows HBM is the bound, and next the work of
// widening: at 6.5 TB/s an SM gets 44 numbers a clock.  A warp widens what it read in registers and multiplies with
// m16n8k16 products whose 16-sided operand is the cache: S^T = K Q^T (16 keys x 8 rows), O^T = V^T P^T (16 channels x 8 rows),
// so that a group of up to 8 query heads costs one product, and the cache's layout gives every lane what its operands hold: 16 bytes
// on end of what was copied, no exchange between lanes.
//
// A block is four warps; each takes 32 of the 128 keys of a step with softmax statistics of its own, and the four are joined
// when a piece ends.  The bytes of a step come by one bulk copy (one for each page, if pages are smaller) into a ring,
// kStages - 1 steps ahead; the warps issue them in turn, which costs each a quarter of the instructions.  Every wait is bounded.
//
// One token of 40 heads over 262 143 keys of 8: 65 us, 6.1 TB/s in steady state and 10 us of start and joining; 275 instructions a unit, issue
// slots 60 % busy, ALU 52 %.  With a copy a lane instead of bulk copies 83 us, with one a warp 78.
#include <cmath>
#include <type_traits>

#include "cache_attention.cuh"
#include "fwd_sm100_common.cuh"

namespace sol {
namespace cache {
namespace {

using namespace ptx;

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kWarpKeys = 32, kStep = kWarps * kWarpKeys;
constexpr int kStages = 3;
constexpr unsigned kAll = 0xffffffffu;
constexpr int kBlocksPerSm = 4;
constexpr long long kLanding = 1 << 20;          // SM clocks that a copy is given to land after a wait has run out, however short the limit
constexpr long long kAnyRows = 1LL << 40;
// Requests of up to so many rows (queries times the query heads of a key / value head) are this kernel's.  It takes as long as it has
// tiles of 16 rows, the other as long for 20 as for 128.  us, this kernel / the other: 16 requests of 8192 keys on 8 heads, 20 rows 93 / 144,
// 40 rows 129 / 145, 60 rows 173 / 149; one of 32 768 keys 38 / 48, 48 / 49, 55 / 50; 32 of 2048, d = 64, 30 / 50, 37 / 51, 47 / 52.
constexpr long long kFewRows = 48;

template <int D, int NB>
struct Cfg {
  static constexpr int kRows = 8 * NB;
  static constexpr int kPartFloats = kRows * (D + 2);            // O, then maximum and sum of each row
  static constexpr int kCodeBytes = D / 8;                       // of a lane, unit and half of the keys or values: 16 or 8
  static constexpr int kStageBytes = kStep / kUnit * Unit<D>::kBytes;
  static constexpr int kRing = kStages * kStageBytes;
  static constexpr int kPad = 4;
  static constexpr int kJoin = kWarps * kRows * (D + kPad) * 4;  // reuses the ring
  static constexpr int kSmem = (kRing > kJoin ? kRing : kJoin) + kWarps * kRows * 8;
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same with accumulators that start at zero.
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {     // an 8 x 8 matrix of 16-bit numbers, two of a row per lane
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
struct Shared {
  uint64_t full[kStages], empty[kStages];        // a step has landed; all warps are done with it
  int abort_flag;
  int missing;                                   // a page of this piece is not there
  long long sums[kWarps];
  Start start;
};

template <class T, int D, int NB>
__global__ void __launch_bounds__(kThreads, NB == 1 ? 4 : 3) cache_attention_kernel(const __grid_constant__ AttnParams p) {
  using C = Cfg<D, NB>;
  using U = Unit<D>;
  constexpr int kSteps16 = D / 16;               // products of 16 channels; also 16-channel tiles of the values
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, t = lane % 4;
  float2* stats = reinterpret_cast<float2*>(smem + C::kSmem - kWarps * C::kRows * 8);    // [warp][row]: maximum, sum
  if (tid == 0) {
    sh.abort_flag = sh.missing = 0;
    for (int x = 0; x < kStages; ++x) { mbar_init(&sh.full[x], 1); mbar_init(&sh.empty[x], kWarps); }
    fence_mbar_init();
  }
  __syncthreads();
  kernel_wait();
  kernel_release();                              // (the joining kernel's blocks find room only as this one's leave)

  using Tiling = Tiles<C::kRows, kStep>;
  const Shares shares = find_share<kThreads, Tiling>(p, blockIdx.x, sh.sums, &sh.start);
  if ((long long)blockIdx.x >= shares.blocks) {
    if (tid == 0) p.records[blockIdx.x] = Record::none();
    return;
  }
  Pieces<Tiling> at;
  at.start(p, sh.start, shares.begin(blockIdx.x), shares.begin(blockIdx.x + 1));
  Record record = Record::none();
  bool ok = true;
  uint32_t fetches = 0;                          // steps of earlier pieces

  while (at.next(p)) {
    const Request r = at.r;
    const int head = at.head, tile = at.tile, s_begin = at.s_begin, s_end = at.s_end;
    const int rows = r.queries * p.group;

    // ---- how the steps come in
    const uint32_t page_bytes = (uint32_t)p.Hk * ((uint32_t)U::kBytes << (p.page_shift - 4));
    const unsigned char* head_data = p.data + (size_t)head * ((size_t)U::kBytes << (p.page_shift - 4));
    const int32_t* table = p.tables + at.b * p.table_stride;
    const int units = (r.keys + kUnit - 1) / kUnit;
    auto unit_of = [&](int step, int i) { return step * (kStep / kUnit) + warp * 2 + i; };
    auto page_at = [&](int unit) {               // -1: there is none
      const int page = unit < units ? table[unit >> (p.page_shift - 4)] : -1;
      return page < p.pages ? page : -1;
    };
    // A step is fetched by one warp, the warps in turn: by one copy, or one for each page if pages are smaller, a lane each.
    const int per = min(kStep / kUnit, 1 << (p.page_shift - 4));               // units of a copy
    auto fetch = [&](int step) {
      if (step >= s_end) return;
      const uint32_t n = fetches + (uint32_t)(step - s_begin), s = n % kStages;
      if (n >= kStages && !__all_sync(kAll, mbar_wait(&sh.empty[s], (n / kStages - 1) & 1, &sh.abort_flag, p.wait_limit))) {
        ok = false;
        return;
      }
      uint64_t* bar = &sh.full[s];
      const int u = step * (kStep / kUnit) + lane * per;
      if (lane * per < kStep / kUnit && u < units) {
        const int page = table[u >> (p.page_shift - 4)];
        if (page >= 0 && page < p.pages) {
          const uint32_t in_page = (uint32_t)u & ((1u << (p.page_shift - 4)) - 1);
          const uint32_t bytes = (uint32_t)min(per, units - u) * U::kBytes;
          mbar_expect_tx(bar, bytes);
          bulk_load_1d(smem + s * C::kStageBytes + lane * per * U::kBytes, head_data + (size_t)(uint32_t)page * page_bytes + in_page * U::kBytes,
                       bytes, bar);
        } else {
          sh.missing = 1;
        }
      }
      __syncwarp();
      if (lane == 0 && (int)n != p.withhold) mbar_arrive(bar);                 // (a test withholds it)
    };

    if (warp < kStages - 1) fetch(s_begin + warp);

    // ---- the rows' queries as the products' 8-sided operand, scaled by a power of two per row so that fp16 holds them
    uint32_t qf[NB][kSteps16][2];
    float sl2[NB][2];                            // of rows 2 t and 2 t + 1
    int sees[NB][2];                             // keys that they see
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int row = tile * C::kRows + nb * 8 + g;
      const bool on = row < rows;
      const int qi = row / p.group, hq = head * p.group + row - qi * p.group;
      float x[D / 4], most = 0.f;
      if (on) {
        const T* src = (const T*)p.q + (r.first + qi) * p.q_s[0] + hq * p.q_s[1] + t * (D / 4);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const uint4 raw = reinterpret_cast<const uint4*>(src)[i];
          const uint32_t wd[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) { const float2 f = Two<T>::widen(wd[j]); x[8 * i + 2 * j] = f.x; x[8 * i + 2 * j + 1] = f.y; }
        }
      } else {
#pragma unroll
        for (int i = 0; i < D / 4; ++i) x[i] = 0.f;
      }
      bool finite = true;
#pragma unroll
      for (int i = 0; i < D / 4; ++i) { most = fmaxf(most, fabsf(x[i])); finite = finite && isfinite(x[i]); }
      most = fmaxf(most, __shfl_xor_sync(kAll, most, 1));
      most = fmaxf(most, __shfl_xor_sync(kAll, most, 2));
      finite = ((__ballot_sync(kAll, finite) >> (4 * g)) & 15u) == 15u;
      // the largest becomes 2^14 to 2^15
      const int e = finite && most > 0.f ? (int)((__float_as_uint(most) >> 23) & 255) - 127 : 14;
      const float up = power2(max(-126, min(127, 14 - e)));
#pragma unroll
      for (int s = 0; s < kSteps16; ++s)
#pragma unroll
        for (int j = 0; j < 2; ++j) qf[nb][s][j] = bits(__floats2half2_rn(x[4 * s + 2 * j] * up, x[4 * s + 2 * j + 1] * up));
      const float mine2 = finite ? p.sl2 / up : NAN;             // a row that is not finite gives NaN
      const int seen = !on ? 0 : p.causal ? r.sees(qi) : r.keys;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        sl2[nb][j] = __shfl_sync(kAll, mine2, (2 * t + j) * 4);
        sees[nb][j] = __shfl_sync(kAll, seen, (2 * t + j) * 4);
      }
    }
    int least = 0x7fffffff;                      // keys that all rows see (rows that are not there do not matter)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (tile * C::kRows + nb * 8 + 2 * t + j < rows) least = min(least, sees[nb][j]);
    least = min(least, __shfl_xor_sync(kAll, least, 1));
    least = min(least, __shfl_xor_sync(kAll, least, 2));

    // exponents are x + nm, x the logit times log2(e): nm = kShift - (a maximum of the row's earlier keys)
    float o[NB][kSteps16][4], nm[NB][2], l[NB][2];
    bool seen[NB][2], fresh = true;              // the row has a maximum; some row has none
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int s = 0; s < kSteps16; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nb][s][i] = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) { nm[nb][j] = 0.f; l[nb][j] = 0.f; seen[nb][j] = false; }
    }

    // one step of 2 x 16 keys, all of which all rows see if `Whole`
    auto work_on = [&](int step, const unsigned char* stage, auto whole) {
      constexpr bool kWhole = decltype(whole)::value;
      const int key0 = step * kStep + warp * kWarpKeys;
      int valid[2];
      if constexpr (!kWhole) {
#pragma unroll
        for (int i = 0; i < 2; ++i) valid[i] = page_at(unit_of(step, i)) >= 0 ? min(kUnit, r.keys - key0 - i * kUnit) : 0;
      }
      float y[NB][2][4];
      // S^T of 2 x 16 keys
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned char* unit = stage + i * U::kBytes;
        uint32_t code[2][D / 32];                // rows g and g + 8, D / 4 channels each
        __half2 sc[2][D / 64];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const unsigned char* src = unit + U::kKeys + (h * 32 + lane) * C::kCodeBytes;
          if constexpr (D == 128) *reinterpret_cast<uint4*>(code[h]) = *reinterpret_cast<const uint4*>(src);
          else *reinterpret_cast<uint2*>(code[h]) = *reinterpret_cast<const uint2*>(src);
        }
        if constexpr (D == 128) {
          const uint32_t x = *reinterpret_cast<const uint32_t*>(unit + U::kKeyScales + lane * 4);
          const __half2 a = scales2(x & 0xffff), c = scales2(x >> 16);
          sc[0][0] = __low2half2(a); sc[0][1] = __high2half2(a); sc[1][0] = __low2half2(c); sc[1][1] = __high2half2(c);
        } else {
          const __half2 a = scales2(*reinterpret_cast<const uint16_t*>(unit + U::kKeyScales + lane * 2));
          sc[0][0] = __low2half2(a); sc[1][0] = __high2half2(a);
        }
#pragma unroll
        for (int w4 = 0; w4 < D / 32; ++w4) {    // channels 8 w4 ... of the lane's D / 4: two products
          uint32_t a[2][4];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            codes8(code[h][w4], a[h]);
#pragma unroll
            for (int x = 0; x < 4; ++x) a[h][x] = bits(__hmul2(half2_of(a[h][x]), sc[h][w4 / 2]));
          }
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint32_t q0 = qf[nb][2 * w4 + x][0], q1 = qf[nb][2 * w4 + x][1];
              if (w4 == 0 && x == 0) mma_first(y[nb][i], a[0][0], a[1][0], a[0][1], a[1][1], q0, q1);
              else mma(y[nb][i], a[0][2 * x], a[1][2 * x], a[0][2 * x + 1], a[1][2 * x + 1], q0, q1);
            }
        }
      }
      // Exponents.  A lane looks at its own four keys of a row, and only if one of the warp's is over the limit are maxima taken.
      bool over = false;
      float mx[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          mx[nb][j] = -INFINITY;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float& x = y[nb][i][2 * h + j];
              x = fmaf(x, sl2[nb][j], nm[nb][j]);
              if constexpr (!kWhole)
                if (g + 8 * h >= valid[i] || key0 + i * kUnit + g + 8 * h >= sees[nb][j]) x = -INFINITY;
              mx[nb][j] = fmaxf(mx[nb][j], x);
            }
          over = over || mx[nb][j] > kMost;
        }
      if (__any_sync(kAll, over) || fresh) {
        fresh = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float top = mx[nb][j];
            top = fmaxf(top, __shfl_xor_sync(kAll, top, 4));
            top = fmaxf(top, __shfl_xor_sync(kAll, top, 8));
            top = fmaxf(top, __shfl_xor_sync(kAll, top, 16));
            // the largest exponent becomes kShift, if it was above (or is the row's first)
            const float by = top == -INFINITY ? 0.f : seen[nb][j] ? fmaxf(0.f, top - kShift) : top - kShift;
            const float f = seen[nb][j] ? ex2(-by) : 1.f;        // (nothing is there yet)
            seen[nb][j] = seen[nb][j] || top != -INFINITY;
            fresh = fresh || !seen[nb][j];
            nm[nb][j] -= by;
            l[nb][j] *= f;
#pragma unroll
            for (int s = 0; s < kSteps16; ++s) { o[nb][s][j] *= f; o[nb][s][2 + j] *= f; }
#pragma unroll
            for (int i = 0; i < 2; ++i) { y[nb][i][j] -= by; y[nb][i][2 + j] -= by; }
          }
        fresh = __any_sync(kAll, fresh);
      }
      // weights, and as the second product's 8-sided operand
      uint32_t pf[NB][2][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float e0 = ex2(y[nb][i][2 * h]), e1 = ex2(y[nb][i][2 * h + 1]);
            l[nb][0] += e0;
            l[nb][1] += e1;
            pf[nb][i][h] = transpose8(bits(__floats2half2_rn(e0, e1)));
          }
      // O^T += V^T P^T
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned char* unit = stage + i * U::kBytes;
        uint32_t vs = *reinterpret_cast<const uint32_t*>(unit + U::kValueScales + ((D == 128 ? g : g / 2) * 4 + t) * 4);
        if constexpr (!kWhole) {                 // what no row may see is multiplied by zero
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (2 * t + (x & 1) + 8 * (x >> 1) >= valid[i]) vs &= ~(0xffu << (8 * x));
        }
        const __half2 sc[2] = {scales2(vs & 0xffff), scales2(vs >> 16)};
        uint32_t a[2][D / 64], c[2][D / 64];     // tokens 8 h + 2 t and + 1, D / 8 channels each
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const unsigned char* src = unit + U::kValues + (h * 32 + lane) * C::kCodeBytes;
          if constexpr (D == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(src);
            a[h][0] = x.x; a[h][1] = x.y; c[h][0] = x.z; c[h][1] = x.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(src);
            a[h][0] = x.x; c[h][0] = x.y;
          }
        }
#pragma unroll
        for (int w4 = 0; w4 < D / 64; ++w4) {    // channels g d / 8 + 8 w4 ...: four tiles of 16
          uint32_t v[2][2][4];                   // half, odd channel: two tokens each
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t x = a[h][w4], z = c[h][w4];
            codes8((x & 0x0f0f0f0fu) | ((z << 4) & 0xf0f0f0f0u), v[h][0]);
            codes8(((x >> 4) & 0x0f0f0f0fu) | (z & 0xf0f0f0f0u), v[h][1]);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[h][q / 4][q % 4] = bits(__hmul2(half2_of(v[h][q / 4][q % 4]), sc[h]));
          }
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              mma(o[nb][4 * w4 + q], v[0][0][q], v[0][1][q], v[1][0][q], v[1][1][q], pf[nb][i][0], pf[nb][i][1]);
        }
      }
    };

    uint32_t n = fetches;
    for (int step = s_begin; ok && step < s_end; ++step, ++n) {
      const uint32_t s = n % kStages;
      if (!__all_sync(kAll, mbar_wait(&sh.full[s], (n / kStages) & 1, &sh.abort_flag, p.wait_limit))) { ok = false; break; }
      const unsigned char* stage = smem + s * C::kStageBytes + warp * 2 * U::kBytes;
      const int key0 = step * kStep + warp * kWarpKeys;
      // (a vote: another warp may be setting the word, and what follows is for whole warps)
      const bool missing = __any_sync(kAll, *(volatile int*)&sh.missing != 0);
      if (key0 + kWarpKeys <= least && !missing) work_on(step, stage, std::true_type{});
      else if (key0 < r.keys) work_on(step, stage, std::false_type{});
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.empty[s]);
      // (into the place of the step before this one, which the other warps are done with by now or soon)
      if ((step - s_begin) % kWarps == warp) fetch(step + kStages - 1);
    }
    if (!ok && lane == 0) {
      sh.abort_flag = 1;
      atomicExch(p.status, (int)SOL_ERR_DEVICE_TIMEOUT);
    }
    __syncthreads();
    if (sh.abort_flag) {                         // a wait ran out: no result, but no copy is left in flight either
      int never = 0;
      if (!ok)
        for (uint32_t x = n; x < n + kStages; ++x) mbar_wait(&sh.full[x % kStages], (x / kStages) & 1, &never, max(p.wait_limit, kLanding));
      if (tid == 0) p.records[blockIdx.x] = Record::none();
      return;
    }
    fetches += (uint32_t)(s_end - s_begin);

    // ---- the four warps' results into one
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float x = l[nb][j];
        x += __shfl_xor_sync(kAll, x, 4);
        x += __shfl_xor_sync(kAll, x, 8);
        x += __shfl_xor_sync(kAll, x, 16);
        if (g == 0) stats[warp * C::kRows + nb * 8 + 2 * t + j] = make_float2(seen[nb][j] ? kShift - nm[nb][j] : -INFINITY, x);
      }
    __syncthreads();                             // (and every warp is done with its ring)
    float* join = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = nb * 8 + 2 * t + j;
        float top = -INFINITY;
        for (int x = 0; x < kWarps; ++x) top = fmaxf(top, stats[x * C::kRows + row].x);
        const float f = top == -INFINITY ? 1.f : seen[nb][j] ? ex2(kShift - nm[nb][j] - top) : 0.f;
        float* dst = join + (warp * C::kRows + row) * (D + C::kPad) + g * (D / 8);
#pragma unroll
        for (int s = 0; s < kSteps16; ++s)
          *reinterpret_cast<float2*>(dst + 2 * s) = make_float2(o[nb][s][j] * f, o[nb][s][2 + j] * f);
      }
    __syncthreads();
    const bool begins = at.begins(), ends = at.ends();
    float* part = p.parts + (size_t)(2 * blockIdx.x + (begins ? 1 : 0)) * C::kPartFloats;
    for (int x = tid; x < C::kRows * D; x += kThreads) {
      const int row = x / D, ch = x - row * D;
      float top = -INFINITY, sum = 0.f, acc = 0.f;
      for (int y = 0; y < kWarps; ++y) top = fmaxf(top, stats[y * C::kRows + row].x);
      for (int y = 0; y < kWarps; ++y) {
        const float2 st = stats[y * C::kRows + row];
        sum += st.y * (top == -INFINITY ? 1.f : ex2(st.x - top));
        acc += join[(y * C::kRows + row) * (D + C::kPad) + ch];
      }
      if (begins && ends) {
        const int full = tile * C::kRows + row;
        if (full < rows) {
          const int qi = full / p.group, hq = head * p.group + full - qi * p.group;
          const float y = sum == 0.f ? 0.f : acc / sum * p.v_scale;
          T* dst = (T*)p.out + (r.first + qi) * p.o_s[0] + hq * p.o_s[1];
          dst[ch] = T(y);
          if (p.lse && ch == 0)
            p.lse[(size_t)(r.first + qi) * p.Hq + hq] = sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + log2f(sum) - kShift) * kLn2;
        }
      } else {
        part[x] = acc;
        if (ch == 0) { part[C::kRows * D + row] = top; part[C::kRows * (D + 1) + row] = sum; }
      }
    }
    if (!begins && ends)                         // the last piece of a cut item: this block's record has it combined
      record = Record{(int)shares.owner(at.item_begin) | head << 16, tile, r.queries, r.first};
    if (tid == 0) sh.missing = 0;
    fence_proxy_async_smem();                    // the next copies go where the warps' results were
    __syncthreads();
  }
  if (tid == 0) p.records[blockIdx.x] = record;
}

// Joins the pieces of the items that several blocks had: of a kernel's blocks, block c had the last piece, blocks from record.from() to c - 1
// the others.  The block that had the first piece left it in its second place, the rest in their first.  A row is added up
// by as many warps as it takes for each to have kAtOnce pieces, up to 16, four channels (two, d = 64) to a lane.
// What bounds this kernel is the way to memory and back, so there are two on its longest path, the records and then the pieces, and
// registers are kept few, for many rows at once.  One launch joins what both attention kernels left.
struct Left {                                    // by a kernel
  const Record* records;
  const float* parts;
  int blocks, rows;                              // rows of an item
};
constexpr int kJoinWarps = 16;
// Pieces of an item up to which join_wide takes the many-row kernel's.  us of a call whose 148 blocks share out items of 256 rows, wide / long, d = 64 and
// 128: 2 pieces 22.6 / 28.4 and 30.4 / 34.6, 4 to 5 23.5 / 24.7 and 29.5 / 31.0, 10 24.5 / 29.8 and 30.8 / 35.5, 13 to 14 25.0 / 27.8 and 31.0 / 33.9,
// 17 to 18 26.6 / 25.5 and 33.4 / 31.5, 37 31.6 / 25.3 and 38.2 / 31.5.
constexpr int kFewPieces = 14;
struct JoinShared {
  float joined[kJoinWarps][128 + 2];
  int counts[kJoinWarps], spans[kJoinWarps];
  Record list[kMostBlocks];
  short last_of[kMostBlocks];
};

// The records with an item, packed: {their number, the most pieces of one}.
__device__ __forceinline__ int2 pack_records(const Left& left, JoinShared& sh) {
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, blocks = left.blocks;
  int n = 0, most_pieces = 0;
  for (int c0 = 0; c0 < blocks; c0 += 32 * kJoinWarps) {
    const int c = c0 + tid;
    Record rec = Record::none();
    if (c < blocks) rec = left.records[c];
    const unsigned some = __ballot_sync(kAll, rec.is());
    const int span = __reduce_max_sync(kAll, rec.is() ? c - rec.from() + 1 : 0);
    __syncthreads();                             // (the last pass's readers)
    if (lane == 0) { sh.counts[warp] = __popc(some); sh.spans[warp] = span; }
    __syncthreads();
    int upto = lane < kJoinWarps ? sh.counts[lane] : 0;          // of warps up to this lane's
    most_pieces = max(most_pieces, __reduce_max_sync(kAll, lane < kJoinWarps ? sh.spans[lane] : 0));
#pragma unroll
    for (int o = 1; o < kJoinWarps; o *= 2) {
      const int y = __shfl_up_sync(kAll, upto, o);
      if (lane >= o) upto += y;
    }
    const int before = __shfl_sync(kAll, upto, (warp + 31) % 32), total = __shfl_sync(kAll, upto, kJoinWarps - 1);
    if (rec.is()) {
      const int k = n + (warp ? before : 0) + __popc(some & ((1u << lane) - 1));
      sh.list[k] = rec;
      sh.last_of[k] = (short)c;
    }
    n += total;
  }
  __syncthreads();
  return make_int2(n, most_pieces);
}

// Where a row of an item belongs, and what becomes of it: acc[kCh] are its channels from `ch`.
template <class T, int kCh>
__device__ __forceinline__ void put_row(const AttnParams& p, const Record& rec, int full, int ch, const float (&acc)[kCh], float sum, float top) {
  const int qi = full / p.group, hq = rec.head() * p.group + full - qi * p.group;
  const long long token = rec.first + qi;
  T* dst = (T*)p.out + token * p.o_s[0] + hq * p.o_s[1] + ch;
  const float inv = sum == 0.f ? 0.f : p.v_scale / sum;
  uint32_t w[kCh / 2];
#pragma unroll
  for (int i = 0; i < kCh / 2; ++i) w[i] = sum == 0.f ? 0u : Two<T>::round(acc[2 * i] * inv, acc[2 * i + 1] * inv);
  if constexpr (kCh == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  else if constexpr (kCh == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(dst) = w[0];
  if (p.lse && ch == 0)
    p.lse[token * p.Hq + hq] = sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + log2f(sum) - kShift) * kLn2;
}

template <int kCh>
__device__ __forceinline__ void load_channels(float (&a)[kCh], const float* src) {
  if constexpr (kCh == 8) {
    *reinterpret_cast<float4*>(a) = reinterpret_cast<const float4*>(src)[0];
    *reinterpret_cast<float4*>(a + 4) = reinterpret_cast<const float4*>(src)[1];
  } else if constexpr (kCh == 4) {
    *reinterpret_cast<float4*>(a) = *reinterpret_cast<const float4*>(src);
  } else {
    *reinterpret_cast<float2*>(a) = *reinterpret_cast<const float2*>(src);
  }
}

// acc, sum and top of a row's pieces x0, x0 + every, ... up to `last`, kAtOnce of them on their way together.
template <int D, int kCh, int kAtOnce>
__device__ __forceinline__ void add_pieces(const Left& left, int from, int last, int x0, int every, int row, int ch, float (&acc)[kCh], float& sum,
                                           float& top) {
  const int rows = left.rows;
  for (; x0 <= last; x0 += every * kAtOnce) {
    float m[kAtOnce], l[kAtOnce], a[kAtOnce][kCh], most = top;
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) {
      const int x = min(x0 + y * every, last);   // (what is too much is read and not used)
      const float* part = left.parts + (size_t)(2 * x + (x == from ? 1 : 0)) * (rows * (D + 2));
      m[y] = part[rows * D + row];
      l[y] = part[rows * (D + 1) + row];
      load_channels(a[y], part + row * D + ch);
    }
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y)
      if (x0 + y * every <= last) most = fmaxf(most, m[y]);
    const float f0 = top == -INFINITY ? 1.f : ex2(top - most);                 // (then acc and sum are 0 or NaN)
#pragma unroll
    for (int i = 0; i < kCh; ++i) acc[i] *= f0;
    sum *= f0;
    top = most;
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) {
      if (x0 + y * every > last) continue;
      const float f = m[y] == -INFINITY ? 1.f : ex2(m[y] - most);              // (a piece without a maximum holds 0 or NaN)
#pragma unroll
      for (int i = 0; i < kCh; ++i) acc[i] += a[y][i] * f;
      sum += l[y] * f;
    }
  }
}

// Rows with many pieces: as many warps to a row as it takes for each to have kAtOnce, up to 16.
template <class T, int D>
__device__ __forceinline__ void join_long(const AttnParams& p, const Left& left, JoinShared& sh, int n, int most_pieces) {
  constexpr int kCh = D / 32, kAtOnce = 5;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rows = left.rows;
  int share = 1;
  while (share < kJoinWarps && share * kAtOnce < most_pieces) share *= 2;
  const int rows_at_once = kJoinWarps / share, tasks = n * rows, part0 = warp % share;
  for (int t0 = blockIdx.x * rows_at_once; t0 < tasks; t0 += gridDim.x * rows_at_once) {
    const int task = t0 + warp / share;
    const bool is = task < tasks;
    const int item = is ? task / rows : 0, row = task - item * rows;
    const Record& rec = sh.list[item];
    const int last = sh.last_of[item], full = rec.tile * rows + row;
    const bool on = is && full < rec.queries * p.group;
    float top = -INFINITY, sum = 0.f, acc[kCh];
#pragma unroll
    for (int i = 0; i < kCh; ++i) acc[i] = 0.f;
    if (on) add_pieces<D, kCh, kAtOnce>(left, rec.from(), last, rec.from() + part0, share, row, lane * kCh, acc, sum, top);
    if (share > 1) {
      __syncthreads();                           // (the last pass's readers)
#pragma unroll
      for (int i = 0; i < kCh; ++i) sh.joined[warp][lane * kCh + i] = acc[i];
      if (lane == 0) { sh.joined[warp][D] = sum; sh.joined[warp][D + 1] = top; }
      __syncthreads();
      if (part0 > 0) continue;
      top = lane < share ? sh.joined[warp + lane][D + 1] : -INFINITY;
#pragma unroll
      for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(kAll, top, o));
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < kCh; ++i) acc[i] = 0.f;
      for (int y = warp; y < warp + share; ++y) {
        const float m = sh.joined[y][D + 1], f = m == -INFINITY ? 1.f : ex2(m - top);
        sum += sh.joined[y][D] * f;
#pragma unroll
        for (int i = 0; i < kCh; ++i) acc[i] += sh.joined[y][lane * kCh + i] * f;
      }
    }
    if (on) put_row<T>(p, rec, full, lane * kCh, acc, sum, top);
  }
}

// Many rows with few pieces: 256 / d rows to a warp, eight channels to a lane, since what a row takes beside its channels is what bounds
// this (one row to a warp: 286 instructions a row, 19 us for 148 items of 256 rows and 64 channels).
template <class T, int D>
__device__ __forceinline__ void join_wide(const AttnParams& p, const Left& left, const JoinShared& sh, int n) {
  constexpr int kLanes = D / 8, kRowsOfWarp = 32 / kLanes;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rows = left.rows, tasks = n * rows;
  const int every = gridDim.x * kJoinWarps * kRowsOfWarp;
  for (int task = (blockIdx.x * kJoinWarps + warp) * kRowsOfWarp + lane / kLanes; task < tasks; task += every) {
    const int item = task / rows, row = task - item * rows;
    const Record& rec = sh.list[item];
    const int full = rec.tile * rows + row, ch = lane % kLanes * 8;
    if (full >= rec.queries * p.group) continue;
    float top = -INFINITY, sum = 0.f, acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    add_pieces<D, 8, 3>(left, rec.from(), sh.last_of[item], rec.from(), 1, row, ch, acc, sum, top);
    put_row<T>(p, rec, full, ch, acc, sum, top);
  }
}

template <class T, int D>
__global__ void __launch_bounds__(32 * kJoinWarps, 2) cache_combine_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ Left few,
                                                                           const __grid_constant__ Left many) {
  __shared__ JoinShared sh;
  kernel_wait();
#pragma unroll 1
  for (int kernel = 0; kernel < 2; ++kernel) {
    const Left& left = kernel ? many : few;
    if (left.blocks == 0) continue;
    const int2 found = pack_records(left, sh);
    if (kernel && found.y <= kFewPieces) join_wide<T, D>(p, left, sh, found.x);
    else join_long<T, D>(p, left, sh, found.x, found.y);
  }
}

// The workspace: status word, then for each of the two kernels a record per block and two partial results per block.
struct Layout {
  size_t few_records, few_parts, many_records, many_parts, total;
  Layout(long long rows, int d) {
    size_t at = 1024;
    auto take = [&](size_t bytes) { const size_t o = at; at = align_up(at + bytes, 1024); return o; };
    few_records = take(kMostBlocks * sizeof(Record));
    few_parts = take(2 * kMostBlocks * (rows <= 8 ? 8 : 16) * (size_t)(d + 2) * sizeof(float));
    many_records = take(rows <= kFewRows ? 0 : kMostChunkBlocks * sizeof(Record));
    many_parts = take(rows <= kFewRows ? 0 : 2 * kMostChunkBlocks * kChunkRows * (size_t)(d + 2) * sizeof(float));
    total = at;
  }
};

template <class T, int D, int NB>
cudaError_t run_few(AttnParams p, long long rows_to, int sms, cudaStream_t stream, Left* left, int* n) {
  using C = Cfg<D, NB>;
  p.rows_from = 0;
  p.rows_to = rows_to;
  int grid = (NB == 1 ? kBlocksPerSm : kBlocksPerSm - 1) * sms;
  if (grid > kMostBlocks) grid = kMostBlocks;
  *left = Left{p.records, p.parts, grid, C::kRows};
  ++*n;
  return launch_after(cache_attention_kernel<T, D, NB>, dim3(grid), kThreads, C::kSmem, C::kSmem, 0, stream, p);
}

template <class T, int D>
cudaError_t run(AttnParams p, char* ws, int max_q, int type, int sms, cudaStream_t stream, int* n) {
  const long long rows = (long long)max_q * p.group;
  const Layout lay(rows, D);
  p.records = reinterpret_cast<Record*>(ws + lay.few_records);
  p.parts = reinterpret_cast<float*>(ws + lay.few_parts);
  Left few{}, many{};
  cudaError_t e = cudaSuccess;
  // With several requests and long ones among them there may be some of either kind.
  const bool split = rows > kFewRows && p.requests > 1;
  if (rows <= 8) e = run_few<T, D, 1>(p, kAnyRows, sms, stream, &few, n);
  else if (rows <= kFewRows || split) e = run_few<T, D, 2>(p, split ? kFewRows : kAnyRows, sms, stream, &few, n);
  if (e != cudaSuccess) return e;
  if (rows > kFewRows) {
    AttnParams q = p;
    q.records = reinterpret_cast<Record*>(ws + lay.many_records);
    q.parts = reinterpret_cast<float*>(ws + lay.many_parts);
    q.rows_from = split ? kFewRows + 1 : 0;
    q.rows_to = kAnyRows;
    many = Left{q.records, q.parts, 0, kChunkRows};
    ++*n;
    e = launch_chunk(q, D, type, sms, stream, &many.blocks);
    if (e != cudaSuccess) return e;
  }
  ++*n;
  return launch_after(cache_combine_kernel<T, D>, dim3(2 * sms), 32 * kJoinWarps, 0, 0, 0, stream, p, few, many);
}

sol_status_t check_attention(const sol_attn_cache_args* a) {
  if (!a) return SOL_ERR_INVALID_ARG;
  sol_status_t s = check(&a->cache);
  if (s != SOL_OK) return s;
  if (a->tokens < 0 || a->requests < 0 || a->max_q < (a->tokens > 0 ? 1 : 0) || a->max_blocks <= 0 || a->Hq <= 0) return SOL_ERR_INVALID_ARG;
  if (a->type != SOL_TYPE_BF16 && a->type != SOL_TYPE_FP16) return SOL_ERR_INVALID_ARG;
  if (std::isnan(a->scale) || std::isinf(a->scale) || a->table_stride < a->max_blocks) return SOL_ERR_INVALID_ARG;
  if (a->Hq > kMaxHeads || a->Hq % a->cache.Hk) return SOL_ERR_UNSUPPORTED_SHAPE;
  if ((long long)a->tokens * (a->Hq / a->cache.Hk) > 0x7fffffffLL) return SOL_ERR_UNSUPPORTED_SHAPE;
  if (a->tokens > 0 && a->q == a->out) return SOL_ERR_INVALID_ARG;             // several blocks read a row's queries
  if (a->tokens > 0 && (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16))) return SOL_ERR_INVALID_ARG;
  if (!strides_ok(a->q_stride, a->tokens, a->Hq) || !strides_ok(a->out_stride, a->tokens, a->Hq) || !aligned(a->lse, 4)) return SOL_ERR_INVALID_ARG;
  if (!rows_apart(a->out_stride, a->tokens, a->Hq)) return SOL_ERR_INVALID_ARG;
  if (a->requests > 0 && (!a->cu_q || !a->kv_lens || !a->block_tables)) return SOL_ERR_INVALID_ARG;
  if (!aligned(a->cu_q, 4) || !aligned(a->kv_lens, 4) || !aligned(a->block_tables, 4)) return SOL_ERR_INVALID_ARG;
  const size_t need = sol_attn_cache_workspace_bytes(a->max_q > 0 ? a->max_q : 1, a->Hq, a->cache.Hk, a->cache.d);
  if (!a->workspace || !aligned(a->workspace, 1024) || a->workspace_bytes < need) return SOL_ERR_WORKSPACE;
  return SOL_OK;
}

}  // namespace
}  // namespace cache
}  // namespace sol

extern "C" {

size_t sol_attn_cache_workspace_bytes(int max_q, int Hq, int Hk, int d) {
  if (max_q <= 0 || Hq <= 0 || Hk <= 0 || Hq > sol::cache::kMaxHeads || Hq % Hk || (d != 64 && d != 128)) return 0;
  const long long rows = (long long)max_q * (Hq / Hk);
  return sol::cache::Layout(rows, d).total;
}

sol_status_t sol_attn_cache_attention(const sol_attn_cache_args* a) {
  using namespace sol;
  sol_status_t s = cache::check_attention(a);
  if (s != SOL_OK) return s;
  if (a->tokens == 0 || a->requests == 0) return SOL_OK;
  if ((s = check_device_arch()) != SOL_OK) return s;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return SOL_ERR_CUDA;
  cache::AttnParams p{};
  p.q = a->q; p.out = a->out; p.lse = a->lse;
  for (int i = 0; i < 2; ++i) { p.q_s[i] = a->q_stride[i]; p.o_s[i] = a->out_stride[i]; }
  p.table_stride = a->table_stride;
  p.cu_q = a->cu_q; p.kv_lens = a->kv_lens; p.tables = a->block_tables;
  p.data = static_cast<const unsigned char*>(a->cache.data);
  p.tokens = a->tokens; p.requests = a->requests; p.max_blocks = a->max_blocks;
  p.Hq = a->Hq; p.Hk = a->cache.Hk; p.group = a->Hq / a->cache.Hk; p.causal = a->causal != 0; p.pages = a->cache.pages;
  p.page_shift = cache::page_shift(a->cache.page_size);
  const float scale = a->scale > 0.f ? a->scale : 1.0f / std::sqrt((float)a->cache.d);
  p.sl2 = std::ldexp(scale * 1.4426950408889634f, a->cache.k_exp);
  p.v_scale = std::ldexp(1.0f, a->cache.v_exp);
  char* ws = static_cast<char*>(a->workspace);
  p.wait_limit = fwd::g_wait_limit;
  p.withhold = fwd::g_withhold_tile;
  p.status = reinterpret_cast<int32_t*>(ws);
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  int n = 0;
  auto typed = [&](auto zero) {
    using T = decltype(zero);
    return a->cache.d == 128 ? cache::run<T, 128>(p, ws, a->max_q, a->type, sms, stream, &n)
                             : cache::run<T, 64>(p, ws, a->max_q, a->type, sms, stream, &n);
  };
  const cudaError_t e = a->type == SOL_TYPE_BF16 ? typed(__nv_bfloat16{}) : typed(__half{});
  count_launches(n);
  return e == cudaSuccess ? SOL_OK : SOL_ERR_CUDA;
}

sol_status_t sol_attn_cache_read_status(void* workspace, sol_stream_t stream) {
  if (!workspace) return SOL_ERR_WORKSPACE;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t word = 0;
  if (cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, st) != cudaSuccess) return SOL_ERR_CUDA;
  if (cudaMemsetAsync(workspace, 0, sizeof(word), st) != cudaSuccess) return SOL_ERR_CUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return SOL_ERR_CUDA;
  return word;
}

}  // extern "C"

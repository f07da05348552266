// Attention of many queries over the 4-bit cache (sol_attn_cache_attention): prompts, chunks of a video.  What the tensor core multiplies is
// not in memory, so tiled TMA loads have nothing to bring: bulk copies bring the cache's units, and warps widen them into the tiles.
//
// A row is one query of one of the query heads that share a key / value head.  A block has two tiles of 128 rows, so that what is widened
// once is multiplied by 256 rows, and the two tiles take turns on the tensor core and the special-function units as in
// fwd_sm100_dense.cu: one warp issues
//   P V (A, t)  Q K^T (A, t + 1)  |  P V (B, t)  Q K^T (B, t + 1)  |  ...
//   softmax  (warps 0-3: tile A, 4-7: tile B) thread = row, with all 128 scores of a tile of keys in registers; at the start of a piece it
//            puts the row's queries into shared memory, scaled by a power of two so that fp16 holds them
//   mma      (warp 8)
//   loader   (warp 9) the cache's units of 16 tokens into a ring of 14
//   widen    (warps 10-15) units to fp16 tiles in a ring of four slots, K0 V0 K1 V1 ..., in the 128-byte swizzle that the tensor core reads
// The cache's values are exact in fp16, so K and V enter the products unrounded.
// 37 heads x 1024 queries x 32 768 keys, d = 128: 545 us, 1165 TFLOP/s; a step of 256 rows x 128 keys 2.13 us (d = 64 1.78), about what
// fwd_sm100_dense.cu takes with tiles that TMA brings: one tile's softmax, P V and Q K^T follow one another.  Tensor pipe 49 % busy.
//
// TMEM: S_A [0, 128)  S_B [128, 256)  O_A [256, 256 + d)  O_B [256 + d, 256 + 2 d).  Every wait is bounded.
#include <atomic>

#include "cache_attention.cuh"
#include "fwd_sm100_common.cuh"

namespace sol {
namespace cache {
namespace {

using namespace ptx;
using fwd::desc_from_lo;
using fwd::kTmemCols;
using fwd::tmem_ld_cols;

constexpr int kThreads = 512;
constexpr int kTileRows = 128, kRows = kChunkRows, kCols = 128;   // of a tile, of a block; keys of a step
constexpr int kUnits = kCols / kUnit;
constexpr int kSlots = 4;
constexpr int kWarpMma = 8, kWarpLoader = 9, kWarpWiden = 10, kWideners = 6;
constexpr int kRaw = 14;                         // units in the raw ring
constexpr int kTmemS = 0, kTmemO = 256;
constexpr int kRegsSoftmax = 200, kRegsOther = 56, kRegsLaunch = 128;   // registers per thread of the roles, and at launch
static_assert(8 * kRegsSoftmax + 8 * kRegsOther <= 16 * kRegsLaunch, "a warpgroup would wait for registers without end");
constexpr unsigned kAll = 0xffffffffu;

using Tiling = Tiles<kRows, kCols>;

template <int D>
struct Cfg {
  static constexpr int kTileBytes = kCols * D * 2;         // a query, K or V tile
  static constexpr int kBoxBytes = kCols * 128;            // 64 channels of it
  static constexpr int kPartFloats = kRows * (D + 2);
  static constexpr size_t kSmem = 1024 + (2 + kSlots) * kTileBytes + kRaw * Unit<D>::kBytes;
};

struct Shared {
  uint64_t q_full[2], q_empty[2];                // per row tile
  uint64_t kv_full[kSlots], kv_empty[kSlots];
  uint64_t raw_full[kRaw], raw_empty[kRaw];      // a unit's bytes are there; its keys and its values are widened
  int raw_valid[kRaw];                           // tokens of it that there are
  uint64_t s_full[2];                            // scores of a tile are in TMEM
  uint64_t p_full[2][2];                         // first / second half of the columns of P are in TMEM
  uint64_t o_full[2], o_free[2];                 // accumulator complete / read
  uint64_t mma_drain;                            // everything that was issued is done
  long long sums[kThreads / 32];
  Start start;
  Pieces<Tiling> pieces[kThreads / 32];          // each warp's place in the block's share: registers are scarce
  uint32_t tmem_base;
  int abort_flag;
  int missing;                                   // a page was not there: from now on softmax looks for itself
};

static_assert(Cfg<128>::kSmem + sizeof(Shared) <= 227 * 1024, "shared memory of a block");

#define WAIT(bar, parity) mbar_wait_inline((bar), (parity), &sm.abort_flag, p.wait_limit)
#define WAIT_ALL(bar, parity) __all_sync(kAll, WAIT(bar, parity))
// (out of line, for the roles that have the registers for a call)
#define WAIT_CALL(bar, parity) mbar_wait((bar), (parity), &sm.abort_flag, p.wait_limit)
#define WAIT_CALL_ALL(bar, parity) __all_sync(kAll, WAIT_CALL(bar, parity))

__device__ __forceinline__ void flag_timeout(Shared& sm, const AttnParams& p) {
  sm.abort_flag = 1;
  atomicExch(p.status, (int)SOL_ERR_DEVICE_TIMEOUT);
}

// Instruction descriptor for kind::f16 with fp16 A / B and fp32 accumulation (see make_idesc_bf16).
__host__ __device__ constexpr uint32_t make_idesc_f16(int M, int N, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Maximum of three; if kNaN, NaN if one is.
template <bool kNaN>
__device__ __forceinline__ float max3(float a, float b, float c) {
  if constexpr (!kNaN) return fmaxf(fmaxf(a, b), c);
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// 2^x of two numbers up to 2^7 on the FMA pipe: x = n + f with n the nearest integer (x plus 1.5 * 2^23 rounds there), 2^f by the polynomial of
// degree 5 with constant 1 whose largest relative error on [-1/2, 1/2] is least, rounded to fp32 (1.1e-7; 1.7e-7 with the steps' roundings, as
// good as the instruction: this goes into lse too.  Degree 4 is off by 2.6e-6), n added to the exponent.
// Below -126 it is 2^-126.  Not for NaN.
__device__ __forceinline__ float2 exp2_fma(float2 x) {
  x = make_float2(fmaxf(x.x, -126.f), fmaxf(x.y, -126.f));
  const float2 magic = make_float2(12582912.f, 12582912.f), minus = make_float2(-12582912.f, -12582912.f);
  const float2 t = __fadd2_rn(x, magic), n = __fadd2_rn(t, minus);
  const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
  float2 q = make_float2(0.00132647285f, 0.00132647285f);
  q = __ffma2_rn(q, f, make_float2(0.00967151299f, 0.00967151299f));
  q = __ffma2_rn(q, f, make_float2(0.0555073358f, 0.0555073358f));
  q = __ffma2_rn(q, f, make_float2(0.240222424f, 0.240222424f));
  q = __ffma2_rn(q, f, make_float2(0.693147004f, 0.693147004f));
  q = __ffma2_rn(q, f, make_float2(1.f, 1.f));
  return make_float2(__uint_as_float(__float_as_uint(q.x) + (__float_as_uint(t.x) << 23)),
                     __uint_as_float(__float_as_uint(q.y) + (__float_as_uint(t.y) << 23)));
}

// Row tiles of a piece that have rows.
__device__ __forceinline__ int tiles_of(const AttnParams& p, const Pieces<Tiling>& at) {
  return at.r.queries * p.group - at.tile * kRows > kTileRows ? 2 : 1;
}

__device__ __forceinline__ bool next_piece(Pieces<Tiling>& at, const AttnParams& p, int lane) {
  __syncwarp();                                  // (readers of the last)
  if (lane == 0) at.more = at.next(p);
  __syncwarp();
  return at.more;
}

// The query that a row of a block is (none: token and head are those of the first row).
struct Place {
  bool on;
  int query, head;
  long long token;
  __device__ Place(const AttnParams& p, const Pieces<Tiling>& at, int row) {
    const int full = at.tile * kRows + row;
    on = full < at.r.queries * p.group;
    query = on ? full / p.group : 0;
    head = at.head * p.group + (on ? full - query * p.group : 0);
    token = at.r.first + query;
  }
};

// 16 bytes of channels 8 x ... of a row into a tile: boxes of 64 channels, rows of 128 bytes, 16-byte chunks swizzled by the row.
template <int D>
__device__ __forceinline__ void put_chunk(unsigned char* tile, int row, int x, uint4 v) {
  *reinterpret_cast<uint4*>(tile + (x >> 3) * Cfg<D>::kBoxBytes + row * 128 + (((x & 7) ^ (row & 7)) << 4)) = v;
}

// Units of 16 tokens into the raw ring, in order, a step's eight by a lane each.
template <int D>
__device__ void loader_role(Shared& sm, const AttnParams& p, Pieces<Tiling>& at, unsigned char* sRaw, int lane) {
  using U = Unit<D>;
  const uint32_t unit_mask = (1u << (p.page_shift - 4)) - 1, head_bytes = (uint32_t)U::kBytes << (p.page_shift - 4);
  uint32_t n = lane;                             // this lane's unit, counted over all pieces
  uint32_t asked = 0;                            // units that it has asked for: lane, lane + kUnits, ...
  bool ok = true;
  while (ok && next_piece(at, p, lane)) {
    const int32_t* table = p.tables + at.b * p.table_stride;
    const int keys = at.r.keys, steps_end = at.s_end;
    const uint32_t head_at = at.head * head_bytes;
    auto page_of = [&](int step) {
      const int u = step * kUnits + lane;
      return lane < kUnits && step < steps_end && u * kUnit < keys ? table[u >> (p.page_shift - 4)] : -1;
    };
    int page = page_of(at.s_begin);
    for (int step = at.s_begin; ok && step < steps_end; ++step, n += kUnits) {
      const int u = step * kUnits + lane;
      const int next_page = page_of(step + 1);
      bool mine = true;
      for (int x = 0; x < kUnits; ++x) {         // one after the other: the first need not wait for room for the last
        if (lane == x) {
          const uint32_t slot = n % kRaw;
          mine = WAIT_CALL(&sm.raw_empty[slot], ((n / kRaw) & 1) ^ 1);
          if (mine) {
            ++asked;
            int valid = max(0, min(keys - u * kUnit, kUnit));
            if (valid > 0 && (page < 0 || page >= p.pages)) { *(volatile int*)&sm.missing = 1; valid = 0; }
            *(volatile int*)&sm.raw_valid[slot] = valid;
            mbar_arrive_expect_tx(&sm.raw_full[slot], valid ? U::kBytes : 0);
            if (valid)
              bulk_load_1d(sRaw + slot * U::kBytes, p.data + (size_t)(uint32_t)page * p.Hk * head_bytes + head_at + ((uint32_t)u & unit_mask) * U::kBytes,
                           U::kBytes, &sm.raw_full[slot]);
          }
        }
        __syncwarp();
      }
      ok = __all_sync(kAll, mine);
      page = next_page;
    }
  }
  if (!ok && lane == 0) flag_timeout(sm, p);
  // The block's shared memory must not go away under a copy, whoever ended the block and why: wait (bounded, not cut short by the flag) for
  // the last units of each lane, but for those whose place in the ring has been given to a later one (their barrier is a phase further).
  // (Three: a lane may be a unit ahead of the others, and then its last but two may have the ring's place still.)
  int never = 0;
  const uint32_t next = __shfl_sync(kAll, asked, (lane + kRaw) % kUnits);
  if (lane < kUnits)
    for (uint32_t back = 1; back <= 3 && back <= asked; ++back) {
      const uint32_t x = lane + (asked - back) * kUnits;
      if ((x + kRaw) / kUnits >= next) mbar_wait(&sm.raw_full[x % kRaw], (x / kRaw) & 1, &never);
    }
}
static_assert(kRaw <= 2 * kUnits, "a lane's last three units are all that can be on their way");

// Raw units to fp16 tiles.  The tasks, eight units of keys and eight of values for each tile of keys, lie one after the other, and
// kWideners warps take them in turn.
template <int D>
__device__ void widen_role(Shared& sm, const AttnParams& p, uint32_t tiles, unsigned char* sKV, unsigned char* sRaw, int me, int lane) {
  using C = Cfg<D>;
  using U = Unit<D>;
  const int g = lane / 4, t = lane % 4;
  bool ok = true;
  for (uint32_t task = me; task < 2 * kUnits * tiles; task += kWideners) {
    const uint32_t m = task / kUnits, slot = m % kSlots;         // tile of the ring
    const bool values = m & 1;
    const uint32_t unit = task % kUnits, n = m / 2 * kUnits + unit, raw_slot = n % kRaw;
    if (!WAIT_CALL_ALL(&sm.raw_full[raw_slot], (n / kRaw) & 1)) { ok = false; break; }
    if (!WAIT_CALL_ALL(&sm.kv_empty[slot], ((m / kSlots) & 1) ^ 1)) { ok = false; break; }
    const unsigned char* raw = sRaw + raw_slot * U::kBytes;
    unsigned char* tile = sKV + slot * C::kTileBytes;
    const int row0 = unit * kUnit;
    if (values) {                                // tokens 8 h + 2 t + e, channels g d / 8 ...: d / 64 words of 8 channels each
      const int valid = *(volatile int*)&sm.raw_valid[raw_slot];
      uint32_t sc = *reinterpret_cast<const uint32_t*>(raw + U::kValueScales + ((D == 128 ? g : g / 2) * 4 + t) * 4);
      if (valid < kUnit) {
#pragma unroll
        for (int x = 0; x < 4; ++x)              // what no row may see is multiplied by zero
          if (2 * t + (x & 1) + 8 * (x >> 1) >= valid) sc &= ~(0xffu << (8 * x));
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[D / 32];
        if constexpr (D == 128) {
          // (odd lanes g write their two chunks the other way round: with that, eight lanes write to eight different groups of banks)
          const uint4 x = *reinterpret_cast<const uint4*>(raw + U::kValues + (h * 32 + lane) * 16);
          w[0] = g & 1 ? x.y : x.x; w[1] = g & 1 ? x.x : x.y; w[2] = g & 1 ? x.w : x.z; w[3] = g & 1 ? x.z : x.w;
        } else {
          *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(raw + U::kValues + (h * 32 + lane) * 8);
        }
        const __half2 both = scales2(h ? sc >> 16 : sc & 0xffff), of[2] = {__low2half2(both), __high2half2(both)};
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int y = 0; y < D / 64; ++y) {
            uint32_t c[4];
            codes8(w[e * (D / 64) + y], c);
#pragma unroll
            for (int x = 0; x < 4; ++x) c[x] = bits(__hmul2(half2_of(c[x]), of[e]));
            put_chunk<D>(tile, row0 + 8 * h + 2 * t + e, g * (D / 64) + (D == 128 ? y ^ (g & 1) : y), make_uint4(c[0], c[1], c[2], c[3]));
          }
      }
    } else {                                     // tokens 8 h + g, channels t d / 4 ...: d / 32 words of 8 channels each
      uint32_t sc;
      if constexpr (D == 128) sc = *reinterpret_cast<const uint32_t*>(raw + U::kKeyScales + lane * 4);
      else sc = *reinterpret_cast<const uint16_t*>(raw + U::kKeyScales + lane * 2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[D / 32];
        __half2 of[2];
        if constexpr (D == 128) {
          // (lanes of the second box write the second half of their channels first: eight groups of banks again)
          const uint4 x = *reinterpret_cast<const uint4*>(raw + U::kKeys + (h * 32 + lane) * 16);
          const __half2 both = scales2(h ? sc >> 16 : sc & 0xffff);
          w[0] = t & 2 ? x.z : x.x; w[1] = t & 2 ? x.w : x.y; w[2] = t & 2 ? x.x : x.z; w[3] = t & 2 ? x.y : x.w;
          of[0] = t & 2 ? __high2half2(both) : __low2half2(both);
          of[1] = t & 2 ? __low2half2(both) : __high2half2(both);
        } else {
          *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(raw + U::kKeys + (h * 32 + lane) * 8);
          const __half2 both = scales2(sc);
          of[0] = of[1] = h ? __high2half2(both) : __low2half2(both);
        }
#pragma unroll
        for (int y = 0; y < D / 32; ++y) {
          uint32_t c[4];
          codes8(w[y], c);
#pragma unroll
          for (int x = 0; x < 4; ++x) c[x] = bits(__hmul2(half2_of(c[x]), of[y / 2]));
          put_chunk<D>(tile, row0 + 8 * h + g, t * (D / 32) + (D == 128 ? y ^ (t & 2) : y), make_uint4(c[0], c[1], c[2], c[3]));
        }
      }
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if ((int)m != p.withhold) mbar_arrive(&sm.kv_full[slot]);  // (a test withholds a tile's)
      mbar_arrive(&sm.raw_empty[raw_slot]);
    }
  }
  if (!ok && lane == 0) flag_timeout(sm, p);
}

template <int D>
__device__ void mma_role(Shared& sm, const AttnParams& p, Pieces<Tiling>& at, unsigned char* sQ, unsigned char* sKV, uint32_t tmem,
                         int lane, const Shares& shares) {
  using C = Cfg<D>;
  const uint32_t idesc_qk = make_idesc_f16(kTileRows, kCols, false);
  const uint32_t idesc_pv = make_idesc_f16(kTileRows, D, true);
  const uint32_t q_lo0 = (smem_addr(sQ) >> 4) | (1u << 16);
  const uint32_t k_lo0 = (smem_addr(sKV) >> 4) | (1u << 16);
  const uint32_t v_lo0 = (smem_addr(sKV) >> 4) | ((uint32_t)(C::kBoxBytes >> 4) << 16);   // MN-major, as in fwd_sm100_dense.cu
  const bool leader = elect_one();
  uint32_t m = 0;                                // ring position of the current K tile
  uint32_t n[2] = {0, 0}, g[2] = {0, 0};         // per row tile: pieces and steps so far
  bool ok = true;
  auto scores = [&](int s, uint32_t slot) {      // S_s = Q_s K^T
    const uint32_t k_lo = k_lo0 + slot * (C::kTileBytes >> 4), q_lo = q_lo0 + s * (C::kTileBytes >> 4);
    tc_fence_after();
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const uint32_t off = ((ks / 4) * C::kBoxBytes + (ks % 4) * 32) >> 4;
      if (leader) mma_ss(tmem + kTmemS + s * kCols, desc_from_lo(q_lo + off), desc_from_lo(k_lo + off), idesc_qk, ks > 0);
    }
    if (leader) mma_commit(&sm.s_full[s]);
  };
  auto values = [&](int s, uint32_t slot, int half, bool first) {              // half of O_s (+)= P_s V
    const uint32_t v_lo = v_lo0 + slot * (C::kTileBytes >> 4);
    tc_fence_after();
#pragma unroll
    for (int kk = 0; kk < kCols / 32; ++kk) {
      const int ks = half * (kCols / 32) + kk;
      if (leader)
        mma_ts(tmem + kTmemO + s * D, tmem + kTmemS + s * kCols + ks * 8, desc_from_lo(v_lo + ((ks * 2048) >> 4)), idesc_pv,
               (first && ks == 0) ? 0u : 1u);
    }
  };
#define NEED(bar, parity) if (!WAIT_CALL_ALL(bar, parity)) { ok = false; break; }
  bool first = true;
  while (ok && next_piece(at, p, lane)) {
    if (first && lane == 0) {                    // the last piece of a cut item is a block's first
      Record record = Record::none();
      if (!at.begins() && at.ends()) record = Record{(int)shares.owner(at.item_begin) | at.head << 16, at.tile, at.r.queries, at.r.first};
      p.records[blockIdx.x] = record;
    }
    first = false;
    const int tiles = tiles_of(p, at), steps = at.s_end - at.s_begin;
    for (int s = 0; s < tiles; ++s) {
      if (s == 0) { NEED(&sm.kv_full[m % kSlots], (m / kSlots) & 1) }
      NEED(&sm.q_full[s], n[s] & 1)
      scores(s, m % kSlots);
      if (steps == 1 && leader) mma_commit(&sm.q_empty[s]);
    }
    if (!ok) break;
    if (leader) mma_commit(&sm.kv_empty[m % kSlots]);
    for (int t = 0; ok && t < steps; ++t, m += 2) {
      const uint32_t v_slot = (m + 1) % kSlots, k_slot = (m + 2) % kSlots;
      const bool last = t == steps - 1;
      for (int s = 0; s < tiles; ++s) {
        if (s == 0) { NEED(&sm.kv_full[v_slot], ((m + 1) / kSlots) & 1) }
        // the first P V of a piece overwrites O: the last piece's has to be read
        if (t == 0 && n[s] > 0) { NEED(&sm.o_free[s], (n[s] - 1) & 1) }
        NEED(&sm.p_full[s][0], g[s] & 1)
        values(s, v_slot, 0, t == 0);
        if (!last && s == 0) { NEED(&sm.kv_full[k_slot], ((m + 2) / kSlots) & 1) }
        NEED(&sm.p_full[s][1], g[s] & 1)
        values(s, v_slot, 1, false);
        ++g[s];
        if (leader) {
          if (last) mma_commit(&sm.o_full[s]);
          if (s == tiles - 1) mma_commit(&sm.kv_empty[v_slot]);
        }
        if (!last) {                             // (S is free behind the P V just issued: MMAs of one thread run in order)
          scores(s, k_slot);
          if (leader) {
            if (t + 1 == steps - 1) mma_commit(&sm.q_empty[s]);
            if (s == tiles - 1) mma_commit(&sm.kv_empty[k_slot]);
          }
        }
      }
    }
    for (int s = 0; s < tiles; ++s) ++n[s];
  }
#undef NEED
  if (!ok && leader) flag_timeout(sm, p);
  __syncwarp();
  // TMEM must not be released, nor shared memory go away, while MMAs use them: wait (bounded) behind everything that was issued, also if it is
  // another role that gives up, before or after this.
  int never = 0;
  if (leader) mma_commit(&sm.mma_drain);
  mbar_wait(&sm.mma_drain, 0, &never);
}

template <class T, int D>
__device__ void softmax_role(Shared& sm, const AttnParams& p, Pieces<Tiling>& at, unsigned char* sQ, uint32_t tmem, int s,
                             int warp_in_group, int lane) {
  using C = Cfg<D>;
  constexpr int kHalf = kCols / 2;
  // With 64 channels the exponentials, not the tensor core, are what a step waits for, and a quarter of them goes to the FMA pipe: 1.78
  // instead of 1.87 us a step.  With 128 the instructions cost more than they free: 2.39 instead of 2.13.
  constexpr bool kPoly = D == 64;
  const uint32_t lane_base = tmem + ((uint32_t)(warp_in_group * 32) << 16);
  const uint32_t t_s = lane_base + kTmemS + s * kCols, t_o = lane_base + kTmemO + s * D;
  const int row = warp_in_group * 32 + lane;
  uint32_t g = 0, n = 0;                         // steps and pieces of this row tile so far
  while (next_piece(at, p, lane)) {
    if (s >= tiles_of(p, at)) continue;
    const Place at_row(p, at, s * kTileRows + row);
    // (a row that is not there sees all: it would have every tile masked)
    const int sees = at_row.on && p.causal ? at.r.sees(at_row.query) : at.r.keys;
    // ---- the row's queries, scaled by a power of two: the largest becomes 2^14 to 2^15 (see cache_attention.cu)
    float sl2;
    bool finite = true;
    {
      if (!WAIT_ALL(&sm.q_empty[s], (n & 1) ^ 1)) { if (lane == 0) flag_timeout(sm, p); return; }
      const uint4* src = reinterpret_cast<const uint4*>((const T*)p.q + at_row.token * p.q_s[0] + at_row.head * p.q_s[1]);
      uint4 raw[D / 8];
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) raw[i] = at_row.on ? src[i] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = Two<T>::widen(w[j]);
          most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
          finite = finite && isfinite(f.x) && isfinite(f.y);
        }
      }
      const int e = finite && most > 0.f ? (int)((__float_as_uint(most) >> 23) & 255) - 127 : 14;
      const float up = power2(max(-126, min(127, 14 - e)));
      sl2 = fmaxf(p.sl2 / up, 1.2e-38f);         // (not zero: what is hidden is -inf before it is scaled)
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = Two<T>::widen(w[j]);
          // (a row that is not finite is zero here, and NaN by its sum)
          w[j] = finite ? bits(__floats2half2_rn(f.x * up, f.y * up)) : 0u;
        }
        put_chunk<D>(sQ + s * C::kTileBytes, row, i, make_uint4(w[0], w[1], w[2], w[3]));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full[s]);
    }
    // exponents are x + nm, x the logit times log2(e): nm = kShift - (a maximum of the row's earlier keys), 0 if it has none yet
    float nm = 0.f, l = 0.f;
    bool seen = false;
    bool ok = true;
    for (int step = at.s_begin; step < at.s_end; ++step, ++g) {
      const int left = sees - step * kCols;      // columns that the row sees
      if (!WAIT_ALL(&sm.s_full[s], g & 1)) { ok = false; break; }
      tc_fence_after();
      // Columns that the row does not see are set to -inf where they lie, 16 at a time: this is rare, and as code between the loads and the
      // maxima it pushed the common path out of the instruction cache (2.63 us a step, 2.09 without it)
      // (by votes: the loader may be setting the word, and the TMEM accesses are for whole warps)
      const bool missing = __any_sync(kAll, *(volatile int*)&sm.missing != 0);
      if (__any_sync(kAll, left < kCols) || missing) {
#pragma unroll 1
        for (int x = 0; x < kUnits; ++x) {
          int seen_here = left - x * kUnit;
          if (missing) {
            const int u = step * kUnits + x, page = u * kUnit < at.r.keys ? p.tables[at.b * p.table_stride + (u >> (p.page_shift - 4))] : -1;
            if (page < 0 || page >= p.pages) seen_here = 0;
          }
          uint32_t c[16];
          tmem_ld_32x32b_x16(t_s + x * kUnit, c);
          tmem_ld_wait();
#pragma unroll
          for (int y = 0; y < 16; ++y)
            if (y >= seen_here) c[y] = __float_as_uint(-INFINITY);
          tmem_st_32x32b_x16(t_s + x * kUnit, c);
        }
        tmem_st_wait();
      }
      uint32_t sr[kCols];
      auto half_max = [&](int c0) {
        constexpr int kQ = kHalf / 4;
        float m[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) m[x] = -INFINITY;
#pragma unroll
        for (int c = 0; c < kQ; c += 2)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            m[x] = max3<kPoly>(m[x], __uint_as_float(sr[c0 + x * kQ + c]), __uint_as_float(sr[c0 + x * kQ + c + 1]));
        return max3<kPoly>(max3<kPoly>(m[0], m[1], m[2]), m[3], m[3]);
      };
      // the maximum of the first half is taken while the second half is on its way
      tmem_ld_cols<kHalf>(t_s, sr);
      tmem_ld_wait();
      tmem_ld_cols<kHalf>(t_s + kHalf, sr + kHalf);
      float mx = half_max(0);
      tmem_ld_wait();
      mx = max3<kPoly>(mx, half_max(kHalf), mx) * sl2;           // (without the polynomial NaN is not among what the maximum is taken of)
      if (kPoly && mx != mx) l = NAN;            // (a key that the row sees is not finite: the polynomial's weight for it may be any number)
      const bool some = mx > -INFINITY;
      if (__any_sync(kAll, some && (!seen || mx + nm > kMost))) {
        const float nm_new = some && (!seen || mx + nm > kMost) ? kShift - mx : nm;
        const float f = seen ? ex2(nm_new - nm) : 1.f;
        if (step > at.s_begin) {
          // (P V of the previous step has landed in O: it was issued before the scores of this one)
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t o[16];
            tmem_ld_32x32b_x16(t_o + c * 16, o);
            tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
            tmem_st_32x32b_x16(t_o + c * 16, o);
          }
        }
        l *= f;
        if (mx == INFINITY) l = NAN;             // (a logit above fp32's range: with nm = -inf all weights would be 0)
        nm = nm_new;
        seen = seen || some;
      }
      // weights 2^(sl2 S + nm), as packed fp32 pairs
      const float2 sl2_2 = make_float2(sl2, sl2), nm2 = make_float2(nm, nm);
      float2 s_a = make_float2(0.f, 0.f), s_b = make_float2(0.f, 0.f);
      auto exps = [&](int c0, int count) {       // columns [c0, c0 + count), fp16 pairs to sr[c0 / 2 ...]
#pragma unroll
        for (int c = 0; c < count; c += 4) {
          const uint32_t* x = sr + c0 + c;
          const float2 xa = __ffma2_rn(make_float2(__uint_as_float(x[0]), __uint_as_float(x[1])), sl2_2, nm2);
          const float2 xb = __ffma2_rn(make_float2(__uint_as_float(x[2]), __uint_as_float(x[3])), sl2_2, nm2);
          const float2 ea = make_float2(ex2(xa.x), ex2(xa.y));
          const float2 eb = kPoly && (c0 + c) % 8 == 4 ? exp2_fma(xb) : make_float2(ex2(xb.x), ex2(xb.y));
          s_a = __fadd2_rn(s_a, ea);
          s_b = __fadd2_rn(s_b, eb);
          sr[(c0 + c) / 2] = bits(__floats2half2_rn(ea.x, ea.y));
          sr[(c0 + c) / 2 + 1] = bits(__floats2half2_rn(eb.x, eb.y));
        }
      };
      auto arrive = [&](int half) {
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[s][half]);
      };
      exps(0, kHalf);
      tmem_st_32x32b_x32(t_s, *reinterpret_cast<uint32_t(*)[32]>(&sr[0]));
      // the store of the first half completes behind the first exponentials of the second
      exps(kHalf, kHalf / 4);
      arrive(0);
      exps(kHalf + kHalf / 4, 3 * kHalf / 4);
      tmem_st_32x32b_x32(t_s + 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[32]));
      arrive(1);
      const float2 sum = __fadd2_rn(s_a, s_b);
      l += sum.x + sum.y;
    }
    if (ok) ok = WAIT_ALL(&sm.o_full[s], n & 1);
    if (!ok) { if (lane == 0) flag_timeout(sm, p); return; }
    // ---- O / l, or a piece's O and statistics
    tc_fence_after();
    if (kPoly && !seen && l == l) l = 0.f;       // (the polynomial's least weight is 2^-126, also for what is hidden)
    if (!finite && seen) l = NAN;                // (a row that is not finite and sees something)
    const bool whole = at.begins() && at.ends();
    const Place to(p, at, s * kTileRows + row);  // (again: registers are scarce in between)
    const float top = seen ? kShift - nm : -INFINITY;
    const float inv = l == 0.f ? 0.f : p.v_scale / l;
    float* part = p.parts + (size_t)(2 * blockIdx.x + (at.begins() ? 1 : 0)) * C::kPartFloats;
    T* orow = (T*)p.out + to.token * p.o_s[0] + to.head * p.o_s[1];
    const int in_block = s * kTileRows + row;
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t a[32];
      tmem_ld_32x32b_x32(t_o + c * 32, a);
      tmem_ld_wait();
      if (c == D / 32 - 1) {                     // the accumulator is in registers: it may be overwritten
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.o_free[s]);
      }
      if (!to.on) continue;
      if (whole) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {            // 16 bytes (8 channels) per store
          uint32_t w[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float b0 = __uint_as_float(a[x * 8 + 2 * y]), b1 = __uint_as_float(a[x * 8 + 2 * y + 1]);
            w[y] = l == 0.f ? 0u : Two<T>::round(b0 * inv, b1 * inv);
          }
          *reinterpret_cast<uint4*>(orow + c * 32 + x * 8) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else {
        float* dst = part + in_block * D + c * 32;
#pragma unroll
        for (int x = 0; x < 4; ++x) st_global_v8(dst + x * 8, *reinterpret_cast<uint32_t(*)[8]>(&a[x * 8]));
      }
    }
    if (to.on && whole && p.lse)
      p.lse[to.token * p.Hq + to.head] = l == 0.f ? -INFINITY : ((seen ? top : 0.f) + log2f(l) - kShift) * kLn2;
    if (!whole) {
      part[kRows * D + in_block] = top;
      part[kRows * (D + 1) + in_block] = l;
    }
    ++n;
  }
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) cache_attention_chunk_kernel(const __grid_constant__ AttnParams p) {
  using C = Cfg<D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ Shared sm;
  unsigned char* sQ = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* sKV = sQ + 2 * C::kTileBytes;
  unsigned char* sRaw = sKV + kSlots * C::kTileBytes;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) {
    sm.abort_flag = sm.missing = 0;
    for (int i = 0; i < kSlots; ++i) { mbar_init(&sm.kv_full[i], kUnits); mbar_init(&sm.kv_empty[i], 1); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.q_full[s], 4); mbar_init(&sm.q_empty[s], 1);
      mbar_init(&sm.s_full[s], 1);
      mbar_init(&sm.p_full[s][0], 4); mbar_init(&sm.p_full[s][1], 4);
      mbar_init(&sm.o_full[s], 1); mbar_init(&sm.o_free[s], 4);
    }
    for (int i = 0; i < kRaw; ++i) { mbar_init(&sm.raw_full[i], 1); mbar_init(&sm.raw_empty[i], 2); }
    mbar_init(&sm.mma_drain, 1);
    fence_mbar_init();
  }
  if (warp == 0) { tmem_alloc(&sm.tmem_base, kTmemCols); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  kernel_wait();
  const Shares shares = find_share<kThreads, Tiling>(p, blockIdx.x, sm.sums, &sm.start);
  if ((long long)blockIdx.x < shares.blocks) {
    if (lane == 0) sm.pieces[warp].start(p, sm.start, shares.begin(blockIdx.x), shares.begin(blockIdx.x + 1));
    __syncwarp();
    // A softmax thread holds a whole row of scores: it takes registers over from the other roles.
    if (warp < 8) {
      set_max_registers_up<kRegsSoftmax>();
      softmax_role<T, D>(sm, p, sm.pieces[warp], sQ, tmem, warp / 4, warp % 4, lane);
    } else {
      set_max_registers_down<kRegsOther>();
      if (warp == kWarpMma) mma_role<D>(sm, p, sm.pieces[warp], sQ, sKV, tmem, lane, shares);
      else if (warp == kWarpLoader) loader_role<D>(sm, p, sm.pieces[warp], sRaw, lane);
      else widen_role<D>(sm, p, (uint32_t)(shares.begin(blockIdx.x + 1) - shares.begin(blockIdx.x)), sKV, sRaw, warp - kWarpWiden, lane);
    }
  } else if (threadIdx.x == 0) {
    p.records[blockIdx.x] = Record::none();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, kTmemCols);
}

template <class T, int D>
cudaError_t launch_instance(const AttnParams& p, int grid, cudaStream_t stream) {
  // the roles share out what the launch brings, which is the compiler's choice within the launch bounds
  static std::atomic<bool> enough{false};
  if (!enough) {
    cudaFuncAttributes a{};
    const cudaError_t e = cudaFuncGetAttributes(&a, cache_attention_chunk_kernel<T, D>);
    if (e != cudaSuccess) return e;
    if (a.numRegs < kRegsLaunch) return cudaErrorInvalidConfiguration;
    enough = true;
  }
  return launch_after(cache_attention_chunk_kernel<T, D>, dim3(grid), kThreads, Cfg<D>::kSmem, Cfg<D>::kSmem, 0, stream, p);
}

}  // namespace

cudaError_t launch_chunk(const AttnParams& p, int d, int type, int sms, cudaStream_t stream, int* grid) {
  *grid = sms < kMostChunkBlocks ? sms : kMostChunkBlocks;
  if (type == SOL_TYPE_BF16)
    return d == 128 ? launch_instance<__nv_bfloat16, 128>(p, *grid, stream) : launch_instance<__nv_bfloat16, 64>(p, *grid, stream);
  return d == 128 ? launch_instance<__half, 128>(p, *grid, stream) : launch_instance<__half, 64>(p, *grid, stream);
}

}  // namespace cache
}  // namespace sol

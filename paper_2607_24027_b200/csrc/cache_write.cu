// Keys and values into the 4-bit cache and back (sol_attn_cache_append, sol_attn_cache_read).
//
// Bound by HBM: 4 d bytes of a token and head on one side, 9 d / 8 on the other; next to that by issuing the instructions, of which
// finding the place takes as many as 16 channels do, and by the L1's accesses.  So a lane has 32 channels of one token, two groups of
// 32 bytes each, which it loads or stores at once, and a warp's tokens lie side by side.
// 7800 tokens x 40 heads x 128 channels, slots half taken: writing 46 us (a group to a lane 62, 16-byte loads 54, tokens apart 53), reading 35.
#include "cache.cuh"
#include "ptx_sm100.cuh"

namespace sol {
namespace {

using cache::Two;

constexpr int kThreads = 128;

struct WriteParams {
  const void *k, *v;                             // append: sources; read: destinations
  long long k_s[2], v_s[2];
  const int32_t* slots;
  unsigned char* data;
  int tokens, Hk, page_shift, slot_end, k_exp, v_exp;
  int aligned32;                                 // every row of k and v starts on a 32-byte boundary
};

// Which token, head, part of 32 channels and side (key or value) a thread has.  A warp has 4 (d = 128) or 8 (d = 64) tokens that follow each
// other in the call, and mostly in the cache too, of one head: then its keys' codes are 256 bytes on end, and its values' fill sectors.
template <int D>
struct Place {
  static constexpr int kParts = D / 32, kTokens = 16 / kParts;
  int part, in_warp, token, head;
  bool is_value;
  __device__ Place(const WriteParams& p) {
    const uint32_t lane = threadIdx.x % 32, warp = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    part = lane % kParts;
    in_warp = lane / kParts % kTokens;
    is_value = lane >= 16;
    const uint32_t of = warp / (uint32_t)p.Hk;
    head = (int)(warp - of * p.Hk);
    token = (int)(of * kTokens) + in_warp;
  }
};

// Four e2m1 pairs to a word, the first number of each in the lower four bits.
__device__ __forceinline__ uint32_t pack_codes(const float2 (&x)[4]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(x[0].x), "f"(x[0].y), "f"(x[1].x), "f"(x[1].y), "f"(x[2].x), "f"(x[2].y), "f"(x[3].x), "f"(x[3].y));
  return r;
}

// Codes of 16 channels in eight words of 16-bit numbers, whose largest magnitude has the bits `most16`; the scale's e4m3 number in `s8`.
template <class T>
__device__ __forceinline__ uint2 codes_of(const uint32_t* w, uint32_t most16, float unscale, uint32_t* s8) {
  const float most = Two<T>::widen(most16).x * unscale;
  // max|x| has at most 11 significant bits and a tie of e4m3 times 6 has 7, so the quotient, rounded to fp32, is a tie only if it is one.
  *s8 = __nv_cvt_float_to_fp8(fminf(__fdiv_rn(most, 6.f), 448.f), __NV_SATFINITE, __NV_E4M3);
  const float s = __low2float(cache::scales2(*s8));
  // x 2^-exp / s by the reciprocal is off by 2^-23 at most, which would break ties (0.75 s and the like).  A quotient that is no
  // tie is 2^-11 or more away from one (x has 11 bits at most, s times a tie 7), so rounding to 12 bits (Veltkamp's
  // splitting) puts ties back in place and moves nothing across one.
  const float inv = s > 0.f ? unscale / s : 0.f;
  const float2 inv2 = make_float2(inv, inv), split2 = make_float2(4097.f, 4097.f), zero2 = make_float2(0.f, 0.f),
               minus2 = make_float2(-1.f, -1.f);
  float2 y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __ffma2_rn(Two<T>::widen(w[i]), inv2, zero2);
  // A quotient is 7 at most with a scale of full precision, less than 9 with a subnormal one (the scale 2^-9 stands for up to 1.5 times itself), which
  // the splitting takes and the conversion makes 6.  Only where the scale is at its end may it be anything, up to an infinity.
  if (most > 6.5f * 448.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = make_float2(fminf(fmaxf(y[i].x, -8.f), 8.f), fminf(fmaxf(y[i].y, -8.f), 8.f));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 c = __ffma2_rn(y[i], split2, zero2);
    y[i] = __ffma2_rn(__ffma2_rn(y[i], minus2, c), minus2, c);
  }
  return make_uint2(pack_codes(*reinterpret_cast<float2(*)[4]>(y)), pack_codes(*reinterpret_cast<float2(*)[4]>(y + 4)));
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(const __grid_constant__ WriteParams p) {
  using U = cache::Unit<D>;
  constexpr int kParts = Place<D>::kParts;
  const Place<D> at(p);
  kernel_wait();
  const int slot = at.token < p.tokens ? p.slots[at.token] : -1;
  const bool stored = slot >= 0 && slot < p.slot_end;
  uint32_t w[2][8], most16[2] = {0, 0};          // largest |x| of each group: 16-bit floats are in the order of their bits
  if (stored) {
    const T* src = at.is_value ? (const T*)p.v + at.token * p.v_s[0] + at.head * p.v_s[1]
                               : (const T*)p.k + at.token * p.k_s[0] + at.head * p.k_s[1];
    const uint4* in = reinterpret_cast<const uint4*>(src + at.part * 32);
    if (p.aligned32) {
      ptx::ld_global_v8(in, w[0]);
      ptx::ld_global_v8(in + 2, w[1]);
    } else {                                     // the interface only asks for 16 bytes
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(&w[i / 2][i % 2 * 4]) = in[i];
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t most2 = w[g][0] & 0x7fff7fffu;
#pragma unroll
      for (int i = 1; i < 8; ++i) most2 = __vmaxu2(most2, w[g][i] & 0x7fff7fffu);
      most16[g] = max(most2 & 0xffffu, most2 >> 16);
    }
  }
  // one element that is not finite marks its token's key
  const bool bad = max(most16[0], most16[1]) >= Two<T>::kInf;
  const unsigned mine = (((1u << kParts) - 1u) * 0x10001u) << (at.in_warp * kParts);
  const bool mark = (__ballot_sync(0xffffffffu, bad) & mine) != 0;
  if (!stored) return;
  if (bad) {                                     // such elements count as zero
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      most16[g] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if ((w[g][i] & 0x7fffu) >= Two<T>::kInf) w[g][i] &= 0xffff0000u;
        if ((w[g][i] >> 16 & 0x7fffu) >= Two<T>::kInf) w[g][i] &= 0xffffu;
        most16[g] = max(most16[g], max(w[g][i] & 0x7fffu, w[g][i] >> 16 & 0x7fffu));
      }
    }
  }
  const float unscale = cache::power2(-(at.is_value ? p.v_exp : p.k_exp));
  uint32_t s8[2];
  const uint2 a = codes_of<T>(w[0], most16[0], unscale, s8), b = codes_of<T>(w[1], most16[1], unscale, s8 + 1);
  unsigned char* unit = p.data + cache::unit_at<D>(slot, at.head, p.page_shift, p.Hk);
  const int i = slot % cache::kUnit, group = 2 * at.part;
  if (at.is_value) {
    unsigned char* dst = unit + U::value_codes(i, group);
    if constexpr (D == 128) {
      *reinterpret_cast<uint2*>(dst) = a;
      *reinterpret_cast<uint2*>(dst + U::kPartStride) = b;       // (a group of 16 channels lies together)
    } else {
      *reinterpret_cast<uint32_t*>(dst) = a.x;                   // (8 channels do)
      *reinterpret_cast<uint32_t*>(dst + U::kPartStride) = a.y;
      *reinterpret_cast<uint32_t*>(dst + 2 * U::kPartStride) = b.x;
      *reinterpret_cast<uint32_t*>(dst + 3 * U::kPartStride) = b.y;
    }
    unit[U::value_scale(i, group)] = (unsigned char)s8[0];
    unit[U::value_scale(i, group + 1)] = (unsigned char)s8[1];
  } else {
    *reinterpret_cast<uint4*>(unit + U::key_codes(i, group)) = make_uint4(a.x, a.y, b.x, b.y);
    if (mark && at.part == 0) s8[0] = 0x7f;
    if constexpr (D == 128) {
      *reinterpret_cast<unsigned short*>(unit + U::key_scale(i, group)) = (unsigned short)(s8[0] | s8[1] << 8);
    } else {
      unit[U::key_scale(i, group)] = (unsigned char)s8[0];
      unit[U::key_scale(i, group + 1)] = (unsigned char)s8[1];
    }
  }
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const __grid_constant__ WriteParams p) {
  using U = cache::Unit<D>;
  const Place<D> at(p);
  kernel_wait();
  if (at.token >= p.tokens) return;
  T* dst = (T*)const_cast<void*>(at.is_value ? p.v : p.k);
  const int slot = p.slots[at.token];
  if (!dst || slot < 0 || slot >= p.slot_end) return;
  const unsigned char* unit = p.data + cache::unit_at<D>(slot, at.head, p.page_shift, p.Hk);
  const int i = slot % cache::kUnit, group = 2 * at.part;
  uint32_t codes[4], s8[2];
  if (at.is_value) {
    const unsigned char* src = unit + U::value_codes(i, group);
    if constexpr (D == 128) {
      *reinterpret_cast<uint2*>(codes) = *reinterpret_cast<const uint2*>(src);
      *reinterpret_cast<uint2*>(codes + 2) = *reinterpret_cast<const uint2*>(src + U::kPartStride);
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x) codes[x] = *reinterpret_cast<const uint32_t*>(src + x * U::kPartStride);
    }
    s8[0] = unit[U::value_scale(i, group)];
    s8[1] = unit[U::value_scale(i, group + 1)];
  } else {
    *reinterpret_cast<uint4*>(codes) = *reinterpret_cast<const uint4*>(unit + U::key_codes(i, group));
    s8[0] = unit[U::key_scale(i, group)];
    s8[1] = unit[U::key_scale(i, group + 1)];
  }
  const float2 both = __half22float2(cache::scales2(s8[0] | s8[1] << 8));
  const float up = cache::power2(at.is_value ? p.v_exp : p.k_exp);
  dst += (at.is_value ? at.token * p.v_s[0] + at.head * p.v_s[1] : at.token * p.k_s[0] + at.head * p.k_s[1]) + at.part * 32;
#pragma unroll
  for (int g = 0; g < 2; ++g) {                  // 16 channels
    const float s = (g ? both.y : both.x) * up;
    uint32_t c[8];
    cache::codes8(codes[2 * g], *reinterpret_cast<uint32_t(*)[4]>(c));
    cache::codes8(codes[2 * g + 1], *reinterpret_cast<uint32_t(*)[4]>(c + 4));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 f = __ffma2_rn(__half22float2(cache::half2_of(c[j])), make_float2(s, s), make_float2(0.f, 0.f));
      c[j] = Two<T>::round(f.x, f.y);
    }
    if (p.aligned32) {
      ptx::st_global_v8(dst + g * 16, c);
    } else {
      reinterpret_cast<uint4*>(dst + g * 16)[0] = make_uint4(c[0], c[1], c[2], c[3]);
      reinterpret_cast<uint4*>(dst + g * 16)[1] = make_uint4(c[4], c[5], c[6], c[7]);
    }
  }
}

enum { kAppend, kRead };

sol_status_t launch(int what, const sol_attn_cache* c, const void* k, const void* v, const int64_t* ks, const int64_t* vs,
                    const int32_t* slots, int tokens, int type, sol_stream_t stream) {
  sol_status_t s = cache::check(c);
  if (s != SOL_OK) return s;
  if (tokens < 0 || (type != SOL_TYPE_BF16 && type != SOL_TYPE_FP16)) return SOL_ERR_INVALID_ARG;
  if (tokens == 0) return SOL_OK;
  if (what == kAppend ? (!k || !v) : (!k && !v)) return SOL_ERR_INVALID_ARG;
  for (int i = 0; i < 2; ++i) {
    const void* x = i ? v : k;
    const int64_t* st = i ? vs : ks;
    if (x && (!st || !cache::aligned(x, 16) || !cache::strides_ok(st, tokens, c->Hk))) return SOL_ERR_INVALID_ARG;
    if (x && what == kRead && !cache::rows_apart(st, tokens, c->Hk)) return SOL_ERR_INVALID_ARG;
  }
  if (!slots || !cache::aligned(slots, 4)) return SOL_ERR_INVALID_ARG;
  if ((s = check_device_arch()) != SOL_OK) return s;
  WriteParams p{};
  p.k = k; p.v = v;
  for (int i = 0; i < 2; ++i) {                  // (a dimension of one has no use for its stride)
    const bool one = (i ? c->Hk : tokens) <= 1;
    p.k_s[i] = k && !one ? ks[i] : 0;
    p.v_s[i] = v && !one ? vs[i] : 0;
  }
  p.slots = slots;
  p.data = static_cast<unsigned char*>(c->data);
  if ((long long)tokens * c->Hk > 0x3fffffffLL) return SOL_ERR_UNSUPPORTED_SHAPE;
  p.tokens = tokens;
  p.Hk = c->Hk; p.page_shift = cache::page_shift(c->page_size); p.slot_end = c->pages * c->page_size;
  p.k_exp = c->k_exp; p.v_exp = c->v_exp;
  p.aligned32 = cache::aligned(k, 32) && cache::aligned(v, 32) &&
                (p.k_s[0] | p.k_s[1] | p.v_s[0] | p.v_s[1]) % 16 == 0;
  const uint32_t of_warp = 16 / (c->d / 32), warps = (((uint32_t)tokens + of_warp - 1) / of_warp) * (uint32_t)c->Hk;
  const uint32_t blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  auto run = [&](auto kernel) {
    return launch_after(kernel, dim3(blocks), kThreads, 0, 0, 0, static_cast<cudaStream_t>(stream), p);
  };
  cudaError_t e;
  if (what == kAppend)
    e = type == SOL_TYPE_BF16 ? (c->d == 128 ? run(cache_append_kernel<__nv_bfloat16, 128>) : run(cache_append_kernel<__nv_bfloat16, 64>))
                              : (c->d == 128 ? run(cache_append_kernel<__half, 128>) : run(cache_append_kernel<__half, 64>));
  else
    e = type == SOL_TYPE_BF16 ? (c->d == 128 ? run(cache_read_kernel<__nv_bfloat16, 128>) : run(cache_read_kernel<__nv_bfloat16, 64>))
                              : (c->d == 128 ? run(cache_read_kernel<__half, 128>) : run(cache_read_kernel<__half, 64>));
  count_launches(1);
  return e == cudaSuccess ? SOL_OK : SOL_ERR_CUDA;
}

}  // namespace
}  // namespace sol

extern "C" {

size_t sol_attn_cache_bytes(int pages, int page_size, int Hk, int d) {
  if (pages <= 0 || Hk <= 0 || Hk > sol::cache::kMaxHeads || (d != 64 && d != 128)) return 0;
  if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128 && page_size != 256) return 0;
  if ((long long)pages * page_size > 0x7fffffffLL) return 0;
  return (size_t)pages * Hk * (page_size / sol::cache::kUnit) * sol::cache::unit_bytes(d);
}

sol_status_t sol_attn_cache_append(const sol_attn_cache* cache, const void* k, const void* v, const int64_t* k_stride,
                                   const int64_t* v_stride, const int32_t* slots, int tokens, int type, sol_stream_t stream) {
  return sol::launch(sol::kAppend, cache, k, v, k_stride, v_stride, slots, tokens, type, stream);
}

sol_status_t sol_attn_cache_read(const sol_attn_cache* cache, void* k, void* v, const int64_t* k_stride, const int64_t* v_stride,
                                 const int32_t* slots, int tokens, int type, sol_stream_t stream) {
  return sol::launch(sol::kRead, cache, k, v, k_stride, v_stride, slots, tokens, type, stream);
}

}  // extern "C"

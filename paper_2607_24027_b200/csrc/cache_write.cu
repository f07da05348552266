// Keys and values into the 4-bit cache and back (sol_attn_cache_append, sol_attn_cache_read).
//
// Bound by HBM: 4 d bytes of a token and head on one side, 9 d / 8 on the other.  A lane has one group of 16 channels of one
// token; d / 16 lanes have a key, the next d / 16 the value, so a warp has 2 (d = 128) or 4 (d = 64) rows of a key and a value.
#include "cache.cuh"

namespace sol {
namespace {

constexpr int kThreads = 128;

struct WriteParams {
  const void *k, *v;                             // append: sources; read: destinations
  long long k_s[2], v_s[2];
  const int32_t* slots;
  unsigned char* data;
  uint32_t rows;                                 // tokens * Hk
  int Hk, page_shift, slot_end, k_exp, v_exp;
};

// Which row, group and side of a row (key or value) a thread has.
template <int D>
struct Place {
  uint32_t row;
  int group, token, head;
  bool is_value;
  __device__ Place(const WriteParams& p) {
    constexpr int kGroups = D / 16;
    group = threadIdx.x % kGroups;
    is_value = (threadIdx.x / kGroups) % 2;
    row = blockIdx.x * (kThreads / (2 * kGroups)) + threadIdx.x / (2 * kGroups);
    token = (int)(row / (uint32_t)p.Hk);
    head = (int)(row - (uint32_t)token * p.Hk);
  }
};

template <class T, int D>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(const WriteParams p) {
  using U = cache::Unit<D>;
  using cache::Two;
  constexpr int kGroups = D / 16;
  const Place<D> at(p);
  kernel_wait();
  const bool on = at.row < p.rows;
  const int slot = on ? p.slots[at.token] : -1;
  const bool stored = slot >= 0 && slot < p.slot_end;
  uint32_t w[8];
  uint32_t most2 = 0;                            // the largest |x| of either half of the words: 16-bit floats are in the order of their bits
  if (stored) {
    const T* src = at.is_value ? (const T*)p.v + at.token * p.v_s[0] + at.head * p.v_s[1]
                               : (const T*)p.k + at.token * p.k_s[0] + at.head * p.k_s[1];
    const uint4* in = reinterpret_cast<const uint4*>(src + at.group * 16);
    const uint4 a = in[0], b = in[1];
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
#pragma unroll
    for (int i = 0; i < 8; ++i) most2 = __vmaxu2(most2, w[i] & 0x7fff7fffu);
  }
  uint32_t most16 = max(most2 & 0xffffu, most2 >> 16);
  // one element that is not finite marks its token's key
  const bool bad = most16 >= Two<T>::kInf;
  const unsigned mine = ((1u << (2 * kGroups)) - 1u) << ((threadIdx.x % 32) / (2 * kGroups) * (2 * kGroups));
  const bool mark = (__ballot_sync(0xffffffffu, bad) & mine) != 0;
  if (!stored) return;
  if (bad) {                                     // such elements count as zero
    most16 = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if ((w[i] & 0x7fffu) >= Two<T>::kInf) w[i] &= 0xffff0000u;
      if ((w[i] >> 16 & 0x7fffu) >= Two<T>::kInf) w[i] &= 0xffffu;
      most16 = max(most16, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
    }
  }
  const float unscale = cache::power2(-(at.is_value ? p.v_exp : p.k_exp)), most = Two<T>::widen(most16).x * unscale;
  // max|x| has at most 11 significant bits and a tie of e4m3 times 6 has 7, so the quotient, rounded to fp32, is a tie only if it is one.
  const __nv_fp8_storage_t s8 = __nv_cvt_float_to_fp8(fminf(__fdiv_rn(most, 6.f), 448.f), __NV_SATFINITE, __NV_E4M3);
  const float s = __half2float(__half(__nv_cvt_fp8_to_halfraw(s8, __NV_E4M3)));
  // x 2^-exp / s by the reciprocal is off by 2^-23 at most, which would break ties (0.75 s and the like).  A quotient that is no
  // tie is 2^-11 or more away from one (x has 11 bits at most, s times a tie 7), so rounding to 12 bits (Veltkamp's
  // splitting) puts ties back in place and moves nothing across one.
  const float inv = s > 0.f ? unscale / s : 0.f;
  const bool over = most > 6.5f * 448.f;         // only then a quotient may pass 7, and much further
  const float2 inv2 = make_float2(inv, inv), split2 = make_float2(4097.f, 4097.f), zero2 = make_float2(0.f, 0.f),
               minus2 = make_float2(-1.f, -1.f);
  unsigned long long codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float2 y = __ffma2_rn(Two<T>::widen(w[i]), inv2, zero2);
    if (over) {
      y.x = fminf(fmaxf(y.x, -8.f), 8.f);
      y.y = fminf(fmaxf(y.y, -8.f), 8.f);
    }
    const float2 c = __ffma2_rn(y, split2, zero2), t = __ffma2_rn(__ffma2_rn(y, minus2, c), minus2, c);
    codes |= (unsigned long long)__nv_cvt_float2_to_fp4x2(t, __NV_E2M1, cudaRoundNearest) << (8 * i);
  }
  unsigned char* unit = p.data + cache::unit_at<D>(slot, at.head, p.page_shift, p.Hk);
  const int i = slot % cache::kUnit;
  if (at.is_value) {
    unsigned char* dst = unit + U::value_codes(i, at.group);
    if constexpr (D == 128) {
      *reinterpret_cast<unsigned long long*>(dst) = codes;
    } else {
      *reinterpret_cast<uint32_t*>(dst) = (uint32_t)codes;
      *reinterpret_cast<uint32_t*>(dst + U::kPartStride) = (uint32_t)(codes >> 32);
    }
    unit[U::value_scale(i, at.group)] = s8;
  } else {
    *reinterpret_cast<unsigned long long*>(unit + U::key_codes(i, at.group)) = codes;
    unit[U::key_scale(i, at.group)] = mark && at.group == 0 ? 0x7f : s8;
  }
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const WriteParams p) {
  using U = cache::Unit<D>;
  using cache::Two;
  const Place<D> at(p);
  kernel_wait();
  if (at.row >= p.rows) return;
  T* dst = (T*)const_cast<void*>(at.is_value ? p.v : p.k);
  const int slot = p.slots[at.token];
  if (!dst || slot < 0 || slot >= p.slot_end) return;
  const unsigned char* unit = p.data + cache::unit_at<D>(slot, at.head, p.page_shift, p.Hk);
  const int i = slot % cache::kUnit;
  unsigned long long codes;
  uint32_t s8;
  if (at.is_value) {
    const unsigned char* src = unit + U::value_codes(i, at.group);
    if constexpr (D == 128)
      codes = *reinterpret_cast<const unsigned long long*>(src);
    else
      codes = *reinterpret_cast<const uint32_t*>(src) | (unsigned long long)*reinterpret_cast<const uint32_t*>(src + U::kPartStride) << 32;
    s8 = unit[U::value_scale(i, at.group)];
  } else {
    codes = *reinterpret_cast<const unsigned long long*>(unit + U::key_codes(i, at.group));
    s8 = unit[U::key_scale(i, at.group)];
  }
  const float s = __low2float(cache::scales2(s8)) * cache::power2(at.is_value ? p.v_exp : p.k_exp);
  uint32_t lo[4], hi[4], w[8];
  cache::codes8((uint32_t)codes, lo);
  cache::codes8((uint32_t)(codes >> 32), hi);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 f = __half22float2(cache::half2_of(j < 4 ? lo[j % 4] : hi[j % 4]));
    w[j] = Two<T>::round(f.x * s, f.y * s);
  }
  dst += at.is_value ? at.token * p.v_s[0] + at.head * p.v_s[1] : at.token * p.k_s[0] + at.head * p.k_s[1];
  uint4* out = reinterpret_cast<uint4*>(dst + at.group * 16);
  out[0] = make_uint4(w[0], w[1], w[2], w[3]);
  out[1] = make_uint4(w[4], w[5], w[6], w[7]);
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
    if (x && (!st || !cache::aligned(x, 16) || !cache::strides_ok(st, 2))) return SOL_ERR_INVALID_ARG;
  }
  if (!slots || !cache::aligned(slots, 4)) return SOL_ERR_INVALID_ARG;
  if ((s = check_device_arch()) != SOL_OK) return s;
  WriteParams p{};
  p.k = k; p.v = v;
  for (int i = 0; i < 2; ++i) { p.k_s[i] = k ? ks[i] : 0; p.v_s[i] = v ? vs[i] : 0; }
  p.slots = slots;
  p.data = static_cast<unsigned char*>(c->data);
  if ((long long)tokens * c->Hk > 0x7fffffffLL) return SOL_ERR_UNSUPPORTED_SHAPE;
  p.rows = (uint32_t)tokens * (uint32_t)c->Hk;
  p.Hk = c->Hk; p.page_shift = cache::page_shift(c->page_size); p.slot_end = c->pages * c->page_size;
  p.k_exp = c->k_exp; p.v_exp = c->v_exp;
  const uint32_t per_block = kThreads / (2 * c->d / 16), blocks = (p.rows + per_block - 1) / per_block;
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

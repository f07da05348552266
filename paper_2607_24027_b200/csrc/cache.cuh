// The 4-bit key / value cache: layout, checks of its description, and the number formats of its entries.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace sol {
namespace cache {

constexpr int kUnit = 16;                        // tokens of a unit (see sol_attn.h)
constexpr int kGroup = 16;                       // channels that share a scale
constexpr int kMaxHeads = 1024;

__host__ __device__ constexpr int unit_bytes(int d) { return 18 * d; }

// Byte offsets in a unit of what belongs to a token and a group of 16 channels; `group` counts from 0 to d / 16 - 1.
template <int D>
struct Unit {
  static constexpr int kBytes = unit_bytes(D);
  static constexpr int kKeys = 0, kValues = 8 * D, kKeyScales = 16 * D, kValueScales = 17 * D;
  static constexpr int kPart = D / 16;           // bytes of a token's values that lie together: d / 8 channels
  __device__ static int key_codes(int token, int group) { return kKeys + token * (D / 2) + group * 8; }
  // A group is one part (d = 128) or two, the second of which lies kPartStride behind the first (d = 64).
  static constexpr int kPartStride = 8 * kPart;  // next g: four lanes of two tokens
  __device__ static int value_codes(int token, int group) {
    const int g = group * 8 / kPart, half = token >> 3, t = (token & 7) >> 1, e = token & 1;
    return kValues + (((half * 8 + g) * 4 + t) * 2 + e) * kPart;
  }
  __device__ static int key_scale(int token, int group) {
    constexpr int kPer = D / 64;
    return kKeyScales + (((token & 7) * 4 + group / kPer) * 2 + (token >> 3)) * kPer + group % kPer;
  }
  __device__ static int value_scale(int token, int group) {
    return kValueScales + (group * 4 + ((token & 7) >> 1)) * 4 + (token >> 3) * 2 + (token & 1);
  }
};

inline sol_status_t check(const sol_attn_cache* c) {
  if (!c || !c->data || (reinterpret_cast<uintptr_t>(c->data) & 15u)) return SOL_ERR_INVALID_ARG;
  if (c->k_exp < -64 || c->k_exp > 64 || c->v_exp < -64 || c->v_exp > 64) return SOL_ERR_INVALID_ARG;
  if (c->pages <= 0 || c->page_size <= 0 || c->Hk <= 0) return SOL_ERR_INVALID_ARG;
  return sol_attn_cache_bytes(c->pages, c->page_size, c->Hk, c->d) ? SOL_OK : SOL_ERR_UNSUPPORTED_SHAPE;
}

inline int page_shift(int page_size) {           // of a supported size
  int s = 4;
  while (1 << s < page_size) ++s;
  return s;
}
inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// Strides of dimensions with more than one entry are multiples of 8 elements.
inline bool strides_ok(const int64_t* s, int a, int b, int c = 1) {
  return (a <= 1 || s[0] % 8 == 0) && (b <= 1 || s[1] % 8 == 0) && (c <= 1 || s[2] % 8 == 0);
}
// Rows of an output do not lie on one another (as those of an expanded tensor do).
inline bool rows_apart(const int64_t* s, int a, int b, int c = 1) { return (a <= 1 || s[0]) && (b <= 1 || s[1]) && (c <= 1 || s[2]); }

#ifdef __CUDACC__
// Where a slot's unit of a head starts.
template <int D>
__device__ __forceinline__ size_t unit_at(int slot, int head, int page_shift, int heads) {
  const int page = slot >> page_shift, unit = (slot & ((1 << page_shift) - 1)) / kUnit;
  return (((size_t)((long long)page * heads + head) << (page_shift - 4)) + unit) * Unit<D>::kBytes;
}

// 16-bit types by name.
template <class T> struct Two;
template <> struct Two<__nv_bfloat16> {
  static constexpr uint32_t kInf = 0x7f80;       // bits of infinity
  __device__ static float2 widen(uint32_t x) { return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&x)); }
  __device__ static uint32_t round(float a, float b) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
};
template <> struct Two<__half> {
  static constexpr uint32_t kInf = 0x7c00;
  __device__ static float2 widen(uint32_t x) { return __half22float2(*reinterpret_cast<__half2*>(&x)); }
  __device__ static uint32_t round(float a, float b) {
    const __half2 r = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
};

// 2^e, -126 <= e <= 127.
__device__ __forceinline__ float power2(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ uint32_t bits(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }
__device__ __forceinline__ __half2 half2_of(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }

// The eight e2m1 numbers of a word, two of a byte to a register (the lower four bits first): exact in fp16.  Written with the word's
// bytes as operands the conversions need nothing beside them; with words that are shifted first each took one or two more instructions
// of the same pipe (a loop of them with its multiplications: 26 against 16 clocks a word and warp).
__device__ __forceinline__ void codes8(uint32_t w, uint32_t (&r)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(w));
}
// Two e4m3 numbers: exact in fp16.
__device__ __forceinline__ __half2 scales2(uint32_t two_bytes) {
  return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two_bytes, __NV_E4M3));
}
#endif

}  // namespace cache
}  // namespace sol

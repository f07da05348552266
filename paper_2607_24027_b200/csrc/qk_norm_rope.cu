// RMS norm of each head of q and k and the position rotation in one pass (sol_attn_qk_norm_rope).
//
// Bound by HBM: every element is read and written once.  A lane holds 8 channels (16 bytes) of a head, so d / 8 lanes hold a
// head and a warp 2 (d = 128) or 4 (d = 64) heads at a time; the partner channels of a pair are in the same lane, or rot / 16
// lanes further.  A warp keeps to one token, whose cos and sin it reads once for all of its heads.  (Next to HBM comes issuing the
// instructions: pairs of fp32 numbers go by one, and partners change places as 16-bit pairs.)
// 72 registers, for 28 warps an SM with four rows each on their way: 32 760 tokens x 80 heads of 128 channels 228 us, 5.9 TB/s; with 88
// registers 255.
#include "cache.cuh"

namespace sol {
namespace {

constexpr int kWarps = 4;
constexpr int kInFlight = 4;                     // head rows of a lane that are loaded before the first is used

struct NormParams {
  const void *q, *k;
  void *q_out, *k_out;
  long long q_s[3], k_s[3], qo_s[3], ko_s[3];
  const float *q_weight, *k_weight, *cos, *sin;
  const int32_t* positions;
  int batch, tokens, Hq, heads, rot, interleaved, table_rows, per_warp;   // heads: of q and k; per_warp: of them, a warp's share
  float eps;
};

template <class T, int D>
__global__ void __launch_bounds__(kWarps * 32, 7) qk_norm_rope_kernel(const __grid_constant__ NormParams p) {
  using cache::Two;
  constexpr int kLanes = D / 8, kRows = 32 / kLanes;
  const int lane = threadIdx.x % 32, sub = lane / kLanes, c0 = (lane % kLanes) * 8;
  const long long token = (long long)blockIdx.x * kWarps + threadIdx.x / 32;
  kernel_wait();
  if (token >= (long long)p.batch * p.tokens) return;
  const int b = (int)(token / p.tokens), n = (int)(token - (long long)b * p.tokens);
  const int pos = p.positions ? p.positions[token] : n;
  if (p.rot > 0 && (pos < 0 || pos >= p.table_rows)) return;
  const int half = p.rot / 2;
  // Pairs: the lane's channel i and its partner, i ^ 1 of the lane (interleaved), or channel i of lane `partner`.  With the norm r, weights w
  // and the partner's weights u, the result is r (x w cos +- y u sin): two factors per channel, formed once for all heads.
  const bool turns = c0 < p.rot, upper = !p.interleaved && c0 >= half;
  const int partner = p.interleaved || !turns ? lane : lane + (upper ? -half : half) / 8;
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  if (turns) {
    const size_t at = (size_t)pos * half + (p.interleaved ? c0 / 2 : (upper ? c0 - half : c0));
    const float4 x = __ldg(reinterpret_cast<const float4*>(p.cos + at)), y = __ldg(reinterpret_cast<const float4*>(p.sin + at));
    if (p.interleaved) {
      cs[0] = cs[1] = x.x; cs[2] = cs[3] = x.y; cs[4] = cs[5] = x.z; cs[6] = cs[7] = x.w;
      sn[0] = -y.x; sn[1] = y.x; sn[2] = -y.y; sn[3] = y.y; sn[4] = -y.z; sn[5] = y.z; sn[6] = -y.w; sn[7] = y.w;
    } else {
      const float4 x1 = __ldg(reinterpret_cast<const float4*>(p.cos + at + 4)), y1 = __ldg(reinterpret_cast<const float4*>(p.sin + at + 4));
      const float f = upper ? 1.f : -1.f;
      cs[0] = x.x; cs[1] = x.y; cs[2] = x.z; cs[3] = x.w; cs[4] = x1.x; cs[5] = x1.y; cs[6] = x1.z; cs[7] = x1.w;
      sn[0] = f * y.x; sn[1] = f * y.y; sn[2] = f * y.z; sn[3] = f * y.w; sn[4] = f * y1.x; sn[5] = f * y1.y; sn[6] = f * y1.z; sn[7] = f * y1.w;
    }
  }
  const int h_begin = blockIdx.y * p.per_warp, h_end = min(p.heads, h_begin + p.per_warp);
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {         // q, then k
    const int first = side ? max(h_begin, p.Hq) - p.Hq : h_begin, end = side ? h_end - p.Hq : min(h_end, p.Hq);
    if (first >= end) continue;
    const float* weight = side ? p.k_weight : p.q_weight;
    const T* src = (side ? (const T*)p.k + b * p.k_s[0] + n * p.k_s[1] : (const T*)p.q + b * p.q_s[0] + n * p.q_s[1]) + c0;
    T* dst = (side ? (T*)p.k_out + b * p.ko_s[0] + n * p.ko_s[1] : (T*)p.q_out + b * p.qo_s[0] + n * p.qo_s[1]) + c0;
    const long long from = side ? p.k_s[2] : p.q_s[2], to = side ? p.ko_s[2] : p.qo_s[2];
    float2 own[4], other[4];
    {
      float w[8], u[8];
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const float4 g = weight ? __ldg(reinterpret_cast<const float4*>(weight + c0 + i)) : make_float4(1.f, 1.f, 1.f, 1.f);
        w[i] = g.x; w[i + 1] = g.y; w[i + 2] = g.z; w[i + 3] = g.w;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = p.interleaved ? w[i ^ 1] : __shfl_sync(0xffffffffu, w[i], partner);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        own[i] = make_float2(w[2 * i] * cs[2 * i], w[2 * i + 1] * cs[2 * i + 1]);
        other[i] = make_float2(u[2 * i] * sn[2 * i], u[2 * i + 1] * sn[2 * i + 1]);
      }
    }
#pragma unroll 1
    for (int h0 = first; h0 < end; h0 += kRows * kInFlight) {
      uint4 raw[kInFlight];
#pragma unroll
      for (int v = 0; v < kInFlight; ++v) {
        const int h = h0 + v * kRows + sub;
        raw[v] = make_uint4(0, 0, 0, 0);
        if (h < end) raw[v] = *reinterpret_cast<const uint4*>(src + h * from);
      }
#pragma unroll
      for (int v = 0; v < kInFlight; ++v) {
        const int h = h0 + v * kRows + sub;
        if (h0 + v * kRows >= end) break;        // (the whole warp)
        const uint32_t w[4] = {raw[v].x, raw[v].y, raw[v].z, raw[v].w};
        float2 x[4], sum2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = Two<T>::widen(w[i]); sum2 = __ffma2_rn(x[i], x[i], sum2); }
        float sum = sum2.x + sum2.y;
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float r = rsqrtf(sum * (1.f / D) + p.eps);
        const float2 r2 = make_float2(r, r);
        uint32_t out[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 y = p.interleaved ? make_float2(x[i].y, x[i].x) : Two<T>::widen(__shfl_sync(0xffffffffu, w[i], partner));
          const float2 z = __ffma2_rn(__ffma2_rn(y, other[i], __ffma2_rn(x[i], own[i], make_float2(0.f, 0.f))), r2, make_float2(0.f, 0.f));
          out[i] = Two<T>::round(z.x, z.y);
        }
        if (h < end) *reinterpret_cast<uint4*>(dst + h * to) = make_uint4(out[0], out[1], out[2], out[3]);
      }
    }
  }
}

}  // namespace
}  // namespace sol

extern "C" sol_status_t sol_attn_qk_norm_rope(const sol_attn_norm_args* a) {
  using sol::cache::aligned;
  if (!a) return SOL_ERR_INVALID_ARG;
  if (a->batch < 0 || a->tokens < 0 || a->Hq < 0 || a->Hk < 0 || a->Hq + a->Hk <= 0) return SOL_ERR_INVALID_ARG;
  if (a->type != SOL_TYPE_BF16 && a->type != SOL_TYPE_FP16) return SOL_ERR_INVALID_ARG;
  if (!(a->eps >= 0.f) || a->rot < 0 || (a->rot > 0 && (!a->cos || !a->sin || a->table_rows <= 0))) return SOL_ERR_INVALID_ARG;
  if (a->Hq > sol::cache::kMaxHeads || a->Hk > sol::cache::kMaxHeads || (a->d != 64 && a->d != 128) || a->rot > a->d || a->rot % 16 ||
      (long long)a->batch * a->tokens > 0x7fffffffLL)
    return SOL_ERR_UNSUPPORTED_SHAPE;
  if (a->batch == 0 || a->tokens == 0) return SOL_OK;
  if ((a->Hq > 0 && (!a->q || !a->q_out)) || (a->Hk > 0 && (!a->k || !a->k_out))) return SOL_ERR_INVALID_ARG;
  for (const void* p : {a->q, a->k, (const void*)a->q_out, (const void*)a->k_out, (const void*)a->q_weight, (const void*)a->k_weight,
                        (const void*)a->cos, (const void*)a->sin})
    if (!aligned(p, 16)) return SOL_ERR_INVALID_ARG;
  if (!aligned(a->positions, 4)) return SOL_ERR_INVALID_ARG;
  const int B = a->batch, N = a->tokens;
  if (!sol::cache::strides_ok(a->q_stride, a->Hq ? B : 0, a->Hq ? N : 0, a->Hq) || !sol::cache::strides_ok(a->q_out_stride, a->Hq ? B : 0, a->Hq ? N : 0, a->Hq) ||
      !sol::cache::strides_ok(a->k_stride, a->Hk ? B : 0, a->Hk ? N : 0, a->Hk) || !sol::cache::strides_ok(a->k_out_stride, a->Hk ? B : 0, a->Hk ? N : 0, a->Hk))
    return SOL_ERR_INVALID_ARG;
  // In place each head lies where it lay; another order, or the other tensor's place, would be written while warps still read it.
  auto lies_as = [&](const void* in, const void* out, const int64_t* si, const int64_t* so, int H) {
    return in != out || ((B <= 1 || si[0] == so[0]) && (N <= 1 || si[1] == so[1]) && (H <= 1 || si[2] == so[2]));
  };
  if ((a->Hq && !sol::cache::rows_apart(a->q_out_stride, B, N, a->Hq)) || (a->Hk && !sol::cache::rows_apart(a->k_out_stride, B, N, a->Hk)))
    return SOL_ERR_INVALID_ARG;
  if (a->Hq && !lies_as(a->q, a->q_out, a->q_stride, a->q_out_stride, a->Hq)) return SOL_ERR_INVALID_ARG;
  if (a->Hk && !lies_as(a->k, a->k_out, a->k_stride, a->k_out_stride, a->Hk)) return SOL_ERR_INVALID_ARG;
  if (a->Hq && a->Hk && (a->q_out == a->k || a->k_out == a->q || a->q_out == a->k_out)) return SOL_ERR_INVALID_ARG;
  const sol_status_t s = sol::check_device_arch();
  if (s != SOL_OK) return s;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return SOL_ERR_CUDA;
  sol::NormParams p{};
  p.q = a->q; p.k = a->k; p.q_out = a->q_out; p.k_out = a->k_out;
  for (int i = 0; i < 3; ++i) {
    p.q_s[i] = a->q_stride[i]; p.k_s[i] = a->k_stride[i]; p.qo_s[i] = a->q_out_stride[i]; p.ko_s[i] = a->k_out_stride[i];
  }
  p.q_weight = a->q_weight; p.k_weight = a->k_weight; p.cos = a->cos; p.sin = a->sin; p.positions = a->positions;
  p.batch = a->batch; p.tokens = a->tokens; p.Hq = a->Hq; p.heads = a->Hq + a->Hk;
  p.rot = a->rot; p.interleaved = a->interleaved != 0; p.table_rows = a->table_rows; p.eps = a->eps;
  // Few tokens: a token's heads are shared out over warps until every SM has 16, down to one load of a warp.
  const long long tokens = (long long)a->batch * a->tokens;
  const int rows = 32 / (a->d / 8);
  int parts = 1;
  while (tokens * parts < 16LL * sms && parts * rows < p.heads) parts *= 2;
  p.per_warp = sol::ceil_div(sol::ceil_div(p.heads, parts), rows) * rows;
  const dim3 grid((unsigned)((tokens + sol::kWarps - 1) / sol::kWarps), (unsigned)sol::ceil_div(p.heads, p.per_warp));
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  auto run = [&](auto kernel) { return sol::launch_after(kernel, grid, sol::kWarps * 32, 0, 0, 0, stream, p); };
  const cudaError_t e = a->type == SOL_TYPE_BF16
      ? (a->d == 128 ? run(sol::qk_norm_rope_kernel<__nv_bfloat16, 128>) : run(sol::qk_norm_rope_kernel<__nv_bfloat16, 64>))
      : (a->d == 128 ? run(sol::qk_norm_rope_kernel<__half, 128>) : run(sol::qk_norm_rope_kernel<__half, 64>));
  sol::count_launches(1);
  return e == cudaSuccess ? SOL_OK : SOL_ERR_CUDA;
}

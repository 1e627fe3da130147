// attend_common.cuh -- what the kernels that write K/V rows share, and the attention kernel and the one that finishes its
// work.
#pragma once

#include "mma.cuh"

namespace kvx {
namespace {

// x / scale to the nearest: a product with the rounded reciprocal, corrected by its residual (Markstein, "Computation
// of elementary functions on the IBM RISC System/6000 processor", 1990).  Quotients that the 8 bits clamp are left as
// they are, as their residual may not be finite.
__device__ __forceinline__ float divided(float x, float scale, float inverse) {
  const float q = x * inverse;
  const float r = fmaf(fmaf(-q, scale, x), inverse, q);
  return fabsf(q) < 512.f ? r : q;
}
__device__ __forceinline__ uint32_t to_e4m3(float2 x, float scale, float inverse) {
  return __nv_cvt_float2_to_fp8x2(make_float2(divided(x.x, scale, inverse), divided(x.y, scale, inverse)), __NV_SATFINITE,
                                  __NV_E4M3);
}

// The sequence that row `token` of a step is of, and the rows from it to that sequence's last; false where there is none.
// A warp calls it as a whole.
__device__ __forceinline__ bool find_row(const int32_t* starts, int32_t num_seqs, int32_t new_tokens, int64_t token, int32_t* seq,
                                         int64_t* back) {
  if (!starts) {
    *seq = (int32_t)(token / new_tokens);
    *back = (int64_t)(*seq + 1) * new_tokens - token;
    return true;
  }
  const int lane = threadIdx.x & 31;
  int32_t lo = 0, hi = num_seqs;  // the last s with starts[s] <= token lies in [lo, hi)
  while (hi - lo > 1) {
    const int32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
    const uint32_t below = __ballot_sync(~0u, at < hi && starts[at] <= token);
    const int32_t n = 31 - __clz(below | 1);
    hi = min(hi, lo + (n + 1) * step);
    lo += n * step;
  }
  *seq = lo;
  *back = starts[lo + 1] - token;
  return token >= starts[lo] && *back > 0;
}

template <class Q>
__device__ __forceinline__ void write_out4(const AttendParams& p, int32_t s, int32_t h, int32_t r, int32_t col, float4 v) {
  const int32_t t = r / p.group, head = h * p.group + r % p.group;
  const int64_t token = (int64_t)s * p.new_tokens + t;
  uint2 o = make_uint2(pack2<Q>(v.x, v.y), pack2<Q>(v.z, v.w));
  *reinterpret_cast<uint2*>(p.out + token * p.out_token + head * p.out_head + col * 2) = o;
}
// Four neighbouring elements of a row's output.
__device__ __forceinline__ void write_out(const AttendParams& p, int32_t s, int32_t h, int32_t r, int32_t col, float4 v) {
  if (p.type == KVX_TYPE_BF16)
    write_out4<Bf16>(p, s, h, r, col, v);
  else
    write_out4<Fp16>(p, s, h, r, col, v);
}

// A row's logarithm of its sum l, which is relative to 2^m.
__device__ __forceinline__ void write_lse(const AttendParams& p, int32_t s, int32_t h, int32_t r, float m, float l) {
  const int32_t t = r / p.group, head = h * p.group + r % p.group;
  const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
  if (p.lse) p.lse[((int64_t)s * p.new_tokens + t) * p.q_heads + head] = lse2 * kLn2;
  if (p.weights) p.row_lse2[((int64_t)s * p.pages.heads + h) * (p.group * p.new_tokens) + r] = lse2;
}
__device__ __forceinline__ float factor(float m, float top) {  // 2^(m - top), 0 for a part without a key
  return m == -INFINITY ? 0.f : ex2(m - top);
}

}  // namespace
}  // namespace kvx

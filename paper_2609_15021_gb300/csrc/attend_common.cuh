// attend_common.cuh -- what the attention kernel and the kernel that finishes its work share.
#pragma once

#include "mma.cuh"

namespace kvx {
namespace {

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

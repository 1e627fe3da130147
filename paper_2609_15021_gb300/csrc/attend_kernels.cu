// attend_kernels.cu -- new tokens' K/V into the pages, and attention over them.

#include "operators.cuh"

namespace kvx {
namespace {

// ---------------------------------------------------------------- append

// Eight elements of one row a thread.  Bound by its bytes (a row in, a row out).
template <class In, bool kFp8>
__global__ void __launch_bounds__(256) append_kernel(const __grid_constant__ AppendParams p) {
  const PagesView& v = p.pages;
  const int32_t row_vecs = v.head_dim / 8, vecs = 2 * v.heads * row_vecs;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t token = i / vecs;
  if (token >= p.tokens) return;
  int32_t rest = (int32_t)(i - token * vecs);
  const int32_t half = rest / (v.heads * row_vecs);
  rest -= half * v.heads * row_vecs;
  const int32_t head = rest / row_vecs, col = (rest - head * row_vecs) * 8;
  int32_t s;
  int64_t back;  // rows of this sequence from this one to its last
  if (p.starts) {
    int32_t lo = 0, hi = p.num_seqs;  // the last s with starts[s] <= token
    while (hi - lo > 1) {
      const int32_t mid = (lo + hi) / 2;
      if (p.starts[mid] <= token) lo = mid; else hi = mid;
    }
    s = lo;
    back = p.starts[s + 1] - token;
    if (token < p.starts[s] || back <= 0) return;
  } else {
    s = (int32_t)(token / p.new_tokens);
    back = (int64_t)(s + 1) * p.new_tokens - token;
  }
  if (rest == 0 && half == 0) check_length(v, s);
  const int64_t pos = length_of(v, s) - back;
  if (pos < 0) return;
  const int64_t at = row_offset(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)pos);
  if (at < 0) return;
  const uint8_t* src = half ? p.value + token * p.value_token + head * p.value_head
                            : p.key + token * p.key_token + head * p.key_head;
  uint8_t* dst = v.base + at + half * v.half_bytes + head * v.head_bytes;
  const uint4 raw = *reinterpret_cast<const uint4*>(src + col * 2);
  if constexpr (!kFp8) {
    *reinterpret_cast<uint4*>(dst + col * 2) = raw;
  } else {
    const typename In::T* e = reinterpret_cast<const typename In::T*>(&raw);
    const float scale = half ? p.v_scale : p.k_scale;
    uint2 packed;
    uint8_t* o = reinterpret_cast<uint8_t*>(&packed);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      o[j] = (uint8_t)__nv_cvt_float_to_fp8(__fdiv_rn(In::up(e[j]), scale), __NV_SATFINITE, __NV_E4M3);
    *reinterpret_cast<uint2*>(dst + col) = packed;
  }
}

// ---------------------------------------------------------------- attention

constexpr float kLog2e = 1.4426950408889634f;

// A score's cap and bias.
__device__ __forceinline__ float finish_score(const AttendParams& p, float s, float slope, int32_t back) {
  if (p.softcap > 0.f) s = p.softcap * tanhf(s / p.softcap);
  return s - slope * back;
}

// One CTA per query row; each of 4 warps takes every fourth key, a lane up to 8
// elements of the rows, and the warps' softmax sums are joined at the end.
template <class Q, class C>
__global__ void __launch_bounds__(128) attend_kernel(const __grid_constant__ AttendParams p) {
  const PagesView& v = p.pages;
  __shared__ float top_s[4], sum_s[4], acc_s[4][256];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int32_t hq = blockIdx.x, s = blockIdx.y, t = blockIdx.z, h = hq / p.group;
  if (threadIdx.x == 0 && hq == 0 && t == 0) check_length(v, s);
  const int64_t token = (int64_t)s * p.new_tokens + t;
  const int32_t pos = length_of(v, s) - p.new_tokens + t;
  const int32_t lo = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
  const typename Q::T* q = reinterpret_cast<const typename Q::T*>(p.q + token * p.q_token + hq * p.q_head);
  const float slope = p.slopes ? p.slopes[hq] : 0.f;
  float qv[8], acc[8];
  for (int i = 0; i < 8; ++i) {
    qv[i] = lane + 32 * i < v.head_dim ? Q::up(q[lane + 32 * i]) : 0.f;
    acc[i] = 0.f;
  }
  float top = -INFINITY, sum = 0.f;
  for (int32_t j = lo + w; j <= pos; j += 4) {
    const int64_t at = row_offset(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)j);
    if (at < 0) continue;
    const typename C::T* key = reinterpret_cast<const typename C::T*>(v.base + at + h * v.head_bytes);
    const typename C::T* val = reinterpret_cast<const typename C::T*>(v.base + at + h * v.head_bytes + v.half_bytes);
    float d = 0.f;
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < v.head_dim) d += qv[i] * C::up(key[lane + 32 * i]);
    for (int m = 16; m; m >>= 1) d += __shfl_xor_sync(~0u, d, m);
    const float score = finish_score(p, d * p.scale * p.k_scale, slope, pos - j);
    const float now = fmaxf(top, score);
    const float keep = now == -INFINITY ? 0.f : exp2f((top - now) * kLog2e);
    const float e = now == -INFINITY ? 0.f : exp2f((score - now) * kLog2e);
    sum = sum * keep + e;
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < v.head_dim) acc[i] = acc[i] * keep + e * C::up(val[lane + 32 * i]);
    top = now;
  }
  for (int i = 0; i < 8; ++i)
    if (lane + 32 * i < v.head_dim) acc_s[w][lane + 32 * i] = acc[i];
  if (lane == 0) {
    top_s[w] = top;
    sum_s[w] = sum;
  }
  __syncthreads();
  top = fmaxf(fmaxf(top_s[0], top_s[1]), fmaxf(top_s[2], top_s[3]));
  sum = 0.f;
  float f[4];
  for (int i = 0; i < 4; ++i) {
    f[i] = top_s[i] == -INFINITY ? 0.f : exp2f((top_s[i] - top) * kLog2e);
    sum += f[i] * sum_s[i];
  }
  typename Q::T* out = reinterpret_cast<typename Q::T*>(p.out + token * p.out_token + hq * p.out_head);
  for (int i = threadIdx.x; i < v.head_dim; i += 128) {
    float o = 0.f;
    for (int k = 0; k < 4; ++k) o += f[k] * acc_s[k][i];
    out[i] = Q::down(sum > 0.f ? o / sum * p.v_scale : (sum == 0.f ? 0.f : sum));
  }
  if (threadIdx.x == 0 && p.lse) p.lse[token * p.q_heads + hq] = logf(sum) + (sum == 0.f ? 0.f : top);
}

// weights[s][h][j] += the rows' probabilities of key j: a warp per key.
template <class Q, class C>
__global__ void __launch_bounds__(128) weights_kernel(const __grid_constant__ AttendParams p) {
  const PagesView& v = p.pages;
  const int lane = threadIdx.x & 31;
  const int32_t h = blockIdx.y, s = blockIdx.z;
  const int32_t n = length_of(v, s);
  for (int32_t j = blockIdx.x * 4 + (threadIdx.x >> 5); j < n; j += gridDim.x * 4) {
    const int64_t at = row_offset(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)j);
    if (at < 0) continue;
    const typename C::T* key = reinterpret_cast<const typename C::T*>(v.base + at + h * v.head_bytes);
    float total = 0.f;
    for (int32_t r = 0; r < p.group * p.new_tokens; ++r) {
      const int32_t t = r / p.group, hq = h * p.group + r % p.group;
      const int64_t token = (int64_t)s * p.new_tokens + t;
      const int32_t pos = n - p.new_tokens + t;
      if (j > pos || (p.window > 0 && j <= pos - p.window)) continue;
      const typename Q::T* q = reinterpret_cast<const typename Q::T*>(p.q + token * p.q_token + hq * p.q_head);
      float d = 0.f;
      for (int i = lane; i < v.head_dim; i += 32) d += Q::up(q[i]) * C::up(key[i]);
      for (int m = 16; m; m >>= 1) d += __shfl_xor_sync(~0u, d, m);
      const float score = finish_score(p, d * p.scale * p.k_scale, p.slopes ? p.slopes[hq] : 0.f, pos - j);
      total += exp2f((score - p.lse[token * p.q_heads + hq]) * kLog2e);
    }
    if (lane == 0) p.weights[s * p.weights_seq + h * p.weights_head + j] += total;
  }
}

template <class Q, class C>
cudaError_t attend(const AttendParams& p, cudaStream_t s) {
  attend_kernel<Q, C><<<dim3(p.q_heads, p.pages.num_seqs, p.new_tokens), 128, 0, s>>>(p);
  if (p.weights)
    weights_kernel<Q, C><<<dim3(64, p.pages.heads, p.pages.num_seqs), 128, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_append(const AppendParams& p, int type, int cache_type, cudaStream_t s) {
  const int64_t n = p.tokens * 2 * p.pages.heads * (p.pages.head_dim / 8);
  const unsigned grid = (unsigned)((n + 255) / 256);
  if (cache_type != KVX_TYPE_E4M3)
    append_kernel<Bf16, false><<<grid, 256, 0, s>>>(p);
  else if (type == KVX_TYPE_BF16)
    append_kernel<Bf16, true><<<grid, 256, 0, s>>>(p);
  else
    append_kernel<Fp16, true><<<grid, 256, 0, s>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_attend(const AttendParams& p, int type, int cache_type, cudaStream_t s) {
  if (cache_type == KVX_TYPE_E4M3)
    return type == KVX_TYPE_BF16 ? attend<Bf16, E4m3>(p, s) : attend<Fp16, E4m3>(p, s);
  return type == KVX_TYPE_BF16 ? attend<Bf16, Bf16>(p, s) : attend<Fp16, Fp16>(p, s);
}

}  // namespace kvx

// attend_kernels.cu -- new tokens' K/V into the pages, and attention over them.

#include <algorithm>

#include "attend_common.cuh"

namespace kvx {
namespace {

// ---------------------------------------------------------------- append

constexpr int kAppendThreads = 128;

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

// A warp finds one token's sequence and place and moves its rows, or a quarter of them (kParts): bound by
// the rows' bytes, in and out.  A lane has four vectors in flight; a vector is 16 bytes of the cache's row,
// twice as much of an input that is narrowed.  16,384 tokens of 4 x 256 bf16 into e4m3 (101 MB): 18.8 us, 5.4 TB/s; with a
// quarter of the instructions' slots free, the narrowing is not far behind the bytes.
template <class In, bool kFp8, int kParts>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5), token = unit / kParts;
  if (token >= p.tokens) return;
  const int part = (int)(unit - token * kParts);
  int32_t s;
  int64_t back;  // rows of this sequence from this one to its last
  if (p.starts) {
    int32_t lo = 0, hi = p.num_seqs;  // the last s with starts[s] <= token lies in [lo, hi)
    while (hi - lo > 1) {
      const int32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
      const uint32_t below = __ballot_sync(~0u, at < hi && p.starts[at] <= token);
      const int32_t n = 31 - __clz(below | 1);
      hi = min(hi, lo + (n + 1) * step);
      lo += n * step;
    }
    s = lo;
    back = p.starts[s + 1] - token;
    if (token < p.starts[s] || back <= 0) return;
  } else {
    s = (int32_t)(token / p.new_tokens);
    back = (int64_t)(s + 1) * p.new_tokens - token;
  }
  if (lane == 0 && part == 0) check_length(v, s);
  const int64_t pos = length_of(v, s) - back;
  if (pos < 0) return;
  const uint32_t row = row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)pos);
  if (row == kNoRow) return;
  uint8_t* to = v.base + row * v.row_bytes;
  const uint8_t* from[2] = {p.key + token * p.key_token, p.value + token * p.value_token};
  const int64_t head_step[2] = {p.key_head, p.value_head};
  const uint32_t half_vecs = v.heads * p.row_vecs.d;  // of K, and of V
  const float inverse[2] = {1.f / p.k_scale, 1.f / p.v_scale};
  for (uint32_t i0 = part * 32 + lane; i0 < 2 * half_vecs; i0 += 4 * 32 * kParts) {
    uint4 raw[4][kFp8 ? 2 : 1];
    uint8_t* dst[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t i = i0 + u * 32 * kParts;
      dst[u] = nullptr;
      if (i < 2 * half_vecs) {
        const uint32_t half = i >= half_vecs, in = i - (half ? half_vecs : 0), head = quotient(p.row_vecs, in);
        const uint32_t col = (in - head * p.row_vecs.d) * 16;  // bytes of the cache's row
        const uint8_t* src = (half ? from[1] : from[0]) + head * (half ? head_step[1] : head_step[0]) + col * (kFp8 ? 2 : 1);
        raw[u][0] = __ldcs(reinterpret_cast<const uint4*>(src));
        if constexpr (kFp8) raw[u][1] = __ldcs(reinterpret_cast<const uint4*>(src) + 1);
        dst[u] = to + (half ? v.half_bytes : 0) + head * v.head_bytes + col;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (!dst[u]) continue;
      if constexpr (!kFp8) {
        *reinterpret_cast<uint4*>(dst[u]) = raw[u][0];
      } else {
        const bool half = i0 + u * 32 * kParts >= half_vecs;
        const float scale = half ? p.v_scale : p.k_scale, by = half ? inverse[1] : inverse[0];
        const uint32_t w[8] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w,
                               raw[u][1].x, raw[u][1].y, raw[u][1].z, raw[u][1].w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          o[k] = to_e4m3(unpack2<In>(w[2 * k]), scale, by) | to_e4m3(unpack2<In>(w[2 * k + 1]), scale, by) << 16;
        *reinterpret_cast<uint4*>(dst[u]) = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
  }
}

template <class In, bool kFp8>
cudaError_t append(const AppendParams& p, int num_sms, cudaStream_t s) {
  constexpr int kWarps = kAppendThreads / 32;
  // a warp per token where that fills the GPU, four where it does not (rows of 4 x 256 to e4m3: 1024 tokens 3.6 us against
  // 3.2, 2048 tokens 4.3 against 5.1)
  if (p.tokens >= 10 * num_sms)
    return launch_after(append_kernel<In, kFp8, 1>, dim3((unsigned)((p.tokens + kWarps - 1) / kWarps)), kAppendThreads, 0, s, p);
  return launch_after(append_kernel<In, kFp8, 4>, dim3((unsigned)((p.tokens * 4 + kWarps - 1) / kWarps)), kAppendThreads, 0, s, p);
}

// ---------------------------------------------------------------- the end of an attention

constexpr int kFinishThreads = 256;

__device__ __forceinline__ const float* part_of(const AttendParams& p, int2 item, int32_t c) {
  const int64_t slot = c ? (item.x / 2 + c) * 2 : item.x;
  return p.parts + slot * (p.part_rows * (p.part_dim + 2));
}

// A row's logarithm of the sum, from its item's parts (a warp).
__device__ __forceinline__ float joined_lse2(const AttendParams& p, int2 item, int32_t row) {
  const int lane = threadIdx.x & 31;
  float top = -INFINITY, sum = 0.f;
  for (int32_t c = lane; c < item.y; c += 32) {
    const float2 ml = *reinterpret_cast<const float2*>(part_of(p, item, c) + p.part_rows * p.part_dim + 2 * row);
    const float now = fmaxf(top, ml.x);
    sum = sum * factor(top, now) + ml.y * factor(ml.x, now);
    top = now;
  }
  float all = top;
  for (int d = 16; d; d >>= 1) all = fmaxf(all, __shfl_xor_sync(~0u, all, d));
  sum *= factor(top, all);
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
  return sum == 0.f ? -INFINITY : all + log2f(sum);
}

// CTAs below `join` join the parts of one query row each: threads by (part, four columns), parts in order
// within a thread and threads in order after that.  The others add a stretch of keys' attention
// weights, a thread per key, so that every sum has one order:
//   weights[s][h][j] += sum over the head's rows of 2^(score - lse2), scores as the attention left them.
// Bound by latency: three dependent loads (an item, its parts' sums, the parts) in 3 to 6 us, some 9 with the weights of
// 53.8k tokens x 8 heads of 8 rows (14 MB of scores).  Four CTAs of weights an SM: seven took as long.
__global__ void __launch_bounds__(kFinishThreads) finish_kernel(const __grid_constant__ AttendParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  const int32_t rows = p.group * p.new_tokens, blocks = (rows + p.part_rows - 1) / p.part_rows;
  const int32_t heads_all = v.heads * v.num_seqs;
  const int64_t join = (int64_t)heads_all * rows;
  __shared__ float4 o_s[kFinishThreads];
  __shared__ float m_s[kFinishThreads], l_s[kFinishThreads];
  if (blockIdx.x < join) {
    const int32_t sh = blockIdx.x / rows, r = blockIdx.x - sh * rows, in = r % p.part_rows;
    const int2 item = p.items[(int64_t)sh * blocks + r / p.part_rows];
    if (item.y == 0) return;
    const int32_t cols = p.part_dim / 4, col = threadIdx.x % cols, groups = kFinishThreads / cols;
    float top = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int32_t c = threadIdx.x / cols; c < item.y; c += groups) {
      const float* part = part_of(p, item, c);
      const float2 ml = *reinterpret_cast<const float2*>(part + p.part_rows * p.part_dim + 2 * in);
      const float4 x = *reinterpret_cast<const float4*>(part + in * p.part_dim + 4 * col);
      const float now = fmaxf(top, ml.x), f0 = factor(top, now), f1 = factor(ml.x, now);
      sum = sum * f0 + ml.y * f1;
      o.x = o.x * f0 + x.x * f1, o.y = o.y * f0 + x.y * f1, o.z = o.z * f0 + x.z * f1, o.w = o.w * f0 + x.w * f1;
      top = now;
    }
    o_s[threadIdx.x] = o, m_s[threadIdx.x] = top, l_s[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= cols) return;
    for (int32_t g = 1; g < groups; ++g) {
      const int32_t i = g * cols + col;
      const float now = fmaxf(top, m_s[i]), f0 = factor(top, now), f1 = factor(m_s[i], now);
      const float4 x = o_s[i];
      sum = sum * f0 + l_s[i] * f1;
      o.x = o.x * f0 + x.x * f1, o.y = o.y * f0 + x.y * f1, o.z = o.z * f0 + x.z * f1, o.w = o.w * f0 + x.w * f1;
      top = now;
    }
    const float by = sum == 0.f ? 0.f : p.v_scale / sum;
    if (sum == 0.f) o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (4 * col < v.head_dim)
      write_out(p, sh / v.heads, sh % v.heads, r, 4 * col, make_float4(o.x * by, o.y * by, o.z * by, o.w * by));
    if (col == 0 && p.lse) {
      const int32_t head = sh % v.heads * p.group + r % p.group;
      p.lse[((int64_t)(sh / v.heads) * p.new_tokens + r / p.group) * p.q_heads + head] =
          (sum == 0.f ? -INFINITY : top + log2f(sum)) * kLn2;
    }
    return;
  }
  const int32_t chunks = (int32_t)((gridDim.x - join) / heads_all);
  const int32_t rest = (int32_t)(blockIdx.x - join), sh = rest / chunks, chunk = rest - sh * chunks;
  const int32_t s = sh / v.heads, h = sh - s * v.heads, length = length_of(v, s);
  const int32_t from = p.window > 0 ? max(0, length - p.new_tokens + 1 - p.window) : 0;
  const float* scores = p.scores + (int64_t)sh * p.score_rows * p.score_stride;
  float* weights = p.weights + s * p.weights_seq + h * p.weights_head;
  for (int32_t r0 = 0; r0 < rows; r0 += kFinishThreads) {  // rows whose sums are kept at once
    const int32_t n = min(rows - r0, kFinishThreads);
    // the first key's scores and weight do not wait for the sums
    int32_t j = from + chunk * kFinishThreads + threadIdx.x;
    float2 ahead[4];
    float before = 0.f;
    auto load = [&]() {
      if (j >= length) return;
      const float2* row = reinterpret_cast<const float2*>(scores + (int64_t)j * p.score_rows + r0);
      before = weights[j];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (2 * k < n) ahead[k] = row[k];
    };
    load();
    __syncthreads();
    for (int32_t r = threadIdx.x >> 5; r < n; r += kFinishThreads / 32) {
      const int2 item = p.items[(int64_t)sh * blocks + (r0 + r) / p.part_rows];
      const float lse2 = item.y == 0 ? p.row_lse2[(int64_t)sh * rows + r0 + r] : joined_lse2(p, item, (r0 + r) % p.part_rows);
      if ((threadIdx.x & 31) == 0) l_s[r] = lse2;
    }
    __syncthreads();
    for (; j < length; j += chunks * kFinishThreads, load()) {
      const float2* row = reinterpret_cast<const float2*>(scores + (int64_t)j * p.score_rows + r0);
      float sum = 0.f;
      auto add = [&](float2 x, int32_t r) {
        if (x.x != -INFINITY) sum += ex2(x.x - l_s[r]);
        if (r + 1 < n && x.y != -INFINITY) sum += ex2(x.y - l_s[r + 1]);
      };
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (2 * k < n) add(ahead[k], 2 * k);
      for (int32_t r = 8; r < n; r += 2) add(row[r / 2], r);
      weights[j] = before + sum;
    }
  }
}

}  // namespace

cudaError_t launch_append(const AppendParams& p, int type, int cache_type, int num_sms, cudaStream_t s) {
  if (cache_type != KVX_TYPE_E4M3) return append<Bf16, false>(p, num_sms, s);  // bytes
  return type == KVX_TYPE_BF16 ? append<Bf16, true>(p, num_sms, s) : append<Fp16, true>(p, num_sms, s);
}

cudaError_t launch_attend(const AttendParams& p, int cache_type, int num_sms, cudaStream_t s) {
  const cudaError_t e = cache_type == KVX_TYPE_E4M3   ? launch_attend_e4m3(p, num_sms, s)
                        : cache_type == KVX_TYPE_BF16 ? launch_attend_bf16(p, num_sms, s)
                                                      : launch_attend_fp16(p, num_sms, s);
  if (e != cudaSuccess) return e;
  const int64_t heads_all = (int64_t)p.pages.heads * p.pages.num_seqs;
  int64_t grid = heads_all * p.group * p.new_tokens;
  if (p.weights) {
    const int64_t most = (p.pages.max_length + kFinishThreads - 1) / kFinishThreads;
    grid += heads_all * std::max<int64_t>(1, std::min(most, 4 * num_sms / heads_all));
  }
  return launch_after(finish_kernel, dim3((unsigned)grid), kFinishThreads, 0, s, p);
}

cudaError_t prepare_attend_kernels() {
  cudaError_t e = prepare_attend_bf16();
  if (e == cudaSuccess) e = prepare_attend_fp16();
  return e == cudaSuccess ? prepare_attend_e4m3() : e;
}

}  // namespace kvx

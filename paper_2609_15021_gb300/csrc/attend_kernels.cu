// attend_kernels.cu -- new tokens' K/V into the pages, and attention over them.

#include <algorithm>

#include "attend_common.cuh"

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
  const uint32_t at = row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)pos);
  if (at == kNoRow) return;
  const uint8_t* src = half ? p.value + token * p.value_token + head * p.value_head
                            : p.key + token * p.key_token + head * p.key_head;
  uint8_t* dst = v.base + at * v.row_bytes + half * v.half_bytes + head * v.head_bytes;
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
    __syncthreads();
    for (int32_t r = threadIdx.x >> 5; r < n; r += kFinishThreads / 32) {
      const int2 item = p.items[(int64_t)sh * blocks + (r0 + r) / p.part_rows];
      const float lse2 = item.y == 0 ? p.row_lse2[(int64_t)sh * rows + r0 + r] : joined_lse2(p, item, (r0 + r) % p.part_rows);
      if ((threadIdx.x & 31) == 0) l_s[r] = lse2;
    }
    __syncthreads();
    for (int32_t j = from + chunk * kFinishThreads + threadIdx.x; j < length; j += chunks * kFinishThreads) {
      const float2* row = reinterpret_cast<const float2*>(scores + (int64_t)j * p.score_rows + r0);
      float sum = 0.f;
      for (int32_t r = 0; r < n; r += 2) {
        const float2 x = row[r / 2];
        if (x.x != -INFINITY) sum += ex2(x.x - l_s[r]);
        if (r + 1 < n && x.y != -INFINITY) sum += ex2(x.y - l_s[r + 1]);
      }
      weights[j] += sum;
    }
  }
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

cudaError_t launch_attend(const AttendParams& p, int cache_type, int num_sms, cudaStream_t s) {
  const cudaError_t e = cache_type == KVX_TYPE_E4M3   ? launch_attend_e4m3(p, num_sms, s)
                        : cache_type == KVX_TYPE_BF16 ? launch_attend_bf16(p, num_sms, s)
                                                      : launch_attend_fp16(p, num_sms, s);
  if (e != cudaSuccess) return e;
  const int64_t heads_all = (int64_t)p.pages.heads * p.pages.num_seqs;
  int64_t grid = heads_all * p.group * p.new_tokens;
  if (p.weights) {
    const int64_t most = (p.pages.max_length + kFinishThreads - 1) / kFinishThreads;
    grid += heads_all * std::max<int64_t>(1, std::min(most, 8 * num_sms / heads_all));
  }
  return launch_after(finish_kernel, dim3((unsigned)grid), kFinishThreads, 0, s, p);
}

cudaError_t prepare_attend_kernels() {
  cudaError_t e = prepare_attend_bf16();
  if (e == cudaSuccess) e = prepare_attend_fp16();
  return e == cudaSuccess ? prepare_attend_e4m3() : e;
}

}  // namespace kvx

// attend_kernels.cu -- new tokens' K/V into the pages, and attention over them.

#include <algorithm>

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

// ---------------------------------------------------------------- attention weights

// weights[s][h][j] += sum over the head's query rows of exp2(score - lse2), from the
// scores that the attention left: a thread per key, so the sums have one order.
__global__ void __launch_bounds__(256) weights_kernel(const __grid_constant__ AttendParams p) {
  const PagesView& v = p.pages;
  const int32_t h = blockIdx.y, s = blockIdx.z, rows = p.group * p.new_tokens;
  const int32_t length = length_of(v, s);
  const int32_t from = p.window > 0 ? max(0, length - p.new_tokens + 1 - p.window) : 0;
  const int64_t item = (int64_t)s * v.heads + h;
  const float* scores = p.scores + item * p.score_rows * p.score_stride;
  const float* lse2 = p.row_lse2 + item * rows;
  float* weights = p.weights + s * p.weights_seq + h * p.weights_head;
  for (int32_t j = from + blockIdx.x * 256 + threadIdx.x; j < length; j += gridDim.x * 256) {
    float sum = 0.f;
    const float2* row = reinterpret_cast<const float2*>(scores + (int64_t)j * p.score_rows);
    for (int32_t r = 0; r < rows; r += 2) {
      const float2 x = row[r / 2];
      if (x.x != -INFINITY) sum += exp2f(x.x - lse2[r]);
      if (r + 1 < rows && x.y != -INFINITY) sum += exp2f(x.y - lse2[r + 1]);
    }
    weights[j] += sum;
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
  if (e != cudaSuccess || !p.weights) return e;
  const int32_t items = p.pages.heads * p.pages.num_seqs;
  const int32_t most = (p.pages.max_length + 255) / 256;
  const int32_t chunks = std::max(1, std::min(most, 16 * num_sms / items));
  weights_kernel<<<dim3(chunks, p.pages.heads, p.pages.num_seqs), 256, 0, s>>>(p);
  return cudaGetLastError();
}

cudaError_t prepare_attend_kernels() {
  cudaError_t e = prepare_attend_bf16();
  if (e == cudaSuccess) e = prepare_attend_fp16();
  return e == cudaSuccess ? prepare_attend_e4m3() : e;
}

}  // namespace kvx

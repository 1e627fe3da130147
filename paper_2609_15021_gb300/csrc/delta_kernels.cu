// delta_kernels.cu -- the gated delta rule token by token, and which sequences go by chunks.
//
//   S_t = a_t S_{t-1} + b_t (v_t - a_t S_{t-1} k_t) k_t^T,   y_t = S_t q_t
#include <algorithm>

#include "delta_common.cuh"

namespace kvx {
namespace {

template <class E, int N, int kRows, bool kPacked>
__global__ void __launch_bounds__(128) delta_kernel(const __grid_constant__ DeltaParams p) {
  wait_for_previous();
  by_tokens<E, N, kRows, kPacked>(p, blockIdx.x, blockIdx.y, blockIdx.z);
}

template <class E, int N>
cudaError_t delta(const DeltaParams& p, int num_sms, cudaStream_t s) {
  constexpr int kSub = kTokenSub<N>;
  constexpr int kMany = N == 16 ? 4 : N == 256 ? 4 : 8, kFew = 2;
  const bool many = (int64_t)p.state.num_seqs * p.heads * p.head_dim >= (int64_t)num_sms * 4 * kSub * kMany;
  const int rows = 4 * kSub * (many ? kMany : kFew);
  const dim3 grid((p.head_dim + rows - 1) / rows, p.heads, p.state.num_seqs);
  const auto kernel = p.state.starts ? (many ? delta_kernel<E, N, kMany, true> : delta_kernel<E, N, kFew, true>)
                                     : (many ? delta_kernel<E, N, kMany, false> : delta_kernel<E, N, kFew, false>);
  return launch_after(kernel, grid, 128, 0, s, p);
}

template <class E>
cudaError_t delta(const DeltaParams& p, int num_sms, cudaStream_t s) {
  switch (p.state_dim) {
    case 16: return delta<E, 16>(p, num_sms, s);
    case 32: return delta<E, 32>(p, num_sms, s);
    case 64: return delta<E, 64>(p, num_sms, s);
    case 128: return delta<E, 128>(p, num_sms, s);
    default: return delta<E, 256>(p, num_sms, s);
  }
}

}  // namespace

bool delta_by_chunks(int64_t tokens, int32_t num_seqs, bool packed, int32_t state_dim, int32_t* by_token) {
  // 16 heads of 128 x 128: a sequence of 16 tokens takes 10 us token by token and 12 by chunks, which take no longer for 64, 24 tokens
  // 16; sixteen sequences of 16 tokens 47 us and 78, of 32 tokens 117 and 74.
  const int32_t few = num_seqs > 1 ? 24 : 16;
  *by_token = INT32_MAX;
  if (!packed || (state_dim != 64 && state_dim != 128) || tokens <= few) return false;
  *by_token = num_seqs > 1 ? few : -1;
  return true;
}

cudaError_t launch_delta(const DeltaParams& p, int type, int num_sms, cudaStream_t s) {
  if (p.pieces) return launch_delta_chunks(p, type, s);
  return type == KVX_TYPE_BF16 ? delta<Bf16>(p, num_sms, s) : delta<Fp16>(p, num_sms, s);
}

}  // namespace kvx

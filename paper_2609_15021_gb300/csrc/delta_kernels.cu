// delta_kernels.cu -- the gated delta rule token by token, and which sequences go by chunks.
//
//   S_t = a_t S_{t-1} + b_t (v_t - a_t S_{t-1} k_t) k_t^T,   y_t = S_t q_t
//
// Rows of the state know nothing of one another, and stay in registers from the first token of a sequence to the last.  One token
// of each sequence is bound by the state's bytes: 96 sequences of 16 heads x 128 x 128 (201 MB) take 34 us, 89 % of the DRAM's
// rate; of several tokens a chain of two sums over a row and what the token before wrote, 0.6 us a token.
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
  // Rows of a warp at once: 8, that many loads are in flight (96 sequences of a token 35 us in a graph, 49 with 2), or 2 where there
  // are too few rows for all SMs (a sequence of 16 tokens 14.5 us, and 16.4).  A row of 16 has four lanes, which end the sums of
  // four rows, and eight rows of 256 would take 165 registers a thread.
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
  // A chunk takes the same for 8 tokens as for 64, so both meet at some number of tokens: at 20 of one sequence and 22 of two (16
  // heads of 128 x 128), at 34 to 38 of four to sixteen; of 8 heads at 22 for up to four sequences, of 16 of 64 x 64 at 18, 22, 27, 32 and 42 for one
  // to sixteen.  In a graph, us token by token and by chunks, of 16 heads of 128 x 128: one of 16 tokens 11.9 and 14.2, of 24 16.6 and
  // 14.2; two of 24 20.9 and 19.5; four of 24 21.8 and 29.4, of 32 27.9 and 29.6; sixteen of 24 52 and 79, of 32 68 and 79.  24 is near
  // where few sequences meet; that many of 25 to 34 tokens go by chunks costs them up to a third.
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

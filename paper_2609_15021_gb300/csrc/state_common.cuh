// state_common.cuh -- what the kernels on state slots share.
#pragma once

#include "mma.cuh"

namespace kvx {
namespace {

// The piece'th of all sequences' pieces of `length` rows (at least one a sequence), counted in their order:
// its sequence, its place there, and how many pieces that sequence has.  False behind the last.  Found by the
// whole CTA; buf: a word a warp and three more.
template <int kThreads>
__device__ __forceinline__ bool find_piece(const StateView& v, int32_t piece, int32_t length, int32_t* buf, int32_t* seq,
                                           int32_t* at, int32_t* of) {
  if (!v.starts) {
    *seq = piece, *at = 0, *of = 1;
    return piece < v.num_seqs;
  }
  if (v.num_seqs == 1) {
    int64_t first, last;
    rows_of(v, 0, &first, &last);
    *seq = 0, *at = piece, *of = max(1, (int32_t)((last - first + length - 1) / length));
    return piece < *of;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kWarps = kThreads / 32;
  int32_t before_all = 0;
  for (int32_t base = 0; base < v.num_seqs; base += kThreads) {
    const int32_t s = base + threadIdx.x;
    int32_t mine = 0;
    if (s < v.num_seqs) {
      int64_t first, last;
      rows_of(v, s, &first, &last);
      mine = max(1, (int32_t)((last - first + length - 1) / length));
    }
    int32_t upto = mine;
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t y = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += y;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = upto;
    if (threadIdx.x == 0) buf[kWarps] = -1;
    __syncthreads();
    int32_t chunk = 0;
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) upto += buf[i];
      chunk += buf[i];
    }
    const int32_t from = before_all + upto - mine;
    if (piece >= from && piece < from + mine) {
      buf[kWarps] = s;
      buf[kWarps + 1] = piece - from;
      buf[kWarps + 2] = mine;
    }
    __syncthreads();
    if (buf[kWarps] >= 0) {
      *seq = buf[kWarps], *at = buf[kWarps + 1], *of = buf[kWarps + 2];
      return true;
    }
    before_all += chunk;
  }
  return false;
}

__device__ __forceinline__ float step_of(const ScanParams& p, float raw, int32_t h) {
  if (p.dt_bias) raw += p.dt_bias[h];
  return p.softplus ? (raw > 20.f ? raw : log1pf(expf(raw))) : raw;
}

}  // namespace
}  // namespace kvx

// state_common.cuh -- what the kernels on state slots share.
#pragma once

#include "mma.cuh"

namespace kvx {
namespace {

// A piece of a sequence, and what a kernel asks about it.
struct Piece {
  int32_t seq, at, of;   // the at'th of its sequence's pieces, `of` in all
  int64_t first, last;   // the sequence's rows
  const uint8_t* in;     // its slots; null where one of them is out of range
  uint8_t* keep;
  bool fresh;
};
__device__ __forceinline__ int32_t pieces_of(int64_t first, int64_t last, int32_t length, int32_t none_up_to) {
  return last - first <= none_up_to ? 0 : max(1, (int32_t)((last - first + length - 1) / length));
}

// The piece'th of all sequences' pieces of `length` rows (at least one of a sequence longer than none_up_to), counted
// in their order: False behind the last.  Up to 32 sequences are looked at by every warp for itself, with one round of loads;
// more by the whole CTA.  buf: a word a warp and three more.
template <int kThreads>
__device__ __forceinline__ bool find_piece(const StateView& v, int32_t piece, int32_t length, int32_t none_up_to, int32_t* buf,
                                           Piece* found) {
  if (v.starts && v.num_seqs <= 32) {
    const int lane = threadIdx.x & 31;
    const bool there = lane < v.num_seqs;
    int64_t first = 0, last = 0;
    int32_t from_slot = 0, to_slot = 0, fresh = 0;
    if (there) {
      rows_of(v, lane, &first, &last);
      from_slot = v.slots_in[lane], to_slot = v.slots_out[lane];
      if (v.fresh) fresh = v.fresh[lane];
    }
    const int32_t mine = there ? pieces_of(first, last, length, none_up_to) : 0;
    int32_t upto = mine;
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t y = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += y;
    }
    const uint32_t at_or_after = __ballot_sync(~0u, piece < upto);
    if (at_or_after == 0) return false;
    const int owner = __ffs(at_or_after) - 1;
    found->seq = owner;
    found->of = __shfl_sync(~0u, mine, owner);
    found->at = piece - (__shfl_sync(~0u, upto, owner) - found->of);
    found->first = __shfl_sync(~0u, first, owner);
    found->last = __shfl_sync(~0u, last, owner);
    found->in = slot_at(v, __shfl_sync(~0u, from_slot, owner), owner);
    found->keep = slot_at(v, __shfl_sync(~0u, to_slot, owner), owner);
    found->fresh = __shfl_sync(~0u, fresh, owner);
    return true;
  }
  auto rest = [&](int32_t s, int32_t at, int32_t of) {
    found->seq = s, found->at = at, found->of = of;
    rows_of(v, s, &found->first, &found->last);
    found->in = slot_of(v, v.slots_in, s);
    found->keep = slot_of(v, v.slots_out, s);
    found->fresh = v.fresh && v.fresh[s];
    return true;
  };
  if (!v.starts) return piece < v.num_seqs && rest(piece, 0, 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kWarps = kThreads / 32;
  int32_t before_all = 0;
  for (int32_t base = 0; base < v.num_seqs; base += kThreads) {
    const int32_t s = base + threadIdx.x;
    int32_t mine = 0;
    if (s < v.num_seqs) {
      int64_t first, last;
      rows_of(v, s, &first, &last);
      mine = pieces_of(first, last, length, none_up_to);
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
    if (buf[kWarps] >= 0) return rest(buf[kWarps], buf[kWarps + 1], buf[kWarps + 2]);
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

// delta_common.cuh -- the gated delta rule token by token, and what its kernels share.
//
// A state row (an element of v) knows nothing of the others, and with what it holds for both vectors, s.k and s.q, taken in one
// pass over it,
//   d = b (v - a s.k),   y = a s.q + d (k.q),   s = a s + d k.
// A row lies over kLanes lanes, 16 bytes each at least, and a lane has kRows rows, whose loads are all in flight at once.  The
// rows' sums meet in a reduction that halves the rows at every step; a row's d goes back to its lanes by as many shuffles
// as there are rows.  Bound by the state's bytes, read and written once.
#pragma once

#include "state_common.cuh"

namespace kvx {
namespace {

__device__ __forceinline__ float decay_of(const DeltaParams& p, float raw, int32_t h) {  // its logarithm
  if (p.dt_bias) raw += p.dt_bias[h];
  return (p.softplus ? (raw > 20.f ? raw : log1pf(expf(raw))) : raw) * p.A[h];
}
__device__ __forceinline__ float step_size(const DeltaParams& p, float raw) { return p.sigmoid ? 1.f / (1.f + expf(-raw)) : raw; }

// Sums of kRows values a lane over the kLanes lanes of a row: lanes that differ in one bit exchange halves of their
// values, then, with one left, its halves.  A lane ends with the sum of value *mine.
template <int kRows, int kLanes>
__device__ __forceinline__ float meet(float (&y)[kRows], int lane, int* mine) {
  int m = kLanes / 2, at = 0;
#pragma unroll
  for (int left = kRows; left > 1; left /= 2, m /= 2) {
    const bool upper = lane & m;
    at = 2 * at + upper;
#pragma unroll
    for (int r = 0; r < left / 2; ++r) {
      const float send = upper ? y[r] : y[r + left / 2], stay = upper ? y[r + left / 2] : y[r];
      y[r] = stay + __shfl_xor_sync(~0u, send, m);
    }
  }
#pragma unroll
  for (int k = m; k; k >>= 1) y[0] += __shfl_xor_sync(~0u, y[0], k);
  *mine = at;
  return y[0];
}

// Rows of a head of a sequence that goes token by token, 4 kRows kSub of them for 128 threads.
template <int N>
constexpr int kTokenSub = N / 4 < 32 ? 128 / N : 1;  // rows that a warp has side by side
template <class E, int N, int kRows, bool kPacked>  // kPacked: sequences have several tokens
__device__ __forceinline__ void by_tokens(const DeltaParams& p, int32_t block, int32_t h, int32_t s) {
  using T = typename E::T;
  constexpr int kLanes = N / 4 < 32 ? N / 4 : 32, kVec = N / kLanes, kSub = kTokenSub<N>;
  static_assert(kRows <= kLanes, "a row's sum ends in a lane");
  const int lane = threadIdx.x & 31, sub = lane / kLanes, in_row = lane % kLanes, col = in_row * kVec;
  const int32_t row0 = (block * 4 + (threadIdx.x >> 5)) * kRows * kSub + sub;  // rows row0 + r * kSub
  const StateView& v = p.state;
  const uint8_t* in = slot_of(v, v.slots_in, s);
  uint8_t* keep = slot_of(v, v.slots_out, s);
  int64_t first, last;
  rows_of(v, s, &first, &last);
  if (last - first > p.by_token) return;
  T* out = reinterpret_cast<T*>(p.out) + h * p.out_head;
  if (!in || !keep) {
    for (int64_t t = first; t < last; ++t)
      for (int r = 0; r < kRows; ++r)
        if (in_row == 0 && row0 + r * kSub < p.head_dim) out[t * p.out_token + row0 + r * kSub] = E::down(0.f);
    return;
  }
  const bool fresh = v.fresh && v.fresh[s];
  const int64_t at = ((int64_t)h * p.head_dim + row0) * N + col;
  float state[kRows][kVec];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int i = 0; i < kVec; i += 4) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (!fresh && row0 + r * kSub < p.head_dim)
        x = __ldcs(reinterpret_cast<const float4*>(in) + (at + r * kSub * N + i) / 4);
      state[r][i] = x.x, state[r][i + 1] = x.y, state[r][i + 2] = x.z, state[r][i + 3] = x.w;
    }
  const int32_t group = h / p.heads_per_group;
  const T* q_at = reinterpret_cast<const T*>(p.q) + group * p.q_head + col;
  const T* k_at = reinterpret_cast<const T*>(p.k) + group * p.k_head + col;
  const T* v_at = reinterpret_cast<const T*>(p.v) + h * p.v_head;
  // A token's rows, loaded while the one before it is at work.
  struct Token {
    uint32_t q[kVec / 2], k[kVec / 2];
    T v[kRows], dt, beta;
  };
  auto load = [&](int64_t t, Token& to) {
#pragma unroll
    for (int i = 0; i < kVec / 2; ++i) {
      to.q[i] = *reinterpret_cast<const uint32_t*>(q_at + t * p.q_token + 2 * i);
      to.k[i] = *reinterpret_cast<const uint32_t*>(k_at + t * p.k_token + 2 * i);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      if (row0 + r * kSub < p.head_dim) to.v[r] = v_at[t * p.v_token + row0 + r * kSub];
    if (p.dt) to.dt = reinterpret_cast<const T*>(p.dt)[t * p.dt_token + h];
    to.beta = reinterpret_cast<const T*>(p.beta)[t * p.beta_token + h];
  };
  Token now, next;
  if (!kPacked || first < last) load(first, now);
  for (int64_t t = first; t < (kPacked ? last : first + 1); ++t) {
    if (kPacked && t + 1 < last) load(t + 1, next);
    float q[kVec], k[kVec];
#pragma unroll
    for (int i = 0; i < kVec; i += 2) {
      const float2 a = unpack2<E>(now.q[i / 2]), b = unpack2<E>(now.k[i / 2]);
      q[i] = a.x, q[i + 1] = a.y, k[i] = b.x, k[i + 1] = b.y;
    }
    float x[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) x[r] = row0 + r * kSub < p.head_dim ? E::up(now.v[r]) : 0.f;
    const float decay = p.dt ? expf(decay_of(p, E::up(now.dt), h)) : 1.f;
    const float beta = step_size(p, E::up(now.beta));
    if (kPacked) now = next;
    float qq = 0.f, kk = 0.f, kq = 0.f;
#pragma unroll
    for (int i = 0; i < kVec; ++i) qq += q[i] * q[i], kk += k[i] * k[i], kq += k[i] * q[i];
#pragma unroll
    for (int m = kLanes / 2; m; m >>= 1) {
      qq += __shfl_xor_sync(~0u, qq, m);
      kk += __shfl_xor_sync(~0u, kk, m);
      kq += __shfl_xor_sync(~0u, kq, m);
    }
    const float q_by = p.normalize ? p.scale * rsqrtf(qq + p.eps) : p.scale, k_by = p.normalize ? rsqrtf(kk + p.eps) : 1.f;
    kq *= q_by * k_by;
#pragma unroll
    for (int i = 0; i < kVec; ++i) q[i] *= q_by, k[i] *= k_by;
    float sk[kRows], sq[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      sk[r] = sq[r] = 0.f;
#pragma unroll
      for (int i = 0; i < kVec; ++i) sk[r] += state[r][i] * k[i], sq[r] += state[r][i] * q[i];
    }
    int mine;
    const float held = meet<kRows, kLanes>(sk, lane, &mine), read = meet<kRows, kLanes>(sq, lane, &mine);
    float xs = x[0];
#pragma unroll
    for (int r = 1; r < kRows; ++r) xs = mine == r ? x[r] : xs;
    const float d = beta * (xs - decay * held);
    if (in_row % (kLanes / kRows) == 0 && row0 + mine * kSub < p.head_dim)
      out[t * p.out_token + row0 + mine * kSub] = E::down(decay * read + d * kq);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const float dr = __shfl_sync(~0u, d, sub * kLanes + r * (kLanes / kRows));  // the lanes that have row r
#pragma unroll
      for (int i = 0; i < kVec; ++i) state[r][i] = state[r][i] * decay + dr * k[i];
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int i = 0; i < kVec; i += 4)
      if (row0 + r * kSub < p.head_dim)
        __stcs(reinterpret_cast<float4*>(keep) + (at + r * kSub * N + i) / 4,
               make_float4(state[r][i], state[r][i + 1], state[r][i + 2], state[r][i + 3]));
}

}  // namespace
}  // namespace kvx

// delta_chunks.cu -- the gated delta rule of prompts, by chunks of 64 tokens.
//
// With c_t the sum of the decays' exponents up to t within a chunk, S the state before it and b, k, q, v a token's,
//   w_t = b_t (v_t - e^{c_t} S k_t - sum_{s<t} e^{c_t - c_s} (k_t . k_s) w_s)
// is what token t writes, so that W = T rhs with T = (I + A)^-1, A_ts = b_t (k_t . k_s) e^{c_t - c_s} below the diagonal and
// rhs_t = b_t (v_t - e^{c_t} S k_t).  Then
//   y_t = e^{c_t} S q_t + sum_{s<=t} (q_t . k_s) e^{c_t - c_s} w_s,   S' = e^{c_63} S + sum_s e^{c_63 - c_s} w_s k_s^T.
// T, the decayed products M of queries and keys, and what else knows nothing of the state are made first, a CTA a chunk and
// head (system_kernel).  Then a CTA walks through the chunks of one sequence with 16 rows of one head's state, an element of
// v each, that know nothing of the other rows (walk_kernel): five products with 16 rows on one side.
//
// Rounding: keys and queries are fp16 numbers times a power of two a row, whose length is below 2^14 and above 2^12, so that a
// bf16 number keeps its bits down to 2^-27 of that and is off by 2^-37 of it below.  The state, rhs and W's decayed copy are each
// two fp16 numbers, 22 bits, times a power of two a row and 16 columns, and so are 2^9 T, M and the W that M is multiplied with.
// (Those two rounded to fp16 once put fp16 outputs off by 3.3e-4 where their own rounding gives 2.1e-4, and bf16 ones by 1.68e-3 instead
// of 1.66e-3, for 3 % less time.)  Sums are fp32.
//
// What bounds it is the walk: chunks of a sequence follow on one another, and each is three products on end (S k, T rhs, the state's
// update) with sums, scales and a barrier between, 3,200 to 3,900 cycles, with no unit near busy.  24k tokens in
// six sequences, 16 heads of 128 x 128, fp16: 728 us (under the profiler the systems are 150 and the walk 589, 282 chunks on end); 2,048 tokens in
// one, bf16: 75 us (18 and 60).  16 rows of the state a CTA, as a matrix instruction has 16, make 128 CTAs of a sequence of 16 heads of
// 128.  (Token by token it is 0.6 us a token.)
//
// A chunk with a number that is not finite, a decay above 1 or a T above 64 (keys with b |k|^2 well above 2) goes token
// by token within the walk.
#include <algorithm>
#include <type_traits>

#include "delta_common.cuh"
#include "tcgen05.cuh"

namespace kvx {
namespace {

constexpr int kChunk = kDeltaChunk, kThreads = 128;
constexpr float kMost = 1024.f;   // of a token's exponent
constexpr float kLargest = 64.f;  // of T
constexpr float kUp = 512.f;      // that T is multiplied by, as what a decay leaves of it is small, and rhs divided by

// What the system kernel leaves of a chunk and head (offsets in bytes): a token's factors, then T and M, each in
// two parts, as 16 x 16 blocks on and below the diagonal, row by row.
constexpr int kTriangle = 10 * 512;
struct Factors {
  float4 by[kChunk];    // of S k_t in rhs, of v_t less that, of w_t in the state, of S q_t in y
  float row[kChunk];    // M's row
  float decay;          // of the whole chunk
  int odd;              // it goes token by token
  float into[4];        // powers of two that are taken out of the third factors, 16 tokens each
  float pad[26];
};
constexpr int kFactors = (int)sizeof(Factors), kHeadBytes = kFactors + 4 * kTriangle;
static_assert(kFactors == 1408 && kHeadBytes == kDeltaHeadBytes && kHeadBytes % 128 == 0, "bulk copies");
// And of a chunk and group: keys and queries as panels of 64 elements, rows of 128 bytes with their vectors permuted.
template <int N>
constexpr int kRowBytes = kChunk * N * 2;

__device__ __forceinline__ int image_at(int row, int vec) { return (vec >> 3) * (kChunk * 128) + row * 128 + (((vec & 7) ^ (row & 7)) << 4); }
// A 16-byte half of a row of a 16 x 16 block; rows four apart would meet in the banks otherwise.
__device__ __forceinline__ int block_at(int i, int j, int row, int half) {
  return (i * (i + 1) / 2 + j) * 512 + row * 32 + ((half ^ (row >> 2 & 1)) << 4);
}
__device__ __forceinline__ int exponent_of(float v) { return min(max((int)(__float_as_uint(v) >> 23 & 255) - 127, -126), 126); }
__device__ __forceinline__ uint32_t half2_of(float a, float b) { return pack2<Fp16>(a, b); }

// ---------------------------------------------------------------- what knows nothing of the state

constexpr int kTokenRows = 8;
template <int N>
__host__ __device__ constexpr int32_t token_ctas(int32_t head_dim) { return (head_dim + 4 * kTokenRows * kTokenSub<N> - 1) / (4 * kTokenRows * kTokenSub<N>); }

constexpr int kDiagonalPitch = 20;
template <int N>
struct SystemShape {
  // keys and queries; when they have been multiplied, in their place: A below the diagonal blocks, T and M, each in two
  // parts, and A's diagonal blocks transposed in 32 bits
  static constexpr int kA = 0, kT = 2 * kTriangle, kM = 4 * kTriangle, kDiagonal = 6 * kTriangle, kThen = kDiagonal + 4 * 16 * kDiagonalPitch * 4;
  static constexpr int kSmem = 2 * kRowBytes<N> > kThen ? 2 * kRowBytes<N> : kThen;
};
__device__ __forceinline__ void split2(float2 x, uint32_t& hi, uint32_t& lo) {
  hi = half2_of(x.x, x.y);
  const float2 rest = fma2(unpack2<Fp16>(hi), make_float2(-1.f, -1.f), x);
  lo = half2_of(rest.x, rest.y);
}

// A chunk and head a CTA, 16 of its tokens a warp; before them the CTAs of the sequences that go token by token, which
// nothing here waits for (a launch of their own took 6 us more).  T is made block by block: on the diagonal by substitution, below it as
// T_ij = -T_ii sum_{j<=k<i} A_ik T_kj, a column of blocks a warp, by products of numbers in two parts (24k tokens of 16 heads 150 us under
// the profiler, and 30 % more with columns by substitution in 32-bit floats, whose longest is the first warp's).  Bound by instructions,
// 3,400 a warp, and by what it reads and writes, which is 81 us of those 150 at the DRAM's rate.
template <class E, int N>
__global__ void __launch_bounds__(kThreads, 5) system_kernel(const __grid_constant__ DeltaParams p) {
  wait_for_previous();
  using S = SystemShape<N>;
  using T = typename E::T;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Factors f;
  __shared__ float key_s[kChunk], query_s[kChunk], by_s[2][kChunk];
  __shared__ float4 token_s[kChunk];  // the exponents' sum up to a token, what it lost, the key's factor, the step
  __shared__ int32_t buf[kThreads / 32 + 3];
  const StateView& v = p.state;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  const int32_t h = blockIdx.y, group = h / p.heads_per_group;
  if ((int32_t)blockIdx.x < p.token_ctas) {
    const int32_t each = token_ctas<N>(p.head_dim), s = blockIdx.x / each;
    by_tokens<E, N, kTokenRows, true>(p, blockIdx.x - s * each, h, s);
    return;
  }
  const int32_t piece = blockIdx.x - p.token_ctas;
  Piece found;
  if (!find_piece<kThreads>(v, piece, kChunk, p.by_token, buf, &found) || !found.in || !found.keep) return;
  const int64_t t0 = found.first + (int64_t)found.at * kChunk;
  const int32_t n = (int32_t)min((int64_t)kChunk, found.last - t0);
  uint8_t* rows_to = p.rows_space + ((int64_t)piece * p.groups + group) * 2 * kRowBytes<N>;
  uint8_t* head_to = p.head_space + ((int64_t)piece * p.heads + h) * kHeadBytes;
  const bool writes_rows = h == group * p.heads_per_group;
  bool odd = false;

  // Keys and queries: lengths, and fp16 numbers that leave the row's below 2^14.
  constexpr int kLanes = N / 8, kAtOnce = 32 / kLanes, kRounds = 16 / kAtOnce;
  const int vec = lane % kLanes, sub = lane / kLanes;
  const T* rows[2] = {reinterpret_cast<const T*>(p.k) + group * p.k_head + vec * 8, reinterpret_cast<const T*>(p.q) + group * p.q_head + vec * 8};
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const int64_t stride = which ? p.q_token : p.k_token;
    uint4 raw[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int row = warp * 16 + i * kAtOnce + sub;
      raw[i] = row < n ? *reinterpret_cast<const uint4*>(rows[which] + (t0 + row) * stride) : make_uint4(0, 0, 0, 0);
    }
    // sums of squares of the rounds' rows meet in a reduction that halves the rounds at every step
    float squares[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x = unpack2<E>(u[j]);
        sum = fma2(x, x, sum);
      }
      squares[i] = sum.x + sum.y;
    }
    int m = kLanes / 2, at = 0;
#pragma unroll
    for (int left = kRounds; left > 1; left /= 2, m /= 2) {
      const bool upper = lane & m;
      at = 2 * at + upper;
#pragma unroll
      for (int k = 0; k < left / 2; ++k) {
        const float send = upper ? squares[k] : squares[k + left / 2], stay = upper ? squares[k + left / 2] : squares[k];
        squares[k] = stay + __shfl_xor_sync(~0u, send, m);
      }
    }
#pragma unroll
    for (; m; m >>= 1) squares[0] += __shfl_xor_sync(~0u, squares[0], m);
    {  // what takes the row's length below 2^14, and a token's factor; a row whose squares vanish counts as zeros
      const int row = warp * 16 + at * kAtOnce + sub;
      const float all = squares[0];
      const int e = all > 0.f ? (((int)(__float_as_uint(all) >> 23) - 127) >> 1) - 13 : 0;  // its root is below 2^(e + 14)
      const float factor = row < n ? (p.normalize ? rsqrtf(all + p.eps) : 1.f) * (which ? p.scale : 1.f) * power_of_two(e) : 0.f;
      odd |= !isfinite(factor) || !isfinite(all);
      by_s[which][row] = power_of_two(-e);
      (which ? query_s : key_s)[row] = all > 0.f ? factor : 0.f;  // of zeros it would only set scales
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int row = warp * 16 + i * kAtOnce + sub;
      const float by = by_s[which][row];
      const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x = mul2(unpack2<E>(u[j]), make_float2(by, by));
        w[j] = half2_of(x.x, x.y);
      }
      const int to = which * kRowBytes<N> + image_at(row, vec);
      *reinterpret_cast<uint4*>(smem + to) = make_uint4(w[0], w[1], w[2], w[3]);
      if (writes_rows) *reinterpret_cast<uint4*>(rows_to + to) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  // Gates, two tokens a lane: sums of exponents up to a token in two parts, whole 64ths (that 64 tokens of up to 2^10 lose no
  // bit of) and the rest, as differences of them count; sums behind a token from the end.
  if (warp == 0) {
    float a[2], rest[2], beta[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int t = 2 * lane + k;
      const bool there = t < n;
      beta[k] = there ? step_size(p, E::up(reinterpret_cast<const T*>(p.beta)[(t0 + t) * p.beta_token + h])) : 0.f;
      a[k] = there && p.dt ? decay_of(p, E::up(reinterpret_cast<const T*>(p.dt)[(t0 + t) * p.dt_token + h]), h) * kLog2e : 0.f;
      odd |= !isfinite(beta[k]) || !(a[k] <= 0.f);
      a[k] = fmaxf(a[k], -kMost);
      rest[k] = a[k] - rintf(a[k] * 64.f) * (1.f / 64);
    }
    float upto = (a[0] - rest[0]) + (a[1] - rest[1]), fine = rest[0] + rest[1], behind = a[0] + a[1];
    for (int m = 1; m < 32; m <<= 1) {
      const float y = __shfl_up_sync(~0u, upto, m), z = __shfl_up_sync(~0u, fine, m), w = __shfl_down_sync(~0u, behind, m);
      if (lane >= m) upto += y, fine += z;
      if (lane + m < 32) behind += w;
    }
    float below = __shfl_up_sync(~0u, upto, 1), below_fine = __shfl_up_sync(~0u, fine, 1), above = __shfl_down_sync(~0u, behind, 1);
    if (lane == 0) below = below_fine = 0.f;
    if (lane == 31) above = 0.f, f.decay = ex2(upto + fine);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      below += a[k] - rest[k], below_fine += rest[k];
      // the sum of both, rounded, and what that lost (Knuth, "The Art of Computer Programming", vol. 2, 4.2.2)
      const float sum = below + below_fine, back = sum - below, low = (below - (sum - back)) + (below_fine - back);
      const int t = 2 * lane + k;
      token_s[t] = make_float4(sum, low, 0.f, beta[k]);
      const float decay = ex2(sum) * ex2(low);
      f.by[t] = make_float4(decay, beta[k] * (1 / kUp), 0.f, decay);
    }
#pragma unroll
    for (int k = 1; k >= 0; --k) {
      f.by[2 * lane + k].z = 2 * lane + k < n ? ex2(above) : 0.f;
      above += a[k];
    }
  }
  __syncthreads();
  if (threadIdx.x < kChunk) {
    float4& by = f.by[threadIdx.x];
    token_s[threadIdx.x].z = key_s[threadIdx.x];
    by.x *= key_s[threadIdx.x], by.z *= key_s[threadIdx.x], by.w *= query_s[threadIdx.x];
    float most = fabsf(by.z);
#pragma unroll
    for (int m = 8; m; m >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, m));
    const int into = min(exponent_of(most) + 1, 126);
    by.z *= power_of_two(-into);
    if (threadIdx.x % 16 == 0) f.into[threadIdx.x / 16] = power_of_two(into);
  }

  // Products of keys with keys and of queries with keys, 16 rows a warp, up to the diagonal.
  const uint32_t base = smem_at(smem);
  float kk[8][4], qk[8][4];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) kk[j][e] = qk[j][e] = 0.f;
  const int a_row = (lane >> 3 & 1) * 8 + (lane & 7), a_vec = lane >> 4;  // of a left factor's matrices, and a right one's transposed
  const int b_row = (lane >> 4) * 8 + (lane & 7), b_vec = lane >> 3 & 1;  // of a right one's
#pragma unroll 2
  for (int s = 0; s < N / 16; ++s) {
    uint32_t ka[4], qa[4];
    load_matrices(ka, base + image_at(warp * 16 + a_row, 2 * s + a_vec));
    load_matrices(qa, base + kRowBytes<N> + image_at(warp * 16 + a_row, 2 * s + a_vec));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j > warp) break;
      uint32_t b[4];
      load_matrices(b, base + image_at(16 * j + b_row, 2 * s + b_vec));
      mma<Fp16>(kk[2 * j], ka, b[0], b[1]);
      mma<Fp16>(kk[2 * j + 1], ka, b[2], b[3]);
      mma<Fp16>(qk[2 * j], qa, b[0], b[1]);
      mma<Fp16>(qk[2 * j + 1], qa, b[2], b[3]);
    }
  }
  __syncthreads();  // the images have been read
  float* diagonal = reinterpret_cast<float*>(smem + S::kDiagonal) + warp * 16 * kDiagonalPitch;  // [s][t]
  float top[2] = {0.f, 0.f};
  const float4 row[2] = {token_s[warp * 16 + g], token_s[warp * 16 + g + 8]};  // of the warp's
  const float query[2] = {query_s[warp * 16 + g], query_s[warp * 16 + g + 8]};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (j > 2 * warp + 1) break;
    const int s = 8 * j + 2 * c;
    const float4 col[2] = {token_s[s], token_s[s + 1]};
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int t = warp * 16 + g + 8 * r;
      float a[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float decay = ex2((row[r].x - col[e].x) + (row[r].y - col[e].y));
        const float by = j < 2 * warp || s + e <= t ? col[e].z * decay : 0.f;
        a[e] = kk[j][2 * r + e] * (by * (row[r].z * row[r].w));
        qk[j][2 * r + e] *= by * query[r];
        top[r] = fmaxf(top[r], fabsf(qk[j][2 * r + e]));
      }
      if (j < 2 * warp) {  // with its sign turned
        uint32_t hi, lo;
        split2(make_float2(a[0] * -kUp, a[1] * -kUp), hi, lo);
        uint8_t* to = smem + S::kA + block_at(warp, j >> 1, g + 8 * r, j & 1) + 4 * c;
        *reinterpret_cast<uint32_t*>(to) = hi;
        *reinterpret_cast<uint32_t*>(to + kTriangle) = lo;
      } else {
        diagonal[(s & 15) * kDiagonalPitch + (t & 15)] = a[0];  // of which what is below the diagonal is read
        diagonal[(s + 1 & 15) * kDiagonalPitch + (t & 15)] = a[1];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 1));
    top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 2));
    odd |= !(top[r] < INFINITY);
    const int e = top[r] > 0.f ? min(13 - exponent_of(top[r]), 126) : 0;  // the row's largest to [2^13, 2^14)
    const float up = power_of_two(e);
    if (c == 0) f.row[warp * 16 + g + 8 * r] = power_of_two(-e);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j > 2 * warp + 1) break;
      uint32_t hi, lo;
      split2(mul2(make_float2(qk[j][2 * r], qk[j][2 * r + 1]), make_float2(up, up)), hi, lo);
      uint8_t* to = smem + S::kM + block_at(warp, j >> 1, g + 8 * r, j & 1) + 4 * c;
      *reinterpret_cast<uint32_t*>(to) = hi;
      *reinterpret_cast<uint32_t*>(to + kTriangle) = lo;
    }
  }
  __syncwarp();
  // A block on the diagonal inverted by substitution, a column a lane (both halves of the warp alike).
  {
    const int col = lane & 15;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i == col ? 1.f : 0.f;
#pragma unroll
    for (int k = 0; k < 15; ++k)
#pragma unroll
      for (int i = (k + 1) / 4 * 4; i < 16; i += 4) {
        const float4 a = *reinterpret_cast<const float4*>(diagonal + k * kDiagonalPitch + i);
        if (i > k) x[i] -= a.x * x[k];
        if (i + 1 > k) x[i + 1] -= a.y * x[k];
        if (i + 2 > k) x[i + 2] -= a.z * x[k];
        if (i + 3 > k) x[i + 3] -= a.w * x[k];
      }
    // T's block, a half of its rows a half of the warp
    uint8_t* to = smem + S::kT;
    const bool upper = lane >= 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = (upper ? x[i + 8] : x[i]) * kUp;
      odd |= !(fabsf(y) <= kLargest * kUp);
      const __half hi = __float2half_rn(y), lo = __float2half_rn(y - __half2float(hi));
      const int at = block_at(warp, warp, i + (upper ? 8 : 0), col >> 3) + (col & 7) * 2;
      *reinterpret_cast<__half*>(to + at) = hi;
      *reinterpret_cast<__half*>(to + kTriangle + at) = lo;
    }
  }
  __syncthreads();
  for (int i = warp + 1; i < 4; ++i) {
    float x[2][4] = {};  // 2^18 times the sum, rows g and g + 8, columns 2 c and the next of each eight
    for (int k = warp; k < i; ++k) {
      uint32_t a[4], a_lo[4], b[4], b_lo[4];
      load_matrices(a, base + S::kA + block_at(i, k, a_row, a_vec));
      load_matrices(a_lo, base + S::kA + kTriangle + block_at(i, k, a_row, a_vec));
      load_matrices_t(b, base + S::kT + block_at(k, warp, a_row, a_vec));
      load_matrices_t(b_lo, base + S::kT + kTriangle + block_at(k, warp, a_row, a_vec));
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        mma<Fp16>(x[u], a, b[2 * u], b[2 * u + 1]);
        mma<Fp16>(x[u], a_lo, b[2 * u], b[2 * u + 1]);
        mma<Fp16>(x[u], a, b_lo[2 * u], b_lo[2 * u + 1]);
      }
    }
    // as a right factor: its columns lie along k
    uint32_t hi[2][2], lo[2][2], a[4], a_lo[4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        split2(mul2(make_float2(x[u][2 * r], x[u][2 * r + 1]), make_float2(1 / kUp, 1 / kUp)), hi[u][r], lo[u][r]);
        hi[u][r] = transpose(hi[u][r]), lo[u][r] = transpose(lo[u][r]);
      }
    load_matrices(a, base + S::kT + block_at(i, i, a_row, a_vec));
    load_matrices(a_lo, base + S::kT + kTriangle + block_at(i, i, a_row, a_vec));
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float y[4] = {};
      mma<Fp16>(y, a, hi[u][0], hi[u][1]);
      mma<Fp16>(y, a_lo, hi[u][0], hi[u][1]);
      mma<Fp16>(y, a, lo[u][0], lo[u][1]);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float2 t = mul2(make_float2(y[2 * r], y[2 * r + 1]), make_float2(1 / kUp, 1 / kUp));
        odd |= !(fabsf(t.x) <= kLargest * kUp) || !(fabsf(t.y) <= kLargest * kUp);
        uint32_t t_hi, t_lo;
        split2(t, t_hi, t_lo);
        uint8_t* to = smem + S::kT + block_at(i, warp, g + 8 * r, u) + 4 * c;
        *reinterpret_cast<uint32_t*>(to) = t_hi;
        *reinterpret_cast<uint32_t*>(to + kTriangle) = t_lo;
      }
    }
    __syncwarp();
  }
  odd = __syncthreads_or(odd);
  if (threadIdx.x == 0) f.odd = odd;
  for (int i = threadIdx.x; i < 4 * kTriangle / 16; i += kThreads)
    reinterpret_cast<uint4*>(head_to + kFactors)[i] = reinterpret_cast<const uint4*>(smem + S::kT)[i];
  __syncthreads();
  for (int i = threadIdx.x; i < kFactors / 16; i += kThreads)
    reinterpret_cast<uint4*>(head_to)[i] = reinterpret_cast<const uint4*>(&f)[i];
}

// ---------------------------------------------------------------- the walk

__device__ __forceinline__ void bulk_load(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes),
               "r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

constexpr int kWalkThreads = 288;  // four warps for the state, four for the outputs, one for the copies

template <int N>
struct WalkShape {
  static constexpr int kSteps = N / 16;  // of 16 along the state's columns
  static constexpr int kT = 2 * kRowBytes<N> + kFactors, kStage = 2 * kRowBytes<N> + kFactors + 2 * kTriangle;
  // left factors as the matrix instruction takes them, 512 bytes for 16 columns and part, and their powers of two
  static constexpr int kM = 2 * kStage, kState = kM + 2 * kTriangle, kRhs = kState + kSteps * 1024, kWrite = kRhs + 4096, kPlain = kWrite + 4096,
                       kStateBy = kPlain + 4096, kRhsBy = kStateBy + kSteps * 64, kPlainBy = kRhsBy + 256, kSmem = kPlainBy + 256;
  static_assert(kSmem <= 231424, "shared memory of an SM");
};

// Two tiles of 16 x 8 sums as 16 columns of a left factor: fp16 parts hi and lo, times powers of two a row, the largest number
// to [2^13, 2^14).
struct Scaled {
  float up[2];
  float2 down;
};
__device__ __forceinline__ Scaled scaled_for(const float (&x)[4], const float (&y)[4]) {
  float top[2] = {fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(y[0]), fabsf(y[1]))),
                  fmaxf(fmaxf(fabsf(x[2]), fabsf(x[3])), fmaxf(fabsf(y[2]), fabsf(y[3])))};
#pragma unroll
  for (int m = 1; m < 4; m <<= 1)
#pragma unroll
    for (int r = 0; r < 2; ++r) top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], m));
  Scaled s;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int e = min(140 - (int)(__float_as_uint(top[r]) >> 23), 126);
    s.up[r] = power_of_two(e);
    (r ? s.down.y : s.down.x) = power_of_two(-e);
  }
  return s;
}
__device__ __forceinline__ void left_factor(const float2 (&v)[4], uint8_t* hi, uint8_t* lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    h[k] = half2_of(v[k].x, v[k].y);
    const float2 rest = fma2(unpack2<Fp16>(h[k]), make_float2(-1.f, -1.f), v[k]);
    l[k] = half2_of(rest.x, rest.y);
  }
  *reinterpret_cast<uint4*>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void times(float2 (&v)[4], const float (&x)[4], const float (&y)[4], const float (&up)[2]) {
  v[0] = mul2(make_float2(x[0], x[1]), make_float2(up[0], up[0])), v[1] = mul2(make_float2(x[2], x[3]), make_float2(up[1], up[1]));
  v[2] = mul2(make_float2(y[0], y[1]), make_float2(up[0], up[0])), v[3] = mul2(make_float2(y[2], y[3]), make_float2(up[1], up[1]));
}
__device__ __forceinline__ void left_load(uint32_t (&a)[4], const uint8_t* at) {
  const uint4 v = *reinterpret_cast<const uint4*>(at);
  a[0] = v.x, a[1] = v.y, a[2] = v.z, a[3] = v.w;
}
__device__ __forceinline__ void add_scaled(float (&d)[4], const float (&x)[4], float2 by) {
  const float2 a = fma2(make_float2(x[0], x[1]), make_float2(by.x, by.x), make_float2(d[0], d[1]));
  const float2 b = fma2(make_float2(x[2], x[3]), make_float2(by.y, by.y), make_float2(d[2], d[3]));
  d[0] = a.x, d[1] = a.y, d[2] = b.x, d[3] = b.y;
}
// Barriers: of all at a chunk's beginning, of the first four where rhs is there, of the eight where w is, and otherwise.
enum { kBegin = 1, kRhsThere, kWThere, kEight };
template <int kCount>
__device__ __forceinline__ void meet(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kCount) : "memory"); }

// A CTA walks with 16 rows of one head's state: four warps have the state in registers, a quarter of its columns each, and make rhs
// and W, 16 tokens each; four make the outputs beside the next chunk's first product; one copies chunks, a chunk ahead.  (With
// four warps for all of it, and what does not wait loaded behind the barriers, a chunk took 3,900 cycles instead of 3,200; a thread
// of the chain that issues the copies costs 300 of these.  Not taken, and measured against 70 us for 2,048 tokens, before bf16 outputs' products had two parts:
// eight warps for the state with 8 tokens each, 146, as all read the state's fragments and shared memory is the bound; the products on
// tcgen05, 97, as one takes 680 cycles from
// its issue to the warps that wait for it, three times a chunk, where mma.sync's steps take 20.)
template <class E, int N>
__global__ void __launch_bounds__(kWalkThreads, 1) walk_kernel(const __grid_constant__ DeltaParams p) {
  wait_for_previous();
  using W = WalkShape<N>;
  using T = typename E::T;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars_s[3];  // of both stages and of M
  __shared__ uint32_t flags_s[2];  // a chunk's: it goes token by token; a wait has run out
  const StateView& v = p.state;
  const int lane = threadIdx.x & 31, all_warps = __shfl_sync(~0u, threadIdx.x >> 5, 0), warp = all_warps & 3, g = lane >> 2, c = lane & 3;
  const int32_t p0 = blockIdx.x * 16, h = blockIdx.y, group = h / p.heads_per_group;
  // Of the sequences that go by chunks the longest first, as they are walked through longest (of more than a warp can look
  // at, in their order).
  int32_t s = -1, first = 0;  // its number, and that of its first chunk
  int64_t begin = 0, end = 0;
  if (v.num_seqs <= 32) {
    if (lane < v.num_seqs) rows_of(v, lane, &begin, &end);
    const int32_t mine = lane < v.num_seqs ? (int32_t)(end - begin) : -1;
    int32_t rank = 0;
    for (int32_t k = 0; k < v.num_seqs; ++k) {
      const int32_t other = __shfl_sync(~0u, mine, k);
      rank += other > mine || (other == mine && k < lane);
    }
    s = __ffs(__ballot_sync(~0u, lane < v.num_seqs && rank == (int32_t)blockIdx.z)) - 1;
    if (s < 0) return;
    first = __reduce_add_sync(~0u, lane < s ? min(pieces_of(begin, end, kChunk, p.by_token), (1 << 30) / 32) : 0);
    begin = __shfl_sync(~0u, begin, s), end = __shfl_sync(~0u, end, s);
  } else {  // every warp for itself
    int32_t before = 0;
    for (int32_t base = 0; base < v.num_seqs && s < 0; base += 32) {
      int64_t a = 0, b = 0;
      if (base + lane < v.num_seqs) rows_of(v, base + lane, &a, &b);
      const int32_t pieces = base + lane < v.num_seqs ? min(pieces_of(a, b, kChunk, p.by_token), (1 << 30) / 32) : 0;
      const uint32_t some = __ballot_sync(~0u, pieces > 0);
      const int at = before + __popc(some) > (int32_t)blockIdx.z ? __fns(some, 0, (int32_t)blockIdx.z - before + 1) : 32;
      first = min(first + (int32_t)__reduce_add_sync(~0u, lane < at ? pieces : 0), p.pieces);
      if (at < 32) s = base + at, begin = __shfl_sync(~0u, a, at), end = __shfl_sync(~0u, b, at);
      before += __popc(some);
    }
    if (s < 0) return;
  }
  first = min(first, p.pieces);
  const int32_t chunks = min(pieces_of(begin, end, kChunk, p.by_token), p.pieces - first);
  if (pieces_of(begin, end, kChunk, p.by_token) == 0) return;
  const uint32_t base = smem_at(smem), bars = smem_at(bars_s);
  if (threadIdx.x == 0) {
    flags_s[0] = flags_s[1] = 0;
    for (int i = 0; i < 3; ++i) bar_init(bars + 8 * i);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");  // what the kernel before has written is read by bulk copies
  }
  __syncthreads();
  const uint8_t* in = slot_of(v, v.slots_in, s);
  uint8_t* keep = slot_of(v, v.slots_out, s);
  T* out = reinterpret_cast<T*>(p.out) + h * p.out_head + p0;
  if (!in || !keep) {
    for (int64_t i = threadIdx.x; i < (end - begin) * 16; i += kWalkThreads)
      if (p0 + i % 16 < p.head_dim) out[(begin + i / 16) * p.out_token + i % 16] = E::down(0.f);
    return;
  }

  auto load_stage = [&](int32_t i) {  // by one thread
    const uint32_t bar = bars + 8 * (i & 1), to = base + (i & 1) * W::kStage;
    if (i >= chunks || (p.stall == 1 && i == 1)) return;
    bar_expect(bar, W::kStage);
    bulk_load(to, p.rows_space + ((int64_t)(first + i) * p.groups + group) * 2 * kRowBytes<N>, 2 * kRowBytes<N>, bar);
    bulk_load(to + 2 * kRowBytes<N>, p.head_space + ((int64_t)(first + i) * p.heads + h) * kHeadBytes, kFactors + 2 * kTriangle, bar);
  };
  auto load_m = [&](int32_t i) {
    constexpr int kBytes = 2 * kTriangle;
    if (p.stall == 2 && i == 0) return;
    bar_expect(bars + 16, kBytes);
    bulk_load(base + W::kM, p.head_space + ((int64_t)(first + i) * p.heads + h) * kHeadBytes + kFactors + 2 * kTriangle, kBytes, bars + 16);
  };
  auto factors_of = [&](int32_t i) -> const Factors& { return *reinterpret_cast<const Factors*>(smem + (i & 1) * W::kStage + 2 * kRowBytes<N>); };
  constexpr uint32_t kOdd = 1, kDead = 2;
  bool dead = false;
  // M's wait, by the warps of the outputs: where it runs out all warps end before the next chunk, as no copy may follow one that is
  // on its way.  (Told by the flag alone: a variable that lives through the loop takes 3 % more time.)
  auto wait_for_m = [&](int32_t i) {
    if (!bar_wait(bars + 16, i & 1, p.wait_cycles)) atomicOr(&flags_s[(i + 1) & 1], kDead);
  };
  float2* state_by = reinterpret_cast<float2*>(smem + W::kStateBy);
  float2* rhs_by = reinterpret_cast<float2*>(smem + W::kRhsBy);
  float2* plain_by = reinterpret_cast<float2*>(smem + W::kPlainBy);
  const int b_row = (lane >> 4) * 8 + (lane & 7), b_vec = lane >> 3 & 1;  // of a right factor's matrices
  int32_t i = 0;

  // S times the keys or queries at `image` of the warp's 16 tokens.  Here and below what products take is loaded for many of
  // them before the first, and every step has sums of its own, so that none waits for another.
  auto read_state = [&](float (&d)[2][4], uint32_t image) {
    constexpr int kAtOnce = 4;
#pragma unroll
    for (int k0 = 0; k0 < W::kSteps; k0 += kAtOnce) {
      uint32_t hi[kAtOnce][4], lo[kAtOnce][4], b[kAtOnce][4];
      float2 by[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        left_load(hi[k], smem + W::kState + (k0 + k) * 1024 + lane * 16);
        left_load(lo[k], smem + W::kState + (k0 + k) * 1024 + 512 + lane * 16);
        load_matrices(b[k], image + image_at(warp * 16 + b_row, 2 * (k0 + k) + b_vec));
        by[k] = state_by[(k0 + k) * 8 + g];
      }
      float x[kAtOnce][2][4] = {};
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
          for (int u = 0; u < 2; ++u) mma<Fp16>(x[k][u], part ? lo[k] : hi[k], b[k][2 * u], b[k][2 * u + 1]);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
        for (int u = 0; u < 2; ++u) add_scaled(d[u], x[k][u], by[k]);
    }
  };
  // A chunk that goes token by token, a row of the state for sixteen lanes; the state in `all`, between two barriers.
  float* all = reinterpret_cast<float*>(smem + W::kState);
  static_assert(W::kSteps * 1024 == 16 * N * 4, "the state's room");
  auto by_tokens = [&](int64_t t0) {
    constexpr int kCols = N / 16;
    const int row = threadIdx.x / 16, part = threadIdx.x % 16;
    const bool used = p0 + row < p.head_dim;
    float x[kCols];
#pragma unroll
    for (int k = 0; k < kCols; ++k) x[k] = all[row * N + k * 16 + part];
    const int64_t stop = min(end, t0 + kChunk);
    for (int64_t t = t0; t < stop; ++t) {
      const T* k_at = reinterpret_cast<const T*>(p.k) + t * p.k_token + group * p.k_head + part;
      const T* q_at = reinterpret_cast<const T*>(p.q) + t * p.q_token + group * p.q_head + part;
      float kk = 0.f, qq = 0.f, kq = 0.f, sk = 0.f, sq = 0.f;
#pragma unroll
      for (int k = 0; k < kCols; ++k) {
        const float a = E::up(k_at[16 * k]), b = E::up(q_at[16 * k]);
        kk += a * a, qq += b * b, kq += a * b, sk += x[k] * a, sq += x[k] * b;
      }
#pragma unroll
      for (int m = 8; m; m >>= 1) {
        kk += __shfl_xor_sync(~0u, kk, m), qq += __shfl_xor_sync(~0u, qq, m), kq += __shfl_xor_sync(~0u, kq, m);
        sk += __shfl_xor_sync(~0u, sk, m), sq += __shfl_xor_sync(~0u, sq, m);
      }
      const float k_by = p.normalize ? rsqrtf(kk + p.eps) : 1.f, q_by = p.normalize ? p.scale * rsqrtf(qq + p.eps) : p.scale;
      const float decay = p.dt ? expf(decay_of(p, E::up(reinterpret_cast<const T*>(p.dt)[t * p.dt_token + h]), h)) : 1.f;
      const float beta = step_size(p, E::up(reinterpret_cast<const T*>(p.beta)[t * p.beta_token + h]));
      const float value = used ? E::up(reinterpret_cast<const T*>(p.v)[t * p.v_token + h * p.v_head + p0 + row]) : 0.f;
      const float d = beta * (value - decay * (sk * k_by));
      if (used && part == 0) out[t * p.out_token + row] = E::down(decay * (sq * q_by) + d * (kq * k_by * q_by));
#pragma unroll
      for (int k = 0; k < kCols; ++k) x[k] = x[k] * decay + d * (E::up(k_at[16 * k]) * k_by);
    }
#pragma unroll
    for (int k = 0; k < kCols; ++k) all[row * N + k * 16 + part] = x[k];
  };

  if (all_warps == 8) {
    // The copies: a chunk's before it begins, and whether it goes token by token.
    if (lane == 0) load_stage(0);
    for (; i < chunks; ++i) {
      dead = dead || !bar_wait(bars + 8 * (i & 1), i >> 1 & 1, p.wait_cycles);
      if (lane == 0 && (dead || factors_of(i).odd)) atomicOr(&flags_s[i & 1], dead ? kDead : kOdd);
      meet<kWalkThreads>(kBegin);
      if (flags_s[i & 1] & kDead) break;
      if (lane == 0) load_m(i), load_stage(i + 1);
      __syncwarp();
    }
  } else if (all_warps >= 4) {
    for (; i < chunks; ++i) {
      const int64_t t0 = begin + (int64_t)i * kChunk;
      const uint32_t rows = base + (i & 1) * W::kStage;
      const Factors& f = factors_of(i);
      meet<kWalkThreads>(kBegin);  // the state and the chunk's copies are there
      const uint32_t flags = flags_s[i & 1];
      if (flags & kDead) break;
      if (flags & kOdd) {
        meet<256>(kEight);
        if (threadIdx.x == 128) flags_s[i & 1] = 0;
        by_tokens(t0);
        wait_for_m(i);
        meet<256>(kEight);
        continue;
      }
      // S q of the warp's 16 tokens
      float y[2][4] = {};
      read_state(y, rows + kRowBytes<N>);
      float by[2][2], m_by[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          by[u][e] = f.by[warp * 16 + 8 * u + 2 * c + e].w;
          m_by[u][e] = f.row[warp * 16 + 8 * u + 2 * c + e];
        }
      wait_for_m(i);
      meet<256>(kWThere);  // S has been read
      // y = e^c S q + M w
      float mw[2][4] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k > warp) break;
        uint32_t hi[4], lo[4], b[4], b_lo[4];
        left_load(hi, smem + W::kPlain + k * 1024 + lane * 16);
        load_matrices(b, base + W::kM + block_at(warp, k, b_row, b_vec));
        left_load(lo, smem + W::kPlain + k * 1024 + 512 + lane * 16);
        load_matrices(b_lo, base + W::kM + kTriangle + block_at(warp, k, b_row, b_vec));
        const float2 undo = plain_by[k * 8 + g];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float x[4] = {};
          mma<Fp16>(x, hi, b[2 * u], b[2 * u + 1]);
          mma<Fp16>(x, lo, b[2 * u], b[2 * u + 1]);
          mma<Fp16>(x, hi, b_lo[2 * u], b_lo[2 * u + 1]);
          add_scaled(mw[u], x, undo);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int64_t t = t0 + warp * 16 + 8 * u + g;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t pair = transpose(pack2<E>(by[u][0] * y[u][2 * r] + m_by[u][0] * mw[u][2 * r],
                                                   by[u][1] * y[u][2 * r + 1] + m_by[u][1] * mw[u][2 * r + 1]));
          if (t < end && p0 + 8 * r < p.head_dim) *reinterpret_cast<uint32_t*>(out + t * p.out_token + 8 * r + 2 * c) = pair;
        }
      }
    }
  }

  // The state: tiles of 16 x 8, rows g and g + 8, columns 2 c and the next.
  constexpr int kTiles = N / 32;  // a warp's
  float state[kTiles][4];
  const int64_t state_at = ((int64_t)h * p.head_dim + p0) * N + warp * kTiles * 8 + 2 * c;
  if (all_warps < 4) {
    // Values of a chunk, as a transposing move takes them: tokens 8 u + lane / 4 of the warp's, elements 2 c and the next
    // of each eight.
    const T* v_at[2];  // of the chunk that is loaded next
    int64_t left = end - begin - warp * 16 - g;
#pragma unroll
    for (int u = 0; u < 2; ++u) v_at[u] = reinterpret_cast<const T*>(p.v) + (begin + warp * 16 + 8 * u + g) * p.v_token + h * p.v_head + p0 + 2 * c;
    const int64_t v_step = kChunk * p.v_token;
    const bool has_row[2] = {true, p0 + 8 < p.head_dim};
    uint32_t raw[2][2];
    auto load_values = [&]() {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int k = 0; k < 2; ++k) raw[u][k] = left > 8 * u && has_row[k] ? *reinterpret_cast<const uint32_t*>(v_at[u] + 8 * k) : 0;
        v_at[u] += v_step;
      }
      left -= kChunk;
    };
    auto values_there = [&](int32_t i) {
      if (odd_carried(odd_carry<E>(raw[0][0]) | odd_carry<E>(raw[0][1]) | odd_carry<E>(raw[1][0]) | odd_carry<E>(raw[1][1]))) atomicOr(&flags_s[i & 1], kOdd);
    };
    load_values();
    const bool fresh = v.fresh && v.fresh[s];
#pragma unroll
    for (int k = 0; k < kTiles; ++k)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float2 x = make_float2(0.f, 0.f);
        if (!fresh && p0 + 8 * r < p.head_dim) x = *reinterpret_cast<const float2*>(in + (state_at + (g + 8 * r) * N + k * 8) * 4);
        state[k][2 * r] = x.x, state[k][2 * r + 1] = x.y;
      }
    auto publish = [&]() {
#pragma unroll
      for (int k = 0; k < kTiles; k += 2) {
        const int step = (warp * kTiles + k) / 2;
        const Scaled by = scaled_for(state[k], state[k + 1]);
        float2 x[4];
        times(x, state[k], state[k + 1], by.up);
        left_factor(x, smem + W::kState + step * 1024 + lane * 16, smem + W::kState + step * 1024 + 512 + lane * 16);
        if (c == 0) state_by[step * 8 + g] = by.down;
      }
    };
    publish();
    values_there(0);
    const int t_row = (lane >> 3 & 1) * 8 + (lane & 7), t_vec = lane >> 4;  // of a factor that is transposed
    for (; i < chunks; ++i) {
      const uint32_t rows = base + (i & 1) * W::kStage;
      const Factors& f = factors_of(i);
      meet<kWalkThreads>(kBegin);  // the state and the chunk's copies are there
      const uint32_t flags = flags_s[i & 1];
      if (flags & kDead) break;
      if (flags & kOdd) {
#pragma unroll
        for (int k = 0; k < kTiles; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) all[(g + 8 * (e >> 1)) * N + (warp * kTiles + k) * 8 + 2 * c + (e & 1)] = state[k][e];
        meet<256>(kEight);
        by_tokens(begin + (int64_t)i * kChunk);
        load_values();
        values_there(i + 1);
        meet<256>(kEight);
#pragma unroll
        for (int k = 0; k < kTiles; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) state[k][e] = all[(g + 8 * (e >> 1)) * N + (warp * kTiles + k) * 8 + 2 * c + (e & 1)];
        meet<128>(kRhsThere);
        publish();
        continue;
      }
      // S k of the warp's 16 tokens
      float sk[2][4] = {};
      read_state(sk, rows);
      float write[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float4 by[2] = {f.by[warp * 16 + 8 * u + 2 * c], f.by[warp * 16 + 8 * u + 2 * c + 1]};
        write[u][0] = by[0].z, write[u][1] = by[1].z;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float2 value = unpack2<E>(transpose(raw[u][r]));
          sk[u][2 * r] = by[0].y * (value.x - by[0].x * sk[u][2 * r]);
          sk[u][2 * r + 1] = by[1].y * (value.y - by[1].x * sk[u][2 * r + 1]);
        }
      }
      {
        const Scaled by = scaled_for(sk[0], sk[1]);
        float2 x[4];
        times(x, sk[0], sk[1], by.up);
        left_factor(x, smem + W::kRhs + warp * 1024 + lane * 16, smem + W::kRhs + warp * 1024 + 512 + lane * 16);
        if (c == 0) rhs_by[warp * 8 + g] = by.down;
      }
      load_values();
      // W = T rhs: a warp's rows of T have as many blocks as it is warps from the first
      float w[2][4] = {};
      auto solve = [&](auto blocks) {
        constexpr int kBlocks = decltype(blocks)::value;
        uint32_t hi[kBlocks][4], lo[kBlocks][4], b[kBlocks][4], b_lo[kBlocks][4];
        float2 undo[kBlocks];
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
          load_matrices(b[k], rows + W::kT + block_at(kBlocks - 1, k, b_row, b_vec));
          load_matrices(b_lo[k], rows + W::kT + kTriangle + block_at(kBlocks - 1, k, b_row, b_vec));
        }
        meet<128>(kRhsThere);
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
          left_load(hi[k], smem + W::kRhs + k * 1024 + lane * 16);
          left_load(lo[k], smem + W::kRhs + k * 1024 + 512 + lane * 16);
          undo[k] = rhs_by[k * 8 + g];
        }
        float x[kBlocks][2][4] = {};
#pragma unroll
        for (int part = 0; part < 3; ++part)
#pragma unroll
          for (int k = 0; k < kBlocks; ++k)
#pragma unroll
            for (int u = 0; u < 2; ++u)
              mma<Fp16>(x[k][u], part == 1 ? lo[k] : hi[k], part == 2 ? b_lo[k][2 * u] : b[k][2 * u], part == 2 ? b_lo[k][2 * u + 1] : b[k][2 * u + 1]);
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int u = 0; u < 2; ++u) add_scaled(w[u], x[k][u], undo[k]);
      };
      if (warp == 0) solve(std::integral_constant<int, 1>());
      else if (warp == 1) solve(std::integral_constant<int, 2>());
      else if (warp == 2) solve(std::integral_constant<int, 3>());
      else solve(std::integral_constant<int, 4>());
      {
        const Scaled by = scaled_for(w[0], w[1]);
        float2 x[4];
        times(x, w[0], w[1], by.up);
        left_factor(x, smem + W::kPlain + warp * 1024 + lane * 16, smem + W::kPlain + warp * 1024 + 512 + lane * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = mul2(x[k], make_float2(write[k >> 1][0], write[k >> 1][1]));
        left_factor(x, smem + W::kWrite + warp * 1024 + lane * 16, smem + W::kWrite + warp * 1024 + 512 + lane * 16);
        if (c == 0) plain_by[warp * 8 + g] = by.down;
      }
      // The state after the chunk.
      {
        uint32_t hi[4][4], lo[4][4], b[4][kTiles / 2][4];
        float2 undo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < kTiles; j += 2) load_matrices_t(b[k][j / 2], rows + image_at(16 * k + t_row, warp * kTiles + j + t_vec));
        const float decay = f.decay;
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) state[j][e] *= decay;
        meet<256>(kWThere);  // S has been read
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          left_load(hi[k], smem + W::kWrite + k * 1024 + lane * 16);
          left_load(lo[k], smem + W::kWrite + k * 1024 + 512 + lane * 16);
          undo[k] = plain_by[k * 8 + g];
          const float into = f.into[k];
          undo[k].x *= into, undo[k].y *= into;
        }
        float x[4][kTiles][4] = {};
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < kTiles; ++j) mma<Fp16>(x[k][j], part ? lo[k] : hi[k], b[k][j / 2][2 * (j & 1)], b[k][j / 2][2 * (j & 1) + 1]);
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
#pragma unroll
          for (int k = 0; k < 4; ++k) add_scaled(state[j], x[k][j], undo[k]);
        }
      }
      publish();
      values_there(i + 1);
    }
  }
  if (__syncthreads_or(dead || ((flags_s[0] | flags_s[1]) & kDead))) {
    if (threadIdx.x == 256) {
      *p.timeout = 1;
      // copies may still be on their way: their end, however short the waits' limit is
      if (i < chunks && !(p.stall == 1 && i == 1)) bar_wait(bars + 8 * (i & 1), i >> 1 & 1, kDefaultWaitCycles);
      if (i > 0 && !(p.stall == 2 && i == 1)) bar_wait(bars + 16, (i - 1) & 1, kDefaultWaitCycles);
    }
    __syncthreads();
    return;
  }
  if (all_warps >= 4) return;
#pragma unroll
  for (int k = 0; k < kTiles; ++k)
#pragma unroll
    for (int r = 0; r < 2; ++r)
      if (p0 + 8 * r < p.head_dim)
        *reinterpret_cast<float2*>(keep + (state_at + (g + 8 * r) * N + k * 8) * 4) = make_float2(state[k][2 * r], state[k][2 * r + 1]);
}

template <class E, int N>
cudaError_t chunks(const DeltaParams& p, cudaStream_t s) {
  DeltaParams q = p;
  q.token_ctas = p.by_token >= 0 ? token_ctas<N>(p.head_dim) * p.state.num_seqs : 0;
  const cudaError_t e = launch_after(system_kernel<E, N>, dim3((unsigned)(q.token_ctas + p.pieces), p.heads), kThreads, SystemShape<N>::kSmem, s, q);
  if (e != cudaSuccess) return e;
  return launch_after(walk_kernel<E, N>, dim3((p.head_dim + 15) / 16, p.heads, p.long_seqs), kWalkThreads, WalkShape<N>::kSmem, s, p);
}

template <class E, int N>
cudaError_t prepare() {
  const cudaError_t e = cudaFuncSetAttribute(system_kernel<E, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, SystemShape<N>::kSmem);
  return e == cudaSuccess ? cudaFuncSetAttribute(walk_kernel<E, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, WalkShape<N>::kSmem) : e;
}

}  // namespace

cudaError_t launch_delta_chunks(const DeltaParams& p, int type, cudaStream_t s) {
  if (type == KVX_TYPE_BF16) return p.state_dim == 64 ? chunks<Bf16, 64>(p, s) : chunks<Bf16, 128>(p, s);
  return p.state_dim == 64 ? chunks<Fp16, 64>(p, s) : chunks<Fp16, 128>(p, s);
}

cudaError_t prepare_delta_kernels() {
  for (auto prepare : {prepare<Bf16, 64>, prepare<Bf16, 128>, prepare<Fp16, 64>, prepare<Fp16, 128>}) {
    const cudaError_t e = prepare();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace kvx

// rotary_kernels.cu -- new tokens' queries and keys normed and rotated by their position, K/V into the pages.
//
//   x = x rsqrt(mean(x^2) + eps) (w + offset),   (a, b) = (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq
//
// A warp has a token, or, of few tokens, a part of one's rows.  A head's row lies over kLanes lanes, 8 elements each; with y the
// row's elements that x is paired with, every element is  by (x c + y s)  with by the row's norm and factors c = w cos t
// and s = +-w' sin t that all heads of a token share: they are made once for the queries and once for the keys.  y is the
// neighbour's place in the lane for neighbouring pairs; else another lane's whole vector where half of rotary_dim
// is a multiple of 8 (eight shuffles); elsewhere it is read again, element by element.
//
// Angles: a position of 2^20 times a frequency has 2^-4 left of a 32-bit product's 24 bits, so turns are taken in 64-bit
// whole numbers: f / 2 pi in units of 2^-64, times the position, of which the whole turns overflow.  Sine and cosine are
// taken of the rest in 32 bits.  (An SM has two units for 64-bit floats.)
//
// Measured: 16,384 tokens of 24 + 2 x 4 heads x 256, bf16 into e4m3 (503 MB): 96 us, 5.2 TB/s, 77 % of the DRAM's rate: what is
// left is its 59 million instructions, at 16 warps an SM.  With the way of pairing read from the parameters instead of a
// template's, and rows by indexes instead of pointers, 123 us; with the next rows in registers of their own, every row's sum made by
// all lanes and 256 threads a CTA, 103.  Two rows in flight a lane and 28 warps an SM take 95 there and 37 instead of 27 for
// 4,864 tokens of 32 + 2 x 8 heads x 128.
#include <algorithm>

#include "attend_common.cuh"

namespace kvx {
namespace {

constexpr int kRotaryThreads = 128, kRotaryWarps = kRotaryThreads / 32;
constexpr int kMaxPairs = 128;
constexpr int kRotaryBatch = 4;  // rows' vectors that a lane has in flight

// position * f / 2 pi less its whole part, from -1/2 to 1/2; NaN for an f that is not finite.
__device__ __forceinline__ float turn_of(int64_t position, float f) {
  const uint32_t bits = __float_as_uint(f);
  const int s = 150 - (int)(bits >> 23 & 255);  // f = m 2^-s
  const uint64_t m = (bits & 0x7FFFFFu) | 0x800000u, unit = 0x28BE60DB9391054Aull;  // 2^64 / 2 pi
  const uint64_t hi = __umul64hi(m, unit), lo = m * unit;
  uint64_t turns;
  if (s <= 0)  // 2^23 and more a position
    turns = s > -64 ? lo << -s : 0;
  else if (s < 64)
    turns = hi << (64 - s) | lo >> s;
  else
    turns = s < 128 ? hi >> (s - 64) : 0;
  turns *= (uint64_t)position;
  const float t = __ll2float_rn((int64_t)turns) * 0x1p-64f;
  return (bits & 0x7F800000u) == 0x7F800000u ? NAN : f < 0.f ? -t : t;
}

enum { kNoTurn, kNeighbours, kVectors, kElements };  // how elements are paired

template <class E, int kLanes, bool kFp8, int kPairs>
__global__ void __launch_bounds__(kRotaryThreads, 4) rotary_kernel(const __grid_constant__ RotaryParams p) {
  wait_for_previous();
  constexpr int kRows = 32 / kLanes;           // heads' rows that a warp takes at once
  constexpr int kEach = kRows * kRotaryBatch;  // and that are in flight: a unit of work
  __shared__ float2 turns[kRotaryWarps][kMaxPairs];  // cosine and sine
  const AppendParams& a = p.append;
  const PagesView& v = a.pages;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / kLanes, vec = lane % kLanes;
  const int64_t at = (int64_t)blockIdx.x * kRotaryWarps + warp, token = p.parts == 1 ? at : at / p.parts;
  if (token >= a.tokens) return;
  const int32_t part = (int32_t)(at - token * p.parts);
  int32_t s;
  int64_t back;
  if (!find_row(a.starts, a.num_seqs, a.new_tokens, token, &s, &back)) return;
  if (lane == 0 && part == 0) check_length(v, s);
  const int64_t place = length_of(v, s) - back;
  const bool used = vec * 8 < v.head_dim;

  // Units: queries', keys', values', in that order.
  const int32_t q_units = (p.q_heads + kEach - 1) / kEach, k_units = (v.heads + kEach - 1) / kEach, units = q_units + 2 * k_units;
  const uint8_t* q_at = p.q + token * p.q_token + sub * p.q_head + vec * 16;
  const uint8_t* k_at = a.key + token * a.key_token + sub * a.key_head + vec * 16;
  const uint8_t* v_at = a.value + token * a.value_token + sub * a.value_head + vec * 16;
  uint4 raw[kRotaryBatch];
  auto load = [&](int32_t u) {
    if (u >= units) return;
    auto from = [&](const uint8_t* base, int64_t head, int32_t h0, int32_t heads) {
      const int32_t rest = used ? heads - h0 - sub : 0;
      const uint8_t* at = base + h0 * head;
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k, at += kRows * head)
        raw[k] = k * kRows < rest ? __ldcs(reinterpret_cast<const uint4*>(at)) : make_uint4(0, 0, 0, 0);
    };
    if (u < q_units)
      from(q_at, p.q_head, u * kEach, p.q_heads);
    else if (u < q_units + k_units)
      from(k_at, a.key_head, (u - q_units) * kEach, v.heads);
    else
      from(v_at, a.value_head, (u - q_units - k_units) * kEach, v.heads);
  };
  int32_t u = part;
  load(u);
  const uint32_t row = place < 0 ? kNoRow : row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)place);
  const int32_t half = p.rotary_dim / 2;
  float2* turn = turns[warp];
  const int64_t position = p.positions ? p.positions[token] : place;
  if (kPairs != kNoTurn && u < q_units + k_units)
    for (int32_t i = lane; i < half; i += 32) {
      float sine, cosine;
      sincospif(2.f * turn_of(position, p.inv_freq[i]), &sine, &cosine);
      turn[i] = make_float2(cosine * p.rotary_scale, sine * p.rotary_scale);
    }
  __syncwarp();

  // How an element of this lane is paired, and its factors of x and of y.  A vector that is not turned is its own partner, with
  // half of the weight in both factors, which is exact and leaves an infinite element infinite.
  const int32_t half_vecs = half / 8;
  const bool turned = vec * 8 < 2 * half;
  const int other = sub * kLanes + (kPairs == kVectors && turned ? (vec < half_vecs ? vec + half_vecs : vec - half_vecs) : vec);
  auto partner = [&](int32_t i) { return kPairs == kNeighbours ? i ^ 1 : i < half ? i + half : i - half; };
  float2 c[4], y_by[4];
  auto factors = [&](const uint8_t* weights) {
    const typename E::T* w = reinterpret_cast<const typename E::T*>(weights);
    auto weight = [&](int32_t i) { return w && i < v.head_dim ? E::up(w[i]) + p.weight_offset : 1.f; };
    float cs[8], ys[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int32_t i = vec * 8 + j;
      cs[j] = weight(i), ys[j] = 0.f;
      if (kPairs == kVectors && !turned) cs[j] = ys[j] = 0.5f * cs[j];
      if (kPairs != kNoTurn && i < 2 * half) {
        const bool low = kPairs == kNeighbours ? !(i & 1) : i < half;
        const float2 t = turn[kPairs == kNeighbours ? i >> 1 : low ? i : i - half];
        cs[j] *= t.x, ys[j] = weight(partner(i)) * (low ? -t.y : t.y);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = make_float2(cs[2 * j], cs[2 * j + 1]), y_by[j] = make_float2(ys[2 * j], ys[2 * j + 1]);
  };
  const float k_inverse = 1.f / a.k_scale, v_inverse = 1.f / a.v_scale;
  auto unpack = [&](const uint4& q, float2 (&x)[4]) { x[0] = unpack2<E>(q.x), x[1] = unpack2<E>(q.y), x[2] = unpack2<E>(q.z), x[3] = unpack2<E>(q.w); };
  auto packed = [&](const float2 (&x)[4]) {
    return make_uint4(pack2<E>(x[0].x, x[0].y), pack2<E>(x[1].x, x[1].y), pack2<E>(x[2].x, x[2].y), pack2<E>(x[3].x, x[3].y));
  };
  // Rows normed and turned, step by step for all of the unit, as none waits for another.
  auto turn_rows = [&](float2 (&x)[kRotaryBatch][4], bool normed, const uint8_t* from, int64_t head, int32_t rest) {
    float by[kRotaryBatch];
    if (normed) {
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k) {
        float2 sum = mul2(x[k][0], x[k][0]);
#pragma unroll
        for (int j = 1; j < 4; ++j) sum = fma2(x[k][j], x[k][j], sum);
        by[k] = sum.x + sum.y;
      }
#pragma unroll
      for (int m = kLanes / 2, left = kRotaryBatch / 2; left; left /= 2, m /= 2) {  // a half of the lanes goes on with a half of the rows
        const bool upper = lane & m;
#pragma unroll
        for (int k = 0; k < left; ++k) {
          const float send = upper ? by[k] : by[k + left], stay = upper ? by[k + left] : by[k];
          by[k] = stay + __shfl_xor_sync(~0u, send, m);
        }
      }
#pragma unroll
      for (int m = kLanes / (2 * kRotaryBatch); m; m >>= 1) by[0] += __shfl_xor_sync(~0u, by[0], m);
      const float mine = rsqrtf(fmaf(by[0], p.inverse_dim, p.eps));
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k) by[k] = __shfl_sync(~0u, mine, sub * kLanes + k * (kLanes / kRotaryBatch));
    }
#pragma unroll
    for (int k = 0; k < kRotaryBatch; ++k) {
      float2 y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int32_t i = vec * 8 + 2 * j;
        if constexpr (kPairs == kNeighbours) {
          y[j] = i < 2 * half ? make_float2(x[k][j].y, x[k][j].x) : make_float2(0.f, 0.f);
        } else if constexpr (kPairs == kVectors) {
          y[j].x = __shfl_sync(~0u, x[k][j].x, other), y[j].y = __shfl_sync(~0u, x[k][j].y, other);
        } else if constexpr (kPairs == kElements) {
          const typename E::T* at = reinterpret_cast<const typename E::T*>(from + k * kRows * head - vec * 16);
          const bool there = k * kRows < rest;
          y[j].x = there && i < 2 * half ? E::up(at[partner(i)]) : 0.f;
          y[j].y = there && i + 1 < 2 * half ? E::up(at[partner(i + 1)]) : 0.f;
        }
      }
      if constexpr (kPairs == kElements) __syncwarp();  // q_out may be q: the row's elements have been read
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[k][j] = mul2(x[k][j], c[j]);
        if constexpr (kPairs != kNoTurn) x[k][j] = fma2(y[j], y_by[j], x[k][j]);
        if (normed) x[k][j] = mul2(x[k][j], make_float2(by[k], by[k]));
      }
    }
  };
  auto put = [&](const float2 (&x)[4], uint8_t* to, float scale, float inverse) {  // into the cache
    if constexpr (kFp8)
      *reinterpret_cast<uint2*>(to) = make_uint2(to_e4m3(x[0], scale, inverse) | to_e4m3(x[1], scale, inverse) << 16,
                                                 to_e4m3(x[2], scale, inverse) | to_e4m3(x[3], scale, inverse) << 16);
    else
      *reinterpret_cast<uint4*>(to) = packed(x);
  };
  constexpr int kCacheVec = kFp8 ? 8 : 16;  // bytes of a vector's elements in the cache
  uint8_t* cache = v.base + (row == kNoRow ? 0 : row) * v.row_bytes + sub * v.head_bytes + vec * kCacheVec;
  bool q_made = false, k_made = false;
  for (; u < units; u += p.parts) {
    if (u < q_units) {
      if (!q_made) factors(p.q_weight), q_made = true;
      const int32_t h0 = u * kEach, rest = used ? p.q_heads - h0 - sub : 0;
      float2 x[kRotaryBatch][4];
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k) unpack(raw[k], x[k]);
      load(u + p.parts);
      turn_rows(x, p.q_weight != nullptr, q_at + h0 * p.q_head, p.q_head, rest);
      uint8_t* to = p.q_out + token * p.out_token + (h0 + sub) * p.out_head + vec * 16;
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k, to += kRows * p.out_head)
        if (k * kRows < rest) *reinterpret_cast<uint4*>(to) = packed(x[k]);
    } else if (u < q_units + k_units) {
      if (!k_made) factors(p.k_weight), k_made = true;
      const int32_t h0 = (u - q_units) * kEach, rest = used ? v.heads - h0 - sub : 0;
      float2 x[kRotaryBatch][4];
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k) unpack(raw[k], x[k]);
      load(u + p.parts);
      turn_rows(x, p.k_weight != nullptr, k_at + h0 * a.key_head, a.key_head, rest);
      uint8_t* to = cache + h0 * v.head_bytes;
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k, to += kRows * v.head_bytes)
        if (k * kRows < rest && row != kNoRow) put(x[k], to, a.k_scale, k_inverse);
    } else {
      const int32_t h0 = (u - q_units - k_units) * kEach, rest = used ? v.heads - h0 - sub : 0;
      uint8_t* to = cache + v.half_bytes + h0 * v.head_bytes;
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k, to += kRows * v.head_bytes) {
        if (!(k * kRows < rest && row != kNoRow)) continue;
        if constexpr (kFp8) {
          float2 x[4];
          unpack(raw[k], x);
          put(x, to, a.v_scale, v_inverse);
        } else {
          *reinterpret_cast<uint4*>(to) = raw[k];
        }
      }
      load(u + p.parts);
    }
  }
}

template <class E, int kLanes>
cudaError_t rotary(const RotaryParams& p, bool fp8, int num_sms, cudaStream_t s) {
  constexpr int kEach = 32 / kLanes * kRotaryBatch;
  const int32_t units = (p.q_heads + kEach - 1) / kEach + 2 * ((p.append.pages.heads + kEach - 1) / kEach);
  // Few tokens: a warp a unit, as one a token leaves SMs idle; many: a warp a token, as every unit makes its sines and factors
  // again.  With a warp a unit and a warp a token, in a graph, us, of 2, 4, 6 and 8 tokens an SM: 32 + 2 x 8 heads x 128 5.2 8.5 11.5 12.5 and
  // 8.0 8.1 8.8 8.9; 16 + 2 x 8 x 96 4.9 5.3 9.1 9.6 and 7.4 7.4 7.8 7.9; 24 + 2 x 4 x 256 into e4m3 6.5 11.5 15.9 20.1 and 10.5 10.6 11.6
  // 11.6; 4 + 2 x 2 x 64 4.1 4.6 7.5 7.6 and 5.6 5.5 5.9 5.9; 64 + 2 x 8 x 128 8.2 11.8 15.6 19.7 and 10.6 10.6 11.7 11.8.
  RotaryParams q = p;
  q.parts = p.append.tokens > 4 * num_sms ? 1 : units;
  q.inverse_dim = 1.f / p.append.pages.head_dim;
  const dim3 grid((unsigned)((p.append.tokens * q.parts + kRotaryWarps - 1) / kRotaryWarps));
  auto launch = [&](auto pairs) {
    constexpr int kPairs = decltype(pairs)::value;
    return launch_after(fp8 ? rotary_kernel<E, kLanes, true, kPairs> : rotary_kernel<E, kLanes, false, kPairs>, grid, kRotaryThreads, 0, s, q);
  };
  if (p.rotary_dim == 0) return launch(std::integral_constant<int, kNoTurn>());
  if (p.interleaved) return launch(std::integral_constant<int, kNeighbours>());
  return p.rotary_dim % 16 == 0 ? launch(std::integral_constant<int, kVectors>()) : launch(std::integral_constant<int, kElements>());
}

template <class E>
cudaError_t rotary(const RotaryParams& p, bool fp8, int num_sms, cudaStream_t s) {
  const int32_t d = p.append.pages.head_dim;
  return d <= 64 ? rotary<E, 8>(p, fp8, num_sms, s) : d <= 128 ? rotary<E, 16>(p, fp8, num_sms, s) : rotary<E, 32>(p, fp8, num_sms, s);
}

}  // namespace

cudaError_t launch_rotary(const RotaryParams& p, int type, int cache_type, int num_sms, cudaStream_t s) {
  const bool fp8 = cache_type == KVX_TYPE_E4M3;
  return type == KVX_TYPE_BF16 ? rotary<Bf16>(p, fp8, num_sms, s) : rotary<Fp16>(p, fp8, num_sms, s);
}

}  // namespace kvx

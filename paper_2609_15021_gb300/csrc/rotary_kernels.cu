// rotary_kernels.cu -- new tokens' queries and keys normed and rotated by their position, K/V into the pages.
//
//   x = x rsqrt(mean(x^2) + eps) (w + offset),   (a, b) = (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq
//
// A warp has a token, or, of few tokens, a part of one's rows.  A head's row lies over kLanes lanes, 8 elements each; with y the
// row's elements that x is paired with, every element is  by (x c + y s)  with by the row's norm and factors c = w cos t
// and s = +-w' sin t that all heads of a token share: they are made once for the queries and once for the keys.  y is the
// neighbour's place in the lane for neighbouring pairs; else another lane's whole vector where half of rotary_dim
// is a multiple of 8 (four shuffles of raw pairs); elsewhere it is read again, element by element.
//
// Angles: a position of 2^20 times a frequency has 2^-4 left of a 32-bit product's 24 bits, so turns are taken in 64-bit
// whole numbers: f / 2 pi in units of 2^-64, times the position, of which the whole turns overflow.  Sine and cosine are
// taken of the rest in 32 bits.  (In 64-bit floats, of which an SM has two units, they took a third of the time.)
#include <algorithm>

#include "attend_common.cuh"

namespace kvx {
namespace {

constexpr int kRotaryThreads = 256, kRotaryWarps = kRotaryThreads / 32;
constexpr int kMaxPairs = 128;
constexpr int kRotaryBatch = 4;  // rows' vectors that a lane has in flight

// position * f / 2 pi less its whole part, from -1/2 to 1/2.
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
  return f < 0.f ? -t : t;
}

enum { kNoTurn, kNeighbours, kVectors, kElements };  // how elements are paired

template <class E, int kLanes, bool kFp8, int kPairs>
__global__ void __launch_bounds__(kRotaryThreads, 2) rotary_kernel(const __grid_constant__ RotaryParams p) {
  wait_for_previous();
  constexpr int kRows = 32 / kLanes;        // heads' rows that a warp takes at once
  constexpr int kEach = kRows * kRotaryBatch;  // and that are in flight: a unit of work
  __shared__ float2 turns[kRotaryWarps][kMaxPairs];  // cosine and sine
  const AppendParams& a = p.append;
  const PagesView& v = a.pages;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / kLanes, vec = lane % kLanes;
  const int64_t at = (int64_t)blockIdx.x * kRotaryWarps + warp, token = at / p.parts;
  if (token >= a.tokens) return;
  const int32_t part = (int32_t)(at - token * p.parts);
  int32_t s;
  int64_t back;
  if (!find_row(a.starts, a.num_seqs, a.new_tokens, token, &s, &back)) return;
  if (lane == 0 && part == 0) check_length(v, s);
  const int64_t place = length_of(v, s) - back;
  const bool used = vec * 8 < v.head_dim;

  // Units: queries', keys', values'.
  const int32_t q_units = (p.q_heads + kEach - 1) / kEach, k_units = (v.heads + kEach - 1) / kEach, units = q_units + 2 * k_units;
  auto set_of = [&](int32_t u) { return u < q_units ? 0 : u < q_units + k_units ? 1 : 2; };
  auto first_of = [&](int32_t u) { return (u - (u < q_units ? 0 : u < q_units + k_units ? q_units : q_units + k_units)) * kEach + sub; };
  auto source = [&](int set, int32_t h) {
    return set == 0 ? p.q + token * p.q_token + h * p.q_head
                    : set == 1 ? a.key + token * a.key_token + h * a.key_head : a.value + token * a.value_token + h * a.value_head;
  };
  uint4 raw[kRotaryBatch], next[kRotaryBatch];
  auto load = [&](int32_t u, uint4 (&to)[kRotaryBatch]) {
    const int set = set_of(u);
    const int32_t h0 = first_of(u), heads = set ? v.heads : p.q_heads;
#pragma unroll
    for (int k = 0; k < kRotaryBatch; ++k) {
      const int32_t h = h0 + k * kRows;
      to[k] = h < heads && used ? __ldcs(reinterpret_cast<const uint4*>(source(set, h)) + vec) : make_uint4(0, 0, 0, 0);
    }
  };
  int32_t u = part;
  if (u < units) load(u, raw);
  const uint32_t row = place < 0 ? kNoRow : row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)place);
  const int32_t half = p.rotary_dim / 2;
  float2* turn = turns[warp];
  const int64_t position = p.positions ? p.positions[token] : place;
  if (kPairs != kNoTurn && set_of(u) < 2)
    for (int32_t i = lane; i < half; i += 32) {
      float sine, cosine;
      sincospif(2.f * turn_of(position, p.inv_freq[i]), &sine, &cosine);
      turn[i] = make_float2(cosine * p.rotary_scale, sine * p.rotary_scale);
    }
  __syncwarp();

  // How an element of this lane is paired.
  const int32_t half_vecs = half / 8;
  const bool turned = vec * 8 < 2 * half;  // some of the lane's are
  const int32_t other = kPairs == kVectors && turned ? (vec < half_vecs ? vec + half_vecs : vec - half_vecs) : vec;
  auto partner = [&](int32_t i) { return kPairs == kNeighbours ? i ^ 1 : i < half ? i + half : i - half; };
  float2 c[4], y_by[4];  // factors of x and of y
  auto factors = [&](int set) {
    const typename E::T* w = reinterpret_cast<const typename E::T*>(set ? p.k_weight : p.q_weight);
    auto weight = [&](int32_t i) { return w && i < v.head_dim ? E::up(w[i]) + p.weight_offset : 1.f; };
    float cs[8], ys[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int32_t i = vec * 8 + j;
      cs[j] = weight(i), ys[j] = 0.f;
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
  int set = -1;
  for (; u < units; u += p.parts) {
    const int32_t ahead = u + p.parts;
    if (ahead < units) load(ahead, next);
    const int now = set_of(u);
    if (now != set && now < 2) factors(now);
    set = now;
    const bool normed = set == 0 ? p.q_weight != nullptr : set == 1 && p.k_weight;
    const int32_t h0 = first_of(u), heads = set ? v.heads : p.q_heads;
    // All rows of the unit step by step, as none waits for another.
    float2 x[kRotaryBatch][4];
#pragma unroll
    for (int k = 0; k < kRotaryBatch; ++k) {
      const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) x[k][j] = unpack2<E>(w[j]);
    }
    if (now < 2) {
      float by[kRotaryBatch];
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k) by[k] = 1.f;
      if (normed) {
#pragma unroll
        for (int k = 0; k < kRotaryBatch; ++k) {
          float2 sum = mul2(x[k][0], x[k][0]);
#pragma unroll
          for (int j = 1; j < 4; ++j) sum = fma2(x[k][j], x[k][j], sum);
          by[k] = sum.x + sum.y;
        }
#pragma unroll
        for (int m = kLanes / 2; m; m >>= 1)
#pragma unroll
          for (int k = 0; k < kRotaryBatch; ++k) by[k] += __shfl_xor_sync(~0u, by[k], m);
#pragma unroll
        for (int k = 0; k < kRotaryBatch; ++k) by[k] = rsqrtf(by[k] * p.inverse_dim + p.eps);
      }
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k) {
        const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
        const int32_t h = h0 + k * kRows;
        float2 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int32_t i = vec * 8 + 2 * j;
          y[j] = make_float2(0.f, 0.f);
          if constexpr (kPairs == kNeighbours) {
            if (i < 2 * half) y[j] = make_float2(x[k][j].y, x[k][j].x);
          } else if constexpr (kPairs == kVectors) {
            const uint32_t o = __shfl_sync(~0u, w[j], sub * kLanes + other);
            y[j] = unpack2<E>(turned ? o : 0);
          } else if constexpr (kPairs == kElements) {
            const typename E::T* from = reinterpret_cast<const typename E::T*>(source(now, h < heads ? h : 0));
            if (i < 2 * half && used) y[j].x = E::up(from[partner(i)]);
            if (i + 1 < 2 * half && used) y[j].y = E::up(from[partner(i + 1)]);
          }
        }
        if constexpr (kPairs == kElements) __syncwarp();  // q_out may be q: the row's elements have been read
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[k][j] = mul2(x[k][j], c[j]);
          if constexpr (kPairs != kNoTurn) x[k][j] = fma2(y[j], y_by[j], x[k][j]);
          x[k][j] = mul2(x[k][j], make_float2(by[k], by[k]));
        }
      }
    }
    if (used && (now == 0 || row != kNoRow)) {
      uint8_t* to = now == 0 ? p.q_out + token * p.out_token : v.base + row * v.row_bytes + (now == 2 ? v.half_bytes : 0);
      const int64_t head = now == 0 ? p.out_head : v.head_bytes;
#pragma unroll
      for (int k = 0; k < kRotaryBatch; ++k) {
        const int32_t h = h0 + k * kRows;
        if (h >= heads) continue;
        if (kFp8 && now > 0) {
          const float scale = now == 2 ? a.v_scale : a.k_scale, inverse = now == 2 ? v_inverse : k_inverse;
          *(reinterpret_cast<uint2*>(to + h * head) + vec) = make_uint2(to_e4m3(x[k][0], scale, inverse) | to_e4m3(x[k][1], scale, inverse) << 16,
                                                                       to_e4m3(x[k][2], scale, inverse) | to_e4m3(x[k][3], scale, inverse) << 16);
        } else if (now == 2) {
          *(reinterpret_cast<uint4*>(to + h * head) + vec) = raw[k];
        } else {
          *(reinterpret_cast<uint4*>(to + h * head) + vec) = make_uint4(pack2<E>(x[k][0].x, x[k][0].y), pack2<E>(x[k][1].x, x[k][1].y),
                                                                       pack2<E>(x[k][2].x, x[k][2].y), pack2<E>(x[k][3].x, x[k][3].y));
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kRotaryBatch; ++k) raw[k] = next[k];
  }
}

template <class E, int kLanes>
cudaError_t rotary(const RotaryParams& p, bool fp8, int num_sms, cudaStream_t s) {
  constexpr int kEach = 32 / kLanes * kRotaryBatch;
  const int32_t units = (p.q_heads + kEach - 1) / kEach + 2 * ((p.append.pages.heads + kEach - 1) / kEach);
  // few tokens: a warp a unit
  RotaryParams q = p;
  q.parts = p.append.tokens >= 8 * num_sms ? 1 : units;
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

// rotary_kernels.cu -- new tokens' queries and keys normed and rotated by their position, K/V into the pages.
//
//   x = x rsqrt(mean(x^2) + eps) (w + offset),   (a, b) = (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq
//
// A head's row lies over kLanes lanes, 8 elements each, so its sum of squares is a reduction of a few steps and a rotation
// of neighbouring pairs stays within a lane.  Of the other kind a lane's partners are another lane's whole vector,
// where half of rotary_dim is a multiple of 8, and come by four shuffles of raw pairs; they are normed here once more, which
// takes less than passing 32-bit numbers.  Elsewhere they are read again, element by element.
//
// Angles: a position of 2^20 times a frequency has 2^-4 left of a 32-bit product's 24 bits, so turns are taken in 64
// bits, p f / 2 pi less its whole part, and their sine and cosine in 32.  That is done once a token, by the CTA that
// has it, for all heads.
//
// Bound by the rows' bytes, in and out.
#include <algorithm>

#include "attend_common.cuh"

namespace kvx {
namespace {

constexpr int kRotaryThreads = 256, kRotaryWarps = kRotaryThreads / 32;
constexpr int kMaxPairs = 128;

template <class E, int kLanes, bool kFp8>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  wait_for_previous();
  constexpr int kRows = 32 / kLanes;  // heads' rows that a warp takes at once
  constexpr int kBatch = 4;           // times that, in flight
  __shared__ float2 turn[kMaxPairs];  // cosine and sine
  const AppendParams& a = p.append;
  const PagesView& v = a.pages;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / kLanes, vec = lane % kLanes;
  const int64_t token = blockIdx.x;
  int32_t s;
  int64_t back;
  if (!find_row(a.starts, a.num_seqs, a.new_tokens, token, &s, &back)) return;
  if (threadIdx.x == 0 && blockIdx.y == 0) check_length(v, s);
  const int64_t place = length_of(v, s) - back;
  const int32_t all = p.q_heads + 2 * v.heads;  // rows of a token: queries, keys, values
  const bool used = vec * 8 < v.head_dim;

  // The place of a row, and its first vectors before the angles are made.
  auto source = [&](int32_t r) -> const uint8_t* {
    if (r < p.q_heads) return p.q + token * p.q_token + r * p.q_head;
    r -= p.q_heads;
    if (r < v.heads) return a.key + token * a.key_token + r * a.key_head;
    return a.value + token * a.value_token + (r - v.heads) * a.value_head;
  };
  const int32_t step = gridDim.y * kRotaryWarps * kRows;
  int32_t r0 = (blockIdx.y * kRotaryWarps + warp) * kRows + sub;
  uint4 raw[kBatch];
  auto load = [&](int32_t r0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      raw[u] = r0 + u * step < all && used ? __ldcs(reinterpret_cast<const uint4*>(source(r0 + u * step)) + vec) : make_uint4(0, 0, 0, 0);
  };
  load(r0);
  const uint32_t row = place < 0 ? kNoRow : row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)place);
  const int32_t half = p.rotary_dim / 2;
  if (threadIdx.x < half) {
    const int64_t position = p.positions ? p.positions[token] : place;
    const double turns = (double)position * (double)p.inv_freq[threadIdx.x] * 0.15915494309189535;  // 1 / 2 pi
    float sine, cosine;
    sincospif(2.f * (float)(turns - rint(turns)), &sine, &cosine);
    turn[threadIdx.x] = make_float2(cosine * p.rotary_scale, sine * p.rotary_scale);
  }
  __syncthreads();

  const bool whole_vectors = half % 8 == 0;
  const int32_t half_vecs = half / 8;
  for (; r0 - sub < all; r0 += kBatch * step) {  // the same for all lanes
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int32_t r = r0 + u * step;
      if (r - sub >= all) break;
      const bool there = r < all && used;
      const bool is_q = r < p.q_heads, is_v = r >= p.q_heads + v.heads;
      const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
      float x[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = unpack2<E>(w[j]);
        x[2 * j] = f.x, x[2 * j + 1] = f.y;
      }
      float by = 1.f;
      const uint8_t* weight = is_q ? p.q_weight : p.k_weight;
      if (p.q_weight || p.k_weight) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
#pragma unroll
        for (int m = kLanes / 2; m; m >>= 1) sum += __shfl_xor_sync(~0u, sum, m);
        by = rsqrtf(sum / v.head_dim + p.eps);
      }
      if (is_v) weight = nullptr;
      auto normed = [&](float (&x)[8], int32_t vec) {
        if (!weight || vec * 8 >= v.head_dim) return;
        const uint4 g = *(reinterpret_cast<const uint4*>(weight) + vec);
        const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = unpack2<E>(gw[j]);
          x[2 * j] = x[2 * j] * by * (f.x + p.weight_offset);
          x[2 * j + 1] = x[2 * j + 1] * by * (f.y + p.weight_offset);
        }
      };
      if (half > 0) {
        if (p.interleaved) {
          normed(x, vec);
          if (!is_v) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int32_t i = vec * 4 + j;
              if (i >= half) break;
              const float2 cs = turn[i];
              const float left = x[2 * j], right = x[2 * j + 1];
              x[2 * j] = left * cs.x - right * cs.y;
              x[2 * j + 1] = right * cs.x + left * cs.y;
            }
          }
        } else if (whole_vectors) {
          const bool low = vec < half_vecs, high = !low && vec < 2 * half_vecs;
          const int32_t other = low ? vec + half_vecs : high ? vec - half_vecs : vec;
          float y[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 f = unpack2<E>(__shfl_sync(~0u, w[j], sub * kLanes + other));
            y[2 * j] = f.x, y[2 * j + 1] = f.y;
          }
          normed(x, vec);
          normed(y, other);
          if (!is_v && (low || high)) {
            const int32_t i0 = (low ? vec : other) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float2 cs = turn[i0 + j];
              x[j] = x[j] * cs.x + (low ? -cs.y : cs.y) * y[j];
            }
          }
        } else {
          normed(x, vec);
          if (there && !is_v) {
            const typename E::T* from = reinterpret_cast<const typename E::T*>(source(r));
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
              const int32_t i = vec * 8 + j;
              if (i >= 2 * half) break;
              const bool low = i < half;
              const int32_t o = low ? i + half : i - half;
              float y = E::up(from[o]);
              if (weight) y = y * by * (E::up(reinterpret_cast<const typename E::T*>(weight)[o]) + p.weight_offset);
              const float2 cs = turn[low ? i : o];
              // x[j] by a number that the compiler does not know would put x into memory
              float mine = 0.f;
#pragma unroll
              for (int k = 0; k < 8; ++k) mine = k == j ? x[k] : mine;
              mine = mine * cs.x + (low ? -cs.y : cs.y) * y;
#pragma unroll
              for (int k = 0; k < 8; ++k) x[k] = k == j ? mine : x[k];
            }
          }
          __syncwarp();  // q_out may be q: its elements have been read
        }
      } else {
        normed(x, vec);
      }
      if (!there) continue;
      if (is_q || !kFp8) {
        uint8_t* to;
        if (is_q) {
          to = p.q_out + token * p.out_token + r * p.out_head;
        } else {
          if (row == kNoRow) continue;
          const int32_t h = r - p.q_heads - (is_v ? v.heads : 0);
          to = v.base + row * v.row_bytes + (is_v ? v.half_bytes : 0) + h * v.head_bytes;
        }
        *(reinterpret_cast<uint4*>(to) + vec) = make_uint4(pack2<E>(x[0], x[1]), pack2<E>(x[2], x[3]), pack2<E>(x[4], x[5]), pack2<E>(x[6], x[7]));
      } else if (row != kNoRow) {
        const int32_t h = r - p.q_heads - (is_v ? v.heads : 0);
        uint8_t* to = v.base + row * v.row_bytes + (is_v ? v.half_bytes : 0) + h * v.head_bytes;
        const float scale = is_v ? a.v_scale : a.k_scale, inverse = 1.f / scale;
        uint32_t o[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          o[k] = to_e4m3(make_float2(x[4 * k], x[4 * k + 1]), scale, inverse) |
                 to_e4m3(make_float2(x[4 * k + 2], x[4 * k + 3]), scale, inverse) << 16;
        *(reinterpret_cast<uint2*>(to) + vec) = make_uint2(o[0], o[1]);
      }
    }
    if (r0 - sub + kBatch * step < all) load(r0 + kBatch * step);
  }
}

template <class E, int kLanes>
cudaError_t rotary(const RotaryParams& p, bool fp8, int num_sms, cudaStream_t s) {
  constexpr int kEach = kRotaryWarps * (32 / kLanes);
  const int32_t all = p.q_heads + 2 * p.append.pages.heads;
  // few tokens: a warp's rows at a time are all that a warp has
  const int parts = p.append.tokens >= 4 * num_sms ? 1 : (all + kEach - 1) / kEach;
  const dim3 grid((unsigned)p.append.tokens, parts);
  return launch_after(fp8 ? rotary_kernel<E, kLanes, true> : rotary_kernel<E, kLanes, false>, grid, kRotaryThreads, 0, s, p);
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

// select_kernels.cu -- the bounds of pages' keys, and the pages that each query picks by them.
//
//   score(page) = max over the head's query rows of step * (w+ . high + w- . low), times the page's size
//
// with w+ and w- the positive and the negative part of the row rounded to whole numbers of its step, low and high the page's
// bounds: one product over twice the elements, and no less than the rounded row's product with any key of the page but for what rounding
// sizes and quotients to the nearest leaves a bound short by, 2^-24 of the page's largest element (a whole number of a
// size is 2^-7 of it).  Everything in the sum is whole and below 2^24, so its order does not show, and the same pages are picked whatever the batch.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "mma.cuh"
#include "pick_border.cuh"

namespace kvx {
namespace {

// ---------------------------------------------------------------- bounds

constexpr int kBoundsThreads = 128;

// The least and the greatest of two pairs of keys; NaN where there is one.
template <class C>
struct Pairs {
  using V = __nv_bfloat162;
};
template <>
struct Pairs<Fp16> {
  using V = __half2;
};
template <class C>
__device__ __forceinline__ uint32_t least2(uint32_t a, uint32_t b) {
  using V = typename Pairs<C>::V;
  const V v = __hmin2_nan(*reinterpret_cast<const V*>(&a), *reinterpret_cast<const V*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <class C>
__device__ __forceinline__ uint32_t most2(uint32_t a, uint32_t b) {
  using V = typename Pairs<C>::V;
  const V v = __hmax2_nan(*reinterpret_cast<const V*>(&a), *reinterpret_cast<const V*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Two e4m3 values as fp16.
__device__ __forceinline__ uint32_t widen2(uint32_t v) {
  uint32_t r;
  asm("{\n .reg .b16 a;\n cvt.u16.u32 a, %1;\n cvt.rn.f16x2.e4m3x2 %0, a;\n}" : "=r"(r) : "r"(v & 0xFFFFu));
  return r;
}

// Quotients by one number, rounded to the nearest: as `divided` of attend_common.cuh, where the number leaves the residuals their
// bits, by division elsewhere.
struct Divisor {
  float by, inverse;
  bool plain;
  __device__ __forceinline__ explicit Divisor(float d) : by(d), inverse(1.f / d), plain(d > 0x1p-80f && d < 0x1p80f) {}
  __device__ __forceinline__ float operator()(float x) const {
    if (!plain) return by > 0.f ? __fdiv_rn(x, by) : 0.f;
    const float q = x * inverse;
    return fmaf(fmaf(-q, by, x), inverse, q);
  }
};

// A warp has one head of two pages, one after the other, whose places are looked up at once: its lanes have a row's vectors, some
// rows at once, and meet at the end, the second page's rows under way; then, where a row is half a warp, one half makes the low
// bounds and the other the high ones.  C: the type that keys are compared in
// (fp16 for e4m3).  Bound by the keys' bytes, of which a lane has eight rows' in
// flight: 2 sequences of 21k and 32.8k tokens, 8 heads x 128, bf16 (117 MB with the bounds): 21 us among other
// calls, 81 % of the DRAM's rate (alone in a graph, whose beginning nothing hides, 25; two pages a warp took 4 less than one, and all of a page's
// loads made first 2 less).  After a step's append it has a page a sequence, and is a launch and four loads on end, 2.3 us in a graph of
// such calls.
template <class C, bool kWide, int kVecs>  // kVecs: vectors of a row, rounded up to a power of two
__global__ void __launch_bounds__(kBoundsThreads) bounds_kernel(const __grid_constant__ BoundsParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  constexpr int kPairs = kWide ? 8 : 4;  // of a vector
  constexpr int kRows = 32 / kVecs, kWarps = kBoundsThreads / 32;
  const int lane = threadIdx.x & 31, vec = lane % kVecs, sub = lane / kVecs;
  const int32_t s = blockIdx.y, unit = (int32_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int32_t n = (int32_t)quotient(p.by_heads, (uint32_t)unit), h = unit - n * v.heads;
  if (unit == 0 && lane == 0) check_length(v, s);
  const int32_t length = length_of(v, s), block = (int32_t)v.by_block.d;
  const int32_t page = (int32_t)quotient(v.by_block, (uint32_t)max(length - p.new_tokens, 0)) + 2 * n;  // and the next
  // The sequence's last page may be another's too, which holds more of it: its bounds are those of all keys that any
  // sequence of the batch holds there, so that all warps that make them write the same.  (A token of each of 48 sequences
  // takes 3.2 us in a graph, 2.4 without the search; of 512 6.8 and 4.0, of 2,000 38 and 13.  A search by the CTA, whose barrier the compiler orders
  // all loads around, takes 5.2 of 512, and two long caches 22.5 instead of 21.2.)
  int32_t reach = length;
  const int32_t last = (int32_t)quotient(v.by_block, (uint32_t)max(length - 1, 0));
  if (v.num_seqs > 1 && length > 0 && length - last * block < block && (page == last || page + 1 == last)) {
    const uint32_t at = quotient(v.by_pack, (uint32_t)last);
    if (at < v.table_len) {
      const int32_t entry = __ldg(v.tables + s * v.table_stride + at);
#pragma unroll 4
      for (int32_t other = lane; other < v.num_seqs; other += 32) {
        const int32_t held = length_of(v, other);
        if (held > length && __ldg(v.tables + other * v.table_stride + at) == entry) reach = max(reach, held);
      }
    }
    reach = __reduce_max_sync(~0u, reach);
  }
  uint32_t row[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
    row[j] = 2 * n + j < p.pages_each && (int64_t)(page + j) * block < length
                 ? row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)(page + j) * block)
                 : kNoRow;
  const int64_t step = v.token_rows * v.row_bytes;
  const bool used = vec * 16 < v.row_bytes;
  constexpr int kAtOnce = 8;  // loads in flight
  uint4 x[kAtOnce];
  auto load = [&](int j, int32_t t0) {
    const uint32_t at = j ? row[1] : row[0];
    if (at == kNoRow || !used) return;
    const uint8_t* from = v.base + at * v.row_bytes + h * v.head_bytes + vec * 16;
    const int32_t held = min(block, reach - (page + j) * block);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) x[i] = __ldcs(reinterpret_cast<const uint4*>(from + min(t0 + i * kRows, held - 1) * step));
  };
  load(0, sub);
  constexpr int kUnrolled = kWide ? 1 : 2;  // (e4m3's code twice took 5 us more where a sequence has one page)
#pragma unroll kUnrolled
  for (int j = 0; j < 2; ++j) {
    const uint32_t here = j ? row[1] : row[0];
    constexpr uint32_t kInf = std::is_same<C, Bf16>::value ? 0x7F807F80u : 0x7C007C00u;
    uint32_t low[kPairs], high[kPairs];
#pragma unroll
    for (int k = 0; k < kPairs; ++k) low[k] = used ? kInf : 0, high[k] = used ? kInf | 0x80008000u : 0;
    if (here != kNoRow && used)
      for (int32_t t0 = sub;;) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < kPairs; ++k) {
            const uint32_t u = kWide ? widen2(w[k / 2] >> k % 2 * 16) : w[k];
            low[k] = least2<C>(low[k], u), high[k] = most2<C>(high[k], u);
          }
        }
        t0 += kAtOnce * kRows;
        if (t0 >= min(block, reach - (page + j) * block)) break;
        load(j, t0);
      }
    if (j == 0) load(1, sub);
    if (here == kNoRow) continue;
    __syncwarp();
#pragma unroll
    for (int m = kVecs; m < 32; m <<= 1)
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        low[k] = least2<C>(low[k], __shfl_xor_sync(~0u, low[k], m));
        high[k] = most2<C>(high[k], __shfl_xor_sync(~0u, high[k], m));
      }
    uint32_t most = 0, carries = 0;  // of both numbers' magnitudes, as their bits are in order
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      carries |= odd_carry<C>(low[k]) | odd_carry<C>(high[k]);
      most = __vmaxu2(most, __vmaxu2(low[k] & 0x7FFF7FFFu, high[k] & 0x7FFF7FFFu));
    }
    const bool odd = __any_sync(~0u, odd_carried(carries));
    most = __reduce_max_sync(~0u, max(most & 0xFFFFu, most >> 16));
    const float size = odd ? FLT_MAX : __fdiv_rn(unpack2<C>(most).x, 127.f);
    const int64_t at = (int64_t)(here / v.page_rows) * v.heads + h;
    if (lane == 0) p.sizes[at] = size;
    if (!used || sub > 1) continue;
    const Divisor by(size);
    const bool both = kRows == 1;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      if (!both && side != sub) continue;
      uint32_t out[kPairs / 2];
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        const float2 y = unpack2<C>(side ? high[k] : low[k]);
        float2 r = make_float2(by(y.x), by(y.y));
        r = side ? make_float2(ceilf(r.x), ceilf(r.y)) : make_float2(floorf(r.x), floorf(r.y));
        const int32_t a = (int32_t)fminf(fmaxf(r.x, -127.f), 127.f), b = (int32_t)fminf(fmaxf(r.y, -127.f), 127.f);
        const uint32_t pair = (uint32_t)(a & 0xFF) | (uint32_t)(b & 0xFF) << 8;
        out[k / 2] = k % 2 ? out[k / 2] | pair << 16 : pair;
      }
      if (odd)
#pragma unroll
        for (int k = 0; k < kPairs / 2; ++k) out[k] = side ? 0x7F7F7F7Fu : 0x81818181u;
      int8_t* to = p.boxes + at * 2 * v.head_dim + side * v.head_dim + vec * 2 * kPairs;
      if constexpr (kWide)
        *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[2], out[3]);
      else
        *reinterpret_cast<uint2*>(to) = make_uint2(out[0], out[1]);
    }
  }
}

template <class C, bool kWide>
cudaError_t bounds(const BoundsParams& p, cudaStream_t s) {
  constexpr int kWarps = kBoundsThreads / 32;
  const dim3 grid((unsigned)((((int64_t)p.pages_each + 1) / 2 * p.pages.heads + kWarps - 1) / kWarps), p.pages.num_seqs);
  const int64_t vecs = p.pages.row_bytes / 16;
  auto kernel = vecs <= 4 ? bounds_kernel<C, kWide, 4> : vecs <= 8 ? bounds_kernel<C, kWide, 8> : vecs <= 16 ? bounds_kernel<C, kWide, 16> : bounds_kernel<C, kWide, 32>;
  return launch_after(kernel, grid, kBoundsThreads, 0, s, p);
}

// ---------------------------------------------------------------- scores

constexpr int kScoreThreads = 2 * kScorePages;  // 16 pages a warp

// Elements of a row of whole queries in shared memory: both bounds', padded to 64, and 8 bytes so that eight rows' reads of
// 8 bytes meet no bank twice.
__host__ __device__ constexpr int32_t score_pitch(int32_t head_dim) { return (2 * head_dim + 63) / 64 * 64 + 4; }
__host__ __device__ constexpr int32_t score_smem(int32_t head_dim, int32_t rows) {
  return (rows + 7) / 8 * 8 * (score_pitch(head_dim) * 2 + 4) + kScorePages * ((rows + 7) / 8 * 8 + 1) * 4;
}
constexpr int32_t kScoreMaxSmem = score_smem(256, kMaxScoreGroup);
static_assert(kScoreMaxSmem <= 232448, "shared memory of an SM");

// Four bytes as whole numbers in fp16: 1024 + (byte ^ 128) put together from bits, less 1152.
__device__ __forceinline__ void halves_of(uint32_t bytes, uint32_t& a, uint32_t& b) {
  const uint32_t u = bytes ^ 0x80808080u;
  const __half2 off = __floats2half2_rn(-1152.f, -1152.f);
  uint32_t w[2] = {__byte_perm(u, 0x64646464u, 0x4140), __byte_perm(u, 0x64646464u, 0x4342)};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const __half2 h = __hadd2(*reinterpret_cast<const __half2*>(&w[k]), off);
    w[k] = *reinterpret_cast<const uint32_t*>(&h);
  }
  a = w[0], b = w[1];
}

// A CTA scores 128 pages of one sequence for one KV head: its queries are made whole numbers in shared memory, as the
// right factor of products of 16 pages by 8 query rows with k over the low and the high bounds.  (Bytes are widened to fp16, in
// which they and all their products are exact, as are the sums in fp32.)  The elements of k are taken in an order that lets
// a lane load 16 neighbouring bytes of a page's bounds.  The bounds are few bytes (4 sequences of 99k to 127k tokens, 4 heads x 256,
// pages of 32: 29 MB, 4 us at the DRAM's rate): what counts is that every CTA makes the queries' whole numbers again, and the loads
// on end before its first product.  Those sequences, 4 queries of 24 heads each, take 18 us.  With 128 pages a CTA, the sizes loaded
// beside the queries and whole numbers by a sum, bounds, choice and attention together take 70 us, 75 with 64 pages and without.
template <class E>
__global__ void __launch_bounds__(kScoreThreads) score_kernel(const __grid_constant__ SelectParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  extern __shared__ __align__(16) uint8_t smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, c = lane & 3;
  const int32_t unit = blockIdx.x / p.score_tiles, h = blockIdx.y;
  const int32_t s = unit / p.score_parts, t0 = (unit - s * p.score_parts) * p.tokens_each;
  const int32_t tokens = min(p.tokens_each, p.new_tokens - t0);
  const int32_t length = length_of(v, s), block = (int32_t)v.by_block.d;
  const int32_t pages = length > 0 ? (int32_t)quotient(v.by_block, (uint32_t)(length - 1)) + 1 : 0;  // up to the last query's
  const int32_t page0 = (blockIdx.x - unit * p.score_tiles) * kScorePages;
  if (pages <= p.budget || page0 >= pages) return;  // all are picked
  const int32_t rows = p.group * tokens, tiles = (rows + 7) / 8;
  const int32_t k_all = 2 * v.head_dim, k_pad = (k_all + 63) / 64 * 64, pitch = score_pitch(v.head_dim);
  __half* q_s = reinterpret_cast<__half*>(smem);                       // [8 tiles rows][pitch]
  float* step_s = reinterpret_cast<float*>(q_s + tiles * 8 * pitch);   // [8 tiles]
  float* dots = step_s + tiles * 8;                                    // [warp][16 pages][8 tiles + 1]

  // A page's bounds are under way while the queries are made ready.
  const int32_t* table = v.tables + s * v.table_stride;
  const uint8_t* box[2];
  float size[2] = {0.f, 0.f};
  bool there[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int32_t page = page0 + warp * 16 + quad + 8 * k;
    uint32_t row = kNoRow;
    if (page < pages) row = row_index(v, table, v.table_len, (uint32_t)page * block);
    there[k] = row != kNoRow;
    const int64_t at = (int64_t)(there[k] ? row / v.page_rows : 0) * v.heads + h;
    box[k] = reinterpret_cast<const uint8_t*>(p.boxes) + at * k_all;
    if (there[k]) size[k] = p.sizes[at];
  }

  // Rows of queries, two vectors of 16 bytes in flight: one row a vector, 8 elements a lane (most heads have one or two rows
  // a warp; four in flight are no faster).
  constexpr int kAtOnce = 2, kWarps = kScoreThreads / 32;
  const bool used = lane * 8 < v.head_dim;
  for (int32_t r0 = warp; r0 < tiles * 8; r0 += kAtOnce * kWarps) {
    uint4 raw[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int32_t r = r0 + k * kWarps, t = r / p.group, i = r - t * p.group;
      raw[k] = make_uint4(0, 0, 0, 0);
      if (r < rows && used)
        raw[k] = *(reinterpret_cast<const uint4*>(p.q + ((int64_t)s * p.new_tokens + t0 + t) * p.q_token + (h * p.group + i) * p.q_head) + lane);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int32_t r = r0 + k * kWarps;
      if (r >= tiles * 8) break;
      uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w}, most = 0, carries = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) carries |= odd_carry<E>(w[j]), most = __vmaxu2(most, w[j] & 0x7FFF7FFFu);
      const bool fine = !__any_sync(~0u, odd_carried(carries));
      most = __reduce_max_sync(~0u, max(most & 0xFFFFu, most >> 16));
      const float step = fine ? __fdiv_rn(unpack2<E>(most).x, 127.f) : 0.f;
      if (lane == 0) step_s[r] = step;
      if (!used) continue;
      const Divisor by(step);
      __half2 up[4], down[4];
      const __half2 zero = __floats2half2_rn(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x = unpack2<E>(fine ? w[j] : 0);
        // to whole numbers by a sum that leaves no fraction; a step that lost bits can leave more than 127
        constexpr float kWhole = 12582912.f;  // 1.5 2^23
        const float2 y = make_float2(by(x.x), by(x.y));
        __half2 whole = __floats2half2_rn((y.x + kWhole) - kWhole, (y.y + kWhole) - kWhole);
        if (!by.plain) whole = __hmax2(__hmin2(whole, __floats2half2_rn(127.f, 127.f)), __floats2half2_rn(-127.f, -127.f));
        up[j] = __hmax2(whole, zero), down[j] = __hmin2(whole, zero);
      }
      uint2* to = reinterpret_cast<uint2*>(q_s + r * pitch + lane * 8);
      to[0] = *reinterpret_cast<const uint2*>(&down[0]), to[1] = *reinterpret_cast<const uint2*>(&down[2]);
      to = reinterpret_cast<uint2*>(q_s + r * pitch + v.head_dim + lane * 8);
      to[0] = *reinterpret_cast<const uint2*>(&up[0]), to[1] = *reinterpret_cast<const uint2*>(&up[2]);
    }
  }
  // what is behind the last element, zeros
  for (int32_t i = threadIdx.x; i < tiles * 8 * (k_pad - k_all); i += kScoreThreads) {
    const int32_t r = i / (k_pad - k_all);
    q_s[r * pitch + k_all + i - r * (k_pad - k_all)] = __float2half_rn(0.f);
  }
  __syncthreads();
  const int32_t dot_pitch = tiles * 8 + 1;
  float* mine = dots + warp * 16 * dot_pitch;
  for (int32_t tile0 = 0; tile0 < tiles; tile0 += 4) {  // 32 rows at a time
    float acc[4][4] = {};
    for (int32_t k0 = 0; k0 < k_pad; k0 += 64) {
      const int32_t at = k0 + c * 16;  // bytes of a page's bounds, and elements of a row
      uint4 x[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) x[k] = there[k] && at < k_all ? __ldg(reinterpret_cast<const uint4*>(box[k] + at)) : make_uint4(0, 0, 0, 0);
      const uint32_t w[2][4] = {{x[0].x, x[0].y, x[0].z, x[0].w}, {x[1].x, x[1].y, x[1].z, x[1].w}};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t a[4];
        halves_of(w[0][u], a[0], a[2]);
        halves_of(w[1][u], a[1], a[3]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (tile0 + t >= tiles) break;
          const uint2 b = *reinterpret_cast<const uint2*>(q_s + ((tile0 + t) * 8 + quad) * pitch + at + 4 * u);
          mma<Fp16>(acc[t], a, b.x, b.y);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (tile0 + t >= tiles) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int32_t r = (tile0 + t) * 8 + 2 * c + (e & 1);
        mine[(quad + 8 * (e >> 1)) * dot_pitch + r] = __fmul_rn(acc[t][e], step_s[r]);
      }
    }
  }
  // times the page's size; -inf where no page is named
  const uint32_t live[2] = {__ballot_sync(~0u, there[0]), __ballot_sync(~0u, there[1])};
  __syncwarp();
  const int32_t in = lane % 16, page = page0 + warp * 16 + in;
  const float low = __shfl_sync(~0u, size[0], in % 8 * 4), high = __shfl_sync(~0u, size[1], in % 8 * 4);
  for (int32_t t = lane / 16; t < tokens && page < pages; t += 2) {
    float top = -INFINITY;
    if (live[in / 8] >> (in % 8 * 4) & 1) {
      for (int32_t r = t * p.group; r < (t + 1) * p.group; ++r) top = fmaxf(top, mine[in * dot_pitch + r]);
      top = __fmul_rn(top, in < 8 ? low : high);
    }
    p.scores[(((int64_t)s * p.new_tokens + t0 + t) * v.heads + h) * p.score_stride + page] = top;
  }
}

// ---------------------------------------------------------------- the best

constexpr int kPickThreads = 512, kPickWarps = kPickThreads / 32;
static_assert(kPickBins == 4 * kPickThreads && kPickWarps <= 32, "a thread has four ranges, a lane a warp's sum");

// Whole numbers in the order of the scores: NaN as -inf, -0 as +0.  None is 0.
__device__ __forceinline__ uint32_t score_rank(float w) {
  const uint32_t u = __float_as_uint(fmaxf(w, -INFINITY) + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t upto_lane(uint32_t v) {
  const int lane = threadIdx.x & 31;
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(~0u, v, d);
    if (lane >= d) v += y;
  }
  return v;
}

// A CTA picks the pages of one query and head: the smallest picked score is the budget'th largest.  It is found by counting
// pages in 2,048 equal ranges of what their ranks span, then of the range that it falls in, until all pages of that are
// picked or it is one rank, of whose pages the first are picked: once or twice as a rule, and without many pages in one
// counter, where digits of the ranks themselves, of which a batch's scores share most, take three rounds.  It waits for its loads,
// barriers and counters, not for bytes: 8 us for 64 lists of 4,000 pages as for 384 of up to 1,000.
// A warp has a stretch of neighbouring pages, so that a page's place among the picked follows from ballots and one sum
// over the warps.
__global__ void __launch_bounds__(kPickThreads) pick_kernel(const __grid_constant__ SelectParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  constexpr int kKept = 8;  // ranks that a lane keeps: those of up to 4,096 pages are read once
  __shared__ int32_t hist[kPickBins];
  __shared__ uint32_t warp_a[kPickWarps], warp_b[kPickWarps];
  __shared__ uint32_t bin_s;
  __shared__ int32_t want_s, count_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t token = blockIdx.x / v.heads, h = blockIdx.x - token * v.heads;
  const int32_t s = token / p.new_tokens, t = token - s * p.new_tokens;
  if (threadIdx.x == 0 && h == 0 && t == 0) check_length(v, s);
  const int32_t at = length_of(v, s) - p.new_tokens + t;  // the query's position
  const int32_t n = at < 0 ? 0 : (int32_t)quotient(v.by_block, (uint32_t)at) + 1;
  int32_t* out = p.selected + ((int64_t)token * v.heads + h) * p.budget;
  const int32_t keep = min(n, p.budget);
  for (int32_t i = keep + threadIdx.x; i < p.budget; i += kPickThreads) out[i] = -1;
  if (n <= p.budget) {
    for (int32_t i = threadIdx.x; i < n; i += kPickThreads) out[i] = i;
    return;
  }
  const float* scores = p.scores + ((int64_t)token * v.heads + h) * p.score_stride;
  const int32_t last = n - p.recent;
  // The ranks of pages that are picked by their scores; 0, which no score has, of the others.
  const int32_t each = (n + kPickThreads - 1) / kPickThreads * 32, from = min(warp * each, n), to = min(from + each, n);
  auto always = [&](int32_t i) { return i < p.sinks || i >= last; };
  auto rank = [&](int32_t i) { return i < to && !always(i) ? score_rank(scores[i]) : 0u; };
  uint32_t kept[kKept];
#pragma unroll
  for (int k = 0; k < kKept; ++k) kept[k] = rank(from + k * 32 + lane);
  auto for_each = [&](auto&& f) {  // of the warp's pages, 32 at once
#pragma unroll
    for (int k = 0; k < kKept; ++k)
      if (from + k * 32 < to) f(from + k * 32 + lane, kept[k]);
    for (int32_t i = from + kKept * 32; i < to; i += 32) f(i + lane, rank(i + lane));
  };
  uint32_t low = UINT32_MAX, high = 0;
  for_each([&](int32_t, uint32_t r) {
    if (r) low = min(low, r), high = max(high, r);
  });
  low = __reduce_min_sync(~0u, low), high = __reduce_max_sync(~0u, high);
  if (lane == 0) warp_a[warp] = low, warp_b[warp] = high;
  for (int32_t i = threadIdx.x; i < kPickBins; i += kPickThreads) hist[i] = 0;
  __syncthreads();
  low = __reduce_min_sync(~0u, warp_a[lane % kPickWarps]), high = __reduce_max_sync(~0u, warp_b[lane % kPickWarps]);
  Border search = {low, high, keep - min(p.sinks + p.recent, n)};  // of those picked by their scores, which are more than that
  if (search.want > 0) {
    for (int pass = 0; pass < kPickPasses; ++pass) {
      const int shift = search.shift();
      low = search.low, high = search.high;
      for_each([&](int32_t, uint32_t r) {
        if (r >= low && r <= high) atomicAdd(&hist[(r - low) >> shift], 1);
      });
      __syncthreads();
      // the range of the want'th largest: sums from the top, four ranges a thread
      int32_t b[4], sum = 0;
      const int32_t top_bin = kPickBins - 1 - 4 * (int32_t)threadIdx.x;
#pragma unroll
      for (int k = 0; k < 4; ++k) b[k] = hist[top_bin - k], sum += b[k];
#pragma unroll
      for (int k = 0; k < 4; ++k) hist[top_bin - k] = 0;
      const int32_t upto = (int32_t)upto_lane(sum);
      if (lane == 31) warp_a[warp] = upto;
      if (threadIdx.x == 0) want_s = 0;  // of the range that one thread names, if any does
      __syncthreads();
      const uint32_t mine = lane < kPickWarps && lane < warp ? warp_a[lane] : 0;
      const int32_t before = upto - sum + (int32_t)__reduce_add_sync(~0u, mine);
      int32_t left = search.want - before;
      if (left > 0 && left <= sum) {  // one thread's
        int k = 0;
        while (left > b[k]) left -= b[k++];
        bin_s = (uint32_t)(top_bin - k), want_s = left, count_s = b[k];
      }
      __syncthreads();
      if (!search.narrow(shift, bin_s, want_s, count_s)) break;
    }
  }
  const uint32_t border = search.rank;
  const int32_t equal = search.equal;
  // A page's place: those picked in front of it.
  uint32_t above = 0, same = 0;
  for_each([&](int32_t i, uint32_t r) {
    above += __popc(__ballot_sync(~0u, i < to && (r > border || always(i))));
    same += __popc(__ballot_sync(~0u, r == border && r != 0));
  });
  __syncthreads();  // warp_a has been read
  if (lane == 0) warp_a[warp] = above, warp_b[warp] = same;
  __syncthreads();
  int32_t a = (int32_t)__reduce_add_sync(~0u, lane < warp ? warp_a[lane % kPickWarps] : 0);
  int32_t e = (int32_t)__reduce_add_sync(~0u, lane < warp ? warp_b[lane % kPickWarps] : 0);
  const uint32_t below = (1u << lane) - 1;
  for_each([&](int32_t i, uint32_t r) {
    const bool is_above = i < to && (r > border || always(i)), is_equal = r == border && r != 0;
    const uint32_t a_bits = __ballot_sync(~0u, is_above), e_bits = __ballot_sync(~0u, is_equal);
    const int32_t my_a = a + __popc(a_bits & below), my_e = e + __popc(e_bits & below);
    const int32_t place = my_a + min(my_e, equal);  // below keep, but where another call writes to the same workspace
    if ((is_above || (is_equal && my_e < equal)) && place < keep) out[place] = i;
    a += __popc(a_bits), e += __popc(e_bits);
  });
}

template <class E>
cudaError_t scores(const SelectParams& p, cudaStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.score_tiles * p.score_parts * p.pages.num_seqs), p.pages.heads);
  return launch_after(score_kernel<E>, grid, kScoreThreads, (size_t)score_smem(p.pages.head_dim, p.group * p.tokens_each), s, p);
}

}  // namespace

cudaError_t launch_bounds(const BoundsParams& p, int cache_type, cudaStream_t s) {
  return cache_type == KVX_TYPE_E4M3 ? bounds<Fp16, true>(p, s) : cache_type == KVX_TYPE_BF16 ? bounds<Bf16, false>(p, s) : bounds<Fp16, false>(p, s);
}

cudaError_t launch_select(const SelectParams& p, int type, cudaStream_t s) {
  if (p.score_tiles) {
    const cudaError_t e = type == KVX_TYPE_BF16 ? scores<Bf16>(p, s) : scores<Fp16>(p, s);
    if (e != cudaSuccess) return e;
  }
  return launch_after(pick_kernel, dim3((unsigned)(p.pages.heads * p.pages.num_seqs * p.new_tokens)), kPickThreads, 0, s, p);
}

cudaError_t prepare_select_kernels() {
  const cudaError_t e = cudaFuncSetAttribute(score_kernel<Bf16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kScoreMaxSmem);
  return e == cudaSuccess ? cudaFuncSetAttribute(score_kernel<Fp16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kScoreMaxSmem) : e;
}

}  // namespace kvx

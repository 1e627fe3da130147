// evict_kernels.cu -- choosing the tokens a cache keeps by their accumulated
// attention weight, and moving their rows into fresh pages.

#include <algorithm>
#include <type_traits>

#include "operators.cuh"

namespace kvx {
namespace {

constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 2048;  // digits of 11, 11 and 10 bits

// Whole numbers in the order of the weights: NaN as -inf, -0 as +0.  None is kNone or kAlways.
constexpr uint32_t kNone = 0, kAlways = UINT32_MAX;
__device__ __forceinline__ uint32_t rank_of(float w) {
  const uint32_t u = __float_as_uint(fmaxf(w, -INFINITY) + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
// Sums over the lanes up to this one.
__device__ __forceinline__ uint32_t sum_upto(uint32_t v) {
  const int lane = threadIdx.x & 31;
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(~0u, v, d);
    if (lane >= d) v += y;
  }
  return v;
}

// One CTA per row of weights (head, sequence, layer).  Tokens that are kept whatever their weight have the largest
// rank of all.  The smallest kept weight is found as the m-th largest rank, 11 bits at a time, by counting the ranks
// that share the bits found so far (the first 11 hold the exponent and two bits more, which spreads weights over enough
// counters that a warp's seldom meet); of the tokens that have just that rank the first ones are kept.  A token's place
// among the kept ones is then
//   #(greater before it) + min(#(equal before it), how many equal ones are kept),
// which one scan of pairs of counts gives.  A thread has neighbouring tokens by fours, so that the scan is over a quarter of
// them.  Up to 4096 * kQuads weights are read once and stay in registers; longer rows are read again, tile by tile, for
// every count.  Bound by its instructions, some 40 a weight and warp, and by the counters' banks: 512 rows of 18k to 32k
// weights (51 MB) take 65 us, a CTA an SM (89 with single tokens in the threads' turns and counts by ballots).
template <int kQuads>
__global__ void __launch_bounds__(kSelectThreads, 1) select_kernel(const __grid_constant__ EvictParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  constexpr int kTile = 4 * kSelectThreads * kQuads;
  __shared__ int32_t hist[kBins];
  __shared__ uint32_t counts[kQuads * kSelectWarps];  // greater | equal << 16 of a warp's quads, then those before
  __shared__ uint32_t warp_counts[kSelectWarps];
  __shared__ uint32_t prefix_s;
  __shared__ int32_t want_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t h = blockIdx.x, s = blockIdx.y, l = blockIdx.z;
  const int32_t n = length_of(v, s), keep = min(n, p.budget);
  const float* w = p.weights + l * p.weights_layer + s * p.weights_seq + h * p.weights_head;
  const int64_t row = ((int64_t)l * v.num_seqs + s) * v.heads + h;
  int32_t* kept = p.kept + row * p.budget;
  float* nw = p.new_weights ? p.new_weights + l * p.new_weights_layer + s * p.new_weights_seq + h * p.new_weights_head
                            : nullptr;
  if (threadIdx.x == 0 && h == 0 && l == 0) {
    check_length(v, s);
    p.new_lengths[s] = keep;
  }
  for (int32_t i = keep + threadIdx.x; i < p.budget; i += kSelectThreads) kept[i] = -1;
  if (n <= p.budget) {  // all of them
    for (int32_t i = threadIdx.x; i < n; i += kSelectThreads) {
      kept[i] = i;
      if (nw) nw[i] = w[i];
    }
    return;
  }
  const int32_t last = n - p.recent;
  const bool aligned = ((uintptr_t)w & 15) == 0;

  uint32_t rank[kQuads][4];  // of tokens base + 4 (1024 k + threadIdx.x) + j
  auto load = [&](int32_t base) {
    float x[kQuads][4];
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const int32_t i = base + 4 * (k * kSelectThreads + (int32_t)threadIdx.x);
      if (aligned && i <= n - 4) {
        *reinterpret_cast<float4*>(x[k]) = *reinterpret_cast<const float4*>(w + i);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[k][j] = i < n - j ? w[i + j] : 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const int32_t i = base + 4 * (k * kSelectThreads + (int32_t)threadIdx.x);
#pragma unroll
      for (int j = 0; j < 4; ++j) rank[k][j] = rank_of(x[k][j]);
      if (i < p.sinks || i > last - 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          rank[k][j] = i >= n - j ? kNone : i + j < p.sinks || i >= last - j ? kAlways : rank[k][j];
      }
    }
  };
  load(0);
  int32_t want = keep;
  uint32_t prefix = 0;
  auto digit = [&](auto at, auto bits) {
    constexpr int kAt = decltype(at)::value, kBits = decltype(bits)::value;
    hist[threadIdx.x] = hist[threadIdx.x + kSelectThreads] = 0;
    __syncthreads();
#pragma unroll 1
    for (int32_t base = 0; base < n; base += kTile) {
      if (n > kTile) load(base);
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (kAt + kBits == 32 || rank[k][j] - prefix < 1u << (kAt + kBits) % 32)
            atomicAdd(&hist[rank[k][j] >> kAt & ((1u << kBits) - 1)], 1);
    }
    __syncthreads();
    // the digit of the want'th largest: sums from the top, two bins a thread
    const int32_t top_bin = kBins - 1 - 2 * (int32_t)threadIdx.x, b0 = hist[top_bin], b1 = hist[top_bin - 1];
    const int32_t upto = (int32_t)sum_upto(b0 + b1);
    if (lane == 31) warp_counts[warp] = upto;
    __syncthreads();
    const uint32_t all = warp_counts[lane];
    const int32_t before = upto - b0 - b1 + (int32_t)__shfl_sync(~0u, sum_upto(all) - all, warp);
    const int32_t left = want - before;
    if (left > 0 && left <= b0 + b1) {  // one thread's
      prefix_s = prefix | (uint32_t)(left > b0 ? top_bin - 1 : top_bin) << kAt;
      want_s = left > b0 ? left - b0 : left;
    }
    __syncthreads();
    prefix = prefix_s;
    want = want_s;
  };
  digit(std::integral_constant<int, 21>(), std::integral_constant<int, 11>());
  digit(std::integral_constant<int, 10>(), std::integral_constant<int, 11>());
  digit(std::integral_constant<int, 0>(), std::integral_constant<int, 10>());
  // want: how many tokens of rank `prefix` itself are kept
  int32_t above_all = 0, equal_all = 0;  // of the tiles before
#pragma unroll 1
  for (int32_t base = 0; base < n; base += kTile) {
    if (n > kTile) load(base);
    __syncthreads();
    uint32_t mine[kQuads];  // greater | equal << 16 of the lanes up to this one
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      uint32_t c = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c += rank[k][j] > prefix ? 1u : rank[k][j] == prefix ? 0x10000u : 0u;
      mine[k] = sum_upto(c);
      if (lane == 31) counts[k * kSelectWarps + warp] = mine[k];
      mine[k] -= c;
    }
    __syncthreads();
    {  // sums before over (k, warp), a count each of the first kQuads warps' threads
      const uint32_t c = warp < kQuads ? counts[threadIdx.x] : 0;
      const uint32_t upto = sum_upto(c);
      if (lane == 31) warp_counts[warp] = upto;
      __syncthreads();
      const uint32_t all = warp_counts[lane], sums = sum_upto(all);
      if (warp < kQuads) counts[threadIdx.x] = __shfl_sync(~0u, sums - all, warp) + upto - c;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        const uint32_t before = counts[k * kSelectWarps + warp] + mine[k];
        int32_t a = above_all + (int32_t)(before & 0xFFFFu), e = equal_all + (int32_t)(before >> 16);
        const int32_t i = base + 4 * (k * kSelectThreads + (int32_t)threadIdx.x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool greater = rank[k][j] > prefix, same = rank[k][j] == prefix;
          if (greater || (same && e < want)) {
            const int32_t at = a + min(e, want);
            kept[at] = i + j;
            if (nw) nw[at] = w[i + j];
          }
          a += greater, e += same;
        }
      }
      const uint32_t tile = __shfl_sync(~0u, sums, 31);
      above_all += (int32_t)(tile & 0xFFFFu), equal_all += (int32_t)(tile >> 16);
    }
  }
}

// A warp has 32 kept tokens of one row: their places, old and new, a lane each, then their K and V rows, eight
// vectors of a lane in flight.  Bound by the rows' bytes, read and written once: 512 rows of 4,096 tokens x 2 x 256 bytes
// (2.1 GB) take 328 us, 6.5 TB/s.
constexpr int kGatherThreads = 128;
__global__ void __launch_bounds__(kGatherThreads) gather_kernel(const __grid_constant__ EvictParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * (kGatherThreads / 32) + (threadIdx.x >> 5), row = unit / p.units;
  const int32_t h = (int32_t)(row % v.heads);
  const int32_t sl = (int32_t)(row / v.heads), l = sl / v.num_seqs, s = sl - l * v.num_seqs;
  if (l >= p.num_layers) return;
  const int32_t to = (int32_t)(unit - row * p.units) * 32 + lane;
  const int32_t n = min(length_of(v, s), p.budget);
  if (to - lane >= n) return;
  uint8_t* base = p.layer_base[l] + h * v.head_bytes;
  uint32_t old_row = kNoRow, new_row = kNoRow;
  if (to < n) {
    old_row = row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)p.kept[row * p.budget + to]);
    new_row = row_index(v, p.new_tables + s * p.new_table_stride, p.new_table_len, (uint32_t)to);
  }
  const uint32_t vecs = p.row_vecs.d, all = 32 * 2 * vecs;
  for (uint32_t i0 = lane; i0 < all; i0 += 8 * 32) {
    uint4 x[8];
    uint8_t* dst[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint32_t i = i0 + u * 32, pair = quotient(p.row_vecs, i), vec = i - pair * vecs, half = pair & 1;
      const uint32_t from = __shfl_sync(~0u, old_row, pair >> 1 & 31), into = __shfl_sync(~0u, new_row, pair >> 1 & 31);
      const int64_t off = half * v.half_bytes + vec * 16;
      x[u] = make_uint4(0, 0, 0, 0);
      dst[u] = i < all && into != kNoRow ? base + into * v.row_bytes + off : nullptr;
      if (dst[u] && from != kNoRow) x[u] = __ldcs(reinterpret_cast<const uint4*>(base + from * v.row_bytes + off));
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (dst[u]) __stcs(reinterpret_cast<uint4*>(dst[u]), x[u]);
  }
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, cudaStream_t s) {
  const PagesView& v = p.pages;
  const dim3 rows(v.heads, v.num_seqs, p.num_layers);
  // no more registers than the longest row fills: 128 rows of 2k to 4k weights take 23.5 us with their gather instead of
  // 32 with the largest form, 12k 26.6 instead of 32.4 (and 28.8 with the smallest, which reads them again)
  auto select = v.max_length <= 4 * kSelectThreads    ? select_kernel<1>
                : v.max_length <= 12 * kSelectThreads ? select_kernel<3>
                                                      : select_kernel<8>;
  const cudaError_t e = launch_after(select, rows, kSelectThreads, 0, s, p);
  const int64_t warps = (int64_t)p.num_layers * v.num_seqs * v.heads * p.units;
  const unsigned grid = (unsigned)((warps + kGatherThreads / 32 - 1) / (kGatherThreads / 32));
  return e != cudaSuccess ? e : launch_after(gather_kernel, dim3(grid), kGatherThreads, 0, s, p);
}

}  // namespace kvx

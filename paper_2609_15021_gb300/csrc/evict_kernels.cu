// evict_kernels.cu -- choosing the tokens a cache keeps by their accumulated
// attention weight, and moving their rows into fresh pages.

#include <algorithm>

#include "operators.cuh"

namespace kvx {
namespace {

constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 2048;  // digits of 11, 11 and 10 bits

// Whole numbers in the order of the weights: NaN as -inf, -0 as +0.  None is kNone or kAlways.
constexpr uint32_t kNone = 0, kAlways = UINT32_MAX;
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (isnan(w)) w = -INFINITY;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA per row of weights (head, sequence, layer).  Tokens that are kept whatever their weight have the largest
// rank of all.  The smallest kept weight is found as the m-th largest
// rank, 11 bits at a time, by counting the ranks that share the bits found so far (the first 11 hold the exponent and
// two bits more, which spreads weights over enough counters that a warp's seldom meet); of the tokens that have just
// that rank the first ones are kept.  A token's place among the kept ones is then
//   #(greater before it) + min(#(equal before it), how many equal ones are kept),
// which one scan of pairs of counts gives.  Up to 1024 * kEach weights are read once and stay in registers; longer
// rows are read again, tile by tile, for every count.  Bound by its instructions, some hundred for a warp's 32 weights:
// 512 rows of 18k to 32k weights (51 MB) take 89 us, a CTA an SM; 128 rows of 4k 8 us.
template <int kEach>
__global__ void __launch_bounds__(kSelectThreads, 1) select_kernel(const __grid_constant__ EvictParams p) {
  wait_for_previous();
  const PagesView& v = p.pages;
  constexpr int kTile = kSelectThreads * kEach;
  __shared__ int32_t hist[kBins];
  __shared__ int32_t above[kEach * kSelectWarps], equal[kEach * kSelectWarps];  // counts, then sums before, by (k, warp)
  __shared__ int32_t warp_above[kSelectWarps], warp_equal[kSelectWarps];
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
  int32_t want = keep;
  uint32_t prefix = 0;

  uint32_t rank[kEach];  // of tokens base + k * 1024 + threadIdx.x
  auto load = [&](int32_t base) {
    float x[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int32_t i = base + k * kSelectThreads + threadIdx.x;
      x[k] = i < n ? w[i] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int32_t i = base + k * kSelectThreads + threadIdx.x;
      rank[k] = i >= n ? kNone : i < p.sinks || i >= last ? kAlways : rank_of(x[k]);
    }
  };
  load(0);
  {
#pragma unroll 1
    for (int shift = 21, width = 11; shift >= 0; width = shift < 11 ? shift : 11, shift -= width) {
      hist[threadIdx.x] = hist[threadIdx.x + kSelectThreads] = 0;
      __syncthreads();
#pragma unroll 1
      for (int32_t base = 0; base < n; base += kTile) {
        if (n > kTile) load(base);
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
          // the bits above the digit, shifted in two steps as the first digit has none
          if ((rank[k] ^ prefix) >> shift >> width == 0)
            atomicAdd(&hist[rank[k] >> shift & ((1 << width) - 1)], 1);
        }
      }
      __syncthreads();
      // the digit of the want'th largest: sums from the top, two bins a thread
      const int32_t top_bin = kBins - 1 - 2 * threadIdx.x, b0 = hist[top_bin], b1 = hist[top_bin - 1];
      int32_t upto = b0 + b1;
      for (int d = 1; d < 32; d <<= 1) {
        const int32_t y = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += y;
      }
      if (lane == 31) warp_above[warp] = upto;
      __syncthreads();
      int32_t before = upto - b0 - b1;
      for (int i = 0; i < warp; ++i) before += warp_above[i];
      const int32_t left = want - before;
      if (left > 0 && left <= b0 + b1) {  // one thread's
        prefix_s = prefix | (uint32_t)(left > b0 ? top_bin - 1 : top_bin) << shift;
        want_s = left > b0 ? left - b0 : left;
      }
      __syncthreads();
      prefix = prefix_s;
      want = want_s;
      if (shift == 0) break;
    }
  }
  // want: how many tokens of rank `prefix` itself are kept
  int32_t above_all = 0, equal_all = 0;  // of the tiles before
#pragma unroll 1
  for (int32_t base = 0; base < n; base += kTile) {
    if (n > kTile) load(base);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const uint32_t gt = __ballot_sync(~0u, rank[k] > prefix), eq = __ballot_sync(~0u, rank[k] == prefix);
      if (lane == 0) above[k * kSelectWarps + warp] = __popc(gt), equal[k * kSelectWarps + warp] = __popc(eq);
    }
    __syncthreads();
    {  // exclusive sums over (k, warp): kEach neighbours a thread of the first 32 threads' warps
      constexpr int kCounts = kEach * kSelectWarps;
      int32_t a = 0, e = 0;
      if (threadIdx.x < kCounts) a = above[threadIdx.x], e = equal[threadIdx.x];
      int32_t ua = a, ue = e;
      for (int d = 1; d < 32; d <<= 1) {
        const int32_t y = __shfl_up_sync(~0u, ua, d), z = __shfl_up_sync(~0u, ue, d);
        if (lane >= d) ua += y, ue += z;
      }
      if (lane == 31) warp_above[warp] = ua, warp_equal[warp] = ue;
      __syncthreads();
      int32_t ba = above_all, be = equal_all, ta = 0, te = 0;
      for (int i = 0; i < kCounts / 32; ++i) {
        if (i < warp) ba += warp_above[i], be += warp_equal[i];
        ta += warp_above[i], te += warp_equal[i];
      }
      if (threadIdx.x < kCounts) above[threadIdx.x] = ba + ua - a, equal[threadIdx.x] = be + ue - e;
      above_all += ta, equal_all += te;
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const bool is_gt = rank[k] > prefix, is_eq = rank[k] == prefix;
      const uint32_t gt = __ballot_sync(~0u, is_gt), eq = __ballot_sync(~0u, is_eq), under = (1u << lane) - 1;
      if ((gt | eq) == 0) continue;
      const int32_t i = base + k * kSelectThreads + threadIdx.x;
      const int32_t e = equal[k * kSelectWarps + warp] + __popc(eq & under);
      if (is_gt || (is_eq && e < want)) {
        const int32_t at = above[k * kSelectWarps + warp] + __popc(gt & under) + min(e, want);
        kept[at] = i;
        if (nw) nw[at] = w[i];
      }
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
  // no more registers than the longest row fills: 128 rows of 2k to 4k weights take 24 us with their gather instead of 35
  // with the largest form, 12k 29 instead of 36 (and 32 with the smallest, which reads them again)
  auto select = v.max_length <= 4 * kSelectThreads    ? select_kernel<4>
                : v.max_length <= 12 * kSelectThreads ? select_kernel<12>
                                                      : select_kernel<32>;
  const cudaError_t e = launch_after(select, rows, kSelectThreads, 0, s, p);
  const int64_t warps = (int64_t)p.num_layers * v.num_seqs * v.heads * p.units;
  const unsigned grid = (unsigned)((warps + kGatherThreads / 32 - 1) / (kGatherThreads / 32));
  return e != cudaSuccess ? e : launch_after(gather_kernel, dim3(grid), kGatherThreads, 0, s, p);
}

}  // namespace kvx

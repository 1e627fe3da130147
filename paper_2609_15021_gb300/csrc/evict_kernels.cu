// evict_kernels.cu -- choosing the tokens a cache keeps by their accumulated
// attention weight, and moving their rows into fresh pages.

#include <algorithm>

#include "operators.cuh"

namespace kvx {
namespace {

constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32;
constexpr int kDigitBits = 8, kBins = 1 << kDigitBits;

// Whole numbers in the order of the weights: NaN as -inf, -0 as +0.
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (isnan(w)) w = -INFINITY;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA per row of weights (head, sequence, layer).  The smallest kept weight is found as the m-th largest
// rank, eight bits at a time, by counting the ranks that share the bits found so far; of the tokens that have just
// that rank the first ones are kept.  A token's place among the kept ones is then
//   #(greater before it) + min(#(equal before it), how many equal ones are kept),
// which one scan of pairs of counts gives.  Up to 1024 * kEach weights are read once and stay in registers; longer
// rows are read again, tile by tile, for every count.  Bound by the weights' bytes, and where rows are few by the
// counts' barriers.
template <int kEach>
__global__ void __launch_bounds__(kSelectThreads, kEach > 16 ? 1 : 2) select_kernel(const __grid_constant__ EvictParams p) {
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
  // the middle: tokens that only their weight keeps
  const int32_t first = p.sinks, last = n - p.recent;
  int32_t want = keep - p.sinks - p.recent;    // of the middle
  uint32_t prefix = want > 0 ? 0 : UINT32_MAX;  // no weight's rank is above UINT32_MAX

  uint32_t rank[kEach];  // of tokens base + k * 1024 + threadIdx.x
  auto load = [&](int32_t base) {
    float x[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int32_t i = base + k * kSelectThreads + threadIdx.x;
      x[k] = i >= first && i < last ? w[i] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) rank[k] = rank_of(x[k]);
  };
  load(0);
  if (want > 0) {
#pragma unroll 1
    for (int shift = 32 - kDigitBits; shift >= 0; shift -= kDigitBits) {
      if (threadIdx.x < kBins) hist[threadIdx.x] = 0;
      __syncthreads();
#pragma unroll 1
      for (int32_t base = 0; base < n; base += kTile) {
        if (n > kTile) load(base);
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
          const int32_t i = base + k * kSelectThreads + threadIdx.x;
          // the bits above the digit, shifted in two steps as the first digit has none
          if (i >= first && i < last && (rank[k] ^ prefix) >> shift >> kDigitBits == 0)
            atomicAdd(&hist[rank[k] >> shift & (kBins - 1)], 1);
        }
      }
      __syncthreads();
      if (warp == 0) {  // the digit of the want'th largest: sums from the top, eight bins a lane
        int32_t mine = 0, bins[kBins / 32];
#pragma unroll
        for (int k = 0; k < kBins / 32; ++k) mine += bins[k] = hist[kBins - 1 - (lane * (kBins / 32) + k)];
        int32_t upto = mine;
        for (int d = 1; d < 32; d <<= 1) {
          const int32_t y = __shfl_up_sync(~0u, upto, d);
          if (lane >= d) upto += y;
        }
        int32_t left = want - (upto - mine);
        if (left > 0 && left <= mine) {  // one lane's
          int k = 0;
#pragma unroll
          for (int j = 0; j < kBins / 32 - 1; ++j)
            if (k == j && left > bins[j]) left -= bins[j], ++k;
          prefix_s = prefix | (uint32_t)(kBins - 1 - (lane * (kBins / 32) + k)) << shift;
          want_s = left;
        }
      }
      __syncthreads();
      prefix = prefix_s;
      want = want_s;
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
      const int32_t i = base + k * kSelectThreads + threadIdx.x;
      const bool middle = i >= first && i < last;
      const uint32_t gt = __ballot_sync(~0u, i < n && (!middle || rank[k] > prefix));
      const uint32_t eq = __ballot_sync(~0u, middle && rank[k] == prefix);
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
      const int32_t i = base + k * kSelectThreads + threadIdx.x;
      const bool middle = i >= first && i < last;
      const bool is_gt = i < n && (!middle || rank[k] > prefix), is_eq = middle && rank[k] == prefix;
      const uint32_t gt = __ballot_sync(~0u, is_gt), eq = __ballot_sync(~0u, is_eq), under = (1u << lane) - 1;
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
// vectors of a lane in flight.  Bound by the rows' bytes, read and written once.
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
  if (v.max_length <= 4 * kSelectThreads)
    select_kernel<4><<<rows, kSelectThreads, 0, s>>>(p);
  else if (v.max_length <= 12 * kSelectThreads)
    select_kernel<12><<<rows, kSelectThreads, 0, s>>>(p);
  else
    select_kernel<32><<<rows, kSelectThreads, 0, s>>>(p);
  const int64_t warps = (int64_t)p.num_layers * v.num_seqs * v.heads * p.units;
  const unsigned grid = (unsigned)((warps + kGatherThreads / 32 - 1) / (kGatherThreads / 32));
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : launch_after(gather_kernel, dim3(grid), kGatherThreads, 0, s, p);
}

}  // namespace kvx

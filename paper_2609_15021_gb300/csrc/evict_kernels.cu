// evict_kernels.cu -- choosing the tokens a cache keeps by their accumulated
// attention weight, and moving their rows into fresh pages.

#include "operators.cuh"

namespace kvx {
namespace {

constexpr int kSelectThreads = 512;

// Whole numbers in the order of the weights: NaN as -inf, -0 as +0.
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (isnan(w)) w = -INFINITY;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum of `v` over the CTA's threads before this one; *total over all.
__device__ __forceinline__ int32_t scan_before(int32_t v, int32_t* warp_sums, int32_t* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int32_t x = v;
  for (int d = 1; d < 32; d <<= 1) {
    const int32_t y = __shfl_up_sync(~0u, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  int32_t before = 0, all = 0;
  for (int i = 0; i < kSelectThreads / 32; ++i) {
    if (i < w) before += warp_sums[i];
    all += warp_sums[i];
  }
  *total = all;
  return before + x - v;
}

// One CTA per (head, sequence, layer): the m-th largest weight of the middle
// tokens, eight bits of its rank at a time, then the kept positions in order.
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const __grid_constant__ EvictParams p) {
  const PagesView& v = p.pages;
  __shared__ int32_t hist[256], warp_sums[kSelectThreads / 32];
  __shared__ uint32_t prefix_s;
  __shared__ int32_t want_s;
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
  // the middle: tokens that only their weight keeps
  const int32_t first = n > keep ? min(p.sinks, n) : n, last = n > keep ? n - p.recent : n;
  int32_t want = keep - p.sinks - p.recent;    // of the middle
  uint32_t prefix = want > 0 ? 0 : UINT32_MAX;  // no weight's rank is above UINT32_MAX
  if (first < last && want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 256; i += kSelectThreads) hist[i] = 0;
      __syncthreads();
      for (int32_t i = first + threadIdx.x; i < last; i += kSelectThreads) {
        const uint32_t r = rank_of(w[i]);
        if (shift == 24 || (r >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(r >> shift) & 255], 1);
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        int b = 255;
        int32_t left = want;
        while (b > 0 && hist[b] < left) left -= hist[b--];
        prefix_s = prefix | ((uint32_t)b << shift);
        want_s = left;
      }
      __syncthreads();
      prefix = prefix_s;
      want = want_s;
    }
  }
  // want: how many tokens of rank `prefix` itself are kept, the first ones
  int32_t out = 0, equal = 0;
  for (int32_t base = 0; base < n; base += kSelectThreads) {
    const int32_t i = base + threadIdx.x;
    const bool middle = i >= first && i < last;
    const uint32_t r = middle ? rank_of(w[i]) : 0;
    const bool tie = middle && r == prefix;
    int32_t all;
    const int32_t ties = equal + scan_before(tie, warp_sums, &all);
    equal += all;
    const bool take = i < n && (!middle || r > prefix || (tie && ties < want));
    const int32_t at = out + scan_before(take, warp_sums, &all);
    out += all;
    if (take && at < keep) {
      kept[at] = i;
      if (nw) nw[at] = w[i];
    }
  }
  for (int32_t i = keep + threadIdx.x; i < p.budget; i += kSelectThreads) kept[i] = -1;
}

// A warp per kept row: its K and V from the old place to the new one.
__global__ void __launch_bounds__(256) gather_kernel(const __grid_constant__ EvictParams p, int64_t rows) {
  const PagesView& v = p.pages;
  const int lane = threadIdx.x & 31;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5;
  if (i >= rows) return;
  const int64_t at = i / p.budget;
  const int32_t to = (int32_t)(i - at * p.budget), pos = p.kept[i];
  if (pos < 0) return;
  const int32_t h = (int32_t)(at % v.heads), s = (int32_t)(at / v.heads % v.num_seqs);
  uint8_t* base = p.layer_base[at / v.heads / v.num_seqs];
  const uint32_t old_row = row_index(v, v.tables + s * v.table_stride, v.table_len, (uint32_t)pos);
  const uint32_t new_row = row_index(v, p.new_tables + s * p.new_table_stride, p.new_table_len, (uint32_t)to);
  if (new_row == kNoRow) return;
  const int32_t vecs = (int32_t)(v.row_bytes / 16);
  for (int32_t k = lane; k < 2 * vecs; k += 32) {
    const int64_t off = (k >= vecs ? v.half_bytes + (k - vecs) * 16 : k * 16) + h * v.head_bytes;
    const uint4 x = old_row == kNoRow ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(base + old_row * v.row_bytes + off);
    *reinterpret_cast<uint4*>(base + new_row * v.row_bytes + off) = x;
  }
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, cudaStream_t s) {
  const PagesView& v = p.pages;
  select_kernel<<<dim3(v.heads, v.num_seqs, p.num_layers), kSelectThreads, 0, s>>>(p);
  const int64_t rows = (int64_t)p.num_layers * v.num_seqs * v.heads * p.budget;
  gather_kernel<<<(unsigned)((rows + 7) / 8), 256, 0, s>>>(p, rows);
  return cudaGetLastError();
}

}  // namespace kvx

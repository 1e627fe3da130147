// attend_kernels.cuh -- attention of each sequence's newest tokens over its pages.
//
//   s_j = scale q.k_j (capped, biased),  m = max s_j,  l = sum exp(s_j - m),
//   o = sum exp(s_j - m) v_j / l
//
// One pass over K and V with the running maximum and sum.  Every K/V row is read
// once and meets all rows of queries that share its head (group x new tokens), so
// the kernel is bound by the cache's bytes, and the products are small: they are taken as
// S^T = K Q^T and O^T = V^T P^T, 16 keys (dims) by 8 query rows a matrix
// instruction, so that a group of up to 8 heads wastes nothing.  mma.sync does them at a few
// per cent of its rate; what the kernel is built for is bytes in flight:
//
//   * The work is cut into steps of 16 or 32 keys of one item (sequence, KV head, block
//     of query rows).  The grid's CTAs take equal runs of the steps of all items,
//     whatever the lengths, which are read on the device (an item counts for kItemSteps
//     more than it has, what beginning and ending one takes).  A run that covers only
//     a part of an item leaves its unnormalised sums in the workspace, and a second kernel
//     joins the parts in their order, a CTA per row.  (Joined by the CTA that came last to
//     an item, the same took 11 us instead of 3 at 38 parts of one sequence: few CTAs, in code
//     that is in no instruction cache.)
//   * In a CTA, three or four warps take the steps in turn.  A warp has a ring of its own in shared
//     memory and shares nothing with the others until a piece ends, so there is no
//     barrier in the loop.
//   * The ring is filled by 16-byte asynchronous copies, row by row, wherever the pages
//     lie.  A row's place is a 32-bit number of rows from the layer's start, so that a
//     vector costs a shuffle, a multiply-add and the copy.  (One bulk copy per row and lane
//     was slower: its addresses are uniform, so a warp issues 32 of them in a loop.)  Rows
//     are kept at a pitch of an odd number of vectors, so ldmatrix reads eight of
//     them without bank conflicts.
//   * The maximum that exponents are relative to is raised only when a score passes it
//     by more than 2^5, so a step needs one vote instead of a reduction over the keys.
//
// An e4m3 cache is widened to fp16 between shared memory and the product, exactly;
// the queries then are fp16 too, each row scaled by a power of two, so that no bit of
// a bf16 value is lost within 2^-24 of the row's largest.  Probabilities are rounded to the
// cache's type (fp16 for e4m3) for the product with V; the sums they are divided by are not.  That is 2^-9 of a term, of
// either sign: in bf16 an output is off by some 2.1e-3 where its own rounding gives 1.6e-3, and a second part of each
// probability would take the product twice.  Over selected pages, of which there are few, it does: what rounding takes
// of a probability is a second factor of V in the same type, and an output is off by its own rounding alone (1.6e-3 in bf16,
// where one part gives 1.9e-3 even if sums are those of the rounded probabilities; times are the same within 3 %).
//
// Measured: bf16, sequences of 21k and 32.8k tokens, 8 heads x 128 with 8 query rows each, weights kept (220 MB of
// K/V): 45 us; fp16, 45 sequences of up to 16k tokens, 8 heads x 96 with 2 rows, cap and slopes (270 MB): 60 us; both
// at 63 % of the DRAM's rate, as they wait for their first rows and for the last CTA.  e4m3, four sequences of 99k to 127k
// tokens, 4 heads x 256 with 24 rows (922 MB): 209 us, 4.4 TB/s: 24 x 256 sums are 192 registers a thread, so there
// are two warps a scheduler and little to hide a step's dependent products and conversions behind.
//
// Over selected pages: four sequences of 99k to 127k tokens, 4 heads x 256 in e4m3, four queries of 6 rows a head with 128 pages
// of 32 tokens each (134 MB): 36 us, 3.7 TB/s; one query of 8 x 128 in bf16 over 64 pages of 16 (4 MB): 9.4 us.
#pragma once

#include <algorithm>
#include <type_traits>

#include "attend_common.cuh"

namespace kvx {
namespace {

constexpr int kMaxCtas = 320;  // of a launch
// Exponents are relative to 2^10 below the largest score so far (fp16 probabilities stay
// normal down to 2^-24 of it), and it is raised when a score passes it by more than 2^5.
constexpr float kBelow = 10.f, kSlack = 15.f;

template <class C, int kDim, int kTiles>  // kTiles: of 8 query rows
struct AttendShape {
  static constexpr int kElem = (int)sizeof(typename C::T);
  static constexpr int kRowBytes = kDim * kElem;
  static constexpr int kPitch = kRowBytes + 16;  // an odd number of vectors
  static constexpr int kBlocks = attend_blocks(kDim, kElem, kTiles), kStep = 16 * kBlocks;  // keys of a step
  static constexpr int kHalfBytes = kStep * kPitch;
  static constexpr int kStageBytes = 2 * kHalfBytes;  // K rows, then V rows
  static constexpr int kWarps = kStageBytes > 16 * 1024 && kBlocks == 2 ? 3 : 4, kThreads = 32 * kWarps;
  static constexpr int kVecs = kRowBytes / 16;
  static constexpr int kRowsPerLoad = 32 / kVecs;
  static constexpr int kLoads = kStep / kRowsPerLoad;  // of K, and of V, by a lane
  static constexpr int kRows = 8 * kTiles;
  // the queries as the products' right factor: [32 dims][tile] x 16 bytes a lane, kept in registers where they fit
  static constexpr bool kQueryInRegs = kDim / 16 * kTiles <= 16;
  static constexpr int kQueryBytes = kQueryInRegs ? 0 : kDim / 16 * kTiles * 256;
  // two CTAs an SM, but one where two stages of every ring are more than half its shared memory
  static constexpr int kCtas = 2 * kWarps * kStageBytes + kQueryBytes > 106 * 1024 ? 1 : 2;
  static constexpr int kFit = ((kCtas == 1 ? 212 : 106) * 1024 - kQueryBytes) / (kWarps * kStageBytes);
  static constexpr int kStages = kFit > 6 ? 6 : kFit;
  static constexpr int kRing = kWarps * kStages * kStageBytes;
  // the ring serves to join the warps' sums too: [warp][row][dim], then [warp][row] maxima and sums
  static constexpr int kSumPitch = kDim + 4;
  static constexpr int kJoin = kWarps * kRows * (kSumPitch + 2) * 4;
  static constexpr int kQueryAt = kRing > kJoin ? kRing : kJoin;
  static constexpr int kSmem = kQueryAt + kQueryBytes;
  static constexpr int kPart = kRows * (kDim + 2);  // floats of a part: sums, then maxima and sums
  static_assert(kStages >= 2, "a ring");
};

// Four e4m3 values as two pairs of fp16.
__device__ __forceinline__ void widen4(uint32_t v, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}"
      : "=r"(lo), "=r"(hi) : "r"(v));
}

// 1 - 2 / (1 + e^2y), and below 1/4, where that would cancel, the series to y^9: within 2^-22 of tanh y, and of y, which
// is what counts once the cap has made an exponent of it.
__device__ __forceinline__ float tanh_of(float y) {
  const float z = y * y;
  const float near = y + y * z * (-1.f / 3 + z * (2.f / 15 + z * (-17.f / 315 + z * (62.f / 2835))));
  const float far = 1.f - 2.f * rcp(1.f + ex2(y * (2.f * kLog2e)));
  return fabsf(y) < 0.25f ? near : far;
}

// The maximum over a column's keys (lanes of equal lane % 4).
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(~0u, v, 4));
  v = fmaxf(v, __shfl_xor_sync(~0u, v, 8));
  return fmaxf(v, __shfl_xor_sync(~0u, v, 16));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor_sync(~0u, v, 4);
  v += __shfl_xor_sync(~0u, v, 8);
  return v + __shfl_xor_sync(~0u, v, 16);
}

// Steps of a sequence, from a multiple of 16 keys (*first) that the first key any of its queries sees is not before.
template <int kStep>
__device__ __forceinline__ int32_t steps_of(const AttendParams& p, int32_t length, int32_t* first) {
  const int32_t lo = p.window > 0 ? max(0, length - p.new_tokens + 1 - p.window) : 0;
  *first = lo & ~15;
  return (length - *first + kStep - 1) / kStep;
}

// What a sequence's item counts for in a run.
__device__ __forceinline__ int32_t run_steps(int32_t steps) { return steps > 0 ? steps + kItemSteps : 0; }

// Sum over the CTA of one value a thread, to all.
template <int kWarps>
__device__ __forceinline__ long long cta_sum(long long v, long long* buf) {
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < kWarps; ++i) v += buf[i];
  return v;
}

__device__ __forceinline__ long long quotient(long long a, long long b) {  // 32 bits where they are enough
  return ((a | b) >> 32) == 0 ? (uint32_t)a / (uint32_t)b : a / b;
}

// The steps of a launch, dealt out to its CTAs in runs of equal length, the first `more` longer by one.
struct Runs {
  long long each, more;
  __device__ __forceinline__ Runs(long long total, long long ctas) {
    each = quotient(total, ctas);
    more = total - each * ctas;
  }
  __device__ __forceinline__ long long begin(long long cta) const { return cta * each + min(cta, more); }
  __device__ __forceinline__ int32_t cta_of(long long step) const {
    const long long longer = more * (each + 1);
    return (int32_t)(step < longer ? quotient(step, each + 1) : more + quotient(step - longer, each));
  }
};

// kSelected: of each query's selected pages alone.  A sequence of the launch then is one query (a sequence's last new_tokens
// tokens after one another), its keys are counted over its list of pages, and its own page, where there are keys behind it, is
// the one place where some are left out.
template <class C, int kDim, int kTiles, bool kSelected>
__global__ void __launch_bounds__(AttendShape<C, kDim, kTiles>::kThreads, AttendShape<C, kDim, kTiles>::kCtas)
    attend_kernel(const __grid_constant__ AttendParams p) {
  using S = AttendShape<C, kDim, kTiles>;
  constexpr bool kWide = S::kElem == 1;  // cache to be widened
  constexpr int kKs = kDim / 16, kRows = S::kRows, kBlocks = S::kBlocks, kStep = S::kStep;
  constexpr int kWarps = S::kWarps, kAttendThreads = S::kThreads;
  constexpr uint32_t kAllKeys = kStep == 32 ? ~0u : 0xFFFFu;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long buf[kWarps + 1];
  __shared__ uint32_t masks[kWarps][S::kStages];
  __shared__ int32_t row_pos[kRows];
  __shared__ float row_slope[kRows], row_scale[kRows];
  __shared__ int32_t found;
  wait_for_previous();
  const PagesView& v = p.pages;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int quad = lane >> 2, sub = lane & 3;
  const int32_t rows = p.group * p.new_tokens;
  const int32_t blocks = (rows + kRows - 1) / kRows;  // of query rows
  const int32_t per_seq = v.heads * blocks;           // items
  // Keys up to a query, and what the launch takes as its sequence's length.
  auto keys_upto = [&](int32_t s) {
    const int32_t of = (int32_t)quotient(p.by_query, (uint32_t)s);
    return max(0, length_of(v, of) - (int32_t)p.by_query.d + 1 + (s - of * (int32_t)p.by_query.d));
  };
  auto keys_of = [&](int32_t s) {
    if (!kSelected) return length_of(v, s);
    const int32_t upto = keys_upto(s), block = (int32_t)v.by_block.d;
    return upto > 0 ? min((int32_t)quotient(v.by_block, (uint32_t)(upto - 1)) + 1, p.budget) * block : 0;
  };
  auto check = [&](int32_t s) {
    if (!kSelected)
      check_length(v, s);
    else if (s == (int32_t)(quotient(p.by_query, (uint32_t)s) * p.by_query.d))
      check_length(v, (int32_t)quotient(p.by_query, (uint32_t)s));
  };

  // All steps, and this CTA's run of them.  Up to 32 sequences are added up by every warp for itself.
  const bool few = v.num_seqs <= 32;
  long long total = 0, upto = 0;  // few: steps of this lane's sequence and those before
  if (few) {
    int32_t first;
    if (blockIdx.x == 0 && threadIdx.x < v.num_seqs) check(threadIdx.x);
    upto = lane < v.num_seqs ? (long long)run_steps(steps_of<kStep>(p, keys_of(lane), &first)) * per_seq : 0;
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += y;
    }
    total = __shfl_sync(~0u, upto, 31);
  } else {
    for (int32_t s = threadIdx.x; s < v.num_seqs; s += kAttendThreads) {
      int32_t first;
      if (blockIdx.x == 0) check(s);
      total += run_steps(steps_of<kStep>(p, keys_of(s), &first));
    }
    total = cta_sum<kWarps>(total, buf) * per_seq;
  }
  for (int32_t s = blockIdx.x; s < v.num_seqs; s += gridDim.x) {  // sequences without a key
    if (keys_of(s) > 0) continue;
    for (int32_t i = threadIdx.x; i < v.heads * rows * (v.head_dim / 4); i += kAttendThreads) {
      const int32_t hr = i / (v.head_dim / 4), col = i % (v.head_dim / 4) * 4;
      write_out(p, s, hr / rows, hr % rows, col, make_float4(0.f, 0.f, 0.f, 0.f));
      if (col == 0) write_lse(p, s, hr / rows, hr % rows, 0.f, 0.f);
    }
    for (int32_t i = threadIdx.x; i < per_seq; i += kAttendThreads) p.items[(int64_t)s * per_seq + i] = make_int2(0, 0);
  }
  const int32_t ctas = (int32_t)min((long long)gridDim.x, max(1ll, quotient(total + p.min_steps - 1, p.min_steps)));
  if (blockIdx.x >= ctas || total == 0) return;
  const Runs runs(total, ctas);
  const long long begin = runs.begin(blockIdx.x), end = runs.begin(blockIdx.x + 1);

  // The sequence that `begin` lies in: every thread takes a sequence's steps, 128 at a time.
  int32_t seq = 0;
  long long seq_begin = 0;  // first step of `seq`'s items
  if (few) {
    seq = __ffs(__ballot_sync(~0u, begin < upto)) - 1;
    seq_begin = seq > 0 ? __shfl_sync(~0u, upto, seq - 1) : 0;
  }
  for (int32_t base = 0; base < v.num_seqs && !few; base += kAttendThreads) {
    int32_t first;
    const int32_t s = base + threadIdx.x;
    const long long mine = s < v.num_seqs ? (long long)run_steps(steps_of<kStep>(p, keys_of(s), &first)) * per_seq : 0;
    long long before = mine;  // inclusive scan over the warp
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(~0u, before, d);
      if (lane >= d) before += y;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = before;
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    long long chunk = 0;
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) before += buf[i];
      chunk += buf[i];
    }
    const long long to = seq_begin + before, from = to - mine;
    if (begin >= from && begin < to) {
      found = s;
      buf[kWarps] = from;
    }
    __syncthreads();
    if (found >= 0) {
      seq = found;
      seq_begin = buf[kWarps];
      break;
    }
    seq_begin += chunk;
  }

  uint8_t* ring = smem + warp * S::kStages * S::kStageBytes;
  const uint32_t ring_at = smem_at(ring);
  uint8_t* query_smem = smem + S::kQueryAt;
  // where a lane's matrices begin in a stage (K: keys 0-7 and 8-15 of 16 dims, or of 2 x 16 to widen; V the same,
  // transposed), and its vectors of a row
  const uint32_t at_lane_k = ((lane & 7) + (((lane >> 3) & 1) << 3)) * S::kPitch + (lane >> 4) * 16;
  const uint32_t at_lane_v = S::kHalfBytes + (kWide ? ((lane & 7) + (((lane >> 3) & 1) << 3)) * S::kPitch + (lane >> 4) * 16
                                                    : ((lane & 7) + ((lane >> 4) << 3)) * S::kPitch + ((lane >> 3) & 1) * 16);
  const int vec = lane % S::kVecs, vec_row = lane / S::kVecs;
  const bool vec_used = vec * 16 < v.head_dim * S::kElem;
  const int vec_bytes = vec_used ? 16 : 0;  // of vectors that no row has, none are copied and zeros written
  const uint32_t at_lane_copy = vec_row * S::kPitch + vec * 16;
  const uint32_t row_bytes = (uint32_t)v.head_dim * S::kElem;

  for (long long at = begin; at < end;) {
    // The piece: steps [i0, i1) of one item.
    int32_t first_key, length, steps;
    for (;;) {
      length = keys_of(seq);
      steps = steps_of<kStep>(p, length, &first_key);
      if (at < seq_begin + (long long)run_steps(steps) * per_seq) break;
      seq_begin += (long long)run_steps(steps) * per_seq;
      if (++seq >= v.num_seqs) return;  // lengths that changed under the kernel
    }
    const int32_t item = (int32_t)quotient(at - seq_begin, run_steps(steps));
    const long long item_begin = seq_begin + (long long)item * run_steps(steps) + kItemSteps;  // its first step's place
    const int32_t i0 = (int32_t)max(0ll, at - item_begin), i1 = (int32_t)min((long long)steps, end - item_begin);
    if (i1 <= i0) break;  // the run ends before the item's first step
    const int32_t h = item / blocks, row0 = (item % blocks) * kRows;
    const int32_t here = min(rows - row0, kRows);  // rows of this block
    const int32_t of = kSelected ? (int32_t)quotient(p.by_query, (uint32_t)seq) : seq;
    const int32_t* table = v.tables + of * v.table_stride;
    const int32_t last = kSelected ? keys_upto(seq) - 1 : 0;  // the query's position
    const int32_t* list = kSelected ? p.selected + ((int64_t)seq * v.heads + h) * p.budget : nullptr;

    // The page of the sequence that key `slot` of the list's n'th page is in, or kNoRow where the query does not see it.
    auto selected = [&](uint32_t n, uint32_t slot) -> uint32_t {
      const int32_t page = __ldg(list + n), before = n ? __ldg(list + n - 1) : -1;
      const int32_t own = (int32_t)quotient(v.by_block, (uint32_t)last);
      const bool seen = page > max(before, -1) && (page < own || (page == own && (int32_t)slot <= last - own * (int32_t)v.by_block.d));
      return seen ? (uint32_t)page : kNoRow;
    };
    // Lane r (and, of 16 keys, r + 16) finds key r of a step, in two parts, so that nothing waits for the table: its entry
    // and the place in the block first, the row when it is used.
    auto look = [&](int32_t i) -> uint2 {
      const uint32_t key = first_key + i * kStep + lane % kStep;
      bool there = i < i1 && (int32_t)key < length;
      uint32_t page = quotient(v.by_block, key);
      const uint32_t slot = key - page * v.by_block.d;
      if (kSelected) {
        page = there ? selected(page, slot) : kNoRow;
        there = page != kNoRow;
        page = there ? page : 0;
      }
      const uint32_t block = quotient(v.by_pack, page), in = page - block * v.by_pack.d;
      const uint32_t entry = there && block < v.table_len ? (uint32_t)__ldg(table + block) : kNoRow;
      return make_uint2(entry, there ? in * v.page_rows + slot * v.token_rows : kNoRow);
    };
    auto row_of = [&](uint2 l, int32_t i) -> uint32_t {
      if (l.x < v.entries && l.y != kNoRow) return l.x * (v.by_pack.d * v.page_rows) + l.y;
      if (l.y != kNoRow) {
        const uint32_t key = first_key + i * kStep + lane % kStep;
        uint32_t page = quotient(v.by_block, key);
        if (kSelected) page = selected(page, key - page * v.by_block.d);
        atomicMin(v.err, (long long)quotient(v.by_pack, page));
      }
      return kNoRow;
    };
    const uint8_t* lane_k = v.base + h * v.head_bytes + (vec_used ? vec * 16 : 0);
    const uint8_t* lane_v = lane_k + v.half_bytes;
    auto issue = [&](int32_t i, uint2 l, uint32_t to) {
      if (i < i1) {
        const uint32_t row = row_of(l, i);
        const uint32_t mask = __ballot_sync(~0u, row != kNoRow) & kAllKeys;
        if (lane == 0) masks[warp][to] = mask;
        const uint32_t dst = ring_at + to * S::kStageBytes + at_lane_copy;
        if (mask == kAllKeys) {
          uint32_t rows_at[S::kLoads];  // in front of the copies where a step has many instructions (211 us, 209.5 so)
#pragma unroll
          for (int k = 0; k < S::kLoads; ++k)
            if (kWide) rows_at[k] = __shfl_sync(~0u, row, k * S::kRowsPerLoad + vec_row);
#pragma unroll
          for (int k = 0; k < S::kLoads; ++k) {
            const uint32_t r = kWide ? rows_at[k] : __shfl_sync(~0u, row, k * S::kRowsPerLoad + vec_row);
            copy_async(dst + k * S::kRowsPerLoad * S::kPitch, lane_k + (uint64_t)r * row_bytes, vec_bytes);
            copy_async(dst + k * S::kRowsPerLoad * S::kPitch + S::kHalfBytes, lane_v + (uint64_t)r * row_bytes, vec_bytes);
          }
        } else {  // rows that there are not: zeros, as V of no key meets a probability of 0
#pragma unroll 1
          for (int k = 0; k < S::kLoads; ++k) {
            const uint32_t r = __shfl_sync(~0u, row, k * S::kRowsPerLoad + vec_row);
            const uint64_t off = r != kNoRow ? (uint64_t)r * row_bytes : 0;
            copy_async(dst + k * S::kRowsPerLoad * S::kPitch, lane_k + off, r != kNoRow ? vec_bytes : 0);
            copy_async(dst + k * S::kRowsPerLoad * S::kPitch + S::kHalfBytes, lane_v + off, r != kNoRow ? vec_bytes : 0);
          }
        }
      }
      commit_async();
    };

    uint2 ahead[S::kStages];
#pragma unroll
    for (int k = 0; k < S::kStages; ++k) ahead[k] = look(i0 + warp + k * kWarps);

    // The first rows are under way while long queries are made ready (24 rows x 256: 211 us instead of 217 over 922 MB), and
    // asked for behind short ones, whose loads would wait for the tables (59.5 us instead of 59 over 270 MB).
    auto start = [&]() {
#pragma unroll
      for (int k = 0; k < S::kStages; ++k) issue(i0 + warp + k * kWarps, ahead[k], k);
    };
    if (!S::kQueryInRegs) start();

    // What is known of the rows, and the queries as the products' right factor: row quad of a tile, dims
    // 2 sub, 2 sub + 1 and those 8 further on (4 sub .. 4 sub + 3 where the cache is widened).
    uint32_t qf[S::kQueryInRegs ? kKs : 1][S::kQueryInRegs ? kTiles : 1][2];
    {
      auto wide = [&](uint32_t raw) { return p.type == KVX_TYPE_BF16 ? unpack2<Bf16>(raw) : unpack2<Fp16>(raw); };
#pragma unroll
      for (int tile = 0; tile < kTiles; ++tile) {
        if (!S::kQueryInRegs && tile % kWarps != warp) continue;
        const int32_t r = row0 + tile * 8 + quad;
        const bool there = r < rows;
        const int32_t t = there ? r / p.group : 0, head = h * p.group + (there ? r % p.group : 0);
        const uint8_t* qrow = p.q + ((int64_t)seq * p.new_tokens + t) * p.q_token + head * p.q_head;
        auto load2 = [&](int col) -> uint32_t {  // two raw neighbouring elements
          return there && col < v.head_dim ? *reinterpret_cast<const uint32_t*>(qrow + col * 2) : 0u;
        };
        uint32_t raw[kKs][2];
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
          for (int e = 0; e < 2; ++e) raw[ks][e] = load2(kWide ? ks * 16 + sub * 4 + e * 2 : ks * 16 + sub * 2 + e * 8);
        int shift = 0;
        if constexpr (kWide) {
          float top = 0.f;
#pragma unroll
          for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 f = wide(raw[ks][e]);
              top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
          top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
          top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
          // the largest to [2^10, 2^11): exponents only
          if (top > 0.f && top < INFINITY) shift = max(-100, min(100, 10 - ilogbf(top)));
        }
        const float up = power_of_two(shift);
        if (sub == 0 && (!S::kQueryInRegs || warp == 0)) {
          row_pos[tile * 8 + quad] = !there ? -1 : kSelected ? INT32_MAX : length - p.new_tokens + t;
          row_slope[tile * 8 + quad] = there && p.slopes ? p.slopes[head] * kLog2e : 0.f;
          row_scale[tile * 8 + quad] = p.scale * p.k_scale * kLog2e * power_of_two(-shift);
        }
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
          uint32_t f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 x = wide(raw[ks][e]);
            f[e] = kWide ? pack2<Fp16>(x.x * up, x.y * up) : raw[ks][e];
          }
          if constexpr (S::kQueryInRegs) {
            qf[ks][tile][0] = f[0], qf[ks][tile][1] = f[1];
          } else {
            *reinterpret_cast<uint2*>(query_smem + ((ks / 2 * kTiles + tile) * 32 + lane) * 16 + ks % 2 * 8) = make_uint2(f[0], f[1]);
          }
        }
      }
    }
    __syncthreads();
    if (S::kQueryInRegs) start();
    uint2 next = look(i0 + warp + S::kStages * kWarps);

    float acc[kKs][kTiles][4];
#pragma unroll
    for (int c = 0; c < kKs; ++c)
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[c][t][e] = 0.f;
    // rows 2 sub and 2 sub + 1 of each tile: what exponents are relative to, and the sums over this lane's keys
    float m[kTiles][2], l[kTiles][2], scale2[kTiles][2];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        m[t][j] = -INFINITY, l[t][j] = 0.f;
        scale2[t][j] = kWide ? row_scale[t * 8 + 2 * sub + j] : p.scale * kLog2e;
      }
    const bool plain_scores = p.softcap == 0.f && !p.slopes;
    const float cap2 = p.softcap * kLog2e, to_cap = p.softcap > 0.f ? 1.f / cap2 : 0.f;  // scores are in powers of two
    // keys below `all_from` or from `all_to` on are not seen by every row
    const int32_t all_to = kSelected ? INT32_MAX : length - p.new_tokens + 1, all_from = p.window > 0 ? length - p.window : INT32_MIN;
    float* scores = p.weights ? p.scores + ((int64_t)seq * v.heads + h) * p.score_stride * p.score_rows : nullptr;

    uint32_t stage = 0;
    for (int32_t i = i0 + warp; i < i1; i += kWarps) {
      wait_async<S::kStages - 1>();
      __syncwarp();
      const uint32_t at_k = ring_at + stage * S::kStageBytes + at_lane_k, at_v = ring_at + stage * S::kStageBytes + at_lane_v;
      const uint32_t mask = masks[warp][stage];
      const int32_t key0 = first_key + i * kStep;

      float sc[kBlocks][kTiles][4];
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[n][t][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < kKs; ks += 2) {  // 32 dims
        uint4 q[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          if constexpr (S::kQueryInRegs)
            q[t] = make_uint4(qf[ks][t][0], qf[ks][t][1], qf[ks + 1][t][0], qf[ks + 1][t][1]);
          else
            q[t] = *reinterpret_cast<const uint4*>(query_smem + ((ks / 2 * kTiles + t) * 32 + lane) * 16);
        }
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) {
          uint32_t b[4], a[4];
          if constexpr (!kWide) {
            load_matrices(a, at_k + n * 16 * S::kPitch + ks * 32);
          } else {
            load_matrices(b, at_k + n * 16 * S::kPitch + ks * 16);
            widen4(b[0], a[0], a[2]);
            widen4(b[1], a[1], a[3]);
          }
#pragma unroll
          for (int t = 0; t < kTiles; ++t) mma<C>(sc[n][t], a, q[t].x, q[t].y);
          if constexpr (!kWide) {
            load_matrices(a, at_k + n * 16 * S::kPitch + ks * 32 + 32);
          } else {
            widen4(b[2], a[0], a[2]);
            widen4(b[3], a[1], a[3]);
          }
#pragma unroll
          for (int t = 0; t < kTiles; ++t) mma<C>(sc[n][t], a, q[t].z, q[t].w);
        }
      }

      // Scores in powers of two; element e of block n, tile t: key 16 n + quad + 8 (e / 2), row 8 t + 2 sub + e % 2.
      const bool whole = mask == kAllKeys && key0 + kStep <= all_to && key0 >= all_from;
      uint32_t unseen[kBlocks] = {};  // a bit for every element of every tile
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = sc[n][t][e] * scale2[t][e & 1];
            if (!plain_scores) {
              const int r = t * 8 + 2 * sub + (e & 1);
              if (p.softcap > 0.f) x = cap2 * tanh_of(x * to_cap);
              if (p.slopes) x += row_slope[r] * (key0 + n * 16 + quad + 8 * (e >> 1) - row_pos[r]);
            }
            sc[n][t][e] = x;
          }
      if (!whole) {
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = n * 16 + quad + 8 * (e >> 1), pos = row_pos[t * 8 + 2 * sub + (e & 1)];
              if (!(mask >> k & 1) || key0 + k > pos || (p.window > 0 && key0 + k <= pos - p.window)) {
                sc[n][t][e] = -INFINITY;
                unseen[n] |= 1u << (4 * t + e);
              }
            }
      }
      if (scores) {
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            const int32_t r = row0 + t * 8 + 2 * sub;
            if (r < p.score_rows) {
              float* to = scores + (int64_t)(key0 + n * 16 + quad) * p.score_rows + r;
              *reinterpret_cast<float2*>(to) = make_float2(sc[n][t][0], sc[n][t][1]);
              *reinterpret_cast<float2*>(to + 8 * p.score_rows) = make_float2(sc[n][t][2], sc[n][t][3]);
            }
          }
      }

      auto lane_max = [&](int t, int j) {
        float top = fmaxf(sc[0][t][j], sc[0][t][2 + j]);
#pragma unroll
        for (int n = 1; n < kBlocks; ++n) top = fmaxf(top, fmaxf(sc[n][t][j], sc[n][t][2 + j]));
        return top;
      };
      bool raise = false;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) raise |= lane_max(t, j) > m[t][j] + kSlack;
      if (__any_sync(~0u, raise)) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float top = fmaxf(m[t][j], column_max(lane_max(t, j)) - kBelow);
            const float keep = factor(m[t][j], top);
            m[t][j] = top;
            l[t][j] *= keep;
#pragma unroll
            for (int c = 0; c < kKs; ++c) acc[c][t][j] *= keep, acc[c][t][2 + j] *= keep;
          }
      }
      uint32_t pf[kBlocks][kTiles][2];
      [[maybe_unused]] uint32_t pf_rest[kBlocks][kTiles][2];  // kSelected: what rounding took
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const float ref[2] = {m[t][0] == -INFINITY ? 0.f : m[t][0], m[t][1] == -INFINITY ? 0.f : m[t][1]};
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sc[n][t][e] = ex2(sc[n][t][e] - ref[e & 1]);
            l[t][e & 1] += sc[n][t][e];
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t pair = pack2<C>(sc[n][t][2 * k], sc[n][t][2 * k + 1]);
            if constexpr (kSelected) {
              const float2 x = fma2(unpack2<C>(pair), make_float2(-1.f, -1.f), make_float2(sc[n][t][2 * k], sc[n][t][2 * k + 1]));
              pf_rest[n][t][k] = transpose(pack2<C>(x.x, x.y));
            }
            pf[n][t][k] = transpose(pair);
          }
        }
      }

      // A value that is not finite must not reach the rows that do not see it (0 x inf): where a
      // step is not seen as a whole and holds such a value, its product is done element by element.
      bool odd = false;
      if (!whole) {
        for (int k = lane; k < S::kHalfBytes / 16; k += 32) {
          if (k * 16 % S::kPitch >= row_bytes) continue;
          const uint4 x = *reinterpret_cast<const uint4*>(ring + stage * S::kStageBytes + S::kHalfBytes + k * 16);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          for (int q = 0; q < 4; ++q) {
            if constexpr (kWide) {
              for (int b = 0; b < 32; b += 8) odd |= (w[q] >> b & 0x7F) == 0x7F;
            } else {
              odd |= odd2<C>(w[q]);
            }
          }
        }
        odd = __any_sync(~0u, odd);
      }
      if (!odd) {
        auto add = [&](int n, int c, const uint32_t (&a)[4]) {
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            mma<C>(acc[c][t], a, pf[n][t][0], pf[n][t][1]);
            if constexpr (kSelected) mma<C>(acc[c][t], a, pf_rest[n][t][0], pf_rest[n][t][1]);
          }
        };
#pragma unroll
        for (int c = 0; c < kKs; c += kWide ? 2 : 1) {
#pragma unroll
          for (int n = 0; n < kBlocks; ++n) {
            uint32_t b[4];
            if constexpr (!kWide) {
              load_matrices_t(b, at_v + n * 16 * S::kPitch + c * 32);
              add(n, c, b);
            } else {
              // a transposed pair of bytes is two neighbouring dims of a key: the even ones are the product's
              // first eight rows, the odd ones the others
              load_matrices_t(b, at_v + n * 16 * S::kPitch + c * 16);
#pragma unroll
              for (int q = 0; q < 4; ++q) b[q] = __byte_perm(b[q], 0, 0x3120);
              uint32_t a[4];
              widen4(b[0], a[0], a[1]);
              widen4(b[1], a[2], a[3]);
              add(n, c, a);
              widen4(b[2], a[0], a[1]);
              widen4(b[3], a[2], a[3]);
              add(n, c + 1, a);
            }
          }
        }
      } else {
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll 1
          for (int k = 0; k < 16; ++k) {
            float pk[kTiles][2];
            bool see[kTiles][2];
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const int from = (k & 7) * 4 + sub;
                pk[t][j] = __shfl_sync(~0u, k < 8 ? sc[n][t][j] : sc[n][t][2 + j], from);
                see[t][j] = !(__shfl_sync(~0u, unseen[n], from) >> (4 * t + (k < 8 ? 0 : 2) + j) & 1);
              }
#pragma unroll
            for (int c = 0; c < kKs; ++c)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const int col = c * 16 + (kWide ? quad * 2 + u : quad + 8 * u);
                if (col >= v.head_dim) continue;
                const uint8_t* at_e =
                    ring + stage * S::kStageBytes + S::kHalfBytes + (n * 16 + k) * S::kPitch + col * S::kElem;
                const float x = C::up(*reinterpret_cast<const typename C::T*>(at_e));
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                  for (int j = 0; j < 2; ++j)
                    if (see[t][j]) acc[c][t][2 * u + j] += pk[t][j] * x;
              }
          }
      }
      __syncwarp();
      issue(i + S::kStages * kWarps, next, stage);
      next = look(i + (S::kStages + 1) * kWarps);
      stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }
    wait_async<0>();
    __syncthreads();

    // The warps' sums joined in shared memory, then written: normalised if the piece is the item.
    float* sums = reinterpret_cast<float*>(smem);
    float* stats = sums + kWarps * kRows * S::kSumPitch;  // [warp][row][m, l]
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = t * 8 + 2 * sub + j;
        const float sum = column_sum(l[t][j]);
        if (r >= here) continue;
        if (quad == 0) {
          stats[2 * (warp * kRows + r)] = m[t][j];
          stats[2 * (warp * kRows + r) + 1] = sum;
        }
        float* to = sums + (warp * kRows + r) * S::kSumPitch;
#pragma unroll
        for (int c = 0; c < kKs; ++c) {
          if constexpr (kWide) {
            *reinterpret_cast<float2*>(to + c * 16 + 2 * quad) = make_float2(acc[c][t][j], acc[c][t][2 + j]);
          } else {
            to[c * 16 + quad] = acc[c][t][j];
            to[c * 16 + quad + 8] = acc[c][t][2 + j];
          }
        }
      }
    __syncthreads();
    const bool whole_item = i0 == 0 && i1 == steps;
    if (i0 == 0 && threadIdx.x == 0) {  // where the item's parts are, and how many
      const int32_t parts = whole_item ? 0 : runs.cta_of(item_begin + steps - 1) - (int32_t)blockIdx.x + 1;
      p.items[(int64_t)seq * per_seq + item] = make_int2(blockIdx.x * 2 + (begin < item_begin), parts);
    }
    float* part = p.parts + ((long long)blockIdx.x * 2 + (begin < item_begin)) * S::kPart;
    for (int idx = threadIdx.x; idx < here * (kDim / 4); idx += kAttendThreads) {
      const int r = idx / (kDim / 4), col = idx % (kDim / 4) * 4;
      float top = -INFINITY, sum = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int g = 0; g < kWarps; ++g) top = fmaxf(top, stats[2 * (g * kRows + r)]);
#pragma unroll
      for (int g = 0; g < kWarps; ++g) {
        const float f = factor(stats[2 * (g * kRows + r)], top);
        const float4 x = *reinterpret_cast<const float4*>(sums + (g * kRows + r) * S::kSumPitch + col);
        sum += f * stats[2 * (g * kRows + r) + 1];
        o.x += f * x.x, o.y += f * x.y, o.z += f * x.z, o.w += f * x.w;
      }
      if (whole_item) {
        const float by = sum == 0.f ? 0.f : p.v_scale / sum;
        if (sum == 0.f) o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (col < v.head_dim) write_out(p, seq, h, row0 + r, col, make_float4(o.x * by, o.y * by, o.z * by, o.w * by));
        if (col == 0) write_lse(p, seq, h, row0 + r, top, sum);
      } else {
        __stcg(reinterpret_cast<float4*>(part + r * kDim + col), o);
        if (col == 0) __stcg(reinterpret_cast<float2*>(part + kRows * kDim + 2 * r), make_float2(top, sum));
      }
    }
    __syncthreads();
    at = item_begin + i1;
  }
}

// f(kernel, shape) for every form of the kernel over a cache of type C.
template <class C, bool kSelected, class F>
cudaError_t for_each_attend(F&& f) {
  cudaError_t e;
#define KVX_EACH(kDim, kTiles) \
  if ((e = f(attend_kernel<C, kDim, kTiles, kSelected>, AttendShape<C, kDim, kTiles>())) != cudaSuccess) return e
  KVX_EACH(64, 1);
  KVX_EACH(64, 2);
  KVX_EACH(64, 4);
  KVX_EACH(128, 1);
  KVX_EACH(128, 2);
  KVX_EACH(128, 4);
  KVX_EACH(256, 1);
  KVX_EACH(256, 2);
  KVX_EACH(256, 3);
#undef KVX_EACH
  return cudaSuccess;
}

template <class C, bool kSelected>
cudaError_t prepare() {
  return for_each_attend<C, kSelected>([](auto kernel, auto shape) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, decltype(shape)::kSmem);
  });
}

// The grid: as many CTAs as are resident, or as many runs of min_steps as there may be.
template <class C, bool kSelected, int kDim, int kTiles>
cudaError_t attend(const AttendParams& p, int num_sms, cudaStream_t s) {
  using S = AttendShape<C, kDim, kTiles>;
  const int grid = (int)std::min<int64_t>(std::min(num_sms * S::kCtas, kMaxCtas), (p.most_steps + p.min_steps - 1) / p.min_steps);
  return launch_after(attend_kernel<C, kDim, kTiles, kSelected>, dim3(grid), S::kThreads, S::kSmem, s, p);
}

template <class C, bool kSelected>
cudaError_t attend(const AttendParams& p, int num_sms, cudaStream_t s) {
  const int pad = attend_pad(p.pages.head_dim), tiles = attend_tiles(p.pages.head_dim, p.group * p.new_tokens);
  switch (pad + tiles) {
    case 65: return attend<C, kSelected, 64, 1>(p, num_sms, s);
    case 66: return attend<C, kSelected, 64, 2>(p, num_sms, s);
    case 68: return attend<C, kSelected, 64, 4>(p, num_sms, s);
    case 129: return attend<C, kSelected, 128, 1>(p, num_sms, s);
    case 130: return attend<C, kSelected, 128, 2>(p, num_sms, s);
    case 132: return attend<C, kSelected, 128, 4>(p, num_sms, s);
    case 257: return attend<C, kSelected, 256, 1>(p, num_sms, s);
    case 258: return attend<C, kSelected, 256, 2>(p, num_sms, s);
    default: return attend<C, kSelected, 256, 3>(p, num_sms, s);
  }
}

}  // namespace
}  // namespace kvx

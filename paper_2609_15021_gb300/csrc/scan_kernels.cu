// scan_kernels.cu -- the selective scan of prompts, in matrix form on the tensor cores.
//
// With a_t = A d_t and c_t the sum of a up to t within a chunk of 128 tokens,
//   y_t = sum_{s <= t} (C_t . B_s) e^{c_t - c_s} d_s x_s + e^{c_t} C_t h_in
//   h_out = e^{c_127} h_in + sum_s e^{c_127 - c_s} d_s x_s B_s^T
// so a chunk is four products of 128 x 128 matrices:
//   G = C B^T,  Y2 = C h_in^T,  Y1 = M X with M = G decayed and masked,  S = B^T W with W = x weighted.
// A CTA has a slice of one head's state (64 or 128 of head_dim) in its threads' registers, as H[state_dim][head_dim] in
// fp32 laid out as S is in tensor memory, and walks the chunks of a segment.  G, Y1, Y2 and S are all of tensor
// memory; M takes the place of G as the product's left factor, so it never passes through shared memory.  The products take
// a quarter of the time that the threads take for the elements between them (an exponential each for G, the splits of W,
// the rounding of H), so there is one CTA an SM with eight warps for them, two for every 32 lanes of tensor memory, and a
// ninth that issues the products and makes the next chunk's weights; Y2 and S are made while the threads are at M, and S
// is read while Y1 is made.  A product with both factors in shared memory is bound by reading them (64 cycles for 16
// of k).  The next chunk's rows (96 KB an SM, some 2000 cycles) come in from the chunk's beginning on, into one buffer
// more and those that a product has done with.
//
// 24k tokens of 16 heads of 128 x 128 in fp16 take 253 us: 61 for the segments' states, 12 for carrying them, 185 for
// the last pass, where a chunk takes some 12,900 cycles: the products 2,600, shared memory 5,400 (what the copies,
// the splits, the products' factors, the state and y write and read of it at 128 bytes a cycle), the threads'
// instructions 4,500; the rest is waiting from one to the next.  15 us of it are the scaling of M's rows, 5 the sums of
// exponents in two parts (in 64-bit floats they took 30).  When it took 230 without them, neither 16 warps (277), nor decays
// taken apart by blocks of 32 tokens, with an eighth of the exponentials (231), nor warps of their own that move y
// (241) made it faster.  2,048 tokens in bf16 take 34.4 us: two chunks a CTA, and three launches.
//
// Rounding: M and the carried state are rounded to the inputs' type for the product that makes y, one rounding
// a term, as y is rounded to that type anyway.  The state itself is kept in fp32: W is split into three bf16 or two fp16
// numbers, whose sum is the weighted x to 22 bits or more, and all are multiplied with B (two bf16 parts, 16 bits, left
// the state off by 2.5e-6 where the recurrence in fp32 is by 5e-7).  In fp16 the state, W and every row of M are scaled by
// powers of two into its range, so that small or large B, C and steps cost no bits.
//
// A long sequence is cut into segments, so that every SM has some: a first pass makes each segment's state from
// nothing (from its last chunk to its first, so that weights need no later decay), a second one carries the states
// through the segments, and the last one starts every segment with its own.

#include <algorithm>

#include "state_common.cuh"
#include "tcgen05.cuh"

namespace kvx {
namespace {

constexpr int kChunk = 128, kThreads = 256, kWarps = kThreads / 32;  // of the elements
// And a group of four warps more, of which one issues.  A thread has 168 registers at the launch, and these four warps
// give up what the eight take (256 * 216 + 128 * 72 = 384 * 168), as spills are dear where shared memory leaves the L1
// cache little: with one warp more and 168 registers for all, 24k tokens of fp16 took 242 us where this took 230.
constexpr int kAllThreads = kThreads + 128, kLaunchRegs = 168, kRegs = 216, kIssuerRegs = 72;
static_assert(kThreads * kRegs + 128 * kIssuerRegs <= kAllThreads * kLaunchRegs, "registers of a CTA");

// Columns of tensor memory.
constexpr uint32_t kG = 0, kY1 = 128, kY2 = 256, kState = 384, kColumns = 512;

constexpr float kMost = 1024.f;  // of a token's exponent

// What a chunk's tokens weigh.
struct Weights {
  float sum[kChunk];     // exponents up to a token, rounded
  union {
    float weight[kChunk];     // d times the decay behind it
    uint8_t top[2][kChunk];   // fp16, once W is made: the exponents of M's largest elements, a row's halves
  };
  float d[kChunk];       // d over 2^low
  __half low[kChunk];    // what the sum lost
  float exponent;        // of the whole chunk
  int shift;             // fp16: the power of two that makes the largest weight less than 1
};

struct Shared {
  Weights weights;
  float largest[2][kWarps];
  int32_t buf[kAllThreads / 32 + 3];
  uint32_t tmem;
  uint64_t bars[5];
};

template <int kP>
struct ScanShape {
  static constexpr int kRows = 2 * kPanel;         // B or C: 128 tokens of up to 128 elements
  static constexpr int kSlice = kP / 64 * kPanel;  // x, its two weighted parts, the rounded state
  // three buffers for B and C of this chunk and the next, three for x and its parts, the state's (the first pass: two
  // for B, four for x and its parts), and one for the third part in bf16: where slices are as large as rows the third of
  // the first ones
  static constexpr int kB = 0, kX = 3 * kRows, kRest = kP == 64 ? kX + 4 * kSlice : kB + 2 * kRows;
  static constexpr int kShared = kX + (kP == 64 ? 5 : 4) * kSlice;
  static constexpr int kSmem = kShared + 2048 + 1024;  // 1024: what aligns the panels to their swizzle
  static_assert(sizeof(Shared) <= 2048 && kSmem <= 232448, "shared memory of an SM");
};

__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 at2(const float* p) { return make_float2(p[0], p[1]); }
__device__ __forceinline__ void put2(float* p, float2 v) { p[0] = v.x, p[1] = v.y; }

// A barrier of the eight warps.
__device__ __forceinline__ void sync_eight() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
// The largest value over their threads.
__device__ __forceinline__ float cta_max(float v, float* buf) {
  for (int m = 16; m; m >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, m));
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  sync_eight();
  v = buf[0];
  for (int i = 1; i < kWarps; ++i) v = fmaxf(v, buf[i]);
  return v;
}
// A barrier of the two warps that have the same lanes of tensor memory.
__device__ __forceinline__ void sync_sides(int lanes) { asm volatile("bar.sync %0, 64;" ::"r"(2 + lanes) : "memory"); }
// A power of two that takes values up to `top` below 2^11.
__device__ __forceinline__ int range_of(float top) {
  return top > 0.f && top < INFINITY ? max(-60, min(60, 10 - ilogbf(top))) : 0;
}

template <class E, int N, int kP, bool kStateOnly>
__global__ void __launch_bounds__(kAllThreads, 1) chunk_kernel(const __grid_constant__ ScanParams p) {
  using S = ScanShape<kP>;
  using T = typename E::T;
  constexpr bool kHalf = std::is_same<E, Fp16>::value;
  constexpr int kCols = kP / 2;  // columns of x, Y and H that a thread has
  constexpr bool kAdds = kStateOnly && !kHalf;  // S adds up over the chunks in tensor memory
  constexpr bool kThree = !kHalf;               // parts of W
  constexpr bool kSpare = kStateOnly || !kThree || kP == 64;  // a buffer of rows more than a chunk takes
  // The last pass's predecessor is the carrying of the states: it waits for that before it reads them.
  const bool carried = !kStateOnly && p.segment_states;
  if (!carried) wait_for_previous();
  extern __shared__ __align__(16) uint8_t raw_smem[];
  uint8_t* smem = raw_smem + (-smem_at(raw_smem) & 1023);
  Shared& sh = *reinterpret_cast<Shared*>(smem + S::kShared);
  Weights& w = sh.weights;
  const StateView& v = p.state;
  const int lane = threadIdx.x & 31, warp = __shfl_sync(~0u, threadIdx.x >> 5, 0);
  const int line = (warp & 3) * 32 + lane;  // of tensor memory: a token of G and Y, an element of state_dim of H
  const int side = warp >> 2;               // which half of the columns
  const int32_t slices = p.head_dim / kP, piece = blockIdx.x / slices, p0 = (blockIdx.x - piece * slices) * kP;
  const int32_t h = blockIdx.y, group = h / p.heads_per_group;
  Piece found;
  if (!find_piece<kAllThreads>(v, piece, p.segment, p.by_token, sh.buf, &found)) {
    if (carried) wait_for_previous();  // no kernel may end before the one before it
    return;
  }
  const int32_t seg = found.at, segs = found.of;
  if (kStateOnly && seg + 1 == segs) return;  // the last segment's state is nobody's start
  const int64_t begin = found.first + (int64_t)seg * p.segment, end = min(found.last, begin + p.segment);
  const uint8_t* in = found.in;
  uint8_t* keep = found.keep;
  if (!in || !keep) {
    if (carried) wait_for_previous();
    if (!kStateOnly)
      for (int64_t i = threadIdx.x; i < (end - begin) * (kP / 2); i += kAllThreads)
        *reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(p.out) + (begin + i / (kP / 2)) * p.out_token + h * p.out_head + p0 +
                                     i % (kP / 2) * 2) = 0;
    return;
  }
  const T* b_at = reinterpret_cast<const T*>(p.b) + group * p.b_group;
  const T* c_at = reinterpret_cast<const T*>(p.c) + group * p.c_group;
  const T* x_at = reinterpret_cast<const T*>(p.x) + h * p.x_head + p0;
  const T* dt_at = reinterpret_cast<const T*>(p.dt) + h;
  const uint32_t base = smem_at(smem), bar_g = smem_at(&sh.bars[0]), bar_y2 = smem_at(&sh.bars[1]),
                 bar_s = smem_at(&sh.bars[2]), bar_y1 = smem_at(&sh.bars[3]), bar_end = smem_at(&sh.bars[4]);
  constexpr uint32_t kLast = S::kX + 3 * S::kSlice;  // the rounded state's, or, in the first pass, x's fourth buffer
  uint32_t b_to = S::kB, c_to = S::kB + S::kRows, spare_to = kStateOnly ? c_to : S::kB + 2 * S::kRows;
  uint32_t x_to = S::kX, hi_to = S::kX + S::kSlice, lo_to = S::kX + 2 * S::kSlice, next_to = kLast;

  // Rows of a chunk, swizzled; those behind the last are zeros.  A thread has one column of vectors of rows that are a
  // multiple of 8 apart, so its place within a row stays.
  auto fetch = [&](const T* src, int64_t stride, int64_t t0, uint32_t to, auto vecs) {
    constexpr int kVecs = decltype(vecs)::value, kApart = kThreads / kVecs;
    const int r0 = threadIdx.x / kVecs, c = threadIdx.x % kVecs;
    const int left = (int)min((int64_t)kChunk, end - t0) - r0;
    const T* from = src + (t0 + r0) * stride + c * 8;
    const uint32_t dst = base + to + panel_at(r0, c);
#pragma unroll
    for (int k = 0; k < kChunk / kApart; ++k, from += kApart * stride) {
      const bool there = k * kApart < left;
      copy_async(dst + k * kApart * 128, there ? from : src + begin * stride, there ? 16 : 0);
    }
  };
  const std::integral_constant<int, N / 8> state_vecs;
  const std::integral_constant<int, kP / 8> slice_vecs;
  // ---- set-up: barriers, tensor memory, the first chunk's rows and weights
  const int64_t chunks = (end - begin + kChunk - 1) / kChunk;
  const int64_t step = kStateOnly ? -kChunk : kChunk;
  int64_t t0 = kStateOnly ? begin + (chunks - 1) * kChunk : begin;
  float exponent = 0.f;  // of the decay over the segment's chunks so far
  auto turn = [&]() {    // the buffers' roles in the next chunk
    const uint32_t b_was = b_to, x_was = x_to;
    if (kStateOnly) {
      b_to = spare_to, spare_to = b_was, x_to = next_to, next_to = x_was;
    } else {
      if (kSpare) b_to = c_to, c_to = spare_to, spare_to = b_was;
      x_to = lo_to, lo_to = hi_to, hi_to = x_was;
    }
  };
  if (warp >= kWarps) {
    give_registers<kIssuerRegs>();
    if (warp > kWarps) return;
    // A chunk's weights, by one warp, four tokens a lane.  Sums behind a token are taken from the end, so that they
    // are exact where their weight is not small; `after`: the exponent of what follows the chunk.  Sums up to a token
    // are of any size, and their differences count: they are taken in two parts, whole 64ths, which 128 tokens of up to 2^10
    // (a decay of 2^-1024 is as good as nothing) lose no bit of, and what is left, and kept as a rounded sum and what that
    // lost, which goes into the factors of a column (d) and of a row of M.
    const float A2 = p.A[h] * kLog2e;
    float d[4];
    auto load_steps = [&](int64_t t0) {
      T raw[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) raw[k] = t0 + 4 * lane + k < end ? dt_at[(t0 + 4 * lane + k) * p.dt_token] : E::down(0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) d[k] = t0 + 4 * lane + k < end ? step_of(p, E::up(raw[k]), h) : 0.f;
    };
    auto weigh = [&](float after) {
      float a[4], rest[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        a[k] = d[k] * A2;
        a[k] = a[k] < -kMost ? -kMost : a[k] > kMost ? kMost : a[k];
        rest[k] = a[k] - rintf(a[k] * 64.f) * (1.f / 64);
      }
      float upto = ((a[0] - rest[0]) + (a[1] - rest[1])) + ((a[2] - rest[2]) + (a[3] - rest[3]));
      float fine = (rest[0] + rest[1]) + (rest[2] + rest[3]);
      float behind = (a[0] + a[1]) + (a[2] + a[3]);
      for (int m = 1; m < 32; m <<= 1) {
        const float y = __shfl_up_sync(~0u, upto, m), f = __shfl_up_sync(~0u, fine, m), z = __shfl_down_sync(~0u, behind, m);
        if (lane >= m) upto += y, fine += f;
        if (lane + m < 32) behind += z;
      }
      float below = __shfl_up_sync(~0u, upto, 1), below_fine = __shfl_up_sync(~0u, fine, 1), above = __shfl_down_sync(~0u, behind, 1);
      if (lane == 0) below = below_fine = 0.f;
      if (lane == 31) above = 0.f, w.exponent = upto + fine;
      above += after;
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        below += a[k] - rest[k], below_fine += rest[k];
        // the sum of both, rounded, and what that lost (Knuth, "The Art of Computer Programming", vol. 2, 4.2.2)
        const float sum = below + below_fine, back = sum - below, low = (below - (sum - back)) + (below_fine - back);
        w.sum[4 * lane + k] = sum;
        w.low[4 * lane + k] = __float2half_rn(low);
        w.d[4 * lane + k] = d[k] * ex2(-low);
      }
#pragma unroll
      for (int k = 3; k >= 0; --k) {
        const float weight = d[k] * ex2(above);
        w.weight[4 * lane + k] = weight;
        above += a[k];
        top = fmaxf(top, fabsf(weight));
      }
      if (kHalf) {
        for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, m));
        if (lane == 0) w.shift = top > 0.f && top < INFINITY ? max(-60, min(60, -1 - ilogbf(top))) : 0;
      }
    };

    if (chunks > 0) load_steps(t0);
    tmem_alloc(smem_at(&sh.tmem), kColumns);
    if (lane == 0) {
      for (uint64_t& bar : sh.bars) bar_init(smem_at(&bar));
      fence_operands();
    }
    if (chunks > 0) weigh(0.f);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = sh.tmem;
    for (int64_t n = 0; n < chunks; ++n, t0 += step) {
      const bool more = n + 1 < chunks;
      tmem_before_sync();
      if (__syncthreads_or(0)) break;
      tmem_after_sync();
      exponent += w.exponent;
      if (!kStateOnly && elected()) {
#pragma unroll
        for (int k = 0; k < N / 16; ++k)
          matrix_product(tmem + kG, operand_k(base + c_to, k), operand_k(base + b_to, k), instruction<E>(false, false, 128), k > 0);
        products_done(bar_g);
      }
      __syncwarp();
      if (more) load_steps(t0 + step);
      __syncthreads_or(0);  // W is there, and G read
      tmem_after_sync();
      if (elected()) {
        if (!kStateOnly) {
#pragma unroll
          for (int k = 0; k < N / 16; ++k)
            matrix_product(tmem + kY2, operand_k(base + c_to, k), operand_rows(base + kLast, k), instruction<E>(false, true, kP), k > 0);
          products_done(bar_y2);
        }
#pragma unroll
        for (int k = 0; k < kChunk / 16; ++k) {
          const bool add = k > 0 || (kAdds && n > 0);
          if (kThree)
            matrix_product(tmem + kState, operand_rows(base + b_to, k), operand_rows(base + S::kRest, k),
                           instruction<E>(true, true, kP), add);
          matrix_product(tmem + kState, operand_rows(base + b_to, k), operand_rows(base + lo_to, k),
                         instruction<E>(true, true, kP), kThree || add);
          matrix_product(tmem + kState, operand_rows(base + b_to, k), operand_rows(base + hi_to, k),
                         instruction<E>(true, true, kP), true);
        }
        if (!p.stall || n > 0) products_done(bar_s);
      }
      if (!kStateOnly) {
        __syncthreads();  // M, and x as the product takes it
        tmem_after_sync();
        if (elected()) {
#pragma unroll
          for (int k = 0; k < kChunk / 16; ++k)
            matrix_product_t(tmem + kY1, tmem + kG + k * 8, operand_rows(base + x_to, k), instruction<E>(false, true, kP), k > 0);
          products_done(bar_y1);
        }
      }
      __syncwarp();
      if (more) weigh(kStateOnly ? exponent : 0.f);  // the others have read this chunk's
      turn();
    }
    tmem_before_sync();
    if (__syncthreads_or(0)) {  // a wait ran out, and products may still be at work
      if (elected()) products_done(bar_end);
      __syncwarp();
      bar_wait(bar_end, 0, kDefaultWaitCycles);
      __syncthreads();
    }
    tmem_after_sync();
    tmem_free(tmem, kColumns);
    return;
  }
  take_registers<kRegs>();
  const float D = p.D ? p.D[h] : 0.f;
  const int64_t all = (int64_t)p.heads * p.head_dim * N;
  const int64_t state_at = ((int64_t)h * p.head_dim + p0 + side * kCols) * N + line;  // + column * N
  float state[kCols];
#pragma unroll
  for (int k = 0; k < kCols; ++k) state[k] = 0.f;
  if (chunks > 0) {
    fetch(b_at, p.b_token, t0, b_to, state_vecs);
    fetch(x_at, p.x_token, t0, x_to, slice_vecs);
    if (!kStateOnly) fetch(c_at, p.c_token, t0, c_to, state_vecs);
  }
  commit_async();
  if (!kStateOnly) {
    if (carried) wait_for_previous();
    const float* from = p.segment_states ? p.segment_states + piece * all : reinterpret_cast<const float*>(in);
    if (line < N && (p.segment_states || !found.fresh)) {
#pragma unroll
      for (int k = 0; k < kCols; ++k) state[k] = from[state_at + k * N];
    }
  }
  if (N == 64)  // S's lanes beyond state_dim: their rows of B^T are zeros
    for (int i = threadIdx.x; i < (kSpare && !kStateOnly ? 3 : 2) * kPanel / 16; i += kThreads)
      *reinterpret_cast<uint4*>(smem + S::kB + (i / (kPanel / 16) * 2 + 1) * kPanel + i % (kPanel / 16) * 16) =
          make_uint4(0, 0, 0, 0);
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  const uint32_t tmem = sh.tmem, my_lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
  bool dead = false;  // a wait ran out: the others are not waited for

  // The state a segment starts from, and the one after every chunk, rounded to shared memory as Y2's right factor.
  float state_scale = 1.f;  // fp16: what undoes the rounded state's scaling
  auto round_state = [&](const float (&state)[kCols]) {
    float scale = 1.f;
    if constexpr (kHalf) {
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < kCols; ++k) top = fmaxf(top, fabsf(state[k]));
      const int e = range_of(cta_max(top, sh.largest[0]));
      scale = power_of_two(e), state_scale = power_of_two(-e);
    }
    if (line < N) {
#pragma unroll
      for (int k = 0; k < kCols; k += 8) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 v = kHalf ? mul2(at2(state + k + 2 * j), twice(scale)) : at2(state + k + 2 * j);
          w[j] = pack2<E>(v.x, v.y);
        }
        *reinterpret_cast<uint4*>(smem + kLast + panel_at(line, (side * kCols + k) / 8)) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    fence_operands();
  };
  if (!kStateOnly && chunks > 0) round_state(state);

  for (int64_t n = 0; n < chunks; ++n, t0 += step) {
    const bool more = n + 1 < chunks;
    const uint32_t parity = n & 1;
    wait_async<0>();
    fence_operands();
    tmem_before_sync();
    if (__syncthreads_or(dead)) break;  // the chunk's rows, its weights and the rounded state are there
    tmem_after_sync();
    const float chunk_exponent = w.exponent;
    exponent += chunk_exponent;
    if (more && kSpare) {
      fetch(kStateOnly ? b_at : c_at, kStateOnly ? p.b_token : p.c_token, t0 + step, spare_to, state_vecs);
      if (kStateOnly) fetch(x_at, p.x_token, t0 + step, next_to, slice_vecs);
    }

    // x weighted, in its parts, vector by vector where it lies
    bool odd;
    float back = 1.f;  // fp16: what undoes the scaling of W
    {
      constexpr int kVecs = kChunk * kP / 8 / kThreads;
      uint4 x[kVecs];
      uint32_t carries = 0;
      float scale = 1.f;
      __half2 top = __floats2half2_rn(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        x[k] = *reinterpret_cast<const uint4*>(smem + x_to + (k * kThreads + threadIdx.x) * 16);
        const uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          carries |= odd_carry<E>(u[j]);
          if constexpr (kHalf) top = __hmax2(top, __habs2(*reinterpret_cast<const __half2*>(&u[j])));
        }
      }
      odd = odd_carried(carries);
      if constexpr (kHalf) {
        const int e = range_of(cta_max(fmaxf(__low2float(top), __high2float(top)), sh.largest[1]));
        scale = power_of_two(e + w.shift), back = power_of_two(-e - w.shift);
      }
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const int i = k * kThreads + threadIdx.x, row = i / 8 % kChunk;
        const uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
        const float weight = w.weight[row] * scale;
        uint32_t hi[4], lo[4], rest[4] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float2 f = mul2(unpack2<E>(u[j]), twice(weight));
          hi[j] = pack2<E>(f.x, f.y);
          f = fma2(unpack2<E>(hi[j]), twice(-1.f), f);
          lo[j] = pack2<E>(f.x, f.y);
          if constexpr (kThree) {
            f = fma2(unpack2<E>(lo[j]), twice(-1.f), f);
            rest[j] = pack2<E>(f.x, f.y);
          }
        }
        if (odd) {  // inf - inf: an infinite x has no other part
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t fine = (odd2<E>(hi[j] & 0xFFFFu) ? 0 : 0xFFFFu) | (odd2<E>(hi[j] & 0xFFFF0000u) ? 0 : 0xFFFF0000u);
            lo[j] &= fine, rest[j] &= fine;
          }
        }
        if constexpr (kThree)
          *reinterpret_cast<uint4*>(smem + S::kRest + i * 16) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
        *reinterpret_cast<uint4*>(smem + hi_to + i * 16) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(smem + lo_to + i * 16) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
    }
    fence_operands();

    float y[kCols];
    // G's columns, 16 of every 32 a side: read by all before M takes their place
    float g[4][16];
    float row_factor = 1.f;  // of M's row
    if constexpr (!kStateOnly) {
      dead = dead || !bar_wait(bar_g, parity, p.wait_cycles);
      tmem_after_sync();
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_load16(g[q], my_lanes + kG + q * 32 + side * 16);
      tmem_wait_loads();
      tmem_before_sync();
    }
    odd = __syncthreads_or(odd);  // W is there, and G read
    tmem_after_sync();
    if constexpr (!kStateOnly) {
      const float sum_t = w.sum[line];
      row_factor = ex2(__half2float(w.low[line]));
      const float by = ex2(sum_t) * row_factor * state_scale;
      auto weighed = [&](int q, int j) {  // elements 2 j and 2 j + 1 of G's q'th columns as M's
        const int u = q * 32 + side * 16 + 2 * j;
        const float2 su = *reinterpret_cast<const float2*>(&w.sum[u]), du = *reinterpret_cast<const float2*>(&w.d[u]);
        const float2 e = fma2(su, twice(-1.f), twice(sum_t));
        const float2 by = mul2(make_float2(ex2(e.x), ex2(e.y)), du), all = mul2(make_float2(g[q][2 * j], g[q][2 * j + 1]), by);
        return make_float2(u <= line ? all.x : 0.f, u + 1 <= line ? all.y : 0.f);
      };
      auto seen = [&](int q) { return q * 32 + side * 16 <= (warp & 3) * 32 + 31; };  // some of the warp's tokens see some of these
      float scale = 1.f;
      if constexpr (kHalf) {  // a row's largest element to [2^14, 2^15)
        float top = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (!seen(q)) continue;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 v = weighed(q, j);
            put2(g[q] + 2 * j, v);
            top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
          }
        }
        w.top[side][line] = (uint8_t)(__float_as_uint(top) >> 23);
        sync_sides(warp & 3);
        const int e = max(w.top[0][line], w.top[1][line]);
        const int shift = e == 255 ? 0 : min(100, 14 + 127 - e);
        scale = power_of_two(shift), row_factor *= power_of_two(-shift);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c0 = q * 32 + side * 16;
        uint32_t m[8];
        if (seen(q)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 v = kHalf ? mul2(at2(g[q] + 2 * j), twice(scale)) : weighed(q, j);
            m[j] = pack2<E>(v.x, v.y);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) m[j] = 0;
        }
        tmem_store8(my_lanes + kG + c0 / 2, m);
      }
      tmem_wait_stores();
      if (odd) {  // a token's x that is not finite must not reach the tokens before it (0 x inf): added below
        for (int i = threadIdx.x; i < S::kSlice / 4; i += kThreads) {
          uint32_t* at = reinterpret_cast<uint32_t*>(smem + x_to) + i;
          if (odd2<E>(*at & 0xFFFFu)) *at &= 0xFFFF0000u;
          if (odd2<E>(*at & 0xFFFF0000u)) *at &= 0xFFFFu;
        }
        fence_operands();
      }
      tmem_before_sync();
      __syncthreads();  // M, and x as the product takes it
      tmem_after_sync();
      // Y2 decayed, and the tokens' own x
      dead = dead || !bar_wait(bar_y2, parity, p.wait_cycles);
      tmem_after_sync();
      if (more) fetch(kSpare ? b_at : c_at, kSpare ? p.b_token : p.c_token, t0 + step, c_to, state_vecs);
#pragma unroll
      for (int k = 0; k < kCols; k += 16) {
        float r[16];
        tmem_load16(r, my_lanes + kY2 + side * kCols + k);
        tmem_wait_loads();
#pragma unroll
        for (int j = 0; j < 16; j += 2) put2(y + k + j, mul2(at2(r + j), twice(by)));
      }
      if (p.D) {
#pragma unroll
        for (int k = 0; k < kCols; k += 8) {
          const uint4 x = *reinterpret_cast<const uint4*>(smem + x_to + panel_at(line, (side * kCols + k) / 8));
          const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            put2(y + k + 2 * j, fma2(unpack2<E>(u[j]), twice(D), at2(y + k + 2 * j)));
          }
        }
      }
    }
    // The state after the chunk.
    dead = dead || !bar_wait(bar_s, parity, p.wait_cycles);
    tmem_after_sync();
    if (!kStateOnly && more) {
      if (!kSpare) fetch(b_at, p.b_token, t0 + step, b_to, state_vecs);
      fetch(x_at, p.x_token, t0 + step, lo_to, slice_vecs);
    }
    commit_async();
    if (!kAdds || !more) {
      const float decay = kStateOnly ? 1.f : ex2(chunk_exponent);
#pragma unroll
      for (int k = 0; k < kCols; k += 16) {
        float r[16];
        tmem_load16(r, my_lanes + kState + side * kCols + k);
        tmem_wait_loads();
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const float2 before = at2(state + k + j), made = at2(r + j);
          put2(state + k + j, kHalf ? fma2(made, twice(back), mul2(before, twice(decay))) : fma2(before, twice(decay), made));
        }
      }
      if (!kStateOnly && more) round_state(state);
    }
    if constexpr (!kStateOnly) {
      dead = dead || !bar_wait(bar_y1, parity, p.wait_cycles);
      tmem_after_sync();
    }
    if constexpr (!kStateOnly) {
#pragma unroll
      for (int k = 0; k < kCols; k += 16) {
        float r[16];
        tmem_load16(r, my_lanes + kY1 + side * kCols + k);
        tmem_wait_loads();
#pragma unroll
        for (int j = 0; j < 16; j += 2) put2(y + k + j, fma2(at2(r + j), twice(row_factor), at2(y + k + j)));
      }
      if (odd) {
        for (int u = 0; u < kChunk && t0 + u < end; ++u) {  // whatever the row's scaling: M's sign decides
          uint32_t m;
          tmem_load1(m, my_lanes + kG + u / 2);
          tmem_wait_loads();
          const float2 mu = unpack2<E>(m);
          const T* xu = x_at + (t0 + u) * p.x_token + side * kCols;
#pragma unroll
          for (int k = 0; k < kCols; ++k) {
            const float x = E::up(xu[k]);
            if (u <= line && !isfinite(x)) y[k] += (u & 1 ? mu.y : mu.x) * x;
            if (p.D && u == line && !isfinite(x)) y[k] += D * x;
          }
        }
      }
      // y through W's place, so that whole rows are written
#pragma unroll
      for (int k = 0; k < kCols; k += 8)
        *reinterpret_cast<uint4*>(smem + hi_to + panel_at(line, (side * kCols + k) / 8)) =
            make_uint4(pack2<E>(y[k], y[k + 1]), pack2<E>(y[k + 2], y[k + 3]), pack2<E>(y[k + 4], y[k + 5]), pack2<E>(y[k + 6], y[k + 7]));
      sync_eight();
      constexpr int kVecs = kP / 8, kApart = kThreads / kVecs;
      const int r0 = threadIdx.x / kVecs, c = threadIdx.x % kVecs;
      T* to = reinterpret_cast<T*>(p.out) + (t0 + r0) * p.out_token + h * p.out_head + p0 + c * 8;
#pragma unroll
      for (int k = 0; k < kChunk / kApart; ++k, to += kApart * p.out_token)
        if (t0 + r0 + k * kApart < end)
          *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(smem + hi_to + panel_at(r0, c) + k * kApart * 128);
    }
    turn();
  }
  if (kStateOnly || seg + 1 == segs) {
    float* to = kStateOnly ? p.segment_states + piece * all : reinterpret_cast<float*>(keep);
    if (line < N) {
#pragma unroll
      for (int k = 0; k < kCols; ++k) to[state_at + k * N] = state[k];
    }
    if (kStateOnly && p0 == 0 && threadIdx.x == 0) p.segment_exponents[(int64_t)piece * p.heads + h] = exponent;
  }
  if (dead) *p.timeout = 1;
  tmem_before_sync();
  if (__syncthreads_or(dead)) {  // products may still be at work: their end, however short the waits' limit is
    bar_wait(bar_end, 0, kDefaultWaitCycles);
    __syncthreads();
  }
  tmem_after_sync();
}

// Carries the states through a sequence's segments, four elements a thread: where the first pass left what a
// segment makes, the state it starts from takes its place.  Rows that overlap (starts that do not ascend) can make more
// segments than there is room for: those are left out here, as they are by the grids of the passes.
__global__ void __launch_bounds__(256) carry_kernel(const __grid_constant__ ScanParams p) {
  wait_for_previous();
  __shared__ int32_t first_s;
  const StateView& v = p.state;
  const int32_t s = blockIdx.z, h = blockIdx.y;
  if (threadIdx.x == 0) first_s = 0;
  __syncthreads();
  int32_t mine = 0;  // pieces of the sequences before, as far as there is room
  for (int32_t i = threadIdx.x; i < s; i += 256) {
    int64_t a, b;
    rows_of(v, i, &a, &b);
    mine = min(mine + pieces_of(a, b, p.segment, p.by_token), p.pieces);
  }
  for (int m = 16; m; m >>= 1) mine += __shfl_xor_sync(~0u, mine, m);
  if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&first_s, mine);
  __syncthreads();
  const uint8_t* in = slot_of(v, v.slots_in, s);
  if (!in || !slot_of(v, v.slots_out, s)) return;
  int64_t a, b;
  rows_of(v, s, &a, &b);
  const int32_t segs = min(pieces_of(a, b, p.segment, p.by_token), p.pieces - first_s);
  const int32_t i = blockIdx.x * 256 + threadIdx.x, vecs = p.head_dim * p.state_dim / 4;
  if (i >= vecs) return;
  float4 state = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!(v.fresh && v.fresh[s])) state = reinterpret_cast<const float4*>(in)[(int64_t)h * vecs + i];
  for (int32_t g0 = 0; g0 < segs; g0 += 8) {  // eight segments' loads at once
    float4 made[8];
    float decay[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t at = (int64_t)(first_s + g0 + k) * p.heads + h;
      made[k] = make_float4(0.f, 0.f, 0.f, 0.f), decay[k] = 0.f;
      if (g0 + k + 1 < segs) {
        made[k] = reinterpret_cast<const float4*>(p.segment_states)[at * vecs + i];
        decay[k] = ex2(p.segment_exponents[at]);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (g0 + k >= segs) break;
      reinterpret_cast<float4*>(p.segment_states)[((int64_t)(first_s + g0 + k) * p.heads + h) * vecs + i] = state;
      state.x = state.x * decay[k] + made[k].x, state.y = state.y * decay[k] + made[k].y;
      state.z = state.z * decay[k] + made[k].z, state.w = state.w * decay[k] + made[k].w;
    }
  }
}

template <class E, int N, int kP>
cudaError_t chunks(const ScanParams& p, cudaStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.pieces * (p.head_dim / kP)), p.heads);
  constexpr int kSmem = ScanShape<kP>::kSmem;
  if (p.segment_states) {
    cudaError_t e = launch_after(chunk_kernel<E, N, kP, true>, grid, kAllThreads, kSmem, s, p);
    if (e != cudaSuccess) return e;
    const dim3 all((p.head_dim * N / 4 + 255) / 256, p.heads, p.state.num_seqs);
    if ((e = launch_after(carry_kernel, all, 256, 0, s, p)) != cudaSuccess) return e;
  }
  return launch_after(chunk_kernel<E, N, kP, false>, grid, kAllThreads, kSmem, s, p);
}

template <class E>
cudaError_t chunks(const ScanParams& p, cudaStream_t s) {
  if (p.head_dim % 128 == 0) return p.state_dim == 64 ? chunks<E, 64, 128>(p, s) : chunks<E, 128, 128>(p, s);
  return p.state_dim == 64 ? chunks<E, 64, 64>(p, s) : chunks<E, 128, 64>(p, s);
}

template <class E, int N, int kP, bool kStateOnly>
cudaError_t prepare(bool* matrix) {
  auto kernel = chunk_kernel<E, N, kP, kStateOnly>;
  cudaFuncAttributes a;
  const cudaError_t e = cudaFuncGetAttributes(&a, kernel);
  if (e != cudaSuccess) return e;
  if (a.numRegs < kLaunchRegs) *matrix = false;  // the eight warps would wait for registers
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ScanShape<kP>::kSmem);
}

template <class E, int N, int kP>
cudaError_t prepare(bool* matrix) {
  const cudaError_t e = prepare<E, N, kP, true>(matrix);
  return e == cudaSuccess ? prepare<E, N, kP, false>(matrix) : e;
}

template <class E>
cudaError_t prepare(bool* matrix) {
  cudaError_t e;
  if ((e = prepare<E, 64, 64>(matrix)) != cudaSuccess || (e = prepare<E, 64, 128>(matrix)) != cudaSuccess) return e;
  if ((e = prepare<E, 128, 64>(matrix)) != cudaSuccess) return e;
  return prepare<E, 128, 128>(matrix);
}

}  // namespace

int32_t scan_segment(const StateView& v, int32_t heads, int32_t head_dim, int32_t state_dim, int num_sms, bool* cut,
                     int32_t* by_token) {
  *cut = false;
  *by_token = INT32_MAX;
  if (!v.starts || head_dim % 64 || (state_dim != 64 && state_dim != 128)) return 0;
  // A CTA of the matrix form takes some 9 us however few tokens a sequence has, a token of the recurrence 0.45 (one
  // sequence of 16 heads: 16 tokens 8.5 us against 9.8, 32 tokens 14.6 against 9.8).  A batch's short sequences are
  // left to the recurrence where most are short or there are CTAs for more than a round of the SMs; that is a launch more
  // and the time of its longest (32 sequences of unlike lengths: 8192 tokens 148 us instead of 174; 4 of them: 64
  // tokens 19 instead of 10).
  constexpr int32_t kShort = 16;
  const int32_t slices = head_dim / (head_dim % 128 ? 64 : 128);
  if (v.tokens <= kShort) return 0;
  const bool both = v.tokens <= 8ll * v.num_seqs || (int64_t)v.num_seqs * heads * slices >= 2 * num_sms;
  *by_token = v.num_seqs > 1 && both ? kShort : -1;
  // two chunks in a row take less than the three launches below (15 us instead of 20), three as long
  if (v.tokens <= 2 * kChunk) return 2 * kChunk;
  const int64_t all = (v.tokens + kChunk - 1) / kChunk * heads * slices;
  const int64_t each = std::max<int64_t>(1, (all + num_sms - 1) / num_sms);
  *cut = v.tokens > each * kChunk;
  return (int32_t)(each * kChunk);
}

cudaError_t launch_scan_chunks(const ScanParams& p, int type, cudaStream_t s) {
  return type == KVX_TYPE_BF16 ? chunks<Bf16>(p, s) : chunks<Fp16>(p, s);
}

cudaError_t prepare_state_kernels(bool* matrix) {
  *matrix = true;
  const cudaError_t e = prepare<Bf16>(matrix);
  return e == cudaSuccess ? prepare<Fp16>(matrix) : e;
}

}  // namespace kvx

// state_kernels.cu -- the recurrent layers' operators on their state slots: the
// short causal convolution and the selective scan.

#include <algorithm>

#include "mma.cuh"

namespace kvx {
namespace {

// ---------------------------------------------------------------- pieces of ragged sequences

// The piece'th of all sequences' pieces of `length` rows (at least one a sequence), counted in their order:
// its sequence, its place there, and how many pieces that sequence has.  False behind the last.  Found by the
// whole CTA; buf: a word a warp and three more.
template <int kThreads>
__device__ __forceinline__ bool find_piece(const StateView& v, int32_t piece, int32_t length, int32_t* buf, int32_t* seq,
                                           int32_t* at, int32_t* of) {
  if (!v.starts) {
    *seq = piece, *at = 0, *of = 1;
    return piece < v.num_seqs;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kWarps = kThreads / 32;
  int32_t before_all = 0;
  for (int32_t base = 0; base < v.num_seqs; base += kThreads) {
    const int32_t s = base + threadIdx.x;
    int32_t mine = 0;
    if (s < v.num_seqs) {
      int64_t first, last;
      rows_of(v, s, &first, &last);
      mine = max(1, (int32_t)((last - first + length - 1) / length));
    }
    int32_t upto = mine;
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t y = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += y;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = upto;
    if (threadIdx.x == 0) buf[kWarps] = -1;
    __syncthreads();
    int32_t chunk = 0;
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) upto += buf[i];
      chunk += buf[i];
    }
    const int32_t from = before_all + upto - mine;
    if (piece >= from && piece < from + mine) {
      buf[kWarps] = s;
      buf[kWarps + 1] = piece - from;
      buf[kWarps + 2] = mine;
    }
    __syncthreads();
    if (buf[kWarps] >= 0) {
      *seq = buf[kWarps], *at = buf[kWarps + 1], *of = buf[kWarps + 2];
      return true;
    }
    before_all += chunk;
  }
  return false;
}

// ---------------------------------------------------------------- convolution

constexpr int kConvThreads = 128, kConvRows = 32;

template <class E>
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = unpack2<E>(w[i]);
    f[2 * i] = x.x, f[2 * i + 1] = x.y;
  }
}

// A thread keeps 8 neighbouring channels' window of kWidth inputs in registers and walks up to 32 rows of
// one sequence, the next four rows' loads in flight behind the four it computes.  Bound by its bytes: a row in and a row out, the window's rows
// read again at the head of a piece (3 of 32, from L2).  The piece at a sequence's head, which alone reads the slot,
// also writes it, so a slot may be updated in place.
template <class E, int kWidth>
__global__ void __launch_bounds__(kConvThreads) conv_kernel(const __grid_constant__ ConvParams p) {
  wait_for_previous();
  constexpr int kPast = kWidth - 1;
  __shared__ int32_t buf[kConvThreads / 32 + 3];
  const StateView& v = p.state;
  int32_t s, piece, pieces;
  if (!find_piece<kConvThreads>(v, blockIdx.x, kConvRows, buf, &s, &piece, &pieces)) return;
  const int32_t c = (blockIdx.y * kConvThreads + threadIdx.x) * 8;
  if (c >= p.channels) return;
  int64_t first, last;
  rows_of(v, s, &first, &last);
  const int64_t begin = first + (int64_t)piece * kConvRows, end = min(last, begin + kConvRows);
  auto in_row = [&](int64_t t) { return *reinterpret_cast<const uint4*>(p.x + (t * p.x_stride + c) * 2); };
  auto out_row = [&](int64_t t) { return reinterpret_cast<uint4*>(p.out + (t * p.out_stride + c) * 2); };
  const uint8_t* in = slot_of(v, v.slots_in, s);
  uint8_t* keep = slot_of(v, v.slots_out, s);
  if (!in || !keep) {
    for (int64_t t = begin; t < end; ++t) *out_row(t) = make_uint4(0, 0, 0, 0);
    return;
  }
  float w[kWidth][8], bias[8] = {}, x[kPast + 4][8];  // the inputs before four rows, and theirs
  {
    float flat[8 * kWidth];
#pragma unroll
    for (int i = 0; i < kWidth; ++i)
      unpack8<E>(*reinterpret_cast<const uint4*>(p.weight + ((int64_t)c * kWidth + 8 * i) * 2), *reinterpret_cast<float(*)[8]>(flat + 8 * i));
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int j = 0; j < kWidth; ++j) w[j][k] = flat[k * kWidth + j];
  }
  if (p.bias) unpack8<E>(*reinterpret_cast<const uint4*>(p.bias + (int64_t)c * 2), bias);
  uint4 old[kPast];  // the inputs before the piece
#pragma unroll
  for (int j = 0; j < kPast; ++j) {
    if (piece > 0)
      old[j] = in_row(begin - kPast + j);
    else if (v.fresh && v.fresh[s])
      old[j] = make_uint4(0, 0, 0, 0);
    else
      old[j] = *reinterpret_cast<const uint4*>(in + ((int64_t)j * p.channels + c) * 2);
    unpack8<E>(old[j], x[j]);
  }
  auto row = [&](int u, uint4* to) {  // of the four
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      y[k] = bias[k];
#pragma unroll
      for (int j = 0; j < kWidth; ++j) y[k] += w[j][k] * x[u + j][k];
    }
    if (p.silu) {
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] *= rcp(1.f + ex2(-kLog2e * y[k]));
    }
    *to = make_uint4(pack2<E>(y[0], y[1]), pack2<E>(y[2], y[3]), pack2<E>(y[4], y[5]), pack2<E>(y[6], y[7]));
  };
  const uint8_t* from = p.x + (begin * p.x_stride + c) * 2;
  uint8_t* to = p.out + (begin * p.out_stride + c) * 2;
  const int64_t from_step = p.x_stride * 2, to_step = p.out_stride * 2;
  int32_t left = (int32_t)(end - begin);
  uint4 next[4];
  if (left >= 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) next[u] = __ldcs(reinterpret_cast<const uint4*>(from + u * from_step));
  }
  for (; left >= 4; left -= 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) unpack8<E>(next[u], x[kPast + u]);
    from += 4 * from_step;
    if (left >= 8) {
#pragma unroll
      for (int u = 0; u < 4; ++u) next[u] = __ldcs(reinterpret_cast<const uint4*>(from + u * from_step));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) row(u, reinterpret_cast<uint4*>(to + u * to_step));
    to += 4 * to_step;
#pragma unroll
    for (int j = 0; j < kPast; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) x[j][k] = x[j + 4][k];
  }
  for (; left > 0; --left, from += from_step, to += to_step) {
    unpack8<E>(*reinterpret_cast<const uint4*>(from), x[kPast]);
    row(0, reinterpret_cast<uint4*>(to));
#pragma unroll
    for (int j = 0; j < kPast; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) x[j][k] = x[j + 1][k];
  }
  if (piece == 0) {
#pragma unroll
    for (int j = 0; j < kPast; ++j) {
      const int64_t t = last - kPast + j;
      uint4 raw = old[0];
#pragma unroll
      for (int k = 1; k < kPast; ++k)
        if (t - first + kPast == k) raw = old[k];
      if (t >= first) raw = in_row(t);
      *reinterpret_cast<uint4*>(keep + ((int64_t)j * p.channels + c) * 2) = raw;
    }
  }
}

template <class E>
cudaError_t conv(const ConvParams& p, cudaStream_t s) {
  const int64_t pieces = p.state.starts ? p.state.tokens / kConvRows + p.state.num_seqs : p.state.num_seqs;
  const dim3 grid((unsigned)pieces, (p.channels / 8 + kConvThreads - 1) / kConvThreads);
  auto kernel = p.width == 2 ? conv_kernel<E, 2> : p.width == 3 ? conv_kernel<E, 3> : conv_kernel<E, 4>;
  return launch_after(kernel, grid, kConvThreads, 0, s, p);
}

// ---------------------------------------------------------------- scan, token by token

__device__ __forceinline__ float step_of(const ScanParams& p, float raw, int32_t h) {
  if (p.dt_bias) raw += p.dt_bias[h];
  return p.softplus ? (raw > 20.f ? raw : log1pf(expf(raw))) : raw;
}

// The recurrence as it stands, for single tokens and for what the matrix form below does not take.  Bound by the
// state's bytes, read and written once: a row of N elements lies over kLanes lanes, 16 bytes each
// at least, and a lane has kRows rows, whose loads are all in flight at once; their sums y meet in one
// reduction that halves the rows at every step.
template <class E, int N, int kRows>
__global__ void __launch_bounds__(128) scan_kernel(const __grid_constant__ ScanParams p) {
  wait_for_previous();
  using T = typename E::T;
  constexpr int kLanes = N / 4 < 32 ? N / 4 : 32, kVec = N / kLanes, kSub = 32 / kLanes;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, in_row = lane % kLanes, col = in_row * kVec;
  const int32_t row0 = (blockIdx.x * 4 + (threadIdx.x >> 5)) * kRows * kSub + sub;  // rows row0 + r * kSub
  const int32_t h = blockIdx.y, s = blockIdx.z;
  const StateView& v = p.state;
  const uint8_t* in = slot_of(v, v.slots_in, s);
  uint8_t* keep = slot_of(v, v.slots_out, s);
  int64_t first, last;
  rows_of(v, s, &first, &last);
  T* out = reinterpret_cast<T*>(p.out) + h * p.out_head;
  if (!in || !keep) {
    for (int64_t t = first; t < last; ++t)
      for (int r = 0; r < kRows; ++r)
        if (in_row == 0 && row0 + r * kSub < p.head_dim) out[t * p.out_token + row0 + r * kSub] = E::down(0.f);
    return;
  }
  const bool fresh = v.fresh && v.fresh[s];
  const int64_t at = ((int64_t)h * p.head_dim + row0) * N + col;
  float state[kRows][kVec];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int i = 0; i < kVec; i += 4) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (!fresh && row0 + r * kSub < p.head_dim)
        x = __ldcs(reinterpret_cast<const float4*>(in) + (at + r * kSub * N + i) / 4);
      state[r][i] = x.x, state[r][i + 1] = x.y, state[r][i + 2] = x.z, state[r][i + 3] = x.w;
    }
  const float A = p.A[h] * kLog2e, D = p.D ? p.D[h] : 0.f;
  const int32_t group = h / p.heads_per_group;
  const T* b_at = reinterpret_cast<const T*>(p.b) + group * p.b_group + col;
  const T* c_at = reinterpret_cast<const T*>(p.c) + group * p.c_group + col;
  const T* x_at = reinterpret_cast<const T*>(p.x) + h * p.x_head;
  for (int64_t t = first; t < last; ++t) {
    uint32_t braw[kVec / 2], craw[kVec / 2];
#pragma unroll
    for (int i = 0; i < kVec / 2; ++i) {
      braw[i] = *reinterpret_cast<const uint32_t*>(b_at + t * p.b_token + 2 * i);
      craw[i] = *reinterpret_cast<const uint32_t*>(c_at + t * p.c_token + 2 * i);
    }
    float x[kRows], y[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      x[r] = row0 + r * kSub < p.head_dim ? E::up(x_at[t * p.x_token + row0 + r * kSub]) : 0.f;
    const float d = step_of(p, E::up(reinterpret_cast<const T*>(p.dt)[t * p.dt_token + h]), h);
    const float decay = ex2(d * A);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const float dx = d * x[r];
      y[r] = 0.f;
#pragma unroll
      for (int i = 0; i < kVec / 2; ++i) {
        const float2 b = unpack2<E>(braw[i]), c = unpack2<E>(craw[i]);
        state[r][2 * i] = state[r][2 * i] * decay + dx * b.x;
        state[r][2 * i + 1] = state[r][2 * i + 1] * decay + dx * b.y;
        y[r] += state[r][2 * i] * c.x + state[r][2 * i + 1] * c.y;
      }
    }
    // Lanes that differ in one bit exchange halves of their rows, then, with one row left, its halves.
    int32_t mine = 0;
    int m = kLanes / 2;
#pragma unroll
    for (int left = kRows; left > 1; left /= 2, m /= 2) {
      const bool upper = lane & m;
      mine = 2 * mine + upper;
#pragma unroll
      for (int r = 0; r < left / 2; ++r) {
        const float send = upper ? y[r] : y[r + left / 2], stay = upper ? y[r + left / 2] : y[r];
        y[r] = stay + __shfl_xor_sync(~0u, send, m);
      }
    }
#pragma unroll
    for (int k = m; k; k >>= 1) y[0] += __shfl_xor_sync(~0u, y[0], k);
    float xs = x[0];
#pragma unroll
    for (int r = 1; r < kRows; ++r) xs = mine == r ? x[r] : xs;
    if (in_row % (kLanes / kRows) == 0 && row0 + mine * kSub < p.head_dim)
      out[t * p.out_token + row0 + mine * kSub] = E::down(y[0] + D * xs);
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int i = 0; i < kVec; i += 4)
      if (row0 + r * kSub < p.head_dim)
        __stcs(reinterpret_cast<float4*>(keep) + (at + r * kSub * N + i) / 4,
               make_float4(state[r][i], state[r][i + 1], state[r][i + 2], state[r][i + 3]));
}

template <class E, int N>
cudaError_t scan(const ScanParams& p, int num_sms, cudaStream_t s) {
  constexpr int kSub = N / 4 < 32 ? 128 / N : 1;
  constexpr int kMany = N == 16 ? 4 : N == 256 ? 4 : 8, kFew = 2;
  // many rows a lane for bandwidth, where that leaves a CTA for every SM; few for latency
  const bool many = (int64_t)p.state.num_seqs * p.heads * p.head_dim >= (int64_t)num_sms * 4 * kSub * kMany;
  const int rows = 4 * kSub * (many ? kMany : kFew);
  const dim3 grid((p.head_dim + rows - 1) / rows, p.heads, p.state.num_seqs);
  return many ? launch_after(scan_kernel<E, N, kMany>, grid, 128, 0, s, p) : launch_after(scan_kernel<E, N, kFew>, grid, 128, 0, s, p);
}

// ---------------------------------------------------------------- scan of prompts, in matrix form

// With a_t = A d_t and c_t the sum of a up to t within a chunk of 64 tokens,
//   y_t = sum_{s <= t} (C_t . B_s) e^{c_t - c_s} d_s x_s + e^{c_t} C_t h_in
//   h_out = e^{c_63} h_in + sum_s e^{c_63 - c_s} d_s x_s B_s^T
// so a chunk is four products of matrices.  A CTA has 64 rows (head_dim) of one head's state in its four
// warps' registers (fp32, 16 rows a warp, all of state_dim) and walks the chunks of a segment; each warp also
// has 16 tokens of y.  The next chunk's rows come in asynchronously behind the products.
//
// Rounding: the weighted products C.B and the carried state are rounded to the inputs' type for the product
// that makes y, one rounding a term, as y is rounded to that type anyway.  The state is kept in fp32: the
// weighted x is split into two numbers of that type, whose sum is x to 16 bits or more, and
// both are multiplied with B.  In fp16 both are scaled by powers of two to stay in its range.
//
// A long sequence is cut into segments, so that every SM has some: a first pass makes each segment's state
// from nothing, a second one carries the states through the segments, and the last one
// starts every segment with its own.  What that costs is the state's product once more.
constexpr int kChunk = 64, kScanThreads = 128, kSlice = 64;

template <int N>
struct ScanShape {
  static constexpr int kBPitch = N * 2 + 16, kXPitch = kSlice * 2 + 16;
  static constexpr int kB = kChunk * kBPitch, kX = kChunk * kXPitch;
  static constexpr int kStage = 2 * kB + kX;  // B, C, x
  static constexpr int kSmem = 2 * kStage + kSlice * kBPitch;  // and the carried state, rounded
};

template <class E, int N, bool kStateOnly>
__global__ void __launch_bounds__(kScanThreads, 2) chunk_kernel(const __grid_constant__ ScanParams p) {
  using S = ScanShape<N>;
  using T = typename E::T;
  constexpr bool kHalf = std::is_same<E, Fp16>::value;
  constexpr int kKs = N / 16;
  wait_for_previous();
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int32_t buf[kScanThreads / 32 + 3];
  __shared__ float sum_s[4][kChunk], weight_s[4][kChunk], d_s[4][kChunk];  // each warp's own
  __shared__ float block_scale[4];  // fp16: of 16 rows of the rounded state
  const StateView& v = p.state;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, sub = lane & 3;
  const int32_t slices = p.head_dim / kSlice, piece = blockIdx.x / slices, p0 = (blockIdx.x - piece * slices) * kSlice;
  const int32_t h = blockIdx.y, group = h / p.heads_per_group;
  int32_t s, seg, segs;
  if (!find_piece<kScanThreads>(v, piece, p.segment, buf, &s, &seg, &segs)) return;
  if (kStateOnly && seg + 1 == segs) return;  // the last segment's state is nobody's start
  int64_t first, last;
  rows_of(v, s, &first, &last);
  const int64_t begin = first + (int64_t)seg * p.segment, end = min(last, begin + p.segment);
  const uint8_t* in = slot_of(v, v.slots_in, s);
  uint8_t* keep = slot_of(v, v.slots_out, s);
  if (!in || !keep) {
    if (!kStateOnly)
      for (int64_t i = threadIdx.x; i < (end - begin) * (kSlice / 2); i += kScanThreads)
        *reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(p.out) + (begin + i / (kSlice / 2)) * p.out_token + h * p.out_head + p0 +
                                     i % (kSlice / 2) * 2) = 0;
    return;
  }
  const T* b_at = reinterpret_cast<const T*>(p.b) + group * p.b_group;
  const T* c_at = reinterpret_cast<const T*>(p.c) + group * p.c_group;
  const T* x_at = reinterpret_cast<const T*>(p.x) + h * p.x_head + p0;
  const T* dt_at = reinterpret_cast<const T*>(p.dt) + h;
  const uint32_t base = smem_at(smem), state_at = base + 2 * S::kStage;

  auto fetch = [&](int64_t t0, int stage) {  // rows behind the last are zeros
    const uint32_t to = base + stage * S::kStage;
    auto rows = [&](const T* src, int64_t stride, int vecs, uint32_t at, int pitch) {
      for (int i = threadIdx.x; i < kChunk * vecs; i += kScanThreads) {
        const int r = i / vecs, k = i % vecs;
        const uint32_t dst = at + r * pitch + k * 16;
        const bool there = t0 + r < end;
        copy_async(dst, src + (there ? t0 + r : t0) * stride + k * 8, there ? 16 : 0);
      }
    };
    rows(b_at, p.b_token, N / 8, to, S::kBPitch);
    if (!kStateOnly) rows(c_at, p.c_token, N / 8, to + S::kB, S::kBPitch);
    rows(x_at, p.x_token, kSlice / 8, to + 2 * S::kB, S::kXPitch);
    commit_async();
  };
  auto step_at = [&](int64_t t) { return t < end ? step_of(p, E::up(dt_at[t * p.dt_token]), h) : 0.f; };

  fetch(begin, 0);
  float d0 = step_at(begin + 2 * lane), d1 = step_at(begin + 2 * lane + 1);
  const float A2 = p.A[h] * kLog2e, D = p.D ? p.D[h] : 0.f;

  // Rows 16 warp + quad and + 8 of the slice, columns 8 n + 2 sub and the next.
  float state[N / 8][4];
  const int32_t row = p0 + warp * 16 + quad;
  const int64_t state_row = ((int64_t)h * p.head_dim + row) * N + 2 * sub;
  const int64_t all = (int64_t)p.heads * p.head_dim * N;
  {
    const float* from = p.segment_states ? p.segment_states + piece * all : reinterpret_cast<const float*>(in);
    const bool none = kStateOnly || (!p.segment_states && v.fresh && v.fresh[s]);
#pragma unroll
    for (int n = 0; n < N / 8; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 x = none ? make_float2(0.f, 0.f) : *reinterpret_cast<const float2*>(from + state_row + j * 8 * N + n * 8);
        state[n][2 * j] = x.x, state[n][2 * j + 1] = x.y;
      }
  }
  // The state as the product that makes y takes it: rounded, in fp16 after scaling 16 rows at a time.
  auto round_state = [&]() {
    float scale = 1.f;
    if constexpr (kHalf) {
      float top = 0.f;
#pragma unroll
      for (int n = 0; n < N / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(state[n][e]));
      for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, m));
      const int e = top > 0.f && top < INFINITY ? max(-100, min(100, 10 - ilogbf(top))) : 0;
      scale = ldexpf(1.f, e);
      if (lane == 0) block_scale[warp] = ldexpf(1.f, -e);
    }
    uint8_t* to = smem + 2 * S::kStage + (warp * 16 + quad) * S::kBPitch + 4 * sub;
#pragma unroll
    for (int n = 0; n < N / 8; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *reinterpret_cast<uint32_t*>(to + j * 8 * S::kBPitch + n * 16) =
            pack2<E>(state[n][2 * j] * scale, state[n][2 * j + 1] * scale);
  };
  if (!kStateOnly) round_state();

  // where a lane's matrices begin: rows as they lie (K-like and, as a left factor, the same), and transposed
  const uint32_t lane_rows = (lane & 7) + (((lane >> 3) & 1) << 3), lane_rows2 = (lane & 7) + ((lane >> 4) << 3);
  float exponent = 0.f;  // of the decay over the segment so far
  int stage = 0;
  for (int64_t t0 = begin; t0 < end; t0 += kChunk, stage ^= 1) {
    // Sums of the chunk's exponents, up to and behind each token (from the end, so that they are exact where
    // their weight is not small): every warp for itself.
    {
      const float a0 = d0 * A2, a1 = d1 * A2;
      float upto = a0 + a1, behind = a0 + a1;
      for (int d = 1; d < 32; d <<= 1) {
        const float y = __shfl_up_sync(~0u, upto, d), z = __shfl_down_sync(~0u, behind, d);
        if (lane >= d) upto += y;
        if (lane + d < 32) behind += z;
      }
      float above = __shfl_down_sync(~0u, behind, 1), below = __shfl_up_sync(~0u, upto, 1);
      if (lane == 31) above = 0.f;
      if (lane == 0) below = 0.f;
      __syncwarp();
      sum_s[warp][2 * lane] = below + a0;
      sum_s[warp][2 * lane + 1] = upto;
      weight_s[warp][2 * lane] = d0 * ex2(above + a1);
      weight_s[warp][2 * lane + 1] = d1 * ex2(above);
      d_s[warp][2 * lane] = d0;
      d_s[warp][2 * lane + 1] = d1;
      __syncwarp();
    }
    const float chunk_exponent = sum_s[warp][kChunk - 1];
    wait_async<0>();
    __syncthreads();  // the chunk's rows and the rounded state are there, and the other stage is free
    if (t0 + kChunk < end) {
      fetch(t0 + kChunk, stage ^ 1);
      d0 = step_at(t0 + kChunk + 2 * lane), d1 = step_at(t0 + kChunk + 2 * lane + 1);
    }
    const uint32_t b_s = base + stage * S::kStage, c_s = b_s + S::kB, x_s = c_s + S::kB;

    if constexpr (!kStateOnly) {
      const int t_row = warp * 16 + quad;  // and + 8
      uint32_t cf[kKs][4];
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks)
        load_matrices(cf[ks], c_s + (warp * 16 + lane_rows) * S::kBPitch + ks * 32 + (lane >> 4) * 16);
      float y[kSlice / 8][4];
#pragma unroll
      for (int q = 0; q < kSlice / 8; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[q][e] = 0.f;
      const float sum_t[2] = {sum_s[warp][t_row], sum_s[warp][t_row + 8]};
      // C h_in, 16 rows of the state at a time
#pragma unroll
      for (int q = 0; q < kSlice / 16; ++q) {
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
          uint32_t b[4];
          load_matrices(b, state_at + (q * 16 + lane_rows2) * S::kBPitch + ks * 32 + ((lane >> 3) & 1) * 16);
          mma<E>(y[2 * q], cf[ks], b[0], b[1]);
          mma<E>(y[2 * q + 1], cf[ks], b[2], b[3]);
        }
        const float scale = kHalf ? block_scale[q] : 1.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float by = ex2(sum_t[e >> 1]) * scale;
          y[2 * q][e] *= by, y[2 * q + 1][e] *= by;
        }
      }
      // the chunk's own tokens, 16 at a time, up to this warp's
#pragma unroll 1
      for (int q = 0; q <= warp; ++q) {
        float g[2][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) g[0][e] = g[1][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
          uint32_t b[4];
          load_matrices(b, b_s + (q * 16 + lane_rows2) * S::kBPitch + ks * 32 + ((lane >> 3) & 1) * 16);
          mma<E>(g[0], cf[ks], b[0], b[1]);
          mma<E>(g[1], cf[ks], b[2], b[3]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = t_row + 8 * (e >> 1), u = q * 16 + k * 8 + 2 * sub + (e & 1);
            g[k][e] = u <= t ? g[k][e] * ex2(sum_t[e >> 1] - sum_s[warp][u]) * d_s[warp][u] : 0.f;
          }
        const uint32_t gf[4] = {pack2<E>(g[0][0], g[0][1]), pack2<E>(g[0][2], g[0][3]), pack2<E>(g[1][0], g[1][1]),
                                pack2<E>(g[1][2], g[1][3])};
        uint32_t xf[kSlice / 16][4];
        bool odd = false;
#pragma unroll
        for (int r = 0; r < kSlice / 16; ++r) {
          load_matrices_t(xf[r], x_s + (q * 16 + lane_rows) * S::kXPitch + r * 32 + (lane >> 4) * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= odd2<E>(xf[r][e]);
        }
        // a token's x that is not finite must not reach the tokens before it (0 x inf)
        if (q == warp && __any_sync(~0u, odd)) {
#pragma unroll 1
          for (int k = 0; k < 16; ++k) {
            const int from = (lane & ~3) | ((k & 7) >> 1);
            float gk[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float lo = k < 8 ? g[0][2 * j] : g[1][2 * j], hi = k < 8 ? g[0][2 * j + 1] : g[1][2 * j + 1];
              gk[j] = __shfl_sync(~0u, k & 1 ? hi : lo, from);
            }
#pragma unroll
            for (int r = 0; r < kSlice / 8; ++r)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const T* at = reinterpret_cast<const T*>(smem + (x_s - base) + (q * 16 + k) * S::kXPitch) + r * 8 + 2 * sub + (e & 1);
                if (q * 16 + k <= t_row + 8 * (e >> 1)) y[r][e] += gk[e >> 1] * E::up(*at);
              }
          }
        } else {
#pragma unroll
          for (int r = 0; r < kSlice / 16; ++r) {
            mma<E>(y[2 * r], gf, xf[r][0], xf[r][1]);
            mma<E>(y[2 * r + 1], gf, xf[r][2], xf[r][3]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t t = t0 + t_row + 8 * j;
        if (t < end) {
          T* to = reinterpret_cast<T*>(p.out) + t * p.out_token + h * p.out_head + p0 + 2 * sub;
          const uint8_t* xt = smem + (x_s - base) + (t_row + 8 * j) * S::kXPitch + 4 * sub;
#pragma unroll
          for (int q = 0; q < kSlice / 8; ++q) {
            const float2 x = unpack2<E>(*reinterpret_cast<const uint32_t*>(xt + q * 16));
            const float a = p.D ? y[q][2 * j] + D * x.x : y[q][2 * j], b = p.D ? y[q][2 * j + 1] + D * x.y : y[q][2 * j + 1];
            *reinterpret_cast<uint32_t*>(to + q * 8) = pack2<E>(a, b);
          }
        }
      }
    }

    // The state: this warp's 16 rows of x^T, weighted, times B.
    uint32_t hi[kChunk / 16][4], lo[kChunk / 16][4];
    float back = 1.f;
    {
      float top = 0.f;
      float2 f[kChunk / 16][4];
#pragma unroll
      for (int ks = 0; ks < kChunk / 16; ++ks) {
        uint32_t a[4];
        load_matrices_t(a, x_s + (ks * 16 + lane_rows2) * S::kXPitch + warp * 32 + ((lane >> 3) & 1) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int u = ks * 16 + 2 * sub + 8 * (e >> 1);
          f[ks][e] = unpack2<E>(a[e]);
          f[ks][e].x *= weight_s[warp][u], f[ks][e].y *= weight_s[warp][u + 1];
          if (kHalf) top = fmaxf(top, fmaxf(fabsf(f[ks][e].x), fabsf(f[ks][e].y)));
        }
      }
      float scale = 1.f;
      if constexpr (kHalf) {
        for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, m));
        const int e = top > 0.f && top < INFINITY ? max(-100, min(100, 10 - ilogbf(top))) : 0;
        scale = ldexpf(1.f, e), back = ldexpf(1.f, -e);
      }
#pragma unroll
      for (int ks = 0; ks < kChunk / 16; ++ks)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = make_float2(f[ks][e].x * scale, f[ks][e].y * scale);
          hi[ks][e] = pack2<E>(x.x, x.y);
          const float2 r = unpack2<E>(hi[ks][e]);
          lo[ks][e] = pack2<E>(x.x - r.x, x.y - r.y);
        }
    }
    const float decay = ex2(chunk_exponent);
#pragma unroll
    for (int n = 0; n < N / 16; ++n) {
      float made[2][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) made[0][e] = made[1][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < kChunk / 16; ++ks) {
        uint32_t b[4];
        load_matrices_t(b, b_s + (ks * 16 + lane_rows) * S::kBPitch + n * 32 + (lane >> 4) * 16);
        mma<E>(made[0], lo[ks], b[0], b[1]);
        mma<E>(made[1], lo[ks], b[2], b[3]);
        mma<E>(made[0], hi[ks], b[0], b[1]);
        mma<E>(made[1], hi[ks], b[2], b[3]);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) state[2 * n + k][e] = state[2 * n + k][e] * decay + made[k][e] * back;
    }
    exponent += chunk_exponent;
    __syncthreads();  // everyone has read the rounded state and this stage
    if (!kStateOnly && t0 + kChunk < end) round_state();
  }

  float* to = nullptr;
  if (kStateOnly) {
    to = p.segment_states + piece * all;
    if (p0 == 0 && threadIdx.x == 0) p.segment_exponents[(int64_t)piece * p.heads + h] = exponent;
  } else if (seg + 1 == segs) {
    to = reinterpret_cast<float*>(keep);
  }
  if (to) {
#pragma unroll
    for (int n = 0; n < N / 8; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *reinterpret_cast<float2*>(to + state_row + j * 8 * N + n * 8) = make_float2(state[n][2 * j], state[n][2 * j + 1]);
  }
}

// Carries the states through a sequence's segments, four elements a thread: where the first pass left what a
// segment makes, the state it starts from takes its place.
__global__ void __launch_bounds__(256) carry_kernel(const __grid_constant__ ScanParams p) {
  wait_for_previous();
  __shared__ int32_t first_s;
  const StateView& v = p.state;
  const int32_t s = blockIdx.z, h = blockIdx.y;
  if (threadIdx.x == 0) first_s = 0;
  __syncthreads();
  int32_t mine = 0;  // pieces of the sequences before
  for (int32_t i = threadIdx.x; i < s; i += 256) {
    int64_t a, b;
    rows_of(v, i, &a, &b);
    mine += max(1, (int32_t)((b - a + p.segment - 1) / p.segment));
  }
  for (int m = 16; m; m >>= 1) mine += __shfl_xor_sync(~0u, mine, m);
  if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&first_s, mine);
  __syncthreads();
  const uint8_t* in = slot_of(v, v.slots_in, s);
  if (!in || !slot_of(v, v.slots_out, s)) return;
  int64_t a, b;
  rows_of(v, s, &a, &b);
  const int32_t segs = max(1, (int32_t)((b - a + p.segment - 1) / p.segment));
  const int32_t i = blockIdx.x * 256 + threadIdx.x, vecs = p.head_dim * p.state_dim / 4;
  if (i >= vecs) return;
  float4 state = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!(v.fresh && v.fresh[s])) state = reinterpret_cast<const float4*>(in)[(int64_t)h * vecs + i];
  for (int32_t g = 0; g < segs; ++g) {
    const int64_t piece = first_s + g;
    float4* at = reinterpret_cast<float4*>(p.segment_states) + (piece * p.heads + h) * vecs + i;
    const float4 made = g + 1 < segs ? *at : make_float4(0.f, 0.f, 0.f, 0.f);
    *at = state;
    if (g + 1 < segs) {
      const float decay = ex2(p.segment_exponents[piece * p.heads + h]);
      state.x = state.x * decay + made.x, state.y = state.y * decay + made.y;
      state.z = state.z * decay + made.z, state.w = state.w * decay + made.w;
    }
  }
}

template <class E, int N>
cudaError_t chunks(ScanParams p, cudaStream_t s) {
  const int64_t pieces = p.state.tokens / p.segment + p.state.num_seqs;
  const dim3 grid((unsigned)(pieces * (p.head_dim / kSlice)), p.heads);
  constexpr int kSmem = ScanShape<N>::kSmem;
  if (p.segment_states) {
    cudaError_t e = launch_after(chunk_kernel<E, N, true>, grid, kScanThreads, kSmem, s, p);
    if (e != cudaSuccess) return e;
    const dim3 all((p.head_dim * N / 4 + 255) / 256, p.heads, p.state.num_seqs);
    if ((e = launch_after(carry_kernel, all, 256, 0, s, p)) != cudaSuccess) return e;
  }
  return launch_after(chunk_kernel<E, N, false>, grid, kScanThreads, kSmem, s, p);
}

template <class E>
cudaError_t scan(const ScanParams& p, int num_sms, cudaStream_t s) {
  if (p.segment) return p.state_dim == 64 ? chunks<E, 64>(p, s) : chunks<E, 128>(p, s);
  switch (p.state_dim) {
    case 16: return scan<E, 16>(p, num_sms, s);
    case 32: return scan<E, 32>(p, num_sms, s);
    case 64: return scan<E, 64>(p, num_sms, s);
    case 128: return scan<E, 128>(p, num_sms, s);
    default: return scan<E, 256>(p, num_sms, s);
  }
}

template <class E, int N>
cudaError_t prepare() {
  cudaError_t e = cudaFuncSetAttribute(chunk_kernel<E, N, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, ScanShape<N>::kSmem);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(chunk_kernel<E, N, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, ScanShape<N>::kSmem);
}

}  // namespace

cudaError_t launch_conv(const ConvParams& p, int type, cudaStream_t s) {
  return type == KVX_TYPE_BF16 ? conv<Bf16>(p, s) : conv<Fp16>(p, s);
}

int32_t scan_segment(const StateView& v, int32_t heads, int32_t head_dim, int32_t state_dim, int num_sms, bool* cut) {
  *cut = false;
  if (!v.starts || head_dim % kSlice || (state_dim != 64 && state_dim != 128)) return 0;
  if (v.tokens < 16ll * v.num_seqs) return 0;  // mostly short ones: a chunk would be mostly empty
  const int64_t all = (v.tokens + kChunk - 1) / kChunk * heads * (head_dim / kSlice);
  const int64_t each = std::max<int64_t>(1, (all + 2 * num_sms - 1) / (2 * num_sms));
  *cut = v.tokens > each * kChunk;
  return (int32_t)(each * kChunk);
}

cudaError_t launch_scan(const ScanParams& p, int type, int num_sms, cudaStream_t s) {
  return type == KVX_TYPE_BF16 ? scan<Bf16>(p, num_sms, s) : scan<Fp16>(p, num_sms, s);
}

cudaError_t prepare_state_kernels() {
  cudaError_t e;
  if ((e = prepare<Bf16, 64>()) != cudaSuccess || (e = prepare<Bf16, 128>()) != cudaSuccess) return e;
  if ((e = prepare<Fp16, 64>()) != cudaSuccess) return e;
  return prepare<Fp16, 128>();
}

}  // namespace kvx

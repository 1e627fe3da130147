// state_kernels.cu -- the recurrent layers' operators on their state slots: the
// short causal convolution, and the selective scan token by token.

#include <algorithm>

#include "state_common.cuh"

namespace kvx {
namespace {

// ---------------------------------------------------------------- convolution

constexpr int kConvThreads = 128, kConvRows = 32;

template <class E>
__device__ __forceinline__ void unpack8(const uint4& v, float2 (&f)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = unpack2<E>(w[i]);
}

// A thread keeps 8 neighbouring channels' window of kWidth inputs in registers and walks up to 32 rows of one sequence.
// Bound by its bytes: a row in and a row out, the window's rows read again at the head of a piece (3 of 32, from L2).
// Rows come through a ring in shared memory, four groups of four ahead, that a thread fills and empties for itself, so
// there is no barrier (with the four next rows in registers, half as many bytes were in flight, and 12,001 rows of 8,192
// channels took 86 us instead of 74).  Two channels go through one fp32 instruction: 72 us, 5.6 TB/s.  Pieces of 48 rows
// are 2 % faster at that size, but leave fewer CTAs where prompts are short.  The piece at a sequence's head, which alone
// reads the slot, also writes it, so a slot may be updated in place.
constexpr int kGroup = 4, kAhead = 4;
template <class E, int kWidth>
__global__ void __launch_bounds__(kConvThreads, 4) conv_kernel(const __grid_constant__ ConvParams p) {
  wait_for_previous();
  constexpr int kPast = kWidth - 1;
  __shared__ int32_t buf[kConvThreads / 32 + 3];
  __shared__ uint4 ring[kAhead + 1][kGroup][kConvThreads];
  const StateView& v = p.state;
  Piece found;
  if (!find_piece<kConvThreads>(v, blockIdx.x, kConvRows, -1, buf, &found)) return;
  const int32_t c = (blockIdx.y * kConvThreads + threadIdx.x) * 8;
  if (c >= p.channels) return;
  const int32_t piece = found.at;
  const int64_t first = found.first, last = found.last;
  const int64_t begin = first + (int64_t)piece * kConvRows, end = min(last, begin + kConvRows);
  auto in_row = [&](int64_t t) { return *reinterpret_cast<const uint4*>(p.x + (t * p.x_stride + c) * 2); };
  auto out_row = [&](int64_t t) { return reinterpret_cast<uint4*>(p.out + (t * p.out_stride + c) * 2); };
  const uint8_t* in = found.in;
  uint8_t* keep = found.keep;
  if (!in || !keep) {
    for (int64_t t = begin; t < end; ++t) *out_row(t) = make_uint4(0, 0, 0, 0);
    return;
  }
  float2 w[kWidth][4], bias[4] = {}, x[kPast + kGroup][4];  // the inputs before four rows, and theirs
  {
    float2 flat[kWidth][4];
#pragma unroll
    for (int i = 0; i < kWidth; ++i)
      unpack8<E>(*reinterpret_cast<const uint4*>(p.weight + ((int64_t)c * kWidth + 8 * i) * 2), flat[i]);
    auto at = [&](int n) { return n & 1 ? flat[n / 8][n % 8 / 2].y : flat[n / 8][n % 8 / 2].x; };
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < kWidth; ++j) w[j][k] = make_float2(at(2 * k * kWidth + j), at((2 * k + 1) * kWidth + j));
  }
  if (p.bias) unpack8<E>(*reinterpret_cast<const uint4*>(p.bias + (int64_t)c * 2), bias);
  uint4 old[kPast];  // the inputs before the piece
#pragma unroll
  for (int j = 0; j < kPast; ++j) {
    if (piece > 0)
      old[j] = in_row(begin - kPast + j);
    else if (found.fresh)
      old[j] = make_uint4(0, 0, 0, 0);
    else
      old[j] = *reinterpret_cast<const uint4*>(in + ((int64_t)j * p.channels + c) * 2);
    unpack8<E>(old[j], x[j]);
  }
  auto row = [&](int u, uint4* to) {  // of the four
    float2 y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      y[k] = bias[k];
#pragma unroll
      for (int j = 0; j < kWidth; ++j) y[k] = fma2(w[j][k], x[u + j][k], y[k]);
    }
    if (p.silu) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 e = mul2(y[k], make_float2(-kLog2e, -kLog2e));
        const float2 one = add2(make_float2(ex2(e.x), ex2(e.y)), make_float2(1.f, 1.f));
        y[k] = mul2(y[k], make_float2(rcp(one.x), rcp(one.y)));
      }
    }
    *to = make_uint4(pack2<E>(y[0].x, y[0].y), pack2<E>(y[1].x, y[1].y), pack2<E>(y[2].x, y[2].y), pack2<E>(y[3].x, y[3].y));
  };
  const uint8_t* from = p.x + (begin * p.x_stride + c) * 2;
  uint8_t* to = p.out + (begin * p.out_stride + c) * 2;
  const int64_t from_step = p.x_stride * 2, to_step = p.out_stride * 2;
  const int32_t rows = (int32_t)(end - begin);
  auto fetch = [&](int32_t r) {  // rows r .. r + 3
#pragma unroll
    for (int u = 0; u < kGroup; ++u)
      if (r + u < rows) copy_async(smem_at(&ring[r / kGroup % (kAhead + 1)][u][threadIdx.x]), from + (r + u) * from_step);
    commit_async();
  };
#pragma unroll
  for (int g = 0; g < kAhead; ++g) fetch(g * kGroup);
#pragma unroll 1
  for (int32_t r = 0; r < rows; r += kGroup) {
    fetch(r + kAhead * kGroup);
    wait_async<kAhead>();
#pragma unroll
    for (int u = 0; u < kGroup; ++u) unpack8<E>(ring[r / kGroup % (kAhead + 1)][u][threadIdx.x], x[kPast + u]);
#pragma unroll
    for (int u = 0; u < kGroup; ++u)
      if (r + u < rows) row(u, reinterpret_cast<uint4*>(to + (r + u) * to_step));
#pragma unroll
    for (int j = 0; j < kPast; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[j][k] = x[j + kGroup][k];
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

// The recurrence as it stands, for sequences of up to by_token tokens and for shapes that the matrix form does not take.
// Bound by the state's bytes, read and written once: a row of N elements lies over kLanes lanes, 16 bytes each
// at least, and a lane has kRows rows, whose loads are all in flight at once; their sums y meet in one
// reduction that halves the rows at every step.  96 sequences of 16 heads of 128 x 128 (202 MB): 32.9 us, 6.1 TB/s.
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
  if (last - first > p.by_token) return;
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
  // many rows a lane for bandwidth, where that leaves a CTA for every SM; few for latency (16 heads of 128 x 128: one
  // sequence 2.9 us against 2.5, four 3.4 against 4.1, 64 22.9 against 27.2)
  const bool many = (int64_t)p.state.num_seqs * p.heads * p.head_dim >= (int64_t)num_sms * 4 * kSub * kMany;
  const int rows = 4 * kSub * (many ? kMany : kFew);
  const dim3 grid((p.head_dim + rows - 1) / rows, p.heads, p.state.num_seqs);
  return many ? launch_after(scan_kernel<E, N, kMany>, grid, 128, 0, s, p) : launch_after(scan_kernel<E, N, kFew>, grid, 128, 0, s, p);
}

template <class E>
cudaError_t scan(const ScanParams& p, int num_sms, cudaStream_t s) {
  switch (p.state_dim) {
    case 16: return scan<E, 16>(p, num_sms, s);
    case 32: return scan<E, 32>(p, num_sms, s);
    case 64: return scan<E, 64>(p, num_sms, s);
    case 128: return scan<E, 128>(p, num_sms, s);
    default: return scan<E, 256>(p, num_sms, s);
  }
}

}  // namespace

cudaError_t launch_conv(const ConvParams& p, int type, cudaStream_t s) {
  return type == KVX_TYPE_BF16 ? conv<Bf16>(p, s) : conv<Fp16>(p, s);
}

cudaError_t launch_scan(const ScanParams& p, int type, int num_sms, cudaStream_t s) {
  if (p.by_token >= 0) {
    const cudaError_t e = type == KVX_TYPE_BF16 ? scan<Bf16>(p, num_sms, s) : scan<Fp16>(p, num_sms, s);
    if (e != cudaSuccess) return e;
  }
  return p.segment ? launch_scan_chunks(p, type, s) : cudaSuccess;
}

}  // namespace kvx

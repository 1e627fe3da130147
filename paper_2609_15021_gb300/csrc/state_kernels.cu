// state_kernels.cu -- the recurrent layers' operators on their state slots: the
// short causal convolution and the selective scan.

#include "operators.cuh"

namespace kvx {
namespace {

// ---------------------------------------------------------------- convolution

// One thread per channel of a sequence, over its tokens.
template <class E>
__global__ void __launch_bounds__(256) conv_kernel(const __grid_constant__ ConvParams p) {
  using T = typename E::T;
  const int32_t c = blockIdx.x * 256 + threadIdx.x, s = blockIdx.y;
  if (c >= p.channels) return;
  const StateView& v = p.state;
  const T* in = reinterpret_cast<const T*>(slot_of(v, v.slots_in, s));
  T* keep = reinterpret_cast<T*>(slot_of(v, v.slots_out, s));
  int64_t first, last;
  rows_of(v, s, &first, &last);
  T* out = reinterpret_cast<T*>(p.out);
  if (!in || !keep) {
    for (int64_t t = first; t < last; ++t) out[t * p.out_stride + c] = E::down(0.f);
    return;
  }
  const int32_t past = p.width - 1;
  float w[4] = {}, x[4] = {};  // the window, x[3] the newest
  for (int j = 0; j < p.width; ++j) w[4 - p.width + j] = E::up(reinterpret_cast<const T*>(p.weight)[(int64_t)c * p.width + j]);
  const bool fresh = v.fresh && v.fresh[s];
  for (int j = 0; j < past; ++j) x[4 - past + j] = fresh ? 0.f : E::up(in[(int64_t)j * p.channels + c]);
  const float bias = p.bias ? E::up(reinterpret_cast<const T*>(p.bias)[c]) : 0.f;
  for (int64_t t = first; t < last; ++t) {
    x[0] = x[1], x[1] = x[2], x[2] = x[3];
    x[3] = E::up(reinterpret_cast<const T*>(p.x)[t * p.x_stride + c]);
    float y = bias + w[0] * x[0] + w[1] * x[1] + w[2] * x[2] + w[3] * x[3];
    if (p.silu) y = y / (1.f + expf(-y));
    out[t * p.out_stride + c] = E::down(y);
  }
  for (int j = 0; j < past; ++j) keep[(int64_t)j * p.channels + c] = E::down(x[4 - past + j]);
}

// ---------------------------------------------------------------- scan

__device__ __forceinline__ float step_of(const ScanParams& p, float raw, int32_t h) {
  if (p.dt_bias) raw += p.dt_bias[h];
  return p.softplus ? (raw > 20.f ? raw : log1pf(expf(raw))) : raw;
}

// A warp holds rows of one head's state, a lane 4 neighbouring elements (N / 32
// of them where N > 128), and walks the tokens.
template <class E, int N>
__global__ void __launch_bounds__(128) scan_kernel(const __grid_constant__ ScanParams p) {
  using T = typename E::T;
  constexpr int kVec = N >= 128 ? N / 32 : 4, kLanes = N / kVec, kRows = 32 / kLanes;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, col = (lane % kLanes) * kVec;
  const int32_t row = (blockIdx.x * 4 + (threadIdx.x >> 5)) * kRows + sub, h = blockIdx.y, s = blockIdx.z;
  const bool live = row < p.head_dim;
  const StateView& v = p.state;
  const float* in = reinterpret_cast<const float*>(slot_of(v, v.slots_in, s));
  float* keep = reinterpret_cast<float*>(slot_of(v, v.slots_out, s));
  int64_t first, last;
  rows_of(v, s, &first, &last);
  T* out = reinterpret_cast<T*>(p.out) + h * p.out_head + row;
  if (!in || !keep) {
    if (live && col == 0)
      for (int64_t t = first; t < last; ++t) out[t * p.out_token] = E::down(0.f);
    return;
  }
  const int64_t at = ((int64_t)h * p.head_dim + (live ? row : 0)) * N + col;
  const bool fresh = v.fresh && v.fresh[s];
  float state[kVec];
  for (int i = 0; i < kVec; ++i) state[i] = fresh ? 0.f : in[at + i];
  const float A = p.A[h], D = p.D ? p.D[h] : 0.f;
  const T* b = reinterpret_cast<const T*>(p.b) + (h / p.heads_per_group) * p.b_group + col;
  const T* c = reinterpret_cast<const T*>(p.c) + (h / p.heads_per_group) * p.c_group + col;
  for (int64_t t = first; t < last; ++t) {
    const float d = step_of(p, E::up(reinterpret_cast<const T*>(p.dt)[t * p.dt_token + h]), h);
    const float decay = expf(d * A);
    const float x = live ? E::up(reinterpret_cast<const T*>(p.x)[t * p.x_token + h * p.x_head + row]) : 0.f;
    float y = 0.f;
    for (int i = 0; i < kVec; ++i) {
      state[i] = state[i] * decay + d * x * E::up(b[t * p.b_token + i]);
      y += state[i] * E::up(c[t * p.c_token + i]);
    }
    for (int m = kLanes / 2; m; m >>= 1) y += __shfl_xor_sync(~0u, y, m);
    if (live && col == 0) out[t * p.out_token] = E::down(y + D * x);
  }
  if (live)
    for (int i = 0; i < kVec; ++i) keep[at + i] = state[i];
}

template <class E, int N>
cudaError_t scan(const ScanParams& p, cudaStream_t s) {
  constexpr int kRows = N >= 128 ? 1 : 128 / N;
  scan_kernel<E, N><<<dim3((p.head_dim + 4 * kRows - 1) / (4 * kRows), p.heads, p.state.num_seqs), 128, 0, s>>>(p);
  return cudaGetLastError();
}

template <class E>
cudaError_t scan(const ScanParams& p, cudaStream_t s) {
  switch (p.state_dim) {
    case 16: return scan<E, 16>(p, s);
    case 32: return scan<E, 32>(p, s);
    case 64: return scan<E, 64>(p, s);
    case 128: return scan<E, 128>(p, s);
    default: return scan<E, 256>(p, s);
  }
}

}  // namespace

cudaError_t launch_conv(const ConvParams& p, int type, cudaStream_t s) {
  const dim3 grid((p.channels + 255) / 256, p.state.num_seqs);
  if (type == KVX_TYPE_BF16)
    conv_kernel<Bf16><<<grid, 256, 0, s>>>(p);
  else
    conv_kernel<Fp16><<<grid, 256, 0, s>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_scan(const ScanParams& p, int type, cudaStream_t s) {
  return type == KVX_TYPE_BF16 ? scan<Bf16>(p, s) : scan<Fp16>(p, s);
}

}  // namespace kvx

// attend_kernels.cuh -- attention of each sequence's newest tokens over its pages.
//
//   s_j = scale q.k_j (capped, biased),  m = max s_j,  l = sum exp(s_j - m),
//   o = sum exp(s_j - m) v_j / l
//
// One pass over K and V with the running maximum and sum.  Every K/V row is read
// once and meets all rows of queries that share its head (group x new tokens), so
// the kernel is bound by the cache's bytes; the products are small matrix ones
// (16 query rows x 16 keys x head_dim), which mma.sync does at a few per cent of
// its rate.  What the kernel is built for is therefore bytes in flight:
//
//   * The work is cut into steps of 16 keys of one item (sequence, KV head, block
//     of query rows).  The grid's CTAs take equal runs of the steps of all items,
//     whatever the lengths, which are read on the device.  A run that covers only a
//     part of an item leaves its unnormalised sums in the workspace, and the CTA that
//     comes last to an item joins the parts, in their order.
//   * In a CTA, teams of kTiles warps (one for every 16 query rows) take the steps in
//     turn.  A team has a ring of its own in shared memory, filled by cp.async
//     from the pages' rows wherever they lie, and shares nothing with the others
//     until a piece ends, so there is no barrier over the CTA in the loop.
//   * 16-byte vectors of a row are permuted within 128 bytes by the row's number, so
//     ldmatrix reads eight rows without bank conflicts.
//
// An e4m3 cache is widened to fp16 between shared memory and the product, exactly;
// the queries then are fp16 too, each row scaled by a power of two, so that no bit of
// a bf16 value is lost within 2^-24 of the row's largest.  Probabilities are rounded to the cache's type (fp16
// for e4m3) for the product with V; the sums they are divided by are not.
#pragma once

#include <algorithm>
#include <type_traits>

#include "operators.cuh"

namespace kvx {
namespace {

constexpr int kStep = 16;          // keys of a step
constexpr int kRowTile = 16;       // query rows of a matrix instruction
constexpr int kAttendThreads = 128;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <class C, int kDim, int kTiles>
struct AttendShape {
  static constexpr int kElem = (int)sizeof(typename C::T);
  static constexpr int kRowBytes = kDim * kElem;
  static constexpr int kVecs = kRowBytes / 16;
  static constexpr int kTeams = kAttendThreads / 32 / kTiles;
  static constexpr int kStageBytes = 2 * kStep * kRowBytes;
  // two CTAs an SM, but one where four rings of 16 KB stages fill its shared memory
  static constexpr int kCtas = kTeams * kStageBytes > 48 * 1024 ? 1 : 2;
  static constexpr int kFit = (kCtas == 1 ? 192 : 96) * 1024 / (kTeams * kStageBytes);
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr bool kQueryInRegs = kDim <= 128;
  static constexpr int kRing = kTeams * kStages * kStageBytes;
  static constexpr int kQueryBytes = kQueryInRegs ? 0 : kTiles * kDim / 16 * 512;
  // the ring serves to join the teams' sums too: [team][tile][row][dim] and maxima and sums
  static constexpr int kJoin = kTeams * kTiles * kRowTile * (kDim + 2) * 4;
  static constexpr int kSmem = (kRing > kJoin ? kRing : kJoin) + kQueryBytes;
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit_async() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void wait_async() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

template <class C>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<C, Bf16>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two numbers in the type of the products (a: low half).
template <class C>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (std::is_same<C, Bf16>::value) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}
// Two e4m3 values (the low 16 bits) as fp16.
__device__ __forceinline__ uint32_t widen2(uint32_t v) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)v, __NV_E4M3);
  return (uint32_t)h.x | ((uint32_t)h.y << 16);
}

// Shared-memory offset of 16-byte vector `vec` of row `row`.
template <int kRowBytes>
__device__ __forceinline__ uint32_t vec_at(int row, int vec) {
  const int x = kRowBytes >= 128 ? row & 7 : (row >> 1) & 3;
  return row * kRowBytes + ((vec ^ x) << 4);
}

template <int kTiles>
__device__ __forceinline__ void team_sync(int team) {
  if constexpr (kTiles == 1)
    __syncwarp();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kTiles * 32) : "memory");
}

__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(~0u, v, 1));
  return fmaxf(v, __shfl_xor_sync(~0u, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor_sync(~0u, v, 1);
  return v + __shfl_xor_sync(~0u, v, 2);
}

// 16-key steps of a sequence, from the step that holds the first key any of its
// queries sees; *first: that step's first key.
__device__ __forceinline__ int32_t steps_of(const AttendParams& p, int32_t length, int32_t* first) {
  const int32_t lo = p.window > 0 ? max(0, length - p.new_tokens + 1 - p.window) : 0;
  *first = lo & ~(kStep - 1);
  return (length - *first + kStep - 1) / kStep;
}

// Sum over the CTA of one value a thread, to all.
__device__ __forceinline__ long long cta_sum(long long v, long long* buf) {
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < kAttendThreads / 32; ++i) v += buf[i];
  return v;
}

template <class Q>
__device__ __forceinline__ void write_out(const AttendParams& p, int32_t s, int32_t h, int32_t r, int32_t col, float v) {
  const int32_t t = r / p.group, head = h * p.group + r % p.group;
  const int64_t token = (int64_t)s * p.new_tokens + t;
  reinterpret_cast<typename Q::T*>(p.out + token * p.out_token + head * p.out_head)[col] = Q::down(v);
}
__device__ __forceinline__ void write_out(const AttendParams& p, int32_t s, int32_t h, int32_t r, int32_t col, float v) {
  if (p.type == KVX_TYPE_BF16)
    write_out<Bf16>(p, s, h, r, col, v);
  else
    write_out<Fp16>(p, s, h, r, col, v);
}

// Normalises a row's sums: m in powers of two, l and o relative to it.
__device__ __forceinline__ void write_lse(const AttendParams& p, int32_t s, int32_t h, int32_t r, float m, float l) {
  const int32_t t = r / p.group, head = h * p.group + r % p.group;
  const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
  if (p.lse) p.lse[((int64_t)s * p.new_tokens + t) * p.q_heads + head] = lse2 * kLn2;
  if (p.weights) p.row_lse2[((int64_t)s * p.pages.heads + h) * (p.group * p.new_tokens) + r] = lse2;
}
__device__ __forceinline__ float factor(float m, float top) {  // exp2(m - top), 0 for a part without a key
  return m == -INFINITY ? 0.f : exp2f(m - top);
}

template <class C, int kDim, int kTiles>
__global__ void __launch_bounds__(kAttendThreads, AttendShape<C, kDim, kTiles>::kCtas)
    attend_kernel(const __grid_constant__ AttendParams p) {
  using S = AttendShape<C, kDim, kTiles>;
  constexpr bool kWide = S::kElem == 1;  // cache to be widened
  constexpr int kKs = kDim / 16;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long buf[kAttendThreads / 32];
  __shared__ uint32_t masks[S::kTeams][S::kStages];
  __shared__ int32_t found[2];
  __shared__ int last_s;
  const PagesView& v = p.pages;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int team = warp / kTiles, tile = warp % kTiles, tlane = threadIdx.x % (32 * kTiles);
  const int quad = lane >> 2, sub = lane & 3;
  const int32_t rows = p.group * p.new_tokens;
  const int32_t blocks = (rows + kRowTile * kTiles - 1) / (kRowTile * kTiles);  // of query rows
  const int32_t per_seq = v.heads * blocks;                                    // items

  // All steps, and this CTA's run of them.
  long long total = 0;
  for (int32_t s = threadIdx.x; s < v.num_seqs; s += kAttendThreads) {
    int32_t first;
    if (blockIdx.x == 0) check_length(v, s);
    total += steps_of(p, length_of(v, s), &first);
  }
  total = cta_sum(total, buf) * per_seq;
  const long long ctas = min((long long)gridDim.x, max(1ll, (total + p.min_steps - 1) / p.min_steps));
  for (int32_t s = blockIdx.x; s < v.num_seqs; s += gridDim.x) {  // sequences without a key
    if (length_of(v, s) > 0) continue;
    for (int32_t i = threadIdx.x; i < v.heads * rows * v.head_dim; i += kAttendThreads) {
      const int32_t hr = i / v.head_dim;
      write_out(p, s, hr / rows, hr % rows, i % v.head_dim, 0.f);
      if (i % v.head_dim == 0) write_lse(p, s, hr / rows, hr % rows, 0.f, 0.f);
    }
  }
  if (blockIdx.x >= ctas) return;
  const long long begin = total * blockIdx.x / ctas, end = total * (blockIdx.x + 1) / ctas;

  // The sequence that `begin` lies in: every thread sums a sequence's steps, 128 at a time.
  int32_t seq = 0;
  long long seq_begin = 0;  // first step of `seq`'s items
  for (int32_t base = 0; base < v.num_seqs; base += kAttendThreads) {
    int32_t first;
    const int32_t s = base + threadIdx.x;
    const long long mine = s < v.num_seqs ? (long long)steps_of(p, length_of(v, s), &first) * per_seq : 0;
    long long before = mine;  // inclusive scan over the warp
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(~0u, before, d);
      if (lane >= d) before += y;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = before;
    __syncthreads();
    long long chunk = 0;
    for (int i = 0; i < kAttendThreads / 32; ++i) {
      if (i < warp) before += buf[i];
      chunk += buf[i];
    }
    const long long to = seq_begin + before, from = to - mine;
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    if (mine > 0 && begin >= from && begin < to) {
      found[0] = s;
      buf[0] = from;
    }
    __syncthreads();
    if (found[0] >= 0) {
      seq = found[0];
      seq_begin = buf[0];
      break;
    }
    seq_begin += chunk;
  }

  uint8_t* ring = smem + team * S::kStages * S::kStageBytes;
  const uint32_t ring_at = smem_at(ring);
  uint8_t* query_smem = smem + (S::kRing > S::kJoin ? S::kRing : S::kJoin);
  const int row_vecs = v.head_dim * S::kElem / 16;

  for (long long at = begin; at < end;) {
    // The piece: steps [i0, i1) of one item.
    int32_t first_key, length, steps;
    for (;;) {
      length = length_of(v, seq);
      steps = steps_of(p, length, &first_key);
      if (at < seq_begin + (long long)steps * per_seq) break;
      seq_begin += (long long)steps * per_seq;
      if (++seq >= v.num_seqs) return;  // lengths that changed under the kernel
    }
    const int32_t item = (int32_t)((at - seq_begin) / steps);
    const long long item_begin = seq_begin + (long long)item * steps;
    const int32_t i0 = (int32_t)(at - item_begin), i1 = (int32_t)min((long long)steps, end - item_begin);
    const int32_t h = item / blocks, row0 = (item % blocks) * (kRowTile * kTiles) + tile * kRowTile;
    const int32_t* table = v.tables + seq * v.table_stride;
    const uint8_t* head_base = v.base + h * v.head_bytes;

    // A step's rows: lane r (and r + 16) finds key r.
    auto look = [&](int32_t i) -> int64_t {
      const int32_t key = first_key + i * kStep + (lane & 15);
      return i < i1 && key < length ? row_offset(v, table, v.table_len, (uint32_t)key) : -1;
    };
    auto issue = [&](int32_t i, int64_t off, int stage) {
      if (i < i1) {
        const uint32_t mask = __ballot_sync(~0u, off >= 0) & 0xFFFFu;
        if (tlane == 0) masks[team][stage] = mask;
        const uint32_t dst = ring_at + stage * S::kStageBytes;
#pragma unroll
        for (int k = 0; k < 2 * kStep * S::kVecs / (32 * kTiles); ++k) {
          const int idx = k * 32 * kTiles + tlane, vec = idx % S::kVecs, row = idx / S::kVecs % kStep,
                    half = idx / S::kVecs / kStep;
          const int64_t o = __shfl_sync(~0u, off, row);
          const bool there = o >= 0 && vec < row_vecs;
          copy_async(dst + half * (kStep * S::kRowBytes) + vec_at<S::kRowBytes>(row, vec),
                     there ? head_base + o + half * v.half_bytes + vec * 16 : v.base, there ? 16 : 0);
        }
      }
      commit_async();
    };

    int64_t ahead[S::kStages];
#pragma unroll
    for (int k = 0; k < S::kStages; ++k) ahead[k] = look(i0 + team + k * S::kTeams);
#pragma unroll
    for (int k = 0; k < S::kStages; ++k) issue(i0 + team + k * S::kTeams, ahead[k], k);
    int64_t off_next = look(i0 + team + S::kStages * S::kTeams);

    // The queries, as the product's left factor: rows quad and quad + 8 of the tile, and what is
    // known of them.
    uint32_t qf[S::kQueryInRegs ? kKs : 1][4];
    float scale2[2], slope[2];
    int32_t pos[2];
    {
      const uint8_t* qrow[2];
      float top[2] = {0.f, 0.f}, shift[2] = {1.f, 1.f};
      for (int j = 0; j < 2; ++j) {
        const int32_t r = row0 + quad + 8 * j;
        const bool there = r < rows;
        const int32_t t = there ? r / p.group : 0, head = h * p.group + (there ? r % p.group : 0);
        qrow[j] = there ? p.q + ((int64_t)seq * p.new_tokens + t) * p.q_token + head * p.q_head : nullptr;
        pos[j] = there ? length - p.new_tokens + t : -1;
        slope[j] = there && p.slopes ? p.slopes[head] : 0.f;
      }
      auto load2 = [&](int j, int col) -> uint32_t {  // two raw neighbouring elements
        return qrow[j] && col < v.head_dim ? *reinterpret_cast<const uint32_t*>(qrow[j] + col * 2) : 0u;
      };
      auto wide = [&](uint32_t raw) -> float2 {
        if (p.type == KVX_TYPE_BF16)
          return make_float2(__uint_as_float(raw << 16), __uint_as_float(raw & 0xFFFF0000u));
        const __half2 hh = *reinterpret_cast<const __half2*>(&raw);
        return __half22float2(hh);
      };
      if constexpr (kWide) {
        for (int ks = 0; ks < kKs; ++ks)
          for (int e = 0; e < 4; ++e) {
            const float2 f = wide(load2(e & 1, ks * 16 + sub * 4 + (e >> 1) * 2));
            top[e & 1] = fmaxf(top[e & 1], fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        for (int j = 0; j < 2; ++j) {
          top[j] = quad_max(top[j]);
          // the largest to [2^10, 2^11): exponents only
          const int e = top[j] > 0.f && top[j] < INFINITY ? 10 - ilogbf(top[j]) : 0;
          shift[j] = ldexpf(1.f, max(-100, min(100, e)));
        }
      }
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks) {
        uint32_t f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (kWide) {  // the k index of a widened K: four neighbours of a lane
            const float2 x = wide(load2(e & 1, ks * 16 + sub * 4 + (e >> 1) * 2));
            f[e] = pack2<Fp16>(x.x * shift[e & 1], x.y * shift[e & 1]);
          } else {
            f[e] = load2(e & 1, ks * 16 + sub * 2 + (e >> 1) * 8);
          }
        }
        if constexpr (S::kQueryInRegs) {
#pragma unroll
          for (int e = 0; e < 4; ++e) qf[ks][e] = f[e];
        } else if (team == 0) {
          *reinterpret_cast<uint4*>(query_smem + ((tile * kKs + ks) * 32 + lane) * 16) = make_uint4(f[0], f[1], f[2], f[3]);
        }
      }
      for (int j = 0; j < 2; ++j) scale2[j] = p.scale * p.k_scale / shift[j];
      if constexpr (!S::kQueryInRegs) __syncthreads();
    }

    float acc[kDim / 8][4];
#pragma unroll
    for (int n = 0; n < kDim / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    const bool plain_scores = p.softcap == 0.f && !p.slopes;
    // keys below `all_from` or from `all_to` on are not seen by every row
    const int32_t all_to = length - p.new_tokens + 1, all_from = p.window > 0 ? length - p.window : INT32_MIN;
    float* scores = p.weights ? p.scores + ((int64_t)seq * v.heads + h) * rows * p.score_stride : nullptr;

    int stage = 0;
    for (int32_t i = i0 + team; i < i1; i += S::kTeams) {
      wait_async<S::kStages - 1>();
      team_sync<kTiles>(team);
      const uint32_t at_k = ring_at + stage * S::kStageBytes, at_v = at_k + kStep * S::kRowBytes;
      const uint32_t mask = masks[team][stage];
      const int32_t key0 = first_key + i * kStep;

      float sc[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks) {
        uint32_t a[4];
        if constexpr (S::kQueryInRegs) {
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] = qf[ks][e];
        } else {
          const uint4 x = *reinterpret_cast<const uint4*>(query_smem + ((tile * kKs + ks) * 32 + lane) * 16);
          a[0] = x.x, a[1] = x.y, a[2] = x.z, a[3] = x.w;
        }
        uint32_t b[4];
        if constexpr (!kWide) {
          load_matrices(b, at_k + vec_at<S::kRowBytes>((lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)));
          mma<C>(sc[0], a, b[0], b[1]);
          mma<C>(sc[1], a, b[2], b[3]);
        } else {
          static_assert(kKs % 2 == 0, "two vectors a load");
          if (ks % 2 == 0) {
            load_matrices(b, at_k + vec_at<S::kRowBytes>((lane & 7) + (((lane >> 3) & 1) << 3), ks + (lane >> 4)));
            uint32_t a2[4];
            if constexpr (S::kQueryInRegs) {
#pragma unroll
              for (int e = 0; e < 4; ++e) a2[e] = qf[ks + 1 < kKs ? ks + 1 : ks][e];
            } else {
              const uint4 x = *reinterpret_cast<const uint4*>(query_smem + ((tile * kKs + ks + 1) * 32 + lane) * 16);
              a2[0] = x.x, a2[1] = x.y, a2[2] = x.z, a2[3] = x.w;
            }
            mma<C>(sc[0], a, widen2(b[0] & 0xFFFF), widen2(b[0] >> 16));
            mma<C>(sc[1], a, widen2(b[1] & 0xFFFF), widen2(b[1] >> 16));
            mma<C>(sc[0], a2, widen2(b[2] & 0xFFFF), widen2(b[2] >> 16));
            mma<C>(sc[1], a2, widen2(b[3] & 0xFFFF), widen2(b[3] >> 16));
          }
        }
      }

      // Scores in powers of two; element e of tile n: row quad + 8 (e / 2), key 8n + 2 sub + e % 2.
      const bool whole = mask == 0xFFFFu && key0 + kStep <= all_to && key0 >= all_from;
      bool seen[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = e >> 1, k = 8 * n + 2 * sub + (e & 1);
          float x = sc[n][e] * scale2[j];
          if (!plain_scores) {
            // tanh y = 1 - 2 / (1 + e^2y): an absolute error of some 2^-22, which is what counts in an exponent
            if (p.softcap > 0.f) x = p.softcap * (1.f - 2.f / (1.f + exp2f(x * (2.f * kLog2e / p.softcap))));
            x += slope[j] * (key0 + k - pos[j]);
          }
          x *= kLog2e;
          seen[n][e] = whole || ((mask >> k & 1) && key0 + k <= pos[j] && (p.window == 0 || key0 + k > pos[j] - p.window));
          sc[n][e] = seen[n][e] ? x : -INFINITY;
        }
      if (scores) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int32_t r = row0 + quad + 8 * j;
          if (r < rows)
#pragma unroll
            for (int n = 0; n < 2; ++n)
              *reinterpret_cast<float2*>(scores + r * p.score_stride + key0 + 8 * n + 2 * sub) =
                  make_float2(sc[n][2 * j], sc[n][2 * j + 1]);
        }
      }

      float top[2], keep[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        top[j] = fmaxf(fmaxf(sc[0][2 * j], sc[0][2 * j + 1]), fmaxf(sc[1][2 * j], sc[1][2 * j + 1]));
        top[j] = fmaxf(m[j], quad_max(top[j]));
      }
      if (__any_sync(~0u, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          keep[j] = factor(m[j], top[j]);
          l[j] *= keep[j];
          m[j] = top[j];
        }
#pragma unroll
        for (int n = 0; n < kDim / 8; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[n][e] *= keep[e >> 1];
      }
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = e >> 1;
          sc[n][e] = exp2f(sc[n][e] - (m[j] == -INFINITY ? 0.f : m[j]));
          l[j] += sc[n][e];
        }
      const uint32_t pf[4] = {pack2<C>(sc[0][0], sc[0][1]), pack2<C>(sc[0][2], sc[0][3]), pack2<C>(sc[1][0], sc[1][1]),
                              pack2<C>(sc[1][2], sc[1][3])};

      // A value that is not finite must not reach the rows that do not see it (0 x inf): where a
      // step is not seen as a whole and holds such a value, its product is done element by element.
      bool odd = false;
      if (!whole) {
        for (int k = lane; k < kStep * S::kVecs; k += 32) {
          const uint4 x = *reinterpret_cast<const uint4*>(ring + stage * S::kStageBytes + kStep * S::kRowBytes + k * 16);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          for (int q = 0; q < 4; ++q) {
            if constexpr (kWide) {
              for (int b = 0; b < 32; b += 8) odd |= (w[q] >> b & 0x7F) == 0x7F;
            } else {
              constexpr uint32_t kInf = std::is_same<C, Bf16>::value ? 0x7F80u : 0x7C00u;
              odd |= (w[q] & kInf) == kInf || (w[q] >> 16 & kInf) == kInf;
            }
          }
        }
        odd = __any_sync(~0u, odd);
      }
      if (!odd) {
#pragma unroll
        for (int c = 0; c < kDim / 16; ++c) {
          uint32_t b[4];
          if constexpr (!kWide) {
            load_matrices_t(b, at_v + vec_at<S::kRowBytes>((lane & 7) + (((lane >> 3) & 1) << 3), c * 2 + (lane >> 4)));
            mma<C>(acc[2 * c], pf, b[0], b[1]);
            mma<C>(acc[2 * c + 1], pf, b[2], b[3]);
          } else if (c % 2 == 0) {
            // a transposed pair of bytes is two neighbouring dims of a key: even dims make one tile, odd ones another
            load_matrices_t(b, at_v + vec_at<S::kRowBytes>((lane & 7) + (((lane >> 3) & 1) << 3), c + (lane >> 4)));
#pragma unroll
            for (int q = 0; q < 4; ++q) b[q] = __byte_perm(b[q], 0, 0x3120);
            mma<C>(acc[2 * c], pf, widen2(b[0] & 0xFFFF), widen2(b[1] & 0xFFFF));
            mma<C>(acc[2 * c + 1], pf, widen2(b[0] >> 16), widen2(b[1] >> 16));
            mma<C>(acc[2 * c + 2], pf, widen2(b[2] & 0xFFFF), widen2(b[3] & 0xFFFF));
            mma<C>(acc[2 * c + 3], pf, widen2(b[2] >> 16), widen2(b[3] >> 16));
          }
        }
      } else {
        for (int k = 0; k < kStep; ++k) {
          const int from = (lane & ~3) | ((k & 7) >> 1);
          float pk[2];
          bool see[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float lo = k < 8 ? sc[0][2 * j] : sc[1][2 * j], hi = k < 8 ? sc[0][2 * j + 1] : sc[1][2 * j + 1];
            const bool slo = k < 8 ? seen[0][2 * j] : seen[1][2 * j], shi = k < 8 ? seen[0][2 * j + 1] : seen[1][2 * j + 1];
            pk[j] = __shfl_sync(~0u, k & 1 ? hi : lo, from);
            see[j] = __shfl_sync(~0u, (int)(k & 1 ? shi : slo), from);
          }
#pragma unroll
          for (int n = 0; n < kDim / 8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int col = kWide ? (n >> 1) * 16 + sub * 4 + 2 * e + (n & 1) : n * 8 + sub * 2 + e;
              const uint8_t* at_e = ring + stage * S::kStageBytes + kStep * S::kRowBytes +
                                    vec_at<S::kRowBytes>(k, col * S::kElem / 16) + col * S::kElem % 16;
              const float x = C::up(*reinterpret_cast<const typename C::T*>(at_e));
              if (see[0]) acc[n][e] += pk[0] * x;
              if (see[1]) acc[n][2 + e] += pk[1] * x;
            }
        }
      }
      team_sync<kTiles>(team);
      issue(i + S::kStages * S::kTeams, off_next, stage);
      off_next = look(i + (S::kStages + 1) * S::kTeams);
      stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }
    wait_async<0>();
    __syncthreads();

    // The teams' sums joined in shared memory, then written: normalised if the piece is the item.
    float* sums = reinterpret_cast<float*>(smem);
    float* stats = sums + S::kTeams * kTiles * kRowTile * kDim;  // [team][tile][row][m, l]
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float whole_l = quad_sum(l[j]);
      const int r = (team * kTiles + tile) * kRowTile + quad + 8 * j;
      if (sub == 0) {
        stats[2 * r] = m[j];
        stats[2 * r + 1] = whole_l;
      }
#pragma unroll
      for (int n = 0; n < kDim / 8; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = kWide ? (n >> 1) * 16 + sub * 4 + 2 * e + (n & 1) : n * 8 + sub * 2 + e;
          sums[r * kDim + col] = acc[n][2 * j + e];
        }
    }
    __syncthreads();
    const int32_t block_row = (item % blocks) * (kRowTile * kTiles);
    const int32_t here = min(rows - block_row, kRowTile * kTiles);  // rows of this block
    const bool whole_item = i0 == 0 && i1 == steps;
    float* part = nullptr;
    if (!whole_item)
      part = p.parts + ((long long)blockIdx.x * 2 + (begin < item_begin)) * (kRowTile * kTiles * (kDim + 2));
    for (int idx = threadIdx.x; idx < here * kDim; idx += kAttendThreads) {
      const int r = idx / kDim, col = idx % kDim;
      float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
      for (int g = 0; g < S::kTeams; ++g) top = fmaxf(top, stats[2 * (g * kTiles * kRowTile + r)]);
#pragma unroll
      for (int g = 0; g < S::kTeams; ++g) {
        const int gr = g * kTiles * kRowTile + r;
        const float f = factor(stats[2 * gr], top);
        sum += f * stats[2 * gr + 1];
        o += f * sums[gr * kDim + col];
      }
      if (whole_item) {
        if (col < v.head_dim) write_out(p, seq, h, block_row + r, col, sum == 0.f ? 0.f : o / sum * p.v_scale);
        if (col == 0) write_lse(p, seq, h, block_row + r, top, sum);
      } else {
        __stcg(part + r * kDim + col, o);
        if (col == 0) {
          __stcg(part + kRowTile * kTiles * kDim + 2 * r, top);
          __stcg(part + kRowTile * kTiles * kDim + 2 * r + 1, sum);
        }
      }
    }
    if (!whole_item) {
      // The CTAs that this item's steps fall to, in order; the one that comes last joins their parts.
      const long long item_end = item_begin + steps;
      const long long c0 = ((item_begin + 1) * ctas + total - 1) / total - 1, c1 = (item_end * ctas + total - 1) / total - 1;
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        int32_t* counter = p.counters + (long long)seq * per_seq + item;
        const int32_t all = (int32_t)(c1 - c0 + 1);
        last_s = atomicAdd(counter, 1) == all - 1;
        if (last_s) {
          __stcg(counter, 0);  // as the next call wants it
          __threadfence();
        }
      }
      __syncthreads();
      if (last_s) {
        for (int idx = threadIdx.x; idx < here * kDim; idx += kAttendThreads) {
          const int r = idx / kDim, col = idx % kDim;
          float top = -INFINITY, sum = 0.f, o = 0.f;
          for (long long c = c0; c <= c1; ++c) {
            const float* from = p.parts + (c * 2 + (total * c / ctas < item_begin)) * (kRowTile * kTiles * (kDim + 2));
            const float pm = __ldcg(from + kRowTile * kTiles * kDim + 2 * r);
            const float pl = __ldcg(from + kRowTile * kTiles * kDim + 2 * r + 1);
            const float po = __ldcg(from + r * kDim + col);
            const float now = fmaxf(top, pm), f0 = factor(top, now), f1 = factor(pm, now);
            sum = sum * f0 + pl * f1;
            o = o * f0 + po * f1;
            top = now;
          }
          if (col < v.head_dim) write_out(p, seq, h, block_row + r, col, sum == 0.f ? 0.f : o / sum * p.v_scale);
          if (col == 0) write_lse(p, seq, h, block_row + r, top, sum);
        }
      }
    }
    __syncthreads();
    at = item_begin + i1;
  }
}

// f(kernel, shape) for every form of the kernel over a cache of type C.
template <class C, class F>
cudaError_t for_each_attend(F&& f) {
  cudaError_t e;
  if ((e = f(attend_kernel<C, 64, 1>, AttendShape<C, 64, 1>())) != cudaSuccess) return e;
  if ((e = f(attend_kernel<C, 64, 2>, AttendShape<C, 64, 2>())) != cudaSuccess) return e;
  if ((e = f(attend_kernel<C, 128, 1>, AttendShape<C, 128, 1>())) != cudaSuccess) return e;
  if ((e = f(attend_kernel<C, 128, 2>, AttendShape<C, 128, 2>())) != cudaSuccess) return e;
  if ((e = f(attend_kernel<C, 256, 1>, AttendShape<C, 256, 1>())) != cudaSuccess) return e;
  return f(attend_kernel<C, 256, 2>, AttendShape<C, 256, 2>());
}

template <class C>
cudaError_t prepare() {
  return for_each_attend<C>([](auto kernel, auto shape) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, decltype(shape)::kSmem);
  });
}

// The grid: as many CTAs as are resident, or as many runs of min_steps as there may be.
template <class C, int kDim, int kTiles>
cudaError_t attend(const AttendParams& p, int num_sms, cudaStream_t s) {
  using S = AttendShape<C, kDim, kTiles>;
  const int grid = (int)std::min<int64_t>((int64_t)num_sms * S::kCtas, std::max<int64_t>(1, p.most_steps / p.min_steps));
  attend_kernel<C, kDim, kTiles><<<grid, kAttendThreads, S::kSmem, s>>>(p);
  return cudaGetLastError();
}

template <class C, int kDim>
cudaError_t attend(const AttendParams& p, int num_sms, cudaStream_t s) {
  return attend_tiles(p) == 1 ? attend<C, kDim, 1>(p, num_sms, s) : attend<C, kDim, 2>(p, num_sms, s);
}

template <class C>
cudaError_t attend(const AttendParams& p, int num_sms, cudaStream_t s) {
  const int pad = attend_pad(p.pages.head_dim);
  return pad == 64 ? attend<C, 64>(p, num_sms, s) : pad == 128 ? attend<C, 128>(p, num_sms, s) : attend<C, 256>(p, num_sms, s);
}

}  // namespace
}  // namespace kvx

// operators.cuh -- what the operators' kernels share: a batch's view of one
// layer's pages, element types, and the launchers operators.cu calls.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kvx_internal.h"

namespace kvx {

// Division of numbers n < 2^31 by d >= 1: with 2^(l-1) < d <= 2^l and m = ceil(2^(31+l) / d), n / d is
// floor(n m / 2^(31+l)), as m is too large by less than 1 and n < 2^31 (Granlund, Montgomery, "Division by
// invariant integers using multiplication", 1994).
struct Div31 {
  uint32_t d, m, shift;  // shift: l - 1, the high word's
};
inline Div31 div31(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return {d, d > 1 ? (uint32_t)(((1ull << (31 + l)) + d - 1) / d) : 0, l ? l - 1 : 0};
}

// One layer's pages as a batch's block tables name them.
struct PagesView {
  uint8_t* base;
  const int32_t* tables;
  const int32_t* lengths;
  long long* err;
  int64_t table_stride;
  int64_t half_bytes;               // K half of a page; the V half follows
  int64_t head_bytes;               // from a head of a page half to the next
  int64_t row_bytes;
  // Head 0's K row of a token has, of its layer's rows, the number page * page_rows + slot * token_rows.
  uint32_t page_rows, token_rows;
  Div31 by_block, by_pack;          // tokens per page, pages per logical block
  uint32_t entries;                 // valid table entries are below this
  uint32_t table_len;
  int32_t heads, head_dim, num_seqs;
  int32_t max_length;               // longer sequences count as this
};

struct AppendParams {
  PagesView pages;
  const uint8_t *key, *value;
  const int32_t* starts;
  int64_t tokens;
  int64_t key_token, key_head, value_token, value_head;  // strides in bytes
  int32_t new_tokens, num_seqs;
  Div31 row_vecs;  // 16-byte vectors of a cached row
  float k_scale, v_scale;
};

struct RotaryParams {
  AppendParams append;
  const uint8_t *q, *q_weight, *k_weight;
  uint8_t* q_out;
  const float* inv_freq;
  const int32_t* positions;
  int64_t q_token, q_head, out_token, out_head;  // strides in bytes
  int32_t q_heads, rotary_dim, interleaved;
  float rotary_scale, eps, weight_offset;
  float inverse_dim;  // 1 / head_dim
  int32_t parts;      // warps of a token
};

struct BoundsParams {
  PagesView pages;
  int8_t* boxes;
  float* sizes;
  int32_t new_tokens, pages_each;  // pages_each: that a sequence's new tokens may lie in
  Div31 by_heads;
};

struct SelectParams {
  PagesView pages;  // base is not used
  const int8_t* boxes;
  const float* sizes;
  const uint8_t* q;
  int32_t* selected;
  int64_t q_token, q_head;  // strides in bytes
  int32_t q_heads, group, new_tokens, budget, sinks, recent;
  float* scores;            // workspace: [query][head][score_stride]
  int64_t score_stride;
  int32_t tokens_each;      // new tokens whose rows a CTA scores at once
  int32_t score_tiles, score_parts;  // of a sequence: of pages, and of new tokens
};
// A CTA of the scores has 128 pages and at most so many rows of queries, but always all of a head's group.
constexpr int32_t kScoreRows = 64, kMaxScoreGroup = 128, kScorePages = 128;
inline int32_t score_tokens(int32_t group, int32_t new_tokens) {
  return group >= kScoreRows ? 1 : kScoreRows / group < new_tokens ? kScoreRows / group : new_tokens;
}

struct AttendParams {
  PagesView pages;
  const uint8_t* q;
  uint8_t* out;
  float *lse, *weights;
  const float* slopes;
  int64_t q_token, q_head, out_token, out_head;  // strides in bytes
  int64_t weights_seq, weights_head;             // strides in elements
  int32_t type, q_heads, group, new_tokens, window;
  float scale, softcap, k_scale, v_scale;
  int64_t most_steps;     // that the batch's items may count for together
  int32_t min_steps;      // the least a CTA is started for
  // workspace
  int2* items;            // [item]: its first part and their number, 0 where there are none
  float* parts;           // [CTA][2][rows of a block][head_dim and 2]: sums of pieces of items
  int32_t part_rows, part_dim;
  float *row_lse2;        // [sequence][head][row], with weights only
  float* scores;          // [sequence][head][score_stride keys][score_rows], with weights only
  int64_t score_stride;
  int32_t score_rows;     // query rows of a head, made even
  // attention over selected pages: pages.num_seqs counts queries then, by_query of them a sequence, and new_tokens is 1
  const int32_t* selected;  // [query][head][budget], or null
  int32_t budget;
  Div31 by_query;
};
// Elements of a row in shared memory, and tiles of 8 query rows that a warp takes at once: what its
// registers hold of sums (at most 4, 3 for rows of 256); more rows are blocks of their own.
inline int attend_pad(int32_t head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }
inline int attend_tiles(int32_t head_dim, int32_t rows) {
  const int most = head_dim > 128 ? 3 : 4, tiles = (rows + 7) / 8, blocks = (tiles + most - 1) / most;
  const int each = (tiles + blocks - 1) / blocks;
  return each == 3 && most == 4 ? 4 : each;
}

// 16-key blocks that a step of the attention takes: two where a warp's sums leave the registers for them and a step's
// rows half of a warp's shared memory (45 sequences of up to 16k tokens, rows of 96 in fp16: 60 us, 75 with one).
constexpr int attend_blocks(int pad, int elem, int tiles) { return tiles == 1 && pad * elem <= 256 ? 2 : 1; }

// What beginning and ending an item of the attention takes, in steps: the 45 sequences took 88 us at 6, 68 at 9, 61 at 12
// and 63 at 16.
constexpr int kItemSteps = 12;

struct EvictParams {
  PagesView pages;                // base is not used
  uint8_t* layer_base[KVX_MAX_LAYERS];
  const float* weights;
  const int32_t* new_tables;
  int32_t *kept, *new_lengths;
  float* new_weights;
  int64_t weights_layer, weights_seq, weights_head;              // strides in elements
  int64_t new_weights_layer, new_weights_seq, new_weights_head;
  int64_t new_table_stride;
  uint32_t new_table_len;
  int32_t budget, sinks, recent, num_layers;
  Div31 row_vecs;  // 16-byte vectors of a row
  int32_t units;   // of 32 kept tokens, of a row of weights
};
static_assert(sizeof(EvictParams) <= 4096, "kernel parameters");

struct StateView {
  uint8_t* base;
  const int32_t *slots_in, *slots_out, *fresh, *starts;
  long long* err;
  int64_t num_slots, slot_bytes, offset;  // offset: of the part the kernel works on
  int64_t tokens;
  int32_t num_seqs;
};

struct ConvParams {
  StateView state;
  const uint8_t *x, *weight, *bias;
  uint8_t* out;
  int64_t x_stride, out_stride;  // in elements
  int32_t channels, width, silu;
};

struct ScanParams {
  StateView state;
  const uint8_t *x, *dt, *b, *c;
  uint8_t* out;
  const float *A, *D, *dt_bias;
  int64_t x_token, x_head, dt_token, b_token, b_group, c_token, c_group, out_token, out_head;  // in elements
  int32_t heads, head_dim, state_dim, heads_per_group, softplus;
  int32_t segment;           // tokens of a segment in the matrix form; 0: no sequence takes it
  int32_t pieces;            // scan_pieces of it
  int32_t by_token;          // sequences of up to so many tokens go token by token; -1: none
  float* segment_states;     // [piece][head][head_dim][state_dim], where sequences are cut into segments
  float* segment_exponents;  // [piece][head]
  long long wait_cycles;     // limit of a wait for the tensor cores
  int* timeout;              // set when one ran out
  bool stall;                // fault point "scan_wait": the first chunk's products are not announced
};
struct DeltaParams {
  StateView state;
  const uint8_t *q, *k, *v, *dt, *beta;
  uint8_t* out;
  const float *A, *dt_bias;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, dt_token, beta_token, out_token, out_head;  // in elements
  int32_t heads, head_dim, state_dim, heads_per_group, groups, softplus, sigmoid, normalize;
  float scale, eps;
  int32_t by_token;          // sequences of up to so many tokens go token by token, the others by chunks; -1: none
  int32_t long_seqs;         // sequences that may go by chunks
  int32_t pieces;            // room for chunks; 0: no sequence goes by chunks
  int32_t token_ctas;        // of the first kernel, of sequences that go token by token
  uint8_t* rows_space;       // workspace: a chunk's and group's keys and queries
  uint8_t* head_space;       // and what else a chunk and head has
  long long wait_cycles;     // limit of a wait for a copy
  int* timeout;              // set when one ran out
  int32_t stall;             // fault points: 1, "delta_wait", the second chunk's copies are not made; 2, "delta_wait_m", the first one's M is not
};
constexpr int32_t kDeltaChunk = 64, kDeltaHeadBytes = 21888;  // tokens; bytes of head_space
// Whether a batch's sequences go by chunks, and which do not (*by_token).
bool delta_by_chunks(int64_t tokens, int32_t num_seqs, bool packed, int32_t state_dim, int32_t* by_token);
// Pieces that the workspace has room for: as many as sequences whose rows do not overlap can have.  No more than there are
// SMs and sequences, where sequences are cut.
inline int64_t scan_pieces(const StateView& v, int32_t segment) { return v.tokens / segment + v.num_seqs; }
// The segment of the matrix form for a batch, 0 where it is not used; *cut: whether a sequence may have several;
// *by_token: up to how many tokens a sequence does not take it.
int32_t scan_segment(const StateView& v, int32_t heads, int32_t head_dim, int32_t state_dim, int num_sms, bool* cut,
                     int32_t* by_token);

cudaError_t launch_append(const AppendParams& p, int type, int cache_type, int num_sms, cudaStream_t s);
cudaError_t launch_attend(const AttendParams& p, int cache_type, int num_sms, cudaStream_t s);
cudaError_t launch_attend_bf16(const AttendParams& p, int num_sms, cudaStream_t s);
cudaError_t launch_attend_fp16(const AttendParams& p, int num_sms, cudaStream_t s);
cudaError_t launch_attend_e4m3(const AttendParams& p, int num_sms, cudaStream_t s);
cudaError_t prepare_attend_bf16();
cudaError_t prepare_attend_fp16();
cudaError_t prepare_attend_e4m3();
cudaError_t launch_attend_selected_bf16(const AttendParams& p, int num_sms, cudaStream_t s);
cudaError_t launch_attend_selected_fp16(const AttendParams& p, int num_sms, cudaStream_t s);
cudaError_t launch_attend_selected_e4m3(const AttendParams& p, int num_sms, cudaStream_t s);
cudaError_t prepare_attend_selected_bf16();
cudaError_t prepare_attend_selected_fp16();
cudaError_t prepare_attend_selected_e4m3();
cudaError_t launch_rotary(const RotaryParams& p, int type, int cache_type, int num_sms, cudaStream_t s);
cudaError_t launch_bounds(const BoundsParams& p, int cache_type, cudaStream_t s);
cudaError_t launch_select(const SelectParams& p, int type, cudaStream_t s);
cudaError_t launch_evict(const EvictParams& p, cudaStream_t s);
cudaError_t launch_conv(const ConvParams& p, int type, cudaStream_t s);
cudaError_t launch_scan(const ScanParams& p, int type, int num_sms, cudaStream_t s);
cudaError_t launch_delta(const DeltaParams& p, int type, int num_sms, cudaStream_t s);
cudaError_t launch_delta_chunks(const DeltaParams& p, int type, cudaStream_t s);
cudaError_t launch_scan_chunks(const ScanParams& p, int type, cudaStream_t s);

#ifdef __CUDACC__
namespace {

// A kernel that is launched while the one before it in the stream still runs, and waits for its end
// (wait_for_previous, its first statement) before it touches memory: only the launch itself overlaps.  It lets its own
// successor start after that wait, so a kernel of a call may read before its own wait what was there before the call's
// kernel in front of it began.
template <class P>
cudaError_t launch_after(void (*kernel)(P), dim3 grid, int threads, size_t smem, cudaStream_t s, const P& p) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = grid;
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = smem;
  c.stream = s;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, p);
}
__device__ __forceinline__ void wait_for_previous() {
  asm volatile("griddepcontrol.wait;\n griddepcontrol.launch_dependents;" ::: "memory");
}

struct Bf16 {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float up(T v) { return __bfloat162float(v); }
  static __device__ __forceinline__ T down(float v) { return __float2bfloat16_rn(v); }
};
struct Fp16 {
  using T = __half;
  static __device__ __forceinline__ float up(T v) { return __half2float(v); }
  static __device__ __forceinline__ T down(float v) { return __float2half_rn(v); }
};
struct E4m3 {
  using T = __nv_fp8_e4m3;
  static __device__ __forceinline__ float up(T v) { return (float)v; }
};

__device__ __forceinline__ uint32_t quotient(const Div31& f, uint32_t n) {
  return f.d > 1 ? __umulhi(f.m, n) >> f.shift : n;
}

// Tokens that sequence `s` holds, between 0 and max_length.
__device__ __forceinline__ int32_t length_of(const PagesView& v, int32_t s) {
  return min(max(v.lengths[s], 0), v.max_length);
}

constexpr uint32_t kNoRow = UINT32_MAX;
// Number in the layer's rows of head 0's K row at `pos`, or kNoRow for a table entry that
// names no page (reported as its logical block).
__device__ __forceinline__ uint32_t row_index(const PagesView& v, const int32_t* table, uint32_t table_len, uint32_t pos) {
  const uint32_t page = quotient(v.by_block, pos), slot = pos - page * v.by_block.d;
  const uint32_t block = quotient(v.by_pack, page), sub = page - block * v.by_pack.d;
  const uint32_t entry = block < table_len ? (uint32_t)__ldg(table + block) : UINT32_MAX;
  if (entry >= v.entries) {
    atomicMin(v.err, (long long)block);
    return kNoRow;
  }
  return (entry * v.by_pack.d + sub) * v.page_rows + slot * v.token_rows;
}

// Reports a length outside [0, max_length] (one thread of a launch calls it per sequence).
__device__ __forceinline__ void check_length(const PagesView& v, int32_t s) {
  const int32_t n = v.lengths[s];
  if (n < 0 || n > v.max_length) atomicMin(v.err, (long long)v.table_len);
}

// Slot i, sequence s's, or null (and reported) where it is out of range.
__device__ __forceinline__ uint8_t* slot_at(const StateView& v, int32_t i, int32_t s) {
  if (i < 0 || i >= v.num_slots) {
    atomicMin(v.err, (long long)s);
    return nullptr;
  }
  return v.base + (int64_t)i * v.slot_bytes + v.offset;
}
__device__ __forceinline__ uint8_t* slot_of(const StateView& v, const int32_t* slots, int32_t s) { return slot_at(v, slots[s], s); }

// Rows of sequence s, cut to the rows there are (a pair of starts that does not ascend within them is reported).
__device__ __forceinline__ void rows_of(const StateView& v, int32_t s, int64_t* first, int64_t* last) {
  if (!v.starts) {
    *first = s;
    *last = s + 1;
    return;
  }
  const int32_t from = v.starts[s], to = v.starts[s + 1];
  if (from < 0 || to < from || to > v.tokens) atomicMin(v.err, (long long)s);
  *first = min((int64_t)max(from, 0), v.tokens);
  *last = max(*first, min((int64_t)to, v.tokens));
}

}  // namespace
#endif

}  // namespace kvx

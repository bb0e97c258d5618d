// Shared by the serving kernels (paged_cache.hip, attention_paged.hip): storage types, division by a
// number that the host knows, and the search for a row's sequence.
#pragma once

#include "sga_internal.h"

namespace sga {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;
template <typename T, int N>
using vec_t = T __attribute__((ext_vector_type(N)));

// n / v for 0 <= n < 2^31 by one multiplication: (umulhi(n, mul) + n) >> shift.
struct FastDiv {
  uint32_t value, mul, shift;
};
inline FastDiv fast_div(uint32_t v) {
  uint32_t s = 0;
  while (s < 31 && (uint32_t(1) << s) < v) ++s;
  const uint64_t m = ((uint64_t(1) << 32) * ((uint64_t(1) << s) - v)) / v + 1;
  return {v, (uint32_t)m, s};
}
__host__ __device__ __forceinline__ uint32_t quotient(uint32_t n, const FastDiv& f) {
  return (uint32_t)((((uint64_t)n * f.mul) >> 32) + n) >> f.shift;
}

// A call's batch as the kernels take it (sga_paged_batch).
struct PagedArgs {
  const int32_t* page_table;
  const int64_t* seq_ptr;
  const int32_t* seq_len;
  int64_t page_stride;      // elements
  uint32_t n_pages;
  int32_t n_seqs, n_tokens, pages_per_seq;
  FastDiv page;
};

// seq_ptr[s], kept inside the packed rows whatever the array holds.
__device__ __forceinline__ int32_t row_of_sequence(const PagedArgs& b, int32_t s) {
  const int64_t p = b.seq_ptr[s];
  return (int32_t)(p < 0 ? 0 : p < b.n_tokens ? p : b.n_tokens);
}

// The largest s in [0, n) with first(s) <= x (0 if none), first non-decreasing: the wavefront's lanes ask at 64 places
// at a time, so that up to 64 sequences cost one load's latency and 4,096 two.  All lanes call it.
template <typename First>
__device__ __forceinline__ int32_t last_not_above(int32_t n, int64_t x, First first) {
  const int lane = threadIdx.x & (kWave - 1);
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const int32_t step = (hi - lo - 1) / kWave + 1;
    const int64_t at = (int64_t)lo + (int64_t)lane * step;
    const int n_below = __popcll(__ballot(at < hi && first((int32_t)(at < hi ? at : hi - 1)) <= x));
    lo += (n_below > 0 ? n_below - 1 : 0) * step;
    hi = hi - lo < step ? hi : lo + step;
  }
  return lo;
}

struct RotaryArgs {
  const double* frequencies;
  float magnitude;
  int32_t channels;
  int32_t interleaved;
  int32_t inverse;
};

// One tensor that passes through the rotation kernel: strides in elements.
struct RowsArg {
  const void* src;
  void* dst;                 // cache: its start; rows: their tensor
  int64_t src_head, src_row, dst_head, dst_row;
  int32_t heads;
  int32_t rotate;
  int32_t paged;
};

struct RotateArgs {
  RowsArg tensor[3];
  int32_t n_tensors;
  int32_t n_rows, d;
  const int64_t* positions;
  int64_t first;
  RotaryArgs rotary;
  PagedArgs batch;           // page_table null: no batch
  int32_t dtype;
  hipStream_t stream;
};
sga_status launch_rotate(const RotateArgs& a);

constexpr size_t kNoteBytes = 32;          // (see Note in attention_paged.hip)

struct PagedAttention {
  const void* Q;
  void* O;
  const void* cache_k;
  const void* cache_v;
  float* lse;
  int64_t q_head, q_row, o_head, o_row;     // elements
  PagedArgs batch;
  int32_t Hq, Hkv;
  FastDiv group;             // Hq / Hkv
  int32_t L, window, n_global, causal;
  float scale;
  uint32_t page_pieces;      // 16-byte pieces from page to page
  float* partials;           // partial states of tiles that are cut; null: none is
  void* notes;               // ... and what is to be joined, one for each workgroup, ahead of them
  int32_t tile_rows, groups, splits, slots;      // the plan's
  int32_t d, dtype;
  hipStream_t stream;
};
// The kernel, the workgroups and the partial states of a call.
struct PagedPlan {
  int32_t tile_rows;         // rows of a tile: which kernel takes the call
  int32_t groups;            // workgroups (tiles of 16 rows: each with an equal share of the work); 0: the call is too large
  int32_t slots, splits;     // tiles of 128 rows: pieces of a key head at most, and more than 1 if tiles may be cut
  size_t bytes;
};
PagedPlan plan_paged(const PagedAttention& a);
sga_status launch_paged(const PagedAttention& a);

}  // namespace sga

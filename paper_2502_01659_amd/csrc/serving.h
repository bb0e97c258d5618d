// Shared by the serving kernels (paged_cache.hip, norm_rotary.hip, drafts.hip, attention_paged.hip): storage types, division by a
// number that the host knows, the search for a row's sequence, and the sines of a position.
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

// cos t and sin t for t = position * f.  The product is held as a rounded part and its error, and multiples of pi / 2
// are taken off in 64 bits (pi / 2 as the sum of two numbers, 2^-107 off), twice: the first time about as many as the rounded part has, whose
// step alone is many turns at far positions, the second time what that and the product's error leave.  Up to |t| = 2^62 the rest
// is within pi / 4 and good to 2^-40; rounded to 32 bits it is within 2^-25, and the Taylor polynomials of degree 9 and 10 are within 2e-9 there.
__device__ __forceinline__ float2 turn_of(int64_t position, double f) {
  constexpr double kQuarters = 0.63661977236758134308, kHigh = 1.57079632679489655800, kLow = 6.12323399573676603587e-17;
  const double p = (double)position;
  const double x = p * f, x_low = __builtin_fma(p, f, -x);
  const double n = __builtin_rint(x * kQuarters);
  double r = __builtin_fma(-n, kHigh, x);
  r = __builtin_fma(-n, kLow, r) + x_low;
  const double rest = __builtin_rint(r * kQuarters);
  r = __builtin_fma(-rest, kHigh, r);
  r = __builtin_fma(-rest, kLow, r);
  const int quarter = (int)(((int64_t)n + (int64_t)rest) & 3);
  const float y = (float)r, z = y * y;
  float s = 2.7557319224e-6f, c = -2.7557319224e-7f;
  s = fmaf(s, z, -1.9841269841e-4f);
  s = fmaf(s, z, 8.3333333333e-3f);
  s = fmaf(s, z, -1.6666666667e-1f);
  s = fmaf(s * z, y, y);
  c = fmaf(c, z, 2.4801587302e-5f);
  c = fmaf(c, z, -1.3888888889e-3f);
  c = fmaf(c, z, 4.1666666667e-2f);
  c = fmaf(c, z, -0.5f);
  c = fmaf(c, z, 1.0f);
  const float cos_t = (quarter & 1) ? s : c, sin_t = (quarter & 1) ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -cos_t : cos_t, quarter >= 2 ? -sin_t : sin_t);
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

// Norm of every head's row before it turns.
struct NormArg {
  const void* weight;        // null: all 1
  float epsilon, offset;
  int32_t dtype;             // the weight's
  int32_t on;
};
struct NormRotateArgs {
  RotateArgs r;
  NormArg norm[3];           // r.tensor's
  const int32_t* depth;      // a draft tree's depths: positions count from the sequence's first new token; null: a row's own place
};
sga_status launch_norm_rotate(const NormRotateArgs& a);

// One tensor of the backward pass.
struct NormGradRows {
  const void *x, *g;
  void* dx;
  int64_t x_head, x_row, g_head, g_row, dx_head, dx_row;
  float* dw;                 // null: not asked for
  NormArg norm;
  int32_t heads;
};
struct NormGradArgs {
  NormGradRows tensor[2];
  int32_t n_tensors, n_rows, d;
  const int64_t* positions;
  int64_t first;
  RotaryArgs rotary;         // inverse
  float* partials;           // [workgroups][d], null: no dw is asked for
  int32_t dtype;
  hipStream_t stream;
};
size_t norm_partial_bytes(int64_t n_rows, int32_t Hq, int32_t Hkv, int32_t d);
sga_status launch_norm_grad(const NormGradArgs& a);

// The next step's pages (sga_pages_advance).
struct PagesArgs {
  PagedArgs from;                    // as it was
  int32_t* page_table;               // as it becomes (may be the same arrays)
  int64_t* seq_ptr;
  int32_t* seq_len;
  int32_t* ring;
  const int64_t* state;
  int64_t* state_out;
  const int32_t* ask;
  const int32_t* kept;               // null: all rows are
  int64_t *positions, *slots;        // null: not asked for
  int32_t give_back, window, n_global;     // give_back: pages behind the window go back
  int32_t segments, per_segment;     // wavefronts of a sequence, columns of each
  void* workspace;
  hipStream_t stream;
};
void plan_pages(PagesArgs& a);
size_t pages_workspace(const PagesArgs& a);
sga_status launch_pages(const PagesArgs& a);

struct TreeArgs {
  PagedArgs batch;
  const int32_t* parent;
  int32_t* depth;
  uint32_t* seen;
  int32_t words;
  int32_t L, window, n_global;
  hipStream_t stream;
};
sga_status launch_tree(const TreeArgs& a);

struct KeepArgs {
  PagedArgs batch;
  char *cache_k, *cache_v;
  const int32_t *path, *count;
  int32_t path_columns;
  int32_t Hkv, layers;
  int64_t layer_bytes, page_bytes, head_bytes, row_bytes;
  hipStream_t stream;
};
sga_status launch_keep(const KeepArgs& a);

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
  const int32_t* depth;      // a draft tree (null: none): the rows' depths and which new tokens they see
  const uint32_t* seen;
  int32_t words;
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

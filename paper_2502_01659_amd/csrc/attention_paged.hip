// Attention of new tokens over a paged cache (sga_attention_paged).
//
// A tile is kRows consecutive rows of one sequence and key head, a row being a new token and one of the query heads
// that share the key head (row = token * group + head).  Keys are met in blocks of 32 aligned ones: those of the
// global tokens before the window, then the window's.  Per block, with matrix instructions of 16 x 16 results,
//     S^T[key][row] = K Q^T          O^T[channel][row] += V^T P^T
// so that a lane holds one row (lane % 16) in both, its running maximum and sum stay with it, and the
// probabilities leave the first product in the registers where the second one reads them: the order of the keys inside
// a product is free, and V is loaded in the order that P has.  Lane (m, g), m = lane % 16, g = lane / 16:
//   K  key m of a 16-key tile, 16-byte pieces g, g + 4, ...   (a product takes the same piece of every key)
//   P  keys 4 g .. 4 g + 3 of both 16-key tiles of the block
//   V  those eight keys, channels m d / 16 ..: d / 16 neighbouring channels of each; a lane swaps its eight rows into
//      columns by itself, so V needs neither LDS nor another lane
//   O  row m, channels g d / 4 .. of it: a run of d / 4 neighbouring channels
#include "serving.h"

#include <type_traits>

namespace sga {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kBlock = 32;            // keys of a block
constexpr int kRows = 16;             // rows of a tile
constexpr int kWaves = 4;             // wavefronts of a workgroup, which take its blocks in turn
constexpr int kPieceBlocks = 4 * kWaves;   // fewest blocks of a piece of a split tile

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// The largest of a row's four lanes (m, 0..3).
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, kWave));
  return fmaxf(x, __shfl_xor(x, 32, kWave));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16, kWave);
  return x + __shfl_xor(x, 32, kWave);
}

__device__ __forceinline__ float4v matrix(vec_t<f16_t, 8> a, vec_t<f16_t, 8> b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float4v matrix(vec_t<bf16_t, 8> a, vec_t<bf16_t, 8> b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float4v matrix(float a, float b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Which rows a tile has, and the blocks of keys that they see.
struct Tile {
  int32_t seq, begin, n_new, length;      // sequence, its first packed row, its rows, its length
  int32_t first, count;                   // the tile's flat rows (token * group + head) within the sequence
  int32_t kept;                           // tokens of the sequence that can be seen
  int32_t lead, base, blocks;             // blocks of global keys, first key of the window's blocks, blocks of both
};

// What one row sees: keys j with lo <= j <= hi or j < lead.
struct Sight {
  int32_t lo, hi, lead;
};
__device__ __forceinline__ Sight sight_of(const PagedAttention& a, int32_t p, int32_t kept) {
  if (p < 0 || p >= a.L) return {0, -1, 0};
  const int32_t last = a.causal ? (p < kept - 1 ? p : kept - 1) : kept - 1;
  if (p < a.n_global) return {0, last, 0};
  const int64_t far = (int64_t)p + a.window;
  return {p > a.window ? p - a.window : 0, far < last ? (int32_t)far : last, a.n_global < last + 1 ? a.n_global : last + 1};
}

// The tile of slot i: sequence s owns the slots from seq_ptr[s] * group / kRows + s, which are enough for it and follow
// from seq_ptr alone.  False: an empty slot.  All lanes call it.
__device__ __forceinline__ bool tile_of(const PagedAttention& a, int32_t slot, Tile& t) {
  const PagedArgs& b = a.batch;
  const int64_t group = a.group.value;
  auto first_slot = [&](int32_t s) { return (int64_t)row_of_sequence(b, s) * group / kRows + s; };
  t.seq = __builtin_amdgcn_readfirstlane(last_not_above(b.n_seqs, slot, first_slot));
  t.begin = __builtin_amdgcn_readfirstlane(row_of_sequence(b, t.seq));
  const int32_t end = __builtin_amdgcn_readfirstlane(row_of_sequence(b, t.seq + 1));
  t.length = __builtin_amdgcn_readfirstlane(b.seq_len[t.seq]);
  t.n_new = end > t.begin ? end - t.begin : 0;
  const int64_t first = ((int64_t)slot - (t.begin * group / kRows + t.seq)) * kRows, rows = t.n_new * group;
  if (first < 0 || first >= rows) return false;
  t.first = (int32_t)first;
  t.count = rows - first < kRows ? (int32_t)(rows - first) : kRows;
  const int64_t room = (int64_t)b.pages_per_seq * b.page.value;
  int64_t kept = t.length < 0 ? 0 : t.length;
  kept = kept < room ? kept : room;
  t.kept = (int32_t)(kept < a.L ? kept : a.L);
  // the rows' keys: positions grow with the rows, and so do both ends of what they see
  const int32_t p0 = t.length - t.n_new + (int32_t)quotient((uint32_t)t.first, a.group);
  const int32_t p1 = t.length - t.n_new + (int32_t)quotient((uint32_t)(t.first + t.count - 1), a.group);
  // (rows before 0 and from L on see nothing; a global row sees from 0 on, and then so does what follows)
  const int32_t from = p0 < 0 ? 0 : p0, to = p1 < a.L ? p1 : a.L - 1;
  t.lead = t.base = t.blocks = 0;
  if (from > to) return true;
  const Sight low = sight_of(a, from, t.kept), high = sight_of(a, to, t.kept);
  // (not causal: a global row sees to the end)
  const int32_t last = low.hi > high.hi ? low.hi : high.hi;
  t.base = low.lo & ~(kBlock - 1);
  int32_t lead = low.lead > high.lead ? low.lead : high.lead;
  lead = lead < t.base ? lead : t.base;
  t.lead = (lead + kBlock - 1) / kBlock;
  t.blocks = t.lead + (last >= t.base ? (last - t.base) / kBlock + 1 : 0);
  return true;
}

// Pieces of a tile: at least kPieceBlocks blocks each.
struct Pieces {
  int32_t count, blocks;
};
__device__ __forceinline__ Pieces pieces_of(int32_t blocks, int32_t splits) {
  int32_t each = (blocks + splits - 1) / splits;
  each = each > kPieceBlocks ? (each + kWaves - 1) / kWaves * kWaves : kPieceBlocks;
  const int32_t n = (blocks + each - 1) / each;
  return {n > 0 ? n : 1, each};
}

// Operands of 16-bit storage: eight values of a lane per product of 32.
template <typename T, int D>
struct Core {
  static constexpr int kSteps = D / 32;      // products over the channels of a 16-key tile
  static constexpr int kRun = D / 16;        // channels of V per lane
  using Piece = vec_t<T, 8>;
  using Run = vec_t<T, kRun>;
  static constexpr int kPieceElems = 8;
  Piece q[kSteps];
  Piece k[2][kSteps];
  Run v[8];

  __device__ __forceinline__ float4v scores(int t) const {
    float4v s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) s = matrix(k[t][i], q[i], s);
    return s;
  }
  // P as the sum of two numbers of the storage type: one alone would add an error as large as the
  // rounding of O to O, and the matrix cores wait for memory here.
  __device__ __forceinline__ void mix(const float (&p)[8], float4v (&o)[kRun]) const {
    Piece high, low;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      high[e] = (T)p[e];
      low[e] = (T)(p[e] - (float)high[e]);
    }
#pragma unroll
    for (int c = 0; c < kRun; ++c) {
      Piece column;
#pragma unroll
      for (int e = 0; e < 8; ++e) column[e] = v[e][c];
      o[c] = matrix(column, high, o[c]);
      o[c] = matrix(column, low, o[c]);
    }
  }
};
// fp32 storage: products of four, every operand used whole.
template <int D>
struct Core<float, D> {
  static constexpr int kSteps = D / 16;      // 16-byte pieces of a key per lane
  static constexpr int kRun = D / 16;
  using Piece = vec_t<float, 4>;
  using Run = vec_t<float, kRun>;
  static constexpr int kPieceElems = 4;
  Piece q[kSteps];
  Piece k[2][kSteps];
  Run v[8];

  __device__ __forceinline__ float4v scores(int t) const {
    float4v s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = matrix(k[t][i][e], q[i][e], s);
    return s;
  }
  __device__ __forceinline__ void mix(const float (&p)[8], float4v (&o)[kRun]) const {
#pragma unroll
    for (int c = 0; c < kRun; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[c] = matrix(v[e][c], p[e], o[c]);
  }
};

// Where the rows of a block's keys are.  kWholeTiles: pages hold multiples of 16 tokens, so a 16-key tile lies in one.
struct Places {
  int64_t tile[2];           // kWholeTiles: element offset of the tile's first row (wave-uniform)
  int64_t key[2], value[8];  // else: of the lane's keys
  uint32_t held;             // bit t: tile t has a page; else bit j: key j of the block has one
};

template <typename T, int D, bool kWholeTiles>
__global__ __launch_bounds__(kWaves* kWave) void paged_kernel(PagedAttention a) {
  using C = Core<T, D>;
  constexpr int kRun = C::kRun;
  constexpr int kStride = D + 4;                          // floats of a row in LDS
  __shared__ __align__(16) float out[kWaves][kRows][kStride];
  __shared__ float tops[kWaves][kRows], sums[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int m = lane & 15, g = lane >> 4;
  const int32_t slot = blockIdx.x, head_kv = blockIdx.y, piece = blockIdx.z;
  Tile tile;
  if (!tile_of(a, slot, tile)) return;
  const Pieces pieces = pieces_of(tile.blocks, a.splits);
  if (piece >= pieces.count) return;
  const int32_t group = (int32_t)a.group.value;

  // this lane's row
  const int32_t flat = tile.first + (m < tile.count ? m : 0);
  const int32_t token = (int32_t)quotient((uint32_t)flat, a.group), head = head_kv * group + (flat - token * group);
  const Sight sight = sight_of(a, tile.length - tile.n_new + token, tile.kept);
  C core;
  {
    const T* q = static_cast<const T*>(a.Q) + (int64_t)head * a.q_head + (int64_t)(tile.begin + token) * a.q_row;
#pragma unroll
    for (int i = 0; i < C::kSteps; ++i)
      core.q[i] = *reinterpret_cast<const typename C::Piece*>(q + (g + 4 * i) * C::kPieceElems);
  }
  // keys that every row sees
  int32_t lo_max = sight.lo, hi_min = sight.hi;
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) {
    lo_max = max(lo_max, __shfl_xor(lo_max, off, kWave));
    hi_min = min(hi_min, __shfl_xor(hi_min, off, kWave));
  }
  lo_max = __builtin_amdgcn_readfirstlane(lo_max);
  hi_min = __builtin_amdgcn_readfirstlane(hi_min);

  const PagedArgs& b = a.batch;
  const int64_t in_head = (int64_t)head_kv * b.page.value * D;
  const T* const cache_k = static_cast<const T*>(a.cache_k) + in_head;
  const T* const cache_v = static_cast<const T*>(a.cache_v) + in_head;
  const int32_t* const table = b.page_table + (int64_t)tile.seq * b.pages_per_seq;

  auto first_key = [&](int32_t block) {
    return block < tile.lead ? block * kBlock : tile.base + (block - tile.lead) * kBlock;
  };
  // element offset of key j's row, -1 if it has no page.  (j may lie behind the last token, up to the block's end.)
  auto place_of = [&](int32_t j) -> int64_t {
    const uint32_t column = quotient((uint32_t)j, b.page);
    if (column >= (uint32_t)b.pages_per_seq) return -1;
    const uint32_t page = (uint32_t)table[column];
    return page < b.n_pages ? (int64_t)page * b.page_stride + (int64_t)((uint32_t)j - column * b.page.value) * D : -1;
  };
  auto find = [&](int32_t block) {
    Places at;
    const int32_t j0 = first_key(block);
    at.held = 0;
    if constexpr (kWholeTiles) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t o = uniform64(place_of(j0 + 16 * t));
        at.held |= (o >= 0 ? 1u : 0u) << t;
        at.tile[t] = o >= 0 ? o : 0;
      }
    } else {
      const int64_t o = place_of(j0 + (lane & 31));
      at.held = (uint32_t)__ballot(o >= 0);
      const int64_t safe = o >= 0 ? o : 0;
#pragma unroll
      for (int t = 0; t < 2; ++t) at.key[t] = __shfl(safe, 16 * t + m, kWave);
#pragma unroll
      for (int e = 0; e < 8; ++e) at.value[e] = __shfl(safe, (e < 4 ? 4 * g + e : 12 + 4 * g + e), kWave);
    }
    return at;
  };
  auto load_k = [&](const Places& at) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const T* row = kWholeTiles ? cache_k + at.tile[t] + m * D : cache_k + at.key[t];
#pragma unroll
      for (int i = 0; i < C::kSteps; ++i)
        core.k[t][i] = *reinterpret_cast<const typename C::Piece*>(row + (g + 4 * i) * C::kPieceElems);
    }
  };
  auto load_v = [&](const Places& at) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const T* row = kWholeTiles ? cache_v + at.tile[e / 4] + (4 * g + e % 4) * D : cache_v + at.value[e];
      core.v[e] = *reinterpret_cast<const typename C::Run*>(row + m * kRun);
    }
  };

  const int32_t first_block = piece * pieces.blocks;
  const int32_t end_block = min(first_block + pieces.blocks, tile.blocks);
  float top, sum;
  float4v o[kRun];

  // One walk over the wavefront's blocks.  only >= 0: for that row alone, with the values of every key that it does not
  // see taken as 0 (a product cannot leave a key out: 0 times an infinity or NaN is NaN).
  auto walk = [&](int only) {
    top = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < kRun; ++c) o[c] = float4v{0.f, 0.f, 0.f, 0.f};
    int32_t block = first_block + wave;
    if (block >= end_block) return;
    Places at = find(block);
    load_k(at);
    load_v(at);
    for (; block < end_block; block += kWaves) {
      const int32_t j0 = first_key(block);
      const uint32_t held = at.held;
      const bool more = block + kWaves < end_block;
      float4v s[2] = {core.scores(0), core.scores(1)};
      if (more) {
        at = find(block + kWaves);
        load_k(at);
      }
      const bool all_held = held == (kWholeTiles ? 3u : ~0u);
      const bool whole = all_held && j0 >= lo_max && j0 + kBlock - 1 <= hi_min;
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = s[e / 4][e % 4] * (a.scale * kLog2e);
      uint32_t seen = 0xFF;
      if (!whole) {
        seen = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int in_block = 16 * (e / 4) + 4 * g + e % 4, j = j0 + in_block;
          const bool there = kWholeTiles ? (held >> (e / 4)) & 1 : (held >> in_block) & 1;
          const bool sees = there && ((j >= sight.lo && j <= sight.hi) || j < sight.lead);
          seen |= (sees ? 1u : 0u) << e;
          p[e] = sees ? p[e] : -INFINITY;
        }
      }
      float best = p[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) best = fmaxf(best, p[e]);
      best = fmaxf(row_max(best), top);
      if (__any(best > top)) {
        const float keep = best > -INFINITY ? __builtin_amdgcn_exp2f(top - best) : 1.f;
        sum *= keep;
#pragma unroll
        for (int c = 0; c < kRun; ++c) o[c] *= keep;
        top = best;
      }
      const float against = top > -INFINITY ? top : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(p[e] - against);
        sum += p[e];
      }
      // values of keys that no row sees (behind the last token, without a page) may be anything
      if (only >= 0 || !all_held || j0 + kBlock > tile.kept) {
        const uint32_t row_seen = __shfl(seen, (lane & 48) | (only >= 0 ? only : 0), kWave);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int in_block = 16 * (e / 4) + 4 * g + e % 4;
          const bool there = kWholeTiles ? (held >> (e / 4)) & 1 : (held >> in_block) & 1;
          const bool use = only >= 0 ? (row_seen >> e) & 1 : there && j0 + in_block < tile.kept;
#pragma unroll
          for (int c = 0; c < kRun; ++c) core.v[e][c] = use ? core.v[e][c] : (T)0.f;
        }
      }
      core.mix(p, o);
      if (more) load_v(at);
    }
  };
  auto deposit = [&](bool mine) {
    const float total = row_sum(sum);
    if (!mine) return;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < kRun; ++c) out[wave][m][(4 * g + r) * kRun + c] = o[c][r];
    if (g == 0) {
      tops[wave][m] = top;
      sums[wave][m] = total;
    }
  };
  walk(-1);
  bool finite = true;
#pragma unroll
  for (int c = 0; c < kRun; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r) finite = finite && __builtin_isfinite(o[c][r]);
  if (__all(finite)) {
    deposit(true);
  } else {
    for (int row = 0; row < tile.count; ++row) {
      walk(row);
      deposit(m == row);
    }
  }
  __syncthreads();

  // the wavefronts' states of a row, added in their order
  constexpr int kPer = D * kRows / (kWaves * kWave);       // channels of a thread: D / 16
  const int row = tid / (D / kPer), channel = tid % (D / kPer) * kPer;
  if (row >= tile.count) return;
  float high = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) high = fmaxf(high, tops[w][row]);
  const float against = high > -INFINITY ? high : 0.f;
  float total = 0.f, x[kPer];
#pragma unroll
  for (int c = 0; c < kPer; ++c) x[c] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (sums[w][row] == 0.f) continue;                     // no key seen
    const float weight = __builtin_amdgcn_exp2f(tops[w][row] - against);
    total += weight * sums[w][row];
#pragma unroll
    for (int c = 0; c < kPer; ++c) x[c] += weight * out[w][row][channel + c];
  }
  if (pieces.count > 1) {
    float* part = a.partials + (((int64_t)slot * a.Hkv + head_kv) * a.splits + piece) * (kRows * (D + 2));
#pragma unroll
    for (int c = 0; c < kPer; ++c) part[row * D + channel + c] = x[c];
    if (channel == 0) {
      part[kRows * D + row] = high;
      part[kRows * (D + 1) + row] = total;
    }
    return;
  }
  const int32_t f = tile.first + row, tok = (int32_t)quotient((uint32_t)f, a.group);
  const int32_t h = head_kv * group + (f - tok * group), at_row = tile.begin + tok;
  const float inv = total != 0.f ? 1.f / total : 0.f;
  T* to = static_cast<T*>(a.O) + (int64_t)h * a.o_head + (int64_t)at_row * a.o_row + channel;
  vec_t<T, kPer> y;
#pragma unroll
  for (int c = 0; c < kPer; ++c) y[c] = (T)(x[c] * inv);
  *reinterpret_cast<vec_t<T, kPer>*>(to) = y;
  if (a.lse && channel == 0)
    a.lse[(int64_t)h * b.n_tokens + at_row] = (high + __builtin_amdgcn_logf(total)) * kLn2;
}

// Joins the pieces of the tiles that are split, in their order.
template <typename T, int D>
__global__ __launch_bounds__(kWaves* kWave) void paged_merge_kernel(PagedAttention a) {
  constexpr int kPer = D / 16;
  const int tid = threadIdx.x;
  const int32_t slot = blockIdx.x, head_kv = blockIdx.y;
  Tile tile;
  if (!tile_of(a, slot, tile)) return;
  const Pieces pieces = pieces_of(tile.blocks, a.splits);
  if (pieces.count <= 1) return;
  const int row = tid / 16, channel = tid % 16 * kPer;
  if (row >= tile.count) return;
  const float* part = a.partials + ((int64_t)slot * a.Hkv + head_kv) * a.splits * (kRows * (D + 2));
  float high = -INFINITY;
  for (int i = 0; i < pieces.count; ++i) high = fmaxf(high, part[(int64_t)i * kRows * (D + 2) + kRows * D + row]);
  const float against = high > -INFINITY ? high : 0.f;
  float total = 0.f, x[kPer];
#pragma unroll
  for (int c = 0; c < kPer; ++c) x[c] = 0.f;
  for (int i = 0; i < pieces.count; ++i) {
    const float* p = part + (int64_t)i * kRows * (D + 2);
    if (p[kRows * (D + 1) + row] == 0.f) continue;
    const float weight = __builtin_amdgcn_exp2f(p[kRows * D + row] - against);
    total += weight * p[kRows * (D + 1) + row];
#pragma unroll
    for (int c = 0; c < kPer; ++c) x[c] += weight * p[row * D + channel + c];
  }
  const int32_t group = (int32_t)a.group.value;
  const int32_t f = tile.first + row, tok = (int32_t)quotient((uint32_t)f, a.group);
  const int32_t h = head_kv * group + (f - tok * group), at_row = tile.begin + tok;
  const float inv = total != 0.f ? 1.f / total : 0.f;
  T* to = static_cast<T*>(a.O) + (int64_t)h * a.o_head + (int64_t)at_row * a.o_row + channel;
  vec_t<T, kPer> y;
#pragma unroll
  for (int c = 0; c < kPer; ++c) y[c] = (T)(x[c] * inv);
  *reinterpret_cast<vec_t<T, kPer>*>(to) = y;
  if (a.lse && channel == 0)
    a.lse[(int64_t)h * a.batch.n_tokens + at_row] = (high + __builtin_amdgcn_logf(total)) * kLn2;
}

template <typename T, int D>
sga_status launch_paged_as(const PagedAttention& a) {
  const dim3 grid((unsigned)a.slots, (unsigned)a.Hkv, (unsigned)a.splits);
  profile_mark_begin(a.stream, "paged_kernel");
  if (a.batch.page.value % 16 == 0) paged_kernel<T, D, true><<<grid, kWaves * kWave, 0, a.stream>>>(a);
  else paged_kernel<T, D, false><<<grid, kWaves * kWave, 0, a.stream>>>(a);
  profile_mark_end(a.stream);
  if (a.splits > 1)
    paged_merge_kernel<T, D><<<dim3((unsigned)a.slots, (unsigned)a.Hkv), kWaves * kWave, 0, a.stream>>>(a);
  return hip_status(hipGetLastError());
}

template <typename T>
sga_status launch_paged_type(const PagedAttention& a) {
  switch (a.d) {
    case 32: return launch_paged_as<T, 32>(a);
    case 64: return launch_paged_as<T, 64>(a);
    case 128: return launch_paged_as<T, 128>(a);
    default: return launch_paged_as<T, 256>(a);
  }
}

}  // namespace

PagedPlan plan_paged(const PagedAttention& a) {
  PagedPlan p{1, 0, 0};
  const int64_t slots = (int64_t)a.batch.n_tokens * a.group.value / kRows + a.batch.n_seqs;
  if (slots * kWaves * kWave >= int64_t(1) << 32) return PagedPlan{0, 0, 0};
  p.slots = (int32_t)slots;
  // keys that a tile meets at most
  const int64_t rows = kRows / (int64_t)a.group.value + 2;
  const int64_t room = (int64_t)a.batch.pages_per_seq * a.batch.page.value;
  int64_t keys = a.L < room ? a.L : room;
  const int64_t wide = (a.causal ? 1 : 2) * (int64_t)a.window + rows + a.n_global + 3 * kBlock;
  if (wide < keys && !(a.n_global > 0 && !a.causal)) keys = wide;
  const int64_t blocks = (keys + kBlock - 1) / kBlock + 2;
  const int64_t most = (blocks + kPieceBlocks - 1) / kPieceBlocks, wanted = (1024 + slots * a.Hkv - 1) / (slots * a.Hkv);
  p.splits = (int32_t)(most < wanted ? most : wanted);
  if (p.splits < 1) p.splits = 1;
  if (p.splits > 1) p.bytes = (size_t)slots * a.Hkv * p.splits * kRows * (a.d + 2) * sizeof(float);
  return p;
}

sga_status launch_paged(const PagedAttention& a) {
  switch (a.dtype) {
    case SGA_F32: return launch_paged_type<float>(a);
    case SGA_F16: return launch_paged_type<f16_t>(a);
    default: return launch_paged_type<bf16_t>(a);
  }
}

}  // namespace sga

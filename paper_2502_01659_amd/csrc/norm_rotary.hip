// Norm of every head of queries and keys with the rotation by position in the same pass, and its gradient.
//
//   r = (mean_c x_c^2 + epsilon)^-1/2,   n_c = x_c r w_c,   y = R n
// with R the rotation of paged_cache.hip, pair by pair.  A row is read and written once and costs about ten operations a channel, so memory bounds
// it, as it does the rotation alone.  A row lies in d / 2V neighbouring lanes (V elements of 16 bytes, two such pieces a lane, those that turn together), which
// add their squares by register exchanges.  Which channels a lane has is the same in every row: a wavefront takes a token with all its heads and keeps the
// token's turns in registers (weights are read from LDS for every row).  Measured: 32,768 tokens, 32 + 8 heads of 128, bf16 128 us
// (5.2 TB/s read and written; a large copy 4.8); into pages, with as many values as keys, fp16 165 (4.9).  16 sequences of 5 to 16 drafts into pages take 7.5, 66 % of the wavefronts' time
// waiting: the search for a row's sequence, its length and depth, its page, then the rows.  (A workgroup for a few tokens, turns
// and weights in LDS, a row's tensor picked by its lane: 166, three quarters of the time waiting for what describes the tensor.)
// The gradient of G = dL/dy: with g = R^T G (the rotation by the negative angle),
//   dx_c = r (w_c g_c - x_c r^2 mean_k(w_k g_k x_k)),   dw_c = sum over rows of g_c x_c r.
// One pass too: x and G are read, dx is written, and a lane keeps its channels' part of dw in registers over all the rows that it
// meets.  Workgroups leave their sums in the workspace and a second, small kernel adds them up in 64 bits, in their order: the same call gives the same
// bits.  Measured: the same tokens 194 + 7 us (5.2 TB/s); 10,007 tokens, 8 + 2 heads of 64, fp32 16 + 4.
#include "serving.h"

namespace sga {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 4;        // (any alignment) tokens of a workgroup, as in paged_cache.hip
constexpr int kMaxGroups = 1 << 20;  // workgroups along the tokens; they stride
// Workgroups of the gradient at most: each leaves a partial sum.  (us, kernel and join, 32,768 tokens, 32 + 8 heads of 128, bf16: 1,024 226 + 5, 1,536 210 + 9, 2,048 200 + 8,
// 4,096 198 + 15.)
constexpr int kGradGroups = 2048;
constexpr int kGradTokens = 16;      // (any alignment) tokens of one round of it at most ...
// ... and no more than leave four workgroups a compute unit their weights and turns, a fourth of its LDS each.  (us, as many as 16 / so / 16 KB less: fp32, 32,768 tokens, 8 + 2 heads
// of 1,024 2,861 / 1,980 / 2,159, 4 heads of 768 705 / 539 / 536.  16 tokens of 1,024 channels would take 68 KB.)
constexpr size_t kGradShared = 40 * 1024;
constexpr int64_t kNone = INT64_MIN;  // (rows of a batch) no position; a program's own positions may be any number

// Sum over groups of kLanes neighbouring lanes, in every one of them.  (The lanes of a group are active together.)
template <int kCtrl>
__device__ __forceinline__ float from_dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kCtrl, 0xF, 0xF, true));
}
template <int kLanes>
__device__ __forceinline__ float group_sum(float x) {
  if constexpr (kLanes >= 2) x += from_dpp<0xB1>(x);       // quad_perm 1 0 3 2
  if constexpr (kLanes >= 4) x += from_dpp<0x4E>(x);       // quad_perm 2 3 0 1
  if constexpr (kLanes >= 8) x += from_dpp<0x141>(x);      // mirrored in 8
  if constexpr (kLanes >= 16) x += from_dpp<0x140>(x);     // mirrored in 16
  if constexpr (kLanes >= 32) x += __shfl_xor(x, 16, kWave);
  if constexpr (kLanes >= 64) x += __shfl_xor(x, 32, kWave);
  return x;
}

constexpr int kMostChannels = 1024;
// A weight as it lies in memory, and what it stands for.  (0 where there are none.)
__device__ __forceinline__ uint32_t raw_weight(const NormArg& n, int c) {
  if (!n.on || !n.weight) return 0;
  return n.dtype == SGA_F32 ? static_cast<const uint32_t*>(n.weight)[c] : static_cast<const uint16_t*>(n.weight)[c];
}
__device__ __forceinline__ float weight_from(const NormArg& n, uint32_t raw) {
  if (!n.weight) return 1.f;
  return (n.dtype == SGA_F32   ? __builtin_bit_cast(float, raw)
          : n.dtype == SGA_F16 ? (float)__builtin_bit_cast(f16_t, (uint16_t)raw)
                               : __builtin_bit_cast(float, raw << 16)) + n.offset;
}

__device__ __forceinline__ float weight_at(const NormArg& n, int c) { return weight_from(n, raw_weight(n, c)); }

__device__ __forceinline__ float inverse_size(float squares, float per, float epsilon) { return rsqrtf(fmaf(squares, per, epsilon)); }

// The channels of item k of a row: V from `at` and V from `at2`; where it turns, its pairs are V k ..  Split, pair e is (at + e, at2 + e), else the
// pairs are (at, at + 1) and so on through all 2 V.
template <int V>
struct Item {
  int at, at2;
  bool turns, split;
  __device__ __forceinline__ Item(const RotaryArgs& r, bool rotates, int k) {
    turns = rotates && k < r.channels / (2 * V);
    split = turns && !r.interleaved;
    at = split ? k * V : k * 2 * V;
    at2 = split ? at + (r.channels >> 1) : at + V;
  }
};

// One pair.
__device__ __forceinline__ void turn(float2 cs, float& a, float& b) {
  const float p = a, q = b;
  a = p * cs.x - q * cs.y;
  b = p * cs.y + q * cs.x;
}

struct NormShape {
  FastDiv heads, tokens;         // one pair a lane: rows (heads) of a token here, tokens here
  FastDiv pairs;                 // that turn
  int32_t all_heads;
  int32_t head_first;            // neighbouring rows in memory are a token's heads, not a head's tokens
  int32_t tokens_log2;           // rows in lanes: tokens of a wavefront at a time
  int32_t slices;                // rows in lanes: wavefronts that share a token's heads
};

// Position and place in the cache of a token's row; all lanes of the wavefront call it.
struct Placed {
  int64_t position, cache_row;   // kNone: none; -1: without a page
};
__device__ __forceinline__ Placed find_in_batch(const NormRotateArgs& a, int32_t row) {
  const PagedArgs& b = a.r.batch;
  const int32_t s = last_not_above(b.n_seqs, row, [&](int32_t i) { return b.seq_ptr[i]; });
  const int64_t begin = b.seq_ptr[s], end = b.seq_ptr[s + 1];
  Placed p{kNone, -1};
  if (begin <= row && row < end) {
    const int64_t slot = (int64_t)b.seq_len[s] - (end - row);
    const int32_t depth = a.depth ? a.depth[row] : 0;
    if (depth >= 0) {
      p.position = a.depth ? (int64_t)b.seq_len[s] - (end - begin) + depth : slot;
      if (slot >= 0 && slot < (int64_t)b.pages_per_seq * b.page.value) {
        const uint32_t column = quotient((uint32_t)slot, b.page), in_page = (uint32_t)slot - column * b.page.value;
        const uint32_t page = (uint32_t)b.page_table[(int64_t)s * b.pages_per_seq + column];
        if (page < b.n_pages) p.cache_row = (int64_t)page * b.page_stride + (int64_t)in_page * a.r.d;
      }
    }
  }
  return p;
}

__device__ __forceinline__ float2 turned_by(const RotaryArgs& r, int64_t position, double frequency) {
  const float2 cs = turn_of(position, frequency);
  return make_float2(r.magnitude * cs.x, r.inverse ? -r.magnitude * cs.y : r.magnitude * cs.y);
}

// 2 V channels of a lane in registers: the weights or the turns of its item, which are the same in every row that it meets.
template <int V>
struct Own {
  float u[V], v[V];
};
template <int V>
__device__ __forceinline__ Own<V> weights_of(const float* w, const Item<V>& item) {
  Own<V> own;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    own.u[e] = w[item.at + e];
    own.v[e] = w[item.at2 + e];
  }
  return own;
}

// Rows in lanes, kLanes of them a row with 2 V elements each.  A wavefront works by itself: it takes one token (or, where a token has fewer heads than the
// wavefront holds rows, several) with all its heads, computes the sines into its own part of LDS while the first rows are on their way, and keeps
// those of its lanes' channels in registers: a lane's channels are the same in every row.  Rows are loaded kBatch at a time
// (us, 1 / 2 / 3 / 4 / 8: 32,768 tokens, 32 + 8 heads of 128, bf16 128 / 129 / 136 / 149 / 196: registers).
constexpr int kBatch = 2;
template <typename T, int V, int kLanes, bool kPaged>
__global__ __launch_bounds__(kThreads) void norm_rotate_kernel(NormRotateArgs a, NormShape shape) {
  using Vec = vec_t<T, V>;
  constexpr int kRows = kWave / kLanes;
  extern __shared__ __align__(16) float shared[];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, d = a.r.d;
  const float per = 1.f / (float)d;
  float* const weights = shared;                                                     // [tensors][d]
  const int pairs = shape.pairs.value, tokens = 1 << shape.tokens_log2;
  float2* const turns = reinterpret_cast<float2*>(shared + ((a.r.n_tensors * d + 3) & ~3)) + wave * tokens * pairs;     // [tokens][pairs]
  // (weights are on their way while the first tokens are looked for)
  constexpr int kHeld = (3 * kMostChannels + kThreads - 1) / kThreads;
  uint32_t held[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = threadIdx.x + j * kThreads;
    if (j * kThreads >= a.r.n_tensors * d) break;
    held[j] = i < d ? raw_weight(a.norm[0], i) : i < 2 * d ? raw_weight(a.norm[1], i - d) : i < 3 * d ? raw_weight(a.norm[2], i - 2 * d) : 0;
  }
  const int k = lane % kLanes, group = lane / kLanes;
  const bool mine = k < d / (2 * V);
  const int token = group & (tokens - 1), apart = kRows >> shape.tokens_log2, head0 = group >> shape.tokens_log2;
  // the heads of all tensors in rounds of `apart`, a slice of these rounds for each of the wavefronts that share a token
  int rounds[3], all_rounds = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    rounds[i] = i < a.r.n_tensors ? (a.r.tensor[i].heads + apart - 1) / apart : 0;
    all_rounds += rounds[i];
  }
  const int64_t waves = (int64_t)gridDim.x * (kThreads / kWave), id = (int64_t)blockIdx.x * (kThreads / kWave) + wave;
  const int slices = shape.slices;
  const int64_t units = ((a.r.n_rows + (int64_t)tokens - 1) >> shape.tokens_log2) * slices;
  auto first_row = [&](int64_t unit) { return (int32_t)((unit / slices) << shape.tokens_log2); };
  auto find = [&](int64_t unit) {                           // of this lane's token
    const int32_t row0 = first_row(unit);
    Placed mine{0, -1};
    if constexpr (kPaged) {
      for (int t = 0; t < tokens; ++t) {
        const Placed p = find_in_batch(a, min(row0 + t, a.r.n_rows - 1));
        if (t == token) mine = p;
      }
    } else if (pairs > 0) {
      mine.position = a.r.positions ? a.r.positions[min(row0 + token, a.r.n_rows - 1)] : a.r.first + row0 + token;
    }
    return mine;
  };
  // (the frequency of this lane's first turn: of every token's, mostly)
  const double own_frequency = pairs > 0 ? a.r.rotary.frequencies[lane - (int)quotient((uint32_t)lane, shape.pairs) * pairs] : 0.0;
  Placed next{0, -1};
  if (id < units) next = find(id);
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = threadIdx.x + j * kThreads;
    if (j * kThreads >= a.r.n_tensors * d) break;
    if (i < a.r.n_tensors * d) weights[i] = i < d ? weight_from(a.norm[0], held[j]) : i < 2 * d ? weight_from(a.norm[1], held[j]) : weight_from(a.norm[2], held[j]);
  }
  __syncthreads();
  for (int64_t unit = id; unit < units; unit += waves) {
    const int64_t first = unit / slices;
    const int slice = (int)(unit - first * slices);
    const int32_t row0 = first_row(unit), row = row0 + token;
    const int begin = all_rounds * slice / slices, end = all_rounds * (slice + 1) / slices;
    const int64_t position = next.position, cache_row = next.cache_row;
    const bool there = row < a.r.n_rows && (!kPaged || position != kNone);
    if (!kPaged && unit + waves < units) next = find(unit + waves);
    // (tensor by tensor, so that what describes one is the same in all lanes and known ahead)
    Vec u[kBatch], v[kBatch];
    auto heads_of = [&](const RowsArg& x, int i, bool& is) {
      const int32_t head = head0 + i * apart;
      is = there && mine && head < x.heads && !(kPaged && x.paged && cache_row < 0);
      return head;
    };
    auto load = [&](const RowsArg& x, int i, int stop) {
      const Item<V> item(a.r.rotary, x.rotate, k);
      const T* const src = static_cast<const T*>(x.src) + (int64_t)row * x.src_row;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        bool is;
        const int64_t head = heads_of(x, min(i + b, stop - 1), is);
        const T* const at = src + (is ? head * x.src_head : 0);
        if (is) {
          u[b] = *reinterpret_cast<const Vec*>(at + item.at);
          v[b] = *reinterpret_cast<const Vec*>(at + item.at2);
        }
      }
    };
    Own<V> cosines{}, sines{};
    auto finish = [&](const RowsArg& t, const NormArg& norm, const float* w_of, int i, int stop) {
      const Item<V> item(a.r.rotary, t.rotate, k);
      T* const dst = static_cast<T*>(t.dst) + (kPaged && t.paged ? cache_row : (int64_t)row * t.dst_row);
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (i + b >= stop) break;
        bool is;
        const int64_t head = heads_of(t, i + b, is);
        float x[V], y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          x[e] = (float)u[b][e];
          y[e] = (float)v[b][e];
        }
        if (norm.on) {
          float squares = 0.f;
          if (is) {
#pragma unroll
            for (int e = 0; e < V; ++e) squares = fmaf(x[e], x[e], fmaf(y[e], y[e], squares));
          }
          const float size = inverse_size(group_sum<kLanes>(squares), per, norm.epsilon);
          if (mine) {
            const Own<V> w = weights_of<V>(w_of, item);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              x[e] = x[e] * size * w.u[e];
              y[e] = y[e] * size * w.v[e];
            }
          }
        }
        if (t.rotate && !a.r.rotary.interleaved) {
          if (item.turns) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float p = x[e], q = y[e];
              x[e] = p * cosines.u[e] - q * sines.u[e];
              y[e] = p * sines.u[e] + q * cosines.u[e];
            }
          }
        } else if (t.rotate) {
          if (item.turns) {
#pragma unroll
            for (int e = 0; e < V; e += 2) {
              const float p = x[e], q = x[e + 1], p2 = y[e], q2 = y[e + 1];
              x[e] = p * cosines.u[e / 2] - q * sines.u[e / 2];
              x[e + 1] = p * sines.u[e / 2] + q * cosines.u[e / 2];
              y[e] = p2 * cosines.u[(V + e) / 2] - q2 * sines.u[(V + e) / 2];
              y[e + 1] = p2 * sines.u[(V + e) / 2] + q2 * cosines.u[(V + e) / 2];
            }
          }
        }
        if (is) {
          Vec p, q;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            p[e] = (T)x[e];
            q[e] = (T)y[e];
          }
          T* const to = dst + head * t.dst_head;
          *reinterpret_cast<Vec*>(to + item.at) = p;
          *reinterpret_cast<Vec*>(to + item.at2) = q;
        }
      }
    };
    const int first_stop = min(end, rounds[0]);
    if (begin < first_stop) load(a.r.tensor[0], begin, first_stop);
    // sines of the wavefront's tokens
    if (pairs > 0) {
      for (int i0 = 0; i0 < tokens * pairs; i0 += kWave) {
        const int i = i0 + lane, t = (int)quotient((uint32_t)i, shape.pairs), p = i - t * pairs;
        // (the position of token t: of the lanes that hold its rows)
        const int from = (t & (tokens - 1)) * kLanes;
        const int64_t at = (int64_t)((uint64_t)(uint32_t)__shfl((int)(position >> 32), from, kWave) << 32 | (uint32_t)__shfl((int)position, from, kWave));
        if (i < tokens * pairs) turns[i] = kPaged && at == kNone ? make_float2(0.f, 0.f) : turned_by(a.r.rotary, at, i0 == 0 ? own_frequency : a.r.rotary.frequencies[p]);
      }
      __builtin_amdgcn_wave_barrier();
      // interleaved, pair e of an item's 2 V channels is (2 e, 2 e + 1); split, (e, V + e)
      const Item<V> item(a.r.rotary, true, k);
      if (item.turns && mine) {
        const float2* const cs = turns + token * pairs + k * V;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          cosines.u[e] = cs[e].x;
          sines.u[e] = cs[e].y;
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
    int before = 0;
#pragma unroll
    for (int which = 0; which < 3; ++which) {
      if (which >= a.r.n_tensors) break;
      const int from = max(begin - before, 0), stop = min(end - before, rounds[which]);
      for (int i = from; i < stop; i += kBatch) {
        if (which > 0 || i > from) load(a.r.tensor[which], i, stop);
        finish(a.r.tensor[which], a.norm[which], weights + which * d, i, stop);
      }
      before += rounds[which];
    }
    if (kPaged && unit + waves < units) next = find(unit + waves);
  }
}

// Any size and alignment: a workgroup takes a few tokens, a wavefront goes over a row, a pair a lane, twice.  (us, 32,768 tokens, 32 + 8 heads of 96, bf16: 32 channels turn, rows
// in lanes, 108 and the gradient 160; 24, which are no multiple of the 16 of a lane's two pieces, so 597 and 1,007.)
template <typename T, bool kPaged>
__global__ __launch_bounds__(kThreads) void norm_rotate_any_kernel(NormRotateArgs a, NormShape shape) {
  extern __shared__ __align__(16) float shared[];
  __shared__ int64_t position[kMaxTokens], cache_row[kMaxTokens];
  const int tid = threadIdx.x, tokens = shape.tokens.value, d = a.r.d;
  const float per = 1.f / (float)d;
  float* const weights = shared;                                                     // [tensors][d]
  float2* const turns = reinterpret_cast<float2*>(shared + ((a.r.n_tensors * d + 3) & ~3));     // [tokens][pairs]
  const int pairs = a.r.rotary.channels >> 1;
  for (int i = tid; i < a.r.n_tensors * d; i += kThreads) {
    const int which = i / d;
    if (a.norm[which].on) weights[i] = weight_at(a.norm[which], i - which * d);
  }
  const int32_t head0 = blockIdx.y * shape.heads.value;
  const int heads = min(shape.all_heads - head0, (int)shape.heads.value);
  const int k = tid % kWave;
  for (int64_t row0_ = (int64_t)blockIdx.x * tokens; row0_ < a.r.n_rows; row0_ += (int64_t)gridDim.x * tokens) {
    const int32_t row0 = (int32_t)row0_;
    const int count = min(a.r.n_rows - row0, tokens);
    __syncthreads();                                          // the rows before these are done with the turns
    if constexpr (kPaged) {
      for (int t = tid / kWave; t < count; t += kThreads / kWave) {
        const Placed p = find_in_batch(a, row0 + t);
        if (k == 0) {
          position[t] = p.position;
          cache_row[t] = p.cache_row;
        }
      }
    } else if (tid < count) {
      position[tid] = a.r.positions ? a.r.positions[row0 + tid] : a.r.first + row0 + tid;
    }
    __syncthreads();
    for (int i = tid; i < count * pairs; i += kThreads) {
      const int t = i / pairs;
      if (!kPaged || position[t] != kNone) turns[i] = turned_by(a.r.rotary, position[t], a.r.rotary.frequencies[i - t * pairs]);
    }
    __syncthreads();
    const uint32_t total = (uint32_t)tokens * shape.heads.value;
    for (uint32_t i = tid / kWave; i < total; i += kThreads / kWave) {
      uint32_t t, h;
      if (shape.head_first) {
        t = quotient(i, shape.heads);
        h = i - t * shape.heads.value;
      } else {
        h = quotient(i, shape.tokens);
        t = i - h * shape.tokens.value;
      }
      if ((int)t >= count || (int)h >= heads) continue;
      h += head0;
      int which = 0;
      while (which < a.r.n_tensors - 1 && (int)h >= a.r.tensor[which].heads) h -= a.r.tensor[which++].heads;
      const RowsArg& x = a.r.tensor[which];
      if (kPaged && (position[t] == kNone || (x.paged && cache_row[t] < 0))) continue;
      const int64_t at = row0 + (int)t;
      const T* const src = static_cast<const T*>(x.src) + (int64_t)h * x.src_head + at * x.src_row;
      T* const dst = static_cast<T*>(x.dst) + (int64_t)h * x.dst_head + (kPaged && x.paged ? cache_row[t] : at * x.dst_row);
      const NormArg& norm = a.norm[which];
      float r = 1.f;
      if (norm.on) {
        float squares = 0.f;
        for (int c = k; c < d; c += kWave) squares = fmaf((float)src[c], (float)src[c], squares);
        r = inverse_size(group_sum<kWave>(squares), per, norm.epsilon);
      }
      const float* const w = weights + which * d;
      for (int j = k; j < (d + 1) / 2; j += kWave) {
        const Item<1> item(a.r.rotary, x.rotate, j);
        const bool two = item.at2 < d;                       // (not the last channel of an odd number)
        float p = (float)src[item.at], q = two ? (float)src[item.at2] : 0.f;
        if (norm.on) {
          p = p * r * w[item.at];
          if (two) q = q * r * w[item.at2];
        }
        if (item.turns) turn(turns[(int)t * pairs + j], p, q);
        dst[item.at] = (T)p;
        if (two) dst[item.at2] = (T)q;
      }
    }
  }
}

constexpr int kMostBlocks = 256 * 8;      // workgroups of wavefronts that each take tokens until there are none: what the chip holds and as much again

template <typename T, int V, int kLanes>
sga_status launch_norm_as(const NormRotateArgs& a) {
  const bool paged = a.r.batch.page_table != nullptr;
  NormShape s{};
  const int pairs = a.r.rotary.channels / 2;
  s.pairs = fast_div(pairs > 0 ? pairs : 1);
  s.pairs.value = pairs;
  const size_t weights = (size_t)((a.r.n_tensors * a.r.d + 3) & ~3) * sizeof(float);
  if constexpr (kLanes > 0) {
    constexpr int kRows = kWave / kLanes;
    int most = 0;
    for (int i = 0; i < a.r.n_tensors; ++i) most = a.r.tensor[i].heads > most ? a.r.tensor[i].heads : most;
    while ((2 << s.tokens_log2) * most <= kRows) ++s.tokens_log2;
    const int apart = kRows >> s.tokens_log2;
    int rounds = 0;
    for (int i = 0; i < a.r.n_tensors; ++i) rounds += (a.r.tensor[i].heads + apart - 1) / apart;
    const int64_t units = ((int64_t)a.r.n_rows + (1 << s.tokens_log2) - 1) >> s.tokens_log2;
    s.slices = 1;
    while (s.slices < rounds && units * s.slices < 1024) ++s.slices;
    const int64_t blocks = (units * s.slices + kThreads / kWave - 1) / (kThreads / kWave);
    const unsigned grid = (unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks);
    const size_t lds = weights + (size_t)(kThreads / kWave) * ((size_t)pairs << s.tokens_log2) * sizeof(float2);
    if (paged) norm_rotate_kernel<T, V, kLanes, true><<<grid, kThreads, lds, a.r.stream>>>(a, s);
    else norm_rotate_kernel<T, V, kLanes, false><<<grid, kThreads, lds, a.r.stream>>>(a, s);
  } else {
    for (int i = 0; i < a.r.n_tensors; ++i) s.all_heads += a.r.tensor[i].heads;
    // tokens and heads of a workgroup: as for the rotation alone
    int tokens = kMaxTokens;
    while (tokens > 1 && a.r.n_rows / tokens < 1024) tokens >>= 1;
    int heads = s.all_heads;
    const int64_t groups = ((int64_t)a.r.n_rows + tokens - 1) / tokens;
    while (heads > 1 && groups * ((s.all_heads + heads - 1) / heads) < 256 && heads * kWave * tokens > kThreads) heads = (heads + 1) / 2;
    s.heads = fast_div(heads);
    s.tokens = fast_div(tokens);
    s.head_first = a.r.tensor[0].src_head <= a.r.tensor[0].src_row;
    const dim3 grid((unsigned)(groups < kMaxGroups ? groups : kMaxGroups), (unsigned)((s.all_heads + heads - 1) / heads));
    const size_t lds = weights + (size_t)tokens * pairs * sizeof(float2);
    if (paged) norm_rotate_any_kernel<T, true><<<grid, kThreads, lds, a.r.stream>>>(a, s);
    else norm_rotate_any_kernel<T, false><<<grid, kThreads, lds, a.r.stream>>>(a, s);
  }
  return hip_status(hipGetLastError());
}

// Lanes that hold a row of `items`: the next power of two from 4 on, 0 where a wavefront is too small.
inline int row_lanes(int items) {
  for (int lanes = 4; lanes <= kWave; lanes *= 2)
    if (items <= lanes) return lanes;
  return 0;
}
inline bool wide_at(const void* p, int64_t head, int64_t row, int V) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (head | row) % V == 0;
}

template <typename T>
sga_status launch_norm_type(const NormRotateArgs& a) {
  constexpr int V = 16 / sizeof(T);
  bool wide = a.r.d % (2 * V) == 0 && a.r.rotary.channels % (2 * V) == 0 && a.r.batch.page_stride % V == 0;
  for (int i = 0; i < a.r.n_tensors; ++i) {
    const RowsArg& x = a.r.tensor[i];
    wide = wide && wide_at(x.src, x.src_head, x.src_row, V) && wide_at(x.dst, x.dst_head, x.dst_row, V);
  }
  switch (wide ? row_lanes(a.r.d / (2 * V)) : 0) {
    case 4: return launch_norm_as<T, V, 4>(a);
    case 8: return launch_norm_as<T, V, 8>(a);
    case 16: return launch_norm_as<T, V, 16>(a);
    case 32: return launch_norm_as<T, V, 32>(a);
    case 64: return launch_norm_as<T, V, 64>(a);
    default: return launch_norm_as<T, 1, 0>(a);
  }
}

// ---- gradient ---------------------------------------------------------------------------------------
struct GradShape {
  FastDiv heads[2], pairs;
  int32_t groups[2];         // workgroups of each tensor
  int32_t tokens[2];         // one pair a lane: tokens of a round; rows in lanes: log2 of a wavefront's tokens
  int32_t head_first[2];
};

// The workgroup's sums of its wavefronts' (in `sums`, [wavefronts][d]), in their order, into the workspace.
__device__ __forceinline__ void leave_sums(const NormGradArgs& a, const float* sums) {
  const int d = a.d;
  __syncthreads();
  float* const out = a.partials + (int64_t)blockIdx.x * d;
  for (int c = threadIdx.x; c < d; c += kThreads) out[c] = (sums[c] + sums[d + c]) + (sums[2 * d + c] + sums[3 * d + c]);
}

// Rows in lanes: a wavefront takes tokens by itself, as in the forward pass.
template <typename T, int V, int kLanes>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(NormGradArgs a, GradShape shape) {
  using Vec = vec_t<T, V>;
  constexpr int kRows = kWave / kLanes;
  extern __shared__ __align__(16) float shared[];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, d = a.d;
  const float per = 1.f / (float)d;
  const int which = (int)blockIdx.x >= shape.groups[0] ? 1 : 0;
  const NormGradRows& x = which ? a.tensor[1] : a.tensor[0];
  const int groups = which ? shape.groups[1] : shape.groups[0], tokens_log2 = which ? shape.tokens[1] : shape.tokens[0], tokens = 1 << tokens_log2;
  const int pairs = shape.pairs.value;
  float* const weights = shared;                                                   // [d]
  float2* const turns = reinterpret_cast<float2*>(shared + ((d + 3) & ~3)) + wave * tokens * pairs;     // [tokens][pairs]
  if (x.norm.on)
    for (int c = threadIdx.x; c < d; c += kThreads) weights[c] = weight_at(x.norm, c);
  __syncthreads();
  const int k = lane % kLanes, group = lane / kLanes;
  const bool mine = k < d / (2 * V);
  const int token = group & (tokens - 1), apart = kRows >> tokens_log2, head0 = group >> tokens_log2;
  const Item<V> item(a.rotary, true, k);
  Own<V> w{}, sums{}, cosines{}, sines{};
  if (x.norm.on && mine) w = weights_of<V>(weights, item);
  const int rounds = (x.heads + apart - 1) / apart;
  const int64_t waves = (int64_t)groups * (kThreads / kWave);
  const int64_t units = ((int64_t)a.n_rows + tokens - 1) >> tokens_log2;
  const double own_frequency = pairs > 0 ? a.rotary.frequencies[lane - (int)quotient((uint32_t)lane, shape.pairs) * pairs] : 0.0;
  auto position_of = [&](int64_t unit) -> int64_t {
    const int32_t row = (int32_t)((unit << tokens_log2) + token);
    return pairs == 0 ? 0 : a.positions ? a.positions[min(row, a.n_rows - 1)] : a.first + row;
  };
  int64_t unit = (int64_t)(blockIdx.x - (which ? shape.groups[0] : 0)) * (kThreads / kWave) + wave;
  int64_t next = unit < units ? position_of(unit) : 0;
  Vec xu, xv, gu, gv;
  for (; unit < units; unit += waves) {
    const int32_t row = (int32_t)((unit << tokens_log2) + token);
    const bool there = row < a.n_rows && mine;
    const int64_t position = next;
    if (unit + waves < units) next = position_of(unit + waves);
    const T* const g = static_cast<const T*>(x.g) + (int64_t)row * x.g_row;
    const T* const xs = static_cast<const T*>(x.x) + (int64_t)row * x.x_row;
    T* const dx = static_cast<T*>(x.dx) + (int64_t)row * x.dx_row;
    auto load = [&](int i) {
      const int64_t head = head0 + i * apart;
      if (there && head < x.heads) {
        gu = *reinterpret_cast<const Vec*>(g + head * x.g_head + item.at);
        gv = *reinterpret_cast<const Vec*>(g + head * x.g_head + item.at2);
        if (x.norm.on) {
          xu = *reinterpret_cast<const Vec*>(xs + head * x.x_head + item.at);
          xv = *reinterpret_cast<const Vec*>(xs + head * x.x_head + item.at2);
        }
      }
    };
    load(0);
    if (pairs > 0) {
      for (int i0 = 0; i0 < tokens * pairs; i0 += kWave) {
        const int i = i0 + lane, t = (int)quotient((uint32_t)i, shape.pairs), p = i - t * pairs, from = (t & (tokens - 1)) * kLanes;
        const int64_t at = (int64_t)((uint64_t)(uint32_t)__shfl((int)(position >> 32), from, kWave) << 32 | (uint32_t)__shfl((int)position, from, kWave));
        if (i < tokens * pairs) turns[i] = turned_by(a.rotary, at, i0 == 0 ? own_frequency : a.rotary.frequencies[p]);
      }
      __builtin_amdgcn_wave_barrier();
      if (item.turns && mine) {
        const float2* const cs = turns + token * pairs + k * V;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          cosines.u[e] = cs[e].x;
          sines.u[e] = cs[e].y;
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
    for (int i = 0; i < rounds; ++i) {
      const int64_t head = head0 + i * apart;
      const bool is = there && head < x.heads;
      float u[V], v[V], p[V], q[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        u[e] = (float)xu[e];
        v[e] = (float)xv[e];
        p[e] = (float)gu[e];
        q[e] = (float)gv[e];
      }
      if (i + 1 < rounds) load(i + 1);                        // (on its way while this round is worked on)
      if (item.split) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float b = p[e], c = q[e];
          p[e] = b * cosines.u[e] - c * sines.u[e];
          q[e] = b * sines.u[e] + c * cosines.u[e];
        }
      } else if (item.turns) {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float b = p[e], c = p[e + 1], b2 = q[e], c2 = q[e + 1];
          p[e] = b * cosines.u[e / 2] - c * sines.u[e / 2];
          p[e + 1] = b * sines.u[e / 2] + c * cosines.u[e / 2];
          q[e] = b2 * cosines.u[(V + e) / 2] - c2 * sines.u[(V + e) / 2];
          q[e + 1] = b2 * sines.u[(V + e) / 2] + c2 * cosines.u[(V + e) / 2];
        }
      }
      if (x.norm.on) {
        float squares = 0.f, mixed = 0.f, wu[V], wv[V];
        if (is) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            wu[e] = w.u[e] * p[e];
            wv[e] = w.v[e] * q[e];
            squares = fmaf(u[e], u[e], fmaf(v[e], v[e], squares));
            mixed = fmaf(wu[e], u[e], fmaf(wv[e], v[e], mixed));
          }
        }
        const float r = inverse_size(group_sum<kLanes>(squares), per, x.norm.epsilon);
        const float share = group_sum<kLanes>(mixed) * r * per;                // mean of w g n
        if (is) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float nu = u[e] * r, nv = v[e] * r;
            sums.u[e] = fmaf(p[e], nu, sums.u[e]);
            sums.v[e] = fmaf(q[e], nv, sums.v[e]);
            p[e] = r * fmaf(-nu, share, wu[e]);
            q[e] = r * fmaf(-nv, share, wv[e]);
          }
        }
      }
      if (is) {
        Vec yu, yv;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          yu[e] = (T)p[e];
          yv[e] = (T)q[e];
        }
        *reinterpret_cast<Vec*>(dx + head * x.dx_head + item.at) = yu;
        *reinterpret_cast<Vec*>(dx + head * x.dx_head + item.at2) = yv;
      }
    }
  }
  if (!a.partials) return;
  // over the rows of a wavefront, then over the wavefronts
#pragma unroll
  for (int off = kLanes; off < kWave; off <<= 1)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sums.u[e] += __shfl_xor(sums.u[e], off, kWave);
      sums.v[e] += __shfl_xor(sums.v[e], off, kWave);
    }
  __syncthreads();                                            // (weights and turns are in the same place)
  if (group == 0 && mine) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      shared[wave * d + item.at + e] = sums.u[e];
      shared[wave * d + item.at2 + e] = sums.v[e];
    }
  }
  leave_sums(a, shared);
}

// Any size and alignment: a wavefront goes over a row, a pair a lane, twice.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_grad_any_kernel(NormGradArgs a, GradShape shape) {
  extern __shared__ __align__(16) float shared[];
  __shared__ int64_t position[kGradTokens];
  const int tid = threadIdx.x, d = a.d, pairs = a.rotary.channels >> 1;
  const float per = 1.f / (float)d;
  const int which = (int)blockIdx.x >= shape.groups[0] ? 1 : 0;
  const int32_t group = blockIdx.x - (which ? shape.groups[0] : 0), groups = shape.groups[which];
  const int tokens = shape.tokens[which];
  const FastDiv heads = which ? shape.heads[1] : shape.heads[0];
  const NormGradRows& x = a.tensor[which];
  float* const weights = shared;                                                   // [d]
  float2* const turns = reinterpret_cast<float2*>(shared + ((d + 3) & ~3));        // [tokens][pairs]
  if (x.norm.on)
    for (int c = tid; c < d; c += kThreads) weights[c] = weight_at(x.norm, c);
  constexpr int kPieces = kMostChannels / 2 / kWave;
  const int k = tid % kWave;
  float sum_u[kPieces] = {}, sum_v[kPieces] = {};
  for (int64_t row0_ = (int64_t)group * tokens; row0_ < a.n_rows; row0_ += (int64_t)groups * tokens) {
    const int32_t row0 = (int32_t)row0_;
    const int count = min(a.n_rows - row0, tokens);
    __syncthreads();
    if (tid < count) position[tid] = a.positions ? a.positions[row0 + tid] : a.first + row0 + tid;
    __syncthreads();
    for (int i = tid; i < count * pairs; i += kThreads) turns[i] = turned_by(a.rotary, position[i / pairs], a.rotary.frequencies[i % pairs]);
    __syncthreads();
    const uint32_t total = (uint32_t)count * heads.value;
    for (uint32_t i = tid / kWave; i < total; i += kThreads / kWave) {
      uint32_t t, h;
      if (shape.head_first[which]) {
        t = quotient(i, heads);
        h = i - t * heads.value;
      } else {
        h = i / (uint32_t)count;
        t = i - h * (uint32_t)count;
      }
      const int64_t at = row0 + (int)t;
      const T* const xs = static_cast<const T*>(x.x) + (int64_t)h * x.x_head + at * x.x_row;
      const T* const g = static_cast<const T*>(x.g) + (int64_t)h * x.g_head + at * x.g_row;
      T* const dx = static_cast<T*>(x.dx) + (int64_t)h * x.dx_head + at * x.dx_row;
      float squares = 0.f, mixed = 0.f;
      auto pair = [&](int j, const Item<1>& item, bool two, float& p, float& q) {
        p = (float)g[item.at];
        q = two ? (float)g[item.at2] : 0.f;
        if (item.turns) turn(turns[(int)t * pairs + j], p, q);
      };
      if (x.norm.on) {
        for (int j = k; j < (d + 1) / 2; j += kWave) {
          const Item<1> item(a.rotary, true, j);
          const bool two = item.at2 < d;
          float p, q;
          pair(j, item, two, p, q);
          const float u = (float)xs[item.at], v = two ? (float)xs[item.at2] : 0.f;
          squares = fmaf(u, u, fmaf(v, v, squares));
          mixed = fmaf(weights[item.at] * p, u, mixed);
          if (two) mixed = fmaf(weights[item.at2] * q, v, mixed);
        }
      }
      const float r = x.norm.on ? inverse_size(group_sum<kWave>(squares), per, x.norm.epsilon) : 1.f;
      const float share = group_sum<kWave>(mixed) * r * per;
#pragma unroll
      for (int n = 0; n < kPieces; ++n) {
        const int j = k + n * kWave;
        if (j >= (d + 1) / 2) break;
        const Item<1> item(a.rotary, true, j);
        const bool two = item.at2 < d;
        float p, q;
        pair(j, item, two, p, q);
        if (x.norm.on) {
          const float nu = (float)xs[item.at] * r, nv = two ? (float)xs[item.at2] * r : 0.f;
          sum_u[n] = fmaf(p, nu, sum_u[n]);
          sum_v[n] = fmaf(q, nv, sum_v[n]);
          p = r * fmaf(-nu, share, weights[item.at] * p);
          if (two) q = r * fmaf(-nv, share, weights[item.at2] * q);
        }
        dx[item.at] = (T)p;
        if (two) dx[item.at2] = (T)q;
      }
    }
  }
  if (!a.partials) return;
  __syncthreads();
  float* const sums = shared + (tid / kWave) * d;
#pragma unroll
  for (int n = 0; n < kPieces; ++n) {
    const int j = k + n * kWave;
    if (j >= (d + 1) / 2) break;
    const Item<1> item(a.rotary, true, j);
    sums[item.at] = sum_u[n];
    if (item.at2 < d) sums[item.at2] = sum_v[n];
  }
  leave_sums(a, shared);
}

// dw of both tensors: 16 channels a workgroup, 64 threads for each, which add every 64th partial sum.
constexpr int kJoinChannels = 16, kJoinParts = 64;
__global__ __launch_bounds__(kJoinChannels* kJoinParts) void norm_join_kernel(NormGradArgs a, int32_t groups0, int32_t groups1) {
  __shared__ double sums[kJoinParts][kJoinChannels + 1];
  const NormGradRows& x = a.tensor[blockIdx.y];
  if (!x.dw) return;
  const int32_t first = blockIdx.y ? groups0 : 0, count = blockIdx.y ? groups1 : groups0;
  const int lane = threadIdx.x % kJoinChannels, part = threadIdx.x / kJoinChannels, c = blockIdx.x * kJoinChannels + lane;
  double sum = 0.0;
  if (c < a.d) {
    const float* p = a.partials + (int64_t)first * a.d + c;
#pragma unroll 8
    for (int32_t i = part; i < count; i += kJoinParts) sum += (double)p[(int64_t)i * a.d];
  }
  sums[part][lane] = sum;
  __syncthreads();
  if (part < 4) {
    for (int i = part + 4; i < kJoinParts; i += 4) sum += sums[i][lane];
    sums[part][lane] = sum;
  }
  __syncthreads();
  if (part == 0 && c < a.d) x.dw[c] = (float)((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
}

// Workgroups of each tensor: in proportion to their heads, kGradGroups in all at most; no more than a fourth of its tokens, and beyond one a compute unit than a sixteenth
// (us, kernel and join, a fourth / a sixteenth: 10,007 tokens, 8 + 2 heads of 64, fp32 18.0 + 4.6 / 16.4 + 4.1).
void grad_groups(int64_t n_rows, int32_t Hq, int32_t Hkv, int32_t (&groups)[2]) {
  const int32_t heads[2] = {Hq, Hkv};
  for (int i = 0; i < 2; ++i) {
    if (heads[i] < 1) {
      groups[i] = 0;
      continue;
    }
    const int64_t most = ((int64_t)kGradGroups * heads[i] + Hq + Hkv - 1) / (Hq + Hkv), few = (n_rows + 3) / 4, many = (n_rows + 15) / 16;
    const int64_t enough = many > 256 ? many : few < 256 ? few : 256;
    groups[i] = (int32_t)(enough < 1 ? 1 : enough < most ? enough : most);
  }
}

template <typename T, int V, int kLanes>
sga_status launch_grad_as(const NormGradArgs& a) {
  GradShape s{};
  grad_groups(a.n_rows, a.tensor[0].heads, a.n_tensors > 1 ? a.tensor[1].heads : 0, s.groups);
  const int pairs = a.rotary.channels / 2;
  s.pairs = fast_div(pairs > 0 ? pairs : 1);
  s.pairs.value = pairs;
  int most = 1;                                       // tokens whose turns a workgroup holds
  for (int i = 0; i < a.n_tensors; ++i) {
    const int heads = a.tensor[i].heads;
    s.heads[i] = fast_div(heads);
    s.head_first[i] = a.tensor[i].x_head <= a.tensor[i].x_row;
    if constexpr (kLanes > 0) {
      while ((2 << s.tokens[i]) * heads <= kWave / kLanes) ++s.tokens[i];
      most = (kThreads / kWave) << s.tokens[i] > most ? (kThreads / kWave) << s.tokens[i] : most;
    } else {
      int t = (128 + heads - 1) / heads;
      t = t > kGradTokens ? kGradTokens : t;
      while (t > 1 && (a.n_rows / t < 256 || (size_t)((a.d + 3) & ~3) * sizeof(float) + (size_t)t * pairs * sizeof(float2) > kGradShared)) t >>= 1;
      s.tokens[i] = t;
      most = t > most ? t : most;
    }
  }
  size_t lds = (size_t)((a.d + 3) & ~3) * sizeof(float) + (size_t)most * pairs * sizeof(float2);
  const size_t sums = (size_t)(kThreads / kWave) * a.d * sizeof(float);
  lds = lds > sums ? lds : sums;
  if (a.n_rows > 0) {
    if constexpr (kLanes > 0) norm_grad_kernel<T, V, kLanes><<<s.groups[0] + s.groups[1], kThreads, lds, a.stream>>>(a, s);
    else norm_grad_any_kernel<T><<<s.groups[0] + s.groups[1], kThreads, lds, a.stream>>>(a, s);
  }
  if (a.partials) {
    const bool any = a.n_rows > 0;                     // (no rows: dw is 0)
    norm_join_kernel<<<dim3((a.d + kJoinChannels - 1) / kJoinChannels, a.n_tensors), kJoinChannels * kJoinParts, 0, a.stream>>>(a, any ? s.groups[0] : 0, any ? s.groups[1] : 0);
  }
  return hip_status(hipGetLastError());
}

template <typename T>
sga_status launch_grad_type(const NormGradArgs& a) {
  constexpr int V = 16 / sizeof(T);
  bool wide = a.d % (2 * V) == 0 && a.rotary.channels % (2 * V) == 0;
  for (int i = 0; i < a.n_tensors; ++i) {
    const NormGradRows& x = a.tensor[i];
    wide = wide && (!x.norm.on || wide_at(x.x, x.x_head, x.x_row, V)) && wide_at(x.g, x.g_head, x.g_row, V) && wide_at(x.dx, x.dx_head, x.dx_row, V);
  }
  switch (wide ? row_lanes(a.d / (2 * V)) : 0) {
    case 4: return launch_grad_as<T, V, 4>(a);
    case 8: return launch_grad_as<T, V, 8>(a);
    case 16: return launch_grad_as<T, V, 16>(a);
    case 32: return launch_grad_as<T, V, 32>(a);
    case 64: return launch_grad_as<T, V, 64>(a);
    default: return launch_grad_as<T, 1, 0>(a);
  }
}

}  // namespace

size_t norm_partial_bytes(int64_t n_rows, int32_t Hq, int32_t Hkv, int32_t d) {
  int32_t groups[2];
  grad_groups(n_rows, Hq, Hkv, groups);
  return (size_t)(groups[0] + groups[1]) * d * sizeof(float);
}

sga_status launch_norm_rotate(const NormRotateArgs& a) {
  switch (a.r.dtype) {
    case SGA_F32: return launch_norm_type<float>(a);
    case SGA_F16: return launch_norm_type<f16_t>(a);
    default: return launch_norm_type<bf16_t>(a);
  }
}

sga_status launch_norm_grad(const NormGradArgs& a) {
  switch (a.dtype) {
    case SGA_F32: return launch_grad_type<float>(a);
    case SGA_F16: return launch_grad_type<f16_t>(a);
    default: return launch_grad_type<bf16_t>(a);
  }
}

}  // namespace sga

// Norm of every head of queries and keys with the rotation by position in the same pass, and its gradient.
//
//   r = (mean_c x_c^2 + epsilon)^-1/2,   n_c = x_c r w_c,   y = R n
// with R the rotation of paged_cache.hip, pair by pair.  A row is read and written once and costs about ten operations a channel, so
// memory bounds it, as it does the rotation alone, and the layout is that one's: a workgroup takes a few tokens with all their heads,
// computes their sines once into LDS and streams the rows past them.  What the norm adds is a sum over the row: it lies in d / 2V
// neighbouring lanes (V elements of 16 bytes, two such pieces a lane, those that turn together), which add their squares by
// register exchanges; weights are in LDS in 32 bits.
// The gradient of G = dL/dy: with g = R^T G (the rotation by the negative angle),
//   dx_c = r (w_c g_c - x_c r^2 mean_k(w_k g_k x_k)),   dw_c = sum over rows of g_c x_c r.
// One pass too: x and G are read, dx is written, and a lane keeps its channels' part of dw in registers over all the rows that it
// meets, since its channels are the same in each.  Workgroups leave their sums in the workspace and a second, small
// kernel adds them up in 64 bits, in their order: the same call gives the same bits.
#include "serving.h"

namespace sga {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 4;        // tokens of a workgroup (as in paged_cache.hip)
constexpr int kMaxGroups = 1 << 20;  // workgroups along the tokens; they stride
constexpr int kGradGroups = 1024;    // workgroups of the gradient at most: each leaves a partial sum
constexpr int kGradTokens = 16;      // tokens of one round of it at most
constexpr int64_t kNone = INT64_MIN;

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

__device__ __forceinline__ float weight_at(const NormArg& n, int c) {
  if (!n.weight) return 1.f;
  const float w = n.dtype == SGA_F32   ? static_cast<const float*>(n.weight)[c]
                  : n.dtype == SGA_F16 ? (float)static_cast<const f16_t*>(n.weight)[c]
                                       : (float)static_cast<const bf16_t*>(n.weight)[c];
  return w + n.offset;
}

__device__ __forceinline__ float inverse_size(float squares, float per, float epsilon) { return rsqrtf(fmaf(squares, per, epsilon)); }

// The channels of item k of a row: V from `at` and V from `at2`; where it turns, its cosines and sines are kTurns V k ..
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

// The pair (a[e], b[e]) if split, else (a[2i], a[2i + 1]) and (b[2i], b[2i + 1]).
template <int V>
__device__ __forceinline__ void turn(const Item<V>& item, const float2* cs, float (&u)[V], float (&v)[V]) {
  if (item.split) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float p = u[e], q = v[e];
      u[e] = p * cs[e].x - q * cs[e].y;
      v[e] = p * cs[e].y + q * cs[e].x;
    }
  } else if constexpr (V > 1) {
#pragma unroll
    for (int e = 0; e < V; e += 2) {
      const float2 c = cs[e / 2], c2 = cs[(V + e) / 2];
      const float p = u[e], q = u[e + 1], p2 = v[e], q2 = v[e + 1];
      u[e] = p * c.x - q * c.y;
      u[e + 1] = p * c.y + q * c.x;
      v[e] = p2 * c2.x - q2 * c2.y;
      v[e + 1] = p2 * c2.y + q2 * c2.x;
    }
  } else {
    const float p = u[0], q = v[0];
    u[0] = p * cs[0].x - q * cs[0].y;
    v[0] = p * cs[0].y + q * cs[0].x;
  }
}

struct NormShape {
  FastDiv heads, tokens;         // rows (heads) of a token here, tokens here
  int32_t all_heads;
  int32_t head_first;            // neighbouring rows in memory are a token's heads, not a head's tokens
  int32_t items;                 // of a row, a lane each (the kernel's lanes are at least as many)
};

// Where tokens row0 .. are: their places in the cache and their positions.
template <bool kPaged>
__device__ __forceinline__ void find_tokens(const NormRotateArgs& a, int32_t row0, int count, int64_t* position, int64_t* cache_row) {
  const int tid = threadIdx.x;
  if constexpr (kPaged) {
    for (int t = tid / kWave; t < count; t += kThreads / kWave) {
      const int32_t row = row0 + t;
      const PagedArgs& b = a.r.batch;
      const int32_t s = last_not_above(b.n_seqs, row, [&](int32_t i) { return b.seq_ptr[i]; });
      const int64_t begin = b.seq_ptr[s], end = b.seq_ptr[s + 1];
      int64_t pos = kNone, place = -1;
      if (begin <= row && row < end) {
        const int64_t slot = (int64_t)b.seq_len[s] - (end - row);
        const int32_t depth = a.depth ? a.depth[row] : 0;
        if (depth >= 0) {
          pos = a.depth ? (int64_t)b.seq_len[s] - (end - begin) + depth : slot;
          if (slot >= 0 && slot < (int64_t)b.pages_per_seq * b.page.value) {
            const uint32_t column = quotient((uint32_t)slot, b.page), in_page = (uint32_t)slot - column * b.page.value;
            const uint32_t page = (uint32_t)b.page_table[(int64_t)s * b.pages_per_seq + column];
            if (page < b.n_pages) place = (int64_t)page * b.page_stride + (int64_t)in_page * a.r.d;
          }
        }
      }
      if ((tid & (kWave - 1)) == 0) {
        position[t] = pos;
        cache_row[t] = place;
      }
    }
  } else if (tid < count) {
    position[tid] = a.r.positions ? a.r.positions[row0 + tid] : a.r.first + row0 + tid;
  }
}

__device__ __forceinline__ void find_turns(const RotaryArgs& r, int count, const int64_t* position, float2* turns) {
  const int pairs = r.channels >> 1;
  for (int i = threadIdx.x; i < count * pairs; i += kThreads) {
    const int t = i / pairs, k = i - t * pairs;
    if (position[t] == kNone) continue;
    const float2 cs = turn_of(position[t], r.frequencies[k]);
    turns[i] = make_float2(r.magnitude * cs.x, r.inverse ? -r.magnitude * cs.y : r.magnitude * cs.y);
  }
}

// kLanes lanes hold a row, 2 V elements each; kLanes 0: a wavefront goes over the row, one pair at a time, twice (any size and
// alignment).
template <typename T, int V, int kLanes, bool kPaged>
__global__ __launch_bounds__(kThreads) void norm_rotate_kernel(NormRotateArgs a, NormShape shape) {
  extern __shared__ __align__(16) float shared[];
  __shared__ int64_t position[kMaxTokens], cache_row[kMaxTokens];
  const int tid = threadIdx.x, tokens = shape.tokens.value, d = a.r.d;
  const float per = 1.f / (float)d;
  float* const weights = shared;                                                     // [tensors][d]
  float2* const turns = reinterpret_cast<float2*>(shared + ((a.r.n_tensors * d + 3) & ~3));     // [tokens][channels / 2]
  const int pairs = a.r.rotary.channels >> 1;
  for (int i = tid; i < a.r.n_tensors * d; i += kThreads) {
    const int which = i / d;
    if (a.norm[which].on) weights[i] = weight_at(a.norm[which], i - which * d);
  }
  const int32_t head0 = blockIdx.y * shape.heads.value;
  const int heads = min(shape.all_heads - head0, (int)shape.heads.value);
  constexpr int kRowLanes = kLanes ? kLanes : kWave;
  const int k = tid % kRowLanes;

  for (int64_t row0_ = (int64_t)blockIdx.x * tokens; row0_ < a.r.n_rows; row0_ += (int64_t)gridDim.x * tokens) {
    const int32_t row0 = (int32_t)row0_;
    const int count = min(a.r.n_rows - row0, tokens);
    __syncthreads();                                          // the rows before these are done with the turns
    find_tokens<kPaged>(a, row0, count, position, cache_row);
    if constexpr (kPaged) __syncthreads();
    struct Row {
      const T* src;
      T* dst;
      int which, t;
      bool there;
    };
    auto locate = [&](uint32_t i) {
      Row row{};
      uint32_t t, h;
      if (shape.head_first) {
        t = quotient(i, shape.heads);
        h = i - t * shape.heads.value;
      } else {
        h = quotient(i, shape.tokens);
        t = i - h * shape.tokens.value;
      }
      if ((int)t >= count || (int)h >= heads) return row;
      h += head0;
      int which = 0;
      while (which < a.r.n_tensors - 1 && (int)h >= a.r.tensor[which].heads) h -= a.r.tensor[which++].heads;
      const RowsArg& x = a.r.tensor[which];
      const int64_t at = row0 + (int)t;
      row.src = static_cast<const T*>(x.src) + (int64_t)h * x.src_head + at * x.src_row;
      row.dst = static_cast<T*>(x.dst) + (int64_t)h * x.dst_head + (kPaged && x.paged ? cache_row[t] : at * x.dst_row);
      row.which = which;
      row.t = (int)t;
      row.there = !kPaged || (position[t] != kNone && !(x.paged && cache_row[t] < 0));
      return row;
    };
    auto make_turns = [&]() {
      if constexpr (!kPaged) __syncthreads();
      find_turns(a.r.rotary, count, position, turns);
      __syncthreads();
    };
    const uint32_t total = (uint32_t)tokens * shape.heads.value, step = kThreads / kRowLanes;
    if constexpr (kLanes > 0) {
      using Vec = vec_t<T, V>;
      auto load = [&](const Row& row, Vec& u, Vec& v) {
        if (!row.there || k >= shape.items) return;
        const Item<V> item(a.r.rotary, a.r.tensor[row.which].rotate, k);
        u = *reinterpret_cast<const Vec*>(row.src + item.at);
        v = *reinterpret_cast<const Vec*>(row.src + item.at2);
      };
      uint32_t i = tid / kLanes;
      Row row = locate(i);
      Vec u = {}, v = {};
      if (i < total) load(row, u, v);                          // (on its way while the sines are computed)
      make_turns();
      for (; i < total; i += step) {
        const Row here = row;
        float x[V], y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          x[e] = (float)u[e];
          y[e] = (float)v[e];
        }
        if (i + step < total) {                                // the next row is on its way while this one is worked on
          row = locate(i + step);
          load(row, u, v);
        }
        if (!here.there) continue;
        const NormArg& norm = a.norm[here.which];
        const Item<V> item(a.r.rotary, a.r.tensor[here.which].rotate, k);
        if (norm.on) {
          float squares = 0.f;
          if (k < shape.items) {
#pragma unroll
            for (int e = 0; e < V; ++e) squares = fmaf(x[e], x[e], fmaf(y[e], y[e], squares));
          }
          const float r = inverse_size(group_sum<kLanes>(squares), per, norm.epsilon);
          const float* const w = weights + here.which * d;
          if (k < shape.items) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              x[e] = x[e] * r * w[item.at + e];
              y[e] = y[e] * r * w[item.at2 + e];
            }
          }
        }
        if (k >= shape.items) continue;
        if (item.turns) turn<V>(item, turns + here.t * pairs + k * V, x, y);
        Vec p, q;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          p[e] = (T)x[e];
          q[e] = (T)y[e];
        }
        *reinterpret_cast<Vec*>(here.dst + item.at) = p;
        *reinterpret_cast<Vec*>(here.dst + item.at2) = q;
      }
    } else {
      make_turns();
      for (uint32_t i = tid / kWave; i < total; i += step) {
        const Row row = locate(i);
        if (!row.there) continue;
        const NormArg& norm = a.norm[row.which];
        float r = 1.f;
        if (norm.on) {
          float squares = 0.f;
          for (int c = k; c < d; c += kWave) squares = fmaf((float)row.src[c], (float)row.src[c], squares);
          r = inverse_size(group_sum<kWave>(squares), per, norm.epsilon);
        }
        const float* const w = weights + row.which * d;
        for (int j = k; j < (d + 1) / 2; j += kWave) {
          const Item<1> item(a.r.rotary, a.r.tensor[row.which].rotate, j);
          const bool two = item.at2 < d;                       // (not the last channel of an odd number)
          float x[1] = {(float)row.src[item.at]}, y[1] = {two ? (float)row.src[item.at2] : 0.f};
          if (norm.on) {
            x[0] = x[0] * r * w[item.at];
            if (two) y[0] = y[0] * r * w[item.at2];
          }
          if (item.turns) turn<1>(item, turns + row.t * pairs + j, x, y);
          row.dst[item.at] = (T)x[0];
          if (two) row.dst[item.at2] = (T)y[0];
        }
      }
    }
  }
}

template <typename T, int V, int kLanes>
sga_status launch_norm_as(const NormRotateArgs& a) {
  const bool paged = a.r.batch.page_table != nullptr;
  NormShape s{};
  for (int i = 0; i < a.r.n_tensors; ++i) s.all_heads += a.r.tensor[i].heads;
  constexpr int kRowLanes = kLanes ? kLanes : kWave;
  // tokens and heads of a workgroup: as for the rotation alone
  int tokens = kMaxTokens;
  while (tokens > 1 && a.r.n_rows / tokens < 1024) tokens >>= 1;
  int heads = s.all_heads;
  const int64_t groups = ((int64_t)a.r.n_rows + tokens - 1) / tokens;
  while (heads > 1 && groups * ((s.all_heads + heads - 1) / heads) < 256 && heads * kRowLanes * tokens > kThreads)
    heads = (heads + 1) / 2;
  s.heads = fast_div(heads);
  s.tokens = fast_div(tokens);
  s.head_first = a.r.tensor[0].src_head <= a.r.tensor[0].src_row;
  s.items = a.r.d / (2 * V);
  const dim3 grid((unsigned)(groups < kMaxGroups ? groups : kMaxGroups), (unsigned)((s.all_heads + heads - 1) / heads));
  const size_t lds = (size_t)((a.r.n_tensors * a.r.d + 3) & ~3) * sizeof(float) + (size_t)tokens * (a.r.rotary.channels / 2) * sizeof(float2);
  if (paged) norm_rotate_kernel<T, V, kLanes, true><<<grid, kThreads, lds, a.r.stream>>>(a, s);
  else norm_rotate_kernel<T, V, kLanes, false><<<grid, kThreads, lds, a.r.stream>>>(a, s);
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
  FastDiv heads[2];
  int32_t groups[2];         // workgroups of each tensor
  int32_t tokens[2];         // tokens of a round
  int32_t items;
  int32_t head_first[2];
};

template <typename T, int V, int kLanes>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(NormGradArgs a, GradShape shape) {
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
  float2* const turns = reinterpret_cast<float2*>(shared + ((d + 3) & ~3));        // [tokens][channels / 2]
  // (behind them, at the end, the wavefronts' sums [4][d], in the same place)
  if (x.norm.on)
    for (int c = tid; c < d; c += kThreads) weights[c] = weight_at(x.norm, c);
  constexpr int kRowLanes = kLanes ? kLanes : kWave;
  constexpr int kPieces = kLanes ? 1 : 8;                       // (d up to 1,024: 512 pairs)
  const int k = tid % kRowLanes;
  float sum_u[kPieces][V], sum_v[kPieces][V];
#pragma unroll
  for (int p = 0; p < kPieces; ++p)
#pragma unroll
    for (int e = 0; e < V; ++e) sum_u[p][e] = sum_v[p][e] = 0.f;

  for (int64_t row0_ = (int64_t)group * tokens; row0_ < a.n_rows; row0_ += (int64_t)groups * tokens) {
    const int32_t row0 = (int32_t)row0_;
    const int count = min(a.n_rows - row0, tokens);
    __syncthreads();
    if (tid < count) position[tid] = a.positions ? a.positions[row0 + tid] : a.first + row0 + tid;
    __syncthreads();
    find_turns(a.rotary, count, position, turns);
    __syncthreads();
    const uint32_t total = (uint32_t)count * heads.value, step = kThreads / kRowLanes;
    struct Row {
      const T *x, *g;
      T* dx;
      int t;
    };
    auto locate = [&](uint32_t i) {
      uint32_t t, h;
      if (shape.head_first[which]) {
        t = quotient(i, heads);
        h = i - t * heads.value;
      } else {
        h = i / (uint32_t)count;
        t = i - h * (uint32_t)count;
      }
      const int64_t at = row0 + (int)t;
      return Row{static_cast<const T*>(x.x) + (int64_t)h * x.x_head + at * x.x_row, static_cast<const T*>(x.g) + (int64_t)h * x.g_head + at * x.g_row,
                 static_cast<T*>(x.dx) + (int64_t)h * x.dx_head + at * x.dx_row, (int)t};
    };
    if constexpr (kLanes > 0) {
      using Vec = vec_t<T, V>;
      const Item<V> item(a.rotary, true, k);
      const bool mine = k < shape.items;
      uint32_t i = tid / kLanes;
      Row row{};
      Vec xu = {}, xv = {}, gu = {}, gv = {};
      auto load = [&](uint32_t at) {
        row = locate(at);
        if (!mine) return;
        gu = *reinterpret_cast<const Vec*>(row.g + item.at);
        gv = *reinterpret_cast<const Vec*>(row.g + item.at2);
        if (x.norm.on) {
          xu = *reinterpret_cast<const Vec*>(row.x + item.at);
          xv = *reinterpret_cast<const Vec*>(row.x + item.at2);
        }
      };
      if (i < total) load(i);
      for (; i < total; i += step) {
        const Row here = row;
        float u[V], v[V], p[V], q[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          u[e] = (float)xu[e];
          v[e] = (float)xv[e];
          p[e] = (float)gu[e];
          q[e] = (float)gv[e];
        }
        if (i + step < total) load(i + step);
        if (mine && item.turns) turn<V>(item, turns + here.t * pairs + k * V, p, q);
        if (x.norm.on) {
          float squares = 0.f, mixed = 0.f, wu[V], wv[V];
          if (mine) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              wu[e] = weights[item.at + e] * p[e];
              wv[e] = weights[item.at2 + e] * q[e];
              squares = fmaf(u[e], u[e], fmaf(v[e], v[e], squares));
              mixed = fmaf(wu[e], u[e], fmaf(wv[e], v[e], mixed));
            }
          }
          const float r = inverse_size(group_sum<kLanes>(squares), per, x.norm.epsilon);
          const float share = group_sum<kLanes>(mixed) * r * per;           // mean of w g n
          if (mine) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float nu = u[e] * r, nv = v[e] * r;
              sum_u[0][e] = fmaf(p[e], nu, sum_u[0][e]);
              sum_v[0][e] = fmaf(q[e], nv, sum_v[0][e]);
              p[e] = r * fmaf(-nu, share, wu[e]);
              q[e] = r * fmaf(-nv, share, wv[e]);
            }
          }
        }
        if (!mine) continue;
        Vec yu, yv;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          yu[e] = (T)p[e];
          yv[e] = (T)q[e];
        }
        *reinterpret_cast<Vec*>(here.dx + item.at) = yu;
        *reinterpret_cast<Vec*>(here.dx + item.at2) = yv;
      }
    } else {
      for (uint32_t i = tid / kWave; i < total; i += step) {
        const Row row = locate(i);
        float squares = 0.f, mixed = 0.f;
        auto pair = [&](int j, const Item<1>& item, bool two, float (&p)[1], float (&q)[1]) {
          p[0] = (float)row.g[item.at];
          q[0] = two ? (float)row.g[item.at2] : 0.f;
          if (item.turns) turn<1>(item, turns + row.t * pairs + j, p, q);
        };
        if (x.norm.on) {
          for (int j = k; j < (d + 1) / 2; j += kWave) {
            const Item<1> item(a.rotary, true, j);
            const bool two = item.at2 < d;
            float p[1], q[1];
            pair(j, item, two, p, q);
            const float u = (float)row.x[item.at], v = two ? (float)row.x[item.at2] : 0.f;
            squares = fmaf(u, u, fmaf(v, v, squares));
            mixed = fmaf(weights[item.at] * p[0], u, mixed);
            if (two) mixed = fmaf(weights[item.at2] * q[0], v, mixed);
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
          float p[1], q[1];
          pair(j, item, two, p, q);
          if (x.norm.on) {
            const float nu = (float)row.x[item.at] * r, nv = two ? (float)row.x[item.at2] * r : 0.f;
            sum_u[n][0] = fmaf(p[0], nu, sum_u[n][0]);
            sum_v[n][0] = fmaf(q[0], nv, sum_v[n][0]);
            p[0] = r * fmaf(-nu, share, weights[item.at] * p[0]);
            if (two) q[0] = r * fmaf(-nv, share, weights[item.at2] * q[0]);
          }
          row.dx[item.at] = (T)p[0];
          if (two) row.dx[item.at2] = (T)q[0];
        }
      }
    }
  }
  if (!a.partials) return;
  // the workgroup's sums: over the rows of a wavefront, then over the wavefronts, in their order
  if constexpr (kLanes > 0) {
#pragma unroll
    for (int off = kLanes; off < kWave; off <<= 1)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sum_u[0][e] += __shfl_xor(sum_u[0][e], off, kWave);
        sum_v[0][e] += __shfl_xor(sum_v[0][e], off, kWave);
      }
  }
  __syncthreads();
  float* const sums = shared + (tid / kWave) * d;
#pragma unroll
  for (int p = 0; p < kPieces; ++p) {
    const int j = k + p * kRowLanes;
    if (tid % kWave >= kRowLanes || j >= (kLanes ? shape.items : (d + 1) / 2)) continue;
    const Item<V> item(a.rotary, true, j);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sums[item.at + e] = sum_u[p][e];
      if (item.at2 + e < d) sums[item.at2 + e] = sum_v[p][e];
    }
  }
  __syncthreads();
  float* const out = a.partials + (int64_t)blockIdx.x * d;
  for (int c = tid; c < d; c += kThreads) out[c] = (shared[c] + shared[d + c]) + (shared[2 * d + c] + shared[3 * d + c]);
}

// dw of both tensors: 32 channels a workgroup, 32 threads for each, which add every 32nd partial sum.
__global__ __launch_bounds__(1024) void norm_join_kernel(NormGradArgs a, int32_t groups0, int32_t groups1) {
  __shared__ double sums[32][33];
  const NormGradRows& x = a.tensor[blockIdx.y];
  if (!x.dw) return;
  const int32_t first = blockIdx.y ? groups0 : 0, count = blockIdx.y ? groups1 : groups0;
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  double sum = 0.0;
  if (c < a.d) {
    const float* p = a.partials + (int64_t)first * a.d + c;
#pragma unroll 8
    for (int32_t i = part; i < count; i += 32) sum += (double)p[(int64_t)i * a.d];
  }
  sums[part][lane] = sum;
  __syncthreads();
  if (part == 0 && c < a.d) {
    sum = 0.0;
    for (int i = 0; i < 32; ++i) sum += sums[i][lane];
    x.dw[c] = (float)sum;
  }
}

// Workgroups of each tensor: in proportion to their heads, as many as have a round of rows each, kGradGroups in all at most.
void grad_groups(int64_t n_rows, int32_t Hq, int32_t Hkv, int32_t (&groups)[2], int32_t (&tokens)[2]) {
  const int32_t heads[2] = {Hq, Hkv};
  for (int i = 0; i < 2; ++i) {
    groups[i] = tokens[i] = 0;
    if (heads[i] < 1) continue;
    int32_t t = (128 + heads[i] - 1) / heads[i];
    t = t < 1 ? 1 : t > kGradTokens ? kGradTokens : t;
    while (t > 1 && n_rows / t < 256) t >>= 1;
    const int64_t most = ((int64_t)kGradGroups * heads[i] + Hq + Hkv - 1) / (Hq + Hkv), rounds = (n_rows + t - 1) / t;
    tokens[i] = t;
    groups[i] = (int32_t)(rounds < most ? (rounds < 1 ? 1 : rounds) : most);
  }
}

template <typename T, int V, int kLanes>
sga_status launch_grad_as(const NormGradArgs& a) {
  GradShape s{};
  grad_groups(a.n_rows, a.tensor[0].heads, a.n_tensors > 1 ? a.tensor[1].heads : 0, s.groups, s.tokens);
  for (int i = 0; i < a.n_tensors; ++i) s.head_first[i] = a.tensor[i].x_head <= a.tensor[i].x_row;
  s.items = a.d / (2 * V);
  s.heads[0] = fast_div(a.tensor[0].heads);
  s.heads[1] = fast_div(a.n_tensors > 1 ? a.tensor[1].heads : 1);
  const int most = s.tokens[0] > s.tokens[1] ? s.tokens[0] : s.tokens[1];
  size_t lds = (size_t)((a.d + 3) & ~3) * sizeof(float) + (size_t)most * (a.rotary.channels / 2) * sizeof(float2);
  const size_t sums = (size_t)(kThreads / kWave) * a.d * sizeof(float);
  lds = lds > sums ? lds : sums;
  if (a.n_rows > 0) norm_grad_kernel<T, V, kLanes><<<s.groups[0] + s.groups[1], kThreads, lds, a.stream>>>(a, s);
  if (a.partials) {
    const bool any = a.n_rows > 0;                     // (no rows: dw is 0)
    norm_join_kernel<<<dim3((a.d + 31) / 32, a.n_tensors), 1024, 0, a.stream>>>(a, any ? s.groups[0] : 0, any ? s.groups[1] : 0);
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
  int32_t groups[2], tokens[2];
  grad_groups(n_rows, Hq, Hkv, groups, tokens);
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

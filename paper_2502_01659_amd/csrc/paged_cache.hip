// Rotary positions and appending to a paged cache: one pass over rows of channels.
//
// Pair (a, b) of a head turns by t = position * frequency: a' = m (a cos t - b sin t), b' = m (a sin t + b cos t);
// the inverse turns by -t.  Every element is read and written once and a pair costs four multiplications, so memory
// bounds it; what could cost more is the sines, and they depend on the token and the pair but not on the head.  A
// workgroup therefore takes a few tokens with all their heads (of Q, K and V together when it appends to a
// cache), computes their sines once into LDS and streams the rows past them, 16 bytes per lane and access.
// Measured (us, read and written): queries of 65,536 tokens, 32 heads of 128, bf16 193 (5.6 TB/s; a large copy 5.0); prompts
// of 33,000 tokens into pages, 32 + 8 + 8 heads of 128, fp16 182 (4.5); 100,003 tokens, 8 heads of 64, fp32 73 (5.6).
#include "serving.h"

namespace sga {
namespace {

constexpr int kThreads = 256;
// tokens of a workgroup at most (us, 8 / 4 / 2: queries of 65,536 tokens, 32 heads of 128, bf16 204 / 193 / 187; prompts of 33,000
// tokens into pages, 32 + 8 + 8 heads, fp16 192 / 187 / 189; 100,003 tokens, 8 heads of 64, fp32 76 / 73 / 76)
constexpr int kMaxTokens = 4;
constexpr int kMaxGroups = 1 << 20;  // workgroups along the tokens (a grid holds fewer than 2^32 threads); they stride

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

struct RotateShape {
  FastDiv items, heads, tokens;   // items of a row, rows (heads) of a token here, tokens here
  int32_t heads_here;             // heads of a workgroup (of all tensors' heads, one behind the other)
  int32_t all_heads;
  int32_t head_first;             // neighbouring rows in memory are a token's heads, not a head's tokens
};

// V elements per access: 16 bytes, or one where sizes or addresses do not allow that.  An item is 2 V channels of a row.
template <typename T, int V, bool kPaged>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a, RotateShape shape) {
  extern __shared__ __align__(16) float2 turns[];          // [tokens][channels / 2]
  __shared__ int64_t position[kMaxTokens], cache_row[kMaxTokens];
  const int tid = threadIdx.x, tokens = shape.tokens.value;
  constexpr int64_t kNone = INT64_MIN;

  for (int64_t row0_ = (int64_t)blockIdx.x * tokens; row0_ < a.n_rows; row0_ += (int64_t)gridDim.x * tokens) {
    const int32_t row0 = (int32_t)row0_;
    const int count = a.n_rows - row0 < tokens ? a.n_rows - row0 : tokens;
    __syncthreads();                                          // the rows before these are done with the turns
    if constexpr (kPaged) {
      for (int t = tid / kWave; t < count; t += kThreads / kWave) {
        const int32_t row = row0 + t;
        const PagedArgs& b = a.batch;
        const int32_t s = last_not_above(b.n_seqs, row, [&](int32_t i) { return b.seq_ptr[i]; });
        const int64_t begin = b.seq_ptr[s], end = b.seq_ptr[s + 1];
        int64_t pos = kNone, place = -1;
        if (begin <= row && row < end) {
          pos = (int64_t)b.seq_len[s] - (end - row);
          if (pos >= 0 && pos < (int64_t)b.pages_per_seq * b.page.value) {
            const uint32_t column = quotient((uint32_t)pos, b.page), in_page = (uint32_t)pos - column * b.page.value;
            const uint32_t page = (uint32_t)b.page_table[(int64_t)s * b.pages_per_seq + column];
            if (page < b.n_pages) place = (int64_t)page * b.page_stride + (int64_t)in_page * a.d;
          }
        }
        if ((tid & (kWave - 1)) == 0) {
          position[t] = pos;
          cache_row[t] = place;
        }
      }
    } else if (tid < count) {
      position[tid] = a.positions ? a.positions[row0 + tid] : a.first + row0 + tid;
    }
    __syncthreads();
    const int pairs = a.rotary.channels >> 1;
    for (int i = tid; i < count * pairs; i += kThreads) {
      const int t = i / pairs, k = i - t * pairs;
      if (kPaged && position[t] == kNone) continue;
      const float2 cs = turn_of(position[t], a.rotary.frequencies[k]);
      const float m = a.rotary.magnitude;
      turns[i] = make_float2(m * cs.x, a.rotary.inverse ? -m * cs.y : m * cs.y);
    }
    __syncthreads();

    using Vec = vec_t<T, V>;
    const int32_t head0 = blockIdx.y * shape.heads_here;
    const int heads = shape.all_heads - head0 < shape.heads_here ? shape.all_heads - head0 : shape.heads_here;
    const int turning = a.rotary.channels / (2 * V);           // items of a row that turn
    const uint32_t total = shape.items.value * (uint32_t)tokens * (uint32_t)shape.heads_here;
    for (uint32_t i = tid; i < total; i += kThreads) {
      const uint32_t row = quotient(i, shape.items), k = i - row * shape.items.value;
      uint32_t t, h;
      if (shape.head_first) {
        t = quotient(row, shape.heads);
        h = row - t * shape.heads.value;
      } else {
        h = quotient(row, shape.tokens);
        t = row - h * shape.tokens.value;
      }
      if ((int)t >= count || (int)h >= heads) continue;
      h += head0;
      int which = 0;
      if (kPaged) {
        while (which < a.n_tensors - 1 && (int)h >= a.tensor[which].heads) h -= a.tensor[which++].heads;
      }
      const RowsArg& x = a.tensor[which];
      const T* src = static_cast<const T*>(x.src) + (int64_t)h * x.src_head + (int64_t)(row0 + (int)t) * x.src_row;
      T* dst = static_cast<T*>(x.dst) + (int64_t)h * x.dst_head;
      if (kPaged) {
        if (position[t] == kNone || (x.paged && cache_row[t] < 0)) continue;
        dst += x.paged ? cache_row[t] : (int64_t)(row0 + (int)t) * x.dst_row;
      } else {
        dst += (int64_t)(row0 + (int)t) * x.dst_row;
      }
      const bool turns_here = (int)k < turning && (!kPaged || x.rotate);
      const bool split = turns_here && !a.rotary.interleaved;
      const int at = split ? (int)k * V : (int)k * 2 * V, at2 = split ? at + pairs : at + V;
      if (V == 1 && at2 >= a.d) {                              // the last channel of an odd number
        dst[at] = src[at];
        continue;
      }
      Vec u, v;
      if constexpr (V == 1) {
        u[0] = src[at];
        v[0] = src[at2];
      } else {
        u = *reinterpret_cast<const Vec*>(src + at);
        v = *reinterpret_cast<const Vec*>(src + at2);
      }
      if (turns_here) {
        const float2* cs = turns + (int)t * pairs + (int)k * V;
        if (split) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float p = (float)u[e], q = (float)v[e], c = cs[e].x, s = cs[e].y;
            u[e] = (T)(p * c - q * s);
            v[e] = (T)(p * s + q * c);
          }
        } else if constexpr (V == 1) {
          const float p = (float)u[0], q = (float)v[0], c = cs[0].x, s = cs[0].y;
          u[0] = (T)(p * c - q * s);
          v[0] = (T)(p * s + q * c);
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const float p = (float)u[e], q = (float)u[e + 1], c = cs[e / 2].x, s = cs[e / 2].y;
            const float p2 = (float)v[e], q2 = (float)v[e + 1], c2 = cs[(V + e) / 2].x, s2 = cs[(V + e) / 2].y;
            u[e] = (T)(p * c - q * s);
            u[e + 1] = (T)(p * s + q * c);
            v[e] = (T)(p2 * c2 - q2 * s2);
            v[e + 1] = (T)(p2 * s2 + q2 * c2);
          }
        }
      }
      if constexpr (V == 1) {
        dst[at] = u[0];
        dst[at2] = v[0];
      } else {
        *reinterpret_cast<Vec*>(dst + at) = u;
        *reinterpret_cast<Vec*>(dst + at2) = v;
      }
    }
  }
}

template <typename T, int V>
sga_status launch_rotate_as(const RotateArgs& a) {
  const bool paged = a.batch.page_table != nullptr;
  RotateShape s{};
  for (int i = 0; i < a.n_tensors; ++i) s.all_heads += a.tensor[i].heads;
  const RowsArg& x = a.tensor[0];
  const bool in_place = !paged && x.src == x.dst;
  const int width = in_place ? a.rotary.channels : a.d;
  const int items = (width + 2 * V - 1) / (2 * V);
  // Tokens of a workgroup: as many as leave 1,024 workgroups, so that the sines of a long call are computed by
  // few and a short one spreads; heads: all, unless the call has fewer workgroups than the chip and a
  // workgroup more than one round of items.
  int tokens = kMaxTokens;
  while (tokens > 1 && a.n_rows / tokens < 1024) tokens >>= 1;
  int heads = s.all_heads;
  const int64_t groups = ((int64_t)a.n_rows + tokens - 1) / tokens;
  while (heads > 1 && groups * ((s.all_heads + heads - 1) / heads) < 256 && heads * items * tokens > kThreads)
    heads = (heads + 1) / 2;
  s.items = fast_div(items);
  s.heads = fast_div(heads);
  s.tokens = fast_div(tokens);
  s.heads_here = heads;
  s.head_first = x.src_head <= x.src_row;
  const dim3 grid((unsigned)(groups < kMaxGroups ? groups : kMaxGroups), (unsigned)((s.all_heads + heads - 1) / heads));
  const size_t lds = (size_t)tokens * (a.rotary.channels / 2) * sizeof(float2);
  if (paged) rotate_kernel<T, V, true><<<grid, kThreads, lds, a.stream>>>(a, s);
  else rotate_kernel<T, V, false><<<grid, kThreads, lds, a.stream>>>(a, s);
  return hip_status(hipGetLastError());
}

template <typename T>
sga_status launch_rotate_type(const RotateArgs& a) {
  constexpr int V = 16 / sizeof(T);
  bool wide = a.d % (2 * V) == 0 && a.rotary.channels % (2 * V) == 0 && a.batch.page_stride % V == 0;
  for (int i = 0; i < a.n_tensors; ++i) {
    const RowsArg& x = a.tensor[i];
    wide = wide && ((reinterpret_cast<uintptr_t>(x.src) | reinterpret_cast<uintptr_t>(x.dst)) & 15) == 0 &&
           (x.src_head | x.src_row | x.dst_head | x.dst_row) % V == 0;
  }
  return wide ? launch_rotate_as<T, V>(a) : launch_rotate_as<T, 1>(a);
}

}  // namespace

sga_status launch_rotate(const RotateArgs& a) {
  switch (a.dtype) {
    case SGA_F32: return launch_rotate_type<float>(a);
    case SGA_F16: return launch_rotate_type<f16_t>(a);
    default: return launch_rotate_type<bf16_t>(a);
  }
}

}  // namespace sga

// What a program does around a step of generation: the next step's pages (sga_pages_advance), trees of drafted tokens
// (sga_draft_tree_build) and the accepted tokens' move into place (sga_cache_keep).
#include "serving.h"

namespace sga {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

// ---- the next step's pages ---------------------------------------------------------------------------
// Sequence s had rows(s) = seq_ptr[s + 1] - seq_ptr[s] new tokens, of which kept[s] stay: l = seq_len - rows + kept.  It asks for
// want tokens more, so it needs columns ceil(l / page) .. ceil((l + want) / page) - 1 of the table; held pages from there on, wholly
// behind the window, or of a sequence that ends go back.  With P and R the sums of needed pages and wanted tokens over the sequences up to
// s, it is granted where R fits the packed rows and P what is free (or where it needs no page).  Free pages are a ring: granted
// sequences take from its front, in their order, and what goes back is put behind its end, in the order (sequence, column), so no
// place that is read is written and neither order nor result depends on how the work runs.
// A call is small: what it costs is launches and chains of dependent loads.  Two kernels: the first counts, a wavefront for each segment
// of a sequence's columns; the second sums what the first counted up to its own sequences (a few kilobytes, from L2), and then goes over the same columns
// again and writes.  It reads nothing but its own columns, the ring's front and what the first one left, so the arrays may be updated in place.
struct SequenceNote {
  int32_t length, want;      // tokens kept, tokens asked for and possible (0 otherwise)
};
struct SegmentNote {
  int32_t need, give;
};
struct PoolNote {
  int64_t first, count;
};

__device__ __forceinline__ PoolNote* pool_note(const PagesArgs& a) { return static_cast<PoolNote*>(a.workspace); }
__device__ __forceinline__ SequenceNote* sequence_notes(const PagesArgs& a) { return reinterpret_cast<SequenceNote*>(pool_note(a) + 1); }
__device__ __forceinline__ SegmentNote* segment_notes(const PagesArgs& a) {
  return reinterpret_cast<SegmentNote*>(sequence_notes(a) + a.from.n_seqs);
}

// What becomes of a sequence's columns.
struct Columns {
  int64_t length, behind;    // tokens; tokens that lie behind the window
  int32_t first_new, end;    // columns that new tokens begin, and the first that none is in
  bool ended;
  __device__ __forceinline__ Columns(const PagesArgs& a, int32_t length_, int32_t want, bool ended_) {
    const int64_t page = a.from.page.value;
    length = length_;
    ended = ended_;
    const int64_t top = a.from.pages_per_seq, f = (length + page - 1) / page, e = (length + want + page - 1) / page;
    first_new = (int32_t)(f < top ? f : top);
    end = (int32_t)(e < top ? e : top);
    behind = a.give_back ? length - a.window : INT64_MIN;
  }
  // an entry's fate: it goes back, or (want > 0 is what makes end > first_new) its column needs a page
  __device__ __forceinline__ bool gives(const PagesArgs& a, int32_t column, bool held) const {
    const int64_t from = (int64_t)column * a.from.page.value;
    return held && (ended || column >= end || (from + a.from.page.value <= behind && from >= a.n_global));
  }
  __device__ __forceinline__ bool needs(int32_t column, bool held) const { return !held && column >= first_new && column < end; }
};

__device__ __forceinline__ int32_t entry_of(const PagesArgs& a, int32_t s, int32_t column) {
  return a.from.page_table[(int64_t)s * a.from.pages_per_seq + column];
}

__global__ __launch_bounds__(kThreads) void pages_count_kernel(PagesArgs a) {
  const int lane = threadIdx.x & (kWave - 1);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const int64_t n = a.from.n_pages;
    int64_t first = a.state[0] % n, count = a.state[1];
    first = first < 0 ? first + n : first;
    count = count < 0 ? 0 : count < n ? count : n;
    *pool_note(a) = PoolNote{first, count};
  }
  const int64_t units = (int64_t)a.from.n_seqs * a.segments;
  for (int64_t unit = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; unit < units; unit += (int64_t)gridDim.x * kWaves) {
    const int32_t s = (int32_t)(unit / a.segments), segment = (int32_t)(unit - (int64_t)s * a.segments);
    int64_t length = a.from.seq_len[s];
    length = length < 0 ? 0 : length;
    if (a.kept) {
      int64_t rows = a.from.seq_ptr[s + 1] - a.from.seq_ptr[s], kept = a.kept[s];
      rows = rows < 0 ? 0 : rows < length ? rows : length;
      kept = kept < 0 ? 0 : kept < rows ? kept : rows;
      length += kept - rows;
    }
    const int32_t ask = a.ask[s];
    const bool ended = ask < 0;
    if (ended) length = 0;
    const int32_t want = ask > 0 && length + ask <= (int64_t)a.from.pages_per_seq * a.from.page.value ? ask : 0;
    const Columns columns(a, (int32_t)length, want, ended);
    const int32_t begin = segment * a.per_segment, end = min(begin + a.per_segment, a.from.pages_per_seq);
    int32_t need = 0, give = 0;
#pragma unroll 4
    for (int32_t c = begin + lane; c < end; c += kWave) {
      const bool held = (uint32_t)entry_of(a, s, c) < a.from.n_pages;
      need += columns.needs(c, held);
      give += columns.gives(a, c, held);
    }
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      need += __shfl_xor(need, off, kWave);
      give += __shfl_xor(give, off, kWave);
    }
    if (lane == 0) {
      segment_notes(a)[unit] = SegmentNote{need, give};
      if (segment == 0) sequence_notes(a)[s] = SequenceNote{(int32_t)length, ended ? -1 : want};
    }
  }
}

__device__ __forceinline__ int64_t sum_up(int64_t x, int64_t (&parts)[kWaves], int64_t& all) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int64_t below = (int64_t)__shfl_up((unsigned long long)x, off, kWave);
    if (lane >= off) x += below;
  }
  __syncthreads();                    // the last sum's readers are done
  if (lane == kWave - 1) parts[wave] = x;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) x += parts[w];
    all += parts[w];
  }
  return x;
}

__global__ __launch_bounds__(kThreads) void pages_write_kernel(PagesArgs a, int32_t units_per_group) {
  __shared__ int64_t parts[kWaves];
  struct Place {
    int64_t rows, pages, given;       // before the sequence
    int32_t granted;
  };
  __shared__ Place places[kThreads];  // of the sequences of the current chunk
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const PoolNote pool = *pool_note(a);
  const int64_t n = a.from.n_pages, page = a.from.page.value;
  const int64_t units = (int64_t)a.from.n_seqs * a.segments;
  const int64_t unit0 = (int64_t)blockIdx.x * units_per_group, unit1 = min(unit0 + units_per_group, units);
  if (unit0 >= units) return;
  const bool last = unit1 == units;
  const int32_t last_seq = (int32_t)((unit1 - 1) / a.segments);
  int64_t rows = 0, wanted = 0, pages = 0, taken = 0, given = 0;       // over the chunks before
  int64_t unit = unit0;
  for (int32_t chunk = 0; chunk <= last_seq; chunk += kThreads) {
    const int32_t s = chunk + tid;
    SequenceNote note{0, 0};
    int64_t need = 0, give = 0;
    if (s < a.from.n_seqs) {
      note = sequence_notes(a)[s];
      for (int i = 0; i < a.segments; ++i) {
        const SegmentNote x = segment_notes(a)[(int64_t)s * a.segments + i];
        need += x.need;
        give += x.give;
      }
    }
    const int64_t want = note.want > 0 ? note.want : 0;
    int64_t all_need, all_want, all_rows, all_taken, all_give;
    const int64_t need_up = pages + sum_up(need, parts, all_need), want_up = wanted + sum_up(want, parts, all_want);
    const bool granted = want > 0 && want_up <= a.from.n_tokens && (need == 0 || need_up <= pool.count);
    const int64_t rows_up = rows + sum_up(granted ? want : 0, parts, all_rows);
    const int64_t taken_up = taken + sum_up(granted ? need : 0, parts, all_taken);
    const int64_t give_up = given + sum_up(give, parts, all_give);
    places[tid] = Place{rows_up - (granted ? want : 0), taken_up - (granted ? need : 0), give_up - give, granted};
    __syncthreads();
    // the workgroup's units of these sequences, a wavefront each
    for (int64_t u = unit + wave; u < unit1 && u < (int64_t)(chunk + kThreads) * a.segments; u += kWaves) {
      const int32_t seq = (int32_t)(u / a.segments), segment = (int32_t)(u - (int64_t)seq * a.segments);
      const Place at = places[seq - chunk];
      const SequenceNote mine = sequence_notes(a)[seq];
      const int32_t want_here = mine.want > 0 ? mine.want : 0;
      const Columns columns(a, mine.length, want_here, mine.want < 0);
      int64_t take = at.pages, back = at.given;
      for (int i = 0; i < segment; ++i) {
        const SegmentNote x = segment_notes(a)[(int64_t)seq * a.segments + i];
        take += x.need;
        back += x.give;
      }
      if (segment == 0 && lane == 0) {
        a.seq_ptr[seq] = at.rows;
        a.seq_len[seq] = mine.length + (at.granted ? want_here : 0);
      }
      const int32_t begin = segment * a.per_segment, end = min(begin + a.per_segment, a.from.pages_per_seq);
      for (int32_t c0 = begin; c0 < end; c0 += kWave) {
        const int32_t c = c0 + lane;
        int32_t entry = c < end ? entry_of(a, seq, c) : -1;
        const bool held = c < end && (uint32_t)entry < a.from.n_pages;
        const bool gives = columns.gives(a, c, held), needs = c < end && columns.needs(c, held);
        const uint64_t giving = __ballot(gives), needing = __ballot(needs), below = (uint64_t(1) << lane) - 1;
        if (gives) {
          const int64_t r = pool.count + back + __popcll(giving & below);
          if (r < n) {                                 // (a page that stands in two tables comes back twice)
            int64_t where = pool.first + r;
            a.ring[where < n ? where : where - n] = entry;
          }
          entry = -1;
        }
        if (needs && at.granted) {
          int64_t where = pool.first + take + __popcll(needing & below);
          entry = a.ring[where < n ? where : where - n];
        }
        if (c < end) a.page_table[(int64_t)seq * a.from.pages_per_seq + c] = entry;
        back += __popcll(giving);
        take += __popcll(needing);
        if (at.granted && (a.positions || a.slots)) {
          // the new tokens in these columns
          const int64_t from = max((int64_t)mine.length, c0 * page), to = min((int64_t)mine.length + want_here, min((int64_t)c0 + kWave, (int64_t)end) * page);
          for (int64_t p0 = from; p0 < to; p0 += kWave) {
            const int64_t p = p0 + lane;
            const uint32_t column = quotient((uint32_t)p, a.from.page);
            const int32_t held_by = __shfl(entry, (int)(column - (uint32_t)c0) & (kWave - 1), kWave);
            if (p < to) {
              const int64_t row = at.rows + p - mine.length;
              if (a.positions) a.positions[row] = p;
              if (a.slots) a.slots[row] = (uint32_t)held_by < a.from.n_pages ? (int64_t)held_by * page + (p - (int64_t)column * page) : -1;
            }
          }
        }
      }
    }
    const int64_t done = (int64_t)(chunk + kThreads) * a.segments;
    if (unit < done) unit = done < unit1 ? done : unit1;
    rows += all_rows;
    wanted += all_want;
    pages += all_need;
    taken += all_taken;
    given += all_give;
  }
  if (last && tid == 0) {
    a.seq_ptr[a.from.n_seqs] = rows;
    const int64_t first = pool.first + taken;
    a.state_out[0] = first < n ? first : first - n;
    a.state_out[1] = (pool.count + given < n ? pool.count + given : n) - taken;
  }
}

__global__ void pages_nothing_kernel(PagesArgs a) {
  a.seq_ptr[0] = 0;
  const int64_t n = a.from.n_pages;
  int64_t first = a.state[0] % n, count = a.state[1];
  a.state_out[0] = first < 0 ? first + n : first;
  a.state_out[1] = count < 0 ? 0 : count < n ? count : n;
}
}  // namespace

void plan_pages(PagesArgs& a) {
  // as many wavefronts as keep the chip's memory busy, as far as a sequence has columns
  const int64_t S = a.from.n_seqs > 0 ? a.from.n_seqs : 1, C = a.from.pages_per_seq;
  int64_t segments = 1024 / S;
  segments = segments < 1 ? 1 : segments > 16 ? 16 : segments;
  int64_t per = (C + segments - 1) / segments;
  per = (per + kWave - 1) / kWave * kWave;
  a.per_segment = (int32_t)per;
  a.segments = (int32_t)((C + per - 1) / per);
}

size_t pages_workspace(const PagesArgs& a) {
  return sizeof(PoolNote) + (size_t)a.from.n_seqs * (sizeof(SequenceNote) + (size_t)a.segments * sizeof(SegmentNote));
}

sga_status launch_pages(const PagesArgs& a) {
  if (a.from.n_seqs == 0) {
    pages_nothing_kernel<<<1, 1, 0, a.stream>>>(a);
    return hip_status(hipGetLastError());
  }
  const int64_t units = (int64_t)a.from.n_seqs * a.segments;
  const int64_t groups = (units + kWaves - 1) / kWaves;
  pages_count_kernel<<<(unsigned)(groups < 65536 ? groups : 65536), kThreads, 0, a.stream>>>(a);
  // (a workgroup sums up all sequences before its own: no more than 1,024 of them do)
  int64_t per = (groups + 1023) / 1024 * kWaves;
  pages_write_kernel<<<(unsigned)((units + per - 1) / per), kThreads, 0, a.stream>>>(a, (int32_t)per);
  return hip_status(hipGetLastError());
}

// ---- trees of drafted tokens ---------------------------------------------------------------------------
// A token's ancestors by doubling: with J_k the 2^k-th ancestor, A_k the ancestors nearer than that and itself as bits, and D_k their number,
//   A_{k+1}(t) = A_k(t) | A_k(J_k(t)),   J_{k+1}(t) = J_k(J_k(t)),   D_{k+1}(t) = D_k(t) + D_k(J_k(t)),
// which takes log2 of the depth steps whatever the tree looks like.  Then what the mask hides of them, by the depths, is taken out.
namespace {

// Parent of token t: an entry that is no earlier token stands for the last token of the context.
__device__ __forceinline__ int32_t parent_of(const TreeArgs& a, int32_t row, int32_t t) {
  const int32_t p = a.parent[row];
  return p >= 0 && p < t ? p : -1;
}

// Whether the mask lets a token at depth i of a sequence with `base` tokens before the new ones see an ancestor at depth j.
__device__ __forceinline__ bool mask_lets(const TreeArgs& a, int64_t base, int32_t i, int32_t j) {
  const int64_t p = base + i, q = base + j;
  if (p < 0 || p >= a.L || q < 0) return false;
  return (int64_t)i - j <= a.window || q < a.n_global || p < a.n_global;
}

// Up to 64 tokens a sequence: a wavefront each, a lane a token, bits in registers.
__global__ __launch_bounds__(kThreads) void tree_wave_kernel(TreeArgs a) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int64_t s_ = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; s_ < a.batch.n_seqs; s_ += (int64_t)gridDim.x * kWaves) {
    const int32_t s = (int32_t)s_, begin = row_of_sequence(a.batch, s), rows = row_of_sequence(a.batch, s + 1) - begin;
    if (rows <= 0) continue;
    const int32_t most = 32 * a.words, n = rows < most ? rows : most;
    const int64_t base = (int64_t)a.batch.seq_len[s] - rows;
    const bool mine = lane < n;
    int32_t jump = mine ? parent_of(a, begin + lane, lane) : -1;
    uint64_t bits = uint64_t(1) << lane;
    int32_t depth = jump >= 0 ? 1 : 0;
    while (__any(jump >= 0)) {
      const int from = jump >= 0 ? jump : lane;
      const uint64_t theirs = (uint64_t)__shfl((unsigned long long)bits, from, kWave);
      const int32_t above = __shfl(depth, from, kWave), next = __shfl(jump, from, kWave);
      if (jump >= 0) {
        bits |= theirs;
        depth += above;
        jump = next;
      }
    }
    // (depths behind the tokens are 0)
    const int64_t p = base + depth;
    if (p < 0 || p >= a.L) bits = 0;
    if (__any(mine && bits && (depth > a.window || base < 0))) {
      for (int j = 0; j < n; ++j) {
        const int32_t at = __builtin_amdgcn_readlane(depth, j);
        if (!mask_lets(a, base, depth, at)) bits &= ~(uint64_t(1) << j);
      }
    }
    if (mine) {
      const int32_t row = begin + lane;
      a.depth[row] = depth;
      a.seen[(int64_t)row * a.words] = (uint32_t)bits;
      if (a.words > 1) a.seen[(int64_t)row * a.words + 1] = (uint32_t)(bits >> 32);
    }
    for (int32_t t = most + lane; t < rows; t += kWave) {       // no room in the tree
      const int32_t row = begin + t;
      a.depth[row] = -1;
      for (int w = 0; w < a.words; ++w) a.seen[(int64_t)row * a.words + w] = 0;
    }
  }
}

// Larger trees: a workgroup each, bits in LDS.
constexpr int kMostWords = 16;
__global__ __launch_bounds__(kThreads) void tree_group_kernel(TreeArgs a) {
  __shared__ int32_t jump[2][32 * kMostWords], depth[2][32 * kMostWords];
  __shared__ uint32_t bits[32 * kMostWords * kMostWords];
  const int tid = threadIdx.x, words = a.words;
  for (int32_t s = blockIdx.x; s < a.batch.n_seqs; s += gridDim.x) {
    const int32_t begin = row_of_sequence(a.batch, s), rows = row_of_sequence(a.batch, s + 1) - begin;
    if (rows <= 0) continue;
    const int32_t most = 32 * words, n = rows < most ? rows : most, used = (n + 31) / 32;
    const int64_t base = (int64_t)a.batch.seq_len[s] - rows;
    __syncthreads();                                  // the sequence before is done with LDS
    for (int32_t t = tid; t < n; t += kThreads) {
      const int32_t p = parent_of(a, begin + t, t);
      jump[0][t] = p;
      depth[0][t] = p >= 0 ? 1 : 0;
    }
    for (int32_t i = tid; i < n * used; i += kThreads) {
      const int32_t t = i / used, w = i - t * used;
      bits[i] = t / 32 == w ? 1u << (t % 32) : 0u;
    }
    int now = 0;
    bool more = true;
    while (more) {
      __syncthreads();
      bool any = false;
      for (int32_t t = tid; t < n; t += kThreads) {
        const int32_t j = jump[now][t];
        jump[1 - now][t] = j >= 0 ? jump[now][j] : -1;
        depth[1 - now][t] = depth[now][t] + (j >= 0 ? depth[now][j] : 0);
        any |= j >= 0;
      }
      // (a row that another thread has already extended holds more of the same ancestors)
      for (int32_t i = tid; i < n * used; i += kThreads) {
        const int32_t t = i / used, w = i - t * used, j = jump[now][t];
        if (j >= 0 && 32 * w <= j) bits[i] |= bits[j * used + w];
      }
      now = 1 - now;
      more = __syncthreads_or(any);
    }
    for (int32_t t = tid; t < n; t += kThreads) a.depth[begin + t] = depth[now][t];
    for (int32_t i = tid; i < rows * words; i += kThreads) {
      const int32_t t = i / words, w = i - t * words;
      uint32_t x = 0;
      if (t < n && w < used) {
        x = bits[t * used + w];
        const int32_t own = depth[now][t];
        const int64_t p = base + own;
        if (p < 0 || p >= a.L) {
          x = 0;
        } else if (own > a.window || base < 0) {
          for (uint32_t left = x; left; left &= left - 1) {
            const int bit = __ffs(left) - 1;
            if (!mask_lets(a, base, own, depth[now][32 * w + bit])) x &= ~(1u << bit);
          }
        }
      }
      a.seen[(int64_t)begin * words + i] = x;
    }
    for (int32_t t = n + tid; t < rows; t += kThreads) a.depth[begin + t] = -1;
  }
}

}  // namespace

sga_status launch_tree(const TreeArgs& a) {
  if (a.words <= 2) {
    const int64_t groups = ((int64_t)a.batch.n_seqs + kWaves - 1) / kWaves;
    tree_wave_kernel<<<(unsigned)(groups < 65536 ? groups : 65536), kThreads, 0, a.stream>>>(a);
  } else {
    tree_group_kernel<<<(unsigned)(a.batch.n_seqs < 65536 ? a.batch.n_seqs : 65536), kThreads, 0, a.stream>>>(a);
  }
  return hip_status(hipGetLastError());
}

// ---- the accepted tokens' move -------------------------------------------------------------------------
// Row base + path[k] of a sequence moves to row base + k.  path[k] >= k, so a place that is written has been read by the places before
// it: a thread that takes the same bytes of a row through all k, in their order, may do so in place, and any number of
// rows that it loads before it stores them are as they were.  Memory bounds it, and at few rows the chain of table lookups, which the workgroup makes for
// kRound rows at once.
namespace {

constexpr int kRound = 64, kAtOnce = 8;

template <typename Piece>
__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a, FastDiv pieces, uint32_t total) {
  __shared__ int64_t from[kRound], to[kRound];
  const int tid = threadIdx.x;
  const PagedArgs& b = a.batch;
  for (int32_t s = blockIdx.x; s < b.n_seqs; s += gridDim.x) {
    const int64_t rows = b.seq_ptr[s + 1] - b.seq_ptr[s], base = (int64_t)b.seq_len[s] - rows;
    const int32_t count = min(a.count[s], a.path_columns);
    auto place = [&](int64_t slot) -> int64_t {
      if (slot < 0 || slot >= (int64_t)b.pages_per_seq * b.page.value) return -1;
      const uint32_t column = quotient((uint32_t)slot, b.page), page = (uint32_t)b.page_table[(int64_t)s * b.pages_per_seq + column];
      return page < b.n_pages ? (int64_t)page * a.page_bytes + (int64_t)((uint32_t)slot - column * b.page.value) * a.row_bytes : -1;
    };
    for (int32_t k0 = 0; k0 < count; k0 += kRound) {
      __syncthreads();
      if (tid < kRound) {
        const int32_t k = k0 + tid;
        int64_t x = -1, y = -1;
        if (k < count) {
          const int32_t p = a.path[(int64_t)s * a.path_columns + k];
          if (p > k && p < rows) {                         // (k itself is there already; what is no new token stays away)
            x = place(base + p);
            y = place(base + k);
          }
        }
        from[tid] = y < 0 ? -1 : x;
        to[tid] = y;
      }
      __syncthreads();
      const int32_t here = min(count - k0, kRound);
      // rows of all layers, keys and values, key heads
      for (uint32_t i = blockIdx.y * kThreads + tid; i < total; i += gridDim.y * kThreads) {
        const uint32_t row = quotient(i, pieces), at = i - row * pieces.value;
        const uint32_t half = row / (uint32_t)a.Hkv, head = row - half * (uint32_t)a.Hkv;
        char* const cache = ((half & 1) ? a.cache_v : a.cache_k) + (int64_t)(half >> 1) * a.layer_bytes + head * a.head_bytes + at * (int64_t)sizeof(Piece);
        for (int32_t k = 0; k < here; k += kAtOnce) {
          Piece x[kAtOnce];
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e)
            if (k + e < here && from[k + e] >= 0) x[e] = *reinterpret_cast<const Piece*>(cache + from[k + e]);
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e)
            if (k + e < here && from[k + e] >= 0) *reinterpret_cast<Piece*>(cache + to[k + e]) = x[e];
        }
      }
    }
  }
}

template <typename Piece>
sga_status launch_keep_as(const KeepArgs& a) {
  const uint32_t pieces = (uint32_t)(a.row_bytes / (int64_t)sizeof(Piece));
  const int64_t total = (int64_t)a.layers * 2 * a.Hkv * pieces;
  if (total >= int64_t(1) << 31) return SGA_ERR_OVERFLOW;
  int64_t across = (total + kThreads - 1) / kThreads;
  across = across < 1 ? 1 : across > 256 ? 256 : across;
  const int32_t groups = a.batch.n_seqs < 16384 ? a.batch.n_seqs : 16384;       // (a grid holds fewer than 2^32 threads)
  keep_kernel<Piece><<<dim3((unsigned)groups, (unsigned)across), kThreads, 0, a.stream>>>(a, fast_div(pieces), (uint32_t)total);
  return hip_status(hipGetLastError());
}

}  // namespace

sga_status launch_keep(const KeepArgs& a) {
  const int64_t all = (int64_t)reinterpret_cast<uintptr_t>(a.cache_k) | (int64_t)reinterpret_cast<uintptr_t>(a.cache_v) | a.layer_bytes |
                      a.head_bytes | a.row_bytes | a.page_bytes;
  if (all % 16 == 0) return launch_keep_as<uint4>(a);
  if (all % 4 == 0) return launch_keep_as<uint32_t>(a);
  return launch_keep_as<uint16_t>(a);
}

}  // namespace sga

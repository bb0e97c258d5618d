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
// A call is small: what it costs is launches, chains of dependent loads and, at hundreds of sequences, one wavefront's walk over them.  Two kernels: the first
// counts, a wavefront for each segment of a sequence's columns; in the second a sequence's first wavefront sums up what the first kernel has left of the sequences
// up to its own (16 bytes for each, from L2, two a lane at a time), while the others ask for their columns, and then each goes over the same columns again
// and writes.  It reads nothing but its own columns, the ring's front and what the first kernel left, so the arrays may be updated in place.
// Measured (us, both kernels): 64 sequences of up to 32,768 tokens, pages of 16 4.3 + 6.1; 700 of up to 40,000, 1 to 2,000 new tokens each 6.0 + 15.4 (every segment's wavefront
// summing up by itself 25 + 6, one column at a time without asking ahead 29 + 13).  Of the latter's 15.4 vector instructions take about 4; 62 % of the wavefronts' time
// is waiting, for the walk of their workgroup's first one and for its loads.
struct alignas(16) SequenceNote {
  int32_t length, want;      // tokens kept; tokens asked for and possible (0 otherwise), -1 where the sequence ends
  int32_t need, give;        // pages
};
struct alignas(8) SegmentNote {
  int32_t need, give;        // of the sequence's segments before it
};
struct alignas(16) PoolNote {
  int64_t first, count;
};

__device__ __forceinline__ PoolNote* pool_note(const PagesArgs& a) { return static_cast<PoolNote*>(a.workspace); }
__device__ __forceinline__ SequenceNote* sequence_notes(const PagesArgs& a) { return reinterpret_cast<SequenceNote*>(pool_note(a) + 1); }
__device__ __forceinline__ SegmentNote* segment_notes(const PagesArgs& a) {
  return reinterpret_cast<SegmentNote*>(sequence_notes(a) + a.from.n_seqs);
}
__device__ __forceinline__ PoolNote read_pool(const PagesArgs& a) {
  const int64_t n = a.from.n_pages;
  const int64_t first = a.state[0] % n, count = a.state[1];
  return PoolNote{first < 0 ? first + n : first, count < 0 ? 0 : count < n ? count : n};
}

// What becomes of a sequence's columns.
struct Columns {
  int32_t first_new, end;    // columns that new tokens begin, and the first that none is in (all go back where the sequence ends)
  int32_t global, behind;    // columns from `global` on and below `behind` lie behind the window
  __device__ __forceinline__ Columns(const PagesArgs& a, int32_t length, int32_t want) {
    auto below = [&](uint32_t tokens) { return (int32_t)quotient(tokens, a.from.page); };
    auto up_to = [&](uint32_t tokens) {
      const uint32_t q = quotient(tokens, a.from.page);
      return (int32_t)(q + (q * a.from.page.value != tokens));
    };
    first_new = min(up_to(length), a.from.pages_per_seq);
    end = want < 0 ? 0 : min(up_to(length + want), a.from.pages_per_seq);       // (what is asked for fits the columns)
    global = up_to(a.n_global);
    behind = a.give_back && length > a.window ? below(length - a.window) : 0;
  }
  // an entry's fate: it goes back, or (want > 0 is what makes end > first_new) its column needs a page
  __device__ __forceinline__ bool gives(int32_t column, bool held) const { return held && (column >= end || (column < behind && column >= global)); }
  __device__ __forceinline__ bool needs(int32_t column, bool held) const { return !held && column >= first_new && column < end; }
};

__device__ __forceinline__ const int32_t* row_of(const PagesArgs& a, int32_t s) {
  return a.from.page_table + (int64_t)s * a.from.pages_per_seq;
}

// Columns of a lane that are asked for at once.  (us, 8 / 4: 700 sequences 15.4 / 19.1 in the second kernel.)
constexpr int kAsked = 8;
constexpr int kMostSegments = 16;

// A workgroup has 4 or more wavefronts: the segments of a sequence, or of several.
__global__ __launch_bounds__(kWave* kMostSegments) void pages_count_kernel(PagesArgs a) {
  __shared__ SegmentNote notes[kMostSegments];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int32_t here = blockDim.x / kWave / a.segments, s = blockIdx.x * here + wave / a.segments, segment = wave % a.segments;
  if (blockIdx.x == 0 && threadIdx.x == 0) *pool_note(a) = read_pool(a);
  const bool there = s < a.from.n_seqs;
  int64_t length = 0;
  int32_t want = 0, need = 0, give = 0;
  if (there) {
    const int32_t begin = segment * a.per_segment, end = min(begin + a.per_segment, a.from.pages_per_seq);
    const int32_t* const row = row_of(a, s);
    int32_t entry[kAsked];
    auto ask = [&](int32_t from) {
#pragma unroll
      for (int i = 0; i < kAsked; ++i) {
        const int32_t c = from + i * kWave + lane;
        entry[i] = c < end ? row[c] : -1;
      }
    };
    ask(begin);
    length = a.from.seq_len[s];
    length = length < 0 ? 0 : length;
    if (a.kept) {
      int64_t rows = a.from.seq_ptr[s + 1] - a.from.seq_ptr[s], kept = a.kept[s];
      rows = rows < 0 ? 0 : rows < length ? rows : length;
      kept = kept < 0 ? 0 : kept < rows ? kept : rows;
      length += kept - rows;
    }
    const int32_t ask_for = a.ask[s];
    if (ask_for < 0) length = 0;
    want = ask_for < 0 ? -1 : length + ask_for <= (int64_t)a.from.pages_per_seq * a.from.page.value ? ask_for : 0;
    const Columns columns(a, (int32_t)length, want);
    for (int32_t c0 = begin; c0 < end; c0 += kAsked * kWave) {
      int32_t now[kAsked];
#pragma unroll
      for (int i = 0; i < kAsked; ++i) now[i] = entry[i];
      if (c0 + kAsked * kWave < end) ask(c0 + kAsked * kWave);
#pragma unroll
      for (int i = 0; i < kAsked; ++i) {
        const int32_t c = c0 + i * kWave + lane;
        const bool held = (uint32_t)now[i] < a.from.n_pages;
        need += __popcll(__ballot(c < end && columns.needs(c, held)));
        give += __popcll(__ballot(columns.gives(c, held)));
      }
    }
    if (lane == 0) notes[wave] = SegmentNote{need, give};
  }
  __syncthreads();
  if (there && lane == 0) {
    SegmentNote before{0, 0};
    for (int i = wave - segment; i < wave; ++i) {
      before.need += notes[i].need;
      before.give += notes[i].give;
    }
    segment_notes(a)[(int64_t)s * a.segments + segment] = before;
    if (segment == a.segments - 1) sequence_notes(a)[s] = SequenceNote{(int32_t)length, want, before.need + need, before.give + give};
  }
}

// Sums of what is asked for and of what goes back stop at 2^31: more tokens or pages than there can be, so that a sum that has stopped passes no
// limit.  The middle one of a + b, a and 2^31 is that, also where both have stopped and a + b is 0.  The others need not stop: a page that is needed
// holds a token that is asked for, so where the tokens fit their packed rows there are fewer than 2^31 pages, and where they do not, nothing
// is granted whatever the pages' sum is.
constexpr uint32_t kFull = 0x80000000;
template <bool kStops>
__device__ __forceinline__ uint32_t sum_of(uint32_t a, uint32_t b) {
  const uint32_t sum = a + b;
  return kStops ? max(min(sum, a), min(max(sum, a), kFull)) : sum;
}
__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return sum_of<true>(a, b); }
template <int kCtrl, int kRows, bool kStops>
__device__ __forceinline__ uint32_t with_lane(uint32_t x) {
  return sum_of<kStops>(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, kRows, 0xF, false));
}
// The sums up to each lane: within 16 lanes by shifts, then the last of 16 and of 32 to those behind them.
template <bool kStops>
__device__ __forceinline__ uint32_t sum_up(uint32_t x) {
  x = with_lane<0x111, 0xF, kStops>(x);
  x = with_lane<0x112, 0xF, kStops>(x);
  x = with_lane<0x114, 0xF, kStops>(x);
  x = with_lane<0x118, 0xF, kStops>(x);
  x = with_lane<0x142, 0xA, kStops>(x);
  return with_lane<0x143, 0xC, kStops>(x);
}
__device__ __forceinline__ uint32_t of_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

constexpr int kEach = 2;               // sequences of a lane at a time (us, 1 / 2 / 4: 700 sequences 16.9 / 15.4 / 17.6)

// A walk over all sequences' notes, a wavefront's: what the sequences of the current kEach * kWave have to themselves and before them.
struct Walk {
  int32_t end = 0;                                         // of the sequences at hand
  uint32_t rows = 0, wanted = 0, pages = 0, taken = 0, given = 0;      // before them
  SequenceNote note[kEach];
  bool granted[kEach];
  uint32_t rows_sum = 0, want_sum = 0, need_sum = 0, taken_sum = 0, give_sum = 0;      // up to and with each lane's
  uint32_t rows_up = 0, taken_up = 0, give_up = 0;         // before each lane's

  __device__ __forceinline__ void next(const PagesArgs& a, const PoolNote& pool) {
    const int lane = threadIdx.x & (kWave - 1);
    rows += of_lane(rows_sum, kWave - 1);
    taken += of_lane(taken_sum, kWave - 1);
    wanted = plus(wanted, of_lane(want_sum, kWave - 1));
    pages += of_lane(need_sum, kWave - 1);
    given = plus(given, of_lane(give_sum, kWave - 1));
    uint32_t want = 0, need = 0, give = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int32_t s = end + lane * kEach + i;
      note[i] = s < a.from.n_seqs ? sequence_notes(a)[s] : SequenceNote{0, 0, 0, 0};
      want = plus(want, max(note[i].want, 0));
      need += note[i].need;
      give = plus(give, note[i].give);
    }
    want_sum = sum_up<true>(want);
    need_sum = sum_up<false>(need);
    give_sum = sum_up<true>(give);
    // (what a lane's sequences follow: the sum up to the lane before)
    auto ahead = [&](uint32_t sum) {
      const uint32_t up = __shfl_up(sum, 1, kWave);
      return lane > 0 ? up : 0u;
    };
    uint32_t want_up = plus(wanted, ahead(want_sum)), need_up = pages + ahead(need_sum);
    give_up = plus(given, ahead(give_sum));
    uint32_t own_rows = 0, own_taken = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      want_up = plus(want_up, max(note[i].want, 0));
      need_up += note[i].need;
      granted[i] = note[i].want > 0 && want_up <= (uint32_t)a.from.n_tokens && (note[i].need == 0 || (int64_t)need_up <= pool.count);
      own_rows += granted[i] ? note[i].want : 0;
      own_taken += granted[i] ? note[i].need : 0;
    }
    // (what is granted fits n_tokens and the ring: 31 bits)
    rows_sum = sum_up<false>(own_rows);
    taken_sum = sum_up<false>(own_taken);
    rows_up = rows + rows_sum - own_rows;
    taken_up = taken + taken_sum - own_taken;
    end += kEach * kWave;
  }
};
// What a sequence's wavefronts have to know of it.
struct Granted {
  int32_t length, want;      // want: -1 where the sequence ends
  int32_t rows;              // new tokens that it gets
  uint32_t row, take, back;  // before it: packed rows, pages taken, pages given back
};

__global__ __launch_bounds__(kWave* kMostSegments) void pages_write_kernel(PagesArgs a, int32_t seqs_per_wave) {
  extern __shared__ int32_t asked_for[];                   // [wavefronts][kAsked][kWave]: what a lane has asked for (it is met in a loop)
  __shared__ Granted told[kMostSegments];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int32_t groups = blockDim.x / kWave / a.segments, S = a.from.n_seqs, group = wave / a.segments, segment = wave % a.segments;
  // this wavefront's sequences, all in the same segment of their columns; the first segment's walks over those before them
  const int64_t s0 = (int64_t)(blockIdx.x * groups + group) * seqs_per_wave;
  const int64_t n = a.from.n_pages, page = a.from.page.value;
  const int32_t begin = segment * a.per_segment, end = min(begin + a.per_segment, a.from.pages_per_seq);
  int32_t* const entries = asked_for + wave * (kAsked * kWave) + lane;
  const PoolNote pool = *pool_note(a);
  const bool moved = a.page_table != a.from.page_table;    // all entries are written, not only those that change
  Walk walk;
  for (int32_t turn = 0; turn < seqs_per_wave; ++turn) {
    const int32_t s = (int32_t)min(s0 + turn, (int64_t)S);
    auto ask = [&](int32_t from) {
      const int32_t* const row = row_of(a, s);
      int32_t entry[kAsked];
#pragma unroll
      for (int i = 0; i < kAsked; ++i) {
        const int32_t c = from + i * kWave + lane;
        entry[i] = c < end ? row[c] : -1;
      }
#pragma unroll
      for (int i = 0; i < kAsked; ++i) entries[i * kWave] = entry[i];
    };
    SegmentNote before{0, 0};
    if (s < S) {
      before = segment_notes(a)[(int64_t)s * a.segments + segment];
      ask(begin);
      if (segment == 0) {
        while (walk.end <= s) walk.next(a, pool);
        const int32_t place = s - (walk.end - kEach * kWave);
        const int owner = place / kEach, which = place % kEach;
        Granted g{0, 0, 0, walk.rows_up, walk.taken_up, walk.give_up};
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          if (i == which) {
            g.length = walk.note[i].length;
            g.want = walk.note[i].want;
            g.rows = walk.granted[i] ? g.want : 0;
          } else if (i < which) {
            g.row += walk.granted[i] ? walk.note[i].want : 0;
            g.take += walk.granted[i] ? walk.note[i].need : 0;
            g.back = plus(g.back, walk.note[i].give);
          }
        }
        if (lane == owner) {
          told[group] = g;
          a.seq_ptr[s] = g.row;
          a.seq_len[s] = g.length + g.rows;
        }
        if (s == S - 1 && lane == kWave - 1) {
          a.seq_ptr[S] = walk.rows + walk.rows_sum;
          const int64_t taken = walk.taken + walk.taken_sum, given = plus(walk.given, walk.give_sum);
          const int64_t first = pool.first + taken;
          a.state_out[0] = first < n ? first : first - n;
          a.state_out[1] = (pool.count + given < n ? pool.count + given : n) - taken;
        }
      }
    }
    __syncthreads();
    const Granted g = told[group];
    __syncthreads();                                       // (the next turn's are told in the same place)
    if (s >= S) continue;
    const int32_t length = __builtin_amdgcn_readfirstlane(g.length), asked = __builtin_amdgcn_readfirstlane(g.want);
    const int32_t new_rows = __builtin_amdgcn_readfirstlane(g.rows);
    int64_t take = (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)g.take) + before.need;
    int64_t back = (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)g.back) + before.give;
    const int64_t first_row = (uint32_t)__builtin_amdgcn_readfirstlane((int)g.row);
    const Columns columns(a, length, asked);
    for (int32_t c0 = begin; c0 < end; c0 += kAsked * kWave) {
      if (c0 > begin) ask(c0);
#pragma unroll 1
      for (int i = 0; i < kAsked; ++i) {
        const int32_t first = c0 + i * kWave, c = first + lane;
        if (first >= end) break;
        int32_t to = entries[i * kWave];
        const bool held = (uint32_t)to < a.from.n_pages;
        const bool gives = columns.gives(c, held), needs = c < end && columns.needs(c, held);
        const uint64_t giving = __ballot(gives), needing = __ballot(needs);
        if (giving) {
          if (gives) {
            const int64_t r = pool.count + back + __popcll(giving & ((uint64_t(1) << lane) - 1));
            if (r < n) {                                   // (a page that stands in two tables comes back twice)
              const int64_t where = pool.first + r;
              a.ring[where < n ? where : where - n] = to;
            }
            to = -1;
          }
          back += __popcll(giving);
        }
        if (needing) {
          if (needs && new_rows > 0) {
            const int64_t where = pool.first + take + __popcll(needing & ((uint64_t(1) << lane) - 1));
            to = a.ring[where < n ? where : where - n];
          }
          take += __popcll(needing);
        }
        if (c < end && (moved || gives || needs)) a.page_table[(int64_t)s * a.from.pages_per_seq + c] = to;
        if (new_rows > 0 && (a.positions || a.slots)) {
          // the new tokens in these columns
          const int64_t from = max((int64_t)length, first * page), stop = min((int64_t)length + new_rows, min((int64_t)first + kWave, (int64_t)end) * page);
          for (int64_t p0 = from; p0 < stop; p0 += kWave) {
            const int64_t p = p0 + lane;
            const uint32_t column = quotient((uint32_t)p, a.from.page);
            const int32_t held_by = __shfl(to, (int)(column - (uint32_t)first) & (kWave - 1), kWave);
            if (p < stop) {
              const int64_t row = first_row + p - length;
              if (a.positions) a.positions[row] = p;
              if (a.slots) a.slots[row] = (uint32_t)held_by < a.from.n_pages ? (int64_t)held_by * page + (p - (int64_t)column * page) : -1;
            }
          }
        }
      }
    }
  }
}

__global__ void pages_nothing_kernel(PagesArgs a) {
  a.seq_ptr[0] = 0;
  const PoolNote pool = read_pool(a);
  a.state_out[0] = pool.first;
  a.state_out[1] = pool.count;
}
}  // namespace

void plan_pages(PagesArgs& a) {
  // segments of about as many columns as a wavefront asks for at once
  const int64_t C = a.from.pages_per_seq;
  int64_t segments = 1;
  while (segments < kMostSegments && segments * kAsked * kWave < C) segments *= 2;
  a.segments = (int32_t)segments;
  a.per_segment = (int32_t)(((C + segments - 1) / segments + kWave - 1) / kWave * kWave);
}

size_t pages_workspace(const PagesArgs& a) {
  return sizeof(PoolNote) + (size_t)a.from.n_seqs * (sizeof(SequenceNote) + (size_t)a.segments * sizeof(SegmentNote));
}

sga_status launch_pages(const PagesArgs& a) {
  if (a.from.n_seqs == 0) {
    pages_nothing_kernel<<<1, 1, 0, a.stream>>>(a);
    return hip_status(hipGetLastError());
  }
  const int waves = a.segments > kWaves ? a.segments : kWaves, here = waves / a.segments;
  pages_count_kernel<<<(unsigned)((a.from.n_seqs + here - 1) / here), waves * kWave, 0, a.stream>>>(a);
  // (a wavefront sums up all sequences before its own: no more than 4,096 times a segment are they read)
  const int32_t each = (a.from.n_seqs + 4095) / 4096;
  pages_write_kernel<<<(unsigned)(((a.from.n_seqs + each - 1) / each + here - 1) / here), waves * kWave, waves * kAsked * kWave * sizeof(int32_t),
                       a.stream>>>(a, each);
  return hip_status(hipGetLastError());
}

// ---- trees of drafted tokens ---------------------------------------------------------------------------
// A token's ancestors by doubling: with J_k the 2^k-th ancestor, A_k the ancestors nearer than that and itself as bits, and D_k their number,
//   A_{k+1}(t) = A_k(t) | A_k(J_k(t)),   J_{k+1}(t) = J_k(J_k(t)),   D_{k+1}(t) = D_k(t) + D_k(J_k(t)),
// which takes log2 of the depth steps whatever the tree looks like.  Then what the mask hides of them, by the depths, is taken out.  Latency bounds it.  Measured (us):
// 16 trees of 5 to 16 tokens 3.0; 256 trees of 16 to 500, window 24 15.7 (256 threads a tree, the window's bits one by one 47.5): half of their tokens follow the one before,
// the middle tree is 14 deep and the deepest 30 to 39, so four to six rounds of three barriers of 16 wavefronts, and 57 % of their time is waiting.
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

// Larger trees: a workgroup each, bits in LDS.  What the window leaves of a token's ancestors, itself and those up to `window` steps away, is
// put together from the same sets on the way: window + 1 as a sum of powers of two, for each of them the set of that size at the place that the ones before
// have led to.  Only where some token's position is below n_global (or below 0), so that the window does not decide alone, are the bits looked at
// one by one.  A thread holds up to kItems words of the rows, always the same word of a row, so that nothing is divided.
constexpr int kMostWords = 16, kMostTokens = 32 * kMostWords, kTreeThreads = 1024, kItems = kMostTokens * kMostWords / kTreeThreads;
__global__ __launch_bounds__(kTreeThreads) void tree_group_kernel(TreeArgs a) {
  __shared__ int32_t jump[2][kMostTokens], depth[2][kMostTokens], reach[kMostTokens];
  __shared__ uint32_t bits[kMostTokens * kMostWords];
  const int tid = threadIdx.x, words = a.words;
  for (int32_t s = blockIdx.x; s < a.batch.n_seqs; s += gridDim.x) {
    const int32_t begin = row_of_sequence(a.batch, s), rows = row_of_sequence(a.batch, s + 1) - begin;
    if (rows <= 0) continue;
    const int32_t most = 32 * words, n = rows < most ? rows : most, used = (n + 31) / 32;
    const int64_t base = (int64_t)a.batch.seq_len[s] - rows;
    const int shift = used <= 1 ? 0 : 32 - __builtin_clz(used - 1);            // words of a row in LDS: a power of two
    const int w = tid & ((1 << shift) - 1), t0 = tid >> shift, apart = kTreeThreads >> shift;
    const bool whole_window = a.window >= n - 1, one_by_one = base < 0 || base < a.n_global;
    __syncthreads();                                  // the sequence before is done with LDS
    if (tid < n) {
      const int32_t p = parent_of(a, begin + tid, tid);
      jump[0][tid] = p;
      depth[0][tid] = p >= 0 ? 1 : 0;
      reach[tid] = tid;
    }
    uint32_t all[kItems], near[kItems];
#pragma unroll
    for (int m = 0; m < kItems; ++m) {
      const int32_t t = t0 + m * apart;
      all[m] = t < n && t / 32 == w ? 1u << (t % 32) : 0u;
      near[m] = 0;
      if (t < n) bits[(t << shift) + w] = all[m];
    }
    __syncthreads();
    int now = 0;
    // round k: `bits` holds the sets of 2^k tokens, jump[now] the 2^k-th ancestors
    for (uint32_t steps = whole_window || one_by_one ? 0u : (uint32_t)a.window + 1;; steps >>= 1) {
      const bool any = __syncthreads_or(tid < n && jump[now][tid] >= 0);
      if (steps & 1 || (!any && steps)) {             // (no jump left: the sets are whole, larger ones are the same)
#pragma unroll
        for (int m = 0; m < kItems; ++m) {
          const int32_t t = t0 + m * apart;
          if (t < n && reach[t] >= 0) near[m] |= bits[(reach[t] << shift) + w];
        }
        __syncthreads();
        if (tid < n && reach[tid] >= 0) reach[tid] = jump[now][reach[tid]];
      }
      if (!any) break;
      uint32_t more[kItems];
#pragma unroll
      for (int m = 0; m < kItems; ++m) {
        const int32_t t = t0 + m * apart, j = t < n ? jump[now][t] : -1;
        more[m] = j >= 0 ? bits[(j << shift) + w] : 0u;
      }
      if (tid < n) {
        const int32_t j = jump[now][tid];
        jump[1 - now][tid] = j >= 0 ? jump[now][j] : -1;
        depth[1 - now][tid] = depth[now][tid] + (j >= 0 ? depth[now][j] : 0);
      }
      __syncthreads();
#pragma unroll
      for (int m = 0; m < kItems; ++m) {
        const int32_t t = t0 + m * apart;
        all[m] |= more[m];
        if (t < n && more[m]) bits[(t << shift) + w] = all[m];
      }
      now = 1 - now;
    }
    if (tid < n) a.depth[begin + tid] = depth[now][tid];
    for (int32_t t = n + tid; t < rows; t += kTreeThreads) a.depth[begin + t] = -1;
#pragma unroll
    for (int m = 0; m < kItems; ++m) {
      const int32_t t = t0 + m * apart;
      if (t >= n || w >= used) continue;
      const int32_t own = depth[now][t];
      const int64_t p = base + own;
      uint32_t x = whole_window || one_by_one ? all[m] : near[m];
      if (p < 0 || p >= a.L) {
        x = 0;
      } else if (one_by_one && (own > a.window || base < 0)) {
        for (uint32_t left = x; left; left &= left - 1) {
          const int bit = __ffs(left) - 1;
          if (!mask_lets(a, base, own, depth[now][32 * w + bit])) x &= ~(1u << bit);
        }
      }
      a.seen[(int64_t)(begin + t) * words + w] = x;
    }
    // words that no token of the sequence has, and rows without room in the tree
    if (used < words)
      for (int32_t i = tid; i < n * (words - used); i += kTreeThreads)
        a.seen[(int64_t)(begin + i / (words - used)) * words + used + i % (words - used)] = 0;
    for (int64_t i = (int64_t)n * words + tid; i < (int64_t)rows * words; i += kTreeThreads) a.seen[(int64_t)begin * words + i] = 0;
  }
}

}  // namespace

sga_status launch_tree(const TreeArgs& a) {
  if (a.words <= 2) {
    const int64_t groups = ((int64_t)a.batch.n_seqs + kWaves - 1) / kWaves;
    tree_wave_kernel<<<(unsigned)(groups < 65536 ? groups : 65536), kThreads, 0, a.stream>>>(a);
  } else {
    tree_group_kernel<<<(unsigned)(a.batch.n_seqs < 65536 ? a.batch.n_seqs : 65536), kTreeThreads, 0, a.stream>>>(a);
  }
  return hip_status(hipGetLastError());
}

// ---- the accepted tokens' move -------------------------------------------------------------------------
// Row base + path[k] of a sequence moves to row base + k.  path[k] >= k, so a place that is written has been read by the places before
// it: a thread that takes the same bytes of a row through all k, in their order, may do so in place, and any number of
// rows that it loads before it stores them are as they were.  Memory bounds it, and at few rows the chain of table lookups, which the workgroup makes for
// kRound rows at once.  Workgroup i runs on XCD i % 8: the parts of a sequence's rows follow each other in the grid, so that with many layers each XCD has some layers' caches to
// itself and finds their address translations.  Measured (us): 64 sequences, up to 5 of 16 tokens, 8 heads of 128, bf16 3.9; 128 sequences, up to 30 of 20 to 100, eight layers,
// fp16 13.8 (4.9 TB/s read and written; sequences before layers in the grid 43).
namespace {

constexpr int kRound = 64;

// kRows rows' pieces at once: loaded, then stored.  (No condition within: the loads would wait for each other's.)
template <int kRows, typename Piece>
__device__ __forceinline__ void move(char* cache, const int64_t* from, const int64_t* to, Piece) {
  Piece x[kRows];
#pragma unroll
  for (int e = 0; e < kRows; ++e) x[e] = *reinterpret_cast<const Piece*>(cache + from[e]);
#pragma unroll
  for (int e = 0; e < kRows; ++e) *reinterpret_cast<Piece*>(cache + to[e]) = x[e];
}

template <typename Piece>
__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a, FastDiv pieces, uint32_t total) {
  __shared__ int64_t from[kRound], to[kRound];
  __shared__ int32_t moves;
  const int tid = threadIdx.x;
  const PagedArgs& b = a.batch;
  for (int32_t s = blockIdx.y; s < b.n_seqs; s += gridDim.y) {
    const int64_t rows = b.seq_ptr[s + 1] - b.seq_ptr[s], base = (int64_t)b.seq_len[s] - rows;
    const int32_t count = min(a.count[s], a.path_columns);
    auto place = [&](int64_t slot) -> int64_t {
      if (slot < 0 || slot >= (int64_t)b.pages_per_seq * b.page.value) return -1;
      const uint32_t column = quotient((uint32_t)slot, b.page), page = (uint32_t)b.page_table[(int64_t)s * b.pages_per_seq + column];
      return page < b.n_pages ? (int64_t)page * a.page_bytes + (int64_t)((uint32_t)slot - column * b.page.value) * a.row_bytes : -1;
    };
    for (int32_t k0 = 0; k0 < count; k0 += kRound) {
      __syncthreads();
      if (tid < kRound) {                                  // (one wavefront) the moves there are, one behind the other
        const int32_t k = k0 + tid;
        int64_t x = -1, y = -1;
        if (k < count) {
          const int32_t p = a.path[(int64_t)s * a.path_columns + k];
          if (p > k && p < rows) {                         // (k itself is there already; what is no new token stays away)
            x = place(base + p);
            y = place(base + k);
          }
        }
        const uint64_t moving = __ballot(x >= 0 && y >= 0);
        if (x >= 0 && y >= 0) {
          const int at = __popcll(moving & ((uint64_t(1) << tid) - 1));
          from[at] = x;
          to[at] = y;
        }
        if (tid == 0) moves = __popcll(moving);
      }
      __syncthreads();
      const int32_t here = __builtin_amdgcn_readfirstlane(moves);
      // rows of all layers, keys and values, key heads
      for (uint32_t i = blockIdx.x * kThreads + tid; here > 0 && i < total; i += gridDim.x * kThreads) {
        const uint32_t row = quotient(i, pieces), at = i - row * pieces.value;
        const uint32_t half = row / (uint32_t)a.Hkv, head = row - half * (uint32_t)a.Hkv;
        char* const cache = ((half & 1) ? a.cache_v : a.cache_k) + (int64_t)(half >> 1) * a.layer_bytes + head * a.head_bytes + at * (int64_t)sizeof(Piece);
        int32_t k = 0;
        for (; k + 8 <= here; k += 8) move<8>(cache, from + k, to + k, Piece{});
        if (here - k >= 4) {
          move<4>(cache, from + k, to + k, Piece{});
          k += 4;
        }
        if (here - k >= 2) {
          move<2>(cache, from + k, to + k, Piece{});
          k += 2;
        }
        if (here > k) move<1>(cache, from + k, to + k, Piece{});
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
  keep_kernel<Piece><<<dim3((unsigned)across, (unsigned)groups), kThreads, 0, a.stream>>>(a, fast_div(pieces), (uint32_t)total);
  return hip_status(hipGetLastError());
}

}  // namespace

sga_status launch_keep(const KeepArgs& a) {
  const int64_t all = (int64_t)reinterpret_cast<uintptr_t>(a.cache_k) | (int64_t)reinterpret_cast<uintptr_t>(a.cache_v) | a.layer_bytes |
                      a.head_bytes | a.row_bytes | a.page_bytes;
  if (all % 16 == 0) return launch_keep_as<vec_t<uint32_t, 4>>(a);
  if (all % 4 == 0) return launch_keep_as<uint32_t>(a);
  return launch_keep_as<uint16_t>(a);
}

}  // namespace sga

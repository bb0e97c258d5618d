// Attention of new tokens over a paged cache (sga_attention_paged), of drafted ones that form a tree too (sga_attention_tree).
//
// Two kernels: paged_kernel for short chunks, which memory bounds, and paged_chunk_kernel (below) for long ones, which the
// matrix cores bound.  In the first a tile is 16 or 32 consecutive rows of one sequence and key head, a row being a new
// token and one of the query heads that share the key head (row = token * group + head).  Keys are met in blocks of 32
// aligned ones: those of the global tokens before the window, then the window's.  Per block, with matrix instructions of
// 16 x 16 results,
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

namespace sga {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kBlock = 32;            // keys of a block
constexpr int kRows = 16;             // rows of a tile, or twice as many where a sequence brings more
constexpr int kWaves = 4;             // wavefronts of a workgroup, which take its blocks in turn
// Pieces of tiles of 128 rows that a call is cut into, three rounds of the places on the chip, and the fewest keys of one: a piece
// costs a prologue of about 4 us and a partial state of 66 KB (d = 128), eight blocks of fp32 products as much as 32 of
// 16-bit ones.  (us, bf16, 32 / 8 heads of 128: 1,024 / 1,536 / 2,048 pieces, eight chunks of 256 behind up to 16k 344 / 329 / 334;
// least piece 512 / 1,024 / 2,048 keys, 512 tokens behind 8k 128 / 111 / 98, four chunks of 64 behind 8k 106 / 64 / 64, 64 channels
// and one head per key head 69 / 70 / 121.)
constexpr int kLeastPiece = 1024, kLeastPieceF32 = 256;
// ... of drafted tokens, which come few at a time (us, least piece 1,024 / 512 / 256, bf16, 32 / 8 heads of 128: eight sequences of 12 tokens behind 500 to
// 3,000 35.7 / 26.0 / 28.8, one of 24 behind 8,000 34.2 / 28.2 / 30.4)
constexpr int kLeastPieceTree = 512;
constexpr int least_piece(bool tree, int dtype) { return dtype == SGA_F32 ? kLeastPieceF32 : tree ? kLeastPieceTree : kLeastPiece; }
constexpr int kChunkPieces = 1536;
// Drafted tokens under a window, or behind contexts of one length: the tiles of 128 rows are all alike.  Where they are more than the places on the
// chip, whole rounds of them are not cut, and what is left is cut into as many pieces as fill the places once more: fewer prologues and hardly any
// partial states.  (Key heads that share the XCDs, so that pieces start in their order.  us, whole calls with their joins, in turn on one card, cut by kChunkPieces / so: 16
// tokens of 64 and of 100 sequences under a window of 2,048, 32 / 8 heads of 128, bf16 144 / 114, 212 / 188; 30 to 200 tokens of 32 sequences under 4,096, 32 / 4 heads,
// fp16 231 / 224.)
constexpr float kAlike = 1.25f;
constexpr int kMostTreeWords = 16;

// Sequences with more rows than this on average take tiles of 128 rows.  (us, short tiles / tiles of 128 rows, 8 heads, behind 4k to 16k; bf16, 32
// sequences: 29 rows d = 64 123 / 137, d = 128 232 / 252, d = 256 427 / 504; 33 rows 191 / 142, 391 / 255, 854 / 511.  Full precision, 8 sequences, where
// a tile of 128 rows costs the same however few rows it has, since the matrix cores bound it: 33 rows d = 32 79 / 104, d = 64 123 / 191, d = 128 284 / 380;
// 64 rows d = 128 370 / 391; 80 rows 451 / 402; 96 rows d = 32 105 / 121, d = 64 169 / 199; 128 rows 127 / 118, 222 / 210; but where all of a
// sequence is 256 tokens or fewer a short tile's chain of loads is what counts: 16 sequences of 80 tokens d = 32 26 / 15, d = 64 30 / 19, the last 80 of
// 256 32 / 22, 42 / 30, of 512 32 / 31, 45 / 47.)
constexpr int token_rows(bool single, int d, int64_t tokens) { return !single || (d <= 64 && tokens <= 256) ? 32 : d > 64 ? 64 : 96; }

// Numerators of fp16 storage are kept 2^kRaise times as large as against the row's largest score: fp16 ends at 2^-25 (2^-14 with all
// its bits), and a long context can hold most of its weight in tokens that are each below that beside a few large ones.  The
// reference is that much lower, lse and sums follow from it, and nothing else changes.  Short chunks raise the reference with every larger score,
// so the largest numerator is 2^15 and what a pair of fp16 numbers loses begins 2^-40 below it; long chunks leave room for scores that grow, and
// lose 2^-35 (kMostNumerators).  (Scores from 2^24 on, whose own step is as large, may pass the end of fp16: such rows are not finite then and are
// redone in 32 bits, see attend_row.)
template <typename T>
constexpr float kRaise = sizeof(T) == 2 && !__is_same(T, bf16_t) ? 15.f : 0.f;
template <typename T>
constexpr float kChunkRaise = sizeof(T) == 2 && !__is_same(T, bf16_t) ? 10.f : 0.f;

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

// Tokens of a sequence that can be seen.  (Of a draft tree: by their places.  A new token's place may lie behind its position, so what the
// mask's L hides is left out of the tree's bits and of the context instead.)
template <bool kTree>
__device__ __forceinline__ int32_t kept_of(const PagedAttention& a, int32_t length) {
  const int64_t room = (int64_t)a.batch.pages_per_seq * a.batch.page.value;
  int64_t kept = length < 0 ? 0 : length;
  kept = kept < room ? kept : room;
  return (int32_t)(kTree || kept < a.L ? kept : a.L);
}

// Drafted tokens.  New token t of a sequence lies at place base + t of the cache, base = length - n_new, but at position base + depth(t), and
// sees of the context, the tokens before base, what the mask shows that position, and of the new tokens those whose bits are set in
// its row of `seen`.  Both kernels meet the context's keys as they do others', and the blocks that reach base as blocks at an edge, in which every key is
// tested: the bits of a block's 32 keys are two words of the row, put together.  All rows of a sequence meet the same keys.  Measured (us, whole calls with their joins, in turn with
// the same call without a tree): 5 to 16 drafts of 64 sequences behind 512 to 32,768, 32 / 8 heads of 128, bf16 417 / 415 (4.8 TB/s, as a large copy); 30 to 200 of 32
// under a window of 4,096, 32 / 4 heads, fp16 224 / 223 on one card, 219 / 218 on another (212 to 232 over six: 690 TFLOP/s of the products that the mask asks for at
// 218; the library's 1,171).
__device__ __forceinline__ Sight context_sight(const PagedAttention& a, const Tile& t, int32_t token) {
  const int32_t base = t.length - t.n_new, depth = a.depth[t.begin + token];
  const int64_t p = (int64_t)base + depth;
  if (depth < 0 || p < 0 || p >= a.L) return {0, -1, 0};
  const int32_t context = base < t.kept ? base : t.kept, last = (context < a.L ? context : a.L) - 1;
  if (p < a.n_global) return {0, last, 0};
  return {p > a.window ? (int32_t)(p - a.window) : 0, last, a.n_global < last + 1 ? a.n_global : last + 1};
}
// The row of `seen` of a token, -1 where it is none of the tree or outside the mask.
__device__ __forceinline__ int32_t tree_row(const PagedAttention& a, const Tile& t, int32_t token) {
  const int32_t depth = a.depth[t.begin + token];
  const int64_t p = (int64_t)(t.length - t.n_new) + depth;
  return depth < 0 || p < 0 || p >= a.L ? -1 : t.begin + token;
}
// Which of the keys j0 .. j0 + 31 a row sees as new tokens; seen: the row's words.
__device__ __forceinline__ uint32_t new_tokens_seen(const PagedAttention& a, const Tile& t, const uint32_t* seen, int32_t j0) {
  const int32_t start = j0 - (t.length - t.n_new), word = start >> 5, shift = start & 31;
  if (start <= -kBlock || word >= a.words || j0 >= t.kept) return 0;
  const uint32_t low = word >= 0 ? seen[word] : 0, high = shift && word + 1 < a.words ? seen[word + 1] : 0;
  const uint32_t bits = shift ? low >> shift | high << (32 - shift) : low;
  return t.kept - j0 < kBlock ? bits & ((1u << (t.kept - j0)) - 1) : bits;
}

__device__ __forceinline__ uint32_t new_tokens_seen(const PagedAttention& a, const Tile& t, int32_t row, int32_t j0) {
  return row < 0 ? 0 : new_tokens_seen(a, t, a.seen + (int64_t)row * a.words, j0);
}

template <bool kTree>
__device__ __forceinline__ Sight row_sight(const PagedAttention& a, const Tile& t, int32_t token) {
  if constexpr (kTree) return context_sight(a, t, token);
  return sight_of(a, t.length - t.n_new + token, t.kept);
}

// Tile t of a sequence.
template <int kTileRows, bool kTree>
__device__ __forceinline__ Tile tile_of(const PagedAttention& a, int32_t seq, int32_t begin, int32_t n_new, int32_t length,
                                        int32_t index) {
  Tile t;
  t.seq = seq;
  t.begin = begin;
  t.n_new = n_new;
  t.length = length;
  const int64_t left = (int64_t)n_new * a.group.value - (int64_t)index * kTileRows;
  t.first = index * kTileRows;
  t.count = left < kTileRows ? (int32_t)left : kTileRows;
  t.kept = kept_of<kTree>(a, length);
  if constexpr (kTree) {
    const int32_t start = max(length - n_new, 0), context = min(start, min(t.kept, a.L));
    t.base = (start < a.n_global || start <= a.window ? 0 : start - a.window) & ~(kBlock - 1);
    t.lead = (min(min(a.n_global, context), t.base) + kBlock - 1) / kBlock;
    t.blocks = t.lead + (t.kept > t.base ? (t.kept - 1 - t.base) / kBlock + 1 : 0);
    return t;
  }
  // the rows' keys: positions grow with the rows, and so do both ends of what they see
  const int32_t p0 = t.length - t.n_new + (int32_t)quotient((uint32_t)t.first, a.group);
  const int32_t p1 = t.length - t.n_new + (int32_t)quotient((uint32_t)(t.first + t.count - 1), a.group);
  // (rows before 0 and from L on see nothing; a global row sees from 0 on, and then so does what follows)
  const int32_t from = p0 < 0 ? 0 : p0, to = p1 < a.L ? p1 : a.L - 1;
  t.lead = t.base = t.blocks = 0;
  if (from > to) return t;
  const Sight low = sight_of(a, from, t.kept), high = sight_of(a, to, t.kept);
  // (not causal: a global row sees to the end)
  const int32_t last = low.hi > high.hi ? low.hi : high.hi;
  t.base = low.lo & ~(kBlock - 1);
  int32_t lead = low.lead > high.lead ? low.lead : high.lead;
  lead = lead < t.base ? lead : t.base;
  t.lead = (lead + kBlock - 1) / kBlock;
  t.blocks = t.lead + (last >= t.base ? (last - t.base) / kBlock + 1 : 0);
  return t;
}

// ---- the division of a call's work ---------------------------------------------------------------------------
// All work lies on one line: sequences, in each its key heads, in each its tiles, each about as long as the keys that
// it meets and kTileCost for itself.  The line is cut into equal shares, one for each workgroup that the chip holds, whatever the
// lengths of the sequences are; a cut falls inside a tile where tiles are long, and the tile's parts are then joined.
// Lengths are estimates (a tile's blocks are counted when it is met; a cut goes to the block in proportion) that follow from
// the sequence alone: tile u < t1 is a0 + u * step long, the others a1.  Causal, the keys grow with the tiles until the
// window is full; otherwise the tiles of global rows see everything and the others a window.
// (us, kTileCost 64 / 256 / 512: a step of 64 sequences of 512 to 32k tokens 371 / 359 / 362, 160 windows of 2,048 127 / 123 / 127,
// drafts at d = 256 60 / 53 / 71; kLeastShare 256 / 512 / 1,024, drafts 72 / 67 / 81.)
constexpr uint32_t kTileCost = 256;
constexpr uint32_t kLeastShare = 512;      // keys of the smallest share
constexpr uint32_t kLeastShareTree = 256;  // ... of drafted tokens (seven behind 2,000, one head of 64, fp32 512 / 256: 17.0 / 15.6 us)
constexpr uint32_t kWholeTiles = 32;       // tiles shorter than this part of a share are not cut
// ... nor are a sequence's tiles that are all shorter than this, as long as a share holds one for each wavefront: a cut costs about as much
// as the unevenness that it takes away.  (us, cut / not: 512 sequences of windows of 128, d = 64 85 / 75, 700 sequences of up to 600
// tokens 158 / 150, documents under +-128, fp32 142 / 138, causal 97 / 89; not with tiles of every length: causal prompts of
// 2,000 tokens, d = 32, 71 / 78, nor up to 32,768 keys, 358 / 394.)
constexpr uint32_t kShortTiles = 768;

__device__ __forceinline__ uint64_t quotient64(uint64_t n, uint64_t d) {
  return (n | d) >> 32 ? n / d : (uint64_t)((uint32_t)n / (uint32_t)d);
}
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((uint32_t)v, lane);
}

struct SequenceWork {
  int32_t begin, n_new, length;
  uint32_t tiles, a0, a1, t1;
  uint64_t per_head;
  // length of the first t tiles
  __device__ __forceinline__ uint64_t before(uint32_t t, uint32_t step) const {
    const uint64_t n = t < t1 ? t : t1;
    return n * a0 + (uint64_t)step * (n * (n - 1) / 2) + (uint64_t)(t - (uint32_t)n) * a1;
  }
  __device__ __forceinline__ uint32_t length_of(uint32_t t, uint32_t step) const { return t < t1 ? a0 + t * step : a1; }
};

template <int kTileRows>
__device__ __forceinline__ uint32_t step_of(const PagedAttention& a) { return a.causal ? kTileRows / a.group.value : 0; }

template <int kTileRows, bool kTree>
__device__ __forceinline__ SequenceWork work_of(const PagedAttention& a, int32_t s) {
  SequenceWork w{};
  const PagedArgs& b = a.batch;
  if (s >= b.n_seqs) return w;
  w.begin = row_of_sequence(b, s);
  const int32_t end = row_of_sequence(b, s + 1);
  w.length = max(b.seq_len[s], 0);
  w.n_new = end > w.begin ? end - w.begin : 0;
  w.tiles = (uint32_t)(((int64_t)w.n_new * a.group.value + kTileRows - 1) / kTileRows);
  if constexpr (kTree) {                     // all tiles meet the same keys
    const int64_t kept = kept_of<true>(a, w.length), reach = (int64_t)a.window + w.n_new + 1 + a.n_global;
    w.a0 = w.a1 = (uint32_t)(reach < kept ? reach : kept) + kTileCost;
    w.per_head = (uint64_t)w.tiles * w.a1;
    return w;
  }
  const int64_t kept = kept_of<kTree>(a, w.length), old = (int64_t)w.length - w.n_new, step = kTileRows / a.group.value;
  int64_t window = (a.causal ? 1 : 2) * (int64_t)a.window + step + 1 + a.n_global;
  window = window < kept ? window : kept;
  w.a1 = (uint32_t)window + kTileCost;
  if (a.causal) {
    int64_t first = old + step + 1;
    first = first < 0 ? 0 : first < window ? first : window;
    w.a0 = (uint32_t)first + kTileCost;
    if (step > 0 && first < window) {
      const int64_t ramp = (window - first + step - 1) / step;
      w.t1 = ramp < w.tiles ? (uint32_t)ramp : w.tiles;
    } else {
      w.a0 = w.a1;
    }
  } else {
    w.a0 = (uint32_t)kept + kTileCost;
    if (old < a.n_global) {
      const int64_t global = ((a.n_global - (old < 0 ? 0 : old)) * (int64_t)a.group.value + kTileRows - 1) / kTileRows;
      w.t1 = global < w.tiles ? (uint32_t)global : w.tiles;
    }
  }
  w.per_head = w.before(w.tiles, (uint32_t)(a.causal ? step : 0));
  return w;
}

// The thread's index, as if read anew: what follows from it is not kept in registers from one part of a share to the next.
__device__ __forceinline__ int thread_again() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// A part of a tile that a share holds: [from, to) of the tile's length `extent`.
struct Part {
  int32_t seq, begin, n_new, length, tile, head;
  uint32_t from, to, extent;
  int32_t there;             // 2: a wavefront's work, 1: the workgroup's
};

// A workgroup's walk along its share.  It lies in LDS, since it is needed between the parts only; the first wavefront
// walks, all its lanes with the same values but where they load a sequence each.
template <int kTileRows, bool kTree>
struct Share {
  SequenceWork work[kWave];  // sequences chunk ..
  uint64_t start[kWave];     // where each begins on the line
  uint64_t behind;           // where the last one ends
  uint64_t at, end, size;    // what is left of the share, and a whole one
  int32_t chunk, lane;       // the current sequence is chunk + lane
  uint32_t head, tile, offset, extent;     // current tile, the place in it, its length
  Part part[kWaves];         // what the workgroup does next: one part, or a whole tile for each wavefront
  int32_t parts, pending;    // how many; and whether the current tile's part is found but not done (it is `ahead`)
  Part ahead;

  // 64 sequences from `from` on, which begins at `base` on the line
  __device__ __forceinline__ void load(const PagedAttention& a, int32_t from, uint64_t base) {
    const int l = threadIdx.x & (kWave - 1);
    const SequenceWork w = work_of<kTileRows, kTree>(a, from + l);
    const uint64_t own = w.per_head * (uint64_t)a.Hkv;
    uint64_t sum = own;
    for (int off = 1; off < kWave && off < a.batch.n_seqs; off <<= 1) {
      const uint64_t below = (uint64_t)__shfl_up((unsigned long long)sum, off, kWave);
      if (l >= off) sum += below;
    }
    work[l] = w;
    chunk = from;
    const int32_t here = min(a.batch.n_seqs - from, kWave);
    behind = base + from_lane(sum, here - 1);
    start[l] = l < here ? base + sum - own : behind;
    __builtin_amdgcn_wave_barrier();
  }
  __device__ __forceinline__ void take_sequence() {
    lane = 63 - __builtin_clzll(__ballot(start[threadIdx.x & (kWave - 1)] <= at) | 1);
  }
  // Finds the place `at`.
  __device__ __forceinline__ void locate(const PagedAttention& a, uint32_t step) {
    take_sequence();
    const SequenceWork& now = work[lane];
    const uint64_t in_seq = at - start[lane];
    head = (uint32_t)quotient64(in_seq, now.per_head);
    const uint64_t in_head = in_seq - head * now.per_head, ramp = now.before(now.t1, step);
    if (in_head >= ramp) {
      tile = now.t1 + (uint32_t)quotient64(in_head - ramp, now.a1);
    } else {
      uint32_t low = 0, high = now.t1;        // before(low) <= in_head < before(high)
      while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if (now.before(mid, step) <= in_head) low = mid; else high = mid;
      }
      tile = low;
    }
    offset = (uint32_t)(in_head - now.before(tile, step));
    extent = now.length_of(tile, step);
  }
  __device__ __forceinline__ bool whole() const {
    const bool all_short = extent < kShortTiles && work[lane].a1 < kShortTiles;
    return (uint64_t)extent * (all_short ? kWaves : kWholeTiles) < size;
  }

  // Share i of the call.  False: there is nothing in it.
  __device__ __forceinline__ bool begin(const PagedAttention& a, uint32_t i) {
    // once over the sequences for the line's length, and if they are not all at hand then, again up to the place
    const int32_t n = a.batch.n_seqs;
    uint64_t base = 0;
    bool counted = false;
    for (int32_t c = 0;;) {
      load(a, c, base);
      base = behind;
      c += kWave;
      if (!counted) {
        if (c < n) continue;
        const uint64_t total = base;
        uint64_t each = total;
        if (a.groups > 1) {
          each = quotient64(total + a.groups - 1, a.groups);
          const uint32_t least = kTree ? kLeastShareTree : kLeastShare;
          each = each > least ? each : least;
        }
        size = each;
        at = each * i;
        end = at + each < total ? at + each : total;
        if (at >= total) return false;
        if (n <= kWave) break;
        counted = true;
        base = 0;
        c = 0;
      } else if (base > at || c >= n) {
        break;
      }
    }
    if (i > 0) {
      locate(a, step_of<kTileRows>(a));
    } else {
      take_sequence();
      head = tile = offset = 0;
      extent = work[lane].length_of(0, step_of<kTileRows>(a));
    }
    return true;
  }
  // The part of the current tile that is in the share, if any.
  __device__ __forceinline__ void find_part(const PagedAttention& a) {
    const bool uncut = !a.partials || whole();
    if (uncut && offset > 0) {              // the share begins inside a tile that is not cut: with its beginning
      at -= offset;
      offset = 0;
    }
    pending = 0;
    if (at >= end) return;
    const uint64_t left = end - at;
    const uint32_t to = offset + left < extent ? offset + (uint32_t)left : extent;
    if (uncut && to < extent) return;
    const SequenceWork& now = work[lane];
    if (tile >= now.tiles || head >= (uint32_t)a.Hkv) return;          // (lengths that change while the call runs)
    ahead = Part{chunk + lane, now.begin, now.n_new, now.length, (int32_t)tile, (int32_t)head, offset, to, extent, 1};
    pending = 1;
  }
  // Goes on behind the part found.
  __device__ __forceinline__ void advance(const PagedAttention& a) {
    at += ahead.to - offset;
    offset = 0;
    if (at < end) {
      if (++tile == work[lane].tiles) {
        tile = 0;
        if (++head == (uint32_t)a.Hkv) {
          head = 0;
          while (at >= behind && chunk + kWave < a.batch.n_seqs) load(a, chunk + kWave, behind);
          take_sequence();
        }
      }
      extent = work[lane].length_of(tile, step_of<kTileRows>(a));
    }
    find_part(a);
  }
  // A whole tile that is short against the share is one wavefront's work: four of them then wait for memory and for their
  // first keys at the same time, and none waits for the others' keys.
  __device__ __forceinline__ bool alone() const {
    return ahead.from == 0 && ahead.to == extent && (uint64_t)extent * kWaves <= size;
  }
  // What the workgroup with share i does first, or next; all wavefronts call it.  False: nothing is left.
  __device__ __forceinline__ bool next(const PagedAttention& a, uint32_t i, bool first) {
    if (threadIdx.x < kWave) {
      pending = first ? 0 : pending;
      parts = 0;
      if (first && begin(a, i)) find_part(a);
      bool more = true;
      while (more && pending) {
        const bool single = alone();
        if (parts > 0 && !single) break;
        part[parts] = ahead;
        part[parts].there = single ? 2 : 1;
        ++parts;
        more = single && parts < kWaves;
        advance(a);
      }
    }
    __syncthreads();
    return parts > 0;
  }
  __device__ __forceinline__ Part mine(int i) const {
    const Part& q = part[i];
    Part p;
    p.seq = __builtin_amdgcn_readfirstlane(q.seq);
    p.begin = __builtin_amdgcn_readfirstlane(q.begin);
    p.n_new = __builtin_amdgcn_readfirstlane(q.n_new);
    p.length = __builtin_amdgcn_readfirstlane(q.length);
    p.tile = __builtin_amdgcn_readfirstlane(q.tile);
    p.head = __builtin_amdgcn_readfirstlane(q.head);
    p.from = __builtin_amdgcn_readfirstlane(q.from);
    p.to = __builtin_amdgcn_readfirstlane(q.to);
    p.extent = __builtin_amdgcn_readfirstlane(q.extent);
    p.there = __builtin_amdgcn_readfirstlane(q.there);
    return p;
  }
};

// Blocks [first, end) of a tile that the part [from, to) of its length `extent` stands for.
__device__ __forceinline__ int32_t block_at(uint32_t place, uint32_t extent, int32_t blocks) {
  if (place == 0) return 0;
  if (place >= extent) return blocks;
  return (int32_t)quotient64((uint64_t)place * (uint32_t)blocks, extent);
}

// A partial state of a tile: O [rows][D], then the rows' references and sums.
template <int D, int kTileRows>
__device__ __forceinline__ float* record_of(const PagedAttention& a, int64_t i) {
  return a.partials + i * (kTileRows * (D + 2));
}
// Each share has two, of the tile that it begins within and of the one that it ends within.
template <int D, int kTileRows>
__device__ __forceinline__ float* record_of_share(const PagedAttention& a, uint32_t share, bool begins_within) {
  return record_of<D, kTileRows>(a, (int64_t)share * 2 + (begins_within ? 0 : 1));
}
// What a workgroup leaves for the kernel that joins: a tile and its parts.
struct alignas(16) Note {
  int32_t count;             // parts of the tile; 0: nothing to join here
  int32_t first;             // the first one's share or record
  int32_t apart;             // (tiles of 128 rows) from a part's record to the next one's
  int32_t begin, n_new, length, tile, head;
};
static_assert(sizeof(Note) == kNoteBytes, "the plan counts on this");
__device__ __forceinline__ Note* notes_of(const PagedAttention& a) { return reinterpret_cast<Note*>(a.notes); }

// Wavefronts per SIMD that registers and the ring of blocks leave to tiles of 128 rows.
__host__ __device__ constexpr int chunk_waves(int row_bytes) { return row_bytes > 256 ? 1 : row_bytes > 128 ? 2 : 3; }

// Which piece of which tile of 128 rows workgroup `rest` of a key head has.  Not causal, a sequence's first tiles may hold global
// rows, which see everything, and the others see a window; causal, all count as its longest one.  The tiles of
// a kind are all cut into as many pieces as make them about the size at which the call has kChunkPieces of them
// (as far as the lengths say; kLeastPiece keys at least), so that uneven sequences keep the chip evenly busy.  The pieces lie in
// the order sequence, kind, piece, tile; the pieces of a tile are `apart` from each other.  False: there is no such piece.  All lanes call it.
template <int kTileRows, bool kTree>
__device__ __forceinline__ bool piece_of(const PagedAttention& a, int32_t rest, Tile& tile, int32_t& index, int32_t& piece,
                                         int32_t& pieces, int32_t& apart) {
  const int l = threadIdx.x & (kWave - 1);
  const int32_t n = a.batch.n_seqs;
  SequenceWork w{};
  int32_t all = 0, rows = 0;                 // tiles that see everything, the others
  float all_length = 0.f, length = 0.f;
  auto look = [&](int32_t s) {
    w = work_of<kTileRows, kTree>(a, s);
    all = a.causal ? 0 : (int32_t)w.t1;
    rows = (int32_t)w.tiles - all;
    all_length = (float)w.a0;
    length = (float)(a.causal && w.t1 > 0 ? max(w.a1, w.length_of(w.t1 - 1, step_of<kTileRows>(a))) : w.a1);
  };
  float total = 0.f, longest = 0.f;
  int32_t tiles = 0;
  for (int32_t c = 0; c < n; c += kWave) {
    look(c + l);
    total += (float)all * all_length + (float)rows * length;
    if constexpr (kTree) {
      tiles += rows;
      longest = fmaxf(longest, rows > 0 ? length : 0.f);
    }
  }
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) total += __shfl_xor(total, off, kWave);
  if constexpr (kTree) {
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      tiles += __shfl_xor(tiles, off, kWave);
      longest = fmaxf(longest, __shfl_xor(longest, off, kWave));
    }
    tiles = __builtin_amdgcn_readfirstlane(tiles);
    const float most = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, longest)));
    const bool alike = __builtin_amdgcn_readfirstlane(longest * (float)tiles <= kAlike * total);
    const int32_t places = 256 * chunk_waves(a.d * (a.dtype == SGA_F32 ? 4 : 2)), whole = tiles * a.Hkv / places * places / a.Hkv;
    if (a.splits > 1 && 8 % a.Hkv == 0 && whole > 0 && alike) {
      const int32_t left = tiles - whole;
      int32_t ordinal = rest;                               // of the tile, over the sequences
      piece = 0;
      pieces = 1;
      apart = max(left, 1);
      if (rest >= whole) {
        if (left == 0) return false;
        pieces = max(1, min(places / (left * a.Hkv), (int32_t)__builtin_amdgcn_readfirstlane((int)(most / (float)least_piece(true, a.dtype)))));
        piece = (rest - whole) / left;
        if (piece >= pieces) return false;
        ordinal = whole + (rest - whole) - piece * left;
      }
      int32_t behind = 0;
      for (int32_t c = 0; c < n; c += kWave) {
        if (n > kWave) look(c + l);
        int32_t sum = rows;
        for (int off = 1; off < kWave && off < n; off <<= 1) {
          const int32_t below = __shfl_up(sum, off, kWave);
          if (l >= off) sum += below;
        }
        const uint64_t begun = __ballot(rows > 0 && behind + sum - rows <= ordinal && ordinal < behind + sum);
        if (begun) {
          const int lane = __builtin_ctzll(begun);
          index = ordinal - behind - __builtin_amdgcn_readlane(sum - rows, lane);
          tile = tile_of<kTileRows, kTree>(a, c + lane, __builtin_amdgcn_readlane(w.begin, lane), __builtin_amdgcn_readlane(w.n_new, lane),
                                           __builtin_amdgcn_readlane(w.length, lane), index);
          return true;
        }
        behind += __builtin_amdgcn_readlane(sum, min(n - c, kWave) - 1);
      }
      return false;
    }
  }
  const float size = fmaxf((float)least_piece(kTree, a.dtype), total * (float)a.Hkv * (1.f / kChunkPieces));
  auto cuts = [&](float x) { return a.splits > 1 ? max(1, (int32_t)(x / size + 0.5f)) : 1; };
  int32_t behind = 0;
  for (int32_t c = 0; c < n; c += kWave) {
    if (n > kWave) look(c + l);
    const int32_t all_cuts = cuts(all_length), row_cuts = cuts(length), own = all * all_cuts + rows * row_cuts;
    int32_t sum = own;
    for (int off = 1; off < kWave && off < n; off <<= 1) {
      const int32_t below = __shfl_up(sum, off, kWave);
      if (l >= off) sum += below;
    }
    const uint64_t begun = __ballot(own > 0 && behind + sum - own <= rest && rest < behind + sum);
    if (begun) {
      const int lane = __builtin_ctzll(begun);
      const int32_t first = __builtin_amdgcn_readlane(all, lane), first_cuts = __builtin_amdgcn_readlane(all_cuts, lane);
      int32_t place = rest - behind - __builtin_amdgcn_readlane(sum - own, lane);
      const bool in_first = place < first * first_cuts;
      pieces = in_first ? first_cuts : __builtin_amdgcn_readlane(row_cuts, lane);
      apart = in_first ? first : __builtin_amdgcn_readlane(rows, lane);
      place -= in_first ? 0 : first * first_cuts;
      piece = (int32_t)((uint32_t)place / (uint32_t)apart);
      index = place - piece * apart + (in_first ? 0 : first);
      tile = tile_of<kTileRows, kTree>(a, c + lane, __builtin_amdgcn_readlane(w.begin, lane), __builtin_amdgcn_readlane(w.n_new, lane),
                                __builtin_amdgcn_readlane(w.length, lane), index);
      return true;
    }
    behind += __builtin_amdgcn_readlane(sum, min(n - c, kWave) - 1);
  }
  return false;
}

__device__ __forceinline__ int32_t first_key(const Tile& t, int32_t block) {
  return block < t.lead ? block * kBlock : t.base + (block - t.lead) * kBlock;
}
// Element offset of token j's row within a key head of the cache, -1 if it has no page.  (j may lie behind the last token,
// up to a block's end.)
__device__ __forceinline__ int64_t place_of(const PagedArgs& b, int32_t seq, int32_t j, int32_t d) {
  const uint32_t column = quotient((uint32_t)j, b.page);
  if (column >= (uint32_t)b.pages_per_seq) return -1;
  const uint32_t page = (uint32_t)b.page_table[(int64_t)seq * b.pages_per_seq + column];
  return page < b.n_pages ? (int64_t)page * b.page_stride + (int64_t)((uint32_t)j - column * b.page.value) * d : -1;
}

// Operands of 16-bit storage: eight values of a lane per product of 32.
template <typename T, int D, int N>
struct Core {
  static constexpr int kSteps = D / 32;      // products over the channels of a 16-key tile
  static constexpr int kRun = D / 16;        // channels of V per lane
  using Piece = vec_t<T, 8>;
  using Run = vec_t<T, kRun>;
  static constexpr int kPieceElems = 8;
  Piece q[N][kSteps];
  Piece k[2][kSteps];
  Run v[8];

  // (a product waits for the one before it on the same sum: the sums take turns)
  __device__ __forceinline__ void scores(float4v (&s)[N][2]) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) s[n][t] = matrix(k[t][i], q[n][i], i ? s[n][t] : float4v{0.f, 0.f, 0.f, 0.f});
  }
  // P as the sum of two numbers of the storage type: one alone would add an error as large as the
  // rounding of O to O, and the matrix cores wait for memory here.  What is left is 2^-22 (bf16 2^-16) of a numerator, or 2^-25 (fp16,
  // whose largest is 2^15).
  __device__ __forceinline__ void mix(const float (&p)[N][8], float4v (&o)[N][kRun]) const {
    Piece high[N], low[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        high[n][e] = (T)p[n][e];
        low[n][e] = (T)(p[n][e] - (float)high[n][e]);
      }
#pragma unroll
    for (int c = 0; c < kRun; ++c) {
      Piece column;
#pragma unroll
      for (int e = 0; e < 8; ++e) column[e] = v[e][c];
#pragma unroll
      for (int n = 0; n < N; ++n) o[n][c] = matrix(column, high[n], o[n][c]);
#pragma unroll
      for (int n = 0; n < N; ++n) o[n][c] = matrix(column, low[n], o[n][c]);
    }
  }
};
// fp32 storage: products of four, every operand used whole.
template <int D, int N>
struct Core<float, D, N> {
  static constexpr int kSteps = D / 16;      // 16-byte pieces of a key per lane
  static constexpr int kRun = D / 16;
  using Piece = vec_t<float, 4>;
  using Run = vec_t<float, kRun>;
  static constexpr int kPieceElems = 4;
  Piece q[N][kSteps];
  Piece k[2][kSteps];
  Run v[8];

  __device__ __forceinline__ void scores(float4v (&s)[N][2]) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int t = 0; t < 2; ++t)
            s[n][t] = matrix(k[t][i][e], q[n][i][e], i || e ? s[n][t] : float4v{0.f, 0.f, 0.f, 0.f});
  }
  __device__ __forceinline__ void mix(const float (&p)[N][8], float4v (&o)[N][kRun]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int c = 0; c < kRun; ++c)
#pragma unroll
        for (int n = 0; n < N; ++n) o[n][c] = matrix(v[e][c], p[n][e], o[n][c]);
  }
};

// Walks the blocks [block, end) in steps of `step` for one row, key by key, and adds nothing for a key that it does not see:
// the products above cannot leave a key out, and 0 times an infinity or NaN in it is NaN.  Only where a tile's result is not
// finite.  A lane ends with channels lane, lane + 64, ...; top and sum are the wavefront's.
template <typename T, int D, bool kTree>
__device__ __forceinline__ void attend_row(const PagedAttention& a, const Tile& tile, int32_t head_kv, int32_t flat,
                                           int32_t block, int32_t end, int32_t step, float& top, float& sum,
                                           float (&o)[(D + 63) / 64]) {
  const int lane = threadIdx.x & (kWave - 1);
  const PagedArgs& b = a.batch;
  const int32_t group = (int32_t)a.group.value, token = (int32_t)quotient((uint32_t)flat, a.group);
  const Sight sight = row_sight<kTree>(a, tile, token);
  const T* const q = static_cast<const T*>(a.Q) + (int64_t)(head_kv * group + (flat - token * group)) * a.q_head +
                     (int64_t)(tile.begin + token) * a.q_row;
  const int64_t in_head = (int64_t)head_kv * b.page.value * D;
  top = -INFINITY;
  sum = 0.f;
#pragma unroll
  for (int c = 0; c < (D + 63) / 64; ++c) o[c] = 0.f;
  for (; block < end; block += step) {
    const int32_t j = first_key(tile, block) + (lane & (kBlock - 1));
    const int64_t at = place_of(b, tile.seq, j, D);
    bool sees = (j >= sight.lo && j <= sight.hi) || j < sight.lead;
    if constexpr (kTree)
      sees |= new_tokens_seen(a, tile, tree_row(a, tile, token), first_key(tile, block)) >> (lane & (kBlock - 1)) & 1;
    sees = sees && at >= 0;
    float s = -INFINITY;
    if (sees) {
      const T* const k = static_cast<const T*>(a.cache_k) + in_head + at;
      float x = 0.f;
      for (int c = 0; c < D; ++c) x = fmaf((float)q[c], (float)k[c], x);
      s = x * (a.scale * kLog2e);
    }
    float best = s;
#pragma unroll
    for (int off = 1; off < kBlock; off <<= 1) best = fmaxf(best, __shfl_xor(best, off, kWave));
    best = fmaxf(best, top);
    const float keep = best > -INFINITY ? __builtin_amdgcn_exp2f(top - best) : 1.f;
    top = best;
    const float p = sees ? __builtin_amdgcn_exp2f(s - (top > -INFINITY ? top : 0.f)) : 0.f;
    sum *= keep;
#pragma unroll
    for (int c = 0; c < (D + 63) / 64; ++c) o[c] *= keep;
    float total = 0.f, mix[(D + 63) / 64] = {};              // (added up by blocks, see the kernel)
    for (uint32_t left = (uint32_t)__ballot(sees); left; left &= left - 1) {
      const int from = __ffs(left) - 1;
      const float w = __shfl(p, from, kWave);
      const int32_t low = __shfl((int32_t)at, from, kWave), high = __shfl((int32_t)(at >> 32), from, kWave);
      const T* const v = static_cast<const T*>(a.cache_v) + in_head + ((int64_t)high << 32 | (uint32_t)low);
      total += w;
#pragma unroll
      for (int c = 0; c < (D + 63) / 64; ++c)
        if (lane + 64 * c < D) mix[c] = fmaf(w, (float)v[lane + 64 * c], mix[c]);
    }
    sum += total;
#pragma unroll
    for (int c = 0; c < (D + 63) / 64; ++c) o[c] += mix[c];
  }
}

// Writes D / 16 channels of a finished row: o / total, and its lse.
template <typename T, int D>
__device__ __forceinline__ void store_row(const PagedAttention& a, const Tile& tile, int32_t head_kv, int32_t row, int32_t channel,
                                          const float (&o)[D / 16], float top, float total) {
  const int32_t group = (int32_t)a.group.value, flat = tile.first + row, token = (int32_t)quotient((uint32_t)flat, a.group);
  const int32_t head = head_kv * group + (flat - token * group), at = tile.begin + token;
  const float inv = total != 0.f ? 1.f / total : 0.f;
  vec_t<T, D / 16> y;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) y[c] = (T)(o[c] * inv);
  *reinterpret_cast<vec_t<T, D / 16>*>(static_cast<T*>(a.O) + (int64_t)head * a.o_head + (int64_t)at * a.o_row + channel) = y;
  if (a.lse && channel == 0) a.lse[(int64_t)head * a.batch.n_tokens + at] = (top + __builtin_amdgcn_logf(total)) * kLn2;
}

// Where the rows of a block's keys are.  kWholeTiles: pages hold multiples of 16 tokens, so a 16-key tile lies in one.
struct Places {
  int64_t tile[2];           // kWholeTiles: element offset of the tile's first row (wave-uniform)
  int64_t key;               // else: of key lane % 32
  uint32_t held;             // bit t: tile t has a page; else bit j: key j of the block has one
};
struct Asked {
  int32_t page, in_page;     // of a key: its page table entry (-1 behind the last column) and the row in that page
};

// N: 16-row groups of a tile, which share the keys that a wavefront loads.
// One share after the other of each workgroup's tiles.  Measured (us alone, TB/s of the keys and values that rows see): one
// token of 64 sequences of 512 to 32,768, 8 key heads of 128, bf16 349 (5.7, a large copy: 5.0), of 160 windows of 2,048, 4 key
// heads, fp16 116 (4.8); a document of six sequences, window 128, fp32, d = 64 137 (43 TFLOP/s of 154: matrix cores 32 % busy.  445 of the 512
// workgroups get five or six tiles, four in a first pass and one or two in a second, so a third of the wavefronts' time passes at the barrier behind it;
// and first loads of short tiles, which two wavefronts per SIMD do not hide).
template <typename T, int D, int N, bool kWholeTiles, bool kTree>
__global__ __launch_bounds__(kWaves* kWave) __attribute__((amdgpu_waves_per_eu(D == 256 ? 1 : 2))) void paged_kernel(
    PagedAttention a) {
  using C = Core<T, D, N>;
  constexpr int kRun = C::kRun, kTileRows = 16 * N;
  constexpr int kStride = D + 4;                          // floats of a row in LDS
  __shared__ __align__(16) float out[kWaves][kTileRows][kStride];
  __shared__ float tops[kWaves][kTileRows], sums[kWaves][kTileRows];
  const int32_t group = (int32_t)a.group.value;
  __shared__ Share<kTileRows, kTree> share;
  for (bool first_part = true;; first_part = false) {
    const bool any = share.next(a, blockIdx.x, first_part);
    if (first_part && a.partials && threadIdx.x == 0) {
      // the tile that ends in this share and began in an earlier one
      const Part& p = share.part[0];
      const bool ends = any && p.from > 0 && p.to == p.extent;
      const int32_t first = ends ? (int32_t)quotient64(share.size * blockIdx.x - p.from, share.size) : 0;
      notes_of(a)[blockIdx.x] = Note{ends ? (int32_t)blockIdx.x - first + 1 : 0, first, 0, p.begin, p.n_new, p.length,
                                     p.tile, p.head};
    }
    if (!any) return;
    const int tid = thread_again(), lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int m = lane & 15, g = lane >> 4;
    const int parts = __builtin_amdgcn_readfirstlane(share.parts);
    const bool alone = __builtin_amdgcn_readfirstlane(share.part[0].there) == 2;      // this wavefront has a tile to itself
    if (!alone || wave < parts) {
      const Part here = share.mine(alone ? wave : 0);
      const int32_t head_kv = here.head;
      const Tile tile = tile_of<kTileRows, kTree>(a, here.seq, here.begin, here.n_new, here.length, here.tile);

      // this lane's rows
      Sight sight[N];
      int32_t seen_row[N];                                   // (of a draft tree)
      C core;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int32_t flat = tile.first + (16 * n + m < tile.count ? 16 * n + m : 0);
        const int32_t token = (int32_t)quotient((uint32_t)flat, a.group), head = head_kv * group + (flat - token * group);
        sight[n] = row_sight<kTree>(a, tile, token);
        if constexpr (kTree) seen_row[n] = tree_row(a, tile, token);
        const T* q = static_cast<const T*>(a.Q) + (int64_t)head * a.q_head + (int64_t)(tile.begin + token) * a.q_row;
#pragma unroll
        for (int i = 0; i < C::kSteps; ++i)
          core.q[n][i] = *reinterpret_cast<const typename C::Piece*>(q + (g + 4 * i) * C::kPieceElems);
      }
      // keys that every row sees
      int32_t lo_max = sight[0].lo, hi_min = sight[0].hi;
#pragma unroll
      for (int n = 1; n < N; ++n) {
        lo_max = max(lo_max, sight[n].lo);
        hi_min = min(hi_min, sight[n].hi);
      }
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
      // Lane l asks for key l % 32 of a block, a block ahead of the loads that need the answer.
      auto ask = [&](int32_t block) {
        const uint32_t j = (uint32_t)(first_key(tile, block) + (lane & 31)), column = quotient(j, b.page);
        Asked q;
        q.in_page = (int32_t)(j - column * b.page.value);
        q.page = column < (uint32_t)b.pages_per_seq ? table[column] : -1;
        return q;
      };
      auto find = [&](const Asked& q) {
        const bool there = (uint32_t)q.page < b.n_pages;
        const int64_t o = there ? (int64_t)q.page * b.page_stride + (int64_t)q.in_page * D : 0;
        const uint32_t held = (uint32_t)__ballot(there);
        Places at;
        if constexpr (kWholeTiles) {
          at.held = (held & 1) | (held >> 15 & 2);
          at.tile[0] = (int64_t)from_lane((uint64_t)o, 0);
          at.tile[1] = (int64_t)from_lane((uint64_t)o, 16);
        } else {
          at.held = held;
          at.key = o;
        }
        return at;
      };
      auto load_k = [&](const Places& at) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const T* row = kWholeTiles ? cache_k + at.tile[t] + m * D : cache_k + __shfl(at.key, 16 * t + m, kWave);
#pragma unroll
          for (int i = 0; i < C::kSteps; ++i)
            core.k[t][i] = *reinterpret_cast<const typename C::Piece*>(row + (g + 4 * i) * C::kPieceElems);
        }
      };
      auto load_v = [&](const Places& at) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const T* row = kWholeTiles ? cache_v + at.tile[e / 4] + (4 * g + e % 4) * D
                                     : cache_v + __shfl(at.key, 16 * (e / 4) + 4 * g + e % 4, kWave);
          core.v[e] = *reinterpret_cast<const typename C::Run*>(row + m * kRun);
        }
      };

      const int32_t first_block = block_at(here.from, here.extent, tile.blocks) + (alone ? 0 : wave);
      const int32_t end_block = block_at(here.to, here.extent, tile.blocks), step = alone ? 1 : kWaves;
      float top[N], sum[N];
      float4v o[N][kRun];
#pragma unroll
      for (int n = 0; n < N; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int c = 0; c < kRun; ++c) o[n][c] = float4v{0.f, 0.f, 0.f, 0.f};
      }
      Places at;
      Asked asked{};
      if (first_block < end_block) {
        at = find(ask(first_block));
        asked = ask(first_block + step);      // (behind the last block: a place in the page table's row, or none)
        load_k(at);
        load_v(at);
      }
      for (int32_t block = first_block; block < end_block; block += step) {
        const int32_t j0 = first_key(tile, block);
        const uint32_t held = at.held;
        const bool more = block + step < end_block;
        float4v s[N][2];
        core.scores(s);
        if (more) {
          at = find(asked);
          asked = ask(block + 2 * step);
          load_k(at);
        }
        const bool all_held = held == (kWholeTiles ? 3u : ~0u);
        const bool whole = all_held && j0 >= lo_max && j0 + kBlock - 1 <= hi_min;
        float p[N][8];
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[n][e] = s[n][e / 4][e % 4] * (a.scale * kLog2e);
          if (!whole) {
            uint32_t drafted = 0;
            if constexpr (kTree) drafted = new_tokens_seen(a, tile, seen_row[n], j0);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int in_block = 16 * (e / 4) + 4 * g + e % 4, j = j0 + in_block;
              const bool there = kWholeTiles ? (held >> (e / 4)) & 1 : (held >> in_block) & 1;
              const bool sees = (j >= sight[n].lo && j <= sight[n].hi) || j < sight[n].lead || (kTree && (drafted >> in_block & 1));
              p[n][e] = there && sees ? p[n][e] : -INFINITY;
            }
          }
          float best = p[n][0];
#pragma unroll
          for (int e = 1; e < 8; ++e) best = fmaxf(best, p[n][e]);
          best = fmaxf(row_max(best) - kRaise<T>, top[n]);
          if (__any(best > top[n])) {
            const float keep = best > -INFINITY ? __builtin_amdgcn_exp2f(top[n] - best) : 1.f;
            sum[n] *= keep;
#pragma unroll
            for (int c = 0; c < kRun; ++c) o[n][c] *= keep;
            top[n] = best;
          }
          // (a block's numerators are added up before they join the row's sum: many small ones beside a few large ones would each
          // be rounded to the sum's step)
          const float against = top[n] > -INFINITY ? top[n] : 0.f;
          float total = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[n][e] = __builtin_amdgcn_exp2f(p[n][e] - against);
            total += p[n][e];
          }
          sum[n] += total;
        }
        // values of keys that no row sees (behind the last token, without a page) may be anything
        if (!all_held || j0 + kBlock > tile.kept) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int in_block = 16 * (e / 4) + 4 * g + e % 4;
            const bool there = kWholeTiles ? (held >> (e / 4)) & 1 : (held >> in_block) & 1;
            const bool use = there && j0 + in_block < tile.kept;
#pragma unroll
            for (int c = 0; c < kRun; ++c) core.v[e][c] = use ? core.v[e][c] : (T)0.f;
          }
        }
        core.mix(p, o);
        if (more) load_v(at);
      }
      bool finite = true;
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int c = 0; c < kRun; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) finite = finite && __builtin_isfinite(o[n][c][r]);
      if (__all(finite)) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const float total = row_sum(sum[n]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < kRun; ++c) out[wave][16 * n + m][(4 * g + r) * kRun + c] = o[n][c][r];
          if (g == 0) {
            tops[wave][16 * n + m] = top[n];
            sums[wave][16 * n + m] = total;
          }
        }
      } else {
        for (int row = 0; row < tile.count; ++row) {
          float x[(D + 63) / 64], row_top, row_total;
          attend_row<T, D, kTree>(a, tile, head_kv, tile.first + row, first_block, end_block, step, row_top, row_total, x);
#pragma unroll
          for (int c = 0; c < (D + 63) / 64; ++c)
            if (lane + 64 * c < D) out[wave][row][lane + 64 * c] = x[c];
          if (lane == 0) {
            tops[wave][row] = row_top;
            sums[wave][row] = row_total;
          }
        }
      }
      constexpr int kPer = D / 16;                             // channels of a thread
      if (alone) {
        __builtin_amdgcn_wave_barrier();
        for (int i = lane; i < 16 * tile.count; i += kWave) {
          float x[kPer];
#pragma unroll
          for (int c = 0; c < kPer; ++c) x[c] = out[wave][i / 16][i % 16 * kPer + c];
          store_row<T, D>(a, tile, head_kv, i / 16, i % 16 * kPer, x, tops[wave][i / 16], sums[wave][i / 16]);
        }
      } else {
        __syncthreads();
        // the wavefronts' states of a row, added in their order
        float* const part = here.from == 0 && here.to == here.extent ? nullptr : record_of_share<D, kTileRows>(a, blockIdx.x, here.from > 0);
        const int channel = tid % 16 * kPer;
        for (int row = tid / 16; row < tile.count; row += kWaves * kWave / 16) {
          float high = -INFINITY;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) high = fmaxf(high, tops[w][row]);
          const float against = high > -INFINITY ? high : 0.f;
          float total = 0.f, x[kPer];
#pragma unroll
          for (int c = 0; c < kPer; ++c) x[c] = 0.f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) {
            if (sums[w][row] == 0.f) continue;                 // no key seen
            const float weight = __builtin_amdgcn_exp2f(tops[w][row] - against);
            total += weight * sums[w][row];
#pragma unroll
            for (int c = 0; c < kPer; ++c) x[c] += weight * out[w][row][channel + c];
          }
          if (part) {
#pragma unroll
            for (int c = 0; c < kPer; ++c) part[row * D + channel + c] = x[c];
            if (channel == 0) {
              part[kTileRows * D + row] = high;
              part[kTileRows * (D + 1) + row] = total;
            }
          } else {
            store_row<T, D>(a, tile, head_kv, row, channel, x, high, total);
          }
        }
      }
    }
    __syncthreads();                                       // the next part's states take the same space
  }
}

// ---- many new tokens: tiles of 128 rows ---------------------------------------------------------------------
// Four wavefronts own 32 rows each and share every block of keys: K and V are copied global -> LDS without registers,
// once per workgroup, into a ring of four blocks, three ahead; the barrier that opens a block also frees the one before
// it.  Products of 32 x 32 x 16 (fp32 storage: x 2): S^T = K Q^T and O^T += V^T P^T, a lane's row is lane % 32 in both, and
// the keys that it holds of S^T are those that it feeds as P.  The scores of the next block are issued ahead of this
// block's exponentials, so matrix and vector units have work at once.
// The reference of a row's exponentials (m) is raised only when a lane's 16 numerators of a block add up to kMostNumerators: what matters
// is that they stay in the range of the storage type, and the sums l and O are in 32 bits whatever their reference.
// P is rounded to the storage type once: fp16 2^-11 of a numerator, and at least 2^-25 where the largest of the row is 2^10 or more; bf16
// 2^-8.  Scores that differ are rounded independently of each other, equal ones alike, so O is off by at most that part
// of the weighted mean of |V|.  The matrix cores bound this kernel, and a second number for P costs a third of its time (us: prompt under a window 1,223 / 1,622, chunks
// behind long contexts 261 / 342).  l sums the unrounded numerators.  Drafted tokens keep this, so that a chain of them is rounded as the same tokens without a tree are: O is 1.4
// times as far from the exact result as its own rounding makes it (bf16 2.3e-3 of its size against 1.7e-3).  A second number would cost them little where memory bounds the
// call and as much as others where it does not (us: 5 to 16 drafts of 64 sequences behind up to 32,768 417 / 430, of 8 behind up to 3,000 26 / 30, 16 under a window of 2,048
// 114 / 119, 30 to 200 under 4,096 225 / 292, 100 behind 4,000 265 / 363).
// Measured (us and TFLOP/s of the products that the mask asks for): a causal prompt of 32,768 tokens, 8 heads of 128, bf16
// 2,310 (950 of a library product's 1,266); the same with 32 heads under a window of 2,048, fp16 1,250 (850: a tile meets
// 68 blocks, eight of them edges that test every key); 16,384 tokens, causal, 8 heads of 64, fp32 2,570 (107 of 154).
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr int kChunkRows = 128, kChunkSlots = 4;
constexpr int kChunkAhead = kChunkSlots - 1;
// (fp16 ends at 65,504.  From 2^10, the largest right after the reference was raised, 16 equal ones have room for a factor of 3.75 and a
// single one of 60, where 2^14 against a largest of 1 left 2^10 and 2^14: us, a prompt of 32,768 tokens under a window of 2,048, 32 heads of 128,
// scores of deviation 1 / 3 / 6 / 12 1,230 / 1,300 / 1,345 / 1,355 against 1,225 / 1,240 / 1,245 / 1,265.)
template <typename T>
constexpr float kMostNumerators = kChunkRaise<T> > 0.f ? 61440.f : 16384.f;

__device__ __forceinline__ floatx16 matrix32(vec_t<f16_t, 8> a, vec_t<f16_t, 8> b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 matrix32(vec_t<bf16_t, 8> a, vec_t<bf16_t, 8> b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Full precision: four products of two, the halves of the wavefront each with its piece.
__device__ __forceinline__ floatx16 matrix32(vec_t<float, 4> a, vec_t<float, 4> b, floatx16 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// The value of the lane 32 positions away.
__device__ __forceinline__ float other_half(float x, int h) {
  const unsigned xi = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(xi, xi, false, false);
  return __builtin_bit_cast(float, h ? r[0] : r[1]);
}

// s_waitcnt vmcnt(N): all but the N most recently issued vector memory operations have completed.
template <int N>
__device__ __forceinline__ void wait_loads_except() {
  static_assert(N >= 0 && N <= 63, "vmcnt immediate");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// kCopies times 16 bytes per lane from k, the lane's offset and 64 bytes for each copy before on, into LDS at `to` + 16 * lane and
// `step` further on each, and then from v likewise: without registers and behind the compiler's back, completion is waited
// for by count (wait_loads_except) and a barrier.  (M0 holds the address in LDS; the compiler's own value is put back.)
template <int kCopies, int kStep, int kApart>
__device__ __forceinline__ void copy_pieces(const char* k, uint32_t k_offset, const char* v, uint32_t v_offset, uint32_t to) {
  uint32_t kept;
  if constexpr (kCopies == 1) {
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %4\n\ts_mov_b32 m0, %0"
        : "=&s"(kept) : "v"(k_offset), "s"(k), "v"(v_offset), "s"(v), "s"(to), "i"(kApart) : "memory", "scc");
  } else {
    static_assert(kCopies % 2 == 0, "copies in pairs");
#pragma unroll
    for (int i = 0; i < kCopies; i += 2)
      asm volatile(
          "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %7\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
          "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\t"
          "s_add_u32 m0, m0, %9\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %6\n\t"
          "s_add_u32 m0, m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %6\n\ts_mov_b32 m0, %0"
          : "=&s"(kept)
          : "v"(k_offset + 64 * i), "v"(k_offset + 64 * i + 64), "s"(k), "v"(v_offset + 64 * i), "v"(v_offset + 64 * i + 64), "s"(v),
            "s"(to + i * kStep), "i"(kStep), "i"(kApart - kStep)
          : "memory", "scc");
  }
}

// The same from an address of each lane's own.
template <int kCopies, int kStep, int kApart>
__device__ __forceinline__ void copy_pieces_from(const char* k, const char* v, uint32_t to) {
  uint32_t kept;
#pragma unroll
  for (int i = 0; i < kCopies; ++i)
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\t"
        "s_add_u32 m0, m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
        : "=&s"(kept) : "v"(k + 64 * i), "v"(v + 64 * i), "s"(to + i * kStep), "i"(kApart) : "memory", "scc");
}

// A block of 32 keys in LDS: groups of 64 bytes of a row, in a group the 32 keys' parts one behind the other.  What the products read then
// differs by constants from one or two addresses per lane, and 16 lanes' pieces (K: four rows apart they would share
// banks, so a row's four pieces are permuted; V: eight rows in a row) meet every bank once.
template <int kRow>
struct ChunkBlock {
  static constexpr int kRowBytes = kRow, kBytes = kBlock * kRowBytes, kGroupBytes = kBlock * 64;
  static constexpr int kCopies = kRow / 128;  // copies of a wavefront: 16 rows of as many groups
  static __device__ __forceinline__ int k_turn(int row) { return row >> 2 & 3; }
};

// Row sizes that the ring fits.
__host__ __device__ constexpr bool chunk_fits(int64_t row_bytes) { return row_bytes >= 128 && row_bytes <= 512; }

template <typename T, int D, bool kWholeTiles, bool kTree>
__global__ __attribute__((amdgpu_waves_per_eu(chunk_waves(sizeof(T) * D), chunk_waves(sizeof(T) * D)))) __launch_bounds__(kWaves* kWave) void
paged_chunk_kernel(PagedAttention a) {
  using B = ChunkBlock<D * (int)sizeof(T)>;
  constexpr int kPieceElems = 16 / sizeof(T);
  using Piece = vec_t<T, kPieceElems>;
  using Numerators = vec_t<T, 8>;
  constexpr bool kSingle = sizeof(T) == 4;
  constexpr int kSlotBytes = 2 * B::kBytes, kPer = 2 * B::kCopies;    // copies of a wavefront per block
  constexpr int kSteps = B::kRowBytes / 32, kTiles = D / 32;
  __shared__ __align__(16) char ring[kChunkSlots * kSlotBytes];
  // Pages that do not hold multiples of 16 tokens: the page of every key of the next kAskBlocks blocks, asked for at once.  (A
  // load into registers between the copies would make its reader wait for all of them.)
  constexpr int kAskBlocks = kTree ? 32 : 64;
  __shared__ int32_t page_of_key[kWholeTiles ? 1 : kAskBlocks * kBlock];
  // (a draft tree) The rows' words of `seen`, for the same reason ahead of the copies.
  __shared__ uint32_t seen_words[kTree ? kChunkRows * kMostTreeWords : 1];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane & 31, h = lane >> 5;
  // Workgroup i runs on XCD i % 8: a key head stays on one XCD, or on 8 / Hkv of them, whose L2 then holds the keys that
  // its tiles share.
  int32_t head_kv, rest;
  {
    const uint32_t id = blockIdx.x, per_head = (uint32_t)a.slots, heads = a.Hkv;
    if (heads % 8 == 0) {
      const uint32_t turn = (id / 8) / per_head;
      head_kv = id % 8 + 8 * turn;
      rest = id / 8 - turn * per_head;
    } else if (8 % heads == 0) {
      head_kv = id % 8 % heads;
      rest = id / 8 * (8 / heads) + id % 8 / heads;
    } else {
      head_kv = id / per_head;
      rest = id - head_kv * per_head;
    }
    if ((uint32_t)rest >= per_head) return;
  }
  const int64_t record = (int64_t)head_kv * a.slots + rest;
  Tile tile;
  int32_t index = 0, piece = 0, pieces = 1, apart = 0;
  const bool any = piece_of<kChunkRows, kTree>(a, rest, tile, index, piece, pieces, apart);
  if (a.partials && tid == 0) {
    const bool cut = any && pieces > 1 && piece == 0;
    // (a seq_ptr that decreases can bring more tiles than the plan counts: pieces behind the last workgroup's have no record)
    const int32_t count = cut ? min(pieces, 1 + (int32_t)((uint32_t)(a.slots - 1 - rest) / (uint32_t)apart)) : 0;
    notes_of(a)[record] = cut ? Note{count, (int32_t)record, apart, tile.begin, tile.n_new, tile.length, index, head_kv} : Note{};
  }
  if (!any) return;
  const int32_t group = (int32_t)a.group.value;
  const PagedArgs& b = a.batch;
  const int32_t first_block = (int32_t)((int64_t)tile.blocks * piece / pieces);
  const int32_t end_block = (int32_t)((int64_t)tile.blocks * (piece + 1) / pieces);

  // this lane's row
  const int32_t own_first = 32 * wave, row = own_first + n;
  const bool exists = row < tile.count;
  const int32_t flat = tile.first + (exists ? row : tile.count - 1);
  const int32_t token = (int32_t)quotient((uint32_t)flat, a.group), head = head_kv * group + (flat - token * group);
  Sight sight = row_sight<kTree>(a, tile, token);
  if constexpr (kTree) {
    for (int i = tid; i < kChunkRows * a.words; i += kWaves * kWave) {
      const int r = i / a.words;
      const int32_t from = r < tile.count ? tree_row(a, tile, (int32_t)quotient((uint32_t)(tile.first + r), a.group)) : -1;
      seen_words[i] = from >= 0 ? a.seen[(int64_t)from * a.words + (i - r * a.words)] : 0;
    }
  }
  if (own_first >= tile.count) sight = Sight{0, -1, 0};                // a wavefront without rows only copies
  Piece qf[kSteps];
  {
    const T* q = static_cast<const T*>(a.Q) + (int64_t)head * a.q_head + (int64_t)(tile.begin + token) * a.q_row + kPieceElems * h;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) qf[i] = *reinterpret_cast<const Piece*>(q + 2 * kPieceElems * i);
    // (a mask puts -inf into scores before the scale: the scale is positive from here on)
    if (!(a.scale > 0.f)) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int e = 0; e < kPieceElems; ++e) qf[i][e] = a.scale == 0.f ? (T)((float)qf[i][e] * 0.f) : -qf[i][e];
    }
  }
  const float factor = a.scale == 0.f ? 1.f : fabsf(a.scale) * kLog2e;
  int32_t lo_min = sight.lo, lo_max = sight.lo, hi_min = sight.hi, hi_max = sight.hi, lead_max = sight.lead;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    lo_min = min(lo_min, __shfl_xor(lo_min, off, kWave));
    lo_max = max(lo_max, __shfl_xor(lo_max, off, kWave));
    hi_min = min(hi_min, __shfl_xor(hi_min, off, kWave));
    hi_max = max(hi_max, __shfl_xor(hi_max, off, kWave));
    lead_max = max(lead_max, __shfl_xor(lead_max, off, kWave));
  }
  lo_min = __builtin_amdgcn_readfirstlane(lo_min);
  lo_max = __builtin_amdgcn_readfirstlane(lo_max);
  hi_min = __builtin_amdgcn_readfirstlane(hi_min);
  hi_max = __builtin_amdgcn_readfirstlane(hi_max);
  lead_max = __builtin_amdgcn_readfirstlane(lead_max);

  // ---- copies
  const int64_t in_head = (int64_t)head_kv * b.page.value * D;
  const char* const cache_k = reinterpret_cast<const char*>(static_cast<const T*>(a.cache_k) + in_head);
  const char* const cache_v = reinterpret_cast<const char*>(static_cast<const T*>(a.cache_v) + in_head);
  // (read as constants: scalar loads, which leave the count of vector memory operations to the copies)
  const auto* const table = (const int32_t __attribute__((address_space(4)))*)(uintptr_t)(b.page_table + (int64_t)tile.seq * b.pages_per_seq);
  // Wavefront w copies 16-key tile w / 2, half of the groups: lane l 16 bytes of row l / 4.  (Bytes from the tile's first row on;
  // the groups follow at 64 bytes.)
  const int copy_row = 16 * (wave / 2) + lane / 4;
  const uint32_t k_in_row = (wave % 2) * (B::kCopies * 64) + ((lane & 3) ^ B::k_turn(copy_row)) * 16;
  const uint32_t v_in_row = (wave % 2) * (B::kCopies * 64) + (lane & 3) * 16;
  const uint32_t k_from = (lane / 4) * B::kRowBytes + k_in_row, v_from = (lane / 4) * B::kRowBytes + v_in_row;
  const uint32_t own_part = (wave % 2) * (B::kCopies * B::kGroupBytes) + (wave / 2) * 1024;
  const uint32_t ring_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(char __attribute__((address_space(3)))*)ring);
  // The place of this wavefront's rows in the block that is copied next: its page's column and the row within it follow each
  // other without divisions, and the column's entry is loaded a block ahead of its use.  An entry that is no page
  // is read as some page (what it copies is hidden), a column behind the last as the last.
  const uint32_t page = b.page.value, columns_step = page == 16 ? 2 : 0, rows_step = page == 16 ? 0 : kBlock;
  const uint32_t last_column = b.pages_per_seq - 1, last_page = b.n_pages - 1;
  int32_t next_block = first_block;
  uint32_t column = 0, in_page = 0, entry = 0, next_at = ring_at + own_part;
  auto look_up = [&]() { entry = (uint32_t)table[min(column, last_column)]; };
  auto start_at = [&](int32_t block) {
    const uint32_t j = (uint32_t)(first_key(tile, block) + 16 * (wave / 2));
    column = quotient(j, b.page);
    in_page = j - column * page;
    look_up();
  };
  auto ask = [&]() {                     // (every wavefront: all have issued the blocks before)
    for (int i = tid; i < kAskBlocks * kBlock; i += kWaves * kWave) {
      const int32_t block = next_block + i / kBlock;
      const uint32_t c = quotient((uint32_t)(first_key(tile, block < end_block ? block : end_block - 1) + i % kBlock), b.page);
      page_of_key[i] = b.page_table[(int64_t)tile.seq * b.pages_per_seq + min(c, last_column)];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  auto issue = [&]() {                   // copies next_block, or the last one again
    if constexpr (kWholeTiles) {
      const uint64_t at = ((uint64_t)min(entry, last_page) * a.page_pieces << 4) + in_page * B::kRowBytes;
      copy_pieces<B::kCopies, B::kGroupBytes, B::kBytes>(cache_k + at, k_from, cache_v + at, v_from, next_at);
    } else {
      const int32_t block = next_block < end_block ? next_block : end_block - 1;
      const uint32_t j = (uint32_t)(first_key(tile, block) + copy_row), in_page = j - quotient(j, b.page) * page;
      const uint32_t held_by = min((uint32_t)page_of_key[(block - first_block) % kAskBlocks * kBlock + copy_row], last_page);
      const uint64_t at = ((uint64_t)held_by * a.page_pieces << 4) + in_page * B::kRowBytes;
      copy_pieces_from<B::kCopies, B::kGroupBytes, B::kBytes>(cache_k + at + k_in_row, cache_v + at + v_in_row, next_at);
    }
    next_at = ring_at + ((next_at - ring_at + kSlotBytes) & (kChunkSlots * kSlotBytes - 1));
    if (++next_block < end_block && kWholeTiles) {
      if (next_block == tile.lead) {
        start_at(next_block);
      } else {
        column += columns_step;
        in_page += rows_step;
        if (in_page >= page) {
          in_page -= page;
          ++column;
        }
        look_up();
      }
    }
  };
  // Opens a block: every wavefront has waited for its own copies of this block and the next one, and everyone is
  // done with the block before, whose slot takes the next copy.
  auto publish = [&]() {
    wait_loads_except<kPer*(kChunkAhead - 2)>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if constexpr (!kWholeTiles)
      if ((next_block - first_block) % kAskBlocks == 0 && next_block < end_block) ask();
    issue();
  };

  // ---- arithmetic
  floatx16 o[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) o[t] = floatx16{0};
  float top = -INFINITY, sum = 0.f;
  const int vi = lane & 15;
  const char* const v_base = ring + B::kBytes + (4 * h + (vi >> 2)) * 64 + (lane >> 4 & 1) * 32 + (vi & 3) * 8;
  const char* const k_base[2] = {ring + n * 64 + (h ^ B::k_turn(n)) * 16, ring + n * 64 + ((2 + h) ^ B::k_turn(n)) * 16};
  auto slot_of = [&](int32_t block) { return (uint32_t)(block - first_block) % kChunkSlots * kSlotBytes; };
  auto meets = [&](int32_t block) {
    const int32_t j0 = first_key(tile, block);
    if constexpr (kTree)
      if (j0 + kBlock > tile.length - tile.n_new && own_first < tile.count) return true;
    return (j0 <= hi_max && j0 + kBlock - 1 >= lo_min) || j0 < lead_max;
  };
  auto read_k = [&](uint32_t slot_at, Piece (&k)[kSteps]) {
    const char* const at[2] = {k_base[0] + slot_at, k_base[1] + slot_at};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) k[i] = *reinterpret_cast<const Piece*>(at[i & 1] + i / 2 * B::kGroupBytes);
  };
  auto products = [&](const Piece (&k)[kSteps], floatx16& s) {
    s = floatx16{0};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) s = matrix32(k[i], qf[i], s);
  };
  // (16-bit) 32 t + 0..31 channels of 16 keys, turned
  auto read_v = [&](uint32_t slot_at, int u, Piece (&v)[kTiles]) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const char* const at = v_base + slot_at + t * B::kGroupBytes + 16 * u * 64;
      const short4v low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)at);
      const short4v high =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(at + 8 * 64));
      const vec_t<short, 8> both = __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
      v[t] = __builtin_bit_cast(Piece, both);
    }
  };
  // Accumulator register r holds key 8 (r / 4) + 4 h + r % 4 of the block.
  auto numerators = [&](const floatx16& s, float against, Numerators (&p)[2]) {
    float total = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = __builtin_amdgcn_exp2f(fmaf(s[r], factor, -against));
      total += x;
      p[r / 8][r % 8] = (T)x;
    }
    return total;
  };
  // the reference of the rows' numerators becomes their largest score so far, or 2^kChunkRaise below it
  auto raise = [&](const floatx16& s) {
    float best = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) best = fmaxf(best, s[r]);
    best = fmaxf(best, other_half(best, h)) * factor - kChunkRaise<T>;
    best = fmaxf(best, top);
    const float keep = best > -INFINITY ? __builtin_amdgcn_exp2f(top - best) : 1.f;
    top = best;
    sum *= keep;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] *= keep;
  };
  auto weigh = [&](uint32_t slot_at, const floatx16& s, float total, Numerators (&p)[2]) {
    if (__any(!(total < kMostNumerators<T>))) {          // (before a row's first key: infinite or NaN)
      raise(s);
      total = numerators(s, top > -INFINITY ? top : 0.f, p);
    }
    sum += total;
    if constexpr (kSingle) {
      // register r: key 8 (r / 4) + 4 h + r % 4, and a lane's channels kTiles n ..
      const char* const at = ring + B::kBytes + slot_at + (kTiles * 4 * n / 64) * B::kGroupBytes + kTiles * 4 * n % 64 + 4 * h * 64;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const vec_t<float, kTiles> v = *reinterpret_cast<const vec_t<float, kTiles>*>(at + (8 * (r / 4) + r % 4) * 64);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[t], p[r / 8][r % 8], o[t], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        Piece v[kTiles];
        read_v(slot_at, u, v);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) o[t] = matrix32(v[t], p[u], o[t]);
      }
    }
  };

  // which keys of the block at key j0 have a page (missing: some key of the workgroup's has none)
  bool missing = false;
  auto held_of = [&](int32_t j0) {
    return missing ? (uint32_t)__ballot(place_of(b, tile.seq, j0 + (lane & 31), D) >= 0) : ~0u;
  };
  // A block that some row of the wavefront does not see whole.
  auto edge = [&](int32_t block) {
    publish();
    const int32_t j0 = first_key(tile, block);
    if (missing || j0 + kBlock > tile.kept) {
      // values that are no token's: 0, whatever memory held, each wavefront in its own rows (every wavefront is here)
      const uint32_t held = held_of(j0);
      char* const dst = ring + slot_of(block) + B::kBytes + own_part;
      if (!(held >> copy_row & 1) || j0 + copy_row >= tile.kept) {
#pragma unroll
        for (int i = 0; i < B::kCopies; ++i) *reinterpret_cast<uint4*>(dst + i * B::kGroupBytes + lane * 16) = uint4{0, 0, 0, 0};
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    if (!meets(block)) return;
    Piece k[kSteps];
    Numerators p[2];
    floatx16 s;
    read_k(slot_of(block), k);
    products(k, s);
    const uint32_t held = held_of(j0);
    uint32_t drafted = 0;
    if constexpr (kTree) drafted = new_tokens_seen(a, tile, seen_words + row * a.words, j0);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int in_block = 8 * (r / 4) + 4 * h + r % 4, j = j0 + in_block;
      const bool sees = (j >= sight.lo && j <= sight.hi) || j < sight.lead || (kTree && (drafted >> in_block & 1));
      s[r] = (held >> in_block & 1) && sees ? s[r] : -INFINITY;
    }
    const float total = numerators(s, top, p);
    weigh(slot_of(block), s, total, p);
  };
  // A block that every row sees whole, its scores at hand; those of the next one are issued ahead of its exponentials.
  uint32_t here = 0;                    // its slot
  auto after = [](uint32_t slot_at) { return (slot_at + kSlotBytes) & (kChunkSlots * kSlotBytes - 1); };
  auto inside = [&](floatx16& s, floatx16& ahead) {
    Piece k[kSteps];
    Numerators p[2];
    read_k(after(here), k);
    products(k, ahead);
    const float total = numerators(s, top, p);
    weigh(here, s, total, p);
    here = after(here);
  };

  if (first_block < end_block) {
    // Does a token's key miss its page?  Asked while Q is on its way: where none does, and that is nearly always, no block
    // asks again.
    const int apart = kWholeTiles ? 16 : 1;
    for (int32_t i = tid; i < (end_block - first_block) * (kBlock / apart); i += kWaves * kWave) {
      const int32_t j = first_key(tile, first_block + i / (kBlock / apart)) + i % (kBlock / apart) * apart;
      const uint32_t c = quotient((uint32_t)j, b.page);
      missing |= (uint32_t)b.page_table[(int64_t)tile.seq * b.pages_per_seq + min(c, last_column)] >= b.n_pages && j < tile.kept;
    }
    missing = __syncthreads_or(missing);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) asm volatile("" : "+v"(qf[i]));   // Q has arrived: from here on only the copies are counted
    if constexpr (kWholeTiles) start_at(first_block);
    else ask();
    for (int i = 0; i < kChunkAhead; ++i) issue();
    // blocks [inner, outer) are seen whole by every row (none where pages are missing)
    int32_t inner = end_block, outer = end_block;
    if (!missing) {
      const int32_t from = lo_max <= tile.base ? 0 : (lo_max - tile.base + kBlock - 1) / kBlock;
      const int32_t to = hi_min + 1 <= tile.base ? 0 : (hi_min + 1 - tile.base) / kBlock;
      inner = max(max(first_block, tile.lead), tile.lead + from);
      outer = min(end_block, tile.lead + to);
      if (inner >= outer) inner = outer = end_block;
    }
    int32_t block = first_block;
    for (; block < inner; ++block) edge(block);
    if (block < outer) {
      floatx16 s_a, s_b;
      here = slot_of(block);
      {
        Piece k[kSteps];
        publish();
        read_k(here, k);
        products(k, s_a);
      }
      for (; block + 2 < outer; block += 2) {
        inside(s_a, s_b);
        publish();
        inside(s_b, s_a);
        publish();
      }
      Numerators p[2];
      if (block + 1 < outer) {
        inside(s_a, s_b);
        publish();
        const float total = numerators(s_b, top, p);
        weigh(here, s_b, total, p);
        block += 2;
      } else {
        const float total = numerators(s_a, top, p);
        weigh(here, s_a, total, p);
        ++block;
      }
    }
    for (; block < end_block; ++block) edge(block);
    // every copy has landed and every wavefront is done with the ring: its space takes the results
    wait_loads_except<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
  if (own_first >= tile.count) return;
  const int own_count = min(tile.count - own_first, 32);
  float* const part = pieces > 1 ? record_of<D, kChunkRows>(a, record) : nullptr;
  auto place_out = [&](int32_t r, int32_t& h_out, int32_t& row_out) {
    const int32_t f = tile.first + own_first + r, tok = (int32_t)quotient((uint32_t)f, a.group);
    h_out = head_kv * group + (f - tok * group);
    row_out = tile.begin + tok;
  };
  bool finite = true;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) finite = finite && __builtin_isfinite(o[t][r]);
  if (!__all(finite)) {
    for (int r = 0; r < own_count; ++r) {
      float x[(D + 63) / 64], row_top, row_total;
      attend_row<T, D, kTree>(a, tile, head_kv, tile.first + own_first + r, first_block, end_block, 1, row_top, row_total, x);
      if (part) {
#pragma unroll
        for (int c = 0; c < (D + 63) / 64; ++c)
          if (lane + 64 * c < D) part[(own_first + r) * D + lane + 64 * c] = x[c];
        if (lane == 0) {
          part[kChunkRows * D + own_first + r] = row_top;
          part[kChunkRows * (D + 1) + own_first + r] = row_total;
        }
        continue;
      }
      int32_t h_out, row_out;
      place_out(r, h_out, row_out);
      const float inv = row_total != 0.f ? 1.f / row_total : 0.f;
      T* to = static_cast<T*>(a.O) + (int64_t)h_out * a.o_head + (int64_t)row_out * a.o_row;
#pragma unroll
      for (int c = 0; c < (D + 63) / 64; ++c)
        if (lane + 64 * c < D) to[lane + 64 * c] = (T)(x[c] * inv);
      if (a.lse && lane == 0)
        a.lse[(int64_t)h_out * b.n_tokens + row_out] = (row_top + __builtin_amdgcn_logf(row_total)) * kLn2;
    }
    return;
  }
  const float total = sum + other_half(sum, h);
  if (part) {
    if (!exists) return;
    // register 4 g + e of tile t: channel 32 t + 8 g + 4 h + e, in full precision kTiles (8 g + 4 h + e) + t
    if constexpr (kSingle) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        vec_t<float, kTiles> w;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) w[t] = o[t][r];
        *reinterpret_cast<vec_t<float, kTiles>*>(part + row * D + kTiles * (8 * (r / 4) + 4 * h + r % 4)) = w;
      }
    } else {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4v*>(part + row * D + 32 * t + 8 * g + 4 * h) =
              float4v{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]};
    }
    if (h == 0) {
      part[kChunkRows * D + row] = top;
      part[kChunkRows * (D + 1) + row] = total;
    }
    return;
  }
  // A lane holds pieces of its own row; the rows go through LDS and leave whole.
  const float inv = total != 0.f ? 1.f / total : 0.f;
  constexpr int kPitch = B::kRowBytes + 16, kRowPieces = B::kRowBytes / 16;
  static_assert(kWaves * 32 * kPitch <= kChunkSlots * kSlotBytes, "the results fit the ring");
  char* const mine = ring + wave * (32 * kPitch);
  if constexpr (kSingle) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      vec_t<float, kTiles> w;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) w[t] = o[t][r] * inv;
      *reinterpret_cast<vec_t<float, kTiles>*>(mine + n * kPitch + kTiles * (8 * (r / 4) + 4 * h + r % 4) * 4) = w;
    }
  } else {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        vec_t<T, 4> w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (T)(o[t][4 * g + e] * inv);
        *reinterpret_cast<vec_t<T, 4>*>(mine + n * kPitch + (32 * t + 8 * g + 4 * h) * 2) = w;
      }
  }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 32 * kRowPieces / kWave; ++i) {
    const int r = lane / kRowPieces + i * (kWave / kRowPieces), at = lane % kRowPieces;
    if (r < own_count) {
      int32_t h_out, row_out;
      place_out(r, h_out, row_out);
      *reinterpret_cast<Piece*>(static_cast<T*>(a.O) + (int64_t)h_out * a.o_head + (int64_t)row_out * a.o_row + at * kPieceElems) =
          *reinterpret_cast<const Piece*>(mine + r * kPitch + at * 16);
    }
  }
  if (a.lse && h == 0 && exists) a.lse[(int64_t)head * b.n_tokens + tile.begin + token] = (top + __builtin_amdgcn_logf(total)) * kLn2;
}

// Joins the parts of a tile, in their order.  The records of four parts are loaded at a time.
template <typename T, int D, int kTileRows, typename Record>
__device__ __forceinline__ void join_parts(const PagedAttention& a, const Note& note, int32_t row0, Record record) {
  constexpr int kPer = D / 16, kAtOnce = 4;
  const Tile tile = tile_of<kTileRows, false>(a, 0, note.begin, note.n_new, note.length, note.tile);
  const int row = row0 + threadIdx.x / 16, channel = threadIdx.x % 16 * kPer;
  if (row >= tile.count) return;
  float high = -INFINITY, total = 0.f, x[kPer];
#pragma unroll
  for (int c = 0; c < kPer; ++c) x[c] = 0.f;
  for (int32_t i = 0; i < note.count; i += kAtOnce) {
    float top[kAtOnce], sum[kAtOnce];
    vec_t<float, kPer> o[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float* const p = record(min(i + k, note.count - 1));
      top[k] = p[kTileRows * D + row];
      sum[k] = p[kTileRows * (D + 1) + row];
      o[k] = *reinterpret_cast<const vec_t<float, kPer>*>(p + row * D + channel);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (i + k >= note.count || sum[k] == 0.f) continue;   // no key seen
      const float best = fmaxf(high, top[k]), against = best > -INFINITY ? best : 0.f;
      const float keep = __builtin_amdgcn_exp2f(high - against), weight = __builtin_amdgcn_exp2f(top[k] - against);
      high = best;
      const float kept = total == 0.f ? 0.f : keep;          // (nothing yet: not 0 times what an infinity leaves)
      total = kept * total + weight * sum[k];
#pragma unroll
      for (int c = 0; c < kPer; ++c) x[c] = kept * x[c] + weight * o[k][c];
    }
  }
  store_row<T, D>(a, tile, note.head, row, channel, x, high, total);
}

// ... tiles that end in a share and begin in an earlier one
template <typename T, int D, int kTileRows>
__global__ __launch_bounds__(kWaves* kWave) void paged_join_kernel(PagedAttention a) {
  const Note note = notes_of(a)[blockIdx.x];
  if (note.count == 0) return;
  join_parts<T, D, kTileRows>(a, note, blockIdx.y * 16,
                              [&](int32_t i) { return record_of_share<D, kTileRows>(a, note.first + i, i > 0); });
}

// ... tiles of 128 rows in pieces (16 rows a workgroup: 64 made a chunk of 32 tokens behind 32k 69 us instead of 48)
template <typename T, int D>
__global__ __launch_bounds__(kWaves* kWave) void paged_chunk_join_kernel(PagedAttention a) {
  const Note note = notes_of(a)[blockIdx.x];
  if (note.count == 0) return;
  join_parts<T, D, kChunkRows>(a, note, blockIdx.y * 16,
                               [&](int32_t i) { return record_of<D, kChunkRows>(a, note.first + (int64_t)i * note.apart); });
}

template <typename T, int D, int N, bool kTree>
sga_status launch_paged_rows(const PagedAttention& a) {
  const dim3 block(kWaves * kWave);
  profile_mark_begin(a.stream, "paged_kernel");
  if (a.batch.page.value % 16 == 0) paged_kernel<T, D, N, true, kTree><<<dim3(a.groups), block, 0, a.stream>>>(a);
  else paged_kernel<T, D, N, false, kTree><<<dim3(a.groups), block, 0, a.stream>>>(a);
  profile_mark_end(a.stream);
  if (a.partials) paged_join_kernel<T, D, 16 * N><<<dim3(a.groups, N), block, 0, a.stream>>>(a);
  return hip_status(hipGetLastError());
}

template <typename T, int D, bool kTree>
sga_status launch_paged_as(const PagedAttention& a) {
  const dim3 block(kWaves * kWave);
  if (a.tile_rows == kChunkRows) {
    if constexpr (chunk_fits(sizeof(T) * D)) {
      int64_t groups = (int64_t)a.slots * a.Hkv;
      if (a.Hkv < 8 && 8 % a.Hkv == 0) groups = (int64_t)(a.slots + 8 / a.Hkv - 1) / (8 / a.Hkv) * 8;
      profile_mark_begin(a.stream, "paged_chunk_kernel");
      if (a.batch.page.value % 16 == 0) paged_chunk_kernel<T, D, true, kTree><<<dim3((unsigned)groups), block, 0, a.stream>>>(a);
      else paged_chunk_kernel<T, D, false, kTree><<<dim3((unsigned)groups), block, 0, a.stream>>>(a);
      profile_mark_end(a.stream);
      if (a.partials) paged_chunk_join_kernel<T, D><<<dim3((unsigned)a.groups, kChunkRows / 16), block, 0, a.stream>>>(a);
    }
    return hip_status(hipGetLastError());
  }
  if constexpr (!(sizeof(T) == 4 && D > 64))        // (the registers do not hold two groups of such rows)
    if (a.tile_rows != kRows) return launch_paged_rows<T, D, 2, kTree>(a);
  return launch_paged_rows<T, D, 1, kTree>(a);
}

template <typename T, bool kTree>
sga_status launch_paged_type(const PagedAttention& a) {
  switch (a.d) {
    case 32: return launch_paged_as<T, 32, kTree>(a);
    case 64: return launch_paged_as<T, 64, kTree>(a);
    case 128: return launch_paged_as<T, 128, kTree>(a);
    default: return launch_paged_as<T, 256, kTree>(a);
  }
}

}  // namespace

PagedPlan plan_paged(const PagedAttention& a) {
  PagedPlan p{kRows, 0, 0, 1, 0};
  const int64_t all_rows = (int64_t)a.batch.n_tokens * a.group.value;
  // (fp32 at d = 64 under a narrow window: a wavefront meets 9 of the 13 blocks of its workgroup's tile, and waits in the others; us,
  // short tiles / tiles of 128 rows, documents of 900 to 4,096 tokens, 8 heads: 128 causal 79 / 90, +-64 80 / 92, +-128 118 / 120, with 16 global
  // rows and pages of 24 139 / 148; 300 causal 120 / 125, 400 156 / 141, +-200 174 / 151.  At d = 32 128 causal 53 / 42, +-64 53 / 42; at d = 128, 256 causal 315 / 296.)
  const bool single = a.dtype == SGA_F32, narrow = single && a.d == 64 && (a.causal ? 1 : 2) * (int64_t)a.window <= 256;
  const int64_t room = (int64_t)a.batch.pages_per_seq * a.batch.page.value, tokens = a.L < room ? a.L : room;      // of a sequence at most
  if (chunk_fits((int64_t)a.d * (single ? 4 : 2)) && !narrow && all_rows > (int64_t)token_rows(single, a.d, tokens) * a.batch.n_seqs)
    p.tile_rows = kChunkRows;
  else if (all_rows > (int64_t)kRows * a.batch.n_seqs && !(a.dtype == SGA_F32 && a.d > 64))
    p.tile_rows = 2 * kRows;
  const int64_t tiles = all_rows / p.tile_rows + a.batch.n_seqs;
  if (tiles >= int64_t(1) << 24) return p;                 // (rows of a sequence are counted in 31 bits)
  // keys that a tile meets at most
  const int64_t step = p.tile_rows / (int64_t)a.group.value;
  int64_t keys = tokens;
  if (a.words > 0) keys = (int64_t)a.L + 32 * a.words < room ? (int64_t)a.L + 32 * a.words : room;      // (new tokens by their places)
  const int64_t window = (a.causal ? 1 : 2) * (int64_t)a.window + step + 1 + a.n_global + 32 * a.words;
  if (window < keys && !(a.n_global > 0 && !a.causal)) keys = window;
  if (p.tile_rows == kChunkRows) {
    // cut where the chip would have less than four rounds of tiles, and where a tile can be long enough for two pieces (see piece_of; full
    // precision would cut from 128 keys on, for which a join does not pay)
    const int64_t least = least_piece(a.words > 0, a.dtype);
    p.splits = tiles * a.Hkv < 2048 && keys > kLeastShare && 2 * (keys + kTileCost) >= 3 * least ? 2 : 1;
    const int64_t slots = tiles + (p.splits > 1 ? (kChunkPieces + a.Hkv - 1) / a.Hkv + 1 : 0);
    if (slots * a.Hkv + 8 >= int64_t(1) << 24) return p;                    // (a grid holds fewer than 2^32 threads)
    p.slots = (int32_t)slots;
    p.groups = (int32_t)(slots * a.Hkv);
    if (p.splits > 1) p.bytes = (size_t)p.groups * (kNoteBytes + kChunkRows * (a.d + 2) * sizeof(float));
    return p;
  }
  // workgroups that the chip holds at once, and that have the least share to do if every tile met all the keys that it can
  const int64_t row_bytes = (int64_t)a.d * (a.dtype == SGA_F32 ? 4 : 2) * (p.tile_rows / kRows);
  const int64_t groups = a.d == 256 ? 256 : row_bytes > 128 ? 512 : 768;
  const int64_t share = a.words > 0 ? kLeastShareTree : kLeastShare, work = (tiles * a.Hkv * (keys + kTileCost) + share - 1) / share;
  p.groups = (int32_t)(work < groups ? (work > 1 ? work : 1) : groups);
  if (p.groups > 1) p.bytes = (size_t)p.groups * (kNoteBytes + 2 * p.tile_rows * (a.d + 2) * sizeof(float));
  return p;
}

sga_status launch_paged(const PagedAttention& a) {
  const bool tree = a.depth != nullptr;
  switch (a.dtype) {
    case SGA_F32: return tree ? launch_paged_type<float, true>(a) : launch_paged_type<float, false>(a);
    case SGA_F16: return tree ? launch_paged_type<f16_t, true>(a) : launch_paged_type<f16_t, false>(a);
    default: return tree ? launch_paged_type<bf16_t, true>(a) : launch_paged_type<bf16_t, false>(a);
  }
}

}  // namespace sga

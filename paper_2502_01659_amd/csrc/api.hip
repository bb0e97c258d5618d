// C ABI of libsga.so: argument validation and dispatch.  See include/sga.h for the contract.
#include "sga_internal.h"
#include "serving.h"

#include <atomic>
#include <cstring>
#include <vector>

using namespace sga;

namespace {

// Profiling state (benchmark use only; not thread-safe).  Event pairs are created while a
// recording runs and destroyed when it is switched off.
struct ProfileState {
  bool on = false;
  bool failed = false;          // an event could not be created: reported by sga_profile_collect
  size_t used = 0;
  const char* kernel = "";      // name of the kernel inside the most recent pair
  std::vector<hipEvent_t> start, stop;
};
ProfileState g_prof;

// ---- scratch of the entry point that allocates nothing ------------------------------------------
// One array per device, in the library's own device image: it exists from the moment the image is
// loaded on a device until the process ends.  In host code `scratch` is only a handle for
// hipGetSymbolAddress; the address a kernel can use is resolved once per device and kept here.
constexpr size_t kScratchBytes = size_t(64) << 20;
__device__ __align__(256) static unsigned char scratch[kScratchBytes];
constexpr int kMaxDevices = 64;
std::atomic<void*> g_scratch_ptr[kMaxDevices];

// Device address of `scratch` on the current device (resolved on the first call per device).
sga_status scratch_of_current_device(void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return SGA_ERR_HIP;
  if (dev < 0 || dev >= kMaxDevices) return SGA_ERR_UNSUPPORTED;
  void* p = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (!p) {
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) {
      (void)hipGetLastError();
      return SGA_ERR_HIP;
    }
    g_scratch_ptr[dev].store(p, std::memory_order_release);
  }
  *out = p;
  return SGA_OK;
}

constexpr uint32_t kPlanMagic = 0x53474150u;   // marks a record written by sga_graph_prepare

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

sga_status check_common(const void* Q, const void* K, const void* V, const void* O, int64_t L,
                        int32_t H, int32_t d, int32_t dtype, int32_t path, const void* ws,
                        size_t ws_bytes) {
  if (!Q || !K || !V || !O) return SGA_ERR_INVALID_ARG;
  if (L < 1 || L >= (int64_t(1) << 31) || H < 1 || H > 65535) return SGA_ERR_INVALID_ARG;
  if (dtype != SGA_F32 && dtype != SGA_F16) return SGA_ERR_INVALID_ARG;
  if (path != SGA_PATH_AUTO && path != SGA_PATH_GATHER && path != SGA_PATH_TILE &&
      path != SGA_PATH_TILE_SPLIT)
    return SGA_ERR_INVALID_ARG;
  if (path == SGA_PATH_TILE_SPLIT && (dtype != SGA_F32 || d != kHeadDim)) return SGA_ERR_UNSUPPORTED;
  if (d != 32 && d != 64 && d != 128 && d != 256) return SGA_ERR_UNSUPPORTED;
  if (path == SGA_PATH_TILE && d < kHeadDim) return SGA_ERR_UNSUPPORTED;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return SGA_ERR_INVALID_ARG;
  if (ws && (reinterpret_cast<uintptr_t>(ws) & 255u)) return SGA_ERR_INVALID_ARG;
  if (!ws && ws_bytes != 0) return SGA_ERR_INVALID_ARG;
  return SGA_OK;
}

}  // namespace

namespace sga {

void profile_mark_begin(hipStream_t stream, const char* kernel) {
  if (!g_prof.on || g_prof.failed) return;
  if (g_prof.used == g_prof.start.size()) {
    hipEvent_t a, b;
    // (no system-scope fence at the records: they only take time stamps on the stream)
    if (hipEventCreateWithFlags(&a, hipEventDisableSystemFence) != hipSuccess) {
      g_prof.failed = true;
      return;
    }
    if (hipEventCreateWithFlags(&b, hipEventDisableSystemFence) != hipSuccess) {
      (void)hipEventDestroy(a);
      g_prof.failed = true;
      return;
    }
    g_prof.start.push_back(a);
    g_prof.stop.push_back(b);
  }
  g_prof.kernel = kernel;
  (void)hipEventRecord(g_prof.start[g_prof.used], stream);
}

void profile_mark_end(hipStream_t stream) {
  if (!g_prof.on || g_prof.failed || g_prof.used >= g_prof.stop.size()) return;
  (void)hipEventRecord(g_prof.stop[g_prof.used], stream);
  ++g_prof.used;
}

}  // namespace sga

extern "C" {

sga_status sga_profile_enable(int32_t on) {
  g_prof.on = on != 0;
  g_prof.used = 0;
  g_prof.failed = false;
  g_prof.kernel = "";
  if (!g_prof.on) {             // the recording's events go with it
    for (hipEvent_t e : g_prof.start) (void)hipEventDestroy(e);
    for (hipEvent_t e : g_prof.stop) (void)hipEventDestroy(e);
    g_prof.start.clear();
    g_prof.stop.clear();
  }
  return SGA_OK;
}

sga_status sga_profile_collect(float* ms_out, int32_t capacity, int32_t* n_out) {
  if (!n_out || (capacity > 0 && !ms_out) || capacity < 0) return SGA_ERR_INVALID_ARG;
  *n_out = 0;
  if (g_prof.failed) return SGA_ERR_HIP;
  for (size_t i = 0; i < g_prof.used; ++i) {
    if (hipEventSynchronize(g_prof.stop[i]) != hipSuccess) return SGA_ERR_HIP;
    if ((int64_t)i >= capacity) continue;
    float ms = 0.f;
    if (hipEventElapsedTime(&ms, g_prof.start[i], g_prof.stop[i]) != hipSuccess) return SGA_ERR_HIP;
    ms_out[i] = ms;
  }
  *n_out = (int32_t)g_prof.used;
  g_prof.used = 0;
  return SGA_OK;
}

const char* sga_profile_last_kernel(void) { return g_prof.kernel; }

const char* sga_status_string(sga_status s) {
  switch (s) {
    case SGA_OK: return "ok";
    case SGA_ERR_INVALID_ARG: return "invalid argument";
    case SGA_ERR_UNSUPPORTED: return "unsupported configuration";
    case SGA_ERR_WORKSPACE: return "workspace or output capacity too small";
    case SGA_ERR_OVERFLOW: return "size overflow";
    case SGA_ERR_HIP: return "HIP runtime error";
    default: return "unknown status";
  }
}

sga_status sga_mask_nnz(const sga_mask_desc* desc, int64_t* nnz_out) {
  if (!nnz_out) return SGA_ERR_INVALID_ARG;
  const sga_status st = mask_validate(desc);
  if (st != SGA_OK) return st;
  *nnz_out = mask_total_edges(*desc);
  return SGA_OK;
}

sga_status sga_build_mask(const sga_mask_desc* desc, int64_t* row_ptr, int32_t* col_idx,
                          int64_t col_capacity, void* stream) {
  const sga_status st = mask_validate(desc);
  if (st != SGA_OK) return st;
  if (!row_ptr || !col_idx) return SGA_ERR_INVALID_ARG;
  if (col_capacity < mask_total_edges(*desc)) return SGA_ERR_WORKSPACE;
  (void)hipGetLastError();   // drop stale errors of earlier, unrelated runtime calls
  return launch_build_mask(*desc, row_ptr, col_idx, static_cast<hipStream_t>(stream));
}

sga_status sga_validate_csr(const int64_t* row_ptr, const int32_t* col_idx, int64_t L,
                            int64_t col_capacity, void* scratch, int64_t* bad_row_out, void* stream) {
  if (!row_ptr || !col_idx || !scratch || (reinterpret_cast<uintptr_t>(scratch) & 7)) return SGA_ERR_INVALID_ARG;
  if (L < 1 || L >= (int64_t(1) << 31) || col_capacity < 0) return SGA_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // drop stale errors of earlier, unrelated runtime calls
  unsigned long long* verdict = static_cast<unsigned long long*>(scratch);
  const sga_status launched = launch_validate_csr(row_ptr, col_idx, L, col_capacity, verdict, st);
  if (launched != SGA_OK) return launched;
  unsigned long long found[2] = {0, 0};   // in the row offsets, in the columns
  if (hipMemcpyAsync(found, verdict, sizeof(found), hipMemcpyDeviceToHost, st) != hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return SGA_ERR_HIP;
  const unsigned long long bad = found[0] < found[1] ? found[0] : found[1];
  if (bad_row_out) *bad_row_out = bad == ~0ull ? -1 : (int64_t)bad;
  return bad == ~0ull ? SGA_OK : SGA_ERR_INVALID_ARG;
}

sga_status sga_workspace_bytes(int64_t L, int32_t H, int32_t d, int32_t dtype, int64_t nnz,
                               size_t* bytes_out) {
  if (!bytes_out) return SGA_ERR_INVALID_ARG;
  if (L < 1 || L >= (int64_t(1) << 31) || H < 1 || H > 65535) return SGA_ERR_INVALID_ARG;
  if (dtype != SGA_F32 && dtype != SGA_F16) return SGA_ERR_INVALID_ARG;
  if (d != 32 && d != 64 && d != 128 && d != 256) return SGA_ERR_UNSUPPORTED;
  if (nnz < -1 || nnz > L * L) return SGA_ERR_INVALID_ARG;
  // (a caller that passes an upper bound of the edge count still gets enough for the shorter
  // work items the kernels may choose from the real count)
  const size_t chosen = plan_workspace(L, H, nnz, dtype, d).total_bytes;
  const size_t shortest = plan_workspace(L, H, nnz, dtype, d, seg_shift_min(dtype)).total_bytes;
  *bytes_out = chosen > shortest ? chosen : shortest;
  return SGA_OK;
}

}  // extern "C"

namespace {

sga_status run_explicit_call(const void* Q, const void* K, const void* V, const int64_t* row_ptr,
                             const int32_t* col_idx, void* O, int64_t L, int32_t H, int32_t d,
                             float scale, void* stream, int32_t dtype, float* lse, void* workspace,
                             size_t workspace_bytes, int32_t path, bool accumulate,
                             const sga_graph_plan* plan = nullptr, bool prepared = false) {
  const sga_status st = check_common(Q, K, V, O, L, H, d, dtype, path, workspace, workspace_bytes);
  if (st != SGA_OK) return st;
  if (!row_ptr || !col_idx) return SGA_ERR_INVALID_ARG;
  if (accumulate && !lse) return SGA_ERR_INVALID_ARG;
  if (prepared) {
    // the plan must have been prepared for exactly these buffers and this problem
    if (!plan || plan->struct_bytes != sizeof(sga_graph_plan) || plan->magic != kPlanMagic)
      return SGA_ERR_INVALID_ARG;
    if (plan->L != L || plan->H != H || plan->d != d || plan->dtype != dtype || plan->row_ptr != row_ptr ||
        plan->col_idx != col_idx || plan->workspace != workspace || plan->workspace_bytes != workspace_bytes)
      return SGA_ERR_INVALID_ARG;
    if (path == SGA_PATH_GATHER) return SGA_ERR_INVALID_ARG;
  }
  AttnArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.O = O; a.lse = lse;
  a.L = L; a.H = H; a.scale = scale; a.dtype = dtype; a.d = d;
  a.stream = static_cast<hipStream_t>(stream);
  a.row_ptr = row_ptr; a.col_idx = col_idx;
  a.ws = workspace; a.ws_bytes = workspace_bytes;
  a.accumulate = accumulate;
  a.split = path == SGA_PATH_TILE_SPLIT;
  if ((path == SGA_PATH_TILE || path == SGA_PATH_TILE_SPLIT) && (!workspace || workspace_bytes < 256))
    return SGA_ERR_WORKSPACE;
  // the MFMA tile kernels work on 64-channel slices (d = 64, 128, 256); d = 32 runs on the per-row kernels
  const bool gather_only = path == SGA_PATH_GATHER || d < kHeadDim;
  (void)hipGetLastError();   // drop stale errors of earlier, unrelated runtime calls
  if (prepared) {
    const bool parts_fit = (plan->flags & SGA_GRAPH_TILE_PARTS_FIT) != 0;
    a.prepared = true;
    a.plan_multi_tiles = parts_fit ? plan->multi_tiles : 0;
    a.plan_tiles_cover_all = (plan->flags & SGA_GRAPH_TILES_COVER_ALL) != 0;
    a.plan_rows_left = parts_fit ? (int64_t)plan->tiles_left * kTile : L;
    a.plan_no_tiles = (int64_t)plan->tiles_left == (L + kTile - 1) / kTile;
    a.plan_long_rows = (plan->flags & SGA_GRAPH_ROW_CHUNKS_FIT) ? plan->long_rows : 0;
    a.plan_rows_even = (plan->flags & SGA_GRAPH_ROWS_EVEN) != 0;
    a.plan_rows_share = (plan->flags & SGA_GRAPH_ROWS_SHARE_KEYS) != 0;
    return launch_tile_explicit(a);
  }
  // (the per-row kernels alone use the workspace for split rows only, and no row of up to kSplitThreshold
  // neighbours is split where there are no longer ones: the verification runs, 11.2 -> 8.4 us)
  if (workspace && workspace_bytes >= 256 && !(gather_only && L <= kSplitThreshold)) clear_workspace(a, !gather_only);
  if (gather_only) return launch_gather_explicit(a, true, false);
  return launch_tile_explicit(a);
}

sga_status run_implicit_call(const void* Q, const void* K, const void* V, const sga_mask_desc* desc,
                             void* O, int64_t L, int32_t H, int32_t d, float scale, void* stream,
                             int32_t dtype, float* lse, void* workspace, size_t workspace_bytes,
                             int32_t path, bool accumulate) {
  sga_status st = check_common(Q, K, V, O, L, H, d, dtype, path, workspace, workspace_bytes);
  if (st != SGA_OK) return st;
  st = mask_validate(desc);
  if (st != SGA_OK) return st;
  if (desc->L != L) return SGA_ERR_INVALID_ARG;
  if (accumulate && !lse) return SGA_ERR_INVALID_ARG;
  const int32_t kind = desc->kind;
  if (kind != SGA_MASK_SLIDING && kind != SGA_MASK_DILATED && kind != SGA_MASK_NONLOCAL &&
      kind != SGA_MASK_DILATED_2D)
    return SGA_ERR_UNSUPPORTED;
  AttnArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.O = O; a.lse = lse;
  a.L = L; a.H = H; a.scale = scale; a.dtype = dtype; a.d = d;
  a.stream = static_cast<hipStream_t>(stream);
  a.mask_kind = kind;
  a.stride = (kind == SGA_MASK_DILATED || kind == SGA_MASK_DILATED_2D) ? desc->stride : 1;
  const int64_t wmax = (L - 1) / a.stride;
  a.window = (int32_t)(desc->window < wmax ? desc->window : wmax);
  // 2-D dilated blocks: the selected rows of a block all see each other
  if (kind == SGA_MASK_DILATED_2D) a.window = (int32_t)(((desc->block < L ? desc->block : L) - 1) / a.stride);
  a.n_global = desc->n_global;
  a.block = desc->block;
  a.ws = workspace; a.ws_bytes = workspace_bytes;
  a.accumulate = accumulate;
  a.split = path == SGA_PATH_TILE_SPLIT;
  a.tiles_allowed = path != SGA_PATH_GATHER;
  (void)hipGetLastError();   // drop stale errors of earlier, unrelated runtime calls
  if (kind == SGA_MASK_NONLOCAL) {
    const int64_t g = desc->n_global < L ? desc->n_global : L;
    if (g > kMaxImplicitGlobal) return SGA_ERR_UNSUPPORTED;
    if (g > 0 && (!workspace || workspace_bytes < plan_workspace(L, H, -1, dtype, d).total_bytes))
      return SGA_ERR_WORKSPACE;
    return launch_gather_implicit(a);
  }
  if (path == SGA_PATH_GATHER || d < kHeadDim)
    return launch_gather_implicit(a);
  // 2-D dilated blocks with fewer than 16 selected rows would leave most of a 32-query tile
  // empty: the per-row kernels handle them
  if (kind == SGA_MASK_DILATED_2D && path == SGA_PATH_AUTO && a.window + 1 < 16)
    return launch_gather_implicit(a);
  return launch_tile_implicit(a);
}

}  // namespace

extern "C" {

sga_status sga_attention_forward(const void* Q, const void* K, const void* V, const int64_t* row_ptr,
                                 const int32_t* col_idx, void* O, int64_t L, int32_t H, int32_t d,
                                 float scale, void* stream, int32_t dtype, float* lse,
                                 void* workspace, size_t workspace_bytes, int32_t path) {
  return run_explicit_call(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype, lse, workspace,
                           workspace_bytes, path, false);
}

sga_status sga_attention_forward_implicit(const void* Q, const void* K, const void* V,
                                          const sga_mask_desc* desc, void* O, int64_t L, int32_t H,
                                          int32_t d, float scale, void* stream, int32_t dtype,
                                          float* lse, void* workspace, size_t workspace_bytes,
                                          int32_t path) {
  return run_implicit_call(Q, K, V, desc, O, L, H, d, scale, stream, dtype, lse, workspace,
                           workspace_bytes, path, false);
}

sga_status sga_attention_accumulate(const void* Q, const void* K, const void* V, const int64_t* row_ptr,
                                    const int32_t* col_idx, void* O, int64_t L, int32_t H, int32_t d,
                                    float scale, void* stream, int32_t dtype, float* lse,
                                    void* workspace, size_t workspace_bytes, int32_t path) {
  return run_explicit_call(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype, lse, workspace,
                           workspace_bytes, path, true);
}

sga_status sga_attention_accumulate_implicit(const void* Q, const void* K, const void* V,
                                             const sga_mask_desc* desc, void* O, int64_t L, int32_t H,
                                             int32_t d, float scale, void* stream, int32_t dtype,
                                             float* lse, void* workspace, size_t workspace_bytes,
                                             int32_t path) {
  return run_implicit_call(Q, K, V, desc, O, L, H, d, scale, stream, dtype, lse, workspace,
                           workspace_bytes, path, true);
}

sga_status sga_graph_prepare(const int64_t* row_ptr, const int32_t* col_idx, int64_t L, int32_t H,
                             int32_t d, int32_t dtype, void* workspace, size_t workspace_bytes,
                             void* stream, sga_graph_plan* plan_out) {
  if (!row_ptr || !col_idx || !plan_out) return SGA_ERR_INVALID_ARG;
  if (L < 1 || L >= (int64_t(1) << 31) || H < 1 || H > 65535) return SGA_ERR_INVALID_ARG;
  if (dtype != SGA_F32 && dtype != SGA_F16) return SGA_ERR_INVALID_ARG;
  if (d != 64 && d != 128 && d != 256) return SGA_ERR_UNSUPPORTED;   // the tile kernels' sizes
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return SGA_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  // the edge count sizes the workspace layout; only the device knows it
  int64_t nnz = -1;
  if (hipMemcpyAsync(&nnz, row_ptr + L, sizeof(nnz), hipMemcpyDeviceToHost, st) != hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return SGA_ERR_HIP;
  if (nnz < 0 || nnz > L * L) return SGA_ERR_INVALID_ARG;
  const WorkspacePlan pl = plan_workspace(L, H, nnz, dtype, d);
  if (pl.total_bytes > workspace_bytes) return SGA_ERR_WORKSPACE;
  AttnArgs a{};
  a.L = L; a.H = H; a.dtype = dtype; a.d = d; a.stream = st;
  a.row_ptr = row_ptr; a.col_idx = col_idx;
  a.ws = workspace; a.ws_bytes = workspace_bytes;
  clear_workspace(a, true);
  launch_tile_analyze(a);
  if (L > kSplitThreshold && tile_parts_in_doubt(pl)) launch_split_prepass(a, true);
  launch_row_lengths(a);
  uint32_t ctr[kNumCounters];
  if (hipGetLastError() != hipSuccess ||
      hipMemcpyAsync(ctr, workspace, sizeof(ctr), hipMemcpyDeviceToHost, st) != hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return SGA_ERR_HIP;
  sga_graph_plan p{};
  p.struct_bytes = sizeof(sga_graph_plan);
  p.magic = kPlanMagic;
  p.L = L; p.nnz = nnz; p.H = H; p.d = d; p.dtype = dtype;
  p.tiles_left = ctr[kCtrTilesBad];
  p.multi_tiles = ctr[kCtrMultiTiles];
  p.tile_parts = ctr[kCtrTilePartsNeeded];
  p.long_rows = ctr[kCtrLongRows];
  p.row_chunks = ctr[kCtrChunksNeeded];
  const bool parts_fit = (int64_t)p.tile_parts <= pl.cap_tparts;
  const bool chunks_fit = (int64_t)p.row_chunks <= pl.cap_items;
  p.flags = (parts_fit ? SGA_GRAPH_TILE_PARTS_FIT : 0) | (chunks_fit ? SGA_GRAPH_ROW_CHUNKS_FIT : 0) |
            (p.tiles_left == 0 && parts_fit ? SGA_GRAPH_TILES_COVER_ALL : 0);
  if (chunks_fit && shared_chunks_possible(L, H, d, dtype, workspace_bytes) &&
      shared_chunks(pl, nnz, L, H, d, dtype, ctr))
    p.flags |= SGA_GRAPH_ROWS_SHARE_KEYS;
  uint64_t squares;
  std::memcpy(&squares, ctr + kCtrLengthSquares, sizeof(squares));
  if ((int64_t)p.tiles_left == pl.n_tiles && p.long_rows == 0 &&
      rows_of_one_length(nnz, L, ctr[kCtrLongestRow], squares))
    p.flags |= SGA_GRAPH_ROWS_EVEN;
  p.row_ptr = row_ptr; p.col_idx = col_idx;
  p.workspace = workspace; p.workspace_bytes = workspace_bytes;
  *plan_out = p;
  return SGA_OK;
}

sga_status sga_attention_forward_prepared(const void* Q, const void* K, const void* V,
                                          const int64_t* row_ptr, const int32_t* col_idx, void* O,
                                          int64_t L, int32_t H, int32_t d, float scale, void* stream,
                                          int32_t dtype, float* lse, void* workspace,
                                          size_t workspace_bytes, int32_t path,
                                          const sga_graph_plan* plan) {
  return run_explicit_call(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype, lse, workspace,
                           workspace_bytes, path, false, plan, true);
}

sga_status sga_attention_accumulate_prepared(const void* Q, const void* K, const void* V,
                                             const int64_t* row_ptr, const int32_t* col_idx, void* O,
                                             int64_t L, int32_t H, int32_t d, float scale,
                                             void* stream, int32_t dtype, float* lse,
                                             void* workspace, size_t workspace_bytes, int32_t path,
                                             const sga_graph_plan* plan) {
  return run_explicit_call(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype, lse, workspace,
                           workspace_bytes, path, true, plan, true);
}

sga_status sga_static_scratch_init(void) {
  void* p = nullptr;
  return scratch_of_current_device(&p);
}

size_t sga_static_scratch_bytes(void) { return kScratchBytes; }

sga_status sga_attention_forward_static(const void* Q, const void* K, const void* V,
                                        const int64_t* row_ptr, const int32_t* col_idx, void* O,
                                        int64_t L, int32_t H, int32_t d, float scale, void* stream,
                                        int32_t dtype, float* lse, int64_t nnz, int32_t path) {
  // the library's own scratch array takes the place of the caller's workspace
  size_t need = 0;
  const sga_status sized = sga_workspace_bytes(L, H, d, dtype, nnz, &need);
  if (sized != SGA_OK) return sized;
  if (nnz < 0) return SGA_ERR_INVALID_ARG;
  if (need > kScratchBytes) return SGA_ERR_WORKSPACE;      // beyond the stated maximum
  void* ws = nullptr;
  const sga_status found = scratch_of_current_device(&ws);
  if (found != SGA_OK) return found;
  return run_explicit_call(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype, lse, ws,
                           kScratchBytes, path, false);
}

}  // extern "C"

// ---- serving ----------------------------------------------------------------------------------
namespace {

int element_bytes(int32_t dtype) { return dtype == SGA_F32 ? 4 : 2; }

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

bool valid_rows(const sga_rows* x, int32_t dtype) { return x && x->data && aligned_to(x->data, element_bytes(dtype)); }

// ... whose address and strides are multiples of 16 bytes
bool wide_rows(const sga_rows* x, int32_t dtype) {
  const int64_t step = 16 / element_bytes(dtype);
  return x && x->data && aligned16(x->data) && x->head_stride % step == 0 && x->row_stride % step == 0;
}

bool serving_dtype(int32_t dtype) { return dtype == SGA_F32 || dtype == SGA_F16 || dtype == SGA_BF16; }

bool valid_rotary(const sga_rotary_desc* r, int32_t d) {
  return r && r->struct_bytes == sizeof(sga_rotary_desc) &&
         (r->layout == SGA_ROTARY_HALF || r->layout == SGA_ROTARY_INTERLEAVED) && r->channels >= 2 && r->channels <= d &&
         r->channels % 2 == 0 && r->frequencies && aligned_to(r->frequencies, 8);
}

RotaryArgs rotary_args(const sga_rotary_desc* r, int32_t inverse) {
  if (!r) return RotaryArgs{nullptr, 1.f, 0, 0, 0};
  return RotaryArgs{r->frequencies, r->magnitude, r->channels, r->layout == SGA_ROTARY_INTERLEAVED, inverse != 0};
}

RowsArg rows_arg(const sga_rows& src, const sga_rows& dst, int32_t heads, bool rotate) {
  return RowsArg{src.data, dst.data, src.head_stride, src.row_stride, dst.head_stride, dst.row_stride, heads, rotate, 0};
}

// In place means the same elements: the same address with other strides would mix them.
bool apart_or_same(const sga_rows& x, const sga_rows& y) {
  return x.data != y.data || (x.head_stride == y.head_stride && x.row_stride == y.row_stride);
}

constexpr int32_t kMaxRotaryDim = 1024;

// What a batch has to be whatever it is used for.  (A batch without tokens needs no arrays.)
bool valid_batch(const sga_paged_batch* b, int32_t Hkv, int32_t d) {
  if (!b || b->struct_bytes != sizeof(sga_paged_batch) || b->n_seqs < 0) return false;
  if (b->n_tokens < 0 || b->n_tokens >= (int64_t(1) << 31)) return false;
  if (b->n_pages < 1 || b->n_pages >= (int64_t(1) << 31) || b->page_size < 1 || b->page_size > 65536) return false;
  if (b->pages_per_seq < 1 || (int64_t)b->pages_per_seq * b->page_size > (int64_t(1) << 31) - 1024) return false;
  if (b->page_stride < (int64_t)Hkv * b->page_size * d || b->page_stride >= (int64_t(1) << 32)) return false;
  if (b->n_tokens == 0 || b->n_seqs == 0) return true;
  return b->page_table && b->seq_ptr && b->seq_len && aligned_to(b->page_table, 4) && aligned_to(b->seq_len, 4) &&
         aligned_to(b->seq_ptr, 8);
}

PagedArgs batch_args(const sga_paged_batch& b) {
  PagedArgs a{};
  a.page_table = b.page_table; a.seq_ptr = b.seq_ptr; a.seq_len = b.seq_len;
  a.page_stride = b.page_stride;
  a.n_pages = (uint32_t)b.n_pages;
  a.n_seqs = b.n_seqs; a.n_tokens = (int32_t)b.n_tokens; a.pages_per_seq = b.pages_per_seq;
  a.page = fast_div((uint32_t)b.page_size);
  return a;
}

// The part of an attention call that its workspace depends on.
sga_status paged_shape(const sga_paged_batch* batch, const sga_mask_desc* mask, int32_t causal, int32_t Hq, int32_t Hkv,
                       int32_t d, int32_t dtype, PagedAttention& a) {
  if (!serving_dtype(dtype) || Hkv < 1 || Hq < 1 || Hq > 65535 || Hq % Hkv != 0) return SGA_ERR_INVALID_ARG;
  if (d != 32 && d != 64 && d != 128 && d != 256) return SGA_ERR_UNSUPPORTED;
  if (!valid_batch(batch, Hkv, d)) return SGA_ERR_INVALID_ARG;
  const sga_status st = mask_validate(mask);
  if (st != SGA_OK) return st;
  if (mask->kind != SGA_MASK_SLIDING && mask->kind != SGA_MASK_GLOBAL_LOCAL) return SGA_ERR_UNSUPPORTED;
  a.batch = batch_args(*batch);
  a.Hq = Hq; a.Hkv = Hkv; a.group = fast_div((uint32_t)(Hq / Hkv));
  a.L = (int32_t)mask->L;
  a.window = mask->window;
  a.n_global = mask->kind == SGA_MASK_GLOBAL_LOCAL ? mask->n_global : 0;
  a.causal = causal != 0;
  a.d = d; a.dtype = dtype;
  return SGA_OK;
}

}  // namespace

extern "C" {

sga_status sga_rotary(const sga_rows* X, const sga_rows* Y, const int64_t* positions, int64_t first, int64_t L, int32_t H,
                      int32_t d, const sga_rotary_desc* rotary, int32_t inverse, int32_t dtype, void* stream) {
  if (!X || !Y || !serving_dtype(dtype) || L < 0 || L >= (int64_t(1) << 31) || H < 1 || H > 65535) return SGA_ERR_INVALID_ARG;
  if (d < 2 || d > kMaxRotaryDim || !valid_rotary(rotary, d)) return SGA_ERR_INVALID_ARG;
  if (L == 0) return SGA_OK;
  if (!valid_rows(X, dtype) || !valid_rows(Y, dtype) || !apart_or_same(*X, *Y)) return SGA_ERR_INVALID_ARG;
  if (positions && !aligned_to(positions, 8)) return SGA_ERR_INVALID_ARG;
  (void)hipGetLastError();   // drop stale errors of earlier, unrelated runtime calls
  RotateArgs a{};
  a.tensor[0] = rows_arg(*X, *Y, H, true);
  a.n_tensors = 1;
  a.n_rows = (int32_t)L; a.d = d;
  a.positions = positions; a.first = first;
  a.rotary = rotary_args(rotary, inverse);
  a.dtype = dtype;
  a.stream = static_cast<hipStream_t>(stream);
  return launch_rotate(a);
}

sga_status sga_cache_append(const sga_rows* K, const sga_rows* V, void* cache_k, void* cache_v, const sga_paged_batch* batch,
                            int32_t Hkv, int32_t d, const sga_rotary_desc* rotary, const sga_rows* Q, const sga_rows* Q_out,
                            int32_t Hq, int32_t dtype, void* stream) {
  if (!K || !V || !serving_dtype(dtype) || Hkv < 1 || Hkv > 65535 || d < 2 || d > kMaxRotaryDim) return SGA_ERR_INVALID_ARG;
  if ((rotary && !valid_rotary(rotary, d)) || !valid_batch(batch, Hkv, d)) return SGA_ERR_INVALID_ARG;
  if ((Q != nullptr) != (Q_out != nullptr) || (Q && (!rotary || Hq < 1 || Hq > 65535))) return SGA_ERR_INVALID_ARG;
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return SGA_OK;
  if (!valid_rows(K, dtype) || !valid_rows(V, dtype) || !cache_k || !cache_v || cache_k == cache_v) return SGA_ERR_INVALID_ARG;
  if (!aligned_to(cache_k, element_bytes(dtype)) || !aligned_to(cache_v, element_bytes(dtype))) return SGA_ERR_INVALID_ARG;
  if (Q && (!valid_rows(Q, dtype) || !valid_rows(Q_out, dtype) || !apart_or_same(*Q, *Q_out))) return SGA_ERR_INVALID_ARG;
  (void)hipGetLastError();
  RotateArgs a{};
  const int64_t head = (int64_t)batch->page_size * d;      // from head to head within a page
  int n = 0;
  if (Q) a.tensor[n++] = rows_arg(*Q, *Q_out, Hq, true);
  a.tensor[n] = rows_arg(*K, sga_rows{cache_k, head, 0}, Hkv, rotary != nullptr);
  a.tensor[n++].paged = 1;
  a.tensor[n] = rows_arg(*V, sga_rows{cache_v, head, 0}, Hkv, false);
  a.tensor[n++].paged = 1;
  a.n_tensors = n;
  a.n_rows = (int32_t)batch->n_tokens; a.d = d;
  a.rotary = rotary_args(rotary, 0);
  a.batch = batch_args(*batch);
  a.dtype = dtype;
  a.stream = static_cast<hipStream_t>(stream);
  return launch_rotate(a);
}

sga_status sga_paged_workspace_bytes(const sga_paged_batch* batch, const sga_mask_desc* mask, int32_t Hq, int32_t Hkv,
                                     int32_t d, int32_t dtype, size_t* bytes_out) {
  if (!bytes_out) return SGA_ERR_INVALID_ARG;
  PagedAttention a{};
  const sga_status st = paged_shape(batch, mask, 0, Hq, Hkv, d, dtype, a);
  if (st != SGA_OK) return st;
  size_t most = 0;
  for (a.causal = 0; a.causal < 2 && batch->n_tokens > 0 && batch->n_seqs > 0; ++a.causal) {
    const PagedPlan p = plan_paged(a);
    if (p.groups == 0) return SGA_ERR_OVERFLOW;
    most = p.bytes > most ? p.bytes : most;
  }
  *bytes_out = most;
  return SGA_OK;
}

sga_status sga_attention_paged(const sga_rows* Q, const void* cache_k, const void* cache_v, const sga_paged_batch* batch,
                               const sga_mask_desc* mask, int32_t causal, const sga_rows* O, int32_t Hq, int32_t Hkv,
                               int32_t d, float scale, int32_t dtype, float* lse, void* workspace, size_t workspace_bytes,
                               void* stream) {
  if (!Q || !O) return SGA_ERR_INVALID_ARG;
  PagedAttention a{};
  const sga_status st = paged_shape(batch, mask, causal, Hq, Hkv, d, dtype, a);
  if (st != SGA_OK) return st;
  if (workspace ? (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 : workspace_bytes != 0) return SGA_ERR_INVALID_ARG;
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return SGA_OK;
  if (!wide_rows(Q, dtype) || !wide_rows(O, dtype) || Q->data == O->data) return SGA_ERR_INVALID_ARG;
  if (!cache_k || !cache_v || !aligned16(cache_k) || !aligned16(cache_v)) return SGA_ERR_INVALID_ARG;
  if (batch->page_stride % (16 / element_bytes(dtype)) != 0 || !aligned_to(lse, 4)) return SGA_ERR_INVALID_ARG;
  const PagedPlan plan = plan_paged(a);
  if (plan.groups == 0) return SGA_ERR_OVERFLOW;
  (void)hipGetLastError();
  a.Q = Q->data; a.q_head = Q->head_stride; a.q_row = Q->row_stride;
  a.O = O->data; a.o_head = O->head_stride; a.o_row = O->row_stride;
  a.cache_k = cache_k; a.cache_v = cache_v;
  a.lse = lse;
  a.scale = scale;
  a.tile_rows = plan.tile_rows;
  a.page_pieces = (uint32_t)(batch->page_stride / (16 / element_bytes(dtype)));
  a.groups = plan.groups;
  a.splits = 1;
  a.slots = plan.slots;
  if (plan.bytes > 0 && workspace_bytes >= plan.bytes) {
    a.splits = plan.splits;
    a.notes = workspace;
    a.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + (size_t)plan.groups * kNoteBytes);
  }
  a.stream = static_cast<hipStream_t>(stream);
  return launch_paged(a);
}

}  // extern "C"

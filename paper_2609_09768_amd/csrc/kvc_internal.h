// Internal declarations shared by the C ABI (api.cpp) and the gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace kvc {

constexpr int kHeadDim = 128;      // D: the only supported head size
constexpr int kHalf = kHeadDim / 2;
// Work tile of the adjustment kernel: up to 1024 16-byte units (8 pairs of
// one head row), four per thread of a 256-thread workgroup, all loaded
// before the first is rotated: 16 rows of 8 kv heads, 128 rows of one.
constexpr int kShiftTileUnits = 1024;
// Requests of fewer than 16,384 reused rows get tiles of at most 16 rows,
// so that they still spread over the CUs (4.1k rows of one kv head: 256
// tiles instead of 32).
inline int shift_tile_rows(int64_t n_reused, int n_kv_heads) {
  const int rows = kShiftTileUnits / (8 * n_kv_heads);  // >= 2 for n_kv_heads <= 64
  return n_reused < 16384 && rows > 16 ? 16 : rows;
}
constexpr int kMaxHidden = 16384;  // widest row the RMS normalisation keeps in registers
// Grid cap of the grid-stride kernels (and of each batch of shift tiles):
// 2^20 workgroups of up to 512 threads
// stay far below HIP's 2^32 work-items per launch and fill the GPU many times.
constexpr int64_t kMaxGrid = int64_t(1) << 20;

// ---- plan (device buffer written by kvc_plan_upload) ----------------------
// [PlanHeader][double2 rot[n_chunks][64]][ShiftTile tiles[n_tiles]], each
// part 256-byte aligned; the offsets follow from n_chunks alone, so the host
// passes them to the kernel with n_tiles and only the header's hash and the
// tile itself are read before the data.
struct PlanHeader {
  uint64_t layout_hash;  // checked by the kernels: a stale plan adjusts nothing
  int32_t n_chunks;
  int32_t n_tiles;
  int64_t n_reused;
  int64_t rot_offset;    // bytes from plan start
  int64_t tile_offset;   // bytes from plan start
};
constexpr uint32_t kTileDeltaZero = 1;  // the chunk keeps its positions
constexpr uint32_t kTileZeroKv = 2;     // the chunk's cached K/V are all zero (separator slot)
struct ShiftTile {       // 16 bytes: one scalar load
  int32_t chunk;
  int32_t row_begin;
  int32_t row_end;
  uint32_t flags;        // kTileDeltaZero | kTileZeroKv
};
inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
inline size_t plan_rot_offset() { return align256(sizeof(PlanHeader)); }
inline size_t plan_tile_offset(int n_chunks) {
  return plan_rot_offset() + align256(sizeof(double) * 2 * kHalf * (size_t)n_chunks);
}

// ---- top-k workspace --------------------------------------------------------
struct TopkState {
  unsigned long long prefix;  // bits of the threshold key found so far
  unsigned long long mask;    // which bits of prefix are fixed
  long long rem;              // how many of the rows matching prefix are still to take
  unsigned int done;          // blocks finished in the current pass
  unsigned int pad;
  unsigned int hist[256];
};
constexpr int kTopkRowsPerBlock = 2048;  // 256 threads x 8 rows
inline int64_t topk_blocks(int64_t n) { return (n + kTopkRowsPerBlock - 1) / kTopkRowsPerBlock; }
// State of the fused selection (one launch for all steps, grid barriers),
// zero at its start: three rotating histograms, the barrier's arrival
// counter, the candidates' count and ranges of keys (largest key, largest
// complement): of all keys, and of those left after each histogram.
constexpr int kTopkMaxLevels = 8;  // histograms of 256 bins that 64-bit keys can take
struct TopkFused {
  unsigned int hist[3][256];
  unsigned int arrive;
  unsigned int cand;
  unsigned long long range[1 + kTopkMaxLevels][2];
  unsigned int pad[26];
};
static_assert(sizeof(TopkFused) == 3 * 1024 + 256, "part of the workspace size");
inline size_t topk_ws_bytes(int64_t n) {
  const size_t state = sizeof(TopkState) > sizeof(TopkFused) ? sizeof(TopkState) : sizeof(TopkFused);
  return align256(state) + align256(size_t(2) * sizeof(unsigned int) * size_t(topk_blocks(n) > 0 ? topk_blocks(n) : 1));
}

// ---- launchers (return hipGetLastError() of their launches) ---------------
// v_zero non-NULL (staging): tiles of zero_kv chunks get zeros in k_dst and
// v_zero instead of a rotation.
hipError_t launch_rope_shift(const void* plan, uint64_t layout_hash, int n_chunks, int n_tiles, int n_kv_heads,
                             const uint16_t* k_src, uint16_t* k_dst, uint16_t* v_zero,
                             hipStream_t s);
// clear, clear_bytes: memory zeroed by the same launch (16-byte units; the
// selection's state), or NULL, 0.
hipError_t launch_kv_deviation(int64_t n_rows, int n_kv_heads, const uint16_t* k_cached,
                               const uint16_t* k_fresh, double* dev, void* clear, size_t clear_bytes,
                               hipStream_t s);
// Adjustment and deviation in one launch, for the small requests it fits.
bool shift_deviation_fits(int64_t n_reused, int n_kv_heads);
hipError_t launch_shift_deviation(const void* plan, uint64_t layout_hash, int n_chunks, int n_tiles, int64_t n_reused,
                                  int n_kv_heads, const uint16_t* k_src, uint16_t* k_dst,
                                  const uint16_t* k_fresh, double* dev, hipStream_t s);
// Bytes at the start of the selection's workspace to be zero when it starts.
size_t topk_clear_bytes(int64_t n);
// cleared: they are; otherwise a launch of its own does it.  spin_limit: looks
// at the arrival counter before a wait of the selection's grid barriers is
// given up (the default takes seconds).
constexpr int kTopkSpinLimit = 1 << 22;
hipError_t launch_select_topk(const double* dev, int64_t n, int64_t k, int64_t n_append,
                              int32_t* idx_out, void* ws, bool cleared, hipStream_t s,
                              int spin_limit = kTopkSpinLimit);
hipError_t launch_scatter_rows(const int32_t* sel, int64_t n_sel, int compact,
                               const uint16_t* k_fresh, const uint16_t* v_fresh,
                               int64_t n_fresh, uint16_t* k_cache, uint16_t* v_cache,
                               int64_t n_rows, int n_kv_heads, hipStream_t s);
// Attention; with ws of at least attention_ws_bytes(...) bytes a selection
// too small to fill the GPU runs with its key range split over several
// workgroups (partials in ws, then a combine launch).
hipError_t launch_attention(const uint16_t* q, int64_t n_q_rows, const int32_t* q_rows,
                            const int32_t* q_pos, int64_t n_sel, const uint16_t* k,
                            const uint16_t* v, int64_t n_kv, int n_q_heads, int n_kv_heads,
                            float scale, uint16_t* out, float* lse, void* ws, size_t ws_bytes,
                            hipStream_t s);
// Bound on the work-items of the attention launch without a key-range split;
// a shape above 2^32 - 1 of them is refused.
int64_t attention_work_items(int64_t n_sel, int n_q_heads, int n_kv_heads);
// Decoder-layer steps around the attention (layer_ops.hip).
hipError_t launch_rms_norm(const uint16_t* x, int64_t n_x_rows, const int32_t* rows, int64_t n,
                           int hidden, const uint16_t* gamma, float eps, uint16_t* out,
                           uint16_t* res_out, hipStream_t s);
// norm: the RMS norms of the query and key heads before the rotation, or NULL.
struct HeadNorm {
  const uint16_t* gamma_q;
  const uint16_t* gamma_k;
  float eps;
};
hipError_t launch_qkv_rope(const uint16_t* y, int64_t n, int n_q, int n_k, int n_v,
                           const int32_t* pos, const double* freqs, uint16_t* q, uint16_t* k,
                           uint16_t* v, hipStream_t s, const HeadNorm* norm = nullptr);
hipError_t launch_swiglu(const uint16_t* gu, int64_t n, int64_t inter, uint16_t* out,
                         hipStream_t s);
size_t attention_ws_bytes(int64_t n_sel, int n_q_heads, int n_kv_heads);

// Projection GEMM of the selected rows (gemm.hip): c = a[rows] w^T (+ res).
hipError_t launch_gemm(int64_t m, int64_t n, int64_t k, const uint16_t* a, int64_t n_a_rows,
                       const int32_t* a_rows, const uint16_t* w, const uint16_t* res, uint16_t* c,
                       hipStream_t s);
// Work-items of a launch of 256 x 256 tiles alone, the choice that has to fit
// one launch for a shape to be accepted (HIP allows fewer than 2^32 of them).
int64_t gemm_work_items(int64_t m, int64_t n);

// ---- copies of the transfer stage (stage_copy.hip) -----------------------------
// Copies for one launch, all from host or all from device memory; 16-byte
// aligned, whole 16-byte units.  A kernel argument, so it stays below 4 KB.
struct CopyList {
  static constexpr int kMax = 160;
  const void* src[kMax];
  void* dst[kMax];
  uint32_t units[kMax];     // 16-byte units of each copy
  uint32_t end_tile[kMax];  // running count of the launch's tiles
  int n = 0;
};
// False when the list is full (or the copy is too large for it).
bool copy_list_add(CopyList* L, void* dst, const void* src, size_t bytes);
// host: the sources are in host memory.
hipError_t launch_copy_list(const CopyList& L, bool host, hipStream_t s);

// ---- pages of a cache pool (pages.hip) ------------------------------------------
// The tables of a kvc_pages, checked: page_rows is 2^page_shift.
struct PageTables {
  int32_t n_pages, page_shift, n_slots, max_pages;
  int32_t* ref;
  int32_t* table;
  int32_t* len;
};
// Scratch of fork, reserve and compact: a copy of the tables and lengths, or
// an entry and a count per page and slot.
inline size_t pages_ws_bytes(int64_t n_pages, int64_t n_slots, int64_t max_pages) {
  const size_t fork = size_t(n_slots) * size_t(max_pages + 1), lists = 2 * size_t(n_pages) + 2 * size_t(n_slots);
  return align256(4 * (fork > lists ? fork : lists) + 4);
}
hipError_t launch_pages_trim(const PageTables& P, const int32_t* keep, hipStream_t s);
hipError_t launch_pages_fork(const PageTables& P, const int32_t* src_of, int32_t* ws, hipStream_t s);
hipError_t launch_pages_reserve(const PageTables& P, const int32_t* n_new, int32_t max_new, int32_t* rows,
                                int32_t* copy_src, int32_t* copy_dst, int32_t* shortage, int32_t* ws, hipStream_t s);
hipError_t launch_pages_compact(const PageTables& P, int32_t* move_src, int32_t* move_dst, int32_t* counts,
                                int32_t* ws, hipStream_t s);
// page_bytes: a multiple of 2 KB; count: device, or NULL (all n_pairs).
hipError_t launch_pages_copy(int32_t n_pages, int64_t page_bytes, int n_layers, uint16_t* k, uint16_t* v,
                             const int32_t* src, const int32_t* dst, int64_t n_pairs, const int32_t* count,
                             hipStream_t s);

// ---- attention over a shared prefix and own pages (prefix_attention.hip) ----------
size_t prefix_attention_ws_bytes(int64_t n_prefix, int n_slots, int n_new, int n_q_heads, int n_kv_heads,
                                 int page_rows, int max_pages);
// Workgroups of its largest launch.
int64_t prefix_attention_workgroups(int64_t n_prefix, int n_slots, int n_new, int n_q_heads, int n_kv_heads,
                                    int page_rows, int max_pages);
hipError_t launch_prefix_attention(const uint16_t* q, int n_new, const uint16_t* kp, const uint16_t* vp,
                                   int64_t n_prefix, const PageTables& pages, const uint16_t* kt, const uint16_t* vt,
                                   int n_q_heads, int n_kv_heads, float scale, uint16_t* out, float* lse, void* ws,
                                   hipStream_t s);

// Its prefix for many rows (attention.hip): parts shares of the keys, results
// [part][kv head][row][D] and [part][kv head][row] (log2), where row r of kv
// head g is head g G + r % G of token r / G.
hipError_t launch_prefix_rows(const uint16_t* q, int64_t rows, int n_q_heads, int n_kv_heads, const uint16_t* k,
                              const uint16_t* v, int64_t n_kv, int parts, float scale, float* part_o, float* part_lse,
                              hipStream_t s);

// ---- packed sequences (attention.hip) -----------------------------------------------
// Sequences of up to kPackShort rows have workgroups of four units (32 queries
// of one head each), longer ones of eight: 40 sequences of 600 rows of 32/8
// heads take 209 us in blocks of four and 231 in blocks of eight, 24 of 1,000
// rows 285 and 275.
constexpr int kPackShort = 768;
constexpr int kPackShortUnits = 4;
constexpr int kPackUnits = 8;
// Work of one workgroup and kv head: a block of units of one sequence over key
// tiles tile0 .. tile0 + n_tiles - 1.  part: where its partial results go, -1
// if it has all of the keys (as in every short sequence).
struct PackItem {
  int32_t row0, len;     // the sequence's first row and its rows
  int32_t block;         // its units are 8 (4) block and those after it
  int32_t tile0, n_tiles;
  int32_t part;
  uint64_t id;           // the plan's, so that one load brings both
};
static_assert(sizeof(PackItem) == 32, "one 32-byte scalar load");
// A block whose keys were cut: parts first .. first + n_parts - 1.
struct PackJoin {
  int32_t row0, len, block, first, n_parts;
  int32_t pad[3];
};
struct PackHeader {
  uint64_t id;
  int32_t n_items, n_short, n_joins, n_parts;  // items of long sequences first
};
// The short sequences' items lie in the order of the queues that work on them,
// each a workgroup for every kv head, two workgroups a CU.
inline int64_t pack_queues(int64_t n_short, int n_kv_heads) {
  const int64_t most = 512 / n_kv_heads;  // >= 8
  return n_short < most ? n_short : most;
}
inline size_t pack_items_offset() { return align256(sizeof(PackHeader)); }
inline size_t pack_joins_offset(int64_t n_items) {
  return pack_items_offset() + align256(sizeof(PackItem) * size_t(n_items));
}
// First item of each queue, and the end of the last one's.
inline size_t pack_queues_offset(int64_t n_items, int64_t n_joins) {
  return pack_joins_offset(n_items) + align256(sizeof(PackJoin) * size_t(n_joins));
}
// Partials of a part: 8 units of 32 queries, D sums and a log-sum each.
inline size_t pack_ws_bytes(int64_t n_parts, int n_kv_heads) {
  return align256(size_t(n_parts) * size_t(n_kv_heads) * 8 * 32 * (kHeadDim + 1) * sizeof(float));
}
hipError_t launch_packed_attention(const void* plan, uint64_t id, int n_items, int n_short, int n_joins, int n_parts,
                                   const uint16_t* q, const uint16_t* k, const uint16_t* v, int n_q_heads,
                                   int n_kv_heads, float scale, uint16_t* out, float* lse, void* ws, hipStream_t s);

// ---- static scratch (static_scratch.hip) -------------------------------------
// Size of the per-GPU device array behind kvc_blend_prefill_layer_noalloc
// (KVC_STATIC_SCRATCH_BYTES in kvc.h).
constexpr size_t kStaticScratchBytes = size_t(16) << 20;
// Device address of that array on the current device (looked up once per
// device with hipGetSymbolAddress, then cached).
hipError_t static_scratch(void** ptr);

}  // namespace kvc

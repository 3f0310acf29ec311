// Attention of a batch over one shared prefix and over rows of their own
// (gfx950).
//
// Sequence s has n_new query tokens at the end of its own rows 0 .. len - 1,
// which lie in pages of a pool and follow a prefix that all sequences share
// (the blended context).  Query i sees the whole prefix and its own rows 0 ..
// t = len - n_new + i:
//   O = softmax_j(scale * <q, k_j>) v_j  over prefix and own rows together.
// A softmax over a union is the weighted mean of the softmaxes over its
// parts, with weights e^(lse of the part), so the key axis is cut into parts
// that are computed apart and joined by a last kernel in a fixed order:
// the prefix into shares of its key tiles, each read once for ALL rows
// (sequence, token, query head of the group) of a kv head, and every
// sequence's own rows into chunks.
//
// Up to 64 rows of a kv head are bound by the bytes of K and V: 512 per key
// and kv head against 4 x 128 FLOP per row.  So the kernel here is built
// around loads in flight.  A workgroup has four waves, and two fit a CU, so that
// one's first loads and joins lie beside the other's tiles; each wave takes
// every fourth 32-key tile of the part by itself, with a K slot and a V
// slot of its own in LDS that loads fill without registers: the next K tile is
// asked for when the scores are done, the next V tile when the product is, so
// 64 to 128 KB per CU are under way, and no barrier is met until the waves join
// their results.  The matrix work of a tile (v_mfma_f32_32x32x16_bf16: S^T = K
// Q^T, O^T += V^T P^T, a lane holds one row and 16 of the keys) takes 512
// cycles, against about 1,500 for a CU's share of HBM to bring its 16 KB.
// 64 rows of a kv head over 32,256 keys of 8 heads and 300 own rows (149.6 MB)
// take 45 us with the join, 3.3 TB/s: a share of the prefix is four tiles a wave
// there, and its first loads and its results count beside them.
// More rows go to the kernel of the other attentions (attention.hip), whose
// eight waves of 32 rows share every tile.
// Scores, softmax and sums are float32; weights are rounded to bf16 for the
// product with V, whose operand they are: each is off by 2^-8 of itself at most,
// and the output is rounded to as many bits.  A part's output is divided by the
// sum of its rounded weights, which makes it a weighted mean of V (over the
// unrounded sum a row that one key dominates is off by that key's rounding, up
// to 0.38 %); the log-sum, the part's weight in the join, takes the sum of the
// unrounded ones and is exact to float32.
#include <algorithm>

#include "bf16_util.h"
#include "kvc_internal.h"

namespace kvc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) v4s lds_v4s;
typedef __attribute__((address_space(1))) const void global_void;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
static_assert(kWaves == 4, "the join gives each wave a quarter of 32 channels");
constexpr int kTile = 32;                       // keys of a tile
constexpr int kKGroup = 4 * kHeadDim + 32;      // bf16 per four K rows in LDS (1088 B, spreads the banks)
constexpr int kKSlot = (kTile / 4) * kKGroup;   // of one wave
constexpr int kVSlot = kTile * kHeadDim;
constexpr int kMaxIds = 64;                     // pages of a chunk: one a lane
// s_waitcnt immediates (vmcnt bits 3:0 and 15:14, expcnt 6:4, lgkmcnt 11:8) as
// the builtin takes them, which the compiler's own wait counting understands:
// at most n vector loads under way; LDS reads done.
constexpr int wait_vm(int n) { return (n & 15) | (n >> 4) << 14 | 7 << 4 | 15 << 8; }
constexpr int kWaitLds = 15 | 3 << 14 | 7 << 4;

// What rows that are not there are loaded as.
__device__ const uint4 zero_row[16] = {};

struct PrefixParams {
  const uint16_t* q;
  int n_new, n_slots, n_q_heads, n_kv_heads, group;
  int rows;        // of a kv head: n_slots x n_new x group
  int slot_rows;   // of a slot: n_new x group
  const uint16_t* kp;
  const uint16_t* vp;
  int n_prefix;
  const uint16_t* kt;
  const uint16_t* vt;
  PageTables pages;
  float scale_log2;
  int prefix_parts, prefix_blocks;  // shares of the prefix, blocks of rows
  int prefix_wgs;                   // workgroups of a kv head for them here (none: the wide kernel has them)
  int own_parts, own_blocks, chunk; // chunks of a slot's rows (chunk rows each), blocks of rows
  float* part_o;    // [part][kv head][row][D], parts of the prefix first
  float* part_lse;  // [part][kv head][row], log2
  uint16_t* out;
  float* lse;
};

__device__ __forceinline__ bf16x8 as_bf16x8(const uint4& u) { return __builtin_bit_cast(bf16x8, u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Memory operations stay on their side of this: the counts of loads under way
// that the kernel waits for go by the order it asks for them.
__device__ __forceinline__ void in_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

__global__ __launch_bounds__(kThreads, 2) void prefix_attn_kernel(const PrefixParams P) {
  // a part of each for every wave
  __shared__ __attribute__((aligned(16))) uint16_t Ks[kWaves * kKSlot];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[kWaves * kVSlot];
  __shared__ float wm[kWaves][32], wl[kWaves][32], wu[kWaves][32];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ql = lane & 31, half = lane >> 5;

  // this workgroup's part of the keys and block of rows
  const unsigned hkv = (unsigned)P.n_kv_heads;
  const int g = (int)(blockIdx.x % hkv);
  unsigned rest = blockIdx.x / hkv;
  const unsigned n_prefix_wgs = (unsigned)P.prefix_wgs;
  const bool own = rest >= n_prefix_wgs;
  int part, row0, row_end, key0, key_end, slot = 0, have = 0;
  int page_id = -1;  // own: lane i has the number of the chunk's page i, -1 where the table names none of the pool
  if (!own) {
    const int rb = (int)(rest % (unsigned)P.prefix_blocks);
    part = (int)(rest / (unsigned)P.prefix_blocks);
    row0 = rb * 32;
    row_end = P.rows;
    const long long tiles = ((long long)P.n_prefix + kTile - 1) / kTile;
    key0 = (int)(tiles * part / P.prefix_parts) * kTile;
    key_end = min((int)std::min<long long>(tiles * (part + 1) / P.prefix_parts * kTile, P.n_prefix), P.n_prefix);
  } else {
    rest -= n_prefix_wgs;
    const int rb = (int)(rest % (unsigned)P.own_blocks);
    rest /= (unsigned)P.own_blocks;
    slot = (int)(rest % (unsigned)P.n_slots);
    const int c = (int)(rest / (unsigned)P.n_slots);
    have = min(max(P.pages.len[slot], 0), P.pages.max_pages << P.pages.page_shift);
    key0 = c * P.chunk;
    if (key0 >= have) return;  // every wave: nothing of this chunk is there, and the join knows it
    key_end = (int)std::min<long long>((long long)key0 + P.chunk, have);
    part = P.prefix_parts + c;
    row0 = slot * P.slot_rows + rb * 32;
    row_end = (slot + 1) * P.slot_rows;
    const int first = key0 >> P.pages.page_shift;  // chunks start with a page
    if (lane <= ((key_end - 1) >> P.pages.page_shift) - first) {
      const int p = P.pages.table[(size_t)slot * P.pages.max_pages + first + lane];
      page_id = p >= 0 && p < P.pages.n_pages ? p : -1;
    }
  }
  // the page of a key of this chunk (the same key in every lane)
  auto page_of = [&](int key) __attribute__((always_inline)) {
    return __builtin_amdgcn_readlane(page_id, (key - key0) >> P.pages.page_shift);
  };

  // query of the row, and how many keys of the tensor the row sees
  bf16x8 qreg[8];
  const int row = row0 + ql;
  const bool in = row < row_end;
  int sees = 0;
  {
    const int tok = row / P.group;
    const uint16_t* qp =
        P.q + ((long long)tok * P.n_q_heads + g * P.group + (row - tok * P.group)) * kHeadDim + half * 8;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
      qreg[ks] = as_bf16x8(in ? *reinterpret_cast<const uint4*>(qp + ks * 16) : make_uint4(0, 0, 0, 0));
    sees = own ? max(have - P.n_new + (tok - slot * P.n_new) + 1, 0) : P.n_prefix;
  }
  in_order();
  // the block's first row sees the fewest keys: it has the earliest token
  const int sees_least = own ? max(have - P.n_new + (row0 / P.group - slot * P.n_new) + 1, 0) : P.n_prefix;

  // A tile: eight loads of four rows of K, then eight of V; lane l of a load
  // fills 16 bytes at the wave's LDS address + 16 l.  LDS pieces are swizzled
  // for the operand reads: K row r's piece p at p ^ (r & 3), V's at
  // p ^ 4 (r & 3).
  const long long row_bytes = (long long)P.n_kv_heads * kHeadDim * 2;
  const int lr = lane >> 4, lp = lane & 15;
  const int k_piece = 16 * (lp ^ lr), v_piece = 16 * (lp ^ (4 * lr));
  const char* zero = reinterpret_cast<const char*>(zero_row);
  const char* const kb = reinterpret_cast<const char*>(own ? P.kt : P.kp) + g * (kHeadDim * 2) + k_piece;
  const char* const vb = reinterpret_cast<const char*>(own ? P.vt : P.vp) + g * (kHeadDim * 2) + v_piece;
  uint16_t* const ks_ = Ks + wave * kKSlot;
  uint16_t* const vs_ = Vs + wave * kVSlot;
  // Loads of a K or V tile (base: kb or vb; row r goes to to + r's place).  A
  // row that is not there is loaded as zeros.
  auto issue = [&](int k0, const char* base, int piece, uint16_t* to, int stride) __attribute__((always_inline)) {
    const char* from[8];
    if (!own && k0 + kTile <= key_end) {
      from[0] = base + (long long)(k0 + lr) * row_bytes;
#pragma unroll
      for (int j = 1; j < 8; ++j) from[j] = from[j - 1] + 4 * row_bytes;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = k0 + 4 * j + lr;
        long long r = key;
        int id = 0;
        if (own) {
          id = page_of(min(k0 + 4 * j, key_end - 1));  // four rows share a page
          r = ((long long)id << P.pages.page_shift) + (key & ((1 << P.pages.page_shift) - 1));
        }
        from[j] = id < 0 || key >= key_end ? zero + piece : base + r * row_bytes;
      }
    }
    // (one place for the loads: the compiler's wait counting goes by it)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      __builtin_amdgcn_global_load_lds((global_void*)from[j], (lds_void*)(to + j * stride), 16, 0, 0);
    in_order();
  };
  auto issue_k = [&](int k0) __attribute__((always_inline)) { issue(k0, kb, k_piece, ks_, kKGroup); };
  auto issue_v = [&](int k0) __attribute__((always_inline)) { issue(k0, vb, v_piece, vs_, 4 * kHeadDim); };

  // Whether any of the pages is outside the pool: its keys are masked like
  // keys past the end.
  const bool gaps = own && __any(page_id < 0 && lane <= ((key_end - 1 - key0) >> P.pages.page_shift));

  // operand reads: A = K rows lane % 32, dims 16 ks + 8 half .. + 8; and
  // A = V^T, dims 32 dt + lane % 32, keys in the order in which the S^T
  // accumulator holds them (8 (e / 4) + 4 half + e % 4), by transposing reads
  const int k_a0 = (ql >> 2) * kKGroup + (lane & 3) * kHeadDim + 8 * (half ^ (lane & 1));
  const int k_e1 = 16 * ((lane >> 1) & 1);
  const int k_rd[2] = {k_a0 + k_e1, k_a0 - k_e1};
  int v_rd[4];
  {
    const int i = lane & 15, gd = (lane >> 4) & 1, sr = i >> 2;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
      v_rd[dt] = (4 * half + sr) * kHeadDim + 32 * (dt ^ sr) + 16 * gd + 4 * (i & 3);
  }

  f32x16 o[4];
  float m_run = -INFINITY, l_run = 0.f, u_run = 0.f;  // sums of the weights as rounded to bf16, and before that
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;

  // Tile i of this wave starts at key0 + 32 (4 i + wave).  Loads return in
  // order, K and V by turns, so whichever is needed next is there when at most
  // eight are left.  A tile past the last is loaded too, as zeros (no memory
  // traffic), so that these counts hold to the end.
  const int n_all = (key_end - key0 + kTile - 1) / kTile;
  const int n = n_all > wave ? (n_all - wave + kWaves - 1) / kWaves : 0;
  auto start = [&](int i) __attribute__((always_inline)) { return i < n ? key0 + kTile * (kWaves * i + wave) : key_end; };
  if (n > 0) {
    issue_k(start(0));  // behind the queries' loads, which are done when the first K tile is

    issue_v(start(0));
    for (int i = 0; i < n; ++i) {
      const int k0 = start(i);
      __builtin_amdgcn_s_waitcnt(wait_vm(8));  // K
      in_order();
      f32x16 s = {};
#pragma unroll
      for (int ks = 0; ks < 8; ++ks)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            as_bf16x8(*reinterpret_cast<const uint4*>(ks_ + k_rd[ks & 1] + 16 * ks)), qreg[ks], s, 0, 0, 0);
      in_order();
      __builtin_amdgcn_s_waitcnt(kWaitLds);  // the slot has been read
      issue_k(start(i + 1));
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= P.scale_log2;
      if (k0 + kTile > sees_least || k0 + kTile > key_end || gaps) {
        // first key that is not seen, for each eight keys (which share a page)
        const int limit = min(sees, key_end);
        int lim[4] = {limit, limit, limit, limit};
        if (gaps) {
#pragma unroll
          for (int j = 0; j < 4; ++j) lim[j] = page_of(min(k0 + 8 * j, key_end - 1)) < 0 ? key0 : limit;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[r] = k0 + (r >> 2) * 8 + half * 4 + (r & 3) >= lim[r >> 2] ? -INFINITY : s[r];
      }
      float mx = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      // The offset of a row's exponents follows the maximum only when that has
      // left it by 2^8: weights up to 2^8 lose nothing, and O is seldom scaled.
      const float mx2 = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
      const float m_new = mx2 > m_run + 8.f ? mx2 : m_run;
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      if (__any(m_new != m_run)) {
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
        l_run *= alpha;
        u_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
      }
      m_run = m_new;
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(s[2 * e] - m_use), p1 = __builtin_amdgcn_exp2f(s[2 * e + 1] - m_use);
        u_run += p0 + p1;
        w[e] = pack_bf16x2(p0, p1);
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[e]), ones, l_run, false);
      }
      const bf16x8 pb[2] = {as_bf16x8(make_uint4(w[0], w[1], w[2], w[3])), as_bf16x8(make_uint4(w[4], w[5], w[6], w[7]))};
      __builtin_amdgcn_s_waitcnt(wait_vm(8));  // V
      in_order();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int kk = j >> 2, dt = j & 3;
        const uint16_t* b = vs_ + v_rd[dt] + kk * 16 * kHeadDim;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(b));
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(b + 8 * kHeadDim));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(make_uint4(l2.x, l2.y, h2.x, h2.y)), pb[kk], o[dt], 0, 0, 0);
      }
      in_order();
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      issue_v(start(i + 1));
    }
    __builtin_amdgcn_s_waitcnt(wait_vm(0));
  }

  // join the waves, 32 channels at a time (16 KB of LDS), in wave order
  float4* const red = reinterpret_cast<float4*>(Ks);
  static_assert(sizeof(Ks) >= kWaves * 4 * 64 * sizeof(float4), "the waves' sums of a quarter of the channels");
  const float l_tot = l_run + __shfl_xor(l_run, 32), u_tot = u_run + __shfl_xor(u_run, 32);
  if (half == 0) {
    wm[wave][ql] = m_run;
    wl[wave][ql] = l_tot;
    wu[wave][ql] = u_tot;
  }
  __syncthreads();  // all waves are done with their slots
  float m = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, wm[w][ql]);
  float l = 0.f, u = 0.f, f[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    f[w] = wm[w][ql] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(wm[w][ql] - m);
    l = fmaf(f[w], wl[w][ql], l);
    u = fmaf(f[w], wu[w][ql], u);
  }
  // (a row that sees no key of the part has the sum 0; one with a NaN among its
  // scores has the sum NaN, whatever its maximum, and keeps it)
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const long long at = ((long long)part * P.n_kv_heads + g) * P.rows + row;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) {
    if (dt) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
      red[(wave * 4 + e) * 64 + lane] = make_float4(o[dt][4 * e], o[dt][4 * e + 1], o[dt][4 * e + 2], o[dt][4 * e + 3]);
    __syncthreads();
    {  // piece `wave` of the four
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float4 x = red[(w * 4 + wave) * 64 + lane];
        a.x = fmaf(f[w], x.x, a.x);
        a.y = fmaf(f[w], x.y, a.y);
        a.z = fmaf(f[w], x.z, a.z);
        a.w = fmaf(f[w], x.w, a.w);
      }
      if (in)
        *reinterpret_cast<float4*>(P.part_o + at * kHeadDim + 32 * dt + 8 * wave + 4 * half) =
            make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
    }
  }
  if (wave == 0 && half == 0 && in) P.part_lse[at] = u == 0.f ? -INFINITY : m + log2f(u);
}

// Joins the parts of a row and head with the weights 2^(lse - max), one
// workgroup each: a lane has the weight of one of 64 parts, each wave adds
// every fourth part (two channels a lane, up to eight parts' loads under way),
// and the waves' sums are added in order.  Bound by the parts' 516 bytes a row,
// and by two rounds of loads.
constexpr int kJoinWaves = 4;
__global__ __launch_bounds__(64 * kJoinWaves) void prefix_join_kernel(const PrefixParams P) {
  __shared__ float2 sums[kJoinWaves][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = (int)(blockIdx.x / (unsigned)P.rows), r = (int)(blockIdx.x - (unsigned)g * (unsigned)P.rows);
  const int tok = r / P.group, h = g * P.group + (r - tok * P.group), slot = tok / P.n_new;
  const int have = min(max(P.pages.len[slot], 0), P.pages.max_pages << P.pages.page_shift);
  const int t = have - P.n_new + (tok - slot * P.n_new);  // its place among the slot's rows
  const int own = t < 0 ? 0 : (int)(((long long)have + P.chunk - 1) / P.chunk);
  const int parts = t < 0 ? 0 : P.prefix_parts + own;
  const long long stride = (long long)P.n_kv_heads * P.rows;
  const float* lp = P.part_lse + (long long)g * P.rows + r;
  const float* op = P.part_o + ((long long)g * P.rows + r) * kHeadDim + 2 * lane;
  float l_first = lane < parts ? lp[lane * stride] : -INFINITY;
  float m = l_first;
  bool nan = l_first != l_first;  // fmaxf passes over NaN: a row of nothing else is not one without keys
  for (int p = lane + 64; p < parts; p += 64) {
    const float l = lp[p * stride];
    m = fmaxf(m, l);
    nan |= l != l;
  }
  nan = __any(nan);
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
  float a = 0.f, b = 0.f, sum = 0.f;
  for (int p0 = 0; p0 < parts && (m != -INFINITY || nan); p0 += 64) {
    const float l = p0 == 0 ? l_first : p0 + lane < parts ? lp[(p0 + lane) * stride] : -INFINITY;
    const float w = __builtin_amdgcn_exp2f(l - m);  // 0 for a part without keys, NaN for one of NaN
    sum += w;
    const int n = min(parts - p0, 64);
    const float* q = op + (long long)p0 * stride * kHeadDim;
#pragma unroll 1
    for (int p = wave; p < n; p += 8 * kJoinWaves) {
      float2 x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[e] = p + e * kJoinWaves < n ? *reinterpret_cast<const float2*>(q + (p + e * kJoinWaves) * stride * kHeadDim)
                                      : make_float2(0.f, 0.f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float we = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), min(p + e * kJoinWaves, 63)));
        a = fmaf(we, x[e].x, a);
        b = fmaf(we, x[e].y, b);
      }
    }
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
  sums[wave][lane] = make_float2(a, b);
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 1; w < kJoinWaves; ++w) {
    a += sums[w][lane].x;
    b += sums[w][lane].y;
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  const long long at = (long long)tok * P.n_q_heads + h;
  *reinterpret_cast<uint32_t*>(P.out + at * kHeadDim + 2 * lane) = pack_bf16x2(a * inv, b * inv);
  if (P.lse && lane == 0) P.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.69314718055994531f;
}

long long div_up(long long a, long long b) { return (a + b - 1) / b; }

constexpr int kCus = 256;
constexpr int kPerCu = 2;  // workgroups of the kernel here that a CU holds (67 KB of LDS each)

// How a call is cut.  Up to 64 rows of a kv head take the kernel here (a
// second block of 32 finds the tiles in L2: 64 rows over 32,256 keys of 8
// heads 47 us, 50 with the wide kernel, of whose eight waves two have work),
// more the wide one, 256 rows a workgroup.  The prefix in as many shares as
// fill the CUs with workgroups, of at least a tile for each wave here, of four
// 64-key tiles there.  A slot's rows in chunks of 256 (two tiles a wave), 512
// where slots and heads alone give every CU a workgroup (16 slots of 8 heads
// and 300 rows 47 us, 50 with 512; 64 slots 170 us, 168 with 512), larger where
// its table holds more than 32 of them, but of no more than 64 pages.
struct Cut {
  bool wide;
  int prefix_parts, prefix_blocks, own_parts, own_blocks, chunk;
};
Cut cut(int64_t n_prefix, int n_slots, int64_t rows, int64_t slot_rows, int n_kv_heads, int page_rows, int max_pages) {
  Cut c;
  c.wide = rows > 64;
  c.prefix_blocks = (int)div_up(rows, c.wide ? 256 : 32);
  const long long most_parts = div_up(n_prefix, c.wide ? 4 * 64 : kTile * kWaves);
  c.prefix_parts = n_prefix == 0 || rows == 0
                       ? 0
                       : (int)std::max<long long>(1, std::min(div_up(c.wide ? kCus : kCus * kPerCu, (long long)n_kv_heads * c.prefix_blocks), most_parts));
  const long long most = (long long)max_pages * page_rows;
  const long long least = (long long)n_slots * n_kv_heads > kCus ? 512 : 256;
  c.chunk = (int)std::min<long long>(std::max<long long>(least, div_up(most, 32 * 128) * 128), (long long)kMaxIds * page_rows);
  c.chunk = std::max(c.chunk / page_rows, 1) * page_rows;  // whole pages
  c.own_parts = (int)div_up(most, c.chunk);
  c.own_blocks = (int)div_up(slot_rows, 32);
  return c;
}

}  // namespace

size_t prefix_attention_ws_bytes(int64_t n_prefix, int n_slots, int n_new, int n_q_heads, int n_kv_heads,
                                 int page_rows, int max_pages) {
  const int64_t slot_rows = (int64_t)n_new * (n_q_heads / n_kv_heads), rows = slot_rows * n_slots;
  const Cut c = cut(n_prefix, n_slots, rows, slot_rows, n_kv_heads, page_rows, max_pages);
  return align256(size_t(c.prefix_parts + c.own_parts) * size_t(n_kv_heads) * size_t(rows) * (kHeadDim + 1) * sizeof(float));
}

int64_t prefix_attention_workgroups(int64_t n_prefix, int n_slots, int n_new, int n_q_heads, int n_kv_heads,
                                    int page_rows, int max_pages) {
  const int64_t slot_rows = (int64_t)n_new * (n_q_heads / n_kv_heads), rows = slot_rows * n_slots;
  const Cut c = cut(n_prefix, n_slots, rows, slot_rows, n_kv_heads, page_rows, max_pages);
  return ((int64_t)c.prefix_parts * c.prefix_blocks + (int64_t)c.own_parts * c.own_blocks * n_slots) * n_kv_heads;
}

hipError_t launch_prefix_attention(const uint16_t* q, int n_new, const uint16_t* kp, const uint16_t* vp,
                                   int64_t n_prefix, const PageTables& pages, const uint16_t* kt, const uint16_t* vt,
                                   int n_q_heads, int n_kv_heads, float scale, uint16_t* out, float* lse, void* ws,
                                   hipStream_t s) {
  PrefixParams P;
  P.q = q;
  P.n_new = n_new;
  P.n_slots = pages.n_slots;
  P.n_q_heads = n_q_heads;
  P.n_kv_heads = n_kv_heads;
  P.group = n_q_heads / n_kv_heads;
  P.slot_rows = n_new * P.group;
  P.rows = P.slot_rows * P.n_slots;
  P.kp = kp;
  P.vp = vp;
  P.n_prefix = (int)n_prefix;
  P.kt = kt;
  P.vt = vt;
  P.pages = pages;
  P.scale_log2 = scale * 1.4426950408889634f;
  const Cut c = cut(n_prefix, P.n_slots, P.rows, P.slot_rows, n_kv_heads, 1 << pages.page_shift, pages.max_pages);
  P.prefix_parts = c.prefix_parts;
  P.prefix_blocks = c.prefix_blocks;
  P.own_parts = c.own_parts;
  P.own_blocks = c.own_blocks;
  P.chunk = c.chunk;
  P.part_o = static_cast<float*>(ws);
  P.part_lse = P.part_o + (size_t)(c.prefix_parts + c.own_parts) * n_kv_heads * P.rows * kHeadDim;
  P.out = out;
  P.lse = lse;
  if (c.wide && c.prefix_parts > 0) {
    const hipError_t e = launch_prefix_rows(q, P.rows, n_q_heads, n_kv_heads, kp, vp, n_prefix, c.prefix_parts, scale,
                                            P.part_o, P.part_lse, s);
    if (e != hipSuccess) return e;
  }
  P.prefix_wgs = c.wide ? 0 : c.prefix_parts * c.prefix_blocks;
  const long long wgs = (P.prefix_wgs + (long long)c.own_parts * c.own_blocks * P.n_slots) * n_kv_heads;
  if (wgs > 0) {
    hipLaunchKernelGGL(prefix_attn_kernel, dim3((unsigned)wgs), dim3(kThreads), 0, s, P);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(prefix_join_kernel, dim3((unsigned)P.rows * (unsigned)n_kv_heads), dim3(64 * kJoinWaves), 0, s, P);
  return hipGetLastError();
}

}  // namespace kvc

// cwl_head_loss: softmax cross entropy of a head's projection over a large vocabulary, with its gradients, logits not kept.
//
//   z = X W,   lse_t = ln sum_v e^(z_tv),   loss_t = w_t (lse_t - z_t,y),   dX = dZ W^T,   dW = X^T dZ,
//   dZ = up (softmax(z) - onehot(y))
//
// Rows without a target or of weight 0 cost nothing: the first kernel lists the others and packs their activations
// together (or, where every row counts, leaves X as it is), and all products run over the packed rows.  These are
// tensor-core products of one persistent kernel, which differ in the way their operands lie and in what becomes of a tile:
//   STATS  z tile -> (max, sum of exponentials) of its columns per row without the target's, and the target's logit
//   EXP    z tile of a piece of the vocabulary -> E = e^(z - r_t) in bf16, to a workspace, with the same statistics
//   DZ     z tile of a piece again, once lse is known -> dZ in bf16, to a workspace (where dW is wanted)
//   DX     piece of E or dZ times W^T; the sums over the pieces are kept in fp32
//   DW     X^T times piece of dZ: whole columns of dW
// (Up to 64 rows, 128 for the loss alone, STATS and EXP are head_few_kernel's.)
//
// Loss and dX in one call take two products, not three: dX = up (sum_(v != y) E_tv W_v - W_y sum_(v != y) E_tv) / sum_v E_tv needs
// the row's sums at the end only.  bf16 has the exponents of fp32, so that any logit of the row will do as the reference r_t as long as no other
// but the target's, which joins at the end, lies 60 above it: the target's, or (many rows) that of column 0.  Where one does, its 64 columns take a reference of their own,
// and head_merge_kernel puts the row's piece on a common one before DX reads it.  The target's column W_y is gathered from W
// and subtracted in fp32, so that it is not among what is rounded to bf16: a token of which the model knows little has
// dX near -up W_y, and where the model is sure of it E_y W_y and W_y would cancel.  Where dW is wanted, the target is an entry
// of dZ like the others, rounded like them, but not as e^(z_y - lse) - 1, of which little would be left where the model is sure:
// -up (1 - q_y) is what the others add up to (head_finish_kernel), or up expm1(z_y - lse) where lse is given.
//
// Roundings to fewer bits: E and dZ to bf16 (2^-9 of a number on the average row: dX's own rounding to bf16 is as large).
// For fp32 gradients they are kept as the sum of two bf16 numbers (2^-17), of up to kThreeTermRows rows, where one number's error
// shows in a whole column of dW, of three (2^-25), each multiplied on its own; and the tensor cores' sums, which are
// truncated at every step of 16 (2.4e-6 of a sum of 256 steps, measured on the logits of d = 4096), are added up in fp32 after
// every kChunkBlocks K blocks, over the terms.  dZ is relative to the first row's up: rows of one weight are then not rounded twice.
//
// bf16 rows that outgrow their reference are rounded a second time when head_merge_kernel puts them on the new one (2^-9 again).
//
// What bounds it (one B200): the tensor cores, under the power cap once a call lasts.  16384 rows, 4096 -> 32000, loss and dX: 6.9 to
// 7.3 ms, of which the two products take 3.0 + 3.1 (1.39 PFLOP/s where a library's product keeps up 1.41, 1.68 in bursts), the gather
// 0.15, listing rows and references 0.05, the merges 0.04; 1536 of 2048 rows: 0.70 to 0.81 ms, 0.30 + 0.33 + 0.053 + 0.017.  Tensor
// pipe active 79 % in EXP and 84 % in DX.  Tiles of 256 x 512 a pair of CTAs, because with 256 x 256 operands reach shared
// memory no faster than they are used; what the epilogue of a tile leaves uncovered is 2 % of it at d = 4096 and 15 % at d = 1024
// (4000 rows of 131072: 0.89 to 0.94 ms, 1.2 PFLOP/s; pipe 66 %): it hands the first 256 columns back before the others, and the
// next tile's products of as many K blocks as the ring holds start there.  fp32 gradients: two products for one, 2.7 ms for 2047
// rows, 2048 -> 50021, dX and dW.
#include "cluster.cuh"
#include "cwl_common.cuh"
#include "pair_mma.cuh"

namespace cwl {
namespace {

constexpr int kHM = 128;                          // rows per CTA tile = TMEM lanes
constexpr int kHK = 64;                           // K elements per stage = one 128-byte swizzle row of bf16
constexpr int kHMaxStages = 8;
constexpr int kHBox = 64 * kHK * 2;               // a box of 64 columns (or rows) x 64 K elements: 8 KB
constexpr int kHLeft = kHM * kHK * 2;             // 16 KB of the left operand a stage
constexpr int kHMaxTile = 512;                    // columns of a pair's tile = fp32 columns of tensor memory
constexpr int kHRing = 192 * 1024;                // 4 stages of 48 KB (tiles of 512 columns) to 8 of 24 KB (of up to 128)
constexpr int kHOutBuf = 4096;                    // staging of a warp: 32 rows of 128 bytes
constexpr int kHEpiWarps = 8;
constexpr int kHThreads = 64 + 32 * kHEpiWarps;   // warp 0: TMA, warp 1: MMA and tensor memory, warps 2..9: epilogue
constexpr int kHBars = 8 * (2 * kHMaxStages + 4);
constexpr size_t kHSmem = 1024 + kHRing + kHEpiWarps * kHOutBuf + kHBars + 32;
constexpr int kHPairs = 74;                       // CTA pairs that schedules are made for (a B200 holds 74)
constexpr int kHRaster = 16;                      // row tiles whose columns are walked together, so that they share W in L2
constexpr int kHeadMaxRows = 1 << 24, kHeadMaxWidth = 1 << 20;   // T and V, d
constexpr int kChunkBlocks = 64;                  // K blocks, times terms, after which the sums of an fp32 gradient leave the tensor memory
constexpr int kThreeTermRows = 512;
// Logits of up to kExactRows rows, of more than kExactWidth activations, or behind fp32 gradients, are added up in fp32 after every
// kLogitChunk K blocks: the truncation of the tensor cores' own sums would show in the loss of a single token that the model is
// sure of (1.6e-5 of one of 0.9, d = 4096), would grow with d, and would be most of what fp32 gradients lose (d = 8192, lse given: 4e-5
// without, 7e-6 with).  It takes tiles of 256 columns, whose operands come in no faster than they are worked on; with one row tile,
// where W's rate in HBM is the bound, that costs nothing.  Elsewhere it costs 7 to 8 % of a call (16384 rows 7.1 -> 7.7 ms, 4096
// rows backward 1.74 -> 1.89; 24 K blocks 5 %, 8 K blocks 17 %) and would bring lse from 2.4e-6 to 6e-7: not worth it beside bf16 gradients.
constexpr int kExactRows = 256, kExactWidth = 8192, kLogitChunk = 16;
constexpr float kAbove = 60.f;                    // a logit this far above the reference takes another one
constexpr float kLog2e = 1.4426950408889634f;

enum : int { HEAD_STATS = 0, HEAD_DZ = 1, HEAD_DX = 2, HEAD_DW = 3, HEAD_EXP = 4 };

struct HeadRows {                                 // the packed rows, written by head_rows_kernel
  int* n;                                         // how many
  int* row;                                       // which row of the call each is
  int* target;
  float* up;                                      // weight times upstream gradient
  float* lse;                                     // known from the start in a backward call
  float* z_target;
  float* ref;                                     // EXP: reference of the row's exponentials (a backward call: lse)
  float* sum;                                     // ... their sum over the pieces so far, without the target's
  float* alpha;                                   // ... what the sums of the pieces before this one are multiplied with (not in a backward call)
  float* scale;                                   // DX: the root of 1 / sum of all (a backward call: up)
  float* of_target;                               // DX, DZ: up times what the other tokens' probabilities add up to (a call that gives the loss)
  unsigned* above;                                // EXP: bit per chunk of columns of the piece that took their own reference
  float* above_ref;                               // ... and that reference
  int above_words, chunks;                        // words and chunks a row (64 columns; in head_few_kernel a block's)
};

struct HeadMaps { CUtensorMap a, a_packed, b; };  // a: of X itself (every row counts), a_packed: of the packed rows

struct HeadParams {
  HeadRows rows;
  int T;
  int m_extent;                                   // rows of the product: 0 = the packed rows, else this many (DW: d)
  int n_extent, n_first;                          // columns of the product; where they start in the right operand
  int k_extent, k_first;                          // K loop: 0 = the packed rows (DW); where it starts in the right operand (DX)
  int tn, n_cols;                                 // columns of a tile, tiles beside one another
  int stages, stage_bytes;                        // of the ring
  int split, kb_per_split;                        // shares of the K loop
  int chunk_kb;                                   // K blocks after which sums leave the tensor memory (0: at the end)
  int terms, term_at;                             // E / dZ is the sum of so many bf16 numbers, each term_at columns after the one before
  int rows_alloc;                                 // rows of the workspace arrays
  float2* part;                                   // STATS, EXP: [2 n_cols][rows_alloc] (max, sum)
  int online;                                     // a call that gives the loss.  EXP: statistics wanted, references may be outgrown
  __nv_bfloat16* dz; int64_t dz_ld;               // EXP, DZ
  float* acc; int acc_groups;                     // fp32 sums [split][128-row tile][group of 4 columns][128 rows][4]
  int acc_in, acc_out;                            // DX, DW: add what is there; leave the sum there instead of in `out`
  const uint32_t* wy;                             // DX from E: W's columns of the targets, [128-row tile][pair of d][128 rows] of 2 bf16
  void* out; int64_t out_ld; int out_f32, out_vec;
  unsigned long long wait_limit_ns;
  int withhold;
  int32_t* status_word;
};

// What W's column of the target is taken away with: up (1 - q_y).  A call that gives the loss has it from the sum without the
// target, however near to 1 the target's probability is; a backward call has lse.
__device__ __forceinline__ float target_factor(const HeadRows& rows, int row, int online) {
  return online ? rows.of_target[row] : -rows.up[row] * expm1f(rows.z_target[row] - rows.lse[row]);
}
// What DX's sums are multiplied with, one after the other: up / sum of all, as two factors, since a target far above the
// reference puts it below what a number holds where its product with the sums is not.
__device__ __forceinline__ float2 row_factors(const HeadRows& rows, int row, int online) {
  const float s = rows.scale[row];
  return online ? make_float2(s, s * rows.up[row]) : make_float2(s, 1.f);
}
// The unit of dZ: the first row's up, unless it is out of the ordinary.
__device__ __forceinline__ float dz_unit(const HeadRows& rows) {
  const float u = rows.up[0];
  return fabsf(u) >= 0x1p-60f && fabsf(u) <= 0x1p60f ? u : 1.f;
}

// What a CTA pair does next: a tile (raster groups of kHRaster row tiles, row tile fastest inside a group), a share of its K
// loop and, one after the other, the chunks of that.
struct HeadWork { int n_m_pairs, n_kb, kb_per_split, n_chunks, chunk_kb; };
struct HeadItem { int m_pair, col, split, chunk, kb0, n_blk; };
__device__ __forceinline__ bool head_item(int i, const HeadWork& w, const HeadParams& p, HeadItem& t) {
  t.chunk = i % w.n_chunks;
  const int64_t total = (int64_t)w.n_m_pairs * p.n_cols * p.split;
  int64_t at = (int64_t)(blockIdx.x >> 1) + (int64_t)(i / w.n_chunks) * (gridDim.x >> 1);
  if (at >= total) return false;
  t.split = (int)(at % p.split);
  at /= p.split;
  const int64_t per_group = (int64_t)kHRaster * p.n_cols;
  const int group = (int)(at / per_group), within = (int)(at - (int64_t)group * per_group);
  const int first = group * kHRaster, size = min(kHRaster, w.n_m_pairs - first);
  t.m_pair = first + within % size;
  t.col = within / size;
  const int end = min((t.split + 1) * w.kb_per_split, w.n_kb);
  t.kb0 = t.split * w.kb_per_split + t.chunk * w.chunk_kb;
  t.n_blk = max(0, min(w.chunk_kb, end - t.kb0));
  return true;
}

// 32 consecutive fp32 columns of this warp's rows, from tensor memory
__device__ __forceinline__ void head_columns(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  tmem_ld32(taddr, r);
  tmem_ld_wait();
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}

// A warp's 32 rows of 128 bytes, staged in `buf` (16-byte pieces swizzled by the row), to rows of an output.
// `row_at(r)` gives the address of row r's first byte or null, `n_bytes` how many of the 128 exist.
template <typename RowAt>
__device__ __forceinline__ void store_staged(uint32_t buf, int lane, int n_bytes, int vec, int elem, RowAt row_at) {
  const int piece = lane & 7;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = (lane >> 3) + 4 * k;
    const uint4 q = get_shared_v4(buf + r * 128 + ((piece ^ (r & 7)) << 4));
    uint8_t* to = row_at(r);
    if (to == nullptr) continue;
    to += piece * 16;
    const int left = n_bytes - piece * 16;
    if (vec && left >= 16) {
      *reinterpret_cast<uint4*>(to) = q;
    } else {
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (elem == 4) {
          if (4 * j < left) reinterpret_cast<uint32_t*>(to)[j] = w[j];
        } else {
          if (4 * j < left) reinterpret_cast<uint16_t*>(to)[2 * j] = (uint16_t)w[j];
          if (4 * j + 2 < left) reinterpret_cast<uint16_t*>(to)[2 * j + 1] = (uint16_t)(w[j] >> 16);
        }
      }
    }
  }
}
__device__ __forceinline__ void stage_bf16(uint32_t buf, int lane, int half, const float (&v)[32]) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const uint4 q = make_uint4(pack_bf16(v[g * 8], v[g * 8 + 1]), pack_bf16(v[g * 8 + 2], v[g * 8 + 3]),
                               pack_bf16(v[g * 8 + 4], v[g * 8 + 5]), pack_bf16(v[g * 8 + 6], v[g * 8 + 7]));
    put_shared_v4(buf + lane * 128 + (((half * 4 + g) ^ (lane & 7)) << 4), q);
  }
}
__device__ __forceinline__ void stage_bf16_row(uint32_t buf, int lane, const float (&v)[64]) {
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    const uint4 q = make_uint4(pack_bf16(v[g * 8], v[g * 8 + 1]), pack_bf16(v[g * 8 + 2], v[g * 8 + 3]),
                               pack_bf16(v[g * 8 + 4], v[g * 8 + 5]), pack_bf16(v[g * 8 + 6], v[g * 8 + 7]));
    put_shared_v4(buf + lane * 128 + ((g ^ (lane & 7)) << 4), q);
  }
}
__device__ __forceinline__ void stage_f32(uint32_t buf, int lane, const float (&v)[32]) {
#pragma unroll
  for (int g = 0; g < 8; ++g)
    put_shared_v4(buf + lane * 128 + ((g ^ (lane & 7)) << 4),
                  make_uint4(__float_as_uint(v[g * 4]), __float_as_uint(v[g * 4 + 1]), __float_as_uint(v[g * 4 + 2]), __float_as_uint(v[g * 4 + 3])));
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// kSums: the epilogue keeps a tile of at most 256 columns in registers and adds the chunks of the K loop up there (STATS, EXP, DZ).
template <int kMode, bool kSums>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kHThreads, 1)
head_kernel(const __grid_constant__ HeadMaps maps, const __grid_constant__ HeadParams p) {
  constexpr bool kLeftMn = kMode == HEAD_DW;      // X^T: its rows (columns of X) are contiguous
  constexpr bool kRightMn = kMode != HEAD_DX;     // W, dZ: their columns are contiguous; W^T: its K dimension is
  extern __shared__ uint8_t head_raw[];
  const uint32_t raw = smem_u32(head_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = head_raw + (base - raw);
  const uint32_t out_bufs = base + kHRing;
  const uint32_t bars = out_bufs + kHEpiWarps * kHOutBuf;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kHMaxStages + s); };
  // the accumulator is two slots of 256 columns: a wide tile takes both, narrow ones take turns
  auto acc_full = [&](int slot) { return bars + 8u * (2 * kHMaxStages + slot); };
  auto acc_empty = [&](int slot) { return bars + 8u * (2 * kHMaxStages + 2 + slot); };
  uint8_t* misc = base_ptr + kHRing + kHEpiWarps * kHOutBuf + kHBars;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);     // its wait limit sits at misc + 16
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();

  if (threadIdx.x == 0) {
    // full: armed by the leader's producer, completed by both CTAs' bytes (only the leader's copy is used); empty, acc_full:
    // one arrival, from the leader's commit, in both CTAs; acc_empty: an arrival per epilogue warp of both, on the leader's
    for (int s = 0; s < kHMaxStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int k = 0; k < 2; ++k) { mbar_init(acc_full(k), 1); mbar_init(acc_empty(k), 2 * kHEpiWarps); }
    *abort_flag = 0;
    *reinterpret_cast<volatile unsigned long long*>(misc + 16) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(&maps.a);
    if (kMode != HEAD_DX) prefetch_tmap(&maps.a_packed);
    prefetch_tmap(&maps.b);
  }
  if (warp == 1) {
    pair_tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kHMaxTile);
    pair_tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  cluster_barrier();                              // the peer's barriers exist before anything signals them
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();

  const int n = *p.rows.n;
  const int m_rows = p.m_extent > 0 ? p.m_extent : n;
  HeadWork work;
  work.n_m_pairs = (m_rows + 2 * kHM - 1) / (2 * kHM);
  // a K block is worked on once for each term, right after one another
  work.n_kb = ((p.k_extent > 0 ? p.k_extent : n) + kHK - 1) / kHK;
  work.kb_per_split = p.k_extent > 0 ? p.kb_per_split : (work.n_kb + p.split - 1) / p.split;
  work.chunk_kb = p.chunk_kb > 0 ? p.chunk_kb : max(work.kb_per_split, 1);
  work.n_chunks = max((min(work.kb_per_split, work.n_kb) + work.chunk_kb - 1) / work.chunk_kb, 1);
  const int terms = kMode == HEAD_DX || kMode == HEAD_DW ? p.terms : 1;     // ... as the operand of this product
  const bool wide = p.tn > 256;
  const int n_stages = p.stages, stage_bytes = p.stage_bytes;
  const CUtensorMap* map_a = kMode != HEAD_DX && n < p.T ? &maps.a_packed : &maps.a;

  if (warp == 0) {
    // ------------------------------------------------------------------------------------- producer (both CTAs)
    uint32_t issued = 0, s = 0, ph = 0;
    const uint32_t leader_full0 = peer_shared(full_bar(0), 0);
    bool ok = true;
    HeadItem t;
    for (int i = 0; ok && head_item(i, work, p, t); ++i) {
      const int n0 = t.col * p.tn, wt = min(p.tn, (p.n_extent - n0 + 31) & ~31);
      const int wa = min(wt, 256), wb = wt - wa;
      const int ca = wa >> 1, cb = wb >> 1, boxes_a = (ca + 63) >> 6, boxes = boxes_a + ((cb + 63) >> 6);
      const uint32_t tx = 2u * (kHLeft + boxes * kHBox);
      // lane 0: the left operand; lanes 1..boxes: a box of the right operand each
      const int bi = lane - 1;
      const bool has_box = bi >= 0 && bi < boxes;
      const int at = p.n_first + n0 + (bi < boxes_a ? (int)rank * ca + bi * 64 : wa + (int)rank * cb + (bi - boxes_a) * 64);
      const int m0 = (t.m_pair * 2 + (int)rank) * kHM;
      const int n_blk = t.n_blk * terms;
      for (int b = 0; b < n_blk; ++b) {
        if (CWL_WITHHELD(p) && i == 0 && b == n_blk - 1) { ok = false; break; }
        const bool step_ok = mbar_wait(empty_bar(s), ph ^ 1u, abort_flag);
        if (!__all_sync(0xffffffffu, step_ok)) { ok = false; break; }
        const int block = terms == 1 ? b : b / terms;
        const int k = (t.kb0 + block) * kHK, second = (b - block * terms) * p.term_at;
        const uint32_t sa = base + s * stage_bytes, sb = sa + kHLeft, full = leader_full0 + 8u * s;
        if (lane == 0) {
          if (rank == 0) mbar_expect_tx(full_bar(s), tx);
          if (kLeftMn) {
            pair_load_2d(sa, map_a, full, m0, k);
            pair_load_2d(sa + kHBox, map_a, full, m0 + 64, k);
          } else {
            pair_load_2d(sa, map_a, full, kMode == HEAD_DX ? second + k : k, m0);
          }
        } else if (has_box) {
          if (kRightMn) pair_load_2d(sb + bi * kHBox, &maps.b, full, kMode == HEAD_DW ? second + at : at, k);
          else pair_load_2d(sb + bi * kHBox, &maps.b, full, p.k_first + k, at);
        }
        ++issued;
        if (++s == (uint32_t)n_stages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok && rank == 0 && lane == 0) {
      // copies already issued get a bounded chance to land before the CTA leaves
      for (uint32_t back = 1; back <= (uint32_t)n_stages && back <= issued; ++back) {
        const uint32_t j = issued - back;
        const unsigned long long t0 = global_timer();
        while (!mbar_try_wait(full_bar(j % n_stages), (j / n_stages) & 1u) && global_timer() - t0 < p.wait_limit_ns) {}
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------- MMA issuer (leader only)
    if (lane == 0 && rank == 0) {
      uint32_t local = 0, s = 0, ph = 0;
      bool ok = true;
      const uint64_t step_a = kLeftMn ? (16 * 128) >> 4 : (16 * 2) >> 4;
      const uint64_t step_b = kRightMn ? (16 * 128) >> 4 : (16 * 2) >> 4;
      const uint64_t desc_a = kLeftMn ? make_smem_desc(base, kHBox, 1024) : make_smem_desc(base, 16, 1024);
      const uint64_t desc_b = kRightMn ? make_smem_desc(base + kHLeft, kHBox, 1024) : make_smem_desc(base + kHLeft, 16, 1024);
      HeadItem t;
      for (int i = 0; ok && head_item(i, work, p, t); ++i) {
        const int n0 = t.col * p.tn, wt = min(p.tn, (p.n_extent - n0 + 31) & ~31);
        const int wa = min(wt, 256), wb = wt - wa;
        const uint32_t idesc_a = pair_idesc(wa, kLeftMn, kRightMn), idesc_b = pair_idesc(wb > 0 ? wb : 32, kLeftMn, kRightMn);
        const uint64_t second = (uint64_t)((((wa >> 1) + 63) >> 6) * kHBox) >> 4;
        const int n_blk = t.n_blk * terms;
        if (n_blk <= 0) continue;                 // nothing to add up: the epilogue takes zeros
        const int slot = wide ? 0 : (int)(local & 1u);
        const uint32_t use = wide ? local : local >> 1;
        if (!mbar_wait(acc_empty(slot), (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        auto mma = [&](uint32_t stage, int half, bool first) {
          const uint64_t da = desc_a + (uint64_t)(((int)stage * stage_bytes) >> 4), db = desc_b + (uint64_t)(((int)stage * stage_bytes) >> 4) + (half ? second : 0);
          const uint32_t to = tmem + (half ? 256u : 256u * (uint32_t)slot);
          const uint32_t idesc = half ? idesc_b : idesc_a;
#pragma unroll
          for (int kk = 0; kk < kHK / 16; ++kk) pair_mma_bf16(to, da + kk * step_a, db + kk * step_b, idesc, first && kk == 0 ? 0u : 1u);
        };
        int b = 0;
        if (wide) {
          // The epilogue hands the first 256 columns back before the others: their MMAs of as many K blocks as the ring
          // holds run ahead meanwhile.
          const int ahead = min(n_blk, n_stages);
          uint32_t s1 = s, ph1 = ph;
          for (; b < ahead; ++b) {
            if (!mbar_wait(full_bar(s1), ph1, abort_flag)) { ok = false; break; }
            tc_fence_after();
            mma(s1, 0, b == 0);
            if (++s1 == (uint32_t)n_stages) { s1 = 0; ph1 ^= 1u; }
          }
          if (ok && !mbar_wait(acc_empty(1), (use & 1u) ^ 1u, abort_flag)) ok = false;
          if (!ok) break;
          tc_fence_after();
          for (int c = 0; c < ahead; ++c) {
            if (wb > 0) mma(s, 1, c == 0);
            pair_commit(empty_bar(s));
            if (++s == (uint32_t)n_stages) { s = 0; ph ^= 1u; }
          }
        }
        for (; b < n_blk; ++b) {
          if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          mma(s, 0, b == 0);
          if (wb > 0) mma(s, 1, b == 0);
          pair_commit(empty_bar(s));
          if (++s == (uint32_t)n_stages) { s = 0; ph ^= 1u; }
        }
        if (ok) pair_commit(acc_full(slot));
        ++local;
      }
      if (!ok) {
        // MMAs in flight get a bounded time to retire before the tensor memory is released
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 1000000ull) {}
      }
    }
  } else {
    // ------------------------------------------------------------------------------------- epilogue (both CTAs)
    const int quad = warp & 3;                    // tensor-memory lanes this warp may read
    const int chalf = (warp - 2) >> 2;            // the two warps of a quadrant take alternate chunks of columns
    const uint32_t buf = out_bufs + (uint32_t)(warp - 2) * kHOutBuf;
    // kSums: the chunks' sums of this warp's columns.  Beside the 64 numbers at work they do not fit 168 registers (320 threads are
    // given them as 384 would be): STATS spills 0.5 KB a thread, EXP 0.7, DZ 0.7, which is in what these sums are said to cost above.
    float held[2][64];
    uint32_t local = 0;
    HeadItem t;
    for (int i = 0; head_item(i, work, p, t); ++i) {
      const int n0 = t.col * p.tn, cols = min(p.tn, p.n_extent - n0);
      const int m_tile = t.m_pair * 2 + (int)rank, row0 = m_tile * kHM + quad * 32, row = row0 + lane;
      const bool live = row < m_rows;
      const bool any = t.n_blk > 0;
      const int slot = wide ? 0 : (int)(local & 1u);
      if (any) {
        if (!__all_sync(0xffffffffu, mbar_wait(acc_full(slot), (wide ? local : local >> 1) & 1u, abort_flag))) break;
        tc_fence_after();
        ++local;
      }
      const uint32_t t_row = tmem + ((uint32_t)(quad * 32) << 16) + 256u * (uint32_t)slot;
      // the first 256 columns of a wide tile are free as soon as this warp is past them
      bool first_held = wide;
      auto past = [&](int c) {
        if (any && first_held && c >= 256) {
          first_held = false;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_in_cluster(peer_shared(acc_empty(0), 0));
        }
      };
      if (kMode == HEAD_STATS || kMode == HEAD_DZ || kMode == HEAD_EXP) {
        // this warp's columns: every other 64
        auto columns = [&](int c, float (&v)[64]) {
          uint32_t r[2][32];
          tmem_ld32(t_row + c, r[0]);
          tmem_ld32(t_row + c + 32, r[1]);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 64; ++j) v[j] = __uint_as_float(r[j >> 5][j & 31]);
        };
        if (kSums) {
          if (row0 < m_rows) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int c = (2 * k + chalf) * 64;
              if (c < cols) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  float v[32];
                  head_columns(t_row + c + h * 32, v);
#pragma unroll
                  for (int j = 0; j < 32; ++j) held[k][h * 32 + j] = t.chunk == 0 ? v[j] : held[k][h * 32 + j] + v[j];
                }
              }
            }
          } else if (kMode == HEAD_DZ) {          // rows that are not there are written as zeros all the same
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int j = 0; j < 64; ++j) held[k][j] = 0.f;
          }
          if (t.chunk + 1 < work.n_chunks) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_in_cluster(peer_shared(acc_empty(slot), 0));
            continue;
          }
        }
        float up = 0.f, ref = kMode == HEAD_STATS ? -INFINITY : 0.f;
        int y = -1;
        if (live) {
          y = p.rows.target[row] - (p.n_first + n0);
          if (y >= cols) y = -1;                  // another tile's
          if (kMode == HEAD_DZ) {
            up = p.rows.up[row] / dz_unit(p.rows);
            ref = p.rows.lse[row];
          } else if (kMode == HEAD_EXP) {
            ref = p.rows.ref[row];
          }
        }
        float m = ref, sum = 0.f;                 // STATS, EXP: the sum so far, relative to m
        auto take = [&](int c, float (&v)[64]) {  // columns [c, c + 64) of the tile; sums and maxima in four chains
          if (cols - c < 64) {
#pragma unroll
            for (int j = 0; j < 64; ++j) v[j] = j < cols - c ? v[j] : -INFINITY;
          }
          const bool mine = (unsigned)(y - c) < 64u;
          float z_y = 0.f;                        // DZ: the target's logit
          if (mine) {
#pragma unroll
            for (int j = 0; j < 64; ++j)
              if (j == y - c) {
                if (kMode == HEAD_DZ) {
                  z_y = v[j];
                } else {
                  p.rows.z_target[row] = v[j];
                  v[j] = -INFINITY;               // the target stays out of E, of the sum and of what a reference is held against
                }
              }
          }
          float own = ref;                        // reference of these columns
          if (kMode == HEAD_STATS || (kMode == HEAD_EXP && p.online)) {
            float t4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int j = 4; j < 64; ++j) t4[j & 3] = fmaxf(t4[j & 3], v[j]);
            const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
            if (kMode == HEAD_STATS) {
              own = top > m ? top : m;            // -inf as long as there was nothing but the target
            } else if (live && top > ref + kAbove) {
              own = top;
              const int chunk = (n0 + c) >> 6;    // tiles start at multiples of 64 here
              atomicOr(p.rows.above + (int64_t)row * p.rows.above_words + (chunk >> 5), 1u << (chunk & 31));
              p.rows.above_ref[(int64_t)row * p.rows.chunks + chunk] = top;
            }
          }
          const float shift = kMode == HEAD_STATS && own == -INFINITY ? 0.f : own * kLog2e;
          float p4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 64; ++j) {
            v[j] = exp2_fast(fmaf(v[j], kLog2e, -shift));
            if (kMode != HEAD_DZ) p4[j & 3] += v[j];
          }
          if (kMode != HEAD_DZ) {
            const float part = (p4[0] + p4[1]) + (p4[2] + p4[3]);
            if (own > m) { sum *= exp2_fast((m - own) * kLog2e); m = own; }
            sum += m > own ? part * exp2_fast((own - m) * kLog2e) : part;
            if (kMode == HEAD_STATS) return;
          } else {
#pragma unroll
            for (int j = 0; j < 64; ++j) v[j] *= up;         // rows that are not there: 0
            if (mine) {
              const float of_target = p.online ? -p.rows.of_target[row] / dz_unit(p.rows) : up * expm1f(z_y - ref);
#pragma unroll
              for (int j = 0; j < 64; ++j) v[j] = j == y - c ? of_target : v[j];
            }
          }
#pragma unroll 1
          for (int term = 0; term < p.terms; ++term) {
            __syncwarp();                         // every lane has read what was staged before
            stage_bf16_row(buf, lane, v);
            if (p.terms > 1) {
#pragma unroll
              for (int j = 0; j < 64; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(v[j]));
            }
            __syncwarp();
            uint8_t* first = reinterpret_cast<uint8_t*>(p.dz + (int64_t)row0 * p.dz_ld + n0 + c + term * p.term_at);
            store_staged(buf, lane, 128, 1, 2, [&](int r) { return first + (int64_t)r * p.dz_ld * 2; });
          }
        };
        if (kSums) {
          if (row0 < m_rows || kMode == HEAD_DZ) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
              if ((2 * k + chalf) * 64 < cols) take((2 * k + chalf) * 64, held[k]);
          }
        } else {
#pragma unroll 1
          for (int c = chalf * 64; c < cols; c += 128) {
            past(c);
            float v[64];
            columns(c, v);
            take(c, v);
          }
        }
        if (kMode != HEAD_DZ && (kMode == HEAD_STATS || p.online) && live)
          p.part[(int64_t)(t.col * 2 + chalf) * p.rows_alloc + row] = make_float2(m, sum);
      } else {
        const int64_t tiles = (int64_t)work.n_m_pairs * 2;
        float* sums = p.acc + ((((int64_t)t.split * tiles + m_tile) * p.acc_groups + n0 / 4) * kHM + quad * 32 + lane) * 4;
        const bool add = p.acc_in || t.chunk > 0, keep = p.acc_out || t.chunk + 1 < work.n_chunks;
        // where this warp's rows go: rows of the call for DX, columns of X for DW
        const int mine = !live ? -1 : kMode == HEAD_DX && n < p.T ? p.rows.row[row] : row;
        const bool from_e = kMode == HEAD_DX && p.wy != nullptr;
        // a backward call's reference is lse from the first piece on: nobody writes alpha
        const float alpha = from_e && p.online && p.acc_in && t.chunk == 0 && live ? p.rows.alpha[row] : 1.f;
        const float up = from_e && live && !keep ? target_factor(p.rows, row, p.online) : 0.f;
        const float2 scale = from_e ? (live && !keep ? row_factors(p.rows, row, p.online) : make_float2(0.f, 0.f))
                                    : make_float2(n > 0 ? dz_unit(p.rows) : 1.f, 1.f);
        const uint32_t* wy = p.wy + ((int64_t)m_tile * p.acc_groups * 2 + n0 / 2) * kHM + quad * 32 + lane;
        const int chunk = keep || p.out_f32 ? 32 : 64;
#pragma unroll 1
        for (int c = chalf * chunk; c < cols; c += 2 * chunk) {
          past(c);
          __syncwarp();
#pragma unroll 1
          for (int h = 0; h < chunk / 32; ++h) {
            const int cc = c + h * 32;
            float v[32];
            if (any && cc < cols) {
              head_columns(t_row + cc, v);
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = 0.f;
            }
            if (add) {
#pragma unroll
              for (int g = 0; g < 8; ++g) {
                if (cc + g * 4 < cols) {
                  const float4 x = *reinterpret_cast<const float4*>(sums + (int64_t)(cc / 4 + g) * kHM * 4);
                  v[g * 4] += x.x * alpha; v[g * 4 + 1] += x.y * alpha; v[g * 4 + 2] += x.z * alpha; v[g * 4 + 3] += x.w * alpha;
                }
              }
            }
            if (keep) {
#pragma unroll
              for (int g = 0; g < 8; ++g)
                if (cc + g * 4 < cols)
                  *reinterpret_cast<float4*>(sums + (int64_t)(cc / 4 + g) * kHM * 4) = make_float4(v[g * 4], v[g * 4 + 1], v[g * 4 + 2], v[g * 4 + 3]);
              continue;
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = v[j] * scale.x * scale.y;
            if (from_e) {
#pragma unroll
              for (int g = 0; g < 16; ++g) {
                if (cc + g * 2 < cols) {
                  const uint32_t x = wy[(int64_t)(cc / 2 + g) * kHM];
                  v[g * 2] -= up * __uint_as_float(x << 16);
                  v[g * 2 + 1] -= up * __uint_as_float(x & 0xFFFF0000u);
                }
              }
            }
            if (p.out_f32) stage_f32(buf, lane, v);
            else stage_bf16(buf, lane, h, v);
          }
          if (!keep) {
            __syncwarp();
            const int es = p.out_f32 ? 4 : 2;
            const int64_t col = n0 + c;
            // the row that lane r holds, asked for by all lanes together
            int to[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) to[k] = __shfl_sync(0xffffffffu, mine, (lane >> 3) + 4 * k);
            store_staged(buf, lane, (cols - c) * es, p.out_vec, es, [&](int r) -> uint8_t* {
              const int q = to[(r - (lane >> 3)) >> 2];
              return q < 0 ? nullptr : reinterpret_cast<uint8_t*>(p.out) + ((int64_t)q * p.out_ld + col) * es;
            });
          }
        }
      }
      if (any) {
        past(256);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_in_cluster(peer_shared(acc_empty(wide ? 1 : slot), 0));
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_barrier();     // neither CTA leaves (or frees tensor memory) while the other may still signal it or write its own
  if (threadIdx.x == 0 && *abort_flag) flag_status(p.status_word, CWL_ERR_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    pair_tmem_dealloc(tmem, kHMaxTile);
  }
}

#include "head_few.cuh"

// ------------------------------------------------------------------------------------------------ rows that count
struct RowsParams {
  const __nv_bfloat16* X; int64_t ldx;
  const __nv_bfloat16* W; int64_t ldw;            // online: a logit of every row is wanted as its reference
  int T, d, V;
  const int32_t* targets; const float* weight; const float* dloss; const float* lse_in;
  float* loss; float* lse;
  void* dX; int64_t lddx; int dx_elem;
  __nv_bfloat16* packed; int64_t packed_ld;
  HeadRows rows;
  int per_block, backward, online, reference;
  int32_t* status_word;
};

constexpr int kRowsThreads = 1024;
constexpr int kRowsColumn = 8192;                 // of W's column 0 kept in shared memory

__device__ __forceinline__ float row_up(const RowsParams& p, int t) {
  float up = p.weight != nullptr ? p.weight[t] : 1.f;
  if (p.dloss != nullptr) up *= p.dloss[t];
  return up;
}
// a row counts if it has a target and its loss or, in a backward call, its gradient is not 0 whatever the logits are
__device__ __forceinline__ bool row_counts(const RowsParams& p, int t) {
  // no branch between the loads: those of many rows go out together
  const unsigned y = (unsigned)__ldg(p.targets + t);
  float up = p.weight != nullptr ? __ldg(p.weight + t) : 1.f;
  if (p.backward && p.dloss != nullptr) up *= __ldg(p.dloss + t);
  return (y < (unsigned)p.V) & (up != 0.f);
}

// Lists the rows that count, packs their activations where some do not, works out their references (of many rows: the logit of column 0),
// and writes the outputs of those that do not.  Every block counts all rows before its own itself (two words a row from L2), so one launch does it.
__global__ void __launch_bounds__(kRowsThreads) head_rows_kernel(const RowsParams p) {
  __shared__ int sums[2][kRowsThreads / 32];
  __shared__ int counts[kRowsThreads];
  __shared__ __align__(16) __nv_bfloat16 column[kRowsColumn];
  pdl_wait();
  pdl_launch_dependents();                        // after the wait and never before it: head_few_kernel fetches W by that
  if (p.online && p.reference) {
#pragma unroll 8
    for (int j = threadIdx.x; j < kRowsColumn; j += kRowsThreads) column[j] = j < p.d ? p.W[(int64_t)j * p.ldw] : __float2bfloat16_rn(0.f);
  }
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t first64 = (int64_t)blockIdx.x * p.per_block;
  const int first = (int)(first64 < p.T ? first64 : p.T);
  const int last = (int)(first64 + p.per_block < p.T ? first64 + p.per_block : p.T);
  int before = 0, total = 0;
#pragma unroll 8
  for (int64_t t = tid; t < p.T; t += kRowsThreads) {
    const int c = row_counts(p, (int)t) ? 1 : 0;
    total += c;
    if (t < first) before += c;
  }
  for (int o = 16; o > 0; o >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, o);
    total += __shfl_xor_sync(0xffffffffu, total, o);
  }
  if (lane == 0) { sums[0][warp] = before; sums[1][warp] = total; }
  __syncthreads();
  before = total = 0;
  for (int w = 0; w < kRowsThreads / 32; ++w) { before += sums[0][w]; total += sums[1][w]; }
  if (blockIdx.x == 0 && tid == 0) *p.rows.n = total;

  // this block's rows, kRowsThreads at a time
  for (int64_t t0 = first; t0 < last; t0 += kRowsThreads) {
    const int64_t t = t0 + tid;
    const bool in = t < last, counts_here = in && row_counts(p, (int)t);
    const unsigned mask = __ballot_sync(0xffffffffu, counts_here);
    __syncthreads();
    if (lane == 0) sums[0][warp] = __popc(mask);
    __syncthreads();
    int at = before + __popc(mask & ((1u << lane) - 1u));
    for (int w = 0; w < kRowsThreads / 32; ++w) {
      if (w < warp) at += sums[0][w];
      before += sums[0][w];
    }
    counts[tid] = counts_here ? at : in ? -1 : -2;
    if (counts_here) {
      p.rows.row[at] = (int)t;
      p.rows.target[at] = p.targets[t];
      p.rows.up[at] = row_up(p, (int)t);
      if (p.backward) {
        p.rows.lse[at] = p.rows.ref[at] = p.lse_in[t];
        p.rows.scale[at] = row_up(p, (int)t);
      }
      if (p.online) {
        p.rows.sum[at] = 0.f;
        for (int w = 0; w < p.rows.above_words; ++w) p.rows.above[(int64_t)at * p.rows.above_words + w] = 0u;
      }
    } else if (in) {
      const bool bad = p.targets[t] >= p.V;
      if (bad) flag_status(p.status_word, CWL_ERR_INVALID_ARG);
      const float v = bad ? NAN : 0.f;
      if (p.loss != nullptr) p.loss[t] = v;
      if (p.lse != nullptr) p.lse[t] = v;
    }
    __syncthreads();
    // a warp a row: into the packed activations, its logit of column 0, or zeros into its gradient
    const int rows_here = (int)(last - t0 < kRowsThreads ? last - t0 : kRowsThreads);
    for (int r = warp; r < rows_here; r += kRowsThreads / 32) {
      const int to = counts[r];
      const bool pack = total < p.T, refer = p.online && p.reference;
      if (to >= 0 && (pack || refer)) {
        const __nv_bfloat16* x = p.X + (t0 + r) * p.ldx;
        __nv_bfloat16* out = p.packed + (int64_t)to * p.packed_ld;
        float z = 0.f;
#pragma unroll 8
        for (int j = lane; j < p.d / 8; j += 32) {
          const uint4 q = __ldg(reinterpret_cast<const uint4*>(x) + j);
          if (pack) reinterpret_cast<uint4*>(out)[j] = q;
          if (refer && j < kRowsColumn / 8) {
            const uint4 c = reinterpret_cast<const uint4*>(column)[j];
            const uint32_t a[4] = {q.x, q.y, q.z, q.w}, b[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              z = fmaf(__uint_as_float(a[k] << 16), __uint_as_float(b[k] << 16), z);
              z = fmaf(__uint_as_float(a[k] & 0xFFFF0000u), __uint_as_float(b[k] & 0xFFFF0000u), z);
            }
          }
        }
        if (pack)
          for (int j = p.d / 8 * 8 + lane; j < p.d; j += 32) out[j] = x[j];
        if (refer) {
          // what the column in shared memory does not hold, and the elements after the last eight
          for (int j = min(p.d / 8 * 8, kRowsColumn) + lane; j < p.d; j += 32)
            z = fmaf(__bfloat162float(x[j]), __bfloat162float(p.W[(int64_t)j * p.ldw]), z);
          for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
          if (lane == 0) p.rows.ref[to] = fabsf(z) < 1e30f ? z : 0.f;
        }
      } else if (to == -1 && p.dX != nullptr) {
        uint8_t* out = reinterpret_cast<uint8_t*>(p.dX) + (t0 + r) * p.lddx * p.dx_elem;
        for (int j = lane; j < p.d; j += 32) {
          if (p.dx_elem == 4) reinterpret_cast<float*>(out)[j] = 0.f;
          else reinterpret_cast<uint16_t*>(out)[j] = 0;
        }
      }
    }
  }
  // the last K block of dW's product reads on to a multiple of 64 rows
  if (blockIdx.x == gridDim.x - 1 && total < p.T) {
    const int64_t end = ((int64_t)total + kHK - 1) / kHK * kHK;
    for (int64_t r = total + warp; r < end; r += kRowsThreads / 32)
      for (int64_t j = lane; j < p.packed_ld; j += 32) p.packed[r * p.packed_ld + j] = __float2bfloat16_rn(0.f);
  }
}

// (max, sum) of a row over the tiles, relative to a reference that is at least `m`: kRowsEach rows a block (32, or one where
// there are few), 256 / kRowsEach threads a row, met in a fixed order.  The first thread of a row gets the result.
constexpr int kFinishThreads = 256;
__device__ __forceinline__ float2 join_sums(const float2& a, const float2& b) {
  const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.f : top;
  // a NaN in a sum stays one; a maximum is NaN only where all logits were
  return make_float2(top, a.y * exp2_fast((a.x - ref) * kLog2e) + b.y * exp2_fast((b.x - ref) * kLog2e));
}
template <int kRowsEach>
__device__ __forceinline__ float2 row_sums(const float2* part, int n_part, int rows_alloc, int64_t row, bool there, float m, float2* met) {
  constexpr int kSlices = kFinishThreads / kRowsEach;
  const int slice = threadIdx.x / kRowsEach;
  float2 all = make_float2(m, 0.f);
  if (there) {
    // eight loads at a time
    for (int c0 = slice; c0 < n_part; c0 += kSlices * 8) {
      float2 x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = c0 + k * kSlices < n_part ? part[(int64_t)(c0 + k * kSlices) * rows_alloc + row] : make_float2(m, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) all = join_sums(all, x[k]);
    }
  }
  met[threadIdx.x] = all;
#pragma unroll
  for (int k = kSlices / 2; k >= 1; k /= 2) {
    __syncthreads();
    if (slice < k) met[threadIdx.x] = all = join_sums(all, met[threadIdx.x + k * kRowsEach]);
  }
  return all;
}

// The target joins the others, whose exponentials add up to `sum` relative to m: relative to its own logit z where that is the larger.
struct JoinedTarget {
  float top, over;                                // log-sum-exp = top + over
  float loss, others;                             // lse - z; what the others' probabilities add up to
  float scale;                                    // root of 1 / the sum of all
};
__device__ __forceinline__ JoinedTarget join_target(float m, float sum, float z) {
  JoinedTarget t;
  const float h = z > m ? exp2_fast((m - z) * (0.5f * kLog2e)) : 1.f;
  const float others = sum * h * h, total = others + (z > m ? 1.f : exp2_fast((z - m) * kLog2e));
  t.top = z > m ? z : m;
  t.over = z > m ? log1pf(others) : logf(total);
  t.loss = z > m ? t.over : m - z + t.over;       // not lse - z, which has been rounded at the size of the logits
  t.others = others / total;
  t.scale = h * rsqrtf(total);
  return t;
}

// Log-sum-exp, loss and the target's share of dZ of every row that counts, from the tiles' maxima and sums.
template <int kRowsEach>
__global__ void __launch_bounds__(kFinishThreads)
head_finish_kernel(HeadRows rows, const float2* part, int n_part, int rows_alloc, const float* weight, float* loss, float* lse) {
  __shared__ float2 met[kFinishThreads];
  pdl_launch_dependents();
  pdl_wait();
  const int n = *rows.n;
  if ((int64_t)blockIdx.x * kRowsEach >= n) return;
  const int64_t row = (int64_t)blockIdx.x * kRowsEach + threadIdx.x % kRowsEach;
  const float2 all = row_sums<kRowsEach>(part, n_part, rows_alloc, row, row < n, -INFINITY, met);
  if (threadIdx.x < kRowsEach && row < n) {
    const JoinedTarget j = join_target(all.x, all.y, rows.z_target[row]);
    const float l = j.top + j.over;
    const int t = rows.row[row];
    rows.lse[row] = l;
    rows.of_target[row] = rows.up[row] * j.others;
    if (lse != nullptr) lse[t] = l;
    if (loss != nullptr) loss[t] = (weight != nullptr ? weight[t] : 1.f) * j.loss;
  }
}

// After EXP of a piece: the rows' sums so far, on the reference that the piece leaves, and what the sums of earlier pieces (in
// head_merge_kernel and in DX) are multiplied with.  Where 64 columns outgrew the reference, all of the row's piece is put
// on the new one.  After the last piece: log-sum-exp, loss, and the factor of dX.
struct MergeParams {
  HeadRows rows;
  const float2* part;
  int n_part, rows_alloc, last;
  __nv_bfloat16* dz; int64_t dz_ld;
  int width, terms, term_at;
  int chunk_cols;                                 // columns that share a reference
  const float* weight; float* loss; float* lse;
};
template <int kRowsEach>
__global__ void __launch_bounds__(kFinishThreads) head_merge_kernel(const MergeParams p) {
  __shared__ float2 met[kFinishThreads];
  __shared__ float old_ref[kRowsEach], new_ref[kRowsEach];
  pdl_launch_dependents();
  pdl_wait();
  const HeadRows& rows = p.rows;
  const int n = *rows.n, r = threadIdx.x % kRowsEach;
  const int row0 = blockIdx.x * kRowsEach, row = row0 + r;
  if (row0 >= n) return;
  const float ref = row < n ? rows.ref[row] : 0.f;
  const float2 all = row_sums<kRowsEach>(p.part, p.n_part, p.rows_alloc, row, row < n, ref, met);
  if (threadIdx.x < kRowsEach) {
    const float m = all.x;
    old_ref[r] = ref;
    new_ref[r] = m;
    if (row < n) {
      const float alpha = m > ref ? exp2_fast((ref - m) * kLog2e) : 1.f;
      const float sum = rows.sum[row] * alpha + all.y;
      rows.alpha[row] = alpha;
      rows.ref[row] = m;
      rows.sum[row] = sum;
      if (p.last) {
        const JoinedTarget j = join_target(m, sum, rows.z_target[row]);
        const int t = rows.row[row];
        if (p.lse != nullptr) p.lse[t] = j.top + j.over;
        p.loss[t] = (p.weight != nullptr ? p.weight[t] : 1.f) * j.loss;
        rows.scale[row] = j.scale;
        rows.of_target[row] = rows.up[row] * j.others;
      }
    }
  }
  __syncthreads();
  // a row to a warp, or to the block; numbers eight at a time
  constexpr int kTogether = kRowsEach == 1 ? kFinishThreads : 32;
  const int lane = threadIdx.x % kTogether;
  for (int r = threadIdx.x / kTogether; r < kRowsEach && row0 + r < n; r += kFinishThreads / kTogether) {
    if (!(new_ref[r] > old_ref[r])) continue;            // as good as always; where all outgrow it, 2048 rows of 32000 take 0.47 ms
    const int64_t at = row0 + r;
    const float from_old = exp2_fast((old_ref[r] - new_ref[r]) * kLog2e);
    auto factor = [&](int c) {
      const int chunk = c / p.chunk_cols;
      const bool above = rows.above[at * rows.above_words + (chunk >> 5)] >> (chunk & 31) & 1u;
      return above ? exp2_fast((rows.above_ref[at * rows.chunks + chunk] - new_ref[r]) * kLog2e) : from_old;
    };
    auto put = [&](__nv_bfloat16* e, float x) {
      for (int k = 0; k < p.terms; ++k) {
        e[k * p.term_at] = __float2bfloat16_rn(x);
        x -= __bfloat162float(e[k * p.term_at]);
      }
    };
    __nv_bfloat16* e = p.dz + at * p.dz_ld;
    const int whole = p.terms == 1 ? p.width / 8 : 0;
#pragma unroll 4
    for (int i = lane; i < whole; i += kTogether) {
      uint4 q = reinterpret_cast<const uint4*>(e)[i];
      const float f = factor(i * 8);
      uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(__uint_as_float(w[k] << 16) * f, __uint_as_float(w[k] & 0xFFFF0000u) * f);
        w[k] = reinterpret_cast<const uint32_t&>(two);
      }
      reinterpret_cast<uint4*>(e)[i] = q;
    }
    for (int c = whole * 8 + lane; c < p.width; c += kTogether) {
      float x = 0.f;
      for (int k = p.terms - 1; k >= 0; --k) x += __bfloat162float(e[c + k * p.term_at]);
      put(e + c, x * factor(c));
    }
    if (kTogether == 32) __syncwarp();
    else __syncthreads();
    for (int w = lane; w < rows.above_words; w += kTogether) rows.above[at * rows.above_words + w] = 0u;
  }
}

// W's columns of the targets, packed as DX's epilogue reads them: [128-row tile][pair of d][128 rows] of two bf16.
// Of few rows: a block a row, a 32-byte sector of W for every number, and the target's logit, which is the row's reference.
// Of many: blocks bring two rows of W (or parts of them) into shared memory and serve all targets from there, so that W is
// read once, in order (16384 rows of 4096, V = 32000: 2.1 GB against 0.26); the reference is head_rows_kernel's.
constexpr int kGatherThreads = 256;
constexpr int kGatherBatch = 8;
__global__ void __launch_bounds__(kGatherThreads)
head_gather_kernel(HeadRows rows, const __nv_bfloat16* X, int64_t ldx, const __nv_bfloat16* W, int64_t ldw, int d, int groups, int online, uint32_t* wy) {
  __shared__ float met[kGatherThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x;
  if (row >= *rows.n) return;
  const int y = rows.target[row], pairs = groups * 2;
  const uint16_t* w = reinterpret_cast<const uint16_t*>(W) + y;
  const uint16_t* x = reinterpret_cast<const uint16_t*>(X) + (int64_t)rows.row[row] * ldx;
  uint32_t* out = wy + (int64_t)(row >> 7) * pairs * kHM + (row & 127);
  float z = 0.f;
  for (int j0 = threadIdx.x; j0 < pairs; j0 += kGatherThreads * kGatherBatch) {
    uint32_t v[kGatherBatch], a[kGatherBatch];
#pragma unroll
    for (int k = 0; k < kGatherBatch; ++k) {
      const int64_t j = (int64_t)(j0 + k * kGatherThreads) * 2;
      v[k] = a[k] = 0u;
      if (j < d) { v[k] = w[j * ldw]; a[k] = x[j]; }
      if (j + 1 < d) { v[k] |= (uint32_t)w[(j + 1) * ldw] << 16; a[k] |= (uint32_t)x[j + 1] << 16; }
    }
#pragma unroll
    for (int k = 0; k < kGatherBatch; ++k) {
      const int j = j0 + k * kGatherThreads;
      if (j < pairs) out[(int64_t)j * kHM] = v[k];
      z = fmaf(__uint_as_float(v[k] << 16), __uint_as_float(a[k] << 16), z);
      z = fmaf(__uint_as_float(v[k] & 0xFFFF0000u), __uint_as_float(a[k] & 0xFFFF0000u), z);
    }
  }
  if (!online) return;
  for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
  if ((threadIdx.x & 31) == 0) met[threadIdx.x >> 5] = z;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < kGatherThreads / 32; ++k) z += met[k];
    rows.ref[row] = fabsf(z) < 1e30f ? z : 0.f;
  }
}
constexpr int kOrderedThreads = 512;
constexpr int kOrderedColumns = 28 * 1024;               // of two rows of W: 112 KB, two blocks an SM
__global__ void __launch_bounds__(kOrderedThreads)
head_gather_ordered_kernel(HeadRows rows, const __nv_bfloat16* W, int64_t ldw, int d, int V, int groups, int columns, uint32_t* wy) {
  extern __shared__ __align__(16) uint8_t gather_raw[];
  uint16_t* first_row = reinterpret_cast<uint16_t*>(gather_raw);
  uint16_t* second_row = first_row + columns;
  pdl_launch_dependents();
  pdl_wait();
  const int n = *rows.n, pair = blockIdx.x, first = blockIdx.y * columns;
  const int width = min(columns, V - first);
  const bool two = pair * 2 + 1 < d;
  const uint16_t* from = reinterpret_cast<const uint16_t*>(W) + (int64_t)pair * 2 * ldw + first;
  // all copies of the block on their way at once
  auto copy = [](void* to, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(src), "r"(bytes) : "memory");
  };
  for (int j = threadIdx.x; j < width / 8; j += kOrderedThreads) {
    copy(first_row + j * 8, from + j * 8, 16);
    copy(second_row + j * 8, two ? from + ldw + j * 8 : from, two ? 16 : 0);
  }
  asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
  for (int j = width / 8 * 8 + threadIdx.x; j < width; j += kOrderedThreads) {
    first_row[j] = from[j];
    second_row[j] = two ? from[ldw + j] : (uint16_t)0;
  }
  __syncthreads();
#pragma unroll 4
  for (int row = threadIdx.x; row < n; row += kOrderedThreads) {
    const unsigned y = (unsigned)(rows.target[row] - first);
    if (y < (unsigned)width)
      wy[((int64_t)(row >> 7) * groups * 2 + pair) * kHM + (row & 127)] = (uint32_t)first_row[y] | (uint32_t)second_row[y] << 16;
  }
}

// Sums of the shares of a K loop, [split][128-row tile][group of 4 columns][128 rows][4], to rows of an output.
// A block takes 32 columns of a 128-row tile.
constexpr int kSumThreads = 256;
__global__ void __launch_bounds__(kSumThreads)
head_sum_kernel(HeadRows rows, int T, int online, int m_extent, int cols, const float* acc, int groups, int split, const uint32_t* wy,
                void* out, int64_t ld, int f32) {
  __shared__ float tile[kHM][33];
  pdl_launch_dependents();
  pdl_wait();
  const int n = *rows.n, m_rows = m_extent > 0 ? m_extent : n;
  const int m_tile = blockIdx.x, col0 = blockIdx.y * 32;
  if ((int64_t)m_tile * kHM >= m_rows) return;
  const int64_t tiles = (int64_t)((m_rows + 2 * kHM - 1) / (2 * kHM)) * 2;
  const float unit = wy == nullptr && n > 0 ? dz_unit(rows) : 1.f;
  constexpr int kEach = 8 * kHM / kSumThreads;
  float4 sums[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) sums[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int k = 0; k < split; ++k) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = e * kSumThreads + threadIdx.x, g = i / kHM, r = i % kHM;
      if (col0 + g * 4 < cols && m_tile * kHM + r < m_rows) {
        const float4 x = *reinterpret_cast<const float4*>(acc + (((k * tiles + m_tile) * groups + col0 / 4 + g) * kHM + r) * 4);
        sums[e].x += x.x; sums[e].y += x.y; sums[e].z += x.z; sums[e].w += x.w;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = e * kSumThreads + threadIdx.x, g = i / kHM, r = i % kHM, row = m_tile * kHM + r;
    float4 s = sums[e];
    if (col0 + g * 4 < cols && row < m_rows) {
      if (wy != nullptr) {
        const float2 f = row_factors(rows, row, online);
        const float up = target_factor(rows, row, online);
        const uint32_t* w = wy + ((int64_t)m_tile * groups * 2 + col0 / 2 + g * 2) * kHM + r;
        const uint32_t x = w[0], y = w[kHM];
        s.x = s.x * f.x * f.y - up * __uint_as_float(x << 16); s.y = s.y * f.x * f.y - up * __uint_as_float(x & 0xFFFF0000u);
        s.z = s.z * f.x * f.y - up * __uint_as_float(y << 16); s.w = s.w * f.x * f.y - up * __uint_as_float(y & 0xFFFF0000u);
      } else {
        s.x *= unit; s.y *= unit; s.z *= unit; s.w *= unit;
      }
    }
    tile[r][g * 4] = s.x; tile[r][g * 4 + 1] = s.y; tile[r][g * 4 + 2] = s.z; tile[r][g * 4 + 3] = s.w;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kHM * 32; i += kSumThreads) {
    const int r = i / 32, c = col0 + i % 32, row = m_tile * kHM + r;
    if (row >= m_rows || c >= cols) continue;
    const int64_t at = (int64_t)(m_extent > 0 || n == T ? row : rows.row[row]) * ld + c;
    if (f32) reinterpret_cast<float*>(out)[at] = tile[r][i % 32];
    else reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(tile[r][i % 32]);
  }
}

// ------------------------------------------------------------------------------------------------------ host: plan
// Columns of a pair's tile and shares of its K loop.  Cost of a K block, in SM clocks: its MMAs (two columns a clock), or its
// operands at the 47 bytes a clock that reach an SM's shared memory, whichever is longer; of a tile, its epilogue, which
// nothing covers; of a share of the K loop, the sums that it hands over.
struct HeadPlan { int tn, n_cols, split; };
HeadPlan head_plan(int m_rows, int cols, int n_kb, bool may_split, int most_tn, int step) {
  const long long m_pairs = ceil_div(m_rows, 2 * kHM);
  HeadPlan best{0, 0, 1};
  double best_cost = 0;
  for (int tn = most_tn; tn >= 64; tn -= step) {
    const int n_cols = ceil_div(cols, tn);
    const int wa = tn < 256 ? tn : 256, wb = tn - wa, boxes = (wa / 2 + 63) / 64 + (wb / 2 + 63) / 64;
    const double mma = 2.0 * tn, bytes = (16 + 8 * boxes) * 1024 / 47.0, block = mma > bytes ? mma : bytes;
    for (int split = 1; split <= (may_split ? 16 : 1); ++split) {
      const int per = ceil_div(n_kb, split);
      if (split > 1 && (per < 8 || (split - 1) * per >= n_kb)) break;
      const double waves = (double)((m_pairs * n_cols * split + kHPairs - 1) / kHPairs);
      // narrow tiles take turns in the tensor memory, so that one's epilogue runs under the next one's products
      const double epilogue = 1500.0 + 10.0 * tn, loop = per * block;
      double cost = tn <= 256 ? waves * (loop > epilogue ? loop : epilogue) + epilogue : waves * (loop + 0.6 * epilogue);
      // written and read once more at about 3 KB a clock by the whole GPU, and a launch
      if (split > 1) cost += 4000.0 + split * 8.0 * m_rows * cols / 3000.0;
      if (best.tn == 0 || cost < best_cost * 0.999) { best = HeadPlan{tn, n_cols, split}; best_cost = cost; }
    }
  }
  return best;
}

constexpr int kOneRowEach = 592;                        // rows up to which finishing takes a block a row: four blocks an SM
constexpr size_t kPieceBytes = (size_t)256 << 20;       // E or dZ of a piece of the vocabulary
constexpr int kPieceMin = 2048;
int head_piece(int rows_alloc, int V, int terms) {
  int64_t most = (int64_t)(kPieceBytes / 2 / terms) / rows_alloc / 512 * 512;
  if (most < kPieceMin) most = kPieceMin;
  const int pieces = (int)((V + most - 1) / most);
  return ceil_div(ceil_div(V, pieces), 512) * 512;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// How a call is carried out, and where its arrays lie in the workspace, whose size is that of the largest way.
struct HeadLayout {
  int rows_alloc, piece, pieces, terms;
  int few;                                              // logits (of STATS, or of EXP) by head_few_kernel
  int stats_pass;                                       // a product for lse alone comes first
  int logit_chunk;                                      // K blocks of the logits' products that are summed in the tensor memory, 0 = all
  int from_e;                                           // dX comes from E and the gathered columns of W, without dZ
  HeadPlan stats, dz, dx, dw;
  int64_t packed_ld;
  int dx_groups, dw_groups, above_words, chunks;
  size_t list, part, packed, above, above_ref, wy, dz_at, acc_x, acc_w, total;
};
constexpr int kLists = 10;
HeadLayout head_layout(int T, int d, int V, bool forward, bool want_dx, bool want_dw, bool f32) {
  HeadLayout l = {};
  l.rows_alloc = (int)(((int64_t)T + 255) / 256 * 256);
  const int terms = !f32 ? 1 : T <= kThreeTermRows ? 3 : 2;
  l.terms = terms;
  const bool grads = want_dx || want_dw;
  l.from_e = want_dx && !want_dw;
  l.stats_pass = forward && !l.from_e;
  l.few = T <= (l.from_e ? kFewExpRows : kFewRows);
  const int k_d = ceil_div(d, kHK), k_t = ceil_div(T, kHK);
  l.logit_chunk = (T <= kExactRows || d > kExactWidth || (grads && f32)) && k_d > kLogitChunk ? kLogitChunk : 0;
  const int most_tn = l.logit_chunk > 0 ? 256 : kHMaxTile;
  l.packed_ld = (d + 7) / 8 * 8;
  l.piece = grads ? head_piece(l.rows_alloc, V, terms) : 0;
  l.pieces = grads ? ceil_div(V, l.piece) : 0;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += align256(bytes); return here; };
  l.list = align256((size_t)l.rows_alloc * 4);
  take(256 + kLists * l.list);
  size_t parts = 0;
  if (l.stats_pass) {
    l.stats = l.few ? HeadPlan{few_columns(V), ceil_div(V, few_columns(V)), 1} : head_plan(T, V, k_d, false, most_tn, 32);
    parts = l.stats.n_cols;
  }
  if (grads) {
    l.dz = l.few && l.from_e ? HeadPlan{few_columns(l.piece), ceil_div(l.piece, few_columns(l.piece)), 1}
                             : head_plan(T, l.piece, k_d, false, most_tn, 64);
    if (l.from_e && forward) parts = l.dz.n_cols;
  }
  l.part = take(parts * 2 * l.rows_alloc * 8);
  l.packed = take((size_t)l.rows_alloc * l.packed_ld * 2);
  if (grads) {
    l.dz_at = take((size_t)l.rows_alloc * l.piece * terms * 2);
    if (want_dx) {
      l.dx = head_plan(T, d, l.piece / kHK * terms, true, kHMaxTile, 32);
      l.dx_groups = ceil_div(d, 4);
      // fp32 gradients pass through the sums at every chunk
      if (l.pieces > 1 || l.dx.split > 1 || terms > 1) l.acc_x = take((size_t)l.dx.split * l.rows_alloc * l.dx_groups * 16);
    }
    if (want_dw) {
      l.dw = head_plan(d, l.piece, k_t * terms, true, kHMaxTile, 32);
      l.dw_groups = l.piece / 4;
      if (l.dw.split > 1 || terms > 1) l.acc_w = take((size_t)l.dw.split * ceil_div(d, 2 * kHM) * 2 * kHM * l.dw_groups * 16);
    }
    if (l.from_e) {
      l.wy = take((size_t)l.rows_alloc * l.dx_groups * 8);
      l.chunks = l.few ? l.dz.n_cols : l.piece / 64;
      l.above_words = ceil_div(l.chunks, 32);
      l.above = take((size_t)l.rows_alloc * l.above_words * 4);
      l.above_ref = take((size_t)l.rows_alloc * l.chunks * 4);
    }
  }
  l.total = at;
  return l;
}

template <int kMode, bool kSums>
cudaError_t launch_head(const HeadMaps& maps, HeadParams p, int most_rows, bool chained, cudaStream_t st) {
  const int wa = p.tn < 256 ? p.tn : 256, wb = p.tn - wa;
  p.stage_bytes = kHLeft + ((wa / 2 + 63) / 64 + (wb / 2 + 63) / 64) * kHBox;
  p.stages = kHRing / p.stage_bytes < kHMaxStages ? kHRing / p.stage_bytes : kHMaxStages;
  static SharedMemoryGrant grant;
  cudaError_t e = grant(head_kernel<kMode, kSums>);
  if (e != cudaSuccess) return e;
  int dev = 0, sms = 0;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  const int64_t tiles = (int64_t)ceil_div(most_rows, 2 * kHM) * p.n_cols * p.split;
  int pairs = sms / 2 < kHPairs ? sms / 2 : kHPairs;
  if (tiles < pairs) pairs = (int)tiles;
  return launch_chained(chained, head_kernel<kMode, kSums>, dim3((unsigned)(2 * pairs)), dim3(kHThreads), kHSmem, st, maps, p);
}

// products whose tiles are logits
template <int kMode>
cudaError_t launch_logits(const HeadMaps& maps, const HeadParams& p, int T, bool chained, cudaStream_t st) {
  return p.chunk_kb > 0 ? launch_head<kMode, true>(maps, p, T, chained, st) : launch_head<kMode, false>(maps, p, T, chained, st);
}

bool bad_operand(const void* ptr, int64_t ld, int64_t cols, int64_t rows) {
  return !aligned16(ptr) || (rows > 1 && (ld < cols || ld % 8 != 0 || ld > ((int64_t)1 << 38)));
}

}  // namespace
}  // namespace cwl

extern "C" size_t cwl_head_loss_workspace_bytes(int32_t T, int32_t d, int32_t V, int32_t want_dx, int32_t want_dw) {
  using namespace cwl;
  if (T <= 0 || d <= 0 || V <= 0 || T > kHeadMaxRows || V > kHeadMaxRows || d > kHeadMaxWidth) return 0;
  // of the loss alone, too: a training loop's evaluation runs in the workspace of its steps
  size_t most = head_layout(T, d, V, true, false, false, false).total;
  for (int f32 = 0; f32 <= 1 && (want_dx != 0 || want_dw != 0); ++f32) {
    for (int forward = 0; forward <= 1; ++forward) {
      const size_t n = head_layout(T, d, V, forward != 0, want_dx != 0, want_dw != 0, f32 != 0).total;
      if (n > most) most = n;
    }
  }
  return most;
}

extern "C" cwl_status cwl_head_loss(const void* X, int64_t ldx, const void* W, int64_t ldw, int32_t T, int32_t d, int32_t V,
                                    const int32_t* targets, const float* weight, const float* dloss,
                                    float* loss, float* lse, void* dX, int64_t lddx, void* dW, int64_t lddw,
                                    cwl_dtype grad_dtype, void* workspace, size_t workspace_bytes,
                                    int32_t* status_word, void* stream) try {
  using namespace cwl;
  if (T < 0 || d <= 0 || V <= 0) return CWL_ERR_INVALID_ARG;
  if (grad_dtype != CWL_F32 && grad_dtype != CWL_BF16) return CWL_ERR_INVALID_ARG;
  if (T > kHeadMaxRows || V > kHeadMaxRows || d > kHeadMaxWidth) return CWL_ERR_UNSUPPORTED;
  const int es = grad_dtype == CWL_F32 ? 4 : 2;
  auto bad_grad = [&](const void* ptr, int64_t ld, int64_t cols, int64_t rows) {
    return ptr != nullptr && ((reinterpret_cast<uintptr_t>(ptr) % es) != 0 || (rows > 1 && ld < cols));
  };
  if (bad_grad(dX, lddx, d, T) || bad_grad(dW, lddw, V, d)) return CWL_ERR_SHAPE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {
    if (dW != nullptr) CWL_CUDA_TRY(cudaMemset2DAsync(dW, (size_t)(d > 1 ? lddw : V) * es, 0, (size_t)V * es, d, st));
    return CWL_OK;
  }
  if (X == nullptr || W == nullptr || targets == nullptr) return CWL_ERR_INVALID_ARG;
  if (loss == nullptr && dX == nullptr && dW == nullptr) return CWL_ERR_INVALID_ARG;
  if (loss == nullptr && lse == nullptr) return CWL_ERR_INVALID_ARG;      // a backward call reads it
  if (loss != nullptr && dloss != nullptr) return CWL_ERR_INVALID_ARG;    // an upstream gradient belongs to a backward call
  if (bad_operand(X, ldx, d, T) || bad_operand(W, ldw, V, d)) return CWL_ERR_SHAPE;
  const bool forward = loss != nullptr;
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
      workspace_bytes < cwl_head_loss_workspace_bytes(T, d, V, dX != nullptr, dW != nullptr))
    return CWL_ERR_WORKSPACE;
  // gradients are written while X and W are still being read
  const MatrixSpan x_at = matrix_span(X, ldx, T, d, 2), w_at = matrix_span(W, ldw, d, V, 2), dx_at = matrix_span(dX, lddx, T, d, es),
                   dw_at = matrix_span(dW, lddw, d, V, es);
  if (overlap(dx_at, x_at) || overlap(dx_at, w_at) || overlap(dw_at, x_at) || overlap(dw_at, w_at) || overlap(dx_at, dw_at)) return CWL_ERR_INVALID_ARG;
  const HeadLayout l = head_layout(T, d, V, forward, dX != nullptr, dW != nullptr, es == 4);
  const bool online = l.from_e && forward;
  // a sector of 32 bytes for each number of the targets' columns, or all of W
  const bool in_order = (int64_t)T * 32 > (int64_t)V * 2;

  uint8_t* ws = static_cast<uint8_t*>(workspace);
  auto list = [&](int i) { return reinterpret_cast<float*>(ws + 256 + i * l.list); };
  HeadRows rows = {};
  rows.n = reinterpret_cast<int*>(ws);
  rows.row = reinterpret_cast<int*>(list(0));
  rows.target = reinterpret_cast<int*>(list(1));
  rows.up = list(2); rows.lse = list(3); rows.z_target = list(4);
  rows.ref = list(5); rows.sum = list(6); rows.alpha = list(7); rows.scale = list(8); rows.of_target = list(9);
  static_assert(kLists == 10, "arrays of a number a row");
  rows.above = reinterpret_cast<unsigned*>(ws + l.above);
  rows.above_ref = reinterpret_cast<float*>(ws + l.above_ref);
  rows.above_words = l.above_words;
  rows.chunks = l.chunks;
  __nv_bfloat16* packed = reinterpret_cast<__nv_bfloat16*>(ws + l.packed);
  __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + l.dz_at);
  float2* part = reinterpret_cast<float2*>(ws + l.part);
  uint32_t* wy = l.from_e ? reinterpret_cast<uint32_t*>(ws + l.wy) : nullptr;
  const int64_t dz_ld = (int64_t)l.piece * l.terms;
  const bool chained = !stream_is_capturing(st);

  RowsParams r = {};
  r.X = static_cast<const __nv_bfloat16*>(X); r.ldx = ldx; r.T = T; r.d = d; r.V = V;
  r.W = static_cast<const __nv_bfloat16*>(W); r.ldw = ldw;
  r.targets = targets; r.weight = weight; r.dloss = dloss; r.lse_in = forward ? nullptr : lse;
  r.loss = loss; r.lse = forward ? lse : nullptr;
  r.dX = dX; r.lddx = lddx; r.dx_elem = es;
  r.packed = packed; r.packed_ld = l.packed_ld; r.rows = rows; r.backward = !forward; r.online = online; r.reference = in_order;
  r.status_word = status_word;
  int blocks = ceil_div(T, 8);
  if (blocks > 148) blocks = 148;
  r.per_block = ceil_div(T, blocks);
  // first of the call's launches: head_few_kernel reads W before its own wait on the strength of this one's
  CWL_CUDA_TRY(launch_chained(chained, head_rows_kernel, dim3((unsigned)blocks), dim3(kRowsThreads), 0, st, r));
  if (l.from_e) {
    const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(W);
    if (in_order) {
      const int parts = ceil_div(V, kOrderedColumns), columns = (ceil_div(V, parts) + 7) / 8 * 8;
      static SharedMemoryGrant grant;
      CWL_CUDA_TRY(grant(head_gather_ordered_kernel));
      CWL_CUDA_TRY(launch_chained(chained, head_gather_ordered_kernel, dim3((unsigned)ceil_div(d, 2), (unsigned)parts), dim3(kOrderedThreads),
                                  (size_t)columns * 4, st, rows, w, ldw, d, V, l.dx_groups, columns, wy));
    } else {
      CWL_CUDA_TRY(launch_chained(chained, head_gather_kernel, dim3((unsigned)T), dim3(kGatherThreads), 0, st, rows, r.X, ldx, w, ldw, d,
                                  l.dx_groups, online ? 1 : 0, wy));
    }
  }

  HeadParams p = {};
  p.rows = rows; p.T = T; p.rows_alloc = l.rows_alloc; p.split = 1; p.terms = 1;
  p.part = part;
  p.wait_limit_ns = training_wait_limit();
  p.withhold = training_withhold();
  p.status_word = status_word;
  HeadMaps logits, maps;
  const uint64_t ux = T > 1 ? ldx : l.packed_ld, uw = d > 1 ? ldw : (V + 7) / 8 * 8;
  if (!encode_map(&logits.a, X, d, T, ux, kHK, kHM) || !encode_map(&logits.a_packed, packed, d, l.rows_alloc, l.packed_ld, kHK, kHM) ||
      !encode_map(&logits.b, W, V, d, uw, 64, kHK))
    return CWL_ERR_CUDA;
  HeadMaps few = logits;
  if (l.few && (!encode_map(&few.a, X, d, T, ux, kHK, few_box(T)) || !encode_map(&few.a_packed, packed, d, l.rows_alloc, l.packed_ld, kHK, few_box(T))))
    return CWL_ERR_CUDA;

  if (l.stats_pass) {
    HeadParams q = p;
    q.n_extent = V; q.k_extent = d; q.tn = l.stats.tn; q.n_cols = l.stats.n_cols; q.kb_per_split = ceil_div(d, kHK); q.chunk_kb = l.logit_chunk;
    CWL_CUDA_TRY(l.few ? launch_few<HEAD_STATS>(few, q, T, chained, st) : launch_logits<HEAD_STATS>(logits, q, T, chained, st));
    const float2* parts = part;
    const int n_part = (l.few ? 1 : 2) * l.stats.n_cols;
    CWL_CUDA_TRY(T <= kOneRowEach ? launch_chained(chained, head_finish_kernel<1>, dim3((unsigned)T), dim3(kFinishThreads), 0, st, rows, parts, n_part,
                                                   l.rows_alloc, weight, loss, lse)
                                  : launch_chained(chained, head_finish_kernel<32>, dim3((unsigned)ceil_div(T, 32)), dim3(kFinishThreads), 0, st, rows,
                                                   parts, n_part, l.rows_alloc, weight, loss, lse));
  }
  for (int piece = 0; piece < l.pieces; ++piece) {
    const int first = piece * l.piece, width = V - first < l.piece ? V - first : l.piece;
    const bool last = piece + 1 == l.pieces;
    HeadParams q = p;
    q.n_extent = width; q.n_first = first; q.k_extent = d; q.kb_per_split = ceil_div(d, kHK); q.chunk_kb = l.logit_chunk;
    q.tn = l.dz.tn; q.n_cols = ceil_div(width, q.tn);
    q.dz = dz; q.dz_ld = dz_ld; q.terms = l.terms; q.term_at = l.piece; q.online = online;
    if (l.from_e) {
      CWL_CUDA_TRY(l.few ? launch_few<HEAD_EXP>(few, q, T, chained, st) : launch_logits<HEAD_EXP>(logits, q, T, chained, st));
      if (online) {
        MergeParams m = {};
        m.rows = rows; m.part = part; m.n_part = l.few ? q.n_cols : 2 * q.n_cols; m.chunk_cols = l.few ? q.tn : 64; m.rows_alloc = l.rows_alloc; m.last = last;
        m.dz = dz; m.dz_ld = dz_ld; m.width = width; m.terms = l.terms; m.term_at = l.piece;
        m.weight = weight; m.loss = loss; m.lse = lse;
        CWL_CUDA_TRY(T <= kOneRowEach ? launch_chained(chained, head_merge_kernel<1>, dim3((unsigned)T), dim3(kFinishThreads), 0, st, m)
                                      : launch_chained(chained, head_merge_kernel<32>, dim3((unsigned)ceil_div(T, 32)), dim3(kFinishThreads), 0, st, m));
      }
    } else {
      q.online = forward;
      CWL_CUDA_TRY(launch_logits<HEAD_DZ>(logits, q, T, chained, st));
    }
    // where E / dZ is several numbers, the last block of each is stored whole, and DX reads no further
    const int64_t stored = (int64_t)(l.terms - 1) * l.piece + width;
    if (dX != nullptr) {
      q = p;
      q.n_extent = d; q.k_extent = width; q.k_first = first; q.terms = l.terms; q.term_at = l.piece;
      q.chunk_kb = l.terms > 1 ? kChunkBlocks / l.terms : 0;
      q.tn = l.dx.tn; q.n_cols = l.dx.n_cols; q.split = l.dx.split; q.kb_per_split = ceil_div(ceil_div(width, kHK), q.split);
      q.acc = reinterpret_cast<float*>(ws + l.acc_x); q.acc_groups = l.dx_groups;
      q.acc_in = piece > 0; q.acc_out = q.split > 1 || !last;
      q.wy = wy; q.online = online;
      q.out = dX; q.out_ld = lddx; q.out_f32 = es == 4;
      q.out_vec = aligned16(dX) && (T == 1 || lddx * es % 16 == 0);
      if (!encode_map(&maps.a, dz, stored, l.rows_alloc, dz_ld, kHK, kHM) || !encode_map(&maps.b, W, V, d, uw, kHK, 64)) return CWL_ERR_CUDA;
      maps.a_packed = maps.a;
      CWL_CUDA_TRY((launch_head<HEAD_DX, false>(maps, q, T, chained, st)));
      if (last && q.split > 1)
        CWL_CUDA_TRY(launch_chained(chained, head_sum_kernel, dim3((unsigned)ceil_div(T, kHM), (unsigned)ceil_div(d, 32)), dim3(kSumThreads), 0, st,
                                    rows, T, online ? 1 : 0, 0, d, static_cast<const float*>(q.acc), q.acc_groups, q.split, static_cast<const uint32_t*>(wy), dX, lddx,
                                    q.out_f32));
    }
    if (dW != nullptr) {
      q = p;
      q.m_extent = d; q.n_extent = width; q.terms = l.terms; q.term_at = l.piece;
      q.chunk_kb = l.terms > 1 ? kChunkBlocks / l.terms : 0;
      q.tn = l.dw.tn; q.n_cols = ceil_div(width, q.tn); q.split = l.dw.split;
      q.acc = reinterpret_cast<float*>(ws + l.acc_w); q.acc_groups = l.dw_groups; q.acc_out = q.split > 1;
      q.out = static_cast<uint8_t*>(dW) + (size_t)first * es; q.out_ld = lddw; q.out_f32 = es == 4;
      q.out_vec = aligned16(q.out) && (d == 1 || lddw * es % 16 == 0);
      if (!encode_map(&maps.a, X, d, T, ux, 64, kHK) || !encode_map(&maps.a_packed, packed, d, l.rows_alloc, l.packed_ld, 64, kHK) ||
          !encode_map(&maps.b, dz, stored, l.rows_alloc, dz_ld, 64, kHK))
        return CWL_ERR_CUDA;
      CWL_CUDA_TRY((launch_head<HEAD_DW, false>(maps, q, d, chained, st)));
      if (q.split > 1)
        CWL_CUDA_TRY(launch_chained(chained, head_sum_kernel, dim3((unsigned)ceil_div(d, kHM), (unsigned)ceil_div(width, 32)), dim3(kSumThreads), 0, st,
                                    rows, T, 0, d, width, static_cast<const float*>(q.acc), q.acc_groups, q.split, static_cast<const uint32_t*>(nullptr), q.out,
                                    lddw, q.out_f32));
    }
  }
  return CWL_OK;
} catch (...) {
  return CWL_ERR_CUDA;                                   // nothing may leave a C entry
}

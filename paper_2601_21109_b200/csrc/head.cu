// cwl_head_loss: softmax cross entropy of a head's projection over a large vocabulary, with its gradients, logits not kept.
//
//   z = X W,   lse_t = ln sum_v e^(z_tv),   loss_t = w_t (lse_t - z_t,y),   dZ = up (softmax(z) - onehot(y)),
//   dX = dZ W^T,   dW = X^T dZ
//
// Rows without a target or of weight 0 cost nothing: the first kernel lists the others and packs their activations
// together (or, where every row counts, leaves X as it is), and all products run over the packed rows.  Then, all of them
// tensor-core products of one persistent kernel that differ in which way their operands lie and in what is done with a
// finished tile:
//   STATS  z tile -> (max, sum of exponentials) of its columns per row, and the target's logit
//   DZ     z tile of a piece of the vocabulary again -> dZ in bf16, to a workspace
//   DX     dZ piece times W^T; sums over the pieces are kept in fp32
//   DW     X^T times dZ piece: whole columns of dW
#include "cluster.cuh"
#include "cwl_common.cuh"
#include "pair_mma.cuh"

namespace cwl {
namespace {

constexpr int kHM = 128;                          // rows per CTA tile = TMEM lanes
constexpr int kHK = 64;                           // K elements per stage = one 128-byte swizzle row of bf16
constexpr int kHStages = 4;
constexpr int kHBox = 64 * kHK * 2;               // a box of 64 columns (or rows) x 64 K elements: 8 KB
constexpr int kHLeft = kHM * kHK * 2;             // 16 KB of the left operand a stage
constexpr int kHMaxTile = 512;                    // columns of a pair's tile = fp32 columns of tensor memory
constexpr int kHStage = kHLeft + 4 * kHBox;       // 48 KB
constexpr int kHRing = kHStages * kHStage;
constexpr int kHOutBuf = 4096;                    // staging of a warp: 32 rows of 128 bytes
constexpr int kHEpiWarps = 8;
constexpr int kHThreads = 64 + 32 * kHEpiWarps;   // warp 0: TMA, warp 1: MMA and tensor memory, warps 2..9: epilogue
constexpr int kHBars = 8 * (2 * kHStages + 2);
constexpr size_t kHSmem = 1024 + kHRing + kHEpiWarps * kHOutBuf + kHBars + 32;
constexpr int kHPairs = 74;                       // CTA pairs that schedules are made for (a B200 holds 74)
constexpr int kHRaster = 16;                      // row tiles whose columns are walked together, so that they share W in L2
constexpr int kHeadMaxRows = 1 << 24, kHeadMaxWidth = 1 << 20;   // T and V, d
constexpr float kLog2e = 1.4426950408889634f;

enum : int { HEAD_STATS = 0, HEAD_DZ = 1, HEAD_DX = 2, HEAD_DW = 3 };

struct HeadRows {                                 // the packed rows, written by head_rows_kernel
  int* n;                                         // how many
  int* row;                                       // which row of the call each is
  int* target;
  float* up;                                      // weight times upstream gradient
  float* lse;
  float* z_target;
};

struct HeadMaps { CUtensorMap a, a_packed, b; };  // a: of X itself (every row counts), a_packed: of the packed rows

struct HeadParams {
  HeadRows rows;
  int T;
  int m_extent;                                   // rows of the product: 0 = the packed rows, else this many (DW: d)
  int n_extent, n_first;                          // columns of the product; where they start in the right operand / output
  int k_extent, k_first;                          // K loop: 0 = the packed rows (DW); where it starts in the right operand (DX)
  int tn, n_cols;                                 // columns of a tile, tiles beside one another
  int split, kb_per_split;                        // shares of the K loop
  int rows_alloc;                                 // rows of the workspace arrays
  float2* part;                                   // STATS: [2 n_cols][rows_alloc] (max, sum)
  __nv_bfloat16* dz; int64_t dz_ld;               // DZ
  float* acc; int acc_groups;                     // fp32 sums [split][128-row tile][group of 4 columns][128 rows][4]
  int acc_in, acc_out;                            // DX, DW: add what is there; leave the sum there instead of in `out`
  void* out; int64_t out_ld; int out_f32, out_vec;
  unsigned long long wait_limit_ns;
  int withhold;
  int32_t* status_word;
};

// A tile of the launch: raster groups of kHRaster row tiles, row tile fastest inside a group.
struct HeadTile { int m_pair, col, split; };
__device__ __forceinline__ bool head_tile(int i, int n_m_pairs, const HeadParams& p, HeadTile& t) {
  const int64_t total = (int64_t)n_m_pairs * p.n_cols * p.split;
  int64_t at = (int64_t)(blockIdx.x >> 1) + (int64_t)i * (gridDim.x >> 1);
  if (at >= total) return false;
  t.split = (int)(at % p.split);
  at /= p.split;
  const int64_t per_group = (int64_t)kHRaster * p.n_cols;
  const int group = (int)(at / per_group), within = (int)(at - (int64_t)group * per_group);
  const int first = group * kHRaster, size = min(kHRaster, n_m_pairs - first);
  t.m_pair = first + within % size;
  t.col = within / size;
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

template <int kMode>
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
  auto empty_bar = [&](int s) { return bars + 8u * (kHStages + s); };
  const uint32_t acc_full = bars + 8u * (2 * kHStages), acc_empty = acc_full + 8u;
  uint8_t* misc = base_ptr + kHRing + kHEpiWarps * kHOutBuf + kHBars;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);     // its wait limit sits at misc + 16
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();

  if (threadIdx.x == 0) {
    // full: armed by the leader's producer, completed by both CTAs' bytes (only the leader's copy is used); empty, acc_full:
    // one arrival, from the leader's commit, in both CTAs; acc_empty: an arrival per epilogue warp of both, on the leader's
    for (int s = 0; s < kHStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, 2 * kHEpiWarps);
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
  const int n_m_pairs = (m_rows + 2 * kHM - 1) / (2 * kHM);
  const int n_kb = ((p.k_extent > 0 ? p.k_extent : n) + kHK - 1) / kHK;
  const int kb_per_split = p.k_extent > 0 ? p.kb_per_split : (n_kb + p.split - 1) / p.split;
  const CUtensorMap* map_a = kMode != HEAD_DX && n < p.T ? &maps.a_packed : &maps.a;

  if (warp == 0) {
    // ------------------------------------------------------------------------------------- producer (both CTAs)
    uint32_t issued = 0, s = 0, ph = 0;
    const uint32_t leader_full0 = peer_shared(full_bar(0), 0);
    bool ok = true;
    HeadTile t;
    for (int i = 0; ok && head_tile(i, n_m_pairs, p, t); ++i) {
      const int n0 = t.col * p.tn, wt = min(p.tn, (p.n_extent - n0 + 31) & ~31);
      const int wa = min(wt, 256), wb = wt - wa;
      const int ca = wa >> 1, cb = wb >> 1, boxes_a = (ca + 63) >> 6, boxes = boxes_a + ((cb + 63) >> 6);
      const uint32_t tx = 2u * (kHLeft + boxes * kHBox);
      // lane 0: the left operand; lanes 1..boxes: a box of the right operand each
      const int bi = lane - 1;
      const bool has_box = bi >= 0 && bi < boxes;
      const int at = p.n_first + n0 + (bi < boxes_a ? (int)rank * ca + bi * 64 : wa + (int)rank * cb + (bi - boxes_a) * 64);
      const int m0 = (t.m_pair * 2 + (int)rank) * kHM;
      const int kb0 = t.split * kb_per_split;
      const int n_blk = min(kb_per_split, n_kb - kb0);
      for (int b = 0; b < n_blk; ++b) {
        if (CWL_WITHHELD(p) && i == 0 && b == n_blk - 1) { ok = false; break; }
        const bool step_ok = mbar_wait(empty_bar(s), ph ^ 1u, abort_flag);
        if (!__all_sync(0xffffffffu, step_ok)) { ok = false; break; }
        const int k = (kb0 + b) * kHK;
        const uint32_t sa = base + s * kHStage, sb = sa + kHLeft, full = leader_full0 + 8u * s;
        if (lane == 0) {
          if (rank == 0) mbar_expect_tx(full_bar(s), tx);
          if (kLeftMn) {
            pair_load_2d(sa, map_a, full, m0, k);
            pair_load_2d(sa + kHBox, map_a, full, m0 + 64, k);
          } else {
            pair_load_2d(sa, map_a, full, k, m0);
          }
        } else if (has_box) {
          if (kRightMn) pair_load_2d(sb + bi * kHBox, &maps.b, full, at, k);
          else pair_load_2d(sb + bi * kHBox, &maps.b, full, p.k_first + k, at);
        }
        ++issued;
        if (++s == kHStages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok && rank == 0 && lane == 0) {
      // copies already issued get a bounded chance to land before the CTA leaves
      for (uint32_t back = 1; back <= (uint32_t)kHStages && back <= issued; ++back) {
        const uint32_t j = issued - back;
        const unsigned long long t0 = global_timer();
        while (!mbar_try_wait(full_bar(j % kHStages), (j / kHStages) & 1u) && global_timer() - t0 < p.wait_limit_ns) {}
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
      HeadTile t;
      for (int i = 0; ok && head_tile(i, n_m_pairs, p, t); ++i) {
        const int n0 = t.col * p.tn, wt = min(p.tn, (p.n_extent - n0 + 31) & ~31);
        const int wa = min(wt, 256), wb = wt - wa;
        const uint32_t idesc_a = pair_idesc(wa, kLeftMn, kRightMn), idesc_b = pair_idesc(wb > 0 ? wb : 32, kLeftMn, kRightMn);
        const uint64_t second = (uint64_t)((((wa >> 1) + 63) >> 6) * kHBox) >> 4;
        const int kb0 = t.split * kb_per_split, n_blk = min(kb_per_split, n_kb - kb0);
        if (n_blk <= 0) continue;                 // nothing to add up: the epilogue takes zeros
        if (!mbar_wait(acc_empty, (local & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        for (int b = 0; b < n_blk; ++b) {
          if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t da = desc_a + (uint64_t)((s * kHStage) >> 4), db = desc_b + (uint64_t)((s * kHStage) >> 4);
#pragma unroll
          for (int kk = 0; kk < kHK / 16; ++kk) {
            pair_mma_bf16(tmem, da + kk * step_a, db + kk * step_b, idesc_a, (b | kk) ? 1u : 0u);
            if (wb > 0) pair_mma_bf16(tmem + 256, da + kk * step_a, db + second + kk * step_b, idesc_b, (b | kk) ? 1u : 0u);
          }
          pair_commit(empty_bar(s));
          if (++s == kHStages) { s = 0; ph ^= 1u; }
        }
        if (ok) pair_commit(acc_full);
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
    const uint32_t leader_empty = peer_shared(acc_empty, 0);
    const uint32_t buf = out_bufs + (uint32_t)(warp - 2) * kHOutBuf;
    uint32_t local = 0;
    HeadTile t;
    for (int i = 0; head_tile(i, n_m_pairs, p, t); ++i) {
      const int n0 = t.col * p.tn, cols = min(p.tn, p.n_extent - n0);
      const int m_tile = t.m_pair * 2 + (int)rank, row0 = m_tile * kHM + quad * 32, row = row0 + lane;
      const bool live = row < m_rows;
      const bool any = min(kb_per_split, n_kb - t.split * kb_per_split) > 0;
      if (any) {
        if (!__all_sync(0xffffffffu, mbar_wait(acc_full, local & 1u, abort_flag))) break;
        tc_fence_after();
        ++local;
      }
      const uint32_t t_row = tmem + ((uint32_t)(quad * 32) << 16);
      if (kMode == HEAD_STATS) {
        const int y = live ? p.rows.target[row] - (p.n_first + n0) : -1;
        float m = -INFINITY, sum = 0.f;
#pragma unroll 1
        for (int c = chalf * 32; c < cols; c += 64) {
          float v[32];
          head_columns(t_row + c, v);
          const int left = cols - c;
          if (left < 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = j < left ? v[j] : -INFINITY;
          }
          float top = m;
#pragma unroll
          for (int j = 0; j < 32; ++j) top = fmaxf(top, v[j]);
          const float ref = top == -INFINITY ? 0.f : top * kLog2e;
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < 32; ++j) part += exp2_fast(fmaf(v[j], kLog2e, -ref));
          sum = sum * exp2_fast(fmaf(m, kLog2e, -ref)) + part;
          m = top;
          if ((unsigned)(y - c) < 32u) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j == y - c) p.rows.z_target[row] = v[j];
          }
        }
        if (live) p.part[(int64_t)(t.col * 2 + chalf) * p.rows_alloc + row] = make_float2(m, sum);
      } else if (kMode == HEAD_DZ) {
        const float up = live ? p.rows.up[row] : 0.f;
        const float ref = live ? p.rows.lse[row] * kLog2e : 0.f;
        const int y = live ? p.rows.target[row] - (p.n_first + n0) : -1;
#pragma unroll 1
        for (int c = chalf * 64; c < cols; c += 128) {
          __syncwarp();                           // every lane has read the chunk before back
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v[32];
            head_columns(t_row + c + h * 32, v);
            const int left = cols - c - h * 32, mine = y - c - h * 32;
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = exp2_fast(fmaf(v[j], kLog2e, -ref));
            if ((unsigned)mine < 32u) {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] -= j == mine ? 1.f : 0.f;
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = live && j < left ? v[j] * up : 0.f;
            stage_bf16(buf, lane, h, v);
          }
          __syncwarp();
          uint8_t* first = reinterpret_cast<uint8_t*>(p.dz + (int64_t)row0 * p.dz_ld + n0 + c);
          store_staged(buf, lane, ((cols - c) * 2 + 15) & ~15, 1, 2, [&](int r) { return first + (int64_t)r * p.dz_ld * 2; });
        }
      } else {
        const int64_t tiles = (int64_t)n_m_pairs * 2;
        float* sums = p.acc + ((((int64_t)t.split * tiles + m_tile) * p.acc_groups + n0 / 4) * kHM + quad * 32 + lane) * 4;
        // where this warp's rows go: rows of the call for DX, columns of X for DW
        const int mine = !live ? -1 : kMode == HEAD_DX && n < p.T ? p.rows.row[row] : row;
        const int chunk = p.acc_out || p.out_f32 ? 32 : 64;
#pragma unroll 1
        for (int c = chalf * chunk; c < cols; c += 2 * chunk) {
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
            if (p.acc_in) {
#pragma unroll
              for (int g = 0; g < 8; ++g) {
                if (cc + g * 4 < cols) {
                  const float4 x = *reinterpret_cast<const float4*>(sums + (int64_t)(cc / 4 + g) * kHM * 4);
                  v[g * 4] += x.x; v[g * 4 + 1] += x.y; v[g * 4 + 2] += x.z; v[g * 4 + 3] += x.w;
                }
              }
            }
            if (p.acc_out) {
#pragma unroll
              for (int g = 0; g < 8; ++g)
                if (cc + g * 4 < cols)
                  *reinterpret_cast<float4*>(sums + (int64_t)(cc / 4 + g) * kHM * 4) = make_float4(v[g * 4], v[g * 4 + 1], v[g * 4 + 2], v[g * 4 + 3]);
            } else if (p.out_f32) {
              stage_f32(buf, lane, v);
            } else {
              stage_bf16(buf, lane, h, v);
            }
          }
          if (!p.acc_out) {
            __syncwarp();
            const int es = p.out_f32 ? 4 : 2;
            const int64_t col = (kMode == HEAD_DW ? p.n_first : 0) + n0 + c;
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
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_in_cluster(leader_empty);
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

// ------------------------------------------------------------------------------------------------ rows that count
struct RowsParams {
  const __nv_bfloat16* X; int64_t ldx;
  int T, d, V;
  const int32_t* targets; const float* weight; const float* dloss; const float* lse_in;
  float* loss; float* lse;
  void* dX; int64_t lddx; int dx_elem;
  __nv_bfloat16* packed; int64_t packed_ld;
  HeadRows rows;
  int per_block, backward;
  int32_t* status_word;
};

constexpr int kRowsThreads = 256;

__device__ __forceinline__ float row_up(const RowsParams& p, int t) {
  float up = p.weight != nullptr ? p.weight[t] : 1.f;
  if (p.dloss != nullptr) up *= p.dloss[t];
  return up;
}
// a row counts if it has a target and its loss or, in a backward call, its gradient is not 0 whatever the logits are
__device__ __forceinline__ bool row_counts(const RowsParams& p, int t) {
  const int y = p.targets[t];
  if (y < 0 || y >= p.V) return false;
  return (p.backward ? row_up(p, t) : p.weight != nullptr ? p.weight[t] : 1.f) != 0.f;
}

// Lists the rows that count, packs their activations where some do not, and writes the outputs of those that do not.
// Every block counts all rows before its own itself (two words a row from L2), so one launch does it.
__global__ void __launch_bounds__(kRowsThreads) head_rows_kernel(const RowsParams p) {
  __shared__ int sums[2][kRowsThreads / 32];
  __shared__ int counts[kRowsThreads];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t first64 = (int64_t)blockIdx.x * p.per_block;
  const int first = (int)(first64 < p.T ? first64 : p.T);
  const int last = (int)(first64 + p.per_block < p.T ? first64 + p.per_block : p.T);
  int before = 0, total = 0;
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
      if (p.lse_in != nullptr) p.rows.lse[at] = p.lse_in[t];
    } else if (in) {
      const bool bad = p.targets[t] >= p.V;
      if (bad) flag_status(p.status_word, CWL_ERR_INVALID_ARG);
      const float v = bad ? NAN : 0.f;
      if (p.loss != nullptr) p.loss[t] = v;
      if (p.lse != nullptr) p.lse[t] = v;
    }
    __syncthreads();
    // a warp a row: into the packed activations, or zeros into its gradient
    const int rows_here = (int)(last - t0 < kRowsThreads ? last - t0 : kRowsThreads);
    for (int r = warp; r < rows_here; r += kRowsThreads / 32) {
      const int to = counts[r];
      if (to >= 0 && total < p.T) {
        const __nv_bfloat16* from = p.X + (t0 + r) * p.ldx;
        __nv_bfloat16* out = p.packed + (int64_t)to * p.packed_ld;
        for (int j = lane; j < p.d / 8; j += 32) reinterpret_cast<uint4*>(out)[j] = reinterpret_cast<const uint4*>(from)[j];
        for (int j = p.d / 8 * 8 + lane; j < p.d; j += 32) out[j] = from[j];
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

// Log-sum-exp and loss of every row that counts, from the tiles' maxima and sums.  32 rows a block, eight threads a row.
constexpr int kFinishThreads = 256;
__global__ void __launch_bounds__(kFinishThreads)
head_finish_kernel(HeadRows rows, const float2* part, int n_part, int rows_alloc, const float* weight, float* loss, float* lse) {
  __shared__ float2 met[kFinishThreads];
  pdl_launch_dependents();
  pdl_wait();
  const int n = *rows.n, lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * 32 + lane;
  if ((int64_t)blockIdx.x * 32 >= n) return;
  float m = -INFINITY, s = 0.f;
  if (row < n) {
    for (int c = slice; c < n_part; c += kFinishThreads / 32) {
      const float2 x = part[(int64_t)c * rows_alloc + row];
      const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
      s = s * exp2_fast((m - ref) * kLog2e) + x.y * exp2_fast((x.x - ref) * kLog2e);
      m = top;
    }
  }
  met[threadIdx.x] = make_float2(m, s);
  __syncthreads();
  if (slice == 0 && row < n) {
    for (int k = 1; k < kFinishThreads / 32; ++k) {
      const float2 x = met[k * 32 + lane];
      const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
      s = s * exp2_fast((m - ref) * kLog2e) + x.y * exp2_fast((x.x - ref) * kLog2e);
      m = top;
    }
    const float l = m + logf(s);
    const int t = rows.row[row];
    rows.lse[row] = l;
    if (lse != nullptr) lse[t] = l;
    if (loss != nullptr) loss[t] = (weight != nullptr ? weight[t] : 1.f) * (l - rows.z_target[row]);
  }
}

// Sums of the shares of a K loop, [split][128-row tile][group of 4 columns][128 rows][4], to rows of an output.
// A block takes 32 columns of a 128-row tile.
constexpr int kSumThreads = 256;
__global__ void __launch_bounds__(kSumThreads)
head_sum_kernel(HeadRows rows, int T, int m_extent, int cols, const float* acc, int groups, int split,
                void* out, int64_t ld, int f32, int vec) {
  __shared__ float tile[kHM][33];
  pdl_launch_dependents();
  pdl_wait();
  const int n = *rows.n, m_rows = m_extent > 0 ? m_extent : n;
  const int m_tile = blockIdx.x, col0 = blockIdx.y * 32;
  if ((int64_t)m_tile * kHM >= m_rows) return;
  const int64_t tiles = (int64_t)((m_rows + 2 * kHM - 1) / (2 * kHM)) * 2;
  for (int i = threadIdx.x; i < 8 * kHM; i += kSumThreads) {
    const int g = i / kHM, r = i % kHM;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col0 + g * 4 < cols) {
      for (int k = 0; k < split; ++k) {
        const float4 x = *reinterpret_cast<const float4*>(acc + (((k * tiles + m_tile) * groups + col0 / 4 + g) * kHM + r) * 4);
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
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
HeadPlan head_plan(int m_rows, int cols, int n_kb, bool may_split) {
  const long long m_pairs = ceil_div(m_rows, 2 * kHM);
  HeadPlan best{0, 0, 1};
  double best_cost = 0;
  for (int tn = kHMaxTile; tn >= 64; tn -= 32) {
    const int n_cols = ceil_div(cols, tn);
    const int wa = tn < 256 ? tn : 256, wb = tn - wa, boxes = (wa / 2 + 63) / 64 + (wb / 2 + 63) / 64;
    const double mma = 2.0 * tn, bytes = (16 + 8 * boxes) * 1024 / 47.0, block = mma > bytes ? mma : bytes;
    for (int split = 1; split <= (may_split ? 16 : 1); ++split) {
      const int per = ceil_div(n_kb, split);
      if (split > 1 && (per < 8 || (split - 1) * per >= n_kb)) break;
      const double waves = (double)((m_pairs * n_cols * split + kHPairs - 1) / kHPairs);
      double cost = waves * (per * block + 1500.0 + 10.0 * tn);
      // written and read once more at about 3 KB a clock by the whole GPU, and a launch
      if (split > 1) cost += 4000.0 + split * 8.0 * m_rows * cols / 3000.0;
      if (best.tn == 0 || cost < best_cost * 0.999) { best = HeadPlan{tn, n_cols, split}; best_cost = cost; }
    }
  }
  return best;
}

constexpr size_t kPieceBytes = (size_t)256 << 20;       // dZ of a piece of the vocabulary
constexpr int kPieceMin = 2048;
int head_piece(int rows_alloc, int V) {
  int64_t most = (int64_t)(kPieceBytes / 2) / rows_alloc / 512 * 512;
  if (most < kPieceMin) most = kPieceMin;
  const int pieces = (int)((V + most - 1) / most);
  return ceil_div(ceil_div(V, pieces), 512) * 512;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

struct HeadLayout {
  int rows_alloc, piece, pieces;
  HeadPlan stats, dz, dx, dw;
  int64_t packed_ld;
  int dx_groups, dw_groups;
  size_t info, part, packed, dz_at, acc_x, acc_w, total;
};
HeadLayout head_layout(int T, int d, int V, bool want_loss, bool want_dx, bool want_dw) {
  HeadLayout l = {};
  l.rows_alloc = (int)(((int64_t)T + 255) / 256 * 256);
  const bool grads = want_dx || want_dw;
  const int k_d = ceil_div(d, kHK), k_t = ceil_div(T, kHK);
  l.packed_ld = (d + 7) / 8 * 8;
  l.piece = grads ? head_piece(l.rows_alloc, V) : 0;
  l.pieces = grads ? ceil_div(V, l.piece) : 0;
  l.stats = head_plan(T, V, k_d, false);
  size_t at = 0;
  l.info = at;
  at += 256 + 5 * align256((size_t)l.rows_alloc * 4);
  l.part = at;
  if (want_loss) at += align256((size_t)2 * l.stats.n_cols * l.rows_alloc * 8);
  l.packed = at;
  at += align256((size_t)l.rows_alloc * l.packed_ld * 2);
  if (grads) {
    l.dz = head_plan(T, l.piece, k_d, false);
    l.dz_at = at;
    at += align256((size_t)l.rows_alloc * l.piece * 2);
    if (want_dx) {
      l.dx = head_plan(T, d, l.piece / kHK, true);
      l.dx_groups = ceil_div(d, 4);
      l.acc_x = at;
      if (l.pieces > 1 || l.dx.split > 1) at += (size_t)l.dx.split * l.rows_alloc * l.dx_groups * 16;
    }
    if (want_dw) {
      l.dw = head_plan(d, l.piece, k_t, true);
      l.dw_groups = l.piece / 4;
      l.acc_w = at;
      if (l.dw.split > 1) at += (size_t)l.dw.split * ceil_div(d, 2 * kHM) * 2 * kHM * l.dw_groups * 16;
    }
  }
  l.total = align256(at);
  return l;
}

template <int kMode>
cudaError_t launch_head(const HeadMaps& maps, const HeadParams& p, int most_rows, bool chained, cudaStream_t st) {
  static SharedMemoryGrant grant;
  cudaError_t e = grant(head_kernel<kMode>);
  if (e != cudaSuccess) return e;
  int dev = 0, sms = 0;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  const int64_t tiles = (int64_t)ceil_div(most_rows, 2 * kHM) * p.n_cols * p.split;
  int pairs = sms / 2 < kHPairs ? sms / 2 : kHPairs;
  if (tiles < pairs) pairs = (int)tiles;
  return launch_chained(chained, head_kernel<kMode>, dim3((unsigned)(2 * pairs)), dim3(kHThreads), kHSmem, st, maps, p);
}

bool bad_operand(const void* ptr, int64_t ld, int64_t cols, int64_t rows) {
  return !aligned16(ptr) || (rows > 1 && (ld < cols || ld % 8 != 0 || ld > ((int64_t)1 << 38)));
}

}  // namespace
}  // namespace cwl

extern "C" size_t cwl_head_loss_workspace_bytes(int32_t T, int32_t d, int32_t V, int32_t want_dx, int32_t want_dw) {
  using namespace cwl;
  if (T <= 0 || d <= 0 || V <= 0 || T > kHeadMaxRows || V > kHeadMaxRows || d > kHeadMaxWidth) return 0;
  return head_layout(T, d, V, true, want_dx != 0, want_dw != 0).total;
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
  if (loss == nullptr && dX == nullptr && dW == nullptr) return CWL_ERR_INVALID_ARG;
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
  if (loss == nullptr && lse == nullptr) return CWL_ERR_INVALID_ARG;      // a backward call reads it
  if (loss != nullptr && dloss != nullptr) return CWL_ERR_INVALID_ARG;    // an upstream gradient belongs to a backward call
  if (bad_operand(X, ldx, d, T) || bad_operand(W, ldw, V, d)) return CWL_ERR_SHAPE;
  const HeadLayout l = head_layout(T, d, V, true, dX != nullptr, dW != nullptr);
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < l.total)
    return CWL_ERR_WORKSPACE;

  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const size_t list = align256((size_t)l.rows_alloc * 4);
  HeadRows rows;
  rows.n = reinterpret_cast<int*>(ws + l.info);
  rows.row = reinterpret_cast<int*>(ws + l.info + 256);
  rows.target = reinterpret_cast<int*>(ws + l.info + 256 + list);
  rows.up = reinterpret_cast<float*>(ws + l.info + 256 + 2 * list);
  rows.lse = reinterpret_cast<float*>(ws + l.info + 256 + 3 * list);
  rows.z_target = reinterpret_cast<float*>(ws + l.info + 256 + 4 * list);
  __nv_bfloat16* packed = reinterpret_cast<__nv_bfloat16*>(ws + l.packed);
  __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + l.dz_at);
  const bool chained = !stream_is_capturing(st);

  RowsParams r = {};
  r.X = static_cast<const __nv_bfloat16*>(X); r.ldx = ldx; r.T = T; r.d = d; r.V = V;
  r.targets = targets; r.weight = weight; r.dloss = dloss; r.lse_in = loss == nullptr ? lse : nullptr;
  r.loss = loss; r.lse = loss != nullptr ? lse : nullptr;
  r.dX = dX; r.lddx = lddx; r.dx_elem = es;
  r.packed = packed; r.packed_ld = l.packed_ld; r.rows = rows; r.backward = loss == nullptr;
  r.status_word = status_word;
  int blocks = ceil_div(T, 16);
  if (blocks > 592) blocks = 592;
  r.per_block = ceil_div(T, blocks);
  CWL_CUDA_TRY(launch_chained(chained, head_rows_kernel, dim3((unsigned)blocks), dim3(kRowsThreads), 0, st, r));

  HeadParams p = {};
  p.rows = rows; p.T = T; p.rows_alloc = l.rows_alloc; p.split = 1;
  p.part = reinterpret_cast<float2*>(ws + l.part);
  p.wait_limit_ns = training_wait_limit();
  p.withhold = training_withhold();
  p.status_word = status_word;
  HeadMaps logits, maps;
  const uint64_t ux = T > 1 ? ldx : l.packed_ld, uw = d > 1 ? ldw : (V + 7) / 8 * 8;
  if (!encode_map(&logits.a, X, d, T, ux, kHK, kHM) || !encode_map(&logits.a_packed, packed, d, l.rows_alloc, l.packed_ld, kHK, kHM) ||
      !encode_map(&logits.b, W, V, d, uw, 64, kHK))
    return CWL_ERR_CUDA;

  if (loss != nullptr) {
    HeadParams q = p;
    q.n_extent = V; q.k_extent = d; q.tn = l.stats.tn; q.n_cols = l.stats.n_cols; q.kb_per_split = ceil_div(d, kHK);
    CWL_CUDA_TRY(launch_head<HEAD_STATS>(logits, q, T, chained, st));
    CWL_CUDA_TRY(launch_chained(chained, head_finish_kernel, dim3((unsigned)ceil_div(T, 32)), dim3(kFinishThreads), 0, st, rows,
                                static_cast<const float2*>(q.part), 2 * l.stats.n_cols, l.rows_alloc, weight, loss, lse));
  }
  for (int piece = 0; piece < l.pieces; ++piece) {
    const int first = piece * l.piece, width = V - first < l.piece ? V - first : l.piece;
    HeadParams q = p;
    q.n_extent = width; q.n_first = first; q.k_extent = d; q.kb_per_split = ceil_div(d, kHK);
    q.tn = l.dz.tn; q.n_cols = ceil_div(width, q.tn);
    q.dz = dz; q.dz_ld = l.piece;
    CWL_CUDA_TRY(launch_head<HEAD_DZ>(logits, q, T, chained, st));
    if (dX != nullptr) {
      q = p;
      q.n_extent = d; q.k_extent = width; q.k_first = first;
      q.tn = l.dx.tn; q.n_cols = l.dx.n_cols; q.split = l.dx.split; q.kb_per_split = ceil_div(ceil_div(width, kHK), q.split);
      const bool last = piece + 1 == l.pieces;
      q.acc = reinterpret_cast<float*>(ws + l.acc_x); q.acc_groups = l.dx_groups;
      q.acc_in = piece > 0; q.acc_out = q.split > 1 || !last;
      q.out = dX; q.out_ld = lddx; q.out_f32 = es == 4;
      q.out_vec = aligned16(dX) && (T == 1 || lddx * es % 16 == 0);
      if (!encode_map(&maps.a, dz, width, l.rows_alloc, l.piece, kHK, kHM) || !encode_map(&maps.b, W, V, d, uw, kHK, 64)) return CWL_ERR_CUDA;
      maps.a_packed = maps.a;
      CWL_CUDA_TRY(launch_head<HEAD_DX>(maps, q, T, chained, st));
      if (last && q.split > 1)
        CWL_CUDA_TRY(launch_chained(chained, head_sum_kernel, dim3((unsigned)ceil_div(T, kHM), (unsigned)ceil_div(d, 32)), dim3(kSumThreads), 0, st,
                                    rows, T, 0, d, static_cast<const float*>(q.acc), q.acc_groups, q.split, dX, lddx, q.out_f32, q.out_vec));
    }
    if (dW != nullptr) {
      q = p;
      q.m_extent = d; q.n_extent = width; q.n_first = 0;
      q.tn = l.dw.tn; q.n_cols = ceil_div(width, q.tn); q.split = l.dw.split;
      q.acc = reinterpret_cast<float*>(ws + l.acc_w); q.acc_groups = l.dw_groups; q.acc_out = q.split > 1;
      q.out = static_cast<uint8_t*>(dW) + (size_t)first * es; q.out_ld = lddw; q.out_f32 = es == 4;
      q.out_vec = aligned16(q.out) && (d == 1 || lddw * es % 16 == 0);
      if (!encode_map(&maps.a, X, d, T, ux, 64, kHK) || !encode_map(&maps.a_packed, packed, d, l.rows_alloc, l.packed_ld, 64, kHK) ||
          !encode_map(&maps.b, dz, width, l.rows_alloc, l.piece, 64, kHK))
        return CWL_ERR_CUDA;
      CWL_CUDA_TRY(launch_head<HEAD_DW>(maps, q, d, chained, st));
      if (q.split > 1)
        CWL_CUDA_TRY(launch_chained(chained, head_sum_kernel, dim3((unsigned)ceil_div(d, kHM), (unsigned)ceil_div(width, 32)), dim3(kSumThreads), 0, st,
                                    rows, T, d, width, static_cast<const float*>(q.acc), q.acc_groups, q.split, q.out, lddw, q.out_f32, q.out_vec));
    }
  }
  return CWL_OK;
} catch (...) {
  return CWL_ERR_CUDA;                                   // nothing may leave a C entry
}

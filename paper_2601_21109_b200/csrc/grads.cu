// cwl_apply_grads: gradient of the adapter factors under a chunk table.
//
//   Y = X W + H' B,  H' = g o (X A)  (g: the per-row gate of cwl_apply)
//   G = g o (dY B^T),   dA = X^T G,   dB = H'^T dY
//
// Two launches of tcgen05 products whose narrow side is the ladder rank R:
//   SHRINK  one output tile per 128 rows: P = X A and Q = dY B^T (K = d_in and d_out), gated, and kept as the sum of two
//           bf16 numbers (16 significant bits: rounded once to 8, the gradients' error would grow by 40 % over that of
//           their own rounding to bf16, and fp32 gradients would not be worth their name);
//   FOLD    one output tile per 128 columns of X or dY: dA = X^T G and dB^T = dY^T H' (K = T), both halves in one pass
//           over X and dY: [G_hi G_lo] is one operand of 2 R columns, and the halves of the product meet in the epilogue.
// X and dY are read by both: no output of FOLD can be summed before all of d_in / d_out went through SHRINK for its rows.
//
// What bounds it (R = 64, T = 16384, 4096 -> 11008: 173 us in bursts, 188 to 203 under lasting load, twice 495 MB at 5.7 to 4.9
// TB/s; T = 4096: 56 us, 4.4 TB/s): no unit as a whole, most likely what the busiest SMs take in.  At T = 4096 SHRINK takes 32.6 us and FOLD 33.4, with DRAM at 49 and
// 47 %, L2 at 28 %, the tensor pipe at 14 and 30 % of their cycles.  [G_hi G_lo] comes into every CTA beside X and dY (in FOLD half of
// 251 MB), and the tiles deal unevenly: 236 CTAs of FOLD on 148 SMs, of which the busiest take in 2.13 MB and the idlest 1.06; the
// busiest of SHRINK 1.50 MB where the mean is 1.30.  Reading the rows that SHRINK read last first, or SHRINK in waves of rows so that
// they could still be in L2, therefore changed nothing: 169 -> 169 to 189 us.  Short ones are bound by the two launches, each with its
// ramp and its meeting of partial sums (T = 2048, 4096 -> 4096: 24.6 us; T = 256, 1024 -> 1024, R = 16: 12 us on the device).
// The K loop of a tile is split over the CTAs of a cluster where the tiles alone do not fill the GPU; the partial
// accumulators meet in distributed shared memory in a fixed order, so results do not depend on timing.
//
// Roles per CTA: warp 0 = TMA producer, warp 1 = tcgen05.mma issuer and owner of the tensor memory, warps 2..5 move the
// accumulator to shared memory; all warps reduce and store.  SHRINK reads the rows of X / dY K-major; A is N-major and
// B K-major, as they lie in memory.  FOLD reads X / dY M-major (their columns are the output rows) and G / H' N-major.
// Every wait is bounded: when one runs out the CTA raises CWL_ERR_TIMEOUT, stores nothing and still meets its cluster (whose
// other CTAs may store what lacks its part).
#include "cluster.cuh"
#include "cwl_common.cuh"
#include "gate.cuh"
#include "tcgen05_common.cuh"

namespace cwl {
namespace {

constexpr int kGM = 128;                        // rows of an accumulator tile = TMEM lanes
constexpr int kGK = 64;                         // K elements per stage
constexpr int kGThreads = 192;
constexpr int kGLeftBytes = kGM * kGK * 2;      // 16 KB of the wide operand per stage
constexpr int kGBoxBytes = 64 * kGK * 2;        // one 64-column box
constexpr int kGMaxStages = 8;
constexpr int kGMaxCluster = 8;

enum : int { PHASE_SHRINK = 0, PHASE_FOLD = 1 };

struct GradMaps { CUtensorMap wide[2], narrow[2]; };   // per side: 0 = X with A / G, 1 = dY with B / H'

struct GradParams {
  int T, R;
  int d[2];                    // d_in, d_out
  int window, window_mode;
  cwl_chunk_table table;
  int n_tiles[2], first;       // output tiles per side; the side whose tiles come first (the one with the longer K loop)
  int n_kb[2];                 // 64-deep K blocks per side
  int split;                   // CTAs of the cluster that share a tile's K loop
  int tile_m, acc_cols;        // FOLD: 128 or 256 columns of X / dY per CTA (one or two accumulators), TMEM columns of one
  int stages, stage_bytes, wide_bytes, narrow_bytes, tmem_cols, ring_bytes;
  int meet_in_ring, meet_off;  // where a cluster's partial sums meet: over the idle ring, or beside it
  __nv_bfloat16* gated[2];     // SHRINK: where side s's result goes: H' (side 0) and G (side 1), [T, gated_ld]
  int gated_ld, lo_col;        // a row: R columns of high halves, then (from column lo_col) R of low halves
  void* out[2]; int64_t ld[2]; // FOLD: dA, dB
  int out_f32;
  unsigned long long wait_limit_ns;
  int withhold;                // test build: SHRINK's last K block is never loaded
  int32_t* status_word;
};

__device__ __forceinline__ void tmem_alloc1(uint32_t dst_smem, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish1() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc1(uint32_t taddr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
__device__ __forceinline__ void umma_bf16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// kind::f16, fp32 accumulate, bf16 x bf16; a_mn / b_mn: that operand lies with its M / N dimension contiguous
__device__ __forceinline__ uint32_t grad_idesc(int n, int a_mn, int b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(kGM >> 4) << 24);
}
__device__ __forceinline__ void store8(void* out, int64_t at, int f32, const float4& a, const float4& b) {
  if (f32) {
    float4* o = reinterpret_cast<float4*>(reinterpret_cast<float*>(out) + at);
    o[0] = a;
    o[1] = b;
  } else {
    *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(out) + at) =
        make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
  }
}
// eight columns of one row of the tile, where rows of the tile are rows of the output: gated H' or G, or dA
template <int kPhase>
__device__ __forceinline__ void store_row8(const GradParams& p, int side, int at, int col, const RowGate& g, const float4& a, const float4& b) {
  if (kPhase == PHASE_SHRINK) {
    if (at < p.T) {
      const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = v[2 * k] * gate_at(g, col + 2 * k), y = v[2 * k + 1] * gate_at(g, col + 2 * k + 1);
        hi[k] = pack_bf16(x, y);
        lo[k] = pack_bf16(x - __uint_as_float(hi[k] << 16), y - __uint_as_float(hi[k] & 0xFFFF0000u));
      }
      __nv_bfloat16* o = p.gated[side] + (int64_t)at * p.gated_ld + col;
      *reinterpret_cast<uint4*>(o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(o + p.lo_col) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  } else if (at < p.d[0]) {
    store8(p.out[0], (int64_t)at * p.ld[0] + col, p.out_f32, a, b);
  }
}

template <int kPhase>
__global__ void __launch_bounds__(kGThreads)
grad_kernel(const __grid_constant__ GradMaps maps, const __grid_constant__ GradParams p) {
  extern __shared__ uint8_t grad_raw[];
  const uint32_t raw = smem_u32(grad_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;         // swizzled boxes need 1024-byte alignment
  uint8_t* base_ptr = grad_raw + (base - raw);
  const uint32_t bars = base + (uint32_t)p.ring_bytes;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kGMaxStages + s); };
  const uint32_t acc_bar = bars + 8u * (2 * kGMaxStages);
  uint8_t* misc = base_ptr + p.ring_bytes + 8 * (2 * kGMaxStages + 1) + 8;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);     // its wait limit sits at misc + 16
  RowGate* gates = reinterpret_cast<RowGate*>(misc + 32);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // which tile, which share of its K loop
  const int split = p.split;
  const int cta = split > 1 ? (int)cluster_rank() : 0;
  int tile = blockIdx.x / split;
  int side = p.first;
  if (tile >= p.n_tiles[side]) { tile -= p.n_tiles[side]; side ^= 1; }
  const int per = (p.n_kb[side] + split - 1) / split;
  const int kb0 = min(cta * per, p.n_kb[side]);
  const int n_blk = min(kb0 + per, p.n_kb[side]) - kb0;
  const int n_acc = kPhase == PHASE_FOLD ? p.tile_m / kGM : 1;
  const int m0 = tile * kGM * n_acc;
  const CUtensorMap* wide = &maps.wide[side];
  const CUtensorMap* narrow = &maps.narrow[side];

  if (tid == 0) {
    for (int s = 0; s < kGMaxStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(acc_bar, 1);
    *abort_flag = 0;
    *reinterpret_cast<volatile unsigned long long*>(misc + 16) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(wide);
    prefetch_tmap(narrow);
  }
  if (warp == 1) {
    tmem_alloc1(smem_u32(const_cast<uint32_t*>(tmem_slot)), (uint32_t)p.tmem_cols);
    tmem_relinquish1();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if (split > 1 && !p.meet_in_ring) cluster_barrier_arrive();
  // SHRINK waits here for the launch ahead, and only then lets FOLD be placed: a FOLD that runs therefore knows that what
  // came before SHRINK is complete.  It reads X and dY at once; all that SHRINK writes, and its own outputs, wait below.
  if (kPhase == PHASE_SHRINK) {
    pdl_wait();
    pdl_launch_dependents();
  } else {
    pdl_launch_dependents();
  }

  const bool narrow_k_major = kPhase == PHASE_SHRINK && side == 1;      // B [R, d_out]: its K dimension is contiguous
  int issued = 0;                                        // of the producer: K blocks whose loads went out
  if (warp == 0) {
    if (lane == 0) {
      const int n_boxes = narrow_k_major ? 1 : p.narrow_bytes / kGBoxBytes;
      const uint32_t tx = (uint32_t)(p.wide_bytes + (narrow_k_major ? p.R * kGK * 2 : n_boxes * kGBoxBytes));
      auto load_wide = [&](int st, int k) {
        const uint32_t sa = base + (uint32_t)(st * p.stage_bytes);
        mbar_expect_tx(full_bar(st), tx);
        if (kPhase == PHASE_SHRINK) {
          tma_load_2d(sa, wide, full_bar(st), k, m0);
        } else {
          for (int j = 0; j < 2 * n_acc; ++j) tma_load_2d(sa + j * kGBoxBytes, wide, full_bar(st), m0 + 64 * j, k);
        }
      };
      auto load_narrow = [&](int st, int k) {
        const uint32_t sb = base + (uint32_t)(st * p.stage_bytes + p.wide_bytes);
        if (narrow_k_major) {
          tma_load_2d(sb, narrow, full_bar(st), k, 0);
        } else {
          for (int j = 0; j < n_boxes; ++j) tma_load_2d(sb + j * kGBoxBytes, narrow, full_bar(st), j * 64, k);
        }
      };
      const int n_load = CWL_WITHHELD(p) && kPhase == PHASE_SHRINK ? n_blk - 1 : n_blk;
      const int ahead = min(n_load, p.stages);           // the ring starts empty
      for (int b = 0; b < ahead; ++b) load_wide(b, (kb0 + b) * kGK);
      if (kPhase == PHASE_FOLD) pdl_wait();
      for (int b = 0; b < ahead; ++b) load_narrow(b, (kb0 + b) * kGK);
      issued = max(ahead, 0);
      int s = 0;
      uint32_t ph = 1;
      for (int b = ahead; b < n_load; ++b) {
        if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag)) break;
        load_wide(s, (kb0 + b) * kGK);
        load_narrow(s, (kb0 + b) * kGK);
        ++issued;
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && n_blk > 0) {
      // FOLD: both halves as one product of 2 R columns where that is at most 256, else one after the other
      const bool halves = kPhase == PHASE_FOLD && 2 * p.R > 256;
      const uint32_t idesc = grad_idesc(kPhase == PHASE_FOLD && !halves ? 2 * p.R : p.R, kPhase == PHASE_FOLD, !narrow_k_major);
      const uint64_t lo_half = (uint64_t)((p.lo_col / 64) * kGBoxBytes) >> 4;
      // one K step of 16 further on: 32 bytes in a K-major tile, 16 rows of 128 bytes in a box with the other order
      const uint64_t step_a = kPhase == PHASE_SHRINK ? (16 * 2) >> 4 : (16 * 128) >> 4;
      const uint64_t step_b = narrow_k_major ? (16 * 2) >> 4 : (16 * 128) >> 4;
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int b = 0; b < n_blk; ++b) {
        if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t sa = base + (uint32_t)(s * p.stage_bytes), sb = sa + p.wide_bytes;
        const uint64_t da = kPhase == PHASE_SHRINK ? make_smem_desc(sa, 16, 1024) : make_smem_desc(sa, kGBoxBytes, 1024);
        const uint64_t db = narrow_k_major ? make_smem_desc(sb, 16, 1024) : make_smem_desc(sb, kGBoxBytes, 1024);
#pragma unroll
        for (int kk = 0; kk < kGK / 16; ++kk) {
          umma_bf16(tmem, da + kk * step_a, db + kk * step_b, idesc, (b | kk) ? 1u : 0u);
          if (kPhase == PHASE_FOLD && n_acc > 1)
            umma_bf16(tmem + p.acc_cols, da + (kGLeftBytes >> 4) + kk * step_a, db + kk * step_b, idesc, (b | kk) ? 1u : 0u);
          if (halves) umma_bf16(tmem + p.lo_col, da + kk * step_a, db + lo_half + kk * step_b, idesc, (b | kk) ? 1u : 0u);
        }
        umma_commit(empty_bar(s));
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
      if (ok) {
        umma_commit(acc_bar);
      } else {
        // MMAs in flight get a bounded time to retire before the tensor memory is released
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 1000000ull) {}
      }
    }
  } else if (kPhase == PHASE_SHRINK) {
    const int mine = (warp & 3) * 32 + lane;             // the row this thread drains
    gates[mine] = table_gate(m0 + mine, p);                // while the main loop runs (a chain of dependent loads)
  }

  if (kPhase == PHASE_FOLD) pdl_wait();                  // every thread, before it writes an output
  // Wait for the accumulator.  A CTA without K blocks (short loops on many CTAs) contributes zeros.
  const int quad = warp & 3, row = quad * 32 + lane;     // of warps 2..5: the TMEM lanes a warp may read, one tile row a lane
  const bool drain = warp >= 2;
  if (drain && n_blk > 0) {
    mbar_wait(acc_bar, 0, abort_flag);
    __syncwarp();
    tc_fence_after();
  }
  auto columns = [&](int acc, int c, uint32_t (&v)[32]) {   // 32 columns of this lane's row of an accumulator
    if (n_blk > 0) {
      const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + acc * p.acc_cols + c;
      tmem_ld32(at, v);
      if (kPhase == PHASE_FOLD) {
        uint32_t lo[32];
        tmem_ld32(at + p.lo_col, lo);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(lo[j]));
      } else {
        tmem_ld_wait();
      }
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = 0;
    }
  };
  const bool by_rows = kPhase == PHASE_SHRINK || side == 0;      // rows of the tile are rows of the output (else its columns)
  if (split == 1) {
    // straight from the accumulator
    if (drain && *abort_flag == 0) {
      for (int acc = 0; acc < n_acc; ++acc) {
        const int at_row = acc * kGM + row;
        for (int c = 0; c < p.R; c += 32) {
          uint32_t v[32];
          columns(acc, c, v);
          if (by_rows) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (c + q * 8 < p.R)
                store_row8<kPhase>(p, side, m0 + at_row, c + q * 8, kPhase == PHASE_SHRINK ? gates[row] : RowGate{},
                                   make_float4(__uint_as_float(v[q * 8]), __uint_as_float(v[q * 8 + 1]), __uint_as_float(v[q * 8 + 2]), __uint_as_float(v[q * 8 + 3])),
                                   make_float4(__uint_as_float(v[q * 8 + 4]), __uint_as_float(v[q * 8 + 5]), __uint_as_float(v[q * 8 + 6]), __uint_as_float(v[q * 8 + 7])));
          } else if (m0 + at_row < p.d[1]) {             // a warp stores 32 neighbours of an output row at a time
            const int n = min(32, p.R - c);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (j < n) {
                const int64_t at = (int64_t)(c + j) * p.ld[1] + m0 + at_row;
                if (p.out_f32) reinterpret_cast<float*>(p.out[1])[at] = __uint_as_float(v[j]);
                else reinterpret_cast<__nv_bfloat16*>(p.out[1])[at] = __float2bfloat16_rn(__uint_as_float(v[j]));
              }
            }
          }
        }
      }
    }
    tc_fence_before();
    __syncthreads();
  } else {
    // Every CTA owns a share of the output: tile_m / split rows of the tile, or R / split columns of it where those are the
    // rows of the output.  The others' accumulators are pushed into its shared memory and added up there, in the order of
    // the CTAs.  Layouts are such that a warp's stores are contiguous: [column group of 4][rows][4] and [column][128 rows].
    if (p.meet_in_ring) {                                // over the ring, once it is idle in the whole cluster
      tc_fence_before();
      cluster_barrier();
      tc_fence_after();
    } else {
      cluster_barrier_wait();                       // the peers run (they arrived at their start)
    }
    const int tile_m = kGM * n_acc;
    const int share = (by_rows ? tile_m : p.R) / split;
    const uint32_t meet = base + (uint32_t)p.meet_off;
    const int part = by_rows ? share * p.R : share * tile_m;         // numbers that one CTA contributes to a share
    if (drain) {
      for (int acc = 0; acc < n_acc; ++acc) {
        const int at_row = acc * kGM + row;
        if (by_rows) {
          const int owner = at_row / share;
          const uint32_t to = peer_shared(meet, owner) + (uint32_t)(cta * part + (at_row - owner * share) * 4) * 4u;
          for (int c = 0; c < p.R; c += 32) {
            uint32_t v[32];
            columns(acc, c, v);
#pragma unroll
            for (int q = 0; q < 8; ++q)
              if (c + q * 4 < p.R)
                st_peer_v4(to + (uint32_t)((c + q * 4) * share) * 4u, v[q * 4], v[q * 4 + 1], v[q * 4 + 2], v[q * 4 + 3]);
          }
        } else {
          for (int c = 0; c < p.R; c += 32) {
            uint32_t v[32];
            columns(acc, c, v);
            const int n = min(32, p.R - c);
            int owner = c / share, left = share - (c - owner * share);
            uint32_t to = peer_shared(meet, owner) + (uint32_t)(cta * part + (share - left) * tile_m + at_row) * 4u;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (j < n) {
                if (left == 0) {
                  left = share;
                  to = peer_shared(meet, ++owner) + (uint32_t)(cta * part + at_row) * 4u;
                }
                st_peer_b32(to, v[j]);
                to += (uint32_t)tile_m * 4u;
                --left;
              }
            }
          }
        }
      }
      tc_fence_before();
    }
    cluster_barrier();                              // this CTA's shares have arrived, and it may leave when it is done
    if (*abort_flag == 0) {
      const float* in = reinterpret_cast<const float*>(base_ptr + p.meet_off);
      // eight numbers of an output row a thread
      for (int i = tid; i < part / 8; i += kGThreads) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        const int line = by_rows ? i % share : i / (tile_m / 8);     // row of the tile in the share, or column of it
        const int col = by_rows ? (i / share) * 8 : (i % (tile_m / 8)) * 8;
        const float* q = in + (by_rows ? col * share + line * 4 : line * tile_m + col);
        const int second = by_rows ? share * 4 : 4;
        for (int r = 0; r < split; ++r, q += part) {
          const float4 x = *reinterpret_cast<const float4*>(q), y = *reinterpret_cast<const float4*>(q + second);
          a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
          b.x += y.x; b.y += y.y; b.z += y.z; b.w += y.w;
        }
        const int at = cta * share + line;
        if (by_rows) {
          store_row8<kPhase>(p, side, m0 + at, col, kPhase == PHASE_SHRINK ? gates[at] : RowGate{}, a, b);
        } else if (m0 + col < p.d[1]) {                  // d_out is a multiple of 16
          store8(p.out[1], (int64_t)at * p.ld[1] + m0 + col, p.out_f32, a, b);
        }
      }
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc1(tmem, (uint32_t)p.tmem_cols);
  }
  if (tid == 0 && *abort_flag != 0) {
    flag_status(p.status_word, CWL_ERR_TIMEOUT);
    // copies that nobody waited for get a bounded chance to land before the CTA leaves
    for (int back = 1; back <= p.stages && back <= issued; ++back) {
      const int j = issued - back;
      const unsigned long long t0 = global_timer();
      while (!mbar_try_wait(full_bar(j % p.stages), (uint32_t)(j / p.stages) & 1u) && global_timer() - t0 < p.wait_limit_ns) {}
    }
  }
}

struct GradLaunch {
  int split, tile_m, acc_cols, stages, stage_bytes, wide_bytes, narrow_bytes, tmem_cols, ring_bytes, meet_in_ring, meet_off;
  size_t smem;
};

// CTAs a tile's K loop (the longer side's, n_kb blocks) is split over: doubled while there is an SM for each and each keeps
// four K blocks; up to `resident` CTAs (two an SM where their shared memory allows it) while each keeps kDeepBlocks, which
// is what the meeting of the partial sums asks for.
constexpr int kDeepBlocks = 8;
int grad_split(int tiles, int n_kb, int resident) {
  int s = 1;
  while (s < kGMaxCluster && ((tiles * s * 2 <= 148 && n_kb / (s * 2) >= 4) || (tiles * s * 2 <= resident && n_kb / (s * 2) >= kDeepBlocks)))
    s *= 2;
  return s;
}

// `columns` of the narrow operand: R, or what both halves of G / H' take; tile_m: 128, or 256 (FOLD)
GradLaunch grad_launch(int R, int columns, int tile_m, int tiles, int n_kb) {
  GradLaunch l;
  l.tile_m = tile_m;
  l.wide_bytes = kGLeftBytes * (tile_m / kGM);
  l.narrow_bytes = ((columns + 63) / 64) * kGBoxBytes;
  l.stage_bytes = l.wide_bytes + l.narrow_bytes;
  // three stages or more in 96 KB let two CTAs share an SM (FOLD's set-up then runs beside SHRINK's end); a deeper stage
  // takes what the SM has
  const bool pair = 3 * l.stage_bytes <= 96 * 1024;
  l.split = grad_split(tiles, n_kb, pair ? 296 : 148);
  const int budget = pair ? 96 * 1024 : 192 * 1024;
  l.stages = budget / l.stage_bytes;
  if (l.stages > kGMaxStages) l.stages = kGMaxStages;
  // a cluster's partial sums, [tile_m][R] fp32: beside a ring of at least three stages where both fit 109 KB (no need to wait
  // for the whole cluster's MMAs before they are sent), else over the ring
  const int meet = l.split == 1 ? 0 : tile_m * R * 4;
  l.meet_in_ring = 0;
  l.ring_bytes = l.stages * l.stage_bytes;
  if (l.split > 1) {
    int beside = (109 * 1024 - meet) / l.stage_bytes;
    if (beside > l.stages) beside = l.stages;
    if (beside >= 3) {
      l.stages = beside;
      l.meet_off = l.stages * l.stage_bytes;
      l.ring_bytes = l.meet_off + meet;
    } else {
      l.meet_in_ring = 1;
      l.meet_off = 0;
      if (l.ring_bytes < meet) l.ring_bytes = meet;
    }
  } else {
    l.meet_off = 0;
  }
  // the epilogue reads 32 columns at a time, from 0 and (low halves) from columns - R on
  const int read = columns - R + (R + 31) / 32 * 32;
  l.acc_cols = 32;
  while (l.acc_cols < read) l.acc_cols *= 2;
  l.tmem_cols = l.acc_cols * (tile_m / kGM);
  l.smem = (size_t)l.ring_bytes + 1024 + 8 * (2 * kGMaxStages + 1) + 8 + 32 + kGM * sizeof(RowGate);
  return l;
}

template <int kPhase>
cudaError_t launch_phase(const GradMaps& maps, const GradParams& p, const GradLaunch& l, bool chained, cudaStream_t st) {
  static SharedMemoryGrant grant;
  const cudaError_t e = grant(grad_kernel<kPhase>);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.n_tiles[0] + p.n_tiles[1]) * l.split));
  cfg.blockDim = dim3(kGThreads);
  cfg.dynamicSmemBytes = l.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = l.split; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = chained ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, grad_kernel<kPhase>, maps, p);
}

// G and H' hold two halves a row: side by side where one product takes both, else the low half from a multiple of 64 on
// (a box's edge), where a product of its own can start
int lo_column(int R) { return 2 * R <= 256 ? R : (R + 63) / 64 * 64; }
// Columns of X / dY per CTA of FOLD: 128, or 256 where both halves of G / H' are wider than 128 columns and would come in
// more often than X and dY themselves (us, 128 -> 256: R = 80 at T = 16384, 4096 -> 11008: 230 -> 188; R = 80 at
// T = 4096, 4096 -> 4096: 44.9 -> 40.8; R = 128 at T = 8192, 4096 -> 4096: 75.8 -> 71.5; but R = 64 at T = 8192: 57.6 ->
// 58.2).  Two accumulators must fit the tensor memory, and the CTAs must still take most SMs for loops of kFoldMinBlocks
// (R = 128 at T = 2048, 4096 -> 4096, loops of 8: 35.0 -> 37.2).
constexpr int kFoldMinCtas = 96, kFoldMinBlocks = 16;
int fold_tile(int R, int d_in, int d_out, int t_blocks) {
  if (R <= 64 || R > 128) return kGM;
  const int tiles = ceil_div(d_in, 2 * kGM) + ceil_div(d_out, 2 * kGM);
  const int split = grad_split(tiles, t_blocks, 148);
  return tiles * split >= kFoldMinCtas && t_blocks / split >= kFoldMinBlocks ? 2 * kGM : kGM;
}
size_t gated_bytes(int T, int R) { return ((size_t)T * (lo_column(R) + R) * 2 + 255) / 256 * 256; }

bool bad_matrix(const void* ptr, int64_t ld, int64_t cols, int elem) {
  return !aligned16(ptr) || ld < cols || (ld * elem) % 16 != 0;
}

}  // namespace
}  // namespace cwl

extern "C" size_t cwl_apply_grads_workspace_bytes(int32_t T, int32_t d_in, int32_t d_out, int32_t R) {
  if (T <= 0 || d_in <= 0 || d_out <= 0 || R <= 0) return 0;
  return 2 * cwl::gated_bytes(T, R);
}

extern "C" cwl_status cwl_apply_grads(const void* X, int64_t ldx, const void* dY, int64_t lddy,
                                      const void* A, int64_t lda, const void* B, int64_t ldb,
                                      int32_t T, int32_t d_in, int32_t d_out, int32_t R,
                                      cwl_chunk_table table, int32_t window, int32_t window_mode,
                                      void* dA, int64_t ldda, void* dB, int64_t lddb, cwl_dtype grad_dtype,
                                      void* workspace, size_t workspace_bytes, int32_t* status_word, void* stream) try {
  using namespace cwl;
  if (T < 0 || d_in <= 0 || d_out <= 0 || R <= 0 || window < 0) return CWL_ERR_INVALID_ARG;
  if (window_mode != CWL_WINDOW_CAUSAL && window_mode != CWL_WINDOW_CENTRED) return CWL_ERR_INVALID_ARG;
  if (grad_dtype != CWL_F32 && grad_dtype != CWL_BF16) return CWL_ERR_INVALID_ARG;
  if (dA == nullptr || dB == nullptr) return CWL_ERR_INVALID_ARG;
  if (d_in % 16 != 0 || d_out % 16 != 0 || R % 16 != 0 || R > CWL_MAX_RANK) return CWL_ERR_UNSUPPORTED;
  const int es = grad_dtype == CWL_F32 ? 4 : 2;
  if (bad_matrix(dA, ldda, R, es) || bad_matrix(dB, lddb, d_out, es)) return CWL_ERR_SHAPE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {                                          // a sum over no rows
    CWL_CUDA_TRY(cudaMemset2DAsync(dA, (size_t)ldda * es, 0, (size_t)R * es, d_in, st));
    CWL_CUDA_TRY(cudaMemset2DAsync(dB, (size_t)lddb * es, 0, (size_t)d_out * es, R, st));
    return CWL_OK;
  }
  if (X == nullptr || dY == nullptr || A == nullptr || B == nullptr) return CWL_ERR_INVALID_ARG;
  if (table.offsets == nullptr || table.rank == nullptr || table.scale == nullptr || table.flags == nullptr ||
      table.n_chunks == nullptr || table.capacity < 0)
    return CWL_ERR_INVALID_ARG;
  if (bad_matrix(X, ldx, d_in, 2) || bad_matrix(dY, lddy, d_out, 2) || bad_matrix(A, lda, R, 2) || bad_matrix(B, ldb, d_out, 2))
    return CWL_ERR_SHAPE;
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
      workspace_bytes < cwl_apply_grads_workspace_bytes(T, d_in, d_out, R))
    return CWL_ERR_WORKSPACE;

  __nv_bfloat16* H = static_cast<__nv_bfloat16*>(workspace);
  __nv_bfloat16* G = reinterpret_cast<__nv_bfloat16*>(static_cast<uint8_t*>(workspace) + gated_bytes(T, R));
  GradParams p = {};
  p.T = T; p.R = R; p.d[0] = d_in; p.d[1] = d_out;
  p.window = window; p.window_mode = window_mode; p.table = table;
  p.gated[0] = H; p.gated[1] = G;
  p.lo_col = lo_column(R);
  p.gated_ld = p.lo_col + R;
  p.out[0] = dA; p.out[1] = dB; p.ld[0] = ldda; p.ld[1] = lddb; p.out_f32 = grad_dtype == CWL_F32;
  p.wait_limit_ns = training_wait_limit();
  p.withhold = training_withhold();
  p.status_word = status_word;

  GradMaps shrink, fold;
  const bool maps_ok =
      encode_map(&shrink.wide[0], X, d_in, T, ldx, kGK, kGM) && encode_map(&shrink.narrow[0], A, R, d_in, lda, 64, kGK) &&
      encode_map(&shrink.wide[1], dY, d_out, T, lddy, kGK, kGM) && encode_map(&shrink.narrow[1], B, d_out, R, ldb, kGK, R) &&
      encode_map(&fold.wide[0], X, d_in, T, ldx, 64, kGK) && encode_map(&fold.narrow[0], G, p.gated_ld, T, p.gated_ld, 64, kGK) &&
      encode_map(&fold.wide[1], dY, d_out, T, lddy, 64, kGK) && encode_map(&fold.narrow[1], H, p.gated_ld, T, p.gated_ld, 64, kGK);
  if (!maps_ok) return CWL_ERR_CUDA;

  auto fill = [&](int columns, int tile_m, int rows0, int rows1, int kb0, int kb1) {
    const int tiles0 = ceil_div(rows0, tile_m), tiles1 = ceil_div(rows1, tile_m);
    p.n_tiles[0] = tiles0; p.n_tiles[1] = tiles1;
    p.n_kb[0] = kb0; p.n_kb[1] = kb1;
    p.first = kb1 > kb0 ? 1 : 0;                         // the longer loops start first
    const GradLaunch l = grad_launch(R, columns, tile_m, tiles0 + tiles1, kb0 > kb1 ? kb0 : kb1);
    p.split = l.split; p.stages = l.stages; p.stage_bytes = l.stage_bytes; p.wide_bytes = l.wide_bytes; p.narrow_bytes = l.narrow_bytes;
    p.tile_m = l.tile_m; p.acc_cols = l.acc_cols;
    p.tmem_cols = l.tmem_cols; p.ring_bytes = l.ring_bytes; p.meet_in_ring = l.meet_in_ring; p.meet_off = l.meet_off;
    return l;
  };
  const bool chained = !stream_is_capturing(st);
  const int t_blocks = ceil_div(T, kGK);
  GradLaunch l = fill(R, kGM, T, T, ceil_div(d_in, kGK), ceil_div(d_out, kGK));
  CWL_CUDA_TRY(launch_phase<PHASE_SHRINK>(shrink, p, l, chained, st));
  l = fill(p.gated_ld, fold_tile(R, d_in, d_out, t_blocks), d_in, d_out, t_blocks, t_blocks);
  CWL_CUDA_TRY(launch_phase<PHASE_FOLD>(fold, p, l, chained, st));
  return CWL_OK;
} catch (...) {
  return CWL_ERR_CUDA;                                   // nothing may leave a C entry
}

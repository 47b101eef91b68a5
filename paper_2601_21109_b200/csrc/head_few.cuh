// Logits of up to 64 rows, 128 where the loss alone is wanted (included by head.cu): STATS and EXP with the operands' places exchanged, Z^T = W^T X^T.
//
// Few rows are bound by the bytes of W.  head_kernel would fill 256 rows of tensor memory with them and spend half of what it
// brings into shared memory on X; here the vocabulary is the M dimension (W's columns are contiguous: an M-major operand),
// the rows are the N dimension, and a stage is W but for a few KB.  A block takes up to 256 columns of the vocabulary: two
// tiles of 128 x kRows, drained every kFewChunk K blocks into fp32 sums of the epilogue's threads, one column of the
// vocabulary and all rows a thread.  Single blocks, no pairs: columns are dealt evenly over the SMs, to eight.
//
// Bound by HBM: one row, 4096 -> 32000: 43.5 us, 262 MB at 6.0 TB/s (head_kernel: 57 with tiles of 448 columns, 84 with sums in
// fp32); 48 rows, EXP: 54 us (88); 128 rows, STATS: 61 to 64 us (66), spills of 0.5 KB a thread among them.
#pragma once

constexpr int kFewRows = 128;                             // of STATS
// EXP keeps a register a row beside E's stores: with 128 rows it spills (100 rows: 157 us against head_kernel's 90)
constexpr int kFewExpRows = 64;
constexpr int kFewChunk = 8;                               // K blocks
constexpr int kFewMaxStages = 8;
constexpr int kFewRing = 200 * 1024;
constexpr int kFewThreads = 64 + 32 * 8;
constexpr int kFewBars = 8 * (2 * kFewMaxStages + 4);
constexpr int kFewMeet = 2 * 8 * kFewRows * 4;           // a number per warp and row, twice
constexpr size_t kFewSmem = 1024 + kFewRing + kFewBars + 32 + kFewMeet + kFewRows * 4;

__device__ __forceinline__ void few_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void few_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void few_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void few_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// 16 consecutive fp32 columns of this thread's lane
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}

// kN (16 or 32) numbers a lane, reduced over the lanes: lane l ends with number l mod kN in its first place.  Each step halves
// what a lane still has to pass on.
template <int kN, typename Op>
__device__ __forceinline__ void reduce_lanes(float (&v)[kN], int lane, Op op) {
  constexpr unsigned all = 0xffffffffu;
  if (kN == 16) {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = op(v[j], __shfl_xor_sync(all, v[j], 16));
  }
#pragma unroll
  for (int w = kN / 2; w >= 1; w /= 2) {
    const bool upper = (lane & w) != 0;
#pragma unroll
    for (int j = 0; j < w; ++j) {
      const float give = upper ? v[j] : v[j + w], keep = upper ? v[j + w] : v[j];
      v[j] = op(keep, __shfl_xor_sync(all, give, w));
    }
  }
}

template <int kMode, int kRows>
__global__ void __launch_bounds__(kFewThreads, 1) head_few_kernel(const __grid_constant__ HeadMaps maps, const __grid_constant__ HeadParams p) {
  extern __shared__ uint8_t few_raw[];
  const uint32_t raw = smem_u32(few_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = few_raw + (base - raw);
  const uint32_t bars = base + kFewRing;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kFewMaxStages + s); };
  auto acc_full = [&](int slot) { return bars + 8u * (2 * kFewMaxStages + slot); };
  auto acc_empty = [&](int slot) { return bars + 8u * (2 * kFewMaxStages + 2 + slot); };
  uint8_t* misc = base_ptr + kFewRing + kFewBars;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);     // its wait limit sits at misc + 16
  volatile int* epi_go = reinterpret_cast<volatile int*>(misc + 8);         // epilogue: this tile is complete
  float* meet = reinterpret_cast<float*>(misc + 32);                        // [2][8 warps][kRows]
  int* targets = reinterpret_cast<int*>(misc + 32 + kFewMeet);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr uint32_t kCols = 4 * kRows < 32 ? 32 : 4 * kRows;               // two slots of two tiles; a power of two

  if (threadIdx.x == 0) {
    for (int s = 0; s < kFewMaxStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int k = 0; k < 2; ++k) { mbar_init(acc_full(k), 1); mbar_init(acc_empty(k), 8); }
    *abort_flag = 0;
    *reinterpret_cast<volatile unsigned long long*>(misc + 16) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(&maps.a);
    prefetch_tmap(&maps.a_packed);
    prefetch_tmap(&maps.b);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int n_kb = (p.k_extent + kHK - 1) / kHK;
  const int n_chunks = (n_kb + kFewChunk - 1) / kFewChunk;
  const int boxes = (p.tn + 63) / 64, m_tiles = (boxes + 1) / 2;
  const int stage_bytes = p.stage_bytes, n_stages = p.stages, x_at = boxes * kHBox;
  // Before pdl_wait().  W is there once head_rows_kernel is past its own wait, after which it lets the next kernel begin: all that was
  // launched before this call has completed then, and nothing of this call writes W (outputs that overlap it are refused).
  // head_rows_kernel has to stay the first launch of the call and to let others begin only after its wait; what is launched
  // between the two (head_gather_kernel, DX, sums) may let the next one begin whenever it likes.  As much of W as the ring holds
  // is fetched beside the kernels ahead (a tenth of it for 4096 -> 32000; one row 53.8 -> 52.1 us, 48 rows 143 -> 139)
  const int ahead = min(n_stages, n_kb - (CWL_WITHHELD(p) ? 1 : 0));
  if (warp == 0 && lane >= 1 && lane <= boxes) {
    for (int b = 0; b < ahead; ++b)
      few_load(base + b * stage_bytes + (lane - 1) * kHBox, &maps.b, full_bar(b), p.n_first + (int)blockIdx.x * p.tn + (lane - 1) * 64, b * kHK);
  }
  pdl_launch_dependents();
  pdl_wait();

  const int n = *p.rows.n;
  const int n_tiles = n > 0 ? p.n_cols : 0;              // nothing to do without rows
  const CUtensorMap* map_x = n < p.T ? &maps.a_packed : &maps.a;

  if (warp == 0) {
    uint32_t issued = 0, s = 0, ph = 0;
    bool ok = true;
    const uint32_t tx = (uint32_t)(boxes * kHBox + kRows * kHK * 2);
    for (int tile = blockIdx.x; ok && tile < n_tiles; tile += gridDim.x) {
      const int at = p.n_first + tile * p.tn;
      for (int b = 0; b < n_kb; ++b) {
        if (CWL_WITHHELD(p) && tile == (int)blockIdx.x && b == n_kb - 1) { ok = false; break; }
        const bool step_ok = mbar_wait(empty_bar(s), ph ^ 1u, abort_flag);
        if (!__all_sync(0xffffffffu, step_ok)) { ok = false; break; }
        const uint32_t to = base + s * stage_bytes;
        if (lane == 0) {
          mbar_expect_tx(full_bar(s), tx);
          few_load(to + x_at, map_x, full_bar(s), b * kHK, 0);
        }
        __syncwarp();
        if (lane >= 1 && lane <= boxes && issued >= (uint32_t)ahead)
          few_load(to + (lane - 1) * kHBox, &maps.b, full_bar(s), at + (lane - 1) * 64, b * kHK);
        ++issued;
        if (++s == (uint32_t)n_stages) { s = 0; ph ^= 1u; }
      }
    }
    if (lane == 0) {
      // what was fetched ahead and came to no use lands before the block leaves
      for (int k = (int)issued; k < ahead; ++k) {
        mbar_expect_tx(full_bar(k), (uint32_t)(boxes * kHBox));
        const unsigned long long t0 = global_timer();
        while (!mbar_try_wait(full_bar(k), 0u) && global_timer() - t0 < p.wait_limit_ns) {}
      }
    }
    if (!ok && lane == 0) {
      // copies already issued get a bounded chance to land before the block leaves
      for (uint32_t back = 1; back <= (uint32_t)n_stages && back <= issued; ++back) {
        const uint32_t j = issued - back;
        const unsigned long long t0 = global_timer();
        while (!mbar_try_wait(full_bar(j % n_stages), (j / n_stages) & 1u) && global_timer() - t0 < p.wait_limit_ns) {}
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // A: M-major, 128 columns of W in two boxes; B: K-major, rows of X
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | ((uint32_t)(kRows >> 3) << 17) | ((uint32_t)(kHM >> 4) << 24);
      uint32_t local = 0, s = 0, ph = 0;
      bool ok = true;
      for (int tile = blockIdx.x; ok && tile < n_tiles; tile += gridDim.x) {
        for (int chunk = 0; ok && chunk < n_chunks; ++chunk, ++local) {
          const int slot = local & 1u;
          if (!mbar_wait(acc_empty(slot), ((local >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const int n_blk = min(kFewChunk, n_kb - chunk * kFewChunk);
          for (int b = 0; b < n_blk; ++b) {
            if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t at = base + s * stage_bytes;
            const uint64_t db = make_smem_desc(at + x_at, 16, 1024);
            for (int m = 0; m < m_tiles; ++m) {
              const uint64_t da = make_smem_desc(at + m * 2 * kHBox, kHBox, 1024);
#pragma unroll
              for (int kk = 0; kk < kHK / 16; ++kk)
                few_mma(tmem + (slot * 2 + m) * kRows, da + kk * ((16 * 128) >> 4), db + kk * ((16 * 2) >> 4), idesc, (b | kk) ? 1u : 0u);
            }
            few_commit(empty_bar(s));
            if (++s == (uint32_t)n_stages) { s = 0; ph ^= 1u; }
          }
          if (ok) few_commit(acc_full(slot));
        }
      }
      if (!ok) {
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 1000000ull) {}
      }
    }
  } else {
    const int quad = warp & 3, m = (warp - 2) >> 2, epi = threadIdx.x - 64, w8 = warp - 2;
    if (epi < kRows) targets[epi] = epi < n ? p.rows.target[epi] - p.n_first : -1;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const bool mine = m < m_tiles;
    constexpr int kPart = kRows < 32 ? kRows : 32;
    uint32_t local = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < n_tiles; tile += gridDim.x) {
      const int in_tile = m * kHM + quad * 32 + lane;            // this thread's column
      const int col = tile * p.tn + in_tile;
      const bool there = in_tile < p.tn && col < p.n_extent;
      float z[kRows];
      for (int chunk = 0; chunk < n_chunks; ++chunk, ++local) {
        const int slot = local & 1u;
        if (!__all_sync(0xffffffffu, mbar_wait(acc_full(slot), (local >> 1) & 1u, abort_flag))) { ok = false; break; }
        tc_fence_after();
        if (mine) {
          const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + (slot * 2 + m) * kRows;
#pragma unroll
          for (int j0 = 0; j0 < kRows; j0 += kPart) {
            uint32_t r[kPart];
#pragma unroll
            for (int j = 0; j < kPart; j += 16) tmem_ld16(at + j0 + j, r + j);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < kPart; ++j) z[j0 + j] = chunk == 0 ? __uint_as_float(r[j]) : z[j0 + j] + __uint_as_float(r[j]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) few_arrive(acc_empty(slot));
      }
      // one thread's word for all, so that the barriers below are never split
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (epi == 0) *epi_go = *abort_flag == 0;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (*epi_go == 0) break;

      // is any row's target among this warp's columns?
      bool held = false;
#pragma unroll
      for (int j = 0; j < kRows; j += 32) held |= (unsigned)(targets[j + (lane & (kPart - 1))] - (col - lane)) < 32u;
      held = __any_sync(0xffffffffu, held);
      if (held && there) {
#pragma unroll
        for (int j = 0; j < kRows; ++j)
          if (targets[j] == col) {
            p.rows.z_target[j] = z[j];
            z[j] = -INFINITY;                                    // the target stays out of E, of the sum and of what a reference is held against
          }
      }
      // the rows' maxima over the block's columns, 32 rows at a time
#pragma unroll
      for (int b = 0; b < kRows; b += kPart) {
        float v[kPart];
#pragma unroll
        for (int j = 0; j < kPart; ++j) v[j] = there ? z[b + j] : -INFINITY;
        reduce_lanes<kPart>(v, lane, [](float x, float y) { return fmaxf(x, y); });
        if (lane < kPart) meet[w8 * kRows + b + lane] = v[0];
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      float* common = meet + 8 * kRows;                          // [kRows]: the rows' references
      if (epi < kRows) {
        float top = -INFINITY;
        for (int w = 0; w < 8; ++w) top = fmaxf(top, meet[w * kRows + epi]);
        float ref = top == -INFINITY ? 0.f : top;
        if (kMode == HEAD_EXP) {
          ref = epi < n ? p.rows.ref[epi] : 0.f;
          if (p.online && epi < n && top > ref + kAbove) {
            ref = top;
            atomicOr(p.rows.above + (int64_t)epi * p.rows.above_words + (tile >> 5), 1u << (tile & 31));
            p.rows.above_ref[(int64_t)epi * p.rows.chunks + tile] = top;
          }
        }
        common[epi] = ref;
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
#pragma unroll
      for (int j = 0; j < kRows; ++j) z[j] = there && j < n ? exp2_fast(fmaf(z[j], kLog2e, -common[j] * kLog2e)) : 0.f;
      if (kMode == HEAD_EXP) {
        if (there) {
          __nv_bfloat16* e = p.dz + col;
          if (p.terms == 1) {
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
              if (j < n) *e = __float2bfloat16_rn(z[j]);
              e += p.dz_ld;
            }
          } else {
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
              float left = z[j];
              for (int term = 0; term < p.terms && j < n; ++term) {
                const __nv_bfloat16 part = __float2bfloat16_rn(left);
                e[term * p.term_at] = part;
                left -= __bfloat162float(part);
              }
              e += p.dz_ld;
            }
          }
        }
        if (p.terms > 1 && tile == n_tiles - 1) {
          // columns up to the end of the last K block of DX, which reads on there
          const int pad = -p.n_extent & (kHK - 1);
          for (int i = epi; i < n * pad; i += 256)
            for (int term = 0; term < p.terms; ++term)
              p.dz[(int64_t)(i / pad) * p.dz_ld + term * p.term_at + p.n_extent + i % pad] = __float2bfloat16_rn(0.f);
        }
        if (!p.online) {
          asm volatile("bar.sync 1, 256;" ::: "memory");         // before the next tile's maxima
          continue;
        }
      }
#pragma unroll
      for (int b = 0; b < kRows; b += kPart) {
        float v[kPart];
#pragma unroll
        for (int j = 0; j < kPart; ++j) v[j] = z[b + j];
        reduce_lanes<kPart>(v, lane, [](float x, float y) { return x + y; });
        if (lane < kPart) meet[w8 * kRows + b + lane] = v[0];
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (epi < n) {
        float sum = 0.f;
        for (int w = 0; w < 8; ++w) sum += meet[w * kRows + epi];
        // the maximum of nothing but the target is -inf
        p.part[(int64_t)tile * p.rows_alloc + epi] = make_float2(kMode == HEAD_STATS && sum == 0.f ? -INFINITY : common[epi], sum);
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");             // before the next tile's maxima
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) flag_status(p.status_word, CWL_ERR_TIMEOUT);
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
  }
}

// Columns of a block: dealt evenly, to eight, over as few turns of 148 blocks as 256 columns a block allow.
constexpr int kFewBlocks = 148;
inline int few_columns(int V) {
  const int turns = (V + kFewBlocks * 256 - 1) / (kFewBlocks * 256);
  const int each = (V + kFewBlocks * turns - 1) / (kFewBlocks * turns);
  return (each + 7) / 8 * 8;
}

template <int kMode, int kRows>
cudaError_t launch_few_rows(const HeadMaps& maps, HeadParams p, bool chained, cudaStream_t st) {
  static SharedMemoryGrant grant;
  const cudaError_t e = grant(head_few_kernel<kMode, kRows>);
  if (e != cudaSuccess) return e;
  p.stage_bytes = (p.tn + 63) / 64 * kHBox + kRows * kHK * 2;
  p.stages = kFewRing / p.stage_bytes < kFewMaxStages ? kFewRing / p.stage_bytes : kFewMaxStages;
  const int blocks = p.n_cols < kFewBlocks ? p.n_cols : kFewBlocks;
  return launch_chained(chained, head_few_kernel<kMode, kRows>, dim3((unsigned)blocks), dim3(kFewThreads), kFewSmem, st, maps, p);
}
inline int few_box(int T) { return T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128; }
template <int kMode>
cudaError_t launch_few(const HeadMaps& maps, const HeadParams& p, int T, bool chained, cudaStream_t st) {
  switch (few_box(T)) {
    case 16: return launch_few_rows<kMode, 16>(maps, p, chained, st);
    case 32: return launch_few_rows<kMode, 32>(maps, p, chained, st);
    case 64: return launch_few_rows<kMode, 64>(maps, p, chained, st);
    default: return launch_few_rows<HEAD_STATS, 128>(maps, p, chained, st);      // EXP has 64 at most
  }
}

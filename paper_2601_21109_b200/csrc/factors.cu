// cwl_orthogonalize and cwl_factor_step: Newton-Schulz orthogonalisation of adapter factors, alone and as a factor's update.
//
//   X_0 = U / (|U|_F + eps),   X_(k+1) = a X_k + b (X_k X_k^T) X_k + c (X_k X_k^T)^2 X_k      (X with its short side first)
//
// Every X_k is a polynomial in G_0 = X_0 X_0^T times X_0, so the iteration is done on R x R matrices, R the short side:
//   P_k = a I + b G_k + c G_k^2,   G_(k+1) = P_k G_k P_k,   Q_(k+1) = P_k Q_k,   O = Q_steps X_0
// U is read twice instead of 2 steps times, and the products over its long side shrink from 2 steps to 1.5 (G_0 is symmetric).
// The price is precision: directions of singular value s enter G_0 as s^2 and are amplified a^(2 steps) times, so G_0 and the
// iteration are in 64 bits (on the tensor cores' 64-bit products; in 32 bits, directions of s = 2e-3 would be off by a
// per cent).  All matrices of the iteration are symmetric and commute: only tiles of the lower triangle are computed.
//
//   GRAM     a block per (factor, pair of 64-row blocks, slice of the long side): partial products in 64 bits
//   ITERATE  R <= 64: a block a factor, all in shared memory.  R > 64: launches of 16 x 16 tiles over L2-resident matrices
//   APPLY    a block per (factor, 128 columns of the long side, 64 rows): Q U in 32 bits, and the update
//
// What bounds it (one B200).  Many factors (448 of R = 64, bf16 gradients, the update: 1.45 ms; floor 0.49, 3.2 GB): GRAM 0.55 ms, 64-bit
// products at 58 % of the 18.5 T/s that a loop of nothing else reaches (0.32 ms), beside 10 bytes an element; iteration 0.13,
// at 90 % of that rate; APPLY 0.75, 10.2 G multiply-adds at 38 % of the units' rate beside 16 bytes an element: 16 warps an SM wait for
// shared memory and for one another's phases (4 x 8 outputs a thread two to an instruction, 8 x 8 outputs, copies ahead through shared
// memory, several tiles a block: 0.79 to 1.01; pairs of tf32 on the tensor cores: 0.675, and O 1.7 times as far
// off).  Few factors: four launches that wait for one another (a pair of 4096 x 64: 56 us, of which the iteration's 17 products in one SM
// 34, 20 of them the SM's 64-bit rate; four SMs a factor with stores to one another took 68 when one took 62).  R > 64: a launch a product of the iteration, 6.6 us each at R = 256 (256 x 11008 and two more: 230 to 250 us, 92 of them
// these; one cooperative launch with a barrier between products: 118).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <math.h>

#include "cwl_common.cuh"

namespace cwl {
namespace {

constexpr int kFewFactors = 16, kMostFactors = 496;   // of a launch: their descriptors are kernel parameters (1 KB, 31 KB)
constexpr int kShort = 64;                         // R up to which the iteration stays in one block

struct Factor {
  const void* u;                                   // gradient, or the matrix to orthogonalise
  float* m;                                        // momentum (step)
  void* out;                                       // fp32 master (step), or the orthogonalised matrix
  __nv_bfloat16* low;                              // bf16 copy of the master, or null
  int ldu, ldm, ldo, ldl;
  int rows, cols;
  float scale;                                     // of the update
  int first;                                       // first block of the launch at hand
};
static_assert(sizeof(Factor) == 64, "descriptors in kernel parameters");

struct FactorCommon {
  int n;
  int step, nesterov, in_type, out_type;
  float beta, keep, lr;                            // step: momentum, 1 - lr weight_decay, learning rate
  int slice;                                       // GRAM: long-side elements a block
  int steps;
  double a, b, c, eps;
  double* partial;                                 // GRAM: [block][64][64]
  float* q;                                        // [factor] R x R, each `q_stride` apart, and at the end of each what U is lifted by
  int64_t q_stride;
};
template <int kMost>
struct FactorArgs {
  FactorCommon c;
  Factor f[kMost];
};
static_assert(sizeof(FactorArgs<kMostFactors>) <= 32 * 1024 - 256, "kernel parameters");

__host__ __device__ __forceinline__ int short_side(const Factor& f) { return f.rows < f.cols ? f.rows : f.cols; }
__host__ __device__ __forceinline__ int long_side(const Factor& f) { return f.rows < f.cols ? f.cols : f.rows; }
__host__ __device__ __forceinline__ int block_pairs(int R) { const int b = (R + 63) / 64; return b * (b + 1) / 2; }
// blocks of APPLY: 128 elements of the long side, 64 of the short one
constexpr int kApplyLong = 128, kApplyShort = 64;
__host__ __device__ __forceinline__ int apply_blocks(const Factor& f) {
  return ((long_side(f) + kApplyLong - 1) / kApplyLong) * ((short_side(f) + kApplyShort - 1) / kApplyShort);
}

// The factor that a block of GRAM works on.
__device__ __forceinline__ int find_factor(const Factor* f, int n, int block) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (f[mid].first <= block) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ float load_typed(const void* p, int64_t at, int type) {
  if (type == CWL_F32) return static_cast<const float*>(p)[at];
  if (type == CWL_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
  return __half2float(static_cast<const __half*>(p)[at]);
}
// four consecutive elements; `vec`: they lie on a boundary of four
__device__ __forceinline__ float4 load4(const void* p, int64_t at, int type, bool vec, int left) {
  if (vec && left >= 4) {
    if (type == CWL_F32) return *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + at);
    if (type == CWL_BF16)
      return make_float4(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16), __uint_as_float(q.y & 0xFFFF0000u));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&q.x)), y = __half22float2(*reinterpret_cast<const __half2*>(&q.y));
    return make_float4(x.x, x.y, y.x, y.y);
  }
  return make_float4(left > 0 ? load_typed(p, at, type) : 0.f, left > 1 ? load_typed(p, at + 1, type) : 0.f,
                     left > 2 ? load_typed(p, at + 2, type) : 0.f, left > 3 ? load_typed(p, at + 3, type) : 0.f);
}
__device__ __forceinline__ void store4_f32(float* p, const float4& v, bool vec, int left) {
  if (vec && left >= 4) {
    *reinterpret_cast<float4*>(p) = v;
  } else {
    if (left > 0) p[0] = v.x;
    if (left > 1) p[1] = v.y;
    if (left > 2) p[2] = v.z;
    if (left > 3) p[3] = v.w;
  }
}
__device__ __forceinline__ void store4_bf16(__nv_bfloat16* p, const float4& v, bool vec, int left) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  if (vec && left >= 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  } else {
    if (left > 0) p[0] = a.x;
    if (left > 1) p[1] = a.y;
    if (left > 2) p[2] = b.x;
    if (left > 3) p[3] = b.y;
  }
}
__device__ __forceinline__ bool vec_rows(const void* p, int ld, int elem) {
  return (reinterpret_cast<uintptr_t>(p) & (4 * elem - 1)) == 0 && (ld & 3) == 0;
}
__device__ __forceinline__ int elem_size(int type) { return type == CWL_F32 ? 4 : 2; }

// Four consecutive elements of U (row r, columns c...), `left` of which exist.  A step's U is the gradient plus the momentum
// after it took the gradient in; with kUpdate the momentum is brought up to date here.
template <bool kUpdate>
__device__ __forceinline__ float4 load_u(const FactorCommon& a, const Factor& f, int r, int c, int left, bool vec_u, bool vec_m) {
  if (left <= 0) return make_float4(0.f, 0.f, 0.f, 0.f);
  const float4 g = load4(f.u, (int64_t)r * f.ldu + c, a.in_type, vec_u, left);
  if (!a.step) return g;
  float* at = f.m + (int64_t)r * f.ldm + c;
  float4 m = load4(at, 0, CWL_F32, vec_m, left);
  if (kUpdate) {
    m = make_float4(fmaf(a.beta, m.x, g.x), fmaf(a.beta, m.y, g.y), fmaf(a.beta, m.z, g.z), fmaf(a.beta, m.w, g.w));
    store4_f32(at, m, vec_m, left);
  }
  if (!a.nesterov) return m;
  return make_float4(fmaf(a.beta, m.x, g.x), fmaf(a.beta, m.y, g.y), fmaf(a.beta, m.z, g.z), fmaf(a.beta, m.w, g.w));
}

// 16 bytes from global to shared memory, of which `bytes` are read and the rest filled with zeros
__device__ __forceinline__ void copy16(void* to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

// Rows of this matrix can be copied 16 bytes at a time.
__device__ __forceinline__ bool wide_rows(const void* p, int ld, int elem) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ((int64_t)ld * elem & 15) == 0;
}
// D += A B, 8 x 8 x 4 in 64 bits.  Lane l holds A[l / 4][l % 4], B[l % 4][l / 4] and D[l / 4][2 (l % 4) + {0, 1}]: with B's
// columns as rows of a symmetric product both operands are read the same way.
__device__ __forceinline__ void mma_f64(double (&d)[2], double a, double b) {
  asm("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};" : "+d"(d[0]), "+d"(d[1]) : "d"(a), "d"(b));
}

__device__ __forceinline__ void lower_tile(int i, int& ti, int& tj) {
  ti = 0;
  while (i > ti) { i -= ti + 1; ++ti; }
  tj = i;
}

// 1 / (norm + eps) as Q and APPLY take it: what Q is multiplied with, and, where fp32 would not hold that times Q (norms near either
// end of its range), the powers of two, one after the other, that APPLY lifts U by instead.  Within 2^32 of 1 the latter are 1.
constexpr int kLiftFrom = 32;
struct SplitUnit { double of_q; float2 lift; };
__device__ __forceinline__ SplitUnit split_unit(double unit) {
  SplitUnit s{unit, make_float2(1.f, 1.f)};
  if (isfinite(unit) && unit != 0.0) {             // a factor that is not finite, or zeros
    const int e = ilogb(unit);
    if (e > kLiftFrom || e < -kLiftFrom) s = SplitUnit{scalbn(unit, -e), make_float2(scalbnf(1.f, e / 2), scalbnf(1.f, e - e / 2))};
  }
  return s;
}
__host__ __device__ __forceinline__ float2* lift_at(float* q, int64_t q_stride) { return reinterpret_cast<float2*>(q + q_stride) - 1; }

// ------------------------------------------------------------------------------------------------------------- GRAM
constexpr int kGramThreads = 256;
constexpr int kGramK = 32;                         // long-side elements staged at a time
constexpr int kGramLd = kGramK + 4;                // doubles a row
// Place of element k of row r.  Lanes of a fragment (four rows by four k) and lanes that store one k of sixteen rows hit
// sixteen different banks of 8 bytes.
__device__ __forceinline__ int gram_at(int r, int k) { return r * kGramLd + (k ^ (r >> 2 & 3)); }

// Raw rows in shared memory, kRun elements each, in pieces of 16 bytes.  The place of a piece depends on its row, so that lanes
// that read the same piece of neighbouring rows hit different banks.
template <int kRun, int kElem>
__device__ __forceinline__ int raw_turn(int row) {
  constexpr int kPitch = kRun * kElem;             // bytes: 64 or more
  return (kPitch < 128 ? row >> 1 : row) & 7 & (kPitch / 16 - 1);
}
// byte offset of element `at` (a multiple of 4) of a row
template <int kRun, int kElem>
__device__ __forceinline__ int raw_at(int row, int at) {
  return row * kRun * kElem + ((at * kElem) ^ (raw_turn<kRun, kElem>(row) << 4));
}
// What one thread copies of every chunk of kRows x kRun elements of a matrix: the same piece of rows some way apart.  Chunks follow
// one another along the rows or along the columns; places outside [.., r_end) x [.., c_end) read as zeros.
template <int kRows, int kRun, int kElem, int kThreads>
struct RawCopy {
  static constexpr int kPieces = kRun * kElem / 16, kStep = kThreads / kPieces, kEach = kRows / kStep;
  static_assert(kThreads % kPieces == 0 && kRows % kStep == 0 && kStep % 8 == 0, "every thread the same piece, at the same turn");
  const uint8_t* src;
  int64_t pitch;
  int to, row, col;
  __device__ __forceinline__ RawCopy(const void* from, int ld, int r0, int c0) {
    const int piece = threadIdx.x & (kPieces - 1);
    row = threadIdx.x / kPieces;
    col = c0 + piece * (16 / kElem);
    pitch = (int64_t)ld * kElem;
    src = static_cast<const uint8_t*>(from) + (r0 + row) * pitch + (int64_t)col * kElem;
    to = row * kRun * kElem + ((piece ^ raw_turn<kRun, kElem>(row)) << 4);
    row += r0;
  }
  // the chunk at (rows, columns) further on from the first one
  __device__ __forceinline__ void start(uint8_t* at, int rows, int cols, int r_end, int c_end) const {
    const int bytes = min(max(c_end - col - cols, 0) * kElem, 16);
    const uint8_t* p = src + rows * pitch + (int64_t)cols * kElem;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const bool there = row + rows + i * kStep < r_end && bytes > 0;
      copy16(at + to + i * kStep * kRun * kElem, there ? p + i * kStep * pitch : src, there ? bytes : 0);
    }
  }
};
template <int kElem>
__device__ __forceinline__ float4 raw_four(const uint8_t* at, bool bf16) {
  if (kElem == 4) return *reinterpret_cast<const float4*>(at);
  const uint2 q = *reinterpret_cast<const uint2*>(at);
  if (bf16)
    return make_float4(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16), __uint_as_float(q.y & 0xFFFF0000u));
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&q.x)), y = __half22float2(*reinterpret_cast<const __half2*>(&q.y));
  return make_float4(x.x, x.y, y.x, y.y);
}
// U of a step from gradient and momentum, both as they are now
__device__ __forceinline__ float4 step_u(const FactorCommon& a, const float4& g, const float4& m) {
  return a.nesterov ? make_float4(fmaf(a.beta, m.x, g.x), fmaf(a.beta, m.y, g.y), fmaf(a.beta, m.z, g.z), fmaf(a.beta, m.w, g.w)) : m;
}

// A block of 64 of the short side (from `first` on) by kGramK of the long side, on its way to shared memory in 64 bits.  Where rows
// allow it the raw elements of the next chunks are already on their way to a ring in shared memory; else they are read
// when they are wanted.
constexpr int kGramRing = 3;
constexpr int kGramRaw = 64 * kGramK * 4;          // bytes of a chunk, 4 an element at most
template <bool kTall, bool kStep, int kElem>
struct GramSide {
  static constexpr int kRows = kTall ? kGramK : 64, kRun = kTall ? 64 : kGramK;   // of a chunk as it lies in memory
  const FactorCommon& a;
  const Factor& f;
  bool wide, vec_u, vec_m, update;
  int first, k_begin, k_end;
  uint8_t* raw;                                    // [kGramRing][gradient, momentum][kGramRaw]
  RawCopy<kRows, kRun, kElem, kGramThreads> copy_u;
  RawCopy<kRows, kRun, 4, kGramThreads> copy_m;
  __device__ __forceinline__ GramSide(const FactorCommon& a_, const Factor& f_, bool wide_, bool vec_u_, bool vec_m_, bool update_, int first_, int k_begin_, int k_end_, uint8_t* raw_)
      : a(a_), f(f_), wide(wide_), vec_u(vec_u_), vec_m(vec_m_), update(update_), first(first_), k_begin(k_begin_), k_end(k_end_), raw(raw_),
        copy_u(f_.u, f_.ldu, kTall ? k_begin_ : first_, kTall ? first_ : k_begin_), copy_m(f_.m, f_.ldm, kTall ? k_begin_ : first_, kTall ? first_ : k_begin_) {}
  __device__ __forceinline__ uint8_t* piece(int slot, int which) const { return raw + (slot * (kStep ? 2 : 1) + which) * kGramRaw; }
  __device__ __forceinline__ void start(int k0, int slot) const {
    if (!wide || k0 >= k_end) return;
    const int R = short_side(f), on = k0 - k_begin, r_end = kTall ? k_end : R, c_end = kTall ? R : k_end;
    copy_u.start(piece(slot, 0), kTall ? on : 0, kTall ? 0 : on, r_end, c_end);
    if (kStep) copy_m.start(piece(slot, 1), kTall ? on : 0, kTall ? 0 : on, r_end, c_end);
  }
  __device__ __forceinline__ void put(double* to, int k0, int slot) const {
    const int R = short_side(f), tid = threadIdx.x;
    const bool bf16 = a.in_type == CWL_BF16;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // four neighbours of a row; lanes take neighbouring rows
      const int row = kTall ? tid & 31 : i * 32 + (tid & 15) + (tid >> 7) * 16, at = kTall ? i * 32 + (tid >> 5) * 4 : (tid >> 4 & 7) * 4;
      const int r = kTall ? k0 + row : first + row, c = kTall ? first + at : k0 + at;
      float4 u;
      if (wide) {
        const float4 g = raw_four<kElem>(piece(slot, 0) + raw_at<kRun, kElem>(row, at), bf16);
        u = g;
        if (kStep) {
          float4 m = *reinterpret_cast<const float4*>(piece(slot, 1) + raw_at<kRun, 4>(row, at));
          if (update) {
            m = make_float4(fmaf(a.beta, m.x, g.x), fmaf(a.beta, m.y, g.y), fmaf(a.beta, m.z, g.z), fmaf(a.beta, m.w, g.w));
            const int left = r < (kTall ? k_end : R) ? (kTall ? R : k_end) - c : 0;
            store4_f32(f.m + (int64_t)r * f.ldm + c, m, true, left);
          }
          u = step_u(a, g, m);
        }
      } else {
        const int left = r < (kTall ? k_end : R) ? (kTall ? R : k_end) - c : 0;
        u = update ? load_u<true>(a, f, r, c, left, vec_u, vec_m) : load_u<false>(a, f, r, c, left, vec_u, vec_m);
      }
      const float v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) to[kTall ? gram_at(at + j, row) : gram_at(row, at + j)] = (double)v[j];
    }
  }
};

template <bool kTall, bool kStep, int kElem>
__device__ __forceinline__ void gram_block(const FactorCommon& a, const Factor& f, uint8_t* gram_raw, double* out) {
  double* rows_i = reinterpret_cast<double*>(gram_raw);
  double* rows_j = rows_i + 64 * kGramLd;
  double* sums = rows_j;                           // 36 tiles of 64, where one block of rows is all there is
  static_assert(64 * kGramLd >= 36 * 64, "room for the tiles");
  uint8_t* ring = gram_raw + 2 * 64 * kGramLd * 8;
  const int R = short_side(f), n = long_side(f), pairs = block_pairs(R);
  const int unit = blockIdx.x - f.first;
  const int slice = unit / pairs;
  int bi = 0, bj = unit % pairs;
  while (bj > bi) { bj -= bi + 1; ++bi; }          // bj <= bi
  const int k_begin = slice * a.slice, k_end = min(n, k_begin + a.slice);
  const bool wide = wide_rows(f.u, f.ldu, kElem) && (!kStep || wide_rows(f.m, f.ldm, 4));
  const bool vec_u = vec_rows(f.u, f.ldu, kElem), vec_m = kStep && vec_rows(f.m, f.ldm, 4);
  // each element is read by one block only where R <= 64: the momentum is brought up to date there
  const GramSide<kTall, kStep, kElem> si(a, f, wide, vec_u, vec_m, kStep && R <= kShort, bi * 64, k_begin, k_end, ring);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, fr = lane >> 2, fc = lane & 3;

  auto pipeline = [&](auto start, auto put, auto multiply) {
#pragma unroll
    for (int i = 0; i < kGramRing - 1; ++i) { start(k_begin + i * kGramK, i); copies_commit(); }
    int slot = 0;
    for (int k0 = k_begin; k0 < k_end; k0 += kGramK) {
      copies_wait<kGramRing - 2>();
      __syncthreads();                             // the chunk has arrived; the one before is done with
      put(k0, slot);
      start(k0 + (kGramRing - 1) * kGramK, slot == 0 ? kGramRing - 1 : slot - 1);
      copies_commit();
      if (++slot == kGramRing) slot = 0;
      __syncthreads();
      multiply();
    }
    copies_wait<0>();
    __syncthreads();
  };
  if (bi == bj) {
    // 36 tiles of the lower triangle, 18 a warp; four warps take a quarter of the K steps each: eight fragments serve 18 products
    const int half = warp >> 2, quarter = warp & 3;
    double acc[18][2];
#pragma unroll
    for (int i = 0; i < 18; ++i) acc[i][0] = acc[i][1] = 0.0;
    pipeline([&](int k0, int slot) { si.start(k0, slot); }, [&](int k0, int slot) { si.put(rows_i, k0, slot); },
             [&]() {
#pragma unroll 1
               for (int s = quarter; s < kGramK / 4; s += 4) {
                 double x[8];
#pragma unroll
                 for (int t = 0; t < 8; ++t) x[t] = rows_i[gram_at(t * 8 + fr, s * 4 + fc)];
                 // in the order of rows: rows 0 to 4 and half of row 5, or the rest (a branch around each half: predicated
                 // products of the other half would take the unit's time all the same)
                 if (half == 0) {
#pragma unroll
                   for (int ti = 0; ti < 8; ++ti)
#pragma unroll
                     for (int tj = 0; tj <= ti; ++tj) {
                       const int at = ti * (ti + 1) / 2 + tj;
                       if (at < 18) mma_f64(acc[at < 18 ? at : 0], x[ti], x[tj]);
                     }
                 } else {
#pragma unroll
                   for (int ti = 0; ti < 8; ++ti)
#pragma unroll
                     for (int tj = 0; tj <= ti; ++tj) {
                       const int at = ti * (ti + 1) / 2 + tj;
                       if (at >= 18) mma_f64(acc[at < 18 ? 0 : at - 18], x[ti], x[tj]);
                     }
                 }
               }
             });
    // the quarters' sums, in their order
    for (int w = 0; w < 4; ++w) {
      if (quarter == w) {
#pragma unroll
        for (int i = 0; i < 18; ++i) {
          double2* to = reinterpret_cast<double2*>(sums + (half * 18 + i) * 64 + fr * 8 + fc * 2);
          double2 v = w == 0 ? make_double2(0.0, 0.0) : *to;
          v.x += acc[i][0];
          v.y += acc[i][1];
          *to = v;
        }
      }
      __syncthreads();
    }
    // as tiles of the lower triangle
    for (int at = threadIdx.x; at < 36 * 32; at += kGramThreads) reinterpret_cast<double2*>(out)[at] = reinterpret_cast<const double2*>(sums)[at];
  } else {
    // a warp a quadrant of 32 x 32 and half of the K steps
    const GramSide<kTall, kStep, kElem> sj(a, f, wide, vec_u, vec_m, false, bj * 64, k_begin, k_end, ring + kGramRing * (kStep ? 2 : 1) * kGramRaw);
    const int qi = (warp >> 1 & 1) * 32, qj = (warp & 1) * 32, half = warp >> 2;
    double acc[4][4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j][0] = acc[i][j][1] = 0.0;
    pipeline([&](int k0, int slot) { si.start(k0, slot); sj.start(k0, slot); },
             [&](int k0, int slot) { si.put(rows_i, k0, slot); sj.put(rows_j, k0, slot); },
             [&]() {
#pragma unroll
               for (int s = 0; s < kGramK / 8; ++s) {
                 double x[4], y[4];
#pragma unroll
                 for (int t = 0; t < 4; ++t) {
                   x[t] = rows_i[gram_at(qi + t * 8 + fr, (s * 2 + half) * 4 + fc)];
                   y[t] = rows_j[gram_at(qj + t * 8 + fr, (s * 2 + half) * 4 + fc)];
                 }
#pragma unroll
                 for (int ti = 0; ti < 4; ++ti)
#pragma unroll
                   for (int tj = 0; tj < 4; ++tj) mma_f64(acc[ti][tj], x[ti], y[tj]);
               }
             });
    static_assert(2 * 64 * kGramLd >= 64 * 64, "room for one half's sums");
    double2* met = reinterpret_cast<double2*>(rows_i);
    auto place = [&](int ti, int tj) { return ((qi + ti * 8 + fr) * 64 + qj + tj * 8 + fc * 2) / 2; };
    if (half == 1) {
#pragma unroll
      for (int ti = 0; ti < 4; ++ti)
#pragma unroll
        for (int tj = 0; tj < 4; ++tj) met[place(ti, tj)] = make_double2(acc[ti][tj][0], acc[ti][tj][1]);
    }
    __syncthreads();
    if (half == 0) {
#pragma unroll
      for (int ti = 0; ti < 4; ++ti)
#pragma unroll
        for (int tj = 0; tj < 4; ++tj) {
          const double2 v = met[place(ti, tj)];
          reinterpret_cast<double2*>(out)[place(ti, tj)] = make_double2(acc[ti][tj][0] + v.x, acc[ti][tj][1] + v.y);
        }
    }
  }
}
template <int kMost, bool kStep, int kElem>
__global__ void __launch_bounds__(kGramThreads, 2) gram_kernel(const __grid_constant__ FactorArgs<kMost> args) {
  extern __shared__ __align__(16) uint8_t gram_raw[];
  pdl_launch_dependents();
  pdl_wait();
  const Factor& f = args.f[find_factor(args.f, args.c.n, blockIdx.x)];
  double* out = args.c.partial + (int64_t)blockIdx.x * 64 * 64;
  if (f.rows > f.cols) gram_block<true, kStep, kElem>(args.c, f, gram_raw, out);
  else gram_block<false, kStep, kElem>(args.c, f, gram_raw, out);
}
// shared memory of GRAM: two blocks of rows in 64 bits, and the ring (twice, where a pair has two of them)
size_t gram_smem(bool step, bool pairs) { return (size_t)2 * 64 * kGramLd * 8 + (size_t)kGramRing * (step ? 2 : 1) * (pairs ? 2 : 1) * kGramRaw; }
// where entry (r, c), r >= c, of a 64 x 64 block on the diagonal lies among its tiles
__device__ __forceinline__ int lower_at(int r, int c) {
  const int ti = r >> 3, tj = c >> 3;
  return (ti * (ti + 1) / 2 + tj) * 64 + (r & 7) * 8 + (c & 7);
}

// Momentum of the factors whose elements GRAM reads more than once (R > 64).
constexpr int kMomentumThreads = 256;
template <int kMost>
__global__ void __launch_bounds__(kMomentumThreads) momentum_kernel(const __grid_constant__ FactorArgs<kMost> args) {
  pdl_launch_dependents();
  pdl_wait();
  const FactorCommon& a = args.c;
  const Factor& f = args.f[blockIdx.y];
  if (short_side(f) <= kShort) return;
  const bool vec_u = vec_rows(f.u, f.ldu, elem_size(a.in_type)), vec_m = vec_rows(f.m, f.ldm, 4);
  const int per_row = (f.cols + 3) / 4;
  const int64_t total = (int64_t)f.rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * kMomentumThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kMomentumThreads) {
    const int r = (int)(i / per_row), c = (int)(i % per_row) * 4;
    load_u<true>(a, f, r, c, f.cols - c, vec_u, vec_m);
  }
}

// Sums of the slices' partial products of factors of R <= 64, into the first slice's place: 64 entries a block, four groups of
// slices, so that one block does not read them all in a row.
constexpr int kSlicesThreads = 256;
template <int kMost>
__global__ void __launch_bounds__(kSlicesThreads) slices_kernel(const __grid_constant__ FactorArgs<kMost> args) {
  __shared__ double met[kSlicesThreads];
  pdl_launch_dependents();
  pdl_wait();
  const Factor& f = args.f[blockIdx.y];
  const int R = short_side(f), t8 = (R + 7) / 8, slices = (long_side(f) + args.c.slice - 1) / args.c.slice;
  if (R > kShort || (int)blockIdx.x >= t8 * (t8 + 1) / 2) return;
  double* part = args.c.partial + (int64_t)f.first * 64 * 64 + blockIdx.x * 64 + (threadIdx.x & 63);
  double s = 0.0;
#pragma unroll 8
  for (int k = threadIdx.x >> 6; k < slices; k += kSlicesThreads / 64) s += part[(int64_t)k * 64 * 64];
  met[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 64) part[0] = met[threadIdx.x] + met[threadIdx.x + 64] + met[threadIdx.x + 128] + met[threadIdx.x + 192];
}

// ---------------------------------------------------------------------------------------------------- ITERATE, R <= 64
constexpr int kIterThreads = 384;                  // 12 warps of three tiles: 36, the lower triangle of 8 x 8
constexpr int kIterTiles = 3;
constexpr int kIterLd = 68;                        // doubles a row
constexpr size_t kIterSmem = ((size_t)4 * 64 * kIterLd + 1) * 8;

// This warp's tiles of the lower triangle, neighbours in the order of rows.  Where the triangle is smaller, the last ones stand
// for the missing; they are not stored.
struct IterMine {
  int count, left[kIterTiles], right[kIterTiles], row[kIterTiles], col[kIterTiles];
  __device__ __forceinline__ IterMine(int n_tiles, int warp, int fr, int fc) {
    const int first = warp * kIterTiles;
    count = min(max(n_tiles - first, 0), kIterTiles);
#pragma unroll
    for (int i = 0; i < kIterTiles; ++i) {
      int ti, tj;
      lower_tile(min(first + i, n_tiles - 1), ti, tj);
      left[i] = (ti * 8 + fr) * kIterLd + fc;
      right[i] = (tj * 8 + fr) * kIterLd + fc;
      row[i] = ti * 8 + fr;
      col[i] = tj * 8 + fc * 2;
    }
  }
};
struct IterSums { double d[kIterTiles][2]; };
// Product of two symmetric, commuting matrices in shared memory.  The tiles advance together and the fragments of several K steps
// are on their way at once, without a branch in between.
__device__ __forceinline__ void iter_product(const double* x, const double* y, const IterMine& w, int k_steps, IterSums& t) {
#pragma unroll
  for (int i = 0; i < kIterTiles; ++i) t.d[i][0] = t.d[i][1] = 0.0;
  if (w.count == 0) return;
#pragma unroll 4
  for (int k = 0; k < k_steps; ++k) {
    double l[kIterTiles], r[kIterTiles];
#pragma unroll
    for (int i = 0; i < kIterTiles; ++i) { l[i] = x[w.left[i] + k * 4]; r[i] = y[w.right[i] + k * 4]; }
#pragma unroll
    for (int i = 0; i < kIterTiles; ++i) mma_f64(t.d[i], l[i], r[i]);
  }
}
template <typename F>
__device__ __forceinline__ void iter_store(double* to, const IterMine& w, const IterSums& t, F value) {
#pragma unroll
  for (int i = 0; i < kIterTiles; ++i) {
    if (i >= w.count) break;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = w.row[i], c = w.col[i] + j;
      const double v = value(r, c, t.d[i][j]);
      if (c <= r) {                                // one value for both halves
        to[r * kIterLd + c] = v;
        to[c * kIterLd + r] = v;
      }
    }
  }
}

template <int kMost>
__global__ void __launch_bounds__(kIterThreads) iterate_kernel(const __grid_constant__ FactorArgs<kMost> args) {
  const FactorCommon& a = args.c;
  extern __shared__ __align__(16) double iter_raw[];
  double* G = iter_raw;
  double* P = G + 64 * kIterLd;
  double* S = P + 64 * kIterLd;
  double* Q = S + 64 * kIterLd;
  double& size_slot = Q[64 * kIterLd];
  pdl_launch_dependents();
  pdl_wait();
  const Factor& f = args.f[blockIdx.x];
  const int R = short_side(f);
  if (R > kShort) return;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, fr = lane >> 2, fc = lane & 3;
  const double* part = a.partial + (int64_t)f.first * 64 * 64;
  const int t8 = (R + 7) / 8, n_tiles = t8 * (t8 + 1) / 2, k_steps = t8 * 2, used = t8 * 8;
#pragma unroll
  for (int e = 0; e < 36 * 64 / kIterThreads; ++e) {
    const int at = e * kIterThreads + tid;
    if (at >= n_tiles * 64) continue;
    const double v = part[at];
    int ti, tj;
    lower_tile(at >> 6, ti, tj);
    const int r = ti * 8 + (at >> 3 & 7), c = tj * 8 + (at & 7);
    if (r >= c) G[r * kIterLd + c] = G[c * kIterLd + r] = v;
  }
  __syncthreads();
  if (tid < 32) {
    double s = tid < R ? G[tid * kIterLd + tid] : 0.0;
    if (tid + 32 < R) s += G[(tid + 32) * kIterLd + tid + 32];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (tid == 0) size_slot = s;
  }
  __syncthreads();
  const double trace = size_slot, size = sqrt(trace) + a.eps;
  const double unit = trace == 0.0 ? 0.0 : 1.0 / size;        // a factor of zeros stays one
  for (int at = tid; at < used * 64; at += kIterThreads) G[(at >> 6) * kIterLd + (at & 63)] *= unit * unit;
  const IterMine mine(n_tiles, warp, fr, fc);
  IterSums t, u;
  for (int step = 0; step < a.steps; ++step) {
    const bool first = step == 0, last = step + 1 == a.steps;
    __syncthreads();
    iter_product(G, G, mine, k_steps, t);
    iter_store(P, mine, t, [&](int r, int c, double v) { return (r == c ? a.a : 0.0) + a.b * G[r * kIterLd + c] + a.c * v; });
    __syncthreads();
    if (!first) iter_product(P, Q, mine, k_steps, u);
    if (!last) iter_product(P, G, mine, k_steps, t);
    __syncthreads();
    if (first) {
      for (int at = tid; at < used * 64; at += kIterThreads) Q[(at >> 6) * kIterLd + (at & 63)] = P[(at >> 6) * kIterLd + (at & 63)];
    } else {
      iter_store(Q, mine, u, [](int, int, double v) { return v; });
    }
    if (last) break;
    iter_store(S, mine, t, [](int, int, double v) { return v; });
    __syncthreads();
    iter_product(P, S, mine, k_steps, t);
    iter_store(G, mine, t, [](int, int, double v) { return v; });
  }
  __syncthreads();
  float* q = a.q + blockIdx.x * a.q_stride;
  const SplitUnit split = split_unit(unit);
  for (int at = tid; at < R * R; at += kIterThreads) q[at] = (float)(Q[(at / R) * kIterLd + at % R] * split.of_q);
  if (tid == 0) *lift_at(q, a.q_stride) = split.lift;
}

// ------------------------------------------------------------------------------------------------- ITERATE, R > 64
// Matrices of padded size Rp (a multiple of 32) in the workspace, of which tiles of the lower half are computed, and mirrored.
struct BigArgs {
  int n, steps, slice;
  double a, b, c, eps;
  const double* partial;
  double* big;                                     // [factor of this list][G, P, S, Q, Q of the next step][stride]
  int64_t stride;
  double* unit;                                    // [factor of this list] what Q is multiplied with at the end
  float* q; int64_t q_stride;
  uint16_t which[kMostFactors], R[kMostFactors];   // place in the call's list, short side
  int first[kMostFactors], slices[kMostFactors];   // GRAM's blocks
};
static_assert(sizeof(BigArgs) <= 8 * 1024, "kernel parameters");
__host__ __device__ __forceinline__ int padded(int R) { return (R + 31) / 32 * 32; }

// Sums of GRAM's partial products, scaled: G_0.  Sixteen blocks a 64 x 64 pair, an entry a thread, whose slices are on their way
// before the trace's.
constexpr int kBigGramThreads = 256, kBigGramShare = 16;
static_assert(64 * 64 == kBigGramThreads * kBigGramShare, "an entry a thread");
__global__ void __launch_bounds__(kBigGramThreads) big_gram_kernel(const __grid_constant__ BigArgs a) {
  __shared__ double met[kBigGramThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const int R = a.R[blockIdx.y], pairs = block_pairs(R), slices = a.slices[blockIdx.y], pair = blockIdx.x / kBigGramShare;
  if (pair >= pairs) return;
  const int Rp = padded(R), tid = threadIdx.x;
  int bi = 0, bj = pair;
  while (bj > bi) { bj -= bi + 1; ++bi; }
  const double* part = a.partial + (int64_t)a.first[blockIdx.y] * 64 * 64;
  // of a block on the diagonal its tiles of the lower triangle are there, all of the others
  const int entries = (bi == bj ? 36 * 64 : 64 * 64) / kBigGramShare, at = (blockIdx.x % kBigGramShare) * entries + tid;
  double v = 0.0;
  if (tid < entries) {
#pragma unroll 16
    for (int k = 0; k < slices; ++k) v += part[((int64_t)k * pairs + pair) * 64 * 64 + at];
  }
  // the trace: every block adds it up in the same order
  double s = 0.0;
  for (int i = tid; i < R; i += kBigGramThreads) {
    const int b = i >> 6, p = b * (b + 1) / 2 + b;
#pragma unroll 16
    for (int k = 0; k < slices; ++k) s += part[((int64_t)k * pairs + p) * 64 * 64 + lower_at(i & 63, i & 63)];
  }
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((tid & 31) == 0) met[tid >> 5] = s;
  __syncthreads();
  double trace = 0.0;
  for (int w = 0; w < kBigGramThreads / 32; ++w) trace += met[w];
  const double unit = trace == 0.0 ? 0.0 : 1.0 / (sqrt(trace) + a.eps);
  double* G = a.big + (int64_t)blockIdx.y * 5 * a.stride;
  if (tid < entries) {
    int r = at >> 6, c = at & 63;
    if (bi == bj) {
      int ti, tj;
      lower_tile(at >> 6, ti, tj);
      r = ti * 8 + (at >> 3 & 7);
      c = tj * 8 + (at & 7);
    }
    const bool other_half = bi == bj && c > r;     // of a tile on the diagonal
    r += bi * 64;
    c += bj * 64;
    if (!other_half && r < Rp && c < Rp) G[(int64_t)r * Rp + c] = G[(int64_t)c * Rp + r] = v * unit * unit;
  }
  if (blockIdx.x == 0 && tid == 0) {
    const SplitUnit split = split_unit(unit);
    a.unit[blockIdx.y] = split.of_q;
    *lift_at(a.q + a.which[blockIdx.y] * a.q_stride, a.q_stride) = split.lift;
  }
}

// One product a launch (two where they do not depend on one another):
//   POLY    P = a I + b G + c G G; in the first step this is Q too
//   SPREAD  S = P G, and Q' = P Q (z = 1, or alone in the last step, where it leaves as fp32, times its unit)
//   GRAM    G = P S
enum : int { BIG_POLY = 0, BIG_SPREAD = 1, BIG_GRAM = 2 };
// A block takes 16 x 16 entries, each of its warps a quarter of the sums, which it brings in itself and waits for alone: at R = 256
// that is 136 blocks a factor (32 x 32 entries: 36, each with all of 2.2 us of products in one SM, twice that where P G and P Q go
// together).
constexpr int kBigThreads = 128;
constexpr int kBigTile = 16;
constexpr int kBigLd = CWL_MAX_RANK + 4;
constexpr size_t kBigSmem = (size_t)(2 * kBigTile * kBigLd + 4 * kBigTile * kBigTile) * 8;
__global__ void __launch_bounds__(kBigThreads) big_product_kernel(const __grid_constant__ BigArgs a, int what, int step) {
  extern __shared__ __align__(16) double big_raw[];
  pdl_launch_dependents();
  pdl_wait();
  const int R = a.R[blockIdx.y], Rp = padded(R);
  int ti = 0, tj = blockIdx.x;
  while (tj > ti) { tj -= ti + 1; ++ti; }
  if (ti >= Rp / kBigTile) return;
  const bool last = step + 1 == a.steps;
  double* G = a.big + (int64_t)blockIdx.y * 5 * a.stride;
  double* P = G + a.stride;
  double* S = P + a.stride;
  double* Q = S + a.stride + (step & 1) * a.stride;
  double* Q_next = S + a.stride + ((step + 1) & 1) * a.stride;
  const bool of_q = what == BIG_SPREAD && (last || blockIdx.z == 1);
  const double* x = what == BIG_POLY ? G : P;
  const double* y = what == BIG_GRAM ? S : of_q ? Q : G;
  double* to = what == BIG_POLY ? P : what == BIG_GRAM ? G : of_q ? Q_next : S;
  double* rows_x = big_raw;
  double* rows_y = rows_x + kBigTile * kBigLd;
  double* sums = rows_y + kBigTile * kBigLd;       // [warp][16][16]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, fr = lane >> 2, fc = lane & 3;
  const int share = Rp / 4, k_first = warp * share;        // Rp is a multiple of 32
  for (int r = 0; r < kBigTile; ++r) {
    for (int c = k_first + lane * 2; c < k_first + share; c += 64) {
      copy16(rows_x + r * kBigLd + c, x + (int64_t)(ti * kBigTile + r) * Rp + c, 16);
      copy16(rows_y + r * kBigLd + c, y + (int64_t)(tj * kBigTile + r) * Rp + c, 16);
    }
  }
  copies_commit();
  // what else this thread's entries are made of, on its way too
  constexpr int kOne = kBigTile * kBigTile, kMine = kOne / kBigThreads;
  double g[kMine] = {};
  if (what == BIG_POLY) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int e = tid + i * kBigThreads;
      g[i] = G[(int64_t)(ti * kBigTile + e / kBigTile) * Rp + tj * kBigTile + e % kBigTile];
    }
  }
  const double unit = of_q || (what == BIG_POLY && a.steps == 1) ? a.unit[blockIdx.y] : 0.0;
  copies_wait<0>();
  __syncwarp();
  double acc[2][2][2] = {};
#pragma unroll 4
  for (int k = k_first; k < k_first + share; k += 4) {
    double u[2], v[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u[t] = rows_x[(t * 8 + fr) * kBigLd + k + fc];
      v[t] = rows_y[(t * 8 + fr) * kBigLd + k + fc];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) mma_f64(acc[i][j], u[i], v[j]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < 2; ++k) sums[warp * kBigTile * kBigTile + (i * 8 + fr) * kBigTile + j * 8 + fc * 2 + k] = acc[i][j][k];
  __syncthreads();
  float* q = a.q + a.which[blockIdx.y] * a.q_stride;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int e = tid + i * kBigThreads;
    const int r = ti * kBigTile + e / kBigTile, c = tj * kBigTile + e % kBigTile;
    if (c > r) continue;                           // one value for both halves
    double v = (sums[e] + sums[e + kOne]) + (sums[e + 2 * kOne] + sums[e + 3 * kOne]);
    if (what == BIG_POLY) v = (r == c ? a.a : 0.0) + a.b * g[i] + a.c * v;
    if (last && (of_q || what == BIG_POLY && step == 0)) {
      if (r < R && c < R) q[(int64_t)r * R + c] = q[(int64_t)c * R + r] = (float)(v * unit);
      if (of_q) continue;
    }
    to[(int64_t)r * Rp + c] = v;
    to[(int64_t)c * Rp + r] = v;
    if (what == BIG_POLY && step == 0) {
      Q_next[(int64_t)r * Rp + c] = v;
      Q_next[(int64_t)c * Rp + r] = v;
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ APPLY
// O = Q U over 64 short-side rows and 128 long-side elements.  Outputs of a thread: 8 x 4 with the lanes along the rows of the
// factor as they lie in memory, whichever side that is.
constexpr int kApplyThreads = 256;
constexpr int kApplyK = 32;
constexpr int kApplyLdX = kApplyLong + 4, kApplyLdQ = kApplyShort + 4;

template <bool kTall, bool kStep, int kElem>
__device__ __forceinline__ void apply_tile(const FactorCommon& a, const Factor& f, const float* q, float2 lift, int long0, int short0, float* xs, float* qs) {
  const int R = short_side(f), n = long_side(f), tid = threadIdx.x;
  const bool vec_u = vec_rows(f.u, f.ldu, kElem), vec_m = kStep && vec_rows(f.m, f.ldm, 4);
  const bool vec_q = (R & 3) == 0;
  // this thread's outputs: short side s0.., long side l0..
  constexpr int kS = kTall ? 4 : 8, kL = kTall ? 8 : 4;
  const int s0 = kTall ? (tid & 15) * 4 : (tid >> 5) * 8, l0 = kTall ? (tid >> 4) * 8 : (tid & 31) * 4;
  float acc[kS][kL];
#pragma unroll
  for (int i = 0; i < kS; ++i)
#pragma unroll
    for (int j = 0; j < kL; ++j) acc[i][j] = 0.f;

  // What comes next is loaded raw, all loads together, and becomes U when it is put into shared memory.
  float4 x[4], mom[kStep ? 4 : 1], y[2];
  const bool inside = vec_u && (!kStep || vec_m) && (kTall ? (R & 3) == 0 : (n & 3) == 0);
  auto place = [&](int k0, int i, int& r, int& c) {
    if (kTall) { r = long0 + i * 32 + (tid >> 3); c = k0 + (tid & 7) * 4; }      // U [long][short]: eight threads 32 of a row
    else { r = k0 + i * 8 + (tid >> 5); c = long0 + (tid & 31) * 4; }            // U [short][long]: a warp 128 of a row
    return r < f.rows ? f.cols - c : 0;
  };
  auto fetch = [&](int k0) {
    int r, c;
    if (inside) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = place(k0, i, r, c) > 0;
        const int64_t at = (int64_t)r * f.ldu + c;
        if (kElem == 4) {
          x[i] = there ? *reinterpret_cast<const float4*>(static_cast<const float*>(f.u) + at) : make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
          const float2 q = there ? *reinterpret_cast<const float2*>(static_cast<const uint16_t*>(f.u) + at) : make_float2(0.f, 0.f);
          x[i].x = q.x;
          x[i].y = q.y;
        }
        if (kStep) mom[kStep ? i : 0] = there ? *reinterpret_cast<const float4*>(f.m + (int64_t)r * f.ldm + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int left = place(k0, i, r, c);
        x[i] = load_u<false>(a, f, r, c, left, vec_u, vec_m);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {                  // Q is symmetric: its row k is the column wanted
      const int k = k0 + i * 16 + (tid >> 4), s = short0 + (tid & 15) * 4, left = k < R ? R - s : 0;
      y[i] = load4(q, (int64_t)k * R + s, CWL_F32, vec_q, left);
    }
  };
  const bool lifted = lift.x != 1.f || lift.y != 1.f;
  auto made = [&](int i) {                         // U from what was loaded
    float4 u = x[i];
    if (inside) {
      u = raw_four<kElem>(reinterpret_cast<const uint8_t*>(&x[i]), a.in_type == CWL_BF16);
      if (kStep) u = step_u(a, u, mom[kStep ? i : 0]);
    }
    if (lifted) u = make_float4(u.x * lift.x * lift.y, u.y * lift.x * lift.y, u.z * lift.x * lift.y, u.w * lift.x * lift.y);
    return u;
  };
  fetch(0);
  for (int k0 = 0; k0 < R; k0 += kApplyK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 u = made(i);
      if (kTall) {
        const int l = i * 32 + (tid >> 3), k = (tid & 7) * 4;
        xs[k * kApplyLdX + l] = u.x; xs[(k + 1) * kApplyLdX + l] = u.y;
        xs[(k + 2) * kApplyLdX + l] = u.z; xs[(k + 3) * kApplyLdX + l] = u.w;
      } else {
        *reinterpret_cast<float4*>(xs + (i * 8 + (tid >> 5)) * kApplyLdX + (tid & 31) * 4) = u;
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<float4*>(qs + (i * 16 + (tid >> 4)) * kApplyLdQ + (tid & 15) * 4) = y[i];
    __syncthreads();
    if (k0 + kApplyK < R) fetch(k0 + kApplyK);
#pragma unroll 8
    for (int k = 0; k < kApplyK; ++k) {
      float sv[kS], lv[kL];
#pragma unroll
      for (int i = 0; i < kS; i += 4) *reinterpret_cast<float4*>(sv + i) = *reinterpret_cast<const float4*>(qs + k * kApplyLdQ + s0 + i);
#pragma unroll
      for (int j = 0; j < kL; j += 4) *reinterpret_cast<float4*>(lv + j) = *reinterpret_cast<const float4*>(xs + k * kApplyLdX + l0 + j);
#pragma unroll
      for (int i = 0; i < kS; ++i)
#pragma unroll
        for (int j = 0; j < kL; ++j) acc[i][j] = fmaf(sv[i], lv[j], acc[i][j]);
    }
  }

  const int out_type = kStep ? CWL_F32 : a.out_type;
  const bool vec_o = vec_rows(f.out, f.ldo, elem_size(out_type)), vec_l = f.low != nullptr && vec_rows(f.low, f.ldl, 2);
  const float by = kStep ? -a.lr * f.scale : 1.f;
  // four neighbours of a row of the factor at a time; a step's masters all come in before the first is written back
  auto at_output = [&](int i, int& r, int& c) {
    r = kTall ? long0 + l0 + i : short0 + s0 + i;
    c = kTall ? short0 + s0 : long0 + l0;
    return r < f.rows ? f.cols - c : 0;
  };
  int r, c;
  float4 p[kStep ? 8 : 1];
  if (kStep) {
    const bool whole = vec_o && (f.cols & 3) == 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int left = at_output(i, r, c);
      const float* at = static_cast<const float*>(f.out) + (int64_t)r * f.ldo + c;
      if (whole) p[kStep ? i : 0] = left > 0 ? *reinterpret_cast<const float4*>(at) : make_float4(0.f, 0.f, 0.f, 0.f);
      else p[kStep ? i : 0] = load4(at, 0, CWL_F32, vec_o, left);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int left = at_output(i, r, c);
    if (left <= 0) continue;
    float4 v = kTall ? make_float4(acc[0][i % kL], acc[1 % kS][i % kL], acc[2 % kS][i % kL], acc[3 % kS][i % kL])
                     : make_float4(acc[i % kS][0], acc[i % kS][1 % kL], acc[i % kS][2 % kL], acc[i % kS][3 % kL]);
    if (kStep) {
      const float4 was = p[kStep ? i : 0];
      v = make_float4(fmaf(by, v.x, a.keep * was.x), fmaf(by, v.y, a.keep * was.y), fmaf(by, v.z, a.keep * was.z), fmaf(by, v.w, a.keep * was.w));
      store4_f32(static_cast<float*>(f.out) + (int64_t)r * f.ldo + c, v, vec_o, left);
      if (f.low != nullptr) store4_bf16(f.low + (int64_t)r * f.ldl + c, v, vec_l, left);
    } else if (out_type == CWL_F32) {
      store4_f32(static_cast<float*>(f.out) + (int64_t)r * f.ldo + c, v, vec_o, left);
    } else {
      store4_bf16(static_cast<__nv_bfloat16*>(f.out) + (int64_t)r * f.ldo + c, v, vec_o, left);
    }
  }
}

template <int kMost, bool kStep, int kElem>
__global__ void __launch_bounds__(kApplyThreads, 2) apply_factors_kernel(const __grid_constant__ FactorArgs<kMost> args) {
  __shared__ __align__(16) float xs[kApplyK * kApplyLdX], qs[kApplyK * kApplyLdQ];
  pdl_launch_dependents();
  pdl_wait();
  const int at = find_factor(args.f, args.c.n, blockIdx.x);
  const Factor& f = args.f[at];
  const int unit = blockIdx.x - f.first, row_tiles = (short_side(f) + kApplyShort - 1) / kApplyShort;
  const int long0 = unit / row_tiles * kApplyLong, short0 = unit % row_tiles * kApplyShort;
  float* q = args.c.q + at * args.c.q_stride;
  const float2 lift = *lift_at(q, args.c.q_stride);
  if (f.rows > f.cols) apply_tile<true, kStep, kElem>(args.c, f, q, lift, long0, short0, xs, qs);
  else apply_tile<false, kStep, kElem>(args.c, f, q, lift, long0, short0, xs, qs);
}

// ------------------------------------------------------------------------------------------------------------- host
size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Long-side elements a block of GRAM: short enough that the blocks fill the GPU evenly, long enough that their sums
// (32 KB a block) stay a small part of what is read.
constexpr int64_t kGramBlocks = 2400;
constexpr int kGramLeast = 128, kGramLeastBig = 256;
struct FactorPlan { int slice, n_big, most_R; int64_t blocks; size_t partial, q, big, unit, total; int64_t q_stride, stride; };
template <typename Item>
FactorPlan factor_plan(const Item* items, int n) {
  FactorPlan p = {};
  int64_t work = 0;
  int big = 0;
  for (int i = 0; i < n; ++i) {
    const int R = items[i].rows < items[i].cols ? items[i].rows : items[i].cols, len = items[i].rows < items[i].cols ? items[i].cols : items[i].rows;
    work += (int64_t)block_pairs(R) * len;
    if (R > p.most_R) p.most_R = R;
    if (R > kShort) { ++p.n_big; if (R > big) big = R; }
  }
  int64_t slice = (work + kGramBlocks - 1) / kGramBlocks;
  slice = (slice + kGramK - 1) / kGramK * kGramK;
  const int least = p.n_big > 0 ? kGramLeastBig : kGramLeast;
  if (slice < least) slice = least;
  if (slice > 1 << 20) slice = 1 << 20;
  p.slice = (int)slice;
  for (int i = 0; i < n; ++i) {
    const int R = items[i].rows < items[i].cols ? items[i].rows : items[i].cols, len = items[i].rows < items[i].cols ? items[i].cols : items[i].rows;
    p.blocks += (int64_t)block_pairs(R) * ceil_div(len, p.slice);
  }
  p.q_stride = ((int64_t)p.most_R * p.most_R + 3) / 4 * 4 + 4;
  p.stride = (int64_t)padded(big) * padded(big);
  p.q = align256((size_t)p.blocks * 64 * 64 * 8);
  p.big = p.q + align256((size_t)p.q_stride * n * 4);
  p.unit = p.big + align256((size_t)p.stride * 5 * p.n_big * 8);
  p.total = p.unit + align256((size_t)p.n_big * 8);
  return p;
}

// Items are worked on in groups whose descriptors fit a launch; the groups follow one another and share the workspace.
template <typename Item>
size_t factor_bytes(const Item* items, int n) {
  size_t most = 0;
  for (int i = 0; i < n; i += kMostFactors) {
    const size_t b = factor_plan(items + i, n - i < kMostFactors ? n - i : kMostFactors).total;
    if (b > most) most = b;
  }
  return most;
}

template <int kMost, bool kStep, int kElem>
cudaError_t launch_gram(const FactorArgs<kMost>& args, int64_t blocks, bool pairs, bool chained, cudaStream_t st) {
  static SharedMemoryGrant grant;
  const cudaError_t e = grant(gram_kernel<kMost, kStep, kElem>);
  if (e != cudaSuccess) return e;
  return launch_chained(chained, gram_kernel<kMost, kStep, kElem>, dim3((unsigned)blocks), dim3(kGramThreads), gram_smem(kStep, pairs), st, args);
}
template <int kMost, bool kStep, int kElem>
cudaError_t launch_apply(const FactorArgs<kMost>& args, int64_t blocks, bool chained, cudaStream_t st) {
  return launch_chained(chained, apply_factors_kernel<kMost, kStep, kElem>, dim3((unsigned)blocks), dim3(kApplyThreads), 0, st, args);
}

template <int kMost, bool kStep, int kElem, typename Item, typename Fill>
cwl_status run_group(const Item* items, int n, FactorCommon common, Fill fill, void* workspace, bool chained, cudaStream_t st) {
  const FactorPlan plan = factor_plan(items, n);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  FactorArgs<kMost> args;
  args.c = common;
  args.c.n = n;
  args.c.slice = plan.slice;
  args.c.partial = reinterpret_cast<double*>(ws);
  args.c.q = reinterpret_cast<float*>(ws + plan.q);
  args.c.q_stride = plan.q_stride;
  BigArgs big;
  big.n = 0; big.steps = common.steps; big.slice = plan.slice;
  big.a = common.a; big.b = common.b; big.c = common.c; big.eps = common.eps;
  big.partial = args.c.partial;
  big.big = reinterpret_cast<double*>(ws + plan.big); big.stride = plan.stride;
  big.unit = reinterpret_cast<double*>(ws + plan.unit);
  big.q = args.c.q; big.q_stride = plan.q_stride;
  int64_t gram_blocks = 0, blocks = 0;
  bool any_small = false;
  int most_R = 0, most_slices = 0;
  int64_t most_elements = 0;
  for (int i = 0; i < n; ++i) {
    Factor& f = args.f[i];
    f = Factor{};
    f.rows = items[i].rows; f.cols = items[i].cols;
    fill(items[i], f);
    f.first = (int)gram_blocks;
    const int R = short_side(f), slices = ceil_div(long_side(f), plan.slice);
    if (R > kShort) {
      big.which[big.n] = (uint16_t)i; big.R[big.n] = (uint16_t)R; big.first[big.n] = f.first; big.slices[big.n] = slices;
      ++big.n;
      if (R > most_R) most_R = R;
      const int64_t e = (int64_t)f.rows * f.cols;
      if (e > most_elements) most_elements = e;
    } else {
      any_small = true;
      if (slices > most_slices) most_slices = slices;
    }
    gram_blocks += (int64_t)block_pairs(R) * slices;
  }
  if (common.step && big.n > 0) {
    const int64_t x = (most_elements / 4 + kMomentumThreads * 4 - 1) / (kMomentumThreads * 4);
    CWL_CUDA_TRY(launch_chained(chained, momentum_kernel<kMost>, dim3((unsigned)(x < 592 ? x + 1 : 592), (unsigned)n), dim3(kMomentumThreads), 0, st, args));
  }
  CWL_CUDA_TRY((launch_gram<kMost, kStep, kElem>(args, gram_blocks, big.n > 0, chained, st)));
  if (any_small) {
    if (most_slices > 1)
      CWL_CUDA_TRY(launch_chained(chained, slices_kernel<kMost>, dim3(36, (unsigned)n), dim3(kSlicesThreads), 0, st, args));
    static SharedMemoryGrant grant;
    CWL_CUDA_TRY(grant(iterate_kernel<kMost>));
    CWL_CUDA_TRY(launch_chained(chained, iterate_kernel<kMost>, dim3((unsigned)n), dim3(kIterThreads), kIterSmem, st, args));
  }
  if (big.n > 0) {
    static SharedMemoryGrant grant;
    CWL_CUDA_TRY(grant(big_product_kernel));
    CWL_CUDA_TRY(launch_chained(chained, big_gram_kernel, dim3((unsigned)(block_pairs(most_R) * kBigGramShare), (unsigned)big.n), dim3(kBigGramThreads), 0, st, big));
    const int t = padded(most_R) / kBigTile, tiles = t * (t + 1) / 2;
    for (int step = 0; step < common.steps; ++step) {
      const bool last = step + 1 == common.steps;
      auto product = [&](int what, int z) {
        return launch_chained(chained, big_product_kernel, dim3((unsigned)tiles, (unsigned)big.n, (unsigned)z), dim3(kBigThreads), kBigSmem, st, big, what, step);
      };
      CWL_CUDA_TRY(product(BIG_POLY, 1));
      if (last && step == 0) break;
      CWL_CUDA_TRY(product(BIG_SPREAD, step == 0 || last ? 1 : 2));
      if (!last) CWL_CUDA_TRY(product(BIG_GRAM, 1));
    }
  }
  for (int i = 0; i < n; ++i) {
    args.f[i].first = (int)blocks;
    blocks += apply_blocks(args.f[i]);
  }
  CWL_CUDA_TRY((launch_apply<kMost, kStep, kElem>(args, blocks, chained, st)));
  return CWL_OK;
}

// A factor's matrices read and written by the same call, by different blocks: none may lie in another's place.
bool shares_memory(const cwl_factor& f, bool step, int in_bytes, int out_bytes) {
  const MatrixSpan at[4] = {matrix_span(f.grad, f.ld_grad, f.rows, f.cols, in_bytes), matrix_span(f.out, f.ld_out, f.rows, f.cols, out_bytes),
                            matrix_span(f.momentum, f.ld_momentum, f.rows, f.cols, 4), matrix_span(f.low, f.ld_low, f.rows, f.cols, 2)};
  for (int i = 0; i < (step ? 4 : 2); ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(at[i], at[j])) return true;
  return false;
}

template <bool kStep, typename Item, typename Fill>
cwl_status run_factors(const Item* items, int n, const FactorCommon& common, Fill fill, void* workspace, size_t workspace_bytes, void* stream) {
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < factor_bytes(items, n)) return CWL_ERR_WORKSPACE;
  for (int i = 0; i < n; ++i)
    if (shares_memory(items[i], kStep, common.in_type == CWL_F32 ? 4 : 2, common.out_type == CWL_F32 ? 4 : 2)) return CWL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool chained = !stream_is_capturing(st);
  for (int i = 0; i < n; i += kMostFactors) {
    const int m = n - i < kMostFactors ? n - i : kMostFactors;
    const bool f32 = common.in_type == CWL_F32;
    const cwl_status s = m <= kFewFactors ? (f32 ? run_group<kFewFactors, kStep, 4>(items + i, m, common, fill, workspace, chained, st)
                                                 : run_group<kFewFactors, kStep, 2>(items + i, m, common, fill, workspace, chained, st))
                                          : (f32 ? run_group<kMostFactors, kStep, 4>(items + i, m, common, fill, workspace, chained, st)
                                                 : run_group<kMostFactors, kStep, 2>(items + i, m, common, fill, workspace, chained, st));
    if (s != CWL_OK) return s;
  }
  return CWL_OK;
}

bool bad_type(cwl_dtype t) { return t != CWL_F32 && t != CWL_BF16 && t != CWL_F16; }
cwl_status check_iteration(const cwl_newton_schulz* ns) {
  if (ns == nullptr || ns->steps < 1 || ns->steps > CWL_MAX_NS_STEPS) return CWL_ERR_INVALID_ARG;
  if (!isfinite(ns->a) || !isfinite(ns->b) || !isfinite(ns->c) || !(ns->eps >= 0.0) || !isfinite(ns->eps)) return CWL_ERR_INVALID_ARG;
  return CWL_OK;
}
constexpr int kMostLong = 1 << 22;
cwl_status check_size(int rows, int cols) {
  if (rows < 1 || cols < 1) return CWL_ERR_INVALID_ARG;
  const int R = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
  return R > CWL_MAX_RANK || n > kMostLong ? CWL_ERR_UNSUPPORTED : CWL_OK;
}
// element alignment, and rows that do not run into one another
bool bad_rows(const void* p, int64_t ld, int rows, int cols, int elem) {
  return (reinterpret_cast<uintptr_t>(p) % elem) != 0 || (rows > 1 && ld < cols) || ld > INT32_MAX || ld < 0;
}
int row_step(int64_t ld, int rows, int cols) { return rows > 1 ? (int)ld : cols; }
int type_bytes(cwl_dtype t) { return t == CWL_F32 ? 4 : 2; }

}  // namespace
}  // namespace cwl

extern "C" size_t cwl_orthogonalize_workspace_bytes(const cwl_factor* factors, int32_t n) {
  if (factors == nullptr || n <= 0) return 0;
  for (int i = 0; i < n; ++i)
    if (cwl::check_size(factors[i].rows, factors[i].cols) != CWL_OK) return 0;
  return cwl::factor_bytes(factors, n);
}

extern "C" cwl_status cwl_orthogonalize(const cwl_factor* factors, int32_t n, cwl_dtype in_dtype, cwl_dtype out_dtype,
                                        const cwl_newton_schulz* iteration, void* workspace, size_t workspace_bytes, void* stream) try {
  using namespace cwl;
  if (n < 0 || (n > 0 && factors == nullptr)) return CWL_ERR_INVALID_ARG;
  if (bad_type(in_dtype) || (out_dtype != CWL_F32 && out_dtype != CWL_BF16)) return CWL_ERR_INVALID_ARG;
  cwl_status s = check_iteration(iteration);
  if (s != CWL_OK) return s;
  for (int i = 0; i < n; ++i) {
    const cwl_factor& f = factors[i];
    if ((s = check_size(f.rows, f.cols)) != CWL_OK) return s;
    if (f.grad == nullptr || f.out == nullptr) return CWL_ERR_INVALID_ARG;
    if (bad_rows(f.grad, f.ld_grad, f.rows, f.cols, type_bytes(in_dtype)) || bad_rows(f.out, f.ld_out, f.rows, f.cols, type_bytes(out_dtype))) return CWL_ERR_SHAPE;
  }
  if (n == 0) return CWL_OK;
  FactorCommon c = {};
  c.in_type = in_dtype; c.out_type = out_dtype;
  c.steps = iteration->steps; c.a = iteration->a; c.b = iteration->b; c.c = iteration->c; c.eps = iteration->eps;
  return run_factors<false>(factors, n, c, [](const cwl_factor& i, Factor& f) {
    f.u = i.grad; f.out = i.out;
    f.ldu = row_step(i.ld_grad, i.rows, i.cols); f.ldo = row_step(i.ld_out, i.rows, i.cols);
  }, workspace, workspace_bytes, stream);
} catch (...) {
  return CWL_ERR_CUDA;                                   // nothing may leave a C entry
}

extern "C" cwl_status cwl_factor_step(const cwl_factor* factors, int32_t n, cwl_dtype grad_dtype, const cwl_newton_schulz* iteration,
                                      float lr, float momentum, float weight_decay, int32_t nesterov,
                                      void* workspace, size_t workspace_bytes, void* stream) try {
  using namespace cwl;
  if (n < 0 || (n > 0 && factors == nullptr) || bad_type(grad_dtype)) return CWL_ERR_INVALID_ARG;
  if (!isfinite(lr) || !isfinite(weight_decay) || !(momentum >= 0.f) || !(momentum < 1.f)) return CWL_ERR_INVALID_ARG;
  cwl_status s = check_iteration(iteration);
  if (s != CWL_OK) return s;
  for (int i = 0; i < n; ++i) {
    const cwl_factor& f = factors[i];
    if ((s = check_size(f.rows, f.cols)) != CWL_OK) return s;
    if (f.grad == nullptr || f.momentum == nullptr || f.out == nullptr || !isfinite(f.scale)) return CWL_ERR_INVALID_ARG;
    if (bad_rows(f.grad, f.ld_grad, f.rows, f.cols, type_bytes(grad_dtype)) || bad_rows(f.momentum, f.ld_momentum, f.rows, f.cols, 4) ||
        bad_rows(f.out, f.ld_out, f.rows, f.cols, 4) || (f.low != nullptr && bad_rows(f.low, f.ld_low, f.rows, f.cols, 2)))
      return CWL_ERR_SHAPE;
  }
  if (n == 0) return CWL_OK;
  FactorCommon c = {};
  c.step = 1; c.nesterov = nesterov != 0; c.in_type = grad_dtype; c.out_type = CWL_F32;
  c.beta = momentum; c.keep = (float)(1.0 - (double)lr * weight_decay); c.lr = lr;
  c.steps = iteration->steps; c.a = iteration->a; c.b = iteration->b; c.c = iteration->c; c.eps = iteration->eps;
  return run_factors<true>(factors, n, c, [](const cwl_factor& i, Factor& f) {
    f.u = i.grad; f.m = static_cast<float*>(i.momentum); f.out = i.out; f.low = static_cast<__nv_bfloat16*>(i.low);
    f.ldu = row_step(i.ld_grad, i.rows, i.cols); f.ldm = row_step(i.ld_momentum, i.rows, i.cols);
    f.ldo = row_step(i.ld_out, i.rows, i.cols); f.ldl = row_step(i.ld_low, i.rows, i.cols);
    f.scale = i.scale;
  }, workspace, workspace_bytes, stream);
} catch (...) {
  return CWL_ERR_CUDA;                                   // nothing may leave a C entry
}

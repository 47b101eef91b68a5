// cwl_token_logprobs: what a logit row says about given tokens -- their log-probability, the row's log-sum-exp and entropy,
// and the top alternatives.
//
//   m = max z,  S = sum e^((z-m)/tau):   lse = m/tau + ln S,   H = ln S - (1/S) sum (z-m)/tau e^((z-m)/tau),
//   logprob(y) = (z_y - m)/tau - ln S,   top K by (z descending, index ascending)
//
// The row is read once.  Every thread keeps the online triple of its own elements and the maximum of each of up to eight
// runs of them (its cells; the batch maxima that the triple needs anyway).  The K-th largest of the maxima of the threads'
// even and odd cells is a lower bound of the row's K-th largest logit, and only cells whose maximum reaches it can hold one of the
// top K: a few per cent of the row are read a second time (from L2), and what reaches the bound is sorted in shared memory.
//
// What bounds it: without alternatives the one pass over the logits (2048 rows of 32000 fp32: 42 to 45 us, 6.2 to 5.9 TB/s; 16384
// rows of 32000 bf16: 163 us, 6.4 TB/s); with K = 64 the instructions of a row and its serial phases (16384 rows of 32000 bf16: 265
// to 276 us, 3.9 TB/s, issue slots 63 % active; 12300 warp instructions a row, of which 6950 are the pass itself, 2100 the cells and
// the fixed part of the selection and 3200 the second reads, the 64 places and their sort).  16384 rows of 500 fp32 with K = 64: 132
// us.  Few rows are cut up over a cluster: one row of 32000 fp32 with K = 20 in 7.5 us (launch, one pass of 16 KB a block, selection,
// the leader's merge), 64 bf16 rows in 10.4 us.
// A warp a row instead of four (24 rows an SM): 263 -> 350 us; the serial parts of a row then take four times as long.  Eight
// blocks an SM instead of seven: 266 -> 271.  Rows cut in two where they do not fill the GPU (777 of 50021 fp32): 32 -> 40.
#include <cmath>

#include "logits_common.cuh"

namespace cwl {
namespace {

constexpr int kLpThreads = 128;       // small blocks, seven to an SM: while one row selects, others stream
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpBatch = 4;           // 16-byte loads in flight per thread
constexpr int kLpBatchVecs = kLpThreads * kLpBatch;
constexpr int kSegs = 8;              // cells per thread
constexpr int kMaxCand = 1152;        // logits above the bound kept for sorting; with fewer than K threads that hold
                                      // anything a slice has at most (CWL_MAX_TOP_K - 1) * 8 + 14 elements, which fit
constexpr int kMaxVecs = 256;         // vectors that reach the bound, gathered in the place of the cells (4 KB) and maxima (1 KB)
constexpr int kMaxTies = 256;         // logits equal to the bound kept for sorting
constexpr int kMaxLpCluster = 8;
constexpr uint32_t kKeyOfMinusInf = 0x007FFFFFu;
constexpr uint32_t kKeyOfMinusZero = 0x7FFFFFFFu;      // no element's: -0 and 0 share the next one

struct LogprobParams {
  const void* logits; int64_t ld; int T, V;
  const int32_t* targets;
  float c, inv_temp;          // log2(e) / temperature, 1 / temperature
  int ordinary;               // temperature within what the short form of the exponent takes
  int top_k;
  float *logprob, *lse, *entropy;
  int32_t* top_ids; float* top_logprobs;
  int32_t* status_word;
};

// larger logit first, lower index first among equals: a larger 64-bit number comes first
__device__ __forceinline__ unsigned long long rank_key(uint32_t key, int idx) {
  return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)idx);
}

struct LpShared {
  alignas(16) unsigned long long cand[kMaxCand + 2];   // candidates
  alignas(16) uint32_t cell[kSegs * kLpThreads];       // order key of every cell's maximum, 0 for an empty cell
  uint32_t half[2 * kLpThreads];                       // the largest of a thread's even cells, of its odd ones
  RowStat part[kLpWarps];
  uint32_t hist[256];
  int ties[kMaxTies];
  int warp_count[kLpWarps];
  uint16_t hits[kSegs * kLpThreads];
  uint32_t thr;
  int n_hits, n_cand, n_ties, n_vecs, rest;
};
// Shared memory of the leader of a cluster that the others write: every CTA's sorted list (top_k places each, a shorter
// one ends in zeros), then every CTA's triple.
static_assert(kMaxLpCluster * CWL_MAX_TOP_K <= kMaxCand, "all lists fit the candidate buffer");
extern __shared__ __align__(16) unsigned long long lp_lists[];
inline size_t lp_lists_bytes(int n_cta, int top_k) { return (size_t)n_cta * (top_k * sizeof(unsigned long long) + 16); }

// Appends the lowest-index elements whose key equals `key` to the candidates until `need` are found.
template <typename T>
__device__ __noinline__ void append_ties_in_order(LpShared& sh, const T* z, int e0, int e1, uint32_t key, int have, int need) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  int found = 0;
  for (uint32_t base = e0; base < (uint32_t)e1 && found < need; base += kLpThreads) {    // unsigned: e1 may be 2^31 - 1
    const uint32_t i = base + tid;
    const bool is = i < (uint32_t)e1 && order_key(Elem<T>::load(z + i)) == key;
    const unsigned bal = __ballot_sync(0xffffffffu, is);
    if (lane == 0) sh.warp_count[wid] = __popc(bal);
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kLpWarps; ++w) {
      if (w < wid) before += sh.warp_count[w];
      all += sh.warp_count[w];
    }
    const int pos = found + before + __popc(bal & ((1u << lane) - 1u));
    if (is && pos < need) sh.cand[have + pos] = rank_key(key, i);
    found += all;
    __syncthreads();
  }
}

// The want-th largest of the threads' half maxima, rounded down to its first bits (all that a 16-bit type has, 16 of
// fp32: a bound that is up to 1/128 lower admits a few logits more).  One warp: a bit per step, from the first in which the
// keys differ.  Where that is the lowest value of all, which the row is then full of (most logits masked with one value), the
// bound is the number above it: fewer may reach it than are wanted, and the rest are ties, the lowest indices of the row.
template <typename T>
__device__ __forceinline__ uint32_t cell_bound(const uint32_t* half, int want) {
  constexpr int kLastBit = Elem<T>::kZeroBits > 0 ? Elem<T>::kZeroBits : 16;
  constexpr int n = 2 * kLpThreads / 32;
  const int lane = threadIdx.x & 31;
  uint32_t k[n], hi = 0, lo = 0xFFFFFFFFu;
#pragma unroll
  for (int i = 0; i < n; ++i) {
    k[i] = half[i * 32 + lane];
    hi = max(hi, k[i]);
    lo = min(lo, k[i]);
  }
  hi = __reduce_max_sync(0xffffffffu, hi);
  lo = __reduce_min_sync(0xffffffffu, lo);
  const int first = 31 - __clz((int)(hi ^ lo));          // -1 when all keys are equal
  // (above -2^-149 that is 0, whose key is not the next one: the search below finds its bound)
  if (lo >= kKeyOfMinusInf && lo + 1 != kKeyOfMinusZero && __popc(__ballot_sync(0xffffffffu, k[0] == lo)) >= 8) {
    int above = 0;
#pragma unroll
    for (int i = 0; i < n; ++i) above += k[i] > lo;
    if ((int)__reduce_add_sync(0xffffffffu, above) < want) return lo + 1;
  }
  uint32_t prefix = first >= 31 ? 0u : hi & ~((2u << first) - 1u);
  if (first < 0) prefix = hi;
  for (int bit = first; bit >= kLastBit; --bit) {
    const uint32_t trial = prefix | (1u << bit);
    int count = 0;
#pragma unroll
    for (int i = 0; i < n; ++i) count += k[i] >= trial;
    if (__reduce_add_sync(0xffffffffu, count) >= want) prefix = trial;
  }
  // exact where it can be: a negative 16-bit value has ones below its bits, and -inf is alone in its range of keys
  if (Elem<T>::kZeroBits > 0) return prefix | ((prefix >> 31) != 0 ? 0u : (1u << kLastBit) - 1u);
  return prefix >= (kKeyOfMinusInf & ~0xFFFFu) && prefix < kKeyOfMinusInf ? kKeyOfMinusInf : prefix;
}

// The digit whose bin of sh.hist holds the rest-th element from the top, into sh.thr, and its rank inside the bin, into
// sh.rest.  One warp: eight bins a lane, the highest in lane 0.
__device__ __forceinline__ void digit_of_rank(LpShared& sh, int rest) {
  const int lane = threadIdx.x & 31, top = 255 - 8 * lane;
  int mine = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) mine += sh.hist[top - i];
  int upto = mine;                                       // elements in this lane's bins and all above
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, upto, off);
    if (lane >= off) upto += o;
  }
  const int owner = __ffs((int)__ballot_sync(0xffffffffu, upto >= rest)) - 1;
  if (lane == owner) {
    int left = rest - (upto - mine), d = top;
    while (d > top - 7 && (int)sh.hist[d] < left) { left -= sh.hist[d]; --d; }
    sh.thr = (uint32_t)d;
    sh.rest = left;
  }
}

// Many candidates (short rows of which a good part is wanted): only those from the want-th largest on stay, ties with it
// included, before the sort, whose work is quadratic.
constexpr int kSortable = 256;
__device__ __noinline__ int tighten_candidates(LpShared& sh, int n, int want) {
  const int tid = threadIdx.x;
  constexpr int kEach = (kMaxCand + kLpThreads - 1) / kLpThreads;
  unsigned long long mine[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) mine[j] = tid + j * kLpThreads < n ? sh.cand[tid + j * kLpThreads] : 0ull;   // no element has key 0
  uint32_t prefix = 0, mask = 0;
  int rest = want;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kLpThreads) sh.hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const uint32_t key = (uint32_t)(mine[j] >> 32);
      if (mine[j] != 0 && (key & mask) == prefix) atomicAdd(&sh.hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid < 32) digit_of_rank(sh, rest);
    __syncthreads();
    prefix |= sh.thr << shift;
    mask |= 255u << shift;
    rest = sh.rest;
    if (tid == 0) sh.n_cand = 0;
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < kEach; ++j)
    if ((uint32_t)(mine[j] >> 32) >= prefix) sh.cand[atomicAdd(&sh.n_cand, 1)] = mine[j];
  __syncthreads();
  return sh.n_cand;
}

// Rows built so that few cells hold everything large: the want-th largest key exactly, eight bits at a time, then the
// candidates above it and the ties with it.
template <typename T>
__device__ __noinline__ uint32_t exact_bound_and_candidates(LpShared& sh, const T* z, int e0, int e1, int want) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, mask = 0;
  int rest = want;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kLpThreads) sh.hist[i] = 0;
    __syncthreads();
    for (uint32_t i = e0 + tid; i < (uint32_t)e1; i += kLpThreads) {
      const uint32_t key = order_key(Elem<T>::load(z + i));
      if ((key & mask) == prefix) atomicAdd(&sh.hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid < 32) digit_of_rank(sh, rest);
    __syncthreads();
    prefix |= sh.thr << shift;
    mask |= 255u << shift;
    rest = sh.rest;
    __syncthreads();
  }
  const uint32_t thr = prefix;                         // an element's own key, and fewer than `want` lie above it
  if (tid == 0) { sh.n_cand = 0; sh.n_ties = 0; }
  __syncthreads();
  for (uint32_t i = e0 + tid; i < (uint32_t)e1; i += kLpThreads) {
    const float v = Elem<T>::load(z + i);
    const uint32_t key = order_key(v);
    if (key > thr) sh.cand[atomicAdd(&sh.n_cand, 1)] = rank_key(key, i);
    else if (key == thr) {
      const int at = atomicAdd(&sh.n_ties, 1);
      if (at < kMaxTies) sh.ties[at] = i;
    }
  }
  __syncthreads();
  return thr;
}

// What lies above the bound goes to the candidates, what equals it to the ties.
__device__ __forceinline__ void take_candidate(LpShared& sh, float v, int i, float bound, bool all) {
  if (v > bound || all) {
    const int at = atomicAdd(&sh.n_cand, 1);
    if (at < kMaxCand) sh.cand[at] = rank_key(order_key(v), i);
  } else if (v == bound) {
    const int at = atomicAdd(&sh.n_ties, 1);
    if (at < kMaxTies) sh.ties[at] = i;
  }
}

// Cells of a short row again, of one vector each: a single batch makes one cell a thread, and where nearly as many
// alternatives are wanted the bound would sink until most of the row lies above it (four rows of 29879 bf16, K = 128, eight
// blocks a row: 23.2 -> 16.1 us; half as many wanted, or two batches, and the second look at the row costs more than it gives:
// K = 64 7.8 -> 8.1, 7248 rows of 8250 fp16 with K = 128 129 -> 141).
constexpr int kFineWant = 96;
template <typename T>
__device__ __noinline__ void fine_cells(LpShared& sh, const uint4* zv, int nv) {
  const int tid = threadIdx.x;
  const uint4 pad = make_uint4(Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked());
  uint4 q[kLpBatch];
  uint32_t half_key[2] = {0u, 0u};
#pragma unroll
  for (int s = 0; s < kLpBatch; ++s) q[s] = s * kLpThreads + tid < nv ? __ldg(zv + s * kLpThreads + tid) : pad;
#pragma unroll
  for (int s = 0; s < kLpBatch; ++s) {
    const uint32_t w[4] = {q[s].x, q[s].y, q[s].z, q[s].w};
    const uint32_t key = s * kLpThreads + tid < nv ? order_key(Elem<T>::max_of(w)) : 0u;
    sh.cell[s * kLpThreads + tid] = key;                 // the cells above stay empty
    half_key[s & 1] = max(half_key[s & 1], key);
  }
  sh.half[tid] = half_key[0];
  sh.half[kLpThreads + tid] = half_key[1];
  __syncthreads();
}

// Leaves in sh.cand a set that holds the `want` largest rank keys of this CTA's elements; returns its size (at least
// `want`).  sh.cell and sh.half hold the maxima.
template <typename T>
__device__ __forceinline__ int select_candidates(LpShared& sh, const T* z, const RowSlice& rs, int want) {
  constexpr int kVec = Elem<T>::kVec;
  const int tid = threadIdx.x, lane = tid & 31;
  const int nv = rs.v1 - rs.v0;
  const uint4* zv = reinterpret_cast<const uint4*>(z + rs.head) + rs.v0;
  // cell (s, t) holds the vectors (s * per_cell + j) * 128 + t, j < per_cell
  int per_cell = kLpBatch * max(1, ((nv + kLpBatchVecs - 1) / kLpBatchVecs + kSegs - 1) / kSegs);
  if (nv <= kLpBatchVecs && want > kFineWant) {
    fine_cells<T>(sh, zv, nv);
    per_cell = 1;
  }
  if (tid < 32) {
    const uint32_t bound = cell_bound<T>(sh.half, want);
    if (lane == 0) { sh.n_hits = 0; sh.n_cand = 0; sh.n_ties = 0; sh.n_vecs = 0; sh.thr = bound; }
  }
  __syncthreads();
  uint32_t thr = sh.thr;
  const uint32_t best = max(sh.half[tid], sh.half[kLpThreads + tid]);
  if (best >= thr && best != 0) {
#pragma unroll
    for (int s = 0; s < kSegs; ++s) {
      const uint32_t key = sh.cell[s * kLpThreads + tid];
      if (key >= thr && key != 0) sh.hits[atomicAdd(&sh.n_hits, 1)] = (uint16_t)(s * kLpThreads + tid);
    }
  }
  __syncthreads();

  // a bound below every element's key (fewer nonempty cells than wanted): everything is above it, -inf too
  const bool all = thr < kKeyOfMinusInf;
  float bound = all ? -CUDART_INF_F : key_value(thr);
  const int n_work = sh.n_hits * per_cell;               // at most 1024 cells of nv / 1024 + 4 vectors each: below 2^29
  const float inv_per_cell = 1.f / (float)per_cell;
  const uint4 pad = make_uint4(Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked());
  // The few vectors that hold anything are gathered (where the cells and their maxima were, which have served) and their
  // elements dealt to all threads: taken in place, every warp would walk all elements of its vectors for a lane or two.
  uint4* vecs = reinterpret_cast<uint4*>(sh.cell);
  int* vec_at = reinterpret_cast<int*>(sh.half);
  constexpr int kAhead = 4;                              // second reads in flight per thread
  for (int w0 = tid; w0 < n_work; w0 += kLpThreads * kAhead) {
    uint4 q[kAhead];
    int at[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int w = w0 + u * kLpThreads;
      int h = (int)((float)w * inv_per_cell);            // w / per_cell, below 1024: off by at most one
      int j = w - h * per_cell;
      if (j < 0) { --h; j += per_cell; }
      if (j >= per_cell) { ++h; j -= per_cell; }
      at[u] = -1;
      q[u] = pad;
      if (w < n_work) {
        const int cell = sh.hits[h];
        const int i = ((cell / kLpThreads) * per_cell + j) * kLpThreads + cell % kLpThreads;
        if (i < nv) { at[u] = i; q[u] = __ldg(zv + i); }
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
      if (at[u] >= 0 && Elem<T>::max_of(w) >= bound) {
        const int slot = atomicAdd(&sh.n_vecs, 1);
        if (slot < kMaxVecs) {
          vecs[slot] = q[u];
          vec_at[slot] = at[u];
        } else {                                         // many vectors reach the bound: element by element, here
          uint4 v = q[u];
          const int first = rs.head + (rs.v0 + at[u]) * kVec;
#pragma unroll 1
          for (int e = 0; e < kVec; ++e) take_candidate(sh, Elem<T>::shift_out(v), first + e, bound, all);
        }
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < min(sh.n_vecs, kMaxVecs) * kVec; i += kLpThreads)
    take_candidate(sh, Elem<T>::to_float(reinterpret_cast<const T*>(vecs)[i]), rs.head + (rs.v0 + vec_at[i / kVec]) * kVec + i % kVec,
                   bound, all);
  if (tid < rs.own_head) take_candidate(sh, Elem<T>::load(z + tid), tid, bound, all);
  if (tid < rs.own_tail) take_candidate(sh, Elem<T>::load(z + rs.tail_start + tid), rs.tail_start + tid, bound, all);
  __syncthreads();
  int n_cand = sh.n_cand, n_ties = sh.n_ties;
  if (n_cand > kMaxCand) {
    thr = exact_bound_and_candidates<T>(sh, z, rs.e0, rs.e1, want);
    n_cand = sh.n_cand;
    n_ties = sh.n_ties;
  }
  if (n_cand < want) {
    if (n_ties <= kMaxTies) {
      for (int i = tid; i < n_ties; i += kLpThreads) sh.cand[n_cand + i] = rank_key(thr, sh.ties[i]);
      n_cand += n_ties;                                  // at most 127 + 256
    } else {
      append_ties_in_order(sh, z, rs.e0, rs.e1, thr, n_cand, want - n_cand);
      n_cand = want;
    }
    if (n_cand < want) {                                 // the bound was the number above the row's lowest
      append_ties_in_order(sh, z, rs.e0, rs.e1, thr - 1, n_cand, want - n_cand);
      n_cand = want;
    }
    __syncthreads();
  }
  if (n_cand > kSortable) n_cand = tighten_candidates(sh, n_cand, want);
  if ((n_cand & 1) != 0) {                               // the sort reads pairs
    if (tid == 0) sh.cand[n_cand] = 0ull;
    __syncthreads();
  }
  return n_cand;
}

// how many of the `n` candidates come before `key`
__device__ __forceinline__ int place_among(const LpShared& sh, unsigned long long key, int n) {
  const ulonglong2* pairs = reinterpret_cast<const ulonglong2*>(sh.cand);
  int before = 0;
#pragma unroll 4
  for (int j = 0; j < (n + 1) / 2; ++j) {
    const ulonglong2 o = pairs[j];
    before += (o.x > key) + (o.y > key);
  }
  return before;
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads, 7)
token_logprobs_kernel(const LogprobParams p, const int log2_cta) {
  pdl_launch_dependents();
  __shared__ LpShared sh;
  const int n_cta = 1 << log2_cta;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int cta = log2_cta > 0 ? (int)cluster_rank() : 0;
  const uint32_t n_rows_at_once = gridDim.x >> log2_cta;
  if (log2_cta > 0) cluster_barrier_arrive();          // waited for before the leader's shared memory is written
  pdl_wait();

  for (uint32_t row = blockIdx.x >> log2_cta; row < (uint32_t)p.T; row += n_rows_at_once) {   // unsigned: T may be 2^31 - 1
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.ld;
    const RowSlice rs = row_slice<T>(z, p.V, cta, log2_cta);
    float z_target = 0.f;
    int target = -1;
    if (cta == 0 && tid == 0 && p.targets != nullptr) {
      target = p.targets[row];
      if (target >= 0 && target < p.V) z_target = Elem<T>::load(z + target);
    }
    RunningStat run;
    run.start(p.ordinary != 0);
    const int nv = rs.v1 - rs.v0;
    const int n_batch = (nv + kLpBatchVecs - 1) / kLpBatchVecs;
    const int per_seg = max(1, (n_batch + kSegs - 1) / kSegs);
    const uint4* src = reinterpret_cast<const uint4*>(z + rs.head) + rs.v0 + tid;
    const uint4 pad = make_uint4(Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked());
    float seg_max = -CUDART_INF_F;
    uint32_t half_key[2] = {0u, 0u};
    int seg = 0, left = per_seg;
    auto load = [&](int b, uint4 (&q)[kLpBatch]) {
      const uint4* at = src + b * kLpBatchVecs;
      if ((b + 1) * kLpBatchVecs <= nv) {
#pragma unroll
        for (int u = 0; u < kLpBatch; ++u) q[u] = __ldg(at + u * kLpThreads);
      } else {
#pragma unroll
        for (int u = 0; u < kLpBatch; ++u)               // a padding vector (-inf) contributes nothing
          q[u] = b * kLpBatchVecs + u * kLpThreads + tid < nv ? __ldg(at + u * kLpThreads) : pad;
      }
    };
    auto process = [&](int b, const uint4 (&q)[kLpBatch]) {
      uint32_t w[4 * kLpBatch];
#pragma unroll
      for (int u = 0; u < kLpBatch; ++u) { w[4 * u] = q[u].x; w[4 * u + 1] = q[u].y; w[4 * u + 2] = q[u].z; w[4 * u + 3] = q[u].w; }
      const float batch_max = Elem<T>::max_of(w);
      run.template take_words<T, 4 * kLpBatch>(w, batch_max, p.c);
      seg_max = max_nan(seg_max, batch_max);
      if (p.top_k > 0) {
        if (--left == 0 || b == n_batch - 1) {
          const uint32_t key = seg * per_seg * kLpBatchVecs + tid < nv ? order_key(seg_max) : 0u;
          sh.cell[seg * kLpThreads + tid] = key;
          if ((seg & 1) == 0) half_key[0] = max(half_key[0], key); else half_key[1] = max(half_key[1], key);
          ++seg;
          seg_max = -CUDART_INF_F;
          left = per_seg;
        }
      }
    };
    for (int b = 0; b < n_batch; b += 2) {
      uint4 q[kLpBatch], r[kLpBatch];
      load(b, q);
      if (b + 1 < n_batch) load(b + 1, r);
      process(b, q);
      if (b + 1 < n_batch) process(b + 1, r);
    }
    if (p.top_k > 0) {
      for (; seg < kSegs; ++seg) sh.cell[seg * kLpThreads + tid] = 0u;
      sh.half[tid] = half_key[0];
      sh.half[kLpThreads + tid] = half_key[1];
    }
    // the warp's maximum first, one rescaling each, then plain sums; the same across the warps
    RowStat a = run.done_at_maximum(p.top_k > 0 ? key_value(max(half_key[0], half_key[1])) : seg_max, p.c);
    if (run.exact_needed) a = exact_stat<T>(reinterpret_cast<const uint4*>(z + rs.head) + rs.v0, tid, kLpThreads, nv, p.c);
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {                        // scalars before the first vector and after the last
      const int i = k == 0 ? tid : rs.tail_start + tid;
      if (tid < (k == 0 ? rs.own_head : rs.own_tail)) absorb_scalar(a, Elem<T>::load(z + i), p.c);
    }
    rescale(a, key_value(__reduce_max_sync(0xffffffffu, order_key(a.m))), p.c);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      a.S += __shfl_xor_sync(0xffffffffu, a.S, off);
      a.U += __shfl_xor_sync(0xffffffffu, a.U, off);
    }
    if (lane == 0) sh.part[wid] = a;
    __syncthreads();
    a = sh.part[lane & (kLpWarps - 1)];                  // every warp sums the parts, in the same order
    rescale(a, key_value(__reduce_max_sync(0xffffffffu, order_key(a.m))), p.c);
#pragma unroll
    for (int off = kLpWarps / 2; off > 0; off >>= 1) {
      a.S += __shfl_xor_sync(0xffffffffu, a.S, off);
      a.U += __shfl_xor_sync(0xffffffffu, a.U, off);
    }
    // A NaN cell maximum would order wrongly: a bad row (its maximum says so) lists nothing.  With several CTAs the others
    // may not know yet; what they list is not used then.
    const bool list = p.top_k > 0 && !(a.m != a.m);
    const int want = min(p.top_k, rs.e1 - rs.e0);
    const int n_cand = list ? select_candidates<T>(sh, z, rs, want) : 0;
    if (log2_cta > 0) {
      // this CTA's sorted list and triple go to the leader, which then finds everything in its own shared memory
      cluster_barrier_wait();
      float* stats = reinterpret_cast<float*>(lp_lists + p.top_k * n_cta);
      for (int i = tid; i < max(n_cand, p.top_k); i += kLpThreads) {
        const unsigned long long key = i < n_cand ? sh.cand[i] : 0ull;
        const int before = i < n_cand ? place_among(sh, key, n_cand) : i;
        if (before < want && i < n_cand) st_peer_u64(peer_shared(&lp_lists[cta * p.top_k + before], 0), key);
        if (i >= (list ? want : 0) && i < p.top_k) st_peer_u64(peer_shared(&lp_lists[cta * p.top_k + i], 0), 0ull);
      }
      if (tid < 3) st_peer_f32(peer_shared(&stats[cta * 4 + tid], 0), tid == 0 ? a.m : tid == 1 ? a.S : a.U);
      cluster_barrier();
      if (cta != 0) return;                              // a cluster has one row (the host launches as many as there are rows)
      const float* mine = stats + (lane & (n_cta - 1)) * 4;
      a = RowStat{mine[0], mine[1], mine[2]};
      rescale(a, key_value(__reduce_max_sync(0xffffffffu, order_key(a.m))), p.c);
      for (int off = n_cta / 2; off > 0; off >>= 1) {
        a.S += __shfl_xor_sync(0xffffffffu, a.S, off);
        a.U += __shfl_xor_sync(0xffffffffu, a.U, off);
      }
    }
    if (cta == 0) {
      const bool bad = bad_max(a.m);
      const float ln_s = logf(a.S);
      if (tid == 0) {
        const float nan = CUDART_NAN_F;
        if (p.lse != nullptr) p.lse[row] = bad ? nan : fmaf(a.m, p.inv_temp, ln_s);
        if (p.entropy != nullptr) p.entropy[row] = bad ? nan : fmaxf(ln_s - (a.U * kRowLn2) / a.S, 0.f);
        if (p.logprob != nullptr) {
          float v;
          if (target >= p.V) { v = nan; flag_status(p.status_word, CWL_ERR_INVALID_ARG); }
          else if (target < 0) v = 0.f;
          else v = bad ? nan : (z_target - a.m) * p.inv_temp - ln_s;
          p.logprob[row] = v;
        }
      }
      if (p.top_k > 0) {
        const int64_t out = (int64_t)row * p.top_k;
        if (bad) {
          for (int j = tid; j < p.top_k; j += kLpThreads) {
            p.top_ids[out + j] = -1;
            p.top_logprobs[out + j] = CUDART_NAN_F;
          }
        } else {
          int n = n_cand;
          if (log2_cta > 0) {
            // every list has at least q entries that reach the smallest of the lists' q-th ones: with q = top_k / n_cta
            // rounded up that is a bound of the row's top_k-th; what reaches it is sorted
            const int q = (p.top_k + n_cta - 1) >> log2_cta;
            unsigned long long bound = lp_lists[(lane & (n_cta - 1)) * p.top_k + q - 1];
            for (int off = n_cta / 2; off > 0; off >>= 1) bound = min(bound, __shfl_xor_sync(0xffffffffu, bound, off));
            if (tid == 0) sh.n_cand = 0;
            __syncthreads();
            for (int i = tid; i < p.top_k << log2_cta; i += kLpThreads) {
              const unsigned long long key = lp_lists[i];
              if (key >= bound && key != 0) sh.cand[atomicAdd(&sh.n_cand, 1)] = key;
            }
            __syncthreads();
            n = sh.n_cand;
            if (tid == 0) sh.cand[n] = 0ull;
            __syncthreads();
          }
          for (int i = tid; i < n; i += kLpThreads) {
            const unsigned long long key = sh.cand[i];
            const int place = place_among(sh, key, n);
            if (place < p.top_k) {
              p.top_ids[out + place] = (int32_t)(0xFFFFFFFFu - (uint32_t)key);
              p.top_logprobs[out + place] = (key_value((uint32_t)(key >> 32)) - a.m) * p.inv_temp - ln_s;
            }
          }
        }
      }
    }
    if (log2_cta > 0) return;
    __syncthreads();
  }
}

// CTAs that share a row (as a power of two).  One per row once the rows fill the GPU; with fewer rows the row is cut so
// that more SMs pull on it, down to slices of 2048 elements, while no more than 592 blocks come of it.  us with 1 : 2 : 4 : 8 blocks a
// row, 50000 fp32 without alternatives: 100 rows 16.0 : 11.4 : 9.2 : 8.0, 148 16.4 : 12.8 : 10.4 : 11.5, 296 20.2 : 15.0 : 17.3 : 17.9,
// 400 21.7 : 17.0 : 19.3 : 22.7, 500 21.8 : 19.4 : 24.8 : 27.4, 600 24.3 : 27.6 : 27.6 : 31.3, 777 27.8 : 30.6 : 34.9 : 39.4; 32000 bf16,
// K = 20: 100 rows 9.0 : 10.9 : 10.7 : 10.4, 296 16.7 : 14.6 : 18.3 : 25.8, 600 19.4 : 21.5 : 29.1 : 47.3; 131072 bf16, K = 20: 148 26.6 :
// 27.2 : 20.2 : 22.1, 296 43.9 : 30.7 : 30.2 : 34.7, 600 49.2 : 45.5 : 47.7 : 61.4.  One bound for all of them: between 297 and some 500
// rows two blocks a row would be 10 to 45 % faster than the one they get, at 222 rows four than two.
int logprob_cluster(int T, int V) {
  int l = 0;
  while ((1 << l) < kMaxLpCluster && ((int64_t)T << (l + 1)) <= 592 && (V >> (l + 1)) >= 2048) ++l;
  return l;
}

template <typename T>
cudaError_t launch_logprobs(const LogprobParams& p, cudaStream_t st) {
  const int l = logprob_cluster(p.T, p.V);
  const int rows = p.T < (1 << 20) ? p.T : (1 << 20);
  const bool chained = !stream_is_capturing(st);
  if (l == 0) return launch_chained(chained, token_logprobs_kernel<T>, dim3(rows), dim3(kLpThreads), 0, st, p, 0);
  return launch_clusters(chained, 1 << l, token_logprobs_kernel<T>, dim3(rows << l), dim3(kLpThreads), lp_lists_bytes(1 << l, p.top_k),
                         st, p, l);
}

}  // namespace
}  // namespace cwl

extern "C" cwl_status cwl_token_logprobs(const void* logits, cwl_dtype dtype, int64_t ld_logits, int32_t T, int32_t V,
                                         const int32_t* targets, float temperature, int32_t top_k,
                                         float* logprob, float* lse, float* entropy, int32_t* top_ids, float* top_logprobs,
                                         int32_t* status_word, void* stream) {
  if (T < 0 || V < 1 || top_k < 0 || !cwl::known_dtype(dtype)) return CWL_ERR_INVALID_ARG;
  if (!(temperature > 0.f) || !std::isfinite(temperature)) return CWL_ERR_INVALID_ARG;
  if (top_k > CWL_MAX_TOP_K) return CWL_ERR_UNSUPPORTED;
  if (top_k > V) return CWL_ERR_INVALID_ARG;
  if (T == 0) return CWL_OK;
  if (logits == nullptr || (top_k > 0 && (top_ids == nullptr || top_logprobs == nullptr))) return CWL_ERR_INVALID_ARG;
  if ((targets == nullptr) != (logprob == nullptr)) return CWL_ERR_INVALID_ARG;
  if (ld_logits < V) return CWL_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) % cwl::elem_size(dtype) != 0) return CWL_ERR_SHAPE;
  const float tau = cwl::usable_temperature(temperature);
  cwl::LogprobParams p{logits, ld_logits, T, V, targets, (float)(1.4426950408889634074 / (double)tau), (float)(1.0 / (double)tau),
                       cwl::ordinary_temperature(tau) ? 1 : 0, top_k, logprob, lse, entropy, top_ids, top_logprobs, status_word};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case CWL_F32: CWL_CUDA_TRY(cwl::launch_logprobs<float>(p, st)); break;
    case CWL_BF16: CWL_CUDA_TRY(cwl::launch_logprobs<__nv_bfloat16>(p, st)); break;
    default: CWL_CUDA_TRY(cwl::launch_logprobs<__half>(p, st)); break;
  }
  return CWL_OK;
}

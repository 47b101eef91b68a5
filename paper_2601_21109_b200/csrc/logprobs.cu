// cwl_token_logprobs: what a logit row says about given tokens -- their log-probability, the row's log-sum-exp and entropy,
// and the top alternatives.
//
//   m = max z,  S = sum e^((z-m)/tau):   lse = m/tau + ln S,   H = ln S - (1/S) sum (z-m)/tau e^((z-m)/tau),
//   logprob(y) = (z_y - m)/tau - ln S,   top K by (z descending, index ascending)
//
// The row is read once.  Every thread keeps the online triple of its own elements (its cell: every 256th 16-byte vector),
// and the maximum of the triple is at the same time the cell's maximum.  The K-th largest of the cell maxima is a lower
// bound of the row's K-th largest logit, and only cells whose maximum reaches it can hold one of the top K: about K of
// 256 cells are read a second time (from L2), and what reaches the bound is sorted in shared memory.
#include <cmath>

#include "logits_common.cuh"

namespace cwl {
namespace {

constexpr int kLpThreads = 256;       // also the number of cells a CTA's elements are dealt to
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpBatch = 4;           // 16-byte loads in flight per thread
constexpr int kMaxCand = 1152;        // logits above the bound kept for sorting; fewer than K nonempty cells hold at most
                                      // (CWL_MAX_TOP_K - 1) * 8 + 14 elements, which fit
constexpr int kMaxTies = 256;         // logits equal to the bound kept for sorting
constexpr int kMaxLpCluster = 8;

struct LogprobParams {
  const void* logits; int64_t ld; int T, V;
  const int32_t* targets;
  float c, inv_temp;          // log2(e) / temperature, 1 / temperature
  int top_k;
  float *logprob, *lse, *entropy;
  int32_t* top_ids; float* top_logprobs;
  int32_t* status_word;
};

// order-preserving map of a float (no NaN) to 32 bits; -0 and +0 are equal
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
// larger logit first, lower index first among equals: a larger 64-bit number comes first
__device__ __forceinline__ unsigned long long rank_key(uint32_t key, int idx) {
  return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)idx);
}

struct LpShared {
  unsigned long long cand[kMaxCand];           // candidates; then the lists of the whole cluster
  unsigned long long top[CWL_MAX_TOP_K];       // this CTA's sorted list; in the leader at the end the row's
  RowStat part[kLpWarps];
  RowStat stat;                                // this CTA's triple, read by the leader
  alignas(16) uint32_t cell[kLpThreads];       // order key of every cell's maximum, 0 for an empty cell
  uint32_t hist[256];
  int ties[kMaxTies];
  int warp_count[kLpWarps];
  uint16_t hits[kLpThreads];
  uint32_t thr;
  int n_hits, n_cand, n_ties, rest;
};
static_assert(kMaxLpCluster * CWL_MAX_TOP_K <= kMaxCand, "the cluster's lists are gathered in the candidate buffer");

// Appends the lowest-index elements whose key equals `key` to the candidates until `need` are found.
template <typename T>
__device__ void append_ties_in_order(LpShared& sh, const T* z, const RowSlice& rs, uint32_t key, int have, int need) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  int found = 0;
  for (int base = rs.e0; base < rs.e1 && found < need; base += kLpThreads) {
    const int i = base + tid;
    const bool is = i < rs.e1 && order_key(Elem<T>::load(z + i)) == key;
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

// The `k` largest rank keys of this CTA's elements, sorted, into sh.top (padded with 0).  sh.cell holds the cell maxima.
template <typename T>
__device__ void local_top(LpShared& sh, const T* z, const RowSlice& rs, int k) {
  constexpr int kVec = Elem<T>::kVec;
  const int tid = threadIdx.x;
  const int n = rs.e1 - rs.e0;
  const int want = min(k, n);
  if (tid == 0) { sh.n_hits = 0; sh.n_cand = 0; sh.n_ties = 0; sh.thr = 0; }
  if (tid < k) sh.top[tid] = 0ull;
  __syncthreads();
  // bound: the want-th largest of the cell maxima (0, below every element's key, when fewer cells hold anything)
  const uint32_t mine = sh.cell[tid];
  int above = 0;
  const uint4* cells = reinterpret_cast<const uint4*>(sh.cell);
#pragma unroll 8
  for (int j = 0; j < kLpThreads / 4; ++j) {
    const uint4 q = cells[j];
    above += (q.x > mine || (q.x == mine && 4 * j + 0 < tid)) + (q.y > mine || (q.y == mine && 4 * j + 1 < tid)) +
             (q.z > mine || (q.z == mine && 4 * j + 2 < tid)) + (q.w > mine || (q.w == mine && 4 * j + 3 < tid));
  }
  if (above == want - 1) sh.thr = mine;
  __syncthreads();
  uint32_t thr = sh.thr;
  if (mine >= thr && mine != 0) sh.hits[atomicAdd(&sh.n_hits, 1)] = (uint16_t)tid;
  __syncthreads();

  auto take = [&](float v, int i) {
    const uint32_t key = order_key(v);
    if (key > thr) {
      const int at = atomicAdd(&sh.n_cand, 1);
      if (at < kMaxCand) sh.cand[at] = rank_key(key, i);
    } else if (key == thr) {
      const int at = atomicAdd(&sh.n_ties, 1);
      if (at < kMaxTies) sh.ties[at] = i;
    }
  };
  const int per_cell = (rs.v1 - rs.v0 + kLpThreads - 1) / kLpThreads;
  const int n_hits = sh.n_hits;
  const uint4* zv = reinterpret_cast<const uint4*>(z + rs.head);
  for (int w = tid; w < n_hits * per_cell; w += kLpThreads) {
    const int h = w / per_cell, j = w - h * per_cell;
    const int i = rs.v0 + sh.hits[h] + j * kLpThreads;
    if (i < rs.v1) {
      float f[kVec];
      Elem<T>::unpack(__ldg(zv + i), f);
#pragma unroll
      for (int e = 0; e < kVec; ++e) take(f[e], rs.head + i * kVec + e);
    }
  }
  if (mine >= thr && mine != 0) {
    if (tid < rs.own_head) take(Elem<T>::load(z + tid), tid);
    if (tid < rs.own_tail) take(Elem<T>::load(z + rs.tail_start + tid), rs.tail_start + tid);
  }
  __syncthreads();
  int n_cand = sh.n_cand, n_ties = sh.n_ties;
  if (n_cand > kMaxCand) {
    // Rows built so that few cells hold everything large: the want-th largest key exactly, eight bits at a time.
    uint32_t prefix = 0, mask = 0;
    int rest = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
      sh.hist[tid] = 0;
      __syncthreads();
      for (int i = rs.e0 + tid; i < rs.e1; i += kLpThreads) {
        const uint32_t key = order_key(Elem<T>::load(z + i));
        if ((key & mask) == prefix) atomicAdd(&sh.hist[(key >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        int d = 255;
        while (d > 0 && (int)sh.hist[d] < rest) { rest -= sh.hist[d]; --d; }
        sh.thr = (uint32_t)d;
        sh.rest = rest;
      }
      __syncthreads();
      prefix |= sh.thr << shift;
      mask |= 255u << shift;
      rest = sh.rest;
      __syncthreads();
    }
    thr = prefix;
    if (tid == 0) { sh.n_cand = 0; sh.n_ties = 0; }
    __syncthreads();
    for (int i = rs.e0 + tid; i < rs.e1; i += kLpThreads) {
      const float v = Elem<T>::load(z + i);
      if (order_key(v) >= thr) take(v, i);
    }
    __syncthreads();
    n_cand = sh.n_cand;               // fewer than want
    n_ties = sh.n_ties;
  }
  if (n_cand < want) {
    const int need = want - n_cand;
    if (n_ties <= kMaxTies) {
      for (int i = tid; i < n_ties && n_cand + i < kMaxCand; i += kLpThreads) sh.cand[n_cand + i] = rank_key(thr, sh.ties[i]);
      n_cand = min(n_cand + n_ties, kMaxCand);
    } else {
      append_ties_in_order(sh, z, rs, thr, n_cand, need);
      n_cand = want;
    }
    __syncthreads();
  }
  for (int i = tid; i < n_cand; i += kLpThreads) {
    const unsigned long long key = sh.cand[i];
    int before = 0;
    for (int j = 0; j < n_cand; ++j) before += sh.cand[j] > key;
    if (before < k) sh.top[before] = key;
  }
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads)
token_logprobs_kernel(const LogprobParams p, const int n_cta) {
  constexpr int kVec = Elem<T>::kVec;
  pdl_launch_dependents();
  __shared__ LpShared sh;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int cta = n_cta > 1 ? (int)cluster_rank() : 0;
  const int n_rows_at_once = gridDim.x / n_cta;
  pdl_wait();

  for (int row = blockIdx.x / n_cta; row < p.T; row += n_rows_at_once) {
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.ld;
    const RowSlice rs = row_slice<T>(z, p.V, cta, n_cta);
    RowStat acc{-CUDART_INF_F, 0.f, 0.f};
    bool any = false;
    float z_target = 0.f;
    int target = -1;
    if (cta == 0 && tid == 0 && p.targets != nullptr) {
      target = p.targets[row];
      if (target >= 0 && target < p.V) z_target = Elem<T>::load(z + target);
    }
    auto take_scalar = [&](float v) {
      any = true;
      const float m_new = max_nan(acc.m, v);
      if (m_new == -CUDART_INF_F) return;
      if (m_new != acc.m) rebase(acc, m_new, p.c);
      absorb(acc, v, p.c);
    };
    if (tid < rs.own_head) take_scalar(Elem<T>::load(z + tid));
    if (tid < rs.own_tail) take_scalar(Elem<T>::load(z + rs.tail_start + tid));
    const uint4* zv = reinterpret_cast<const uint4*>(z + rs.head);
    const uint4 pad = make_uint4(Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked());
    if (rs.v0 + tid < rs.v1) any = true;
    for (int i = rs.v0 + tid; i < rs.v1; i += kLpThreads * kLpBatch) {
      uint4 q[kLpBatch];
#pragma unroll
      for (int u = 0; u < kLpBatch; ++u) {
        const int at = i + u * kLpThreads;
        q[u] = at < rs.v1 ? __ldg(zv + at) : pad;      // a padding vector (-inf) contributes nothing
      }
#pragma unroll
      for (int u = 0; u < kLpBatch; ++u) {
        float f[kVec];
        Elem<T>::unpack(q[u], f);
        float m_new = acc.m;
#pragma unroll
        for (int e = 0; e < kVec; ++e) m_new = max_nan(m_new, f[e]);
        if (m_new == -CUDART_INF_F) continue;
        if (m_new != acc.m) rebase(acc, m_new, p.c);
#pragma unroll
        for (int e = 0; e < kVec; ++e) absorb(acc, f[e], p.c);
      }
    }
    if (p.top_k > 0) sh.cell[tid] = any ? order_key(acc.m) : 0u;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      RowStat o;
      o.m = __shfl_xor_sync(0xffffffffu, acc.m, off);
      o.S = __shfl_xor_sync(0xffffffffu, acc.S, off);
      o.U = __shfl_xor_sync(0xffffffffu, acc.U, off);
      acc = merge(acc, o, p.c);
    }
    if (lane == 0) sh.part[wid] = acc;
    __syncthreads();
    RowStat a = sh.part[0];
    for (int w = 1; w < kLpWarps; ++w) a = merge(a, sh.part[w], p.c);
    // A NaN cell maximum would order wrongly: a bad row (its maximum says so) lists nothing.  With several CTAs the others
    // may not know yet; what they list is not used then.
    const bool list = p.top_k > 0 && !(a.m != a.m);
    if (list) local_top<T>(sh, z, rs, p.top_k);
    if (n_cta > 1) {
      if (tid == 0) sh.stat = a;
      __syncthreads();
      cluster_barrier();                          // every CTA's triple and list are in its shared memory
      if (cta == 0) {
        for (int r = 1; r < n_cta; ++r) {
          const uint32_t at = peer_shared(&sh.stat, r);
          RowStat o{ld_peer_f32(at), ld_peer_f32(at + 4), ld_peer_f32(at + 8)};
          a = merge(a, o, p.c);
        }
        if (p.top_k > 0) {
          const int all = n_cta * p.top_k;
          for (int i = tid; i < all; i += kLpThreads) {
            const int r = i / p.top_k;
            sh.cand[i] = ld_peer_u64(peer_shared(&sh.top[i - r * p.top_k], r));
          }
          __syncthreads();
          for (int i = tid; i < all; i += kLpThreads) {
            const unsigned long long key = sh.cand[i];
            const int r = i / p.top_k;
            int rank = i - r * p.top_k;           // keys before it in its own list, then in the others
            for (int o = 0; o < n_cta && rank < p.top_k; ++o) {
              if (o == r) continue;
              const unsigned long long* l = sh.cand + o * p.top_k;
              int lo = 0, hi = p.top_k;
              while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (l[mid] > key) lo = mid + 1; else hi = mid;
              }
              rank += lo;
            }
            if (rank < p.top_k) sh.top[rank] = key;
          }
        }
      }
    }
    __syncthreads();
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
      if (tid < p.top_k) {
        const unsigned long long key = sh.top[tid];
        const int64_t at = (int64_t)row * p.top_k + tid;
        const float v = key_value((uint32_t)(key >> 32));
        p.top_ids[at] = bad ? -1 : (int32_t)(0xFFFFFFFFu - (uint32_t)key);
        p.top_logprobs[at] = bad ? CUDART_NAN_F : (v - a.m) * p.inv_temp - ln_s;
      }
    }
    if (n_cta > 1) cluster_barrier();             // the leader has read the others' shared memory
    else __syncthreads();
  }
}

// CTAs that share a row.  One per row once the rows fill the GPU; with fewer rows the row is cut so that more SMs pull
// on it, down to slices of 2048 elements.
int logprob_cluster(int T, int V) {
  int c = 1;
  while (c < kMaxLpCluster && (int64_t)T * c * 2 <= 296 && V / (c * 2) >= 2048) c *= 2;
  return c;
}

template <typename T>
cudaError_t launch_logprobs(const LogprobParams& p, cudaStream_t st) {
  const int c = logprob_cluster(p.T, p.V);
  const int rows = p.T < (1 << 20) ? p.T : (1 << 20);
  return launch_clusters(!stream_is_capturing(st), c, token_logprobs_kernel<T>, dim3(rows * c), dim3(kLpThreads), 0, st, p, c);
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
  cwl::LogprobParams p{logits, ld_logits, T, V, targets, (float)(1.4426950408889634074 / (double)temperature),
                       (float)(1.0 / (double)temperature), top_k, logprob, lse, entropy, top_ids, top_logprobs, status_word};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case CWL_F32: CWL_CUDA_TRY(cwl::launch_logprobs<float>(p, st)); break;
    case CWL_BF16: CWL_CUDA_TRY(cwl::launch_logprobs<__nv_bfloat16>(p, st)); break;
    default: CWL_CUDA_TRY(cwl::launch_logprobs<__half>(p, st)); break;
  }
  return CWL_OK;
}

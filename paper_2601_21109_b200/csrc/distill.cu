// cwl_distill_topk: distillation from a teacher's top logits, loss and gradient in one pass over the student's logits.
//
//   q = softmax(z / tau),  loss = w tau^2 ( sum_j p_j ln(p_j / q_j) + p_rest ln(p_rest / q_rest) )
//   dz_v = dloss w tau ( q_v (sum p + p_rest) - p_v - [v outside the entries] p_rest q_v / q_rest )
//
// The statistics of a row must be known before its first gradient can be written, so the row stays in shared memory in
// between: one CTA holds it, or a cluster of up to eight CTAs holds a contiguous slice each and exchanges (m, S) through
// distributed shared memory.  Logits cross HBM once and the gradient once.  The entries' logits are lifted out of the
// row (their places become -inf) before the sums run: what is summed is then the mass outside the entries itself, not a
// difference of two nearly equal sums, and the elementwise gradient leaves those places 0 for the entries' own values.
#include <cmath>

#include "logits_common.cuh"

namespace cwl {
namespace {

constexpr int kDsThreads = 256;
constexpr int kDsWarps = kDsThreads / 32;
constexpr int kMaxDsCluster = 8;
constexpr int kDsSliceMax = 208 * 1024;      // bytes of a row one CTA can hold

struct DistillParams {
  const void* logits; int64_t ld; int T, V;
  const int32_t* ids; const float* values; int64_t ld_teacher; int K;
  int mode;
  float temperature, c, inv_temp;
  const float *weight, *dloss;
  float* loss;
  void* dlogits; int64_t ld_d;
  int32_t* status_word;
};

struct DsShared {
  float m_all[kMaxDsCluster], s_all[kMaxDsCluster], in_all[kMaxDsCluster];   // every CTA's max, outside sum, entries' sum
  int id[CWL_MAX_TOP_K];          // -1 for padding
  float p[CWL_MAX_TOP_K];         // teacher probability
  float z[CWL_MAX_TOP_K];         // student logits of the entries (in the leader: of all CTAs)
  float red[kDsWarps], red2[kDsWarps];
  double red_d[kDsWarps];
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() {
  asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}

// Writes one row slice of gradients: whole 16-byte vectors where the output row starts at the same offset from a 16-byte
// boundary as the input row, element by element otherwise.  value(i, f) fills f with the gradients of vector i.
template <typename T, typename F, typename G>
__device__ __forceinline__ void store_slice(T* d, bool same_phase, const RowSlice& rs, F vec_value, G scalar_value) {
  constexpr int kVec = Elem<T>::kVec;
  const int tid = threadIdx.x;
  for (int i = rs.v0 + tid; i < rs.v1; i += kDsThreads) {
    float f[kVec];
    vec_value(i, f);
    T* out = d + rs.head + (int64_t)i * kVec;
    if (same_phase) {
      *reinterpret_cast<uint4*>(out) = Elem<T>::pack(f);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) out[e] = Elem<T>::from_float(f[e]);
    }
  }
  if (tid < rs.own_head) d[tid] = Elem<T>::from_float(scalar_value(tid));
  if (tid < rs.own_tail) d[rs.tail_start + tid] = Elem<T>::from_float(scalar_value(rs.tail_start + tid));
}

template <typename T>
__global__ void __launch_bounds__(kDsThreads)
distill_kernel(const DistillParams p, const int log2_cta) {
  constexpr int kVec = Elem<T>::kVec;
  const int n_cta = 1 << log2_cta;
  pdl_launch_dependents();
  extern __shared__ __align__(16) uint8_t ds_raw[];
  __shared__ DsShared sh;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int cta = n_cta > 1 ? (int)cluster_rank() : 0;
  const int n_rows_at_once = gridDim.x >> log2_cta;
  if (n_cta > 1) cluster_barrier();                // the peers run before anything is written to their shared memory
  pdl_wait();

  for (int row = blockIdx.x >> log2_cta; row < p.T; row += n_rows_at_once) {
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.ld;
    T* d = p.dlogits != nullptr ? reinterpret_cast<T*>(p.dlogits) + (int64_t)row * p.ld_d : nullptr;
    const RowSlice rs = row_slice<T>(z, p.V, cta, log2_cta);
    const bool same_phase = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(d)) & 15u) == 0;
    const float w = p.weight != nullptr ? p.weight[row] : 1.f;
    if (w == 0.f) {                                // a row that is not trained on: not read (the whole cluster agrees)
      if (d != nullptr)
        store_slice<T>(d, same_phase, rs, [](int, float (&f)[kVec]) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) f[e] = 0.f;
        }, [](int) { return 0.f; });
      if (p.loss != nullptr && cta == 0 && tid == 0) p.loss[row] = 0.f;
      continue;
    }
    // shared-memory image of the slice: element i of the row at smem[i - e0 + lead], vectors on 16-byte boundaries
    const int lead = (kVec - rs.own_head % kVec) % kVec;
    T* sm = reinterpret_cast<T*>(ds_raw);
    const uint32_t sm_addr = (uint32_t)__cvta_generic_to_shared(sm);
    auto at = [&](int i) { return i - rs.e0 + lead; };
    const uint4* zv = reinterpret_cast<const uint4*>(z + rs.head);
    const uint32_t vec_base = sm_addr + (uint32_t)(rs.v1 > rs.v0 ? at(rs.head + rs.v0 * kVec) : 0) * (uint32_t)sizeof(T);
    for (int i = rs.v0 + tid; i < rs.v1; i += kDsThreads) cp_async16(vec_base + (uint32_t)(i - rs.v0) * 16u, zv + i);
    if (tid < rs.own_head) sm[at(tid)] = z[tid];
    if (tid < rs.own_tail) sm[at(rs.tail_start + tid)] = z[rs.tail_start + tid];

    // teacher entries, while the row is on its way (K <= 128: the first four warps, one entry a thread)
    const bool renorm = p.mode == CWL_TEACHER_LOGITS;
    int id = -1;
    float u = -CUDART_INF_F;       // the entry's value
    double lp;                     // ln p of the entry
    if (tid < p.K) {
      id = p.ids[(int64_t)row * p.ld_teacher + tid];
      if (id >= p.V) { flag_status(p.status_word, CWL_ERR_INVALID_ARG); id = -1; }
      if (id >= 0) u = p.values[(int64_t)row * p.ld_teacher + tid];
      sh.id[tid] = id;
    }
    float u_max = 0.f;
    if (renorm) {
      const float mx = warp_max_nan(u);
      if (lane == 0) sh.red[wid] = mx;
      __syncthreads();
      u_max = sh.red[0];
      for (int i = 1; i < kDsWarps; ++i) u_max = max_nan(u_max, sh.red[i]);
    }
    float pj = id >= 0 ? expf(renorm ? (u - u_max) * p.inv_temp : u) : 0.f;
    double p_sum = warp_sum((double)pj);
    if (lane == 0) sh.red_d[wid] = p_sum;
    __syncthreads();
    p_sum = 0.0;
    for (int i = 0; i < kDsWarps; ++i) p_sum += sh.red_d[i];
    float p_in = (float)p_sum, p_rest = 0.f;
    if (renorm) {
      lp = ((double)u - (double)u_max) / (double)p.temperature - log(p_sum);
      pj *= p_sum == 0.0 ? 0.f : (float)(1.0 / p_sum);           // no entries at all: nothing to learn from this row
      p_in = p_sum == 0.0 ? 0.f : p_sum == p_sum ? 1.f : CUDART_NAN_F;
    } else {
      lp = (double)u;
      p_rest = p_sum == p_sum ? (float)fmax(0.0, 1.0 - p_sum) : CUDART_NAN_F;
    }
    if (tid < p.K) sh.p[tid] = pj;
    cp_async_wait_all();
    __syncthreads();                               // slice and entries are in shared memory

    // lift the entries out of the slice
    float z_id = 0.f;
    float p_id = -1.f;             // probability of the entry's id: over all its occurrences, at the first of them; else -1
    bool mine = false;
    if (id >= 0) {
      mine = id >= rs.e0 && id < rs.e1;
      if (mine) z_id = Elem<T>::to_float(sm[at(id)]);
      p_id = 0.f;
      for (int j = 0; j < p.K; ++j) {
        if (sh.id[j] == id) {
          if (j < tid) { p_id = -1.f; break; }
          p_id += sh.p[j];
        }
      }
    }
    __syncthreads();
    if (mine) sm[at(id)] = Elem<T>::from_float(-CUDART_INF_F);
    __syncthreads();

    // maximum over the slice and its entries, then the sums relative to it
    float m = mine ? z_id : -CUDART_INF_F;
    const uint4* sv = reinterpret_cast<const uint4*>(ds_raw + (vec_base - sm_addr));
    const int n_vec = rs.v1 - rs.v0;
    for (int i = tid; i < n_vec; i += kDsThreads) {
      float f[kVec];
      Elem<T>::unpack(sv[i], f);
#pragma unroll
      for (int e = 0; e < kVec; ++e) m = max_nan(m, f[e]);
    }
    if (tid < rs.own_head) m = max_nan(m, Elem<T>::to_float(sm[at(tid)]));
    if (tid < rs.own_tail) m = max_nan(m, Elem<T>::to_float(sm[at(rs.tail_start + tid)]));
    m = warp_max_nan(m);
    if (lane == 0) sh.red[wid] = m;
    __syncthreads();
    m = sh.red[0];
    for (int i = 1; i < kDsWarps; ++i) m = max_nan(m, sh.red[i]);
    __syncthreads();
    const float m0 = bad_max(m) ? 0.f : m;         // a slice of -inf only sums to 0; NaN and +inf are told by m
    float s = 0.f;
    for (int i = tid; i < n_vec; i += kDsThreads) {
      float f[kVec];
      Elem<T>::unpack(sv[i], f);
#pragma unroll
      for (int e = 0; e < kVec; ++e) s += exp2_fast((f[e] - m0) * p.c);
    }
    if (tid < rs.own_head) s += exp2_fast((Elem<T>::to_float(sm[at(tid)]) - m0) * p.c);
    if (tid < rs.own_tail) s += exp2_fast((Elem<T>::to_float(sm[at(rs.tail_start + tid)]) - m0) * p.c);
    float s_in = mine && p_id >= 0.f ? exp2_fast((z_id - m0) * p.c) : 0.f;   // once per distinct id (p_id is -1 at repeats)
    s = warp_sum(s);
    s_in = warp_sum(s_in);
    if (lane == 0) { sh.red[wid] = s; sh.red2[wid] = s_in; }
    __syncthreads();
    s = 0.f; s_in = 0.f;
    for (int i = 0; i < kDsWarps; ++i) { s += sh.red[i]; s_in += sh.red2[i]; }
    if (n_cta > 1) {
      if (tid < n_cta) {
        st_peer_f32(peer_shared(&sh.m_all[cta], tid), m);
        st_peer_f32(peer_shared(&sh.s_all[cta], tid), s);
        st_peer_f32(peer_shared(&sh.in_all[cta], tid), s_in);
      }
      if (mine) st_peer_f32(peer_shared(&sh.z[tid], 0), z_id);
      cluster_barrier();
      float m_row = sh.m_all[0];
      for (int r = 1; r < n_cta; ++r) m_row = max_nan(m_row, sh.m_all[r]);
      s = 0.f; s_in = 0.f;
      for (int r = 0; r < n_cta; ++r) {
        const float mr = sh.m_all[r];
        if (mr == -CUDART_INF_F) continue;
        const float scale = exp2_fast((mr - m_row) * p.c);
        s += sh.s_all[r] * scale;
        s_in += sh.in_all[r] * scale;
      }
      m = m_row;
    } else if (mine) {
      sh.z[tid] = z_id;
    }
    if (bad_max(m)) { m = 0.f; s = CUDART_NAN_F; }
    const float s_row = s + s_in;

    if (p.loss != nullptr && cta == 0) {
      // the few terms of the loss in fp64: they nearly cancel where the student is close to the teacher
      const double ln_s = log((double)s_row);
      double term = 0.0;
      if (n_cta == 1) __syncthreads();
      if (id >= 0 && !(pj == 0.f)) term = (double)pj * (lp - (((double)sh.z[tid] - (double)m) / (double)p.temperature - ln_s));
      if (tid == 0 && !(p_rest == 0.f)) term += (double)p_rest * (log((double)p_rest) - (log((double)s) - ln_s));
      if (tid == 0 && !(s_row == s_row)) term = (double)CUDART_NAN_F;
      term = warp_sum(term);
      __syncthreads();
      if (lane == 0) sh.red_d[wid] = term;
      __syncthreads();
      if (tid == 0) {
        double kl = 0.0;
        for (int i = 0; i < kDsWarps; ++i) kl += sh.red_d[i];
        p.loss[row] = (float)((double)w * p.temperature * p.temperature * kl);
      }
    }
    if (d != nullptr) {
      const float up = w * p.temperature * (p.dloss != nullptr ? p.dloss[row] : 1.f);
      const float total = p_in + p_rest;
      const float inv_s = 1.f / s_row;
      // outside the entries: q_v (total - p_rest / q_rest); with no mass outside there is nothing to scale
      const float outside = s > 0.f ? total - p_rest * (s_row / s) : (s == s ? 0.f : s);
      const float k_out = outside * up * inv_s;
      store_slice<T>(d, same_phase, rs, [&](int i, float (&f)[kVec]) {
        Elem<T>::unpack(sv[i - rs.v0], f);
#pragma unroll
        for (int e = 0; e < kVec; ++e) f[e] = exp2_fast((f[e] - m) * p.c) * k_out;
      }, [&](int i) { return exp2_fast((Elem<T>::to_float(sm[at(i)]) - m) * p.c) * k_out; });
      __syncthreads();                             // the entries' places now hold 0: put their own values there
      if (mine && p_id >= 0.f) d[id] = Elem<T>::from_float((exp2_fast((z_id - m) * p.c) * inv_s * total - p_id) * up);
    }
    // the next row overwrites the shared arrays; the peers must have read this CTA's
    if (n_cta > 1) cluster_barrier(); else __syncthreads();
  }
}

// CTAs that share a row: as few as hold it in slices of kSliceWanted bytes (three CTAs fit an SM, so that one loads while
// another sums and a third writes), more while the rows do not fill the GPU.
constexpr int kSliceWanted = 66 * 1024;
int distill_cluster(int T, int64_t row_bytes) {
  int c = 1;
  while (c < kMaxDsCluster && row_bytes / c > kSliceWanted) c *= 2;
  while (c < kMaxDsCluster && (int64_t)T * c * 2 <= 296 && row_bytes / (c * 2) >= 8192) c *= 2;
  return c;
}

template <typename T>
cudaError_t launch_distill(const DistillParams& p, cudaStream_t st) {
  const int64_t row_bytes = (int64_t)p.V * sizeof(T);
  const int c = distill_cluster(p.T, row_bytes);
  int log2_cta = 0;
  while ((1 << log2_cta) < c) ++log2_cta;
  // one slice: its vectors, and head and tail scalars in a vector of their own each
  const size_t smem = (size_t)((row_bytes / 16 + c - 1) / c) * 16 + 32;
  if (smem > 40 * 1024) {                          // beyond what a kernel may use without asking
    const cudaError_t e = cudaFuncSetAttribute(distill_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDsSliceMax + 64);
    if (e != cudaSuccess) return e;
  }
  const int rows = p.T < (1 << 20) ? p.T : (1 << 20);
  return launch_clusters(!stream_is_capturing(st), c, distill_kernel<T>, dim3(rows * c), dim3(kDsThreads), smem, st, p, log2_cta);
}

}  // namespace
}  // namespace cwl

extern "C" cwl_status cwl_distill_topk(const void* logits, cwl_dtype dtype, int64_t ld_logits, int32_t T, int32_t V,
                                       const int32_t* teacher_ids, const float* teacher_values, int64_t ld_teacher, int32_t K,
                                       cwl_teacher_mode mode, float temperature, const float* weight, const float* dloss,
                                       float* loss, void* dlogits, int64_t ld_dlogits, int32_t* status_word, void* stream) {
  if (T < 0 || V < 1 || K < 1 || !cwl::known_dtype(dtype)) return CWL_ERR_INVALID_ARG;
  if (mode != CWL_TEACHER_LOGITS && mode != CWL_TEACHER_LOGPROBS) return CWL_ERR_INVALID_ARG;
  if (!(temperature > 0.f) || !std::isfinite(temperature)) return CWL_ERR_INVALID_ARG;
  if (K > CWL_MAX_TOP_K) return CWL_ERR_UNSUPPORTED;
  const size_t es = cwl::elem_size(dtype);
  if ((int64_t)V * (int64_t)es > CWL_MAX_DISTILL_ROW_BYTES) return CWL_ERR_UNSUPPORTED;
  if (T == 0) return CWL_OK;
  if (logits == nullptr || teacher_ids == nullptr || teacher_values == nullptr || (loss == nullptr && dlogits == nullptr))
    return CWL_ERR_INVALID_ARG;
  if (ld_logits < V || ld_teacher < K || (dlogits != nullptr && ld_dlogits < V)) return CWL_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) % es != 0 || reinterpret_cast<uintptr_t>(dlogits) % es != 0) return CWL_ERR_SHAPE;
  if (dlogits == logits && ld_dlogits != ld_logits) return CWL_ERR_SHAPE;
  cwl::DistillParams p{logits, ld_logits, T, V, teacher_ids, teacher_values, ld_teacher, K, (int)mode, temperature,
                       (float)(1.4426950408889634074 / (double)temperature), (float)(1.0 / (double)temperature), weight, dloss,
                       loss, dlogits, ld_dlogits, status_word};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case CWL_F32: CWL_CUDA_TRY(cwl::launch_distill<float>(p, st)); break;
    case CWL_BF16: CWL_CUDA_TRY(cwl::launch_distill<__nv_bfloat16>(p, st)); break;
    default: CWL_CUDA_TRY(cwl::launch_distill<__half>(p, st)); break;
  }
  return CWL_OK;
}

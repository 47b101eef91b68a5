// cwl_distill_topk: distillation from a teacher's top logits, loss and gradient in one pass over the student's logits.
//
//   q = softmax(z / tau),  loss = w tau^2 ( sum_j p_j ln(p_j / q_j) + p_rest ln(p_rest / q_rest) )
//   dz_v = dloss w tau ( q_v (sum p + p_rest) - p_v - [v outside the entries] p_rest q_v / q_rest )
//
// The statistics of a row must be known before its first gradient can be written, so the row stays in shared memory in
// between.  Logits cross HBM once and the gradient once.  The entries' logits are lifted out of the row (their places
// become -inf) before the sums run: what is summed is then the mass outside the entries itself, not a difference of two
// nearly equal sums, and the elementwise gradient leaves those places 0 for the entries' own values.
//
// Three kernels.  The loss alone of many rows: a stream over them.  Short rows: one block of 128 threads a row, many
// blocks to an SM, which overlap one another's phases.  Longer rows, and few rows: one persistent block an SM that
// pipelines rows through up to three buffers, alone or in a cluster of up to eight blocks that hold a contiguous slice of
// each row and exchange (m, S) through distributed shared memory.
//
// What bounds them: HBM, with the logits read once and the gradient written once.  16384 rows of 32000 fp32, gradient
// (clusters of two): 660 to 710 us, by GPU and how long it has been under load, 6.3 to 5.9 TB/s; 2048 rows of 32000 bf16, loss and
// gradient, a quarter of weight 0 (a block a row): 46.5 us, 4.9 TB/s -- ten rows a block, of which the first has no other to hide
// behind; 16384 short rows of 32 KB: fp32 164 us, 6.6 TB/s, bf16 209 us, 5.1 TB/s; the loss alone of 1000 rows of 131072 fp16: 52
// to 56 us, 5.0 to 4.7 TB/s -- one wave of blocks, all of which start and end together, on SMs of six or seven -- and of 16384 rows
// of 32000 fp32: 310 us, 6.8 TB/s.  Seven rows of 32003 fp32 (eight blocks a row): 7 us on the device.
#include <atomic>
#include <cmath>

#include "logits_common.cuh"
#include "tcgen05_common.cuh"

namespace cwl {
namespace {

constexpr int kDsThreads = 128;           // of the kernel for short rows; at least CWL_MAX_TOP_K
constexpr int kDsWarps = kDsThreads / 32;
constexpr int kMaxDsCluster = 8;
// Rows for one small block each: up to 16 KB always, up to 44 KB when there are four blocks an SM of them.  Small blocks against
// the pipelined kernel, us: 16384 rows of 32 KB 181 : 247, of 48 KB 279 : 286; at 300, 592, 900, 2000 rows of 17 KB 8.0 : 9.6, 8.9 :
// 15.3, 14.6 : 22.1, 19.6 : 40.9; of 32 KB (bf16) 14.1 : 13.0, 16.9 : 17.2, 20.0 : 24.3, 33.4 : 46.0; of 44 KB 13.1 : 13.0, 15.6 :
// 17.6, 20.5 : 24.3, 34.6 : 46.8.  (Rows of 17 and 22 KB would gain from 400 rows on.)
constexpr int kSmallRowBytes = 16 * 1024;
constexpr int kSmallManyRowBytes = 44 * 1024;
constexpr int kSmallManyRows = 592;

struct DistillParams {
  const void* logits; int64_t ld; int T, V;
  const int32_t* ids; const float* values; int64_t ld_teacher; int K;
  int mode;
  float temperature, c, inv_temp;
  double inv_temp_d;
  int ordinary;               // temperature within what the short form of the exponent takes
  const float *weight, *dloss;
  float* loss;
  void* dlogits; int64_t ld_d;
  int32_t* status_word;
  unsigned long long wait_limit_ns;
  int withhold;               // test build: the slice of row number 1 is never copied
};

struct DsShared {
  int id[CWL_MAX_TOP_K];          // -1 for padding
  float p[CWL_MAX_TOP_K];         // teacher probability
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

// Writes one row slice of gradients in 16-byte vectors.  Where the output row starts at the same offset from a 16-byte
// boundary as the input row, the vectors are those of the input: vec_value(i, f) fills f with the gradients of vector i.
// Otherwise they lie across the input's, and are put together element by element (scalar_value); the elements before the
// first and after the last whole vector go out one by one.
template <typename T, int kThreads, typename F, typename G>
__device__ __forceinline__ void store_slice(int tid, T* d, bool same_phase, const RowSlice& rs, F vec_value, G scalar_value) {
  constexpr int kVec = Elem<T>::kVec;
  if (same_phase) {
    for (int i = rs.v0 + tid; i < rs.v1; i += kThreads) {
      float f[kVec];
      vec_value(i, f);
      *reinterpret_cast<uint4*>(d + rs.head + (int64_t)i * kVec) = Elem<T>::pack(f);
    }
    if (tid < rs.own_head) d[tid] = Elem<T>::from_float(scalar_value(tid));
    if (tid < rs.own_tail) d[rs.tail_start + tid] = Elem<T>::from_float(scalar_value(rs.tail_start + tid));
  } else {
    const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(d + rs.e0) & 15u);
    const int first = min(rs.e0 + (int)(((16u - off) & 15u) / sizeof(T)), rs.e1);
    const int n = (rs.e1 - first) / kVec, last = first + n * kVec;
    for (int i = tid; i < n; i += kThreads) {
      float f[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) f[e] = scalar_value(first + i * kVec + e);
      *reinterpret_cast<uint4*>(d + first + (int64_t)i * kVec) = Elem<T>::pack(f);
    }
    if (tid < first - rs.e0) d[rs.e0 + tid] = Elem<T>::from_float(scalar_value(rs.e0 + tid));
    if (tid < rs.e1 - last) d[last + tid] = Elem<T>::from_float(scalar_value(last + tid));
  }
}
template <typename T, int kThreads>
__device__ __forceinline__ void zero_slice(int tid, T* d, bool same_phase, const RowSlice& rs) {
  store_slice<T, kThreads>(tid, d, same_phase, rs, [](int, float (&f)[Elem<T>::kVec]) {
#pragma unroll
    for (int e = 0; e < Elem<T>::kVec; ++e) f[e] = 0.f;
  }, [](int) { return 0.f; });
}

// One entry of the teacher, and what all entries of its row share.
struct Entry {
  int id;               // -1: padding
  float value;
  float p;              // probability
  double lp;            // its logarithm
  float p_id;           // probability of the id over all its occurrences, at the first of them; -1 elsewhere
  float z;              // the student's logit
  float p_in, p_rest;   // sum of the entries' probabilities; what is left to the rest
};
struct EntryRest { double lp; int id; float p, p_id, z; };   // what the loss and the entry's own gradient take of it
__device__ __forceinline__ void load_entry(const DistillParams& p, int row, int j, Entry& en) {
  en.id = -1; en.value = 0.f; en.p = 0.f; en.lp = 0.0; en.p_id = -1.f; en.z = 0.f; en.p_in = 0.f; en.p_rest = 0.f;
  if (j < p.K) {
    en.id = __ldg(p.ids + (int64_t)row * p.ld_teacher + j);
    en.value = __ldg(p.values + (int64_t)row * p.ld_teacher + j);
  }
}
// apart from the loads, so that they can be under way while another row is worked on
__device__ __forceinline__ void check_entry(const DistillParams& p, Entry& en) {
  if (en.id >= p.V) { flag_status(p.status_word, CWL_ERR_INVALID_ARG); en.id = -1; }
  if (en.id < 0) { en.id = -1; en.value = 0.f; }
}
// the entry's weight before normalisation (also left in en.p); v_max: the largest value of the row, for CWL_TEACHER_LOGITS
__device__ __forceinline__ double entry_weight(const DistillParams& p, float v_max, Entry& en) {
  if (en.id >= 0) en.p = expf(p.mode == CWL_TEACHER_LOGITS ? (en.value - v_max) * p.inv_temp : en.value);
  return (double)en.p;
}
__device__ __forceinline__ void finish_entry(const DistillParams& p, float v_max, double p_sum, Entry& en) {
  if (p.mode == CWL_TEACHER_LOGITS) {
    // no entries at all: nothing to learn from this row
    en.lp = ((double)en.value - (double)v_max) * p.inv_temp_d - log(p_sum);
    en.p *= p_sum == 0.0 ? 0.f : (float)(1.0 / p_sum);
    en.p_in = p_sum == 0.0 ? 0.f : p_sum == p_sum ? 1.f : CUDART_NAN_F;
    en.p_rest = 0.f;
  } else {
    en.lp = (double)en.value;
    en.p_in = (float)p_sum;
    en.p_rest = p_sum == p_sum ? (float)fmax(0.0, 1.0 - p_sum) : CUDART_NAN_F;
  }
}
__device__ __forceinline__ float merged_probability(const int* ids, const float* probs, int K, int j) {
  const int id = ids[j];
  float sum = 0.f;
  bool seen = false;
  for (int k = 0; k < K; ++k) {
    if (ids[k] == id) {
      seen = seen || k < j;
      sum += probs[k];
    }
  }
  return seen ? -1.f : sum;
}
// 1 / x within 2^-23, of sums between 1 and 2^30
__device__ __forceinline__ float inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// What a row's logits come to: its maximum m and S = sum 2^((z - m) c) over all of it, and the same of what lies outside the
// entries, relative to an m_out.  That is m itself where the mass outside shows beside it; where it does not (kNear) it is the
// largest logit outside: however far that lies below the row's maximum, the mass outside then has its logarithm and its elements
// their shares of it.
struct RowMass {
  float m, s_row;
  float m_out, s_out;     // m and 0 where nothing lies outside
  float scale;            // 2^((m_out - m) c)
};
constexpr float kNear = 0x1p-40f;      // 2^-126, below which an exponential is 0, is nothing beside it
__device__ __forceinline__ RowMass bad_mass() { return RowMass{0.f, CUDART_NAN_F, 0.f, CUDART_NAN_F, 1.f}; }
__device__ __forceinline__ RowMass near_mass(float m, float s_out, float s_in) { return RowMass{m, s_out + s_in, m, s_out, 1.f}; }
// An outside that lies below the maximum by more than kMaskedExponent is masked (with fp32's or bf16's lowest value), like -inf.
__device__ __forceinline__ RowMass far_mass(float m, float s_in, float m_out, float s_out, float c) {
  const float below = (m_out - m) * c;
  const bool none = !(below > kMaskedExponent);
  RowMass r{m, 0.f, none ? m : m_out, none ? 0.f : s_out, none ? 0.f : exp2_fast(below)};
  r.s_row = s_in + r.s_out * r.scale;
  return r;
}
// a part's sum relative to m
__device__ __forceinline__ float part_sum(float2 part, float m, float c) {
  return part.x == -CUDART_INF_F ? 0.f : part.y * exp2_fast((part.x - m) * c);
}
// What the teacher leaves to the rest.  1 - sum p of a record that holds everything is not 0 but its rounding: an fp32 log-
// probability u of a few operations is off by a few 2^-24 (1 + |u|), and sum p (1 + |u|) is at most 1 + ln 128 < 6.  A remainder
// that small is taken for none where the student has no more than that outside the entries either; its logarithm there may be
// -inf or that of a mask, and would make an infinite loss, or any, of the rounding.
constexpr float kRecordRounding = 1.f / (1 << 20);
__device__ __forceinline__ float rest_of(float p_rest, const RowMass& r) {
  return p_rest <= kRecordRounding && r.s_out * r.scale <= kRecordRounding * r.s_row ? 0.f : p_rest;
}
// No entries, and no rest: the row's loss and gradient are 0 whatever its logits are.
__device__ __forceinline__ bool nothing_taught(float p_in, float p_rest) { return p_in + p_rest == 0.f; }
// This entry's share of the loss (thread 0 adds the rest's), in fp64: the terms nearly cancel where the student is close
// to the teacher.
__device__ __forceinline__ double loss_term(const DistillParams& p, int id, float prob, double lp, float z, float p_in, float p_rest,
                                            const RowMass& r, int tid) {
  double term = 0.0;
  const double ln_s = log((double)r.s_row);
  if (id >= 0 && !(prob == 0.f)) term = (double)prob * (lp - (((double)z - (double)r.m) * p.inv_temp_d - ln_s));
  if (tid == 0 && !(p_rest == 0.f)) {
    const double ln_out = log((double)r.s_out) + ((double)r.m_out - (double)r.m) * p.inv_temp_d;
    term += (double)p_rest * (log((double)p_rest) - (ln_out - ln_s));
  }
  if (tid == 0 && !(r.s_row == r.s_row) && !nothing_taught(p_in, p_rest)) term = (double)CUDART_NAN_F;
  return term;
}
// outside the entries the gradient is 2^((z - m_out) c) times this: total q_v - p_rest q_v / q_rest; with no mass outside
// there is nothing to scale
__device__ __forceinline__ float outside_factor(float total, float p_rest, const RowMass& r) {
  const float k = total * r.scale * inverse(r.s_row) - p_rest * inverse(r.s_out);
  return r.s_out == 0.f ? 0.f : k;
}
__device__ __forceinline__ float entry_gradient(const DistillParams& p, float z, float p_id, float total, float m, float s_row) {
  return exp2_fast((z - m) * p.c) * inverse(s_row) * total - p_id;
}

template <typename T>
__global__ void __launch_bounds__(kDsThreads)
distill_small_kernel(const DistillParams p) {
  constexpr int kVec = Elem<T>::kVec;
  pdl_launch_dependents();
  extern __shared__ __align__(128) uint8_t ds_raw[];
  __shared__ DsShared sh;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  pdl_wait();

  for (uint32_t row = blockIdx.x; row < (uint32_t)p.T; row += gridDim.x) {     // unsigned: T may be 2^31 - 1
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.ld;
    T* d = p.dlogits != nullptr ? reinterpret_cast<T*>(p.dlogits) + (int64_t)row * p.ld_d : nullptr;
    const RowSlice rs = row_slice<T>(z, p.V, 0, 0);
    const bool same_phase = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(d)) & 15u) == 0;
    const float w = p.weight != nullptr ? p.weight[row] : 1.f;
    if (w == 0.f) {                                // a row that is not trained on: not read
      if (d != nullptr) zero_slice<T, kDsThreads>(tid, d, same_phase, rs);
      if (p.loss != nullptr && tid == 0) p.loss[row] = 0.f;
      continue;
    }
    // shared-memory image of the row: element i at sm[i + lead], vectors on 16-byte boundaries
    const int lead = (kVec - rs.head % kVec) % kVec;
    T* sm = reinterpret_cast<T*>(ds_raw);
    const uint4* zv = reinterpret_cast<const uint4*>(z + rs.head);
    const uint32_t vec_base = (uint32_t)__cvta_generic_to_shared(sm + rs.head + lead);
    for (int i = tid; i < rs.v1; i += kDsThreads) cp_async16(vec_base + (uint32_t)i * 16u, zv + i);
    if (tid < rs.own_head) sm[lead + tid] = z[tid];
    if (tid < rs.own_tail) sm[lead + rs.tail_start + tid] = z[rs.tail_start + tid];

    // teacher entries, one a thread, while the row is on its way
    Entry en;
    load_entry(p, row, tid, en);
    check_entry(p, en);
    if (tid < p.K) sh.id[tid] = en.id;
    float v_max = 0.f;
    if (p.mode == CWL_TEACHER_LOGITS) {
      const float mx = warp_max_nan(en.id >= 0 ? en.value : -CUDART_INF_F);
      if (lane == 0) sh.red[wid] = mx;
      __syncthreads();
      v_max = sh.red[0];
      for (int i = 1; i < kDsWarps; ++i) v_max = max_nan(v_max, sh.red[i]);
    }
    double p_sum = warp_sum(entry_weight(p, v_max, en));
    if (lane == 0) sh.red_d[wid] = p_sum;
    __syncthreads();
    p_sum = 0.0;
    for (int i = 0; i < kDsWarps; ++i) p_sum += sh.red_d[i];
    finish_entry(p, v_max, p_sum, en);
    if (tid < p.K) sh.p[tid] = en.p;
    cp_async_wait_all();
    __syncthreads();                               // row and entries are in shared memory
    // lift the entries out of the row
    if (en.id >= 0) {
      en.z = Elem<T>::to_float(sm[lead + en.id]);
      en.p_id = merged_probability(sh.id, sh.p, p.K, tid);
    }
    __syncthreads();
    if (en.id >= 0) sm[lead + en.id] = Elem<T>::from_float(-CUDART_INF_F);
    __syncthreads();

    // maximum over the row and its entries, then the sums relative to it
    const uint4* sv = reinterpret_cast<const uint4*>(sm + rs.head + lead);
    auto row_max = [&](float m) {
      for (int i = tid; i < rs.v1; i += kDsThreads) {
        const uint4 q = sv[i];
        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
        m = max_nan(m, Elem<T>::max_of(words));
      }
      if (tid < rs.own_head) m = max_nan(m, Elem<T>::to_float(sm[lead + tid]));
      if (tid < rs.own_tail) m = max_nan(m, Elem<T>::to_float(sm[lead + rs.tail_start + tid]));
      m = key_value(__reduce_max_sync(0xffffffffu, order_key(m)));
      if (lane == 0) sh.red[wid] = m;
      __syncthreads();
      m = sh.red[0];
      for (int i = 1; i < kDsWarps; ++i) m = max_nan(m, sh.red[i]);
      __syncthreads();
      return m;
    };
    auto sum_outside = [&](float m) {              // this warp's
      float s = 0.f;
      for (int i = tid; i < rs.v1; i += kDsThreads) {
        float f[kVec];
        Elem<T>::unpack(sv[i], f);
#pragma unroll
        for (int e = 0; e < kVec; ++e) s += exp2_fast((f[e] - m) * p.c);
      }
      if (tid < rs.own_head) s += exp2_fast((Elem<T>::to_float(sm[lead + tid]) - m) * p.c);
      if (tid < rs.own_tail) s += exp2_fast((Elem<T>::to_float(sm[lead + rs.tail_start + tid]) - m) * p.c);
      return warp_sum(s);
    };
    float m = row_max(en.id >= 0 ? en.z : -CUDART_INF_F);
    const bool bad = bad_max(m);
    if (bad) m = 0.f;
    const float s_warp = sum_outside(m);
    const float s_in_warp = warp_sum(en.p_id >= 0.f ? exp2_fast((en.z - m) * p.c) : 0.f);   // once per distinct id
    if (lane == 0) { sh.red[wid] = s_warp; sh.red2[wid] = s_in_warp; }
    __syncthreads();
    float s_out = 0.f, s_in = 0.f;
    for (int i = 0; i < kDsWarps; ++i) { s_out += sh.red[i]; s_in += sh.red2[i]; }
    RowMass r = bad ? bad_mass() : near_mass(m, s_out, s_in);
    if (!bad && s_out < kNear) {
      __syncthreads();                             // sh.red was read
      const float m_out = row_max(-CUDART_INF_F);
      const float s_far = sum_outside(m_out == -CUDART_INF_F ? 0.f : m_out);
      if (lane == 0) sh.red[wid] = s_far;
      __syncthreads();
      s_out = 0.f;
      for (int i = 0; i < kDsWarps; ++i) s_out += sh.red[i];
      r = far_mass(m, s_in, m_out, s_out, p.c);
    }
    const float rest = rest_of(en.p_rest, r);
    const float k = outside_factor(en.p_in + rest, rest, r);

    if (p.loss != nullptr) {
      const double term = warp_sum(loss_term(p, en.id, en.p, en.lp, en.z, en.p_in, rest, r, tid));
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
      const float k_out = k * up;
      if (nothing_taught(en.p_in, rest)) {
        zero_slice<T, kDsThreads>(tid, d, same_phase, rs);
      } else {
        store_slice<T, kDsThreads>(tid, d, same_phase, rs, [&](int i, float (&f)[kVec]) {
          Elem<T>::unpack(sv[i], f);
#pragma unroll
          for (int e = 0; e < kVec; ++e) f[e] = exp2_fast((f[e] - r.m_out) * p.c) * k_out;
        }, [&](int i) { return exp2_fast((Elem<T>::to_float(sm[lead + i]) - r.m_out) * p.c) * k_out; });
      }
      __syncthreads();                             // the entries' places now hold 0: put their own values there
      if (en.p_id >= 0.f) d[en.id] = Elem<T>::from_float(entry_gradient(p, en.z, en.p_id, en.p_in + rest, r.m, r.s_row) * up);
    }
    __syncthreads();                               // the next row overwrites the shared arrays
  }
}

// --------------------------------------------------------------------------------------------- the loss alone, many rows
// Nothing has to stay for a gradient: rows stream through registers as in logprobs.cu, one block of 128 threads a row,
// seven or eight blocks an SM.  A bit per element in shared memory marks the entries; a vector that holds one (64 of 4000, say) has
// it replaced by -inf before it is summed, so that the mass outside the entries is again a sum of its own.
// Eight blocks against seven: 16384 rows of 32000 fp16 213 -> 200 us, 4000 rows 61 -> 59; but rows that seven an SM hold at
// once are spread more evenly that way: 1000 rows of 131072 fp16, back to back, 55 us (52 to 56 by GPU), with eight 58.
constexpr int kLossThreads = 128;
constexpr int kLossWarps = kLossThreads / 32;
constexpr int kLossBatch = 4;
// From five blocks an SM on; with fewer rows the pipelined kernel, which cuts rows up.  Stream against pipeline, us, at 200, 400,
// 600, 740, 1200 rows: 32 KB (fp32) 7.4 : 7.9, 9.2 : 11.7, 11.2 : 15.4, 11.8 : 16.8, 16.7 : 24.1; 64 KB (bf16) 11.7 : 9.2, 16.3 : 13.3,
// 17.4 : 17.1, 17.7 : 18.5, 24.3 : 26.9; 256 KB (fp16) 34.9 : 21.6, 45.3 : 35.7, 48.0 : 49.5, 48.6 : 58.1, 67.7 : 89.3; 512 KB (fp32)
// 42.0 : 35.9, 52.4 : 62.4, 61.2 : 90.9, 65.5 : 111.5, 119.7 : 175.0.  One bound for all sizes and types: fp32 rows, whose sums cost
// half as much a byte, would gain from the stream from 300 rows on.
constexpr int kLossMinRows = 740;

struct LossShared {
  double red_d[kLossWarps];
  float red[kLossWarps];
  float2 part[kLossWarps];                     // (m, S) of every warp's elements outside the entries
  float m_in[kLossWarps], s_in[kLossWarps];    // and of its entries
  int id[CWL_MAX_TOP_K];
  int repeated;                                // some id occurs twice
};

template <typename T>
__device__ __noinline__ RowStat exact_masked_stat(const uint4* v, const uint32_t* marks, int first, int stride, int n, float c) {
  constexpr int kVec = Elem<T>::kVec;
  RowStat a{-CUDART_INF_F, 0.f, 0.f};
  for (int i = first; i < n; i += stride) {
    uint4 q = v[i];
    const int pos = (i + 1) * kVec;
    Elem<T>::mask_out(q, (marks[pos >> 5] >> (pos & 31)) & ((1u << kVec) - 1u));
    float f[kVec];
    Elem<T>::unpack(q, f);
#pragma unroll
    for (int e = 0; e < kVec; ++e) absorb_scalar(a, f[e], c);
  }
  return a;
}

template <typename T, int kBlocks>
__global__ void __launch_bounds__(kLossThreads, kBlocks)
distill_loss_kernel(const DistillParams p, const int mark_words) {
  constexpr int kVec = Elem<T>::kVec;
  pdl_launch_dependents();
  extern __shared__ __align__(128) uint8_t ds_raw[];
  LossShared& sh = *reinterpret_cast<LossShared*>(ds_raw);
  uint32_t* marks = reinterpret_cast<uint32_t*>(ds_raw + sizeof(LossShared));   // element i of a row: bit i - head + kVec
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  for (int i = tid; i < mark_words; i += kLossThreads) marks[i] = 0;
  if (tid == 0) sh.repeated = 0;
  pdl_wait();
  __syncthreads();

  for (int row = blockIdx.x; row < p.T; row += gridDim.x) {
    const float w = p.weight != nullptr ? __ldg(p.weight + row) : 1.f;
    if (w == 0.f) {
      if (tid == 0) p.loss[row] = 0.f;
      continue;
    }
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.ld;
    const RowSlice rs = row_slice<T>(z, p.V, 0, 0);
    Entry en;
    load_entry(p, row, tid, en);
    check_entry(p, en);
    bool counts = false;                       // the first entry of its id
    const int pos = en.id - rs.head + kVec;
    if (tid < p.K) sh.id[tid] = en.id;
    if (en.id >= 0) {
      en.z = Elem<T>::load(z + en.id);
      const uint32_t bit = 1u << (pos & 31);
      counts = (atomicOr(marks + (pos >> 5), bit) & bit) == 0;
      if (!counts) sh.repeated = 1;
    }
    __syncthreads();                           // all marks are set
    if (sh.repeated != 0) {                    // which of two marked it depends on timing, and so would the order of the sums
      counts = en.id >= 0;
      for (int k = 0; k < tid && counts; ++k) counts = sh.id[k] != en.id;
    }

    RunningSum run;
    run.start(p.ordinary != 0);
    const int nv = rs.v1;
    const uint4* src = reinterpret_cast<const uint4*>(z + rs.head) + tid;
    const uint4 pad = make_uint4(Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked(), Elem<T>::masked());
    auto load = [&](int first, uint4 (&q)[kLossBatch]) {
#pragma unroll
      for (int u = 0; u < kLossBatch; ++u) q[u] = first + u * kLossThreads < nv ? __ldg(src + (first - tid) + u * kLossThreads) : pad;
    };
    auto process = [&](int first, uint4 (&q)[kLossBatch]) {
      uint32_t words[4 * kLossBatch];
#pragma unroll
      for (int u = 0; u < kLossBatch; ++u) {
        const int v = min(first + u * kLossThreads, nv - 1);
        const int at = (v + 1) * kVec;
        const uint32_t bits = (marks[at >> 5] >> (at & 31)) & ((1u << kVec) - 1u);
        if (bits != 0) Elem<T>::mask_out(q[u], bits);
        words[4 * u] = q[u].x; words[4 * u + 1] = q[u].y; words[4 * u + 2] = q[u].z; words[4 * u + 3] = q[u].w;
      }
      run.template take_words<T, 4 * kLossBatch>(words, Elem<T>::max_of(words), p.c);
    };
    constexpr int kStep = kLossBatch * kLossThreads;
    for (int i = tid; i - tid < nv; i += 2 * kStep) {
      uint4 q[kLossBatch], r[kLossBatch];
      load(i, q);
      const bool two = i - tid + kStep < nv;
      if (two) load(i + kStep, r);
      process(i, q);
      if (two) process(i + kStep, r);
    }
    RowStat a = run.done(p.c);
    if (run.exact_needed) a = exact_masked_stat<T>(src - tid, marks, tid, kLossThreads, nv, p.c);
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {              // scalars before the first vector and after the last
      const int i = k == 0 ? tid : rs.tail_start + tid;
      if (tid < (k == 0 ? rs.own_head : rs.own_tail)) {
        const int at = i - rs.head + kVec;
        if (((marks[at >> 5] >> (at & 31)) & 1u) == 0) absorb_scalar(a, Elem<T>::load(z + i), p.c);
      }
    }
    rescale(a, key_value(__reduce_max_sync(0xffffffffu, order_key(a.m))), p.c);
    a.S = warp_sum(a.S);
    if (lane == 0) sh.part[wid] = make_float2(a.m, a.S);

    // the teacher's side
    float v_max = 0.f;
    if (p.mode == CWL_TEACHER_LOGITS) {
      const float mx = warp_max_nan(en.id >= 0 ? en.value : -CUDART_INF_F);
      if (lane == 0) sh.red[wid] = mx;
      __syncthreads();
      v_max = max_nan(max_nan(sh.red[0], sh.red[1]), max_nan(sh.red[2], sh.red[3]));
    }
    const double weight = warp_sum(entry_weight(p, v_max, en));
    const float mw = key_value(__reduce_max_sync(0xffffffffu, order_key(counts ? en.z : -CUDART_INF_F)));
    const float sw = warp_sum(counts && !bad_max(mw) ? exp2_fast((en.z - mw) * p.c) : 0.f);
    if (lane == 0) { sh.red_d[wid] = weight; sh.m_in[wid] = mw; sh.s_in[wid] = sw; }
    __syncthreads();                           // every thread is done with the marks
    if (en.id >= 0) marks[pos >> 5] = 0;
    if (tid == 0) sh.repeated = 0;
    finish_entry(p, v_max, (sh.red_d[0] + sh.red_d[1]) + (sh.red_d[2] + sh.red_d[3]), en);
    // all parts together: lanes 0..3 outside the entries, 4..7 the entries
    const int k = lane & (2 * kLossWarps - 1);
    const bool outside = k < kLossWarps;
    const float2 part = outside ? sh.part[k] : make_float2(sh.m_in[k - kLossWarps], sh.s_in[k - kLossWarps]);
    const float m = key_value(__reduce_max_sync(0xffffffffu, order_key(part.x)));
    const float mine = lane < 2 * kLossWarps ? part_sum(part, m, p.c) : 0.f;
    const float s_out = warp_sum(outside ? mine : 0.f), s_in = warp_sum(outside ? 0.f : mine);
    RowMass r = bad_max(m) ? bad_mass() : near_mass(m, s_out, s_in);
    if (!bad_max(m) && s_out < kNear) {
      const float m_out = key_value(__reduce_max_sync(0xffffffffu, order_key(outside ? part.x : -CUDART_INF_F)));
      r = far_mass(m, s_in, m_out, warp_sum(lane < kLossWarps ? part_sum(part, m_out, p.c) : 0.f), p.c);
    }
    const double term = warp_sum(loss_term(p, en.id, en.p, en.lp, en.z, en.p_in, rest_of(en.p_rest, r), r, tid));
    __syncthreads();                           // red_d was read
    if (lane == 0) sh.red_d[wid] = term;
    __syncthreads();
    if (tid == 0) {
      const double kl = (sh.red_d[0] + sh.red_d[1]) + (sh.red_d[2] + sh.red_d[3]);
      p.loss[row] = (float)((double)w * p.temperature * p.temperature * kl);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ long rows, few rows
constexpr int kEntryThreads = 128;             // warps 0..3 (prepare) and 4..7 (finish): one teacher entry a thread
constexpr int kSumThreads = 256;               // warps 8..15 and 16..23: sums and gradients of every other row
constexpr int kSumGroups = 2;
constexpr int kSumWarps = kSumThreads / 32;
constexpr int kPipeThreads = 2 * kEntryThreads + kSumGroups * kSumThreads + 32;   // the last warp copies slices in
constexpr int kMaxBuffers = 3;
constexpr int kSlots = 3;                      // rows under way between the roles of a block
constexpr int kClusterSlots = 6;               // rows under way between the blocks of a cluster
constexpr int kParts = kSumWarps + 1;          // parts of a slice's statistics: its sum warps', its entries'
constexpr int kAtOnce = 4;                       // vectors of a sum thread in the works at once
constexpr int kCopyBytes = 16 * 1024;          // piece of a slice that one bulk copy brings

struct DsPipe {
  alignas(8) unsigned long long full[kMaxBuffers], ready[kMaxBuffers], xchg[kClusterSlots];
  alignas(16) int misc[8];                     // [1] gave up, [4..5] wait limit in ns (the layout mbar_wait expects)
  float2 slot[kClusterSlots][kMaxDsCluster * kParts];   // (m, S) of every part of the row
  float z[kClusterSlots][CWL_MAX_TOP_K];       // student logits of the entries (in the first block: of all slices)
  EntryRest entry[kSlots][CWL_MAX_TOP_K];      // from prepare to finish
  float mass[kSlots][2];                       // sum of the teacher's probabilities, and what they leave to the rest
  int id[CWL_MAX_TOP_K];
  float p[CWL_MAX_TOP_K];
  float red[kEntryThreads / 32], red2[kEntryThreads / 32];
  double red_d[kEntryThreads / 32], red_loss[kEntryThreads / 32];
  int red_n[kEntryThreads / 32];
  int repeated;                                // some id occurs twice
};

struct PipePlan {
  int log2_cta, n_buffers, buffer_bytes;
};

// A row's masses from the parts of its slices, a part a lane of the warp (of eight slices, up to three).  Every sum warp waits
// for it: a block that has the row to itself reads its entries' part as it stands (2048 rows of 32000 bf16: 47.5 -> 46.5 us).
__device__ __forceinline__ RowMass row_statistics(const float2* part, int n_cta, float c) {
  const int lane = threadIdx.x & 31;
  float m = -CUDART_INF_F, s_out = 0.f, s_in = 0.f;
  if (n_cta == 1) {
    const float2 q = part[lane % kSumWarps], e = part[kSumWarps];
    m = max_nan(key_value(__reduce_max_sync(0xffffffffu, order_key(q.x))), e.x);
    s_out = part_sum(q, m, c);
    s_in = part_sum(e, m, c);
#pragma unroll
    for (int off = kSumWarps / 2; off > 0; off >>= 1) s_out += __shfl_xor_sync(0xffffffffu, s_out, off);
  } else {
    for (int i = lane; i < n_cta * kParts; i += 32) m = max_nan(m, part[i].x);
    m = key_value(__reduce_max_sync(0xffffffffu, order_key(m)));
    for (int i = lane; i < n_cta * kParts; i += 32) {
      const float v = part_sum(part[i], m, c);
      if (i % kParts == kSumWarps) s_in += v; else s_out += v;
    }
    s_out = warp_sum(s_out);
    s_in = warp_sum(s_in);
  }
  if (bad_max(m)) return bad_mass();
  if (s_out >= kNear) return near_mass(m, s_out, s_in);
  float m_out = -CUDART_INF_F;
  for (int i = lane; i < n_cta * kParts; i += 32)
    if (i % kParts != kSumWarps) m_out = max_nan(m_out, part[i].x);
  m_out = key_value(__reduce_max_sync(0xffffffffu, order_key(m_out)));
  s_out = 0.f;
  for (int i = lane; i < n_cta * kParts; i += 32)
    if (i % kParts != kSumWarps) s_out += part_sum(part[i], m_out, c);
  return far_mass(m, s_in, m_out, warp_sum(s_out), c);
}

__device__ __forceinline__ void prepare_barrier() { __syncwarp(); asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ void finish_barrier() { __syncwarp(); asm volatile("bar.sync 2, 128;" ::: "memory"); }
// the gradients of row n's slice are stored: the sum warps say so and go on, the finish warps wait for it
__device__ __forceinline__ void stored_arrive(int slot) { __syncwarp(); asm volatile("bar.arrive %0, 416;" ::"r"(3 + slot) : "memory"); }
__device__ __forceinline__ void stored_wait(int slot) { __syncwarp(); asm volatile("bar.sync %0, 416;" ::"r"(3 + slot) : "memory"); }
static_assert(kEntryThreads == 128 && kSumThreads == 256, "the barriers' counts");

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Stores to the shared memory of a block of the cluster that count their bytes on an mbarrier there: no fence, and so no
// wait for the gradients that the same thread has stored before.
__device__ __forceinline__ void st_async_f32(uint32_t cluster_addr, float v, uint32_t cluster_bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];"
               ::"r"(cluster_addr), "r"(__float_as_uint(v)), "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void st_async_2f32(uint32_t cluster_addr, float a, float b, uint32_t cluster_bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];"
               ::"r"(cluster_addr), "r"(__float_as_uint(a)), "r"(__float_as_uint(b)), "r"(cluster_bar) : "memory");
}
// The bounded wait of mbar_wait, ordered after what the whole cluster did before its arrivals.
__device__ __forceinline__ bool mbar_try_wait_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (mbar_try_wait_cluster(bar, parity)) return true;
  const unsigned long long t0 = global_timer();
  for (uint32_t spins = 1;; ++spins) {
    if (mbar_try_wait_cluster(bar, parity)) return true;
    if ((spins & 255u) == 0) {
      if (*abort_flag) return false;
      if (global_timer() - t0 > wait_limit(abort_flag)) { *abort_flag = 1; return false; }
    }
  }
}
__device__ __forceinline__ void bulk_copy_in(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// The rows first, first + stride, ... in groups of 32, a row a lane of the warp: their weights come with one load a group,
// a group ahead, and rows of weight 0 cost nothing.
struct RowCursor {
  const float* weight;
  int T, stride, base, row;      // first row of the group; the row at hand
  unsigned live;                 // rows of the group that are still to come
  float mine, ahead;             // this lane's weight in the group, in the next one
  __device__ __forceinline__ float weight_of(int64_t r) const { return r < T ? (weight != nullptr ? __ldg(weight + r) : 1.f) : 0.f; }
  __device__ __forceinline__ void enter(int64_t first) {
    base = (int)min(first, (int64_t)T);
    mine = ahead;
    ahead = weight_of(first + (int64_t)(32 + (threadIdx.x & 31)) * stride);
    live = __ballot_sync(0xffffffffu, mine != 0.f);           // a NaN is trained on, and 0 past the end
  }
  __device__ __forceinline__ void start(const float* w, int rows, int first, int step) {
    weight = w; T = rows; stride = step; row = first;
    ahead = weight_of(first + (int64_t)(threadIdx.x & 31) * stride);
    enter(first);
  }
  __device__ __forceinline__ bool next(float& w) {
    while (live == 0) {
      const int64_t after = (int64_t)base + 32ll * stride;
      if (after >= T) return false;
      enter(after);
    }
    const int k = __ffs((int)live) - 1;
    live &= live - 1;
    row = base + k * stride;
    w = __shfl_sync(0xffffffffu, mine, k);
    return true;
  }
};
// position in a ring of `size` places, and how often it went round (mod 2)
struct Ring {
  int at = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int size) {
    if (++at == size) { at = 0; phase ^= 1u; }
  }
};

// One block: rows first, first + stride, ...; rows of weight 0 take no part in the numbering below.  Row number n goes
// through buffer n % n_buffers:
//   copy warp        brings the slice in (full), as soon as row n - n_buffers has left the buffer
//   prepare warps    entries of the teacher; once the slice is there, lift the entries out of it (ready)
//   sum warps        two groups for every other row, so that one sums while the other waits or stores: sum what is left;
//                    each warp's (m, S), and the entries', go to every block of the cluster (xchg), and once all have
//                    arrived the gradient of the slice is stored (stored)
//   finish warps     loss (in the first block of the cluster); gradient of the entries
// How far they drift apart: row k needs its copy, so its block's finish is past row k - n_buffers wherever prepare or the
// sums are at row k: three slots and `stored` barriers serve a block.  Past row k - 3 also means that every block has sent
// its statistics of row k - 3, so its finish is past row k - 6: six slots serve a cluster.
// Every wait on a barrier in memory is bounded; one that runs out raises CWL_ERR_TIMEOUT, after which nothing is stored
// any more, but the loops run to their end so that no other warp or block is left waiting.
template <typename T>
__global__ void __launch_bounds__(kPipeThreads, 1)
distill_pipe_kernel(const DistillParams p, const PipePlan plan) {
  constexpr int kVec = Elem<T>::kVec;
  pdl_launch_dependents();
  extern __shared__ __align__(128) uint8_t ds_raw[];
  DsPipe& sh = *reinterpret_cast<DsPipe*>(ds_raw + plan.n_buffers * plan.buffer_bytes);
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int log2_cta = plan.log2_cta, n_cta = 1 << log2_cta;
  const int cta = log2_cta > 0 ? (int)cluster_rank() : 0;
  const int first = blockIdx.x >> log2_cta, stride = gridDim.x >> log2_cta;
  volatile int* abort_flag = sh.misc + 1;
  auto full_bar = [&](int b) { return smem_u32(&sh.full[b]); };
  auto ready_bar = [&](int b) { return smem_u32(&sh.ready[b]); };
  auto xchg_bar = [&](int k) { return smem_u32(&sh.xchg[k]); };
  if (tid == 0) {
    for (int b = 0; b < kMaxBuffers; ++b) { mbar_init(full_bar(b), 1); mbar_init(ready_bar(b), 1); }
    for (int k = 0; k < kClusterSlots; ++k) mbar_init(xchg_bar(k), 1);
    sh.misc[1] = 0;
    *reinterpret_cast<volatile unsigned long long*>(sh.misc + 4) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (log2_cta > 0) cluster_barrier();             // the peers' barriers exist before anything arrives on them
  pdl_wait();

  auto row_of = [&](int row) { return reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.ld; };
  auto lead_of = [&](const RowSlice& rs) { return (kVec - rs.own_head % kVec) % kVec; };
  auto cluster_addr = [&](const void* ptr, uint32_t block) { return log2_cta > 0 ? peer_shared(ptr, block) : smem_u32(ptr); };
  // one part of a row's statistics to every block of the cluster, from the first lanes of a warp
  auto send_part = [&](int slot, int part, float m, float s) {
    if (lane < n_cta)
      st_async_2f32(cluster_addr(&sh.slot[slot][cta * kParts + part], lane), m, s,
                    cluster_addr(&sh.xchg[slot], lane));
    __syncwarp();
  };
  // element i of the row sits at image[i - e0 + lead]; its vectors begin after own_head + lead elements
  auto image_of = [&](int buffer) { return reinterpret_cast<T*>(ds_raw + buffer * plan.buffer_bytes); };

  if (wid < kEntryThreads / 32) {
    // ---------------------------------------------------------------------------------------------- prepare warps
    RowCursor at;
    at.start(p.weight, p.T, first, stride);
    float w, w_after;
    bool more = at.next(w);
    Entry en;
    if (more) load_entry(p, at.row, tid, en);
    Ring buf, slot, cslot;
    for (; more; buf.step(plan.n_buffers), slot.step(kSlots), cslot.step(kClusterSlots)) {
      const int row = at.row;
      more = at.next(w_after);
      Entry after;
      if (more) load_entry(p, at.row, tid, after);       // a row ahead
      check_entry(p, en);
      const T* z = row_of(row);
      const RowSlice rs = row_slice<T>(z, p.V, cta, log2_cta);
      T* sm = image_of(buf.at) + lead_of(rs) - rs.e0;         // element i of the row at sm[i]
      float v_max = 0.f;
      if (p.mode == CWL_TEACHER_LOGITS) {
        const float mx = warp_max_nan(en.id >= 0 ? en.value : -CUDART_INF_F);
        if (lane == 0) sh.red[wid] = mx;
        prepare_barrier();
        v_max = max_nan(max_nan(sh.red[0], sh.red[1]), max_nan(sh.red[2], sh.red[3]));
      }
      const double part = warp_sum(entry_weight(p, v_max, en));
      const int valid = __popc(__ballot_sync(0xffffffffu, en.id >= 0));
      if (lane == 0) { sh.red_d[wid] = part; sh.red_n[wid] = valid; }
      prepare_barrier();
      const int n_valid = (sh.red_n[0] + sh.red_n[1]) + (sh.red_n[2] + sh.red_n[3]);
      finish_entry(p, v_max, (sh.red_d[0] + sh.red_d[1]) + (sh.red_d[2] + sh.red_d[3]), en);
      if (tid < p.K) { sh.id[tid] = en.id; sh.p[tid] = en.p; }
      if (tid == 0) sh.repeated = 0;
      const bool mine = en.id >= rs.e0 && en.id < rs.e1;
      mbar_wait(full_bar(buf.at), buf.phase, abort_flag);
      __syncwarp();
      if (tid < rs.own_head) sm[tid] = z[tid];
      if (tid < rs.own_tail) sm[rs.tail_start + tid] = z[rs.tail_start + tid];
      prepare_barrier();                                 // head and tail scalars are there too
      if (mine) en.z = Elem<T>::to_float(sm[en.id]);
      prepare_barrier();                                 // every entry was read: each leaves its number in its place
      if (mine) Elem<T>::put_number(sm + en.id, tid);
      prepare_barrier();
      if (mine && Elem<T>::number_at(sm + en.id) != tid) sh.repeated = 1;
      const float mw = key_value(__reduce_max_sync(0xffffffffu, order_key(mine ? en.z : -CUDART_INF_F)));
      if (lane == 0) sh.red[wid] = mw;
      prepare_barrier();
      en.p_id = mine ? en.p : -1.f;
      if (sh.repeated && mine) en.p_id = merged_probability(sh.id, sh.p, p.K, tid);
      if (mine) {
        sm[en.id] = Elem<T>::from_float(-CUDART_INF_F);
        if (p.loss != nullptr)
          st_async_f32(cluster_addr(&sh.z[cslot.at][tid], 0), en.z, cluster_addr(&sh.xchg[cslot.at], 0));
      }
      // (m, S) of this slice's entries, every distinct id once
      const float me = max_nan(max_nan(sh.red[0], sh.red[1]), max_nan(sh.red[2], sh.red[3]));
      const float sw = warp_sum(en.p_id >= 0.f && !bad_max(me) ? exp2_fast((en.z - me) * p.c) : 0.f);
      if (lane == 0) sh.red2[wid] = sw;
      if (tid < p.K) sh.entry[slot.at][tid] = EntryRest{en.lp, en.id, en.p, en.p_id, en.z};
      prepare_barrier();
      if (tid == 0) {
        sh.mass[slot.at][0] = en.p_in;
        sh.mass[slot.at][1] = en.p_rest;
        // what will arrive for this row: every part of its statistics and, in the first block, every entry's logit
        mbar_expect_tx(xchg_bar(cslot.at),
                       (uint32_t)(n_cta * kParts * sizeof(float2)) + (p.loss != nullptr && cta == 0 ? (uint32_t)n_valid * 4u : 0u));
        mbar_arrive(ready_bar(buf.at));
      }
      if (wid == 0) send_part(cslot.at, kSumWarps, me, (sh.red2[0] + sh.red2[1]) + (sh.red2[2] + sh.red2[3]));
      en = after;
    }
  } else if (wid < 2 * kEntryThreads / 32) {
    // ----------------------------------------------------------------------------------------------- finish warps
    const int ft = tid - kEntryThreads, fw = wid - kEntryThreads / 32;
    RowCursor at;
    at.start(p.weight, p.T, first, stride);
    float w;
    Ring slot, cslot;
    for (; at.next(w); slot.step(kSlots), cslot.step(kClusterSlots)) {
      const int row = at.row;
      const float dl = p.dloss != nullptr ? __ldg(p.dloss + row) : 1.f;
      const bool ok = mbar_wait_cluster(xchg_bar(cslot.at), cslot.phase, abort_flag);
      __syncwarp();
      const RowMass r = row_statistics(sh.slot[cslot.at], n_cta, p.c);
      EntryRest e{0.0, -1, 0.f, -1.f, 0.f};
      if (ft < p.K) e = sh.entry[slot.at][ft];
      const float p_in = sh.mass[slot.at][0], p_rest = rest_of(sh.mass[slot.at][1], r);
      if (p.loss != nullptr && cta == 0) {
        const double term = warp_sum(loss_term(p, e.id, e.p, e.lp, ft < p.K ? sh.z[cslot.at][ft] : 0.f, p_in, p_rest, r, ft));
        if (lane == 0) sh.red_loss[fw] = term;
        finish_barrier();
        if (ft == 0 && ok) {
          const double kl = (sh.red_loss[0] + sh.red_loss[1]) + (sh.red_loss[2] + sh.red_loss[3]);
          p.loss[row] = (float)((double)w * p.temperature * p.temperature * kl);
        }
      }
      stored_wait(slot.at);
      if (p.dlogits != nullptr && e.p_id >= 0.f && ok && *abort_flag == 0) {
        T* d = reinterpret_cast<T*>(p.dlogits) + (int64_t)row * p.ld_d;
        d[e.id] = Elem<T>::from_float(entry_gradient(p, e.z, e.p_id, p_in + p_rest, r.m, r.s_row) * (w * p.temperature * dl));
      }
    }
  } else if (wid == kPipeThreads / 32 - 1) {
    // -------------------------------------------------------------------------------------------------- copy warp
    RowCursor loads;
    loads.start(p.weight, p.T, first, stride);
    int loaded = 0;
    uint32_t copied = 0, odd = 0;                            // buffers that were filled at all; filled an odd number of times
    Ring buf, past;                                          // `past`: slot of the row whose buffer comes free next
    float w;
    while (loads.next(w)) {
      if (loaded >= plan.n_buffers) { stored_wait(past.at); past.step(kSlots); }
      if (lane == 0 && !(CWL_WITHHELD(p) && loaded == 1)) {
        copied |= 1u << buf.at;
        odd ^= 1u << buf.at;
        asm volatile("fence.proxy.async;" ::: "memory");   // the buffer was read and written with ordinary accesses
        const T* z = row_of(loads.row);
        const RowSlice rs = row_slice<T>(z, p.V, cta, log2_cta);
        const uint32_t bytes = (uint32_t)(rs.v1 - rs.v0) * 16u;
        const uint8_t* src = reinterpret_cast<const uint8_t*>(z + rs.head) + (int64_t)rs.v0 * 16;
        const uint32_t dst = smem_u32(image_of(buf.at) + rs.own_head + lead_of(rs));
        mbar_expect_tx(full_bar(buf.at), bytes);                // an arrival that expects no bytes completes at once
        for (uint32_t off = 0; off < bytes; off += kCopyBytes)
          bulk_copy_in(dst + off, src + off, min(bytes - off, (uint32_t)kCopyBytes), full_bar(buf.at));
      }
      __syncwarp();
      buf.step(plan.n_buffers);
      ++loaded;
    }
    for (int n = min(loaded, plan.n_buffers); n > 0; --n) { stored_wait(past.at); past.step(kSlots); }   // every row counts this warp
    // Where a wait ran out, copies may still be on their way: they get a bounded chance to land.
    for (int b = 0; b < kMaxBuffers; ++b) {
      if (lane != 0 || ((copied >> b) & 1u) == 0) continue;
      const unsigned long long t0 = global_timer();
      while (!mbar_try_wait(full_bar(b), ((odd >> b) & 1u) ^ 1u) && global_timer() - t0 < p.wait_limit_ns) {}
    }
    __syncwarp();
  } else {
    // -------------------------------------------------------------------------------------------------- sum warps
    const int group = (tid - 2 * kEntryThreads) / kSumThreads;
    const int st = (tid - 2 * kEntryThreads) % kSumThreads, sw = st >> 5;
    // rows of weight 0 are not read; their zeros go out first, while the first slices come in
    if (p.weight != nullptr) {
      int turn = 0;
      for (int64_t row0 = first; row0 < p.T; row0 += 32ll * stride) {
        const int64_t mine = row0 + (int64_t)lane * stride;
        unsigned dead = __ballot_sync(0xffffffffu, mine < p.T && __ldg(p.weight + min(mine, (int64_t)p.T - 1)) == 0.f);
        for (; dead != 0; dead &= dead - 1) {
          if ((turn++ & (kSumGroups - 1)) != group) continue;
          const int64_t row = row0 + (int64_t)(__ffs((int)dead) - 1) * stride;
          if (p.dlogits != nullptr) {
            const T* z = row_of((int)row);
            T* d = reinterpret_cast<T*>(p.dlogits) + row * p.ld_d;
            zero_slice<T, kSumThreads>(st, d, ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(d)) & 15u) == 0,
                                       row_slice<T>(z, p.V, cta, log2_cta));
          }
          if (p.loss != nullptr && cta == 0 && st == 0) p.loss[row] = 0.f;
        }
      }
    }
    RowCursor at;
    at.start(p.weight, p.T, first, stride);
    Ring buf, slot, cslot;
    float w;
    int turn = 0;
    for (; at.next(w); buf.step(plan.n_buffers), slot.step(kSlots), cslot.step(kClusterSlots)) {
      if ((turn++ & (kSumGroups - 1)) != group) continue;
      const int row = at.row;
      const T* z = row_of(row);
      T* d = p.dlogits != nullptr ? reinterpret_cast<T*>(p.dlogits) + (int64_t)row * p.ld_d : nullptr;
      const RowSlice rs = row_slice<T>(z, p.V, cta, log2_cta);
      const bool same_phase = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(d)) & 15u) == 0;
      const float up = w * p.temperature * (p.dloss != nullptr ? __ldg(p.dloss + row) : 1.f);
      const T* sm = image_of(buf.at) + lead_of(rs) - rs.e0;
      const uint4* sv = reinterpret_cast<const uint4*>(image_of(buf.at) + rs.own_head + lead_of(rs));
      const int nv = rs.v1 - rs.v0;
      mbar_wait(ready_bar(buf.at), buf.phase, abort_flag);
      __syncwarp();

      RunningSum run;
      run.start(p.ordinary != 0);
      int i = st;
      for (; i + (kAtOnce - 1) * kSumThreads < nv; i += kAtOnce * kSumThreads) {
        uint32_t words[4 * kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const uint4 q = sv[i + u * kSumThreads];
          words[4 * u] = q.x; words[4 * u + 1] = q.y; words[4 * u + 2] = q.z; words[4 * u + 3] = q.w;
        }
        run.template take_words<T, 4 * kAtOnce>(words, Elem<T>::max_of(words), p.c);
      }
      for (; i < nv; i += kSumThreads) {
        const uint4 q = sv[i];
        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
        run.template take_words<T, 4>(words, Elem<T>::max_of(words), p.c);
      }
      RowStat a = run.done(p.c);
      if (run.exact_needed) a = exact_stat<T>(sv, st, kSumThreads, nv, p.c);
      if (st < rs.own_head) absorb_scalar(a, Elem<T>::to_float(sm[st]), p.c);
      if (st < rs.own_tail) absorb_scalar(a, Elem<T>::to_float(sm[rs.tail_start + st]), p.c);
      rescale(a, key_value(__reduce_max_sync(0xffffffffu, order_key(a.m))), p.c);
      send_part(cslot.at, sw, a.m, warp_sum(a.S));
      const bool ok = mbar_wait_cluster(xchg_bar(cslot.at), cslot.phase, abort_flag);
      __syncwarp();
      if (d != nullptr && ok && *abort_flag == 0) {
        const RowMass r = row_statistics(sh.slot[cslot.at], n_cta, p.c);
        const float m = r.m_out;                                   // what the elements outside are relative to
        const float p_in = sh.mass[slot.at][0], rest = rest_of(sh.mass[slot.at][1], r);
        const float k_out = outside_factor(p_in + rest, rest, r) * up;
        if (nothing_taught(p_in, rest)) {
          zero_slice<T, kSumThreads>(st, d, same_phase, rs);
        } else if (fabsf(m) <= kOrdinaryLogit && p.ordinary != 0) {
          const float M = m * p.c;
          const float k = k_out * exp2_fast(-fmaf(m, p.c, -M));
          const uint64_t c2 = pair(p.c, p.c), minus_m = pair(-M, -M), k2 = pair(k, k), zero = pair(0.f, 0.f);
          auto grad_vec = [&](const uint4& q, float (&f)[kVec]) {
            const uint32_t words[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < kVec / 2; ++e) {
              float t0, t1;
              unpair(fma_pair(Elem<T>::unpack_pair(words + e * Elem<T>::kPairWords), c2, minus_m), t0, t1);
              unpair(fma_pair(pair(exp2_fast(t0), exp2_fast(t1)), k2, zero), f[2 * e], f[2 * e + 1]);
            }
          };
          if (same_phase) {
            const uint4* in = sv + st;
            uint4* out = reinterpret_cast<uint4*>(d + rs.head) + rs.v0 + st;
            int left = nv - st;
            for (; left > (kAtOnce - 1) * kSumThreads; left -= kAtOnce * kSumThreads, in += kAtOnce * kSumThreads, out += kAtOnce * kSumThreads) {
              uint4 q[kAtOnce];
#pragma unroll
              for (int u = 0; u < kAtOnce; ++u) q[u] = in[u * kSumThreads];
#pragma unroll
              for (int u = 0; u < kAtOnce; ++u) {
                float f[kVec];
                grad_vec(q[u], f);
                out[u * kSumThreads] = Elem<T>::pack(f);
              }
            }
            for (; left > 0; left -= kSumThreads, in += kSumThreads, out += kSumThreads) {
              float f[kVec];
              grad_vec(*in, f);
              *out = Elem<T>::pack(f);
            }
            if (st < rs.own_head) d[st] = Elem<T>::from_float(exp2_fast((Elem<T>::to_float(sm[st]) - m) * p.c) * k_out);
            if (st < rs.own_tail) {
              const int x = rs.tail_start + st;
              d[x] = Elem<T>::from_float(exp2_fast((Elem<T>::to_float(sm[x]) - m) * p.c) * k_out);
            }
          } else {
            store_slice<T, kSumThreads>(st, d, false, rs, [](int, float (&)[kVec]) {},
                                        [&](int x) { return exp2_fast(fmaf(Elem<T>::to_float(sm[x]), p.c, -M)) * k; });
          }
        } else {
          store_slice<T, kSumThreads>(st, d, same_phase, rs, [&](int v, float (&f)[kVec]) {
            Elem<T>::unpack(sv[v - rs.v0], f);
#pragma unroll
            for (int e = 0; e < kVec; ++e) f[e] = exp2_fast((f[e] - m) * p.c) * k_out;
          }, [&](int x) { return exp2_fast((Elem<T>::to_float(sm[x]) - m) * p.c) * k_out; });
        }
      }
      stored_arrive(slot.at);
    }
  }
  __syncthreads();
  if (tid == 0 && *abort_flag != 0) flag_status(p.status_word, CWL_ERR_TIMEOUT);
  if (log2_cta > 0) {
    cluster_barrier();                             // nobody leaves while a peer may still write to it
    if (*abort_flag != 0) {                        // a block that gave up has not waited for all that is sent to it
      const unsigned long long t0 = global_timer();
      while (global_timer() - t0 < 1000000ull) {}
    }
  }
}

static_assert(sizeof(DsPipe) + CWL_MAX_DISTILL_ROW_BYTES / kMaxDsCluster + 160 <= 227 * 1024, "the longest row fits a cluster");
// How the long-row kernel runs: as few blocks a row as hold it in slices of kSliceWanted bytes (two buffers fit), more
// while the rows do not fill the GPU, down to slices of 8 KB.  Half the slice with a third buffer costs more in exchanges than
// the buffer gives (us, slices up to 66 KB -> up to 104 KB: 2587 rows of 142736 bf16 417 -> 286; 4096 rows of 50000 fp32 298
// -> 258, of 100000 fp32 635 -> 551, of 25000 fp32 154 -> 133).
constexpr int kSliceWanted = 104 * 1024;
PipePlan pipe_plan(int T, int64_t row_bytes) {
  PipePlan plan;
  plan.log2_cta = 0;
  while ((1 << plan.log2_cta) < kMaxDsCluster && (row_bytes >> plan.log2_cta) > kSliceWanted) ++plan.log2_cta;
  while ((1 << plan.log2_cta) < kMaxDsCluster && ((int64_t)T << (plan.log2_cta + 1)) <= 148 && (row_bytes >> (plan.log2_cta + 1)) >= 8192)
    ++plan.log2_cta;
  const int c = 1 << plan.log2_cta;
  // one slice: its vectors, and head and tail scalars in a vector of their own each
  plan.buffer_bytes = ((int)((row_bytes / 16 + c - 1) / c) * 16 + 32 + 127) / 128 * 128;
  plan.n_buffers = (227 * 1024 - (int)sizeof(DsPipe)) / plan.buffer_bytes;
  if (plan.n_buffers > kMaxBuffers) plan.n_buffers = kMaxBuffers;
  return plan;
}

// Clusters of long-row blocks that fit the GPU at once, one block an SM; the rows are dealt to that many.  Asked with all of an
// SM's shared memory: the plans' own shares go down to a fifth of it, but 800 threads of 72 registers leave no room for a second.
template <typename T>
int resident_clusters(int log2_cta) {
  constexpr int kDevices = 32;
  static std::atomic<int> known[kDevices][4];      // by device and log2_cta
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) dev = kDevices;
  if (dev < kDevices) {
    const int seen = known[dev][log2_cta].load(std::memory_order_relaxed);
    if (seen > 0) return seen;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(148u >> log2_cta << log2_cta);
  cfg.blockDim = dim3(kPipeThreads);
  cfg.dynamicSmemBytes = 227 * 1024;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 1u << log2_cta; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, distill_pipe_kernel<T>, &cfg) != cudaSuccess || n <= 0) {
    cudaGetLastError();
    return 148 >> log2_cta;
  }
  if (dev < kDevices) known[dev][log2_cta].store(n, std::memory_order_relaxed);
  return n;
}

template <typename T, int kBlocks>
cudaError_t launch_loss(const DistillParams& p, bool chained, cudaStream_t st) {
  const int words = (p.V + 2 * Elem<T>::kVec + 31) / 32;
  static SharedMemoryGrant grant;
  const cudaError_t e = grant(distill_loss_kernel<T, kBlocks>);
  if (e != cudaSuccess) return e;
  const int rows = p.T < (1 << 20) ? p.T : (1 << 20);
  return launch_chained(chained, distill_loss_kernel<T, kBlocks>, dim3(rows), dim3(kLossThreads),
                        sizeof(LossShared) + words * sizeof(uint32_t), st, p, words);
}

template <typename T>
cudaError_t launch_distill(const DistillParams& p, cudaStream_t st) {
  const int64_t row_bytes = (int64_t)p.V * sizeof(T);
  const bool chained = !stream_is_capturing(st);
  if (row_bytes <= kSmallRowBytes || (row_bytes <= kSmallManyRowBytes && p.T >= kSmallManyRows && p.dlogits != nullptr)) {
    const size_t smem = (size_t)(row_bytes / 16) * 16 + 32;
    const int rows = p.T < (1 << 20) ? p.T : (1 << 20);
    return launch_chained(chained, distill_small_kernel<T>, dim3(rows), dim3(kDsThreads), smem, st, p);
  }
  if (p.dlogits == nullptr && p.T >= kLossMinRows) {
    return p.T <= 7 * 148 ? launch_loss<T, 7>(p, chained, st) : launch_loss<T, 8>(p, chained, st);
  }
  const PipePlan plan = pipe_plan(p.T, row_bytes);
  const size_t smem = (size_t)plan.n_buffers * plan.buffer_bytes + sizeof(DsPipe);
  static SharedMemoryGrant grant;
  const cudaError_t e = grant(distill_pipe_kernel<T>);
  if (e != cudaSuccess) return e;
  const int clusters = resident_clusters<T>(plan.log2_cta);
  const int rows = p.T < clusters ? p.T : clusters;
  return launch_clusters(chained, 1 << plan.log2_cta, distill_pipe_kernel<T>, dim3(rows << plan.log2_cta), dim3(kPipeThreads), smem, st,
                         p, plan);
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
  const float tau = cwl::usable_temperature(temperature);
  cwl::DistillParams p{logits, ld_logits, T, V, teacher_ids, teacher_values, ld_teacher, K, (int)mode, tau,
                       (float)(1.4426950408889634074 / (double)tau), (float)(1.0 / (double)tau), 1.0 / (double)tau,
                       cwl::ordinary_temperature(tau) ? 1 : 0, weight, dloss,
                       loss, dlogits, ld_dlogits, status_word, cwl::training_wait_limit(), cwl::training_withhold()};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case CWL_F32: CWL_CUDA_TRY(cwl::launch_distill<float>(p, st)); break;
    case CWL_BF16: CWL_CUDA_TRY(cwl::launch_distill<__nv_bfloat16>(p, st)); break;
    default: CWL_CUDA_TRY(cwl::launch_distill<__half>(p, st)); break;
  }
  return CWL_OK;
}

#ifdef CWL_TEST_HOOKS
namespace cwl {
std::atomic<unsigned long long> g_training_wait_limit_ns{kTrainingWaitLimitNs};
std::atomic<int> g_training_withhold{0};
}  // namespace cwl
extern "C" void cwl_debug_training_set(int64_t wait_limit_ns, int32_t withhold) {
  cwl::g_training_wait_limit_ns.store(wait_limit_ns > 0 ? (unsigned long long)wait_limit_ns : cwl::kTrainingWaitLimitNs);
  cwl::g_training_withhold.store(withhold != 0 ? 1 : 0);
}
#endif

// Shared pieces of the kernels that walk logit rows of several types (logprobs.cu, distill.cu): 16-byte access to rows
// that may start at any element, the online softmax triple, clusters of CTAs that share a row.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "cluster.cuh"
#include "cwl_common.cuh"

namespace cwl {

constexpr float kRowLn2 = 0.6931471805599453f;
constexpr float kMaskedLogit = -1.0e30f;
constexpr float kMaskedExponent = -1.0e30f;   // stands for -inf where a weight of 0 is multiplied with its exponent

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// maximum that a NaN on either side wins: the maximum of a row then tells a bad row by itself
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// true for a row maximum that leaves the softmax undefined: NaN, +inf, or nothing but -inf
__device__ __forceinline__ bool bad_max(float m) { return !(m < CUDART_INF_F) || m == -CUDART_INF_F; }

// Two fp32 numbers in one 64-bit register: one instruction slot does both.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ void unpair(uint64_t p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Element types of a logit row: how many sit in 16 bytes, how they become fp32 and how a gradient is rounded back.
template <typename T> struct Elem;
template <> struct Elem<float> {
  static constexpr int kVec = 4;
  static constexpr int kZeroBits = 0;     // low bits that are 0 in every value's fp32 form
  static __device__ __forceinline__ float load(const float* p) { return __ldg(p); }
  static __device__ __forceinline__ float to_float(float v) { return v; }
  static __device__ __forceinline__ float from_float(float v) { return v; }
  // a small whole number in the place of an element
  static __device__ __forceinline__ void put_number(float* p, int n) { *reinterpret_cast<volatile int*>(p) = n; }
  static __device__ __forceinline__ int number_at(const float* p) { return *reinterpret_cast<const volatile int*>(p); }
  static __device__ __forceinline__ void unpack(const uint4& q, float (&f)[4]) {
    f[0] = __uint_as_float(q.x); f[1] = __uint_as_float(q.y); f[2] = __uint_as_float(q.z); f[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  // the first element of a vector, which moves up by one
  static __device__ __forceinline__ float shift_out(uint4& q) {
    const float f = __uint_as_float(q.x);
    q.x = q.y; q.y = q.z; q.z = q.w;
    return f;
  }
  static __device__ __forceinline__ uint32_t masked() { return 0xFF800000u; }   // -inf
  // the elements of a vector whose bits are set become -inf
  static __device__ __forceinline__ void mask_out(uint4& q, uint32_t bits) {
    if (bits & 1u) q.x = 0xFF800000u;
    if (bits & 2u) q.y = 0xFF800000u;
    if (bits & 4u) q.z = 0xFF800000u;
    if (bits & 8u) q.w = 0xFF800000u;
  }
  // maximum of the elements of n words, NaN wins
  template <int n> static __device__ __forceinline__ float max_of(const uint32_t (&w)[n]) {
    float m = __uint_as_float(w[0]);
#pragma unroll
    for (int i = 1; i < n; ++i) m = max_nan(m, __uint_as_float(w[i]));
    return m;
  }
  // two elements, -inf (and whatever lies below kMaskedLogit) made finite: of weight 0 beside an ordinary maximum
  static constexpr int kPairWords = 2;
  static __device__ __forceinline__ uint64_t unpack_pair(const uint32_t* w) { return pair(__uint_as_float(w[0]), __uint_as_float(w[1])); }
  static __device__ __forceinline__ uint64_t unpack_pair_floored(const uint32_t* w) {
    return pair(fmaxf(__uint_as_float(w[0]), kMaskedLogit), fmaxf(__uint_as_float(w[1]), kMaskedLogit));
  }
};
template <> struct Elem<__nv_bfloat16> {
  static constexpr int kVec = 8;
  static constexpr int kZeroBits = 16;
  static __device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(__ldg(p)); }
  static __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
  static __device__ __forceinline__ void put_number(__nv_bfloat16* p, int n) { *reinterpret_cast<volatile unsigned short*>(p) = (unsigned short)n; }
  static __device__ __forceinline__ int number_at(const __nv_bfloat16* p) { return *reinterpret_cast<const volatile unsigned short*>(p); }
  static __device__ __forceinline__ void unpack(const uint4& q, float (&f)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float shift_out(uint4& q) {
    const float f = __uint_as_float(q.x << 16);
    q.x = __funnelshift_r(q.x, q.y, 16); q.y = __funnelshift_r(q.y, q.z, 16); q.z = __funnelshift_r(q.z, q.w, 16); q.w >>= 16;
    return f;
  }
  static __device__ __forceinline__ uint32_t masked() { return 0xFF80FF80u; }
  static __device__ __forceinline__ void mask_out(uint4& q, uint32_t bits) {
    auto word = [](uint32_t w, uint32_t two) {
      if (two & 1u) w = (w & 0xFFFF0000u) | 0xFF80u;
      if (two & 2u) w = (w & 0x0000FFFFu) | (0xFF80u << 16);
      return w;
    };
    q.x = word(q.x, bits); q.y = word(q.y, bits >> 2); q.z = word(q.z, bits >> 4); q.w = word(q.w, bits >> 6);
  }
  template <int n> static __device__ __forceinline__ float max_of(const uint32_t (&w)[n]) {
    uint32_t m = w[0];
#pragma unroll
    for (int i = 1; i < n; ++i) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i]));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
  static constexpr int kPairWords = 1;
  static __device__ __forceinline__ uint64_t unpack_pair(const uint32_t* w) {
    return pair(__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint64_t unpack_pair_floored(const uint32_t* w) {
    uint32_t y;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(w[0]), "r"(0xF149F149u));     // kMaskedLogit in bf16, twice
    return pair(__uint_as_float(y << 16), __uint_as_float(y & 0xFFFF0000u));
  }
};
template <> struct Elem<__half> {
  static constexpr int kVec = 8;
  static constexpr int kZeroBits = 13;
  static __device__ __forceinline__ float load(const __half* p) { return __half2float(__ldg(p)); }
  static __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
  static __device__ __forceinline__ void put_number(__half* p, int n) { *reinterpret_cast<volatile unsigned short*>(p) = (unsigned short)n; }
  static __device__ __forceinline__ int number_at(const __half* p) { return *reinterpret_cast<const volatile unsigned short*>(p); }
  static __device__ __forceinline__ void unpack(const uint4& q, float (&f)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      f[2 * i] = v.x; f[2 * i + 1] = v.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float shift_out(uint4& q) {
    const float f = __half2float(__ushort_as_half((unsigned short)(q.x & 0xFFFFu)));
    q.x = __funnelshift_r(q.x, q.y, 16); q.y = __funnelshift_r(q.y, q.z, 16); q.z = __funnelshift_r(q.z, q.w, 16); q.w >>= 16;
    return f;
  }
  static __device__ __forceinline__ uint32_t masked() { return 0xFC00FC00u; }
  static __device__ __forceinline__ void mask_out(uint4& q, uint32_t bits) {
    auto word = [](uint32_t w, uint32_t two) {
      if (two & 1u) w = (w & 0xFFFF0000u) | 0xFC00u;
      if (two & 2u) w = (w & 0x0000FFFFu) | (0xFC00u << 16);
      return w;
    };
    q.x = word(q.x, bits); q.y = word(q.y, bits >> 2); q.z = word(q.z, bits >> 4); q.w = word(q.w, bits >> 6);
  }
  template <int n> static __device__ __forceinline__ float max_of(const uint32_t (&w)[n]) {
    uint32_t m = w[0];
#pragma unroll
    for (int i = 1; i < n; ++i) asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i]));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return max_nan(v.x, v.y);
  }
  static constexpr int kPairWords = 1;
  static __device__ __forceinline__ uint64_t unpack_pair(const uint32_t* w) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(w));
    return pair(v.x, v.y);
  }
  static __device__ __forceinline__ uint64_t unpack_pair_floored(const uint32_t* w) {
    uint32_t y;
    asm("max.f16x2 %0, %1, %2;" : "=r"(y) : "r"(w[0]), "r"(0xFBFFFBFFu));      // the type's lowest value, twice
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&y));
    return pair(v.x, v.y);
  }
};

// Online softmax statistics of what a thread (then a warp, a CTA, a cluster) has seen:
//   m = max z,  S = sum 2^t,  U = sum t 2^t,  t = (z - m) c,  c = log2(e) / temperature.
struct RowStat { float m, S, U; };

// Moves a triple to a new (not smaller) maximum; m == -inf means nothing was seen.  A NaN or +inf maximum is told by m
// alone, S and U are then of no account.
__device__ __forceinline__ void rebase(RowStat& a, float m_new, float c) {
  const float dt = (a.m - m_new) * c;     // <= 0; -inf for an empty triple
  const float sc = exp2_fast(dt);
  a.U = sc > 0.f ? (a.U + dt * a.S) * sc : 0.f;
  a.S = sc > 0.f ? a.S * sc : 0.f;
  a.m = m_new;
}
__device__ __forceinline__ void absorb(RowStat& a, float z, float c) {
  // z - m first: exact when z == m however large m is, so rows of the type's lowest value keep their uniform softmax
  const float t = fmaxf((z - a.m) * c, kMaskedExponent);
  const float e = exp2_fast(t);
  a.S += e;
  a.U = fmaf(t, e, a.U);
}
__device__ __forceinline__ void absorb_scalar(RowStat& a, float v, float c) {
  const float m_new = max_nan(a.m, v);
  if (m_new == -CUDART_INF_F) return;
  if (m_new != a.m) rebase(a, m_new, c);
  absorb(a, v, c);
}

// A thread's running statistic over batches of 16-byte vectors, for rows whose maximum is an ordinary number (|m| up to
// kOrdinaryLogit, and a temperature between 1/100 and 100).  Two elements a step: t = z c - M, M = m c rounded once, and
// -inf is replaced beforehand by a finite value of weight 0 (for 16-bit types one instruction for two elements, and so
// is the maximum): 4.5 instruction slots an element, the exponential among them, where the plain form takes 8; a row of
// 16-bit logits is bound by them.  The reference m follows the maximum only when that runs ahead by kLead powers of two,
// which leaves the sums far below fp32's range and saves the rescaling of nearly every batch.  A batch is summed by itself, so
// that a large term is met by as few additions as there are batches (16384 rows of 32000 bf16: error of the log-probabilities
// against 64 bits 6.6e-8 -> 3.1e-8, 267.7 -> 270.3 us).  A thread that met an extraordinary maximum says so in the end
// (`exact_needed`), and its elements are taken again in the form t = (z - m) c with the exponent clamped.
constexpr float kOrdinaryLogit = 16384.f;
constexpr float kLead = 8.f;
template <bool kWithU>
struct Running {
  float m, M, limit;           // reference; m c rounded; the batch maximum up to which the reference stays
  uint64_t S2, U2;             // sums over even and odd elements
  bool exact_needed;
  __device__ __forceinline__ void start(bool ordinary_temperature) {
    m = -CUDART_INF_F; M = 0.f; limit = -CUDART_INF_F; S2 = 0; U2 = 0; exact_needed = !ordinary_temperature;
  }
  template <typename T, int n>
  __device__ __forceinline__ void take_words(const uint32_t (&w)[n], float batch_max, float c) {
    if (!(batch_max <= limit)) {                        // well above the reference, or a NaN
      const float m_new = max_nan(m, batch_max);
      exact_needed = exact_needed || !(fabsf(m_new) <= kOrdinaryLogit);
      const float M_new = m_new * c;
      const float dt = M - M_new;
      const float sc = m == -CUDART_INF_F ? 0.f : exp2_fast(dt);
      const uint64_t sc2 = pair(sc, sc), zero = pair(0.f, 0.f);
      if (kWithU) U2 = fma_pair(fma_pair(pair(dt, dt), S2, U2), sc2, zero);
      S2 = fma_pair(S2, sc2, zero);
      m = m_new; M = M_new;
      limit = m_new + kLead / c;
    }
    if (m == -CUDART_INF_F) return;                     // nothing but -inf so far
    const uint64_t c2 = pair(c, c), minus_m = pair(-M, -M);
    uint64_t batch = 0;
#pragma unroll
    for (int i = 0; i < n; i += Elem<T>::kPairWords) {
      // without U no exponent is multiplied by its weight of 0, and -inf may stay
      const uint64_t t = fma_pair(kWithU ? Elem<T>::unpack_pair_floored(w + i) : Elem<T>::unpack_pair(w + i), c2, minus_m);
      float t0, t1;
      unpair(t, t0, t1);
      const uint64_t x = pair(exp2_fast(t0), exp2_fast(t1));
      batch = i == 0 ? x : add_pair(batch, x);
      if (kWithU) U2 = fma_pair(t, x, U2);
    }
    S2 = add_pair(S2, batch);
  }
  // the triple relative to m itself instead of the rounded M; of no account where exact_needed is set
  __device__ __forceinline__ RowStat done(float c) const {
    if (m == -CUDART_INF_F) return RowStat{m, 0.f, 0.f};
    float s0, s1, u0, u1;
    unpair(S2, s0, s1);
    unpair(U2, u0, u1);
    const float S = s0 + s1, U = u0 + u1;
    const float d = fmaf(m, c, -M), sc = exp2_fast(-d);
    return RowStat{m, S * sc, (U - d * S) * sc};
  }
  // The triple relative to the maximum itself, the largest of the batches'.  Its own term, the same instruction on the same number
  // as in the sum, is taken out and put back as the 1 that it is: S >= 1, and a near-certain token's ln S has no rounding of an
  // exponential in it.
  __device__ __forceinline__ RowStat done_at_maximum(float top, float c) const {
    if (m == -CUDART_INF_F) return RowStat{m, 0.f, 0.f};
    float s0, s1, u0, u1;
    unpair(S2, s0, s1);
    unpair(U2, u0, u1);
    const float S = s0 + s1, U = u0 + u1;
    const float d = fmaf(top, c, -M), sc = exp2_fast(-d);
    return RowStat{top, fmaf(fmaxf(S - exp2_fast(d), 0.f), sc, 1.f), fmaf(-d, S, U) * sc};
  }
};
using RunningStat = Running<true>;
using RunningSum = Running<false>;
// The exact form over the vectors first, first + stride, ... below n.
template <typename T>
__device__ __noinline__ RowStat exact_stat(const uint4* v, int first, int stride, int n, float c) {
  RowStat a{-CUDART_INF_F, 0.f, 0.f};
  for (int i = first; i < n; i += stride) {
    float f[Elem<T>::kVec];
    Elem<T>::unpack(v[i], f);
#pragma unroll
    for (int e = 0; e < Elem<T>::kVec; ++e) absorb_scalar(a, f[e], c);
  }
  return a;
}
// the temperature that is calculated with: its reciprocal has to be an fp32 number, times log2 e too
inline float usable_temperature(float t) { return t < 0x1p-127f ? 0x1p-127f : t; }
inline bool ordinary_temperature(float t) { return t >= 0.01f && t <= 100.f; }

// order-preserving map of a float to 32 bits; -0 and +0 are equal, a NaN (as max_nan makes them) comes above +inf
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
// a triple rescaled to a maximum that is not smaller; empty triples stay empty
__device__ __forceinline__ void rescale(RowStat& a, float m_new, float c) {
  if (m_new == a.m || m_new == -CUDART_INF_F) return;
  rebase(a, m_new, c);
}

// Where the elements of a row sit for one of the 2^log2_cta CTAs that share it: scalars up to the first 16-byte boundary
// (CTA 0), whole 16-byte vectors dealt out in contiguous runs, scalars after the last vector (last CTA).
struct RowSlice {
  int head;        // elements before the first vector of the row
  int v0, v1;      // this CTA's vectors
  int e0, e1;      // this CTA's elements, contiguous
  int own_head, own_tail, tail_start;
};
template <typename T>
__device__ __forceinline__ RowSlice row_slice(const T* z, int V, int cta, int log2_cta) {
  const int n_cta = 1 << log2_cta;
  RowSlice s;
  const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(z) & 15u);
  s.head = min((int)(((16u - off) & 15u) / sizeof(T)), V);
  const int n_vec = (V - s.head) / Elem<T>::kVec;
  const int per = (n_vec + n_cta - 1) >> log2_cta;
  s.v0 = min(cta * per, n_vec);
  s.v1 = min(s.v0 + per, n_vec);
  s.tail_start = s.head + n_vec * Elem<T>::kVec;
  s.own_head = cta == 0 ? s.head : 0;
  s.own_tail = cta == n_cta - 1 ? V - s.tail_start : 0;
  s.e0 = cta == 0 ? 0 : s.head + s.v0 * Elem<T>::kVec;
  s.e1 = cta == n_cta - 1 ? V : s.head + s.v1 * Elem<T>::kVec;
  return s;
}

// Launch in clusters of `cluster` CTAs, chained to the launch ahead like launch_chained.  A kernel that executes cluster
// instructions (asynchronous stores among them) needs this launch for clusters of one CTA too: started without the
// attribute such a kernel ended in an illegal instruction.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_clusters(bool chained, int cluster, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem,
                                   cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  attr[n].id = cudaLaunchAttributeClusterDimension;
  attr[n].val.clusterDim.x = cluster; attr[n].val.clusterDim.y = 1; attr[n].val.clusterDim.z = 1;
  ++n;
  if (chained) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

inline size_t elem_size(cwl_dtype t) { return t == CWL_F32 ? 4 : 2; }
inline bool known_dtype(cwl_dtype t) { return t == CWL_F32 || t == CWL_BF16 || t == CWL_F16; }

}  // namespace cwl

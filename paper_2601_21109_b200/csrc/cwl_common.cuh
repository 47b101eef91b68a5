// Shared host/device helpers of the CUDA library (never included by the CPU oracle).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "cwl.h"

#define CWL_CUDA_TRY(expr)                        \
  do {                                            \
    cudaError_t _e = (expr);                      \
    if (_e != cudaSuccess) return CWL_ERR_CUDA;   \
  } while (0)

namespace cwl {

constexpr int kQ24 = 1 << 24;

// Records a device-side problem without trapping: bit `code` of the caller's status word.
__device__ __forceinline__ void flag_status(int32_t* status_word, int code) {
  if (status_word != nullptr) atomicOr(status_word, 1 << code);
}

__host__ __device__ __forceinline__ int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A matrix in memory: `rows` of `width` bytes, `pitch` apart (at least their width, where there are several).
struct MatrixSpan { uintptr_t at; int64_t rows, width, pitch; };
inline MatrixSpan matrix_span(const void* at, int64_t ld, int64_t rows, int64_t cols, int elem) {
  return MatrixSpan{reinterpret_cast<uintptr_t>(at), rows, cols * elem, (rows > 1 ? ld : cols) * elem};
}
// Do two matrices have a byte in common?  Rows that lie between the other's rows (columns of one buffer) do not count.
inline bool overlap(const MatrixSpan& a, const MatrixSpan& b) {
  if (a.at == 0 || b.at == 0 || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
  if (a.at > b.at) return overlap(b, a);
  const int64_t off = (int64_t)(b.at - a.at);      // a begins first
  if (off >= (a.rows - 1) * a.pitch + a.width) return false;
  if (a.pitch == b.pitch) {
    const int64_t within = off % a.pitch;          // where b's rows lie in a's
    return within < a.width || within + b.width > a.pitch;
  }
  for (int64_t i = 0; i < b.rows; ++i) {           // the last of a's rows that begins before a row of b ends
    const int64_t begin = off + i * b.pitch, end = begin + b.width;
    const int64_t k = (end - 1) / a.pitch < a.rows - 1 ? (end - 1) / a.pitch : a.rows - 1;
    if (k * a.pitch + a.width > begin) return true;
  }
  return false;
}

// Programmatic dependent launch.  A kernel launched with launch_chained() may have its CTAs placed while the kernel
// before it in the stream is still running; it must call pdl_wait() before its first access to global memory, which
// returns once that kernel has completed and its writes are visible.  pdl_launch_dependents() lets the NEXT chained
// launch do the same with respect to this kernel.  Both do nothing in a kernel launched the ordinary way.
// A kernel may read before pdl_wait() what no kernel since a COMPLETED one has written: the first kernel of its call has to wait
// before it lets others begin, and every launch of the call up to the reader must leave that memory alone (head_few_kernel and W).
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// true while `stream` records into a CUDA graph (chained launches then keep the plain stream order)
inline bool stream_is_capturing(cudaStream_t stream) {
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(stream, &st) != cudaSuccess) { cudaGetLastError(); return true; }
  return st != cudaStreamCaptureStatusNone;
}

template <typename... KArgs, typename... Args>
inline cudaError_t launch_chained(bool chained, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem,
                                  cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = chained ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Lets a kernel without static shared memory take all that a block may have (227 KB), once per device.
class SharedMemoryGrant {
 public:
  template <typename Kernel>
  cudaError_t operator()(Kernel* kernel) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < kDevices && done_[dev].load(std::memory_order_acquire))) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e == cudaSuccess && dev < kDevices) done_[dev].store(true, std::memory_order_release);
    return e;
  }

 private:
  static constexpr int kDevices = 32;
  std::atomic<bool> done_[kDevices] = {};
};

}  // namespace cwl

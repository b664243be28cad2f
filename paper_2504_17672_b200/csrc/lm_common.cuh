// Shared by the operators of the local step (lm_*.cu): the handle, argument checks, element types.
#pragma once

#include "../../include/cocodc_lm.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

struct cocodc_lm {
  int device = 0;
  int sm_count = 0;
  int* d_status = nullptr;
  std::atomic<long long> launches{0};
};

namespace cocodc_lm_impl {

// The source files whose kernels need more shared memory than any kernel may have opt them in, at creation of a handle (the
// attribute is per device and outlives the handle).
bool embed_prepare();
bool glu_prepare();

struct DeviceScope {
  int prev = -1;
  bool switched = false, ok = true;
  explicit DeviceScope(int dev) {
    ok = cudaGetDevice(&prev) == cudaSuccess;
    if (ok && prev != dev) ok = switched = cudaSetDevice(dev) == cudaSuccess;
  }
  ~DeviceScope() { if (switched) cudaSetDevice(prev); }
};

// Launches with programmatic dependence on the stream's previous kernel: the next kernel's blocks may become resident once
// all blocks of this one have called may_follow(), and touch global memory only after wait_for_previous() (which
// returns when the previous kernel is done and its writes are visible), so that launch and set-up hide behind its end.
// What they read may thus have been written during their own lifetime: ordinary loads only, none through the read-only path (__ldg,
// ld.global.nc, const __restrict__ pointers), which is for data that no one writes while the kernel exists.
// The status is this launch's own, whatever the thread has left of older errors; what would read its results is not launched after a failure.
template <typename... P, typename... A>
inline cocodc_status start(cocodc_lm* lm, void (*kernel)(P...), dim3 grid, unsigned threads, unsigned smem, cudaStream_t st,
                           unsigned cluster, const A&... args) {
  cudaLaunchAttribute attrs[2] = {};
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = cluster;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = grid;
  config.blockDim = dim3(threads);
  config.dynamicSmemBytes = smem;
  config.stream = st;
  config.attrs = attrs;
  config.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&config, kernel, P(args)...) != cudaSuccess) {
    cudaGetLastError();                                // reported here, nobody else is to find it
    return COCODC_ERR_CUDA;
  }
  lm->launches.fetch_add(1, std::memory_order_relaxed);
  return COCODC_OK;
}

inline bool known_type(int32_t t) { return t == COCODC_F32 || t == COCODC_BF16 || t == COCODC_F16; }
inline int type_bytes(int32_t t) { return t == COCODC_F32 ? 4 : 2; }
inline int index_bytes(int32_t t) { return t == COCODC_I32 ? 4 : 8; }
inline bool on_boundary(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
// Rows that start on 16-byte boundaries: what vector loads and tensor maps need.
inline bool rows_aligned(const void* p, int64_t stride, int esize) {
  return on_boundary(p, 16) && (stride * esize) % 16 == 0;
}
// Sizes whose products with an element size stay far inside 64 bits.
inline bool sane(int64_t n) { return n >= 0 && n <= (int64_t(1) << 40); }

// The bytes [lo, hi) that a matrix spans, from its first element to its last; empty for no rows.
struct Span {
  uintptr_t lo, hi;
  uintptr_t pitch, width;    // bytes from row to row (0: one row) and of a row
};
inline Span span(const void* p, int64_t rows, int64_t stride, int64_t width, int esize) {
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  if (!p || rows < 1 || width < 1) return Span{b, b, 0, 0};
  const uintptr_t pitch = (uintptr_t)stride * (uintptr_t)esize, w = (uintptr_t)width * (uintptr_t)esize;
  return Span{b, b + (uintptr_t)(rows - 1) * pitch + w, rows > 1 ? pitch : 0, w};
}
// Whether two matrices have a byte in common.  Those with rows equally far apart (one row: as far as the other's) may be different
// columns of one buffer; where rows are not equally far apart, spans that meet count as matrices that do.
inline bool meet(const Span& a, const Span& b) {
  if (a.lo >= a.hi || b.lo >= b.hi || a.lo >= b.hi || b.lo >= a.hi) return false;
  const uintptr_t pitch = a.pitch ? a.pitch : b.pitch;
  if (pitch == 0 || (b.pitch && b.pitch != pitch) || a.width > pitch || b.width > pitch) return true;
  const uintptr_t d = b.lo >= a.lo ? (b.lo - a.lo) % pitch : (pitch - (a.lo - b.lo) % pitch) % pitch;   // b's first column from a's
  return d < a.width || d + b.width > pitch;
}

// ---- device side -------------------------------------------------------------------------------
// see start()
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void may_follow() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// All threads of the cluster have come here, and what they wrote to shared memory before is visible to all after.  (The lanes of a warp
// come to an .aligned instruction together, which after a branch only __syncwarp() promises.)
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 bytes by an ordinary load.  As volatile assembly it stays behind wait_for_previous(), and where it was written: plain C++
// loads took more registers in k_logprobs (4000 x 50257 bf16 with eight alternatives: 92 -> 96 us).
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }

// The token id at t as a row number: -1 for "no token", also for an id outside [0, V), which is recorded.
__device__ __forceinline__ long long token_at(const void* ids, int is64, long long t, long long V, int* status) {
  const long long v = is64 ? static_cast<const long long*>(ids)[t] : (long long)static_cast<const int*>(ids)[t];
  if (v < V) return v < 0 ? -1 : v;
  record(status, COCODC_ERR_INVALID_ARG);
  return -1;
}

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Calls f with a value of the C++ type that a type code stands for.
template <typename F> cocodc_status with_type(int32_t t, F&& f) {
  if (t == COCODC_F32) return f(float());
  if (t == COCODC_BF16) return f(__nv_bfloat16());
  return f(__half());
}

}  // namespace cocodc_lm_impl

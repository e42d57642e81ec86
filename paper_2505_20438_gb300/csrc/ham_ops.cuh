// What the operators after a macro-step's attention share (ham_norm.cu, ham_fp8.cu, ham_sample.cu):
// the 8-bit row format's device code, argument checks and the launch with programmatic dependence.
//
// 8-bit rows (ham.h, "8-bit rows and weights"): e4m3 codes, one E8M0 scale byte s for each block of
// 128 elements (value = code * 2^(s - 127)), a row's scale bytes padded to a multiple of four.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ham_internal.cuh"

namespace ham {

constexpr int kFp8Block = 128;
// Scale bytes of a row of k elements: one a block, padded to whole 32-bit words.
__host__ __device__ inline int fp8_scale_bytes(int k) {
  return ((k + 4 * kFp8Block - 1) / (4 * kFp8Block)) * 4;
}
// Exponent e of the scale 2^e of a block whose largest magnitude is `a` (not negative): E - 8 for
// a = m 2^E with 0.5 <= m < 1, within [-124, 119], so that the scaled block is below 256 (nothing
// saturates) and 2^e and 2^-e are normal numbers; 0 for a block of zeros.  E is read from the
// exponent field; numbers below the normal range (E <= -126) and infinities end at the clamp.
__device__ __forceinline__ int fp8_exponent(float a) {
  const int E = (int)((__float_as_uint(a) >> 23) & 0xffu) - 126;
  return a > 0.f ? min(max(E - 8, kFp8ExpMin), kFp8ExpMax) : 0;
}
__device__ __forceinline__ float fp8_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// Four fp32 values -> four e4m3 codes (value i in byte i), each times `p` (a power of two: exact),
// rounded to nearest even, saturating at +-448.
__device__ __forceinline__ uint32_t fp8_codes4(float a, float b, float c, float d, float p) {
  const __nv_fp8x2_storage_t lo =
      __nv_cvt_float2_to_fp8x2(make_float2(a * p, b * p), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t hi =
      __nv_cvt_float2_to_fp8x2(make_float2(c * p, d * p), __NV_SATFINITE, __NV_E4M3);
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// Set this thread's error message (printf style) and return `status`.
int op_fail(int status, const char *fmt, ...);
inline bool op_aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline bool op_overlap(const void *a, size_t na, const void *b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && na && nb && x < y + nb && y < x + na;
}
// SMs of the current device (cached per device).
int device_sms();
// Let `kernel` have `bytes` of dynamic shared memory, once a device.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, bool (&done)[64], int dev) {
  if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
  return e;
}

// TMA map of a row-major [rows][cols] matrix of bytes (cols a multiple of 16) with a box of
// {box_cols, box_rows}, with the 128-byte swizzle; boxes past the end read zeros.
// Returns a CUresult.
int make_bytes_tensor_map(CUtensorMap *map, const void *base, int64_t rows, int64_t cols,
                          int box_cols, int box_rows);

// TMA map of a stretch of `bytes` of memory (a multiple of 2048) as rows of 2048 bytes, with a box of
// box_bytes of them one after the other; boxes past the end read zeros.  Returns a CUresult.
int make_stretch_tensor_map(CUtensorMap *map, const void *base, int64_t bytes, int box_bytes);

// Launch kKernel so that it may be scheduled before the kernel before it on the stream has ended.
// Every kernel launched this way waits (griddepcontrol.wait) before it reads anything that an
// earlier kernel may have written and before it writes, and lets its own successor start only after
// that wait: at any time at most one kernel before it is still running.
//
// Small calls are bound by the host, so the launch goes to the driver's entry point (0.7 to 1.4 us of a
// call's 15 to 22 less than the runtime's); where that has no context yet, through the runtime.
using DriverLaunch = CUresult (*)(const CUlaunchConfig *, CUfunction, void **, void **);
DriverLaunch driver_launch();  // null if there is none

template <auto kKernel, typename... P>
cudaError_t launch_with(dim3 grid, dim3 block, size_t smem, dim3 cluster, cudaStream_t stream, void (*)(P...),
                        P... args) {
  void *values[] = {const_cast<void *>(static_cast<const void *>(&args))...};
  const bool clustered = cluster.x * cluster.y * cluster.z > 1;
  static CUfunction known[64] = {};              // by device; written with the same value by any thread
  int dev = 0;
  cudaGetDevice(&dev);
  const DriverLaunch launch = driver_launch();
  if (launch && dev >= 0 && dev < 64) {
    cudaFunction_t f = reinterpret_cast<cudaFunction_t>(known[dev]);
    if (!f && cudaGetFuncBySymbol(&f, reinterpret_cast<const void *>(kKernel)) != cudaSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    known[dev] = reinterpret_cast<CUfunction>(f);
    CUlaunchConfig cfg = {};
    cfg.gridDimX = grid.x, cfg.gridDimY = grid.y, cfg.gridDimZ = grid.z;
    cfg.blockDimX = block.x, cfg.blockDimY = block.y, cfg.blockDimZ = block.z;
    cfg.sharedMemBytes = (unsigned)smem;
    cfg.hStream = stream;
    CUlaunchAttribute attr[2];
    attr[0].id = CU_LAUNCH_ATTRIBUTE_PROGRAMMATIC_STREAM_SERIALIZATION;
    attr[0].value.programmaticStreamSerializationAllowed = 1;
    attr[1].id = CU_LAUNCH_ATTRIBUTE_CLUSTER_DIMENSION;
    attr[1].value.clusterDim.x = cluster.x;
    attr[1].value.clusterDim.y = cluster.y;
    attr[1].value.clusterDim.z = cluster.z;
    cfg.attrs = attr;
    cfg.numAttrs = clustered ? 2 : 1;
    if (f && launch(&cfg, known[dev], values, nullptr) == CUDA_SUCCESS) return cudaSuccess;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster.x;
  attr[1].val.clusterDim.y = cluster.y;
  attr[1].val.clusterDim.z = cluster.z;
  cfg.attrs = attr;
  cfg.numAttrs = clustered ? 2 : 1;
  return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(kKernel), values);
}
template <auto kKernel, typename... A>
cudaError_t launch_after(dim3 grid, dim3 block, size_t smem, dim3 cluster, cudaStream_t stream, A... args) {
  return launch_with<kKernel>(grid, block, smem, cluster, stream, kKernel, args...);
}

}  // namespace ham

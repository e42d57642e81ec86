// What the products with 8-bit weights share (ham_fp8.cu, ham_experts.cu): the handle, the weights' blocks, the pair
// kernels' launches.  (Each has its own parts of K, and its own order of the same role's code: a mend in one pair kernel's
// scale words, waits or end is to be looked for in the other's.)
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include "ham_mx.cuh"
#include "ham_ops.cuh"

// One weight: codes [tile][K block][part][128 x 128].  Some experts': blocks of 128 x 128 too, as ham_experts.cu says.
struct ham_fp8_weight {
  int32_t n = 0, k = 0, parts = 1;   // parts: 2 for a gated weight (gate, up)
  int32_t experts = 0;               // 0: one weight
  bool sorts = false;                // its calls may take memory of the device's pool for sorted rows
  int32_t tiles = 0, kbs = 0, sk = 0;
  int device = 0;
  uint8_t *codes = nullptr;    // 128 x 128 swizzled blocks, and behind them in the same allocation
  uint8_t *scales = nullptr;   // [(experts)][tiles][parts][sk]
  int32_t *err = nullptr;      // the device error word
  uint64_t wait_ns = ham::kWaitLimitNs;  // limit of the kernels' waits
  CUtensorMap map;             // codes as one stretch, boxes of half a block (experts: a block)
};

namespace ham {
// One weight that `sorts` less on a device: with the last one the pool's memory goes back.
void experts_weight_freed(int dev);

namespace {

constexpr int kTile = 128;             // weight rows of a tile
constexpr int kBlockBytes = 128 * 128; // a tile's K block

// Shared memory that a CTA with `cols` columns of tensor memory asks for at least, in kernels whose CTAs
// wait for one another: an SM's 228 KB then run out before its 512 columns do, so that no CTA of a
// cluster ever waits for columns that a CTA of another cluster holds (two clusters could otherwise each
// hold what the other waits for).
constexpr int smem_floor(int cols) { return (228 * 1024 * (cols / 32) + 16) / 17; }

// Registers a thread that the pair kernels are launched with.  From the roles on the first four warps' threads have fewer
// and the epilogue's eight more, which hold a tile's sums in 128 of them; together they are what the launch has: a kernel
// compiled to fewer would wait for the rest forever, so the host looks before it launches one.
constexpr int kPairThreads = 384;       // warps: copies, products, 2 x scales, 8 x epilogue
constexpr int kLaunchRegs = 168;

// Pairs that are resident at once (a pair lies within one group of SMs, which need not hold a whole number
// of them); a persistent grid is no larger.
template <typename K>
int resident_pairs(K kernel, int smem, int (&known)[64], int dev) {
  if (dev >= 0 && dev < 64 && known[dev] > 0) return known[dev];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(device_sms() / 2 * 2));
  cfg.blockDim = dim3(kPairThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = device_sms() / 2;
  }
  if (dev >= 0 && dev < 64) known[dev] = n;
  return n;
}

}  // namespace
}  // namespace ham

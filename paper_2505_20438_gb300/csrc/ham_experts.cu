// Products of 8-bit rows with the weights of their experts (ham.h, "A feed-forward block made of experts"): slots i of
// expert e, offsets[e] <= i < offsets[e + 1],
//
//   Y[i][n] = sum_k X[i][k] W_e[n][k]
//   H[i][f] = silu(G) U,  G = X[order[i] / top_k] Wg_e^T, U = X[order[i] / top_k] Wu_e^T,  encoded as 8-bit rows
//
// Weights are laid out once as [expert][half tile][K block][128 x 128], each block 16 KiB in the shared-memory layout
// of the 128-byte swizzle.  A half tile is 128 features of a plain weight; of a gated one 64 features, 16 rows of the
// gate and the same features' 16 rows of the up projection in turn, so that a warp's 32 lanes of tensor memory hold
// both numbers of 16 features.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <new>

#include "ham_fp8.cuh"

namespace ham {
namespace {

constexpr int kMostExperts = 512, kMostTop = 32;

// Row r of half tile h of a gated weight: the feature, and whether it is the up projection's row.
__host__ __device__ inline int gated_feature(int h, int r) { return h * 64 + (r / 32) * 16 + r % 16; }
__host__ __device__ inline bool gated_up(int r) { return r & 16; }

// One thread per 16-byte piece of the laid-out weights of one expert.
template <bool kGated>
__global__ void lay_out_experts_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ up, int n, int k,
                                       int kbs, int64_t pieces, uint8_t *__restrict__ dst) {
  const int64_t p = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (p >= pieces) return;
  const int in = (int)(p % (kBlockBytes / 16)), r = in / 8, c = in % 8;
  const int64_t block = p / (kBlockBytes / 16);  // half tile * kbs + K block
  const int half = (int)(block / kbs);
  const int64_t row = kGated ? gated_feature(half, r) : (int64_t)half * kTile + r;
  const uint8_t *from = kGated && gated_up(r) ? up : codes;
  const int col = (int)(block % kbs) * kFp8Block + 16 * c;
  uint4 v = make_uint4(0, 0, 0, 0);
  if (row < n && col < k) v = *reinterpret_cast<const uint4 *>(from + row * k + col);
  *reinterpret_cast<uint4 *>(dst + block * kBlockBytes + r * 128 + ((c ^ (r & 7)) << 4)) = v;
}
// [experts][tiles][sk] -> [experts][tiles][parts][sk]
__global__ void lay_out_expert_scales_kernel(const uint8_t *__restrict__ scales, int64_t rows, int sk, int part,
                                             int parts, uint8_t *__restrict__ dst) {
  const int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (i < rows * sk) dst[(i / sk * parts + part) * sk + i % sk] = scales[i];
}

struct ExpertArgs {
  const uint8_t *w, *ws;   // the handle's layout
  const uint8_t *x, *xs;   // rows
  const int32_t *offsets, *order;  // order: gated
  void *out;
  uint8_t *out_scales;     // gated
  int32_t *err;
  int experts, slots, top_k, n, k, kbs, sk, out_sk, tiles, halves, f32;
};

__device__ __forceinline__ float code_value(uint32_t byte) {
  uint32_t lo, hi;
  e4m3x4_to_f16x2(byte, lo, hi);
  return __half2float(__ushort_as_half((unsigned short)(lo & 0xffffu)));
}
__device__ __forceinline__ float scale_value(uint8_t s) {
  return s == 255 ? __uint_as_float(0x7fffffffu) : s ? __uint_as_float((uint32_t)s << 23) : 0x1p-127f;
}

// A thread a feature, a block 128 features of one slot.
template <bool kGated>
__global__ void __launch_bounds__(128) experts_kernel(ExpertArgs a) {
  __shared__ float x[kFp8Block];
  __shared__ float top[4];
  const int slot = blockIdx.x, tile = blockIdx.y, tid = threadIdx.x;
  grid_dependency_wait();
  grid_launch_dependents();
  int expert = -1;
  for (int e = 0; e < a.experts; ++e) {
    const int from = a.offsets[e], to = a.offsets[e + 1];
    if (from < 0 || to > a.slots || from > to) {
      if (tid == 0) record_error(a.err, HAM_DEVERR_ROUTE);
      return;
    }
    if (slot >= from && slot < to) expert = e;
  }
  if (expert < 0) return;
  int row = slot;
  if (kGated) {
    const int o = a.order[slot];
    if (o < 0 || o >= a.slots) {
      if (tid == 0) record_error(a.err, HAM_DEVERR_ROUTE);
      row = 0;
    } else {
      row = o / a.top_k;
    }
  }
  const int f = tile * kTile + tid;
  float sum[2] = {0.f, 0.f};
  for (int kb = 0; kb < a.kbs; ++kb) {
    __syncthreads();
    const int col = kb * kFp8Block + tid;
    x[tid] = col < a.k ? code_value(a.x[(int64_t)row * a.k + col]) : 0.f;
    __syncthreads();
    const float sx = scale_value(a.xs[(int64_t)row * a.sk + kb]);
#pragma unroll
    for (int p = 0; p < (kGated ? 2 : 1); ++p) {
      const int half = kGated ? tile * 2 + tid / 64 : tile, r = kGated ? (tid % 64) / 16 * 32 + p * 16 + tid % 16 : tid;
      const uint8_t *w = a.w + (((int64_t)expert * a.halves + half) * a.kbs + kb) * kBlockBytes + r * 128;
      float part = 0.f;
      for (int c = 0; c < 8; ++c) {
        const uint4 v = *reinterpret_cast<const uint4 *>(w + ((c ^ (r & 7)) << 4));
        const uint32_t word[4] = {v.x, v.y, v.z, v.w};
        for (int i = 0; i < 16; ++i) part = fmaf(x[16 * c + i], code_value(word[i / 4] >> 8 * (i % 4) & 0xffu), part);
      }
      const float sw = scale_value(a.ws[(((int64_t)expert * a.tiles + tile) * (kGated ? 2 : 1) + p) * a.sk + kb]);
      sum[p] += part * sx * sw;
    }
  }
  if constexpr (!kGated) {
    if (f >= a.n) return;
    const int64_t to = (int64_t)slot * a.n + f;
    if (a.f32) static_cast<float *>(a.out)[to] = sum[0];
    else static_cast<__nv_bfloat16 *>(a.out)[to] = __float2bfloat16_rn(sum[0]);
  } else {
    const float h = silu_mul(sum[0], sum[1]);
    const float m = warp_max_f32(fabsf(h));
    if ((tid & 31) == 0) top[tid >> 5] = m;
    __syncthreads();
    const int e = fp8_exponent(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
    if (f < a.n) static_cast<uint8_t *>(a.out)[(int64_t)slot * a.n + f] = (uint8_t)fp8_codes4(h, 0, 0, 0, fp8_pow2(-e));
    uint8_t *s = a.out_scales + (int64_t)slot * a.out_sk;
    if (tid == 0) s[tile] = (uint8_t)(e + 127);
    if (tile == a.tiles - 1 && tid > 0 && tile + tid < a.out_sk) s[tile + tid] = 127;
  }
}

int check_experts(const ham_fp8_weight *w, const void *xc, const void *xs, int64_t slots, const void *offsets,
                  const void *out) {
  if (slots == 0) return HAM_OK;
  if (!xc || !xs || !offsets || !out) return op_fail(HAM_EINVAL, "codes, scales, offsets and the output are required");
  if (!op_aligned(xc, 16) || !op_aligned(out, 16)) return op_fail(HAM_EINVAL, "codes and the output must be 16-byte aligned");
  if (!op_aligned(xs, 4) || !op_aligned(offsets, 4)) return op_fail(HAM_EINVAL, "scales and offsets must be 4-byte aligned");
  return HAM_OK;
}

int run_experts(ham_fp8_weight *w, ExpertArgs a, void *stream) {
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev != w->device) cudaSetDevice(w->device);
  a.w = w->codes;
  a.ws = w->scales;
  a.err = w->err;
  a.experts = w->experts;
  a.n = w->n;
  a.k = w->k;
  a.kbs = w->kbs;
  a.sk = w->sk;
  a.out_sk = fp8_scale_bytes(w->n);
  a.tiles = w->tiles;
  a.halves = w->tiles * w->parts;
  const dim3 grid((unsigned)a.slots, (unsigned)a.tiles);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = w->parts == 2 ? launch_after<experts_kernel<true>>(grid, dim3(128), 0, dim3(1), s, a)
                                      : launch_after<experts_kernel<false>>(grid, dim3(128), 0, dim3(1), s, a);
  const int rc = e == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "experts launch: %s", cudaGetErrorString(e));
  if (dev != w->device) cudaSetDevice(dev);
  return rc;
}

}  // namespace
}  // namespace ham

using ham::op_aligned;
using ham::op_fail;
using ham::op_overlap;

extern "C" {

int ham_fp8_experts_alloc(int32_t experts, int32_t n, int32_t k, const void *codes, const void *scales,
                          const void *codes_up, const void *scales_up, ham_fp8_weight **out) {
  if (!out) return op_fail(HAM_EINVAL, "out is required");
  *out = nullptr;
  if (experts < 1 || experts > ham::kMostExperts)
    return op_fail(HAM_EINVAL, "experts %d outside 1..%d", experts, ham::kMostExperts);
  if (n < 1 || n > (1 << 22)) return op_fail(HAM_EINVAL, "n %d outside 1..2^22", n);
  if (k < 16 || k % 16 != 0 || k > (1 << 20)) return op_fail(HAM_EINVAL, "k %d must be a multiple of 16 in 16..2^20", k);
  if (!codes || !scales) return op_fail(HAM_EINVAL, "codes and scales are required");
  if (!codes_up != !scales_up) return op_fail(HAM_EINVAL, "codes_up and scales_up come together");
  if (codes_up && n % 16 != 0) return op_fail(HAM_EINVAL, "n %d of a gated weight must be a multiple of 16", n);
  for (const void *p : {codes, codes_up})
    if (!op_aligned(p, 16)) return op_fail(HAM_EINVAL, "codes must be 16-byte aligned");
  ham_fp8_weight *w = new (std::nothrow) ham_fp8_weight();
  if (!w) return op_fail(HAM_ENOMEM, "host allocation failed");
  w->experts = experts;
  w->n = n;
  w->k = k;
  w->parts = codes_up ? 2 : 1;
  w->tiles = (n + ham::kTile - 1) / ham::kTile;
  w->kbs = (k + ham::kFp8Block - 1) / ham::kFp8Block;
  w->sk = ham::fp8_scale_bytes(k);
  cudaGetDevice(&w->device);
  const int64_t blocks = (int64_t)w->tiles * w->kbs * w->parts;  // of one expert
  if (blocks > ((int64_t)1 << 42) / ham::kBlockBytes / experts) {
    delete w;
    return op_fail(HAM_EUNSUPPORTED, "weights of %d x %d x %d are too large", experts, n, k);
  }
  const int64_t scale_rows = (int64_t)experts * w->tiles;
  const size_t code_bytes = (size_t)blocks * experts * ham::kBlockBytes, scale_bytes = (size_t)scale_rows * w->parts * w->sk;
  cudaError_t e = cudaMalloc(reinterpret_cast<void **>(&w->codes), code_bytes + scale_bytes + 4);
  if (e != cudaSuccess) {
    cudaGetLastError();
    ham_fp8_weight_free(w);
    return op_fail(HAM_ENOMEM, "weights of %d x %d x %d: %s", experts, n, k, cudaGetErrorString(e));
  }
  w->scales = w->codes + code_bytes;             // (whole words)
  w->err = reinterpret_cast<int32_t *>(w->scales + scale_bytes);
  const int64_t pieces = blocks * (ham::kBlockBytes / 16);
  const unsigned grid = (unsigned)((pieces + 255) / 256);
  for (int64_t i = 0; i < experts && e == cudaSuccess; ++i) {
    const uint8_t *from = static_cast<const uint8_t *>(codes) + i * n * k;
    uint8_t *to = w->codes + i * blocks * ham::kBlockBytes;
    if (codes_up)
      ham::lay_out_experts_kernel<true><<<grid, 256>>>(from, static_cast<const uint8_t *>(codes_up) + i * n * k, n, k,
                                                       w->kbs, pieces, to);
    else
      ham::lay_out_experts_kernel<false><<<grid, 256>>>(from, nullptr, n, k, w->kbs, pieces, to);
    e = cudaGetLastError();
  }
  for (int p = 0; p < w->parts && e == cudaSuccess; ++p) {
    ham::lay_out_expert_scales_kernel<<<(unsigned)((scale_rows * w->sk + 255) / 256), 256>>>(
        static_cast<const uint8_t *>(p ? scales_up : scales), scale_rows, w->sk, p, w->parts, w->scales);
    e = cudaGetLastError();
  }
  if (e == cudaSuccess) e = cudaMemset(w->err, 0, 4);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess || ham::make_stretch_tensor_map(&w->map, w->codes, (int64_t)code_bytes, ham::kBlockBytes) != 0) {
    cudaGetLastError();
    ham_fp8_weight_free(w);
    return op_fail(HAM_ECUDA, "weight layout: %s", cudaGetErrorString(e));
  }
  *out = w;
  return HAM_OK;
}

int ham_fp8_experts_gated(ham_fp8_weight *w, const void *x_codes, const void *x_scales, int32_t rows,
                          const int32_t *offsets, const int32_t *order, int32_t top_k, void *codes, void *scales,
                          void *stream) {
  ham::ApiRange nvtx_range("ham_fp8_experts_gated");
  if (!w) return op_fail(HAM_EINVAL, "null handle");
  if (!w->experts || w->parts != 2) return op_fail(HAM_EINVAL, "ham_fp8_experts_gated takes experts' gated weights");
  if (rows < 0 || rows > (1 << 24)) return op_fail(HAM_EINVAL, "rows %d outside 0..2^24", rows);
  if (top_k < 1 || top_k > ham::kMostTop) return op_fail(HAM_EINVAL, "top_k %d outside 1..%d", top_k, ham::kMostTop);
  const int64_t slots = (int64_t)rows * top_k;
  if (slots > (1 << 26)) return op_fail(HAM_EINVAL, "rows * top_k %lld above 2^26", (long long)slots);
  const int rc = ham::check_experts(w, x_codes, x_scales, slots, offsets, codes);
  if (rc || slots == 0) return rc;
  if (!order || !op_aligned(order, 4)) return op_fail(HAM_EINVAL, "order is required, 4-byte aligned");
  if (!scales || !op_aligned(scales, 4)) return op_fail(HAM_EINVAL, "the output's scales are required, 4-byte aligned");
  struct Span { const void *p; size_t n; };
  const Span outs[2] = {{codes, (size_t)slots * w->n}, {scales, (size_t)slots * ham::fp8_scale_bytes(w->n)}};
  const Span ins[4] = {{x_codes, (size_t)rows * w->k}, {x_scales, (size_t)rows * w->sk},
                       {offsets, 4 * ((size_t)w->experts + 1)}, {order, 4 * (size_t)slots}};
  for (const Span &o : outs)
    for (const Span &i : ins)
      if (op_overlap(o.p, o.n, i.p, i.n)) return op_fail(HAM_EINVAL, "an output overlaps an input");
  if (op_overlap(outs[0].p, outs[0].n, outs[1].p, outs[1].n)) return op_fail(HAM_EINVAL, "two outputs overlap");
  ham::ExpertArgs a{};
  a.x = static_cast<const uint8_t *>(x_codes);
  a.xs = static_cast<const uint8_t *>(x_scales);
  a.offsets = offsets;
  a.order = order;
  a.top_k = top_k;
  a.slots = (int)slots;
  a.out = codes;
  a.out_scales = static_cast<uint8_t *>(scales);
  return ham::run_experts(w, a, stream);
}

int ham_fp8_experts_linear(ham_fp8_weight *w, const void *x_codes, const void *x_scales, int32_t slots,
                           const int32_t *offsets, void *out, int32_t out_dtype, void *stream) {
  ham::ApiRange nvtx_range("ham_fp8_experts_linear");
  if (!w) return op_fail(HAM_EINVAL, "null handle");
  if (!w->experts || w->parts != 1) return op_fail(HAM_EINVAL, "ham_fp8_experts_linear takes experts' plain weights");
  if (out_dtype != HAM_DTYPE_BF16 && out_dtype != HAM_DTYPE_F32) return op_fail(HAM_EINVAL, "out_dtype %d", out_dtype);
  if (slots < 0 || slots > (1 << 26)) return op_fail(HAM_EINVAL, "slots %d outside 0..2^26", slots);
  const int rc = ham::check_experts(w, x_codes, x_scales, slots, offsets, out);
  if (rc || slots == 0) return rc;
  const int f32 = out_dtype == HAM_DTYPE_F32;
  const size_t ob = (size_t)slots * w->n * (f32 ? 4 : 2);
  if (op_overlap(out, ob, x_codes, (size_t)slots * w->k) || op_overlap(out, ob, x_scales, (size_t)slots * w->sk) ||
      op_overlap(out, ob, offsets, 4 * ((size_t)w->experts + 1)))
    return op_fail(HAM_EINVAL, "out overlaps an input");
  ham::ExpertArgs a{};
  a.x = static_cast<const uint8_t *>(x_codes);
  a.xs = static_cast<const uint8_t *>(x_scales);
  a.offsets = offsets;
  a.top_k = 1;
  a.slots = slots;
  a.out = out;
  a.f32 = f32;
  return ham::run_experts(w, a, stream);
}

}  // extern "C"

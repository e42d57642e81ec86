// Residual addition with root-mean-square norm (bf16 or 8-bit output), and the encoder of bf16 rows.
//
//   h = x + r,  y = h / sqrt(mean(h^2) + eps) * w        (fp32; sums over the row in fp32)
//   sum = bf16(h),  out = bf16(y),  (codes, scales) = 8-bit rows of y
//
// The norm takes the fp32 sum h, not the bf16 one that goes on as the residual: each output is the
// formula's value rounded once.  One pass over memory: a block holds its row in registers, 8
// consecutive elements a thread and group, so that a 128-element scale block is 16 neighbouring
// lanes and its largest magnitude four shuffles away.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>

#include "ham_ops.cuh"
#include "ham_ptx.cuh"

namespace ham {

int op_fail(int status, const char *fmt, ...) {
  char buf[400];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return set_last_error(status, buf);
}

namespace {

constexpr int kNormMaxHidden = 32768;

struct NormArgs {
  const uint4 *x, *r;      // [rows][hidden / 8]; r nullable
  const uint4 *w;          // [hidden / 8]
  uint4 *sum, *out;        // nullable
  uint2 *codes;            // nullable [rows][hidden / 8]
  uint8_t *scales;         // with codes: [rows][sk]
  int hidden, vecs, blocks, sk;   // vecs = hidden / 8, blocks = ceil(hidden / 128)
  float eps;
  int far;                 // the outputs pass L2: nothing is gained by keeping them there
};
template <typename V>
__device__ __forceinline__ void put(V *p, const V &v, int far) {
  if (far) __stcs(p, v);
  else *p = v;
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8]) {
  f[0] = bf_lo(v.x), f[1] = bf_hi(v.x), f[2] = bf_lo(v.y), f[3] = bf_hi(v.y);
  f[4] = bf_lo(v.z), f[5] = bf_hi(v.z), f[6] = bf_lo(v.w), f[7] = bf_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                    pack_bf16x2(f[6], f[7]));
}
// The 8-bit form of the 16 lanes' block of 128 values (lanes past the row hold zeros); the block's
// first lane gets the scale byte to write.
__device__ __forceinline__ uint2 encode8(const float (&y)[8], uint32_t &scale) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(y[i]));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(kFull, a, o));
  const int e = fp8_exponent(a);
  const float p = fp8_pow2(-e);
  scale = (uint32_t)(e + 127);
  return make_uint2(fp8_codes4(y[0], y[1], y[2], y[3], p), fp8_codes4(y[4], y[5], y[6], y[7], p));
}

// A number's sum over the block; `part`: its warps' sums.
__device__ __forceinline__ float block_sum(float s, float *part) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  if ((tid & 31) == 0) part[tid >> 5] = s;
  __syncthreads();
  s = (tid & 31) < (blockDim.x >> 5) ? part[tid & 31] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  return s;
}

// A block is one row, a thread the groups tid, tid + threads, ... of 8 elements.  Many rows are bound by
// memory (16384 rows of 4096, residual in, sum and 8-bit rows out: 68.1 us, 6.9 TB/s counted at the bytes
// of the operands), few by the chain of launch, reads and the row's sum (8 rows: 1.65 us).
template <int kGroups>
__global__ void __launch_bounds__(kGroups >= 4 ? 1024 : 512) add_norm_kernel(NormArgs a) {
  __shared__ float part[32];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int64_t row = blockIdx.x;
  const int64_t at = row * a.vecs;
  grid_dependency_wait();
  grid_launch_dependents();
  float h[kGroups][8];
  uint4 vx[kGroups], vr[kGroups];
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    const int v = tid + g * threads;
    vx[g] = vr[g] = make_uint4(0, 0, 0, 0);
    if (v < a.vecs) {
      vx[g] = __ldcs(a.x + at + v);
      if (a.r) vr[g] = __ldcs(a.r + at + v);
    }
  }
  float s = 0.f;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    float r[8];
    unpack8(vx[g], h[g]);
    unpack8(vr[g], r);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[g][i] += r[i];
      s = fmaf(h[g][i], h[g][i], s);
    }
  }
  if (a.sum) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int v = tid + g * threads;
      if (v < a.vecs) put(a.sum + at + v, pack8(h[g]), a.far);
    }
  }
  uint4 vw[kGroups];
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    const int v = tid + g * threads;
    vw[g] = v < a.vecs ? __ldg(a.w + v) : make_uint4(0, 0, 0, 0);
  }
  float mean = block_sum(s, part) / (float)a.hidden + a.eps;
  // Where the squares leave fp32's range (elements from some 1e18 on; a row below 1e-15 with next to no eps) they
  // are summed again, and the row normed, in another unit, a power of two.
  if (__builtin_expect(!(mean >= 0x1p-100f && mean <= 0x1p126f), 0)) {
    const float unit = mean < 1.f ? 0x1p80f : 0x1p-80f;
    s = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[g][i] *= unit;
        s = fmaf(h[g][i], h[g][i], s);
      }
    __syncthreads();                             // (the sums are read)
    mean = block_sum(s, part) / (float)a.hidden + a.eps * unit * unit;
  }
  const float inv = rsqrtf(mean);
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    const int v = tid + g * threads;
    float w[8], y[8];
    unpack8(vw[g], w);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = h[g][i] * inv * w[i];
    if (a.out && v < a.vecs) put(a.out + at + v, pack8(y), a.far);
    if (a.codes) {  // (whole warps take part in the shuffles)
      uint32_t scale;
      const uint2 c = encode8(y, scale);
      if (v < a.vecs) {
        put(a.codes + at + v, c, a.far);
        if ((tid & 15) == 0) a.scales[row * a.sk + (v >> 4)] = (uint8_t)scale;
      }
    }
  }
  if (a.codes && tid < a.sk - a.blocks) a.scales[row * a.sk + a.blocks + tid] = 127;  // padding
}

// bf16 rows -> 8-bit rows: 16 threads a block of 128 elements, kEncodeEach such blocks a thread, read
// together; the places of a row's padding get scale 1 and no codes.  Bound by memory (16384 rows of 4096:
// 30.9 us, 96% of the copy rate; with one block a thread 36, and 40 with all rows' blocks numbered through,
// which takes a 64-bit division a thread; with four 31).
constexpr int kEncodeEach = 2;
__global__ void __launch_bounds__(256) encode_kernel(const uint4 *__restrict__ x, uint2 *codes,
                                                     uint8_t *scales, int vecs, int sk) {
  const int threads = blockDim.x, first = blockIdx.y * kEncodeEach * threads + threadIdx.x;
  const int64_t row = blockIdx.x;
  grid_dependency_wait();
  grid_launch_dependents();
  uint4 in[kEncodeEach];
#pragma unroll
  for (int j = 0; j < kEncodeEach; ++j) {
    const int v = first + j * threads;
    in[j] = v < vecs ? __ldcs(x + row * vecs + v) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < kEncodeEach; ++j) {
    const int v = first + j * threads;
    float y[8];
    unpack8(in[j], y);
    uint32_t scale;
    const uint2 c = encode8(y, scale);
    if (v < vecs) codes[row * vecs + v] = c;
    if ((v >> 4) < sk && (v & 15) == 0) scales[row * sk + (v >> 4)] = (uint8_t)scale;
  }
}

// bf16 weight [n][k] -> codes and one scale for each 128 x 128 block: a block of threads a weight
// block (two reads of it, the second from L1 / L2).  Done once for a weight; 16384 x 4096 takes 41 us,
// 73% of the copy rate.
__global__ void __launch_bounds__(256) encode_weight_kernel(const uint4 *__restrict__ w, uint2 *codes,
                                                            uint8_t *scales, int n, int vecs, int sk) {
  __shared__ float part[8];
  const int tid = threadIdx.x, v = blockIdx.x * 16 + (tid & 15);
  const int64_t row0 = (int64_t)blockIdx.y * kFp8Block;
  grid_dependency_wait();
  grid_launch_dependents();
  float a = 0.f;
  for (int r = tid >> 4; r < kFp8Block; r += 16)
    if (row0 + r < n && v < vecs) {
      float y[8];
      unpack8(w[(row0 + r) * vecs + v], y);
#pragma unroll
      for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(y[i]));
    }
  a = warp_max_f32(a);
  if ((tid & 31) == 0) part[tid >> 5] = a;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) a = fmaxf(a, part[i]);
  const int e = fp8_exponent(a);
  const float p = fp8_pow2(-e);
  for (int r = tid >> 4; r < kFp8Block; r += 16)
    if (row0 + r < n && v < vecs) {
      float y[8];
      unpack8(w[(row0 + r) * vecs + v], y);
      codes[(row0 + r) * vecs + v] = make_uint2(fp8_codes4(y[0], y[1], y[2], y[3], p),
                                                fp8_codes4(y[4], y[5], y[6], y[7], p));
    }
  if (tid == 0) scales[(int64_t)blockIdx.y * sk + blockIdx.x] = (uint8_t)(e + 127);
}

int check_rows(const char *what, int32_t rows, int32_t width, int32_t most) {
  if (rows < 0) return op_fail(HAM_EINVAL, "rows %d is negative", rows);
  if (width < 16 || width % 16 != 0 || width > most)
    return op_fail(HAM_EINVAL, "%s %d must be a multiple of 16 in 16..%d", what, width, most);
  return HAM_OK;
}

}  // namespace
}  // namespace ham

using ham::op_aligned;
using ham::op_fail;
using ham::op_overlap;

extern "C" {

int ham_add_norm(const void *x, const void *residual, const void *weight, float eps, int32_t rows,
                 int32_t hidden, void *sum_out, void *out, void *codes, void *scales, void *stream) {
  ham::ApiRange nvtx_range("ham_add_norm");
  int rc = ham::check_rows("hidden", rows, hidden, ham::kNormMaxHidden);
  if (rc) return rc;
  if (!(eps >= 0.f)) return op_fail(HAM_EINVAL, "eps must not be negative");
  if (rows == 0) return HAM_OK;
  if (!codes != !scales) return op_fail(HAM_EINVAL, "codes and scales come together");
  if (!out && !codes) return op_fail(HAM_EINVAL, "out, or codes and scales, are required");
  if (!x || !weight) return op_fail(HAM_EINVAL, "x and weight are required");
  for (const void *p : {x, residual, weight, (const void *)sum_out, (const void *)out, (const void *)codes})
    if (!op_aligned(p, 16)) return op_fail(HAM_EINVAL, "x, residual, weight, sum_out, out and codes must be 16-byte aligned");
  if (!op_aligned(scales, 4)) return op_fail(HAM_EINVAL, "scales must be 4-byte aligned");
  const size_t e = (size_t)rows * hidden, sb = (size_t)rows * ham::fp8_scale_bytes(hidden);
  struct Span { const void *p; size_t n; };
  const Span outs[4] = {{sum_out, 2 * e}, {out, 2 * e}, {codes, e}, {scales, sb}};
  for (int i = 0; i < 4; ++i) {
    // (a 16-bit output may be x or residual itself: a row is read whole before it is written)
    for (const void *in : {x, residual})
      if (op_overlap(outs[i].p, outs[i].n, in, 2 * e) && !(i < 2 && outs[i].p == in))
        return op_fail(HAM_EINVAL, "an output overlaps x or residual");
    if (op_overlap(outs[i].p, outs[i].n, weight, 2 * (size_t)hidden))
      return op_fail(HAM_EINVAL, "an output overlaps weight");
    for (int j = 0; j < i; ++j)
      if (op_overlap(outs[i].p, outs[i].n, outs[j].p, outs[j].n))
        return op_fail(HAM_EINVAL, "two outputs overlap");
  }
  ham::NormArgs a;
  a.x = static_cast<const uint4 *>(x);
  a.r = static_cast<const uint4 *>(residual);
  a.w = static_cast<const uint4 *>(weight);
  a.sum = static_cast<uint4 *>(sum_out);
  a.out = static_cast<uint4 *>(out);
  a.codes = static_cast<uint2 *>(codes);
  a.scales = static_cast<uint8_t *>(scales);
  a.hidden = hidden;
  a.vecs = hidden / 8;
  a.blocks = (hidden + ham::kFp8Block - 1) / ham::kFp8Block;
  a.sk = ham::fp8_scale_bytes(hidden);
  a.eps = eps;
  a.far = 2 * e * (!!sum_out + !!out) + e * !!codes > ((size_t)64 << 20);
  // Few rows: short chains a thread.  Many: more of a row a thread, so that more rows are in flight an SM.  (At most
  // 256 / 512 threads a row, us, inputs from memory: 16384 rows of 4096 73 / 79 with residual and 8-bit output, 49 / 60 of
  // x alone to bf16; of 3008 38 / 46, of 5136 65 / 69, of 8192 89 / 101; 1333 rows of 4096 6.1 / 7.2, of 5136 7.6 / 8.2 (with
  // residual 11.0 / 10.5); 608 of 4096 3.8 / 3.5, of 5136 4.3 / 3.9, of 8192 5.2 / 6.2; 400 of 5136 3.8 / 3.5, with residual
  // 5.7 / 5.0; from 12288 on both are the same kernel.)
  const int most = rows >= 4 * ham::device_sms() ? 256 : 512;
  int groups = 1;
  while (groups < 4 && a.vecs > groups * most) groups *= 2;
  const int threads = ((a.vecs + groups - 1) / groups + 31) / 32 * 32;
  const dim3 grid((unsigned)rows), block((unsigned)threads);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t ce = groups == 1   ? ham::launch_after<ham::add_norm_kernel<1>>(grid, block, 0, dim3(1), s, a)
                         : groups == 2 ? ham::launch_after<ham::add_norm_kernel<2>>(grid, block, 0, dim3(1), s, a)
                                       : ham::launch_after<ham::add_norm_kernel<4>>(grid, block, 0, dim3(1), s, a);
  return ce == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "norm launch: %s", cudaGetErrorString(ce));
}

int ham_fp8_encode(const void *x, int32_t rows, int32_t k, void *codes, void *scales, void *stream) {
  ham::ApiRange nvtx_range("ham_fp8_encode");
  int rc = ham::check_rows("k", rows, k, 1 << 20);
  if (rc) return rc;
  if (rows == 0) return HAM_OK;
  if (!x || !codes || !scales) return op_fail(HAM_EINVAL, "x, codes and scales are required");
  if (!op_aligned(x, 16) || !op_aligned(codes, 16) || !op_aligned(scales, 4))
    return op_fail(HAM_EINVAL, "x and codes must be 16-byte aligned, scales 4-byte aligned");
  const size_t e = (size_t)rows * k;
  const int sk = ham::fp8_scale_bytes(k);
  const size_t sb = (size_t)rows * sk;
  if (op_overlap(x, 2 * e, codes, e) || op_overlap(x, 2 * e, scales, sb) || op_overlap(codes, e, scales, sb))
    return op_fail(HAM_EINVAL, "x, codes and scales must not overlap");
  // a row in as few blocks of threads as hold it, of equal shares
  const int share = sk * 16 / ham::kEncodeEach, parts = (share + 255) / 256;
  const int threads = ((share + parts - 1) / parts + 31) / 32 * 32;
  const cudaError_t ce = ham::launch_after<ham::encode_kernel>(
      dim3((unsigned)rows, (unsigned)parts), dim3((unsigned)threads), 0, dim3(1),
      static_cast<cudaStream_t>(stream), static_cast<const uint4 *>(x), static_cast<uint2 *>(codes),
      static_cast<uint8_t *>(scales), k / 8, sk);
  return ce == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "encode launch: %s", cudaGetErrorString(ce));
}

int ham_fp8_encode_weight(const void *w, int32_t n, int32_t k, void *codes, void *scales, void *stream) {
  ham::ApiRange nvtx_range("ham_fp8_encode_weight");
  int rc = ham::check_rows("k", n, k, 1 << 20);
  if (rc) return rc;
  if (n < 1 || n > 65535 * ham::kFp8Block) return op_fail(HAM_EINVAL, "n %d outside 1..%d", n, 65535 * ham::kFp8Block);
  if (!w || !codes || !scales) return op_fail(HAM_EINVAL, "w, codes and scales are required");
  if (!op_aligned(w, 16) || !op_aligned(codes, 16) || !op_aligned(scales, 4))
    return op_fail(HAM_EINVAL, "w and codes must be 16-byte aligned, scales 4-byte aligned");
  const size_t e = (size_t)n * k;
  const int sk = ham::fp8_scale_bytes(k), nb = (n + ham::kFp8Block - 1) / ham::kFp8Block;
  const size_t sb = (size_t)nb * sk;
  if (op_overlap(w, 2 * e, codes, e) || op_overlap(w, 2 * e, scales, sb) || op_overlap(codes, e, scales, sb))
    return op_fail(HAM_EINVAL, "w, codes and scales must not overlap");
  // one block a scale byte, the padding's too (no elements there: scale 1)
  const cudaError_t ce = ham::launch_after<ham::encode_weight_kernel>(
      dim3((unsigned)sk, (unsigned)nb), dim3(256), 0, dim3(1),
      static_cast<cudaStream_t>(stream), static_cast<const uint4 *>(w), static_cast<uint2 *>(codes),
      static_cast<uint8_t *>(scales), n, k / 8, sk);
  return ce == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "encode launch: %s", cudaGetErrorString(ce));
}

}  // extern "C"

// The two ends of a feed-forward block made of experts: which experts a row takes, with the grouping of the chosen
// (row, expert) pairs by expert, and the weighted sum of a row's results.
//
//   s = softmax(l) or 1 / (1 + exp(-max(l, -80))),  v = s + bias
//   groups of experts by the sum of their two largest v, the best stay; of those the top_k largest v
//   weight = scale s (/ sum of the chosen s);  slots: the pairs in order of (expert, row, place)
//   out[t] = add[t] + sum_j weight[t][j] y[place[t][j]]
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cfloat>

#include "ham_ops.cuh"
#include "ham_ptx.cuh"

namespace ham {
namespace {

constexpr int kMostExperts = 512, kMostTop = 32;
constexpr int kChooseWarps = 8;          // rows of a block

struct RouteArgs {
  const void *logits;      // [rows][experts] bf16 or f32
  const float *bias;       // nullable
  int f32, rows, experts, top_k, sigmoid, groups, top_groups, renorm;
  float scale;
  int32_t *expert;         // [rows][top_k]
  float *weight;
  int32_t *offsets, *order, *place;
};

// A logit as the formulas take it: -inf rules out (NaN too).
__device__ __forceinline__ float read_logit(const RouteArgs &a, int64_t at) {
  float l = a.f32 ? static_cast<const float *>(a.logits)[at]
                  : __bfloat162float(static_cast<const __nv_bfloat16 *>(a.logits)[at]);
  if (!(l > -INFINITY)) return -INFINITY;
  l = fminf(l, FLT_MAX);
  return a.sigmoid ? fmaxf(l, -80.f) : l;
}
__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }
// exp(l - top), l <= top, the difference's rounding (which a large one would carry over) put right.
__device__ __forceinline__ float exp_difference(float l, float top) {
  const float x = l - top, part = x - l;
  const float off = (l - (x - part)) - (top + part);   // (a difference's error, exactly: the two-sum)
  const float e = expf(x);
  return e > 0.f ? fmaf(e, off, e) : 0.f;
}
// A number's place in the order of floats, as an unsigned one; 0: ruled out.
__device__ __forceinline__ uint32_t rank_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);   // (-0 -> +0)
  return x > -INFINITY ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float value_of(uint32_t r) {
  return __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r);
}
template <typename T>
__device__ __forceinline__ T warp_sum(T x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kFull, x, o);
  return x;
}
// The largest x over the warp and the lowest index that has it (-1: every x is -inf).
__device__ __forceinline__ int warp_best(float x, int index, float &best) {
  const uint32_t r = rank_of(x), top = __reduce_max_sync(kFull, r);
  best = top ? value_of(top) : -INFINITY;
  const int at = __reduce_min_sync(kFull, r == top ? index : INT32_MAX);
  return top ? at : -1;
}
__device__ __forceinline__ int warp_best(double x, int index, double &best) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const double y = __shfl_xor_sync(kFull, x, o);
    const int j = __shfl_xor_sync(kFull, index, o);
    if (y > x || (y == x && j < index)) x = y, index = j;
  }
  best = x;
  return x > -INFINITY ? index : -1;
}

// One row's experts by a warp, lane j < top_k getting the j-th (-1: none).  Values in T; in fp32 `unsure` says that
// two values that a decision lies between are nearer than their errors: the caller then computes the row in fp64.
//
// fp32 errors, relative to the row's largest score: of a sigmoid two units of expf, a sum and a quotient, below 2^-21;
// of a softmax the rounding of l - max (|x| exp(x) <= 0.37 units), expf, 21 additions and a product, below 2^-19.
// A value adds half a unit of itself.  Equal logits with equal biases are equal exactly, however they are computed.
template <typename T, int kPer>
__device__ __forceinline__ int choose_row(const RouteArgs &a, int row, const int (&group)[kPer], T *shared, float &peak,
                                          T &total, bool &unsure) {
  constexpr bool kCheck = sizeof(T) == 4;
  const int lane = threadIdx.x & 31;
  const int64_t base = (int64_t)row * a.experts;
  const T none = -INFINITY;
  T l[kPer], v[kPer];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = lane + 32 * i;
    const float x = e < a.experts ? read_logit(a, base + e) : -INFINITY;
    m = fmaxf(m, x);
    l[i] = x;
  }
  m = warp_max_f32(m);
  peak = m;
  total = 1;
  unsure = false;
  if (!(m > -INFINITY)) return -1;
  const bool values = a.bias || a.top_groups < a.groups;   // else the logits decide
  T smax = 0, cmax = 0;
  if (values || !a.renorm) {
    if (a.sigmoid) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = l[i] > none ? T(1) / (T(1) + exp_of(-l[i])) : T(0);
    } else {
      T z = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) z += v[i] = l[i] > none ? exp_of(l[i] - T(m)) : T(0);
      total = warp_sum(z);
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = v[i] / total;
    }
  }
  T tol = 0, group_tol = 0;
  if (values) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = lane + 32 * i;
      if (kCheck) smax = fmax(smax, v[i]);
      if (a.bias && e < a.experts) v[i] += T(a.bias[e]);
      if (!(l[i] > none) || !(v[i] > none)) l[i] = v[i] = none;
      else if (kCheck) cmax = fmax(cmax, fabs(v[i]));
    }
    if constexpr (kCheck) {
      smax = warp_max_f32(smax), cmax = warp_max_f32(cmax);
      const T off = smax * (a.sigmoid ? 0x1p-21f : 0x1p-19f);
      tol = 2 * off + cmax * 0x1p-22f;
      group_tol = 4 * off + cmax * 0x1p-20f;
    }
  }
  if (a.top_groups < a.groups) {
    // each group's two largest values by a few lanes
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (lane + 32 * i < a.experts) shared[lane + 32 * i] = v[i];
    __syncwarp();
    const int each = a.experts / a.groups;
    int lanes = 32;
    while (lanes * a.groups > 32) lanes >>= 1;
    const int g = lane / lanes, sub = lane % lanes;
    T first = none, second = none;
    if (g < a.groups)
      for (int i = sub; i < each; i += lanes) {
        const T x = shared[g * each + i];
        if (x > first) second = first, first = x;
        else if (x > second) second = x;
      }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
      const T x = __shfl_xor_sync(kFull, first, o), y = __shfl_xor_sync(kFull, second, o);
      second = fmax(fmin(first, x), fmax(second, y));
      first = fmax(first, x);
    }
    T sum = first > none && second > none ? first + second : first;
    if (sub) sum = none;
    uint32_t stays = 0;
    T last = none;
    for (int j = 0; j <= a.top_groups; ++j) {
      T best;
      const int at = warp_best(sum, g, best);
      if (at < 0) break;
      if (j < a.top_groups) {
        stays |= 1u << at;
        last = best;
        if (g == at) sum = none;
      } else if (kCheck && !(last - best > group_tol)) {
        unsure = true;
        return -1;
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (!(stays >> group[i] & 1u)) l[i] = v[i] = none;
  }
  if (!a.bias) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = l[i];
  }
  int mine = -1;
  T value = none, before = none;
  int at_before = -1;
  const int rounds = kCheck && a.bias ? a.top_k + 1 : a.top_k;
  for (int j = 0; j < rounds; ++j) {
    T x = v[0];
    int e = lane;
#pragma unroll
    for (int i = 1; i < kPer; ++i)
      if (v[i] > x) x = v[i], e = lane + 32 * i;
    T best;
    const int at = warp_best(x, e, best);
    if (at < 0) break;
    if (kCheck && a.bias && j > 0 && !(before - best > tol))
      unsure = unsure || a.bias[at] != a.bias[at_before] || read_logit(a, base + at) != read_logit(a, base + at_before);
    if (lane == j && j < a.top_k) mine = at, value = best;
    before = best, at_before = at;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (lane + 32 * i == at) v[i] = none;
  }
  return mine;
}

template <int kPer>
__device__ __noinline__ int choose_row_again(const RouteArgs &a, int row, const int (&group)[kPer], double *shared,
                                             float &peak, double &total) {
  bool unsure;
  return choose_row<double, kPer>(a, row, group, shared, peak, total, unsure);
}

// A warp a row.
template <int kPer>
__global__ void __launch_bounds__(kChooseWarps * 32) choose_kernel(RouteArgs a) {
  __shared__ double shared[kChooseWarps][kPer * 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int group[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) group[i] = min(lane + 32 * i, a.experts - 1) / (a.experts / a.groups);
  grid_dependency_wait();
  grid_launch_dependents();
  for (int row = blockIdx.x * kChooseWarps + warp; row < a.rows; row += gridDim.x * kChooseWarps) {
    float peak, z;
    bool unsure;
    int mine = choose_row<float, kPer>(a, row, group, reinterpret_cast<float *>(shared[warp]), peak, z, unsure);
    if (unsure) {
      double z64;
      __syncwarp();
      mine = choose_row_again<kPer>(a, row, group, shared[warp], peak, z64);
      z = (float)z64;
    }
    // the weights, from the chosen experts' logits alone: lane j has the j-th
    float s = 0.f;
    const float l = mine >= 0 ? read_logit(a, (int64_t)row * a.experts + mine) : -INFINITY;
    if (a.sigmoid) {
      if (mine >= 0) s = 1.f / (1.f + expf(-l));
    } else {
      const float top = a.renorm ? warp_max_f32(l) : peak;  // (a quotient: any common factor will do)
      if (mine >= 0) s = exp_difference(l, top);
      if (!a.renorm) s /= z;
    }
    if (a.renorm) {
      const float sum = warp_sum(s);
      if (mine >= 0) s /= sum;
    }
    if (lane < a.top_k) {
      const int64_t to = (int64_t)row * a.top_k + lane;
      a.expert[to] = mine;
      a.weight[to] = s * a.scale;
    }
  }
}

// ------------------------------------------------------------------------------------
// Grouping: a stable counting sort of the pairs by expert, by one cluster
// ------------------------------------------------------------------------------------
// A warp takes a stretch of the pairs, 32 at a time, and counts each expert's in a histogram of its own (the lanes
// with equal experts find one another, one of them counts: no atomics, so that every run gives the same order).  The
// histograms' running sums over warps, then CTAs (through distributed shared memory), then experts are where each
// warp's pairs of an expert begin; a second walk places them.
constexpr int kGroupThreads = 1024, kGroupWarps = 32, kGroupCtas = 8;

__global__ void __launch_bounds__(kGroupThreads) group_kernel(RouteArgs a, int64_t n) {
  extern __shared__ int32_t hist[];              // [warps][experts]
  __shared__ int32_t count[kMostExperts], first[kMostExperts], part[kGroupWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, E = a.experts;
  const int ctas = gridDim.x, rank = blockIdx.x;
  int32_t *mine = hist + warp * E;
  for (int e = lane; e < E; e += 32) mine[e] = 0;
  const int64_t stretch = ((n + ctas * kGroupWarps - 1) / (ctas * kGroupWarps) + 31) / 32 * 32;
  const int64_t from = (rank * kGroupWarps + warp) * stretch, to = min(n, from + stretch);
  grid_dependency_wait();
  grid_launch_dependents();
  __syncwarp();
  for (int64_t i = from; i < to; i += 32) {
    const int e = i + lane < to ? a.expert[i + lane] : -1;
    const uint32_t same = __match_any_sync(kFull, e);
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  for (int e = tid; e < E; e += kGroupThreads) {
    int run = 0;
    for (int w = 0; w < kGroupWarps; ++w) {
      const int c = hist[w * E + e];
      hist[w * E + e] = run;
      run += c;
    }
    count[e] = run;
  }
  if (ctas > 1) cluster_sync_all();
  else __syncthreads();
  int before = 0, all = 0;                       // this expert's, of the CTAs before and of all
  if (tid < E)
    for (int q = 0; q < ctas; ++q) {
      uint32_t c;
      if (ctas > 1) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(cluster_map_shared(smem_u32(&count[tid]), q)));
      else c = (uint32_t)count[tid];
      if (q < rank) before += (int)c;
      all += (int)c;
    }
  int run = all;                                 // over the experts up to this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kFull, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) part[warp] = run;
  if (ctas > 1) cluster_sync_all();              // (the counts have been read)
  else __syncthreads();
  int lead = 0, total = 0;
  for (int w = 0; w < kGroupWarps; ++w) {
    if (w < warp) lead += part[w];
    total += part[w];
  }
  if (tid < E) {
    first[tid] = lead + run - all + before;
    if (rank == 0) {
      a.offsets[tid] = lead + run - all;
      if (tid == 0) a.offsets[E] = total;
    }
  }
  __syncthreads();
  for (int64_t i = from; i < to; i += 32) {
    const int e = i + lane < to ? a.expert[i + lane] : -1;
    const uint32_t same = __match_any_sync(kFull, e);
    int at = -1;
    if (e >= 0) {
      at = first[e] + mine[e] + __popc(same & ((1u << lane) - 1));
      a.order[at] = (int32_t)(i + lane);
    }
    if (i + lane < to) a.place[i + lane] = at;
    __syncwarp();
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
  }
  for (int64_t i = total + rank * kGroupThreads + tid; i < n; i += ctas * kGroupThreads) a.order[i] = -1;
}

// ------------------------------------------------------------------------------------
// The weighted sum of a row's results
// ------------------------------------------------------------------------------------
struct CombineArgs {
  const void *y;           // [rows * top_k][n]
  const float *weight;     // [rows][top_k]
  const int32_t *place;
  const __nv_bfloat16 *add;  // nullable
  __nv_bfloat16 *out;
  int64_t slots;
  int top_k, n, f32;
};

// kEach neighbouring columns of a row a thread.
template <int kEach, bool kF32>
__global__ void __launch_bounds__(256) combine_kernel(CombineArgs a) {
  const int64_t row = blockIdx.x;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * kEach;
  grid_dependency_wait();
  grid_launch_dependents();
  if (c >= a.n) return;
  float sum[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum[i] = a.add ? __bfloat162float(a.add[row * a.n + c + i]) : 0.f;
  for (int j = 0; j < a.top_k; ++j) {
    const int64_t at = a.place[row * a.top_k + j];
    if (at < 0 || at >= a.slots) continue;
    const float w = a.weight[row * a.top_k + j];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int64_t from = at * a.n + c + i;
      const float y = kF32 ? static_cast<const float *>(a.y)[from]
                           : __bfloat162float(static_cast<const __nv_bfloat16 *>(a.y)[from]);
      sum[i] = fmaf(w, y, sum[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) a.out[row * a.n + c + i] = __float2bfloat16_rn(sum[i]);
}

template <int kPer>
cudaError_t launch_choose(const RouteArgs &a, cudaStream_t s) {
  const int blocks = (a.rows + kChooseWarps - 1) / kChooseWarps;
  return launch_after<choose_kernel<kPer>>(dim3((unsigned)blocks), dim3(kChooseWarps * 32), 0, dim3(1), s, a);
}

}  // namespace
}  // namespace ham

using ham::op_aligned;
using ham::op_fail;
using ham::op_overlap;

extern "C" {

int ham_route(const void *logits, int32_t logits_dtype, const float *bias, int32_t rows, int32_t experts,
              int32_t top_k, int32_t score, int32_t groups, int32_t top_groups, int32_t renorm, float scale,
              int32_t *expert, float *weight, int32_t *offsets, int32_t *order, int32_t *place, void *stream) {
  ham::ApiRange nvtx_range("ham_route");
  if (logits_dtype != HAM_DTYPE_BF16 && logits_dtype != HAM_DTYPE_F32)
    return op_fail(HAM_EINVAL, "logits_dtype %d", logits_dtype);
  if (score != HAM_SCORE_SOFTMAX && score != HAM_SCORE_SIGMOID) return op_fail(HAM_EINVAL, "score %d", score);
  if (rows < 0 || rows > (1 << 24)) return op_fail(HAM_EINVAL, "rows %d outside 0..2^24", rows);
  if (experts < 1 || experts > ham::kMostExperts)
    return op_fail(HAM_EINVAL, "experts %d outside 1..%d", experts, ham::kMostExperts);
  if (groups < 1 || groups > 32 || experts % groups != 0)
    return op_fail(HAM_EINVAL, "groups %d must divide the %d experts, 32 at most", groups, experts);
  if (top_groups < 1 || top_groups > groups) return op_fail(HAM_EINVAL, "top_groups %d outside 1..%d", top_groups, groups);
  const int most = experts / groups * top_groups;
  if (top_k < 1 || top_k > ham::kMostTop || top_k > most)
    return op_fail(HAM_EINVAL, "top_k %d outside 1..%d", top_k, most < ham::kMostTop ? most : ham::kMostTop);
  if (!(scale > -INFINITY && scale < INFINITY)) return op_fail(HAM_EINVAL, "scale must be finite");
  if (rows == 0) return HAM_OK;
  if (!logits || !expert || !weight || !offsets || !order || !place)
    return op_fail(HAM_EINVAL, "logits and the five outputs are required");
  const int f32 = logits_dtype == HAM_DTYPE_F32;
  for (const void *p : {(const void *)bias, (const void *)expert, (const void *)weight, (const void *)offsets,
                        (const void *)order, (const void *)place})
    if (!op_aligned(p, 4)) return op_fail(HAM_EINVAL, "pointers must be 4-byte aligned");
  if (!op_aligned(logits, f32 ? 4 : 2)) return op_fail(HAM_EINVAL, "logits must be aligned to their elements");
  const size_t pairs = (size_t)rows * top_k;
  struct Span { const void *p; size_t n; };
  const Span outs[5] = {{expert, 4 * pairs}, {weight, 4 * pairs}, {offsets, 4 * ((size_t)experts + 1)},
                        {order, 4 * pairs}, {place, 4 * pairs}};
  for (int i = 0; i < 5; ++i) {
    if (op_overlap(outs[i].p, outs[i].n, logits, (size_t)rows * experts * (f32 ? 4 : 2)) ||
        op_overlap(outs[i].p, outs[i].n, bias, 4 * (size_t)experts))
      return op_fail(HAM_EINVAL, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (op_overlap(outs[i].p, outs[i].n, outs[j].p, outs[j].n)) return op_fail(HAM_EINVAL, "two outputs overlap");
  }
  ham::RouteArgs a;
  a.logits = logits;
  a.bias = bias;
  a.f32 = f32;
  a.rows = rows;
  a.experts = experts;
  a.top_k = top_k;
  a.sigmoid = score == HAM_SCORE_SIGMOID;
  a.groups = groups;
  a.top_groups = top_groups;
  a.renorm = renorm != 0;
  a.scale = scale;
  a.expert = expert;
  a.weight = weight;
  a.offsets = offsets;
  a.order = order;
  a.place = place;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t ce = experts <= 32    ? ham::launch_choose<1>(a, s)
                   : experts <= 64  ? ham::launch_choose<2>(a, s)
                   : experts <= 128 ? ham::launch_choose<4>(a, s)
                   : experts <= 256 ? ham::launch_choose<8>(a, s)
                                    : ham::launch_choose<16>(a, s);
  if (ce == cudaSuccess) {
    static bool done[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !done[dev]) {
      ce = cudaFuncSetAttribute(ham::group_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                ham::kGroupWarps * ham::kMostExperts * 4);
      if (ce == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
    }
    const int ctas = pairs <= 8192 ? 1 : ham::kGroupCtas;
    if (ce == cudaSuccess)
      ce = ham::launch_after<ham::group_kernel>(dim3((unsigned)ctas), dim3(ham::kGroupThreads),
                                                (size_t)ham::kGroupWarps * experts * 4, dim3((unsigned)ctas), s, a,
                                                (int64_t)pairs);
  }
  return ce == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "route launch: %s", cudaGetErrorString(ce));
}

int ham_experts_combine(const void *y, int32_t y_dtype, const float *weight, const int32_t *place, const void *add,
                        int32_t rows, int32_t top_k, int32_t n, void *out, void *stream) {
  ham::ApiRange nvtx_range("ham_experts_combine");
  if (y_dtype != HAM_DTYPE_BF16 && y_dtype != HAM_DTYPE_F32) return op_fail(HAM_EINVAL, "y_dtype %d", y_dtype);
  if (rows < 0 || rows > (1 << 24)) return op_fail(HAM_EINVAL, "rows %d outside 0..2^24", rows);
  if (top_k < 1 || top_k > ham::kMostTop) return op_fail(HAM_EINVAL, "top_k %d outside 1..%d", top_k, ham::kMostTop);
  if (n < 1 || n > (1 << 20)) return op_fail(HAM_EINVAL, "n %d outside 1..2^20", n);
  if (rows == 0) return HAM_OK;
  if (!y || !weight || !place || !out) return op_fail(HAM_EINVAL, "y, weight, place and out are required");
  if (!op_aligned(y, 16) || !op_aligned(add, 16) || !op_aligned(out, 16))
    return op_fail(HAM_EINVAL, "y, add and out must be 16-byte aligned");
  if (!op_aligned(weight, 4) || !op_aligned(place, 4))
    return op_fail(HAM_EINVAL, "weight and place must be 4-byte aligned");
  const int f32 = y_dtype == HAM_DTYPE_F32;
  const size_t pairs = (size_t)rows * top_k, ob = (size_t)rows * n * 2;
  if (op_overlap(out, ob, y, pairs * n * (f32 ? 4 : 2)) || op_overlap(out, ob, weight, 4 * pairs) ||
      op_overlap(out, ob, place, 4 * pairs) || (op_overlap(out, ob, add, ob) && out != add))
    return op_fail(HAM_EINVAL, "out overlaps an input");
  ham::CombineArgs a;
  a.y = y;
  a.weight = weight;
  a.place = place;
  a.add = static_cast<const __nv_bfloat16 *>(add);
  a.out = static_cast<__nv_bfloat16 *>(out);
  a.slots = (int64_t)pairs;
  a.top_k = top_k;
  a.n = n;
  a.f32 = f32;
  const dim3 grid((unsigned)rows, (unsigned)((n + 255) / 256));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t ce = f32 ? ham::launch_after<ham::combine_kernel<1, true>>(grid, dim3(256), 0, dim3(1), s, a)
                             : ham::launch_after<ham::combine_kernel<1, false>>(grid, dim3(256), 0, dim3(1), s, a);
  return ce == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "combine launch: %s", cudaGetErrorString(ce));
}

}  // extern "C"

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

#include <algorithm>
#include <cfloat>

#include "ham_ops.cuh"
#include "ham_ptx.cuh"

namespace ham {
namespace {

constexpr int kMostExperts = 512, kMostTop = 32;
constexpr int kChooseWarps = 4;  // warps (rows) of a block

struct RouteArgs {
  const void *logits;      // [rows][experts] bf16 or f32
  const float *bias;       // nullable
  int f32, wide;           // wide: rows of whole 16 bytes
  int rows, experts, top_k, sigmoid, groups, top_groups, renorm;
  float scale;
  int32_t *expert;         // [rows][top_k]
  float *weight;
  int32_t *offsets, *order, *place;
};

// A logit as the formulas take it: -inf rules out (NaN too).
__device__ __forceinline__ float a_logit(const RouteArgs &a, float l) {
  l = l > -INFINITY ? fminf(l, FLT_MAX) : -INFINITY;
  return a.sigmoid && l > -INFINITY ? fmaxf(l, -80.f) : l;
}
__device__ __forceinline__ float read_logit(const RouteArgs &a, int64_t at) {
  return a_logit(a, a.f32 ? static_cast<const float *>(a.logits)[at]
                          : __bfloat162float(static_cast<const __nv_bfloat16 *>(a.logits)[at]));
}
// exp(l - top), l <= top, the difference's rounding (which a large one would carry over) put right.
__device__ __forceinline__ float exp_difference(float l, float top) {
  const float x = l - top, part = x - l;
  const float off = (l - (x - part)) - (top + part);   // (a difference's error, exactly: the two-sum)
  const float e = expf(x);
  return e > 0.f ? fmaf(e, off, e) : 0.f;
}
// A number's place in the order of floats, as an unsigned one; kNoRank: -inf, ruled out.
constexpr uint32_t kNoRank = 0x007fffffu;
__device__ __forceinline__ uint32_t rank_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);   // (-0 -> +0)
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
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
__device__ __forceinline__ int warp_best(double x, int index) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const double y = __shfl_xor_sync(kFull, x, o);
    const int j = __shfl_xor_sync(kFull, index, o);
    if (y > x || (y == x && j < index)) x = y, index = j;
  }
  return x > -INFINITY ? index : -1;
}

// One row's experts by a warp in fp64, lane j < top_k getting the j-th (-1: none): for the rows in which fp32 cannot tell
// two values apart.  `shared`: the row's values.
__device__ __noinline__ int choose_exactly(const RouteArgs &a, int row, double *shared) {
  const int lane = threadIdx.x & 31, each = a.experts / a.groups;
  const int64_t base = (int64_t)row * a.experts;
  double m = -INFINITY, z = 0;
  for (int e = lane; e < a.experts; e += 32) m = fmax(m, (double)read_logit(a, base + e));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(kFull, m, o));
  if (!a.sigmoid) {
    for (int e = lane; e < a.experts; e += 32) z += exp((double)read_logit(a, base + e) - m);
    z = warp_sum(z);
  }
  for (int e = lane; e < a.experts; e += 32) {
    const double l = read_logit(a, base + e);
    double v = a.sigmoid ? 1 / (1 + exp(-l)) : exp(l - m) / z;
    if (a.bias) v += a.bias[e];
    shared[e] = l > -INFINITY && v > -INFINITY ? v : -INFINITY;
  }
  __syncwarp();
  uint32_t stays = kFull;
  if (a.top_groups < a.groups) {
    double first = -INFINITY, second = -INFINITY;
    if (lane < a.groups)
      for (int i = 0; i < each; ++i) {
        const double x = shared[lane * each + i];
        if (x > first) second = first, first = x;
        else if (x > second) second = x;
      }
    double sum = first > -INFINITY && second > -INFINITY ? first + second : first;
    stays = 0;
    for (int j = 0; j < a.top_groups; ++j) {
      const int at = warp_best(sum, lane);
      if (at < 0) break;
      stays |= 1u << at;
      if (lane == at) sum = -INFINITY;
    }
  }
  int mine = -1;
  for (int j = 0; j < a.top_k; ++j) {
    double x = -INFINITY;
    int e = INT32_MAX;
    for (int i = lane; i < a.experts; i += 32)
      if (stays >> i / each & 1u) {
        // (without a bias the logits decide; an expert that was taken is ruled out)
        const double y = a.bias || !(shared[i] > -INFINITY) ? shared[i] : (double)read_logit(a, base + i);
        if (y > x) x = y, e = i;
      }
    const int at = warp_best(x, e);
    if (at < 0) break;
    if (lane == j) mine = at;
    if (lane == (at & 31)) shared[at] = -INFINITY;
    __syncwarp();
  }
  __syncwarp();
  return mine;
}

// ------------------------------------------------------------------------------------
// The choice: a warp a row
// ------------------------------------------------------------------------------------
// A lane has kPer neighbouring experts, in registers: scores, values and the groups' sums (a group that lies in whole
// lanes takes two shuffles a doubling) need no shared memory.  Each lane brings its three largest to its front, in order;
// then the warp's largest first one is taken top_k times, a reduction, a ballot and a shift of the owner's each, and a lane
// that runs out brings up one more.  (16384 rows of 256 in 8 groups with one, two, three, four and all of them in order at first:
// 35.4, 29.8, 29.2, 29.8 and 30.7 us a call, grouping and all; 8192 rows of 512: 26.2, 20.1, 20.0, 20.7, 26.0.)  Deciding in fp32
// and only where two values are nearer than their errors in fp64, for those values alone, costs a few comparisons a row:
// with whole rows computed again 16384 rows of 256 with sigmoid and bias take 47.6 us, so 25.9; in groups 54.3, so 29.2.
//
// A warp has one row: blocks that stay and take rows in turn, 4 an SM of 8 warps, have a last turn that is a third full (an eighth
// slower when it was tried, on an earlier form).
//
// Bound by instructions, some 1050 a row of 256 experts in 8 groups: of the 29.2 us that 16384 rows take, 21 are the
// choice (of 20.0 where the logits alone decide, 11.4), and reading the logits takes 2.5.  bf16 logits, read one by one, cost
// as much: 30.7 and 20.4 us.
//
// What is known of a call where its kernel is made: nothing; that the logits decide alone; sigmoid and a bias; these and groups
// of 2^i whole lanes.  (Asked for in the kernel, the flags cost 16384 rows of 256 with sigmoid and a bias 27.5 us a call
// instead of 25.9, where the logits alone decide 23.0 instead of 20.0.)
enum { kAnyChoice, kByLogits, kSigmoidBias, kSigmoidBiasGroups };
// Lane's experts: lane * kPer .. lane * kPer + kPer - 1.
template <int kPer, int kMode>
struct Chooser {
  float bias[kPer];        // this lane's experts'
  int each, lanes, group;  // experts of a group; the lanes that hold one (0: it does not lie in 2^i whole lanes), this lane's

  __device__ __forceinline__ explicit Chooser(const RouteArgs &a) {
    const int lane = threadIdx.x & 31;
    each = a.experts / a.groups;
    lanes = each % kPer == 0 ? each / kPer : 0;
    if (lanes & (lanes - 1)) lanes = 0;
    group = lane * kPer / each;
#pragma unroll
    for (int i = 0; i < kPer; ++i) bias[i] = a.bias && lane * kPer + i < a.experts ? a.bias[lane * kPer + i] : 0.f;
  }

  __device__ __forceinline__ void read(const RouteArgs &a, int row, float (&l)[kPer]) const {
    const int e0 = (threadIdx.x & 31) * kPer;
    const int64_t base = (int64_t)row * a.experts + e0;
    if (kPer >= 4 && a.f32 && a.wide) {
#pragma unroll
      for (int i = 0; i < kPer; i += 4) {
        float4 x = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (e0 + i < a.experts) x = *reinterpret_cast<const float4 *>(static_cast<const float *>(a.logits) + base + i);
        l[i] = a_logit(a, x.x), l[i + 1] = a_logit(a, x.y), l[i + 2] = a_logit(a, x.z), l[i + 3] = a_logit(a, x.w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) l[i] = e0 + i < a.experts ? read_logit(a, base + i) : -INFINITY;
    }
  }

  // The row's experts, lane j < top_k getting the j-th (-1: none).  `unsure`: two values that a decision lies between are
  // nearer than their errors.  `shared`: room for the row's values.
  //
  // The errors, relative to the row's largest score: of a sigmoid two units of expf, half a unit of a sum and one of a
  // reciprocal, below 2^-21;
  // of a softmax the rounding of l - max (|x| exp(x) <= 0.37 units), expf, 21 additions and a quotient, below 2^-19.  A
  // value adds half a unit of itself; the bound takes the row's largest for all.  (So a bias far beyond the scores, the lowest
  // finite number as a mask, has every row decided in fp64: 16384 rows of 256 then take 395 us, in groups 721.  A mask of -inf
  // costs nothing.)  Equal logits with equal biases are equal exactly, however they are computed.
  __device__ __forceinline__ int choose(const RouteArgs &a, int row, float *shared, float &peak, float &z, bool &unsure) const {
    const int lane = threadIdx.x & 31;
    float l[kPer];
    read(a, row, l);
    float m = l[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) m = fmaxf(m, l[i]);
    m = warp_max_f32(m);
    peak = m;
    z = 1.f;
    unsure = false;
    if (!(m > -INFINITY)) return -1;
    constexpr bool kAll = kMode == kSigmoidBiasGroups, kBoth = kAll || kMode == kSigmoidBias;
    const bool grouped = kAll || (kMode == kAnyChoice && a.top_groups < a.groups);
    const bool has_bias = kBoth || (kMode == kAnyChoice && a.bias), sigmoid = kBoth || a.sigmoid;
    uint32_t k[kPer];                            // the experts' places in the order
    float tol = 0.f, group_tol = 0.f;
    if (kMode != kByLogits && (has_bias || grouped || !(a.renorm || sigmoid))) {  // (else the logits' quotients suffice)
      float v[kPer];
      if (sigmoid) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(v[i]) : "f"(1.f + expf(-l[i])));  // (0 where ruled out)
        }
      } else {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += v[i] = expf(l[i] - m);
        z = warp_sum(sum);
        const float back = 1.f / z;
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] *= back;
      }
      if (has_bias || grouped) {
        float smax = 0.f, cmax = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          smax = fmaxf(smax, v[i]);
          v[i] += bias[i];
          if (!(l[i] > -INFINITY && v[i] > -INFINITY)) v[i] = -INFINITY;
          else cmax = fmaxf(cmax, fabsf(v[i]));
        }
        smax = warp_max_f32(smax), cmax = warp_max_f32(cmax);
        const float off = smax * (sigmoid ? 0x1p-21f : 0x1p-19f);
        tol = 2 * off + cmax * 0x1p-22f;
        group_tol = 4 * off + cmax * 0x1p-20f;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (!(v[i] > -INFINITY)) l[i] = -INFINITY;
      }
      if (grouped) {
        uint32_t stays;
        if (!keep_groups(a, l, v, shared, group_tol, stays)) {
          unsure = true;
          return -1;
        }
        if (kAll || lanes) {
          if (!(stays >> group & 1u)) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) l[i] = v[i] = -INFINITY;
          }
        } else {
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (!(stays >> (lane * kPer + i) / each & 1u)) l[i] = v[i] = -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) k[i] = rank_of(has_bias ? v[i] : l[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) k[i] = rank_of(l[i]);
    }
    // Each lane's largest few in order at its front (passes from the back that change neighbours' places, so that equal ones
    // keep theirs), then the warp's largest first one, again and again; a lane that has no more in order makes all pass once more.
    constexpr int kFront = kPer < 3 ? kPer : 3;
    uint32_t id[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) id[i] = i;
    const auto pass = [&](int from) {
#pragma unroll
      for (int i = kPer - 2; i >= 0; --i)
        if (i >= from) {
          const bool swap = k[i] < k[i + 1];
          const uint32_t x = k[i], y = id[i];
          k[i] = max(x, k[i + 1]), k[i + 1] = min(x, k[i + 1]);
          id[i] = swap ? id[i + 1] : y, id[i + 1] = swap ? y : id[i + 1];
        }
    };
#pragma unroll
    for (int i = 0; i < kFront; ++i) pass(i);
    int front = kFront;                          // in order
    int mine = -1;                               // lane j: the j-th; with a bias the one after the last too
    uint32_t rank = kNoRank;
    const int rounds = min(a.top_k + (has_bias ? 1 : 0), 32);
    for (int j = 0; j < rounds; ++j) {
      const uint32_t top = __reduce_max_sync(kFull, k[0]);
      if (top == kNoRank) break;
      const int owner = __ffs(__ballot_sync(kFull, k[0] == top)) - 1;
      const int e = owner * kPer + (int)__shfl_sync(kFull, id[0], owner);
      if (lane == j) mine = e, rank = top;
      if (lane == owner) {
#pragma unroll
        for (int i = 0; i + 1 < kFront; ++i) k[i] = k[i + 1], id[i] = id[i + 1];
        k[kFront - 1] = kNoRank;
        --front;
      }
      if (kPer > kFront && __any_sync(kFull, front == 0)) {
        pass(0);
        front = min(front + 1, kFront);
      }
    }
    if (has_bias) {
      uint32_t next = __shfl_down_sync(kFull, rank, 1);
      int e = __shfl_down_sync(kFull, mine, 1);
      if (a.top_k == 32) {                       // (a lane for each: the one after the last is still to come)
        const uint32_t top = __reduce_max_sync(kFull, k[0]);
        if (lane == 31) next = top, e = -1;
      }
      const bool near = lane < a.top_k && next > kNoRank && !(value_of(rank) - value_of(next) > tol);
      if (__any_sync(kFull, near)) {
        const int64_t base = (int64_t)row * a.experts;
        const bool differ = near && (e < 0 || a.bias[mine] != a.bias[e] || read_logit(a, base + mine) != read_logit(a, base + e));
        if (__any_sync(kFull, differ)) {
          // A sigmoid's value is its own logit's alone: where what follows is far enough away, the few chosen are put in
          // order by their exact values.
          const uint32_t follows = __reduce_max_sync(kFull, k[0]);
          const bool apart = follows == kNoRank || value_of(__shfl_sync(kFull, rank, rounds - 1)) - value_of(follows) > tol;
          if (!sigmoid || rounds > 31 || !apart) {
            unsure = true;
          } else {
            double exact = -INFINITY;
            if (mine >= 0) exact = 1 / (1 + exp(-(double)read_logit(a, base + mine))) + a.bias[mine];
            int at = 0;                            // of this lane's among the others
            for (int j = 0; j < rounds; ++j) {
              const double other = __shfl_sync(kFull, exact, j);
              const int o = __shfl_sync(kFull, mine, j);
              at += o >= 0 && (other > exact || (other == exact && o < mine));
            }
            if (mine < 0) at = 32;
            int sorted = -1;
            for (int j = 0; j < rounds; ++j)
              if (__shfl_sync(kFull, at, j) == lane) sorted = j;
            const int chosen = __shfl_sync(kFull, mine, max(sorted, 0));
            mine = sorted >= 0 ? chosen : -1;
          }
        } else if (__shfl_sync(kFull, near, a.top_k - 1)) {
          // The one after the last is exactly the last's equal: what is still to come and near may be larger all the same.
          const int last = __shfl_sync(kFull, mine, a.top_k - 1);
          const float value = value_of(__shfl_sync(kFull, rank, a.top_k - 1)), b = a.bias[last], x = read_logit(a, base + last);
          bool other = false;
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (k[i] > kNoRank && !(value - value_of(k[i]) > tol)) {
              const int e = lane * kPer + (int)id[i];
              other |= a.bias[e] != b || read_logit(a, base + e) != x;
            }
          unsure = __any_sync(kFull, other);
        }
      }
      if (lane >= a.top_k) mine = -1;
    }
    return mine;
  }

  // The top_groups groups of the largest sums of two values, a bit each; false: two sums are too near to one another.
  __device__ __forceinline__ bool keep_groups(const RouteArgs &a, const float (&l)[kPer], const float (&v)[kPer], float *shared,
                                              float tol, uint32_t &stays) const {
    const int lane = threadIdx.x & 31;
    float first = -INFINITY, second = -INFINITY;
    int g = group, step = lanes;                 // the group that this lane works at, the lanes that do
    if (kMode == kSigmoidBiasGroups || lanes) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        second = fmaxf(second, fminf(first, v[i]));
        first = fmaxf(first, v[i]);
      }
    } else {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (lane * kPer + i < a.experts) shared[lane * kPer + i] = v[i];
      __syncwarp();
      step = 32;
      while (step * a.groups > 32) step >>= 1;
      g = lane / step;
      if (g < a.groups)
        for (int i = lane % step; i < each; i += step) {
          const float x = shared[g * each + i];
          second = fmaxf(second, fminf(first, x));
          first = fmaxf(first, x);
        }
    }
    for (int o = step >> 1; o > 0; o >>= 1) {
      const float x = __shfl_xor_sync(kFull, first, o), y = __shfl_xor_sync(kFull, second, o);
      second = fmaxf(fminf(first, x), fmaxf(second, y));
      first = fmaxf(first, x);
    }
    // (Whether a group has an expert left is asked of its largest value: a sum of two finite ones may be infinite.)
    const bool live = g < a.groups && first > -INFINITY;
    const float sum = second > -INFINITY ? first + second : first;
    const bool passes = __any_sync(kFull, live && fabsf(sum) == INFINITY);   // fp32's range: the exact sums decide
    int before = 0;                              // groups that come before this one
    for (int i = 0; i < a.groups; ++i) {
      const float other = __shfl_sync(kFull, sum, i * step);
      before += other > sum || (other == sum && i < g);
    }
    const bool kept = live && before < a.top_groups;
    const uint32_t least = __reduce_min_sync(kFull, kept ? rank_of(sum) : kFull);
    const uint32_t most = __reduce_max_sync(kFull, live && !kept ? rank_of(sum) : kNoRank);
    stays = __reduce_or_sync(kFull, kept ? 1u << g : 0u);
    if (!passes && (most == kNoRank || value_of(least) - value_of(most) > tol)) return true;
    if (kMode != kSigmoidBiasGroups && (!a.sigmoid || !lanes)) return false;
    // Exactly, a sigmoid's value being its own logit's alone: the values that may be a group's two largest, one a lane at a
    // time.
    uint32_t wanted = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (v[i] > -INFINITY && !(v[i] < (second > -INFINITY ? second : first) - tol)) wanted |= 1u << i;
    double first64 = -INFINITY, second64 = -INFINITY;
    while (__any_sync(kFull, wanted)) {
      const int at = __ffs(wanted) - 1;
      float x = -INFINITY, b = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i == at) x = l[i], b = bias[i];
      const double exact = at >= 0 ? 1 / (1 + exp(-(double)x)) + b : -INFINITY;
      second64 = fmax(second64, fmin(first64, exact));
      first64 = fmax(first64, exact);
      wanted &= wanted - 1;
    }
    for (int o = step >> 1; o > 0; o >>= 1) {
      const double x = __shfl_xor_sync(kFull, first64, o), y = __shfl_xor_sync(kFull, second64, o);
      second64 = fmax(fmin(first64, x), fmax(second64, y));
      first64 = fmax(first64, x);
    }
    const double sum64 = second64 > -INFINITY ? first64 + second64 : first64;
    before = 0;
    for (int i = 0; i < a.groups; ++i) {
      const double other = __shfl_sync(kFull, sum64, i * step);
      before += other > sum64 || (other == sum64 && i < g);
    }
    stays = __reduce_or_sync(kFull, live && before < a.top_groups ? 1u << g : 0u);
    return true;
  }
};

// A row by a warp.
template <int kPer, int kMode>
__device__ __forceinline__ void choose_row(const RouteArgs &a, int row, double *shared) {
  const int lane = threadIdx.x & 31;
  const Chooser<kPer, kMode> chooser(a);
  float peak, z;
  bool unsure;
  int mine = chooser.choose(a, row, reinterpret_cast<float *>(shared), peak, z, unsure);
  if (unsure) {
    __syncwarp();
    mine = choose_exactly(a, row, shared);
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

template <int kPer, int kMode>
__global__ void __launch_bounds__(kChooseWarps * 32) choose_kernel(const __grid_constant__ RouteArgs a) {
  __shared__ double shared[kChooseWarps][kPer * 32];
  const int warp = threadIdx.x >> 5;
  grid_dependency_wait();
  grid_launch_dependents();
  const int64_t row = (int64_t)blockIdx.x * kChooseWarps + warp;
  if (row < a.rows) choose_row<kPer, kMode>(a, (int)row, shared[warp]);
}

// ------------------------------------------------------------------------------------
// Grouping: a stable counting sort of the pairs by expert, by one cluster
// ------------------------------------------------------------------------------------
// A warp takes a stretch of rows, 32 at a time, and counts each expert's in a histogram of its own.  The
// histograms' running sums over warps, then CTAs (through distributed shared memory), then experts are where each warp's
// pairs of an expert begin.  A second walk places them: a row has an expert once at most, so that the rows of 32 that
// have it are bits of a word (or-ed together in any order), and a pair's place is the bits before its own.  (With the
// lanes of equal experts finding one another, 32 pairs at a time, 131072 pairs took 27 us.)
//
// A CTA that has no more than kStaged pairs puts them in their order in shared memory and writes each expert's one after
// another (1024 rows of 8 of 64: 7.9 us a call against 9.4 with scattered words; 16384 rows of 256 20.0 against 22.0).
constexpr int kGroupThreads = 1024, kGroupWarps = 32, kGroupCtas = 16, kStaged = 16384;
// (Pitch of the histograms: odd, so that four lanes that add up eight warps each of one expert's meet no bank twice.)
__host__ __device__ constexpr int group_pitch(int experts) { return experts | 1; }
__host__ __device__ constexpr int group_smem(int experts, bool staged) {
  return 2 * kGroupWarps * group_pitch(experts) * 4 + (staged ? kStaged * 4 : 0);
}
// (Rows of a warp.)
__host__ __device__ constexpr int group_stretch(int rows, int ctas) {
  return ((rows + ctas * kGroupWarps - 1) / (ctas * kGroupWarps) + 31) & ~31;
}
static_assert(group_smem(kMostExperts, true) <= 220 * 1024, "shared memory");

// kOnce: the stretch is 32 rows, whose bits the first walk finds and counts for both.  (16384 rows of 8 of 64: 15.0 us a call
// otherwise, so 14.2; 1333 rows of 4 of 60 8.0 and 7.2.  Asked for in the kernel, it cost 65536 rows of 2 of 64 7%.)
//
// (Every thread of a block of kGroupThreads, of every block of the cluster; hist: [2][warps][pitch], and the staged pairs.)
template <bool kOnce>
__device__ __forceinline__ void group_pairs(const RouteArgs &a, int32_t *hist, bool staged) {
  __shared__ int32_t count[kMostExperts], first[kMostExperts], local[kMostExperts], part[2][kGroupWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, E = a.experts, K = a.top_k, pitch = group_pitch(E);
  const int ctas = gridDim.x, rank = blockIdx.x;   // (one cluster)
  int32_t *mine = hist + warp * pitch;
  uint32_t *rows_of = reinterpret_cast<uint32_t *>(hist + (kGroupWarps + warp) * pitch);
  uint32_t *stage = reinterpret_cast<uint32_t *>(hist + 2 * kGroupWarps * pitch);
  const int stretch = kOnce ? 32 : group_stretch(a.rows, ctas);
  const int64_t row0 = (int64_t)rank * kGroupWarps * stretch;                                // the CTA's first
  const int64_t from = row0 + (int64_t)warp * stretch, to = min((int64_t)a.rows, from + stretch);
  const uint32_t one_kth = 65536 / K + 1;        // x / K = x one_kth / 65536 for x < 1024
  int e[8];                                      // experts of 8 x 32 pairs
  const auto read = [&](int64_t p0, int i0, int pairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = i0 + 32 * i + lane < pairs ? a.expert[p0 + i0 + 32 * i + lane] : -1;
  };
  const auto mark = [&](int i0) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (e[i] >= 0) atomicOr(&rows_of[e[i]], 1u << ((i0 + 32 * i + lane) * one_kth >> 16));
  };
  for (int x = lane; x < E; x += 32) mine[x] = 0, rows_of[x] = 0;
  __syncwarp();
  const int64_t first_pair = from * K;
  const int most = to > from ? (int)min((int64_t)stretch, to - from) * K : 0;
  for (int i0 = 0; i0 < most; i0 += 8 * 32) {
    read(first_pair, i0, most);
    if (kOnce) {
      mark(i0);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e[i] >= 0) atomicAdd(&mine[e[i]], 1);    // (of whole numbers: any order)
    }
  }
  __syncthreads();
  for (int x = tid >> 2; x < (E + 7) / 8 * 8; x += kGroupThreads / 4) {
    const int w0 = (tid & 3) * (kGroupWarps / 4);
    int c[kGroupWarps / 4], run = 0;
#pragma unroll
    for (int i = 0; i < kGroupWarps / 4; ++i) {
      c[i] = run;
      if (x < E) run += kOnce ? __popc((uint32_t)hist[(kGroupWarps + w0 + i) * pitch + x]) : hist[(w0 + i) * pitch + x];
    }
    int upto = run;
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const int y = __shfl_up_sync(kFull, upto, o, 4);
      if ((tid & 3) >= o) upto += y;
    }
    if (x < E) {
#pragma unroll
      for (int i = 0; i < kGroupWarps / 4; ++i) hist[(w0 + i) * pitch + x] = upto - run + c[i];
      if ((tid & 3) == 3) count[x] = upto;
    }
  }
  if (ctas > 1) cluster_sync_all();
  else __syncthreads();
  int before = 0, all = 0, own = 0;              // this expert's, of the CTAs before, of all, of this one
  if (tid < E) {
    own = count[tid];
    if (ctas > 1) {
      uint32_t c[kGroupCtas];
#pragma unroll
      for (int q = 0; q < kGroupCtas; ++q) {
        c[q] = 0;
        if (q < ctas)
          asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c[q]) : "r"(cluster_map_shared(smem_u32(&count[tid]), q)));
      }
#pragma unroll
      for (int q = 0; q < kGroupCtas; ++q) {
        if (q < rank) before += (int)c[q];
        all += (int)c[q];
      }
    } else {
      all = own;
    }
  }
  int run = all, own_run = own;                  // over the experts up to this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kFull, run, o), y = __shfl_up_sync(kFull, own_run, o);
    if (lane >= o) run += x, own_run += y;
  }
  if (lane == 31) part[0][warp] = run, part[1][warp] = own_run;
  if (ctas > 1) cluster_sync_all();              // (the counts have been read)
  else __syncthreads();
  const int warps = (E + 31) / 32;               // that have experts
  const int all_of = lane < warps ? part[0][lane] : 0, own_of = lane < warps ? part[1][lane] : 0;
  const int total = __reduce_add_sync(kFull, all_of), owned = __reduce_add_sync(kFull, own_of);
  const int lead = __reduce_add_sync(kFull, lane < warp ? all_of : 0), own_lead = __reduce_add_sync(kFull, lane < warp ? own_of : 0);
  if (tid < E) {
    first[tid] = lead + run - all + before;
    local[tid] = own_lead + own_run - own;
    if (rank == 0) {
      a.offsets[tid] = lead + run - all;
      if (tid == 0) a.offsets[E] = total;
    }
  }
  __syncthreads();
  for (int64_t r0 = from; r0 < to; r0 += 32) {
    const int64_t p0 = r0 * K;
    const int pairs = (int)min((int64_t)32, to - r0) * K;
    if (!kOnce) {
      for (int i0 = 0; i0 < pairs; i0 += 8 * 32) {
        read(p0, i0, pairs);
        mark(i0);
      }
      __syncwarp();
    }
    for (int i0 = 0; i0 < pairs; i0 += 8 * 32) {
      if (pairs > 8 * 32) read(p0, i0, pairs);
      int at[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        at[i] = -1;
        if (e[i] < 0) continue;
        const int p = i0 + 32 * i + lane;
        const int r = mine[e[i]] + __popc(rows_of[e[i]] & ((1u << (p * one_kth >> 16)) - 1));
        at[i] = first[e[i]] + r;
        if (staged) stage[local[e[i]] + r] = (uint32_t)((int)(p0 - row0 * K) + p) << 9 | (uint32_t)e[i];
        else a.order[at[i]] = (int32_t)(p0 + p);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i0 + 32 * i + lane < pairs) a.place[p0 + i0 + 32 * i + lane] = at[i];
    }
    if (kOnce) break;
    __syncwarp();
    for (int x = lane; x < E; x += 32) {
      mine[x] += __popc(rows_of[x]);
      rows_of[x] = 0;
    }
    __syncwarp();
  }
  if (staged) {
    __syncthreads();
    for (int p = tid; p < owned; p += kGroupThreads) {
      const uint32_t v = stage[p];
      const int e = (int)(v & 511u);
      a.order[first[e] + p - local[e]] = (int32_t)(row0 * K + (v >> 9));
    }
  }
  const int64_t n = (int64_t)a.rows * K;
  for (int64_t i = total + rank * kGroupThreads + tid; i < n; i += ctas * kGroupThreads) a.order[i] = -1;
}

template <bool kOnce>
__global__ void __launch_bounds__(kGroupThreads) group_kernel(const __grid_constant__ RouteArgs a, int staged) {
  extern __shared__ int32_t hist[];
  grid_dependency_wait();
  grid_launch_dependents();
  group_pairs<kOnce>(a, hist, staged != 0);
}

// A few rows: the choice and the grouping by one block.  (us with one launch / with two, of 2, 8 and 32 choices.  64 experts: 8 rows
// 4.2 / 4.4, 4.5 / 4.8, 6.1 / 6.3; 16 rows 4.5 / 4.4, 5.0 / 4.9, 7.2 / 7.2; 256 experts: 8 rows 5.3 / 5.2, 5.8 / 5.8, 7.9 / 7.8; 16 rows
// 5.7 / 5.3, 6.4 / 5.9, 9.6 / 8.8; 32 rows of 8 choices 5.9 / 5.2 and 7.8 / 6.2.  Up to 16 for the sake of calls outside
// graphs, where a launch is two of the host's.  With more than 256 experts the block's 64 registers a thread spill 204 bytes.)
constexpr int kFewRows = 16;
static_assert(kFewRows <= kGroupWarps, "a warp has one row");
template <int kPer>
__global__ void __launch_bounds__(kGroupThreads) route_few_kernel(const __grid_constant__ RouteArgs a) {
  extern __shared__ int32_t hist[];              // the grouping's, before that [warps][values]
  grid_dependency_wait();
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5;
  if (warp < a.rows) choose_row<kPer, kAnyChoice>(a, warp, reinterpret_cast<double *>(hist) + warp * (kPer * 32));
  __syncthreads();
  group_pairs<true>(a, hist, false);
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
  int top_k, n;
};

// kEach neighbouring numbers as they lie in memory, read at once (16 bytes at a time at most).
template <typename T, int kEach>
struct alignas(sizeof(T) * kEach < 16 ? sizeof(T) * kEach : 16) Piece {
  T v[kEach];
};
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// kEach neighbouring columns of a row a thread, kGroups times (a block's columns apart).  The results of kTogether
// places are read before any is added.  (4096 rows of 8 x 4096 in bf16: 62 us where numbers were converted as they were
// read, so that each read was waited for.)
constexpr int kTogether = 4;
template <int kEach, int kGroups, typename Y>
__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ CombineArgs a) {
  const int64_t row = blockIdx.x;
  const int c0 = (blockIdx.y * kGroups * blockDim.x + threadIdx.x) * kEach;
  grid_dependency_wait();
  grid_launch_dependents();
  float sum[kGroups][kEach];
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    const int c = c0 + g * (int)blockDim.x * kEach;
    Piece<uint16_t, kEach> p = {};
    if (a.add && c < a.n) p = *reinterpret_cast<const Piece<uint16_t, kEach> *>(a.add + row * a.n + c);
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum[g][i] = as_float(p.v[i]);
  }
  for (int j0 = 0; j0 < a.top_k; j0 += kTogether) {
    Piece<Y, kEach> p[kTogether][kGroups];
    float w[kTogether];
    bool live[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int64_t pair = row * a.top_k + j0 + j;
      const int64_t at = j0 + j < a.top_k ? a.place[pair] : -1;
      live[j] = at >= 0 && at < a.slots;
      w[j] = live[j] ? a.weight[pair] : 0.f;
      const Y *y = static_cast<const Y *>(a.y) + at * a.n + c0;
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
        if (live[j] && c0 + g * (int)blockDim.x * kEach < a.n) p[j][g] = *reinterpret_cast<const Piece<Y, kEach> *>(y + g * (int)blockDim.x * kEach);
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j)
      if (live[j]) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int i = 0; i < kEach; ++i) sum[g][i] = fmaf(w[j], as_float(p[j][g].v[i]), sum[g][i]);
      }
  }
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    const int c = c0 + g * (int)blockDim.x * kEach;
    if (c >= a.n) continue;
    Piece<uint16_t, kEach> p;
#pragma unroll
    for (int i = 0; i < kEach; ++i) p.v[i] = __bfloat16_as_ushort(__float2bfloat16_rn(sum[g][i]));
    *reinterpret_cast<Piece<uint16_t, kEach> *>(a.out + row * a.n + c) = p;
  }
}
template <int kEach, int kGroups>
cudaError_t launch_combine(const CombineArgs &a, int rows, bool f32, cudaStream_t s) {
  // a row in as few blocks of threads as hold it, of equal shares
  const int share = (a.n + kEach * kGroups - 1) / (kEach * kGroups), parts = (share + 255) / 256;
  const dim3 grid((unsigned)rows, (unsigned)parts), block((unsigned)(((share + parts - 1) / parts + 31) / 32 * 32));
  return f32 ? launch_after<combine_kernel<kEach, kGroups, float>>(grid, block, 0, dim3(1), s, a)
             : launch_after<combine_kernel<kEach, kGroups, uint16_t>>(grid, block, 0, dim3(1), s, a);
}

// CTAs of a grouping cluster at most: 16 need a group of SMs that holds as many.
int group_ctas(int dev) {
  static int known[64] = {};
  if (dev >= 0 && dev < 64 && known[dev]) return known[dev];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kGroupCtas);
  cfg.blockDim = dim3(kGroupThreads);
  cfg.dynamicSmemBytes = (size_t)group_smem(kMostExperts, true);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kGroupCtas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const auto fit = [&](auto kernel) {
    int n = 0;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
           cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess && n > 0;
  };
  const bool fits = fit(group_kernel<true>) && fit(group_kernel<false>);
  if (!fits) cudaGetLastError();
  const int ctas = fits ? kGroupCtas : 8;
  if (dev >= 0 && dev < 64) known[dev] = ctas;
  return ctas;
}

// Launches of Kernel<kPer> for the experts' number.
template <int kPer>
cudaError_t launch_route(const RouteArgs &a, cudaStream_t s) {
  static bool few_done[64] = {}, once_done[64] = {}, done[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (a.rows <= kFewRows) {
    constexpr int kMost = std::max(kGroupWarps * kPer * 32 * 8, group_smem(kPer * 32, false));
    const cudaError_t e = allow_smem(route_few_kernel<kPer>, kMost, few_done, dev);
    return e != cudaSuccess ? e : launch_after<route_few_kernel<kPer>>(dim3(1), dim3(kGroupThreads), (size_t)kMost, dim3(1), s, a);
  }
  const dim3 grid((unsigned)(((int64_t)a.rows + kChooseWarps - 1) / kChooseWarps)), block(kChooseWarps * 32);
  const int each = a.experts / a.groups, lanes = each / kPer;
  const bool grouped = a.top_groups < a.groups;
  cudaError_t e = !a.bias && !grouped && (a.renorm || a.sigmoid) ? launch_after<choose_kernel<kPer, kByLogits>>(grid, block, 0, dim3(1), s, a)
                  : a.sigmoid && a.bias && !grouped ? launch_after<choose_kernel<kPer, kSigmoidBias>>(grid, block, 0, dim3(1), s, a)
                  : a.sigmoid && a.bias && each % kPer == 0 && (lanes & (lanes - 1)) == 0
                      ? launch_after<choose_kernel<kPer, kSigmoidBiasGroups>>(grid, block, 0, dim3(1), s, a)
                      : launch_after<choose_kernel<kPer, kAnyChoice>>(grid, block, 0, dim3(1), s, a);
  if (e == cudaSuccess) e = allow_smem(group_kernel<true>, group_smem(kMostExperts, true), once_done, dev);
  if (e == cudaSuccess) e = allow_smem(group_kernel<false>, group_smem(kMostExperts, true), done, dev);
  if (e != cudaSuccess) return e;
  // The steps lie where a warp would have a second stretch of 32 rows, however many the choices.  (The whole call with one
  // block / a cluster of eight / of sixteen, us, 64 experts.  2 choices: 1024 rows 5.8 / 6.5 / 6.6, 2048 rows 7.9 / 6.7 / 6.8,
  // 8192 rows 18 / 8.0 / 8.2, 16384 rows 36 / 12.7 / 10.5; 8: 7.8 / 8.6 / 8.7, 12.4 / 8.9 / 9.0, 47 / 11.1 / 11.2, 87 / 18.7 / 14.3; 32:
  // 28.4 / 29.4 / 29.4, 54 / 29.7 / 29.8, 196 / 35.4 / 35.5, 380 / 68 / 45.  256 experts, 8 choices: 9.4 / 10.4 / 10.7, 15.3 / 11.2 / 11.6,
  // 58 / 15.4 / 15.9, 108 / 25.3 / 20.1; 2 and 32 alike.)
  const int ctas = a.rows <= 1024 ? 1 : a.rows <= 8192 ? 8 : group_ctas(dev);
  const int stretch = group_stretch(a.rows, ctas);
  const int staged = (int64_t)stretch * kGroupWarps * a.top_k <= kStaged;
  const dim3 cluster((unsigned)ctas);
  const size_t smem = (size_t)group_smem(a.experts, staged);
  return stretch == 32 ? launch_after<group_kernel<true>>(cluster, dim3(kGroupThreads), smem, cluster, s, a, staged)
                       : launch_after<group_kernel<false>>(cluster, dim3(kGroupThreads), smem, cluster, s, a, staged);
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
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {                               // no slots: what a call before left there is no grouping of this batch
    const size_t bytes = 4 * ((size_t)experts + 1);
    if (!offsets) return HAM_OK;
    if (!op_aligned(offsets, 4)) return op_fail(HAM_EINVAL, "pointers must be 4-byte aligned");
    if (op_overlap(offsets, bytes, bias, 4 * (size_t)experts)) return op_fail(HAM_EINVAL, "an output overlaps an input");
    const cudaError_t ce = cudaMemsetAsync(offsets, 0, bytes, s);
    return ce == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "route: %s", cudaGetErrorString(ce));
  }
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
  a.wide = f32 && experts % 4 == 0 && op_aligned(logits, 16);
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
  const cudaError_t ce = experts <= 32    ? ham::launch_route<1>(a, s)
                         : experts <= 64  ? ham::launch_route<2>(a, s)
                         : experts <= 128 ? ham::launch_route<4>(a, s)
                         : experts <= 256 ? ham::launch_route<8>(a, s)
                                          : ham::launch_route<16>(a, s);
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
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Two pieces of 16 bytes a thread for many rows, one for few (us with one / two: 8 rows of 8 x 4096 2.2 / 2.9, 4096 rows 48.8 /
  // 46.6, 8192 rows of 2 x 4096 44.5 / 37.1, of 4 x 2048 29.7 / 27.4; with four 51.5, 39.2 and 32.9).
  const cudaError_t ce = n % 8 == 0   ? (rows < 4 * ham::device_sms() ? ham::launch_combine<8, 1>(a, rows, f32, s)
                                                                      : ham::launch_combine<8, 2>(a, rows, f32, s))
                         : n % 2 == 0 ? ham::launch_combine<2, 4>(a, rows, f32, s)
                                      : ham::launch_combine<1, 4>(a, rows, f32, s);
  return ce == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "combine launch: %s", cudaGetErrorString(ce));
}

}  // extern "C"

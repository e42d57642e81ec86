// The choice of a token from a row of logits and a given random number: temperature, top-k, top-p and
// min-p, then the inverse of the running sum in index order.
//
//   w_i = trunc(2^31 exp((l_i - max l) / T))        a whole number: the token's weight
//   order: by l, largest first, equal ones by index
//   kept:  the first k; of these the shortest prefix whose weights reach p times the k's; of these
//          the ones with w_i >= min_p 2^31
//   token: the first index at which the running sum of the kept weights exceeds floor(u S), S their sum
//
// Sums are of whole numbers, so that neither the order of the additions nor the launch's shape can
// change an answer.  Weights are below one part in 2^31 of the likeliest token's where they are 0.
//
// A row is never sorted: histograms find where the order is cut, and the tokens next to the cut are listed
// and cut exactly.  Two kernels do this; the launch takes the second where many rows wait on one another.
//
// Few rows (sample_kernel): a row is held in the shared memory of a cluster of CTAs and read from global
// memory once.  A histogram over 512 bins of (max - l) / T, which grows as the order goes on, of counts (for
// top-k) or of counts and weights (top-p alone) finds the bin of the cut: every CTA adds up the cluster's
// histograms for itself, 16 bytes a load, so that this costs one cluster barrier (2048 bins, added up by
// shares and read back, took 8500 cycles against 3000).  Then
//  - where at most 2048 tokens lie up to that bin they are listed, in index order, in the first CTA's
//    shared memory; that CTA makes the exact cuts and picks the token;
//  - otherwise the bin's own tokens are listed there and the first CTA finds the cut among them for all
//    (where they too are more than 2048: histograms over 512 parts of the bin, then over the values of l
//    in the part until one is left); then the cluster sums the kept weights by stretches of the index.
// One row of 128256 fp32 logits takes 10.9 us (top-k and top-p), of which the reads are less than one: the rest is a chain of
// some ten barriers and shared-memory steps.
//
// Many rows (sample_alone_kernel): a CTA a row, two an SM, so that no row waits for a place in shared memory
// and no step for a cluster.  The first pass over the row, which the memory's rate bounds (23 us for 256 rows
// of 128256 in fp32, 19 at the rate of a copy), leaves the largest logit of each group of 128 (or 256)
// tokens; what comes after reads the groups that matter, from the L2 where they are still there:
//  - top-k: the groups whose largest logit is among the k largest of them, in whose bins the k tokens lie
//    (k = 50: 31 us in all, where the clusters took 106);
//  - larger k, and top-p alone: the first pass also counts tokens by finer bins, on a scale that does not need
//    the maximum.  For k they give the tokens to list (60 to 88 us; the shared atomics take 0.8 us a million).
//    For top-p they bound each bin's weight, which leaves the cut to a few bins, and one more pass sums
//    weights and lists the bins' tokens (86 us; clusters 195; histograms of all weights took 150);
//  - no cut: one more pass of exponentials, whose instructions bound it (52 us; clusters 77).
// A bound that does not hold is seen, exactly, and the row goes the way of the other kernel's steps.  (Two CTAs an SM
// leave 64 registers a thread, of which 88 bytes spill in fp32 and 136 in bf16, as ptxas reports them.)
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cmath>

#include "ham_mx.cuh"
#include "ham_ops.cuh"

namespace ham {
namespace {

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr int kBins = 512;
constexpr int kList = 2048;             // tokens that one CTA takes by itself
constexpr int kRanked = 128;            // ... that it compares with one another
constexpr float kFine = 2147483648.f;   // 2^31
constexpr float kLastBin = 511.f;
constexpr float kBinsPerX = 23.78f;     // bins of x = (l - max) / T: 511 reach to -21.4886, and below
                                        // -31 log 2 = -21.4876 a weight is 0
constexpr int kSampleMaxVocab = 1 << 18;
constexpr int kMaxCluster = 8;           // (8 CTAs hold the largest vocabulary in fp32)
constexpr int kSampleSmem = 220 * 1024, kSampleSmem2 = 112 * 1024;  // one and two CTAs an SM

struct SampleArgs {
  const void *logits;
  const float *u, *temperature, *top_p, *min_p;  // all but u nullable
  const int32_t *top_k;
  int32_t *tokens;
  float *probs;
  int vocab, slice;       // elements of a CTA, a multiple of 8
};

// Weights are added in two halves (weight = high 2^16 + low): at most 2^16 tokens of a CTA keep each
// half's sum within 32 bits.
constexpr int kSliceMost = 1 << 16;
struct __align__(16) Histogram { uint32_t count[kBins], low[kBins], high[kBins]; };

// Groups of a row that one CTA reads by itself: a vector a lane of a warp.  (The row's first vector may
// begin before the row.)
constexpr int kGroups = kSampleMaxVocab / 4 / 32 + 1;
constexpr int kCopies = 8;               // histograms of such a CTA, one for two warps
constexpr int kPart = 256;               // tokens that a warp of it lists at once
constexpr int kFineBins = 4096, kFineCopies = 3, kFineEach = kFineBins / 2 / kSampleThreads;
constexpr float kFinePerX = 4.f * kBinsPerX;
constexpr int kQuad = 4;                 // groups that a warp of it has on their way, and takes together
constexpr int kQuads = (kGroups + kQuad - 1) / kQuad;

// What a CTA shares with its cluster beside the logits.
struct SampleShared {
  Histogram h;
  __align__(16) float list_l[kList];      // the row's listed tokens, by index
  int32_t list_i[kList];
  uint32_t own[kGroups];                  // this CTA's: their places among its logits
  uint64_t sorted[kGroups];
  uint64_t total_mass, warp_mass[kSampleWarps];
  uint32_t warp_count[kSampleWarps];
  float best, warp_best[kSampleWarps];
  uint32_t key_max, key_min, warp_max[kSampleWarps], warp_min[kSampleWarps];
  uint64_t kept;
  uint32_t ties, warp_ties[kSampleWarps];
  int first;                              // first index of the largest logit
  uint64_t found_before_mass, found_mass, aim;
  uint32_t found_before_count, found_count;
  int found, members;
  float cut_value;
  uint32_t cut_ties, cut_same;
  uint64_t cut_key, cut_mass;
};
static_assert(kFineBins * kFineCopies * 4 <= sizeof(Histogram) * kCopies, "finer histogram");
static_assert(kQuads * 8 + kSampleWarps * kPart * 4 <= sizeof(Histogram) * kCopies, "lists");
static_assert(offsetof(SampleShared, sorted) + sizeof(SampleShared::sorted) - offsetof(SampleShared, list_l) >=
                  kSampleWarps * kQuad * 512, "the groups on their way");
static_assert(kQuad * 32 * 8 <= kSampleWarps * kPart, "a quad's tokens");
static_assert(kGroups >= kList && kGroups * 2 >= kSampleWarps * kPart, "lists");

// What a CTA that reads a row by itself has beside it.
struct RowShared {
  Histogram h[kCopies];
  uint32_t group_max[kGroups];            // keys of the groups' largest logits
  uint4 edge[2];                          // the first and the last vector, where they stick out of the row
};

__device__ __forceinline__ float load_logit(const float *p) { return *p; }
__device__ __forceinline__ float load_logit(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
// Keys in the order of the logits (-0 as 0).
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// A row's largest logit and temperature.  -x = (best - l) / t rounded to nearest as a division is: with r
// the rounded reciprocal of t, q = d r and its remainder d - q t (exact in a fused multiply-add), q + rem r
// rounds to the quotient (Markstein, IBM J. Res. Dev. 34, 1990).  Where a step leaves fp32's range the
// weight is right all the same: an x that underflows is one whose exponential is 1, and an overflow
// makes it NaN or -inf, which weigh 0, as a NaN logit does.
struct Scale {
  float best, t, r, bins;   // bins = kBinsPerX / t
};
__device__ __forceinline__ Scale scale_of(float best, float t) {
  t = fminf(fmaxf(t, 0x1p-60f), 0x1p60f);
  return Scale{best, t, __frcp_rn(t), __fdiv_rn(kBinsPerX, t)};
}
__device__ __forceinline__ uint32_t weight_of(float l, const Scale &c) {
  const float d = __fsub_rn(c.best, l), q = __fmul_rn(d, c.r);
  const float x = __fmaf_rn(__fmaf_rn(-q, c.t, d), c.r, q);
  return (uint32_t)(expf(-x) * kFine);           // (NaN: 0)
}
// Where l lies in the order, in bins (the fraction: the part of the bin); it grows as l falls, so bins
// and parts follow the order.  From kLastBin on weights are 0 and the token is left out, as is NaN.
__device__ __forceinline__ float place_of(float l, const Scale &c) { return __fmul_rn(__fsub_rn(c.best, l), c.bins); }
__device__ __forceinline__ bool has_bin(float place) { return place < kLastBin; }
__device__ __forceinline__ int part_of(float place, int bin) { return (int)((place - (float)bin) * (float)kBins); }

__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t a) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint4 ld_cluster_u32x4(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void cp_async16(uint4 *to, const uint4 *from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename T>
__device__ __forceinline__ float ld_cluster_logit(uint32_t a) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(ld_cluster_u32(a));
  uint16_t v;
  asm volatile("ld.shared::cluster.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return __uint_as_float((uint32_t)v << 16);
}
template <typename T>
__device__ __forceinline__ uint32_t peer(const T *p, int rank) { return cluster_map_shared(smem_u32(p), (uint32_t)rank); }

// Where the order is cut: kept are the logits above `value` and, of the ones equal to it, all or (with
// by_index) the first `ties` by index.
struct Cut {
  float value = -INFINITY;
  bool by_index = false;
  uint32_t ties = 0;
  uint64_t mass = 0;       // weight of what is kept
};
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}

// Inclusive running sums of a weight over the block's threads, in thread order; `all`: their sum.
__device__ __forceinline__ uint64_t block_scan(SampleShared &s, uint64_t mass, uint64_t &all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t m = __shfl_up_sync(kFull, mass, o);
    if (lane >= o) mass += m;
  }
  __syncthreads();                               // (the array's last readers are done)
  if (lane == 31) s.warp_mass[warp] = mass;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int q = 0; q < kSampleWarps; ++q) {
    if (q == warp) mass += all;
    all += s.warp_mass[q];
  }
  return mass;
}

// A warp's view of one value of each CTA of the cluster: lane q holds that of CTA q (0 past them).
__device__ __forceinline__ uint32_t sum8(uint32_t v) { return __reduce_add_sync(kFull, v); }
__device__ __forceinline__ uint64_t sum8(uint64_t v) {
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return __shfl_sync(kFull, v, 0);
}

// A vector of 16 bytes of logits.
template <typename T>
struct Vec {
  static constexpr int kN = 16 / (int)sizeof(T);
  float l[kN];
  __device__ __forceinline__ explicit Vec(const uint4 &v) {
    const T *e = reinterpret_cast<const T *>(&v);
#pragma unroll
    for (int j = 0; j < kN; ++j) l[j] = load_logit(e + j);
  }
  // (fmaxf and fminf pass over NaN)
  __device__ __forceinline__ float largest() const {
    float m = l[0];
#pragma unroll
    for (int j = 1; j < kN; ++j) m = fmaxf(m, l[j]);
    return m;
  }
  __device__ __forceinline__ float smallest() const {
    float m = l[0];
#pragma unroll
    for (int j = 1; j < kN; ++j) m = fminf(m, l[j]);
    return m;
  }
};

constexpr float kWhole = 12582912.f;     // 1.5 2^23

template <typename T, bool kAlone>
struct Row {
  static constexpr int kN = Vec<T>::kN;
  SampleShared &s;
  uint4 *data;             // this CTA's logits (-inf before and after them)
  int first_index;         // index of the first vector's first element (slice further on in the next CTA)
  int slice, vecs, ctas, rank, tid;
  Scale c;
  // kAlone: the row stays in global memory, and this CTA reads it in groups, a warp a run of them
  RowShared *w;
  const uint4 *from;       // the row's vectors, of which whole0 .. whole1 - 1 lie in it whole
  int whole0, whole1, groups, g0, g1;
  bool infinite;           // the largest logit is: those like it are as likely as one another, nothing else is

  __device__ void sync() const {
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
  }
  template <typename V>
  __device__ __forceinline__ uint32_t lane32(const V *p) const {
    const int q = tid & 31;
    return q < ctas ? ld_cluster_u32(peer(p, q)) : 0u;
  }
  __device__ __forceinline__ uint64_t lane64(const uint64_t *p) const {
    const int q = tid & 31;
    return q < ctas ? ld_cluster_u64(peer(p, q)) : 0ull;
  }
  __device__ __forceinline__ Histogram &hist() const {
    if constexpr (kAlone) return w->h[tid >> 6];
    return s.h;
  }
  __device__ __forceinline__ uint4 vector(int v) const {
    if (v >= whole0 && v < whole1) return __ldg(from + v);
    const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    return v < vecs ? w->edge[v > 0] : make_uint4(none, none, none, none);
  }
  __device__ __forceinline__ Vec<T> logits(const uint4 &v) const {
    Vec<T> x(v);
    if (infinite)
#pragma unroll
      for (int j = 0; j < kN; ++j) x.l[j] = x.l[j] == INFINITY ? 0.f : -INFINITY;
    return x;
  }
  __device__ __forceinline__ float logit_at(int place) const {
    const int v = place / kN;
    const uint4 *x = v >= whole0 && v < whole1 ? from + v : &w->edge[v > 0];
    const float l = load_logit(reinterpret_cast<const T *>(x) + place % kN);
    return !infinite ? l : l == INFINITY ? 0.f : -INFINITY;
  }
  // For this warp's quads of groups, any of which has want(group): f(group, vector) for the four, then
  // end(quad); all lanes together.  The groups come through shared memory (the lists' place), a quad on
  // its way and each lane's vector by itself.  Every other pass goes down: what was read last is still in
  // the L2.
  template <bool kDown, typename P, typename F, typename E>
  __device__ __forceinline__ void run(P want, F f, E end) const {
    const int lane = tid & 31;
    uint4 *ring = reinterpret_cast<uint4 *>(s.list_l) + (tid >> 5) * kQuad * 32 + lane;
    int b = kDown ? (g1 - g0 + 31) / 32 * 32 : -32;   // of the next quad: its window of 32 groups,
    uint32_t mask = 0;                                // and the window's quads from it on
    const auto next = [&]() {
      while (!mask) {
        b += kDown ? -32 : 32;
        if (kDown ? b < 0 : b >= g1 - g0) return -1;
        const int g = g0 + b + lane;
        mask = __ballot_sync(kFull, g < g1 && want(g));
        mask = (mask | mask >> 1 | mask >> 2 | mask >> 3) & 0x11111111u;
      }
      const int at = kDown ? 31 - __clz(mask) : __ffs(mask) - 1;
      mask ^= 1u << at;
      return g0 + b + at;
    };
    const auto load = [&](int g, int i) {
      if (g >= 0) {
        const int v = (g + i) * 32 + lane;
        if (v >= whole0 && v < whole1) cp_async16(ring + i * 32, from + v);
        else ring[i * 32] = vector(v);
      }
      cp_async_commit();
    };
    int g = next();
#pragma unroll
    for (int i = 0; i < kQuad; ++i) load(g, kDown ? kQuad - 1 - i : i);
    while (g >= 0) {
      const int then = next();
#pragma unroll
      for (int n = 0; n < kQuad; ++n) {
        const int i = kDown ? kQuad - 1 - n : n;
        cp_async_wait<kQuad - 1>();
        f(g + i, logits(ring[i * 32]));
        load(then, i);
      }
      end(g / kQuad);
      g = then;
    }
    cp_async_wait<0>();
  }
  // f(group, vector) for the few of this warp's groups for which want(group), four at once; the lists
  // stay as they are.
  template <typename P, typename F>
  __device__ __forceinline__ void run_few(P want, F f) const {
    const int lane = tid & 31;
    for (int b = 0; b < g1 - g0; b += 32) {
      const int mine = g0 + b + lane;
      uint32_t mask = __ballot_sync(kFull, mine < g1 && want(mine));
      while (mask) {
        constexpr int kAtOnce = 4;
        int g[kAtOnce];
        uint4 v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j, mask &= mask - 1) g[j] = mask ? g0 + b + __ffs(mask) - 1 : -1;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
          if (g[j] >= 0) v[j] = vector(g[j] * 32 + lane);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
          if (g[j] >= 0) f(g[j], logits(v[j]));
      }
    }
  }
  __device__ __forceinline__ float max_of(int g) const { return logit_of(w->group_max[g]); }
  // f(vector) for every vector of this CTA's logits that has a weight, in any order.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if constexpr (kAlone) {
      run<true>([&](int g) { return has_bin(place_of(max_of(g), c)); }, [&](int, const Vec<T> &x) { f(x); }, [](int) {});
    } else {
#pragma unroll 2
      for (int v = tid; v < vecs; v += kSampleThreads) f(Vec<T>(data[v]));
    }
  }
  // This thread's stretch of the vectors: the threads' stretches follow one another in index order.  (An
  // odd number of vectors each, so that a warp's loads of 16 bytes fall on different banks.)
  __device__ __forceinline__ void stretch(int &v0, int &v1) const {
    const int per = ((vecs + kSampleThreads - 1) / kSampleThreads) | 1;
    v0 = min(vecs, tid * per);
    v1 = min(vecs, v0 + per);
  }
  // The vectors of this thread's stretch (bit i: vector v0 + i) for which pred(vector).
  template <typename P>
  __device__ __forceinline__ uint32_t which(P pred) const {
    int v0, v1;
    stretch(v0, v1);
    uint32_t mask = 0;
#pragma unroll 2
    for (int v = v0; v < v1; ++v) mask |= (uint32_t)pred(Vec<T>(data[v])) << (v - v0);
    return mask;
  }
  // The histogram of the logits by bin(place, l) where in(place, l), of counts and / or weights.
  // Computed for the whole vector first: a vector's chains of arithmetic overlap.
  template <bool kMasses, typename I, typename B>
  __device__ __forceinline__ void histogram(I in, B bin) const {
    Histogram &h = hist();
    each([&](const Vec<T> &x) {
      float f[kN];
      uint32_t w[kN];
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        f[j] = place_of(x.l[j], c);
        if (kMasses) w[j] = weight_of(x.l[j], c);
      }
#pragma unroll
      for (int j = 0; j < kN; ++j)
        if (in(f[j], x.l[j])) {
          const int b = bin(f[j], x.l[j]);
          atomicAdd(&h.count[b], 1u);
          if (kMasses) add_mass(h, b, w[j]);
        }
    });
  }
  template <bool kMasses>
  __device__ __forceinline__ void histogram_of_bins() const {
    histogram<kMasses>([](float f, float) { return has_bin(f); }, [](float f, float) { return (int)f; });
  }
  __device__ void clear(Histogram *h, int many) const {
    uint4 *p = reinterpret_cast<uint4 *>(h);
    for (int i = tid; i < many * (int)(sizeof(Histogram) / 16); i += kSampleThreads) p[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  __device__ void clear() const {
    if constexpr (kAlone) clear(w->h, kCopies);
    else clear(&s.h, 1);
  }
  __device__ __forceinline__ void add_mass(Histogram &h, int bin, uint32_t w) const {
    atomicAdd(&h.low[bin], w & 0xffffu);
    if (w >> 16) atomicAdd(&h.high[bin], w >> 16);
  }
  // The share of a row's weight that top-p reaches for: whole numbers from here on (a sum reaches the
  // fp64 product if it reaches the whole number above).
  static __device__ uint64_t aim_of(double p, uint64_t mass) { return (uint64_t)ceil(fmax(p * (double)mass, 1.)); }
  // The first bin at which the running count (or weight) of the whole row's histogram, begun at the
  // given sums, reaches the aim (p > 0: the aim is that share of the row's weight, left in s.aim);
  // s.found (-1: none), its own and the earlier sums.  All CTAs of the cluster call it; the histograms
  // must stand until their next barrier.
  __device__ void find(bool by_mass, bool masses, uint32_t count0, uint64_t mass0, uint64_t aim, double p = 0.) const {
    sync();                                      // every CTA's histogram is complete
    constexpr int kThreads = kBins / 4;          // four bins a thread; a group of threads a histogram
    static_assert(kThreads % 32 == 0 && 3 * kThreads <= kSampleThreads && 2 * kBins <= kList, "threads");
    const int lane = tid & 31, warp = tid >> 5, group = tid / kThreads, quad = tid % kThreads;
    uint64_t m4[4] = {0, 0, 0, 0}, m_sum = 0, mi = 0;
    uint32_t c4[4], c_sum = 0, ci = 0;
    if (group == 0 || (masses && group < 3)) {
      static_assert(kCopies == kMaxCluster, "histograms of a row");
      const int offset = (group == 0 ? 0 : group == 1 ? 2 : 1) * kBins + quad * 4;  // count, high, low
      uint4 v[kMaxCluster];
#pragma unroll
      for (int q = 0; q < kMaxCluster; ++q) {
        if constexpr (kAlone) v[q] = *reinterpret_cast<const uint4 *>(w->h[q].count + offset);
        else v[q] = q < ctas ? ld_cluster_u32x4(peer(s.h.count + offset, q)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int q = 0; q < kMaxCluster; ++q) m4[0] += v[q].x, m4[1] += v[q].y, m4[2] += v[q].z, m4[3] += v[q].w;
      if (group)
#pragma unroll
        for (int j = 0; j < 4; ++j) s.sorted[(group - 1) * kBins + quad * 4 + j] = m4[j];
    }
    if (masses) __syncthreads();
    if (tid < kThreads) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c4[j] = (uint32_t)m4[j], c_sum += c4[j];
        m4[j] = masses ? (s.sorted[quad * 4 + j] << 16) + s.sorted[kBins + quad * 4 + j] : 0;
        m_sum += m4[j];
      }
      ci = c_sum, mi = m_sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t c = __shfl_up_sync(kFull, ci, o);
        const uint64_t m = __shfl_up_sync(kFull, mi, o);
        if (lane >= o) ci += c, mi += m;
      }
      if (lane == 31) s.warp_count[warp] = ci, s.warp_mass[warp] = mi;
      if (tid == 0) s.found = -1;
    }
    __syncthreads();
    if (tid < kThreads) {
      uint32_t run_c = count0 + ci - c_sum;
      uint64_t run_m = mass0 + mi - m_sum, all = 0;
#pragma unroll
      for (int q = 0; q < kThreads / 32; ++q) {
        const uint64_t m = s.warp_mass[q];
        if (q < warp) run_c += s.warp_count[q], run_m += m;
        all += m;
      }
      if (p > 0.) aim = aim_of(p, all);
      if (tid == 0) s.total_mass = all, s.aim = aim;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t c1 = run_c + c4[j];
        const uint64_t m1 = run_m + m4[j];
        if ((by_mass ? m1 : c1) >= aim && (by_mass ? run_m : run_c) < aim) {
          s.found = tid * 4 + j;
          s.found_before_count = run_c, s.found_before_mass = run_m;
          s.found_count = c4[j], s.found_mass = m4[j];
        }
        run_c = c1, run_m = m1;
      }
    }
    __syncthreads();
  }
  // Largest and smallest key (of the row) among this CTA's kmax / kmin.
  __device__ void key_range(uint32_t &kmax, uint32_t &kmin) const {
    kmax = __reduce_max_sync(kFull, kmax);
    kmin = __reduce_min_sync(kFull, kmin);
    if ((tid & 31) == 0) s.warp_max[tid >> 5] = kmax, s.warp_min[tid >> 5] = kmin;
    __syncthreads();
    if (tid == 0) {
      for (int q = 1; q < kSampleWarps; ++q) kmax = max(kmax, s.warp_max[q]), kmin = min(kmin, s.warp_min[q]);
      s.key_max = kmax, s.key_min = kmin;
    }
    sync();
    kmax = __reduce_max_sync(kFull, lane32(&s.key_max));
    kmin = __reduce_min_sync(kFull, (tid & 31) < ctas ? lane32(&s.key_min) : 0xffffffffu);
    sync();                                      // (read before the next call writes them)
  }
  // The exact cut within the bin that find() gave for the aim, by histograms of the whole cluster.
  __device__ Cut cut_by_bins(bool by_mass, uint64_t aim) const {
    Cut k;
    const int b1 = s.found;
    uint32_t count = s.found_before_count;
    uint64_t mass = s.found_before_mass;
    sync();                                      // (before the histogram's next use)
    clear();                                     // parts of the bin
    histogram<true>([&](float f, float) { return has_bin(f) && (int)f == b1; },
                    [&](float f, float) { return part_of(f, b1); });
    find(by_mass, true, count, mass, aim);
    const int b2 = s.found;
    count = s.found_before_count, mass = s.found_before_mass;
    // values of l within the part, until one is left
    // (a part is 2^-9 of a bin, so that its ends are numbers of 18 bits)
    const float begin = (float)b1 + (float)b2 * (1.f / kBins), end = begin + 1.f / kBins;
    uint32_t lo = 0, hi = 0xffffffffu;
    for (;;) {
      uint32_t kmax = 0, kmin = 0xffffffffu;
      each([&](const Vec<T> &x) {
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const float f = place_of(x.l[j], c);
          const uint32_t key = key_of(x.l[j]);
          if (f >= begin && f < end && key >= lo && key <= hi) kmax = max(kmax, key), kmin = min(kmin, key);
        }
      });
      key_range(kmax, kmin);
      int shift = 0;
      while (((kmax - kmin) >> shift) >= (uint32_t)kBins) ++shift;
      clear();
      histogram<true>(
          [&](float f, float l) { return f >= begin && f < end && key_of(l) >= kmin && key_of(l) <= kmax; },
          [&](float, float l) { return (int)((kmax - key_of(l)) >> shift); });
      find(by_mass, true, count, mass, aim);
      count = s.found_before_count, mass = s.found_before_mass;
      const uint32_t bin = (uint32_t)s.found;
      if (shift == 0) {                          // one value, held by s.found_count tokens
        const uint32_t key = kmax - bin;
        const uint64_t many = s.found_count, w = s.found_mass / many;
        // (by weight: the fewest whose weights reach the aim; the bin's own do, so w > 0)
        const uint64_t keep = by_mass ? (aim - mass + w - 1) / w : aim - count;
        k.value = logit_of(key);
        k.ties = (uint32_t)keep;
        k.by_index = keep < many;
        k.mass = mass + keep * w;
        return k;
      }
      hi = kmax - (bin << shift);
      const uint32_t down = ((bin + 1) << shift) - 1;
      lo = kmax - kmin < down ? kmin : kmax - down;
    }
  }
  // Weight of l if the cut and min_p keep it (those equal to the cut's value too: where some of them are
  // cut off, the caller keeps the first by index).
  __device__ __forceinline__ uint32_t kept(const Cut &k, uint32_t least, float l) const {
    const uint32_t v = weight_of(l, c);
    return l >= k.value && v >= least ? v : 0u;
  }
  // Lists this CTA's tokens of the bins first .. last, by index; the row's number of them.  If that is at
  // most kList, pull() then makes the row's list.
  __device__ uint32_t list(int first, int last) const {
    const float begin = (float)first, end = (float)(last + 1);  // (last < 511: a token up to it has a bin)
    const auto in = [&](float l) {
      const float f = place_of(l, c);
      return f < end && f >= begin;
    };
    if constexpr (kAlone) {
      return list_alone([&](int g) { return place_of(max_of(g), c) < end; }, in);
    } else {
      // the vectors that may hold some, by their largest and smallest logits; then their tokens
      const uint32_t mask =
          first == 0 ? which([&](const Vec<T> &x) { return place_of(x.largest(), c) < end; })
                     : which([&](const Vec<T> &x) { return place_of(x.largest(), c) < end && place_of(x.smallest(), c) >= begin; });
      int v0, v1;
      stretch(v0, v1);
      uint32_t many = 0;
      for (uint32_t m = mask; m; m &= m - 1) {
        const Vec<T> x(data[v0 + __ffs(m) - 1]);
#pragma unroll
        for (int j = 0; j < kN; ++j) many += in(x.l[j]);
      }
      uint64_t cta;
      uint32_t at = (uint32_t)block_scan(s, many, cta) - many;
      if (tid == 0) s.ties = (uint32_t)cta;
      if (many && cta <= kList)
        for (uint32_t m = mask; m; m &= m - 1) {
          const int v = v0 + __ffs(m) - 1;
          const Vec<T> x(data[v]);
#pragma unroll
          for (int j = 0; j < kN; ++j)
            if (in(x.l[j])) s.own[at++] = v * kN + j;
        }
      sync();
      return sum8(lane32(&s.ties));
    }
  }
  // The same by one CTA: its row's list at once, where it has at most kList.  A warp notes the places of
  // its groups' tokens (from kPart on: finds them again when it knows where they go).
  template <typename P, typename I>
  __device__ uint32_t list_alone(P want, I in) const {
    const int lane = tid & 31, warp = tid >> 5;
    uint32_t *part = reinterpret_cast<uint32_t *>(s.sorted) + warp * kPart;
    uint32_t many = 0;                           // of the warp
    const auto note = [&](int g, const Vec<T> &x, auto to) {
      uint32_t mine = 0;
#pragma unroll
      for (int j = 0; j < kN; ++j) mine += in(x.l[j]);
      if (!__any_sync(kFull, mine)) return;
      uint32_t upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += v;
      }
      uint32_t at = many + upto - mine;
      if (mine)
#pragma unroll
        for (int j = 0; j < kN; ++j)
          if (in(x.l[j])) to(at++, (uint32_t)((g * 32 + lane) * kN + j), x.l[j]);
      many += __shfl_sync(kFull, upto, 31);
    };
    run_few(want, [&](int g, const Vec<T> &x) {
      note(g, x, [&](uint32_t at, uint32_t place, float) {
        if (at < (uint32_t)kPart) part[at] = place;
      });
    });
    __syncthreads();                             // (the counts' last readers are done)
    if (lane == 0) s.warp_count[warp] = many;
    __syncthreads();
    uint32_t all = 0, before = 0;
    for (int q = 0; q < kSampleWarps; ++q) {
      if (q < warp) before += s.warp_count[q];
      all += s.warp_count[q];
    }
    if (all > (uint32_t)kList) return all;
    if (many <= (uint32_t)kPart) {
      for (uint32_t i = lane; i < many; i += 32) {
        const uint32_t place = part[i];
        s.list_l[before + i] = logit_at((int)place);
        s.list_i[before + i] = first_index + (int)place;
      }
    } else {
      many = before;
      run_few(want, [&](int g, const Vec<T> &x) {
        note(g, x, [&](uint32_t at, uint32_t place, float l) {
          s.list_l[at] = l;
          s.list_i[at] = first_index + (int)place;
        });
      });
    }
    __syncthreads();
    return all;
  }
  // The CTAs' lists of list(), one after the other.
  __device__ void pull(uint32_t all) const {
    if (kAlone) return;
    uint32_t upto = lane32(&s.ties);             // lane q: the tokens of CTAs 0 .. q
#pragma unroll
    for (int o = 1; o < kMaxCluster; o <<= 1) {
      const uint32_t v = __shfl_up_sync(kFull, upto, o);
      if ((tid & 31) >= o) upto += v;
    }
    for (uint32_t i0 = 0; i0 < all; i0 += kSampleThreads) {
      const uint32_t i = i0 + tid;
      int q = 0;
      uint32_t before = 0;
#pragma unroll
      for (int p = 0; p < kMaxCluster - 1; ++p) {
        const uint32_t v = __shfl_sync(kFull, upto, p);
        if (p < ctas - 1 && i >= v) q = p + 1, before = v;
      }
      if (i < all) {
        const uint32_t place = ld_cluster_u32(peer(&s.own[i - before], q));
        s.list_l[i] = ld_cluster_logit<T>(peer(data, q) + place * (uint32_t)sizeof(T));
        s.list_i[i] = first_index + (q - rank) * slice + (int)place;
      }
    }
    __syncthreads();
  }
  // A listed token's place in the order: by l, largest first, equal ones by index; and which one it is.
  static_assert(kList <= 1 << 11 && kSampleMaxVocab <= 1 << 18, "keys");
  __device__ __forceinline__ uint64_t sort_key(int i) const {
    return ((uint64_t)~key_of(s.list_l[i]) << 32) | (uint32_t)(s.list_i[i] << 11 | i);
  }
  static __device__ __forceinline__ int listed_of(uint64_t key) { return (int)key & 2047; }
  __device__ __forceinline__ uint32_t listed_weight(int i) const { return weight_of(s.list_l[i], c); }
  // For a few keys of s.sorted: how many come before each in the order and their weights (s.own, of the list),
  // by comparing it with every other; as many threads a key as there are, of which the first has the key's
  // token `i` and the sums (else i = -1).  (Top-k 50 of one row: 10.5 us, 11.5 if they are sorted; top-k
  // 200: the same.)
  struct Rank {
    int i;
    uint32_t count;
    uint64_t mass, key;
  };
  __device__ Rank rank_of(int n) const {
    int lanes = 1;
    while (lanes < 32 && 2 * lanes * n <= kSampleThreads) lanes *= 2;
    const int i = tid / lanes, part = tid & (lanes - 1);
    Rank r{-1, 0, 0, 0};
    if (i < n) {
      r.key = s.sorted[i];
      for (int j = part; j < n; j += lanes) {
        const uint64_t other = s.sorted[j];
        if (other < r.key) ++r.count, r.mass += s.own[listed_of(other)];
      }
      if (part == 0) r.i = listed_of(r.key);
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
      r.count += __shfl_xor_sync(kFull, r.count, o);
      r.mass += __shfl_xor_sync(kFull, r.mass, o);
    }
    return r;
  }
  // Sorts the first `many` keys of s.sorted (by l, largest first, equal ones by place in the list): a
  // bitonic network, distances below a warp in registers, the others in shared memory.
  __device__ void sort(int many) const {
    uint64_t *key = s.sorted;
    int n = 32;
    while (n < many) n *= 2;
    for (int i = many + tid; i < n; i += kSampleThreads) key[i] = ~0ull;
    __syncthreads();
    for (int size = 32; size <= n; size *= 2) {
      for (int step = size / 2; step >= 32; step /= 2) {
        for (int q = tid; q < n / 2; q += kSampleThreads) {
          const int i = 2 * q - (q & (step - 1)), o = i + step;
          const uint64_t x = key[i], y = key[o];
          if ((x > y) == ((i & size) == 0)) key[i] = y, key[o] = x;
        }
        __syncthreads();
      }
      for (int i = tid; i < n; i += kSampleThreads) {  // (whole warps)
        uint64_t x = key[i];
        for (int sub = size == 32 ? 2 : size; sub <= size; sub *= 2)
          for (int step = min(sub / 2, 16); step > 0; step /= 2) {
            const uint64_t y = __shfl_xor_sync(kFull, x, step);
            const bool low = (i & step) == 0, up = (i & sub) == 0;
            if ((x > y) == (low == up)) x = y;
          }
        key[i] = x;
      }
      __syncthreads();
    }
  }
  // The exact cut among the `n` listed tokens, by this CTA alone: a histogram over 512 bins (`bins`; else
  // the cut is known to lie in bin `bin`), one over the 512 parts of the cut's bin, then the part's tokens
  // ranked or sorted.  count0, mass0: those of the tokens before bin `bin`; s.own: the list's weights.
  // s.cut_key: the last token kept.
  __device__ Cut cut_list(int n, bool bins, int bin, bool by_mass, uint64_t aim, uint32_t count0, uint64_t mass0) const {
    float base = (float)bin, mult = bins ? 1.f : (float)kBins;
    for (;;) {
      clear(&s.h, 1);
      for (int i = tid; i < n; i += kSampleThreads) {
        const float at = (place_of(s.list_l[i], c) - base) * mult;  // (exact)
        if (at >= 0.f && at < (float)kBins) {
          atomicAdd(&s.h.count[(int)at], 1u);
          add_mass(s.h, (int)at, s.own[i]);
        }
      }
      __syncthreads();
      // (at most 2^11 tokens of 2^31: count and weight in one number)
      const uint64_t mine = ((uint64_t)s.h.count[tid] << 48) + ((uint64_t)s.h.high[tid] << 16) + s.h.low[tid];
      uint64_t all;
      const uint64_t run = block_scan(s, mine, all), ran = run - mine;
      constexpr uint64_t kMass = (1ull << 48) - 1;
      const uint64_t upto = by_mass ? mass0 + (run & kMass) : count0 + (run >> 48);
      const uint64_t before = by_mass ? mass0 + (ran & kMass) : count0 + (ran >> 48);
      if (upto >= aim && before < aim) {
        s.found = tid;
        s.found_before_count = count0 + (uint32_t)(ran >> 48), s.found_before_mass = mass0 + (ran & kMass);
      }
      if (tid == 0) s.members = 0;
      __syncthreads();
      base += (float)s.found / mult;
      count0 = s.found_before_count, mass0 = s.found_before_mass;
      if (mult > 1.f) break;
      mult = (float)kBins;
      __syncthreads();
    }
    const float end = base + 1.f / kBins;
    for (int i = tid; i < n; i += kSampleThreads) {
      const float f = place_of(s.list_l[i], c);
      if (f >= base && f < end) s.sorted[atomicAdd(&s.members, 1)] = sort_key(i);
    }
    __syncthreads();
    const int many = s.members;
    const auto cut_at = [&](uint64_t key, uint32_t w, uint64_t before, uint64_t mass) {
      if (before < aim && before + (by_mass ? w : 1u) >= aim) s.cut_key = key, s.cut_mass = mass + w;
    };
    if (many <= kRanked) {
      const Rank r = rank_of(many);
      if (r.i >= 0) cut_at(r.key, s.own[r.i], by_mass ? mass0 + r.mass : (uint64_t)count0 + r.count, mass0 + r.mass);
    } else {
      sort(many);
      uint64_t at = mass0;
      for (int i0 = 0; i0 < many; i0 += kSampleThreads) {
        const int i = i0 + tid;
        const uint64_t key = i < many ? s.sorted[i] : ~0ull;
        const uint32_t w = i < many ? s.own[listed_of(key)] : 0u;
        uint64_t part;
        const uint64_t before = at + block_scan(s, w, part) - w;
        if (i < many) cut_at(key, w, by_mass ? before : (uint64_t)count0 + i, before);
        at += part;
      }
    }
    if (tid == 0) s.cut_ties = s.cut_same = 0;
    __syncthreads();
    const uint64_t key = s.cut_key;              // its equals, and how many of them are kept
    for (int i = tid; i < many; i += kSampleThreads)
      if ((s.sorted[i] ^ key) >> 32 == 0) {
        atomicAdd(&s.cut_same, 1u);
        if (s.sorted[i] <= key) atomicAdd(&s.cut_ties, 1u);
      }
    if (tid == 0) s.cut_value = logit_of(~(uint32_t)(key >> 32));
    __syncthreads();
    return Cut{s.cut_value, s.cut_ties < s.cut_same, s.cut_ties, s.cut_mass};
  }
  // Leaves the listed tokens after the cut's without a weight.
  __device__ void drop(int n) const {
    for (int i = tid; i < n; i += kSampleThreads)
      if (sort_key(i) > s.cut_key) s.own[i] = 0;
    __syncthreads();
  }
  // The exact cut within the bin that find() gave for the aim, made by the first CTA for the cluster.
  __device__ Cut cut(bool by_mass, uint64_t aim) const {
    if (s.found_count > (uint32_t)kList) return cut_by_bins(by_mass, aim);
    const uint32_t count = s.found_before_count;
    const uint64_t mass = s.found_before_mass;
    const int bin = s.found;
    __syncthreads();
    const int many = (int)list(bin, bin);
    if (rank == 0) {
      pull(many);
      for (int i = tid; i < many; i += kSampleThreads) s.own[i] = listed_weight(i);  // (its places are pulled)
      cut_list(many, false, bin, by_mass, aim, count, mass);
    }
    sync();
    Cut k;
    k.value = __uint_as_float(ld_cluster_u32(peer(&s.cut_value, 0)));
    k.ties = ld_cluster_u32(peer(&s.cut_ties, 0));
    k.by_index = k.ties < ld_cluster_u32(peer(&s.cut_same, 0));
    k.mass = ld_cluster_u64(peer(&s.cut_mass, 0));
    return k;
  }
  // The choice among the first CTA's list of `all` tokens up to bin `last`, by that CTA alone.  k > 0:
  // top-k, which cuts in bin `last` (-1: not known), before which lie `before` tokens.  p >= 0: top-p, of the weight
  // `row_mass` (0: of the list's, after top-k).  Up to a token a thread are ranked or sorted; of more,
  // only the cuts' parts are.
  __device__ void choose(const SampleArgs &a, int row, int all, int last, uint32_t before, int k, double p,
                         uint64_t row_mass, uint32_t least) const {
    constexpr int kPer = kList / kSampleThreads;
    uint32_t *list_w = s.own;                    // (its places are pulled)
    uint64_t whole = row_mass;
    if (k > all) k = 0;
    if (all <= kSampleThreads) {
      if (tid < all) list_w[tid] = listed_weight(tid);
      if (tid < all) s.sorted[tid] = sort_key(tid);
      __syncthreads();
      Rank r;
      if (all <= kRanked) {
        r = rank_of(all);
      } else {
        sort(all);
        r.i = tid < all ? listed_of(s.sorted[tid]) : -1;
        r.count = (uint32_t)tid;
        const uint32_t w = r.i >= 0 ? list_w[r.i] : 0;
        uint64_t sum;
        r.mass = block_scan(s, w, sum) - w;
      }
      const uint32_t w = r.i >= 0 && (k <= 0 || (int)r.count < k) ? list_w[r.i] : 0;
      uint64_t sum, aim = ~0ull;
      block_scan(s, w, sum);
      if (p >= 0.) {
        if (tid == 0) s.aim = aim_of(p, row_mass ? row_mass : sum);
        __syncthreads();
        aim = s.aim;
      }
      if (r.i >= 0) list_w[r.i] = r.mass < aim ? w : 0u;
    } else {
      for (int i = tid; i < all; i += kSampleThreads) list_w[i] = listed_weight(i);
      __syncthreads();
      if (k > 0) {
        cut_list(all, last < 0, max(last, 0), false, (uint64_t)k, before, 0);
        drop(all);
      }
      if (p >= 0.) {
        if (!row_mass) {
          uint64_t mine = 0;
          for (int i = tid; i < all; i += kSampleThreads) mine += list_w[i];
          block_scan(s, mine, whole);
        }
        if (tid == 0) s.aim = aim_of(p, whole);
        __syncthreads();
        cut_list(all, true, 0, true, s.aim, 0, 0);
        drop(all);
      }
    }
    __syncthreads();
    uint64_t mass = 0;
    uint32_t w[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid * kPer + j;
      w[j] = i < all ? list_w[i] : 0u;
      if (w[j] < least) w[j] = 0;
      mass += w[j];
    }
    uint64_t sum = block_scan(s, mass, whole) - mass;
    if (tid == 0) s.aim = pick(a.u[row], whole);
    __syncthreads();
    const uint64_t aim = s.aim;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (sum <= aim && aim < sum + w[j]) {
        a.tokens[row] = s.list_i[tid * kPer + j];
        if (a.probs) a.probs[row] = (float)((double)w[j] / (double)whole);
      }
      sum += w[j];
    }
  }
  // Top-k (k > 0) and top-p (p >= 0) by the histograms of the bins, which are clear.  True: the tokens up to the cut are
  // few, and the first CTA has chosen among them; else where the order is cut.
  __device__ bool cuts(const SampleArgs &a, int row, int k, double p, uint32_t least, Cut &cut_at) const {
    const bool by_k = k > 0, by_p = p >= 0.;
    if (by_k) histogram_of_bins<false>();        // counts alone if top-k comes first
    else histogram_of_bins<true>();
    find(!by_k, !by_k, 0, 0, (uint64_t)k, by_k ? 0. : p);
    const bool all_in = s.found < 0;             // fewer than k tokens have any weight
    const int last = all_in ? kBins - 2 : s.found;
    const uint32_t before = all_in ? 0 : s.found_before_count;
    const uint64_t whole = by_k ? 0 : s.total_mass;
    uint64_t aim = s.aim;
    const uint32_t all = all_in ? kList : before + s.found_count;
    if (all <= (uint32_t)kList) {
      const uint32_t listed = list(0, last);
      if (listed <= (uint32_t)kList) {           // (all_in: known only now)
        if (rank == 0) pull(listed);
        if (ctas > 1) cluster_arrive();          // (the others' lists are pulled)
        if (rank == 0) choose(a, row, (int)listed, last, before, all_in ? 0 : k, p, whole, least);
        if (ctas > 1) cluster_wait();
        return true;
      }
    }
    if (by_k) {
      if (by_p) {                                // (top-p wants the weight that top-k keeps)
        sync();
        clear();
        histogram_of_bins<true>();
        find(false, true, 0, 0, (uint64_t)k);
      }
      if (!all_in) cut_at = cut(false, (uint64_t)k);
      if (by_p) {
        aim = aim_of(p, all_in ? s.total_mass : cut_at.mass);
        sync();
        clear();
        histogram_of_bins<true>();
        find(true, true, 0, 0, aim);
      }
    }
    if (by_p) cut_at = cut(true, aim);
    return false;
  }
  // Turns the quads' numbers into the running sums before them; their sum.
  template <typename N>
  __device__ uint64_t sum_before(N *of) const {
    const int quads = (groups + kQuad - 1) / kQuad, per = (quads + kSampleThreads - 1) / kSampleThreads;
    const int i0 = min(quads, tid * per), i1 = min(quads, i0 + per);
    uint64_t mine = 0, all;
    for (int i = i0; i < i1; ++i) mine += of[i];
    uint64_t at = block_scan(s, mine, all) - mine;
    for (int i = i0; i < i1; ++i) {
      const N v = of[i];
      of[i] = (N)at;
      at += v;
    }
    __syncthreads();
    return all;
  }
  // The quad in which the running sum of `mass` passes the aim of u, left in s.first, and the sum before
  // it; `mass` is turned into running sums.
  __device__ uint64_t find_quad(const SampleArgs &a, int row, uint64_t *mass, uint64_t &total) const {
    const int quads = (groups + kQuad - 1) / kQuad;
    total = sum_before(mass);
    if (tid == 0) s.aim = pick(a.u[row], total), s.first = 0;
    __syncthreads();
    const uint64_t aim = s.aim;
    for (int q = tid; q < quads; q += kSampleThreads)
      if (mass[q] <= aim && aim < (q + 1 < quads ? mass[q + 1] : total)) s.first = q;
    __syncthreads();
    return mass[s.first];
  }
  // A warp's sum of numbers below 2^36: two parts that 32 lanes add up in 32 bits.
  static __device__ __forceinline__ uint64_t warp_sum(uint64_t lanes) {
    const uint32_t low = __reduce_add_sync(kFull, (uint32_t)lanes & 0xffffffu);
    const uint32_t high = __reduce_add_sync(kFull, (uint32_t)(lanes >> 24));
    return ((uint64_t)high << 24) + low;
  }
  // The token of that quad, by one warp; weigh(group, vector, to): the kept weights of a lane's logits.
  template <typename W>
  __device__ void pick_of_quad(const SampleArgs &a, int row, uint64_t before, uint64_t total, W weigh) const {
    const int lane = tid & 31;
    const uint64_t aim = s.aim;
    uint4 v[kQuad];
#pragma unroll
    for (int i = 0; i < kQuad; ++i) v[i] = vector((s.first * kQuad + i) * 32 + lane);
#pragma unroll
    for (int i = 0; i < kQuad; ++i) {
      const int g = s.first * kQuad + i;
      uint32_t to[kN];
      weigh(g, logits(v[i]), to);
      uint64_t sum = 0;
#pragma unroll
      for (int j = 0; j < kN; ++j) sum += to[j];
      uint64_t at = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t u = __shfl_up_sync(kFull, at, o);
        if (lane >= o) at += u;
      }
      const uint64_t upto = before + __shfl_sync(kFull, at, 31);
      at += before - sum;
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        if (at <= aim && aim < at + to[j]) {
          a.tokens[row] = first_index + (g * 32 + lane) * kN + j;
          if (a.probs) a.probs[row] = (float)((double)to[j] / (double)total);
        }
        at += to[j];
      }
      before = upto;
    }
  }
  // Which of the finer bins l lies in, on a scale that needs no row's maximum: the nearest whole number,
  // up to 2^22, in the low bits of a float (and itself, less 1.5 2^23).
  __device__ __forceinline__ static float fine_place(float l, float fine_bins) { return __fmaf_rn(l, fine_bins, kWhole); }
  // Tokens of the finer bin n below that of the largest logit (where they lie too low for a weight, those
  // may count as higher ones: the bins take turns).
  __device__ __forceinline__ uint32_t fine_count(float top, int n) const {
    const uint32_t *fine = reinterpret_cast<const uint32_t *>(w->h);
    uint32_t many = 0;
    for (int q = 0; q < kFineCopies; ++q) many += fine[q * kFineBins + ((__float_as_int(top) - n) & (kFineBins - 1))];
    return many;
  }
  __device__ __forceinline__ bool has_fine_bins(float fine_bins) const { return fabsf(c.best * fine_bins) < 0x1p21f; }
  // The first of the block's numbers, a thread's, whose running sum reaches k; which one, and the sum
  // before it, in s.found and s.found_before_count, and with it in s.found_count.
  __device__ void first_to_reach(uint32_t k, uint32_t mine, uint32_t before) const {
    uint64_t all;
    const uint32_t upto = before + (uint32_t)block_scan(s, mine, all);
    if (tid == 0) s.found = -1;
    __syncthreads();
    if (upto >= k && upto - mine < k) s.found = tid, s.found_before_count = upto - mine, s.found_count = upto;
    __syncthreads();
  }
  // Lists the row's tokens up to the finer bin of the k-th, or up to a 512th of it; their number.
  // 0: the bins do not tell it, or it is too many.
  __device__ uint32_t list_first(uint32_t k, float fine_bins) const {
    if (!has_fine_bins(fine_bins) || k > (uint32_t)kList) return 0;
    const float top = fine_place(c.best, fine_bins);
    uint32_t count[kFineEach], sum = 0;
#pragma unroll
    for (int j = 0; j < kFineEach; ++j) sum += count[j] = fine_count(top, kFineEach * tid + j);
    first_to_reach(k, sum, 0);
    if (s.found == tid) {
      uint32_t upto = s.found_before_count;
      bool found = false;
#pragma unroll
      for (int j = 0; j < kFineEach; ++j) {
        if (!found && upto + count[j] >= k) {
          found = true;
          s.members = kFineEach * tid + j;
          s.found_before_count = upto, s.found_count = upto + count[j];
        }
        upto += count[j];
      }
    }
    __syncthreads();
    // (the last bins may hold tokens that have no place among the others)
    if (s.found < 0 || s.members >= kFineBins / 2 - 8) return 0;
    const float bin = top - (float)s.members;
    uint32_t listed;
    if (s.found_count <= (uint32_t)kList) {
      const auto in = [&](float l) { return fine_place(l, fine_bins) >= bin; };
      listed = list_alone([&](int g) { return in(max_of(g)); }, in);
    } else {
      const uint32_t before = s.found_before_count;
      const float at = kWhole - bin;             // l's part of the bin: -1/2 .. 1/2
      const auto part = [&](float l) { return __fmaf_rn(l, fine_bins, at); };
      clear(&s.h, 1);
      run<true>([&](int g) { return fine_place(max_of(g), fine_bins) >= bin; }, [&](int, const Vec<T> &x) {
#pragma unroll
        for (int j = 0; j < kN; ++j)
          if (fine_place(x.l[j], fine_bins) == bin) atomicAdd(&s.h.count[min(max((int)((0.5f - part(x.l[j])) * (float)kBins), 0), kBins - 1)], 1u);
      }, [](int) {});
      __syncthreads();
      first_to_reach(k, s.h.count[tid], before);
      if (s.found < 0 || s.found_count > (uint32_t)kList) return 0;
      const float least = 0.5f - (float)(s.found + 1) / (float)kBins;
      const auto in = [&](float l) { return part(l) >= least; };
      listed = list_alone([&](int g) { return in(max_of(g)); }, in);
    }
    return listed >= k && listed <= (uint32_t)kList ? listed : 0u;
  }
  // Top-p alone.  The counts of the finer bins, taken as the row was read, bound each bin's weight from
  // both sides (by its ends' weights, 1.1% apart), and so the share of the row's weight up to each bin:
  // they leave the cut to a few bins.  One pass then sums the weights of the row, of its groups' tokens
  // above those bins, and lists the bins' own, among which the cut is made.  False, with nothing chosen:
  // the bounds do not hold the cut (fine_place out of range), or hold too many tokens.
  __device__ bool top_p(const SampleArgs &a, int row, double p, uint32_t least, float fine_bins) const {
    const int lane = tid & 31, warp = tid >> 5;
    if (!has_fine_bins(fine_bins)) return false;
    const float top = fine_place(c.best, fine_bins), over = __fmaf_rn(c.best, fine_bins, kWhole - top);
    // ---- the bounds
    float lo[kFineEach], hi[kFineEach], sum_lo = 0.f, sum_hi = 0.f;
#pragma unroll
    for (int j = 0; j < kFineEach; ++j) {
      const int n = kFineEach * tid + j;
      const uint32_t many = fine_count(top, n);
      const float d = (float)n + over + 0.5f;    // of the bin's far end
      sum_lo = lo[j] = sum_lo + (float)many * expf(-d / kFinePerX);
      sum_hi = hi[j] = sum_hi + (float)many * expf(-fmaxf(d - 1.f, 0.f) / kFinePerX);
    }
    float run_lo = sum_lo, run_hi = sum_hi;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float x = __shfl_up_sync(kFull, run_lo, o), y = __shfl_up_sync(kFull, run_hi, o);
      if (lane >= o) run_lo += x, run_hi += y;
    }
    if (lane == 31) s.warp_max[warp] = __float_as_uint(run_lo), s.warp_min[warp] = __float_as_uint(run_hi);
    if (tid == 0) s.key_min = s.key_max = kFineBins / 2 - 1;
    __syncthreads();
    float all_lo = 0.f, all_hi = 0.f;
    run_lo -= sum_lo, run_hi -= sum_hi;
    for (int q = 0; q < kSampleWarps; ++q) {
      const float x = __uint_as_float(s.warp_max[q]), y = __uint_as_float(s.warp_min[q]);
      if (q < warp) run_lo += x, run_hi += y;
      all_lo += x, all_hi += y;
    }
    constexpr float kSlack = 4e-6f;              // for these sums' rounding
#pragma unroll
    for (int j = kFineEach - 1; j >= 0; --j) {
      const float l = run_lo + lo[j], h = run_hi + hi[j];
      if (h >= ((float)p - kSlack) * (h + fmaxf(all_lo - l, 0.f))) atomicMin(&s.key_min, (uint32_t)(kFineEach * tid + j));
      if (l >= ((float)p + kSlack) * (l + fmaxf(all_hi - h, 0.f))) atomicMin(&s.key_max, (uint32_t)(kFineEach * tid + j));
    }
    __syncthreads();                             // (and the bins are read)
    const float above = top - (float)s.key_min + 1.f, from_bin = top - (float)s.key_max;
    // ---- the pass; a warp's list is filled from its end, as its groups go down
    uint64_t *mass = reinterpret_cast<uint64_t *>(w->h);
    uint32_t *part = reinterpret_cast<uint32_t *>(mass + kQuads) + warp * kPart;
    for (int q = tid; q < kQuads; q += kSampleThreads) mass[q] = 0;
    __syncthreads();
    uint64_t whole = 0, upper = 0, sum = 0;
    uint32_t many = 0;
    run<true>([&](int g) { return weight_of(max_of(g), c) > 0; }, [&](int g, const Vec<T> &x) {
      uint32_t mine = 0;
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const uint32_t v = weight_of(x.l[j], c);
        const float f = fine_place(x.l[j], fine_bins);
        whole += v;
        if (f >= above) {
          upper += v;
          if (v >= least) sum += v;
        } else {
          mine += f >= from_bin;
        }
      }
      if (!__any_sync(kFull, mine)) return;
      uint32_t after = mine;                     // of this lane and those after it
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_down_sync(kFull, after, o);
        if (lane + o < 32) after += v;
      }
      uint32_t at = many + after;
      if (mine)
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const float f = fine_place(x.l[j], fine_bins);
          if (f < above && f >= from_bin) {
            if (at <= (uint32_t)kPart) part[kPart - at] = (uint32_t)((g * 32 + lane) * kN + j);
            --at;
          }
        }
      many += __shfl_sync(kFull, after, 0);
    }, [&](int q) {
      const uint64_t all = warp_sum(sum);
      if (lane == 0) mass[q] = all;
      sum = 0;
    });
    // ---- the row's list, and its sums
    if (lane == 0) s.warp_count[warp] = many;
    uint64_t row_mass, upper_mass;
    block_scan(s, whole, row_mass);
    block_scan(s, upper, upper_mass);
    uint32_t all = 0, before = 0, longest = 0;
    for (int q = 0; q < kSampleWarps; ++q) {
      const uint32_t v = s.warp_count[q];
      if (q < warp) before += v;
      all += v;
      longest = max(longest, v);
    }
    if (longest > (uint32_t)kPart || all > (uint32_t)kList) return false;
    uint32_t *list_w = s.own;
    uint64_t listed = 0;
    for (uint32_t i = lane; i < many; i += 32) {
      const uint32_t place = part[kPart - many + i];
      const float l = logit_at((int)place);
      const uint32_t v = weight_of(l, c);
      s.list_l[before + i] = l;
      s.list_i[before + i] = (int)place;
      list_w[before + i] = v;
      listed += v;
    }
    uint64_t list_mass;
    block_scan(s, listed, list_mass);
    const uint64_t aim = aim_of(p, row_mass);
    if (upper_mass >= aim || upper_mass + list_mass < aim) return false;
    __syncthreads();
    cut_list((int)all, true, 0, true, aim, 0, upper_mass);
    drop((int)all);
    constexpr int kTokens = kQuad * 32 * kN;
    for (int i = tid; i < (int)all; i += kSampleThreads)
      if (list_w[i] >= max(least, 1u))
        atomicAdd(reinterpret_cast<unsigned long long *>(mass + s.list_i[i] / kTokens), (unsigned long long)list_w[i]);
    __syncthreads();
    // ---- the quad, and in it the token
    uint64_t total;
    const uint64_t ahead = find_quad(a, row, mass, total);
    uint32_t *of_quad = part - warp * kPart;     // the listed ones of the quad
    for (int i = tid; i < kTokens; i += kSampleThreads) of_quad[i] = 0;
    __syncthreads();
    for (int i = tid; i < (int)all; i += kSampleThreads)
      if (s.list_i[i] / kTokens == s.first && list_w[i] >= least) of_quad[s.list_i[i] % kTokens] = list_w[i];
    __syncthreads();
    if (warp == 0)
      pick_of_quad(a, row, ahead, total, [&](int g, const Vec<T> &x, uint32_t (&to)[kN]) {
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const uint32_t v = weight_of(x.l[j], c);
          to[j] = fine_place(x.l[j], fine_bins) >= above ? v >= least ? v : 0u
                                                         : of_quad[(g % kQuad * 32 + lane) * kN + j];
        }
      });
    return true;
  }
  // floor(u S), below S
  static __device__ uint64_t pick(float u, uint64_t whole) {
    const double v = fmin(fmax((double)u, 0.), 1.);  // (a NaN becomes 0)
    const uint64_t aim = (uint64_t)floor(v * (double)whole);
    return aim >= whole ? whole - 1 : aim;
  }
};

constexpr int kSampleFixed = (int)(sizeof(SampleShared) + 15) / 16 * 16;  // shared memory before the logits
static_assert(kBins == kSampleThreads, "a thread a bin");
constexpr int kAloneSmem = kSampleFixed + (int)sizeof(RowShared);
static_assert(kAloneSmem <= kSampleSmem2, "two CTAs an SM");

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SampleShared &s = *reinterpret_cast<SampleShared *>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = gridDim.x, rank = blockIdx.x, row = blockIdx.y;
  uint4 *store = reinterpret_cast<uint4 *>(smem_raw + kSampleFixed);
  const int begin = min(a.vocab, rank * a.slice), n = min(a.vocab, begin + a.slice) - begin;
  for (int i = tid; i < kBins; i += kSampleThreads) s.h.count[i] = s.h.low[i] = s.h.high[i] = 0;
  grid_dependency_wait();
  grid_launch_dependents();
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const float min_p = a.min_p ? a.min_p[row] : 0.f;
  // ---- the row's slice to shared memory at its own 16-byte phase, and the largest logit
  const T *src = static_cast<const T *>(a.logits) + (int64_t)row * a.vocab + begin;
  constexpr int kVec = Vec<T>::kN, kAtOnce = 8;
  const int phase = (int)(((uintptr_t)src & 15u) / sizeof(T));
  const int vecs = n > 0 ? (phase + n + kVec - 1) / kVec : 0;
  const int whole0 = phase ? 1 : 0, whole1 = (phase + n) / kVec;   // vectors inside the slice
  const uint4 *from = reinterpret_cast<const uint4 *>(src - phase);  // (read from whole0 on)
  float best = -INFINITY;
  for (int i0 = whole0 + tid; i0 < whole1; i0 += kAtOnce * kSampleThreads) {
    uint4 v[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (i0 + j * kSampleThreads < whole1) v[j] = __ldcs(from + i0 + j * kSampleThreads);
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (i0 + j * kSampleThreads < whole1) {
        store[i0 + j * kSampleThreads] = v[j];
        best = fmaxf(best, Vec<T>(v[j]).largest());
      }
  }
  if (tid < 2 * kVec) {                          // the first and the last vector, where they stick out
    const int v = tid < kVec ? 0 : vecs - 1, i = v * kVec + tid % kVec - phase;
    if (vecs > 0 && (v < whole0 || v >= whole1)) {
      const float x = i >= 0 && i < n ? load_logit(src + i) : -INFINITY;
      best = fmaxf(best, x);
      T *to = reinterpret_cast<T *>(store) + v * kVec + tid % kVec;
      if constexpr (sizeof(T) == 4) *to = x;
      else *to = (T)(__float_as_uint(x) >> 16);
    }
  }
  best = warp_max_f32(best);
  if (lane == 0) s.warp_best[warp] = best;
  __syncthreads();
  best = warp_max_f32(lane < kSampleWarps ? s.warp_best[lane] : -INFINITY);
  if (tid == 0) s.best = best;
  Row<T, false> r{s, store, rank * a.slice - phase, a.slice, vecs, ctas, rank, tid, Scale{}, nullptr, nullptr, 0, 0, 0, 0, 0, false};
  r.sync();
  best = warp_max_f32(lane < ctas ? __uint_as_float(r.lane32(&s.best)) : -INFINITY);
  const bool greedy = !(temperature > 0.f);
  if (best == INFINITY) {                        // as likely as one another, and nothing else is
    best = 0.f;
    T *l = reinterpret_cast<T *>(store);
    for (int i = tid; i < vecs * kVec; i += kSampleThreads) {
      const uint32_t to = load_logit(l + i) == INFINITY ? 0u : 0xff800000u;
      if constexpr (sizeof(T) == 4) l[i] = __uint_as_float(to);
      else l[i] = (T)(to >> 16);
    }
    __syncthreads();
  }
  r.c = scale_of(best, greedy ? 1.f : temperature);
  if (best == -INFINITY || greedy) {             // (the same in every CTA of the cluster)
    int first = INT32_MAX;
    if (best != -INFINITY)
      for (int v = tid; v < vecs && first == INT32_MAX; v += kSampleThreads) {
        const Vec<T> x(store[v]);
#pragma unroll
        for (int j = kVec - 1; j >= 0; --j)
          if (x.l[j] == best) first = r.first_index + v * kVec + j;
      }
    first = __reduce_min_sync(kFull, first);
    if (lane == 0) s.warp_ties[warp] = (uint32_t)first;
    __syncthreads();
    first = __reduce_min_sync(kFull, lane < kSampleWarps ? (int)s.warp_ties[lane] : INT32_MAX);
    if (tid == 0) s.first = first;
    r.sync();
    if (rank == 0 && warp == 0) {
      first = __reduce_min_sync(kFull, lane < ctas ? (int)r.lane32(&s.first) : INT32_MAX);
      const bool none = best == -INFINITY;
      if (lane == 0) {
        a.tokens[row] = none ? -1 : first;
        if (a.probs) a.probs[row] = none ? 0.f : 1.f;
      }
    }
    r.sync();
    return;
  }
  const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
  const double share = by_p ? fmax((double)p, 0x1p-80) : 1.;  // (at least the likeliest token)
  // w >= min_p 2^31 for whole w (the product is exact in fp32): at least the whole number above
  const uint32_t least = min_p > 0.f ? (uint32_t)ceilf(fminf(min_p, 1.f) * kFine) : 0u;
  Cut cut;
  if ((by_k || by_p) && r.cuts(a, row, by_k ? k : 0, by_p ? share : -1., least, cut)) return;
  // ---- the kept weights of each thread's stretch of the slice, in index order
  uint32_t ties_before = 0, ties_mine = 0;
  if (cut.by_index) {
    int v0, v1;
    r.stretch(v0, v1);
    for (int v = v0; v < v1; ++v) {
      const Vec<T> x(store[v]);
#pragma unroll
      for (int j = 0; j < kVec; ++j) ties_mine += x.l[j] == cut.value;
    }
    uint64_t cta;
    ties_before = (uint32_t)block_scan(s, ties_mine, cta) - ties_mine;
    r.sync();                                    // (s.ties: its last readers are done)
    if (tid == 0) s.ties = (uint32_t)cta;
    r.sync();
    const uint32_t theirs = r.lane32(&s.ties);
    ties_before += sum8(lane < rank ? theirs : 0u);
  }
  int v0, v1;
  r.stretch(v0, v1);
  uint64_t sum = 0;
  if (cut.value == -INFINITY) {
    for (int v = v0; v < v1; ++v) {
      const Vec<T> x(store[v]);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const uint32_t w = weight_of(x.l[j], r.c);
        sum += w >= least ? w : 0u;
      }
    }
  } else {                                       // (few of a long row's: only their vectors are weighed)
    uint32_t ties = ties_before;
    for (uint32_t mask = r.which([&](const Vec<T> &x) { return x.largest() >= cut.value; }); mask; mask &= mask - 1) {
      const Vec<T> x(store[v0 + __ffs(mask) - 1]);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const uint32_t w = r.kept(cut, least, x.l[j]);
        if (!(cut.by_index && x.l[j] == cut.value && ties++ >= cut.ties)) sum += w;
      }
    }
  }
  uint64_t cta;
  uint64_t before = block_scan(s, sum, cta) - sum;
  if (tid == 0) s.kept = cta;
  r.sync();
  const uint64_t theirs = r.lane64(&s.kept), total = sum8(theirs);
  before += sum8(lane < rank ? theirs : (uint64_t)0);
  if (warp == 0) {
    const uint64_t v = Row<T, false>::pick(a.u[row], total);
    if (lane == 0) s.aim = v;
  }
  __syncthreads();
  const uint64_t aim = s.aim;
  // one thread of the cluster has the token in its stretch: its warp looks for it, a lane a logit
  const uint32_t owner = __ballot_sync(kFull, before <= aim && aim < before + sum);
  if (owner) {
    const int o = __ffs(owner) - 1;
    const int from = __shfl_sync(kFull, v0, o) * kVec, to = __shfl_sync(kFull, v1, o) * kVec;
    uint64_t at = __shfl_sync(kFull, before, o);
    uint32_t ties = __shfl_sync(kFull, ties_before, o);
    const T *logits = reinterpret_cast<const T *>(store);
    for (int i0 = from; i0 < to; i0 += 32) {
      const float l = i0 + lane < to ? load_logit(logits + i0 + lane) : -INFINITY;
      uint32_t w = r.kept(cut, least, l);
      if (cut.by_index) {
        const uint32_t equal = __ballot_sync(kFull, l == cut.value);
        if (l == cut.value && ties + __popc(equal & ((1u << lane) - 1u)) >= cut.ties) w = 0;
        ties += __popc(equal);
      }
      uint64_t run = w;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint64_t v = __shfl_up_sync(kFull, run, d);
        if (lane >= d) run += v;
      }
      const uint32_t over = __ballot_sync(kFull, at + run > aim);
      if (over) {
        if (lane == __ffs(over) - 1) {
          a.tokens[row] = r.first_index + i0 + lane;
          if (a.probs) a.probs[row] = (float)((double)w / (double)total);
        }
        break;
      }
      at += __shfl_sync(kFull, run, 31);
    }
  }
  r.sync();  // (a peer may still read this CTA's sums)
}

// The same choice with a row a CTA, two of them an SM.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_alone_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SampleShared &s = *reinterpret_cast<SampleShared *>(smem_raw);
  RowShared &w = *reinterpret_cast<RowShared *>(smem_raw + kSampleFixed);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.x;
  constexpr int kVec = Vec<T>::kN;
  {
    uint4 *p = reinterpret_cast<uint4 *>(w.h);
    for (int i = tid; i < (int)sizeof(w.h) / 16; i += kSampleThreads) p[i] = make_uint4(0, 0, 0, 0);
  }
  grid_dependency_wait();
  grid_launch_dependents();
  const T *src = static_cast<const T *>(a.logits) + (int64_t)row * a.vocab;
  const int phase = (int)(((uintptr_t)src & 15u) / sizeof(T));
  const int vecs = (phase + a.vocab + kVec - 1) / kVec, groups = (vecs + 31) / 32;
  const int per = (groups + kSampleWarps * kQuad - 1) / (kSampleWarps * kQuad) * kQuad;  // (whole quads)
  const int g0 = min(groups, warp * per), g1 = min(groups, g0 + per);
  Row<T, true> r{s, nullptr, -phase, 0, vecs, 1, 0, tid, Scale{}, &w, reinterpret_cast<const uint4 *>(src - phase),
                 phase ? 1 : 0, (phase + a.vocab) / kVec, groups, g0, g1, false};
  // the vectors that stick out of the row, by the warps that read them
  for (int e = 0; e < 2; ++e) {
    const int v = e ? vecs - 1 : 0, g = v / 32, i = v * kVec + lane - phase;
    if (g >= g0 && g < g1 && lane < kVec) {
      const float x = i >= 0 && i < a.vocab ? load_logit(src + i) : -INFINITY;
      T *to = reinterpret_cast<T *>(&w.edge[e]) + lane;
      if constexpr (sizeof(T) == 4) *to = x;
      else *to = (T)(__float_as_uint(x) >> 16);
    }
  }
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const float min_p = a.min_p ? a.min_p[row] : 0.f;
  const bool greedy = !(temperature > 0.f), by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
  // Top-k by the groups' largest logits or by the finer counts: 256 rows of 128256 fp32 logits (1002 groups), k = 50 34 /
  // 42 us, 250 47 / 52, 400 54 / 58, 600 63 / 62, 1000 132 / 69 (the list too long); in bf16 (501 groups), k = 200 39 / 46,
  // 400 50 / 54, 500 98 / 56.
  const bool fine = !greedy && (by_k ? 2 * (int64_t)k > groups : by_p);
  const float fine_bins = fine ? __fdiv_rn(kFinePerX, scale_of(0.f, temperature).t) : 0.f;
  uint32_t *const fine_counts = reinterpret_cast<uint32_t *>(w.h) + warp % kFineCopies * kFineBins;
  __syncthreads();
  // ---- the groups' largest logits, and the row's
  uint32_t most = 0;
  r.template run<false>([](int) { return true; }, [&](int g, const Vec<T> &x) {
    if (g >= groups) return;
    const uint32_t m = __reduce_max_sync(kFull, key_of(fmaxf(x.largest(), -INFINITY)));
    if (lane == 0) w.group_max[g] = m;
    most = max(most, m);
    if (fine) {                                  // (what lies too far below the largest so far has no weight)
      const float least_place = Row<T, true>::fine_place(logit_of(most), fine_bins) - (float)(kFineBins / 2);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float f = Row<T, true>::fine_place(x.l[i], fine_bins);
        if (f >= least_place) atomicAdd(fine_counts + (__float_as_int(f) & (kFineBins - 1)), 1u);
      }
    }
  }, [](int) {});
  if (lane == 0) s.warp_max[warp] = most;
  __syncthreads();
  most = __reduce_max_sync(kFull, lane < kSampleWarps ? s.warp_max[lane] : 0u);
  float best = logit_of(most);
  if (best == INFINITY) {                        // as likely as one another, and nothing else is
    best = 0.f;
    r.infinite = true;
    for (int g = tid; g < groups; g += kSampleThreads)
      w.group_max[g] = key_of(w.group_max[g] == most ? 0.f : -INFINITY);
    __syncthreads();
  }
  const bool none = best == -INFINITY;
  r.c = scale_of(best, greedy ? 1.f : temperature);
  if (none || greedy) {
    if (tid == 0) s.first = groups;
    __syncthreads();
    for (int g = tid; g < groups; g += kSampleThreads)
      if (logit_of(w.group_max[g]) == best) {
        atomicMin(&s.first, g);
        break;
      }
    __syncthreads();
    if (warp == 0) {
      int first = INT32_MAX;
      const Vec<T> x = r.logits(r.vector(s.first * 32 + lane));
#pragma unroll
      for (int j = kVec - 1; j >= 0; --j)
        if (x.l[j] == best) first = (s.first * 32 + lane) * kVec + j - phase;
      first = __reduce_min_sync(kFull, first);
      if (lane == 0) {
        a.tokens[row] = none ? -1 : first;
        if (a.probs) a.probs[row] = none ? 0.f : 1.f;
      }
    }
    return;
  }
  const double share = by_p ? fmax((double)p, 0x1p-80) : 1.;  // (at least the likeliest token)
  const uint32_t least = min_p > 0.f ? (uint32_t)ceilf(fminf(min_p, 1.f) * kFine) : 0u;
  Cut cut;
  if (by_k && !fine) {
    // k groups' largest logits are k tokens: what the row's k-th place is, or before it
    for (int g = tid; g < groups; g += kSampleThreads) {
      const float f = place_of(logit_of(w.group_max[g]), r.c);
      if (has_bin(f)) atomicAdd(&w.h[0].count[(int)f], 1u);
    }
    r.find(false, false, 0, 0, (uint64_t)k);
    if (s.found >= 0) {
      const uint32_t listed = r.list(0, s.found);
      if (listed <= (uint32_t)kList) {
        r.choose(a, row, (int)listed, -1, 0, k, by_p ? share : -1., 0, least);
        return;
      }
    }
    r.clear();
  }
  if (fine) {
    if (by_k) {
      const uint32_t listed = r.infinite ? 0u : r.list_first((uint32_t)k, fine_bins);
      if (listed) {
        r.choose(a, row, (int)listed, -1, 0, k, by_p ? share : -1., 0, least);
        return;
      }
    } else if (!r.infinite && r.top_p(a, row, share, least, fine_bins)) {
      return;
    }
    __syncthreads();
    r.clear();
  }
  if ((by_k || by_p) && r.cuts(a, row, by_k ? k : 0, by_p ? share : -1., least, cut)) return;
  // ---- the kept weights of each quad
  __syncthreads();                               // (what was here was read)
  uint64_t *mass = reinterpret_cast<uint64_t *>(w.h);
  uint32_t *ties = reinterpret_cast<uint32_t *>(mass + kQuads);
  const auto wanted = [&](int g) {
    const float m = r.max_of(g);
    return m >= cut.value && weight_of(m, r.c) >= max(least, 1u);
  };
  for (int q = tid; q < kQuads; q += kSampleThreads) mass[q] = 0, ties[q] = 0;
  __syncthreads();
  uint64_t sum = 0;
  const auto leave = [&](int q) {
    const uint64_t all = Row<T, true>::warp_sum(sum);
    if (lane == 0) mass[q] = all;
    sum = 0;
  };
  uint32_t tied = 0;                             // equals of the cut's value before the group
  const auto weigh = [&](int g, const Vec<T> &x, uint32_t (&to)[kVec]) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) to[j] = r.kept(cut, least, x.l[j]);
    if (cut.by_index) {                          // (all but the first of those by index are left out)
      uint32_t mine = 0;
#pragma unroll
      for (int j = 0; j < kVec; ++j) mine += x.l[j] == cut.value;
      uint32_t upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += v;
      }
      if (g % kQuad == 0) tied = ties[g / kQuad];
      uint32_t at = tied + upto - mine;
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (x.l[j] == cut.value && at++ >= cut.ties) to[j] = 0;
      tied += __shfl_sync(kFull, upto, 31);
    }
  };
  if (cut.value == -INFINITY && !least) {
    r.template run<true>(wanted, [&](int, const Vec<T> &x) {
#pragma unroll
      for (int j = 0; j < kVec; ++j) sum += weight_of(x.l[j], r.c);
    }, leave);
  } else {
    if (cut.by_index) {
      r.template run<false>(wanted, [&](int, const Vec<T> &x) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) tied += x.l[j] == cut.value;
      }, [&](int q) {
        tied = __reduce_add_sync(kFull, tied);
        if (lane == 0) ties[q] = tied;
        tied = 0;
      });
      __syncthreads();
      r.sum_before(ties);
    }
    r.template run<false>(wanted, [&](int g, const Vec<T> &x) {
      uint32_t to[kVec];
      weigh(g, x, to);
#pragma unroll
      for (int j = 0; j < kVec; ++j) sum += to[j];
    }, leave);
  }
  __syncthreads();
  // the quad in which the running sum passes the aim, and in it the token
  uint64_t total;
  const uint64_t before = r.find_quad(a, row, mass, total);
  if (warp == 0) r.pick_of_quad(a, row, before, total, weigh);
}

template <typename T>
cudaError_t launch_sample(SampleArgs a, int rows, cudaStream_t stream) {
  static bool done[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  // As many CTAs a row as find an SM each at once (of more than 1024 logits); where there are none that hold the
  // row, the fewest that leave room for two on an SM.  (us with 1, 2, 4, 8 CTAs a row: 8 x 32000 fp32, k 50, 11.3,
  // 10.5, 9.4, 9.3; 24 x 50001 fp32, p 0.9, -, 21.9, 18.9, 23.8; 40 x 50001 bf16, p 0.9 and flat, -, 27.0, 30.8, 42.2;
  // 76 x 32000 fp32, no cut, 9.4, 8.3, 12.7, 13.9; 100 x 32000 bf16, p 0.9, 22.4, 25.6, 33.0, 30.9; 32 x 128256 fp32, p
  // 0.9, four 25.3, eight 29.0; 38 rows, four 46.1, eight 42.3.)
  auto bytes = [&](int c) {
    return ((a.vocab + c - 1) / c + 7) / 8 * 8 * (int)sizeof(T) + 32 + kSampleFixed;
  };
  const int sms = device_sms();
  // (With a CTA an SM, clusters of four or eight find fewer places than there are SMs: a cluster lies within one group
  // of them.)
  const auto at_once = [&](int c) {
    return c <= 2 || bytes(c) <= kSampleSmem2 ? (int64_t)rows * c <= sms : (int64_t)rows * c * 16 <= sms * 15;
  };
  int ctas = kMaxCluster;
  while (ctas > 1 && (!at_once(ctas) || a.vocab <= 1024 * ctas)) ctas /= 2;
  if (!at_once(ctas) || bytes(ctas) > kSampleSmem || a.vocab > kSliceMost * ctas)
    for (ctas = 1; ctas < kMaxCluster && bytes(ctas) > kSampleSmem2;) ctas *= 2;
  a.slice = ((a.vocab + ctas - 1) / ctas + 7) / 8 * 8;
  if (dev < 0 || dev >= 64 || !done[dev]) {
    cudaError_t e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSampleSmem);
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(sample_alone_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAloneSmem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) done[dev] = true;
  }
  // A CTA a row where the clusters' CTAs would take turns: from one and a half times what the SMs hold at
  // once.  (fp32 rows of 128256: at 48, 384 CTAs, clusters / alone took 17 / 29 us without cuts, 26 / 20
  // with k = 50, 45 / 54 with p = 0.9; at 96 they took 31 / 32, 44 / 23 and 79 / 57.  A row that one CTA
  // holds waits for no other, and is read once: 1000 rows of 32000 in bf16, 40 / 53, 58 / 61, 105 / 115.  Rows of 50001
  // in fp32 and bf16: at 80, 160 CTAs, 15 / 18 and 13 / 21, 22 / 16 and 17 / 18, 35 / 34 and 34 / 37; at 160, 320 CTAs, 23 /
  // 25 and 18 / 24, 33 / 19 and 27 / 22, 52 / 47 and 49 / 47.)
  if (ctas > 1 && rows * ctas > 3 * sms)
    return launch_after<sample_alone_kernel<T>>(dim3((unsigned)rows), dim3(kSampleThreads), (size_t)kAloneSmem, dim3(1), stream, a);
  return launch_after<sample_kernel<T>>(dim3((unsigned)ctas, (unsigned)rows), dim3(kSampleThreads),
                      (size_t)bytes(ctas), dim3((unsigned)ctas), stream, a);
}

}  // namespace
}  // namespace ham

using ham::op_aligned;
using ham::op_fail;
using ham::op_overlap;

extern "C" int ham_sample(const void *logits, int32_t logits_dtype, int32_t rows, int32_t vocab, const float *u,
                          const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                          int32_t *tokens, float *probs, void *stream) {
  ham::ApiRange nvtx_range("ham_sample");
  if (logits_dtype != HAM_DTYPE_BF16 && logits_dtype != HAM_DTYPE_F32)
    return op_fail(HAM_EINVAL, "logits_dtype %d", logits_dtype);
  if (rows < 0 || rows > 65535) return op_fail(HAM_EINVAL, "rows %d outside 0..65535", rows);
  if (vocab < 1) return op_fail(HAM_EINVAL, "vocab %d is not positive", vocab);
  if (vocab > ham::kSampleMaxVocab)
    return op_fail(HAM_EUNSUPPORTED, "vocab %d above %d", vocab, ham::kSampleMaxVocab);
  if (rows == 0) return HAM_OK;
  if (!logits || !u || !tokens) return op_fail(HAM_EINVAL, "logits, u and tokens are required");
  if (!op_aligned(logits, 16)) return op_fail(HAM_EINVAL, "logits must be 16-byte aligned");
  for (const void *p : {(const void *)u, (const void *)temperature, (const void *)top_k, (const void *)top_p,
                        (const void *)min_p, (const void *)tokens, (const void *)probs})
    if (!op_aligned(p, 4)) return op_fail(HAM_EINVAL, "the per-row arrays must be 4-byte aligned");
  const size_t each = 4 * (size_t)rows, all = (size_t)rows * vocab * (logits_dtype == HAM_DTYPE_F32 ? 4 : 2);
  for (const void *out : {(const void *)tokens, (const void *)probs}) {
    for (const void *in : {(const void *)u, (const void *)temperature, (const void *)top_k, (const void *)top_p,
                           (const void *)min_p})
      if (op_overlap(out, each, in, each)) return op_fail(HAM_EINVAL, "an output overlaps an input");
    if (op_overlap(out, each, logits, all)) return op_fail(HAM_EINVAL, "an output overlaps an input");
  }
  if (op_overlap(tokens, each, probs, each)) return op_fail(HAM_EINVAL, "two outputs overlap");
  ham::SampleArgs a;
  a.logits = logits;
  a.u = u;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.tokens = tokens;
  a.probs = probs;
  a.vocab = vocab;
  a.slice = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = logits_dtype == HAM_DTYPE_F32 ? ham::launch_sample<float>(a, rows, s)
                                                      : ham::launch_sample<uint16_t>(a, rows, s);
  return e == cudaSuccess ? HAM_OK : op_fail(HAM_ECUDA, "sample launch: %s", cudaGetErrorString(e));
}

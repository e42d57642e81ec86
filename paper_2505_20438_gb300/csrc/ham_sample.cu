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
// A row is held in the shared memory of a cluster of CTAs and read from global memory once.  Nothing is
// sorted.  A histogram over 2048 bins of (max - l) / T, which grows as the order goes on, of counts (for
// top-k) or of weights (top-p alone) finds the bin in which the order is cut; every CTA sums its share
// of the bins over the cluster, so that this costs two cluster barriers.  Then
//  - where at most 2048 tokens lie up to that bin (the usual case) they are listed, in index order, in
//    the first CTA's shared memory, and that CTA makes the exact cuts, ranking only the tokens of the
//    cuts' bins against one another, and picks the token;
//  - otherwise the cluster goes on as a whole: histograms over 2048 parts of the bin, then over the
//    values of l in the part until one is left, whose equal tokens are kept by index; then the sums of
//    the kept weights by stretches of the index.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>

#include "ham_mx.cuh"
#include "ham_ops.cuh"

namespace ham {
namespace {

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr int kBins = 2048;
constexpr int kList = 2048;             // tokens that one CTA ranks by itself
constexpr float kFine = 2147483648.f;   // 2^31
constexpr float kLeast = -21.49f;       // below -31 log 2 = -21.4876 a weight is 0
constexpr float kBinsPerX = 95.25f;     // bins of x = (l - max) / T: 2047 reach beyond kLeast
constexpr float kLastBin = 2047.f;
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

struct Histogram { uint32_t count[kBins], low[kBins], high[kBins]; };  // weight = high 2^16 + low

// What a CTA shares with its cluster beside the logits and the running sums of its share of the bins.
struct SampleShared {
  Histogram h;
  float list_l[kList];                    // first CTA: the listed tokens, by index
  int32_t list_i[kList];
  uint64_t total_mass, warp_mass[kSampleWarps];
  uint32_t total_count, warp_count[kSampleWarps];
  float best, warp_best[kSampleWarps];
  uint32_t key_max, key_min, warp_max[kSampleWarps], warp_min[kSampleWarps];
  uint64_t kept, warp_kept[kSampleWarps];
  uint32_t ties, warp_ties[kSampleWarps];
  int first;                              // first index of the largest logit
  uint64_t found_before_mass, found_mass;
  uint32_t found_before_count, found_count;
  int found, members;
};

__device__ __forceinline__ float load_logit(const float *p) { return *p; }
__device__ __forceinline__ float load_logit(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
// NaN counts as ruled out; -0 as 0.
__device__ __forceinline__ float clean(float l) { return l != l ? -INFINITY : l + 0.f; }
// Keys in the order of the (cleaned) logits.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
// A row's temperature, and x = (l - best) / t rounded to nearest as a division is: with r the rounded
// reciprocal of t, q = a r and its remainder a - q t (exact in a fused multiply-add), q + rem r rounds
// to the quotient (Markstein, IBM J. Res. Dev. 34, 1990), in the range where nothing underflows.
struct Scale {
  float best, t, r, bins;   // bins = kBinsPerX / t
  bool plain;               // t within 2^-60 .. 2^60
};
__device__ __forceinline__ Scale scale_of(float best, float t) {
  return Scale{best, t, __frcp_rn(t), __fdiv_rn(kBinsPerX, t), t > 0x1p-60f && t < 0x1p60f};
}
__device__ __forceinline__ float x_of(float l, const Scale &c) {
  if (l == c.best) return 0.f;
  const float a = __fsub_rn(l, c.best);
  if (!c.plain || a > -0x1p-30f || a < -0x1p30f) return __fdiv_rn(a, c.t);
  const float q = __fmul_rn(a, c.r);
  return __fmaf_rn(__fmaf_rn(-q, c.t, a), c.r, q);
}
__device__ __forceinline__ uint32_t weight_of(float x) {
  return x >= kLeast ? (uint32_t)(expf(x) * kFine) : 0u;
}
// Where l lies in the order, in bins (the fraction: the part of the bin); it grows as l falls, so bins
// and parts follow the order.  From kLastBin on weights are 0 and the token is left out.
__device__ __forceinline__ float place_of(float l, const Scale &c) {
  return l == c.best ? 0.f : __fmul_rn(__fsub_rn(c.best, l), c.bins);
}
__device__ __forceinline__ bool has_bin(float place) { return place < kLastBin; }
__device__ __forceinline__ int part_of(float place, int bin) { return (int)((place - (float)bin) * (float)kBins); }

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t a) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t a, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
template <typename T>
__device__ __forceinline__ uint32_t peer(const T *p, int rank) { return cluster_map_shared(smem_u32(p), (uint32_t)rank); }

// Where the order is cut (depth 0: not at all): kept are the tokens of bins before b1, of b1 those of
// parts before b2, and of that part all (depth 2) or those with keys above `key` and the first `ties`
// by index of the ones equal to it (depth 3).
struct Cut {
  int depth = 0, b1 = 0, b2 = 0;
  uint32_t key = 0, ties = 0;
  uint64_t mass = 0;       // weight of what is kept
  bool by_index = false;   // some of the equal tokens are cut off
};

// Inclusive running sums over the block's threads, in thread order, of a count and a weight; the
// block's sums in `count_all`, `mass_all`.
__device__ __forceinline__ void block_scan(SampleShared &s, uint32_t &count, uint64_t &mass, uint32_t &count_all,
                                           uint64_t &mass_all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t c = __shfl_up_sync(kFull, count, o);
    const uint64_t m = __shfl_up_sync(kFull, mass, o);
    if (lane >= o) count += c, mass += m;
  }
  __syncthreads();                               // (the arrays' last readers are done)
  if (lane == 31) s.warp_count[warp] = count, s.warp_mass[warp] = mass;
  __syncthreads();
  count_all = 0, mass_all = 0;
#pragma unroll
  for (int q = 0; q < kSampleWarps; ++q) {
    if (q == warp) count += count_all, mass += mass_all;
    count_all += s.warp_count[q], mass_all += s.warp_mass[q];
  }
}

template <typename T>
struct Row {
  SampleShared &s;
  uint64_t *run_mass;      // running sums of this CTA's share of the bins
  uint32_t *run_count;
  const T *data;           // this CTA's logits
  int begin, n, ctas, rank, tid;
  Scale c;

  __device__ void sync() const {
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
  }
  __device__ __forceinline__ float logit(int i) const { return clean(load_logit(data + i)); }
  __device__ void clear() const {
    for (int i = tid; i < kBins; i += kSampleThreads) s.h.count[i] = s.h.low[i] = s.h.high[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void add_mass(int bin, uint32_t w) const {
    if (w & 0xffffu) atomicAdd(&s.h.low[bin], w & 0xffffu);
    if (w >> 16) atomicAdd(&s.h.high[bin], w >> 16);
  }
  __device__ __forceinline__ void add(int bin, uint32_t w) const {
    atomicAdd(&s.h.count[bin], 1u);
    add_mass(bin, w);
  }
  // The first bin at which the running count (or weight) of the whole row's histogram, begun at the
  // given sums, reaches the aim (aim_p > 0: that share of the row's weight, at least 1); s.found (-1:
  // none), its own and the earlier sums.  All CTAs of the cluster call it.
  __device__ void find(bool by_mass, uint64_t count0, uint64_t mass0, uint64_t aim_count, double aim_mass,
                       double aim_p = 0.) const {
    sync();                                      // every CTA's histogram is complete
    const int share = kBins / ctas, per = (share + kSampleThreads - 1) / kSampleThreads;
    uint32_t cn[4], cs = 0, ca;
    uint64_t m[4], ms = 0, ma;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      cn[j] = 0, m[j] = 0;
      const int i = tid * per + j;
      if (j < per && i < share) {
        const int bin = rank * share + i;
        uint64_t hi = 0, lo = 0;
#pragma unroll 4
        for (int q = 0; q < ctas; ++q) {
          cn[j] += ld_cluster_u32(peer(&s.h.count[bin], q));
          hi += ld_cluster_u32(peer(&s.h.high[bin], q));
          lo += ld_cluster_u32(peer(&s.h.low[bin], q));
        }
        m[j] = (hi << 16) + lo;
      }
      cs += cn[j], ms += m[j];
    }
    uint32_t cb = cs;
    uint64_t mb = ms;
    block_scan(s, cb, mb, ca, ma);
    cb -= cs, mb -= ms;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = tid * per + j;
      cb += cn[j], mb += m[j];
      if (j < per && i < share) run_count[i] = cb, run_mass[i] = mb;
    }
    if (tid == 0) {
      s.total_count = ca, s.total_mass = ma;
      s.found = -1;
    }
    sync();                                      // every CTA's running sums are complete
    uint32_t qc[kMaxCluster];
    uint64_t qm[kMaxCluster], all = 0;
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q) {
      qc[q] = 0, qm[q] = 0;
      if (q < ctas) {
        qc[q] = ld_cluster_u32(peer(&s.total_count, q));
        qm[q] = ld_cluster_u64(peer(&s.total_mass, q));
      }
      all += qm[q];
    }
    if (aim_p > 0.) aim_mass = fmax(aim_p * (double)all, 1.);
    uint64_t base_c = count0, base_m = mass0;
    int at = -1;
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q) {
      if (at < 0 && q < ctas) {
        if (by_mass ? (double)(base_m + qm[q]) >= aim_mass : base_c + qc[q] >= aim_count) at = q;
        else base_c += qc[q], base_m += qm[q];
      }
    }
    if (at >= 0)
      for (int i = tid; i < share; i += kSampleThreads) {
        const uint64_t c1 = base_c + ld_cluster_u32(peer(&run_count[i], at));
        const uint64_t m1 = base_m + ld_cluster_u64(peer(&run_mass[i], at));
        const uint64_t c0 = i ? base_c + ld_cluster_u32(peer(&run_count[i - 1], at)) : base_c;
        const uint64_t m0 = i ? base_m + ld_cluster_u64(peer(&run_mass[i - 1], at)) : base_m;
        const bool after = by_mass ? (double)m1 >= aim_mass : c1 >= aim_count;
        const bool before = by_mass ? !((double)m0 >= aim_mass) : c0 < aim_count;
        if (after && before) {
          s.found = at * share + i;
          s.found_before_count = (uint32_t)c0, s.found_before_mass = m0;
          s.found_count = (uint32_t)(c1 - c0), s.found_mass = m1 - m0;
        }
      }
    __syncthreads();
  }
  __device__ uint64_t whole_mass() const {       // after a find
    uint64_t all = 0;
    for (int q = 0; q < ctas; ++q) all += ld_cluster_u64(peer(&s.total_mass, q));
    return all;
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
    for (int q = 0; q < ctas; ++q) {
      const uint32_t a = ld_cluster_u32(peer(&s.key_max, q)), b = ld_cluster_u32(peer(&s.key_min, q));
      kmax = q ? max(kmax, a) : a;
      kmin = q ? min(kmin, b) : b;
    }
    sync();                                      // (read before the next call writes them)
  }
  // The exact cut within the bin that find() gave for the aim, by the whole cluster.
  __device__ Cut cut(bool by_mass, uint64_t aim_count, double aim_mass) const {
    Cut k;
    k.depth = 2, k.b1 = s.found;
    uint64_t count = s.found_before_count, mass = s.found_before_mass;
    __syncthreads();                             // (before the histogram's next use)
    sync();
    clear();                                     // parts of the bin
    for (int i = tid; i < n; i += kSampleThreads) {
      const float l = logit(i), f = place_of(l, c);
      if (has_bin(f) && (int)f == k.b1) add(part_of(f, k.b1), weight_of(x_of(l, c)));
    }
    __syncthreads();
    find(by_mass, count, mass, aim_count, aim_mass);
    k.b2 = s.found;
    k.mass = s.found_before_mass + s.found_mass;
    count = s.found_before_count, mass = s.found_before_mass;
    if (s.found_count == 1 || (!by_mass && count + s.found_count == aim_count)) return k;
    // values of l within the part, until one is left
    uint32_t lo = 0, hi = 0xffffffffu;
    for (;;) {
      uint32_t kmax = 0, kmin = 0xffffffffu;
      for (int i = tid; i < n; i += kSampleThreads) {
        const float l = logit(i), f = place_of(l, c);
        if (has_bin(f) && (int)f == k.b1 && part_of(f, k.b1) == k.b2) {
          const uint32_t key = key_of(l);
          if (key >= lo && key <= hi) kmax = max(kmax, key), kmin = min(kmin, key);
        }
      }
      key_range(kmax, kmin);
      int shift = 0;
      while (((kmax - kmin) >> shift) >= (uint32_t)kBins) ++shift;
      clear();
      for (int i = tid; i < n; i += kSampleThreads) {
        const float l = logit(i), f = place_of(l, c);
        if (has_bin(f) && (int)f == k.b1 && part_of(f, k.b1) == k.b2) {
          const uint32_t key = key_of(l);
          if (key >= kmin && key <= kmax) add((int)((kmax - key) >> shift), weight_of(x_of(l, c)));
        }
      }
      __syncthreads();
      find(by_mass, count, mass, aim_count, aim_mass);
      count = s.found_before_count, mass = s.found_before_mass;
      const uint32_t bin = (uint32_t)s.found;
      if (shift == 0) {                          // one value, held by s.found_count tokens
        k.depth = 3, k.key = kmax - bin;
        const uint64_t many = s.found_count, w = s.found_mass / many;
        uint64_t keep = many;
        if (!by_mass) {
          keep = aim_count - count;
        } else if (w > 0) {
          const double want = ceil((aim_mass - (double)mass) / (double)w);
          keep = want < 1. ? 1 : want > (double)many ? many : (uint64_t)want;
          while (keep > 1 && (double)(mass + (keep - 1) * w) >= aim_mass) --keep;
          while (keep < many && (double)(mass + keep * w) < aim_mass) ++keep;
        }
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
  // Weight of logit i if the cut and min_p keep it (tie: it is one of the cut's equal tokens, of which
  // the caller keeps the first by index).
  __device__ __forceinline__ uint32_t kept(const Cut &k, double least, int i, bool &tie) const {
    const float l = logit(i), f = place_of(l, c);
    tie = false;
    if (!has_bin(f)) return 0;
    if (k.depth > 0) {
      const int b = (int)f;
      if (b > k.b1) return 0;
      if (b == k.b1) {
        const int part = part_of(f, b);
        if (part > k.b2) return 0;
        if (part == k.b2 && k.depth > 2) {
          const uint32_t key = key_of(l);
          if (key < k.key) return 0;
          tie = k.by_index && key == k.key;
        }
      }
    }
    const uint32_t w = weight_of(x_of(l, c));
    return (double)w < least ? 0 : w;
  }
  // The warps' stretches of the slice, in index order.
  __device__ __forceinline__ void stretch(int &i0, int &i1) const {
    const int each = (n + kSampleWarps * 32 - 1) / (kSampleWarps * 32) * 32;
    i0 = min(n, (tid >> 5) * each);
    i1 = min(n, i0 + each);
  }
  // Lists the tokens up to bin `last` in the first CTA, by index, if they are at most kList; their
  // number over the row.
  __device__ uint32_t list(int last) const {
    const int lane = tid & 31, warp = tid >> 5;
    const float end = (float)(last + 1);         // (last < 2047: a token up to it has a bin)
    int i0, i1;
    stretch(i0, i1);
    uint32_t many = 0;
    for (int i = i0 + lane; i < i1; i += 32) many += place_of(logit(i), c) < end;
    many = __reduce_add_sync(kFull, many);
    if (lane == 0) s.warp_ties[warp] = many;
    __syncthreads();
    if (tid == 0) {
      uint32_t all = 0;
      for (int q = 0; q < kSampleWarps; ++q) all += s.warp_ties[q];
      s.ties = all;
    }
    sync();
    uint32_t at = 0, all = 0;
    for (int q = 0; q < ctas; ++q) {
      const uint32_t v = ld_cluster_u32(peer(&s.ties, q));
      if (q < rank) at += v;
      all += v;
    }
    if (all > (uint32_t)kList) return all;
    for (int q = 0; q < warp; ++q) at += s.warp_ties[q];
    if (many) {
      const uint32_t to_l = peer(s.list_l, 0), to_i = peer(s.list_i, 0);
      for (int i = i0; i < i1; i += 32) {
        const float l = i + lane < i1 ? logit(i + lane) : -INFINITY;
        const bool in = i + lane < i1 && place_of(l, c) < end;
        const uint32_t who = __ballot_sync(kFull, in);
        if (in) {
          const uint32_t to = at + __popc(who & ((1u << lane) - 1u));
          st_cluster_u32(to_l + 4 * to, __float_as_uint(l));
          st_cluster_u32(to_i + 4 * to, (uint32_t)(begin + i + lane));
        }
        at += __popc(who);
      }
    }
    sync();
    return all;
  }
  // The choice among the first CTA's list of `all` tokens (up to bin `last`), by that CTA alone.
  // k > 0: top-k cuts in bin `last`, before which the list holds `before` tokens.  p >= 0: top-p, of the
  // weight `row_mass` (0: of the list's, after top-k).
  __device__ void choose(const SampleArgs &a, int row, uint32_t all, int last, uint32_t before, int k, double p,
                         uint64_t row_mass, double least) const {
    constexpr int kPer = kList / kSampleThreads;
    // each thread: kPer neighbouring tokens of the list
    float l[kPer];
    uint32_t w[kPer];
    int bin[kPer];
    uint32_t *members = s.h.count;               // (the histogram's counts are not needed here)
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t i = tid * kPer + j;
      l[j] = i < all ? s.list_l[i] : -INFINITY;
      bin[j] = i < all ? (int)place_of(l[j], c) : kBins;
      w[j] = i < all ? weight_of(x_of(l[j], c)) : 0;
    }
    // the bin's tokens that `which` picks, listed in any order: each then counts those before it
    auto collect = [&](int b, auto which) {
      __syncthreads();
      if (tid == 0) s.members = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (bin[j] == b && which(j)) members[atomicAdd(&s.members, 1)] = tid * kPer + j;
      __syncthreads();
    };
    auto earlier = [&](uint32_t o, float lo, uint32_t i, float li) { return lo > li || (lo == li && o < i); };
    if (k > 0 && all > (uint32_t)k) {            // of bin `last`, the first k - before
      collect(last, [](int) { return true; });
      const int m = s.members;
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (bin[j] == last) {
          uint32_t rank_in = 0;
          for (int q = 0; q < m; ++q) {
            const uint32_t o = members[q];
            rank_in += earlier(o, s.list_l[o], tid * kPer + j, l[j]);
          }
          if (before + rank_in >= (uint32_t)k) w[j] = 0;
        }
    }
    uint64_t mass = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) mass += w[j];
    uint32_t none = 0, none_all;
    uint64_t sum = mass, whole;
    block_scan(s, none, sum, none_all, whole);
    if (p >= 0.) {
      const double aim = fmax(p * (double)(row_mass ? row_mass : whole), 1.);
      for (int i = tid; i < kBins; i += kSampleThreads) s.h.low[i] = s.h.high[i] = 0;
      if (tid == 0) s.found = -1;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (w[j]) add_mass(bin[j], w[j]);
      __syncthreads();
      uint64_t m[kBins / kSampleThreads], ms = 0;
#pragma unroll
      for (int j = 0; j < kBins / kSampleThreads; ++j) {
        const int b = tid * (kBins / kSampleThreads) + j;
        m[j] = ((uint64_t)s.h.high[b] << 16) + s.h.low[b];
        ms += m[j];
      }
      uint64_t run = ms, run_all;
      block_scan(s, none, run, none_all, run_all);
      run -= ms;
#pragma unroll
      for (int j = 0; j < kBins / kSampleThreads; ++j) {
        if (!((double)run >= aim) && (double)(run + m[j]) >= aim) {
          s.found = tid * (kBins / kSampleThreads) + j;
          s.found_before_mass = run;
        }
        run += m[j];
      }
      __syncthreads();
      const int b = s.found;
      const uint64_t mass0 = s.found_before_mass;
      collect(b, [&](int j) { return w[j] > 0; });
      const int many = s.members;
      uint32_t gone = 0;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        if (bin[j] == b && w[j]) {
          uint64_t run_in = mass0;
          for (int q = 0; q < many; ++q) {
            const uint32_t o = members[q];
            const float lo = s.list_l[o];
            if (earlier(o, lo, tid * kPer + j, l[j])) run_in += weight_of(x_of(lo, c));
          }
          if ((double)run_in >= aim) gone |= 1u << j;
        } else if (bin[j] > b) {
          gone |= 1u << j;
        }
      }
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (gone >> j & 1u) w[j] = 0;
    }
    mass = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if ((double)w[j] < least) w[j] = 0;
      mass += w[j];
    }
    sum = mass;
    block_scan(s, none, sum, none_all, whole);
    const double u = fmin(fmax((double)a.u[row], 0.), 1.);   // (a NaN becomes 0)
    uint64_t aim = (uint64_t)floor(u * (double)whole);
    if (aim >= whole) aim = whole - 1;
    sum -= mass;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (sum <= aim && aim < sum + w[j]) {
        a.tokens[row] = s.list_i[tid * kPer + j];
        if (a.probs) a.probs[row] = (float)((double)w[j] / (double)whole);
      }
      sum += w[j];
    }
  }
};

// Bytes of shared memory before the logits: SampleShared and the running sums of a share of the bins.
__host__ __device__ constexpr int sample_fixed(int ctas) {
  return (int)(sizeof(SampleShared) + 15) / 16 * 16 + kBins / ctas * 12;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SampleShared &s = *reinterpret_cast<SampleShared *>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = gridDim.x, rank = blockIdx.x, row = blockIdx.y;
  uint64_t *run_mass = reinterpret_cast<uint64_t *>(smem_raw + (sizeof(SampleShared) + 15) / 16 * 16);
  uint32_t *run_count = reinterpret_cast<uint32_t *>(run_mass + kBins / ctas);
  T *store = reinterpret_cast<T *>(smem_raw + sample_fixed(ctas));
  const int begin = min(a.vocab, rank * a.slice), n = min(a.vocab, begin + a.slice) - begin;
  for (int i = tid; i < kBins; i += kSampleThreads) s.h.count[i] = s.h.low[i] = s.h.high[i] = 0;
  grid_dependency_wait();
  grid_launch_dependents();
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  // ---- the row's slice to shared memory at its own 16-byte phase, and the largest logit
  const T *src = static_cast<const T *>(a.logits) + (int64_t)row * a.vocab + begin;
  constexpr int kVec = 16 / (int)sizeof(T), kAtOnce = 8;
  const int phase = (int)(((uintptr_t)src & 15u) / sizeof(T));
  T *data = store + phase;
  float best = -INFINITY;
  const int head = min(n, phase ? kVec - phase : 0), vecs = (n - head) / kVec;
  const uint4 *from = reinterpret_cast<const uint4 *>(src + head);
  uint4 *to = reinterpret_cast<uint4 *>(data + head);
  for (int i0 = tid; i0 < vecs; i0 += kAtOnce * kSampleThreads) {
    uint4 v[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (i0 + j * kSampleThreads < vecs) v[j] = __ldcs(from + i0 + j * kSampleThreads);
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (i0 + j * kSampleThreads < vecs) {
        to[i0 + j * kSampleThreads] = v[j];
        const T *e = reinterpret_cast<const T *>(&v[j]);
#pragma unroll
        for (int q = 0; q < kVec; ++q) best = fmaxf(best, load_logit(e + q));  // (fmaxf passes over NaN)
      }
  }
  for (int j = tid; j < n - vecs * kVec; j += kSampleThreads) {  // the ends
    const int i = j < head ? j : j + vecs * kVec;
    data[i] = src[i];
    best = fmaxf(best, load_logit(src + i));
  }
  best = warp_max_f32(best);
  if (lane == 0) s.warp_best[warp] = best;
  __syncthreads();
  for (int q = 0; q < kSampleWarps; ++q) best = fmaxf(best, s.warp_best[q]);
  if (tid == 0) s.best = best;
  Row<T> r{s, run_mass, run_count, data, begin, n, ctas, rank, tid, Scale{}};
  r.sync();
  for (int q = 0; q < ctas; ++q) best = fmaxf(best, __uint_as_float(ld_cluster_u32(peer(&s.best, q))));
  best = clean(best);
  const bool greedy = !(temperature > 0.f);
  r.c = scale_of(best, greedy ? 1.f : temperature);
  if (best == -INFINITY || greedy) {             // (the same in every CTA of the cluster)
    int first = INT32_MAX;
    if (best != -INFINITY)
      for (int i = tid; i < n && first == INT32_MAX; i += kSampleThreads)
        if (r.logit(i) == best) first = begin + i;
    first = __reduce_min_sync(kFull, first);
    if (lane == 0) s.warp_ties[warp] = (uint32_t)first;
    __syncthreads();
    if (tid == 0) {
      for (int q = 1; q < kSampleWarps; ++q) first = min(first, (int)s.warp_ties[q]);
      s.first = first;
    }
    r.sync();
    if (rank == 0 && tid == 0) {
      for (int q = 0; q < ctas; ++q) first = min(first, (int)ld_cluster_u32(peer(&s.first, q)));
      const bool none = best == -INFINITY;
      a.tokens[row] = none ? -1 : first;
      if (a.probs) a.probs[row] = none ? 0.f : 1.f;
    }
    r.sync();
    return;
  }
  const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
  const double share = by_p ? fmax((double)p, 0x1p-80) : 1.;  // (at least the likeliest token)
  const double least = (a.min_p ? (double)fminf(a.min_p[row], 1.f) : 0.) * (double)kFine;
  Cut cut;
  if (by_k || by_p) {
    // counts if top-k comes first, else weights
#pragma unroll 4
    for (int i = tid; i < n; i += kSampleThreads) {
      const float l = r.logit(i), f = place_of(l, r.c);
      if (has_bin(f)) {
        if (by_k) atomicAdd(&s.h.count[(int)f], 1u);
        else r.add_mass((int)f, weight_of(x_of(l, r.c)));
      }
    }
    __syncthreads();
    r.find(!by_k, 0, 0, (uint64_t)k, 0., share);
    // (fewer than k tokens have any weight: the last bin closes the list)
    const int last = s.found < 0 ? kBins - 2 : s.found;
    const uint32_t before = s.found < 0 ? 0 : s.found_before_count;
    const bool all_in = s.found < 0;
    const uint64_t whole = r.whole_mass();
    const uint32_t all = r.list(last);
    if (all <= (uint32_t)kList) {
      if (rank == 0) r.choose(a, row, all, last, before, by_k && !all_in ? k : 0, by_p ? share : -1.,
                              by_k ? 0 : whole, least);
      return;                                    // (no shared memory of a peer is read from here on)
    }
    double aim = fmax(share * (double)whole, 1.);
    auto histogram = [&](bool counts) {
      r.sync();
      r.clear();
      for (int i = tid; i < n; i += kSampleThreads) {
        const float l = r.logit(i), f = place_of(l, r.c);
        if (!has_bin(f)) continue;
        if (counts) atomicAdd(&s.h.count[(int)f], 1u);
        r.add_mass((int)f, weight_of(x_of(l, r.c)));
      }
      __syncthreads();
    };
    if (by_k) {
      if (by_p) {                                // (top-p wants the weight that top-k keeps)
        histogram(true);
        r.find(false, 0, 0, (uint64_t)k, 0.);
      }
      if (!all_in) cut = r.cut(false, (uint64_t)k, 0.);
      if (by_p) {
        aim = fmax(share * (double)(all_in ? r.whole_mass() : cut.mass), 1.);
        histogram(false);
        r.find(true, 0, 0, 0, aim);
      }
    }
    if (by_p) cut = r.cut(true, 0, aim);
  }
  // ---- the kept weights of each warp's stretch of the slice, in index order
  int i0, i1;
  r.stretch(i0, i1);
  uint32_t ties_before = 0;
  if (cut.by_index) {
    uint32_t ties = 0;
    for (int i = i0 + lane; i < i1; i += 32) {
      bool tie;
      r.kept(cut, least, i, tie);
      ties += tie;
    }
    ties = __reduce_add_sync(kFull, ties);
    r.sync();                                    // (s.ties: its last readers are done)
    if (lane == 0) s.warp_ties[warp] = ties;
    __syncthreads();
    if (tid == 0) {
      uint32_t all = 0;
      for (int q = 0; q < kSampleWarps; ++q) all += s.warp_ties[q];
      s.ties = all;
    }
    r.sync();
    for (int q = 0; q < rank; ++q) ties_before += ld_cluster_u32(peer(&s.ties, q));
    for (int q = 0; q < warp; ++q) ties_before += s.warp_ties[q];
  }
  // one step of 32 tokens: this lane's kept weight (ties: those before this step)
  auto step = [&](int i, uint32_t &ties) -> uint32_t {
    bool tie = false;
    uint32_t w = i < i1 ? r.kept(cut, least, i, tie) : 0u;
    if (cut.by_index) {
      const uint32_t all = __ballot_sync(kFull, tie);
      if (tie && ties + __popc(all & ((1u << lane) - 1u)) >= cut.ties) w = 0;
      ties += __popc(all);
    }
    return w;
  };
  uint64_t sum = 0;
  uint32_t ties = ties_before;
#pragma unroll 4
  for (int i = i0; i < i1; i += 32) sum += step(i + lane, ties);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
  if (lane == 0) s.warp_kept[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    uint64_t all = 0;
    for (int q = 0; q < kSampleWarps; ++q) all += s.warp_kept[q];
    s.kept = all;
  }
  r.sync();
  uint64_t before = 0, total = 0;
  for (int q = 0; q < ctas; ++q) {
    const uint64_t v = ld_cluster_u64(peer(&s.kept, q));
    if (q < rank) before += v;
    total += v;
  }
  for (int q = 0; q < warp; ++q) before += s.warp_kept[q];
  const double u = fmin(fmax((double)a.u[row], 0.), 1.);   // (a NaN becomes 0)
  uint64_t aim = (uint64_t)floor(u * (double)total);
  if (aim >= total) aim = total - 1;
  if (before <= aim && aim < before + sum) {     // one warp of the cluster
    ties = ties_before;
    for (int i = i0; i < i1; i += 32) {
      const uint32_t w = step(i + lane, ties);
      uint64_t run = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t v = __shfl_up_sync(kFull, run, o);
        if (lane >= o) run += v;
      }
      const uint32_t over = __ballot_sync(kFull, before + run > aim);
      if (over) {
        if (lane == __ffs(over) - 1) {
          a.tokens[row] = begin + i + lane;
          if (a.probs) a.probs[row] = (float)((double)w / (double)total);
        }
        break;
      }
      before += __shfl_sync(kFull, run, 31);
    }
  }
  r.sync();  // (a peer may still read this CTA's sums)
}

template <typename T>
cudaError_t launch_sample(SampleArgs a, int rows, cudaStream_t stream) {
  static bool done[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  // the fewest CTAs a row that leave room for two on an SM; more while all rows' CTAs find an SM each
  int ctas = 1;
  auto bytes = [&](int c) {
    return ((a.vocab + c - 1) / c + 7) / 8 * 8 * (int)sizeof(T) + 16 + sample_fixed(c);
  };
  while (ctas < kMaxCluster && (bytes(ctas) > kSampleSmem2 ||
                                ((int64_t)rows * ctas * 2 <= device_sms() && a.vocab > 2048 * ctas)))
    ctas *= 2;
  a.slice = ((a.vocab + ctas - 1) / ctas + 7) / 8 * 8;
  if (dev < 0 || dev >= 64 || !done[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSampleSmem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) done[dev] = true;
  }
  return launch_after(sample_kernel<T>, dim3((unsigned)ctas, (unsigned)rows), dim3(kSampleThreads),
                      (size_t)bytes(ctas), dim3((unsigned)ctas), stream, a);
}

}  // namespace
}  // namespace ham

using ham::op_aligned;
using ham::op_fail;

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

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
// A row is held in the shared memory of a cluster of CTAs and read from global memory once.  The cuts
// of the order are found without sorting: histograms (count and weight) over 2048 bins of x = (l - max)
// / T, which falls as the order goes on; then over 2048 parts of the bin that holds the cut; then, if
// that still holds several tokens, over their l itself until one value is left, whose ties are kept
// by index.  Of a histogram's bins each CTA sums its share over the cluster, so that a level costs two
// cluster barriers.
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
constexpr float kFine = 2147483648.f;   // 2^31
constexpr float kLeast = -21.49f;       // below -31 log 2 = -21.4876 a weight is 0
constexpr float kBinsPerX = 95.25f;     // kBins bins from x = 0 to beyond kLeast
constexpr int kSampleMaxVocab = 1 << 18;
constexpr int kMaxCluster = 8;           // (8 CTAs hold the largest vocabulary in fp32)
constexpr int kSampleSmem = 220 * 1024;

struct SampleArgs {
  const void *logits;
  const float *u, *temperature, *top_p, *min_p;  // all but u nullable
  const int32_t *top_k;
  int32_t *tokens;
  float *probs;
  int vocab, slice;       // elements of a CTA, a multiple of 8
};

struct Histogram { uint32_t count[kBins], low[kBins], high[kBins]; };  // weight = high 2^16 + low

// What a CTA shares with its cluster beside the logits.
struct SampleShared {
  Histogram h[2];
  uint64_t run_mass[kBins];               // running sums of the CTA's share of the bins
  uint32_t run_count[kBins];
  uint64_t total_mass, warp_mass[kSampleWarps];
  uint32_t total_count, warp_count[kSampleWarps];
  float best, warp_best[kSampleWarps];
  uint32_t key_max, key_min, warp_max[kSampleWarps], warp_min[kSampleWarps];
  uint64_t kept;                          // of this CTA
  uint32_t ties;
  int first;                              // first index of the largest logit
  uint64_t base_mass, found_before_mass, found_mass;
  uint32_t found_before_count, found_count;
  int found;
  uint64_t warp_kept[kSampleWarps];
  uint32_t warp_ties[kSampleWarps];
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
__device__ __forceinline__ float x_of(float l, float best, float t) {
  return l == best ? 0.f : __fdiv_rn(__fsub_rn(l, best), t);
}
__device__ __forceinline__ uint32_t weight_of(float x) {
  return x < kLeast ? 0u : (uint32_t)(expf(x) * kFine);
}
// The bin of x and the part of the bin; both fall as x grows.
__device__ __forceinline__ int bin_of(float x, int &part) {
  const float f = -x * kBinsPerX;
  const int b = (int)f;
  part = (int)((f - (float)b) * (float)kBins);
  return b;
}

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
template <typename T>
__device__ __forceinline__ uint32_t peer(const T *p, int rank) { return cluster_map_shared(smem_u32(p), (uint32_t)rank); }

// Where the order is cut: a token is kept if its bin comes before b1, or is b1 and (depth > 1) its part
// comes before b2, or is b2 and (depth > 2) its key is above `key`, or equal with fewer than `ties` such
// tokens before it by index.  depth 0 keeps all.
struct Cut {
  int depth = 0, b1 = 0, b2 = 0;
  uint32_t key = 0, ties = 0;
  uint64_t mass = 0;       // weight of what is kept
  bool by_index = false;   // some of the equal tokens are cut off
};

template <typename T>
struct Row {
  SampleShared &s;
  const T *data;           // this CTA's logits
  int n, ctas, rank, tid;
  float best, t;

  __device__ void sync() const {
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
  }
  __device__ void clear(Histogram &h) const {
    for (int i = tid; i < kBins; i += kSampleThreads) h.count[i] = h.low[i] = h.high[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void add(Histogram &h, int bin, uint32_t w) const {
    atomicAdd(&h.count[bin], 1u);
    if (w) {
      atomicAdd(&h.low[bin], w & 0xffffu);
      atomicAdd(&h.high[bin], w >> 16);
    }
  }
  // The first bin at which the running count (or weight) of the whole row's histogram, begun at the
  // given sums, reaches the aim; s.found (-1: none), its own and the earlier sums.  All CTAs call it.
  __device__ void find(const Histogram &h, bool by_mass, uint64_t count0, uint64_t mass0, uint64_t aim_count,
                       double aim_mass) const {
    sync();                                      // every CTA's histogram is complete
    const int share = kBins / ctas, per = (share + kSampleThreads - 1) / kSampleThreads;
    uint32_t c[4];
    uint64_t m[4], cs = 0, ms = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[j] = 0, m[j] = 0;
      const int i = tid * per + j;
      if (j < per && i < share) {
        const int bin = rank * share + i;
        for (int q = 0; q < ctas; ++q) {
          c[j] += ld_cluster_u32(peer(&h.count[bin], q));
          m[j] += ((uint64_t)ld_cluster_u32(peer(&h.high[bin], q)) << 16) + ld_cluster_u32(peer(&h.low[bin], q));
        }
      }
      cs += c[j], ms += m[j];
    }
    uint32_t ci = (uint32_t)cs;
    uint64_t mi = ms;
    const int lane = tid & 31, warp = tid >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t cu = __shfl_up_sync(kFull, ci, o);
      const uint64_t mu = __shfl_up_sync(kFull, mi, o);
      if (lane >= o) ci += cu, mi += mu;
    }
    if (lane == 31) s.warp_count[warp] = ci, s.warp_mass[warp] = mi;
    __syncthreads();
    uint32_t cb = ci - (uint32_t)cs;
    uint64_t mb = mi - ms;
    for (int q = 0; q < warp; ++q) cb += s.warp_count[q], mb += s.warp_mass[q];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = tid * per + j;
      cb += c[j], mb += m[j];
      if (j < per && i < share) s.run_count[i] = cb, s.run_mass[i] = mb;
    }
    if (tid == kSampleThreads - 1) s.total_count = cb, s.total_mass = mb;
    if (tid == 0) s.found = -1;
    sync();                                      // every CTA's running sums are complete
    uint64_t base_c = count0, base_m = mass0;
    for (int q = 0; q < ctas; ++q) {
      const uint64_t qc = ld_cluster_u32(peer(&s.total_count, q)), qm = ld_cluster_u64(peer(&s.total_mass, q));
      const bool here = by_mass ? (double)(base_m + qm) >= aim_mass : base_c + qc >= aim_count;
      if (here) {
        for (int i = tid; i < share; i += kSampleThreads) {
          const uint64_t c1 = base_c + ld_cluster_u32(peer(&s.run_count[i], q));
          const uint64_t m1 = base_m + ld_cluster_u64(peer(&s.run_mass[i], q));
          const uint64_t c0 = i ? base_c + ld_cluster_u32(peer(&s.run_count[i - 1], q)) : base_c;
          const uint64_t m0 = i ? base_m + ld_cluster_u64(peer(&s.run_mass[i - 1], q)) : base_m;
          const bool after = by_mass ? (double)m1 >= aim_mass : c1 >= aim_count;
          const bool before = by_mass ? !((double)m0 >= aim_mass) : c0 < aim_count;
          if (after && before) {
            s.found = q * share + i;
            s.found_before_count = (uint32_t)c0, s.found_before_mass = m0;
            s.found_count = (uint32_t)(c1 - c0), s.found_mass = m1 - m0;
          }
        }
        break;
      }
      base_c += qc, base_m += qm;
    }
    __syncthreads();
  }
  // Largest and smallest key (of the row) among this CTA's kmax / kmin.
  __device__ void key_range(uint32_t &kmax, uint32_t &kmin) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      kmax = max(kmax, __shfl_xor_sync(kFull, kmax, o));
      kmin = min(kmin, __shfl_xor_sync(kFull, kmin, o));
    }
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
  // The cut of the order at which the count (or the weight) reaches the aim.  h[0] holds the bins.
  __device__ Cut cut(bool by_mass, uint64_t aim_count, double aim_mass) const {
    Cut c;
    find(s.h[0], by_mass, 0, 0, aim_count, aim_mass);
    if (s.found < 0) {                           // (fewer tokens than k have any weight)
      for (int q = 0; q < ctas; ++q) c.mass += ld_cluster_u64(peer(&s.total_mass, q));
      return c;
    }
    c.depth = 1, c.b1 = s.found;
    c.mass = s.found_before_mass + s.found_mass;
    uint64_t count = s.found_before_count, mass = s.found_before_mass;
    if (s.found_count == 1 || (!by_mass && count + s.found_count == aim_count)) return c;
    // parts of the bin
    clear(s.h[1]);
    for (int i = tid; i < n; i += kSampleThreads) {
      const float x = x_of(clean(load_logit(data + i)), best, t);
      int part;
      if (x >= kLeast && bin_of(x, part) == c.b1) add(s.h[1], part, weight_of(x));
    }
    __syncthreads();
    find(s.h[1], by_mass, count, mass, aim_count, aim_mass);
    c.depth = 2, c.b2 = s.found;
    c.mass = s.found_before_mass + s.found_mass;
    count = s.found_before_count, mass = s.found_before_mass;
    if (s.found_count == 1 || (!by_mass && count + s.found_count == aim_count)) return c;
    // values of l within the part, until one is left
    uint32_t lo = 0, hi = 0xffffffffu;
    for (;;) {
      uint32_t kmax = 0, kmin = 0xffffffffu;
      for (int i = tid; i < n; i += kSampleThreads) {
        const float l = clean(load_logit(data + i)), x = x_of(l, best, t);
        int part;
        if (x >= kLeast && bin_of(x, part) == c.b1 && part == c.b2) {
          const uint32_t k = key_of(l);
          if (k >= lo && k <= hi) kmax = max(kmax, k), kmin = min(kmin, k);
        }
      }
      key_range(kmax, kmin);
      int shift = 0;
      while (((kmax - kmin) >> shift) >= (uint32_t)kBins) ++shift;
      clear(s.h[1]);
      for (int i = tid; i < n; i += kSampleThreads) {
        const float l = clean(load_logit(data + i)), x = x_of(l, best, t);
        int part;
        if (x >= kLeast && bin_of(x, part) == c.b1 && part == c.b2) {
          const uint32_t k = key_of(l);
          if (k >= kmin && k <= kmax) add(s.h[1], (int)((kmax - k) >> shift), weight_of(x));
        }
      }
      __syncthreads();
      find(s.h[1], by_mass, count, mass, aim_count, aim_mass);
      count = s.found_before_count, mass = s.found_before_mass;
      const uint32_t bin = (uint32_t)s.found;
      if (shift == 0) {                          // one value, held by s.found_count tokens
        c.depth = 3, c.key = kmax - bin;
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
        c.ties = (uint32_t)keep;
        c.by_index = keep < many;
        c.mass = mass + keep * w;
        return c;
      }
      hi = kmax - (bin << shift);
      const uint32_t down = ((bin + 1) << shift) - 1;
      lo = kmax - kmin < down ? kmin : kmax - down;
    }
  }
  // Weight of logit i if the cut and min_p keep it (tie: it is one of the cut's equal tokens, of which
  // the caller keeps the first by index).
  __device__ __forceinline__ uint32_t kept(const Cut &c, double least, int i, bool &tie) const {
    const float l = clean(load_logit(data + i)), x = x_of(l, best, t);
    tie = false;
    if (!(x >= kLeast)) return 0;
    const uint32_t w = weight_of(x);
    if ((double)w < least) return 0;
    if (c.depth > 0) {
      int part;
      const int b = bin_of(x, part);
      if (b > c.b1) return 0;
      if (b == c.b1 && c.depth > 1) {
        if (part > c.b2) return 0;
        if (part == c.b2 && c.depth > 2) {
          const uint32_t k = key_of(l);
          if (k < c.key) return 0;
          tie = c.by_index && k == c.key;
        }
      }
    }
    return w;
  }
};

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(SampleArgs a) {
  extern __shared__ uint8_t smem_raw[];
  SampleShared &s = *reinterpret_cast<SampleShared *>(smem_raw);
  T *store = reinterpret_cast<T *>(smem_raw + (sizeof(SampleShared) + 15) / 16 * 16);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = gridDim.x, rank = blockIdx.x, row = blockIdx.y;
  const int begin = min(a.vocab, rank * a.slice), n = min(a.vocab, begin + a.slice) - begin;
  grid_dependency_wait();
  grid_launch_dependents();
  // ---- the row's slice to shared memory at its own 16-byte phase, and the largest logit
  const T *src = static_cast<const T *>(a.logits) + (int64_t)row * a.vocab + begin;
  constexpr int kVec = 16 / (int)sizeof(T);
  const int phase = (int)(((uintptr_t)src & 15u) / sizeof(T));
  T *data = store + phase;
  float best = -INFINITY;
  const int head = min(n, phase ? kVec - phase : 0), vecs = (n - head) / kVec;
  for (int i = tid; i < vecs; i += kSampleThreads) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4 *>(src + head) + i);
    *(reinterpret_cast<uint4 *>(data + head) + i) = v;
    const T *e = reinterpret_cast<const T *>(&v);
#pragma unroll
    for (int j = 0; j < kVec; ++j) best = fmaxf(best, load_logit(e + j));  // (fmaxf passes over NaN)
  }
  for (int j = tid; j < n - vecs * kVec; j += kSampleThreads) {  // the ends
    const int i = j < head ? j : j + vecs * kVec;
    data[i] = src[i];
    best = fmaxf(best, load_logit(src + i));
  }
  best = warp_max_f32(best);
  if (lane == 0) s.warp_best[warp] = best;
  for (int i = tid; i < kBins; i += kSampleThreads) s.h[0].count[i] = s.h[0].low[i] = s.h[0].high[i] = 0;
  __syncthreads();
  best = s.warp_best[0];
  for (int q = 1; q < kSampleWarps; ++q) best = fmaxf(best, s.warp_best[q]);
  if (tid == 0) s.best = best;
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  const bool greedy = !(temperature > 0.f);
  Row<T> r{s, data, n, ctas, rank, tid, best, greedy ? 1.f : temperature};
  r.sync();
  for (int q = 0; q < ctas; ++q) best = fmaxf(best, __uint_as_float(ld_cluster_u32(peer(&s.best, q))));
  best = clean(best);
  r.best = best;
  if (best == -INFINITY || greedy) {             // (the same in every CTA of the cluster)
    int first = INT32_MAX;
    if (best != -INFINITY)
      for (int i = tid; i < n && first == INT32_MAX; i += kSampleThreads)
        if (clean(load_logit(data + i)) == best) first = begin + i;
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
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
  const double least = (a.min_p ? (double)fminf(a.min_p[row], 1.f) : 0.) * (double)kFine;
  Cut c;
  if (by_k || by_p) {
    for (int i = tid; i < n; i += kSampleThreads) {
      const float x = x_of(clean(load_logit(data + i)), best, r.t);
      int part;
      if (x >= kLeast) r.add(s.h[0], bin_of(x, part), weight_of(x));
    }
    __syncthreads();
    if (by_k) c = r.cut(false, (uint64_t)k, 0.);
    if (by_p) {
      uint64_t mass = c.mass;
      if (!by_k) {                               // the whole row's weight
        r.find(s.h[0], false, 0, 0, ~0ull, 0.);
        for (int q = 0; q < ctas; ++q) mass += ld_cluster_u64(peer(&s.total_mass, q));
      }
      c = r.cut(true, 0, fmax((double)p * (double)mass, 1.));
    }
  }
  // ---- the kept weights of each warp's stretch of the slice, in index order
  const int stretch = (n + kSampleWarps * 32 - 1) / (kSampleWarps * 32) * 32;
  const int i0 = min(n, warp * stretch), i1 = min(n, i0 + stretch);
  uint32_t ties_before = 0;
  if (c.by_index) {
    uint32_t ties = 0;
    for (int i = i0 + lane; i < i1; i += 32) {
      bool tie;
      r.kept(c, least, i, tie);
      ties += tie;
    }
    ties = __reduce_add_sync(kFull, ties);
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
    uint32_t w = i < i1 ? r.kept(c, least, i, tie) : 0u;
    if (c.by_index) {
      const uint32_t all = __ballot_sync(kFull, tie);
      if (tie && ties + __popc(all & ((1u << lane) - 1u)) >= c.ties) w = 0;
      ties += __popc(all);
    }
    return w;
  };
  uint64_t sum = 0;
  uint32_t ties = ties_before;
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
  const int fixed = (int)(sizeof(SampleShared) + 15) / 16 * 16 + 16;
  // the fewest CTAs whose shared memory holds a row; more while all rows' CTAs find an SM each
  int ctas = 1;
  auto bytes = [&](int c) {
    return ((a.vocab + c - 1) / c + 7) / 8 * 8 * (int)sizeof(T) + fixed;
  };
  while (ctas < kMaxCluster && (bytes(ctas) > kSampleSmem ||
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

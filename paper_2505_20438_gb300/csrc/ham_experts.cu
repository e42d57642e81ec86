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
#include <atomic>
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

// ------------------------------------------------------------------------------------
// The kernel: pairs of CTAs, 256 rows of weights by up to 224 slots
// ------------------------------------------------------------------------------------
// The weights are the product's M: a pair of CTAs (cta_group::2) multiplies two half tiles, one a CTA (128 lanes of its
// tensor memory), with the N rows of one expert's slots.  N is what the expert has, up to the next multiple of 32, so
// that a few rows cost a few rows' products and many experts of uneven counts leave no lanes idle.  More than 224 slots
// are cut into tiles of equal size, more than 128 into two halves of N, each for four warps of the epilogue.
//
// Each CTA copies its half tile's K block (16 KiB, one stretch) and half of the N rows (of a gated product by index, four
// rows a copy, or sorted before) into its own shared memory alone.  Sums take parts of K as the products of one weight do
// (ham_fp8.cu), of equal size and at most kExpertPart blocks (or one more, for an even number), in two sums of 224 columns
// in turn, so that two parts' products are on their way while the epilogue deals with the tile before; it adds them in
// registers.  Errors against 64-bit sums, relative to the outputs' norm, of K 512, 1024, 1408, 2048, 4096, 8192: 3.4e-8,
// 6.0e-8, 7.2e-8, 6.5e-8, 8.7e-8, 9.8e-8 (an fp32 product in the usual order 2.7e-8, 4.1e-8, 4.7e-8, 6.0e-8, 8.6e-8, 1.3e-7).
// With parts of 16 blocks they were 1.1e-7 from K 2048 on; the more parts cost gated halves of 64, 128, 192 slots an expert
// 0.4, 3 and 4% at K 4096, of 512 there 3%, at K 2048 (two parts instead of one) 1, 6 and 9% of 64, 128 and 512, plain
// products 2% at most.  Parts of 8: 6.5e-8, 7.2e-8 and 8.2e-8 at 2048, 4096 and 8192, and 507 us for 4096 rows' gated halves
// (parts of 11 457, of 16 444).
//
// A thread of the epilogue has one feature (a lane) and up to 128 slots (columns).  Plain outputs are neighbours across
// a warp's lanes.  Of a gated product 16 lanes hold the gate and 16 the up projection of 16 features: half a warp reads
// both of half the slots, the other half those of the others (with lanes exchanged by shuffles 4096 rows of 8 experts took
// 474 us, 460 so).  A slot's largest magnitude over the 128 features of a scale is wanted from both CTAs' warps: 16 bits of
// each (exponent and seven bits, all that the scale depends on) through shared memory and the pair's.
//
// What bounds it.  Few rows: the weights' bytes.  8 rows of 8 of 64 experts (K 4096, 2048 features) take 119 us, 87% of the
// copy rate with the sorting and the first and last tile's latencies, some 7 us, in it; the second products (K 2048, 4096
// features) 59 us, 87%.  Many rows: no one thing.  4096 rows of 8 of 64 experts take 457 to 507 us, 25 of them the sorting, and
// 226 to 231 for the second products, 2.4 PFLOP/s; a stream of such calls, which the card's power limit slows down, 540 and 265.
// A K block of the usual tile, 171 slots of 512, is 27 KB a CTA in 0.33 us: 83 GB/s an SM, 12.6 TB/s in all, where the dense pair
// kernel's 32 KB come at 93 and feed 256 rows.  Without any epilogue the calls took 410 and 198 (of 446 and 224, with parts of 16
// blocks), with half of the products 356 and 178, without the weights' copies 354 and 181: each alone is an eighth to a fifth.
// The gated epilogue's sums, results and maxima pass its 216 registers: 180 bytes a thread are spilled (the plain one's none).
//
// Measured and not taken: copies by index for many rows (1430 us gated: 84 clocks for four rows, whoever issues them from one
// warp); three sums of 128 columns and tiles of 256 slots (520 us); deeper rings where tiles are narrow (no faster); the next tile's looking up moved ahead (2 to 8% slower);
// weights marked to leave the L2 first (478 against 453 us).
struct ExpertArgs {
  const uint8_t *ws;       // the handle's scales
  const uint8_t *xs;       // the rows'
  const int32_t *offsets, *order;
  int gather, boxes;       // the rows are order's, not the slots' own; row maps
  void *out;
  uint8_t *out_scales;     // gated
  int32_t *err;
  int experts, slots, top_k, n, kbs, part, sk, out_sk, tiles, f32;   // part: K blocks of one accumulator, even
  uint64_t wait_ns;
};

constexpr int kExpertPart = 11;         // K blocks of one accumulator, or one more
constexpr int kExpertStages = 6;
constexpr int kExpertStageBytes = 2 * kBlockBytes;  // the weights' block, 64 + 64 rows
constexpr int kExpertSf = 4;            // scale slots (of four K blocks each)
constexpr int kExpertSfBytes = 3 * 512; // the CTA's half tile, both halves of N
constexpr int kExpertFew = 72, kExpertMany = 216;  // registers of the first four warps' threads, of the epilogue's
static_assert(4 * kExpertFew + 8 * kExpertMany <= 12 * kLaunchRegs, "registers");
constexpr int kTileSlots = 224, kSfCol = 448;  // columns of one of the two sums, and behind both the scales
constexpr int kGroup = 2;               // K blocks that one accumulator takes, then the other
constexpr int kKeyBytes = 2 * 2 * 8 * 128 * 2;   // [half][every other tile][warp of the pair][slot]
constexpr int kCodeBytes = 2 * 128 * 64;         // [half][slot][feature]
constexpr int kPowerBytes = 2 * 128 * 4;         // [half][slot]
constexpr int kExpertBars = 288;
constexpr int kExpertUsed = 1024 + kExpertStages * kExpertStageBytes + kExpertSf * kExpertSfBytes + kExpertBars;
constexpr int kTurnPitch = 144, kTurnBytes = 16 * kTurnPitch;  // plain: a warp's 32 features of 32 slots, slots in pairs
constexpr int expert_smem(bool gated) {
  const int used = kExpertUsed + (gated ? kKeyBytes + kCodeBytes + kPowerBytes : 8 * kTurnBytes);
  return used > smem_floor(512) ? used : smem_floor(512);
}
static_assert(expert_smem(true) + (kMostExperts + 1) * 4 + 32 * 16 + 128 <= 227 * 1024, "shared memory");

// A tile: slots of one expert by one pair of half tiles.  A CTA brings the rows of (n0 + n1) / 2 neighbouring slots, the
// first n0 / 2 of them for the first half.
struct ExpertTile {
  int expert, ct, slot0, count;
  int n0, n1;                           // columns of the two halves (multiples of 32; n1 may be 0)
  // The tile's slot that is column j of half h: the first CTA's rows, then the second one's.
  __device__ __forceinline__ int slot_at(int h, int j) const {
    const int mine = (h ? n1 : n0) / 2, first = h ? n0 / 2 : 0;
    return first + j + (j < mine ? 0 : (n0 + n1) / 2 - mine);
  }
};

// The rows of the slots, one after another, for products with more rows than a copy by index keeps up with.
constexpr int kSortWarps = 8;
__global__ void __launch_bounds__(kSortWarps * 32) sort_rows_kernel(const uint4 *__restrict__ x, const uint32_t *__restrict__ xs,
                                                                    const int32_t *order, const int32_t *offsets, int experts, int slots, int top_k,
                                                                    int vecs, int words, uint4 *codes, uint32_t *scales,
                                                                    int32_t *err) {
  const int lane = threadIdx.x & 31;
  const int64_t slot = (int64_t)blockIdx.x * kSortWarps + (threadIdx.x >> 5);
  grid_dependency_wait();
  grid_launch_dependents();
  if (slot >= slots) return;
  int64_t row = order[slot];                     // (on its way with the offsets)
  if (slot < offsets[0] || slot >= offsets[experts]) return;
  if (row < 0 || row >= slots) {
    if (lane == 0) record_error(err, HAM_DEVERR_ROUTE);
    row = 0;
  }
  row /= top_k;
  for (int w = lane; w < words; w += 32) scales[slot * words + w] = xs[row * words + w];
  int v = lane;
  for (; v + 7 * 32 < vecs; v += 8 * 32) {
    uint4 r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[row * vecs + v + 32 * i];
#pragma unroll
    for (int i = 0; i < 8; ++i) codes[slot * vecs + v + 32 * i] = r[i];
  }
  for (; v < vecs; v += 32) codes[slot * vecs + v] = x[row * vecs + v];
}

// Maps of the rows with boxes of 16, 32 and 64 of them, as far as a CTA's may be that many; of rows by index the first
// alone, with boxes of one.
constexpr int kBoxes = 3;
struct RowMaps {
  CUtensorMap of[kBoxes];
};

// u g / (1 + exp(-g)), of two numbers, from t = exp(-|g|), which never overflows: g t / (1 + t) below zero, g / (1 + t)
// above; the reciprocal, of a number in 1..2, with one step of Newton's (a quotient's general form tests for and mends
// cases that do not occur here).
__device__ __forceinline__ float2 silu_mul2(float2 g, float2 u) {
  const float2 one = make_float2(1.f, 1.f), t = make_float2(expf(-fabsf(g.x)), expf(-fabsf(g.y)));
  const float2 d = add2(t, one);
  float2 r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(d.y));
  r = fma2(r, fma2(make_float2(-d.x, -d.y), r, one), r);
  const float2 s = mul2(make_float2(g.x < 0.f ? t.x : 1.f, g.y < 0.f ? t.y : 1.f), r);
  return mul2(mul2(g, s), u);
}

template <bool kGated>
__global__ void __launch_bounds__(kPairThreads, 1)
    experts_kernel(const __grid_constant__ RowMaps tx, const __grid_constant__ CUtensorMap tw, ExpertArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *sf = ring + kExpertStages * kExpertStageBytes;
  // full, sf_full and sum_free: the ones of a pair's first CTA are used
  uint64_t *full = reinterpret_cast<uint64_t *>(sf + kExpertSf * kExpertSfBytes);
  uint64_t *empty = full + kExpertStages;
  uint64_t *sf_full = empty + kExpertStages;   // an arrival a CTA
  uint64_t *sf_empty = sf_full + kExpertSf;
  uint64_t *sum_full = sf_empty + kExpertSf;   // [epilogue group][its parts in turn]
  uint64_t *sum_free = sum_full + 4;           // [sum][half]: an arrival a warp of the pair that takes it
  uint64_t *keys_full = sum_free + 4;          // [half][every other tile]: an arrival a warp of the pair
  uint64_t *drained = keys_full + 4;           // every product issued is complete
  static_assert((2 * kExpertStages + 2 * kExpertSf + 13) * 8 <= kExpertBars, "barriers");
  uint16_t *keys = reinterpret_cast<uint16_t *>(reinterpret_cast<uint8_t *>(full) + kExpertBars);
  uint8_t *code_rows = reinterpret_cast<uint8_t *>(keys) + kKeyBytes;
  float *powers = reinterpret_cast<float *>(code_rows + kCodeBytes);
  __shared__ int starts[kMostExperts + 1];     // row tiles of the experts before
  __shared__ int parts_of[12], bad_shared;
  __shared__ int4 gathered[32];                // the rows of a tile's copies by index
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_shared, issued_shared;
  volatile int *abort_flag = &abort_shared;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int side = (int)cluster_rank();
  const uint32_t both = 3u;
  const int clusters = gridDim.x / 2, cluster = blockIdx.x / 2;
  const int cols = kGated ? a.tiles : (a.tiles + 1) / 2;    // pairs of half tiles
  // A wait ran out (or the pair has given up already): both CTAs stop.
  const auto give_up = [&] {
    if (*abort_flag) return;
    record_error(a.err, HAM_DEVERR_TIMEOUT);
    *abort_flag = 1;
    st_cluster_u32(cluster_map_shared(smem_u32(&abort_shared), side ^ 1), 1u);
  };
  if (tid == 0) {
    for (int s = 0; s < kExpertStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < kExpertSf; ++s) {
      mbar_init(&sf_full[s], 2);
      mbar_init(&sf_empty[s], 1);
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(&sum_full[s], 1);
      mbar_init(&sum_free[s], 8);
      mbar_init(&keys_full[s], 8);
    }
    mbar_init(drained, 1);
    abort_shared = 0;
    bad_shared = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) {
    for (int i = 0; i < a.boxes; ++i) prefetch_tensormap(&tx.of[i]);
    prefetch_tensormap(&tw);
  }
  cluster_sync_all();
  // Tensor memory is taken before the dependency wait and before the next kernel may start (as in ham_fp8.cu).
  if (warp == 1) tmem_alloc_pair<512>(&tmem_slot);
  tc_fence_before();
  grid_dependency_wait();
  // ---------------------------------------------------------------- the experts' row tiles, added up
  {
    int tiles_of[2], sum = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = 2 * tid + i;
      tiles_of[i] = 0;
      if (e < a.experts) {
        const int from = a.offsets[e], to = a.offsets[e + 1];
        if (from < 0 || to < from || to > a.slots) bad_shared = 1;
        else tiles_of[i] = (to - from + kTileSlots - 1) / kTileSlots;
      }
      sum += tiles_of[i];
    }
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(kFull, run, o);
      if (lane >= o) run += x;
    }
    if (lane == 31) parts_of[warp] = run;
    __syncthreads();
    tc_fence_after();
    for (int w = 0; w < warp; ++w) run += parts_of[w];
    run -= sum;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (2 * tid + i <= a.experts) starts[2 * tid + i] = run;
      run += tiles_of[i];
    }
    __syncthreads();
  }
  if (bad_shared && tid == 0) record_error(a.err, HAM_DEVERR_ROUTE);
  const int64_t total = bad_shared ? 0 : (int64_t)starts[a.experts] * cols;
  const uint32_t tmem = *const_cast<volatile uint32_t *>(&tmem_slot);
  // Tile w: an expert's tiles lie together, its row tiles next to one another (they share their weights).
  const auto tile_of = [&](int64_t w) {
    int lo = 0, hi = a.experts;                  // starts[lo] * cols <= w < starts[hi] * cols
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((int64_t)starts[mid] * cols <= w) lo = mid;
      else hi = mid;
    }
    ExpertTile t;
    t.expert = lo;
    const int from = a.offsets[lo], rows = a.offsets[lo + 1] - from, rt = starts[lo + 1] - starts[lo];
    const int64_t at = w - (int64_t)starts[lo] * cols;
    int r = 0;
    t.ct = (int)at;
    if (rt > 1) t.ct = (int)(at / rt), r = (int)(at % rt);
    const int each = ((rows + rt - 1) / rt + 31) & ~31;
    t.slot0 = from + r * each;
    t.count = min(each, rows - r * each);
    const int n = (t.count + 31) & ~31;
    t.n0 = n > 128 ? (n / 2 + 31) & ~31 : n;
    t.n1 = n - t.n0;
    return t;
  };
  // The row of the tile's slot i (past the last: the last).
  const auto row_of = [&](const ExpertTile &t, int i) {
    const int slot = t.slot0 + min(i, t.count - 1);
    if (!a.gather) return slot;
    const int o = a.order[slot];
    if ((uint32_t)o >= (uint32_t)a.slots) {
      record_error(a.err, HAM_DEVERR_ROUTE);
      return 0;
    }
    return o / a.top_k;
  };
  // The copies of a tile by warp 0: of a CTA's rows those that the tile has (what lies in the others' place does not
  // matter: a row's sums are its own), up to the next multiple of 16; by index, of four.
  struct Source { int w, bytes, copies, row; };
  const auto source_of = [&](int64_t w) {
    const ExpertTile t = tile_of(w);
    const int n = (t.n0 + t.n1) / 2, each = a.gather ? 4 : 16;
    Source from;
    from.bytes = 2 * kBlockBytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int copies = (min(max(t.count - s * n, 0), n) + each - 1) / each;
      from.bytes += copies * each * 128;
      if (s == side) from.copies = copies;
    }
    from.row = t.slot0 + side * n;
    if (a.gather && lane < from.copies) {
      const int i = side * n + lane * 4;
      gathered[lane] = make_int4(row_of(t, i), row_of(t, i + 1), row_of(t, i + 2), row_of(t, i + 3));
    }
    __syncwarp();
    const int half = kGated ? t.ct * 2 + side : min(t.ct * 2 + side, a.tiles - 1);
    from.w = (t.expert * (a.tiles * (kGated ? 2 : 1)) + half) * a.kbs;
    return from;
  };
  // Request a tile's K block kb for stage s (one thread); the bytes of both CTAs count at the first one's barrier.
  const auto request = [&](int s, const Source &from, int kb, uint64_t pol) {
    const uint32_t bar = cluster_map_shared(smem_u32(&full[s]), 0);
    uint8_t *dst = ring + s * kExpertStageBytes;
    if (side == 0) mbar_arrive_tx(&full[s], (uint32_t)from.bytes);
    tma_load_2d_pair(dst, &tw, 0, (from.w + kb) * (kBlockBytes / 2048), bar, pol);
    dst += kBlockBytes;
    if (a.gather) {
#pragma unroll 1
      for (int c0 = 0; c0 < from.copies; c0 += 4) {
        int4 r[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) r[c] = gathered[c0 + c];
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c0 + c < from.copies) tma_gather4_pair(dst + (c0 + c) * 512, &tx.of[0], kb * kFp8Block, r[c], bar, pol);
      }
    } else {
      int done = 0;
#pragma unroll
      for (int i = kBoxes - 1; i >= 0; --i)
        if (from.copies >> i & 1) {
          tma_load_2d_pair(dst + done * 2048, &tx.of[i], kb * kFp8Block, from.row + done * 16, bar, pol);
          done += 1 << i;
        }
    }
  };
  int issued = 0;
  if (warp < 4) {
    setmaxnreg_dec<kExpertFew>();
    if (warp == 0) {
      // ------------------------------------------------------------ copies
      const uint64_t pol = policy_evict_last();
      bool ok = true;
      int it = 0;
      for (int64_t w = cluster; w < total && ok; w += clusters) {
        const Source from = source_of(w);
        for (int kb = 0; kb < a.kbs; ++kb, ++it) {
          if (it >= kExpertStages &&
              !warp_wait(&empty[it % kExpertStages], (uint32_t)(it / kExpertStages - 1) & 1u, abort_flag)) {
            ok = false;
            break;
          }
          if (elect_one()) request(it % kExpertStages, from, kb, pol);
          __syncwarp();
          issued = it + 1;
        }
      }
      if (!ok && lane == 0) give_up();
    } else if (warp == 1) {
      // ------------------------------------------------------------ products (a pair's first CTA)
      if (side == 0 && elect_one()) {
        const uint64_t blocks = smem_desc_sw128(smem_u32(ring), 16, 1024), words = smem_desc_plain(smem_u32(sf), 0, 128);
        constexpr uint32_t kNextByte = idesc_mx(256, 128, 1) - idesc_mx(256, 128, 0);
        bool ok = true;
        int s = 0, slot = 0;                     // of the block, of the scale word
        uint32_t phase = 0, word_phase = 0, which = 0;
        uint32_t part = 0, singles = 0, given[2] = {0, 0};  // parts, tiles of one half, each group's parts so far
        uint32_t used[2][2] = {{0, 0}, {0, 0}};    // [sum][half]: how often
        // Both halves of a sum are free.
        const auto free_sum = [&](int b) {
          for (int h = 0; h < 2; ++h) {
            const uint32_t n = b ? used[1][h] : used[0][h];
            if (n && !thread_wait_cluster(&sum_free[b * 2 + h], (n - 1) & 1u, abort_flag)) return false;
          }
          return true;
        };
        for (int64_t w = cluster; w < total && ok; w += clusters) {
          const ExpertTile t = tile_of(w);
          const int halves = t.n1 ? 2 : 1;
          const uint32_t alone = halves == 1 && (singles++ & 1);  // the second group's turn
          const uint32_t idesc_half[2] = {idesc_mx(256, t.n0, 0), idesc_mx(256, t.n1, 0)};
          for (int g = 0, in = 0; g < a.kbs; g += kGroup) {  // in: blocks of this part so far
            const bool two = g + 1 < a.kbs, ends = g + kGroup >= a.kbs || in + kGroup >= a.part;
            const int s1 = s + 1 == kExpertStages ? 0 : s + 1;
            if ((g & 3) == 0) {
              ok = ok && thread_wait_cluster(&sf_full[slot], word_phase, abort_flag);
              which ^= 16;
            }
            ok = ok && thread_wait_cluster(&full[s], phase, abort_flag);
            if (in == 0) ok = ok && free_sum(part & 1);
            if (!ok) break;
            tc_fence_after();
            const uint32_t sft = tmem + kSfCol + which;
            if ((g & 3) == 0) {
#pragma unroll
              for (int p = 0; p < 3; ++p)
                tc_copy_scales_of<2>(sft + p * 4, words + (uint32_t)(slot * (kExpertSfBytes / 16) + p * 32));
              tc_commit_pair(&sf_empty[slot], both);
              if (++slot == kExpertSf) slot = 0, word_phase ^= 1;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (h >= halves) break;
              const uint32_t acc = tmem + (part & 1) * kTileSlots + (h ? t.n0 : 0), idesc = idesc_half[h] + (g & 3) * kNextByte;
#pragma unroll
              for (int j = 0; j < kGroup; ++j) {
                if (j && !two) break;
                const int st = j ? s1 : s;
                if (j && !h) {
                  ok = thread_wait_cluster(&full[s1], phase ^ (s1 == 0), abort_flag);
                  if (!ok) break;
                  tc_fence_after();
                }
                const uint64_t wt = blocks + (uint32_t)(st * (kExpertStageBytes / 16)), x = wt + (uint32_t)(kBlockBytes + (h ? t.n0 / 2 * 128 : 0)) / 16;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                  tc_mma_mx<2>(acc, wt + kk * 2, x + kk * 2, idesc + j * kNextByte, sft, sft + 4 + 4 * h, in + j + kk > 0);
                if (h == halves - 1) tc_commit_pair(&empty[st], both);
              }
              if (!ok) break;
              if (ends) {
                if (h || alone) tc_commit_pair(&sum_full[2 + (given[1]++ & 1)], both);
                else tc_commit_pair(&sum_full[given[0]++ & 1], both);
                if (part & 1) ++used[1][h];
                else ++used[0][h];
              }
            }
            if (!ok) break;
            s += two ? 2 : 1;
            if (s >= kExpertStages) s -= kExpertStages, phase ^= 1;
            in += kGroup;
            if (ends) {
              in = 0;
              ++part;
            }
          }
        }
        if (!ok) give_up();
        tc_commit_pair(drained, both);
      }
      __syncwarp();
    } else {
      // ------------------------------------------------------------ scale words
      // Two warps take turns at the words (of four K blocks each), and each loads its next before it passes one on.
      if (warp == 2) grid_launch_dependents();
      const int groups = (a.kbs + 3) / 4, turn = warp - 2;
      uint32_t x[8], ws;
      int64_t w = cluster, known = -1;           // known: the tile of the rows below
      int g = turn, rows[8], wrow = 0;
      const auto load = [&] {
        if (w != known) {
          const ExpertTile t = tile_of(w);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int i = lane + 32 * (j & 3);
            rows[j] = i < (j < 4 ? t.n0 : t.n1) ? row_of(t, t.slot_at(j >> 2, i)) : -1;
          }
          wrow = kGated ? (t.expert * a.tiles + t.ct) * 2 + (lane >> 4) : t.expert * a.tiles + min(t.ct * 2 + side, a.tiles - 1);
          known = w;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          x[j] = rows[j] >= 0 ? __ldg(reinterpret_cast<const uint32_t *>(a.xs + (int64_t)rows[j] * a.sk) + g) : 0x7f7f7f7fu;
        ws = __ldg(reinterpret_cast<const uint32_t *>(a.ws + (int64_t)wrow * a.sk) + g);
      };
      // the gi-th word of this cluster's tiles is word g of tile w
      const auto settle = [&] {
        while (g >= groups) g -= groups, w += clusters;
      };
      settle();
      if (w < total) load();
      for (int64_t gi = turn; w < total; gi += 2) {
        const int slot = (int)(gi % kExpertSf);
        if (gi >= kExpertSf && !warp_wait(&sf_empty[slot], (uint32_t)(gi / kExpertSf - 1) & 1u, abort_flag, a.wait_ns)) {
          if (lane == 0) give_up();
          break;
        }
        uint4 *dst = reinterpret_cast<uint4 *>(sf + slot * kExpertSfBytes) + lane;
        dst[0] = make_uint4(ws, ws, ws, ws);
        dst[32] = make_uint4(x[0], x[1], x[2], x[3]);
        dst[64] = make_uint4(x[4], x[5], x[6], x[7]);
        g += 2;
        settle();
        if (w < total) load();
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(cluster_map_shared(smem_u32(&sf_full[slot]), 0));
      }
    }
  } else {
    setmaxnreg_inc<kExpertMany>();
    // ------------------------------------------------------------ epilogue: a feature a thread
    // Four warps take the first half's sums, four the second's; tiles of one half in turn.
    const int quarter = warp & 3, group = (warp - 4) >> 2;
    const uint32_t free_bar = cluster_map_shared(smem_u32(sum_free), 0);
    const int parts = (a.kbs + a.part - 1) / a.part;
    uint32_t first = 0, singles = 0;             // parts, tiles of one half so far
    uint32_t got = 0, taken = 0;                 // parts, tiles that this group took
    for (int64_t w = cluster; w < total; w += clusters) {
      const ExpertTile t = tile_of(w);
      const int halves = t.n1 ? 2 : 1;
      int half = group;
      const uint32_t sum = first;
      first += parts;
      if (halves == 1) {
        if ((singles++ & 1) != (uint32_t)group) continue;
        half = 0;
      }
      const int n = half ? t.n1 : t.n0;
      // Plain: a feature's sums, slot after slot.  Gated: the gate's of feature 16 quarter + lane % 16 and from 64 on the up
      // projection's, 16 columns of each 32, the first ones (lanes 0..15) or the others.
      float v[128];
      bool ok = true;
#pragma unroll 1
      for (int c = 0; c < parts; ++c) {
        const int b = (int)(sum + c & 1);
        // (a group waits for parts of its own alone, each barrier's phases in order: of them two at most are full and
        // not yet taken)
        ok = warp_wait_cluster(&sum_full[group * 2 + (got & 1)], (got >> 1) & 1u, abort_flag);
        ++got;
        if (!ok) {
          if (lane == 0) give_up();
          break;
        }
        tc_fence_after();
        const uint32_t acc = tmem + b * kTileSlots + (half ? t.n0 : 0) + ((uint32_t)(quarter * 32) << 16);
        const auto load = [&](int q, float *first, float *second) {  // 32 columns: plain; gated: the gate's, the up's
          if constexpr (kGated) {
            tmem_ld16x2(acc + q * 32, *reinterpret_cast<uint32_t(*)[16]>(first));
            tmem_ld16x2(acc + q * 32 + (16u << 16), *reinterpret_cast<uint32_t(*)[16]>(second));
          } else {
            tmem_ld32(acc + q * 32, *reinterpret_cast<uint32_t(*)[32]>(first));
          }
        };
        if (c == 0) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q * 32 < n) load(q, v + q * (kGated ? 16 : 32), v + 64 + q * 16);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q * 32 < n) {
              float f[32];
              load(q, f, f + 16);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const int at = !kGated ? q * 32 + j : j < 16 ? q * 16 + j : 48 + q * 16 + j;
                const float2 s = add2(make_float2(v[at], v[at + 1]), make_float2(f[j], f[j + 1]));
                v[at] = s.x, v[at + 1] = s.y;
              }
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(free_bar + (b * 2 + half) * 8);
      }
      if constexpr (!kGated) {
        if (!ok) break;
        const int f0 = t.ct * 256 + side * 128 + quarter * 32;
        if (!a.f32 && (a.n & 7) == 0) {
          // Pairs of slots as words, turned in shared memory: a lane then writes 8 features of two slots.  (Straight from
          // the registers, 2 bytes a lane, 4096 rows of 8 experts took 248 us.)
          uint8_t *turn = reinterpret_cast<uint8_t *>(keys) + (warp - 4) * kTurnBytes;
          const int pair = lane >> 2, c = (lane & 3) * 8;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (q * 32 >= n) continue;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j)
              *reinterpret_cast<uint32_t *>(turn + j * kTurnPitch + lane * 4) = pack_bf16x2(v[q * 32 + 2 * j], v[q * 32 + 2 * j + 1]);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint4 x = *reinterpret_cast<const uint4 *>(turn + (pair + 8 * i) * kTurnPitch + c * 4);
              const uint4 y = *reinterpret_cast<const uint4 *>(turn + (pair + 8 * i) * kTurnPitch + c * 4 + 16);
              const int slot = t.slot_at(half, q * 32 + 2 * (pair + 8 * i));   // (and the next: 16 columns are neighbours)
              if (f0 + c < a.n) {
                __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(a.out) + (int64_t)(t.slot0 + slot) * a.n + f0 + c;
                if (slot < t.count)
                  *reinterpret_cast<uint4 *>(out) = make_uint4(__byte_perm(x.x, x.y, 0x5410), __byte_perm(x.z, x.w, 0x5410),
                                                               __byte_perm(y.x, y.y, 0x5410), __byte_perm(y.z, y.w, 0x5410));
                if (slot + 1 < t.count)
                  *reinterpret_cast<uint4 *>(out + a.n) = make_uint4(__byte_perm(x.x, x.y, 0x7632), __byte_perm(x.z, x.w, 0x7632),
                                                                     __byte_perm(y.x, y.y, 0x7632), __byte_perm(y.z, y.w, 0x7632));
              }
            }
          }
        } else if (f0 + lane < a.n) {
#pragma unroll
          for (int q = 0; q < 8; ++q) {            // (16 columns are neighbouring slots)
            const int slot = t.slot_at(half, q * 16), live = q * 16 < n ? t.count - slot : 0;
            if (live <= 0) continue;
            const int64_t to = (int64_t)(t.slot0 + slot) * a.n + f0 + lane;
            if (a.f32) {
              float *out = static_cast<float *>(a.out) + to;
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (j < live) out[(int64_t)j * a.n] = v[q * 16 + j];
            } else {
              __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(a.out) + to;
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (j < live) out[(int64_t)j * a.n] = __float2bfloat16_rn(v[q * 16 + j]);
            }
          }
        }
      } else {
        const int buffer = group * 2 + (taken & 1);
        uint16_t *key = keys + buffer * (8 * 128);
        float h[64];                             // columns 32 (i / 16) + 16 (lane / 16) + i % 16
        if (ok) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (q * 32 < n) {
#pragma unroll
              for (int i = 16 * q; i < 16 * q + 16; i += 2) {
                const float2 s = silu_mul2(make_float2(v[i], v[i + 1]), make_float2(v[64 + i], v[64 + i + 1]));
                h[i] = s.x, h[i + 1] = s.y;
              }
            } else {
#pragma unroll
              for (int i = 16 * q; i < 16 * q + 16; ++i) h[i] = 0.f;
            }
          }
          // the largest over the 16 lanes of a column (NaN counts for nothing): lanes swap what the other half of
          // them will go on with, and end with those of h[4 (lane % 16)] .. h[4 (lane % 16) + 3]
          float m[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const bool high = lane & 8;
            const float other = __shfl_xor_sync(kFull, high ? h[i] : h[32 + i], 8);
            m[i] = fmaxf(fabsf(high ? h[32 + i] : h[i]), fabsf(other));
          }
#pragma unroll
          for (int o = 4, c = 16; o > 0; o >>= 1, c >>= 1)
#pragma unroll
            for (int i = 0; i < c; ++i) {
              const bool high = lane & o;
              const float other = __shfl_xor_sync(kFull, high ? m[i] : m[c + i], o);
              m[i] = fmaxf(high ? m[c + i] : m[i], other);
            }
          uint32_t b[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bits = __float_as_uint(m[i]);
            // (infinity's key is infinity: with the bit that keeps small numbers from being none it would be NaN)
            b[i] = bits > 0x7f800000u ? 0u : min((bits >> 16) | (bits != 0u), 0x7f80u);
          }
          const uint32_t b01 = b[0] | b[1] << 16, b23 = b[2] | b[3] << 16;
          uint16_t *mine = key + (side * 4 + quarter) * 128 + (lane & 12) * 8 + (lane & 16) + (lane & 3) * 4;
          *reinterpret_cast<uint2 *>(mine) = make_uint2(b01, b23);
          asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(cluster_map_shared(smem_u32(mine), side ^ 1)), "r"(b01), "r"(b23)
                       : "memory");
          __syncwarp();
          if (lane < 2) mbar_arrive_cluster(cluster_map_shared(smem_u32(&keys_full[buffer]), lane));
          ok = warp_wait_cluster(&keys_full[buffer], (taken >> 1) & 1u, abort_flag);
          if (!ok && lane == 0) give_up();
        }
        ++taken;
        ok = named_barrier_and(1 + group, 128, ok);  // (they meet below: all go on or none)
        if (!ok) break;
        float *power = powers + group * 128;
        {
          const int column = quarter * 32 + lane, slot = t.slot_at(half, column);  // a slot's scale a thread
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) top = max(top, (uint32_t)key[i * 128 + column]);
          const int e = fp8_exponent(__uint_as_float(top << 16));
          power[column] = fp8_pow2(-e);
          if (side == 0 && column < n && slot < t.count) {
            uint8_t *s = a.out_scales + (int64_t)(t.slot0 + slot) * a.out_sk;
            s[t.ct] = (uint8_t)(e + 127);
            if (t.ct == a.tiles - 1)
              for (int b = a.tiles; b < a.out_sk; ++b) s[b] = 127;  // padding
          }
        }
        named_barrier(1 + group, 128);
        uint8_t *codes = code_rows + group * (128 * 64);
        // (rows of an odd 16 change places with their neighbours, or both halves of a warp would write to the same banks)
        uint8_t *to = codes + (lane & 16) * 64 + quarter * 16 + (lane & 15);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q * 32 < n) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 p = *reinterpret_cast<const float4 *>(power + q * 32 + (lane & 16) + i);
              const int at = 16 * q + i;
              const float2 x = mul2(make_float2(h[at], h[at + 1]), make_float2(p.x, p.y));
              const float2 y = mul2(make_float2(h[at + 2], h[at + 3]), make_float2(p.z, p.w));
              const uint32_t c = fp8_codes4(x.x, x.y, y.x, y.y, 1.f);
#pragma unroll
              for (int j = 0; j < 4; ++j) to[(q * 32 + i + (j ^ (lane >> 4))) * 64] = (uint8_t)(c >> 8 * j);
            }
          }
        named_barrier(1 + group, 128);
        const int c = (lane & 3) * 16, col = t.ct * kTile + side * 64 + c;
        for (int r = quarter * 8 + (lane >> 2); r < n; r += 32) {
          const int slot = t.slot_at(half, r);
          if (slot < t.count && col < a.n)         // (n is a multiple of 16)
            *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(a.out) + (int64_t)(t.slot0 + slot) * a.n + col) =
                *reinterpret_cast<const uint4 *>(codes + (r ^ (r >> 4 & 1)) * 64 + c);
        }
        named_barrier(1 + group, 128);             // (read before the next tile's are written)
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  if (tid == 0) issued_shared = issued;
  cluster_sync_all();                            // (the roles of both CTAs have ended)
  if (warp < 2 && lane == 0) thread_wait(drained, 0u, abort_flag, false);
  __syncwarp();
  if (*abort_flag) {
    // The copies of both CTAs count at the first one's barrier: the CTA that has requested fewer requests what it lacks
    // (nothing reads the stages any more), and the first waits for the last of them to land.
    if (warp == 0) {
      const int theirs = (int)ld_cluster_u32(cluster_map_shared(smem_u32(&issued_shared), side ^ 1));
      for (; issued < theirs; ++issued) {
        const Source from = source_of(cluster + (int64_t)(issued / a.kbs) * clusters);
        if (elect_one()) request(issued % kExpertStages, from, issued % a.kbs, policy_evict_last());
        __syncwarp();
      }
    }
    cluster_sync_all();
    if (tid == 0 && side == 0)
      for (int t = max(0, issued - kExpertStages); t < issued; ++t)
        thread_wait(&full[t % kExpertStages], (uint32_t)(t / kExpertStages) & 1u, abort_flag, false);
    __syncwarp();
    cluster_sync_all();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair<512>(tmem);
  }
}

template <bool kGated>
cudaError_t launch_experts(const RowMaps &tx, const CUtensorMap &tw, const ExpertArgs &a, int dev, cudaStream_t s) {
  static bool done[64] = {};
  static int resident[64] = {};
  constexpr auto kKernel = experts_kernel<kGated>;
  constexpr int kSmem = expert_smem(kGated);
  if (dev < 0 || dev >= 64 || !done[dev]) {
    cudaFuncAttributes f;
    const cudaError_t e = cudaFuncGetAttributes(&f, kKernel);
    if (e != cudaSuccess) return e;
    if (f.numRegs < kLaunchRegs) return cudaErrorLaunchOutOfResources;
  }
  const cudaError_t e = allow_smem(kKernel, kSmem, done, dev);
  if (e != cudaSuccess) return e;
  const int64_t cols = kGated ? a.tiles : (a.tiles + 1) / 2;
  const int64_t most = ((int64_t)a.slots / kTileSlots + std::min(a.slots, a.experts)) * cols;  // tiles at most
  const int64_t pairs = std::min<int64_t>(resident_pairs(kKernel, kSmem, resident, dev), most);
  return launch_after<kKernel>(dim3((unsigned)(2 * pairs)), dim3(kPairThreads), (size_t)kSmem, dim3(2, 1, 1), s, tx, tw, a);
}

// The device's pool for sorted rows: memory is ordered by the stream (a captured call's belongs to its graph) and goes to
// no other stream before its own is known to be done with it.  Up to kKeepBytes stay with the pool, until the last gated
// weights of the device are freed.
constexpr uint64_t kKeepBytes = (uint64_t)1 << 30;
std::atomic<cudaMemPool_t> pools[64];
std::atomic<int> sorting_weights[64];            // by device
cudaMemPool_t row_pool(int dev) {
  if (dev < 0 || dev >= 64) return nullptr;
  cudaMemPool_t pool = pools[dev].load();
  if (pool) return pool;
  cudaMemPoolProps props = {};
  props.allocType = cudaMemAllocationTypePinned;
  props.location.type = cudaMemLocationTypeDevice;
  props.location.id = dev;
  if (cudaMemPoolCreate(&pool, &props) != cudaSuccess) {
    cudaGetLastError();
    return nullptr;
  }
  uint64_t keep = kKeepBytes;
  int no = 0;
  cudaMemPoolSetAttribute(pool, cudaMemPoolAttrReleaseThreshold, &keep);
  for (cudaMemPoolAttr reuse : {cudaMemPoolReuseFollowEventDependencies, cudaMemPoolReuseAllowOpportunistic,
                                cudaMemPoolReuseAllowInternalDependencies})
    cudaMemPoolSetAttribute(pool, reuse, &no);
  cudaMemPool_t first = nullptr;
  if (!pools[dev].compare_exchange_strong(first, pool)) {   // (another thread's came first)
    cudaMemPoolDestroy(pool);
    pool = first;
  }
  return pool;
}

int check_experts(const ham_fp8_weight *w, const void *xc, const void *xs, int64_t slots, const void *offsets,
                  const void *out) {
  if (slots == 0) return HAM_OK;
  if (!xc || !xs || !offsets || !out) return op_fail(HAM_EINVAL, "codes, scales, offsets and the output are required");
  if (!op_aligned(xc, 16) || !op_aligned(out, 16)) return op_fail(HAM_EINVAL, "codes and the output must be 16-byte aligned");
  if (!op_aligned(xs, 4) || !op_aligned(offsets, 4)) return op_fail(HAM_EINVAL, "scales and offsets must be 4-byte aligned");
  return HAM_OK;
}

int run_experts(ham_fp8_weight *w, const void *x_codes, int32_t rows, ExpertArgs a, void *stream) {
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev != w->device) cudaSetDevice(w->device);
  a.ws = w->scales;
  a.err = w->err;
  a.experts = w->experts;
  a.n = w->n;
  a.kbs = w->kbs;
  const int parts = (w->kbs + kExpertPart - 1) / kExpertPart;   // of equal size
  a.part = ((w->kbs + parts - 1) / parts + kGroup - 1) / kGroup * kGroup;
  a.sk = w->sk;
  a.out_sk = fp8_scale_bytes(w->n);
  a.tiles = w->tiles;
  a.wait_ns = w->wait_ns;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  uint8_t *sorted = nullptr;
  // Rows by index, or sorted first?  A copy by index takes its thread some 80 clocks for four rows, a box of neighbouring
  // rows four a row, so that a K block costs some 35 ns more, from 16 slots an expert on 4.5 ns a slot; sorting takes 2.8 us
  // and the rows' bytes twice.  (us by index / sorted, K 4096, 2048 features of 32 experts, 4, 8, 16, 24, 32, 64, 128 slots
  // an expert in the mean: 88.3 / 84.6, 95.9 / 91.0, 100.5 / 92.7, 113.8 / 93.3, 122.6 / 93.6, 162.3 / 97.5, 237.5 / 111.4; K 1024, 512
  // features of 16, 16, 32, 64, 96 slots: 11.8 / 14.9, 12.8 / 15.5, 16.0 / 17.0, 17.6 / 17.3.)
  const int64_t blocks = (int64_t)std::min(a.slots, a.experts) * a.tiles * a.kbs / (device_sms() / 2);  // a pair's
  const int64_t more_ns = blocks * std::max<int64_t>(35, (int64_t)a.slots * 9 / (2 * a.experts));
  if (a.gather && more_ns > 2800 + (int64_t)a.slots * w->k / 3400) {
    const size_t codes = (size_t)a.slots * w->k, scales = (size_t)a.slots * w->sk;
    cudaMemPool_t pool = row_pool(w->device);
    if (pool && cudaMallocFromPoolAsync(reinterpret_cast<void **>(&sorted), codes + scales, pool, s) != cudaSuccess) {
      cudaGetLastError();
      sorted = nullptr;                            // (by index, then)
    }
    if (sorted) {
      e = launch_after<sort_rows_kernel>(dim3((unsigned)((a.slots + kSortWarps - 1) / kSortWarps)), dim3(kSortWarps * 32), 0, dim3(1), s,
                                         static_cast<const uint4 *>(x_codes), reinterpret_cast<const uint32_t *>(a.xs), a.order,
                                         a.offsets, a.experts, a.slots, a.top_k, w->k / 16, w->sk / 4,
                                         reinterpret_cast<uint4 *>(sorted), reinterpret_cast<uint32_t *>(sorted + codes), a.err);
      x_codes = sorted;
      a.xs = sorted + codes;
      a.gather = 0;
      rows = a.slots;
    }
  }
  RowMaps tx;
  int rc = HAM_OK;
  a.boxes = a.gather || a.slots <= 32 ? 1 : a.slots <= 64 ? 2 : 3;   // (a CTA's rows: half of the slots' next 32, 112 at most)
  for (int i = 0; i < a.boxes; ++i)
    if (make_bytes_tensor_map(&tx.of[i], x_codes, rows, w->k, kFp8Block, a.gather ? 1 : 16 << i) != 0)
      rc = op_fail(HAM_ECUDA, "tensor map of the rows");
  if (rc == HAM_OK && e == cudaSuccess)
    e = w->parts == 2 ? launch_experts<true>(tx, w->map, a, w->device, s) : launch_experts<false>(tx, w->map, a, w->device, s);
  if (sorted) cudaFreeAsync(sorted, s);
  if (rc == HAM_OK && e != cudaSuccess) rc = op_fail(HAM_ECUDA, "experts launch: %s", cudaGetErrorString(e));
  if (dev != w->device) cudaSetDevice(dev);
  return rc;
}

}  // namespace

void experts_weight_freed(int dev) {
  if (dev < 0 || dev >= 64 || --sorting_weights[dev] != 0) return;
  const cudaMemPool_t pool = pools[dev].load();
  if (!pool) return;
  // (memory whose use has not ended would stay with the pool)
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemPoolTrimTo(pool, 0) != cudaSuccess) cudaGetLastError();
}

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
  if (blocks > ((int64_t)1 << 41) / ham::kBlockBytes / experts) {
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
  if (codes_up && w->device >= 0 && w->device < 64) {
    ham::row_pool(w->device);                    // (not first in a call, which may be captured)
    ++ham::sorting_weights[w->device];
    w->sorts = true;
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
  a.xs = static_cast<const uint8_t *>(x_scales);
  a.offsets = offsets;
  a.order = order;
  a.gather = 1;
  a.top_k = top_k;
  a.slots = (int)slots;
  a.out = codes;
  a.out_scales = static_cast<uint8_t *>(scales);
  return ham::run_experts(w, x_codes, rows, a, stream);
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
  a.xs = static_cast<const uint8_t *>(x_scales);
  a.offsets = offsets;
  a.top_k = 1;
  a.slots = slots;
  a.out = out;
  a.f32 = f32;
  return ham::run_experts(w, x_codes, slots, a, stream);
}

}  // extern "C"

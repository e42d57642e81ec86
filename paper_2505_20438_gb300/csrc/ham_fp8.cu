// Products with 8-bit weights (e4m3 codes, a power-of-two scale for each 128 x 128 block) of 8-bit
// rows (a scale for each 128 elements), on the block-scaled tensor-core products of sm_103a, and the
// first half of a gated feed-forward block made of two of them:
//
//   Y[t][n] = sum_b 2^(sx[t][b] + sw[n / 128][b] - 254) sum_{k in block b} X[t][k] W[n][k]
//   H[t][f] = silu(G[t][f]) U[t][f],  G = X W_g^T, U = X W_u^T,  encoded as 8-bit rows
//
// The scales are E8M0 bytes, so tcgen05 kind::mxf8f6f4 applies them inside the product (its scale
// blocks are 32 elements of K: four products of a 128-block use the same byte) and sums stay in fp32
// accumulators in tensor memory.  Four consecutive blocks' bytes are one 32-bit word of a row; a word serves
// four K steps, the instruction descriptor selecting the byte, so that the scales of an operand tile are
// copied to tensor memory (512 bytes a copy) once every four steps.
//
// The tensor cores add 32 terms of K exactly to the fp32 sum and cut the result off at its last place, toward
// zero, so that one accumulator's error is a bias that grows with K: measured against 64-bit sums, relative to
// the outputs' norm, 5.9e-8 at K 1024, 1.1e-7 at 2048, 2.3e-7 at 4096, 1.3e-6 at 16384 (a plain fp32 product:
// 4.1e-8, 5.9e-8, 8.6e-8, 2.0e-7).  So an accumulator takes kSumNext blocks of K, 1024 terms (the pair kernel's first
// in a tile kSumFirst; the streaming kernel's up to kSumMost where more accumulators would cost a CTA an SM), and the
// parts are added in fp32, in order: 0.9 to 1.1e-7 at every K from 2048 on with the pair kernel, 0.5 to 0.9e-7 with the
// streaming one (up to 2.4e-7 where its accumulators are few).
//
// Weights are laid out once (ham_fp8_weight_alloc) as [tile of 128 rows][K block][128 x 128], each
// block 16 KiB in the shared-memory layout of the 128-byte swizzle, so that a weight tile's K range is
// one contiguous stretch of memory (a gated weight: gate and up block after block).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>
#include <new>

#include "ham_mx.cuh"
#include "ham_ops.cuh"

struct ham_fp8_weight {
  int32_t n = 0, k = 0, parts = 1;   // parts: 2 for a gated weight (gate, up)
  int32_t tiles = 0, kbs = 0, sk = 0;
  int device = 0;
  uint8_t *codes = nullptr;    // [tiles][kbs][parts][128 x 128 swizzled], and behind them in the same allocation
  uint8_t *scales = nullptr;   // [tiles][parts][sk]
  int32_t *err = nullptr;      // the device error word
  uint64_t wait_ns = ham::kWaitLimitNs;  // limit of the kernels' waits
  CUtensorMap map;             // codes as one stretch, boxes of half a block
};

namespace ham {
namespace {

constexpr int kTile = 128;             // weight rows of a tile
constexpr int kSumFirst = 16, kSumNext = 8, kSumMost = 32;  // K blocks of one accumulator
constexpr int kBlockBytes = 128 * 128; // a tile's K block

// One thread per 16-byte piece of the laid-out weight.
__global__ void lay_out_weight_kernel(const uint8_t *__restrict__ codes, int n, int k, int part, int parts,
                                      int kbs, int64_t pieces, uint8_t *__restrict__ dst) {
  const int64_t p = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (p >= pieces) return;
  const int in = (int)(p % (kBlockBytes / 16)), r = in / 8, c = in % 8;
  const int64_t block = p / (kBlockBytes / 16);  // tile * kbs + kb
  const int64_t row = block / kbs * kTile + r;
  const int col = (int)(block % kbs) * kFp8Block + 16 * c;
  uint4 v = make_uint4(0, 0, 0, 0);
  if (row < n && col < k) v = *reinterpret_cast<const uint4 *>(codes + row * k + col);
  *reinterpret_cast<uint4 *>(dst + (block * parts + part) * kBlockBytes + r * 128 + ((c ^ (r & 7)) << 4)) = v;
}
__global__ void lay_out_scales_kernel(const uint8_t *__restrict__ scales, int tiles, int sk, int part,
                                      int parts, uint8_t *__restrict__ dst) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < tiles * sk) dst[((int64_t)(i / sk) * parts + part) * sk + i % sk] = scales[i];
}

// Shared memory that a CTA with `cols` columns of tensor memory asks for at least, in kernels whose CTAs
// wait for one another: an SM's 228 KB then run out before its 512 columns do, so that no CTA of a
// cluster ever waits for columns that a CTA of another cluster holds (two clusters could otherwise each
// hold what the other waits for).
constexpr int smem_floor(int cols) { return (228 * 1024 * (cols / 32) + 16) / 17; }

struct ProductArgs {
  const uint8_t *w, *ws;   // the handle's layout
  const uint8_t *xs;       // [rows][sk]
  void *out;               // [rows][n], or [rows][n] codes of a gated product
  uint8_t *out_scales;     // gated: [rows][out_sk]
  int32_t *err;
  int rows, n, kbs, sk, out_sk;
  int part, first_part;    // K blocks that one accumulator takes; of the pair kernel's first one in a tile
  int sums;                // the streaming kernel: accumulators
  int nt, box;             // the streaming kernel: rows of X a CTA takes (a multiple of 16), rows it loads
  int stages, stage_bytes, tmem_cols;
  int tiles;               // weight tiles
  uint64_t wait_ns;        // limit of the waits that may be shortened (the others end with them)
  int f32;                 // fp32 output
};

__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.f + expf(-g)) * u; }

// Four neighbouring outputs of one row from column c (a multiple of 4), within the row's n.
__device__ __forceinline__ void store4(const ProductArgs &a, int64_t row, int c, float4 v) {
  const int64_t at = row * a.n + c;
  if (c + 4 <= a.n && (a.n & 3) == 0) {
    if (a.f32)
      *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = v;
    else
      *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) =
          make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    return;
  }
  const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < a.n) {
      if (a.f32) static_cast<float *>(a.out)[at + i] = f[i];
      else static_cast<__nv_bfloat16 *>(a.out)[at + i] = __float2bfloat16_rn(f[i]);
    }
}

// ------------------------------------------------------------------------------------
// Few rows: the weights stream
// ------------------------------------------------------------------------------------
// A CTA multiplies one weight tile's (128 rows: the product's M; gated: the gate's and the up's tile)
// K range with nt rows of X (its N).  The K blocks are cut over the CTAs of a cluster, which add their
// fp32 accumulators through distributed shared memory, in the order of the ranges.  Weight blocks are
// requested before the dependency wait: nothing on the stream writes them.
//
// Bound by the weights' bytes where there are enough of them: the head of 128256 features of 4096 for 64 rows
// takes 85.6 us (96% of the copy rate), a gated half of 16384 features for 8 rows 23.4 to 24.4 (82 to 85%), 14.9
// for 8 rows of 16384 in 4096 (66%).  A 4096 x 4096 weight, 16 MB, takes 7.1 us against 2.5 at that rate: the chain
// of launch, first blocks, products, the cluster's sums and stores stands alone.
constexpr int kStreamThreads = 256;
constexpr int kStreamSf = 4;            // scale slots (of four K blocks each)
constexpr int kStreamSmem2 = 104 * 1024; // shared memory of a CTA: two share an SM
constexpr int kStreamSmem3 = 72 * 1024;  // ... three

constexpr int kStreamStages = 12;       // at most
constexpr int kStreamBars = (2 * kStreamStages + 2 * kStreamSf + 1) * 8;
// Bytes of a scale slot (the weight tiles', the rows') and of everything beside the ring.
__host__ __device__ constexpr int stream_sf_bytes(int parts) { return (parts + 1) * 512; }
constexpr int stream_sf_columns(int parts) { return 2 * (parts + 1) * 4; }
// Accumulators that `columns` of tensor memory hold beside the scales.
constexpr int stream_sums(int parts, int nt, int columns) { return (columns - stream_sf_columns(parts)) / (parts * nt); }
constexpr int kMaxSplits = 8;
constexpr int stream_fixed(int parts) { return 1024 + kStreamSf * stream_sf_bytes(parts) + kStreamBars; }

template <int kParts>
__global__ void __launch_bounds__(kStreamThreads)
    fp8_stream_kernel(const __grid_constant__ CUtensorMap tx, ProductArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *sf = ring + (size_t)a.stages * a.stage_bytes;
  uint64_t *full = reinterpret_cast<uint64_t *>(sf + kStreamSf * stream_sf_bytes(kParts));
  uint64_t *empty = full + kStreamStages, *sf_full = empty + kStreamStages;
  uint64_t *sf_empty = sf_full + kStreamSf, *acc_full = sf_empty + kStreamSf;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_shared;
  volatile int *abort_flag = &abort_shared;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int tile = blockIdx.x, splits = gridDim.y, rank = blockIdx.y;  // a cluster: the splits
  // The CTA's rows begin at row n0 and are loaded from row x0 on: a part that would pass the last row
  // begins earlier instead, since a copy's rows past the end cost more than others (gated, 16384
  // features of 4096: 300 rows took 67 us, 512 rows 50).
  const int n0 = blockIdx.z * a.nt, x0 = min(n0, a.rows - a.box);
  const int kb0 = (int)((int64_t)rank * a.kbs / splits), kb1 = (int)((int64_t)(rank + 1) * a.kbs / splits);
  const int nk = kb1 - kb0, stages = a.stages;
  const int g0 = kb0 >> 2;                            // first scale word
  const int ng = ((kb1 + 3) >> 2) - g0;
  if (tid == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < kStreamSf; ++s) {
      mbar_init(&sf_full[s], 1);
      mbar_init(&sf_empty[s], 1);
    }
    mbar_init(acc_full, 1);
    abort_shared = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) prefetch_tensormap(&tx);
  __syncthreads();
  // Tensor memory is taken before the dependency wait (after it, 1.3 us of a call of 6.5 were spent on
  // it) and before the next kernel may start: a kernel that holds columns and waits for this one while
  // this one still wants some would keep both waiting.  Of the kernels that may still run before this
  // one, those that take columns do so before they let anything start, or fill their SMs' shared memory.
  if (warp > 0) {
    if (warp == 1) tmem_alloc_n(&tmem_slot, (uint32_t)a.tmem_cols);
    tc_fence_before();
    named_barrier(1, kStreamThreads - 32);
    tc_fence_after();
    grid_dependency_wait();  // (bounded waits count from here: the kernel before may still have run long)
  }
  int issued = 0;

  if (warp == 0) {
    // ------------------------------------------------------------ copies
    if (lane == 0) {
      const uint64_t pol_x = policy_evict_last();
      const uint8_t *src = a.w + ((int64_t)tile * a.kbs + kb0) * (kParts * kBlockBytes);
      const int xbytes = a.box * 128;
      auto load_w = [&](int t, int s) {
        mbar_arrive_tx(&full[s], (uint32_t)(kParts * kBlockBytes + xbytes));
        bulk_load(ring + s * a.stage_bytes, src + (int64_t)t * (kParts * kBlockBytes),
                  (uint32_t)(kParts * kBlockBytes), &full[s]);
      };
      const int pre = min(stages, nk);
      for (int t = 0; t < pre; ++t) load_w(t, t);
      grid_dependency_wait();
      for (int t = 0; t < nk; ++t) {
        const int s = t % stages;
        if (t >= pre) {
          if (!thread_wait(&empty[s], (uint32_t)(t / stages - 1) & 1u, abort_flag, true, a.wait_ns)) break;
          load_w(t, s);
        }
        tma_load_2d(ring + s * a.stage_bytes + kParts * kBlockBytes, &tx, (kb0 + t) * kFp8Block, x0, &full[s],
                    pol_x);
        issued = t + 1;
      }
      if (issued < nk && !*abort_flag) {
        record_error(a.err, HAM_DEVERR_TIMEOUT);
        *abort_flag = 1;
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ products
    const uint32_t tmem = *const_cast<volatile uint32_t *>(&tmem_slot);
    const uint32_t sf_tmem = tmem + a.sums * kParts * a.nt;  // two buffers of (kParts + 1) * 4 columns
    uint32_t acc = tmem;
    int in = 0;                                       // blocks of the accumulator so far
    bool ok = true;
    for (int t = 0; t < nk; ++t) {
      const int s = t % stages, kb = kb0 + t, g = (kb >> 2) - g0;
      const bool first = t == 0 || (kb & 3) == 0;     // a new scale word
      const uint32_t sft = sf_tmem + (uint32_t)((g & 1) * (kParts + 1) * 4);
      if (first && !warp_wait(&sf_full[g % kStreamSf], (uint32_t)(g / kStreamSf) & 1u, abort_flag, a.wait_ns)) { ok = false; break; }
      if (!warp_wait(&full[s], (uint32_t)(t / stages) & 1u, abort_flag, a.wait_ns)) { ok = false; break; }
      if (elect_one()) {
        tc_fence_after();
        if (first) {
          const uint32_t from = smem_u32(sf + (g % kStreamSf) * stream_sf_bytes(kParts));
#pragma unroll
          for (int p = 0; p <= kParts; ++p) tc_copy_scales<1>(sft + p * 4, from + p * 512);
          tc_commit(&sf_empty[g % kStreamSf]);
        }
        const uint32_t wa = smem_u32(ring + s * a.stage_bytes), xa = wa + kParts * kBlockBytes;
        const uint32_t idesc = idesc_mx(kTile, a.nt, kb & 3);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int p = 0; p < kParts; ++p)
            tc_mma_mx<1>(acc + p * a.nt, smem_desc_sw128(wa + p * kBlockBytes + kk * 32, 16, 1024),
                         smem_desc_sw128(xa + kk * 32, 16, 1024), idesc, sft + p * 4, sft + kParts * 4,
                         in > 0 || kk > 0);
        tc_commit(&empty[s]);
      }
      __syncwarp();
      if (++in == a.part) in = 0, acc += kParts * a.nt;
    }
    if (!ok && lane == 0 && !*abort_flag) {
      record_error(a.err, HAM_DEVERR_TIMEOUT);
      *abort_flag = 1;
    }
    __syncwarp();
    if (elect_one()) tc_commit(acc_full);  // also after an abort: what was issued completes
    __syncwarp();
  } else if (warp == 2) {
    // ------------------------------------------------------------ scale words
    uint32_t w[kParts];
#pragma unroll
    for (int p = 0; p < kParts; ++p) w[p] = 0;
    grid_launch_dependents();
    for (int g = 0; g < ng; ++g) {
      const int slot = g % kStreamSf;
      uint32_t x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = lane + 32 * j;
        x[j] = 0x7f7f7f7fu;
        if (r < a.box)
          x[j] = __ldg(reinterpret_cast<const uint32_t *>(a.xs + (int64_t)(x0 + r) * a.sk) + g0 + g);
      }
#pragma unroll
      for (int p = 0; p < kParts; ++p)
        w[p] = __ldg(reinterpret_cast<const uint32_t *>(a.ws + ((int64_t)tile * kParts + p) * a.sk) + g0 + g);
      if (g >= kStreamSf &&
          !warp_wait(&sf_empty[slot], (uint32_t)(g / kStreamSf - 1) & 1u, abort_flag, a.wait_ns)) {
        if (lane == 0 && !*abort_flag) {
          record_error(a.err, HAM_DEVERR_TIMEOUT);
          *abort_flag = 1;
        }
        break;
      }
      uint4 *dst = reinterpret_cast<uint4 *>(sf + slot * stream_sf_bytes(kParts)) + lane;
#pragma unroll
      for (int p = 0; p < kParts; ++p) dst[p * 32] = make_uint4(w[p], w[p], w[p], w[p]);
      dst[kParts * 32] = make_uint4(x[0], x[1], x[2], x[3]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sf_full[slot]);
    }
  }

  // ---------------------------------------------------------------- epilogue (every warp)
  // Accumulators -> shared memory [part][row][128 features] (the ring, free by now), then each CTA of
  // the cluster adds its share of the rows: a warp a row, a lane four features.
  __syncwarp();
  bool ok = warp_wait(acc_full, 0u, abort_flag);  // (ends with the others, whose limit may be shorter)
  if (!ok && lane == 0 && !*abort_flag) {
    record_error(a.err, HAM_DEVERR_TIMEOUT);
    *abort_flag = 1;
  }
  ok = ok && !__any_sync(kFull, *abort_flag != 0);
  const uint32_t tmem = *const_cast<volatile uint32_t *>(&tmem_slot);
  float *acc = reinterpret_cast<float *>(ring);
  if (ok) {
    tc_fence_after();
    const int quarter = warp & 3, sums = (nk + a.part - 1) / a.part;  // accumulators in use
    const uint32_t t_row = tmem + ((uint32_t)(quarter * 32) << 16);
    for (int c = (warp >> 2) * 16; c < kParts * a.nt; c += 32) {
      float v[16];
      tmem_ld16(t_row + c, *reinterpret_cast<uint32_t(*)[16]>(v));
      tmem_wait_ld();
      for (int i = 1; i < sums; ++i) {
        float u[16];
        tmem_ld16(t_row + i * kParts * a.nt + c, *reinterpret_cast<uint32_t(*)[16]>(u));
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] += u[j];
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[(c + j) * kTile + quarter * 32 + lane] = v[j];
    }
  }
  tc_fence_before();
  if (splits > 1) cluster_sync_all();
  else __syncthreads();
  if (warp == 1) {
    if (!ok && lane == 0) thread_wait(acc_full, 0u, abort_flag, false);  // products in flight
    __syncwarp();
    tc_fence_after();
    tmem_dealloc_n(tmem, (uint32_t)a.tmem_cols);
  }
  if (ok) {
    const uint32_t base = smem_u32(acc) + lane * 16;
    for (int r = n0 - x0 + rank * 8 + warp; r < a.box; r += splits * 8) {
      float4 v[kParts];
#pragma unroll
      for (int p = 0; p < kParts; ++p) {
        const uint32_t at = base + (uint32_t)((p * a.nt + r) * kTile * 4);
        if (splits == 1) {
          v[p] = *reinterpret_cast<const float4 *>(acc + (p * a.nt + r) * kTile + lane * 4);
        } else {
          v[p] = ld_cluster_f4(cluster_map_shared(at, 0));
          for (int q = 1; q < splits; ++q) {
            const float4 o = ld_cluster_f4(cluster_map_shared(at, q));
            v[p].x += o.x, v[p].y += o.y, v[p].z += o.z, v[p].w += o.w;
          }
        }
      }
      const int c = tile * kTile + lane * 4;
      if constexpr (kParts == 1) {
        if (c < a.n) store4(a, x0 + r, c, v[0]);
      } else {
        const float h[4] = {silu_mul(v[0].x, v[1].x), silu_mul(v[0].y, v[1].y), silu_mul(v[0].z, v[1].z),
                            silu_mul(v[0].w, v[1].w)};
        const float m = warp_max_f32(fmaxf(fmaxf(fabsf(h[0]), fabsf(h[1])), fmaxf(fabsf(h[2]), fabsf(h[3]))));
        const int e = fp8_exponent(m);
        if (c < a.n)  // (n is a multiple of 16; features past it are zeros)
          *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(a.out) + (int64_t)(x0 + r) * a.n + c) =
              fp8_codes4(h[0], h[1], h[2], h[3], fp8_pow2(-e));
        uint8_t *s = a.out_scales + (int64_t)(x0 + r) * a.out_sk;
        if (lane == 0) s[tile] = (uint8_t)(e + 127);
        else if (tile == a.tiles - 1 && lane < a.out_sk - tile) s[tile + lane] = 127;  // padding
      }
    }
  }
  if (splits > 1) cluster_sync_all();  // (a peer may still read this CTA's accumulators)
  if (tid == 0 && *abort_flag)  // after an abort, this CTA's copies land before it exits
    for (int t = max(0, issued - stages); t < issued; ++t)
      thread_wait(&full[t % stages], (uint32_t)(t / stages) & 1u, abort_flag, false);
}

// ------------------------------------------------------------------------------------
// Many rows: pairs of CTAs, tiles of 256 x 256
// ------------------------------------------------------------------------------------
// A pair of CTAs (cta_group::2) computes 256 rows of X by two weight tiles (a gated weight: the gate's
// and the up's tile of the same features): each CTA holds 128 of the rows (its lanes of tensor memory)
// and loads its rows and half of the weight rows, into its own shared memory alone (the library is also what
// every rank of a job on several GPUs loads, so no load here is a cluster multicast).  The pairs are
// persistent.
//
// The tile's sums are two accumulators of 128 columns each, of three in tensor memory: one takes a group of
// two K blocks, then the other takes them, so that a part of K ends in the first a group's products before it
// ends in the second, the first of the next part has an accumulator of its own at once, and the second takes
// the one that the epilogue has emptied meanwhile.  With one accumulator of 256 columns, two of which share
// 64, a part cost 0.6 to 0.9 us more.  (Groups of four blocks, which hold most of the ring, took 4096 x 16384
// x 4096 from 172 to 205 us.)  The epilogue holds the sums of the parts before in registers.  A tile's first part is
// the longer one, since the epilogue of the tile before still runs beside it: with parts of 12 and 8 blocks the
// gated 4096 x 4096 x 16384 took 320 us instead of 306, with 8 alone 344, with 16 alone 305.
//
// Bound by the tensor cores: 8192 rows, K 4096, 6144 features 120 us (3.44 PFLOP/s, 89% of twice the measured
// bf16 rate), 4096 rows, K 16384, 4096 features 172 us (83%), gated 4096 rows of 4096 in 16384 features
// 305 to 310 us (92 to 94%); run without a break the card's power limit makes that 141, 196 and 362 us.  Few
// tiles leave pairs without work in the last round, and the first tile's loads and the last one's epilogue
// stand alone (2048 rows, 4096 x 4096: 27 us, 66%).  With one accumulator for all of K these took 119, 169,
// 302 and 26.5 us; a pair takes 64 bytes a clock an SM from L2 at the products' full rate.
constexpr int kPairThreads = 384;       // warps: copies, products, 2 x scales, 8 x epilogue
// Registers a thread: the launch's, and from the roles on those of the first four warps and of the epilogue's
// eight, which hold a tile's sums in 128 of them.  Together they are what the launch has: a kernel compiled
// to fewer would wait for the rest forever, so the host looks before it launches one.
constexpr int kLaunchRegs = 168, kFewRegs = 56, kManyRegs = 224;
static_assert(4 * kFewRegs + 8 * kManyRegs <= 12 * kLaunchRegs && kPairThreads == 384, "registers");
constexpr int kPairStages = 6;
constexpr int kPairStageBytes = 2 * kBlockBytes;
constexpr int kPairSf = 4;
constexpr int kPairSfBytes = 3 * 512;   // the CTA's 128 rows, the weight rows of both halves
constexpr int kPairSums = 3, kPairSfCol = 448;  // accumulators of 128 columns, then the scales
constexpr int kGroup = 2;               // K blocks that one accumulator takes, then the other
constexpr int kTurn = 17;               // floats a row of a warp's turning space: 16 columns, padded
constexpr int kPairUsed = 1024 + kPairStages * kPairStageBytes + kPairSf * kPairSfBytes + 256 + 8 * 32 * kTurn * 4;
constexpr int kPairSmem = kPairUsed > smem_floor(512) ? kPairUsed : smem_floor(512);
static_assert(kPairSmem <= 226 * 1024, "shared memory");

// 32 accumulator columns (from column c of n) of a warp's 32 rows (those from own0 on), a row a lane, to the
// output through shared memory, 16 columns at a time, so that neighbouring lanes write neighbours, kEach
// elements each: what n is a multiple of, up to 16 bytes.  Loads from shared memory are issued four at a time,
// before their stores.  (3344 rows, K 544, some 15550 features, which the outputs bound: bf16 35 us straight,
// turned 50 with 8 elements, 60 with 4, 71 with 1 (89 with the loads one by one); fp32 53, and 55 with 4.
// 16 bytes a lane straight from the registers took 57 and 117; a value at a time, a row a lane, 164 for 3000 x
// 5003 outputs of 2000 columns that take 38 turned.)
template <int kEach, bool kF32>
__device__ __forceinline__ void store_turned(const ProductArgs &a, int row0, int own0, int c, const float *f, float *turn) {
  constexpr int kLanes = 16 / kEach;             // a row's
  constexpr int kSteps = 16 / kEach, kAtOnce = kSteps < 4 ? kSteps : 4;
  const int lane = threadIdx.x & 31, at = lane % kLanes * kEach;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 16; ++j) turn[lane * kTurn + j] = f[16 * h + j];
    __syncwarp();
    const int col = c + 16 * h + at;
#pragma unroll
    for (int i0 = 0; i0 < kSteps; i0 += kAtOnce) {
      const int r0 = i0 * 2 * kEach + lane / kLanes;
      float x[kAtOnce][kEach];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[i][j] = turn[(r0 + i * 2 * kEach) * kTurn + at + j];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int row = row0 + r0 + i * 2 * kEach;
        if (row < own0 || col >= a.n) continue;
        const int64_t to = (int64_t)row * a.n + col;
        if constexpr (kF32) {
          float *y = static_cast<float *>(a.out) + to;
          if constexpr (kEach == 1) *y = x[i][0];
          if constexpr (kEach == 2) *reinterpret_cast<float2 *>(y) = make_float2(x[i][0], x[i][1]);
          if constexpr (kEach == 4) *reinterpret_cast<float4 *>(y) = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
        } else {
          __nv_bfloat16 *y = static_cast<__nv_bfloat16 *>(a.out) + to;
          if constexpr (kEach == 1) *y = __float2bfloat16_rn(x[i][0]);
          if constexpr (kEach == 2) *reinterpret_cast<uint32_t *>(y) = pack_bf16x2(x[i][0], x[i][1]);
          if constexpr (kEach == 4)
            *reinterpret_cast<uint2 *>(y) = make_uint2(pack_bf16x2(x[i][0], x[i][1]), pack_bf16x2(x[i][2], x[i][3]));
          if constexpr (kEach == 8)
            *reinterpret_cast<uint4 *>(y) = make_uint4(pack_bf16x2(x[i][0], x[i][1]), pack_bf16x2(x[i][2], x[i][3]),
                                                       pack_bf16x2(x[i][4], x[i][5]), pack_bf16x2(x[i][6], x[i][7]));
        }
      }
    }
  }
}
// The same in units of what n is a multiple of.
__device__ __forceinline__ void store_turned(const ProductArgs &a, int row0, int own0, int c, const float *f, float *turn) {
  if (a.f32) {
    if ((a.n & 3) == 0) store_turned<4, true>(a, row0, own0, c, f, turn);
    else if ((a.n & 1) == 0) store_turned<2, true>(a, row0, own0, c, f, turn);
    else store_turned<1, true>(a, row0, own0, c, f, turn);
  } else {
    if ((a.n & 7) == 0) store_turned<8, false>(a, row0, own0, c, f, turn);
    else if ((a.n & 3) == 0) store_turned<4, false>(a, row0, own0, c, f, turn);
    else if ((a.n & 1) == 0) store_turned<2, false>(a, row0, own0, c, f, turn);
    else store_turned<1, false>(a, row0, own0, c, f, turn);
  }
}
// The same straight from the registers, 32 bytes at a time a lane, where rows begin at multiples of them.
__device__ __forceinline__ void store_straight(const ProductArgs &a, int row, int own0, int c, const float *f) {
  if (row < own0) return;
  char *dst = static_cast<char *>(a.out) + ((int64_t)row * a.n + c) * (a.f32 ? 4 : 2);
  if (a.f32) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(f[8 * q + j]);
      if (c + 8 * q < a.n) st_global_32(dst + 32 * q, w);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = pack_bf16x2(f[16 * q + 2 * j], f[16 * q + 2 * j + 1]);
      if (c + 16 * q < a.n) st_global_32(dst + 32 * q, w);
    }
  }
}

// kMore: K may be several accumulators' (a plain product of one needs no registers for sums, and stores
// straight from the accumulator; a gated one holds its 128 values a thread in any case).
template <bool kGated, bool kMore>
__global__ void __launch_bounds__(kPairThreads, 1)
    fp8_pair_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw,
                    ProductArgs a, int row_tiles, int col_tiles) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *sf = ring + kPairStages * kPairStageBytes;
  // full, sf_full and sum_free: the ones of a pair's first CTA are used
  uint64_t *full = reinterpret_cast<uint64_t *>(sf + kPairSf * kPairSfBytes);
  uint64_t *empty = full + kPairStages;
  uint64_t *sf_full = empty + kPairStages;     // an arrival a CTA
  uint64_t *sf_empty = sf_full + kPairSf;
  uint64_t *sum_full = sf_empty + kPairSf;     // [half][every other part of K]
  uint64_t *sum_free = sum_full + 4;           // the same: an arrival a warp of the pair that takes the half
  uint64_t *drained = sum_free + 4;            // every product issued is complete
  static_assert((2 * kPairStages + 2 * kPairSf + 9) * 8 <= 256, "barriers");
  float *turn = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(full) + 256);  // [8 warps][32][kTurn]
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_shared, issued_shared;
  __shared__ float row_max[2][128];            // gated: largest magnitude of a row's half
  volatile int *abort_flag = &abort_shared;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int side = (int)cluster_rank();
  const uint32_t both = 3u;
  const int clusters = gridDim.x / 2, cluster = blockIdx.x / 2, total = row_tiles * col_tiles;
  // This CTA's 128 rows of row tile rt: the tile's, but none past the last (as in the streaming kernel,
  // a tile that would pass it begins earlier); an odd last weight tile has no second, so its own is loaded
  // twice.
  auto row_of = [&](int rt) { return min(rt * 256 + side * 128, a.rows - 128); };
  // A wait ran out (or the pair has given up already): both CTAs stop.
  const auto give_up = [&] {
    if (*abort_flag) return;
    record_error(a.err, HAM_DEVERR_TIMEOUT);
    *abort_flag = 1;
    st_cluster_u32(cluster_map_shared(smem_u32(&abort_shared), side ^ 1), 1u);
  };
  // Where tile w begins: this CTA's rows, and K block 0 of the weight's two stretches of 64 rows that it takes, one
  // a half of the sums: plain, its half of each tile (so that a half of the sums is a tile); gated, of the gate's
  // or the up's tile.
  struct Source { int x, w0, w1; };
  const auto source_of = [&](int w) {
    constexpr int kRows = kBlockBytes / 2048;    // of a block in the map
    const int ct = w / row_tiles;
    Source from{row_of(w % row_tiles), 0, 0};
    if constexpr (kGated) {
      from.w0 = (ct * a.kbs * 2 + side) * kRows;
      from.w1 = from.w0 + kRows / 2;
    } else {
      from.w0 = min(ct * 2, a.tiles - 1) * a.kbs * kRows + side * (kRows / 2);
      from.w1 = min(ct * 2 + 1, a.tiles - 1) * a.kbs * kRows + side * (kRows / 2);
    }
    return from;
  };
  // Request a tile's K block kb for stage s; the bytes of both CTAs count at the first one's barrier.
  const auto request = [&](int s, const Source &from, int kb, uint64_t pol) {
    if (side == 0) mbar_arrive_tx(&full[s], 2 * kPairStageBytes);
    const uint32_t bar = cluster_map_shared(smem_u32(&full[s]), 0);
    uint8_t *dst = ring + s * kPairStageBytes;
    const int down = kb * (kGated ? 2 : 1) * (kBlockBytes / 2048);
    tma_load_2d_pair(dst, &tx, kb * kFp8Block, from.x, bar, pol);
    tma_load_2d_pair(dst + kBlockBytes, &tw, 0, from.w0 + down, bar, pol);
    tma_load_2d_pair(dst + kBlockBytes + kBlockBytes / 2, &tw, 0, from.w1 + down, bar, pol);
  };
  if (tid == 0) {
    for (int s = 0; s < kPairStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < kPairSf; ++s) {
      mbar_init(&sf_full[s], 2);
      mbar_init(&sf_empty[s], 1);
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(&sum_full[s], 1);
      mbar_init(&sum_free[s], 8);
    }
    mbar_init(drained, 1);
    abort_shared = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) {
    prefetch_tensormap(&tx);
    prefetch_tensormap(&tw);
  }
  cluster_sync_all();
  if (warp > 0) {  // (tensor memory: as in the streaming kernel)
    if (warp == 1) tmem_alloc_pair<512>(&tmem_slot);
    tc_fence_before();
    named_barrier(5, kPairThreads - 32);
    tc_fence_after();
    grid_dependency_wait();
  }
  const uint32_t tmem = *const_cast<volatile uint32_t *>(&tmem_slot);  // (not warp 0's)
  int issued = 0;
  if (warp < 4) {
    if constexpr (kMore) setmaxnreg_dec<kFewRegs>();
    if (warp == 0) {
      // ------------------------------------------------------------ copies
      if (lane == 0) {
        const uint64_t pol = policy_evict_last();
        grid_dependency_wait();
        bool ok = true;
        int it = 0;
        for (int w = cluster; w < total && ok; w += clusters) {
          const Source from = source_of(w);
          for (int kb = 0; kb < a.kbs; ++kb, ++it) {
            if (it >= kPairStages &&
                !thread_wait(&empty[it % kPairStages], (uint32_t)(it / kPairStages - 1) & 1u, abort_flag, true)) {
              ok = false;
              break;
            }
            request(it % kPairStages, from, kb, pol);
            issued = it + 1;
          }
        }
        if (!ok) give_up();
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------ products (a pair's first CTA)
      // One thread waits and issues: what it does between two blocks' products is on their way (a division a
      // block took 4096 x 16384 x 4096 from 185 to 215 us, waits with a limit of their own from 173 to 184, and
      // those of the copies from 170 to 175).
      if (side == 0 && elect_one()) {
        const uint64_t blocks = smem_desc_sw128(smem_u32(ring), 16, 1024), words = smem_desc_plain(smem_u32(sf), 0, 128);
        constexpr uint32_t kNextByte = idesc_mx(256, 128, 1) - idesc_mx(256, 128, 0);
        const int tiles = (total - cluster + clusters - 1) / clusters;
        bool ok = true;
        int s = 0, slot = 0, sum = 0;            // of the block, of the scale word, of the first half's accumulator
        uint32_t phase = 0, word_phase = 0, n = 0, which = 0;
        for (int t = 0; t < tiles && ok; ++t) {
          for (int g = 0, in = 0, most = a.first_part; g < a.kbs; g += kGroup) {  // in: blocks of this part so far
            const bool two = g + 1 < a.kbs, ends = g + kGroup >= a.kbs || in + kGroup >= most;
            const int s1 = s + 1 == kPairStages ? 0 : s + 1;
            if ((g & 3) == 0) {
              ok = ok && thread_wait_cluster(&sf_full[slot], word_phase, abort_flag);
              which ^= 16;
            }
            ok = ok && thread_wait_cluster(&full[s], phase, abort_flag);
            // (the accumulator three before: the other half's, two or one parts before)
            if (in == 0 && n >= 2) ok = ok && thread_wait_cluster(&sum_free[2 + (n & 1)], (n - 2) >> 1 & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
            const uint32_t sft = tmem + kPairSfCol + which;
            if ((g & 3) == 0) {
#pragma unroll
              for (int p = 0; p < 3; ++p)
                tc_copy_scales_of<2>(sft + p * 4, words + (uint32_t)(slot * (kPairSfBytes / 16) + p * 32));
              tc_commit_pair(&sf_empty[slot], both);
              if (++slot == kPairSf) slot = 0, word_phase ^= 1;
            }
            const uint32_t idesc = idesc_mx(256, 128, 0) + (g & 3) * kNextByte;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (h && in == 0 && n >= 1) {
                if (!thread_wait_cluster(&sum_free[(n - 1) & 1], (n - 1) >> 1 & 1u, abort_flag)) { ok = false; break; }
                tc_fence_after();
              }
              const uint32_t acc = tmem + (uint32_t)((sum + h) % kPairSums * 128);
#pragma unroll
              for (int j = 0; j < kGroup; ++j) {
                if (j && !two) break;
                const int st = j ? s1 : s;
                if (j && !h) {
                  ok = thread_wait_cluster(&full[s1], phase ^ (s1 == 0), abort_flag);
                  if (!ok) break;
                  tc_fence_after();
                }
                const uint64_t x = blocks + (uint32_t)(st * (kPairStageBytes / 16)), wt = x + (uint32_t)(kBlockBytes + h * 64 * 128) / 16;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                  tc_mma_mx<2>(acc, x + kk * 2, wt + kk * 2, idesc + j * kNextByte, sft, sft + 4 + 4 * h, in + j + kk > 0);
                if (h) tc_commit_pair(&empty[st], both);
              }
              if (!ok) break;
              if (ends) tc_commit_pair(&sum_full[h * 2 + (n & 1)], both);
            }
            if (!ok) break;
            s += two ? 2 : 1;
            if (s >= kPairStages) s -= kPairStages, phase ^= 1;
            in += kGroup;
            if (ends) {
              in = 0, ++n;
              most = a.part;
              sum = sum == 0 ? 2 : sum - 1;      // (two further on, of three)
            }
          }
        }
        if (!ok) give_up();
        tc_commit_pair(drained, both);
      }
      __syncwarp();
    } else {
      // ------------------------------------------------------------ scale words
      // Two warps take turns at the words (of four K blocks each), and each loads its next before it
      // passes one on: the passing on, released at cluster scope, takes about as long as four K blocks'
      // products do (with one warp it set the pace: 16384 columns, 4096 x 4096, 199 us against 163).
      if (warp == 2) grid_launch_dependents();
      const int groups = (a.kbs + 3) / 4, turn = warp - 2;
      uint32_t x[4], ws[2];
      auto load = [&](int w, int g) {
        const int rt = w % row_tiles, ct = w / row_tiles, x_row = row_of(rt);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[j] = __ldg(reinterpret_cast<const uint32_t *>(a.xs + (int64_t)(x_row + lane + 32 * j) * a.sk) + g);
#pragma unroll
        for (int p = 0; p < 2; ++p) {  // the tile's scale rows: [tile][part]
          const int row = kGated ? ct * 2 + p : min(ct * 2 + p, a.tiles - 1);
          ws[p] = __ldg(reinterpret_cast<const uint32_t *>(a.ws + (int64_t)row * a.sk) + g);
        }
      };
      // the gi-th word of this cluster's tiles is word g of tile w
      int w = cluster, g = turn;
      auto settle = [&] {
        while (g >= groups) g -= groups, w += clusters;
      };
      settle();
      if (w < total) load(w, g);
      for (int gi = turn; w < total; gi += 2) {
        const int slot = gi % kPairSf;
        if (gi >= kPairSf && !warp_wait(&sf_empty[slot], (uint32_t)(gi / kPairSf - 1) & 1u, abort_flag, a.wait_ns)) {
          if (lane == 0) give_up();
          break;
        }
        uint4 *dst = reinterpret_cast<uint4 *>(sf + slot * kPairSfBytes) + lane;
        dst[0] = make_uint4(x[0], x[1], x[2], x[3]);
        dst[32] = make_uint4(ws[0], ws[0], ws[kGated], ws[kGated]);
        dst[64] = make_uint4(ws[!kGated], ws[!kGated], ws[1], ws[1]);
        g += 2;
        settle();
        if (w < total) load(w, g);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(cluster_map_shared(smem_u32(&sf_full[slot]), 0));
      }
    }
  } else {
    if constexpr (kMore) setmaxnreg_inc<kManyRegs>();
    // ------------------------------------------------------------ epilogue: two threads a row
    // Four warps take one half's sums, four the other's: a weight tile's, or 64 features of the gate and of the
    // up of a gated one.
    const int quarter = warp & 3, half = (warp - 4) >> 2, lane_row = quarter * 32 + lane;
    const uint32_t free_bar = cluster_map_shared(smem_u32(sum_free + half * 2), 0);
    // rows begin at multiples of 32 bytes
    const bool straight = (a.n * (kGated ? 1 : a.f32 ? 4 : 2) & 31) == 0 && ((uintptr_t)a.out & 31u) == 0;
    const int parts = 1 + (max(a.kbs - a.first_part, 0) + a.part - 1) / a.part;
    int n = 0, sum = half;                       // parts of K so far; the accumulator
    // The half's next accumulator, complete (false: the wait ran out, or another one), and its release.
    const auto take = [&](uint32_t &acc) {
      if (!warp_wait_cluster(&sum_full[half * 2 + (n & 1)], (uint32_t)(n >> 1) & 1u, abort_flag)) {
        if (lane == 0) give_up();
        return false;
      }
      tc_fence_after();
      acc = tmem + (uint32_t)(sum * 128) + ((uint32_t)(quarter * 32) << 16);
      sum = sum == 0 ? 2 : sum - 1;              // (two further on, of three)
      return true;
    };
    const auto release = [&] {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_relaxed(free_bar + (n & 1) * 8);
      ++n;
    };
    for (int w = cluster; w < total; w += clusters) {
      const int rt = w % row_tiles, ct = w / row_tiles;
      const int row0 = row_of(rt) + quarter * 32, row = row0 + lane, own0 = rt * 256 + side * 128;
      // 32 columns of a plain product
      const auto store = [&](int c, const float *f) {
        if (c >= a.n) return;
        if (straight) store_straight(a, row, own0, c, f);
        else store_turned(a, row0, own0, c, f, turn + (warp - 4) * 32 * kTurn);
      };
      if constexpr (!kMore) {                    // 64 columns at a time, no sums to hold
        uint32_t acc;
        if (!take(acc)) break;
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
          float f[64];
#pragma unroll
          for (int q = 0; q < 2; ++q) tmem_ld32(acc + i * 64 + q * 32, *reinterpret_cast<uint32_t(*)[32]>(f + q * 32));
          tmem_wait_ld();
          if (i == 1) release();
#pragma unroll
          for (int q = 0; q < 2; ++q) store(ct * 256 + half * 128 + i * 64 + q * 32, f + q * 32);
        }
      } else {
        float v[128];                              // the tile's sums, part after part of K
        if constexpr (!kGated)
#pragma unroll
          for (int j = 0; j < 128; ++j) v[j] = 0.f;
        bool ok = true;
#pragma unroll 1
        for (int c = 0; c < parts; ++c) {
          uint32_t acc;
          ok = take(acc);
          if (!ok) break;
          if (kGated && c == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) tmem_ld32(acc + q * 32, *reinterpret_cast<uint32_t(*)[32]>(v + q * 32));
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              float t[64];
              tmem_ld32(acc + q * 64, *reinterpret_cast<uint32_t(*)[32]>(t));
              tmem_ld32(acc + q * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(t + 32));
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 64; ++j) v[q * 64 + j] += t[j];
            }
          }
          release();
        }
        if (kGated) ok = named_barrier_and(1 + quarter, 64, ok);  // (they meet below: both go on or neither)
        if (!ok) break;
        if constexpr (!kGated) {
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            float u[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) u[j] = q < 2 ? (q == 0 ? v[j] : v[32 + j]) : (q == 2 ? v[64 + j] : v[96 + j]);
            store(ct * 256 + half * 128 + q * 32, u);
          }
        } else {
          float h[64], m = 0.f;
#pragma unroll
          for (int j = 0; j < 64; ++j) {
            h[j] = silu_mul(v[j], v[64 + j]);
            m = fmaxf(m, fabsf(h[j]));
          }
          row_max[half][lane_row] = m;             // a block's scale is that of both halves
          named_barrier(1 + quarter, 64);
          m = fmaxf(m, row_max[half ^ 1][lane_row]);
          named_barrier(1 + quarter, 64);          // (read before the next tile's is written)
          const int e = fp8_exponent(m);
          const float p = fp8_pow2(-e);
          const int c = ct * kTile + half * 64;
          if (row >= own0) {
            uint32_t code[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) code[q] = fp8_codes4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3], p);
            uint8_t *dst = static_cast<uint8_t *>(a.out) + (int64_t)row * a.n + c;
            if (straight && c + 64 <= a.n) {
              st_global_32(dst, *reinterpret_cast<uint32_t(*)[8]>(code));
              st_global_32(dst + 32, *reinterpret_cast<uint32_t(*)[8]>(code + 8));
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if (c + 16 * q < a.n)              // (n is a multiple of 16)
                  *reinterpret_cast<uint4 *>(dst + 16 * q) =
                      make_uint4(code[4 * q], code[4 * q + 1], code[4 * q + 2], code[4 * q + 3]);
            }
            if (half == 0) {
              uint8_t *s = a.out_scales + (int64_t)row * a.out_sk;
              s[ct] = (uint8_t)(e + 127);
              if (ct == a.tiles - 1)
                for (int b = a.tiles; b < a.out_sk; ++b) s[b] = 127;  // padding
            }
          }
        }
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
    // Both stages of a block count at the first CTA's barrier: the CTA that has requested fewer requests what
    // it lacks (nothing reads the stages any more), and the first waits for the last of them to land.
    if (tid == 0) {
      const int theirs = (int)ld_cluster_u32(cluster_map_shared(smem_u32(&issued_shared), side ^ 1));
      for (; issued < theirs; ++issued)
        request(issued % kPairStages, source_of(cluster + issued / a.kbs * clusters), issued % a.kbs, policy_evict_last());
    }
    cluster_sync_all();
    if (tid == 0 && side == 0)
      for (int t = max(0, issued - kPairStages); t < issued; ++t)
        thread_wait(&full[t % kPairStages], (uint32_t)(t / kPairStages) & 1u, abort_flag, false);
    __syncwarp();
    cluster_sync_all();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair<512>(tmem);
  }
}

// ------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, bool (&done)[64], int dev) {
  if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
  return e;
}

// Pairs that are resident at once (a pair lies within one group of SMs, which need not hold a whole number
// of them); a persistent grid is no larger.
template <typename K>
int resident_pairs(K kernel, int (&known)[64], int dev) {
  if (dev >= 0 && dev < 64 && known[dev] > 0) return known[dev];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(device_sms() / 2 * 2));
  cfg.blockDim = dim3(kPairThreads);
  cfg.dynamicSmemBytes = (size_t)kPairSmem;
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

template <int kParts>
cudaError_t launch_stream(const CUtensorMap &tx, ProductArgs a, int dev, cudaStream_t stream) {
  static bool done[64] = {};
  const int sms = device_sms();
  const int zt = (a.rows + a.nt - 1) / a.nt;
  // K is cut over a cluster until there are more CTAs than SMs, at least two blocks each.  (8 rows, us with 1, 2, 4, 8
  // CTAs a tile: K 4096 with 8 tiles 16.4, 10.2, 6.8, 5.6, 32 tiles 16.9, 10.5, 7.9, 7.6, 64 tiles 16.9, 11.8, 9.8, 14.1,
  // 128 tiles 18.2, 14.5, 19.1, 22.4, 192 tiles 20.3, 19.2, 23.6, 31.6; 32 tiles with K 1024 5.9, 4.9, 4.6, 5.6.)
  int splits = 1;
  while (splits < kMaxSplits && splits * 4 <= a.kbs && (int64_t)a.tiles * zt * splits <= sms) splits *= 2;
  a.stage_bytes = kParts * kBlockBytes + a.nt * 128;
  // Accumulators of kSumNext blocks, as far as the columns of three CTAs an SM go (over one wave, of two), of
  // kSumMost at most in any case: with more columns, then with more splits, if that is what it takes.  (Head of
  // 128256 features of 4096 for 64 rows: 87 us with one accumulator, 98 with two of 16 blocks and two CTAs an SM, 101
  // with two splits of 16; 8 rows of 16384 in 32768 features: 81 with seven of 19 or with one of 128 blocks, 99 with
  // eight splits.)
  int per, cols;
  for (;; splits *= 2) {
    per = (a.kbs + splits - 1) / splits;              // K blocks of a CTA
    const int want = (per + kSumNext - 1) / kSumNext, least = (per + kSumMost - 1) / kSumMost;
    const bool last = splits == kMaxSplits || splits * 4 > a.kbs, waves = (int64_t)a.tiles * zt * splits > 2 * sms;
    int room = stream_sums(kParts, a.nt, waves ? 128 : 256);
    if (room < least) room = stream_sums(kParts, a.nt, 256);
    if (room < least && last) room = stream_sums(kParts, a.nt, 512);
    a.sums = std::min(want, std::max(room, 1));
    if (a.sums >= least || last) break;
  }
  a.part = (per + a.sums - 1) / a.sums;
  for (cols = 32; cols < a.sums * kParts * a.nt + stream_sf_columns(kParts);) cols *= 2;
  // A grid of one wave runs fastest with the deepest rings that leave two CTAs an SM; over several waves
  // a third CTA covers the others' beginnings and ends (head of 128256 features, 64 rows: 96 us with
  // two an SM, 85 with three; 40960 features of 8 rows: 40 and 28; 28672 + 28672 features of 8 rows: 38.3 with either;
  // a second projection of 16384 in 4096 features: 14.1 with two, 14.8 with three).
  a.tmem_cols = cols;
  const bool three = (int64_t)a.tiles * zt * splits > 2 * sms && 3 * cols <= 512;
  const int budget = three ? kStreamSmem3 : kStreamSmem2;
  a.stages = std::min(std::min(per, kStreamStages), (budget - stream_fixed(kParts)) / a.stage_bytes);
  const int acc = kParts * a.nt * kTile * 4;          // the epilogue's, in the ring
  a.stages = std::max(std::max(a.stages, 2), (acc + a.stage_bytes - 1) / a.stage_bytes);
  const int smem = std::max(a.stages * a.stage_bytes + stream_fixed(kParts), splits > 1 ? smem_floor(cols) : 0);
  cudaError_t e = allow_smem(fp8_stream_kernel<kParts>, 226 * 1024, done, dev);
  if (e != cudaSuccess) return e;
  return launch_after<fp8_stream_kernel<kParts>>(dim3((unsigned)a.tiles, (unsigned)splits, (unsigned)zt),
                      dim3(kStreamThreads), (size_t)smem, dim3(1, (unsigned)splits, 1), stream, tx, a);
}

template <bool kGated, bool kMore>
cudaError_t launch_pair(const CUtensorMap &tx, const CUtensorMap &tw, const ProductArgs &a, int dev,
                        cudaStream_t stream) {
  static bool done[64] = {};
  static int resident[64] = {};
  const int row_tiles = (a.rows + 255) / 256, col_tiles = kGated ? a.tiles : (a.tiles + 1) / 2;
  constexpr auto kKernel = fp8_pair_kernel<kGated, kMore>;
  if (kMore && (dev < 0 || dev >= 64 || !done[dev])) {
    cudaFuncAttributes f;
    const cudaError_t e = cudaFuncGetAttributes(&f, kKernel);
    if (e != cudaSuccess) return e;
    if (f.numRegs < kLaunchRegs) return cudaErrorLaunchOutOfResources;
  }
  const cudaError_t e = allow_smem(kKernel, kPairSmem, done, dev);
  if (e != cudaSuccess) return e;
  const int64_t pairs = std::min<int64_t>(resident_pairs(kKernel, resident, dev), (int64_t)row_tiles * col_tiles);
  return launch_after<kKernel>(dim3((unsigned)(2 * pairs)), dim3(kPairThreads), (size_t)kPairSmem, dim3(2, 1, 1),
                               stream, tx, tw, a, row_tiles, col_tiles);
}

int run_product(ham_fp8_weight *w, const void *x_codes, const void *x_scales, int32_t rows, void *out,
                void *out_scales, int f32, void *stream) {
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev != w->device) cudaSetDevice(w->device);
  ProductArgs a{};
  a.w = w->codes;
  a.ws = w->scales;
  a.xs = static_cast<const uint8_t *>(x_scales);
  a.out = out;
  a.out_scales = static_cast<uint8_t *>(out_scales);
  a.err = w->err;
  a.rows = rows;
  a.n = w->n;
  a.kbs = w->kbs;
  a.sk = w->sk;
  a.out_sk = fp8_scale_bytes(w->n);
  a.tiles = w->tiles;
  a.f32 = f32;
  a.wait_ns = w->wait_ns;
  const int64_t tiles = (int64_t)((rows + 255) / 256) * (w->parts == 2 ? w->tiles : (w->tiles + 1) / 2);
  // The pair kernel where its tiles (of 256 x 256; a tile takes 43 us at K 16384, whoever else is idle) occupy an
  // eighth of the SMs, gated ones a sixteenth.  Stream / pair kernel, us: 16 tiles (512 x 2048) 8.6 / 6.4 at K 512,
  // 10.4 / 10.1 at 2048, 12.8 / 15.7 at 4096, 25.5 / 43 at 16384; 21 tiles (768 x 1792) 7.9 / 6.7, 11.1 / 10.4,
  // 15.6 / 15.7, 45 / 43; 64 tiles (300 x 8192) 8.0 / 7.2, 14.5 / 11.7, 23 / 17, 76 / 54.  Gated, whose stream kernel
  // fills an SM's tensor memory with 128 rows: 8 tiles (129 x 1024) 9.5 / 10.0 at K 1024, 12.3 / 16.6 at 4096; 12 tiles
  // (640 x 512) 19 / 10, 24 / 17, 39 / 45 at 16384; 16 tiles (256 x 2048) 29 / 10, 36 / 18, 59 / 46.
  const bool pair = rows > 128 && tiles * (w->parts == 2 ? 16 : 8) >= device_sms();
  a.first_part = kSumFirst;                           // the pair kernel's parts
  a.part = kSumNext;
  // the streaming kernel's row parts, of equal size: 128 rows at most, fewer where K is so long that a CTA needs
  // several accumulators even with every split (gated from 32768 on, plain from 98304)
  const int blocks = (w->kbs + kMaxSplits - 1) / kMaxSplits, needs = (blocks + kSumMost - 1) / kSumMost;
  int most = 128;
  while (most > 16 && stream_sums(w->parts, most, 512) < needs) most -= 16;
  const int row_parts = (rows + most - 1) / most;
  a.nt = ((rows + row_parts - 1) / row_parts + 15) / 16 * 16;
  a.box = std::min(a.nt, rows);
  CUtensorMap tx;
  int rc = HAM_OK;
  if (make_bytes_tensor_map(&tx, x_codes, rows, w->k, kFp8Block, pair ? 128 : a.box) != 0) {
    rc = op_fail(HAM_ECUDA, "tensor map of the rows");
  } else {
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = pair ? (w->parts == 2 ? launch_pair<true, true>(tx, w->map, a, w->device, s)
                                                : a.first_part < a.kbs ? launch_pair<false, true>(tx, w->map, a, w->device, s) : launch_pair<false, false>(tx, w->map, a, w->device, s))
                               : (w->parts == 2 ? launch_stream<2>(tx, a, w->device, s)
                                                : launch_stream<1>(tx, a, w->device, s));
    if (e != cudaSuccess) rc = op_fail(HAM_ECUDA, "product launch: %s", cudaGetErrorString(e));
  }
  if (dev != w->device) cudaSetDevice(dev);
  return rc;
}

int check_product(const ham_fp8_weight *w, const void *xc, const void *xs, int32_t rows, const void *out) {
  if (!w) return op_fail(HAM_EINVAL, "null handle");
  if (rows < 0 || rows > (1 << 24)) return op_fail(HAM_EINVAL, "rows %d outside 0..2^24", rows);
  if (rows == 0) return HAM_OK;
  if (!xc || !xs || !out) return op_fail(HAM_EINVAL, "codes, scales and the output are required");
  if (!op_aligned(xc, 16) || !op_aligned(out, 16) || !op_aligned(xs, 4))
    return op_fail(HAM_EINVAL, "codes and the output must be 16-byte aligned, scales 4-byte aligned");
  return HAM_OK;
}

}  // namespace
}  // namespace ham

using ham::op_aligned;
using ham::op_fail;
using ham::op_overlap;

extern "C" {

int ham_fp8_weight_free(ham_fp8_weight *w) {
  if (!w) return HAM_OK;
  int dev = 0;
  cudaGetDevice(&dev);
  cudaSetDevice(w->device);
  cudaFree(w->codes);
  cudaSetDevice(dev);
  delete w;
  return HAM_OK;
}

int ham_fp8_weight_alloc(int32_t n, int32_t k, const void *codes, const void *scales, const void *codes_up,
                         const void *scales_up, ham_fp8_weight **out) {
  if (!out) return op_fail(HAM_EINVAL, "out is required");
  *out = nullptr;
  if (n < 1 || n > (1 << 22)) return op_fail(HAM_EINVAL, "n %d outside 1..2^22", n);
  if (k < 16 || k % 16 != 0 || k > (1 << 20)) return op_fail(HAM_EINVAL, "k %d must be a multiple of 16 in 16..2^20", k);
  if (!codes || !scales) return op_fail(HAM_EINVAL, "codes and scales are required");
  if (!codes_up != !scales_up) return op_fail(HAM_EINVAL, "codes_up and scales_up come together");
  if (codes_up && n % 16 != 0) return op_fail(HAM_EINVAL, "n %d of a gated weight must be a multiple of 16", n);
  for (const void *p : {codes, codes_up})
    if (!op_aligned(p, 16)) return op_fail(HAM_EINVAL, "codes must be 16-byte aligned");
  ham_fp8_weight *w = new (std::nothrow) ham_fp8_weight();
  if (!w) return op_fail(HAM_ENOMEM, "host allocation failed");
  w->n = n;
  w->k = k;
  w->parts = codes_up ? 2 : 1;
  w->tiles = (n + ham::kTile - 1) / ham::kTile;
  w->kbs = (k + ham::kFp8Block - 1) / ham::kFp8Block;
  w->sk = ham::fp8_scale_bytes(k);
  cudaGetDevice(&w->device);
  const int64_t blocks = (int64_t)w->tiles * w->kbs;
  if (blocks * w->parts * 128 > INT32_MAX) {
    delete w;
    return op_fail(HAM_EUNSUPPORTED, "weight of %d x %d is too large", n, k);
  }
  const size_t code_bytes = (size_t)blocks * w->parts * ham::kBlockBytes, scale_bytes = (size_t)w->tiles * w->parts * w->sk;
  cudaError_t e = cudaMalloc(reinterpret_cast<void **>(&w->codes), code_bytes + scale_bytes + 4);
  if (e != cudaSuccess) {
    cudaGetLastError();
    ham_fp8_weight_free(w);
    return op_fail(HAM_ENOMEM, "weight of %d x %d: %s", n, k, cudaGetErrorString(e));
  }
  w->scales = w->codes + code_bytes;             // (whole words)
  w->err = reinterpret_cast<int32_t *>(w->scales + scale_bytes);
  const int64_t pieces = blocks * (ham::kBlockBytes / 16);
  for (int p = 0; p < w->parts && e == cudaSuccess; ++p) {
    ham::lay_out_weight_kernel<<<(unsigned)((pieces + 255) / 256), 256>>>(
        static_cast<const uint8_t *>(p ? codes_up : codes), n, k, p, w->parts, w->kbs, pieces, w->codes);
    e = cudaGetLastError();
    if (e != cudaSuccess) break;
    ham::lay_out_scales_kernel<<<(unsigned)((w->tiles * w->sk + 255) / 256), 256>>>(
        static_cast<const uint8_t *>(p ? scales_up : scales), w->tiles, w->sk, p, w->parts, w->scales);
    e = cudaGetLastError();
  }
  if (e == cudaSuccess) e = cudaMemset(w->err, 0, 4);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess || ham::make_stretch_tensor_map(&w->map, w->codes, blocks * w->parts * ham::kBlockBytes,
                                                       ham::kBlockBytes / 2) != 0) {
    cudaGetLastError();
    ham_fp8_weight_free(w);
    return op_fail(HAM_ECUDA, "weight layout: %s", cudaGetErrorString(e));
  }
  *out = w;
  return HAM_OK;
}

int ham_fp8_linear(ham_fp8_weight *w, const void *x_codes, const void *x_scales, int32_t rows, void *out,
                   int32_t out_dtype, void *stream) {
  ham::ApiRange nvtx_range("ham_fp8_linear");
  int rc = ham::check_product(w, x_codes, x_scales, rows, out);
  if (rc) return rc;
  if (w->parts != 1) return op_fail(HAM_EINVAL, "a gated weight serves ham_fp8_gated");
  if (out_dtype != HAM_DTYPE_BF16 && out_dtype != HAM_DTYPE_F32) return op_fail(HAM_EINVAL, "out_dtype %d", out_dtype);
  if (rows == 0) return HAM_OK;
  const int f32 = out_dtype == HAM_DTYPE_F32;
  const size_t ob = (size_t)rows * w->n * (f32 ? 4 : 2);
  if (op_overlap(out, ob, x_codes, (size_t)rows * w->k) || op_overlap(out, ob, x_scales, (size_t)rows * w->sk))
    return op_fail(HAM_EINVAL, "out must not overlap the input rows");
  return ham::run_product(w, x_codes, x_scales, rows, out, nullptr, f32, stream);
}

int ham_fp8_gated(ham_fp8_weight *w, const void *x_codes, const void *x_scales, int32_t rows, void *codes,
                  void *scales, void *stream) {
  ham::ApiRange nvtx_range("ham_fp8_gated");
  int rc = ham::check_product(w, x_codes, x_scales, rows, codes);
  if (rc) return rc;
  if (w->parts != 2) return op_fail(HAM_EINVAL, "ham_fp8_gated takes a gated weight (gate and up)");
  if (rows == 0) return HAM_OK;
  if (!scales || !op_aligned(scales, 4)) return op_fail(HAM_EINVAL, "the output's scales are required, 4-byte aligned");
  const size_t ob = (size_t)rows * w->n, sb = (size_t)rows * ham::fp8_scale_bytes(w->n);
  const size_t xb = (size_t)rows * w->k, xsb = (size_t)rows * w->sk;
  if (op_overlap(codes, ob, x_codes, xb) || op_overlap(codes, ob, x_scales, xsb) ||
      op_overlap(scales, sb, x_codes, xb) || op_overlap(scales, sb, x_scales, xsb) || op_overlap(codes, ob, scales, sb))
    return op_fail(HAM_EINVAL, "inputs and outputs must not overlap");
  return ham::run_product(w, x_codes, x_scales, rows, codes, scales, 0, stream);
}

int ham_fp8_weight_set_wait_limit_ns(ham_fp8_weight *w, uint64_t ns) {
  if (!w) return op_fail(HAM_EINVAL, "null handle");
  if (ns > ham::kWaitLimitNs)
    return op_fail(HAM_EINVAL, "limit %llu ns above the default %llu", (unsigned long long)ns,
                   (unsigned long long)ham::kWaitLimitNs);
  w->wait_ns = ns ? ns : ham::kWaitLimitNs;
  return HAM_OK;
}

int ham_fp8_weight_status(ham_fp8_weight *w, void *stream, int32_t *device_code) {
  if (!w) return op_fail(HAM_EINVAL, "null handle");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t code = 0;
  cudaError_t ce = cudaMemcpyAsync(&code, w->err, 4, cudaMemcpyDeviceToHost, s);
  if (ce == cudaSuccess) ce = cudaMemsetAsync(w->err, 0, 4, s);
  if (ce == cudaSuccess) ce = cudaStreamSynchronize(s);
  if (ce != cudaSuccess) return op_fail(HAM_ECUDA, "status read: %s", cudaGetErrorString(ce));
  if (device_code) *device_code = code;
  if (code != 0) return op_fail(HAM_EDEVICE, "device error word = %d", code);
  return HAM_OK;
}

}  // extern "C"

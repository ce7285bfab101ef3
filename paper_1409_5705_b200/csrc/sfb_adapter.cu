// Low-rank adapters of many requests beside the shared W (sfb_adapter_* in sfb.h): the logits of samples, each with the adapter
// (a set of factor pairs) that its request names, and the gradients of the samples and of the adapters' factors.
//
// Launches of a forward pass:  adapter_rank_kernel (s = V x), adapter_product_kernel (y = W x, with scale U^T s at the end);
// of a backward pass:  adapter_index_kernel, adapter_rank_kernel (t = U dy; s again where it is not given), adapter_product_kernel
// (dx), adapter_gradient_kernel (dU, dV).
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <new>

#include "sfb_tc.h"
#include "sfb_tile.cuh"

namespace sfb {
namespace {

using namespace ptx;

constexpr int BM = 128, BK = 64, kSlice = 16;       // rows of the accumulator, k-block, ranks of a slice
constexpr int kMaxTile = 256;                       // samples of a tile, at most
constexpr int kTileBytesA = BM * BK * 2;
constexpr int kMaxParts = 16;                       // of the contraction of adapter_rank_kernel
constexpr int kMaxStages = 8;
constexpr int kRing = 196608;                       // bytes of operand stages

__host__ __device__ constexpr int stage_bytes(int tn) { return kTileBytesA + tn * BK * 2; }
int stages_of(int tn) { return std::min(kMaxStages, kRing / stage_bytes(tn)); }

// Samples of a tile: the fewest columns that hold n, up to 256.
int tile_of(int64_t n) { return n <= 16 ? 16 : n <= 32 ? 32 : n <= 64 ? 64 : n <= 128 ? 128 : kMaxTile; }

// ---------------------------------------------------------------------------------------------------------
// Which adapters the samples of a tile take: list[0 .. count), in the order of their first samples, and each sample's place in it
// (-1: none).  By all threads of a block.
// ---------------------------------------------------------------------------------------------------------
struct TileList {
  int32_t id[kMaxTile];
  int32_t place[kMaxTile];
  int32_t list[kMaxTile];
  uint32_t firsts[kMaxTile / 32];
  int32_t count;
};

__device__ __forceinline__ void build_list(TileList& L, const int32_t* ids, int first, int n, int tn, int adapters, uint32_t* status) {
  for (int t = threadIdx.x; t < kMaxTile; t += blockDim.x) {
    int id = t < tn && first + t < n ? ids[first + t] : -1;
    if (id < -1 || id >= adapters) {
      atomicOr(status, SFB_STATUS_ADAPTER_RANGE);
      id = -1;
    }
    L.id[t] = id;
  }
  __syncthreads();
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  for (int w = threadIdx.x >> 5; w < kMaxTile / 32; w += warps) {
    const int t = w * 32 + lane, id = L.id[t];
    int f = t;
    if (w * 32 < tn) {
      for (int u = (t & ~3) - 4; u >= 0; u -= 4) {                     // downwards: the last hit is the first sample
        const int4 v = *reinterpret_cast<const int4*>(&L.id[u]);
        if (v.w == id) f = u + 3;
        if (v.z == id) f = u + 2;
        if (v.y == id) f = u + 1;
        if (v.x == id) f = u;
      }
      if (f == t)
        for (int u = t - 1; u >= (t & ~3); --u)
          if (L.id[u] == id) f = u;
    }
    const uint32_t m = __ballot_sync(0xffffffffu, id >= 0 && f == t);
    if (lane == 0) L.firsts[w] = m;
    L.place[t] = f;                                                    // for now: the sample that has the place
  }
  __syncthreads();
  for (int t = threadIdx.x; t < kMaxTile; t += blockDim.x) {
    const int f = L.place[t];
    int at = __popc(L.firsts[f >> 5] & ((1u << (f & 31)) - 1));
    for (int w = 0; w < (f >> 5); ++w) at += __popc(L.firsts[w]);
    if (L.id[t] >= 0 && f == t) L.list[at] = L.id[t];
    L.place[t] = L.id[t] >= 0 ? at : -1;
  }
  if (threadIdx.x == 0) {
    int c = 0;
    for (int w = 0; w < kMaxTile / 32; ++w) c += __popc(L.firsts[w]);
    L.count = c;
  }
  __syncthreads();
}

// ---------------------------------------------------------------------------------------------------------
// p_i = F[a_i] z_i:  the adapters' factors as the rows of the accumulator, 16 ranks (a slice) of one adapter after another, the
// samples of a tile as its columns; each sample takes the rows of its own adapter, so what another adapter or sample holds does not
// reach it.  Grid: parts of the contraction x tiles of samples x groups of the tile's slices, eight slices at a time.
// Warps: 0 TMA producer, 1 MMA issuer and TMEM owner, 2..5 epilogue.
// ---------------------------------------------------------------------------------------------------------
constexpr int kRankThreads = 192;
struct RankParams {
  int32_t n, tn, kseg, stages;
  int32_t rank, adapters;
  const int32_t* ids;
  float* out;                  // [parts][n][rank]
  uint32_t* status;
};

__global__ void __launch_bounds__(kRankThreads, 1)
adapter_rank_kernel(const __grid_constant__ CUtensorMap tmF, const __grid_constant__ CUtensorMap tmZ, const __grid_constant__ RankParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ alignas(16) TileList L;
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2];
  __shared__ uint32_t tmem_slot, abort_word;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int part = blockIdx.x, parts = gridDim.x, first = blockIdx.y * p.tn;
  const int kbeg = static_cast<int>(static_cast<int64_t>(part) * p.kseg / parts), kend = static_cast<int>(static_cast<int64_t>(part + 1) * p.kseg / parts);
  const int cols = max(p.tn, 32), stage = stage_bytes(p.tn);
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], 4); }
    abort_word = 0;
    fence_barrier_init();
    prefetch_tmap(&tmF); prefetch_tmap(&tmZ);
  }
  if (warp == 1) { tmem_alloc(&tmem_slot, 2 * cols); tmem_relinquish(); }
  pdl_wait();
  pdl_launch_dependents();
  build_list(L, p.ids, first, p.n, p.tn, p.adapters, p.status);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  const int per = (p.rank + kSlice - 1) / kSlice, slices = L.count * per, chunks = (slices + 7) / 8;

  if (warp == 0) {
    uint32_t s = 0, ph = 0;
    bool ok = true;
    for (int c = blockIdx.z; c < chunks && ok; c += gridDim.z) {
      const int ns = min(8, slices - c * 8);
      for (int k = kbeg; k < kend; ++k) {
        if (!mbar_wait_warp(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
        if (elect_one()) {
          mbar_expect_tx(&full[s], ns * (kSlice * BK * 2) + p.tn * BK * 2);
          uint8_t* st = smem + s * stage;
          tma_load_2d(st + kTileBytesA, &tmZ, k * BK, first, &full[s]);
          for (int j = 0; j < ns; ++j) {
            const int g = c * 8 + j, at = g / per;
            tma_load_3d(st + j * (kSlice * BK * 2), &tmF, k * BK, (g - at * per) * kSlice, L.list[at], &full[s]);
          }
        }
        if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1; }
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = umma_idesc_bf16(BM, p.tn);
    uint32_t s = 0, ph = 0, i = 0;
    bool ok = true;
    for (int c = blockIdx.z; c < chunks && ok; c += gridDim.z, ++i) {
      const uint32_t a = i & 1, aph = (i >> 1) & 1, d_tmem = tmem_base + a * cols;
      if (!mbar_wait_warp(&tempty[a], aph ^ 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      for (int k = kbeg; k < kend; ++k) {
        if (!mbar_wait_warp(&full[s], ph, abort_flag)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t da = umma_desc_k128(smem_u32(smem + s * stage)), db = umma_desc_k128(smem_u32(smem + s * stage + kTileBytesA));
#pragma unroll
          for (int j = 0; j < BK / 16; ++j) umma_bf16(d_tmem, da + 2 * j, db + 2 * j, idesc, (k - kbeg) | j ? 1u : 0u);
          umma_commit(&empty[s]);
        }
        if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1; }
      }
      if (ok && elect_one()) umma_commit(&tfull[a]);
    }
  } else {
    const int q = warp & 3;
    float* out = p.out + static_cast<int64_t>(part) * p.n * p.rank;
    uint32_t i = 0;
    for (int c = blockIdx.z; c < chunks; c += gridDim.z, ++i) {
      const uint32_t a = i & 1, aph = (i >> 1) & 1;
      if (!mbar_wait_warp(&tfull[a], aph, abort_flag)) break;
      tc_fence_after();
      const int g = c * 8 + q * 2 + (lane >> 4), at = g < slices ? g / per : -2, r = (g - at * per) * kSlice + (lane & 15);
#pragma unroll 1
      for (int t0 = 0; t0 < p.tn; t0 += 32) {
        uint32_t acc[32];
        tmem_ld_32x32(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + a * cols + t0, acc);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j)                 // (places behind a tile of 16 are -1)
          if (L.place[t0 + j] == at && r < p.rank) out[static_cast<int64_t>(first + t0 + j) * p.rank + r] = __uint_as_float(acc[j]);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tempty[a]);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (abort_word) {
    if (threadIdx.x == 0) atomicOr(p.status, SFB_STATUS_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, 2 * cols); }
}

// The products p_i as adapter_rank_kernel leaves them, or as the caller has them (one part).
struct Ranked {
  const float* at;
  int32_t parts;
  int64_t stride;              // entries from a part to the next
};
__device__ __forceinline__ float ranked(const Ranked& s, int64_t at) {
  float v = s.at[at];
  for (int c = 1; c < s.parts; ++c) v += s.at[c * s.stride + at];
  return v;
}

// ---------------------------------------------------------------------------------------------------------
// y_i = A z_i + scale F[a_i]^T p_i for a tile of 128 rows of A (rows of W; with MN, of its transpose: columns of W) and tn samples.  The
// contraction is cut over the CTAs of a cluster; each of them finishes some of the samples, adding the parts in rank order and the
// adapter's term in fp32.
// ---------------------------------------------------------------------------------------------------------
constexpr int kProdThreads = 192;
struct ProductParams {
  int32_t n, tn, tiles, m;     // samples; of a tile; tiles of samples; rows of A
  int32_t kseg, stages, parts; // k-blocks; operand stages; CTAs of a cluster
  int32_t rank, adapters;
  const int32_t* ids;
  const float* scale;
  const __nv_bfloat16* F;      // [adapters][rank][ldf]
  int64_t ldf;
  Ranked p;
  float* p_out;                // may be null: [n][rank]
  __nv_bfloat16* Y;
  int64_t ldy;
  uint32_t* status;
};

template <bool MN>
__global__ void __launch_bounds__(kProdThreads, 1)
adapter_product_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmZ, const __grid_constant__ ProductParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], done;
  __shared__ uint32_t tmem_slot, abort_word;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int mine = static_cast<int>(blockIdx.x) % p.parts, tile = static_cast<int>(blockIdx.x) / p.parts;
  const int mt = tile / p.tiles, m0 = mt * BM, first = (tile - mt * p.tiles) * p.tn;
  const int kbeg = mine * p.kseg / p.parts, nk = (mine + 1) * p.kseg / p.parts - kbeg;
  const int cols = max(p.tn, 32), stage = stage_bytes(p.tn);
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    mbar_init(&done, 1);
    abort_word = 0;
    fence_barrier_init();
    prefetch_tmap(&tmA); prefetch_tmap(&tmZ);
  }
  if (warp == 1) { tmem_alloc(&tmem_slot, cols); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();

  if (warp == 0) {
    bool ok = true;
    for (int k = 0; k < nk && ok; ++k) {
      const uint32_t s = k % p.stages, ph = (k / p.stages) & 1;
      ok = mbar_wait_warp(&empty[s], ph ^ 1, abort_flag);
      if (ok && elect_one()) {
        uint8_t* st = smem + s * stage;
        mbar_expect_tx(&full[s], stage);
        if (MN) {
          tma_load_2d(st, &tmA, m0, (kbeg + k) * BK, &full[s]);
          tma_load_2d(st + kTileBytesA / 2, &tmA, m0 + 64, (kbeg + k) * BK, &full[s]);
        } else {
          tma_load_2d(st, &tmA, (kbeg + k) * BK, m0, &full[s]);
        }
        tma_load_2d(st + kTileBytesA, &tmZ, (kbeg + k) * BK, first, &full[s]);
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = umma_idesc_bf16(BM, p.tn) | (MN ? 1u << 15 : 0u);
    bool ok = true;
    for (int k = 0; k < nk && ok; ++k) {
      const uint32_t s = k % p.stages, ph = (k / p.stages) & 1;
      ok = mbar_wait_warp(&full[s], ph, abort_flag);
      tc_fence_after();
      if (ok && elect_one()) {
        const uint32_t a = smem_u32(smem + s * stage);
        const uint64_t da = MN ? umma_desc_mn128(a) : umma_desc_k128(a), db = umma_desc_k128(a + kTileBytesA);
#pragma unroll
        for (int j = 0; j < BK / 16; ++j) umma_bf16(tmem_base, da + (MN ? 128 : 2) * j, db + 2 * j, idesc, k | j ? 1u : 0u);
        umma_commit(&empty[s]);
      }
    }
    if (ok && elect_one()) umma_commit(&done);
  } else {
    // the accumulator to shared memory (the operand stages', which nothing uses any more): [sample][128 rows]
    const int q = warp & 3;
    if (mbar_wait_warp(&done, 0, abort_flag)) {
      tc_fence_after();
      float* to = reinterpret_cast<float*>(smem) + q * 32 + lane;
#pragma unroll 1
      for (int t0 = 0; t0 < p.tn; t0 += 32) {
        uint32_t acc[32];
        tmem_ld_32x32(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + t0, acc);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (t0 + j < p.tn) to[(t0 + j) * BM] = __uint_as_float(acc[j]);
      }
    }
  }
  __syncwarp();
  if (p.parts > 1) { cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  if (!abort_word) {
    const uint32_t base = smem_u32(smem);
    const int t1 = (mine + 1) * p.tn / p.parts;
    for (int t = mine * p.tn / p.parts + warp; t < t1; t += kProdThreads / 32) {
      const int64_t i = first + t;
      if (i >= p.n) break;
      const int id = p.ids[i];
      const bool has = id >= 0 && id < p.adapters;
      const float sc = has ? p.scale[id] : 0.f;
      float s[SFB_ADAPTER_MAX_RANK / 32];
#pragma unroll
      for (int u = 0; u < SFB_ADAPTER_MAX_RANK / 32; ++u) {
        const int r = u * 32 + lane;
        s[u] = has && r < p.rank ? ranked(p.p, i * p.rank + r) : 0.f;
        if (p.p_out && mt == 0 && r < p.rank) p.p_out[i * p.rank + r] = s[u];
        s[u] *= sc;
      }
#pragma unroll 1
      for (int g = 0; g < BM / 32; ++g) {
        const int m = m0 + g * 32 + lane;
        float v = 0.f;
        const uint32_t at = base + (t * BM + g * 32 + lane) * 4;
        for (int c = 0; c < p.parts; ++c) {
          float w;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w) : "r"(mapa_u32(at, c)) : "memory");
          v = c ? v + w : w;
        }
        if (has) {
          const __nv_bfloat16* f = p.F + static_cast<int64_t>(id) * p.rank * p.ldf + m;
#pragma unroll
          for (int u = 0; u < SFB_ADAPTER_MAX_RANK / 32; ++u) {
            const int left = min(32, p.rank - u * 32);
            for (int r = 0; r < left; ++r) {
              const float w = m < p.m ? __bfloat162float(f[(u * 32 + r) * p.ldf]) : 0.f;
              v = fmaf(w, __shfl_sync(0xffffffffu, s[u], r), v);
            }
          }
        }
        if (m < p.m) p.Y[i * p.ldy + m] = __float2bfloat16_rn(v);
      }
    }
  }
  __syncwarp();
  if (p.parts > 1) { cluster_arrive(); cluster_wait(); }               // no CTA leaves while a peer still reads its part
  tc_fence_before();
  __syncthreads();
  if (abort_word) {
    if (threadIdx.x == 0) atomicOr(p.status, SFB_STATUS_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, cols); }
}

// ---------------------------------------------------------------------------------------------------------
// The samples of each adapter, one adapter after another, in their order: a warp per adapter goes over all ids, counts the samples
// of lower adapters and its own, then writes its own.  No sample without an adapter is among them.
// ---------------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) adapter_index_kernel(const int32_t* ids, int32_t n, int32_t adapters, int32_t* order, int32_t* begin, int32_t* count,
                                                            uint32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  const int a = static_cast<int>(blockIdx.x) * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (a >= adapters) return;
  int below = 0, own = 0;
  bool bad = false;
  for (int64_t b = 0; b < n; b += 128) {
    int id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) id[u] = b + u * 32 + lane < n ? ids[b + u * 32 + lane] : -1;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      bad |= id[u] < -1 || id[u] >= adapters;
      below += id[u] >= 0 && id[u] < a;
      own += id[u] == a;
    }
  }
  below = __reduce_add_sync(0xffffffffu, below);
  own = __reduce_add_sync(0xffffffffu, own);
  if (a == 0 && bad) atomicOr(status, SFB_STATUS_ADAPTER_RANGE);
  if (lane == 0) { begin[a] = below; count[a] = own; }
  int64_t at = below;
  if (own > 0) {
    for (int64_t b = 0; b < n; b += 128) {
      int id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) id[u] = b + u * 32 + lane < n ? ids[b + u * 32 + lane] : -1;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t m = __ballot_sync(0xffffffffu, id[u] == a);
        if (id[u] == a) order[at + __popc(m & ((1u << lane) - 1))] = static_cast<int32_t>(b + u * 32 + lane);
        at += __popc(m);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------------
// dF[a] = scale sum_{i of a} p_i z_i^T for a tile of 128 columns of z: the columns are the accumulator's rows, the ranks its
// columns, the samples the contraction, 64 of them at a time, gathered by the order that adapter_index_kernel wrote (so no sample of
// another adapter is in the product).  p as a (hi, lo) pair of bf16, 2^-17 of it lost; z is bf16 as it is.
// Warps: 0..3 loaders (z by asynchronous copies, p from fp32), 4 MMA issuer and TMEM owner, 5..8 epilogue.
// ---------------------------------------------------------------------------------------------------------
constexpr int kGradThreads = 288, kGradStages = 4, kGradLag = 2;
struct GradSide {
  const __nv_bfloat16* z;      // [n][ldz]
  int64_t ldz;
  int32_t width, tiles;        // columns; tiles of 128 of them (0: not wanted)
  Ranked p;
  float* out;                  // [adapters][rank][width]
};
struct GradParams {
  GradSide side[2];
  int32_t rank, adapters;
  const int32_t *order, *begin, *count;
  const float* scale;
  uint32_t* status;
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// v = hi + lo, as near as two bf16 come.  (What overflows in the rounding is cut off instead; an infinity has no rest.)
__device__ __forceinline__ void two_words(float v, float& hi, float& lo) {
  hi = __bfloat162float(__float2bfloat16_rn(v));
  if (isinf(hi)) hi = isinf(v) ? v : __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  lo = isinf(hi) ? 0.f : v - hi;
}

__global__ void __launch_bounds__(kGradThreads, 1) adapter_gradient_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kGradStages], empty[kGradStages], tfull[2], tempty[2];
  __shared__ uint32_t tmem_slot, abort_word;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int rp = (p.rank + 15) & ~15, panels = (rp + 63) / 64, word = panels * 8192, stage = kTileBytesA + 2 * word;
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    for (int i = 0; i < kGradStages; ++i) { mbar_init(&full[i], 128); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], 4); }
    abort_word = 0;
    fence_barrier_init();
  }
  if (warp == 4) { tmem_alloc(&tmem_slot, 256); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();
  const int64_t items0 = static_cast<int64_t>(p.side[0].tiles) * p.adapters, items = items0 + static_cast<int64_t>(p.side[1].tiles) * p.adapters;
  auto locate = [&](int64_t it, int& side, int& a, int& m0) {
    side = it >= items0;
    if (side) it -= items0;
    const int tiles = p.side[side].tiles;
    a = static_cast<int>(it / tiles);
    m0 = static_cast<int>(it - static_cast<int64_t>(a) * tiles) * BM;
  };

  if (warp < 4) {
    uint32_t g = 0;                                  // k-blocks so far
    bool ok = true;
    const int tid = threadIdx.x, c16 = tid & 15, r0 = tid >> 4, kb_row = tid >> 1, half = tid & 1;
    for (int64_t it = blockIdx.x; it < items && ok; it += gridDim.x) {
      int side, a, m0;
      locate(it, side, a, m0);
      const GradSide& sd = p.side[side];
      const int count = p.count[a], nk = (count + BK - 1) / BK;
      const int32_t* order = p.order + p.begin[a];
      const float sc = p.scale[a];
      const int col = m0 + c16 * 8, left = sd.width - col;
      const uint32_t bytes = left >= 8 ? 16 : left > 0 ? left * 2 : 0;
      for (int k = 0; k < nk; ++k, ++g) {
        const uint32_t s = g % kGradStages, ph = (g / kGradStages) & 1;
        if (!mbar_wait(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
        const uint32_t st = smem_u32(smem + s * stage);
        int64_t row[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) { const int at = k * BK + r0 + j * 8; row[j] = at < count ? order[at] : -1; }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int kr = r0 + j * 8;
          const uint32_t to = st + (c16 >> 3) * (kTileBytesA / 2) + kr * 128 + (((c16 & 7) ^ (kr & 7)) << 4);
          const uint32_t b = row[j] >= 0 ? bytes : 0;
          cp_async_16(to, b ? sd.z + row[j] * sd.ldz + col : sd.z, b);
        }
        cp_async_commit();
        // p of sample kb_row: every other piece of eight ranks
        const int at = k * BK + kb_row;
        const int64_t i = at < count ? order[at] : -1;
        for (int ch = half; ch < rp / 8; ch += 2) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float h[2], l[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int r = ch * 8 + j * 2 + e;
              two_words(i >= 0 && r < p.rank ? sc * ranked(sd.p, i * p.rank + r) : 0.f, h[e], l[e]);
            }
            hi[j] = pack2(h[0], h[1]);
            lo[j] = pack2(l[0], l[1]);
          }
          const uint32_t to = st + kTileBytesA + (ch >> 3) * 8192 + kb_row * 128 + (((ch & 7) ^ (kb_row & 7)) << 4);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + word), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
        }
        if (g >= kGradLag) {
          cp_async_wait<kGradLag>();
          fence_proxy_async_smem();
          mbar_arrive(&full[(g - kGradLag) % kGradStages]);
        }
      }
    }
    cp_async_wait<0>();
    fence_proxy_async_smem();
    if (ok)
      for (uint32_t j = g > kGradLag ? g - kGradLag : 0; j < g; ++j) mbar_arrive(&full[j % kGradStages]);
  } else if (warp == 4) {
    const uint32_t idesc = umma_idesc_bf16(BM, rp) | kIdescMnMajor;
    uint32_t g = 0, i = 0;
    bool ok = true;
    for (int64_t it = blockIdx.x; it < items && ok; it += gridDim.x) {
      int side, a, m0;
      locate(it, side, a, m0);
      const int nk = (p.count[a] + BK - 1) / BK;
      if (nk == 0) continue;
      const uint32_t b = i & 1, bph = (i >> 1) & 1, d_tmem = tmem_base + b * 128;
      ++i;
      if (!mbar_wait_warp(&tempty[b], bph ^ 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      for (int k = 0; k < nk; ++k, ++g) {
        const uint32_t s = g % kGradStages, ph = (g / kGradStages) & 1;
        if (!mbar_wait_warp(&full[s], ph, abort_flag)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint32_t st = smem_u32(smem + s * stage);
          const uint64_t da = umma_desc_mn128(st), dh = umma_desc_mn128(st + kTileBytesA), dl = umma_desc_mn128(st + kTileBytesA + word);
#pragma unroll
          for (int j = 0; j < BK / 16; ++j) {
            umma_bf16(d_tmem, da + 128 * j, dh + 128 * j, idesc, k | j ? 1u : 0u);
            umma_bf16(d_tmem, da + 128 * j, dl + 128 * j, idesc, 1u);
          }
          umma_commit(&empty[s]);
        }
      }
      if (ok && elect_one()) umma_commit(&tfull[b]);
    }
  } else {
    const int q = warp & 3;
    uint32_t i = 0;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
      int side, a, m0;
      locate(it, side, a, m0);
      const GradSide& sd = p.side[side];
      const bool any = p.count[a] > 0;
      const uint32_t b = i & 1, bph = (i >> 1) & 1;
      const int m = m0 + q * 32 + lane;
      float* out = sd.out + static_cast<int64_t>(a) * p.rank * sd.width + m;
      if (any) {
        ++i;
        if (!mbar_wait_warp(&tfull[b], bph, abort_flag)) break;
        tc_fence_after();
      }
#pragma unroll 1
      for (int r0 = 0; r0 < p.rank; r0 += 32) {
        uint32_t acc[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[j] = 0u;
        if (any) {
          tmem_ld_32x32(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + b * 128 + r0, acc);
          tmem_ld_wait();
        }
        if (m < sd.width) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (r0 + j < p.rank) out[static_cast<int64_t>(r0 + j) * sd.width] = __uint_as_float(acc[j]);
        }
      }
      if (any) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&tempty[b]);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (abort_word) {
    if (threadIdx.x == 0) atomicOr(p.status, SFB_STATUS_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 4) { tc_fence_after(); tmem_dealloc(tmem_base, 256); }
}

// ---------------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------------
// Parts of the contraction of adapter_rank_kernel: as many as give every SM a block, of four k-blocks at least.
int rank_parts(int64_t n, int64_t d) {
  const int64_t tiles = (n + tile_of(n) - 1) / tile_of(n), kseg = (d + BK - 1) / BK;
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({kMaxParts, kModelSms / tiles, kseg / 4})));
}
// Most samples x parts of a call of up to n samples.
int64_t rank_rows(int64_t n, int64_t d) {
  int64_t most = 0;
  for (int64_t tiles = 1; tiles <= kModelSms; ++tiles) {
    const int64_t m = std::min(n, tiles * kMaxTile);
    most = std::max(most, m * rank_parts(m, d));
    if (m == n) return most;
  }
  return std::max(most, n);
}

struct AdapterLayout {
  size_t status, s, t, order, begin, count, total;
};

int check(const sfb_adapter_config* c) {
  if (!c || c->rows <= 0 || c->cols <= 0 || c->adapters <= 0 || c->rank <= 0 || c->max_samples < 0 || c->ldw < 0 || c->ldu < 0 || c->ldv < 0)
    return SFB_ERR_ARG;
  const int64_t ldw = c->ldw ? c->ldw : c->cols, ldu = c->ldu ? c->ldu : c->rows, ldv = c->ldv ? c->ldv : c->cols;
  if (ldw < c->cols || ldu < c->rows || ldv < c->cols || ldw % 8 || ldu % 8 || ldv % 8) return SFB_ERR_SHAPE;
  if (c->rank > SFB_ADAPTER_MAX_RANK || c->adapters > 65536 || c->rows > (1 << 26) || c->cols > (1 << 26) || c->max_samples > (1 << 22))
    return SFB_ERR_SHAPE;
  if (((std::max(c->rows, c->cols) + BM - 1) / BM) * (c->max_samples / kMaxTile + 1) > (1ll << 28)) return SFB_ERR_SHAPE;
  if (std::max({ldw, ldu, ldv}) > (1ll << 30) || ldu * c->rank > (1ll << 35) || ldv * c->rank > (1ll << 35)) return SFB_ERR_SHAPE;
  return SFB_OK;
}

AdapterLayout layout_of(const sfb_adapter_config& c) {
  AdapterLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off += (bytes + kAlign - 1) / kAlign * kAlign; return at; };
  L.status = take(4);
  L.s = take(static_cast<size_t>(rank_rows(c.max_samples, c.cols)) * c.rank * 4);
  L.t = take(static_cast<size_t>(rank_rows(c.max_samples, c.rows)) * c.rank * 4);
  L.order = take(static_cast<size_t>(c.max_samples) * 4);
  L.begin = take(static_cast<size_t>(c.adapters) * 4);
  L.count = take(static_cast<size_t>(c.adapters) * 4);
  L.total = off;
  return L;
}

bool al(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace
}  // namespace sfb

struct sfb_adapters {
  sfb_adapter_config cfg;              // pitches filled in
  sfb::AdapterLayout lay;
  const void *W, *U, *V;
  const float* scale;
  char* ws;
  cudaStream_t stream;
  int device, last_cuda;
  CUtensorMap mapU, mapV;              // boxes of 64 entries x 16 ranks of an adapter
  sfb::TcState* tc;

  template <typename T>
  T* at(size_t off) const { return reinterpret_cast<T*>(ws + off); }
};

namespace sfb {
namespace {

struct OnDevice {                      // the handle's device is current for the length of a call
  int before = -1, mine;
  cudaError_t err;
  explicit OnDevice(int device) : mine(device) {
    err = cudaGetDevice(&before);
    if (err == cudaSuccess && before != mine) err = cudaSetDevice(mine);
  }
  ~OnDevice() {
    if (before >= 0 && before != mine) cudaSetDevice(before);
  }
};

bool factor_map(sfb_adapters* h, CUtensorMap* m, const void* base, int64_t width, int64_t pitch) {
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(h->cfg.rank), static_cast<cuuint64_t>(h->cfg.adapters)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(pitch) * 2, static_cast<cuuint64_t>(pitch) * 2 * h->cfg.rank};
  cuuint32_t box[3] = {BK, kSlice, 1}, estr[3] = {1, 1, 1};
  return h->tc->encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// p = F[a] z for n samples into `out`; *got: where and in how many parts.
cudaError_t rank_products(sfb_adapters* h, int64_t n, const void* Z, int64_t ldz, int64_t d, const CUtensorMap& mapF, const int32_t* ids, float* out,
                          Ranked* got) {
  const int tn = tile_of(n), parts = rank_parts(n, d), tiles = static_cast<int>((n + tn - 1) / tn);
  CUtensorMap mz;
  if (!make_map(h->tc, &mz, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, const_cast<void*>(Z), d, n, ldz * 2, BK, tn)) return cudaErrorInvalidValue;
  RankParams p{};
  p.n = static_cast<int32_t>(n); p.tn = tn; p.kseg = static_cast<int32_t>((d + BK - 1) / BK); p.stages = stages_of(tn);
  p.rank = h->cfg.rank; p.adapters = h->cfg.adapters; p.ids = ids; p.out = out; p.status = h->at<uint32_t>(h->lay.status);
  const int per = (h->cfg.rank + kSlice - 1) / kSlice, chunks = (std::min(tn, h->cfg.adapters) * per + 7) / 8;
  const int groups = std::max(1, std::min(chunks, kModelSms / (parts * tiles)));
  const int smem = p.stages * stage_bytes(tn) + 1024;
  cudaError_t e = allow_smem<adapter_rank_kernel>(kRing + 1024);
  if (e != cudaSuccess) return e;
  *got = Ranked{out, parts, n * h->cfg.rank};
  return launch_kernel(adapter_rank_kernel, dim3(parts, tiles, groups), dim3(kRankThreads), smem, h->stream, 1, mapF, mz, p);
}

// CTAs of a cluster: as many as leave every SM one and each four k-blocks.
int product_parts(int64_t tiles, int64_t kseg) {
  int best = 1;
  for (int s = 2; s <= 8; s *= 2)
    if (tiles * s <= kModelSms && kseg >= 4 * s) best = s;
  return best;
}

template <bool MN>
cudaError_t product(sfb_adapters* h, int64_t n, const void* Z, int64_t ldz, const int32_t* ids, const Ranked& s, float* p_out, void* Y, int64_t ldy) {
  const sfb_adapter_config& c = h->cfg;
  const int64_t m = MN ? c.cols : c.rows, d = MN ? c.rows : c.cols;
  const int tn = tile_of(n);
  CUtensorMap ma, mz;
  if (!make_map(h->tc, &ma, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, const_cast<void*>(h->W), c.cols, c.rows, c.ldw * 2, BK, MN ? BK : BM) ||
      !make_map(h->tc, &mz, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, const_cast<void*>(Z), d, n, ldz * 2, BK, tn))
    return cudaErrorInvalidValue;
  ProductParams p{};
  p.n = static_cast<int32_t>(n); p.tn = tn; p.tiles = static_cast<int32_t>((n + tn - 1) / tn); p.m = static_cast<int32_t>(m);
  p.kseg = static_cast<int32_t>((d + BK - 1) / BK); p.stages = stages_of(tn);
  const int64_t tiles = (m + BM - 1) / BM * p.tiles;
  p.parts = product_parts(tiles, p.kseg);
  p.rank = c.rank; p.adapters = c.adapters; p.ids = ids; p.scale = h->scale;
  p.F = static_cast<const __nv_bfloat16*>(MN ? h->V : h->U); p.ldf = MN ? c.ldv : c.ldu;
  p.p = s; p.p_out = p_out; p.Y = static_cast<__nv_bfloat16*>(Y); p.ldy = ldy; p.status = h->at<uint32_t>(h->lay.status);
  const int smem = p.stages * stage_bytes(tn) + 1024;
  cudaError_t e = allow_smem<adapter_product_kernel<MN>>(kRing + 1024);
  if (e != cudaSuccess) return e;
  return launch_kernel(adapter_product_kernel<MN>, dim3(static_cast<unsigned>(tiles * p.parts)), dim3(kProdThreads), smem, h->stream, p.parts, ma, mz, p);
}

int fail(sfb_adapters* h, cudaError_t e) {
  h->last_cuda = static_cast<int>(e);
  return SFB_ERR_CUDA;
}

}  // namespace
}  // namespace sfb

using namespace sfb;

#define ACK(x)                                  \
  do {                                          \
    const cudaError_t e_ = (x);                 \
    if (e_ != cudaSuccess) return fail(h, e_);  \
  } while (0)

extern "C" int sfb_adapter_workspace_bytes(const sfb_adapter_config* cfg, size_t* out_bytes) {
  if (!out_bytes) return SFB_ERR_ARG;
  const int rc = check(cfg);
  if (rc) return rc;
  *out_bytes = layout_of(*cfg).total;
  return SFB_OK;
}

extern "C" int sfb_adapter_init(const sfb_adapter_config* cfg, const void* W_dev, const void* U_dev, const void* V_dev, const float* scale_dev,
                                void* workspace_dev, size_t workspace_bytes, sfb_adapters** out) {
  if (!out) return SFB_ERR_ARG;
  *out = nullptr;
  const int rc = check(cfg);
  if (rc) return rc;
  if (!W_dev || !U_dev || !V_dev || !scale_dev || !workspace_dev) return SFB_ERR_ARG;
  if (!al(W_dev, 16) || !al(U_dev, 16) || !al(V_dev, 16) || !al(scale_dev, 4) || !al(workspace_dev, kAlign)) return SFB_ERR_ALIGN;
  const AdapterLayout lay = layout_of(*cfg);
  if (workspace_bytes < lay.total) return SFB_ERR_WORKSPACE;
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SFB_ERR_CUDA;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return SFB_ERR_CUDA;
  if (major != 10) return SFB_ERR_ARCH;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess) return SFB_ERR_CUDA;
  if (qres != cudaDriverEntryPointSuccess || !fn) return SFB_ERR_CUDA;
  sfb_adapters* h = new (std::nothrow) sfb_adapters();
  TcState* st = new (std::nothrow) TcState();
  if (!h || !st) { delete h; delete st; return SFB_ERR_ARG; }
  h->tc = st;
  st->encode = reinterpret_cast<EncodeTiledFn>(fn);
  h->cfg = *cfg;
  sfb_adapter_config& c = h->cfg;
  if (!c.ldw) c.ldw = c.cols;
  if (!c.ldu) c.ldu = c.rows;
  if (!c.ldv) c.ldv = c.cols;
  h->lay = lay;
  h->W = W_dev; h->U = U_dev; h->V = V_dev; h->scale = scale_dev;
  h->ws = static_cast<char*>(workspace_dev);
  h->stream = static_cast<cudaStream_t>(cfg->stream);
  h->device = dev;
  h->last_cuda = 0;
  if (!factor_map(h, &h->mapU, U_dev, c.rows, c.ldu) || !factor_map(h, &h->mapV, V_dev, c.cols, c.ldv) ||
      cudaMemsetAsync(h->ws + lay.status, 0, 4, h->stream) != cudaSuccess) {
    sfb_adapter_destroy(h);
    return SFB_ERR_CUDA;
  }
  *out = h;
  return SFB_OK;
}

extern "C" int sfb_adapter_forward(sfb_adapters* h, int64_t n, const void* X_dev, int64_t ldx, const int32_t* ids_dev, void* Y_dev, int64_t ldy,
                                   float* S_dev) {
  if (!h || n < 0) return SFB_ERR_ARG;
  const sfb_adapter_config& c = h->cfg;
  if (n > c.max_samples) return SFB_ERR_SHAPE;
  if (n == 0) return SFB_OK;
  if (!X_dev || !ids_dev || !Y_dev) return SFB_ERR_ARG;
  if (ldx < c.cols || ldy < c.rows || ldx % 8 || ldy % 8 || std::max(ldx, ldy) > (1ll << 30)) return SFB_ERR_SHAPE;
  if (!al(X_dev, 16) || !al(Y_dev, 16) || !al(ids_dev, 4) || !al(S_dev, 4)) return SFB_ERR_ALIGN;
  const OnDevice on(h->device);
  ACK(on.err);
  Ranked s{};
  ACK(rank_products(h, n, X_dev, ldx, c.cols, h->mapV, ids_dev, h->at<float>(h->lay.s), &s));
  ACK(product<false>(h, n, X_dev, ldx, ids_dev, s, S_dev, Y_dev, ldy));
  return SFB_OK;
}

extern "C" int sfb_adapter_backward(sfb_adapters* h, int64_t n, const void* dY_dev, int64_t lddy, const void* X_dev, int64_t ldx,
                                    const int32_t* ids_dev, const float* S_dev, void* dX_dev, int64_t lddx, float* dU_dev, float* dV_dev) {
  if (!h || n < 0) return SFB_ERR_ARG;
  const sfb_adapter_config& c = h->cfg;
  if (n > c.max_samples) return SFB_ERR_SHAPE;
  if (!al(dU_dev, 4) || !al(dV_dev, 4)) return SFB_ERR_ALIGN;
  const OnDevice on(h->device);
  ACK(on.err);
  if (n == 0) {
    const size_t pairs = static_cast<size_t>(c.adapters) * c.rank * 4;
    if (dU_dev) ACK(cudaMemsetAsync(dU_dev, 0, pairs * c.rows, h->stream));
    if (dV_dev) ACK(cudaMemsetAsync(dV_dev, 0, pairs * c.cols, h->stream));
    return SFB_OK;
  }
  if (!dY_dev || !X_dev || !ids_dev) return SFB_ERR_ARG;
  if (lddy < c.rows || ldx < c.cols || lddy % 8 || ldx % 8 || std::max(lddy, ldx) > (1ll << 30)) return SFB_ERR_SHAPE;
  if (dX_dev && (lddx < c.cols || lddx % 8 || lddx > (1ll << 30))) return SFB_ERR_SHAPE;
  if (!al(dY_dev, 16) || !al(X_dev, 16) || !al(dX_dev, 16) || !al(ids_dev, 4) || !al(S_dev, 4)) return SFB_ERR_ALIGN;
  uint32_t* status = h->at<uint32_t>(h->lay.status);
  int32_t *order = h->at<int32_t>(h->lay.order), *begin = h->at<int32_t>(h->lay.begin), *count = h->at<int32_t>(h->lay.count);
  if (dU_dev || dV_dev)
    ACK(launch_kernel(adapter_index_kernel, dim3((c.adapters + 7) / 8), dim3(256), 0, h->stream, 1, ids_dev, static_cast<int32_t>(n), c.adapters, order,
                      begin, count, status));
  Ranked s{S_dev, 1, 0}, t{};
  if (dU_dev && !S_dev) ACK(rank_products(h, n, X_dev, ldx, c.cols, h->mapV, ids_dev, h->at<float>(h->lay.s), &s));
  if (dX_dev || dV_dev) ACK(rank_products(h, n, dY_dev, lddy, c.rows, h->mapU, ids_dev, h->at<float>(h->lay.t), &t));
  if (dX_dev) ACK(product<true>(h, n, dY_dev, lddy, ids_dev, t, nullptr, dX_dev, lddx));
  if (dU_dev || dV_dev) {
    GradParams p{};
    if (dU_dev)
      p.side[0] = GradSide{static_cast<const __nv_bfloat16*>(dY_dev), lddy, static_cast<int32_t>(c.rows), static_cast<int32_t>((c.rows + BM - 1) / BM), s, dU_dev};
    if (dV_dev)
      p.side[1] = GradSide{static_cast<const __nv_bfloat16*>(X_dev), ldx, static_cast<int32_t>(c.cols), static_cast<int32_t>((c.cols + BM - 1) / BM), t, dV_dev};
    p.rank = c.rank; p.adapters = c.adapters; p.order = order; p.begin = begin; p.count = count; p.scale = h->scale; p.status = status;
    const int64_t items = (static_cast<int64_t>(p.side[0].tiles) + p.side[1].tiles) * c.adapters;
    const int panels = ((c.rank + 15) / 16 * 16 + 63) / 64, smem = kGradStages * (kTileBytesA + 2 * panels * 8192) + 1024;
    ACK(allow_smem<adapter_gradient_kernel>(kGradStages * (kTileBytesA + 4 * 8192) + 1024));
    ACK(launch_kernel(adapter_gradient_kernel, dim3(static_cast<unsigned>(std::min<int64_t>(items, sm_count()))), dim3(kGradThreads), smem, h->stream, 1, p));
  }
  return SFB_OK;
}

extern "C" int sfb_adapter_get_status(sfb_adapters* h, uint32_t* status_out) {
  if (!h || !status_out) return SFB_ERR_ARG;
  const OnDevice on(h->device);
  ACK(on.err);
  ACK(cudaMemcpyAsync(status_out, h->ws + h->lay.status, 4, cudaMemcpyDeviceToHost, h->stream));
  ACK(cudaMemsetAsync(h->ws + h->lay.status, 0, 4, h->stream));
  ACK(cudaStreamSynchronize(h->stream));
  return SFB_OK;
}

extern "C" int sfb_adapter_last_cuda_error(sfb_adapters* h) { return h ? h->last_cuda : 0; }

extern "C" int sfb_adapter_destroy(sfb_adapters* h) {
  if (!h) return SFB_ERR_ARG;
  delete h->tc;
  delete h;
  return SFB_OK;
}

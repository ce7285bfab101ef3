// Low-rank adapters of many requests beside the shared W (sfb_adapter_* in sfb.h): the logits of samples, each with the adapter
// (a set of factor pairs) that its request names, and the gradients of the samples and of the adapters' factors.
//
// Launches of a forward pass of up to 64 samples:  adapter_dot_kernel or, for many entries, adapter_rank_kernel (s = V x), adapter_few_kernel
// (y = W x + scale U^T s).  Of more:  adapter_index_kernel and adapter_copy_kernel (where the samples had better be taken in the order of their
// adapters, or copied because of the way their rows lie), adapter_dot_kernel or adapter_rank_kernel and adapter_sum_kernel (s, and what follows
// it), adapter_pair_kernel (y).
// Of a backward pass:  adapter_index_kernel (the samples of each adapter), the products as in a forward pass (t = U dy, dx), adapter_words_kernel
// where none of them has done its work, adapter_gradient_kernel (dU, dV), adapter_join_kernel where few adapters' samples are cut into shares.
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
constexpr int kMaxParts = 32;                       // of the contraction of adapter_rank_kernel
constexpr int kMaxStages = 8;
// The tensor cores cut off what an fp32 accumulator cannot hold, always towards zero: 1.4e-8 of the sum an instruction of 16 (measured:
// -1.1e-6 after 78 of them, -8e-6 after 512).  Sums that leave in fp32 are taken out, and added up with rounding, every 12 k-blocks.
constexpr int kDrain = 12;
constexpr int kListPitch = kMaxTile + 8;            // entries of a tile's list: their number, then the adapters
constexpr int kSmallRing = 98304;                   // bytes of operand stages where two blocks share an SM,
constexpr int kFewRing = 73728;                     // of adapter_rank_kernel beside one of adapter_few_kernel

__host__ __device__ constexpr int stage_bytes(int tn) { return kTileBytesA + tn * BK * 2; }

// Samples of a tile: the fewest columns that hold n, up to 256.
int tile_of(int64_t n) { return n <= 16 ? 16 : n <= 32 ? 32 : n <= 64 ? 64 : n <= 128 ? 128 : kMaxTile; }

// ---------------------------------------------------------------------------------------------------------
// Which adapters the samples of a tile take: list[0 .. count), in the order of their first samples, and each sample's place in it
// (-1: none).  By all threads of a block.
// ---------------------------------------------------------------------------------------------------------
template <int MOST>
struct TileList {
  int32_t id[MOST];
  int32_t place[MOST];
  int32_t list[MOST];
  uint32_t firsts[MOST / 32];
  int32_t count;
};

template <int MOST>
__device__ __forceinline__ void build_list(TileList<MOST>& L, const int32_t* ids, int first, int n, int tn, int adapters, uint32_t* status) {
  for (int t = threadIdx.x; t < MOST; t += blockDim.x) {
    int id = t < tn && first + t < n ? ids[first + t] : -1;
    if (id < -1 || id >= adapters) {
      atomicOr(status, SFB_STATUS_ADAPTER_RANGE);
      id = -1;
    }
    L.id[t] = id;
  }
  __syncthreads();
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  for (int w = threadIdx.x >> 5; w < MOST / 32; w += warps) {
    const int t = w * 32 + lane, id = L.id[t];
    int f = t;
    if (w * 32 < tn) {
      const uint32_t same = __match_any_sync(0xffffffffu, id);
      f = w * 32 + __ffs(same) - 1;
      if (__any_sync(0xffffffffu, w > 0 && id >= 0))
#pragma unroll 4
        for (int u = w * 32 - 4; u >= 0; u -= 4) {                     // downwards: the last hit is the first sample
          const int4 v = *reinterpret_cast<const int4*>(&L.id[u]);
          f = v.x == id ? u : v.y == id ? u + 1 : v.z == id ? u + 2 : v.w == id ? u + 3 : f;
        }
    }
    const uint32_t m = __ballot_sync(0xffffffffu, id >= 0 && f == t);
    if (lane == 0) L.firsts[w] = m;
    L.place[t] = f;                                                    // for now: the sample that has the place
  }
  __syncthreads();
  for (int t = threadIdx.x; t < MOST; t += blockDim.x) {
    const int f = L.place[t];
    int at = __popc(L.firsts[f >> 5] & ((1u << (f & 31)) - 1));
    for (int w = 0; w < (f >> 5); ++w) at += __popc(L.firsts[w]);
    if (L.id[t] >= 0 && f == t) L.list[at] = L.id[t];
    L.place[t] = L.id[t] >= 0 ? at : -1;
  }
  if (threadIdx.x == 0) {
    int c = 0;
    for (int w = 0; w < MOST / 32; ++w) c += __popc(L.firsts[w]);
    L.count = c;
  }
  __syncthreads();
}

// The products p_i as adapter_rank_kernel leaves them, or as the caller has them (one part).
struct Ranked {
  const float* at;
  int32_t parts;
  int64_t stride;              // entries from a part to the next
};
__device__ __forceinline__ float ranked(const Ranked& s, int64_t at) {
  float v = 0.f;
  for (int c = 0; c < s.parts; c += 8) {             // eight on their way
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = c + u < s.parts ? __ldcg(s.at + (c + u) * s.stride + at) : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) v += x[u];
  }
  return v;
}

// Where adapter_index_kernel has found that it pays, more than 64 samples are taken in the order of their adapters: position i is sample
// order[i] then.  (sorted null: never.)
struct Sorting {
  const uint32_t* sorted;
  const int32_t *order, *ids;  // of the positions
  __device__ __forceinline__ bool on() const { return sorted && *sorted; }
};

constexpr int kUnit = 8;                             // ranks of a unit of the adapters' term (see Term)

// v = w0 + w1, 2^-16 of v apart: two words of bf16.  (What overflows in the rounding to the first word is cut off instead; of what is not
// finite there is no rest.)
__device__ __forceinline__ void two_words(float v, float (&w)[2]) {
  w[0] = __bfloat162float(__float2bfloat16_rn(v));
  if (isinf(w[0]) && !isinf(v)) w[0] = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  w[1] = isfinite(v) ? v - w[0] : 0.f;
}
// Rank r of row i of pb (see Term).
__device__ __forceinline__ void put_pair(__nv_bfloat16* pb, int64_t i, int per, int r, float v) {
  float w[2];
  two_words(v, w);
  __nv_bfloat16* to = pb + (i * per + r / kUnit) * (2 * kUnit) + r % kUnit;
  to[0] = __float2bfloat16_rn(w[0]);
  to[kUnit] = __float2bfloat16_rn(w[1]);
}

// ---------------------------------------------------------------------------------------------------------
// p_i = F[a_i] z_i:  the adapters' factors as the rows of the accumulator, 16 ranks (a slice) of one adapter after another, up to 128
// samples as its columns; each sample takes the rows of its own adapter, so what another adapter or sample holds does not reach it.
// Eight slices (a chunk) at a time; the contraction in parts.  Bound by the way of z and F to the SMs, and by latency at either end of a
// block.  Grid: parts x tiles of samples x groups of chunks, two blocks an SM.
// FEW, up to 64 samples: one tile, a block an SM, chunks and parts shared out once the chunks are known; the block that finishes the last
// part of a chunk adds them (in their order) and writes p and pb, the first one the list, so that the product is the next launch.
// Warps: 0 TMA producer, 1 MMA issuer and TMEM owner, 2..9 epilogue (TMEM lane quarter q; 32 of every 64 samples), whose sums stay in
// registers from drain to drain.
// ---------------------------------------------------------------------------------------------------------
constexpr int kRankThreads = 320, kRankTile = 128, kFewChunks = 64;
// FEW: parts of the contraction that the grid's blocks make for each chunk.
__host__ __device__ inline int few_rank_parts(int blocks, int chunks, int kseg) {
  const int most = blocks / chunks < kMaxParts ? blocks / chunks : kMaxParts, parts = most < kseg / 4 ? most : kseg / 4;
  return parts < 1 ? 1 : parts;
}
struct RankParams {
  int32_t n, tn, kseg, stages;
  int32_t rank, adapters;
  int32_t boxed;               // slices that one copy of factors brings
  const int32_t* ids;
  float* out;                  // [parts][n][rank], by positions
  uint32_t* status;
  Sorting sort;                // not FEW
  // FEW
  const float* scale;
  float* p;                    // [n][rank]
  __nv_bfloat16* pb;           // see Term
  int32_t *lists, *place;
  uint32_t* arrived;           // [kFewChunks]
};

template <bool FEW>
__global__ void __launch_bounds__(kRankThreads, 2)
adapter_rank_kernel(const __grid_constant__ CUtensorMap tmF, const __grid_constant__ CUtensorMap tmZ, const __grid_constant__ CUtensorMap tmSorted,
                    const __grid_constant__ RankParams p) {
  constexpr int kHeld = FEW ? 1 : 2;                 // times 32 samples of an epilogue warp
  extern __shared__ uint8_t smem_raw[];
  __shared__ alignas(16) TileList<kRankTile> L;
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2];
  __shared__ uint32_t tmem_slot, abort_word, last;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int first = FEW ? 0 : blockIdx.y * p.tn;
  const int cols = max(p.tn, 32), stage = stage_bytes(p.tn);
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], 8); }
    abort_word = 0;
    fence_barrier_init();
    prefetch_tmap(&tmF); prefetch_tmap(&tmZ);
  }
  pdl_wait();
  if (warp == 1) { tmem_alloc(&tmem_slot, 2 * cols); tmem_relinquish(); }
  pdl_launch_dependents();
  const bool sorted = !FEW && p.sort.on();
  build_list(L, sorted ? p.sort.ids : p.ids, first, p.n, p.tn, p.adapters, p.status);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  const int per = (p.rank + kSlice - 1) / kSlice, slices = L.count * per, chunks = (slices + 7) / 8;
  // this block's chunks [c0, c0 + step, ..) and its part of their contraction
  int c0 = blockIdx.z, step = gridDim.z, part = blockIdx.x, parts = gridDim.x;
  if (FEW) {
    // (the grid has a block for each chunk at least: up to 64 samples have 64 chunks at most)
    parts = chunks ? few_rank_parts(gridDim.x, chunks, p.kseg) : 1;
    step = max(chunks, 1);
    c0 = blockIdx.x % step;
    part = blockIdx.x / step;
    if (part >= parts) c0 = chunks;                  // nothing
  }
  const int kbeg = static_cast<int>(static_cast<int64_t>(part) * p.kseg / parts), kend = static_cast<int>(static_cast<int64_t>(part + 1) * p.kseg / parts);
  if (FEW) {
    if (blockIdx.x == 0) {
      if (threadIdx.x == 0) p.lists[0] = L.count;
      const int per_pb = (p.rank + kUnit - 1) / kUnit, per8 = per_pb * kUnit;
      for (int t = threadIdx.x; t < p.tn; t += kRankThreads) {
        if (t < L.count) p.lists[1 + t] = L.list[t];
        if (t < p.n) p.place[t] = L.place[t];
      }
      for (int x = threadIdx.x; x < p.n * per8; x += kRankThreads) {       // samples without an adapter, and what lies behind the ranks
        const int t = x / per8, r = x - t * per8;
        if (r >= p.rank || L.place[t] < 0) put_pair(p.pb, t, per_pb, r, 0.f);
        if (r < p.rank && L.place[t] < 0) p.p[t * p.rank + r] = 0.f;
      }
    }
  }

  if (warp == 0) {
    uint32_t s = 0, ph = 0;
    bool ok = true;
    for (int c = c0; c < chunks && ok; c += step) {
      const int ns = min(8, slices - c * 8);
      for (int k = kbeg; k < kend; ++k) {
        if (!mbar_wait_warp(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
        if (elect_one()) {
          mbar_expect_tx(&full[s], ns * (kSlice * BK * 2) + p.tn * BK * 2);
          uint8_t* st = smem + s * stage;
          tma_load_2d(st + kTileBytesA, sorted ? &tmSorted : &tmZ, k * BK, first, &full[s]);
          for (int j = 0; j < ns; j += p.boxed) {
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
    for (int c = c0; c < chunks && ok; c += step) {
      for (int k0 = kbeg; k0 < kend && ok; k0 += kDrain, ++i) {
        const uint32_t a = i & 1, aph = (i >> 1) & 1, d_tmem = tmem_base + a * cols;
        if (!mbar_wait_warp(&tempty[a], aph ^ 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        for (int k = k0; k < min(k0 + kDrain, kend); ++k) {
          if (!mbar_wait_warp(&full[s], ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          if (elect_one()) {
            const uint64_t da = umma_desc_k128(smem_u32(smem + s * stage)), db = umma_desc_k128(smem_u32(smem + s * stage + kTileBytesA));
#pragma unroll
            for (int j = 0; j < BK / 16; ++j) umma_bf16(d_tmem, da + 2 * j, db + 2 * j, idesc, (k - k0) | j ? 1u : 0u);
            umma_commit(&empty[s]);
          }
          if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1; }
        }
        if (ok && elect_one()) umma_commit(&tfull[a]);
      }
    }
  } else {
    const int q = warp & 3, h = (warp - 2) >> 2;
    float* out = p.out + static_cast<int64_t>(part) * p.n * p.rank;
    uint32_t i = 0;
    bool ok = true;
    for (int c = c0; c < chunks && ok; c += step) {
      const int g = c * 8 + q * 2 + (lane >> 4), at = g < slices ? g / per : -2, r = (g - at * per) * kSlice + (lane & 15);
      uint32_t own[kHeld];                           // of 32 samples: those of this lane's adapter (places behind a tile of 16 are -1)
      bool any[kHeld];
      float sum[kHeld][32];
#pragma unroll
      for (int x = 0; x < kHeld; ++x) {
        const int t0 = h * 32 + x * 64;
        own[x] = 0;
        if (t0 < p.tn && r < p.rank) {
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const int4 v = *reinterpret_cast<const int4*>(&L.place[t0 + j]);
            own[x] |= ((v.x == at ? 1u : 0u) | (v.y == at ? 2u : 0u) | (v.z == at ? 4u : 0u) | (v.w == at ? 8u : 0u)) << j;
          }
        }
        any[x] = __any_sync(0xffffffffu, own[x]) != 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) sum[x][j] = 0.f;
      }
      for (int k0 = kbeg; k0 < kend; k0 += kDrain, ++i) {
        const uint32_t a = i & 1, aph = (i >> 1) & 1;
        if (!mbar_wait_warp(&tfull[a], aph, abort_flag)) { ok = false; break; }
        tc_fence_after();
#pragma unroll
        for (int x = 0; x < kHeld; ++x) {
          if (!any[x]) continue;
#pragma unroll
          for (int j0 = 0; j0 < 32; j0 += 16) {
            uint32_t acc[16];
            tmem_ld_32x16(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + a * cols + h * 32 + x * 64 + j0, acc);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[x][j0 + j] += __uint_as_float(acc[j]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&tempty[a]);
      }
      if (!ok) break;
#pragma unroll
      for (int x = 0; x < kHeld; ++x) {
        float* to = out + static_cast<int64_t>(first + h * 32 + x * 64) * p.rank + r;
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (own[x] >> j & 1) to[static_cast<int64_t>(j) * p.rank] = sum[x][j];
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (FEW && !abort_word) {
    for (int c = c0; c < chunks; c += step) {
      if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(&p.arrived[c], 1u) == static_cast<uint32_t>(parts) - 1;
        if (last) p.arrived[c] = 0;                  // for the next launch
        __threadfence();
      }
      __syncthreads();
      if (last) {
        const int per_pb = (p.rank + kUnit - 1) / kUnit;
        for (int x = threadIdx.x; x < p.n * p.rank; x += kRankThreads) {
          const int t = x / p.rank, r = x - t * p.rank, at = L.place[t];
          if (at < 0 || (at * per + r / kSlice) / 8 != c) continue;
          const float v = ranked(Ranked{p.out, parts, static_cast<int64_t>(p.n) * p.rank}, x);
          p.p[x] = v;
          put_pair(p.pb, t, per_pb, r, p.scale[L.list[at]] * v);
        }
      }
      __syncthreads();
    }
  }
  if (abort_word) {
    if (threadIdx.x == 0) atomicOr(p.status, SFB_STATUS_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, 2 * cols); }
}

constexpr int kEpi = 8;                             // epilogue warps of the products
// acc: row m (this lane's) of the positions i .. i + 31; sample: of position i + lane.  Even lanes store two rows of every other sample, odd
// lanes of the ones between; by a warp, whose rows begin at m - lane.  sorted: the samples do not follow one another.  (First all exchanges, then all stores, without a branch where the chunk
// is whole: with one behind each exchange a tile's end took 6.5 us.)
__device__ __forceinline__ void store_chunk(__nv_bfloat16* Y, int64_t ldy, int i, int n, bool sorted, int sample, int m, int most, const uint32_t (&acc)[32],
                                            int lane) {
  const int second = lane & 1;
  uint32_t two[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float x = __uint_as_float(acc[2 * j]), y = __uint_as_float(acc[2 * j + 1]);
    const float got = __shfl_xor_sync(0xffffffffu, second ? x : y, 1);
    const __nv_bfloat162 v = __floats2bfloat162_rn(second ? got : x, second ? y : got);
    two[j] = *reinterpret_cast<const uint32_t*>(&v);
  }
  const int r = m & ~1;
  __nv_bfloat16* to = Y + r;
  if (i + 32 <= n && m - lane + 32 <= most && !sorted) {
    to += static_cast<int64_t>(i + second) * ldy;
#pragma unroll
    for (int j = 0; j < 16; ++j) *reinterpret_cast<uint32_t*>(to + 2 * j * ldy) = two[j];
  } else if (i + 32 <= n && m - lane + 32 <= most) {
#pragma unroll
    for (int j = 0; j < 16; ++j) *reinterpret_cast<uint32_t*>(to + __shfl_sync(0xffffffffu, sample, 2 * j + second) * ldy) = two[j];
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int64_t at = __shfl_sync(0xffffffffu, sample, 2 * j + second) * ldy;
      if (i + second + 2 * j >= n || r >= most) continue;
      if (r + 1 < most) *reinterpret_cast<uint32_t*>(to + at) = two[j];
      else *reinterpret_cast<uint16_t*>(to + at) = static_cast<uint16_t>(two[j] & 0xffffu);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------
// The adapters' term, scale F[a_i]^T p_i, of the three products below is more contraction behind the k-blocks of A: the factors of the
// adapters in the tile's list, in units of 8 ranks, against  scale p  of the samples as two words of bf16 (2^-16 of the term; with one word
// its rounding was as large as that of the result), with zeros where a sample has another adapter.  (us with one word and with two: 37 samples of
// 64 adapters of 16 ranks, 10,000 x 20,000, 75.0 and 75.4; 64 of 32 of 128, 3,000 x 3,000, 28.4 and 32.3; 8,192 of 8 of 64, 10,000 x 5,000, 785
// and 808; 300 of 32 of 128, 5,000 x 2,000, 83 and 90; gradients of 1,024 of 64 of 8, 1,000 x 20,000, 116.5 and 120.5.)  Zeros do not hide what is not finite: some warps look
// through the factors in shared memory and replace what is not finite by zeros, and the end of the tile adds those entries alone to their
// own samples, in fp32.
// (In fp32 FMAs from global memory, as it was for up to 64 samples, a tile's term is a chain of loads: 64 samples of 8 ranks took 99 us a
// tile of 325,000 x 10,000, whose rows of W stream by in 57.)
// ---------------------------------------------------------------------------------------------------------
struct Term {
  int32_t rank, adapters;
  int32_t boxed;               // units that one copy of factors brings: a power of two that divides those of an adapter
  const int32_t *ids, *lists, *place;
  const float* scale;
  const __nv_bfloat16* F;      // [adapters][rank][ldf]
  int64_t ldf;
  const float* p;              // [n][rank]
  const uint4* pb;             // [n][units of an adapter][2]: scale p, first and second words of its eight ranks, zeros behind
};
__device__ __forceinline__ int units_of(const Term& t) { return (t.rank + kUnit - 1) / kUnit; }
// What the tensor cores have left out of the term of sample i at row m: the factors that are not finite.
__device__ __noinline__ float odd_term(const Term& p, int i, int m) {
  const int id = p.ids[i];
  if (id < 0 || id >= p.adapters) return 0.f;
  const __nv_bfloat16* f = p.F + static_cast<int64_t>(id) * p.rank * p.ldf + m;
  const float* s = p.p + static_cast<int64_t>(i) * p.rank;
  const float sc = p.scale[id];
  float v = 0.f;
  for (int r = 0; r < p.rank; ++r) {
    const float x = __bfloat162float(f[r * p.ldf]);
    if (!isfinite(x)) v = fmaf(x, sc * s[r], v);
  }
  return v;
}
// The factors of units [g0, g0 + nu) into a stage, by `warps` warps, w of them, each some of the copies (one warp, the producer's, took 90 ns a
// copy, 1.4 us a k-block of 16).  held: of the 32 units that unit g0 is among, the adapter and the first rank of each, by the lanes.
struct Held { int a, y; };
__device__ __forceinline__ Held hold_units(const int32_t* list, int g, int units, int per) {
  Held h{0, 0};
  if (g < units) {
    const int at = g / per;
    h.a = list[1 + at];
    h.y = (g - at * per) * kUnit;
  }
  return h;
}
template <int WARPS, int UNITS>
__device__ __forceinline__ void load_units(uint8_t* st, uint64_t* landed, const CUtensorMap& tmF, const Held& held, int g0, int nu, int boxed, int m0, int w) {
  constexpr int kMost = UNITS / WARPS;              // copies of a warp, for each of the two panels
  int a[kMost], y[kMost];
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int j = (w + i * WARPS) * boxed;
    a[i] = __shfl_sync(0xffffffffu, held.a, (g0 + j) & 31);
    y[i] = __shfl_sync(0xffffffffu, held.y, (g0 + j) & 31);
  }
  if (!elect_one()) return;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int j = (w + i * WARPS) * boxed;
    if (j >= nu) break;
    tma_load_3d(st + j * (kUnit * 128), &tmF, m0, y[i], a[i], landed);
    tma_load_3d(st + kTileBytesA / 2 + j * (kUnit * 128), &tmF, m0 + 64, y[i], a[i], landed);
  }
}
__device__ __forceinline__ uint4 lds_v4(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
// Replaces what is not finite of the factors of `nu` units in a stage by zeros; whether there was anything.  By THREADS threads, t of them.
template <int THREADS, int UNITS>
__device__ __forceinline__ uint32_t clean_units(uint8_t* st, int t, int nu) {
  // bit 15 / 31: the exponent of the low / high half is all ones
  auto found = [](uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
  constexpr int kBatch = 4, kPieces = 2 * UNITS * 64 / THREADS;       // of a thread, in both panels
  uint32_t bad = 0;
#pragma unroll 1
  for (int b = 0; b < kPieces; b += kBatch) {        // (loads first: with a branch behind each of them a block took 1.3 us)
    uint32_t hit = 0;
    uint4 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = (b + u) * THREADS + t, panel = i / (UNITS * 64), in = i % (UNITS * 64);
      v[u] = lds_v4(smem_u32(st) + panel * (kTileBytesA / 2) + in * 16);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int in = ((b + u) * THREADS + t) % (UNITS * 64);
      const uint32_t f = found(v[u].x) | found(v[u].y) | found(v[u].z) | found(v[u].w);
      hit |= in < nu * 64 ? f : 0u;
    }
    if (hit) {
      bad = 1;
#pragma unroll 1
      for (int u = 0; u < kBatch; ++u) {
        const int i = (b + u) * THREADS + t, panel = i / (UNITS * 64), in = i % (UNITS * 64);
        if (in >= nu * 64) continue;
        const uint32_t at = smem_u32(st) + panel * (kTileBytesA / 2) + in * 16;
        uint4 w = lds_v4(at);
        w.x &= ~((found(w.x) >> 15) * 0xffffu); w.y &= ~((found(w.y) >> 15) * 0xffffu);
        w.z &= ~((found(w.z) >> 15) * 0xffffu); w.w &= ~((found(w.w) >> 15) * 0xffffu);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
      }
    }
  }
  return bad;
}
// Up to 64 samples: both words are one operand, four units a k-block.  (A ring of second words, as for more samples, leaves room for one place
// of 64 samples: 37 samples of 64 adapters of 16 ranks, 10,000 x 20,000, 75.4 us and 76.0 with it; 64 of 64 of 64, 10,000 x 5,000, 52.5 and 54.4.)
constexpr int kFewUnits = BK / (2 * kUnit);
// Row t of the samples' operand of a k-block of `nu` units, first words and then second ones (row: this thread has one), and, beside an odd last unit, zeros in the factors'
// operand.  By THREADS threads, t of them.
template <int THREADS>
__device__ __forceinline__ void write_units(const uint4 (&words)[2 * kFewUnits], uint8_t* st, int t, bool row, int nu) {
  if (row) {
    const uint32_t to = smem_u32(st) + kTileBytesA + t * 128;
#pragma unroll
    for (int j = 0; j < 2 * kFewUnits; ++j)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + ((j ^ (t & 7)) << 4)), "r"(words[j].x), "r"(words[j].y),
                   "r"(words[j].z), "r"(words[j].w) : "memory");
  }
  if (nu & 1)
    for (int x = t; x < 128; x += THREADS)
      *reinterpret_cast<uint4*>(st + (x >> 6) * (kTileBytesA / 2) + nu * (kUnit * 128) + (x & 63) * 16) = make_uint4(0, 0, 0, 0);
}
// The words of the units [g0, g0 + nu) of a sample whose first unit is `at` (below zero: no adapter): zeros for those that are not its own.
__device__ __forceinline__ void read_units(const uint4* src, int at, int g0, int nu, int per, uint4 (&words)[2 * kFewUnits]) {
#pragma unroll
  for (int j = 0; j < kFewUnits; ++j) {
    const int u = g0 + j - at;
    const bool own = at >= 0 && j < nu && u >= 0 && u < per;
    words[j] = own ? src[2 * u] : make_uint4(0, 0, 0, 0);
    words[kFewUnits + j] = own ? src[2 * u + 1] : make_uint4(0, 0, 0, 0);
  }
}

// ---------------------------------------------------------------------------------------------------------
// y_i = A z_i + scale F[a_i]^T p_i for up to 64 samples: the rows of A (rows of W; with MN, of its transpose: columns of W) are the rows
// of the accumulator, 128 of them a tile.  Bound by the way of W to the SMs: two CTAs an SM, up to 192 KB of loads under way on it.  A tile
// a cluster, whose CTAs share the contraction and the k-blocks of the term; the parts are added in rank order, each CTA finishing some of
// the samples.  The loads of A and z do not wait for the launch before (adapter_rank_kernel lets this one start once those before it are
// done).  325,000 x 10,000 with 64 samples: 955 to 1,130 us by the GPU, 6.9 to 5.8 TB/s.  (A CTA an SM that takes its even share of all tiles, with parts through
// global memory: 1,030; 10,000 x 20,000 with 37 samples of 64 adapters 84, here 77.)
// Warps: 0 TMA producer, 1 MMA issuer and TMEM owner, 2..5 epilogue, 6 and 7 the samples' operand of the term and the
// loads of its factors, 8 and 9 the look at them.
// ---------------------------------------------------------------------------------------------------------
constexpr int kWrite = 2, kClean = 2, kBuild = kWrite + kClean;      // warps that write the samples' operand of the term, that look
                                                                     // through the factors
constexpr int kFewThreads = 32 * (6 + kBuild), kFewMost = 64, kMaxCluster = 8;
struct FewParams {
  Term term;
  int32_t n, m;                // samples; rows of A
  int32_t kseg, stages, parts; // k-blocks; operand stages; CTAs of a cluster
  __nv_bfloat16* Y;
  int64_t ldy;
  uint32_t* status;
};

// One k-block of A and z into a stage; by the producer's warp.
template <int TN, bool MN>
__device__ __forceinline__ void few_load(uint8_t* st, uint64_t* full, const CUtensorMap& tmA, const CUtensorMap& tmZ, int k, int m0, uint64_t keep) {
  if (!elect_one()) return;
  mbar_expect_tx(full, stage_bytes(TN));
  if (MN) {
    tma_load_2d(st, &tmA, m0, k * BK, full);
    tma_load_2d(st + kTileBytesA / 2, &tmA, m0 + 64, k * BK, full);
  } else {
    tma_load_2d(st, &tmA, k * BK, m0, full);
  }
  tma_load_2d_hint(st + kTileBytesA, &tmZ, k * BK, 0, full, keep);     // (every tile reads the samples)
}
template <bool MN>
__device__ __forceinline__ void few_mma(uint32_t st, uint32_t d_tmem, uint32_t idesc, bool first) {
  const uint64_t da = MN ? umma_desc_mn128(st) : umma_desc_k128(st), db = umma_desc_k128(st + kTileBytesA);
#pragma unroll
  for (int j = 0; j < BK / 16; ++j) umma_bf16(d_tmem, da + (MN ? 128 : 2) * j, db + 2 * j, idesc, !first || j ? 1u : 0u);
}
__device__ __forceinline__ void few_mma_units(uint32_t st, uint32_t d_tmem, uint32_t idesc, int nu) {
  const uint64_t da = umma_desc_mn128(st), db = umma_desc_k128(st + kTileBytesA);
  for (int j = 0; j < (nu + 1) / 2; ++j) {           // two units each: their first words, their second ones
    umma_bf16(d_tmem, da + 128 * j, db + 2 * j, idesc, 1u);
    umma_bf16(d_tmem, da + 128 * j, db + kFewUnits + 2 * j, idesc, 1u);
  }
}

template <int TN, bool MN>
__global__ void __launch_bounds__(kFewThreads, 2)
adapter_few_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmZ, const __grid_constant__ CUtensorMap tmF,
                   const __grid_constant__ FewParams p) {
  constexpr int kStage = stage_bytes(TN), kCols = TN < 32 ? 32 : TN;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], free_[kMaxStages], landed[kMaxStages], built[kMaxStages], done;
  __shared__ uint32_t tmem_slot, abort_word, odd;    // odd: some factor here was not finite
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int mine = static_cast<int>(blockIdx.x) % p.parts, m0 = static_cast<int>(blockIdx.x) / p.parts * BM;
  const int kbeg = mine * p.kseg / p.parts, nk = (mine + 1) * p.kseg / p.parts - kbeg;
  const int per = units_of(p.term);
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); mbar_init(&free_[i], 1); mbar_init(&landed[i], 1); mbar_init(&built[i], kBuild); }
    mbar_init(&done, 1);
    abort_word = odd = 0;
    fence_barrier_init();
    prefetch_tmap(&tmA); prefetch_tmap(&tmZ); prefetch_tmap(&tmF);
  }
  if (warp == 1) { tmem_alloc(&tmem_slot, kCols); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();                           // (not before this block has its columns of TMEM: the next launch takes some before it waits)
  const uint32_t tmem_base = tmem_slot;

  if (warp == 0) {
    const uint64_t keep = policy_evict_last();
    uint32_t s = 0, ph = 0;
    bool ok = true;
    auto next = [&]() { if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1; } };
    for (int k = 0; k < nk && ok; ++k, next()) {
      ok = mbar_wait_warp(&empty[s], ph ^ 1, abort_flag);
      if (ok) few_load<TN, MN>(smem + s * kStage, &full[s], tmA, tmZ, kbeg + k, m0, keep);
    }
    pdl_wait();
    const int units = p.term.lists[0] * per;
    for (int g0 = mine * kFewUnits; g0 < units && ok; g0 += p.parts * kFewUnits, next()) {
      ok = mbar_wait_warp(&empty[s], ph ^ 1, abort_flag);
      if (ok && elect_one()) {
        mbar_expect_tx(&landed[s], min(kFewUnits, units - g0) * 2 * kUnit * 128);
        mbar_arrive(&free_[s]);
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc_f = umma_idesc_bf16(BM, TN) | 1u << 15, idesc = MN ? idesc_f : umma_idesc_bf16(BM, TN);
    uint32_t s = 0, fph = 0, bph = 0;                // the phases of full and of built, a bit per stage
    bool ok = true;
    auto next = [&]() { if (++s == static_cast<uint32_t>(p.stages)) s = 0; };
    for (int k = 0; k < nk && ok; ++k, next()) {
      ok = mbar_wait_warp(&full[s], (fph >> s) & 1, abort_flag);
      fph ^= 1u << s;
      tc_fence_after();
      if (ok && elect_one()) {
        few_mma<MN>(smem_u32(smem + s * kStage), tmem_base, idesc, k == 0);
        umma_commit(&empty[s]);
      }
    }
    pdl_wait();
    const int units = p.term.lists[0] * per;
    for (int g0 = mine * kFewUnits; g0 < units && ok; g0 += p.parts * kFewUnits, next()) {
      ok = mbar_wait_warp(&built[s], (bph >> s) & 1, abort_flag);
      bph ^= 1u << s;
      tc_fence_after();
      if (ok && elect_one()) {
        few_mma_units(smem_u32(smem + s * kStage), tmem_base, idesc_f, min(kFewUnits, units - g0));
        umma_commit(&empty[s]);
      }
    }
    if (ok && elect_one()) umma_commit(&done);
  } else if (warp < 6) {
    pdl_wait();
    // the accumulator to shared memory (the operand stages', which nothing uses any more): [sample][128 rows]
    const int q = warp & 3;
    if (mbar_wait_warp(&done, 0, abort_flag)) {
      tc_fence_after();
      float* to = reinterpret_cast<float*>(smem) + q * 32 + lane;
#pragma unroll 1
      for (int t0 = 0; t0 < TN; t0 += 32) {
        uint32_t acc[32];
        tmem_ld_32x32(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + t0, acc);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (t0 + j < TN) to[(t0 + j) * BM] = __uint_as_float(acc[j]);
      }
    }
  } else {
    pdl_wait();
    const bool writes = warp < 6 + kWrite;
    const int t = (writes ? warp - 6 : warp - 6 - kWrite) * 32 + lane;     // this thread's sample, or share of the factors
    const int units = p.term.lists[0] * per, at = writes && t < p.n ? p.term.place[t] * per : -1;
    const uint4* src = p.term.pb + t * per * 2;
    uint32_t s = static_cast<uint32_t>(nk) % p.stages, ph = 0, bad = 0;    // ph: the phases of free_, or of landed, a bit per stage
    uint4 words[2 * kFewUnits];
    if (writes) read_units(src, at, mine * kFewUnits, min(kFewUnits, units - mine * kFewUnits), per, words);
    for (int g0 = mine * kFewUnits; g0 < units; g0 += p.parts * kFewUnits) {
      const int nu = min(kFewUnits, units - g0);
      if (!mbar_wait_warp(writes ? &free_[s] : &landed[s], (ph >> s) & 1, abort_flag)) break;
      ph ^= 1u << s;
      uint32_t wrote = 1;
      if (writes) {
        load_units<kWrite, kFewUnits>(smem + s * kStage, &landed[s], tmF, hold_units(p.term.lists, (g0 & ~31) + lane, units, per), g0, nu, p.term.boxed, m0, warp - 6);
        write_units<32 * kWrite>(words, smem + s * kStage, t, t < TN, nu);
      } else bad |= wrote = clean_units<32 * kClean, kFewUnits>(smem + s * kStage, t, nu);
      if (wrote) fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&built[s]);
      if (writes) read_units(src, at, g0 + p.parts * kFewUnits, min(kFewUnits, units - g0 - p.parts * kFewUnits), per, words);
      if (++s == static_cast<uint32_t>(p.stages)) s = 0;
    }
    if (bad) odd = 1;
  }
  __syncwarp();
  if (p.parts > 1) { cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  if (!abort_word) {
    bool any = false;
    for (int c = 0; c < p.parts; ++c) {
      uint32_t w;
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(w) : "r"(mapa_u32(smem_u32(&odd), c)) : "memory");
      any |= w != 0;
    }
    // a lane takes two rows of a sample, a warp half of its 128
    const int t1 = min((mine + 1) * TN / p.parts, p.n);
    for (int x = mine * TN / p.parts * 2 + warp; x < 2 * t1; x += kFewThreads / 32) {
      const int t = x >> 1, row = (x & 1) * 64 + 2 * lane, m = m0 + row;
      const uint32_t at = smem_u32(smem) + (t * BM + row) * 4;
      float2 v = make_float2(0.f, 0.f);
      for (int c = 0; c < p.parts; ++c) {
        float2 w;
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(w.x), "=f"(w.y) : "r"(mapa_u32(at, c)) : "memory");
        v = c ? make_float2(v.x + w.x, v.y + w.y) : w;
      }
      if (any) {
        if (m < p.m) v.x += odd_term(p.term, t, m);
        if (m + 1 < p.m) v.y += odd_term(p.term, t, m + 1);
      }
      __nv_bfloat16* y = p.Y + t * p.ldy + m;
      if (m + 1 < p.m) *reinterpret_cast<__nv_bfloat162*>(y) = __floats2bfloat162_rn(v.x, v.y);
      else if (m < p.m) *y = __float2bfloat16_rn(v.x);
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
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, kCols); }
}

// ---------------------------------------------------------------------------------------------------------
// The same for more samples, on pairs of CTAs (cta_group::2): a tile of 256 rows of A x tn samples (128 or 256), a CTA 128 of the rows in
// its TMEM; it loads its own rows and its half of the samples, 32 KB a k-block.  Two accumulators: the end of a tile runs beside the next
// one's products.  Whole rounds of tiles are taken whole, the k-blocks of the rest are shared out (Segments in sfb_tile.cuh); the pair that
// finishes a tile has its term.
// Bound by the tensor cores where the contraction is long: 4,096 samples, 10,000 x 20,000: 1,260 to 1,340 us in a stream of gradients, 1.22 to
// 1.30 PFLOP/s at the power cap (8,192, 10,000 x 5,000: 640 to 710 us, and 592 by itself, the tensor pipe 83 % busy).  Where it is short, by what a
// k-block of the term waits for: it takes a stage only once that is free, and its copies, the look at them and the other CTA's word come to
// 4,500 cycles, of which the stages ahead cover 2,500 (1,024 samples of 64 adapters of 8 ranks, 1,000 x 20,000: 61 us for 4.3 rounds of tiles of
// 16 + 3 k-blocks; with one word 57, 16,000 cycles a tile, 9,700 of them products).
//
// Warps: 0 TMA producer, 1 MMA issuer (leader CTA) and TMEM owner, 2..9 epilogue (TMEM lane quarter q, half h of the columns), 10..13
// the samples' operand of the term and the loads of its factors, 14..17 the look at them, 18, 19 and, in the other CTA, 1 hand that CTA's on to the leader.
// ---------------------------------------------------------------------------------------------------------
constexpr int kPairBuild = 4, kHand = 3, kPairThreads = 32 * (2 + kEpi + 2 * kPairBuild + kHand - 1), kGroup = 8;      // kGroup: tiles of samples that follow one another
constexpr int kPairUnits = BK / kUnit;              // units of a k-block of the term: their first words in its stage, the second ones in a ring
// Operand stages, and places of the ring of second words behind them.  (With both words in one stage, four units a k-block, six stages, half of
// the factors' places are empty, and as many fewer factors are under way: 333 samples of 150 adapters of 128 ranks, 9,000 x 1,000, 301 us, here
// 221; 300 of 32 of 128, 5,000 x 2,000, 109 and 90; 700 of 16 of 32, 4,000 x 4,000, 56.7 and 57.1; long contractions the same.  14 single places, of
// which k-blocks take two or three: long contractions 7 % longer.)
constexpr int kPairStages = 5, kPairStage = 2 * kTileBytesA, kPairSecond = 4;
constexpr int kPairSmem = kPairStages * kPairStage + kPairSecond * kTileBytesA + 1024;
// The words of the units [g0, g0 + nu) of a sample whose first unit is `at` (below zero: no adapter), zeros for those that are not its own, to
// row t of two operands: by copies of this thread, which make zeros without reading.  (With a number of bytes that is zero instead: 99 us of the 90
// above, 146 of the 135 of 150 samples of 128 adapters of 32 ranks, 20,000 x 3,000.)
__device__ __forceinline__ void copy_words(uint32_t first, uint32_t second, int t, const uint4* src, int at, int g0, int nu, int per) {
#pragma unroll
  for (int j = 0; j < kPairUnits; ++j) {
    const int u = g0 + j - at;
    const bool own = at >= 0 && j < nu && u >= 0 && u < per;
    const uint4* from = own ? src + 2 * u : src;
    const uint32_t to = t * 128 + ((j ^ (t & 7)) << 4);
    cp_async_16_or_zero(first + to, from, own);
    cp_async_16_or_zero(second + to, from + 1, own);
  }
}
constexpr int kPartFloats = BM * kMaxTile;          // what a CTA leaves of a tile
struct PairParams {
  Term term;
  Sorting sort;
  int32_t n, tn, tilesT, tilesM, m;
  int32_t kseg, cut, whole;    // k-blocks; see Segments
  __nv_bfloat16* Y;
  int64_t ldy;
  float* partial;              // [pairs][2][kPartFloats]
  uint32_t* ready;             // [pairs][2][kEpi]
  uint32_t* status;
};

__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity, volatile uint32_t* abort) {      // by a whole warp
  const long long t0 = clock64();
  bool got = false;
  for (uint32_t i = 0; i < kMaxPolls; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t"
        ".reg .pred P;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 P, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, P;\n\t"
        "}\n"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(kWaitHintNs) : "memory");
    if (ok) { got = true; break; }
    if (*abort) break;
    if (clock64() - t0 > kMaxWaitCycles) { *abort = 1; break; }
  }
  return __all_sync(0xffffffffu, got);
}

template <bool MN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
adapter_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmZ, const __grid_constant__ CUtensorMap tmSorted,
                    const __grid_constant__ CUtensorMap tmF, const __grid_constant__ PairParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kPairStages], empty[kPairStages];       // full, built, tempty: the leader's are in use
  __shared__ uint64_t free_[kPairStages], built[kPairStages];      // of a k-block of factors: the stage is free for the samples' operand;
                                                                   // this CTA has its operands
  __shared__ uint64_t landed[kPairStages], joined[kPairStages];    // its factors are here; the leader's: the other CTA has built its operands
  __shared__ uint64_t second[kPairSecond];                         // a place for second words is free
  __shared__ uint64_t tfull[2], tempty[2], looked[2], taken[2];    // looked: whether factors of a tile were not finite is known; taken: read
  __shared__ uint32_t tmem_slot, abort_word, odd[2][kPairBuild];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, half = p.tn / 2;
  const Segments segs(p.kseg, p.cut != 0, p.whole, p.tilesT * p.tilesM, pair, gridDim.x >> 1);
  const int per = units_of(p.term);
  // Tiles that run at the same time: kGroup tiles of samples against as many rows of A as there are pairs for.
  auto tile_coords = [&](int tile, int& m0, int& tt) {
    const int in = kGroup * p.tilesM, g = tile / in, width = min(kGroup, p.tilesT - g * kGroup), at = tile - g * in;
    m0 = at / width * (2 * BM) + static_cast<int>(rank) * BM;
    tt = g * kGroup + at % width;
  };

  // Hands on, in the other CTA, the term's k-blocks in the stages s with s % kHand == h: a release to the cluster, 1,650 cycles of a warp that has
  // no accesses of its own.  A stage is built again only once its k-block is multiplied, so once the warp that it belongs to has seen it: no
  // warp looks for a phase that it could miss.
  auto hand_on = [&](int h) {
    uint32_t s = 0, bph = 0;
    bool ok = true;
    for (int i = 0; i < segs.n && ok; ++i) {
      const Segment sg = segs.get(i);
      int m0, tt;
      tile_coords(sg.tile, m0, tt);
      s = (s + sg.k1 - sg.k0) % kPairStages;
      for (int left = sg.k1 == p.kseg ? p.term.lists[static_cast<int64_t>(tt) * kListPitch] * per : 0; left > 0 && ok; left -= kPairUnits) {
        if (static_cast<int>(s % kHand) == h) {
          ok = mbar_wait_warp(&built[s], (bph >> s) & 1, abort_flag);
          bph ^= 1u << s;
          fence_proxy_async_smem();                  // the words are generic writes
          if (ok && lane == 0) mbar_arrive_cluster(mapa_u32(smem_u32(&joined[s]), 0));
        }
        if (++s == static_cast<uint32_t>(kPairStages)) s = 0;
      }
    }
  };

  if (threadIdx.x == 0) {
    for (int i = 0; i < kPairStages; ++i) {
      mbar_init(&full[i], 1); mbar_init(&empty[i], 1); mbar_init(&free_[i], 1); mbar_init(&landed[i], 1); mbar_init(&joined[i], 1);
      mbar_init(&built[i], 33 * kPairBuild);         // the threads that write words, the warps that look
    }
    for (int i = 0; i < kPairSecond; ++i) mbar_init(&second[i], 1);
    for (int i = 0; i < 2; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], 2 * kEpi); mbar_init(&looked[i], kPairBuild); mbar_init(&taken[i], kEpi); }
    abort_word = 0;
    fence_barrier_init();
    prefetch_tmap(&tmA); prefetch_tmap(&tmZ); prefetch_tmap(&tmF);
  }
  if (warp == 1) { tmem_alloc_pair(&tmem_slot, 512); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  pdl_launch_dependents();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();

  if (warp == 0) {
    // ---------------- TMA producer ----------------
    const uint64_t pol = policy_evict_normal();
    const CUtensorMap* tz = p.sort.on() ? &tmSorted : &tmZ;
    uint32_t s = 0, ph = 0;
    bool ok = true;
    for (int i = 0; i < segs.n && ok; ++i) {
      const Segment sg = segs.get(i);
      int m0, tt;
      tile_coords(sg.tile, m0, tt);
      const int z0 = tt * p.tn + static_cast<int>(rank) * half;
      const int count = sg.k1 == p.kseg ? p.term.lists[static_cast<int64_t>(tt) * kListPitch] : 0;
      auto loads = [&](int k0, int k1) {
        for (int k = k0; k < k1; ++k) {
          if (!mbar_wait_warp(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
          uint8_t* st = smem + s * kPairStage;
          if (elect_one()) {
            if (rank == 0) mbar_expect_tx(&full[s], 2 * (kTileBytesA + half * BK * 2));
            const uint32_t bar = mapa_u32(smem_u32(&full[s]), 0);
            if (MN) {
              tma_load_2d_pair(st, &tmA, m0, k * BK, bar, pol);
              tma_load_2d_pair(st + kTileBytesA / 2, &tmA, m0 + 64, k * BK, bar, pol);
            } else {
              tma_load_2d_pair(st, &tmA, k * BK, m0, bar, pol);
            }
            tma_load_2d_pair(st + kTileBytesA, tz, k * BK, z0, bar, pol);
          }
          if (++s == static_cast<uint32_t>(kPairStages)) { s = 0; ph ^= 1; }
        }
      };
      loads(sg.k0, sg.k1);
      const int units = count * per, more = (units + kPairUnits - 1) / kPairUnits;
      for (int k = 0; k < more && ok; ++k) {
        if (!mbar_wait_warp(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
        const int nu = min(kPairUnits, units - k * kPairUnits);
        if (elect_one()) {
          mbar_expect_tx(&landed[s], nu * 2 * kUnit * 128);
          mbar_arrive(&free_[s]);
        }
        if (++s == static_cast<uint32_t>(kPairStages)) { s = 0; ph ^= 1; }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    if (rank == 0) {
      const uint32_t idesc = umma_idesc_bf16(2 * BM, p.tn) | (MN ? 1u << 15 : 0u), idesc_f = umma_idesc_bf16(2 * BM, p.tn) | 1u << 15;
      uint32_t s = 0, l = 0, fph = 0, bph = 0;       // stage, place of second words; the phases of full and of built, a bit per stage
      bool ok = true;
      for (int i = 0; i < segs.n && ok; ++i) {
        const Segment sg = segs.get(i);
        int m0, tt;
        tile_coords(sg.tile, m0, tt);
        const int count = sg.k1 == p.kseg ? p.term.lists[static_cast<int64_t>(tt) * kListPitch] : 0;
        const uint32_t a = i & 1, aph = (i >> 1) & 1, d_tmem = tmem_base + a * kMaxTile;
        if (!mbar_wait_warp(&tempty[a], aph ^ 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        for (int k = sg.k0; k < sg.k1; ++k) {
          if (!mbar_wait_warp(&full[s], (fph >> s) & 1, abort_flag)) { ok = false; break; }
          fph ^= 1u << s;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t st = smem_u32(smem + s * kPairStage);
            const uint64_t da = MN ? umma_desc_mn128(st) : umma_desc_k128(st), db = umma_desc_k128(st + kTileBytesA);
#pragma unroll
            for (int j = 0; j < BK / 16; ++j) umma_bf16_pair(d_tmem, da + (MN ? 128 : 2) * j, db + 2 * j, idesc, (k - sg.k0) | j ? 1u : 0u);
            umma_commit_pair(&empty[s], 3);
          }
          if (++s == static_cast<uint32_t>(kPairStages)) s = 0;
        }
        for (int left = count * per; left > 0 && ok; left -= kPairUnits) {
          if (!mbar_wait_warp(&built[s], (bph >> s) & 1, abort_flag) || !mbar_wait_cluster(&joined[s], (bph >> s) & 1, abort_flag)) { ok = false; break; }
          bph ^= 1u << s;
          fence_proxy_async_smem();                  // the words are generic writes; the other CTA's are fenced where they are handed on
          tc_fence_after();
          const int ns = (min(kPairUnits, left) + 1) / 2;                  // two units each: of their first words, of their second ones
          if (elect_one()) {
            const uint32_t st = smem_u32(smem + s * kPairStage);
            const uint64_t da = umma_desc_mn128(st), db = umma_desc_k128(st + kTileBytesA);
            const uint64_t dl = umma_desc_k128(smem_u32(smem + kPairStages * kPairStage + l * kTileBytesA));
            for (int j = 0; j < ns; ++j) {
              umma_bf16_pair(d_tmem, da + 128 * j, db + 2 * j, idesc_f, 1u);
              umma_bf16_pair(d_tmem, da + 128 * j, dl + 2 * j, idesc_f, 1u);
            }
            umma_commit_pair(&empty[s], 3);
            umma_commit_pair(&second[l], 3);
          }
          if (++l == kPairSecond) l = 0;
          if (++s == static_cast<uint32_t>(kPairStages)) s = 0;
        }
        if (ok && elect_one()) umma_commit_pair(&tfull[a], 3);
      }
    } else {
      hand_on(kHand - 1);
    }
  } else if (warp < 2 + kEpi) {
    // ---------------- epilogue ----------------
    const int e = warp - 2, q = warp & 3, h = e >> 2, cols = half;     // columns of this warp: half of tn
    const int32_t* order = p.sort.on() ? p.sort.order : nullptr;
    const uint32_t tempty0 = mapa_u32(smem_u32(&tempty[0]), 0), tempty1 = mapa_u32(smem_u32(&tempty[1]), 0);
    bool ok = true;
    for (int i = 0; i < segs.n && ok; ++i) {
      const Segment sg = segs.get(i);
      int m0, tt;
      tile_coords(sg.tile, m0, tt);
      const uint32_t a = i & 1, aph = (i >> 1) & 1;
      if (!mbar_wait_warp(&tfull[a], aph, abort_flag) || !mbar_wait_warp(&looked[a], aph, abort_flag)) { ok = false; break; }
      tc_fence_after();
      uint32_t any = 0;
#pragma unroll
      for (int w = 0; w < kPairBuild; ++w) any |= odd[a][w];
      __syncwarp();
      if (lane == 0) mbar_arrive(&taken[a]);
      const uint32_t t_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + a * kMaxTile + h * cols;
      const bool leave = sg.k1 < p.kseg;
      const int from = leave ? pair : segs.first_part(sg);
      const int slot = (static_cast<int>(rank) * kEpi + e);
      if (!leave && from < pair) {
        for (int j = from; j < pair && ok; ++j) ok = __all_sync(0xffffffffu, lane != 0 || flag_wait(p.ready + j * 2 * kEpi + slot, abort_flag));
        if (!ok) break;
        if (lane == 0)
          for (int j = from; j < pair; ++j) p.ready[j * 2 * kEpi + slot] = 0;               // for the next launch
        __syncwarp();
      }
      const int row = q * 32 + lane, m = m0 + row;
      const int64_t mine = (static_cast<int64_t>(h) * cols) * BM + row;                     // of a CTA's part: [column][128 rows]
#pragma unroll 1
      for (int c = 0; c < cols; c += 32) {
        uint32_t acc[32];
        tmem_ld_32x32(t_addr + c, acc);
        tmem_ld_wait();
        if (c + 32 >= cols) {                        // the last read of the accumulator: hand it back
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(a ? tempty1 : tempty0);
        }
        if (leave) {
          float* to = p.partial + (static_cast<int64_t>(pair) * 2 + rank) * kPartFloats + mine + static_cast<int64_t>(c) * BM;
#pragma unroll
          for (int j = 0; j < 32; ++j) __stcg(to + j * BM, __uint_as_float(acc[j]));
          continue;
        }
        for (int w = from; w < pair; ++w) {
          const float* in = p.partial + (static_cast<int64_t>(w) * 2 + rank) * kPartFloats + mine + static_cast<int64_t>(c) * BM;
          float x[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) x[j] = __ldcg(in + j * BM);
#pragma unroll
          for (int j = 0; j < 32; ++j) acc[j] = __float_as_uint(__uint_as_float(acc[j]) + x[j]);
        }
        const int i0 = tt * p.tn + h * cols + c, sample = order && i0 + lane < p.n ? order[i0 + lane] : i0 + lane;
        if (any) {
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const int i = __shfl_sync(0xffffffffu, sample, j);
            if (i0 + j < p.n && m < p.m) acc[j] = __float_as_uint(__uint_as_float(acc[j]) + odd_term(p.term, i, m));
          }
        }
        store_chunk(p.Y, p.ldy, i0, p.n, order != nullptr, sample, m, p.m, acc, lane);
      }
      __syncwarp();
      if (leave && lane == 0) {
        __threadfence();
        st_release(p.ready + pair * 2 * kEpi + slot, 1u);
      }
    }
  } else if (warp >= 2 + kEpi + 2 * kPairBuild) {
    // ---------------- hand on the other CTA's operands ----------------
    // (1,024 samples, 1,000 x 20,000, eight k-blocks of the term a tile: 98 us with releases by each of the eight warps that make the operands, 89
    // with one warp that hands all on, 76 with two in turn.  With both words in one stage, 333 samples of 150 adapters of 128 ranks, 9,000 x 1,000:
    // 351 with two in turn, 311 with two by stages, 300 with three.)
    if (rank == 1) hand_on(warp - 2 - kEpi - 2 * kPairBuild);
  } else {
    // ---------------- the samples' operand of the term, and its factors ----------------
    const bool writes = warp < 2 + kEpi + kPairBuild;
    const int w = warp - 2 - kEpi - (writes ? 0 : kPairBuild), t = w * 32 + lane;    // this thread's sample of the CTA's half of the tile, or
    uint32_t s = 0, ph = 0;                          // share of the factors; ph: the phases of free_, or of landed, a bit per stage
    uint32_t l = 0, lph = 0;                         // place of second words, and phase
    bool ok = true;
    for (int i = 0; i < segs.n && ok; ++i) {
      const Segment sg = segs.get(i);
      int m0, tt;
      tile_coords(sg.tile, m0, tt);
      s = (s + sg.k1 - sg.k0) % kPairStages;
      const int units = sg.k1 == p.kseg ? p.term.lists[static_cast<int64_t>(tt) * kListPitch] * per : 0;
      const int smp = tt * p.tn + static_cast<int>(rank) * half + t;
      const int at = writes && t < half && smp < p.n ? p.term.place[smp] * per : -1;   // this sample's first unit
      const uint4* src = p.term.pb + (at >= 0 ? static_cast<int64_t>(smp) * per * 2 : 0);
      const uint32_t a = i & 1, aph = (i >> 1) & 1;
      const int32_t* list = p.term.lists + static_cast<int64_t>(tt) * kListPitch;
      Held held = hold_units(list, lane, writes ? units : 0, per);
      if (!writes && !mbar_wait_warp(&taken[a], aph ^ 1, abort_flag)) break;
      uint32_t bad = 0;
      for (int g0 = 0; g0 < units; g0 += kPairUnits) {
        const int nu = min(kPairUnits, units - g0);
        uint8_t* st = smem + s * kPairStage;
        if (!mbar_wait_warp(writes ? &free_[s] : &landed[s], (ph >> s) & 1, abort_flag)) { ok = false; break; }
        ph ^= 1u << s;
        if (writes) {
          load_units<kPairBuild, kPairUnits>(st, &landed[s], tmF, held, g0, nu, p.term.boxed, m0, w);
          if (!mbar_wait_warp(&second[l], lph ^ 1, abort_flag)) { ok = false; break; }
          if (t < half) copy_words(smem_u32(st) + kTileBytesA, smem_u32(smem + kPairStages * kPairStage + l * kTileBytesA), t, src, at, g0, nu, per);
          if (nu & 1)                                // beside an odd last unit, zeros in the factors' operand
            cp_async_16(smem_u32(st) + (t >> 6) * (kTileBytesA / 2) + nu * (kUnit * 128) + (t & 63) * 16, src, 0);
          cp_async_arrive(&built[s]);                // (the copies arrive by themselves)
          if (++l == kPairSecond) { l = 0; lph ^= 1; }
          if (((g0 + kPairUnits) & 31) == 0) held = hold_units(list, g0 + kPairUnits + lane, units, per);
        } else {
          const uint32_t wrote = clean_units<32 * kPairBuild, kPairUnits>(st, t, nu);
          bad |= wrote;
          if (wrote) fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&built[s]);
        }
        if (++s == static_cast<uint32_t>(kPairStages)) s = 0;
      }
      bad = __any_sync(0xffffffffu, bad);
      if (!writes && lane == 0) {
        odd[a][w] = bad;
        mbar_arrive(&looked[a]);
      }
    }
    cp_async_wait_all();
  }

  // ---------------- teardown ----------------
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (abort_word) {
    if (threadIdx.x == 0) atomicOr(p.status, SFB_STATUS_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    __syncthreads();
  }
  cluster_arrive();
  cluster_wait();
  if (warp == 1) { tc_fence_after(); tmem_dealloc_pair(tmem_base, 512); }
}

// ---------------------------------------------------------------------------------------------------------
// scale p of the samples in the order of adapter_index_kernel, as three words of bf16 (24 bits): [position][word][rp], rp the rank rounded
// up to 16 with zeros: what adapter_gradient_kernel takes.  adapter_sum_kernel writes them where it forms p anyway (a launch less: 5 us a
// call), adapter_words_kernel elsewhere.
// ---------------------------------------------------------------------------------------------------------
struct WordsParams {
  Ranked p[2];                 // at null: not wanted
  __nv_bfloat16* out[2];       // both null: none
  const int32_t *ids, *order, *begin, *count;
  const int32_t* position;     // of a sample in `order`
  int64_t* work;               // [adapters * shares + 1]: what a column tile takes of the shares of adapters before each one (see adapter_work)
  const float* scale;
  int32_t rank, adapters, shares;
};
// What a tile of dF[a] costs, in k-blocks: its contraction, and its end.
__device__ __forceinline__ int adapter_work(int count) { return (count + BK - 1) / BK + 1; }
// Share c of `shares` of an adapter's samples, in whole k-blocks: where it begins, and how many they are.
__device__ __forceinline__ int share_of(int count, int shares, int c, int* first) {
  const int each = ((count + BK - 1) / BK + shares - 1) / shares * BK;
  *first = min(c * each, count);
  return min(each, count - *first);
}
// v = w0 + w1 + w2.  (What overflows in the rounding to the first word is cut off instead; of what is not finite there is no rest.)
__device__ __forceinline__ void three_words(float v, float (&w)[3]) {
  w[0] = __bfloat162float(__float2bfloat16_rn(v));
  if (isinf(w[0]) && !isinf(v)) w[0] = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  const float rest = isfinite(v) ? v - w[0] : 0.f;
  w[1] = __bfloat162float(__float2bfloat16_rn(rest));
  w[2] = rest - w[1];
}
// The words of eight values (scaled) to `to`, `to` + rp and `to` + 2 rp.
__device__ __forceinline__ void put_words(__nv_bfloat16* to, int rp, const float (&x)[8]) {
  uint32_t w[3][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float u[3], v[3];
    three_words(x[2 * j], u);
    three_words(x[2 * j + 1], v);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(u[k], v[k]);
      w[k][j] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(to + k * rp) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
}
// work, by a block of 256 threads.
__device__ __forceinline__ void sum_work(const WordsParams& p, int64_t (&sums)[256]) {
  const int all_shares = p.adapters * p.shares, each = (all_shares + 255) / 256;
  const int from = min(static_cast<int>(threadIdx.x) * each, all_shares), to = min(from + each, all_shares);
  auto work = [&](int x) {
    int first;
    return adapter_work(share_of(p.count[x / p.shares], p.shares, x % p.shares, &first));
  };
  int64_t s = 0;
  for (int a = from; a < to; ++a) s += work(a);
  sums[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 32) {                            // a lane the eight sums from 8 * lane on
    int64_t v[8], all = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) { v[u] = all; all += sums[threadIdx.x * 8 + u]; }
    int64_t before = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, before, o);
      if (static_cast<int>(threadIdx.x) >= o) before += x;
    }
    before -= all;
#pragma unroll
    for (int u = 0; u < 8; ++u) sums[threadIdx.x * 8 + u] = before + v[u];
  }
  __syncthreads();
  s = sums[threadIdx.x];
  for (int a = from; a < to; ++a) { p.work[a] = s; s += work(a); }
  if (to == all_shares && from < to) p.work[all_shares] = s;
}

__global__ void __launch_bounds__(256) adapter_words_kernel(const __grid_constant__ WordsParams p) {
  __shared__ int64_t sums[256];
  pdl_launch_dependents();
  pdl_wait();
  const int rp = (p.rank + 15) & ~15, pieces = rp / 8;
  const int64_t total = static_cast<int64_t>(p.begin[p.adapters - 1] + p.count[p.adapters - 1]) * pieces;
  const int side = blockIdx.y;
  if (side == 2) {
    if (blockIdx.x == 0) sum_work(p, sums);
    return;
  }
  if (!p.out[side]) return;
  for (int64_t x = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; x < total; x += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t at = x / pieces;
    const int c = static_cast<int>(x - at * pieces), i = p.order[at];
    const float sc = p.scale[p.ids[i]];
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = c * 8 + j;
      v[j] = r < p.rank ? sc * ranked(p.p[side], static_cast<int64_t>(i) * p.rank + r) : 0.f;
    }
    put_words(p.out[side] + at * 3 * rp + c * 8, rp, v);
  }
}

// ---------------------------------------------------------------------------------------------------------
// More than 64 samples: p from its parts, zeros for a sample without an adapter, and scale p as two words (pb).  In the first blocks the lists of
// the tiles of the product.
// ---------------------------------------------------------------------------------------------------------
struct SumParams {
  Ranked p;
  const int32_t* ids;
  Sorting sort;
  const float* scale;
  int64_t n;
  int32_t rank, adapters;
  float* out;                  // by samples; all else by positions
  __nv_bfloat16* pb;
  int32_t tiles, tn;           // a block per tile of tn samples
  int32_t* lists;              // [tiles][kListPitch]
  int32_t* place;              // per sample its place in its tile's list
  uint32_t* status;
  WordsParams words;           // of p (p[1], from here) and of the other side's products
};

// Blocks 0 .. tiles: a tile's list; what the gradients' blocks share the work by.
__device__ __forceinline__ void lists_and_work(const SumParams& p, int tile, const int32_t* ids) {
  __shared__ alignas(16) TileList<kMaxTile> L;
  __shared__ int64_t sums[256];
  if (tile < p.tiles) {
    const int first = tile * p.tn;
    build_list(L, ids, first, static_cast<int>(p.n), p.tn, p.adapters, p.status);
    int32_t* to = p.lists + static_cast<int64_t>(tile) * kListPitch;
    if (threadIdx.x == 0) to[0] = L.count;
    for (int t = threadIdx.x; t < p.tn; t += 256) {
      if (t < L.count) to[1 + t] = L.list[t];
      if (first + t < p.n) p.place[first + t] = L.place[t];
    }
  } else {
    sum_work(p.words, sums);
  }
}

__global__ void __launch_bounds__(256) adapter_sum_kernel(const __grid_constant__ SumParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int tile = blockIdx.x;
  const bool sorted = p.sort.on();
  const int32_t* ids = sorted ? p.sort.ids : p.ids;
  const bool wanted = p.words.out[0] || p.words.out[1];
  const int more = p.tiles + (wanted ? 1 : 0);
  if (tile < more) {
    lists_and_work(p, tile, ids);
    return;
  }
  const int per = (p.rank + kUnit - 1) / kUnit, rp = (p.rank + 15) & ~15;
  const int64_t blocks = gridDim.x - more;
  // four lanes a unit, each some of the parts (by whole warps: a unit behind the last one is formed, not written)
  const int turn = threadIdx.x & 3;
  for (int64_t base = static_cast<int64_t>(tile - more) * 64; base < p.n * per; base += blocks * 64) {
    const int64_t at = base + (threadIdx.x >> 2), x = min(at, p.n * per - 1), i = x / per;
    const int r0 = static_cast<int>(x - i * per) * kUnit, id = ids[i];
    const bool has = id >= 0 && id < p.adapters;
    const float sc = has ? p.scale[id] : 0.f;
    float v[kUnit];
    const int64_t sample = sorted ? p.sort.order[i] : i, from = i * p.rank + r0, into = sample * p.rank + r0;
    if (p.rank % kUnit == 0) {                       // (rows of p are whole pieces of 32 bytes then)
#pragma unroll
      for (int j = 0; j < kUnit; ++j) v[j] = 0.f;
      if (has) {
#pragma unroll 4
        for (int c = turn; c < p.p.parts; c += 4) {
          const float4* in = reinterpret_cast<const float4*>(p.p.at + c * p.p.stride + from);
          const float4 a = in[0], b = in[1];
          v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
        }
      }
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        v[j] += __shfl_xor_sync(0xffffffffu, v[j], 1);
        v[j] += __shfl_xor_sync(0xffffffffu, v[j], 2);
      }
      if (turn || at >= p.n * per) continue;
    } else {
      if (turn || at >= p.n * per) continue;
#pragma unroll
      for (int j = 0; j < kUnit; ++j) v[j] = has && r0 + j < p.rank ? ranked(p.p, from + j) : 0.f;
    }
    if (p.rank % kUnit == 0 && (reinterpret_cast<uintptr_t>(p.out) & 15) == 0) {
      float4* to = reinterpret_cast<float4*>(p.out + into);
      to[0] = make_float4(v[0], v[1], v[2], v[3]);
      to[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int j = 0; j < kUnit; ++j)
        if (r0 + j < p.rank) p.out[into + j] = v[j];
    }
    uint32_t w[2][kUnit / 2];
#pragma unroll
    for (int j = 0; j < kUnit / 2; ++j) {
      float a[2], b[2];
      two_words(has ? sc * v[2 * j] : 0.f, a);
      two_words(has ? sc * v[2 * j + 1] : 0.f, b);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const __nv_bfloat162 ab = __floats2bfloat162_rn(a[k], b[k]);
        w[k][j] = *reinterpret_cast<const uint32_t*>(&ab);
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) reinterpret_cast<uint4*>(p.pb)[2 * x + k] = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
    if (!wanted || !has) continue;
    const int64_t row = (static_cast<int64_t>(p.words.position[sample]) * 3) * rp + r0;
    const bool behind = r0 + 2 * kUnit == rp && r0 + kUnit >= p.rank;        // a piece of zeros follows
    const float zeros[kUnit] = {};
    for (int side = 0; side < 2; ++side) {
      __nv_bfloat16* to = p.words.out[side];
      if (!to) continue;
      float u[kUnit];
#pragma unroll
      for (int j = 0; j < kUnit; ++j) u[j] = r0 + j < p.rank ? sc * (side ? v[j] : ranked(p.words.p[0], into + j)) : 0.f;
      put_words(to + row, rp, u);
      if (behind) put_words(to + row + kUnit, rp, zeros);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------
// adapter_rank_kernel and adapter_sum_kernel in one for few entries in all, in fp32 FMAs: a block takes four ranks of one sample, its threads
// pieces of 16 bytes of the contraction.  Bound by latency: ids, then the factors, then the block's sum, where the tensor cores have tiles to
// set up, parts to add and a list ahead of their first load.  (us a forward pass, those and this one: 1 sample of 16 ranks, 10,000 x 5,000:
// 24.5 and 22.3; 16, 2,000 x 3,000: 17 and 11; 64, 22 and 12; 37, 10,000 x 20,000: 77.6 and 72.7; 64 of 64 ranks, 2,000 x 10,000: 30.8 and 27.5,
// 2,000 x 20,000: 40.0 and 41.6; 64 of 128 and 30 adapters, 2,000 x 20,000: 64 and 72; 100 of 16, 2,000 x 3,000: 40 and 27; 200 of 16, 5,000 x
// 10,000: 68 and 56.  Gradients: 128 samples of 4 ranks, 64 x 256: 34 and 22; 1,000 of 16, 2,000 x 3,000: 61 and 62.)
// ---------------------------------------------------------------------------------------------------------
constexpr int kDotRanks = 4;
struct DotParams {
  SumParams s;                 // s.p: not used
  const __nv_bfloat16 *F, *Z;
  int64_t ldf, ldz;
  int32_t d;
};
__device__ __forceinline__ void dot8(const uint4& a, const uint4& b, float& sum) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    sum = fmaf(__uint_as_float(x[j] << 16), __uint_as_float(y[j] << 16), sum);
    sum = fmaf(__uint_as_float(x[j] & 0xffff0000u), __uint_as_float(y[j] & 0xffff0000u), sum);
  }
}

__global__ void __launch_bounds__(256) adapter_dot_kernel(const __grid_constant__ DotParams p) {
  __shared__ float part[8][kDotRanks];
  pdl_wait();
  pdl_launch_dependents();
  const SumParams& q = p.s;
  const bool sorted = q.sort.on(), wanted = q.words.out[0] || q.words.out[1];
  const int more = q.tiles + (wanted ? 1 : 0), block = static_cast<int>(blockIdx.x) - more;
  if (block < 0) {
    lists_and_work(q, blockIdx.x, sorted ? q.sort.ids : q.ids);
    return;
  }
  const int rank = q.rank, per8 = (rank + kUnit - 1) / kUnit * kUnit, groups = per8 / kDotRanks;
  const int i = block / groups, r0 = (block - i * groups) * kDotRanks, sample = sorted ? q.sort.order[i] : i, id = q.ids[sample];
  const bool has = id >= 0 && id < q.adapters;
  float sum[kDotRanks] = {};
  if (has && r0 < rank) {
    const __nv_bfloat16* z = p.Z + sample * p.ldz;
    const __nv_bfloat16* f[kDotRanks];
#pragma unroll
    for (int r = 0; r < kDotRanks; ++r) f[r] = p.F + (static_cast<int64_t>(id) * rank + min(r0 + r, rank - 1)) * p.ldf;
    const int whole = p.d / 8;
#pragma unroll 2
    for (int c = threadIdx.x; c < whole; c += 256) {
      const uint4 a = *reinterpret_cast<const uint4*>(z + c * 8);
      uint4 b[kDotRanks];
#pragma unroll
      for (int r = 0; r < kDotRanks; ++r) b[r] = *reinterpret_cast<const uint4*>(f[r] + c * 8);
#pragma unroll
      for (int r = 0; r < kDotRanks; ++r) dot8(a, b[r], sum[r]);
    }
    const int e = whole * 8 + threadIdx.x;
    if (e < p.d)
#pragma unroll
      for (int r = 0; r < kDotRanks; ++r) sum[r] = fmaf(__bfloat162float(z[e]), __bfloat162float(f[r][e]), sum[r]);
  }
#pragma unroll
  for (int r = 0; r < kDotRanks; ++r) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5][r] = sum[r];
  }
  __syncthreads();
  const int rp = (rank + 15) & ~15, r = r0 + threadIdx.x;
  // the last block of a sample also has the words behind the ranks
  if (r >= (r0 + kDotRanks == per8 ? rp : r0 + kDotRanks)) return;
  float v = 0.f;
  if (threadIdx.x < kDotRanks)
#pragma unroll
    for (int w = 0; w < 8; ++w) v += part[w][threadIdx.x];
  const int64_t at = static_cast<int64_t>(sample) * rank + r;
  const float sc = has ? q.scale[id] : 0.f;
  if (r < rank) q.out[at] = v;
  if (r < per8) put_pair(q.pb, i, per8 / kUnit, r, has && r < rank ? sc * v : 0.f);
  if (!wanted || !has) return;
  const int64_t row = static_cast<int64_t>(q.words.position[sample]) * 3 * rp + r;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    __nv_bfloat16* to = q.words.out[side];
    if (!to) continue;
    float w[3];
    three_words(r < rank ? sc * (side ? v : ranked(q.words.p[0], at)) : 0.f, w);
#pragma unroll
    for (int k = 0; k < 3; ++k) to[row + k * rp] = __float2bfloat16_rn(w[k]);
  }
}

// ---------------------------------------------------------------------------------------------------------
// [rows][pitch_in] to [rows][pitch_out], `pieces` of 16 bytes a row.  A row of a box is 128 bytes, four sectors of L2; where the rows of an
// operand are an odd multiple of 16 bytes apart, half of them are five, and the products of many samples, which move their operands
// through L2 at its rate, take up to 1.4 times as long (8,192 samples, 10,000 x 5,000 in a loop: pitches of 5,000 entries 997 us, 5,008 774,
// 5,056 720).  Such operands are copied where the copy, 4 bytes an entry at HBM's rate and a launch, costs less than that, which it does from
// 3,500 uses of a row on: us without and with it, of X for 8,192 samples and 2,200 rows of 5,000 entries 205 and 216, 3,000 277 and 281, 3,500 310
// and 310, 4,000 340 and 334; of W, 10,000 x 5,000, for 2,200 samples 247 and 261, 3,000 327 and 331, 3,500 375 and 373, 4,000 426 and 419.
// ---------------------------------------------------------------------------------------------------------
// Samples that are taken in the order of their adapters come here too (if_sorted: only then is there anything to do).
constexpr int64_t kCopyUses = 4096;
__global__ void __launch_bounds__(256) adapter_copy_kernel(const uint4* in, int64_t pitch_in, uint4* out, int64_t pitch_out, int64_t rows, int64_t pieces,
                                                           const __grid_constant__ Sorting sort, bool if_sorted) {
  pdl_launch_dependents();
  pdl_wait();
  const bool sorted = sort.on();
  if (if_sorted && !sorted) return;
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256, step_r = step / pieces, step_c = step - step_r * pieces;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  int64_t r = first / pieces, c = first - r * pieces;
  while (r < rows) {
    uint4 v[4];
    int64_t to[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      to[u] = r < rows ? r * pitch_out + c : -1;
      if (r < rows) v[u] = __ldcs(in + (sorted ? sort.order[r] : r) * pitch_in + c);
      r += step_r;
      c += step_c;
      if (c >= pieces) { c -= pieces; ++r; }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (to[u] >= 0) out[to[u]] = v[u];
  }
}

// ---------------------------------------------------------------------------------------------------------
// The samples of each adapter, one adapter after another, in their order, and those without one behind them: a block per adapter, each of its
// warps (8, beyond 2,048 samples 32) over a share of the ids, counts the samples of lower adapters and its own, then writes its own.
//
// Whether the products had better take the samples in that order: a tile of samples reads the factors of each adapter among them, and its
// share of the term grows by as much, while samples in order have to be copied.  More blocks (tiles of them) count the adapters of each 128
// samples as they come, and the last block of all compares the bytes: a factor's entries times the ranks of the pairs of a tile and an
// adapter that there are fewer of, against those of the samples, read and written.  (Gradients, us as the samples come and in order: 1,024
// samples of 64 adapters of 8 ranks at random, 1,000 x 20,000: 150 and 122; 2,000 of 100 adapters of 32 ranks, 5,000 x 5,000: 390 and 206;
// 4,096 of 8 adapters of 128, 4,000 x 20,000: 1,093 and 793.  Finding out that it does not pay, a forward pass of 8,192 samples of 64 adapters of
// 16 ranks, one request after another, 10,000 x 5,000: 776 to 785 and 787 to 799.)
//
// Every block reads all ids, adapters x samples reads: 6 us of a call for 64 adapters and 1,024 samples, 12 for 32 and 4,096.
// ---------------------------------------------------------------------------------------------------------
struct IndexParams {
  const int32_t* ids;
  int32_t n, adapters, rank16;
  int32_t *order, *begin, *count, *position;
  int32_t* sorted_ids;
  int32_t tiles;               // 0: the samples stay as they are
  int64_t width, d;            // entries of a factor that a tile reads, of a sample
  uint32_t *tally, *sorted;    // [3]: pairs, adapters with samples, blocks done
  uint32_t* status;
};

constexpr int kIndexWarps = 32;                      // at most
__device__ __forceinline__ void index_adapter(const IndexParams& p, int a, int (&below_of)[kIndexWarps], int (&own_of)[kIndexWarps]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int64_t share = (static_cast<int64_t>(p.n) + 256 * warps - 1) / (256 * warps) * 256, from = warp * share, to = min(static_cast<int64_t>(p.n), from + share);
  bool bad = false;
  auto key = [&](int64_t i) {                        // samples without an adapter come last
    const int id = i < to ? p.ids[i] : -1;
    bad |= id < -1 || id >= p.adapters;
    return i < to ? (id >= 0 && id < p.adapters ? id : p.adapters) : p.adapters + 1;
  };
  int below = 0, own = 0;
  for (int64_t b = from; b < to; b += 256) {
    int id[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) id[u] = key(b + u * 32 + lane);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      below += id[u] < a;
      own += id[u] == a;
    }
  }
  if (a == 0 && bad) atomicOr(p.status, SFB_STATUS_ADAPTER_RANGE);
  below = __reduce_add_sync(0xffffffffu, below);
  own = __reduce_add_sync(0xffffffffu, own);
  if (lane == 0) { below_of[warp] = below; own_of[warp] = own; }
  __syncthreads();
  int64_t at = 0;
  int total = 0;
  for (int w = 0; w < warps; ++w) {
    at += below_of[w] + (w < warp ? own_of[w] : 0);
    total += own_of[w];
  }
  if (threadIdx.x == 0) {
    if (a < p.adapters) { p.begin[a] = static_cast<int32_t>(at); p.count[a] = total; }
    if (p.tiles && a < p.adapters && total) atomicAdd(p.tally + 1, 1u);
  }
  if (own == 0) return;
  for (int64_t b = from; b < to; b += 256) {
    int id[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) id[u] = key(b + u * 32 + lane);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint32_t m = __ballot_sync(0xffffffffu, id[u] == a);
      if (id[u] == a) {
        const int64_t to_at = at + __popc(m & ((1u << lane) - 1));
        p.order[to_at] = static_cast<int32_t>(b + u * 32 + lane);
        p.position[b + u * 32 + lane] = static_cast<int32_t>(to_at);
        if (p.tiles) p.sorted_ids[to_at] = a < p.adapters ? a : -1;
      }
      at += __popc(m);
    }
  }
}

__global__ void __launch_bounds__(32 * kIndexWarps) adapter_index_kernel(const __grid_constant__ IndexParams p) {
  __shared__ alignas(16) TileList<kRankTile> L;
  __shared__ int below_of[kIndexWarps], own_of[kIndexWarps];
  pdl_launch_dependents();
  pdl_wait();
  const int tile = static_cast<int>(blockIdx.x) - p.adapters - 1;
  if (tile < 0) {
    index_adapter(p, blockIdx.x, below_of, own_of);
  } else {
    build_list(L, p.ids, tile * kRankTile, p.n, kRankTile, p.adapters, p.status);
    if (threadIdx.x == 0) atomicAdd(p.tally, static_cast<uint32_t>(L.count));
  }
  if (p.tiles && threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(p.tally + 2, 1u) == gridDim.x - 1) {
      __threadfence();
      const int64_t fewer = static_cast<int64_t>(__ldcg(p.tally)) - p.tiles - __ldcg(p.tally + 1);
      *p.sorted = fewer * p.rank16 * p.width > 2ll * p.n * p.d;
      p.tally[0] = p.tally[1] = p.tally[2] = 0;      // for the next launch
    }
  }
}

// ---------------------------------------------------------------------------------------------------------
// dF[a] = sum_{i of a} (scale p_i) z_i^T for a tile of 256 columns of z (128 where the ranks fill the accumulators): the columns are the
// rows of two accumulators, the ranks of the three words their columns (added at the end), the samples the contraction, 64 of them at a
// time, gathered in the order of adapter_index_kernel (so no sample of another adapter is in the product).
// Warps: 0..7 loaders (asynchronous copies of 16 bytes into both operands, which arrive at the stage's barrier by themselves: a loader that
// waited for its copies and fenced them had one k-block under way), 8 MMA issuer and TMEM owner, 9..16 epilogue, four of them a half of
// the columns.
// Bound by the instructions around a k-block, of which an adapter with few samples has one a tile: 1,024 samples of 64 adapters, 21,000
// columns, 8 ranks: 63 us with tiles of 128 columns, 40 with 256, 33 with two blocks an SM, which share its TMEM (up to 16 ranks: with more
// a block has no second accumulator then, and 24 to 32 ranks take 1.2 times as long).
// ---------------------------------------------------------------------------------------------------------
constexpr int kLoaders = 8, kGradThreads = 32 * (kLoaders + 9), kGradBuffers = 8, kGradStages = 8, kGradRing = 196608;
struct GradSide {
  const __nv_bfloat16* z;      // [n][ldz]
  int64_t ldz;
  int32_t width, tiles;        // columns; tiles of them (0: not wanted)
  const __nv_bfloat16* words;
  float* out;                  // [adapters][rank][width]: of the first share
  float* more;                 // [shares - 1][adapters][rank][width]: of the others
};
struct GradParams {
  GradSide side[2];
  int32_t rank, adapters, shares, stages;
  const int32_t *order, *begin, *count;
  const int64_t* work;
  uint32_t* status;
};
// Columns of an accumulator for the three words of all ranks; halves of a tile; panels of 64 ranks; bytes of a stage.
__host__ __device__ inline int grad_pitch(int rank) { return (3 * ((rank + 15) / 16 * 16) + 31) / 32 * 32; }
__host__ __device__ inline int grad_halves(int rank) { return grad_pitch(rank) <= 256 ? 2 : 1; }
__host__ __device__ inline int grad_blocks(int rank) { return grad_pitch(rank) <= 64 ? 2 : 1; }           // that share an SM
__host__ __device__ inline int grad_panels(int rank) { return (3 * ((rank + 15) / 16 * 16) + 63) / 64; }
__host__ __device__ inline int grad_stage(int rank) { return grad_halves(rank) * kTileBytesA + grad_panels(rank) * 8192; }

// A block's tiles: those whose work begins in its share of all work, the columns of an adapter one after another, so that a block
// keeps an adapter's samples at hand.
struct GradWalk {
  const GradParams& p;
  GradSide sd;
  int side, a, tile, count, begin;      // a: share a % shares of adapter a / shares
  int64_t at, end;             // where the tile's work begins; the end of the block's part of all work
  __device__ __forceinline__ GradWalk(const GradParams& p_) : p(p_) {
    const int64_t each = p.work[p.adapters * p.shares], first = each * p.side[0].tiles, all = first + each * p.side[1].tiles;
    at = all * blockIdx.x / gridDim.x;
    end = all * (blockIdx.x + 1) / gridDim.x;
    side = at >= first;
    sd = side ? p.side[1] : p.side[0];
    const int64_t base = side ? first : 0, tiles = sd.tiles;
    int lo = 0, len = at < end ? p.adapters * p.shares : 1;     // the last adapter whose work begins at or before `at`
    const int lane = threadIdx.x & 31;
    while (len > 1) {
      const int step = (len + 31) / 32, x = lane * step;
      const int j = 31 - __clz(__ballot_sync(0xffffffffu, x < len && (x == 0 || base + p.work[lo + x] * tiles <= at)));
      lo += j * step;
      len = min(step, len - j * step);
    }
    a = lo;
    if (at >= end) return;
    load();
    const int64_t from = base + p.work[a] * tiles, w = adapter_work(count);
    tile = static_cast<int>((at - from + w - 1) / w);
    at = from + tile * w;
    settle();
  }
  __device__ __forceinline__ void load() {
    const int of = a / p.shares;
    int first;
    count = share_of(p.count[of], p.shares, a - of * p.shares, &first);
    begin = p.begin[of] + first;
  }
  // where the share's dF goes
  __device__ __forceinline__ float* out() const {
    const int of = a / p.shares, c = a - of * p.shares;
    const int64_t entries = static_cast<int64_t>(p.rank) * sd.width;
    return (c ? sd.more + static_cast<int64_t>(c - 1) * p.adapters * entries : sd.out) + of * entries;
  }
  __device__ __forceinline__ void settle() {
    while (at < end && tile >= sd.tiles) {
      tile = 0;
      if (++a == p.adapters * p.shares) {
        a = 0;
        if (++side > 1) { at = end; return; }
        sd = p.side[1];
      }
      load();
    }
  }
  __device__ __forceinline__ bool valid() const { return at < end; }
  __device__ __forceinline__ void next() {
    at += adapter_work(count);
    ++tile;
    settle();
  }
};

__device__ __forceinline__ void grad_load(const GradParams& p, uint8_t* smem, uint64_t* full, uint64_t* empty, volatile uint32_t* abort_flag) {
  const int rp = (p.rank + 15) & ~15, pieces = 3 * rp / 8, stage = grad_stage(p.rank), halves = grad_halves(p.rank), shift = halves + 3;
  const int tid = threadIdx.x;
  // of z: pieces of 16 bytes, c of the rows r0, r0 + step, ..; of the words: pieces wc, wc + 4, .. of row wr
  const int c = tid & ((1 << shift) - 1), r0 = tid >> shift, step = (32 * kLoaders) >> shift, wr = tid >> 2, wc = tid & 3;
  const uint32_t base = smem_u32(smem);
  const uint32_t to_z = (c >> 3) * (kTileBytesA / 2) + r0 * 128 + (((c & 7) ^ (r0 & 7)) << 4), to_w = halves * kTileBytesA + wr * 128;
  uint32_t s = 0, ph = 0;
  int known = -1, known_k = -1;                      // the adapter and the k-block of the samples in row
  int32_t row[8];
  for (GradWalk it(p); it.valid(); it.next()) {
    const GradSide& sd = it.sd;
    const int nk = (it.count + BK - 1) / BK;
    const int col = it.tile * (halves * BM) + c * 8, left = sd.width - col;
    const uint32_t bytes = left >= 8 ? 16 : left > 0 ? left * 2 : 0;
    const __nv_bfloat16* z = sd.z + (bytes ? col : 0);
    const __nv_bfloat16* words = sd.words + (static_cast<int64_t>(it.begin) + wr) * 3 * rp + wc * 8;
    for (int k = 0; k < nk; ++k, words += BK * 3 * rp) {
      const int here = it.count - k * BK;            // samples from here on
      if (known != it.a || known_k != k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) row[j] = r0 + j * step < min(here, BK) ? p.order[it.begin + k * BK + r0 + j * step] : -1;
        known = it.a;
        known_k = k;
      }
      const int rows = min(BK, (here + 15) & ~15);   // whole instructions of 16
      if (!mbar_wait(&empty[s], ph ^ 1, abort_flag)) return;
      const uint32_t st = base + s * stage;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j * step >= rows) break;
        cp_async_16(st + to_z + j * step * 128, row[j] >= 0 ? z + row[j] * sd.ldz : z, row[j] >= 0 ? bytes : 0);
      }
      if (wr < rows) {
        const uint32_t b = wr < here ? 16 : 0;
        const __nv_bfloat16* from = b ? words : sd.words;
        for (int ch = wc; ch < pieces; ch += 4, from += b ? 32 : 0)
          cp_async_16(st + to_w + (ch >> 3) * 8192 + (((ch & 7) ^ (wr & 7)) << 4), from, b);
      }
      cp_async_arrive(&full[s]);
      if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1; }
    }
  }
  cp_async_wait_all();
}

template <int BLOCKS>
__global__ void __launch_bounds__(kGradThreads, BLOCKS) adapter_gradient_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kGradStages], empty[kGradStages], tfull[kGradBuffers], tempty[kGradBuffers];
  __shared__ uint32_t tmem_slot, abort_word;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  volatile uint32_t* abort_flag = &abort_word;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int rp = (p.rank + 15) & ~15, N = 3 * rp, stage = grad_stage(p.rank);
  constexpr uint32_t kColumns = 512 / BLOCKS;
  const uint32_t pitch = grad_pitch(p.rank), halves = grad_halves(p.rank), each = min(static_cast<uint32_t>(kGradBuffers), kColumns / pitch) / halves;
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) { mbar_init(&full[i], 32 * kLoaders); mbar_init(&empty[i], 1); }
    for (int i = 0; i < kGradBuffers; ++i) { mbar_init(&tfull[i], 1); mbar_init(&tempty[i], 4); }
    abort_word = 0;
    fence_barrier_init();
  }
  if (warp == kLoaders) { tmem_alloc(&tmem_slot, kColumns); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();

  if (warp < kLoaders) {
    grad_load(p, smem, full, empty, abort_flag);
  } else if (warp == kLoaders) {
    // more than 256 columns: 192 (three panels), then the rest
    const uint32_t n1 = N <= 256 ? N : 192, n2 = N - n1;
    const uint32_t idesc1 = umma_idesc_bf16(BM, n1) | kIdescMnMajor, idesc2 = umma_idesc_bf16(BM, n2 ? n2 : 16) | kIdescMnMajor;
    uint32_t s = 0, ph = 0, b = 0, bph = 0;          // stage and phase; accumulator (of each half) and phase
    bool ok = true;
    for (GradWalk it(p); it.valid() && ok; it.next()) {
      const int nk = (it.count + BK - 1) / BK;
      for (int k0 = 0; k0 < nk && ok; k0 += kDrain) {
        for (uint32_t h = 0; h < halves && ok; ++h) ok = mbar_wait_warp(&tempty[h * each + b], bph ^ 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        for (int k = k0; k < min(k0 + kDrain, nk); ++k) {
          if (!mbar_wait_warp(&full[s], ph, abort_flag)) { ok = false; break; }
          fence_proxy_async_smem();                  // the loaders' copies are generic writes: ahead of the tensor core's reads
          tc_fence_after();
          const int steps = min(BK / 16, (it.count - k * BK + 15) / 16);
          if (elect_one()) {
            const uint32_t st = smem_u32(smem + s * stage), bt = st + halves * kTileBytesA;
            const uint64_t db = umma_desc_mn128(bt), db2 = umma_desc_mn128(bt + 3 * 8192);
            for (uint32_t h = 0; h < halves; ++h) {
              const uint64_t da = umma_desc_mn128(st + h * kTileBytesA);
              const uint32_t d_tmem = tmem_base + (h * each + b) * pitch;
              for (int j = 0; j < steps; ++j) {
                umma_bf16(d_tmem, da + 128 * j, db + 128 * j, idesc1, (k - k0) | j ? 1u : 0u);
                if (n2) umma_bf16(d_tmem + 192, da + 128 * j, db2 + 128 * j, idesc2, (k - k0) | j ? 1u : 0u);
              }
            }
            umma_commit(&empty[s]);
          }
          if (++s == static_cast<uint32_t>(p.stages)) { s = 0; ph ^= 1; }
        }
        if (ok && elect_one())
          for (uint32_t h = 0; h < halves; ++h) umma_commit(&tfull[h * each + b]);
        if (++b == each) { b = 0; bph ^= 1; }
      }
    }
  } else {
    const int q = warp & 3;
    const uint32_t h = (warp - kLoaders - 1) >> 2;
    uint32_t b = 0, bph = 0;
    bool ok = h < halves;
    for (GradWalk it(p); it.valid() && ok; it.next()) {
      const GradSide& sd = it.sd;
      const int m = (it.tile * static_cast<int>(halves) + static_cast<int>(h)) * BM + q * 32 + lane, nk = (it.count + BK - 1) / BK;
      const bool in = m < sd.width;
      const int64_t width = sd.width;
      float* const out = it.out() + m;
      if (nk == 0 && in) {
        float* to = out;
        for (int r = 0; r < p.rank; ++r, to += width) *to = 0.f;
      }
      for (int k0 = 0; k0 < nk; k0 += kDrain) {
        if (!mbar_wait_warp(&tfull[h * each + b], bph, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t t_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + (h * each + b) * pitch;
        float* to = out;
#pragma unroll 1
        for (int r0 = 0; r0 < p.rank; r0 += 8, to += 8 * width) {
          uint32_t w0[8], w1[8], w2[8];
          tmem_ld_32x8(t_addr + r0, w0);
          tmem_ld_32x8(t_addr + rp + r0, w1);
          tmem_ld_32x8(t_addr + 2 * rp + r0, w2);
          tmem_ld_wait();
          float v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {               // (an infinite entry of z times a second word may be NaN, or the other infinity)
            const float first = __uint_as_float(w0[j]), rest = __uint_as_float(w1[j]) + __uint_as_float(w2[j]);
            v[j] = isfinite(first) ? first + rest : first;
          }
          const int live = in ? p.rank - r0 : 0;
          if (k0) {
            float old[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) old[j] = j < live ? to[j * width] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += old[j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < live) to[j * width] = v[j];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&tempty[h * each + b]);
        if (++b == each) { b = 0; bph ^= 1; }
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
  if (warp == kLoaders) { tc_fence_after(); tmem_dealloc(tmem_base, kColumns); }
}

// The shares of dF added up, in their order.  (16-byte pieces where there are only whole ones.)
__global__ void __launch_bounds__(256) adapter_join_kernel(float* out, const float* more, int64_t entries, int shares) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256, first = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (entries % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0) {
    for (int64_t x = first; x < entries / 4; x += step) {
      float4 v = reinterpret_cast<float4*>(out)[x];
      for (int c = 0; c + 1 < shares; ++c) {
        const float4 w = reinterpret_cast<const float4*>(more + c * entries)[x];
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
      }
      reinterpret_cast<float4*>(out)[x] = v;
    }
  } else {
    for (int64_t x = first; x < entries; x += step) {
      float v = out[x];
      for (int c = 0; c + 1 < shares; ++c) v += more[c * entries + x];
      out[x] = v;
    }
  }
}

// ---------------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------------
// Samples of a tile of adapter_rank_kernel; parts of its contraction: as many as give every SM two blocks, of four k-blocks at least.
int rank_tile(int64_t n) { return std::min(tile_of(n), kRankTile); }
int rank_parts(int64_t n, int64_t d) {
  const int64_t tiles = std::max<int64_t>(1, (n + rank_tile(n) - 1) / rank_tile(n)), kseg = (d + BK - 1) / BK;     // (a handle's n may be 0)
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({kMaxParts, 2 * kModelSms / tiles, kseg / 4})));
}
// Chunks of a tile, at most; blocks up to 64 samples: one an SM, and no more than there can be parts of chunks.
int rank_chunks(const sfb_adapter_config& c, int64_t n) { return (std::min(rank_tile(n), c.adapters) * ((c.rank + kSlice - 1) / kSlice) + 7) / 8; }
int few_rank_blocks(const sfb_adapter_config& c, int64_t n, int64_t d) { return std::max(1, std::min(kModelSms, rank_chunks(c, n) * rank_parts(n, d))); }
// Most samples x parts of a call of up to n samples.
int64_t rank_rows(int64_t n, int64_t d) {
  int64_t most = 0;
  for (int64_t tiles = 1; tiles <= 2 * kModelSms; ++tiles) {
    const int64_t m = std::min(n, tiles * kRankTile);
    most = std::max(most, m * rank_parts(m, d));
    if (m == n) return most;
  }
  return std::max(most, n);
}

// Shares that the samples of every adapter are cut into for the gradients: as many as the SMs have room for beside one another, of four
// k-blocks at least on average, since a block takes the k-blocks of a tile one after another.
// (us, gradients with one share and with these: 8,192 samples of one adapter of 16 ranks, 4,096 x 4,096: 427 and 253; 2,048, 1,000 x 1,000: 80 and
// 60; 12,000 of 8 adapters of 1 rank, 40 x 100: 137 and 76.)
int grad_shares(const sfb_adapter_config& c, int64_t n) {
  const int64_t tile = grad_halves(c.rank) * BM, items = ((c.rows + tile - 1) / tile + (c.cols + tile - 1) / tile) * c.adapters;
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({8, grad_blocks(c.rank) * kModelSms / items, n / c.adapters / (4 * BK)})));
}

// Whether adapter_dot_kernel is the one that forms the products of n samples with factors of d entries: up to these products, and samples x units
// of ranks.
constexpr int64_t kDotMost = 48 << 20, kDotUnits = 2048;
bool use_dot(const sfb_adapter_config& c, int64_t n, int64_t d) {
  return n * c.rank * d <= kDotMost && n * ((c.rank + kUnit - 1) / kUnit) <= kDotUnits;
}
// Entries of a factor that a tile reads once for each adapter among its samples, in a product from d entries to m.
int64_t sort_width(const sfb_adapter_config& c, int64_t n, int64_t m, int64_t d) { return m + (use_dot(c, n, d) ? 0 : d); }
// Whether n samples, each with an adapter at random, had better be taken in the order of their adapters (see adapter_index_kernel), and would
// read 32 MB less of factors, 5 us, which is what finding out takes.
bool sort_may_pay(const sfb_adapter_config& c, int64_t n, int64_t m, int64_t d) {
  const int64_t tiles = (n + kRankTile - 1) / kRankTile, rank16 = (c.rank + kSlice - 1) / kSlice * kSlice;
  const int64_t fewer = tiles * std::min<int64_t>(c.adapters, kRankTile) - tiles - c.adapters, less = fewer * rank16 * sort_width(c, n, m, d);
  return n > kFewMost && less > 2 * n * d && less > 16 << 20;
}

bool pitch_odd(int64_t pitch) { return pitch % 16 != 0; }      // of bf16 entries: not a multiple of 32 bytes

struct AdapterLayout {
  size_t status, ready, arrived, tally, sorted, s, t, ssum, tsum, pb, swords, twords, order, sorted_ids, begin, count, position, work, gparts, lists,
      place, partial, wcopy, zcopy, total;
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
  const size_t n = static_cast<size_t>(c.max_samples), rp = (static_cast<size_t>(c.rank) + 15) / 16 * 16;
  L.status = take(4);
  L.ready = take(kModelSms * kEpi * 4);              // these are cleared with the status word
  L.arrived = take(kFewChunks * 4);
  L.tally = take(3 * 4);
  L.sorted = take(4);
  L.s = take(static_cast<size_t>(rank_rows(c.max_samples, c.cols)) * c.rank * 4);
  L.t = take(static_cast<size_t>(rank_rows(c.max_samples, c.rows)) * c.rank * 4);
  L.ssum = take(n * c.rank * 4);
  L.tsum = take(n * c.rank * 4);
  L.pb = take(n * ((static_cast<size_t>(c.rank) + kUnit - 1) / kUnit) * kUnit * 4);
  L.swords = take(n * 3 * rp * 2);
  L.twords = take(n * 3 * rp * 2);
  L.lists = take((n / kMaxTile + 1) * kListPitch * 4);
  L.place = take(n * 4);
  L.partial = take(n > kFewMost ? static_cast<size_t>(kModelSms) * kPartFloats * 4 : 0);
  // copies of operands whose rows, without gaps between them, are an odd multiple of 16 bytes apart (see adapter_copy_kernel)
  const bool odd_w = pitch_odd(c.ldw ? c.ldw : c.cols) && c.max_samples >= kCopyUses;
  const bool odd_x = pitch_odd(round_up(c.cols, 8)) && c.rows >= kCopyUses, odd_y = pitch_odd(round_up(c.rows, 8)) && c.cols >= kCopyUses;
  L.wcopy = take(odd_w ? static_cast<size_t>(c.rows) * round_up(c.cols, BK) * 2 : 0);
  const bool sorts = sort_may_pay(c, c.max_samples, c.rows, c.cols) || sort_may_pay(c, c.max_samples, c.cols, c.rows);
  L.zcopy = take(n <= kFewMost ? 0 : std::max(odd_x || sorts ? n * round_up(c.cols, BK) * 2 : 0, odd_y || sorts ? n * round_up(c.rows, BK) * 2 : 0));
  L.order = take(n * 4);
  L.sorted_ids = take(sorts ? n * 4 : 0);
  L.begin = take(static_cast<size_t>(c.adapters) * 4);
  L.position = take(n * 4);
  const size_t shares = grad_shares(c, c.max_samples);
  L.work = take((static_cast<size_t>(c.adapters) * shares + 1) * 8);
  L.gparts = take((shares - 1) * c.adapters * c.rank * (round_up(c.rows, 4) + round_up(c.cols, 4)) * 4);
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
  int device, last_cuda, max_pairs;
  CUtensorMap mapU, mapV;              // boxes of 64 entries x `boxed_slices` times 16 ranks of an adapter
  CUtensorMap unitU, unitV;            // x `boxed` units of 8 ranks,
  CUtensorMap fewU, fewV;              // `boxed_few` of them
  int32_t boxed, boxed_few, boxed_slices;
  sfb::EncodeTiledFn encode;           // cuTensorMapEncodeTiled

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

// A matrix [outer x inner], boxes with the 128-byte swizzle.  Operands that are streamed once are asked for 256 bytes at a time (64 samples,
// 10,000 x 20,000: 71.2 us, 73.8 with boxes alone; 325,000 x 10,000: 1,025 and 1,056), those that tiles share in L2 by boxes alone (1,024 samples,
// 10,000 x 20,000: 390 us, 442 with 256 bytes; 8,192, 10,000 x 5,000, whose operands are copied: 790 and 795).
bool operand_map(sfb_adapters* h, CUtensorMap* m, const void* base, int64_t inner, int64_t outer, int64_t pitch, int box_inner, int box_outer,
                 CUtensorMapL2promotion promotion) {
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(outer)}, strides[1] = {static_cast<cuuint64_t>(pitch) * 2};
  cuuint32_t box[2] = {static_cast<cuuint32_t>(box_inner), static_cast<cuuint32_t>(box_outer)}, estr[2] = {1, 1};
  return h->encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool factor_map(sfb_adapters* h, CUtensorMap* m, const void* base, int64_t width, int64_t pitch, int ranks) {
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(h->cfg.rank), static_cast<cuuint64_t>(h->cfg.adapters)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(pitch) * 2, static_cast<cuuint64_t>(pitch) * 2 * h->cfg.rank};
  cuuint32_t box[3] = {BK, static_cast<cuuint32_t>(ranks), 1}, estr[3] = {1, 1, 1};
  return h->encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// allow_smem for a kernel that runs beside another one: the SM's memory as shared memory from the start (as much as the first of the two
// asks for by itself would keep the second one out until it is done).
template <auto Kernel>
cudaError_t allow_beside(int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(Kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (e == cudaSuccess) e = allow_smem<Kernel>(bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// The samples' operand: as it is, or a copy whose rows lie better; and in the order of their adapters, where sort.on() says so.
struct Samples {
  const void* given;
  int64_t given_pitch;
  const void* at;
  int64_t pitch;
  const void* in_order;
  int64_t pitch_in_order;
  Sorting sort;
};

SumParams sum_params(const sfb_adapters* h, int64_t n, const Sorting& sort, const int32_t* ids, float* out, const WordsParams& words) {
  SumParams p{};
  p.ids = ids; p.sort = sort; p.scale = h->scale; p.n = n; p.rank = h->cfg.rank; p.adapters = h->cfg.adapters; p.out = out;
  p.status = h->at<uint32_t>(h->lay.status);
  p.pb = h->at<__nv_bfloat16>(h->lay.pb);
  p.tn = tile_of(n); p.tiles = static_cast<int32_t>((n + p.tn - 1) / p.tn); p.lists = h->at<int32_t>(h->lay.lists); p.place = h->at<int32_t>(h->lay.place);
  p.words = words;
  return p;
}

// p = F[a] z for n samples.  *got: where, and in how many parts.  *all: it is in `sum` in one part, with all that a product with the other
// factors (MN: with V) takes, and the words that are wanted.  So it is up to 64 samples, but for the words; for more adapter_sum_kernel has to
// follow.
template <bool MN>
cudaError_t rank_products(sfb_adapters* h, int64_t n, const Samples& z, const int32_t* ids, float* out, float* sum, const WordsParams& words, Ranked* got,
                          bool* all) {
  const sfb_adapter_config& c = h->cfg;
  const int64_t d = MN ? c.rows : c.cols;
  const int tn = rank_tile(n), parts = rank_parts(n, d), tiles = static_cast<int>((n + tn - 1) / tn);
  *all = use_dot(c, n, d);
  if (*all) {
    *got = Ranked{sum, 1, 0};
    DotParams p{};
    p.s = sum_params(h, n, z.sort, ids, sum, words);
    p.F = static_cast<const __nv_bfloat16*>(MN ? h->U : h->V); p.Z = static_cast<const __nv_bfloat16*>(z.given);
    p.ldf = MN ? c.ldu : c.ldv; p.ldz = z.given_pitch; p.d = static_cast<int32_t>(d);
    const int64_t blocks = n * ((c.rank + kUnit - 1) / kUnit) * (kUnit / kDotRanks) + p.s.tiles + (words.out[0] || words.out[1] ? 1 : 0);
    return launch_kernel(adapter_dot_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, h->stream, 1, p);
  }
  const CUtensorMap& mf = MN ? h->mapU : h->mapV;
  CUtensorMap mz, ms;
  if (!operand_map(h, &mz, z.at, d, n, z.pitch, BK, tn, CU_TENSOR_MAP_L2_PROMOTION_L2_256B) ||
      (z.in_order != z.at && !operand_map(h, &ms, z.in_order, d, n, z.pitch_in_order, BK, tn, CU_TENSOR_MAP_L2_PROMOTION_L2_256B)))
    return cudaErrorInvalidValue;
  if (z.in_order == z.at) ms = mz;
  RankParams p{};
  p.sort = z.sort;
  p.n = static_cast<int32_t>(n); p.tn = tn; p.kseg = static_cast<int32_t>((d + BK - 1) / BK);
  p.stages = std::min(kMaxStages, (n <= kFewMost ? kFewRing : kSmallRing) / stage_bytes(tn));
  p.rank = c.rank; p.adapters = c.adapters; p.boxed = h->boxed_slices; p.ids = ids; p.out = out; p.status = h->at<uint32_t>(h->lay.status);
  const int chunks = rank_chunks(c, n);
  const int smem = p.stages * stage_bytes(tn) + 1024;
  if (n <= kFewMost) {
    p.scale = h->scale; p.p = sum; p.pb = h->at<__nv_bfloat16>(h->lay.pb);
    p.lists = h->at<int32_t>(h->lay.lists); p.place = h->at<int32_t>(h->lay.place); p.arrived = h->at<uint32_t>(h->lay.arrived);
    const cudaError_t e = allow_beside<adapter_rank_kernel<true>>(kFewRing + 1024);
    if (e != cudaSuccess) return e;
    *got = Ranked{sum, 1, 0};
    return launch_kernel(adapter_rank_kernel<true>, dim3(few_rank_blocks(c, n, d)), dim3(kRankThreads), smem, h->stream, 1, mf, mz, ms, p);
  }
  const int groups = std::max(1, std::min(chunks, 2 * kModelSms / (parts * tiles)));
  const cudaError_t e = allow_smem<adapter_rank_kernel<false>>(kSmallRing + 1024);
  if (e != cudaSuccess) return e;
  *got = Ranked{out, parts, n * c.rank};
  return launch_kernel(adapter_rank_kernel<false>, dim3(parts, tiles, groups), dim3(kRankThreads), smem, h->stream, 1, mf, mz, ms, p);
}

// CTAs of a cluster of adapter_few_kernel, each with four k-blocks at least: up to four as long as nine tenths of the places, two an SM,
// hold them all, more only where every CTA has an SM of its own.  (us with one sample: 10,000 x 20,000, 79 tiles, 1 CTA 75, 3 CTAs 64; 5,000 x
// 10,000, 40 tiles, 3 CTAs 22.6, 6 CTAs 25.5; 18,944 x 10,000, 148 tiles, 1 CTA 61, 2 CTAs 65.)
int few_parts(int64_t tiles, int64_t kseg) {
  int best = 1;
  for (int s = 2; s <= kMaxCluster; ++s)
    if (tiles * s <= (s <= 4 ? 2 * kModelSms * 9 / 10 : kModelSms) && kseg >= 4 * s) best = s;
  return best;
}

// Copies a bf16 operand [outer x inner] to workspace, with round_up(inner, BK) entries from row to row.
cudaError_t copy_operand(sfb_adapters* h, const void* from, int64_t pitch, int64_t outer, int64_t inner, size_t room, const Sorting& sort, bool if_sorted) {
  return launch_kernel(adapter_copy_kernel, dim3(grid1d(outer * ((inner + 7) / 8), 1024)), dim3(256), 0, h->stream, 1, static_cast<const uint4*>(from),
                       pitch / 8, h->at<uint4>(room), round_up(inner, BK) / 8, outer, (inner + 7) / 8, sort, if_sorted);
}
bool fits(int64_t outer, int64_t inner, size_t bytes) { return bytes >= static_cast<size_t>(outer) * round_up(inner, BK) * 2; }

// Z [n x d] where the products take it.
cudaError_t placed(sfb_adapters* h, int64_t n, const void* Z, int64_t ldz, int64_t d, int64_t uses, const Sorting& sort, Samples* z) {
  const size_t room = h->lay.order - h->lay.zcopy;
  const bool copy = n > kFewMost && pitch_odd(ldz) && uses >= kCopyUses && fits(n, d, room);
  *z = Samples{Z, ldz, Z, ldz, Z, ldz, sort};
  if (!copy && !sort.sorted) return cudaSuccess;
  z->in_order = h->at<char>(h->lay.zcopy);
  z->pitch_in_order = round_up(d, BK);
  if (copy) { z->at = z->in_order; z->pitch = z->pitch_in_order; }
  return copy_operand(h, Z, ldz, n, d, h->lay.zcopy, sort, !copy);
}

// What adapter_rank_kernel or adapter_sum_kernel leaves for the products.
template <bool MN>
Term term_of(const sfb_adapters* h, const int32_t* ids, const float* p) {
  const sfb_adapter_config& c = h->cfg;
  return Term{c.rank, c.adapters, h->boxed, ids, h->at<int32_t>(h->lay.lists), h->at<int32_t>(h->lay.place), h->scale,
              static_cast<const __nv_bfloat16*>(MN ? h->V : h->U), MN ? c.ldv : c.ldu, p, h->at<uint4>(h->lay.pb)};
}

template <int TN, bool MN>
cudaError_t few(sfb_adapters* h, int64_t n, const void* Z, int64_t ldz, const Term& term, void* Y, int64_t ldy) {
  const sfb_adapter_config& c = h->cfg;
  const int64_t m = MN ? c.cols : c.rows, d = MN ? c.rows : c.cols;
  CUtensorMap ma, mz;
  if (!operand_map(h, &ma, h->W, c.cols, c.rows, c.ldw, BK, MN ? BK : BM, CU_TENSOR_MAP_L2_PROMOTION_L2_256B) ||
      !operand_map(h, &mz, Z, d, n, ldz, BK, TN, CU_TENSOR_MAP_L2_PROMOTION_L2_256B))
    return cudaErrorInvalidValue;
  const CUtensorMap& mf = MN ? h->fewV : h->fewU;
  FewParams p{};
  p.term = term;
  p.term.boxed = h->boxed_few;
  p.n = static_cast<int32_t>(n); p.m = static_cast<int32_t>(m);
  p.kseg = static_cast<int32_t>((d + BK - 1) / BK);
  p.Y = static_cast<__nv_bfloat16*>(Y); p.ldy = ldy; p.status = h->at<uint32_t>(h->lay.status);
  const int64_t tiles = (m + BM - 1) / BM;
  p.parts = few_parts(tiles, p.kseg);
  p.stages = std::min(kMaxStages, kSmallRing / stage_bytes(TN));
  const cudaError_t e = allow_beside<adapter_few_kernel<TN, MN>>(kSmallRing + 1024);
  if (e != cudaSuccess) return e;
  return launch_kernel(adapter_few_kernel<TN, MN>, dim3(static_cast<unsigned>(tiles * p.parts)), dim3(kFewThreads), p.stages * stage_bytes(TN) + 1024,
                       h->stream, p.parts, ma, mz, mf, p);
}

// Cycles of a plan of adapter_pair_kernel: its k-blocks on a pair, 7,000 to start and to end, 9,000 and 2,000 a part to leave and to take
// over parts of tiles.
struct PairPlan { int cut, whole, pairs; };
PairPlan plan_pairs(int64_t tiles, int64_t kseg, int tn, int64_t most) {
  const double per_kb = std::max(2.1 * tn, (BM + tn / 2) * BK * 2 / 60.0), tile = std::max(static_cast<double>(kseg) * per_kb, 8000.0 * tn / kMaxTile);
  const int64_t rounds = (tiles + most - 1) / most, full = tiles / most, whole = std::max<int64_t>(0, full - 1) * most, rest = tiles - whole;
  PairPlan best{0, 0, static_cast<int>(std::min(tiles, most))};
  double cost = static_cast<double>(rounds) * tile + 7000.0;
  const int64_t cap = full > 0 ? most : std::max<int64_t>(1, std::min(most, rest * kseg / 4));
  for (int64_t parts = 2; (full > 0 && parts == 2) || (parts - 1) * rest < cap; ++parts) {
    const int64_t pairs = full > 0 ? most : std::min(cap, parts * rest), shared = (rest * kseg + pairs - 1) / pairs;
    const double c = static_cast<double>(whole / most) * tile + static_cast<double>(shared) * per_kb + 16000.0 + 2000.0 * static_cast<double>(parts);
    if (c < cost && rest % pairs != 0) { cost = c; best = PairPlan{1, static_cast<int>(whole), static_cast<int>(pairs)}; }
  }
  return best;
}

template <bool MN>
cudaError_t pairs(sfb_adapters* h, int64_t n, const Samples& z, const Term& term, void* Y, int64_t ldy) {
  const sfb_adapter_config& c = h->cfg;
  const int64_t m = MN ? c.cols : c.rows, d = MN ? c.rows : c.cols;
  const int tn = tile_of(n);
  const void* W = h->W;
  int64_t ldw = c.ldw;
  if (pitch_odd(ldw) && n >= kCopyUses && fits(c.rows, c.cols, h->lay.zcopy - h->lay.wcopy)) {
    const cudaError_t e = copy_operand(h, W, ldw, c.rows, c.cols, h->lay.wcopy, Sorting{}, false);
    if (e != cudaSuccess) return e;
    W = h->at<char>(h->lay.wcopy);
    ldw = round_up(c.cols, BK);
  }
  CUtensorMap ma, mz, ms;
  if (!operand_map(h, &ma, W, c.cols, c.rows, ldw, BK, MN ? BK : BM, CU_TENSOR_MAP_L2_PROMOTION_NONE) ||
      !operand_map(h, &mz, z.at, d, n, z.pitch, BK, tn / 2, CU_TENSOR_MAP_L2_PROMOTION_NONE) ||
      (z.in_order != z.at && !operand_map(h, &ms, z.in_order, d, n, z.pitch_in_order, BK, tn / 2, CU_TENSOR_MAP_L2_PROMOTION_NONE)))
    return cudaErrorInvalidValue;
  if (z.in_order == z.at) ms = mz;
  PairParams p{};
  p.sort = z.sort;
  p.n = static_cast<int32_t>(n); p.tn = tn; p.tilesT = static_cast<int32_t>((n + tn - 1) / tn);
  p.tilesM = static_cast<int32_t>((m + 2 * BM - 1) / (2 * BM)); p.m = static_cast<int32_t>(m);
  p.kseg = static_cast<int32_t>((d + BK - 1) / BK);
  const PairPlan plan = plan_pairs(static_cast<int64_t>(p.tilesT) * p.tilesM, p.kseg, tn, h->max_pairs);
  p.cut = plan.cut; p.whole = plan.whole;
  p.term = term; p.Y = static_cast<__nv_bfloat16*>(Y); p.ldy = ldy;
  p.partial = h->at<float>(h->lay.partial); p.ready = h->at<uint32_t>(h->lay.ready); p.status = h->at<uint32_t>(h->lay.status);
  return launch_kernel_if(static_cast<int64_t>(p.tilesT) * p.tilesM <= plan.pairs, adapter_pair_kernel<MN>, dim3(2u * static_cast<unsigned>(plan.pairs)),
                          dim3(kPairThreads), kPairSmem, h->stream, 1, ma, mz, ms, MN ? h->unitV : h->unitU, p);
}

// y = A z + scale F^T p.  Unless all is there already, p of more than 64 samples goes from its parts to `to` first, and to the words that are
// wanted; *s: p where it is afterwards.
template <bool MN>
cudaError_t product(sfb_adapters* h, int64_t n, const Samples& z, const int32_t* ids, bool all, Ranked* s, float* to, void* Y, int64_t ldy,
                    const WordsParams& words) {
  const sfb_adapter_config& c = h->cfg;
  if (n <= kFewMost) {
    const Term term = term_of<MN>(h, ids, s->at);
    return n <= 16 ? few<16, MN>(h, n, z.at, z.pitch, term, Y, ldy) : n <= 32 ? few<32, MN>(h, n, z.at, z.pitch, term, Y, ldy)
                                                                             : few<kFewMost, MN>(h, n, z.at, z.pitch, term, Y, ldy);
  }
  if (!all) {
    SumParams p = sum_params(h, n, z.sort, ids, to, words);
    p.p = *s;
    const cudaError_t e = launch_kernel(adapter_sum_kernel, dim3(p.tiles + (words.out[0] || words.out[1] ? 1 : 0) + grid1d(n * ((c.rank + kUnit - 1) / kUnit), 64)),
                                        dim3(256), 0, h->stream, 1, p);
    if (e != cudaSuccess) return e;
    *s = Ranked{to, 1, 0};
  }
  return pairs<MN>(h, n, z, term_of<MN>(h, ids, to), Y, ldy);
}

// The samples by adapters.  sort (may be null): also finds out whether the products, from d entries to m, had better take them so.
cudaError_t index_samples(sfb_adapters* h, int64_t n, const int32_t* ids, int64_t m, int64_t d, Sorting* sort) {
  const AdapterLayout& l = h->lay;
  const sfb_adapter_config& c = h->cfg;
  IndexParams p{};
  p.ids = ids; p.n = static_cast<int32_t>(n); p.adapters = c.adapters; p.rank16 = (c.rank + kSlice - 1) / kSlice * kSlice;
  p.order = h->at<int32_t>(l.order); p.begin = h->at<int32_t>(l.begin); p.count = h->at<int32_t>(l.count); p.position = h->at<int32_t>(l.position); p.sorted_ids = h->at<int32_t>(l.sorted_ids);
  p.tally = h->at<uint32_t>(l.tally); p.sorted = h->at<uint32_t>(l.sorted); p.status = h->at<uint32_t>(l.status);
  if (sort) {
    p.tiles = static_cast<int32_t>((n + kRankTile - 1) / kRankTile);
    p.width = sort_width(c, n, m, d); p.d = d;
    *sort = Sorting{p.sorted, p.order, p.sorted_ids};
  }
  return launch_kernel(adapter_index_kernel, dim3(c.adapters + 1 + p.tiles), dim3(n <= 2048 ? 256 : 32 * kIndexWarps), 0, h->stream, 1, p);
}
// ... whether there is room for that too.
bool sorts(const sfb_adapter_config& c, const AdapterLayout& lay, int64_t n, int64_t m, int64_t d) {
  return sort_may_pay(c, n, m, d) && lay.begin > lay.sorted_ids && fits(n, d, lay.order - lay.zcopy);
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

extern "C" int sfb_adapter_get_plan(const sfb_adapter_config* cfg, int64_t samples, int32_t backward, int32_t* factors, int32_t* factor_blocks,
                                    int32_t* in_order, int32_t* share_blocks) {
  const int rc = check(cfg);
  if (rc) return rc;
  if (samples < 0 || !factors || !factor_blocks || !in_order || !share_blocks) return SFB_ERR_ARG;
  if (samples > cfg->max_samples) return SFB_ERR_SHAPE;
  const sfb_adapter_config& c = *cfg;
  const int64_t d = backward ? c.rows : c.cols, m = backward ? c.cols : c.rows;
  const int kseg = static_cast<int>((d + BK - 1) / BK);
  *factors = use_dot(c, samples, d) ? 0 : 1;
  *factor_blocks = 0;
  if (*factors) {
    const int parts = samples <= kFewMost ? few_rank_parts(few_rank_blocks(c, samples, d), rank_chunks(c, samples), kseg) : rank_parts(samples, d);
    *factor_blocks = (kseg + parts - 1) / parts;
  }
  *in_order = sorts(c, layout_of(c), samples, m, d) ? 1 : 0;
  const int64_t blocks = (samples + BK - 1) / BK;
  *share_blocks = backward ? static_cast<int32_t>((blocks + grad_shares(c, samples) - 1) / grad_shares(c, samples)) : 0;
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
  if (!h) return SFB_ERR_ARG;
  h->encode = reinterpret_cast<EncodeTiledFn>(fn);
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
  h->max_pairs = std::min(sm_count(), kModelSms) / 2;
  h->boxed = h->boxed_slices = 1;
  while (h->boxed_slices < 8 && (c.rank + kSlice - 1) / kSlice % (2 * h->boxed_slices) == 0) h->boxed_slices *= 2;
  while (h->boxed < kPairUnits && (c.rank + kUnit - 1) / kUnit % (2 * h->boxed) == 0) h->boxed *= 2;
  h->boxed_few = std::min(h->boxed, kFewUnits);
  if (!factor_map(h, &h->mapU, U_dev, c.rows, c.ldu, kSlice * h->boxed_slices) || !factor_map(h, &h->mapV, V_dev, c.cols, c.ldv, kSlice * h->boxed_slices) ||
      !factor_map(h, &h->unitU, U_dev, c.rows, c.ldu, kUnit * h->boxed) || !factor_map(h, &h->unitV, V_dev, c.cols, c.ldv, kUnit * h->boxed) ||
      !factor_map(h, &h->fewU, U_dev, c.rows, c.ldu, kUnit * h->boxed_few) || !factor_map(h, &h->fewV, V_dev, c.cols, c.ldv, kUnit * h->boxed_few) ||
      prepare_pair_kernel(adapter_pair_kernel<false>, kPairThreads, kPairSmem, &h->max_pairs) != cudaSuccess ||
      prepare_pair_kernel(adapter_pair_kernel<true>, kPairThreads, kPairSmem, &h->max_pairs) != cudaSuccess || h->max_pairs < 1 ||
      cudaMemsetAsync(h->ws + lay.status, 0, lay.s - lay.status, h->stream) != cudaSuccess) {
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
  float* sum = S_dev ? S_dev : h->at<float>(h->lay.ssum);
  Sorting sort{};
  Samples z;
  if (sorts(c, h->lay, n, c.rows, c.cols)) ACK(index_samples(h, n, ids_dev, c.rows, c.cols, &sort));
  ACK(placed(h, n, X_dev, ldx, c.cols, c.rows, sort, &z));
  bool all;
  ACK(rank_products<false>(h, n, z, ids_dev, h->at<float>(h->lay.s), sum, WordsParams{}, &s, &all));
  ACK(product<false>(h, n, z, ids_dev, all, &s, sum, Y_dev, ldy, WordsParams{}));
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
  Sorting sort{};
  const bool sorting = dX_dev && sorts(c, h->lay, n, c.cols, c.rows);
  if (dU_dev || dV_dev || sorting) ACK(index_samples(h, n, ids_dev, c.cols, c.rows, sorting ? &sort : nullptr));
  Ranked s{S_dev, 1, 0}, t{};
  bool all = false;
  Samples z{X_dev, ldx, X_dev, ldx, X_dev, ldx, Sorting{}};
  if (dU_dev && !S_dev) ACK(rank_products<false>(h, n, z, ids_dev, h->at<float>(h->lay.s), h->at<float>(h->lay.ssum), WordsParams{}, &s, &all));
  WordsParams w{};
  w.out[0] = dU_dev ? h->at<__nv_bfloat16>(h->lay.swords) : nullptr; w.out[1] = dV_dev ? h->at<__nv_bfloat16>(h->lay.twords) : nullptr;
  w.p[0] = s;
  w.ids = ids_dev; w.order = order; w.begin = begin; w.count = count; w.position = h->at<int32_t>(h->lay.position);
  w.work = h->at<int64_t>(h->lay.work); w.scale = h->scale; w.rank = c.rank; w.adapters = c.adapters;
  w.shares = grad_shares(c, n);
  all = false;
  z = Samples{dY_dev, lddy, dY_dev, lddy, dY_dev, lddy, Sorting{}};
  if (dX_dev) ACK(placed(h, n, dY_dev, lddy, c.rows, c.cols, sort, &z));
  if (dX_dev || dV_dev) ACK(rank_products<true>(h, n, z, ids_dev, h->at<float>(h->lay.t), h->at<float>(h->lay.tsum), w, &t, &all));
  if (dX_dev) ACK(product<true>(h, n, z, ids_dev, all, &t, h->at<float>(h->lay.tsum), dX_dev, lddx, w));
  if (dU_dev || dV_dev) {
    if (!all && (!dX_dev || n <= kFewMost)) {
      w.p[1] = t;
      ACK(launch_kernel(adapter_words_kernel, dim3(grid1d(n * ((c.rank + 15) / 16 * 2), 256), 3), dim3(256), 0, h->stream, 1, w));
    }
    GradParams p{};
    const int tile = grad_halves(c.rank) * BM;
    const int64_t pairs_all = static_cast<int64_t>(c.adapters) * c.rank, others = (w.shares - 1) * pairs_all;
    float* more = h->at<float>(h->lay.gparts);
    if (dU_dev)
      p.side[0] = GradSide{static_cast<const __nv_bfloat16*>(dY_dev), lddy, static_cast<int32_t>(c.rows), static_cast<int32_t>((c.rows + tile - 1) / tile), w.out[0], dU_dev, more};
    if (dV_dev)
      p.side[1] = GradSide{static_cast<const __nv_bfloat16*>(X_dev), ldx, static_cast<int32_t>(c.cols), static_cast<int32_t>((c.cols + tile - 1) / tile), w.out[1], dV_dev, more + others * round_up(c.rows, 4)};
    p.rank = c.rank; p.adapters = c.adapters; p.shares = w.shares; p.order = order; p.begin = begin; p.count = count; p.work = w.work; p.status = status;
    const int64_t items = (static_cast<int64_t>(p.side[0].tiles) + p.side[1].tiles) * c.adapters * w.shares;
    const int stage = grad_stage(c.rank);
    const int blocks = grad_blocks(c.rank);
    p.stages = std::min(kGradStages, kGradRing / blocks / stage);
    const int smem = p.stages * stage + 1024;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(items, blocks * sm_count())));
    if (blocks == 2) {
      ACK(allow_beside<adapter_gradient_kernel<2>>(kGradRing / 2 + 1024));
      ACK(launch_kernel(adapter_gradient_kernel<2>, grid, dim3(kGradThreads), smem, h->stream, 1, p));
    } else {
      ACK(allow_smem<adapter_gradient_kernel<1>>(kGradRing + 1024));
      ACK(launch_kernel(adapter_gradient_kernel<1>, grid, dim3(kGradThreads), smem, h->stream, 1, p));
    }
    for (const GradSide& sd : p.side)
      if (sd.tiles && w.shares > 1)
        ACK(launch_kernel(adapter_join_kernel, dim3(grid1d(pairs_all * sd.width / 4 + 1, 256)), dim3(256), 0, h->stream, 1, sd.out,
                          static_cast<const float*>(sd.more), pairs_all * sd.width, w.shares));
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
  if (*status_out & SFB_STATUS_TIMEOUT) ACK(cudaMemsetAsync(h->ws + h->lay.ready, 0, h->lay.s - h->lay.ready, h->stream));
  return SFB_OK;
}

extern "C" int sfb_adapter_last_cuda_error(sfb_adapters* h) { return h ? h->last_cuda : 0; }

extern "C" int sfb_adapter_destroy(sfb_adapters* h) {
  if (!h) return SFB_ERR_ARG;
  delete h;
  return SFB_OK;
}

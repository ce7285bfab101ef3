// Samples from token ids, the gradient of that with respect to the table, and dropout (sfb_embed_*, sfb_dropout_* in sfb.h).
//
//   lookup, dropout   embed_rows_kernel, dropout_kernel: a thread takes groups of eight entries of the output rows
//   gradient          dE[t] = alpha s sum_{i: id_i = t} m_i dX_i:
//     sort_kernel     the samples in the order of their tokens (stable: a token's samples stay in their order); meanwhile other SMs zero dE
//                     (where it is written whole)
//     gradient_kernel chunks of that order, whichever tokens they hold: a thread adds the samples of a chunk for a group of columns and
//                     writes the sum where the token changes.  Work is even however often a token comes up.  A token that goes beyond
//                     a chunk leaves a part in each.
//     join_kernel     adds the parts of such tokens in their order
//   or, for few samples, gradient_few_kernel alone
// Sums are in fp32, in an order that depends on the ids alone: the same bits from call to call.
// All are to be bound by HBM: the rows read once, the table's rows written once.  What each has reached of that stands beside it.
#include <algorithm>
#include <cmath>
#include <new>

#include "sfb_elem.cuh"
#include "sfb_ptx.cuh"

namespace {

using sfb::DropParams;
using sfb::Divisor;
using sfb::Generator;
using sfb::groups_of;
using sfb::kGroup;
using sfb::pdl_launch_dependents;
using sfb::pdl_wait;
using sfb::Raw;

// A matrix of groups, cut into pieces of kThreads * N of them, of which a thread takes N, kThreads apart.
constexpr int kThreads = 256;
struct Grid {
  Divisor groups;                      // of a row
  uint32_t rows, tail;                 // tail: entries of a row's last group
  __device__ __forceinline__ int count(uint32_t group) const { return group + 1 < groups.d ? kGroup : static_cast<int>(tail); }
};
struct Place { uint32_t row, group; };
// The first place of a piece (a division of 64 bits where there are that many), and others by their distance from it.
template <int N>
__device__ __forceinline__ Place first_place(const Grid& g, int64_t piece) {
  const uint64_t first = static_cast<uint64_t>(piece) * (kThreads * N);
  const uint32_t row = first < 0x7fffffffull ? g.groups(static_cast<uint32_t>(first)) : static_cast<uint32_t>(first / g.groups.d);
  return Place{row, static_cast<uint32_t>(first - static_cast<uint64_t>(row) * g.groups.d)};
}
__device__ __forceinline__ Place place_at(const Grid& g, const Place& first, int k) {
  const uint32_t n = first.group + threadIdx.x + k * kThreads, q = g.groups(n);
  return Place{first.row + q, n - q * g.groups.d};
}
// A matrix of rows `pitch` bytes apart.
template <typename T>
__device__ __forceinline__ T* address(void* base, uint32_t pitch, const Place& at) {
  return reinterpret_cast<T*>(static_cast<char*>(base) + static_cast<uint64_t>(at.row) * pitch) + at.group * static_cast<uint64_t>(kGroup);
}
template <typename T>
__device__ __forceinline__ const T* address(const void* base, uint32_t pitch, const Place& at) {
  return address<const T>(const_cast<void*>(base), pitch, at);
}

// ---- lookup ------------------------------------------------------------------------------------------------------------------------
struct RowsParams {
  const void* table;
  void* out;
  const int32_t* ids;
  int64_t pieces;
  Grid grid;
  uint32_t tokens, pitch_in, pitch_out;
  float factor;                        // scale, times the dropout's factor
  bool wide_in, wide_out;
  uint32_t* status;
  DropParams drop;
};

// Blocks take pieces in turn, the ids of the next one under way while one is copied.
// 16,384 samples of 2,000 from 325,000 tokens, fp32 to bf16, with dropout: 32 us for 120 MB (19 at the rate of a plain copy); a row that comes up again is
// read from L2, and it is the loads of 196 MB through it, 64 KB under way an SM at most (four blocks with
// two groups of 32 bytes a thread), and the generator's instructions (half of all issue slots) that take
// the time; without dropout 28 where that is 37 (calls one by one, caches cold).  Rows that are not on 16-byte boundaries go entry by entry: 95 at 2,001
// columns without gaps.  One launch's latency for few samples (2.5 us at 7 of 5,000).
template <typename In, typename Out, bool DROP, int N>
__global__ void __launch_bounds__(kThreads, N == 1 ? 1 : 4) embed_rows_kernel(const __grid_constant__ RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  Generator generator;
  if constexpr (DROP) generator.begin(p.drop);
  Place next[N];
  int32_t id[N];
  auto look = [&](int64_t piece) {
    const Place first = first_place<N>(p.grid, piece);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      next[k] = place_at(p.grid, first, k);
      id[k] = next[k].row < p.grid.rows ? p.ids[next[k].row] : -1;
    }
  };
  look(blockIdx.x);
  for (int64_t piece = blockIdx.x; piece < p.pieces; piece += gridDim.x) {
    Raw<In> raw[N];
    bool named[N];
    Place at[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      at[k] = next[k];
      named[k] = static_cast<uint32_t>(id[k]) < p.tokens;
      if (!named[k] && id[k] != -1 && at[k].group == 0) atomicOr(p.status, SFB_STATUS_INDEX_RANGE);
      if (named[k])
        sfb::load_group(address<In>(p.table, p.pitch_in, Place{static_cast<uint32_t>(id[k]), at[k].group}), p.grid.count(at[k].group), p.wide_in, raw[k]);
    }
    if (N > 1 && piece + gridDim.x < p.pieces) look(piece + gridDim.x);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (at[k].row >= p.grid.rows) break;
      float v[kGroup] = {};
      if (named[k]) {
        sfb::unpack(raw[k], v);
        if constexpr (DROP) generator.drop(v, at[k].row, at[k].group, p.drop.last);
#pragma unroll
        for (int j = 0; j < kGroup; ++j) v[j] *= p.factor;
      }
      Raw<Out> r;
      sfb::pack(v, r);
      sfb::store_group(address<Out>(p.out, p.pitch_out, at[k]), p.grid.count(at[k].group), p.wide_out, r);
    }
  }
}

// ---- dropout -----------------------------------------------------------------------------------------------------------------------
// y = factor x where kept, 0 where not, plus r; y may be x or r.
struct DropoutParams {
  const void *x, *r;
  void* y;
  Grid grid;
  uint32_t pitch_x, pitch_r, pitch_y;
  bool wide;
  DropParams drop;
};

// (One group a thread and 2,048 threads an SM: what takes the time where entries are of 16 bits is the generator, and more threads hide more of it
// than more loads a thread do.  us at 8,192 x 5,000 bf16 with a residual: 47; with two and four groups a thread 53 and 63.)
template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads, 2048 / kThreads) dropout_kernel(const __grid_constant__ DropoutParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const Place at = place_at(p.grid, first_place<1>(p.grid, blockIdx.x), 0);
  const bool there = at.row < p.grid.rows;
  const int count = p.grid.count(at.group);
  Raw<T> raw, more;
  if (there) {
    sfb::load_group(address<T>(p.x, p.pitch_x, at), count, p.wide, raw);
    if constexpr (RESIDUAL) sfb::load_group(address<T>(p.r, p.pitch_r, at), count, p.wide, more);
  }
  Generator generator;
  generator.begin(p.drop);
  if (!there) return;
  float v[kGroup];
  sfb::unpack(raw, v);
  if (p.drop.threshold) generator.drop(v, at.row, at.group, p.drop.last);
  if constexpr (RESIDUAL) {
    float u[kGroup];
    sfb::unpack(more, u);
#pragma unroll
    for (int j = 0; j < kGroup; ++j) v[j] = fmaf(v[j], p.drop.factor, u[j]);
  } else {
#pragma unroll
    for (int j = 0; j < kGroup; ++j) v[j] *= p.drop.factor;
  }
  sfb::pack(v, raw);
  sfb::store_group(address<T>(p.y, p.pitch_y, at), count, p.wide, raw);
}

// ---- the samples in the order of their tokens ----------------------------------------------------------------------------------------
// A radix sort by digits of up to ten bits, least significant first, stable.  Up to kSortMost samples one cluster does it all: a CTA takes
// its share of the samples, a warp a run of them; the lanes of a warp that hold the same digit find one another by a ballot a bit.
// More samples take three launches a digit (counts of tiles, their sums, the move), each tile as a CTA of the cluster does it.
constexpr int kSortThreads = 1024, kSortWarps = 32, kSortPer = 8, kSortTile = kSortThreads * kSortPer;
constexpr int kSortCtas = 16;          // (more than 8: a launch that asks for them)
constexpr int64_t kSortMost = static_cast<int64_t>(kSortThreads) * 4 * kSortCtas;
constexpr int kMaxBits = 10, kMaxBins = 1 << kMaxBits;

struct SortParams {
  const int32_t* ids;                  // of the first digit; the others read `in`
  const uint2* in;                     // (key, sample)
  uint2* out;
  int64_t n;
  uint32_t tokens;                     // a sample that names none of them takes this as its key
  int bits, shift;                     // of the digit
  uint32_t* counts;                    // several launches: [bin][tile]
  uint32_t* totals;                    // ... and [bin]
  int64_t tiles;
  uint32_t* status;
};

struct SortShared {
  uint16_t rank[kSortWarps][kMaxBins]; // of a warp: how many of a digit so far, then how many in the warps before it
  uint32_t total[kMaxBins];            // of the CTA
  uint32_t base[kMaxBins];             // where the CTA's of a digit begin
  uint32_t scan[kSortWarps];
  uint32_t part[kSortThreads];         // of a share of the bins, the CTAs' totals
  uint32_t shares[kSortCtas];          // what the CTAs' shares of the bins hold
};

// Digits of a tile that begins at `first`: key and the rank within the CTA among those of the same digit, of each of a thread's samples.
template <int PER>
__device__ __forceinline__ void rank_tile(SortShared& s, const SortParams& p, int64_t first, uint2 (&e)[PER], uint16_t (&rank)[PER]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << p.bits;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int64_t i = first + warp * (32 * PER) + j * 32 + lane;
    e[j] = make_uint2(0, static_cast<uint32_t>(i));
    if (i >= p.n) continue;
    if (p.ids) {
      const int32_t id = p.ids[i];
      const bool named = id >= 0 && static_cast<uint32_t>(id) < p.tokens;
      if (!named && id != -1) atomicOr(p.status, SFB_STATUS_INDEX_RANGE);
      e[j].x = named ? static_cast<uint32_t>(id) : p.tokens;
    } else {
      e[j] = __ldcg(p.in + i);
    }
  }
  // (its own warp's counts: no other looks at them before the barrier)
  for (int i = lane; i < bins / 2; i += 32) reinterpret_cast<uint32_t*>(s.rank[warp])[i] = 0;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const bool there = first + warp * (32 * PER) + j * 32 + lane < p.n;
    const uint32_t digit = (e[j].x >> p.shift) & (bins - 1);
    uint32_t same = __ballot_sync(0xffffffffu, there);
    if (!same) break;
    for (int b = 0; b < p.bits; ++b) {
      const bool bit = (digit >> b) & 1;
      const uint32_t vote = __ballot_sync(0xffffffffu, bit);
      same &= bit ? vote : ~vote;
    }
    const uint32_t before = there ? s.rank[warp][digit] : 0;
    __syncwarp();
    rank[j] = static_cast<uint16_t>(before + __popc(same & ((1u << lane) - 1)));
    if (there && lane == __ffs(same) - 1) s.rank[warp][digit] = static_cast<uint16_t>(before + __popc(same));
    __syncwarp();
  }
  __syncthreads();
  if (threadIdx.x < bins) {
    uint32_t sum = 0;
#pragma unroll
    for (int w0 = 0; w0 < kSortWarps; w0 += 16) {        // (loads that do not wait for stores)
      uint32_t c[16];
#pragma unroll
      for (int w = 0; w < 16; ++w) c[w] = s.rank[w0 + w][threadIdx.x];
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        s.rank[w0 + w][threadIdx.x] = static_cast<uint16_t>(sum);
        sum += c[w];
      }
    }
    s.total[threadIdx.x] = sum;
  }
}

// The sums of what lies in smaller bins, to base (thread by bin; a value of 0 beyond the bins).
__device__ __forceinline__ uint32_t scan_bins(SortShared& s, uint32_t value) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t sum = value;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) s.scan[warp] = sum;
  __syncthreads();
  uint32_t ahead = 0;
  for (int w = 0; w < warp; ++w) ahead += s.scan[w];
  return ahead + sum - value;
}

template <int PER>
__device__ __forceinline__ void move_tile(const SortShared& s, const SortParams& p, int64_t first, const uint2 (&e)[PER],
                                          const uint16_t (&rank)[PER]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (first + warp * (32 * PER) + j * 32 + lane >= p.n) break;
    const uint32_t digit = (e[j].x >> p.shift) & ((1u << p.bits) - 1);
    __stcg(p.out + s.base[digit] + s.rank[warp][digit] + rank[j], e[j]);
  }
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cluster(const uint32_t* here, int cta) {
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(here))), "r"(cta));
  return there;
}
__device__ __forceinline__ uint32_t cluster_read(const uint32_t* here, int cta) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(in_cluster(here, cta)) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_write(uint32_t* here, int cta, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cluster(here, cta)), "r"(v) : "memory");
}

// Where the sorted samples and what goes with them lie; two buffers that the digits take in turn, the last one writes the first.
struct Order {
  uint2* entries[2];                   // (key, sample)
  uint32_t* crossing;                  // [0]: how many chunks hold the beginning of a token that goes beyond them, then which
};

// Where the CTAs' samples of each digit begin, to their `base`.  A CTA takes a share of the bins: the totals of all CTAs there, added up over CTAs
// and bins; what lies in the shares before it comes to every CTA as one number.
__device__ __forceinline__ void place_digits(SortShared& s, int bits, int ctas, int cta) {
  const int bins = 1 << bits, t = threadIdx.x;
  cluster_sync();                      // every CTA's totals are there
  if (ctas == 1) {
    const uint32_t base = scan_bins(s, t < bins ? s.total[t] : 0);
    if (t < bins) s.base[t] = base;
    __syncthreads();
    return;
  }
  const int share = bins < ctas ? 1 : bins / ctas, first = cta * share, at = t % share, from = t / share;        // bins * ctas threads at most: one each
  const bool mine = from < ctas && first < bins;
  s.part[t] = mine ? cluster_read(&s.total[first + at], from) : 0;
  __syncthreads();
  uint32_t before = 0, all = 0;        // of this bin: in the CTAs before `from`, in all
  if (mine) {
    for (int c = 0; c < ctas; ++c) {
      const uint32_t v = s.part[c * share + at];
      all += v;
      if (c < from) before += v;
    }
  }
  __syncthreads();
  // the share's bins in turn: the threads of the first CTA hold their totals
  const uint32_t ahead = scan_bins(s, t < share && mine ? all : 0);
  if (t < share) s.part[t] = ahead;
  __syncthreads();
  if (mine) cluster_write(&s.base[first + at], from, s.part[at] + before);
  uint32_t whole = 0;
  if (t < kSortWarps) whole = __reduce_add_sync(0xffffffffu, s.scan[t]);
  if (t < ctas) cluster_write(&s.shares[cta], t, first < bins ? whole : 0);
  cluster_sync();
  if (t < bins) {
    uint32_t v = s.base[t];
    for (int c = 0; c < t / share; ++c) v += s.shares[c];
    s.base[t] = v;
  }
  __syncthreads();
}

// dE, all of it: what the rows that samples name cost twice is less than a list of the others (16,384 samples, 50,000 x 2,000: 7 us for 43 MB, 8 for bits
// of the tokens; with 100 tokens the bits took 26, of threads that queue for few words).
struct ZeroParams {
  float* table;
  int64_t ldt, tokens, dim;
  bool wide;
};
// Rows that start on 16-byte boundaries by copies of zeros from shared memory, a row a thread; what lies behind the last 16 bytes, and
// other rows, by stores.  `zeros`: kZeroBytes of shared memory.
constexpr int kZeroBytes = 4096;
template <int THREADS, typename F>
__device__ __forceinline__ void zero_rows(const ZeroParams& p, uint4* zeros, int64_t block, int64_t blocks, F&& wanted) {
  for (int i = threadIdx.x; i < kZeroBytes / 16; i += THREADS) zeros[i] = make_uint4(0, 0, 0, 0);
  sfb::ptx::fence_proxy_async_smem();
  __syncthreads();
  if (p.wide) {
    const int64_t bytes = p.dim / 4 * 16;
    for (int64_t row = static_cast<int64_t>(threadIdx.x) * blocks + block; row < p.tokens; row += blocks * THREADS) {
      if (!wanted(row)) continue;
      float* to = p.table + row * p.ldt;
      for (int64_t at = 0; at < bytes; at += kZeroBytes)
        sfb::ptx::bulk_store(reinterpret_cast<char*>(to) + at, zeros, static_cast<uint32_t>(min(static_cast<int64_t>(kZeroBytes), bytes - at)));
      for (int64_t col = p.dim / 4 * 4; col < p.dim; ++col) to[col] = 0.f;
    }
    sfb::ptx::tma_commit_group();
    sfb::ptx::tma_wait_group<0>();     // (the copies read this block's shared memory)
    return;
  }
  const int lane = threadIdx.x & 31, warps = THREADS / 32;
  for (int64_t row = block * warps + (threadIdx.x >> 5); row < p.tokens; row += blocks * warps)
    if (wanted(row))
      for (int64_t col = lane; col < p.dim; col += 32) p.table[row * p.ldt + col] = 0.f;
}

template <int THREADS>
__device__ __forceinline__ void zero_rows(const ZeroParams& p, uint4* zeros, int64_t block, int64_t blocks) {
  zero_rows<THREADS>(p, zeros, block, blocks, [](int64_t) { return true; });
}

// The first cluster sorts, the others zero.  (65,000 samples, two digits: 25 us, of barriers, ballots and remote reads; nothing of it is HBM's.  Having the
// other CTAs ask L2 for the samples' rows meanwhile made the gradient 2 us faster and the sort 3 us slower.)
template <int PER>
__global__ void __launch_bounds__(kSortThreads, 1) sort_kernel(SortParams p, const __grid_constant__ Order o, const __grid_constant__ ZeroParams zero, int digits, int ctas) {
  extern __shared__ __align__(128) unsigned char shared[];
  SortShared& s = *reinterpret_cast<SortShared*>(shared);
  pdl_launch_dependents();
  pdl_wait();
  const int cta = blockIdx.x;
  if (cta >= ctas) {
    zero_rows<kSortThreads>(zero, reinterpret_cast<uint4*>(shared), cta - ctas, gridDim.x - ctas);
    return;
  }
  const int64_t first = static_cast<int64_t>(cta) * (kSortThreads * PER);
  if (cta == 0 && threadIdx.x == 0) o.crossing[0] = 0;
  uint2 e[PER];
  uint16_t rank[PER];
  for (int d = 0; d < digits; ++d) {
    const int to = (digits - 1 - d) & 1;
    p.out = o.entries[to];
    p.shift = d * p.bits;
    rank_tile<PER>(s, p, first, e, rank);
    place_digits(s, p.bits, ctas, cta);
    move_tile<PER>(s, p, first, e, rank);
    cluster_sync();                    // the order is written, the places are read
    p.ids = nullptr;
    p.in = o.entries[to];
  }
}

__global__ void __launch_bounds__(256) zero_kernel(const __grid_constant__ ZeroParams p) {
  __shared__ __align__(128) uint4 zeros[kZeroBytes / 16];
  pdl_launch_dependents();
  pdl_wait();
  zero_rows<256>(p, zeros, blockIdx.x, gridDim.x);
}

// The same for more samples, a launch each.
__global__ void __launch_bounds__(kSortThreads, 1) sort_count_kernel(const __grid_constant__ SortParams p, uint32_t* crossing) {
  extern __shared__ __align__(128) unsigned char shared[];
  SortShared& s = *reinterpret_cast<SortShared*>(shared);
  pdl_launch_dependents();
  pdl_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) crossing[0] = 0;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortTile;
  uint2 e[kSortPer];
  uint16_t rank[kSortPer];
  rank_tile<kSortPer>(s, p, first, e, rank);
  if (threadIdx.x < (1 << p.bits)) p.counts[threadIdx.x * p.tiles + blockIdx.x] = s.total[threadIdx.x];
}

// A warp a bin: how many of it lie in the tiles before each, and in all.
__global__ void __launch_bounds__(256) sort_sum_kernel(const __grid_constant__ SortParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int bin = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (bin >= (1 << p.bits)) return;
  uint32_t* c = p.counts + bin * p.tiles;
  uint32_t sum = 0;
  for (int64_t at = 0; at < p.tiles; at += 32) {
    const uint32_t v = at + lane < p.tiles ? c[at + lane] : 0;
    uint32_t upto = v;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
      const uint32_t u = __shfl_up_sync(0xffffffffu, upto, k);
      if (lane >= k) upto += u;
    }
    if (at + lane < p.tiles) c[at + lane] = sum + upto - v;
    sum += __shfl_sync(0xffffffffu, upto, 31);
  }
  if (lane == 0) p.totals[bin] = sum;
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_move_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ __align__(128) unsigned char shared[];
  SortShared& s = *reinterpret_cast<SortShared*>(shared);
  pdl_launch_dependents();
  pdl_wait();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortTile;
  uint2 e[kSortPer];
  uint16_t rank[kSortPer];
  rank_tile<kSortPer>(s, p, first, e, rank);
  const bool bin = threadIdx.x < (1 << p.bits);
  const uint32_t base = scan_bins(s, bin ? p.totals[threadIdx.x] : 0);
  if (bin) s.base[threadIdx.x] = base + p.counts[threadIdx.x * p.tiles + blockIdx.x];
  __syncthreads();
  move_tile<kSortPer>(s, p, first, e, rank);
}

// ---- the gradient ------------------------------------------------------------------------------------------------------------------
struct GradientParams {
  const uint2* order;                  // (key, sample)
  uint32_t* crossing;
  float* parts;                        // [2 chunks][groups][8]: what a chunk's first token has of an earlier one's, and its last one's
                                       // beginning
  int64_t n;
  int32_t per;                         // samples a chunk
  uint32_t chunks;
  uint32_t tokens;
  Divisor groups;
  const void* dx;
  int64_t lddx, dim;
  bool wide_in, wide_out;
  float* table;
  int64_t lddt;
  float factor;                        // alpha, scale, the dropout's factor
  bool add;
  DropParams drop;
};

// us, caches cold: 16,384 samples bf16 of 2,000 with dropout to 50,000 tokens 30 (66 MB of samples), 65,000 of 1,000 added to 325,000 tokens 65 (130 MB, and
// 167 MB of rows read and written): what is under way are two samples' loads of each of 32 warps an SM, as many as their 64 registers leave room for (22 to
// 26 of them at work on average); more samples ahead took as many warps away as they brought loads.
constexpr int kAhead = 2;          // samples under way a thread

template <typename T, bool DROP, bool ADD>
__global__ void __launch_bounds__(kThreads, 4) gradient_kernel(const __grid_constant__ GradientParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t place = blockIdx.x * kThreads + threadIdx.x, chunk = p.chunks - 1 - p.groups(place), group = place - p.groups(place) * p.groups.d;
  Generator generator;
  if constexpr (DROP) generator.begin(p.drop);
  if (chunk >= p.chunks) return;
  const uint32_t n = static_cast<uint32_t>(p.n), first = chunk * p.per, last = min(n, first + p.per);
  const int64_t col = static_cast<int64_t>(group) * kGroup;
  const int count = static_cast<int>(min(static_cast<int64_t>(kGroup), p.dim - col));
  const T* dx = static_cast<const T*>(p.dx) + col;
  float* table = p.table + col;
  float* parts = p.parts + (2 * static_cast<int64_t>(chunk) * p.groups.d + group) * kGroup;
  auto entry = [&](uint32_t i) { return i < last ? p.order[i] : make_uint2(p.tokens, 0); };
  uint2 next[kAhead];
#pragma unroll
  for (int q = 0; q < kAhead; ++q) next[q] = entry(first + q);
  const uint32_t first_key = next[0].x;
  if (first_key == p.tokens) return;
  // what the chunk's first token has of an earlier chunk's, and whether its last one goes on
  const uint32_t lead_key = first > 0 && p.order[first - 1].x == first_key ? first_key : p.tokens;
  const uint32_t trail_key = last < n ? p.order[last].x : p.tokens;
  float sum[kGroup] = {};
  for (uint32_t i = first; i < last; i += kAhead) {
    uint2 e[kAhead];
    Raw<T> raw[kAhead];
    Raw<float> old[ADD ? kAhead : 1];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      e[q] = next[q];
      if (e[q].x < p.tokens) sfb::load_group(dx + e[q].y * p.lddx, count, p.wide_in, raw[q]);
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) next[q] = entry(i + kAhead + q);
    bool ends[kAhead], whole[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      ends[q] = e[q].x != (q + 1 < kAhead ? e[q + 1].x : next[0].x) && e[q].x < p.tokens;
      whole[q] = ends[q] && e[q].x != lead_key && (e[q].x != trail_key || i + q + 1 < last);
      if constexpr (ADD) {             // (with the samples: nothing waits for a row by itself)
        if (whole[q]) sfb::load_group(table + e[q].x * p.lddt, count, p.wide_out, old[q]);
      }
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if (e[q].x == p.tokens) break;   // nothing follows
      float v[kGroup];
      sfb::unpack(raw[q], v);
      if constexpr (DROP) generator.drop(v, e[q].y, group, p.drop.last);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) sum[j] += v[j];
      if (!ends[q]) continue;
      Raw<float> r;
      float* to = table + e[q].x * p.lddt;
      if (whole[q]) {
        float o[kGroup] = {};
        if constexpr (ADD) sfb::unpack(old[q], o);
#pragma unroll
        for (int j = 0; j < kGroup; ++j) o[j] = fmaf(p.factor, sum[j], o[j]);
        sfb::pack(o, r);
      } else {
        const bool begins = e[q].x != lead_key;
        to = parts + (begins ? static_cast<int64_t>(p.groups.d) * kGroup : 0);
        sfb::pack(sum, r);
        if (begins && group == 0) p.crossing[1 + atomicAdd(p.crossing, 1u)] = chunk;
      }
      sfb::store_group(to, whole[q] ? count : kGroup, p.wide_out || !whole[q], r);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) sum[j] = 0.f;
    }
  }
}

// Up to kFew samples, in one launch: a warp has a sample and 32 groups of columns.  It compares the sample's token with all others; the first
// sample of a token adds them all, in their order.  Other blocks zero rows that are no sample's token.
constexpr int kFew = 256;
template <typename T, bool DROP, bool ADD>
__global__ void __launch_bounds__(kThreads) gradient_few_kernel(const __grid_constant__ GradientParams p, const __grid_constant__ ZeroParams zero, const int32_t* given,
                                                                uint32_t zeros, uint32_t* status) {
  __shared__ __align__(128) uint4 shared[kZeroBytes / 16];
  __shared__ __align__(16) int32_t ids[kFew];
  pdl_launch_dependents();
  pdl_wait();
  const int n = static_cast<int>(p.n), lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kFew; i += kThreads) ids[i] = i < n ? given[i] : -1;
  __syncthreads();
  if (blockIdx.x < zeros) {
    zero_rows<kThreads>(zero, shared, blockIdx.x, zeros, [&](int64_t row) {
      const int4* q = reinterpret_cast<const int4*>(ids);
      const int t = static_cast<int>(row);
      bool found = false;
#pragma unroll 4
      for (int i = 0; i < (n + 3) / 4; ++i) {
        const int4 w = q[i];
        found |= w.x == t || w.y == t || w.z == t || w.w == t;
      }
      return !found;
    });
    return;
  }
  Generator generator;
  if constexpr (DROP) generator.begin(p.drop);
  const uint32_t slabs = (p.groups.d + 31) / 32, item = (blockIdx.x - zeros) * (kThreads / 32) + (threadIdx.x >> 5);
  const int i = static_cast<int>(item / slabs);
  if (i >= n) return;
  const uint32_t slab = item % slabs, group = slab * 32 + lane;
  const int32_t id = ids[i];
  if (static_cast<uint32_t>(id) >= p.tokens) {
    if (id != -1 && slab == 0 && lane == 0) atomicOr(status, SFB_STATUS_INDEX_RANGE);
    return;
  }
  uint32_t same[kFew / 32];
  bool first = true;
#pragma unroll
  for (int b = 0; b < kFew / 32; ++b) {
    same[b] = __ballot_sync(0xffffffffu, ids[b * 32 + lane] == id);
    const uint32_t before = i >= (b + 1) * 32 ? 0xffffffffu : i > b * 32 ? (1u << (i - b * 32)) - 1 : 0;
    first &= !(same[b] & before);
  }
  if (!first) return;
  const int64_t col = static_cast<int64_t>(group) * kGroup;
  const int count = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(kGroup), p.dim - col)));
  float* to = p.table + static_cast<int64_t>(id) * p.lddt + col;
  Raw<float> r{};
  if constexpr (ADD) {
    if (count) sfb::load_group(to, count, p.wide_out, r);
  }
  float sum[kGroup] = {};
  constexpr int kTogether = 4;
  int at[kTogether], have = 0;
  auto take = [&]() {
    Raw<T> raw[kTogether];
#pragma unroll
    for (int q = 0; q < kTogether; ++q)
      if (q < have && count) sfb::load_group(static_cast<const T*>(p.dx) + at[q] * p.lddx + col, count, p.wide_in, raw[q]);
#pragma unroll
    for (int q = 0; q < kTogether; ++q) {
      if (q >= have || !count) break;
      float v[kGroup];
      sfb::unpack(raw[q], v);
      if constexpr (DROP) generator.drop(v, at[q], group, p.drop.last);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) sum[j] += v[j];
    }
    have = 0;
  };
#pragma unroll
  for (int b = 0; b < kFew / 32; ++b) {
#pragma unroll 1
    for (uint32_t left = same[b]; left; left &= left - 1) {
      const int j = b * 32 + __ffs(left) - 1;
#pragma unroll
      for (int q = 0; q < kTogether; ++q)
        if (q == have) at[q] = j;
      if (++have == kTogether) take();
    }
  }
  if (have) take();
  if (!count) return;
  float v[kGroup];
  sfb::unpack(r, v);
#pragma unroll
  for (int j = 0; j < kGroup; ++j) v[j] = fmaf(p.factor, sum[j], v[j]);
  sfb::pack(v, r);
  sfb::store_group(to, count, p.wide_out, r);
}

// Warps take (token, 32 groups) in turn and add the token's parts in their order.  Where there are more than kSerial, the block does so afterwards:
// eight warps add contiguous shares of the parts, the first adds the shares.
constexpr int kSerial = 16;
__device__ __forceinline__ void add_parts(const GradientParams& p, uint32_t chunk, uint32_t group, int64_t from, int64_t to, float (&sum)[kGroup]) {
  for (int64_t k0 = from; k0 < to; k0 += 4) {
    Raw<float> r[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t k = k0 + q, slot = k == 0 ? 2 * static_cast<int64_t>(chunk) + 1 : 2 * (chunk + k);
      if (k < to) sfb::load_group(p.parts + (slot * p.groups.d + group) * kGroup, kGroup, true, r[q]);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (k0 + q >= to) break;
      float v[kGroup];
      sfb::unpack(r[q], v);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) sum[j] += v[j];
    }
  }
}
__device__ __forceinline__ void store_joined(const GradientParams& p, uint32_t key, uint32_t group, const float (&sum)[kGroup]) {
  const int64_t col = static_cast<int64_t>(group) * kGroup;
  const int count = static_cast<int>(min(static_cast<int64_t>(kGroup), p.dim - col));
  float* to = p.table + key * p.lddt + col;
  Raw<float> r{};
  float v[kGroup];
  if (p.add) sfb::load_group(to, count, p.wide_out, r);
  sfb::unpack(r, v);
#pragma unroll
  for (int j = 0; j < kGroup; ++j) v[j] = fmaf(p.factor, sum[j], v[j]);
  sfb::pack(v, r);
  sfb::store_group(to, count, p.wide_out, r);
}

// (Two blocks an SM: with the registers of four, spills took half of the time.  us at 16,384 samples, 50,000 x 2,000: 6; with three and four 8, 11.)
__global__ void __launch_bounds__(256, 2) join_kernel(const __grid_constant__ GradientParams p) {
  __shared__ float shares[8][32][kGroup + 1];
  __shared__ struct { uint32_t chunk, slab, key; int64_t parts; } later[8];
  __shared__ uint32_t left;
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t count = p.crossing[0], slabs = (p.groups.d + 31) / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint64_t items = static_cast<uint64_t>(count) * slabs;
  // (a block's warps far apart in the list, where tokens of many parts may follow one another)
  for (uint64_t first = blockIdx.x; first < items; first += static_cast<uint64_t>(gridDim.x) * 8) {
    if (threadIdx.x == 0) left = 0;
    __syncthreads();
    const uint64_t item = first + static_cast<uint64_t>(warp) * gridDim.x;
    if (item < items) {
      const uint32_t chunk = p.crossing[1 + item / slabs], slab = static_cast<uint32_t>(item % slabs), group = slab * 32 + lane;
      const uint32_t key = p.order[(static_cast<int64_t>(chunk) + 1) * p.per - 1].x;
      int64_t parts = 1;               // the chunk's own, and one of each chunk behind it that begins with this token
      for (int got = 32; got == 32; parts += got) {
        const int64_t at = (chunk + parts + lane) * p.per;
        const uint32_t there = at < p.n ? p.order[at].x : p.tokens;
        got = __popc(__ballot_sync(0xffffffffu, there == key));
      }
      if (parts > kSerial) {
        if (lane == 0) {
          const uint32_t at = atomicAdd(&left, 1u);
          later[at].chunk = chunk, later[at].slab = slab, later[at].key = key, later[at].parts = parts;
        }
      } else if (group < p.groups.d) {
        float sum[kGroup] = {};
        add_parts(p, chunk, group, 0, parts, sum);
        store_joined(p, key, group, sum);
      }
    }
    __syncthreads();
    for (uint32_t q = 0; q < left; ++q) {
      const uint32_t group = later[q].slab * 32 + lane;
      const int64_t parts = later[q].parts, each = (parts + 7) / 8, from = warp * each, to = min(parts, from + each);
      float sum[kGroup] = {};
      if (group < p.groups.d) add_parts(p, later[q].chunk, group, from, to, sum);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) shares[warp][lane][j] = sum[j];
      __syncthreads();
      if (warp == 0 && group < p.groups.d) {
        for (int w = 1; w < 8; ++w)
#pragma unroll
          for (int j = 0; j < kGroup; ++j) sum[j] += shares[w][lane][j];
        store_joined(p, later[q].key, group, sum);
      }
      __syncthreads();
    }
  }
}

}  // namespace

// ---- host --------------------------------------------------------------------------------------------------------------------------
struct sfb_embed {
  sfb_embed_config cfg;
  const void* table;
  char* ws;
  int device;
  int last_cuda;
};

namespace {

using sfb::OnDevice;

template <typename H>
int fail(H* h, cudaError_t e) {
  h->last_cuda = static_cast<int>(e);
  return SFB_ERR_CUDA;
}

constexpr int64_t kPieces = static_cast<int64_t>(sfb::kModelSms) * 1024;
constexpr int kPerLeast = 4, kPerMost = 64;
constexpr int64_t kBlocksMost = (1ll << 31) - 1;

// Of a matrix that the element-wise kernels take: up to 2^31 rows, rows less than 4 GB apart.
bool fits(int64_t n, int64_t pitch, int32_t dtype) { return n < (1ll << 31) && pitch < static_cast<int64_t>((1ull << 32) / sfb::size_of(dtype)); }
Grid grid_of(int64_t n, int64_t cols) {
  const int64_t groups = groups_of(cols);
  return Grid{Divisor(static_cast<uint32_t>(groups)), static_cast<uint32_t>(n), static_cast<uint32_t>(cols - (groups - 1) * kGroup)};
}

// Samples a chunk: one full round of threads, which end together (us at 16,384 samples, 50,000 x 2,000, and at 65,000 added to 325,000 x 1,000, with a join
// of more registers spilled: 110 and 103; with two rounds 114 and 102, four 121 and 109); but no fewer than 4, and no more than 64, where parts are a small share of what is read.
int samples_per_chunk(int64_t n, int64_t groups) {
  const int64_t chunks = std::max<int64_t>(1, kPieces / groups);
  return static_cast<int>(std::max<int64_t>(kPerLeast, std::min<int64_t>(kPerMost, (n + chunks - 1) / chunks)));
}

struct EmbedLayout {
  size_t status, crossing, entries[2], counts, totals, parts, bytes;
  int64_t tiles;
};

EmbedLayout layout_of(const sfb_embed_config& c) {
  EmbedLayout l{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 1023) / 1024 * 1024;
    return at;
  };
  const int64_t n = c.max_ids, groups = groups_of(c.dim);
  l.tiles = (n + kSortTile - 1) / kSortTile;
  l.status = take(16);
  // chunks: the most that any number of samples up to n is cut into, and their parts
  const int64_t chunks = std::max({static_cast<int64_t>(1), (n + kPerMost - 1) / kPerMost, std::min((n + kPerLeast - 1) / kPerLeast, kPieces / groups)});
  l.crossing = take((chunks + 1) * 4);
  for (size_t& e : l.entries) e = take(n * 8);
  l.counts = take(l.tiles * kMaxBins * 4);
  l.totals = take(kMaxBins * 4);
  l.parts = take(static_cast<size_t>(chunks) * 2 * groups * kGroup * 4);
  l.bytes = off;
  return l;
}

int check(const sfb_embed_config* c) {
  if (!c || c->tokens <= 0 || c->dim <= 0 || c->ldt < 0 || c->max_ids < 0 || !std::isfinite(c->scale)) return SFB_ERR_ARG;
  if (!sfb::is_dtype(c->table_dtype) || !sfb::is_dtype(c->out_dtype)) return SFB_ERR_ARG;
  if (c->tokens > (1ll << 30) || c->dim > (1ll << 24) || c->max_ids > (1ll << 26)) return SFB_ERR_SHAPE;
  // (a launch's blocks: groups of columns of chunks of 64 samples are numbered in 31 bits)
  if ((c->max_ids + kPerMost - 1) / kPerMost * groups_of(c->dim) > kBlocksMost - kThreads) return SFB_ERR_SHAPE;
  if ((c->ldt && c->ldt < c->dim) || c->ldt >= (1ll << 32) / static_cast<int64_t>(sfb::size_of(c->table_dtype))) return SFB_ERR_SHAPE;
  return SFB_OK;
}

template <typename In, typename Out, bool DROP>
cudaError_t launch_rows(RowsParams p, cudaStream_t s) {
  const int64_t all = static_cast<int64_t>(p.grid.rows) * p.grid.groups.d;
  // (groups a thread, their loads under way together, once that still is a block for each SM)
  constexpr int N = 2;
  if (all < static_cast<int64_t>(sfb::kModelSms) * kThreads * N) {
    p.pieces = (all + kThreads - 1) / kThreads;
    return sfb::launch_kernel(embed_rows_kernel<In, Out, DROP, 1>, dim3(static_cast<unsigned>(p.pieces)), dim3(kThreads), 0, s, 1, p);
  }
  p.pieces = (all + kThreads * N - 1) / (kThreads * N);
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(p.pieces, sfb::sm_count() * 4));
  return sfb::launch_kernel(embed_rows_kernel<In, Out, DROP, N>, dim3(blocks), dim3(kThreads), 0, s, 1, p);
}
template <typename In, typename Out>
cudaError_t launch_rows(const RowsParams& p, bool drop, cudaStream_t s) {
  return drop ? launch_rows<In, Out, true>(p, s) : launch_rows<In, Out, false>(p, s);
}
template <typename In>
cudaError_t launch_rows(const RowsParams& p, int32_t out, bool drop, cudaStream_t s) {
  if (out == SFB_F32) return launch_rows<In, float>(p, drop, s);
  if (out == SFB_BF16) return launch_rows<In, __nv_bfloat16>(p, drop, s);
  return launch_rows<In, __half>(p, drop, s);
}

template <typename T, bool RESIDUAL>
cudaError_t launch_dropout(const DropoutParams& p, cudaStream_t s) {
  const int64_t all = static_cast<int64_t>(p.grid.rows) * p.grid.groups.d;
  return sfb::launch_kernel(dropout_kernel<T, RESIDUAL>, dim3(static_cast<unsigned>((all + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, 1, p);
}
template <typename T>
cudaError_t launch_dropout(const DropoutParams& p, cudaStream_t s) {
  return p.r ? launch_dropout<T, true>(p, s) : launch_dropout<T, false>(p, s);
}

template <int PER>
cudaError_t launch_sort(const SortParams& p, const Order& o, const ZeroParams& zero, int digits, int ctas, int zeros, cudaStream_t s) {
  cudaError_t e = sfb::allow_smem<sort_kernel<PER>>(sizeof(SortShared));
  if (e == cudaSuccess) e = sfb::allow_clusters<sort_kernel<PER>>();
  return e == cudaSuccess ? sfb::launch_kernel(sort_kernel<PER>, dim3(ctas + zeros), dim3(kSortThreads), sizeof(SortShared), s, ctas, p, o, zero, digits, ctas) : e;
}

cudaError_t sort_samples(const EmbedLayout& l, char* ws, const sfb_embed_config& c, int64_t n, const int32_t* ids, const Order& o, const ZeroParams* zero) {
  int bits = 1;
  while ((1ll << bits) <= c.tokens) ++bits;            // of the keys 0 .. tokens
  const int digits = (bits + kMaxBits - 1) / kMaxBits;
  SortParams p{};
  p.ids = ids;
  p.n = n;
  p.tokens = static_cast<uint32_t>(c.tokens);
  p.bits = (bits + digits - 1) / digits;
  p.status = reinterpret_cast<uint32_t*>(ws + l.status);
  const cudaStream_t s = static_cast<cudaStream_t>(c.stream);
  cudaError_t e = cudaSuccess;
  if (n <= kSortMost) {
    // As many CTAs as there are for the sort; but the fewest where zeroing takes longer than that anyway (100 MB: 16 us), since clusters of few CTAs leave
    // more SMs to it (us at 16,384 samples, 50,000 x 2,000: with 16 CTAs 75, with 4 71).
    const bool few = zero && c.tokens * c.dim * 4 > (100ll << 20);
    const int per = few || n > 2 * kSortThreads * kSortCtas ? 4 : n > kSortThreads * kSortCtas ? 2 : 1;
    int ctas = 1;
    while (static_cast<int64_t>(ctas) * kSortThreads * per < n) ctas *= 2;
    // CTAs that zero, in clusters like the one that sorts: as many as a chip of 148 SMs has room for beside it
    int zeros = 0;
    if (zero) {
      const int room = ctas <= 2 ? 148 : ctas == 4 ? 132 : ctas == 8 ? 120 : 112;
      zeros = static_cast<int>(std::min<int64_t>(room - ctas, (c.tokens + 31) / 32));
      zeros = std::max(1, zeros / ctas) * ctas;
    }
    if (per == 1) return launch_sort<1>(p, o, zero ? *zero : ZeroParams{}, digits, ctas, zeros, s);
    if (per == 2) return launch_sort<2>(p, o, zero ? *zero : ZeroParams{}, digits, ctas, zeros, s);
    return launch_sort<4>(p, o, zero ? *zero : ZeroParams{}, digits, ctas, zeros, s);
  }
  p.tiles = (n + kSortTile - 1) / kSortTile;
  p.counts = reinterpret_cast<uint32_t*>(ws + l.counts);
  p.totals = reinterpret_cast<uint32_t*>(ws + l.totals);
  e = sfb::allow_smem<sort_count_kernel>(sizeof(SortShared));
  if (e == cudaSuccess) e = sfb::allow_smem<sort_move_kernel>(sizeof(SortShared));
  for (int d = 0; d < digits && e == cudaSuccess; ++d) {
    const int to = (digits - 1 - d) & 1;
    p.out = o.entries[to];
    p.shift = d * p.bits;
    const dim3 tiles(static_cast<unsigned>(p.tiles));
    e = sfb::launch_kernel(sort_count_kernel, tiles, dim3(kSortThreads), sizeof(SortShared), s, 1, p, o.crossing);
    if (e == cudaSuccess) e = sfb::launch_kernel(sort_sum_kernel, dim3(((1 << p.bits) + 7) / 8), dim3(256), 0, s, 1, p);
    if (e == cudaSuccess) e = sfb::launch_kernel(sort_move_kernel, tiles, dim3(kSortThreads), sizeof(SortShared), s, 1, p);
    p.ids = nullptr;
    p.in = p.out;
  }
  if (e == cudaSuccess && zero)
    e = sfb::launch_kernel(zero_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((c.tokens + 31) / 32, sfb::sm_count() * 4))), dim3(256), 0, s, 1, *zero);
  return e;
}

template <typename T, bool DROP>
cudaError_t launch_gradient(const GradientParams& p, unsigned blocks, cudaStream_t s) {
  return p.add ? sfb::launch_kernel(gradient_kernel<T, DROP, true>, dim3(blocks), dim3(kThreads), 0, s, 1, p)
               : sfb::launch_kernel(gradient_kernel<T, DROP, false>, dim3(blocks), dim3(kThreads), 0, s, 1, p);
}
template <typename T>
cudaError_t launch_few(const GradientParams& p, const ZeroParams& zero, const int32_t* ids, uint32_t zeros, uint32_t* status, bool drop, unsigned blocks, cudaStream_t s) {
  auto launch = [&](auto kernel) { return sfb::launch_kernel(kernel, dim3(blocks), dim3(kThreads), 0, s, 1, p, zero, ids, zeros, status); };
  if (p.add) return drop ? launch(gradient_few_kernel<T, true, true>) : launch(gradient_few_kernel<T, false, true>);
  return drop ? launch(gradient_few_kernel<T, true, false>) : launch(gradient_few_kernel<T, false, false>);
}
template <typename T>
cudaError_t launch_gradient(const GradientParams& p, bool drop, unsigned blocks, cudaStream_t s) {
  return drop ? launch_gradient<T, true>(p, blocks, s) : launch_gradient<T, false>(p, blocks, s);
}

}  // namespace

extern "C" int sfb_dropout_init(float p, const uint64_t* rng_dev, void* stream, sfb_dropout** out) {
  if (!out) return SFB_ERR_ARG;
  *out = nullptr;
  if (!rng_dev || !(p >= 0.f && p <= 1.f)) return SFB_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(rng_dev) & 7u) return SFB_ERR_ALIGN;
  int dev = 0;
  const int rc = sfb::this_device(&dev);
  if (rc) return rc;
  sfb_dropout* h = new (std::nothrow) sfb_dropout();
  if (!h) return SFB_ERR_ARG;
  h->drop.rng = rng_dev;
  h->drop.threshold = static_cast<uint32_t>(std::nearbyint(static_cast<double>(p) * 65536.0));
  h->drop.last = (h->drop.threshold << 16) - 1;        // (of 65536: all ones)
  h->drop.factor = h->drop.threshold < 65536 ? static_cast<float>(65536.0 / (65536.0 - h->drop.threshold)) : 0.f;
  h->stream = static_cast<cudaStream_t>(stream);
  h->device = dev;
  *out = h;
  return SFB_OK;
}

extern "C" int sfb_dropout_apply(sfb_dropout* h, uint64_t call, int64_t n, int64_t cols, int32_t dtype, const void* X_dev, int64_t ldx,
                                 const void* R_dev, int64_t ldr, void* Y_dev, int64_t ldy) {
  if (!h || n < 0 || cols <= 0 || !sfb::is_dtype(dtype)) return SFB_ERR_ARG;
  if (n == 0) return SFB_OK;
  if (!X_dev || !Y_dev) return SFB_ERR_ARG;
  if (!R_dev) ldr = ldx;
  if (cols > (1ll << 30) || ldx < cols || ldy < cols || ldr < cols) return SFB_ERR_SHAPE;
  if (!fits(n, ldx, dtype) || !fits(n, ldy, dtype) || !fits(n, ldr, dtype)) return SFB_ERR_SHAPE;
  if (!sfb::lies_aligned(X_dev, dtype) || !sfb::lies_aligned(Y_dev, dtype) || !sfb::lies_aligned(R_dev, dtype)) return SFB_ERR_ALIGN;
  const int64_t groups = groups_of(cols);
  if (n > kBlocksMost / groups * kThreads) return SFB_ERR_SHAPE;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  const int64_t size = static_cast<int64_t>(sfb::size_of(dtype));
  DropoutParams p{X_dev, R_dev, Y_dev, grid_of(n, cols), static_cast<uint32_t>(ldx * size), static_cast<uint32_t>(ldr * size), static_cast<uint32_t>(ldy * size), false, h->drop};
  p.wide = sfb::lies_wide(X_dev, ldx, dtype) && sfb::lies_wide(Y_dev, ldy, dtype) && (!R_dev || sfb::lies_wide(R_dev, ldr, dtype));
  p.drop.call = call;
  const cudaError_t e = dtype == SFB_F32 ? launch_dropout<float>(p, h->stream)
                        : dtype == SFB_BF16 ? launch_dropout<__nv_bfloat16>(p, h->stream) : launch_dropout<__half>(p, h->stream);
  return e == cudaSuccess ? SFB_OK : fail(h, e);
}

extern "C" int sfb_dropout_last_cuda_error(sfb_dropout* h) { return h ? h->last_cuda : 0; }

extern "C" int sfb_dropout_destroy(sfb_dropout* h) {
  if (!h) return SFB_ERR_ARG;
  delete h;
  return SFB_OK;
}

extern "C" int sfb_embed_workspace_bytes(const sfb_embed_config* cfg, size_t* out_bytes) {
  if (!out_bytes) return SFB_ERR_ARG;
  const int rc = check(cfg);
  if (rc) return rc;
  *out_bytes = layout_of(*cfg).bytes;
  return SFB_OK;
}

extern "C" int sfb_embed_init(const sfb_embed_config* cfg, const void* table_dev, void* workspace_dev, size_t workspace_bytes, sfb_embed** out) {
  if (!out) return SFB_ERR_ARG;
  *out = nullptr;
  const int rc = check(cfg);
  if (rc) return rc;
  if (!table_dev || !workspace_dev) return SFB_ERR_ARG;
  if (!sfb::lies_aligned(table_dev, cfg->table_dtype) || (reinterpret_cast<uintptr_t>(workspace_dev) & 1023u)) return SFB_ERR_ALIGN;
  if (workspace_bytes < layout_of(*cfg).bytes) return SFB_ERR_WORKSPACE;
  int dev = 0;
  const int on = sfb::this_device(&dev);
  if (on) return on;
  sfb_embed* h = new (std::nothrow) sfb_embed();
  if (!h) return SFB_ERR_ARG;
  h->cfg = *cfg;
  if (!h->cfg.ldt) h->cfg.ldt = cfg->dim;
  h->table = table_dev;
  h->ws = static_cast<char*>(workspace_dev);
  h->device = dev;
  if (cudaMemsetAsync(h->ws, 0, 16, static_cast<cudaStream_t>(cfg->stream)) != cudaSuccess) {
    delete h;
    return SFB_ERR_CUDA;
  }
  *out = h;
  return SFB_OK;
}

extern "C" int sfb_embed_forward(sfb_embed* h, int64_t n, const int32_t* ids_dev, void* X_dev, int64_t ldx, const sfb_dropout* drop, uint64_t call) {
  if (!h || n < 0 || (drop && drop->device != h->device)) return SFB_ERR_ARG;
  const sfb_embed_config& c = h->cfg;
  if (n > c.max_ids) return SFB_ERR_SHAPE;
  if (n == 0) return SFB_OK;
  if (!ids_dev || !X_dev) return SFB_ERR_ARG;
  if (ldx < c.dim) return SFB_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(ids_dev) & 3u) || !sfb::lies_aligned(X_dev, c.out_dtype)) return SFB_ERR_ALIGN;
  if (!fits(n, ldx, c.out_dtype)) return SFB_ERR_SHAPE;
  const bool drops = drop && drop->drop.threshold > 0;
  const float factor = c.scale * (drops ? drop->drop.factor : 1.f);
  if (!std::isfinite(factor)) return SFB_ERR_ARG;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  RowsParams p{};
  p.table = h->table;
  p.out = X_dev;
  p.ids = ids_dev;
  p.grid = grid_of(n, c.dim);
  p.tokens = static_cast<uint32_t>(c.tokens);
  p.pitch_in = static_cast<uint32_t>(c.ldt * static_cast<int64_t>(sfb::size_of(c.table_dtype)));
  p.pitch_out = static_cast<uint32_t>(ldx * static_cast<int64_t>(sfb::size_of(c.out_dtype)));
  p.factor = factor;
  p.wide_in = sfb::lies_wide(h->table, c.ldt, c.table_dtype);
  p.wide_out = sfb::lies_wide(X_dev, ldx, c.out_dtype);
  p.status = reinterpret_cast<uint32_t*>(h->ws);
  if (drops) {
    p.drop = drop->drop;
    p.drop.call = call;
  }
  const cudaStream_t s = static_cast<cudaStream_t>(c.stream);
  const cudaError_t e = c.table_dtype == SFB_F32 ? launch_rows<float>(p, c.out_dtype, drops, s)
                        : c.table_dtype == SFB_BF16 ? launch_rows<__nv_bfloat16>(p, c.out_dtype, drops, s) : launch_rows<__half>(p, c.out_dtype, drops, s);
  return e == cudaSuccess ? SFB_OK : fail(h, e);
}

extern "C" int sfb_embed_backward(sfb_embed* h, int64_t n, const int32_t* ids_dev, const void* dX_dev, int64_t lddx, const sfb_dropout* drop,
                                  uint64_t call, float alpha, int32_t add, float* dE_dev, int64_t ldde) {
  if (!h || n < 0 || (drop && drop->device != h->device) || !dE_dev || !std::isfinite(alpha) || (add != 0 && add != 1)) return SFB_ERR_ARG;
  const sfb_embed_config& c = h->cfg;
  if (n > c.max_ids || ldde < c.dim) return SFB_ERR_SHAPE;
  if (n > 0 && (!ids_dev || !dX_dev)) return SFB_ERR_ARG;
  if (n > 0 && lddx < c.dim) return SFB_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(ids_dev) & 3u) || !sfb::lies_aligned(dX_dev, c.out_dtype) || !sfb::lies_aligned(dE_dev, SFB_F32)) return SFB_ERR_ALIGN;
  const bool drops = drop && drop->drop.threshold > 0;
  const float factor = c.scale * alpha * (drops ? drop->drop.factor : 1.f);
  if (!std::isfinite(factor)) return SFB_ERR_ARG;
  if (n == 0 && add) return SFB_OK;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  const EmbedLayout l = layout_of(c);
  const cudaStream_t s = static_cast<cudaStream_t>(c.stream);
  GradientParams p{};
  p.n = n;
  p.groups = Divisor(static_cast<uint32_t>(groups_of(c.dim)));
  p.tokens = static_cast<uint32_t>(c.tokens);
  p.dx = dX_dev;
  p.lddx = lddx;
  p.dim = c.dim;
  p.wide_in = sfb::lies_wide(dX_dev, lddx, c.out_dtype);
  p.wide_out = sfb::lies_wide(dE_dev, ldde, SFB_F32);
  p.table = dE_dev;
  p.lddt = ldde;
  p.factor = factor;
  p.add = add != 0;
  if (drops) {
    p.drop = drop->drop;
    p.drop.call = call;
  }
  Order o{};
  for (int k = 0; k < 2; ++k) o.entries[k] = reinterpret_cast<uint2*>(h->ws + l.entries[k]);
  o.crossing = reinterpret_cast<uint32_t*>(h->ws + l.crossing);
  const ZeroParams zero{dE_dev, ldde, c.tokens, c.dim, p.wide_out};
  const int64_t slabs = (p.groups.d + 31) / 32;
  cudaError_t e;
  if (n <= kFew) {
    const unsigned zeros = add ? 0 : static_cast<unsigned>(std::min<int64_t>((c.tokens + 31) / 32, sfb::sm_count() * 4));
    const unsigned blocks = zeros + static_cast<unsigned>((n * slabs + kThreads / 32 - 1) / (kThreads / 32));
    uint32_t* status = reinterpret_cast<uint32_t*>(h->ws + l.status);
    e = c.out_dtype == SFB_F32 ? launch_few<float>(p, zero, ids_dev, zeros, status, drops, blocks, s)
        : c.out_dtype == SFB_BF16 ? launch_few<__nv_bfloat16>(p, zero, ids_dev, zeros, status, drops, blocks, s)
                                  : launch_few<__half>(p, zero, ids_dev, zeros, status, drops, blocks, s);
    return e == cudaSuccess ? SFB_OK : fail(h, e);
  }
  e = sort_samples(l, h->ws, c, n, ids_dev, o, add ? nullptr : &zero);
  if (e != cudaSuccess) return fail(h, e);
  p.order = o.entries[0];
  p.crossing = o.crossing;
  p.parts = reinterpret_cast<float*>(h->ws + l.parts);
  p.per = samples_per_chunk(n, p.groups.d);
  p.chunks = static_cast<uint32_t>((n + p.per - 1) / p.per);
  const unsigned blocks = static_cast<unsigned>((static_cast<int64_t>(p.chunks) * p.groups.d + kThreads - 1) / kThreads);
  e = c.out_dtype == SFB_F32 ? launch_gradient<float>(p, drops, blocks, s)
      : c.out_dtype == SFB_BF16 ? launch_gradient<__nv_bfloat16>(p, drops, blocks, s) : launch_gradient<__half>(p, drops, blocks, s);
  // (a single chunk has nothing that goes beyond it)
  if (e == cudaSuccess && p.chunks > 1) {
    const unsigned joins = static_cast<unsigned>(std::min<int64_t>(static_cast<int64_t>(sfb::sm_count()) * 2, (static_cast<int64_t>(p.chunks - 1) * slabs + 7) / 8));
    e = sfb::launch_kernel(join_kernel, dim3(joins), dim3(256), 0, s, 1, p);
  }
  return e == cudaSuccess ? SFB_OK : fail(h, e);
}

extern "C" int sfb_embed_get_status(sfb_embed* h, uint32_t* status_out) {
  if (!h || !status_out) return SFB_ERR_ARG;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  const cudaStream_t s = static_cast<cudaStream_t>(h->cfg.stream);
  cudaError_t e = cudaMemcpyAsync(status_out, h->ws, sizeof(uint32_t), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(h->ws, 0, sizeof(uint32_t), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  return e == cudaSuccess ? SFB_OK : fail(h, e);
}

extern "C" int sfb_embed_last_cuda_error(sfb_embed* h) { return h ? h->last_cuda : 0; }

extern "C" int sfb_embed_destroy(sfb_embed* h) {
  if (!h) return SFB_ERR_ARG;
  delete h;
  return SFB_OK;
}

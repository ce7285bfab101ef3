// Samples from token ids, the gradient of that with respect to the table, and dropout (sfb_embed_*, sfb_dropout_* in sfb.h).
//
//   lookup, dropout   embed_rows_kernel, dropout_kernel: a thread takes groups of eight entries of the output rows
//   gradient          dE[t] = alpha s sum_{i: id_i = t} m_i dX_i, in three launches:
//     sort_kernel     the samples in the order of their tokens (stable: a token's samples stay in their order)
//     gradient_kernel chunks of that order, whichever tokens they hold: a thread adds the samples of a chunk for a group of columns and
//                     writes the sum where the token changes.  Work is even however often a token comes up.  A token that goes beyond
//                     a chunk leaves a part in each.  Other blocks zero the rows that no sample names.
//     join_kernel     adds the parts of such tokens in their order
// Sums are in fp32, in an order that depends on the ids alone: the same bits from call to call.
// All are bound by HBM: the rows read once, the table's rows written once.
#include <algorithm>
#include <cmath>
#include <new>

#include "sfb_elem.cuh"

namespace {

using sfb::DropParams;
using sfb::Divisor;
using sfb::Generator;
using sfb::groups_of;
using sfb::kGroup;
using sfb::pdl_launch_dependents;
using sfb::pdl_wait;
using sfb::Raw;

// A matrix of groups, cut into blocks of kThreads * N of them: row and group of each that a thread takes, N of them kThreads apart.
constexpr int kThreads = 256;
template <int N>
struct Places {
  int64_t row;
  uint32_t group;
  // A block's first place by a division of 64 bits where there are that many, the others by their distance from it.
  __device__ __forceinline__ Places(const Divisor& groups, int64_t block) {
    const uint64_t first = static_cast<uint64_t>(block) * (kThreads * N);
    if (first < 0x7fffffffull) {
      row = groups(static_cast<uint32_t>(first));
    } else {
      row = static_cast<int64_t>(first / groups.d);
    }
    group = static_cast<uint32_t>(first - static_cast<uint64_t>(row) * groups.d);
  }
  __device__ __forceinline__ void at(const Divisor& groups, int k, int64_t& r, uint32_t& g) const {
    const uint32_t n = group + threadIdx.x + k * kThreads, q = groups(n);
    r = row + q;
    g = n - q * groups.d;
  }
};

// ---- lookup ------------------------------------------------------------------------------------------------------------------------
struct RowsParams {
  const void* table;
  int64_t ldt, tokens, n, dim;
  const int32_t* ids;
  void* out;
  int64_t ldo;
  Divisor groups;
  float factor;                        // scale, times the dropout's factor
  bool wide_in, wide_out;
  uint32_t* status;
  DropParams drop;
};

template <typename In, typename Out, bool DROP, int N>
__global__ void __launch_bounds__(kThreads) embed_rows_kernel(const __grid_constant__ RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const Places<N> places(p.groups, blockIdx.x);
  Generator generator;
  if constexpr (DROP) generator.begin(p.drop);
  Raw<In> raw[N];
  int64_t row[N];
  uint32_t group[N];
  bool named[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    places.at(p.groups, k, row[k], group[k]);
    const int32_t id = row[k] < p.n ? p.ids[row[k]] : -1;
    named[k] = id >= 0 && id < p.tokens;
    if (!named[k] && id != -1 && group[k] == 0) atomicOr(p.status, SFB_STATUS_INDEX_RANGE);
    const int64_t col = static_cast<int64_t>(group[k]) * kGroup;
    if (named[k])
      sfb::load_group(static_cast<const In*>(p.table) + id * p.ldt + col, static_cast<int>(min(static_cast<int64_t>(kGroup), p.dim - col)), p.wide_in, raw[k]);
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (row[k] >= p.n) break;
    float v[kGroup] = {};
    if (named[k]) {
      sfb::unpack(raw[k], v);
      if constexpr (DROP) generator.drop(v, static_cast<uint32_t>(row[k]), group[k], p.drop.threshold);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) v[j] *= p.factor;
    }
    const int64_t col = static_cast<int64_t>(group[k]) * kGroup;
    Raw<Out> r;
    sfb::pack(v, r);
    sfb::store_group(static_cast<Out*>(p.out) + row[k] * p.ldo + col, static_cast<int>(min(static_cast<int64_t>(kGroup), p.dim - col)), p.wide_out, r);
  }
}

// ---- dropout -----------------------------------------------------------------------------------------------------------------------
// y = factor x where kept, 0 where not, plus r; y may be x or r.
struct DropoutParams {
  const void *x, *r;
  void* y;
  int64_t ldx, ldr, ldy, n, cols;
  Divisor groups;
  bool wide;
  DropParams drop;
};

template <typename T, bool RESIDUAL, int N>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const __grid_constant__ DropoutParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const Places<N> places(p.groups, blockIdx.x);
  Raw<T> raw[N], more[RESIDUAL ? N : 1];
  int64_t row[N];
  uint32_t group[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    places.at(p.groups, k, row[k], group[k]);
    if (row[k] >= p.n) continue;
    const int64_t col = static_cast<int64_t>(group[k]) * kGroup;
    const int count = static_cast<int>(min(static_cast<int64_t>(kGroup), p.cols - col));
    sfb::load_group(static_cast<const T*>(p.x) + row[k] * p.ldx + col, count, p.wide, raw[k]);
    if constexpr (RESIDUAL) sfb::load_group(static_cast<const T*>(p.r) + row[k] * p.ldr + col, count, p.wide, more[k]);
  }
  Generator generator;
  generator.begin(p.drop);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (row[k] >= p.n) break;
    float v[kGroup];
    sfb::unpack(raw[k], v);
    generator.drop(v, static_cast<uint32_t>(row[k]), group[k], p.drop.threshold);
    if constexpr (RESIDUAL) {
      float u[kGroup];
      sfb::unpack(more[k], u);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) v[j] = fmaf(v[j], p.drop.factor, u[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kGroup; ++j) v[j] *= p.drop.factor;
    }
    const int64_t col = static_cast<int64_t>(group[k]) * kGroup;
    Raw<T> r;
    sfb::pack(v, r);
    sfb::store_group(static_cast<T*>(p.y) + row[k] * p.ldy + col, static_cast<int>(min(static_cast<int64_t>(kGroup), p.cols - col)), p.wide, r);
  }
}

// ---- the samples in the order of their tokens ----------------------------------------------------------------------------------------
// A radix sort by digits of up to ten bits, least significant first, stable.  Up to kSortMost samples one cluster does it all: a CTA takes
// its share of the samples, a warp a run of them; the lanes of a warp that hold the same digit find one another by a ballot a bit.
// More samples take three launches a digit (counts of tiles, their sums, the move), each tile as a CTA of the cluster does it.
constexpr int kSortThreads = 1024, kSortWarps = 32, kSortPer = 8, kSortTile = kSortThreads * kSortPer;
constexpr int kSortCtas = 8;
constexpr int64_t kSortMost = static_cast<int64_t>(kSortTile) * kSortCtas;
constexpr int kMaxBits = 10, kMaxBins = 1 << kMaxBits;

struct SortParams {
  const int32_t* ids;                  // of the first digit; the others read keys_in, at_in
  const uint32_t *keys_in, *at_in;
  uint32_t *keys_out, *at_out;
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
  uint32_t base[kMaxBins];
  uint32_t scan[kSortWarps];
};

// Digits of a tile that begins at `first`: key and the rank within the CTA among those of the same digit, of each of a thread's samples.
template <int PER>
__device__ __forceinline__ void rank_tile(SortShared& s, const SortParams& p, int64_t first, uint32_t (&key)[PER], uint32_t (&at)[PER],
                                          uint16_t (&rank)[PER]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << p.bits;
  for (int i = threadIdx.x; i < kSortWarps * kMaxBins / 2; i += kSortThreads) reinterpret_cast<uint32_t*>(s.rank)[i] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int64_t i = first + warp * (32 * PER) + j * 32 + lane;
    key[j] = 0;
    at[j] = static_cast<uint32_t>(i);
    if (i >= p.n) continue;
    if (p.ids) {
      const int32_t id = p.ids[i];
      const bool named = id >= 0 && static_cast<uint32_t>(id) < p.tokens;
      if (!named && id != -1) atomicOr(p.status, SFB_STATUS_INDEX_RANGE);
      key[j] = named ? static_cast<uint32_t>(id) : p.tokens;
    } else {
      key[j] = __ldcg(p.keys_in + i);
      at[j] = __ldcg(p.at_in + i);
    }
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const bool there = first + warp * (32 * PER) + j * 32 + lane < p.n;
    const uint32_t digit = (key[j] >> p.shift) & (bins - 1);
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
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = s.rank[w][threadIdx.x];
      s.rank[w][threadIdx.x] = static_cast<uint16_t>(sum);
      sum += c;
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
__device__ __forceinline__ void move_tile(const SortShared& s, const SortParams& p, int64_t first, const uint32_t (&key)[PER],
                                          const uint32_t (&at)[PER], const uint16_t (&rank)[PER]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (first + warp * (32 * PER) + j * 32 + lane >= p.n) break;
    const uint32_t digit = (key[j] >> p.shift) & ((1u << p.bits) - 1);
    const uint32_t to = s.base[digit] + s.rank[warp][digit] + rank[j];
    __stcg(p.keys_out + to, key[j]);
    __stcg(p.at_out + to, at[j]);
  }
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_read(const uint32_t* here, int cta) {
  uint32_t v, there;
  const uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(here));
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(a), "r"(cta));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(there) : "memory");
  return v;
}

// Where the sorted samples and what goes with them lie; two buffers that the digits take in turn, the last one writes the first.
struct Order {
  uint32_t *keys[2], *at[2];
  uint32_t* touched;                   // a bit for each token that some sample names
  uint32_t* crossing;                  // [0]: how many chunks hold the beginning of a token that goes beyond them, then which
  int64_t words;                       // of touched; 0: not wanted
};

__device__ __forceinline__ void mark(const Order& o, uint32_t key, uint32_t tokens) {
  if (key < tokens) atomicOr(o.touched + (key >> 5), 1u << (key & 31));
}

template <int PER>
__global__ void __launch_bounds__(kSortThreads, 1) sort_kernel(SortParams p, const __grid_constant__ Order o, int digits, int ctas) {
  extern __shared__ __align__(16) unsigned char shared[];
  SortShared& s = *reinterpret_cast<SortShared*>(shared);
  pdl_launch_dependents();
  pdl_wait();
  const int cta = blockIdx.x;
  const int64_t first = static_cast<int64_t>(cta) * (kSortThreads * PER);
  if (cta == 0 && threadIdx.x == 0) o.crossing[0] = 0;
  for (int64_t i = static_cast<int64_t>(cta) * kSortThreads + threadIdx.x; i < o.words; i += static_cast<int64_t>(ctas) * kSortThreads) o.touched[i] = 0;
  uint32_t key[PER], at[PER];
  uint16_t rank[PER];
  for (int d = 0; d < digits; ++d) {
    const int to = (digits - 1 - d) & 1;
    p.keys_out = o.keys[to];
    p.at_out = o.at[to];
    p.shift = d * p.bits;
    rank_tile<PER>(s, p, first, key, at, rank);
    cluster_sync();                    // every CTA's totals are there (and, the first time, the bits are clear)
    uint32_t all = 0, before = 0;
    if (threadIdx.x < (1 << p.bits)) {
      for (int c = 0; c < ctas; ++c) {
        const uint32_t v = c == cta ? s.total[threadIdx.x] : cluster_read(&s.total[threadIdx.x], c);
        all += v;
        if (c < cta) before += v;
      }
    }
    const uint32_t base = scan_bins(s, all) + before;
    if (threadIdx.x < (1 << p.bits)) s.base[threadIdx.x] = base;
    __syncthreads();
    move_tile<PER>(s, p, first, key, at, rank);
    if (d == 0 && o.words) {
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (first + (threadIdx.x >> 5) * (32 * PER) + j * 32 + (threadIdx.x & 31) < p.n) mark(o, key[j], p.tokens);
    }
    cluster_sync();                    // the order is written, the totals are read
    p.ids = nullptr;
    p.keys_in = o.keys[to];
    p.at_in = o.at[to];
  }
}

// The same for more samples, a launch each.
__global__ void __launch_bounds__(256) sort_clear_kernel(const __grid_constant__ Order o) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i == 0) o.crossing[0] = 0;
  if (i < o.words) o.touched[i] = 0;
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_count_kernel(const __grid_constant__ SortParams p, const __grid_constant__ Order o) {
  extern __shared__ __align__(16) unsigned char shared[];
  SortShared& s = *reinterpret_cast<SortShared*>(shared);
  pdl_launch_dependents();
  pdl_wait();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortTile;
  uint32_t key[kSortPer], at[kSortPer];
  uint16_t rank[kSortPer];
  rank_tile<kSortPer>(s, p, first, key, at, rank);
  if (threadIdx.x < (1 << p.bits)) p.counts[threadIdx.x * p.tiles + blockIdx.x] = s.total[threadIdx.x];
  if (p.ids && o.words) {
#pragma unroll
    for (int j = 0; j < kSortPer; ++j)
      if (first + (threadIdx.x >> 5) * (32 * kSortPer) + j * 32 + (threadIdx.x & 31) < p.n) mark(o, key[j], p.tokens);
  }
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
  extern __shared__ __align__(16) unsigned char shared[];
  SortShared& s = *reinterpret_cast<SortShared*>(shared);
  pdl_launch_dependents();
  pdl_wait();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortTile;
  uint32_t key[kSortPer], at[kSortPer];
  uint16_t rank[kSortPer];
  rank_tile<kSortPer>(s, p, first, key, at, rank);
  const bool bin = threadIdx.x < (1 << p.bits);
  const uint32_t base = scan_bins(s, bin ? p.totals[threadIdx.x] : 0);
  if (bin) s.base[threadIdx.x] = base + p.counts[threadIdx.x * p.tiles + blockIdx.x];
  __syncthreads();
  move_tile<kSortPer>(s, p, first, key, at, rank);
}

// ---- the gradient ------------------------------------------------------------------------------------------------------------------
struct GradientParams {
  const uint32_t *keys, *at;           // in order
  const uint32_t* touched;
  uint32_t* crossing;
  float* parts;                        // [2 chunks][groups][8]: what a chunk's first token has of an earlier one's, and its last one's
                                       // beginning
  int64_t n;
  int32_t per;                         // samples a chunk
  uint32_t chunks, work;               // work: blocks that add; the others zero
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

__device__ __forceinline__ void store_sum(const GradientParams& p, uint32_t key, uint32_t group, const float (&sum)[kGroup]) {
  const int64_t col = static_cast<int64_t>(group) * kGroup;
  const int count = static_cast<int>(min(static_cast<int64_t>(kGroup), p.dim - col));
  float* to = p.table + key * p.lddt + col;
  Raw<float> r;
  float v[kGroup] = {};
  if (p.add) {
    sfb::load_group(to, count, p.wide_out, r);
    sfb::unpack(r, v);
  }
#pragma unroll
  for (int j = 0; j < kGroup; ++j) v[j] = fmaf(p.factor, sum[j], v[j]);
  sfb::pack(v, r);
  sfb::store_group(to, count, p.wide_out, r);
}

constexpr int kAhead = 4;              // samples under way a thread

template <typename T, bool DROP>
__global__ void __launch_bounds__(kThreads) gradient_kernel(const __grid_constant__ GradientParams p) {
  pdl_launch_dependents();
  pdl_wait();
  if (blockIdx.x >= p.work) {          // rows that no sample names
    const Places<4> places(p.groups, blockIdx.x - p.work);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      int64_t row;
      uint32_t group;
      places.at(p.groups, k, row, group);
      if (row >= p.tokens || (p.touched[row >> 5] >> (row & 31) & 1)) continue;
      const int64_t col = static_cast<int64_t>(group) * kGroup;
      const Raw<float> zero{};
      sfb::store_group(p.table + row * p.lddt + col, static_cast<int>(min(static_cast<int64_t>(kGroup), p.dim - col)), p.wide_out, zero);
    }
    return;
  }
  const uint32_t place = blockIdx.x * kThreads + threadIdx.x, chunk = p.groups(place), group = place - chunk * p.groups.d;
  if (chunk >= p.chunks) return;
  const int64_t first = static_cast<int64_t>(chunk) * p.per, last = min(p.n, first + p.per);
  const int64_t col = static_cast<int64_t>(group) * kGroup;
  const int count = static_cast<int>(min(static_cast<int64_t>(kGroup), p.dim - col));
  const T* dx = static_cast<const T*>(p.dx) + col;
  uint32_t key = p.keys[first];
  if (key == p.tokens) return;
  Generator generator;
  if constexpr (DROP) generator.begin(p.drop);
  bool lead = first > 0 && p.keys[first - 1] == key;
  float sum[kGroup] = {};
  auto leave = [&](bool trail) {
    if (!lead && !trail) {
      store_sum(p, key, group, sum);
      return;
    }
    Raw<float> r;
    sfb::pack(sum, r);
    sfb::store_group(p.parts + ((2 * static_cast<int64_t>(chunk) + !lead) * p.groups.d + group) * kGroup, kGroup, true, r);
    if (!lead && group == 0) p.crossing[1 + atomicAdd(p.crossing, 1u)] = chunk;
  };
  for (int64_t i = first; i < last; i += kAhead) {
    uint32_t keys[kAhead], at[kAhead];
    Raw<T> raw[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) keys[q] = i + q < last ? p.keys[i + q] : p.tokens;
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      at[q] = keys[q] < p.tokens ? p.at[i + q] : 0;
      if (keys[q] < p.tokens) sfb::load_group(dx + at[q] * p.lddx, count, p.wide_in, raw[q]);
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if (keys[q] == p.tokens) break;  // nothing follows
      if (keys[q] != key) {
        leave(false);
        key = keys[q];
        lead = false;
#pragma unroll
        for (int j = 0; j < kGroup; ++j) sum[j] = 0.f;
      }
      float v[kGroup];
      sfb::unpack(raw[q], v);
      if constexpr (DROP) generator.drop(v, at[q], group, p.drop.threshold);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) sum[j] += v[j];
    }
  }
  leave(last < p.n && p.keys[last] == key);
}

// Blocks take (token, 32 groups) in turn: eight warps add contiguous shares of the parts, the first adds the shares.
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ GradientParams p) {
  __shared__ float shares[8][32][kGroup + 1];
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t count = p.crossing[0], slabs = (p.groups.d + 31) / 32;
  const int share = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (uint64_t item = blockIdx.x; item < static_cast<uint64_t>(count) * slabs; item += gridDim.x) {
    const uint32_t chunk = p.crossing[1 + item / slabs], group = static_cast<uint32_t>(item % slabs) * 32 + lane;
    const uint32_t key = p.keys[(static_cast<int64_t>(chunk) + 1) * p.per - 1];
    // the chunks behind it that begin with this token
    int64_t more = 0;
    for (int got = 256; got == 256; more += got) {
      const int64_t at = (static_cast<int64_t>(chunk) + 1 + more + threadIdx.x) * p.per;
      got = __syncthreads_count(at < p.n && p.keys[at] == key);
    }
    const int64_t each = (more + 1 + 7) / 8, from = share * each, to = min(more + 1, from + each);
    float sum[kGroup] = {};
    if (group < p.groups.d) {
#pragma unroll 4
      for (int64_t k = from; k < to; ++k) {
        const int64_t slot = k == 0 ? 2 * static_cast<int64_t>(chunk) + 1 : 2 * (chunk + k);
        Raw<float> r;
        float v[kGroup];
        sfb::load_group(p.parts + (slot * p.groups.d + group) * kGroup, kGroup, true, r);
        sfb::unpack(r, v);
#pragma unroll
        for (int j = 0; j < kGroup; ++j) sum[j] += v[j];
      }
    }
#pragma unroll
    for (int j = 0; j < kGroup; ++j) shares[share][lane][j] = sum[j];
    __syncthreads();
    if (share == 0 && group < p.groups.d) {
      for (int w = 1; w < 8 && w * each <= more; ++w)
#pragma unroll
        for (int j = 0; j < kGroup; ++j) sum[j] += shares[w][lane][j];
      store_sum(p, key, group, sum);
    }
    __syncthreads();
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

constexpr int kPer[] = {4, 8, 16, 32, 64};
constexpr int64_t kBlocksMost = (1ll << 31) - 1;

// Samples a chunk: the fewest (more, smaller pieces of work) that still are two full rounds of threads or, beyond that, keep what is left
// of tokens that go beyond a chunk a small part of what is read.
int samples_per_chunk(int64_t n, int64_t groups) {
  for (const int per : kPer)
    if ((n + per - 1) / per * groups <= static_cast<int64_t>(sfb::kModelSms) * 2048) return per;
  return 64;
}

struct EmbedLayout {
  size_t status, crossing, touched, keys[2], at[2], counts, totals, parts, bytes;
  int64_t words, tiles;
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
  l.words = (c.tokens + 31) / 32;
  l.tiles = (n + kSortTile - 1) / kSortTile;
  l.status = take(16);
  // chunks: the most that any number of samples up to n is cut into, and their parts
  int64_t chunks = 1;
  for (const int per : kPer) {
    // the rule takes `per` up to this many samples
    const int64_t most = per == 64 ? n : std::min(n, static_cast<int64_t>(sfb::kModelSms) * 2048 / groups * per);
    chunks = std::max(chunks, (most + per - 1) / per);
  }
  l.crossing = take((chunks + 1) * 4);
  l.touched = take(l.words * 4);
  for (int k = 0; k < 2; ++k) {
    l.keys[k] = take(n * 4);
    l.at[k] = take(n * 4);
  }
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
  if (c->ldt && c->ldt < c->dim) return SFB_ERR_SHAPE;
  return SFB_OK;
}

template <typename In, typename Out, bool DROP>
cudaError_t launch_rows(const RowsParams& p, cudaStream_t s) {
  const int64_t all = p.n * p.groups.d;
  // (four groups a thread, their loads under way together, once that still is a block for each SM)
  if (all >= static_cast<int64_t>(sfb::kModelSms) * kThreads * 4)
    return sfb::launch_kernel(embed_rows_kernel<In, Out, DROP, 4>, dim3(static_cast<unsigned>((all + kThreads * 4 - 1) / (kThreads * 4))), dim3(kThreads), 0, s, 1, p);
  return sfb::launch_kernel(embed_rows_kernel<In, Out, DROP, 1>, dim3(static_cast<unsigned>((all + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, 1, p);
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
  const int64_t all = p.n * p.groups.d;
  if (all >= static_cast<int64_t>(sfb::kModelSms) * kThreads * 4)
    return sfb::launch_kernel(dropout_kernel<T, RESIDUAL, 4>, dim3(static_cast<unsigned>((all + kThreads * 4 - 1) / (kThreads * 4))), dim3(kThreads), 0, s, 1, p);
  return sfb::launch_kernel(dropout_kernel<T, RESIDUAL, 1>, dim3(static_cast<unsigned>((all + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, 1, p);
}
template <typename T>
cudaError_t launch_dropout(const DropoutParams& p, cudaStream_t s) {
  return p.r ? launch_dropout<T, true>(p, s) : launch_dropout<T, false>(p, s);
}

template <int PER>
cudaError_t launch_sort(const SortParams& p, const Order& o, int digits, int ctas, cudaStream_t s) {
  const cudaError_t e = sfb::allow_smem<sort_kernel<PER>>(sizeof(SortShared));
  return e == cudaSuccess ? sfb::launch_kernel(sort_kernel<PER>, dim3(ctas), dim3(kSortThreads), sizeof(SortShared), s, ctas, p, o, digits, ctas) : e;
}

cudaError_t sort_samples(const EmbedLayout& l, char* ws, const sfb_embed_config& c, int64_t n, const int32_t* ids, const Order& o) {
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
  if (n <= kSortMost) {
    const int per = n <= kSortThreads * kSortCtas ? 1 : n <= 2 * kSortThreads * kSortCtas ? 2 : n <= 4 * kSortThreads * kSortCtas ? 4 : 8;
    int ctas = 1;
    while (static_cast<int64_t>(ctas) * kSortThreads * per < n) ctas *= 2;
    if (per == 1) return launch_sort<1>(p, o, digits, ctas, s);
    if (per == 2) return launch_sort<2>(p, o, digits, ctas, s);
    if (per == 4) return launch_sort<4>(p, o, digits, ctas, s);
    return launch_sort<8>(p, o, digits, ctas, s);
  }
  p.tiles = (n + kSortTile - 1) / kSortTile;
  p.counts = reinterpret_cast<uint32_t*>(ws + l.counts);
  p.totals = reinterpret_cast<uint32_t*>(ws + l.totals);
  cudaError_t e = sfb::allow_smem<sort_count_kernel>(sizeof(SortShared));
  if (e == cudaSuccess) e = sfb::allow_smem<sort_move_kernel>(sizeof(SortShared));
  if (e == cudaSuccess) e = sfb::launch_kernel(sort_clear_kernel, dim3(static_cast<unsigned>(std::max<int64_t>(1, (o.words + 255) / 256))), dim3(256), 0, s, 1, o);
  for (int d = 0; d < digits && e == cudaSuccess; ++d) {
    const int to = (digits - 1 - d) & 1;
    p.keys_out = o.keys[to];
    p.at_out = o.at[to];
    p.shift = d * p.bits;
    const dim3 tiles(static_cast<unsigned>(p.tiles));
    e = sfb::launch_kernel(sort_count_kernel, tiles, dim3(kSortThreads), sizeof(SortShared), s, 1, p, o);
    if (e == cudaSuccess) e = sfb::launch_kernel(sort_sum_kernel, dim3(((1 << p.bits) + 7) / 8), dim3(256), 0, s, 1, p);
    if (e == cudaSuccess) e = sfb::launch_kernel(sort_move_kernel, tiles, dim3(kSortThreads), sizeof(SortShared), s, 1, p);
    p.ids = nullptr;
    p.keys_in = p.keys_out;
    p.at_in = p.at_out;
  }
  return e;
}

template <typename T>
cudaError_t launch_gradient(const GradientParams& p, bool drop, unsigned blocks, cudaStream_t s) {
  return drop ? sfb::launch_kernel(gradient_kernel<T, true>, dim3(blocks), dim3(kThreads), 0, s, 1, p)
              : sfb::launch_kernel(gradient_kernel<T, false>, dim3(blocks), dim3(kThreads), 0, s, 1, p);
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
  if (n > (1ll << 32) || cols > (1ll << 30) || ldx < cols || ldy < cols || ldr < cols) return SFB_ERR_SHAPE;
  if (!sfb::lies_aligned(X_dev, dtype) || !sfb::lies_aligned(Y_dev, dtype) || !sfb::lies_aligned(R_dev, dtype)) return SFB_ERR_ALIGN;
  const int64_t groups = groups_of(cols);
  if (n > kBlocksMost / groups * kThreads) return SFB_ERR_SHAPE;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  DropoutParams p{X_dev, R_dev, Y_dev, ldx, ldr, ldy, n, cols, Divisor(static_cast<uint32_t>(groups)), false, h->drop};
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
  if (n > kBlocksMost / groups_of(c.dim) * kThreads) return SFB_ERR_SHAPE;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  const bool drops = drop && drop->drop.threshold > 0;
  RowsParams p{};
  p.table = h->table;
  p.ldt = c.ldt;
  p.tokens = c.tokens;
  p.n = n;
  p.dim = c.dim;
  p.ids = ids_dev;
  p.out = X_dev;
  p.ldo = ldx;
  p.groups = Divisor(static_cast<uint32_t>(groups_of(c.dim)));
  p.factor = c.scale * (drops ? drop->drop.factor : 1.f);
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
  if (n == 0 && add) return SFB_OK;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  const EmbedLayout l = layout_of(c);
  const bool drops = drop && drop->drop.threshold > 0;
  Order o{};
  for (int k = 0; k < 2; ++k) {
    o.keys[k] = reinterpret_cast<uint32_t*>(h->ws + l.keys[k]);
    o.at[k] = reinterpret_cast<uint32_t*>(h->ws + l.at[k]);
  }
  o.touched = reinterpret_cast<uint32_t*>(h->ws + l.touched);
  o.crossing = reinterpret_cast<uint32_t*>(h->ws + l.crossing);
  o.words = add ? 0 : l.words;
  const cudaStream_t s = static_cast<cudaStream_t>(c.stream);
  cudaError_t e = n > 0 ? sort_samples(l, h->ws, c, n, ids_dev, o)
                        : sfb::launch_kernel(sort_clear_kernel, dim3(static_cast<unsigned>(std::max<int64_t>(1, (o.words + 255) / 256))), dim3(256), 0, s, 1, o);
  if (e != cudaSuccess) return fail(h, e);
  GradientParams p{};
  p.keys = o.keys[0];
  p.at = o.at[0];
  p.touched = o.touched;
  p.crossing = o.crossing;
  p.parts = reinterpret_cast<float*>(h->ws + l.parts);
  p.n = n;
  p.groups = Divisor(static_cast<uint32_t>(groups_of(c.dim)));
  p.per = samples_per_chunk(n, p.groups.d);
  p.chunks = static_cast<uint32_t>((n + p.per - 1) / p.per);
  const int64_t work = (static_cast<int64_t>(p.chunks) * p.groups.d + kThreads - 1) / kThreads;
  const int64_t zero = add ? 0 : (c.tokens * p.groups.d + kThreads * 4 - 1) / (kThreads * 4);
  if (work * kThreads > kBlocksMost || work + zero > kBlocksMost) return SFB_ERR_SHAPE;
  p.work = static_cast<uint32_t>(work);
  p.tokens = static_cast<uint32_t>(c.tokens);
  p.dx = dX_dev;
  p.lddx = lddx;
  p.dim = c.dim;
  p.wide_in = sfb::lies_wide(dX_dev, lddx, c.out_dtype);
  p.wide_out = sfb::lies_wide(dE_dev, ldde, SFB_F32);
  p.table = dE_dev;
  p.lddt = ldde;
  p.factor = c.scale * alpha * (drops ? drop->drop.factor : 1.f);
  p.add = add != 0;
  if (drops) {
    p.drop = drop->drop;
    p.drop.call = call;
  }
  const unsigned blocks = static_cast<unsigned>(work + zero);
  e = c.out_dtype == SFB_F32 ? launch_gradient<float>(p, drops, blocks, s)
      : c.out_dtype == SFB_BF16 ? launch_gradient<__nv_bfloat16>(p, drops, blocks, s) : launch_gradient<__half>(p, drops, blocks, s);
  // (a single chunk has nothing that goes beyond it)
  if (e == cudaSuccess && p.chunks > 1) {
    const int64_t slabs = (p.groups.d + 31) / 32;
    const unsigned joins = static_cast<unsigned>(std::min<int64_t>(static_cast<int64_t>(sfb::sm_count()) * 8, static_cast<int64_t>(p.chunks - 1) * slabs));
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

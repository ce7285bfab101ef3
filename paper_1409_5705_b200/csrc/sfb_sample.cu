// One class drawn for each row of logits (sfb_sample in sfb.h).
//
// sample_kernel: a cluster of CTAs has a row.  The row is read once, into shared memory (what does not fit there is read again), and then gone over
// as often as the filters want:
//   1. the largest logit m (all that a greedy answer takes, but for its place); for top-k a bound that the k largest come up to, from the largest
//      logits of lanes.  A small top-k lists what comes up to it, and the rest follows from that list.
//   2. (top-k, top-p) counts of the logits by their distance from m, in up to 1024 bins
//   3. (top-k) the bin of the k-th largest; (top-p) between which bins the nucleus ends, by bounds on what weights of a bin can come to, and
//      between which it is likely to, by the bins' middles
//   4. where what lies up to there fits a list, it is gathered, and the rest follows from that: the CTA that has the list looks for the filters'
//      ends and the draw in it, by whole-number sums over ever narrower bins (find_end)
//   5. else the logits of the bins in question alone, once they are that few (the likely ones first, listed with the sum of all weights in one go;
//      the weights then say whether the end is among them); until then they are counted (or their weights summed) by ordered key in bins of
//      fewer and fewer keys.  Out comes a key and how many of the logits with that key are kept, the first ones: all filters keep a beginning
//      of the order by falling logit and rising index.
//   6. sums of the weights that are kept by warp, whose shares of the row follow one another: prefix sums say which warp the random
//      number falls on, and that warp goes over its share once more
// sample_plain_kernel: rows without top-k and top-p, as soon as there is one for each CTA: one pass, relative to the largest logit so far.
//
// Whole numbers come out: a class is right or wrong.  So the weights exp((z - m) / T) are taken in 64 bits (an error of 1e-7 in a sum over
// 325,000 classes would move one draw in a hundred to the class beside), by a table of 256 powers of two and a polynomial of the third
// degree (table-driven exponentials: P. T. P. Tang, ACM Trans. Math. Softw. 15, 1989): eight operations of 64 bits, 2e-13.  Sums by key are whole
// numbers, so that their order changes nothing; the others are added in a fixed order.
//
// What bounds it (us, caches cold): a single row is a chain of passes of a few thousand logits a CTA, barriers of the cluster (0.3 each) and code
// that is met for the first time (325,000 bf16 classes, top-k and top-p: 20, of which the row's bytes would take 0.1).  Many rows with filters: the
// instructions of a look at each logit, some 10 to 20 for each that may count, 18 for its weight (64 rows of 325,000, mixed settings: 98 to 116; bytes 7;
// 37 rows of 99,999 fp32 at temperatures that keep most classes: 60).  Without filters: 64-bit arithmetic, 8 operations at 0.22 cycles a weight
// and SM (2,048 rows of 10,000 fp32: 47 to 51; 24 of them the weights, bytes 13).
#include <algorithm>
#include <cmath>
#include <new>

#include "sfb_elem.cuh"

namespace {

using sfb::pdl_launch_dependents;
using sfb::pdl_wait;

// What follows from the threads of a CTA (N): two bins, and two places of the list of logits that are gathered, for each.
constexpr int kEach = 2;
template <int N>
struct Of {
  static constexpr int kWarps = N / 32, kBins = kEach * N, kList = kEach * N;
};
constexpr unsigned long long kOut = 1ull << 63;          // the weight of what a filter has left out of a list
constexpr double kGrain = 1125899906842624.0;            // weights of a list are whole numbers, 2^-50 of the largest
constexpr float kWidest = 32.f;              // bins of 2 reach to e^-32 of the largest weight at most
constexpr float kFar = 104.f;                // weights below e^-104 of the largest count as zero: below what min-p can be, 2^-149, and 2^30 of them below 1e-36
constexpr int kMaxCtas = 16;                 // (more than eight: a launch that asks for them)
constexpr int kTable = 256;
constexpr uint32_t kSmall = 64;              // logits that are compared each with each, at most

struct SampleParams {
  const void* z;
  int64_t ldz, classes;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t *ids, *kept;
  float* logp;
  int32_t ctas, share, resident;             // of a row; vectors of 16 bytes that a CTA has at most, and that its shared memory holds
  int32_t fraction, place_bits;              // F; of a class's number
  bool wide;
};

constexpr float kNone = -INFINITY, kLargest = 3.4028234663852886e38f;

// ---- types -------------------------------------------------------------------------------------------------------------------------
// kLow: bits of an fp32 word that such a value leaves zero.  A vector's largest value (which is no NaN where one is not), and a running
// smallest one, which is NaN from the first NaN on.
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <typename T> struct Type;
template <> struct Type<float> {
  static constexpr int kLow = 0;
  using Pair = float;
  static __device__ __forceinline__ Pair most(const uint4& w) {
    return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
  }
  static __device__ __forceinline__ Pair least(const uint4& w, Pair so_far) {
    return min_nan(min_nan(so_far, min_nan(__uint_as_float(w.x), __uint_as_float(w.y))), min_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
  }
  static __device__ __forceinline__ Pair all(float v) { return v; }
  static __device__ __forceinline__ Pair larger(Pair a, Pair b) { return fmaxf(a, b); }
  static __device__ __forceinline__ float largest(Pair v) { return v; }
  static __device__ __forceinline__ float smallest(Pair v) { return v; }
};
#define SFB_SAMPLE_TYPE(T, T2, LOW, BOTH, FLOAT)                                                                                    \
  template <> struct Type<T> {                                                                                                      \
    static constexpr int kLow = LOW;                                                                                                \
    using Pair = T2;                                                                                                                \
    static __device__ __forceinline__ T2 of(uint32_t w) { return *reinterpret_cast<T2*>(&w); }                                      \
    static __device__ __forceinline__ T2 most(const uint4& w) { return __hmax2(__hmax2(of(w.x), of(w.y)), __hmax2(of(w.z), of(w.w))); } \
    static __device__ __forceinline__ T2 least(const uint4& w, T2 so_far) {                                                         \
      return __hmin2_nan(__hmin2_nan(so_far, __hmin2_nan(of(w.x), of(w.y))), __hmin2_nan(of(w.z), of(w.w)));                        \
    }                                                                                                                               \
    static __device__ __forceinline__ T2 all(float v) { return BOTH(v, v); }                                                        \
    static __device__ __forceinline__ T2 larger(T2 a, T2 b) { return __hmax2(a, b); }                                               \
    static __device__ __forceinline__ float largest(T2 v) { return fmaxf(FLOAT(__low2##LOW(v)), FLOAT(__high2##LOW(v))); }          \
    static __device__ __forceinline__ float smallest(T2 v) { return min_nan(FLOAT(__low2##LOW(v)), FLOAT(__high2##LOW(v))); }       \
  };
#define __low216 __low2bfloat16
#define __high216 __high2bfloat16
#define __low213 __low2half
#define __high213 __high2half
SFB_SAMPLE_TYPE(__nv_bfloat16, __nv_bfloat162, 16, __floats2bfloat162_rn, __bfloat162float)
SFB_SAMPLE_TYPE(__half, __half2, 13, __floats2half2_rn, __half2float)
#undef __low216
#undef __high216
#undef __low213
#undef __high213
#undef SFB_SAMPLE_TYPE

// Whole numbers that are ordered like the values (-0 counts as 0).
template <int LOW>
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return (u >> 31 ? ~u : u | 0x80000000u) >> LOW;
}
template <int LOW>
__device__ __forceinline__ float value_of(uint32_t key) {
  const uint32_t u = key << LOW;
  return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~(u | ((1u << LOW) - 1)));
}

// ---- shared memory -------------------------------------------------------------------------------------------------------------------
template <int N, bool FILTERS>
struct Shared {
  static constexpr int kWarps = Of<N>::kWarps, kBins = FILTERS ? Of<N>::kBins : 2, kList = FILTERS ? Of<N>::kList : 2;
  union {
    uint32_t count[kBins];
    unsigned long long mass[kBins];
    unsigned long long list[kList];          // of this CTA
  };
  union {
    unsigned long long order[kList];         // of all of the row's CTAs (also parts of the bins' sums)
    struct {                                 // of the row's warps, in their order: what is kept ahead of each
      double upto[kMaxCtas * kWarps];
      uint32_t ties_ahead[kMaxCtas * kWarps];
    };
  };
  unsigned long long value[kList];           // (bits of) weights of the order (also this CTA's share of the bins, summed over the row)
  double power[kTable];                      // 2^(j / 256)
  double scan[kWarps];                       // (also of the other types that are scanned)
  double part[2][kWarps];
  uint32_t part_count[kWarps];
  float part_most[kWarps], part_least[kWarps];
  uint32_t listed, found[2], first;
  uint32_t low_before, likely_before, likely_upto;
  float last_bin;
  double found_at;
  unsigned long long found_sum, found_entry, small_entry[kSmall], small_value[kSmall];
  uint32_t small;
  // what the row's CTAs have written here
  float most[kMaxCtas], least[kMaxCtas];
  double sums[2][kMaxCtas];
  uint32_t counts[kMaxCtas];
  // the row's warps, in their order: what is kept, but for the last key, of which there are `ties`
  alignas(16) double sum[kMaxCtas * kWarps];
  uint32_t ties[kMaxCtas * kWarps], keeps[kMaxCtas * kWarps];
  double total;
  int32_t winner;
};

__device__ __forceinline__ uint32_t remote(const void* here, int cta) {
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(here))), "r"(cta));
  return there;
}
__device__ __forceinline__ uint32_t read(const uint32_t* here, int cta) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote(here, cta)) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long read(const unsigned long long* here, int cta) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(remote(here, cta)) : "memory");
  return v;
}
__device__ __forceinline__ void write(uint32_t* here, int cta, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote(here, cta)), "r"(v) : "memory");
}
__device__ __forceinline__ void write(float* here, int cta, float v) { write(reinterpret_cast<uint32_t*>(here), cta, __float_as_uint(v)); }
__device__ __forceinline__ void write(double* here, int cta, double v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(remote(here, cta)), "l"(__double_as_longlong(v)) : "memory");
}
// All of the row's threads.
__device__ __forceinline__ void row_sync(int ctas) {
  if (ctas == 1) __syncthreads();
  else asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// ---- weights -------------------------------------------------------------------------------------------------------------------------
// 2^(j / kTable), by the exponential series.
struct Powers { double of[kTable]; };
constexpr Powers powers() {
  Powers p{};
  for (int j = 0; j < kTable; ++j) {
    long double x = 0.693147180559945309417232121458L * j / kTable, term = 1.0L, sum = 1.0L;
    for (int i = 1; i < 24; ++i) sum += term *= x / i;
    p.of[j] = static_cast<double>(sum);
  }
  return p;
}
__device__ const Powers kPowers = powers();

// exp((z - m) / T), 0 for z below `far`.  Where m is infinite: 1 for such logits (m, per are 0 here and far is infinite).
struct Weight {
  const double* power;
  double m, per;                             // 256 log2(e) / T
  float far;
  // For finite z from `far` to m: two factors of it.
  __device__ __forceinline__ void factors(float z, double& s, double& e) const {
    // (z - m) per = k + f, |f| <= 1/2: the sum with 1.5 * 2^52 leaves k in the low bits
    const double d = static_cast<double>(z) - m;
    const double shifted = fma(d, per, 6755399441055744.0);
    const int k = __double2loint(shifted);
    const double f = fma(d, per, 6755399441055744.0 - shifted);
    // 2^(f / 256): (ln 2 / 256)^j / j!
    constexpr double c1 = 0.6931471805599453 / kTable, c2 = c1 * c1 / 2, c3 = c2 * c1 / 3;
    e = fma(fma(fma(c3, f, c2), f, c1), f, 1.0);
    const double t = power[k & (kTable - 1)];
    s = __hiloint2double(__double2hiint(t) + ((k >> 8) << 20), __double2loint(t));
  }
  __device__ __forceinline__ double operator()(float z) const {
    double s, e;
    factors(fminf(fmaxf(z, far), kLargest), s, e);
    return z >= far ? s * e : 0.0;
  }
};

// 2^n, and the n of the power of two that a positive number is not below, for what is far from the type's ends.
__device__ __forceinline__ double power_of_two(int n) { return __hiloint2double((1023 + n) << 20, 0); }
__device__ __forceinline__ int log2_of(double v) { return (__double2hiint(v) >> 20) - 1023; }

__device__ __forceinline__ Weight weight_of(const double* power, float m, float temperature, double per) {
  return isinf(m) ? Weight{power, 0.0, 0.0, m} : Weight{power, m, per, fmaxf(m - kFar * temperature, -kLargest)};
}
__device__ __forceinline__ double per_of(float temperature) { return 369.3299304757463 / temperature; }        // 256 log2(e)

template <typename V>
__device__ __forceinline__ V shuffle_up(V v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }
__device__ __forceinline__ uint32_t warp_sum(uint32_t v) { return __reduce_add_sync(0xffffffffu, v); }
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// (Functions of their own, not copies at each call: a CTA goes through the kernel once, and waits for its instructions.)
// What lies in the threads before this one; the whole in `all`.
template <int N, bool FILTERS, typename V>
__device__ __noinline__ V block_scan(Shared<N, FILTERS>& s, V value, V& all) {
  constexpr int kWarps = Of<N>::kWarps;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  V* part = reinterpret_cast<V*>(s.scan);
  V sum = value;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V v = shuffle_up(sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) part[warp] = sum;
  __syncthreads();
  V upto = lane < kWarps ? part[lane] : 0;
#pragma unroll
  for (int o = 1; o < kWarps; o <<= 1) {
    const V v = shuffle_up(upto, o);
    if (lane >= o) upto += v;
  }
  all = __shfl_sync(0xffffffffu, upto, kWarps - 1);
  const V ahead = __shfl_sync(0xffffffffu, upto, max(warp - 1, 0));
  __syncthreads();
  return (warp ? ahead : 0) + (sum - value);
}
// The threads' sum (of small whole numbers).
template <int N, bool FILTERS>
__device__ __noinline__ uint32_t block_sum(Shared<N, FILTERS>& s, uint32_t value) {
  constexpr int kWarps = Of<N>::kWarps;
  const uint32_t v = warp_sum(value);
  if ((threadIdx.x & 31) == 0) s.part_count[threadIdx.x >> 5] = v;
  __syncthreads();
  const uint32_t all = warp_sum((threadIdx.x & 31) < kWarps ? s.part_count[threadIdx.x & 31] : 0u);
  __syncthreads();
  return all;
}

// ---- a CTA's share of a row ------------------------------------------------------------------------------------------------------------
template <typename T>
struct Slice {
  static constexpr int kV = 16 / sizeof(T);
  const T* z;                                // of the share
  uint4* held;
  int vectors, resident;
  int64_t entries;
  bool wide;

  __device__ __forceinline__ uint4 fetch(int i) const {
    const int64_t at = static_cast<int64_t>(i) * kV;
    if (wide && at + kV <= entries) return reinterpret_cast<const uint4*>(z)[i];
    uint4 w;
    T* e = reinterpret_cast<T*>(&w);
#pragma unroll
    for (int j = 0; j < kV; ++j) e[j] = at + j < entries ? z[at + j] : sfb::from_float<T>(kNone);
    return w;
  }
  __device__ __forceinline__ uint4 vector(int i) const { return i < resident ? held[i] : fetch(i); }
  static __device__ __forceinline__ void widen(const uint4& w, float (&v)[kV]) {
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int j = 0; j < kV; ++j) v[j] = sfb::to_float(e[j]);
  }
};

// A vector of one value.
template <typename T>
__device__ __forceinline__ uint4 filled(float v) {
  uint4 w;
  T* e = reinterpret_cast<T*>(&w);
#pragma unroll
  for (int j = 0; j < Slice<T>::kV; ++j) e[j] = sfb::from_float<T>(v);
  return w;
}

// Calls f(z, place in the share) for the logits of a warp's vectors from `gate` to `top`, one after another.
template <typename T, typename F>
__device__ __forceinline__ void each_hit(const Slice<T>& s, int from, int to, float gate, float top, F&& f) {
  const int first = from + (threadIdx.x & 31);
  uint4 next = first < to ? s.vector(first) : make_uint4(0, 0, 0, 0);
#pragma unroll 1
  for (int i = first; i < to; i += 32) {
    const uint4 w = next;
    if (i + 32 < to) next = s.vector(i + 32);
    if (!(Type<T>::largest(Type<T>::most(w)) >= gate)) continue;
    float v[Slice<T>::kV];
    Slice<T>::widen(w, v);
    uint32_t hits = 0;
#pragma unroll
    for (int j = 0; j < Slice<T>::kV; ++j) hits |= (v[j] >= gate && v[j] <= top ? 1u : 0u) << j;
#pragma unroll 1
    for (; hits; hits &= hits - 1) {
      const int at = i * Slice<T>::kV + __ffs(hits) - 1;
      f(sfb::to_float(i < s.resident ? reinterpret_cast<const T*>(s.held)[at] : s.z[at]), at);
    }
  }
}
// Calls f(values) for the vectors that hold one.
template <typename T, typename F>
__device__ __forceinline__ void each_vector(const Slice<T>& s, int from, int to, float gate, F&& f) {
#pragma unroll 1
  for (int i = from + (threadIdx.x & 31); i < to; i += 32) {
    const uint4 w = s.vector(i);
    if (!(Type<T>::largest(Type<T>::most(w)) >= gate)) continue;
    float v[Slice<T>::kV];
    Slice<T>::widen(w, v);
    f(v);
  }
}

// ---- keys ------------------------------------------------------------------------------------------------------------------------------
struct Range { uint32_t low, high; };

// The keys that bins [first, last] can hold (and some more beside them: the bins were found in 32 bits).
template <int LOW, int kBins>
__device__ __forceinline__ Range range_of(float m, double unit, int first, int last) {
  Range r{key_of<LOW>(-kLargest), key_of<LOW>(m)};
  if (isinf(m)) {
    if (last == 0) r.low = r.high;
    return r;
  }
  auto at = [&](int bin, double sign) { return m - bin * unit + sign * 1e-6 * (fabs(static_cast<double>(m)) + (bin + 1) * unit); };
  if (first > 0) r.high = min(r.high, key_of<LOW>(static_cast<float>(at(first, 1.0))) + 1);
  if (last < kBins - 1) {
    const uint32_t k = key_of<LOW>(static_cast<float>(at(last + 1, -1.0)));
    r.low = max(r.low, k > 0 ? k - 1 : 0);
  }
  r.high = max(r.high, r.low);
  return r;
}
template <int kBins>
__device__ __forceinline__ int shift_of(const Range& r) {
  const uint32_t width = r.high - r.low;     // the largest distance
  return width < kBins ? 0 : __clz(kBins) + 1 - __clz(width);
}

// The bins' sums over the row's CTAs, two a thread.  Every CTA has passed a row_sync since it filled its own.  Each adds a share of the bins,
// then all read the shares: a sixteenth of what it is if all read all.
template <int N, bool FILTERS, typename V>
__device__ __noinline__ void sum_bins(Shared<N, FILTERS>& s, const V* bins, int ctas, int cta, V (&out)[kEach]) {
  if (ctas == 1) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) out[j] = bins[threadIdx.x * kEach + j];
    __syncthreads();
    return;
  }
  const int share = Of<N>::kBins / ctas, groups = N / share, mine = threadIdx.x % share, group = threadIdx.x / share;      // of two CTAs each
  V* part = reinterpret_cast<V*>(s.order);
  V* summed = reinterpret_cast<V*>(s.value);
  part[threadIdx.x] = read(&bins[cta * share + mine], 2 * group) + read(&bins[cta * share + mine], 2 * group + 1);
  __syncthreads();
  if (threadIdx.x < share) {
    V v = 0;
    for (int g = 0; g < groups; ++g) v += part[g * share + threadIdx.x];
    summed[threadIdx.x] = v;
  }
  row_sync(ctas);
  const int owner = threadIdx.x * kEach / share, at = threadIdx.x * kEach % share;
#pragma unroll
  for (int j = 0; j < kEach; ++j) out[j] = read(&summed[at + j], owner);
}

// Adds to a whole number of 64 bits in shared memory by its halves: the hardware adds 32 bits at a time, and takes many threads at one address in
// its stride, where a 64-bit addition is a loop that each of them wins once.
__device__ __forceinline__ void add(unsigned long long* to, unsigned long long v) {
  uint32_t* half = reinterpret_cast<uint32_t*>(to);
  const uint32_t low = static_cast<uint32_t>(v), old = atomicAdd(half, low), high = static_cast<uint32_t>(v >> 32) + (old + low < old ? 1 : 0);
  if (high) atomicAdd(half + 1, high);
}

// What the CTAs have listed, CTA by CTA: entries.  Returns how many; -1: more than `most`, or than one of the lists holds.  (Every
// CTA has passed a row_sync since it listed.)
template <int N, bool FILTERS>
__device__ __noinline__ int collect(Shared<N, FILTERS>& s, int ctas, int most, bool wanted, unsigned long long* to) {
  const int lane = threadIdx.x & 31;
  const uint32_t n = lane < ctas ? read(&s.listed, lane) : 0;
  uint32_t upto = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = shuffle_up(upto, o);
    if (lane >= o) upto += v;
  }
  const uint32_t all = __shfl_sync(0xffffffffu, upto, 31);
  if (all > most || __any_sync(0xffffffffu, n > Shared<N, FILTERS>::kList)) return -1;
  if (!wanted) return static_cast<int>(all);
  for (uint32_t i0 = 0; i0 < all; i0 += N) {
    const uint32_t i = i0 + threadIdx.x;
    uint32_t c = 0, begin = 0;               // the CTA that has it: the first whose sum goes beyond it
    for (int q = 0; q < ctas - 1; ++q) {
      const uint32_t end = __shfl_sync(0xffffffffu, upto, q);
      if (i >= end) c = q + 1, begin = end;
    }
    if (i < all) to[i] = read(&s.list[i - begin], c);
  }
  return static_cast<int>(all);
}

// Entries of lists: falling keys and rising places in one number, places in its low `bits` bits.
__device__ __forceinline__ uint32_t key_in(unsigned long long entry, int bits) { return ~static_cast<uint32_t>(entry >> bits); }
__device__ __forceinline__ uint32_t place_in(unsigned long long entry, int bits) { return static_cast<uint32_t>(entry) & ((1u << bits) - 1); }

// Entries in ascending order are logits in the order by falling logit and rising place.  The last entry of the beginning of that order whose
// values (value null: 1 each; kOut: none) first come to `target` (1 or more), or the last of all: looked for among [low, high] first, among all where
// it is not there (from_first: no entry lies before the range).  By sums of bins of the range, then of the bin that it is in, until that has few entries, which are compared each with each.
template <int N, bool FILTERS>
__device__ __noinline__ unsigned long long find_end(Shared<N, FILTERS>& s, const unsigned long long* list, const unsigned long long* value, int n,
                                                    unsigned long long low, unsigned long long high, unsigned long long target, bool from_first) {
  constexpr int kBins = Shared<N, FILTERS>::kBins;
  auto worth = [&](int i) { return value ? (value[i] == kOut ? 0 : value[i]) : 1ull; };
  unsigned long long before = 0, all;
  if (!from_first) {
    for (int i = threadIdx.x; i < n; i += N) before += list[i] < low ? worth(i) : 0;
    block_scan(s, before, before);
  }
  for (bool begins = true;; begins = false) {
    const unsigned long long width = high - low;
    const int shift = width < kBins ? 0 : __clz(kBins) + 33 - __clzll(static_cast<long long>(width));
    for (int b = threadIdx.x; b < kBins; b += N) s.mass[b] = 0;
    if (threadIdx.x == 0) s.small = 0, s.found[0] = 0, s.found_sum = before;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += N) {
      const unsigned long long v = worth(i);
      if (v && list[i] >= low && list[i] <= high) add(&s.mass[(list[i] - low) >> shift], v);
    }
    __syncthreads();
    unsigned long long mass[kEach], sum = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) mass[j] = s.mass[threadIdx.x * kEach + j], sum += mass[j];
    unsigned long long upto = before + block_scan(s, sum, all);
    if (begins && (target <= before || target > before + all) && (low > 0 || ~high > 0)) {
      low = before = 0;
      high = ~0ull;
      begins = true;
      continue;
    }
    const unsigned long long want = min(target, before + all);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      if (upto < want && upto + mass[j] >= want) s.found[0] = threadIdx.x * kEach + j, s.found_sum = upto;
      upto += mass[j];
    }
    __syncthreads();
    low += static_cast<unsigned long long>(s.found[0]) << shift;
    high = min(high, low + ((1ull << shift) - 1));
    before = s.found_sum;
    for (int i = threadIdx.x; i < n; i += N) {
      if (list[i] < low || list[i] > high || !worth(i)) continue;
      const uint32_t at = atomicAdd(&s.small, 1u);
      if (at < kSmall) s.small_entry[at] = list[i], s.small_value[at] = worth(i);
    }
    __syncthreads();
    const uint32_t count = s.small;
    if (count <= kSmall) {
      if (threadIdx.x < count) {
        const unsigned long long me = s.small_entry[threadIdx.x], mine = s.small_value[threadIdx.x];
        unsigned long long ahead = before;
#pragma unroll 4
        for (uint32_t j = 0; j < count; ++j)
          if (s.small_entry[j] < me) ahead += s.small_value[j];
        if (ahead < want && ahead + mine >= want) s.found_entry = me;
      }
      __syncthreads();
      const unsigned long long end = s.found_entry;
      __syncthreads();
      return end;
    }
    __syncthreads();
  }
}

// FILTERS: top-k or top-p may be asked for (without them a smaller kernel, of which more threads fit an SM).
template <typename T, int N, bool FILTERS>
__global__ void __launch_bounds__(N, (FILTERS ? 1024 : 1536) / N) sample_kernel(const __grid_constant__ SampleParams p) {
  constexpr int LOW = Type<T>::kLow, kV = Slice<T>::kV;
  extern __shared__ __align__(16) unsigned char dynamic[];
  constexpr int kWarps = Of<N>::kWarps, kBins = Of<N>::kBins, kList = Of<N>::kList;
  __shared__ Shared<N, FILTERS> s;
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kTable; i += N) s.power[i] = kPowers.of[i];
  if (threadIdx.x == 0) s.listed = 0, s.first = 0xffffffffu;
  const int ctas = p.ctas, bits = p.place_bits;
  if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  pdl_wait();

  const int64_t row = blockIdx.x / ctas;
  const int cta = blockIdx.x % ctas;
  const int64_t first = static_cast<int64_t>(cta) * p.share * kV;             // entry of the row
  Slice<T> slice;
  slice.z = static_cast<const T*>(p.z) + row * p.ldz + first;
  slice.held = reinterpret_cast<uint4*>(dynamic);
  slice.entries = max(static_cast<int64_t>(0), min(static_cast<int64_t>(p.share) * kV, p.classes - first));
  slice.vectors = static_cast<int>((slice.entries + kV - 1) / kV);
  slice.resident = min(slice.vectors, p.resident);
  slice.wide = p.wide;
  const int per_warp = (p.share + kWarps - 1) / kWarps;
  const int from = min(warp * per_warp, slice.vectors), to = min(from + per_warp, slice.vectors);
  const float temperature = p.temperature ? p.temperature[row] : 1.f;
  const int32_t top_k = FILTERS && p.top_k ? p.top_k[row] : 0;
  const float top_p = FILTERS && p.top_p ? p.top_p[row] : 1.f;
  const double min_p = p.min_p ? fmin(1.0, fmax(0.0, static_cast<double>(p.min_p[row]))) : 0.0;

  // 1. the row comes in
  float m, least, k_gate = -kLargest;        // at least top_k logits are no smaller than k_gate
  {
    typename Type<T>::Pair high = Type<T>::all(kNone), low = Type<T>::all(INFINITY);
    float tail = INFINITY;
    for (int i = from + lane; i < to; i += 4 * 32) {
      uint4 w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (i + 32 * q < to) w[q] = slice.fetch(i + 32 * q);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (i + 32 * q >= to) break;
        if (i + 32 * q < slice.resident) slice.held[i + 32 * q] = w[q];
        high = Type<T>::larger(high, Type<T>::most(w[q]));
        if (static_cast<int64_t>(i + 32 * q + 1) * kV <= slice.entries) {
          low = Type<T>::least(w[q], low);
        } else {                             // (what lies behind the row's end is minus infinity too, but no hole)
          float v[kV];
          Slice<T>::widen(w[q], v);
          for (int j = 0; (i + 32 * q) * kV + j < slice.entries; ++j) tail = min_nan(tail, v[j]);
        }
      }
    }
    m = fmaxf(Type<T>::largest(high), kNone);
    // A bound below the k-th largest: of the warps' `rounds`-th largest lanes the one that so many warps come up to that they have top_k logits
    // together.  About half of the warps, where that takes more than a lane of each: the least of all would be a poor bound.
    constexpr int kMostRounds = 16;
    const int warps = ctas * kWarps, rounds = top_k <= warps ? 1 : static_cast<int>(min((2ll * top_k + warps - 1) / warps, static_cast<long long>(kMostRounds + 1)));
    const bool gated = top_k > 1 && rounds <= kMostRounds;
    float gate = kNone;
    if (gated) {
      uint32_t key = key_of<0>(m), best = 0;
#pragma unroll 1
      for (int q = 0; q < rounds; ++q) {
        best = __reduce_max_sync(0xffffffffu, key);
        if (lane == __ffs(__ballot_sync(0xffffffffu, key == best)) - 1) key = 0;
      }
      gate = fmaxf(value_of<0>(best), kNone);            // (where a warp has fewer logits: minus infinity)
    }
    least = min_nan(Type<T>::smallest(low), tail);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      least = min_nan(least, __shfl_xor_sync(0xffffffffu, least, o));
    }
    if (lane == 0) s.part_most[warp] = m, s.part_least[warp] = least;
    __syncthreads();
    m = s.part_most[0];
    least = s.part_least[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s.part_most[w]), least = min_nan(least, s.part_least[w]);
    float* gates = reinterpret_cast<float*>(s.sum);      // of the row's warps (whose sums come in the end)
    if (ctas > 1) {
      asm volatile("barrier.cluster.wait;" ::: "memory");          // (all of the row's CTAs are there)
      if (threadIdx.x < ctas) write(&s.most[cta], threadIdx.x, m), write(&s.least[cta], threadIdx.x, least);
      if (gated && lane < ctas) write(&gates[cta * kWarps + warp], lane, gate);
      row_sync(ctas);
      for (int c = 0; c < ctas; ++c) m = fmaxf(m, s.most[c]), least = min_nan(least, s.least[c]);
    } else if (gated) {
      if (lane == 0) gates[warp] = gate;
      __syncthreads();
    }
    m += 0.f;
    if (gated) {
      const int wanted = (top_k + rounds - 1) / rounds;            // warps
      if (threadIdx.x < warps) {
        const float mine = gates[threadIdx.x];
        int larger = 0;
#pragma unroll 4
        for (int w = 0; w < warps; w += 4) {
          const float4 g = *reinterpret_cast<const float4*>(&s.sum[w / 2]);
          const float of[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) larger += of[j] > mine || (of[j] == mine && w + j < static_cast<int>(threadIdx.x));
        }
        if (larger == wanted - 1) s.part_most[0] = mine;
      }
      __syncthreads();
      k_gate = fmaxf(k_gate, s.part_most[0]);
      __syncthreads();
    }
  }
  const bool holes = !(least > kNone);       // some logit is minus infinity or no number
  if (m == kNone) {                          // nothing to draw from
    if (cta == 0 && threadIdx.x == 0) {
      p.ids[row] = -1;
      if (p.logp) p.logp[row] = kNone;
      if (p.kept) p.kept[row] = 0;
    }
    return;                                  // (nothing of another CTA's is read any more)
  }
  if (!(temperature > 0.f) || top_k == 1 || top_p <= 0.f) {                   // nothing to draw: the first place of m
    uint32_t at = 0xffffffffu;
    each_hit(slice, from, to, m, INFINITY, [&](float, int i) { at = min(at, static_cast<uint32_t>(first + i)); });
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) atomicMin(&s.first, at);
    __syncthreads();
    if (threadIdx.x == 0 && ctas > 1) write(&s.counts[cta], 0, s.first);
    row_sync(ctas);
    if (cta == 0 && threadIdx.x == 0) {
      at = s.first;
      for (int c = 1; c < ctas; ++c) at = min(at, s.counts[c]);
      p.ids[row] = static_cast<int32_t>(at);
      if (p.logp) p.logp[row] = 0.f;
      if (p.kept) p.kept[row] = 1;
    }
    return;
  }
  const bool endless = isinf(m);
  const Weight weight = weight_of(s.power, m, temperature, per_of(temperature));
  const double u = fmax(0.0, static_cast<double>(p.u[row]));
  const bool nucleus = top_p < 1.f;

  // Sums of this CTA's threads, to every CTA.
  auto spread = [&](double a, double b, uint32_t n) {
    a = warp_sum(a);
    b = warp_sum(b);
    n = warp_sum(n);
    if (lane == 0) s.part[0][warp] = a, s.part[1][warp] = b, s.part_count[warp] = n;
    __syncthreads();
    if (warp == 0) {
      a = warp_sum(lane < kWarps ? s.part[0][lane] : 0.0);
      b = warp_sum(lane < kWarps ? s.part[1][lane] : 0.0);
      n = warp_sum(lane < kWarps ? s.part_count[lane] : 0u);
      if (lane < ctas) write(&s.sums[0][cta], lane, a), write(&s.sums[1][cta], lane, b), write(&s.counts[cta], lane, n);
    }
  };
  auto gathered = [&](double& a, double& b, uint32_t& n) {                    // (after a row_sync, and before the next)
    a = b = 0.0;
    n = 0;
    for (int c = 0; c < ctas; ++c) a += s.sums[0][c], b += s.sums[1][c], n += s.counts[c];
  };

  // Adds a logit to this CTA's list.
  auto list = [&](float z, int i) {
    const uint32_t at = atomicAdd(&s.listed, 1u);
    if (at < kList) s.list[at] = static_cast<unsigned long long>(~key_of<LOW>(z)) << bits | static_cast<uint32_t>(first + i);
  };
  // Room for all lists in the place of CTA 0's share of the row; how many there are (-1: no list of all that can be kept), and among which keys
  // top-k and the nucleus end.
  const int room = 2 * kList;
  unsigned long long *entry = reinterpret_cast<unsigned long long*>(dynamic), *value = entry + room;        // (p.resident is twice kList at least)
  int in_list = -1;
  Range k_keys{}, p_keys{};
  auto collect_all = [&]() {                 // (after a row_sync)
    in_list = collect(s, ctas, room, cta == 0, entry);
    row_sync(ctas);                          // (the lists are read)
    if (in_list >= 0) return;
    if (threadIdx.x == 0) s.listed = 0;      // (too many, or too many in one CTA's share)
    __syncthreads();
  };

  // 2. counts by distance
  bool cuts = false;                         // top-k leaves something out
  uint32_t k = 0, k_bin = 0, k_before = 0, k_upto = 0, low_bin = 0, high_bin = 0, nucleus_before = 0, nucleus_upto = 0, likely_low = 0, likely_high = 0,
           likely = 0;
  const bool filters = FILTERS && (top_k > 0 || nucleus);
  const float reach = holes ? kWidest : fminf(kWidest, fmaxf((m - least) / temperature, 1.f / 1024));
  const float scale = endless ? 0.f : fminf(kBins / reach / temperature, 1e30f);                                 // bins a unit
  const double unit = scale > 0.f ? 1.0 / scale : INFINITY, width = scale > 0.f ? unit / temperature : 0.0;      // in logits; in exponents
  // (the difference first: m itself is in bin 0)
  auto bin_of = [&](float z) {
    return endless ? (z == m ? 0u : kBins - 1) : min(__float2uint_rz((m - z) * scale), static_cast<uint32_t>(kBins - 1));
  };
  bool unbinned = false;                     // the list was made without bins
  if (FILTERS && k_gate > -kLargest && static_cast<int64_t>(top_k) * 6 <= room) {      // (those from k_gate on are a few times top_k)
    each_hit(slice, from, to, k_gate, INFINITY, list);
    row_sync(ctas);
    collect_all();
    if (in_list >= 0) {
      cuts = unbinned = true;
      k = static_cast<uint32_t>(top_k);
      k_keys = p_keys = Range{key_of<LOW>(k_gate), key_of<LOW>(m)};
    }
  }
  if (filters && in_list < 0) {
    for (int b = threadIdx.x; b < kBins; b += N) s.count[b] = 0;
    __syncthreads();
    // (all logits; those from k_gate on, where they are top_k or more and nothing is asked of the others)
    if (k_gate > -kLargest) {
      each_hit(slice, from, to, k_gate, INFINITY, [&](float z, int) { atomicAdd(&s.count[bin_of(z)], 1u); });
    } else {
      uint4 next = from + lane < to ? slice.vector(from + lane) : make_uint4(0, 0, 0, 0);
#pragma unroll 1
      for (int i = from + lane; i < to; i += 32) {
        float v[kV];
        Slice<T>::widen(next, v);
        if (i + 32 < to) next = slice.vector(i + 32);
#pragma unroll
        for (int j = 0; j < kV; ++j)
          if (v[j] > kNone) atomicAdd(&s.count[bin_of(v[j])], 1u);
      }
    }
    row_sync(ctas);
    uint32_t count[kEach], before[kEach], mine = 0, finite;
    sum_bins(s, s.count, ctas, cta, count);
#pragma unroll
    for (int j = 0; j < kEach; ++j) mine += count[j];
    before[0] = block_scan(s, mine, finite);
#pragma unroll
    for (int j = 1; j < kEach; ++j) before[j] = before[j - 1] + count[j - 1];

    // 3. the bin of the k-th largest, and bins of the nucleus's end.  With S the sum of the weights, that is the first bin up to which they
    // come to top_p S, or behind which (1 - top_p) S or less is left.  A bin's weights lie within a factor of the one at its middle: so what bins
    // up to, or behind, which these sums have bounds (low_bin .. high_bin), and are about what the middles come to (likely_low .. likely_high, which
    // the weights themselves have to bear out).
    cuts = top_k > 0 && (static_cast<uint32_t>(top_k) < finite || k_gate > -kLargest);
    k = cuts ? static_cast<uint32_t>(top_k) : finite;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (before[j] < k && before[j] + count[j] >= k) {
        s.found[0] = threadIdx.x * kEach + j;
        s.found[1] = before[j] + count[j];
        s.low_before = before[j];
      }
    __syncthreads();
    k_bin = s.found[0];
    nucleus_upto = k_upto = s.found[1];
    nucleus_before = k_before = s.low_before;
    low_bin = high_bin = k_bin;
    if (nucleus) {
      // (in fp32: sums of up to 1024 bins are off by less than 1e-5 of the whole, bins that were found in 32 bits by less than that; the last
      // bin has what lies beyond it too, and where the temperature is that high, differences beyond fp32)
      const float share = top_p, rest = 1.f - share, per_bin = static_cast<float>(width), spread_by = __expf(0.5f * per_bin) * 1.0001f, near = 1e-4f + 0.12f * per_bin;
      constexpr float lost = 2e-5f;
      float mid = 0.f, all_mid, bin_mid[kEach];
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int b = threadIdx.x * kEach + j;
        const uint32_t c = before[j] < k ? min(count[j], k - before[j]) : 0;
        bin_mid[j] = b < kBins - 1 ? c * __expf(-(b + 0.5f) * per_bin) : 0.f;
        if (b == kBins - 1) s.last_bin = c * (temperature < 1e36f ? __expf(-b * per_bin) : 1.f);
        mid += bin_mid[j];
      }
      mid = block_scan(s, mid, all_mid);
      const float last = s.last_bin, some = lost * all_mid;
      const float all_low = (all_mid - some) / spread_by, all_high = (all_mid + some) * spread_by + last;
      uint32_t early = 0, open = 0;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const bool end = threadIdx.x * kEach + j == kBins - 1;
        mid += bin_mid[j];
        const float left = end ? 0.f : fmaxf(all_mid - mid, 0.f);
        const float high = end ? all_high : (mid + some) * spread_by, low = (mid - some) / spread_by;
        const float left_low = end ? 0.f : (left - some) / spread_by, left_high = end ? 0.f : (left + some) * spread_by + last;
        early += high < share * all_low || left_low > rest * all_high;
        open += !(low >= share * all_high || left_high <= rest * all_low);
        // the same by the middles alone, and a little to either side
        early += (mid * (1 + near) < share * all_mid || left * (1 - near) > rest * all_mid ? 1u : 0u) << 16;
        open += (mid * (1 - near) >= share * all_mid || left * (1 + near) <= rest * all_mid ? 0u : 1u) << 16;
      }
      early = block_sum(s, early);
      open = block_sum(s, open);
      low_bin = min(early & 0xffffu, k_bin);
      high_bin = min(max(open & 0xffffu, low_bin), k_bin);
      likely_low = min(max(early >> 16, low_bin), high_bin);
      likely_high = min(max(open >> 16, likely_low), high_bin);
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const uint32_t b = threadIdx.x * kEach + j;
        if (b == high_bin) s.found[1] = before[j] + count[j];
        if (b == low_bin) s.low_before = before[j];
        if (b == likely_low) s.likely_before = before[j];
        if (b == likely_high) s.likely_upto = before[j] + count[j];
      }
      __syncthreads();
      nucleus_upto = s.found[1];
      nucleus_before = s.low_before;
      likely = s.likely_upto - s.likely_before;
    }
  }

  // The weights of all logits, where something takes their sum, and of those in the bins before the nucleus's end; what lies in the bins of that end
  // is listed, where it is no more than a list holds (and not all that can be kept is listed below).
  const bool listed_all = filters && in_list < 0 && (cuts ? k_upto : nucleus_upto) <= room;
  const bool few = filters && nucleus && !cuts && !listed_all && likely <= kList;
  double all = 0.0, over = 0.0;
  uint32_t over_count = 0;
  if (!cuts && (nucleus || min_p == 0.0)) {
    if (few) {
      const float low_edge = static_cast<float>(likely_low), high_edge = static_cast<float>(likely_high + 1);
      uint4 next = from + lane < to ? slice.vector(from + lane) : make_uint4(0, 0, 0, 0);
#pragma unroll 1
      for (int i = from + lane; i < to; i += 32) {
        float v[kV];
        Slice<T>::widen(next, v);
        if (i + 32 < to) next = slice.vector(i + 32);
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < kV; ++j) {
          const double w = weight(v[j]);
          const float x = endless ? (v[j] == m ? 0.f : INFINITY) : (m - v[j]) * scale;         // as bin_of has it
          all += w;
          if (x < low_edge && v[j] > kNone) over += w, ++over_count;
          else if ((x < high_edge || likely_high == kBins - 1) && v[j] > kNone) hits |= 1u << j;
        }
        for (; hits; hits &= hits - 1) {
          const int e = i * kV + __ffs(hits) - 1;
          list(sfb::to_float(i < slice.resident ? reinterpret_cast<const T*>(slice.held)[e] : slice.z[e]), e);
        }
      }
    } else {
#pragma unroll 2
      for (int i = from + lane; i < to; i += 32) {
        float v[kV];
        Slice<T>::widen(slice.vector(i), v);
#pragma unroll
        for (int j = 0; j < kV; ++j) all += weight(v[j]);
      }
    }
  }

  uint32_t last_key = 0, last_ties = 0xffffffffu;        // of what is kept: all above the key, and so many that have it
  int listed = -1;                           // in s.order, s.value: of the nucleus's end
  if (filters) {
    // Of a range of keys the first and the last entry.
    auto first_of = [&](const Range& r) { return static_cast<unsigned long long>(~r.high) << bits; };
    auto last_of = [&](const Range& r) { return (static_cast<unsigned long long>(~r.low) << bits) + ((1ull << bits) - 1); };
    double above = 0.0, whole = 0.0;
    uint32_t none;
    // 4. all that can be kept, where that is little enough for a list, which takes the place of CTA 0's share of the row
    if (listed_all) {
      const uint32_t top_bin = cuts ? k_bin : high_bin;
      each_hit(slice, from, to, fmaxf(value_of<LOW>(range_of<LOW, kBins>(m, unit, 0, top_bin).low), k_gate), INFINITY, [&](float z, int i) {
        if (z > kNone && bin_of(z) <= top_bin) list(z, i);
      });
      spread(all, 0.0, 0u);
      row_sync(ctas);
      gathered(whole, above, none);
      k_keys = range_of<LOW, kBins>(m, unit, k_bin, k_bin);
      p_keys = range_of<LOW, kBins>(m, unit, likely_low, likely_high);
      collect_all();
    }
    {
      const int n = in_list;
      if (n >= 0) {
        if (cta != 0) return;
        for (int i = threadIdx.x; i < n; i += N) value[i] = __double2ull_rn(weight(value_of<LOW>(key_in(entry[i], bits))) * kGrain);
        __syncthreads();
        unsigned long long total = 0;
        uint32_t kept = 0;
        auto leave_out = [&](unsigned long long end) {
          for (int i = threadIdx.x; i < n; i += N)
            if (entry[i] > end) value[i] = kOut;
          __syncthreads();
        };
        if (cuts) leave_out(find_end(s, entry, nullptr, n, first_of(k_keys), last_of(k_keys), k, unbinned));
        if (nucleus) {
          double goal = whole * kGrain;
          if (cuts) {
            for (int i = threadIdx.x; i < n; i += N) total += value[i] != kOut ? value[i] : 0;
            block_scan(s, total, total);
            goal = static_cast<double>(total);
          }
          goal = fmin(fmax(ceil(static_cast<double>(top_p) * goal), 1.0), 9.0e18);
          leave_out(find_end(s, entry, value, n, first_of(p_keys), last_of(p_keys), __double2ull_rn(goal), unbinned));
        }
        // The draw, in the order of the places: sums by shares of the row, by shares of the share that the random number falls on, until what is
        // left is little enough to compare each with each.
        total = 0;
        for (int i = threadIdx.x; i < n; i += N) {
          if (min_p > 0.0 && value[i] != kOut && weight(value_of<LOW>(key_in(entry[i], bits))) < min_p) value[i] = kOut;
          if (value[i] == kOut) continue;
          ++kept;
          total += value[i];
        }
        kept = block_sum(s, kept);
        block_scan(s, total, total);
        // the first sum beyond u of the whole; at most the last one
        const unsigned long long goal = min(u < 1.0 ? __double2ull_rz(u * static_cast<double>(total)) : total, total - 1);
        int64_t base = 0, size = p.classes;
        unsigned long long ahead = 0;
        if (threadIdx.x == 0) s.listed = 0;
        __syncthreads();
        bool few_kept = kept <= kSmall;
        if (few_kept) {
          for (int i = threadIdx.x; i < n; i += N)
            if (value[i] != kOut) s.small_entry[atomicAdd(&s.listed, 1u)] = static_cast<unsigned long long>(place_in(entry[i], bits)) << 32 | i;
          __syncthreads();
        }
        while (!few_kept) {
          const uint32_t part = static_cast<uint32_t>((size + kBins - 1) / kBins);
          for (int b = threadIdx.x; b < kBins; b += N) s.mass[b] = 0;
          if (threadIdx.x == 0) s.listed = 0;
          __syncthreads();
          for (int i = threadIdx.x; i < n; i += N) {
            const int64_t at = static_cast<int64_t>(place_in(entry[i], bits)) - base;
            if (value[i] != kOut && at >= 0 && at < size) add(&s.mass[static_cast<uint32_t>(at) / part], value[i]);
          }
          __syncthreads();
          unsigned long long mass[kEach], sum = 0, none;
#pragma unroll
          for (int j = 0; j < kEach; ++j) mass[j] = s.mass[threadIdx.x * kEach + j], sum += mass[j];
          unsigned long long upto = ahead + block_scan(s, sum, none);
#pragma unroll
          for (int j = 0; j < kEach; ++j) {
            if (upto <= goal && upto + mass[j] > goal) s.found[0] = threadIdx.x * kEach + j, s.found_sum = upto;
            upto += mass[j];
          }
          __syncthreads();
          base += static_cast<int64_t>(s.found[0]) * part;
          size = min(static_cast<int64_t>(part), size - static_cast<int64_t>(s.found[0]) * part);
          ahead = s.found_sum;
          for (int i = threadIdx.x; i < n; i += N) {
            const int64_t at = static_cast<int64_t>(place_in(entry[i], bits)) - base;
            if (value[i] == kOut || at < 0 || at >= size) continue;
            const uint32_t to_at = atomicAdd(&s.listed, 1u);
            if (to_at < kSmall) s.small_entry[to_at] = static_cast<unsigned long long>(place_in(entry[i], bits)) << 32 | i;
          }
          __syncthreads();
          if (part == 1 || s.listed <= kSmall) break;
          __syncthreads();
        }
        const uint32_t left = min(s.listed, kSmall);     // (one place has one entry)
        if (threadIdx.x < left) {
          const unsigned long long me = s.small_entry[threadIdx.x];
          const int i = static_cast<int>(static_cast<uint32_t>(me));
          unsigned long long upto = ahead;
          for (uint32_t j = 0; j < left; ++j)
            if (s.small_entry[j] < me) upto += value[static_cast<uint32_t>(s.small_entry[j])];
          if (upto <= goal && upto + value[i] > goal) {
            p.ids[row] = static_cast<int32_t>(me >> 32);
            if (p.logp) p.logp[row] = static_cast<float>(log(weight(value_of<LOW>(key_in(entry[i], bits))) * kGrain / static_cast<double>(total)));
            if (p.kept) p.kept[row] = static_cast<int32_t>(kept);
          }
        }
        return;
      }
    }

    // All lists to every CTA.
    auto gather = [&]() {                    // (after a row_sync)
      const int n = collect(s, ctas, kList, true, s.order);
      row_sync(ctas);                        // (the lists are read)
      if (threadIdx.x == 0) s.listed = 0;
      return n;
    };
    auto list_range = [&](const Range& r) {  // of keys; no more of them than a list holds
      each_hit(slice, from, to, fmaxf(value_of<LOW>(r.low), k_gate), value_of<LOW>(r.high), [&](float z, int i) {
        const uint32_t key = key_of<LOW>(z);
        if (key >= r.low && key <= r.high) list(z, i);
      });
      row_sync(ctas);
      return gather();
    };
    // The last entry of a list that is kept: its key, and how many of that key are kept with it.
    auto ends_at = [&](int n, unsigned long long end) {
      uint32_t ties = 0;
      for (int i = threadIdx.x; i < n; i += N) ties += key_in(s.order[i], bits) == key_in(end, bits) && s.order[i] <= end;
      last_ties = block_sum(s, ties);
      last_key = key_in(end, bits);
    };

    // 5. the k-th largest
    if (cuts) {
      Range r = range_of<LOW, kBins>(m, unit, k_bin, k_bin);
      const bool few_k = k_upto - k_before <= kList;
      if (few_k) {
        each_hit(slice, from, to, fmaxf(value_of<LOW>(r.low), k_gate), value_of<LOW>(r.high), [&](float z, int i) {
          if (bin_of(z) == k_bin) list(z, i);
        });
        row_sync(ctas);
        const int n = gather();
        ends_at(n, find_end(s, s.order, nullptr, n, first_of(r), last_of(r), k - k_before, true));
      }
      while (!few_k) {
        const int shift = shift_of<kBins>(r);
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += N) s.count[b] = 0;
        __syncthreads();
        uint32_t over = 0;
        each_hit(slice, from, to, fmaxf(value_of<LOW>(r.low), k_gate), INFINITY, [&](float z, int) {
          const uint32_t key = key_of<LOW>(z);
          if (key > r.high) ++over;
          else if (key >= r.low) atomicAdd(&s.count[(r.high - key) >> shift], 1u);
        });
        spread(0.0, 0.0, over);
        row_sync(ctas);
        double unused;
        uint32_t some[kEach], inside, sum = 0;
        gathered(unused, unused, over);
        sum_bins(s, s.count, ctas, cta, some);
#pragma unroll
        for (int j = 0; j < kEach; ++j) sum += some[j];
        uint32_t a = over + block_scan(s, sum, inside);
        if (shift > 0 && inside <= kList) {
          const int n = list_range(r);
          ends_at(n, find_end(s, s.order, nullptr, n, first_of(r), last_of(r), k - over, true));
          break;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          if (a < k && a + some[j] >= k) {
            s.found[0] = threadIdx.x * kEach + j;
            s.found[1] = k - a;
          }
          a += some[j];
        }
        __syncthreads();
        const uint32_t high = r.high - (s.found[0] << shift), span = (1u << shift) - 1;
        if (shift == 0) {
          last_key = high;
          last_ties = s.found[1];
          break;
        }
        r = Range{max(r.low, high > span ? high - span : 0u), high};
      }
    }

    // the nucleus
    if (nucleus) {
      Range r = few ? range_of<LOW, kBins>(m, unit, likely_low, likely_high) : range_of<LOW, kBins>(m, unit, low_bin, high_bin);
      r.low = max(r.low, last_key);
      r.high = max(r.high, r.low);
      const uint32_t cut_key = last_key, cut_ties = last_ties;       // of top-k; key 0: none
      const double cut_weight = cuts ? weight(value_of<LOW>(cut_key)) : 0.0;
      const float cut_value = cuts ? value_of<LOW>(cut_key) : kNone;
      double target = 0.0;
      bool cut_inside = cuts && high_bin == k_bin;
      // A list of n logits that follow others with the sum `above`, behind them what top-k leaves of its last key (where that is in reach):
      // where the target is met.  False: not within a list that had to hold it.
      auto meet = [&](int n, bool sure) {
        const double goal = fmax(ceil((target - above) * kGrain), 1.0);
        unsigned long long sum = 0;
        for (int i = threadIdx.x; i < n; i += N) {
          s.value[i] = __double2ull_rn(weight(value_of<LOW>(key_in(s.order[i], bits))) * kGrain);
          sum += s.value[i];
        }
        block_scan(s, sum, sum);
        if (!sure && !(above < target && goal <= static_cast<double>(sum))) return false;
        if (sum > 0 && !(cut_inside && goal > static_cast<double>(sum))) {
          ends_at(n, find_end(s, s.order, s.value, n, first_of(r), last_of(r), __double2ull_rn(fmin(goal, 9.0e18)), true));
        } else if (cut_inside) {
          const double more = ceil((goal - static_cast<double>(sum)) / (cut_weight * kGrain));
          last_key = cut_key;
          last_ties = more >= cut_ties || !(cut_weight > 0.0) ? cut_ties : more > 1.0 ? static_cast<uint32_t>(more) : 1u;
        } else {                             // (weights that are too small for the sums: all is kept)
          last_key = cuts ? cut_key : 0;
          last_ties = cuts ? cut_ties : 0xffffffffu;
          listed = -1;
        }
        return true;
      };
      // sums of the weights: of all that top-k leaves, and of those above the range (by bins at first, then by keys)
      const bool few_left = nucleus_upto - nucleus_before <= kList;
      if (few) {                             // (the sums are there already, and the list)
        spread(over, all, 0u);
        row_sync(ctas);
        double sum_all;
        gathered(above, sum_all, none);
        target = static_cast<double>(top_p) * sum_all;
        listed = gather();
        if (!meet(listed, false)) {          // (the end lies outside the likely bins)
          listed = -1;
          r = range_of<LOW, kBins>(m, unit, low_bin, high_bin);
        }
      }
      // Sums by key are of weights as whole numbers: in units of about 2^-F of the largest weight that the range can have, or finer ones where all weights
      // come to none.  Each is off by half a unit, and equal ones all by the same, so a bin near whose edge the target falls may be the wrong one.
      // The sums of its own weights in 64 bits say so when it is gone over, and the search goes on beside it, within `bound`, which is sure.
      Range bound = r;
      int finer = 0;
      if (listed < 0)
      for (bool begins = true;; begins = false) {
        const int shift = shift_of<kBins>(r);
        // (the largest weight is below 2^(most + 1))
        const int most = endless ? 0 : max(-160, __double2int_rd((value_of<LOW>(r.high) - weight.m) * weight.per * (1.0 / kTable)));
        int unit_bits = p.fraction - 1 - most + finer;
        const double units = power_of_two(unit_bits);
        __syncthreads();
        if (!few_left)
          for (int b = threadIdx.x; b < kBins; b += N) s.mass[b] = 0;
        __syncthreads();
        double over = 0.0, within = 0.0;
        uint32_t inside = 0;
        each_vector(slice, from, to, begins && cuts ? cut_value : value_of<LOW>(r.low), [&](const float (&v)[kV]) {
#pragma unroll
          for (int j = 0; j < kV; ++j) {
            const bool there = v[j] > cut_value;                             // (equal ones are added below)
            const double w = there ? weight(v[j]) : 0.0;
            if (begins && cuts) all += w;
            if (few_left) {
              if (bin_of(v[j]) < low_bin) over += w;
              continue;
            }
            const uint32_t key = key_of<LOW>(v[j]);
            if (key > r.high) {
              over += w;
            } else if (there && key >= r.low) {
              ++inside;
              if (!begins) within += w;
              if (shift == 0) atomicAdd(&s.count[r.high - key], 1u);         // (a bin is one key: its weight comes in below)
              else add(&s.mass[(r.high - key) >> shift], static_cast<unsigned long long>(__double2ll_rn(w * units)));
            }
          }
        });
        if (few_left)
          each_hit(slice, from, to, value_of<LOW>(r.low), value_of<LOW>(r.high), [&](float z, int i) {
            const uint32_t bin = bin_of(z);
            if (z > cut_value && bin >= low_bin && bin <= high_bin) list(z, i);
          });
        spread(over, begins ? all : within, inside);
        row_sync(ctas);
        double sum;                          // of all that top-k leaves but for its last key; then of the range
        gathered(above, sum, inside);
        if (begins) {
          if (cuts) sum += cut_ties * cut_weight;
          target = static_cast<double>(top_p) * sum;
        }
        if (few_left) {
          meet(gather(), true);
          break;
        }
        cut_inside = cuts && cut_key >= r.low && cut_key <= r.high;
        if (!begins) {
          if (cut_inside) sum += cut_ties * cut_weight;
          const bool before = above >= target && r.high < bound.high, behind = above + sum < target && r.low > bound.low;
          if (before || behind) {
            if (before) bound.low = r.high + 1;
            else bound.high = r.low - 1;
            r = bound;
            finer = 0;
            row_sync(ctas);                  // (the sums are read)
            continue;
          }
          bound = r;
        }
        if (shift > 0 && inside <= kList) {
          meet(list_range(Range{max(r.low, cut_key + 1), r.high}), true);
          break;
        }
        unsigned long long some[kEach], mine = 0, mass;
        if (shift == 0) {                    // counts of keys: their weights by 64-bit products, in units of 2^-62 of what holds them all
          uint32_t count[kEach];
          sum_bins(s, s.count, ctas, cta, count);
          unit_bits = 60 - log2_of(begins ? fmax(sum - above, 1e-12 * sum) : fmax(sum, 1e-60));
#pragma unroll
          for (int j = 0; j < kEach; ++j) {
            const uint32_t at = threadIdx.x * kEach + j;
            double here = count[j] ? count[j] * weight(value_of<LOW>(r.high - at)) : 0.0;
            if (cut_inside && r.high - cut_key == at) here += cut_ties * cut_weight;
            some[j] = __double2ull_rn(here * power_of_two(unit_bits));
          }
        } else {
          sum_bins(s, s.mass, ctas, cta, some);
#pragma unroll
          for (int j = 0; j < kEach; ++j)
            if (cut_inside && (r.high - cut_key) >> shift == threadIdx.x * kEach + j) some[j] += cut_ties * __double2ull_rn(cut_weight * units);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) mine += some[j];
        unsigned long long ahead = block_scan(s, mine, mass);
        if (mass == 0 && shift > 0 && finer < 400) {     // (half a unit each at most: in units of 2^-F of that they come to 2^61 at most)
          finer += p.fraction;
          continue;
        }
        // in whole numbers: what the target leaves for the bins, and at least one and at most what they hold, so that one thread finds it
        const double left = ceil((target - above) * power_of_two(unit_bits));
        const unsigned long long want = min(left > 1.0 ? __double2ull_rn(left) : 1ull, mass);
        if (mass == 0 && threadIdx.x == 0) s.found[0] = 0, s.found_at = above;       // (no weight in the range)
        finer = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          if (ahead < want && ahead + some[j] >= want) {
            s.found[0] = threadIdx.x * kEach + j;
            s.found_at = above + ahead * power_of_two(-unit_bits);
          }
          ahead += some[j];
        }
        __syncthreads();
        const uint32_t top = r.high - (s.found[0] << shift), span = (1u << shift) - 1;
        if (shift == 0) {
          const double w = weight(value_of<LOW>(top)), ties = ceil((target - s.found_at) / w);
          last_key = top;
          last_ties = !(w > 0.0) || ties >= 4294967295.0 ? 0xffffffffu : ties > 1.0 ? static_cast<uint32_t>(ties) : 1u;
          if (top == cut_key) last_ties = min(last_ties, cut_ties);
          break;
        }
        r = Range{max(r.low, top > span ? top - span : 0u), top};
      }
    }
  }

  // 6. the draw
  const float last_value = last_key ? value_of<LOW>(last_key) : kNone;
  const double last_weight = last_key ? weight(last_value) : 0.0;
  if (last_weight < min_p) last_ties = 0;
  {
    double sum = all;
    uint32_t keeps = 0, ties = 0;
    if (listed >= 0 && min_p == 0.0) {       // what lies in the bins before, and what is kept of the list
      sum = over;
      keeps = over_count;
      const int64_t begin = first + static_cast<int64_t>(from) * kV, end = first + static_cast<int64_t>(to) * kV;
      unsigned long long more = 0;           // (in whole numbers: their order says nothing)
      for (int i = lane; i < listed; i += 32) {
        const uint32_t place = place_in(s.order[i], bits), key = key_in(s.order[i], bits);
        if (place < begin || place >= end) continue;
        if (key == last_key) ++ties;
        else if (key > last_key) more += s.value[i], ++keeps;
      }
      sum += static_cast<double>(more) / kGrain;
    } else if (!last_key && min_p == 0.0) {
      if (!holes) {
        if (lane == 0) keeps = static_cast<uint32_t>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(to) * kV, slice.entries) - static_cast<int64_t>(from) * kV));
      } else {
        each_hit(slice, from, to, -kLargest, INFINITY, [&](float, int) { ++keeps; });
      }
    } else {
      // (a bound on logits that min-p keeps, in 32 bits: the weights decide)
      float gate = last_key ? last_value : -kLargest;
      if (min_p > 0.0 && !endless) {
        const float by = m + temperature * (__logf(static_cast<float>(min_p)) - 1e-3f) - 1e-6f * fabsf(m);
        if (by > gate) gate = by;            // (not where it is no number)
      }
      sum = 0.0;
      each_vector(slice, from, to, gate, [&](const float (&v)[kV]) {
#pragma unroll
        for (int j = 0; j < kV; ++j) {
          const double w = weight(v[j]);
          const bool keep = v[j] > last_value && w >= min_p;                  // (minus infinity and what is no number is not above)
          if (keep) sum += w;
          keeps += keep;
          ties += v[j] == last_value;
        }
      });
    }
    sum = warp_sum(sum);
    keeps = warp_sum(keeps);
    ties = last_key ? warp_sum(ties) : 0;
    const int at = cta * kWarps + warp;
    if (lane < ctas) write(&s.sum[at], lane, sum), write(&s.keeps[at], lane, keeps), write(&s.ties[at], lane, ties);
  }
  row_sync(ctas);
  if (warp == 0) {                           // the row's warps, a few of them a lane
    constexpr int kMost = kMaxCtas * kWarps / 32;
    const int each_lane = (ctas * kWarps + 31) / 32;
    double sum[kMost], mine = 0.0;
    uint32_t ties[kMost], mine_ties = 0, kept = 0;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      const int i = lane * each_lane + j;
      const bool there = j < each_lane && i < ctas * kWarps;
      sum[j] = there ? s.sum[i] : 0.0;
      ties[j] = there ? s.ties[i] : 0u;
      kept += there ? s.keeps[i] : 0u;
      mine_ties += ties[j];
    }
    uint32_t ties_ahead = mine_ties;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = shuffle_up(ties_ahead, o);
      if (lane >= o) ties_ahead += v;
    }
    ties_ahead -= mine_ties;
    uint32_t first_ties[kMost];
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      first_ties[j] = ties_ahead;
      const uint32_t take = ties_ahead < last_ties ? min(ties[j], last_ties - ties_ahead) : 0;
      sum[j] += take * last_weight;
      kept += take;
      ties_ahead += ties[j];
      mine += sum[j];
    }
    double upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double v = shuffle_up(upto, o);
      if (lane >= o) upto += v;
    }
    const double total = __shfl_sync(0xffffffffu, upto, 31);
    upto = shuffle_up(upto, 1);              // (not upto - mine: what one lane's sums end with, the next one's begin with)
    if (lane == 0) upto = 0.0;
    kept = warp_sum(kept);
    const double target = u < 1.0 ? u * total : INFINITY;
    int found = 0x7fffffff, last = -1;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      const int i = lane * each_lane + j;
      if (j < each_lane && i < ctas * kWarps) {
        s.upto[i] = upto;
        s.ties_ahead[i] = first_ties[j];
        upto += sum[j];
        if (sum[j] > 0.0) {
          last = i;
          if (upto > target) found = min(found, i);
        }
      }
    }
    found = __reduce_min_sync(0xffffffffu, found);
    last = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) {
      s.total = total;
      s.winner = found != 0x7fffffff ? found : last;
      if (cta == 0 && p.kept) p.kept[row] = static_cast<int32_t>(kept);
    }
  }
  __syncthreads();
  const int winner = s.winner;
  if (winner == cta * kWarps + warp) {
    const double total = s.total, target = u < 1.0 ? u * total : INFINITY;
    double upto = s.upto[winner];
    uint32_t seen = s.ties_ahead[winner];
    int at = -1, last_at = -1;               // of the slice
    double w_at = 0.0, last_w = 0.0;
    for (int i0 = from; i0 < to; i0 += 32) {
      const int i = i0 + lane;
      float v[kV];
      double w[kV], sum = 0.0;
      uint32_t ties = 0;
      if (i < to) Slice<T>::widen(slice.vector(i), v);
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        if (i >= to) v[j] = kNone;
        if (last_key && v[j] == last_value) ++ties;
      }
      uint32_t ahead = ties;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = shuffle_up(ahead, o);
        if (lane >= o) ahead += t;
      }
      const uint32_t here = __shfl_sync(0xffffffffu, ahead, 31);
      ahead += seen - ties;
      seen += here;
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        w[j] = 0.0;
        if (last_key && v[j] == last_value) {
          if (ahead++ < last_ties) w[j] = last_weight;
        } else if (v[j] > last_value) {      // (minus infinity and what is no number is not)
          w[j] = weight(v[j]);
          if (w[j] < min_p) w[j] = 0.0;
        }
        sum += w[j];
        if (w[j] > 0.0) last_at = i * kV + j, last_w = w[j];
      }
      double incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double t = shuffle_up(incl, o);
        if (lane >= o) incl += t;
      }
      const uint32_t over = __ballot_sync(0xffffffffu, sum > 0.0 && upto + incl > target);
      if (over) {
        if (lane == __ffs(over) - 1) {
          double a = upto + (incl - sum);
#pragma unroll
          for (int j = 0; j < kV; ++j) {
            if (w[j] > 0.0 && (at < 0 || a <= target)) at = i * kV + j, w_at = w[j];
            a += w[j];
          }
        } else {
          at = -1;
        }
        last_at = at;
        last_w = w_at;
        break;
      }
      upto += __shfl_sync(0xffffffffu, incl, 31);
    }
    // the place that was found, or, where rounding leaves the target behind the last one, that
    const int best_at = __reduce_max_sync(0xffffffffu, last_at);
    if (best_at >= 0 && last_at == best_at) {
      p.ids[row] = static_cast<int32_t>(first + best_at);
      if (p.logp) p.logp[row] = static_cast<float>(log(last_w / total));
    }
  }
}

// 16 bytes that the launch ahead may have written while this one began: no load of constant data (__ldg), which may be older than pdl_wait, or come
// before it.  (volatile: in its place among the other asm; us at 2,048 rows of 10,000 fp32, caches cold: 53; with plain loads, which the compiler keeps
// in order with more, 55.)
__device__ __forceinline__ uint4 load_coherent(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Many rows without top-k and top-p: a CTA a row, whose warps go over their shares of it once, from global memory, with sums relative to the
// largest logit that each has seen (when a larger one comes up, what it has is rescaled).  Sums and largest logits of the warps say which one the
// random number falls on, and that warp goes over its share again.  Rows with min-p, which needs the largest logit first, are gone over twice.
template <typename T, int N>
__global__ void __launch_bounds__(N, 1280 / N) sample_plain_kernel(const __grid_constant__ SampleParams p) {
  constexpr int kV = Slice<T>::kV, kWarps = N / 32, kAhead = 2;
  __shared__ double power[kTable], sum_of[kWarps], upto_of[kWarps], total_of;
  __shared__ float most_of[kWarps];
  __shared__ uint32_t keeps_of[kWarps];
  __shared__ int winner_of;
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kTable; i += N) power[i] = kPowers.of[i];
  pdl_wait();
  const int64_t row = blockIdx.x;
  Slice<T> slice;
  slice.z = static_cast<const T*>(p.z) + row * p.ldz;
  slice.held = nullptr;
  slice.entries = p.classes;
  slice.vectors = p.share;
  slice.resident = 0;
  slice.wide = p.wide;
  const int per_warp = (p.share + kWarps - 1) / kWarps, from = min(warp * per_warp, p.share), to = min(from + per_warp, p.share);
  const float temperature = p.temperature ? p.temperature[row] : 1.f;
  const double min_p = p.min_p ? fmin(1.0, fmax(0.0, static_cast<double>(p.min_p[row]))) : 0.0;
  const bool draws = temperature > 0.f;
  __syncthreads();                           // the table is there

  float most = kNone;                        // of the warp
  double sum[2] = {0.0, 0.0};
  bool holes = false;
  const double per = draws ? per_of(temperature) : 0.0;
  Weight weight{power, 0.0, 0.0, 0.f};
  for (int i0 = from; i0 < to; i0 += kAhead * 32) {
    uint4 w[kAhead];
    uint32_t ragged = 0;
    typename Type<T>::Pair high = Type<T>::all(kNone), low = Type<T>::all(INFINITY);
    if (slice.wide && i0 + kAhead * 32 <= to && static_cast<int64_t>(i0 + kAhead * 32) * kV <= slice.entries) {
      const uint4* z = reinterpret_cast<const uint4*>(slice.z) + i0 + lane;
#pragma unroll
      for (int q = 0; q < kAhead; ++q) w[q] = load_coherent(z + q * 32);
    } else {
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const int i = i0 + q * 32 + lane;
        w[q] = i < to ? slice.fetch(i) : filled<T>(kNone);
        if (i < to && static_cast<int64_t>(i + 1) * kV <= slice.entries) continue;
        // (what lies behind the row's end, or the warp's, is no hole)
        if (i < to) {
          float v[kV];
          Slice<T>::widen(w[q], v);
          for (int j = 0; static_cast<int64_t>(i) * kV + j < slice.entries; ++j) holes |= !(v[j] > kNone);
        }
        ragged |= 1u << q;
      }
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      high = Type<T>::larger(high, Type<T>::most(w[q]));
      if (!(ragged >> q & 1)) low = Type<T>::least(w[q], low);
    }
    holes |= !(Type<T>::smallest(low) > kNone);
    const float here = fmaxf(Type<T>::largest(high), kNone) + 0.f;
    if (__any_sync(0xffffffffu, here > most)) {
      float larger = here;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) larger = fmaxf(larger, __shfl_xor_sync(0xffffffffu, larger, o));
      if (draws) {
        weight = weight_of(power, larger, temperature, per);
        const double by = most > kNone ? weight(most) : 0.0;
        sum[0] *= by;
        sum[1] *= by;
      }
      most = larger;
    }
    if (!draws || min_p > 0.0 || most == kNone) continue;
    if (isinf(most)) {
      for (int q = 0; q < kAhead; ++q) {
        float v[kV];
        Slice<T>::widen(w[q], v);
        for (int j = 0; j < kV; ++j) sum[0] += v[j] == most ? 1.0 : 0.0;
      }
      continue;
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      float v[kV];
      Slice<T>::widen(w[q], v);
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        double s, e;
        weight.factors(fmaxf(v[j], weight.far), s, e);
        if (v[j] >= weight.far) sum[j & 1] = fma(s, e, sum[j & 1]);
      }
    }
  }
  const bool some_holes = __any_sync(0xffffffffu, holes);
  if (lane == 0) most_of[warp] = most;
  __syncthreads();
  float m = most_of[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) m = fmaxf(m, most_of[w]);
  if (m == kNone || !draws) {                // nothing to draw from, or nothing to draw: the first place of m
    int at = 0x7fffffff;
    if (m != kNone && most == m) each_hit(slice, from, to, m, INFINITY, [&](float, int i) { at = min(at, i); });
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) keeps_of[warp] = at;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kWarps; ++w) at = min(at, static_cast<int>(keeps_of[w]));
      p.ids[row] = m == kNone ? -1 : at;
      if (p.logp) p.logp[row] = m == kNone ? kNone : 0.f;
      if (p.kept) p.kept[row] = m == kNone ? 0 : 1;
    }
    return;
  }
  // what the warp has, relative to the row's largest logit
  const Weight row_weight = weight_of(power, m, temperature, per);
  double mine, scale = 1.0;
  uint32_t keeps = 0;
  if (min_p > 0.0) {
    weight = row_weight;
    mine = 0.0;
    each_vector(slice, from, to, -kLargest, [&](const float (&v)[kV]) {
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        const double w = weight(v[j]);
        const bool keep = v[j] > kNone && w >= min_p;
        if (keep) mine += w;
        keeps += keep;
      }
    });
    mine = warp_sum(mine);
  } else {
    scale = most > kNone ? row_weight(most) : 0.0;
    mine = warp_sum(sum[0] + sum[1]) * scale;
    if (some_holes) each_hit(slice, from, to, -kLargest, INFINITY, [&](float, int) { ++keeps; });
    else if (lane == 0) keeps = static_cast<uint32_t>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(to) * kV, p.classes) - static_cast<int64_t>(from) * kV));
  }
  keeps = warp_sum(keeps);
  if (lane == 0) sum_of[warp] = mine, keeps_of[warp] = keeps;
  __syncthreads();
  if (threadIdx.x == 0) {
    const double u = fmax(0.0, static_cast<double>(p.u[row]));
    double total = 0.0;
    uint32_t kept = 0;
    for (int w = 0; w < kWarps; ++w) upto_of[w] = total, total += sum_of[w], kept += keeps_of[w];
    const double target = u < 1.0 ? u * total : INFINITY;
    int found = -1, last = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (!(sum_of[w] > 0.0)) continue;
      last = w;
      if (found < 0 && upto_of[w] + sum_of[w] > target) found = w;
    }
    winner_of = found >= 0 ? found : last;
    total_of = total;
    if (p.kept) p.kept[row] = static_cast<int32_t>(kept);
  }
  __syncthreads();
  // over that share again, relative to its own largest logit as before: each warp a part of it, then the one that the random number falls on
  const int winner = winner_of, share_from = min(winner * per_warp, p.share), share_to = min(share_from + per_warp, p.share);
  const double u = fmax(0.0, static_cast<double>(p.u[row])), total = total_of, target = u < 1.0 ? u * total : INFINITY;
  if (!(min_p > 0.0)) {
    weight = weight_of(power, most_of[winner], temperature, per);
    scale = row_weight(most_of[winner]);
  }
  const int per_part = ((share_to - share_from + kWarps - 1) / kWarps + 31) / 32 * 32, part_from = min(share_from + warp * per_part, share_to),
            part_to = min(part_from + per_part, share_to);
  double part = 0.0;
  for (int i = part_from + lane; i < part_to; i += 32) {
    float v[kV];
    Slice<T>::widen(slice.fetch(i), v);
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      const double w = v[j] > kNone ? weight(v[j]) : 0.0;
      if (w >= min_p) part += w;
    }
  }
  part = warp_sum(part) * scale;
  __syncthreads();                           // (upto_of is read below alone)
  if (lane == 0) sum_of[warp] = part;
  __syncthreads();
  double upto = upto_of[winner], last_upto = upto;
  int chosen = -1, last_part = 0;
  for (int w = 0; w < kWarps; ++w) {
    if (sum_of[w] > 0.0) last_part = w, last_upto = upto;
    if (chosen < 0 && sum_of[w] > 0.0 && upto + sum_of[w] > target) {
      chosen = w;
      break;
    }
    upto += sum_of[w];
  }
  if (chosen < 0) chosen = last_part, upto = last_upto;
  if (warp != chosen) return;
  int at = -1, last_at = -1;
  double w_at = 0.0, last_w = 0.0;
  for (int i0 = part_from; i0 < part_to; i0 += 32) {
    const int i = i0 + lane;
    float v[kV];
    double w[kV], here = 0.0;
    if (i < part_to) Slice<T>::widen(slice.fetch(i), v);
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      w[j] = i < part_to && v[j] > kNone ? weight(v[j]) : 0.0;
      w[j] = w[j] < min_p ? 0.0 : w[j] * scale;
      here += w[j];
      if (w[j] > 0.0) last_at = i * kV + j, last_w = w[j];
    }
    double incl = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double t = shuffle_up(incl, o);
      if (lane >= o) incl += t;
    }
    const uint32_t over = __ballot_sync(0xffffffffu, here > 0.0 && upto + incl > target);
    if (over) {
      if (lane == __ffs(over) - 1) {
        double a = upto + (incl - here);
#pragma unroll
        for (int j = 0; j < kV; ++j) {
          if (w[j] > 0.0 && (at < 0 || a <= target)) at = i * kV + j, w_at = w[j];
          a += w[j];
        }
      }
      last_at = at;
      last_w = w_at;
      break;
    }
    upto += __shfl_sync(0xffffffffu, incl, 31);
  }
  const int best_at = __reduce_max_sync(0xffffffffu, last_at);
  if (best_at >= 0 && last_at == best_at) {
    p.ids[row] = best_at;
    if (p.logp) p.logp[row] = static_cast<float>(log(last_w / total));
  }
}

}  // namespace

struct sfb_sampler {
  sfb_sampler_config cfg;
  int device;
  int last_cuda;
};

namespace {

int check(const sfb_sampler_config* c) {
  if (!c || c->classes <= 0 || c->max_samples < 0 || !sfb::is_dtype(c->dtype)) return SFB_ERR_ARG;
  if (c->classes > (1ll << 30) || c->max_samples > (1ll << 27)) return SFB_ERR_SHAPE;
  return SFB_OK;
}

constexpr int kHeldMost = 192 << 10;         // of a CTA's shared memory, for the row
constexpr int kHeldFour = 40 << 10;          // ... where four CTAs of half the threads are on an SM
constexpr int kHeldTwo = 79 << 10;           // ... where two CTAs are (the rest of the row is read from L2 again)
constexpr int kShareMost = 128 << 10;        // bytes of a row that a CTA has, at most: what is under way at a time then stays in L2

// CTAs that are there at a time, two on an SM, in clusters of so many (what the driver says for 148 SMs: a cluster lies within a part of the chip).
int slots(int ctas) { return ctas <= 2 ? 296 : ctas == 4 ? 284 : ctas == 8 ? 264 : 224; }

template <typename T, int N, bool FILTERS>
cudaError_t launch(SampleParams p, int64_t n, cudaStream_t s) {
  // (the lists have room in the place of the row: at least for twice what one CTA lists)
  if (FILTERS) p.resident = std::max(p.resident, 2 * Of<N>::kList);
  cudaError_t e = sfb::allow_smem<sample_kernel<T, N, FILTERS>>(kHeldMost);
  if (e == cudaSuccess && p.ctas > 8) e = sfb::allow_clusters<sample_kernel<T, N, FILTERS>>();
  if (e != cudaSuccess) return e;
  return sfb::launch_kernel(sample_kernel<T, N, FILTERS>, dim3(static_cast<unsigned>(n * p.ctas)), dim3(N), static_cast<size_t>(p.resident) * 16, s, p.ctas, p);
}

template <typename T>
cudaError_t launch(SampleParams p, int64_t n, cudaStream_t s) {
  const int64_t vectors = (p.classes * static_cast<int64_t>(sizeof(T)) + 15) / 16;
  // More CTAs a row where all rows still are under way at once, and a CTA has enough of its row.
  int ctas = 1;
  while (ctas < 8 && vectors * 16 > static_cast<int64_t>(kShareMost) * ctas) ctas *= 2;
  while (ctas < kMaxCtas && n * ctas * 2 <= slots(ctas * 2) && vectors * 16 > (16 << 10) * ctas) ctas *= 2;
  p.ctas = ctas;
  p.share = static_cast<int32_t>((vectors + ctas - 1) / ctas);
  p.resident = std::min(p.share, (n * ctas <= 112 ? kHeldMost : kHeldTwo) / 16);
  const bool small = p.share <= kHeldFour / 16 && n * ctas > 2 * sfb::kModelSms;
  if (p.top_k || p.top_p) return small ? launch<T, 256, true>(p, n, s) : launch<T, 512, true>(p, n, s);
  // (with a row for each CTA nothing but the random number's share is read twice)
  if (ctas == 1) return sfb::launch_kernel(sample_plain_kernel<T, 256>, dim3(static_cast<unsigned>(n)), dim3(256), 0, s, 1, p);
  return launch<T, 512, false>(p, n, s);
}

}  // namespace

extern "C" int sfb_sampler_init(const sfb_sampler_config* cfg, sfb_sampler** out) {
  if (!out) return SFB_ERR_ARG;
  *out = nullptr;
  const int rc = check(cfg);
  if (rc) return rc;
  int dev = 0;
  const int on = sfb::this_device(&dev);
  if (on) return on;
  sfb_sampler* h = new (std::nothrow) sfb_sampler();
  if (!h) return SFB_ERR_ARG;
  h->cfg = *cfg;
  h->device = dev;
  *out = h;
  return SFB_OK;
}

extern "C" int sfb_sample(sfb_sampler* h, int64_t n, const void* Z_dev, int64_t ldz, const float* u_dev, const float* temperature_dev,
                          const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev, int32_t* ids_dev, float* logp_dev,
                          int32_t* kept_dev) {
  if (!h || n < 0) return SFB_ERR_ARG;
  const sfb_sampler_config& c = h->cfg;
  if (n > c.max_samples) return SFB_ERR_SHAPE;
  if (n == 0) return SFB_OK;
  if (!Z_dev || !u_dev || !ids_dev) return SFB_ERR_ARG;
  if (ldz < c.classes) return SFB_ERR_SHAPE;
  const uintptr_t words = reinterpret_cast<uintptr_t>(u_dev) | reinterpret_cast<uintptr_t>(temperature_dev) | reinterpret_cast<uintptr_t>(top_k_dev) |
                          reinterpret_cast<uintptr_t>(top_p_dev) | reinterpret_cast<uintptr_t>(min_p_dev) | reinterpret_cast<uintptr_t>(ids_dev) |
                          reinterpret_cast<uintptr_t>(logp_dev) | reinterpret_cast<uintptr_t>(kept_dev);
  if ((words & 3u) || !sfb::lies_aligned(Z_dev, c.dtype)) return SFB_ERR_ALIGN;
  const sfb::OnDevice on(h->device);
  if (on.err != cudaSuccess) {
    h->last_cuda = static_cast<int>(on.err);
    return SFB_ERR_CUDA;
  }
  SampleParams p{};
  p.z = Z_dev;
  p.ldz = ldz;
  p.classes = c.classes;
  p.u = u_dev;
  p.temperature = temperature_dev;
  p.top_k = top_k_dev;
  p.top_p = top_p_dev;
  p.min_p = min_p_dev;
  p.ids = ids_dev;
  p.logp = logp_dev;
  p.kept = kept_dev;
  int bits = 0;
  while ((1ll << bits) < c.classes) ++bits;
  p.place_bits = bits;
  p.fraction = 62 - bits;                    // the weights are 1 at most: their sum is below 2^63
  p.wide = sfb::lies_wide(Z_dev, ldz, c.dtype);
  const cudaStream_t s = static_cast<cudaStream_t>(c.stream);
  const cudaError_t e = c.dtype == SFB_F32 ? launch<float>(p, n, s) : c.dtype == SFB_BF16 ? launch<__nv_bfloat16>(p, n, s) : launch<__half>(p, n, s);
  if (e == cudaSuccess) return SFB_OK;
  h->last_cuda = static_cast<int>(e);
  return SFB_ERR_CUDA;
}

extern "C" int sfb_sampler_last_cuda_error(sfb_sampler* h) { return h ? h->last_cuda : 0; }

extern "C" int sfb_sampler_destroy(sfb_sampler* h) {
  if (!h) return SFB_ERR_ARG;
  delete h;
  return SFB_OK;
}

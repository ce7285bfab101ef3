// One class drawn for each row of logits (sfb_sample in sfb.h).
//
// A cluster of up to eight CTAs has a row.  The row is read once, into shared memory (what does not fit there is read again), and then
// gone over as often as the filters want:
//   1. the largest logit m and the first place that has it (all that a greedy answer takes)
//   2. (top-k, top-p) how many logits lie in each 1/32 of (m - z) / T below 32: 1024 counts
//   3. (top-k) counts of ordered keys within the part of 2 that holds the k-th largest, until a bin is a single key
//   4. (top-p) bounds on the sums of weights by 2 say within which keys the nucleus ends; the weights of these are summed by key until a
//      bin is a single key
//   5. sums of the weights that are kept by warp, whose shares of the row follow one another: prefix sums say which warp the random
//      number falls on, and that warp goes over its share once more
// A filter's result is a key and how many of the logits with that key are kept, the first ones: all filters keep a beginning of the
// order by falling logit and rising index.
//
// Whole numbers come out: a class is right or wrong.  So the weights exp((z - m) / T) are taken in 64 bits (an error of 1e-7 in a sum over
// 325,000 classes would move one draw in a hundred to the class beside), by a table of 64 powers of two and a polynomial of the fourth
// degree: ten operations, 4e-14.  Sums by key are whole numbers (2^-F of the largest weight), so that their order changes nothing; the
// others are added in a fixed order.
//
// Bound by HBM (the row, once) where little is kept, by the 64-bit unit where all classes are weighed: 0.16 cycles an SM and class.
#include <algorithm>
#include <cmath>
#include <new>

#include "sfb_elem.cuh"

namespace {

using sfb::pdl_launch_dependents;
using sfb::pdl_wait;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 1024, kEach = kBins / kThreads;
constexpr float kPerUnit = 32.f;             // bins of 2 in a factor e
constexpr float kFar = 45.f;                 // weights below e^-45 of the largest count as zero: all of them together are below 1e-13
constexpr int kMaxCtas = 8;

struct SampleParams {
  const void* z;
  int64_t ldz, classes;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t *ids, *kept;
  float* logp;
  int32_t ctas, share, resident;             // of a row; vectors of 16 bytes that a CTA has at most, and that its shared memory holds
  int32_t fraction;                          // F
  bool wide;
};

template <typename T> struct Type;
template <> struct Type<float> { static constexpr int kLow = 0; };           // bits of an fp32 word that such a value leaves zero
template <> struct Type<__nv_bfloat16> { static constexpr int kLow = 16; };
template <> struct Type<__half> { static constexpr int kLow = 13; };

constexpr float kNone = -INFINITY;

// Ordered like the values.
template <int LOW>
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return (u >> 31 ? ~u : u | 0x80000000u) >> LOW;
}
template <int LOW>
__device__ __forceinline__ float value_of(uint32_t key) {
  const uint32_t u = key << LOW;
  return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~(u | ((1u << LOW) - 1)));
}

struct Shared {
  union {
    uint32_t count[kBins];
    unsigned long long mass[kBins];
  };
  double power[64];                          // 2^(j / 64)
  double scan[kWarps];                       // (also of the other types that are scanned)
  unsigned long long best;                   // of this CTA: key of the largest, ~ its index
  unsigned long long warp_best[kWarps];
  double above, all;                         // of this CTA: weights above the keys looked at; all kept ones
  uint32_t above_count;
  double warp_above[kWarps], warp_all[kWarps];
  uint32_t warp_count[kWarps];
  double sum[kWarps];                        // of this CTA's warps: what is kept, but for the last key, of which there are `ties`
  uint32_t ties[kWarps], keeps[kWarps];
  uint32_t found[2];
  double found_at;
  // the row's warps, in their order
  double upto[kMaxCtas * kWarps];
  uint32_t ties_ahead[kMaxCtas * kWarps];
  double total;
  uint32_t kept;
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
__device__ __forceinline__ double read(const double* here, int cta) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(remote(here, cta)) : "memory");
  return v;
}
// All of the row's threads.
__device__ __forceinline__ void row_sync(int ctas) {
  if (ctas == 1) __syncthreads();
  else asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// exp((z - m) / T).
struct Weight {
  const double* power;
  double m, per;                             // 64 log2(e) / T
  float top, far;                            // m, and below which weights are zero
  __device__ __forceinline__ double operator()(float z) const {
    // t = (z - m) per = k + f, |f| <= 1/2: the sum with 1.5 * 2^52 leaves k in the low bits
    const double d = static_cast<double>(z) - m;
    const double shifted = fma(d, per, 6755399441055744.0);
    const int k = __double2loint(shifted);
    const double f = fma(d, per, -(shifted - 6755399441055744.0));
    // 2^(f / 64): (ln 2 / 64)^j / j!
    constexpr double c1 = 0.6931471805599453 / 64, c2 = c1 * c1 / 2, c3 = c2 * c1 / 3, c4 = c3 * c1 / 4;
    const double s = power[k & 63], e = fma(fma(fma(fma(c4, f, c3), f, c2), f, c1), f, 1.0);
    const double r = s * e;
    const double w = __hiloint2double(__double2hiint(r) + ((k >> 6) << 20), __double2loint(r));
    return z == top ? 1.0 : z < far ? 0.0 : w;
  }
};

template <typename V>
__device__ __forceinline__ V shuffle_up(V v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }

// What lies in the threads before this one; the whole in `all`.
template <typename V>
__device__ __forceinline__ V block_scan(Shared& s, V value, V& all) {
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
  V ahead = 0, whole = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w == warp) ahead = whole;
    whole += part[w];
  }
  __syncthreads();
  all = whole;
  return ahead + sum - value;
}

// A CTA's share of a row.
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
  // No numbers count as minus infinity, and -0 as 0.
  static __device__ __forceinline__ void widen(const uint4& w, float (&v)[kV]) {
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int j = 0; j < kV; ++j) v[j] = fmaxf(sfb::to_float(e[j]), kNone) + 0.f;
  }
  __device__ __forceinline__ void values(int i, float (&v)[kV]) const { widen(i < resident ? held[i] : fetch(i), v); }
};

// Calls f(z) for the logits of a warp's vectors.
template <typename T, typename F>
__device__ __forceinline__ void each(const Slice<T>& s, int from, int to, F&& f) {
  for (int i = from + (threadIdx.x & 31); i < to; i += 32) {
    float v[Slice<T>::kV];
    s.values(i, v);
#pragma unroll
    for (int j = 0; j < Slice<T>::kV; ++j) f(v[j]);
  }
}

__device__ __forceinline__ uint32_t warp_sum(uint32_t v) { return __reduce_add_sync(0xffffffffu, v); }
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A range of keys and what lies above it.
struct Range { uint32_t low, high; };

// The keys that bins [first, last] can hold (and some more beside them: the bins were found in 32 bits).
template <int LOW>
__device__ __forceinline__ Range range_of(float m, double unit, int first, int last) {
  Range r{key_of<LOW>(-3.4028234663852886e38f), key_of<LOW>(m)};
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
__device__ __forceinline__ int shift_of(const Range& r) {
  const uint32_t width = r.high - r.low;     // the largest distance
  return width < kBins ? 0 : 32 - __clz(width) - 10;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleParams p) {
  constexpr int LOW = Type<T>::kLow, kV = Slice<T>::kV;
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ Shared s;
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < 64) s.power[threadIdx.x] = exp2(threadIdx.x / 64.0);
  pdl_wait();

  const int64_t row = blockIdx.x / p.ctas;
  const int cta = blockIdx.x % p.ctas;
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

  // 1. the row comes in
  unsigned long long best = 0;               // (minus infinity, which is above key 0, has no place)
  {
    float most = kNone;
    int at = -1;
    for (int i = from + lane; i < to; i += 4 * 32) {
      uint4 w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (i + 32 * q < to) w[q] = slice.fetch(i + 32 * q);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (i + 32 * q >= to) break;
        if (i + 32 * q < slice.resident) slice.held[i + 32 * q] = w[q];
        float v[kV];
        Slice<T>::widen(w[q], v);
#pragma unroll
        for (int j = 0; j < kV; ++j)
          if (v[j] > most) {
            most = v[j];
            at = (i + 32 * q) * kV + j;
          }
      }
    }
    if (at >= 0) best = static_cast<unsigned long long>(key_of<LOW>(most)) << 32 | ~static_cast<uint32_t>(first + at);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) s.warp_best[warp] = best;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) best = max(best, s.warp_best[w]);
    if (p.ctas > 1) {
      if (threadIdx.x == 0) s.best = best;
      row_sync(p.ctas);
      for (int c = 0; c < p.ctas; ++c) best = max(best, read(&s.best, c));
    }
  }
  const float temperature = p.temperature ? p.temperature[row] : 1.f;
  const int32_t top_k = p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f;
  const double min_p = p.min_p ? fmin(1.0, fmax(0.0, static_cast<double>(p.min_p[row]))) : 0.0;
  if (best == 0 || !(temperature > 0.f) || top_k == 1 || top_p <= 0.f) {      // nothing to draw from, or nothing to draw
    if (cta == 0 && threadIdx.x == 0) {
      p.ids[row] = best ? static_cast<int32_t>(~static_cast<uint32_t>(best)) : -1;
      if (p.logp) p.logp[row] = best ? 0.f : kNone;
      if (p.kept) p.kept[row] = best ? 1 : 0;
    }
    row_sync(p.ctas);                        // (no CTA leaves while another reads its shared memory)
    return;
  }
  const float m = value_of<LOW>(static_cast<uint32_t>(best >> 32));
  const Weight weight{s.power, m, 92.33248261893196 / temperature, m,
                      isinf(m) ? m : m - kFar * temperature};                // 64 log2(e)
  const double unit = static_cast<double>(temperature) / kPerUnit;

  uint32_t last_key = 0, last_ties = 0xffffffffu;        // of what is kept: all above the key, and so many that have it
  if (top_k > 0 || top_p < 1.f) {
    // 2. counts by distance
    for (int b = threadIdx.x; b < kBins; b += kThreads) s.count[b] = 0;
    __syncthreads();
    const float scale = fminf(kPerUnit / temperature, 1e30f);
    each(slice, from, to, [&](float z) {
      if (z == kNone) return;
      const float x = z == m ? 0.f : isinf(m) ? kBins : fminf(m - z, 3.4028234663852886e38f) * scale;
      atomicAdd(&s.count[min(static_cast<int>(fminf(x, kBins - 1.f)), kBins - 1)], 1u);
    });
    row_sync(p.ctas);
    uint32_t count[kEach] = {}, before[kEach], mine = 0, finite;
    for (int c = 0; c < p.ctas; ++c)
#pragma unroll
      for (int j = 0; j < kEach; ++j) count[j] += read(&s.count[threadIdx.x * kEach + j], c);
#pragma unroll
    for (int j = 0; j < kEach; ++j) mine += count[j];
    before[0] = block_scan(s, mine, finite);
#pragma unroll
    for (int j = 1; j < kEach; ++j) before[j] = before[j - 1] + count[j - 1];
    if (threadIdx.x == 0) s.found[0] = 0;
    row_sync(p.ctas);                        // the counts are read

    // 3. the k-th largest
    const bool cuts = top_k > 0 && static_cast<uint32_t>(top_k) < finite;
    const uint32_t k = cuts ? static_cast<uint32_t>(top_k) : finite;
    if (cuts) {
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (before[j] < k && before[j] + count[j] >= k) s.found[0] = threadIdx.x * kEach + j;
      __syncthreads();
      Range r = range_of<LOW>(m, unit, s.found[0], s.found[0]);
      for (;;) {
        const int shift = shift_of(r);
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) s.count[b] = 0;
        if (threadIdx.x == 0) s.found[0] = 0, s.found[1] = 1;
        __syncthreads();
        uint32_t above = 0;
        each(slice, from, to, [&](float z) {
          const uint32_t key = key_of<LOW>(z);
          if (z == kNone || key < r.low) return;
          if (key > r.high) ++above;
          else atomicAdd(&s.count[(r.high - key) >> shift], 1u);
        });
        above = warp_sum(above);
        if (lane == 0) s.warp_count[warp] = above;
        row_sync(p.ctas);
        uint32_t some[kEach] = {}, a = 0, whole, sum = 0;
        for (int c = 0; c < p.ctas; ++c) {
#pragma unroll
          for (int j = 0; j < kEach; ++j) some[j] += read(&s.count[threadIdx.x * kEach + j], c);
          a += warp_sum(lane < kWarps ? read(&s.warp_count[lane], c) : 0u);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) sum += some[j];
        a += block_scan(s, sum, whole);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          if (a < k && a + some[j] >= k) {
            s.found[0] = threadIdx.x * kEach + j;
            s.found[1] = k - a;
          }
          a += some[j];
        }
        row_sync(p.ctas);                    // all is read, and found
        const uint32_t high = r.high - (s.found[0] << shift), span = (1u << shift) - 1;
        if (shift == 0) {
          last_key = high;
          last_ties = s.found[1];
          break;
        }
        r = Range{max(r.low, high > span ? high - span : 0u), high};
      }
    }

    // 4. the nucleus.  With S the sum of the weights, it ends in the first bin up to which they come to top_p S, or behind which
    // (1 - top_p) S or less is left.  A bin's weights lie within a factor of e^(1/32): what bins up to, or behind, which these sums have bounds.
    if (top_p < 1.f) {
      double low = 0.0, high = 0.0, all_low, all_high, bin_low[kEach], bin_high[kEach];
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int b = threadIdx.x * kEach + j;
        const uint32_t c = before[j] < k ? min(count[j], k - before[j]) : 0;
        bin_low[j] = b < kBins - 1 ? c * static_cast<double>(expf(-(b + 1) / kPerUnit)) : 0.0;
        bin_high[j] = c * static_cast<double>(expf(-b / kPerUnit));
        low += bin_low[j];
        high += bin_high[j];
      }
      low = block_scan(s, low, all_low);
      high = block_scan(s, high, all_high);
      __syncthreads();
      if (threadIdx.x == 0) s.found[0] = s.found[1] = kBins - 1;
      __syncthreads();
      const double share = top_p, rest = 1.0 - share, slack = 1e-5;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const uint32_t b = threadIdx.x * kEach + j;
        low += bin_low[j];
        high += bin_high[j];
        const bool early = high * (1 + slack) < share * all_low || (all_low - low) * (1 - slack) > rest * all_high;
        const bool enough = low * (1 - slack) >= share * all_high || (all_high - high) * (1 + slack) <= rest * all_low;
        if (!early) atomicMin(&s.found[0], b);
        if (enough) atomicMin(&s.found[1], b);
      }
      __syncthreads();
      Range r = range_of<LOW>(m, unit, s.found[0], max(s.found[0], s.found[1]));
      r.low = max(r.low, last_key);
      r.high = max(r.high, r.low);
      const uint32_t cut_key = last_key, cut_ties = last_ties;       // of top-k; key 0: none
      const double cut_weight = cuts ? weight(value_of<LOW>(cut_key)) : 0.0;
      const double grain = ldexp(1.0, p.fraction), back = ldexp(1.0, -p.fraction);
      double target = 0.0;
      for (bool begins = true;; begins = false) {
        const int shift = shift_of(r);
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) s.mass[b] = 0;
        if (threadIdx.x == 0) s.found[0] = kBins, s.found[1] = 0;
        __syncthreads();
        double above = 0.0, all = 0.0;
        each(slice, from, to, [&](float z) {
          const uint32_t key = key_of<LOW>(z);
          if (z == kNone || key <= cut_key || (!begins && key < r.low)) return;
          const double w = weight(z);
          all += w;
          if (key > r.high) above += w;
          else if (key >= r.low) atomicAdd(&s.mass[(r.high - key) >> shift], static_cast<unsigned long long>(__double2ll_rn(w * grain)));
        });
        above = warp_sum(above);
        all = warp_sum(all);
        if (lane == 0) s.warp_above[warp] = above, s.warp_all[warp] = all;
        row_sync(p.ctas);
        unsigned long long some[kEach] = {}, sum = 0, whole;
        above = all = 0.0;
        for (int c = 0; c < p.ctas; ++c) {
#pragma unroll
          for (int j = 0; j < kEach; ++j) some[j] += read(&s.mass[threadIdx.x * kEach + j], c);
          above += warp_sum(lane < kWarps ? read(&s.warp_above[lane], c) : 0.0);
          if (begins) all += warp_sum(lane < kWarps ? read(&s.warp_all[lane], c) : 0.0);
        }
        if (begins) target = share * (all + (cuts ? cut_ties * cut_weight : 0.0));
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          if (cuts && cut_key >= r.low && cut_key <= r.high && (r.high - cut_key) >> shift == threadIdx.x * kEach + j)
            some[j] += cut_ties * static_cast<unsigned long long>(__double2ll_rn(cut_weight * grain));
          sum += some[j];
        }
        const unsigned long long ahead = block_scan(s, sum, whole);
        unsigned long long upto = ahead;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          upto += some[j];
          if (some[j]) atomicMax(&s.found[1], threadIdx.x * kEach + j);
          if (some[j] && above + upto * back >= target) atomicMin(&s.found[0], threadIdx.x * kEach + j);
        }
        __syncthreads();
        const uint32_t bin = s.found[0] < kBins ? s.found[0] : s.found[1];   // (rounding may leave the target just beyond the last one)
        if (bin / kEach == threadIdx.x) {
          upto = ahead;
#pragma unroll
          for (int j = 0; j < kEach; ++j)
            if (threadIdx.x * kEach + j < bin) upto += some[j];
          s.found_at = above + upto * back;
        }
        row_sync(p.ctas);                    // all is read, and found
        const uint32_t top = r.high - (bin << shift), span = (1u << shift) - 1;
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

  // 5. the draw
  const double last_weight = last_key ? weight(value_of<LOW>(last_key)) : 0.0;
  if (last_weight < min_p) last_ties = 0;
  {
    double sum = 0.0;
    uint32_t keeps = 0, ties = 0;
    each(slice, from, to, [&](float z) {
      const uint32_t key = key_of<LOW>(z);
      if (z == kNone || key < last_key) return;
      if (key == last_key) {
        ++ties;
        return;
      }
      const double w = weight(z);
      if (w < min_p) return;
      sum += w;
      ++keeps;
    });
    sum = warp_sum(sum);
    keeps = warp_sum(keeps);
    ties = warp_sum(ties);
    if (lane == 0) s.sum[warp] = sum, s.keeps[warp] = keeps, s.ties[warp] = ties;
  }
  row_sync(p.ctas);
  const double u = fmax(0.0, static_cast<double>(p.u[row]));
  if (warp == 0) {                           // the row's warps, a few of them a lane
    constexpr int kMost = kMaxCtas * kWarps / 32;
    const int each_lane = (p.ctas * kWarps + 31) / 32;
    double sum[kMost], mine = 0.0;
    uint32_t ties[kMost], mine_ties = 0, kept = 0;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      const int i = lane * each_lane + j, c = i / kWarps;
      const bool there = j < each_lane && c < p.ctas;
      sum[j] = there ? read(&s.sum[i % kWarps], c) : 0.0;
      ties[j] = there ? read(&s.ties[i % kWarps], c) : 0u;
      kept += there ? read(&s.keeps[i % kWarps], c) : 0u;
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
    const double target = u * total;
    int found = 0x7fffffff, last = -1;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      const int i = lane * each_lane + j;
      if (j < each_lane && i < p.ctas * kWarps) {
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
    const double total = s.total, target = u * total;
    double upto = s.upto[winner];
    uint32_t seen = s.ties_ahead[winner];
    int at = -1, last_at = -1;               // of the slice
    double w_at = 0.0, last_w = 0.0;
    for (int i0 = from; i0 < to; i0 += 32) {
      const int i = i0 + lane;
      float v[kV];
      double w[kV], sum = 0.0;
      uint32_t ties = 0;
      if (i < to) slice.values(i, v);
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        if (i >= to) v[j] = kNone;
        if (v[j] != kNone && key_of<LOW>(v[j]) == last_key) ++ties;
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
        const uint32_t key = key_of<LOW>(v[j]);
        w[j] = 0.0;
        if (v[j] == kNone || key < last_key) continue;
        if (key == last_key) {
          if (ahead++ < last_ties) w[j] = last_weight;
        } else {
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
  row_sync(p.ctas);                          // (no CTA leaves while another reads its shared memory)
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

constexpr int kHeldMost = 200 << 10;         // of a CTA's shared memory, for the row
constexpr int kHeldTwo = 96 << 10;           // ... where two CTAs are to share an SM

template <typename T>
cudaError_t launch(SampleParams p, int64_t n, cudaStream_t s) {
  const int64_t vectors = (p.classes * static_cast<int64_t>(sizeof(T)) + 15) / 16;
  // As many CTAs a row as leave room for two of them on an SM; more where there are few rows and enough of each.
  int ctas = 1;
  while (ctas < kMaxCtas && (vectors * 16 > static_cast<int64_t>(kHeldTwo) * ctas || (n * ctas < sfb::kModelSms && vectors * 16 > (16 << 10) * ctas))) ctas *= 2;
  p.ctas = ctas;
  p.share = static_cast<int32_t>((vectors + ctas - 1) / ctas);
  p.resident = std::min(p.share, kHeldMost / 16);
  const cudaError_t e = sfb::allow_smem<sample_kernel<T>>(kHeldMost);
  return e == cudaSuccess ? sfb::launch_kernel(sample_kernel<T>, dim3(static_cast<unsigned>(n * ctas)), dim3(kThreads), static_cast<size_t>(p.resident) * 16, s, ctas, p) : e;
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

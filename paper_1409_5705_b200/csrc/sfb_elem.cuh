// What the element-wise operators share: groups of eight entries of fp32, bf16 or fp16, the generator of the dropout, and the host side
// of a handle.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sfb_internal.h"

namespace sfb {

// ---- eight entries --------------------------------------------------------------------------------------------------------------
// A group is the unit of all of these operators: 16 bytes of a 16-bit type, and what one call of the generator decides.
constexpr int kGroup = 8;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// A group as it lies in memory, so that several loads are under way before the first is used.
template <typename T> struct Raw { uint4 w[sizeof(T) / 2]; };

template <typename T>
__device__ __forceinline__ void unpack(const Raw<T>& r, float (&v)[kGroup]) {
  const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
  for (int j = 0; j < kGroup; ++j) v[j] = to_float(e[j]);
}
template <typename T>
__device__ __forceinline__ void pack(const float (&v)[kGroup], Raw<T>& r) {
  T* e = reinterpret_cast<T*>(&r);
#pragma unroll
  for (int j = 0; j < kGroup; ++j) e[j] = from_float<T>(v[j]);
}
// The first `count` (1 .. 8) entries at p, the rest zeros; 16 bytes at a time where the rows lie so (`wide`) and the group is whole.
// (Plain loads: an operator in place writes what it has read.)
template <typename T>
__device__ __forceinline__ void load_group(const T* p, int count, bool wide, Raw<T>& r) {
  if (wide && count == kGroup) {
#pragma unroll
    for (int q = 0; q < static_cast<int>(sizeof(T) / 2); ++q) r.w[q] = reinterpret_cast<const uint4*>(p)[q];
  } else {
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int j = 0; j < kGroup; ++j) e[j] = j < count ? p[j] : from_float<T>(0.f);
  }
}
template <typename T>
__device__ __forceinline__ void store_group(T* p, int count, bool wide, const Raw<T>& r) {
  if (wide && count == kGroup) {
#pragma unroll
    for (int q = 0; q < static_cast<int>(sizeof(T) / 2); ++q) reinterpret_cast<uint4*>(p)[q] = r.w[q];
  } else {
    const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
      if (j < count) p[j] = e[j];
  }
}

inline int64_t groups_of(int64_t cols) { return (cols + kGroup - 1) / kGroup; }
inline size_t size_of(int32_t dtype) { return dtype == SFB_F32 ? 4 : 2; }
inline bool is_dtype(int32_t dtype) { return dtype >= SFB_F32 && dtype <= SFB_F16; }
// Whether rows of that pitch from p on all start on a 16-byte boundary.
inline bool lies_wide(const void* p, int64_t pitch, int32_t dtype) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(pitch) * size_of(dtype)) & 15u) == 0;
}
inline bool lies_aligned(const void* p, int32_t dtype) { return (reinterpret_cast<uintptr_t>(p) & (size_of(dtype) - 1)) == 0; }

// ---- division of numbers below 2^31 by one that a launch knows: floor(n / d) = floor(n m / 2^(31 + l)) with l = ceil(log2 d) and
// m = floor(2^(31 + l) / d) + 1, since 0 < m d - 2^(31 + l) <= d <= 2^l ------------------------------------------------------------
struct Divisor {
  uint32_t d, m, shift;
  Divisor() = default;
  explicit Divisor(uint32_t by) : d(by), m(0), shift(0) {
    if (by <= 1) return;
    int l = 0;
    while ((1u << l) < by) ++l;
    m = static_cast<uint32_t>(((1ull << (31 + l)) / by) + 1);
    shift = static_cast<uint32_t>(l - 1);
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return m ? __umulhi(n, m) >> shift : n; }
};

#ifdef __CUDACC__
// ---- the generator: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) --------------
// Ten rounds of two 32 x 32 -> 64-bit products; 128 bits, which eight entries share by 16.
__device__ __forceinline__ uint4 philox(uint4 c, uint2 k) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = static_cast<uint64_t>(0xD2511F53u) * c.x, b = static_cast<uint64_t>(0xCD9E8D57u) * c.z;
    c = make_uint4(static_cast<uint32_t>(b >> 32) ^ c.y ^ k.x, static_cast<uint32_t>(b), static_cast<uint32_t>(a >> 32) ^ c.w ^ k.y,
                   static_cast<uint32_t>(a));
    k.x += 0x9E3779B9u;
    k.y += 0xBB67AE85u;
  }
  return c;
}
#endif

// What a kernel takes of a dropout: an entry is kept where its 16 bits are at least `threshold`.
struct DropParams {
  const uint64_t* rng;                 // seed, offset; device memory
  uint64_t call;                       // added to the offset
  uint32_t threshold;                  // round(65536 p), 0 .. 65536
  uint32_t last;                       // 65536 threshold - 1, where that is not 0
  float factor;                        // 65536 / (65536 - threshold); 0 where nothing is kept
};

#ifdef __CUDACC__
// Called by whole warps.
struct Generator {
  uint2 key{}, offset{};
  __device__ __forceinline__ void begin(const DropParams& p) {
    const uint64_t seed = p.rng[0], at = p.rng[1] + p.call;
    key = make_uint2(same(static_cast<uint32_t>(seed)), same(static_cast<uint32_t>(seed >> 32)));
    offset = make_uint2(same(static_cast<uint32_t>(at)), same(static_cast<uint32_t>(at >> 32)));
  }
  // A value that is the same in all lanes, known to be: what follows from it alone is computed once a warp.
  static __device__ __forceinline__ uint32_t same(uint32_t v) { return __reduce_or_sync(0xffffffffu, v); }
  // Zeroes the dropped ones of a group's entries (whatever they are: infinities and NaN too).  `last`: (threshold << 16) - 1, which 16 bits
  // on top of a word exceed where they are at least the threshold, whatever lies below them.
  __device__ __forceinline__ void drop(float (&v)[kGroup], uint32_t row, uint32_t group, uint32_t last) const {
    const uint4 w = philox(make_uint4(group, row, offset.x, offset.y), key);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = (u[j] << 16) > last ? v[2 * j] : 0.f;
      v[2 * j + 1] = u[j] > last ? v[2 * j + 1] : 0.f;
    }
  }
};
#endif

// ---- handles -----------------------------------------------------------------------------------------------------------------------
struct OnDevice {                            // the handle's device is current for the length of a call
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

// The current device, or an error code where it is not one of compute capability 10.x.
inline int this_device(int* dev) {
  int major = 0;
  if (cudaGetDevice(dev) != cudaSuccess) return SFB_ERR_CUDA;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev) != cudaSuccess) return SFB_ERR_CUDA;
  return major == 10 ? SFB_OK : SFB_ERR_ARCH;
}

}  // namespace sfb

// The state of a dropout's handle, which the lookup's kernels take too.
struct sfb_dropout {
  sfb::DropParams drop;
  cudaStream_t stream;
  int device;
  int last_cuda;
};

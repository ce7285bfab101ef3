// Global norm of a list of gradient tensors, and their copies rescaled where it is above a limit (sfb_clip_* in sfb.h).
//
// The table, made once: pieces of at most 16 KB of a tensor, each with its addresses, entries and type, so that tensors of any
// number and length are one even list.  Two launches:
//   clip_sum_kernel    blocks take pieces in turn; a thread's squares go into fp64 sums, a block's sum to its place
//   clip_scale_kernel  every block adds the blocks' sums in the same order, and takes its pieces from the list's end backwards: what
//                      the first pass read last is still in L2
// Squares and sums in fp64, so the norm and the factor are those of 64 bits but for their last rounding.
// Bound by HBM: one read for the norm, one read and one write for the copies, less what L2 holds of the second read.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <vector>

#include "sfb_internal.h"

namespace {

using sfb::pdl_launch_dependents;
using sfb::pdl_wait;

constexpr int kThreads = 256;
constexpr int64_t kPieceBytes = 16384;               // four 16-byte loads a thread
// Blocks an SM.  (The sum's squares in fp64 want more threads than its loads do: us with 4, 6 and 8 of its blocks, 500 M fp32 1,030, 1,011 and 1,022;
// 40 M of three types 57.1, 55.5 and 55.0; 21 M bf16 25.7, 24.8 and 25.8.)
constexpr int kSumBlocks = 6, kScaleBlocks = 4;

struct Piece {
  const char* src;
  char* dst;
  int32_t count;
  int32_t dtype;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// The entries of 16 bytes.
__device__ __forceinline__ void widen(const uint4& w, float (&v)[4], const float*) {
  v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ void widen(const uint4& w, float (&v)[8], const __nv_bfloat16*) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(u[j] << 16);
    v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(const uint4& w, float (&v)[8], const __half*) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[j]));
    v[2 * j] = f.x;
    v[2 * j + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 narrow(const float (&v)[4], const float*) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint32_t two(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ uint32_t two(__half2 v) { return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ uint4 narrow(const float (&v)[8], const __nv_bfloat16*) {
  return make_uint4(two(__floats2bfloat162_rn(v[0], v[1])), two(__floats2bfloat162_rn(v[2], v[3])), two(__floats2bfloat162_rn(v[4], v[5])),
                    two(__floats2bfloat162_rn(v[6], v[7])));
}
__device__ __forceinline__ uint4 narrow(const float (&v)[8], const __half*) {
  return make_uint4(two(__floats2half2_rn(v[0], v[1])), two(__floats2half2_rn(v[2], v[3])), two(__floats2half2_rn(v[4], v[5])),
                    two(__floats2half2_rn(v[6], v[7])));
}

// The squares of entries of up to 32 bits are exact in fp64.  Two sums, so that a thread does not wait for each addition.
template <int N>
__device__ __forceinline__ void add_squares(const float (&v)[N], double (&sum)[2]) {
#pragma unroll
  for (int j = 0; j < N; ++j) sum[j & 1] = fma(static_cast<double>(v[j]), static_cast<double>(v[j]), sum[j & 1]);
}

// Entries [0, n) of a piece: up to the first 16-byte boundary and behind the last one singly, the rest 16 bytes at a time, four of
// them under way.
template <typename T>
__device__ __forceinline__ void sum_piece(const T* p, int n, double (&sum)[2]) {
  constexpr int kV = 16 / sizeof(T);
  const int lead = min(n, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(T)));
  const int vecs = (n - lead) / kV;
  for (int i = threadIdx.x; i < lead; i += kThreads) { const float v[1] = {to_f(p[i])}; add_squares(v, sum); }
  for (int i = lead + vecs * kV + threadIdx.x; i < n; i += kThreads) { const float v[1] = {to_f(p[i])}; add_squares(v, sum); }
  const uint4* q = reinterpret_cast<const uint4*>(p + lead);
  for (int i = threadIdx.x; i < vecs; i += 4 * kThreads) {
    uint4 w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = i + u * kThreads < vecs ? q[i + u * kThreads] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {                    // (what lies behind the last one is zero)
      float v[kV];
      widen(w[u], v, static_cast<const T*>(nullptr));
      add_squares(v, sum);
    }
  }
}

// dst = coef * src, or src bit for bit where coef is 1; the two may be the same addresses.  Where they lie differently to a 16-byte boundary,
// entry by entry.
template <typename T>
__device__ __forceinline__ void scale_piece(const T* src, T* dst, int n, float coef) {
  constexpr int kV = 16 / sizeof(T);
  const int lead = min(n, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) & 15) / sizeof(T)));
  const bool same = ((reinterpret_cast<uintptr_t>(src) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0;
  const int vecs = (n - lead) / kV;
  const bool copy = coef == 1.f;
  auto scaled = [&](T v) { return copy ? v : from_f<T>(to_f(v) * coef); };
  for (int i = threadIdx.x; i < lead; i += kThreads) dst[i] = scaled(src[i]);
  for (int i = lead + vecs * kV + threadIdx.x; i < n; i += kThreads) dst[i] = scaled(src[i]);
  uint4* d = reinterpret_cast<uint4*>(dst + lead);
  if (!same) {
    for (int i = threadIdx.x; i < vecs * kV; i += kThreads) dst[lead + i] = scaled(src[lead + i]);
    return;
  }
  const uint4* q = reinterpret_cast<const uint4*>(src + lead);
  for (int i = threadIdx.x; i < vecs; i += 4 * kThreads) {
    uint4 w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * kThreads < vecs) w[u] = __ldcs(q + i + u * kThreads);          // (not read again, nor what is written)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u * kThreads >= vecs) break;
      if (!copy) {
        float v[kV];
        widen(w[u], v, static_cast<const T*>(nullptr));
#pragma unroll
        for (int j = 0; j < kV; ++j) v[j] *= coef;
        w[u] = narrow(v, static_cast<const T*>(nullptr));
      }
      __stcs(d + i + u * kThreads, w[u]);
    }
  }
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += part[w];
  __syncthreads();
  return s;
}

__global__ void __launch_bounds__(kThreads, kSumBlocks) clip_sum_kernel(const Piece* pieces, int64_t n, double* part) {
  pdl_launch_dependents();
  pdl_wait();
  double sums[2] = {};
  Piece next = blockIdx.x < n ? pieces[blockIdx.x] : Piece{};
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const Piece c = next;
    if (i + gridDim.x < n) next = pieces[i + gridDim.x];
    if (c.dtype == SFB_F32) sum_piece(reinterpret_cast<const float*>(c.src), c.count, sums);
    else if (c.dtype == SFB_BF16) sum_piece(reinterpret_cast<const __nv_bfloat16*>(c.src), c.count, sums);
    else sum_piece(reinterpret_cast<const __half*>(c.src), c.count, sums);
  }
  const double sum = block_sum(sums[0] + sums[1]);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The sum of `parts` values, the same in every block: each thread some of them in their order, then block_sum.
__device__ __forceinline__ double total_of(const double* part, int parts) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
  return block_sum(s);
}

__global__ void __launch_bounds__(kThreads) clip_total_kernel(const double* part, int parts, double* sum) {
  pdl_launch_dependents();
  pdl_wait();
  const double s = total_of(part, parts);
  if (threadIdx.x == 0) *sum = s;
}

__global__ void __launch_bounds__(kThreads, kScaleBlocks) clip_scale_kernel(const Piece* pieces, int64_t n, const double* part, int parts, float max_norm,
                                                              float* result) {
  pdl_launch_dependents();
  pdl_wait();
  const double norm = sqrt(total_of(part, parts));
  const bool finite = isfinite(norm);
  const float coef = finite && norm > static_cast<double>(max_norm) ? static_cast<float>(static_cast<double>(max_norm) / norm) : 1.f;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    result[0] = static_cast<float>(norm);
    result[1] = finite ? coef : 0.f;
  }
  Piece next = n > blockIdx.x ? pieces[n - 1 - blockIdx.x] : Piece{};
  for (int64_t i = n - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
    const Piece c = next;
    if (i >= gridDim.x) next = pieces[i - gridDim.x];
    if (coef == 1.f && c.src == c.dst) continue;
    if (c.dtype == SFB_F32) scale_piece(reinterpret_cast<const float*>(c.src), reinterpret_cast<float*>(c.dst), c.count, coef);
    else if (c.dtype == SFB_BF16)
      scale_piece(reinterpret_cast<const __nv_bfloat16*>(c.src), reinterpret_cast<__nv_bfloat16*>(c.dst), c.count, coef);
    else scale_piece(reinterpret_cast<const __half*>(c.src), reinterpret_cast<__half*>(c.dst), c.count, coef);
  }
}

constexpr int kMaxParts = 148 * 16;          // blocks of the sum, at most

int64_t piece_entries(int32_t dtype) { return kPieceBytes / (dtype == SFB_F32 ? 4 : 2); }

// The pieces of all tensors, or an error code.
int64_t count_pieces(int64_t tensors, const int64_t* counts, const int32_t* dtypes) {
  if (tensors < 0 || (tensors > 0 && (!counts || !dtypes))) return SFB_ERR_ARG;
  int64_t n = 0;
  for (int64_t t = 0; t < tensors; ++t) {
    if (dtypes[t] < SFB_F32 || dtypes[t] > SFB_F16) return SFB_ERR_ARG;
    if (counts[t] < 0 || counts[t] > (1LL << 46)) return SFB_ERR_SHAPE;
    n += (counts[t] + piece_entries(dtypes[t]) - 1) / piece_entries(dtypes[t]);
    if (n > (1LL << 32)) return SFB_ERR_SHAPE;
  }
  return n;
}

// Whether some dst lies over another tensor's src or dst, or over its own src by a part: its entries would be scaled twice, or be
// changed before they are read.
struct Span { uintptr_t lo, hi; int64_t t; };
bool overlapping(int64_t tensors, const void* const* src, void* const* dst, const int64_t* counts, const int32_t* dtypes) {
  std::vector<Span> to, from;
  to.reserve(tensors);
  from.reserve(tensors);
  for (int64_t t = 0; t < tensors; ++t) {
    if (counts[t] == 0) continue;
    const uintptr_t s = reinterpret_cast<uintptr_t>(src[t]), d = dst ? reinterpret_cast<uintptr_t>(dst[t]) : s;
    const uintptr_t bytes = static_cast<uintptr_t>(counts[t]) * (dtypes[t] == SFB_F32 ? 4 : 2);
    from.push_back(Span{s, s + bytes, t});
    to.push_back(Span{d, d + bytes, t});
  }
  std::sort(to.begin(), to.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
  for (size_t i = 1; i < to.size(); ++i)
    if (to[i].lo < to[i - 1].hi) return true;
  for (const Span& f : from) {                       // the dsts do not overlap: those over f follow one another
    auto it = std::upper_bound(to.begin(), to.end(), f.lo, [](uintptr_t v, const Span& a) { return v < a.hi; });
    for (; it != to.end() && it->lo < f.hi; ++it)
      if (it->t != f.t || it->lo != f.lo) return true;
  }
  return false;
}

constexpr size_t kPartBytes = static_cast<size_t>(kMaxParts) * 8;

}  // namespace

struct sfb_clip {
  char* ws;
  int64_t pieces;
  int blocks;
  cudaStream_t stream;
  int device;
  int last_cuda;
};

namespace {

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

int fail(sfb_clip* h, cudaError_t e) {
  h->last_cuda = static_cast<int>(e);
  return SFB_ERR_CUDA;
}

int launch_sum(sfb_clip* h) {
  const cudaError_t e = sfb::launch_kernel(clip_sum_kernel, dim3(h->blocks), dim3(kThreads), 0, h->stream, 1,
                                           reinterpret_cast<const Piece*>(h->ws + kPartBytes), h->pieces, reinterpret_cast<double*>(h->ws));
  return e == cudaSuccess ? SFB_OK : fail(h, e);
}

int launch_scale(sfb_clip* h, float max_norm, const double* part, int parts, float* result) {
  const unsigned blocks = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(h->pieces, sfb::sm_count() * kScaleBlocks)));
  const cudaError_t e = sfb::launch_kernel(clip_scale_kernel, dim3(blocks), dim3(kThreads), 0, h->stream, 1,
                                           reinterpret_cast<const Piece*>(h->ws + kPartBytes), h->pieces, part, parts, max_norm, result);
  return e == cudaSuccess ? SFB_OK : fail(h, e);
}

}  // namespace

extern "C" int sfb_clip_workspace_bytes(int64_t tensors, const int64_t* counts, const int32_t* dtypes, size_t* out_bytes) {
  if (!out_bytes) return SFB_ERR_ARG;
  const int64_t n = count_pieces(tensors, counts, dtypes);
  if (n < 0) return static_cast<int>(n);
  *out_bytes = kPartBytes + static_cast<size_t>(n) * sizeof(Piece);
  return SFB_OK;
}

extern "C" int sfb_clip_init(int64_t tensors, const void* const* src, void* const* dst, const int64_t* counts, const int32_t* dtypes,
                             void* workspace_dev, size_t workspace_bytes, void* stream, sfb_clip** out) {
  if (!out) return SFB_ERR_ARG;
  *out = nullptr;
  size_t need = 0;
  const int rc = sfb_clip_workspace_bytes(tensors, counts, dtypes, &need);
  if (rc) return rc;
  if (!workspace_dev || (tensors > 0 && !src)) return SFB_ERR_ARG;
  for (int64_t t = 0; t < tensors; ++t) {
    const uintptr_t s = reinterpret_cast<uintptr_t>(src[t]), d = dst ? reinterpret_cast<uintptr_t>(dst[t]) : s;
    if (counts[t] > 0 && (!s || !d)) return SFB_ERR_ARG;
    if ((s | d) & (dtypes[t] == SFB_F32 ? 3u : 1u)) return SFB_ERR_ALIGN;
  }
  if (reinterpret_cast<uintptr_t>(workspace_dev) & 15u) return SFB_ERR_ALIGN;
  if (workspace_bytes < need) return SFB_ERR_WORKSPACE;
  try {
    if (overlapping(tensors, src, dst, counts, dtypes)) return SFB_ERR_ARG;
  } catch (const std::exception&) {
    return SFB_ERR_ARG;
  }
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SFB_ERR_CUDA;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return SFB_ERR_CUDA;
  if (major != 10) return SFB_ERR_ARCH;
  sfb_clip* h = nullptr;
  try {
    std::vector<Piece> table;
    table.reserve((need - kPartBytes) / sizeof(Piece));
    for (int64_t t = 0; t < tensors; ++t) {
      const int64_t most = piece_entries(dtypes[t]), size = dtypes[t] == SFB_F32 ? 4 : 2;
      for (int64_t at = 0; at < counts[t]; at += most)
        table.push_back(Piece{static_cast<const char*>(src[t]) + at * size,
                              (dst ? static_cast<char*>(dst[t]) : static_cast<char*>(const_cast<void*>(src[t]))) + at * size,
                              static_cast<int32_t>(std::min(most, counts[t] - at)), dtypes[t]});
    }
    h = new sfb_clip();
    h->ws = static_cast<char*>(workspace_dev);
    h->pieces = static_cast<int64_t>(table.size());
    h->blocks = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(h->pieces, std::min(sfb::sm_count() * kSumBlocks, kMaxParts))));
    h->stream = static_cast<cudaStream_t>(stream);
    h->device = dev;
    h->last_cuda = 0;
    if (!table.empty()) {
      cudaError_t e = cudaMemcpyAsync(h->ws + kPartBytes, table.data(), table.size() * sizeof(Piece), cudaMemcpyHostToDevice, h->stream);
      if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
      if (e != cudaSuccess) { delete h; return SFB_ERR_CUDA; }
    }
  } catch (const std::exception&) {
    delete h;
    return SFB_ERR_ARG;
  }
  *out = h;
  return SFB_OK;
}

extern "C" int sfb_clip_sum(sfb_clip* h, double* sum_dev) {
  if (!h || !sum_dev) return SFB_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(sum_dev) & 7u) return SFB_ERR_ALIGN;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  const int rc = launch_sum(h);
  if (rc) return rc;
  const cudaError_t e = sfb::launch_kernel(clip_total_kernel, dim3(1), dim3(kThreads), 0, h->stream, 1,
                                           reinterpret_cast<const double*>(h->ws), h->blocks, sum_dev);
  return e == cudaSuccess ? SFB_OK : fail(h, e);
}

extern "C" int sfb_clip_scale(sfb_clip* h, float max_norm, const double* sum_dev, float* result_dev) {
  if (!h || !sum_dev || !result_dev || !(max_norm >= 0.f)) return SFB_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(sum_dev) & 7u) || (reinterpret_cast<uintptr_t>(result_dev) & 3u)) return SFB_ERR_ALIGN;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  return launch_scale(h, max_norm, sum_dev, 1, result_dev);
}

extern "C" int sfb_clip_gradients(sfb_clip* h, float max_norm, float* result_dev) {
  if (!h || !result_dev || !(max_norm >= 0.f)) return SFB_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(result_dev) & 3u) return SFB_ERR_ALIGN;
  const OnDevice on(h->device);
  if (on.err != cudaSuccess) return fail(h, on.err);
  const int rc = launch_sum(h);
  return rc ? rc : launch_scale(h, max_norm, reinterpret_cast<const double*>(h->ws), h->blocks, result_dev);
}

extern "C" int sfb_clip_last_cuda_error(sfb_clip* h) { return h ? h->last_cuda : 0; }

extern "C" int sfb_clip_destroy(sfb_clip* h) {
  if (!h) return SFB_ERR_ARG;
  delete h;
  return SFB_OK;
}

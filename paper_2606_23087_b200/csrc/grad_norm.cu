// The 2-norm over a list of gradients, and the factor that brings it down to a limit.
//
//   norm = sqrt(sum over all elements of g^2),  factor = norm > max_norm ? max_norm / norm : 1
//
// Bound by HBM: every element is read once.  117 M fp32 elements 71 us (6.6 TB/s), with eight CTAs an SM instead of six 81, with four 73 to 77;
// any alignment alike.  A thread squares and adds the elements of a chunk in fp32 and the chunks in fp64; where a
// chunk's sum is outside the numbers whose squares fp32 holds to full precision it takes the chunk's squares in fp64 too.  CTA i owns
// the i-th line of the workspace, and the join adds the lines in a fixed order: no atomics, the same bits on every run of a device.
#include <algorithm>
#include <cmath>

#include "operators.cuh"

namespace ft {

constexpr int kGradThreads = 256;
constexpr uint32_t kGradVecs = 4;                                  // 16-byte accesses of a thread a chunk
constexpr uint32_t kGradChunk = kGradThreads * kGradVecs * 16;     // bytes
constexpr uint32_t kGradPerLaunch = 320;                           // tensors a launch takes at most (kernel arguments hold 32 KiB)
constexpr uint32_t kGradFew = 16;                                  // tensors of the launch with a small argument block
constexpr uint32_t kGradCtasPerSm = 6;
constexpr uint32_t kGradLines = 2048;                              // of the workspace, at most

struct GradTensorArg {
  const void* p;       // on a 16-byte boundary, at or before the tensor's first element
  uint64_t first, end; // bytes from p on that the tensor has
  uint64_t chunk0;     // chunks of the tensors before this one
  uint32_t bf16;
};
template <uint32_t kCap>
struct GradArgs {
  uint64_t chunks;
  double* lines;
  uint32_t n, add;  // add: to what the lines hold
  GradTensorArg t[kCap];
};

template <typename T>
__device__ __forceinline__ float squares(const uint4 (&v)[kGradVecs]) {
  F2 s[2] = {f2(0.f), f2(0.f)};
#pragma unroll
  for (uint32_t i = 0; i < kGradVecs; ++i) {
    F2 x[Pack<T>::kElems / 2];
    Pack<T>::widen(v[i], x);
#pragma unroll
    for (int j = 0; j < Pack<T>::kElems / 2; ++j) s[j & 1] = fma(x[j], x[j], s[j & 1]);
  }
  return sum(s[0] + s[1]);
}
template <typename T>
__device__ __noinline__ double squares_in_double(uint4 v) {
  float x[Pack<T>::kElems];
  Pack<T>::widen(v, x);
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < Pack<T>::kElems; ++j) s = ::fma((double)x[j], (double)x[j], s);
  return s;
}

// this thread's share of a chunk of a tensor
template <typename T>
__device__ __forceinline__ double grad_chunk(const GradTensorArg& t, uint64_t at) {
  uint4 v[kGradVecs];
#pragma unroll
  for (uint32_t i = 0; i < kGradVecs; ++i) {
    const uint64_t b = at + i * (kGradThreads * 16);
    const uint8_t* p = static_cast<const uint8_t*>(t.p) + b;
    v[i] = make_uint4(0, 0, 0, 0);
    if (b >= t.first && b + 16 <= t.end) {
      v[i] = *reinterpret_cast<const uint4*>(p);
    } else if (b + 16 > t.first && b < t.end) {  // the tensor's ends: no byte outside it is read
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (uint32_t j = 0; j < 16; j += sizeof(T)) {
        if (b + j < t.first || b + j >= t.end) continue;
        if constexpr (sizeof(T) == 4) w[j / 4] = *reinterpret_cast<const uint32_t*>(p + j);
        else w[j / 4] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + j) << 8 * (j % 4);
      }
      v[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  const float s = squares<T>(v);
  if (s > 0x1p-80f && s < 0x1p100f) return s;
  uint32_t any = 0;
#pragma unroll
  for (uint32_t i = 0; i < kGradVecs; ++i) any |= v[i].x | v[i].y | v[i].z | v[i].w;
  double d = 0.0;
  if (any)
    for (uint32_t i = 0; i < kGradVecs; ++i) d += squares_in_double<T>(v[i]);
  return d;
}

__device__ __forceinline__ double block_sum_double(double x) {  // for thread 0
  __shared__ double part[32];
#pragma unroll
  for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  if (threadIdx.x == 0)
    for (uint32_t w = 1; w < blockDim.x / 32; ++w) x += part[w];
  return x;
}

template <uint32_t kCap>
__global__ void __launch_bounds__(kGradThreads, kGradCtasPerSm) k_grad_squares(const __grid_constant__ GradArgs<kCap> a) {
  let_next_start();
  after_previous();
  double s = 0.0;
  // a contiguous share of the chunks
  const uint64_t c0 = a.chunks * blockIdx.x / gridDim.x, c1 = a.chunks * (blockIdx.x + 1) / gridDim.x;
  uint32_t lo = 0, hi = a.n;  // the last tensor whose first chunk is not behind c0
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (a.t[mid].chunk0 <= c0) lo = mid; else hi = mid;
  }
  for (uint64_t c = c0; c < c1; ++c) {
    while (lo + 1 < a.n && a.t[lo + 1].chunk0 <= c) ++lo;
    const GradTensorArg& t = a.t[lo];
    const uint64_t at = (c - t.chunk0) * kGradChunk + threadIdx.x * 16;
    s += t.bf16 ? grad_chunk<__nv_bfloat16>(t, at) : grad_chunk<float>(t, at);
  }
  s = block_sum_double(s);
  if (threadIdx.x == 0) a.lines[blockIdx.x] = a.add ? a.lines[blockIdx.x] + s : s;
}

__global__ void __launch_bounds__(kGradThreads) k_grad_join(const double* lines, uint32_t n, const double* more, double* sumsq, float* norm,
                                                           float* factor, double max_norm) {
  after_previous();
  double s = 0.0;
  for (uint32_t i = threadIdx.x; i < n; i += kGradThreads) s += lines[i];
  s = block_sum_double(s);
  if (threadIdx.x) return;
  if (more) s += *more;
  if (sumsq) *sumsq = s;
  const double r = sqrt(s);
  if (norm) *norm = (float)r;
  if (factor) *factor = r > max_norm ? (float)(max_norm / r) : r == r ? 1.f : (float)r;
}

template <uint32_t kCap>
static cudaError_t grad_squares(const ft_grad_tensor* t, uint32_t n, uint32_t grid, uint64_t chunks, double* lines, bool add, cudaStream_t st) {
  GradArgs<kCap> a;
  a.chunks = chunks;
  a.lines = lines;
  a.n = 0;
  a.add = add;
  uint64_t at = 0;
  for (uint32_t i = 0; i < n; ++i) {
    if (t[i].n == 0) continue;
    GradTensorArg& d = a.t[a.n++];
    d.first = reinterpret_cast<uintptr_t>(t[i].grad) & 15;
    d.p = static_cast<const uint8_t*>(t[i].grad) - d.first;
    d.end = d.first + t[i].n * dtype_size(t[i].dtype);
    d.chunk0 = at;
    d.bf16 = t[i].dtype == FT_BF16;
    at += (d.end + kGradChunk - 1) / kGradChunk;
  }
  return launch_chained(k_grad_squares<kCap>, dim3(grid), kGradThreads, 0, st, a);
}

static uint32_t grad_grid(const ft_pool* p) { return std::min<uint32_t>(kGradLines, kGradCtasPerSm * (uint32_t)p->sm_count); }

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_grad_norm_workspace(ft_pool* p, uint64_t* bytes) {
  if (!p || !bytes) return FT_ERR_INVALID_ARG;
  *bytes = grad_grid(p) * sizeof(double);
  return FT_OK;
}

FT_EXPORT int32_t pool_grad_norm(ft_pool* p, const ft_grad_tensor* tensors, uint32_t n_tensors, double max_norm, const double* more,
                                 double* sumsq, float* norm, float* factor, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (n_tensors && !tensors) return FT_ERR_INVALID_ARG;
  for (uint32_t i = 0; i < n_tensors; ++i) {
    const ft_grad_tensor& t = tensors[i];
    if (!dtype_ok(t.dtype)) return FT_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    if (!t.grad || !aligned_to(t.grad, dtype_size(t.dtype))) return FT_ERR_INVALID_ARG;
    if (t.n > (1ull << 40)) return FT_ERR_CAPACITY;
  }
  if ((factor && !(max_norm >= 0.0)) || !aligned_to(more, 8) || !aligned_to(sumsq, 8) || !aligned_to(norm, 4) || !aligned_to(factor, 4)) return FT_ERR_INVALID_ARG;
  if (!workspace || !aligned_to(workspace, 256)) return FT_ERR_INVALID_ARG;
  const uint32_t most = grad_grid(p);
  if (workspace_bytes < most * sizeof(double)) return FT_ERR_CAPACITY;
  double* lines = static_cast<double*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const auto chunks_of = [](const ft_grad_tensor& t) {
    return t.n ? ((reinterpret_cast<uintptr_t>(t.grad) & 15) + t.n * dtype_size(t.dtype) + kGradChunk - 1) / kGradChunk : 0;
  };
  uint64_t all = 0;
  for (uint32_t i = 0; i < n_tensors; ++i) all += chunks_of(tensors[i]);
  // every launch takes as many CTAs: those after the first add to its lines
  const uint32_t grid = (uint32_t)std::min<uint64_t>(most, all);
  bool add = false;
  for (uint32_t i0 = 0; i0 < n_tensors;) {
    uint32_t i1 = i0, used = 0;
    uint64_t chunks = 0;
    for (; i1 < n_tensors && used < kGradPerLaunch; ++i1) {
      const uint64_t c = chunks_of(tensors[i1]);
      chunks += c;
      used += c != 0;
    }
    if (chunks) {
      FT_CUDA(used <= kGradFew ? (grad_squares<kGradFew>(tensors + i0, i1 - i0, grid, chunks, lines, add, st))
                               : (grad_squares<kGradPerLaunch>(tensors + i0, i1 - i0, grid, chunks, lines, add, st)));
      p->gpu_launches += 1;
      add = true;
    }
    i0 = i1;
  }
  FT_CUDA(launch_chained(k_grad_join, dim3(1), kGradThreads, 0, st, static_cast<const double*>(lines), grid, more, sumsq, norm, factor, max_norm));
  p->gpu_launches += 1;
  return FT_OK;
}

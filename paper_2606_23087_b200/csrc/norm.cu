// Layer norm over the rows of a matrix, forward and backward.
//
//   forward    mean = sum(x) / c,  var = sum((x - mean)^2) / c,  rstd = (var + eps)^-1/2,  y = (x - mean) rstd w + b
//   backward   xhat = (x - mean) rstd,  a = w dy,
//              dx = rstd (a - sum(a)/c - xhat sum(a xhat)/c),  dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// Both are bound by HBM: a row is read once (two rows backward) and written once, with a dozen operations an element.
//
//   k_norm          a CTA holds one row at a time in registers: the variance is taken about the mean, not from a difference
//                   of sums.  16-byte chunks of the following rows are on their way into shared memory meanwhile
//   k_norm_grad     the same walk; a thread always owns the same columns, so the sums over rows stay in its registers
//                   until the CTA has seen its last row.  No atomics: partial sums go to the workspace, one line a CTA
//   k_norm_join     adds the lines of partial sums in line order
//   k_norm_wide, k_norm_grad_sums, k_norm_grad_cols   rows too long for a CTA's registers
#include <algorithm>
#include <cmath>

#include "operators.cuh"

namespace ft {

struct NormArgs {
  uint64_t rows, ldx, ldy;
  uint32_t cols, param_dtype;
  const void *x, *weight, *bias;
  void* y;
  float *mean, *rstd;
  float eps;
};

struct NormGradArgs {
  uint64_t rows, lddy, ldx, lddx;
  uint32_t cols, param_dtype;
  const void *dy, *x, *weight;
  const float *mean, *rstd;
  void* dx;
  float* partial;  // [lines][2][cols]
};

constexpr int kNormMaxThreads = 512;
// Rows in shared memory or under way to it: four, or two where the backward pass holds two operands of 64 bytes a thread
// (four stages of those would take 256 KiB at 512 threads).
template <int kOperands, int V>
constexpr int kNormStages = kOperands * V <= 4 ? 4 : 2;

// sum over the block of N values a thread; every thread gets them.  `red` is one of two buffers used in turn: a buffer
// is written again only behind the barrier of the other one's use.
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float (*red)[kNormMaxThreads / 32]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  const int nw = blockDim.x >> 5;
  if (nw == 1) return;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) red[i][threadIdx.x >> 5] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float s = red[i][0];
    for (int w = 1; w < nw; ++w) s += red[i][w];
    v[i] = s;
  }
}

// Rows as this thread sees them: chunk k of thread t holds the E elements from (k * blockDim + t) * E on.  With 16-byte
// chunks (kVec) a row travels through a ring of kStages rows in shared memory, filled by asynchronous copies that the
// same thread issues and waits for, so the ring needs no barrier.  Otherwise (odd widths, odd strides) E = 1 and the
// chunks come straight into registers.
template <typename T, int V, bool kVec, int kStages>
struct RowRing {
  static constexpr int E = kVec ? Pack<T>::kElems : 1;
  const T* base;
  uint64_t ld, rows;
  uint32_t cols;
  uint4* ring;  // [kStages][V][blockDim], kVec only

  __device__ __forceinline__ uint32_t at(int k) const { return (k * blockDim.x + threadIdx.x) * E; }
  __device__ __forceinline__ void fetch(uint64_t row, uint32_t stage) {
    if constexpr (kVec) {
      if (row < rows) {
        const T* p = base + row * ld;
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (at(k) < cols) copy16_async(ring + (stage * V + k) * blockDim.x + threadIdx.x, p + at(k));
      }
    }
  }
  __device__ __forceinline__ void take(uint64_t row, uint32_t stage, float (&f)[V * E]) const {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (at(k) < cols) {
        if constexpr (kVec) Pack<T>::widen(ring[(stage * V + k) * blockDim.x + threadIdx.x], f + k * E);
        else f[k] = widen1(base[row * ld + at(k)]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) f[k * E + e] = 0.f;
      }
    }
  }
  __device__ __forceinline__ void store(void* out, uint64_t row, uint64_t ldo, const float (&f)[V * E]) const {
    T* p = static_cast<T*>(out) + row * ldo;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (at(k) < cols) {
        if constexpr (kVec) *reinterpret_cast<uint4*>(p + at(k)) = Pack<T>::narrow(f + k * E);
        else p[at(k)] = narrow1<T>(f[k]);
      }
    }
  }
};

template <typename T, int V, bool kVec>
__global__ void __launch_bounds__(kNormMaxThreads) k_norm(NormArgs a) {
  extern __shared__ __align__(16) uint4 ring[];
  __shared__ float red[2][1][kNormMaxThreads / 32];
  constexpr int kStages = kNormStages<1, V>;
  using Ring = RowRing<T, V, kVec, kStages>;
  constexpr int E = Ring::E, N = V * E;
  Ring in{static_cast<const T*>(a.x), a.ldx, a.rows, a.cols, ring};
  const uint64_t step = gridDim.x;
  uint64_t row = blockIdx.x;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) { in.fetch(row + s * step, s); copy_async_commit(); }
  float w[N], b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t c = in.at(i / E) + i % E;
    w[i] = c < a.cols ? (a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f) : 0.f;
    b[i] = c < a.cols && a.bias ? load_as(a.bias, a.param_dtype, c) : 0.f;
  }
  uint32_t stage = 0;
  for (; row < a.rows; row += step) {
    in.fetch(row + (kStages - 1) * step, (stage + kStages - 1) % kStages);
    copy_async_commit();
    copy_async_wait<kStages - 1>();
    float x[N];
    in.take(row, stage, x);
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) s[0] += x[i];
    block_sum(s, red[0]);
    const float mean = s[0] / a.cols;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] -= mean;
      if (in.at(i / E) < a.cols) s[0] += x[i] * x[i];
    }
    block_sum(s, red[1]);
    const float rstd = rsqrtf(s[0] / a.cols + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = x[i] * rstd * w[i] + b[i];
    in.store(a.y, row, a.ldy, x);
    stage = (stage + 1) % kStages;
  }
}

template <typename T, int V, bool kVec>
__global__ void __launch_bounds__(kNormMaxThreads) k_norm_grad(NormGradArgs a) {
  extern __shared__ __align__(16) uint4 ring[];
  __shared__ float red[2][2][kNormMaxThreads / 32];
  constexpr int kStages = kNormStages<2, V>;
  using Ring = RowRing<T, V, kVec, kStages>;
  constexpr int E = Ring::E, N = V * E;
  Ring in_x{static_cast<const T*>(a.x), a.ldx, a.rows, a.cols, ring};
  Ring in_g{static_cast<const T*>(a.dy), a.lddy, a.rows, a.cols, ring + kStages * V * blockDim.x};
  const uint64_t step = gridDim.x;
  uint64_t row = blockIdx.x;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    in_x.fetch(row + s * step, s); in_g.fetch(row + s * step, s);
    copy_async_commit();
  }
  float w[N], dw[N], db[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t c = in_x.at(i / E) + i % E;
    w[i] = c < a.cols ? (a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f) : 0.f;
    dw[i] = db[i] = 0.f;
  }
  uint32_t stage = 0;
  for (; row < a.rows; row += step) {
    in_x.fetch(row + (kStages - 1) * step, (stage + kStages - 1) % kStages);
    in_g.fetch(row + (kStages - 1) * step, (stage + kStages - 1) % kStages);
    copy_async_commit();
    copy_async_wait<kStages - 1>();
    const float mean = a.mean[row], rstd = a.rstd[row];
    float x[N], g[N];
    in_x.take(row, stage, x);
    in_g.take(row, stage, g);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = in_x.at(i / E) < a.cols ? (x[i] - mean) * rstd : 0.f;
      dw[i] += g[i] * x[i];
      db[i] += g[i];
      g[i] *= w[i];
      s[0] += g[i];
      s[1] += g[i] * x[i];
    }
    block_sum(s, red[stage & 1]);
    const float c0 = s[0] / a.cols, c1 = s[1] / a.cols;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = rstd * (g[i] - c0 - x[i] * c1);
    in_x.store(a.dx, row, a.lddx, x);
    stage = (stage + 1) % kStages;
  }
  float* line = a.partial + (uint64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t c = in_x.at(i / E) + i % E;
    if (c < a.cols) { line[c] = dw[i]; line[a.cols + c] = db[i]; }
  }
}

// dw and db from the lines of partial sums: 32 columns a CTA, eight warps over the lines, joined in a fixed order
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(32 * kJoinWarps) k_norm_join(const float* __restrict__ partial, uint32_t lines, uint32_t cols,
                                                               float* dweight, float* dbias, uint32_t accumulate) {
  __shared__ float part[kJoinWarps][32];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;  // column of [dw | db]
  float s = 0.f;
  if (c < 2ull * cols)
    for (uint32_t l = warp; l < lines; l += kJoinWarps) s += partial[(uint64_t)l * 2 * cols + c];
  part[warp][lane] = s;
  __syncthreads();
  if (warp || c >= 2ull * cols) return;
#pragma unroll
  for (int w = 1; w < kJoinWarps; ++w) s += part[w][lane];
  float* out = c < cols ? dweight : dbias;
  if (!out) return;
  const uint64_t i = c < cols ? c : c - cols;
  out[i] = accumulate ? out[i] + s : s;
}

// ---- rows beyond a CTA's registers: every pass reads the row again (from L2, a row at a time a CTA) ----------------

template <typename T>
__global__ void __launch_bounds__(kNormMaxThreads) k_norm_wide(NormArgs a) {
  __shared__ float red[2][1][kNormMaxThreads / 32];
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    float s[1] = {0.f};
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) s[0] += widen1(x[c]);
    block_sum(s, red[0]);
    const float mean = s[0] / a.cols;
    s[0] = 0.f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) { const float d = widen1(x[c]) - mean; s[0] += d * d; }
    block_sum(s, red[1]);
    const float rstd = rsqrtf(s[0] / a.cols + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float w = a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f, b = a.bias ? load_as(a.bias, a.param_dtype, c) : 0.f;
      y[c] = narrow1<T>((widen1(x[c]) - mean) * rstd * w + b);
    }
  }
}

// sums[row] = (sum(a), sum(a xhat)) / cols
template <typename T>
__global__ void __launch_bounds__(kNormMaxThreads) k_norm_grad_sums(NormGradArgs a, float2* sums) {
  __shared__ float red[2][2][kNormMaxThreads / 32];
  uint32_t turn = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const T *x = static_cast<const T*>(a.x) + row * a.ldx, *dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f};
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float g = widen1(dy[c]) * (a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f);
      s[0] += g;
      s[1] += g * ((widen1(x[c]) - mean) * rstd);
    }
    block_sum(s, red[turn]);
    if (threadIdx.x == 0) sums[row] = make_float2(s[0] / a.cols, s[1] / a.cols);
  }
}

// CTA (column block, line): its columns of the rows line, line + lines, ...
template <typename T>
__global__ void __launch_bounds__(256) k_norm_grad_cols(NormGradArgs a, const float2* __restrict__ sums) {
  const uint64_t c = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= a.cols) return;
  const float w = a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f;
  float dw = 0.f, db = 0.f;
  for (uint64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float g = widen1(static_cast<const T*>(a.dy)[row * a.lddy + c]), mean = a.mean[row], rstd = a.rstd[row];
    const float xhat = (widen1(static_cast<const T*>(a.x)[row * a.ldx + c]) - mean) * rstd;
    const float2 s = sums[row];
    dw += g * xhat;
    db += g;
    static_cast<T*>(a.dx)[row * a.lddx + c] = narrow1<T>(rstd * (g * w - s.x - xhat * s.y));
  }
  float* line = a.partial + (uint64_t)blockIdx.y * 2 * a.cols;
  line[c] = dw;
  line[a.cols + c] = db;
}

// ---- launch geometry ----------------------------------------------------------------------------------------------

constexpr uint32_t kNormHeld = 16;  // elements of a row a thread holds at most
constexpr uint32_t kNormMaxCols = kNormHeld * kNormMaxThreads;
constexpr uint32_t kNormMaxLines = 1024;  // lines of partial sums: the grid of the backward kernel at most
constexpr uint32_t kNormWideLines = 64;
constexpr uint32_t kNormColsLimit = 1u << 30;  // column counters are 32-bit

struct NormShape {
  uint32_t threads, chunks;  // chunks a thread
  bool vec;
};

// A row in 16-byte chunks where every row of every operand starts on a 16-byte boundary, else element by element.
static NormShape norm_shape(uint32_t cols, bool vec, uint32_t elems, bool few_rows) {
  NormShape s;
  s.vec = vec;
  const uint32_t n = vec ? cols / elems : cols, most = vec ? kNormHeld / elems : kNormHeld;
  s.chunks = 1;
  while (s.chunks < most && (n + s.chunks - 1) / s.chunks > (few_rows ? kNormMaxThreads : 128u)) s.chunks *= 2;
  s.threads = ((n + s.chunks - 1) / s.chunks + 31) / 32 * 32;
  return s;
}

template <typename T, typename F>
static void with_chunks(const NormShape& s, F&& f) {
  if (s.vec) {
    switch (s.chunks) {
      case 1: f(std::integral_constant<int, 1>{}, std::true_type{}); return;
      case 2: f(std::integral_constant<int, 2>{}, std::true_type{}); return;
      default:
        if constexpr (Pack<T>::kElems == 4) f(std::integral_constant<int, 4>{}, std::true_type{});
        return;
    }
  }
  switch (s.chunks) {
    case 1: f(std::integral_constant<int, 1>{}, std::false_type{}); return;
    case 2: f(std::integral_constant<int, 2>{}, std::false_type{}); return;
    case 4: f(std::integral_constant<int, 4>{}, std::false_type{}); return;
    case 8: f(std::integral_constant<int, 8>{}, std::false_type{}); return;
    default: f(std::integral_constant<int, 16>{}, std::false_type{}); return;
  }
}

template <typename K>
static cudaError_t ctas_per_sm(K kernel, uint32_t threads, size_t smem, int* n) {
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(n, kernel, (int)threads, smem);
  *n = std::max(1, *n);
  return e;
}

template <typename T>
static cudaError_t norm_launch(const ft_pool* p, const NormArgs& a, bool vec, cudaStream_t st) {
  if (a.cols > kNormMaxCols) {
    k_norm_wide<T><<<(unsigned)std::min<uint64_t>(a.rows, 4ull * p->sm_count), kNormMaxThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  const NormShape s = norm_shape(a.cols, vec, Pack<T>::kElems, a.rows <= (uint64_t)p->sm_count);
  cudaError_t e = cudaSuccess;
  with_chunks<T>(s, [&](auto v, auto is_vec) {
    auto kernel = k_norm<T, decltype(v)::value, decltype(is_vec)::value>;
    const size_t smem = s.vec ? (size_t)kNormStages<1, decltype(v)::value> * s.chunks * s.threads * 16 : 0;
    int per_sm = 1;
    if ((e = ctas_per_sm(kernel, s.threads, smem, &per_sm)) != cudaSuccess) return;
    kernel<<<(unsigned)std::min<uint64_t>(a.rows, (uint64_t)per_sm * p->sm_count), s.threads, smem, st>>>(a);
    e = cudaGetLastError();
  });
  return e;
}

template <typename T>
static cudaError_t norm_grad_launch(const ft_pool* p, const NormGradArgs& a, bool vec, float2* sums, uint32_t* lines, cudaStream_t st) {
  if (a.cols > kNormMaxCols) {
    k_norm_grad_sums<T><<<(unsigned)std::min<uint64_t>(a.rows, 4ull * p->sm_count), kNormMaxThreads, 0, st>>>(a, sums);
    *lines = (uint32_t)std::min<uint64_t>(a.rows, kNormWideLines);
    k_norm_grad_cols<T><<<dim3((a.cols + 255u) / 256u, *lines), 256, 0, st>>>(a, sums);
    return cudaGetLastError();
  }
  const NormShape s = norm_shape(a.cols, vec, Pack<T>::kElems, a.rows <= (uint64_t)p->sm_count);
  cudaError_t e = cudaSuccess;
  with_chunks<T>(s, [&](auto v, auto is_vec) {
    auto kernel = k_norm_grad<T, decltype(v)::value, decltype(is_vec)::value>;
    const size_t smem = s.vec ? 2ull * kNormStages<2, decltype(v)::value> * s.chunks * s.threads * 16 : 0;
    int per_sm = 1;
    if ((e = ctas_per_sm(kernel, s.threads, smem, &per_sm)) != cudaSuccess) return;
    *lines = (uint32_t)std::min<uint64_t>(std::min<uint64_t>(a.rows, (uint64_t)per_sm * p->sm_count), kNormMaxLines);
    kernel<<<*lines, s.threads, smem, st>>>(a);
    e = cudaGetLastError();
  });
  return e;
}

// bytes of the backward pass's workspace: the lines of partial sums, and for wide rows two numbers a row
static uint64_t norm_grad_ws(const ft_pool* p, uint64_t rows, uint32_t cols) {
  const bool wide = cols > kNormMaxCols;
  const uint64_t lines = wide ? kNormWideLines : std::min<uint64_t>(std::min<uint64_t>(rows, 16ull * p->sm_count), kNormMaxLines);
  return align_up_sz(lines * 2 * cols * sizeof(float), 256) + (wide ? rows * sizeof(float2) : 0);
}

static bool rows_in_16(const void* p, uint64_t ld, uint32_t es) { return aligned_to(p, 16) && ld * es % 16 == 0; }

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_layer_norm(ft_pool* p, uint64_t rows, uint32_t cols, const void* x, uint64_t ldx, uint32_t dtype, const void* weight,
                                  const void* bias, uint32_t param_dtype, float eps, void* y, uint64_t ldy, float* mean, float* rstd,
                                  void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (cols == 0 || !dtype_ok(dtype) || !dtype_ok(param_dtype) || !(eps >= 0.f) || std::isinf(eps)) return FT_ERR_INVALID_ARG;
  if (cols > kNormColsLimit) return FT_ERR_CAPACITY;
  if (rows == 0) return FT_OK;
  const uint32_t es = dtype_size(dtype), ps = dtype_size(param_dtype);
  if (!x || !y || ldx < cols || ldy < cols || !aligned_to(x, es) || !aligned_to(y, es)) return FT_ERR_INVALID_ARG;
  if (!aligned_to(weight, ps) || !aligned_to(bias, ps) || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return FT_ERR_INVALID_ARG;
  NormArgs a;
  a.rows = rows; a.ldx = ldx; a.ldy = ldy; a.cols = cols; a.param_dtype = param_dtype;
  a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.mean = mean; a.rstd = rstd; a.eps = eps;
  const bool vec = cols * es % 16 == 0 && rows_in_16(x, ldx, es) && rows_in_16(y, ldy, es);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  FT_CUDA(dtype == FT_F32 ? norm_launch<float>(p, a, vec, st) : norm_launch<__nv_bfloat16>(p, a, vec, st));
  p->gpu_launches += 1;
  return FT_OK;
}

FT_EXPORT int32_t pool_layer_norm_grad_workspace(ft_pool* p, uint64_t rows, uint32_t cols, uint64_t* bytes) {
  if (!p || cols == 0 || !bytes) return FT_ERR_INVALID_ARG;
  if (cols > kNormColsLimit) return FT_ERR_CAPACITY;
  *bytes = rows ? norm_grad_ws(p, rows, cols) : 0;
  return FT_OK;
}

FT_EXPORT int32_t pool_layer_norm_grad(ft_pool* p, uint64_t rows, uint32_t cols, const void* dy, uint64_t lddy, const void* x, uint64_t ldx,
                                       uint32_t dtype, const void* weight, uint32_t param_dtype, const float* mean, const float* rstd,
                                       void* dx, uint64_t lddx, float* dweight, float* dbias, uint32_t accumulate, void* workspace,
                                       uint64_t workspace_bytes, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (cols == 0 || !dtype_ok(dtype) || !dtype_ok(param_dtype)) return FT_ERR_INVALID_ARG;
  if (!aligned_to(dweight, 4) || !aligned_to(dbias, 4)) return FT_ERR_INVALID_ARG;
  if (cols > kNormColsLimit) return FT_ERR_CAPACITY;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {  // sums over no rows
    if (!accumulate && dweight) FT_CUDA(cudaMemsetAsync(dweight, 0, (size_t)cols * 4, st));
    if (!accumulate && dbias) FT_CUDA(cudaMemsetAsync(dbias, 0, (size_t)cols * 4, st));
    return FT_OK;
  }
  const uint32_t es = dtype_size(dtype);
  if (!dy || !x || !mean || !rstd || !dx || lddy < cols || ldx < cols || lddx < cols) return FT_ERR_INVALID_ARG;
  if (!aligned_to(dy, es) || !aligned_to(x, es) || !aligned_to(dx, es) || !aligned_to(weight, dtype_size(param_dtype))) return FT_ERR_INVALID_ARG;
  if (!aligned_to(mean, 4) || !aligned_to(rstd, 4) || !workspace || !aligned_to(workspace, 256)) return FT_ERR_INVALID_ARG;
  if (workspace_bytes < norm_grad_ws(p, rows, cols)) return FT_ERR_CAPACITY;
  NormGradArgs a;
  a.rows = rows; a.lddy = lddy; a.ldx = ldx; a.lddx = lddx; a.cols = cols; a.param_dtype = param_dtype;
  a.dy = dy; a.x = x; a.weight = weight; a.mean = mean; a.rstd = rstd; a.dx = dx; a.partial = static_cast<float*>(workspace);
  float2* sums = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + align_up_sz((size_t)kNormWideLines * 2 * cols * sizeof(float), 256));
  const bool vec = cols * es % 16 == 0 && rows_in_16(dy, lddy, es) && rows_in_16(x, ldx, es) && rows_in_16(dx, lddx, es);
  uint32_t lines = 0;
  FT_CUDA(dtype == FT_F32 ? norm_grad_launch<float>(p, a, vec, sums, &lines, st) : norm_grad_launch<__nv_bfloat16>(p, a, vec, sums, &lines, st));
  p->gpu_launches += cols > kNormMaxCols ? 2 : 1;
  if (dweight || dbias) {
    k_norm_join<<<(unsigned)((2ull * cols + 31) / 32), 32 * kJoinWarps, 0, st>>>(a.partial, lines, cols, dweight, dbias, accumulate);
    FT_CUDA(cudaGetLastError());
    p->gpu_launches += 1;
  }
  return FT_OK;
}

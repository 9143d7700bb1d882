// Layer norm over the rows of a matrix, forward and backward.
//
//   forward    mean = sum(x) / c,  var = sum((x - mean)^2) / c,  rstd = (var + eps)^-1/2,  y = (x - mean) rstd w + b
//   backward   xhat = (x - mean) rstd,  a = w dy,
//              dx = rstd (a - sum(a)/c - xhat sum(a xhat)/c),  dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// Both are bound by HBM: a row is read once (two rows backward) and written once, with a dozen operations an element.  32768 rows x
// 3584 in bf16: forward 83 to 90 us (5.2 to 5.7 TB/s; 60 % of the issue slots), backward 122 to 129 us (5.5 to 5.8 TB/s, 7 us of it for joining
// the lines).  Rows off 16-byte boundaries go element by element: 127 and 198 us in bf16, 94 and 124 for half the rows in fp32.
//
//   k_norm          a few warps (one for rows up to 4096 elements, where there are rows enough) hold a row in registers: the
//                   variance is taken about the mean, not from a difference of sums
//   k_norm_grad     groups of warps hold a row each; a thread always owns the same columns, so the sums over rows stay in
//                   its registers until its last row, while 16-byte chunks of the following rows are on their way into
//                   shared memory.  No atomics: partial sums go to the workspace, one line a CTA
//   k_norm_join     adds the lines of partial sums in line order
//   k_norm_wide, k_norm_grad_sums, k_norm_grad_cols   rows too long for that: forward beyond 16384 elements, backward beyond 8192 (4096
//                   where they are off 16 bytes), at 1 to 1.5 and 1.2 to 2 TB/s of the bytes that must move
#include <algorithm>
#include <cmath>
#include <utility>

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

// ---- forward ------------------------------------------------------------------------------------------------------

// Sum over a block of kN threads, for every thread.  `red` is one of two zeroed buffers used in turn: a buffer is written
// again only behind the barrier of the other one's use.
template <int kN>
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = warp_sum(v);
  if constexpr (kN == 32) return v;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  const float4* r = reinterpret_cast<const float4*>(red);
  v = 0.f;
#pragma unroll
  for (int w = 0; w < (kN + 127) / 128; ++w) v += (r[w].x + r[w].y) + (r[w].z + r[w].w);
  return v;
}

// rows of all that a group takes: first, first + step, ...
__device__ __forceinline__ uint32_t rows_from(uint64_t all, uint64_t first, uint64_t step) { return first < all ? (uint32_t)((all - first + step - 1) / step) : 0; }

// A thread's chunks of the rows that its group of kN threads goes through: chunk k of thread t holds the E elements from
// (k kN + t) E on.  Where the rows allow it (kVec) a chunk is 16 bytes, and the following rows' chunks are on their way into a
// ring in shared memory: a thread reads only what it has fetched itself, so the ring needs no barrier.  Otherwise a chunk is
// one element and the next row's are fetched into registers.  Where the row has no such chunk the values are zero.  kN is a
// constant, so that chunks are offsets in the instructions; a quarter of the first version's instructions were addresses.
template <typename T, int V, bool kVec, int kN, int kThreads, int kStages>
struct RowFeed {
  static constexpr int E = kVec ? Pack<T>::kElems : 1;
  const T* p;        // the thread's first chunk of the row to be fetched next
  uint64_t step;     // elements from that row to the group's next one
  uint32_t left;     // rows still to be fetched
  uint32_t chunks;   // chunks of this thread that the row has
  uint32_t slot;     // shared-memory address of this thread's places: [kStages][V][kThreads] of 16 bytes
  T next[kVec ? 1 : V];

  __device__ __forceinline__ void init(const void* base, uint64_t ld, uint64_t row, uint64_t row_step, uint32_t rows, uint32_t cols, uint32_t t, const uint4* s) {
    p = static_cast<const T*>(base) + row * ld + t * E;
    step = row_step * ld;
    left = rows;
    const uint32_t n = cols / E;
    chunks = n > t ? (n - t + kN - 1) / kN : 0;
    slot = shared_address(s);
    if constexpr (kVec) {  // chunks that the rows do not have are never fetched
#pragma unroll
      for (int i = 0; i < kStages * V; ++i)
        if (i % V >= (int)chunks) store_shared16(slot + i * kThreads * 16, make_uint4(0, 0, 0, 0));
    }
  }
  __device__ __forceinline__ bool has(int k) const { return k < (int)chunks; }
  __device__ __forceinline__ void fetch(uint32_t stage) {
    if (left == 0) return;
    --left;
    const uint32_t to = slot + stage * (V * kThreads * 16);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if constexpr (kVec) {
        if (has(k)) copy16_async(to + k * kThreads * 16, p + k * kN * E);
      } else {
        next[k] = has(k) ? p[k * kN] : narrow1<T>(0.f);
      }
    }
    p += step;
  }
  __device__ __forceinline__ void take(uint32_t stage, F2 (&f)[V * E / 2]) const {
    const uint32_t from = slot + stage * (V * kThreads * 16);
    if constexpr (kVec) {
#pragma unroll
      for (int k = 0; k < V; ++k) Pack<T>::widen(load_shared16(from + k * kThreads * 16), f + k * (E / 2));
    } else {
#pragma unroll
      for (int k = 0; k < V; k += 2) f[k / 2] = f2(widen1(next[k]), widen1(next[k + 1]));
    }
  }
  __device__ __forceinline__ void store(T* q, const F2 (&f)[V * E / 2]) const {  // q: the thread's first chunk of the output row
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (!has(k)) continue;
      if constexpr (kVec) {
        *reinterpret_cast<uint4*>(q + k * kN * E) = Pack<T>::narrow(f + k * (E / 2));
      } else {
        const float2 p = parts(f[k / 2]);
        q[k * kN] = narrow1<T>(k % 2 ? p.y : p.x);
      }
    }
  }
};

// Rows in shared memory or under way to it: four, or three where those would not fit (fp32 rows beyond 12288 columns).
template <int V, int kN>
constexpr int kNormStages = V * kN <= 3072 ? 4 : 3;
constexpr size_t kSmemMost = 227 * 1024;  // of a CTA

template <typename T, int V, bool kVec, int kN>
__global__ void __launch_bounds__(kN, kVec && V * Pack<T>::kElems <= 16 ? 896 / kN : 512 / kN) k_norm(NormArgs a) {
  extern __shared__ __align__(16) uint4 ring[];  // [kStages][V][kN]
  __shared__ __align__(16) float red[2][(kN / 32 + 3) / 4 * 4];
  constexpr int E = kVec ? Pack<T>::kElems : 1, N = V * E / 2, kStages = kNormStages<V, kN>;  // N pairs
  RowFeed<T, V, kVec, kN, kN, kStages> in;
  const uint32_t n_rows = rows_from(a.rows, blockIdx.x, gridDim.x);
  in.init(a.x, a.ldx, blockIdx.x, gridDim.x, n_rows, a.cols, threadIdx.x, ring + threadIdx.x);
  if constexpr (kVec) {
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) { in.fetch(s); copy_async_commit(); }
  } else {
    in.fetch(0);
  }
  if (kN > 32 && threadIdx.x < sizeof(red) / 4) (&red[0][0])[threadIdx.x] = 0.f;
  F2 w[N], b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float wv[2], bv[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = ((2 * i + j) / E * kN + threadIdx.x) * E + (2 * i + j) % E;
      wv[j] = c < a.cols && a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f;
      bv[j] = c < a.cols && a.bias ? load_as(a.bias, a.param_dtype, c) : 0.f;
    }
    w[i] = f2(wv[0], wv[1]);
    b[i] = f2(bv[0], bv[1]);
  }
  if (kN > 32) __syncthreads();
  const float inv = 1.f / a.cols;
  T* q = static_cast<T*>(a.y) + blockIdx.x * a.ldy + threadIdx.x * E;
  const uint64_t q_step = gridDim.x * a.ldy;
  uint32_t stage = 0;
  for (uint32_t r = 0; r < n_rows; ++r) {
    F2 x[N], s[2] = {f2(0.f), f2(0.f)};
    if constexpr (kVec) {
      in.fetch((stage + kStages - 1) % kStages);
      copy_async_commit();
      copy_async_wait<kStages - 1>();
    }
    in.take(stage, x);
    if constexpr (!kVec) in.fetch(0);
#pragma unroll
    for (int i = 0; i < N; ++i) s[i & 1] = s[i & 1] + x[i];
    const float mean = block_sum<kN>(sum(s[0] + s[1]), red[0]) * inv;
    s[0] = s[1] = f2(0.f);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = x[i] + f2(-mean);
      if constexpr (kVec) {
        if (in.has(i / (E / 2))) s[i & 1] = fma(x[i], x[i], s[i & 1]);
      } else {  // a pair is two chunks
        const float2 p = parts(x[i]);
        const F2 d = f2(in.has(2 * i) ? p.x : 0.f, in.has(2 * i + 1) ? p.y : 0.f);
        s[i & 1] = fma(d, d, s[i & 1]);
      }
    }
    const float rstd = rsqrtf(block_sum<kN>(sum(s[0] + s[1]), red[1]) * inv + a.eps);
    if (threadIdx.x == 0) {
      const uint64_t row = blockIdx.x + (uint64_t)r * gridDim.x;
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fma(x[i] * f2(rstd), w[i], b[i]);
    in.store(q, x);
    q += q_step;
    stage = (stage + 1) % kStages;
  }
}

// ---- backward -----------------------------------------------------------------------------------------------------

// Rows in shared memory or under way to it: four, or three where those would not fit.
template <int V, int kThreads>
constexpr int kGradStages = V * kThreads <= 1024 ? 4 : 3;
// Groups of n threads in a CTA, one CTA an SM: 512 threads of 128 registers, or 256 of 255 where a thread holds 32 elements.
constexpr int kGradGroups(int elems, int n) { return elems > 16 ? 256 / n : 512 / n; }

// The CTA's threads form groups of kN; group i of the grid takes the rows i, i + groups, ...
template <typename T, int V, bool kVec, int kN, int kGroups>
__global__ void __launch_bounds__(kN * kGroups, 1) k_norm_grad(NormGradArgs a) {
  extern __shared__ __align__(16) uint4 ring[];  // weights; then [2][kStages][V][kThreads], at the end the groups' sums
  constexpr int E = kVec ? Pack<T>::kElems : 1, N = V * E / 2, kThreads = kN * kGroups, kStages = kGradStages<V, kN * kGroups>, nw = kN / 32;  // N pairs
  __shared__ float2 red[2][kThreads / 32], stats[4][kThreads / 32];
  const uint32_t group = threadIdx.x / kN, t = threadIdx.x % kN;
  // The weights stay in shared memory, a thread's registers being taken by its row and its sums: by fours (pairs of single
  // elements), so that the lanes of an access read one range.
  constexpr int Q = kVec ? 4 : 2;
  float* weights = reinterpret_cast<float*>(ring);  // [V E / Q][kN][Q]
  uint4* rows = ring + V * E * kN / 4;
  for (uint32_t i = threadIdx.x; i < V * E * kN; i += kThreads) {
    const uint32_t th = i / Q % kN, e = i / Q / kN * Q + i % Q;  // the thread and which of its V E elements
    const uint32_t c = (e / E * kN + th) * E + e % E;
    weights[i] = c < a.cols ? (a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f) : 0.f;
  }
  const uint64_t step = (uint64_t)gridDim.x * kGroups, first = (uint64_t)blockIdx.x * kGroups + group;
  const uint32_t n_rows = rows_from(a.rows, first, step);
  RowFeed<T, V, kVec, kN, kThreads, kStages> in_x, in_g;
  in_x.init(a.x, a.ldx, first, step, n_rows, a.cols, t, rows + threadIdx.x);
  in_g.init(a.dy, a.lddy, first, step, n_rows, a.cols, t, rows + kStages * V * kThreads + threadIdx.x);
  // A row's two statistics come three rows ahead as well, a copy a warp (taken one row ahead they cost 25 of 160 us: each
  // row's are 4 bytes of a sector of their own).
  const uint32_t lane = threadIdx.x & 31, stat_at = shared_address(&stats[0][threadIdx.x >> 5]);
  const float* stat = (lane ? a.rstd : a.mean) + first;
  uint32_t stat_row = 0;
  const auto fetch_stats = [&] {
    if (lane < 2 && stat_row < n_rows) {
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(stat_at + (stat_row % 4) * (uint32_t)sizeof(stats[0]) + lane * 4), "l"(stat) : "memory");
      stat += step;
    }
    ++stat_row;
  };
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    fetch_stats();
    if (kVec && s < kStages - 1) { in_x.fetch(s); in_g.fetch(s); }
    copy_async_commit();
  }
  if constexpr (!kVec) { in_x.fetch(0); in_g.fetch(0); }
  __syncthreads();
  F2 dw[N], db[N];
#pragma unroll
  for (int i = 0; i < N; ++i) dw[i] = db[i] = f2(0.f);
  const float inv = 1.f / a.cols;
  T* q = static_cast<T*>(a.dx) + first * a.lddx + t * E;
  const uint64_t q_step = step * a.lddx;
  uint32_t stage = 0, turn = 0;
  for (uint32_t r = 0; r < n_rows; ++r) {
    F2 x[N], g[N];
    fetch_stats();
    if constexpr (kVec) {
      in_x.fetch((stage + kStages - 1) % kStages);
      in_g.fetch((stage + kStages - 1) % kStages);
    }
    copy_async_commit();
    copy_async_wait<kVec ? kStages - 1 : 3>();
    __syncwarp();
    const float2 st = stats[r % 4][threadIdx.x >> 5];
    const float mean = st.x, rstd = st.y;
    in_x.take(stage, x);
    in_g.take(stage, g);
    if constexpr (!kVec) { in_x.fetch(0); in_g.fetch(0); }
    F2 s0 = f2(0.f), s1 = f2(0.f);
    const F2 by = f2(rstd), less = f2(-mean);
#pragma unroll
    for (int i = 0; i < N; i += Q / 2) {
      F2 w[Q / 2];
      const float* p = weights + (i / (Q / 2) * kN + t) * Q;
      if constexpr (kVec) {
        Pack<float>::widen(*reinterpret_cast<const uint4*>(p), w);
      } else {
        const float2 v = *reinterpret_cast<const float2*>(p);
        w[0] = f2(v.x, v.y);
      }
#pragma unroll
      for (int j = 0; j < Q / 2; ++j) {  // beyond the row dy and w are zero
        x[i + j] = (x[i + j] + less) * by;
        dw[i + j] = fma(g[i + j], x[i + j], dw[i + j]);
        db[i + j] = db[i + j] + g[i + j];
        g[i + j] = g[i + j] * w[j];
        s0 = s0 + g[i + j];
        s1 = fma(g[i + j], x[i + j], s1);
      }
    }
    // both sums over the warp in five exchanges: the lower half of the lanes goes on with the first, the upper half with the second
    const float a0 = sum(s0), a1 = sum(s1);
    const bool upper = (threadIdx.x & 16) != 0;
    float s = (upper ? a1 : a0) + __shfl_xor_sync(0xFFFFFFFFu, upper ? a0 : a1, 16);
#pragma unroll
    for (int d = 8; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    float c0, c1;
    if constexpr (nw == 1) {
      c0 = __shfl_sync(0xFFFFFFFFu, s, 0);
      c1 = __shfl_sync(0xFFFFFFFFu, s, 16);
    } else {
      if ((threadIdx.x & 15) == 0) reinterpret_cast<float*>(&red[turn][threadIdx.x >> 5])[upper ? 1 : 0] = s;
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kN) : "memory");
      const float2* r = &red[turn][group * nw];
      c0 = r[0].x; c1 = r[0].y;
#pragma unroll
      for (int i = 1; i < nw; ++i) { c0 += r[i].x; c1 += r[i].y; }
      turn ^= 1;  // written again only behind the next row's barrier
    }
    c0 *= inv;
    c1 *= inv;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fma(x[i], f2(-c1), g[i] + f2(-c0)) * by;
    in_x.store(q, x);
    q += q_step;
    stage = (stage + 1) % kStages;
  }
  let_next_start();
  // the groups' sums, in group order
  if constexpr (kGroups > 1) {
    uint64_t* sums = reinterpret_cast<uint64_t*>(rows);  // [kGroups - 1][2 N][kN] pairs
    copy_async_wait<0>();
    __syncthreads();
    if (group) {
      uint64_t* mine = sums + (group - 1) * (2 * N * kN) + t;
#pragma unroll
      for (int i = 0; i < N; ++i) { mine[2 * i * kN] = dw[i].v; mine[(2 * i + 1) * kN] = db[i].v; }
    }
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int i = 0; i < N; ++i)
      for (int o = 0; o < kGroups - 1; ++o) {
        dw[i] = dw[i] + F2{sums[o * (2 * N * kN) + 2 * i * kN + t]};
        db[i] = db[i] + F2{sums[o * (2 * N * kN) + (2 * i + 1) * kN + t]};
      }
  }
  float* line = a.partial + (uint64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float2 w2 = parts(dw[i]), b2 = parts(db[i]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = ((2 * i + j) / E * kN + t) * E + (2 * i + j) % E;
      if (c < a.cols) { line[c] = j ? w2.y : w2.x; line[a.cols + c] = j ? b2.y : b2.x; }
    }
  }
}

// dw and db from the lines of partial sums: 32 columns a CTA, its warps over the lines, joined in a fixed order
constexpr int kJoinWarps = 16;
__global__ void __launch_bounds__(32 * kJoinWarps) k_norm_join(const float* partial, uint32_t lines, uint32_t cols,
                                                               float* dweight, float* dbias, uint32_t accumulate) {
  __shared__ float part[kJoinWarps][32];
  after_previous();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;  // column of [dw | db]
  float s = 0.f;
  if (c < 2ull * cols) {
#pragma unroll 5
    for (uint32_t l = warp; l < lines; l += kJoinWarps) s += partial[(uint64_t)l * 2 * cols + c];
  }
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

// ---- long rows: every pass reads the row again (from L2, a row at a time a CTA) ---------------------------------------

constexpr int kWideThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kWideThreads) k_norm_wide(NormArgs a) {
  __shared__ __align__(16) float red[2][kWideThreads / 32];
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    float s = 0.f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) s += widen1(x[c]);
    const float mean = block_sum<kWideThreads>(s, red[0]) / a.cols;
    s = 0.f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) { const float d = widen1(x[c]) - mean; s += d * d; }
    const float rstd = rsqrtf(block_sum<kWideThreads>(s, red[1]) / a.cols + a.eps);
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
__global__ void __launch_bounds__(kWideThreads) k_norm_grad_sums(NormGradArgs a, float2* sums) {
  __shared__ __align__(16) float red[2][kWideThreads / 32];
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = static_cast<const T*>(a.x) + row * a.ldx, *dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s0 = 0.f, s1 = 0.f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float g = widen1(dy[c]) * (a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f);
      s0 += g;
      s1 += g * ((widen1(x[c]) - mean) * rstd);
    }
    s0 = block_sum<kWideThreads>(s0, red[0]);
    s1 = block_sum<kWideThreads>(s1, red[1]);
    if (threadIdx.x == 0) sums[row] = make_float2(s0 / a.cols, s1 / a.cols);
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

constexpr uint32_t kNormWideLines = 64;
constexpr uint32_t kNormColsLimit = 1u << 30;  // column counters are 32-bit

// f with the number n of `list` as a constant
template <typename F, int... N>
static void with_number(uint32_t n, std::integer_sequence<int, N...>, F&& f) {
  (void)((n == (uint32_t)N && (f(std::integral_constant<int, N>{}), true)) || ...);
}
template <typename K>
static cudaError_t allow_smem(K kernel, size_t smem) {
  return smem > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) : cudaSuccess;
}

// Threads a row: multiples of 32, so that few of them have nothing (3584 bf16 elements are 224 threads x 2 chunks of 8).
template <typename F>
static void with_threads(uint32_t n, F&& f) {
  with_number(n <= 256 ? (n + 31) / 32 * 32 : (n + 127) / 128 * 128, std::integer_sequence<int, 32, 64, 96, 128, 160, 192, 224, 256, 384, 512>{}, f);
}

template <typename T, bool kVec, int kElems>
static constexpr int kChunks = kVec ? (kElems < Pack<T>::kElems ? 1 : kElems / Pack<T>::kElems) : kElems;

template <typename T, bool kVec, int V>
static cudaError_t norm_rows(const ft_pool* p, const NormArgs& a, cudaStream_t st) {
  const uint32_t n = a.cols / (kVec ? Pack<T>::kElems : 1);
  cudaError_t e = cudaErrorInvalidConfiguration;
  with_threads((n + V - 1) / V, [&](auto k) {
    constexpr int kN = decltype(k)::value;
    auto kernel = k_norm<T, V, kVec, kN>;
    constexpr size_t smem = kVec ? (size_t)kNormStages<V, kN> * V * kN * 16 : 0;
    static_assert(smem + 2 * (kN / 32 + 3) / 4 * 16 <= kSmemMost, "every instance can be launched");
    if ((e = allow_smem(kernel, smem)) != cudaSuccess) return;
    int per_sm = 1;
    if (a.rows > (uint64_t)p->sm_count) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kN, smem);
    if (e != cudaSuccess) return;
    kernel<<<(unsigned)std::min<uint64_t>(a.rows, (uint64_t)std::max(1, per_sm) * p->sm_count), kN, smem, st>>>(a);
    e = cudaGetLastError();
  });
  return e;
}

// Elements a thread: 16 (82 us for 32768 rows x 3584 in bf16), 32 for rows beyond 256 x 16 (80 us for 14336 x 8192, 99 with
// 16); few where there are few rows, which are a matter of latency.
template <typename T, bool kVec>
static cudaError_t norm_launch(const ft_pool* p, const NormArgs& a, cudaStream_t st) {
  constexpr uint32_t E = kVec ? Pack<T>::kElems : 1;
  constexpr int kFew = kChunks<T, kVec, 4>, kMany = kChunks<T, kVec, 16>, kLong = kChunks<T, kVec, 32>;
  const uint32_t n = a.cols / E;
  if (n > kLong * 512u) {
    k_norm_wide<T><<<(unsigned)std::min<uint64_t>(a.rows, 4ull * p->sm_count), kWideThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  if (a.rows <= 2ull * p->sm_count && n <= kFew * 512u) return norm_rows<T, kVec, kFew>(p, a, st);
  return n <= kMany * 256u ? norm_rows<T, kVec, kMany>(p, a, st) : norm_rows<T, kVec, kLong>(p, a, st);
}

template <typename T, bool kVec, int V, int kN>
static cudaError_t norm_grad_rows(ft_pool* p, const NormGradArgs& a, uint32_t* lines, cudaStream_t st) {
  constexpr int E = kVec ? Pack<T>::kElems : 1, kGroups = kGradGroups(V * E, kN);
  constexpr size_t kRows = kVec ? 2ull * kGradStages<V, kN * kGroups> * V * kN * kGroups * 16 : 0, kSums = (kGroups - 1) * 2ull * V * E * kN * 4;
  constexpr size_t smem = (size_t)V * E * kN * 4 + (kRows > kSums ? kRows : kSums);
  static_assert(smem + 6 * (kN * kGroups / 32) * sizeof(float2) <= kSmemMost, "every instance can be launched");
  auto kernel = k_norm_grad<T, V, kVec, kN, kGroups>;
  const cudaError_t e = allow_smem(kernel, smem);
  if (e != cudaSuccess) return e;
  *lines = (uint32_t)std::min<uint64_t>((a.rows + kGroups - 1) / kGroups, (uint64_t)p->sm_count);
  kernel<<<*lines, kN * kGroups, smem, st>>>(a);
  return cudaGetLastError();
}

// 16 elements a thread (121 us for 32768 rows x 3584 in bf16, 135 with 32), which 256 threads make 4096; 32 up to 8192.
template <typename T, bool kVec>
static cudaError_t norm_grad_launch(ft_pool* p, const NormGradArgs& a, float2* sums, uint32_t* lines, cudaStream_t st) {
  constexpr uint32_t E = kVec ? Pack<T>::kElems : 1;
  constexpr int kFew = kChunks<T, kVec, 4>, kMany = kChunks<T, kVec, 16>, kLong = kChunks<T, true, 32>;
  const uint32_t n = a.cols / E;
  if (n <= 32u * kFew) return norm_grad_rows<T, kVec, kFew, 32>(p, a, lines, st);
  cudaError_t e = cudaErrorInvalidConfiguration;
  if (n <= kMany * 256u) {
    with_threads((n + kMany - 1) / kMany, [&](auto k) {
      constexpr int kN = decltype(k)::value;
      if constexpr (kN <= 256) e = norm_grad_rows<T, kVec, kMany, kN>(p, a, lines, st);
    });
  } else if (kVec && n <= kLong * 256u) {
    with_threads((n + kLong - 1) / kLong, [&](auto k) {
      constexpr int kN = decltype(k)::value;
      if constexpr (kVec && kN > 128 && kN <= 256) e = norm_grad_rows<T, true, kLong, kN>(p, a, lines, st);
    });
  } else {
    k_norm_grad_sums<T><<<(unsigned)std::min<uint64_t>(a.rows, 4ull * p->sm_count), kWideThreads, 0, st>>>(a, sums);
    *lines = (uint32_t)std::min<uint64_t>(a.rows, kNormWideLines);
    k_norm_grad_cols<T><<<dim3((a.cols + 255u) / 256u, *lines), 256, 0, st>>>(a, sums);
    p->gpu_launches += 1;
    e = cudaGetLastError();
  }
  return e;
}

// bytes of the backward pass's workspace: the lines of partial sums, and for long rows two numbers a row (which rows those are
// depends on the operands' alignment too: 4096 elements are the least)
static uint64_t norm_grad_ws(const ft_pool* p, uint64_t rows, uint32_t cols) {
  const uint64_t lines = std::min<uint64_t>(rows, std::max<uint64_t>(p->sm_count, kNormWideLines));
  return align_up_sz(lines * 2 * cols * sizeof(float), 256) + (cols > 4096 ? rows * sizeof(float2) : 0);
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
  using B = __nv_bfloat16;
  FT_CUDA(dtype == FT_F32 ? (vec ? norm_launch<float, true>(p, a, st) : norm_launch<float, false>(p, a, st))
                          : (vec ? norm_launch<B, true>(p, a, st) : norm_launch<B, false>(p, a, st)));
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
  float2* sums = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + norm_grad_ws(p, rows, cols)) - rows;  // at the workspace's end
  const bool vec = cols * es % 16 == 0 && rows_in_16(dy, lddy, es) && rows_in_16(x, ldx, es) && rows_in_16(dx, lddx, es);
  uint32_t lines = 0;
  using B = __nv_bfloat16;
  FT_CUDA(dtype == FT_F32 ? (vec ? norm_grad_launch<float, true>(p, a, sums, &lines, st) : norm_grad_launch<float, false>(p, a, sums, &lines, st))
                          : (vec ? norm_grad_launch<B, true>(p, a, sums, &lines, st) : norm_grad_launch<B, false>(p, a, sums, &lines, st)));
  p->gpu_launches += 1;
  if (dweight || dbias) {
    FT_CUDA(launch_chained(k_norm_join, dim3((unsigned)((2ull * cols + 31) / 32)), 32 * kJoinWarps, 0, st, static_cast<const float*>(a.partial), lines, cols,
                           dweight, dbias, accumulate));
    p->gpu_launches += 1;
  }
  return FT_OK;
}

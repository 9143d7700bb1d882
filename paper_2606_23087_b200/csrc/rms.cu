// Root-mean-square norm over the rows of a matrix, forward with the residual's addition and an 8-bit output, and backward.
//
//   forward    s = x + residual,  rstd = (sum(s^2) / c + eps)^-1/2,  y = s rstd w;  of every 128 columns of a row
//              scale = max|y| / 448,  q = e4m3(y / scale)
//   backward   xhat = s rstd,  a = w dy,  ds = rstd (a - xhat sum(a xhat) / c) + dsum,  dw = sum over rows of dy xhat
//
// Both are bound by HBM: each row is read and written once.  32768 rows x 3584 in bf16: with a residual 142 us (6.6 TB/s, the copy rate), without
// one 73, with an 8-bit output 127; backward with dsum 154 us (6.1 TB/s, 6 us of it for joining the lines).  Rows off 16-byte boundaries go element by
// element: 198 and 263 us.
//
//   k_rms           a few warps hold a row in registers, the rows that follow are on their way into shared memory
//   k_rms_grad      groups of warps hold a row each; a thread always owns the same columns, so the sums over rows stay in its registers.
//                   No atomics: partial sums go to the workspace, one line a CTA
//   k_rms_join      adds the lines of partial sums in line order
//   k_rms_wide, k_rms_grad_sums, k_rms_grad_cols   rows too long for that, and 8-bit outputs of rows off 16-byte boundaries
#include <algorithm>
#include <cmath>

#include <cuda_fp8.h>

#include "rows.cuh"

namespace ft {

constexpr uint32_t kRmsGroup = 128;  // columns that share a scale
constexpr float kFp8Most = 448.f;
constexpr float kFp8Least = 0x1p-110f;  // the least magnitude that a group is scaled by: its inverse is finite

struct RmsArgs {
  uint64_t rows, ldx, ldr, lds, ldy, ldq, ldqs;
  uint32_t cols, param_dtype, rows_each;  // rows_each: of a CTA
  const void *x, *residual, *weight;
  void *sum, *y;
  uint8_t* q;
  float *q_scale, *rstd;
  float eps;
};

struct RmsGradArgs {
  uint64_t rows, lddy, lds, lddsum, lddx;
  uint32_t cols, param_dtype;
  const void *dy, *s, *dsum, *weight;
  const float* rstd;
  void* dx;
  float* partial;  // [lines][cols]
};

// the scale of a group whose largest magnitude is `top`, and what its values are multiplied by
__device__ __forceinline__ float2 rms_scale(float top) {
  if (!(top < INFINITY)) return make_float2(__uint_as_float(0x7FC00000u), 0.f);  // a value that is not finite: the group reads back as NaN
  if (top == 0.f) return make_float2(0.f, 0.f);
  top = fmaxf(top, kFp8Least);
  return make_float2(top / kFp8Most, kFp8Most / top);
}
// E weights of consecutive columns from c on, 16 bytes at a time where they lie so; ones without weights or where the row has ended
template <int E>
__device__ __forceinline__ void weights_from(const void* weight, uint32_t dtype, uint32_t c, bool there, F2 (&w)[E / 2]) {
#pragma unroll
  for (int i = 0; i < E / 2; ++i) w[i] = f2(1.f);
  if (!weight || !there) return;
  if (dtype == FT_F32) {
    const float* p = static_cast<const float*>(weight) + c;
    if (aligned16(p)) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) Pack<float>::widen(*reinterpret_cast<const uint4*>(p + 4 * i), w + 2 * i);
      return;
    }
  } else if (E == 8 && aligned16(static_cast<const __nv_bfloat16*>(weight) + c)) {
    Pack<__nv_bfloat16>::widen(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(weight) + c), reinterpret_cast<F2*>(w));
    return;
  }
#pragma unroll
  for (int i = 0; i < E / 2; ++i) w[i] = f2(load_as(weight, dtype, c + 2 * i), load_as(weight, dtype, c + 2 * i + 1));
}

// ---- forward ------------------------------------------------------------------------------------------------------

// CTAs of an SM: 896 threads of 72 registers, 512 where a thread holds 32 elements or goes element by element.
template <typename T, int V, bool kVec, int kN>
constexpr int kRmsCtas = kVec && V * Pack<T>::kElems <= 16 ? 896 / kN : 512 / kN;
// Rows in shared memory or under way to it: as many as leave room for those CTAs, from two to four; two where a call has few rows.
constexpr int stages_within(size_t budget, size_t stage) { return budget / stage < 2 ? 2 : budget / stage > 4 ? 4 : (int)(budget / stage); }
template <int kStreams, typename T, int V, int kN>
constexpr int kRmsStages = V * Pack<T>::kElems <= 8 ? 2 : stages_within(kSmemMost / kRmsCtas<T, V, true, kN> - 2048, (size_t)kStreams * V * kN * 16);

template <typename T, int V, bool kVec, int kN, bool kRes>
__global__ void __launch_bounds__(kN, (kRmsCtas<T, V, kVec, kN>)) k_rms(RmsArgs a) {
  extern __shared__ __align__(16) uint4 ring[];  // [streams][kStages][V][kN]
  __shared__ __align__(16) float red[2][(kN / 32 + 3) / 4 * 4];
  constexpr int E = kVec ? Pack<T>::kElems : 1, N = V * E / 2, kStages = kRmsStages<kRes ? 2 : 1, T, V, kN>;  // N pairs
  using Feed = RowFeed<T, V, kVec, kN, kN, kStages>;
  Feed in, add;
  let_next_start();
  after_previous();
  const uint64_t row0 = (uint64_t)blockIdx.x * a.rows_each;
  const uint32_t n_rows = (uint32_t)min((uint64_t)a.rows_each, a.rows - row0);
  in.init(a.x, a.ldx, row0, 1, n_rows, a.cols, threadIdx.x, ring + threadIdx.x);
  if constexpr (kRes) add.init(a.residual, a.ldr, row0, 1, n_rows, a.cols, threadIdx.x, ring + kStages * V * kN + threadIdx.x);
  const auto fetch = [&](uint32_t s) {
    in.fetch(s);
    if constexpr (kRes) add.fetch(s);
    if constexpr (kVec) copy_async_commit();
  };
  if constexpr (kVec) {
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(s);
  } else {
    fetch(0);
  }
  if (kN > 32 && threadIdx.x < sizeof(red) / 4) (&red[0][0])[threadIdx.x] = 0.f;
  F2 w[N];
#pragma unroll
  for (int k = 0; k < V * E; k += kVec ? E : 2) {
    const uint32_t c = (k / E * kN + threadIdx.x) * E;
    if constexpr (kVec) {
      weights_from<E>(a.weight, a.param_dtype, c, in.has(k / E), *reinterpret_cast<F2(*)[E / 2]>(w + k / 2));
    } else {
      w[k / 2] = f2(in.has(k) && a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f, in.has(k + 1) && a.weight ? load_as(a.weight, a.param_dtype, c + kN) : 1.f);
    }
  }
  if (kN > 32) __syncthreads();
  const float inv = 1.f / a.cols;
  T* sum_out = a.sum ? static_cast<T*>(a.sum) + row0 * a.lds + threadIdx.x * E : nullptr;
  T* y_out = a.y ? static_cast<T*>(a.y) + row0 * a.ldy + threadIdx.x * E : nullptr;
  uint32_t stage = 0;
  for (uint32_t r = 0; r < n_rows; ++r) {
    F2 x[N], ss[2] = {f2(0.f), f2(0.f)};
    if constexpr (kVec) {
      fetch((stage + kStages - 1) % kStages);
      copy_async_wait<kStages - 1>();
    }
    in.take(stage, x);
    if constexpr (kRes) {
      F2 b[N];
      add.take(stage, b);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = x[i] + b[i];
    }
    if constexpr (!kVec) fetch(0);
    if (sum_out) {
      in.store(sum_out, x);
      sum_out += a.lds;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) ss[i & 1] = fma(x[i], x[i], ss[i & 1]);  // beyond the row x is zero
    const float rstd = rsqrtf(block_sum<kN>(sum(ss[0] + ss[1]), red[r & 1]) * inv + a.eps);
    const uint64_t row = row0 + r;
    if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = x[i] * f2(rstd) * w[i];
    if (y_out) {
      in.store(y_out, x);
      y_out += a.ldy;
    }
    if constexpr (kVec) {
      if (a.q) {
        // the lanes that share a group: 16 of a bf16 row, all 32 of an fp32 row
#pragma unroll
        for (int k = 0; k < V; ++k) {
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < E / 2; ++i) {
            const float2 v = parts(x[k * (E / 2) + i]);
            top = max_with_nan(top, max_with_nan(fabsf(v.x), fabsf(v.y)));
          }
#pragma unroll
          for (int d = kRmsGroup / E / 2; d; d >>= 1) top = max_with_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
          if (!in.has(k)) continue;
          const float2 scale = rms_scale(top);
          const uint32_t c = (k * kN + threadIdx.x) * E;
          if (c % kRmsGroup == 0) a.q_scale[row * a.ldqs + c / kRmsGroup] = scale.x;
          uint32_t q[E / 4];
#pragma unroll
          for (int i = 0; i < E / 4; ++i) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(parts(x[k * (E / 2) + 2 * i] * f2(scale.y)), __NV_SATFINITE, __NV_E4M3);
            q[i] = lo | (uint32_t)__nv_cvt_float2_to_fp8x2(parts(x[k * (E / 2) + 2 * i + 1] * f2(scale.y)), __NV_SATFINITE, __NV_E4M3) << 16;
          }
          uint8_t* to = a.q + row * a.ldq + c;
          if constexpr (E == 8) *reinterpret_cast<uint2*>(to) = make_uint2(q[0], q[1]);
          else *reinterpret_cast<uint32_t*>(to) = q[0];
        }
      }
    }
    stage = (stage + 1) % kStages;
  }
}

// Any row, by single elements: three passes over it, from cache behind the first.  A warp takes the groups of 8-bit columns.
constexpr int kRmsWideThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kRmsWideThreads) k_rms_wide(RmsArgs a) {
  __shared__ __align__(16) float red[2][kRmsWideThreads / 32];
  uint32_t turn = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
    const auto value = [&](uint32_t c) { return widen1(x[c]) + (res ? widen1(res[c]) : 0.f); };
    const auto weight = [&](uint32_t c) { return a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f; };
    float s = 0.f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += kRmsWideThreads) {
      const float v = value(c);
      s = fmaf(v, v, s);
    }
    const float rstd = rsqrtf(block_sum<kRmsWideThreads>(s, red[turn]) / a.cols + a.eps);
    if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
    if (a.q) {
      for (uint32_t c0 = threadIdx.x / 32 * kRmsGroup; c0 < a.cols; c0 += kRmsWideThreads / 32 * kRmsGroup) {
        float y[4], top = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t c = c0 + 32 * i + (threadIdx.x & 31);
          y[i] = c < a.cols ? value(c) * rstd * weight(c) : 0.f;
          top = max_with_nan(top, fabsf(y[i]));
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) top = max_with_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const float2 scale = rms_scale(top);
        if ((threadIdx.x & 31) == 0) a.q_scale[row * a.ldqs + c0 / kRmsGroup] = scale.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t c = c0 + 32 * i + (threadIdx.x & 31);
          if (c < a.cols) a.q[row * a.ldq + c] = (uint8_t)__nv_cvt_float_to_fp8(y[i] * scale.y, __NV_SATFINITE, __NV_E4M3);
        }
      }
      if (a.sum || a.y) __syncthreads();  // sum and y may lie where x or the residual do
    }
    for (uint32_t c = threadIdx.x; (a.sum || a.y) && c < a.cols; c += kRmsWideThreads) {
      const float v = value(c);
      if (a.sum) static_cast<T*>(a.sum)[row * a.lds + c] = narrow1<T>(v);
      if (a.y) static_cast<T*>(a.y)[row * a.ldy + c] = narrow1<T>(v * rstd * weight(c));
    }
  }
}

// ---- backward -----------------------------------------------------------------------------------------------------

// Threads of a CTA, one CTA an SM.  Where the rows are in shared memory a thread reads s twice from there, for the row's sum and for dx,
// instead of keeping it, which leaves registers for 21 warps of 16 elements a thread (with both operands kept 14: 32768 rows x 3584 in
// bf16 with dsum 192 us, not 154) or 32 of 8.  Without dsum w dy is read again too.  Element by element both are kept.
constexpr int kRmsGradThreads(bool vec, int elems) { return vec ? (elems > 16 ? 512 : elems > 8 ? 672 : 1024) : (elems > 16 ? 256 : 512); }
// Groups of kN threads: as many as that, and as leave room for two of their rows in shared memory.
template <int kStreams, typename T, int V, bool kVec, int kN>
constexpr int kRmsGradGroups = [] {
  const int most = kRmsGradThreads(kVec, V * (kVec ? Pack<T>::kElems : 1)) / kN;
  if (!kVec) return most;
  const size_t row = 2ull * kStreams * V * kN * 16, room = kSmemMost - 1024 - (size_t)V * Pack<T>::kElems * kN * 4;
  const int fit = (int)(room / row) < most ? (int)(room / row) : most;
  return fit > 15 ? 15 : fit;  // a group has a named barrier, of which there are sixteen
}();
// Rows in shared memory or under way to it: as many as fit beside the weights.
template <int kStreams, typename T, int V, int kN, int kThreads>
constexpr int kRmsGradStages = stages_within(kSmemMost - 1024 - (size_t)V * Pack<T>::kElems * kN * 4, (size_t)kStreams * V * kThreads * 16);

// The CTA's threads form groups of kN; group i of the grid takes the rows i, i + groups, ...
template <typename T, int V, bool kVec, int kN, int kGroups, bool kRes>
__global__ void __launch_bounds__(kN * kGroups, 1) k_rms_grad(RmsGradArgs a) {
  extern __shared__ __align__(16) uint4 ring[];  // weights; then [streams][kStages][V][kThreads], at the end the groups' sums
  constexpr int E = kVec ? Pack<T>::kElems : 1, N = V * E / 2, kThreads = kN * kGroups, kStages = kRmsGradStages<kRes ? 3 : 2, T, V, kN, kThreads>, nw = kN / 32;
  __shared__ float red[2][kThreads / 32], stats[4][kThreads / 32];
  const uint32_t group = threadIdx.x / kN, t = threadIdx.x % kN;
  constexpr int Q = kVec ? 4 : 2;
  after_previous();
  float* weights = reinterpret_cast<float*>(ring);  // [V E / Q][kN][Q]
  uint4* rows = ring + V * E * kN / 4;
  for (uint32_t i = threadIdx.x; i < V * E * kN; i += kThreads) {
    const uint32_t th = i / Q % kN, e = i / Q / kN * Q + i % Q;  // the thread and which of its V E elements
    const uint32_t c = (e / E * kN + th) * E + e % E;
    weights[i] = c < a.cols ? (a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f) : 0.f;
  }
  const uint64_t step = (uint64_t)gridDim.x * kGroups, first = (uint64_t)blockIdx.x * kGroups + group;
  const uint32_t n_rows = rows_from(a.rows, first, step);
  using Feed = RowFeed<T, V, kVec, kN, kThreads, kStages>;
  // Element by element a bf16 row of dsum is asked for where its turn begins: a row ahead it takes more registers than there are (32768 rows x
  // 3583 337 us, so 268; 16384 fp32 rows 213, so 228).
  constexpr bool kAheadD = kVec || sizeof(T) == 4;
  Feed in_s, in_g, in_d;
  in_s.init(a.s, a.lds, first, step, n_rows, a.cols, t, rows + threadIdx.x);
  in_g.init(a.dy, a.lddy, first, step, n_rows, a.cols, t, rows + kStages * V * kThreads + threadIdx.x);
  if constexpr (kRes && kAheadD) in_d.init(a.dsum, a.lddsum, first, step, n_rows, a.cols, t, rows + 2 * kStages * V * kThreads + threadIdx.x);
  const auto fetch = [&](uint32_t s) {
    in_s.fetch(s);
    in_g.fetch(s);
    if constexpr (kRes && kAheadD) in_d.fetch(s);
  };
  [[maybe_unused]] const T* d_row = static_cast<const T*>(a.dsum) + first * a.lddsum + t;  // dsum's current row, where it is not fetched ahead
  // a row's rstd comes three rows ahead as well, a copy a warp
  const uint32_t lane = threadIdx.x & 31, stat_at = shared_address(&stats[0][threadIdx.x >> 5]);
  const float* stat = a.rstd + first;
  uint32_t stat_row = 0;
  const auto fetch_stats = [&] {
    if (lane == 0 && stat_row < n_rows) {
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(stat_at + (stat_row % 4) * (uint32_t)sizeof(stats[0])), "l"(stat) : "memory");
      stat += step;
    }
    ++stat_row;
  };
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    fetch_stats();
    if (kVec && s < kStages - 1) fetch(s);
    copy_async_commit();
  }
  if constexpr (!kVec) fetch(0);
  __syncthreads();
  F2 dw[N];
#pragma unroll
  for (int i = 0; i < N; ++i) dw[i] = f2(0.f);
  const float inv = 1.f / a.cols;
  T* q = static_cast<T*>(a.dx) + first * a.lddx + t * E;
  const uint64_t q_step = step * a.lddx;
  uint32_t stage = 0, turn = 0;
  // the sum over the group's threads
  const auto group_sum = [&](float v) {
    v = warp_sum(v);
    if constexpr (nw > 1) {
      if (lane == 0) red[turn][threadIdx.x >> 5] = v;
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kN) : "memory");
      const float* r1 = &red[turn][group * nw];
      v = r1[0];
#pragma unroll
      for (int i = 1; i < nw; ++i) v += r1[i];
      turn ^= 1;  // written again only behind the next row's barrier
    }
    return v;
  };
  for (uint32_t r = 0; r < n_rows; ++r) {
    fetch_stats();
    if constexpr (kVec) fetch((stage + kStages - 1) % kStages);
    copy_async_commit();
    copy_async_wait<kVec ? kStages - 1 : 3>();
    __syncwarp();
    const float rstd = stats[r % 4][threadIdx.x >> 5];
    const F2 by = f2(rstd);
    F2 s1[2] = {f2(0.f), f2(0.f)};
    if constexpr (kVec) {
      F2 a_kept[kRes ? N : 1];
      const auto weights_of = [&](int k, F2 (&w)[E / 2]) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i)
          Pack<float>::widen(*reinterpret_cast<const uint4*>(weights + ((k * E / 4 + i) * kN + t) * 4), w + 2 * i);
      };
#pragma unroll
      for (int k = 0; k < V; ++k) {
        F2 x[E / 2], g[E / 2], w[E / 2];
        in_s.take_chunk(stage, k, x);
        in_g.take_chunk(stage, k, g);
        weights_of(k, w);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {  // beyond the row dy and w are zero
          const F2 xhat = x[i] * by;
          dw[k * (E / 2) + i] = fma(g[i], xhat, dw[k * (E / 2) + i]);
          const F2 wg = g[i] * w[i];
          if constexpr (kRes) a_kept[k * (E / 2) + i] = wg;
          s1[i & 1] = fma(wg, xhat, s1[i & 1]);
        }
      }
      const float c1 = group_sum(sum(s1[0] + s1[1])) * inv;
      const F2 less = f2(-c1);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        F2 x[E / 2], g[E / 2], w[E / 2], d[E / 2];
        in_s.take_chunk(stage, k, x);
        if constexpr (kRes) {
          in_d.take_chunk(stage, k, d);
        } else {
          in_g.take_chunk(stage, k, g);
          weights_of(k, w);
        }
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          if constexpr (kRes) d[i] = fma(fma(x[i] * by, less, a_kept[k * (E / 2) + i]), by, d[i]);
          else d[i] = fma(x[i] * by, less, g[i] * w[i]) * by;
        }
        if (in_s.has(k)) *reinterpret_cast<uint4*>(q + k * kN * E) = Pack<T>::narrow(d);
      }
    } else {
      F2 x[N], g[N], d_ahead[kRes && kAheadD ? N : 1];
      [[maybe_unused]] T d[kRes && !kAheadD ? V : 1];
      in_s.take(stage, x);
      in_g.take(stage, g);
      if constexpr (kRes && kAheadD) {
        in_d.take(stage, d_ahead);
      } else if constexpr (kRes) {
#pragma unroll
        for (int k = 0; k < V; ++k) d[k] = in_s.has(k) ? d_row[k * kN] : narrow1<T>(0.f);
        d_row += step * a.lddsum;
      }
      fetch(0);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 v = *reinterpret_cast<const float2*>(weights + (i * kN + t) * Q);
        x[i] = x[i] * by;
        dw[i] = fma(g[i], x[i], dw[i]);
        g[i] = g[i] * f2(v.x, v.y);
        s1[i & 1] = fma(g[i], x[i], s1[i & 1]);
      }
      const float c1 = group_sum(sum(s1[0] + s1[1])) * inv;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const F2 v = fma(x[i], f2(-c1), g[i]);
        if constexpr (kRes && kAheadD) x[i] = fma(v, by, d_ahead[i]);
        else if constexpr (kRes) x[i] = fma(v, by, f2(widen1(d[2 * i]), widen1(d[2 * i + 1])));
        else x[i] = v * by;
      }
      in_s.store(q, x);
    }
    q += q_step;
    stage = (stage + 1) % kStages;
  }
  let_next_start();
  // the groups' sums, in group order
  if constexpr (kGroups > 1) {
    uint64_t* sums = reinterpret_cast<uint64_t*>(rows);  // [kGroups - 1][N][kN] pairs
    copy_async_wait<0>();
    __syncthreads();
    if (group) {
      uint64_t* mine = sums + (group - 1) * (N * kN) + t;
#pragma unroll
      for (int i = 0; i < N; ++i) mine[i * kN] = dw[i].v;
    }
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int i = 0; i < N; ++i)
      for (int o = 0; o < kGroups - 1; ++o) dw[i] = dw[i] + F2{sums[o * (N * kN) + i * kN + t]};
  }
  float* line = a.partial + (uint64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float2 w2 = parts(dw[i]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t c = ((2 * i + j) / E * kN + t) * E + (2 * i + j) % E;
      if (c < a.cols) line[c] = j ? w2.y : w2.x;
    }
  }
}

// dw from the lines of partial sums: 32 columns a CTA, its warps over the lines, joined in a fixed order
constexpr int kRmsJoinWarps = 16;
__global__ void __launch_bounds__(32 * kRmsJoinWarps) k_rms_join(const float* partial, uint32_t lines, uint32_t cols, float* dweight, uint32_t accumulate) {
  __shared__ float part[kRmsJoinWarps][32];
  after_previous();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 5
    for (uint32_t l = warp; l < lines; l += kRmsJoinWarps) s += partial[(uint64_t)l * cols + c];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp || c >= cols) return;
#pragma unroll
  for (int w = 1; w < kRmsJoinWarps; ++w) s += part[w][lane];
  dweight[c] = accumulate ? dweight[c] + s : s;
}

// Long rows: sums[row] = sum(a xhat) / cols
template <typename T>
__global__ void __launch_bounds__(kRmsWideThreads) k_rms_grad_sums(RmsGradArgs a, float* sums) {
  __shared__ __align__(16) float red[2][kRmsWideThreads / 32];
  uint32_t turn = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const T *x = static_cast<const T*>(a.s) + row * a.lds, *dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const float rstd = a.rstd[row];
    float s = 0.f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += kRmsWideThreads)
      s += widen1(dy[c]) * (a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f) * (widen1(x[c]) * rstd);
    s = block_sum<kRmsWideThreads>(s, red[turn]);
    if (threadIdx.x == 0) sums[row] = s / a.cols;
  }
}

// CTA (column block, line): its columns of the rows line, line + lines, ...
template <typename T>
__global__ void __launch_bounds__(256) k_rms_grad_cols(RmsGradArgs a, const float* sums) {
  const uint64_t c = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= a.cols) return;
  const float w = a.weight ? load_as(a.weight, a.param_dtype, c) : 1.f;
  float dw = 0.f;
  for (uint64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float g = widen1(static_cast<const T*>(a.dy)[row * a.lddy + c]), rstd = a.rstd[row];
    const float xhat = widen1(static_cast<const T*>(a.s)[row * a.lds + c]) * rstd;
    dw += g * xhat;
    float d = rstd * (g * w - xhat * sums[row]);
    if (a.dsum) d += widen1(static_cast<const T*>(a.dsum)[row * a.lddsum + c]);
    static_cast<T*>(a.dx)[row * a.lddx + c] = narrow1<T>(d);
  }
  a.partial[(uint64_t)blockIdx.y * a.cols + c] = dw;
}

// ---- launch geometry ----------------------------------------------------------------------------------------------

constexpr uint32_t kRmsWideLines = 64;
constexpr uint32_t kRmsColsLimit = 1u << 30;  // column counters are 32-bit

template <typename T, bool kVec, int V, bool kRes>
static cudaError_t rms_rows(const ft_pool* p, const RmsArgs& a, cudaStream_t st) {
  const uint32_t n = a.cols / (kVec ? Pack<T>::kElems : 1);
  cudaError_t e = cudaErrorInvalidConfiguration;
  with_threads((n + V - 1) / V, [&](auto k) {
    constexpr int kN = decltype(k)::value;
    auto kernel = k_rms<T, V, kVec, kN, kRes>;
    constexpr size_t smem = kVec ? (size_t)(kRes ? 2 : 1) * kRmsStages<kRes ? 2 : 1, T, V, kN> * V * kN * 16 : 0;
    if constexpr (smem + 2 * (kN / 32 + 3) / 4 * 16 > kSmemMost) return;  // rms_launch takes no such rows here
    else if ((e = allow_smem(kernel, smem)) != cudaSuccess) return;
    // Few consecutive rows a CTA: what is read and written at a time then lies close together.  (Persistent CTAs that take every n-th
    // row drift apart: 32768 rows x 3584 with a residual 164 us against 142, without one 88 against 73.  From 4 to 8 rows make little
    // difference; with 2 the weights' loads show.)  A CTA each for rows that do not fill the device.
    const uint64_t resident = (uint64_t)kRmsCtas<T, V, kVec, kN> * p->sm_count;
    RmsArgs b = a;
    b.rows_each = (uint32_t)std::max<uint64_t>(std::min<uint64_t>(a.rows / resident, 6), std::max<uint64_t>(1, a.rows >> 30));
    e = launch_chained(kernel, dim3((unsigned)((a.rows + b.rows_each - 1) / b.rows_each)), kN, smem, st, b);
  });
  return e;
}

// Elements a thread: 16, 32 for rows beyond 256 x 16; few where there are few rows, which are a matter of latency.
template <typename T, bool kVec, bool kRes>
static cudaError_t rms_launch(const ft_pool* p, const RmsArgs& a, cudaStream_t st) {
  constexpr uint32_t E = kVec ? Pack<T>::kElems : 1;
  constexpr int kFew = kChunks<T, kVec, 4>, kMany = kChunks<T, kVec, 16>, kLong = kChunks<T, kVec, 32>;
  const uint32_t n = a.cols / E;
  constexpr uint32_t kMost = kVec && kRes && sizeof(T) == 4 ? 384 : 512;  // threads whose two rows of two operands fit in shared memory
  if (n > kLong * kMost || (!kVec && a.q)) {
    k_rms_wide<T><<<(unsigned)std::min<uint64_t>(a.rows, 4ull * p->sm_count), kRmsWideThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  if (a.rows <= 2ull * p->sm_count && n <= kFew * 512u) return rms_rows<T, kVec, kFew, kRes>(p, a, st);
  return n <= kMany * 256u ? rms_rows<T, kVec, kMany, kRes>(p, a, st) : rms_rows<T, kVec, kLong, kRes>(p, a, st);
}
template <typename T>
static cudaError_t rms_typed(const ft_pool* p, const RmsArgs& a, bool vec, cudaStream_t st) {
  if (a.residual) return vec ? rms_launch<T, true, true>(p, a, st) : rms_launch<T, false, true>(p, a, st);
  return vec ? rms_launch<T, true, false>(p, a, st) : rms_launch<T, false, false>(p, a, st);
}

template <typename T, bool kVec, int V, int kN, bool kRes>
static cudaError_t rms_grad_rows(ft_pool* p, const RmsGradArgs& a, uint32_t* lines, cudaStream_t st) {
  constexpr int E = kVec ? Pack<T>::kElems : 1, kStreams = kRes ? 3 : 2, kGroups = kRmsGradGroups<kStreams, T, V, kVec, kN>;
  constexpr size_t kRows = kVec ? (size_t)kStreams * kRmsGradStages<kStreams, T, V, kN, kN * kGroups> * V * kN * kGroups * 16 : 0, kSums = (kGroups - 1) * (size_t)V * E * kN * 4;
  constexpr size_t smem = (size_t)V * E * kN * 4 + (kRows > kSums ? kRows : kSums);
  static_assert(smem + 6 * (kN * kGroups / 32) * sizeof(float) <= kSmemMost, "every instance can be launched");
  auto kernel = k_rms_grad<T, V, kVec, kN, kGroups, kRes>;
  const cudaError_t e = allow_smem(kernel, smem);
  if (e != cudaSuccess) return e;
  *lines = (uint32_t)std::min<uint64_t>((a.rows + kGroups - 1) / kGroups, (uint64_t)p->sm_count);
  return launch_chained(kernel, dim3(*lines), kN * kGroups, smem, st, a);
}

// Whether rows with dsum may go 8 elements a thread in groups of kN, and not 16.  More warps hide more, and twice as many threads reduce and issue:
// 8 do better where 2, 4 or 8 groups make a CTA, and with two elements a word only where next to all of a group's threads have some.
// us, 8 against 16 elements a thread, 0.7 GB in sustained passes: bf16 28672 x 4096 155 and 162, 30464 x 3840 157 and 160, 57344 x 2048 146 and
// 161, 61440 x 1792 145 and 152, 65536 x 1024 89 and 93; but 32768 x 3584 (7/8 of the threads) 162 and 154, 36864 x 3200 173 and 158, 76000 x 1536
// (5 groups) 192 and 152, 229376 x 512 (15) 194 and 173.  fp32 16384 x 3584 144 and 189, 18432 x 3200 144 and 190, 22528 x 2560 148 and 168,
// 57344 x 1024 150 and 183; 114000 x 512 185 and 166.  Without dsum 16: 32768 x 3584 in bf16 124, 8 140.
template <typename T, int kN>
constexpr bool kRmsGradEight = [] {
  const int groups = kRmsGradGroups<3, T, kChunks<T, true, 8>, true, kN>;
  return groups == 2 || groups == 4 || groups == 8;
}();

// 16 elements a thread, which 256 threads make 4096, or 8 and 512 threads; 32 up to 8192.
template <typename T, bool kVec, bool kRes>
static cudaError_t rms_grad_launch(ft_pool* p, const RmsGradArgs& a, float* sums, uint32_t* lines, cudaStream_t st) {
  constexpr uint32_t E = kVec ? Pack<T>::kElems : 1;
  constexpr int kFew = kChunks<T, kVec, 4>, kEight = kChunks<T, true, 8>, kMany = kChunks<T, kVec, 16>, kLong = kChunks<T, true, 32>;
  const uint32_t n = a.cols / E;
  if (n <= 32u * kFew) return rms_grad_rows<T, kVec, kFew, 32, kRes>(p, a, lines, st);
  cudaError_t e = cudaErrorInvalidConfiguration;
  if (n <= kMany * 256u) {
    bool eight = false;
    if constexpr (kVec && kRes)
      with_threads((n + kEight - 1) / kEight, [&](auto k) {
        constexpr int kN = decltype(k)::value;
        if constexpr (kRmsGradEight<T, kN>)
          if ((eight = sizeof(T) == 4 || 16 * (n / kEight) >= 15u * kN)) e = rms_grad_rows<T, kVec, kEight, kN, kRes>(p, a, lines, st);
      });
    if (!eight)
      with_threads((n + kMany - 1) / kMany, [&](auto k) {
        constexpr int kN = decltype(k)::value;
        if constexpr (kN <= 256) e = rms_grad_rows<T, kVec, kMany, kN, kRes>(p, a, lines, st);
      });
  } else if (kVec && n <= kLong * 256u) {
    with_threads((n + kLong - 1) / kLong, [&](auto k) {
      constexpr int kN = decltype(k)::value;
      if constexpr (kVec && kN > 128 && kN <= 256) e = rms_grad_rows<T, true, kLong, kN, kRes>(p, a, lines, st);
    });
  } else {
    k_rms_grad_sums<T><<<(unsigned)std::min<uint64_t>(a.rows, 4ull * p->sm_count), kRmsWideThreads, 0, st>>>(a, sums);
    *lines = (uint32_t)std::min<uint64_t>(a.rows, kRmsWideLines);
    k_rms_grad_cols<T><<<dim3((a.cols + 255u) / 256u, *lines), 256, 0, st>>>(a, sums);
    p->gpu_launches += 1;
    e = cudaGetLastError();
  }
  return e;
}
template <typename T>
static cudaError_t rms_grad_typed(ft_pool* p, const RmsGradArgs& a, bool vec, float* sums, uint32_t* lines, cudaStream_t st) {
  if (a.dsum) return vec ? rms_grad_launch<T, true, true>(p, a, sums, lines, st) : rms_grad_launch<T, false, true>(p, a, sums, lines, st);
  return vec ? rms_grad_launch<T, true, false>(p, a, sums, lines, st) : rms_grad_launch<T, false, false>(p, a, sums, lines, st);
}

// bytes of the backward pass's workspace: the lines of partial sums, and for long rows a number a row (which rows those are depends on
// the operands' alignment too: 4096 elements are the least)
static uint64_t rms_grad_lines_ws(const ft_pool* p, uint64_t rows, uint32_t cols) {
  return align_up_sz(std::min<uint64_t>(rows, std::max<uint64_t>(p->sm_count, kRmsWideLines)) * cols * sizeof(float), 256);
}
static uint64_t rms_grad_ws(const ft_pool* p, uint64_t rows, uint32_t cols) {
  return rms_grad_lines_ws(p, rows, cols) + (cols > 4096 ? rows * sizeof(float) : 0);
}

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_rms_norm(ft_pool* p, uint64_t rows, uint32_t cols, const void* x, uint64_t ldx, const void* residual, uint64_t ldr,
                                uint32_t dtype, const void* weight, uint32_t param_dtype, float eps, void* sum, uint64_t lds, void* y,
                                uint64_t ldy, void* q, uint64_t ldq, float* q_scale, uint64_t ldqs, float* rstd, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (cols == 0 || !dtype_ok(dtype) || !dtype_ok(param_dtype) || !(eps >= 0.f) || std::isinf(eps)) return FT_ERR_INVALID_ARG;
  if (cols > kRmsColsLimit) return FT_ERR_CAPACITY;
  if (rows == 0) return FT_OK;
  const uint32_t es = dtype_size(dtype), ps = dtype_size(param_dtype);
  // a matrix that is there: its stride and alignment
  const auto bad = [&](const void* m, uint64_t ld, uint64_t least, uint32_t size) { return m && (ld < least || !aligned_to(m, size)); };
  if (!x || (!y && !q && !sum) || bad(x, ldx, cols, es) || bad(residual, ldr, cols, es) || bad(sum, lds, cols, es) || bad(y, ldy, cols, es) ||
      bad(q, ldq, cols, 1) || !q != !q_scale || bad(q_scale, ldqs, (cols + kRmsGroup - 1) / kRmsGroup, 4) || !aligned_to(weight, ps) || !aligned_to(rstd, 4))
    return FT_ERR_INVALID_ARG;
  const auto lands = [&](const void* out, uint64_t ld) { return on_other_rows(rows, out, ld, x, ldx) || on_other_rows(rows, out, ld, residual, ldr); };
  if (lands(sum, lds) || lands(y, ldy) || (sum && sum == y)) return FT_ERR_INVALID_ARG;
  RmsArgs a;
  a.rows = rows; a.cols = cols; a.param_dtype = param_dtype; a.eps = eps;
  a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.weight = weight;
  a.sum = sum; a.lds = lds; a.y = y; a.ldy = ldy; a.q = static_cast<uint8_t*>(q); a.ldq = ldq; a.q_scale = q_scale; a.ldqs = ldqs; a.rstd = rstd;
  const auto in16 = [&](const void* m, uint64_t ld) { return !m || rows_in_16(m, ld, es); };
  const uint32_t qa = es == 2 ? 8 : 4;  // bytes of an access to q
  const bool vec = cols * es % 16 == 0 && in16(x, ldx) && in16(residual, ldr) && in16(sum, lds) && in16(y, ldy) && aligned_to(q, qa) && (!q || ldq % qa == 0);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  FT_CUDA(dtype == FT_F32 ? rms_typed<float>(p, a, vec, st) : rms_typed<__nv_bfloat16>(p, a, vec, st));
  p->gpu_launches += 1;
  return FT_OK;
}

FT_EXPORT int32_t pool_rms_norm_grad_workspace(ft_pool* p, uint64_t rows, uint32_t cols, uint64_t* bytes) {
  if (!p || cols == 0 || !bytes) return FT_ERR_INVALID_ARG;
  if (cols > kRmsColsLimit) return FT_ERR_CAPACITY;
  *bytes = rows ? rms_grad_ws(p, rows, cols) : 0;
  return FT_OK;
}

FT_EXPORT int32_t pool_rms_norm_grad(ft_pool* p, uint64_t rows, uint32_t cols, const void* dy, uint64_t lddy, const void* s, uint64_t lds,
                                     const void* dsum, uint64_t lddsum, uint32_t dtype, const void* weight, uint32_t param_dtype,
                                     const float* rstd, void* dx, uint64_t lddx, float* dweight, uint32_t accumulate, void* workspace,
                                     uint64_t workspace_bytes, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (cols == 0 || !dtype_ok(dtype) || !dtype_ok(param_dtype) || !aligned_to(dweight, 4)) return FT_ERR_INVALID_ARG;
  if (cols > kRmsColsLimit) return FT_ERR_CAPACITY;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {  // a sum over no rows
    if (!accumulate && dweight) FT_CUDA(cudaMemsetAsync(dweight, 0, (size_t)cols * 4, st));
    return FT_OK;
  }
  const uint32_t es = dtype_size(dtype);
  if (!dy || !s || !rstd || !dx || lddy < cols || lds < cols || lddx < cols || (dsum && lddsum < cols)) return FT_ERR_INVALID_ARG;
  if (!aligned_to(dy, es) || !aligned_to(s, es) || !aligned_to(dsum, es) || !aligned_to(dx, es) || !aligned_to(weight, dtype_size(param_dtype))) return FT_ERR_INVALID_ARG;
  if (on_other_rows(rows, dx, lddx, dy, lddy) || on_other_rows(rows, dx, lddx, s, lds) || on_other_rows(rows, dx, lddx, dsum, lddsum)) return FT_ERR_INVALID_ARG;
  if (!aligned_to(rstd, 4) || !workspace || !aligned_to(workspace, 256)) return FT_ERR_INVALID_ARG;
  if (workspace_bytes < rms_grad_ws(p, rows, cols)) return FT_ERR_CAPACITY;
  RmsGradArgs a;
  a.rows = rows; a.cols = cols; a.param_dtype = param_dtype;
  a.dy = dy; a.lddy = lddy; a.s = s; a.lds = lds; a.dsum = dsum; a.lddsum = lddsum; a.weight = weight; a.rstd = rstd; a.dx = dx; a.lddx = lddx;
  a.partial = static_cast<float*>(workspace);
  float* sums = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + rms_grad_lines_ws(p, rows, cols));
  const bool vec = cols * es % 16 == 0 && rows_in_16(dy, lddy, es) && rows_in_16(s, lds, es) && rows_in_16(dx, lddx, es) && (!dsum || rows_in_16(dsum, lddsum, es));
  uint32_t lines = 0;
  FT_CUDA(dtype == FT_F32 ? rms_grad_typed<float>(p, a, vec, sums, &lines, st) : rms_grad_typed<__nv_bfloat16>(p, a, vec, sums, &lines, st));
  p->gpu_launches += 1;
  if (dweight) {
    FT_CUDA(launch_chained(k_rms_join, dim3((cols + 31) / 32), 32 * kRmsJoinWarps, 0, st, static_cast<const float*>(a.partial), lines, cols, dweight, accumulate));
    p->gpu_launches += 1;
  }
  return FT_OK;
}

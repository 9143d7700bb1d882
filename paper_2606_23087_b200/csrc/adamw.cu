// One AdamW step over a list of tensors.
//
//   g' = s g (s: the device-side gradient scale, or 1)
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by HBM: every array is read and written once, 16 operations an element.  One launch serves up to kAdamwPerLaunch
// tensors: their descriptors travel as kernel arguments (no upload, nothing for the caller to keep), a CTA finds its
// tensor by a binary search over the tensors' first chunks, and a warp takes 256 elements at a time.
//
// 8-bit states.  A block of 256 elements of a tensor holds m and r = sqrt(v) as float8 (e4m3) values times one scale a
// block and state.  Keeping r instead of v halves the range that the format has to cover: its 18 octaves are 36 octaves of
// v.  The scale is the smallest power of two that brings the block's largest value to 448 or less: products with it are
// exact, so a value that needs no rounding survives any number of steps, and no precision is lost to it, e4m3 being a
// floating format itself.  A positive r never rounds to zero (its floor is 2^-9 of the scale), because m / (0 + eps) would
// be a step without bound.  m, v and r are taken with one rounding an operation (no contraction), which makes the stored
// bytes the same on every launch shape.  A block that holds a value that is not finite reads back as NaN.
#include <algorithm>
#include <cmath>

#include <cuda_fp8.h>

#include "operators.cuh"

namespace ft {

constexpr uint32_t kAdamwBlock = 256;      // elements that share a scale; a warp's share of a round
constexpr int kAdamwThreads = 256;
constexpr uint32_t kAdamwChunk = 8 * 256;  // elements a CTA updates: one block a warp
constexpr uint32_t kAdamwPerLaunch = 320;  // tensors a launch takes at most (kernel arguments hold 32 KiB)
constexpr uint32_t kAdamwFew = 8;          // tensors of the launch with a small argument block

struct AdamwTensorArg {
  void *param, *m, *v, *copy;
  const void* grad;
  float *m_scale, *v_scale;
  uint64_t n;
  uint64_t first_chunk;  // chunks of the tensors before this one
  float keep;            // 1 - lr * weight decay
  uint16_t kind;         // see adamw_kind
  uint16_t pad;
};

struct AdamwConst {
  float b1, c1, b2, c2;   // c: 1 - b
  float step, inv, eps;   // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  const float* grad_scale;
};

template <uint32_t kCap>
struct AdamwArgs {
  AdamwConst k;
  uint32_t n;
  AdamwTensorArg t[kCap];
};

// kind bits: 1 parameters bf16, 2 gradients bf16, 4 states in 8 bits, 8 every array's blocks start on 16-byte boundaries
// (8 for float8 states, whose lanes hold 8 bytes)
enum { kParamBf16 = 1, kGradBf16 = 2, kState8 = 4, kVec = 8 };

// A lane's eight elements of a block: the consecutive ones 8 lane .. 8 lane + 7 where the arrays allow wide accesses,
// else lane, lane + 32, ... (each access of the warp still covers one contiguous range).
template <bool kV>
__device__ __forceinline__ uint32_t elem_of(uint32_t lane, int i) { return kV ? lane * 8 + i : lane + 32 * i; }

template <typename T, bool kV>
__device__ __forceinline__ void load8(const T* p, uint32_t lane, uint32_t left, float (&f)[8]) {
  if constexpr (kV) {
    if (lane * 8 + 8 <= left) {
      if constexpr (sizeof(T) == 4) {
        Pack<float>::widen(*reinterpret_cast<const uint4*>(p + lane * 8), f);
        Pack<float>::widen(*reinterpret_cast<const uint4*>(p + lane * 8 + 4), f + 4);
      } else {
        Pack<__nv_bfloat16>::widen(*reinterpret_cast<const uint4*>(p + lane * 8), f);
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = elem_of<kV>(lane, i) < left ? widen1(p[elem_of<kV>(lane, i)]) : 0.f;
}
template <typename T, bool kV>
__device__ __forceinline__ void store8(T* p, uint32_t lane, uint32_t left, const float (&f)[8]) {
  if constexpr (kV) {
    if (lane * 8 + 8 <= left) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint4*>(p + lane * 8) = Pack<float>::narrow(f);
        *reinterpret_cast<uint4*>(p + lane * 8 + 4) = Pack<float>::narrow(f + 4);
      } else {
        *reinterpret_cast<uint4*>(p + lane * 8) = Pack<__nv_bfloat16>::narrow(f);
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (elem_of<kV>(lane, i) < left) p[elem_of<kV>(lane, i)] = narrow1<T>(f[i]);
}

__device__ __forceinline__ void widen_fp8x2(uint16_t q, float* f) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(q, __NV_E4M3);
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h));
  f[0] = x.x;
  f[1] = x.y;
}
template <bool kV>
__device__ __forceinline__ void load_state8(const uint8_t* p, uint32_t lane, uint32_t left, float scale, float (&f)[8]) {
  uint16_t q[4];
  if (kV && lane * 8 + 8 <= left) {
    const uint2 v = *reinterpret_cast<const uint2*>(p + lane * 8);
    q[0] = (uint16_t)v.x; q[1] = (uint16_t)(v.x >> 16); q[2] = (uint16_t)v.y; q[3] = (uint16_t)(v.y >> 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t e0 = elem_of<kV>(lane, 2 * i), e1 = elem_of<kV>(lane, 2 * i + 1);
      q[i] = (uint16_t)((e0 < left ? p[e0] : 0) | ((e1 < left ? p[e1] : 0) << 8));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) widen_fp8x2(q[i], f + 2 * i);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(f[i], scale);
}

// the block's scale (lane 0 stores it) and its values rounded to float8
template <bool kV, bool kFloor>
__device__ __forceinline__ void store_state8(uint8_t* p, float* scale_out, uint32_t lane, uint32_t left, const float (&f)[8]) {
  // fmaxf drops a NaN: not finite is looked for in the bits, whose order is that of the magnitudes
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (elem_of<kV>(lane, i) < left) top = max(top, __float_as_uint(f[i]) & 0x7FFFFFFFu);
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  float scale = 0.f, inv = 0.f;
  if (top >= 0x7F800000u) {
    scale = __uint_as_float(0x7FC00000u);
  } else if (top) {
    // top = m 2^x with m in [1, 2): 448 = 1.75 2^8, so 2^(x - 8) does where m <= 1.75, else 2^(x - 7)
    int x = (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    x = max(-100, min(100, x));
    scale = __uint_as_float((uint32_t)(x + 127) << 23);
    inv = __uint_as_float((uint32_t)(127 - x) << 23);
  }
  if (lane == 0) *scale_out = scale;
  uint16_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = f[2 * i] * inv, b = f[2 * i + 1] * inv;
    if (kFloor) {
      a = a > 0.f ? fmaxf(a, 0.001953125f) : a;
      b = b > 0.f ? fmaxf(b, 0.001953125f) : b;
    }
    q[i] = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  }
  if (kV && lane * 8 + 8 <= left) {
    *reinterpret_cast<uint2*>(p + lane * 8) = make_uint2(q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t e0 = elem_of<kV>(lane, 2 * i), e1 = elem_of<kV>(lane, 2 * i + 1);
    if (e0 < left) p[e0] = (uint8_t)q[i];
    if (e1 < left) p[e1] = (uint8_t)(q[i] >> 8);
  }
}

template <typename P, typename G, bool k8, bool kV>
__device__ __forceinline__ void adamw_block(const AdamwTensorArg& t, const AdamwConst& k, uint64_t e0, uint32_t lane) {
  const uint32_t left = (uint32_t)min((uint64_t)kAdamwBlock, t.n - e0);
  float g[8], m[8], r[8], w[8];
  load8<G, kV>(static_cast<const G*>(t.grad) + e0, lane, left, g);
  load8<P, kV>(static_cast<const P*>(t.param) + e0, lane, left, w);
  if constexpr (k8) {
    load_state8<kV>(static_cast<const uint8_t*>(t.m) + e0, lane, left, t.m_scale[e0 / kAdamwBlock], m);
    load_state8<kV>(static_cast<const uint8_t*>(t.v) + e0, lane, left, t.v_scale[e0 / kAdamwBlock], r);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __fmul_rn(r[i], r[i]);
  } else {
    load8<float, kV>(static_cast<const float*>(t.m) + e0, lane, left, m);
    load8<float, kV>(static_cast<const float*>(t.v) + e0, lane, left, r);
  }
  const float s = k.grad_scale ? *k.grad_scale : 1.f;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = __fmul_rn(g[i], s);
    m[i] = __fadd_rn(__fmul_rn(k.b1, m[i]), __fmul_rn(k.c1, x));
    v[i] = __fadd_rn(__fmul_rn(k.b2, r[i]), __fmul_rn(k.c2, __fmul_rn(x, x)));
    r[i] = __fsqrt_rn(v[i]);
    w[i] = w[i] * t.keep - k.step * __fdividef(m[i], fmaf(r[i], k.inv, k.eps));
  }
  store8<P, kV>(static_cast<P*>(t.param) + e0, lane, left, w);
  if (t.copy) store8<__nv_bfloat16, kV>(static_cast<__nv_bfloat16*>(t.copy) + e0, lane, left, w);
  if constexpr (k8) {
    store_state8<kV, false>(static_cast<uint8_t*>(t.m) + e0, t.m_scale + e0 / kAdamwBlock, lane, left, m);
    store_state8<kV, true>(static_cast<uint8_t*>(t.v) + e0, t.v_scale + e0 / kAdamwBlock, lane, left, r);
  } else {
    store8<float, kV>(static_cast<float*>(t.m) + e0, lane, left, m);
    store8<float, kV>(static_cast<float*>(t.v) + e0, lane, left, v);
  }
}

template <uint32_t kCap>
__global__ void __launch_bounds__(kAdamwThreads) k_adamw(const __grid_constant__ AdamwArgs<kCap> a) {
  uint32_t lo = 0, hi = a.n;  // the last tensor whose first chunk is not behind this one
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (a.t[mid].first_chunk <= blockIdx.x) lo = mid; else hi = mid;
  }
  const AdamwTensorArg& t = a.t[lo];
  const uint64_t e0 = (blockIdx.x - t.first_chunk) * kAdamwChunk + (threadIdx.x >> 5) * kAdamwBlock;
  if (e0 >= t.n) return;
  const uint32_t lane = threadIdx.x & 31;
  using B = __nv_bfloat16;
  switch (t.kind) {
    case 0: adamw_block<float, float, false, false>(t, a.k, e0, lane); break;
    case 1: adamw_block<B, float, false, false>(t, a.k, e0, lane); break;
    case 2: adamw_block<float, B, false, false>(t, a.k, e0, lane); break;
    case 3: adamw_block<B, B, false, false>(t, a.k, e0, lane); break;
    case 4: adamw_block<float, float, true, false>(t, a.k, e0, lane); break;
    case 5: adamw_block<B, float, true, false>(t, a.k, e0, lane); break;
    case 6: adamw_block<float, B, true, false>(t, a.k, e0, lane); break;
    case 7: adamw_block<B, B, true, false>(t, a.k, e0, lane); break;
    case 8: adamw_block<float, float, false, true>(t, a.k, e0, lane); break;
    case 9: adamw_block<B, float, false, true>(t, a.k, e0, lane); break;
    case 10: adamw_block<float, B, false, true>(t, a.k, e0, lane); break;
    case 11: adamw_block<B, B, false, true>(t, a.k, e0, lane); break;
    case 12: adamw_block<float, float, true, true>(t, a.k, e0, lane); break;
    case 13: adamw_block<B, float, true, true>(t, a.k, e0, lane); break;
    case 14: adamw_block<float, B, true, true>(t, a.k, e0, lane); break;
    default: adamw_block<B, B, true, true>(t, a.k, e0, lane); break;
  }
}

static uint16_t adamw_kind(const ft_adamw_tensor& t) {
  const bool s8 = t.state_bits == 8;
  const bool vec = aligned_to(t.param, 16) && aligned_to(t.grad, 16) && aligned_to(t.copy, 16) && aligned_to(t.m, s8 ? 8 : 16) &&
                   aligned_to(t.v, s8 ? 8 : 16);
  return (uint16_t)((t.param_dtype == FT_BF16 ? kParamBf16 : 0) | (t.grad_dtype == FT_BF16 ? kGradBf16 : 0) | (s8 ? kState8 : 0) | (vec ? kVec : 0));
}

template <uint32_t kCap>
static cudaError_t adamw_launch(const AdamwConst& k, double lr, const ft_adamw_tensor* t, uint32_t n, uint64_t chunks, cudaStream_t st) {
  AdamwArgs<kCap> a;
  a.k = k;
  a.n = 0;
  uint64_t at = 0;
  for (uint32_t i = 0; i < n; ++i) {
    if (t[i].n == 0) continue;
    AdamwTensorArg& d = a.t[a.n++];
    d.param = t[i].param; d.m = t[i].m; d.v = t[i].v; d.copy = t[i].copy; d.grad = t[i].grad;
    d.m_scale = t[i].m_scale; d.v_scale = t[i].v_scale; d.n = t[i].n; d.first_chunk = at;
    d.keep = (float)(1.0 - lr * t[i].weight_decay);
    d.kind = adamw_kind(t[i]); d.pad = 0;
    at += (t[i].n + kAdamwChunk - 1) / kAdamwChunk;
  }
  k_adamw<kCap><<<(unsigned)chunks, kAdamwThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_adamw_step(ft_pool* p, const ft_adamw_tensor* tensors, uint32_t n_tensors, const ft_adamw_config* cfg, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (!cfg || (n_tensors && !tensors)) return FT_ERR_INVALID_ARG;
  if (!std::isfinite(cfg->lr) || !(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) ||
      !(cfg->eps >= 0.0) || !std::isfinite(cfg->eps) || cfg->step == 0 || !aligned_to(cfg->grad_scale, 4))
    return FT_ERR_INVALID_ARG;
  for (uint32_t i = 0; i < n_tensors; ++i) {
    const ft_adamw_tensor& t = tensors[i];
    if (!dtype_ok(t.param_dtype) || !dtype_ok(t.grad_dtype) || (t.state_bits != 8 && t.state_bits != 32) || !std::isfinite(t.weight_decay))
      return FT_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    const uintptr_t sa = t.state_bits == 8 ? 1 : 4;
    if (!t.param || !t.grad || !t.m || !t.v || !aligned_to(t.param, dtype_size(t.param_dtype)) || !aligned_to(t.grad, dtype_size(t.grad_dtype)) ||
        !aligned_to(t.m, sa) || !aligned_to(t.v, sa) || !aligned_to(t.copy, 2))
      return FT_ERR_INVALID_ARG;
    if (t.state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4))) return FT_ERR_INVALID_ARG;
    if (t.n > (1ull << 40)) return FT_ERR_CAPACITY;
  }
  AdamwConst k;
  k.b1 = (float)cfg->beta1; k.c1 = (float)(1.0 - cfg->beta1);
  k.b2 = (float)cfg->beta2; k.c2 = (float)(1.0 - cfg->beta2);
  k.step = (float)(cfg->lr / (1.0 - std::pow(cfg->beta1, (double)cfg->step)));
  k.inv = (float)(1.0 / std::sqrt(1.0 - std::pow(cfg->beta2, (double)cfg->step)));
  k.eps = (float)cfg->eps;
  k.grad_scale = cfg->grad_scale;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // as many tensors a launch as its arguments hold and its grid can index
  for (uint32_t i0 = 0; i0 < n_tensors;) {
    uint32_t i1 = i0, used = 0;
    uint64_t chunks = 0;
    while (i1 < n_tensors && used < kAdamwPerLaunch) {
      const uint64_t c = (tensors[i1].n + kAdamwChunk - 1) / kAdamwChunk;
      if (chunks + c > 0x7FFFFFFFull) break;
      chunks += c;
      used += c != 0;
      ++i1;
    }
    if (chunks) {
      FT_CUDA(used <= kAdamwFew ? adamw_launch<kAdamwFew>(k, cfg->lr, tensors + i0, i1 - i0, chunks, st)
                                : adamw_launch<kAdamwPerLaunch>(k, cfg->lr, tensors + i0, i1 - i0, chunks, st));
      p->gpu_launches += 1;
    }
    i0 = i1;
  }
  return FT_OK;
}

// One AdamW step over a list of tensors.
//
//   g' = s g (s: the device-side gradient scale, or 1)
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by HBM: every array is read and written once, 16 operations an element: 117 M elements with fp32 states and a bf16 copy 514 us
// (6.85 TB/s).  With 8-bit states by issue slots: 82 M bf16 elements 171 to 184 us from card to card (4.5 to 4.8 TB/s, 55 instructions an element, 74 %
// of the slots), and where a tensor's arrays are off 16 bytes, element by element, 270 us for 80 M against 158; fp32 states lose nothing there.  One launch serves up to kAdamwPerLaunch
// tensors of one kind: their descriptors travel as kernel arguments (no upload, nothing for the caller to keep), a CTA finds its
// tensor by a binary search over the tensors' first chunks, and a warp takes blocks of 256 elements.
//
// 8-bit states.  A block of 256 elements of a tensor holds m and r = sqrt(v) as float8 (e4m3) values times one scale a
// block and state.  Keeping r instead of v halves the range that the format has to cover: its 18 octaves are 36 octaves of
// v.  The scale is the smallest power of two that brings the block's largest value to 448 or less: products with it are
// exact, so a value that needs no rounding survives any number of steps, and no precision is lost to it, e4m3 being a
// floating format itself.  A positive r never rounds to zero (its floor is 2^-9 of the scale), because m / (0 + eps) would
// be a step without bound.  m, v and r are taken with one rounding an operation (no contraction), which makes the stored
// bytes the same on every launch shape.  A block that holds a value that is not finite reads back as NaN.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <type_traits>

#include <cuda_fp8.h>

#include "operators.cuh"

namespace ft {

constexpr uint32_t kAdamwBlock = 256;      // elements that share a scale
constexpr int kAdamwThreads = 256;
constexpr uint32_t kAdamwPerLaunch = 320;  // tensors a launch takes at most (kernel arguments hold 32 KiB)
constexpr uint32_t kAdamwFew = 8;          // tensors of the launch with a small argument block

struct AdamwTensorArg {
  void *param, *m, *v, *copy;
  const void* grad;
  float *m_scale, *v_scale;
  uint64_t n;
  uint64_t first_chunk;  // chunks of the tensors before this one
  float keep;            // 1 - lr * weight decay
};

struct AdamwConst {         // pairs of equal values, as the kernel's operations take them
  float2 b1, c1, b2, c2;    // c: 1 - b
  float2 step, inv, eps;    // -lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  float2 minus_zero;        // see rounded_product
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

// A lane's eight elements as they are stored; those beyond the tensor are zero.
template <typename T, bool kV>
struct Raw8 {
  static constexpr int kQuads = sizeof(T) == 4 ? 2 : 1;
  uint4 q[kQuads];
  __device__ __forceinline__ void load(const T* p, uint32_t lane, uint32_t left) {
    if (kV && lane * 8 + 8 <= left) {
#pragma unroll
      for (int i = 0; i < kQuads; ++i) q[i] = *reinterpret_cast<const uint4*>(p + lane * 8 + i * (8 / kQuads));
      return;
    }
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = elem_of<kV>(lane, i) < left ? p[elem_of<kV>(lane, i)] : narrow1<T>(0.f);
    memcpy(q, v, sizeof(v));
  }
  // (every operation below is taken by pairs, each value rounded by itself)
  __device__ __forceinline__ void widen(F2 (&f)[4]) const {
#pragma unroll
    for (int i = 0; i < kQuads; ++i) Pack<T>::widen(q[i], f + i * (4 / kQuads));
  }
};
template <typename T, bool kV>
__device__ __forceinline__ void store8(T* p, uint32_t lane, uint32_t left, const F2 (&f)[4]) {
  if constexpr (kV) {
    if (lane * 8 + 8 <= left) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint4*>(p + lane * 8) = Pack<float>::narrow(f);
        *reinterpret_cast<uint4*>(p + lane * 8 + 4) = Pack<float>::narrow(f + 2);
      } else {
        *reinterpret_cast<uint4*>(p + lane * 8) = Pack<__nv_bfloat16>::narrow(f);
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = parts(f[i]);
    if (elem_of<kV>(lane, 2 * i) < left) p[elem_of<kV>(lane, 2 * i)] = narrow1<T>(v.x);
    if (elem_of<kV>(lane, 2 * i + 1) < left) p[elem_of<kV>(lane, 2 * i + 1)] = narrow1<T>(v.y);
  }
}

template <bool kV>
struct RawState8 {
  uint2 q;
  float scale;
  __device__ __forceinline__ void load(const uint8_t* p, const float* scale_of_block, uint32_t lane, uint32_t left) {
    scale = *scale_of_block;
    if (kV && lane * 8 + 8 <= left) {
      q = *reinterpret_cast<const uint2*>(p + lane * 8);
      return;
    }
    uint8_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = elem_of<kV>(lane, i) < left ? p[elem_of<kV>(lane, i)] : 0;
    memcpy(&q, v, sizeof(v));
  }
  __device__ __forceinline__ void widen(F2 (&f)[4]) const {
    const uint16_t pair[4] = {(uint16_t)q.x, (uint16_t)(q.x >> 16), (uint16_t)q.y, (uint16_t)(q.y >> 16)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(pair[i], __NV_E4M3);
      const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h));
      f[i] = f2(x.x, x.y);
    }
  }
};

// the block's scale (lane 0 stores it) and its values rounded to float8; `top`: bits of its largest magnitude
template <bool kV, bool kRoot>
__device__ __forceinline__ void store_state8(uint8_t* p, float* scale_out, uint32_t lane, uint32_t left, uint32_t top, const F2 (&f)[4]) {
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
  uint32_t q[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(parts(f[2 * i] * f2(inv)), __NV_SATFINITE, __NV_E4M3);
    q[i] = lo | (uint32_t)__nv_cvt_float2_to_fp8x2(parts(f[2 * i + 1] * f2(inv)), __NV_SATFINITE, __NV_E4M3) << 16;
    if (kRoot && ((q[i] - 0x01010101u) & ~q[i] & 0x80808080u)) {  // some byte is zero: a positive root takes the smallest value, 1
      const float2 a = parts(f[2 * i]), b = parts(f[2 * i + 1]);
      const float r[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (r[j] > 0.f && !(q[i] >> 8 * j & 0xFF)) q[i] |= 1u << 8 * j;
    }
  }
  if (kV && lane * 8 + 8 <= left) {
    *reinterpret_cast<uint2*>(p + lane * 8) = make_uint2(q[0], q[1]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (elem_of<kV>(lane, i) < left) p[elem_of<kV>(lane, i)] = (uint8_t)(q[i / 4] >> 8 * (i % 4));
}

// a b rounded by itself: the assembler makes one operation of a product of pairs and the sum that follows, .rn or not, but
// not of a multiply-add with an addend that it does not know (-0, which changes nothing)
__device__ __forceinline__ F2 f2(float2 v) { return f2(v.x, v.y); }
__device__ __forceinline__ F2 rounded_product(F2 a, F2 b, const AdamwConst& k) { return fma(a, b, f2(k.minus_zero)); }

__device__ __forceinline__ float reciprocal(float x) {  // 1 ulp; x is zero or normal
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float inverse_root(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Square roots of pairs by one step of Heron's method from an approximate inverse root, the residual taken exactly by a
// multiply-add: r = s + (v - s s) / (2 s), off by less than 2^-43 of r before its one rounding (eight of __fsqrt_rn a lane were a
// third of the kernel's instructions).  v lies in [2^-100, 2^104] or is zero.
__device__ __forceinline__ F2 root(F2 v) {
  const float2 a = parts(v);
  const F2 y = f2(inverse_root(fmaxf(a.x, 0x1p-126f)), inverse_root(fmaxf(a.y, 0x1p-126f)));
  const F2 s = v * y;
  return fma(fma(s * f2(-1.f), s, v), y * f2(0.5f), s);
}

constexpr uint32_t kRootBelow = 0x53800000u;  // bits of 2^40

// what a block is made from
template <typename P, typename G, bool k8, bool kV>
struct AdamwLoads {
  Raw8<G, kV> g;
  Raw8<P, kV> w;
  std::conditional_t<k8, RawState8<kV>, Raw8<float, kV>> m, v;
  __device__ __forceinline__ void load(const AdamwTensorArg& t, uint64_t e0, uint32_t lane) {
    const uint32_t left = (uint32_t)min((uint64_t)kAdamwBlock, t.n - e0);
    g.load(static_cast<const G*>(t.grad) + e0, lane, left);
    w.load(static_cast<const P*>(t.param) + e0, lane, left);
    if constexpr (k8) {
      m.load(static_cast<const uint8_t*>(t.m) + e0, t.m_scale + e0 / kAdamwBlock, lane, left);
      v.load(static_cast<const uint8_t*>(t.v) + e0, t.v_scale + e0 / kAdamwBlock, lane, left);
    } else {
      m.load(static_cast<const float*>(t.m) + e0, lane, left);
      v.load(static_cast<const float*>(t.v) + e0, lane, left);
    }
  }
};

template <typename P, typename G, bool k8, bool kV>
__device__ __forceinline__ void adamw_block(const AdamwLoads<P, G, k8, kV>& in, const AdamwTensorArg& t, const AdamwConst& k, uint64_t e0, uint32_t lane) {
  const uint32_t left = (uint32_t)min((uint64_t)kAdamwBlock, t.n - e0);
  F2 g[4], m[4], v[4], r[4], w[4];
  in.g.widen(g);
  in.w.widen(w);
  in.m.widen(m);
  F2 b1 = f2(k.b1);
  if constexpr (k8) {
    b1 = b1 * f2(in.m.scale);  // the scale is a power of two: b1 (scale q) and (b1 scale) q round alike
    in.v.widen(r);
#pragma unroll
    for (int i = 0; i < 4; ++i) { r[i] = r[i] * f2(in.v.scale); v[i] = r[i] * r[i]; }
  } else {
    in.v.widen(v);
  }
  const float s = k.grad_scale ? *k.grad_scale : 1.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const F2 x = g[i] * f2(s);
    m[i] = rounded_product(b1, m[i], k) + rounded_product(f2(k.c1), x, k);
    v[i] = rounded_product(f2(k.b2), v[i], k) + rounded_product(f2(k.c2), x * x, k);
  }
  uint32_t most = 0;  // bits of the largest v of the warp; a NaN's are above all
  if constexpr (k8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = parts(v[i]);
      most = max(most, max(__float_as_uint(a.x), __float_as_uint(a.y)));
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    // v is brought up by an even power of two, so that root() sees no subnormal number; blocks with a v too large for that (a
    // gradient above some 10^6) or not finite take the function
    if (most < kRootBelow) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = root(v[i] * f2(0x1p64f)) * f2(0x1p-32f);
    }
  }
  if (!k8 || most >= kRootBelow) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = parts(v[i]);
      r[i] = f2(sqrtf(a.x), sqrtf(a.y));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 d = parts(fma(r[i], f2(k.inv), f2(k.eps)));
    w[i] = fma(m[i] * f2(reciprocal(d.x), reciprocal(d.y)), f2(k.step), w[i] * f2(t.keep));
  }
  store8<P, kV>(static_cast<P*>(t.param) + e0, lane, left, w);
  if (t.copy) store8<__nv_bfloat16, kV>(static_cast<__nv_bfloat16*>(t.copy) + e0, lane, left, w);
  if constexpr (k8) {
    uint32_t top = 0;  // bits of the largest |m|, whose order is that of the magnitudes and which keep a NaN in sight
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = parts(m[i]);
      top = max(top, max(__float_as_uint(a.x) & 0x7FFFFFFFu, __float_as_uint(a.y) & 0x7FFFFFFFu));
    }
    store_state8<kV, false>(static_cast<uint8_t*>(t.m) + e0, t.m_scale + e0 / kAdamwBlock, lane, left, __reduce_max_sync(0xFFFFFFFFu, top), m);
    // the largest root is the largest v's
    store_state8<kV, true>(static_cast<uint8_t*>(t.v) + e0, t.v_scale + e0 / kAdamwBlock, lane, left, __float_as_uint(__fsqrt_rn(__uint_as_float(most))), r);
  } else {
    store8<float, kV>(static_cast<float*>(t.m) + e0, lane, left, m);
    store8<float, kV>(static_cast<float*>(t.v) + e0, lane, left, v);
  }
}

// Blocks of a warp whose loads go out together.  8-bit states bring little in a block: with one block a warp, 32 warps an SM
// keep some 25 KiB on their way, which held the kernel at 3.7 TB/s.
template <bool k8>
constexpr uint32_t kAdamwAtOnce = k8 ? 2 : 1;
template <bool k8>
constexpr uint32_t kAdamwChunk = kAdamwAtOnce<k8> * (kAdamwThreads / 32) * kAdamwBlock;  // elements of a CTA

template <typename P, typename G, bool k8, bool kV, uint32_t kCap>
__device__ __forceinline__ void adamw_cta(const AdamwArgs<kCap>& a) {
  uint32_t lo = 0, hi = a.n;  // the last tensor whose first chunk is not behind this one
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (a.t[mid].first_chunk <= blockIdx.x) lo = mid; else hi = mid;
  }
  const AdamwTensorArg& t = a.t[lo];
  const uint64_t e0 = (blockIdx.x - t.first_chunk) * kAdamwChunk<k8> + (threadIdx.x >> 5) * kAdamwBlock;
  const uint32_t lane = threadIdx.x & 31;
  constexpr uint32_t kAtOnce = kAdamwAtOnce<k8>, kNext = kAdamwThreads / 32 * kAdamwBlock;
  AdamwLoads<P, G, k8, kV> in[kAtOnce];
#pragma unroll
  for (uint32_t i = 0; i < kAtOnce; ++i)
    if (e0 + i * kNext < t.n) in[i].load(t, e0 + i * kNext, lane);
#pragma unroll
  for (uint32_t i = 0; i < kAtOnce; ++i)
    if (e0 + i * kNext < t.n) adamw_block(in[i], t, a.k, e0 + i * kNext, lane);
}

template <typename P, typename G, bool k8, bool kV, uint32_t kCap>
__global__ void __launch_bounds__(kAdamwThreads, 4) k_adamw(const __grid_constant__ AdamwArgs<kCap> a) {
  adamw_cta<P, G, k8, kV>(a);
}

static uint32_t adamw_kind(const ft_adamw_tensor& t) {
  const bool s8 = t.state_bits == 8;
  const bool vec = aligned_to(t.param, 16) && aligned_to(t.grad, 16) && aligned_to(t.copy, 16) && aligned_to(t.m, s8 ? 8 : 16) &&
                   aligned_to(t.v, s8 ? 8 : 16);
  return (t.param_dtype == FT_BF16 ? kParamBf16 : 0) | (t.grad_dtype == FT_BF16 ? kGradBf16 : 0) | (s8 ? kState8 : 0) | (vec ? kVec : 0);
}

template <typename P, typename G, bool k8, bool kV, uint32_t kCap>
static cudaError_t adamw_launch(const AdamwConst& k, double lr, const ft_adamw_tensor* t, uint32_t n, uint32_t kind, uint64_t chunks, cudaStream_t st) {
  AdamwArgs<kCap> a;
  a.k = k;
  a.n = 0;
  uint64_t at = 0;
  for (uint32_t i = 0; i < n; ++i) {
    if (t[i].n == 0 || adamw_kind(t[i]) != kind) continue;
    AdamwTensorArg& d = a.t[a.n++];
    d.param = t[i].param; d.m = t[i].m; d.v = t[i].v; d.copy = t[i].copy; d.grad = t[i].grad;
    d.m_scale = t[i].m_scale; d.v_scale = t[i].v_scale; d.n = t[i].n; d.first_chunk = at;
    d.keep = (float)(1.0 - lr * t[i].weight_decay);
    at += (t[i].n + kAdamwChunk<k8> - 1) / kAdamwChunk<k8>;
  }
  k_adamw<P, G, k8, kV, kCap><<<(unsigned)chunks, kAdamwThreads, 0, st>>>(a);
  return cudaGetLastError();
}

// The tensors of one kind: as many a launch as its arguments hold and its grid can index.  (One kernel for all kinds, with a
// branch in it, has the registers of its most demanding kind.)
template <typename P, typename G, bool k8, bool kV>
static int32_t adamw_tensors(ft_pool* p, const AdamwConst& k, double lr, const ft_adamw_tensor* t, uint32_t n, uint32_t kind, cudaStream_t st) {
  for (uint32_t i0 = 0; i0 < n;) {
    uint32_t i1 = i0, used = 0;
    uint64_t chunks = 0;
    while (i1 < n && used < kAdamwPerLaunch) {
      const uint64_t c = adamw_kind(t[i1]) == kind ? (t[i1].n + kAdamwChunk<k8> - 1) / kAdamwChunk<k8> : 0;
      if (chunks + c > 0x7FFFFFFFull) break;
      chunks += c;
      used += c != 0;
      ++i1;
    }
    if (chunks) {
      FT_CUDA(used <= kAdamwFew ? (adamw_launch<P, G, k8, kV, kAdamwFew>(k, lr, t + i0, i1 - i0, kind, chunks, st))
                                : (adamw_launch<P, G, k8, kV, kAdamwPerLaunch>(k, lr, t + i0, i1 - i0, kind, chunks, st)));
      p->gpu_launches += 1;
    }
    i0 = i1;
  }
  return FT_OK;
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
  const auto both = [](double x) { return make_float2((float)x, (float)x); };
  AdamwConst k;
  k.b1 = both(cfg->beta1); k.c1 = both(1.0 - cfg->beta1);
  k.b2 = both(cfg->beta2); k.c2 = both(1.0 - cfg->beta2);
  k.step = both(-cfg->lr / (1.0 - std::pow(cfg->beta1, (double)cfg->step)));
  k.inv = both(1.0 / std::sqrt(1.0 - std::pow(cfg->beta2, (double)cfg->step)));
  // the quotient flushes divisors below the normal numbers to zero: m = r = 0 would be 0 / 0
  k.eps = both(cfg->eps > 0.0 ? std::max(cfg->eps, (double)FLT_MIN) : 0.0);
  k.minus_zero = both(-0.0);
  k.grad_scale = cfg->grad_scale;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint32_t kinds = 0;  // a bit a kind that the list has
  for (uint32_t i = 0; i < n_tensors; ++i)
    if (tensors[i].n) kinds |= 1u << adamw_kind(tensors[i]);
  using B = __nv_bfloat16;
  using Run = int32_t (*)(ft_pool*, const AdamwConst&, double, const ft_adamw_tensor*, uint32_t, uint32_t, cudaStream_t);
  static const Run run[16] = {  // by kind
      adamw_tensors<float, float, false, false>, adamw_tensors<B, float, false, false>, adamw_tensors<float, B, false, false>, adamw_tensors<B, B, false, false>,
      adamw_tensors<float, float, true, false>,  adamw_tensors<B, float, true, false>,  adamw_tensors<float, B, true, false>,  adamw_tensors<B, B, true, false>,
      adamw_tensors<float, float, false, true>,  adamw_tensors<B, float, false, true>,  adamw_tensors<float, B, false, true>,  adamw_tensors<B, B, false, true>,
      adamw_tensors<float, float, true, true>,   adamw_tensors<B, float, true, true>,   adamw_tensors<float, B, true, true>,   adamw_tensors<B, B, true, true>};
  for (uint32_t kind = 0; kind < 16; ++kind)
    if (kinds >> kind & 1) {
      const int32_t rc = run[kind](p, k, cfg->lr, tensors, n_tensors, kind, st);
      if (rc != FT_OK) return rc;
    }
  return FT_OK;
}

// What the operators of the backbone's last layer and of its optimizer share: element types, reductions over a warp and
// a block, per-thread asynchronous copies, and the checks of their arguments.
#pragma once
#include <cuda_bf16.h>

#include "flowpool_internal.cuh"

namespace ft {

// Two fp32 values that one instruction takes through an operation, each rounded by itself.
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ F2 f2(float both) { return f2(both, both); }
__device__ __forceinline__ float2 parts(F2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 operator*(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ float sum(F2 a) { const float2 p = parts(a); return p.x + p.y; }

// 16 bytes of a row in its stored type <-> fp32.  Widening bf16 is exact; narrowing rounds to nearest even.
template <typename T>
struct Pack;
template <>
struct Pack<float> {
  static constexpr int kElems = 4;
  static __device__ __forceinline__ void widen(const uint4 v, float* f) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 narrow(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ void widen(const uint4 v, F2* f) {
    f[0] = f2(__uint_as_float(v.x), __uint_as_float(v.y));
    f[1] = f2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ uint4 narrow(const F2* f) {
    const float2 a = parts(f[0]), b = parts(f[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
};
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
struct Pack<__nv_bfloat16> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ void widen(const uint4 v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ uint4 narrow(const float* f) {
    return make_uint4(bf16x2(f[0], f[1]), bf16x2(f[2], f[3]), bf16x2(f[4], f[5]), bf16x2(f[6], f[7]));
  }
  static __device__ __forceinline__ void widen(const uint4 v, F2* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint4 narrow(const F2* f) {
    const float2 a = parts(f[0]), b = parts(f[1]), c = parts(f[2]), d = parts(f[3]);
    return make_uint4(bf16x2(a.x, a.y), bf16x2(b.x, b.y), bf16x2(c.x, c.y), bf16x2(d.x, d.y));
  }
};
__device__ __forceinline__ float widen1(float x) { return x; }
__device__ __forceinline__ float widen1(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T narrow1(float x);
template <>
__device__ __forceinline__ float narrow1<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow1<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// element i of an array whose type is known at run time
__device__ __forceinline__ float load_as(const void* p, uint32_t dtype, uint64_t i) {
  return dtype == FT_F32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
  return x;
}

// NaN wins, unlike in fmaxf
__device__ __forceinline__ float max_with_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float exp2_fast(float x) {  // 2 ulp; results below 2^-126 are zero
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- rows with a label (a token of the vocabulary) and rows without one -------------------------------------------

constexpr int32_t kNoLabel = -100;
__device__ __forceinline__ bool has_label(int32_t l, uint32_t vocab) { return (uint32_t)l < vocab; }

// this thread's share of the rows among the first n that count
__device__ __forceinline__ uint32_t count_labels(const int32_t* labels, uint32_t n, uint32_t vocab) {
  const uint32_t head = min(n, (uint32_t)((16 - (reinterpret_cast<uintptr_t>(labels) & 15)) & 15) / 4), quads = (n - head) / 4;
  uint32_t c = 0;
  if (threadIdx.x < head) c += has_label(labels[threadIdx.x], vocab);
  const int4* q = reinterpret_cast<const int4*>(labels + head);
#pragma unroll 8
  for (uint32_t i = threadIdx.x; i < quads; i += blockDim.x) {
    const int4 l = q[i];
    c += has_label(l.x, vocab) + has_label(l.y, vocab) + has_label(l.z, vocab) + has_label(l.w, vocab);
  }
  const uint32_t r = head + 4 * quads + threadIdx.x;
  if (r < n) c += has_label(labels[r], vocab);
  return c;
}

// 32 bytes in one access: a whole sector a lane, where 16 bytes would write it in halves
__device__ __forceinline__ void store32(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// 16 bytes at a shared-memory address (32 bits: a generic pointer kept in a structure is read as one, at twice the latency)
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16_async(uint32_t shared_dst, const void* gmem_src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(shared_dst), "l"(gmem_src) : "memory");
}
__device__ __forceinline__ uint4 load_shared16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void store_shared16(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A chain of kernels of one call: each lets the next one be set up while it runs, and waits at its start for the one before
// (which has waited for the one before it) to have ended with its stores visible.  Such a kernel takes no `const __restrict__`
// pointer and no __ldg to memory that the one before writes: those loads need not stay behind the wait.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... P, typename... A>
inline cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, uint32_t threads, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<A&&>(args)...);
}

inline bool dtype_ok(uint32_t t) { return t == FT_BF16 || t == FT_F32; }
inline uint32_t dtype_size(uint32_t t) { return t == FT_F32 ? 4u : 2u; }
inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// A matrix written where one is read has that one's stride: with another, a row lands on rows that are still to be read.
inline bool on_other_rows(uint64_t rows, const void* out, uint64_t ld_out, const void* in, uint64_t ld_in) {
  return out && out == in && rows > 1 && ld_out != ld_in;
}
inline bool on_pool_device(const ft_pool* p) {
  int d = -1;
  return cudaGetDevice(&d) == cudaSuccess && d == p->device;
}

}  // namespace ft

#define FT_EXPORT extern "C" __attribute__((visibility("default")))

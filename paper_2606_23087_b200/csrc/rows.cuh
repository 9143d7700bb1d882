// Rows of a matrix that groups of threads go through: what the norms share.  Asynchronous row feeds, sums over a block, launch geometry.
#pragma once
#include <algorithm>
#include <utility>

#include "operators.cuh"

namespace ft {

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
  __device__ __forceinline__ void take_chunk(uint32_t stage, int k, F2 (&f)[kVec ? E / 2 : 1]) const {  // one of them, from shared memory
    if constexpr (kVec) Pack<T>::widen(load_shared16(slot + (stage * V + k) * kThreads * 16), f);
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

constexpr size_t kSmemMost = 227 * 1024;  // of a CTA

// f with the number n of `list` as a constant
template <typename F, int... N>
inline void with_number(uint32_t n, std::integer_sequence<int, N...>, F&& f) {
  (void)((n == (uint32_t)N && (f(std::integral_constant<int, N>{}), true)) || ...);
}
template <typename K>
inline cudaError_t allow_smem(K kernel, size_t smem) {
  return smem > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) : cudaSuccess;
}

// Threads a row: multiples of 32, so that few of them have nothing (3584 bf16 elements are 224 threads x 2 chunks of 8).
template <typename F>
inline void with_threads(uint32_t n, F&& f) {
  with_number(n <= 256 ? (n + 31) / 32 * 32 : (n + 127) / 128 * 128, std::integer_sequence<int, 32, 64, 96, 128, 160, 192, 224, 256, 384, 512>{}, f);
}

template <typename T, bool kVec, int kElems>
constexpr int kChunks = kVec ? (kElems < Pack<T>::kElems ? 1 : kElems / Pack<T>::kElems) : kElems;

inline bool rows_in_16(const void* p, uint64_t ld, uint32_t es) { return aligned_to(p, 16) && ld * es % 16 == 0; }

}  // namespace ft

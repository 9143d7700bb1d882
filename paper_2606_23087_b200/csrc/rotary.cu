// Rotary positions with several axes over the heads of queries, keys, or their gradients.
//
//   angle_i = pos[axis_i][row] freq_i;  (a, b) -> (a cos - b sin, a sin + b cos) for the pair i of every head
//
// The rotation's transpose is the rotation by the negated angle: one kernel serves both directions.
//
// Angles.  A position times a frequency loses what matters of a far position's angle in fp32 (at 10^5 some 2^-7 radians), so
// the angle is taken in turns, as a 64-bit fraction: the host rounds freq / 2 pi modulo one turn to 64 bits, the product with
// a 32-bit position wraps modulo one turn by itself.  freq / 2 pi, below 1.28, is off by 1.64 x 2^-64 as an 80-bit product, by half of 2^-64
// each where a turn is added and where it is rounded: the angle by less than 2^-31 of a turn for any position.  Its rounding to fp32, for the
// sine, is up to 2^-26 of a turn.
//
// Bound by HBM: every element is read and written once.  32768 rows x 32 heads x 128 in bf16: 82 us (6.55 TB/s, the copy rate).  A CTA
// works out the sines and cosines of its rows once into shared memory; a thread takes the same pairs of one head in each of its rows,
// which are on their way while the table is made.
#include <algorithm>
#include <cmath>

#include "operators.cuh"

namespace ft {

constexpr uint32_t kRotaryThreads = 256;
constexpr uint32_t kRotaryTensors = 4;  // of one launch

struct RotaryTensorArg {
  const void* src;
  void* dst;
  uint64_t src_row, src_head, dst_row, dst_head;
  uint32_t heads_end;  // heads of the tensors up to this one
};
struct RotaryArgs {
  uint64_t rows, pos_ld;
  const int32_t* pos;
  uint32_t pairs, dim, heads, n;       // heads: of all tensors
  uint32_t units, turned, slots;       // of a head: pieces of work, those of them that turn; heads that a CTA takes at a time
  RotaryTensorArg t[kRotaryTensors];
  uint64_t turns[FT_ROTARY_MAX_PAIRS];  // of pair i at position 1, in 2^-64
  uint8_t axis[FT_ROTARY_MAX_PAIRS];
};

// One piece of work of a head: kE pairs (two accesses of kE elements), or as many elements behind the last pair to be copied.
template <typename T, int kE>
struct RotaryPiece {
  static constexpr bool kVec = kE > 1;
  T x[2 * kE];
  static __device__ __forceinline__ void move(T* to, const T* from) {
    if constexpr (kVec) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
    else *to = *from;
  }
  __device__ __forceinline__ void load(const T* p, uint32_t second, bool two) {
    move(x, p);
    if (two) move(x + kE, p + second);
  }
  __device__ __forceinline__ void store(T* p, uint32_t second, bool two) const {
    move(p, x);
    if (two) move(p + second, x + kE);
  }
  // cs: the table's place of the piece's first pair (see rotary_place)
  template <bool kInterleaved>
  __device__ __forceinline__ void turn(const float2* cs, uint32_t turned) {
    float2 c[kE];
    if constexpr (kVec) {
#pragma unroll
      for (int i = 0; i < kE; i += 2) *reinterpret_cast<float4*>(c + i) = *reinterpret_cast<const float4*>(cs + i * turned);
    } else {
      c[0] = cs[0];
    }
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      T &ta = kInterleaved ? x[2 * i] : x[i], &tb = kInterleaved ? x[2 * i + 1] : x[kE + i];
      const float a = widen1(ta), b = widen1(tb);
      ta = narrow1<T>(fmaf(a, c[i].x, -(b * c[i].y)));
      tb = narrow1<T>(fmaf(a, c[i].y, b * c[i].x));
    }
  }
};
// Where the table holds pair p: two pairs of each piece side by side, then the next two of each, so that the pieces of a head, which
// neighbouring lanes hold, read one range (a piece's pairs in a row were read at a quarter of the rate, and bound the kernel).
template <int kE>
__device__ __forceinline__ uint32_t rotary_place(uint32_t p, uint32_t turned) {
  if constexpr (kE == 1) return p;
  const uint32_t piece = p / kE, i = p % kE;
  return (i / 2 * turned + piece) * 2 + i % 2;
}

// An element of the tables among the arguments, by an ordinary load: lanes that index constant memory each by themselves are served one
// after the other.
__device__ __forceinline__ uint64_t load_argument(const uint64_t* p) { uint64_t v; asm("ld.u64 %0, [%1];" : "=l"(v) : "l"(p)); return v; }
__device__ __forceinline__ uint32_t load_argument(const uint8_t* p) { uint32_t v; asm("ld.u8 %0, [%1];" : "=r"(v) : "l"(p)); return v; }

// CTA (row tile, heads): kRows rows, `slots` heads.  kE: pairs of a piece, 16 bytes of each element's row or a single one.
template <typename T, int kE, bool kInterleaved, int kRows>
__global__ void __launch_bounds__(kRotaryThreads) k_rotary(const __grid_constant__ RotaryArgs a) {
  extern __shared__ __align__(16) float2 table[];  // [kRows][pairs]
  let_next_start();
  after_previous();
  const uint64_t row0 = (uint64_t)blockIdx.x * kRows;
  const uint32_t rows = (uint32_t)min((uint64_t)kRows, a.rows - row0);
  const uint32_t slot = threadIdx.x / a.units, unit = threadIdx.x - slot * a.units, head = blockIdx.y * a.slots + slot;
  const bool active = slot < a.slots && head < a.heads, turned = unit < a.turned;
  RotaryPiece<T, kE> piece[kRows];
  // where the piece lies in its head, how far its second half is, and whether there is one (the last copied piece may be half)
  uint32_t at, second;
  if (turned) {
    at = kInterleaved ? unit * 2 * kE : unit * kE;
    second = kInterleaved ? kE : a.pairs;
  } else {
    at = 2 * a.pairs + (unit - a.turned) * 2 * kE;
    second = kE;
  }
  const bool two = at + second < a.dim;
  uint32_t which = 0;
#pragma unroll
  for (uint32_t i = 0; i + 1 < kRotaryTensors; ++i) which += i + 1 < a.n && head >= a.t[i].heads_end;
  const RotaryTensorArg& t = a.t[which];
  const uint32_t h = head - (which ? a.t[which - 1].heads_end : 0);
  if (active) {
    const T* src = static_cast<const T*>(t.src) + row0 * t.src_row + h * t.src_head + at;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      if (r < rows) piece[r].load(src + r * t.src_row, second, two);
  }
  for (uint32_t i = threadIdx.x; i < rows * a.pairs; i += kRotaryThreads) {
    const uint32_t r = i / a.pairs, p = i - r * a.pairs;
    const int32_t position = a.pos[load_argument(a.axis + p) * a.pos_ld + row0 + r];
    const int64_t turns = (int64_t)(load_argument(a.turns + p) * (uint64_t)(int64_t)position);  // of a turn, from -1/2 on
    float s, c;
    sincospif((float)turns * 0x1p-63f, &s, &c);
    table[r * a.pairs + rotary_place<kE>(p, a.turned)] = make_float2(c, s);
  }
  __syncthreads();
  if (!active) return;
  T* dst = static_cast<T*>(t.dst) + row0 * t.dst_row + h * t.dst_head + at;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= rows) break;
    if (turned) piece[r].template turn<kInterleaved>(table + r * a.pairs + unit * (kE == 1 ? 1 : 2), a.turned);
    piece[r].store(dst + r * t.dst_row, second, two);
  }
}

// Rows of a CTA: four, so that a thread has 128 bytes on their way; one where that gives fewer CTAs than SMs.
template <typename T, int kE, bool kInterleaved>
static cudaError_t rotary_launch(const ft_pool* p, RotaryArgs& a, cudaStream_t st) {
  a.turned = a.pairs / kE;
  const uint32_t rest = a.dim - 2 * a.pairs, copied = (rest + 2 * kE - 1) / (2 * kE);
  bool in_place = true;
  for (uint32_t i = 0; i < a.n; ++i) in_place &= a.t[i].src == a.t[i].dst;
  a.units = a.turned + (in_place ? 0 : copied);
  a.slots = std::max(1u, std::min(a.heads, kRotaryThreads / a.units));
  const uint32_t y = (a.heads + a.slots - 1) / a.slots;
  if ((a.rows + 3) / 4 * y < (uint64_t)p->sm_count)
    return launch_chained(k_rotary<T, kE, kInterleaved, 1>, dim3((unsigned)a.rows, y), kRotaryThreads, a.pairs * sizeof(float2), st, a);
  return launch_chained(k_rotary<T, kE, kInterleaved, 4>, dim3((unsigned)((a.rows + 3) / 4), y), kRotaryThreads, 4 * a.pairs * sizeof(float2), st, a);
}

template <typename T>
static cudaError_t rotary_typed(const ft_pool* p, RotaryArgs& a, bool interleaved, bool vec, cudaStream_t st) {
  constexpr int E = Pack<T>::kElems;
  if (vec) return interleaved ? rotary_launch<T, E, true>(p, a, st) : rotary_launch<T, E, false>(p, a, st);
  return interleaved ? rotary_launch<T, 1, true>(p, a, st) : rotary_launch<T, 1, false>(p, a, st);
}

// every access of 16 bytes of the tensor's heads starts on a 16-byte boundary
static bool rotary_in_16(const ft_rotary_tensor& t) {
  const uint64_t es = dtype_size(t.dtype), strides = t.dst_row | t.dst_head | t.src_row | t.src_head;
  return aligned_to(t.src, 16) && aligned_to(t.dst, 16) && strides * es % 16 == 0;
}

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_rotary(ft_pool* p, uint64_t rows, const int32_t* pos, uint64_t pos_ld, const ft_rotary_config* cfg,
                              const ft_rotary_tensor* tensors, uint32_t n_tensors, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (!cfg || !cfg->freq || cfg->pairs == 0 || cfg->head_dim < 2ull * cfg->pairs || (n_tensors && !tensors)) return FT_ERR_INVALID_ARG;
  if (cfg->head_dim > FT_ROTARY_MAX_DIM || rows >> 31) return FT_ERR_CAPACITY;
  RotaryArgs a;
  uint32_t axes = 0;
  for (uint32_t i = 0; i < cfg->pairs; ++i) {
    const double f = cfg->freq[i];
    a.axis[i] = cfg->axis ? cfg->axis[i] : 0;
    if (!(std::fabs(f) <= 8.0) || a.axis[i] > 2) return FT_ERR_INVALID_ARG;
    axes = std::max<uint32_t>(axes, a.axis[i]);
    long double t = f * 0.159154943091895335768883763372514362L;  // turns a position, of which whole ones count nothing
    t -= (long double)(int64_t)t;
    if (t < 0) t += 1;
    const long double units = t * 0x1p64L;
    uint64_t u = units < 0x1p64L ? (uint64_t)units : 0;
    if (units < 0x1p64L && units - (long double)u >= 0.5L) ++u;
    a.turns[i] = cfg->inverse ? 0 - u : u;
  }
  if (rows && (!pos || !aligned_to(pos, 4) || (axes && pos_ld < rows))) return FT_ERR_INVALID_ARG;
  for (uint32_t i = 0; i < n_tensors; ++i) {
    const ft_rotary_tensor& t = tensors[i];
    if (!dtype_ok(t.dtype)) return FT_ERR_INVALID_ARG;
    if (t.heads == 0 || rows == 0) continue;
    if (t.heads > FT_ROTARY_MAX_HEADS) return FT_ERR_CAPACITY;
    const uint32_t es = dtype_size(t.dtype);
    if (!t.src || !t.dst || !aligned_to(t.src, es) || !aligned_to(t.dst, es)) return FT_ERR_INVALID_ARG;
    // heads of a row and rows apart from one another in what is written
    const uint64_t heads = t.heads, dim = cfg->head_dim;
    if ((heads > 1 && t.dst_head < dim) || (rows > 1 && t.dst_row < dim) ||
        (heads > 1 && rows > 1 && t.dst_row < (heads - 1) * t.dst_head + dim && t.dst_head < (rows - 1) * t.dst_row + dim))
      return FT_ERR_INVALID_ARG;
    if (t.src == t.dst && (t.src_row != t.dst_row || t.src_head != t.dst_head)) return FT_ERR_INVALID_ARG;
  }
  if (rows == 0) return FT_OK;
  a.rows = rows; a.pos = pos; a.pos_ld = pos_ld; a.pairs = cfg->pairs; a.dim = cfg->head_dim;
  // tensors of one type that all take 16-byte accesses, or all do not, share launches
  for (uint32_t kind = 0; kind < 4; ++kind) {
    const uint32_t dtype = kind & 1 ? FT_F32 : FT_BF16, e = 16 / dtype_size(dtype);
    const bool vec = (kind & 2) != 0;
    a.n = a.heads = 0;
    const auto launch = [&]() -> int32_t {
      if (a.n == 0) return FT_OK;
      cudaStream_t st = static_cast<cudaStream_t>(stream);
      FT_CUDA(dtype == FT_F32 ? rotary_typed<float>(p, a, cfg->interleaved, vec, st) : rotary_typed<__nv_bfloat16>(p, a, cfg->interleaved, vec, st));
      p->gpu_launches += 1;
      a.n = a.heads = 0;
      return FT_OK;
    };
    for (uint32_t i = 0; i < n_tensors; ++i) {
      const ft_rotary_tensor& t = tensors[i];
      if (t.heads == 0 || t.dtype != dtype || (rotary_in_16(t) && cfg->pairs % e == 0 && cfg->head_dim % e == 0) != vec) continue;
      a.heads += t.heads;
      a.t[a.n++] = RotaryTensorArg{t.src, t.dst, t.src_row, t.src_head, t.dst_row, t.dst_head, a.heads};
      if (a.n == kRotaryTensors) {
        const int32_t rc = launch();
        if (rc != FT_OK) return rc;
      }
    }
    const int32_t rc = launch();
    if (rc != FT_OK) return rc;
  }
  return FT_OK;
}

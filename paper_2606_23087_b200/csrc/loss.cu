// Softmax cross entropy of rows against a vocabulary, with its gradients, without a matrix of logits.
//
//   z = x W^T,  lse = log(sum(exp(z))),  loss = lse - z[label]
//   d = g (exp(z - lse) - [v = label]),  dx = d W,  dW = d^T x
//
//   k_pick    takes the rows that count out of a piece of the rows: a dense copy of their x, their labels and row
//             numbers.  Rows labelled -100 cost no products, and what they hold cannot reach dW as 0 * NaN.  It also
//             takes each row's reference: the label's logit, x . W[label], by fp32 FMAs
//   k_logits  z by tiles; a row of a tile gives the sum of e = exp(z - reference) over the columns that are not its label,
//             and with gradients e itself in bf16 (rounding e costs 2^-8 of a probability, rounding z would cost 2^-8 of z)
//   k_join    adds a row's sums to S: loss = log(1 + S), lse = reference + loss
//   k_finish  d = f e with one factor f = g exp(reference - lse) a row: f goes to the row's x for dW (rounded to bf16; for few rows as two bf16 values) and to
//             the row's sums for dx, so e is not touched again but for the label's element, (exp(-loss) - 1) exp(lse - reference)
//   k_dx, k_dw  the two products
//
// Bound by the tensor cores, long calls by the card's power limit: 16384 rows that count x 32768 x 3584 with gradients 8.4 to 8.9 ms (1.29 to
// 1.37 PFLOP/s), 2460 x 32768 x 1024 470 to 483 us (1.02 to 1.05 PFLOP/s); few rows by W and launches: 24 x 32768 x 1024 forward 33 to 34 us, with
// gradients 95.
//
// Why a reference known before any logit: with each tile's own maximum, the usual choice, e has to be read, scaled and
// written again once lse is known (1.1 ms of 10.7 for 16384 rows x 32768).  bf16 has fp32's range, so any reference that is not
// far below lse serves as well as the maximum; the label's logit is that, unless a row's loss is above 41.  Such a row gets its
// maximum as reference, and its row tile's logits are worked out once more (k_logits<., true, .>, which returns at once where
// there is none): one such row in each 256 of 16384 x 32768 x 3584 makes the forward call 5.9 ms instead of 2.5.  And it makes small losses exact: the label's term of the sum is 1, not a difference of two large numbers,
// and the tensor cores' truncating additions do not touch the one logit that a loss depends on most (2.6e-6 -> 0.7e-6 of the loss
// over 3584; see kPartBlocks for the rest).
#include <algorithm>

#include "mma_pair.cuh"

namespace ft {

constexpr uint32_t kStatCols = 128;  // columns of the vocabulary that share a row's sum
constexpr uint32_t kTileCost = 6;    // what a tile of dx costs beside its products, in blocks of K
// The tensor cores truncate at every addition of 16 products, all one way, which shows in a loss as 0.24e-6 of it for each 1024 of K.
// Tiles of 256 rows are summed in parts of kPartBlocks blocks of K, the parts joined in registers: 0.2e-6 at any K, for 3 to 5 % of a call
// (200 rows x 32768 x 3584 76.6 -> 80.4 us; parts of 8 blocks 83.8).  Tiles of 512 rows have no registers for that: they are for
// rows beyond 256 and K up to kHighBlocks blocks, where a loss comes to be off by 1e-6 (3000 rows x 32768 x 5120, with gradients: 2.39 ms
// in parts, 2.24 ms in high tiles and off by 1.2e-6).
constexpr uint32_t kPartBlocks = 16;
// Rounding f x to bf16 makes dW's error 2.3e-3 of its norm, where the rounding of a bf16 dW alone is 1.7e-3.  Up to kTwiceUpTo rows, where
// dW's bytes and not the product take the time, x goes in as two bf16 values, over twice the K: 1.7e-3, for 2 to 3 % of the call (60 rows x
// 32768 x 3584 195 -> 199 us); 250 rows would pay 17 % (219 -> 256 us).
constexpr uint32_t kTwiceUpTo = 128;
static_assert(2 * kTwiceUpTo <= kMmaTile, "both values of f x fit in xc");
constexpr uint32_t kHighBlocks = 66;
constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kMinusInf = 0xFF800000u;
constexpr float kSumLimit = 0x1p60f;  // a row's sum above this wants another reference
constexpr int32_t kNoLabel = -100;
constexpr uint32_t kPieceRowsMost = 65536;
constexpr uint32_t kHighRows = 2 * kMmaTile;  // rows of a tile of dx and dw

struct LossPiece {
  uint32_t rows, hidden, vocab, ld_p, tiles, slots;  // tiles: of kStatCols columns; slots: tiles that dx_slots holds
  uint32_t padded;  // rows of xc and p: `rows` in whole tiles
  uint32_t twice;   // dw takes f x as two bf16 values, the second one behind the whole blocks of K of the first
  uint32_t pairs;   // CTA pairs of the products
  uint64_t row0, ldx, ldw, lddx;
  const __nv_bfloat16 *x, *w;
  const int32_t* labels;
  const float* grad_loss;
  uint32_t grad_stride, dw_dtype, add_dw, last;
  float *loss, *lse;
  __nv_bfloat16* dx;
  void* dw;
  uint64_t call_seq;
  // workspace
  uint32_t* count;         // rows of the piece that count; slices of dx's product
  int32_t *row_of, *label; // [count] row in the piece, label
  uint32_t* redo;          // [1 + row tiles] whether any, and which row tiles need another reference
  float *ref, *target;     // [count] the reference, and the label's logit
  float* factor;           // [count] lse - reference, then f
  float2* stat;            // [tiles][rows] maximum of z and sum of e of a row in a tile, the label's column apart
  __nv_bfloat16* xc;       // [padded][hidden]
  __nv_bfloat16* p;        // [padded][ld_p] e
  float* dx_slots;         // [slots][256][512] dx by slices of the vocabulary and tiles, columns first
  float* dw_acc;           // [vocab][hidden]: bf16 dw of several pieces
};

constexpr uint32_t kPickRows = 32;    // rows of a CTA; 8 where that alone fills the device, a row a warp
constexpr uint32_t kPickFew = 8;
constexpr uint32_t kPickFewUpTo = 4096;

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

// A CTA takes kRows rows; where they go it learns by counting the labels before them itself (a piece's labels stay in L2),
// so nothing has to wait for another CTA.
template <uint32_t kRows>
__global__ void __launch_bounds__(256) k_pick(PoolView v, LossPiece a) {
  __shared__ uint32_t warp_count[8];
  __shared__ int32_t dest[32], s_label[32];
  __shared__ uint8_t s_from[32];  // the rows of the CTA that count, in order
  let_next_start();
  const uint32_t r0 = blockIdx.x * kRows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t* labels = a.labels + a.row0;
  if (blockIdx.x == 0)
    for (uint32_t i = threadIdx.x; i <= a.padded / kMmaTile; i += blockDim.x) a.redo[i] = 0;
  const uint32_t mine = __reduce_add_sync(0xFFFFFFFFu, count_labels(labels, r0, a.vocab));
  if (lane == 0) warp_count[warp] = mine;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) before += warp_count[w];
  const uint32_t r = r0 + lane;
  const int32_t l = lane < kRows && r < a.rows ? labels[r] : kNoLabel;
  const bool counts = has_label(l, a.vocab);
  const uint32_t mask = __ballot_sync(0xFFFFFFFFu, counts), pos = before + __popc(mask & ((1u << lane) - 1)), total = before + __popc(mask);
  if (warp == 0) {
    dest[lane] = counts ? (int32_t)pos : -1;
    s_label[lane] = l;
    if (counts) {
      s_from[pos - before] = (uint8_t)lane;
      a.row_of[pos] = (int32_t)r;
      a.label[pos] = l;
    } else if (lane < kRows && r < a.rows) {
      a.loss[a.row0 + r] = 0.f;
      a.lse[a.row0 + r] = 0.f;
      if (l != kNoLabel) note_error(v, a.call_seq, FT_ERR_BAD_TOKEN_ID, (uint32_t)(a.row0 + r));
    }
    if (blockIdx.x == gridDim.x - 1 && lane == 0) *a.count = total;
  }
  __syncthreads();
  const uint32_t vecs = a.hidden / 8, rows = min(kRows, a.rows - r0);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  if (blockIdx.x == gridDim.x - 1) {  // the product over rows runs to a whole block of K: those rows' x must be finite
    const uint32_t end = (total + kMmaK - 1) / kMmaK * kMmaK;
    uint4* tail = reinterpret_cast<uint4*>(a.xc + (uint64_t)total * a.hidden);
    for (uint32_t c = threadIdx.x; c < (end - total) * vecs; c += blockDim.x) {
      tail[c] = zero;
      if (a.twice) tail[(uint64_t)end * vecs + c] = zero;
    }
  }
  for (uint32_t k = warp; k < rows; k += 8)
    if (a.dx && dest[k] < 0) {
      uint4* dst = reinterpret_cast<uint4*>(a.dx + (a.row0 + r0 + k) * a.lddx);
      for (uint32_t c = lane; c < vecs; c += 32) dst[c] = zero;
    }
  // the rows that count, two a warp at a time (a short row's loads alone do not cover memory's latency) where there are many
  constexpr uint32_t kAtOnce = kRows == kPickFew ? 1 : 2;
  for (uint32_t q = kAtOnce * warp; q < total - before; q += kAtOnce * 8) {
    const uint4 *src[kAtOnce], *wl[kAtOnce];
    float dot[kAtOnce] = {};
    const uint32_t two = min(kAtOnce, total - before - q);
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i) {
      const uint32_t k = s_from[q + (i < two ? i : 0)];
      src[i] = reinterpret_cast<const uint4*>(a.x + (a.row0 + r0 + k) * a.ldx);
      wl[i] = reinterpret_cast<const uint4*>(a.w + (uint64_t)s_label[k] * a.ldw);
    }
    uint4* __restrict__ dst = reinterpret_cast<uint4*>(a.xc + (uint64_t)(before + q) * a.hidden);
#pragma unroll(4 / kAtOnce)
    for (uint32_t c = lane; c < vecs; c += 32) {
      uint4 xv[kAtOnce], wv[kAtOnce];
#pragma unroll
      for (uint32_t i = 0; i < kAtOnce; ++i) { xv[i] = __ldg(src[i] + c); wv[i] = __ldg(wl[i] + c); }
#pragma unroll
      for (uint32_t i = 0; i < kAtOnce; ++i) {
        float f[8], g[8];
        Pack<__nv_bfloat16>::widen(xv[i], f);
        Pack<__nv_bfloat16>::widen(wv[i], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot[i] = fmaf(f[e], g[e], dot[i]);
        if (i < two) dst[i * vecs + c] = xv[i];
      }
    }
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i) {
      const float d = warp_sum(dot[i]);
      if (lane == 0 && i < two) a.ref[before + q + i] = a.target[before + q + i] = d;
    }
  }
}

// ---- the three products ---------------------------------------------------------------------------------------------

__device__ __forceinline__ float exp2_fast(float x) {  // 2 ulp; results below 2^-126 are zero
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 32 bytes in one access: a whole sector a lane, where 16 bytes would write it in halves
__device__ __forceinline__ void store32(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void load32(const float* p, float (&v)[8]) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(p) : "memory");
}

__device__ __forceinline__ void give_up(const PoolView& v, uint64_t call_seq, bool lost) {
  if (lost && threadIdx.x == 0) note_error(v, call_seq, FT_ERR_TIMEOUT, blockIdx.x);
}

// z by tiles; a lane owns a row's 128 columns.  kRedo: only the row tiles whose reference has changed.
template <bool kKeep, bool kRedo, int kHigh>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
k_logits(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_e,
         const __grid_constant__ PoolView v, const __grid_constant__ LossPiece a) {
  __shared__ uint8_t s_tile[kRedo ? kPieceRowsMost / kMmaTile : 1];
  __shared__ uint32_t s_tiles;
  let_next_start();
  after_previous();
  const uint32_t n = *a.count, n_tiles = (a.vocab + kMmaTile - 1) / kMmaTile, k_blocks = (a.hidden + kMmaK - 1) / kMmaK;
  uint32_t blocks = (n + kMmaTile - 1) / kMmaTile;
  if constexpr (kRedo) {
    if (a.redo[0] == 0) return;
    if (threadIdx.x == 0) {
      uint32_t c = 0;
      for (uint32_t t = 0; t < blocks; ++t)
        if (a.redo[1 + t]) s_tile[c++] = (uint8_t)t;
      s_tiles = c;
    }
    __syncthreads();
    blocks = s_tiles;
  }
  const uint32_t m_tiles = (blocks + kHigh - 1) / kHigh, tiles = m_tiles * n_tiles;
  // A pair takes the parts of a tile's K one after the other.
  constexpr uint32_t kPart = kHigh == 1 ? kPartBlocks : 0xFFFFFFu;
  const uint32_t k_parts = (k_blocks + kPart - 1) / kPart;
  bool lost;
  uint32_t z[kStatCols / 32][32];
  int32_t label = kNoLabel;
  float ref = 0.f;
  mma_pair_tiles<false, false, kHigh>(map_x, map_w, (tiles + a.pairs - 1) / a.pairs * a.pairs * k_parts, v, &lost,
    [&](uint32_t item) {
      const uint32_t round = item / a.pairs, i = item % a.pairs + round / k_parts * a.pairs, part = round % k_parts;
      if (i >= tiles) return MmaTile{0, 0, 0, 0, 0};
      // bands of 2048 rows, all columns of a band before the next: a band's x stays in L2
      constexpr uint32_t kBand = 8 / kHigh;
      const uint32_t band = i / (kBand * n_tiles), in = i - band * kBand * n_tiles, rows = min(kBand, m_tiles - band * kBand), m = band * kBand + in % rows;
      return MmaTile{(kRedo ? (uint32_t)s_tile[m] : m * kHigh) * kMmaTile, in / rows * kMmaTile, part * kPart, min((part + 1) * kPart, k_blocks),
                     min((uint32_t)kHigh, blocks - m * kHigh)};
    },
    [&](const MmaTile& t, uint32_t row) {
      const uint32_t m = t.m + row + (threadIdx.x & 31);
      label = m < n ? a.label[m] : kNoLabel;
      ref = m < n ? a.ref[m] : 0.f;
    },
    [&](const MmaTile& t, uint32_t, uint32_t tmem, uint32_t row, uint32_t col0, auto&& release) {
      const uint32_t c0 = t.n + col0;
      if (c0 >= a.vocab) return;
      if (kHigh == 2 || t.k0 == 0) {
#pragma unroll
        for (uint32_t c = 0; c < kStatCols / 32; ++c) tmem_load32(tmem + 32 * c, z[c]);
        tmem_wait();
      } else {
#pragma unroll
        for (uint32_t c = 0; c < kStatCols / 32; ++c) {
          uint32_t part[32];
          tmem_load32(tmem + 32 * c, part);
          tmem_wait();
#pragma unroll
          for (uint32_t j = 0; j < 32; ++j) z[c][j] = __float_as_uint(__uint_as_float(z[c][j]) + __uint_as_float(part[j]));
        }
      }
      release();  // the products go on while the exponentials are taken
      if (kHigh == 1 && t.k1 < k_blocks) return;
      const uint32_t m = t.m + row + (threadIdx.x & 31), cols = min(kStatCols, a.vocab - c0);
      const uint32_t label_at = (uint32_t)label - c0;
      [[maybe_unused]] const uint32_t keep = m < n ? 0xFFFFFFFFu : 0u;  // rows beyond the last one that counts: zeros, which the product over rows adds
      if (label_at < kStatCols) {
#pragma unroll
        for (uint32_t j = 0; j < kStatCols; ++j)
          if (j == label_at) z[j / 32][j % 32] = kMinusInf;
      }
      if (cols < kStatCols) {  // beyond the vocabulary
#pragma unroll
        for (uint32_t j = 0; j < kStatCols; ++j)
          if (j >= cols) z[j / 32][j % 32] = kMinusInf;
      }
      float top = -INFINITY;
      F2 sums = f2(0.f);
      const F2 minus_ref = f2(-ref), scale = f2(kLog2e);
      const auto take_exp = [&](uint32_t c) {  // of two columns
        const float x0 = __uint_as_float(z[c / 32][c % 32]), x1 = __uint_as_float(z[c / 32][c % 32 + 1]);
        const float2 t = parts((f2(x0, x1) + minus_ref) * scale);
        const F2 e = f2(exp2_fast(t.x), exp2_fast(t.y));
        top = fmaxf(top, fmaxf(x0, x1));
        sums = sums + e;
        return e;
      };
      if constexpr (kKeep) {
#pragma unroll
        for (uint32_t c = 0; c < kStatCols; c += 64) {
          if (c >= cols) break;
          MmaOut().put<false>(&map_e, (int32_t)(c0 + c), (int32_t)(t.m + row), [&](uint32_t j) {
            F2 e[4];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) e[k] = take_exp(c + 8 * j + 2 * k);
            const uint4 w = Pack<__nv_bfloat16>::narrow(e);
            return make_uint4(w.x & keep, w.y & keep, w.z & keep, w.w & keep);
          });
        }
      } else {
#pragma unroll
        for (uint32_t c = 0; c < kStatCols; c += 2) take_exp(c);
      }
      if (m < n) a.stat[(uint64_t)(c0 / kStatCols) * a.rows + m] = make_float2(top, sum(sums));
    });
  give_up(v, a.call_seq, lost);
}

// The work of a product in tiles of 512 rows.  Tile `t` of `all` = m_tiles x n_tiles (columns first) x slices of K;
// where the last round has 512-row tiles for at most half the pairs, those are dealt out as two 256-row halves.
struct HighTiles {
  uint32_t blocks, n_tiles, tiles, all, split;  // blocks: of 256 rows; tiles: of one slice; split: whole tiles in front of the halves
  __device__ __forceinline__ HighTiles(uint32_t rows, uint32_t cols, uint32_t slices, uint32_t pairs) {
    blocks = (rows + kMmaTile - 1) / kMmaTile;
    n_tiles = (cols + kMmaTile - 1) / kMmaTile;
    tiles = (blocks + 1) / 2 * n_tiles;
    all = split = tiles * slices;
    const uint32_t rest = all % pairs;
    if (blocks > 1 && rest * 2 <= pairs) split -= rest;
  }
  __device__ __forceinline__ uint32_t items() const { return split + 2 * (all - split); }
  // rounds of all pairs, in tiles of 256 rows
  __device__ __forceinline__ uint32_t rounds(uint32_t pairs) const {
    return min(2u, blocks) * ((split + pairs - 1) / pairs) + (split < all ? 1 : 0);
  }
  __device__ __forceinline__ uint32_t tile_of(uint32_t i) const { return i < split ? i : split + (i - split) / 2; }
  __device__ __forceinline__ MmaTile at(uint32_t i, uint32_t k_each, uint32_t k_blocks) const {
    const uint32_t tile = tile_of(i), slice = tile / tiles, t = tile - slice * tiles, half = i < split ? 0 : (i - split) & 1;
    const uint32_t block = t / n_tiles * 2 + half, left = blocks > block ? blocks - block : 0;
    return MmaTile{block * kMmaTile, t % n_tiles * kMmaTile, min(slice * k_each, k_blocks), min((slice + 1) * k_each, k_blocks),
                   min(i < split ? 2u : 1u, left)};
  }
};

// Slices of K = vocab for dx's tiles: they rarely divide among the pairs, and few rows have few tiles at all.  Taken is the
// number of slices with the least rounds of tiles times blocks of K a tile, plus what a tile costs beside its products and
// what the slices cost in traffic (in blocks of K of 256 rows, some 0.35 us).  Not sensitive: kTileCost from 1 to 10 is within
// 1 % at 200 to 5000 rows.
__device__ __forceinline__ uint32_t dx_slices(const LossPiece& a, uint32_t n) {  // a whole warp: a lane a number of slices
  const uint32_t k_blocks = (a.vocab + kMmaK - 1) / kMmaK, s = (threadIdx.x & 31) + 1;
  const HighTiles h(n, a.hidden, s, a.pairs);
  uint32_t cost = h.rounds(a.pairs) * ((k_blocks + s - 1) / s + kTileCost) + (s > 1 ? s * h.blocks * h.n_tiles / 4 : 0);
  if (s > k_blocks || (s > 1 && h.all > a.slots)) cost = 0x7FFFFFFu;
  const uint32_t best = __reduce_min_sync(0xFFFFFFFFu, cost);
  return __ffs(__ballot_sync(0xFFFFFFFFu, cost == best));
}

// ---- joining the tiles of a row -------------------------------------------------------------------------------------

// 32 rows a CTA, a lane a row, the CTA's warps share the tiles; warp 0 gets the result.
constexpr int kJoinRowWarps = 16;
__device__ __forceinline__ float2 join_tiles(const LossPiece& a, uint32_t n, uint32_t m) {
  __shared__ float2 part[kJoinRowWarps][32];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float top = -INFINITY, sum = 0.f;
  if (m < n) {
#pragma unroll 8
    for (uint32_t t = warp; t < a.tiles; t += kJoinRowWarps) {
      const float2 s = a.stat[(uint64_t)t * a.rows + m];
      top = fmaxf(top, s.x);
      sum += s.y;
    }
  }
  part[warp][lane] = make_float2(top, sum);
  __syncthreads();
  if (warp == 0) {
#pragma unroll
    for (int w = 1; w < kJoinRowWarps; ++w) { top = fmaxf(top, part[w][lane].x); sum += part[w][lane].y; }
  }
  return make_float2(top, sum);
}
// loss and lse from the sum over the columns that are not the label, and lse - reference for k_finish (in factor); returns the loss
__device__ __forceinline__ float store_loss(const LossPiece& a, uint32_t m, float sum) {
  const float ref = a.ref[m], target = a.target[m];
  const float above = ref == target ? log1pf(sum) : logf(sum + expf(target - ref)), loss = (ref - target) + above;
  const uint64_t row = a.row0 + a.row_of[m];
  a.loss[row] = loss;
  a.lse[row] = ref + above;  // not target + loss, which is no number where the label's logit is -inf
  a.factor[m] = above;
  return loss;
}

__global__ void __launch_bounds__(32 * kJoinRowWarps) k_join(LossPiece a) {
  let_next_start();
  after_previous();
  const uint32_t n = *a.count, m = blockIdx.x * 32 + (threadIdx.x & 31);
  if (blockIdx.x * 32 >= n) return;
  if (a.dx && blockIdx.x == 0 && threadIdx.x / 32 == 1) {
    const uint32_t slices = dx_slices(a, n);
    if (threadIdx.x == 32) a.count[1] = slices;
  }
  const float2 s = join_tiles(a, n, m);
  if (threadIdx.x >= 32 || m >= n) return;
  // (a label's logit of -inf is no reference either: z - reference is inf or no number)
  if ((s.y > kSumLimit || a.ref[m] == -INFINITY) && s.x < INFINITY && s.x > -INFINITY) {
    a.ref[m] = s.x;
    a.redo[1 + m / kMmaTile] = 1;
    a.redo[0] = 1;
  } else {
    store_loss(a, m, s.y);
  }
}

// Row tiles with new references: their rows' sums once more.  With gradients: f, the label's element of e, and f x.
template <bool kGrad>
__global__ void __launch_bounds__(32 * kJoinRowWarps) k_finish(LossPiece a) {
  __shared__ float s_f[32];
  let_next_start();
  after_previous();
  const uint32_t n = *a.count, r0 = blockIdx.x * 32, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, m = r0 + lane;
  if (r0 >= n) return;
  const bool again = a.redo[1 + r0 / kMmaTile] != 0;
  if (!kGrad && !again) return;
  float sum = 0.f;
  if (again) sum = join_tiles(a, n, m).y;
  if (warp == 0 && m < n) {
    const float loss = again ? store_loss(a, m, sum) : a.loss[a.row0 + a.row_of[m]];
    if constexpr (kGrad) {
      const float g = a.grad_loss ? a.grad_loss[(a.row0 + a.row_of[m]) * a.grad_stride] : 1.f;
      const float above = a.factor[m];
      // The label's element outweighs the row's others together, so f takes up its rounding (at most 2^-8): f q is the label's d,
      // and dw's error that of f x's rounding alone (2.3e-3 of its norm instead of 2.7e-3, the output's own 1.7e-3 included).
      const float e = expm1f(-loss) * expf(above);
      const __nv_bfloat16 q = __float2bfloat16_rn(e);
      const float r = e / __bfloat162float(q), f = g * expf(-above) * (r > 0.99f && r < 1.01f ? r : 1.f);
      a.factor[m] = f;
      s_f[lane] = f;
      a.p[(uint64_t)m * a.ld_p + a.label[m]] = q;
    }
  }
  if constexpr (kGrad) {
    __syncthreads();
    const uint32_t vecs = a.hidden / 8, second = (n + kMmaK - 1) / kMmaK * kMmaK;
    for (uint32_t k = warp; k < 32 && r0 + k < n; k += kJoinRowWarps) {
      uint4* x = reinterpret_cast<uint4*>(a.xc + (uint64_t)(r0 + k) * a.hidden);
      const float f = s_f[k];
#pragma unroll 4
      for (uint32_t c = lane; c < vecs; c += 32) {
        float t[8];
        Pack<__nv_bfloat16>::widen(x[c], t);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= f;
        const uint4 first = x[c] = Pack<__nv_bfloat16>::narrow(t);
        if (a.twice) {
          float b[8];
          Pack<__nv_bfloat16>::widen(first, b);
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] -= b[e];
          x[(uint64_t)second * vecs + c] = Pack<__nv_bfloat16>::narrow(t);
        }
      }
    }
  }
}

// 16 values of a row, rounded to bf16; `left` of them exist (a multiple of 8)
__device__ __forceinline__ void store_bf16x16(__nv_bfloat16* p, const float* f, uint32_t left, bool wide) {
  uint32_t w[8];
#pragma unroll
  for (uint32_t j = 0; j < 8; ++j) w[j] = bf16x2(f[2 * j], f[2 * j + 1]);
  if (wide && left >= 16) {
    store32(p, w);
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    if (left >= 16) *reinterpret_cast<uint4*>(p + 8) = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
// a lane's 128 columns out of tensor memory, and the accumulator given back
template <class Release>
__device__ __forceinline__ void take_columns(uint32_t tmem, uint32_t (&z)[4][32], Release&& release) {
#pragma unroll
  for (uint32_t c = 0; c < 4; ++c) {
    if (tmem == kNone) {
#pragma unroll
      for (uint32_t j = 0; j < 32; ++j) z[c][j] = 0;
    } else {
      tmem_load32(tmem + 32 * c, z[c]);
    }
  }
  tmem_wait();
  release();
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
k_dx(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ PoolView v,
     const __grid_constant__ LossPiece a) {
  let_next_start();
  after_previous();
  const uint32_t n = *a.count, k_blocks = (a.vocab + kMmaK - 1) / kMmaK;
  const uint32_t slices = n ? a.count[1] : 1, each = (k_blocks + slices - 1) / slices;
  const HighTiles work(n, a.hidden, slices, a.pairs);
  const bool wide = ((reinterpret_cast<uintptr_t>(a.dx) | a.lddx * 2) & 31) == 0;
  bool lost;
  mma_pair_tiles<false, true, 2>(map_p, map_w, work.items(), v, &lost,
    [&](uint32_t i) { return work.at(i, each, k_blocks); }, [](const MmaTile&, uint32_t) {},
    [&](const MmaTile& t, uint32_t i, uint32_t tmem, uint32_t row, uint32_t col0, auto&& release) {
      const uint32_t r = t.m % kHighRows + row + (threadIdx.x & 31), m = t.m + row + (threadIdx.x & 31), c0 = t.n + col0;
      if (c0 >= a.hidden) return;
      uint32_t z[4][32];
      take_columns(tmem, z, release);
      if (slices > 1) {  // columns first: a warp's store is one line
        float* slot = a.dx_slots + ((uint64_t)work.tile_of(i) * kMmaTile + col0) * kHighRows + r;
#pragma unroll
        for (uint32_t c = 0; c < 128; ++c) slot[c * kHighRows] = __uint_as_float(z[c / 32][c % 32]);
      } else if (m < n) {
        const uint32_t cols = min(128u, a.hidden - c0);
        const float f = a.factor[m];
        __nv_bfloat16* dx = a.dx + (a.row0 + a.row_of[m]) * a.lddx + c0;
#pragma unroll
        for (uint32_t c = 0; c < 128; c += 16) {
          if (c >= cols) break;
          float d[16];
#pragma unroll
          for (uint32_t j = 0; j < 16; ++j) d[j] = f * __uint_as_float(z[(c + j) / 32][(c + j) % 32]);
          store_bf16x16(dx + c, d, cols - c, wide);
        }
      }
    });
  give_up(v, a.call_seq, lost);
}

// dx of a counted row from several slices: f times their sum, in slice order, rounded once.  A CTA takes 32 rows and kCols
// columns and turns them over in shared memory: the slices hold columns, dx rows.  64 columns, a line of dx, unless that
// gives fewer CTAs than SMs; then 16 (8 rows x 1024, 32 slices: 20.7 -> 12.0 us; 2460 rows x 1024: 16.7 us, 21.7 with 16).
template <uint32_t kCols>
__global__ void __launch_bounds__(256) k_dx_join(LossPiece a) {
  constexpr uint32_t kEach = kCols / 8;  // columns of a warp
  __shared__ float turned[32][kCols + 4];
  let_next_start();
  after_previous();
  const uint32_t n = *a.count;
  if (n == 0) return;
  const uint32_t slices = a.count[1], col_parts = (a.hidden + kCols - 1) / kCols, parts = (n + 31) / 32 * col_parts;
  if (slices == 1) return;
  const HighTiles work(n, a.hidden, slices, a.pairs);
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (uint32_t i = blockIdx.x; i < parts; i += gridDim.x) {
    const uint32_t r0 = i / col_parts * 32, c0 = i % col_parts * kCols, m = r0 + lane;
    const uint64_t tile = (uint64_t)(r0 / kHighRows) * work.n_tiles + c0 / kMmaTile, slice = (uint64_t)work.tiles * kMmaTile * kHighRows;
    const float* slot = a.dx_slots + (tile * kMmaTile + c0 % kMmaTile + warp * kEach) * kHighRows + r0 % kHighRows + lane;
    const float f = m < n ? a.factor[m] : 0.f;
    float s[kEach] = {};
#pragma unroll(32 / kEach)
    for (uint32_t k = 0; k < slices; ++k) {
#pragma unroll
      for (uint32_t j = 0; j < kEach; ++j) s[j] += slot[k * slice + j * kHighRows];
    }
    __syncthreads();  // the part before this one has been written out
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) turned[lane][warp * kEach + j] = f * s[j];
    __syncthreads();
    const uint32_t r = threadIdx.x / kEach, c = threadIdx.x % kEach * 8;
    if (r < 32 && r0 + r < n && c0 + c < a.hidden)
      *reinterpret_cast<uint4*>(a.dx + (a.row0 + a.row_of[r0 + r]) * a.lddx + c0 + c) = Pack<__nv_bfloat16>::narrow(&turned[r][c]);
  }
}

// dw leaves by TMA.  fp32 sums that are added to (accumulation, or later pieces) are added on their way out, each element once.
// 200 rows x 32768 x 3584: 83 us, 93 us with direct stores of 32 bytes a lane.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
k_dw(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_out,
     const __grid_constant__ PoolView v, const __grid_constant__ LossPiece a) {
  let_next_start();
  after_previous();
  const uint32_t n = *a.count, blocks = (n + kMmaK - 1) / kMmaK, k_blocks = a.twice ? 2 * blocks : blocks;
  const HighTiles work(a.vocab, a.hidden, 1, a.pairs);
  const bool in_fp32 = a.dw_dtype == FT_F32 || !a.last;  // a bf16 dw of several pieces is summed in fp32 until the last one
  bool lost;
  mma_pair_tiles<true, true, 2>(map_p, map_x, work.items(), v, &lost,
    [&](uint32_t i) {
      MmaTile t = work.at(i, k_blocks, k_blocks);
      if (a.twice) t.again = blocks;
      return t;
    },
    [](const MmaTile&, uint32_t) {},
    [&](const MmaTile& t, uint32_t, uint32_t tmem, uint32_t row, uint32_t col0, auto&& release) {
      const int32_t c0 = (int32_t)(t.n + col0), m0 = (int32_t)(t.m + row);
      if (c0 >= (int32_t)a.hidden) return;
      uint32_t z[4][32];
      take_columns(tmem, z, release);
      if (m0 >= (int32_t)a.vocab) return;
      const MmaOut out;
      if (in_fp32) {
#pragma unroll
        for (uint32_t c = 0; c < 128; c += 32) {
          if (c0 + c >= a.hidden) break;
          const auto quad = [&](uint32_t j) { return make_uint4(z[c / 32][4 * j], z[c / 32][4 * j + 1], z[c / 32][4 * j + 2], z[c / 32][4 * j + 3]); };
          if (a.add_dw) out.put<true>(&map_out, c0 + (int32_t)c, m0, quad);
          else out.put<false>(&map_out, c0 + (int32_t)c, m0, quad);
        }
        return;
      }
      if (a.add_dw) {  // the last of several pieces
        const uint32_t m = (uint32_t)m0 + (threadIdx.x & 31);
        const float* sums = a.dw_acc + (uint64_t)m * a.hidden + c0;
#pragma unroll
        for (uint32_t c = 0; c < 128; c += 8) {
          float b[8] = {};
          if (m < a.vocab && c0 + c < a.hidden) load32(sums + c, b);
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j) z[c / 32][c % 32 + j] = __float_as_uint(__uint_as_float(z[c / 32][c % 32 + j]) + b[j]);
        }
      }
#pragma unroll
      for (uint32_t c = 0; c < 128; c += 64) {
        if (c0 + c >= a.hidden) break;
        out.put<false>(&map_out, c0 + (int32_t)c, m0, [&](uint32_t j) {
          float d[8];
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k) d[k] = __uint_as_float(z[(c + 8 * j + k) / 32][(c + 8 * j + k) % 32]);
          return Pack<__nv_bfloat16>::narrow(d);
        });
      }
    });
  give_up(v, a.call_seq, lost);
}

// ---- workspace ----------------------------------------------------------------------------------------------------

// Carves the workspace for pieces of `rows` rows; returns its bytes.  `acc`: a bf16 dw of several pieces.  Few rows have room for
// slices of dx that give each pair two tiles: `sms` of them, 512 KiB each.
static uint64_t loss_carve(LossPiece* a, uint8_t* base, uint32_t rows, uint32_t hidden, uint32_t vocab, uint32_t sms, bool grad, bool acc) {
  uint64_t off = 0;
  auto take = [&](uint64_t bytes) { const uint64_t o = off; off += align_up_sz(bytes, 256); return base + o; };
  const uint64_t padded = align_up_sz(rows, kMmaTile);
  a->rows = rows;
  a->padded = (uint32_t)padded;
  a->tiles = (vocab + kStatCols - 1) / kStatCols;
  a->ld_p = (uint32_t)align_up_sz(vocab, 64);  // whole lines
  const uint64_t dx_tiles = (padded + kHighRows - 1) / kHighRows * ((hidden + kMmaTile - 1) / kMmaTile);
  a->slots = (uint32_t)std::max<uint64_t>(dx_tiles, sms);
  a->count = reinterpret_cast<uint32_t*>(take(8));
  a->row_of = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->label = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->redo = reinterpret_cast<uint32_t*>(take(4ull * (1 + padded / kMmaTile)));
  a->ref = reinterpret_cast<float*>(take(4ull * rows));
  a->target = reinterpret_cast<float*>(take(4ull * rows));
  a->factor = reinterpret_cast<float*>(take(4ull * rows));
  a->stat = reinterpret_cast<float2*>(take(8ull * rows * a->tiles));
  a->xc = reinterpret_cast<__nv_bfloat16*>(take(2ull * padded * hidden));
  a->p = reinterpret_cast<__nv_bfloat16*>(take(grad ? 2ull * padded * a->ld_p : 0));
  a->dx_slots = reinterpret_cast<float*>(take(grad ? 4ull * a->slots * kHighRows * kMmaTile : 0));
  a->dw_acc = reinterpret_cast<float*>(take(acc ? 4ull * vocab * hidden : 0));
  return off;
}

struct LossWork {
  uint32_t hidden, vocab, sms;
  bool grad, bf16_dw;
  uint64_t rows;
  uint64_t bytes(uint32_t piece) const {
    LossPiece a;
    return loss_carve(&a, nullptr, piece, hidden, vocab, sms, grad, grad && bf16_dw && piece < rows);
  }
  uint32_t least_rows() const { return (uint32_t)std::min<uint64_t>(rows, 256); }
  // pieces of the rows whose probabilities take 4 GiB
  uint32_t best_rows() const {
    const uint64_t most = grad ? std::max<uint64_t>(256, (4ull << 30) / (2ull * vocab) / 256 * 256) : kPieceRowsMost;
    return (uint32_t)std::min<uint64_t>(rows, std::min<uint64_t>(most, kPieceRowsMost));
  }
  uint64_t least() const { return std::min(bytes(least_rows()), bytes(best_rows())); }
  uint64_t best() const { return std::max(bytes(least_rows()), bytes(best_rows())); }
  // the largest piece that fits: all rows, or a multiple of 256
  uint32_t piece_for(uint64_t have) const {
    if (bytes(best_rows()) <= have) return best_rows();
    uint32_t lo = 1, hi = (best_rows() + 255) / 256;  // in units of 256 rows
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (bytes(mid * 256) <= have) lo = mid; else hi = mid;
    }
    return std::min(lo * 256, best_rows());
  }
};

static int32_t token_loss(ft_pool* p, LossPiece a, uint64_t rows, bool grad, void* workspace, uint64_t workspace_bytes, uint32_t accumulate,
                          cudaStream_t st) {
  const LossWork work{a.hidden, a.vocab, (uint32_t)p->sm_count, grad, a.dw_dtype == FT_BF16, rows};
  if (!workspace || !aligned_to(workspace, 256)) return FT_ERR_INVALID_ARG;
  if (workspace_bytes < work.least()) return FT_ERR_CAPACITY;
  const uint32_t piece = work.piece_for(workspace_bytes);
  loss_carve(&a, static_cast<uint8_t*>(workspace), piece, a.hidden, a.vocab, (uint32_t)p->sm_count, grad, grad && a.dw_dtype == FT_BF16 && piece < rows);
  a.call_seq = status_seq(p);
  CUtensorMap map_x, map_w, map_p = {}, map_e = {}, map_dw = {};
  if (mma_map(&map_x, a.xc, a.hidden, a.padded, a.hidden) != CUDA_SUCCESS || mma_map(&map_w, a.w, a.hidden, a.vocab, a.ldw) != CUDA_SUCCESS ||
      (grad && (mma_map(&map_p, a.p, a.vocab, a.padded, a.ld_p) != CUDA_SUCCESS || mma_map(&map_e, a.p, a.vocab, a.padded, a.ld_p, 32) != CUDA_SUCCESS)))
    return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  a.pairs = (uint32_t)p->sm_count / 2;
  const unsigned grid = 2 * a.pairs;
  if (!p->loss_attr_set) {  // once per pool, hence once per device the pool lives on
    for (auto k : {k_logits<false, false, 1>, k_logits<false, false, 2>, k_logits<false, true, 1>, k_logits<true, false, 1>, k_logits<true, false, 2>,
                   k_logits<true, true, 1>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMmaSmem));
    FT_CUDA(cudaFuncSetAttribute(k_dx, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMmaSmem));
    FT_CUDA(cudaFuncSetAttribute(k_dw, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMmaSmem));
    p->loss_attr_set = true;
  }
  for (uint64_t r0 = 0; r0 < rows; r0 += piece) {
    a.row0 = r0;
    a.rows = (uint32_t)std::min<uint64_t>(piece, rows - r0);
    a.add_dw = r0 > 0 || accumulate;
    a.last = r0 + a.rows == rows;
    a.twice = grad && a.rows <= kTwiceUpTo;
    if (grad) {
      const bool fp32 = a.dw_dtype == FT_F32 || !a.last;
      if (mma_map(&map_dw, a.dw_dtype == FT_F32 || a.last ? a.dw : a.dw_acc, a.hidden, a.vocab, a.hidden, 32, fp32) != CUDA_SUCCESS)
        return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    }
    const dim3 joins((a.rows + 31) / 32);
    const uint32_t join_threads = 32 * kJoinRowWarps;
    const bool high = a.rows > kMmaTile && a.hidden <= kHighBlocks * kMmaK;
    if (a.rows <= kPickFewUpTo) k_pick<kPickFew><<<(a.rows + kPickFew - 1) / kPickFew, 256, 0, st>>>(p->view, a);
    else k_pick<kPickRows><<<(a.rows + kPickRows - 1) / kPickRows, 256, 0, st>>>(p->view, a);
    FT_CUDA(cudaGetLastError());
    if (grad) {
      FT_CUDA(launch_chained(high ? k_logits<true, false, 2> : k_logits<true, false, 1>, grid, kMmaThreads, kMmaSmem, st, map_x, map_w, map_e, p->view, a));
      FT_CUDA(launch_chained(k_join, joins, join_threads, 0, st, a));
      FT_CUDA(launch_chained(k_logits<true, true, 1>, grid, kMmaThreads, kMmaSmem, st, map_x, map_w, map_e, p->view, a));
      FT_CUDA(launch_chained(k_finish<true>, joins, join_threads, 0, st, a));
      FT_CUDA(launch_chained(k_dx, grid, kMmaThreads, kMmaSmem, st, map_p, map_w, p->view, a));
      const uint64_t parts = (uint64_t)joins.x * ((a.hidden + 63) / 64), most = (uint64_t)p->sm_count * 8;
      if (parts < (uint64_t)p->sm_count) FT_CUDA(launch_chained(k_dx_join<16>, dim3((unsigned)parts * 4), 256, 0, st, a));
      else FT_CUDA(launch_chained(k_dx_join<64>, dim3((unsigned)std::min(parts, most)), 256, 0, st, a));
      FT_CUDA(launch_chained(k_dw, grid, kMmaThreads, kMmaSmem, st, map_p, map_x, map_dw, p->view, a));
    } else {
      FT_CUDA(launch_chained(high ? k_logits<false, false, 2> : k_logits<false, false, 1>, grid, kMmaThreads, kMmaSmem, st, map_x, map_w, map_e, p->view, a));
      FT_CUDA(launch_chained(k_join, joins, join_threads, 0, st, a));
      FT_CUDA(launch_chained(k_logits<false, true, 1>, grid, kMmaThreads, kMmaSmem, st, map_x, map_w, map_e, p->view, a));
      FT_CUDA(launch_chained(k_finish<false>, joins, join_threads, 0, st, a));
    }
    p->gpu_launches += grad ? 8 : 5;
  }
  return FT_OK;
}

// the checks that both entry points share, in argument order
static int32_t loss_args(uint64_t rows, uint32_t hidden, uint32_t vocab, const void* x, uint64_t ldx, const void* w, uint64_t ldw,
                         const void* labels, const void* loss, const void* lse) {
  if (hidden == 0 || hidden % 8 || vocab == 0) return FT_ERR_INVALID_ARG;
  if (rows >> 31 || vocab >> 31) return FT_ERR_CAPACITY;
  if (rows == 0) return FT_OK;
  if (!x || !aligned_to(x, 16) || ldx < hidden || ldx % 8 || !w || !aligned_to(w, 16) || ldw < hidden || ldw % 8) return FT_ERR_INVALID_ARG;
  if (!labels || !aligned_to(labels, 4) || !loss || !aligned_to(loss, 4) || !lse || !aligned_to(lse, 4)) return FT_ERR_INVALID_ARG;
  return FT_OK;
}

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_token_loss_workspace(ft_pool* p, uint64_t rows, uint32_t hidden, uint32_t vocab, uint32_t with_grad, uint32_t dw_dtype,
                                            uint64_t* least, uint64_t* best) {
  if (!p || hidden == 0 || hidden % 8 || vocab == 0 || !dtype_ok(dw_dtype) || !least || !best) return FT_ERR_INVALID_ARG;
  if (rows >> 31 || vocab >> 31) return FT_ERR_CAPACITY;
  const LossWork work{hidden, vocab, (uint32_t)p->sm_count, with_grad != 0, dw_dtype == FT_BF16, rows};
  *least = rows ? work.least() : 0;
  *best = rows ? work.best() : 0;
  return FT_OK;
}

FT_EXPORT int32_t pool_token_loss(ft_pool* p, uint64_t rows, uint32_t hidden, uint32_t vocab, const void* x, uint64_t ldx, const void* w,
                                  uint64_t ldw, const int32_t* labels, float* loss, float* lse, void* workspace, uint64_t workspace_bytes,
                                  void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  const int32_t rc = loss_args(rows, hidden, vocab, x, ldx, w, ldw, labels, loss, lse);
  if (rc != FT_OK || rows == 0) return rc;
  LossPiece a = {};
  a.hidden = hidden; a.vocab = vocab; a.ldx = ldx; a.ldw = ldw;
  a.x = static_cast<const __nv_bfloat16*>(x); a.w = static_cast<const __nv_bfloat16*>(w);
  a.labels = labels; a.loss = loss; a.lse = lse; a.dw_dtype = FT_F32;
  return token_loss(p, a, rows, false, workspace, workspace_bytes, 0, static_cast<cudaStream_t>(stream));
}

FT_EXPORT int32_t pool_token_loss_grad(ft_pool* p, uint64_t rows, uint32_t hidden, uint32_t vocab, const void* x, uint64_t ldx, const void* w,
                                       uint64_t ldw, const int32_t* labels, const float* grad_loss, uint32_t grad_stride, float* loss,
                                       float* lse, void* dx, uint64_t lddx, void* dw, uint32_t dw_dtype, uint32_t accumulate,
                                       void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  const int32_t rc = loss_args(rows, hidden, vocab, x, ldx, w, ldw, labels, loss, lse);
  if (rc != FT_OK) return rc;
  if (!aligned_to(grad_loss, 4) || grad_stride > 1 || !dtype_ok(dw_dtype) || (accumulate && dw_dtype != FT_F32)) return FT_ERR_INVALID_ARG;
  if (!dw || !aligned_to(dw, 16)) return FT_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (!accumulate) FT_CUDA(cudaMemsetAsync(dw, 0, (size_t)vocab * hidden * dtype_size(dw_dtype), st));
    return FT_OK;
  }
  if (!dx || !aligned_to(dx, 16) || lddx < hidden || lddx % 8) return FT_ERR_INVALID_ARG;
  LossPiece a = {};
  a.hidden = hidden; a.vocab = vocab; a.ldx = ldx; a.ldw = ldw; a.lddx = lddx;
  a.x = static_cast<const __nv_bfloat16*>(x); a.w = static_cast<const __nv_bfloat16*>(w);
  a.labels = labels; a.loss = loss; a.lse = lse; a.grad_loss = grad_loss; a.grad_stride = grad_stride;
  a.dx = static_cast<__nv_bfloat16*>(dx); a.dw = dw; a.dw_dtype = dw_dtype;
  return token_loss(p, a, rows, true, workspace, workspace_bytes, accumulate, st);
}

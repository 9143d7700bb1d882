// Softmax cross entropy of rows against a vocabulary, with its gradients, without a matrix of logits.
//
//   z = x W^T,  lse = log(sum(exp(z))),  loss = lse - z[label]
//   d = g (exp(z - lse) - [v = label]),  dx = d W,  dW = d^T x
//
//   k_pick    takes the rows that count out of a piece of the rows: a dense copy of their x, their labels and row
//             numbers.  Rows labelled -100 cost no products, and what they hold cannot reach dW as 0 * NaN
//   k_logits  z by tiles; of a tile, each row keeps its maximum and the sum of exp(z - maximum), and with gradients
//             exp(z - maximum) itself in bf16 (relative to the tile's own maximum, so rounding it costs 2^-8 of a
//             probability, where rounding z would cost 2^-8 of z)
//   k_join    joins the tiles' maxima and sums: lse, loss
//   k_scale   turns exp(z - tile maximum) into d: one factor a row and tile, and the label's element from its own logit
//   k_dx, k_dw  the two products
#include <algorithm>

#include "operators.cuh"

namespace ft {

constexpr uint32_t kTile = 64;  // rows and columns of a tile
constexpr int32_t kNoLabel = -100;
constexpr uint32_t kPieceRowsMost = 65536;

struct LossPiece {
  uint32_t rows, hidden, vocab, ld_p, tiles;  // tiles: tiles of the vocabulary
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
  uint32_t* count;         // rows of the piece that count
  int32_t *row_of, *label; // [count] row in the piece, label
  float *target, *row_lse; // [count]
  float2* stat;            // [tiles][rows] maximum and sum of a row in a tile
  __nv_bfloat16* xc;       // [rows][hidden]
  __nv_bfloat16* p;        // [rows][ld_p]
  float* dw_acc;           // [vocab][hidden]: bf16 dw of several pieces
};

constexpr uint32_t kPickRows = 64;

__global__ void __launch_bounds__(256) k_pick(PoolView v, LossPiece a) {
  __shared__ uint32_t before, warp_count[2];
  __shared__ int32_t dest[kPickRows];
  const uint32_t r0 = blockIdx.x * kPickRows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t* labels = a.labels + a.row0;
  if (threadIdx.x == 0) before = 0;
  __syncthreads();
  uint32_t mine = 0;
  for (uint32_t r = threadIdx.x; r < r0; r += blockDim.x) { const int32_t l = labels[r]; mine += l >= 0 && (uint32_t)l < a.vocab; }
  mine = __reduce_add_sync(0xFFFFFFFFu, mine);
  if (lane == 0 && mine) atomicAdd(&before, mine);
  const uint32_t r = r0 + threadIdx.x;
  bool counts = false;
  int32_t l = kNoLabel;
  uint32_t mask = 0;
  if (threadIdx.x < kPickRows) {
    if (r < a.rows) l = labels[r];
    counts = l >= 0 && (uint32_t)l < a.vocab;
    mask = __ballot_sync(0xFFFFFFFFu, counts);
    if (lane == 0) warp_count[warp] = __popc(mask);
  }
  __syncthreads();
  if (threadIdx.x < kPickRows) {
    const uint32_t pos = before + (warp ? warp_count[0] : 0) + __popc(mask & ((1u << lane) - 1));
    dest[threadIdx.x] = counts ? (int32_t)pos : -1;
    if (counts) {
      a.row_of[pos] = (int32_t)r;
      a.label[pos] = l;
    } else if (r < a.rows) {
      a.loss[a.row0 + r] = 0.f;
      a.lse[a.row0 + r] = 0.f;
      if (l != kNoLabel) note_error(v, a.call_seq, FT_ERR_BAD_TOKEN_ID, (uint32_t)(a.row0 + r));
    }
  }
  const uint32_t total = before + warp_count[0] + warp_count[1];
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *a.count = total;
  __syncthreads();
  const uint32_t vecs = a.hidden / 8, rows = min(kPickRows, a.rows - r0);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  for (uint32_t k = warp; k < rows; k += blockDim.x / 32) {
    if (dest[k] >= 0) {
      const uint4* src = reinterpret_cast<const uint4*>(a.x + (a.row0 + r0 + k) * a.ldx);
      uint4* dst = reinterpret_cast<uint4*>(a.xc + (uint64_t)dest[k] * a.hidden);
      for (uint32_t c = lane; c < vecs; c += 32) dst[c] = src[c];
    } else if (a.dx) {
      uint4* dst = reinterpret_cast<uint4*>(a.dx + (a.row0 + r0 + k) * a.lddx);
      for (uint32_t c = lane; c < vecs; c += 32) dst[c] = zero;
    }
  }
}

// 64 x 64 tile of A B^T in fp32 by a 16 x 16 block, four rows and four columns a thread; fetch_a(m, k), fetch_b(n, k)
template <class FA, class FB>
__device__ __forceinline__ void tile_product(uint32_t m0, uint32_t n0, uint32_t K, FA fetch_a, FB fetch_b, float (&acc)[4][4]) {
  __shared__ float sa[16][kTile + 1], sb[16][kTile + 1];
  const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (uint32_t k0 = 0; k0 < K; k0 += 16) {
    for (uint32_t i = threadIdx.x; i < 16 * kTile; i += 256) {
      const uint32_t k = i % 16, m = i / 16;
      sa[k][m] = k0 + k < K ? fetch_a(m0 + m, k0 + k) : 0.f;
      sb[k][m] = k0 + k < K ? fetch_b(n0 + m, k0 + k) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += sa[k][ty * 4 + i] * sb[k][tx * 4 + j];
    __syncthreads();
  }
}

template <bool kKeep>
__global__ void __launch_bounds__(256) k_logits(LossPiece a) {
  const uint32_t n = *a.count, m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
  if (m0 >= n) return;
  float z[4][4] = {};
  tile_product(m0, n0, a.hidden, [&](uint32_t m, uint32_t k) { return m < n ? __bfloat162float(a.xc[(uint64_t)m * a.hidden + k]) : 0.f; },
               [&](uint32_t v, uint32_t k) { return v < a.vocab ? __bfloat162float(a.w[(uint64_t)v * a.ldw + k]) : 0.f; }, z);
  const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = m0 + ty * 4 + i;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + tx * 4 + j < a.vocab) top = fmaxf(top, z[i][j]);
#pragma unroll
    for (int d = 8; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t v = n0 + tx * 4 + j;
      if (v >= a.vocab) continue;
      const float e = expf(z[i][j] - top);
      sum += e;
      if (m < n && (int32_t)v == a.label[m]) a.target[m] = z[i][j];
      if (kKeep && m < n) a.p[(uint64_t)m * a.ld_p + v] = __float2bfloat16_rn(e);
    }
#pragma unroll
    for (int d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (m < n && tx == 0) a.stat[(uint64_t)blockIdx.x * a.rows + m] = make_float2(top, sum);
  }
}

// 32 rows a CTA, its warps share the tiles
constexpr int kJoinRowWarps = 8;
__global__ void __launch_bounds__(32 * kJoinRowWarps) k_join(LossPiece a) {
  __shared__ float2 part[kJoinRowWarps][32];
  const uint32_t n = *a.count, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, m = blockIdx.x * 32 + lane;
  if (blockIdx.x * 32 >= n) return;
  float top = -INFINITY, sum = 0.f;
  auto add = [&](float2 s) {
    const float t = fmaxf(top, s.x);
    // an empty side contributes nothing (and -inf - -inf must not be formed for it)
    sum = (sum == 0.f ? 0.f : sum * expf(top - t)) + (s.y == 0.f ? 0.f : s.y * expf(s.x - t));
    top = t;
  };
  if (m < n)
    for (uint32_t t = warp; t < a.tiles; t += kJoinRowWarps) add(a.stat[(uint64_t)t * a.rows + m]);
  part[warp][lane] = make_float2(top, sum);
  __syncthreads();
  if (warp || m >= n) return;
#pragma unroll
  for (int w = 1; w < kJoinRowWarps; ++w) add(part[w][lane]);
  const float lse = top + logf(sum);
  a.row_lse[m] = lse;
  const uint64_t row = a.row0 + a.row_of[m];
  a.lse[row] = lse;
  a.loss[row] = lse - a.target[m];
}

__global__ void __launch_bounds__(256) k_scale(LossPiece a) {
  const uint32_t n = *a.count;
  for (uint32_t m = blockIdx.y; m < n; m += gridDim.y) {
    const float lse = a.row_lse[m], g = a.grad_loss ? a.grad_loss[(a.row0 + a.row_of[m]) * a.grad_stride] : 1.f;
    for (uint32_t v = blockIdx.x * 256 + threadIdx.x; v < a.vocab; v += gridDim.x * 256) {
      __nv_bfloat16* e = a.p + (uint64_t)m * a.ld_p + v;
      const float f = g * expf(a.stat[(uint64_t)(v / kTile) * a.rows + m].x - lse);
      *e = __float2bfloat16_rn((int32_t)v == a.label[m] ? g * expm1f(a.target[m] - lse) : f * __bfloat162float(*e));
    }
  }
}

__global__ void __launch_bounds__(256) k_dx(LossPiece a) {
  const uint32_t n = *a.count, m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
  if (m0 >= n) return;
  float c[4][4] = {};
  tile_product(m0, n0, a.vocab, [&](uint32_t m, uint32_t k) { return m < n ? __bfloat162float(a.p[(uint64_t)m * a.ld_p + k]) : 0.f; },
               [&](uint32_t h, uint32_t k) { return h < a.hidden ? __bfloat162float(a.w[(uint64_t)k * a.ldw + h]) : 0.f; }, c);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t m = m0 + threadIdx.x / 16 * 4 + i, h = n0 + threadIdx.x % 16 * 4 + j;
      if (m < n && h < a.hidden) a.dx[(a.row0 + a.row_of[m]) * a.lddx + h] = __float2bfloat16_rn(c[i][j]);
    }
}

__global__ void __launch_bounds__(256) k_dw(LossPiece a) {
  const uint32_t n = *a.count, m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
  float c[4][4] = {};
  tile_product(m0, n0, n, [&](uint32_t v, uint32_t k) { return v < a.vocab ? __bfloat162float(a.p[(uint64_t)k * a.ld_p + v]) : 0.f; },
               [&](uint32_t h, uint32_t k) { return h < a.hidden ? __bfloat162float(a.xc[(uint64_t)k * a.hidden + h]) : 0.f; }, c);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t v = m0 + threadIdx.x / 16 * 4 + i, h = n0 + threadIdx.x % 16 * 4 + j;
      if (v >= a.vocab || h >= a.hidden) continue;
      const uint64_t at = (uint64_t)v * a.hidden + h;
      if (a.dw_dtype == FT_F32) {
        float* d = static_cast<float*>(a.dw) + at;
        *d = a.add_dw ? *d + c[i][j] : c[i][j];
      } else {
        const float s = a.add_dw ? a.dw_acc[at] + c[i][j] : c[i][j];
        if (a.last) static_cast<__nv_bfloat16*>(a.dw)[at] = __float2bfloat16_rn(s);
        else a.dw_acc[at] = s;
      }
    }
}

// ---- workspace ----------------------------------------------------------------------------------------------------

// Carves the workspace for pieces of `rows` rows; returns its bytes.  `several`: more than one piece.
static uint64_t loss_carve(LossPiece* a, uint8_t* base, uint32_t rows, uint32_t hidden, uint32_t vocab, bool grad, bool acc) {
  uint64_t off = 0;
  auto take = [&](uint64_t bytes) { const uint64_t o = off; off += align_up_sz(bytes, 256); return base + o; };
  const uint64_t padded = align_up_sz(rows, kTile);
  a->rows = rows;
  a->tiles = (vocab + kTile - 1) / kTile;
  a->ld_p = (uint32_t)align_up_sz(vocab, 8);
  a->count = reinterpret_cast<uint32_t*>(take(4));
  a->row_of = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->label = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->target = reinterpret_cast<float*>(take(4ull * rows));
  a->row_lse = reinterpret_cast<float*>(take(4ull * rows));
  a->stat = reinterpret_cast<float2*>(take(8ull * rows * a->tiles));
  a->xc = reinterpret_cast<__nv_bfloat16*>(take(2ull * padded * hidden));
  a->p = reinterpret_cast<__nv_bfloat16*>(take(grad ? 2ull * padded * a->ld_p : 0));
  a->dw_acc = reinterpret_cast<float*>(take(acc ? 4ull * vocab * hidden : 0));
  return off;
}

struct LossWork {
  uint32_t hidden, vocab;
  bool grad, bf16_dw;
  uint64_t rows;
  uint64_t bytes(uint32_t piece) const {
    LossPiece a;
    return loss_carve(&a, nullptr, piece, hidden, vocab, grad, grad && bf16_dw && piece < rows);
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
  const LossWork work{a.hidden, a.vocab, grad, a.dw_dtype == FT_BF16, rows};
  if (!workspace || !aligned_to(workspace, 256)) return FT_ERR_INVALID_ARG;
  if (workspace_bytes < work.least()) return FT_ERR_CAPACITY;
  const uint32_t piece = work.piece_for(workspace_bytes);
  loss_carve(&a, static_cast<uint8_t*>(workspace), piece, a.hidden, a.vocab, grad, grad && a.dw_dtype == FT_BF16 && piece < rows);
  a.call_seq = status_seq(p);
  for (uint64_t r0 = 0; r0 < rows; r0 += piece) {
    a.row0 = r0;
    a.rows = (uint32_t)std::min<uint64_t>(piece, rows - r0);
    a.add_dw = r0 > 0 || accumulate;
    a.last = r0 + a.rows == rows;
    const uint32_t row_tiles = (a.rows + kTile - 1) / kTile;
    k_pick<<<(a.rows + kPickRows - 1) / kPickRows, 256, 0, st>>>(p->view, a);
    if (grad) k_logits<true><<<dim3(a.tiles, row_tiles), 256, 0, st>>>(a);
    else k_logits<false><<<dim3(a.tiles, row_tiles), 256, 0, st>>>(a);
    k_join<<<(a.rows + 31) / 32, 32 * kJoinRowWarps, 0, st>>>(a);
    p->gpu_launches += 3;
    if (grad) {
      const uint32_t h_tiles = (a.hidden + kTile - 1) / kTile;
      k_scale<<<dim3(std::min(8u, (a.vocab + 255) / 256), std::min(a.rows, 4096u)), 256, 0, st>>>(a);
      k_dx<<<dim3(h_tiles, row_tiles), 256, 0, st>>>(a);
      k_dw<<<dim3(h_tiles, a.tiles), 256, 0, st>>>(a);
      p->gpu_launches += 3;
    }
    FT_CUDA(cudaGetLastError());
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
  const LossWork work{hidden, vocab, with_grad != 0, dw_dtype == FT_BF16, rows};
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

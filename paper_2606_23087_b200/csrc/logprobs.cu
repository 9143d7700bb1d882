// Log probabilities of given tokens, entropies and the likeliest alternatives of rows against a vocabulary, without a matrix of logits
// where no alternatives are asked for.
//
//   z = x W^T, u = (z - max) scale log2(e), S = sum(2^u), U = sum(u 2^u)
//   logprob = (z_token - max) scale - ln S,  entropy = ln S - ln 2 U / S
//
//   k_score_pick  takes the rows that count out of a piece of the rows: a dense copy of their x, their tokens and row numbers
//   k_score       z by tiles; a row of a tile gives max, S and U of 128 columns (a segment), each about the segment's own maximum: every
//                 term of U is negative, so nothing cancels in an entropy; the token's logit; and with alternatives z itself in fp32
//   k_score_join  joins a row's segments.  Alternatives: the `top` segments with the largest maxima (equal ones: the first) hold the `top`
//                 largest logits, so only those are read again
//
// Bound by the tensor cores, few rows by W.
#include <algorithm>
#include <cmath>

#include "mma_pair.cuh"

namespace ft {

constexpr uint32_t kSegCols = 128;     // columns of a segment: an epilogue warp's
// The tensor cores truncate at every addition of 16 products, all one way: tiles of 256 rows are summed in parts of kScorePart blocks of K,
// the parts joined in registers.  Tiles of 512 rows have no registers for that: they are for rows beyond 256 and K up to kScoreHigh blocks.
constexpr uint32_t kScorePart = 16, kScoreHigh = 66;
constexpr uint32_t kScoreRowsMost = 65536;  // of a piece
constexpr float kScoreLog2e = 1.4426950408889634f, kScoreLn2 = 0.6931471805599453f;
constexpr float kLeastExponent = -300.f;    // 2^-300 is zero; finite, so that its product with zero is one

struct ScorePiece {
  uint32_t rows, hidden, vocab, segs, padded, pairs, top, ld_z;
  uint64_t row0, ldx;
  const __nv_bfloat16* x;
  const int32_t* tokens;
  float scale;
  float *logprob, *entropy, *top_logprobs;
  int32_t* top_ids;
  uint64_t call_seq;
  // workspace
  uint32_t* count;          // rows of the piece that count
  int32_t *row_of, *token;  // [count] row in the piece, token
  float* target;            // [count] the token's logit
  float *most, *sum, *moment;  // [segs][rows] max, S, U of a row's segment
  __nv_bfloat16* xc;        // [padded][hidden]
  float* z;                 // [padded][ld_z]
};

__device__ __forceinline__ float max_with_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A CTA takes kRows rows; where they go it learns by counting the tokens before them itself, so nothing has to wait for another CTA.
constexpr uint32_t kScorePickRows = 32, kScorePickFew = 8, kScorePickFewUpTo = 4096;
template <uint32_t kRows>
__global__ void __launch_bounds__(256) k_score_pick(PoolView v, ScorePiece a) {
  __shared__ uint32_t warp_count[8];
  __shared__ int32_t dest[32];
  let_next_start();
  const uint32_t r0 = blockIdx.x * kRows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = r0 + lane;
  const int32_t* tokens = a.tokens + a.row0;
  const uint32_t mine = __reduce_add_sync(0xFFFFFFFFu, count_labels(tokens, r0, a.vocab));
  if (lane == 0) warp_count[warp] = mine;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) before += warp_count[w];
  const int32_t t = lane < kRows && r < a.rows ? tokens[r] : kNoLabel;
  const bool counts = has_label(t, a.vocab);
  const uint32_t mask = __ballot_sync(0xFFFFFFFFu, counts), pos = before + __popc(mask & ((1u << lane) - 1));
  if (warp == 0) {
    dest[lane] = counts ? (int32_t)pos : -1;
    if (counts) {
      a.row_of[pos] = (int32_t)r;
      a.token[pos] = t;
    } else if (lane < kRows && r < a.rows) {
      const uint64_t row = a.row0 + r;
      a.logprob[row] = 0.f;
      if (a.entropy) a.entropy[row] = 0.f;
      for (uint32_t i = 0; i < a.top; ++i) { a.top_ids[row * a.top + i] = -1; a.top_logprobs[row * a.top + i] = 0.f; }
      if (t != kNoLabel) note_error(v, a.call_seq, FT_ERR_BAD_TOKEN_ID, (uint32_t)row);
    }
    if (blockIdx.x == gridDim.x - 1 && lane == 0) *a.count = before + __popc(mask);
  }
  __syncthreads();
  const uint32_t vecs = a.hidden / 8, rows = min(kRows, a.rows - r0);
  for (uint32_t k = warp; k < rows; k += 8) {
    if (dest[k] < 0) continue;
    const uint4* src = reinterpret_cast<const uint4*>(a.x + (a.row0 + r0 + k) * a.ldx);
    uint4* dst = reinterpret_cast<uint4*>(a.xc + (uint64_t)dest[k] * a.hidden);
#pragma unroll 8
    for (uint32_t c = lane; c < vecs; c += 32) dst[c] = src[c];
  }
}

// z by tiles; a lane owns a row's segment
template <bool kKeep, int kHigh>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
k_score(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_z,
        const __grid_constant__ PoolView v, const __grid_constant__ ScorePiece a) {
  let_next_start();
  after_previous();
  const uint32_t n = a.tokens ? *a.count : a.rows, n_tiles = (a.vocab + kMmaTile - 1) / kMmaTile, k_blocks = (a.hidden + kMmaK - 1) / kMmaK;
  const uint32_t blocks = (n + kMmaTile - 1) / kMmaTile, m_tiles = (blocks + kHigh - 1) / kHigh, tiles = m_tiles * n_tiles;
  constexpr uint32_t kPart = kHigh == 1 ? kScorePart : 0xFFFFFFu;
  const uint32_t k_parts = (k_blocks + kPart - 1) / kPart;
  bool lost;
  uint32_t z[kSegCols / 32][32];
  int32_t token = kNoLabel;
  mma_pair_tiles<false, false, kHigh>(map_x, map_w, (tiles + a.pairs - 1) / a.pairs * a.pairs * k_parts, v, &lost,
    [&](uint32_t item) {  // a pair takes the parts of a tile's K one after the other
      const uint32_t round = item / a.pairs, i = item % a.pairs + round / k_parts * a.pairs, part = round % k_parts;
      if (i >= tiles) return MmaTile{0, 0, 0, 0, 0};
      // bands of 2048 rows, all columns of a band before the next: a band's x stays in L2
      constexpr uint32_t kBand = 8 / kHigh;
      const uint32_t band = i / (kBand * n_tiles), in = i - band * kBand * n_tiles, rows = min(kBand, m_tiles - band * kBand), m = band * kBand + in % rows;
      return MmaTile{m * kHigh * kMmaTile, in / rows * kMmaTile, part * kPart, min((part + 1) * kPart, k_blocks), min((uint32_t)kHigh, blocks - m * kHigh)};
    },
    [&](const MmaTile& t, uint32_t row) {
      const uint32_t m = t.m + row + (threadIdx.x & 31);
      token = a.tokens && m < n ? a.token[m] : kNoLabel;
    },
    [&](const MmaTile& t, uint32_t, uint32_t tmem, uint32_t row, uint32_t col0, auto&& release) {
      const uint32_t c0 = t.n + col0;
      if (c0 >= a.vocab) return;
      if (kHigh == 2 || t.k0 == 0) {
#pragma unroll
        for (uint32_t c = 0; c < kSegCols / 32; ++c) tmem_load32(tmem + 32 * c, z[c]);
        tmem_wait();
      } else {
#pragma unroll
        for (uint32_t c = 0; c < kSegCols / 32; ++c) {
          uint32_t part[32];
          tmem_load32(tmem + 32 * c, part);
          tmem_wait();
#pragma unroll
          for (uint32_t j = 0; j < 32; ++j) z[c][j] = __float_as_uint(__uint_as_float(z[c][j]) + __uint_as_float(part[j]));
        }
      }
      release();  // the products go on while the exponentials are taken
      if (kHigh == 1 && t.k1 < k_blocks) return;
      const uint32_t m = t.m + row + (threadIdx.x & 31), cols = min(kSegCols, a.vocab - c0), token_at = (uint32_t)token - c0;
      if (token_at < kSegCols) {
        uint32_t own = 0;
#pragma unroll
        for (uint32_t j = 0; j < kSegCols; ++j) own = j == token_at ? z[j / 32][j % 32] : own;
        a.target[m] = __uint_as_float(own);
      }
      if (cols < kSegCols) {  // beyond the vocabulary
#pragma unroll
        for (uint32_t j = 0; j < kSegCols; ++j)
          if (j >= cols) z[j / 32][j % 32] = 0xFF800000u;
      }
      if constexpr (kKeep) {
#pragma unroll
        for (uint32_t c = 0; c < kSegCols; c += 32)
          MmaOut().put<false>(&map_z, (int32_t)(c0 + c), (int32_t)(t.m + row),
                              [&](uint32_t j) { return make_uint4(z[c / 32][4 * j], z[c / 32][4 * j + 1], z[c / 32][4 * j + 2], z[c / 32][4 * j + 3]); });
      }
      float top = -INFINITY;
#pragma unroll
      for (uint32_t j = 0; j < kSegCols; j += 2) top = fmaxf(top, fmaxf(__uint_as_float(z[j / 32][j % 32]), __uint_as_float(z[j / 32][j % 32 + 1])));
      F2 sums = f2(0.f), moments = f2(0.f);
      const F2 less = f2(top == -INFINITY ? 0.f : -top), scale = f2(a.scale * kScoreLog2e);
#pragma unroll
      for (uint32_t j = 0; j < kSegCols; j += 2) {
        const float2 t2 = parts((f2(__uint_as_float(z[j / 32][j % 32]), __uint_as_float(z[j / 32][j % 32 + 1])) + less) * scale);
        const float u0 = max_with_nan(t2.x, kLeastExponent), u1 = max_with_nan(t2.y, kLeastExponent);
        const F2 e = f2(exp2_fast(u0), exp2_fast(u1));
        sums = sums + e;
        moments = fma(e, f2(u0, u1), moments);
      }
      if (m < n) {
        const uint64_t at = (uint64_t)(c0 / kSegCols) * a.rows + m;
        a.most[at] = top;
        a.sum[at] = sum(sums);
        a.moment[at] = sum(moments);
      }
    });
  give_up(v, a.call_seq, lost);
}

// ---- joining the segments of a row ----------------------------------------------------------------------------------

// An order of (value, place): larger values first, equal ones by place.  A NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint64_t order_key(float z, uint32_t place) {
  const uint32_t b = __float_as_uint(fmaxf(z, -INFINITY) + 0.f);
  return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~place;
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}
__device__ __forceinline__ uint32_t key_place(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ uint64_t warp_max(uint64_t key) {
  const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(key >> 32));
  const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
  return (uint64_t)hi << 32 | lo;
}

constexpr uint32_t kScoreJoinWarps = 16;  // rows of a CTA: a sector of the segments' numbers serves eight of them
constexpr uint32_t kFewPicks = 64;        // logits that a row's alternatives are usually among

// A warp a row.
__global__ void __launch_bounds__(32 * kScoreJoinWarps) k_score_join(ScorePiece a) {
  __shared__ uint64_t s_picks[kScoreJoinWarps][kFewPicks];
  after_previous();
  const uint32_t n = a.tokens ? *a.count : a.rows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, m = blockIdx.x * kScoreJoinWarps + warp;
  if (m >= n) return;
  const uint64_t row = a.row0 + (a.tokens ? (uint32_t)a.row_of[m] : m);
  float most = -INFINITY;
  uint64_t seg_key = 0;  // the lane's first segment in the order
  for (uint32_t s = lane; s < a.segs; s += 32) {
    const float v = a.most[(uint64_t)s * a.rows + m];
    most = fmaxf(most, v);
    seg_key = max(seg_key, order_key(v, s));
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
  const float about = most == -INFINITY ? 0.f : most, to_log2 = a.scale * kScoreLog2e;
  float sum = 0.f, moment = 0.f;
  for (uint32_t s = lane; s < a.segs; s += 32) {
    const uint64_t at = (uint64_t)s * a.rows + m;
    const float v = a.most[at], u = max_with_nan(((v == -INFINITY ? 0.f : v) - about) * to_log2, kLeastExponent), e = exp2f(u), part = a.sum[at];
    if (v == -INFINITY && part == 0.f) continue;  // nothing in it (a sum of NaN stays)
    sum = fmaf(part, e, sum);
    moment = fmaf(e, fmaf(part, u, a.moment[at]), moment);
  }
  sum = warp_sum(sum);
  moment = warp_sum(moment);
  const float log_sum = logf(sum);
  if (lane == 0) {
    if (a.tokens) a.logprob[row] = (a.target[m] - about) * a.scale - log_sum;
    if (a.entropy) a.entropy[row] = log_sum - kScoreLn2 * moment / sum;
  }
  if (a.top == 0) return;
  // the first `top` segments, lane j the j-th
  const uint32_t segs = min(a.top, a.segs);
  uint32_t my_seg = 0;
  float least = 0.f;
  for (uint32_t j = 0; j < segs; ++j) {
    const uint64_t key = warp_max(seg_key);
    if (lane == j) my_seg = key_place(key);
    least = key_value(key);
    if (key == seg_key) {
      seg_key = 0;
      for (uint32_t s = lane; s < a.segs; s += 32) {
        const uint64_t k = order_key(a.most[(uint64_t)s * a.rows + m], s);
        if (k < key) seg_key = max(seg_key, k);
      }
    }
  }
  if (segs < a.top) least = -INFINITY;
  // their logits that are not below the last one's maximum; where those are many, not below the `top`-th largest of the lanes' maxima either
  const float* z = a.z + (uint64_t)m * a.ld_z;
  const auto each = [&](auto&& f) {  // f(key) of the lane's logits in the segments
    for (uint32_t j = 0; j < segs; ++j) {
      const uint32_t c = __shfl_sync(0xFFFFFFFFu, my_seg, j) * kSegCols + lane * 4;
      const float4 q = *reinterpret_cast<const float4*>(z + c);
      f(order_key(q.x, c));
      f(order_key(q.y, c + 1));
      f(order_key(q.z, c + 2));
      f(order_key(q.w, c + 3));
    }
  };
  bool few = false;
  uint32_t found = 0;
  for (int round = 0; round < 2 && !few; ++round) {
    found = 0;
    uint64_t mine = 0;
    each([&](uint64_t key) {
      const bool take = key_value(key) >= least;
      const uint32_t mask = __ballot_sync(0xFFFFFFFFu, take), at = found + __popc(mask & ((1u << lane) - 1));
      if (take && at < kFewPicks) s_picks[warp][at] = key;
      found += __popc(mask);
      mine = max(mine, key);
    });
    few = found <= kFewPicks;
    if (few || round == 1) break;
    for (uint32_t j = 0; j < a.top; ++j) {
      const uint64_t key = warp_max(mine);
      least = key_value(key);
      if (mine == key) mine = 0;
    }
    __syncwarp();
  }
  __syncwarp();
  uint64_t pick[kFewPicks / 32] = {}, last = ~0ull;
  if (few) {
#pragma unroll
    for (uint32_t i = 0; i < kFewPicks / 32; ++i) pick[i] = i * 32 + lane < found ? s_picks[warp][i * 32 + lane] : 0;
  }
  for (uint32_t j = 0; j < a.top; ++j) {
    uint64_t best = 0;
    if (few) {
#pragma unroll
      for (uint32_t i = 0; i < kFewPicks / 32; ++i)
        if (pick[i] < last) best = max(best, pick[i]);
    } else {  // many equal logits: all of the segments again
      each([&](uint64_t key) {
        if (key < last) best = max(best, key);
      });
    }
    last = warp_max(best);
    if (lane == 0) {
      const bool there = last != 0 && key_place(last) < a.vocab;
      a.top_ids[row * a.top + j] = there ? (int32_t)key_place(last) : -1;
      a.top_logprobs[row * a.top + j] = there ? (key_value(last) - about) * a.scale - log_sum : -INFINITY;
    }
  }
}

// ---- workspace ----------------------------------------------------------------------------------------------------

static uint64_t score_carve(ScorePiece* a, uint8_t* base, uint32_t rows, uint32_t hidden, uint32_t vocab, uint32_t top) {
  uint64_t off = 0;
  auto take = [&](uint64_t bytes) { const uint64_t o = off; off += align_up_sz(bytes, 256); return base + o; };
  const uint64_t padded = align_up_sz(rows, kMmaTile);
  a->rows = rows;
  a->padded = (uint32_t)padded;
  a->segs = (vocab + kSegCols - 1) / kSegCols;
  a->ld_z = a->segs * kSegCols;
  a->count = reinterpret_cast<uint32_t*>(take(4));
  a->row_of = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->token = reinterpret_cast<int32_t*>(take(4ull * rows));
  a->target = reinterpret_cast<float*>(take(4ull * rows));
  a->most = reinterpret_cast<float*>(take(4ull * rows * a->segs));
  a->sum = reinterpret_cast<float*>(take(4ull * rows * a->segs));
  a->moment = reinterpret_cast<float*>(take(4ull * rows * a->segs));
  a->xc = reinterpret_cast<__nv_bfloat16*>(take(2ull * padded * hidden));
  a->z = reinterpret_cast<float*>(take(top ? 4ull * padded * a->ld_z : 0));
  return off;
}

struct ScoreWork {
  uint32_t hidden, vocab, top;
  uint64_t rows;
  uint64_t bytes(uint32_t piece) const {
    ScorePiece a;
    return score_carve(&a, nullptr, piece, hidden, vocab, top);
  }
  uint32_t least_rows() const { return (uint32_t)std::min<uint64_t>(rows, kMmaTile); }
  uint32_t best_rows() const {  // with alternatives, pieces whose logits take 4 GiB
    const uint64_t most = top ? std::max<uint64_t>(kMmaTile, (4ull << 30) / (4ull * vocab) / kMmaTile * kMmaTile) : kScoreRowsMost;
    return (uint32_t)std::min<uint64_t>(rows, std::min<uint64_t>(most, kScoreRowsMost));
  }
  uint64_t least() const { return bytes(least_rows()); }
  uint64_t best() const { return bytes(best_rows()); }
  // the largest piece that fits: all rows, or a multiple of 256
  uint32_t piece_for(uint64_t have) const {
    if (bytes(best_rows()) <= have) return best_rows();
    uint32_t lo = 1, hi = (best_rows() + kMmaTile - 1) / kMmaTile;  // in units of 256 rows
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (bytes(mid * kMmaTile) <= have) lo = mid; else hi = mid;
    }
    return std::min(lo * kMmaTile, best_rows());
  }
};

static int32_t token_logprobs(ft_pool* p, ScorePiece a, const __nv_bfloat16* w, uint64_t ldw, uint64_t rows, void* workspace, uint64_t workspace_bytes,
                              cudaStream_t st) {
  const ScoreWork work{a.hidden, a.vocab, a.top, rows};
  if (!workspace || !aligned_to(workspace, 256)) return FT_ERR_INVALID_ARG;
  if (workspace_bytes < work.least()) return FT_ERR_CAPACITY;
  const uint32_t piece = work.piece_for(workspace_bytes);
  score_carve(&a, static_cast<uint8_t*>(workspace), piece, a.hidden, a.vocab, a.top);
  a.call_seq = status_seq(p);
  a.pairs = (uint32_t)p->sm_count / 2;
  CUtensorMap map_x, map_w, map_z = {};
  if (mma_map(&map_w, w, a.hidden, a.vocab, ldw) != CUDA_SUCCESS || (a.top && mma_map(&map_z, a.z, a.ld_z, a.padded, a.ld_z, 32, true) != CUDA_SUCCESS))
    return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  if (!p->score_attr_set) {  // once per pool, hence once per device the pool lives on
    for (auto k : {k_score<false, 1>, k_score<false, 2>, k_score<true, 1>, k_score<true, 2>})
      FT_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMmaSmem));
    p->score_attr_set = true;
  }
  for (uint64_t r0 = 0; r0 < rows; r0 += piece) {
    a.row0 = r0;
    a.rows = (uint32_t)std::min<uint64_t>(piece, rows - r0);
    if ((a.tokens ? mma_map(&map_x, a.xc, a.hidden, a.padded, a.hidden) : mma_map(&map_x, a.x + r0 * a.ldx, a.hidden, a.rows, a.ldx)) != CUDA_SUCCESS)
      return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    if (a.tokens) {
      if (a.rows <= kScorePickFewUpTo) k_score_pick<kScorePickFew><<<(a.rows + kScorePickFew - 1) / kScorePickFew, 256, 0, st>>>(p->view, a);
      else k_score_pick<kScorePickRows><<<(a.rows + kScorePickRows - 1) / kScorePickRows, 256, 0, st>>>(p->view, a);
      FT_CUDA(cudaGetLastError());
      p->gpu_launches += 1;
    }
    const bool high = a.rows > kMmaTile && a.hidden <= kScoreHigh * kMmaK;
    const auto kernel = a.top ? (high ? k_score<true, 2> : k_score<true, 1>) : (high ? k_score<false, 2> : k_score<false, 1>);
    FT_CUDA(launch_chained(kernel, 2 * a.pairs, kMmaThreads, kMmaSmem, st, map_x, map_w, map_z, p->view, a));
    FT_CUDA(launch_chained(k_score_join, dim3((a.rows + kScoreJoinWarps - 1) / kScoreJoinWarps), 32 * kScoreJoinWarps, 0, st, a));
    p->gpu_launches += 2;
  }
  return FT_OK;
}

}  // namespace ft

using namespace ft;

FT_EXPORT int32_t pool_token_logprobs_workspace(ft_pool* p, uint64_t rows, uint32_t hidden, uint32_t vocab, uint32_t top, uint64_t* least, uint64_t* best) {
  if (!p || hidden == 0 || hidden % 8 || vocab == 0 || !least || !best) return FT_ERR_INVALID_ARG;
  if (rows >> 31 || vocab >> 31 || top > FT_LOGPROBS_MAX_TOP) return FT_ERR_CAPACITY;
  const ScoreWork work{hidden, vocab, top, rows};
  *least = rows ? work.least() : 0;
  *best = rows ? work.best() : 0;
  return FT_OK;
}

FT_EXPORT int32_t pool_token_logprobs(ft_pool* p, uint64_t rows, uint32_t hidden, uint32_t vocab, const void* x, uint64_t ldx, const void* w,
                                      uint64_t ldw, const int32_t* tokens, float logit_scale, float* logprob, float* entropy, uint32_t top,
                                      int32_t* top_ids, float* top_logprobs, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!p || !on_pool_device(p)) return FT_ERR_INVALID_ARG;
  p->call_seq++;
  if (hidden == 0 || hidden % 8 || vocab == 0) return FT_ERR_INVALID_ARG;
  if (rows >> 31 || vocab >> 31) return FT_ERR_CAPACITY;
  if (rows == 0) return FT_OK;
  if (!x || !aligned_to(x, 16) || ldx < hidden || ldx % 8 || !w || !aligned_to(w, 16) || ldw < hidden || ldw % 8) return FT_ERR_INVALID_ARG;
  if (!aligned_to(tokens, 4) || !(logit_scale > 0.f) || std::isinf(logit_scale) || !tokens != !logprob || !aligned_to(logprob, 4) || !aligned_to(entropy, 4))
    return FT_ERR_INVALID_ARG;
  if (top > FT_LOGPROBS_MAX_TOP) return FT_ERR_CAPACITY;
  if ((top && (!top_ids || !top_logprobs)) || !aligned_to(top_ids, 4) || !aligned_to(top_logprobs, 4)) return FT_ERR_INVALID_ARG;
  ScorePiece a = {};
  a.hidden = hidden; a.vocab = vocab; a.ldx = ldx; a.x = static_cast<const __nv_bfloat16*>(x); a.tokens = tokens; a.scale = logit_scale;
  a.logprob = logprob; a.entropy = entropy; a.top = top; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
  return token_logprobs(p, a, static_cast<const __nv_bfloat16*>(w), ldw, rows, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

// Orthogonalisation of a matrix by Newton-Schulz products, and the update of weight matrices that uses it (Muon: a momentum,
// whose singular values are all brought near one before it is applied).
//
// With X = U / |U| (Frobenius norm: all singular values are at most 1), each step maps every singular value s of X by the
// odd quintic p(s) = a s + b s^3 + c s^5 and leaves the singular vectors:
//     A = X X^T,   B = b A + c A^2,   X <- a X + B X,      (a, b, c) = (3.4445, -4.7750, 2.0315)
// p rises by 3.44 at zero and keeps [0, 1.203] in itself (its largest value, at s = 0.555, is 1.2024), so after five steps
// everything that was above 0.01 or so lies in [0.68, 1.21].  X is the m x n matrix with m <= n: a tall one is worked on
// transposed.  A and B are symmetric: only tiles on and above the diagonal are computed, and written to both places.
//
// Products.  p multiplies small singular values, and with them the rounding errors beside them, by up to 3.44^steps, so the
// products are kept to float accuracy: every operand is two f16 terms (split_f16.h, 23 bits), three products on the
// half-precision matrix cores each (frag_product.h).  Since the entries of X, A and B are bounded by their spectral norms
// (1.203, 1.45, 2.81), their scales are constants.  (With a I in B the sums of B X would carry a X from their beginning and be
// rounded at its size throughout: three times the error after one step.)  All three live in fragment order only; X in two of them, by rows (the
// contraction of X X^T runs along n) and by columns (that of B X along m): the tile that a block has finished goes through
// LDS and leaves in both.
//
// All matrices of an update go through each phase in one launch: two launches and three a step for all of them.
#include <algorithm>

#include "common.h"
#include "elem.h"
#include "frag_product.h"

namespace vcnn {

static constexpr int kThreads = 256;
static constexpr int kNormBlocks = 256;  // of a matrix
static constexpr int kExpX = 14, kExpA = 14, kExpB = 14;  // 2^14 times those is below 65504
static constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
static constexpr int kTileWords = 2048;  // 16-byte words of a 128 x 128 tile of one term

enum { MUON_A = 0, MUON_B = 1 };

struct MuonBatch {
  MuonTensor t[kMuonBatch];
  unsigned first[kMuonBatch + 1];  // index of a matrix' first block; [tensors]: grid size
  int tensors;
  float momentum, keep, lr;  // keep = 1 - lr * weight decay
  int nesterov;
  int turn;                  // which of the two copies of X by columns is read
};

// The buffers of a matrix in the workspace, in 16-byte words (terms: hi, then lo).
__host__ __device__ __forceinline__ int64_t x_term(const MuonTensor& t) { return (int64_t)t.mt * t.nt * kTileWords; }
__host__ __device__ __forceinline__ int64_t a_term(const MuonTensor& t) { return (int64_t)t.mt * t.mt * kTileWords; }
__device__ __forceinline__ uint4* x_rows(const MuonTensor& t) { return t.work; }
__device__ __forceinline__ uint4* x_cols(const MuonTensor& t, int turn) { return t.work + (2 + 2 * turn) * x_term(t); }
__device__ __forceinline__ uint4* mat_a(const MuonTensor& t) { return t.work + 6 * x_term(t); }
__device__ __forceinline__ uint4* mat_b(const MuonTensor& t) { return mat_a(t) + 2 * a_term(t); }
static inline int64_t work_words(const MuonTensor& t) { return 6 * x_term(t) + 4 * a_term(t) + kNormBlocks * 8 / 16; }
__device__ __forceinline__ double* norms(const MuonTensor& t) { return reinterpret_cast<double*>(mat_b(t) + 2 * a_term(t)); }

__device__ __forceinline__ int tensor_of(const MuonBatch& b) {
  int t = 0;
  while (t + 1 < b.tensors && blockIdx.x >= b.first[t + 1]) ++t;
  return t;
}

// The matrix to orthogonalise, from the gradient and the momentum as updated.
__device__ __forceinline__ float direction(const MuonBatch& b, float g, float m) {
  return b.nesterov ? fmaf(b.momentum, m, g) : m;
}

// ---- momentum, sum of squares -----------------------------------------------------------------------------------------
// In double: the squares of floats and their sums leave no range and lose nothing that matters.
__global__ __launch_bounds__(kThreads) void muon_moment_kernel(MuonBatch b) {
  const MuonTensor& t = b.t[tensor_of(b)];
  const int block = blockIdx.x - b.first[tensor_of(b)];
  const int64_t count = (int64_t)t.rows * t.cols;
  double sum = 0.;
  for (int64_t i = (int64_t)block * kThreads + threadIdx.x; i < count; i += (int64_t)t.norm_blocks * kThreads) {
    float u = t.g[i];
    if (t.m) {
      const float m = fmaf(b.momentum, t.m[i], u);
      t.m[i] = m;
      u = direction(b, u, m);
    }
    sum += (double)u * u;
  }
  __shared__ double waves[kThreads / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) norms(t)[block] = waves[0] + waves[1] + waves[2] + waves[3];
}
// 1 / |U|; zero for a matrix of zeros, NaN where an element is not finite.  Called by whole blocks;
// `waves`: four doubles of LDS, free again afterwards.
__device__ __forceinline__ double inverse_norm(const MuonTensor& t, double* waves) {
  double sum = (int)threadIdx.x < t.norm_blocks ? norms(t)[threadIdx.x] : 0.;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = waves[0] + waves[1] + waves[2] + waves[3];
  __syncthreads();
  if (!(sum < __builtin_inf())) return __builtin_nan("");
  return sum > 0. ? 1. / sqrt(sum) : 0.;
}

// ---- a wave's 64 x 64 values in LDS -----------------------------------------------------------------------------------
// Element (i, j) at 64 i + (j ^ shift(i)): conflict-free along j, for a row's four neighbours in eight rows at a time, and for
// rows four apart.
__device__ __forceinline__ int shift_of(int i) { return (i & 7) << 2 ^ (i & 4) << 3; }
__device__ __forceinline__ int at64(int i, int j) { return i * 64 + (j ^ shift_of(i)); }

// Writes the values as two row tiles by four steps of fragments: rows i and contraction j, or (COLS) rows j and contraction i.
// change(v, word, row, k): eight values of row `row`, contraction k .. k + 7 (both within the wave's part); word: their place.
template <bool COLS, typename F>
__device__ __forceinline__ void put_fragments(const float* v64, uint4* dst, int64_t term, int row_tile, int step, int steps,
                                              int exponent, F change) {
  const int lane = threadIdx.x & 63;
#pragma unroll 2
  for (int f = 0; f < 8; ++f) {
    const int row = (f >> 2) * 32 + (lane & 31), k = (f & 3) * 16 + (lane >> 5) * 8;
    float v[8];
    if (COLS) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = v64[at64(k + e, row)];
    } else {
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const float4 p = *reinterpret_cast<const float4*>(v64 + at64(row, k + e));
        v[e] = p.x, v[e + 1] = p.y, v[e + 2] = p.z, v[e + 3] = p.w;
      }
    }
    const int64_t word = ((int64_t)(row_tile + (f >> 2)) * steps + step + (f & 3)) * 64 + lane;
    change(v, word, row, k);
    uint32_t s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = split_f16(v[e], exponent);
    uint4 hi, lo;
    pack_terms(s, &hi, &lo);
    dst[word] = hi, dst[term + word] = lo;
  }
}

// ---- X = U / |U| in both orders ---------------------------------------------------------------------------------------
__global__ __launch_bounds__(kThreads) void muon_begin_kernel(MuonBatch b) {
  __shared__ __attribute__((aligned(16))) float smem[4][64 * 64];
  const MuonTensor& t = b.t[tensor_of(b)];
  const int tile = blockIdx.x - b.first[tensor_of(b)], it = tile % t.mt, jt = tile / t.mt;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i0 = it * kFragTile + (wave & 1) * 64, j0 = jt * kFragTile + (wave >> 1) * 64;
  const double inverse = inverse_norm(t, reinterpret_cast<double*>(smem[0]));
  float* const v64 = smem[wave];
#pragma unroll 4
  for (int r = 0; r < 64; ++r) {  // rows of the matrix as stored: of X, or of a tall matrix its columns
    const int i = t.tall ? lane : r, j = t.tall ? r : lane;
    float x = 0.f;
    if (i0 + i < t.small && j0 + j < t.large) {
      const int64_t at = t.tall ? (int64_t)(j0 + j) * t.small + i0 + i : (int64_t)(i0 + i) * t.large + j0 + j;
      const float g = t.g[at];
      x = (float)((t.m ? direction(b, g, t.m[at]) : g) * inverse);
    }
    v64[at64(i, j)] = x;
  }
  const auto as_is = [](float (&)[8], int64_t, int, int) {};
  put_fragments<false>(v64, x_rows(t), x_term(t), i0 / 32, j0 / 16, t.nt * 8, kExpX, as_is);
  put_fragments<true>(v64, x_cols(t, b.turn), x_term(t), j0 / 32, i0 / 16, t.mt * 8, kExpX, as_is);
}

// ---- products -----------------------------------------------------------------------------------------------------------
// The tile (it, jt) of rows by columns, both along `steps` steps, as this wave's 64 x 64 part in LDS.
__device__ __forceinline__ float* tile_product(const uint4* rows, int64_t rows_term, const uint4* cols, int64_t cols_term,
                                               int it, int jt, int steps, float scale, uint4* smem) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint4* const a = rows + (int64_t)(4 * it + wave) * steps * 64 + lane;
  const uint4* const c = cols + (int64_t)(4 * jt + wave) * steps * 64 + lane;
  constexpr int S = FragSlab<2>::STEPS;
  f32x16 acc[2][2];
  frag_product<2>(steps / S, smem, rows_term, cols_term, [&](int sl) { return a + sl * (S * 64); },
                  [&](int sl) { return c + sl * (S * 64); }, acc);
  float* const v64 = reinterpret_cast<float*>(smem) + wave * (64 * 64);
#pragma unroll
  for (int mi = 0; mi < 2; ++mi)
#pragma unroll
    for (int ni = 0; ni < 2; ++ni)
#pragma unroll
      for (int q = 0; q < 16; ++q) v64[at64(mi * 32 + acc_row(q, lane), ni * 32 + (lane & 31))] = acc[mi][ni][q] * scale;
  return v64;
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// the two terms at `word` of a matrix, joined and scaled back
__device__ __forceinline__ void join8(const uint4* src, int64_t term, int64_t word, float scale, float (&v)[8]) {
  const f16x8 hi = __builtin_bit_cast(f16x8, src[word]), lo = __builtin_bit_cast(f16x8, src[term + word]);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = fmaf((float)lo[e], 1.f / 2048.f, (float)hi[e]) * scale;
}

// MUON_A: A = X X^T.  MUON_B: B = b A + c A A^T.
template <int WHAT>
__global__ __launch_bounds__(kThreads, 2) void muon_square_kernel(MuonBatch b) {
  extern __shared__ uint4 smem16[];
  const MuonTensor& t = b.t[tensor_of(b)];
  int it = blockIdx.x - b.first[tensor_of(b)], jt = 0;
  while (it > jt) it -= ++jt;  // column jt of the upper triangle has jt + 1 tiles
  const int wave = threadIdx.x >> 6;
  const uint4* const src = WHAT == MUON_A ? x_rows(t) : mat_a(t);
  const int64_t src_term = WHAT == MUON_A ? x_term(t) : a_term(t);
  const float* const v64 = tile_product(src, src_term, src, src_term, it, jt, (WHAT == MUON_A ? t.nt : t.mt) * 8,
                                        pow2(WHAT == MUON_A ? -2 * kExpX : -2 * kExpA), smem16);
  const int i0 = it * kFragTile + (wave & 1) * 64, j0 = jt * kFragTile + (wave >> 1) * 64;
  uint4* const dst = WHAT == MUON_A ? mat_a(t) : mat_b(t);
  const auto polynomial = [&](float (&v)[8], int64_t word, int, int) {
    if (WHAT == MUON_A) return;
    float a8[8];
    join8(mat_a(t), a_term(t), word, pow2(-kExpA), a8);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(kC, v[e], kB * a8[e]);
  };
  constexpr int exponent = WHAT == MUON_A ? kExpA : kExpB;
  put_fragments<false>(v64, dst, a_term(t), i0 / 32, j0 / 16, t.mt * 8, exponent, polynomial);
  if (it != jt) put_fragments<true>(v64, dst, a_term(t), j0 / 32, i0 / 16, t.mt * 8, exponent, polynomial);
}

// X <- a X + B X; the last one: the result, or the weights moved by it.
template <bool LAST>
__global__ __launch_bounds__(kThreads, 2) void muon_apply_kernel(MuonBatch b) {
  extern __shared__ uint4 smem16[];
  const MuonTensor& t = b.t[tensor_of(b)];
  const int tile = blockIdx.x - b.first[tensor_of(b)], it = tile % t.mt, jt = tile / t.mt;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* const v64 = tile_product(mat_b(t), a_term(t), x_cols(t, b.turn), x_term(t), it, jt, t.mt * 8,
                                        pow2(-kExpB - kExpX), smem16);
  const int i0 = it * kFragTile + (wave & 1) * 64, j0 = jt * kFragTile + (wave >> 1) * 64;
#pragma unroll 2
  for (int f = 0; f < 8; ++f) {  // a X, from X by rows (whose place the same lanes write below)
    const int row = (f >> 2) * 32 + (lane & 31), k = (f & 3) * 16 + (lane >> 5) * 8;
    float x[8];
    join8(x_rows(t), x_term(t), ((int64_t)(i0 / 32 + (f >> 2)) * (t.nt * 8) + j0 / 16 + (f & 3)) * 64 + lane, pow2(-kExpX), x);
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      float4* const p = reinterpret_cast<float4*>(v64 + at64(row, k + e));
      const float4 v = *p;
      *p = make_float4(fmaf(kA, x[e], v.x), fmaf(kA, x[e + 1], v.y), fmaf(kA, x[e + 2], v.z), fmaf(kA, x[e + 3], v.w));
    }
  }
  if constexpr (!LAST) {
    const auto as_is = [](float (&)[8], int64_t, int, int) {};
    put_fragments<false>(v64, x_rows(t), x_term(t), i0 / 32, j0 / 16, t.nt * 8, kExpX, as_is);
    put_fragments<true>(v64, x_cols(t, b.turn ^ 1), x_term(t), j0 / 32, i0 / 16, t.mt * 8, kExpX, as_is);
  } else {
    const float step = b.lr * t.factor;
#pragma unroll 4
    for (int r = 0; r < 64; ++r) {
      const int i = t.tall ? lane : r, j = t.tall ? r : lane;
      if (i0 + i >= t.small || j0 + j >= t.large) continue;
      const int64_t at = t.tall ? (int64_t)(j0 + j) * t.small + i0 + i : (int64_t)(i0 + i) * t.large + j0 + j;
      const float o = v64[at64(i, j)];
      if (t.out) {
        t.out[at] = o;
      } else {
        const float w = fmaf(-step, o, b.keep * t.w[at]);
        t.w[at] = w;
        if (t.w16) st(reinterpret_cast<bf16*>(t.w16) + at, w);
      }
    }
  }
}

// ---- launches -----------------------------------------------------------------------------------------------------------
static void lay_out(MuonTensor* t) {
  t->tall = t->rows > t->cols;
  t->small = std::min(t->rows, t->cols), t->large = std::max(t->rows, t->cols);
  t->mt = (int)ceil_div(t->small, kFragTile), t->nt = (int)ceil_div(t->large, kFragTile);
  t->norm_blocks = (int)std::min<int64_t>(kNormBlocks, ceil_div((int64_t)t->rows * t->cols, 4 * kThreads));
}

size_t muon_workspace(int tensors, const int32_t* rows, const int32_t* cols) {
  int64_t most = 0;
  for (int t0 = 0; t0 < tensors; t0 += kMuonBatch) {  // batches follow one another in the same memory
    int64_t words = 0;
    for (int t = t0; t < std::min(tensors, t0 + kMuonBatch); ++t) {
      MuonTensor m{};
      m.rows = rows[t], m.cols = cols[t];
      lay_out(&m);
      words += work_words(m);
    }
    most = std::max(most, words);
  }
  return (size_t)most * 16;
}

template <typename K, typename N>
static vcnn_status launch_phase(const char* what, K kernel, MuonBatch* b, size_t lds, hipStream_t st, N blocks_of) {
  int64_t blocks = 0;
  for (int t = 0; t < b->tensors; ++t) {
    b->first[t] = (unsigned)blocks;
    blocks += blocks_of(b->t[t]);
  }
  if (blocks > 0x7fffffffLL) return fail(VCNN_ERR_UNSUPPORTED, "%s: too many tiles", what);
  b->first[b->tensors] = (unsigned)blocks;
  if (lds) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), lds, st, *b);
  return check_launch(what);
}

vcnn_status launch_muon(const MuonTensor* tensors, int count, float lr, float momentum, int nesterov, float weight_decay,
                        int steps, void* workspace, hipStream_t st) {
  constexpr size_t lds = FragSlab<2>::LDS_BYTES;
  static_assert(lds >= 4 * 64 * 64 * sizeof(float), "a tile fits the slabs' memory");
  MuonBatch b{};
  b.tensors = count;
  b.lr = lr, b.momentum = momentum, b.nesterov = nesterov, b.keep = 1.f - lr * weight_decay;
  uint4* work = (uint4*)workspace;
  for (int t = 0; t < b.tensors; ++t) {
    b.t[t] = tensors[t];
    lay_out(&b.t[t]);
    b.t[t].work = work;
    work += work_words(b.t[t]);
  }
  const auto tiles = [](const MuonTensor& t) { return (int64_t)t.mt * t.nt; };
  const auto triangle = [](const MuonTensor& t) { return (int64_t)t.mt * (t.mt + 1) / 2; };
  if (vcnn_status s = launch_phase("muon moment", muon_moment_kernel, &b, 0, st, [](const MuonTensor& t) { return t.norm_blocks; })) return s;
  if (vcnn_status s = launch_phase("muon begin", muon_begin_kernel, &b, 0, st, tiles)) return s;
  for (int i = 0; i < steps; ++i, b.turn ^= 1) {
    if (vcnn_status s = launch_phase("muon A", muon_square_kernel<MUON_A>, &b, lds, st, triangle)) return s;
    if (vcnn_status s = launch_phase("muon B", muon_square_kernel<MUON_B>, &b, lds, st, triangle)) return s;
    if (vcnn_status s = i + 1 < steps ? launch_phase("muon apply", muon_apply_kernel<false>, &b, lds, st, tiles)
                                      : launch_phase("muon apply", muon_apply_kernel<true>, &b, lds, st, tiles))
      return s;
  }
  return VCNN_OK;
}

}  // namespace vcnn

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
// products are kept to float accuracy: every operand v is two f16 terms, hi + lo of v times a power of two, and a product is
// the three products hi hi + hi lo + lo hi on the half-precision matrix cores, in one float accumulator; what is left out, lo lo,
// is 2^-22 of a product at most.  (With a I in B the sums of B X would carry a X from their beginning and be rounded at its
// size throughout: three times the error after one step.)
// The terms are of X by rows (the contraction of X X^T runs along n), X by columns (that of B X along m), A and B, in fragment
// order, frag[16-row tile][step of 32][lane][8]: word `lane` holds row lane % 16 and elements 8 (lane / 16) + 0..7 of the step,
// what the lane feeds to one v_mfma_f32_16x16x32_f16 (1.9 PFLOP/s on this card with operands in registers; the 32 x 32 x 16
// form, by the power it draws, 1.6); X itself stays in floats beside them, for a X.  The tile that a block has finished goes
// through LDS and leaves in all of them.
//
// The powers of two.  Float products keep a row, or a column, that is far smaller than the others to its own accuracy: a X and B X
// scale row by row and column by column (the gradients of maps that are seldom active are such rows).  Under one power for all,
// terms lose bits of what lies below 2^-16 of the norm, down to nothing.  So row i of X has a power d_i of its own, and
// column j a power e_j:
//     X by rows  d_i X_ij,    A  d_i A_ij,    B  d_i B_ij,    X by columns  X_ij e_j
// A sum of products of two rows then carries d_i d_k, of B and a column d_i e_j, and the columns k of A and B, whose contribution
// to row i is in proportion to |X_k|, need no power.  d_i |X_i| is kept below 2^14, which keeps rows of A below 1.21 and of B
// below 2.82 of that (|x| <= |X_i| times the largest of s and of |b s + c s^3|), within f16.  A step multiplies the norm of a row or
// column by 0.63 (the least of a + b s^2 + c s^4) to 3.4445, so d follows from the diagonal of A, d_i^2 |X_i|^2, one step ahead; e
// from the largest entry of the column, which the blocks of a step collect by a maximum in memory (of integers, the same in any
// order) and which bounds the norm to sqrt(m) of itself: the terms of what is below 2^-10 of it (m = 4096) are off by up to 2^-33
// of it.  d of the first X is found like that too.  Beside one power for all and no X in floats this costs 2 to 6 % (4096 x 4096
// 4.04 ms, not 3.94; 1024 x 4096 393 us, not 378; 64 x 800 82, not 79), most of it for writing X once more.
//
// Tiles.  256 x 256 and 128 x 128 from slabs in LDS; where there are too few of those for the chip, 64 x 64 with the
// contraction divided over the block's eight waves, which read their fragments straight from the caches.
//
// All matrices of an update go through each phase in one launch: two at first, then a step in two (all matrices of at most 64
// rows), three, or four (long sums over few tiles, shared by blocks).  4096 x 4096 and 8192 x 2048 together take 5.53 ms, five
// steps: 1.05 PFLOP/s of f16 products (B X of both 1.15, X X^T 1.03, A^2 0.91, whose tiles come in 1.3 rounds of what the chip
// holds), a plain f16 product of 8192^3 1.32.  The products draw so much power that the clock falls to 1.9 GHz; the
// matrix cores are then busy 57 % of the time in B X, 50 in X X^T and 45 in A^2.  1024 x 4096 takes 0.40 ms, bound by the rate at which a CU reads its
// cache (X X^T) and by the latency of 32 steps (B X); 64 x 800 79 us and 500 x 800 beside three smaller ones 170, by that of
// the launches.
#include <algorithm>

#include "common.h"
#include "elem.h"
#include "bf16_core.h"
#include "mma_core.h"

namespace vcnn {

static constexpr int kThreads = 256;
static constexpr int kNormBlocks = 1024;  // of a matrix, at most
static constexpr int kJoinBlocks = 256;  // of a phase whose sums are shared by several blocks
static constexpr int kSharedSteps = 64;  // of the longest, from which on sums are shared
static constexpr int kPad = 128;         // sides in the workspace are multiples of it
static constexpr int kRowTop = 14, kColTop = 15;  // d_i |X_i| < 2^14 (2.82 * 2^14 < 65504), e_j X_ij < 2^15
static constexpr float kGrowth = 3.5f, kMost = 1.25f;  // of a row's norm in a step, and of any row: a little above the bounds
static constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
static constexpr int kTileWords = kPad * kPad / 8;  // 16-byte words of a 128 x 128 tile of one term

enum { MUON_A = 0, MUON_B = 1 };

struct MuonBatch {
  MuonTensor t[kMuonBatch];
  unsigned first[kMuonBatch + 1];  // index of a matrix' first block; [tensors]: grid size
  int tensors;
  float momentum, keep, lr;  // keep = 1 - lr * weight decay
  int nesterov;
  int turn;                  // which of the two copies of X by columns, and of the powers, is read
  int third;                 // which of the three arrays of columns' largest entries is
  int small;                 // all matrices have at most 64 rows (as X)
  float* shares;             // [kJoinBlocks][64 * 64]: sums of blocks that share a tile
};

// The buffers of a matrix in the workspace, in 16-byte words (terms: hi, then lo).
__host__ __device__ __forceinline__ int64_t x_term(const MuonTensor& t) { return (int64_t)t.mt * t.nt * kTileWords; }
__host__ __device__ __forceinline__ int64_t a_term(const MuonTensor& t) { return (int64_t)t.mt * t.mt * kTileWords; }
__device__ __forceinline__ uint4* x_rows(const MuonTensor& t) { return t.work; }
__device__ __forceinline__ uint4* x_cols(const MuonTensor& t, int turn) { return t.work + (2 + 2 * turn) * x_term(t); }
__device__ __forceinline__ uint4* mat_a(const MuonTensor& t) { return t.work + 6 * x_term(t); }
__device__ __forceinline__ uint4* mat_b(const MuonTensor& t) { return mat_a(t) + 2 * a_term(t); }
__device__ __forceinline__ double* norms(const MuonTensor& t) { return reinterpret_cast<double*>(mat_b(t) + 2 * a_term(t)); }
// X as floats, 64 x 64 parts as in LDS below: the one at (i0, j0).
__device__ __forceinline__ float4* x_floats(const MuonTensor& t, int i0, int j0) {
  return reinterpret_cast<float4*>(mat_b(t) + 2 * a_term(t) + kNormBlocks * 8 / 16) + ((int64_t)(i0 / 64) * t.pn + j0 / 64) * 1024;
}
// Per row: 1 / d_i (two turns).  Per column: 1 / e_j (two turns), the bits of its largest magnitude (three).  And the largest
// magnitudes of U that the blocks of muon_moment_kernel saw, [gn] of a row and [gm] of a column.
__host__ __device__ __forceinline__ int64_t row_pitch(const MuonTensor& t) { return (int64_t)t.mt * kPad; }
__host__ __device__ __forceinline__ int64_t col_pitch(const MuonTensor& t) { return (int64_t)t.nt * kPad; }
__device__ __forceinline__ float* inv_d(const MuonTensor& t, int turn) {
  return reinterpret_cast<float*>(x_floats(t, t.pm * 64, 0)) + turn * row_pitch(t);
}
__device__ __forceinline__ float* inv_e(const MuonTensor& t, int turn) { return inv_d(t, 2) + turn * col_pitch(t); }
__device__ __forceinline__ uint32_t* col_most(const MuonTensor& t, int third) {
  return reinterpret_cast<uint32_t*>(inv_e(t, 2 + third));
}
__device__ __forceinline__ uint32_t* row_seen(const MuonTensor& t, int g) { return col_most(t, 3) + g * row_pitch(t); }
__device__ __forceinline__ uint32_t* col_seen(const MuonTensor& t, int g) { return row_seen(t, t.gn) + g * col_pitch(t); }
static inline int64_t work_words(const MuonTensor& t) {
  return 6 * x_term(t) + 4 * a_term(t) + kNormBlocks * 8 / 16 + (int64_t)t.pm * t.pn * 1024 +
         ((2 + t.gn) * row_pitch(t) + (5 + t.gm) * col_pitch(t)) / 4;
}

// The power of two that takes what is at most `bound` below 2^top, up to 2^126, whose reciprocal is the smallest normal float.
// (Any would do for zero.)
__device__ __forceinline__ float power_for(float bound, int top) {
  const int exponent = __float_as_int(bound) >> 23 & 255;  // bound < 2^(exponent - 126)
  return __int_as_float((min(top + 126 - exponent, 126) + 127) << 23);
}
__device__ __forceinline__ float inverse_power(float p) { return __int_as_float(0x7f000000 - __float_as_int(p)); }
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }  // (a NaN is the largest)

__device__ __forceinline__ int tensor_of(const MuonBatch& b) {
  int t = 0;
  while (t + 1 < b.tensors && blockIdx.x >= b.first[t + 1]) ++t;
  return t;
}

// The matrix to orthogonalise, from the gradient and the momentum as updated.
__device__ __forceinline__ float direction(const MuonBatch& b, float g, float m) {
  return b.nesterov ? fmaf(b.momentum, m, g) : m;
}

// ---- momentum, sum of squares, largest magnitudes ------------------------------------------------------------------------
// What a block of 256 threads sees of the 64 x 64 part at (i0, j0) of X in the matrix as stored: thread (wave, lane) has column
// `lane` of rows wave * 16 + 0..15, which of a tall matrix are X's columns.
struct Part {
  int64_t at0;
  int pitch, rows_left, cols_left;  // of the stored matrix
  __device__ __forceinline__ Part(const MuonTensor& t, int i0, int j0)
      : at0(t.tall ? (int64_t)j0 * t.small + i0 : (int64_t)i0 * t.large + j0), pitch(t.tall ? t.small : t.large),
        rows_left(t.tall ? t.large - j0 : t.small - i0), cols_left(t.tall ? t.small - i0 : t.large - j0) {}
  __device__ __forceinline__ bool there(int r) const {
    return (int)(threadIdx.x >> 6) * 16 + r < rows_left && (int)(threadIdx.x & 63) < cols_left;
  }
  // (behind the end: the last one's, which nobody uses, so that loads wait for no condition)
  __device__ __forceinline__ int64_t at(int r) const {
    return at0 + (int64_t)min((int)(threadIdx.x >> 6) * 16 + r, rows_left - 1) * pitch + min((int)(threadIdx.x & 63), cols_left - 1);
  }
};

// A block takes one of gm x gn groups of parts.  Sums in double: the squares of floats and their sums leave no range and lose
// nothing that matters.
__global__ __launch_bounds__(kThreads) void muon_moment_kernel(MuonBatch b) {
  __shared__ uint32_t over_rows[2][kThreads / 64][64], over_cols[2][64];  // parts take turns: one barrier each
  __shared__ double waves[kThreads / 64];
  const int at_tensor = tensor_of(b);
  const MuonTensor& t = b.t[at_tensor];
  const int block = blockIdx.x - b.first[at_tensor], gi = block / t.gn, gj = block % t.gn;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // (at most 2^18 parts a side, 256 groups)
  const int p0 = (unsigned)(t.pm * gi) / t.gm, p1 = (unsigned)(t.pm * (gi + 1)) / t.gm;
  const int q0 = (unsigned)(t.pn * gj) / t.gn, q1 = (unsigned)(t.pn * (gj + 1)) / t.gn;
  double sum = 0.;
  int turn = 0;
  for (int p = p0; p < p1; ++p)
    for (int q = q0; q < q1; ++q, turn ^= 1) {
      const Part part(t, p * 64, q * 64);
      float g[16], m[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) g[r] = t.g[part.at(r)];
      if (t.m) {
#pragma unroll
        for (int r = 0; r < 16; ++r) m[r] = t.m[part.at(r)];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          m[r] = fmaf(b.momentum, m[r], g[r]), g[r] = direction(b, g[r], m[r]);
          if (part.there(r)) t.m[part.at(r)] = m[r];
        }
      }
      uint32_t v[16], most = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (!part.there(r)) g[r] = 0.f;
        sum += (double)g[r] * g[r];
        v[r] = magnitude(g[r]), most = max(most, v[r]);
      }
      // over the lanes: each step keeps the half of the rows that a bit of the lane chooses; lane 4 r has row r in the end
#pragma unroll
      for (int n = 8, d = 32; n > 0; n >>= 1, d >>= 1) {
        const bool up = lane & d;
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = max(up ? v[i + n] : v[i], (uint32_t)__shfl_xor((int)(up ? v[i] : v[i + n]), d));
      }
      v[0] = max(v[0], (uint32_t)__shfl_xor((int)v[0], 2));
      v[0] = max(v[0], (uint32_t)__shfl_xor((int)v[0], 1));
      over_rows[turn][wave][lane] = most;
      if (lane % 4 == 0) over_cols[turn][wave * 16 + lane / 4] = v[0];
      __syncthreads();
      if (threadIdx.x < 128) {  // of a column as stored, of a row as stored: of X's row or column; this thread's in every part
        const auto& waves_most = over_rows[turn];
        most = threadIdx.x < 64 ? max(max(waves_most[0][lane], waves_most[1][lane]), max(waves_most[2][lane], waves_most[3][lane]))
                                : over_cols[turn][lane];
        const bool row = (threadIdx.x < 64) == (bool)t.tall;
        uint32_t* const seen = row ? row_seen(t, gj) + p * 64 + lane : col_seen(t, gi) + q * 64 + lane;
        *seen = (row ? q > q0 : p > p0) ? max(*seen, most) : most;
      }
    }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) waves[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) norms(t)[block] = waves[0] + waves[1] + waves[2] + waves[3];
}
// 1 / |U| from a thread's share of the sum of squares; zero for a matrix of zeros, NaN where an element is not finite.  Called
// by whole blocks; `waves`: four doubles of LDS, free again afterwards.
__device__ __forceinline__ double inverse_norm(double sum, double* waves) {
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
// Element (i, j) at 64 i + (j ^ shift(i)), shift a multiple of four: the accumulators' writes (sixteen neighbours of rows four
// apart), the reads of rows (four neighbours of sixteen rows) and of columns (sixteen neighbours of rows eight apart) each meet
// all 64 banks.
__device__ __forceinline__ int shift_of(int i) { return (i & 7) << 2 ^ (i & 4) << 3 ^ (i & 8) << 1 ^ (i & 16) << 1; }
__device__ __forceinline__ int at64(int i, int j) { return i * 64 + (j ^ shift_of(i)); }

// Eight values as two terms.
__device__ __forceinline__ void split8(const float (&v)[8], uint4* hi, uint4* lo) {
  f16x8 h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    h[e] = (_Float16)v[e];
    l[e] = (_Float16)(v[e] - (float)h[e]);
  }
  *hi = __builtin_bit_cast(uint4, h), *lo = __builtin_bit_cast(uint4, l);
}
__device__ __forceinline__ void join8(const uint4* src, int64_t term, int64_t word, float (&v)[8]) {
  const f16x8 hi = __builtin_bit_cast(f16x8, src[word]), lo = __builtin_bit_cast(f16x8, src[term + word]);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)hi[e] + (float)lo[e];
}

// Fragment f (of four row tiles by two steps) of the 64 x 64 values: rows i and contraction j, or (COLS) rows j and
// contraction i.  word0: the word of fragment 0; change(v, word, row, k): eight values, their place, row and first contraction.
template <bool COLS, typename F>
__device__ __forceinline__ void put_fragment(const float* v64, uint4* dst, int64_t term, int64_t word0, int steps, int f,
                                             F change) {
  const int lane = threadIdx.x & 63;
  const int row = (f >> 1) * 16 + (lane & 15), k = (f & 1) * 32 + (lane >> 4) * 8;
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
  const int64_t word = word0 + ((int64_t)(f >> 1) * steps + (f & 1)) * 64 + lane;
  change(v, word, row, k);
  uint4 hi, lo;
  split8(v, &hi, &lo);
  dst[word] = hi, dst[term + word] = lo;
}
// Word (without the lane) of the fragment at row i0, contraction j0.
__device__ __forceinline__ int64_t word_of(int i0, int j0, int steps) { return ((int64_t)(i0 / 16) * steps + j0 / 32) * 64; }
// Eight values times eight of an array, or times one.
__device__ __forceinline__ void times8(float (&v)[8], const float* by) {  // (16-byte aligned)
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const float4 p = *reinterpret_cast<const float4*>(by + e);
    v[e] *= p.x, v[e + 1] *= p.y, v[e + 2] *= p.z, v[e + 3] *= p.w;
  }
}
__device__ __forceinline__ void times8(float (&v)[8], float by) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= by;
}
// Place p of the 1024 of four values: row i, columns j .. j + 3.
__device__ __forceinline__ int row_at(int p) { return p >> 4; }
__device__ __forceinline__ int col_at(int p) { return (p & 15) << 2 ^ shift_of(p >> 4); }

// ---- X = U / |U| in both orders ---------------------------------------------------------------------------------------
// A block makes one 64 x 64 part.
__global__ __launch_bounds__(kThreads) void muon_begin_kernel(MuonBatch b) {
  __shared__ __attribute__((aligned(16))) float v64[64 * 64];
  __shared__ uint32_t seen[2][kThreads / 64][64];  // of rows, of columns
  __shared__ float power[2][64];                   // the same
  const int at_tensor = tensor_of(b);
  const MuonTensor& t = b.t[at_tensor];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int at_part = blockIdx.x - b.first[at_tensor];
  // neighbouring parts lie along the rows as stored
  const int i0 = (t.tall ? at_part % t.pm : at_part / t.pn) * 64, j0 = (t.tall ? at_part / t.pm : at_part % t.pn) * 64;
  const Part part(t, i0, j0);
  float x[16];  // of sixteen rows of the matrix as stored: of X, or of a tall matrix its columns
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = t.g[part.at(r)];
  if (t.m) {
    float m[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) m[r] = t.m[part.at(r)];
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = direction(b, x[r], m[r]);
  }
  double sum = 0.;
#pragma unroll 4
  for (int i = threadIdx.x; i < t.gm * t.gn; i += kThreads) sum += norms(t)[i];
  // of row `lane` and of column `lane`, a wave every fourth group
  const auto largest = [&](const uint32_t* from, int64_t pitch, int groups) {
    uint32_t most = 0;
#pragma unroll 8
    for (int g = wave; g < groups; g += kThreads / 64) most = max(most, from[g * pitch + lane]);
    return most;
  };
  const uint32_t of_row = largest(row_seen(t, 0) + i0, row_pitch(t), t.gn);
  const uint32_t of_col = largest(col_seen(t, 0) + j0, col_pitch(t), t.gm);
  seen[0][wave][lane] = of_row, seen[1][wave][lane] = of_col;
  const double inverse = inverse_norm(sum, reinterpret_cast<double*>(v64));
#pragma unroll
  for (int r = 0; r < 16; ++r)
    v64[t.tall ? at64(lane, wave * 16 + r) : at64(wave * 16 + r, lane)] = part.there(r) ? (float)(x[r] * inverse) : 0.f;
  if (wave < 2) {
    const uint32_t most = max(max(seen[wave][0][lane], seen[wave][1][lane]), max(seen[wave][2][lane], seen[wave][3][lane]));
    const float bound = (float)(__uint_as_float(most) * inverse);
    if (wave == 0) {
      const float d = power_for(fminf(bound * sqrtf((float)t.large), 1.f), kRowTop);
      power[0][lane] = d;
      if (j0 == 0) inv_d(t, b.turn)[i0 + lane] = inverse_power(d);
    } else {
      const float e = power_for(bound, kColTop);
      power[1][lane] = e;
      if (i0 == 0 && !b.small) {
        inv_e(t, b.turn)[j0 + lane] = inverse_power(e);
        col_most(t, b.third)[j0 + lane] = magnitude(bound);
        col_most(t, (b.third + 1) % 3)[j0 + lane] = 0;
      }
    }
  }
  __syncthreads();
  float4* const kept = x_floats(t, i0, j0) + threadIdx.x;
#pragma unroll
  for (int n = 0; n < 4; ++n) kept[n * kThreads] = reinterpret_cast<const float4*>(v64)[n * kThreads + threadIdx.x];
  const int by_rows = t.nt * (kPad / 32), by_cols = t.mt * (kPad / 32);
#pragma unroll
  for (int f = 2 * wave; f < 2 * wave + 2; ++f) {
    put_fragment<false>(v64, x_rows(t), x_term(t), word_of(i0, j0, by_rows), by_rows, f,
                        [&](float (&v)[8], int64_t, int row, int) { times8(v, power[0][row]); });
    if (!b.small)
      put_fragment<true>(v64, x_cols(t, b.turn), x_term(t), word_of(j0, i0, by_cols), by_cols, f,
                         [&](float (&v)[8], int64_t, int row, int) { times8(v, power[1][row]); });
  }
}

// ---- products -----------------------------------------------------------------------------------------------------------
// A block's tile: C[i][j] = sum over `steps` steps (of 32) of rows i of one operand times rows j of the other, handed out
// as 64 x 64 parts in LDS.  Row tiles behind the last one read that one again.
struct Operand {
  const uint4* src;
  int64_t term;
  int row_tile;   // first of the tile
  int row_tiles;  // of the operand
  int pitch;      // steps of a row tile
  __device__ __forceinline__ const uint4* frag(int row, int t) const {
    return src + t * term + (int64_t)min(row_tile + row, row_tiles - 1) * pitch * 64;
  }
};

// The accumulators of TA x 4 tiles (register q of lane l: row 4 (l / 16) + q, column l % 16), four by four from row tile
// `first` on, as values in LDS (still times the powers of both operands' rows).
template <int TA>
__device__ __forceinline__ void spread(const f32x4 (&acc)[TA][4], int first, float* v64) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        v64[at64(i * 16 + (lane >> 4) * 4 + q, j * 16 + (lane & 15))] = acc[first + i][j][q];
}

// Tiles of 16 TA WM x 64 WN, a wave 16 TA x 64 of them.  A slab is one step of both operands, both terms; it goes to LDS by
// direct loads, 1 KB each, while the slab before is multiplied: wave w brings four row tiles of it.  A wave's row tiles are
// multiplied in two halves h, in the order  hi_h Bhi, lo_h Bhi, hi_h Blo:  while a half is multiplied the other's fragments
// are read, Bhi of the next slab while the last products are made, Blo while the first are.  One barrier a slab, before the
// last products: behind it the next slab is there, and this one's place is free for the one after.
// RING slabs in LDS, RING - 1 ahead: four where a CU has one tile only and nothing else to do while a slab is on its way.
template <int TA_, int WM_, int WN_, int RING_>
struct SlabTile {
  static constexpr int TA = TA_, WM = WM_, WN = WN_, RING = RING_, WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int BM = 16 * TA * WM, BN = 64 * WN;
  static constexpr int ROWS = TA * WM + 4 * WN;  // row tiles of both operands
  static constexpr int WORDS = ROWS * 128;       // of a slab
  static constexpr size_t LDS = RING * WORDS * 16;
  static_assert(ROWS == 4 * WAVES && TA % 4 == 0, "four row tiles a wave, parts of 64 x 64");
  static_assert(LDS >= WAVES * 64 * 64 * 4, "the parts fit the slabs' memory");

  // part(v64, i0, j0, f0, f1): a 64 x 64 part at (i0, j0) within the tile, for one wave: fragments 0 .. 8 are its own
  template <typename F>
  __device__ static __forceinline__ void run(const Operand& a, const Operand& b, int steps, uint4* smem, F part) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint4* src[4][2];  // [row tile][term]: wave-uniform
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int row = 4 * wave + r;
        src[r][t] = row < TA * WM ? a.frag(row, t) : b.frag(row - TA * WM, t);
      }
    auto stage = [&](int s, int n) {  // load n of eight of slab s (behind the last: that one again, for nobody)
      load_to_lds16(src[n / 2][n % 2] + (int64_t)min(s, steps - 1) * 64, lane * 16,
                    smem + (s % RING) * WORDS + (4 * wave * 2 + n) * 64);
    };
    constexpr int H = TA / 2, LEFT = 8 * (RING - 2);  // loads that may be on their way when the next slab has to be there
    constexpr int WAIT = 0x0F70 | (LEFT & 15) | (LEFT >> 4) << 14;  // vmcnt(LEFT)
    const int ra = (wave % WM) * TA, rb = TA * WM + (wave / WM) * 4;
    f32x4 acc[TA][4];
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    uint4 fa[2][2][H], fb[2][4];  // [half][term], [term]
    auto read_a = [&](int s, int h) {
      const uint4* const buf = smem + (s % RING) * WORDS + lane;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < H; ++i) fa[h][t][i] = buf[((ra + h * H + i) * 2 + t) * 64];
    };
    auto read_b = [&](int s, int t) {
      const uint4* const buf = smem + (s % RING) * WORDS + lane;
#pragma unroll
      for (int j = 0; j < 4; ++j) fb[t][j] = buf[((rb + j) * 2 + t) * 64];
    };
    // loads n0 .. n1 of slab s among the products: one waits its turn behind those of the other waves, and the matrix cores
    // are not to wait with it
    auto multiply = [&](int h, int ta, int tb, int s, int n0, int n1) {
      constexpr int PRODUCTS = 4 * H;
#pragma unroll
      for (int n = 0; n < PRODUCTS; ++n) {
        const int i = n / 4, j = n % 4;
        acc[h * H + i][j] = mfma_f16(fa[h][ta][i], fb[tb][j], acc[h * H + i][j]);
        if (n1 > n0 && n % (PRODUCTS / 2) == PRODUCTS / 2 - 1 && n0 + n / (PRODUCTS / 2) < n1) {
          __builtin_amdgcn_sched_barrier(0);
          stage(s, n0 + n / (PRODUCTS / 2));
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int s = 0; s < RING - 1; ++s)
#pragma unroll
      for (int n = 0; n < 8; ++n) stage(s, n);
    __builtin_amdgcn_s_waitcnt(WAIT);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_b(0, 0), read_a(0, 0);
    for (int s = 0; s < steps; ++s) {
      read_b(s, 1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(0, 0, 0, s + RING - 1, 0, 2);
      read_a(s, 1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(0, 1, 0, s + RING - 1, 2, 4);
      multiply(0, 0, 1, s + RING - 1, 4, 6);
      multiply(1, 0, 0, s + RING - 1, 6, 8);
      multiply(1, 1, 0, 0, 0, 0);
      __builtin_amdgcn_s_waitcnt(WAIT);  // this wave's share of the next slab has landed
      __builtin_amdgcn_s_barrier();      // everyone's has, and everyone has read this one
      asm volatile("" ::: "memory");
      read_b(s + 1, 0), read_a(s + 1, 0);
      __builtin_amdgcn_sched_barrier(0);
      multiply(1, 0, 1, 0, 0, 0);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): nothing more is on its way to LDS
    __syncthreads();
    float* const v64 = reinterpret_cast<float*>(smem) + wave * (64 * 64);
#pragma unroll
    for (int h = 0; h < TA / 4; ++h) {
      spread(acc, 4 * h, v64);
      wave_sync();
      part(v64, (ra / 4 + h) * 64, (wave / WM) * 64, 0, 8);
      wave_sync();
    }
  }
};

// A tile of 64 x 64, every eighth step a wave's; the waves' sums are added in order.  A wave's fragments come at the rate of the
// CU's cache, a step of all eight in a microsecond, so where a few tiles have long sums each is shared by several blocks, which
// leave theirs in memory to a kernel of their own (muon_join_kernel; the last block to arrive adding them by itself was slower
// than no sharing: its fences write all of an L2 back).
struct FewTile {
  static constexpr int WAVES = 8, THREADS = 512, BM = 64, BN = 64;
  static constexpr size_t LDS = WAVES * 64 * 64 * 4;

  // part(v64, 0, 0, f0, f1): the whole tile for every wave, fragments f0 .. f1 are its own
  template <typename F>
  __device__ static __forceinline__ void run(const Operand& a, const Operand& b, int steps, uint4* smem, F part) {
    sum<3>(a, b, 0, steps, smem);
    __syncthreads();
    const int wave = threadIdx.x >> 6;
    part(reinterpret_cast<float*>(smem), 0, 0, wave, wave + 1);
  }
  // Steps s0 .. s0 + steps by three term products or all four, as values in LDS; every thread writes places n * 512 + threadIdx.x (of four values), n < 2.
  template <int PRODUCTS>
  __device__ static __forceinline__ void sum(const Operand& a, const Operand& b, int s0, int steps, uint4* smem) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint4* src[8][2];  // [row tile of either operand][term]: wave-uniform
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int t = 0; t < 2; ++t) src[r][t] = (r < 4 ? a.frag(r, t) : b.frag(r - 4, t)) + (int64_t)(s0 + wave) * 64;
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    uint4 f[8][2], g[8][2];
    const int mine = wave < steps ? (steps - 1 - wave) / WAVES + 1 : 0;
    auto fetch = [&](int s, uint4 (&to)[8][2]) {  // (behind the last: that one again)
      const int64_t at = (int64_t)min(s, mine - 1) * (WAVES * 64);
#pragma unroll
      for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int t = 0; t < 2; ++t) to[r][t] = (src[r][t] + at)[lane];
    };
    auto products = [&](const uint4 (&x)[8][2]) {
#pragma unroll
      for (int p = 0; p < PRODUCTS; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = mfma_f16(x[i][p >> 1], x[4 + j][p & 1], acc[i][j]);
    };
    if (mine > 0) {
      fetch(0, f);
      int s = 0;
      for (; s + 1 < mine; s += 2) {
        fetch(s + 1, g);
        products(f);
        fetch(s + 2, f);
        products(g);
      }
      if (s < mine) products(f);
    }
    float* const all = reinterpret_cast<float*>(smem);
    spread(acc, 0, all + wave * (64 * 64));
    __syncthreads();
    float4* const sums = reinterpret_cast<float4*>(all);  // (the waves' parts lie alike: places are added)
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      float4 v = sums[n * 512 + threadIdx.x];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) {
        const float4 u = sums[w * 1024 + n * 512 + threadIdx.x];
        v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
      }
      sums[n * 512 + threadIdx.x] = v;
    }
  }
};

// Consecutive blocks go to the eight XCDs in turn.  Each takes a contiguous eighth of a matrix' tiles, in patches eight tiles
// wide, so that what its blocks stream at one time is shared in its L2 (34 TB/s; a miss of it is served at 10).
__device__ __forceinline__ int xcd_item(int block, int total) {
  const int per = total / 8;
  return block < per * 8 ? (block % 8) * per + block / 8 : block;
}
// Tile `item` of rows x cols ones.
__device__ __forceinline__ void tile_of(int item, int rows, int cols, int* it, int* jt) {
  const int band = item / (8 * cols), in = item - band * 8 * cols, wide = min(8, rows - band * 8);
  *jt = in / wide, *it = band * 8 + in % wide;
}
// Tile `item` of those on and above the diagonal (it <= jt) of n x n: bands of eight columns, row by row.
__device__ __forceinline__ void triangle_of(int item, int n, int* it, int* jt) {
  int band = 0, wide = min(8, n);
  for (int in_band; item >= (in_band = wide * band + wide * (wide + 1) / 2);) {
    item -= in_band;
    band += 8, wide = min(8, n - band);
  }
  if (item < wide * band) {
    *it = item / wide, *jt = band + item % wide;
    return;
  }
  item -= wide * band;
  int j = 0;
  while (item > j) item -= ++j;  // column j of the band's own triangle has j + 1 tiles
  *it = band + item, *jt = band + j;
}

// d_i for the X that this step makes, from d_i^2 A_ii and 1 / d_i of this one.
__device__ __forceinline__ float next_power(float diagonal, float inverse) {
  return power_for(fminf(sqrtf(diagonal) * inverse * kGrowth, kMost), kRowTop);
}

// A 64 x 64 part of A (MUON_A: the values themselves) or B (MUON_B: b A + c times the values) at (i0, j0), and at (j0, i0) where
// that is another place: fragments f0 .. f1.  The values carry the powers of row and column; that of the contraction goes.
template <int WHAT>
__device__ __forceinline__ void put_symmetric(const MuonBatch& b, const MuonTensor& t, const float* v64, int i0, int j0, bool both, int f0, int f1) {
  if (max(i0, j0) >= t.small) return;
  uint4* const dst = WHAT == MUON_A ? mat_a(t) : mat_b(t);
  const int steps = t.mt * (kPad / 32), lane = threadIdx.x & 63;
  const float* const inverse = inv_d(t, b.turn);
  const auto polynomial = [&](float (&v)[8], int64_t word, const float* by) {
    times8(v, by);
    if (WHAT == MUON_A) return;
    float a8[8];
    join8(mat_a(t), a_term(t), word, a8);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(kC, v[e], kB * a8[e]);
  };
  if (WHAT == MUON_A && i0 == j0 && f0 == 0)
    inv_d(t, b.turn ^ 1)[i0 + lane] = inverse_power(next_power(v64[at64(lane, lane)], inverse[i0 + lane]));
#pragma unroll 2
  for (int f = f0; f < f1; ++f) {
    put_fragment<false>(v64, dst, a_term(t), word_of(i0, j0, steps), steps, f,
                        [&](float (&v)[8], int64_t word, int, int k) { polynomial(v, word, inverse + j0 + k); });
    if (both)
      put_fragment<true>(v64, dst, a_term(t), word_of(j0, i0, steps), steps, f,
                         [&](float (&v)[8], int64_t word, int, int k) { polynomial(v, word, inverse + i0 + k); });
  }
}

// MUON_A: A = X X^T.  MUON_B: B = b A + c A A^T.
template <typename TILE, int WHAT>
__global__ __launch_bounds__(TILE::THREADS, 2) void muon_square_kernel(MuonBatch b) {
  extern __shared__ uint4 smem16[];
  static_assert(TILE::BM == TILE::BN, "the tiles of a symmetric matrix");
  const int at_tensor = tensor_of(b);
  const MuonTensor& t = b.t[at_tensor];
  const int tiles = (t.small + TILE::BM - 1) / TILE::BM;
  int it, jt;
  triangle_of(xcd_item(blockIdx.x - b.first[at_tensor], tiles * (tiles + 1) / 2), tiles, &it, &jt);
  const int pitch = (WHAT == MUON_A ? t.nt : t.mt) * (kPad / 32), depth = WHAT == MUON_A ? t.large : t.small;
  Operand x{WHAT == MUON_A ? x_rows(t) : mat_a(t), WHAT == MUON_A ? x_term(t) : a_term(t), it * (TILE::BM / 16), t.mt * (kPad / 16), pitch};
  Operand y = x;
  y.row_tile = jt * (TILE::BM / 16);
  TILE::run(x, y, (depth + 31) / 32, smem16, [&](const float* v64, int i1, int j1, int f0, int f1) {
    put_symmetric<WHAT>(b, t, v64, it * TILE::BM + i1, jt * TILE::BN + j1, it != jt, f0, f1);
  });
}

// A = X X^T where t.parts blocks share a tile's steps: their sums ...
__global__ __launch_bounds__(FewTile::THREADS, 2) void muon_share_kernel(MuonBatch b) {
  extern __shared__ uint4 smem16[];
  const int at_tensor = tensor_of(b);
  const MuonTensor& t = b.t[at_tensor];
  const int block = blockIdx.x - b.first[at_tensor], part = block % t.parts, tiles = (t.small + 63) / 64;
  int it, jt;
  triangle_of(block / t.parts, tiles, &it, &jt);
  Operand x{x_rows(t), x_term(t), it * 4, t.mt * (kPad / 16), t.nt * (kPad / 32)};
  Operand y = x;
  y.row_tile = jt * 4;
  const int steps = (t.large + 31) / 32;
  const int s0 = (int)((int64_t)steps * part / t.parts), s1 = (int)((int64_t)steps * (part + 1) / t.parts);
  FewTile::sum<4>(x, y, s0, s1 - s0, smem16);  // (the fragments' way here takes longer than the products)
#pragma unroll
  for (int n = 0; n < 2; ++n)
    reinterpret_cast<float4*>(b.shares)[blockIdx.x * 1024 + n * 512 + threadIdx.x] = reinterpret_cast<const float4*>(smem16)[n * 512 + threadIdx.x];
}
// ... and their join, a block a tile, in the order of the blocks.
__global__ __launch_bounds__(FewTile::THREADS) void muon_join_kernel(MuonBatch b) {
  __shared__ __attribute__((aligned(16))) float v64[64 * 64];
  int tile = blockIdx.x, at_tensor = 0, n = 0;
  for (;; ++at_tensor, tile -= n) {
    n = (b.first[at_tensor + 1] - b.first[at_tensor]) / b.t[at_tensor].parts;
    if (tile < n) break;
  }
  const MuonTensor& t = b.t[at_tensor];
  const float4* const from = reinterpret_cast<const float4*>(b.shares) + (int64_t)(b.first[at_tensor] + tile * t.parts) * 1024 + threadIdx.x;
  float4 v[2] = {from[0], from[512]};
#pragma unroll 4
  for (int p = 1; p < t.parts; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 u = from[p * 1024 + h * 512];
      v[h].x += u.x, v[h].y += u.y, v[h].z += u.z, v[h].w += u.w;
    }
#pragma unroll
  for (int h = 0; h < 2; ++h) reinterpret_cast<float4*>(v64)[h * 512 + threadIdx.x] = v[h];
  __syncthreads();
  int it, jt;
  triangle_of(tile, (t.small + 63) / 64, &it, &jt);
  const int wave = threadIdx.x >> 6;
  put_symmetric<MUON_A>(b, t, v64, it * 64, jt * 64, it != jt, wave, wave + 1);
}

// X' of a 64 x 64 part at (i0, j0) to where the next step finds it; after the last one: the result, or the weights moved by it.
// Fragments f0 .. f1 are this wave's.  COLS: X is read by columns too.  d, e: the powers that X' has in the part's row, and column,
// `lane`.
template <bool LAST, bool COLS = true>
__device__ __forceinline__ void put_next(const MuonBatch& b, const MuonTensor& t, const float* v64, int i0, int j0, int f0, int f1,
                                         float d, float e) {
  const int lane = threadIdx.x & 63;
  const int steps_n = t.nt * (kPad / 32), steps_m = t.mt * (kPad / 32);
  if constexpr (!LAST) {
    uint32_t largest = 0;  // of column `lane`, in the rows of the wave's fragments
#pragma unroll 2
    for (int f = f0; f < f1; ++f) {
      put_fragment<false>(v64, x_rows(t), x_term(t), word_of(i0, j0, steps_n), steps_n, f,
                          [&](float (&v)[8], int64_t, int row, int) { times8(v, __shfl(d, row)); });
      if (COLS)
        put_fragment<true>(v64, x_cols(t, b.turn ^ 1), x_term(t), word_of(j0, i0, steps_m), steps_m, f,
                           [&](float (&v)[8], int64_t, int col, int) {  // sixteen columns, four lanes each
                             uint32_t most = 0;
#pragma unroll
                             for (int n = 0; n < 8; ++n) most = max(most, magnitude(v[n]));
                             most = max(most, (uint32_t)__shfl_xor((int)most, 16));
                             most = max(most, (uint32_t)__shfl_xor((int)most, 32));
                             if (lane >> 4 == f >> 1) largest = max(largest, most);
                             times8(v, __shfl(e, col));
                           });
    }
    if (COLS) {
      if (lane >> 4 >= f0 >> 1 && lane >> 4 <= (f1 - 1) >> 1)
        atomicMax(col_most(t, (b.third + 1) % 3) + j0 + lane, largest);
      if (i0 == 0 && f0 == 0) inv_e(t, b.turn ^ 1)[j0 + lane] = inverse_power(e), col_most(t, (b.third + 2) % 3)[j0 + lane] = 0;
    }
  } else {
    const float step = b.lr * t.factor;
    const int64_t at0 = t.tall ? (int64_t)j0 * t.small + i0 : (int64_t)i0 * t.large + j0;
    const int pitch = t.tall ? t.small : t.large;
    const int rows_left = t.tall ? t.large - j0 : t.small - i0, cols_left = t.tall ? t.small - i0 : t.large - j0;
    if (lane >= cols_left) return;
#pragma unroll 1
    for (int r0 = f0 * 8; r0 < min(f1 * 8, rows_left); r0 += 8) {  // rows of the matrix as stored
      float w[8];
      if (!t.out) {
#pragma unroll
        for (int r = 0; r < 8; ++r) w[r] = r0 + r < rows_left ? t.w[at0 + (int64_t)(r0 + r) * pitch + lane] : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        if (r0 + r >= rows_left) break;
        const int64_t at = at0 + (int64_t)(r0 + r) * pitch + lane;
        const float o = v64[t.tall ? at64(lane, r0 + r) : at64(r0 + r, lane)];
        if (t.out) {
          t.out[at] = o;
        } else {
          const float v = fmaf(-step, o, b.keep * w[r]);
          t.w[at] = v;
          if (t.w16) st(reinterpret_cast<bf16*>(t.w16) + at, v);
        }
      }
    }
  }
}

// X <- a X + B X of such a part, given d_i e_j B X.  Waves that share a part all come here.
template <bool LAST>
__device__ __forceinline__ void put_applied(const MuonBatch& b, const MuonTensor& t, float* v64, int i0, int j0, int f0, int f1) {
  const int lane = threadIdx.x & 63;
  const bool inside = i0 < t.small && j0 < t.large;  // (the same for all waves that share a part)
  float d = 0.f, e = 0.f;
  if (inside) {
    if (!LAST) {
      d = inverse_power(inv_d(t, b.turn ^ 1)[i0 + lane]);
      const float bound = __uint_as_float(col_most(t, b.third)[j0 + lane]) * (kGrowth * sqrtf((float)t.small));
      e = power_for(fminf(bound, kMost), kColTop);
    }
    float4* const x = x_floats(t, i0, j0);
    const float *const by_row = inv_d(t, b.turn) + i0, *const by_col = inv_e(t, b.turn) + j0;
#pragma unroll 4
    for (int n = f0 * 2; n < f1 * 2; ++n) {
      const int p = n * 64 + lane;
      const float row = by_row[row_at(p)];
      const float4 col = *reinterpret_cast<const float4*>(by_col + col_at(p)), v = x[p];
      float4* const at = reinterpret_cast<float4*>(v64) + p;
      float4 u = *at;
      u.x = fmaf(kA, v.x, u.x * row * col.x), u.y = fmaf(kA, v.y, u.y * row * col.y);
      u.z = fmaf(kA, v.z, u.z * row * col.z), u.w = fmaf(kA, v.w, u.w * row * col.w);
      *at = u;
      if (!LAST) x[p] = u;
    }
  }
  if (f1 - f0 < 8) __syncthreads();  // (a part of several waves)
  else wave_sync();
  if (inside) put_next<LAST>(b, t, v64, i0, j0, f0, f1, d, e);
}

template <typename TILE, bool LAST>
__global__ __launch_bounds__(TILE::THREADS, 2) void muon_apply_kernel(MuonBatch b) {
  extern __shared__ uint4 smem16[];
  const int at_tensor = tensor_of(b);
  const MuonTensor& t = b.t[at_tensor];
  const int tiles_m = (t.small + TILE::BM - 1) / TILE::BM, tiles_n = (t.large + TILE::BN - 1) / TILE::BN;
  int it, jt;
  tile_of(xcd_item(blockIdx.x - b.first[at_tensor], tiles_m * tiles_n), tiles_m, tiles_n, &it, &jt);
  const Operand x{mat_b(t), a_term(t), it * (TILE::BM / 16), t.mt * (kPad / 16), t.mt * (kPad / 32)};
  const Operand y{x_cols(t, b.turn), x_term(t), jt * (TILE::BN / 16), t.nt * (kPad / 16), t.mt * (kPad / 32)};
  TILE::run(x, y, (t.small + 31) / 32, smem16, [&](float* v64, int i1, int j1, int f0, int f1) {
    put_applied<LAST>(b, t, v64, it * TILE::BM + i1, jt * TILE::BN + j1, f0, f1);
  });
}

// Matrices of at most 64 rows (as X): a block adds the shares of A by itself, makes B of it and then its 64 columns of X, in place
// of three launches with a few blocks each.  The products are small (a wave makes two 16 x 16 tiles of either) and their sums
// short, so that float products would round little: these are float products, of X kept in floats beside the terms that the
// shares are made of.  (With term products here the error was up to twice that of float products, 64 x 800 in 68 us, not 76: a
// float product has an eighth of the rate, and a block waits 1 us for each.)
template <bool LAST>
__global__ __launch_bounds__(512) void muon_small_kernel(MuonBatch b) {
  __shared__ __attribute__((aligned(16))) float v64[64 * 64], x64[64 * 64];
  const int at_tensor = tensor_of(b);
  const MuonTensor& t = b.t[at_tensor];
  const int j0 = (blockIdx.x - b.first[at_tensor]) * 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rt = (wave >> 1) * 16, ct = (wave & 1) * 32, in = lane & 15, k4 = lane >> 4;  // rows, columns of the wave's tiles
  float4* const kept = x_floats(t, 0, j0) + threadIdx.x;
  const float* const inverse = inv_d(t, b.turn);
  const float4* const from = reinterpret_cast<const float4*>(b.shares) + (int64_t)t.share0 * 1024 + threadIdx.x;
  const float4 x[2] = {kept[0], kept[512]};
  float4 v[2] = {from[0], from[512]};
#pragma unroll 4
  for (int p = 1; p < t.parts; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 u = from[p * 1024 + h * 512];
      v[h].x += u.x, v[h].y += u.y, v[h].z += u.z, v[h].w += u.w;
    }
#pragma unroll
  for (int h = 0; h < 2; ++h) {  // d_i A_ij
    const int p = h * 512 + threadIdx.x;
    const float4 by = *reinterpret_cast<const float4*>(inverse + col_at(p));
    reinterpret_cast<float4*>(v64)[p] = make_float4(v[h].x * by.x, v[h].y * by.y, v[h].z * by.z, v[h].w * by.w);
    reinterpret_cast<float4*>(x64)[p] = x[h];
  }
  __syncthreads();
  const float diagonal = v64[at64(lane, lane)], by = inverse[lane];
  // v_mfma_f32_16x16x4_f32: lane l holds row l % 16 of one operand, column l % 16 of the other, contraction l / 16
  const auto product = [&](auto column, f32x4 (&acc)[2]) {  // two halves of the sum at once
    f32x4 part[2][2] = {};
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = h * 32 + n * 4 + k4;
        const float row = v64[at64(rt + in, k)];
#pragma unroll
        for (int c = 0; c < 2; ++c)
          part[h][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(row, column(k, ct + c * 16 + in), part[h][c], 0, 0, 0);
      }
#pragma unroll
    for (int c = 0; c < 2; ++c) acc[c] = part[0][c] + part[1][c];
  };
  f32x4 acc[2];
  product([&](int k, int j) { return v64[at64(j, k)]; }, acc);  // d_i d_j A^2
  __syncthreads();
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const float by_col = inverse[ct + c * 16 + in];
#pragma unroll
    for (int q = 0; q < 4; ++q) {  // d_i B in A's place: every value is one lane's own
      float* const at = v64 + at64(rt + 4 * k4 + q, ct + c * 16 + in);
      *at = fmaf(kC, acc[c][q] * by_col, kB * *at);
    }
  }
  __syncthreads();
  product([&](int k, int j) { return x64[at64(k, j)]; }, acc);
  __syncthreads();
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = at64(rt + 4 * k4 + q, ct + c * 16 + in);
      v64[at] = fmaf(kA, x64[at], acc[c][q] * inverse[rt + 4 * k4 + q]);
    }
  __syncthreads();
  if (!LAST) {
#pragma unroll
    for (int h = 0; h < 2; ++h) kept[h * 512] = reinterpret_cast<const float4*>(v64)[h * 512 + threadIdx.x];
  }
  const float d = next_power(diagonal * inverse_power(by), by);
  if (!LAST && j0 == 0 && wave == 0) inv_d(t, b.turn ^ 1)[lane] = inverse_power(d);
  put_next<LAST, false>(b, t, v64, 0, j0, wave, wave + 1, d, 0.f);
}

// ---- launches -----------------------------------------------------------------------------------------------------------
static void lay_out(MuonTensor* t) {
  t->tall = t->rows > t->cols;
  t->small = std::min(t->rows, t->cols), t->large = std::max(t->rows, t->cols);
  t->mt = (int)ceil_div(t->small, kPad), t->nt = (int)ceil_div(t->large, kPad);
  t->pm = (int)ceil_div(t->small, 64), t->pn = (int)ceil_div(t->large, 64);
  // groups of parts that a block of muon_moment_kernel takes: a block of muon_begin_kernel reads what all of a row, and all of a
  // column, have seen
  t->gm = std::min(t->pm, 32), t->gn = std::min(t->pn, std::max(32, 256 / t->gm));
}

// At the start of the workspace: the shares.
static constexpr size_t kJoinBytes = (size_t)kJoinBlocks * 64 * 64 * sizeof(float);

size_t muon_workspace(int tensors, const int32_t* rows, const int32_t* cols) {
  if (tensors == 0) return 0;
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
  return (size_t)most * 16 + kJoinBytes;
}

template <typename K, typename N>
static vcnn_status launch_phase(const char* what, K kernel, MuonBatch* b, int threads, size_t lds, hipStream_t st, N blocks_of) {
  // the matrices whose blocks take longest first: their larger side stands for both
  std::stable_sort(b->t, b->t + b->tensors, [](const MuonTensor& x, const MuonTensor& y) { return x.large > y.large; });
  int64_t blocks = 0;
  for (int t = 0; t < b->tensors; ++t) {
    b->first[t] = (unsigned)blocks;
    blocks += blocks_of(b->t[t]);
  }
  if (blocks > 0x7fffffffLL) return fail(VCNN_ERR_UNSUPPORTED, "%s: too many tiles", what);
  b->first[b->tensors] = (unsigned)blocks;
  if (lds) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), lds, st, *b);
  return check_launch(what);
}

// Tiles of a phase: of the whole X, or on and above the diagonal.
template <typename TILE>
static int64_t tiles_of(const MuonTensor& t, bool triangle) {
  const int64_t m = ceil_div(t.small, TILE::BM);
  return triangle ? m * (m + 1) / 2 : m * ceil_div(t.large, TILE::BN);
}
using TileDeep = SlabTile<4, 2, 2, 4>;  // 128 x 128, a tile a CU
using TileTwo = SlabTile<4, 2, 2, 2>;   // 128 x 128, two tiles a CU
using TileWide = SlabTile<8, 2, 4, 2>;  // 256 x 256

// The tile of a phase, by how many there are for 256 CUs; launch(tile) with its type.  Measured, us a phase (Few / Deep / Two
// / Wide): X X^T of 1024 x 4096 (36 tiles of 128) 28 / 69 / 96 / 215, of 2048 x 2048 (136) 50 / 45 / 56 / 118; B X of 1024 x 4096
// (256) 50 / 34 / 39 / 74, of 2048 x 4096 (512) 168 / 115 / 100 / 134, of 4096 x 4096 (1024) 536 / 397 / 361 / 329 (B X
// without what writing X in floats too has added since, 2 and some 15 us at the first and the last of these sizes).
template <typename F>
static vcnn_status with_tile(const MuonBatch& b, bool triangle, F launch) {
  int64_t few = 0, two = 0, wide = 0;
  for (int t = 0; t < b.tensors; ++t) {
    few += tiles_of<FewTile>(b.t[t], triangle);
    two += tiles_of<TileTwo>(b.t[t], triangle);
    wide += tiles_of<TileWide>(b.t[t], triangle);
  }
  if (few <= 512) return launch(FewTile());
  if (two <= 256) return launch(TileDeep());
  if (wide >= 256) return launch(TileWide());
  return launch(TileTwo());
}

// The shares of A = X X^T: blocks share its sums as far as there are idle CUs, `each` steps a block at least.
static vcnn_status launch_shares(MuonBatch* b, int64_t tiles, int each, int most, hipStream_t st) {
  for (int t = 0; t < b->tensors; ++t)
    b->t[t].parts = (int)std::max<int64_t>(1, std::min<int64_t>({kJoinBlocks / tiles, most, ceil_div(b->t[t].large, 32) / each}));
  if (vcnn_status s = launch_phase("muon share", muon_share_kernel, b, FewTile::THREADS, FewTile::LDS, st,
                                   [](const MuonTensor& t) { return tiles_of<FewTile>(t, true) * t.parts; }))
    return s;
  for (int t = 0; t < b->tensors; ++t) b->t[t].share0 = (int)b->first[t];
  return VCNN_OK;
}

template <int WHAT>
static vcnn_status launch_square(MuonBatch* b, hipStream_t st) {
  if constexpr (WHAT == MUON_A) {  // its sums are long where A is small
    int64_t few = 0, longest = 0;
    for (int t = 0; t < b->tensors; ++t) {
      few += tiles_of<FewTile>(b->t[t], true);
      longest = std::max(longest, ceil_div(b->t[t].large, 32));
    }
    if (few * 2 <= kJoinBlocks && longest >= kSharedSteps) {
      if (vcnn_status s = launch_shares(b, few, 16, kJoinBlocks, st)) return s;
      hipLaunchKernelGGL(muon_join_kernel, dim3((unsigned)few), dim3(FewTile::THREADS), 0, st, *b);
      return check_launch("muon join");
    }
  }
  return with_tile(*b, true, [&](auto tile) {
    using TILE = decltype(tile);
    return launch_phase("muon square", muon_square_kernel<TILE, WHAT>, b, TILE::THREADS, TILE::LDS, st,
                        [](const MuonTensor& t) { return tiles_of<TILE>(t, true); });
  });
}
template <bool LAST>
static vcnn_status launch_apply(MuonBatch* b, hipStream_t st) {
  return with_tile(*b, false, [&](auto tile) {
    using TILE = decltype(tile);
    return launch_phase("muon apply", muon_apply_kernel<TILE, LAST>, b, TILE::THREADS, TILE::LDS, st,
                        [](const MuonTensor& t) { return tiles_of<TILE>(t, false); });
  });
}

vcnn_status launch_muon(const MuonTensor* tensors, int count, float lr, float momentum, int nesterov, float weight_decay,
                        int steps, void* workspace, hipStream_t st) {
  MuonBatch b{};
  b.tensors = count;
  b.lr = lr, b.momentum = momentum, b.nesterov = nesterov, b.keep = 1.f - lr * weight_decay;
  b.shares = (float*)workspace;
  uint4* work = (uint4*)((char*)workspace + kJoinBytes);
  for (int t = 0; t < b.tensors; ++t) {
    b.t[t] = tensors[t];
    lay_out(&b.t[t]);
    b.t[t].work = work;
    work += work_words(b.t[t]);
  }
  b.small = 1;  // a step is two launches then (64 x 800: five steps 76 us, with three launches each 107)
  for (int t = 0; t < b.tensors; ++t) b.small = b.small && b.t[t].small <= 64;
  const auto groups = [](const MuonTensor& t) { return t.gm * t.gn; };
  const auto parts = [](const MuonTensor& t) { return (int64_t)t.pm * t.pn; };
  if (vcnn_status s = launch_phase("muon moment", muon_moment_kernel, &b, kThreads, 0, st, groups)) return s;
  if (vcnn_status s = launch_phase("muon begin", muon_begin_kernel, &b, kThreads, 0, st, parts)) return s;
  for (int i = 0; i < steps; ++i, b.turn ^= 1, b.third = (b.third + 1) % 3) {
    if (b.small) {
      const auto columns = [](const MuonTensor& t) { return ceil_div(t.large, 64); };
      if (vcnn_status s = launch_shares(&b, b.tensors, 8, 16, st)) return s;
      if (vcnn_status s = i + 1 < steps ? launch_phase("muon small", muon_small_kernel<false>, &b, 512, 0, st, columns)
                                        : launch_phase("muon small", muon_small_kernel<true>, &b, 512, 0, st, columns))
        return s;
      continue;
    }
    if (vcnn_status s = launch_square<MUON_A>(&b, st)) return s;
    if (vcnn_status s = launch_square<MUON_B>(&b, st)) return s;
    if (vcnn_status s = i + 1 < steps ? launch_apply<false>(&b, st) : launch_apply<true>(&b, st)) return s;
  }
  return VCNN_OK;
}

}  // namespace vcnn

// Root-mean-square norm of the rows of a matrix, with the residual's addition before it, in training and with an 8-bit
// output, and the quantisation of rows alone:
//     h = x + r (rounded to the storage type),   s = 1 / sqrt(mean(h^2) + eps),   y = h s g
//     q = round(127 u / a),  u = h g (or x),  a = max |u|,  scale = a s / 127 (or a / 127)
// s cancels in q, so q depends on the products u and their largest magnitude alone: no error of the sum reaches it.
//     dh = dh_above + s (t - h s^2 mean(t h)),  t = dy g;    dg = sum over rows of dy h s
//
// All of it is bandwidth: a row is read once, kept in registers over the reduction (NV groups of 16 bytes a thread), and
// written.  A row of at most 128 groups belongs to one wave (no barrier; four rows a block), a longer one to a block of as
// many waves as its groups fill (at most eight), one of more than 16384 elements is read twice.  Rows start wherever the row
// length puts them: a group is loaded as a 16-byte type of alignment one, which the target serves at full width, and only
// the last group of a row whose length is no multiple of it goes by elements.  bfloat16, with the residual: 8192 x 5120 to 8
// bits 61 us (4.8 TB/s; a large copy 5.1), 4096 x 4096 forward 22 and backward 26 us (read from the last-level cache in part).
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "elem.h"

namespace vcnn {

static constexpr int kWaveThreads = 256;  // of a block with a row per wave
static constexpr int kMaxWaves = 16;
static constexpr int kKeptThreads = 512;  // most of a row that is kept in registers (32 elements a thread)

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct __attribute__((packed, aligned(1))) Loose16 { uint32_t w[4]; };
struct __attribute__((packed, aligned(1))) Loose8 { uint32_t w[2]; };
struct __attribute__((packed, aligned(1))) Loose4 { uint32_t w; };

// A group of 16 bytes of one row.
template <typename T>
struct Group {
  static constexpr int N = 16 / sizeof(T);
};
__device__ __forceinline__ void unpack(const Loose16& p, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(p.w[i]);
}
__device__ __forceinline__ void unpack(const Loose16& p, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(p.w[i] << 16), v[2 * i + 1] = __uint_as_float(p.w[i] & 0xffff0000u);
}
__device__ __forceinline__ Loose16 pack(const float (&v)[4]) {
  Loose16 p;
#pragma unroll
  for (int i = 0; i < 4; ++i) p.w[i] = __float_as_uint(v[i]);
  return p;
}
__device__ __forceinline__ Loose16 pack(const float (&v)[8]) {  // nearest even
  Loose16 p;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    p.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){v[2 * i], v[2 * i + 1]}, bf16x2));
  return p;
}

// Elements c .. c + N of a row of `cols` (zeros behind its end).
template <typename T>
__device__ __forceinline__ Loose16 load_group(const T* row, int c, int cols) {
  constexpr int N = Group<T>::N;
  if (c + N <= cols) return *reinterpret_cast<const Loose16*>(row + c);
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = c + i < cols ? ld(row + c + i) : 0.f;
  return pack(v);
}
template <typename T>
__device__ __forceinline__ void store_group(T* row, int c, int cols, const Loose16& p) {
  constexpr int N = Group<T>::N;
  if (c + N <= cols) {
    *reinterpret_cast<Loose16*>(row + c) = p;
    return;
  }
  float v[N];
  unpack(p, v);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c + i < cols) st(row + c + i, v[i]);
}
template <int N>
__device__ __forceinline__ void load_gain(const float* gain, int c, int cols, float (&g)[N]) {
  if (c + N <= cols) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const Loose16 p = *reinterpret_cast<const Loose16*>(gain + c + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) g[i + j] = __uint_as_float(p.w[j]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = c + i < cols ? gain[c + i] : 0.f;
  }
}
// N integers of at most 127 (still as floats) to bytes.
__device__ __forceinline__ uint32_t pack_bytes(float a, float b, float c, float d) {
  return ((uint32_t)(int)a & 255u) | ((uint32_t)(int)b & 255u) << 8 | ((uint32_t)(int)c & 255u) << 16 | (uint32_t)(int)d << 24;
}
template <int N>
__device__ __forceinline__ void store_bytes(int8_t* row, int c, int cols, const float (&v)[N]) {
  if (c + N <= cols) {
    if constexpr (N == 8) {
      Loose8 p;
      p.w[0] = pack_bytes(v[0], v[1], v[2], v[3]), p.w[1] = pack_bytes(v[4], v[5], v[6], v[7]);
      *reinterpret_cast<Loose8*>(row + c) = p;
    } else {
      Loose4 p;
      p.w = pack_bytes(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<Loose4*>(row + c) = p;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c + i < cols) row[c + i] = (int8_t)(int)v[i];
}

// ---- reductions over a row's threads -----------------------------------------------------------------------------------
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
struct RowSums {  // one slot per wave; rows of even and odd turns take turns, so that a row needs one barrier
  float sum[2][kMaxWaves];
  uint32_t most[2][kMaxWaves];
  double wide[2][kMaxWaves], again[kMaxWaves];
  __device__ __forceinline__ float* of(float, int turn) { return sum[turn]; }
  __device__ __forceinline__ double* of(double, int turn) { return wide[turn]; }
};
// Sum (and largest magnitude's bits) over the row's threads, in every thread.
template <bool WAVE, typename S>
__device__ __forceinline__ void row_reduce(RowSums& s, int turn, S& sum, uint32_t& most) {
  sum = wave_sum(sum), most = wave_max(most);
  if constexpr (!WAVE) {
    S* const sums = s.of(sum, turn);
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) sums[wave] = sum, s.most[turn][wave] = most;
    __syncthreads();
    sum = 0, most = 0;
    for (int w = 0; w < waves; ++w) sum += sums[w], most = max(most, s.most[turn][w]);
  }
}
template <bool WAVE>
__device__ __forceinline__ double row_reduce(RowSums& s, double sum) {
  sum = wave_sum(sum);
  if constexpr (!WAVE) {
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.again[wave] = sum;
    __syncthreads();
    sum = 0.;
    for (int w = 0; w < waves; ++w) sum += s.again[w];
  }
  return sum;
}
// What a thread adds its share of a row in.  Kept rows: at most 32 elements, in float.  Rows read twice: any number, and the
// roundings of equal elements do not cancel, so the groups of one load, each added in float, are added in double (a row of
// 3.2 million elements of 1.1 came out 1e-5 off in float; forward takes 1 to 4 % longer, 4096 x 20000 of bfloat16 85.3 us, not
// 84.0, backward the same).
template <int NV>
using RowSum = std::conditional_t<(NV > 0), float, double>;

// round(127 u / a), ties to even, for |u| <= a, a > 0: the quotient in float is off by at most 127 * 2^-23 = 1.5e-5, so only
// a quotient within 1e-4 of the middle between two integers (one in 5000) needs the one rounded once in double, which is
// never moved across the middle: 127 u has 31 bits, and so the quotient is either the middle or 2^-32 of itself away.
__device__ __forceinline__ float to_i8(float u, float a, float inverse) {
  const float t = u * inverse;
  float q = rintf(t);
  if (!(fabsf(t - q) < 0.4999f)) q = (float)rint((double)u * 127.0 / (double)a);  // (and where inverse overflows: tiny a)
  return q;
}

enum { NORM_PLAIN = 0, NORM_I8 = 1, QUANT_I8 = 2 };

// Waves a SIMD of the kernel that keeps nv groups of `group` elements a thread: its registers (the elements, their gain, and
// two tensors' groups of the next row) are held to it, and no more blocks are launched than that makes resident, for a block
// that comes later has nothing on its way yet.
constexpr int waves_for(int nv, int group) {
  const int registers = nv * (2 * group + 8);
  return registers <= 24 ? 6 : registers <= 48 ? 4 : registers <= 72 ? 3 : 2;
}

struct NormArgs {
  const void* x;
  const void* residual;  // null: none
  const float* gain;
  void* h;               // x + residual (written with a residual only)
  void* y;               // NORM_PLAIN: elements of x's type; else int8
  float* stat;           // NORM_PLAIN: rstd (nullable); else scale
  int rows, cols;
  float eps;
};

template <typename T, int MODE, int NV, bool WAVE>
__global__ __launch_bounds__(WAVE ? kWaveThreads : NV ? kKeptThreads : 1024, NV ? waves_for(NV, 16 / (int)sizeof(T)) : 4) void norm_kernel(NormArgs a) {
  constexpr int N = Group<T>::N;
  __shared__ RowSums sums;
  const int per_row = WAVE ? 64 : blockDim.x, tid = WAVE ? threadIdx.x & 63 : threadIdx.x;
  const int rows_at_once = WAVE ? kWaveThreads / 64 : 1;
  const int cols = a.cols;
  float gain[NV ? NV : 1][N];
  if constexpr (NV > 0 && MODE != QUANT_I8) {
#pragma unroll
    for (int k = 0; k < NV; ++k) load_gain(a.gain, (k * per_row + tid) * N, cols, gain[k]);
  }
  const bool added = MODE != QUANT_I8 && a.residual;
  const int64_t stride = (int64_t)gridDim.x * rows_at_once;
  int64_t row = (int64_t)blockIdx.x * rows_at_once + (WAVE ? threadIdx.x >> 6 : 0);
  // a row's groups are on their way while the row before is reduced and written
  Loose16 px[NV ? NV : 1], pr[NV ? NV : 1];
  auto fetch = [&](int64_t at) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * per_row + tid) * N;
      if (c >= cols) continue;
      px[k] = load_group(reinterpret_cast<const T*>(a.x) + at * cols, c, cols);
      if (added) pr[k] = load_group(reinterpret_cast<const T*>(a.residual) + at * cols, c, cols);
    }
  };
  if (NV > 0 && row < a.rows) fetch(row);
  int turn = 0;
  for (; row < a.rows; row += stride, turn ^= 1) {
    const T* const x = reinterpret_cast<const T*>(a.x) + row * cols;
    T* const h = reinterpret_cast<T*>(a.h) + row * cols;
    // the group at c, the residual added and the sum stored
    auto take = [&](int c, const Loose16& gx, const Loose16& gr, float (&v)[N]) {
      unpack(gx, v);
      if (!added) return;
      float w[N];
      unpack(gr, w);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += w[i];
      const Loose16 ph = pack(v);
      unpack(ph, v);
      store_group(h, c, cols, ph);
    };
    RowSum<NV> sum = 0;
    uint32_t most = 0;
    auto count = [&](const float (&v)[N], const float (&g)[N]) {
      float part = NV > 0 ? (float)sum : 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (MODE != QUANT_I8) part = fmaf(v[i], v[i], part);
        if (MODE == NORM_I8) most = max(most, __float_as_uint(v[i] * g[i]) & 0x7fffffffu);
        if (MODE == QUANT_I8) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
      }
      sum = NV > 0 ? part : sum + part;
    };
    float v[NV ? NV : 1][N];
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * per_row + tid) * N;
        if (c < cols) {
          take(c, px[k], pr[k], v[k]);
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) v[k][i] = 0.f;
        }
      }
      if (row + stride < a.rows) fetch(row + stride);
#pragma unroll
      for (int k = 0; k < NV; ++k) count(v[k], gain[k]);
    } else {
      for (int c = tid * N; c < cols; c += per_row * N) {
        px[0] = load_group(x, c, cols);
        if (added) pr[0] = load_group(reinterpret_cast<const T*>(a.residual) + row * cols, c, cols);
        take(c, px[0], pr[0], v[0]);
        if (MODE == NORM_I8) load_gain(a.gain, c, cols, gain[0]);
        count(v[0], gain[0]);
      }
    }
    row_reduce<WAVE>(sums, turn, sum, most);
    const T* const kept = added ? h : x;  // (rows read twice: every thread meets its own elements again)
    float rstd = 1.f;
    if (MODE != QUANT_I8) {
      const float total = (float)sum, mean = total / (float)cols + a.eps;
      rstd = 1.f / sqrtf(mean);
      // squares beyond the float range (or not finite), or so small that their roundings, up to 2^-150 each, are seen in the
      // mean (only with an eps as small): once more in double
      if (!(total < __builtin_inff()) || mean < 0x1p-120f) {
        double wide = 0.;
        if constexpr (NV > 0) {
#pragma unroll
          for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) wide += (double)v[k][i] * v[k][i];
        } else {
          for (int c = tid * N; c < cols; c += per_row * N) {
            unpack(load_group(kept, c, cols), v[0]);
#pragma unroll
            for (int i = 0; i < N; ++i) wide += (double)v[0][i] * v[0][i];
          }
        }
        rstd = (float)(1.0 / sqrt(row_reduce<WAVE>(sums, wide) / cols + (double)a.eps));
      }
    }
    float most_f = __uint_as_float(most), scale = 0.f;
    const float inverse = 127.f / most_f;
    bool fine = true;
    if (MODE != NORM_PLAIN) {
      scale = MODE == NORM_I8 ? most_f * rstd / 127.f : most_f / 127.f;
      fine = most < 0x7f800000u && !isnan(rstd);
      if (!fine) scale = __builtin_nanf("");
    }
    if (a.stat && tid == 0) a.stat[row] = MODE == NORM_PLAIN ? rstd : scale;
    auto give = [&](int c, const float (&u)[N], const float (&g)[N]) {
      float o[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (MODE == NORM_PLAIN) o[i] = u[i] * rstd * g[i];
        else o[i] = fine && most != 0 ? to_i8(MODE == NORM_I8 ? u[i] * g[i] : u[i], most_f, inverse) : 0.f;
      }
      if constexpr (MODE == NORM_PLAIN) store_group(reinterpret_cast<T*>(a.y) + row * cols, c, cols, pack(o));
      else store_bytes(reinterpret_cast<int8_t*>(a.y) + row * cols, c, cols, o);
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * per_row + tid) * N;
        if (c < cols) give(c, v[k], gain[k]);
      }
    } else {
      for (int c = tid * N; c < cols; c += per_row * N) {
        unpack(load_group(kept, c, cols), v[0]);
        if (MODE != QUANT_I8) load_gain(a.gain, c, cols, gain[0]);
        give(c, v[0], gain[0]);
      }
    }
  }
}

// Threads and blocks of a row kernel: threads == 64 stands for a row per wave.
struct RowShape {
  int nv;       // groups a thread keeps; 0: rows are read twice
  int threads;  // of a row
  int blocks;
};
// quarters: rows by four waves where that will do, since blocks of four fill a CU evenly (8192 x 5120: blocks of five 79 us, of
// four 64); all eight where rows are few and a row's own time counts.
static RowShape row_shape(int64_t rows, int cols, int group, bool quarters) {
  const int64_t groups = ceil_div(cols, group);
  RowShape s;
  if (groups <= 128) s.nv = groups <= 64 ? 1 : 2, s.threads = 64;
  else if (cols > 32 * kKeptThreads) s.nv = 0, s.threads = 1024;
  else {
    const int most = quarters && rows > 512 && groups <= 4 * 256 ? 256 : kKeptThreads;
    s.nv = (int)ceil_div(groups, most);
    if (s.nv > 4) s.nv = s.nv <= 6 ? 6 : 8;
    s.threads = most == 256 ? 256 : (int)ceil_div(ceil_div(groups, s.nv), 64) * 64;
  }
  const int64_t blocks = s.threads == 64 ? ceil_div(rows, kWaveThreads / 64) : rows;
  const int waves = s.threads == 64 ? kWaveThreads / 64 : s.threads / 64;
  const int resident = s.nv ? std::max(2, 4 * waves_for(s.nv, group) / waves) : 2;
  s.blocks = (int)std::min<int64_t>(blocks, 256 * resident);
  return s;
}

// launch(nv, wave): the two as types
template <typename T, typename F>
static void with_shape(const RowShape& s, F launch) {
  using std::integral_constant;
  if (s.threads == 64) {
    if (s.nv == 1) launch(integral_constant<int, 1>(), std::true_type());
    else launch(integral_constant<int, 2>(), std::true_type());
  } else if (s.nv == 0) launch(integral_constant<int, 0>(), std::false_type());
  else if (s.nv == 1) launch(integral_constant<int, 1>(), std::false_type());
  else if (s.nv == 2) launch(integral_constant<int, 2>(), std::false_type());
  else if (s.nv == 3) launch(integral_constant<int, 3>(), std::false_type());
  else if (s.nv == 4) launch(integral_constant<int, 4>(), std::false_type());
  else if constexpr (Group<T>::N == 4) {  // (32 elements a thread at most)
    if (s.nv == 6) launch(integral_constant<int, 6>(), std::false_type());
    else launch(integral_constant<int, 8>(), std::false_type());
  }
}

template <typename T, int MODE>
static void launch_norm_typed(const NormArgs& a, hipStream_t st) {
  const RowShape s = row_shape(a.rows, a.cols, Group<T>::N, true);
  with_shape<T>(s, [&](auto nv, auto wave) {
    hipLaunchKernelGGL((norm_kernel<T, MODE, decltype(nv)::value, decltype(wave)::value>), dim3(s.blocks),
                       dim3(s.threads == 64 ? kWaveThreads : s.threads), 0, st, a);
  });
}

vcnn_status launch_rmsnorm(int dtype, int rows, int cols, float eps, const void* x, const void* residual, const float* gain,
                           void* h, void* y, float* rstd, hipStream_t st) {
  const NormArgs a{x, residual, gain, h, y, rstd, rows, cols, eps};
  if (dtype == VCNN_BF16) launch_norm_typed<bf16, NORM_PLAIN>(a, st);
  else launch_norm_typed<float, NORM_PLAIN>(a, st);
  return check_launch("rmsnorm");
}
vcnn_status launch_rmsnorm_i8(int dtype, int rows, int cols, float eps, const void* x, const void* residual,
                              const float* gain, void* h, int8_t* q, float* scale, hipStream_t st) {
  const NormArgs a{x, residual, gain, h, q, scale, rows, cols, eps};
  if (dtype == VCNN_BF16) launch_norm_typed<bf16, NORM_I8>(a, st);
  else launch_norm_typed<float, NORM_I8>(a, st);
  return check_launch("rmsnorm_i8");
}
vcnn_status launch_quant_rows_i8(int dtype, int rows, int cols, const void* x, int8_t* q, float* scale, hipStream_t st) {
  const NormArgs a{x, nullptr, nullptr, nullptr, q, scale, rows, cols, 0.f};
  if (dtype == VCNN_BF16) launch_norm_typed<bf16, QUANT_I8>(a, st);
  else launch_norm_typed<float, QUANT_I8>(a, st);
  return check_launch("quant_rows_i8");
}

// ---- backward ------------------------------------------------------------------------------------------------------------
// A block takes every gridDim-th row (or four) and adds their share of dg in registers; the blocks' shares are added in
// ascending order by a second kernel, so that dg has the same bits in every run.
struct NormBwdArgs {
  const void* h;
  const float* gain;
  const float* rstd;
  const void* dy;
  const void* above;  // gradient that reaches h beside the norm (nullable)
  void* dh;           // nullable
  float* partial;     // [blocks][cols] (nullable: no dg)
  int rows, cols;
};

static constexpr int kNormBwdBlocks = 512;

template <typename T, int NV, bool WAVE>
__global__ __launch_bounds__(WAVE ? kWaveThreads : NV ? kKeptThreads : 1024) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int N = Group<T>::N, K = NV ? NV : 1;
  __shared__ RowSums sums;
  __shared__ float shares[WAVE ? 3 * 64 * K * N : 1];
  const int per_row = WAVE ? 64 : blockDim.x, tid = WAVE ? threadIdx.x & 63 : threadIdx.x;
  const int rows_at_once = WAVE ? kWaveThreads / 64 : 1, wave = threadIdx.x >> 6;
  const int cols = a.cols;
  float* const partial = a.partial ? a.partial + (int64_t)blockIdx.x * cols : nullptr;
  float gain[K][N], dg[K][N];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (NV > 0) load_gain(a.gain, (k * per_row + tid) * N, cols, gain[k]);
#pragma unroll
    for (int i = 0; i < N; ++i) dg[k][i] = 0.f;
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * rows_at_once + (WAVE ? wave : 0); row < a.rows;
       row += (int64_t)gridDim.x * rows_at_once, turn ^= 1) {
    const T* const h = reinterpret_cast<const T*>(a.h) + row * cols;
    const T* const dy = reinterpret_cast<const T*>(a.dy) + row * cols;
    const T* const above = a.above ? reinterpret_cast<const T*>(a.above) + row * cols : nullptr;
    T* const dh = reinterpret_cast<T*>(a.dh) + row * cols;
    const float rstd = a.rstd[row];
    Loose16 ph[K], pd[K], pa[K];
    RowSum<NV> dot = 0;
    // t z, z = h s: of the magnitude of dy, so that the sum stays in range wherever h is
    auto meet = [&](const Loose16& gh, const Loose16& gd, const float (&g)[N], float (&z)[N], float (&d)[N]) {
      unpack(gh, z), unpack(gd, d);
      float part = NV > 0 ? (float)dot : 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] *= rstd, part = fmaf(d[i] * g[i], z[i], part);
      dot = NV > 0 ? part : dot + part;
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * per_row + tid) * N;
        if (c < cols) {
          ph[k] = load_group(h, c, cols), pd[k] = load_group(dy, c, cols);
          if (above) pa[k] = load_group(above, c, cols);
        } else {
          ph[k] = pd[k] = Loose16{{0, 0, 0, 0}};
        }
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float z[N], d[N];
        meet(ph[k], pd[k], gain[k], z, d);
#pragma unroll
        for (int i = 0; i < N; ++i) dg[k][i] = fmaf(d[i], z[i], dg[k][i]);
      }
    } else {
      for (int c = tid * N; c < cols; c += per_row * N) {
        float z[N], d[N];
        load_gain(a.gain, c, cols, gain[0]);
        meet(load_group(h, c, cols), load_group(dy, c, cols), gain[0], z, d);
        if (partial) {  // (this thread's own elements, turn after turn)
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (c + i < cols) partial[c + i] = (row == blockIdx.x ? 0.f : partial[c + i]) + d[i] * z[i];
        }
      }
    }
    uint32_t none = 0;
    row_reduce<WAVE>(sums, turn, dot, none);
    if (!a.dh) continue;
    const float mean = (float)dot / (float)cols;
    auto give = [&](int c, const Loose16& gh, const Loose16& gd, const Loose16& ga, const float (&g)[N]) {
      float hv[N], d[N], o[N];
      unpack(gh, hv), unpack(gd, d);
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = rstd * (d[i] * g[i] - hv[i] * rstd * mean);
      if (above) {
        float w[N];
        unpack(ga, w);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] += w[i];
      }
      store_group(dh, c, cols, pack(o));
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * per_row + tid) * N;
        if (c < cols) give(c, ph[k], pd[k], pa[k], gain[k]);
      }
    } else {
      for (int c = tid * N; c < cols; c += per_row * N) {
        if (above) pa[0] = load_group(above, c, cols);
        load_gain(a.gain, c, cols, gain[0]);
        give(c, load_group(h, c, cols), load_group(dy, c, cols), pa[0], gain[0]);
      }
    }
  }
  if constexpr (NV > 0) {
    if (!partial) return;
    if constexpr (WAVE) {  // the four waves' shares, in order
      if (wave > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int i = 0; i < N; ++i) shares[((wave - 1) * NV * N + k * N + i) * 64 + tid] = dg[k][i];
      }
      __syncthreads();
      if (wave > 0) return;
#pragma unroll
      for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int i = 0; i < N; ++i) dg[k][i] += shares[(w * NV * N + k * N + i) * 64 + tid];
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * per_row + tid) * N;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (c + i < cols) partial[c + i] = dg[k][i];
    }
  }
}

// dg[c] = the blocks' shares: 64 threads a column take every 64th, and their sums are added in pairs, always the same ones.
__global__ __launch_bounds__(1024) void gain_grad_kernel(const float* partial, float* dg, int blocks, int cols) {
  __shared__ float sums[64][17];
  const int in = threadIdx.x & 15, col = (blockIdx.y * gridDim.x + blockIdx.x) * 16 + in, part = threadIdx.x >> 4;
  float s = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int b = part; b < blocks; b += 64) s += partial[(int64_t)b * cols + col];
  }
  sums[part][in] = s;
  for (int n = 32; n > 0; n >>= 1) {
    __syncthreads();
    if (part < n) sums[part][in] += sums[part + n][in];
  }
  if (part == 0 && col < cols) dg[col] = sums[0][in];
}

size_t rmsnorm_bwd_partial_bytes(int rows, int cols) {
  return (size_t)std::min(rows, kNormBwdBlocks) * cols * sizeof(float);
}

template <typename T>
static int launch_norm_bwd_typed(const NormBwdArgs& a, hipStream_t st) {
  RowShape s = row_shape(a.rows, a.cols, Group<T>::N, false);
  s.blocks = std::min(s.blocks, kNormBwdBlocks);
  with_shape<T>(s, [&](auto nv, auto wave) {
    hipLaunchKernelGGL((norm_bwd_kernel<T, decltype(nv)::value, decltype(wave)::value>), dim3(s.blocks),
                       dim3(s.threads == 64 ? kWaveThreads : s.threads), 0, st, a);
  });
  return s.blocks;
}

vcnn_status launch_rmsnorm_bwd(int dtype, int rows, int cols, const void* h, const float* gain, const float* rstd,
                               const void* dy, const void* above, void* dh, float* dgain, float* partial, hipStream_t st) {
  const NormBwdArgs a{h, gain, rstd, dy, above, dh, dgain ? partial : nullptr, rows, cols};
  const int blocks = dtype == VCNN_BF16 ? launch_norm_bwd_typed<bf16>(a, st) : launch_norm_bwd_typed<float>(a, st);
  if (vcnn_status s = check_launch("rmsnorm_bwd")) return s;
  if (!dgain) return VCNN_OK;
  const unsigned groups = (unsigned)ceil_div(cols, 16), wide = std::min(groups, 1u << 16);  // (2^32 threads are no grid's width)
  hipLaunchKernelGGL(gain_grad_kernel, dim3(wide, (unsigned)ceil_div(groups, wide)), dim3(1024), 0, st, partial, dgain, blocks, cols);
  return check_launch("rmsnorm_bwd gain");
}

}  // namespace vcnn

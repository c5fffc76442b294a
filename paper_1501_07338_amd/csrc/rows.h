// What the kernels over the rows of a matrix share: groups of 16 bytes of a row, sums over a wave, and how a row is divided over
// threads and rows over blocks.
#pragma once
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

// What a thread adds its share of a row in.  Kept rows: at most 32 elements, in float.  Rows read twice: any number, and the
// roundings of equal elements do not cancel, so the groups of one load, each added in float, are added in double (a row of
// 3.2 million elements of 1.1 came out 1e-5 off in float; forward takes 1 to 4 % longer, 4096 x 20000 of bfloat16 85.3 us, not
// 84.0, backward the same).
template <int NV>
using RowSum = std::conditional_t<(NV > 0), float, double>;

// Waves a SIMD of the kernel that keeps nv groups of `group` elements a thread: its registers (the elements, their gain, and
// two tensors' groups of the next row) are held to it, and no more blocks are launched than that makes resident, for a block
// that comes later has nothing on its way yet.
constexpr int waves_for(int nv, int group) {
  const int registers = nv * (2 * group + 8);
  return registers <= 24 ? 6 : registers <= 48 ? 4 : registers <= 72 ? 3 : 2;
}

// Threads and blocks of a row kernel: threads == 64 stands for a row per wave.
struct RowShape {
  int nv;       // groups a thread keeps; 0: rows are read twice
  int threads;  // of a row
  int blocks;
};
// quarters: rows by four waves where that will do, since blocks of four fill a CU evenly (8192 x 5120: blocks of five 79 us, of
// four 64); all eight where rows are few and a row's own time counts.
// waves_of: waves_for, or its like of a kernel that keeps more.
static RowShape row_shape(int64_t rows, int cols, int group, bool quarters, int (*waves_of)(int, int) = waves_for) {
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
  const int resident = s.nv ? std::max(2, 4 * waves_of(s.nv, group) / waves) : 2;
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

}  // namespace vcnn

// The forward pass of a fully connected layer in 8-bit integers (v_mfma_i32_16x16x64_i8):
//     y[b][o] = act(bias[o] + xscale[b] wscale[o] sum_i xq[b][i] wq[o][i])
// The sums are whole numbers, exact in 32 bits up to 131071 terms of at most 2^14, so neither the order of a sum nor its
// division over waves and blocks changes a bit of the result.  A sum is rounded to float (2^-24) in the epilogue, multiplied
// by the two scales and rounded once more to the type of y.
//
// Three kernels.  One or two samples: dot products of whole rows (i8_dot_kernel; 4096 -> 16384 in 11.9 us with the call's own,
// the next kernel 15.1).  Up to 32, or 128 where the layer is small: the weights are read once and nothing of them is reused,
// so a block owns 16 outputs, its eight waves take every eighth 128 bytes of the rows and feed the matrix cores from global
// memory, all operands of four such steps in flight at once with up to 16 samples, of two with more (i8_rows_kernel; 48 samples
// 4096 -> 4096 in 11.2 us, two rounds of loads).  More: tiles of 256 x 256 or 128 x 128 from slabs of 64 bytes of both operands in LDS (i8_tile_kernel), the
// contraction divided over blocks where the tiles alone do not fill the chip; their shares are added by i8_join_kernel.
// 4096 x 8192 -> 8192 takes 246 us, 2.23 POP/s: 53 % of what the instruction reaches with operands in registers (4.2, bound by
// power).
#include <algorithm>

#include "common.h"
#include "elem.h"
#include "bf16_core.h"

namespace vcnn {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct __attribute__((packed, aligned(1))) Loose16i { uint32_t w[4]; };

struct I8Args {
  const int8_t* x;      // [batch][k]
  const int8_t* w;      // [out][k]
  const float* xscale;
  const float* wscale;
  const float* bias;    // nullable
  void* y;              // [batch][out]
  int32_t* partial;     // given: [splits][batch][out] sums instead of y
  int batch, k, out, act;
  int tiles_b, tiles_o, slabs_per_split;
};

__device__ __forceinline__ uint4 load16_whole(const int8_t* p) {
  const Loose16i v = *reinterpret_cast<const Loose16i*>(p);
  return make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
}
// 16 bytes of a row of k from byte c on, zeros behind its end: nothing is read there, but the row's last 16 bytes, shifted.
__device__ __forceinline__ uint4 load16(const int8_t* row, int c, int k) {
  if (c + 16 <= k) return load16_whole(row + c);
  uint64_t lo = 0, hi = 0;
  if (c < k) {
    if (k >= 16) {
      const uint4 v = load16_whole(row + k - 16);
      lo = v.x | (uint64_t)v.y << 32, hi = v.z | (uint64_t)v.w << 32;
      const int n = 8 * (c + 16 - k);  // 8 .. 120 bits
      if (n >= 64) lo = hi >> (n - 64), hi = 0;
      else lo = lo >> n | hi << (64 - n), hi >>= n;
    } else {
#pragma unroll 1
      for (int i = k - 1; i >= c; --i) hi = hi << 8 | lo >> 56, lo = lo << 8 | (uint8_t)row[i];
    }
  }
  return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}
__device__ __forceinline__ i32x4 mfma_i8(uint4 a, uint4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// SMOOTH: act may be one of the smooth ones.
template <bool SMOOTH>
__device__ __forceinline__ float finish(int sum, float scale, float bias, int act) {
  const float v = fmaf((float)sum, scale, bias);
  if (act == VCNN_ACT_RELU) return v < 0.f ? 0.f : v;  // (a NaN, from a row that could not be quantised, stays one)
  if (SMOOTH && act == VCNN_ACT_TANH) return tanhf(v);
  if (SMOOTH && act == VCNN_ACT_SIGMOID) return 1.f / (1.f + expf(-v));
  return v;
}

// What four neighbouring outputs o .. o + 3 have in common for all samples.
struct Outputs {
  float scale[4], bias[4];
  bool whole;  // (rows of a multiple of four outputs: every group is aligned to its own size)
};
template <typename T>
__device__ __forceinline__ Outputs outputs_of(const I8Args& a, int o) {
  Outputs p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = min(o + i, a.out - 1);
    p.scale[i] = a.wscale[j], p.bias[i] = a.bias ? a.bias[j] : 0.f;
  }
  p.whole = a.out % 4 == 0 && (reinterpret_cast<uintptr_t>(a.y) & (4 * sizeof(T) - 1)) == 0;
  return p;
}
// The four of sample b.
template <typename T, bool SMOOTH = true>
__device__ __forceinline__ void put4(const I8Args& a, const Outputs& p, int b, float xscale, int o, const int (&sum)[4]) {
  T* const y = reinterpret_cast<T*>(a.y) + (int64_t)b * a.out + o;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = finish<SMOOTH>(sum[i], xscale * p.scale[i], p.bias[i], a.act);
  if (p.whole) {
    st4(y, make_float4(v[0], v[1], v[2], v[3]));
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (o + i < a.out) st(y + i, v[i]);
}

// ---- very few samples ---------------------------------------------------------------------------------------------------
// Nothing is reused but the samples, so there is no product for the matrix cores: a wave reads whole rows of weights, 1 KB a
// load, four rows and four such loads of each at once, against the same bytes of the samples held in registers.
__device__ __forceinline__ int dot16(uint4 a, uint4 b, int c) {
  c = __builtin_amdgcn_sdot4((int)a.x, (int)b.x, c, false);
  c = __builtin_amdgcn_sdot4((int)a.y, (int)b.y, c, false);
  c = __builtin_amdgcn_sdot4((int)a.z, (int)b.z, c, false);
  return __builtin_amdgcn_sdot4((int)a.w, (int)b.w, c, false);
}
template <int CTRL>
__device__ __forceinline__ int add_ror(int v) {  // v + v of the lane CTRL (row_ror: 1 .. 15) places on in each sixteen
  return v + __builtin_amdgcn_update_dpp(0, v, 0x120 + CTRL, 0xf, 0xf, false);
}

template <typename T, int NB>
__global__ __launch_bounds__(256) void i8_dot_kernel(I8Args a) {
  constexpr int ROWS = 4, AHEAD = 4;
  const int lane = threadIdx.x & 63;
  const int o0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * ROWS;
  if (o0 >= a.out) return;
  int sum[NB][ROWS];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sum[n][r] = 0;
  const int8_t* w[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) w[r] = a.w + (int64_t)min(o0 + r, a.out - 1) * a.k;
  int c = 0;
  for (; c + AHEAD * 1024 <= a.k; c += AHEAD * 1024) {
    uint4 fw[AHEAD][ROWS];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int r = 0; r < ROWS; ++r) fw[u][r] = load16_whole(w[r] + c + u * 1024 + lane * 16);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int8_t* const x = a.x + (int64_t)min(n, a.batch - 1) * a.k + c + lane * 16;
      uint4 fx[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) fx[u] = load16_whole(x + u * 1024);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) sum[n][r] = dot16(fw[u][r], fx[u], sum[n][r]);
    }
  }
  for (; c < a.k; c += 1024) {
    uint4 fw[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) fw[r] = load16(w[r], c + lane * 16, a.k);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const uint4 fx = load16(a.x + (int64_t)min(n, a.batch - 1) * a.k, c + lane * 16, a.k);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) sum[n][r] = dot16(fw[r], fx, sum[n][r]);
    }
  }
  int mine = 0;  // lane 4 n + r finishes output r of sample n
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      int v = add_ror<1>(add_ror<2>(add_ror<4>(add_ror<8>(sum[n][r]))));
      v += __shfl_xor(v, 16);
      v += __shfl_xor(v, 32);
      if (lane == n * ROWS + r) mine = v;
    }
  const int b = lane / ROWS, o = o0 + lane % ROWS;
  if (b >= NB || b >= a.batch || o >= a.out) return;
  st(reinterpret_cast<T*>(a.y) + (int64_t)b * a.out + o,
     finish<true>(mine, a.xscale[b] * a.wscale[o], a.bias ? a.bias[o] : 0.f, a.act));
}

// ---- few samples -------------------------------------------------------------------------------------------------------
// Lane l holds row l % 16 of either operand and, of the 128 bytes of a step, the 16 from 16 (l / 16) on and the 16 that are 64
// further: each load takes 64 neighbouring bytes of a row (with 32 neighbouring bytes a lane, in two loads that share every
// 64, 32 samples of 16 Mi weights took 9.2 us, not 9.0).  With one tile of samples four steps are on their way at once, with
// more two, for the registers of four leave a CU one block: 16 samples 4096 -> 4096 6.9 and 7.8 us (four, two).  Of 20 to 128
// samples, 88 layers of 500 to 8192 inputs and 500 to 10000 outputs, two steps are faster by 2 % in the mean: 48 samples 4000 ->
// 4096 10.7 us, not 12.7, 4096 -> 4096 11.2 either way.  They lose where a wave's steps are few and leave a remainder: 60 samples
// 3000 -> 5000 15.0 us, not 14.0, 2000 -> 10000 17.5, not 15.4; but 3000 -> 4096 10.7, not 13.2, so that no rule by the number of
// inputs separates the two.
static constexpr int kRowsThreads = 512;

template <typename T, int NB>
__global__ __launch_bounds__(kRowsThreads) void i8_rows_kernel(I8Args a) {
  constexpr int AHEAD = NB == 1 ? 4 : 2, WAVES = kRowsThreads / 64;
  __shared__ int share[WAVES - 1][NB][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int o0 = blockIdx.x * 16, row = lane & 15, at = (lane >> 4) * 16;
  const int8_t* const w = a.w + (int64_t)min(o0 + row, a.out - 1) * a.k;
  const int8_t* x[NB];
  i32x4 acc[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    x[n] = a.x + (int64_t)min(n * 16 + row, a.batch - 1) * a.k;
    acc[n] = (i32x4){0, 0, 0, 0};
  }
  const int whole = a.k / 128;
  int s = wave;
  for (; s + WAVES * (AHEAD - 1) < whole; s += WAVES * AHEAD) {
    uint4 fw[AHEAD][2], fx[AHEAD][NB][2];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int c = (s + WAVES * u) * 128 + at;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const Loose16i p = *reinterpret_cast<const Loose16i*>(w + c + 64 * i);
        fw[u][i] = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const Loose16i q = *reinterpret_cast<const Loose16i*>(x[n] + c + 64 * i);
          fx[u][n][i] = make_uint4(q.w[0], q.w[1], q.w[2], q.w[3]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[n] = mfma_i8(fw[u][i], fx[u][n][i], acc[n]);
  }
  for (; s * 128 < a.k; s += WAVES) {
    const int c = s * 128 + at;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 fw = load16(w, c + 64 * i, a.k);
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[n] = mfma_i8(fw, load16(x[n], c + 64 * i, a.k), acc[n]);
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) share[wave - 1][n][q][lane] = acc[n][q];
  }
  __syncthreads();
  if (wave > 0) return;
  const int o = o0 + 4 * (lane >> 4);  // register q: row 4 (l / 16) + q, column l % 16
  const Outputs out = outputs_of<T>(a, o);
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    int sum[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[q] = acc[n][q];
#pragma unroll
      for (int v = 0; v < WAVES - 1; ++v) sum[q] += share[v][n][q][lane];
    }
    const int b = n * 16 + (lane & 15);
    if (b < a.batch && o < a.out) put4<T>(a, out, b, a.xscale[b], o, sum);
  }
}

// ---- tiles -------------------------------------------------------------------------------------------------------------
// BO outputs x BB samples by waves of 16 TO x 16 TB, on the 16 x 16 x 64 form: with operands in registers it reaches 4.2 POP/s
// on this card, the 32 x 32 x 32 form 2.7.
template <int BO_, int BB_, int TO_, int TB_, int RING_, bool AHEAD_>
struct I8Tile {
  static constexpr int BO = BO_, BB = BB_, TO = TO_, TB = TB_;
  static constexpr int WO = BO / (16 * TO), THREADS = WO * (BB / (16 * TB)) * 64, WAVES = THREADS / 64;
  static constexpr int RING = RING_;                 // slabs in LDS
  static constexpr bool AHEAD = AHEAD_;              // a wave reads a whole step ahead (else half a one)
  static constexpr int WORDS = (BO + BB) * 4;        // 16-byte words of a slab of 64 bytes a row
  static constexpr size_t LDS = (size_t)RING * WORDS * 16;
  static constexpr int LO = BO * 4 / THREADS, LB = BB * 4 / THREADS;  // words a thread brings of one
  static_assert(TO % 2 == 0 && TB % 2 == 0 && LDS >= (size_t)WAVES * 32 * 4 * TO * 16, "the sums fit the slabs' memory");
};

// Places of a slab in LDS: word c of the four of row r at place c ^ swizzle(r).  Lane l reads word l / 16 of row l % 16, and
// the banks serve sixteen lanes of a 16-byte read at a time, four runs of four neighbours (0-3, 12-15, 20-23 and 24-27, the
// others of the first 32, the same of the last 32): these then meet 256 different bytes.
__device__ __forceinline__ int swizzle(int r) {
  const int h = r >> 2 & 3;
  return h >> 1 | ((h ^ h >> 1) & 1) << 1;  // 0 2 3 1
}

// Lane l of a 16 x 16 accumulator has sums 4 (l / 16) + q of column l % 16.  They go through LDS, 32 samples at a time and
// every wave for itself, so that a sample's neighbouring outputs are finished and stored by neighbouring lanes; word c of
// sample r at place c ^ (r % 8).
template <typename T, typename TILE>
__device__ __forceinline__ void i8_store(const I8Args& a, const i32x4 (&acc)[TILE::TO][TILE::TB], int o0, int b0, uint4* smem) {
  constexpr int WR = 4 * TILE::TO;  // words of four sums a sample
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ow = o0 + (wave % TILE::WO) * 16 * TILE::TO, bw = b0 + (wave / TILE::WO) * 16 * TILE::TB;
  constexpr int ROWS = 64 / WR, TURNS = 32 / ROWS;  // samples that the lanes store at once
  static_assert(64 % WR == 0, "a lane keeps its outputs");
  uint4* const mine = smem + wave * (32 * WR);
  const int c0 = lane % WR, r0 = lane / WR, o = ow + 4 * c0;
  const Outputs out = outputs_of<T>(a, o);
#pragma unroll
  for (int j = 0; j < TILE::TB; j += 2) {
    const int b0j = bw + j * 16;
    float xs[TURNS];  // (all on their way before the first is needed)
    if (!a.partial) {
#pragma unroll
      for (int n = 0; n < TURNS; ++n) xs[n] = a.xscale[min(b0j + n * ROWS + r0, a.batch - 1)];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < TILE::TO; ++i) {
        const int r = h * 16 + (lane & 15), c = i * 4 + (lane >> 4);
        mine[r * WR + (c ^ (r & 7))] = __builtin_bit_cast(uint4, acc[i][j + h]);
      }
    wave_sync();
    auto turn = [&](int n, float scale, bool smooth) {
      const int r = n * ROWS + r0, b = b0j + r;
      const uint4 v = mine[r * WR + (c0 ^ (r & 7))];
      if (b >= a.batch || o >= a.out) return;
      const int sum[4] = {(int)v.x, (int)v.y, (int)v.z, (int)v.w};
      if (a.partial) {
        int32_t* const p = a.partial + ((int64_t)blockIdx.y * a.batch + b) * a.out + o;
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (o + u < a.out) p[u] = sum[u];
      } else if (smooth) {
        put4<T, true>(a, out, b, scale, o, sum);
      } else {
        put4<T, false>(a, out, b, scale, o, sum);
      }
    };
    if (!a.partial && a.act >= VCNN_ACT_TANH) {  // (their code is long: not once a turn)
#pragma unroll 1
      for (int n = 0; n < TURNS; ++n) turn(n, a.xscale[min(b0j + n * ROWS + r0, a.batch - 1)], true);
    } else {
#pragma unroll
      for (int n = 0; n < TURNS; ++n) turn(n, xs[n], false);
    }
    wave_sync();
  }
}

// Consecutive blocks go to the eight XCDs in turn: each takes a contiguous eighth of the tiles, in patches of eight tiles of
// samples by as many of outputs as it comes to, so that the blocks at work share what they read in its L2.
__device__ __forceinline__ void tile_of(const I8Args& a, int* to, int* tb) {
  const int total = a.tiles_o * a.tiles_b, per = total / 8, block = blockIdx.x;
  const int item = block < per * 8 ? (block % 8) * per + block / 8 : block;
  const int group = item / (8 * a.tiles_o), in = item - group * 8 * a.tiles_o, wide = min(8, a.tiles_b - group * 8);
  *to = in / wide, *tb = group * 8 + in % wide;
}

__device__ const uint4 kZeros = {0, 0, 0, 0};

// Rows that start on 16 bytes.  Slabs of 64 bytes a row, one step of the instruction, go to a ring of four by direct loads,
// three slabs ahead; a wave reads the second half of a step's outputs while it multiplies the first, and the first of the
// next step while it multiplies the second, so that neither the loads nor the barrier (one a slab) leave the matrix cores
// without operands.
template <typename T, typename TILE>
__global__ __launch_bounds__(TILE::THREADS, 2) void i8_tile_kernel(I8Args a) {
  constexpr int TO = TILE::TO, TB = TILE::TB, LO = TILE::LO, LB = TILE::LB, L = LO + LB, THREADS = TILE::THREADS;
  extern __shared__ uint4 smem16[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int to, tb;
  tile_of(a, &to, &tb);
  const int o0 = to * TILE::BO, b0 = tb * TILE::BB;
  const int s0 = blockIdx.y * a.slabs_per_split, slabs = min((a.k + 63) / 64 - s0, a.slabs_per_split);
  const int8_t* const w0 = a.w + (int64_t)o0 * a.k + (int64_t)s0 * 64;  // rows behind the last read that one again
  const int8_t* const x0 = a.x + (int64_t)b0 * a.k + (int64_t)s0 * 64;
  const int place = ((tid & 3) ^ swizzle(tid >> 2)) * 16;  // of this thread's word within a row (THREADS / 4 rows on: the same)
  static_assert(THREADS % 128 == 0, "the swizzle repeats");
  uint32_t offset[L];  // (at most 256 rows of 131071 bytes)
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int r = (i < LO ? i : i - LO) * (THREADS / 4) + (tid >> 2);
    offset[i] = (uint32_t)(i < LO ? min(r, a.out - 1 - o0) : min(r, a.batch - 1 - b0)) * (uint32_t)a.k + place;
  }
  const int limit = min(a.k - s0 * 64, slabs * 64);  // bytes of a row that are this block's
  auto stage = [&](int s, int i) {                   // load i of L; behind the last slab: zeros
    uint4* const to = smem16 + (s % TILE::RING) * TILE::WORDS + i * THREADS + wave * 64;
    const int8_t* const from = (i < LO ? w0 : x0) + s * 64;
    if (s * 64 + 64 <= limit) load_to_lds16(from, offset[i], to);
    else load_to_lds16(s * 64 + place < limit ? reinterpret_cast<const uint4*>(from + offset[i]) : &kZeros, to);
  };
  i32x4 acc[TO][TB];
#pragma unroll
  for (int i = 0; i < TO; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
  const int wo = (wave % TILE::WO) * 16 * TO, wb = (wave / TILE::WO) * 16 * TB;
  const int mine = (lane & 15) * 4 + ((lane >> 4) ^ swizzle(lane & 15));  // this lane's word of a 16-row tile
  constexpr bool AHEAD = TILE::AHEAD;
  constexpr int H = AHEAD ? TO : TO / 2;  // row tiles of a set of fragments
  uint4 fo[2][H], fb[2][TB];
  auto read_o = [&](int s, int p, int first) {
    const uint4* const buf = smem16 + (s % TILE::RING) * TILE::WORDS + mine;
#pragma unroll
    for (int i = 0; i < H; ++i) fo[p][i] = buf[(wo + (first + i) * 16) * 4];
  };
  auto read_b = [&](int s, int p) {
    const uint4* const buf = smem16 + (s % TILE::RING) * TILE::WORDS + mine;
#pragma unroll
    for (int j = 0; j < TB; ++j) fb[p][j] = buf[(TILE::BO + wb + j * 16) * 4];
  };
  // The products of set po, loads l0 .. l1 of slab s among them: a load waits its turn behind those of the other waves, and the
  // matrix cores are not to wait with it.
  auto multiply = [&](int first, int po, int pb, int s, int l0, int l1) {
    const int every = H * TB / (l1 - l0);
#pragma unroll
    for (int n = 0; n < H * TB; ++n) {
      const int i = n / TB, j = n % TB;
      acc[first + i][j] = mfma_i8(fo[po][i], fb[pb][j], acc[first + i][j]);
      if (n % every == every / 2) {
        __builtin_amdgcn_sched_barrier(0);
        stage(s, l0 + n / every);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  constexpr int R = TILE::RING;
  static_assert((R - 2) * L < 64, "the counts fit");
  constexpr auto all_but = [](int n) { return 0x0F70 | (n & 15) | n >> 4 << 14; };  // vmcnt(n)
#pragma unroll
  for (int s = 0; s < R - 1; ++s)
#pragma unroll
    for (int i = 0; i < L; ++i) stage(s, i);
  __builtin_amdgcn_s_waitcnt(all_but((R - 2) * L));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_b(0, 0), read_o(0, 0, 0);
  auto step = [&](int s, int p) {
    // slab s + 1 is there, for everyone; slab s - 1 has been read by everyone
    __builtin_amdgcn_s_waitcnt(all_but((R - 3) * L));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if constexpr (AHEAD) {
      read_b(s + 1, p ^ 1), read_o(s + 1, p ^ 1, 0);
      __builtin_amdgcn_sched_barrier(0);
      multiply(0, p, p, s + R - 1, 0, L);
    } else {
      read_o(s, 1, H);
      __builtin_amdgcn_sched_barrier(0);
      multiply(0, 0, p, s + R - 1, 0, L / 2);
      __builtin_amdgcn_sched_barrier(0);
      read_b(s + 1, p ^ 1), read_o(s + 1, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      multiply(H, 1, p, s + R - 1, L / 2, L);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  for (int s = 0; s < slabs; s += 2) {
    step(s, 0);
    step(s + 1, 1);
  }
  __builtin_amdgcn_s_waitcnt(0x0070);  // nothing more is on its way to LDS, or from it
  __syncthreads();
  i8_store<T, TILE>(a, acc, o0, b0, smem16);
}

// Rows that start anywhere: a slab goes through registers, fetched HELD slabs before it is multiplied and put into one of two
// places in LDS while the one before is.
template <typename T, typename TILE>
__global__ __launch_bounds__(TILE::THREADS, 2) void i8_tile_loose_kernel(I8Args a) {
  constexpr int TO = TILE::TO, TB = TILE::TB, LO = TILE::LO, L = TILE::LO + TILE::LB, THREADS = TILE::THREADS;
  constexpr int HELD = L <= 2 ? 4 : 2;
  extern __shared__ uint4 smem16[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int to, tb;
  tile_of(a, &to, &tb);
  const int o0 = to * TILE::BO, b0 = tb * TILE::BB;
  const int s0 = blockIdx.y * a.slabs_per_split, s1 = min((a.k + 63) / 64, s0 + a.slabs_per_split);
  const int8_t* const w0 = a.w + (int64_t)o0 * a.k;
  const int8_t* const x0 = a.x + (int64_t)b0 * a.k;
  const int place = ((tid & 3) ^ swizzle(tid >> 2)) * 16;
  uint32_t offset[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int r = (i < LO ? i : i - LO) * (THREADS / 4) + (tid >> 2);
    offset[i] = (uint32_t)(i < LO ? min(r, a.out - 1 - o0) : min(r, a.batch - 1 - b0)) * (uint32_t)a.k;
  }
  uint4 held[HELD][L];
  auto fetch = [&](int s, uint4 (&to)[L]) {  // (zeros behind the last slab)
    if (s < s1 && (s + 1) * 64 <= a.k) {
#pragma unroll
      for (int i = 0; i < L; ++i) to[i] = load16_whole((i < LO ? w0 : x0) + (int64_t)s * 64 + offset[i] + place);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) to[i] = load16((i < LO ? w0 : x0) + offset[i], s < s1 ? s * 64 + place : a.k, a.k);
    }
  };
  auto put = [&](int s, const uint4 (&from)[L]) {
#pragma unroll
    for (int i = 0; i < L; ++i) smem16[(s & 1) * TILE::WORDS + i * THREADS + tid] = from[i];
  };
  i32x4 acc[TO][TB];
#pragma unroll
  for (int i = 0; i < TO; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
  const int wo = (wave % TILE::WO) * 16 * TO, wb = (wave / TILE::WO) * 16 * TB;
  const int mine = (lane & 15) * 4 + ((lane >> 4) ^ swizzle(lane & 15));
#pragma unroll
  for (int u = 0; u < HELD; ++u) fetch(s0 + u, held[u]);
  put(s0, held[0]);
  fetch(s0 + HELD, held[0]);
  for (int s = s0; s < s1; s += HELD) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {  // (slabs behind the last are zeros, so that every turn is the same)
      __syncthreads();                // slab s + u is there, the other place is free
      const uint4* const buf = smem16 + ((s + u) & 1) * TILE::WORDS + mine;
      uint4 fo[TO], fb[TB];
#pragma unroll
      for (int j = 0; j < TB; ++j) fb[j] = buf[(TILE::BO + wb + j * 16) * 4];
#pragma unroll
      for (int i = 0; i < TO; ++i) fo[i] = buf[(wo + i * 16) * 4];
      put(s + u + 1, held[(u + 1) % HELD]);
      fetch(s + u + 1 + HELD, held[(u + 1) % HELD]);
#pragma unroll
      for (int i = 0; i < TO; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = mfma_i8(fo[i], fb[j], acc[i][j]);
    }
  }
  __syncthreads();
  i8_store<T, TILE>(a, acc, o0, b0, smem16);
}

// The blocks' shares of four neighbouring outputs.
template <typename T>
__global__ __launch_bounds__(256) void i8_join_kernel(I8Args a, int splits) {
  const int groups = (a.out + 3) / 4;
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= (int64_t)groups * a.batch) return;
  const int b = (int)(n / groups), o = (int)(n % groups) * 4;
  int sum[4] = {0, 0, 0, 0};
  const int32_t* p = a.partial + (int64_t)b * a.out + o;
  for (int s = 0; s < splits; ++s, p += (int64_t)a.batch * a.out) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (o + u < a.out) sum[u] += p[u];
  }
  put4<T>(a, outputs_of<T>(a, o), b, a.xscale[b], o, sum);
}

// ---- the choice ----------------------------------------------------------------------------------------------------------
struct I8Plan {
  int few;             // 16-sample tiles of the kernel for few samples (0: tiles)
  int tile;            // 256 or 128
  int splits, slabs_per_split;
  size_t workspace_bytes;
};

static I8Plan i8_plan(int batch, int k, int out, size_t budget) {
  I8Plan p{};
  // Without tiles or with them, us: 64 samples of 16 Mi weights (4096 x 4096) 13 and 16, of 64 Mi 28 and 25; 65 samples of 1 Mi
  // 8 and 10, of 4 Mi 15 and 14.
  const int64_t weights = (int64_t)k * out;
  if (batch <= 32 || (batch <= 64 && weights <= 1 << 25) || (batch <= 128 && weights <= 1 << 20)) {
    p.few = batch <= 64 ? (int)ceil_div(batch, 16) : 8;
    return p;
  }
  const int slabs = (int)ceil_div(k, 64);
  p.tile = ceil_div(batch, 256) * ceil_div(out, 256) >= 192 ? 256 : 128;  // (1024 4096 -> 16384, 256 large tiles: 75 us either way)
  p.splits = 1, p.slabs_per_split = slabs;
  if (p.tile == 256) return p;
  // How many blocks share a sum: a slab takes a CU's one block 0.28 us and each further round of 256 blocks as long, the
  // join 4 us and the time of the shares, written and read at some 3.3 TB/s (within 10 % of what 65 to 512 samples took,
  // 1024 x 1024 to 8192 x 8192).
  const int64_t tiles = ceil_div(batch, 128) * ceil_div(out, 128);
  const double share = (double)batch * out * 4;
  double best = 0.28 * slabs * ceil_div(tiles, 256);
  for (int n = 2; n <= 16 && n * 4 <= slabs && n * share <= (double)budget; ++n) {
    const int each = (int)ceil_div(slabs, n), real = (int)ceil_div(slabs, each);
    const double us = 0.28 * each * ceil_div(tiles * real, 256) + 4 + real * share * 2 / 3.3e6;
    if (us < best) best = us, p.splits = real, p.slabs_per_split = each;
  }
  if (p.splits > 1) p.workspace_bytes = (size_t)p.splits * batch * out * 4;
  return p;
}

size_t fc_i8_workspace(int batch, int in_f, int out_f) { return i8_plan(batch, in_f, out_f, (size_t)1 << 30).workspace_bytes; }

template <typename T, typename TILE>
static void launch_tile(const I8Args& a, const I8Plan& p, hipStream_t st) {
  const bool aligned = a.k % 16 == 0 && ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15) == 0;
  const auto kernel = aligned ? i8_tile_kernel<T, TILE> : i8_tile_loose_kernel<T, TILE>;
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)TILE::LDS);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles_o * a.tiles_b), (unsigned)p.splits), dim3(TILE::THREADS), TILE::LDS, st, a);
}

template <typename T>
static vcnn_status launch_fc_i8_typed(I8Args a, void* workspace, size_t bytes, hipStream_t st) {
  const I8Plan p = i8_plan(a.batch, a.k, a.out, bytes);
  if (p.few) {
    const dim3 grid((unsigned)ceil_div(a.out, 16));
    if (a.batch == 1) hipLaunchKernelGGL((i8_dot_kernel<T, 1>), grid, dim3(256), 0, st, a);
    else if (a.batch == 2) hipLaunchKernelGGL((i8_dot_kernel<T, 2>), grid, dim3(256), 0, st, a);
    else if (p.few == 1) hipLaunchKernelGGL((i8_rows_kernel<T, 1>), grid, dim3(kRowsThreads), 0, st, a);
    else if (p.few == 2) hipLaunchKernelGGL((i8_rows_kernel<T, 2>), grid, dim3(kRowsThreads), 0, st, a);
    else if (p.few == 3) hipLaunchKernelGGL((i8_rows_kernel<T, 3>), grid, dim3(kRowsThreads), 0, st, a);
    else if (p.few == 4) hipLaunchKernelGGL((i8_rows_kernel<T, 4>), grid, dim3(kRowsThreads), 0, st, a);
    else hipLaunchKernelGGL((i8_rows_kernel<T, 8>), grid, dim3(kRowsThreads), 0, st, a);
    return check_launch("fc_fwd_i8");
  }
  a.tiles_b = (int)ceil_div(a.batch, p.tile), a.tiles_o = (int)ceil_div(a.out, p.tile);
  a.slabs_per_split = p.slabs_per_split;
  a.partial = p.splits > 1 ? (int32_t*)workspace : nullptr;
  if (p.tile == 256) launch_tile<T, I8Tile<256, 256, 8, 4, 4, false>>(a, p, st);
  else launch_tile<T, I8Tile<128, 128, 4, 2, 4, true>>(a, p, st);
  if (vcnn_status s = check_launch("fc_fwd_i8")) return s;
  if (p.splits == 1) return VCNN_OK;
  hipLaunchKernelGGL((i8_join_kernel<T>), dim3((unsigned)ceil_div(ceil_div(a.out, 4) * a.batch, 256)), dim3(256), 0, st, a,
                     p.splits);
  return check_launch("fc_fwd_i8 join");
}

vcnn_status launch_fc_i8(int dtype, int batch, int in_f, int out_f, int act, const int8_t* xq, const float* xscale,
                         const int8_t* wq, const float* wscale, const float* bias, void* y, void* workspace, size_t bytes,
                         hipStream_t st) {
  I8Args a{};
  a.x = xq, a.w = wq, a.xscale = xscale, a.wscale = wscale, a.bias = bias, a.y = y;
  a.batch = batch, a.k = in_f, a.out = out_f, a.act = act;
  return dtype == VCNN_BF16 ? launch_fc_i8_typed<bf16>(a, workspace, bytes, st)
                            : launch_fc_i8_typed<float>(a, workspace, bytes, st);
}

}  // namespace vcnn

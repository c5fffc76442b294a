// The forward pass of a fully connected layer in 8-bit integers (v_mfma_i32_*_i8, twice the rate of the 16-bit forms):
//     y[b][o] = act(bias[o] + xscale[b] wscale[o] sum_i xq[b][i] wq[o][i])
// The sums are whole numbers, exact in 32 bits up to 131071 terms of at most 2^14, so neither the order of a sum nor its
// division over waves and blocks changes a bit of the result.  A sum is rounded to float (2^-24) in the epilogue, multiplied
// by the two scales and rounded once more to the type of y.
//
// Two kernels.  Few samples (at most 64): the weights are read once and nothing of them is reused, so a block owns 16
// outputs, its four waves take every fourth 128 bytes of the rows and feed the matrix cores from global memory, all
// operands of four such steps in flight at once (i8_rows_kernel).  More: tiles of 256 x 256 or 128 x 128 from slabs of 128
// bytes of both operands in LDS (i8_tile_kernel), the contraction divided over blocks where the tiles alone do not fill the
// chip; their shares are added by i8_join_kernel.
#include <algorithm>

#include "common.h"
#include "elem.h"
#include "bf16_core.h"

namespace vcnn {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

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
// load_to_lds16 (bf16_core.h) from a wave-uniform address and a byte offset per lane.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds16(const int8_t* base, uint32_t offset, uint4* lds_base) {
  const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds_base);
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ i32x4 mfma_i8(uint4 a, uint4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x16 mfma_i8(uint4 a, uint4 b, i32x16 c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

__device__ __forceinline__ float finish(int sum, float scale, float bias, int act) {
  const float v = fmaf((float)sum, scale, bias);
  if (act == VCNN_ACT_RELU) return v < 0.f ? 0.f : v;  // (a NaN, from a row that could not be quantised, stays one)
  if (act == VCNN_ACT_TANH) return tanhf(v);
  if (act == VCNN_ACT_SIGMOID) return 1.f / (1.f + expf(-v));
  return v;
}

// Four neighbouring outputs o .. o + 3 of one sample.
template <typename T>
__device__ __forceinline__ void put4(const I8Args& a, int b, int o, const int (&sum)[4], bool whole) {
  const float xs = a.xscale[b];
  T* const y = reinterpret_cast<T*>(a.y) + (int64_t)b * a.out + o;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = min(o + i, a.out - 1);
    v[i] = finish(sum[i], xs * a.wscale[j], a.bias ? a.bias[j] : 0.f, a.act);
  }
  if (whole) {  // (rows of a multiple of four outputs: every group is aligned to its own size)
    st4(y, make_float4(v[0], v[1], v[2], v[3]));
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (o + i < a.out) st(y + i, v[i]);
}
template <typename T>
__device__ __forceinline__ bool whole_groups(const I8Args& a) {
  return a.out % 4 == 0 && (reinterpret_cast<uintptr_t>(a.y) & (4 * sizeof(T) - 1)) == 0;
}

// ---- few samples -------------------------------------------------------------------------------------------------------
// Lane l holds row l % 16 of either operand and, of the 128 bytes of a step, the 32 from 32 (l / 16) on as two
// instructions' words: a row's 128 bytes are read whole, and the order of a sum's terms is free.
template <typename T, int NB>
__global__ __launch_bounds__(256) void i8_rows_kernel(I8Args a) {
  constexpr int AHEAD = NB <= 2 ? 4 : 2;
  __shared__ int share[3][NB][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int o0 = blockIdx.x * 16, row = lane & 15, at = (lane >> 4) * 32;
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
  for (; s + 4 * (AHEAD - 1) < whole; s += 4 * AHEAD) {
    uint4 fw[AHEAD][2], fx[AHEAD][NB][2];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int c = (s + 4 * u) * 128 + at;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const Loose16i p = *reinterpret_cast<const Loose16i*>(w + c + 16 * i);
        fw[u][i] = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const Loose16i q = *reinterpret_cast<const Loose16i*>(x[n] + c + 16 * i);
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
  for (; s * 128 < a.k; s += 4) {
    const int c = s * 128 + at;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 fw = load16(w, c + 16 * i, a.k);
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[n] = mfma_i8(fw, load16(x[n], c + 16 * i, a.k), acc[n]);
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
  const bool whole4 = whole_groups<T>(a);
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    int sum[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[q] = acc[n][q];
#pragma unroll
      for (int v = 0; v < 3; ++v) sum[q] += share[v][n][q][lane];
    }
    const int b = n * 16 + (lane & 15), o = o0 + 4 * (lane >> 4);  // register q: row 4 (l / 16) + q, column l % 16
    if (b < a.batch && o < a.out) put4<T>(a, b, o, sum, whole4);
  }
}

// ---- tiles -------------------------------------------------------------------------------------------------------------
// A block owns BO outputs x BB samples, a wave 64 TO/2 ... (TO x TB accumulators of 32 x 32).  A slab is 128 bytes of every
// row of both operands, eight words of 16; word c of row r lies at place c ^ (r % 8), so that the eight rows that eight
// neighbouring lanes read at one time lie on different banks.
template <typename T, int BO, int BB, int TO, int TB, bool ALIGNED>
__global__ __launch_bounds__(BO / (32 * TO) * (BB / (32 * TB)) * 64) void i8_tile_kernel(I8Args a) {
  constexpr int THREADS = BO / (32 * TO) * (BB / (32 * TB)) * 64;
  constexpr int LO = BO * 8 / THREADS, LB = BB * 8 / THREADS;  // words of a slab a thread stages
  constexpr int WORDS = (BO + BB) * 8;
  extern __shared__ uint4 smem16[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tile = blockIdx.x, to = tile % a.tiles_o, tb = tile / a.tiles_o;
  const int o0 = to * BO, b0 = tb * BB;
  const int total = (a.k + 127) / 128;
  const int s0 = blockIdx.y * a.slabs_per_split, s1 = min(total, s0 + a.slabs_per_split);
  const int8_t* const w0 = a.w + (int64_t)o0 * a.k;  // first rows of the tile; rows behind the last read that one again
  const int8_t* const x0 = a.x + (int64_t)b0 * a.k;
  const int place = ((tid & 7) ^ (tid >> 3 & 7)) * 16;  // of this thread's word within a row of a slab
  uint32_t offset[LO + LB];                             // (at most 256 rows of 131071 bytes)
#pragma unroll
  for (int i = 0; i < LO + LB; ++i) {
    const int r = (i < LO ? i : i - LO) * (THREADS / 8) + (tid >> 3);
    offset[i] = (uint32_t)(i < LO ? min(r, a.out - 1 - o0) : min(r, a.batch - 1 - b0)) * (uint32_t)a.k + place;
  }
  uint4 held[ALIGNED ? 1 : LO + LB];
  // direct loads where rows start on 16 bytes, else through registers: fetched before a slab is multiplied, put behind it
  auto begin = [&](int s, uint4* buf) {
    if ((s + 1) * 128 > a.k) {  // ends inside
#pragma unroll 1
      for (int i = 0; i < LO + LB; ++i) {
        const int r = (i < LO ? i : i - LO) * (THREADS / 8) + (tid >> 3);
        const int8_t* const row = i < LO ? w0 + (int64_t)min(r, a.out - 1 - o0) * a.k : x0 + (int64_t)min(r, a.batch - 1 - b0) * a.k;
        buf[i * THREADS + tid] = load16(row, s * 128 + place, a.k);
      }
      return;
    }
    if constexpr (ALIGNED) {
#pragma unroll
      for (int i = 0; i < LO + LB; ++i)
        load_to_lds16((i < LO ? w0 : x0) + (int64_t)s * 128, offset[i], buf + i * THREADS + wave * 64);
    } else {
#pragma unroll
      for (int i = 0; i < LO + LB; ++i) held[i] = load16_whole((i < LO ? w0 : x0) + (int64_t)s * 128 + offset[i]);
    }
  };
  auto put = [&](int s, uint4* buf) {
    if constexpr (!ALIGNED)
      if ((s + 1) * 128 <= a.k) {
#pragma unroll
        for (int i = 0; i < LO + LB; ++i) buf[i * THREADS + tid] = held[i];
      }
  };
  const int wo = (wave % (BO / (32 * TO))) * 32 * TO, wb = (wave / (BO / (32 * TO))) * 32 * TB;
  i32x16 acc[TO][TB];
#pragma unroll
  for (int i = 0; i < TO; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;
  const int r32 = lane & 31, half = lane >> 5;
  begin(s0, smem16);
  put(s0, smem16);
  for (int s = s0; s < s1; ++s) {
    const uint4* const W = smem16 + ((s - s0) & 1) * WORDS;
    uint4* const next = smem16 + (((s - s0) & 1) ^ 1) * WORDS;
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's share of the slab has landed
    __syncthreads();                     // everyone's has, and the other buffer is free
    if (s + 1 < s1) begin(s + 1, next);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int c = 2 * t + half;
      uint4 fo[TO], fb[TB];
#pragma unroll
      for (int i = 0; i < TO; ++i) fo[i] = W[(wo + i * 32 + r32) * 8 + (c ^ (r32 & 7))];
#pragma unroll
      for (int j = 0; j < TB; ++j) fb[j] = W[BO * 8 + (wb + j * 32 + r32) * 8 + (c ^ (r32 & 7))];
#pragma unroll
      for (int i = 0; i < TO; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = mfma_i8(fo[i], fb[j], acc[i][j]);
    }
    if (s + 1 < s1) put(s + 1, next);
  }
  // The sums go through LDS, 32 samples at a time and every wave for itself, so that a sample's neighbouring outputs are
  // finished and stored by neighbouring lanes; word c of sample r at place c ^ (r % 8), as above.
  __syncthreads();
  const bool whole4 = whole_groups<T>(a);
  constexpr int WR = 8 * TO;  // words of four sums a sample
  uint4* const mine = smem16 + wave * (32 * WR);
#pragma unroll
  for (int j = 0; j < TB; ++j) {
#pragma unroll
    for (int i = 0; i < TO; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {  // register q: row 8 (q / 4) + 4 (l / 32) + q % 4, column l % 32
        const int c = i * 8 + 2 * g + half;
        mine[r32 * WR + (c ^ (r32 & 7))] = make_uint4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
      }
    // (a wave's LDS accesses keep their order)
#pragma unroll 2
    for (int n = lane; n < 32 * WR; n += 64) {
      const int r = n / WR, c = n % WR, b = b0 + wb + j * 32 + r, o = o0 + wo + 4 * c;
      const uint4 v = mine[r * WR + (c ^ (r & 7))];
      if (b >= a.batch || o >= a.out) continue;
      const int sum[4] = {(int)v.x, (int)v.y, (int)v.z, (int)v.w};
      if (a.partial) {
        int32_t* const p = a.partial + ((int64_t)blockIdx.y * a.batch + b) * a.out + o;
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (o + u < a.out) p[u] = sum[u];
      } else {
        put4<T>(a, b, o, sum, whole4);
      }
    }
  }
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
  put4<T>(a, b, o, sum, whole_groups<T>(a));
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
  if (batch <= 64) {
    p.few = (int)ceil_div(batch, 16);
    if (p.few == 3) p.few = 4;
    return p;
  }
  const int64_t big = ceil_div(batch, 256) * ceil_div(out, 256);
  p.tile = big >= 192 ? 256 : 128;
  const int64_t tiles = ceil_div(batch, p.tile) * ceil_div(out, p.tile);
  const int slabs = (int)ceil_div(k, 128);
  const int64_t room = p.tile == 256 ? 256 : 512;  // blocks resident at once
  int splits = 1;
  if (tiles * 2 <= room) splits = (int)std::min<int64_t>({room / tiles, slabs / 4, 16});
  splits = std::max(splits, 1);
  while (splits > 1 && (size_t)splits * batch * out * 4 > budget) --splits;
  p.slabs_per_split = (int)ceil_div(slabs, splits);
  p.splits = (int)ceil_div(slabs, p.slabs_per_split);
  if (p.splits > 1) p.workspace_bytes = (size_t)p.splits * batch * out * 4;
  return p;
}

size_t fc_i8_workspace(int batch, int in_f, int out_f) { return i8_plan(batch, in_f, out_f, (size_t)1 << 30).workspace_bytes; }

template <typename T, int BO, int BB, int TO, int TB, bool ALIGNED>
static void launch_tile(const I8Args& a, const I8Plan& p, hipStream_t st) {
  constexpr size_t lds = 2 * (BO + BB) * 128;
  const auto kernel = i8_tile_kernel<T, BO, BB, TO, TB, ALIGNED>;
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles_o * a.tiles_b), (unsigned)p.splits),
                     dim3(BO / (32 * TO) * (BB / (32 * TB)) * 64), lds, st, a);
}

template <typename T>
static vcnn_status launch_fc_i8_typed(I8Args a, void* workspace, size_t bytes, hipStream_t st) {
  const I8Plan p = i8_plan(a.batch, a.k, a.out, bytes);
  if (p.few) {
    const dim3 grid((unsigned)ceil_div(a.out, 16)), block(256);
    if (p.few == 1) hipLaunchKernelGGL((i8_rows_kernel<T, 1>), grid, block, 0, st, a);
    else if (p.few == 2) hipLaunchKernelGGL((i8_rows_kernel<T, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((i8_rows_kernel<T, 4>), grid, block, 0, st, a);
    return check_launch("fc_fwd_i8");
  }
  a.tiles_b = (int)ceil_div(a.batch, p.tile), a.tiles_o = (int)ceil_div(a.out, p.tile);
  a.slabs_per_split = p.slabs_per_split;
  a.partial = p.splits > 1 ? (int32_t*)workspace : nullptr;
  const bool aligned = a.k % 16 == 0 && ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15) == 0;
  if (p.tile == 256) {
    if (aligned) launch_tile<T, 256, 256, 4, 2, true>(a, p, st);
    else launch_tile<T, 256, 256, 4, 2, false>(a, p, st);
  } else {
    if (aligned) launch_tile<T, 128, 128, 2, 2, true>(a, p, st);
    else launch_tile<T, 128, 128, 2, 2, false>(a, p, st);
  }
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

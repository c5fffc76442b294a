// A matrix product of 16-bit operands with float sums on the matrix cores, for the products of a layer with many outputs:
//     out[b][a] = sum over k of  A(a, k) B(b, k)
// Each operand lies in memory as rows that run along k, or as rows of k that run along a (or b): the second kind is turned round
// on its way from LDS to the registers (ds_read_b64_tr_b16: sixteen lanes read four rows of sixteen elements, and each gets a
// column of four), so that no transposed copy is ever written.  An operand may come in planes, a high and a low term (or three)
// in turn for every 64 elements; the products high x high, low x high and high x low are then made of one slab into the same sums.
//
// What bounds it.  On operands of zeros a step of 256 x 256 x 32 takes 1820 clocks of which the matrix cores are busy 1031, without
// its loads 1440: a CU's loads to LDS wait for one another, 16 rows of 64 bytes each (rows of 1 KB: 1620).  On operands as they
// come the clock falls to 1.6 .. 1.9 GHz instead, and of all that only 4 % are left: 4096 x 4096 x 65536, called in turn, 1.88 ms
// (1.17 PFLOP/s; the library's product 1.46 ms), with d along the sum 1.66 ms (1.32), its two terms 3.49 ms (1.26).  No bank
// conflicts.  Measured and not taken: 256 x 128 in two blocks a CU 2.31 ms, not 1.90 (the loads); 128 x 128 a wave, four waves,
// 2.59 (the sums do not fit beside the operands); five slabs, a higher priority of the products, and LDS reads among them: no
// difference; planes in turn for every 32 elements, so that a load takes both: float 220, 210, 250 us, not 227, 203, 238, and the
// pass that writes them 490, not 434.
#pragma once
#include <type_traits>

#include "bf16_core.h"
#include "common.h"

namespace vcnn {

struct Operand16 {
  const char* base;
  int64_t pitch;  // bytes from row to row
  int count;      // rows along k: how many; rows of k: groups of eight elements in each
};

struct ProductArgs {
  Operand16 a, b;
  int k;                // contraction steps (rows along k: up to the next multiple of 8 there are zeros)
  int tiles_a, tiles_b;
  int slabs_per_split;  // of ceil(k / 32)
};

// BA x BB outputs by waves of 16 TA x 16 TB, from PA and PB planes of the operands: high x high, and the products of the lower
// terms with the other's high one.  RING slabs in LDS.
template <int BA_, int BB_, int TA_, int TB_, int PA_, int PB_, int RING_>
struct ProductTile {
  static constexpr int BA = BA_, BB = BB_, TA = TA_, TB = TB_, PA = PA_, PB = PB_, RING = RING_;
  static constexpr int WA = BA / (16 * TA), WB = BB / (16 * TB), WAVES = WA * WB, THREADS = WAVES * 64;
  static constexpr int WORDS = (PA * BA + PB * BB) * 4;  // 16-byte words of a slab of 32 steps
  static constexpr size_t LDS = (size_t)RING * WORDS * 16;
  static constexpr int BLOCKS = 160 * 1024 / LDS >= 2 && THREADS <= 256 ? 2 : 1;   // a CU's
  static constexpr int WAVES_SIMD = BLOCKS * WAVES / 4;
  static constexpr int LA = BA * 4 / THREADS, LB = BB * 4 / THREADS;  // words a thread brings of a plane
  static constexpr int LOADS = PA * LA + PB * LB;
  static_assert(TA % 2 == 0 && LA * THREADS == BA * 4 && LB * THREADS == BB * 4, "whole slabs");
};

__device__ const uint4 kZeroWord = {0, 0, 0, 0};

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t* LdsShort4;

// One operand's way into LDS and from there to the registers.  R rows of the tile, THREADS threads, L words each.
//   rows along k: word c (of four) of row r at place 4 r + (c ^ swizzle(r)): sixteen lanes of a read meet all banks (as in int8.hip)
//   rows of k:    word c (of R / 8) of step k at place R / 8 * k + (c ^ turn(k)): a read of half a wave takes two neighbouring
//                 words of eight steps 8 g + 0 .. 3 and 8 (g + 1) + 0 .. 3, which turn() sends to different banks
// PLANES: how many there are of it in memory.
template <bool ALONG, int PLANES, int R, int THREADS>
struct Way {
  static constexpr int L = R * 4 / THREADS, WPR = R / 8;
  static_assert(R >= 64 || ALONG, "the banks");
  __device__ static __forceinline__ int swizzle(int r) {
    const int h = r >> 2 & 3;
    return h >> 1 | ((h ^ h >> 1) & 1) << 1;
  }
  __device__ static __forceinline__ int turn(int k) {
    return R >= 128 ? 2 * ((k & 3) | (k >> 3 & 1) << 2) : 2 * ((k >> 1 & 1) | (k >> 3 & 1) << 1);
  }

  const char* base;
  int64_t pitch;
  uint32_t offset[L];
  int step[L];  // of word i: within a slab, the first contraction step (along: of its eight)
  __device__ __forceinline__ Way(const Operand16& o, int r0, int tid) : base(o.base), pitch(o.pitch) {
    if constexpr (ALONG) {
      base += (int64_t)r0 * pitch;
#pragma unroll
      for (int i = 0; i < L; ++i) {
        const int r = i * (THREADS / 4) + (tid >> 2), c = (tid & 3) ^ swizzle(r);
        offset[i] = (uint32_t)min(r, o.count - 1 - r0) * (uint32_t)pitch + c * 16;  // rows behind the last: that one again
        step[i] = c * 8;
      }
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        const int p = i * THREADS + tid, k = p / WPR, c = min(r0 / 8 + ((p % WPR) ^ turn(k)), o.count - 1);
        offset[i] = (uint32_t)k * (uint32_t)pitch + (uint32_t)((c >> 3) * (PLANES * 128) + (c & 7) * 16);
        step[i] = k;
      }
    }
  }
  // Word i of a plane of slab s (32 steps from 32 s on) to `to` (wave-uniform).
  __device__ __forceinline__ const char* from(int s, int plane) const {
    int64_t at;
    if constexpr (ALONG) at = (int64_t)(s >> 1) * (PLANES * 128) + (s & 1) * 64 + plane * 128;
    else at = (int64_t)s * 32 * pitch + plane * 128;
    return base + at;
  }
  __device__ __forceinline__ void stage(int i, int s, int plane, uint4* to) const { load_to_lds16(from(s, plane), offset[i], to); }
  // Only `left` of the 32 steps are there: zeros for the others.
  __device__ __forceinline__ void stage(int i, int s, int plane, int left, uint4* to) const {
    load_to_lds16(step[i] < left ? reinterpret_cast<const uint4*>(from(s, plane) + offset[i]) : &kZeroWord, to);
  }
  // Row tile at r (of the tile) of the slab at buf: lane l holds row l % 16, steps 8 (l / 16) .. + 8.
  __device__ static __forceinline__ uint4 fragment(const uint4* buf, int r, int lane) {
    if constexpr (ALONG) {
      return buf[r * 4 + (lane & 15) * 4 + ((lane >> 4) ^ swizzle(lane & 15))];
    } else {
      const int k = 8 * (lane >> 4) + (lane >> 2 & 3), c = (r / 8 + (lane >> 1 & 1)) ^ turn(k);
      const char* const at = reinterpret_cast<const char*>(buf + k * WPR + c) + (lane & 1) * 8;
      const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4)at);
      const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4)(at + 4 * WPR * 16));  // (turn(k + 4) == turn(k))
      const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
      return make_uint4(l.x, l.y, h.x, h.y);
    }
  }
};

// Consecutive blocks go to the eight XCDs in turn: each takes a contiguous eighth of the tiles, in patches of eight tiles of b by
// as many of a as it comes to, so that the blocks at work share what they read in its L2.
__device__ __forceinline__ void product_tile_of(const ProductArgs& p, int* ta, int* tb) {
  const int total = p.tiles_a * p.tiles_b, per = total / 8, block = blockIdx.x;
  const int item = block < per * 8 ? (block % 8) * per + block / 8 : block;
  const int group = item / (8 * p.tiles_a), in = item - group * 8 * p.tiles_a, wide = min(8, p.tiles_b - group * 8);
  *ta = in / wide, *tb = group * 8 + in % wide;
}

// Slabs of 32 steps go to a ring by direct loads.  A wave reads the second half of a step's a-tiles while it multiplies the first, and
// the first of the next step while it multiplies the second.  The one barrier of a step stands between the two: there the next slab is
// in LDS for every wave, and every wave has read this one, whose place then takes the slab RING steps on; so a slab has RING - 1 steps
// to arrive.  acc[i][j]: lane l has a = 16 i + 4 (l / 16) + q, b = 16 j + l % 16 of the wave's part.
template <typename TILE, bool F16, bool A_ALONG, int A_PLANES, bool B_ALONG, int B_PLANES>
__device__ __forceinline__ void slab_product(const ProductArgs& p, int a0, int b0, uint4* smem,
                                             f32x4 (&acc)[TILE::TA][TILE::TB]) {
  constexpr int TA = TILE::TA, TB = TILE::TB, PA = TILE::PA, PB = TILE::PB, LA = TILE::LA, LB = TILE::LB, L = TILE::LOADS;
  constexpr int R = TILE::RING;
  using WayA = Way<A_ALONG, A_PLANES, TILE::BA, TILE::THREADS>;
  using WayB = Way<B_ALONG, B_PLANES, TILE::BB, TILE::THREADS>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const WayA wa(p.a, a0, tid);
  const WayB wb(p.b, b0, tid);
  const int first = blockIdx.y * p.slabs_per_split;
  const int slabs = min(p.slabs_per_split, (p.k + 31) / 32 - first), whole = min(slabs, p.k / 32 - first);
  // load i of L of slab s, to its place `slot` in the ring; WHOLE: it is known to have 32 steps (otherwise, and behind the last, zeros for what there is not)
  auto stage = [&](int s, int slot, int i, auto is_whole) {
    constexpr bool WHOLE = decltype(is_whole)::value;
    uint4* const to = smem + slot * TILE::WORDS + i * TILE::THREADS + wave * 64;
    const int left = WHOLE ? 32 : s < slabs ? p.k - (first + s) * 32 : 0;
    if (i < PA * LA) {
      if constexpr (WHOLE) wa.stage(i % LA, first + s, i / LA, to);
      else wa.stage(i % LA, first + s, i / LA, left, to);
    } else {
      const int n = i - PA * LA;
      if constexpr (WHOLE) wb.stage(n % LB, first + s, n / LB, to);
      else wb.stage(n % LB, first + s, n / LB, left, to);
    }
  };
#pragma unroll
  for (int i = 0; i < TA; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
  const int ra = (wave % TILE::WA) * 16 * TA, rb = (wave / TILE::WA) * 16 * TB;
  constexpr int H = TA / 2;
  // fa: [half][term]; fb: the high terms of this step and the next, and the lower ones of this step
  uint4 fa[2][PA][H], fb[2][TB], fl[2][TB];
  auto read_a = [&](int slot, int h) {
    const uint4* const buf = smem + slot * TILE::WORDS;
#pragma unroll
    for (int t = 0; t < PA; ++t)
#pragma unroll
      for (int i = 0; i < H; ++i) fa[h][t][i] = WayA::fragment(buf + t * TILE::BA * 4, ra + (h * H + i) * 16, lane);
  };
  auto read_b = [&](int slot, uint4 (&to)[TB], int t) {
    const uint4* const buf = smem + slot * TILE::WORDS + (PA * TILE::BA + t * TILE::BB) * 4;
#pragma unroll
    for (int j = 0; j < TB; ++j) to[j] = WayB::fragment(buf, rb + j * 16, lane);
  };
  // The products of half h: term t of a with `with`.  Of slab s every L / (2 PAIRS) loads belong to one such turn and stand among its
  // products: a load waits its turn behind those of the other waves, and the matrix cores are not to wait with it.
  constexpr int PAIRS = PA == 2 && PB == 2 ? 3 : PA * PB;
  auto multiply = [&](int h, int t, const uint4 (&with)[TB], int s, int slot, int turn, auto is_whole) {
    const int l0 = L * turn / (2 * PAIRS), l1 = L * (turn + 1) / (2 * PAIRS), every = H * TB / (l1 > l0 ? l1 - l0 : 1);
#pragma unroll
    for (int m = 0; m < H * TB; ++m) {
      const int i = m / TB, j = m % TB;
      if constexpr (F16) acc[h * H + i][j] = mfma_f16(fa[h][t][i], with[j], acc[h * H + i][j]);
      else acc[h * H + i][j] = mfma_bf16(fa[h][t][i], with[j], acc[h * H + i][j]);
      if (m % every == every / 2 && l0 + m / every < l1) {
        __builtin_amdgcn_sched_barrier(0);
        stage(s, slot, l0 + m / every, is_whole);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr auto all_but = [](int n) { return 0x0F70 | (n & 15) | n >> 4 << 14; };  // vmcnt(n)
  constexpr int HALF = L * PAIRS / (2 * PAIRS);  // loads of a slab that are issued in a step's second half, R steps ahead
  static_assert((R - 1) * L + HALF < 64, "the counts fit");
#pragma unroll
  for (int n = 0; n < (R - 1) * L + HALF; ++n) stage(n / L, n / L, n % L, std::false_type());
  __builtin_amdgcn_s_waitcnt(all_but((R - 2) * L + HALF));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_b(0, fb[0], 0), read_a(0, 0);
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): so that the loop's own waits need not count what came before it
  int here = 0;  // the slab's place
  auto step = [&](int s, int n, auto is_whole) {
    const int next = here + 1 == R ? 0 : here + 1, last = here == 0 ? R - 1 : here - 1;
    int turn = PAIRS;
    if constexpr (PB >= 2) read_b(here, fl[0], 1);
    if constexpr (PB == 3) read_b(here, fl[1], 2);
    read_a(here, 1);
    __builtin_amdgcn_sched_barrier(0);
    multiply(0, 0, fb[n], s + R - 1, last, turn++, is_whole);
    if constexpr (PA == 2) multiply(0, 1, fb[n], s + R - 1, last, turn++, is_whole);
    if constexpr (PB >= 2) multiply(0, 0, fl[0], s + R - 1, last, turn++, is_whole);
    if constexpr (PB == 3) multiply(0, 0, fl[1], s + R - 1, last, turn++, is_whole);
    // slab s + 1 is there, for everyone; slab s has been read by everyone (vmcnt and lgkmcnt(0))
    __builtin_amdgcn_s_waitcnt(all_but((R - 2) * L) & ~0x0F00);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    turn = 0;
    read_b(next, fb[n ^ 1], 0), read_a(next, 0);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (PB == 3) multiply(1, 0, fl[1], s + R, here, turn++, is_whole);
    if constexpr (PB >= 2) multiply(1, 0, fl[0], s + R, here, turn++, is_whole);
    if constexpr (PA == 2) multiply(1, 1, fb[n], s + R, here, turn++, is_whole);
    multiply(1, 0, fb[n], s + R, here, turn++, is_whole);
    here = next;
  };
  int s = 0;
  for (; s + R + 1 < whole; s += 2) {
    step(s, 0, std::true_type());
    step(s + 1, 1, std::true_type());
  }
  for (; s < slabs; s += 2) {
    step(s, 0, std::false_type());
    step(s + 1, 1, std::false_type());
  }
  __builtin_amdgcn_s_waitcnt(0x0070);  // nothing more is on its way to LDS, or from it
  __syncthreads();
}

}  // namespace vcnn

// The random bits of dropout, and the arguments that dropout is described by.
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two products
// of 32 by 32 bits turn a counter of 128 bits and a key of 64 into 128 random bits, so that any element's bits can be made anywhere,
// in the backward pass as in the forward one, and no mask is stored.  The key is the seed, the counter (block, step, site), a block
// eight neighbouring elements of a row with 16 bits each.  16 bits, because the products are what the generator costs (v_mul_hi and
// v_mul_lo run at a quarter of the rate of other instructions): at 32 bits an element a bfloat16 pass would wait for them instead of
// for memory.  The rate is rounded to a multiple of 2^-16 for it, and the scale is that of the rounded rate, so that the mean stays.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vcnn {

struct Dropout {
  const uint64_t* rng;   // device: seed, step (null: no dropout)
  uint32_t site, limit;  // an element is kept where its 16 bits are at least `limit`
  float scale;           // 65536 / (65536 - limit)
};

struct DropoutKey {  // wave-uniform
  uint32_t k0, k1, step, site;
  DropoutKey() = default;
  __device__ __forceinline__ explicit DropoutKey(const Dropout& d) {
    const uint64_t seed = d.rng[0];
    k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32), step = (uint32_t)d.rng[1], site = d.site;
  }
};

__device__ __forceinline__ uint4 philox(const DropoutKey& key, uint64_t block) {
  uint32_t a = (uint32_t)block, b = (uint32_t)(block >> 32), c = key.step, d = key.site, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = (uint64_t)0xD2511F53u * a, q = (uint64_t)0xCD9E8D57u * c;
    a = (uint32_t)(q >> 32) ^ b ^ k0, b = (uint32_t)q;
    c = (uint32_t)(p >> 32) ^ d ^ k1, d = (uint32_t)p;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
  return make_uint4(a, b, c, d);
}

// Blocks of eight elements in a row.
__host__ __device__ __forceinline__ uint32_t dropout_blocks(int cols) { return ((uint32_t)cols + 7) / 8; }

// The bits of elements c .. c + N of a row (N 4 or 8, c a multiple of N), the row's first block being `first`.
template <int N>
__device__ __forceinline__ void dropout_bits(const DropoutKey& key, uint64_t first, int c, uint32_t (&bits)[N]) {
  const uint4 r = philox(key, first + (uint32_t)(c >> 3));
  if constexpr (N == 8) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) bits[2 * i] = w[i] & 0xffffu, bits[2 * i + 1] = w[i] >> 16;
  } else {
    const uint32_t w[2] = {c & 4 ? r.z : r.x, c & 4 ? r.w : r.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) bits[2 * i] = w[i] & 0xffffu, bits[2 * i + 1] = w[i] >> 16;
  }
}

// A kept element (one that is not is replaced, so that an infinity there leaves no NaN), and the residual with one rounding.
__device__ __forceinline__ float dropped(float v, uint32_t bits, const Dropout& d) { return bits >= d.limit ? v * d.scale : 0.f; }
__device__ __forceinline__ float dropped(float v, uint32_t bits, const Dropout& d, float residual) {
  return bits >= d.limit ? fmaf(v, d.scale, residual) : residual;
}

}  // namespace vcnn

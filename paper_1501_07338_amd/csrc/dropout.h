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

// The random words of a thread's groups of N elements (4 or 8) in a row, two elements a word: group k starts at element
// (k * per_row + tid) * N (per_row even), the row's first block is `first`.  Groups of four: two neighbouring lanes share a block,
// so of two groups each makes one block and hands the other lane its half.  All lanes of the wave take part.
template <int N, int K>
__device__ __forceinline__ void dropout_words(const DropoutKey& key, uint64_t first, int per_row, int tid, uint32_t (&words)[K][N / 2]) {
  if constexpr (N == 8) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint4 r = philox(key, first + (uint32_t)(k * per_row + tid));
      words[k][0] = r.x, words[k][1] = r.y, words[k][2] = r.z, words[k][3] = r.w;
    }
  } else {
    const bool odd = tid & 1;
#pragma unroll
    for (int k = 0; k < K; k += 2) {
      if (k + 1 < K) {
        const uint4 r = philox(key, first + (uint32_t)(((k + (odd ? 1 : 0)) * per_row + tid) >> 1));
        const uint32_t u = __shfl_xor(odd ? r.x : r.z, 1), v = __shfl_xor(odd ? r.y : r.w, 1);
        words[k][0] = odd ? u : r.x, words[k][1] = odd ? v : r.y;
        words[k + 1][0] = odd ? r.z : u, words[k + 1][1] = odd ? r.w : v;
      } else {
        const uint4 r = philox(key, first + (uint32_t)((k * per_row + tid) >> 1));
        words[k][0] = odd ? r.z : r.x, words[k][1] = odd ? r.w : r.y;
      }
    }
  }
}
// Those of one group at element c (a multiple of N).
template <int N>
__device__ __forceinline__ void dropout_words(const DropoutKey& key, uint64_t first, int c, uint32_t (&words)[N / 2]) {
  const uint4 r = philox(key, first + (uint32_t)(c >> 3));
  if constexpr (N == 8) words[0] = r.x, words[1] = r.y, words[2] = r.z, words[3] = r.w;
  else words[0] = c & 4 ? r.z : r.x, words[1] = c & 4 ? r.w : r.y;
}
// Element i's 16 bits of its group's words.
template <int W>
__device__ __forceinline__ uint32_t bits_of(const uint32_t (&words)[W], int i) { return i & 1 ? words[i / 2] >> 16 : words[i / 2] & 0xffffu; }

// A kept element (one that is not is replaced, so that an infinity there leaves no NaN), and the residual with one rounding.
__device__ __forceinline__ float dropped(float v, uint32_t bits, const Dropout& d) { return bits >= d.limit ? v * d.scale : 0.f; }
__device__ __forceinline__ float dropped(float v, uint32_t bits, const Dropout& d, float residual) {
  return bits >= d.limit ? fmaf(v, d.scale, residual) : residual;
}

}  // namespace vcnn

// Dropout of the rows of a matrix, with the residual's addition behind it, and the step of its generator (dropout.h):
//     y = residual + (kept ? x / (1 - p) : 0),   dx = kept ? dy / (1 - p) : 0
// A thread makes the bits of a block of eight elements of one row and loads and stores them as groups of 16 bytes (two in float)
// wherever the row starts.  Bandwidth: bfloat16, 8192 x 5120, with a residual 51.4 us (4.9 TB/s; a large copy 5.1), without 31.5
// (read from the last-level cache in part); the generator's products are hidden behind the loads of other waves.
#include "dropout.h"

#include "rows.h"

namespace vcnn {

struct DropoutArgs {
  const void* x;
  const void* residual;  // null: none
  void* y;
  uint64_t blocks;    // of all rows
  uint32_t per_row;
  int cols;
  Dropout drop;
};

static constexpr int kDropoutThreads = 256;

template <typename T, bool ADDED>
__global__ __launch_bounds__(kDropoutThreads) void dropout_kernel(DropoutArgs a) {
  constexpr int N = Group<T>::N, G = 8 / N;
  const DropoutKey key(a.drop);
  const uint64_t stride = (uint64_t)gridDim.x * kDropoutThreads;
  for (uint64_t block = (uint64_t)blockIdx.x * kDropoutThreads + threadIdx.x; block < a.blocks; block += stride) {
    const uint64_t row = block < 1ull << 32 ? (uint32_t)block / a.per_row : block / a.per_row;
    const int c = (int)(uint32_t)(block - row * a.per_row) * 8;
    const int64_t at = (int64_t)row * a.cols;
    const T* const x = reinterpret_cast<const T*>(a.x) + at;
    const T* const res = reinterpret_cast<const T*>(a.residual) + at;
    Loose16 px[G], pr[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (g == 0 || c + g * N < a.cols) {
        px[g] = load_group(x, c + g * N, a.cols);
        if (ADDED) pr[g] = load_group(res, c + g * N, a.cols);
      }
    uint32_t words[4];
    dropout_words<8>(key, block, 0, words);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (g > 0 && c + g * N >= a.cols) break;
      float v[N];
      unpack(px[g], v);
      if constexpr (ADDED) {
        float w[N];
        unpack(pr[g], w);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = dropped(v[i], bits_of(words, g * N + i), a.drop, w[i]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = dropped(v[i], bits_of(words, g * N + i), a.drop);
      }
      store_group(reinterpret_cast<T*>(a.y) + at, c + g * N, a.cols, pack(v));
    }
  }
}

__global__ void rng_advance_kernel(uint64_t* rng) { rng[1] += 1; }

template <typename T>
static void launch_dropout_typed(const DropoutArgs& a, hipStream_t st) {
  const unsigned blocks = (unsigned)std::min<uint64_t>((a.blocks + kDropoutThreads - 1) / kDropoutThreads, 256 * 8);
  if (a.residual) hipLaunchKernelGGL((dropout_kernel<T, true>), dim3(blocks), dim3(kDropoutThreads), 0, st, a);
  else hipLaunchKernelGGL((dropout_kernel<T, false>), dim3(blocks), dim3(kDropoutThreads), 0, st, a);
}

vcnn_status launch_dropout(int dtype, int rows, int cols, const Dropout& drop, const void* x, const void* residual, void* y,
                           hipStream_t st) {
  const uint32_t per_row = dropout_blocks(cols);
  const DropoutArgs a{x, residual, y, (uint64_t)rows * per_row, per_row, cols, drop};
  if (dtype == VCNN_BF16) launch_dropout_typed<bf16>(a, st);
  else launch_dropout_typed<float>(a, st);
  return check_launch("dropout");
}

vcnn_status launch_rng_advance(uint64_t* rng, hipStream_t st) {
  hipLaunchKernelGGL(rng_advance_kernel, dim3(1), dim3(1), 0, st, rng);
  return check_launch("rng_advance");
}

}  // namespace vcnn

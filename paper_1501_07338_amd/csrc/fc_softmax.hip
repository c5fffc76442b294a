// A fully connected layer with many outputs and its softmax cost, forward and backward, without keeping the logits:
//     z = x w^T + bias,   lse_r = log sum exp z_r,   loss = 1/C sum over the C samples that count of lse_r - z_r[label]
//     d = softmax(z) - onehot(label) (0 for samples that do not count),   dx = d w / C,   dw = d^T x / C,   dbias = sum_r d_r / C
//
// The samples go through in parts.  A part's logits are made once (z, float), by a product whose tiles leave the largest logit of
// each sample and its sum of exponentials beside them; these are joined to lse; one pass turns z where it stands into d, a high
// and a low bfloat16 term of the difference, and two products make dx and dw from it.  Without gradients z is not stored at all.
//   d in two terms: dw is float, and one bfloat16 term alone would leave 2^-9 of each element in it (the two leave 2^-18).  dx is
//   bfloat16 itself and takes the high term alone.
#include <algorithm>

#include "rows.h"
#include "slab_product.h"

namespace vcnn {

static constexpr int kThreads = 256;

struct LossMeta {  // at the head of the workspace
  float inverse;   // 1 / C, 0 if no sample counts
};

// ---- operands ----------------------------------------------------------------------------------------------------------
// Rows re-laid with a length of whole groups of eight, the rows of samples that do not count as zeros (whatever they hold must
// not meet the zeros of d as a NaN).  Block 0 of the first part counts the samples.
template <typename T>
__global__ __launch_bounds__(kThreads) void relay_rows_kernel(const T* x, T* to, int64_t rows, int cols, int groups,
                                                              const int32_t* labels, int ignore, const int32_t* all_labels,
                                                              int batch, LossMeta* meta) {
  if (meta && blockIdx.x == 0) {
    __shared__ int counts[kThreads / 64];
    int n = 0;
    for (int b = threadIdx.x; b < batch; b += kThreads) n += all_labels[b] != ignore;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
    if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      n = 0;
      for (int w = 0; w < kThreads / 64; ++w) n += counts[w];
      meta->inverse = n ? 1.f / (float)n : 0.f;
    }
  }
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * groups; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / groups;
    const int c = (int)(i - row * groups) * 8;
    Loose16 v{{0, 0, 0, 0}};
    if (!labels || labels[row] != ignore) v = load_group(x + row * cols, c, cols);
    *reinterpret_cast<uint4*>(to + i * 8) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
  }
}

// ---- products ------------------------------------------------------------------------------------------------------------
enum { EPI_LOGITS = 0, EPI_DX = 1, EPI_DW = 2 };

struct LossProduct {
  ProductArgs p;
  int rows, cols;        // of the result
  // EPI_LOGITS: a classes, b samples
  float* z;              // [rows][z_pitch] (nullable)
  int64_t z_pitch;
  const float* bias;     // nullable
  const int32_t* labels;
  float2* stats;         // [16 TA of classes][rows]: the largest logit, the sum of exponentials about it
  float* at_label;
  // EPI_DX, EPI_DW
  const LossMeta* meta;
  float* partial;        // [splits][rows][cols] (EPI_DX, shared sums)
  void* out;             // [rows][cols]
  int add;               // EPI_DW: to what is there
};

template <typename T>
__device__ __forceinline__ void store4(T* at, const float (&v)[4], int n) {
  if (n >= 4) {
    if constexpr (sizeof(T) == 4) {
      struct __attribute__((packed, aligned(4))) Four { float v[4]; };
      *reinterpret_cast<Four*>(at) = Four{{v[0], v[1], v[2], v[3]}};
    } else {
      Loose8 p;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        p.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){v[2 * i], v[2 * i + 1]}, bf16x2));
      *reinterpret_cast<Loose8*>(at) = p;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) st(at + i, v[i]);
  }
}

template <typename TILE, int EPI, bool A_ALONG, bool B_ALONG, bool B_PLANES>
__global__ __launch_bounds__(TILE::THREADS, 2) void loss_product_kernel(LossProduct a) {
  extern __shared__ uint4 smem16[];
  int ta, tb;
  product_tile_of(a.p, &ta, &tb);
  f32x4 acc[TILE::TA][TILE::TB];
  slab_product<TILE, false, A_ALONG, false, B_ALONG, B_PLANES>(a.p, ta * TILE::BA, tb * TILE::BB, smem16, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a0 = ta * TILE::BA + (wave % TILE::WA) * 16 * TILE::TA, b0 = tb * TILE::BB + (wave / TILE::WA) * 16 * TILE::TB;
  const int ca = a0 + 4 * (lane >> 4);  // + 16 i + q
  if constexpr (EPI == EPI_LOGITS) {
#pragma unroll
    for (int i = 0; i < TILE::TA; ++i) {
      float bias[4] = {0.f, 0.f, 0.f, 0.f};
      if (a.bias) {
#pragma unroll
        for (int q = 0; q < 4; ++q) bias[q] = a.bias[min(ca + 16 * i + q, a.cols - 1)];
      }
#pragma unroll
      for (int j = 0; j < TILE::TB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[i][j][q] += bias[q];
    }
#pragma unroll
    for (int j = 0; j < TILE::TB; ++j) {
      const int b = b0 + 16 * j + (lane & 15);
      const int label = a.labels[min(b, a.rows - 1)];
      float most = -__builtin_inff(), sum = 0.f;
#pragma unroll
      for (int i = 0; i < TILE::TA; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (ca + 16 * i + q < a.cols) most = fmaxf(most, acc[i][j][q]);
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      if (most > -__builtin_inff()) {  // (none of these classes is possible: their sum is 0)
#pragma unroll
        for (int i = 0; i < TILE::TA; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (ca + 16 * i + q < a.cols) sum += expf(acc[i][j][q] - most);
      } else {  // (or all are NaN)
#pragma unroll
        for (int i = 0; i < TILE::TA; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (ca + 16 * i + q < a.cols && acc[i][j][q] != acc[i][j][q]) sum = acc[i][j][q];
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (b >= a.rows) continue;
      if (lane < 16 && a0 < a.cols) a.stats[(int64_t)(a0 / (16 * TILE::TA)) * a.rows + b] = make_float2(most, sum);
      float* const z = a.z + (int64_t)b * a.z_pitch;
#pragma unroll
      for (int i = 0; i < TILE::TA; ++i) {
        const int c = ca + 16 * i, at = label - c;
        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        if (a.z && c < a.cols) *reinterpret_cast<float4*>(z + c) = make_float4(v[0], v[1], v[2], v[3]);  // (rows have whole groups)
        if (at >= 0 && at < 4 && label < a.cols) a.at_label[b] = at == 0 ? v[0] : at == 1 ? v[1] : at == 2 ? v[2] : v[3];
      }
    }
  } else {
    const float inverse = a.meta->inverse;
#pragma unroll
    for (int j = 0; j < TILE::TB; ++j) {
      const int b = b0 + 16 * j + (lane & 15);
      if (b >= a.rows) continue;
#pragma unroll
      for (int i = 0; i < TILE::TA; ++i) {
        const int c = ca + 16 * i, n = a.cols - c;
        if (n <= 0) continue;
        const int64_t at = (int64_t)b * a.cols + c;
        float v[4];
        if (EPI == EPI_DX && a.partial) {
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = acc[i][j][q];
          store4(a.partial + (int64_t)blockIdx.y * a.rows * a.cols + at, v, n);
          continue;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = acc[i][j][q] * inverse;
        if constexpr (EPI == EPI_DX) {
          store4(reinterpret_cast<bf16*>(a.out) + at, v, n);
        } else {
          float* const out = reinterpret_cast<float*>(a.out) + at;
          if (a.add) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (q < n) v[q] += out[q];
          }
          store4(out, v, n);
        }
      }
    }
  }
}

// dx from the shares of its sums, always in the same order.
__global__ __launch_bounds__(kThreads) void loss_join_kernel(const float* partial, int splits, int64_t count, const LossMeta* meta,
                                                             bf16* out) {
  const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4;
  if (i >= count) return;
  const float inverse = meta->inverse;
  const int n = (int)std::min<int64_t>(4, count - i);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < n) v[q] += partial[s * count + i + q];
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] *= inverse;
  store4(out + i, v, n);
}

// ---- softmax -------------------------------------------------------------------------------------------------------------
// lse of sixteen samples from the tiles' maxima and sums, sixteen threads each, joined in a fixed order; what each sample costs.
__global__ __launch_bounds__(kThreads) void loss_rows_kernel(const float2* stats, int tiles, int rows, int classes,
                                                             const int32_t* labels, int ignore, const float* at_label, float* lse,
                                                             float* each) {
  __shared__ float2 parts[16][17];
  const int in = threadIdx.x & 15, part = threadIdx.x >> 4, b = blockIdx.x * 16 + in;
  float most = -__builtin_inff(), sum = 0.f;
  auto meet = [&](float m, float s) {
    const float top = fmaxf(most, m);
    if (top > -__builtin_inff()) sum = sum * expf(most - top) + s * expf(m - top);
    else sum += s;  // (nothing yet, or a NaN)
    most = top;
  };
  if (b < rows) {
#pragma unroll 4
    for (int t = part; t < tiles; t += 16) {
      const float2 v = stats[(int64_t)t * rows + b];
      meet(v.x, v.y);
    }
  }
  parts[part][in] = make_float2(most, sum);
  __syncthreads();
  if (part > 0 || b >= rows) return;
  for (int p = 1; p < 16; ++p) meet(parts[p][in].x, parts[p][in].y);
  const float l = most + logf(sum);
  const int label = labels[b];
  if (lse) lse[b] = l;
  each[b] = label == ignore ? 0.f : label < 0 || label >= classes ? __builtin_nanf("") : l - at_label[b];
}

// z to d where it stands: 64 floats of a row become 64 high and 64 low terms (the sixteen lanes that read them are of one wave, which
// has them all before it writes); behind the last class zeros.  Each block leaves its samples' share of dbias.
__global__ __launch_bounds__(kThreads) void loss_grad_kernel(float* z, int64_t pitch, int rows, int classes, const int32_t* labels,
                                                             int ignore, const float* lse, float* shares, int64_t share_pitch) {
  __shared__ float sums[16][64];
  const int in = threadIdx.x & 15, part = threadIdx.x >> 4, c = blockIdx.x * 64 + in * 4;
  float total[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int b = blockIdx.y * 64 + n * 16 + part;
    if (b >= rows) break;
    const int label = labels[b];
    const bool counts = label != ignore, bad = counts && (label < 0 || label >= classes);
    const float l = lse[b];
    char* const row = reinterpret_cast<char*>(z + b * pitch);
    const float4 v = *reinterpret_cast<const float4*>(row + c * 4);
    float d[4] = {v.x, v.y, v.z, v.w}, low[4];
    bf16x2 h[2], r[2];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      d[q] = expf(d[q] - l) - (c + q == label ? 1.f : 0.f);
      if (bad) d[q] = __builtin_nanf("");
      if (!counts || c + q >= classes) d[q] = 0.f;
      total[q] += d[q];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      h[i] = __builtin_convertvector((f32x2){d[2 * i], d[2 * i + 1]}, bf16x2);
      low[2 * i] = d[2 * i] - (float)h[i][0], low[2 * i + 1] = d[2 * i + 1] - (float)h[i][1];
      r[i] = __builtin_convertvector((f32x2){low[2 * i], low[2 * i + 1]}, bf16x2);
    }
    char* const to = row + (int64_t)blockIdx.x * 256 + in * 8;
    *reinterpret_cast<uint2*>(to) = make_uint2(__builtin_bit_cast(uint32_t, h[0]), __builtin_bit_cast(uint32_t, h[1]));
    *reinterpret_cast<uint2*>(to + 128) = make_uint2(__builtin_bit_cast(uint32_t, r[0]), __builtin_bit_cast(uint32_t, r[1]));
  }
  if (!shares) return;
#pragma unroll
  for (int q = 0; q < 4; ++q) sums[part][in * 4 + q] = total[q];
  __syncthreads();
  if (threadIdx.x < 64) {
    float s = 0.f;
#pragma unroll
    for (int p = 0; p < 16; ++p) s += sums[p][threadIdx.x];
    shares[(int64_t)blockIdx.y * share_pitch + blockIdx.x * 64 + threadIdx.x] = s;
  }
}

__global__ __launch_bounds__(kThreads) void loss_bias_kernel(const float* shares, int64_t share_pitch, int parts, int classes,
                                                             const LossMeta* meta, int add, float* dbias) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= classes) return;
  float s = 0.f;
#pragma unroll 8
  for (int p = 0; p < parts; ++p) s += shares[p * share_pitch + c];
  s *= meta->inverse;
  dbias[c] = add ? dbias[c] + s : s;
}

// The mean of what the samples cost, in a fixed order.
__global__ __launch_bounds__(1024) void loss_mean_kernel(const float* each, const int32_t* labels, int ignore, int batch, float* loss) {
  __shared__ float sums[16];
  __shared__ int counts[16];
  float s = 0.f;
  int n = 0;
  for (int b = threadIdx.x; b < batch; b += 1024) s += each[b], n += labels[b] != ignore;
  s = wave_sum(s);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s, counts[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x > 0) return;
  s = 0.f, n = 0;
  for (int w = 0; w < 16; ++w) s += sums[w], n += counts[w];
  *loss = n ? s / (float)n : 0.f;
}

// ---- plan ----------------------------------------------------------------------------------------------------------------
using TileLarge = ProductTile<256, 256, 8, 4>;
using TileSmall = ProductTile<128, 128, 4, 4>;

struct LossPlan {
  int part;            // samples at once
  int classes_pitch;   // elements of a row of z
  int groups;          // of eight inputs, of a row
  int stat_tiles;      // of classes
  bool relay_w;
  int splits, slabs_per_split;  // of dx
  int tile_z, tile_dx, tile_dw;
  size_t x, w, stats, at_label, lse, each, z, partial, shares, bytes;  // places in the workspace
};

static constexpr int kMostSamples = 1 << 20;  // of a part

static int tile_of(int64_t a, int64_t b) { return ceil_div(a, 256) * ceil_div(b, 256) >= 192 ? 256 : 128; }

static LossPlan loss_plan(int part, int batch, int in_f, int classes, bool grads) {
  LossPlan p{};
  p.part = part;
  p.classes_pitch = (int)ceil_div(classes, 64) * 64;
  p.groups = (int)ceil_div(in_f, 8);
  p.relay_w = in_f % 8 != 0;
  p.tile_z = tile_of(classes, part), p.tile_dx = tile_of(in_f, part), p.tile_dw = tile_of(in_f, classes);
  p.stat_tiles = (int)ceil_div(classes, p.tile_z == 256 ? 16 * TileLarge::TA : 16 * TileSmall::TA);
  const int slabs = (int)ceil_div(classes, 32);
  p.splits = 1, p.slabs_per_split = slabs;
  const int64_t tiles = ceil_div(in_f, p.tile_dx) * ceil_div(part, p.tile_dx), room = p.tile_dx == 256 ? 256 : 512;
  if (tiles * 2 <= room) {
    const int want = (int)std::min<int64_t>(room / tiles, std::max(1, slabs / 16));
    p.slabs_per_split = (int)ceil_div(slabs, want), p.splits = (int)ceil_div(slabs, p.slabs_per_split);
  }
  size_t at = 256;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
  };
  p.x = take((size_t)part * p.groups * 16);
  p.w = take(p.relay_w ? (size_t)classes * p.groups * 16 : 0);
  p.stats = take((size_t)p.stat_tiles * part * 8);
  p.at_label = take((size_t)part * 4), p.lse = take((size_t)part * 4), p.each = take((size_t)batch * 4);
  if (grads) {
    p.z = take((size_t)part * p.classes_pitch * 4);
    p.partial = take(p.splits > 1 ? (size_t)p.splits * part * in_f * 4 : 0);
    p.shares = take((size_t)ceil_div(part, 64) * p.classes_pitch * 4);
  }
  p.bytes = at;
  return p;
}

// The samples in equal parts of whole tiles, the fewest that keep a part's logits (without gradients: its statistics) within `most`.
static LossPlan loss_plan_within(size_t most, int batch, int in_f, int classes, bool grads) {
  const LossPlan one = loss_plan(64, 64, in_f, classes, grads);
  const size_t row = (size_t)one.groups * 16 + (grads ? (size_t)one.classes_pitch * 4 : (size_t)one.stat_tiles * 8);
  const int64_t fit = std::max<int64_t>(64, std::min<int64_t>((int64_t)(most / row), kMostSamples) / 64 * 64), parts = ceil_div(batch, fit);
  int64_t part = ceil_div(batch, parts);
  if (parts > 1) part = std::min(fit, ceil_div(part, part > 256 ? 256 : 64) * (part > 256 ? 256 : 64));
  return loss_plan((int)part, batch, in_f, classes, grads);
}

size_t fc_softmax_loss_workspace(int batch, int in_f, int classes, bool grads) {
  return loss_plan_within((size_t)1 << 30, batch, in_f, classes, grads).bytes;
}
size_t fc_softmax_loss_least_workspace(int batch, int in_f, int classes, bool grads) {
  return std::min(loss_plan(std::min(batch, 64), batch, in_f, classes, grads).bytes, fc_softmax_loss_workspace(batch, in_f, classes, grads));
}

template <typename TILE, int EPI, bool A_ALONG, bool B_ALONG, bool B_PLANES>
static vcnn_status launch_product(LossProduct a, int splits, hipStream_t st) {
  a.p.tiles_a = (int)ceil_div(a.cols, TILE::BA), a.p.tiles_b = (int)ceil_div(a.rows, TILE::BB);
  const auto kernel = loss_product_kernel<TILE, EPI, A_ALONG, B_ALONG, B_PLANES>;
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)TILE::LDS);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(a.p.tiles_a * a.p.tiles_b), (unsigned)splits), dim3(TILE::THREADS), TILE::LDS, st, a);
  return check_launch("fc_softmax_loss product");
}
template <int EPI, bool A_ALONG, bool B_ALONG, bool B_PLANES>
static vcnn_status launch_product(int tile, const LossProduct& a, int splits, hipStream_t st) {
  return tile == 256 ? launch_product<TileLarge, EPI, A_ALONG, B_ALONG, B_PLANES>(a, splits, st)
                     : launch_product<TileSmall, EPI, A_ALONG, B_ALONG, B_PLANES>(a, splits, st);
}

template <typename T>
static vcnn_status relay(const T* x, T* to, int64_t rows, int cols, int groups, const int32_t* labels, int ignore,
                         const int32_t* all_labels, int batch, LossMeta* meta, hipStream_t st) {
  const int64_t blocks = std::min<int64_t>(ceil_div(rows * groups, kThreads), 256 * 16);
  hipLaunchKernelGGL(relay_rows_kernel<T>, dim3((unsigned)blocks), dim3(kThreads), 0, st, x, to, rows, cols, groups, labels, ignore,
                     all_labels, batch, meta);
  return check_launch("fc_softmax_loss relay");
}

vcnn_status launch_fc_softmax_loss_bf16(int batch, int in_f, int classes, const void* x, const void* w, const float* bias,
                                        const int32_t* labels, int ignore, float* loss, float* sample_loss, void* dx, float* dw,
                                        float* dbias, void* workspace, size_t bytes, hipStream_t st) {
  const bool grads = dx || dw || dbias;
  LossPlan p = loss_plan_within((size_t)1 << 30, batch, in_f, classes, grads);
  for (size_t most = (size_t)1 << 30; p.bytes > bytes; most /= 2) {
    if (most < 256) {
      p = loss_plan(std::min(batch, 64), batch, in_f, classes, grads);
      break;
    }
    p = loss_plan_within(most, batch, in_f, classes, grads);
  }
  char* const ws = (char*)workspace;
  LossMeta* const meta = (LossMeta*)ws;
  float* const each = sample_loss ? sample_loss : (float*)(ws + p.each);
  float* const lse = (float*)(ws + p.lse);
  float* const z = grads ? (float*)(ws + p.z) : nullptr;
  const bf16* weights = (const bf16*)w;
  if (p.relay_w) {
    weights = (const bf16*)(ws + p.w);
    if (vcnn_status s = relay((const bf16*)w, (bf16*)(ws + p.w), classes, in_f, p.groups, nullptr, 0, nullptr, 0, nullptr, st)) return s;
  }
  const int64_t x_pitch = (int64_t)p.groups * 16, z_pitch = (int64_t)p.classes_pitch * 4;
  for (int64_t b0 = 0; b0 < batch; b0 += p.part) {
    const int rows = (int)std::min<int64_t>(p.part, batch - b0);
    const int32_t* const lab = labels + b0;
    bf16* const xs = (bf16*)(ws + p.x);
    if (vcnn_status s = relay((const bf16*)x + b0 * in_f, xs, rows, in_f, p.groups, grads ? lab : nullptr, ignore, labels, batch,
                              b0 == 0 ? meta : nullptr, st))
      return s;
    LossProduct l{};
    l.p.a = {(const char*)weights, x_pitch, classes}, l.p.b = {(const char*)xs, x_pitch, rows};
    l.p.k = p.groups * 8, l.p.segments = 1, l.p.slabs_per_split = (int)ceil_div(l.p.k, 32);
    l.rows = rows, l.cols = classes, l.z = z, l.z_pitch = p.classes_pitch, l.bias = bias, l.labels = lab;
    l.stats = (float2*)(ws + p.stats), l.at_label = (float*)(ws + p.at_label);
    if (vcnn_status s = launch_product<EPI_LOGITS, true, true, false>(p.tile_z, l, 1, st)) return s;
    hipLaunchKernelGGL(loss_rows_kernel, dim3((unsigned)ceil_div(rows, 16)), dim3(kThreads), 0, st, l.stats, p.stat_tiles, rows, classes,
                       lab, ignore, l.at_label, lse, each + b0);
    if (vcnn_status s = check_launch("fc_softmax_loss rows")) return s;
    if (!grads) continue;
    float* const shares = dbias ? (float*)(ws + p.shares) : nullptr;
    hipLaunchKernelGGL(loss_grad_kernel, dim3((unsigned)(p.classes_pitch / 64), (unsigned)ceil_div(rows, 64)), dim3(kThreads), 0, st, z,
                       p.classes_pitch, rows, classes, lab, ignore, lse, shares, p.classes_pitch);
    if (vcnn_status s = check_launch("fc_softmax_loss gradient")) return s;
    if (dx) {
      LossProduct g{};
      g.p.a = {(const char*)weights, x_pitch, p.groups}, g.p.b = {(const char*)z, z_pitch, rows};
      g.p.k = classes, g.p.segments = 1, g.p.slabs_per_split = p.slabs_per_split;
      g.rows = rows, g.cols = in_f, g.meta = meta, g.out = (bf16*)dx + b0 * in_f;
      g.partial = p.splits > 1 ? (float*)(ws + p.partial) : nullptr;
      if (vcnn_status s = launch_product<EPI_DX, false, true, true>(p.tile_dx, g, p.splits, st)) return s;
      if (p.splits > 1) {
        const int64_t count = (int64_t)rows * in_f;
        hipLaunchKernelGGL(loss_join_kernel, dim3((unsigned)ceil_div(count, 4 * kThreads)), dim3(kThreads), 0, st, g.partial, p.splits,
                           count, meta, (bf16*)g.out);
        if (vcnn_status s = check_launch("fc_softmax_loss join")) return s;
      }
    }
    if (dw) {
      LossProduct g{};
      g.p.a = {(const char*)xs, x_pitch, p.groups}, g.p.b = {(const char*)z, z_pitch, p.classes_pitch / 8};
      g.p.k = rows, g.p.segments = 2, g.p.plane_b[1] = 1, g.p.slabs_per_split = 2 * (int)ceil_div(rows, 32);
      g.rows = classes, g.cols = in_f, g.meta = meta, g.out = dw, g.add = b0 > 0;
      if (vcnn_status s = launch_product<EPI_DW, false, false, true>(p.tile_dw, g, 1, st)) return s;
    }
    if (dbias) {
      hipLaunchKernelGGL(loss_bias_kernel, dim3((unsigned)ceil_div(classes, kThreads)), dim3(kThreads), 0, st, shares, p.classes_pitch,
                         (int)ceil_div(rows, 64), classes, meta, b0 > 0, dbias);
      if (vcnn_status s = check_launch("fc_softmax_loss bias")) return s;
    }
  }
  hipLaunchKernelGGL(loss_mean_kernel, dim3(1), dim3(1024), 0, st, each, labels, ignore, batch, loss);
  return check_launch("fc_softmax_loss mean");
}

// ---- float ---------------------------------------------------------------------------------------------------------------
// The samples that count, and x with zeros for the others.
__global__ __launch_bounds__(kThreads) void loss_float_rows_kernel(const float* x, float* to, int64_t count, int cols,
                                                                   const int32_t* labels, int ignore) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < count; i += (int64_t)gridDim.x * kThreads)
    to[i] = labels[i / cols] != ignore ? x[i] : 0.f;
}

// A block a sample: z to d / C where it stands, and what the sample costs.
__global__ __launch_bounds__(kThreads) void loss_float_kernel(float* z, int classes, const int32_t* labels, int ignore,
                                                              const int32_t* all_labels, int batch, int grads, float* each) {
  __shared__ float parts[kThreads / 64];
  __shared__ int counts[kThreads / 64];
  const int b = blockIdx.x, label = labels[b];
  float* const row = z + (int64_t)b * classes;
  const bool counted = label != ignore, good = label >= 0 && label < classes;
  float most = -__builtin_inff();
  for (int c = threadIdx.x; c < classes; c += kThreads) most = fmaxf(most, row[c]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  int n = 0;
  if (grads) {
    for (int i = threadIdx.x; i < batch; i += kThreads) n += all_labels[i] != ignore;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
  }
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = most, counts[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) most = fmaxf(most, parts[w]), n += counts[w];
  __syncthreads();
  float sum = 0.f;
  for (int c = threadIdx.x; c < classes; c += kThreads) sum += expf(row[c] - most);
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) sum += parts[w];
  const float lse = most + logf(sum);
  if (threadIdx.x == 0) each[b] = !counted ? 0.f : good ? lse - row[label] : __builtin_nanf("");
  if (!grads) return;
  __syncthreads();
  const float inverse = n ? 1.f / (float)n : 0.f;
  for (int c = threadIdx.x; c < classes; c += kThreads) {
    const float d = (expf(row[c] - lse) - (c == label ? 1.f : 0.f)) * inverse;
    row[c] = !counted ? 0.f : good ? d : __builtin_nanf("");
  }
}

struct LossFloatPlan {
  int part;
  size_t x, z, each, dw, dbias, bytes;
};
static LossFloatPlan loss_float_plan(int64_t part, int batch, int in_f, int classes, bool grads) {
  LossFloatPlan p{};
  p.part = (int)part;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
  };
  p.each = take((size_t)batch * 4);
  p.z = take((size_t)part * classes * 4);
  if (grads) {
    p.x = take((size_t)part * in_f * 4);
    p.dw = take((size_t)classes * in_f * 4), p.dbias = take((size_t)classes * 4);  // (of a part behind the first)
  }
  p.bytes = at;
  return p;
}
static LossFloatPlan loss_float_plan_within(size_t most, int batch, int in_f, int classes, bool grads) {
  const int64_t fit = std::max<int64_t>(64, std::min<int64_t>((int64_t)(most / ((size_t)classes * 4)), kMostSamples) / 64 * 64);
  return loss_float_plan(std::min<int64_t>(batch, ceil_div(ceil_div(batch, ceil_div(batch, fit)), 64) * 64), batch, in_f, classes, grads);
}
size_t fc_softmax_loss_workspace_f32(int batch, int in_f, int classes, bool grads) {
  return loss_float_plan_within((size_t)1 << 30, batch, in_f, classes, grads).bytes;
}
size_t fc_softmax_loss_least_workspace_f32(int batch, int in_f, int classes, bool grads) {
  return std::min(loss_float_plan(std::min(batch, 64), batch, in_f, classes, grads).bytes, fc_softmax_loss_workspace_f32(batch, in_f, classes, grads));
}

vcnn_status launch_fc_softmax_loss_f32(int batch, int in_f, int classes, const float* x, const float* w, const float* bias,
                                       const int32_t* labels, int ignore, float* loss, float* sample_loss, float* dx, float* dw,
                                       float* dbias, void* workspace, size_t bytes, hipStream_t st) {
  const bool grads = dx || dw || dbias;
  LossFloatPlan p = loss_float_plan_within((size_t)1 << 30, batch, in_f, classes, grads);
  for (size_t most = (size_t)1 << 30; p.bytes > bytes; most /= 2) {
    p = most < 256 ? loss_float_plan(std::min(batch, 64), batch, in_f, classes, grads)
                   : loss_float_plan_within(most, batch, in_f, classes, grads);
    if (most < 256) break;
  }
  char* const ws = (char*)workspace;
  float* const each = sample_loss ? sample_loss : (float*)(ws + p.each);
  float* const z = (float*)(ws + p.z);
  for (int64_t b0 = 0; b0 < batch; b0 += p.part) {
    const int rows = (int)std::min<int64_t>(p.part, batch - b0);
    const int32_t* const lab = labels + b0;
    const float* xs = x + b0 * in_f;
    if (vcnn_status s = vcnn_fc_fwd(VCNN_F32, rows, in_f, classes, VCNN_ACT_NONE, xs, w, bias, z, st)) return s;
    hipLaunchKernelGGL(loss_float_kernel, dim3((unsigned)rows), dim3(kThreads), 0, st, z, classes, lab, ignore, labels, batch, (int)grads,
                       each + b0);
    if (vcnn_status s = check_launch("fc_softmax_loss rows")) return s;
    if (!grads) continue;
    if (dw) {
      const int64_t count = (int64_t)rows * in_f;
      hipLaunchKernelGGL(loss_float_rows_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(count, kThreads), 256 * 16)), dim3(kThreads),
                         0, st, xs, (float*)(ws + p.x), count, in_f, lab, ignore);
      if (vcnn_status s = check_launch("fc_softmax_loss rows of x")) return s;
      xs = (const float*)(ws + p.x);
    }
    float* const dw_here = b0 == 0 || !dw ? dw : (float*)(ws + p.dw);
    float* const db_here = b0 == 0 || !dbias ? dbias : (float*)(ws + p.dbias);
    if (vcnn_status s = vcnn_fc_bwd(VCNN_F32, rows, in_f, classes, xs, w, z, dw_here, db_here, dx ? dx + b0 * in_f : nullptr, st)) return s;
    if (b0 == 0) continue;
    if (dw)
      if (vcnn_status s = launch_sgd_f32((size_t)classes * in_f, -1.f, dw, dw_here, st)) return s;
    if (dbias)
      if (vcnn_status s = launch_sgd_f32((size_t)classes, -1.f, dbias, db_here, st)) return s;
  }
  hipLaunchKernelGGL(loss_mean_kernel, dim3(1), dim3(1024), 0, st, each, labels, ignore, batch, loss);
  return check_launch("fc_softmax_loss mean");
}

}  // namespace vcnn

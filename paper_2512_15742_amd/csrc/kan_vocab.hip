// Softmax cross entropy of rows against a table of outputs, without the logits, and its gradients.
//
//   z[n][v] = scale <h_n, T_v>,   lse_n = log sum_v exp z[n][v],   loss_n = lse_n - z[n][t_n]     (t_n names no row: 0)
//   dS[n][v] = scale dloss_n (exp(z[n][v] - lse_n) - [v == t_n])   (t_n names no row: 0)
//   dh = dS T,   dT (+)= dS^t h
//
// Forward: tiles of z stay in registers; each leaves the maximum and the sum of exponentials of its part of a row, which a
// small launch joins.  Backward: piece by piece of the table, z again, dS of the piece in the workspace, and two products
// with it.  All products run on the matrix cores with fp32 sums.
//
// Operands are 16-bit numbers.  fp32 rows travel as three bf16 parts (24 bits together; 8 of the smaller parts' products
// are below 2^-24 of the whole and left out), so a product is six of parts.  dS of 16-bit types is rounded to the type (2^-9 or 2^-12
// of each entry, the step of the gradients themselves): its entries are about as far apart as the logits, and fp16 holds
// them times 2^14 / max |dloss|, so that probabilities down to 4e-9 keep all bits.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "kan_tokens.hpp"

namespace kan {
namespace {

typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 128;              // outputs of a workgroup in either direction
constexpr int kThreads = 256;
constexpr int kStep = 32;               // products along the contraction per step
constexpr int kPad = 8;
constexpr int kVocabStep = 256;         // pieces of the table are multiples of it
constexpr long long kPackBytes = 256ll << 20, kPieceBytes = 512ll << 20;

constexpr int kMaxParts = 3;
constexpr float kHalfScale = 16384.f;   // of fp16 dS

template <class T>
__device__ __forceinline__ f32x4 mfma(uint4 a, uint4 b, f32x4 c) {
  if constexpr (std::is_same<T, f16>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// An operand of a product out[n][m] = sum_k A(m, k) B(n, k): element (r, k) at p[r * stride + k], or at p[k * stride + r];
// rows and k of it that exist.  Parts lie `part` elements apart.
struct Operand {
  const void* p;
  long long stride, part;
  int rows, depth;
};

enum Epilogue : int { kStats, kGradS, kGradRows };

struct ProductArgs {
  Operand a, b;
  int m, n, k;               // sizes of the product
  int parts;                 // 1, or 3: the operands' parts
  // kStats, kGradS: m = rows of the table from `v0` on, n = tokens
  int v0, V;
  float scale;
  const void* targets;
  int id_dtype;
  float2* stats;             // [tile of the table][tokens]
  float* target_z;
  const float *lse, *weight;
  void* ds;                  // [part][n][ds_stride]
  long long ds_stride, ds_part;
  // kGradRows: out[n][m], in the type of the rows or added to fp32 sums
  void* out;
  long long out_stride;
  int out_dtype;             // type of out
  int add;                   // add onto it
  const float* factor;       // null, or what the sums are multiplied with
};

// Which parts of A and B the products of three parts each take, the smallest first.
__device__ constexpr int kPartA[6] = {2, 1, 0, 1, 0, 0}, kPartB[6] = {0, 1, 2, 0, 1, 0};

__device__ __forceinline__ void store_any(void* p, int dtype, long long at, float v, bool add) {
  if (dtype == KAN_F32) ((float*)p)[at] = add ? ((float*)p)[at] + v : v;
  else if (dtype == KAN_F16) ((f16*)p)[at] = (f16)(add ? (float)((f16*)p)[at] + v : v);
  else ((bf16*)p)[at] = (bf16)(add ? (float)((bf16*)p)[at] + v : v);
}

// T: type of the 16-bit operands; AK, BK: their k is contiguous.
template <class T, bool AK, bool BK, int EPI>
__global__ __launch_bounds__(kThreads) void kan_vocab_product_kernel(const ProductArgs g) {
  __shared__ __attribute__((aligned(16))) T sA[kTile][kStep + kPad];
  __shared__ __attribute__((aligned(16))) T sB[kTile][kStep + kPad];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64, lr = lane & 15, lk = lane >> 4;
  const int m0 = blockIdx.x * kTile, n0 = blockIdx.y * kTile;
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto fetch = [&](const Operand& o, int part, int r0, int k0, auto contiguous, T (*dst)[kStep + kPad]) {
    const T* const p = (const T*)o.p + part * o.part;
#pragma unroll 4
    for (int i = 0; i < kTile * kStep / kThreads; ++i) {
      const int e = i * kThreads + tid;
      const int r = decltype(contiguous)::value ? e / kStep : e % kTile, k = decltype(contiguous)::value ? e % kStep : e / kTile;
      const bool in = r0 + r < o.rows && k0 + k < o.depth;
      const long long at = decltype(contiguous)::value ? (long long)(r0 + r) * o.stride + k0 + k : (long long)(k0 + k) * o.stride + r0 + r;
      dst[r][k] = in ? p[at] : (T)0.f;
    }
  };
  const int combos = g.parts == 1 ? 1 : 6;
  for (int q = 0; q < combos; ++q) {
    const int pa = g.parts == 1 ? 0 : kPartA[q], pb = g.parts == 1 ? 0 : kPartB[q];
    for (int k0 = 0; k0 < g.k; k0 += kStep) {
      __syncthreads();
      fetch(g.a, pa, m0, k0, std::integral_constant<bool, AK>{}, sA);
      fetch(g.b, pb, n0, k0, std::integral_constant<bool, BK>{}, sB);
      __syncthreads();
      uint4 fa[4], fb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fa[i] = *(const uint4*)&sA[wm + i * 16 + lr][lk * 8];
        fb[i] = *(const uint4*)&sB[wn + i * 16 + lr][lk * 8];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = mfma<T>(fa[i], fb[j], acc[i][j]);
    }
  }

  // acc[i][j][r]: m = wm + 16 i + 4 lk + r, n = wn + 16 j + lr
  if constexpr (EPI == kStats) {
    __shared__ float2 sStat[2][kTile];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + wn + 16 * j + lr;
      const uint32_t target = n < g.n ? row_of(g.targets, g.id_dtype, n, (uint32_t)g.V) : (uint32_t)g.V;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int v = g.v0 + m0 + wm + 16 * i + 4 * lk + r;
          acc[i][j][r] *= g.scale;
          if (v < g.V) top = fmaxf(top, acc[i][j][r]);
          if ((uint32_t)v == target && v < g.V) g.target_z[n] = acc[i][j][r];
        }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float at = fminf(fmaxf(top, -FLT_MAX), FLT_MAX);      // (finite, so that nothing below subtracts infinities)
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (g.v0 + m0 + wm + 16 * i + 4 * lk + r < g.V) sum += __expf(acc[i][j][r] - at);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (lk == 0) sStat[wave & 1][wn + 16 * j + lr] = make_float2(at, sum);
    }
    __syncthreads();
    if (tid < kTile && n0 + tid < g.n) {
      const float2 x = sStat[0][tid], y = sStat[1][tid];
      const float at = fmaxf(x.x, y.x);
      g.stats[(long long)((g.v0 + m0) / kTile) * g.n + n0 + tid] = make_float2(at, x.y * __expf(x.x - at) + y.y * __expf(y.x - at));
    }
  } else if constexpr (EPI == kGradS) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + wn + 16 * j + lr;
      if (n >= g.n) continue;
      const uint32_t target = row_of(g.targets, g.id_dtype, n, (uint32_t)g.V);
      const float lse = g.lse[n], weight = g.weight[n];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = m0 + wm + 16 * i + 4 * lk + r, v = g.v0 + m;
          if (m >= g.ds_stride) continue;
          float d = 0.f;
          if (v < g.V && target < (uint32_t)g.V) d = (__expf(acc[i][j][r] * g.scale - lse) - ((uint32_t)v == target ? 1.f : 0.f)) * weight;
          T* dst = (T*)g.ds + (long long)n * g.ds_stride + m;
          for (int p = 0; p < g.parts; ++p) {
            const T hi = (T)d;
            dst[p * g.ds_part] = hi;
            d -= (float)hi;
          }
        }
    }
  } else {
    const float factor = g.factor ? *g.factor : 1.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + wn + 16 * j + lr;
      if (n >= g.n) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = m0 + wm + 16 * i + 4 * lk + r;
          if (m < g.m) store_any(g.out, g.out_dtype, (long long)n * g.out_stride + m, acc[i][j][r] * factor, g.add);
        }
    }
  }
}

// Rows in the form the products take: 16-bit parts of `width` columns (zeros behind the last).  With targets: rows whose
// target names no row are zeros, whatever they hold.
template <class I, class T, int PARTS>
__global__ __launch_bounds__(kThreads) void kan_vocab_pack_kernel(const I* __restrict__ src, long long rows, int D, int width, long long part,
                                                                  const void* __restrict__ targets, int id_dtype, uint32_t V, T* __restrict__ dst) {
  const int C = width / 8;
  const long long items = rows * C;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < items; i += (long long)gridDim.x * kThreads) {
    const long long row = i / C;
    const int c = (int)(i - row * C) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < D && (!targets || row_of(targets, id_dtype, row, V) < V)) load_cols(src + row * D, c, D, v);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      store8(dst + p * part + row * width + c, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] -= (float)(T)v[k];
    }
  }
}

// lse and loss of a token from the statistics of the table's tiles.
__global__ __launch_bounds__(256) void kan_vocab_join_kernel(const float2* __restrict__ stats, int tiles, const float* __restrict__ target_z,
                                                             const void* __restrict__ targets, int id_dtype, uint32_t V, int N, float* __restrict__ loss,
                                                             float* __restrict__ lse) {
  // 16 tokens a workgroup, 16 lanes share a token's tiles
  __shared__ float2 sStat[16][16];
  const int at = threadIdx.x & 15, share = threadIdx.x >> 4, n = blockIdx.x * 16 + at;
  float top = -INFINITY, sum = 0.f;
  if (n < N)
    for (int t = share; t < tiles; t += 16) {
      const float2 s = stats[(long long)t * N + n];
      const float m = fmaxf(top, s.x);
      sum = sum * __expf(top - m) + s.y * __expf(s.x - m);
      top = m;
    }
  sStat[share][at] = make_float2(top, sum);
  __syncthreads();
  if (share == 0 && n < N) {
    float m = top;
    for (int k = 1; k < 16; ++k) m = fmaxf(m, sStat[k][at].x);
    float s = 0.f;
    for (int k = 0; k < 16; ++k) s += sStat[k][at].y * __expf(sStat[k][at].x - m);
    const float l = m + __logf(s);
    lse[n] = l;
    loss[n] = row_of(targets, id_dtype, n, V) < V ? l - target_z[n] : 0.f;
  }
}

// Weights of the tokens' gradients; fp16: scaled so that the largest is 2^14, and the factor that takes this back.
__global__ __launch_bounds__(1024) void kan_vocab_weight_kernel(const float* __restrict__ dloss, const void* __restrict__ targets, int id_dtype, uint32_t V,
                                                                long long N, float scale, int half, float* __restrict__ weight, float* __restrict__ factor) {
  __shared__ float sMax[16];
  float mul = scale;
  if (half) {
    float top = 0.f;
    for (long long n = threadIdx.x; n < N; n += 1024)
      if (row_of(targets, id_dtype, n, V) < V) top = fmaxf(top, fabsf(dloss[n]));
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((threadIdx.x & 63) == 0) sMax[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int w = 0; w < 16; ++w) top = fmaxf(top, sMax[w]);
    mul = top > 0.f ? kHalfScale / top : 0.f;
    if (threadIdx.x == 0) *factor = scale * top / kHalfScale;
  }
  for (long long n = threadIdx.x; n < N; n += 1024) weight[n] = row_of(targets, id_dtype, n, V) < V ? dloss[n] * mul : 0.f;
}

__global__ __launch_bounds__(kThreads) void kan_vocab_round_kernel(const float* __restrict__ src, long long n, int dtype, const float* factor, void* __restrict__ dst) {
  const float f = factor ? *factor : 1.f;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) store_any(dst, dtype, i, src[i] * f, false);
}

struct Plan {
  int parts;
  bool pack_table;            // the table's rows go through the workspace
  long long width;            // columns of packed rows
  int piece, pieces;          // rows of the table that are dealt with at a time
  size_t h, table, stats, target_z, weight, factor, ds, dh, bytes;
};

Plan make_plan(long long N, int V, int D, int dtype, bool backward) {
  Plan p = {};
  p.parts = dtype == KAN_F32 ? 3 : 1;
  p.pack_table = p.parts > 1 || D % 8 != 0;
  p.width = ((long long)D + 63) / 64 * 64;
  const long long all = ((long long)V + kVocabStep - 1) / kVocabStep * kVocabStep;
  long long piece = all;
  auto limit = [&](long long budget, long long row_bytes) { piece = std::min(piece, std::max(1ll, budget / (row_bytes * kVocabStep)) * kVocabStep); };
  if (p.pack_table) limit(kPackBytes, p.parts * p.width * 2);
  if (backward) limit(kPieceBytes, p.parts * N * 2);
  p.piece = (int)std::min(piece, (long long)INT32_MAX / kVocabStep * kVocabStep);
  p.pieces = (int)((V + (long long)p.piece - 1) / p.piece);
  size_t at = 0;
  auto take = [&](long long bytes) {
    const size_t was = at;
    at += (size_t)(bytes + 255) / 256 * 256;
    return was;
  };
  p.h = take(backward || p.pack_table ? p.parts * N * p.width * 2 : 0);
  p.table = take(p.pack_table ? p.parts * (long long)p.piece * p.width * 2 : 0);
  p.stats = take(backward ? 0 : (all / kTile) * N * 8);
  p.target_z = take(backward ? 0 : N * 4);
  p.weight = take(backward ? N * 4 : 0);
  p.factor = take(backward ? 4 : 0);
  p.ds = take(backward ? p.parts * N * (long long)p.piece * 2 : 0);
  p.dh = take(backward && (p.pieces > 1) ? N * D * 4ll : 0);
  p.bytes = at;
  return p;
}

template <class T, bool AK, bool BK, int EPI>
hipError_t launch_product(const ProductArgs& g, hipStream_t s) {
  const dim3 grid((unsigned)((g.m + kTile - 1) / kTile), (unsigned)((g.n + kTile - 1) / kTile));
  hipLaunchKernelGGL((kan_vocab_product_kernel<T, AK, BK, EPI>), grid, dim3(kThreads), 0, s, g);
  return hipGetLastError();
}

hipError_t pack(const void* src, long long rows, int D, long long width, int dtype, const void* targets, int id_dtype, int V, void* dst, hipStream_t s) {
  const long long items = rows * (width / 8);
  const dim3 grid((unsigned)std::min((items + kThreads - 1) / kThreads, 1ll << 16));
  const long long part = rows * width;
  if (dtype == KAN_F32)
    hipLaunchKernelGGL((kan_vocab_pack_kernel<float, bf16, 3>), grid, dim3(kThreads), 0, s, (const float*)src, rows, D, (int)width, part, targets, id_dtype,
                       (uint32_t)V, (bf16*)dst);
  else if (dtype == KAN_F16)
    hipLaunchKernelGGL((kan_vocab_pack_kernel<f16, f16, 1>), grid, dim3(kThreads), 0, s, (const f16*)src, rows, D, (int)width, part, targets, id_dtype,
                       (uint32_t)V, (f16*)dst);
  else
    hipLaunchKernelGGL((kan_vocab_pack_kernel<bf16, bf16, 1>), grid, dim3(kThreads), 0, s, (const bf16*)src, rows, D, (int)width, part, targets, id_dtype,
                       (uint32_t)V, (bf16*)dst);
  return hipGetLastError();
}

// f(T{}): the type of the 16-bit operands.
template <class F>
kan_status with_operand(int dtype, F&& f) {
  if (dtype == KAN_F16) return f(f16{});
  return f(bf16{});
}

// The rows of the table from v0 on as an operand whose k is the width.
kan_status table_rows(const VocabArgs& a, const Plan& p, unsigned char* ws, int v0, int rows, Operand* out, hipStream_t s) {
  const char* const src = (const char*)a.table + (long long)v0 * a.D * float_bytes(a.dtype);
  if (!p.pack_table) {
    *out = {src, a.D, 0, rows, a.D};
    return KAN_OK;
  }
  *out = {ws + p.table, p.width, rows * p.width, rows, a.D};
  return run_named("kan_vocab_pack", s, [&] { return pack(src, rows, a.D, p.width, a.dtype, nullptr, 0, 0, ws + p.table, s); });
}

}  // namespace

size_t vocab_workspace(long long N, int V, int D, int dtype, bool backward) { return N == 0 ? 0 : make_plan(N, V, D, dtype, backward).bytes; }

kan_status run_vocab_loss(const VocabArgs& a, hipStream_t s) {
  const Plan p = make_plan(a.N, a.V, a.D, a.dtype, false);
  unsigned char* const ws = (unsigned char*)a.ws;
  return with_operand(a.dtype, [&](auto t) -> kan_status {
    typedef decltype(t) T;
    ProductArgs g = {};
    g.n = (int)a.N;
    g.k = a.D;
    g.parts = p.parts;
    g.V = a.V;
    g.scale = a.scale;
    g.targets = a.targets;
    g.id_dtype = a.id_dtype;
    g.stats = (float2*)(ws + p.stats);
    g.target_z = (float*)(ws + p.target_z);
    kan_status st;
    g.b = {a.h, a.D, 0, (int)a.N, a.D};
    if (p.pack_table) {
      st = run_named("kan_vocab_pack", s, [&] { return pack(a.h, a.N, a.D, p.width, a.dtype, nullptr, 0, 0, ws + p.h, s); });
      if (st != KAN_OK) return st;
      g.b = {ws + p.h, p.width, a.N * p.width, (int)a.N, a.D};
    }
    for (int v0 = 0, i = 0; i < p.pieces; ++i, v0 += p.piece) {
      g.v0 = v0;
      g.m = std::min(p.piece, a.V - v0);
      if ((st = table_rows(a, p, ws, v0, g.m, &g.a, s)) != KAN_OK) return st;
      st = run_named("kan_vocab_loss", s, [&] { return launch_product<T, true, true, kStats>(g, s); });
      if (st != KAN_OK) return st;
    }
    return run_named("kan_vocab_join", s, [&] {
      hipLaunchKernelGGL(kan_vocab_join_kernel, dim3((unsigned)((a.N + 15) / 16)), dim3(256), 0, s, g.stats, (a.V + kTile - 1) / kTile, g.target_z, a.targets,
                         a.id_dtype, (uint32_t)a.V, (int)a.N, a.loss, a.lse);
      return hipGetLastError();
    });
  });
}

kan_status run_vocab_grad(const VocabArgs& a, hipStream_t s) {
  const Plan p = make_plan(a.N, a.V, a.D, a.dtype, true);
  unsigned char* const ws = (unsigned char*)a.ws;
  const int half = a.dtype == KAN_F16;
  float* const factor = half ? (float*)(ws + p.factor) : nullptr;
  return with_operand(a.dtype, [&](auto t) -> kan_status {
    typedef decltype(t) T;
    kan_status st = run_named("kan_vocab_weight", s, [&] {
      hipLaunchKernelGGL(kan_vocab_weight_kernel, dim3(1), dim3(1024), 0, s, a.dloss, a.targets, a.id_dtype, (uint32_t)a.V, a.N, a.scale, half,
                         (float*)(ws + p.weight), factor);
      return hipGetLastError();
    });
    if (st != KAN_OK) return st;
    st = run_named("kan_vocab_pack", s, [&] { return pack(a.h, a.N, a.D, p.width, a.dtype, a.targets, a.id_dtype, a.V, ws + p.h, s); });
    if (st != KAN_OK) return st;
    const Operand h = {ws + p.h, p.width, a.N * p.width, (int)a.N, a.D};
    for (int v0 = 0, i = 0; i < p.pieces; ++i, v0 += p.piece) {
      const int rows = std::min(p.piece, a.V - v0);
      ProductArgs g = {};
      g.parts = p.parts;
      g.v0 = v0;
      g.V = a.V;
      g.scale = a.scale;
      g.targets = a.targets;
      g.id_dtype = a.id_dtype;
      g.lse = a.lse;
      g.weight = (const float*)(ws + p.weight);
      g.ds = ws + p.ds;
      g.ds_stride = p.piece;
      g.ds_part = a.N * (long long)p.piece;
      g.m = rows;
      g.n = (int)a.N;
      g.k = a.D;
      Operand table;
      if ((st = table_rows(a, p, ws, v0, rows, &table, s)) != KAN_OK) return st;
      g.a = table;
      g.b = h;
      st = run_named("kan_vocab_ds", s, [&] { return launch_product<T, true, true, kGradS>(g, s); });
      if (st != KAN_OK) return st;
      // dh (+)= dS T: k = rows of the piece
      const bool direct = p.pieces == 1;
      g.m = a.D;
      g.k = rows;
      g.a = {table.p, table.stride, table.part, a.D, rows};
      g.b = {ws + p.ds, p.piece, g.ds_part, (int)a.N, rows};
      g.out = direct ? a.dh : (void*)(ws + p.dh);
      g.out_stride = a.D;
      g.out_dtype = direct ? a.dtype : KAN_F32;
      g.add = i > 0;
      g.factor = direct ? factor : nullptr;
      st = run_named("kan_vocab_dh", s, [&] { return launch_product<T, false, true, kGradRows>(g, s); });
      if (st != KAN_OK) return st;
      // dT (+)= dS^t h: k = tokens
      g.n = rows;
      g.k = (int)a.N;
      g.a = {h.p, h.stride, h.part, a.D, (int)a.N};
      g.b = {ws + p.ds, p.piece, g.ds_part, rows, (int)a.N};
      g.out = (char*)a.dtable + (long long)v0 * a.D * float_bytes(a.dtype);
      g.out_dtype = a.dtype;
      g.add = a.accumulate;
      g.factor = factor;
      st = run_named("kan_vocab_dtable", s, [&] { return launch_product<T, false, false, kGradRows>(g, s); });
      if (st != KAN_OK) return st;
    }
    if (p.pieces == 1) return KAN_OK;
    return run_named("kan_vocab_round", s, [&] {
      const long long n = a.N * a.D;
      hipLaunchKernelGGL(kan_vocab_round_kernel, dim3((unsigned)std::min((n + kThreads - 1) / kThreads, 1ll << 14)), dim3(kThreads), 0, s,
                         (const float*)(ws + p.dh), n, a.dtype, factor, a.dh);
      return hipGetLastError();
    });
  });
}

}  // namespace kan

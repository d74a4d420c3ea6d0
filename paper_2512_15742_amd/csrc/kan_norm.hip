// The norm in front of a block and the norm behind it, with gate and residual scale, in one pass over the residual stream.
//
//   y = x + scale * sigma(gate) * w_after * v * rv,   rv = 1 / sqrt(mean(v^2) + eps)     (v: the block's output)
//   u = w_before * y * ry,                            ry = 1 / sqrt(mean(y^2) + eps)     (u: the next block's input)
//
// Backward, from y, v, gate and the gradients dy, du (t = du w_before, m = v rv, s = sigma(gate)):
//   gy = dy + ry (t - y ry mean(t y ry))                       = dx, the gradient of the stream in front of the block
//   q  = scale s gy w_after,   dv = rv (q - m mean(q m)),   dgate = scale gy w_after m sigma(gate) sigma(-gate)
//   dw_before = sum du y ry,   dw_after = sum scale s gy m     (over the tokens)
//
// Bound by the bytes of the rows: each is read once, a row stays in the registers of one to sixteen waves, eight columns a
// lane at a time (8192 rows of 2048 in bf16 with fp32 blocks and gates forward 49 us, 5.4 TB/s; of 4096 in bf16 backward 111 us,
// 4.8 TB/s; a large copy reaches 5.1).  Norms, means and the sums of the weights' gradients are fp32; means are sums times a rounded 1 / D,
// roots and sigma the hardware's (exact division and roots left the same errors, of 7e-8 to 1.2e-7 in fp32).  The u of the forward pass is
// formed from the fp32 y, not from its rounded copy.  Backward: up to 512 groups of waves (2,048 for up to 512 columns) take rows in turn and keep
// the sums of their rows' weight gradients; a second launch adds the groups' sums in a fixed order.  Where a lane has sixteen columns
// (backward: widths that are no multiple of eight above 4,089, all above 8,192) some of that lies in scratch memory.
#include <algorithm>
#include <type_traits>

#include "kan_tokens.hpp"

namespace kan {
namespace {

constexpr int kMaxGroups = 512;         // groups of waves of a backward launch (of wide rows), each with a partial sum of the weights' gradients
constexpr int kMaxBlocks = 1 << 20;     // workgroups of a forward launch: they take rows in turn
constexpr int kReduceThreads = 1024;    // 16 columns, 64 shares of the groups

// Rows whose width is no multiple of eight: a lane's eight columns begin where row n's place in the array is one, so that all
// its accesses are aligned; those in front of the row (c < 0) and behind it are left out.
// WHOLE: widths that are multiples of eight, no lane has a part of eight columns.
template <bool WHOLE, int COLS>      // columns that the lanes have
__device__ __forceinline__ int first_shift(long long n, int D) { return !WHOLE && D + 7 <= COLS ? (int)((n * D) & 7) : 0; }
template <bool WHOLE>
__device__ __forceinline__ bool within(int c, int D) { return WHOLE || (c >= 0 && c + 8 <= D); }
// room: elements from the row's first to the array's end.  A part of eight columns is read with its neighbours in other rows,
// which are then left out; only at the array's end it is read one by one (rows of fewer than eight columns may begin in it).
template <bool WHOLE, class T>
__device__ __forceinline__ void load_part(const T* row, int c, int D, long long room, float (&out)[8]) {
  if (WHOLE || c + 8 <= room) {
    load8(row + c, out);
    if (!within<WHOLE>(c, D))
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] = c + i >= 0 && c + i < D ? out[i] : 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = c + i >= 0 && c + i < D ? (float)row[c + i] : 0.f;
  }
}
template <bool WHOLE, class T>
__device__ __forceinline__ void load_vector(const T* w, int c, int D, float (&out)[8]) {
  if (within<WHOLE>(c, D)) {
    load8(w + c, out);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = c + i >= 0 && c + i < D ? (float)w[c + i] : 0.f;
  }
}
template <bool WHOLE, class T>
__device__ __forceinline__ void store_part(T* row, int c, int D, const float (&in)[8]) {
  if (within<WHOLE>(c, D)) {
    store8(row + c, in);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i >= 0 && c + i < D) row[c + i] = (T)in[i];
  }
}

template <bool WHOLE>
__device__ __forceinline__ void load_weight(const void* w, int dtype, int c, int D, float (&out)[8]) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = 1.f;
  } else if (dtype == KAN_F32) {
    load_vector<WHOLE>((const float*)w, c, D, out);
  } else if (dtype == KAN_F16) {
    load_vector<WHOLE>((const f16*)w, c, D, out);
  } else {
    load_vector<WHOLE>((const bf16*)w, c, D, out);
  }
}

// Sums of K values over the W waves of a row, the same in every lane.  The scratch has to be another one than that of the call
// before: the barrier here is then the only one, since nobody passes the next call's before everybody has read this one's.
template <int W, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*scratch)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v[k] += __shfl_xor(v[k], d);
  if constexpr (W > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) scratch[wave][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += scratch[w][k];
      v[k] = s;
    }
  }
}

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
// sigma(z) and its derivative sigma(z) sigma(-z): both from e^-|z|, so that nothing cancels (1 - sigma(z) is 0 from z = 17 on).
__device__ __forceinline__ void sigmoid_and_slope(float z, float& s, float& slope) {
  const float e = __expf(-fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + e), least = e * r;       // least: the smaller of sigma(z), sigma(-z)
  s = z < 0.f ? least : r;
  slope = fmaf(-least, least, least);
}

// W waves a row, W == 1: four rows a workgroup.
template <class S, class B, int W, int P, bool WHOLE>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void kan_norm_kernel(const NormArgs a) {
  __shared__ float sSum[2][2][W][1];
  const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int D = a.D;
  const float inv = 1.f / (float)D;
  const long long rows = (long long)gridDim.x * (W == 1 ? 4 : 1);
  int odd = 0;       // (each row has one or two sums: the scratch of a row is another one than that of the row before)
  for (long long n = W == 1 ? (long long)blockIdx.x * 4 + (threadIdx.x >> 6) : (long long)blockIdx.x; n < a.N; n += rows, odd ^= 1) {
    float x[P][8], v[P][8], g[P][8], w[P][8];
    const int shift = first_shift<WHOLE, 512 * W * P>(n, D);
    const long long room = (a.N - n) * D;
  #pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * 64 * W + t) * 8 - shift;
  #pragma unroll
      for (int i = 0; i < 8; ++i) x[p][i] = v[p][i] = g[p][i] = 0.f;
      if (c < D) {
        load_part<WHOLE>((const S*)a.x + n * D, c, D, room, x[p]);
        if (a.v) {
          load_part<WHOLE>((const B*)a.v + n * D, c, D, room, v[p]);
          if (a.gate) load_part<WHOLE>((const B*)a.gate + n * D, c, D, room, g[p]);
          load_weight<WHOLE>(a.w_after, a.weight_dtype, c, D, w[p]);
        }
      }
    }
    if (a.v) {
      float ss[1] = {0.f};
  #pragma unroll
      for (int p = 0; p < P; ++p)
  #pragma unroll
        for (int i = 0; i < 8; ++i) ss[0] += v[p][i] * v[p][i];
      row_sums<W, 1>(ss, sSum[odd][0]);
      const float r = a.scale * rsqrtf(ss[0] * inv + a.eps);
  #pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * 64 * W + t) * 8 - shift;
        if (c < D) {
  #pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float s = a.gate ? sigmoid(g[p][i]) : 1.f;
            x[p][i] += s * (w[p][i] * (v[p][i] * r));
          }
          store_part<WHOLE>((S*)a.y + n * D, c, D, x[p]);
          if (!within<WHOLE>(c, D))
  #pragma unroll
            for (int i = 0; i < 8; ++i)
              if (c + i < 0 || c + i >= D) x[p][i] = 0.f;
        }
      }
    }
    if (a.u) {
      float ss[1] = {0.f};
  #pragma unroll
      for (int p = 0; p < P; ++p)
  #pragma unroll
        for (int i = 0; i < 8; ++i) ss[0] += x[p][i] * x[p][i];
      row_sums<W, 1>(ss, sSum[odd][1]);
      const float r = rsqrtf(ss[0] * inv + a.eps);
  #pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * 64 * W + t) * 8 - shift;
        if (c < D) {
          load_weight<WHOLE>(a.w_before, a.weight_dtype, c, D, w[p]);
  #pragma unroll
          for (int i = 0; i < 8; ++i) x[p][i] = w[p][i] * (x[p][i] * r);
          store_part<WHOLE>((B*)a.u + n * D, c, D, x[p]);
        }
      }
    }
  }
}

// Eight columns of a row as they lie in memory; zeros past its end.
template <class T>
struct Raw {
  typedef T V8 __attribute__((ext_vector_type(8)));
  V8 v;
  template <bool WHOLE>
  __device__ __forceinline__ void load(const void* row, int c, int D, long long room) {      // (as load_part)
    const T* const p = (const T*)row + c;
    if (WHOLE || c + 8 <= room) {
      __builtin_memcpy(&v, p, sizeof(v));
      if (!within<WHOLE>(c, D))
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i >= 0 && c + i < D ? v[i] : (T)0.f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i >= 0 && c + i < D ? p[i] : (T)0.f;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (T)0.f;
  }
  __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
};

// W waves a row, weights and their sums in registers (P == 1): 128 of them where widths are multiples of eight, so that two rows
// share a CU and the loads of one run beside the sums of the other (8192 rows of 4096 in bf16: 111 us; the next row fetched
// ahead, with 155 registers and one row a CU, 122).
template <class S, class B, int W, int P, bool WHOLE>
__global__ __launch_bounds__(64 * W, P == 1 && WHOLE ? 4 : (W == 16 ? 4 : 2)) void kan_norm_grad_kernel(const NormArgs a, int groups) {
  __shared__ float sSum[2][W][3];
  __shared__ float sSum1[2][W][1];
  const int t = threadIdx.x, group = blockIdx.x, D = a.D;
  const int shift = first_shift<WHOLE, 512 * W * P>(group, D);      // (the same for all rows of the group: it has one, or one of each 512 n)
  static_assert(kMaxGroups % 8 == 0, "");
  const float inv = 1.f / (float)D;
  float sum1[P][8], sum2[P][8], w1[P][8], w2[P][8];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * 64 * W + t) * 8 - shift;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum1[p][i] = sum2[p][i] = w1[p][i] = w2[p][i] = 0.f;
    if (c < D) {
      if (a.du) load_weight<WHOLE>(a.w_before, a.weight_dtype, c, D, w1[p]);
      if (a.v) load_weight<WHOLE>(a.w_after, a.weight_dtype, c, D, w2[p]);
      if (!within<WHOLE>(c, D))
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < 0 || c + i >= D) w1[p][i] = w2[p][i] = 0.f;
    }
  }
  struct Row {
    Raw<S> y[P], dy[P];
    Raw<B> du[P], v[P], g[P];
  };
  auto load = [&](long long n, Row& r) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * 64 * W + t) * 8 - shift;
      r.y[p].clear(), r.dy[p].clear(), r.du[p].clear(), r.v[p].clear(), r.g[p].clear();
      if (c < D) {
        if (a.du) {
          r.y[p].template load<WHOLE>((const S*)a.x + n * D, c, D, (a.N - n) * D);
          r.du[p].template load<WHOLE>((const B*)a.du + n * D, c, D, (a.N - n) * D);
        }
        if (a.dy) r.dy[p].template load<WHOLE>((const S*)a.dy + n * D, c, D, (a.N - n) * D);
        if (a.v) r.v[p].template load<WHOLE>((const B*)a.v + n * D, c, D, (a.N - n) * D);
        if (a.gate) r.g[p].template load<WHOLE>((const B*)a.gate + n * D, c, D, (a.N - n) * D);
      }
    }
  };
  auto work = [&](long long n, const Row& r, int odd) {
    float ss[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss[0] += r.y[p][i] * r.y[p][i];
        ss[1] += r.du[p][i] * w1[p][i] * r.y[p][i];
        ss[2] += r.v[p][i] * r.v[p][i];
      }
    row_sums<W, 3>(ss, sSum[odd]);
    const float ry = rsqrtf(ss[0] * inv + a.eps), rv = rsqrtf(ss[2] * inv + a.eps), mean = ss[1] * ry * inv;
    float sq[1] = {0.f}, q[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * 64 * W + t) * 8 - shift;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        q[p][i] = r.dy[p][i];
        if (a.du) {
          const float hat = r.y[p][i] * ry;
          sum1[p][i] += r.du[p][i] * hat;
          q[p][i] += ry * (r.du[p][i] * w1[p][i] - hat * mean);
        }
      }
      if (c < D) store_part<WHOLE>((S*)a.dx + n * D, c, D, q[p]);
      if (a.v) {
        float dg[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float s = 1.f, slope = 0.f;
          if (a.gate) sigmoid_and_slope(r.g[p][i], s, slope);
          const float m = r.v[p][i] * rv, e = a.scale * q[p][i];
          sum2[p][i] += s * e * m;
          dg[i] = e * (w2[p][i] * m) * slope;
          q[p][i] = s * e * w2[p][i];
          sq[0] += q[p][i] * m;
        }
        if (a.gate && c < D) store_part<WHOLE>((B*)a.dgate + n * D, c, D, dg);
      }
    }
    if (a.v) {
      row_sums<W, 1>(sq, sSum1[odd]);
      const float qm = sq[0] * inv;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int c = (p * 64 * W + t) * 8 - shift;
#pragma unroll
        for (int i = 0; i < 8; ++i) q[p][i] = rv * (q[p][i] - r.v[p][i] * rv * qm);
        if (c < D) store_part<WHOLE>((B*)a.dv + n * D, c, D, q[p]);
      }
    }
  };
  for (long long n = group, odd = 0; n < a.N; n += groups, odd ^= 1) {
    Row r;
    load(n, r);
    work(n, r, (int)odd);
  }
  // sums[0]: w_before, then w_after, as far as they are asked for
  float* dst = a.partial + (long long)group * D;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c = (p * 64 * W + t) * 8 - shift;
    if (c < D) {
      if (a.dw_before) store_part<WHOLE>(dst, c, D, sum1[p]);
      if (a.dw_after) store_part<WHOLE>(dst + (a.dw_before ? (long long)groups * D : 0), c, D, sum2[p]);
    }
  }
}

// Sum in a tree: log2(K) roundings one behind the other in place of K.
template <int K>
__device__ __forceinline__ float tree_sum(float (&v)[K]) {
#pragma unroll
  for (int d = K / 2; d >= 1; d /= 2)
#pragma unroll
    for (int k = 0; k < d; ++k) v[k] += v[k + d];
  return v[0];
}

// 16 columns a workgroup, 64 shares of the groups.
__global__ __launch_bounds__(kReduceThreads) void kan_norm_reduce_kernel(const float* __restrict__ partial, int groups, int D, void* first, void* second,
                                                                         int dtype) {
  __shared__ float sSum[64][17];
  const int lane = threadIdx.x & 15, share = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
  const float* const src = partial + (long long)blockIdx.y * groups * D;
  float s = 0.f;
  if (c < D) {
    for (int r = share; r < groups; r += 8 * 64) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = r + u * 64 < groups ? src[(long long)(r + u * 64) * D + c] : 0.f;
      s += tree_sum(v);
    }
  }
  sSum[share][lane] = s;
  __syncthreads();
  if (share == 0 && c < D) {
    float v[64];
#pragma unroll
    for (int k = 0; k < 64; ++k) v[k] = sSum[k][lane];
    s = tree_sum(v);
    void* const out = blockIdx.y == 0 ? first : second;
    if (dtype == KAN_F32) ((float*)out)[c] = s;
    else if (dtype == KAN_F16) ((f16*)out)[c] = (f16)s;
    else ((bf16*)out)[c] = (bf16)s;
  }
}

// f(W, P): waves per row and groups of eight columns a lane.  Backward a row takes more registers, and more waves.
template <bool GRAD, class F>
hipError_t with_shape(int D, F&& f) {
  const int cols = D + (D % 8 ? 7 : 0);
#define KAN_SHAPE(W, P) if (cols <= 512 * W * P) return f(std::integral_constant<int, W>{}, std::integral_constant<int, P>{})
  KAN_SHAPE(1, 1);
  if constexpr (GRAD) {
    KAN_SHAPE(2, 1);
    KAN_SHAPE(4, 1);
    KAN_SHAPE(8, 1);
  } else {
    KAN_SHAPE(1, 2);
    KAN_SHAPE(4, 1);
    KAN_SHAPE(4, 2);
  }
  KAN_SHAPE(8, 2);
  return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
#undef KAN_SHAPE
}

// f(S{}, B{}): the block's type is the stream's, or fp32.
template <class F>
hipError_t with_types(int stream, int block, F&& f) {
  return with_float(stream, [&](auto s) {
    if (block == stream) return f(s, s);
    return f(s, float{});
  });
}

// (rows of up to 512 columns have a wave each: more groups, so that a CU has eight of them; 4000 x 333 36 -> 22 us.  1024 groups
// of two waves lose on the partial sums: 999 x 1000 14 -> 17 us)
int grad_groups(long long N, int D) { return (int)std::min((long long)kMaxGroups * (D <= 512 ? 4 : 1), N); }

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  return with_types(a.stream_dtype, a.block_dtype, [&](auto st, auto bl) {
    typedef decltype(st) S;
    typedef decltype(bl) B;
    return with_shape<false>(a.D, [&](auto w, auto p) {
      constexpr int W = decltype(w)::value, P = decltype(p)::value;
      const long long blocks = std::min(W == 1 ? (a.N + 3) / 4 : a.N, (long long)kMaxBlocks);
      if (a.D % 8 == 0) hipLaunchKernelGGL((kan_norm_kernel<S, B, W, P, true>), dim3((unsigned)blocks), dim3(W == 1 ? 256 : 64 * W), 0, s, a);
      else hipLaunchKernelGGL((kan_norm_kernel<S, B, W, P, false>), dim3((unsigned)blocks), dim3(W == 1 ? 256 : 64 * W), 0, s, a);
      return hipGetLastError();
    });
  });
}

size_t norm_grad_workspace(int D, long long N, int sums) {
  return ((size_t)sums * grad_groups(N, D) * D * 4 + 255) / 256 * 256;
}

kan_status run_norm_grad(const NormArgs& a, hipStream_t s) {
  const int groups = grad_groups(a.N, a.D);
  kan_status st = KAN_OK;
  if (groups > 0) st = run_named("kan_norm_grad", s, [&] {
    return with_types(a.stream_dtype, a.block_dtype, [&](auto str, auto bl) {
      typedef decltype(str) S;
      typedef decltype(bl) B;
      return with_shape<true>(a.D, [&](auto w, auto p) {
        constexpr int W = decltype(w)::value, P = decltype(p)::value;
        if (a.D % 8 == 0) hipLaunchKernelGGL((kan_norm_grad_kernel<S, B, W, P, true>), dim3(groups), dim3(64 * W), 0, s, a, groups);
        else hipLaunchKernelGGL((kan_norm_grad_kernel<S, B, W, P, false>), dim3(groups), dim3(64 * W), 0, s, a, groups);
        return hipGetLastError();
      });
    });
  });
  const int sums = (a.dw_before ? 1 : 0) + (a.dw_after ? 1 : 0);
  if (st != KAN_OK || sums == 0) return st;
  return run_named("kan_norm_reduce", s, [&] {
    hipLaunchKernelGGL(kan_norm_reduce_kernel, dim3((a.D + 15) / 16, sums), dim3(kReduceThreads), 0, s, a.partial, groups, a.D,
                       a.dw_before ? a.dw_before : a.dw_after, a.dw_after, a.weight_dtype);
    return hipGetLastError();
  });
}

}  // namespace kan

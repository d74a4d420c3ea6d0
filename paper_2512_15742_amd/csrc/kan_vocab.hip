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
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kStep = 32;               // products along the contraction per step
constexpr int kTile = 256;              // results of a workgroup in either direction
constexpr int kSlots = 4;               // steps whose operands LDS holds
constexpr int kVocabStep = 256;         // pieces of the table are multiples of it
constexpr long long kPackBytes = 256ll << 20, kPieceBytes = 512ll << 20;

constexpr float kHalfScale = 16384.f;   // of fp16 dS

template <class T>
__device__ __forceinline__ f32x16 mfma(uint4 a, uint4 b, f32x16 c) {
  if constexpr (std::is_same<T, f16>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// An operand of a product out[n][m] = sum_k A(m, k) B(n, k): element (r, k) at p[r * stride + k], or at p[k * stride + r];
// the rows and k of it that exist (k contiguous: a multiple of 8).  Parts lie `part` elements apart.
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

__device__ __forceinline__ void store_any(void* p, int dtype, long long at, float v, bool add) {
  if (dtype == KAN_F32) ((float*)p)[at] = add ? ((float*)p)[at] + v : v;
  else if (dtype == KAN_F16) ((f16*)p)[at] = (f16)(add ? (float)((f16*)p)[at] + v : v);
  else ((bf16*)p)[at] = (bf16)(add ? (float)((bf16*)p)[at] + v : v);
}

// 64 lanes x 16 bytes from the buffer r at each lane's `off` into LDS at `lds`, `lds` + 16, ...; zeros past the buffer's end.
// The compiler does not count these copies: the waits are explicit (copies_done).
__device__ __forceinline__ void copy_to_lds(const u32x4 r, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(r) : "memory", "m0");
}
// All but the newest N of this wave's copies have landed, and its own LDS reads are done.
template <int N>
__device__ __forceinline__ void copies_done() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// Which parts of A and B the six products of three parts each take, the smallest first: two bits a product.
constexpr uint32_t kPartA = 2u | 1u << 2 | 0u << 4 | 1u << 6 | 0u << 8 | 0u << 10;
constexpr uint32_t kPartB = 0u | 1u << 2 | 2u << 4 | 0u << 6 | 1u << 8 | 0u << 10;

// One operand's tile of R rows: a step of it is R x 32 numbers, 64 R bytes of LDS.
//   k contiguous: [row][4 pieces of 8 k], piece c of row r at place c ^ (r >> 1 & 3), so that eight lanes side by side, which
//   read one piece of eight rows, meet eight different groups of four banks;
//   k strided: [k][R / 16 pieces of 16 rows], piece u of row k at place u ^ {0, 2, 5, 7}[k & 3] (R = 64: u ^ (k & 3)): a
//   transposing read takes one piece of four k in 16 lanes, and two neighbouring ones in 32.
// The memory pipeline writes LDS in the order of the lanes, so the places are chosen by what each lane asks for.
template <class T, bool K, int R>
struct Tile {
  static constexpr int kBytes = R * kStep * 2;
  static constexpr int kCopies = kBytes / 4096;        // per wave of four
  static_assert(kBytes % 4096 == 0, "whole copies for each of four waves");
  uint32_t off[kCopies];
  uint32_t chunk;                  // k contiguous: first k of the lane's piece
  const char* base;                // of the tile at k = 0, part 0
  long long step, part;            // bytes
  long long limit;                 // k contiguous: bytes from base to the end of the last row
  uint32_t read;                   // byte of the lane's first fragment read

  __device__ __forceinline__ static uint32_t mix(uint32_t k) { return R == 64 ? k & 3u : (0x7520u >> (4 * (k & 3u))) & 7u; }

  // wave and lane as the copies are dealt, first: this wave's first row within the tile
  __device__ __forceinline__ void init(const Operand& o, int r0, int wave, int lane, int first) {
    const long long row = o.stride * 2;
    part = o.part * 2;
    if constexpr (K) {
      base = (const char*)o.p + (long long)r0 * row;
      step = kStep * 2;
      limit = (long long)(min(o.rows - r0, R) - 1) * row + (long long)o.depth * 2;
      const uint32_t l = lane;
      chunk = (l & 3u) ^ (l >> 3 & 3u);
#pragma unroll
      for (int j = 0; j < kCopies; ++j) off[j] = (uint32_t)((wave * kCopies + j) * 16 + (lane >> 2)) * (uint32_t)row + chunk * 16u;
      chunk *= 8u;
      const uint32_t r = first + (lane & 31);
      read = r * 64u + ((uint32_t)(lane >> 5) ^ (r >> 1 & 3u)) * 16u;
    } else {
      base = (const char*)o.p + (long long)r0 * 2;
      step = kStep * row;
      limit = row;
      chunk = (uint32_t)r0 * 2u;
#pragma unroll
      for (int j = 0; j < kCopies; ++j) {
        const uint32_t u = (uint32_t)(wave * kCopies + j) * 64u + lane, k = u / (R / 8), c = u % (R / 8);
        off[j] = k * (uint32_t)row + (((c >> 1) ^ mix(k)) * 2u + (c & 1u)) * 16u;
      }
      // lane 16 g + i reads four rows at k = 8 (g >> 1) + i / 4, piece first / 16 + (g & 1)
      const uint32_t k = (uint32_t)(lane >> 5) * 8u + (lane >> 2 & 3u);
      read = k * (R * 2u) + ((((uint32_t)first >> 4) + (lane >> 4 & 1u)) ^ mix(k)) * 32u + (lane & 3u) * 8u;
    }
  }
  // The buffer of the next copies: aimed at k = 0 of a part, then moved on a step at a time.
  uint64_t at;
  long long left;                  // bytes from there to the end of the operand
  __device__ __forceinline__ void aim(uint32_t p, int depth) {
    at = (uint64_t)(uintptr_t)base + (uint64_t)p * (uint64_t)part;
    left = K ? limit : (long long)depth * limit - (long long)chunk;
  }
  __device__ __forceinline__ void move() {
    at += (uint64_t)step;
    left -= step;
  }
  __device__ __forceinline__ u32x4 buffer() const {
    u32x4 r = {(uint32_t)at, (uint32_t)(at >> 32), (uint32_t)max(min(left, 0x7fffff00ll), 0ll), 0x00020000u};
    return r;
  }
  __device__ __forceinline__ void copy(const u32x4& r, int j, int wave, uint32_t lds, int k0, int depth) const {
    uint32_t o = off[j];
    if constexpr (K) o = k0 + (int)chunk < depth ? o : 0xfffffff0u;      // (the row behind it is somebody else's)
    copy_to_lds(r, o, lds + (uint32_t)(wave * kCopies + j) * 1024u);
  }
  // Fragment of rows first + 32 b .. + 31, k = 16 h .. 16 h + 15: one read, or its half j of two.
  static constexpr int kReads = K ? 1 : 2;
  __device__ __forceinline__ void fragment(const unsigned char* slot, int b, int h, int j, uint4& f) const {
    if constexpr (K) {
      f = *(const uint4*)(slot + ((read + b * 2048) ^ (h * 32)));
    } else {
      // rows 32 b further: pieces 2 b further, under the same exclusive or (first is a multiple of 32 b's range)
      const uint32_t at = ((read ^ (uint32_t)(b * 64)) + h * (16 * R * 2) + j * (4 * R * 2));
      const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(slot + at));
      const uint2 w = __builtin_bit_cast(uint2, v);
      if (j == 0) f.x = w.x, f.y = w.y;
      else f.z = w.x, f.w = w.y;
    }
  }
};

// Workgroup of four waves: WM x WN of them, each RB x CB blocks of 32 x 32 results.
//
// A step is 32 of the contraction.  LDS holds four of them; the fragments of a step are read into registers while the step
// before is multiplied, and the copies of the fourth next one are sent out, one or two between each two MFMAs.  One barrier
// a step: behind it every wave's copies of step s + 1 have landed and nobody reads slot s % 4 any more.
template <class T, bool AK, bool BK, int EPI, int RB, int CB, int WM, int WN>
__global__ __launch_bounds__(kThreads, 1) void kan_vocab_product_kernel(const ProductArgs g) {
  constexpr int BM = 32 * RB * WM, BN = 32 * CB * WN;
  typedef Tile<T, AK, BM> TA;
  typedef Tile<T, BK, BN> TB;
  constexpr int kSlot = TA::kBytes + TB::kBytes, kCopies = TA::kCopies + TB::kCopies;
  __shared__ __attribute__((aligned(1024))) unsigned char sRing[kSlots * kSlot];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ln = lane & 31, lh = lane >> 5;
  const int wm = (wave % WM) * 32 * RB, wn = (wave / WM) * 32 * CB;
  // Runs of consecutive work items per XCD; eight tiles of n by as many of m as it has workgroups.
  int mt, nt;
  {
    const unsigned W = gridDim.x, L = blockIdx.x, xcd = L & 7u, q = W >> 3, r = W & 7u;
    const unsigned item = xcd * q + min(xcd, r) + (L >> 3);
    const unsigned nmt = (unsigned)(g.m + BM - 1) / BM, nnt = (unsigned)(g.n + BN - 1) / BN;
    const unsigned group = item / (8 * nmt), first = group * 8, width = min(8u, nnt - first), in = item - first * nmt;
    mt = (int)(in / width);
    nt = (int)(first + in % width);
  }
  const int m0 = mt * BM, n0 = nt * BN;
  TA A;
  TB B;
  A.init(g.a, m0, wave, lane, wm);
  B.init(g.b, n0, wave, lane, wn);
  const int depth_a = g.a.depth, depth_b = g.b.depth;
  const int ksteps = (g.k + kStep - 1) / kStep, total = g.parts == 1 ? ksteps : 6 * ksteps;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)sRing;

  // The next copies: product of parts, k, slot.  Past the last one everything is behind the buffers' ends.
  int cq = 0, ck = 0, cs = 0;
  u32x4 ra, rb;
  A.aim(g.parts == 1 ? 0u : kPartA & 3u, depth_a);
  B.aim(g.parts == 1 ? 0u : kPartB & 3u, depth_b);
  ra = A.buffer();
  rb = B.buffer();
  auto copy = [&](int j) {
    if (j < TA::kCopies) A.copy(ra, j, wave, lds0 + (uint32_t)(cs * kSlot), ck, depth_a);
    else B.copy(rb, j - TA::kCopies, wave, lds0 + (uint32_t)(cs * kSlot + TA::kBytes), ck, depth_b);
  };
  auto next = [&] {
    cs = (cs + 1) & (kSlots - 1);
    ck += kStep;
    A.move();
    B.move();
    if (ck >= g.k) {
      ck = 0;
      ++cq;
      if (g.parts > 1 && cq < 6) {
        A.aim(kPartA >> (2 * cq) & 3u, depth_a);
        B.aim(kPartB >> (2 * cq) & 3u, depth_b);
      } else {
        A.left = B.left = 0;
      }
    }
    ra = A.buffer();
    rb = B.buffer();
  };
  f32x16 acc[RB][CB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
#pragma unroll
    for (int j = 0; j < kCopies; ++j) copy(j);
    next();
  }
  struct Frags {
    uint4 a[2][RB], b[2][CB];
  };
  Frags f[2];
  constexpr int kReadsA = 2 * RB * TA::kReads, kReadsAll = kReadsA + 2 * CB * TB::kReads;
  auto read = [&](const unsigned char* slot, int i, Frags& to) {
    if (i < kReadsA) {
      const int j = i % TA::kReads, b = i / TA::kReads % RB, h = i / TA::kReads / RB;
      A.fragment(slot, b, h, j, to.a[h][b]);
    } else {
      i -= kReadsA;
      const int j = i % TB::kReads, b = i / TB::kReads % CB, h = i / TB::kReads / CB;
      B.fragment(slot + TA::kBytes, b, h, j, to.b[h][b]);
    }
  };
  copies_done<(kSlots - 1) * kCopies>();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int i = 0; i < kReadsAll; ++i) read(sRing, i, f[0]);

  auto step = [&](auto P, int s) {
    constexpr int p = decltype(P)::value, kMfmas = 2 * RB * CB, kSpread = kMfmas > 4 ? kMfmas - 2 : kMfmas;
    copies_done<(kSlots - 2) * kCopies>();
    __builtin_amdgcn_s_barrier();
    const unsigned char* const slot = sRing + ((s + 1) & (kSlots - 1)) * kSlot;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kMfmas; ++i) {
      const int h = i / (RB * CB), a = i / CB % RB, b = i % CB;
      acc[a][b] = mfma<T>(f[p].a[h][a], f[p].b[h][b], acc[a][b]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = i * kReadsAll / kSpread; u < (i + 1) * kReadsAll / kSpread && u < kReadsAll; ++u) read(slot, u, f[p ^ 1]);
#pragma unroll
      for (int u = i * kCopies / kMfmas; u < (i + 1) * kCopies / kMfmas; ++u) copy(u);
      __builtin_amdgcn_sched_barrier(0);
    }
    next();
  };
  int s = 0;
  for (; s + 2 <= total; s += 2) {
    step(std::integral_constant<int, 0>{}, s);
    step(std::integral_constant<int, 1>{}, s + 1);
  }
  if (s < total) step(std::integral_constant<int, 0>{}, s);
  copies_done<0>();
  __syncthreads();

  // acc[i][j][r]: m = wm + 32 i + 8 (r / 4) + 4 lh + r % 4, n = wn + 32 j + ln
  if constexpr (EPI == kStats) {
    float2* const sStat = (float2*)sRing;         // [WM][BN]
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      const int n = n0 + wn + 32 * j + ln;
      const uint32_t target = n < g.n ? row_of(g.targets, g.id_dtype, n, (uint32_t)g.V) : (uint32_t)g.V;
      // The lane's place of the target's row: 16 i + r of those above, or none.
      const uint32_t at_row = target - (uint32_t)(g.v0 + m0 + wm);
      const uint32_t mine = target < (uint32_t)g.V && at_row < 32u * RB && (at_row >> 2 & 1u) == (uint32_t)lh
                                ? (at_row >> 5) * 16u + (at_row >> 3 & 3u) * 4u + (at_row & 3u) : 0xffffu;
      int rows = g.V - (g.v0 + m0 + wm + 4 * lh);
      asm volatile("" : "+v"(rows));       // (compared anew: 64 masks kept for all j would not fit the scalar registers)
      float top = -INFINITY, target_z = 0.f;
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float z = acc[i][j][r] * g.scale;
          target_z = mine == (uint32_t)(16 * i + r) ? z : target_z;
          z = 32 * i + 8 * (r >> 2) + (r & 3) < rows ? z : -INFINITY;
          top = fmaxf(top, z);
          acc[i][j][r] = z;
        }
      if (mine != 0xffffu) g.target_z[n] = target_z;
      top = fmaxf(top, __shfl_xor(top, 32));
      const float at = fminf(fmaxf(top, -FLT_MAX), FLT_MAX);      // (finite, so that nothing below subtracts infinities)
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += __expf(acc[i][j][r] - at);
      sum += __shfl_xor(sum, 32);
      if (lh == 0) sStat[(wave % WM) * BN + wn + 32 * j + ln] = make_float2(at, sum);
    }
    __syncthreads();
    for (int c = tid; c < BN; c += kThreads)
      if (n0 + c < g.n) {
        float at = sStat[c].x, sum = 0.f;
#pragma unroll
        for (int w = 1; w < WM; ++w) at = fmaxf(at, sStat[w * BN + c].x);
#pragma unroll
        for (int w = 0; w < WM; ++w) sum += sStat[w * BN + c].y * __expf(sStat[w * BN + c].x - at);
        g.stats[(long long)((g.v0 + m0) / BM) * g.n + n0 + c] = make_float2(at, sum);
      }
  } else if constexpr (EPI == kGradS) {
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      const int n = n0 + wn + 32 * j + ln;
      if (n >= g.n) continue;
      const uint32_t target = row_of(g.targets, g.id_dtype, n, (uint32_t)g.V);
      const float lse = g.lse[n], weight = g.weight[n];
      const bool named = target < (uint32_t)g.V;
      const int m_first = m0 + wm + 4 * lh;
      int rows = named ? g.V - (g.v0 + m_first) : 0, hit = named ? (int)(target - (uint32_t)(g.v0 + m_first)) : -1;
      asm volatile("" : "+v"(rows), "+v"(hit));
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int m = m_first + 32 * i + 8 * q;
          if (m >= g.ds_stride) continue;
          float d[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int at = 32 * i + 8 * q + r;
            const float p = __expf(acc[i][j][4 * q + r] * g.scale - lse);
            d[r] = at < rows ? (at == hit ? p - 1.f : p) * weight : 0.f;
          }
          T* dst = (T*)g.ds + (long long)n * g.ds_stride + m;
          for (int p = 0; p < g.parts; ++p) {
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 t;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              t[r] = (T)d[r];
              d[r] -= (float)t[r];
            }
            *(T4*)(dst + p * g.ds_part) = t;
          }
        }
    }
  } else {
    const float factor = g.factor ? *g.factor : 1.f;
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      const int n = n0 + wn + 32 * j + ln;
      if (n >= g.n) continue;
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int m = m0 + wm + 32 * i + 8 * (r >> 2) + 4 * lh + (r & 3);
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
  const long long tiles = (long long)((g.m + kTile - 1) / kTile) * ((g.n + kTile - 1) / kTile);
  hipLaunchKernelGGL((kan_vocab_product_kernel<T, AK, BK, EPI, 4, 4, 2, 2>), dim3((unsigned)tiles), dim3(kThreads), 0, s, g);
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
  *out = {ws + p.table, p.width, rows * p.width, rows, (int)p.width};
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
    g.b = {a.h, a.D, 0, (int)a.N, a.D};      // (packed rows: zeros up to the next multiple of 64)
    if (p.pack_table) {
      st = run_named("kan_vocab_pack", s, [&] { return pack(a.h, a.N, a.D, p.width, a.dtype, nullptr, 0, 0, ws + p.h, s); });
      if (st != KAN_OK) return st;
      g.b = {ws + p.h, p.width, a.N * p.width, (int)a.N, (int)p.width};
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
    const Operand h = {ws + p.h, p.width, a.N * p.width, (int)a.N, (int)p.width};
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
      g.b = {ws + p.ds, p.piece, g.ds_part, (int)a.N, (rows + 7) / 8 * 8};      // (zeros behind the last row)
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

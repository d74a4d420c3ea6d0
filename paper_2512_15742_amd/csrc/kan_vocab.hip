// Softmax cross entropy of rows against a table of outputs, without the logits, and its gradients.
//
//   z[n][v] = scale <h_n, T_v>,   lse_n = log sum_v exp z[n][v],   loss_n = lse_n - z[n][t_n]     (t_n names no row: 0)
//   dS[n][v] = scale dloss_n (exp(z[n][v] - lse_n) - [v == t_n])   (t_n names no row: 0)
//   dh = dS T,   dT (+)= dS^t h
//
// Forward: tiles of z stay in registers; each leaves the maximum and the sum of exponentials of its part of a row, which a
// small launch joins.  Backward: piece by piece of the table (z formed once more: dS of 8,192 x 131,072 tokens and rows would
// be 2.1 GB, pieces of 256 MiB, of each part, take 1.5 % longer than all of it), dS of the piece in the workspace, and two products with it.
// All products run on the matrix cores with fp32 sums.
//
// Operands are 16-bit numbers.  fp32 rows travel as three bf16 parts (24 bits together; of the nine products of parts the three
// that are at most 2^-24 of the whole are left out), so a product is six of parts.  dS of 16-bit types is rounded to the type (at
// most 2^-8 or 2^-11 of each entry, the step of the gradients themselves).  It is held in units of max |dloss|, so that the equal
// weights of a mean are not all off by the same rounding (1/255 by 2^-8.01, and all gradients with it); fp16 in 2^-14 of that, so that
// probabilities down to 4e-9 keep all bits.
//
// Bound: few tokens by the bytes of the table (one token x 65,536 x 2,048 in bf16 51 us, 5.3 TB/s); many by the matrix cores and
// the power that they draw (8,192 x 131,072 x 2,048: the loss 3.6 ms, 1.21 PFLOP/s; loss and gradients 15.0 ms, 1.17 PFLOP/s over
// four products; the clock falls to 1.7 GHz, matrix units busy 62 % of it in the loss, 50 % with dS, 69 % in the
// gradients).  Between, launches and tiles that do not fill the CUs (500 x 10,007 x 256 in fp32 114 us in seven launches).
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
constexpr int kVocabStep = 256;         // pieces of the table are multiples of it
constexpr long long kPackBytes = 256ll << 20, kPieceBytes = 256ll << 20;

constexpr float kHalfUnit = 16384.f;    // the largest weight of fp16 dS

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

enum Epilogue : int { kStats, kGradS, kGradRows, kGradTable };

struct ProductArgs {
  Operand a, b;
  int m, n, k;               // sizes of the product
  const int* count;          // null, or how many of n (kGradTable: of k) there are
  int parts;                 // 1, or 3: the operands' parts
  int splits;                // shares of the contraction, each with a slice of its own in out
  // kStats, kGradS: m = rows of the table from `v0` on, n = tokens
  int v0, V;
  float scale;
  float2* stats;             // [tile of the table][tokens]
  const int* targets;        // kGradS
  const float *lse, *weight;
  void* ds;                  // [part][n][ds_stride]
  long long ds_stride, ds_part;
  // kGradRows, kGradTable: out[n][m]
  void* out;
  long long out_stride, out_slice;
  int out_dtype;
  int add;                   // add onto it
  const float* factor;       // null, or what the sums are multiplied with
};

// Columns c .. c + 7 of a row of D, added onto what is there or not.
__device__ __forceinline__ void store_any(void* p, int dtype, long long row, int c, int D, float (&v)[8], bool add) {
  auto put = [&](auto t) {
    typedef decltype(t) T;
    T* const at = (T*)p + row;
    if (add) {
      float old[8];
      load_cols(at, c, D, old);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += old[i];
    }
    store_cols(at, c, D, v);
  };
  if (dtype == KAN_F32) put(float{});
  else if (dtype == KAN_F16) put(f16{});
  else put(bf16{});
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

// Which parts of A and B the six products of three parts each take (dT of fp32 rows), the smallest first: two bits a product.
constexpr uint32_t kPartA = 2u | 1u << 2 | 0u << 4 | 1u << 6 | 0u << 8 | 0u << 10;
constexpr uint32_t kPartB = 0u | 1u << 2 | 2u << 4 | 0u << 6 | 1u << 8 | 0u << 10;

// One operand's tile of R rows: a step of it is R x 32 numbers, 64 R bytes of LDS.
//   k contiguous: [row][4 pieces of 8 k], piece c of row r at place c ^ (r >> 2 & 3), so that sixteen lanes side by side, which
//   read one piece of sixteen rows, meet all banks once (c ^ (r >> 1 & 3) does so for eight lanes: half of the clocks of the
//   LDS were conflicts);
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
      chunk = (l & 3u) ^ (l >> 4 & 3u);
#pragma unroll
      for (int j = 0; j < kCopies; ++j) off[j] = (uint32_t)((wave * kCopies + j) * 16 + (lane >> 2)) * (uint32_t)row + chunk * 16u;
      chunk *= 8u;
      const uint32_t r = first + (lane & 31);
      read = r * 64u + ((uint32_t)(lane >> 5) ^ (r >> 2 & 3u)) * 16u;
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
  // The buffer of the next copies: aimed at some k of a part, then moved on a step at a time.
  uint64_t at;
  uint32_t bytes;                  // k contiguous: from there to the end of the last row; strided: of one k
  int deep;                        // k that are left
  __device__ __forceinline__ void aim(uint32_t p, int depth, int k0) {
    at = (uint64_t)(uintptr_t)base + (uint64_t)((long long)p * part + (long long)(k0 / kStep) * step);
    bytes = K ? (uint32_t)limit - (uint32_t)k0 * 2u : (uint32_t)limit;
    deep = depth - k0;
  }
  __device__ __forceinline__ void move() {
    at += (uint32_t)step;
    if (K) bytes -= kStep * 2u;
    deep -= kStep;
  }
  __device__ __forceinline__ u32x4 buffer() const {
    // (a strided step's last row ends where the tile's columns begin behind it: fewer bytes by r0)
    const uint32_t n = K ? bytes : (uint32_t)min(deep, kStep) * bytes - chunk;
    u32x4 r = {(uint32_t)at, (uint32_t)(at >> 32), deep > 0 ? n : 0u, 0x00020000u};
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
// A step is 32 of the contraction.  LDS holds kSlots of them; the fragments of a step are read into registers while the step
// before is multiplied, and the copies of the kSlots-th next one are sent out, one or two between each two MFMAs.  One barrier
// a step: behind it every wave's copies of step s + 1 have landed and nobody reads slot s % kSlots any more.
template <int RB_, int CB_, int WM_, int WN_, int SLOTS_>
struct Shape {
  static constexpr int RB = RB_, CB = CB_, WM = WM_, WN = WN_, kSlots = SLOTS_;
  static constexpr int BM = 32 * RB * WM, BN = 32 * CB * WN, kLds = kSlots * (BM + BN) * kStep * 2;
};

// Which tile, and which share of the contraction, a workgroup has: runs of consecutive work items per XCD; eight tiles of n by as many
// of m as it has workgroups.
__device__ __forceinline__ bool place(unsigned block, unsigned nmt, unsigned nnt, unsigned splits, int* mt, int* nt, int* split) {
  const unsigned tiles = nmt * nnt, W = tiles * splits, L = block, xcd = L & 7u, q = W >> 3, r = W & 7u;
  if (L >= W) return false;
  const unsigned work = xcd * q + min(xcd, r) + (L >> 3), item = work % tiles;
  *split = (int)(work / tiles);
  const unsigned group = item / (8 * nmt), first = group * 8, width = min(8u, nnt - first), in = item - first * nmt;
  *mt = (int)(in / width);
  *nt = (int)(first + in % width);
  return true;
}

// What becomes of a tile's sums, acc[i][j][r]: m = m0 + wm + 32 i + 8 (r / 4) + 4 lh + r % 4, n = n0 + wn + 32 j + ln.  All waves are done with
// the LDS.
template <class T, int EPI, class S>
__device__ __forceinline__ void finish(const ProductArgs& g, f32x16 (&acc)[S::RB][S::CB], const int m0, const int n0, const int split, const int n_here,
                                       unsigned char* const sRing) {
  constexpr int RB = S::RB, CB = S::CB, WM = S::WM, BM = S::BM, BN = S::BN;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, lh = lane >> 5;
  const int wm = (wave % WM) * 32 * RB, wn = (wave / WM) * 32 * CB;
  if constexpr (EPI == kStats) {
    // In units of log 2: the exponentials are the hardware's, of base 2.
    float2* const sStat = (float2*)sRing;         // [WM][BN]
    const float scale = g.scale * 1.44269504088896f;
    const int here = g.V - g.v0 - m0 - wm;       // rows of the table from the wave's first on (differences: v0 + m0 + wm may pass 2^31)
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      int rows = here - 4 * lh;
      asm volatile("" : "+v"(rows));       // (compared anew: 64 masks kept for all j would not fit the scalar registers)
      const bool whole = here >= 32 * RB;
      float z[RB][16], top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) z[i][r] = acc[i][j][r] * scale;
      if (!whole) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) z[i][r] = 32 * i + 8 * (r >> 2) + (r & 3) < rows ? z[i][r] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, z[i][r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const float at = fminf(fmaxf(top, -FLT_MAX), FLT_MAX);      // (finite, so that nothing below subtracts infinities)
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(z[i][r] - at);
      sum += __shfl_xor(sum, 32);
      if (lh == 0) sStat[(wave % WM) * BN + wn + 32 * j + ln] = make_float2(at, sum);
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    for (int c = tid; c < BN; c += kThreads)
      if (n0 + c < g.n) {
        float at = sStat[c].x, sum = 0.f;
#pragma unroll
        for (int w = 1; w < WM; ++w) at = fmaxf(at, sStat[w * BN + c].x);
#pragma unroll
        for (int w = 0; w < WM; ++w) sum += sStat[w * BN + c].y * __builtin_amdgcn_exp2f(sStat[w * BN + c].x - at);
        g.stats[(long long)((g.v0 + m0) / BM) * g.n + n0 + c] = make_float2(at, sum);
      }
  } else {
    // Blocks of 32 rows n go through LDS, each wave's through its own part, so that 4 RB lanes write the pieces of one row:
    // row r's four columns u at place u ^ r.
    constexpr int kUnits = 8 * RB, kGroup = 4 * RB;
    static_assert(4 * 32 * kUnits * 16 <= S::kLds, "the blocks of four waves");
    float4* const mine = (float4*)sRing + wave * (32 * kUnits);
    const float factor = EPI != kGradS && g.factor ? *g.factor : 1.f;
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      const int nb = n0 + wn + 32 * j;
      if (nb >= n_here) break;
      if constexpr (EPI == kGradS) {
        const int n = min(nb + ln, n_here - 1);
        const float lse = g.lse[n] * 1.44269504088896f, weight = g.weight[n], scale = g.scale * 1.44269504088896f;
        const int here = g.V - g.v0 - m0 - wm;
        int rows = here - 4 * lh, hit = (int)((uint32_t)g.targets[n] - (uint32_t)(g.v0 + m0) - (uint32_t)(wm + 4 * lh));
        asm volatile("" : "+v"(rows), "+v"(hit));
        // (a target, or the table's end, among the wave's rows)
        const bool special = __any((unsigned)hit < 32u * RB) || here < 32 * RB;
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int at = 32 * i + 8 * (r >> 2) + (r & 3);
            const float p = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], scale, -lse));
            acc[i][j][r] = p * weight;
            if (special) acc[i][j][r] = at < rows ? (at == hit ? p - 1.f : p) * weight : 0.f;
          }
      }
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          mine[ln * kUnits + ((8 * i + 2 * q + lh) ^ (ln & (kUnits - 1)))] =
              make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
      __builtin_amdgcn_wave_barrier();
#pragma unroll 4
      for (int r = lane / kGroup; r < 32; r += 64 / kGroup) {
        const int u = (lane % kGroup) * 2, n = nb + r, m = m0 + wm + u * 4;
        const float4 x = mine[r * kUnits + (u ^ (r & (kUnits - 1)))], y = mine[r * kUnits + ((u + 1) ^ (r & (kUnits - 1)))];
        if (n >= n_here) continue;
        float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        if constexpr (EPI == kGradS) {
          if (m >= g.ds_stride) continue;
          T* const dst = (T*)g.ds + (long long)n * g.ds_stride + m;
          for (int p = 0; p < g.parts; ++p) {
            store8(dst + p * g.ds_part, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] -= (float)(T)v[i];
          }
        } else {
          if (m >= g.m) continue;
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] *= factor;
          store_any(g.out, g.out_dtype, split * g.out_slice + n * g.out_stride, m, g.m, v, g.add);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

template <class T, bool AK, bool BK, int EPI, class S>
__device__ __forceinline__ void product(const ProductArgs& g, const unsigned block, unsigned char* const sRing) {
  constexpr int RB = S::RB, CB = S::CB, WM = S::WM, WN = S::WN, kSlots = S::kSlots, BM = S::BM, BN = S::BN;
  typedef Tile<T, AK, BM> TA;
  typedef Tile<T, BK, BN> TB;
  constexpr int kSlot = TA::kBytes + TB::kBytes, kCopies = TA::kCopies + TB::kCopies;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wave % WM) * 32 * RB, wn = (wave / WM) * 32 * CB;
  const int n_here = EPI != kGradTable && g.count ? min(g.n, *g.count) : g.n, k_here = EPI == kGradTable && g.count ? min(g.k, *g.count) : g.k;
  int mt, nt, split;
  const unsigned nnt = (unsigned)(n_here + BN - 1) / BN;
  if (!place(block, (unsigned)(g.m + BM - 1) / BM, nnt, (unsigned)g.splits, &mt, &nt, &split)) return;
  const int m0 = mt * BM, n0 = nt * BN;
  TA A;
  TB B;
  A.init(g.a, m0, wave, lane, wm);
  B.init(g.b, n0, wave, lane, wn);
  const int depth_a = min(g.a.depth, AK ? g.a.depth : k_here), depth_b = min(g.b.depth, BK ? g.b.depth : k_here);
  const int ksteps = (k_here + kStep - 1) / kStep, all = g.parts == 1 ? ksteps : 6 * ksteps;
  const int s0 = (int)((long long)all * split / g.splits), total = (int)((long long)all * (split + 1) / g.splits) - s0;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)sRing;

  // The next copies: product of parts, k, slot.  Past the last one everything is behind the buffers' ends.
  // With one tile of n every row of the table is read by one workgroup: each begins at another k, since rows of 2^n bytes in step
  // would meet in the same memory channels.
  const int turn = EPI != kGradRows && nnt == 1 && g.parts == 1 && ksteps > 1 ? (int)((unsigned)mt * 5u % (unsigned)ksteps) : 0;
  int cq = g.parts == 1 ? 0 : s0 / max(ksteps, 1), ck = (s0 - cq * ksteps + turn) * kStep, cs = 0, left = total;
  u32x4 ra, rb;
  A.aim(g.parts == 1 ? 0u : kPartA >> (2 * cq) & 3u, depth_a, ck);
  B.aim(g.parts == 1 ? 0u : kPartB >> (2 * cq) & 3u, depth_b, ck);
  ra = A.buffer();
  rb = B.buffer();
  auto copy = [&](int j) __attribute__((always_inline)) {
    if (j < TA::kCopies) A.copy(ra, j, wave, lds0 + (uint32_t)(cs * kSlot), ck, depth_a);
    else B.copy(rb, j - TA::kCopies, wave, lds0 + (uint32_t)(cs * kSlot + TA::kBytes), ck, depth_b);
  };
  auto next = [&]() __attribute__((always_inline)) {
    cs = cs + 1 == kSlots ? 0 : cs + 1;
    ck += kStep;
    A.move();
    B.move();
    if (--left <= 0) {
      A.deep = B.deep = 0;
    } else if (ck >= k_here) {
      ck = 0;
      cq += g.parts > 1 ? 1 : 0;
      A.aim(g.parts == 1 ? 0u : kPartA >> (2 * cq) & 3u, depth_a, 0);
      B.aim(g.parts == 1 ? 0u : kPartB >> (2 * cq) & 3u, depth_b, 0);
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
  auto read = [&](const unsigned char* slot, int i, Frags& to) __attribute__((always_inline)) {
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

  int rs = 0;
  auto step = [&](auto P) __attribute__((always_inline)) {
    constexpr int p = decltype(P)::value, kMfmas = 2 * RB * CB, kSpread = kMfmas > 4 ? kMfmas - 2 : kMfmas;
    copies_done<(kSlots - 2) * kCopies>();
    __builtin_amdgcn_s_barrier();
    rs = rs + 1 == kSlots ? 0 : rs + 1;
    const unsigned char* const slot = sRing + rs * kSlot;
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
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
  }
  if (s < total) step(std::integral_constant<int, 0>{});
  copies_done<0>();
  __syncthreads();

  finish<T, EPI, S>(g, acc, m0, n0, split, n_here, sRing);
}

constexpr int waves_of(int lds) { return lds <= 81920 ? 2 : 1; }      // workgroups of four waves that a CU is to hold
template <class T, bool AK, bool BK, int EPI, class S>
__global__ __launch_bounds__(kThreads, waves_of(S::kLds)) void kan_vocab_product_kernel(const ProductArgs g) {
  __shared__ __attribute__((aligned(1024))) unsigned char sRing[S::kLds];
  product<T, AK, BK, EPI, S>(g, blockIdx.x, sRing);
}
// dh and dT of a piece in one launch, so that the tiles of one fill the CUs that the last round of the other leaves.
template <class T, class S>
__global__ __launch_bounds__(kThreads, waves_of(S::kLds)) void kan_vocab_grads_kernel(const ProductArgs rows, const ProductArgs table, unsigned row_blocks) {
  __shared__ __attribute__((aligned(1024))) unsigned char sRing[S::kLds];
  if (blockIdx.x < row_blocks) product<T, false, true, kGradRows, S>(rows, blockIdx.x, sRing);
  else product<T, false, false, kGradTable, S>(table, blockIdx.x - row_blocks, sRing);
}

// ---- fp32: products with the table ------------------------------------------------------------------------------------
// z and dh read the table as it is and split it into its parts in registers.  (Parts in the workspace are one and a half times its bytes, written twice
// and read three times, by tiles whose steps are six times as many: loss and gradients of 65 x 100,000 x 2,048 so 2,916 us, of 128 x 30,000 x 2,048 824, of
// 500 x 1,300 x 4,000 397; now 1,148, 420 and 203.)  The product of the first parts and the smaller ones have sums of their own.  Bound by the
// reads of the table up to about 64 tokens (64 x 30,000 x 1,024: 42 us for the loss, 176 with gradients), by the matrix cores beyond (1,024 x 30,000 x
// 2,048: the loss 633 us, 1.19 PFLOP/s of the parts).

// The next bf16 part of two numbers, and what is left of them.
__device__ __forceinline__ uint32_t next_part(float& x, float& y, bool last = false) {
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 t = {(bf16)x, (bf16)y};
  const uint32_t both = __builtin_bit_cast(uint32_t, t);
  if (!last) {
    x -= __builtin_bit_cast(float, both << 16);
    y -= __builtin_bit_cast(float, both & 0xffff0000u);
  }
  return both;
}

struct FewSums {
  f32x16 high, low;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 16; ++i) high[i] = low[i] = 0.f;
  }
  // v: eight k of a row of A; b: a row of B, its parts `part` further
  __device__ __forceinline__ void add(float (&v)[8], const bf16* b, long long part) {
    uint4 a[3];
#pragma unroll
    for (int p = 0; p < 3; ++p) a[p] = make_uint4(next_part(v[0], v[1]), next_part(v[2], v[3]), next_part(v[4], v[5]), next_part(v[6], v[7]));
    uint4 w[3];
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p] = *(const uint4*)(b + p * part);
    low = mfma<bf16>(a[2], w[0], low);
    low = mfma<bf16>(a[1], w[1], low);
    low = mfma<bf16>(a[0], w[2], low);
    low = mfma<bf16>(a[1], w[0], low);
    low = mfma<bf16>(a[0], w[1], low);
    high = mfma<bf16>(a[0], w[0], high);
  }
};

// Few tokens, or few rows of the table: a workgroup has z of 32 rows of the table and 32 tokens, whose parts come from L2.  Four waves share
// the columns, 64 at a time, and add their sums through LDS.
constexpr int kFewRows = 32;
template <int EPI>
__global__ __launch_bounds__(kThreads) void kan_vocab_few_kernel(const ProductArgs g) {
  __shared__ float sSum[4][16][64];
  __shared__ float2 sStat[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ln = lane & 31, lh = lane >> 5;
  const int n_here = g.count ? min(g.n, *g.count) : g.n, m0 = (int)blockIdx.x * kFewRows, n0 = (int)blockIdx.y * 32;
  if (n0 >= n_here) return;
  const float* const row = (const float*)g.a.p + (long long)min(m0 + ln, g.m - 1) * g.a.stride;
  const bf16* const b = (const bf16*)g.b.p + (long long)min(n0 + ln, n_here - 1) * g.b.stride;
  FewSums sums;
  sums.clear();
  for (int k0 = wave * 64; k0 < g.k; k0 += 256) {
    float v[4][8];
    if (k0 + 64 <= g.k) {
#pragma unroll
      for (int h = 0; h < 4; ++h) load8(row + k0 + 16 * h + 8 * lh, v[h]);
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = k0 + 16 * h + 8 * lh + i;
          v[h][i] = k < g.k ? row[k] : 0.f;
        }
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) sums.add(v[h], b + k0 + 16 * h + 8 * lh, g.b.part);      // (zeros behind B's last column)
  }
  const float scale = g.scale * 1.44269504088896f;
  const int m = 8 * wave + 4 * lh, rows = g.m - m0 - m;       // the lane's four rows of token ln
  const int n = n0 + ln;
#pragma unroll
  for (int i = 0; i < 16; ++i) sSum[wave][i][lane] = sums.high[i] + sums.low[i];
  __syncthreads();
  float z[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) z[q] = (sSum[0][4 * wave + q][lane] + sSum[1][4 * wave + q][lane]) + (sSum[2][4 * wave + q][lane] + sSum[3][4 * wave + q][lane]);
  if constexpr (EPI == kStats) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      z[q] = q < rows ? z[q] * scale : -INFINITY;
      top = fmaxf(top, z[q]);
    }
    top = fmaxf(top, __shfl_xor(top, 32));
    const float at = fminf(fmaxf(top, -FLT_MAX), FLT_MAX);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += __builtin_amdgcn_exp2f(z[q] - at);
    sum += __shfl_xor(sum, 32);
    if (lh == 0) sStat[wave][ln] = make_float2(at, sum);
    __syncthreads();
    if (threadIdx.x < 32 && n < g.n) {
      float all = sStat[0][ln].x, total = 0.f;
#pragma unroll
      for (int w = 1; w < 4; ++w) all = fmaxf(all, sStat[w][ln].x);
#pragma unroll
      for (int w = 0; w < 4; ++w) total += sStat[w][ln].y * __builtin_amdgcn_exp2f(sStat[w][ln].x - all);
      g.stats[(long long)((g.v0 + m0) / kFewRows) * g.n + n] = make_float2(all, total);
    }
  } else {
    if (n < n_here) {
      const float lse = g.lse[n] * 1.44269504088896f, weight = g.weight[n];
      const int hit = (int)((uint32_t)g.targets[n] - (uint32_t)(g.v0 + m0) - (uint32_t)m);
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float e = __builtin_amdgcn_exp2f(fmaf(z[q], scale, -lse));
        v[q] = q < rows ? (q == hit ? e - 1.f : e) * weight : 0.f;
      }
      bf16* dst = (bf16*)g.ds + (long long)n * g.ds_stride + m0 + m;
#pragma unroll
      for (int p = 0; p < 3; ++p, dst += g.ds_part) {
        typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 t;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          t[q] = (bf16)v[q];
          v[q] -= (float)t[q];
        }
        *(bf16x4*)dst = t;
      }
    }
  }
}

// dh's slices of up to 32 tokens: four waves take 32 columns each of the same rows of the table.
__global__ __launch_bounds__(kThreads) void kan_vocab_few_rows_kernel(const ProductArgs g) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ln = lane & 31, lh = lane >> 5;
  const int n_here = min(g.n, *g.count), d0 = (int)blockIdx.x * 128 + wave * 32, split = blockIdx.y;
  if (n_here == 0 || d0 >= g.m) return;
  const float* const column = (const float*)g.a.p + min(d0 + ln, g.m - 1);
  const bf16* const b = (const bf16*)g.b.p + (long long)min(ln, n_here - 1) * g.b.stride;
  FewSums sums;
  sums.clear();
  const long long steps = (g.k + 31) / 32;
  const int s0 = (int)(steps * split / g.splits), s1 = (int)(steps * (split + 1) / g.splits);
  for (int s = s0; s < s1; ++s) {
    float v[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[h][i] = column[(long long)min(32 * s + 16 * h + 8 * lh + i, g.k - 1) * g.a.stride];
#pragma unroll
    for (int h = 0; h < 2; ++h) sums.add(v[h], b + 32 * s + 16 * h + 8 * lh, g.b.part);       // (dS is zero behind the last row)
  }
  float* const out = (float*)g.out + split * g.out_slice + ln * g.out_stride;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int d = d0 + 8 * (i >> 2) + 4 * lh + (i & 3);
    if (ln < n_here && d < g.m) out[d] = sums.high[i] + sums.low[i] + (g.add ? out[d] : 0.f);
  }
}

// Tiles of 32 WM rows of the table (dh: columns) and 32 CB WN tokens.  A wave has 32 of the rows as fragments straight from memory, two steps of
// 32 ahead, and splits the next half of a step while this one is multiplied; the tokens' parts pass through LDS for all waves, a ring of three
// steps.  One barrier a step, in front of its last six products.
template <int CB_, int WM_>
struct SplitShape {
  static constexpr int RB = 1, CB = CB_, WM = WM_, WN = 4 / WM_;
  static constexpr int BM = 32 * WM, BN = 32 * CB * WN, kHeld = (BN + 63) / 64 * 64, kSlots = 3, kLds = kSlots * 3 * kHeld * kStep * 2;
};
// AK: z (else dh): the contraction is over the columns of the table.
template <bool AK, int EPI, class S>
__device__ __forceinline__ void split_product(const ProductArgs& g, const unsigned block, unsigned char* const sRing) {
  constexpr int CB = S::CB, BM = S::BM, BN = S::BN, kSlots = S::kSlots, kAhead = 2;
  typedef Tile<bf16, true, S::kHeld> TB;
  constexpr int kSlot = 3 * TB::kBytes, kCopies = 3 * TB::kCopies;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, lh = lane >> 5;
  const int wm = wave % S::WM * 32, n_here = g.count ? min(g.n, *g.count) : g.n;
  int mt, nt, split;
  if (!place(block, (unsigned)(g.m + BM - 1) / BM, (unsigned)(n_here + BN - 1) / BN, (unsigned)g.splits, &mt, &nt, &split)) return;
  const int m0 = mt * BM, n0 = nt * BN;
  const int steps = (g.k + kStep - 1) / kStep, s0 = (int)((long long)steps * split / g.splits), s1 = (int)((long long)steps * (split + 1) / g.splits);
  TB B;
  B.init(g.b, n0, wave, lane, wave / S::WM * 32 * CB);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)sRing;
  // (a step past the last one: a buffer of no bytes)
  auto copy = [&](int s, int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      B.aim((uint32_t)p, s < s1 ? g.b.depth : 0, s * kStep);
      const u32x4 r = B.buffer();
#pragma unroll
      for (int j = 0; j < TB::kCopies; ++j) B.copy(r, j, wave, lds0 + (uint32_t)(slot * kSlot + p * TB::kBytes), s * kStep, g.b.depth);
    }
  };
  // A: rows past the last one repeat it.  Bytes from the tile's first element on.
  const char* const a0 = (const char*)g.a.p + (AK ? (long long)m0 * g.a.stride * 4 : (long long)m0 * 4);
  const long long row = g.a.stride * 4;
  const uint32_t r0 = (uint32_t)(min(m0 + wm + ln, g.m - 1) - m0), ao = AK ? r0 * (uint32_t)row + lh * 32u : r0 * 4u + lh * 8u * (uint32_t)row;
  // Half h of a step: eight numbers of k = 16 h + 8 lh on.  (Always loads, so that the compiler's waits count the same loads on every way.)
  float a[kAhead][2][8];
  auto fetch = [&](int s, int h, auto P) __attribute__((always_inline)) {
    constexpr int to = decltype(P)::value;
    const int k0 = min(s, s1 - 1) * kStep;
    if (k0 + kStep <= g.k) {
      if constexpr (AK) {
        load8((const float*)(a0 + (long long)k0 * 4 + ao) + 16 * h, a[to][h]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) a[to][h][e] = *(const float*)(a0 + (long long)(k0 + 16 * h + e) * row + ao);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int k = k0 + 16 * h + e;
        a[to][h][e] = k + 8 * lh < g.k ? *(const float*)(a0 + (AK ? (long long)k * 4 : (long long)k * row) + ao) : 0.f;
      }
      __builtin_amdgcn_s_waitcnt(0);
    }
  };
  // Parts of both halves: one is multiplied while the other is formed, two numbers at a time.
  uint32_t parts[2][3][4];
  auto cut = [&](int h, int pair, int p, auto P) __attribute__((always_inline)) {
    constexpr int from = decltype(P)::value;
    parts[h][p][pair] = next_part(a[from][h][2 * pair], a[from][h][2 * pair + 1], p == 2);
    asm volatile("" : "+v"(parts[h][p][pair]));       // (formed here, beside the products, not where it is used)
  };
  f32x16 high[1][CB], low[CB];
#pragma unroll
  for (int j = 0; j < CB; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) high[0][j][r] = low[j][r] = 0.f;
  uint4 w[2][3];
  int slot = 0;
  auto read = [&](int s, int group, int to) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 3; ++p) B.fragment(sRing + s * kSlot + p * TB::kBytes, group % CB, group / CB, 0, w[to][p]);
  };
  // Groups of six products: half h of a block of 32 tokens.  Behind the first of them the next group's fragments are asked for, between the
  // others the next half's parts are formed.
  auto step = [&](int s, auto now) __attribute__((always_inline)) {
    const std::integral_constant<int, (decltype(now)::value + 1) % kAhead> next;
    const int last = slot >= 1 ? slot - 1 : kSlots - 1, after = slot + 1 == kSlots ? 0 : slot + 1;
    copy(s + kSlots - 1, last);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 2 * CB; ++q) {
      const int h = q / CB, j = q % CB;
      if (j == 0) {
        fetch(s + kAhead, h, now);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (q == 2 * CB - 1) {
        // The last reads of this slot are done, and the next one is there.  Behind its copies are those of kSlots - 2 later ones, and the loads
        // of as many steps and this one, four each at least, where the step that these are for exists (the compiler leaves out those that nothing needs).
        if (s + kAhead < s1) copies_done<kCopies * (kSlots - 2) + 4 * (kSlots - 1)>();
        else copies_done<kCopies * (kSlots - 2)>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
      uint4 v[3];
#pragma unroll
      for (int p = 0; p < 3; ++p) v[p] = make_uint4(parts[h][p][0], parts[h][p][1], parts[h][p][2], parts[h][p][3]);
      const uint4(&b)[3] = w[q & 1];
      constexpr int kSmall = 5, kPartsA[] = {2, 1, 0, 1, 0}, kPartsB[] = {0, 1, 2, 0, 1};
#pragma unroll
      for (int m = 0; m <= kSmall; ++m) {
        if (m < kSmall) low[j] = mfma<bf16>(v[kPartsA[m]], b[kPartsB[m]], low[j]);
        else high[0][j] = mfma<bf16>(v[0], b[0], high[0][j]);
        __builtin_amdgcn_sched_barrier(0);
        if (m == 0) read(q == 2 * CB - 1 ? after : slot, q == 2 * CB - 1 ? 0 : q + 1, (q + 1) & 1);
        const int first = j * 12 / CB, count = (j + 1) * 12 / CB - first;
#pragma unroll
        for (int c = first + m * count / (kSmall + 1); c < first + (m + 1) * count / (kSmall + 1); ++c) {
          if (h == 0) cut(1, c / 3, c % 3, now);
          else cut(0, c / 3, c % 3, next);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    slot = after;
  };
  if (s0 < s1) {
#pragma unroll
    for (int i = 0; i < kSlots - 1; ++i) copy(s0 + i, i);
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    fetch(s0, 0, even);
    fetch(s0, 1, even);
    fetch(s0 + 1, 0, odd);
    fetch(s0 + 1, 1, odd);
#pragma unroll
    for (int c = 0; c < 12; ++c) cut(0, c / 3, c % 3, even);
    copies_done<kCopies * (kSlots - 2)>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(0, 0, 0);
    int s = s0;
    for (; s + 2 <= s1; s += 2) {
      step(s, even);
      step(s + 1, odd);
    }
    if (s < s1) step(s, even);
  }
  copies_done<0>();
  __syncthreads();
#pragma unroll
  for (int j = 0; j < CB; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) high[0][j][r] += low[j][r];
  finish<bf16, EPI, S>(g, high, m0, n0, split, n_here, sRing);
}
template <bool AK, int EPI, class S>
__global__ __launch_bounds__(kThreads, 2) void kan_vocab_split_kernel(const ProductArgs g) {
  __shared__ __attribute__((aligned(1024))) unsigned char sRing[S::kLds];
  split_product<AK, EPI, S>(g, blockIdx.x, sRing);
}
// dh and dT of a piece in one launch, as kan_vocab_grads_kernel.
template <class R, class S>
__global__ __launch_bounds__(kThreads, 2) void kan_vocab_split_grads_kernel(const ProductArgs rows, const ProductArgs table, unsigned row_blocks) {
  __shared__ __attribute__((aligned(1024))) unsigned char sRing[R::kLds > S::kLds ? R::kLds : S::kLds];
  if (blockIdx.x < row_blocks) split_product<false, kGradRows, R>(rows, blockIdx.x, sRing);
  else product<bf16, false, false, kGradTable, S>(table, blockIdx.x - row_blocks, sRing);
}

// z from its slices [slice][token][row] (few tiles: shares of the columns each): a wave has 256 rows of the table and a token.
constexpr int kSumRows = 256;
template <int EPI>
__global__ __launch_bounds__(kThreads) void kan_vocab_sums_kernel(const ProductArgs g, const float* __restrict__ src, int slices, unsigned chunks) {
  const int lane = threadIdx.x & 63, n = (int)(blockIdx.x / chunks) * 4 + (threadIdx.x >> 6), n_here = g.count ? min(g.n, *g.count) : g.n;
  if (n >= n_here) return;
  const unsigned chunk = blockIdx.x % chunks;
  const int m = (int)chunk * kSumRows + lane * 4, rows = g.m - m;
  float z[4] = {0.f, 0.f, 0.f, 0.f};
  if (rows > 0) {
#pragma unroll 4
    for (int k = 0; k < slices; ++k) {
      const float4 t = *(const float4*)(src + k * g.out_slice + n * g.out_stride + m);       // (rows of whole float4)
      z[0] += t.x, z[1] += t.y, z[2] += t.z, z[3] += t.w;
    }
  }
  const float scale = g.scale * 1.44269504088896f;
  if constexpr (EPI == kStats) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      z[q] = q < rows ? z[q] * scale : -INFINITY;
      top = fmaxf(top, z[q]);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float at = fminf(fmaxf(top, -FLT_MAX), FLT_MAX);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += __builtin_amdgcn_exp2f(z[q] - at);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) g.stats[((long long)(g.v0 / kSumRows) + chunk) * g.n + n] = make_float2(at, sum);
  } else {
    const float lse = g.lse[n] * 1.44269504088896f, weight = g.weight[n];
    const int hit = (int)((uint32_t)g.targets[n] - (uint32_t)g.v0 - (uint32_t)m);
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float e = __builtin_amdgcn_exp2f(fmaf(z[q], scale, -lse));
      v[q] = q < rows ? (q == hit ? e - 1.f : e) * weight : 0.f;
    }
    uint2* dst = (uint2*)((bf16*)g.ds + (long long)n * g.ds_stride + m);
#pragma unroll
    for (int p = 0; p < 3; ++p, dst = (uint2*)((bf16*)dst + g.ds_part)) *dst = make_uint2(next_part(v[0], v[1]), next_part(v[2], v[3]));
  }
}

// Which tokens have a target that names a row: their numbers in order, from the back of the list those of the others; how
// many; what their weights are multiplied with, and the factor that takes this back.
struct Index {
  int* list;                 // [N]
  int* count;
  float *mul, *factor;
};
// What the weights dloss are multiplied with, and the sums after it: the largest weight `top` is at `unit` (0: as it is).
// (Weights below 1e-30 and above 2^126 are not brought there, so that nothing here leaves fp32's range.)
__device__ __forceinline__ float within_fp32(float top) { return fminf(fmaxf(top, 1e-30f), 0x1p126f); }
__device__ __forceinline__ float scale_of(float scale, float unit, float top) { return unit != 0.f ? unit / within_fp32(top) : scale; }
__device__ __forceinline__ float factor_of(float scale, float unit, float top) { return unit != 0.f ? scale * (within_fp32(top) / unit) : 1.f; }
// (infinite and NaN weights spoil their own rows alone)
__device__ __forceinline__ float larger(float top, float dloss) { return fabsf(dloss) <= FLT_MAX ? fmaxf(top, fabsf(dloss)) : top; }

__global__ __launch_bounds__(1024) void kan_vocab_index_kernel(const float* __restrict__ dloss, const void* __restrict__ targets, int id_dtype, uint32_t V, int N,
                                                               float scale, float unit, const Index x) {
  __shared__ int sCount[16];
  __shared__ float sMax[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0;
  float top = 0.f;
  for (int n0 = 0; n0 < N; n0 += 1024) {
    const int n = n0 + threadIdx.x;
    const bool named = n < N && row_of(targets, id_dtype, n, V) < V;
    const uint64_t all = __ballot(named);
    if (lane == 0) sCount[wave] = __popcll(all);
    __syncthreads();
    int at = before, sum = 0;
    for (int w = 0; w < 16; ++w) {
      at += w < wave ? sCount[w] : 0;
      sum += sCount[w];
    }
    at += __popcll(all & ((1ull << lane) - 1));
    if (named) {
      x.list[at] = n;
      if (unit != 0.f) top = larger(top, dloss[n]);
    } else if (n < N) {
      x.list[N - 1 - (n - at)] = n;
    }
    before += sum;
    __syncthreads();
  }
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) sMax[wave] = top;
  __syncthreads();
  if (threadIdx.x != 0) return;
  *x.count = before;
  for (int w = 0; w < 16; ++w) top = fmaxf(top, sMax[w]);
  *x.mul = scale_of(scale, unit, top);
  *x.factor = factor_of(scale, unit, top);
}

// Rows in the form the products take: 16-bit parts of `width` columns (zeros behind the last).
struct PackArgs {
  const void* src;
  void* dst;
  long long rows;
};
template <class I, class T, int PARTS>
__device__ __forceinline__ void pack_item(const I* row, int c, int D, T* dst, long long part) {
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < D) load_cols(row, c, D, v);
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    store8(dst + p * part, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] -= (float)(T)v[k];
  }
}
template <class I, class T, int PARTS>
__device__ __forceinline__ void pack_rows(const PackArgs& a, int D, int width, unsigned block, unsigned blocks) {
  const int C = width / 8;
  const long long items = a.rows * C;
  for (long long i = (long long)block * kThreads + threadIdx.x; i < items; i += (long long)blocks * kThreads) {
    const long long row = i / C;
    const int c = (int)(i - row * C) * 8;
    pack_item<I, T, PARTS>((const I*)a.src + row * D, c, D, (T*)a.dst + row * width + c, a.rows * width);
  }
}
template <class I, class T, int PARTS>
__global__ __launch_bounds__(kThreads) void kan_vocab_pack_kernel(const PackArgs a, const PackArgs b, unsigned blocks_a, int D, int width) {
  if (blockIdx.x < blocks_a) pack_rows<I, T, PARTS>(a, D, width, blockIdx.x, blocks_a);
  else pack_rows<I, T, PARTS>(b, D, width, blockIdx.x - blocks_a, gridDim.x - blocks_a);
}

// The same for the tokens that count, one behind the other, with their targets, lse and weights; zeros for the gradients of
// the others.  Up to kOwnIndex tokens each workgroup counts the tokens in front of its own itself, beyond the index is there.
constexpr int kOwnIndex = 4096, kTokensPerBlock = 4;
struct TokenArgs {
  const void* h;
  const void* targets;
  const float *lse, *dloss;
  void *packed, *dh;
  int* target;
  float *lse_out, *weight;
  Index x;
  int N, D, width, id_dtype;
  uint32_t V;
  float scale, unit;
  int own_index;
  unsigned blocks;
  PackArgs table;            // and rows of the table by the workgroups behind
};
template <class I, class T, int PARTS>
__device__ __forceinline__ void pack_token(const TokenArgs& a, int n, int at, bool named, float mul, int c) {
  if (!named) {
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < a.D) store_cols((I*)a.dh + (long long)n * a.D, c, a.D, zero);
    return;
  }
  pack_item<I, T, PARTS>((const I*)a.h + (long long)n * a.D, c, a.D, (T*)a.packed + (long long)at * a.width + c, (long long)a.N * a.width);
  if (c == 0) {
    a.target[at] = (int)row_of(a.targets, a.id_dtype, n, a.V);
    a.lse_out[at] = a.lse[n];
    a.weight[at] = a.dloss[n] * mul;
  }
}
template <class I, class T, int PARTS>
__global__ __launch_bounds__(kThreads) void kan_vocab_tokens_kernel(const TokenArgs a) {
  if (blockIdx.x >= a.blocks) {
    pack_rows<I, T, PARTS>(a.table, a.D, a.width, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    return;
  }
  if (!a.own_index) {
    const int C = a.width / 8, count = *a.x.count;
    const float mul = *a.x.mul;
    const long long items = (long long)a.N * C;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < items; i += (long long)a.blocks * kThreads) {
      const int at = (int)(i / C);
      pack_token<I, T, PARTS>(a, a.x.list[at], at, at < count, mul, (int)(i - (long long)at * C) * 8);
    }
    return;
  }
  __shared__ int sFront[4], sAll[4];
  __shared__ float sMax[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * kTokensPerBlock;
  int front = 0, all = 0;
  float top = 0.f;
#pragma unroll 4
  for (int n = threadIdx.x; n < a.N; n += kThreads)
    if (row_of(a.targets, a.id_dtype, n, a.V) < a.V) {
      ++all;
      front += n < first ? 1 : 0;
      if (a.unit != 0.f) top = larger(top, a.dloss[n]);
    }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    front += __shfl_xor(front, d);
    all += __shfl_xor(all, d);
    top = fmaxf(top, __shfl_xor(top, d));
  }
  if (lane == 0) {
    sFront[wave] = front;
    sAll[wave] = all;
    sMax[wave] = top;
  }
  __syncthreads();
  front = sFront[0] + sFront[1] + sFront[2] + sFront[3];
  all = sAll[0] + sAll[1] + sAll[2] + sAll[3];
  top = fmaxf(fmaxf(sMax[0], sMax[1]), fmaxf(sMax[2], sMax[3]));
  const float mul = scale_of(a.scale, a.unit, top);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *a.x.count = all;
    *a.x.factor = factor_of(a.scale, a.unit, top);
  }
  const int n = first + wave;           // a wave has a token
  if (n >= a.N) return;
  int at = front;
  bool named = false;
#pragma unroll
  for (int k = 0; k < kTokensPerBlock; ++k) {
    const bool t = first + k < a.N && row_of(a.targets, a.id_dtype, min(first + k, a.N - 1), a.V) < a.V;
    at += k < wave && t ? 1 : 0;
    named = k == wave ? t : named;
  }
  if (lane == 0 && named) a.x.list[at] = n;
  for (int c = lane * 8; c < a.width; c += 512) pack_token<I, T, PARTS>(a, n, at, named, mul, c);
}

// lse of a token from the statistics of the table's tiles, and its loss: the logit of its target is formed anew.
struct JoinArgs {
  const float2* stats;
  const void *h, *table, *targets;
  float *loss, *lse;
  int tiles, N, D, id_dtype;
  uint32_t V;
  float scale;
};
template <class I, int TOKENS>
__global__ __launch_bounds__(256) void kan_vocab_join_kernel(const JoinArgs a) {
  // TOKENS a workgroup.  Statistics: TOKENS lanes side by side have a token each, the groups of them share the tiles; the
  // target's logit: 256 / TOKENS lanes side by side have one token.
  constexpr int G = 256 / TOKENS, U = TOKENS == 1 ? 4 : 16;
  __shared__ float2 sStat[G][TOKENS];
  __shared__ float sTarget[TOKENS][4];
  const int at = threadIdx.x % TOKENS, share = threadIdx.x / TOKENS, n = blockIdx.x * TOKENS + at;
  const int in = threadIdx.x % G, of = threadIdx.x / G, nt = blockIdx.x * TOKENS + of;
  const uint32_t target = nt < a.N ? row_of(a.targets, a.id_dtype, nt, a.V) : a.V;
  float top = -FLT_MAX, sum = 0.f;
  for (int t0 = share; t0 < a.tiles; t0 += U * G) {
    float2 s[U];
#pragma unroll
    for (int k = 0; k < U; ++k) s[k] = t0 + G * k < a.tiles && n < a.N ? a.stats[(long long)(t0 + G * k) * a.N + n] : make_float2(-FLT_MAX, 0.f);
    float m = top;
#pragma unroll
    for (int k = 0; k < U; ++k) m = fmaxf(m, s[k].x);
    sum *= __builtin_amdgcn_exp2f(top - m);
#pragma unroll
    for (int k = 0; k < U; ++k) sum += s[k].y * __builtin_amdgcn_exp2f(s[k].x - m);
    top = m;
  }
  float dot = 0.f;
  if (target < a.V) {
    const I *const h = (const I*)a.h + (long long)nt * a.D, *const w = (const I*)a.table + (long long)target * a.D;
#pragma unroll 4
    for (int c = in * 8; c < a.D; c += G * 8) {
      float x[8], y[8];
      load_cols(h, c, a.D, x);
      load_cols(w, c, a.D, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot = fmaf(x[i], y[i], dot);
    }
  }
#pragma unroll
  for (int d = min(G, 64) / 2; d >= 1; d >>= 1) dot += __shfl_xor(dot, d);
  if (in % 64 == 0) sTarget[of][in / 64] = dot;
  if constexpr (TOKENS == 1) {       // a wave's share first
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      const float t = __shfl_xor(top, d), u = __shfl_xor(sum, d), m = fmaxf(top, t);
      sum = sum * __builtin_amdgcn_exp2f(top - m) + u * __builtin_amdgcn_exp2f(t - m);
      top = m;
    }
  }
  constexpr int R = TOKENS == 1 ? 4 : G;
  if (TOKENS > 1 || share % 64 == 0) sStat[TOKENS == 1 ? share / 64 : share][at] = make_float2(top, sum);
  __syncthreads();
  if (share == 0 && n < a.N) {
    float m = sStat[0][at].x, s = 0.f;
#pragma unroll
    for (int k = 1; k < R; ++k) m = fmaxf(m, sStat[k][at].x);
#pragma unroll
    for (int k = 0; k < R; ++k) s += sStat[k][at].y * __builtin_amdgcn_exp2f(sStat[k][at].x - m);
    float z = 0.f;
#pragma unroll
    for (int k = 0; k < (G + 63) / 64; ++k) z += sTarget[at][k];
    const float l = 0.693147180559945f * (m + __builtin_amdgcn_logf(s));
    a.lse[n] = l;
    a.loss[n] = row_of(a.targets, a.id_dtype, n, a.V) < a.V ? l - z * a.scale : 0.f;
  }
}

// dh from its slices: row i of them is token list[i]'s.  SHARES groups of lanes add a share of the slices each.
template <int SHARES>
__global__ __launch_bounds__(kThreads) void kan_vocab_round_kernel(const float* __restrict__ src, int slices, long long slice, int N, int D, const Index x, int dtype,
                                                                   void* __restrict__ dst) {
  constexpr int kItems = kThreads / SHARES;
  __shared__ float sSum[SHARES == 1 ? 1 : SHARES][kItems][9];
  const int C = (D + 7) / 8, share = threadIdx.x / kItems, at = threadIdx.x % kItems;
  const long long items = (long long)min(*x.count, N) * C;
  const float f = *x.factor;
  for (long long i0 = (long long)blockIdx.x * kItems; i0 < items; i0 += (long long)gridDim.x * kItems) {
    const long long i = i0 + at, row = min(i, items - 1) / C;
    const int c = (int)(min(i, items - 1) - row * C) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = share; k < slices; k += SHARES) {
      float t[8];
      load_cols(src + k * slice + row * D, c, D, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += t[e];
    }
    if constexpr (SHARES > 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sSum[share][at][e] = v[e];
      __syncthreads();
      if (share == 0)
#pragma unroll
        for (int k = 1; k < SHARES; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += sSum[k][at][e];
    }
    if (share == 0 && i < items) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= f;
      store_any(dst, dtype, (long long)x.list[row] * D, c, D, v, false);
    }
    if constexpr (SHARES > 1) __syncthreads();
  }
}

// ---- which tiles, and how many shares of the contraction ---------------------------------------------------------------
constexpr int kCus = 256;
enum TileKind : int { k256x256, k256x128, k256x64, k128x64, kTileKinds };
constexpr int kTileM[] = {256, 256, 256, 128}, kTileN[] = {256, 128, 64, 64};
// Workgroups that fit a CU, and ns of a step of 32 and of a tile's beginning and end, with that many on it and with one: with the
// statistics of z, and with rows that leave through LDS (measured on products of 8192 x 131072 x 2048, 2000 x 32000 x 1024,
// 1111 x 50021 x 1000 and 500 x 10007 x 1536).
constexpr long long kPerCu[] = {1, 2, 2, 3};
struct Cost {
  long long step, stats, rows;
};
constexpr Cost kFull[] = {{830, 5000, 15000}, {915, 7500, 11000}, {590, 9000, 6500}, {500, 6000, 4500}};
constexpr Cost kAlone[] = {{830, 5000, 13000}, {420, 4500, 8000}, {330, 4500, 6000}, {245, 4000, 4300}};

long long tiles_of(int kind, long long m, long long n) { return ((m + kTileM[kind] - 1) / kTileM[kind]) * ((n + kTileN[kind] - 1) / kTileN[kind]); }
long long steps_of(long long k, int parts) { return (k + kStep - 1) / kStep * (parts == 1 ? 1 : 6); }
// of a tile with `on` workgroups on its CU
long long tile_ns(int kind, long long steps, bool stats, long long on) {
  const Cost &f = kFull[kind], &a = kAlone[kind];
  const long long full = steps * f.step + (stats ? f.stats : f.rows), alone = steps * a.step + (stats ? a.stats : a.rows);
  return kPerCu[kind] == 1 ? full : alone + (full - alone) * (on - 1) / (kPerCu[kind] - 1);
}
// until the last of `tiles` is done
long long rounds_ns(int kind, long long tiles, long long steps, bool stats) {
  const long long slots = kCus * kPerCu[kind], rest = tiles % slots;
  return tiles / slots * tile_ns(kind, steps, stats, kPerCu[kind]) + (rest ? tile_ns(kind, steps, stats, (rest + kCus - 1) / kCus) : 0);
}

// The tiles that are done first.
int pick_tiles(long long m, long long n, long long steps, bool stats) {
  int best = 0;
  long long least = -1;
  for (int kind = 0; kind < kTileKinds; ++kind) {
    const long long c = rounds_ns(kind, tiles_of(kind, m, n), steps, stats);
    if (least < 0 || c < least) {
      least = c;
      best = kind;
    }
  }
  return best;
}

// dh and dT of a piece of V rows, which share a launch: tiles of both (from `first` on), and the shares in which dh's long contraction is done where it
// has few tiles: each adds a slice of N x D sums that is written and read once.  At most `most` workgroups fit a CU; row_ns(kind, steps, on), row_tiles(kind):
// ns of a tile of dh, and how many.  Returns ns.
template <class Ns, class Tiles>
long long pick_shares(long long N, long long V, long long D, int parts, int first, long long most, long long steps, Ns&& row_ns, Tiles&& row_tiles, int* kind, int* slices) {
  long long least = -1;
  const long long table_steps = steps_of(N, parts);
  for (int k = first; k < kTileKinds; ++k)
    for (int s = 1; s <= 32 && (s == 1 || steps / s >= 8); ++s) {
      const long long n1 = row_tiles(k) * s, n2 = tiles_of(k, D, V), per = std::min(most, kPerCu[k]), slots = kCus * per, row_steps = (steps + s - 1) / s;
      const long long on = std::min(per, (n1 + n2 + kCus - 1) / kCus);
      const long long rows = row_ns(k, row_steps, on), table = tile_ns(k, table_steps, false, on);
      // the longest, if all have a place at once; else dh's rounds, or the CUs' work in all and the end of the last tiles, dT's
      long long c = std::max(rows, table);
      if (n1 + n2 > slots) c = std::max((n1 + slots - 1) / slots * rows, (n1 * rows + n2 * table) / slots + tile_ns(k, table_steps, false, 1) / 2);
      c += N * D * 8 * (s - 1) / 4000;
      if (least < 0 || c < least) {
        least = c;
        *kind = k;
        *slices = s;
      }
    }
  return least;
}
void pick_grads(long long N, long long V, long long D, int* kind, int* slices) {
  pick_shares(N, V, D, 1, 0, 3, steps_of(V, 1), [](int k, long long steps, long long on) { return tile_ns(k, steps, false, on); },
              [&](int k) { return tiles_of(k, D, N); }, kind, slices);
}

// f(S{}) for the shape of a kind.
template <class F>
hipError_t with_tiles(int kind, F&& f) {
  if (kind == k256x256) return f(Shape<4, 4, 2, 2, 4>{});
  if (kind == k256x128) return f(Shape<4, 2, 2, 2, 3>{});
  if (kind == k256x64) return f(Shape<2, 2, 4, 1, 4>{});
  return f(Shape<2, 1, 2, 2, 4>{});
}

template <class T, int EPI>
hipError_t launch_product(const ProductArgs& g, int kind, hipStream_t s) {
  return with_tiles(kind, [&](auto shape) {
    hipLaunchKernelGGL((kan_vocab_product_kernel<T, true, true, EPI, decltype(shape)>), dim3((unsigned)tiles_of(kind, g.m, g.n)), dim3(kThreads), 0, s, g);
    return hipGetLastError();
  });
}

template <class T>
hipError_t launch_grads(const ProductArgs& rows, const ProductArgs& table, int kind, hipStream_t s) {
  // (a multiple of eight, so that the second product's workgroups find their XCDs as the first's do)
  const unsigned row_blocks = (unsigned)((tiles_of(kind, rows.m, rows.n) * rows.splits + 7) / 8 * 8);
  return with_tiles(kind, [&](auto shape) {
    hipLaunchKernelGGL((kan_vocab_grads_kernel<T, decltype(shape)>), dim3(row_blocks + (unsigned)tiles_of(kind, table.m, table.n)), dim3(kThreads), 0, s, rows,
                       table, row_blocks);
    return hipGetLastError();
  });
}

template <int EPI>
hipError_t launch_few(const ProductArgs& g, hipStream_t s) {
  hipLaunchKernelGGL((kan_vocab_few_kernel<EPI>), dim3((unsigned)(g.m + kFewRows - 1) / kFewRows, (unsigned)(g.n + 31) / 32), dim3(kThreads), 0, s, g);
  return hipGetLastError();
}
hipError_t launch_few_rows(const ProductArgs& g, hipStream_t s) {
  hipLaunchKernelGGL(kan_vocab_few_rows_kernel, dim3((unsigned)(g.m + 127) / 128, (unsigned)g.splits), dim3(kThreads), 0, s, g);
  return hipGetLastError();
}

// fp32: tiles of kan_vocab_split_kernel, and the kernels for few (z: kSplitKinds stands for kan_vocab_few_kernel).
enum SplitKind : int { k128x32, k128x64s, k128x96, k128x128, k64x128, kSplitKinds };
constexpr int kSplitM[] = {128, 128, 128, 128, 64}, kSplitN[] = {32, 64, 96, 128, 128};
// ns of a step of 32 with one and two workgroups on a CU (measured on products of 30,000 x 4,000, 94,000 x 1,530, 13,000 x 1,700 and 5,000 x 3,500 with 1
// to 400 tokens; beyond about 2,300 it is the matrix cores and their power).
constexpr long long kSplitAlone[] = {1100, 1150, 1250, 1350, 1000}, kSplitFull[] = {2000, 2200, 2500, 2600, 2000};
long long split_tiles(int kind, long long m, long long n) { return ((m + kSplitM[kind] - 1) / kSplitM[kind]) * ((n + kSplitN[kind] - 1) / kSplitN[kind]); }
// z of m rows of the table and n tokens.  Few: every column takes a workgroup 10 ns, and the GPU 30 to 50 ps (the more of its 32 tokens exist the more
// cache lines of these it reads).  Loss in us, few and split: 1 x 94,000 x 1,530 141 and 171, 32 x 94,000 x 1,530 248 and 194, 32 x 1,300 x 4,000 47 and 99,
// 64 x 13,000 x 1,700 74 and 58, 200 x 2,000 x 1,024 31 and 43, 400 x 2,000 x 1,024 48 and 44.  Tiles that leave CUs idle: shares of the columns, whose sums are
// written, read and added (500 x 1,300 x 4,000 whole 146, in shares 56, 128 x 5,000 x 3,500 108 and 49).
int pick_split(long long m, long long n, long long D, int* slices) {
  const long long groups = (m + kFewRows - 1) / kFewRows * ((n + 31) / 32), steps = (D + kStep - 1) / kStep;
  int best = kSplitKinds;
  long long least = n > 1 << 20 ? INT64_MAX : D * std::max(10000ll, groups * (30 + 6 * std::min(n, 32ll) / 10)) / 1000;      // (65,536 blocks of tokens a launch)
  *slices = 1;
  for (int kind = 0; kind < kSplitKinds; ++kind)
    for (int s = 1; s <= 16 && (s == 1 || steps / s >= 8); ++s) {
      const long long tiles = split_tiles(kind, m, n) * s, rest = tiles % (2 * kCus);
      if (s > 1 && tiles > 2 * kCus) break;
      const long long c = (steps + s - 1) / s * (tiles / (2 * kCus) * kSplitFull[kind] + (rest > kCus ? kSplitFull[kind] : rest ? kSplitAlone[kind] : 0)) +
                          (s == 1 ? 0 : 6000 + m * n * 8 * s / 4000);
      if (c < least) {
        least = c;
        best = kind;
        *slices = s;
      }
    }
  return best;
}

template <bool AK, int EPI>
hipError_t launch_split(const ProductArgs& g, int kind, hipStream_t s) {
  auto launch = [&](auto shape) {
    hipLaunchKernelGGL((kan_vocab_split_kernel<AK, EPI, decltype(shape)>), dim3((unsigned)(split_tiles(kind, g.m, g.n) * g.splits)), dim3(kThreads), 0, s, g);
    return hipGetLastError();
  };
  if (kind == k128x32) return launch(SplitShape<1, 4>{});
  if (kind == k128x64s) return launch(SplitShape<2, 4>{});
  if (kind == k128x96) return launch(SplitShape<3, 4>{});
  if constexpr (AK)
    if (kind == k64x128) return launch(SplitShape<2, 2>{});
  return launch(SplitShape<4, 4>{});
}
hipError_t launch_split_grads(const ProductArgs& rows, const ProductArgs& table, int kind, hipStream_t s) {
  const unsigned row_blocks = (unsigned)((split_tiles(k128x128, rows.m, rows.n) * rows.splits + 7) / 8 * 8);
  auto launch = [&](auto shape) {
    hipLaunchKernelGGL((kan_vocab_split_grads_kernel<SplitShape<4, 4>, decltype(shape)>), dim3(row_blocks + (unsigned)tiles_of(kind, table.m, table.n)), dim3(kThreads), 0, s,
                       rows, table, row_blocks);
    return hipGetLastError();
  };
  if (kind == k256x128) return launch(Shape<4, 2, 2, 2, 3>{});
  if (kind == k256x64) return launch(Shape<2, 2, 4, 1, 4>{});
  return launch(Shape<2, 1, 2, 2, 4>{});
}
// z, in slices or at once, and what becomes of it.
template <int EPI>
hipError_t launch_fp32(const ProductArgs& g, int kind, int slices, float* sums, hipStream_t s) {
  if (kind == kSplitKinds) return launch_few<EPI>(g, s);
  if (slices == 1) return launch_split<true, EPI>(g, kind, s);
  ProductArgs z = g;
  z.splits = slices;
  z.out = sums;
  z.out_stride = (g.m + 3) / 4 * 4;
  z.out_slice = z.out_stride * g.n;
  z.out_dtype = KAN_F32;
  const hipError_t e = launch_split<true, kGradRows>(z, kind, s);
  if (e != hipSuccess) return e;
  const unsigned chunks = (unsigned)(g.m + kSumRows - 1) / kSumRows;
  hipLaunchKernelGGL((kan_vocab_sums_kernel<EPI>), dim3(chunks * ((unsigned)(g.n + 3) / 4)), dim3(kThreads), 0, s, z, (const float*)sums, slices, chunks);
  return hipGetLastError();
}

struct Plan {
  int parts;
  bool pack_table, pack_rows; // the table's rows, h go through the workspace
  long long width;            // columns of packed rows
  int piece, pieces;          // rows of the table that are dealt with at a time
  int slices, z_slices;       // of dh; fp32: of z
  int z_kind, rows_kind;      // tiles of z, of dh (fp32: SplitKind, kSplitKinds for few; else dh has dT's)
  int grad_kind;              // tiles of dT
  bool together;              // fp32: dh and dT in one launch
  int stat_rows;              // of the table that share statistics
  size_t h, table, sums, stats, list, target, lse, weight, scalars, ds, dh, bytes;
};

Plan make_plan(long long N, int V, int D, int dtype, bool backward) {
  Plan p = {};
  const bool fp32 = dtype == KAN_F32;
  p.parts = fp32 ? 3 : 1;
  p.pack_table = !fp32 && D % 8 != 0;
  p.pack_rows = fp32 || p.pack_table;
  p.width = ((long long)D + 63) / 64 * 64;
  const long long all = ((long long)V + kVocabStep - 1) / kVocabStep * kVocabStep;
  long long piece = all;
  auto limit = [&](long long budget, long long row_bytes) { piece = std::min(piece, std::max(1ll, budget / (row_bytes * kVocabStep)) * kVocabStep); };
  // Packed pieces that the memory-side cache holds.
  if (p.pack_table) limit(kPackBytes, p.width * 2);
  // (fewer than 2^24 workgroups a launch, whose threads have 32 bits: tiles of 128 x 64, fp32: 32 rows)
  limit(1ll << 36, N);
  limit(fp32 ? 1ll << 28 : 1ll << 30, 1);
  if (backward) {
    limit(kPieceBytes, N * 2);      // (of a part)
    limit(1ll << 35, D);
    limit(1ll << 25, 1);           // (32 rows of dS: 32-bit offsets)
  }
  p.pieces = (int)((all + piece - 1) / piece);
  p.piece = (int)((all / kVocabStep + p.pieces - 1) / p.pieces * kVocabStep);       // (of one size)
  p.pieces = (int)((all + p.piece - 1) / p.piece);
  const long long rows = std::min(p.piece, V);
  if (fp32) {
    p.z_kind = pick_split(rows, N, D, &p.z_slices);
    p.stat_rows = p.z_kind == kSplitKinds ? kFewRows : p.z_slices > 1 ? kSumRows : kSplitM[p.z_kind];
  } else {
    p.z_kind = pick_tiles(rows, N, steps_of(D, 1), !backward);
    p.stat_rows = kTileM[p.z_kind];
  }
  if (backward && fp32) {
    // dh: the fewest blocks of 32 tokens, two workgroups a CU (four: 2 to 4 % longer, one: up to 20 %), slices of 256 rows of the table or more.  Narrow rows of up
    // to 32 tokens: four a CU, 64 rows or more (32 x 1,000 x 256 39 us for 44).
    p.grad_kind = pick_tiles(D, rows, steps_of(N, 3), false);
    if (N <= 32 && D <= 256) {
      p.rows_kind = kSplitKinds;
      p.slices = (int)std::max(1ll, std::min({256ll, 4ll * kCus / ((D + 127) / 128), rows / 64}));
    } else {
      p.rows_kind = N <= 32 ? k128x32 : N <= 64 ? k128x64s : (N + 95) / 96 * 3 < (N + 127) / 128 * 4 ? k128x96 : k128x128;
      p.slices = (int)std::max(1ll, std::min({128ll, 2ll * kCus / split_tiles(p.rows_kind, D, N), rows / 256}));
    }
    if (p.rows_kind == k128x128) {       // or with dT, if that is done before both launches are
      const long long tiles = split_tiles(k128x128, D, N), steps = (rows + kStep - 1) / kStep, n = tiles * p.slices;
      auto ns = [](int, long long steps, long long on) { return steps * (on > 1 ? kSplitFull[k128x128] : kSplitAlone[k128x128]) + 8000; };
      const long long apart = (n + 2 * kCus - 1) / (2 * kCus) * ns(0, steps / p.slices, n > kCus ? 2 : 1) + N * D * 8 * (p.slices - 1) / 4000 + 3000 +
                              rounds_ns(p.grad_kind, tiles_of(p.grad_kind, D, rows), steps_of(N, 3), false);
      int kind, slices;
      p.together = pick_shares(N, rows, D, 3, k256x128, 2, steps, ns, [=](int) { return tiles; }, &kind, &slices) < apart;
      if (p.together) {
        p.grad_kind = kind;
        p.slices = slices;
      }
    }
  } else if (backward) {
    pick_grads(N, rows, D, &p.grad_kind, &p.slices);
  }
  size_t at = 0;
  auto take = [&](long long bytes) {
    const size_t was = at;
    at += (size_t)(bytes + 255) / 256 * 256;
    return was;
  };
  p.h = take(backward || p.pack_rows ? p.parts * N * p.width * 2 : 0);
  p.table = take(p.pack_table ? (long long)p.piece * p.width * 2 : 0);
  p.sums = take(p.z_slices > 1 ? p.z_slices * N * (long long)p.piece * 4 : 0);
  if (!backward) {
    p.stats = take(all / p.stat_rows * N * 8);
  } else {
    p.list = take(N * 4);
    p.target = take(N * 4);
    p.lse = take(N * 4);
    p.weight = take(N * 4);
    p.scalars = take(12);
    p.ds = take(p.parts * N * (long long)p.piece * 2);
    p.dh = take((long long)p.slices * N * D * 4);
  }
  p.bytes = at;
  return p;
}

// Launches f(I{}, T{}, parts): type of the rows, of their 16-bit parts, how many.
template <class F>
hipError_t with_parts(int dtype, F&& f) {
  if (dtype == KAN_F32) return f(float{}, bf16{}, std::integral_constant<int, 3>{});
  if (dtype == KAN_F16) return f(f16{}, f16{}, std::integral_constant<int, 1>{});
  return f(bf16{}, bf16{}, std::integral_constant<int, 1>{});
}

unsigned item_blocks(long long items) { return (unsigned)std::min((items + kThreads - 1) / kThreads, 1ll << 15); }

// Rows of a, and of b (none: no rows), in the form the products take.
kan_status pack(const PackArgs& a, const PackArgs& b, int D, long long width, int dtype, hipStream_t s) {
  return run_named("kan_vocab_pack", s, [&] {
    return with_parts(dtype, [&](auto i, auto t, auto parts) {
      const unsigned first = item_blocks(a.rows * (width / 8)), second = item_blocks(b.rows * (width / 8));
      hipLaunchKernelGGL((kan_vocab_pack_kernel<decltype(i), decltype(t), decltype(parts)::value>), dim3(first + second), dim3(kThreads), 0, s, a, b, first, D,
                         (int)width);
      return hipGetLastError();
    });
  });
}

// f(T{}): the type of the 16-bit operands.
template <class F>
kan_status with_operand(int dtype, F&& f) {
  if (dtype == KAN_F16) return f(f16{});
  return f(bf16{});
}

// The rows of the table from v0 on as an operand whose k is the width, and what has to be packed for it.
Operand table_rows(const VocabArgs& a, const Plan& p, unsigned char* ws, int v0, int rows, PackArgs* job) {
  const char* const src = (const char*)a.table + (long long)v0 * a.D * float_bytes(a.dtype);
  *job = {};
  if (!p.pack_table) return {src, a.D, 0, rows, a.D};
  *job = {src, ws + p.table, rows};
  return {ws + p.table, p.width, rows * p.width, rows, (int)p.width};
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
    g.splits = 1;
    g.V = a.V;
    g.scale = a.scale;
    g.stats = (float2*)(ws + p.stats);
    kan_status st;
    g.b = p.pack_rows ? Operand{ws + p.h, p.width, a.N * p.width, (int)a.N, (int)p.width} : Operand{a.h, a.D, 0, (int)a.N, a.D};
    for (int i = 0; i < p.pieces; ++i) {
      const int v0 = i * p.piece;
      PackArgs job;
      g.v0 = v0;
      g.m = std::min(p.piece, a.V - v0);
      g.a = table_rows(a, p, ws, v0, g.m, &job);
      if (p.pack_table || (p.pack_rows && i == 0)) {
        const PackArgs rows = {a.h, ws + p.h, i == 0 ? a.N : 0};
        if ((st = pack(job, rows, a.D, p.width, a.dtype, s)) != KAN_OK) return st;
      }
      st = run_named("kan_vocab_loss", s, [&] { return p.parts == 3 ? launch_fp32<kStats>(g, p.z_kind, p.z_slices, (float*)(ws + p.sums), s) : launch_product<T, kStats>(g, p.z_kind, s); });
      if (st != KAN_OK) return st;
    }
    return run_named("kan_vocab_join", s, [&] {
      const int rows = p.stat_rows;
      const JoinArgs j = {g.stats, a.h, a.table, a.targets, a.loss, a.lse, (a.V - 1) / rows + 1, (int)a.N, a.D, a.id_dtype, (uint32_t)a.V, a.scale};
      return with_float(a.dtype, [&](auto i) {
        if (a.N <= 1024) hipLaunchKernelGGL((kan_vocab_join_kernel<decltype(i), 1>), dim3((unsigned)a.N), dim3(256), 0, s, j);
        else hipLaunchKernelGGL((kan_vocab_join_kernel<decltype(i), 16>), dim3((unsigned)((a.N + 15) / 16)), dim3(256), 0, s, j);
        return hipGetLastError();
      });
    });
  });
}

kan_status run_vocab_grad(const VocabArgs& a, hipStream_t s) {
  const Plan p = make_plan(a.N, a.V, a.D, a.dtype, true);
  unsigned char* const ws = (unsigned char*)a.ws;
  const int N = (int)a.N;
  const Index x = {(int*)(ws + p.list), (int*)(ws + p.scalars), (float*)(ws + p.scalars) + 1, (float*)(ws + p.scalars) + 2};
  const bool own_index = N <= kOwnIndex;
  const float unit = a.dtype == KAN_F32 ? 0.f : a.dtype == KAN_F16 ? kHalfUnit : 1.f;
  kan_status st = KAN_OK;
  if (!own_index) {
    st = run_named("kan_vocab_index", s, [&] {
      hipLaunchKernelGGL(kan_vocab_index_kernel, dim3(1), dim3(1024), 0, s, a.dloss, a.targets, a.id_dtype, (uint32_t)a.V, N, a.scale, unit, x);
      return hipGetLastError();
    });
    if (st != KAN_OK) return st;
  }
  TokenArgs ta = {a.h, a.targets, a.lse, a.dloss, ws + p.h, a.dh, (int*)(ws + p.target), (float*)(ws + p.lse), (float*)(ws + p.weight), x, N, a.D, (int)p.width,
                  a.id_dtype, (uint32_t)a.V, a.scale, unit, own_index, 0, {}};
  ta.blocks = own_index ? (unsigned)(N + kTokensPerBlock - 1) / kTokensPerBlock : item_blocks(N * (p.width / 8));
  return with_operand(a.dtype, [&](auto t) -> kan_status {
    typedef decltype(t) T;
    const Operand h = {ws + p.h, p.width, a.N * p.width, N, (int)p.width};
    for (int i = 0; i < p.pieces; ++i) {
      const int v0 = i * p.piece, rows = std::min(p.piece, a.V - v0);
      const long long ds_part = a.N * (long long)p.piece;
      PackArgs job;
      const Operand table = table_rows(a, p, ws, v0, rows, &job);
      if (i == 0) {
        ta.table = job;
        st = run_named("kan_vocab_tokens", s, [&] {
          return with_parts(a.dtype, [&](auto in, auto out, auto parts) {
            hipLaunchKernelGGL((kan_vocab_tokens_kernel<decltype(in), decltype(out), decltype(parts)::value>),
                               dim3(ta.blocks + item_blocks(job.rows * (p.width / 8))), dim3(kThreads), 0, s, ta);
            return hipGetLastError();
          });
        });
      } else if (p.pack_table) {
        st = pack(job, PackArgs{}, a.D, p.width, a.dtype, s);
      }
      if (st != KAN_OK) return st;
      ProductArgs g = {};
      g.count = x.count;
      g.parts = p.parts;
      g.splits = 1;
      g.v0 = v0;
      g.V = a.V;
      g.scale = a.scale;
      g.targets = ta.target;
      g.lse = ta.lse_out;
      g.weight = ta.weight;
      g.ds = ws + p.ds;
      g.ds_stride = p.piece;
      g.ds_part = ds_part;
      g.m = rows;
      g.n = N;
      g.k = a.D;
      g.a = table;
      g.b = h;
      st = run_named("kan_vocab_ds", s, [&] { return p.parts == 3 ? launch_fp32<kGradS>(g, p.z_kind, p.z_slices, (float*)(ws + p.sums), s) : launch_product<T, kGradS>(g, p.z_kind, s); });
      if (st != KAN_OK) return st;
      // dh (+)= dS T: k = rows of the piece
      ProductArgs r = g;
      r.m = a.D;
      r.k = rows;
      r.splits = p.slices;
      r.a = {table.p, table.stride, table.part, a.D, rows};
      r.b = {ws + p.ds, p.piece, ds_part, N, (rows + 7) / 8 * 8};      // (zeros behind the last row)
      r.out = ws + p.dh;
      r.out_stride = a.D;
      r.out_slice = a.N * a.D;
      r.out_dtype = KAN_F32;
      r.add = i > 0;
      // dT (+)= dS^t h: k = tokens
      g.m = a.D;
      g.n = rows;
      g.k = N;
      g.a = {h.p, h.stride, h.part, a.D, N};
      g.b = {ws + p.ds, p.piece, ds_part, rows, N};
      g.out = (char*)a.dtable + (long long)v0 * a.D * float_bytes(a.dtype);
      g.out_stride = a.D;
      g.out_dtype = a.dtype;
      g.add = a.accumulate;
      g.factor = x.factor;
      if (p.parts == 3 && !p.together) {
        st = run_named("kan_vocab_rows", s, [&] { return p.rows_kind == kSplitKinds ? launch_few_rows(r, s) : launch_split<false, kGradRows>(r, p.rows_kind, s); });
        if (st != KAN_OK) return st;
        r.m = 0;            // (then there are no tiles of it)
      }
      st = run_named("kan_vocab_grads", s, [&] { return p.together ? launch_split_grads(r, g, p.grad_kind, s) : launch_grads<T>(r, g, p.grad_kind, s); });
      if (st != KAN_OK) return st;
    }
    return run_named("kan_vocab_round", s, [&] {
      auto round = [&](auto shares) {
        constexpr int S = decltype(shares)::value;
        hipLaunchKernelGGL((kan_vocab_round_kernel<S>), dim3(item_blocks(a.N * ((a.D + 7) / 8) * S)), dim3(kThreads), 0, s, (const float*)(ws + p.dh), p.slices,
                           a.N * a.D, N, a.D, x, a.dtype, a.dh);
      };
      if (p.slices >= 4 && a.N * a.D < (1 << 19)) round(std::integral_constant<int, 8>{});
      else round(std::integral_constant<int, 1>{});
      return hipGetLastError();
    });
  });
}

}  // namespace kan

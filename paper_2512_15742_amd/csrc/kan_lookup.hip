// Rows of a table by token id, and the table's gradient.
//
//   y[n][:]       = scale * T[id_n][:]                      (an id that names no row: zeros)
//   dT[v][:] (+)= scale * sum over n with id_n = v of dy[n][:]
//
// Forward: a copy with an indirection, bound by the bytes of y and of the rows.  An item is eight columns of one token,
// four items a thread, so that the ids, then the rows of all four are on their way before the first is used.
//
// Gradient: the sums of a row are those of a run of tokens sorted by (id, position), so the order of every sum is fixed
// and no atomics add floats.  Up to kRankTokens tokens one launch finds each token's place by counting the tokens in
// front of it; beyond, a radix sort with 9 bits a pass.  The sorted order is cut into chunks of equal length, whatever
// the histogram of the ids: a chunk sums its runs in fp32, writes the rows of runs that lie within it, and leaves what
// a run has in it when the run goes on in another chunk; a last launch joins those parts in their order.  So a token
// that is a tenth of a batch costs no more than others.
//
// Measured, and the bytes at a large copy's 5.1 TB/s: 16,384 tokens of 4,096 columns, bf16 table, fp32 rows 86 us (78); gradient of a
// table of 65,536 such rows 168 us (131): 98 for the sort, beside which the whole table is written as zeros (537 MB at 5.5 TB/s),
// 64 for the sums, 9 for the joining; gradient of 65,536 rows of ten columns from 1,048,576 edges 79 us (9): 41 for the sort, whose
// launches follow one another, 28 for the sums, where a lane has one column of ten in sixteen, 14 for the joining.
#include <algorithm>
#include <type_traits>

#include "kan_tokens.hpp"

namespace kan {
namespace {

constexpr int kThreads = 256;
constexpr unsigned kMaxBlocks = 1u << 22;

// ---- forward --------------------------------------------------------------------------------------------------------
template <class T, class O, int U>
__global__ __launch_bounds__(kThreads) void kan_lookup_kernel(const T* __restrict__ table, uint32_t V, int D, const void* __restrict__ ids,
                                                              int id_dtype, long long N, float scale, O* __restrict__ y, long long blocks) {
  const uint32_t C = (uint32_t)(D + 7) / 8;              // items per row
  for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
    const long long first = b * (kThreads * U), n0 = first / C;
    const uint32_t r0 = (uint32_t)(first - n0 * C) + threadIdx.x;
    long long n[U];
    int c[U];
    uint32_t id[U];
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t local = r0 + u * kThreads, row = local / C;
      n[u] = n0 + row;
      c[u] = (int)(local - row * C) * 8;
      id[u] = n[u] < N ? row_of(ids, id_dtype, n[u], V) : V;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (id[u] < V) {
        load_cols(table + (long long)id[u] * D, c[u], D, v[u]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (n[u] >= N) continue;
      const float by = id[u] < V ? scale : 0.f;        // (0 * infinity would be no zero)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] *= by;
      store_cols(y + n[u] * D, c[u], D, v[u]);
    }
  }
}

// ---- sorting the tokens ---------------------------------------------------------------------------------------------
constexpr int kRankTokens = 8192;           // keys of all tokens in LDS
constexpr int kRankThreads = 1024;          // 64 tokens, 16 waves that share the counting
constexpr int kSortThreads = 1024;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;      // a pass; two for tables of up to 2^18 rows
constexpr int kInlineTiles = 64;            // up to here a tile adds the counts of the others itself

// Zeros for every element of the gradient: blocks blockIdx.x = first .. first + blocks - 1 of a launch.
__device__ __forceinline__ void fill_zero(unsigned char* p, long long bytes, unsigned block, unsigned blocks) {
  const long long head = min(bytes, (long long)(-(uintptr_t)p & 15u)), n16 = (bytes - head) / 16, done = head + n16 * 16;
  uint4* q = (uint4*)(p + head);
  for (long long i = (long long)block * blockDim.x + threadIdx.x; i < n16; i += (long long)blocks * blockDim.x) q[i] = uint4{0, 0, 0, 0};
  if (block == 0 && threadIdx.x < 16) {
    if (threadIdx.x < head) p[threadIdx.x] = 0;
    if (done + threadIdx.x < bytes) p[done + threadIdx.x] = 0;
  }
}

__global__ __launch_bounds__(kRankThreads) void kan_lookup_rank_kernel(const void* __restrict__ ids, int id_dtype, int N, uint32_t V,
                                                                       uint2* __restrict__ sorted, unsigned rank_blocks, unsigned char* fill, long long fill_bytes) {
  __shared__ __attribute__((aligned(16))) uint32_t sKey[kRankTokens];
  __shared__ uint32_t sCount[16][64];
  if (blockIdx.x >= rank_blocks) {
    fill_zero(fill, fill_bytes, blockIdx.x - rank_blocks, gridDim.x - rank_blocks);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int padded = (N + 63) & ~63;
#pragma unroll
  for (int i = 0; i < kRankTokens / kRankThreads; ++i) {
    const int n = i * kRankThreads + threadIdx.x;
    if (n < padded) sKey[n] = n < N ? row_of(ids, id_dtype, n, V) : 0xffffffffu;
  }
  __syncthreads();
  const int mine = blockIdx.x * 64 + lane;       // (blocks are of whole runs of 64: mine < padded)
  const uint32_t key = sKey[mine];
  uint32_t count = 0;
  // Tokens in front of the 64: equal keys count; behind: they do not; among them: by position.
  const int quads = padded / 4, from = blockIdx.x * 16, to = from + 16;
  const uint4* const k4 = (const uint4*)sKey;
#pragma unroll 4
  for (int q = wave; q < from; q += 16) {
    const uint4 k = k4[q];
    count += (k.x <= key) + (k.y <= key) + (k.z <= key) + (k.w <= key);
  }
#pragma unroll 4
  for (int q = to + wave; q < quads; q += 16) {
    const uint4 k = k4[q];
    count += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
  }
  {
    const uint4 k = k4[from + wave];
    const int at = (from + wave) * 4;
    count += (k.x < key || (k.x == key && at < mine)) ? 1u : 0u;
    count += (k.y < key || (k.y == key && at + 1 < mine)) ? 1u : 0u;
    count += (k.z < key || (k.z == key && at + 2 < mine)) ? 1u : 0u;
    count += (k.w < key || (k.w == key && at + 3 < mine)) ? 1u : 0u;
  }
  sCount[wave][lane] = count;
  __syncthreads();
  if (wave == 0 && mine < N) {
    uint32_t place = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) place += sCount[w][lane];
    sorted[place] = make_uint2(key, (uint32_t)mine);
  }
}

// How often each digit occurs in each tile of `per` x 1024 keys.
__global__ __launch_bounds__(kSortThreads) void kan_lookup_count_kernel(const void* __restrict__ ids, int id_dtype, const uint2* __restrict__ pairs,
                                                                        long long N, uint32_t V, int shift, int per, uint32_t* __restrict__ counts,
                                                                        unsigned tiles, unsigned char* fill, long long fill_bytes) {
  __shared__ uint32_t sHist[kDigits];
  if (blockIdx.x >= tiles) {
    fill_zero(fill, fill_bytes, blockIdx.x - tiles, gridDim.x - tiles);
    return;
  }
  if (threadIdx.x < kDigits) sHist[threadIdx.x] = 0;
  __syncthreads();
  const long long first = (long long)blockIdx.x * per * kSortThreads;
#pragma unroll 4
  for (int r = 0; r < per; ++r) {
    const long long n = first + r * kSortThreads + threadIdx.x;
    if (n < N) atomicAdd(&sHist[((pairs ? pairs[n].x : row_of(ids, id_dtype, n, V)) >> shift) & (kDigits - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kDigits) counts[(size_t)blockIdx.x * kDigits + threadIdx.x] = sHist[threadIdx.x];
}

// counts[tile][digit] -> keys of that digit in the tiles in front; their sum over all tiles behind the last tile's row.
// A workgroup has 16 digits, 64 threads share the tiles of each.
__global__ __launch_bounds__(kSortThreads) void kan_lookup_scan_kernel(uint32_t* __restrict__ counts, unsigned tiles) {
  __shared__ uint32_t sSum[64][17];
  const unsigned digit = blockIdx.x * 16 + (threadIdx.x & 15), t = threadIdx.x >> 4, per = (tiles + 63) / 64;
  const unsigned a = min(tiles, t * per), b = min(tiles, a + per);
  uint32_t sum = 0;
#pragma unroll 8
  for (unsigned i = a; i < b; ++i) sum += counts[(size_t)i * kDigits + digit];
  sSum[t][threadIdx.x & 15] = sum;
  __syncthreads();
  uint32_t before = 0;
  for (unsigned i = 0; i < t; ++i) before += sSum[i][threadIdx.x & 15];
  for (unsigned i = a; i < b; ++i) {
    const uint32_t c = counts[(size_t)i * kDigits + digit];
    counts[(size_t)i * kDigits + digit] = before;
    before += c;
  }
  if (t == 63) counts[(size_t)tiles * kDigits + digit] = before;
}

// One pass of the sort: pairs (key, position) that agree in the digit keep their order.  A wave takes 64 PER pairs in a row, 64
// at a time: lanes of equal digits find each other with a ballot per bit, a counter per wave and digit carries on.  The tile is
// sorted in LDS first, so that neighbouring lanes write neighbouring places.
template <int PER>
__global__ __launch_bounds__(kSortThreads) void kan_lookup_scatter_kernel(const void* __restrict__ ids, int id_dtype, const uint2* __restrict__ in,
                                                                          long long N, uint32_t V, int shift, const uint32_t* __restrict__ counts,
                                                                          unsigned tiles, int scanned, uint2* __restrict__ out, unsigned char* fill,
                                                                          long long fill_bytes) {
  __shared__ uint32_t sOff[16][kDigits];
  __shared__ uint32_t sPart[2][kDigits];
  __shared__ uint32_t sWave[2][8];
  __shared__ uint32_t sTo[kDigits];
  __shared__ uint2 sPair[PER * kSortThreads];
  if (blockIdx.x >= tiles) {
    fill_zero(fill, fill_bytes, blockIdx.x - tiles, gridDim.x - tiles);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < 16 * kDigits; i += kSortThreads) (&sOff[0][0])[i] = 0;
  const long long tile = (long long)blockIdx.x * PER * kSortThreads, first = tile + wave * (64 * PER) + lane;
  uint2 pair[PER];
  uint32_t rank[PER];
#pragma unroll
  for (int r = 0; r < PER; ++r) {
    const long long n = first + r * 64;
    pair[r] = n >= N ? make_uint2(0u, 0u) : (in ? in[n] : make_uint2(row_of(ids, id_dtype, n, V), (uint32_t)n));
  }
  // keys of a digit in all tiles, and in those in front of this one
  uint32_t total = 0, before = 0;
  {
    const int digit = tid & (kDigits - 1), part = tid >> kDigitBits;
    if (scanned) {
      if (part == 0) {
        total = counts[(size_t)tiles * kDigits + digit];
        before = counts[(size_t)blockIdx.x * kDigits + digit];
      }
    } else {
#pragma unroll 8
      for (unsigned i = part; i < tiles; i += 2) {
        const uint32_t c = counts[(size_t)i * kDigits + digit];
        total += c;
        before += i < blockIdx.x ? c : 0u;
      }
    }
    if (part == 1) {
      sPart[0][digit] = total;
      sPart[1][digit] = before;
    }
  }
  __syncthreads();
  volatile uint32_t* const mine = sOff[wave];
#pragma unroll
  for (int r = 0; r < PER; ++r) {
    const bool live = first + r * 64 < N;
    const uint32_t digit = (pair[r].x >> shift) & (kDigits - 1);
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
      const uint64_t m = __ballot((digit >> b) & 1u);
      same &= (digit >> b) & 1u ? m : ~m;
    }
    const uint32_t at = live ? mine[digit] : 0u;
    rank[r] = at + __popcll(same & ((1ull << lane) - 1));
    __builtin_amdgcn_wave_barrier();
    if (live && (same >> lane) == 1ull) mine[digit] = rank[r] + 1;       // the last of its lanes
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  uint32_t here = 0, scan_all = 0, scan_here = 0;      // keys of this digit in the tile; of it and of smaller ones in its wave
  if (tid < kDigits) {
    total += sPart[0][tid];
    before += sPart[1][tid];
#pragma unroll
    for (int w = 0; w < 16; ++w) here += sOff[w][tid];
    scan_all = total;
    scan_here = here;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(scan_all, d), q = __shfl_up(scan_here, d);
      if (lane >= d) {
        scan_all += o;
        scan_here += q;
      }
    }
    if (lane == 63) {
      sWave[0][wave] = scan_all;
      sWave[1][wave] = scan_here;
    }
  }
  __syncthreads();
  if (tid < kDigits) {
    uint32_t all = before + scan_all - total, at = scan_here - here;
    for (int w = 0; w < wave; ++w) {
      all += sWave[0][w];
      at += sWave[1][w];
    }
    sTo[tid] = all - at;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      const uint32_t c = sOff[w][tid];
      sOff[w][tid] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < PER; ++r)
    if (first + r * 64 < N) sPair[sOff[wave][(pair[r].x >> shift) & (kDigits - 1)] + rank[r]] = pair[r];
  __syncthreads();
  const int live = (int)min((long long)PER * kSortThreads, N - tile);
#pragma unroll
  for (int r = 0; r < PER; ++r) {
    const int i = r * kSortThreads + tid;
    if (i < live) {
      const uint2 p = sPair[i];
      out[sTo[(p.x >> shift) & (kDigits - 1)] + (uint32_t)i] = p;
    }
  }
}

// ---- sums over runs of the sorted tokens ----------------------------------------------------------------------------
struct SumArgs {
  const uint2* sorted;       // (row, token)
  float* parts;              // [chunk][2][D]: what the chunk has of the run that began in front of it, and of the one that
                             // goes on behind it (a run that does both: the first)
  long long N;
  uint32_t V;
  int D, chunk, lanes;       // tokens per chunk (a multiple of 8), lanes per chunk and column tile
  int accumulate;
  float scale;
};

template <int VEC, class O>
__device__ __forceinline__ void put(O* dst, int c, int D, float (&sum)[VEC], const SumArgs& a) {
  if constexpr (VEC == 8) {
    float old[8];
    if (a.accumulate) load_cols(dst, c, D, old);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = a.accumulate ? old[i] + sum[i] * a.scale : sum[i] * a.scale;
    store_cols(dst, c, D, sum);
  } else {
    dst[c] = (O)(a.accumulate ? (float)dst[c] + sum[0] * a.scale : sum[0] * a.scale);
  }
}

// Wide rows: eight columns a lane, a wave has a chunk of its own, whose keys and positions are scalars.  Narrow rows: a lane
// has one column, and 64 / lanes chunks share a wave.  The keys of the next eight tokens are on their way while eight rows are.
template <class I, class O, bool WIDE>
__global__ __launch_bounds__(kThreads) void kan_lookup_sum_kernel(const I* __restrict__ dy, O* __restrict__ dtable, const SumArgs a) {
  constexpr int VEC = WIDE ? 8 : 1;
  const int lanes = WIDE ? 64 : a.lanes;
  const int lane = threadIdx.x % lanes;
  const int group = WIDE ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / lanes;
  const long long chunk = (long long)blockIdx.x * (kThreads / lanes) + group;
  const int c = (blockIdx.y * lanes + lane) * VEC;
  const long long first = chunk * a.chunk, end = min(a.N, first + a.chunk);
  if (first >= a.N || c >= a.D) return;
  float sum[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
  uint32_t run = a.sorted[first].x;
  bool from_before = first > 0 && a.sorted[first - 1].x == run;
  float* const parts = a.parts + chunk * 2 * a.D;
  auto flush = [&](bool goes_on) {
    if (run < a.V) {
      if (from_before || goes_on) {
        float* const p = parts + (from_before ? 0 : a.D);
        if constexpr (WIDE) store_cols(p, c, a.D, sum);
        else p[c] = sum[0];
      } else {
        put<VEC>(dtable + (long long)run * a.D, c, a.D, sum, a);
      }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
    from_before = false;
  };
  typedef I Raw __attribute__((ext_vector_type(VEC)));
  const bool whole = c + VEC <= a.D;
  uint32_t key[2][8];
  Raw raw[2][8];
  auto fetch = [&](long long p, int b) {       // (the arrays are padded: sixteen tokens behind the last one)
    uint32_t at[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint2 t = a.sorted[p + u];
      key[b][u] = t.x;
      at[u] = t.y;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool live = p + u < end && key[b][u] < a.V;
      const I* const row = dy + (long long)(live ? at[u] : 0u) * a.D;
      if (whole) {
        __builtin_memcpy(&raw[b][u], row + c, sizeof(Raw));
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) raw[b][u][i] = c + i < a.D ? row[c + i] : (I)0.f;
      }
    }
  };
  auto take = [&](long long p, int b) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p + u < end) {
        if (key[b][u] != run) {
          flush(false);
          run = key[b][u];
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += (float)raw[b][u][i];
      }
    }
  };
  fetch(first, 0);
  for (long long p = first; p < end; p += 16) {
    if (p + 8 < end) fetch(p + 8, 1);
    take(p, 0);
    if (p + 16 < end) fetch(p + 16, 0);
    if (p + 8 < end) take(p + 8, 1);
  }
  flush(end < a.N && a.sorted[end].x == run);
}

// The runs that begin in a chunk and go on behind it: their parts, in order.  A group of lanes looks at a chunk and adds the
// parts of a run that reaches up to kShort chunks further by itself; longer ones are left to all groups of the workgroup
// together, a share of the parts each.
constexpr int kJoinThreads = 1024, kShort = 16;
template <class O, bool WIDE>
__global__ __launch_bounds__(kJoinThreads) void kan_lookup_join_kernel(O* __restrict__ dtable, const SumArgs a, long long chunks) {
  constexpr int VEC = WIDE ? 8 : 1;
  __shared__ float sSum[kJoinThreads * VEC];
  __shared__ uint32_t sLong[kJoinThreads];        // chunks (of this workgroup) whose run is long
  const int lanes = WIDE ? 64 : a.lanes, groups = kJoinThreads / lanes;
  const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
  const int c = (blockIdx.y * lanes + lane) * VEC;
  const long long chunk = (long long)blockIdx.x * groups + group;
  const long long first = min(chunk, chunks - 1) * a.chunk, end = first + a.chunk;
  const uint32_t run = a.sorted[min(end, a.N - 1)].x, last_in = a.sorted[min(end, a.N) - 1].x, first_in = a.sorted[first].x, in_front = a.sorted[max(first - 1, 0ll)].x;
  const bool mine = chunk < chunks && end < a.N && run < a.V && last_in == run && !(first > 0 && first_in == run && in_front == run);
  int reach = 1;                  // chunks behind this one that the run is known to reach
  for (int i = 0; i < kShort; i += lanes) {
    const long long k = chunk + 2 + i + lane;
    const uint64_t on = __ballot(mine && k < chunks && a.sorted[min(k, chunks - 1) * a.chunk].x == run) >> (threadIdx.x & 63 & ~(lanes - 1));
    const int n = min(lanes, on == ~0ull ? 64 : __ffsll((long long)~on) - 1);
    reach += reach == 1 + i ? n : 0;
  }
  const bool far = mine && reach > kShort;
  if (lane == 0) sLong[group] = far ? 1u : 0u;
  auto add = [&](float (&sum)[VEC], long long from, long long p0, long long p1) {
    for (long long p = p0; p < p1; p += 8) {
      float v[8][VEC];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const long long q = min(p + u, p1 - 1);
        const float* const src = a.parts + (from + q) * 2 * a.D + (q == 0 ? a.D : 0);
        if constexpr (WIDE) load_cols(src, c, a.D, v[u]);
        else v[u][0] = src[c];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += p + u < p1 ? v[u][i] : 0.f;
    }
  };
  float sum[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
  if (mine && !far && c < a.D) {
    add(sum, chunk, 0, reach + 1);
    put<VEC>(dtable + (long long)run * a.D, c, a.D, sum, a);
  }
  __syncthreads();
  for (int g = 0; g < groups; ++g) {
    if (!sLong[g]) continue;
    const long long from = (long long)blockIdx.x * groups + g;
    const uint32_t key = a.sorted[(from + 1) * a.chunk].x;
    long long last = from + 1, past = chunks;       // the run reaches `last` and does not reach `past`
    while (past - last > 1) {                       // a 64th of what is between them is left
      const long long step = (past - last + 63) / 64, k = last + ((threadIdx.x & 63) + 1) * step;
      const uint64_t on = __ballot(k < past && a.sorted[min(k, chunks - 1) * a.chunk].x == key);
      const int n = __popcll(on);
      past = min(past, last + (n + 1) * step);
      last += n * step;
    }
    const long long parts = last - from + 1, per = (parts + groups - 1) / groups;
    const long long p0 = group * per, p1 = c < a.D ? min(parts, p0 + per) : 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
    add(sum, from, p0, p1);
#pragma unroll
    for (int i = 0; i < VEC; ++i) sSum[(group * VEC + i) * lanes + lane] = sum[i];
    __syncthreads();
    if (group == 0 && c < a.D) {
      const int busy = (int)min((long long)groups, (parts + per - 1) / per);
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
      for (int h = 0; h < busy; ++h)
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += sSum[(h * VEC + i) * lanes + lane];
      put<VEC>(dtable + (long long)key * a.D, c, a.D, sum, a);
    }
    __syncthreads();
  }
}

// ---- plan of a gradient ----------------------------------------------------------------------------------------------
struct GradPlan {
  bool rank;                 // one counting launch in place of the radix sort
  unsigned tiles;            // radix sort, in tiles of per x 1024 keys
  int passes, per;
  int chunk, lanes;
  bool wide;
  long long chunks;
  size_t sorted[2], counts, parts, bytes;      // byte offsets of the workspace
};

GradPlan plan_grad(int V, int D, long long N) {
  GradPlan p = {};
  p.rank = N <= kRankTokens;
  // Small tiles while they leave CUs idle; a tile's counts are added by every other one, or by a launch of their own.
  p.per = N <= (1 << 20) ? 4 : 8;
  p.tiles = (unsigned)((N + p.per * kSortThreads - 1) / (p.per * kSortThreads));
  p.passes = 0;
  if (!p.rank)
    while (p.passes < 4 && ((uint64_t)V >> (kDigitBits * p.passes)) != 0) ++p.passes;       // (V itself is the key of ids that name no row)
  // Chunks of 16 tokens while there are few, so that many waves share them; of 32 and 64 where that leaves 1024 and 2048 waves
  // busy (fewer rows are written in parts: 66 against 70 us for 16,384 tokens x 4096); longer ones where there would be more
  // than 2^14 of them, so that a run of most tokens has few parts.
  p.chunk = N / 64 * ((D + 511) / 512) >= 2048 ? 64 : N / 32 * ((D + 511) / 512) >= 1024 ? 32 : 16;
  while ((N + p.chunk - 1) / p.chunk > (1 << 14)) p.chunk *= 2;
  p.chunks = (N + p.chunk - 1) / p.chunk;
  // Up to 64 columns a lane takes one; wider rows: eight a lane, sixteen-byte loads of 16-bit types.
  p.wide = D > 64;
  p.lanes = 1;
  while (p.lanes < D && p.lanes < 64) p.lanes *= 2;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) / 256 * 256;
    return was;
  };
  const size_t list = ((size_t)N + 16) * 8;
  for (int i = 0; i < (p.rank ? 1 : 2); ++i) p.sorted[i] = take(list);
  p.counts = take(p.rank ? 0 : ((size_t)p.tiles + 1) * kDigits * 4);
  p.parts = take((size_t)p.chunks * 2 * D * 4);
  p.bytes = at;
  return p;
}

}  // namespace

hipError_t launch_lookup(const LookupArgs& a, hipStream_t s) {
  const long long items = a.N * ((a.D + 7) / 8);
  return with_float(a.table_dtype, [&](auto t) {
    return with_float(a.y_dtype, [&](auto o) {
      typedef decltype(t) T;
      typedef decltype(o) O;
      // one item a thread until every CU has four workgroups, then four
      if (items <= 256 * 4 * kThreads) {
        const long long blocks = (items + kThreads - 1) / kThreads;
        hipLaunchKernelGGL((kan_lookup_kernel<T, O, 1>), dim3((unsigned)blocks), dim3(kThreads), 0, s, (const T*)a.table, (uint32_t)a.V, a.D,
                           a.ids, a.id_dtype, a.N, a.scale, (O*)a.y, blocks);
      } else {
        const long long blocks = (items + 4 * kThreads - 1) / (4 * kThreads);
        hipLaunchKernelGGL((kan_lookup_kernel<T, O, 4>), dim3((unsigned)std::min(blocks, (long long)kMaxBlocks)), dim3(kThreads), 0, s,
                           (const T*)a.table, (uint32_t)a.V, a.D, a.ids, a.id_dtype, a.N, a.scale, (O*)a.y, blocks);
      }
      return hipGetLastError();
    });
  });
}

size_t lookup_grad_workspace(int V, int D, long long N) { return N == 0 ? 0 : plan_grad(V, D, N).bytes; }

kan_status run_lookup_grad(const LookupGradArgs& a, hipStream_t s) {
  const long long table_bytes = (long long)a.V * a.D * float_bytes(a.dtable_dtype);
  const long long fill = a.accumulate ? 0 : table_bytes;
  const unsigned fill_blocks = (unsigned)std::min(2048ll, (fill + 16 * kSortThreads - 1) / (16 * kSortThreads));
  if (a.N == 0) {
    if (!fill) return KAN_OK;
    return run_named("kan_lookup_fill", s, [&] {
      hipLaunchKernelGGL(kan_lookup_rank_kernel, dim3(fill_blocks), dim3(kRankThreads), 0, s, a.ids, a.id_dtype, 0, (uint32_t)a.V,
                         (uint2*)nullptr, 0u, (unsigned char*)a.dtable, fill);
      return hipGetLastError();
    });
  }
  const GradPlan p = plan_grad(a.V, a.D, a.N);
  unsigned char* const ws = (unsigned char*)a.ws;
  uint2* const sorted[2] = {(uint2*)(ws + p.sorted[0]), (uint2*)(ws + p.sorted[1])};
  int now = 0;
  kan_status st;
  if (p.rank) {
    const unsigned blocks = (unsigned)((a.N + 63) / 64);
    st = run_named("kan_lookup_rank", s, [&] {
      hipLaunchKernelGGL(kan_lookup_rank_kernel, dim3(blocks + fill_blocks), dim3(kRankThreads), 0, s, a.ids, a.id_dtype, (int)a.N,
                         (uint32_t)a.V, sorted[0], blocks, (unsigned char*)a.dtable, fill);
      return hipGetLastError();
    });
    if (st != KAN_OK) return st;
  } else {
    uint32_t* const counts = (uint32_t*)(ws + p.counts);
    // The zeros are written beside the sort, whose launches leave most of the GPU idle: a share in each.
    const int shares = 2 * p.passes;
    const long long share = (fill / shares + 255) / 256 * 256;
    for (int pass = 0; pass < p.passes; ++pass) {
      const uint2* const in = pass == 0 ? nullptr : sorted[now];
      const int to = pass == 0 ? 0 : now ^ 1;
      unsigned char* part[2];
      long long bytes[2];
      unsigned fb[2];
      for (int k = 0; k < 2; ++k) {
        const int which = 2 * pass + k;
        const long long from = std::min(fill, which * share);
        part[k] = (unsigned char*)a.dtable + from;
        bytes[k] = which == shares - 1 ? fill - from : std::min(share, fill - from);
        fb[k] = (unsigned)std::min(1024ll, (bytes[k] + 16 * kSortThreads - 1) / (16 * kSortThreads));
      }
      st = run_named("kan_lookup_sort", s, [&] {
        hipLaunchKernelGGL(kan_lookup_count_kernel, dim3(p.tiles + fb[0]), dim3(kSortThreads), 0, s, a.ids, a.id_dtype, in, a.N, (uint32_t)a.V,
                           kDigitBits * pass, p.per, counts, p.tiles, part[0], bytes[0]);
        const bool scan = p.tiles > kInlineTiles;
        if (scan) hipLaunchKernelGGL(kan_lookup_scan_kernel, dim3(kDigits / 16), dim3(kSortThreads), 0, s, counts, p.tiles);
        auto scatter = [&](auto per) {
          hipLaunchKernelGGL((kan_lookup_scatter_kernel<decltype(per)::value>), dim3(p.tiles + fb[1]), dim3(kSortThreads), 0, s, a.ids, a.id_dtype, in,
                             a.N, (uint32_t)a.V, kDigitBits * pass, counts, p.tiles, (int)scan, sorted[to], part[1], bytes[1]);
        };
        if (p.per == 4) scatter(std::integral_constant<int, 4>{});
        else scatter(std::integral_constant<int, 8>{});
        return hipGetLastError();
      });
      if (st != KAN_OK) return st;
      now = to;
    }
  }
  SumArgs q = {sorted[now], (float*)(ws + p.parts), a.N, (uint32_t)a.V, a.D, p.chunk, p.lanes, a.accumulate, a.scale};
  const int cols = p.lanes * (p.wide ? 8 : 1);
  const unsigned per_block = kThreads / p.lanes, col_tiles = (unsigned)((a.D + cols - 1) / cols);
  const dim3 grid((unsigned)((p.chunks + per_block - 1) / per_block), col_tiles), join((unsigned)((p.chunks + kJoinThreads / p.lanes - 1) / (kJoinThreads / p.lanes)), col_tiles);
  st = run_named("kan_lookup_sum", s, [&] {
    return with_float(a.dy_dtype, [&](auto i) {
      return with_float(a.dtable_dtype, [&](auto o) {
        typedef decltype(i) I;
        typedef decltype(o) O;
        if (p.wide) hipLaunchKernelGGL((kan_lookup_sum_kernel<I, O, true>), grid, dim3(kThreads), 0, s, (const I*)a.dy, (O*)a.dtable, q);
        else hipLaunchKernelGGL((kan_lookup_sum_kernel<I, O, false>), grid, dim3(kThreads), 0, s, (const I*)a.dy, (O*)a.dtable, q);
        return hipGetLastError();
      });
    });
  });
  if (st != KAN_OK || p.chunks < 2) return st;
  return run_named("kan_lookup_join", s, [&] {
    return with_float(a.dtable_dtype, [&](auto o) {
      typedef decltype(o) O;
      if (p.wide) hipLaunchKernelGGL((kan_lookup_join_kernel<O, true>), join, dim3(kJoinThreads), 0, s, (O*)a.dtable, q, p.chunks);
      else hipLaunchKernelGGL((kan_lookup_join_kernel<O, false>), join, dim3(kJoinThreads), 0, s, (O*)a.dtable, q, p.chunks);
      return hipGetLastError();
    });
  });
}

}  // namespace kan

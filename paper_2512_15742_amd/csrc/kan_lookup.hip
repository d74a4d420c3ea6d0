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
// front of it; beyond, a radix sort with 8 bits a pass.  The sorted order is cut into chunks of equal length, whatever
// the histogram of the ids: a chunk sums its runs in fp32, writes the rows of runs that lie within it, and leaves what
// a run has in it when the run goes on in another chunk; a last launch joins those parts in their order.  So a token
// that is a tenth of a batch costs no more than others.
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
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] *= scale;
      store_cols(y + n[u] * D, c[u], D, v[u]);
    }
  }
}

// ---- sorting the tokens ---------------------------------------------------------------------------------------------
constexpr int kRankTokens = 8192;           // keys of all tokens in LDS
constexpr int kRankThreads = 1024;          // 64 tokens, 16 waves that share the counting
constexpr int kSortThreads = 1024, kSortPer = 16, kSortTile = kSortThreads * kSortPer;
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
                                                                       uint32_t* __restrict__ order, uint32_t* __restrict__ keys,
                                                                       unsigned rank_blocks, unsigned char* fill, long long fill_bytes) {
  __shared__ __attribute__((aligned(16))) uint32_t sKey[kRankTokens];
  __shared__ uint32_t sCount[16][64];
  if (blockIdx.x >= rank_blocks) {
    fill_zero(fill, fill_bytes, blockIdx.x - rank_blocks, gridDim.x - rank_blocks);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int padded = (N + 63) & ~63;
  for (int i = threadIdx.x; i < padded; i += kRankThreads) sKey[i] = i < N ? row_of(ids, id_dtype, i, V) : 0xffffffffu;
  __syncthreads();
  const int mine = blockIdx.x * 64 + lane;       // (blocks are of whole runs of 64: mine < padded)
  const uint32_t key = sKey[mine];
  uint32_t count = 0;
  const int quads = padded / 4;
  for (int q = wave; q < quads; q += 16) {
    const uint4 k = ((const uint4*)sKey)[q];
    const int at = q * 4;
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
    order[place] = (uint32_t)mine;
    keys[place] = key;
  }
}

// How often each digit occurs in each tile of keys.
__global__ __launch_bounds__(kSortThreads) void kan_lookup_count_kernel(const void* __restrict__ ids, int id_dtype, const uint32_t* __restrict__ keys,
                                                                        long long N, uint32_t V, int shift, uint32_t* __restrict__ counts,
                                                                        unsigned tiles, unsigned char* fill, long long fill_bytes) {
  __shared__ uint32_t sHist[256];
  if (blockIdx.x >= tiles) {
    fill_zero(fill, fill_bytes, blockIdx.x - tiles, gridDim.x - tiles);
    return;
  }
  if (threadIdx.x < 256) sHist[threadIdx.x] = 0;
  __syncthreads();
  const long long first = (long long)blockIdx.x * kSortTile;
#pragma unroll 4
  for (int r = 0; r < kSortPer; ++r) {
    const long long n = first + r * kSortThreads + threadIdx.x;
    if (n < N) atomicAdd(&sHist[((keys ? keys[n] : row_of(ids, id_dtype, n, V)) >> shift) & 255u], 1u);
  }
  __syncthreads();
  if (threadIdx.x < 256) counts[(size_t)blockIdx.x * 256 + threadIdx.x] = sHist[threadIdx.x];
}

// counts[tile][digit] -> keys of that digit in the tiles in front; their sum over all tiles behind the last tile's row.
__global__ __launch_bounds__(256) void kan_lookup_scan_kernel(uint32_t* __restrict__ counts, unsigned tiles) {
  __shared__ uint32_t sSum[256];
  const unsigned digit = blockIdx.x, t = threadIdx.x, per = (tiles + 255) / 256;
  const unsigned a = min(tiles, t * per), b = min(tiles, a + per);
  uint32_t sum = 0;
  for (unsigned i = a; i < b; ++i) sum += counts[(size_t)i * 256 + digit];
  sSum[t] = sum;
  __syncthreads();
  uint32_t before = 0;
  for (unsigned i = 0; i < t; ++i) before += sSum[i];
  for (unsigned i = a; i < b; ++i) {
    const uint32_t c = counts[(size_t)i * 256 + digit];
    counts[(size_t)i * 256 + digit] = before;
    before += c;
  }
  if (t == 255) counts[(size_t)tiles * 256 + digit] = before;
}

// One pass of the sort: keys that agree in the digit keep their order.  A wave takes 1024 keys in a row, 64 at a time: lanes
// of equal digits find each other with a ballot per bit, a counter per wave and digit carries on.
__global__ __launch_bounds__(kSortThreads) void kan_lookup_scatter_kernel(const void* __restrict__ ids, int id_dtype,
                                                                          const uint32_t* __restrict__ keys_in, const uint32_t* __restrict__ order_in,
                                                                          long long N, uint32_t V, int shift, const uint32_t* __restrict__ counts,
                                                                          unsigned tiles, int scanned, uint32_t* __restrict__ keys_out,
                                                                          uint32_t* __restrict__ order_out) {
  __shared__ uint32_t sOff[16][256];
  __shared__ uint32_t sPart[2][4][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < 16 * 256; i += kSortThreads) (&sOff[0][0])[i] = 0;
  // keys of a digit in all tiles, and in those in front of this one
  {
    const int digit = tid & 255, part = tid >> 8;
    uint32_t total = 0, before = 0;
    if (scanned) {
      if (part == 0) {
        total = counts[(size_t)tiles * 256 + digit];
        before = counts[(size_t)blockIdx.x * 256 + digit];
      }
    } else {
      for (unsigned i = part; i < tiles; i += 4) {
        const uint32_t c = counts[(size_t)i * 256 + digit];
        total += c;
        before += i < blockIdx.x ? c : 0u;
      }
    }
    sPart[0][part][digit] = total;
    sPart[1][part][digit] = before;
  }
  __syncthreads();
  const long long first = (long long)blockIdx.x * kSortTile + wave * (64 * kSortPer) + lane;
  uint32_t key[kSortPer], rank[kSortPer];
#pragma unroll
  for (int r = 0; r < kSortPer; ++r) {
    const long long n = first + r * 64;
    key[r] = n < N ? (keys_in ? keys_in[n] : row_of(ids, id_dtype, n, V)) : 0u;
  }
  volatile uint32_t* const mine = sOff[wave];
#pragma unroll
  for (int r = 0; r < kSortPer; ++r) {
    const bool live = first + r * 64 < N;
    const uint32_t digit = (key[r] >> shift) & 255u;
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
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
  if (tid < 256) {
    uint32_t before = 0;
    for (int p = 0; p < 4; ++p) before += sPart[1][p][tid];
    // keys of smaller digits: summed in 64 lanes of four, then within the four
    sPart[0][0][tid] += sPart[0][1][tid] + sPart[0][2][tid] + sPart[0][3][tid];
    sPart[1][0][tid] = before;
  }
  __syncthreads();
  if (tid < 256) {
    uint32_t smaller = 0;
    for (int d = 0; d < tid; ++d) smaller += sPart[0][0][d];
    uint32_t at = smaller + sPart[1][0][tid];
    for (int w = 0; w < 16; ++w) {
      const uint32_t c = sOff[w][tid];
      sOff[w][tid] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortPer; ++r) {
    const long long n = first + r * 64;
    if (n < N) {
      const uint32_t to = sOff[wave][(key[r] >> shift) & 255u] + rank[r];
      keys_out[to] = key[r];
      order_out[to] = order_in ? order_in[n] : (uint32_t)n;
    }
  }
}

// ---- sums over runs of the sorted tokens ----------------------------------------------------------------------------
struct SumArgs {
  const uint32_t *order, *keys;
  float* parts;              // [chunk][2][D]: what the chunk has of the run that began in front of it, and of the one that
                             // goes on behind it (a run that does both: the first)
  long long N;
  uint32_t V;
  int D, chunk, lanes;       // tokens per chunk (a multiple of 8), lanes per chunk and column tile
  int accumulate;
  float scale;
};

template <class O>
__device__ __forceinline__ void put_row(O* dst, int c, int cols, int D, const float* sum, float scale, int accumulate) {
  for (int i = 0; i < cols; ++i)
    if (c + i < D) dst[c + i] = (O)(accumulate ? (float)dst[c + i] + sum[i] * scale : sum[i] * scale);
}

// Narrow rows: a lane has one column and 64 / lanes chunks share a wave; wide rows: eight columns a lane.
template <class I, class O, int VEC>
__global__ __launch_bounds__(kThreads) void kan_lookup_sum_kernel(const I* __restrict__ dy, O* __restrict__ dtable, const SumArgs a) {
  const int lane = threadIdx.x % a.lanes;
  const long long chunk = (long long)blockIdx.x * (kThreads / a.lanes) + threadIdx.x / a.lanes;
  const int c = (blockIdx.y * a.lanes + lane) * VEC;
  const long long first = chunk * a.chunk, end = min(a.N, first + a.chunk);
  if (first >= a.N || c >= a.D) return;
  float sum[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
  uint32_t run = a.keys[first];
  bool from_before = first > 0 && a.keys[first - 1] == run;
  float* const parts = a.parts + chunk * 2 * a.D;
  auto flush = [&](bool goes_on) {
    if (run < a.V) {
      if (from_before || goes_on) {
        float* const p = parts + (from_before ? 0 : a.D);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (c + i < a.D) p[c + i] = sum[i];
      } else {
        O* const dst = dtable + (long long)run * a.D;
        if constexpr (VEC == 8) {
          if (c + 8 <= a.D) {
            float v[8], old[8];
            if (a.accumulate) load8(dst + c, old);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = a.accumulate ? old[i] + sum[i] * a.scale : sum[i] * a.scale;
            store8(dst + c, v);
          } else {
            put_row(dst, c, VEC, a.D, sum, a.scale, a.accumulate);
          }
        } else {
          put_row(dst, c, VEC, a.D, sum, a.scale, a.accumulate);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
    from_before = false;
  };
  for (long long p = first; p < end; p += 8) {
    uint32_t key[8], at[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {       // (the arrays are padded to a multiple of eight)
      key[u] = a.keys[p + u];
      at[u] = a.order[p + u];
    }
    float v[8][VEC];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool live = p + u < end && key[u] < a.V;
      const I* const row = dy + (long long)(live ? at[u] : 0u) * a.D;
      if constexpr (VEC == 8) {
        if (live) load_cols(row, c, a.D, v[u]);
      } else {
        if (live) v[u][0] = (float)row[c];
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p + u < end) {
        if (key[u] != run) {
          flush(false);
          run = key[u];
        }
        if (run < a.V) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) sum[i] += v[u][i];
        }
      }
    }
  }
  flush(end < a.N && a.keys[end] == run);
}

// The run that begins in a chunk and goes on behind it: its parts, in order.  16 (narrow rows) or 4 groups of lanes take a
// share of the parts each.
template <class O, int VEC>
__global__ __launch_bounds__(kThreads) void kan_lookup_join_kernel(O* __restrict__ dtable, const SumArgs a, long long chunks) {
  __shared__ float sSum[kThreads * VEC];
  const long long chunk = blockIdx.x;
  const long long end = (chunk + 1) * a.chunk;
  if (end >= a.N) return;
  const uint32_t run = a.keys[end];
  if (run >= a.V || a.keys[end - 1] != run) return;
  const long long first = chunk * a.chunk;
  if (first > 0 && a.keys[first] == run && a.keys[first - 1] == run) return;       // it began further in front
  // chunks behind this one that the run reaches
  long long last = chunk + 1;
  for (;;) {
    const long long k = last + 1 + (threadIdx.x & 63);
    const uint64_t on = __ballot(k < chunks && a.keys[k * a.chunk] == run);
    const int n = on == ~0ull ? 64 : __ffsll((long long)~on) - 1;
    last += n;
    if (n < 64) break;
  }
  const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes, groups = kThreads / a.lanes;
  const int c = (blockIdx.y * a.lanes + lane) * VEC;
  const long long parts = last - chunk + 1, per = (parts + groups - 1) / groups;
  const long long p0 = group * per, p1 = min(parts, p0 + per);
  float sum[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
#pragma unroll 4
  for (long long p = p0; p < p1; ++p) {
    const float* const src = a.parts + (chunk + p) * 2 * a.D + (p == 0 ? a.D : 0);
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] += c + i < a.D ? src[c + i] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) sSum[(group * VEC + i) * a.lanes + lane] = sum[i];
  __syncthreads();
  if (group != 0 || c >= a.D) return;
  const int busy = (int)min((long long)groups, (parts + per - 1) / per);
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
  for (int g = 0; g < busy; ++g)
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] += sSum[(g * VEC + i) * a.lanes + lane];
  put_row(dtable + (long long)run * a.D, c, VEC, a.D, sum, a.scale, a.accumulate);
}

// ---- plan of a gradient ----------------------------------------------------------------------------------------------
struct GradPlan {
  bool rank;                 // one counting launch in place of the radix sort
  unsigned tiles;            // radix sort
  int passes;
  int chunk, lanes, vec;
  long long chunks;
  size_t keys[2], order[2], counts, parts, bytes;      // byte offsets of the workspace
};

GradPlan plan_grad(int V, int D, long long N) {
  GradPlan p = {};
  p.rank = N <= kRankTokens;
  p.tiles = (unsigned)((N + kSortTile - 1) / kSortTile);
  p.passes = 0;
  if (!p.rank)
    while (p.passes < 4 && ((uint64_t)V >> (8 * p.passes)) != 0) ++p.passes;       // (V itself is the key of ids that name no row)
  // Chunks of 32 tokens; longer ones where that leaves more than 2^14 of them, so that a run of most tokens has few parts.
  p.chunk = 32;
  while ((N + p.chunk - 1) / p.chunk > (1 << 14)) p.chunk *= 2;
  p.chunks = (N + p.chunk - 1) / p.chunk;
  // Up to 64 columns a lane takes one; wider rows: eight a lane, sixteen-byte loads of 16-bit types.
  p.vec = D <= 64 ? 1 : 8;
  const int need = (D + p.vec - 1) / p.vec;
  p.lanes = 1;
  while (p.lanes < need && p.lanes < 64) p.lanes *= 2;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) / 256 * 256;
    return was;
  };
  const size_t list = ((size_t)N + 8) * 4;
  for (int i = 0; i < (p.rank ? 1 : 2); ++i) {
    p.keys[i] = take(list);
    p.order[i] = take(list);
  }
  p.counts = take(p.rank ? 0 : ((size_t)p.tiles + 1) * 256 * 4);
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
                         (uint32_t*)nullptr, (uint32_t*)nullptr, 0u, (unsigned char*)a.dtable, fill);
      return hipGetLastError();
    });
  }
  const GradPlan p = plan_grad(a.V, a.D, a.N);
  unsigned char* const ws = (unsigned char*)a.ws;
  uint32_t* keys[2] = {(uint32_t*)(ws + p.keys[0]), (uint32_t*)(ws + p.keys[1])};
  uint32_t* order[2] = {(uint32_t*)(ws + p.order[0]), (uint32_t*)(ws + p.order[1])};
  int now = 0;
  kan_status st;
  if (p.rank) {
    const unsigned blocks = (unsigned)((a.N + 63) / 64);
    st = run_named("kan_lookup_rank", s, [&] {
      hipLaunchKernelGGL(kan_lookup_rank_kernel, dim3(blocks + fill_blocks), dim3(kRankThreads), 0, s, a.ids, a.id_dtype, (int)a.N,
                         (uint32_t)a.V, order[0], keys[0], blocks, (unsigned char*)a.dtable, fill);
      return hipGetLastError();
    });
    if (st != KAN_OK) return st;
  } else {
    uint32_t* const counts = (uint32_t*)(ws + p.counts);
    for (int pass = 0; pass < p.passes; ++pass) {
      const uint32_t* const kin = pass == 0 ? nullptr : keys[now];
      const uint32_t* const oin = pass == 0 ? nullptr : order[now];
      const int to = pass == 0 ? 0 : now ^ 1;
      const unsigned fb = pass == 0 ? fill_blocks : 0;
      st = run_named("kan_lookup_sort", s, [&] {
        hipLaunchKernelGGL(kan_lookup_count_kernel, dim3(p.tiles + fb), dim3(kSortThreads), 0, s, a.ids, a.id_dtype, kin, a.N, (uint32_t)a.V,
                           8 * pass, counts, p.tiles, (unsigned char*)a.dtable, fill);
        const bool scan = p.tiles > kInlineTiles;
        if (scan) hipLaunchKernelGGL(kan_lookup_scan_kernel, dim3(256), dim3(256), 0, s, counts, p.tiles);
        hipLaunchKernelGGL(kan_lookup_scatter_kernel, dim3(p.tiles), dim3(kSortThreads), 0, s, a.ids, a.id_dtype, kin, oin, a.N, (uint32_t)a.V,
                           8 * pass, counts, p.tiles, (int)scan, keys[to], order[to]);
        return hipGetLastError();
      });
      if (st != KAN_OK) return st;
      now = to;
    }
  }
  SumArgs q = {order[now], keys[now], (float*)(ws + p.parts), a.N, (uint32_t)a.V, a.D, p.chunk, p.lanes, a.accumulate, a.scale};
  const unsigned per_block = kThreads / p.lanes, col_tiles = (unsigned)((a.D + p.lanes * p.vec - 1) / (p.lanes * p.vec));
  const dim3 grid((unsigned)((p.chunks + per_block - 1) / per_block), col_tiles), join((unsigned)p.chunks, col_tiles);
  st = run_named("kan_lookup_sum", s, [&] {
    return with_float(a.dy_dtype, [&](auto i) {
      return with_float(a.dtable_dtype, [&](auto o) {
        typedef decltype(i) I;
        typedef decltype(o) O;
        if (p.vec == 1) hipLaunchKernelGGL((kan_lookup_sum_kernel<I, O, 1>), grid, dim3(kThreads), 0, s, (const I*)a.dy, (O*)a.dtable, q);
        else hipLaunchKernelGGL((kan_lookup_sum_kernel<I, O, 8>), grid, dim3(kThreads), 0, s, (const I*)a.dy, (O*)a.dtable, q);
        return hipGetLastError();
      });
    });
  });
  if (st != KAN_OK || p.chunks < 2) return st;
  return run_named("kan_lookup_join", s, [&] {
    return with_float(a.dtable_dtype, [&](auto o) {
      typedef decltype(o) O;
      if (p.vec == 1) hipLaunchKernelGGL((kan_lookup_join_kernel<O, 1>), join, dim3(kThreads), 0, s, (O*)a.dtable, q, p.chunks);
      else hipLaunchKernelGGL((kan_lookup_join_kernel<O, 8>), join, dim3(kThreads), 0, s, (O*)a.dtable, q, p.chunks);
      return hipGetLastError();
    });
  });
}

}  // namespace kan

// Shared by the operators around the KAN blocks of a language model (kan_lookup.hip, kan_norm.hip, kan_vocab.hip and
// their dispatcher kan_tokens_api.hip): element types, ids, loads of eight elements.  Not part of the public C-ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/kan.h"

namespace kan {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int kMaxWidth = 1 << 20;      // columns of a table or a row that the entry points take

inline bool is_float_dtype(int t) { return t == KAN_F32 || t == KAN_F16 || t == KAN_BF16; }
inline int float_bytes(int t) { return t == KAN_F32 ? 4 : 2; }
inline bool is_id_dtype(int t) { return t == KAN_U16 || t == KAN_U32 || t == KAN_I64; }
inline int id_bytes(int t) { return t == KAN_U16 ? 2 : (t == KAN_U32 ? 4 : 8); }

// f(T{}) for the element type of a dtype code (checked by the entry points).
template <class F>
inline hipError_t with_float(int dtype, F&& f) {
  if (dtype == KAN_F32) return f(float{});
  if (dtype == KAN_F16) return f(f16{});
  return f(bf16{});
}

// One launch, bracketed by the timing hooks of kan_prof_begin (kan_api.hip).
kan_status run_launch(const char* name, hipStream_t s, hipError_t (*f)(const void*), const void* args);
template <class F>
kan_status run_named(const char* name, hipStream_t s, const F& f) {
  return run_launch(name, s, [](const void* a) -> hipError_t { return (*(const F*)a)(); }, &f);
}

// ---- table lookup (kan_lookup.hip) --------------------------------------------------------------------------------
struct LookupArgs {
  const void* table;
  const void* ids;
  void* y;
  long long N;
  int V, D;
  int table_dtype, id_dtype, y_dtype;
  float scale;
};
hipError_t launch_lookup(const LookupArgs&, hipStream_t);

struct LookupGradArgs {
  const void* dy;
  const void* ids;
  void* dtable;
  void* ws;
  long long N;
  int V, D;
  int dy_dtype, id_dtype, dtable_dtype;
  int accumulate;
  float scale;
};
constexpr long long kLookupGradMaxTokens = 1ll << 30;      // positions and row numbers of the sort have 32 bits
size_t lookup_grad_workspace(int V, int D, long long N);
kan_status run_lookup_grad(const LookupGradArgs&, hipStream_t);

// ---- norms around a block (kan_norm.hip) ---------------------------------------------------------------------------
constexpr int kNormMaxWidth = 16384;
struct NormArgs {
  const void *x, *v, *gate;                  // forward: x = stream in front; backward: x = stream behind (y)
  const void *dy, *du;                       // backward
  const void *w_before, *w_after;
  void *y, *u;                               // forward
  void *dx, *dv, *dgate;                     // backward
  void *dw_before, *dw_after;
  float* partial;                            // backward: [2][blocks][D]
  long long N;
  int D;
  int stream_dtype, block_dtype, weight_dtype;
  float scale, eps;
};
size_t norm_grad_workspace(int D, long long N, int sums);
hipError_t launch_norm(const NormArgs&, hipStream_t);
kan_status run_norm_grad(const NormArgs&, hipStream_t);

// ---- vocabulary loss (kan_vocab.hip) ------------------------------------------------------------------------------
struct VocabArgs {
  const void *h, *table, *targets;
  const float* dloss;                        // backward
  float *loss, *lse;                         // backward reads lse
  void *dh, *dtable;
  void* ws;
  long long N;
  int V, D;
  int dtype, id_dtype, accumulate;
  float scale;
};
constexpr long long kVocabMaxTokens = 1ll << 24;
size_t vocab_workspace(long long N, int V, int D, int dtype, bool backward);
kan_status run_vocab_loss(const VocabArgs&, hipStream_t);
kan_status run_vocab_grad(const VocabArgs&, hipStream_t);

// ---- device side ---------------------------------------------------------------------------------------------------
#if defined(__HIPCC__)

// Eight elements at an address that is aligned to one element: gfx950 takes a 16-byte access at any address, so rows of odd
// widths need no form of their own.
template <class T>
__device__ __forceinline__ void load8(const T* p, float (&out)[8]) {
  typedef T V8 __attribute__((ext_vector_type(8)));
  V8 r;
  __builtin_memcpy(&r, p, sizeof(r));
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = (float)r[i];
}
template <class T>
__device__ __forceinline__ void store8(T* p, const float (&in)[8]) {
  typedef T V8 __attribute__((ext_vector_type(8)));
  V8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (T)in[i];
  __builtin_memcpy(p, &r, sizeof(r));
}
// The same for columns c .. c + 7 of a row of D: those past its end are 0, and are not written.
template <class T>
__device__ __forceinline__ void load_cols(const T* row, int c, int D, float (&out)[8]) {
  if (c + 8 <= D) {
    load8(row + c, out);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = c + i < D ? (float)row[c + i] : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void store_cols(T* row, int c, int D, const float (&in)[8]) {
  if (c + 8 <= D) {
    store8(row + c, in);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < D) row[c + i] = (T)in[i];
  }
}

// Row that id n names, or V when it names none (negative or past the table).
__device__ __forceinline__ uint32_t row_of(const void* ids, int dtype, long long n, uint32_t V) {
  if (dtype == KAN_I64) {
    const uint64_t t = ((const uint64_t*)ids)[n];
    return t < V ? (uint32_t)t : V;
  }
  const uint32_t t = dtype == KAN_U16 ? ((const uint16_t*)ids)[n] : ((const uint32_t*)ids)[n];
  return min(t, V);
}

#endif
}  // namespace kan

// Entry points of the operators around the KAN blocks of a language model (include/kan.h): host-side validation, then the
// launches of kan_lookup.hip, kan_norm.hip and kan_vocab.hip.

#include <math.h>

#include "kan_tokens.hpp"

using namespace kan;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool float_aligned(const void* p, int dtype) { return aligned(p, float_bytes(dtype)); }
bool flag(int32_t v) { return v == 0 || v == 1; }

kan_status check_ws(const void* ws, size_t ws_bytes, size_t need) {
  return need == 0 || (ws && aligned(ws, 256) && ws_bytes >= need) ? KAN_OK : KAN_ERR_WORKSPACE;
}

kan_status check_table(int32_t V, int32_t D, int32_t id_dtype) {
  if (!is_id_dtype(id_dtype)) return KAN_ERR_DTYPE;
  if (V < 1 || D < 1 || D > kMaxWidth || (id_dtype == KAN_U16 && V > 65536)) return KAN_ERR_SHAPE;
  return KAN_OK;
}

kan_status check_norm(const kan_block_norm* b) {
  if (!b) return KAN_ERR_NULL;
  if (!is_float_dtype(b->stream_dtype) || !is_float_dtype(b->block_dtype) || !is_float_dtype(b->weight_dtype)) return KAN_ERR_DTYPE;
  if (b->block_dtype != b->stream_dtype && b->block_dtype != KAN_F32) return KAN_ERR_UNSUPPORTED;
  if (b->D < 1) return KAN_ERR_SHAPE;
  if (b->D > kNormMaxWidth) return KAN_ERR_UNSUPPORTED;
  if (!(b->eps > 0.f) || !isfinite(b->eps) || !float_aligned(b->w_before, b->weight_dtype) || !float_aligned(b->w_after, b->weight_dtype)) return KAN_ERR_SHAPE;
  return KAN_OK;
}

NormArgs norm_args(const kan_block_norm* b, int64_t N) {
  NormArgs a = {};
  a.w_before = b->w_before;
  a.w_after = b->w_after;
  a.N = N;
  a.D = b->D;
  a.stream_dtype = b->stream_dtype;
  a.block_dtype = b->block_dtype;
  a.weight_dtype = b->weight_dtype;
  a.scale = b->scale;
  a.eps = b->eps;
  return a;
}

constexpr int64_t kMaxRows = int64_t(1) << 40;      // rows of a lookup or a norm: offsets have 64 bits

kan_status check_vocab(int64_t N, int32_t V, int32_t D, int32_t dtype) {
  if (!is_float_dtype(dtype)) return KAN_ERR_DTYPE;
  if (N < 0 || N > kVocabMaxTokens || V < 1 || D < 1 || D > kMaxWidth) return KAN_ERR_SHAPE;
  return KAN_OK;
}
// 16-bit rows of whole 16-byte pieces are read as such where they lie.
bool rows_aligned(const void* p, int dtype, int D) { return aligned(p, dtype != KAN_F32 && D % 8 == 0 ? 16 : float_bytes(dtype)); }

}  // namespace

extern "C" {

kan_status kan_lookup_forward(const void* table, int32_t table_dtype, int32_t V, int32_t D, const void* ids, int32_t id_dtype, int64_t N, float scale, void* y,
                              int32_t y_dtype, void* stream) {
  kan_status st = check_table(V, D, id_dtype);
  if (st != KAN_OK) return st;
  if (!is_float_dtype(table_dtype) || !is_float_dtype(y_dtype)) return KAN_ERR_DTYPE;
  if (N < 0 || N > kMaxRows / D) return KAN_ERR_SHAPE;
  if (N == 0) return KAN_OK;
  if (!table || !ids || !y) return KAN_ERR_NULL;
  if (!float_aligned(table, table_dtype) || !float_aligned(y, y_dtype) || !aligned(ids, id_bytes(id_dtype))) return KAN_ERR_SHAPE;
  const LookupArgs a = {table, ids, y, N, V, D, table_dtype, id_dtype, y_dtype, scale};
  return run_named("kan_lookup", (hipStream_t)stream, [&] { return launch_lookup(a, (hipStream_t)stream); });
}

size_t kan_lookup_backward_workspace_bytes(int32_t V, int32_t D, int64_t N) {
  if (V < 1 || D < 1 || D > kMaxWidth || N < 0 || N > kLookupGradMaxTokens) return (size_t)-1;
  return lookup_grad_workspace(V, D, N);
}

kan_status kan_lookup_backward(const void* dy, int32_t dy_dtype, const void* ids, int32_t id_dtype, int64_t N, int32_t V, int32_t D, float scale, void* dtable,
                               int32_t dtable_dtype, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  kan_status st = check_table(V, D, id_dtype);
  if (st != KAN_OK) return st;
  if (!is_float_dtype(dy_dtype) || !is_float_dtype(dtable_dtype)) return KAN_ERR_DTYPE;
  if (N < 0 || N > kLookupGradMaxTokens || !flag(accumulate)) return KAN_ERR_SHAPE;
  if (!dtable || (N > 0 && (!dy || !ids))) return KAN_ERR_NULL;
  if (!float_aligned(dtable, dtable_dtype) || (N > 0 && (!float_aligned(dy, dy_dtype) || !aligned(ids, id_bytes(id_dtype))))) return KAN_ERR_SHAPE;
  st = check_ws(ws, ws_bytes, lookup_grad_workspace(V, D, N));
  if (st != KAN_OK) return st;
  const LookupGradArgs a = {dy, ids, dtable, ws, N, V, D, dy_dtype, id_dtype, dtable_dtype, accumulate, scale};
  return run_lookup_grad(a, (hipStream_t)stream);
}

kan_status kan_block_norm_forward(const kan_block_norm* b, const void* x, const void* v, const void* gate, int64_t N, void* y, void* u, void* stream) {
  kan_status st = check_norm(b);
  if (st != KAN_OK) return st;
  if (N < 0 || N > kMaxRows / b->D) return KAN_ERR_SHAPE;
  if (N == 0) return KAN_OK;
  if (!v && (gate || y)) return KAN_ERR_UNSUPPORTED;
  if (!x || (!v && !u) || (v && !y)) return KAN_ERR_NULL;
  for (const void* p : {x, (const void*)y})
    if (!float_aligned(p, b->stream_dtype)) return KAN_ERR_SHAPE;
  for (const void* p : {v, gate, (const void*)u})
    if (!float_aligned(p, b->block_dtype)) return KAN_ERR_SHAPE;
  NormArgs a = norm_args(b, N);
  a.x = x;
  a.v = v;
  a.gate = gate;
  a.y = y;
  a.u = u;
  return run_named("kan_norm", (hipStream_t)stream, [&] { return launch_norm(a, (hipStream_t)stream); });
}

size_t kan_block_norm_backward_workspace_bytes(const kan_block_norm* b, int64_t N) {
  if (check_norm(b) != KAN_OK || N < 0 || N > kMaxRows / b->D) return (size_t)-1;
  return norm_grad_workspace(b->D, N, 2);
}

kan_status kan_block_norm_backward(const kan_block_norm* b, const void* y, const void* dy, const void* du, const void* v, const void* gate, int64_t N, void* dx,
                                   void* dv, void* dgate, void* dw_before, void* dw_after, void* ws, size_t ws_bytes, void* stream) {
  kan_status st = check_norm(b);
  if (st != KAN_OK) return st;
  if (N < 0 || N > kMaxRows / b->D) return KAN_ERR_SHAPE;
  if ((dw_before && !b->w_before) || (dw_after && !b->w_after)) return KAN_ERR_UNSUPPORTED;
  for (const void* p : {(const void*)dw_before, (const void*)dw_after})
    if (!float_aligned(p, b->weight_dtype)) return KAN_ERR_SHAPE;
  if (N > 0) {      // (arrays of no rows may be NULL)
    if ((!du && dw_before) || (!v && (gate || dv || dw_after)) || (!gate && dgate)) return KAN_ERR_UNSUPPORTED;
    if ((!dy && !du) || !dx || (du && !y) || (v && !dv) || (gate && !dgate)) return KAN_ERR_NULL;
    for (const void* p : {y, dy, (const void*)dx})
      if (!float_aligned(p, b->stream_dtype)) return KAN_ERR_SHAPE;
    for (const void* p : {du, v, gate, (const void*)dv, (const void*)dgate})
      if (!float_aligned(p, b->block_dtype)) return KAN_ERR_SHAPE;
  }
  const int sums = (dw_before ? 1 : 0) + (dw_after ? 1 : 0);
  st = check_ws(ws, ws_bytes, norm_grad_workspace(b->D, N, sums));
  if (st != KAN_OK) return st;
  NormArgs a = norm_args(b, N);
  a.x = y;
  a.v = v;
  a.gate = gate;
  a.dy = dy;
  a.du = du;
  a.dx = dx;
  a.dv = dv;
  a.dgate = dgate;
  a.dw_before = dw_before;
  a.dw_after = dw_after;
  a.partial = (float*)ws;
  return run_norm_grad(a, (hipStream_t)stream);
}

size_t kan_vocab_loss_workspace_bytes(int64_t N, int32_t V, int32_t D, int32_t dtype, int32_t backward) {
  if (check_vocab(N, V, D, dtype) != KAN_OK || !flag(backward)) return (size_t)-1;
  return vocab_workspace(N, V, D, dtype, backward != 0);
}

kan_status kan_vocab_loss_forward(const void* h, const void* table, int32_t dtype, int64_t N, int32_t V, int32_t D, const void* targets, int32_t id_dtype,
                                  float scale, float* loss, float* lse, void* ws, size_t ws_bytes, void* stream) {
  kan_status st = check_vocab(N, V, D, dtype);
  if (st == KAN_OK) st = check_table(V, D, id_dtype);
  if (st != KAN_OK) return st;
  if (N == 0) return KAN_OK;
  if (!h || !table || !targets || !loss || !lse) return KAN_ERR_NULL;
  if (!rows_aligned(h, dtype, D) || !rows_aligned(table, dtype, D) || !aligned(targets, id_bytes(id_dtype)) || !aligned(loss, 4) || !aligned(lse, 4))
    return KAN_ERR_SHAPE;
  st = check_ws(ws, ws_bytes, vocab_workspace(N, V, D, dtype, false));
  if (st != KAN_OK) return st;
  VocabArgs a = {};
  a.h = h;
  a.table = table;
  a.targets = targets;
  a.loss = loss;
  a.lse = lse;
  a.ws = ws;
  a.N = N;
  a.V = V;
  a.D = D;
  a.dtype = dtype;
  a.id_dtype = id_dtype;
  a.scale = scale;
  return run_vocab_loss(a, (hipStream_t)stream);
}

kan_status kan_vocab_loss_backward(const void* h, const void* table, int32_t dtype, int64_t N, int32_t V, int32_t D, const void* targets, int32_t id_dtype,
                                   float scale, const float* lse, const float* dloss, void* dh, void* dtable, int32_t accumulate, void* ws, size_t ws_bytes,
                                   void* stream) {
  kan_status st = check_vocab(N, V, D, dtype);
  if (st == KAN_OK) st = check_table(V, D, id_dtype);
  if (st != KAN_OK) return st;
  if (!flag(accumulate)) return KAN_ERR_SHAPE;
  if (!dtable) return KAN_ERR_NULL;
  if (!float_aligned(dtable, dtype)) return KAN_ERR_SHAPE;
  if (N == 0) {      // no tokens: the sums over them
    const LookupGradArgs a = {nullptr, nullptr, dtable, nullptr, 0, V, D, dtype, id_dtype, dtype, accumulate, 1.f};
    return run_lookup_grad(a, (hipStream_t)stream);
  }
  if (!h || !table || !targets || !lse || !dloss || !dh) return KAN_ERR_NULL;
  if (!rows_aligned(h, dtype, D) || !rows_aligned(table, dtype, D) || !float_aligned(dh, dtype) || !aligned(targets, id_bytes(id_dtype)) || !aligned(lse, 4) ||
      !aligned(dloss, 4))
    return KAN_ERR_SHAPE;
  st = check_ws(ws, ws_bytes, vocab_workspace(N, V, D, dtype, true));
  if (st != KAN_OK) return st;
  VocabArgs a = {};
  a.h = h;
  a.table = table;
  a.targets = targets;
  a.dloss = dloss;
  a.lse = const_cast<float*>(lse);
  a.dh = dh;
  a.dtable = dtable;
  a.ws = ws;
  a.N = N;
  a.V = V;
  a.D = D;
  a.dtype = dtype;
  a.id_dtype = id_dtype;
  a.accumulate = accumulate;
  a.scale = scale;
  return run_vocab_grad(a, (hipStream_t)stream);
}

}  // extern "C"

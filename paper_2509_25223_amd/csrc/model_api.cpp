// Host side of include/rla_model.h: argument validation (no HIP call until it
// passes), workspace planning and launches.
#include <math.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "host.hpp"
#include "model.hpp"
#include "rla_model.h"

namespace rla {
namespace {

bool is_index(int32_t t) { return t == RLA_INDEX_I32 || t == RLA_INDEX_I64; }
size_t index_size(int32_t t) { return t == RLA_INDEX_I64 ? 8 : 4; }

// `n` rows of `width` bytes, `step` apart.
struct Bytes {
  const void* at;
  size_t width, n = 1, step = 0;
};
Bytes rows_of(const void* at, int64_t n, int64_t D, int64_t stride, size_t el) {
  return {at, (size_t)D * el, (size_t)n, (size_t)stride * el};
}
// They meet `out` (one piece).
bool meet(const Bytes& in, const Bytes& out) {
  if (in.n <= 1 || in.step == in.width) return overlap(in.at, in.n * in.width, out.at, out.width);
  if (!in.at || !out.at || out.width == 0) return false;
  const uintptr_t a = (uintptr_t)in.at, o = (uintptr_t)out.at;
  const size_t k = o < a + in.width ? 0 : (o - a - in.width) / in.step + 1;   // the first row that ends behind its start
  return k < in.n && a + k * in.step < o + out.width;
}
// No output (one piece each) lies over an input or another output.
template <size_t N, size_t M> bool apart(const Bytes (&outs)[N], const Bytes (&ins)[M]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = 0; j < i; ++j)
      if (meet(outs[j], outs[i])) return false;
    for (const Bytes& in : ins)
      if (meet(in, outs[i])) return false;
  }
  return true;
}

// ---------------------------------------------------------------------------
// embedding
// ---------------------------------------------------------------------------
rla_status check_embed(const rla_embed_problem* q, bool gradient, EmbedParams& p) {
  if (!q) return RLA_ERR_NULL_ARG;
  if (!is_type(q->dtype) || !is_type(q->table_dtype) || !is_index(q->index)) return RLA_ERR_DTYPE;
  if (q->tokens < 0 || q->tokens > kMaxTokens || q->vocab < 1 || q->vocab > (gradient ? (1 << 22) - 1 : INT32_MAX) ||
      q->width < 1 || q->width > (1 << 20))
    return RLA_ERR_SHAPE;
  if (!stride(q->dout_stride, q->width, p.dos) || times(times(q->tokens, p.dos), 4) < 0) return RLA_ERR_SHAPE;
  if (!isfinite(q->scale)) return RLA_ERR_VALUE;
  p.n = q->tokens;
  p.V = q->vocab;
  p.D = q->width;
  p.scale = q->scale;
  p.ids.wide = q->index == RLA_INDEX_I64;
  return RLA_OK;
}
size_t embed_bytes(const EmbedParams& p) {
  EmbedParams plan = p;
  return p.n == 0 ? 0 : embed_plan(plan, p.n < kEmbedSlice ? p.n : kEmbedSlice, nullptr);
}

}  // namespace
}  // namespace rla

using namespace rla;

extern "C" size_t rla_embed_workspace_size(const rla_embed_problem* q) {
  EmbedParams p;
  return check_embed(q, true, p) == RLA_OK ? embed_bytes(p) : 0;
}

extern "C" rla_status rla_embed_forward(const rla_embed_problem* q, const void* ids, const void* table, void* out,
                                        void* stream) {
  EmbedParams p;
  const rla_status st = check_embed(q, false, p);
  if (st != RLA_OK) return st;
  if (p.n == 0) return RLA_OK;
  if (!ids || !table || !out) return RLA_ERR_NULL_ARG;
  const size_t tb = (size_t)p.V * p.D * elem(q->table_dtype), ob = (size_t)p.n * p.D * elem(q->dtype);
  if (!aligned(ids, index_size(q->index)) || !aligned(table, elem(q->table_dtype)) || !aligned(out, elem(q->dtype)) ||
      overlap(table, tb, out, ob) || overlap(ids, (size_t)p.n * index_size(q->index), out, ob))
    return RLA_ERR_VALUE;
  p.ids.p = ids;
  p.table = table;
  p.out = out;
  return to_status(launch_embed_forward(p, q->table_dtype == RLA_BF16, q->dtype == RLA_BF16,
                                        reinterpret_cast<hipStream_t>(stream)));
}

extern "C" rla_status rla_embed_backward(const rla_embed_problem* q, const void* ids, const void* dout, const float* base,
                                         float* dtable, void* workspace, size_t workspace_bytes, void* stream) {
  EmbedParams p;
  rla_status st = check_embed(q, true, p);
  if (st != RLA_OK) return st;
  if (!dtable || (p.n > 0 && (!ids || !dout))) return RLA_ERR_NULL_ARG;
  const size_t tb = (size_t)p.V * p.D * 4;
  if (!aligned(ids, index_size(q->index)) || !aligned(dout, elem(q->dtype)) || !aligned(base, 4) || !aligned(dtable, 4) ||
      (base != dtable && overlap(base, tb, dtable, tb)) ||
      (p.n > 0 && (overlap(dout, ((size_t)(p.n - 1) * p.dos + p.D) * elem(q->dtype), dtable, tb) ||
                   overlap(ids, (size_t)p.n * index_size(q->index), dtable, tb))))
    return RLA_ERR_VALUE;
  st = check_workspace(embed_bytes(p), workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  p.ids.p = ids;
  p.dout = dout;
  p.base = base;
  p.dtable = dtable;
  return to_status(launch_embed_backward(p, q->dtype == RLA_BF16, reinterpret_cast<unsigned char*>(workspace),
                                         reinterpret_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// log probabilities
// ---------------------------------------------------------------------------
namespace rla {
namespace {

rla_status check_logprob(const rla_logprob_problem* q, LogprobParams& p) {
  if (!q) return RLA_ERR_NULL_ARG;
  if (!is_type(q->dtype) || !is_index(q->index)) return RLA_ERR_DTYPE;
  if (q->rows < 0 || q->rows > kMaxTokens || q->vocab < 1 || q->vocab > (1 << 30) || q->top < 0 || q->top > kMaxTop ||
      q->top > q->vocab)
    return RLA_ERR_SHAPE;
  if (!stride(q->logits_stride, q->vocab, p.xs) || times(times(q->rows, p.xs), 4) < 0) return RLA_ERR_SHAPE;
  if (!(q->scale > 0.f) || isinf(q->scale * 1.4426950408889634f)) return RLA_ERR_VALUE;   // (kernels use scale log2 e)
  p.n = q->rows;
  p.V = q->vocab;
  p.scale = q->scale;
  p.top = q->top;
  p.targets.wide = q->index == RLA_INDEX_I64;
  return RLA_OK;
}
size_t logits_bytes(const rla_logprob_problem* q, const LogprobParams& p) {
  return p.n == 0 ? 0 : ((size_t)(p.n - 1) * p.xs + p.V) * elem(q->dtype);
}

}  // namespace
}  // namespace rla

extern "C" size_t rla_logprob_workspace_size(const rla_logprob_problem* q) {
  LogprobParams p;
  return check_logprob(q, p) == RLA_OK ? logprob_plan(p, q->dtype == RLA_BF16, nullptr) : 0;
}

extern "C" rla_status rla_logprob_forward(const rla_logprob_problem* q, const void* logits, const void* targets,
                                          float* logprob, float* lse, float* entropy, float* top_logprobs,
                                          int32_t* top_ids, void* workspace, size_t workspace_bytes, void* stream) {
  LogprobParams p;
  rla_status st = check_logprob(q, p);
  if (st != RLA_OK) return st;
  if (p.n == 0) return RLA_OK;
  if (!logits || (logprob && !targets) || (p.top > 0 && (!top_logprobs || !top_ids))) return RLA_ERR_NULL_ARG;
  if (!aligned(logits, elem(q->dtype)) || !aligned(targets, index_size(q->index))) return RLA_ERR_VALUE;
  const size_t row = 4 * (size_t)p.n;
  const Bytes ins[] = {{logits, logits_bytes(q, p)}, {logprob ? targets : nullptr, index_size(q->index) * (size_t)p.n}};
  const Bytes outs[] = {
      {logprob, row}, {lse, row}, {entropy, row}, {p.top ? top_logprobs : nullptr, row * p.top}, {p.top ? top_ids : nullptr, row * p.top}};
  for (const Bytes& o : outs)
    if (!aligned(o.at, 4)) return RLA_ERR_VALUE;
  if (!apart(outs, ins)) return RLA_ERR_VALUE;
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  const size_t size = logprob_plan(p, q->dtype == RLA_BF16, ws);
  st = check_workspace(p.parts == 1 ? 0 : size, workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  p.x = logits;
  p.targets.p = targets;
  p.logprob = logprob;
  p.lse = lse;
  p.entropy = entropy;
  p.top_lp = top_logprobs;
  p.top_ids = top_ids;
  return to_status(launch_logprob_forward(p, q->dtype == RLA_BF16, reinterpret_cast<hipStream_t>(stream)));
}

extern "C" rla_status rla_logprob_backward(const rla_logprob_problem* q, const void* logits, const void* targets,
                                           const float* lse, const float* entropy, const float* dlogprob,
                                           const float* dentropy, void* dlogits, void* stream) {
  LogprobParams p;
  const rla_status st = check_logprob(q, p);
  if (st != RLA_OK) return st;
  if (p.n == 0) return RLA_OK;
  if (!logits || !lse || !dlogits || (dlogprob && !targets) || (dentropy && !entropy)) return RLA_ERR_NULL_ARG;
  const size_t el = elem(q->dtype);
  if (!aligned(logits, el) || !aligned(dlogits, el) || !aligned(targets, index_size(q->index))) return RLA_ERR_VALUE;
  const size_t out = (size_t)p.n * p.V * el, row = 4 * (size_t)p.n;
  for (const float* a : {lse, entropy, dlogprob, dentropy})
    if (!aligned(a, 4) || overlap(a, row, dlogits, out)) return RLA_ERR_VALUE;
  if (targets && overlap(targets, index_size(q->index) * (size_t)p.n, dlogits, out)) return RLA_ERR_VALUE;
  if ((logits != dlogits || p.xs != p.V) && overlap(logits, logits_bytes(q, p), dlogits, out)) return RLA_ERR_VALUE;
  p.x = logits;
  p.targets.p = targets;
  p.lse_in = lse;
  p.entropy_in = entropy;
  p.dlogprob = dlogprob;
  p.dentropy = dentropy;
  p.dx = dlogits;
  return to_status(launch_logprob_backward(p, q->dtype == RLA_BF16, reinterpret_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// gated linear recurrence
// ---------------------------------------------------------------------------
namespace rla {
namespace {

rla_status check_glr(const rla_glr_problem* q, GlrParams& p) {
  if (!q) return RLA_ERR_NULL_ARG;
  if (!is_type(q->dtype)) return RLA_ERR_DTYPE;
  const rla_status st = tokens(q->batch, q->seq_len, q->num_seqs, q->cu_seqlens, p.map);
  if (st != RLA_OK) return st;
  if (q->channels < 1 || q->channels >= (1 << 23)) return RLA_ERR_SHAPE;
  if (q->normalize != 0 && q->normalize != 1) return RLA_ERR_VALUE;
  p.D = q->channels;
  if (!stride(q->x_stride, p.D, p.xs) || !stride(q->r_stride, p.D, p.rs) || !stride(q->i_stride, p.D, p.is) ||
      !stride(q->z_stride, p.D, p.zs) || !stride(q->do_stride, p.D, p.dos))
    return RLA_ERR_SHAPE;
  for (int64_t s : {p.xs, p.rs, p.is, p.zs, p.dos})   // (a tile's rows: 32-bit offsets of bytes)
    if (s >= (1 << 23) || times(times(p.map.ntok, s), 4) < 0) return RLA_ERR_SHAPE;
  if (times(times(p.map.nseq, p.D), 4) < 0) return RLA_ERR_SHAPE;
  p.normalize = q->normalize;
  return RLA_OK;
}
rla_status check_glr_scan(const rla_glr_problem* q, GlrParams& p) {
  const rla_status st = check_glr(q, p);
  if (st == RLA_OK) glr_plan(p, q->cu_seqlens != nullptr);
  return st;
}

struct GlrPlan {
  size_t map = 0, sum = 0, ck = 0, pA = 0, total = 0;
  size_t used = 0;   // by this call: as far as its own cut needs the room
};
GlrPlan plan_glr(const rla_glr_problem* q, const GlrParams& p, bool backward) {
  GlrPlan w;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = up(off + bytes);
    return at;
  };
  const size_t D = (size_t)p.D;
  if (q->cu_seqlens) {
    w.map = take(token_map_bytes(p.map.ntok, p.map.nseq));
    w.used = off;
  }
  w.sum = take(8 * (size_t)p.room_sum * D);
  if (!p.apart) w.used = off;
  if (backward) {
    w.ck = take(4 * (size_t)p.room_tiles * D);
    w.pA = take(4 * (size_t)p.room_chunks * D);
    w.used = off;
  }
  w.total = off;
  return w;
}
void set_workspace(GlrParams& p, const GlrPlan& w, unsigned char* ws) {
  p.sum = reinterpret_cast<float*>(ws + w.sum);
  p.ck = reinterpret_cast<float*>(ws + w.ck);
  p.pA = reinterpret_cast<float*>(ws + w.pA);
}

rla_status glr_inputs(const rla_glr_problem* q, GlrParams& p, const void* x, const void* r, const float* A, const void* i,
                      const void* z, const float* h0) {
  if (!A || (p.map.ntok > 0 && (!x || !r))) return RLA_ERR_NULL_ARG;
  for (const void* a : {x, r, i, z})
    if (!aligned(a, elem(q->dtype))) return RLA_ERR_VALUE;
  if (!aligned(A, 4) || !aligned(h0, 4)) return RLA_ERR_VALUE;
  p.x = x; p.r = r; p.A = A; p.i = i; p.z = z; p.h0 = h0;
  return RLA_OK;
}
// Outputs over nothing that is read, or each other.
template <size_t N>
bool glr_apart(const rla_glr_problem* q, const GlrParams& p, const void* dO, const float* dh_final, const Bytes (&outs)[N]) {
  const size_t el = elem(q->dtype), sbytes = (size_t)p.map.nseq * (size_t)p.D * 4;
  const Bytes ins[] = {rows_of(p.x, p.map.ntok, p.D, p.xs, el), rows_of(p.r, p.map.ntok, p.D, p.rs, el),
                       rows_of(p.i, p.map.ntok, p.D, p.is, el), rows_of(p.z, p.map.ntok, p.D, p.zs, el),
                       rows_of(dO, p.map.ntok, p.D, p.dos, el), {p.A, (size_t)p.D * 4}, {p.h0, sbytes}, {dh_final, sbytes},
                       {q->cu_seqlens, ((size_t)p.map.nseq + 1) * 4}};
  return apart(outs, ins);
}
size_t state_bytes(const GlrParams& p) { return (size_t)p.map.nseq * (size_t)p.D * 4; }

hipError_t copy_states(const void* from, void* to, size_t bytes, hipStream_t stream) {
  return to && bytes ? launch_copy_words(from, to, (int64_t)(bytes / 2), stream) : hipSuccess;
}

}  // namespace
}  // namespace rla

extern "C" size_t rla_glr_workspace_size(const rla_glr_problem* q, int op) {
  GlrParams p;
  if ((op != RLA_GLR_FORWARD && op != RLA_GLR_BACKWARD) || check_glr_scan(q, p) != RLA_OK) return 0;
  return plan_glr(q, p, op == RLA_GLR_BACKWARD).total;
}

extern "C" rla_status rla_glr_forward(const rla_glr_problem* q, const void* x, const void* r, const float* A, const void* i,
                                      const void* z, const float* h_init, void* o, float* h_final, int save,
                                      void* workspace, size_t workspace_bytes, void* stream_) {
  GlrParams p;
  rla_status st = check_glr_scan(q, p);
  if (st == RLA_OK) st = glr_inputs(q, p, x, r, A, i, z, h_init);
  if (st != RLA_OK) return st;
  if (p.map.ntok > 0 && !o) return RLA_ERR_NULL_ARG;
  const size_t sbytes = state_bytes(p);
  if (!aligned(o, elem(q->dtype)) || !aligned(h_final, 4) || overlap(h_init, sbytes, h_final, sbytes)) return RLA_ERR_VALUE;
  const GlrPlan w = plan_glr(q, p, save != 0);
  st = check_workspace(w.used, workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  const Bytes outs[] = {{o, (size_t)p.map.ntok * p.D * elem(q->dtype)}, {h_final, sbytes}};
  if (!glr_apart(q, p, nullptr, nullptr, outs)) return RLA_ERR_VALUE;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  if (p.map.ntok == 0) return to_status(copy_states(h_init, h_final, sbytes, stream));
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  set_workspace(p, w, ws);
  p.o = o;
  p.hfin = h_final;
  hipError_t e = hipSuccess;
  if (q->cu_seqlens) e = launch_token_map(q->cu_seqlens, p.map.nseq, p.map.ntok, ws + w.map, true, p.map, stream);
  if (e == hipSuccess) e = launch_glr_forward(p, q->dtype == RLA_BF16, save != 0, true, stream);
  return to_status(e);
}

extern "C" rla_status rla_glr_backward(const rla_glr_problem* q, const void* x, const void* r, const float* A, const void* i,
                                       const void* z, const float* h_init, const void* dO, const float* dh_final, void* dx,
                                       void* dr, float* dA, void* di, void* dz, float* dh_init, int use_saved,
                                       void* workspace, size_t workspace_bytes, void* stream_) {
  GlrParams p;
  rla_status st = check_glr_scan(q, p);
  if (st == RLA_OK) st = glr_inputs(q, p, x, r, A, i, z, h_init);
  if (st != RLA_OK) return st;
  if (!dA || (p.map.ntok > 0 && (!dO || !dx || !dr || (i && !di) || (z && !dz)))) return RLA_ERR_NULL_ARG;
  const size_t el = elem(q->dtype), sbytes = state_bytes(p);
  for (const void* a : {dO, (const void*)dx, (const void*)dr, (const void*)di, (const void*)dz})
    if (!aligned(a, el)) return RLA_ERR_VALUE;
  if (!aligned(dh_final, 4) || !aligned(dA, 4) || !aligned(dh_init, 4) || overlap(dh_final, sbytes, dh_init, sbytes) ||
      overlap(h_init, sbytes, dh_init, sbytes))
    return RLA_ERR_VALUE;
  const GlrPlan w = plan_glr(q, p, true);
  st = check_workspace(w.total, workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  const size_t tbytes = (size_t)p.map.ntok * p.D * el;
  const Bytes outs[] = {{dx, tbytes}, {dr, tbytes}, {i ? di : nullptr, tbytes}, {z ? dz : nullptr, tbytes},
                        {dA, (size_t)p.D * 4}, {dh_init, sbytes}};
  if (!glr_apart(q, p, dO, dh_final, outs)) return RLA_ERR_VALUE;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  const bool bf16 = q->dtype == RLA_BF16;
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  set_workspace(p, w, ws);
  hipError_t e = hipSuccess;
  if (p.map.ntok > 0) {
    if (q->cu_seqlens) e = launch_token_map(q->cu_seqlens, p.map.nseq, p.map.ntok, ws + w.map, !use_saved, p.map, stream);
    if (e == hipSuccess && !use_saved) e = launch_glr_forward(p, bf16, true, false, stream);
    p.dO = dO; p.dhfin = dh_final; p.dx = dx; p.dr = dr; p.di = di; p.dz = dz; p.dh0 = dh_init;
    if (e == hipSuccess) e = launch_glr_backward(p, bf16, stream);
  } else {
    e = copy_states(dh_final, dh_init, sbytes, stream);
  }
  if (e == hipSuccess)
    e = launch_column_sums(p.pA, p.map.ntok > 0 ? p.nchunk : 0, p.D, p.D, 1, dA, nullptr, stream);
  return to_status(e);
}

extern "C" rla_status rla_glr_decode(const rla_glr_problem* q, const void* x, const void* r, const float* A, const void* i,
                                     const void* z, const float* h_in, void* o, float* h_out, void* stream) {
  GlrParams p;
  rla_status st = check_glr(q, p);
  if (st != RLA_OK) return st;
  if (q->cu_seqlens) return RLA_ERR_UNSUPPORTED;
  if (p.map.nseq == 0) return RLA_OK;
  if (glr_decode_wgs(p) > kMaxWgs) return RLA_ERR_SHAPE;
  st = glr_inputs(q, p, x, r, A, i, z, h_in);
  if (st != RLA_OK) return st;
  if (!h_out || (p.map.ntok > 0 && !o)) return RLA_ERR_NULL_ARG;
  const size_t sbytes = state_bytes(p);
  if (!aligned(o, elem(q->dtype)) || !aligned(h_out, 4) || (h_in != h_out && overlap(h_in, sbytes, h_out, sbytes)))
    return RLA_ERR_VALUE;
  // (in place: a thread reads what it writes)
  GlrParams in = p;
  if (in.h0 == h_out) in.h0 = nullptr;
  if (in.x == o && in.xs == p.D) in.x = nullptr;
  if (in.r == o && in.rs == p.D) in.r = nullptr;
  if (in.i == o && in.is == p.D) in.i = nullptr;
  if (in.z == o && in.zs == p.D) in.z = nullptr;
  const Bytes outs[] = {{o, (size_t)p.map.ntok * p.D * elem(q->dtype)}, {h_out, sbytes}};
  if (!glr_apart(q, in, nullptr, nullptr, outs)) return RLA_ERR_VALUE;
  p.o = o;
  p.hfin = h_out;
  return to_status(launch_glr_decode(p, q->dtype == RLA_BF16, reinterpret_cast<hipStream_t>(stream)));
}

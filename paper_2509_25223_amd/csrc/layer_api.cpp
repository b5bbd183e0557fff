// Host side of include/rla_layer.h: argument validation (no HIP call until it
// passes), workspace planning and launches.
#include <math.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "layer.hpp"
#include "rla_layer.h"
#include "ssm.hpp"

namespace rla {
namespace {

constexpr size_t kWsAlign = 256;
size_t up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool is_type(int32_t t) { return t == RLA_F32 || t == RLA_BF16; }
size_t elem(int32_t t) { return t == RLA_BF16 ? 2 : 4; }
rla_status to_status(hipError_t e) { return e == hipSuccess ? RLA_OK : RLA_ERR_HIP; }

// Byte ranges intersect (empty or NULL ones never do).
bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  if (!a || !b || an == 0 || bn == 0) return false;
  return (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}

// a * b, or -1 where it passes 2^62 (a, b >= 0)
int64_t times(int64_t a, int64_t b) {
  if (a < 0 || b < 0) return -1;
  if (a == 0 || b == 0) return 0;
  return a > ((int64_t)1 << 62) / b ? -1 : a * b;
}

// Row stride in elements: 0 stands for rows next to each other.
bool stride(int64_t given, int64_t width, int64_t& out) {
  out = given == 0 ? width : given;
  return out >= width;
}

constexpr int64_t kMaxTokens = INT32_MAX - 4096;

// Tokens of a problem: dense [B, T] or packed.
rla_status tokens(int64_t B, int64_t T, int64_t num_seqs, const int32_t* cu, TokenMap& m) {
  if (B < 0 || T < 0) return RLA_ERR_SHAPE;
  if (cu) {
    if (B != 1 || num_seqs < 0) return RLA_ERR_SHAPE;
    if (!aligned(cu, 4)) return RLA_ERR_VALUE;
    m.nseq = (int32_t)(num_seqs < ((int64_t)1 << 30) ? num_seqs : -1);
    m.ntok = T;
  } else {
    m.nseq = (int32_t)(B < ((int64_t)1 << 30) ? B : -1);
    m.ntok = times(B, T);
    m.T = T;
  }
  return m.nseq < 0 || m.ntok < 0 || m.ntok > kMaxTokens ? RLA_ERR_SHAPE : RLA_OK;
}

rla_status check_workspace(size_t need, const void* ws, size_t bytes) {
  if (need == 0) return RLA_OK;
  if (!ws || bytes < need) return RLA_ERR_WORKSPACE;
  return aligned(ws, kWsAlign) ? RLA_OK : RLA_ERR_VALUE;
}

// ---------------------------------------------------------------------------
// convolution
// ---------------------------------------------------------------------------
rla_status check_conv(const rla_conv_problem* q, ConvParams& p) {
  if (!q) return RLA_ERR_NULL_ARG;
  if (!is_type(q->dtype)) return RLA_ERR_DTYPE;
  const rla_status st = tokens(q->batch, q->seq_len, q->num_seqs, q->cu_seqlens, p.map);
  if (st != RLA_OK) return st;
  if (q->channels < 1 || q->channels > INT32_MAX / 64 || q->taps < 2 || q->taps > 4) return RLA_ERR_SHAPE;
  if (q->silu != 0 && q->silu != 1) return RLA_ERR_VALUE;
  if (!stride(q->x_stride, q->channels, p.xs) || !stride(q->dy_stride, q->channels, p.dys)) return RLA_ERR_SHAPE;
  // token counts times a row, and the states, as byte counts
  if (times(times(p.map.ntok, p.xs > p.dys ? p.xs : p.dys), 4) < 0 || times(times(p.map.nseq, 3 * q->channels), 4) < 0)
    return RLA_ERR_SHAPE;
  p.D = q->channels;
  p.taps = q->taps;
  p.silu = q->silu;
  return RLA_OK;
}

size_t conv_part_bytes(const ConvParams& p) {
  return up(sizeof(float) * (size_t)conv_backward_rows(p.map.ntok, p.D) * (size_t)(p.taps + 1) *
            (size_t)p.D);
}
// (sequences looked up in place need none; packed calls take a workspace all the same, so
// that callers need not know how many those are)
size_t conv_map_bytes(const rla_conv_problem* q, const ConvParams& p) {
  if (!q->cu_seqlens) return 0;
  return p.map.nseq > kConvInPlace ? token_map_bytes(p.map.ntok, p.map.nseq) : kWsAlign;
}

// Packed: where sequences lie, looked up in place or by a map in ws.
hipError_t conv_sequences(const rla_conv_problem* q, unsigned char* ws, ConvParams& p, hipStream_t stream) {
  if (p.map.nseq > kConvInPlace)
    return launch_token_map(q->cu_seqlens, p.map.nseq, p.map.ntok, ws, true, p.map, stream);
  p.cu = q->cu_seqlens;
  return hipSuccess;
}

rla_status conv_pointers(const rla_conv_problem* q, const ConvParams& p, const void* x, const float* weight,
                         const float* bias, const void* s0) {
  if (!weight || (p.map.ntok > 0 && !x)) return RLA_ERR_NULL_ARG;
  if (!aligned(x, elem(q->dtype)) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(s0, elem(q->dtype))) return RLA_ERR_VALUE;
  return RLA_OK;
}

// Final states (or initial states' gradients) of a call without tokens: the
// initial ones.
hipError_t copy_states(const void* from, void* to, size_t bytes, hipStream_t stream) {
  if (!to || bytes == 0) return hipSuccess;
  return launch_copy_words(from, to, (int64_t)(bytes / 2), stream);
}

}  // namespace
}  // namespace rla

using namespace rla;

extern "C" size_t rla_conv_workspace_size(const rla_conv_problem* q, int backward) {
  ConvParams p;
  if (check_conv(q, p) != RLA_OK || !(backward ? conv_backward_fits(p) : conv_forward_fits(p, q->dtype == RLA_BF16)))
    return 0;
  return conv_map_bytes(q, p) + (backward ? conv_part_bytes(p) : 0);
}

extern "C" rla_status rla_conv_forward(const rla_conv_problem* q, const void* x, const float* weight,
                                       const float* bias, const void* state_init, void* y, void* state_final,
                                       void* workspace, size_t workspace_bytes, void* stream_) {
  ConvParams p;
  rla_status st = check_conv(q, p);
  if (st == RLA_OK && !conv_forward_fits(p, q->dtype == RLA_BF16)) st = RLA_ERR_SHAPE;
  if (st == RLA_OK) st = conv_pointers(q, p, x, weight, bias, state_init);
  if (st != RLA_OK) return st;
  if (p.map.ntok > 0 && !y) return RLA_ERR_NULL_ARG;
  if (!aligned(y, elem(q->dtype)) || !aligned(state_final, elem(q->dtype))) return RLA_ERR_VALUE;
  const size_t el = elem(q->dtype), sbytes = (size_t)p.map.nseq * (p.taps - 1) * p.D * el;
  if (overlap(state_init, sbytes, state_final, sbytes)) return RLA_ERR_VALUE;
  st = check_workspace(conv_map_bytes(q, p), workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  if (p.map.ntok == 0) return to_status(copy_states(state_init, state_final, sbytes, stream));
  p.x = x; p.weight = weight; p.bias = bias; p.state0 = state_init; p.y = y; p.state_fin = state_final;
  hipError_t e = hipSuccess;
  if (q->cu_seqlens) e = conv_sequences(q, reinterpret_cast<unsigned char*>(workspace), p, stream);
  if (e == hipSuccess) e = launch_conv_forward(p, q->dtype == RLA_BF16, stream);
  return to_status(e);
}

extern "C" rla_status rla_conv_backward(const rla_conv_problem* q, const void* x, const float* weight,
                                        const float* bias, const void* state_init, const void* dy,
                                        const void* dstate_final, void* dx, float* dweight, float* dbias,
                                        void* dstate_init, void* workspace, size_t workspace_bytes, void* stream_) {
  ConvParams p;
  rla_status st = check_conv(q, p);
  if (st == RLA_OK && !conv_backward_fits(p)) st = RLA_ERR_SHAPE;
  if (st == RLA_OK) st = conv_pointers(q, p, x, weight, bias, state_init);
  if (st != RLA_OK) return st;
  if (!dweight || (p.map.ntok > 0 && (!dy || !dx))) return RLA_ERR_NULL_ARG;
  const size_t el = elem(q->dtype), sbytes = (size_t)p.map.nseq * (p.taps - 1) * p.D * el;
  if (!aligned(dy, el) || !aligned(dx, el) || !aligned(dstate_final, el) || !aligned(dweight, 4) ||
      !aligned(dbias, 4) || !aligned(dstate_init, el) || overlap(dstate_final, sbytes, dstate_init, sbytes))
    return RLA_ERR_VALUE;
  const size_t map_bytes = conv_map_bytes(q, p);
  st = check_workspace(map_bytes + conv_part_bytes(p), workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  p.x = x; p.weight = weight; p.bias = bias; p.state0 = state_init; p.dy = dy; p.dstate_fin = dstate_final;
  p.dx = dx; p.dstate0 = dstate_init;
  p.part = reinterpret_cast<float*>(ws + map_bytes);
  hipError_t e = hipSuccess;
  if (p.map.ntok == 0) e = copy_states(dstate_final, dstate_init, sbytes, stream);
  else if (q->cu_seqlens) e = conv_sequences(q, ws, p, stream);
  if (e == hipSuccess) e = launch_conv_backward(p, q->dtype == RLA_BF16, dweight, dbias, stream);
  return to_status(e);
}

extern "C" rla_status rla_conv_decode(const rla_conv_problem* q, const void* x, const float* weight,
                                      const float* bias, const void* state_in, void* y, void* state_out,
                                      void* stream_) {
  ConvParams p;
  rla_status st = check_conv(q, p);
  if (st != RLA_OK) return st;
  if (q->cu_seqlens) return RLA_ERR_UNSUPPORTED;
  if (p.map.nseq == 0) return RLA_OK;
  if (!conv_decode_fits(p, q->dtype == RLA_BF16)) return RLA_ERR_SHAPE;
  st = conv_pointers(q, p, x, weight, bias, state_in);
  if (st != RLA_OK) return st;
  if (!state_out || (p.map.ntok > 0 && !y)) return RLA_ERR_NULL_ARG;
  const size_t sbytes = (size_t)p.map.nseq * (p.taps - 1) * p.D * elem(q->dtype);
  if (!aligned(y, elem(q->dtype)) || !aligned(state_out, elem(q->dtype)) ||
      (state_in != state_out && overlap(state_in, sbytes, state_out, sbytes)))
    return RLA_ERR_VALUE;
  p.x = x; p.weight = weight; p.bias = bias; p.state0 = state_in; p.y = y; p.state_fin = state_out;
  return to_status(launch_conv_decode(p, q->dtype == RLA_BF16, reinterpret_cast<hipStream_t>(stream_)));
}

// ---------------------------------------------------------------------------
// norms
// ---------------------------------------------------------------------------
namespace rla {
namespace {

constexpr int64_t kMaxRows = INT32_MAX - 4096, kMaxWidth = (int64_t)1 << 24;

rla_status check_addnorm(const rla_addnorm_problem* q, AddNormParams& p) {
  if (!q) return RLA_ERR_NULL_ARG;
  if (!is_type(q->dtype) || !is_type(q->residual_dtype)) return RLA_ERR_DTYPE;
  if (q->dtype == RLA_F32 && q->residual_dtype != RLA_F32) return RLA_ERR_DTYPE;
  if (q->rows < 0 || q->rows > kMaxRows || q->width < 1 || q->width > kMaxWidth) return RLA_ERR_SHAPE;
  if (!stride(q->x_stride, q->width, p.xs) || !stride(q->dn_stride, q->width, p.dns)) return RLA_ERR_SHAPE;
  if (times(times(q->rows, p.xs > p.dns ? p.xs : p.dns), 4) < 0) return RLA_ERR_SHAPE;
  if (!(q->eps >= 0.f) || isinf(q->eps)) return RLA_ERR_VALUE;
  p.rows = q->rows;
  p.width = q->width;
  p.eps = q->eps;
  p.wgs = addnorm_backward_wgs(q->rows, q->width, q->dtype == RLA_BF16);
  return RLA_OK;
}
size_t addnorm_bytes(const AddNormParams& p) { return up(sizeof(float) * 2 * (size_t)p.wgs * (size_t)p.width); }

rla_status check_gatenorm(const rla_gatenorm_problem* q, GateNormParams& p, int64_t& part_rows) {
  if (!q) return RLA_ERR_NULL_ARG;
  if (!is_type(q->dtype) || !is_type(q->x_dtype)) return RLA_ERR_DTYPE;
  if (q->dtype == RLA_F32 && q->x_dtype != RLA_F32) return RLA_ERR_DTYPE;
  if (q->tokens < 0 || q->heads < 1 || q->heads > (1 << 20) || q->width < 1 || q->width > kMaxWidth) return RLA_ERR_SHAPE;
  p.rows = times(q->tokens, q->heads);
  if (p.rows < 0 || p.rows > kMaxRows) return RLA_ERR_SHAPE;
  const int64_t token = q->heads * q->width;
  if (!stride(q->x_stride, token, p.xs) || !stride(q->gate_stride, token, p.gs) || !stride(q->do_stride, token, p.dos))
    return RLA_ERR_SHAPE;
  for (int64_t s : {p.xs, p.gs, p.dos})
    if (times(times(q->tokens, s), 4) < 0) return RLA_ERR_SHAPE;
  if (!(q->eps >= 0.f) || isinf(q->eps)) return RLA_ERR_VALUE;
  if ((q->gate_first & ~1) || (q->weight_per_head & ~1)) return RLA_ERR_VALUE;
  p.heads = q->heads;
  p.width = q->width;
  p.eps = q->eps;
  p.first = q->gate_first;
  p.wstride = q->weight_per_head ? q->width : 0;
  p.groups = gatenorm_backward_groups(p.rows > 0 ? p.rows : q->heads, q->heads, q->width, q->dtype == RLA_BF16, part_rows,
                                      q->weight_per_head != 0);
  return RLA_OK;
}

}  // namespace
}  // namespace rla

extern "C" size_t rla_addnorm_workspace_size(const rla_addnorm_problem* q) {
  AddNormParams p;
  return check_addnorm(q, p) == RLA_OK ? addnorm_bytes(p) : 0;
}

extern "C" rla_status rla_addnorm_forward(const rla_addnorm_problem* q, const void* x, const void* residual,
                                          const float* weight, const float* scale, void* n, void* residual_out,
                                          void* stream) {
  AddNormParams p;
  const rla_status st = check_addnorm(q, p);
  if (st != RLA_OK) return st;
  if (p.rows == 0) return RLA_OK;
  if (!x || !weight || !n || !residual_out) return RLA_ERR_NULL_ARG;
  const size_t el = elem(q->dtype), rl = elem(q->residual_dtype), bytes = (size_t)p.rows * p.width * rl;
  if (!aligned(x, el) || !aligned(n, el) || !aligned(residual, rl) || !aligned(residual_out, rl) ||
      !aligned(weight, 4) || !aligned(scale, 4) ||
      (residual != residual_out && overlap(residual, bytes, residual_out, bytes)))
    return RLA_ERR_VALUE;
  p.x = x; p.residual = residual; p.weight = weight; p.scale = scale; p.n = n; p.residual_out = residual_out;
  return to_status(launch_addnorm(p, q->dtype == RLA_BF16, q->residual_dtype == RLA_BF16, false,
                                  reinterpret_cast<hipStream_t>(stream)));
}

extern "C" rla_status rla_addnorm_backward(const rla_addnorm_problem* q, const void* dn, const void* dresidual_out,
                                           const void* residual_out, const void* x, const float* weight,
                                           const float* scale, void* dx, void* dresidual, float* dweight,
                                           float* dscale, void* workspace, size_t workspace_bytes, void* stream_) {
  AddNormParams p;
  rla_status st = check_addnorm(q, p);
  if (st != RLA_OK) return st;
  if (!weight || !dweight || (scale && !dscale)) return RLA_ERR_NULL_ARG;
  if (p.rows > 0 && (!dn || !residual_out || !dx || (scale && !x))) return RLA_ERR_NULL_ARG;
  const size_t el = elem(q->dtype), rl = elem(q->residual_dtype), bytes = (size_t)p.rows * p.width * rl;
  if (!aligned(dn, el) || !aligned(x, el) || !aligned(dx, el) || !aligned(dresidual_out, rl) ||
      !aligned(residual_out, rl) || !aligned(dresidual, rl) || !aligned(weight, 4) || !aligned(scale, 4) ||
      !aligned(dweight, 4) || !aligned(dscale, 4) || overlap(residual_out, bytes, dresidual, bytes) ||
      (dresidual != dresidual_out && overlap(dresidual_out, bytes, dresidual, bytes)))
    return RLA_ERR_VALUE;
  st = check_workspace(addnorm_bytes(p), workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  p.dn = dn; p.dresidual_out = dresidual_out; p.residual_in = residual_out; p.x = x; p.weight = weight;
  p.scale = scale; p.dx = dx; p.dresidual = dresidual;
  p.part = reinterpret_cast<float*>(workspace);
  // (without rows the kernel writes sums of nothing: zeros)
  hipError_t e = launch_addnorm(p, q->dtype == RLA_BF16, q->residual_dtype == RLA_BF16, true, stream);
  if (e == hipSuccess)
    e = launch_column_sums(p.part, p.wgs, (scale ? 2 : 1) * p.width, p.width, 1, dweight, scale ? dscale : nullptr, stream);
  return to_status(e);
}

extern "C" size_t rla_gatenorm_workspace_size(const rla_gatenorm_problem* q) {
  GateNormParams p;
  int64_t part_rows = 0;
  if (check_gatenorm(q, p, part_rows) != RLA_OK) return 0;
  return up(sizeof(float) * (size_t)part_rows * (size_t)p.width);
}

extern "C" rla_status rla_gatenorm_forward(const rla_gatenorm_problem* q, const void* x, const void* gate,
                                           const float* weight, void* o, void* stream) {
  GateNormParams p;
  int64_t part_rows = 0;
  const rla_status st = check_gatenorm(q, p, part_rows);
  if (st != RLA_OK) return st;
  if (p.rows == 0) return RLA_OK;
  if (!x || !gate || !weight || !o) return RLA_ERR_NULL_ARG;
  if (!aligned(x, elem(q->x_dtype)) || !aligned(gate, elem(q->dtype)) || !aligned(o, elem(q->dtype)) ||
      !aligned(weight, 4))
    return RLA_ERR_VALUE;
  p.x = x; p.gate = gate; p.weight = weight; p.o = o;
  return to_status(launch_gatenorm(p, q->dtype == RLA_BF16, q->x_dtype == RLA_BF16, false,
                                   reinterpret_cast<hipStream_t>(stream)));
}

extern "C" rla_status rla_gatenorm_backward(const rla_gatenorm_problem* q, const void* dO, const void* x,
                                            const void* gate, const float* weight, void* dx, void* dgate,
                                            float* dweight, void* workspace, size_t workspace_bytes, void* stream_) {
  GateNormParams p;
  int64_t part_rows = 0;
  rla_status st = check_gatenorm(q, p, part_rows);
  if (st != RLA_OK) return st;
  if (!weight || !dweight) return RLA_ERR_NULL_ARG;
  if (p.rows > 0 && (!dO || !x || !gate || !dx || !dgate)) return RLA_ERR_NULL_ARG;
  if (!aligned(x, elem(q->x_dtype)) || !aligned(dx, elem(q->x_dtype)) || !aligned(gate, elem(q->dtype)) ||
      !aligned(dO, elem(q->dtype)) || !aligned(dgate, elem(q->dtype)) || !aligned(weight, 4) || !aligned(dweight, 4))
    return RLA_ERR_VALUE;
  st = check_workspace(up(sizeof(float) * (size_t)part_rows * (size_t)p.width), workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  p.x = x; p.gate = gate; p.weight = weight; p.dO = dO; p.dx = dx; p.dgate = dgate;
  p.part = reinterpret_cast<float*>(workspace);
  hipError_t e = launch_gatenorm(p, q->dtype == RLA_BF16, q->x_dtype == RLA_BF16, true, stream);
  // weights per head: rows of all heads' groups side by side
  const int64_t cols = q->weight_per_head ? p.heads * p.width : p.width;
  const int64_t rows = q->weight_per_head ? p.groups / p.heads : part_rows;
  if (e == hipSuccess) e = launch_column_sums(p.part, rows, cols, cols, 1, dweight, nullptr, stream);
  return to_status(e);
}

// ---------------------------------------------------------------------------
// selective scan
// ---------------------------------------------------------------------------
namespace rla {
namespace {

// Workgroups that fill the card: chunks are added up to this many.  The training step of
// 4 x 4096 tokens x 4096 channels x 16 states (256 workgroups without chunks), us of the
// forward's two passes and the gradients' two: 1024: 161 + 347 + 200 + 1161; 512: 166 + 373
// + 201 + 1193; 2048: 187 + 343 + 220 + 1155; 256, no summaries: 533 and 1814.
constexpr int64_t kSsmFill = 1024, kSsmMinChunk = 64;

rla_status check_ssm(const rla_ssm_problem* q, SsmParams& p) {
  if (!q) return RLA_ERR_NULL_ARG;
  if (!is_type(q->dtype)) return RLA_ERR_DTYPE;
  const rla_status st = tokens(q->batch, q->seq_len, q->num_seqs, q->cu_seqlens, p.map);
  if (st != RLA_OK) return st;
  if (q->states < 1 || q->states > 64 || q->groups < 1 || q->channels < q->groups || q->channels >= (1 << 24) ||
      q->channels % q->groups != 0)
    return RLA_ERR_SHAPE;
  if (q->softplus != 0 && q->softplus != 1) return RLA_ERR_VALUE;
  p.D = q->channels;
  p.N = q->states;
  p.G = q->groups;
  p.Dg = p.D / p.G;
  p.softplus = q->softplus;
  if (!stride(q->u_stride, p.D, p.us) || !stride(q->delta_stride, p.D, p.dts) || !stride(q->z_stride, p.D, p.zs) ||
      !stride(q->do_stride, p.D, p.dos) || !stride(q->b_stride, p.G * p.N, p.bs) || !stride(q->c_stride, p.G * p.N, p.cs))
    return RLA_ERR_SHAPE;
  for (int64_t s : {p.us, p.dts, p.zs, p.dos, p.bs, p.cs})   // (24-bit row offsets)
    if (s >= (1 << 24) || times(times(p.map.ntok, s), 4) < 0) return RLA_ERR_SHAPE;
  if (times(times(p.map.nseq, p.D), p.N * 4) < 0) return RLA_ERR_SHAPE;
  const int64_t cb = ssm_channels(p.N);
  p.bpg = (int32_t)((p.Dg + cb - 1) / cb);
  const int64_t blocks = p.G * p.bpg, T = q->cu_seqlens ? p.map.ntok : p.map.T;
  const int64_t seqs = q->cu_seqlens ? 1 : p.map.nseq > 0 ? p.map.nseq : 1;
  int64_t n = (kSsmFill + blocks * seqs - 1) / (blocks * seqs);
  n = n < T / kSsmMinChunk ? n : T / kSsmMinChunk;
  n = n < 1 ? 1 : n > kSsmMaxChunks ? kSsmMaxChunks : n;
  p.L = ((T + n - 1) / n + kSsmTile - 1) / kSsmTile * kSsmTile;
  if (p.L == 0) p.L = kSsmTile;
  p.cps = (int32_t)((T + p.L - 1) / p.L);
  if (p.cps * blocks * seqs > INT32_MAX / 2) return RLA_ERR_SHAPE;
  p.nchunk = (int32_t)(p.cps * (q->cu_seqlens ? 1 : p.map.nseq));
  return RLA_OK;
}

// A forward or a backward: also few enough workgroups for a launch.
rla_status check_ssm_scan(const rla_ssm_problem* q, SsmParams& p) {
  const rla_status st = check_ssm(q, p);
  return st == RLA_OK && ssm_wgs(p) > kMaxWgs ? RLA_ERR_SHAPE : st;
}

struct SsmPlan {
  size_t map = 0, flags = 0, S = 0, sumd = 0, ck = 0, E = 0, pBC = 0, pA = 0, pD = 0, total = 0;
};
SsmPlan plan_ssm(const rla_ssm_problem* q, const SsmParams& p, bool backward) {
  SsmPlan w;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = up(off + bytes);
    return at;
  };
  const size_t NP = (size_t)ssm_padded(p.N), D = (size_t)p.D, nc = (size_t)p.nchunk;
  if (q->cu_seqlens) w.map = take(token_map_bytes(p.map.ntok, p.map.nseq));
  if (p.cps > 1) {
    w.flags = take(4 * nc);
    w.S = take(4 * nc * D * NP);
    w.sumd = take(4 * nc * D);
  }
  if (backward) {
    w.ck = take(4 * nc * (size_t)(p.L / kSsmSub) * D * NP);
    if (p.cps > 1) w.E = take(4 * nc * D * NP);
    w.pBC = take(4 * (size_t)(p.G * p.bpg) * (size_t)p.map.ntok * 2 * (size_t)p.N);
    w.pA = take(4 * nc * D * (size_t)p.N);
    w.pD = take(4 * nc * 2 * D);
  }
  w.total = off;
  return w;
}
void set_workspace(SsmParams& p, const SsmPlan& w, unsigned char* ws, bool backward) {
  auto f = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  p.flags = reinterpret_cast<int32_t*>(ws + w.flags);
  p.S = f(w.S);
  p.sumd = f(w.sumd);
  if (!backward) return;
  p.ck = f(w.ck);
  p.E = f(w.E);
  p.pBC = f(w.pBC);
  p.pA = f(w.pA);
  p.pD = f(w.pD);
}

rla_status ssm_inputs(const rla_ssm_problem* q, SsmParams& p, const void* u, const void* delta, const float* A,
                      const void* B, const void* C, const float* skip, const void* z, const float* dbias, const float* h0) {
  if (!A || (p.map.ntok > 0 && (!u || !delta || !B || !C))) return RLA_ERR_NULL_ARG;
  const size_t el = elem(q->dtype);
  for (const void* a : {u, delta, B, C, z})
    if (!aligned(a, el)) return RLA_ERR_VALUE;
  for (const float* a : {A, skip, dbias, h0})
    if (!aligned(a, 4)) return RLA_ERR_VALUE;
  p.u = u; p.delta = delta; p.A = A; p.B = B; p.C = C; p.skip = skip; p.z = z; p.dbias = dbias; p.h0 = h0;
  return RLA_OK;
}

size_t ssm_state_bytes(const SsmParams& p) { return (size_t)p.map.nseq * (size_t)p.D * (size_t)p.N * 4; }

}  // namespace
}  // namespace rla

extern "C" size_t rla_ssm_workspace_size(const rla_ssm_problem* q, int op) {
  SsmParams p;
  if (check_ssm_scan(q, p) != RLA_OK || (op != RLA_SSM_FORWARD && op != RLA_SSM_BACKWARD)) return 0;
  return plan_ssm(q, p, op == RLA_SSM_BACKWARD).total;
}

extern "C" rla_status rla_ssm_forward(const rla_ssm_problem* q, const void* u, const void* delta, const float* A,
                                      const void* B, const void* C, const float* skip, const void* z,
                                      const float* delta_bias, const float* h_init, void* o, float* h_final, int save,
                                      void* workspace, size_t workspace_bytes, void* stream_) {
  SsmParams p;
  rla_status st = check_ssm_scan(q, p);
  if (st == RLA_OK) st = ssm_inputs(q, p, u, delta, A, B, C, skip, z, delta_bias, h_init);
  if (st != RLA_OK) return st;
  if (p.map.ntok > 0 && !o) return RLA_ERR_NULL_ARG;
  const size_t sbytes = ssm_state_bytes(p);
  if (!aligned(o, elem(q->dtype)) || !aligned(h_final, 4) || overlap(h_init, sbytes, h_final, sbytes))
    return RLA_ERR_VALUE;
  const SsmPlan w = plan_ssm(q, p, save != 0);
  st = check_workspace(w.total, workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  if (p.map.ntok == 0) return to_status(copy_states(h_init, h_final, sbytes, stream));
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  set_workspace(p, w, ws, save != 0);
  p.o = o;
  p.hfin = h_final;
  hipError_t e = hipSuccess;
  if (q->cu_seqlens) e = launch_token_map(q->cu_seqlens, p.map.nseq, p.map.ntok, ws + w.map, true, p.map, stream);
  if (e == hipSuccess) e = launch_ssm_forward(p, q->dtype == RLA_BF16, stream);
  return to_status(e);
}

extern "C" rla_status rla_ssm_backward(const rla_ssm_problem* q, const void* u, const void* delta, const float* A,
                                       const void* B, const void* C, const float* skip, const void* z,
                                       const float* delta_bias, const float* h_init, const void* dO,
                                       const float* dh_final, void* du, void* ddelta, float* dA, void* dB, void* dC,
                                       float* dskip, void* dz, float* ddelta_bias, float* dh_init, int use_saved,
                                       void* workspace, size_t workspace_bytes, void* stream_) {
  SsmParams p;
  rla_status st = check_ssm_scan(q, p);
  if (st == RLA_OK) st = ssm_inputs(q, p, u, delta, A, B, C, skip, z, delta_bias, h_init);
  if (st != RLA_OK) return st;
  if (!dA || (skip && !dskip) || (delta_bias && !ddelta_bias)) return RLA_ERR_NULL_ARG;
  if (p.map.ntok > 0 && (!dO || !du || !ddelta || !dB || !dC || (z && !dz))) return RLA_ERR_NULL_ARG;
  const size_t el = elem(q->dtype), sbytes = ssm_state_bytes(p);
  for (const void* a : {(const void*)dO, (const void*)du, (const void*)ddelta, (const void*)dB, (const void*)dC, (const void*)dz})
    if (!aligned(a, el)) return RLA_ERR_VALUE;
  for (const float* a : {dh_final, (const float*)dA, (const float*)dskip, (const float*)ddelta_bias, (const float*)dh_init})
    if (!aligned(a, 4)) return RLA_ERR_VALUE;
  if (overlap(dh_final, sbytes, dh_init, sbytes)) return RLA_ERR_VALUE;
  const SsmPlan w = plan_ssm(q, p, true);
  st = check_workspace(w.total, workspace, workspace_bytes);
  if (st != RLA_OK) return st;
  hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
  const bool bf16 = q->dtype == RLA_BF16;
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  set_workspace(p, w, ws, true);
  hipError_t e = hipSuccess;
  if (p.map.ntok > 0) {
    if (q->cu_seqlens)
      e = launch_token_map(q->cu_seqlens, p.map.nseq, p.map.ntok, ws + w.map, !use_saved, p.map, stream);
    if (e == hipSuccess && !use_saved) e = launch_ssm_forward(p, bf16, stream);
    p.dO = dO; p.dhfin = dh_final; p.du = du; p.ddelta = ddelta; p.dB = dB; p.dC = dC; p.dz = dz; p.dh0 = dh_init;
    if (e == hipSuccess) e = launch_ssm_backward(p, bf16, stream);
  } else {
    e = copy_states(dh_final, dh_init, sbytes, stream);
  }
  const int64_t rows = p.map.ntok > 0 ? p.nchunk : 0;
  if (e == hipSuccess) e = launch_column_sums(p.pA, rows, p.D * p.N, p.D * p.N, 1, dA, nullptr, stream);
  if (e == hipSuccess && (skip || delta_bias))
    e = launch_column_sums(p.pD, rows, 2 * p.D, p.D, 1, skip ? dskip : nullptr, delta_bias ? ddelta_bias : nullptr, stream);
  return to_status(e);
}

extern "C" rla_status rla_ssm_decode(const rla_ssm_problem* q, const void* u, const void* delta, const float* A,
                                     const void* B, const void* C, const float* skip, const void* z,
                                     const float* delta_bias, const float* h_in, void* o, float* h_out, void* stream) {
  SsmParams p;
  rla_status st = check_ssm(q, p);
  if (st != RLA_OK) return st;
  if (q->cu_seqlens) return RLA_ERR_UNSUPPORTED;
  if (p.map.nseq == 0) return RLA_OK;
  if (ssm_decode_wgs(p) > kMaxWgs) return RLA_ERR_SHAPE;
  st = ssm_inputs(q, p, u, delta, A, B, C, skip, z, delta_bias, h_in);
  if (st != RLA_OK) return st;
  if (!h_out || (p.map.ntok > 0 && !o)) return RLA_ERR_NULL_ARG;
  const size_t sbytes = ssm_state_bytes(p);
  if (!aligned(o, elem(q->dtype)) || !aligned(h_out, 4) || (h_in != h_out && overlap(h_in, sbytes, h_out, sbytes)))
    return RLA_ERR_VALUE;
  p.o = o;
  p.hfin = h_out;
  return to_status(launch_ssm_decode(p, q->dtype == RLA_BF16, reinterpret_cast<hipStream_t>(stream)));
}

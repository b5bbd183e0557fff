// Shared by the host sides of rla_layer.h and rla_model.h: argument checks.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime.h>

#include "layer.hpp"
#include "rla.h"

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

}  // namespace
}  // namespace rla

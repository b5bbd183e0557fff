// The norms around a block, RMS(y) = y / sqrt(mean(y^2) + eps):
//   addnorm   residual_out = residual + scale x,  n = RMS(residual_out) weight
//   gatenorm  per head: o = RMS(x) weight SiLU(g), or RMS(x SiLU(g)) weight
// All are bound by HBM: a row is read once into registers, its statistics are
// sums over the row's lanes, and its outputs are written from the same
// registers.  With y^ = y inv, inv = 1 / sqrt(mean(y^2) + eps), a gradient d of
// y^ gives y the gradient inv (d - y^ mean(d y^)); the backward reads the rows
// again and takes inv anew, so nothing but the inputs is kept for it.  In a narrow
// row d - y^ mean(d y^) is the small difference of near equal terms (in a row of
// one value: eps inv^2 d), so each value's own term is taken out of both sums
// first (NormGrad).  Weight
// gradients: a lane keeps the sums of its columns over all its rows, written
// once per workgroup (or group of lanes) and summed by launch_column_sums.
//
// bf16, rows of 2048 with an fp32 stream (16384 of them) and of 128 (262144), us:
//   addnorm forward 88 (403 MB, 4.6 TB/s), gradients 109 (604 MB, 5.5 TB/s)
//   gatenorm forward 32 (201 MB, 6.3 TB/s: a part from the 256 MB last-level cache),
//   gradients 58 (336 MB, 5.8 TB/s)
// Of a few rows, latency: gatenorm 3.9 us (777 tokens x 16 heads of 128), of which two
// dependent round trips to memory; addnorm 5.7 (32 rows of 2048), where x, scale, stream
// and weight of each of a lane's four pieces are waited for one after the other.
#include "layer.hpp"

namespace rla {

namespace {

// Sum over aligned groups of L lanes; every lane gets it.
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
  v = group_sum<L < 16 ? L : 16>(v);
  if constexpr (L >= 32) v += __shfl_xor(v, 16);
  if constexpr (L >= 64) v += __shfl_xor(v, 32);
  return v;
}

// inv (d_i - y^_i mean(d y^)), from the row's sums S of y^2 and P of d y:
//   inv (d_i eps inv^2 + (d_i (S - y_i^2) - y_i (P - d_i y_i)) inv^2 / width)
struct NormGrad {
  float S, P, inv, k, floor;
  __device__ __forceinline__ NormGrad(float sum_yy, float sum_dy, float width, float eps) : S(sum_yy), P(sum_dy) {
    inv = rsqrtf(S / width + eps);
    k = inv * inv / width;
    floor = eps * inv * inv;
  }
  __device__ __forceinline__ float of(float d, float y) const {
    const float yy = y * y, dy = d * y;   // rounded as in the sums, not fused into the differences
    const float others = __builtin_fmaf(d, S - yy, -(y * (P - dy)));
    return inv * __builtin_fmaf(others, k, d * floor);
  }
};

// A row's piece at column c, `left` values of which exist (0 or less: none).  FULL:
// pieces are whole or absent, and an absent one's lane reads the row's start
// instead and takes zeros.  (The zeros are a branch behind the load, which waits for it.)
template <typename T, int V, bool FULL>
__device__ __forceinline__ void row_load(const T* row, int64_t c, int left, float (&x)[V]) {
  if constexpr (FULL) {
    load_piece<T, V, true>(row + (left > 0 ? c : 0), V, x);
    if (left <= 0)
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = 0.f;
  } else {
    load_piece<T, V>(row + c, left, x);
  }
}
template <typename T, int V, bool FULL, bool NT = false>
__device__ __forceinline__ void row_store(T* row, int64_t c, int left, const float (&x)[V]) {
  if constexpr (FULL) {
    if (left > 0) store_piece<T, V, true, NT>(row + c, V, x);
  } else {
    store_piece<T, V>(row + c, left, x);
  }
}

// Rows on L lanes, NP pieces of V values a lane: piece j of lane l starts at
// column (j L + l) V.
template <int L, int NP, int V> struct RowLanes {
  __device__ __forceinline__ static int lane() { return (int)threadIdx.x % L; }
  __device__ __forceinline__ static int64_t col(int j) { return (int64_t)(j * L + lane()) * V; }
  __device__ __forceinline__ static int left(int j, int64_t width) {
    const int64_t l = width - col(j);
    return l >= V ? V : (int)l;
  }
};

// Sum over the row's L lanes; rows of more than a wave: over the workgroup.
template <int L>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  v = lanes_sum<(L < 64 ? L : 64)>(v);
  if constexpr (L > 64) {
    const int w = threadIdx.x >> 6;
    __syncthreads();   // the previous sum is read
    if ((threadIdx.x & 63) == 0) lds[w] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < L / 64; ++i) v += lds[i];
  }
  return v;
}

// Two sums at once; `turn` alternates, so that one barrier a call is enough.
template <int L>
__device__ __forceinline__ void row_sums(float& a, float& b, float (&lds)[2][kWaves][2], int turn) {
  a = lanes_sum<(L < 64 ? L : 64)>(a);
  b = lanes_sum<(L < 64 ? L : 64)>(b);
  if constexpr (L > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      lds[turn][w][0] = a;
      lds[turn][w][1] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < L / 64; ++i) {
      a += lds[turn][i][0];
      b += lds[turn][i][1];
    }
  }
}

// ---------------------------------------------------------------------------
// Before a block.  A row is taken by a wave (up to 4 pieces a lane: 2048 bf16
// channels) or a workgroup; wider rows (NP = 0) are read twice, their sum
// first.
// ---------------------------------------------------------------------------
template <typename T, typename R, int L, int NP, bool FULL, bool NT>
__global__ __launch_bounds__(kThreads) void addnorm_fwd_kernel(AddNormParams p) {
  constexpr int V = kPiece<T>, N = NP ? NP : 1;
  typedef RowLanes<L, N, V> RL;
  __shared__ float lds[kWaves];
  const int64_t row = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (row >= p.rows) return;   // whole rows of lanes (L = kThreads: never)
  const T* x = reinterpret_cast<const T*>(p.x) + row * p.xs;
  const R* res = p.residual ? reinterpret_cast<const R*>(p.residual) + row * p.width : nullptr;
  T* n = reinterpret_cast<T*>(p.n) + row * p.width;
  R* out = reinterpret_cast<R*>(p.residual_out) + row * p.width;

  auto stream = [&](int64_t c, int left, float (&r)[V]) {   // the new stream's piece
    float s[V];
    row_load<T, V, FULL>(x, c, left, r);
    if (p.scale) {
      row_load<float, V, FULL>(p.scale, c, left, s);
#pragma unroll
      for (int e = 0; e < V; ++e) r[e] *= s[e];
    }
    if (res) {
      row_load<R, V, FULL>(res, c, left, s);
#pragma unroll
      for (int e = 0; e < V; ++e) r[e] += s[e];
    }
  };
  auto finish = [&](int64_t c, int left, const float (&r)[V], float inv) {
    float w[V];
    row_store<R, V, FULL, NT>(out, c, left, r);
    row_load<float, V, FULL>(p.weight, c, left, w);
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] *= r[e] * inv;
    row_store<T, V, FULL, NT>(n, c, left, w);
  };
  float ss = 0.f;
  if constexpr (NP > 0) {
    float r[N][V];
#pragma unroll
    for (int j = 0; j < N; ++j) stream(RL::col(j), RL::left(j, p.width), r[j]);
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) ss = __builtin_fmaf(r[j][e], r[j][e], ss);
    const float inv = rsqrtf(row_sum<L>(ss, lds) / (float)p.width + p.eps);
#pragma unroll
    for (int j = 0; j < N; ++j) finish(RL::col(j), RL::left(j, p.width), r[j], inv);
  } else {
    for (int64_t c = RL::col(0); c < p.width; c += L * V) {
      float r[V];
      stream(c, (int)min(p.width - c, (int64_t)V), r);
#pragma unroll
      for (int e = 0; e < V; ++e) ss = __builtin_fmaf(r[e], r[e], ss);
    }
    const float inv = rsqrtf(row_sum<L>(ss, lds) / (float)p.width + p.eps);
    for (int64_t c = RL::col(0); c < p.width; c += L * V) {
      float r[V];
      const int left = (int)min(p.width - c, (int64_t)V);
      stream(c, left, r);
      finish(c, left, r, inv);
    }
  }
}

// Rows blockIdx.x * (kThreads / L) + ..., a grid apart.  Column sums: [workgroup][2][width]
// (dweight, dscale), the workgroup's waves added in LDS.  NP = 0: the row in
// two passes, and the sums kept in the workgroup's partial row itself.
template <typename T, typename R, int L, int NP, bool FULL, bool NT>
__global__ __launch_bounds__(kThreads) void addnorm_bwd_kernel(AddNormParams p) {
  constexpr int V = kPiece<T>, N = NP ? NP : 1;
  typedef RowLanes<L, N, V> RL;
  __shared__ float lds[2][kWaves][2];
  int turn = 0;
  constexpr int kSub = kThreads / L;
  const bool scaled = p.scale != nullptr;
  float* part = p.part + (int64_t)blockIdx.x * (scaled ? 2 : 1) * p.width;
  const float wd = (float)p.width;

  struct Piece {
    float r[V], dn[V], w[V];
  };
  auto load = [&](int64_t row, int64_t c, int left, Piece& q) {
    row_load<R, V, FULL>(reinterpret_cast<const R*>(p.residual_in) + row * p.width, c, left, q.r);
    row_load<T, V, FULL>(reinterpret_cast<const T*>(p.dn) + row * p.dns, c, left, q.dn);
  };
  auto finish = [&](int64_t row, int64_t c, int left, const Piece& q, const NormGrad& ng, float (&dw)[V], float (&ds)[V]) {
    float dr[V], t[V];
    if (p.dresidual_out) {
      row_load<R, V, FULL>(reinterpret_cast<const R*>(p.dresidual_out) + row * p.width, c, left, dr);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) dr[e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      dw[e] = __builtin_fmaf(q.dn[e], q.r[e] * ng.inv, dw[e]);
      dr[e] += ng.of(q.dn[e] * q.w[e], q.r[e]);
    }
    if (p.dresidual) row_store<R, V, FULL, NT>(reinterpret_cast<R*>(p.dresidual) + row * p.width, c, left, dr);
    if (scaled) {
      row_load<T, V, FULL>(reinterpret_cast<const T*>(p.x) + row * p.xs, c, left, t);
#pragma unroll
      for (int e = 0; e < V; ++e) ds[e] = __builtin_fmaf(dr[e], t[e], ds[e]);
      row_load<float, V, FULL>(p.scale, c, left, t);
#pragma unroll
      for (int e = 0; e < V; ++e) dr[e] *= t[e];
    }
    row_store<T, V, FULL, NT>(reinterpret_cast<T*>(p.dx) + row * p.width, c, left, dr);
  };

  if constexpr (NP > 0) {
    __shared__ float sums[L < kThreads ? kSub : 1][L < kThreads ? L * N * V : 1];
    float dw[N][V], ds[N][V], w[N][V];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      row_load<float, V, FULL>(p.weight, RL::col(j), RL::left(j, p.width), w[j]);
#pragma unroll
      for (int e = 0; e < V; ++e) dw[j][e] = ds[j][e] = 0.f;
    }
    for (int64_t row = (int64_t)blockIdx.x * kSub + threadIdx.x / L; row < p.rows; row += (int64_t)gridDim.x * kSub) {
      Piece q[N];
      float ss = 0.f, sd = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) load(row, RL::col(j), RL::left(j, p.width), q[j]);
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          q[j].w[e] = w[j][e];
          ss += q[j].r[e] * q[j].r[e];
          sd += q[j].dn[e] * w[j][e] * q[j].r[e];
        }
      row_sums<L>(ss, sd, lds, turn);
      turn ^= 1;
      const NormGrad ng(ss, sd, wd, p.eps);
#pragma unroll
      for (int j = 0; j < N; ++j) finish(row, RL::col(j), RL::left(j, p.width), q[j], ng, dw[j], ds[j]);
    }
    auto write = [&](const float (&a)[N][V], float* to) {
      if constexpr (L == kThreads) {
#pragma unroll
        for (int j = 0; j < N; ++j) row_store<float, V, FULL>(to, RL::col(j), RL::left(j, p.width), a[j]);
      } else {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int e = 0; e < V; ++e) sums[threadIdx.x / L][RL::col(j) + e] = a[j][e];
        __syncthreads();
        for (int c = threadIdx.x; c < L * N * V; c += kThreads) {
          if (c >= p.width) break;
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < kSub; ++i) s += sums[i][c];
          to[c] = s;
        }
      }
    };
    write(dw, part);
    if (scaled) write(ds, part + p.width);
  } else {
    for (int64_t c = threadIdx.x; c < (scaled ? 2 : 1) * p.width; c += kThreads) part[c] = 0.f;
    __syncthreads();
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
      float ss = 0.f, sd = 0.f;
      for (int64_t c = RL::col(0); c < p.width; c += L * V) {
        const int left = (int)min(p.width - c, (int64_t)V);
        Piece q;
        load(row, c, left, q);
        row_load<float, V, FULL>(p.weight, c, left, q.w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          ss += q.r[e] * q.r[e];
          sd += q.dn[e] * q.w[e] * q.r[e];
        }
      }
      row_sums<L>(ss, sd, lds, turn);
      turn ^= 1;
      const NormGrad ng(ss, sd, wd, p.eps);
      for (int64_t c = RL::col(0); c < p.width; c += L * V) {
        const int left = (int)min(p.width - c, (int64_t)V);
        Piece q;
        float dw[V], ds[V];
        load(row, c, left, q);
        row_load<float, V, FULL>(p.weight, c, left, q.w);
        load_piece<float, V, FULL>(part + c, left, dw);
        if (scaled) load_piece<float, V, FULL>(part + p.width + c, left, ds);
        finish(row, c, left, q, ng, dw, ds);
        store_piece<float, V, FULL>(part + c, left, dw);
        if (scaled) store_piece<float, V, FULL>(part + p.width + c, left, ds);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// After a block.  A head's row is taken by L lanes, NP pieces each; rows wider than
// that (NP = 0) are read twice.
// ---------------------------------------------------------------------------
template <typename T, typename X, int L, int NP, bool FULL, bool FIRST, bool NT>
__global__ __launch_bounds__(kThreads) void gatenorm_fwd_kernel(GateNormParams p) {
  constexpr int V = kPiece<T>, N = NP ? NP : 1;
  typedef RowLanes<L, N, V> RL;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (row >= p.rows) return;
  const int64_t tok = (uint32_t)row / (uint32_t)p.heads, h = row - tok * p.heads;
  const X* x = reinterpret_cast<const X*>(p.x) + tok * p.xs + h * p.width;
  const T* g = reinterpret_cast<const T*>(p.gate) + tok * p.gs + h * p.width;
  const float* weight = p.weight + h * p.wstride;
  T* o = reinterpret_cast<T*>(p.o) + row * p.width;

  auto load = [&](int64_t c, int left, float (&y)[V], float (&act)[V]) {
    row_load<X, V, FULL>(x, c, left, y);
    row_load<T, V, FULL>(g, c, left, act);
  };
  auto gate = [&](float (&y)[V], float (&act)[V], float& ss) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      act[e] *= sigmoid_fast(act[e]);
      if (FIRST) y[e] *= act[e];
      ss = __builtin_fmaf(y[e], y[e], ss);
    }
  };
  auto finish = [&](int64_t c, int left, const float (&y)[V], const float (&act)[V], float inv) {
    float w[V];
    row_load<float, V, FULL>(weight, c, left, w);
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] *= y[e] * inv * (FIRST ? 1.f : act[e]);
    row_store<T, V, FULL, NT>(o, c, left, w);
  };
  float ss = 0.f;
  if constexpr (NP > 0) {
    float y[N][V], act[N][V];
#pragma unroll
    for (int j = 0; j < N; ++j) load(RL::col(j), RL::left(j, p.width), y[j], act[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) gate(y[j], act[j], ss);
    const float inv = rsqrtf(lanes_sum<L>(ss) / (float)p.width + p.eps);
#pragma unroll
    for (int j = 0; j < N; ++j) finish(RL::col(j), RL::left(j, p.width), y[j], act[j], inv);
  } else {
    float y[V], act[V];
    for (int64_t c = RL::col(0); c < p.width; c += L * V) {
      load(c, (int)min(p.width - c, (int64_t)V), y, act);
      gate(y, act, ss);
    }
    const float inv = rsqrtf(lanes_sum<L>(ss) / (float)p.width + p.eps);
    for (int64_t c = RL::col(0); c < p.width; c += L * V) {
      const int left = (int)min(p.width - c, (int64_t)V);
      load(c, left, y, act);
      gate(y, act, ss);
      finish(c, left, y, act, inv);
    }
  }
}

// Groups of L lanes take rows `groups` apart, a multiple of the heads: a group
// stays with one head.  Column sums: [group][width] for weights per head (rows of
// [groups / heads][heads][width]), else [workgroup][width].
template <typename T, typename X, int L, int NP, bool FULL, bool FIRST, bool NT>
__global__ __launch_bounds__(kThreads) void gatenorm_bwd_kernel(GateNormParams p) {
  constexpr int V = kPiece<T>, N = NP ? NP : 1, kSub = kThreads / L;
  typedef RowLanes<L, N, V> RL;
  const int64_t group = (int64_t)blockIdx.x * kSub + threadIdx.x / L;
  const int64_t h = (uint32_t)group % (uint32_t)p.heads, first = (uint32_t)group / (uint32_t)p.heads;
  const int64_t step = p.groups / p.heads, tokens = p.rows / p.heads;
  const float* weight = p.weight + h * p.wstride;
  const float wd = (float)p.width;

  struct Piece {
    float x[V], g[V], d[V];
  };
  auto load = [&](int64_t tok, int64_t c, int left, Piece& q) {
    row_load<X, V, FULL>(reinterpret_cast<const X*>(p.x) + tok * p.xs + h * p.width, c, left, q.x);
    row_load<T, V, FULL>(reinterpret_cast<const T*>(p.gate) + tok * p.gs + h * p.width, c, left, q.g);
    row_load<T, V, FULL>(reinterpret_cast<const T*>(p.dO) + tok * p.dos + h * p.width, c, left, q.d);
  };
  auto stats = [&](const Piece& q, const float (&w)[V], float& ss, float& sd) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float act = q.g[e] * sigmoid_fast(q.g[e]);
      const float y = FIRST ? q.x[e] * act : q.x[e];
      ss += y * y;
      sd += (FIRST ? q.d[e] : q.d[e] * act) * w[e] * y;
    }
  };
  auto finish = [&](int64_t tok, int64_t c, int left, const Piece& q, const float (&w)[V], const NormGrad& ng, float (&dw)[V]) {
    float dx[V], dg[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float act;
      const float slope = silu_grad_f(q.g[e], act);
      const float y = FIRST ? q.x[e] * act : q.x[e], hat = y * ng.inv;
      const float dn = FIRST ? q.d[e] : q.d[e] * act;
      const float dy = ng.of(dn * w[e], y);
      dw[e] = __builtin_fmaf(dn, hat, dw[e]);
      dx[e] = FIRST ? dy * act : dy;
      dg[e] = (FIRST ? dy * q.x[e] : q.d[e] * hat * w[e]) * slope;
    }
    const int64_t at = (tok * p.heads + h) * p.width;
    row_store<X, V, FULL, NT>(reinterpret_cast<X*>(p.dx) + at, c, left, dx);
    row_store<T, V, FULL, NT>(reinterpret_cast<T*>(p.dgate) + at, c, left, dg);
  };

  if constexpr (NP > 0) {
    float w[N][V], dw[N][V];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      row_load<float, V, FULL>(weight, RL::col(j), RL::left(j, p.width), w[j]);
#pragma unroll
      for (int e = 0; e < V; ++e) dw[j][e] = 0.f;
    }
    if (group < p.groups) {
      for (int64_t tok = first; tok < tokens; tok += step) {
        Piece q[N];
        float ss = 0.f, sd = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) load(tok, RL::col(j), RL::left(j, p.width), q[j]);
#pragma unroll
        for (int j = 0; j < N; ++j) stats(q[j], w[j], ss, sd);
        const NormGrad ng(lanes_sum<L>(ss), lanes_sum<L>(sd), wd, p.eps);
#pragma unroll
        for (int j = 0; j < N; ++j) finish(tok, RL::col(j), RL::left(j, p.width), q[j], w[j], ng, dw[j]);
      }
    }
    if (p.wstride) {   // per head: each group its own
      if (group < p.groups)
#pragma unroll
        for (int j = 0; j < N; ++j)
          row_store<float, V, FULL>(p.part + group * p.width, RL::col(j), RL::left(j, p.width), dw[j]);
      return;
    }
    __shared__ float sums[kSub][L * N * V];
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) sums[threadIdx.x / L][RL::col(j) + e] = dw[j][e];
    __syncthreads();
    for (int c = threadIdx.x; c < L * N * V && c < p.width; c += kThreads) {
      float s = 0.f;
      for (int i = 0; i < kSub; ++i) s += sums[i][c];
      p.part[(int64_t)blockIdx.x * p.width + c] = s;
    }
  } else {   // the sums in the group's partial row itself
    if (group >= p.groups) return;
    float* part = p.part + group * p.width;
    for (int64_t c = RL::col(0); c < p.width; c += L * V) {
      const float zero[V] = {};
      store_piece<float, V, FULL>(part + c, (int)min(p.width - c, (int64_t)V), zero);
    }
    for (int64_t tok = first; tok < tokens; tok += step) {
      float ss = 0.f, sd = 0.f;
      Piece q;
      float w[V], dw[V];
      for (int64_t c = RL::col(0); c < p.width; c += L * V) {
        const int left = (int)min(p.width - c, (int64_t)V);
        load(tok, c, left, q);
        row_load<float, V, FULL>(weight, c, left, w);
        stats(q, w, ss, sd);
      }
      const NormGrad ng(lanes_sum<L>(ss), lanes_sum<L>(sd), wd, p.eps);
      for (int64_t c = RL::col(0); c < p.width; c += L * V) {
        const int left = (int)min(p.width - c, (int64_t)V);
        load(tok, c, left, q);
        row_load<float, V, FULL>(weight, c, left, w);
        load_piece<float, V, FULL>(part + c, left, dw);
        finish(tok, c, left, q, w, ng, dw);
        store_piece<float, V, FULL>(part + c, left, dw);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
struct Shape {
  int L, NP;
};
// addnorm forward: a wave a row up to 4 pieces a lane (a narrow row leaves lanes idle: of
// 64 bf16 values 56 of the 64), then a workgroup, then two passes.
// Backward, where a lane holds its columns' sums beside the row: a wave a row of one
// piece a lane, then a workgroup (16384 rows of 2048 bf16 values with an fp32 stream: a
// wave with 4 pieces 195 us, one to a SIMD; a workgroup 109).
Shape addnorm_shape(int64_t width, int V, bool backward) {
  const int64_t pieces = (width + V - 1) / V;
  if (pieces <= 64) return Shape{64, 1};
  if (!backward && pieces <= 128) return Shape{64, 2};
  if (!backward && pieces <= 256) return Shape{64, 4};
  for (int NP : {1, 2, 4})
    if (pieces <= kThreads * NP) return Shape{kThreads, NP};
  return Shape{kThreads, 0};
}
// gatenorm: the fewest lanes that hold a row in a piece each, then more pieces
Shape gatenorm_shape(int64_t width, int V) {
  const int64_t pieces = (width + V - 1) / V;
  for (int L : {8, 16, 32, 64})
    if (pieces <= L) return Shape{L, 1};
  if (pieces <= 256) return Shape{64, 4};
  return Shape{64, 0};
}
// Workgroups that keep sums over many rows: enough to fill the card, few enough that the
// sums stay small beside the rows.  More where a workgroup leaves one row of sums for
// many rows at a time (gatenorm, one weight for all heads).
constexpr int64_t kBwdWgs = 512, kBwdRowWgs = 1024, kBwdNarrowWgs = 1024;

template <typename T, typename R, int L, int NP, bool FULL, bool NT>
hipError_t addnorm_forward(const AddNormParams& p, hipStream_t stream) {
  // (more rows than a launch holds: several)
  constexpr int64_t sub = kThreads / L, most = kMaxWgs * sub;
  AddNormParams part = p;
  for (int64_t row = 0; row < p.rows; row += most) {
    part.rows = min(p.rows - row, most);
    part.x = reinterpret_cast<const T*>(p.x) + row * p.xs;
    if (p.residual) part.residual = reinterpret_cast<const R*>(p.residual) + row * p.width;
    part.n = reinterpret_cast<T*>(p.n) + row * p.width;
    part.residual_out = reinterpret_cast<R*>(p.residual_out) + row * p.width;
    hipLaunchKernelGGL((addnorm_fwd_kernel<T, R, L, NP, FULL, NT>), dim3((uint32_t)((part.rows + sub - 1) / sub)),
                       dim3(kThreads), 0, stream, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename T, typename R, int L, int NP, bool FULL, bool NT>
hipError_t addnorm_backward(const AddNormParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((addnorm_bwd_kernel<T, R, L, NP, FULL, NT>), dim3((uint32_t)p.wgs), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}
template <typename T, typename R, bool FULL, bool NT>
hipError_t addnorm_shaped(const AddNormParams& p, bool backward, hipStream_t stream) {
  const Shape s = addnorm_shape(p.width, kPiece<T>, backward);
  if (backward) {
    if (s.L == 64) return addnorm_backward<T, R, 64, 1, FULL, NT>(p, stream);
    if (s.NP == 1) return addnorm_backward<T, R, kThreads, 1, FULL, NT>(p, stream);
    if (s.NP == 2) return addnorm_backward<T, R, kThreads, 2, FULL, NT>(p, stream);
    if (s.NP == 4) return addnorm_backward<T, R, kThreads, 4, FULL, NT>(p, stream);
    return addnorm_backward<T, R, kThreads, 0, FULL, NT>(p, stream);
  }
  if (s.L == 64) {
    if (s.NP == 1) return addnorm_forward<T, R, 64, 1, FULL, NT>(p, stream);
    if (s.NP == 2) return addnorm_forward<T, R, 64, 2, FULL, NT>(p, stream);
    return addnorm_forward<T, R, 64, 4, FULL, NT>(p, stream);
  }
  // (one piece of 256 lanes is four of a wave)
  if (s.NP == 2) return addnorm_forward<T, R, kThreads, 2, FULL, NT>(p, stream);
  if (s.NP == 4) return addnorm_forward<T, R, kThreads, 4, FULL, NT>(p, stream);
  return addnorm_forward<T, R, kThreads, 0, FULL, NT>(p, stream);
}
template <typename T, typename R> hipError_t addnorm(const AddNormParams& p, bool backward, hipStream_t stream) {
  if (p.width % kPiece<T> != 0) return addnorm_shaped<T, R, false, false>(p, backward, stream);
  return p.rows * p.width * (int64_t)(sizeof(T) + sizeof(R)) > kNtBytes ? addnorm_shaped<T, R, true, true>(p, backward, stream)
                                                                        : addnorm_shaped<T, R, true, false>(p, backward, stream);
}

template <typename T, typename X, int L, int NP, bool FULL, bool NT>
hipError_t gatenorm_run(const GateNormParams& p, bool backward, hipStream_t stream) {
  constexpr int64_t sub = kThreads / L;
  if (backward) {
    const dim3 grid((uint32_t)((p.groups + sub - 1) / sub));
    if (p.first) hipLaunchKernelGGL((gatenorm_bwd_kernel<T, X, L, NP, FULL, true, NT>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((gatenorm_bwd_kernel<T, X, L, NP, FULL, false, NT>), grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
  }
  // (more rows than a launch holds: several, of whole tokens each)
  const int64_t tokens = p.rows / p.heads, most = kMaxWgs * sub / p.heads;
  GateNormParams part = p;
  for (int64_t tok = 0; tok < tokens; tok += most) {
    part.rows = min(tokens - tok, most) * p.heads;
    part.x = reinterpret_cast<const X*>(p.x) + tok * p.xs;
    part.gate = reinterpret_cast<const T*>(p.gate) + tok * p.gs;
    part.o = reinterpret_cast<T*>(p.o) + tok * p.heads * p.width;
    const dim3 grid((uint32_t)((part.rows + sub - 1) / sub));
    if (p.first) hipLaunchKernelGGL((gatenorm_fwd_kernel<T, X, L, NP, FULL, true, NT>), grid, dim3(kThreads), 0, stream, part);
    else hipLaunchKernelGGL((gatenorm_fwd_kernel<T, X, L, NP, FULL, false, NT>), grid, dim3(kThreads), 0, stream, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename T, typename X, bool FULL, bool NT>
hipError_t gatenorm_shaped(const GateNormParams& p, bool backward, hipStream_t stream) {
  const Shape s = gatenorm_shape(p.width, kPiece<T>);
  if (s.L == 8) return gatenorm_run<T, X, 8, 1, FULL, NT>(p, backward, stream);
  if (s.L == 16) return gatenorm_run<T, X, 16, 1, FULL, NT>(p, backward, stream);
  if (s.L == 32) return gatenorm_run<T, X, 32, 1, FULL, NT>(p, backward, stream);
  if (s.NP == 1) return gatenorm_run<T, X, 64, 1, FULL, NT>(p, backward, stream);
  if (s.NP == 4) return gatenorm_run<T, X, 64, 4, FULL, NT>(p, backward, stream);
  return gatenorm_run<T, X, 64, 0, FULL, NT>(p, backward, stream);
}
template <typename T, typename X> hipError_t gatenorm(const GateNormParams& p, bool backward, hipStream_t stream) {
  if (p.width % kPiece<T> != 0) return gatenorm_shaped<T, X, false, false>(p, backward, stream);
  const int64_t written = p.rows * p.width * (int64_t)(sizeof(T) + (backward ? sizeof(X) : 0));
  return written > kNtBytes ? gatenorm_shaped<T, X, true, true>(p, backward, stream)
                            : gatenorm_shaped<T, X, true, false>(p, backward, stream);
}

}  // namespace

int64_t addnorm_backward_wgs(int64_t rows, int64_t width, bool bf16) {
  const int64_t sub = kThreads / addnorm_shape(width, bf16 ? 8 : 4, true).L;
  return max((int64_t)1, min(sub == 1 ? kBwdRowWgs : kBwdWgs, (rows + sub - 1) / sub));
}

int64_t gatenorm_backward_groups(int64_t rows, int64_t heads, int64_t width, bool bf16, int64_t& part_rows, bool per_head) {
  const Shape s = gatenorm_shape(width, bf16 ? 8 : 4);
  const int64_t sub = kThreads / s.L;
  int64_t groups = min(rows, (per_head || s.NP == 0 ? kBwdWgs : kBwdNarrowWgs) * sub);
  groups = max((int64_t)1, groups / heads) * heads;   // whole sets of heads
  part_rows = per_head || s.NP == 0 ? groups : (groups + sub - 1) / sub;
  return groups;
}

hipError_t launch_addnorm(const AddNormParams& p, bool bf16, bool res_bf16, bool backward, hipStream_t stream) {
  if (!bf16) return addnorm<float, float>(p, backward, stream);
  return res_bf16 ? addnorm<u16, u16>(p, backward, stream) : addnorm<u16, float>(p, backward, stream);
}

hipError_t launch_gatenorm(const GateNormParams& p, bool bf16, bool x_bf16, bool backward, hipStream_t stream) {
  if (!bf16) return gatenorm<float, float>(p, backward, stream);
  return x_bf16 ? gatenorm<u16, u16>(p, backward, stream) : gatenorm<u16, float>(p, backward, stream);
}

}  // namespace rla

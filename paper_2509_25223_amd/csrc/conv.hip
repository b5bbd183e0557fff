// Short causal depthwise convolution of a layer's projections:
//   pre_t = bias + sum_i weight_i x_{t-W+1+i},  y_t = pre_t or SiLU(pre_t)
// A channel is W multiply-adds a token, so every kernel here is bound by HBM:
// each value is read once (twice where a stretch's first rows are its
// neighbour's last) and written once.  A thread owns a piece of a row (forward and
// single tokens: 16 bytes, 8 bf16 or 4 fp32 channels; gradients: 4 channels) and
// walks a stretch of tokens with the last W - 1 rows in registers, so the taps cost no
// loads; the lanes of a wave take adjacent pieces of one row, so that an access of a
// wave is 1 KB of adjacent bytes (bf16 gradients: 512).
// bf16, four taps, bias and SiLU, us (and of the 5.4 TB/s of a large copy's traffic):
//   forward, 16384 x 6144 (403 MB)             84.3   4.8 TB/s
//   forward, 20011 x 2048 packed, of wider rows 35.6   4.6 TB/s
//   gradients, 16384 x 6144 (604 MB)            126   4.8 TB/s
// The forward has its loads in flight a batch of 8 rows ahead of their use; in the
// gradients, SiLU' is some 25 instructions a value and shares the time with the loads.
//
// Rows before a sequence's start are its state's, [W-1][D] with the oldest first:
// the row m before the start is state row W-2-m.
#include "layer.hpp"

namespace rla {

namespace {

// state row r of sequence n for the piece at channel c
template <typename T, int W, int V, bool FULL>
__device__ __forceinline__ void load_state(const void* state, int n, int r, int64_t D, int64_t c, int left,
                                           float (&x)[V]) {
  if (state == nullptr || n < 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = 0.f;
    return;
  }
  load_piece<T, V, FULL>(reinterpret_cast<const T*>(state) + ((int64_t)n * (W - 1) + r) * D + c, left, x);
}

// the piece's taps and bias
template <int W, int V, bool FULL>
__device__ __forceinline__ void load_taps(const ConvParams& p, int64_t c, int left, float (&w)[V * W], float (&b)[V]) {
  load_piece<float, V * W, FULL>(p.weight + c * W, left * W, w);
  if (p.bias) load_piece<float, V, FULL>(p.bias + c, left, b);
  else
#pragma unroll
    for (int e = 0; e < V; ++e) b[e] = 0.f;
}

template <int W, int V>
__device__ __forceinline__ float tap_sum(const float (&w)[V * W], float bias, int e, float x, const float (&win)[W - 1][V]) {
  float s = bias;
#pragma unroll
  for (int j = W - 2; j >= 0; --j) s = __builtin_fmaf(w[e * W + W - 2 - j], win[j][e], s);
  return __builtin_fmaf(w[e * W + W - 1], x, s);
}

// Packed sequences without a map (few of them): offset i, the running maximum being the
// caller's.  The same value in every lane, loaded as scalars.
__device__ __forceinline__ int32_t offset(const ConvParams& p, int i) {
  const int32_t v = ((ConstPtr<int32_t>)(uint64_t)p.cu)[min(i, p.map.nseq)];
  return min(max(v, 0), (int32_t)p.map.ntok);
}
__device__ __forceinline__ int seq_of(const ConvParams& p, int64_t t) {
  if (!p.cu) return p.map.seq_of(t);
  int32_t m = 0, below = 0;   // offsets up to t
  for (int i = 0; i <= p.map.nseq; ++i) {
    m = max(m, offset(p, i));
    below += m <= (int32_t)t ? 1 : 0;
  }
  return below > p.map.nseq ? -1 : below - 1;
}
__device__ __forceinline__ bool is_empty(const ConvParams& p, int n) {
  if (!p.cu) return p.map.empty[n];
  int32_t m = 0;
  for (int i = 0; i <= n; ++i) m = max(m, offset(p, i));
  return offset(p, n + 1) <= m;
}

// Tokens t and around: bit i of `before`: token t - i starts a sequence (i < 3); bit i of
// `bits`: token t + i does (i < 32, with WIDE 64; set past the end); t's sequence.
template <bool WIDE>
__device__ __forceinline__ void tokens_around(const ConvParams& p, int64_t t, bool want, uint32_t& before, uint64_t& bits,
                                              int& n) {
  if (p.cu) {
    uint64_t b = t < 3 ? 7ull >> t : 0ull;   // bit i: token t - 2 + i; token 0 and those in front
    int32_t m = 0, below = 0;
    constexpr int U = 8;
    for (int i0 = 0; i0 <= p.map.nseq; i0 += U) {
      int32_t v[U];
#pragma unroll
      for (int i = 0; i < U; ++i) v[i] = offset(p, i0 + i);   // (past the last: the last again)
#pragma unroll
      for (int i = 0; i < U; ++i) {
        m = max(m, v[i]);
        const uint32_t d = (uint32_t)(m - (int32_t)t + 2);
        b |= d < 64 ? 1ull << d : 0ull;
        below += i0 + i <= p.map.nseq && m <= (int32_t)t ? 1 : 0;
      }
    }
    const int64_t left = p.map.ntok - t + 2;
    if (left < 64) b |= ~0ull << left;
    before = (uint32_t)((b >> 2 & 1) | (b & 2) | (b << 2 & 4));
    bits = b >> 2;
    n = below > p.map.nseq ? -1 : below - 1;
    return;
  }
  bits = p.map.start_bits(t);
  before = (uint32_t)bits & 1u;
  const int64_t t1 = t > 2 ? t - 2 : 0;
  const uint32_t near = p.map.start_bits(t1);
#pragma unroll
  for (int i = 1; i < 3; ++i) before |= (t - i < 0 ? 1u : (near >> (t - i - t1)) & 1u) << i;
  if constexpr (WIDE) bits |= t + 32 < p.map.ntok ? (uint64_t)p.map.start_bits(t + 32) << 32 : ~0ull << 32;
  n = want ? p.map.seq_of(t) : 0;
}

// win[j] = the row before token t by j + 1, from x or the state; returns how many
// tokens of t's sequence lie before t (W - 1 for that many or more)
template <typename T, int W, int V, bool FULL>
__device__ __forceinline__ int load_window(const ConvParams& p, const T* x, int64_t t, uint32_t before, int n, int64_t c,
                                           int left, float (&win)[W - 1][V]) {
  int pos = 0;
  while (pos < W - 1 && !((before >> pos) & 1u)) ++pos;
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    if (j < pos) load_piece<T, V, FULL>(x + (t - 1 - j) * p.xs + c, left, win[j]);
    else load_state<T, W, V, FULL>(p.state0, n, W - 2 - (j - pos), p.D, c, left, win[j]);
  }
  return pos;
}

template <typename T, int W, int V, bool FULL>
__device__ __forceinline__ void load_state_window(const ConvParams& p, int n, int64_t c, int left, float (&win)[W - 1][V]) {
#pragma unroll
  for (int j = 0; j < W - 1; ++j) load_state<T, W, V, FULL>(p.state0, n, W - 2 - j, p.D, c, left, win[j]);
}

template <bool SILU> __device__ __forceinline__ float activation(float s) { return SILU ? s * sigmoid_fast(s) : s; }

template <typename T, int W, int TT, bool SILU, bool NT, bool FULL>
__device__ __forceinline__ void conv_fwd_stretch(const ConvParams& p, int64_t t0, int64_t c, int left) {
  constexpr int V = kPiece<T>;
  const T* x = reinterpret_cast<const T*>(p.x);
  T* y = reinterpret_cast<T*>(p.y);
  T* fin = reinterpret_cast<T*>(p.state_fin);
  float w[V * W], bias[V], win[W - 1][V];
  load_taps<W, V, FULL>(p, c, left, w, bias);
  uint32_t before;
  uint64_t around;
  int n;
  tokens_around<false>(p, t0, p.map.seq || p.state0 || fin, before, around, n);
  const uint32_t bits = (uint32_t)around;
  load_window<T, W, V, FULL>(p, x, t0, before, n, c, left, win);
  auto token = [&](const float (&xv)[V], int64_t t) {
    float o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      o[e] = activation<SILU>(tap_sum<W, V>(w, bias[e], e, xv[e], win));
    }
    store_piece<T, V, FULL, NT>(y + t * p.D + c, left, o);
#pragma unroll
    for (int j = W - 2; j > 0; --j)
#pragma unroll
      for (int e = 0; e < V; ++e) win[j][e] = win[j - 1][e];
#pragma unroll
    for (int e = 0; e < V; ++e) win[0][e] = xv[e];
  };
  // no start behind the first token: one sequence, loads a batch ahead of their use
  if (t0 + TT <= p.map.ntok && (bits & (((1u << TT) - 1u) << 1)) == 0 && n >= 0) {
    constexpr int U = TT < 8 ? TT : 8;
    typename RowVec<T, V>::type raw[2][U];
#pragma unroll
    for (int k = 0; k < U; ++k) load_raw<T, V, FULL>(x + (t0 + k) * p.xs + c, left, raw[0][k]);
#pragma unroll
    for (int k0 = 0; k0 < TT; k0 += U) {
      if (k0 + U < TT)
#pragma unroll
        for (int k = 0; k < U; ++k) load_raw<T, V, FULL>(x + (t0 + k0 + U + k) * p.xs + c, left, raw[(k0 / U + 1) & 1][k]);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        float xv[V];
#pragma unroll
        for (int e = 0; e < V; ++e) xv[e] = to_f<T>(raw[k0 / U & 1][k][e]);
        token(xv, t0 + k0 + k);
      }
    }
    return;
  }
  const int count = (int)min((int64_t)TT, p.map.ntok - t0);
  for (int k = 0; k < count; ++k) {
    if (k > 0 && ((bits >> k) & 1u)) {
      n = seq_of(p, t0 + k);
      load_state_window<T, W, V, FULL>(p, n, c, left, win);
    }
    float xv[V];
    if (n < 0) {   // outside every sequence
#pragma unroll
      for (int e = 0; e < V; ++e) xv[e] = 0.f;
      store_piece<T, V, FULL>(y + (t0 + k) * p.D + c, left, xv);
      continue;
    }
    load_piece<T, V, FULL>(x + (t0 + k) * p.xs + c, left, xv);
    token(xv, t0 + k);
    if (fin && ((bits >> (k + 1)) & 1u)) {   // the sequence's last token: the window is its state
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        store_piece<T, V, FULL>(fin + ((int64_t)n * (W - 1) + W - 2 - j) * p.D + c, left, win[j]);
    }
  }
}

// Workgroups past `main_wgs`: the states of sequences without tokens are copied
// (from NULL: zeros).
template <typename T, int W>
__device__ __forceinline__ void copy_empty_states(const ConvParams& p, const void* from, void* to, uint32_t wg,
                                                  uint32_t wgs) {
  const int64_t row = (W - 1) * p.D;
  for (int64_t n = wg; n < p.map.nseq; n += wgs) {
    if (!is_empty(p, (int)n)) continue;
    for (int64_t i = threadIdx.x; i < row; i += kThreads)
      reinterpret_cast<T*>(to)[n * row + i] = from ? reinterpret_cast<const T*>(from)[n * row + i] : from_f<T>(0.f);
  }
}

constexpr uint32_t kEmptyWgs = 32;

template <typename T, int W, int TT, bool SILU, bool NT>
__global__ __launch_bounds__(kThreads) void conv_fwd_kernel(ConvParams p, uint32_t pieces, uint32_t count,
                                                            uint32_t main_wgs) {
  constexpr int V = kPiece<T>;
  if (blockIdx.x >= main_wgs) {
    copy_empty_states<T, W>(p, p.state0, p.state_fin, blockIdx.x - main_wgs, kEmptyWgs);
    return;
  }
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  if (id >= count) return;
  const int64_t t0 = (int64_t)(id / pieces) * TT, c = (int64_t)(id % pieces) * V;
  const int left = (int)min(p.D - c, (int64_t)V);
  if (left == V) conv_fwd_stretch<T, W, TT, SILU, NT, true>(p, t0, c, left);
  else conv_fwd_stretch<T, W, TT, SILU, NT, false>(p, t0, c, left);
}

// Single tokens: a thread owns a piece of one sequence, loads its state before it
// writes any (in place works).  256 sequences x 6144 channels of bf16, four taps: 8.5 us
// for 25 MB.  What bounds it is latency: each load stands behind the branch that parts
// a whole piece from a row's last one, and is waited for there, so the three rows of the
// state, the taps and the token's row are round trips to memory one after the other.
template <typename T, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_decode_kernel(ConvParams p, uint32_t pieces, uint32_t count) {
  constexpr int V = kPiece<T>;
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  if (id >= count) return;
  const int n = (int)(id / pieces);
  const int64_t c = (int64_t)(id % pieces) * V;
  const int left = (int)min(p.D - c, (int64_t)V);
  float w[V * W], bias[V], win[W - 1][V];
  load_state_window<T, W, V, false>(p, n, c, left, win);
  load_taps<W, V, false>(p, c, left, w, bias);
  for (int64_t k = 0; k < p.map.T; ++k) {
    const int64_t t = n * p.map.T + k;
    float xv[V], o[V];
    load_piece<T, V>(reinterpret_cast<const T*>(p.x) + t * p.xs + c, left, xv);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      o[e] = activation<SILU>(tap_sum<W, V>(w, bias[e], e, xv[e], win));
#pragma unroll
      for (int j = W - 2; j > 0; --j) win[j][e] = win[j - 1][e];
      win[0][e] = xv[e];
    }
    store_piece<T, V>(reinterpret_cast<T*>(p.y) + t * p.D + c, left, o);
  }
  T* fin = reinterpret_cast<T*>(p.state_fin);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) store_piece<T, V>(fin + ((int64_t)n * (W - 1) + W - 2 - j) * p.D + c, left, win[j]);
}

// ---------------------------------------------------------------------------
// Backward.  dpre_t = dy_t (SiLU'(pre_t)); the row u steps before t gets
// weight_{W-1-u} dpre_t.  A thread walks its stretch and the W - 1 tokens behind
// it, with the last W - 1 rows and their gradients so far in registers: a row's
// gradient is complete W - 1 tokens later, or where its sequence ends, and is
// written once.  dweight and dbias are summed over the stretch in registers,
// over the workgroup's stretches in LDS, and over the workgroups by
// launch_column_sums.
// ---------------------------------------------------------------------------
constexpr int kBwdTokens = 32;

constexpr int kBwdV = 4;   // channels a thread (8: registers for two waves a SIMD only)

template <typename T, int W, bool SILU, bool NT, bool FULL>
__device__ __forceinline__ void conv_bwd_stretch(const ConvParams& p, int64_t t0, int64_t c, int left, float (&dw)[kBwdV * W],
                                                 float (&db)[kBwdV]) {
  constexpr int V = kBwdV, TT = kBwdTokens;
  const T* x = reinterpret_cast<const T*>(p.x);
  const T* dy = reinterpret_cast<const T*>(p.dy);
  T* dx = reinterpret_cast<T*>(p.dx);
  const T* dfin = reinterpret_cast<const T*>(p.dstate_fin);
  T* dst0 = reinterpret_cast<T*>(p.dstate0);
  float w[V * W], bias[V], win[W - 1][V], g[W - 1][V];
  load_taps<W, V, FULL>(p, c, left, w, bias);
  uint32_t before;
  uint64_t bits;
  int n;
  tokens_around<true>(p, t0, true, before, bits, n);
  const int pos0 = load_window<T, W, V, FULL>(p, x, t0, before, n, c, left, win);
#pragma unroll
  for (int j = 0; j < W - 1; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) g[j][e] = 0.f;

  // one token: its gradient into the rows of the window, g[W-2] then complete
  auto token = [&](const float (&xv)[V], const float (&dyv)[V], bool own, float (&done)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float d = dyv[e], act;
      if (SILU) d *= silu_grad_f(tap_sum<W, V>(w, bias[e], e, xv[e], win), act);
      if (own) {
        db[e] += d;
        dw[e * W + W - 1] = __builtin_fmaf(d, xv[e], dw[e * W + W - 1]);
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        if (own) dw[e * W + W - 2 - j] = __builtin_fmaf(d, win[j][e], dw[e * W + W - 2 - j]);
        g[j][e] = __builtin_fmaf(w[e * W + W - 2 - j], d, g[j][e]);
      }
      done[e] = g[W - 2][e];
#pragma unroll
      for (int j = W - 2; j > 0; --j) {
        win[j][e] = win[j - 1][e];
        g[j][e] = g[j - 1][e];
      }
      win[0][e] = xv[e];
      g[0][e] = w[e * W + W - 1] * d;
    }
  };

  if (t0 + TT + W - 1 <= p.map.ntok && (bits & (((1ull << (TT + W - 2)) - 1ull) << 1)) == 0 &&
      !((bits & 1ull) && dst0) && n >= 0) {
    constexpr int U = 5, TE = TT + W - 1;   // tokens a batch, loaded a batch ahead (35 = 7 x 5 for four taps)
    typename RowVec<T, V>::type rx[2][U], ry[2][U];
    auto load = [&](int k0, int to) {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int64_t t = t0 + min(k0 + k, TE - 1);
        load_raw<T, V, FULL>(x + t * p.xs + c, left, rx[to][k]);
        load_raw<T, V, FULL>(dy + t * p.dys + c, left, ry[to][k]);
      }
    };
    load(0, 0);
#pragma unroll
    for (int k0 = 0; k0 < TE; k0 += U) {
      if (k0 + U < TE) load(k0 + U, (k0 / U + 1) & 1);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (k0 + k >= TE) break;
        float xv[V], dyv[V], done[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          xv[e] = to_f<T>(rx[k0 / U & 1][k][e]);
          dyv[e] = to_f<T>(ry[k0 / U & 1][k][e]);
        }
        token(xv, dyv, k0 + k < TT, done);
        if (k0 + k >= W - 1) store_piece<T, V, FULL, NT>(dx + (t0 + k0 + k - (W - 1)) * p.D + c, left, done);
      }
    }
    return;
  }

  // any starts: `start` is the current sequence's first token (further back than the
  // window: as good as anywhere there)
  int64_t start = pos0 < W - 1 ? t0 - pos0 : t0 - 64;
  const int64_t own_end = min(t0 + TT, p.map.ntok);
  // gradient of the row `back` + 1 tokens before t (a token of the sequence, or a row of
  // its state), if this thread's to write; at the sequence's end its final state's too
  auto emit = [&](int64_t t, int back, float (&v)[V], bool end) {
    const int64_t at = t - 1 - back;
    if (end && dfin && n >= 0) {
      float f[V];
      load_piece<T, V, FULL>(dfin + ((int64_t)n * (W - 1) + W - 2 - back) * p.D + c, left, f);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] += f[e];
    }
    if (at >= start) {
      if (at >= t0 && at < own_end) store_piece<T, V, FULL>(dx + at * p.D + c, left, v);
    } else if (dst0 && n >= 0 && start >= t0 && start < own_end) {
      const int64_t r = W - 1 - (start - at);   // the row start - at before the start
      store_piece<T, V, FULL>(dst0 + ((int64_t)n * (W - 1) + r) * p.D + c, left, v);
    }
  };
  // rows kAhead tokens ahead of their use (whose they are shows when they are used)
  constexpr int kAhead = 4;
  typename RowVec<T, V>::type ax[kAhead], ay[kAhead];
  auto ahead = [&](int64_t t, int to) {
    t = min(t, p.map.ntok - 1);
    load_raw<T, V, FULL>(x + t * p.xs + c, left, ax[to]);
    load_raw<T, V, FULL>(dy + t * p.dys + c, left, ay[to]);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) ahead(t0 + i, i);
  for (int k = 0; k <= TT + W - 2; ++k) {
    const int64_t t = t0 + k;
    if (k > 0 && ((bits >> k) & 1ull)) {   // the sequence ended before t (or all tokens did)
#pragma unroll
      for (int j = 0; j < W - 1; ++j) emit(t, j, g[j], true);
      if (t >= own_end) return;
      n = seq_of(p, t);
      start = t;
      load_state_window<T, W, V, FULL>(p, n, c, left, win);
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) g[j][e] = 0.f;
    }
    float xv[V], dyv[V], done[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      xv[e] = to_f<T>(ax[0][e]);
      dyv[e] = to_f<T>(ay[0][e]);
    }
#pragma unroll
    for (int i = 1; i < kAhead; ++i) {
      ax[i - 1] = ax[i];
      ay[i - 1] = ay[i];
    }
    ahead(t + kAhead, kAhead - 1);
    if (n >= 0) {
      token(xv, dyv, k < TT, done);
      emit(t + 1, W - 1, done, false);   // the row W - 1 before t
    } else if (k < TT) {   // outside every sequence
#pragma unroll
      for (int e = 0; e < V; ++e) xv[e] = 0.f;
      store_piece<T, V, FULL>(dx + t * p.D + c, left, xv);
    }
  }
}

// lanes: adjacent pieces (kLanes of them), then stretches
// (three waves a SIMD, 168 registers: whole pieces of one sequence fit, while a row's
// partial piece and stretches with starts spill 57 to 125.  For 16384 tokens x 6144
// channels of bf16 two waves took 1.05 times as long; four, where whole pieces spill
// too, 1.74 times)
template <typename T, int W, bool SILU, bool NT>
__global__ __launch_bounds__(kThreads, 3) void conv_bwd_kernel(ConvParams p, uint32_t lanes, uint32_t groups,
                                                            uint32_t main_wgs) {
  constexpr int V = kBwdV;
  if (blockIdx.x >= main_wgs) {
    copy_empty_states<T, W>(p, p.dstate_fin, p.dstate0, blockIdx.x - main_wgs, kEmptyWgs);
    return;
  }
  __shared__ float sums[kThreads][V * (W + 1) + 1];
  const uint32_t row = blockIdx.x / groups, lane = threadIdx.x % lanes, sub = threadIdx.x / lanes, subs = kThreads / lanes;
  const int64_t c = ((int64_t)(blockIdx.x % groups) * lanes + lane) * V;
  const int64_t t0 = ((int64_t)row * subs + sub) * kBwdTokens;
  const int left = (int)min(max(p.D - c, (int64_t)0), (int64_t)V);
  float dw[V * W], db[V];
#pragma unroll
  for (int e = 0; e < V * W; ++e) dw[e] = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) db[e] = 0.f;
  if (left > 0 && t0 < p.map.ntok) {
    if (left == V) conv_bwd_stretch<T, W, SILU, NT, true>(p, t0, c, left, dw, db);
    else conv_bwd_stretch<T, W, SILU, NT, false>(p, t0, c, left, dw, db);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int i = 0; i < W; ++i) sums[threadIdx.x][i * V + e] = dw[e * W + i];
    sums[threadIdx.x][W * V + e] = db[e];
  }
  __syncthreads();
  // (tap, channel) of the workgroup's channels, over its stretches in order
  const int width = (int)lanes * V;
  for (int o = threadIdx.x; o < width * (W + 1); o += kThreads) {
    const int i = o / width, cc = o % width;
    const int64_t ch = (int64_t)(blockIdx.x % groups) * width + cc;
    if (ch >= p.D) continue;
    float s = 0.f;
    for (uint32_t q = 0; q < subs; ++q) s += sums[q * lanes + cc / V][i * V + cc % V];
    p.part[((int64_t)row * (W + 1) + i) * p.D + ch] = s;
  }
}

struct BwdGrid {
  uint32_t lanes, groups;
  int64_t rows;
};
BwdGrid bwd_grid(int64_t ntok, int64_t D) {
  const int64_t pieces = (D + kBwdV - 1) / kBwdV;
  uint32_t lanes = 1;
  while (lanes < 64 && lanes < pieces) lanes *= 2;
  const int64_t per = (int64_t)(kThreads / lanes) * kBwdTokens;
  return BwdGrid{lanes, (uint32_t)((pieces + lanes - 1) / lanes), (ntok + per - 1) / per};
}

// Stretches of 16 tokens, or of 4 where those would leave most of the card idle.  With
// ordinary stores, 16: 96 us for 16384 tokens x 6144 channels of bf16, 35 for 20011 x
// 2048; 8: 100 and 38; 32: 96 and 42.  On both sides of the line, us of a call with
// stretches of 4 / of 16 (of 512, 2048 and 8192 channels alike to a tenth; here 2048):
//   threads, parts of the line     1/8        1/4        1/2          1          2          4
//   bf16                       6.4/12.2   8.1/12.7  16.4/18.6  26.7/25.9  47.4/40.2  89.7/60.6
//   fp32                       6.1/12.6   7.3/13.3  12.8/19.2  20.8/26.5  34.9/38.2  61.5/57.3
// (fp32, whose pieces are half as many channels, crosses at two to four times the line)
constexpr int64_t kFillThreads = 256 * 4 * 64 * 2;

int64_t forward_threads(int64_t ntok, int64_t D, int64_t V) { return (ntok + 15) / 16 * ((D + V - 1) / V); }

template <typename T, int W, int TT, bool SILU, bool NT>
hipError_t forward_run(const ConvParams& p, hipStream_t stream) {
  const int64_t pieces = (p.D + kPiece<T> - 1) / kPiece<T>, count = (p.map.ntok + TT - 1) / TT * pieces;
  const uint32_t wgs = (uint32_t)((count + kThreads - 1) / kThreads);
  const uint32_t extra = (p.map.seq || p.cu) && p.state_fin ? kEmptyWgs : 0;
  hipLaunchKernelGGL((conv_fwd_kernel<T, W, TT, SILU, NT>), dim3(wgs + extra), dim3(kThreads), 0, stream, p,
                     (uint32_t)pieces, (uint32_t)count, wgs);
  return hipGetLastError();
}
template <typename T, int W, bool SILU> hipError_t forward_sized(const ConvParams& p, hipStream_t stream) {
  const bool small = forward_threads(p.map.ntok, p.D, kPiece<T>) < kFillThreads;
  if (small) return forward_run<T, W, 4, SILU, false>(p, stream);
  return p.map.ntok * p.D * (int64_t)sizeof(T) > kNtBytes ? forward_run<T, W, 16, SILU, true>(p, stream)
                                                          : forward_run<T, W, 16, SILU, false>(p, stream);
}
template <typename T, int W> hipError_t forward(const ConvParams& p, hipStream_t stream) {
  return p.silu ? forward_sized<T, W, true>(p, stream) : forward_sized<T, W, false>(p, stream);
}

template <typename T, int W> hipError_t decode(const ConvParams& p, hipStream_t stream) {
  const int64_t pieces = (p.D + kPiece<T> - 1) / kPiece<T>, count = pieces * p.map.nseq;
  const dim3 grid((uint32_t)((count + kThreads - 1) / kThreads));
  if (p.silu)
    hipLaunchKernelGGL((conv_decode_kernel<T, W, true>), grid, dim3(kThreads), 0, stream, p, (uint32_t)pieces, (uint32_t)count);
  else
    hipLaunchKernelGGL((conv_decode_kernel<T, W, false>), grid, dim3(kThreads), 0, stream, p, (uint32_t)pieces, (uint32_t)count);
  return hipGetLastError();
}

template <typename T, int W, bool SILU> hipError_t backward_sized(const ConvParams& p, hipStream_t stream) {
  const BwdGrid g = bwd_grid(p.map.ntok, p.D);
  const int64_t wgs = g.rows * g.groups;
  const dim3 grid((uint32_t)wgs + ((p.map.seq || p.cu) && p.dstate0 ? kEmptyWgs : 0));
  if (p.map.ntok * p.D * (int64_t)sizeof(T) > kNtBytes)
    hipLaunchKernelGGL((conv_bwd_kernel<T, W, SILU, true>), grid, dim3(kThreads), 0, stream, p, g.lanes, g.groups, (uint32_t)wgs);
  else
    hipLaunchKernelGGL((conv_bwd_kernel<T, W, SILU, false>), grid, dim3(kThreads), 0, stream, p, g.lanes, g.groups, (uint32_t)wgs);
  return hipGetLastError();
}
template <typename T, int W> hipError_t backward(const ConvParams& p, hipStream_t stream) {
  return p.silu ? backward_sized<T, W, true>(p, stream) : backward_sized<T, W, false>(p, stream);
}

#define RLA_CONV_DISPATCH(fn)                                                          \
  if (bf16)                                                                            \
    return p.taps == 2 ? fn<u16, 2>(p, stream) : p.taps == 3 ? fn<u16, 3>(p, stream)   \
                                                             : fn<u16, 4>(p, stream);  \
  return p.taps == 2 ? fn<float, 2>(p, stream) : p.taps == 3 ? fn<float, 3>(p, stream) \
                                                             : fn<float, 4>(p, stream)

hipError_t dispatch_backward(const ConvParams& p, bool bf16, hipStream_t stream) { RLA_CONV_DISPATCH(backward); }

}  // namespace

hipError_t launch_conv_forward(const ConvParams& p, bool bf16, hipStream_t stream) { RLA_CONV_DISPATCH(forward); }
hipError_t launch_conv_decode(const ConvParams& p, bool bf16, hipStream_t stream) { RLA_CONV_DISPATCH(decode); }

int64_t conv_backward_rows(int64_t ntok, int64_t D) { return bwd_grid(ntok, D).rows; }

// (with a workgroup to spare for the last threads, and those of empty sequences)
bool conv_forward_fits(const ConvParams& p, bool bf16) {
  return forward_threads(p.map.ntok, p.D, bf16 ? 8 : 4) <= (kMaxWgs - 1 - kEmptyWgs) * kThreads;
}
bool conv_backward_fits(const ConvParams& p) {
  const BwdGrid g = bwd_grid(p.map.ntok, p.D);
  return g.rows * g.groups <= kMaxWgs - kEmptyWgs;
}
bool conv_decode_fits(const ConvParams& p, bool bf16) {
  const int64_t V = bf16 ? 8 : 4;
  return (p.D + V - 1) / V * p.map.nseq <= (kMaxWgs - 1) * kThreads;
}

hipError_t launch_conv_backward(const ConvParams& p, bool bf16, float* dweight, float* dbias, hipStream_t stream) {
  if (p.map.ntok > 0) {
    const hipError_t e = dispatch_backward(p, bf16, stream);
    if (e != hipSuccess) return e;
  }
  return launch_column_sums(p.part, conv_backward_rows(p.map.ntok, p.D), (int64_t)(p.taps + 1) * p.D, p.D, p.taps,
                            dweight, dbias, stream);
}

}  // namespace rla

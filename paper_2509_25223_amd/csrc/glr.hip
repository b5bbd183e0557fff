// Gated linear recurrence, one state a channel:
//   a_t = exp(A sigmoid(r_t)),  b_t = m_t sigmoid(i_t) x_t,  m_t = sqrt(1 - a_t^2) or 1
//   h_t = a_t h_{t-1} + b_t,    o_t = h_t or h_t SiLU(z_t)
// and, with g_t = dO_t SiLU(z_t) and l_t = g_t + a_{t+1} l_{t+1} (the last token of a
// sequence: g_t + dh_final), its gradients
//   dx = l m s_i,  di = l m x s_i (1 - s_i),  dz = dO h SiLU'(z),  dh_init = a_1 l_1
//   d(log a) = l h_{t-1} a - l s_i x a^2 / m,  dr = d(log a) A s_r (1 - s_r),  dA = sum d(log a) s_r
//
// Two tokens' steps are one, (a2, b2) (a1, b1) = (a2 a1, a2 b1 + b2), so a stretch of tokens is
// a pair (P, S): h behind it is P h + S.  A workgroup takes 64 channels (128 bytes of
// bf16: whole lines of the caches) of a chunk of tokens, a tile at a time: a thread 4
// channels of kTok tokens in registers, the stretches of a wave (4) by exchanges between lanes,
// those of the workgroup's waves one after the other in LDS, where the state is carried from
// tile to tile.  Then each thread goes through its tokens from the state before
// them.  Everything is read once and written once.  The backward goes through the tiles
// from the last one; it takes h anew from the state before each tile, which the forward
// kept (or which is computed again), and carries l the other way.
// Sequences lie side by side along one axis of tokens, dense ones too: where one
// starts, the state is its own, whatever came before (never a factor 0: NaN and
// infinities of a sequence stay there).  Few channels: the tokens are cut into chunks, and a pass
// before leaves each chunk's pair.
#include "model.hpp"

namespace rla {

namespace {

constexpr int kGlrThreads = 512, kGlrWaves = kGlrThreads / 64, kV = 4;
constexpr int kLanes = kGlrChannels / kV;        // of a token's row: 16
constexpr int kSegs = kGlrThreads / kLanes;      // stretches of a tile
constexpr int kTok = 4;                          // tokens of a stretch
constexpr int kGlrTile = kSegs * kTok;           // 128

// A stretch of tokens: (P, S), P = -1 where a sequence starts in it (then S alone is the state
// behind it).
struct Step {
  float P, S;
};
__device__ __forceinline__ float apply(const Step& s, float h) { return s.P < 0.f ? s.S : __builtin_fmaf(s.P, h, s.S); }
// first a, then b
__device__ __forceinline__ Step join(const Step& a, const Step& b) {
  return Step{a.P < 0.f || b.P < 0.f ? -1.f : a.P * b.P, apply(b, a.S)};
}

__device__ __forceinline__ float sigmoid_of(float x, float& rest) {   // and 1 - sigmoid, with its digits
  const float e = __expf(-x), s = __builtin_amdgcn_rcpf(1.f + e);
  rest = e < 3e38f ? e * s : 1.f;
  return s;
}

// 1 - e^y for y <= 0: near 0 by the series
__device__ __forceinline__ float one_minus_exp(float y, float ey) {
  float p = 1.f / 40320.f;
  p = __builtin_fmaf(p, y, 1.f / 5040.f);
  p = __builtin_fmaf(p, y, 1.f / 720.f);
  p = __builtin_fmaf(p, y, 1.f / 120.f);
  p = __builtin_fmaf(p, y, 1.f / 24.f);
  p = __builtin_fmaf(p, y, 1.f / 6.f);
  p = __builtin_fmaf(p, y, 0.5f);
  p = __builtin_fmaf(p, y, 1.f);
  return y > -0.5f ? -y * p : 1.f - ey;
}

// a and m of a token from its gate's sigmoid
__device__ __forceinline__ void decay(float A, float sr, bool norm, float& a, float& m) {
  const float l = A * sr;
  a = __expf(l);
  m = norm ? __builtin_amdgcn_sqrtf(fmaxf(one_minus_exp(2.f * l, a * a), 0.f)) : 1.f;
}

// Where a thread's tokens lie: bits of the tokens t .. t + kTok.
struct Place {
  uint32_t in = 0;       // of a sequence (and of this chunk)
  uint32_t starts = 0;   // first of a sequence, or of a gap
  int32_t seq[kTok];
};
__device__ __forceinline__ Place place_of(const GlrParams& p, int64_t t, int64_t end) {
  Place q;
  const int64_t left = end - t;
  const uint32_t there = left >= kTok ? (1u << kTok) - 1u : left > 0 ? (1u << left) - 1u : 0u;
  if (!there) {
#pragma unroll
    for (int k = 0; k < kTok; ++k) q.seq[k] = -1;
    return q;
  }
  // (bit kTok too: whether the last token ends its sequence; past the last of all they are set)
  q.starts = p.map.start_bits(t) & ((there << 1) | 1u);
  q.in = there;
  if (p.map.seq) {
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      q.seq[k] = (there >> k) & 1u ? p.map.seq[t + k] : -1;
      if (q.seq[k] < 0) q.in &= ~(1u << k);
    }
  } else {
    const int32_t n = (int32_t)((uint32_t)t / (uint32_t)p.map.T);
    q.seq[0] = n;
#pragma unroll
    for (int k = 1; k < kTok; ++k) q.seq[k] = q.seq[k - 1] + ((q.starts >> k) & 1u);
  }
  return q;
}

template <typename T, bool FULL>
__device__ __forceinline__ void load4(const void* base, int64_t stride, int64_t t, int64_t c, int left, bool there, float (&x)[kV]) {
  if (there) load_piece<T, kV, FULL>(reinterpret_cast<const T*>(base) + t * stride + c, left, x);
  else
#pragma unroll
    for (int e = 0; e < kV; ++e) x[e] = 0.f;
}

// What a workgroup's waves share: each wave's pair per channel, and the state before it.
struct GlrLds {
  Step wave[kGlrWaves][kGlrChannels];
  float before[kGlrWaves][kGlrChannels];
};

// The state before the thread's stretch, from the stretches' pairs and the state before the
// tile.  FORWARD: stretches in order, else from the last one.  `carry` and `pair` are those of channel
// threadIdx.x (the first 64 threads'): the state, or the pair of everything so far.
template <bool FORWARD>
__device__ __forceinline__ void state_before(const Step (&own)[kV], GlrLds& s, float& carry, Step& pair, float (&h)[kV]) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, l = lane % kLanes, seg = lane / kLanes;
  Step incl[kV], excl[kV];
#pragma unroll
  for (int e = 0; e < kV; ++e) {
    incl[e] = own[e];
#pragma unroll
    for (int d = kLanes; d < 64; d <<= 1) {
      Step o;
      o.P = FORWARD ? __shfl_up(incl[e].P, d) : __shfl_down(incl[e].P, d);
      o.S = FORWARD ? __shfl_up(incl[e].S, d) : __shfl_down(incl[e].S, d);
      if (FORWARD ? lane >= d : lane + d < 64) incl[e] = join(o, incl[e]);
    }
    excl[e].P = FORWARD ? __shfl_up(incl[e].P, kLanes) : __shfl_down(incl[e].P, kLanes);
    excl[e].S = FORWARD ? __shfl_up(incl[e].S, kLanes) : __shfl_down(incl[e].S, kLanes);
  }
  const bool outer = FORWARD ? seg == 64 / kLanes - 1 : seg == 0, first = FORWARD ? seg == 0 : seg == 64 / kLanes - 1;
  if (outer)
#pragma unroll
    for (int e = 0; e < kV; ++e) s.wave[w][l * kV + e] = incl[e];
  __syncthreads();
  if (threadIdx.x < kGlrChannels) {
#pragma unroll
    for (int v = 0; v < kGlrWaves; ++v) {
      const int u = FORWARD ? v : kGlrWaves - 1 - v;
      const Step x = s.wave[u][threadIdx.x];
      s.before[u][threadIdx.x] = carry;
      carry = apply(x, carry);
      pair = join(pair, x);
    }
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kV; ++e) {
    h[e] = s.before[w][l * kV + e];
    if (!first) h[e] = apply(excl[e], h[e]);
  }
}

// Channel threadIdx.x of the first 64 threads: the state before chunk c, from the pairs
// of the chunks before it (FORWARD) or behind it.
template <bool FORWARD> __device__ __forceinline__ float chunk_state(const GlrParams& p, int c, int64_t channel) {
  float h = 0.f;
  if (p.apart || channel >= p.D) return h;
  for (int k = FORWARD ? 0 : p.nchunk - 1; k != c; k += FORWARD ? 1 : -1) {
    const float* at = p.sum + ((int64_t)k * 2) * p.D + channel;
    h = apply(Step{at[0], at[p.D]}, h);
  }
  return h;
}

// the thread's channels of a state row, zeros without one
template <bool FULL>
__device__ __forceinline__ void load_state(const float* state, int32_t n, int64_t D, int64_t c, int left, float (&h)[kV]) {
  if (state && n >= 0) load_piece<float, kV, FULL>(state + (int64_t)n * D + c, left, h);
  else
#pragma unroll
    for (int e = 0; e < kV; ++e) h[e] = 0.f;
}

// The thread's tokens as a, b; tokens outside every sequence have b = 0.
template <typename T, bool HAS_I, bool FULL>
__device__ __forceinline__ void load_steps(const GlrParams& p, const Place& q, int64_t t, int64_t c, int left, const float (&A)[kV],
                                           float (&a)[kTok][kV], float (&b)[kTok][kV]) {
#pragma unroll
  for (int k = 0; k < kTok; ++k) {
    const bool in = (q.in >> k) & 1u;
    float x[kV], r[kV], i[kV];
    load4<T, FULL>(p.x, p.xs, t + k, c, left, in, x);
    load4<T, FULL>(p.r, p.rs, t + k, c, left, in, r);
    if (HAS_I) load4<T, FULL>(p.i, p.is, t + k, c, left, in, i);
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      float m;
      decay(A[e], sigmoid_fast(r[e]), p.normalize, a[k][e], m);
      b[k][e] = m * x[e];
      if (HAS_I) b[k][e] *= sigmoid_fast(i[e]);
      if (!in) a[k][e] = 1.f, b[k][e] = 0.f;
    }
  }
}

// The stretch's pair.
template <bool FULL>
__device__ __forceinline__ void steps_pair(const GlrParams& p, const Place& q, int64_t c, int left, const float (&a)[kTok][kV],
                                           const float (&b)[kTok][kV], Step (&own)[kV]) {
#pragma unroll
  for (int e = 0; e < kV; ++e) own[e] = Step{1.f, 0.f};
#pragma unroll
  for (int k = 0; k < kTok; ++k) {
    if ((q.starts >> k) & 1u) {
      float h[kV];
      load_state<FULL>(p.h0, q.seq[k], p.D, c, left, h);
#pragma unroll
      for (int e = 0; e < kV; ++e) own[e] = Step{-1.f, h[e]};
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      own[e].P = own[e].P < 0.f ? -1.f : own[e].P * a[k][e];
      own[e].S = __builtin_fmaf(a[k][e], own[e].S, b[k][e]);
    }
  }
}

// ---------------------------------------------------------------------------
// forward.  blockIdx.x: block of channels, fastest, then chunk; behind them workgroups that copy the
// states of sequences without tokens.  SUMMARY: the chunk's pair only.
// ---------------------------------------------------------------------------
constexpr uint32_t kGlrEmptyWgs = 16;
__device__ __forceinline__ void copy_empty(const GlrParams& p, const float* from, float* to, uint32_t wg) {
  for (int64_t n = wg; n < p.map.nseq; n += kGlrEmptyWgs) {
    if (!p.map.empty[n]) continue;
    for (int64_t c = threadIdx.x; c < p.D; c += kGlrThreads) to[n * p.D + c] = from ? from[n * p.D + c] : 0.f;
  }
}

template <typename T, bool HAS_I, bool HAS_Z, bool SUMMARY, bool FULL>
__global__ __launch_bounds__(kGlrThreads) void glr_fwd_kernel(GlrParams p, uint32_t blocks, int save) {
  __shared__ GlrLds lds;
  const uint32_t chunk = blockIdx.x / blocks;
  if (chunk >= (uint32_t)p.nchunk) {
    copy_empty(p, p.h0, p.hfin, blockIdx.x - p.nchunk * blocks);
    return;
  }
  const int64_t block = (int64_t)(blockIdx.x - chunk * blocks) * kGlrChannels;
  const int64_t c = block + (threadIdx.x % kLanes) * kV, own_channel = block + threadIdx.x;
  const int left = (int)min(p.D - c, (int64_t)kV);
  const int64_t t0 = chunk * p.L, end = min(t0 + p.L, p.map.ntok);
  float A[kV];
  if (left > 0) load_piece<float, kV, FULL>(p.A + c, left, A);
  float carry = SUMMARY || threadIdx.x >= kGlrChannels ? 0.f : chunk_state<true>(p, (int)chunk, own_channel);
  Step pair{1.f, 0.f};
  for (int tile = 0; t0 + (int64_t)tile * kGlrTile < end; ++tile) {
    const int64_t t = t0 + (int64_t)tile * kGlrTile + (threadIdx.x / kLanes) * kTok;
    if (save && !SUMMARY && threadIdx.x < kGlrChannels && own_channel < p.D)
      p.ck[((int64_t)chunk * p.tiles + tile) * p.D + own_channel] = carry;
    Place q = place_of(p, left > 0 ? t : end, end);
    float a[kTok][kV], b[kTok][kV], h[kV];
    Step own[kV];
    load_steps<T, HAS_I, FULL>(p, q, t, c, left, A, a, b);
    steps_pair<FULL>(p, q, c, left, a, b, own);
    state_before<true>(own, lds, carry, pair, h);
    if (SUMMARY) continue;
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      if (t + k >= end || left <= 0) break;
      if ((q.starts >> k) & 1u) load_state<FULL>(p.h0, q.seq[k], p.D, c, left, h);
      const bool in = (q.in >> k) & 1u;
      float o[kV], z[kV];
      if (HAS_Z) load4<T, FULL>(p.z, p.zs, t + k, c, left, in, z);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        h[e] = __builtin_fmaf(a[k][e], h[e], b[k][e]);
        o[e] = HAS_Z ? h[e] * z[e] * sigmoid_fast(z[e]) : h[e];
        if (!in) o[e] = 0.f;
      }
      if (p.o) store_piece<T, kV, FULL>(reinterpret_cast<T*>(p.o) + (t + k) * p.D + c, left, o);
      if (p.hfin && in && ((q.starts >> (k + 1)) & 1u))
        store_piece<float, kV, FULL>(p.hfin + (int64_t)q.seq[k] * p.D + c, left, h);
    }
  }
  if (SUMMARY && threadIdx.x < kGlrChannels && own_channel < p.D) {
    float* at = p.sum + (int64_t)chunk * 2 * p.D + own_channel;
    at[0] = pair.P;
    at[p.D] = pair.S;
  }
}

// ---------------------------------------------------------------------------
// backward.  The message from a token to the one before it is u_t = a_t l_t, l_t = g_t + u_{t+1};
// a sequence's last token gets dh_final, its first one's message is dh_init.
// ---------------------------------------------------------------------------
template <typename T, bool HAS_I, bool HAS_Z, bool SUMMARY, bool FULL>
__global__ __launch_bounds__(kGlrThreads) void glr_bwd_kernel(GlrParams p, uint32_t blocks) {
  __shared__ GlrLds lds;
  const uint32_t chunk = blockIdx.x / blocks;
  if (chunk >= (uint32_t)p.nchunk) {
    copy_empty(p, p.dhfin, p.dh0, blockIdx.x - p.nchunk * blocks);
    return;
  }
  const int64_t block = (int64_t)(blockIdx.x - chunk * blocks) * kGlrChannels;
  const int64_t c = block + (threadIdx.x % kLanes) * kV, own_channel = block + threadIdx.x;
  const int left = (int)min(p.D - c, (int64_t)kV);
  const int64_t t0 = chunk * p.L, end = min(t0 + p.L, p.map.ntok);
  float A[kV], dA[kV] = {0.f, 0.f, 0.f, 0.f};
  if (left > 0) load_piece<float, kV, FULL>(p.A + c, left, A);
  float carry = SUMMARY || threadIdx.x >= kGlrChannels ? 0.f : chunk_state<false>(p, (int)chunk, own_channel);
  Step pair{1.f, 0.f};
  for (int tile = (int)((end - t0 + kGlrTile - 1) / kGlrTile) - 1; tile >= 0; --tile) {
    const int64_t t = t0 + (int64_t)tile * kGlrTile + (threadIdx.x / kLanes) * kTok;
    Place q = place_of(p, left > 0 ? t : end, end);
    const uint32_t ends = q.starts >> 1;   // last of a sequence
    float a[kTok][kV], b[kTok][kV], h[kV], before[kTok][kV];
    Step own[kV];
    load_steps<T, HAS_I, FULL>(p, q, t, c, left, A, a, b);
    if (!SUMMARY) {
      float state = 0.f;
      Step none{1.f, 0.f};
      if (threadIdx.x < kGlrChannels && own_channel < p.D) state = p.ck[((int64_t)chunk * p.tiles + tile) * p.D + own_channel];
      steps_pair<FULL>(p, q, c, left, a, b, own);
      state_before<true>(own, lds, state, none, h);
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        if ((q.starts >> k) & 1u) load_state<FULL>(p.h0, q.seq[k], p.D, c, left, h);
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          before[k][e] = h[e];
          h[e] = __builtin_fmaf(a[k][e], h[e], b[k][e]);
        }
      }
    }
    // g, and the messages' pairs from the last token on
    float g[kTok][kV];
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      const bool in = (q.in >> k) & 1u;
      float z[kV];
      load4<T, FULL>(p.dO, p.dos, t + k, c, left, in, g[k]);
      if (HAS_Z) {
        load4<T, FULL>(p.z, p.zs, t + k, c, left, in, z);
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float d = g[k][e];
          float silu;
          const float slope = silu_grad_f(z[e], silu);
          g[k][e] = d * silu;
          if (!SUMMARY) z[e] = in ? d * __builtin_fmaf(a[k][e], before[k][e], b[k][e]) * slope : 0.f;
        }
        if (!SUMMARY && t + k < end && left > 0)
          store_piece<T, kV, FULL>(reinterpret_cast<T*>(p.dz) + (t + k) * p.D + c, left, z);
      }
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) own[e] = Step{1.f, 0.f};
#pragma unroll
    for (int k = kTok - 1; k >= 0; --k) {
      if ((ends >> k) & 1u) {
        float d[kV];
        load_state<FULL>(p.dhfin, q.seq[k], p.D, c, left, d);
#pragma unroll
        for (int e = 0; e < kV; ++e) own[e] = Step{-1.f, d[e]};
      }
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        own[e].P = own[e].P < 0.f ? -1.f : own[e].P * a[k][e];
        own[e].S = a[k][e] * (own[e].S + g[k][e]);
      }
    }
    float u[kV];
    state_before<false>(own, lds, carry, pair, u);
    if (SUMMARY) continue;
#pragma unroll
    for (int k = kTok - 1; k >= 0; --k) {
      if (t + k >= end || left <= 0) continue;
      const bool in = (q.in >> k) & 1u;
      if ((ends >> k) & 1u) load_state<FULL>(p.dhfin, q.seq[k], p.D, c, left, u);
      float x[kV], r[kV], i[kV];
      load4<T, FULL>(p.x, p.xs, t + k, c, left, in, x);
      load4<T, FULL>(p.r, p.rs, t + k, c, left, in, r);
      if (HAS_I) load4<T, FULL>(p.i, p.is, t + k, c, left, in, i);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        float rest_r, rest_i = 0.f, si = 1.f, a1, m;
        const float sr = sigmoid_of(r[e], rest_r);
        if (HAS_I) si = sigmoid_of(i[e], rest_i);
        decay(A[e], sr, p.normalize, a1, m);
        const float l = g[k][e] + u[e], lm = l * m * si;
        float dlog = l * before[k][e] * a1;
        if (p.normalize && m > 0.f) dlog -= l * si * x[e] * (a1 * a1) * __builtin_amdgcn_rcpf(m);
        i[e] = in ? lm * x[e] * rest_i : 0.f;
        x[e] = in ? lm : 0.f;
        r[e] = in ? dlog * (A[e] * sr) * rest_r : 0.f;
        dA[e] += in ? dlog * sr : 0.f;
        u[e] = a[k][e] * l;
      }
      store_piece<T, kV, FULL>(reinterpret_cast<T*>(p.dx) + (t + k) * p.D + c, left, x);
      store_piece<T, kV, FULL>(reinterpret_cast<T*>(p.dr) + (t + k) * p.D + c, left, r);
      if (HAS_I) store_piece<T, kV, FULL>(reinterpret_cast<T*>(p.di) + (t + k) * p.D + c, left, i);
      if (p.dh0 && in && (q.starts >> k) & 1u) store_piece<float, kV, FULL>(p.dh0 + (int64_t)q.seq[k] * p.D + c, left, u);
    }
  }
  if (SUMMARY) {
    if (threadIdx.x < kGlrChannels && own_channel < p.D) {
      float* at = p.sum + (int64_t)chunk * 2 * p.D + own_channel;
      at[0] = pair.P;
      at[p.D] = pair.S;
    }
    return;
  }
  // dA over the workgroup's stretches
#pragma unroll
  for (int e = 0; e < kV; ++e)
#pragma unroll
    for (int d = kLanes; d < 64; d <<= 1) dA[e] += __shfl_xor(dA[e], d);
  if ((threadIdx.x & 63) < kLanes)
#pragma unroll
    for (int e = 0; e < kV; ++e) lds.before[threadIdx.x >> 6][(threadIdx.x % kLanes) * kV + e] = dA[e];
  __syncthreads();
  if (threadIdx.x < kGlrChannels && own_channel < p.D) {
    float sum = 0.f;
    for (int w = 0; w < kGlrWaves; ++w) sum += lds.before[w][threadIdx.x];
    p.pA[(int64_t)chunk * p.D + own_channel] = sum;
  }
}

// Single tokens: a thread owns 4 channels of a sequence, whose state it reads before it
// writes (in place works).
template <typename T, bool HAS_I, bool HAS_Z, bool FULL>
__global__ __launch_bounds__(kThreads) void glr_decode_kernel(GlrParams p, uint32_t pieces, uint32_t count) {
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  if (id >= count) return;
  const int64_t n = id / pieces, c = (int64_t)(id % pieces) * kV;
  const int left = (int)min(p.D - c, (int64_t)kV);
  float A[kV], h[kV];
  load_piece<float, kV, FULL>(p.A + c, left, A);
  load_state<FULL>(p.h0, (int32_t)n, p.D, c, left, h);
  for (int64_t k = 0; k < p.map.T; ++k) {
    const int64_t t = n * p.map.T + k;
    float x[kV], r[kV], i[kV], z[kV];
    load4<T, FULL>(p.x, p.xs, t, c, left, true, x);
    load4<T, FULL>(p.r, p.rs, t, c, left, true, r);
    if (HAS_I) load4<T, FULL>(p.i, p.is, t, c, left, true, i);
    if (HAS_Z) load4<T, FULL>(p.z, p.zs, t, c, left, true, z);
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      float a, m;
      decay(A[e], sigmoid_fast(r[e]), p.normalize, a, m);
      float b = m * x[e];
      if (HAS_I) b *= sigmoid_fast(i[e]);
      h[e] = __builtin_fmaf(a, h[e], b);
      x[e] = HAS_Z ? h[e] * z[e] * sigmoid_fast(z[e]) : h[e];
    }
    store_piece<T, kV, FULL>(reinterpret_cast<T*>(p.o) + t * p.D + c, left, x);
  }
  store_piece<float, kV, FULL>(p.hfin + n * p.D + c, left, h);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
uint32_t blocks_of(const GlrParams& p) { return (uint32_t)((p.D + kGlrChannels - 1) / kGlrChannels); }

template <typename F> hipError_t with(bool bf16, bool i, bool z, bool full, F f) {
  auto types = [&](auto T) {
    auto gates = [&](auto I) {
      auto out = [&](auto Z) {
        if (full) f(T, I, Z, std::true_type());
        else f(T, I, Z, std::false_type());
      };
      if (z) out(std::true_type());
      else out(std::false_type());
    };
    if (i) gates(std::true_type());
    else gates(std::false_type());
  };
  if (bf16) types(u16());
  else types(float());
  return hipGetLastError();
}

}  // namespace

void glr_plan(GlrParams& p, bool packed) {
  const int64_t blocks = blocks_of(p), ntok = p.map.ntok;
  constexpr int64_t fill = 512;   // workgroups that fill the card
  int64_t want = max((int64_t)1, fill / blocks);
  p.apart = 0;
  if (!packed && p.map.nseq >= want) {   // whole sequences
    const int64_t T = max(p.map.T, (int64_t)1), each = max(p.map.nseq / want, (kGlrTile + T - 1) / T);
    p.L = each * p.map.T;
    p.apart = 1;
  } else {
    want = min(want, (ntok + kGlrTile - 1) / kGlrTile);
    p.L = ((ntok + max(want, (int64_t)1) - 1) / max(want, (int64_t)1) + kGlrTile - 1) / kGlrTile * kGlrTile;
  }
  if (p.L < 1) p.L = kGlrTile;
  const int64_t n = (ntok + p.L - 1) / p.L;
  p.nchunk = (int32_t)n;
  p.tiles = (int32_t)((p.L + kGlrTile - 1) / kGlrTile);
  if (n <= 1) p.apart = 1;
}

int64_t glr_decode_wgs(const GlrParams& p) { return ((p.D + kV - 1) / kV * p.map.nseq + kThreads - 1) / kThreads; }

hipError_t launch_glr_forward(const GlrParams& p, bool bf16, bool save, bool outputs, hipStream_t stream) {
  const uint32_t blocks = blocks_of(p), main = blocks * p.nchunk;
  hipError_t e = hipSuccess;
  if (!p.apart) {
    e = with(bf16, p.i, false, p.D % kV == 0, [&](auto T, auto I, auto Z, auto F) {
      hipLaunchKernelGGL((glr_fwd_kernel<decltype(T), I.value, Z.value, true, F.value>), dim3(main), dim3(kGlrThreads), 0, stream, p,
                         blocks, 0);
    });
    if (e != hipSuccess) return e;
  }
  GlrParams q = p;
  if (!outputs) q.o = nullptr, q.hfin = nullptr;
  const uint32_t extra = p.map.seq && q.hfin ? kGlrEmptyWgs : 0;
  return with(bf16, p.i, p.z && outputs, p.D % kV == 0, [&](auto T, auto I, auto Z, auto F) {
    hipLaunchKernelGGL((glr_fwd_kernel<decltype(T), I.value, Z.value, false, F.value>), dim3(main + extra), dim3(kGlrThreads), 0,
                       stream, q, blocks, save ? 1 : 0);
  });
}

hipError_t launch_glr_backward(const GlrParams& p, bool bf16, hipStream_t stream) {
  const uint32_t blocks = blocks_of(p), main = blocks * p.nchunk, extra = p.map.seq && p.dh0 ? kGlrEmptyWgs : 0;
  if (!p.apart) {
    const hipError_t e = with(bf16, p.i, p.z, p.D % kV == 0, [&](auto T, auto I, auto Z, auto F) {
      hipLaunchKernelGGL((glr_bwd_kernel<decltype(T), I.value, Z.value, true, F.value>), dim3(main), dim3(kGlrThreads), 0, stream, p,
                         blocks);
    });
    if (e != hipSuccess) return e;
  }
  return with(bf16, p.i, p.z, p.D % kV == 0, [&](auto T, auto I, auto Z, auto F) {
    hipLaunchKernelGGL((glr_bwd_kernel<decltype(T), I.value, Z.value, false, F.value>), dim3(main + extra), dim3(kGlrThreads), 0,
                       stream, p, blocks);
  });
}

hipError_t launch_glr_decode(const GlrParams& p, bool bf16, hipStream_t stream) {
  const uint32_t pieces = (uint32_t)((p.D + kV - 1) / kV), count = pieces * (uint32_t)p.map.nseq;
  return with(bf16, p.i, p.z, p.D % kV == 0, [&](auto T, auto I, auto Z, auto F) {
    hipLaunchKernelGGL((glr_decode_kernel<decltype(T), I.value, Z.value, F.value>), dim3((count + kThreads - 1) / kThreads),
                       dim3(kThreads), 0, stream, p, pieces, count);
  });
}

}  // namespace rla

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
// bf16: whole lines of the caches) of a chunk of tokens, a tile of 128 at a time: a thread 2
// channels of 8 tokens in registers, the two stretches of a wave by an exchange between its halves.  The
// 8 waves' pairs go to LDS, and after the tile's one barrier each wave goes through all of them
// for itself, so that none waits for another's state; the carried state is every wave's own.  Then
// each thread goes through its tokens from the state before them.  Everything is read once
// and written once.  The backward goes through the tiles from the last one; it takes h anew from the
// state before each tile, which the forward kept (or which is computed again), and carries l the
// other way.
// Sequences lie side by side along one axis of tokens, dense ones too: where one
// starts, the state is its own, whatever came before (never a factor 0: NaN and
// infinities of a sequence stay there).  Too few workgroups: the tokens are cut into chunks, and a
// pass before leaves each chunk's pair, at the price of reading x, r, i (backward: r, dO, z) twice.
//
// What bounds it: HBM and the vector ALU together.  bf16, both gates, normalized, 4 x 4096 x 4096: forward 168 to
// 184 us from card to card (671 MB, 3.6 to 4.0 TB/s; vector ALUs at work 54 % of the time), backward 280 to 296 (1.2 GB,
// 4.2 TB/s, 57 %).  Its 2 channels x 8 tokens x 6 values take 252 registers with both gates, two waves a SIMD; what they do
// not hold lies in LDS, each thread's own (96 KB).  fp32 with both gates spills 30 of them (116 bytes a lane), the bf16
// forward with both gates 2.  Measured there and not kept: 16 waves a workgroup and loads a tile further ahead (the same
// time), 16 tokens a stretch (spills), two workgroups a CU of 32 channels each, half lines (forward 205 us, backward 336).
// Loads behind branches, in turn waited for one by one, had cost three times as much (1283 us, now 455).
#include <math.h>

#include "model.hpp"

namespace rla {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kGlrThreads = 512, kGlrWaves = kGlrThreads / 64;
constexpr int kV = 2;                            // channels of a thread
constexpr int kLanes = kGlrChannels / kV;        // of a token's row: 32
constexpr int kSegs = kGlrThreads / kLanes;      // stretches of a tile: 16
constexpr int kTok = 8;                          // tokens of a stretch
constexpr int kTile = kSegs * kTok;              // 128

// A stretch of tokens: (P, S), P = -1 where a sequence starts in it (then S alone is the state
// behind it).
struct Step {
  float P, S;
};
__device__ __forceinline__ float apply(const Step& s, float h) {
  const float next = __builtin_fmaf(s.P, h, s.S);
  return s.P < 0.f ? s.S : next;
}
// first a, then b
__device__ __forceinline__ Step join(const Step& a, const Step& b) {
  const float both = a.P * b.P;
  return Step{fminf(a.P, b.P) < 0.f ? -1.f : both, apply(b, a.S)};
}

// e^l and m = sqrt(1 - e^2l) for l = ln 2 y <= 0: near 0 by the series (to y = -0.18, l = -1/8, off by
// less than a rounding), else as it stands (3.5 roundings of e^2l there)
constexpr float series(int n) {   // (2 ln 2)^n / n!
  double v = 1;
  for (int i = 1; i <= n; ++i) v *= 2 * 0.69314718055994530942 / i;
  return (float)v;
}
template <bool NORM> __device__ __forceinline__ void decay(float y, float& a, float& m) {
  a = __builtin_amdgcn_exp2f(y);
  m = 1.f;
  if (NORM) {
    float p = series(6);
    p = __builtin_fmaf(p, y, series(5));
    p = __builtin_fmaf(p, y, series(4));
    p = __builtin_fmaf(p, y, series(3));
    p = __builtin_fmaf(p, y, series(2));
    p = -y * __builtin_fmaf(p, y, series(1));
    float far = __builtin_fmaf(-a, a, 1.f);
    // (both computed, one selected: the compiler would branch around the series, value by value)
    asm volatile("" : "+v"(p), "+v"(far));
    m = __builtin_amdgcn_sqrtf(y > -0.18f ? p : far);
  }
}

// The channels of a thread, and of a workgroup's 64: the last block and the last piece of a
// row are moved back to its end, so that all are whole.  What lies in two of them is computed by
// both, to the same bits.  (WHOLE false: rows of a single channel.)
template <bool WHOLE> struct Channels {
  int64_t c;
  int left;
  __device__ __forceinline__ Channels(int64_t D, uint32_t b) {
    const int64_t block = WHOLE ? max(min((int64_t)b * kGlrChannels, D - kGlrChannels), (int64_t)0) : 0;
    c = block + (threadIdx.x % kLanes) * kV;
    if (WHOLE) c = min(c, D - kV);
    left = WHOLE ? kV : (int)max((int64_t)0, min(D - c, (int64_t)kV));
  }
  template <typename T> __device__ __forceinline__ void load(const T* row, float (&x)[kV]) const {
    load_piece<T, kV, WHOLE>(row + c, left, x);
  }
  template <typename T> __device__ __forceinline__ void store(T* row, const float (&x)[kV]) const {
    store_piece<T, kV, WHOLE>(row + c, left, x);
  }
  __device__ __forceinline__ void state(const float* rows, int32_t n, int64_t D, float (&h)[kV]) const {
    if (rows && n >= 0) load(rows + (int64_t)n * D, h);
    else
#pragma unroll
      for (int e = 0; e < kV; ++e) h[e] = 0.f;
  }
};

// Workgroups are dealt to the 8 XCDs in turn.  Each takes adjacent blocks of channels: the lines of a row
// lie in all channels of its L2, where every eighth block's would share two of them (16384 x 2048
// forward 139 us, before 147; 3001 x 514 of fp32 with gradients 45, before 49).
constexpr uint32_t kXcds = 8;
__device__ __forceinline__ uint32_t work_of(uint32_t wg, uint32_t count) {
  const uint32_t xcd = wg % kXcds, each = count / kXcds, more = count % kXcds;
  return xcd * each + min(xcd, more) + wg / kXcds;
}

// What a workgroup works on; blocks of channels vary fastest.
template <bool WHOLE> struct Work {
  uint32_t chunk;
  Channels<WHOLE> ch;
  int64_t t0, end, channel;   // (channel: the lane's own, of the states that waves carry)
  bool owner;                 // the first wave's lanes write what there is one of per channel
  __device__ __forceinline__ Work(const GlrParams& p, uint32_t blocks)
      : Work(p, blocks, work_of(blockIdx.x, blocks * p.nchunk)) {}
  __device__ __forceinline__ Work(const GlrParams& p, uint32_t blocks, uint32_t id)
      : chunk(id / blocks), ch(p.D, id - chunk * blocks) {
    t0 = chunk * p.L;
    end = min(t0 + p.L, p.map.ntok);
    channel = ch.c + (threadIdx.x & 63) / kLanes;
    owner = threadIdx.x < 64 && channel < p.D;
  }
  __device__ __forceinline__ int tiles() const { return (int)((end - t0 + kTile - 1) / kTile); }
};

// One tensor's rows of the thread's tokens, as stored: a tile's base and the rows' distance are the
// workgroup's, a thread adds an offset of 32 bits.  Past the chunk's end the last row again: loads
// without branches, all in flight at once.
template <typename T> struct Rows {
  typedef typename RowVec<T, kV>::type Vec;
  Vec v[kTok];
  template <bool WHOLE>
  __device__ __forceinline__ void load(const void* base, int64_t stride, int64_t tile, const Work<WHOLE>& w) {
    const char* row = reinterpret_cast<const char*>(reinterpret_cast<const T*>(base) + tile * stride);
    const uint32_t first = threadIdx.x / kLanes * kTok, step = (uint32_t)stride * (uint32_t)sizeof(T);
    const uint32_t col = (uint32_t)w.ch.c * (uint32_t)sizeof(T);
    if (tile + kTile <= w.end) {
      const uint32_t off = first * step + col;
#pragma unroll
      for (int k = 0; k < kTok; ++k) take<WHOLE>(row + (int64_t)k * step + off, w.ch.left, v[k]);
    } else {
      const uint32_t last = (uint32_t)(w.end - tile) - 1;
#pragma unroll
      for (int k = 0; k < kTok; ++k) take<WHOLE>(row + (min(first + k, last) * step + col), w.ch.left, v[k]);
    }
  }
  template <bool WHOLE> __device__ __forceinline__ static void take(const char* at, int left, Vec& x) {
    load_raw<T, kV, WHOLE>(reinterpret_cast<const T*>(at), left, x);
  }
  __device__ __forceinline__ float at(int k, int e) const { return to_f<T>(v[k][e]); }
  // rows of tokens that `in` does not have
  __device__ __forceinline__ void put(uint32_t in, float x) {
#pragma unroll
    for (int k = 0; k < kTok; ++k)
      if (!((in >> k) & 1u))
#pragma unroll
        for (int e = 0; e < kV; ++e) v[k][e] = from_f<T>(x);
  }
};
// ... written, of a tensor with rows next to each other
template <typename T, bool WHOLE>
__device__ __forceinline__ void store_row(const GlrParams& p, void* base, int64_t tile, int k, const Work<WHOLE>& w, const float (&x)[kV]) {
  const uint32_t off = (threadIdx.x / kLanes * kTok * (uint32_t)p.D + (uint32_t)w.ch.c) * (uint32_t)sizeof(T);
  char* row = reinterpret_cast<char*>(reinterpret_cast<T*>(base) + (tile + k) * p.D);
  store_piece<T, kV, WHOLE>(reinterpret_cast<T*>(row + off), w.ch.left, x);
}

// Whether no sequence starts in the tile or right behind it, and all of it is of one, in this
// chunk: then no token needs a look at where it lies.  The same for the whole workgroup.
__device__ __forceinline__ bool plain_tile(const GlrParams& p, int64_t tile, int64_t end) {
  if (tile + kTile > end) return false;
  if (!p.map.seq) {
    const uint32_t r = (uint32_t)tile % (uint32_t)p.map.T;
    return r > 0 && r + kTile < (uint32_t)p.map.T;
  }
  uint32_t bits = p.map.start_bits(tile + kTile) & 1u;
#pragma unroll
  for (int i = 0; i < kTile / 32; ++i) bits |= p.map.start_bits(tile + 32 * i);
  return bits == 0 && p.map.seq_of(tile) >= 0;
}

// Where a thread's tokens lie.  Bit k: token t + k ...
struct Place {
  int64_t t;
  uint32_t in = (1u << kTok) - 1u;   // is of a sequence (and of this chunk)
  uint32_t there = in;               // is of this chunk
  uint32_t starts = 0;               // is the first of a sequence, or of a gap
  uint32_t ends = 0;                 // is the last one of it
  __device__ __forceinline__ Place(const GlrParams& p, int64_t t_, int64_t end, bool plain) : t(t_) {
    if (plain) return;
    const int64_t left = end - t;
    there = left >= kTok ? there : left > 0 ? (1u << left) - 1u : 0u;
    in = there;
    if (!there) return;
    const uint32_t bits = p.map.start_bits(t);   // (past the last token of all they are set)
    starts = bits & there;
    ends = (bits >> 1) & there;
    if (p.map.seq) {
#pragma unroll
      for (int k = 0; k < kTok; ++k)
        if (p.map.seq[min(t + k, end - 1)] < 0) in &= ~(1u << k);
    }
  }
  __device__ __forceinline__ int32_t seq(const GlrParams& p, int k) const { return p.map.seq_of(t + k); }
};

// What a workgroup's waves hand each other: their pairs by channel, of two tiles in turn.
struct GlrLds {
  Step wave[2][kGlrWaves][kGlrChannels];
};

// The pair of the wave's stretches before the thread's (FORWARD: in time, else behind it) into
// `before`; the wave's own to LDS.
template <bool FORWARD>
__device__ __forceinline__ void wave_steps(const Step (&own)[kV], Step (&wave)[kGlrChannels], Step (&before)[kV]) {
  static_assert(kLanes == 32, "two stretches a wave");
  const int lane = threadIdx.x & 63, l = lane % kLanes;
  const bool later = FORWARD ? lane >= kLanes : lane < kLanes;
#pragma unroll
  for (int e = 0; e < kV; ++e) {
    const Step other{__shfl_xor(own[e].P, kLanes), __shfl_xor(own[e].S, kLanes)};
    before[e].P = later ? other.P : 1.f;
    before[e].S = later ? other.S : 0.f;
    const Step both = join(other, own[e]);
    if (later) wave[l * kV + e] = both;
  }
}

// After the barrier: the state before the thread's stretch.  Each wave goes through all waves' pairs
// for itself, a lane for one channel (kV (lane % kLanes) + lane / kLanes), whose state it carries from
// tile to tile (PAIR: the pair of everything so far).
template <bool FORWARD, bool PAIR>
__device__ __forceinline__ void state_before(const Step (&wave)[kGlrWaves][kGlrChannels], const Step (&before)[kV], float& carry,
                                             Step& pair, float (&h)[kV]) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, own = (lane % kLanes) * kV + lane / kLanes;
  float mine = carry;
#pragma unroll
  for (int v = 0; v < kGlrWaves; ++v) {
    const int u = FORWARD ? v : kGlrWaves - 1 - v;
    const Step x = wave[u][own];
    mine = u == w ? carry : mine;
    carry = apply(x, carry);
    if (PAIR) pair = join(pair, x);
  }
#pragma unroll
  for (int e = 0; e < kV; ++e) h[e] = apply(before[e], __shfl(mine, e * kLanes + lane % kLanes));
}

// The state of the lane's channel before chunk c, from the pairs of the chunks before it (FORWARD)
// or behind it.
template <bool FORWARD> __device__ __forceinline__ float chunk_state(const GlrParams& p, int c, int64_t channel) {
  float h = 0.f;
  if (p.apart || channel >= p.D) return h;
  const int count = FORWARD ? c : p.nchunk - 1 - c;
  constexpr int U = 8;   // loads in flight
  for (int k0 = 0; k0 < count; k0 += U) {
    Step x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(k0 + u, count - 1), chunk = FORWARD ? k : p.nchunk - 1 - k;
      const float* at = p.sum + ((int64_t)chunk * 2) * p.D + channel;
      x[u] = Step{at[0], at[p.D]};
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u < count) h = apply(x[u], h);
  }
  return h;
}
__device__ __forceinline__ void write_pair(const GlrParams& p, uint32_t chunk, int64_t channel, const Step& pair) {
  float* at = p.sum + (int64_t)chunk * 2 * p.D + channel;
  at[0] = pair.P;
  at[p.D] = pair.S;
}

constexpr uint32_t kGlrEmptyWgs = 16;
__device__ __forceinline__ void copy_empty(const GlrParams& p, const float* from, float* to, uint32_t wg) {
  for (int64_t n = wg; n < p.map.nseq; n += kGlrEmptyWgs) {
    if (!p.map.empty[n]) continue;
    for (int64_t c = threadIdx.x; c < p.D; c += kGlrThreads) to[n * p.D + c] = from ? from[n * p.D + c] : 0.f;
  }
}

// The pair of the thread's stretch.
template <bool PLAIN, bool WHOLE>
__device__ __forceinline__ void stretch_forward(const GlrParams& p, const Place& q, const Channels<WHOLE>& ch,
                                                const float (&a)[kTok][kV], const float (&b)[kTok][kV], Step (&own)[kV]) {
#pragma unroll
  for (int e = 0; e < kV; ++e) own[e] = Step{1.f, 0.f};
#pragma unroll
  for (int k = 0; k < kTok; ++k) {
    if (!PLAIN && ((q.starts >> k) & 1u)) {
      float h[kV];
      ch.state(p.h0, q.seq(p, k), p.D, h);
#pragma unroll
      for (int e = 0; e < kV; ++e) own[e].S = h[e];
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      own[e].P *= a[k][e];
      own[e].S = __builtin_fmaf(a[k][e], own[e].S, b[k][e]);
    }
  }
  if (!PLAIN && q.starts)
#pragma unroll
    for (int e = 0; e < kV; ++e) own[e].P = -1.f;
}

// ---------------------------------------------------------------------------
// forward.  Behind the chunks' workgroups those that copy the states of sequences without
// tokens.  SUMMARY: the chunk's pair only (16384 x 2048, bf16: 50 us, then 72 for the rest).
// ---------------------------------------------------------------------------
template <typename T, bool HAS_I, bool HAS_Z, bool NORM, bool SUMMARY, bool WHOLE>
__global__ __launch_bounds__(kGlrThreads, sizeof(T) == 2 ? 4 : 2) void glr_fwd_kernel(GlrParams p, uint32_t blocks, int save) {
  __shared__ GlrLds lds;
  if (blockIdx.x >= blocks * p.nchunk) {
    copy_empty(p, p.h0, p.hfin, blockIdx.x - p.nchunk * blocks);
    return;
  }
  const Work<WHOLE> w(p, blocks);
  float A[kV];
  w.ch.load(p.A, A);
#pragma unroll
  for (int e = 0; e < kV; ++e) A[e] *= kLog2e;
  float carry = SUMMARY ? 0.f : chunk_state<true>(p, (int)w.chunk, w.channel);
  Step pair{1.f, 0.f};
  // the next tile's rows are on their way while this one's are worked on
  Rows<T> x, r, i, z, x1, r1, i1;
  auto load = [&](int64_t tile) {
    r1.load(p.r, p.rs, tile, w);
    x1.load(p.x, p.xs, tile, w);
    if (HAS_I) i1.load(p.i, p.is, tile, w);
  };
  load(w.t0);
  const int tiles = w.tiles();
  for (int n = 0; n < tiles; ++n) {
    const int64_t tile = w.t0 + (int64_t)n * kTile;
    const bool plain = plain_tile(p, tile, w.end);
    r = r1;
    x = x1;
    if (HAS_I) i = i1;
    // (in this order: loads complete in the order of their issue)
    if (HAS_Z && !SUMMARY) z.load(p.z, p.zs, tile, w);
    if (n + 1 < tiles) load(tile + kTile);
    if (save && !SUMMARY && w.owner) p.ck[((int64_t)w.chunk * p.tiles + n) * p.D + w.channel] = carry;
    const Place q(p, tile + threadIdx.x / kLanes * kTok, w.end, plain);
    if (!plain) {   // tokens of no sequence: a = 1 and zeros
      r.put(q.in, -INFINITY);
      x.put(q.in, 0.f);
      if (HAS_I) i.put(q.in, 0.f);
      if (HAS_Z && !SUMMARY) z.put(q.in, 0.f);
    }
    float a[kTok][kV], b[kTok][kV], h[kV];
    Step own[kV], before[kV];
#pragma unroll
    for (int k = 0; k < kTok; ++k)
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        float m;
        decay<NORM>(A[e] * sigmoid_fast(r.at(k, e)), a[k][e], m);
        b[k][e] = m * x.at(k, e);
        if (HAS_I) b[k][e] *= sigmoid_fast(i.at(k, e));
      }
    if (plain) stretch_forward<true>(p, q, w.ch, a, b, own);
    else stretch_forward<false>(p, q, w.ch, a, b, own);
    wave_steps<true>(own, lds.wave[n & 1][threadIdx.x >> 6], before);
    __syncthreads();
    state_before<true, SUMMARY>(lds.wave[n & 1], before, carry, pair, h);
    if (SUMMARY) continue;
    auto finish = [&](auto only) {
      constexpr bool PLAIN = decltype(only)::value;
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        if (!PLAIN) {
          if (!((q.there >> k) & 1u)) break;
          if ((q.starts >> k) & 1u) w.ch.state(p.h0, q.seq(p, k), p.D, h);
        }
        float out[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          h[e] = __builtin_fmaf(a[k][e], h[e], b[k][e]);
          out[e] = h[e];
          if (HAS_Z) out[e] *= z.at(k, e) * sigmoid_fast(z.at(k, e));
        }
        if (p.o) store_row<T>(p, p.o, tile, k, w, out);
        if (!PLAIN && p.hfin && ((q.in & q.ends) >> k) & 1u) w.ch.store(p.hfin + (int64_t)q.seq(p, k) * p.D, h);
      }
    };
    if (plain) finish(std::true_type());
    else finish(std::false_type());
  }
  if (SUMMARY && w.owner) write_pair(p, w.chunk, w.channel, pair);
}

// A gate's s = sigmoid(z), and 1 - s with all its digits (from s alone it has an error of 6e-8, which for an open
// gate is most of it: 1e-3 at z = 10, all at 17).
__device__ __forceinline__ float gate(float z, float& rest) {
  const float e = __expf(-z), s = __builtin_amdgcn_rcpf(1.f + e);
  rest = __builtin_amdgcn_fmed3f(e * s, 0.f, 1.f);   // (infinity times 0: 0, and s is a factor of all that it is used for)
  return s;
}

// Computed here, not moved behind what follows.
__device__ __forceinline__ void here(float& x) { asm volatile("" : "+v"(x)); }
// Every second token: keeps the scheduler from taking the tokens' independent chains all at once,
// for which there are not registers enough.
__device__ __forceinline__ void few_registers(int k) {
  if (k % 2 == 0) __builtin_amdgcn_sched_barrier(0);
}

// ---------------------------------------------------------------------------
// backward.  The message from a token to the one before it is u_t = a_t l_t, l_t = g_t + u_{t+1};
// a sequence's last token gets dh_final, its first one's message is dh_init.  A tile's states and
// messages need nothing of each other, so one barrier a tile serves both.
// ---------------------------------------------------------------------------
template <typename T, bool HAS_I, bool HAS_Z, bool NORM, bool SUMMARY, bool WHOLE>
__global__ __launch_bounds__(kGlrThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void glr_bwd_kernel(GlrParams p, uint32_t blocks) {
  __shared__ GlrLds fwd, rev;
  // What a thread has no registers for, two tokens a slot: 1 - s of the gates and, with both, r's s, read where the
  // gradients are written (the output gate's slope instead of s, read right behind the barrier: 296 us, not 286).
  constexpr bool kParkS = HAS_I && HAS_Z;
  constexpr int kRestI = 1, kS = 2, kParked = SUMMARY ? 0 : 1 + HAS_I + kParkS;
  __shared__ floatx4 parked[kParked ? kParked : 1][kTok / 2][kParked ? kGlrThreads : 1];
  if (blockIdx.x >= blocks * p.nchunk) {
    copy_empty(p, p.dhfin, p.dh0, blockIdx.x - p.nchunk * blocks);
    return;
  }
  const Work<WHOLE> w(p, blocks);
  float A[kV], dA[kV] = {0.f, 0.f};
  w.ch.load(p.A, A);
  float carry = SUMMARY ? 0.f : chunk_state<false>(p, (int)w.chunk, w.channel);
  Step pair{1.f, 0.f};
  Rows<T> x, r, i, z, d;
  auto load = [&](int64_t tile) {
    r.load(p.r, p.rs, tile, w);
    d.load(p.dO, p.dos, tile, w);
    if (HAS_Z) z.load(p.z, p.zs, tile, w);
    if (HAS_I && !SUMMARY) i.load(p.i, p.is, tile, w);
  };
  const int tiles = w.tiles();
  load(w.t0 + (int64_t)(tiles - 1) * kTile);
  for (int n = tiles - 1; n >= 0; --n) {
    const int64_t tile = w.t0 + (int64_t)n * kTile;
    const bool plain = plain_tile(p, tile, w.end);
    float state = 0.f;
    if (!SUMMARY) {
      x.load(p.x, p.xs, tile, w);
      if (w.channel < p.D) state = p.ck[((int64_t)w.chunk * p.tiles + n) * p.D + w.channel];
    }
    const Place q(p, tile + threadIdx.x / kLanes * kTok, w.end, plain);
    if (!plain) {   // tokens of no sequence: a = 1 and zeros
      r.put(q.in, -INFINITY);
      d.put(q.in, 0.f);
      if (HAS_Z) z.put(q.in, 0.f);
      if (!SUMMARY) x.put(q.in, 0.f);
      if (HAS_I && !SUMMARY) i.put(q.in, 0.f);
    }
    // closed, closed_i: 1 - s of the gates, of two tokens; slope: dO SiLU'(z)
    float a[kTok][kV], m[kTok][kV], sr[kTok][kV], si[kTok][kV], g[kTok][kV], slope[kTok][kV], h[kV], u[kV];
    Step own[kV], before[kV], behind[kV];
    floatx4 closed, closed_i;
    static_assert(2 * kV == 4, "two tokens a slot");
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      few_registers(k);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        float rest;
        sr[k][e] = gate(r.at(k, e), rest);
        if (!SUMMARY) closed[k % 2 * kV + e] = rest;
        decay<NORM && !SUMMARY>(A[e] * kLog2e * sr[k][e], a[k][e], m[k][e]);
        if (HAS_I && !SUMMARY) {
          si[k][e] = gate(i.at(k, e), rest);
          closed_i[k % 2 * kV + e] = rest;
        } else {
          si[k][e] = 1.f;
        }
        g[k][e] = d.at(k, e);
        if (HAS_Z) {
          float silu;
          slope[k][e] = silu_grad_f(z.at(k, e), silu) * g[k][e];
          g[k][e] *= silu;
          here(slope[k][e]);
        }
        here(a[k][e]);
        here(m[k][e]);
        here(sr[k][e]);
        here(g[k][e]);
        if (HAS_I && !SUMMARY) here(si[k][e]);
      }
      if constexpr (!SUMMARY) {
        if (k % 2) {
          parked[0][k / 2][threadIdx.x] = closed;
          if constexpr (HAS_I) parked[kRestI][k / 2][threadIdx.x] = closed_i;
          if constexpr (kParkS) parked[kS][k / 2][threadIdx.x] = floatx4{sr[k - 1][0], sr[k - 1][1], sr[k][0], sr[k][1]};
        }
      }
    }
    if (n > 0) load(tile - kTile);
    // messages from the last token on
#pragma unroll
    for (int e = 0; e < kV; ++e) own[e] = Step{1.f, 0.f};
    auto messages = [&](auto only) {
      constexpr bool PLAIN = decltype(only)::value;
#pragma unroll
      for (int k = kTok - 1; k >= 0; --k) {
        if (!PLAIN && ((q.ends >> k) & 1u)) {
          w.ch.state(p.dhfin, q.seq(p, k), p.D, u);
#pragma unroll
          for (int e = 0; e < kV; ++e) own[e].S = u[e];
        }
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          own[e].P *= a[k][e];
          own[e].S = a[k][e] * (own[e].S + g[k][e]);
        }
      }
      if (!PLAIN && q.ends)
#pragma unroll
        for (int e = 0; e < kV; ++e) own[e].P = -1.f;
    };
    if (plain) messages(std::true_type());
    else messages(std::false_type());
    wave_steps<false>(own, rev.wave[n & 1][threadIdx.x >> 6], behind);
    if (!SUMMARY) {   // states
      float b[kTok][kV];
#pragma unroll
      for (int k = 0; k < kTok; ++k)
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          b[k][e] = m[k][e] * si[k][e] * x.at(k, e);
        }
      if (plain) stretch_forward<true>(p, q, w.ch, a, b, own);
      else stretch_forward<false>(p, q, w.ch, a, b, own);
      wave_steps<true>(own, fwd.wave[n & 1][threadIdx.x >> 6], before);
    }
    __syncthreads();
    state_before<false, SUMMARY>(rev.wave[n & 1], behind, carry, pair, u);
    if (SUMMARY) continue;
    Step none{1.f, 0.f};
    state_before<true, false>(fwd.wave[n & 1], before, state, none, h);
    auto finish = [&](auto only) {
      constexpr bool PLAIN = decltype(only)::value;
      float prev[kTok][kV];
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        few_registers(k);
        if (!PLAIN && ((q.starts >> k) & 1u)) w.ch.state(p.h0, q.seq(p, k), p.D, h);
        float dz[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float b = m[k][e] * si[k][e] * x.at(k, e);
          prev[k][e] = h[e];
          h[e] = __builtin_fmaf(a[k][e], h[e], b);
          if (HAS_Z) dz[e] = slope[k][e] * h[e];
        }
        if (HAS_Z && (PLAIN || ((q.there >> k) & 1u))) store_row<T>(p, p.dz, tile, k, w, dz);
      }
#pragma unroll
      for (int k = kTok - 1; k >= 0; --k) {
        few_registers(k);
        if constexpr (!SUMMARY)
          if (k % 2) {
            closed = parked[0][k / 2][threadIdx.x];
            if constexpr (kParkS) {
              const floatx4 s = parked[kS][k / 2][threadIdx.x];
#pragma unroll
              for (int e = 0; e < kV; ++e) sr[k - 1][e] = s[e], sr[k][e] = s[kV + e];
            }
            if constexpr (HAS_I) closed_i = parked[kRestI][k / 2][threadIdx.x];
          }
        if (!PLAIN) {
          if (!((q.there >> k) & 1u)) continue;
          if ((q.ends >> k) & 1u) w.ch.state(p.dhfin, q.seq(p, k), p.D, u);
        }
        float dx[kV], dr[kV], di[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float l = g[k][e] + u[e];
          const float into = l * m[k][e] * si[k][e];
          float dlog = prev[k][e];
          if (NORM) {
            const float over = m[k][e] > 0.f ? __builtin_amdgcn_rcpf(m[k][e]) : 0.f;
            dlog = __builtin_fmaf(-(si[k][e] * x.at(k, e)), a[k][e] * over, dlog);
          }
          u[e] = a[k][e] * l;
          dlog *= u[e] * sr[k][e];
          dx[e] = into;
          if (HAS_I) di[e] = into * x.at(k, e) * closed_i[k % 2 * kV + e];
          dr[e] = dlog * A[e] * closed[k % 2 * kV + e];
          dA[e] += dlog;
        }
        store_row<T>(p, p.dx, tile, k, w, dx);
        store_row<T>(p, p.dr, tile, k, w, dr);
        if (HAS_I) store_row<T>(p, p.di, tile, k, w, di);
        if (!PLAIN && p.dh0 && ((q.in & q.starts) >> k) & 1u) w.ch.store(p.dh0 + (int64_t)q.seq(p, k) * p.D, u);
      }
    };
    if (plain) finish(std::true_type());
    else finish(std::false_type());
  }
  if (SUMMARY) {
    if (w.owner) write_pair(p, w.chunk, w.channel, pair);
    return;
  }
  // dA over the workgroup's stretches
  __syncthreads();
  float* sums = reinterpret_cast<float*>(&fwd);
#pragma unroll
  for (int e = 0; e < kV; ++e) {
    dA[e] += __shfl_xor(dA[e], kLanes);
    if ((threadIdx.x & 63) < kLanes) sums[(threadIdx.x >> 6) * kGlrChannels + threadIdx.x % kLanes * kV + e] = dA[e];
  }
  __syncthreads();
  if (w.owner) {
    const int own = threadIdx.x % kLanes * kV + threadIdx.x / kLanes;
    float sum = 0.f;
    for (int v = 0; v < kGlrWaves; ++v) sum += sums[v * kGlrChannels + own];
    p.pA[(int64_t)w.chunk * p.D + w.channel] = sum;
  }
}

// Single tokens: a thread owns 4 channels of a sequence, whose state it reads before it
// writes (in place works: a row's last piece is its own, in part).  256 x 4096, bf16: 5.2 us for 18.9 MB, in
// most part a launch and one trip to memory; 5 and 8 tokens at once 11.8 and 16.1, what 61 and 92 MB take.
constexpr int kDecV = 4;
template <typename T, bool HAS_I, bool HAS_Z, bool NORM, bool FULL>
__global__ __launch_bounds__(kThreads) void glr_decode_kernel(GlrParams p, uint32_t pieces, uint32_t count) {
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  if (id >= count) return;
  const int64_t n = id / pieces, c = (int64_t)(id % pieces) * kDecV;
  const int left = (int)min(p.D - c, (int64_t)kDecV);
  float A[kDecV], h[kDecV];
  load_piece<float, kDecV, FULL>(p.A + c, left, A);
  if (p.h0) load_piece<float, kDecV, FULL>(p.h0 + n * p.D + c, left, h);
  else
#pragma unroll
    for (int e = 0; e < kDecV; ++e) h[e] = 0.f;
  for (int64_t k = 0; k < p.map.T; ++k) {
    const int64_t t = n * p.map.T + k;
    float x[kDecV], r[kDecV], i[kDecV], z[kDecV];
    load_piece<T, kDecV, FULL>(reinterpret_cast<const T*>(p.x) + t * p.xs + c, left, x);
    load_piece<T, kDecV, FULL>(reinterpret_cast<const T*>(p.r) + t * p.rs + c, left, r);
    if (HAS_I) load_piece<T, kDecV, FULL>(reinterpret_cast<const T*>(p.i) + t * p.is + c, left, i);
    if (HAS_Z) load_piece<T, kDecV, FULL>(reinterpret_cast<const T*>(p.z) + t * p.zs + c, left, z);
#pragma unroll
    for (int e = 0; e < kDecV; ++e) {
      float a, m;
      decay<NORM>(A[e] * kLog2e * sigmoid_fast(r[e]), a, m);
      float b = m * x[e];
      if (HAS_I) b *= sigmoid_fast(i[e]);
      h[e] = __builtin_fmaf(a, h[e], b);
      x[e] = HAS_Z ? h[e] * (z[e] * sigmoid_fast(z[e])) : h[e];
    }
    store_piece<T, kDecV, FULL>(reinterpret_cast<T*>(p.o) + t * p.D + c, left, x);
  }
  store_piece<float, kDecV, FULL>(p.hfin + n * p.D + c, left, h);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
uint32_t blocks_of(const GlrParams& p) { return (uint32_t)((p.D + kGlrChannels - 1) / kGlrChannels); }

template <typename F> hipError_t with(const GlrParams& p, bool bf16, bool i, bool z, bool whole, F f) {
  auto types = [&](auto T) {
    auto gates = [&](auto I) {
      auto out = [&](auto Z) {
        auto norm = [&](auto N) {
          if (whole) f(T, I, Z, N, std::true_type());
          else f(T, I, Z, N, std::false_type());
        };
        if (p.normalize) norm(std::true_type());
        else norm(std::false_type());
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
  constexpr int64_t tile = kTile;
  // Whole sequences where they give every CU a workgroup: then no pass before is needed.  Else chunks, for two
  // workgroups a CU (16384 x 2048: 124 us, one a CU 139).  4096 x 4096 with gradients, us: 1 to 3 sequences, cut, 190, 341,
  // 509; 4, whole, 441 (cut in two each 775); 5 and 8, whole, in a second round of workgroups, 736 and 925.
  constexpr int64_t cus = 256;
  const int64_t apart = max((int64_t)1, cus / blocks), want = max((int64_t)1, 2 * cus / blocks);
  p.apart = 0;
  if (!packed && p.map.nseq >= apart) {
    const int64_t T = max(p.map.T, (int64_t)1), each = max(p.map.nseq / want, (tile + T - 1) / T);
    p.L = max(each, (int64_t)1) * p.map.T;
    p.apart = 1;
  } else {
    const int64_t n = max((int64_t)1, min(want, (ntok + tile - 1) / tile));
    p.L = ((ntok + n - 1) / n + tile - 1) / tile * tile;
  }
  if (p.L < 1) p.L = tile;
  const int64_t n = (ntok + p.L - 1) / p.L;
  p.nchunk = (int32_t)n;
  p.tiles = (int32_t)((p.L + tile - 1) / tile);
  if (n <= 1) p.apart = 1;
  // Room in the workspace for as many as any call of up to this many tokens has, cut this way or that, so that it serves
  // smaller calls too.  Chunks of a tile or more: `all` at most; whole sequences: fewer than 2 want, since
  // each >= nseq / want rounded down.  A chunk has up to 1 + all / apart tiles, one of them begun.
  const int64_t all = (ntok + tile - 1) / tile;
  p.room_sum = want > 1 && all > 1 ? min(want, all) : 0;
  p.room_chunks = min(2 * want, all);
  p.room_tiles = all == 0 ? 0 : all + p.room_chunks + (all + apart - 1) / apart + 2;
}

int64_t glr_decode_wgs(const GlrParams& p) { return ((p.D + kDecV - 1) / kDecV * p.map.nseq + kThreads - 1) / kThreads; }

hipError_t launch_glr_forward(const GlrParams& p, bool bf16, bool save, bool outputs, hipStream_t stream) {
  const uint32_t blocks = blocks_of(p), main = blocks * p.nchunk;
  hipError_t e = hipSuccess;
  if (!p.apart) {
    e = with(p, bf16, p.i, false, p.D >= kV, [&](auto T, auto I, auto Z, auto N, auto F) {
      hipLaunchKernelGGL((glr_fwd_kernel<decltype(T), I.value, Z.value, N.value, true, F.value>), dim3(main), dim3(kGlrThreads), 0, stream, p,
                         blocks, 0);
    });
    if (e != hipSuccess) return e;
  }
  GlrParams q = p;
  if (!outputs) q.o = nullptr, q.hfin = nullptr;
  const uint32_t extra = p.map.seq && q.hfin ? kGlrEmptyWgs : 0;
  return with(p, bf16, p.i, p.z && outputs, p.D >= kV, [&](auto T, auto I, auto Z, auto N, auto F) {
    hipLaunchKernelGGL((glr_fwd_kernel<decltype(T), I.value, Z.value, N.value, false, F.value>), dim3(main + extra), dim3(kGlrThreads), 0,
                       stream, q, blocks, save ? 1 : 0);
  });
}

hipError_t launch_glr_backward(const GlrParams& p, bool bf16, hipStream_t stream) {
  const uint32_t blocks = blocks_of(p), main = blocks * p.nchunk, extra = p.map.seq && p.dh0 ? kGlrEmptyWgs : 0;
  if (!p.apart) {
    const hipError_t e = with(p, bf16, p.i, p.z, p.D >= kV, [&](auto T, auto I, auto Z, auto N, auto F) {
      hipLaunchKernelGGL((glr_bwd_kernel<decltype(T), I.value, Z.value, N.value, true, F.value>), dim3(main), dim3(kGlrThreads), 0, stream, p,
                         blocks);
    });
    if (e != hipSuccess) return e;
  }
  return with(p, bf16, p.i, p.z, p.D >= kV, [&](auto T, auto I, auto Z, auto N, auto F) {
    hipLaunchKernelGGL((glr_bwd_kernel<decltype(T), I.value, Z.value, N.value, false, F.value>), dim3(main + extra), dim3(kGlrThreads), 0,
                       stream, p, blocks);
  });
}

hipError_t launch_glr_decode(const GlrParams& p, bool bf16, hipStream_t stream) {
  const uint32_t pieces = (uint32_t)((p.D + kDecV - 1) / kDecV), count = pieces * (uint32_t)p.map.nseq;
  return with(p, bf16, p.i, p.z, p.D % kDecV == 0, [&](auto T, auto I, auto Z, auto N, auto F) {
    hipLaunchKernelGGL((glr_decode_kernel<decltype(T), I.value, Z.value, N.value, F.value>), dim3((count + kThreads - 1) / kThreads),
                       dim3(kThreads), 0, stream, p, pieces, count);
  });
}

}  // namespace rla

// Shared by the selective scan's kernels (ssm_fwd.hip, ssm_bwd.hip).
//
// Layout of the work.  A channel's states are spread over LPC lanes of NS states each
// (16 states: four lanes of four), a wave holds 64 / LPC channels and a workgroup
// four times that (`kCB`), all of one group of B and C.  Workgroups are (block of
// channels) x (chunk of tokens).  The states are diagonal, so there is no matrix
// product in the recurrence: a state costs a product and an exponential for its
// decay, its input's product and two multiply-adds a token, on the vector ALUs.
//
// A sequence of several chunks is scanned in two passes: the first leaves every
// chunk's end state from a zero start and the sum of its steps s; since the decay
// over a chunk is exp(A sum s), the second pass folds the chunks before its own
// into its start state by itself.
//
// Four lanes of four states with as many chunks as fill the card, against eight lanes of
// two states, which fill it without chunks: 16384 tokens in 4 sequences x 4096 channels
// x 16 states, bf16, forward 161 + 347 against 490 us, gradients 200 + 1161 against 1547
// (the sums over a channel's lanes and what is once per channel double with the lanes):
// the forward alone would be 18 us shorter with eight, the step is 168 us shorter with
// four, and both directions share the layout.  Eight waves a workgroup instead of four:
// forward 527, gradients 1660.
#pragma once

#include "layer.hpp"

namespace rla {

struct SsmParams {
  TokenMap map;
  int64_t D = 0, N = 0, G = 1, Dg = 0;
  int64_t us = 0, dts = 0, zs = 0, bs = 0, cs = 0, dos = 0;
  int32_t softplus = 0, cps = 1, nchunk = 1, bpg = 1;   // chunks per dense sequence, chunks, blocks per group
  int64_t L = 0;                                          // tokens per chunk, a multiple of kSsmTile
  const void* u = nullptr;
  const void* delta = nullptr;
  const float* A = nullptr;
  const void* B = nullptr;
  const void* C = nullptr;
  const float* skip = nullptr;
  const void* z = nullptr;
  const float* dbias = nullptr;
  const float* h0 = nullptr;
  void* o = nullptr;
  float* hfin = nullptr;
  const void* dO = nullptr;
  const float* dhfin = nullptr;
  void* du = nullptr;
  void* ddelta = nullptr;
  void* dB = nullptr;
  void* dC = nullptr;
  void* dz = nullptr;
  float* dh0 = nullptr;
  // workspace (NP: states padded to the kernels' 8, 16, 32 or 64)
  float* S = nullptr;        // [nchunk][D][NP] end states from a zero start
  float* sumd = nullptr;     // [nchunk][D] sums of the steps
  int32_t* flags = nullptr;  // [nchunk] kHasStart, kClosed
  float* ck = nullptr;       // [nchunk][L / 16][D][NP] states before every 16 tokens (saving forward)
  float* E = nullptr;        // [nchunk][D][NP] the reverse pass's S
  float* pBC = nullptr;      // [G * bpg][ntok][2][N] a block's sums of dB, dC
  float* pA = nullptr;       // [nchunk][D][N]
  float* pD = nullptr;       // [nchunk][2][D] dskip, ddelta_bias
};

constexpr int kSsmTile = 32;   // tokens staged at a time in the forward
constexpr int kSsmSub = 16;    // tokens between saved states, staged at a time in the backward
constexpr int kHasStart = 1;   // a sequence starts at one of the chunk's tokens
constexpr int kClosed = 2;     // ... after its first one, or right behind the chunk
constexpr int kSsmMaxChunks = 64;   // of packed tokens, or of a dense sequence

// states padded, and a workgroup's channels
inline int ssm_padded(int64_t N) { return N <= 8 ? 8 : N <= 16 ? 16 : N <= 32 ? 32 : 64; }
inline int ssm_channels(int64_t N) { return N <= 16 ? 64 : N <= 32 ? 32 : 16; }

hipError_t launch_ssm_forward(const SsmParams& p, bool bf16, hipStream_t stream);
hipError_t launch_ssm_decode(const SsmParams& p, bool bf16, hipStream_t stream);
// workgroups of a forward or a backward, of single tokens (at most kMaxWgs of them can run)
inline int64_t ssm_wgs(const SsmParams& p) { return p.G * p.bpg * p.nchunk; }
int64_t ssm_decode_wgs(const SsmParams& p);
// Packed: the states of sequences without tokens, `to` = `from` (NULL: zeros).
hipError_t launch_ssm_empty(const SsmParams& p, const float* from, float* to, hipStream_t stream);
hipError_t launch_ssm_backward(const SsmParams& p, bool bf16, hipStream_t stream);

// ---------------------------------------------------------------------------
// device side
// ---------------------------------------------------------------------------
constexpr float kLog2e = 1.44269504088896f, kLn2 = 0.693147180559945f;

// log(1 + e^x) = max(x, 0) + log(1 + e) with e = e^-|x| <= 1.  With w = 1 + e rounded,
// what the rounding took, e - (w - 1), is added to log(w): to first order the lost part
// over w, and over 1 instead of w it is off by e 2^-24 (a plain log(1 + e) loses all
// digits of small steps).
__device__ __forceinline__ float softplus_exact(float x) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(x)), w = 1.f + e;
  return fmaxf(x, 0.f) + __builtin_fmaf(__builtin_amdgcn_logf(w), kLn2, e - (w - 1.f));
}

template <int NS_, int LPC_, int W_ = 4> struct SsmLanes {
  static constexpr int NS = NS_, LPC = LPC_, NP = NS * LPC;
  static constexpr int kW = W_, kThr = 64 * W_;           // waves, threads of a workgroup
  static_assert(kThr <= kThreads, "kMaxWgs");
  static constexpr int kCW = 64 / LPC, kCB = kW * kCW;    // channels of a wave, of a workgroup
  // rows of LDS tiles [token][channel]: four rows apart on different banks
  static constexpr int kRow = kCB + kCB / 4;
  __device__ __forceinline__ static int q() { return (int)threadIdx.x % LPC; }
  __device__ __forceinline__ static int ch() { return (int)threadIdx.x / LPC; }
};

// NS floats from 4-byte aligned memory, `left` of which exist
template <int NS> __device__ __forceinline__ void load_states(const float* p, int left, float (&h)[NS]) {
  load_piece<float, NS>(p, left, h);
}

// x of another lane (every lane of the pattern exists: no value to fall back on, which
// would cost an instruction to set)
template <int CTRL> __device__ __forceinline__ float lane_dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
// lane j of every quad
template <int J> __device__ __forceinline__ float quad_lane(float x) { return lane_dpp<J * 0x55>(x); }

template <typename F> __device__ __forceinline__ void over4(const F& f) {
  f(std::integral_constant<int, 0>());
  f(std::integral_constant<int, 1>());
  f(std::integral_constant<int, 2>());
  f(std::integral_constant<int, 3>());
}

// The kernel's parameters read again from where the launch put them: a kernel with
// some forty pointers and strides would otherwise keep them all in scalar registers
// through its loops, and spill.  Only for kernels whose one argument is SsmParams.
typedef ConstPtr<SsmParams> SsmArgs;
__device__ __forceinline__ SsmArgs fresh_args() {
  uint64_t a = (uint64_t)(__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(a));
  return (SsmArgs)a;
}

// Waves that share a SIMD are served oldest first: one would run ahead to its end and
// leave the other alone there, with half of the ALU idle.  A priority that falls with
// the tile, modulo 4, keeps them within a few tiles of each other.
__device__ __forceinline__ void even_pace(int tile) {
  switch (tile & 3) {
    case 0: __builtin_amdgcn_s_setprio(3); break;
    case 1: __builtin_amdgcn_s_setprio(2); break;
    case 2: __builtin_amdgcn_s_setprio(1); break;
    default: __builtin_amdgcn_s_setprio(0);
  }
}

// Loaded values have arrived here.  Without it a loop that uses values loaded in front
// of it waits for every load at that use in each turn, the next tile's among them.
template <int N> __device__ __forceinline__ void settle(float (&x)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) asm volatile("" : "+v"(x[e]));
}

__device__ __forceinline__ TokenMap fresh_map(SsmArgs a) {
  TokenMap m;
  m.ntok = a->map.ntok;
  m.T = a->map.T;
  m.seq = a->map.seq;
  m.starts = a->map.starts;
  return m;
}

// x, but not known to be the same in the next turn of a loop: comparisons with it stay
// where they are used, and their masks out of the scalar registers in between.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

template <typename V> __device__ __forceinline__ V settled(V x) {
  if constexpr (sizeof(V) == 2) {
    u16 w = __builtin_bit_cast(u16, x);
    asm volatile("" : "+v"(w));
    return __builtin_bit_cast(V, w);
  } else {
    struct Words { uint32_t w[sizeof(V) / 4]; } t = __builtin_bit_cast(Words, x);
#pragma unroll
    for (int e = 0; e < (int)sizeof(V) / 4; ++e) asm volatile("" : "+v"(t.w[e]));
    return __builtin_bit_cast(V, t);
  }
}

// base + a lane's 32-bit offset in bytes
template <typename T> __device__ __forceinline__ const T* at(const void* base, int64_t elems, uint32_t bytes) {
  return reinterpret_cast<const T*>(reinterpret_cast<const char*>(reinterpret_cast<const T*>(base) + elems) + bytes);
}
template <typename T> __device__ __forceinline__ T* at(void* base, int64_t elems, uint32_t bytes) {
  return reinterpret_cast<T*>(reinterpret_cast<char*>(reinterpret_cast<T*>(base) + elems) + bytes);
}

// v[j] summed over the LPC lanes of a channel; lane q keeps token q & 3's.
template <int LPC> __device__ __forceinline__ float tokens_over_lanes(float (&v)[4]) {
  const int lane = threadIdx.x;
  if constexpr (LPC >= 16)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += lane_dpp<0x140>(v[j]);   // row_mirror
  if constexpr (LPC >= 8)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += lane_dpp<0x141>(v[j]);   // row_half_mirror
  const bool b0 = lane & 1, b1 = lane & 2;
  const float x0 = (b0 ? v[1] : v[0]) + lane_dpp<0xB1>(b0 ? v[0] : v[1]);
  const float x1 = (b0 ? v[3] : v[2]) + lane_dpp<0xB1>(b0 ? v[2] : v[3]);
  return (b1 ? x1 : x0) + lane_dpp<0x4E>(b1 ? x0 : x1);
}

// A state carried through the chunks first, first + dir, .. (count of them): h = exp(A sum)
// h + x, with each chunk's x and sum of steps; four chunks' loads at a time.
template <typename SL>
__device__ __forceinline__ void carry_through(const SsmParams& p, const float* x, int first, int dir, int count, int64_t c,
                                              int n0, const float (&A2)[SL::NS], float (&h)[SL::NS]) {
  constexpr int NS = SL::NS;
  for (int i = 0; i < count; i += 4) {
    float v[4][NS], sum[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t cc = first + dir * min(i + u, count - 1);
      load_piece<float, NS, true>(x + (cc * p.D + c) * SL::NP + n0, NS, v[u]);
      sum[u] = p.sumd[cc * p.D + c];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u < count)
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          // (a state that is zero stays so: no infinity times it where A is positive)
          const float carried = h[n] == 0.f ? 0.f : __builtin_amdgcn_exp2f(sum[u] * A2[n]) * h[n];
          h[n] = carried + v[u][n];
        }
  }
}

// Packed: the last chunk before `chunk` that has `flag`, or (ahead) the first behind it;
// there is one.  At most kSsmMaxChunks chunks: a lane each.
__device__ __forceinline__ int find_chunk(const SsmParams& p, int chunk, int flag, bool ahead) {
  const int lane = threadIdx.x & 63;
  const uint64_t got = __ballot(lane < p.nchunk && (ahead ? lane > chunk : lane < chunk) && (p.flags[lane] & flag));
  return ahead ? __ffsll((unsigned long long)got) - 1 : 63 - __clzll((long long)got);
}

// Chunk c: first token, number of tokens.
__device__ __forceinline__ void chunk_range(const SsmParams& p, int c, int64_t& t0, int& len) {
  if (p.map.seq) {
    t0 = (int64_t)c * p.L;
    len = (int)min(p.L, p.map.ntok - t0);
  } else {
    const int b = c / p.cps, j = c - b * p.cps;
    t0 = b * p.map.T + j * p.L;
    len = (int)min(p.L, p.map.T - j * p.L);
  }
}

// Starts in a chunk: offsets of the last one (-1: none) and of the first one after
// its first token up to the token behind it (len + 1: none).
__device__ __forceinline__ void chunk_starts(const SsmParams& p, int64_t t0, int len, int& last, int& first) {
  last = -1;
  first = len + 1;
  if (!p.map.seq) {
    if (t0 % p.map.T == 0) last = 0;
    if ((t0 + len) % p.map.T == 0) first = len;
    return;
  }
  const int lane = threadIdx.x & 63;
  for (int base = 0; base <= len; base += 64 * 32) {
    const int at = base + lane * 32;
    uint32_t bits = at <= len && t0 + at < p.map.ntok ? p.map.start_bits(t0 + at) : (at <= len ? ~0u : 0u);
    const int n = len - at;   // offsets at .. at + min(n, 31)
    if (n >= 0 && n < 31) bits &= (2u << n) - 1u;
    const uint32_t ahead = at == 0 ? bits & ~1u : bits, inside = n >= 0 && n <= 31 ? bits & ~(1u << n) : bits;
    const uint64_t any = __ballot(ahead != 0);
    if (any && first > len) {
      const int l = __ffsll((unsigned long long)any) - 1;
      const uint32_t w = __shfl(ahead, l);
      first = base + l * 32 + __ffs(w) - 1;
    }
    const uint64_t got = __ballot(inside != 0);
    if (got) {
      const int l = 63 - __clzll((long long)got);
      const uint32_t w = __shfl(inside, l);
      last = base + l * 32 + 31 - __clz(w);
    }
  }
  last = __builtin_amdgcn_readfirstlane(last);
  first = __builtin_amdgcn_readfirstlane(first);
}

// ---------------------------------------------------------------------------
// Staging: tiles of TT tokens x kCB channels, a thread's (token, piece of V
// channels), and of B and C a (token, VB states).  A tile is loaded, as stored, one
// turn ahead of its use.  No load depends on a branch of a lane's own, nor leaves an
// older value in its register (either makes the loads behind it wait for those in
// front): tokens past the chunk read its last one, channels past the block its last
// one, states past the last the last, an absent gate the steps, and all of them are
// masked where they are used.
// ---------------------------------------------------------------------------
constexpr int kStU = 1, kStZ = 2, kStO = 4, kStB = 8, kStC = 16;

template <typename T, typename SL, int TT, int WHAT> struct SsmStage {
  static constexpr int V = TT * SL::kCB / SL::kThr, kPer = SL::kCB / V;
  static constexpr int VB = TT * SL::NP >= SL::kThr ? TT * SL::NP / SL::kThr : 1, kPerB = SL::NP / VB;
  typedef typename RowVec<T, V>::type Vec;
  typedef typename RowVec<T, VB>::type VecB;
  Vec u, d, z, o;
  VecB b, c;
  int seq = 0, seqb = 0;   // of the tokens (packed)

  // token and first channel; token and first state
  __device__ __forceinline__ static int r() { return (int)threadIdx.x / kPer; }
  __device__ __forceinline__ static int pc() { return (int)threadIdx.x % kPer * V; }
  __device__ __forceinline__ static int rb() { return min((int)threadIdx.x / kPerB, TT - 1); }
  __device__ __forceinline__ static int pb() { return (int)threadIdx.x % kPerB * VB; }
  // threads that stage B and C (8 states: half of them, the others repeat the last token)
  __device__ __forceinline__ static bool owns_b() { return TT * SL::NP >= SL::kThr || (int)threadIdx.x < TT * SL::NP; }
  __device__ __forceinline__ bool inside(int k, int end, bool packed) const { return k + r() < end && (!packed || seq >= 0); }
  __device__ __forceinline__ bool inside_b(int k, int end, bool packed) const { return k + rb() < end && (!packed || seqb >= 0); }

  // the piece of row `row` (< 32, its stride < 2^24) from column `col` on, of `width` columns
  template <int N>
  __device__ __forceinline__ static typename RowVec<T, N>::type piece(const void* base, int64_t first, uint32_t row,
                                                                      int64_t stride, int col, bool whole, int width) {
    typedef typename RowVec<T, N>::type Out;
    const uint32_t off = __umul24(row, (uint32_t)stride);
    if (whole) return *at<Out>(base, first, (off + (uint32_t)col) * (uint32_t)sizeof(T));
    Out x;
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = *at<T>(base, first, (off + (uint32_t)min(col + e, width - 1)) * (uint32_t)sizeof(T));
    return x;
  }
  template <typename Q> __device__ __forceinline__ static const Q* at(const void* base, int64_t first, uint32_t bytes) {
    return reinterpret_cast<const Q*>(reinterpret_cast<const char*>(reinterpret_cast<const T*>(base) + first) + bytes);
  }

  // tokens from t on, of which `left` >= 1 are the chunk's; nc channels from c0 on
  __device__ __forceinline__ void load(int64_t t, int left, int64_t c0, int64_t g, int nc) {
    const SsmArgs a = fresh_args();
    const uint32_t rr = min(r(), left - 1), rrb = min(rb(), left - 1);
    const int N = (int)a->N;
    const bool all = nc == SL::kCB, states = N == SL::NP, gated = (WHAT & kStZ) && a->z != nullptr;
    // (all of the scalar loads first, one wait for them)
    const void *pd = a->delta, *pu = a->u, *po = a->dO, *pz = gated ? a->z : a->delta, *pb_ = a->B, *pc_ = a->C;
    const int64_t sd = a->dts, su = a->us, so = a->dos, sz = gated ? a->zs : a->dts, sb = a->bs, sc = a->cs;
    if (a->map.seq) {
      seq = a->map.seq[t + rr];
      seqb = a->map.seq[t + rrb];
    }
    d = piece<V>(pd, t * sd + c0, rr, sd, pc(), all, nc);
    if constexpr (WHAT & kStU) u = piece<V>(pu, t * su + c0, rr, su, pc(), all, nc);
    if constexpr (WHAT & kStO) o = piece<V>(po, t * so + c0, rr, so, pc(), all, nc);
    if constexpr (WHAT & kStZ) z = piece<V>(pz, t * sz + c0, rr, sz, pc(), all, nc);
    if constexpr (WHAT & kStB) b = piece<VB>(pb_, t * sb + g * N, rrb, sb, pb(), states, N);
    if constexpr (WHAT & kStC) c = piece<VB>(pc_, t * sc + g * N, rrb, sc, pb(), states, N);
  }
  // The tile has arrived.  Memory operations are counted in order: a wait for these
  // loads behind the stores of the tile before would be one for the stores too.
  __device__ __forceinline__ void settle() {
    d = settled(d);
    if constexpr (WHAT & kStU) u = settled(u);
    if constexpr (WHAT & kStO) o = settled(o);
    if constexpr (WHAT & kStZ) z = settled(z);
    if constexpr (WHAT & kStB) b = settled(b);
    if constexpr (WHAT & kStC) c = settled(c);
    asm volatile("" : "+v"(seq), "+v"(seqb));
  }
  // steps of the thread's channels
  __device__ __forceinline__ void steps(const float (&bias)[V], bool softplus, float (&s)[V]) const {
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = to_f<T>(d[e]) + bias[e];
    if (softplus)
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] = softplus_exact(s[e]);
  }
};

}  // namespace rla

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
  float* dA = nullptr;
  void* dB = nullptr;
  void* dC = nullptr;
  float* dskip = nullptr;
  void* dz = nullptr;
  float* ddbias = nullptr;
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

// states padded, and a workgroup's channels
inline int ssm_padded(int64_t N) { return N <= 8 ? 8 : N <= 16 ? 16 : N <= 32 ? 32 : 64; }
inline int ssm_channels(int64_t N) { return N <= 16 ? 64 : N <= 32 ? 32 : 16; }

hipError_t launch_ssm_forward(const SsmParams& p, bool bf16, hipStream_t stream);
hipError_t launch_ssm_decode(const SsmParams& p, bool bf16, hipStream_t stream);
// Packed: the states of sequences without tokens, `to` = `from` (NULL: zeros).
hipError_t launch_ssm_empty(const SsmParams& p, const float* from, float* to, hipStream_t stream);
hipError_t launch_ssm_backward(const SsmParams& p, bool bf16, hipStream_t stream);

// ---------------------------------------------------------------------------
// device side
// ---------------------------------------------------------------------------
constexpr float kLog2e = 1.44269504088896f, kLn2 = 0.693147180559945f;

// log(1 + e^x) to a few ulp: with w = 1 + e rounded, log(w) e / (w - 1) corrects the
// rounding of w to first order (a plain log(1 + e) loses all digits of small steps)
__device__ __forceinline__ float softplus_exact(float x) {
  const float e = __expf(x), w = 1.f + e, d = w - 1.f;
  const float l = __builtin_amdgcn_logf(w) * kLn2;
  const float s = d == 0.f ? e : l * e * __builtin_amdgcn_rcpf(d);
  return x > 20.f ? x : s;
}

template <int NS_, int LPC_> struct SsmLanes {
  static constexpr int NS = NS_, LPC = LPC_, NP = NS * LPC;
  static constexpr int kCW = 64 / LPC, kCB = kWaves * kCW;   // channels of a wave, of a workgroup
  // rows of LDS tiles [token][channel]: four rows apart on different banks
  static constexpr int kRow = kCB + kCB / 4;
  __device__ __forceinline__ static int q() { return (int)threadIdx.x % LPC; }
  __device__ __forceinline__ static int ch() { return (int)threadIdx.x / LPC; }
};

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));

// NS floats from 4-byte aligned memory, `left` of which exist
template <int NS> __device__ __forceinline__ void load_states(const float* p, int left, float (&h)[NS]) {
  load_piece<float, NS>(p, left, h);
}

// lane j of every quad
template <int J> __device__ __forceinline__ float quad_lane(float x) { return dpp<J * 0x55>(x); }

// v[j] summed over the LPC lanes of a channel; lane q keeps token q & 3's.
template <int LPC> __device__ __forceinline__ float tokens_over_lanes(float (&v)[4]) {
  const int lane = threadIdx.x;
  if constexpr (LPC >= 16)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += dpp<0x140>(v[j]);   // row_mirror
  if constexpr (LPC >= 8)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += dpp<0x141>(v[j]);   // row_half_mirror
  const bool b0 = lane & 1, b1 = lane & 2;
  const float x0 = (b0 ? v[1] : v[0]) + dpp<0xB1>(b0 ? v[0] : v[1]);
  const float x1 = (b0 ? v[3] : v[2]) + dpp<0xB1>(b0 ? v[2] : v[3]);
  return (b1 ? x1 : x0) + dpp<0x4E>(b1 ? x0 : x1);
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

}  // namespace rla

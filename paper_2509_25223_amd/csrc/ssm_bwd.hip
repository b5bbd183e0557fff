// Selective scan, backward (layout of the work: ssm.hpp).  With a_t = exp(s_t A),
// x_t = s_t u_t and dy_t the gradient of C_t . h_t + skip u_t:
//   dh_t = dy_t C_t + a_{t+1} dh_{t+1}
//   dC_t = sum_c dy_t h_t        dB_t = sum_c dh_t x_t        (over a group's channels)
//   q_t  = dh_t a_t h_{t-1}      dA   = sum_t s_t q_t
//   ds_t = sum_n A q_t + u_t sum_n dh_t B_t
//   du_t = s_t sum_n dh_t B_t + skip dy_t
// A chunk is walked backwards, 16 tokens at a time: from the saved state before
// them the 16 states are formed again and stay in registers with their decays,
// then the same lanes run the reverse recurrence.  (Going back through h_{t-1} =
// (h_t - x_t B_t) / a_t would need no saved state and lose all digits.)
//
// Two sums cross lanes.  Those over a channel's states are over a quad (or 8, 16
// lanes); four tokens are reduced together and left on one lane each.  Those over
// channels (dB, dC) are 4 tokens x NS states a lane over the wave's channels,
// halved lane bit by lane bit (two instructions a pair, where a sum of one value
// over 16 lanes costs 4 a value); then over the waves in LDS, and over the blocks
// of channels by a last kernel, from fp32 partial sums.  No atomics.
//
// The vector ALU bounds it: 29 instructions a token, channel and state (counters).  15 are
// the recurrence and its products (the exponential, at a quarter of their rate, one of
// them), 4 the sums over channels; the others bring a token's values to the lanes, sum
// over a channel's lanes, and are what is once a token and channel.  16384 tokens in
// 4 sequences x 4096 channels x 16 states, bf16: chunk summaries 195 us (88 % with the ALUs
// at work), gradients 1112 (83 %; 1.3 GB: 0.25 ms), sums of dB and dC 36.  Two waves a SIMD at
// 255 registers; fp32 spills 2 of them.
#include "ssm.hpp"

namespace rla {

namespace {

// halves of a pair: lanes with the bit clear get a summed over the two lanes that
// differ in it, the others b
__device__ __forceinline__ float half32(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float half16(float a, float b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// x of lane ^ 4
__device__ __forceinline__ float across4(float x) {
  int y = __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x104, 0xF, 0xF, true);          // row_shl:4
  y = __builtin_amdgcn_update_dpp(y, __builtin_bit_cast(int, x), 0x114, 0xF, 0xA, false);       // row_shr:4
  return __builtin_bit_cast(float, y);
}
// The same halving by lane bit 3, of (a0, a2) and of (a1, a3): an add that the lanes of
// two of a row's four banks execute, then one for the other two (selecting what to add
// first takes three instructions, not two).  In asm, as the compiler knows no masked
// add; a value just written may be read across lanes two instructions later.
__device__ __forceinline__ void half8(float a0, float a1, float a2, float a3, float& b0, float& b1) {
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %0, %2, %2 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
      "v_add_f32_dpp %1, %3, %3 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
      "v_add_f32_dpp %0, %4, %4 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0xc"
      : "=&v"(b0), "=&v"(b1) : "v"(a0), "v"(a1), "v"(a2), "v"(a3));
}
// and by lane bit 2
__device__ __forceinline__ float half4(float b0, float b1) {
  float c;
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %0, %1, %1 row_shl:4 row_mask:0xf bank_mask:0x5\n\t"
      "v_add_f32_dpp %0, %2, %2 row_shr:4 row_mask:0xf bank_mask:0xa"
      : "=&v"(c) : "v"(b0), "v"(b1));
  return c;
}

// v[j][n] summed over the wave's channels.  The lane keeps kKeep values, of token
// `tok` and the states from `st` on.
template <typename SL> struct ChannelSums {
  static constexpr int NS = SL::NS, LPC = SL::LPC;
  static constexpr int kKeep = LPC >= 16 ? NS : LPC == 8 ? NS / 2 : 1;
  __device__ __forceinline__ static int tok() { return (threadIdx.x >> 4) & 1 | (threadIdx.x >> 4) & 2; }
  __device__ __forceinline__ static int st() {
    const int lane = threadIdx.x;
    if constexpr (LPC >= 16) return 0;
    else if constexpr (LPC == 8 || NS == 2) return (lane >> 3 & 1) * (NS / 2);
    else return (lane >> 3 & 1) * 2 + (lane >> 2 & 1);
  }
  __device__ __forceinline__ static void run(const float (&v)[4][NS], float (&out)[kKeep]) {
    float a[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      // bit 5: tokens 0, 1 or 2, 3; bit 4: the first or second of them
      a[n] = half16(half32(v[0][n], v[2][n]), half32(v[1][n], v[3][n]));
    }
    if constexpr (LPC >= 16) {
#pragma unroll
      for (int n = 0; n < NS; ++n) out[n] = a[n];
    } else {
      float b[NS / 2];
      if constexpr (NS == 2) {
        const bool b3 = threadIdx.x & 8;
        b[0] = (b3 ? a[1] : a[0]) + lane_dpp<0x128>(b3 ? a[0] : a[1]);   // row_ror:8
      } else {
        half8(a[0], a[1], a[2], a[3], b[0], b[1]);
      }
      if constexpr (LPC == 8) {
#pragma unroll
        for (int n = 0; n < NS / 2; ++n) out[n] = b[n];
      } else if constexpr (NS == 2) {
        out[0] = b[0] + across4(b[0]);
      } else {
        out[0] = half4(b[0], b[1]);
      }
    }
  }
};

// E[chunk]: the gradient of the state entering the chunk, from zero behind it (or,
// where its sequence ends inside, from the final state's).
template <typename T, typename SL>
__global__ __launch_bounds__(SL::kThr) void ssm_rev_kernel(SsmParams p) {
  constexpr int NS = SL::NS, NP = SL::NP, kRow = SL::kRow, TT = kSsmTile;
  typedef SsmStage<T, SL, TT, kStO | kStZ | kStC> St;
  constexpr int V = St::V, VB = St::VB;
  __shared__ __attribute__((aligned(16))) float sD[TT][kRow], sG[TT][kRow], sC[TT][NP];
  const int nblk = (int)p.G * p.bpg, turn = (int)blockIdx.x / nblk, blk = (int)blockIdx.x - turn * nblk;
  // (dense: all but a sequence's first chunk)
  const int chunk = p.map.seq ? turn : turn / (p.cps - 1) * p.cps + turn % (p.cps - 1) + 1;
  const int g = blk / p.bpg;
  const int64_t c0 = g * p.Dg + (int64_t)(blk - g * p.bpg) * SL::kCB;
  const int nc = (int)min((int64_t)SL::kCB, (g + 1) * p.Dg - c0);
  int64_t t0;
  int len, last, first;
  chunk_range(p, chunk, t0, len);
  if (p.map.start_bits(t0) & 1u) return;   // nothing flows out in front
  chunk_starts(p, t0, len, last, first);
  const bool closed = first <= len;
  const int end = closed ? first : len;

  const int q = SL::q(), ch = SL::ch(), n0 = q * NS;
  const bool live = ch < nc;
  const int64_t c = c0 + (live ? ch : 0);
  const int nleft = (int)p.N - n0;
  float A2[NS], dh[NS];
  load_states<NS>(p.A + c * p.N + n0, nleft, A2);
#pragma unroll
  for (int n = 0; n < NS; ++n) A2[n] *= kLog2e;
  const int seq = closed && p.dhfin ? p.map.seq_of(t0 + end - 1) : -1;
  if (seq >= 0) load_states<NS>(p.dhfin + ((int64_t)seq * p.D + c) * p.N + n0, nleft, dh);
  else
#pragma unroll
    for (int n = 0; n < NS; ++n) dh[n] = 0.f;

  St st;
  const int r = St::r(), pc = St::pc(), rb = St::rb(), pb = St::pb(), pleft0 = nc - pc, bleft0 = (int)p.N - pb;
  float bias[V];
#pragma unroll
  for (int e = 0; e < V; ++e) bias[e] = p.dbias && e < pleft0 ? p.dbias[c0 + pc + e] : 0.f;
  settle(A2);
  settle(dh);
  settle(bias);
  const int k_last = (end - 1) / TT * TT;
  const bool packed = p.map.seq != nullptr, sp = p.softplus != 0, gated = p.z != nullptr;
  st.load(t0 + k_last, end - k_last, c0, g, nc);
  for (int k = k_last; k >= 0; k -= TT) {
    even_pace((k_last - k) / TT);
    const bool in = st.inside(k, end, packed);
    const int pleft = fresh(pleft0), bleft = fresh(bleft0);
    float s[V];
    st.steps(bias, sp, s);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool use = in && e < pleft;
      float gy = to_f<T>(st.o[e]);
      if (gated) {
        const float z = to_f<T>(st.z[e]);
        gy *= z * sigmoid_fast(z);
      }
      sD[r][pc + e] = use ? s[e] : 0.f;
      sG[r][pc + e] = use ? gy : 0.f;
    }
    if (st.owns_b()) {
      const bool inb = st.inside_b(k, end, packed);
#pragma unroll
      for (int e = 0; e < VB; ++e) sC[rb][pb + e] = inb && e < bleft ? to_f<T>(st.c[e]) : 0.f;
    }
    __syncthreads();
    if (k >= TT) st.load(t0 + k - TT, TT, c0, g, nc);
struct Four {
      float d, g, c[4][NS];
    };
    auto fetch = [&](int i, Four& f) {
      f.d = sD[i + (q & 3)][ch];
      f.g = sG[i + (q & 3)][ch];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NS; ++n) f.c[j][n] = sC[i + j][n0 + n];
    };
    Four f[2];
    fetch(TT - 4, f[1]);
#pragma unroll
    for (int i = TT - 4; i >= 0; i -= 4) {
      if (i > 0) fetch(i - 4, f[(i / 4 + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
      const Four& now = f[(i / 4) & 1];
      float e[4][NS], x[4][NS];
      over4([&](auto J) {
        constexpr int j = decltype(J)::value;
        const float dj = quad_lane<j>(now.d);
#pragma unroll
        for (int n = 0; n < NS; ++n) e[j][n] = dj * A2[n];
      });
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NS; ++n) e[j][n] = __builtin_amdgcn_exp2f(e[j][n]);
      over4([&](auto J) {   // through the decay at once: a C dy + a dh
        constexpr int j = decltype(J)::value;
        const float gj = quad_lane<j>(now.g);
#pragma unroll
        for (int n = 0; n < NS; ++n) x[j][n] = e[j][n] * (gj * now.c[j][n]);
      });
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 3; j >= 0; --j)
#pragma unroll
        for (int n = 0; n < NS; ++n) dh[n] = __builtin_fmaf(e[j][n], dh[n], x[j][n]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
  }
  if (live) store_piece<float, NS, true>(p.E + ((int64_t)chunk * p.D + c) * NP + n0, NS, dh);
}

template <typename T, typename SL>
__global__ __launch_bounds__(SL::kThr, 2) void ssm_bwd_kernel(SsmParams p) {
  constexpr int NS = SL::NS, LPC = SL::LPC, NP = SL::NP, kRow = SL::kRow, TT = kSsmSub;
  typedef SsmStage<T, SL, TT, kStU | kStZ | kStO | kStB | kStC> St;
  constexpr int V = St::V, VB = St::VB;
  typedef ChannelSums<SL> CS;
  __shared__ __attribute__((aligned(16))) float sD[TT][kRow], sX[TT][kRow], sG[TT][kRow];
  __shared__ __attribute__((aligned(16))) float sI[TT][kRow], sQ[TT][kRow], sY[TT][kRow];
  __shared__ __attribute__((aligned(16))) float sB[TT][NP], sC[TT][NP];
  // each thread's own: the tile as loaded, its channels' bias and skip (registers are what
  // this kernel is short of)
  __shared__ __attribute__((aligned(16))) T sOwn[4][SL::kThr][V];
  __shared__ float sBias[SL::kCB], sSkip[SL::kCB];
  __shared__ __attribute__((aligned(16))) float sBC[SL::kW][2][TT][NP];   // a wave's sums of dB, dC

  const int tid = threadIdx.x, wave = tid >> 6;
  const int nblk = (int)p.G * p.bpg, chunk = (int)blockIdx.x / nblk, blk = (int)blockIdx.x - chunk * nblk;
  const int g = blk / p.bpg;
  const int64_t c0 = g * p.Dg + (int64_t)(blk - g * p.bpg) * SL::kCB;
  const int nc = (int)min((int64_t)SL::kCB, (g + 1) * p.Dg - c0);
  int64_t t0;
  int len;
  chunk_range(p, chunk, t0, len);

  const int q = SL::q(), ch = SL::ch(), n0 = q * NS;
  const bool live = ch < nc;
  const int64_t c = c0 + (live ? ch : 0);
  const int nleft = (int)p.N - n0;
  float A2[NS], dA[NS], carry[NS];
  load_states<NS>(p.A + c * p.N + n0, nleft, A2);
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    A2[n] *= kLog2e;
    dA[n] = 0.f;
  }
  auto state_of = [&](const float* base, int seq, float (&h)[NS]) {
    if (base && seq >= 0) {
      const SsmArgs a = fresh_args();
      load_states<NS>(base + ((int64_t)seq * a->D + c) * a->N + n0, nleft, h);
      settle(h);   // here, and not in every tile's turn of the code that follows
    } else {
#pragma unroll
      for (int n = 0; n < NS; ++n) h[n] = 0.f;
    }
  };
  // the gradient behind the chunk's last token
  int seq = p.map.seq_of(t0 + len - 1);
  if (p.map.seq ? t0 + len >= p.map.ntok || (p.map.start_bits(t0 + len) & 1u) : (t0 + len) % p.map.T == 0) {
    state_of(p.dhfin, seq, carry);
  } else {   // the chunks behind, up to the first that closes the sequence
    const int cc = p.map.seq ? find_chunk(p, chunk, kClosed, true) : chunk / p.cps * p.cps + p.cps - 1;
    load_piece<float, NS, true>(p.E + ((int64_t)cc * p.D + c) * NP + n0, NS, carry);
    carry_through<SL>(p, p.E, cc - 1, -1, cc - 1 - chunk, c, n0, A2, carry);
  }

  St st;
  const int r = St::r(), pc = St::pc(), rb = St::rb(), pb = St::pb(), pleft0 = nc - pc, bleft0 = (int)p.N - pb;
  const uint32_t fout = (r * (uint32_t)p.D + pc) * (uint32_t)sizeof(T), fck = ((live ? ch : 0) * NP + n0) * 4;
  float dskip[V], ddb[V];
#pragma unroll
  for (int e = 0; e < V; ++e) dskip[e] = ddb[e] = 0.f;
  if (tid < SL::kCB) {
    sBias[tid] = p.dbias && tid < nc ? p.dbias[c0 + tid] : 0.f;
    sSkip[tid] = p.skip && tid < nc ? p.skip[c0 + tid] : 0.f;
  }
  __syncthreads();
  float ck[NS];
  auto load_tile = [&](int k) {
    st.load(t0 + k, len - k, c0, g, nc);
    const SsmArgs a = fresh_args();
    const int64_t sub = (int64_t)chunk * (a->L / kSsmSub) + k / kSsmSub;
    load_piece<float, NS, true>(at<float>(a->ck, (sub * a->D + c0) * NP, fck), NS, ck);
  };
  settle(A2);
  settle(carry);
  const int k_last = (len - 1) / TT * TT;
  const bool packed = p.map.seq != nullptr, sp = p.softplus != 0, gated = p.z != nullptr;
  const bool starts_seq = t0 % p.map.T == 0;   // (dense)
  load_tile(k_last);
  for (int k = k_last; k >= 0; k -= TT) {
    const SsmArgs a = fresh_args();
    even_pace((k_last - k) / TT);
    // ---- these tokens into LDS ----
    const uint32_t valid = len - k >= TT ? (1u << TT) - 1u : (1u << (len - k)) - 1u;
    // (a dense chunk's only start is its first token)
    const uint32_t bits = packed ? fresh_map(a).start_bits(t0 + k) & valid : k == 0 && starts_seq ? 1u : 0u;
    const int pleft = fresh(pleft0), bleft = fresh(bleft0);
    const bool here = st.inside(k, len, packed);
    {
      float s[V], bias[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        bias[e] = sBias[pc + e];
        sOwn[0][tid][e] = st.u[e];
        sOwn[1][tid][e] = st.d[e];
        sOwn[2][tid][e] = st.z[e];
        sOwn[3][tid][e] = st.o[e];
      }
      st.steps(bias, sp, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool use = here && e < pleft;
        float gy = to_f<T>(st.o[e]);
        if (gated) {
          const float z = to_f<T>(st.z[e]);
          gy *= z * sigmoid_fast(z);
        }
        sD[r][pc + e] = use ? s[e] : 0.f;
        sX[r][pc + e] = use ? s[e] * to_f<T>(st.u[e]) : 0.f;
        sG[r][pc + e] = use ? gy : 0.f;
      }
      if (st.owns_b()) {
        const bool inb = st.inside_b(k, len, packed);
#pragma unroll
        for (int e = 0; e < VB; ++e) {
          sB[rb][pb + e] = inb && e < bleft ? to_f<T>(st.b[e]) : 0.f;
          sC[rb][pb + e] = inb && e < bleft ? to_f<T>(st.c[e]) : 0.f;
        }
      }
    }
    float h[NS], hck[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) hck[n] = ck[n];
    __syncthreads();
    if (k >= TT) load_tile(k - TT);

    // ---- the states again, then the reverse recurrence ----
    // one stretch [lo, hi) of a sequence at a time, from the last; nearly always all 16
    auto stretch = [&](auto WHOLE, int lo, int hi) {
      constexpr bool whole = decltype(WHOLE)::value;
      auto inside = [&](int t) { return whole || (t >= lo && t < hi); };
      float decay[TT][NS], hg[TT / 4][NS];   // decays; states before every 4 tokens
      // as in the forward, passes over four tokens' states of independent instructions
#pragma unroll
      for (int i = 0; i < TT; i += 4) {
        const float dv = sD[i + (q & 3)][ch], xv = sX[i + (q & 3)][ch];
        float x[4][NS], c4[4][NS];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            x[j][n] = sB[i + j][n0 + n];
            c4[j][n] = sC[i + j][n0 + n];
          }
        over4([&](auto J) {
          constexpr int j = decltype(J)::value;
          const float dj = quad_lane<j>(dv), xj = quad_lane<j>(xv);
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            decay[i + j][n] = dj * A2[n];
            x[j][n] *= xj;
          }
        });
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int n = 0; n < NS; ++n) decay[i + j][n] = __builtin_amdgcn_exp2f(decay[i + j][n]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NS; ++n) hg[i / 4][n] = h[n];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (inside(i + j))
#pragma unroll
            for (int n = 0; n < NS; ++n) x[j][n] = h[n] = __builtin_fmaf(decay[i + j][n], h[n], x[j][n]);
        if (gated) {
          float y[4];
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = n == 0 ? x[j][n] * c4[j][n] : __builtin_fmaf(x[j][n], c4[j][n], y[j]);
          const float yt = tokens_over_lanes<LPC>(y);
          if ((LPC == 4 || q < 4) && inside(i + q)) sY[i + q][ch] = yt;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = TT - 4; i >= 0; i -= 4) {
        const float dv = sD[i + (q & 3)][ch], xv = sX[i + (q & 3)][ch], gv = sG[i + (q & 3)][ch];
        float x[4][NS], ah[4][NS], v[4][NS];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int n = 0; n < NS; ++n) x[j][n] = sB[i + j][n0 + n];
        // the states again, from the decays; dy h for dC
        float ht[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) ht[n] = hg[i / 4][n];
        over4([&](auto J) {
          constexpr int j = decltype(J)::value;
          const float gj = quad_lane<j>(gv), xj = quad_lane<j>(xv);
          if (inside(i + j))
#pragma unroll
            for (int n = 0; n < NS; ++n) {
              ah[j][n] = decay[i + j][n] * ht[n];
              ht[n] = __builtin_fmaf(xj, x[j][n], ah[j][n]);
            }
#pragma unroll
          for (int n = 0; n < NS; ++n) v[j][n] = inside(i + j) ? gj * ht[n] : 0.f;
        });
        float oB[CS::kKeep], oC[CS::kKeep];
        CS::run(v, oC);
        __builtin_amdgcn_sched_barrier(0);
        // dh of each token, from behind
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int n = 0; n < NS; ++n) x[j][n] = sC[i + j][n0 + n];
        over4([&](auto J) {
          constexpr int j = 3 - decltype(J)::value;
          const float gj = quad_lane<j>(gv);
          if (inside(i + j))
#pragma unroll
            for (int n = 0; n < NS; ++n) {
              x[j][n] = __builtin_fmaf(gj, x[j][n], carry[n]);
              carry[n] = x[j][n] * decay[i + j][n];
            }
        });
        __builtin_amdgcn_sched_barrier(0);
        float into[4], qa[4];
        over4([&](auto J) {
          constexpr int j = decltype(J)::value;
          const float dj = quad_lane<j>(dv), xj = quad_lane<j>(xv);
          if (inside(i + j)) {
#pragma unroll
            for (int n = 0; n < NS; ++n) {
              const float qn = x[j][n] * ah[j][n], b = sB[i + j][n0 + n];
              v[j][n] = x[j][n] * xj;
              into[j] = n == 0 ? x[j][n] * b : __builtin_fmaf(x[j][n], b, into[j]);
              qa[j] = n == 0 ? A2[n] * qn : __builtin_fmaf(A2[n], qn, qa[j]);
              dA[n] = __builtin_fmaf(dj, qn, dA[n]);
            }
          } else {
            into[j] = qa[j] = 0.f;
#pragma unroll
            for (int n = 0; n < NS; ++n) v[j][n] = 0.f;
          }
        });
        const float it = tokens_over_lanes<LPC>(into), qt = tokens_over_lanes<LPC>(qa);
        if ((LPC == 4 || q < 4) && inside(i + q)) {
          sI[i + q][ch] = it;
          sQ[i + q][ch] = qt;
        }
        CS::run(v, oB);
        if (inside(i + CS::tok())) {
#pragma unroll
          for (int n = 0; n < CS::kKeep; ++n) {
            sBC[wave][0][i + CS::tok()][n0 + CS::st() + n] = oB[n];
            sBC[wave][1][i + CS::tok()][n0 + CS::st() + n] = oC[n];
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    for (int hi = TT; hi > 0;) {
      const uint32_t below = bits & ((1u << hi) - 1u);
      const int lo = below ? 31 - __clz(below) : 0;
      const bool starts = below != 0;
      const int64_t t = t0 + k + lo;
      if (starts) {
        state_of(a->h0, p.map.seq_of(t), h);
      } else {
#pragma unroll
        for (int n = 0; n < NS; ++n) h[n] = hck[n];
      }
      if (lo == 0 && hi == TT) stretch(std::true_type(), lo, hi);
      else stretch(std::false_type(), lo, hi);
      if (starts) {   // what flows out is the initial state's; in front, another sequence ends
        const SsmArgs a = fresh_args();
        const TokenMap map = fresh_map(a);
        const int sq = map.seq_of(t);
        if (a->dh0 && live && sq >= 0) store_piece<float, NS>(a->dh0 + ((int64_t)sq * a->D + c) * a->N + n0, nleft, carry);
        state_of(a->dhfin, k + lo > 0 ? map.seq_of(t - 1) : -1, carry);
      }
      hi = lo;
    }
    st.settle();
    settle(ck);
    __syncthreads();

    // ---- gradients of the activations (the thread's own places of the tiles) ----
    // no branches among the values: a wait for one would be for the stores in front too
    {
      float du[V], dd[V], dz[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool use = here && e < pleft;   // else outside every sequence, or past the chunk: zeros
        const float u = to_f<T>(sOwn[0][tid][e]), skip = sSkip[pc + e], gy = sG[r][pc + e], into = sI[r][pc + e];
        const float slope = sp ? sigmoid_fast(to_f<T>(sOwn[1][tid][e]) + sBias[pc + e]) : 1.f;
        float act;
        const float zs = silu_grad_f(to_f<T>(sOwn[2][tid][e]), act);
        du[e] = use ? __builtin_fmaf(sD[r][pc + e], into, skip * gy) : 0.f;
        dd[e] = use ? __builtin_fmaf(u, into, kLn2 * sQ[r][pc + e]) * slope : 0.f;
        dz[e] = use ? to_f<T>(sOwn[3][tid][e]) * __builtin_fmaf(skip, u, sY[r][pc + e]) * zs : 0.f;
        dskip[e] += use ? gy * u : 0.f;
        ddb[e] += dd[e];
      }
      // a thread's values of the sums over the waves: (token, dB or dC, states)
      constexpr int E = TT * 2 * NP / SL::kThr, kPerT = 2 * NP / E;
      const int ft = fresh(tid), et = ft / kPerT, w = ft % kPerT * E / NP, n1 = ft % kPerT * E % NP;
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float* from = &sBC[0][w][et][n1 + e];
        v[e] = from[0];
#pragma unroll
        for (int m = 1; m < SL::kW; ++m) v[e] += from[m * 2 * TT * NP];
      }
      const int64_t first = (t0 + k) * a->D + c0, N = a->N;
      float* part = a->pBC + (((int64_t)blk * a->map.ntok + t0 + k) * 2) * N;
      T *pu = at<T>(a->du, first, fout), *pd = at<T>(a->ddelta, first, fout), *pz = at<T>(a->dz, first, fout);
      if (k + r < len) {
        if (nc == SL::kCB) {
          store_piece<T, V, true>(pu, V, du);
          store_piece<T, V, true>(pd, V, dd);
          if (gated) store_piece<T, V, true>(pz, V, dz);
        } else {
          store_piece<T, V>(pu, pleft, du);
          store_piece<T, V>(pd, pleft, dd);
          if (gated) store_piece<T, V>(pz, pleft, dz);
        }
      }
      if (k + et < len) {
        if (N == NP) store_piece<float, E, true>(part + (et * 2 + w) * NP + n1, E, v);
        else store_piece<float, E>(part + (et * 2 + w) * N + n1, fresh((int)N - n1), v);
      }
    }
  }
  if (live) store_piece<float, NS>(p.pA + ((int64_t)chunk * p.D + c) * p.N + n0, nleft, dA);
  // the threads' tokens of a channel
  __syncthreads();
#pragma unroll
  for (int e = 0; e < V; ++e) {
    sD[r][pc + e] = dskip[e];
    sX[r][pc + e] = ddb[e];
  }
  __syncthreads();
  for (int i = tid; i < 2 * nc; i += SL::kThr) {
    const int w = i / nc, cc = i % nc;
    float v = 0.f;
#pragma unroll
    for (int t = 0; t < TT; ++t) v += w ? sX[t][cc] : sD[t][cc];
    p.pD[((int64_t)chunk * 2 + w) * p.D + c0 + cc] = v;
  }
}

// dB, dC [tokens][G][N] from the blocks' sums (in their order); a value a thread, or
// several where there are more values than a launch has threads
template <typename T>
__global__ __launch_bounds__(kThreads) void ssm_bc_kernel(SsmParams p) {
  const int64_t per = p.map.ntok * 2 * p.N;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < per; i += (int64_t)gridDim.x * kThreads) {
    const int64_t t = i / (2 * p.N);
    const int w = (int)(i / p.N & 1), n = (int)(i % p.N);
    T* out = reinterpret_cast<T*>(w ? p.dC : p.dB);
    for (int g = 0; g < p.G; ++g) {
      float v = 0.f;
      for (int b = 0; b < p.bpg; ++b) v += p.pBC[((int64_t)g * p.bpg + b) * per + i];
      out[(t * p.G + g) * p.N + n] = from_f<T>(v);
    }
  }
}

template <typename T, typename SL> hipError_t backward(const SsmParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)ssm_wgs(p));
  if (p.cps > 1) {
    const dim3 part((uint32_t)(p.G * p.bpg * (p.map.seq ? p.nchunk : p.nchunk / p.cps * (p.cps - 1))));
    hipLaunchKernelGGL((ssm_rev_kernel<T, SL>), part, dim3(SL::kThr), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((ssm_bwd_kernel<T, SL>), grid, dim3(SL::kThr), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t per = p.map.ntok * 2 * p.N;
  hipLaunchKernelGGL(ssm_bc_kernel<T>, dim3((uint32_t)min((per + kThreads - 1) / kThreads, kMaxWgs)), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template <typename T> hipError_t dispatch(const SsmParams& p, hipStream_t stream) {
  switch (ssm_padded(p.N)) {
    case 8: return backward<T, SsmLanes<2, 4>>(p, stream);
    case 16: return backward<T, SsmLanes<4, 4>>(p, stream);
    case 32: return backward<T, SsmLanes<4, 8>>(p, stream);
    default: return backward<T, SsmLanes<4, 16>>(p, stream);
  }
}

}  // namespace

hipError_t launch_ssm_backward(const SsmParams& p, bool bf16, hipStream_t stream) {
  const hipError_t e = bf16 ? dispatch<u16>(p, stream) : dispatch<float>(p, stream);
  if (e != hipSuccess || !p.map.seq || !p.dh0) return e;
  return launch_ssm_empty(p, p.dhfin, p.dh0, stream);
}

}  // namespace rla

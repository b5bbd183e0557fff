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
// halved lane bit by lane bit (2 to 3 instructions a pair, where a sum of one value
// over 16 lanes costs 4 a value); then over the waves in LDS, and over the blocks
// of channels by a last kernel, from fp32 partial sums.  No atomics.
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
  int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x104, 0xF, 0x5, false);   // row_shl:4
  y = __builtin_amdgcn_update_dpp(y, __builtin_bit_cast(int, x), 0x114, 0xF, 0xA, false);       // row_shr:4
  return __builtin_bit_cast(float, y);
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
    const int lane = threadIdx.x;
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
      const bool b3 = lane & 8;
      float b[NS / 2];
#pragma unroll
      for (int n = 0; n < NS / 2; ++n)
        b[n] = (b3 ? a[n + NS / 2] : a[n]) + dpp<0x128>(b3 ? a[n] : a[n + NS / 2]);   // row_ror:8
      if constexpr (LPC == 8) {
#pragma unroll
        for (int n = 0; n < NS / 2; ++n) out[n] = b[n];
      } else if constexpr (NS == 2) {
        out[0] = b[0] + across4(b[0]);
      } else {
        const bool b2 = lane & 4;
        out[0] = (b2 ? b[1] : b[0]) + across4(b2 ? b[0] : b[1]);
      }
    }
  }
};

// E[chunk]: the gradient of the state entering the chunk, from zero behind it (or,
// where its sequence ends inside, from the final state's).
template <typename T, typename SL>
__global__ __launch_bounds__(kThreads) void ssm_rev_kernel(SsmParams p) {
  constexpr int NS = SL::NS, NP = SL::NP, kRow = SL::kRow, TT = kSsmTile;
  constexpr int V = TT * SL::kCB / kThreads, kPer = SL::kCB / V;
  constexpr int VB = TT * NP / kThreads, kPerB = NP / VB;
  __shared__ __attribute__((aligned(16))) float sD[TT][kRow], sG[TT][kRow], sC[TT][NP];
  const int tid = threadIdx.x;
  const int nblk = (int)p.G * p.bpg, chunk = (int)blockIdx.x / nblk, blk = (int)blockIdx.x - chunk * nblk;
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

  const int r = tid / kPer, pc = tid % kPer * V, pleft = nc - pc;
  const int rb = tid / kPerB, pb = tid % kPerB * VB, bleft = (int)p.N - pb;
  const T* dg = reinterpret_cast<const T*>(p.delta) + c0 + pc;
  const T* og = reinterpret_cast<const T*>(p.dO) + c0 + pc;
  const T* zg = reinterpret_cast<const T*>(p.z) + c0 + pc;
  const T* cg = reinterpret_cast<const T*>(p.C) + g * p.N + pb;
  float bias[V];
#pragma unroll
  for (int e = 0; e < V; ++e) bias[e] = p.dbias && e < pleft ? p.dbias[c0 + pc + e] : 0.f;
  typename RowVec<T, V>::type rd, ro, rz;
  typename RowVec<T, VB>::type rc;
  bool in = false, inb = false;
  auto load_tile = [&](int k) {
    const int64_t t = t0 + k + r, tb = t0 + k + rb;
    in = k + r < end && (!p.map.seq || p.map.seq[t] >= 0);
    inb = k + rb < end && (!p.map.seq || p.map.seq[tb] >= 0);
    if (in) {
      load_raw<T, V>(dg + t * p.dts, pleft, rd);
      load_raw<T, V>(og + t * p.dos, pleft, ro);
      if (p.z) load_raw<T, V>(zg + t * p.zs, pleft, rz);
    }
    if (inb) load_raw<T, VB>(cg + tb * p.cs, bleft, rc);
  };
  const int k_last = (end - 1) / TT * TT;
  load_tile(k_last);
  for (int k = k_last; k >= 0; k -= TT) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool use = in && e < pleft;
      const float raw = to_f<T>(rd[e]) + bias[e], z = p.z ? to_f<T>(rz[e]) : 0.f;
      sD[r][pc + e] = use ? (p.softplus ? softplus_exact(raw) : raw) : 0.f;
      sG[r][pc + e] = use ? to_f<T>(ro[e]) * (p.z ? z * sigmoid_fast(z) : 1.f) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < VB; ++e) sC[rb][pb + e] = inb && e < bleft ? to_f<T>(rc[e]) : 0.f;
    __syncthreads();
    if (k >= TT) load_tile(k - TT);
#pragma unroll 1
    for (int i = TT - 4; i >= 0; i -= 4) {
      const float dv = sD[i + (q & 3)][ch], gv = sG[i + (q & 3)][ch];
      auto token = [&](auto J) {
        constexpr int j = decltype(J)::value;
        const float dj = quad_lane<j>(dv), gj = quad_lane<j>(gv);
#pragma unroll
        for (int n = 0; n < NS; ++n)
          dh[n] = __builtin_amdgcn_exp2f(dj * A2[n]) * __builtin_fmaf(gj, sC[i + j][n0 + n], dh[n]);
      };
      token(std::integral_constant<int, 3>());
      token(std::integral_constant<int, 2>());
      token(std::integral_constant<int, 1>());
      token(std::integral_constant<int, 0>());
    }
    __syncthreads();
  }
  if (live) store_piece<float, NS, true>(p.E + ((int64_t)chunk * p.D + c) * NP + n0, NS, dh);
}

template <typename T, typename SL>
__global__ __launch_bounds__(kThreads) void ssm_bwd_kernel(SsmParams p) {
  constexpr int NS = SL::NS, LPC = SL::LPC, NP = SL::NP, kRow = SL::kRow, TT = kSsmSub;
  constexpr int V = TT * SL::kCB / kThreads, kPer = SL::kCB / V;   // staging: channels a thread, threads a token
  constexpr int VB = TT * NP >= kThreads ? TT * NP / kThreads : 1, kPerB = NP / VB;
  typedef ChannelSums<SL> CS;
  __shared__ __attribute__((aligned(16))) float sD[TT][kRow], sX[TT][kRow], sG[TT][kRow];
  __shared__ __attribute__((aligned(16))) float sI[TT][kRow], sQ[TT][kRow], sY[TT][kRow];
  __shared__ __attribute__((aligned(16))) float sB[TT][NP], sC[TT][NP];
  __shared__ float sdB[kWaves][TT][NP], sdC[kWaves][TT][NP];

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
    if (base && seq >= 0) load_states<NS>(base + ((int64_t)seq * p.D + c) * p.N + n0, nleft, h);
    else
#pragma unroll
      for (int n = 0; n < NS; ++n) h[n] = 0.f;
  };
  // the gradient behind the chunk's last token
  int seq = p.map.seq_of(t0 + len - 1);
  if (p.map.seq ? t0 + len >= p.map.ntok || (p.map.start_bits(t0 + len) & 1u) : (t0 + len) % p.map.T == 0) {
    state_of(p.dhfin, seq, carry);
  } else {   // the chunks behind, up to the first that closes the sequence
    int cc = chunk + 1;
    while (!(p.flags[cc] & kClosed)) ++cc;
    load_states<NS>(p.E + ((int64_t)cc * p.D + c) * NP + n0, NS, carry);
    for (--cc; cc > chunk; --cc) {
      float s[NS];
      load_states<NS>(p.E + ((int64_t)cc * p.D + c) * NP + n0, NS, s);
      const float sum = p.sumd[(int64_t)cc * p.D + c];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const float back = carry[n] == 0.f ? 0.f : __builtin_amdgcn_exp2f(sum * A2[n]) * carry[n];
        carry[n] = back + s[n];
      }
    }
  }

  const int r = tid / kPer, pc = tid % kPer * V, pleft = nc - pc;
  const int rb = tid / kPerB, pb = tid % kPerB * VB, bleft = (int)p.N - pb;
  const T* ug = reinterpret_cast<const T*>(p.u) + c0 + pc;
  const T* dg = reinterpret_cast<const T*>(p.delta) + c0 + pc;
  const T* zg = reinterpret_cast<const T*>(p.z) + c0 + pc;
  const T* og = reinterpret_cast<const T*>(p.dO) + c0 + pc;
  const T* bg = reinterpret_cast<const T*>(p.B) + g * p.N + pb;
  const T* cg = reinterpret_cast<const T*>(p.C) + g * p.N + pb;
  float bias[V], skip[V], dskip[V], ddb[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    bias[e] = p.dbias && e < pleft ? p.dbias[c0 + pc + e] : 0.f;
    skip[e] = p.skip && e < pleft ? p.skip[c0 + pc + e] : 0.f;
    dskip[e] = ddb[e] = 0.f;
  }
  typename RowVec<T, V>::type ru, rd, rz, ro;
  typename RowVec<T, VB>::type rB, rC;
  float ck[NS];
  bool in = false, inb = false;
  auto load_tile = [&](int k) {
    const int64_t t = t0 + k + r, tb = t0 + k + rb;
    in = k + r < len && (!p.map.seq || p.map.seq[t] >= 0);
    inb = rb < TT && k + rb < len && (!p.map.seq || p.map.seq[tb] >= 0);
    if (in) {
      load_raw<T, V>(ug + t * p.us, pleft, ru);
      load_raw<T, V>(dg + t * p.dts, pleft, rd);
      load_raw<T, V>(og + t * p.dos, pleft, ro);
      if (p.z) load_raw<T, V>(zg + t * p.zs, pleft, rz);
    }
    if (inb) {
      load_raw<T, VB>(bg + tb * p.bs, bleft, rB);
      load_raw<T, VB>(cg + tb * p.cs, bleft, rC);
    }
    const int64_t sub = (int64_t)chunk * (p.L / kSsmSub) + k / kSsmSub;
    load_states<NS>(p.ck + (sub * p.D + c) * NP + n0, NS, ck);
  };
  const int k_last = (len - 1) / TT * TT;
  load_tile(k_last);
  for (int k = k_last; k >= 0; k -= TT) {
    // ---- these tokens into LDS ----
    float s[V], u[V], gy[V], o[V], z[V], slope[V];
    const bool here = in;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool use = here && e < pleft;
      const float raw = (use ? to_f<T>(rd[e]) : 0.f) + bias[e];
      u[e] = use ? to_f<T>(ru[e]) : 0.f;
      o[e] = use ? to_f<T>(ro[e]) : 0.f;
      z[e] = use && p.z ? to_f<T>(rz[e]) : 0.f;
      s[e] = use ? (p.softplus ? softplus_exact(raw) : raw) : 0.f;
      slope[e] = p.softplus ? sigmoid_fast(raw) : 1.f;
      gy[e] = p.z ? o[e] * (z[e] * sigmoid_fast(z[e])) : o[e];
      sD[r][pc + e] = s[e];
      sX[r][pc + e] = s[e] * u[e];
      sG[r][pc + e] = gy[e];
    }
    if (rb < TT)
#pragma unroll
      for (int e = 0; e < VB; ++e) {
        sB[rb][pb + e] = inb && e < bleft ? to_f<T>(rB[e]) : 0.f;
        sC[rb][pb + e] = inb && e < bleft ? to_f<T>(rC[e]) : 0.f;
      }
    float h[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = ck[n];
    __syncthreads();
    if (k >= TT) load_tile(k - TT);

    // ---- the states again ----
    const uint32_t valid = len - k >= TT ? (1u << TT) - 1u : (1u << (len - k)) - 1u;
    const uint32_t bits = p.map.start_bits(t0 + k) & valid;
    float a[TT][NS], ah[TT][NS];   // decays; decayed states a h_{t-1}
#pragma unroll
    for (int i = 0; i < TT; i += 4) {
      const float dv = sD[i + (q & 3)][ch], xv = sX[i + (q & 3)][ch];
      float y[4];
      auto token = [&](auto J) {
        constexpr int j = decltype(J)::value;
        if ((bits >> (i + j)) & 1u) state_of(p.h0, p.map.seq_of(t0 + k + i + j), h);
        const float dj = quad_lane<j>(dv), xj = quad_lane<j>(xv);
        float acc = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          a[i + j][n] = __builtin_amdgcn_exp2f(dj * A2[n]);
          ah[i + j][n] = a[i + j][n] * h[n];
          h[n] = __builtin_fmaf(xj, sB[i + j][n0 + n], ah[i + j][n]);
          acc = __builtin_fmaf(h[n], sC[i + j][n0 + n], acc);
        }
        y[j] = acc;
      };
      token(std::integral_constant<int, 0>());
      token(std::integral_constant<int, 1>());
      token(std::integral_constant<int, 2>());
      token(std::integral_constant<int, 3>());
      if (p.z) {
        const float yt = tokens_over_lanes<LPC>(y);
        if (q < 4) sY[i + q][ch] = yt;
      }
    }

    // ---- the reverse recurrence ----
#pragma unroll
    for (int i = TT - 4; i >= 0; i -= 4) {
      const float dv = sD[i + (q & 3)][ch], xv = sX[i + (q & 3)][ch], gv = sG[i + (q & 3)][ch];
      float into[4], qa[4], vB[4][NS], vC[4][NS];
      auto token = [&](auto J) {
        constexpr int j = decltype(J)::value;
        const float dj = quad_lane<j>(dv), xj = quad_lane<j>(xv), gj = quad_lane<j>(gv);
        float acc = 0.f, acq = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          const float b = sB[i + j][n0 + n], cc = sC[i + j][n0 + n];
          const float dh = __builtin_fmaf(gj, cc, carry[n]);
          const float qn = dh * ah[i + j][n];
          vC[j][n] = gj * __builtin_fmaf(xj, b, ah[i + j][n]);
          vB[j][n] = dh * xj;
          acc = __builtin_fmaf(dh, b, acc);
          acq = __builtin_fmaf(A2[n], qn, acq);
          dA[n] = __builtin_fmaf(dj, qn, dA[n]);
          carry[n] = dh * a[i + j][n];
        }
        into[j] = acc;
        qa[j] = acq;
        if ((bits >> (i + j)) & 1u) {   // a sequence's first token: what flows out is its initial state's
          const int64_t t = t0 + k + i + j;
          if (p.dh0 && live) {
            const int sq = p.map.seq_of(t);
            if (sq >= 0) store_piece<float, NS>(p.dh0 + ((int64_t)sq * p.D + c) * p.N + n0, nleft, carry);
          }
          state_of(p.dhfin, k + i + j > 0 ? p.map.seq_of(t - 1) : -1, carry);
        }
      };
      token(std::integral_constant<int, 3>());
      token(std::integral_constant<int, 2>());
      token(std::integral_constant<int, 1>());
      token(std::integral_constant<int, 0>());
      const float it = tokens_over_lanes<LPC>(into), qt = tokens_over_lanes<LPC>(qa);
      if (q < 4) {
        sI[i + q][ch] = it;
        sQ[i + q][ch] = qt;
      }
      float oB[CS::kKeep], oC[CS::kKeep];
      CS::run(vB, oB);
      CS::run(vC, oC);
#pragma unroll
      for (int n = 0; n < CS::kKeep; ++n) {
        sdB[wave][i + CS::tok()][n0 + CS::st() + n] = oB[n];
        sdC[wave][i + CS::tok()][n0 + CS::st() + n] = oC[n];
      }
    }
    __syncthreads();

    // ---- gradients of the activations ----
    if (k + r < len) {
      float du[V], dd[V], dz[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float into = sI[r][pc + e], ds = __builtin_fmaf(u[e], into, kLn2 * sQ[r][pc + e]);
        du[e] = __builtin_fmaf(s[e], into, skip[e] * gy[e]);
        dd[e] = ds * slope[e];
        float act;
        dz[e] = p.z ? o[e] * __builtin_fmaf(skip[e], u[e], sY[r][pc + e]) * silu_grad_f(z[e], act) : 0.f;
        if (!here) du[e] = dd[e] = dz[e] = 0.f;   // outside every sequence
        dskip[e] = __builtin_fmaf(gy[e], u[e], dskip[e]);
        ddb[e] += dd[e];
      }
      const int64_t at = (t0 + k + r) * p.D + c0 + pc;
      store_piece<T, V>(reinterpret_cast<T*>(p.du) + at, pleft, du);
      store_piece<T, V>(reinterpret_cast<T*>(p.ddelta) + at, pleft, dd);
      if (p.z) store_piece<T, V>(reinterpret_cast<T*>(p.dz) + at, pleft, dz);
    }
    for (int i = tid; i < TT * 2 * NP; i += kThreads) {
      const int t = i / (2 * NP), w = i / NP & 1, n = i % NP;
      if (k + t >= len || n >= p.N) continue;
      float v = 0.f;
#pragma unroll
      for (int m = 0; m < kWaves; ++m) v += w ? sdC[m][t][n] : sdB[m][t][n];
      p.pBC[(((int64_t)blk * p.map.ntok + t0 + k + t) * 2 + w) * p.N + n] = v;
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
  for (int i = tid; i < 2 * nc; i += kThreads) {
    const int w = i / nc, cc = i % nc;
    float v = 0.f;
#pragma unroll
    for (int t = 0; t < TT; ++t) v += w ? sX[t][cc] : sD[t][cc];
    p.pD[((int64_t)chunk * 2 + w) * p.D + c0 + cc] = v;
  }
}

// dB, dC [tokens][G][N] from the blocks' sums (in their order)
template <typename T>
__global__ __launch_bounds__(kThreads) void ssm_bc_kernel(SsmParams p) {
  const int64_t per = p.map.ntok * 2 * p.N, i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= per) return;
  const int64_t t = i / (2 * p.N);
  const int w = (int)(i / p.N & 1), n = (int)(i % p.N);
  T* out = reinterpret_cast<T*>(w ? p.dC : p.dB);
  for (int g = 0; g < p.G; ++g) {
    float v = 0.f;
    for (int b = 0; b < p.bpg; ++b) v += p.pBC[((int64_t)g * p.bpg + b) * per + i];
    out[(t * p.G + g) * p.N + n] = from_f<T>(v);
  }
}

template <typename T, typename SL> hipError_t backward(const SsmParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)(p.G * p.bpg * p.nchunk));
  if (p.map.seq ? p.nchunk > 1 : p.cps > 1) {
    hipLaunchKernelGGL((ssm_rev_kernel<T, SL>), grid, dim3(kThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((ssm_bwd_kernel<T, SL>), grid, dim3(kThreads), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t per = p.map.ntok * 2 * p.N;
  hipLaunchKernelGGL(ssm_bc_kernel<T>, dim3((uint32_t)((per + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, p);
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

// Selective scan, forward and single tokens (layout of the work: ssm.hpp).
//
//   s_t = softplus(delta_t + bias);  h_t = exp(s_t A) h_{t-1} + s_t u_t B_t
//   o_t = (C_t . h_t + skip u_t) z_t sigmoid(z_t)
//
// What bounds it is the vector ALU: 16 states are 16 (product, exponential, product,
// two multiply-adds) a token and channel, against 8 bytes of bf16 activations.
// Everything that is once per (token, channel) is kept out of the lanes that hold
// states: a tile of 32 tokens is staged by threads that own (token, piece of
// channels), which form the steps and s u for it and, after the scan, add the
// skip, gate and store.  exp(s A) is v_exp_f32 of s (A log2 e).
//
// 16384 tokens in 4 sequences x 4096 channels x 16 states, bf16: chunk summaries 161 us,
// scan 344 with the saved states, 87 and 77 % of the time with the vector ALUs at work, 5.5
// and 7.9 instructions a token, channel and state (counters; HBM: 0.8 GB, 0.15 ms).  16384
// tokens of one sequence x 2048 channels: 108 and 180.
#include "ssm.hpp"

namespace rla {

namespace {

template <typename T, typename SL, bool SUMMARY>
__global__ __launch_bounds__(SL::kThr) void ssm_fwd_kernel(SsmParams p) {
  constexpr int NS = SL::NS, LPC = SL::LPC, NP = SL::NP, kRow = SL::kRow, TT = kSsmTile;
  typedef SsmStage<T, SL, TT, SUMMARY ? kStU | kStB : kStU | kStZ | kStB | kStC> St;
  constexpr int V = St::V, VB = St::VB;
  __shared__ __attribute__((aligned(16))) float sD[TT][kRow], sX[TT][kRow], sY[SUMMARY ? 1 : TT][kRow];
  __shared__ __attribute__((aligned(16))) float sB[TT][NP], sC[SUMMARY ? 1 : TT][NP];

  const int tid = threadIdx.x;
  const int nblk = (int)p.G * p.bpg, turn = (int)blockIdx.x / nblk, blk = (int)blockIdx.x - turn * nblk;
  // (dense summaries: all but a sequence's last chunk)
  const int chunk = SUMMARY && !p.map.seq ? turn / (p.cps - 1) * p.cps + turn % (p.cps - 1) : turn;
  const int g = blk / p.bpg;
  const int64_t c0 = g * p.Dg + (int64_t)(blk - g * p.bpg) * SL::kCB;   // first channel
  const int nc = (int)min((int64_t)SL::kCB, (g + 1) * p.Dg - c0);
  int64_t t0;
  int len;
  chunk_range(p, chunk, t0, len);
  int last, first;
  chunk_starts(p, t0, len, last, first);
  if constexpr (SUMMARY) {
    if (blk == 0 && tid == 0 && p.map.seq) p.flags[chunk] = (last >= 0 ? kHasStart : 0) | (first <= len ? kClosed : 0);
    if (first == len || (p.map.seq && t0 + len >= p.map.ntok)) return;   // nothing continues behind it
    if (p.map.seq && first < len && p.map.start_bits(t0 + len) & 1u) return;
  }

  // the lane's channel and states
  const int q = SL::q(), ch = SL::ch(), n0 = q * NS;
  const bool live = ch < nc;
  const int64_t c = c0 + (live ? ch : 0);
  const int nleft = (int)p.N - n0;
  float A2[NS], h[NS];
  load_states<NS>(p.A + c * p.N + n0, nleft, A2);
#pragma unroll
  for (int n = 0; n < NS; ++n) A2[n] *= kLog2e;
  auto start_state = [&](int seq) {
    if (p.h0 && seq >= 0) {
      load_states<NS>(p.h0 + ((int64_t)seq * p.D + c) * p.N + n0, nleft, h);
      settle(h);   // here, and not in every tile's turn of the code that follows
    } else {
#pragma unroll
      for (int n = 0; n < NS; ++n) h[n] = 0.f;
    }
  };
  auto end_state = [&](int seq) {
    if (p.hfin && seq >= 0 && live) store_piece<float, NS>(p.hfin + ((int64_t)seq * p.D + c) * p.N + n0, nleft, h);
  };

  St st;
  const int r = St::r(), pc = St::pc(), rb = St::rb(), pb = St::pb(), pleft0 = nc - pc, bleft0 = (int)p.N - pb;
  const uint32_t fout = (r * (uint32_t)p.D + pc) * (uint32_t)sizeof(T);
  float bias[V], skip[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    bias[e] = p.dbias && e < pleft0 ? p.dbias[c0 + pc + e] : 0.f;
    skip[e] = p.skip && e < pleft0 ? p.skip[c0 + pc + e] : 0.f;
  }
  // tiles from the one of the last start on (summary), or all
  const int k_first = SUMMARY && last > 0 ? last / TT * TT : 0;
  int seq = p.map.seq || p.h0 || p.hfin ? p.map.seq_of(t0) : 0;
  if (SUMMARY) {
    if (last >= 0) seq = p.map.seq_of(t0 + last);
    start_state(last >= 0 ? seq : -1);
  } else if (last >= 0 && p.map.start_bits(t0) & 1u) {
    start_state(seq);
  } else {   // the chunks before, from the last one with a start on
    const int cc = p.map.seq ? find_chunk(p, chunk, kHasStart, false) : chunk / p.cps * p.cps;
    load_piece<float, NS, true>(p.S + ((int64_t)cc * p.D + c) * NP + n0, NS, h);
    carry_through<SL>(p, p.S, cc + 1, 1, chunk - 1 - cc, c, n0, A2, h);
  }
  float total = 0.f;   // sum of the channel's steps
  float* const ck = p.ck;

  settle(A2);
  settle(h);
  settle(bias);
  settle(skip);
  const bool packed = p.map.seq != nullptr, sp = p.softplus != 0;
  st.load(t0 + k_first, len - k_first, c0, g, nc);
  for (int k = k_first; k < len; k += TT) {
    even_pace(k / TT);
    // ---- this tile into LDS ----
    const uint32_t valid = len - k >= TT ? ~0u : (1u << (len - k)) - 1u;
    // (the chunk's first token, and dense chunks' only start: its state is set)
    uint32_t bits = SUMMARY || !packed ? 0u : fresh_map(fresh_args()).start_bits(t0 + k) & valid;
    if (k == 0) bits &= ~1u;
    const int pleft = fresh(pleft0), bleft = fresh(bleft0);
    const bool in = st.inside(k, len, packed);
    const typename St::Vec uu = st.u, zz = st.z;
    {
      float s[V];
      st.steps(bias, sp, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool use = in && e < pleft && (!SUMMARY || k + r >= last);
        sD[r][pc + e] = use ? s[e] : 0.f;
        sX[r][pc + e] = use ? s[e] * to_f<T>(st.u[e]) : 0.f;
      }
      if (st.owns_b()) {
        const bool inb = st.inside_b(k, len, packed) && (!SUMMARY || k + rb >= last);
#pragma unroll
        for (int e = 0; e < VB; ++e) {
          sB[rb][pb + e] = inb && e < bleft ? to_f<T>(st.b[e]) : 0.f;
          if (!SUMMARY) sC[rb][pb + e] = inb && e < bleft ? to_f<T>(st.c[e]) : 0.f;
        }
      }
    }
    __syncthreads();
    if (k + TT < len) st.load(t0 + k + TT, len - k - TT, c0, g, nc);

    // ---- the scan: four tokens at a time, the next four's values on their way ----
    struct Four {
      float d, x, b[4][NS], c[4][NS];
    };
    auto fetch = [&](int i, Four& f) {
      f.d = sD[i + (q & 3)][ch];
      f.x = sX[i + (q & 3)][ch];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          f.b[j][n] = sB[i + j][n0 + n];
          if (!SUMMARY) f.c[j][n] = sC[i + j][n0 + n];
        }
    };
    auto scan4 = [&](auto STARTS, int i, const Four& f) {
      if (!SUMMARY && ck && (i & (kSsmSub - 1)) == 0 && k + i < len && live) {
        const int64_t sub = (int64_t)chunk * (fresh_args()->L / kSsmSub) + (k + i) / kSsmSub;
        store_piece<float, NS, true>(ck + (sub * p.D + c) * NP + n0, NS, h);
      }
      if (SUMMARY) total += f.d;
      // in passes over the four tokens' states, each of independent instructions: one
      // wave then keeps the ALU busy through their latencies
      float e[4][NS], x[4][NS], y[4];
      over4([&](auto J) {
        constexpr int j = decltype(J)::value;
        const float dj = quad_lane<j>(f.d);
#pragma unroll
        for (int n = 0; n < NS; ++n) e[j][n] = dj * A2[n];
      });
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NS; ++n) e[j][n] = __builtin_amdgcn_exp2f(e[j][n]);
      over4([&](auto J) {
        constexpr int j = decltype(J)::value;
        const float xj = quad_lane<j>(f.x);
#pragma unroll
        for (int n = 0; n < NS; ++n) x[j][n] = xj * f.b[j][n];
      });
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (decltype(STARTS)::value && ((bits >> (i + j)) & 1u)) {
          end_state(seq);
          seq = p.map.seq_of(t0 + k + i + j);
          start_state(seq);
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) x[j][n] = h[n] = __builtin_fmaf(e[j][n], h[n], x[j][n]);
      }
      if (!SUMMARY) {
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = n == 0 ? x[j][n] * f.c[j][n] : __builtin_fmaf(x[j][n], f.c[j][n], y[j]);
        const float yt = tokens_over_lanes<LPC>(y);
        if (LPC == 4 || q < 4) sY[i + q][ch] = yt;
      }
    };
    if (bits == 0) {
      Four f[2];
      fetch(0, f[0]);
#pragma unroll
      for (int i = 0; i < TT; i += 4) {
        if (i + 4 < TT) fetch(i + 4, f[(i / 4 + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
        scan4(std::false_type(), i, f[(i / 4) & 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < TT; i += 4) {
        Four f;
        fetch(i, f);
        scan4(std::true_type(), i, f);
      }
    }
    st.settle();
    __syncthreads();

    // ---- skip, gate, store ----
    if (!SUMMARY && p.o && k + r < len) {   // (no outputs: the backward's recomputation)
      const SsmArgs a = fresh_args();
      const bool gated = a->z != nullptr;
      float y[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        y[e] = __builtin_fmaf(skip[e], to_f<T>(uu[e]), sY[r][pc + e]);
        if (gated) {
          const float zf = to_f<T>(zz[e]);
          y[e] *= zf * sigmoid_fast(zf);
        }
        if (!in) y[e] = 0.f;
      }
      store_piece<T, V>(at<T>(a->o, (t0 + k) * a->D + c0, fout), pleft, y);
    }
  }
  if constexpr (SUMMARY) {
    if (!live) return;
    store_piece<float, NS, true>(p.S + ((int64_t)chunk * p.D + c) * NP + n0, NS, h);
    total = group_sum<4>(total);   // the quad's lanes took a token of four each
    if (q == 0) p.sumd[(int64_t)chunk * p.D + c] = total;
  } else {
    // the last sequence ends with the chunk
    if (p.map.seq ? t0 + len >= p.map.ntok || (p.map.start_bits(t0 + len) & 1u) : (t0 + len) % p.map.T == 0)
      end_state(seq);
  }
}

// final (or, in the backward, initial) states of sequences without tokens
__global__ __launch_bounds__(kThreads) void ssm_empty_kernel(const int32_t* empty, int32_t nseq, int64_t row,
                                                             const float* from, float* to) {
  for (int64_t n = blockIdx.x; n < nseq; n += gridDim.x) {
    if (!empty[n]) continue;
    for (int64_t i = threadIdx.x; i < row; i += kThreads) to[n * row + i] = from ? from[n * row + i] : 0.f;
  }
}

// Single tokens.  A lane holds NS states of a channel of SEQS sequences through the
// call's tokens: the states are read and written once, which is what the call costs
// (HBM).  A workgroup's life is little more than one round of loads, so what is in
// flight bounds the rate: with one sequence a lane 4 KB a workgroup, 32 KB a CU.  Two
// sequences a lane from kPairWgs workgroups of one each: 4096 channels of 16 states,
// bf16, n sequences, time a call in us (states cold) with one / two / four a lane
//   n     16           32           64            128           256
//    5.0/5.0/6.0  7.5/6.3/6.8  12.7/10.5/9.3  21.8/18.1/17.3  39.0/32.6/35.0
// (256: 4.1 TB/s).  A call of pairs touches its states once: past the caches.
constexpr int64_t kPairWgs = 2048;
template <typename T, typename SL, int SEQS>
__global__ __launch_bounds__(SL::kThr) void ssm_decode_kernel(SsmParams p) {
  constexpr int NS = SL::NS, LPC = SL::LPC;
  typedef typename RowVec<float, NS>::type States;
  const int q = SL::q(), n0 = q * NS;
  const int64_t id = (int64_t)blockIdx.x * SL::kCB + SL::ch();   // (group of sequences, channel)
  const int64_t groups = (p.map.nseq + SEQS - 1) / SEQS;
  if (id >= groups * p.D) return;   // whole channels of lanes
  const int64_t s0 = (uint32_t)id / (uint32_t)p.D, c = id - s0 * p.D, g = (uint32_t)c / (uint32_t)p.Dg;
  const int nleft = (int)p.N - n0;
  auto seq = [&](int i) { return min(s0 * SEQS + i, (int64_t)p.map.nseq - 1); };   // past the last: the last, not stored
  float A2[NS], h[SEQS][NS];
#pragma unroll
  for (int i = 0; i < SEQS; ++i) {
    const float* from = p.h0 + (seq(i) * p.D + c) * p.N + n0;
    if (!p.h0) {
#pragma unroll
      for (int n = 0; n < NS; ++n) h[i][n] = 0.f;
    } else if (SEQS > 1 && p.N == SL::NP) {
      const States v = __builtin_nontemporal_load(reinterpret_cast<const States*>(from));
#pragma unroll
      for (int n = 0; n < NS; ++n) h[i][n] = v[n];
    } else {
      load_states<NS>(from, nleft, h[i]);
    }
  }
  load_states<NS>(p.A + c * p.N + n0, nleft, A2);
#pragma unroll
  for (int n = 0; n < NS; ++n) A2[n] *= kLog2e;
  const float bias = p.dbias ? p.dbias[c] : 0.f, skip = p.skip ? p.skip[c] : 0.f;
  for (int64_t k = 0; k < p.map.T; ++k) {
    T u[SEQS], d[SEQS], z[SEQS];
    typename RowVec<T, NS>::type b[SEQS], cc[SEQS];
#pragma unroll
    for (int i = 0; i < SEQS; ++i) {
      const int64_t t = seq(i) * p.map.T + k;
      u[i] = reinterpret_cast<const T*>(p.u)[t * p.us + c];
      d[i] = reinterpret_cast<const T*>(p.delta)[t * p.dts + c];
      z[i] = p.z ? reinterpret_cast<const T*>(p.z)[t * p.zs + c] : u[i];
      load_raw<T, NS>(reinterpret_cast<const T*>(p.B) + t * p.bs + g * p.N + n0, nleft, b[i]);
      load_raw<T, NS>(reinterpret_cast<const T*>(p.C) + t * p.cs + g * p.N + n0, nleft, cc[i]);
    }
#pragma unroll
    for (int i = 0; i < SEQS; ++i) {
      const float uf = to_f<T>(u[i]), raw = to_f<T>(d[i]) + bias, zf = to_f<T>(z[i]);
      const float step = p.softplus ? softplus_exact(raw) : raw, x = step * uf;
      float y = 0.f;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        h[i][n] = __builtin_fmaf(__builtin_amdgcn_exp2f(step * A2[n]), h[i][n], x * to_f<T>(b[i][n]));
        y = __builtin_fmaf(h[i][n], to_f<T>(cc[i][n]), y);
      }
      y = group_sum<LPC>(y);
      y = __builtin_fmaf(skip, uf, y);
      if (p.z) y *= zf * sigmoid_fast(zf);
      if (q == 0 && s0 * SEQS + i < p.map.nseq)
        reinterpret_cast<T*>(p.o)[((s0 * SEQS + i) * p.map.T + k) * p.D + c] = from_f<T>(y);
    }
  }
#pragma unroll
  for (int i = 0; i < SEQS; ++i) {
    if (s0 * SEQS + i >= p.map.nseq) break;
    float* to = p.hfin + ((s0 * SEQS + i) * p.D + c) * p.N + n0;
    if (SEQS > 1 && p.N == SL::NP) store_piece<float, NS, true, true>(to, NS, h[i]);
    else store_piece<float, NS>(to, nleft, h[i]);
  }
}

template <typename T, typename SL> hipError_t forward(const SsmParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)ssm_wgs(p));   // blocks of channels fastest: rows are contiguous
  if (p.cps > 1) {
    const dim3 part((uint32_t)(p.G * p.bpg * (p.map.seq ? p.nchunk : p.nchunk / p.cps * (p.cps - 1))));
    hipLaunchKernelGGL((ssm_fwd_kernel<T, SL, true>), part, dim3(SL::kThr), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((ssm_fwd_kernel<T, SL, false>), grid, dim3(SL::kThr), 0, stream, p);
  return hipGetLastError();
}
template <typename T, typename SL, int SEQS> hipError_t decode_run(const SsmParams& p, hipStream_t stream) {
  hipLaunchKernelGGL((ssm_decode_kernel<T, SL, SEQS>), dim3((uint32_t)ssm_decode_wgs(p)), dim3(SL::kThr), 0, stream, p);
  return hipGetLastError();
}
int decode_seqs(const SsmParams& p) { return p.map.nseq * p.D / ssm_channels(p.N) >= kPairWgs ? 2 : 1; }
template <typename T, typename SL> hipError_t decode(const SsmParams& p, hipStream_t stream) {
  return decode_seqs(p) == 2 ? decode_run<T, SL, 2>(p, stream) : decode_run<T, SL, 1>(p, stream);
}

template <typename T> hipError_t dispatch(const SsmParams& p, bool single, hipStream_t stream) {
  switch (ssm_padded(p.N)) {
    case 8: return single ? decode<T, SsmLanes<2, 4>>(p, stream) : forward<T, SsmLanes<2, 4>>(p, stream);
    case 16: return single ? decode<T, SsmLanes<4, 4>>(p, stream) : forward<T, SsmLanes<4, 4>>(p, stream);
    case 32: return single ? decode<T, SsmLanes<4, 8>>(p, stream) : forward<T, SsmLanes<4, 8>>(p, stream);
    default: return single ? decode<T, SsmLanes<4, 16>>(p, stream) : forward<T, SsmLanes<4, 16>>(p, stream);
  }
}

}  // namespace

int64_t ssm_decode_wgs(const SsmParams& p) {
  const int64_t seqs = decode_seqs(p), cb = ssm_channels(p.N);
  return ((p.map.nseq + seqs - 1) / seqs * p.D + cb - 1) / cb;
}
hipError_t launch_ssm_forward(const SsmParams& p, bool bf16, hipStream_t stream) {
  const hipError_t e = bf16 ? dispatch<u16>(p, false, stream) : dispatch<float>(p, false, stream);
  if (e != hipSuccess || !p.map.seq || !p.hfin) return e;
  return launch_ssm_empty(p, p.h0, p.hfin, stream);
}
hipError_t launch_ssm_empty(const SsmParams& p, const float* from, float* to, hipStream_t stream) {
  hipLaunchKernelGGL(ssm_empty_kernel, dim3(32), dim3(kThreads), 0, stream, p.map.empty, p.map.nseq, p.D * p.N, from, to);
  return hipGetLastError();
}
hipError_t launch_ssm_decode(const SsmParams& p, bool bf16, hipStream_t stream) {
  return bf16 ? dispatch<u16>(p, true, stream) : dispatch<float>(p, true, stream);
}

}  // namespace rla

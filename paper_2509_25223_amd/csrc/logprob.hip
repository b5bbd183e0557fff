// Log probabilities of rows of logits, z = scale x: lse = log sum e^z, z_y - lse for a
// row's token y, the entropy lse - sum p z, the `top` largest logits; and their
// gradient by the logits, scale (g (1[j = y] - p_j) - e p_j (z_j - lse + H)).
//
// A row is read once, into registers: with its largest value mx known, the sums are of
// 2^((x - mx) k), k = scale log2 e, and of these times (x - mx) k.  Taken as
// fma(x, k, -c) with c = mx k rounded, a value is two instructions; what c lost (one factor
// for the whole row) is taken out of the sums at the end.  A row longer than the registers of a
// workgroup hold, or one of few rows, is read in parts by several, each leaving its largest
// value, sums and alternatives, which logprob_join merges.
//
// Alternatives: values are compared as whole numbers in their order (0: none, -inf or NaN).
// Of 64 lanes' largest values the `top`-th is a bound that at least `top` values of
// the row reach; values from the bound on are collected in LDS and ranked by
// counting, (value, place) being different for each.  Where more reach the bound than LDS
// has room for (equal or neighbouring large logits), it is raised by bisection until exactly
// `top` do.
#include "model.hpp"

namespace rla {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kInf = __builtin_huge_valf();

// Ordered like the values; 0 for what can be no alternative.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0 equals 0)
  return x > -kInf ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0u;
}
__device__ __forceinline__ float from_order_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  v = group_sum<16>(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Over the L lanes of a row (64, or the workgroup); `slot`: LDS of its own for each use
// between two barriers.
template <int L, typename Op> __device__ __forceinline__ float over_waves(float v, float (&slot)[kWaves], Op op) {
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = op(op(slot[0], slot[1]), op(slot[2], slot[3]));
  }
  return v;
}
template <int L> __device__ __forceinline__ void row_barrier() {
  if constexpr (L > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// The `want`-th largest of the 64 lanes' keys, or 0 if fewer are not 0.
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t key, int want) {
  uint32_t t = 0;
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
    if (__popcll(__ballot(key >= (t | bit))) >= want) t |= bit;
  return t;
}

struct Candidate {
  uint32_t key;
  int32_t at;
};
template <int L> constexpr int kRoom = L > 64 ? 256 : 128;

template <int L> struct TopLds {
  uint32_t bound[kWaves];
  int32_t count, sums[2][kWaves];
  Candidate list[kRoom<L>];
};

// Sum over a row's lanes of a whole number.
template <int L> __device__ __forceinline__ int row_count(int c, TopLds<L>& s, int turn) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) c += __shfl_xor(c, d);
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) s.sums[turn & 1][threadIdx.x >> 6] = c;
    __syncthreads();
    c = s.sums[turn & 1][0] + s.sums[turn & 1][1] + s.sums[turn & 1][2] + s.sums[turn & 1][3];
  }
  return c;
}

// The largest `want` of the values that for_each(f) hands to f(key, place), place by place the same
// each time; out(rank, key, place) for each.  A row's L lanes call it together.
template <int L, typename Each, typename Out>
__device__ __forceinline__ void select_top(int want, TopLds<L>& s, Each for_each, Out out) {
  const int lane = threadIdx.x & 63, w = L > 64 ? threadIdx.x >> 6 : 0;
  uint32_t best = 0;
  for_each([&](uint32_t k, int) { best = max(best, k); });
  uint32_t bound = kth_of_lanes(best, want);
  if (lane == 0) s.bound[w] = bound;
  if (threadIdx.x % L == 0) s.count = 0;
  row_barrier<L>();
  if constexpr (L > 64) bound = max(max(s.bound[0], s.bound[1]), max(s.bound[2], s.bound[3]));
  bound = max(bound, 1u);
  int turn = 0;
  auto reach = [&](uint32_t t) {
    int c = 0;
    for_each([&](uint32_t k, int) { c += k >= t ? 1 : 0; });
    return row_count<L>(c, s, turn++);
  };
  int32_t last = 0x7fffffff;   // of the values equal to the bound, those up to this place
  if (reach(bound) > kRoom<L>) {
    // the largest bound that `want` values reach, then the place that leaves `want`
    uint32_t t = 0;
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
      if (reach(t | bit) >= want) t |= bit;
    bound = t;
    const int above = t == 0xffffffffu ? 0 : reach(t + 1);
    int32_t place = 0;   // fewer than want - above equal values lie before it
    for (int32_t bit = 1 << 30; bit; bit >>= 1) {
      int c = 0;
      const int32_t upto = place | bit;
      for_each([&](uint32_t k, int at) { c += k == t && at < upto ? 1 : 0; });
      if (row_count<L>(c, s, turn++) < want - above) place = upto;
    }
    last = place;
  }
  for_each([&](uint32_t k, int at) {
    if (k > bound || (k == bound && at <= last)) {
      const int j = atomicAdd(&s.count, 1);
      s.list[j] = Candidate{k, at};
    }
  });
  row_barrier<L>();
  const int count = s.count;
  for (int j = threadIdx.x % L; j < count; j += L) {
    const Candidate own = s.list[j];
    int rank = 0;
    for (int i = 0; i < count; ++i) {
      const Candidate c = s.list[i];
      rank += c.key > own.key || (c.key == own.key && c.at < own.at) ? 1 : 0;
    }
    if (rank < want) out(rank, own.key, own.at);
  }
  for (int j = count + threadIdx.x % L; j < want; j += L) out(j, 0u, -1);
}

// A row's outputs from its largest value mx, s = sum e^(z - z_max) and e = sum of these times
// (x - mx) k.
struct RowResult {
  float mx, ln;   // ln s
  bool none;      // nothing but -inf
  float scale;
  __device__ __forceinline__ RowResult(float mx_, float s, float scale_)
      : mx(mx_), ln(logf(s)), none(s == 0.f), scale(scale_) {}
  __device__ __forceinline__ float of(float x) const { return none ? -kInf : (x - mx) * scale - ln; }
  __device__ __forceinline__ float lse() const { return none ? -kInf : mx * scale + ln; }
  __device__ __forceinline__ float entropy(float s, float e) const { return none ? 0.f : ln - kLn2 * (e / s); }
};

// What one lane writes of a row.
template <typename T>
__device__ __forceinline__ void write_row(const LogprobParams& p, int64_t row, const RowResult& r, float s, float e) {
  if (p.lse) p.lse[row] = r.lse();
  if (p.entropy) p.entropy[row] = r.entropy(s, e);
  if (p.logprob) {
    const int64_t y = p.targets[row];
    p.logprob[row] = y >= 0 && y < p.V ? r.of(to_f<T>(reinterpret_cast<const T*>(p.x)[row * p.xs + y])) : 0.f;
  }
}

// ---------------------------------------------------------------------------
// L lanes a part of a row, N pieces a lane.  Part: row / part = id / p.parts, id % p.parts.
// ---------------------------------------------------------------------------
template <typename T, int L, int N, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_fwd_kernel(LogprobParams p, int64_t first) {
  constexpr int V = kPiece<T>, kSub = kThreads / L;
  __shared__ float slots[3][kWaves];
  __shared__ TopLds<L> top[TOP ? kSub : 1];
  const int64_t id = first + (int64_t)blockIdx.x * kSub + threadIdx.x / L;
  if (id >= p.n * p.parts) return;   // (whole rows of lanes)
  const int64_t row = id / p.parts, part = id - row * p.parts;
  const int64_t c0 = part * p.width;
  const int width = (int)min(p.width, p.V - c0);
  const T* x = reinterpret_cast<const T*>(p.x) + row * p.xs + c0;
  const int lane = threadIdx.x % L;

  typename RowVec<T, V>::type raw[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = (j * L + lane) * V, left = width - c;
    if (left >= V) {
      raw[j] = *reinterpret_cast<const typename RowVec<T, V>::type*>(x + c);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) raw[j][e] = e < left ? x[c + e] : from_f<T>(-kInf);
    }
  }
  float mx = -kInf;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) mx = fmaxf(mx, to_f<T>(raw[j][e]));
  mx = over_waves<L>(wave_max(mx), slots[0], [](float a, float b) { return fmaxf(a, b); });
  const float k = p.scale * kLog2e, m0 = mx == -kInf ? 0.f : mx, c = m0 * k;
  float s = 0.f, ent = 0.f;
  auto add = [&](float d) {
    const float y = __builtin_amdgcn_exp2f(d);
    s += y;
    ent = __builtin_fmaf(y, fmaxf(d, -1000.f), ent);   // (0 times -inf)
  };
  if (__builtin_fabsf(c) > 1e30f) {   // c could overflow (a row at the type's lowest value)
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) add((to_f<T>(raw[j][e]) - m0) * k);
  } else if (p.entropy) {
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) add(__builtin_fmaf(to_f<T>(raw[j][e]), k, -c));
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) s += __builtin_amdgcn_exp2f(__builtin_fmaf(to_f<T>(raw[j][e]), k, -c));
  }
  if (p.entropy) ent = over_waves<L>(wave_sum(ent), slots[2], [](float a, float b) { return a + b; });
  s = over_waves<L>(wave_sum(s), slots[1], [](float a, float b) { return a + b; });
  if (__builtin_fabsf(c) <= 1e30f) {   // the factor 2^(mx k - c) out of the sums
    const float lost = __builtin_fmaf(m0, k, -c), f = __builtin_amdgcn_exp2f(-lost);
    ent = (ent - lost * s) * f;
    s *= f;
  }
  const RowResult r(m0, s, p.scale);
  if (p.parts == 1) {
    if (lane == 0) write_row<T>(p, row, r, s, ent);
  } else if (lane == 0) {
    *reinterpret_cast<floatx4*>(p.stat + id * 4) = floatx4{mx, s, ent, 0.f};
  }
  if constexpr (TOP) {
    auto each = [&](auto&& f) {
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) f(order_key(to_f<T>(raw[j][e])), (j * L + lane) * V + e);
    };
    const int want = min(p.top, width);
    const int64_t base = id * p.top;
    select_top<L>(want, top[threadIdx.x / L], each, [&](int rank, uint32_t key, int at) {
      if (p.parts == 1) {
        p.top_lp[base + rank] = key ? r.of(from_order_key(key)) : r.ln == r.ln ? -kInf : r.ln;
        p.top_ids[base + rank] = key ? at : -1;
      } else {
        p.cand_x[base + rank] = key ? from_order_key(key) : -kInf;
        p.cand_i[base + rank] = key ? (int)c0 + at : -1;
      }
    });
    if (p.parts > 1)   // (a last part narrower than `top`)
      for (int j = want + lane; j < p.top; j += L) {
        p.cand_x[base + j] = -kInf;
        p.cand_i[base + j] = -1;
      }
  }
}

// A wave a row: its parts merged.
template <typename T, bool TOP> __global__ __launch_bounds__(kThreads) void logprob_join_kernel(LogprobParams p) {
  __shared__ TopLds<64> top[TOP ? kWaves : 1];
  const int64_t row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (row >= p.n) return;
  const int lane = threadIdx.x & 63;
  const float k = p.scale * kLog2e;
  float mx = -kInf, s = 0.f, e = 0.f;
  for (int64_t j = lane; j < p.parts; j += 64) mx = fmaxf(mx, p.stat[(row * p.parts + j) * 4]);
  mx = wave_max(mx);
  const float m0 = mx == -kInf ? 0.f : mx;
  for (int64_t j = lane; j < p.parts; j += 64) {
    const floatx4 t = *reinterpret_cast<const floatx4*>(p.stat + (row * p.parts + j) * 4);
    const float d = t[0] == -kInf ? -1000.f : (t[0] - m0) * k, f = __builtin_amdgcn_exp2f(d);
    s = __builtin_fmaf(t[1], f, s);
    e = __builtin_fmaf(__builtin_fmaf(t[1], fmaxf(d, -1000.f), t[2]), f, e);
  }
  s = wave_sum(s);
  e = wave_sum(e);
  const RowResult r(m0, s, p.scale);
  if (lane == 0) write_row<T>(p, row, r, s, e);
  if constexpr (TOP) {
    const int64_t count = p.parts * p.top;
    auto each = [&](auto&& f) {
      for (int64_t j = lane; j < count; j += 64) {
        const int32_t at = p.cand_i[row * count + j];
        f(at < 0 ? 0u : order_key(p.cand_x[row * count + j]), at);
      }
    };
    select_top<64>(p.top, top[threadIdx.x >> 6], each, [&](int rank, uint32_t key, int at) {
      p.top_lp[row * p.top + rank] = key ? r.of(from_order_key(key)) : r.ln == r.ln ? -kInf : r.ln;
      p.top_ids[row * p.top + rank] = key ? at : -1;
    });
  }
}

// ---------------------------------------------------------------------------
// Gradient: L lanes a row, or N pieces a lane of one
// ---------------------------------------------------------------------------
// The log probability z - lse is off by half a step of lse: 1.5e-5 at 256.  Rows farther out
// (large logits, a row at the type's lowest value) are read once more for their largest value and
// the logarithm of the sum beside it.
constexpr float kFarLse = 256.f;
template <typename T, int L> __device__ __forceinline__ void far_row(const LogprobParams& p, const T* x, float& mx, float& ln) {
  __shared__ float slots[2][kWaves];
  const float k = p.scale * kLog2e;
  float m = -kInf, s = 0.f;
  for (int64_t j = threadIdx.x % L; j < p.V; j += L) m = fmaxf(m, to_f<T>(x[j]));
  m = over_waves<L>(wave_max(m), slots[0], [](float a, float b) { return fmaxf(a, b); });
  for (int64_t j = threadIdx.x % L; j < p.V; j += L) s += __builtin_amdgcn_exp2f((to_f<T>(x[j]) - m) * k);
  s = over_waves<L>(wave_sum(s), slots[1], [](float a, float b) { return a + b; });
  mx = m;
  ln = logf(s);
}

template <typename T, int L, int N, bool NT>
__global__ __launch_bounds__(kThreads) void logprob_bwd_kernel(LogprobParams p, int64_t first, uint32_t segs) {
  constexpr int V = kPiece<T>, kSub = kThreads / L;
  const int64_t id = first + (int64_t)blockIdx.x * kSub + threadIdx.x / L;
  const int64_t row = id / segs;
  if (row >= p.n) return;
  const int64_t c0 = (id - row * segs) * (L * N * V) + (threadIdx.x % L) * V;
  const T* x = reinterpret_cast<const T*>(p.x) + row * p.xs;
  T* dx = reinterpret_cast<T*>(p.dx) + row * p.V;
  float in[N][V];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int64_t c = c0 + j * (L * V);
    load_piece<T, V>(x + c, (int)min(p.V - c, (int64_t)V), in[j]);
  }
  const float lse = p.lse_in[row];
  int64_t y = -1;
  float g = 0.f, de = 0.f, H = 0.f;
  if (p.dlogprob) {
    y = p.targets[row];
    if (y >= 0 && y < p.V) g = p.dlogprob[row];
    else y = -1;
  }
  if (p.dentropy) {
    de = p.dentropy[row];
    H = p.entropy_in[row];
  }
  const bool none = lse == -kInf;
  float mx = 0.f, ln = lse;
  if (__builtin_fabsf(lse) > kFarLse && __builtin_fabsf(lse) < kInf) far_row<T, L>(p, x, mx, ln);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int64_t c = c0 + j * (L * V);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = __builtin_fmaf(in[j][e] - mx, p.scale, -ln);   // log p
      const float pr = __builtin_amdgcn_exp2f(d * kLog2e);
      float t = -pr * __builtin_fmaf(de, fmaxf(d, -1000.f) + H, g);
      if (c + e == y) t += g;
      in[j][e] = none ? 0.f : t * p.scale;
    }
    store_piece<T, V, false, NT>(dx + c, (int)min(p.V - c, (int64_t)V), in[j]);
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
constexpr int64_t kMaxGrid = (int64_t)1 << 23;   // workgroups a launch

template <typename T, int L, int N> hipError_t forward(const LogprobParams& p, hipStream_t stream) {
  const int64_t sub = kThreads / L, wgs = (p.n * p.parts + sub - 1) / sub;
  for (int64_t w = 0; w < wgs; w += kMaxGrid) {
    const dim3 grid((uint32_t)min(wgs - w, kMaxGrid));
    if (p.top) hipLaunchKernelGGL((logprob_fwd_kernel<T, L, N, true>), grid, dim3(kThreads), 0, stream, p, w * sub);
    else hipLaunchKernelGGL((logprob_fwd_kernel<T, L, N, false>), grid, dim3(kThreads), 0, stream, p, w * sub);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// Values in a lane's registers: 64 at most.
template <typename T> hipError_t forward(const LogprobParams& p, hipStream_t stream) {
  constexpr int V = kPiece<T>;
  const int64_t pieces = (p.width + V - 1) / V;
  hipError_t e;
  if (pieces <= 64) e = forward<T, 64, 1>(p, stream);
  else if (pieces <= 128) e = forward<T, 64, 2>(p, stream);
  else if (pieces <= 256) e = forward<T, 256, 1>(p, stream);
  else if (pieces <= 512) e = forward<T, 256, 2>(p, stream);
  else if (pieces <= 1024) e = forward<T, 256, 4>(p, stream);
  else if (V == 8 || pieces <= 2048) e = forward<T, 256, 8>(p, stream);
  else e = forward<T, 256, 64 / V>(p, stream);
  if (e != hipSuccess || p.parts == 1) return e;
  const dim3 grid((uint32_t)((p.n + kWaves - 1) / kWaves));
  if (p.top) hipLaunchKernelGGL((logprob_join_kernel<T, true>), grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((logprob_join_kernel<T, false>), grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template <typename T, int L, int N> hipError_t backward(const LogprobParams& p, hipStream_t stream) {
  constexpr int V = kPiece<T>;
  const int64_t sub = kThreads / L, segs = (p.V + L * N * V - 1) / (L * N * V), wgs = (p.n * segs + sub - 1) / sub;
  const bool nt = p.n * p.V * (int64_t)sizeof(T) > kNtBytes;
  for (int64_t w = 0; w < wgs; w += kMaxGrid) {
    const dim3 grid((uint32_t)min(wgs - w, kMaxGrid));
    if (nt) hipLaunchKernelGGL((logprob_bwd_kernel<T, L, N, true>), grid, dim3(kThreads), 0, stream, p, w * sub, (uint32_t)segs);
    else hipLaunchKernelGGL((logprob_bwd_kernel<T, L, N, false>), grid, dim3(kThreads), 0, stream, p, w * sub, (uint32_t)segs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename T> hipError_t backward(const LogprobParams& p, hipStream_t stream) {
  const int64_t pieces = (p.V + kPiece<T> - 1) / kPiece<T>;
  return pieces <= 128 ? backward<T, 64, 1>(p, stream) : backward<T, 256, 4>(p, stream);
}

}  // namespace

size_t logprob_plan(LogprobParams& p, bool bf16, unsigned char* ws) {
  const int64_t most = 64 * kThreads, piece = bf16 ? 8 : 4;   // values that a workgroup holds
  constexpr int64_t fill = 1024, least = 1024;                // workgroups, values a part
  int64_t parts = (p.V + most - 1) / most;
  if (p.n * parts < fill) parts = max(parts, min(min((fill + p.n - 1) / max(p.n, (int64_t)1), p.V / least), (int64_t)64));
  p.width = ((p.V + parts - 1) / parts + piece - 1) / piece * piece;
  p.parts = (p.V + p.width - 1) / p.width;
  if (p.parts == 1) return 0;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* at = ws + off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  const size_t all = (size_t)p.n * (size_t)p.parts;
  p.stat = reinterpret_cast<float*>(take(16 * all));
  p.cand_x = reinterpret_cast<float*>(take(4 * all * (size_t)p.top));
  p.cand_i = reinterpret_cast<int32_t*>(take(4 * all * (size_t)p.top));
  return off;
}

hipError_t launch_logprob_forward(const LogprobParams& p, bool bf16, hipStream_t stream) {
  return bf16 ? forward<u16>(p, stream) : forward<float>(p, stream);
}
hipError_t launch_logprob_backward(const LogprobParams& p, bool bf16, hipStream_t stream) {
  return bf16 ? backward<u16>(p, stream) : backward<float>(p, stream);
}

}  // namespace rla

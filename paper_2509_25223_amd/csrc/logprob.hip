// Log probabilities of rows of logits, z = scale x: lse = log sum e^z, z_y - lse for a
// row's token y, the entropy lse - sum p z, the `top` largest logits; and their
// gradient by the logits, scale (g (1[j = y] - p_j) - e p_j (z_j - lse + H)).
//
// A row is read once, into registers: with its largest value mx known, the sums are of 2^((x - mx) k),
// k = scale log2 e, and of these times (x - mx) k.  A row longer than the registers of a
// workgroup hold, or one of few rows, is read in parts by several, each leaving its largest
// value, sums and alternatives, which logprob_join merges.  Many rows are bound by HBM and the vector ALU
// (16384 x 32768 of bf16: 176 us for 1.07 GB, 6.1 TB/s, the ALUs at work 93 % of the time; 4001 x 50001 96 us, 4.2 TB/s,
// 106 with five alternatives), few by latency (one of 32768 in fp32 with twenty alternatives: 10.1 us; 64 of
// 131072 with eight: 10.9, and 6.2 to join them).  All sums are fp32, in one order.
//
// Alternatives: values are compared as whole numbers in their order (0: none, -inf or NaN).
// Of a wave's 64 lanes' largest values the q-th is a bound that q values of the wave reach (its upper
// 16 bits are enough), and the r-th of the waves' bounds one that q r >= `top` values of the row do;
// values from the bound on are collected in LDS by the few lanes whose largest reaches it, and
// ranked by counting, (value, place) being different for each.  Where more reach the bound than LDS
// has room for, the row is read again: first with the largest of the waves' `top`-th lanes as the bound
// (a few hundred neighbouring tokens allowed), then, if that does not do (equal large logits), by
// bisection until exactly `top` reach it (64 rows of 131072, eight alternatives: 16 us; 500 allowed
// tokens in each 30; all equal 135).
//
// The gradient recomputes p from lse, and holds a row in the same way (below).
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
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  v = fmaxf(v, dpp<0x140>(v));
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = group_sum<16>(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Barrier of a row's L lanes (64, or the workgroup).
template <int L> __device__ __forceinline__ void row_barrier() {
  if constexpr (L > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}
template <int N, typename Op> __device__ __forceinline__ float over(const float (&x)[N], Op op) {
  float v = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) v = op(v, x[i]);
  return v;
}
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };

// A bound, in the upper 16 bits of a key, that `want` of the 64 lanes' keys reach; 0 if fewer are
// not 0.
__device__ __forceinline__ uint32_t bound_of_lanes(uint32_t key, int want) {
  uint32_t t = 0;
  for (uint32_t bit = 0x80000000u; bit > 0xffffu; bit >>= 1)
    if (__popcll(__ballot(key >= (t | bit))) >= want) t |= bit;
  return t;
}
constexpr uint32_t kLowestKey = 0x00800000u;   // of the lowest finite value

struct Candidate {
  uint32_t key;
  int32_t at;
};
template <int L> constexpr int kRoom = L > 64 ? 256 : 128;

template <int L> struct TopLds {
  uint32_t bound[L / 64];   // of each wave
  int32_t count, sums[2][L / 64];
  Candidate list[kRoom<L>];
};

// Sum over a row's lanes of a whole number.
template <int L> __device__ __forceinline__ int row_count(int c, TopLds<L>& s, int turn) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) c += __shfl_xor(c, d);
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) s.sums[turn & 1][threadIdx.x >> 6] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < L / 64; ++w) c += s.sums[turn & 1][w];
  }
  return c;
}
template <int L> __device__ __forceinline__ void collect(TopLds<L>& s, uint32_t key, int at) {
  const int j = atomicAdd(&s.count, 1);
  if (j < kRoom<L>) s.list[j] = Candidate{key, at};
}

// More than fit were collected: anew, from the largest of the waves' own bounds on, if a wave has `want`
// lanes of values (a mask that leaves a stretch of tokens; `own`: the lane's largest key).
template <int L, typename Each>
__device__ __forceinline__ void collect_stretch(int want, uint32_t own, TopLds<L>& s, Each for_each) {
  const uint32_t wave = bound_of_lanes(own, want);
  __syncthreads();   // (all have read the count)
  if ((threadIdx.x & 63) == 0) s.bound[threadIdx.x >> 6] = wave;
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  uint32_t bound = kLowestKey;
#pragma unroll
  for (int w = 0; w < L / 64; ++w) bound = max(bound, s.bound[w]);
  for_each([&](uint32_t k, int at) {
    if (k >= bound) collect(s, k, at);
  });
  __syncthreads();
}

// Still more: the largest bound that `want` values reach (the row's largest key `most`, if that many
// equal it), of the values equal to it those up to the place that leaves `want`, collected anew.
// for_each(f) hands all of the lane's (key, place < places) to f.
template <int L, typename Each>
__device__ __forceinline__ void collect_exactly(int want, uint32_t most, int places, TopLds<L>& s, Each for_each) {
  int turn = 0;
  auto reach = [&](uint32_t t) {
    int c = 0;
    for_each([&](uint32_t k, int) { c += k >= t ? 1 : 0; });
    return row_count<L>(c, s, turn++);
  };
  uint32_t t = most;
  int above = 0;
  if (reach(most) < want) {
    t = 0;
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
      if (reach(t | bit) >= want) t |= bit;
    above = reach(t + 1);
  }
  int32_t last = 0;   // fewer than want - above equal values lie before it
  for (int32_t bit = 1 << (31 - __builtin_clz(places)); bit; bit >>= 1) {
    int c = 0;
    const int32_t upto = last | bit;
    for_each([&](uint32_t k, int at) { c += k == t && at < upto ? 1 : 0; });
    if (row_count<L>(c, s, turn++) < want - above) last = upto;
  }
  if (threadIdx.x % L == 0) s.count = 0;
  row_barrier<L>();
  for_each([&](uint32_t k, int at) {
    if (k > t || (k == t && at <= last)) collect(s, k, at);
  });
  row_barrier<L>();
}

// out(rank, key, place) of the collected ones' largest `want` (key 0, place -1 past the last).
template <int L, typename Out> __device__ __forceinline__ void rank_collected(int want, const TopLds<L>& s, Out out) {
  const int count = s.count;
  for (int j = threadIdx.x % L; j < count; j += L) {
    const Candidate own = s.list[j];
    int rank = 0;
#pragma unroll 8
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

// The lane's values of a part, as stored: N pieces of V, piece j of lane l from column (j L + l) V on,
// -inf past its end.
template <typename T, int L, int N> struct Part {
  static constexpr int V = kPiece<T>;
  typedef typename RowVec<T, V>::type Vec;
  Vec raw[N];
  __device__ __forceinline__ static int col(int j, int lane) { return (j * L + lane) * V; }
  // Whole pieces without branches, so that all are in flight at once (past the end the last
  // one again), then what is not whole.
  __device__ __forceinline__ void load(const T* x, int width, int lane) {
    if (width >= V)
#pragma unroll
      for (int j = 0; j < N; ++j) raw[j] = *reinterpret_cast<const Vec*>(x + min(col(j, lane), width - V));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (width >= (j + 1) * L * V) continue;
      const int c = col(j, lane), left = width - c;
      if (left >= V) continue;
#pragma unroll
      for (int e = 0; e < V; ++e) raw[j][e] = e < left ? x[c + e] : from_f<T>(-kInf);
    }
  }
  // Before each pass: values are converted anew, kept they would take twice the registers.
  __device__ __forceinline__ void again() {
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      Words w = __builtin_bit_cast(Words, raw[j]);
      asm volatile("" : "+v"(w));
      raw[j] = __builtin_bit_cast(Vec, w);
    }
  }
  template <typename F> __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) f(j, e, to_f<T>(raw[j][e]));
  }
};

// The logit of a row's token (`there`: it has one).
template <typename T> __device__ __forceinline__ float given_logit(const LogprobParams& p, int64_t row, bool& there) {
  const int64_t y = p.targets[row];
  there = y >= 0 && y < p.V;
  return there ? to_f<T>(reinterpret_cast<const T*>(p.x)[row * p.xs + y]) : 0.f;
}
// What one lane writes of a row.
__device__ __forceinline__ void write_row(const LogprobParams& p, int64_t row, const RowResult& r, float s, float e, float given,
                                          bool there) {
  if (p.lse) p.lse[row] = r.lse();
  if (p.entropy) p.entropy[row] = r.entropy(s, e);
  if (p.logprob) p.logprob[row] = there ? r.of(given) : 0.f;
}

// ---------------------------------------------------------------------------
// L lanes a part of a row, N pieces a lane.  Part: row / part = id / p.parts, id % p.parts.
// ---------------------------------------------------------------------------
// (1024 lanes, up to 7 pieces: in 64 registers, for two rows on a CU)
template <typename T, int L, int N, bool TOP>
__global__ __launch_bounds__(L > kThreads ? L : kThreads, !TOP && L == 1024 && N <= 7 ? 8 : 1)
void logprob_fwd_kernel(LogprobParams p, int64_t first) {
  constexpr int V = kPiece<T>, kSub = L > kThreads ? 1 : kThreads / L, W = L / 64;
  __shared__ float slots[3][kSub][W];
  __shared__ TopLds<L> tops[TOP ? kSub : 1];
  const int sub = L > 64 ? 0 : threadIdx.x / L, w = L > 64 ? threadIdx.x >> 6 : 0, lane = threadIdx.x % L;
  const int64_t id = first + (int64_t)blockIdx.x * kSub + threadIdx.x / L;
  if (id >= p.n * p.parts) return;   // (whole rows of lanes)
  TopLds<L>& top = tops[TOP ? sub : 0];
  const int64_t row = p.parts == 1 ? id : id / p.parts, part = id - row * p.parts;
  const int64_t c0 = part * p.width;
  const int width = (int)min(p.width, p.V - c0), want = TOP ? min(p.top, width) : 0;
  const T* x = reinterpret_cast<const T*>(p.x) + row * p.xs + c0;

  Part<T, L, N> v;
  v.load(x, width, lane);
  float given = 0.f;
  bool there = false;
  if (p.logprob && p.parts == 1 && lane == 0) given = given_logit<T>(p, row, there);

  float own = -kInf;   // the lane's largest
  v.each([&](int, int, float z) { own = fmaxf(own, z); });
  float mx = wave_max(own);
  // (a wave's q-th; the workgroup's: the r-th of its waves', so that r waves have q each)
  const int q = (want + max(W / 2, 1) - 1) / max(W / 2, 1);
  uint32_t bound = 0;
  if constexpr (TOP) bound = bound_of_lanes(order_key(own), q);
  if ((threadIdx.x & 63) == 0) {
    slots[0][sub][w] = mx;
    if (TOP) top.bound[w] = bound;
  }
  if (TOP && lane == 0) top.count = 0;
  row_barrier<L>();
  if constexpr (L > 64) {
    mx = over(slots[0][0], Max());
    if constexpr (TOP) bound = bound_of_lanes((threadIdx.x & 63) < W ? top.bound[threadIdx.x & (W - 1)] : 0u, (want + q - 1) / q);
  }

  if constexpr (TOP) {
    const float least = from_order_key(max(bound, kLowestKey));
    v.again();
    if (own >= least) {
      int at = lane * V;   // (computed here: kept from the loads, the pieces' columns take registers)
      asm volatile("" : "+v"(at));
      v.each([&](int j, int e, float z) {
        if (z >= least) collect(top, order_key(z), at + j * (L * V) + e);
      });
    }
  }
  // (the difference first: mx k alone could overflow, in a row at the type's lowest value)
  const float k = p.scale * kLog2e, m0 = mx == -kInf ? 0.f : mx;
  float s = 0.f, ent = 0.f;
  if (p.entropy) {
    v.again();
    v.each([&](int, int, float z) {
      const float d = (z - m0) * k, y = __builtin_amdgcn_exp2f(d);
      s += y;
      ent = __builtin_fmaf(y, fmaxf(d, -1000.f), ent);   // (0 times -inf)
    });
  } else {
    v.again();   // (in each branch: what both convert would be taken out of them)
    v.each([&](int, int, float z) { s += __builtin_amdgcn_exp2f((z - m0) * k); });
  }
  s = wave_sum(s);
  if (p.entropy) ent = wave_sum(ent);
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) {
      slots[1][0][w] = s;
      slots[2][0][w] = ent;
    }
    __syncthreads();
    s = over(slots[1][0], Add());
    ent = over(slots[2][0], Add());
  } else if (TOP) {
    row_barrier<L>();
  }
  const RowResult r(m0, s, p.scale);
  if (lane == 0) {
    if (p.parts == 1) write_row(p, row, r, s, ent, given, there);
    else *reinterpret_cast<floatx4*>(p.stat + id * 4) = floatx4{mx, s, ent, 0.f};
  }
  if constexpr (TOP) {
    auto again = [&](auto&& f) {   // (read again: rare, and registers are few)
      for (int i = lane; i < width; i += L) f(order_key(to_f<T>(x[i])), i);
    };
    if constexpr (L > 64)
      if (top.count > kRoom<L>) collect_stretch<L>(want, order_key(own), top, again);
    if (top.count > kRoom<L>) collect_exactly<L>(want, order_key(mx), width, top, again);
    const int64_t base = id * p.top;
    rank_collected<L>(want, top, [&](int rank, uint32_t key, int at) {
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

// A wave a row: its parts merged.  What the lane's first part, its first alternative and the row's
// token need is loaded at once, before anything waits.
template <typename T, bool TOP> __global__ __launch_bounds__(kThreads) void logprob_join_kernel(LogprobParams p) {
  __shared__ TopLds<64> tops[TOP ? kWaves : 1];
  const int64_t row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (row >= p.n) return;
  const int lane = threadIdx.x & 63;
  const float k = p.scale * kLog2e;
  const int64_t count = TOP ? p.parts * p.top : 0;
  auto stat = [&](int64_t j) {
    return *reinterpret_cast<const floatx4*>(p.stat + (row * p.parts + min(j, p.parts - 1)) * 4);
  };
  const floatx4 t0 = stat(lane);
  float x0 = 0.f;
  int32_t at0 = -1;
  if (TOP) {
    const int64_t j = row * count + min((int64_t)lane, count - 1);
    x0 = p.cand_x[j];
    at0 = p.cand_i[j];
  }
  bool there = false;
  const float given = p.logprob ? given_logit<T>(p, row, there) : 0.f;
  float mx = t0[0], s = 0.f, e = 0.f;
  for (int64_t j = lane + 64; j < p.parts; j += 64) mx = fmaxf(mx, stat(j)[0]);
  mx = wave_max(mx);
  const float m0 = mx == -kInf ? 0.f : mx;
  auto add = [&](const floatx4& t) {
    const float d = t[0] == -kInf ? -1000.f : (t[0] - m0) * k, f = __builtin_amdgcn_exp2f(d);
    s = __builtin_fmaf(t[1], f, s);
    e = __builtin_fmaf(__builtin_fmaf(t[1], fmaxf(d, -1000.f), t[2]), f, e);
  };
  if (lane < p.parts) add(t0);
  for (int64_t j = lane + 64; j < p.parts; j += 64) add(stat(j));
  s = wave_sum(s);
  e = wave_sum(e);
  const RowResult r(m0, s, p.scale);
  if (lane == 0) write_row(p, row, r, s, e, given, there);
  if constexpr (TOP) {
    TopLds<64>& top = tops[threadIdx.x >> 6];
    auto each = [&](auto&& f) {
      if (lane < count) f(at0 < 0 ? 0u : order_key(x0), at0);
      for (int64_t j = lane + 64; j < count; j += 64) {
        const int32_t at = p.cand_i[row * count + j];
        f(at < 0 ? 0u : order_key(p.cand_x[row * count + j]), at);
      }
    };
    uint32_t bound = kLowestKey;
    if (count > kRoom<64>) {
      uint32_t best = 0;
      each([&](uint32_t key, int) { best = max(best, key); });
      bound = max(bound_of_lanes(best, p.top), bound);
    }
    if (lane == 0) top.count = 0;
    row_barrier<64>();
    each([&](uint32_t key, int at) {
      if (key >= bound) collect(top, key, at);
    });
    row_barrier<64>();
    if (top.count > kRoom<64>) collect_exactly<64>(p.top, order_key(mx), (int)p.V, top, each);
    rank_collected<64>(p.top, top, [&](int rank, uint32_t key, int at) {
      p.top_lp[row * p.top + rank] = key ? r.of(from_order_key(key)) : r.ln == r.ln ? -kInf : r.ln;
      p.top_ids[row * p.top + rank] = key ? at : -1;
    });
  }
}

// ---------------------------------------------------------------------------
// Gradient.  lse is rounded to fp32, so e^(z - lse) is off by up to half a step of it: 1.9e-6 at 63,
// 7.6e-6 at 255.  The row's own sum of these, by which they are divided, takes that out, and what the
// shift c and the factor k are off by.  Rows farther out (large logits, a row at the type's lowest
// value; an infinite lse: scale times finite logits is, or there is nothing but -inf) take the
// differences from their largest value instead.
// ---------------------------------------------------------------------------
constexpr float kFarLse = 256.f;
// Of one row: log2 p = (x - b) k - c - log2 s.  g and de hold the factor `scale`, and in gs, des that of 1 / s.
struct RowGradient {
  float lse, k, b = 0.f, c, g = 0.f, gs, de = 0.f, des, H = 0.f;
  int y = -1;
  bool far, entropy;
  __device__ __forceinline__ RowGradient(const LogprobParams& p, int64_t row)
      : lse(p.lse_in[row]), k(p.scale * kLog2e), c(lse * kLog2e), far(__builtin_fabsf(lse) > kFarLse), entropy(p.dentropy) {
    if (p.dlogprob) {
      const int64_t t = p.targets[row];
      if (t >= 0 && t < p.V) {
        y = (int)t;
        g = p.dlogprob[row] * p.scale;
      }
    }
    if (entropy) {
      de = p.dentropy[row] * p.scale;
      H = p.entropy_in[row];
    }
    gs = g;
    des = de;
  }
  __device__ __forceinline__ void from(float mx) {
    b = mx;
    c = 0.f;
    if (mx == -kInf) b = g = gs = de = des = 0.f;   // nothing but -inf
  }
  __device__ __forceinline__ float log2_of(float x) const { return __builtin_fmaf(x - b, k, -c); }
  __device__ __forceinline__ float term(float x) const { return __builtin_amdgcn_exp2f(log2_of(x)); }
  // The row's sum of terms.  Further from 1 than the roundings (lse, k and c a step each at most, the sum
  // 128 half steps), the lse given is not of this row alone, and stands.
  __device__ __forceinline__ void divide(float s) {
    if (s == 0.f || (!far && !(__builtin_fabsf(s - 1.f) <= __builtin_fmaf(__builtin_fabsf(lse), 0x1p-21f, 0x1p-17f)))) return;
    gs = g / s;
    des = de / s;
    H -= logf(s);   // (what is added to log p)
  }
  template <typename T, int V>
  __device__ __forceinline__ void write(T* dx, int col, int width, const typename RowVec<T, V>::type& raw, int nt) const {
    float d[V];
    if (entropy) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float t = log2_of(to_f<T>(raw[e]));
        d[e] = -__builtin_amdgcn_exp2f(t) * __builtin_fmaf(des, __builtin_fmaf(fmaxf(t, -1000.f), kLn2, H), gs);   // (0 times -inf)
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] = -term(to_f<T>(raw[e])) * gs;
    }
    const uint32_t at = (uint32_t)(y - col);
    if (at < (uint32_t)V)
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] += (uint32_t)e == at ? g : 0.f;
    if (nt) store_piece<T, V, false, true>(dx + col, width - col, d);
    else store_piece<T, V, false, false>(dx + col, width - col, d);
  }
};
template <int L, typename Op> __device__ __forceinline__ float over_row(float a, float* slots, Op op) {
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = a;
    __syncthreads();
    a = slots[0];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) a = op(a, slots[w]);
  }
  return a;
}

// L lanes a row, which they hold, N pieces each: read once, written once.
template <typename T, int L, int N>
__global__ __launch_bounds__(L > kThreads ? L : kThreads, L == 1024 ? 8 : 1)
void logprob_bwd_kernel(LogprobParams p, int64_t first, int nt) {
  constexpr int V = kPiece<T>, kSub = L > kThreads ? 1 : kThreads / L;
  __shared__ float slots[2][L / 64];
  const int lane = threadIdx.x % L, width = (int)p.V;
  const int64_t row = first + (int64_t)blockIdx.x * kSub + threadIdx.x / L;
  if (row >= p.n) return;   // (whole rows of lanes)
  Part<T, L, N> v;
  v.load(reinterpret_cast<const T*>(p.x) + row * p.xs, width, lane);
  RowGradient r(p, row);
  if (r.far) {
    float mx = -kInf;
    v.each([&](int, int, float z) { mx = fmaxf(mx, z); });
    r.from(over_row<L>(wave_max(mx), slots[0], Max()));
  }
  float s = 0.f;
  v.again();
  v.each([&](int, int, float z) { s += r.term(z); });
  r.divide(over_row<L>(wave_sum(s), slots[1], Add()));
  v.again();
  T* dx = reinterpret_cast<T*>(p.dx) + row * p.V;
#pragma unroll
  for (int j = 0; j < N; ++j) r.write<T, V>(dx, v.col(j, lane), width, v.raw[j], nt);
}

// Longer rows: a workgroup a piece a lane, many a row, which trust its lse as far as it costs no more than
// the exponents' own rounding (fp32: to 32, half a step 9.5e-7) or the outputs' (bf16: to 256, 2^-8 of theirs).  Any
// other row is left to one of its workgroups (in place, others would write what it reads again; not to the
// first, which for 8 n workgroups a row would all lie on one XCD), and read twice, far out three times.
constexpr int kLongLanes = 1024;
// A lane's N pieces from column c0 on, -inf past the row's end (loads without branches: there its last piece).
template <typename T, int N>
__device__ __forceinline__ void load_ahead(const T* x, int c0, int width, typename RowVec<T, kPiece<T>>::type (&raw)[N]) {
  constexpr int V = kPiece<T>, kSpan = kLongLanes * V;
#pragma unroll
  for (int u = 0; u < N; ++u) raw[u] = *reinterpret_cast<const typename RowVec<T, V>::type*>(x + min(c0 + u * kSpan, width - V));
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int c = c0 + u * kSpan, left = width - c;
    if (left >= V) continue;
#pragma unroll
    for (int e = 0; e < V; ++e) raw[u][e] = e < left ? x[c + e] : from_f<T>(-kInf);
  }
}
template <typename T> constexpr float kTrustedLse = sizeof(T) == 4 ? 32.f : kFarLse;
template <typename T> __global__ __launch_bounds__(kLongLanes, 8) void logprob_bwd_long_kernel(LogprobParams p, int64_t first, uint32_t segs, int nt) {
  constexpr int L = kLongLanes, V = kPiece<T>, kSpan = L * V, kAhead = 4;
  typedef typename RowVec<T, V>::type Vec;
  __shared__ float slots[2][L / 64];
  const int64_t id = first + blockIdx.x, row = id / segs;
  const int seg = (int)(id - row * segs), width = (int)p.V, lane = threadIdx.x;
  const T* x = reinterpret_cast<const T*>(p.x) + row * p.xs;
  T* dx = reinterpret_cast<T*>(p.dx) + row * p.V;
  Vec raw[1];
  const int own = seg * kSpan + lane * V;
  load_ahead<T, 1>(x, own, width, raw);
  RowGradient r(p, row);
  if (!(__builtin_fabsf(r.lse) > kTrustedLse<T>)) {
    r.write<T, V>(dx, own, width, raw[0], nt);
    return;
  }
  if (seg != (int)(row % segs)) return;
  auto all = [&](auto f) {
    for (int c0 = lane * V; c0 < width; c0 += kAhead * kSpan) {
      Vec z[kAhead];
      load_ahead<T, kAhead>(x, c0, width, z);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) f(c0 + u * kSpan, z[u]);
    }
  };
  if (r.far) {
    float mx = -kInf;
    all([&](int, const Vec& z) {
#pragma unroll
      for (int e = 0; e < V; ++e) mx = fmaxf(mx, to_f<T>(z[e]));
    });
    r.from(over_row<L>(wave_max(mx), slots[0], Max()));
  }
  float s = 0.f;
  all([&](int, const Vec& z) {
#pragma unroll
    for (int e = 0; e < V; ++e) s += r.term(to_f<T>(z[e]));
  });
  r.divide(over_row<L>(wave_sum(s), slots[1], Add()));
  all([&](int c, const Vec& z) { r.write<T, V>(dx, c, width, z, nt); });
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
constexpr int64_t kMaxLanes = (int64_t)1 << 31;   // of a launch

template <typename T, int L, int N, bool TOP> hipError_t forward(const LogprobParams& p, hipStream_t stream) {
  const int64_t sub = L > kThreads ? 1 : kThreads / L, wgs = (p.n * p.parts + sub - 1) / sub;
  const dim3 threads(L > kThreads ? L : kThreads);
  constexpr int64_t most = kMaxLanes / (L > kThreads ? L : kThreads);
  for (int64_t w = 0; w < wgs; w += most) {
    const dim3 grid((uint32_t)min(wgs - w, most));
    hipLaunchKernelGGL((logprob_fwd_kernel<T, L, N, TOP>), grid, threads, 0, stream, p, w * sub);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// Lanes of a row: few rows take the most; of many, 64 up to 4 pieces a lane, 256 up to 6, or 16 with
// alternatives (whose search costs each wave the same), then 1024.  us, bf16: 16384 x 32768 on 1024 lanes
// (256 of 16 pieces) 167 (189), with five alternatives 257 (232); 4001 x 49152 with five on 1024 lanes (512
// of 12) 90 (114).
constexpr int64_t kFewRows = 512;
template <typename T, int L, bool TOP> hipError_t forward_pieces(const LogprobParams& p, int64_t n, hipStream_t stream) {
  if (n <= 1) return forward<T, L, 1, TOP>(p, stream);
  if (n <= 2) return forward<T, L, 2, TOP>(p, stream);
  if constexpr (L == 64) return forward<T, L, 4, TOP>(p, stream);
  else {
    if (n <= 4) return forward<T, L, 4, TOP>(p, stream);
    if (n <= 5) return forward<T, L, 5, TOP>(p, stream);
    if constexpr (L == 256 && !TOP) return forward<T, L, 6, TOP>(p, stream);
    else {
      if (n <= 6) return forward<T, L, 6, TOP>(p, stream);
      if (n <= 7) return forward<T, L, 7, TOP>(p, stream);
      if (n <= 8) return forward<T, L, 8, TOP>(p, stream);
      if (n <= 10) return forward<T, L, 10, TOP>(p, stream);
      if (n <= 13) return forward<T, L, 13, TOP>(p, stream);
      return forward<T, L, 16, TOP>(p, stream);
    }
  }
}
template <typename T, bool TOP> hipError_t forward_lanes(const LogprobParams& p, hipStream_t stream) {
  constexpr int V = kPiece<T>;
  const int64_t pieces = (p.width + V - 1) / V;
  const bool few = p.n * p.parts <= kFewRows;
  const int64_t lanes = pieces <= 64 * (few ? 1 : 4) ? 64 : pieces <= 256 * (few ? 1 : TOP ? 16 : 6) ? 256 : 1024;
  const int64_t n = (pieces + lanes - 1) / lanes;
  return lanes == 64    ? forward_pieces<T, 64, TOP>(p, n, stream)
         : lanes == 256 ? forward_pieces<T, 256, TOP>(p, n, stream)
                        : forward_pieces<T, 1024, TOP>(p, n, stream);
}
template <typename T> hipError_t forward(const LogprobParams& p, hipStream_t stream) {
  const hipError_t e = p.top ? forward_lanes<T, true>(p, stream) : forward_lanes<T, false>(p, stream);
  if (e != hipSuccess || p.parts == 1) return e;
  const dim3 grid((uint32_t)((p.n + kWaves - 1) / kWaves));
  if (p.top) hipLaunchKernelGGL((logprob_join_kernel<T, true>), grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((logprob_join_kernel<T, false>), grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

// `launch` for all of `wgs` workgroups, from workgroup w on: as many as a launch holds at a time.
template <typename F> hipError_t backward_launches(int64_t wgs, int64_t threads, F launch) {
  const int64_t most = kMaxLanes / threads;
  for (int64_t w = 0; w < wgs; w += most) {
    launch(dim3((uint32_t)min(wgs - w, most)), w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename T, int L, int N> hipError_t backward(const LogprobParams& p, int nt, hipStream_t stream) {
  constexpr int threads = L > kThreads ? L : kThreads, sub = threads / L;
  return backward_launches((p.n + sub - 1) / sub, threads, [&](dim3 grid, int64_t w) {
    hipLaunchKernelGGL((logprob_bwd_kernel<T, L, N>), grid, dim3(threads), 0, stream, p, w * sub, nt);
  });
}
// Lanes of a row, as many as hold it in registers for two rows of 1024 on a CU (fp32: 20480 logits, bf16: 40960); of
// few rows more, for latency.  us: 16384 x 32768 of bf16 415 (2.15 GB, the 5.2 TB/s of a large copy), rows at 400 422;
// 3000 x 20003 of fp32 76 and 77.  Longer: 4001 x 50001 of bf16 145, at 400 309; 2000 x 151936 of fp32 396, at 100 665, at
// 400 816; 1 x 131072 of fp32 2.3, 18, 22.
template <typename T> hipError_t backward(const LogprobParams& p, hipStream_t stream) {
  const int64_t pieces = (p.V + kPiece<T> - 1) / kPiece<T>;
  const int nt = p.n * p.V * (int64_t)sizeof(T) > kNtBytes;
  const bool few = p.n <= kFewRows;
  if (pieces <= 64) return backward<T, 64, 1>(p, nt, stream);
  if (!few && pieces <= 128) return backward<T, 64, 2>(p, nt, stream);
  if (!few && pieces <= 256) return backward<T, 64, 4>(p, nt, stream);
  if (pieces <= 256) return backward<T, 256, 1>(p, nt, stream);
  if (pieces <= 512) return backward<T, 256, 2>(p, nt, stream);
  if (!few && pieces <= 1024) return backward<T, 256, 4>(p, nt, stream);
  if (!few && pieces <= 1536) return backward<T, 256, 6>(p, nt, stream);
  // (a few rows of bf16, whose digits are the outputs': sooner done by several workgroups each, 1 x 32768 2.7, not 4.7)
  if (!few || sizeof(T) == 4) {
    const int64_t n = (pieces + 1023) / 1024;
    if constexpr (sizeof(T) == 4)
      if (n <= 1) return backward<T, 1024, 1>(p, nt, stream);
    if (n <= 2) return backward<T, 1024, 2>(p, nt, stream);
    if (n <= 3) return backward<T, 1024, 3>(p, nt, stream);
    if (n <= 4) return backward<T, 1024, 4>(p, nt, stream);
    if (n <= 5) return backward<T, 1024, 5>(p, nt, stream);
  }
  constexpr int64_t span = kLongLanes * kPiece<T>;
  const int64_t segs = (p.V + span - 1) / span;
  return backward_launches(p.n * segs, kLongLanes, [&](dim3 grid, int64_t w) {
    hipLaunchKernelGGL((logprob_bwd_long_kernel<T>), grid, dim3(kLongLanes), 0, stream, p, w, (uint32_t)segs, nt);
  });
}

}  // namespace

size_t logprob_plan(LogprobParams& p, bool bf16, unsigned char* ws) {
  // Values that a workgroup holds; few long rows: as many workgroups as CUs, of no less than 32768 values
  // (64 rows of 131072 with entropy and eight alternatives: 16.4 us, in one part each 19.3).
  const int64_t piece = bf16 ? 8 : 4, most = 16 * 1024 * piece;
  constexpr int64_t cus = 256, least = 32768;
  int64_t parts = (p.V + most - 1) / most;
  if (p.n * parts < cus) parts = max(parts, min(cus / max(p.n, (int64_t)1), p.V / least));
  p.width = ((p.V + parts - 1) / parts + piece - 1) / piece * piece;
  p.parts = (p.V + p.width - 1) / p.width;
  // Room for as many parts as any call of up to this many rows has: a workspace serves smaller calls too.
  const int64_t base = (p.V + most - 1) / most, few = max(base, p.V / least);
  const size_t all = (size_t)max(base > 1 ? p.n * base : 0, few > 1 ? min(cus, p.n * few) : 0);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* at = ws + off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
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

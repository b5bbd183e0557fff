// Embedding lookup, out_t = scale table[id_t], and the table's gradient: row v gets
// scale times the sum, in the order of t, of dout_t where id_t = v.
//
// The gradient sorts (id, t) by id, stably, and sums stretches of equal ids: every row of the table is
// written once, in one order of summation, and nothing is added by atomics (they count
// tokens and mark rows only).  Ids without a row sort behind the others and are dropped.  Few tokens:
//   embed_rank    counts for each token those before it, and marks the rows that have one
// More, in two passes of a counting sort over the id's low and high bits:
//   embed_count   a tile of tokens counts its low digits; clears what is counted later
//   embed_sort    a tile moves its tokens to their places among all: the counts of smaller
//                 digits, of the same digit in earlier tiles, and in the tile itself
//                 (first pass: also counts the high digits by the tile that a token lands in,
//                 and marks the rows that have a token)
//   embed_sort    second pass; other workgroups write the rows without a token
// Then:
//   embed_sums    a group of lanes takes `chunk` sorted tokens and writes the sums of the ids
//                 that start there and end there or in the next chunk; of longer runs
//                 each chunk leaves its part (few tokens: others write the rows without one)
//   embed_join    adds these parts
// 16384 tokens as frequent as words, 32768 x 2048, bf16 rows into an fp32 table, us: 4.6, 10.0, 42.0 (224 MB of
// zeros at 5.3 TB/s, the second pass beside them), 26 (67 MB read at random, 45 written), 6.2; all bytes
// at 5.0 TB/s would take 67.  Few tokens of a narrow table are bound by the launches, two to three.
#include "model.hpp"

namespace rla {

namespace {

// Pieces of V values of a row, the i-th from column i V.  FULL: the last one moved back to the row's end,
// so that all are whole (what two of them cover is computed by both, to the same bits; not where
// a row is added to in place).
template <int V, bool FULL> __device__ __forceinline__ int64_t piece_col(int64_t i, int64_t D) {
  return FULL ? min(i * V, D - V) : i * V;
}
bool full(const EmbedParams& p, int V) { return p.D % V == 0 || (p.D >= V && (!p.base || p.base != p.dtable)); }

// The id as a sorting key: V for one without a row.
__device__ __forceinline__ uint32_t key_of(const EmbedParams& p, int64_t t) {
  const int64_t id = p.ids[t];
  return id >= 0 && id < p.V ? (uint32_t)id : (uint32_t)p.V;
}

// ---------------------------------------------------------------------------
// lookup: a thread a piece of a row (16384 rows of 2048, fp32 to bf16: 24.1 us; 256 of bf16: 2.8)
// ---------------------------------------------------------------------------
template <typename X, typename T, bool FULL, bool NT>
__global__ __launch_bounds__(kThreads) void embed_fwd_kernel(EmbedParams p, uint32_t pieces, uint32_t count) {
  constexpr int V = kPiece<T>;
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  if (id >= count) return;
  const uint32_t t = id / pieces;
  const int64_t c = piece_col<V, FULL>(id % pieces, p.D);
  const int left = (int)min(p.D - c, (int64_t)V);
  const uint32_t row = key_of(p, t);
  float x[V];
  if (row < (uint32_t)p.V) {
    load_piece<X, V, FULL>(reinterpret_cast<const X*>(p.table) + (int64_t)row * p.D + c, left, x);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] *= p.scale;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = 0.f;
  }
  store_piece<T, V, FULL, NT>(reinterpret_cast<T*>(p.out) + (int64_t)t * p.D + c, left, x);
}

// ---------------------------------------------------------------------------
// sorting
// ---------------------------------------------------------------------------
constexpr int kEmbedTile = 1024, kEmbedLargeTile = 4096;   // tokens of a tile: of up to 65536 tokens, of more

__global__ __launch_bounds__(kThreads) void embed_count_kernel(EmbedParams p) {
  extern __shared__ int32_t lds[];
  const int tid = threadIdx.x, bins = 1 << p.bits1;
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  for (int b = tid; b < bins; b += kThreads) lds[b] = 0;
  // what later kernels count in
  const int64_t all = (int64_t)gridDim.x * kThreads, own = (int64_t)blockIdx.x * kThreads + tid;
  for (int64_t i = own; i < (int64_t)p.tiles << p.bits2; i += all) p.count2[i] = 0;
  for (int64_t i = own; i < p.V / 32 + 1; i += all) p.present[i] = 0;
  __syncthreads();
  for (int i = tid; i < p.tile && t0 + i < p.n; i += kThreads) atomicAdd(&lds[key_of(p, t0 + i) & (bins - 1)], 1);
  __syncthreads();
  for (int b = tid; b < bins; b += kThreads) p.count1[(int64_t)blockIdx.x * bins + b] = lds[b];
}

// A tile's tokens to their places.  Each wave has a quarter of the tile, in order, ROUNDS of 64; lds:
// [kWaves][bins] next places by wave and digit, then kThreads sums.
template <bool SECOND, int ROUNDS>
__device__ __forceinline__ void sort_tile(const EmbedParams& p, int tile, int32_t* lds) {
  const int bits = SECOND ? p.bits2 : p.bits1, bins = 1 << bits;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int32_t* counts = SECOND ? p.count2 : p.count1;
  int32_t* place = lds;
  int32_t* sums = lds + kWaves * bins;
  const int64_t first = (int64_t)tile * p.tile + (int64_t)w * (ROUNDS * 64) + lane;
  auto digit = [&](uint32_t k) { return (int)((SECOND ? k >> p.bits1 : k) & (uint32_t)(bins - 1)); };

  uint32_t key[ROUNDS];
  int32_t pos[ROUNDS];
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const int64_t i = min(first + j * 64, p.n - 1);
    key[j] = SECOND ? (uint32_t)p.key1[i] : key_of(p, i);
    pos[j] = SECOND ? p.pos1[i] : (int32_t)i;
  }
  // a thread's digits: how many tokens have each, and how many of those lie in earlier tiles
  constexpr int kMost = (1 << 11) / kThreads, kAhead = 8;   // digits of a thread; loads in flight
  const int per = (bins + kThreads - 1) / kThreads;
  int32_t before[kMost], all[kMost], total = 0;
#pragma unroll
  for (int j = 0; j < kMost; ++j) {
    before[j] = all[j] = 0;
    const int b = tid * per + j;
    if (j >= per || b >= bins) continue;
    for (int i0 = 0; i0 < p.tiles; i0 += kAhead) {
      int32_t c[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) c[u] = counts[(int64_t)min(i0 + u, p.tiles - 1) * bins + b];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        all[j] += i0 + u < p.tiles ? c[u] : 0;
        before[j] += i0 + u < tile ? c[u] : 0;
      }
    }
    total += all[j];
  }
  for (int b = tid; b < kWaves * bins; b += kThreads) place[b] = 0;
  // places before the thread's digits: over the wave's lanes, then over the waves
  int32_t at = total;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int32_t o = __shfl_up(at, d);
    at += lane >= d ? o : 0;
  }
  if (lane == 63) sums[w] = at;
  at -= total;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kWaves - 1; ++v) at += v < w ? sums[v] : 0;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j)
    if (first + j * 64 < p.n) atomicAdd(&place[w * bins + digit(key[j])], 1);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kMost; ++j) {
    const int b = tid * per + j;
    if (j >= per || b >= bins) continue;
    int32_t next = at + before[j];
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const int32_t c = place[v * bins + b];
      place[v * bins + b] = next;
      next += c;
    }
    at += all[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const bool there = first + j * 64 < p.n;
    const uint32_t k = key[j];
    const int d = digit(k);
    // lanes of the same digit
    uint64_t same = __ballot(there);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? set : ~set;
    }
    if (!there) continue;
    const int rank = __popcll(same & ((1ull << lane) - 1));
    const int32_t to = place[w * bins + d] + rank;
    // (a wave's accesses to LDS keep their order; the compiler is told so)
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    if (rank == 0) place[w * bins + d] = to + __popcll(same);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    if (SECOND) {
      p.key[to] = (int32_t)k;
      p.pos[to] = pos[j];
    } else {
      p.key1[to] = (int32_t)k;
      p.pos1[to] = pos[j];
      // one lane for all of a key (and of a tile that they land in: two at most), or a frequent id's tokens
      // wait for each other (16384 tokens, 10 % of one id: 17 us, now 10)
      uint64_t equal = same;
      for (int b = 0; b < p.bits2; ++b) {
        const uint32_t bit = k >> (p.bits1 + b) & 1u;
        const uint64_t set = __ballot(bit);
        equal &= bit ? set : ~set;
      }
      const uint64_t odd = __ballot(to / p.tile & 1);
      equal &= to / p.tile & 1 ? odd : ~odd;
      if ((equal & ((1ull << lane) - 1)) == 0) {
        atomicAdd(&p.count2[(((int64_t)(to / p.tile)) << p.bits2) + (k >> p.bits1)], __popcll(equal));
        if (k < (uint32_t)p.V) atomicOr(&p.present[k >> 5], 1u << (k & 31));
      }
    }
  }
}

template <int ROUNDS> __global__ __launch_bounds__(kThreads) void embed_sort1_kernel(EmbedParams p) {
  extern __shared__ int32_t lds[];
  sort_tile<false, ROUNDS>(p, blockIdx.x, lds);
}

// Rows without a token, by workgroup.
constexpr int kFillPieces = 8;   // 16-byte pieces a thread

template <bool FULL, bool NT> __device__ __forceinline__ void fill_rows(const EmbedParams& p, uint32_t pieces, int64_t wg) {
  const int64_t first = wg * (kThreads * kFillPieces) + threadIdx.x;
#pragma unroll
  for (int j = 0; j < kFillPieces; ++j) {
    const int64_t id = first + j * kThreads;
    const int64_t v = id / pieces, c = piece_col<4, FULL>(id - v * pieces, p.D);
    if (v >= p.V || (p.present[v >> 5] >> (v & 31)) & 1u) continue;
    const int left = (int)min(p.D - c, (int64_t)4);
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.base) load_piece<float, 4, FULL>(p.base + v * p.D + c, left, x);
    store_piece<float, 4, FULL, NT>(p.dtable + v * p.D + c, left, x);
  }
}

template <int ROUNDS, bool FULL, bool NT>
__global__ __launch_bounds__(kThreads) void embed_sort2_kernel(EmbedParams p, uint32_t pieces) {
  extern __shared__ int32_t lds[];
  if ((int)blockIdx.x < p.tiles) sort_tile<true, ROUNDS>(p, blockIdx.x, lds);
  else fill_rows<FULL, NT>(p, pieces, (int64_t)blockIdx.x - p.tiles);
}

// Up to kRankTokens: a token's place is the number of tokens before it in the order, counted over all of
// them, kRanked tokens a workgroup, 32 lanes each.  The same workgroups find the rows that have a
// token, kRankWords words of bits each.  One launch for three, whose 2 n^2 operations are 4 us of the
// card's at 8192 tokens (4099: 6.1 us in all).  The whole gradient, us, against the counting sort: 6 tokens
// 10.3 (15.5), 600 of 64 values 14.3 (20.1), 3000 14.4 (21.7), 8000 17.7 (25.5), 8192 of 1024 40 (46); on from
// there, 64 tokens a workgroup: 12288 of 1024 53 (50), 16384 60 (52).
constexpr int kRankTokens = 8192, kRankThreads = 1024, kRanked = 32, kRankWords = 1024;
__global__ __launch_bounds__(kRankThreads) void embed_rank_kernel(EmbedParams p) {
  __shared__ uint4 keys[kRankTokens / 4];
  __shared__ uint32_t bits[kRankWords];
  __shared__ int32_t counts[kRankThreads / kRanked][kRanked];
  uint32_t* key = reinterpret_cast<uint32_t*>(keys);
  const int tid = threadIdx.x, n = (int)p.n, slices = kRankThreads / kRanked;
  const int all = (n + 4 * slices - 1) / (4 * slices) * (4 * slices);   // (whole reads of 4 for each slice; past n: behind all)
  const uint32_t word0 = blockIdx.x * kRankWords;
  for (int i = tid; i < kRankWords; i += kRankThreads) bits[i] = 0;
  __syncthreads();
  auto load = [&](auto type) {
    typedef decltype(type) Id;
    const Id* ids = reinterpret_cast<const Id*>(p.ids.p);
    constexpr int kAhead = 4;
    for (int i0 = tid; i0 < all; i0 += kAhead * kRankThreads) {
      Id id[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) id[u] = ids[min(i0 + u * kRankThreads, n - 1)];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + u * kRankThreads;
        const bool row = id[u] >= 0 && id[u] < p.V;
        const uint32_t k = row ? (uint32_t)id[u] : (uint32_t)p.V, word = (k >> 5) - word0;
        if (i < all) key[i] = i < n ? k : 0xffffffffu;
        if (row && word < kRankWords) atomicOr(&bits[word], 1u << (k & 31u));   // (past n: the last again)
      }
    }
  };
  if (p.ids.wide) load(int64_t());
  else load(int32_t());
  __syncthreads();
  const int first = blockIdx.x * kRanked, i = first + tid % kRanked, slice = tid / kRanked;
  const uint32_t own = first < n ? key[min(i, n - 1)] : 0u;
  int count = 0;
  if (first < n) {
    // (of equal keys the earlier tokens)
    const int each = all / (4 * slices), g0 = slice * each, block = first / 4;
#pragma unroll 4
    for (int g = g0; g < g0 + each; ++g) {
      const uint4 k = keys[g];
      const uint32_t below = own + (g < block ? 1u : 0u);
      count += k.x < below ? 1 : 0;
      count += k.y < below ? 1 : 0;
      count += k.z < below ? 1 : 0;
      count += k.w < below ? 1 : 0;
    }
    static_assert(kRanked <= 4 * (kRankThreads / kRanked), "the workgroup's own tokens: a read of 4 a slice");
    const int g = block + slice, j = 4 * g;
    if (j < i) {   // (slices behind the workgroup's tokens: never)
      const uint4 k = keys[g];
      count += k.x == own ? 1 : 0;
      count += k.y == own && j + 1 < i ? 1 : 0;
      count += k.z == own && j + 2 < i ? 1 : 0;
      count += k.w == own && j + 3 < i ? 1 : 0;
    }
    counts[slice][tid % kRanked] = count;
  }
  __syncthreads();
  if (tid < kRanked && i < n) {
    int rank = 0;
    for (int v = 0; v < slices; ++v) rank += counts[v][tid];
    p.key[rank] = (int32_t)own;
    p.pos[rank] = i;
  }
  for (int64_t w = tid; w < kRankWords && word0 + w <= p.V / 32; w += kRankThreads) p.present[word0 + w] = bits[w];
}

// ---------------------------------------------------------------------------
// sums
// ---------------------------------------------------------------------------
// Whether the run of key k that fills the end of chunk c (tokens up to i1) ends in the
// next chunk.
__device__ __forceinline__ bool ends_next(const EmbedParams& p, int64_t i1, int32_t k) {
  const int64_t i2 = min(i1 + p.chunk, p.n);
  const int32_t last = p.key[i2 - 1], behind = p.key[min(i2, p.n - 1)];
  return last != k || i2 == p.n || behind != k;
}

// L lanes a chunk of sorted tokens, a piece of the columns a lane (blockIdx.y: which L pieces).
// BASE: what the sums are added to is loaded with the rows, for each token (those of one run hit the caches).
// From workgroup `fill` on (0: none) others write the rows without a token.
template <typename T, int L, bool FULL, bool BASE>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(EmbedParams p, uint32_t fill, uint32_t pieces, bool nt) {
  constexpr int V = kPiece<T>, kAhead = BASE ? 4 : 8;
  if (fill && blockIdx.x >= fill) {
    const int64_t wg = (int64_t)(blockIdx.x - fill) * gridDim.y + blockIdx.y;
    if (nt) fill_rows<FULL, true>(p, pieces, wg);
    else fill_rows<FULL, false>(p, pieces, wg);
    return;
  }
  const int64_t c = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (c >= p.chunks) return;
  const int64_t piece = (int64_t)blockIdx.y * L + threadIdx.x % L, col = piece_col<V, FULL>(piece, p.D);
  if (piece * V >= p.D) return;
  const int left = (int)min(p.D - col, (int64_t)V);
  int64_t i = c * p.chunk, end = min(i + p.chunk, p.n);
  const int32_t kFirst = p.key[i], kLast = p.key[end - 1], kBefore = p.key[max(i - 1, (int64_t)0)],
                kEarlier = p.key[max(i - p.chunk - 1, (int64_t)0)], kBehind = p.key[min(end, p.n - 1)];
  const bool goes_on = end < p.n && kBehind == kLast, short_tail = ends_next(p, end, kLast);
  bool head = false;   // the first run began in an earlier chunk, which leaves it in parts
  if (c > 0 && kBefore == kFirst) {
    const bool began_before = c == 1 || kEarlier != kFirst;
    const bool ends_here = kLast != kFirst || !goes_on;
    if (began_before && ends_here) {   // the previous chunk's
      while (i < end && p.key[i] == kFirst) ++i;
    } else {
      head = true;
    }
  }
  bool tail = false;   // the last run goes on beyond the next chunk
  if (goes_on && !(head && kFirst == kLast)) {
    if (short_tail) {
      while (end < p.n && p.key[end] == kLast) ++end;
    } else {
      tail = true;
    }
  }
  if (i >= end) return;
  float sum[V], base[V];
#pragma unroll
  for (int e = 0; e < V; ++e) sum[e] = base[e] = 0.f;
  int32_t k = p.key[i];
  auto flush = [&](bool last) {
    if (k >= (int32_t)p.V) return;
    if (head || (last && tail)) {
      store_piece<float, V, FULL>(p.part + (c * 2 + (head ? 0 : 1)) * p.D + col, left, sum);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] = BASE ? __builtin_fmaf(p.scale, sum[e], base[e]) : p.scale * sum[e];
      store_piece<float, V, FULL>(p.dtable + (int64_t)k * p.D + col, left, sum);
    }
  };
  const T* dout = reinterpret_cast<const T*>(p.dout) + col;
  for (; i < end; i += kAhead) {
    int32_t kk[kAhead];
    typename RowVec<T, V>::type raw[kAhead];
    float bb[BASE ? kAhead : 1][V];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {   // (past the end: the last again, not used)
      const int64_t at = min(i + u, end - 1);
      kk[u] = p.key[at];
      load_raw<T, V, FULL>(dout + (int64_t)p.pos[at] * p.dos, left, raw[u]);
      if constexpr (BASE) load_piece<float, V, FULL>(p.base + min((int64_t)kk[u], p.V - 1) * p.D + col, left, bb[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i + u >= end) break;
      if (kk[u] != k) {
        flush(false);
        head = false;
        k = kk[u];
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sum[e] += to_f<T>(raw[u][e]);
        if constexpr (BASE) base[e] = bb[u][e];
      }
    }
  }
  flush(true);
}

// Runs that a chunk left in parts: its tail and the following chunks' heads.  A workgroup looks at
// `per` chunks (at most 64) for such runs; 256 columns, a lane 4 of them, the parts over the waves.
template <bool FULL> __global__ __launch_bounds__(kThreads) void embed_join_kernel(EmbedParams p, int32_t per) {
  __shared__ float sums[kWaves][64][4];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t c0 = (int64_t)blockIdx.y * per, piece = (int64_t)blockIdx.x * 64 + lane, col = piece_col<4, FULL>(piece, p.D);
  const int left = piece * 4 < p.D ? (int)min(p.D - col, (int64_t)4) : 0;
  bool split = false;
  if (lane < per && c0 + lane + 1 < p.chunks) {
    const int64_t i = (c0 + lane) * p.chunk, end = i + p.chunk;
    const int32_t k = p.key[end - 1];
    const bool whole = i > 0 && p.key[i] == k && p.key[i - 1] == k;   // inside a run that began earlier
    split = k < (int32_t)p.V && p.key[end] == k && !whole && !ends_next(p, end, k);
  }
  for (uint64_t left_runs = __ballot(split); left_runs; left_runs &= left_runs - 1) {
    const int64_t c = c0 + __builtin_ctzll(left_runs);
    const int32_t k = p.key[(c + 1) * p.chunk];
    // parts: the tail of c, the heads of c + 1 .. c + count
    int64_t count = 0;
    while (true) {
      const int64_t d = c + 1 + count + lane;
      const uint64_t in = __ballot(d < p.chunks && p.key[min(d, (int64_t)p.chunks - 1) * p.chunk] == k);
      const int run = in == ~0ull ? 64 : __builtin_ctzll(~in);
      count += run;
      if (run < 64) break;
    }
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (left > 0) {
      constexpr int kAhead = 8;   // loads in flight (past the last: it again, not used)
      for (int64_t j0 = w; j0 <= count; j0 += kAhead * kWaves) {
        float x[kAhead][4];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int64_t j = min(j0 + u * kWaves, count);
          load_piece<float, 4, FULL>(p.part + ((c + j) * 2 + (j == 0 ? 1 : 0)) * p.D + col, left, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] += j0 + u * kWaves <= count ? x[u][e] : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[w][lane][e] = s[e];
    __syncthreads();
    if (w == 0 && left > 0) {
      float b[4] = {0.f, 0.f, 0.f, 0.f};
      if (p.base) load_piece<float, 4, FULL>(p.base + (int64_t)k * p.D + col, left, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        for (int v = 1; v < kWaves; ++v) s[e] += sums[v][lane][e];
        s[e] = __builtin_fmaf(p.scale, s[e], b[e]);
      }
      store_piece<float, 4, FULL>(p.dtable + (int64_t)k * p.D + col, left, s);
    }
    __syncthreads();
  }
}

// without tokens: dtable = base
__global__ __launch_bounds__(kThreads) void embed_copy_kernel(const float* base, float* dtable, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads)
    dtable[i] = base ? base[i] : 0.f;
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
template <typename X, typename T, bool FULL> hipError_t forward(const EmbedParams& p, hipStream_t stream) {
  const int64_t pieces = (p.D + kPiece<T> - 1) / kPiece<T>;
  const bool nt = p.n * p.D * (int64_t)sizeof(T) > kNtBytes;
  // (more pieces than a launch holds: several, of whole rows each)
  const int64_t most = max((int64_t)1, ((int64_t)1 << 31) / pieces);
  EmbedParams part = p;
  for (int64_t t = 0; t < p.n; t += most) {
    part.n = min(p.n - t, most);
    part.ids.p = reinterpret_cast<const char*>(p.ids.p) + t * (p.ids.wide ? 8 : 4);
    part.out = reinterpret_cast<T*>(p.out) + t * p.D;
    const uint32_t count = (uint32_t)(part.n * pieces);
    const dim3 grid((count + kThreads - 1) / kThreads);
    if (nt) hipLaunchKernelGGL((embed_fwd_kernel<X, T, FULL, true>), grid, dim3(kThreads), 0, stream, part, (uint32_t)pieces, count);
    else hipLaunchKernelGGL((embed_fwd_kernel<X, T, FULL, false>), grid, dim3(kThreads), 0, stream, part, (uint32_t)pieces, count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename X, typename T> hipError_t forward(const EmbedParams& p, hipStream_t stream) {
  return full(p, kPiece<T>) ? forward<X, T, true>(p, stream) : forward<X, T, false>(p, stream);
}

// Workgroups that write the rows without a token (in place: none).
int64_t fill_wgs(const EmbedParams& p) {
  const int64_t pieces = (p.D + 3) / 4, count = p.base == p.dtable ? 0 : p.V * pieces;
  return (count + kThreads * kFillPieces - 1) / (kThreads * kFillPieces);
}
bool nt_table(const EmbedParams& p) { return p.V * p.D * 4 > kNtBytes; }

template <typename T, int L, bool FULL> hipError_t sums(const EmbedParams& p, hipStream_t stream) {
  constexpr int V = kPiece<T>, sub = kThreads / L;
  dim3 grid((uint32_t)((p.chunks + sub - 1) / sub), (uint32_t)((p.D + L * V - 1) / (L * V)));
  const uint32_t fill = p.n <= kRankTokens ? grid.x : 0;
  if (fill) grid.x += (uint32_t)((fill_wgs(p) + grid.y - 1) / grid.y);
  const uint32_t pieces = (uint32_t)((p.D + 3) / 4);
  if (p.base) hipLaunchKernelGGL((embed_sums_kernel<T, L, FULL, true>), grid, dim3(kThreads), 0, stream, p, fill, pieces, nt_table(p));
  else hipLaunchKernelGGL((embed_sums_kernel<T, L, FULL, false>), grid, dim3(kThreads), 0, stream, p, fill, pieces, nt_table(p));
  return hipGetLastError();
}
template <typename T, bool FULL> hipError_t sums(const EmbedParams& p, hipStream_t stream) {
  const int64_t pieces = (p.D + kPiece<T> - 1) / kPiece<T>;
  if (pieces <= 8) return sums<T, 8, FULL>(p, stream);
  if (pieces <= 16) return sums<T, 16, FULL>(p, stream);
  if (pieces <= 32) return sums<T, 32, FULL>(p, stream);
  if (pieces <= 64) return sums<T, 64, FULL>(p, stream);
  if (pieces <= 128) return sums<T, 128, FULL>(p, stream);
  return sums<T, 256, FULL>(p, stream);
}

template <int ROUNDS, bool FULL> hipError_t sort_and_fill(const EmbedParams& p, hipStream_t stream) {
  const size_t lds1 = 4 * ((size_t)kWaves * (1 << p.bits1) + kThreads), lds2 = 4 * ((size_t)kWaves * (1 << p.bits2) + kThreads);
  hipLaunchKernelGGL(embed_count_kernel, dim3(p.tiles), dim3(kThreads), 4u << p.bits1, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(embed_sort1_kernel<ROUNDS>, dim3(p.tiles), dim3(kThreads), lds1, stream, p);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((uint32_t)(p.tiles + fill_wgs(p)));
  const uint32_t pieces = (uint32_t)((p.D + 3) / 4);
  if (nt_table(p)) hipLaunchKernelGGL((embed_sort2_kernel<ROUNDS, FULL, true>), grid, dim3(kThreads), lds2, stream, p, pieces);
  else hipLaunchKernelGGL((embed_sort2_kernel<ROUNDS, FULL, false>), grid, dim3(kThreads), lds2, stream, p, pieces);
  return hipGetLastError();
}
hipError_t rank(const EmbedParams& p, hipStream_t stream) {
  const int64_t words = p.V / 32 + 1, wgs = max((p.n + kRanked - 1) / kRanked, (words + kRankWords - 1) / kRankWords);
  hipLaunchKernelGGL(embed_rank_kernel, dim3((uint32_t)wgs), dim3(kRankThreads), 0, stream, p);
  return hipGetLastError();
}

// One slice's gradient.
template <typename T> hipError_t backward(const EmbedParams& p, hipStream_t stream) {
  constexpr int V = kPiece<T>;
  static_assert(kEmbedTile == 4 * 64 * kWaves && kEmbedLargeTile == 16 * 64 * kWaves, "rounds of a wave");
  hipError_t e;
  if (p.n <= kRankTokens) e = rank(p, stream);
  else if (p.tile == kEmbedTile) e = full(p, 4) ? sort_and_fill<4, true>(p, stream) : sort_and_fill<4, false>(p, stream);
  else e = full(p, 4) ? sort_and_fill<16, true>(p, stream) : sort_and_fill<16, false>(p, stream);
  if (e != hipSuccess) return e;
  e = full(p, V) ? sums<T, true>(p, stream) : sums<T, false>(p, stream);
  if (e != hipSuccess || p.chunks < 3) return e;   // (a run in parts spans a whole chunk and its neighbours)
  const int32_t per = (p.chunks + 127) / 128;
  const dim3 grid((uint32_t)((p.D + 255) / 256), (uint32_t)((p.chunks + per - 1) / per));
  if (full(p, 4)) hipLaunchKernelGGL(embed_join_kernel<true>, grid, dim3(kThreads), 0, stream, p, per);
  else hipLaunchKernelGGL(embed_join_kernel<false>, grid, dim3(kThreads), 0, stream, p, per);
  return hipGetLastError();
}

}  // namespace

size_t embed_plan(EmbedParams& p, int64_t tokens, unsigned char* ws) {
  int bits = 1;
  while (((int64_t)1 << bits) < p.V + 1) ++bits;
  p.bits1 = (bits + 1) / 2;
  p.bits2 = bits - p.bits1;
  p.n = tokens;
  p.tile = tokens <= 65536 ? kEmbedTile : kEmbedLargeTile;
  p.tiles = (int32_t)((tokens + p.tile - 1) / p.tile);
  // (few tokens: more groups of lanes; up to 64 in two chunks, which leave no parts to be added)
  p.chunk = tokens <= 64 ? 32 : tokens <= 8192 ? 8 : 16;
  while (p.chunk * 4096 < tokens) p.chunk *= 2;
  p.chunks = (int32_t)((tokens + p.chunk - 1) / p.chunk);
  // Room for as many tiles and chunks as any call of up to this many tokens has: a workspace serves smaller calls too.
  const int64_t tiles = max((int64_t)p.tiles, min((tokens + kEmbedTile - 1) / kEmbedTile, (int64_t)65536 / kEmbedTile));
  const int64_t chunks = tokens <= kRankTokens ? p.chunks : max((int64_t)kRankTokens / 8, min((tokens + 15) / 16, (int64_t)4096));
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* at = ws + off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  p.present = reinterpret_cast<uint32_t*>(take(4 * (size_t)(p.V / 32 + 1)));
  for (int32_t** a : {&p.key, &p.pos}) *a = reinterpret_cast<int32_t*>(take(4 * (size_t)tokens));
  if (tokens > kRankTokens) {
    p.count1 = reinterpret_cast<int32_t*>(take(4 * ((size_t)tiles << p.bits1)));
    p.count2 = reinterpret_cast<int32_t*>(take(4 * ((size_t)tiles << p.bits2)));
    for (int32_t** a : {&p.key1, &p.pos1}) *a = reinterpret_cast<int32_t*>(take(4 * (size_t)tokens));
  }
  p.part = reinterpret_cast<float*>(take(p.chunks < 3 ? 0 : 8 * (size_t)chunks * (size_t)p.D));
  return off;
}

hipError_t launch_embed_forward(const EmbedParams& p, bool table_bf16, bool bf16, hipStream_t stream) {
  if (table_bf16) return bf16 ? forward<u16, u16>(p, stream) : forward<u16, float>(p, stream);
  return bf16 ? forward<float, u16>(p, stream) : forward<float, float>(p, stream);
}

hipError_t launch_embed_backward(const EmbedParams& p, bool bf16, unsigned char* ws, hipStream_t stream) {
  EmbedParams q = p;
  if (p.n == 0) {
    const int64_t n = p.base == p.dtable ? 0 : p.V * p.D;
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL(embed_copy_kernel, dim3((uint32_t)min((n + kThreads - 1) / kThreads, (int64_t)2048)), dim3(kThreads), 0,
                       stream, p.base, p.dtable, n);
    return hipGetLastError();
  }
  for (int64_t t = 0; t < p.n; t += kEmbedSlice) {
    const int64_t n = min(p.n - t, kEmbedSlice);
    embed_plan(q, n, ws);
    q.ids.p = reinterpret_cast<const char*>(p.ids.p) + t * (p.ids.wide ? 8 : 4);
    q.dout = reinterpret_cast<const char*>(p.dout) + t * p.dos * (bf16 ? 2 : 4);
    if (t > 0) q.base = p.dtable;
    const hipError_t e = bf16 ? backward<u16>(q, stream) : backward<float>(q, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace rla

// Packed tokens: which sequence each token belongs to, where sequences start,
// and which are empty; and the column sums that end the gradients of shared
// parameters.
#include "layer.hpp"

namespace rla {

namespace {

constexpr int kMapTokens = 1024;   // tokens per workgroup
constexpr int kNone = 0x7fffffff;

// Sequence n is [m_n, m_{n+1}), m_i the running maximum of the clamped offsets,
// so token t's sequence is F(t) - 1 with F(t) the first offset beyond t.  An
// offset v is beyond every token before it: F(t) is the smallest index i among
// the offsets v > t, a minimum over the tokens' places (any order of offsets,
// one pass over them).  The last workgroup takes the running maximum itself,
// for the empty sequences.
__global__ __launch_bounds__(kThreads) void token_map_kernel(const int32_t* cu, int32_t nseq, int64_t ntok,
                                                             int32_t* seq, uint32_t* starts, int32_t* empty) {
  __shared__ int32_t first[kMapTokens + 2];
  __shared__ int32_t part[kThreads];
  const int tid = threadIdx.x;
  auto offset = [&](int32_t i) {
    const int64_t v = cu[i];
    return v < 0 ? (int64_t)0 : (v > ntok ? ntok : v);
  };
  if (blockIdx.x == gridDim.x - 1) {
    int64_t before = 0;   // running maximum up to this stretch
    __shared__ int64_t top[kThreads];
    for (int64_t base = 0; base <= nseq; base += kThreads) {
      const int64_t i = base + tid;
      top[tid] = i <= nseq ? offset((int32_t)i) : 0;
      __syncthreads();
      for (int d = 1; d < kThreads; d <<= 1) {
        const int64_t o = tid >= d ? top[tid - d] : 0;
        __syncthreads();
        if (o > top[tid]) top[tid] = o;
        __syncthreads();
      }
      const int64_t below = tid ? max(before, top[tid - 1]) : before;   // m_{i-1}
      if (i >= 1 && i <= nseq) empty[i - 1] = max(below, top[tid]) == below;
      const int64_t last = top[kThreads - 1];
      __syncthreads();
      if (last > before) before = last;
    }
    return;
  }
  // places a .. a + kMapTokens of this workgroup and one for all beyond
  const int64_t a = (int64_t)blockIdx.x * kMapTokens;
  for (int j = tid; j < kMapTokens + 2; j += kThreads) first[j] = kNone;
  __syncthreads();
  for (int64_t i = tid; i <= nseq; i += kThreads) {
    const int64_t v = offset((int32_t)i);
    if (v >= a) atomicMin(&first[min(v - a, (int64_t)kMapTokens + 1)], (int32_t)i);
  }
  __syncthreads();
  // suffix minima: 4 places a thread, then over the threads behind it
  constexpr int kPer = kMapTokens / kThreads;
  int32_t own = kNone;
  for (int e = kPer - 1; e >= 0; --e) own = min(own, first[tid * kPer + e]);
  part[tid] = own;
  __syncthreads();
  for (int d = 1; d < kThreads; d <<= 1) {
    const int32_t o = tid + d < kThreads ? part[tid + d] : kNone;
    __syncthreads();
    part[tid] = min(part[tid], o);
    __syncthreads();
  }
  int32_t run = min(first[kMapTokens], first[kMapTokens + 1]);
  if (tid + 1 < kThreads) run = min(run, part[tid + 1]);
  // token a + j - 1 looks at the places from j on
  __syncthreads();
  for (int e = kPer - 1; e >= 0; --e) {
    const int j = tid * kPer + e;
    run = min(run, first[j]);
    first[j] = run;
  }
  if (tid == 0) first[kMapTokens] = min(first[kMapTokens], first[kMapTokens + 1]);
  __syncthreads();
  auto sequence = [&](int j) {   // of token a + j - 1
    const int32_t f = first[j];
    return f == kNone ? -1 : f - 1;
  };
  for (int e = 0; e < kMapTokens; e += kThreads) {
    const int64_t t = a + e + tid;
    const int s = sequence(e + tid + 1);
    if (t < ntok) seq[t] = s;
    const bool start = t >= ntok || t == 0 || s != sequence(e + tid);
    const uint64_t bits = __ballot(start);
    if ((tid & 31) == 0 && t < ntok + 64) starts[t >> 5] = (uint32_t)(bits >> (tid & 32));
  }
}

// 64 columns a workgroup, from `first` on, 16 groups of rows: a group's rows in order,
// then the groups.
constexpr int kSumGroups = 16;
__global__ __launch_bounds__(64 * kSumGroups) void column_sums_kernel(const float* part, int64_t rows, int64_t first,
                                                                      int64_t cols, int64_t inner, int32_t outer,
                                                                      float* out, float* out2) {
  __shared__ float s[kSumGroups][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t c = first + (int64_t)blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (c < cols) {
    constexpr int kAhead = 16;   // loads in flight
    int64_t r = g;
    for (; r + (kAhead - 1) * kSumGroups < rows; r += kAhead * kSumGroups) {
      float v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = part[(r + u * kSumGroups) * cols + c];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) sum += v[u];
    }
    for (; r < rows; r += kSumGroups) sum += part[r * cols + c];
  }
  s[g][lane] = sum;
  __syncthreads();
  if (g != 0 || c >= cols) return;
#pragma unroll
  for (int i = 1; i < kSumGroups; ++i) sum += s[i][lane];
  const int64_t i = c / inner, j = c % inner;
  if (i < outer) {
    if (out) out[j * outer + i] = sum;
  } else if (out2) {
    out2[j] = sum;
  }
}

__global__ __launch_bounds__(kThreads) void copy_words_kernel(const u16* src, u16* dst, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads)
    dst[i] = src ? src[i] : (u16)0;
}

}  // namespace

hipError_t launch_copy_words(const void* src, void* dst, int64_t n, hipStream_t stream) {
  hipLaunchKernelGGL(copy_words_kernel, dim3((uint32_t)min((n + kThreads - 1) / kThreads, (int64_t)1024)),
                     dim3(kThreads), 0, stream, reinterpret_cast<const u16*>(src), reinterpret_cast<u16*>(dst), n);
  return hipGetLastError();
}

hipError_t launch_token_map(const int32_t* cu, int32_t nseq, int64_t ntok, unsigned char* ws, bool build, TokenMap& map,
                            hipStream_t stream) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  int32_t* seq = reinterpret_cast<int32_t*>(ws);
  uint32_t* starts = reinterpret_cast<uint32_t*>(ws + up(4 * (size_t)ntok));
  int32_t* empty = reinterpret_cast<int32_t*>(ws + up(4 * (size_t)ntok) + up(4 * ((size_t)ntok / 32 + 3)));
  map.seq = seq;
  map.starts = starts;
  map.empty = empty;
  if (!build) return hipSuccess;
  // (the words past the last token's reach 64 tokens beyond it)
  const int64_t wgs = (ntok + 64 + kMapTokens - 1) / kMapTokens + 1;
  hipLaunchKernelGGL(token_map_kernel, dim3((uint32_t)wgs), dim3(kThreads), 0, stream, cu, nseq, ntok, seq, starts,
                     empty);
  return hipGetLastError();
}

hipError_t launch_column_sums(const float* part, int64_t rows, int64_t cols, int64_t inner, int32_t outer, float* out,
                              float* out2, hipStream_t stream) {
  // (more columns than a launch holds: several)
  constexpr int64_t most = UINT32_MAX / (64 * kSumGroups) * 64;
  for (int64_t c = 0; c < cols; c += most) {
    const int64_t wgs = (min(cols - c, most) + 63) / 64;
    hipLaunchKernelGGL(column_sums_kernel, dim3((uint32_t)wgs), dim3(64 * kSumGroups), 0, stream, part, rows, c, cols,
                       inner, outer, out, out2);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace rla

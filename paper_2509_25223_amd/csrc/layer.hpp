// Shared by the operators around a mixing layer (conv.hip, ssm*.hip,
// norm.hip) and their host side (layer_api.cpp): rows of any alignment, the
// map from tokens to sequences, launch parameters.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace rla {

// Workgroups of kThreads that a launch can have: a HIP grid holds fewer than 2^32 threads.
constexpr int64_t kMaxWgs = UINT32_MAX / kThreads;

// ---------------------------------------------------------------------------
// Rows.  V values of a row starting at p, of which n exist.  Activations are
// aligned to their elements only (odd channel counts, slices of projections):
// gfx950 loads 16 bytes from any address, so a whole piece is one access, and
// only a row's last piece is read value by value.
// ---------------------------------------------------------------------------
template <typename T, int V> struct RowVec {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
// (as stored: what is loaded ahead is converted where it is used)
template <typename T, int V, bool FULL = false>
__device__ __forceinline__ void load_raw(const T* p, int n, typename RowVec<T, V>::type& x) {
  if (FULL || n >= V) {
    x = *reinterpret_cast<const typename RowVec<T, V>::type*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = e < n ? p[e] : from_f<T>(0.f);
  }
}
template <typename T, int V, bool FULL = false>
__device__ __forceinline__ void load_piece(const T* p, int n, float (&x)[V]) {
  if (FULL || n >= V) {
    const typename RowVec<T, V>::type v = *reinterpret_cast<const typename RowVec<T, V>::type*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = to_f<T>(v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = e < n ? to_f<T>(p[e]) : 0.f;
  }
}
template <typename T, int V, bool FULL = false, bool NT = false>
__device__ __forceinline__ void store_piece(T* p, int n, const float (&x)[V]) {
  if (FULL || n >= V) {
    typename RowVec<T, V>::type v;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = from_f<T>(x[e]);
    if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<typename RowVec<T, V>::type*>(p));
    else *reinterpret_cast<typename RowVec<T, V>::type*>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) p[e] = from_f<T>(x[e]);
  }
}
// NT: calls that write more than this much store it non-temporally, past the caches that
// the inputs come through: writing 201 MB of a convolution's output in 86 us, not 96,
// its gradients' 201 MB in 150, not 162, the residual addition's 201 and 201 MB in 85 and
// 182, not 88 and 195; but 67 MB of a gated norm in 35 us, not 32.
constexpr int64_t kNtBytes = (int64_t)96 << 20;

// values of a 16-byte piece
template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);

// 1 / (1 + e^-z), the reciprocal by v_rcp_f32 (1 ulp; a rounded division is ten
// instructions)
__device__ __forceinline__ float sigmoid_fast(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
// SiLU'(z), and SiLU(z)
__device__ __forceinline__ float silu_grad_f(float z, float& silu) {
  const float s = sigmoid_fast(z);
  silu = z * s;
  return s * __builtin_fmaf(z, 1.f - s, 1.f);
}

// ---------------------------------------------------------------------------
// Tokens and sequences.  Dense: sequence t / T.  Packed: a map built per call
// in the workspace (launch_token_map): seq[t], -1 outside every sequence;
// starts: bit t set where token t's sequence is not token t - 1's (and for t =
// 0), bits past the end set; empty[n]: sequence n has no token.
// ---------------------------------------------------------------------------
// (constant while a kernel reads it: address space 4, scalar loads where t is uniform)
template <typename T> using ConstPtr = const __attribute__((address_space(4))) T*;
struct TokenMap {
  int64_t ntok = 0, T = 1;           // dense: tokens per sequence (packed: unused)
  int32_t nseq = 0;
  const int32_t* seq = nullptr;      // packed
  const uint32_t* starts = nullptr;
  const int32_t* empty = nullptr;

  __device__ __forceinline__ int seq_of(int64_t t) const {
    return seq ? ((ConstPtr<int32_t>)(uint64_t)seq)[t] : (int)((uint32_t)t / (uint32_t)T);
  }
  // start bits of tokens t .. t + 31
  __device__ __forceinline__ uint32_t start_bits(int64_t t) const {
    if (seq) {
      const uint32_t w = (uint32_t)t >> 5, s = (uint32_t)t & 31u;
      const ConstPtr<uint32_t> words = (ConstPtr<uint32_t>)(uint64_t)starts;
      const uint64_t two = (uint64_t)words[w] | ((uint64_t)words[w + 1] << 32);
      return (uint32_t)(two >> s);
    }
    const uint32_t r = (uint32_t)t % (uint32_t)T;
    uint32_t bits = 0;
    for (int64_t i = r == 0 ? 0 : T - r; i < 32; i += T) bits |= 1u << i;
    const int64_t left = ntok - t;
    return left >= 32 ? bits : bits | (~0u << (left < 0 ? 0 : left));
  }
};
inline size_t token_map_bytes(int64_t ntok, int64_t nseq) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  return up(4 * (size_t)ntok) + up(4 * ((size_t)ntok / 32 + 3)) + up(4 * (size_t)nseq);
}
// Points `map` (packed) at its arrays in ws; `build`: launches what fills them.
hipError_t launch_token_map(const int32_t* cu, int32_t nseq, int64_t ntok, unsigned char* ws, bool build,
                            TokenMap& map, hipStream_t stream);

// ---------------------------------------------------------------------------
// Sums over the rows of part [rows][cols]: the last step of every gradient of
// a shared parameter (fixed order).  Column i * inner + j goes to out[j * outer
// + i] for i < outer, else to out2[j] (NULL: dropped).
// ---------------------------------------------------------------------------
hipError_t launch_column_sums(const float* part, int64_t rows, int64_t cols, int64_t inner, int32_t outer, float* out,
                              float* out2, hipStream_t stream);

struct ConvParams {
  TokenMap map;
  const int32_t* cu = nullptr;   // packed sequences few enough to be looked up in place (no map)
  int64_t D = 0, xs = 0, dys = 0;
  int32_t taps = 4, silu = 0;
  const void* x = nullptr;
  const float* weight = nullptr;
  const float* bias = nullptr;
  const void* state0 = nullptr;
  void* y = nullptr;
  void* state_fin = nullptr;
  const void* dy = nullptr;
  const void* dstate_fin = nullptr;
  void* dx = nullptr;
  void* dstate0 = nullptr;
  float* part = nullptr;   // [tiles][taps + 1][D] sums of dweight, dbias
};
// Up to this many packed sequences a thread goes through the offsets itself; more, and
// the map is built once a call.  20011 tokens of bf16, us in place / from a map (with the
// launch that builds it):
//   sequences                        8           16           24           32           64
//   2048 channels, forward   47.3/51.5    48.9/52.1    49.4/51.8    51.1/51.3    57.6/52.6
//              gradients     69.5/73.0    73.8/76.0    74.5/76.2    75.4/74.7    93.7/85.0
//   512, forward             18.0/23.5    18.9/23.8    19.6/23.6    21.2/23.7    27.4/23.7
//   6144, forward           100.5/108.2  105.7/110.4  108.2/111.1  107.5/108.8  123.8/110.5
constexpr int32_t kConvInPlace = 24;
hipError_t launch_conv_forward(const ConvParams& p, bool bf16, hipStream_t stream);
hipError_t launch_conv_decode(const ConvParams& p, bool bf16, hipStream_t stream);
int64_t conv_backward_rows(int64_t ntok, int64_t D);
// few enough workgroups for a launch
bool conv_forward_fits(const ConvParams& p, bool bf16);
bool conv_backward_fits(const ConvParams& p);
bool conv_decode_fits(const ConvParams& p, bool bf16);
hipError_t launch_conv_backward(const ConvParams& p, bool bf16, float* dweight, float* dbias, hipStream_t stream);

// dst = src (NULL: zeros), `n` 16-bit words
hipError_t launch_copy_words(const void* src, void* dst, int64_t n, hipStream_t stream);

struct AddNormParams {
  int64_t rows = 0, width = 0, xs = 0, dns = 0, wgs = 0;
  float eps = 0.f;
  const void* x = nullptr;
  const void* residual = nullptr;
  const float* weight = nullptr;
  const float* scale = nullptr;
  void* n = nullptr;
  void* residual_out = nullptr;
  const void* residual_in = nullptr;   // backward: the forward's residual_out
  const void* dn = nullptr;
  const void* dresidual_out = nullptr;
  void* dx = nullptr;
  void* dresidual = nullptr;
  float* part = nullptr;               // [wgs][1, or 2 with scale][width]
};
int64_t addnorm_backward_wgs(int64_t rows, int64_t width, bool bf16);
hipError_t launch_addnorm(const AddNormParams& p, bool bf16, bool res_bf16, bool backward, hipStream_t stream);

struct GateNormParams {
  int64_t rows = 0, heads = 1, width = 0, xs = 0, gs = 0, dos = 0, wstride = 0, groups = 0;
  float eps = 0.f;
  int32_t first = 0;
  const void* x = nullptr;
  const void* gate = nullptr;
  const float* weight = nullptr;
  void* o = nullptr;
  const void* dO = nullptr;
  void* dx = nullptr;
  void* dgate = nullptr;
  float* part = nullptr;
};
// Groups of lanes in the backward, and the rows of its partial sums.
int64_t gatenorm_backward_groups(int64_t rows, int64_t heads, int64_t width, bool bf16, int64_t& part_rows, bool per_head);
hipError_t launch_gatenorm(const GateNormParams& p, bool bf16, bool x_bf16, bool backward, hipStream_t stream);

}  // namespace rla

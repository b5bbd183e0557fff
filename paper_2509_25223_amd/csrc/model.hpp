// Shared by the operators at a language model's ends and the gated linear
// recurrence (embed.hip, logprob.hip, glr.hip) and their host side
// (model_api.cpp): launch parameters and plans of their workspaces.
#pragma once

#include "layer.hpp"

namespace rla {

// Token ids as given: int64 or int32.
struct Ids {
  const void* p = nullptr;
  int32_t wide = 0;
  __device__ __forceinline__ int64_t operator[](int64_t t) const {
    return wide ? reinterpret_cast<const int64_t*>(p)[t] : (int64_t)reinterpret_cast<const int32_t*>(p)[t];
  }
};

// ---------------------------------------------------------------------------
// embedding
// ---------------------------------------------------------------------------
struct EmbedParams {
  int64_t n = 0, V = 1, D = 1, dos = 0;
  float scale = 1.f;
  Ids ids;
  const void* table = nullptr;
  void* out = nullptr;
  const void* dout = nullptr;
  const float* base = nullptr;
  float* dtable = nullptr;
  // the gradient's workspace: a slice of tokens sorted by id in two passes
  int32_t bits1 = 0, bits2 = 0;        // digits of the two passes
  int32_t tile = 0, tiles = 0;         // tokens a workgroup sorts, and how many do
  int32_t chunk = 0, chunks = 0;       // sorted tokens a group of lanes sums, and how many do
  int32_t* count1 = nullptr;           // [tiles][2^bits1]
  int32_t* count2 = nullptr;           // [tiles][2^bits2]
  uint32_t* present = nullptr;         // bit v: a token points at row v
  int32_t *key1 = nullptr, *pos1 = nullptr, *key = nullptr, *pos = nullptr;
  float* part = nullptr;               // [chunks][2][D]
};
// Tokens of a call are taken in slices of this many (one for nearly all calls), later ones
// added in place.
constexpr int64_t kEmbedSlice = (int64_t)1 << 22;
size_t embed_plan(EmbedParams& p, int64_t tokens, unsigned char* ws);   // sets the fields above; returns the bytes
hipError_t launch_embed_forward(const EmbedParams& p, bool table_bf16, bool bf16, hipStream_t stream);
hipError_t launch_embed_backward(const EmbedParams& p, bool bf16, unsigned char* ws, hipStream_t stream);

// ---------------------------------------------------------------------------
// log probabilities
// ---------------------------------------------------------------------------
constexpr int kMaxTop = 64;
struct LogprobParams {
  int64_t n = 0, V = 1, xs = 0;
  float scale = 1.f;
  int32_t top = 0;
  Ids targets;
  const void* x = nullptr;
  float *logprob = nullptr, *lse = nullptr, *entropy = nullptr, *top_lp = nullptr;
  int32_t* top_ids = nullptr;
  // rows in parts (one: no workspace)
  int64_t parts = 1, width = 0;        // values of a part
  float* stat = nullptr;               // [n][parts][4]: largest, sum, sum of products
  float* cand_x = nullptr;             // [n][parts][top]
  int32_t* cand_i = nullptr;
  // backward
  const float *lse_in = nullptr, *entropy_in = nullptr, *dlogprob = nullptr, *dentropy = nullptr;
  void* dx = nullptr;
};
size_t logprob_plan(LogprobParams& p, bool bf16, unsigned char* ws);
hipError_t launch_logprob_forward(const LogprobParams& p, bool bf16, hipStream_t stream);
hipError_t launch_logprob_backward(const LogprobParams& p, bool bf16, hipStream_t stream);

// ---------------------------------------------------------------------------
// gated linear recurrence
// ---------------------------------------------------------------------------
struct GlrParams {
  TokenMap map;
  int64_t D = 0, xs = 0, rs = 0, is = 0, zs = 0, dos = 0;
  int32_t normalize = 0;
  const void *x = nullptr, *r = nullptr, *i = nullptr, *z = nullptr;
  const float *A = nullptr, *h0 = nullptr;
  void* o = nullptr;
  float* hfin = nullptr;
  const void* dO = nullptr;
  const float* dhfin = nullptr;
  void *dx = nullptr, *dr = nullptr, *di = nullptr, *dz = nullptr;
  float *dA = nullptr, *dh0 = nullptr;
  // all tokens in chunks of L, of `tiles` tiles each
  int64_t L = 0;
  int32_t nchunk = 0, tiles = 0;
  int32_t apart = 0;                   // every chunk starts with a sequence: none needs another's state
  int64_t room_sum = 0, room_chunks = 0, room_tiles = 0;   // rows of D that the workspace has for sum (two each), pA, ck
  float* sum = nullptr;                // [nchunk][2][D]: a chunk's decay and state from zeros (forward, then backward)
  float* ck = nullptr;                 // [nchunk][tiles][D]: states before the tiles
  float* pA = nullptr;                 // [nchunk][D]
};
constexpr int kGlrChannels = 64;       // of a workgroup
void glr_plan(GlrParams& p, bool packed);   // the chunks: some hundred workgroups, or one for each 64 channels
int64_t glr_decode_wgs(const GlrParams& p);
hipError_t launch_glr_forward(const GlrParams& p, bool bf16, bool save, bool outputs, hipStream_t stream);
hipError_t launch_glr_backward(const GlrParams& p, bool bf16, hipStream_t stream);
hipError_t launch_glr_decode(const GlrParams& p, bool bf16, hipStream_t stream);

}  // namespace rla

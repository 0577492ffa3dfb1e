// Host-side launch interface of the sequence operators (internal to the library):
// embedding.hip, gated_scan.hip and token_scores.hip. The callers have checked
// sizes, types and alignment.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace dlvm {

hipError_t launch_embedding_forward(int dtype, int64_t vocab, int64_t width, int64_t tokens,
                                    const void* table, const int32_t* ids, float scale, void* out,
                                    hipStream_t s);
size_t embedding_backward_ws(int64_t vocab, int64_t width, int64_t tokens);
hipError_t launch_embedding_backward(int dtype, int64_t vocab, int64_t width, int64_t tokens,
                                     const int32_t* ids, const void* dout, float scale,
                                     bool accumulate, float* dtable, void* ws, hipStream_t s);

// One call of the gated recurrence; the backward fields are null in a forward call.
struct GatedScan {
  int dtype;
  bool coupled;
  int64_t T, B, H;
  const void* z; int64_t ldz;
  const void* x; int64_t ldx;
  const float* h0;       // [B, H] or null
  const int32_t* lens;   // [B] or null
  void* hs; int64_t ldh; // written by the forward call, read by the backward call
  float* hT;             // forward: [B, H] or null
  const void* dhs; int64_t lddh;
  const float* dhT;
  void* dz; int64_t lddz;
  void* dx; int64_t lddx;
  float* dh0;
};
size_t gated_scan_ws(int dtype, int64_t T, int64_t B, int64_t H);
hipError_t launch_gated_scan_forward(const GatedScan& c, void* ws, hipStream_t s);
hipError_t launch_gated_scan_backward(const GatedScan& c, void* ws, hipStream_t s);

constexpr int kTopMax = 32;
// One call of the token scores.
struct TokenScores {
  int dtype;
  int64_t rows, classes;
  const void* logits; int64_t ld;
  float scale;
  const int32_t* tokens;
  float* logp;
  float* lse;
  float* entropy;
  int top;
  int32_t* top_ids;
  float* top_logp;
};
size_t token_scores_ws(int64_t rows, int64_t classes, int top);
hipError_t launch_token_scores(const TokenScores& c, void* ws, hipStream_t s);
hipError_t launch_token_scores_backward(int dtype, int out_dtype, int64_t rows, int64_t classes,
                                        const void* logits, int64_t ld, float scale,
                                        const int32_t* tokens, const float* lse,
                                        const float* entropy, const float* dlogp,
                                        const float* dentropy, void* dlogits, int64_t ld_out,
                                        hipStream_t s);

}  // namespace dlvm

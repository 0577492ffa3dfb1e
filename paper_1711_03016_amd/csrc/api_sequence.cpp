// C ABI of the sequence operators: argument checks of the token embeddings, the
// gated linear recurrence and the token scores, and the calls of their launches.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <initializer_list>

#include "dlvm.h"
#include "api_common.hpp"
#include "sequence.hpp"

using namespace dlvm::api;

namespace {

constexpr int64_t kMaxVocab = int64_t(1) << 24;
constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxWidth = int64_t(1) << 20;
constexpr int64_t kMaxRows = INT32_MAX;
// Strides beyond this could take a row's offset past 63 bits.
constexpr int64_t kMaxStride = int64_t(1) << 31;
// The scale of scores is multiplied by log2(e) in float32.
constexpr float kMaxScale = 2e38f;

dlvm_status embedding_sizes(int32_t dtype, int64_t vocab, int64_t width, int64_t tokens, float scale) {
  if (!valid_dtype(dtype)) return fail(DLVM_ERR_INVALID_ARG, "bad dtype");
  if (vocab < 1 || width < 1 || tokens < 1) return fail(DLVM_ERR_INVALID_ARG, "sizes must be positive");
  if (!std::isfinite(scale)) return fail(DLVM_ERR_INVALID_ARG, "scale must be finite");
  if (vocab > kMaxVocab || width > kMaxWidth || tokens > kMaxTokens)
    return fail(DLVM_ERR_UNSUPPORTED, "vocab at most 2^24, width at most 2^20, tokens at most 2^30");
  return DLVM_OK;
}

bool scan_fits(int64_t steps, int64_t batch, int64_t width) {
  return steps <= (int64_t(1) << 30) && batch <= INT32_MAX && width <= INT32_MAX &&
         batch * width <= INT32_MAX && batch * steps <= INT32_MAX;
}

dlvm_status scan_sizes(int32_t dtype, int32_t mode, int64_t steps, int64_t batch, int64_t width) {
  if (!valid_dtype(dtype)) return fail(DLVM_ERR_INVALID_ARG, "bad dtype");
  if (mode != DLVM_SCAN_FREE && mode != DLVM_SCAN_COUPLED) return fail(DLVM_ERR_INVALID_ARG, "bad mode");
  if (steps < 1 || batch < 1 || width < 1) return fail(DLVM_ERR_INVALID_ARG, "sizes must be positive");
  if (!scan_fits(steps, batch, width))
    return fail(DLVM_ERR_UNSUPPORTED, "batch * width and batch * steps at most 2^31 - 1, steps at most 2^30");
  return DLVM_OK;
}

dlvm_status scan_stride(int64_t ld, int64_t width) {
  if (ld < width) return fail(DLVM_ERR_INVALID_ARG, "row strides must be at least the width");
  // the rows that 64 neighbouring states lie in are addressed with 32 bits
  if (ld > kMaxStride || (63 / width + 1) * ld > (int64_t(1) << 30) - 1)
    return fail(DLVM_ERR_UNSUPPORTED, "row strides times the rows that hold 64 states at most 2^30");
  return DLVM_OK;
}

dlvm_status score_sizes(int32_t dtype, int64_t rows, int64_t classes, int64_t ld, float scale) {
  if (!valid_dtype(dtype)) return fail(DLVM_ERR_INVALID_ARG, "bad dtype");
  if (rows < 1 || classes < 1) return fail(DLVM_ERR_INVALID_ARG, "sizes must be positive");
  if (ld < classes) return fail(DLVM_ERR_INVALID_ARG, "the row stride must be at least the classes");
  if (!std::isfinite(scale) || scale <= 0) return fail(DLVM_ERR_INVALID_ARG, "scale must be finite and positive");
  if (rows > kMaxRows || classes > (int64_t(1) << 30) || ld > kMaxStride)
    return fail(DLVM_ERR_UNSUPPORTED, "rows below 2^31, classes at most 2^30, row strides at most 2^31");
  if (scale > kMaxScale) return fail(DLVM_ERR_UNSUPPORTED, "scale at most 2e38");
  return DLVM_OK;
}

template <typename... P> bool all_aligned16(const P*... p) { return (aligned16(p) && ...); }

// Where a tensor lies: rows of `row` bytes, `pitch` bytes from one to the next.
struct Span {
  const void* at;
  __int128 rows, row, pitch;
};
Span piece(const void* at, int64_t count, size_t size) {
  const __int128 bytes = static_cast<__int128>(count) * static_cast<int64_t>(size);
  return Span{at, 1, bytes, bytes};
}
Span strided(const void* at, int dtype, int64_t rows, int64_t width, int64_t ld) {
  const int64_t e = static_cast<int64_t>(elem_size(dtype));
  if (ld == width) return piece(at, rows * width, elem_size(dtype));
  return Span{at, rows, static_cast<__int128>(width) * e, static_cast<__int128>(ld) * e};
}

// Whether two tensors share a byte; null ones do not. Rows of one stride may lie between those of
// the other tensor (the halves of a product). Rows of two strides are not followed: they are
// taken as apart unless they start together.
bool share(Span a, Span b) {
  if (a.at == nullptr || b.at == nullptr) return false;
  const __int128 d = static_cast<__int128>(reinterpret_cast<uintptr_t>(b.at)) -
                     static_cast<__int128>(reinterpret_cast<uintptr_t>(a.at));  // b begins d after a
  const auto length = [](const Span& s) { return (s.rows - 1) * s.pitch + s.row; };
  if (d >= length(a) || -d >= length(b)) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  // one row: of the other's pitch if it fits between two of its rows, else it meets one
  Span* const one = a.rows == 1 ? &a : b.rows == 1 ? &b : nullptr;
  if (one != nullptr) {
    const Span& many = one == &a ? b : a;
    if (one->row > many.pitch - many.row) return true;
    one->pitch = many.pitch;
  }
  if (a.pitch != b.pitch) return d == 0;
  __int128 q = d / a.pitch, r = d % a.pitch;  // row j of b begins r bytes after row j + q of a does
  if (r < 0) {
    r += a.pitch;
    q -= 1;
  }
  const auto meet = [&](__int128 k) { return k > -b.rows && k < a.rows; };  // a row j of b and row j + k of a
  return (r < a.row && meet(q)) || (r + b.row > a.pitch && meet(q + 1));
}

// Whether no output shares memory with an input or another output.
bool apart(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
  for (const Span* o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Span& i : inputs)
      if (share(*o, i)) return false;
    for (const Span* p = outputs.begin(); p != o; ++p)
      if (share(*o, *p)) return false;
  }
  return true;
}

dlvm_status overlap() { return fail(DLVM_ERR_INVALID_ARG, "an output must not overlap an input or another output"); }

dlvm_status misaligned() {
  return fail(DLVM_ERR_MISALIGNED, "device pointers must be 16-byte aligned");
}

}  // namespace

extern "C" {

dlvm_status dlvm_embedding_forward(int32_t dtype, int64_t vocab, int64_t width, int64_t tokens,
                                   const void* table, const int32_t* ids, float scale, void* out,
                                   void* stream) {
  const dlvm_status st = embedding_sizes(dtype, vocab, width, tokens, scale);
  if (st != DLVM_OK) return st;
  if (table == nullptr || ids == nullptr || out == nullptr)
    return fail(DLVM_ERR_INVALID_ARG, "null argument");
  if (!all_aligned16(table, ids, out)) return misaligned();
  if (!apart({strided(out, dtype, tokens, width, width)},
             {strided(table, dtype, vocab, width, width), piece(ids, tokens, 4)}))
    return overlap();
  const hipError_t e = dlvm::launch_embedding_forward(dtype, vocab, width, tokens, table, ids, scale,
                                                      out, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DLVM_OK : hip_fail(e, "embedding launch");
}

size_t dlvm_embedding_backward_ws_bytes(int64_t vocab, int64_t width, int64_t tokens) {
  if (vocab < 1 || width < 1 || tokens < 1 || vocab > kMaxVocab || width > kMaxWidth ||
      tokens > kMaxTokens)
    return 0;
  return dlvm::embedding_backward_ws(vocab, width, tokens);
}

dlvm_status dlvm_embedding_backward(int32_t dtype, int64_t vocab, int64_t width, int64_t tokens,
                                    const int32_t* ids, const void* dout, float scale,
                                    int32_t accumulate, float* dtable, void* ws, size_t ws_bytes,
                                    void* stream) {
  const dlvm_status st = embedding_sizes(dtype, vocab, width, tokens, scale);
  if (st != DLVM_OK) return st;
  if (accumulate != 0 && accumulate != 1) return fail(DLVM_ERR_INVALID_ARG, "accumulate is 0 or 1");
  if (ids == nullptr || dout == nullptr || dtable == nullptr)
    return fail(DLVM_ERR_INVALID_ARG, "null argument");
  if (ws == nullptr || ws_bytes < dlvm::embedding_backward_ws(vocab, width, tokens))
    return fail(DLVM_ERR_WORKSPACE, "workspace missing or too small");
  if (!all_aligned16(ids, dout, dtable, ws)) return misaligned();
  if (!apart({piece(dtable, vocab * width, 4),
              piece(ws, static_cast<int64_t>(dlvm::embedding_backward_ws(vocab, width, tokens)), 1)},
             {piece(ids, tokens, 4), strided(dout, dtype, tokens, width, width)}))
    return overlap();
  const hipError_t e = dlvm::launch_embedding_backward(dtype, vocab, width, tokens, ids, dout, scale,
                                                       accumulate != 0, dtable, ws,
                                                       static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DLVM_OK : hip_fail(e, "embedding gradient launch");
}

size_t dlvm_gated_scan_ws_bytes(int32_t dtype, int64_t steps, int64_t batch, int64_t width) {
  if (!valid_dtype(dtype) || steps < 1 || batch < 1 || width < 1 || !scan_fits(steps, batch, width))
    return 0;
  return dlvm::gated_scan_ws(dtype, steps, batch, width);
}

dlvm_status dlvm_gated_scan_forward(int32_t dtype, int32_t mode, int64_t steps, int64_t batch,
                                    int64_t width, const void* z, int64_t ldz, const void* x,
                                    int64_t ldx, const float* h0, const int32_t* lens, void* hs,
                                    int64_t ldh, float* hT, void* ws, size_t ws_bytes,
                                    void* stream) {
  dlvm_status st = scan_sizes(dtype, mode, steps, batch, width);
  for (const int64_t ld : {ldz, ldx, ldh})
    if (st == DLVM_OK) st = scan_stride(ld, width);
  if (st != DLVM_OK) return st;
  if (z == nullptr || x == nullptr || hs == nullptr) return fail(DLVM_ERR_INVALID_ARG, "null argument");
  if (ws != nullptr && ws_bytes < dlvm::gated_scan_ws(dtype, steps, batch, width))
    return fail(DLVM_ERR_WORKSPACE, "workspace is smaller than dlvm_gated_scan_ws_bytes");
  if (!all_aligned16(z, x, h0, lens, hs, hT, ws)) return misaligned();
  const int64_t rows = steps * batch, states = batch * width;
  if (!apart({strided(hs, dtype, rows, width, ldh), piece(hT, states, 4),
              piece(ws, static_cast<int64_t>(dlvm::gated_scan_ws(dtype, steps, batch, width)), 1)},
             {strided(z, dtype, rows, width, ldz), strided(x, dtype, rows, width, ldx),
              piece(h0 == hT ? nullptr : h0, states, 4), piece(lens, batch, 4)}))
    return overlap();
  dlvm::GatedScan c{};
  c.dtype = dtype;
  c.coupled = mode == DLVM_SCAN_COUPLED;
  c.T = steps; c.B = batch; c.H = width;
  c.z = z; c.ldz = ldz; c.x = x; c.ldx = ldx;
  c.h0 = h0; c.lens = lens;
  c.hs = hs; c.ldh = ldh; c.hT = hT;
  const hipError_t e = dlvm::launch_gated_scan_forward(c, ws, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DLVM_OK : hip_fail(e, "gated scan launch");
}

dlvm_status dlvm_gated_scan_backward(int32_t dtype, int32_t mode, int64_t steps, int64_t batch,
                                     int64_t width, const void* z, int64_t ldz, const void* x,
                                     int64_t ldx, const float* h0, const int32_t* lens,
                                     const void* hs, int64_t ldh, const void* dhs, int64_t lddh,
                                     const float* dhT, void* dz, int64_t lddz, void* dx,
                                     int64_t lddx, float* dh0, void* ws, size_t ws_bytes,
                                     void* stream) {
  dlvm_status st = scan_sizes(dtype, mode, steps, batch, width);
  for (const int64_t ld : {ldz, ldx, ldh, dhs ? lddh : width, lddz, lddx})
    if (st == DLVM_OK) st = scan_stride(ld, width);
  if (st != DLVM_OK) return st;
  if (z == nullptr || x == nullptr || hs == nullptr || dz == nullptr || dx == nullptr)
    return fail(DLVM_ERR_INVALID_ARG, "null argument");
  if (dhs == nullptr && dhT == nullptr)
    return fail(DLVM_ERR_INVALID_ARG, "one of dhs and dhT is required");
  if (ws != nullptr && ws_bytes < dlvm::gated_scan_ws(dtype, steps, batch, width))
    return fail(DLVM_ERR_WORKSPACE, "workspace is smaller than dlvm_gated_scan_ws_bytes");
  if (!all_aligned16(z, x, h0, lens, hs, dhs, dhT, dz, dx, dh0, ws)) return misaligned();
  const int64_t rows = steps * batch, states = batch * width;
  if (!apart({strided(dz, dtype, rows, width, lddz), strided(dx, dtype, rows, width, lddx), piece(dh0, states, 4),
              piece(ws, static_cast<int64_t>(dlvm::gated_scan_ws(dtype, steps, batch, width)), 1)},
             {strided(z, dtype, rows, width, ldz), strided(x, dtype, rows, width, ldx),
              strided(hs, dtype, rows, width, ldh), strided(dhs, dtype, rows, width, lddh),
              piece(h0, states, 4), piece(lens, batch, 4), piece(dhT == dh0 ? nullptr : dhT, states, 4)}))
    return overlap();
  dlvm::GatedScan c{};
  c.dtype = dtype;
  c.coupled = mode == DLVM_SCAN_COUPLED;
  c.T = steps; c.B = batch; c.H = width;
  c.z = z; c.ldz = ldz; c.x = x; c.ldx = ldx;
  c.h0 = h0; c.lens = lens;
  c.hs = const_cast<void*>(hs); c.ldh = ldh;
  c.dhs = dhs; c.lddh = lddh; c.dhT = dhT;
  c.dz = dz; c.lddz = lddz; c.dx = dx; c.lddx = lddx; c.dh0 = dh0;
  const hipError_t e = dlvm::launch_gated_scan_backward(c, ws, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DLVM_OK : hip_fail(e, "gated scan gradient launch");
}

size_t dlvm_token_logprobs_ws_bytes(int64_t rows, int64_t classes, int32_t top) {
  if (rows < 1 || classes < 1 || rows > kMaxRows || classes > (int64_t(1) << 30) || top < 0 ||
      top > DLVM_TOP_MAX || top > classes)
    return 0;
  return dlvm::token_scores_ws(rows, classes, top);
}

dlvm_status dlvm_token_logprobs(int32_t dtype, int64_t rows, int64_t classes, const void* logits,
                                int64_t ld, float scale, const int32_t* tokens, float* logp,
                                float* lse, float* entropy, int32_t top, int32_t* top_ids,
                                float* top_logp, void* ws, size_t ws_bytes, void* stream) {
  const dlvm_status st = score_sizes(dtype, rows, classes, ld, scale);
  if (st != DLVM_OK) return st;
  if (top < 0 || top > DLVM_TOP_MAX || top > classes)
    return fail(DLVM_ERR_INVALID_ARG, "top must be in [0, 32] and at most the classes");
  if (logits == nullptr || (tokens == nullptr) != (logp == nullptr) ||
      (top > 0) != (top_ids != nullptr) || (top > 0) != (top_logp != nullptr))
    return fail(DLVM_ERR_INVALID_ARG, "null argument (tokens and logp, top_ids and top_logp go together)");
  if (logp == nullptr && lse == nullptr && entropy == nullptr && top == 0)
    return fail(DLVM_ERR_INVALID_ARG, "no output is asked for");
  if (ws != nullptr && ws_bytes < dlvm::token_scores_ws(rows, classes, top))
    return fail(DLVM_ERR_WORKSPACE, "workspace is smaller than dlvm_token_logprobs_ws_bytes");
  if (!all_aligned16(logits, tokens, logp, lse, entropy, top_ids, top_logp, ws)) return misaligned();
  if (!apart({piece(logp, rows, 4), piece(lse, rows, 4), piece(entropy, rows, 4), piece(top_ids, rows * top, 4),
              piece(top_logp, rows * top, 4),
              piece(ws, static_cast<int64_t>(dlvm::token_scores_ws(rows, classes, top)), 1)},
             {strided(logits, dtype, rows, classes, ld), piece(tokens, rows, 4)}))
    return overlap();
  const dlvm::TokenScores c{dtype, rows, classes, logits, ld, scale, tokens, logp, lse, entropy,
                            top, top_ids, top_logp};
  const hipError_t e = dlvm::launch_token_scores(c, ws, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DLVM_OK : hip_fail(e, "token scores launch");
}

dlvm_status dlvm_token_logprobs_backward(int32_t dtype, int32_t out_dtype, int64_t rows,
                                         int64_t classes, const void* logits, int64_t ld,
                                         float scale, const int32_t* tokens, const float* lse,
                                         const float* entropy, const float* dlogp,
                                         const float* dentropy, void* dlogits, int64_t ld_out,
                                         void* stream) {
  dlvm_status st = score_sizes(dtype, rows, classes, ld, scale);
  if (st == DLVM_OK) st = score_sizes(out_dtype, rows, classes, ld_out, scale);
  if (st != DLVM_OK) return st;
  if (dtype == DLVM_BF16 && out_dtype != DLVM_BF16)
    return fail(DLVM_ERR_UNSUPPORTED, "bf16 logits give a bf16 gradient");
  if (logits == nullptr || lse == nullptr || dlogits == nullptr)
    return fail(DLVM_ERR_INVALID_ARG, "null argument");
  if (dlogp == nullptr && dentropy == nullptr)
    return fail(DLVM_ERR_INVALID_ARG, "one of dlogp and dentropy is required");
  if ((dlogp != nullptr && tokens == nullptr) || (dentropy != nullptr && entropy == nullptr))
    return fail(DLVM_ERR_INVALID_ARG, "dlogp needs tokens, and dentropy needs entropy");
  if (dlogits == logits && (dtype != out_dtype || ld != ld_out))
    return fail(DLVM_ERR_INVALID_ARG, "a gradient in place has the type and stride of the logits");
  if (!all_aligned16(logits, tokens, lse, entropy, dlogp, dentropy, dlogits)) return misaligned();
  if (!apart({strided(dlogits, out_dtype, rows, classes, ld_out)},
             {strided(dlogits == logits ? nullptr : logits, dtype, rows, classes, ld), piece(tokens, rows, 4),
              piece(lse, rows, 4), piece(entropy, rows, 4), piece(dlogp, rows, 4), piece(dentropy, rows, 4)}))
    return overlap();
  const hipError_t e = dlvm::launch_token_scores_backward(dtype, out_dtype, rows, classes, logits, ld,
                                                          scale, tokens, lse, entropy, dlogp,
                                                          dentropy, dlogits, ld_out,
                                                          static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DLVM_OK : hip_fail(e, "token scores gradient launch");
}

}  // extern "C"

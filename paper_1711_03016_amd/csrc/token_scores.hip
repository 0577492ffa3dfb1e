// Scores of tokens under rows of logits: log probabilities of given tokens,
// log-sum-exp, entropy and the largest alternatives, and the gradient of the log
// probabilities and the entropy.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace dlvm {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// The order of alternatives as whole numbers: greater is better. NaN counts as
// -infinity and -0 as 0; among equal logits the lower class is greater.
__device__ __forceinline__ uint64_t rank_key(float z, uint32_t c) {
  if (z != z) z = -INFINITY;
  const uint32_t u = __float_as_uint(z + 0.0f);
  const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return (static_cast<uint64_t>(k) << 32) | (0xffffffffu - c);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t k = static_cast<uint32_t>(key >> 32);
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
__device__ __forceinline__ uint32_t key_class(uint64_t key) {
  return 0xffffffffu - static_cast<uint32_t>(key);
}

// A part of a row: the maximum m of its logits and, with y = (z - m) scale log2(e)
// (differences of the logits themselves: a product rounded before the subtraction is
// off by as much as the exponent where logits are as large as the type's lowest value),
// s = sum 2^y and w = sum 2^y y. All terms of w have one sign, so that the entropy
// log s - w / s has no cancellation beyond its own size. y is clamped to a finite
// value where a class is masked, so that its term is 0 and not 0 times infinity.
struct Part {
  float m, s, w;
};
// Nothing left: every class is masked, by -infinity or by the type's lowest value.
__device__ __forceinline__ bool masked_everywhere(const Part& p, float scale) {
  return p.s == 0.0f || (p.s == p.s && p.m * scale < -1e30f);
}
__device__ __forceinline__ float below(float z, float m, float c2) {
  return fmaxf((z - m) * c2, -1e30f);
}
__device__ __forceinline__ Part join(const Part& a, const Part& b, float c2) {
  const float m = fmaxf(a.m, b.m);
  Part r{m, 0.0f, 0.0f};
  if (a.s != 0.0f) {
    const float d = below(a.m, m, c2), e = exp2f(d);
    r.s += a.s * e;
    r.w += (a.w + d * a.s) * e;
  }
  if (b.s != 0.0f) {
    const float d = below(b.m, m, c2), e = exp2f(d);
    r.s += b.s * e;
    r.w += (b.w + d * b.s) * e;
  }
  return r;
}

template <typename T>
__global__ __launch_bounds__(256) void dlvm_token_scores_kernel(TokenScores k) {
  __shared__ Part parts[256];
  __shared__ uint64_t best[256];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int64_t V = k.classes;
  const T* z = static_cast<const T*>(k.logits) + row * k.ld;
  const float c2 = k.scale * kLog2e;
  Part p{-INFINITY, 0.0f, 0.0f};
  for (int64_t c = tid; c < V; c += 256) {
    const float v = load_as_f32(z + c);
    const Part one{v, v != v || v == INFINITY ? NAN : v == -INFINITY ? 0.0f : 1.0f, 0.0f};
    p = join(p, one, c2);
  }
  parts[tid] = p;
  __syncthreads();
  for (int o = 128; o >= 1; o >>= 1) {
    if (tid < o) parts[tid] = join(parts[tid], parts[tid + o], c2);
    __syncthreads();
  }
  p = parts[0];
  const bool empty = masked_everywhere(p, k.scale);
  const float ls = log2f(p.s) * kLn2;
  if (tid == 0) {
    if (k.lse) k.lse[row] = empty ? -INFINITY : p.m * k.scale + ls;
    if (k.entropy) k.entropy[row] = empty ? 0.0f : ls - p.w / p.s * kLn2;
    if (k.logp) {
      const int32_t t = k.tokens[row];
      k.logp[row] = t == -1 ? 0.0f
                    : t < 0 || t >= V ? NAN
                    : empty ? -INFINITY
                            : (load_as_f32(z + t) - p.m) * k.scale - ls;
    }
  }
  uint64_t last = ~uint64_t(0);
  for (int r = 0; r < k.top; ++r) {
    uint64_t b = 0;
    for (int64_t c = tid; c < V; c += 256) {
      const uint64_t key = rank_key(load_as_f32(z + c), static_cast<uint32_t>(c));
      if (key < last && key > b) b = key;
    }
    best[tid] = b;
    __syncthreads();
    for (int o = 128; o >= 1; o >>= 1) {
      if (tid < o && best[tid + o] > best[tid]) best[tid] = best[tid + o];
      __syncthreads();
    }
    last = best[0];
    __syncthreads();
    if (tid == 0) {
      k.top_ids[row * k.top + r] = static_cast<int32_t>(key_class(last));
      k.top_logp[row * k.top + r] = empty ? -INFINITY : (key_logit(last) - p.m) * k.scale - ls;
    }
  }
}

template <typename T, typename TD>
__global__ __launch_bounds__(256) void dlvm_token_scores_grad_kernel(
    int64_t V, const T* logits, int64_t ld, float scale, const int32_t* __restrict__ tokens,
    const float* __restrict__ lse, const float* __restrict__ entropy, const float* __restrict__ dlogp,
    const float* __restrict__ dentropy, TD* dlogits, int64_t ld_out) {
  const int64_t row = blockIdx.x;
  const T* z = logits + row * ld;
  TD* d = dlogits + row * ld_out;
  const float l = lse[row];
  const float ge = dentropy ? dentropy[row] : 0.0f, H = dentropy ? entropy[row] : 0.0f;
  float gl = 0.0f;
  int64_t t = -1;
  if (dlogp) {
    t = tokens[row];
    gl = t == -1 ? 0.0f : t < 0 || t >= V ? NAN : dlogp[row];
  }
  for (int64_t c = threadIdx.x; c < V; c += 256) {
    float g = 0.0f;
    if (l != -INFINITY) {
      const float lp = load_as_f32(z + c) * scale - l;
      const float p = __expf(lp);
      g = gl * ((c == t ? 1.0f : 0.0f) - p);
      if (dentropy) g -= ge * (p == 0.0f ? 0.0f : p * (lp + H));
    }
    d[c] = store_cast<TD>(g * scale);
  }
}

}  // namespace

size_t token_scores_ws(int64_t, int64_t, int) { return 256; }

hipError_t launch_token_scores(const TokenScores& c, void*, hipStream_t s) {
  launch_kernel(c.dtype == F32 ? dlvm_token_scores_kernel<float> : dlvm_token_scores_kernel<bf16_t>,
                dim3(static_cast<uint32_t>(c.rows)), dim3(256), s, c);
  return hipGetLastError();
}

namespace {
template <typename T, typename TD>
hipError_t grad(int64_t rows, int64_t V, const void* logits, int64_t ld, float scale,
                const int32_t* tokens, const float* lse, const float* entropy, const float* dlogp,
                const float* dentropy, void* dlogits, int64_t ld_out, hipStream_t s) {
  launch_kernel(dlvm_token_scores_grad_kernel<T, TD>, dim3(static_cast<uint32_t>(rows)), dim3(256), s,
                V, static_cast<const T*>(logits), ld, scale, tokens, lse, entropy, dlogp, dentropy,
                static_cast<TD*>(dlogits), ld_out);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_token_scores_backward(int dtype, int out_dtype, int64_t rows, int64_t classes,
                                        const void* logits, int64_t ld, float scale,
                                        const int32_t* tokens, const float* lse,
                                        const float* entropy, const float* dlogp,
                                        const float* dentropy, void* dlogits, int64_t ld_out,
                                        hipStream_t s) {
  auto f = dtype == BF16 ? grad<bf16_t, bf16_t> : out_dtype == BF16 ? grad<float, bf16_t> : grad<float, float>;
  return f(rows, classes, logits, ld, scale, tokens, lse, entropy, dlogp, dentropy, dlogits, ld_out, s);
}

}  // namespace dlvm

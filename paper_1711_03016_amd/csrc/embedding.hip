// Token embeddings: the lookup with scaling, and the gradient of the table.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace dlvm {
namespace {

// One wavefront per token.
template <typename T>
__global__ __launch_bounds__(256) void dlvm_embedding_kernel(int64_t V, int64_t E, int64_t N,
                                                             const T* __restrict__ table,
                                                             const int32_t* __restrict__ ids,
                                                             float scale, T* __restrict__ out) {
  const int lane = threadIdx.x & 63;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (i >= N) return;
  const int32_t id = ids[i];
  const bool ok = id >= 0 && id < V;
  const T* row = table + (ok ? id : 0) * E;
  const float other = id == -1 ? 0.0f : NAN;
  for (int64_t c = lane; c < E; c += 64)
    out[i * E + c] = store_cast<T>(ok ? scale * load_as_f32(row + c) : other);
}

// One workgroup per row of the table: the tokens of the row in ascending order.
template <typename T>
__global__ __launch_bounds__(256) void dlvm_embedding_grad_kernel(
    int64_t E, int64_t N, const int32_t* __restrict__ ids, const T* __restrict__ dout, float scale,
    bool accumulate, float* __restrict__ dtable) {
  const int lane = threadIdx.x & 63;
  const int32_t v = blockIdx.x;
  for (int64_t c0 = 0; c0 < E; c0 += 256) {
    const int64_t c = c0 + threadIdx.x;
    float sum = 0.0f;
    bool any = false;
    for (int64_t i0 = 0; i0 < N; i0 += 64) {
      uint64_t m = __ballot(i0 + lane < N && ids[i0 + lane] == v);
      any = any || m != 0;
      for (; m != 0; m &= m - 1) {
        const int64_t i = i0 + __builtin_ctzll(m);
        if (c < E) sum += load_as_f32(dout + i * E + c);
      }
    }
    float* d = dtable + v * E + c;
    if (c < E && (any || !accumulate)) *d = (accumulate ? *d : 0.0f) + scale * sum;
  }
}

}  // namespace

hipError_t launch_embedding_forward(int dtype, int64_t vocab, int64_t width, int64_t tokens,
                                    const void* table, const int32_t* ids, float scale, void* out,
                                    hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>((tokens + 3) / 4));
  if (dtype == F32)
    launch_kernel(dlvm_embedding_kernel<float>, grid, dim3(256), s, vocab, width, tokens,
                  static_cast<const float*>(table), ids, scale, static_cast<float*>(out));
  else
    launch_kernel(dlvm_embedding_kernel<bf16_t>, grid, dim3(256), s, vocab, width, tokens,
                  static_cast<const bf16_t*>(table), ids, scale, static_cast<bf16_t*>(out));
  return hipGetLastError();
}

size_t embedding_backward_ws(int64_t, int64_t, int64_t) { return 256; }

hipError_t launch_embedding_backward(int dtype, int64_t vocab, int64_t width, int64_t tokens,
                                     const int32_t* ids, const void* dout, float scale,
                                     bool accumulate, float* dtable, void*, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(vocab));
  if (dtype == F32)
    launch_kernel(dlvm_embedding_grad_kernel<float>, grid, dim3(256), s, width, tokens, ids,
                  static_cast<const float*>(dout), scale, accumulate, dtable);
  else
    launch_kernel(dlvm_embedding_grad_kernel<bf16_t>, grid, dim3(256), s, width, tokens, ids,
                  static_cast<const bf16_t*>(dout), scale, accumulate, dtable);
  return hipGetLastError();
}

}  // namespace dlvm

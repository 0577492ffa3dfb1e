// The gated linear recurrence h_t = a_t h_{t-1} + u_t, a = sigmoid(z), u = x or
// (1 - a) x, and its gradient.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace dlvm {
namespace {

// a = sigmoid(z) and c = 1 - a, each to float32 accuracy on its own (1 - a from a
// rounded a loses its digits where the gate is open): with s = exp(-|z|) one is
// 1 / (1 + s) and the other s / (1 + s).
__device__ __forceinline__ void gate(float z, float& a, float& c) {
  const float s = __expf(-fabsf(z));
  const float r = 1.0f / (1.0f + s);
  a = z >= 0.0f ? r : s * r;
  c = z >= 0.0f ? s * r : r;
  if (z != z) a = c = z;
}

__device__ __forceinline__ int32_t length_of(const int32_t* lens, int64_t b, int64_t T) {
  if (lens == nullptr) return static_cast<int32_t>(T);
  const int32_t n = lens[b];
  return n < 0 ? 0 : n > T ? static_cast<int32_t>(T) : n;
}

// One thread per state.
template <typename E, bool COUPLED>
__global__ __launch_bounds__(256) void dlvm_gated_scan_kernel(GatedScan k) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (j >= k.B * k.H) return;
  const int64_t b = j / k.H, c = j - b * k.H;
  const int32_t n = length_of(k.lens, b, k.T);
  float h = k.h0 ? k.h0[j] : 0.0f;
  for (int64_t t = 0; t < k.T; ++t) {
    const int64_t r = t * k.B + b;
    float shown = 0.0f;
    if (t < n) {
      float a, q;
      gate(load_as_f32(static_cast<const E*>(k.z) + r * k.ldz + c), a, q);
      const float x = load_as_f32(static_cast<const E*>(k.x) + r * k.ldx + c);
      h = a * h + (COUPLED ? q * x : x);
      shown = h;
    }
    static_cast<E*>(k.hs)[r * k.ldh + c] = store_cast<E>(shown);
  }
  if (k.hT) k.hT[j] = h;
}

// mu is the adjoint of the state after step t, on the way back from the last step.
template <typename E, bool COUPLED>
__global__ __launch_bounds__(256) void dlvm_gated_scan_grad_kernel(GatedScan k) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (j >= k.B * k.H) return;
  const int64_t b = j / k.H, c = j - b * k.H;
  const int32_t n = length_of(k.lens, b, k.T);
  float mu = k.dhT ? k.dhT[j] : 0.0f;
  for (int64_t t = k.T - 1; t >= 0; --t) {
    const int64_t r = t * k.B + b;
    float gz = 0.0f, gx = 0.0f;
    if (t < n) {
      float a, q;
      gate(load_as_f32(static_cast<const E*>(k.z) + r * k.ldz + c), a, q);
      const float x = load_as_f32(static_cast<const E*>(k.x) + r * k.ldx + c);
      const float prev = t > 0 ? load_as_f32(static_cast<const E*>(k.hs) + (r - k.B) * k.ldh + c)
                               : k.h0 ? k.h0[j] : 0.0f;
      const float lam = mu + (k.dhs ? load_as_f32(static_cast<const E*>(k.dhs) + r * k.lddh + c) : 0.0f);
      gx = COUPLED ? q * lam : lam;
      gz = lam * (COUPLED ? prev - x : prev) * (a * q);
      mu = a * lam;
    }
    static_cast<E*>(k.dz)[r * k.lddz + c] = store_cast<E>(gz);
    static_cast<E*>(k.dx)[r * k.lddx + c] = store_cast<E>(gx);
  }
  if (k.dh0) k.dh0[j] = mu;
}

}  // namespace

size_t gated_scan_ws(int, int64_t, int64_t, int64_t) { return 256; }

hipError_t launch_gated_scan_forward(const GatedScan& c, void*, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>((c.B * c.H + 255) / 256));
  auto f = c.dtype == F32 ? (c.coupled ? dlvm_gated_scan_kernel<float, true> : dlvm_gated_scan_kernel<float, false>)
                          : (c.coupled ? dlvm_gated_scan_kernel<bf16_t, true> : dlvm_gated_scan_kernel<bf16_t, false>);
  launch_kernel(f, grid, dim3(256), s, c);
  return hipGetLastError();
}

hipError_t launch_gated_scan_backward(const GatedScan& c, void*, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>((c.B * c.H + 255) / 256));
  auto f = c.dtype == F32
               ? (c.coupled ? dlvm_gated_scan_grad_kernel<float, true> : dlvm_gated_scan_grad_kernel<float, false>)
               : (c.coupled ? dlvm_gated_scan_grad_kernel<bf16_t, true> : dlvm_gated_scan_grad_kernel<bf16_t, false>);
  launch_kernel(f, grid, dim3(256), s, c);
  return hipGetLastError();
}

}  // namespace dlvm

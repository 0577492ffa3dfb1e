// The gated linear recurrence h_t = a_t h_{t-1} + u_t, a = sigmoid(z), u = x or
// (1 - a) x, and its gradient.
//
// A step is the map h -> a h + u; maps compose, (A2, U2) after (A1, U1) being
// (A2 A1, A2 U1 + U2), so a stretch of time is summed up by one pair of numbers for each
// state. The adjoint is the same recurrence backwards: mu -> a (mu + dh). Both calls
// read their tensors once where there are states enough to fill the GPU:
//  - many states, or few steps: a thread takes its states through all steps;
//  - else a workgroup takes 64 V states, its eight waves eight steps each of every 64:
//    each sums its steps up in registers, the sums are exchanged through LDS, and each
//    goes through its steps again from the state before them;
//  - few states and many steps: time is cut into segments besides. A first launch sums
//    every segment up, and the second starts each from the sums before it. That reads the
//    inputs a second time, from the Infinity Cache as far as they fit: the second launch
//    begins with the segments that the first read last.
// What bounds them is memory; the arithmetic (two transcendental functions to an element)
// takes about half of what the vector units could do in that time.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace dlvm {
namespace {

constexpr int kUnroll = 8;  // steps of a thread that are in flight together
constexpr int kWaves = 8;   // waves of a workgroup that share the steps

// V neighbouring states of a row (rows start on V elements).
template <typename E, int V> struct alignas(sizeof(E) * V) Cols {
  E v[V];
};

// a = sigmoid(z) and c = 1 - a, each to float32 accuracy on its own (1 - a from a
// rounded a loses its digits where the gate is open). z of +-infinity gives 0 and 1, NaN
// stays NaN.
__device__ __forceinline__ void gate(float z, float& a, float& c) {
  const float e = __builtin_amdgcn_exp2f(z * -1.44269504088896340736f);
  a = __builtin_amdgcn_rcpf(1.0f + e);
  c = z < 0.0f ? 1.0f - a : e * a;
}

__device__ __forceinline__ int32_t length_of(const int32_t* lens, int32_t b, int64_t T) {
  if (lens == nullptr) return static_cast<int32_t>(T);
  const int32_t n = lens[b];
  return n < 0 ? 0 : n > T ? static_cast<int32_t>(T) : n;
}

// Segments of time of one call. sums[s * N + j] is what segment s does to state j.
struct Cut {
  int S;               // segments (1: none)
  int32_t len;         // steps of one
  int tiles;           // workgroups of a segment
  float* init;         // [N] copy of the first state (the caller's may be overwritten in place)
  float2* sums;
};

// Of a thread: its first state, batch entry and column.
struct Place {
  bool on;
  int32_t j, b, c;
};
template <int V> __device__ __forceinline__ Place place_of(int tile, int lane, const GatedScan& k) {
  Place p;
  const int64_t j = (static_cast<int64_t>(tile) * 64 + lane) * V;
  p.on = j < k.B * k.H;
  p.j = p.on ? static_cast<int32_t>(j) : 0;
  p.b = p.j / static_cast<int32_t>(k.H);
  p.c = p.j - p.b * static_cast<int32_t>(k.H);
  return p;
}

template <typename E, int V>
__device__ __forceinline__ Cols<E, V> load_cols(const E* p) {
  return *reinterpret_cast<const Cols<E, V>*>(p);
}

// ---------------------------------------------------------------------------
// Forward. NW is kWaves, or 1 for a thread that takes its states alone.
// ---------------------------------------------------------------------------
template <typename E, bool COUPLED, int V, int NW>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void dlvm_gated_scan_kernel(GatedScan k, Cut cut) {
  constexpr int U = kUnroll;
  __shared__ float2 sums[2][NW == 1 ? 1 : NW][NW == 1 ? 1 : 64 * V];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const int w = NW == 1 ? 0 : wave;
  const int s = cut.S - 1 - static_cast<int>(blockIdx.x) / cut.tiles;
  const int block = static_cast<int>(blockIdx.x) % cut.tiles;
  const Place p = place_of<V>(NW == 1 ? block * 4 + wave : block, lane, k);
  if (NW == 1 && !p.on) return;
  const int32_t begin = s * cut.len;
  const int32_t end = k.T - begin < cut.len ? static_cast<int32_t>(k.T) : begin + cut.len;
  const int32_t n = length_of(k.lens, p.b, k.T);
  const int32_t live = !p.on ? 0 : n < end ? n : end;  // steps below it are read
  const E* pz = static_cast<const E*>(k.z) + p.b * k.ldz + p.c;
  const E* px = static_cast<const E*>(k.x) + p.b * k.ldx + p.c;
  E* ph = static_cast<E*>(k.hs) + p.b * k.ldh + p.c;
  const int64_t sz = k.B * k.ldz, sx = k.B * k.ldx, sh = k.B * k.ldh;

  float h[V];
  const float* first = cut.S > 1 ? cut.init : k.h0;
#pragma unroll
  for (int v = 0; v < V; ++v) h[v] = first ? first[p.j + v] : 0.0f;
  Cols<E, V> z[U] = {}, x[U] = {};
  const auto fetch = [&](int32_t t0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (t0 + u < live) {
        z[u] = load_cols<E, V>(pz + (t0 + u) * sz);
        x[u] = load_cols<E, V>(px + (t0 + u) * sx);
      }
  };
  fetch(begin + w * U);
  // every wave has its first state before one of them can write hT over it
#pragma unroll
  for (int v = 0; v < V; ++v) asm volatile("" : "+v"(h[v]));
  for (int q = 0; q < s; ++q)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float2 m = cut.sums[q * (k.B * k.H) + p.j + v];
      h[v] = m.x * h[v] + m.y;
    }

  int phase = 0;
  for (int32_t t0 = begin; t0 < end; t0 += NW * U) {
    const int32_t t = t0 + w * U;
    float a[U][V], q[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float c;
        gate(load_as_f32(&z[u].v[v]), a[u][v], c);
        const float xv = load_as_f32(&x[u].v[v]);
        q[u][v] = COUPLED ? c * xv : xv;
        if (t + u >= live) {
          a[u][v] = 1.0f;
          q[u][v] = 0.0f;
        }
      }
    fetch(t + NW * U);
    float now[V];
#pragma unroll
    for (int v = 0; v < V; ++v) now[v] = h[v];
    if (NW > 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float A = a[0][v], Q = q[0][v];
#pragma unroll
        for (int u = 1; u < U; ++u) {
          Q = a[u][v] * Q + q[u][v];
          A *= a[u][v];
        }
        sums[phase][w][lane * V + v] = make_float2(A, Q);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (i == w) now[v] = h[v];
          const float2 m = sums[phase][i][lane * V + v];
          h[v] = m.x * h[v] + m.y;
        }
      phase ^= 1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Cols<E, V> o;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        now[v] = a[u][v] * now[v] + q[u][v];
        o.v[v] = store_cast<E>(t + u < n ? now[v] : 0.0f);
      }
      if (p.on && t + u < end) *reinterpret_cast<Cols<E, V>*>(ph + (t + u) * sh) = o;
    }
    if (NW == 1)
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = now[v];
  }
  if (k.hT != nullptr && p.on && s == cut.S - 1 && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) k.hT[p.j + v] = h[v];
}

// ---------------------------------------------------------------------------
// Gradient, from the last step backwards. The states before a thread's eight steps are
// recomputed from the one before the first of them, the only row of hs that it reads.
// ---------------------------------------------------------------------------
template <typename E, bool COUPLED, int V, int NW>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void dlvm_gated_scan_grad_kernel(GatedScan k, Cut cut) {
  constexpr int U = kUnroll;
  __shared__ float2 sums[2][NW == 1 ? 1 : NW][NW == 1 ? 1 : 64 * V];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const int w = NW == 1 ? 0 : wave;
  const int s = static_cast<int>(blockIdx.x) / cut.tiles;
  const int block = static_cast<int>(blockIdx.x) % cut.tiles;
  const Place p = place_of<V>(NW == 1 ? block * 4 + wave : block, lane, k);
  if (NW == 1 && !p.on) return;
  const int32_t begin = s * cut.len;
  const int32_t end = k.T - begin < cut.len ? static_cast<int32_t>(k.T) : begin + cut.len;
  const int32_t n = length_of(k.lens, p.b, k.T);
  const int32_t live = !p.on ? 0 : n < end ? n : end;
  const E* pz = static_cast<const E*>(k.z) + p.b * k.ldz + p.c;
  const E* px = static_cast<const E*>(k.x) + p.b * k.ldx + p.c;
  const E* ph = static_cast<const E*>(k.hs) + p.b * k.ldh + p.c;
  const E* pd = static_cast<const E*>(k.dhs) + p.b * k.lddh + p.c;
  E* gz = static_cast<E*>(k.dz) + p.b * k.lddz + p.c;
  E* gx = static_cast<E*>(k.dx) + p.b * k.lddx + p.c;
  const int64_t sz = k.B * k.ldz, sx = k.B * k.ldx, sh = k.B * k.ldh, sd = k.B * k.lddh;
  const int64_t tz = k.B * k.lddz, tx = k.B * k.lddx;
  const bool has_d = k.dhs != nullptr;

  float mu[V];
  const float* first = cut.S > 1 ? cut.init : k.dhT;
#pragma unroll
  for (int v = 0; v < V; ++v) mu[v] = first ? first[p.j + v] : 0.0f;
  Cols<E, V> z[U] = {}, x[U] = {}, d[U] = {}, before = {};
  const auto fetch = [&](int32_t t0) {
    if (t0 < begin) return;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (t0 + u < live) {
        z[u] = load_cols<E, V>(pz + (t0 + u) * sz);
        x[u] = load_cols<E, V>(px + (t0 + u) * sx);
        if (has_d) d[u] = load_cols<E, V>(pd + (t0 + u) * sd);
      }
    if (t0 > 0 && t0 < live) before = load_cols<E, V>(ph + (t0 - 1) * sh);
  };
  const int32_t last = begin + (end - begin - 1) / (NW * U) * (NW * U);
  fetch(last + w * U);
  // every wave has its adjoint before one of them can write dh0 over it
#pragma unroll
  for (int v = 0; v < V; ++v) asm volatile("" : "+v"(mu[v]));
  for (int q = cut.S - 1; q > s; --q)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float2 m = cut.sums[q * (k.B * k.H) + p.j + v];
      mu[v] = m.x * mu[v] + m.y;
    }

  int phase = 0;
  for (int32_t t0 = last; t0 >= begin; t0 -= NW * U) {
    const int32_t t = t0 + w * U;
    float a[U][V], c[U][V], xs[U][V], hp[U][V], dh[U][V];
#pragma unroll
    for (int v = 0; v < V; ++v)
      hp[0][v] = t > 0 ? load_as_f32(&before.v[v]) : k.h0 ? k.h0[p.j + v] : 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        gate(load_as_f32(&z[u].v[v]), a[u][v], c[u][v]);
        xs[u][v] = load_as_f32(&x[u].v[v]);
        dh[u][v] = has_d ? load_as_f32(&d[u].v[v]) : 0.0f;
        if (t + u >= live) {
          a[u][v] = 1.0f;
          dh[u][v] = 0.0f;
        }
        if (u + 1 < U) hp[u + 1][v] = a[u][v] * hp[u][v] + (COUPLED ? c[u][v] * xs[u][v] : xs[u][v]);
      }
    fetch(t - NW * U);
    float now[V];
#pragma unroll
    for (int v = 0; v < V; ++v) now[v] = mu[v];
    if (NW > 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float A = 1.0f, M = 0.0f;
#pragma unroll
        for (int u = U - 1; u >= 0; --u) {
          M = a[u][v] * (M + dh[u][v]);
          A *= a[u][v];
        }
        sums[phase][w][lane * V + v] = make_float2(A, M);
      }
      __syncthreads();
#pragma unroll
      for (int i = NW - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (i == w) now[v] = mu[v];
          const float2 m = sums[phase][i][lane * V + v];
          mu[v] = m.x * mu[v] + m.y;
        }
      phase ^= 1;
    }
#pragma unroll
    for (int u = U - 1; u >= 0; --u) {
      Cols<E, V> oz, ox;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float lam = now[v] + dh[u][v];
        const float prev = COUPLED ? hp[u][v] - xs[u][v] : hp[u][v];
        const bool in = t + u < live;
        oz.v[v] = store_cast<E>(in ? lam * prev * (a[u][v] * c[u][v]) : 0.0f);
        ox.v[v] = store_cast<E>(in ? (COUPLED ? c[u][v] * lam : lam) : 0.0f);
        now[v] = a[u][v] * lam;
      }
      if (p.on && t + u < end) {
        *reinterpret_cast<Cols<E, V>*>(gz + (t + u) * tz) = oz;
        *reinterpret_cast<Cols<E, V>*>(gx + (t + u) * tx) = ox;
      }
    }
    if (NW == 1)
#pragma unroll
      for (int v = 0; v < V; ++v) mu[v] = now[v];
  }
  if (k.dh0 != nullptr && p.on && s == 0 && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) k.dh0[p.j + v] = mu[v];
}

// ---------------------------------------------------------------------------
// What each segment does to its states (one column a lane): the waves take equal
// stretches of it, whose sums are composed in order. ADJOINT: of the gradient, backwards
// (the stretches are read forwards, the last wave's applied first).
// ---------------------------------------------------------------------------
template <typename E, bool COUPLED, bool ADJOINT>
__global__ __launch_bounds__(64 * kWaves) void dlvm_gated_scan_sums_kernel(GatedScan k, Cut cut) {
  constexpr int U = 2 * kUnroll;
  __shared__ float2 sums[kWaves][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  // the forward call needs no sum of the last segment, the gradient none of the first
  const int s = static_cast<int>(blockIdx.x) / cut.tiles + (ADJOINT ? 1 : 0);
  const Place p = place_of<1>(static_cast<int>(blockIdx.x) % cut.tiles, lane, k);
  const int32_t begin = s * cut.len;
  const int32_t end = k.T - begin < cut.len ? static_cast<int32_t>(k.T) : begin + cut.len;
  const int32_t n = length_of(k.lens, p.b, k.T);
  const int32_t live = !p.on ? 0 : n < end ? n : end;
  const E* pz = static_cast<const E*>(k.z) + p.b * k.ldz + p.c;
  const int64_t sz = k.B * k.ldz;
  const E* pu = ADJOINT ? static_cast<const E*>(k.dhs) + p.b * k.lddh + p.c
                        : static_cast<const E*>(k.x) + p.b * k.ldx + p.c;
  const int64_t su = ADJOINT ? k.B * k.lddh : k.B * k.ldx;
  const bool has_u = ADJOINT ? k.dhs != nullptr : true;
  if (p.on && wave == 0 && s == (ADJOINT ? cut.S - 1 : 0)) {
    const float* first = ADJOINT ? k.dhT : k.h0;
    cut.init[p.j] = first ? first[p.j] : 0.0f;
  }

  const int32_t stretch = (cut.len + kWaves * U - 1) / (kWaves * U) * U;
  const int32_t t_end = begin + (wave + 1) * stretch < end ? begin + (wave + 1) * stretch : end;
  float A = 1.0f, Q = 0.0f;
  for (int32_t t0 = begin + wave * stretch; t0 < t_end; t0 += U) {
    E z[U] = {}, v[U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (t0 + u < live && t0 + u < t_end) {
        z[u] = pz[(t0 + u) * sz];
        if (has_u) v[u] = pu[(t0 + u) * su];
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float a, c;
      gate(load_as_f32(&z[u]), a, c);
      float q = has_u ? load_as_f32(&v[u]) : 0.0f;
      const bool in = t0 + u < live && t0 + u < t_end;
      if (ADJOINT) {
        // mu -> A mu + Q before this earlier stretch of steps, step t after: A' = A a, and its
        // own dh reaches through a and all steps before it
        A = in ? A * a : A;
        Q = in ? Q + A * q : Q;
      } else {
        q = COUPLED ? c * q : q;
        Q = in ? a * Q + q : Q;
        A = in ? A * a : A;
      }
    }
  }
  sums[wave][lane] = make_float2(A, Q);
  __syncthreads();
  if (wave == 0 && p.on) {
    float2 m = make_float2(1.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float2 o = sums[ADJOINT ? kWaves - 1 - i : i][lane];
      m = make_float2(o.x * m.x, o.x * m.y + o.y);
    }
    cut.sums[s * (k.B * k.H) + p.j] = m;
  }
}

// ---------------------------------------------------------------------------
// Choice of the variant.
// ---------------------------------------------------------------------------
constexpr int64_t kBlocks = 512;       // workgroups that fill the GPU: two on a compute unit
constexpr int32_t kShortest = 128;     // steps of a segment at least

// Segments of a call of N states, and the steps of one.
int segments(int64_t T, int64_t N, int32_t* len) {
  const int64_t tiles = (N + 63) / 64;
  int64_t S = tiles >= kBlocks ? 1 : (kBlocks + tiles - 1) / tiles;
  if (S > T / kShortest) S = T / kShortest;
  if (S < 1) S = 1;
  const int64_t step = int64_t(kWaves) * kUnroll;
  int64_t L = S == 1 ? T : ((T + S - 1) / S + step - 1) / step * step;
  *len = static_cast<int32_t>(L);
  return static_cast<int>((T + L - 1) / L);
}

struct Variant {
  int V;
  bool alone;  // a thread takes its states through all steps
};
// Widest vectors that rows and columns allow, as long as the states fill the GPU: with
// two waves on every SIMD when a thread goes alone, with two workgroups to a compute unit
// when waves share the steps. Few steps leave nothing to share.
Variant variant(const GatedScan& c, bool cut, int widest) {
  const int64_t N = c.B * c.H;
  int V = widest;
  const int64_t lds[] = {c.H, c.ldz, c.ldx, c.ldh, c.dhs ? c.lddh : 0, c.dz ? c.lddz : 0, c.dx ? c.lddx : 0};
  for (const int64_t ld : lds)
    while (ld % V != 0) V /= 2;
  const auto waves = [&](int v) { return (N + 64 * v - 1) / (64 * v); };
  if (cut) return Variant{1, false};
  if (c.T <= 2 * kUnroll || waves(1) >= 8192) {
    while (V > 1 && waves(V) < 2048) V /= 2;
    return Variant{V, true};
  }
  while (V > 1 && waves(V) < kBlocks) V /= 2;
  return Variant{V, false};
}

template <typename E, bool COUPLED, bool GRAD>
hipError_t run(const GatedScan& c, void* ws, hipStream_t s) {
  const int64_t N = c.B * c.H;
  Cut cut{};
  cut.S = 1;
  cut.len = static_cast<int32_t>(c.T);
  if (ws != nullptr) cut.S = segments(c.T, N, &cut.len);
  const Variant v = variant(c, cut.S > 1, GRAD ? 2 : 4);
  const int64_t waves = (N + 64 * v.V - 1) / (64 * v.V);
  cut.tiles = static_cast<int>(v.alone ? (waves + 3) / 4 : waves);
  if (cut.S > 1) {
    cut.init = static_cast<float*>(ws);
    cut.sums = reinterpret_cast<float2*>(cut.init + (N + 63) / 64 * 64);
    launch_kernel(dlvm_gated_scan_sums_kernel<E, COUPLED, GRAD>, dim3(cut.tiles * (cut.S - 1)),
                  dim3(64 * kWaves), s, c, cut);
  }
  const dim3 grid(static_cast<uint32_t>(cut.tiles) * cut.S), block(v.alone ? 256 : 64 * kWaves);
  if constexpr (GRAD) {
    auto f = v.V == 2 ? (v.alone ? dlvm_gated_scan_grad_kernel<E, COUPLED, 2, 1>
                                 : dlvm_gated_scan_grad_kernel<E, COUPLED, 2, kWaves>)
                      : (v.alone ? dlvm_gated_scan_grad_kernel<E, COUPLED, 1, 1>
                                 : dlvm_gated_scan_grad_kernel<E, COUPLED, 1, kWaves>);
    launch_kernel(f, grid, block, s, c, cut);
  } else {
    auto f = v.V == 4   ? (v.alone ? dlvm_gated_scan_kernel<E, COUPLED, 4, 1>
                                   : dlvm_gated_scan_kernel<E, COUPLED, 4, kWaves>)
             : v.V == 2 ? (v.alone ? dlvm_gated_scan_kernel<E, COUPLED, 2, 1>
                                   : dlvm_gated_scan_kernel<E, COUPLED, 2, kWaves>)
                        : (v.alone ? dlvm_gated_scan_kernel<E, COUPLED, 1, 1>
                                   : dlvm_gated_scan_kernel<E, COUPLED, 1, kWaves>);
    launch_kernel(f, grid, block, s, c, cut);
  }
  return hipGetLastError();
}

template <bool GRAD> hipError_t run_any(const GatedScan& c, void* ws, hipStream_t s) {
  return c.dtype == F32 ? (c.coupled ? run<float, true, GRAD>(c, ws, s) : run<float, false, GRAD>(c, ws, s))
                        : (c.coupled ? run<bf16_t, true, GRAD>(c, ws, s) : run<bf16_t, false, GRAD>(c, ws, s));
}

}  // namespace

size_t gated_scan_ws(int, int64_t T, int64_t B, int64_t H) {
  int32_t len = 0;
  const int64_t N = B * H, S = segments(T, N, &len);
  return S == 1 ? 256 : static_cast<size_t>((N + 63) / 64 * 64) * 4 + static_cast<size_t>(S) * N * 8;
}

hipError_t launch_gated_scan_forward(const GatedScan& c, void* ws, hipStream_t s) {
  return run_any<false>(c, ws, s);
}

hipError_t launch_gated_scan_backward(const GatedScan& c, void* ws, hipStream_t s) {
  return run_any<true>(c, ws, s);
}

}  // namespace dlvm

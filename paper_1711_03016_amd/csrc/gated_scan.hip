// The gated linear recurrence h_t = a_t h_{t-1} + u_t, a = sigmoid(z), u = x or
// (1 - a) x, and its gradient.
//
// A step is the map h -> a h + u; maps compose, (A2, U2) after (A1, U1) being
// (A2 A1, A2 U1 + U2), so a stretch of time is summed up by one pair of numbers for each
// state. The adjoint is the same recurrence backwards: mu -> a (mu + dh). One state to a
// lane: wider vectors leave fewer waves (63 against 45 us with four states of bf16 to a lane,
// T = 32, 2^20 states).
//  - ALONE, many states or few steps: a thread takes its state through all steps;
//  - SHARED: a workgroup takes 64 states, its eight waves eight steps each of every 64:
//    each wave sums its steps up in registers, the sums are exchanged through LDS, and each
//    goes through its steps again from the state before them;
//  - CHAINED, the forward call of few states and many steps: each block of time has a
//    workgroup of its own, which publishes the map of its block, takes the state before it
//    from what the workgroups of earlier blocks have published, and publishes the state
//    after it. Every tensor is read once.
//  - SHARED in segments of time, the gradient of few states and many steps: a first launch
//    sums every segment up, and the second starts each from the sums after it (and before it,
//    where it recomputes the states). That reads z, dhs and, for the states, x again, from the
//    Infinity Cache as far as they fit. (Chained, the gradient's blocks are too short for the
//    waiting: its registers hold twelve steps of a wave, where the forward call's 32 steps
//    take 56 us chained and 74 in segments, T = 4096, 8192 states of bf16.)
// What bounds them is memory; the arithmetic (two transcendental functions to an element)
// takes about half of what the vector units could do in that time.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace dlvm {
namespace {

enum Mode { ALONE, SHARED, CHAINED };
constexpr int kWaves = 8;          // waves of a workgroup that share the steps
constexpr int kUnroll = 8;         // steps of a thread that are in flight together
constexpr int kChainedUnroll = 32; // and in a block of a chain

// a = sigmoid(z) and c = 1 - a, each with its own relative error (1 - a from a rounded a
// loses its digits where the gate is open): below (|z| + 16) 2^-23, since the argument of the
// exponential is rounded. z of +-infinity gives 0 and 1, NaN stays NaN.
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

// Segments of time of a gradient call. sums[s * N + j] is the map (A, M) of segment s for the
// adjoint of state j, and A with states[s * N + j] that for the state.
struct Cut {
  int S;               // segments (1: none)
  int32_t len;         // steps of one
  int tiles;           // workgroups of a segment
  float* init;         // [N] copy of the last adjoint (the caller's may be overwritten in place)
  float2* sums;
  float* states;       // where the states are recomputed
};

// ---------------------------------------------------------------------------
// The chain of a CHAINED call. words[(i * tiles + tile) * 64 + lane] is, of block i of time
// and the lane's state, first kEmpty, then the block's map (A, Q), then (kState, the state
// after it): 64 bits that are written and read whole, so that a word needs no flag beside it
// and no order with other memory. (A is a product of gates, never negative; a NaN is stored
// as the one that is not kEmpty.) This is the decoupled look-back of the single-pass prefix
// sums of D. Merrill and M. Garland (2016), for maps in place of sums.
//
// A workgroup takes the next block of its tile by a ticket, so every earlier block is
// taken by a workgroup that runs already, and that publishes its map without waiting for
// anything. The first block that has no state yet finds the states before it, so it goes
// on: every wait ends. Should a workspace be used by two calls at once after all, a bound on
// the rounds of waiting ends it with NaN. The state before a block comes from the nearest
// earlier block whose state is known, by the maps between, applied one after the other in
// time: the same roundings wherever the known state was found.
// ---------------------------------------------------------------------------
constexpr int kWindow = 64;            // earlier blocks that a workgroup looks at
constexpr int kRounds = 1 << 17;       // about a tenth of a second
constexpr uint32_t kEmpty = 0xffffffffu;
constexpr float kState = -1.0f;
constexpr int kTicketStride = 32;      // a ticket to every 128 bytes

struct Chain {
  int blocks, tiles;                   // blocks of time; workgroups of one block
  uint32_t* tickets;
  uint64_t* words;
};

__global__ __launch_bounds__(256) void dlvm_gated_scan_clear_kernel(Chain chain, int64_t n) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i < chain.tiles) chain.tickets[i * kTicketStride] = 0;
  if (i < n) chain.words[i] = ~uint64_t(0);
}

typedef __attribute__((address_space(1))) uint64_t Word;

// The words of a tile in block b, one to a lane: a scalar address.
__device__ __forceinline__ Word* words_of(const Chain& chain, int tile, int b) {
  Word* w = (Word*)chain.words + (static_cast<int64_t>(b) * chain.tiles + tile) * 64;
  asm("" : "+s"(w));
  return w;
}

__device__ __forceinline__ void publish(const Chain& chain, int tile, int b, int lane, float x, float y) {
  const uint32_t hi = x != x ? 0x7fc00000u : __float_as_uint(x);
  __hip_atomic_store(words_of(chain, tile, b) + lane, static_cast<uint64_t>(hi) << 32 | __float_as_uint(y),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The state before block i (> 0) of the lane's state. All waves of the workgroup call it.
__device__ __forceinline__ float state_before(const Chain& chain, int tile, int i, int wave, int lane,
                                              uint64_t (*window)[64]) {
  constexpr int each = kWindow / kWaves;
  const auto ready = [](uint64_t m) { return static_cast<uint32_t>(m >> 32) != kEmpty; };
  const auto state = [](uint64_t m) { return static_cast<uint32_t>(m >> 32) == __float_as_uint(kState); };
  const auto load = [&](int b) {
    return b >= 0 ? __hip_atomic_load(words_of(chain, tile, b) + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                  : static_cast<uint64_t>(__float_as_uint(kState)) << 32;
  };
  int look = kWaves;  // the nearest blocks first: a block's words are as many bytes as a step's inputs
#pragma unroll 1
  for (int round = 0; round < kRounds; ++round) {
    if (look == kWaves) {
      window[wave][lane] = load(i - 1 - wave);
    } else {
      uint64_t m[each];
#pragma unroll
      for (int e = 0; e < each; ++e) m[e] = load(i - 1 - (wave * each + e));
#pragma unroll
      for (int e = 0; e < each; ++e) window[wave * each + e][lane] = m[e];
    }
    __syncthreads();
    // how far back every lane finds a state, with no gap before it
    int far = 0;
    bool found = false, gap = false;
#pragma unroll 1
    while (far < look) {
#pragma unroll 4
      for (int e = 0; e < each; ++e) {
        const uint64_t v = window[far + e][lane];
        gap = gap || (!found && !ready(v));
        found = found || state(v);
      }
      far += each;
      if (__ballot(gap) != 0 || __ballot(found) == ~uint64_t(0)) break;
    }
    const bool whole = __ballot(gap) == 0;
    const bool done = whole && __ballot(found) == ~uint64_t(0);
    float h = 0.0f;
    if (done) {
#pragma unroll 4
      for (int k = far - 1; k >= 0; --k) {
        const uint64_t v = window[k][lane];
        const float A = __uint_as_float(static_cast<uint32_t>(v >> 32));
        const float Q = __uint_as_float(static_cast<uint32_t>(v));
        h = state(v) ? Q : fmaf(A, h, Q);
      }
    }
    __syncthreads();
    if (done) return h;
    if (whole) look = kWindow;
    else __builtin_amdgcn_s_sleep(1);
  }
  return NAN;
}

// Of a thread: whether it has a state, which, and the state's batch entry and column;
// b0 and c0 are those of the wave's first lane. (A lane without a state has the first's.)
struct Place {
  bool on;
  int32_t j, b, c, b0, c0;
};
__device__ __forceinline__ Place place_of(int tile, int lane, const GatedScan& k) {
  Place p;
  const int32_t H = static_cast<int32_t>(k.H);
  const int32_t first = tile * 64;
  p.on = static_cast<int64_t>(first) + lane < k.B * k.H;
  p.j = p.on ? first + lane : first;
  p.b0 = first / H;
  p.c0 = first - p.b0 * H;
  p.b = p.j / H;
  p.c = p.j - p.b * H;
  return p;
}

// The rows of one tensor as a wave sees them: a scalar address for each step, and the
// lane's distance from the first lane's element, which fits 32 bits (checked by the
// caller), so that the addresses of many loads in flight take no vector registers.
template <typename E> struct Rows {
  typedef __attribute__((address_space(1))) char Byte;
  typedef __attribute__((address_space(1))) E Elem;
  Byte* base;
  int64_t step;
  uint32_t at;
  __device__ __forceinline__ Rows(const void* t, int64_t ld, int64_t B, const Place& p)
      : base((Byte*)(static_cast<E*>(const_cast<void*>(t)) + (p.b0 * ld + p.c0))),
        step(B * ld * static_cast<int64_t>(sizeof(E))),
        at(static_cast<uint32_t>((p.b - p.b0) * ld + p.c - p.c0) * static_cast<uint32_t>(sizeof(E))) {}
  __device__ __forceinline__ Byte* row(int32_t t) const { return base + t * step; }
  __device__ __forceinline__ Elem& in(Byte* row) const {
    asm("" : "+s"(row));  // keeps the scalar part of the address apart from the lane's
    return *(Elem*)(row + at);
  }
};

// The largest of the wave's values.
__device__ __forceinline__ int32_t wave_max(int32_t v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const int32_t w = __shfl_xor(v, o, 64);
    v = w > v ? w : v;
  }
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int32_t wave_min(int32_t v) { return -wave_max(-v); }

// The tile of a workgroup, of n: workgroups go to the eight XCDs in turn, and neighbouring
// tiles to one of them, since the rows of an odd width begin and end inside cache lines,
// which only a common L2 reads and writes once (777 steps of 13 x 1001 float32: forward 30
// against 34 us, gradient 47 against 53; even widths as before or up to 3% faster).
__device__ __forceinline__ int neighbours(int n) {
  const int b = static_cast<int>(blockIdx.x) % n, per = n / 8;
  return b < per * 8 ? b % 8 * per + b / 8 : b;
}

// The block of time and the tile of states of a workgroup (and, ALONE, of a wave).
template <int MODE>
__device__ __forceinline__ void work_of(const Chain& chain, int wave, int& block, int& tile) {
  if (MODE == CHAINED) {
    __shared__ uint32_t taken;
    tile = static_cast<int>(blockIdx.x % static_cast<uint32_t>(chain.tiles));
    if (threadIdx.x == 0)
      taken = __hip_atomic_fetch_add(chain.tickets + tile * kTicketStride, 1u, __ATOMIC_RELAXED,
                                     __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const uint32_t next = __builtin_amdgcn_readfirstlane(taken);
    block = next < static_cast<uint32_t>(chain.blocks) ? static_cast<int>(next) : chain.blocks;
  } else {
    block = 0;
    tile = neighbours(chain.tiles) * (MODE == ALONE ? 4 : 1) + (MODE == ALONE ? wave : 0);
  }
}

// ---------------------------------------------------------------------------
// Forward.
// ---------------------------------------------------------------------------
template <typename E, bool COUPLED, int MODE>
__global__ __launch_bounds__(MODE == ALONE ? 256 : 64 * kWaves) void dlvm_gated_scan_kernel(GatedScan k, Chain chain) {
  constexpr int U = MODE == CHAINED ? kChainedUnroll : kUnroll, NW = MODE == ALONE ? 1 : kWaves;
  __shared__ float2 sums[MODE == SHARED ? 2 : 1][MODE == ALONE ? 1 : NW][MODE == ALONE ? 1 : 64];
  __shared__ uint64_t window[MODE == CHAINED ? kWindow : 1][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const int w = MODE == ALONE ? 0 : wave;
  int block, tile;
  work_of<MODE>(chain, wave, block, tile);
  if (MODE == CHAINED && block >= chain.blocks) return;
  const Place p = place_of(tile, lane, k);
  if (MODE == ALONE && __ballot(p.on) == 0) return;  // whole waves: the others compare their lengths
  const int32_t begin = block * (NW * U);
  const int32_t T = static_cast<int32_t>(k.T);
  const int32_t end = MODE != CHAINED || T - begin < NW * U ? T : begin + NW * U;
  const int32_t n = length_of(k.lens, p.b, k.T);
  const int32_t live = !p.on ? 0 : n < end ? n : end;  // steps below it are read
  const Rows<E> pz(k.z, k.ldz, k.B, p), px(k.x, k.ldx, k.B, p), ph(k.hs, k.ldh, k.B, p);

  float h = k.h0 != nullptr && block == 0 ? k.h0[p.j] : 0.0f;
  E z[U] = {}, x[U] = {};
  // Steps below `sure` are live in every lane, those from `over` on in none (the waves of a
  // workgroup have the same states, so the same bounds).
  const int32_t sure = k.lens == nullptr ? end : wave_min(p.on ? live : end);
  const int32_t over = MODE == CHAINED || k.lens == nullptr ? end : wave_max(live);
  // Loads without conditions, steps behind the last that is live in any lane from that
  // one: in a branch of its own each load would be waited for before the next is sent.
  const int32_t stop = (k.lens == nullptr ? end : wave_max(live > begin ? live : begin + 1)) - 1;
  const auto fetch = [&](int32_t t0) {
    if (t0 >= over) return;
    const int32_t from = t0 < stop ? t0 : stop;
    auto rz = pz.row(from), rx = px.row(from);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      z[u] = pz.in(rz);
      x[u] = px.in(rx);
      const bool more = t0 + u < stop;
      rz += more ? pz.step : 0;
      rx += more ? px.step : 0;
    }
  };
  fetch(begin + w * U);
  asm volatile("" : "+v"(h));  // every wave has its first state before one can write hT over it

  int phase = 0;
  int32_t t0 = begin;
  for (; t0 < over; t0 += NW * U) {
    const int32_t t = t0 + w * U;
    float a[U], q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float c;
      gate(load_as_f32(&z[u]), a[u], c);
      const float xv = load_as_f32(&x[u]);
      q[u] = COUPLED ? c * xv : xv;
    }
    const bool whole = t + U <= sure;
    if (!whole)
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (t + u >= live) {
          a[u] = 1.0f;
          q[u] = 0.0f;
        }
    if (MODE != CHAINED) fetch(t + NW * U);
    float now = h;
    if (MODE != ALONE) {
      float A = a[0], Q = q[0];
#pragma unroll
      for (int u = 1; u < U; ++u) {
        Q = a[u] * Q + q[u];
        A *= a[u];
      }
      sums[phase][w][lane] = make_float2(A, Q);
      __syncthreads();
      float Aw = 1.0f, Qw = 0.0f;  // the maps of the waves before this one, and of all
      A = 1.0f;
      Q = 0.0f;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        if (i == w) {
          Aw = A;
          Qw = Q;
        }
        const float2 m = sums[phase][i][lane];
        Q = fmaf(m.x, Q, m.y);
        A *= m.x;
      }
      if (MODE == CHAINED && block > 0) {
        if (w == 0) publish(chain, tile, block, lane, A, Q);
        h = state_before(chain, tile, block, wave, lane, window);
      }
      now = fmaf(Aw, h, Qw);
      h = fmaf(A, h, Q);  // as state_before finds it from the map
      if (MODE == CHAINED && w == 0) publish(chain, tile, block, lane, kState, h);
      if (MODE == SHARED) phase ^= 1;
    }
    auto rh = ph.row(t);
    if (whole && p.on) {
#pragma unroll
      for (int u = 0; u < U; ++u, rh += ph.step) {
        now = a[u] * now + q[u];
        ph.in(rh) = store_cast<E>(now);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u, rh += ph.step) {
        now = a[u] * now + q[u];
        if (p.on && t + u < end) ph.in(rh) = store_cast<E>(t + u < n ? now : 0.0f);
      }
    }
    if (MODE == ALONE) h = now;
    if (MODE == CHAINED) break;  // a block is one round
  }
  if (MODE != CHAINED && p.on)
    for (int32_t t = t0 + w; t < end; t += NW) ph.in(ph.row(t)) = store_cast<E>(0.0f);
  if (k.hT != nullptr && p.on && w == 0 && end == T) k.hT[p.j] = h;
}

// ---------------------------------------------------------------------------
// Gradient, from the last step backwards. The states before a thread's eight steps are
// recomputed from the one before the first of them. In float32 that is a row of hs. The rows of
// bf16 are rounded, and where the state follows the input, h - x is smaller than what they are
// off by: there a pass forwards through z and x finds those states in float32 first, and keeps
// each in the two bf16 of dz and dx at its first step until the same thread comes back to it
// and writes the gradients. (The gradient of 32 steps of 2^20 states takes 84 us with that pass
// and 70 with the rows of hs, 4096 steps of 8192 states 139 and 102.)
// ---------------------------------------------------------------------------
template <typename E> constexpr bool kRecompute = sizeof(E) == 2;

template <typename E, bool COUPLED, int MODE>
__global__ __launch_bounds__(MODE == ALONE ? 256 : 64 * kWaves) void dlvm_gated_scan_grad_kernel(GatedScan k, Cut cut) {
  constexpr int U = kUnroll, NW = MODE == ALONE ? 1 : kWaves;
  __shared__ float2 sums[2][NW][MODE == ALONE ? 1 : 64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const int w = MODE == ALONE ? 0 : wave;
  const int block = neighbours(cut.tiles);
  const int s = static_cast<int>(blockIdx.x) / cut.tiles;
  const Place p = place_of(MODE == ALONE ? block * 4 + wave : block, lane, k);
  if (MODE == ALONE && __ballot(p.on) == 0) return;  // whole waves: the others compare their lengths
  const int64_t N = k.B * k.H;
  const int32_t T = static_cast<int32_t>(k.T);
  const int32_t begin = s * cut.len;
  const int32_t end = T - begin < cut.len ? T : begin + cut.len;
  const int32_t n = length_of(k.lens, p.b, k.T);
  const int32_t live = !p.on ? 0 : n < end ? n : end;
  const bool has_d = k.dhs != nullptr;
  const Rows<E> pz(k.z, k.ldz, k.B, p), px(k.x, k.ldx, k.B, p), ph(k.hs, k.ldh, k.B, p);
  const Rows<E> pd(has_d ? k.dhs : k.z, has_d ? k.lddh : k.ldz, k.B, p);
  const Rows<E> gz(k.dz, k.lddz, k.B, p), gx(k.dx, k.lddx, k.B, p);

  const float* first = cut.S > 1 ? cut.init : k.dhT;
  float mu = first != nullptr ? first[p.j] : 0.0f;
  E z[U] = {}, x[U] = {}, d[U] = {};
  float before = 0.0f;
  // as in the forward call
  const int32_t sure = k.lens == nullptr ? end : wave_min(p.on ? live : end);
  const int32_t over = k.lens == nullptr ? end : wave_max(live);
  const int32_t rounds = over > begin ? (over - begin + NW * U - 1) / (NW * U) : 0;
  const int32_t last = begin + (rounds - 1) * (NW * U);  // first step of the last round
  const int32_t stop = (k.lens == nullptr ? end : wave_max(live > begin ? live : begin + 1)) - 1;
  int phase = 0;
  float start = k.h0 != nullptr ? k.h0[p.j] : 0.0f;  // the first state; recomputed, the segment's
  if constexpr (kRecompute<E>) {
    for (int q = 0; q < s; ++q) start = fmaf(cut.sums[q * N + p.j].x, start, cut.states[q * N + p.j]);
    const auto forwards = [&](int32_t t0) {
      const int32_t from = t0 < stop ? t0 : stop;
      auto rz = pz.row(from), rx = px.row(from);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        z[u] = pz.in(rz);
        x[u] = px.in(rx);
        const bool more = t0 + u < stop;
        rz += more ? pz.step : 0;
        rx += more ? px.step : 0;
      }
    };
    const auto park = [&](int32_t t, float h) {
      const uint32_t bits = __float_as_uint(h);
      gz.in(gz.row(t)) = static_cast<E>(bits >> 16);
      gx.in(gx.row(t)) = static_cast<E>(bits);
    };
    // a thread that goes through all steps has no need of the last of its rounds
    const int32_t finish = MODE == ALONE ? last : last + NW * U;
    float h = start;
    if (finish > begin) forwards(begin + w * U);
    for (int32_t t0 = begin; t0 < finish; t0 += NW * U) {
      const int32_t t = t0 + w * U;
      float a[U], q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float c;
        gate(load_as_f32(&z[u]), a[u], c);
        const float xv = load_as_f32(&x[u]);
        q[u] = COUPLED ? c * xv : xv;
      }
      if (t + U > sure)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (t + u >= live) {
            a[u] = 1.0f;
            q[u] = 0.0f;
          }
      if (t0 + NW * U < finish) forwards(t + NW * U);
      if (MODE == ALONE) {
#pragma unroll
        for (int u = 0; u < U; ++u) h = a[u] * h + q[u];
        if (p.on) park(t + U, h);
      } else {
        float A = a[0], Q = q[0];
#pragma unroll
        for (int u = 1; u < U; ++u) {
          Q = a[u] * Q + q[u];
          A *= a[u];
        }
        sums[phase][w][lane] = make_float2(A, Q);
        __syncthreads();
        float now = h;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
          if (i == w) now = h;
          const float2 m = sums[phase][i][lane];
          h = fmaf(m.x, h, m.y);
        }
        phase ^= 1;
        if (p.on && t < end) park(t, now);
      }
    }
  }
  const auto fetch = [&](int32_t t0) {
    if (t0 < begin) return;
    const int32_t from = t0 < stop ? t0 : stop;
    auto rz = pz.row(from), rx = px.row(from), rd = pd.row(from);
    if constexpr (kRecompute<E>)  // of steps behind the last live one: any row, not used
      before = __uint_as_float(static_cast<uint32_t>(gz.in(gz.row(from))) << 16 |
                               static_cast<uint32_t>(gx.in(gx.row(from))));
    else
      before = ph.in(ph.row(from > 0 ? from - 1 : 0));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      z[u] = pz.in(rz);
      x[u] = px.in(rx);
      d[u] = pd.in(rd);
      const bool more = t0 + u < stop;
      rz += more ? pz.step : 0;
      rx += more ? px.step : 0;
      rd += more ? pd.step : 0;
    }
  };
  fetch(last + w * U);
  asm volatile("" : "+v"(mu));  // every wave has its adjoint before one can write dh0 over it
  for (int q = cut.S - 1; q > s; --q) {
    const float2 m = cut.sums[q * N + p.j];
    mu = fmaf(m.x, mu, m.y);
  }

  if (p.on)
    for (int32_t t = last + NW * U + w; t < end; t += NW) {
      gz.in(gz.row(t)) = store_cast<E>(0.0f);
      gx.in(gx.row(t)) = store_cast<E>(0.0f);
    }
  for (int32_t t0 = last; t0 >= begin; t0 -= NW * U) {
    const int32_t t = t0 + w * U;
    float a[U], c[U], f[U], dh[U];  // f: dz over the adjoint that passes the gate
    float prev = t > 0 ? before : start;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      gate(load_as_f32(&z[u]), a[u], c[u]);
      const float xv = load_as_f32(&x[u]);
      dh[u] = load_as_f32(&d[u]);
      f[u] = (COUPLED ? prev - xv : prev) * c[u];
      prev = a[u] * prev + (COUPLED ? c[u] * xv : xv);
    }
    const bool whole = has_d && t + U <= sure;
    if (!whole)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (t + u >= live) a[u] = 1.0f;
        if (t + u >= live || !has_d) dh[u] = 0.0f;
      }
    fetch(t - NW * U);
    float now = mu;
    if (MODE == SHARED) {
      float A = 1.0f, M = 0.0f;
#pragma unroll
      for (int u = U - 1; u >= 0; --u) {
        M = a[u] * (M + dh[u]);
        A *= a[u];
      }
      sums[phase][w][lane] = make_float2(A, M);
      __syncthreads();
      float Aw = 1.0f, Mw = 0.0f;  // the maps of the waves after this one, and of all
      A = 1.0f;
      M = 0.0f;
#pragma unroll
      for (int i = NW - 1; i >= 0; --i) {
        if (i == w) {
          Aw = A;
          Mw = M;
        }
        const float2 m = sums[phase][i][lane];
        M = fmaf(m.x, M, m.y);
        A *= m.x;
      }
      now = fmaf(Aw, mu, Mw);
      mu = fmaf(A, mu, M);
      phase ^= 1;
    }
    auto rz = gz.row(t + U - 1), rx = gx.row(t + U - 1);
    if (whole && p.on) {
#pragma unroll
      for (int u = U - 1; u >= 0; --u, rz -= gz.step, rx -= gx.step) {
        const float lam = now + dh[u];
        now = a[u] * lam;
        gz.in(rz) = store_cast<E>(f[u] * now);
        gx.in(rx) = store_cast<E>(COUPLED ? c[u] * lam : lam);
      }
    } else {
#pragma unroll
      for (int u = U - 1; u >= 0; --u, rz -= gz.step, rx -= gx.step) {
        const float lam = now + dh[u];
        now = a[u] * lam;
        const bool in = t + u < live;
        if (p.on && t + u < end) {
          gz.in(rz) = store_cast<E>(in ? f[u] * now : 0.0f);
          gx.in(rx) = store_cast<E>(in ? (COUPLED ? c[u] * lam : lam) : 0.0f);
        }
      }
    }
    if (MODE == ALONE) mu = now;
  }
  if (k.dh0 != nullptr && p.on && w == 0 && begin == 0) k.dh0[p.j] = mu;
}

// ---------------------------------------------------------------------------
// The maps of each segment of the gradient: of the adjoint after it to that before it (but the
// first) and, where the states are recomputed, of the state before it to that after it (but the
// last). The waves take equal stretches, read forwards, whose maps are composed.
// ---------------------------------------------------------------------------
template <typename E, bool COUPLED>
__global__ __launch_bounds__(64 * kWaves) void dlvm_gated_scan_sums_kernel(GatedScan k, Cut cut) {
  constexpr int U = 2 * kUnroll;
  constexpr bool kStates = kRecompute<E>;
  __shared__ float2 sums[kWaves][64];
  __shared__ float states[kStates ? kWaves : 1][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const int s = static_cast<int>(blockIdx.x) / cut.tiles + (kStates ? 0 : 1);
  const Place p = place_of(static_cast<int>(blockIdx.x) % cut.tiles, lane, k);
  const int32_t T = static_cast<int32_t>(k.T);
  const int32_t begin = s * cut.len;
  const int32_t end = T - begin < cut.len ? T : begin + cut.len;
  const int32_t n = length_of(k.lens, p.b, k.T);
  // what a segment has no need of is read from z, whose rows are read anyway
  const bool has_d = k.dhs != nullptr && s > 0, has_x = kStates && s < cut.S - 1;
  const Rows<E> pz(k.z, k.ldz, k.B, p), px(has_x ? k.x : k.z, has_x ? k.ldx : k.ldz, k.B, p);
  const Rows<E> pd(has_d ? k.dhs : k.z, has_d ? k.lddh : k.ldz, k.B, p);
  if (p.on && wave == 0 && s == cut.S - 1) cut.init[p.j] = k.dhT != nullptr ? k.dhT[p.j] : 0.0f;

  const int32_t stretch = (cut.len + kWaves * U - 1) / (kWaves * U) * U;
  const int32_t t_begin = begin + wave * stretch;
  const int32_t t_end = t_begin + stretch < end ? t_begin + stretch : end;
  const int32_t live = !p.on ? 0 : n < t_end ? n : t_end;
  const int32_t t_live = k.lens == nullptr ? t_end : wave_max(live);  // no step is live in any lane beyond
  float A = 1.0f, M = 0.0f, Q = 0.0f;
  for (int32_t t0 = t_begin; t0 < t_live; t0 += U) {
    E z[U], x[U], d[U];
    auto rz = pz.row(t0), rx = px.row(t0), rd = pd.row(t0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      z[u] = pz.in(rz);
      if (kStates) x[u] = px.in(rx);
      d[u] = pd.in(rd);
      const bool more = t0 + u + 1 < t_live;
      rz += more ? pz.step : 0;
      rx += more ? px.step : 0;
      rd += more ? pd.step : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float a, c;
      gate(load_as_f32(&z[u]), a, c);
      const float dh = has_d ? load_as_f32(&d[u]) : 0.0f;
      const bool in = t0 + u < live;
      // the adjoint of a step reaches the state before the stretch through the gates up to its own
      A = in ? A * a : A;
      M = in ? fmaf(A, dh, M) : M;
      if (kStates) {
        const float xv = load_as_f32(&x[u]);
        Q = in ? a * Q + (COUPLED ? c * xv : xv) : Q;
      }
    }
  }
  sums[wave][lane] = make_float2(A, M);
  if (kStates) states[wave][lane] = Q;
  __syncthreads();
  if (wave == 0 && p.on) {
    float2 m = make_float2(1.0f, 0.0f);
    const int64_t at = s * (k.B * k.H) + p.j;
#pragma unroll
    for (int i = kWaves - 1; i >= 0; --i) {
      const float2 o = sums[i][lane];
      m = make_float2(o.x * m.x, fmaf(o.x, m.y, o.y));
    }
    cut.sums[at] = m;
    if (kStates) {
      float q = 0.0f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) q = fmaf(sums[i][lane].x, q, states[i][lane]);
      cut.states[at] = q;
    }
  }
}

// ---------------------------------------------------------------------------
// Choice of the variant, for N states: alone where a thread to each state fills the GPU for
// so few steps, chained, or in segments, where the tiles of states leave compute units idle
// for so many steps that it pays for another launch and the waiting, or the second reading.
// Forward and gradient in us, bf16, T steps of so many tiles of 64 states (a training step takes
// both, so their sum decides):
//                          alone          shared
//   1024 tiles, T 16    4.4 and 6.5    6.1 and 16.2
//   512 tiles, T 32     5.7 and 10.1   4.4 and 9.6
//   1024 tiles, T 32    6.1 and 11.4   7.0 and 16.0
//   1024 tiles, T 64    9.4 and 18.4   7.7 and 16.5
//   2048 tiles, T 64   14.3 and 29.2  13.5 and 30.2   (float32 22.2 and 28.7, 23.8 and 36.5)
//   2048 tiles, T 128  26.4 and 54.5  23.7 and 54.1
//   4096 tiles, T 64   23.4 and 44.0  24.9 and 58.2
// Forward, bf16, in one piece against chained: 8 tiles, T 1024 20.8 and 9.5, T 16384 295 and
// 21; 128 tiles, T 1024 22 and 16, T 4096 76 and 44; 188 tiles, T 1024 24 and 27, T 2048 43
// and 43. Gradient in one piece against segments, both launches: bf16, 128 tiles, T 2048 106 and
// 73; 160 tiles, T 777 46 and 37; 204 tiles, T 777 50 and 59, in float32 44 and 52. Few
// steps do not pay: 160 tiles, T 300 20 and 25, in float32 16 and 19, 8 tiles 18.0 and 18.8.
// Where sequences end at lengths the longest hold a few compute units longest: 192 tiles,
// T 2048 105 and 95; 320 tiles, T 2048 158 and 159, in float32 179 and 166; 384 tiles, T 1024,
// float32 89 and 100.
// ---------------------------------------------------------------------------
constexpr int64_t kBlocks = 512;       // two workgroups on a compute unit
constexpr int64_t kUncut = 192;        // tiles from which a gradient is not cut
constexpr int64_t kUncutRagged = 352;  // where sequences have lengths
constexpr int64_t kUnchained = 160;    // and a forward call not chained
constexpr int32_t kShortest = 128;     // steps of a segment at least
constexpr int64_t kCutSteps = 384;     // steps from which a gradient is cut

bool alone(int64_t T, int64_t N) {
  const int64_t tiles = (N + 63) / 64;
  return T <= 2 * kUnroll || tiles >= 4096 || T * 32 <= tiles;
}
bool chained(int64_t T, int64_t N) {
  return !alone(T, N) && (N + 63) / 64 < kUnchained && T >= 2 * kWaves * kChainedUnroll;
}

// Segments of a gradient, and the steps of one.
int segments(int64_t T, int64_t N, bool ragged, int32_t* len) {
  const int64_t tiles = (N + 63) / 64, step = kWaves * kUnroll;
  int64_t S = alone(T, N) || tiles >= (ragged ? kUncutRagged : kUncut) ? 1 : (kBlocks + tiles - 1) / tiles;
  if (S > T / kShortest) S = T / kShortest;
  if (T < kCutSteps) S = 1;
  const int64_t L = S == 1 ? T : ((T + S - 1) / S + step - 1) / step * step;
  *len = static_cast<int32_t>(L);
  return static_cast<int>((T + L - 1) / L);
}

int blocks_of(int64_t T) {
  constexpr int steps = kWaves * kChainedUnroll;
  return static_cast<int>((T + steps - 1) / steps);
}

template <typename E, bool COUPLED> hipError_t forward(const GatedScan& c, void* ws, hipStream_t s) {
  const int64_t N = c.B * c.H;
  Chain chain{1, static_cast<int>((N + 63) / 64), nullptr, nullptr};
  if (alone(c.T, N)) {
    chain.tiles = (chain.tiles + 3) / 4;
    launch_kernel(dlvm_gated_scan_kernel<E, COUPLED, ALONE>, dim3(chain.tiles), dim3(256), s, c, chain);
  } else if (ws == nullptr || !chained(c.T, N)) {
    launch_kernel(dlvm_gated_scan_kernel<E, COUPLED, SHARED>, dim3(chain.tiles), dim3(64 * kWaves), s, c, chain);
  } else {
    chain.blocks = blocks_of(c.T);
    chain.tickets = static_cast<uint32_t*>(ws);
    chain.words = reinterpret_cast<uint64_t*>(chain.tickets + chain.tiles * kTicketStride);
    const int64_t n = static_cast<int64_t>(chain.blocks) * chain.tiles * 64;
    launch_kernel(dlvm_gated_scan_clear_kernel, dim3(static_cast<uint32_t>((n + 255) / 256)), dim3(256), s, chain, n);
    launch_kernel(dlvm_gated_scan_kernel<E, COUPLED, CHAINED>, dim3(chain.tiles * chain.blocks),
                  dim3(64 * kWaves), s, c, chain);
  }
  return hipGetLastError();
}

template <typename E, bool COUPLED> hipError_t backward(const GatedScan& c, void* ws, hipStream_t s) {
  const int64_t N = c.B * c.H;
  Cut cut{1, static_cast<int32_t>(c.T), static_cast<int>((N + 63) / 64), nullptr, nullptr, nullptr};
  if (alone(c.T, N)) {
    cut.tiles = (cut.tiles + 3) / 4;
    launch_kernel(dlvm_gated_scan_grad_kernel<E, COUPLED, ALONE>, dim3(cut.tiles), dim3(256), s, c, cut);
    return hipGetLastError();
  }
  const dim3 block(64 * kWaves);
  if (ws != nullptr) cut.S = segments(c.T, N, c.lens != nullptr, &cut.len);
  if (cut.S > 1) {
    cut.init = static_cast<float*>(ws);
    cut.sums = reinterpret_cast<float2*>(cut.init + (N + 63) / 64 * 64);
    cut.states = reinterpret_cast<float*>(cut.sums + cut.S * N);
    launch_kernel(dlvm_gated_scan_sums_kernel<E, COUPLED && kRecompute<E>>,
                  dim3(cut.tiles * (cut.S - (kRecompute<E> ? 0 : 1))), block, s, c, cut);
  }
  launch_kernel(dlvm_gated_scan_grad_kernel<E, COUPLED, SHARED>, dim3(cut.tiles * cut.S), block, s, c, cut);
  return hipGetLastError();
}

}  // namespace

size_t gated_scan_ws(int dtype, int64_t T, int64_t B, int64_t H) {
  int32_t len = 0;
  const int64_t N = B * H, S = segments(T, N, true, &len);  // as many as without lengths, or more
  const size_t tiles = static_cast<size_t>((N + 63) / 64);
  const size_t maps = dtype == BF16 ? 12 : 8;  // bytes of a segment's
  size_t bytes = S == 1 ? 256 : tiles * 64 * 4 + static_cast<size_t>(S) * N * maps;
  if (chained(T, N)) {
    const size_t chain = tiles * (kTicketStride * 4 + static_cast<size_t>(blocks_of(T)) * 64 * 8);
    bytes = chain > bytes ? chain : bytes;
  }
  return bytes;
}

hipError_t launch_gated_scan_forward(const GatedScan& c, void* ws, hipStream_t s) {
  if (c.dtype == F32) return (c.coupled ? forward<float, true> : forward<float, false>)(c, ws, s);
  return (c.coupled ? forward<bf16_t, true> : forward<bf16_t, false>)(c, ws, s);
}

hipError_t launch_gated_scan_backward(const GatedScan& c, void* ws, hipStream_t s) {
  if (c.dtype == F32) return (c.coupled ? backward<float, true> : backward<float, false>)(c, ws, s);
  return (c.coupled ? backward<bf16_t, true> : backward<bf16_t, false>)(c, ws, s);
}

}  // namespace dlvm

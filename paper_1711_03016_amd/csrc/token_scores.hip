// Scores of tokens under rows of logits: log probabilities of given tokens,
// log-sum-exp, entropy and the largest alternatives, and the gradient of the log
// probabilities and the entropy.
//
// The scores are taken in one pass over the logits. Each thread keeps the running
// maximum m of its logits and the sums s = sum 2^t and w = sum 2^t t, t the distance of
// scale z log2(e) from that maximum; they are rescaled once for every 16 logits, when a new
// maximum is known. The entropy is log s - w / s: all terms of w have one sign, so it
// has no cancellation beyond its own size. Alternatives are collected in the same pass:
// from the first tile of a row comes a bound that at least `top` logits reach (the
// top-th largest of 64 maxima of disjoint parts of it, taken again after 2, 4, ... tiles),
// and the few logits that reach it are kept in LDS, in lists of the waves that are cut back
// to the `top` best when full. So the common logit costs one comparison for eight, and any
// order of logits is right.
// A row is a wave's where it is short or there are many, else a workgroup's of four or
// eight; with a workspace, a call of few long rows cuts them into parts, joined by a second
// launch.
// bf16 logits are bound by both memory and arithmetic (about ten operations for two
// bytes, the exponential four of them), float32 ones by memory.
#include <math.h>

#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace dlvm {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
// Up to this size scale z log2(e) is taken in one operation from a maximum rounded
// after the product (whose rounding is accounted for); beyond, from differences of the
// logits themselves: the rounding of a product the size of the type's lowest value is
// larger than any exponent.
constexpr float kPlain = 16384.0f;

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

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float log2_(float v) { return __builtin_amdgcn_logf(v); }

// Sum and maximum over the wave, the same bits in every lane: rotations within rows of 16
// lanes, then the four rows in order.
__device__ __forceinline__ float lane_value(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = row16_sum(v);
  return ((lane_value(v, 0) + lane_value(v, 16)) + lane_value(v, 32)) + lane_value(v, 48);
}
__device__ __forceinline__ float wave_max(float v) {
  v = row16_max(v);
  return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
__device__ __forceinline__ int bits_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32),
                                   __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0));
}

// Of a set of logits: their maximum m and, with t = (z - m) scale log2(e) + r, s = sum 2^t
// and w = sum 2^t t. (r: what a maximum rounded after its product is off by; 0 once the set is
// complete.)
struct Part {
  float m, s, w;
};

// Nothing left: every class is masked, by -infinity or by the type's lowest value.
__device__ __forceinline__ bool masked_everywhere(const Part& p, float scale) {
  return p.s == 0.0f || (p.s == p.s && p.m * scale < -1e30f);
}

// p moved to the maximum m >= p.m, d = (p.m - m) scale log2(e) - r. (Nothing to move where
// the set is empty, whose d may be infinite. One of masked classes alone may have a d of the
// size of the type's lowest value: e is 0 there, and long before d reaches -1e4, so that it is
// multiplied with a finite number. NaN and +infinity come through in s.)
__device__ __forceinline__ void move_to(Part& p, float m, float d) {
  const float e = exp2_(d);
  p.w = p.s == 0.0f ? 0.0f : (p.w + p.s * fmaxf(d, -1e4f)) * e;
  p.s = p.s == 0.0f ? 0.0f : p.s * e;
  p.m = m;
}

template <typename T> struct Vec;
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  struct __attribute__((packed, aligned(2))) Raw { uint32_t w[4]; } raw;
  __device__ __forceinline__ float operator[](int i) const {
    return __uint_as_float(i % 2 == 0 ? raw.w[i / 2] << 16 : raw.w[i / 2] & 0xffff0000u);
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  struct __attribute__((packed, aligned(4))) Raw { uint32_t w[4]; } raw;
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(raw.w[i]); }
};

// ---------------------------------------------------------------------------
// Alternatives. The list of a wave: keys in LDS, no more than kList; `tau` is the greatest
// key that is not wanted any more, `bound` the least logit that may be wanted. (A wave's
// row of up to kList classes fits whole.)
// ---------------------------------------------------------------------------
constexpr int kList = 256;

struct Wanted {
  uint64_t tau;
  float bound;
  int n;
  bool strict;  // the list has been cut back: of equal logits only some are wanted
};

// Cuts the list back to its `top` best, in order.
__device__ __forceinline__ void cut_back(volatile uint64_t* list, Wanted& f, int top) {
  const int lane = threadIdx.x & 63;
  uint64_t mine[kList / 64];
  int rank[kList / 64];
#pragma unroll
  for (int i = 0; i < kList / 64; ++i) {
    mine[i] = lane + 64 * i < f.n ? list[lane + 64 * i] : 0;
    rank[i] = 0;
  }
#pragma unroll 1
  for (int j = 0; j < f.n; ++j) {
    const uint64_t other = list[j];
#pragma unroll
    for (int i = 0; i < kList / 64; ++i) rank[i] += other > mine[i];
  }
#pragma unroll
  for (int i = 0; i < kList / 64; ++i)
    if (lane + 64 * i < f.n && rank[i] < top) list[rank[i]] = mine[i];
  if (f.n >= top) {
    f.n = top;
    const uint64_t last = list[top - 1];
    const uint32_t high = __builtin_amdgcn_readfirstlane(static_cast<int>(last >> 32));
    const uint32_t low = __builtin_amdgcn_readfirstlane(static_cast<int>(last));
    f.tau = static_cast<uint64_t>(high) << 32 | low;
    f.bound = key_logit(f.tau);
    f.strict = true;
  }
}

// How many keys of a list are greater.
__device__ __forceinline__ int greater_of(const uint64_t* list, int n, uint64_t key) {
  int rank = 0;
#pragma unroll 8
  for (int j = 0; j < n; ++j) rank += list[j] > key;
  return rank;
}

// One logit of each lane, where it may be wanted, at the end of the list as far as there is
// room; counted all the same.
__device__ __forceinline__ void append(volatile uint64_t* list, Wanted& f, float z, uint32_t c, bool valid) {
  bool wanted = valid && !(z < f.bound);
  if (__ballot(wanted) == 0) return;
  const uint64_t key = rank_key(z, c);
  if (f.strict) wanted = wanted && key > f.tau;
  const uint64_t take = __ballot(wanted);
  const int at = f.n + bits_below(take);
  if (wanted && at < kList) list[at] = key;
  f.n += __builtin_popcountll(take);
}

// The logits of one tile, class c0 + i of each lane's U vectors of N, 64 classes at a time with
// room made before each: for the tile that would overflow the list. It reads them again.
template <typename T, int N, int U>
__device__ __forceinline__ void append_carefully(volatile uint64_t* list, Wanted& f, int top, const T* z,
                                                 int c0, int stride, int c1) {
#pragma unroll 1
  for (int i = 0; i < U * N; ++i) {
    const int c = c0 + (i / N) * stride + i % N;
    const bool valid = c < c1;
    const float v = valid ? load_as_f32(z + c) : 0.0f;
    if (f.n + 64 > kList) cut_back(list, f, top);
    append(list, f, v, static_cast<uint32_t>(c), valid);
  }
}

// A number that at least `top` of the wave's 64 reach: the top-th largest with its last 16
// bits cleared, found bit by bit from counts of those that reach a number. (One comparison a
// bit: 64 values ranked against each other cost more than the rest of a tile.)
__device__ __forceinline__ uint32_t reached_by(uint32_t mine, int top) {
  uint32_t reached = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    const uint32_t with = reached | (1u << b);
    if (__builtin_popcountll(__ballot(mine >= with)) >= top) reached = with;
  }
  return reached;
}
__device__ __forceinline__ float reached_by(float v, int top) {
  const uint32_t reached = reached_by(static_cast<uint32_t>(rank_key(v, 0) >> 32), top);
  constexpr uint32_t lowest = 0x007fffffu;  // of -infinity
  return key_logit(static_cast<uint64_t>(reached < lowest ? lowest : reached) << 32);
}

// Maximum over each two, four or eight lanes, in all of them.
template <int LANES> __device__ __forceinline__ float max_of(float v) {
  static_assert(LANES == 2 || LANES == 4 || LANES == 8, "");
  v = fmaxf(v, row_rot<0xB1>(v));                     // the other lane of a pair
  if (LANES > 2) v = fmaxf(v, row_rot<0x4E>(v));      // the other pair of four
  return LANES > 4 ? fmaxf(v, row_rot<0x141>(v)) : v;  // the other four
}

// ---------------------------------------------------------------------------
// Scores. NW waves share a row (or a part of one); NW = 1: four rows to a workgroup.
// ---------------------------------------------------------------------------
constexpr int kLogits = 16;  // of a thread in a tile (32 of bf16 took registers for waves: 233 against 218 us)
constexpr int kUnroll = 4;   // vectors of a thread of the gradient in flight

struct Cut {
  int parts;          // of a row (1: whole rows)
  int64_t len;        // classes of a part
  Part* stats;        // [rows * parts]
  uint64_t* keys;     // [rows * parts][top], falling, 0 where a part has fewer
};

// The scores of a row from its complete sums; z is the token's logit.
__device__ __forceinline__ void write_scores(const TokenScores& k, int64_t row, const Part& p, float log_s,
                                             bool masked, float z) {
  if (k.lse != nullptr) k.lse[row] = masked ? -INFINITY : p.m * k.scale + log_s;
  if (k.entropy != nullptr) k.entropy[row] = masked ? 0.0f : log_s - p.w / p.s * kLn2;
  if (k.logp != nullptr) {
    const int32_t t = k.tokens[row];
    k.logp[row] = t == -1                     ? 0.0f
                  : t < 0 || t >= k.classes   ? NAN
                  : masked                    ? -INFINITY
                                              : (z - p.m) * k.scale - log_s;
  }
}
__device__ __forceinline__ void write_top(const TokenScores& k, int64_t row, int rank, uint64_t key,
                                          const Part& p, float log_s, bool masked) {
  k.top_ids[row * k.top + rank] = static_cast<int32_t>(key_class(key));
  k.top_logp[row * k.top + rank] = masked ? -INFINITY : (key_logit(key) - p.m) * k.scale - log_s;
}

template <typename T>
__device__ __forceinline__ float token_logit(const TokenScores& k, int64_t row) {
  if (k.tokens == nullptr) return 0.0f;
  const int32_t t = k.tokens[row];
  return t >= 0 && t < k.classes ? load_as_f32(static_cast<const T*>(k.logits) + row * k.ld + t) : 0.0f;
}

template <typename T, int NW, bool TOP, bool PARTS>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void dlvm_token_scores_kernel(TokenScores k, Cut cut) {
  constexpr int N = Vec<T>::N, WAVES = NW == 1 ? 4 : NW, U = kLogits / N;
  constexpr int tile = 64 * NW * N * U;  // classes
  __shared__ uint64_t lists[TOP ? WAVES : 1][TOP ? kList : 1];
  __shared__ float heads[TOP && NW > 1 ? 2 : 1][64];
  __shared__ float red[3][WAVES];
  __shared__ int counts[WAVES];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const int tid = NW == 1 ? lane : threadIdx.x;
  int64_t row = NW == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + wave : blockIdx.x;
  int part = 0;
  if (PARTS) {
    part = static_cast<int>(blockIdx.x % static_cast<uint32_t>(cut.parts));
    row = blockIdx.x / static_cast<uint32_t>(cut.parts);
  }
  if (row >= k.rows) return;  // only whole waves of NW = 1, which meet no barrier
  const T* z = static_cast<const T*>(k.logits) + row * k.ld;
  const int classes = static_cast<int>(k.classes);
  const int c0 = PARTS ? part * static_cast<int>(cut.len) : 0;
  const int c1 = PARTS && classes - c0 > cut.len ? c0 + static_cast<int>(cut.len) : classes;
  const float c2 = k.scale * kLog2e;
  const float zt = !PARTS && tid == 0 ? token_logit<T>(k, row) : 0.0f;

  Part p{-INFINITY, 0.0f, 0.0f};
  float r = 0.0f;
  Wanted f{0, -INFINITY, 0, false};
  uint64_t* list = TOP ? lists[wave] : nullptr;

  // The vectors of the tile that starts at class `at`, without a branch for each (it would be
  // waited for before the next is sent): a vector that would reach over the end of the row
  // is taken N classes before it. first_of(at, u) is the first class of the thread's u-th, and
  // from twice_of on its elements are classes that no other vector has.
  constexpr int stride = 64 * NW * N;
  const bool tiny = c1 - c0 < N;  // not one vector: an element to each of the first threads
  const int mine = tid * (tiny ? 1 : N);
  const auto first_of = [&](int at, int u) {
    const int c = at + u * stride + mine;
    return tiny || c <= c1 - N ? c : c1 - N;
  };
  const auto twice_of = [&](int at, int u) {
    const int c = at + u * stride + mine;
    return c >= c1 ? N : tiny || c <= c1 - N ? 0 : c - (c1 - N);
  };
  Vec<T> v[U];
  const auto load = [&](int at) {
    if (tiny) {
      if (c0 + tid < c1)
        v[0].raw.w[0] = sizeof(T) == 2 ? reinterpret_cast<const uint16_t*>(z)[c0 + tid]
                                       : reinterpret_cast<const uint32_t*>(z)[c0 + tid];
    } else if (c1 - at >= tile) {
      const T* from = z + at + mine;
#pragma unroll
      for (int u = 0; u < U; ++u) v[u].raw = *reinterpret_cast<const typename Vec<T>::Raw*>(from + u * stride);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at + u * stride < c1)
          v[u].raw = *reinterpret_cast<const typename Vec<T>::Raw*>(z + first_of(at, u));
    }
  };

  // One tile, all of whose vectors are there (WHOLE) or not.
  unsigned done = 0;  // tiles
  const auto pass = [&](auto all, int at) {
    constexpr bool whole = decltype(all)::value;
    ++done;
    float zs[U][N], top_of[U];
    float big = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      top_of[u] = -INFINITY;
      if (!whole && at + u * stride >= c1) continue;
#pragma unroll
      for (int i = 0; i < N; ++i) zs[u][i] = v[u][i];
      if (!whole) {
        const int from = twice_of(at, u), to = tiny ? 1 : N;
#pragma unroll
        for (int i = 0; i < N; ++i) zs[u][i] = i >= from && i < to ? zs[u][i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) top_of[u] = fmaxf(top_of[u], zs[u][i]);
      big = fmaxf(big, top_of[u]);
    }
    if (c1 - at > tile) load(at + tile);

    // the maximum so far, and the sums moved to it
    const float m = fmaxf(p.m, big);
    const float ref = m == -INFINITY ? 0.0f : m;  // nothing yet: any reference does
    float M = ref * c2;
    const bool plain = __all(fabsf(M) < kPlain) != 0;
    const float r_new = plain ? fmaf(ref, c2, -M) : 0.0f;
    move_to(p, m, (p.m - ref) * c2 + (r_new - r));
    r = r_new;
    if (plain) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!whole && at + u * stride >= c1) break;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float t = fmaf(zs[u][i], c2, -M);
          const float e = exp2_(t);
          p.s += e;
          p.w = fmaf(e, fmaxf(t, -1e4f), p.w);  // a masked class: 0 times a finite number
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!whole && at + u * stride >= c1) break;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float t = (zs[u][i] - ref) * c2;
          const float e = exp2_(t);
          p.s += e;
          p.w = fmaf(e, fmaxf(t, -1e4f), p.w);
        }
      }
    }

    if (TOP) {
      // after 1, 2, 4, ... tiles: what the maxima so far tell (each wave reads one set while
      // the next is written to the other)
      if ((done & (done - 1)) == 0) {
        float head = m;
        if constexpr (NW > 1) {  // of NW threads, so that 64 heads cover the workgroup
          float* set = heads[__builtin_ctz(done) % 2];
          head = max_of<NW>(m);
          if (lane % NW == 0) set[(wave * 64 + lane) / NW] = head;
          __syncthreads();
          head = set[lane];
        }
        f.bound = fmaxf(f.bound, lane_value(reached_by(head, k.top), 0));
      }
      const int had = f.n;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if ((whole || at + u * stride < c1) && __any(!(top_of[u] < f.bound))) {
          const int c = whole ? at + u * stride + mine : first_of(at, u);
          const int from = whole ? 0 : twice_of(at, u), to = whole || !tiny ? N : 1;
#pragma unroll
          for (int i = 0; i < N; ++i)
            append(list, f, zs[u][i], static_cast<uint32_t>(c + i), whole || (i >= from && i < to));
        }
      if (f.n > kList) {  // never in a tiny row
        f.n = had;
        append_carefully<T, N, U>(list, f, k.top, z, at + tid * N, stride, c1);
      }
    }
  };
  load(c0);
  int at = c0;
  for (; c1 - at >= tile; at += tile) pass(std::true_type{}, at);
  if (at < c1) pass(std::false_type{}, at);

  // the row's maximum, then its sums
  float m = wave_max(p.m);
  if (NW > 1) {
    if (lane == 0) {
      red[0][wave] = m;
      counts[wave] = f.n;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, red[0][w]);
  }
  move_to(p, m, (p.m - m) * c2 - r);
  p.s = wave_sum(p.s);
  p.w = wave_sum(p.w);
  if (NW > 1) {
    if (lane == 0) {
      red[1][wave] = p.s;
      red[2][wave] = p.w;
    }
    __syncthreads();
    p.s = red[1][0];
    p.w = red[2][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      p.s += red[1][w];
      p.w += red[2][w];
    }
  }
  const float log_s = log2_(p.s) * kLn2;
  const bool masked = masked_everywhere(p, k.scale);
  if (tid == 0) {
    if (PARTS)
      cut.stats[blockIdx.x] = p;
    else
      write_scores(k, row, p, log_s, masked, zt);
  }
  if (!TOP) return;

  // the rank of each kept key among all of them
  const auto put = [&](uint64_t key, int rank) {
    if (rank >= k.top) return;
    if (PARTS)
      cut.keys[static_cast<int64_t>(blockIdx.x) * k.top + rank] = key;
    else
      write_top(k, row, rank, key, p, log_s, masked);
  };
  if (NW == 1) {
    __builtin_amdgcn_wave_barrier();
    for (int i = lane; i < f.n; i += 64) {
      const uint64_t key = list[i];
      put(key, greater_of(list, f.n, key));
    }
  } else {
    int total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) total += counts[w];
    for (int w = 0; w < NW; ++w)  // the threads in turn over the lists of the waves
      for (int i = (tid + 64 * NW - 64 * w) % (64 * NW); i < counts[w]; i += 64 * NW) {
        const uint64_t key = lists[w][i];
        int rank = 0;
        for (int o = 0; o < NW; ++o) rank += greater_of(lists[o], counts[o], key);
        put(key, rank);
      }
    if (PARTS && tid >= total && tid < k.top)
      cut.keys[static_cast<int64_t>(blockIdx.x) * k.top + tid] = 0;
  }
}

// The parts of a row: their sums joined in order, and the best of their keys. Those below what
// `top` of the parts' first keys reach are not ranked (64 first keys or all, never fewer
// than `top`). All loads are sent before the first is waited for.
constexpr int kMaxParts = 64;
constexpr int kJoinKeys = kMaxParts * kTopMax / 256;  // of a thread

template <typename T>
__global__ __launch_bounds__(256) void dlvm_token_scores_join_kernel(TokenScores k, Cut cut) {
  __shared__ uint64_t keys[256 * kJoinKeys];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x;
  const float c2 = k.scale * kLog2e;
  const int total = cut.parts * k.top;
  const uint64_t* from = cut.keys + row * total;
  const int own = lane < cut.parts ? lane : 0;
  Part p = cut.stats[row * cut.parts + own];
  uint64_t mine[kJoinKeys] = {};
  uint32_t first = 0;
  if (k.top > 0) {
    const int j = lane / cut.parts;
    const bool has = j < 64 / cut.parts && j < k.top;
    first = has ? static_cast<uint32_t>(from[(lane - j * cut.parts) * k.top + j] >> 32) : 0;
#pragma unroll
    for (int i = 0; i < kJoinKeys; ++i)
      if (256 * i < total) mine[i] = from[tid + 256 * i < total ? tid + 256 * i : total - 1];
  }
  const float zt = tid == 0 ? token_logit<T>(k, row) : 0.0f;
  if (tid == 0) count = 0;
  if (lane >= cut.parts) p = Part{-INFINITY, 0.0f, 0.0f};
  const float m = wave_max(p.m);
  move_to(p, m, (p.m - m) * c2);
  p.s = wave_sum(p.s);
  p.w = wave_sum(p.w);
  const float log_s = log2_(p.s) * kLn2;
  const bool masked = masked_everywhere(p, k.scale);
  if (tid == 0) write_scores(k, row, p, log_s, masked, zt);
  if (k.top == 0) return;
  const uint32_t least = reached_by(first, k.top);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kJoinKeys; ++i)
    if (tid + 256 * i < total && mine[i] != 0 && static_cast<uint32_t>(mine[i] >> 32) >= least)
      keys[atomicAdd(&count, 1)] = mine[i];
  __syncthreads();
  const int n = count;
  for (int i = tid; i < n; i += 256) {
    const uint64_t key = keys[i];
    const int rank = greater_of(keys, n, key);
    if (rank < k.top) write_top(k, row, rank, key, p, log_s, masked);
  }
}

// ---------------------------------------------------------------------------
// Gradient: with p = exp(y - lse) one pass over the logits, -p (dlogp + dentropy (log p + H))
// and dlogp more at the token. NT threads take a stretch of a row: a wave where the row is
// short (16384 rows of 100 bf16 10 us, 22 with 256 threads, of 1000 14 and 22), else a
// workgroup (2048 rows of 50001 float32 133 us, 141 with waves).
// ---------------------------------------------------------------------------
struct ScoresGrad {
  int64_t rows, classes;
  const void* logits; int64_t ld;
  float scale;
  const int32_t* tokens;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* dlogits; int64_t ld_out;
  int chunks;  // stretches of a row
};

template <typename TD, int N> struct __attribute__((packed, aligned(sizeof(TD)))) OutVec {
  TD v[N];
};

template <typename T, typename TD, int NT>
__global__ __launch_bounds__(256) void dlvm_token_scores_grad_kernel(ScoresGrad k) {
  constexpr int N = Vec<T>::N, U = kUnroll;
  const int tid = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t item = NT == 64 ? static_cast<int64_t>(blockIdx.x) * 4 +
                                      __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6))
                                : blockIdx.x;
  const int64_t row = item / k.chunks;
  if (row >= k.rows) return;
  const int64_t at = (item - row * k.chunks) * (NT * N * U);
  const T* z = static_cast<const T*>(k.logits) + row * k.ld;  // may be dlogits: not restrict
  TD* d = static_cast<TD*>(k.dlogits) + row * k.ld_out;
  const float lse = k.lse[row];
  const float ge = k.dentropy != nullptr ? k.dentropy[row] : 0.0f;
  const float H = k.dentropy != nullptr ? k.entropy[row] : 0.0f;
  float gl = 0.0f;
  int64_t token = -1;
  if (k.dlogp != nullptr) {
    token = k.tokens[row];
    gl = token == -1 ? 0.0f : token < 0 || token >= k.classes ? NAN : k.dlogp[row];
  }
  if (token == -1 && ge == 0.0f) {  // no adjoint: a row of padding, whatever its logits hold
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c = at + (u * NT + tid) * N;
      if (c + N <= k.classes)
        *reinterpret_cast<OutVec<TD, N>*>(d + c) = OutVec<TD, N>{};
      else
        for (int64_t i = c; i < k.classes; ++i) d[i] = store_cast<TD>(0.0f);
    }
    return;
  }
  const bool masked = lse == -INFINITY && gl == gl;
  // -scale p (gl + ge (log p + H)) = p (a + b max(log p, -1e4)); p is 0 where the maximum acts
  const float a = masked ? 0.0f : -k.scale * fmaf(ge, H, gl), b = masked ? 0.0f : -k.scale * ge;
  const float hot = masked ? 0.0f : k.scale * gl;
  const float ref = masked ? INFINITY : lse;  // every p of a masked row is 0

  const auto gradient = [&](float v) {
    const float lp = fmaf(v, k.scale, -ref);
    const float p = exp2_(lp * kLog2e);
    return p * fmaf(b, fmaxf(lp, -1e4f), a);
  };
  Vec<T> v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = at + (u * NT + tid) * N;
    if (c + N <= k.classes) v[u].raw = *reinterpret_cast<const typename Vec<T>::Raw*>(z + c);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t c = at + (u * NT + tid) * N;
    if (c + N <= k.classes) {
      float g[N];
#pragma unroll
      for (int i = 0; i < N; ++i) g[i] = gradient(v[u][i]);
      const int64_t own = token - c;
      if (own >= 0 && own < N)
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] += own == i ? hot : 0.0f;
      OutVec<TD, N> o;
#pragma unroll
      for (int i = 0; i < N; ++i) o.v[i] = store_cast<TD>(g[i]);
      *reinterpret_cast<OutVec<TD, N>*>(d + c) = o;
    } else {
      for (int64_t i = c; i < k.classes; ++i)
        d[i] = store_cast<TD>(gradient(load_as_f32(z + i)) + (i == token ? hot : 0.0f));
    }
  }
}

// ---------------------------------------------------------------------------
// Choice of the variant.
// ---------------------------------------------------------------------------
// us of scores with 5 alternatives, in rows x classes of bf16, by the waves to a row:
//                   1      4      8
//   256 x 1500     6.5           6.2
//   1024 x 1500    6.6          10.8
//   512 x 4000     9.8    6.4    7.2   (700 x 4000 6.8 and 8.3, 512 x 8000 8.4 and 8.2)
//   512 x 131072  89     36     32
//   1024 x 4000   10.3    7.5   11.1
//   1024 x 131072 94     54     55
//   4096 x 4000   15.3   17.6   31.9
//   4096 x 16000  33.7   37.5   52.6
//   4096 x 32000  55.6   56.3   73.6
//   4096 x 65536         103    104
//   4096 x 131072        194    185
//   4096 x 8000 float32   31     32     41
//   4096 x 32000 float32  94     96     93
// (A workgroup of more waves waits longer for the last of them at each of its barriers and
// ranks more keys at the end; few rows want the waves.) Whole rows against parts and their
// join, of both launches with what lies between: with 20 alternatives 8 x 32000 12.9 and
// 11.4, 8 x 50000 14.9 and 11.2, with 5 1 x 32000 9.4 and 10.3, 32 x 32000 10.3 and 10.2,
// 96 x 50000 12.2 and 12.6; with none 1 x 50000 6.9 and 8.9, 1 x 100000 10.8 and 10.5,
// 8 x 131072 13.1 and 11.1.
constexpr int64_t kWaveRow = 2048;      // classes up to which a wave takes a row
constexpr int64_t kWaveRows = 4096;     // rows from which it takes one
constexpr int64_t kWaveRowOfMany = 16384;  // of up to so many classes
constexpr int64_t kFourRows = 512;      // rows from which four waves take one, else eight,
constexpr int64_t kFourBytes = 96 << 10;  // if it has up to so many bytes
constexpr int64_t kCutRow = 32768;      // classes from which a row is cut into parts,
constexpr int64_t kCutPlain = 98304;    // or these without alternatives,
constexpr int64_t kCutRows = 128;       // where there are fewer rows
constexpr int64_t kPartLen = 4096;      // classes of a part at least (as fast with 8192)
constexpr int64_t kBlocks = 512;        // workgroups that fill the GPU
constexpr int64_t kTurn = 1 << 22;      // workgroups of a launch (its threads are counted in 32 bits)

int parts_of(int64_t rows, int64_t classes, int top, int64_t* len) {
  *len = classes;
  if (classes < (top > 0 ? kCutRow : kCutPlain) || rows >= kCutRows) return 1;
  int64_t S = kBlocks / rows;
  if (S > classes / kPartLen) S = classes / kPartLen;
  if (S > kMaxParts) S = kMaxParts;
  const int64_t L = ((classes + S - 1) / S + 511) / 512 * 512;
  *len = L;
  return static_cast<int>((classes + L - 1) / L);
}

template <typename T> hipError_t scores(const TokenScores& c, void* ws, hipStream_t s) {
  Cut cut{1, c.classes, nullptr, nullptr};
  if (ws != nullptr) cut.parts = parts_of(c.rows, c.classes, c.top, &cut.len);
  if (cut.parts > 1) {
    cut.keys = static_cast<uint64_t*>(ws);
    cut.stats = reinterpret_cast<Part*>(cut.keys + c.rows * cut.parts * c.top);
    launch_kernel(c.top > 0 ? dlvm_token_scores_kernel<T, 8, true, true>
                            : dlvm_token_scores_kernel<T, 8, false, true>,
                  dim3(static_cast<uint32_t>(c.rows * cut.parts)), dim3(512), s, c, cut);
    launch_kernel(dlvm_token_scores_join_kernel<T>, dim3(static_cast<uint32_t>(c.rows)), dim3(256), s, c, cut);
    return hipGetLastError();
  }
  for (int64_t r0 = 0; r0 < c.rows; r0 += kTurn) {
    TokenScores t = c;
    t.rows = c.rows - r0 < kTurn ? c.rows - r0 : kTurn;
    t.logits = static_cast<const T*>(c.logits) + r0 * c.ld;
    if (c.tokens != nullptr) t.tokens += r0;
    if (c.logp != nullptr) t.logp += r0;
    if (c.lse != nullptr) t.lse += r0;
    if (c.entropy != nullptr) t.entropy += r0;
    if (c.top > 0) {
      t.top_ids += r0 * c.top;
      t.top_logp += r0 * c.top;
    }
    const uint32_t rows = static_cast<uint32_t>(t.rows);
    if (c.classes <= kWaveRow || (c.rows >= kWaveRows && c.classes <= kWaveRowOfMany))
      launch_kernel(c.top > 0 ? dlvm_token_scores_kernel<T, 1, true, false>
                              : dlvm_token_scores_kernel<T, 1, false, false>,
                    dim3((rows + 3) / 4), dim3(256), s, t, cut);
    else if (c.rows >= kFourRows && c.classes * static_cast<int64_t>(sizeof(T)) <= kFourBytes)
      launch_kernel(c.top > 0 ? dlvm_token_scores_kernel<T, 4, true, false>
                              : dlvm_token_scores_kernel<T, 4, false, false>,
                    dim3(rows), dim3(256), s, t, cut);
    else
      launch_kernel(c.top > 0 ? dlvm_token_scores_kernel<T, 8, true, false>
                              : dlvm_token_scores_kernel<T, 8, false, false>,
                    dim3(rows), dim3(512), s, t, cut);
  }
  return hipGetLastError();
}

template <typename T, typename TD> hipError_t grad(ScoresGrad g, hipStream_t s) {
  const int NT = g.classes <= kWaveRow ? 64 : 256;
  const int64_t stretch = NT * Vec<T>::N * kUnroll;
  const int64_t chunks = (g.classes + stretch - 1) / stretch;
  g.chunks = static_cast<int>(chunks);
  const int64_t turn = kTurn / chunks;
  for (int64_t r0 = 0, rows = g.rows; r0 < rows; r0 += turn) {
    ScoresGrad h = g;
    h.rows = rows - r0 < turn ? rows - r0 : turn;
    h.logits = static_cast<const T*>(g.logits) + r0 * g.ld;
    h.dlogits = static_cast<TD*>(g.dlogits) + r0 * g.ld_out;
    h.lse = g.lse + r0;
    h.tokens = g.tokens ? g.tokens + r0 : nullptr;
    h.entropy = g.entropy ? g.entropy + r0 : nullptr;
    h.dlogp = g.dlogp ? g.dlogp + r0 : nullptr;
    h.dentropy = g.dentropy ? g.dentropy + r0 : nullptr;
    const int64_t items = h.rows * chunks;
    launch_kernel(NT == 64 ? dlvm_token_scores_grad_kernel<T, TD, 64> : dlvm_token_scores_grad_kernel<T, TD, 256>,
                  dim3(static_cast<uint32_t>(NT == 64 ? (items + 3) / 4 : items)), dim3(256), s, h);
  }
  return hipGetLastError();
}

}  // namespace

size_t token_scores_ws(int64_t rows, int64_t classes, int top) {
  int64_t len = 0;
  const int64_t parts = parts_of(rows, classes, top, &len);
  return parts == 1 ? 256 : static_cast<size_t>(rows * parts) * (top * 8 + sizeof(Part));
}

hipError_t launch_token_scores(const TokenScores& c, void* ws, hipStream_t s) {
  return c.dtype == F32 ? scores<float>(c, ws, s) : scores<bf16_t>(c, ws, s);
}

hipError_t launch_token_scores_backward(int dtype, int out_dtype, int64_t rows, int64_t classes,
                                        const void* logits, int64_t ld, float scale,
                                        const int32_t* tokens, const float* lse,
                                        const float* entropy, const float* dlogp,
                                        const float* dentropy, void* dlogits, int64_t ld_out,
                                        hipStream_t s) {
  const ScoresGrad g{rows, classes, logits, ld, scale, tokens, lse, entropy, dlogp, dentropy,
                     dlogits, ld_out, 1};
  if (dtype == BF16) return grad<bf16_t, bf16_t>(g, s);
  return out_dtype == BF16 ? grad<float, bf16_t>(g, s) : grad<float, float>(g, s);
}

}  // namespace dlvm

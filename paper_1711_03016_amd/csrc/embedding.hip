// Token embeddings: the lookup with scaling, and the gradient of the table by
// sorted tokens.
//
// The gradient, dtable[v] = scale * sum of dout[i] over the tokens i with id v, uses no
// floating-point atomics: the tokens are sorted by id, equal pieces of the sorted list are
// summed, and the sums of rows that run over a piece's end are joined in the order of the
// pieces. The sort leaves most of the GPU idle, so its launches fill the table with zeros; of a
// large one, the launch that sums the pieces zeroes the rows without a token instead, most of
// its bytes.
#include <math.h>

#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"
#include "sequence.hpp"

namespace dlvm {
namespace {

// VEC elements of a row, at any alignment of the element type.
template <typename T, int VEC> struct __attribute__((packed, aligned(sizeof(T)))) Elems {
  T v[VEC];
};

// ---------------------------------------------------------------------------
// Lookup. The output is taken as N * chunks vectors of VEC elements, one to a thread
// and four in flight, so rows of any width fill the wavefronts; the last vector of a
// row whose width is not a multiple of VEC starts VEC elements before its end (the
// overlap is written twice with the same values).
// ---------------------------------------------------------------------------
constexpr int kLookupUnroll = 4;

// n / d for n < 2^31 by a multiplication: ceil(2^(31 + l) / d) with 2^l >= d fits 32 bits,
// and its error n (m d - 2^(31 + l)) / (d 2^(31 + l)) stays below 1 / d.
struct Divisor {
  uint32_t m;
  int shift;
};
Divisor divisor(uint32_t d) {
  int l = 0;
  while ((uint64_t(1) << l) < d) ++l;
  const uint64_t two = uint64_t(1) << (31 + l);
  return Divisor{static_cast<uint32_t>((two + d - 1) / d), l};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, Divisor d) {
  return static_cast<uint32_t>((static_cast<uint64_t>(n) * d.m) >> 31 >> d.shift);
}

template <typename T, int VEC>
__global__ __launch_bounds__(256) void dlvm_embedding_kernel(uint32_t V, int64_t E, uint32_t chunks,
                                                             Divisor by_chunks, uint32_t total,
                                                             const T* __restrict__ table,
                                                             const int32_t* __restrict__ ids,
                                                             float scale, T* __restrict__ out) {
  using Vec = Elems<T, VEC>;
  const uint32_t stride = gridDim.x * 256;  // total + 4 stride < 2^32
  for (uint32_t q = blockIdx.x * 256 + threadIdx.x; q < total; q += kLookupUnroll * stride) {
    int32_t id[kLookupUnroll];
    int64_t to[kLookupUnroll], from[kLookupUnroll];
    Vec w[kLookupUnroll];
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
      const uint32_t p = q + u * stride < total ? q + u * stride : q;
      const uint32_t i = divide(p, by_chunks);
      int64_t c = static_cast<int64_t>(p - i * chunks) * VEC;
      if (c + VEC > E) c = E - VEC;
      id[u] = ids[i];
      from[u] = c;
      to[u] = i * E + c;
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
      from[u] += (static_cast<uint32_t>(id[u]) < V ? id[u] : 0) * E;
      w[u] = *reinterpret_cast<const Vec*>(table + from[u]);
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
      const bool ok = static_cast<uint32_t>(id[u]) < V;
      const float other = id[u] == -1 ? 0.0f : NAN;
#pragma unroll
      for (int k = 0; k < VEC; ++k)
        w[u].v[k] = store_cast<T>(ok ? scale * load_as_f32(&w[u].v[k]) : other);
      if (q + u * stride < total) *reinterpret_cast<Vec*>(out + to[u]) = w[u];
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient, the sort: stable, by digits of kDigitBits from the lowest, two launches to a
// digit: blocks of tokens count their digits, and place them from the counts of all
// blocks. Counts are whole numbers, so nothing depends on an order of execution, and a
// frequent id costs no more than others. Each wave of a block owns consecutive
// tokens; the lanes of one digit find each other by a ballot to each of its bits. Up to
// kSmallSort tokens are placed by one launch that counts those before each, beside which other
// workgroups zero the table (8000 tokens of 32000 x 1024: gradient 39 us, 54 by
// digits; 1000 tokens placed in 5.2 us, 6.8 by one workgroup and digits in LDS, 8000 in 14.8 and
// 15.8). Ids outside the table are taken as V, one more than the last row: they come last and
// are left out of the sums. (Choosing a row's tokens from all ids, one workgroup to some rows
// and without a sort, took 52 us for 200001 tokens of 1021 rows, for the sake of the most
// frequent row alone.)
// ---------------------------------------------------------------------------
constexpr int kDigitBits = 10;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortThreads = kDigits;                // one thread to a digit
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSmallSort = 8 * kSortThreads;
constexpr int64_t kSortTokens = int64_t(1) << 18;    // tokens of one sort
// Numbers of a table that is filled beside a sort by digits: 9000 tokens of 131072 x 512
// float32 take 77 us (lookup too), 88 with the rows without a token zeroed beside the sums,
// 40000 of 100000 x 301 84 and 90; 65536 of 131072 x 1024 215 and 214.
constexpr int64_t kFillBeside = int64_t(1) << 26;

__device__ __forceinline__ int32_t row_of(int32_t id, int32_t V) {
  return static_cast<uint32_t>(id) < static_cast<uint32_t>(V) ? id : V;
}

// Set bits below the lane's.
__device__ __forceinline__ int bits_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32),
                                   __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0));
}

// Ranks of W vectors of 64 digits (lanes `on`) among the equal ones of the wave so far, whose
// counts are kept in `counts`.
template <int W>
__device__ __forceinline__ void rank_digits(const int32_t (&digit)[W], const bool (&on)[W],
                                            int32_t (&rank)[W], volatile int32_t* counts) {
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const uint64_t valid = __ballot(on[i]);
    if (valid == 0) break;  // the vectors behind the last token
    uint32_t low = static_cast<uint32_t>(valid), high = static_cast<uint32_t>(valid >> 32);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
      const int32_t bit = __builtin_amdgcn_sbfe(digit[i], b, 1);  // 0 or -1
      const uint64_t set = __ballot(bit < 0);
      low &= ~(static_cast<uint32_t>(set) ^ bit);
      high &= ~(static_cast<uint32_t>(set >> 32) ^ bit);
    }
    const uint64_t same = static_cast<uint64_t>(high) << 32 | low;
    const int before = bits_below(same);
    if (on[i]) {
      const int32_t so_far = counts[digit[i]];
      rank[i] = so_far + before;
      if (before == 0) counts[digit[i]] = so_far + __builtin_popcountll(same);
    }
  }
}

// Exclusive sum of one number of each of kSortThreads threads.
__device__ __forceinline__ int32_t exclusive_sum(int32_t v, int32_t* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t up = __shfl_up(incl, o, 64);
    if (lane >= o) incl += up;
  }
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int32_t at = incl - v;
  for (int w = 0; w < wave; ++w) at += sums[w];
  return at;
}

// The waves' counts of the thread's digit, and their sum.
__device__ __forceinline__ int32_t take_counts(const int32_t (*counts)[kDigits], int32_t (&n)[kSortWaves]) {
  int32_t all = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    n[w] = counts[w][threadIdx.x];
    all += n[w];
  }
  return all;
}
// Turns them into places: `base` is where the digit begins.
__device__ __forceinline__ void place_waves(int32_t (*counts)[kDigits], const int32_t (&n)[kSortWaves],
                                            int32_t base) {
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    counts[w][threadIdx.x] = base;
    base += n[w];
  }
}

// kZeroQuads vectors of `numbers` zeros by a workgroup, the b-th.
constexpr int64_t kZeroQuads = 8 * kSortThreads;
__device__ __forceinline__ void zero_part(float* __restrict__ to, int64_t numbers, int b) {
  const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const int64_t q0 = b * kZeroQuads + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kZeroQuads / kSortThreads; ++u) {
    const int64_t at = 4 * (q0 + u * kSortThreads);
    if (at + 4 <= numbers)
      *reinterpret_cast<float4*>(to + at) = zero;
    else
      for (int64_t i = at; i < numbers; ++i) to[i] = 0.0f;
  }
}

// Where the tokens of a pass come from: ids (first pass) or pairs sorted by lower digits; the
// workgroups that sort, and what those behind them zero.
struct SortIn {
  const int32_t* ids;
  const int32_t* row;
  const int32_t* tok;
  int blocks;
  float* zero;
  int64_t zeros;
};

// W tokens of a block to each thread.
template <int W>
__global__ __launch_bounds__(kSortThreads) void dlvm_embedding_count_kernel(int32_t V, int32_t N, int shift,
                                                                            int bits, SortIn in,
                                                                            int32_t* __restrict__ counts) {
  __shared__ int32_t hist[kDigits];
  if (static_cast<int>(blockIdx.x) >= in.blocks)
    return zero_part(in.zero, in.zeros, static_cast<int>(blockIdx.x) - in.blocks);
  hist[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < W; ++u) {
    const int32_t i = (blockIdx.x * W + u) * kSortThreads + threadIdx.x;
    if (i < N) {
      const int32_t row = in.ids != nullptr ? row_of(in.ids[i], V) : in.row[i];
      atomicAdd(&hist[(row >> shift) & ((1 << bits) - 1)], 1);
    }
  }
  __syncthreads();
  counts[blockIdx.x * kDigits + threadIdx.x] = hist[threadIdx.x];
}

template <int W>
__global__ __launch_bounds__(kSortThreads) void dlvm_embedding_place_kernel(
    int32_t V, int32_t N, int shift, int bits, SortIn in, const int32_t* __restrict__ counts,
    int32_t* __restrict__ row_out, int32_t* __restrict__ tok_out) {
  constexpr int kCounts = 8;  // in flight
  __shared__ int32_t places[kSortWaves][kDigits];
  __shared__ int32_t sums[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (static_cast<int>(blockIdx.x) >= in.blocks)
    return zero_part(in.zero, in.zeros, static_cast<int>(blockIdx.x) - in.blocks);
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) places[w][tid] = 0;
  int32_t row[W], tok[W], digit[W], rank[W];
  bool on[W];
#pragma unroll
  for (int u = 0; u < W; ++u) {
    const int32_t i = blockIdx.x * (kSortThreads * W) + wave * 64 * W + u * 64 + lane;
    on[u] = i < N;
    const int32_t at = on[u] ? i : N - 1;
    row[u] = in.ids != nullptr ? row_of(in.ids[at], V) : in.row[at];
    tok[u] = in.ids != nullptr ? at : in.tok[at];
    digit[u] = (row[u] >> shift) & ((1 << bits) - 1);
  }
  // of the thread's digit: tokens of earlier blocks, and of all
  const auto counted = [&](int b, int end) {
    int32_t n = 0;
    for (; b < end; b += kCounts) {
      int32_t c[kCounts];
#pragma unroll
      for (int u = 0; u < kCounts; ++u) c[u] = counts[(b + u < end ? b + u : b) * kDigits + tid];
      if (b + kCounts <= end) {
#pragma unroll
        for (int u = 0; u < kCounts; ++u) n += c[u];
      } else {
#pragma unroll
        for (int u = 0; u < kCounts; ++u) n += b + u < end ? c[u] : 0;
      }
    }
    return n;
  };
  const int32_t earlier = counted(0, blockIdx.x), all = earlier + counted(blockIdx.x, in.blocks);
  const int32_t first = exclusive_sum(all, sums);  // its barrier also follows the zeros above
  rank_digits<W>(digit, on, rank, places[wave]);
  __syncthreads();
  int32_t n[kSortWaves];
  take_counts(places, n);
  place_waves(places, n, first + earlier);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < W; ++u)
    if (on[u]) {
      const int32_t at = places[wave][digit[u]] + rank[u];
      row_out[at] = row[u];
      tok_out[at] = tok[u];
    }
}

// One row of zeros by a wave.
__device__ __forceinline__ void zero_row(float* __restrict__ row, int64_t E) {
  using Quad = Elems<float, 4>;
  const Quad zero{{0.0f, 0.0f, 0.0f, 0.0f}};
  int64_t c = 4 * (threadIdx.x & 63);
  for (; c + 4 <= E; c += 256) *reinterpret_cast<Quad*>(row + c) = zero;
  for (; c < E; ++c) row[c] = 0.0f;
}

// The sort of few tokens: a token's place is the number of tokens that come before it. Each of
// the first `blocks` workgroups places 64 tokens, one to a lane, whose waves compare them with
// equal shares of all ids; each of the others zeroes kZeroQuads vectors of the table, of rows
// with a token too (leaving those out cost more than it saved: 32003 x 1001 float32 in 23.7 us,
// now 18.8, 6.8 TB/s).
__global__ __launch_bounds__(kSortThreads) void dlvm_embedding_sort_kernel(
    int32_t V, int64_t E, int32_t N, int blocks, const int32_t* __restrict__ ids,
    int32_t* __restrict__ row_out, int32_t* __restrict__ tok_out, float* __restrict__ dtable) {
  __shared__ int32_t before[kSortWaves][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int own = static_cast<int>(blockIdx.x);
  if (own >= blocks) return zero_part(dtable, V * E, own - blocks);
  const int32_t tok = own * 64 + lane;
  const int32_t row = row_of(ids[tok < N ? tok : N - 1], V);
  int32_t n = 0;
  for (int c = wave; c < blocks; c += kSortWaves) {
    const int32_t* chunk = ids + c * 64;
    const int count = N - c * 64 < 64 ? N - c * 64 : 64;
    if (c == own) {  // of equal ids the earlier lane's comes first
      for (int j = 0; j < count; ++j) n += __builtin_amdgcn_readlane(row, j) < row + (j < lane ? 1 : 0);
    } else {
      const int32_t bound = row + (c < own ? 1 : 0);
      if (count == 64) {
#pragma unroll
        for (int j = 0; j < 64; ++j) n += row_of(chunk[j], V) < bound;
      } else {
        for (int j = 0; j < count; ++j) n += row_of(chunk[j], V) < bound;
      }
    }
  }
  before[wave][lane] = n;
  __syncthreads();
  if (wave == 0 && tok < N) {
    int32_t at = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) at += before[w][lane];
    row_out[at] = row;
    tok_out[at] = tok;
  }
}

// ---------------------------------------------------------------------------
// Gradient, the sums: a wave sums one piece of the sorted list over a slab of
// 64 * VEC * G columns (G vectors a lane, each contiguous over the wave), eight rows in
// flight. Rows that begin and end inside a piece are written; what belongs to a row that
// began in an earlier piece goes to `head`, the start of one that goes on in the next
// piece to `tail` (float32, without the scale). The workgroups behind those of the pieces zero
// the rows that have no token, 64 to a wave, each found absent by a search of the list.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void zero_absent(int32_t V, int64_t E, int32_t N, int64_t first,
                                            const int32_t* __restrict__ sid, float* __restrict__ dtable) {
  const int lane = threadIdx.x & 63;
  const int64_t v = first + lane;
  int32_t lo = 0, hi = N;  // the first place that holds v or more
  while (lo < hi) {
    const int32_t mid = (lo + hi) >> 1;
    if (sid[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  const bool absent = v < V && !(lo < N && sid[lo] == v);
  for (uint64_t todo = __ballot(absent); todo != 0; todo &= todo - 1)
    zero_row(dtable + (first + __builtin_ctzll(todo)) * E, E);
}

template <int VEC, int G>
__device__ __forceinline__ void store_row(float* __restrict__ to, const int64_t (&c)[G], const bool (&on)[G],
                                          bool add, float scale, float (&acc)[G][VEC]) {
  using Sum = Elems<float, VEC>;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (on[g]) {
      Sum s;
#pragma unroll
      for (int k = 0; k < VEC; ++k) s.v[k] = scale * acc[g][k];
      if (add) {
        const Sum old = *reinterpret_cast<const Sum*>(to + c[g]);
#pragma unroll
        for (int k = 0; k < VEC; ++k) s.v[k] += old.v[k];
      }
      *reinterpret_cast<Sum*>(to + c[g]) = s;
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[g][k] = 0.0f;
  }
}

template <typename T, int VEC, int G>
__global__ __launch_bounds__(256) void dlvm_embedding_pieces_kernel(
    int32_t V, int64_t E, int P, int pieces, int slabs, int sum_blocks, int32_t total,
    const int32_t* __restrict__ stok, const int32_t* __restrict__ sid, const T* __restrict__ dout,
    float scale, bool accumulate, float* __restrict__ head, float* __restrict__ tail,
    float* __restrict__ dtable) {
  using Vec = Elems<T, VEC>;
  constexpr int kUnroll = 8;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  if (static_cast<int>(blockIdx.x) >= sum_blocks) {
    zero_absent(V, E, total, (static_cast<int64_t>(blockIdx.x - sum_blocks) * 4 + wave) * 64, sid, dtable);
    return;
  }
  const int task = static_cast<int>(blockIdx.x) * 4 + wave;
  const int piece = task / slabs;
  if (piece >= pieces) return;
  const int32_t p0 = piece * P;
  const int n = total - p0 < P ? total - p0 : P;
  const int32_t tok = lane < n ? stok[p0 + lane] : 0;
  const int32_t id = lane < n ? sid[p0 + lane] : -1;
  const int32_t before = p0 > 0 ? sid[p0 - 1] : -1;
  const int32_t after = p0 + n < total ? sid[p0 + n] : -1;
  const int64_t c0 = static_cast<int64_t>(task - piece * slabs) * (64 * VEC * G) + lane * VEC;
  bool on[G];  // E is a multiple of VEC
  int64_t c[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    on[g] = c0 + g * 64 * VEC < E;
    c[g] = on[g] ? c0 + g * 64 * VEC : 0;
  }
  float acc[G][VEC];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[g][k] = 0.0f;
  int32_t cur = __builtin_amdgcn_readlane(id, 0);
  bool begins = cur != before;
  const int64_t part = static_cast<int64_t>(piece) * E;

  for (int i0 = 0; i0 < n; i0 += kUnroll) {
    Vec w[kUnroll][G];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = i0 + u < n ? i0 + u : n - 1;
      const T* row = dout + static_cast<int64_t>(__builtin_amdgcn_readlane(tok, i)) * E;
#pragma unroll
      for (int g = 0; g < G; ++g) w[u][g] = *reinterpret_cast<const Vec*>(row + c[g]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool live = i0 + u < n;
      const int32_t next = live ? __builtin_amdgcn_readlane(id, i0 + u) : cur;
      if (next != cur) {
        if (begins)  // rows come in order: not V, after which there is none
          store_row<VEC, G>(dtable + cur * E, c, on, accumulate, scale, acc);
        else
          store_row<VEC, G>(head + part, c, on, false, 1.0f, acc);
        cur = next;
        begins = true;
      }
      if (live)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int k = 0; k < VEC; ++k) acc[g][k] += load_as_f32(&w[u][g].v[k]);
    }
  }
  if (cur == V) return;
  if (begins && cur != after)
    store_row<VEC, G>(dtable + cur * E, c, on, accumulate, scale, acc);
  else
    store_row<VEC, G>((begins ? tail : head) + part, c, on, false, 1.0f, acc);
}

// ---------------------------------------------------------------------------
// Gradient, the joins: the rows that run over the end of the piece they begin in: the
// piece's tail and the heads of the following pieces up to the row's last, added in
// order. Rows of few parts take one wave to 256 columns; rows that fill at least
// kJoinLong whole pieces a workgroup, whose waves take equal ranges of the parts and
// are added in order. A workgroup of the second kind looks at one piece in kJoinLong,
// so each long row is found by the first of them that lies inside it.
// ---------------------------------------------------------------------------
constexpr int kJoinWaves = 16;
constexpr int kJoinCols = 256;
constexpr int kJoinLong = 8;

// Whether row `id` has tokens on both sides of the end of piece q, given that it has one
// in the piece or before.
__device__ __forceinline__ bool crosses(const int32_t* sid, int32_t total, int P, int64_t q, int32_t id) {
  const int64_t end = (q + 1) * P;
  return end < total && sid[end] == id;
}
// Lanes before the first that is not set.
__device__ __forceinline__ int leading_ones(uint64_t m) { return ~m == 0 ? 64 : __builtin_ctzll(~m); }
// Whether the row of a piece's last position began in an earlier piece.
__device__ __forceinline__ bool came_in(const int32_t* sid, int P, int64_t q) {
  const int64_t p0 = q * P;
  return p0 > 0 && sid[p0] == sid[p0 + P - 1] && sid[p0 - 1] == sid[p0];
}

// Sum of the parts [from, to) of the row that begins in piece p, columns c + 64 j.
__device__ __forceinline__ void add_parts(int64_t E, int64_t p, int from, int to, int64_t c,
                                          const float* __restrict__ head,
                                          const float* __restrict__ tail, float (&acc)[4]) {
  int64_t at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    at[j] = c + 64 * j < E ? c + 64 * j : 0;
    acc[j] = 0.0f;
  }
  if (from == 0 && to > 0)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = tail[p * E + at[j]];
  for (int k0 = from > 0 ? from : 1; k0 < to; k0 += 8) {
    float w[8][4];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float* src = head + (p + (k0 + u < to ? k0 + u : to - 1)) * E;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[u][j] = src[at[j]];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (k0 + u >= to) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += w[u][j];
    }
  }
}

__global__ __launch_bounds__(64 * kJoinWaves) void dlvm_embedding_join_kernel(
    int32_t V, int64_t E, int P, int pieces, int slabs, int short_blocks, int32_t total,
    const int32_t* __restrict__ sid, float scale, bool accumulate, const float* __restrict__ head,
    const float* __restrict__ tail, float* __restrict__ dtable) {
  __shared__ float part[kJoinWaves][kJoinCols];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));

  if (static_cast<int>(blockIdx.x) < short_blocks) {
    const int task = blockIdx.x * kJoinWaves + wave;
    const int p = task / slabs;
    if (p >= pieces || static_cast<int64_t>(p + 1) * P >= total) return;
    const int32_t id = sid[(p + 1) * P - 1];
    if (id == V || !crosses(sid, total, P, p, id) || came_in(sid, P, p)) return;
    // parts after the first: pieces p + 1 .. p + more, the last the one whose end it does not cross
    const bool on = lane <= kJoinLong && crosses(sid, total, P, p + 1 + lane, id);
    const int more = __builtin_ctzll(~__ballot(on)) + 1;
    if (more > kJoinLong) return;
    const int64_t c = static_cast<int64_t>(task - p * slabs) * kJoinCols + lane;
    float acc[4];
    add_parts(E, p, 0, more + 1, c, head, tail, acc);
    float* d = dtable + id * E + c;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + 64 * j < E) d[64 * j] = (accumulate ? d[64 * j] : 0.0f) + scale * acc[j];
    return;
  }

  const int task = blockIdx.x - short_blocks;
  const int64_t q = static_cast<int64_t>(task / slabs + 1) * kJoinLong - 1;
  if (q >= pieces || (q + 1) * P >= total) return;
  const int32_t id = sid[(q + 1) * P - 1];
  if (id == V || !crosses(sid, total, P, q, id)) return;
  // where the row begins: here or in one of the kJoinLong - 1 pieces before
  const bool in = lane < kJoinLong && came_in(sid, P, q - lane);
  const int back = __builtin_ctzll(~__ballot(in));
  if (back >= kJoinLong) return;  // found by an earlier workgroup
  const int64_t p = q - back;
  // the first end that the row does not cross, by 64 pieces, then one by one
  int more = 1;
  for (int far = 64; far == 64; more += 64 * far)
    far = leading_ones(__ballot(crosses(sid, total, P, p + more + 64 * lane + 63, id)));
  more += leading_ones(__ballot(crosses(sid, total, P, p + more + lane, id)));
  if (more <= kJoinLong) return;
  const int parts = more + 1, each = (parts + kJoinWaves - 1) / kJoinWaves;
  const int from = wave * each, to = from + each < parts ? from + each : parts;
  const int64_t slab = static_cast<int64_t>(task - task / slabs * slabs) * kJoinCols;
  float acc[4];
  add_parts(E, p, from, to, slab + lane, head, tail, acc);
#pragma unroll
  for (int j = 0; j < 4; ++j) part[wave][lane + 64 * j] = acc[j];
  __syncthreads();
  const int64_t c = slab + threadIdx.x;
  if (threadIdx.x < kJoinCols && c < E) {
    float s = part[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) s += part[w][threadIdx.x];
    float* d = dtable + id * E + c;
    *d = (accumulate ? *d : 0.0f) + scale * s;
  }
}

// Positions of a piece. Long pieces store and read fewer partial sums; short ones keep
// enough waves in flight when tokens are few: 65536 tokens of 1024 columns take a join of 20 us
// in pieces of 16, 8.6 in pieces of 64; 4099 of 1001 sums of 11.7 us and 24.
int piece_len(int64_t width, int64_t tokens) {
  const int64_t waves = tokens * ((width + 511) / 512);
  return waves >= 64 * 2048 ? 64 : waves >= 32 * 2048 ? 32 : 16;
}

// Tokens of a block to a thread: a block's place in the sort waits for the counts of all
// blocks, so they grow with the tokens (us to place 20000 tokens with one, two and four: 6.8,
// 7.4 and 10.4, 65536: 10.3, 9.2 and 10.5, 200001: two 15.6, four 13.9).
int sort_width(int64_t n) { return n <= (1 << 15) ? 1 : n <= (1 << 17) ? 2 : 4; }
int sort_blocks(int64_t n) {
  const int64_t block = int64_t(kSortThreads) * sort_width(n);
  return static_cast<int>((n + block - 1) / block);
}

// Workspace of a gradient call: pairs (row, token) before and after a pass, counts, partial sums.
struct GradWs {
  size_t row[2], tok[2], counts, head, tail, total;
  int P;
  int64_t chunk, pieces;
};
GradWs grad_ws(int64_t width, int64_t tokens) {
  const auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  GradWs w;
  w.chunk = tokens < kSortTokens ? tokens : kSortTokens;
  w.P = piece_len(width, w.chunk);
  w.pieces = (w.chunk + w.P - 1) / w.P;
  const size_t list = up(static_cast<size_t>(w.chunk) * 4);
  for (int i = 0; i < 2; ++i) {
    w.row[i] = 2 * i * list;
    w.tok[i] = (2 * i + 1) * list;
  }
  w.counts = 4 * list;
  w.head = w.counts + static_cast<size_t>(sort_blocks(w.chunk)) * kDigits * 4;
  w.tail = w.head + up(static_cast<size_t>(w.pieces) * width * 4);
  w.total = w.tail + up(static_cast<size_t>(w.pieces) * width * 4);
  return w;
}

// The call's n tokens sorted by row; returns which of the two lists holds them. If the table is
// to be zeroed (`zero`), its launches may do that, and then say so.
int sort_tokens(const GradWs& w, int32_t V, int64_t E, int32_t n, const int32_t* ids, char* ws, bool& zero,
                float* dtable, hipStream_t s) {
  const auto list = [&](size_t at) { return reinterpret_cast<int32_t*>(ws + at); };
  int bits = 1;  // of the largest key, V
  while ((V >> bits) != 0) ++bits;
  const int passes = (bits + kDigitBits - 1) / kDigitBits, digit_bits = (bits + passes - 1) / passes;
  if (n <= kSmallSort) {
    const int blocks = (n + 63) / 64;
    const int64_t others = zero ? (V * E + 4 * kZeroQuads - 1) / (4 * kZeroQuads) : 0;
    launch_kernel(dlvm_embedding_sort_kernel, dim3(static_cast<uint32_t>(blocks + others)), dim3(kSortThreads),
                  s, V, E, n, blocks, ids, list(w.row[0]), list(w.tok[0]), dtable);
    zero = false;
    return 0;
  }
  // a table that is not too large is filled beside the sort, an equal part by each launch
  const int blocks = sort_blocks(n);
  const int64_t all = zero && V * E <= kFillBeside ? V * E : 0;
  const int64_t each = ((all + 2 * passes - 1) / (2 * passes) + 3) / 4 * 4;
  const dim3 grid(static_cast<uint32_t>(blocks + (each + 4 * kZeroQuads - 1) / (4 * kZeroQuads)));
  if (all > 0) zero = false;
  int64_t done = 0;
  const auto with_zeros = [&](SortIn in) {
    in.blocks = blocks;
    in.zero = dtable + done;
    in.zeros = std::min(all - done, each);
    done += in.zeros;
    return in;
  };
  const int width = sort_width(n);
  const auto count = width == 1   ? dlvm_embedding_count_kernel<1>
                     : width == 2 ? dlvm_embedding_count_kernel<2> : dlvm_embedding_count_kernel<4>;
  const auto place = width == 1   ? dlvm_embedding_place_kernel<1>
                     : width == 2 ? dlvm_embedding_place_kernel<2> : dlvm_embedding_place_kernel<4>;
  int to = 0;
  for (int shift = 0; shift < bits; shift += digit_bits, to ^= 1) {
    const SortIn in = shift == 0 ? SortIn{ids, nullptr, nullptr}
                                 : SortIn{nullptr, list(w.row[to ^ 1]), list(w.tok[to ^ 1])};
    launch_kernel(count, grid, dim3(kSortThreads), s, V, n, shift, digit_bits, with_zeros(in), list(w.counts));
    launch_kernel(place, grid, dim3(kSortThreads), s, V, n, shift, digit_bits, with_zeros(in),
                  static_cast<const int32_t*>(list(w.counts)), list(w.row[to]), list(w.tok[to]));
  }
  return to ^ 1;
}

template <typename T, int VEC>
void lookup(int64_t V, int64_t E, int64_t N, const void* table, const int32_t* ids, float scale,
            void* out, hipStream_t s) {
  const int64_t chunks = (E + VEC - 1) / VEC;
  const int64_t step = (int64_t(1) << 30) / chunks / 4 * 4;  // tokens of one launch (ids stay aligned)
  for (int64_t i0 = 0; i0 < N; i0 += step) {
    const int64_t n = N - i0 < step ? N - i0 : step, total = n * chunks;
    // every compute unit has eight workgroups before a thread takes a second vector; 65536
    // rows of 1024 bf16 take 51 us with four to a thread, 75 with one
    int64_t blocks = (total + 255) / 256;
    if (blocks > 2048) blocks = (blocks + kLookupUnroll - 1) / kLookupUnroll;
    launch_kernel(dlvm_embedding_kernel<T, VEC>, dim3(static_cast<uint32_t>(blocks)), dim3(256), s,
                  static_cast<uint32_t>(V), E, static_cast<uint32_t>(chunks),
                  divisor(static_cast<uint32_t>(chunks)), static_cast<uint32_t>(total),
                  static_cast<const T*>(table), ids + i0, scale, static_cast<T*>(out) + i0 * E);
  }
}

// One chunk of tokens, sorted.
struct Chunk {
  int32_t V;
  int64_t E;
  int32_t n;
  const int32_t *row, *tok;
  float scale;
  bool add, zero;  // added to the table; whether rows without a token are still to be zeroed
  float *head, *tail, *dtable;
  int P;
};

template <typename T, int VEC, int G>
void sum_pieces(const Chunk& c, const T* dout, hipStream_t s) {
  const int64_t pieces = (c.n + c.P - 1) / c.P, slabs = (c.E + 64 * VEC * G - 1) / (64 * VEC * G);
  const int64_t sum_blocks = (pieces * slabs + 3) / 4, zero_blocks = c.zero ? (c.V + 255) / 256 : 0;
  launch_kernel(dlvm_embedding_pieces_kernel<T, VEC, G>, dim3(static_cast<uint32_t>(sum_blocks + zero_blocks)),
                dim3(256), s, c.V, c.E, c.P, static_cast<int>(pieces), static_cast<int>(slabs),
                static_cast<int>(sum_blocks), c.n, c.tok, c.row, dout, c.scale, c.add, c.head, c.tail, c.dtable);
}

// The widest vector that divides the row, and as many to a lane as leave none idle (160
// columns: 20.6 us with vectors of two in two slabs, 22.0 with vectors of four on 40 lanes).
template <typename T> void sum_pieces_any(const Chunk& c, const T* dout, hipStream_t s) {
  const int64_t E = c.E;
  auto f = E % 4 == 0 && E >= 512 ? sum_pieces<T, 4, 2>
           : E % 4 == 0 && E >= 256 ? sum_pieces<T, 4, 1>
           : E % 2 == 0 && E >= 256 ? sum_pieces<T, 2, 2>
           : E % 2 == 0 && E >= 128 ? sum_pieces<T, 2, 1>
           : E >= 256 ? sum_pieces<T, 1, 4> : sum_pieces<T, 1, 1>;
  f(c, dout, s);
}

}  // namespace

hipError_t launch_embedding_forward(int dtype, int64_t vocab, int64_t width, int64_t tokens,
                                    const void* table, const int32_t* ids, float scale, void* out,
                                    hipStream_t s) {
  if (dtype == F32)
    (width >= 4 ? lookup<float, 4> : lookup<float, 1>)(vocab, width, tokens, table, ids, scale, out, s);
  else
    (width >= 8 ? lookup<bf16_t, 8> : lookup<bf16_t, 1>)(vocab, width, tokens, table, ids, scale, out, s);
  return hipGetLastError();
}

size_t embedding_backward_ws(int64_t, int64_t width, int64_t tokens) {
  return grad_ws(width, tokens).total;
}

hipError_t launch_embedding_backward(int dtype, int64_t vocab, int64_t width, int64_t tokens,
                                     const int32_t* ids, const void* dout, float scale,
                                     bool accumulate, float* dtable, void* ws, hipStream_t s) {
  const GradWs w = grad_ws(width, tokens);
  char* base = static_cast<char*>(ws);
  const auto list = [&](size_t at) { return reinterpret_cast<int32_t*>(base + at); };
  const int32_t V = static_cast<int32_t>(vocab);
  // more tokens than one sort takes: the following ones are added to the table
  for (int64_t t0 = 0; t0 < tokens; t0 += w.chunk) {
    const int32_t n = static_cast<int32_t>(tokens - t0 < w.chunk ? tokens - t0 : w.chunk);
    const bool add = accumulate || t0 > 0;
    bool zero = !add;
    const int at = sort_tokens(w, V, width, n, ids + t0, base, zero, dtable, s);
    const Chunk c{V, width, n, list(w.row[at]), list(w.tok[at]), scale, add, zero,
                  reinterpret_cast<float*>(base + w.head), reinterpret_cast<float*>(base + w.tail), dtable, w.P};
    if (dtype == F32)
      sum_pieces_any<float>(c, static_cast<const float*>(dout) + t0 * width, s);
    else
      sum_pieces_any<bf16_t>(c, static_cast<const bf16_t*>(dout) + t0 * width, s);
    const int pieces = (n + c.P - 1) / c.P;
    const int slabs = static_cast<int>((width + kJoinCols - 1) / kJoinCols);
    const int short_blocks = (pieces * slabs + kJoinWaves - 1) / kJoinWaves;
    if (pieces == 1) continue;  // nothing runs over its end
    launch_kernel(dlvm_embedding_join_kernel, dim3(short_blocks + pieces / kJoinLong * slabs),
                  dim3(64 * kJoinWaves), s, V, width, c.P, pieces, slabs, short_blocks, n, c.row, scale, c.add,
                  static_cast<const float*>(c.head), static_cast<const float*>(c.tail), dtable);
  }
  return hipGetLastError();
}

}  // namespace dlvm

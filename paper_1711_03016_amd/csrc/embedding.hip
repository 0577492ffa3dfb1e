// Token embeddings: the lookup with scaling, and the gradient of the table by
// sorted tokens.
//
// The gradient, dtable[v] = scale * sum of dout[i] over the tokens i with id v, runs in
// three launches and no floating-point atomics: tokens are grouped by id in their
// order (and the rows without a token are zeroed by the same launch, which is most of
// the bytes of a large table), equal pieces of the grouped list are summed, and the
// sums of rows that run over a piece's end are joined in the order of the pieces.
#include <math.h>

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
// Gradient, launch 1: tokens grouped by id. Every workgroup reads all ids (a few
// hundred KB, from the L2) and takes those whose low bits are its number, so frequent
// ids, which are neighbours in most vocabularies, fall to different workgroups. The
// ids of lower-numbered groups, counted on the way, are where its list starts: no
// launch has to scan counts. Each of its waves owns a contiguous range of tokens, a row
// of counters and a list in LDS of the tokens it took, so that they are placed in one
// order (ranges ascending; within 256 tokens every fourth one, from each of the first
// four) without any order between waves; a wave whose list is full (one id
// is a tenth of many tokens) reads its range again instead. What a vector of 64 ids
// costs in the reading is what bounds it, 256 times over: three comparisons with scalar
// counts of their masks, and a branch. The rows that have
// no token are zeroed before the tokens are placed.
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortRows = 512;                       // rows of one group at most
constexpr int kSortMinGroups = 256;                  // a workgroup on every compute unit
constexpr int64_t kSortTokens = int64_t(1) << 18;    // tokens of one sorting launch
constexpr int kSortUnroll = 8;
constexpr int kSortList = 1536;                      // tokens of a wave's list
constexpr int kSortRowBits = 9;                      // 2^9 = kSortRows; the rest: token in the wave's range
static_assert((1 << kSortRowBits) == kSortRows && kSortTokens / kSortWaves <= (1 << (32 - kSortRowBits)), "");

// Set bits below the lane's.
__device__ __forceinline__ int bits_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32),
                                   __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0));
}

// Places of the tokens of one vector in a wave's part of the grouped list: `row` of the
// lane's token (-1: none), one row of the vector at a time; `next` the wave's counters, of
// which that of the row last placed is kept in `hot` and `at_hot` (a frequent id is
// placed vector after vector without waiting for LDS).
__device__ __forceinline__ void place_tokens(int row, int32_t tok, int32_t id, volatile int32_t* next,
                                             int& hot, int32_t& at_hot, int32_t* __restrict__ stok,
                                             int32_t* __restrict__ sid) {
  uint64_t todo = __ballot(row >= 0);
  while (todo != 0) {
    const int one = __builtin_amdgcn_readlane(row, __builtin_ctzll(todo));
    const uint64_t same = __ballot(row == one);
    if (one != hot) {
      if (hot >= 0) next[hot] = at_hot;
      hot = one;
      at_hot = __builtin_amdgcn_readfirstlane(next[one]);
    }
    if (row == one) {
      const int32_t at = at_hot + bits_below(same);
      stok[at] = tok;
      sid[at] = id;
    }
    at_hot += __builtin_popcountll(same);
    todo &= ~same;
  }
}

// Four consecutive ids of a lane from token i on, -1 behind `end` (ids start on 16 bytes,
// i is a multiple of 4).
__device__ __forceinline__ int4 load_ids(const int32_t* __restrict__ ids, int32_t i, int32_t end) {
  int4 v = make_int4(-1, -1, -1, -1);
  if (i + 4 <= end) {
    v = *reinterpret_cast<const int4*>(ids + i);
  } else if (i < end) {
    v.x = ids[i];
    if (i + 1 < end) v.y = ids[i + 1];
    if (i + 2 < end) v.z = ids[i + 2];
  }
  return v;
}

template <bool ZERO>
__global__ __launch_bounds__(kSortThreads) void dlvm_embedding_group_kernel(
    uint32_t V, int64_t E, int32_t N, int log_groups, const int32_t* __restrict__ ids,
    int32_t* __restrict__ count, int32_t* __restrict__ stok, int32_t* __restrict__ sid,
    float* __restrict__ dtable) {
  __shared__ int32_t hist[kSortWaves][kSortRows];
  __shared__ uint32_t list[kSortWaves][kSortList];
  __shared__ int32_t lower[kSortWaves];
  __shared__ int32_t sums[kSortRows / 64];
  __shared__ uint8_t used[kSortRows];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t me = blockIdx.x, mask = (1u << log_groups) - 1;
  const int R = static_cast<int>((V + mask) >> log_groups);
  for (int w = 0; w < kSortWaves; ++w)
    if (tid < R) hist[w][tid] = 0;
  __syncthreads();

  const int32_t span = (N + 4 * kSortThreads - 1) / (4 * kSortThreads) * 256;  // tokens of a wave
  const int32_t first = wave * span;
  const int32_t end = first + span < N ? first + span : N;
  int32_t below = 0, taken = 0;  // of this wave
  for (int32_t i0 = first; i0 < end; i0 += 256 * kSortUnroll) {
    int4 id[kSortUnroll];
#pragma unroll
    for (int u = 0; u < kSortUnroll; ++u) id[u] = load_ids(ids, i0 + 256 * u + 4 * lane, end);
#pragma unroll
    for (int u = 0; u < kSortUnroll; ++u) {
      const uint32_t v[4] = {static_cast<uint32_t>(id[u].x), static_cast<uint32_t>(id[u].y),
                             static_cast<uint32_t>(id[u].z), static_cast<uint32_t>(id[u].w)};
      bool hit[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool valid = v[j] < V;
        hit[j] = valid && (v[j] & mask) == me;
        below += __builtin_popcountll(__ballot(valid && (v[j] & mask) < me));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t match = __ballot(hit[j]);
        if (match == 0) continue;
        const int32_t at = taken + bits_below(match);
        if (hit[j] && at < kSortList)
          list[wave][at] = static_cast<uint32_t>(i0 - first + 256 * u + 4 * lane + j) << kSortRowBits |
                           v[j] >> log_groups;
        taken += __builtin_popcountll(match);
      }
    }
  }
  if (lane == 0) lower[wave] = below;
  if (taken <= kSortList) {
    for (int j = lane; j < taken; j += 64) atomicAdd(&hist[wave][list[wave][j] & (kSortRows - 1)], 1);
  } else {
    for (int32_t i = first + lane; i < end; i += 64) {
      const uint32_t v = static_cast<uint32_t>(ids[i]);
      if (v < V && (v & mask) == me) atomicAdd(&hist[wave][v >> log_groups], 1);
    }
  }
  __syncthreads();

  // counts to places: exclusive sums over the rows, and within a row over the waves
  int32_t mine = 0, incl = 0;
  if (tid < kSortRows) {
    if (tid < R)
      for (int w = 0; w < kSortWaves; ++w) mine += hist[w][tid];
    used[tid] = mine != 0;
    incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int32_t up = __shfl_up(incl, o, 64);
      if (lane >= o) incl += up;
    }
    if (lane == 63) sums[wave] = incl;
  }
  __syncthreads();
  if (tid < kSortRows) {
    int32_t at = incl - mine;
    for (int w = 0; w < kSortWaves; ++w) at += lower[w];
    for (int w = 0; w < wave; ++w) at += sums[w];
    if (tid == kSortRows - 1 && me == mask) *count = at + mine;
    if (tid < R)
      for (int w = 0; w < kSortWaves; ++w) {
        const int32_t n = hist[w][tid];
        hist[w][tid] = at;
        at += n;
      }
  }
  __syncthreads();

  if (ZERO) {
    using Vec = Elems<float, 4>;
    const Vec zero{{0.0f, 0.0f, 0.0f, 0.0f}};
    for (int r = wave; r < R; r += kSortWaves) {
      const uint32_t v = (static_cast<uint32_t>(r) << log_groups) + me;
      if (used[r] || v >= V) continue;
      float* row = dtable + v * E;
      int64_t c = 4 * lane;
      for (; c + 4 <= E; c += 256) *reinterpret_cast<Vec*>(row + c) = zero;
      for (; c < E; ++c) row[c] = 0.0f;
    }
  }

  volatile int32_t* next = hist[wave];
  int hot = -1;
  int32_t at_hot = 0;
  if (taken <= kSortList) {
    for (int j = 0; j < taken; j += 64) {
      const uint32_t e = j + lane < taken ? list[wave][j + lane] : 0;
      const int row = j + lane < taken ? static_cast<int>(e & (kSortRows - 1)) : -1;
      place_tokens(row, first + static_cast<int32_t>(e >> kSortRowBits),
                   static_cast<int32_t>((e & (kSortRows - 1)) << log_groups | me), next, hot, at_hot,
                   stok, sid);
    }
    return;
  }
  for (int32_t i0 = first; i0 < end; i0 += 256) {
    const int4 id = load_ids(ids, i0 + 4 * lane, end);
    const int32_t v[4] = {id.x, id.y, id.z, id.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u = static_cast<uint32_t>(v[j]);
      const int row = u < V && (u & mask) == me ? static_cast<int>(u >> log_groups) : -1;
      place_tokens(row, i0 + 4 * lane + j, v[j], next, hot, at_hot, stok, sid);
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient, launch 2: a wave sums one piece of the grouped list over a slab of
// 64 * VEC * G columns (G vectors a lane, each contiguous over the wave), eight rows in
// flight. Rows that begin and end inside a piece are written; what belongs to a row that
// began in an earlier piece goes to `head`, the start of one that goes on in the next
// piece to `tail` (float32, without the scale).
// ---------------------------------------------------------------------------
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
    int64_t E, int P, int pieces, int slabs, const int32_t* __restrict__ count,
    const int32_t* __restrict__ stok, const int32_t* __restrict__ sid, const T* __restrict__ dout,
    float scale, bool accumulate, float* __restrict__ head, float* __restrict__ tail,
    float* __restrict__ dtable) {
  using Vec = Elems<T, VEC>;
  constexpr int kUnroll = 8;
  const int lane = threadIdx.x & 63;
  const int task = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int piece = task / slabs;
  if (piece >= pieces) return;
  const int32_t total = *count;
  const int32_t p0 = piece * P;
  if (p0 >= total) return;
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
        if (begins)
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
  if (begins && cur != after)
    store_row<VEC, G>(dtable + cur * E, c, on, accumulate, scale, acc);
  else
    store_row<VEC, G>((begins ? tail : head) + part, c, on, false, 1.0f, acc);
}

// ---------------------------------------------------------------------------
// Gradient, launch 3: the rows that run over the end of the piece they begin in: the
// piece's tail and the heads of the following pieces up to the row's last, added in
// order. Rows of few parts take one wave to 256 columns; rows that fill at least
// kJoinLong whole pieces a workgroup, whose waves take equal ranges of the parts and
// are added in order. A workgroup of the second kind looks at one piece in kJoinLong,
// so each long row is found by the first of them that lies inside it.
// ---------------------------------------------------------------------------
constexpr int kJoinWaves = 8;
constexpr int kJoinCols = 256;
constexpr int kJoinLong = 8;

// Whether row `id` has tokens on both sides of the end of piece q, given that it has one
// in the piece or before.
__device__ __forceinline__ bool crosses(const int32_t* sid, int32_t total, int P, int64_t q, int32_t id) {
  const int64_t end = (q + 1) * P;
  return end < total && sid[end] == id;
}
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
    int64_t E, int P, int pieces, int slabs, int short_blocks, const int32_t* __restrict__ count,
    const int32_t* __restrict__ sid, float scale, bool accumulate, const float* __restrict__ head,
    const float* __restrict__ tail, float* __restrict__ dtable) {
  __shared__ float part[kJoinWaves][kJoinCols];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const int32_t total = *count;

  if (static_cast<int>(blockIdx.x) < short_blocks) {
    const int task = blockIdx.x * kJoinWaves + wave;
    const int p = task / slabs;
    if (p >= pieces || static_cast<int64_t>(p + 1) * P >= total) return;
    const int32_t id = sid[(p + 1) * P - 1];
    if (!crosses(sid, total, P, p, id) || came_in(sid, P, p)) return;
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
  if (!crosses(sid, total, P, q, id)) return;
  // where the row begins: here or in one of the kJoinLong - 1 pieces before
  const bool in = lane < kJoinLong && came_in(sid, P, q - lane);
  const int back = __builtin_ctzll(~__ballot(in));
  if (back >= kJoinLong) return;  // found by an earlier workgroup
  const int64_t p = q - back;
  int more = 1;
  for (;;) {
    const uint64_t stop = ~__ballot(crosses(sid, total, P, p + more + lane, id));
    if (stop != 0) {
      more += __builtin_ctzll(stop);
      break;
    }
    more += 64;
  }
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
// enough waves in flight when tokens are few.
int piece_len(int64_t width, int64_t tokens) {
  const int64_t waves = tokens * ((width + 511) / 512);
  return waves >= 64 * 2048 ? 64 : waves >= 32 * 2048 ? 32 : 16;
}

struct GradWs {
  size_t count, stok, sid, head, tail, total;
  int P;
  int64_t chunk, pieces;
};
GradWs grad_ws(int64_t width, int64_t tokens) {
  const auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  GradWs w;
  w.chunk = tokens < kSortTokens ? tokens : kSortTokens;
  w.P = piece_len(width, w.chunk);
  w.pieces = (w.chunk + w.P - 1) / w.P;
  w.count = 0;
  w.stok = 256;
  w.sid = w.stok + up(static_cast<size_t>(w.chunk) * 4);
  w.head = w.sid + up(static_cast<size_t>(w.chunk) * 4);
  w.tail = w.head + up(static_cast<size_t>(w.pieces) * width * 4);
  w.total = w.tail + up(static_cast<size_t>(w.pieces) * width * 4);
  return w;
}

template <typename T, int VEC>
void lookup(int64_t V, int64_t E, int64_t N, const void* table, const int32_t* ids, float scale,
            void* out, hipStream_t s) {
  const int64_t chunks = (E + VEC - 1) / VEC;
  const int64_t step = (int64_t(1) << 30) / chunks / 4 * 4;  // tokens of one launch (ids stay aligned)
  for (int64_t i0 = 0; i0 < N; i0 += step) {
    const int64_t n = N - i0 < step ? N - i0 : step, total = n * chunks;
    // every compute unit has eight workgroups before a thread takes a second vector
    int64_t blocks = (total + 255) / 256;
    if (blocks > 2048) blocks = (blocks + kLookupUnroll - 1) / kLookupUnroll;
    launch_kernel(dlvm_embedding_kernel<T, VEC>, dim3(static_cast<uint32_t>(blocks)), dim3(256), s,
                  static_cast<uint32_t>(V), E, static_cast<uint32_t>(chunks),
                  divisor(static_cast<uint32_t>(chunks)), static_cast<uint32_t>(total),
                  static_cast<const T*>(table), ids + i0, scale, static_cast<T*>(out) + i0 * E);
  }
}

template <typename T, int VEC, int G>
void sum_pieces(const GradWs& w, int64_t E, int64_t n, char* ws, const T* dout, float scale,
                bool accumulate, float* dtable, hipStream_t s) {
  const int64_t pieces = (n + w.P - 1) / w.P, slabs = (E + 64 * VEC * G - 1) / (64 * VEC * G);
  launch_kernel(dlvm_embedding_pieces_kernel<T, VEC, G>, dim3(static_cast<uint32_t>((pieces * slabs + 3) / 4)),
                dim3(256), s, E, w.P, static_cast<int>(pieces), static_cast<int>(slabs),
                reinterpret_cast<const int32_t*>(ws + w.count), reinterpret_cast<const int32_t*>(ws + w.stok),
                reinterpret_cast<const int32_t*>(ws + w.sid), dout, scale, accumulate,
                reinterpret_cast<float*>(ws + w.head), reinterpret_cast<float*>(ws + w.tail), dtable);
}

// The widest vector that divides the row, and as many to a lane as leave none idle.
template <typename T>
void sum_pieces_any(const GradWs& w, int64_t E, int64_t n, char* ws, const T* dout, float scale,
                    bool accumulate, float* dtable, hipStream_t s) {
  auto f = E % 4 == 0 && E >= 512 ? sum_pieces<T, 4, 2>
           : E % 4 == 0 && E >= 256 ? sum_pieces<T, 4, 1>
           : E % 2 == 0 && E >= 256 ? sum_pieces<T, 2, 2>
           : E % 2 == 0 && E >= 128 ? sum_pieces<T, 2, 1>
           : E >= 256 ? sum_pieces<T, 1, 4> : sum_pieces<T, 1, 1>;
  f(w, E, n, ws, dout, scale, accumulate, dtable, s);
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
  int32_t* count = reinterpret_cast<int32_t*>(base + w.count);
  int32_t* stok = reinterpret_cast<int32_t*>(base + w.stok);
  int32_t* sid = reinterpret_cast<int32_t*>(base + w.sid);
  int log_groups = 0;
  while ((1 << log_groups) < kSortMinGroups || ((vocab - 1) >> log_groups) + 1 > kSortRows) ++log_groups;
  // more tokens than one sort takes: the following ones are added to the table
  for (int64_t t0 = 0; t0 < tokens; t0 += w.chunk) {
    const int64_t n = tokens - t0 < w.chunk ? tokens - t0 : w.chunk;
    const bool add = accumulate || t0 > 0;
    launch_kernel(add ? dlvm_embedding_group_kernel<false> : dlvm_embedding_group_kernel<true>,
                  dim3(1u << log_groups), dim3(kSortThreads), s, static_cast<uint32_t>(vocab), width,
                  static_cast<int32_t>(n), log_groups, ids + t0, count, stok, sid, dtable);
    if (dtype == F32)
      sum_pieces_any<float>(w, width, n, base, static_cast<const float*>(dout) + t0 * width, scale, add,
                            dtable, s);
    else
      sum_pieces_any<bf16_t>(w, width, n, base, static_cast<const bf16_t*>(dout) + t0 * width, scale, add,
                             dtable, s);
    const int pieces = static_cast<int>((n + w.P - 1) / w.P);
    const int slabs = static_cast<int>((width + kJoinCols - 1) / kJoinCols);
    const int short_blocks = (pieces * slabs + kJoinWaves - 1) / kJoinWaves;
    launch_kernel(dlvm_embedding_join_kernel, dim3(short_blocks + pieces / kJoinLong * slabs),
                  dim3(64 * kJoinWaves), s, width, w.P, pieces, slabs, short_blocks, count, sid, scale,
                  add, reinterpret_cast<const float*>(base + w.head),
                  reinterpret_cast<const float*>(base + w.tail), dtable);
  }
  return hipGetLastError();
}

}  // namespace dlvm

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

template <typename T, int VEC>
__global__ __launch_bounds__(256) void dlvm_embedding_kernel(uint32_t V, int64_t E, uint32_t chunks,
                                                             int64_t total,
                                                             const T* __restrict__ table,
                                                             const int32_t* __restrict__ ids,
                                                             float scale, T* __restrict__ out) {
  using Vec = Elems<T, VEC>;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
  int64_t q = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  for (; q < total; q += kLookupUnroll * stride) {
    int32_t id[kLookupUnroll];
    int64_t to[kLookupUnroll], from[kLookupUnroll];
    Vec w[kLookupUnroll];
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
      const int64_t p = q + u * stride;
      const int64_t i = (p < total ? p : q) / chunks;
      int64_t c = ((p < total ? p : q) - i * chunks) * VEC;
      if (c + VEC > E) c = E - VEC;
      id[u] = ids[i];
      from[u] = (static_cast<uint32_t>(id[u]) < V ? id[u] : 0) * E + c;
      to[u] = i * E + c;
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) w[u] = *reinterpret_cast<const Vec*>(table + from[u]);
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
// launch has to scan counts. Each of its waves owns a contiguous range of tokens and
// a row of counters, so the second reading places the tokens of one id in ascending
// order without any order between waves. The rows that have no token are zeroed between
// the two readings, whose latency the stores hide.
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortRows = 512;                       // rows of one group at most
constexpr int kSortMinGroups = 512;                  // two workgroups on every compute unit
constexpr int64_t kSortTokens = int64_t(1) << 18;    // tokens of one sorting launch
constexpr int kSortUnroll = 8;

template <bool ZERO>
__global__ __launch_bounds__(kSortThreads) void dlvm_embedding_group_kernel(
    uint32_t V, int64_t E, int32_t N, int log_groups, const int32_t* __restrict__ ids,
    int32_t* __restrict__ count, int32_t* __restrict__ stok, int32_t* __restrict__ sid,
    float* __restrict__ dtable) {
  __shared__ int32_t hist[kSortWaves][kSortRows];
  __shared__ int32_t lower[kSortWaves];
  __shared__ int32_t sums[kSortRows / 64];
  __shared__ uint8_t used[kSortRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t me = blockIdx.x, mask = (1u << log_groups) - 1;
  const int R = static_cast<int>((V + mask) >> log_groups);
  for (int j = tid; j < kSortWaves * R; j += kSortThreads) hist[j / R][j % R] = 0;
  __syncthreads();

  const int32_t span = (N + kSortThreads - 1) / kSortThreads * 64;  // tokens of a wave
  const int32_t first = wave * span;
  const int32_t end = first + span < N ? first + span : N;
  int32_t below = 0;
  for (int32_t i0 = first; i0 < end; i0 += 64 * kSortUnroll) {
    int32_t id[kSortUnroll];
#pragma unroll
    for (int u = 0; u < kSortUnroll; ++u) {
      const int32_t i = i0 + 64 * u + lane;
      id[u] = i < end ? ids[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < kSortUnroll; ++u) {
      const uint32_t v = static_cast<uint32_t>(id[u]);
      if (v < V) {
        below += (v & mask) < me;
        if ((v & mask) == me) atomicAdd(&hist[wave][v >> log_groups], 1);
      }
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) below += __shfl_xor(below, o, 64);
  if (lane == 0) lower[wave] = below;
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

  volatile int32_t* place = hist[wave];
  for (int32_t i0 = first; i0 < end; i0 += 64 * kSortUnroll) {
    int32_t id[kSortUnroll];
#pragma unroll
    for (int u = 0; u < kSortUnroll; ++u) {
      const int32_t i = i0 + 64 * u + lane;
      id[u] = i < end ? ids[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < kSortUnroll; ++u) {
      const uint32_t v = static_cast<uint32_t>(id[u]);
      uint64_t todo = __ballot(v < V && (v & mask) == me);
      while (todo != 0) {                             // one id of these 64 tokens at a time
        const int32_t one = __builtin_amdgcn_readlane(id[u], __builtin_ctzll(todo));
        const uint64_t same = __ballot(id[u] == one);
        const int32_t base = place[one >> log_groups];
        if (id[u] == one) {
          const int32_t at = base + __builtin_amdgcn_mbcnt_hi(
                                        static_cast<uint32_t>(same >> 32),
                                        __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(same), 0));
          stok[at] = i0 + 64 * u + lane;
          sid[at] = one;
        }
        if (lane == 0) place[one >> log_groups] = base + __builtin_popcountll(same);
        todo &= ~same;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient, launch 2: a wave sums one piece of the grouped list over 64 * VEC
// columns, eight rows in flight. Rows that begin and end inside a piece are written;
// what belongs to a row that began in an earlier piece goes to `head`, the start of one
// that goes on in the next piece to `tail` (float32, without the scale).
// ---------------------------------------------------------------------------
template <typename T, int VEC>
__global__ __launch_bounds__(256) void dlvm_embedding_pieces_kernel(
    int64_t E, int P, int pieces, int slabs, const int32_t* __restrict__ count,
    const int32_t* __restrict__ stok, const int32_t* __restrict__ sid, const T* __restrict__ dout,
    float scale, bool accumulate, float* __restrict__ head, float* __restrict__ tail,
    float* __restrict__ dtable) {
  using Vec = Elems<T, VEC>;
  using Sum = Elems<float, VEC>;
  constexpr int kUnroll = 8;
  const int lane = threadIdx.x & 63;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int piece = __builtin_amdgcn_readfirstlane(static_cast<int>(task / slabs));
  if (piece >= pieces) return;
  const int32_t total = *count;
  const int32_t p0 = piece * P;
  if (p0 >= total) return;
  const int n = total - p0 < P ? total - p0 : P;
  const int64_t c = ((task - static_cast<int64_t>(piece) * slabs) * 64 + lane) * VEC;
  const bool on = c < E;  // E is a multiple of VEC
  const int32_t tok = lane < n ? stok[p0 + lane] : 0;
  const int32_t id = lane < n ? sid[p0 + lane] : -1;
  const int32_t before = p0 > 0 ? sid[p0 - 1] : -1;
  const int32_t after = p0 + n < total ? sid[p0 + n] : -1;
  float acc[VEC] = {};
  int32_t cur = __builtin_amdgcn_readlane(id, 0);
  bool begins = cur != before;

  const auto flush = [&](bool ends) {
    if (on) {
      Sum s;
#pragma unroll
      for (int k = 0; k < VEC; ++k) s.v[k] = acc[k];
      if (begins && ends) {
        Sum* d = reinterpret_cast<Sum*>(dtable + cur * E + c);
#pragma unroll
        for (int k = 0; k < VEC; ++k) s.v[k] *= scale;
        if (accumulate) {
          const Sum old = *d;
#pragma unroll
          for (int k = 0; k < VEC; ++k) s.v[k] += old.v[k];
        }
        *d = s;
      } else {
        *reinterpret_cast<Sum*>((begins ? tail : head) + static_cast<int64_t>(piece) * E + c) = s;
      }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
  };

  for (int i0 = 0; i0 < n; i0 += kUnroll) {
    Vec w[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = i0 + u < n ? i0 + u : n - 1;
      const int64_t t = __builtin_amdgcn_readlane(tok, i);
      w[u] = *reinterpret_cast<const Vec*>(dout + t * E + (on ? c : 0));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (i0 + u >= n) break;
      const int32_t next = __builtin_amdgcn_readlane(id, i0 + u);
      if (next != cur) {
        flush(true);
        cur = next;
        begins = true;
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) acc[k] += load_as_f32(&w[u].v[k]);
    }
  }
  flush(cur != after);
}

// Gradient, launch 3: the rows that run over the end of the piece they begin in. Their
// parts, the piece's tail and the heads of the following pieces, are shared out over the
// eight waves of a workgroup in order, and the waves' sums added in order.
constexpr int kJoinWaves = 8;
constexpr int kJoinCols = 256;

__global__ __launch_bounds__(64 * kJoinWaves) void dlvm_embedding_join_kernel(
    int64_t E, int P, int pieces, const int32_t* __restrict__ count, const int32_t* __restrict__ sid,
    float scale, bool accumulate, const float* __restrict__ head, const float* __restrict__ tail,
    float* __restrict__ dtable) {
  __shared__ float part[kJoinWaves][kJoinCols];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int p = blockIdx.x;
  const int32_t total = *count;
  const int64_t end = static_cast<int64_t>(p + 1) * P;
  if (end >= total) return;
  const int32_t id = sid[end - 1];
  if (sid[end] != id) return;                                    // ends with the piece
  if (p > 0 && sid[end - P] == id && sid[end - P - 1] == id) return;  // began before it
  // the last piece that holds a part of the row
  int last = p + 1;
  for (;;) {
    const int64_t q = last + lane;                               // does the row run over q's end?
    const bool on = (q + 1) * P < total && sid[(q + 1) * P] == id;
    const uint64_t stop = ~__ballot(on);
    if (stop != 0) {
      last += __builtin_ctzll(stop);
      break;
    }
    last += 64;
  }
  const int parts = last - p + 1;                                // tail[p], head[p + 1 .. last]
  const int each = (parts + kJoinWaves - 1) / kJoinWaves;
  const int from = wave * each, to = from + each < parts ? from + each : parts;
  const int64_t c0 = static_cast<int64_t>(blockIdx.y) * kJoinCols + lane;
  float acc[4] = {};
#pragma unroll 4
  for (int k = from; k < to; ++k) {
    const float* src = k == 0 ? tail + static_cast<int64_t>(p) * E : head + static_cast<int64_t>(p + k) * E;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c0 + 64 * j < E) acc[j] += src[c0 + 64 * j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) part[wave][lane + 64 * j] = acc[j];
  __syncthreads();
  const int64_t c = static_cast<int64_t>(blockIdx.y) * kJoinCols + threadIdx.x;
  if (threadIdx.x < kJoinCols && c < E) {
    float s = part[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) s += part[w][threadIdx.x];
    float* d = dtable + id * E + c;
    *d = accumulate ? *d + scale * s : scale * s;
  }
}

// Positions of a piece. Long pieces store and read fewer partial sums; short ones keep
// enough waves in flight when tokens are few.
int piece_len(int64_t width, int64_t tokens) {
  const int64_t waves = tokens * ((width + 255) / 256);
  return waves >= 64 * 8192 ? 64 : waves >= 32 * 4096 ? 32 : 16;
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
  const int64_t chunks = (E + VEC - 1) / VEC, total = N * chunks;
  int64_t blocks = (total + 255) / 256;
  // enough workgroups for every compute unit before a thread takes a second vector
  if (blocks > 2048) blocks = (blocks + kLookupUnroll - 1) / kLookupUnroll;
  if (blocks > (1 << 20)) blocks = 1 << 20;
  launch_kernel(dlvm_embedding_kernel<T, VEC>, dim3(static_cast<uint32_t>(blocks)), dim3(256), s,
                static_cast<uint32_t>(V), E, static_cast<uint32_t>(chunks), total,
                static_cast<const T*>(table), ids, scale, static_cast<T*>(out));
}

template <typename T, int VEC>
void sum_pieces(const GradWs& w, int64_t E, int64_t n, char* ws, const T* dout, float scale,
                bool accumulate, float* dtable, hipStream_t s) {
  const int64_t pieces = (n + w.P - 1) / w.P, slabs = (E + 64 * VEC - 1) / (64 * VEC);
  launch_kernel(dlvm_embedding_pieces_kernel<T, VEC>, dim3(static_cast<uint32_t>((pieces * slabs + 3) / 4)),
                dim3(256), s, E, w.P, static_cast<int>(pieces), static_cast<int>(slabs),
                reinterpret_cast<const int32_t*>(ws + w.count), reinterpret_cast<const int32_t*>(ws + w.stok),
                reinterpret_cast<const int32_t*>(ws + w.sid), dout, scale, accumulate,
                reinterpret_cast<float*>(ws + w.head), reinterpret_cast<float*>(ws + w.tail), dtable);
}

// The widest vector that divides the row, but no wider than leaves each lane one.
template <typename T>
void sum_pieces_any(const GradWs& w, int64_t E, int64_t n, char* ws, const T* dout, float scale,
                    bool accumulate, float* dtable, hipStream_t s) {
  if (sizeof(T) == 2 && E % 8 == 0 && E >= 512)
    sum_pieces<T, sizeof(T) == 2 ? 8 : 4>(w, E, n, ws, dout, scale, accumulate, dtable, s);
  else if (E % 4 == 0 && E >= 256)
    sum_pieces<T, 4>(w, E, n, ws, dout, scale, accumulate, dtable, s);
  else if (E % 2 == 0 && E >= 128)
    sum_pieces<T, 2>(w, E, n, ws, dout, scale, accumulate, dtable, s);
  else
    sum_pieces<T, 1>(w, E, n, ws, dout, scale, accumulate, dtable, s);
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
    const uint32_t pieces = static_cast<uint32_t>((n + w.P - 1) / w.P);
    launch_kernel(dlvm_embedding_join_kernel,
                  dim3(pieces, static_cast<uint32_t>((width + kJoinCols - 1) / kJoinCols)),
                  dim3(64 * kJoinWaves), s, width, w.P, static_cast<int>(pieces), count, sid, scale, add,
                  reinterpret_cast<const float*>(base + w.head),
                  reinterpret_cast<const float*>(base + w.tail), dtable);
  }
  return hipGetLastError();
}

}  // namespace dlvm

// Embedding: rows of a table by ID, scaled, and the gradient of the table.
//
//   y_i = scale table[ids_i],   dtable_v = scale sum_{i: ids_i = v} dy_i
//
// Both are bound by memory.  The gradient's rows are summed in a fixed order and without atomics:
// (id, position) pairs are sorted by id, stably, so that a row's positions stand together in
// ascending order; the sorted positions are cut into chunks, and a group of lanes sums a chunk's
// rows, several of them in flight.  A run of equal ids that lies in one chunk is written at once;
// one that goes past a chunk's end (words come thousands of times) leaves a part in each of its
// chunks, and a second kernel adds those.
#include "hg_dense.hpp"
#include "hg_device.hpp"

namespace hg {
namespace {

constexpr int kBlock = 256;

// ---- forward -------------------------------------------------------------------

// 16 bytes of the result a lane; `across` lanes share a row (as many as it has vectors, or the
// block), and a lane has kAhead rows in flight.
template <typename T, typename O>
__global__ __launch_bounds__(kBlock) void k_embed(hg_embed_args A, int32_t across) {
  constexpr int V = kVec<O>, kAhead = 4;
  const int down = kBlock / across;
  const int r = threadIdx.x / across, lane = threadIdx.x - r * across;
  if (r >= down) return;
  const int64_t rows = int64_t(down) * kAhead;
  for (int64_t i0 = int64_t(blockIdx.x) * rows; i0 < A.n; i0 += int64_t(gridDim.x) * rows) {
    int64_t id[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t i = i0 + u * down + r;
      id[u] = i < A.n ? A.ids[i] : -1;
    }
    for (int64_t c = int64_t(lane) * V; c < A.dim; c += int64_t(across) * V) {
      const int n = int(min<int64_t>(V, A.dim - c));
      Vec<T, V> t[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const T rest = T(id[u] == -1 ? 0.0f : __builtin_nanf(""));
        if (id[u] >= 0 && id[u] < A.nodes) {
          t[u].load(static_cast<const T *>(A.table) + id[u] * A.table_stride + c, n);
        } else {
#pragma unroll
          for (int k = 0; k < V; ++k) t[u].e[k] = rest;
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int64_t i = i0 + u * down + r;
        Vec<O, V> y;
#pragma unroll
        for (int k = 0; k < V; ++k)
          y.e[k] = O(id[u] == -1 ? 0.0f : float(t[u].e[k]) * A.scale);
        if (i < A.n)
          y.template store<Move::kStreamed>(static_cast<O *>(A.y) + i * A.y_stride + c, n);
      }
    }
  }
}

// ---- the sort ------------------------------------------------------------------

// An id (below `nodes`; `nodes`: it counts for nothing) and its position.
struct Pair {
  uint32_t id, at;
};

__device__ __forceinline__ Pair pair_of(const int64_t *ids, int64_t i, int64_t nodes) {
  const int64_t v = ids[i];
  return Pair{v >= 0 && v < nodes ? uint32_t(v) : uint32_t(nodes), uint32_t(i)};
}

// Lanes (that are `in`) with this lane's digit.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool in) {
  uint64_t same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const bool one = digit >> b & 1;
    const uint64_t ones = __ballot(one);
    same &= one ? ones : ~ones;
  }
  return same;
}

// How many of this wavefront's pairs before this one have its digit; count [digits] holds those of
// the rounds before, and then of this one too.
__device__ __forceinline__ uint32_t take_place(uint32_t *count, uint32_t digit, int bits, bool in) {
  const uint64_t same = same_digit(digit, bits, in);
  const uint32_t before = __popcll(same & lanes_below());
  const uint32_t seen = in ? count[digit] : 0;
  wave_sync();
  if (in && before == 0) count[digit] = seen + __popcll(same);
  wave_sync();
  return seen + before;
}

// Exclusive sums over the block of one value a thread (red: LDS [wavefronts]).
template <int kThreads>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *red, uint32_t *total) {
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(s, d, 64);
    if (lane_id() >= d) s += o;
  }
  __syncthreads();
  if (lane_id() == 63) red[threadIdx.x >> 6] = s;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < int(threadIdx.x >> 6)) before += red[w];
    all += red[w];
  }
  *total = all;
  return before + s - v;
}

// Marks of the ids that are there, cleared by `threads` threads of which this is `t`.
__device__ __forceinline__ void clear(uint8_t *marks, int64_t nodes, int64_t t, int64_t threads) {
  const u32x4 none = {0, 0, 0, 0};
  for (int64_t v = t * 16; v < nodes; v += threads * 16)
    *reinterpret_cast<u32x4 *>(marks + v) = none;  // (whole pieces: the array ends at one)
}

// All of the sort in one block's LDS.
constexpr int kSmallThreads = 1024;
__global__ __launch_bounds__(kSmallThreads) void k_sort_small(const int64_t *ids, int32_t n,
                                                              int64_t nodes, int32_t passes,
                                                              int32_t digit, Pair *out,
                                                              uint8_t *marks) {
  constexpr int kWaves = kSmallThreads / 64, kRounds = int(kSortSmall) / kSmallThreads;
  constexpr int kBins = 1 << kSmallDigitBits;
  __shared__ Pair pairs[kSortSmall];
  __shared__ uint32_t count[kWaves][kBins];
  __shared__ uint32_t red[kWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int rounds = (n + kSmallThreads - 1) / kSmallThreads;
  const int first = wave * rounds * 64 + lane;
  if (marks) clear(marks, nodes, threadIdx.x, kSmallThreads);
  Pair p[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int i = first + r * 64;
    p[r] = r < rounds && i < n ? pair_of(ids, i, nodes) : Pair{0, 0};
  }
  __syncthreads();
  if (marks) {
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
      if (r < rounds && first + r * 64 < n && p[r].id < nodes) marks[p[r].id] = 1;
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * digit;
    for (int t = threadIdx.x; t < kWaves * kBins; t += kSmallThreads) (&count[0][0])[t] = 0;
    __syncthreads();
    uint32_t place[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (r < rounds)
        place[r] = take_place(count[wave], p[r].id >> shift & ((1u << digit) - 1), digit,
                              first + r * 64 < n);
    }
    __syncthreads();
    // a digit's pairs of all wavefronts, then the digits before it
    uint32_t sum = 0, all;
    const int d = threadIdx.x;
    if (d < kBins)
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = count[w][d];
        count[w][d] = sum;
        sum += c;
      }
    const uint32_t before = block_scan<kSmallThreads>(d < kBins ? sum : 0, red, &all);
    if (d < kBins)
      for (int w = 0; w < kWaves; ++w) count[w][d] += before;
    __syncthreads();
    const bool last = pass + 1 == passes;
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
      if (r < rounds && first + r * 64 < n) {
        const uint32_t to = count[wave][p[r].id >> shift & ((1u << digit) - 1)] + place[r];
        (last ? out : pairs)[to] = p[r];
      }
    if (last) return;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
      if (r < rounds && first + r * 64 < n) p[r] = pairs[first + r * 64];
  }
}

// A pass of the sort over more pairs: counts by tile, their sums, the pairs to their places.
// The first pass takes them from the ids.
struct SortPass {
  const int64_t *ids;  // or
  const Pair *from;
  Pair *to;
  int64_t n, nodes, tiles;
  int32_t shift, digit;
  uint32_t *counts;  // [digits, tiles]
  uint32_t *totals;  // [digits]
  uint8_t *marks;    // with ids
  __device__ __forceinline__ Pair at(int64_t i) const {
    return ids ? pair_of(ids, i, nodes) : from[i];
  }
  __device__ __forceinline__ uint32_t digit_of(Pair p) const {
    return p.id >> shift & ((1u << digit) - 1);
  }
};

template <int kItems>
__global__ __launch_bounds__(kBlock) void k_sort_count(SortPass A) {
  __shared__ uint32_t count[1 << kMostDigitBits];
  const int bins = 1 << A.digit;
  for (int d = threadIdx.x; d < bins; d += kBlock) count[d] = 0;
  if (A.ids && A.marks)
    clear(A.marks, A.nodes, int64_t(blockIdx.x) * kBlock + threadIdx.x, int64_t(gridDim.x) * kBlock);
  __syncthreads();
  const int64_t first = int64_t(blockIdx.x) * kBlock * kItems + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kItems; ++u)
    if (first + u * kBlock < A.n) atomicAdd(&count[A.digit_of(A.at(first + u * kBlock))], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += kBlock) A.counts[d * A.tiles + blockIdx.x] = count[d];
}

// A block for each digit: what the tiles before have of it.
__global__ __launch_bounds__(kBlock) void k_sort_scan(SortPass A) {
  __shared__ uint32_t red[kBlock / 64];
  uint32_t *const row = A.counts + blockIdx.x * A.tiles;
  uint32_t before = 0;
  for (int64_t t = threadIdx.x; t - threadIdx.x < A.tiles; t += kBlock) {
    uint32_t all;
    const uint32_t v = t < A.tiles ? row[t] : 0;
    const uint32_t s = block_scan<kBlock>(v, red, &all);
    if (t < A.tiles) row[t] = before + s;
    before += all;
  }
  if (threadIdx.x == 0) A.totals[blockIdx.x] = before;
}

template <int kItems>
__global__ __launch_bounds__(kBlock) void k_sort_place(SortPass A) {
  constexpr int kWaves = kBlock / 64, kBins = 1 << kMostDigitBits;
  __shared__ uint32_t count[kWaves][kBins];
  __shared__ uint32_t red[kWaves];
  const int bins = 1 << A.digit;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int w = 0; w < kWaves; ++w)
    for (int d = threadIdx.x; d < bins; d += kBlock) count[w][d] = 0;
  const int64_t first = (int64_t(blockIdx.x) * kWaves + wave) * kItems * 64 + lane;
  Pair p[kItems];
#pragma unroll
  for (int r = 0; r < kItems; ++r)
    p[r] = first + r * 64 < A.n ? A.at(first + r * 64) : Pair{0, 0};
  __syncthreads();
  uint32_t place[kItems];
#pragma unroll
  for (int r = 0; r < kItems; ++r)
    place[r] = take_place(count[wave], A.digit_of(p[r]), A.digit, first + r * 64 < A.n);
  if (A.ids && A.marks) {
#pragma unroll
    for (int r = 0; r < kItems; ++r)
      if (first + r * 64 < A.n && p[r].id < A.nodes) A.marks[p[r].id] = 1;
  }
  // the pairs of smaller digits, those of earlier tiles, those of earlier wavefronts
  uint32_t smaller = 0;
  for (int d0 = 0; d0 < bins; d0 += kBlock) {
    const int d = d0 + threadIdx.x;
    uint32_t all;
    const uint32_t s = block_scan<kBlock>(d < bins ? A.totals[d] : 0, red, &all);
    if (d < bins) {
      uint32_t at = smaller + s + A.counts[d * A.tiles + blockIdx.x];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = count[w][d];
        count[w][d] = at;
        at += c;
      }
    }
    smaller += all;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kItems; ++r)
    if (first + r * 64 < A.n) A.to[count[wave][A.digit_of(p[r])] + place[r]] = p[r];
}

// ---- the sums ------------------------------------------------------------------

struct Sums {
  const Pair *pairs;  // sorted
  int64_t n, nodes, dim;
  const void *dy;
  int64_t dy_stride;
  void *out;
  int64_t out_stride;
  float scale;
  int64_t chunk, chunks;
  float *parts;  // [chunks, 2, dim]: of the run that came into a chunk, of the one that starts there
  int64_t slices, sum_blocks, blocks;
  const uint8_t *marks;  // NULL: no row is there
  int64_t fill_rows;     // of a block that fills
  __device__ __forceinline__ uint32_t id(int64_t i) const { return pairs[i].id; }
};

// N sums to a row of the table, n of them in it.
template <typename O, bool kAdd, int N>
__device__ __forceinline__ void put_row(const Sums &A, uint32_t row, int64_t c, const float *v,
                                        int n) {
  O *const to = static_cast<O *>(A.out) + int64_t(row) * A.out_stride + c;
  Vec<O, N> t;
  if (kAdd) t.load(to, n);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float s = v[k] * A.scale;
    t.e[k] = O(kAdd ? float(t.e[k]) + s : s);
  }
  t.store(to, n);
}

// G lanes sum a chunk, for G V columns.  Blocks past sum_blocks fill rows that no id names.
template <typename T, typename O, bool kAdd, int G>
__global__ __launch_bounds__(kBlock) void k_embed_sum(Sums A) {
  constexpr int V = kVec<T>, kAhead = 8;
  for (int64_t b = blockIdx.x; b < A.blocks; b += gridDim.x) {
    if (b >= A.sum_blocks) {
      if constexpr (!kAdd) {
        constexpr int W = kVec<O>;
        const int64_t r0 = (b - A.sum_blocks) * A.fill_rows;
        const uint32_t rows = uint32_t(min(A.fill_rows, A.nodes - r0));
        const uint32_t across = uint32_t((A.dim + W - 1) / W);
        Vec<O> none;
#pragma unroll
        for (int k = 0; k < W; ++k) none.e[k] = O(0.0f);
        for (uint64_t t = threadIdx.x; t < uint64_t(rows) * across; t += kBlock) {
          const int64_t r = r0 + int64_t(t / across), c = int64_t(t % across) * W;
          if (A.marks && A.marks[r]) continue;
          none.template store<Move::kStreamed>(static_cast<O *>(A.out) + r * A.out_stride + c,
                                               int(min<int64_t>(W, A.dim - c)));
        }
      }
      continue;
    }
    const int64_t chunk = b / A.slices * (kBlock / G) + threadIdx.x / G;
    const int64_t c = (b % A.slices * G + threadIdx.x % G) * V;
    if (chunk >= A.chunks || c >= A.dim) continue;
    const int n = int(min<int64_t>(V, A.dim - c));
    const int64_t first = chunk * A.chunk, last = min(first + A.chunk, A.n);
    const uint32_t before = first > 0 ? A.id(first - 1) : ~0u;
    const uint32_t after = last < A.n ? A.id(last) : ~0u;
    uint32_t now = A.id(first);
    float s[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = 0.0f;
    const auto part = [&](int which) {
      Vec<float, V> t;
#pragma unroll
      for (int k = 0; k < V; ++k) t.e[k] = s[k];
      t.store(A.parts + (2 * chunk + which) * A.dim + c, n);
    };
    const auto leave = [&](bool ends) {
      if (now >= A.nodes) return;
      if (now == before)
        part(0);
      else if (!ends)
        part(1);
      else
        put_row<O, kAdd, V>(A, now, c, s, n);
    };
    for (int64_t e = first; e < last; e += kAhead) {
      Pair p[kAhead];
      Vec<T> r[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        p[u] = e + u < last ? A.pairs[e + u] : Pair{uint32_t(A.nodes), 0};
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (p[u].id < A.nodes)
          r[u].template load<Move::kStreamed>(
              static_cast<const T *>(A.dy) + int64_t(p[u].at) * A.dy_stride + c, n);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (e + u < last) {
          if (p[u].id != now) {
            leave(true);
            now = p[u].id;
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] = 0.0f;
          }
          if (now < A.nodes) {
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] += float(r[u].e[k]);
          }
        }
      }
    }
    leave(now != after);
  }
}

// Adds the parts of the runs that go past a chunk's end: a block for the chunk that a run starts in,
// 32 lanes across 128 columns, 8 down that take turns over the parts.
template <typename O, bool kAdd>
__global__ __launch_bounds__(kBlock) void k_embed_join(Sums A, int64_t places) {
  constexpr int kDown = kBlock / 32, N = 4;
  __shared__ float red[kDown][32][N + 1];
  const int lane = threadIdx.x & 31, turn = threadIdx.x >> 5;
  const int64_t slices = (A.dim + 127) / 128;
  for (int64_t b = blockIdx.x; b < places; b += gridDim.x) {
    const int64_t chunk = b / slices;
    // (what leaves a place is the same for the whole block)
    const int64_t next = (chunk + 1) * A.chunk;
    const uint32_t run = A.id(next - 1);
    if (run >= A.nodes || A.id(next) != run) continue;
    if (chunk > 0 && A.id(chunk * A.chunk - 1) == run) continue;
    // the last chunk that it comes into: doubled steps, then halved ones
    int64_t last = chunk + 1, step = 1;
    while (last + step < A.chunks && A.id((last + step) * A.chunk) == run) {
      last += step;
      step *= 2;
    }
    for (; step > 0; step /= 2)
      if (last + step < A.chunks && A.id((last + step) * A.chunk) == run) last += step;
    const int64_t c = (b % slices * 32 + lane) * N;
    const int n = int(max<int64_t>(0, min<int64_t>(N, A.dim - c)));
    float s[N] = {};
    if (n > 0) {
      // part 0 is the chunk's own, the others came into their chunks
#pragma unroll 4
      for (int64_t k = turn; k <= last - chunk; k += kDown) {
        Vec<float, N> t;
        t.load(A.parts + (2 * (chunk + k) + (k == 0)) * A.dim + c, n);
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] += t.e[j];
      }
    }
    __syncthreads();  // the last place's sums have been read
#pragma unroll
    for (int j = 0; j < N; ++j) red[turn][lane][j] = s[j];
    __syncthreads();
    if (turn == 0 && n > 0) {
      for (int t = 1; t < kDown; ++t)
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] += red[t][lane][j];
      put_row<O, kAdd, N>(A, run, c, s, n);
    }
  }
}

// ---- launches ------------------------------------------------------------------

template <typename T, typename O>
hipError_t forward(const hg_embed_args &A, hipStream_t stream) {
  const int64_t vectors = ceil_div<int64_t>(A.dim, kVec<O>);
  const int64_t across = std::min<int64_t>(vectors, kBlock);
  const int64_t blocks = ceil_div<int64_t>(A.n, kBlock / across * 4);
  hipLaunchKernelGGL((k_embed<T, O>), dim3(unsigned(std::min(blocks, kMostBlocks))), dim3(kBlock), 0,
                     stream, A, int32_t(across));
  return hipGetLastError();
}
template <typename T>
hipError_t forward(const hg_embed_args &A, hipStream_t stream) {
  switch (A.out_dtype) {
    case HG_DT_F32: return forward<T, float>(A, stream);
    case HG_DT_F16: return forward<T, _Float16>(A, stream);
    default: return forward<T, __bf16>(A, stream);
  }
}

hipError_t sort(const hg_embed_grad_args &A, const EmbedPlan &p, hipStream_t stream,
                const Pair **sorted) {
  char *const ws = static_cast<char *>(A.workspace);
  Pair *to = reinterpret_cast<Pair *>(ws + p.pairs), *other = reinterpret_cast<Pair *>(ws + p.other);
  uint8_t *const marks = A.add ? nullptr : reinterpret_cast<uint8_t *>(ws + p.marks);
  if (p.small) {
    hipLaunchKernelGGL(k_sort_small, dim3(1), dim3(kSmallThreads), 0, stream, A.ids, int32_t(A.n),
                       A.nodes, p.passes, p.digit, to, marks);
    *sorted = to;
    return hipGetLastError();
  }
  SortPass S{};
  S.ids = A.ids;
  S.n = A.n;
  S.nodes = A.nodes;
  S.tiles = p.tiles;
  S.digit = p.digit;
  S.counts = reinterpret_cast<uint32_t *>(ws + p.counts);
  S.totals = reinterpret_cast<uint32_t *>(ws + p.totals);
  S.marks = marks;
  const dim3 tiles(unsigned(p.tiles)), block(kBlock);
  for (int pass = 0; pass < p.passes; ++pass) {
    S.shift = pass * p.digit;
    S.to = to;
    if (p.tile == 1024)
      hipLaunchKernelGGL(k_sort_count<4>, tiles, block, 0, stream, S);
    else
      hipLaunchKernelGGL(k_sort_count<16>, tiles, block, 0, stream, S);
    hipLaunchKernelGGL(k_sort_scan, dim3(1u << p.digit), block, 0, stream, S);
    if (p.tile == 1024)
      hipLaunchKernelGGL(k_sort_place<4>, tiles, block, 0, stream, S);
    else
      hipLaunchKernelGGL(k_sort_place<16>, tiles, block, 0, stream, S);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    S.ids = nullptr;
    S.from = to;
    std::swap(to, other);
  }
  *sorted = S.from;
  return hipSuccess;
}

template <typename T, typename O, bool kAdd>
hipError_t gradient(const hg_embed_grad_args &A, hipStream_t stream) {
  const EmbedPlan p = embed_plan(A.n, A.nodes, A.dim, kAdd);
  Sums S{};
  if (A.n > 0) {
    const hipError_t e = sort(A, p, stream, &S.pairs);
    if (e != hipSuccess) return e;
  }
  char *const ws = static_cast<char *>(A.workspace);
  S.n = A.n;
  S.nodes = A.nodes;
  S.dim = A.dim;
  S.dy = A.dy;
  S.dy_stride = A.dy_stride;
  S.out = A.dtable;
  S.out_stride = A.dtable_stride;
  S.scale = A.scale;
  S.chunk = p.chunk;
  S.chunks = p.chunks;
  S.parts = reinterpret_cast<float *>(ws + p.parts);
  S.marks = A.n > 0 ? reinterpret_cast<uint8_t *>(ws + p.marks) : nullptr;
  const int64_t vectors = ceil_div<int64_t>(A.dim, kVec<T>);
  int64_t lanes = 8;
  while (lanes < vectors && lanes < kBlock) lanes *= 2;
  S.slices = ceil_div<int64_t>(vectors, lanes);
  S.sum_blocks = ceil_div<int64_t>(p.chunks, kBlock / lanes) * S.slices;
  // a block fills some 64 KB
  S.fill_rows = std::max<int64_t>(1, 65536 / (A.dim * int64_t(sizeof(O))));
  S.blocks = S.sum_blocks + (kAdd ? 0 : ceil_div<int64_t>(A.nodes, S.fill_rows));
  if (S.blocks == 0) return hipSuccess;
  const dim3 grid(unsigned(std::min(S.blocks, kMostBlocks))), block(kBlock);
  switch (lanes) {
    case 8: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 8>), grid, block, 0, stream, S); break;
    case 16: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 16>), grid, block, 0, stream, S); break;
    case 32: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 32>), grid, block, 0, stream, S); break;
    case 64: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 64>), grid, block, 0, stream, S); break;
    case 128: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 128>), grid, block, 0, stream, S); break;
    default: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 256>), grid, block, 0, stream, S);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.chunks < 2) return e;
  const int64_t places = (p.chunks - 1) * ceil_div<int64_t>(A.dim, 128);
  hipLaunchKernelGGL((k_embed_join<O, kAdd>), dim3(unsigned(std::min(places, kMostBlocks))), block, 0,
                     stream, S, places);
  return hipGetLastError();
}
template <typename T>
hipError_t gradient(const hg_embed_grad_args &A, hipStream_t stream) {
  if (A.add) return gradient<T, float, true>(A, stream);
  return A.out_dtype == HG_DT_F32 ? gradient<T, float, false>(A, stream)
                                  : gradient<T, T, false>(A, stream);
}

}  // namespace

hipError_t launch_embed(const hg_embed_args &A, hipStream_t stream) {
  if (A.n <= 0) return hipSuccess;
  switch (A.table_dtype) {
    case HG_DT_F32: return forward<float>(A, stream);
    case HG_DT_F16: return forward<_Float16>(A, stream);
    default: return forward<__bf16>(A, stream);
  }
}

int64_t embed_grad_workspace(int64_t n, int64_t nodes, int64_t dim, bool add) {
  return n > 0 ? embed_plan(n, nodes, dim, add).total : 0;
}

hipError_t launch_embed_grad(const hg_embed_grad_args &A, hipStream_t stream) {
  if (A.nodes <= 0) return hipSuccess;
  switch (A.dtype) {
    case HG_DT_F32: return gradient<float>(A, stream);
    case HG_DT_F16: return gradient<_Float16>(A, stream);
    default: return gradient<__bf16>(A, stream);
  }
}

}  // namespace hg

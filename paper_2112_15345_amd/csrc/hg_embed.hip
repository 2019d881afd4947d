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
// block), and a lane has kAhead rows in flight.  65537 words of 1024 columns, float32 to bfloat16: 40 us, 4.9
// TB/s; with 16 bytes of the row a lane, 8 of the result, 42.
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
__device__ __forceinline__ uint32_t take_place(uint16_t *count, uint32_t digit, int bits, bool in) {
  const uint64_t same = same_digit(digit, bits, in);
  const uint32_t before = __popcll(same & lanes_below());
  const uint32_t seen = in ? count[digit] : 0;
  wave_sync();
  if (in && before == 0) count[digit] = uint16_t(seen + __popcll(same));
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

// Zeros into a table's rows: pieces of some 64 KB, of which a launch takes those from `first` on in
// the blocks past `own`.  The sort's kernels wait for their loads and leave the memory idle, so
// they carry this on the side (the sums are written after them, over the zeros).
struct Fill {
  void *out;
  int64_t stride, rows, dim;
  int32_t size;  // bytes of an element
  int64_t rows_of_piece;  // 0: the rows follow each other without gaps, and are filled as one
  int64_t first, own;
};
constexpr int64_t kFillBytes = 65536;
__device__ __forceinline__ void fill_bytes(void *at, int n) {
  Vec<uint8_t, 16> none;
#pragma unroll
  for (int k = 0; k < 16; ++k) none.e[k] = 0;
  none.template store<Move::kStreamed>(static_cast<uint8_t *>(at), n);
}
// Whether this block fills.
__device__ __forceinline__ bool filled(const Fill &F) {
  if (int64_t(blockIdx.x) < F.own) return false;
  const int64_t piece = F.first + blockIdx.x - F.own;
  uint8_t *const out = static_cast<uint8_t *>(F.out);
  if (F.rows_of_piece == 0) {
    const int64_t bytes = F.rows * F.dim * F.size, end = min(bytes, (piece + 1) * kFillBytes);
    for (int64_t c = piece * kFillBytes + threadIdx.x * 16; c < end; c += blockDim.x * 16)
      fill_bytes(out + c, int(min<int64_t>(16, bytes - c)));
    return true;
  }
  const int64_t r0 = piece * F.rows_of_piece, bytes = F.dim * F.size;
  const uint32_t rows = uint32_t(min(F.rows_of_piece, F.rows - r0));
  const uint32_t across = uint32_t((bytes + 15) / 16);
  for (uint64_t t = threadIdx.x; t < uint64_t(rows) * across; t += blockDim.x) {
    // (either there is one row, or few enough pieces of 16 bytes for 32 bits)
    const int64_t row = rows == 1 ? 0 : uint32_t(t) / across;
    const int64_t c = (int64_t(t) - row * across) * 16;
    fill_bytes(out + (r0 + row) * F.stride * F.size + c, int(min<int64_t>(16, bytes - c)));
  }
  return true;
}

// All of the sort in one block's LDS.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortRounds = int(kSortTile) / kSortThreads;
static_assert(kSortSmall == kSortTile, "as many pairs a thread");
__global__ __launch_bounds__(kSortThreads) void k_sort_small(const int64_t *ids, int32_t n,
                                                             int64_t nodes, int32_t passes,
                                                             int32_t digit, Pair *out, Fill fill) {
  constexpr int kBins = 1 << kSmallDigitBits;
  __shared__ Pair pairs[kSortSmall];
  __shared__ uint16_t count[kSortWaves][kBins];
  __shared__ uint32_t base[kBins];
  __shared__ uint32_t red[kSortWaves];
  if (filled(fill)) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int rounds = (n + kSortThreads - 1) / kSortThreads;
  const int first = wave * rounds * 64 + lane;
  Pair p[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int i = first + r * 64;
    p[r] = r < rounds && i < n ? pair_of(ids, i, nodes) : Pair{0, 0};
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * digit;
    const auto digit_of = [&](Pair q) { return q.id >> shift & ((1u << digit) - 1); };
    for (int t = threadIdx.x; t < kSortWaves * kBins; t += kSortThreads) (&count[0][0])[t] = 0;
    __syncthreads();
    uint32_t place[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      if (r < rounds)
        place[r] = take_place(count[wave], digit_of(p[r]), digit, first + r * 64 < n);
    }
    __syncthreads();
    // a digit's pairs of all wavefronts, then the digits before it
    uint32_t sum = 0, all;
    const int d = threadIdx.x;
    if (d < kBins)
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = count[w][d];
        count[w][d] = uint16_t(sum);
        sum += c;
      }
    const uint32_t before = block_scan<kSortThreads>(d < kBins ? sum : 0, red, &all);
    if (d < kBins) base[d] = before;
    __syncthreads();
    const bool last = pass + 1 == passes;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (r < rounds && first + r * 64 < n) {
        const uint32_t to = base[digit_of(p[r])] + count[wave][digit_of(p[r])] + place[r];
        if (last)
          out[to] = p[r];
        else
          pairs[to] = p[r];
      }
    if (last) return;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (r < rounds && first + r * 64 < n) p[r] = pairs[first + r * 64];
  }
}

// A pass of the sort over more pairs: counts by tile, then the pairs to their places.  The first
// pass takes them from the ids.
struct SortPass {
  const int64_t *ids;  // or
  const Pair *from;
  Pair *to;
  int64_t n, nodes, tiles;
  int32_t shift, digit;
  uint32_t *counts;  // of tile t and digit d at t by_tile + d by_digit
  int64_t by_tile, by_digit;
  uint32_t *totals;  // [digits], with k_sort_scan; else NULL
  Fill fill;
  __device__ __forceinline__ Pair at(int64_t i) const {
    return ids ? pair_of(ids, i, nodes) : from[i];
  }
  __device__ __forceinline__ uint32_t digit_of(Pair p) const {
    return p.id >> shift & ((1u << digit) - 1);
  }
};

__global__ __launch_bounds__(kSortThreads) void k_sort_count(SortPass A) {
  __shared__ uint32_t count[1 << kMostDigitBits];
  if (filled(A.fill)) return;
  const int bins = 1 << A.digit;
  const int64_t first = int64_t(blockIdx.x) * kSortTile + threadIdx.x;
  Pair p[kSortRounds];
#pragma unroll
  for (int u = 0; u < kSortRounds; ++u)
    if (first + u * kSortThreads < A.n) p[u] = A.at(first + u * kSortThreads);
  for (int d = threadIdx.x; d < bins; d += kSortThreads) count[d] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kSortRounds; ++u)
    if (first + u * kSortThreads < A.n) atomicAdd(&count[A.digit_of(p[u])], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += kSortThreads)
    A.counts[blockIdx.x * A.by_tile + d * A.by_digit] = count[d];
}

// A block for each digit: what the tiles before have of it.
__global__ __launch_bounds__(kBlock) void k_sort_scan(SortPass A) {
  __shared__ uint32_t red[kBlock / 64];
  uint32_t *const row = A.counts + blockIdx.x * A.by_digit;  // (by_tile is 1)
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

__global__ __launch_bounds__(kSortThreads) void k_sort_place(SortPass A) {
  constexpr int kBins = 1 << kMostDigitBits;
  __shared__ uint16_t count[kSortWaves][kBins];
  __shared__ uint32_t base[kBins];
  __shared__ uint32_t red[kSortWaves];
  if (filled(A.fill)) return;
  const int bins = 1 << A.digit;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t first = (int64_t(blockIdx.x) * kSortWaves + wave) * kSortRounds * 64 + lane;
  Pair p[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r)
    p[r] = first + r * 64 < A.n ? A.at(first + r * 64) : Pair{0, 0};
  for (int d = 2 * lane; d < bins; d += 128) *reinterpret_cast<uint32_t *>(&count[wave][d]) = 0;
  // the pairs of smaller digits, and those of this one in earlier tiles
  uint32_t smaller = 0;
  for (int d0 = 0; d0 < bins; d0 += kSortThreads) {
    const int d = d0 + threadIdx.x;
    uint32_t earlier = 0, total = 0, all;
    if (d < bins) {
      if (A.totals) {
        earlier = A.counts[blockIdx.x * A.by_tile + d * A.by_digit];
        total = A.totals[d];
      } else {
        // (loads of tiles that are not there, to have 32 at once, cost more: 15.2 us a pass of 37
        // tiles, not 12.4)
#pragma unroll 16
        for (int t = 0; t < int(A.tiles); ++t) {
          const uint32_t c = A.counts[t * A.by_tile + d * A.by_digit];
          earlier += t < int(blockIdx.x) ? c : 0;
          total += c;
        }
      }
    }
    const uint32_t s = block_scan<kSortThreads>(total, red, &all);  // (a barrier at least)
    if (d < bins) base[d] = smaller + s + earlier;
    smaller += all;
  }
  uint32_t place[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r)
    place[r] = take_place(count[wave], A.digit_of(p[r]), A.digit, first + r * 64 < A.n);
  __syncthreads();
  // those of earlier wavefronts
  for (int d = threadIdx.x; d < bins; d += kSortThreads) {
    uint32_t c[kSortWaves], sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) c[w] = count[w][d];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      count[w][d] = uint16_t(sum);
      sum += c[w];
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r)
    if (first + r * 64 < A.n) {
      const uint32_t d = A.digit_of(p[r]);
      A.to[base[d] + count[wave][d] + place[r]] = p[r];
    }
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
  int32_t *ends;  // [chunks]: the last chunk of the run that starts there and goes on, or 0
  int64_t slices, blocks;
  __device__ __forceinline__ uint32_t id(int64_t i) const { return pairs[i].id; }
};

template <typename O, int N>
__device__ __forceinline__ O *row_at(const Sums &A, uint32_t row, int64_t c) {
  return static_cast<O *>(A.out) + int64_t(row) * A.out_stride + c;
}
// A pair; uniform: the same for all lanes of a wavefront, by the scalar unit (nothing writes pairs in
// the kernels that read them so).
template <bool kUniform>
__device__ __forceinline__ Pair pair_at(const Sums &A, int64_t i) {
  if constexpr (kUniform) {
    typedef const __attribute__((address_space(4))) uint64_t Word;
    const uint64_t w = ((Word *)(A.pairs))[i];
    return Pair{uint32_t(w), uint32_t(w >> 32)};
  } else {
    return A.pairs[i];
  }
}

// N sums to a row of the table, n of them in it; `old` (kAdd): what it has.
template <typename O, bool kAdd, int N>
__device__ __forceinline__ void put_row(const Sums &A, uint32_t row, int64_t c, const float *v,
                                        int n, const Vec<O, N> &old) {
  Vec<O, N> t;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float s = v[k] * A.scale;
    t.e[k] = O(kAdd ? float(old.e[k]) + s : s);
  }
  t.template store<Move::kStreamed>(row_at<O, N>(A, row, c), n);
}

// The last chunk that a run which goes past the end of `chunk` comes into: doubled steps, then
// halved ones.
__device__ __forceinline__ int64_t end_of_run(const Sums &A, int64_t chunk, uint32_t run) {
  int64_t last = chunk + 1, step = 1;
  while (last + step < A.chunks && A.id((last + step) * A.chunk) == run) {
    last += step;
    step *= 2;
  }
  for (; step > 0; step /= 2)
    if (last + step < A.chunks && A.id((last + step) * A.chunk) == run) last += step;
  return last;
}

// G lanes sum a chunk, for G V columns.  (16 bytes of dy a lane: with 16 bytes of a wider result a
// lane instead, 8 of dy, the text's gradient of 50001 x 1024 took 97 us here, not 49.)
template <typename T, typename O, bool kAdd, int G>
__global__ __launch_bounds__(kBlock) void k_embed_sum(Sums A) {
  constexpr int V = kVec<T>, kAhead = 8;
  for (int64_t b = blockIdx.x; b < A.blocks; b += gridDim.x) {
    int64_t chunk = b / A.slices * (kBlock / G) + threadIdx.x / G;
    // (the same for a wavefront's lanes: the pairs are read once for all of them)
    if (G >= 64) chunk = int64_t(__builtin_amdgcn_readfirstlane(int(chunk)));
    const int64_t c = (b % A.slices * G + threadIdx.x % G) * V;
    if (chunk >= A.chunks || c >= A.dim) continue;
    const int n = int(min<int64_t>(V, A.dim - c));
    const int64_t first = chunk * A.chunk, last = min(first + A.chunk, A.n);
    const uint32_t before = first > 0 ? pair_at<(G >= 64)>(A, first - 1).id : ~0u;
    const uint32_t after = last < A.n ? pair_at<(G >= 64)>(A, last).id : ~0u;
    uint32_t now = pair_at<(G >= 64)>(A, first).id;
    float s[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = 0.0f;
    Vec<O, V> old;
    const auto leave = [&](bool ends) {
      if (now >= A.nodes) return;
      if (now == before || !ends) {
        Vec<float, V> t;
#pragma unroll
        for (int k = 0; k < V; ++k) t.e[k] = s[k];
        t.store(A.parts + (2 * chunk + (now != before)) * A.dim + c, n);
      } else {
        put_row<O, kAdd, V>(A, now, c, s, n, old);
      }
    };
    // pairs are read one round ahead of the rows that they name
    Pair p[kAhead + 1];
    const auto read = [&](int64_t e) {
#pragma unroll
      for (int u = 0; u <= kAhead; ++u)
        p[u] = e + u < last ? pair_at<(G >= 64)>(A, e + u) : Pair{uint32_t(A.nodes), 0};
    };
    read(first);
    for (int64_t e = first; e < last; e += kAhead) {
      uint32_t id[kAhead];
      Vec<T> r[kAhead];
      Vec<O, V> t[kAdd ? kAhead : 1];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        id[u] = p[u].id;
        if (id[u] < A.nodes) {
          r[u].template load<Move::kStreamed>(
              static_cast<const T *>(A.dy) + int64_t(p[u].at) * A.dy_stride + c, n);
          // the row that a run's sum is added to, where it ends: loaded with the others (150001
          // rows of 128 floats: 87 us where each waited for its own, now 51)
          if (kAdd && id[u] != p[u + 1].id) t[kAdd ? u : 0].load(row_at<O, V>(A, id[u], c), n);
        }
      }
      if (e + kAhead < last) read(e + kAhead);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (e + u < last) {
          if (id[u] != now) {
            leave(true);
            now = id[u];
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] = 0.0f;
          }
          if (now < A.nodes) {
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] += float(r[u].e[k]);
            if constexpr (kAdd) old = t[u];
          }
        }
      }
    }
    leave(now != after);
    if (c == 0)
      A.ends[chunk] = now < A.nodes && now == after && now != before
                          ? int32_t(end_of_run(A, chunk, now)) : 0;
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
    const int64_t last = A.ends[chunk];
    if (last == 0) continue;  // (the same for the whole block)
    const uint32_t run = A.id((chunk + 1) * A.chunk);
    const int64_t c = (b % slices * 32 + lane) * N;
    const int n = int(max<int64_t>(0, min<int64_t>(N, A.dim - c)));
    float s[N] = {};
    if (n > 0) {
      // part 0 is the chunk's own, the others came into their chunks
#pragma unroll 8
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
      Vec<O, N> old;
      if (kAdd) old.load(row_at<O, N>(A, run, c), n);
      put_row<O, kAdd, N>(A, run, c, s, n, old);
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

// Sorts the pairs; the sort's kernels take turns with the pieces to fill.
hipError_t sort(const hg_embed_grad_args &A, const EmbedPlan &p, Fill fill, int64_t pieces,
                hipStream_t stream, const Pair **sorted) {
  char *const ws = static_cast<char *>(A.workspace);
  Pair *to = reinterpret_cast<Pair *>(ws + p.pairs), *other = reinterpret_cast<Pair *>(ws + p.other);
  const bool few = p.tiles <= kFewTiles;
  int64_t launches = p.small ? 1 : 2 * p.passes;
  // blocks of a launch that has `own` for itself
  const auto grid = [&](int64_t own) {
    const int64_t share = ceil_div<int64_t>(pieces - fill.first, launches--);
    fill.own = own;
    return dim3(unsigned(own + share));
  };
  const auto next = [&](dim3 g) { fill.first += g.x - fill.own; };
  if (p.small) {
    const dim3 g = grid(1);
    hipLaunchKernelGGL(k_sort_small, g, dim3(kSortThreads), 0, stream, A.ids, int32_t(A.n), A.nodes,
                       p.passes, p.digit, to, fill);
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
  S.by_tile = few ? int64_t(1) << p.digit : 1;
  S.by_digit = few ? 1 : p.tiles;
  S.totals = few ? nullptr : reinterpret_cast<uint32_t *>(ws + p.totals);
  for (int pass = 0; pass < p.passes; ++pass) {
    S.shift = pass * p.digit;
    S.to = to;
    dim3 g = grid(p.tiles);
    S.fill = fill;
    hipLaunchKernelGGL(k_sort_count, g, dim3(kSortThreads), 0, stream, S);
    next(g);
    if (!few) hipLaunchKernelGGL(k_sort_scan, dim3(1u << p.digit), dim3(kBlock), 0, stream, S);
    g = grid(p.tiles);
    S.fill = fill;
    hipLaunchKernelGGL(k_sort_place, g, dim3(kSortThreads), 0, stream, S);
    next(g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    S.ids = nullptr;
    S.from = to;
    std::swap(to, other);
  }
  *sorted = S.from;
  return hipSuccess;
}

// Zeros alone.
__global__ __launch_bounds__(kBlock) void k_fill(Fill fill) { filled(fill); }

template <typename T, typename O, bool kAdd>
hipError_t gradient(const hg_embed_grad_args &A, hipStream_t stream) {
  Fill fill{A.dtable, A.dtable_stride, A.nodes, A.dim, int32_t(sizeof(O)), 0, 0, 0};
  int64_t pieces = 0;
  if (!kAdd) {
    const int64_t row = A.dim * int64_t(sizeof(O));
    // (a launch has fewer than 2^32 threads, of 1024 in a block; as one, 2^21 pieces are 128 GB)
    const int64_t most = int64_t(1) << 21;
    if ((A.nodes == 1 || A.dtable_stride == A.dim) && A.nodes <= most * kFillBytes / row) {
      pieces = ceil_div<int64_t>(A.nodes * row, kFillBytes);
    } else {
      fill.rows_of_piece =
          std::max(ceil_div<int64_t>(A.nodes, most), std::max<int64_t>(1, kFillBytes / row));
      pieces = ceil_div<int64_t>(A.nodes, fill.rows_of_piece);
    }
  }
  if (A.n == 0) {
    if (pieces > 0)
      hipLaunchKernelGGL(k_fill, dim3(unsigned(pieces)), dim3(kBlock), 0, stream, fill);
    return hipGetLastError();
  }
  const EmbedPlan p = embed_plan(A.n, A.nodes, A.dim);
  char *const ws = static_cast<char *>(A.workspace);
  Sums S{};
  hipError_t e = sort(A, p, fill, pieces, stream, &S.pairs);
  if (e != hipSuccess) return e;
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
  S.ends = reinterpret_cast<int32_t *>(ws + p.ends);
  const int64_t vectors = ceil_div<int64_t>(A.dim, kVec<T>);
  int64_t lanes = 8;
  while (lanes < vectors && lanes < kBlock) lanes *= 2;
  S.slices = ceil_div<int64_t>(vectors, lanes);
  S.blocks = ceil_div<int64_t>(p.chunks, kBlock / lanes) * S.slices;
  const dim3 grid(unsigned(std::min(S.blocks, kMostBlocks))), block(kBlock);
  switch (lanes) {
    case 8: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 8>), grid, block, 0, stream, S); break;
    case 16: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 16>), grid, block, 0, stream, S); break;
    case 32: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 32>), grid, block, 0, stream, S); break;
    case 64: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 64>), grid, block, 0, stream, S); break;
    case 128: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 128>), grid, block, 0, stream, S); break;
    default: hipLaunchKernelGGL((k_embed_sum<T, O, kAdd, 256>), grid, block, 0, stream, S);
  }
  e = hipGetLastError();
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

int64_t embed_grad_workspace(int64_t n, int64_t nodes, int64_t dim) {
  return n > 0 ? embed_plan(n, nodes, dim).total : 0;
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

// bf_embed.cu -- the token embedding out_t = scale * W[id_t] and its gradient
// dW_v = scale * sum over t with id_t = v of dout_t.
//
// The gradient sorts the positions by token (stable: by token, then position)
// and sums each token's rows in that order, so its result does not depend on
// when blocks run, and a token that fills half of the batch costs no more than
// others: tiles of kTile sorted positions are summed apart, the tokens that lie
// within one tile are written, and one that goes on in the next leaves a
// partial row, which the last kernel adds up.  Both directions are bound by
// memory: every thread moves 16 bytes at a time where the rows allow it.
#include "bf_elem.cuh"
#include "bf_launches.cuh"
#include "bf_learn.h"

namespace bfk {

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kTile = 32;  // sorted positions summed by one group of lanes

// Sixteen bytes, still as read.
template <typename E>
__device__ __forceinline__ void add_to(float* sum, const uint4& u) {
  float2 v[Vec<E>::kWidth / 2];
  unpack<E>(u, v);
#pragma unroll
  for (uint32_t i = 0; i < Vec<E>::kWidth; ++i) sum[i] += i % 2 ? v[i / 2].y : v[i / 2].x;
}
template <int N>
__device__ __forceinline__ void read_floats(const float* p, float* f) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 v = *reinterpret_cast<const float4*>(p + i);
    f[i] = v.x;
    f[i + 1] = v.y;
    f[i + 2] = v.z;
    f[i + 3] = v.w;
  }
}
// N neighbouring elements from 32-bit values, where they make up whole vectors or half of one.
template <typename E, int N>
__device__ __forceinline__ void write_n(E* p, const float* f) {
  if constexpr (N * sizeof(E) == 16) {
    float2 v[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = make_float2(f[2 * i], f[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = pack<E>(v);
  } else if constexpr (N * sizeof(E) == 32) {
    write_n<E, N / 2>(p, f);
    write_n<E, N / 2>(p + N / 2, f + N / 2);
  } else {
    static_assert(N * sizeof(E) == 8, "a half, one or two vectors");
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(make_float2(f[0], f[1]), E()), pack2(make_float2(f[2], f[3]), E()));
  }
}

// ---- forward: kPieces pieces of N elements a thread, all read before the first is written ----
//
// Bound by memory: 16,384 rows of 2,048 bf16 21 us, 6.4 TB/s (1 piece a thread 27 us, 4 27, 8 39);
// rows of 2,047, which start at any element, 35 us (75 us element by element).

constexpr uint32_t kPieces = 2;

template <typename E>
__device__ __forceinline__ uint4 scaled(const uint4& u, float scale) {
  float2 f[Vec<E>::kWidth / 2];
  unpack<E>(u, f);
#pragma unroll
  for (uint32_t i = 0; i < Vec<E>::kWidth / 2; ++i) f[i] = make_float2(f[i].x * scale, f[i].y * scale);
  return pack<E>(f);
}

// `aligned`: every row of both matrices is a row of 16-byte vectors; else a piece
// is one of the output row's vectors, wherever its elements lie in the table's row.
template <typename E, bool aligned, typename I>
__global__ void __launch_bounds__(kThreads) embed_kernel(const EmbedArgs a, I pieces, uint32_t per_row) {
  const I first = (I)blockIdx.x * (kThreads * kPieces) + threadIdx.x;
  I row[kPieces];
  int64_t id[kPieces];
  Unaligned<E> u[kPieces] = {};
  const Extent all(static_cast<const E*>(a.src), a.vocab, a.lds, a.width);
#pragma unroll
  for (uint32_t k = 0; k < kPieces; ++k) {
    row[k] = (first + k * kThreads) / per_row;
    id[k] = first + k * kThreads < pieces ? a.tokens[row[k]] : -1;
  }
#pragma unroll
  for (uint32_t k = 0; k < kPieces; ++k) {
    const uint32_t v = (uint32_t)(first + k * kThreads - row[k] * per_row);
    if (id[k] < 0 || id[k] >= (int64_t)a.vocab) continue;
    const E* w = static_cast<const E*>(a.src) + (uint64_t)id[k] * a.lds;
    if constexpr (aligned) {
      u[k].lo = *reinterpret_cast<const uint4*>(w + (uint64_t)v * Vec<E>::kWidth);
    } else {
      const Window<E> o(static_cast<E*>(a.dst) + (uint64_t)row[k] * a.ldd, a.width);
      if (v < o.vectors) u[k].load(w, a.width, (int64_t)v * Vec<E>::kWidth - o.shift, all);
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < kPieces; ++k) {
    if (first + k * kThreads >= pieces) continue;
    const uint32_t v = (uint32_t)(first + k * kThreads - row[k] * per_row);
    E* out = static_cast<E*>(a.dst) + (uint64_t)row[k] * a.ldd;
    const uint32_t nan = sizeof(E) == 4 ? 0x7FC00000u : 0x7FFF7FFFu;  // a NaN in each 16-bit type too
    const uint4 f = id[k] >= (int64_t)a.vocab ? make_uint4(nan, nan, nan, nan) : scaled<E>(u[k].take(), a.scale);
    if constexpr (aligned) *reinterpret_cast<uint4*>(out + (uint64_t)v * Vec<E>::kWidth) = f;
    else Window<E>(out, a.width).put(v, f);
  }
}

// ---- sort by token: 9 bits a pass, a count and a placing kernel each ----
//
// Bound by waiting (16,384 tokens of 131,072: two passes), so it runs beside the
// clearing of the gradient, which takes 80 us there; a pass of 81,920 tokens of
// 500 takes 4 + 10 us.

constexpr uint32_t kBits = 9, kBins = 1u << kBits, kSortThreads = kBins;
constexpr uint32_t kMaxSortTiles = 128;

struct SortArgs {
  const int64_t* tokens;  // first pass: keys are made from these
  const uint32_t *key_in, *pos_in;
  uint32_t *key_out, *pos_out;
  uint32_t* hist;  // a row of kBins counts per tile
  uint32_t* runs;  // first pass clears it: number of runs over several tiles
  uint32_t rows, tiles, tile, shift, vocab;
  // rows of the table's gradient that this launch's other blocks clear
  void* fill;
  uint64_t ld;
  uint32_t fill_first, fill_end, width;
};

// Tokens outside the vocabulary sort behind it, as `vocab`.
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, uint32_t i) {
  if (!a.tokens) return a.key_in[i];
  const int64_t id = a.tokens[i];
  return id >= 0 && id < (int64_t)a.vocab ? (uint32_t)id : a.vocab;
}

// Clearing the gradient takes longer than sorting the positions, and the sort
// fills a few blocks only: its launches' other blocks clear, a warp per row.
template <typename D>
__device__ __forceinline__ void fill_rows(const SortArgs& a) {
  const uint32_t warps = (gridDim.x - a.tiles) * (kSortThreads / 32), lane = threadIdx.x % 32;
  for (uint64_t row = a.fill_first + (blockIdx.x - a.tiles) * (kSortThreads / 32) + threadIdx.x / 32; row < a.fill_end;
       row += warps) {
    const Window<D> w(static_cast<D*>(a.fill) + row * a.ld, a.width);
    for (uint32_t v = lane; v < w.vectors; v += 32) w.store(v, make_uint4(0, 0, 0, 0));
  }
}

template <typename D>
__global__ void __launch_bounds__(kSortThreads) sort_count(const SortArgs a) {
  let_next_start();
  if (blockIdx.x >= a.tiles) {
    fill_rows<D>(a);
    return;
  }
  __shared__ uint32_t bins[kBins];
  bins[threadIdx.x] = 0;
  wait_for_previous();
  if (a.tokens && blockIdx.x == 0 && threadIdx.x == 0) *a.runs = 0;
  __syncthreads();
  const uint32_t first = blockIdx.x * a.tile, end = min(a.rows, first + a.tile);
  for (uint32_t i = first + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&bins[(key_of(a, i) >> a.shift) % kBins], 1u);
  __syncthreads();
  a.hist[blockIdx.x * kBins + threadIdx.x] = bins[threadIdx.x];
}

template <typename D>
__global__ void __launch_bounds__(kSortThreads) sort_place(const SortArgs a) {
  constexpr uint32_t kWarps = kSortThreads / 32;
  let_next_start();
  if (blockIdx.x >= a.tiles) {
    fill_rows<D>(a);
    return;
  }
  __shared__ uint32_t next[kBins];           // where the tile's next item of each digit goes
  __shared__ uint16_t ahead[kWarps][kBins];  // items of a digit in the round's earlier warps
  __shared__ uint32_t warp_sum[kWarps];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  wait_for_previous();
  // Thread d: the digit's items in all tiles and in those before this one.
  uint32_t all = 0, before = 0;
#pragma unroll 16
  for (uint32_t t = 0; t < a.tiles; ++t) {
    const uint32_t n = a.hist[t * kBins + threadIdx.x];
    all += n;
    before += t < blockIdx.x ? n : 0;
  }
  uint32_t sum = all;
#pragma unroll
  for (uint32_t o = 1; o < 32; o *= 2) {
    const uint32_t up = __shfl_up_sync(~0u, sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 31) warp_sum[warp] = sum;
  __syncthreads();
  for (uint32_t w = 0; w < warp; ++w) sum += warp_sum[w];
  next[threadIdx.x] = sum - all + before;
  const uint32_t first = blockIdx.x * a.tile, end = min(a.rows, first + a.tile);
  for (uint32_t base = first; base < end; base += kSortThreads) {
    const uint32_t i = base + threadIdx.x;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) ahead[w][threadIdx.x] = 0;
    __syncthreads();
    const bool in = i < end;
    const uint32_t key = in ? key_of(a, i) : 0, digit = in ? (key >> a.shift) % kBins : kBins;
    const uint32_t pos = in && !a.tokens ? a.pos_in[i] : i;
    const uint32_t same = __match_any_sync(~0u, digit), rank = __popc(same & ((1u << lane) - 1));
    if (in && rank == 0) ahead[warp][digit] = (uint16_t)__popc(same);
    __syncthreads();
    uint32_t count = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) {  // thread d: digit d over the warps
      const uint32_t n = ahead[w][threadIdx.x];
      ahead[w][threadIdx.x] = (uint16_t)count;
      count += n;
    }
    __syncthreads();
    if (in) {
      const uint32_t to = next[digit] + ahead[warp][digit] + rank;
      a.key_out[to] = key;
      a.pos_out[to] = pos;
    }
    __syncthreads();
    next[threadIdx.x] += count;
  }
}

// Up to kSmallSort positions: all passes in one block, the keys in shared memory.
constexpr uint32_t kSmallSort = 2 * kSortThreads;

template <typename D>
__global__ void __launch_bounds__(kSortThreads) sort_small(const SortArgs a) {
  constexpr uint32_t kWarps = kSortThreads / 32;
  let_next_start();
  if (blockIdx.x >= a.tiles) {
    fill_rows<D>(a);
    return;
  }
  __shared__ uint32_t key[2][kSmallSort], next[kBins], warp_sum[kWarps];
  __shared__ uint16_t pos[2][kSmallSort], ahead[kWarps][kBins];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) *a.runs = 0;
  for (uint32_t i = threadIdx.x; i < a.rows; i += kSortThreads) {
    key[0][i] = key_of(a, i);
    pos[0][i] = (uint16_t)i;
  }
  uint32_t from = 0;
  for (uint32_t shift = 0; shift == 0 || (shift < 32 && (a.vocab >> shift)); shift += kBits, from = 1 - from) {
    next[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < a.rows; i += kSortThreads) atomicAdd(&next[(key[from][i] >> shift) % kBins], 1u);
    __syncthreads();
    const uint32_t all = next[threadIdx.x];
    uint32_t sum = all;
#pragma unroll
    for (uint32_t o = 1; o < 32; o *= 2) {
      const uint32_t up = __shfl_up_sync(~0u, sum, o);
      if (lane >= o) sum += up;
    }
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    for (uint32_t w = 0; w < warp; ++w) sum += warp_sum[w];
    next[threadIdx.x] = sum - all;
    for (uint32_t base = 0; base < a.rows; base += kSortThreads) {
      const uint32_t i = base + threadIdx.x;
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) ahead[w][threadIdx.x] = 0;
      __syncthreads();
      const bool in = i < a.rows;
      const uint32_t k = in ? key[from][i] : 0, digit = in ? (k >> shift) % kBins : kBins;
      const uint32_t same = __match_any_sync(~0u, digit), rank = __popc(same & ((1u << lane) - 1));
      if (in && rank == 0) ahead[warp][digit] = (uint16_t)__popc(same);
      __syncthreads();
      uint32_t count = 0;
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) {
        const uint32_t n = ahead[w][threadIdx.x];
        ahead[w][threadIdx.x] = (uint16_t)count;
        count += n;
      }
      __syncthreads();
      if (in) {
        const uint32_t to = next[digit] + ahead[warp][digit] + rank;
        key[1 - from][to] = k;
        pos[1 - from][to] = pos[from][i];
      }
      __syncthreads();
      next[threadIdx.x] += count;
    }
    __syncthreads();
  }
  for (uint32_t i = threadIdx.x; i < a.rows; i += kSortThreads) {
    a.key_out[i] = key[from][i];
    a.pos_out[i] = pos[from][i];
  }
}

// ---- sums by token ----

struct SumArgs {
  EmbedArgs e;
  const uint32_t *key, *pos;
  float* partial;   // per tile: the part of a token that began before it, and of one that goes on after it
  uint32_t* runs;   // number of tokens that go on after the tile they began in, then their tiles, in any order
  uint32_t tiles;
  uint32_t part_width;  // the width, up to whole vectors
};

// N values to columns of a row that starts anywhere, the first `count` of them: two 16-bit ones a store where they share a word.
template <typename D, int N, int first>
__device__ __forceinline__ void write_pairs(D* p, const float* f, uint32_t count) {
  if (first == 1 && count > 0) p[0] = from_f32<D>(f[0]);
#pragma unroll
  for (int j = first; j < N; j += 2) {
    if (j + 1 < N && j + 1 < (int)count) *reinterpret_cast<uint32_t*>(p + j) = pack2(make_float2(f[j], f[j + 1]), D());
    else if (j < (int)count) p[j] = from_f32<D>(f[j]);
  }
}
template <typename D, int N>
__device__ __forceinline__ void write_some(D* p, const float* f, uint32_t count) {
  if constexpr (sizeof(D) == 4) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < (int)count) p[j] = f[j];
  } else {
    if ((uintptr_t)p % 4) write_pairs<D, N, 1>(p, f, count);
    else write_pairs<D, N, 0>(p, f, count);
  }
}

template <typename D, int N, bool aligned>
__device__ __forceinline__ void put_sum(const SumArgs& a, uint32_t key, uint32_t c, float* sum) {
  D* out = static_cast<D*>(a.e.dst) + (uint64_t)key * a.e.ldd + c;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    sum[j] *= a.e.scale;
    if (a.e.accumulate && (aligned || c + j < a.e.width)) sum[j] += to_f32(out[j]);
  }
  if constexpr (aligned) write_n<D, N>(out, sum);
  else write_some<D, N>(out, sum, a.e.width - c);
}

// `lanes` threads per tile, N columns a thread at a time; kAhead rows are read
// before they are added, whatever tokens they belong to.  81,920 rows of 256 f32
// 17 us, 4.9 TB/s; 16,384 rows of 2,048 bf16 23 us beside 8,500 rows written.
// Tiles of 16 or 64 positions: the same within 2 us.  Rows that start anywhere
// (not `aligned`): 16,384 rows of 2,047 bf16 into 131,072, whole gradient 139 us (169 us
// element by element, 107 us aligned).
template <typename S, typename D, bool aligned>
__global__ void __launch_bounds__(kThreads, sizeof(S) == 2 ? 3 : 4) sum_kernel(const SumArgs a, uint32_t lanes) {
  constexpr int N = Vec<S>::kWidth;
  constexpr uint32_t kAhead = aligned ? 8 : 4;
  const Extent all(static_cast<const S*>(a.e.src), a.e.rows, a.e.lds, a.e.width);
  __shared__ uint32_t keys[kThreads / 32 * (kTile + 2)];  // with the neighbours on both sides
  __shared__ uint32_t poss[kThreads / 32 * kTile];
  let_next_start();
  wait_for_previous();
  const uint32_t groups = kThreads / lanes, group = threadIdx.x / lanes, lane = threadIdx.x % lanes;
  const uint32_t rows = (uint32_t)a.e.rows, tile0 = blockIdx.x * groups;
  for (uint32_t i = threadIdx.x; i < groups * (kTile + 2); i += kThreads) {
    const int64_t at = (int64_t)(tile0 + i / (kTile + 2)) * kTile + i % (kTile + 2) - 1;
    keys[i] = at >= 0 && at < rows ? a.key[at] : 0xFFFFFFFFu;
  }
  for (uint32_t i = threadIdx.x; i < groups * kTile; i += kThreads) {
    const uint64_t at = (uint64_t)tile0 * kTile + i;
    poss[i] = at < rows ? a.pos[at] : 0;
  }
  __syncthreads();
  const uint32_t tile = tile0 + group;
  if (tile >= a.tiles) return;
  const uint32_t *key = keys + group * (kTile + 2) + 1, *pos = poss + group * kTile;
  const uint32_t count = min(kTile, rows - tile * kTile), last = key[count - 1];
  if (lane == 0 && last < a.e.vocab && key[count] == last && (key[0] != last || key[-1] != last))
    a.runs[1 + atomicAdd(a.runs, 1u)] = tile;
  float* part = a.partial + (uint64_t)tile * 2 * a.part_width;
  for (uint32_t c = lane * N; c < a.e.width; c += lanes * N) {
    float sum[N] = {};
    bool began = key[-1] != key[0];  // the token's first row lies in this tile
    for (uint32_t k = 0; k < count; k += kAhead) {
      Unaligned<S> piece[kAhead];
#pragma unroll
      for (uint32_t i = 0; i < kAhead; ++i) {
        piece[i].off = 0;
        if (k + i >= count || key[k + i] >= a.e.vocab) continue;
        const S* row = static_cast<const S*>(a.e.src) + (uint64_t)pos[k + i] * a.e.lds;
        if constexpr (aligned) piece[i].lo = *reinterpret_cast<const uint4*>(row + c);
        else piece[i].load(row, a.e.width, c, all);
      }
#pragma unroll
      for (uint32_t i = 0; i < kAhead; ++i) {
        if (k + i >= count || key[k + i] >= a.e.vocab) break;
        add_to<S>(sum, piece[i].take());
        if (key[k + i] == key[k + i + 1]) {
          if (k + i + 1 == count) write_n<float, N>(part + (began ? a.part_width : 0) + c, sum);
          continue;
        }
        if (began) put_sum<D, N, aligned>(a, key[k + i], c, sum);
        else write_n<float, N>(part + c, sum);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] = 0.0f;
        began = true;
      }
    }
  }
}

// Tokens over several tiles: a block adds up one's partial rows, in the tiles'
// order: each of its groups of `lanes` threads a stretch of them, then the stretches.
constexpr uint32_t kJoinThreads = 512;

template <typename D, int N, bool aligned>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const SumArgs a, uint32_t lanes) {
  constexpr uint32_t kAhead = 8;  // partial rows read before they are added
  __shared__ float stretch[kJoinThreads * N];
  wait_for_previous();
  const uint32_t groups = kJoinThreads / lanes, group = threadIdx.x / lanes, lane = threadIdx.x % lanes;
  const uint32_t runs = *a.runs;
  for (uint32_t r = blockIdx.x; r < runs; r += gridDim.x) {
    const uint32_t tile = a.runs[1 + r], key = a.key[(uint64_t)tile * kTile + kTile - 1];
    // The last tile that begins with this token: among the next 32, or by 32 probes at a time.
    const uint32_t near = tile + 1 + threadIdx.x % 32;
    const uint32_t other = __ballot_sync(~0u, near >= a.tiles || a.key[(uint64_t)near * kTile] != key);
    uint32_t lo = tile + (other ? __ffs(other) - 1 : 32), hi = other ? lo + 1 : a.tiles;
    while (hi - lo > 1) {
      const uint32_t step = (hi - lo + 31) / 32, probe = lo + threadIdx.x % 32 * step;
      const uint32_t at_most = __ballot_sync(~0u, probe == lo || (probe < hi && a.key[(uint64_t)probe * kTile] <= key));
      lo += (31 - __clz(at_most)) * step;
      hi = min(hi, lo + step);
    }
    const uint32_t each = (lo - tile + groups - 1) / groups, first = tile + 1 + group * each, end = min(lo + 1, first + each);
    for (uint32_t c0 = 0; c0 < a.e.width; c0 += lanes * N) {
      const uint32_t c = c0 + lane * N;
      float sum[N] = {};
      if (c < a.e.width) {
        for (uint32_t t = first; t < end; t += kAhead) {
          float f[kAhead][N] = {};
#pragma unroll
          for (uint32_t i = 0; i < kAhead; ++i)
            if (t + i < end) read_floats<N>(a.partial + (uint64_t)(t + i) * 2 * a.part_width + c, f[i]);
#pragma unroll
          for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += f[i][j];
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < N; ++j) stretch[j * kJoinThreads + threadIdx.x] = sum[j];
      __syncthreads();
      if (group == 0 && c < a.e.width) {
        read_floats<N>(a.partial + ((uint64_t)tile * 2 + 1) * a.part_width + c, sum);
        for (uint32_t g = 0; g < groups; ++g)
#pragma unroll
          for (int j = 0; j < N; ++j) sum[j] += stretch[j * kJoinThreads + g * lanes + lane];
        put_sum<D, N, aligned>(a, key, c, sum);
      }
    }
  }
}

uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }
uint32_t div_up(uint64_t a, uint32_t b) { return (uint32_t)((a + b - 1) / b); }

// Whether every row of a matrix allows pieces of 16 bytes of type size `size`.
bool rows_of_16(const void* p, uint64_t ld, uint32_t width, uint32_t size) {
  return ((uintptr_t)p | (ld * size) | (uint64_t)width * size) % 16 == 0;
}

template <typename S, typename D, bool aligned>
cudaError_t launch_sums(const SumArgs& a, cudaStream_t st) {
  constexpr int N = Vec<S>::kWidth;
  uint32_t lanes = 32;
  while (lanes < kThreads && lanes * N < a.e.width) lanes *= 2;
  cudaError_t e = launch_after(sum_kernel<S, D, aligned>, div_up(a.tiles, kThreads / lanes), kThreads, st, a, lanes);
  if (e != cudaSuccess) return e;
  const uint32_t blocks = a.tiles < 608 ? a.tiles : 608;
  return launch_after(join_kernel<D, N, aligned>, blocks, kJoinThreads, st, a, lanes);
}

// Columns of a partial row: whole vectors of 16-bit elements.
uint32_t part_width(uint32_t width) { return div_up(width, 8) * 8; }

template <typename S, typename D>
cudaError_t launch_grad(const EmbedArgs& a, void* workspace, cudaStream_t st) {
  char* at = static_cast<char*>(workspace);
  const auto take = [&](uint64_t bytes) {
    char* p = at;
    at += align256(bytes);
    return p;
  };
  const uint32_t rows = (uint32_t)a.rows, tiles = div_up(rows, kTile);
  SortArgs s = {};
  s.rows = rows;
  s.vocab = a.vocab;
  s.tile = div_up(div_up(rows, kMaxSortTiles), kSortThreads) * kSortThreads;
  if (s.tile < 2 * kSortThreads) s.tile = 2 * kSortThreads;
  s.tiles = div_up(rows, s.tile);
  s.fill = a.dst;
  s.ld = a.ldd;
  s.width = a.width;
  uint32_t *key[2] = {}, *pos[2] = {};
  if (rows) {
    for (uint32_t k = 0; k < 2; ++k) {
      key[k] = (uint32_t*)take(4 * a.rows);
      pos[k] = (uint32_t*)take(4 * a.rows);
    }
    s.hist = (uint32_t*)take(4ull * kBins * kMaxSortTiles);
    s.runs = (uint32_t*)take(4ull * (tiles + 1));
  }
  uint32_t passes = rows ? 1 : 0;
  while (passes && passes * kBits < 32 && (a.vocab >> (passes * kBits))) ++passes;
  const bool small = rows && rows <= kSmallSort;
  const uint32_t launches = passes && !small ? 2 * passes : 1;
  const uint64_t fill_bytes = a.accumulate ? 0 : (uint64_t)a.vocab * a.width * sizeof(D);
  const uint64_t most = fill_bytes / launches / (16 * kSortThreads) + 1;  // blocks with 16 bytes a thread to clear
  const uint32_t fillers = a.accumulate ? 0 : most < 456 ? (uint32_t)most : 456;
  uint32_t from = 0;
  for (uint32_t l = 0; l < launches; ++l) {
    s.tokens = l < 2 ? a.tokens : nullptr;
    s.shift = l / 2 * kBits;
    s.key_in = key[from];
    s.pos_in = pos[from];
    s.key_out = key[1 - from];
    s.pos_out = pos[1 - from];
    s.fill_first = (uint32_t)((uint64_t)a.vocab * l / launches);
    s.fill_end = (uint32_t)((uint64_t)a.vocab * (l + 1) / launches);
    if (s.tiles + fillers == 0) continue;
    // The first launch waits for all earlier work: the gradient may be in use.
    const cudaError_t e = small  ? launch_plain(sort_small<D>, s.tiles + fillers, kSortThreads, st, s)
                          : l == 0 ? launch_plain(sort_count<D>, s.tiles + fillers, kSortThreads, st, s)
                          : l % 2 ? launch_after(sort_place<D>, s.tiles + fillers, kSortThreads, st, s)
                                  : launch_after(sort_count<D>, s.tiles + fillers, kSortThreads, st, s);
    if (e != cudaSuccess) return e;
    if (small || l % 2) from = 1 - from;
  }
  if (rows == 0) return cudaSuccess;
  const SumArgs m = {a, key[from], pos[from], (float*)at, s.runs, tiles, part_width(a.width)};
  const bool aligned = rows_of_16(a.src, a.lds, a.width, sizeof(S)) && rows_of_16(a.dst, a.ldd, a.width, sizeof(D));
  return aligned ? launch_sums<S, D, true>(m, st) : launch_sums<S, D, false>(m, st);
}

template <typename S>
cudaError_t launch_grad_from(const EmbedArgs& a, void* workspace, cudaStream_t st) {
  switch (a.dst_dtype) {
    case BF_BF16: return launch_grad<S, __nv_bfloat16>(a, workspace, st);
    case BF_F16: return launch_grad<S, __half>(a, workspace, st);
    default: return launch_grad<S, float>(a, workspace, st);
  }
}

template <typename E, bool aligned>
cudaError_t launch_embed_pieces(const EmbedArgs& a, cudaStream_t st) {
  const uint32_t per_row = div_up(a.width + (aligned ? 0 : Vec<E>::kWidth - 1), Vec<E>::kWidth);
  const uint64_t pieces = a.rows * per_row, blocks = (pieces + kThreads * kPieces - 1) / (kThreads * kPieces);
  if (blocks > 0x7FFFFFFFu) return cudaErrorInvalidValue;
  if (pieces + kThreads * kPieces < (1ull << 32))
    return launch_plain(embed_kernel<E, aligned, uint32_t>, (uint32_t)blocks, kThreads, st, a, (uint32_t)pieces, per_row);
  return launch_plain(embed_kernel<E, aligned, uint64_t>, (uint32_t)blocks, kThreads, st, a, pieces, per_row);
}

template <typename E>
cudaError_t launch_embed_typed(const EmbedArgs& a, cudaStream_t st) {
  return rows_of_16(a.src, a.lds, a.width, sizeof(E)) && rows_of_16(a.dst, a.ldd, a.width, sizeof(E))
             ? launch_embed_pieces<E, true>(a, st) : launch_embed_pieces<E, false>(a, st);
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs& a, cudaStream_t st) {
  switch (a.src_dtype) {
    case BF_BF16: return launch_embed_typed<__nv_bfloat16>(a, st);
    case BF_F16: return launch_embed_typed<__half>(a, st);
    default: return launch_embed_typed<float>(a, st);
  }
}

uint64_t embed_grad_bytes(uint64_t rows, uint32_t width) {
  if (rows == 0) return 0;
  const uint64_t tiles = (rows + kTile - 1) / kTile;
  return 4 * align256(4 * rows) + align256(4ull * kBins * kMaxSortTiles) + align256(4 * (tiles + 1)) +
         align256(4 * 2 * tiles * part_width(width));
}

cudaError_t launch_embed_grad(const EmbedArgs& a, void* workspace, cudaStream_t st) {
  switch (a.src_dtype) {
    case BF_BF16: return launch_grad_from<__nv_bfloat16>(a, workspace, st);
    case BF_F16: return launch_grad_from<__half>(a, workspace, st);
    default: return launch_grad_from<float>(a, workspace, st);
  }
}

}  // namespace bfk

// bf_embed.cu -- the token embedding out_t = scale * W[id_t] and its gradient
// dW_v = scale * sum over t with id_t = v of dout_t.
//
// The gradient sorts the positions by token (stable: by token, then position)
// and sums each token's rows in that order, so its result does not depend on
// when blocks run, and a token that fills half of the batch costs no more than
// others: a block sums kTile sorted positions, writes the tokens that lie
// within its tile and leaves a partial row for one that goes on in the next.
#include "bf_elem.cuh"
#include "bf_learn.h"

namespace bfk {

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kTile = 32;        // sorted positions summed by a block
constexpr uint32_t kSortTile = 1024;  // positions counted and placed by a block
constexpr uint32_t kBins = 256;       // 8 bits of the token a pass

template <typename S, typename D>
__global__ void __launch_bounds__(kThreads) embed_kernel(const EmbedArgs a) {
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t id = a.tokens[row];
    D* out = static_cast<D*>(a.dst) + row * a.ldd;
    const bool in = id >= 0 && id < (int64_t)a.vocab;
    const float other = id < 0 ? 0.0f : __int_as_float(0x7FC00000);
    const S* w = static_cast<const S*>(a.src) + (in ? (uint64_t)id : 0) * a.lds;
    for (uint32_t c = threadIdx.x; c < a.width; c += kThreads)
      out[c] = from_f32<D>(in ? to_f32(w[c]) * a.scale : other);
  }
}

// ---- sort by token ----

struct SortArgs {
  const int64_t* tokens;  // first pass: keys are made from these
  const uint32_t *key_in, *pos_in;
  uint32_t *key_out, *pos_out;
  uint32_t* hist;  // kBins rows of `tiles`
  uint32_t rows, tiles, shift, vocab;
};

// Tokens outside the vocabulary sort behind it, as `vocab`.
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, uint32_t i) {
  if (!a.tokens) return a.key_in[i];
  const int64_t id = a.tokens[i];
  return id >= 0 && id < (int64_t)a.vocab ? (uint32_t)id : a.vocab;
}

__global__ void __launch_bounds__(kThreads) sort_count(const SortArgs a) {
  __shared__ uint32_t bins[kBins];
  bins[threadIdx.x] = 0;
  __syncthreads();
  for (uint32_t k = threadIdx.x; k < kSortTile; k += kThreads) {
    const uint32_t i = blockIdx.x * kSortTile + k;
    if (i < a.rows) atomicAdd(&bins[(key_of(a, i) >> a.shift) % kBins], 1u);
  }
  __syncthreads();
  a.hist[threadIdx.x * a.tiles + blockIdx.x] = bins[threadIdx.x];
}

// Exclusive sums of the counts in place, digit by digit and tile by tile; one block.
__global__ void __launch_bounds__(1024) sort_scan(uint32_t* hist, uint32_t n) {
  __shared__ uint32_t warp_sum[32];
  uint32_t before = 0;
  for (uint32_t base = 0; base < n; base += 1024) {
    const uint32_t i = base + threadIdx.x, lane = threadIdx.x % 32;
    const uint32_t v = i < n ? hist[i] : 0;
    uint32_t sum = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t up = __shfl_up_sync(~0u, sum, o);
      if (lane >= (uint32_t)o) sum += up;
    }
    if (lane == 31) warp_sum[threadIdx.x / 32] = sum;
    __syncthreads();
    uint32_t ahead = 0, total = 0;
    for (uint32_t w = 0; w < 32; ++w) {
      if (w < threadIdx.x / 32) ahead += warp_sum[w];
      total += warp_sum[w];
    }
    if (i < n) hist[i] = before + ahead + sum - v;
    before += total;
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kThreads) sort_place(const SortArgs a) {
  __shared__ uint32_t next[kBins];                   // where the tile's next item of each digit goes
  __shared__ uint32_t ahead[kThreads / 32][kBins];   // items of a digit in the round's earlier warps
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  next[threadIdx.x] = a.hist[threadIdx.x * a.tiles + blockIdx.x];
  for (uint32_t k = 0; k < kSortTile; k += kThreads) {
    const uint32_t i = blockIdx.x * kSortTile + k + threadIdx.x;
    for (uint32_t w = 0; w < kThreads / 32; ++w) ahead[w][threadIdx.x] = 0;
    __syncthreads();
    const bool in = i < a.rows;
    const uint32_t key = in ? key_of(a, i) : 0, digit = in ? (key >> a.shift) % kBins : kBins;
    const uint32_t same = __match_any_sync(~0u, digit), rank = __popc(same & ((1u << lane) - 1));
    if (in && rank == 0) ahead[warp][digit] = __popc(same);
    __syncthreads();
    uint32_t sum = 0;
    for (uint32_t w = 0; w < kThreads / 32; ++w) {  // thread d: digit d over the warps
      const uint32_t n = ahead[w][threadIdx.x];
      ahead[w][threadIdx.x] = sum;
      sum += n;
    }
    __syncthreads();
    if (in) {
      const uint32_t to = next[digit] + ahead[warp][digit] + rank;
      a.key_out[to] = key;
      a.pos_out[to] = a.tokens ? i : a.pos_in[i];
    }
    __syncthreads();
    next[threadIdx.x] += sum;
  }
}

// ---- sums by token ----

struct SumArgs {
  EmbedArgs e;
  const uint32_t *key, *pos;
  float* partial;  // per tile: the part of a token that began before it, and of one that goes on after it
  uint32_t tiles;
};

template <typename D>
__device__ __forceinline__ void put_sum(const SumArgs& a, uint32_t key, uint32_t c, float sum) {
  D* out = static_cast<D*>(a.e.dst) + (uint64_t)key * a.e.ldd + c;
  sum *= a.e.scale;
  *out = from_f32<D>(a.e.accumulate ? to_f32(*out) + sum : sum);
}

template <typename S, typename D>
__global__ void __launch_bounds__(kThreads) sum_kernel(const SumArgs a) {
  __shared__ uint32_t key[kTile + 2];  // with the neighbours on both sides
  __shared__ uint32_t pos[kTile];
  const uint32_t rows = (uint32_t)a.e.rows, first = blockIdx.x * kTile, count = min(kTile, rows - first);
  for (uint32_t k = threadIdx.x; k < kTile + 2; k += kThreads) {
    const int64_t i = (int64_t)first + k - 1;
    key[k] = i >= 0 && i < rows && k < count + 2 ? a.key[i] : 0xFFFFFFFFu;
    if (k < count) pos[k] = a.pos[first + k];
  }
  __syncthreads();
  float* part = a.partial + (uint64_t)blockIdx.x * 2 * a.e.width;
  for (uint32_t c = threadIdx.x; c < a.e.width; c += kThreads) {
    float sum = 0.0f;
    bool began = key[0] != key[1];  // the token's first row lies in this tile
    for (uint32_t k = 0; k < count; ++k) {
      const uint32_t now = key[k + 1];
      if (now >= a.e.vocab) break;  // sorted behind all tokens
      sum += to_f32(static_cast<const S*>(a.e.src)[(uint64_t)pos[k] * a.e.lds + c]);
      if (now == key[k + 2]) {
        if (k + 1 == count) part[began ? a.e.width + c : c] = sum;
        continue;
      }
      if (began) put_sum<D>(a, now, c, sum);
      else part[c] = sum;
      sum = 0.0f;
      began = true;
    }
  }
}

// Tokens over several tiles: the block of the tile where one begins adds up its partial rows, in the tiles' order.
template <typename D>
__global__ void __launch_bounds__(kThreads) join_kernel(const SumArgs a) {
  const uint32_t rows = (uint32_t)a.e.rows, last = min(rows, (blockIdx.x + 1) * kTile) - 1, first = blockIdx.x * kTile;
  const uint32_t key = a.key[last];
  if (key >= a.e.vocab || last + 1 >= rows || a.key[last + 1] != key) return;       // ends here
  if (a.key[first] == key && first > 0 && a.key[first - 1] == key) return;          // began before
  for (uint32_t c = threadIdx.x; c < a.e.width; c += kThreads) {
    float sum = a.partial[((uint64_t)blockIdx.x * 2 + 1) * a.e.width + c];
    for (uint32_t t = blockIdx.x + 1; t < a.tiles && a.key[t * kTile] == key; ++t)
      sum += a.partial[(uint64_t)t * 2 * a.e.width + c];
    put_sum<D>(a, key, c, sum);
  }
}

uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

template <typename S, typename D>
cudaError_t launch_sums(const SumArgs& a, cudaStream_t st) {
  if (!a.e.accumulate) {
    cudaError_t e = cudaMemset2DAsync(a.e.dst, a.e.ldd * sizeof(D), 0, a.e.width * sizeof(D), a.e.vocab, st);
    if (e != cudaSuccess) return e;
  }
  if (a.e.rows == 0) return cudaSuccess;
  sum_kernel<S, D><<<a.tiles, kThreads, 0, st>>>(a);
  join_kernel<D><<<a.tiles, kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

template <typename S>
cudaError_t launch_sums_from(const SumArgs& a, cudaStream_t st) {
  switch (a.e.dst_dtype) {
    case BF_BF16: return launch_sums<S, __nv_bfloat16>(a, st);
    case BF_F16: return launch_sums<S, __half>(a, st);
    default: return launch_sums<S, float>(a, st);
  }
}

template <typename S>
cudaError_t launch_embed_typed(const EmbedArgs& a, cudaStream_t st) {
  const uint32_t grid = (uint32_t)(a.rows < (1u << 30) ? a.rows : (1u << 30));
  embed_kernel<S, S><<<grid, kThreads, 0, st>>>(a);
  return cudaGetLastError();
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
  const uint64_t sort_tiles = (rows + kSortTile - 1) / kSortTile, tiles = (rows + kTile - 1) / kTile;
  return 4 * align256(4 * rows) + align256(4 * kBins * sort_tiles) + align256(4 * 2 * tiles * width);
}

cudaError_t launch_embed_grad(const EmbedArgs& a, void* workspace, cudaStream_t st) {
  char* at = static_cast<char*>(workspace);
  const auto take = [&](uint64_t bytes) {
    char* p = at;
    at += align256(bytes);
    return p;
  };
  const uint32_t rows = (uint32_t)a.rows, sort_tiles = (rows + kSortTile - 1) / kSortTile;
  uint32_t* key[2] = {(uint32_t*)take(4 * a.rows), (uint32_t*)take(4 * a.rows)};
  uint32_t* pos[2] = {(uint32_t*)take(4 * a.rows), (uint32_t*)take(4 * a.rows)};
  uint32_t* hist = (uint32_t*)take(4ull * kBins * sort_tiles);
  uint32_t from = 0;
  for (uint32_t shift = 0; rows && (shift == 0 || (shift < 32 && (a.vocab >> shift))); shift += 8) {
    const SortArgs s = {shift == 0 ? a.tokens : nullptr, key[from], pos[from], key[1 - from], pos[1 - from], hist, rows,
                        sort_tiles, shift, a.vocab};
    sort_count<<<sort_tiles, kThreads, 0, st>>>(s);
    sort_scan<<<1, 1024, 0, st>>>(hist, kBins * sort_tiles);
    sort_place<<<sort_tiles, kThreads, 0, st>>>(s);
    from = 1 - from;
  }
  const SumArgs s = {a, key[from], pos[from], (float*)at, (rows + kTile - 1) / kTile};
  switch (a.src_dtype) {
    case BF_BF16: return launch_sums_from<__nv_bfloat16>(s, st);
    case BF_F16: return launch_sums_from<__half>(s, st);
    default: return launch_sums_from<float>(s, st);
  }
}

}  // namespace bfk

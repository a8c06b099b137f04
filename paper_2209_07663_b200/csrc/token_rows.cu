// Rows by token and their gradient (mono_token_rows, mono_token_rows_grad): kernels and host side.
#include <climits>

#include "operators.cuh"
#include "table_layout.cuh"

using namespace mono;

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------
// Rows by token.  out[i] = scale * weight[token i]: nothing is reused, so bytes bound it.
// A thread moves VEC columns at once and keeps four such moves in flight behind the read of its token(s): four pieces of one row
// where rows are wide, one piece of each of four rows where `lanes` threads cover a row.
// ---------------------------------------------------------------------------
constexpr int kMoves = 4;

template <typename W, typename O, int VEC, int ROWS>
__global__ void __launch_bounds__(kThreads) token_rows_kernel(const W* __restrict__ weight, int64_t weight_stride, TokenList tokens, float scale,
                                                              O* __restrict__ out, int64_t out_stride, int vectors, int lanes) {
  after_previous_kernel();
  constexpr int PIECES = kMoves / ROWS;
  const int lane = threadIdx.x & (lanes - 1), groups = kThreads / lanes;
  const int64_t row0 = (int64_t)blockIdx.x * groups * ROWS + threadIdx.x / lanes;
  const int v0 = blockIdx.y * lanes * PIECES + lane;
  uint32_t t[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int64_t i = row0 + r * groups;
    t[r] = i < tokens.n ? tokens.at(i) : kNoToken;
  }
  Vec<W, VEC> in[kMoves];
#pragma unroll
  for (int k = 0; k < kMoves; ++k) {
    const int r = k / PIECES, v = v0 + (k % PIECES) * lanes;
    if (t[r] != kNoToken && v < vectors) {
      in[k] = *reinterpret_cast<const Vec<W, VEC>*>(weight + t[r] * weight_stride + (int64_t)v * VEC);
    }
  }
#pragma unroll
  for (int k = 0; k < kMoves; ++k) {
    const int r = k / PIECES, v = v0 + (k % PIECES) * lanes;
    const int64_t i = row0 + r * groups;
    if (i >= tokens.n || v >= vectors) continue;
    Vec<O, VEC> o;
#pragma unroll
    for (int c = 0; c < VEC; ++c) o.v[c] = from_float<O>(t[r] != kNoToken ? scale * to_float(in[k].v[c]) : 0.0f);
    *reinterpret_cast<Vec<O, VEC>*>(out + i * out_stride + (int64_t)v * VEC) = o;
  }
}

template <typename W, typename O, int VEC>
int launch_token_rows(const mono_matrix_t& weight, const TokenList& tokens, float scale, const mono_matrix_t& out, cudaStream_t s) {
  const int vectors = (int)(weight.cols / VEC);
  const auto launch = [&](auto rows_of_a_thread, int lanes) {
    constexpr int ROWS = decltype(rows_of_a_thread)::value;
    const int64_t rows = (int64_t)(kThreads / lanes) * ROWS, columns = (int64_t)lanes * (kMoves / ROWS);
    const dim3 grid((unsigned)((tokens.n + rows - 1) / rows), (unsigned)((vectors + columns - 1) / columns));
    return launch_operator(token_rows_kernel<W, O, VEC, ROWS>, grid, kThreads, 0, s, static_cast<const W*>(weight.data), weight.stride, tokens, scale,
                           static_cast<O*>(out.data), out.stride, vectors, lanes);
  };
  int lanes = 1;
  if (vectors > 64) {
    while (lanes < kThreads && lanes * kMoves < vectors) lanes *= 2;
    return launch(Width<1>(), lanes);
  }
  while (lanes < vectors) lanes *= 2;
  return launch(Width<4>(), lanes);
}

// ---------------------------------------------------------------------------
// Gradient.  The tokens are sorted stably by row (radix sort, least digit first; tokens without a row last), so that
// the terms of a row are consecutive; the sorted positions are cut into chunks of kChunk, every chunk adds up its rows in order
// and writes those that begin and end in it.  What a row has in a chunk that it does not begin and end in is a partial
// sum in the workspace: `head` if it began in an earlier chunk, `tail` if it begins here; join_rows_kernel adds
// a row's tail and heads.  All orders follow from the sorted tokens, so the result has the same bits every time.
// ---------------------------------------------------------------------------
constexpr int kChunk = 64;
constexpr int kSortThreads = 256;
constexpr int kSortKeys = 8;                               // keys of a thread
constexpr int kSortTile = kSortThreads * kSortKeys;
constexpr int kMaxDigitBits = 9;
constexpr int kMaxDigits = 1 << kMaxDigitBits;
constexpr int kCoarse = 16;                                // tiles whose digit counts are also kept summed up

struct Entry { uint32_t row, at; };                        // a token's row (vocab: none) and its position

struct SortPlan {
  int passes, bits;                                        // digits of `bits` bits each
  int64_t tiles, coarse;
};

SortPlan plan_sort(int64_t n, int64_t vocab) {
  int width = 1;
  while (((uint64_t)vocab >> width) != 0) ++width;         // rows 0 .. vocab, the last one for tokens without a row
  SortPlan p;
  p.passes = (width + kMaxDigitBits - 1) / kMaxDigitBits;
  p.bits = (width + p.passes - 1) / p.passes;
  p.tiles = (n + kSortTile - 1) / kSortTile;
  p.coarse = (p.tiles + kCoarse - 1) / kCoarse;
  return p;
}

struct GradWorkspace {
  Entry* a;
  Entry* b;
  uint32_t* counts;        // [tiles][digits]
  uint32_t* coarse;        // [coarse][digits]
  float* partial;          // [chunks][2][cols]: head, tail
  int64_t bytes;
};

GradWorkspace carve(char* base, int64_t n, int64_t vocab, int64_t cols) {
  const SortPlan p = plan_sort(n, vocab);
  int64_t at = 0;
  const auto take = [&](int64_t bytes) { char* r = base + at; at += (bytes + 255) / 256 * 256; return r; };
  GradWorkspace w;
  w.a = reinterpret_cast<Entry*>(take(n * (int64_t)sizeof(Entry)));
  w.b = reinterpret_cast<Entry*>(take(n * (int64_t)sizeof(Entry)));
  w.counts = reinterpret_cast<uint32_t*>(take(p.tiles * kMaxDigits * 4));
  w.coarse = reinterpret_cast<uint32_t*>(take(p.coarse * kMaxDigits * 4));
  w.partial = reinterpret_cast<float*>(take((n + kChunk - 1) / kChunk * 2 * cols * 4));
  w.bytes = at;
  return w;
}

// The keys of a tile: from the caller's tokens in the first pass, from the pass before in the others.
struct Keys {
  TokenList tokens;
  const Entry* entries;    // nullptr: the tokens
  __device__ __forceinline__ Entry at(int64_t i) const {
    if (entries) return entries[i];
    const uint32_t t = tokens.at(i);
    return {t == kNoToken ? (uint32_t)tokens.vocab : t, (uint32_t)i};
  }
};

__global__ void __launch_bounds__(kSortThreads) count_digits_kernel(Keys keys, int64_t n, int shift, int bits, uint32_t* __restrict__ counts) {
  after_previous_kernel();
  __shared__ uint32_t count[kMaxDigits];
  const int digits = 1 << bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
#pragma unroll
  for (int k = 0; k < kSortKeys; ++k) {
    const int64_t i = base + k * kSortThreads + threadIdx.x;
    if (i < n) atomicAdd(&count[(keys.at(i).row >> shift) & (digits - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) counts[(int64_t)blockIdx.x * kMaxDigits + d] = count[d];
}

// counts summed over kCoarse tiles each
__global__ void __launch_bounds__(kSortThreads) sum_counts_kernel(const uint32_t* __restrict__ counts, int64_t tiles, int bits, uint32_t* __restrict__ coarse) {
  after_previous_kernel();
  const int64_t first = (int64_t)blockIdx.x * kCoarse, last = first + kCoarse < tiles ? first + kCoarse : tiles;
  for (int d = threadIdx.x; d < 1 << bits; d += kSortThreads) {
    uint32_t sum = 0;
    for (int64_t t = first; t < last; ++t) sum += counts[t * kMaxDigits + d];
    coarse[(int64_t)blockIdx.x * kMaxDigits + d] = sum;
  }
}

// Where the tile's keys of each digit go: the keys of lower digits of all tiles, then those of this digit of earlier tiles.
// Keys keep their order: warp w has the tile's keys [w * 256, (w + 1) * 256), 32 at a time, and a key's place among the equal digits of its 32 is
// what __match_any_sync says.
__global__ void __launch_bounds__(kSortThreads) scatter_keys_kernel(Keys keys, int64_t n, int shift, int bits, const uint32_t* __restrict__ counts,
                                                                    const uint32_t* __restrict__ coarse, int64_t n_coarse, Entry* __restrict__ sorted) {
  after_previous_kernel();
  constexpr int kWarps = kSortThreads / 32;
  __shared__ uint32_t next[kWarps][kMaxDigits];             // counts of the warps, then the place of a warp's next key of a digit
  __shared__ uint32_t warp_sum[kWarps];
  const int digits = 1 << bits, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t tile = blockIdx.x, base = tile * kSortTile + warp * (32 * kSortKeys);
  for (int d = threadIdx.x; d < kWarps * kMaxDigits; d += kSortThreads) next[0][d] = 0;
  __syncthreads();
  Entry e[kSortKeys];
#pragma unroll
  for (int k = 0; k < kSortKeys; ++k) {
    const int64_t i = base + k * 32 + lane;
    if (i < n) {
      e[k] = keys.at(i);
      atomicAdd(&next[warp][(e[k].row >> shift) & (digits - 1)], 1u);
    }
  }
  // of two digits each (neighbours, so that the scan runs in their order): all keys, and those of earlier tiles
  constexpr int kPer = kMaxDigits / kSortThreads;
  uint32_t total[kPer] = {}, before[kPer] = {};
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int d = threadIdx.x * kPer + j;
    if (d >= digits) continue;
    for (int64_t c = 0; c < n_coarse; ++c) {
      const uint32_t x = coarse[c * kMaxDigits + d];
      total[j] += x;
      if (c < tile / kCoarse) before[j] += x;
    }
    for (int64_t t = tile / kCoarse * kCoarse; t < tile; ++t) before[j] += counts[t * kMaxDigits + d];
  }
  uint32_t mine = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) mine += total[j];
  uint32_t scan = mine;
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, scan, s);
    if (lane >= s) scan += x;
  }
  if (lane == 31) warp_sum[warp] = scan;
  __syncthreads();
  uint32_t start = scan - mine;
  for (int w = 0; w < warp; ++w) start += warp_sum[w];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int d = threadIdx.x * kPer + j;
    uint32_t place = start + before[j];
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t c = next[w][d];
      next[w][d] = place;
      place += c;
    }
    start += total[j];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortKeys; ++k) {
    const bool there = base + k * 32 + lane < n;
    const uint32_t digit = there ? (e[k].row >> shift) & (digits - 1) : kMaxDigits;
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
    const uint32_t rank = __popc(same & ((1u << lane) - 1));
    uint32_t place = 0;
    if (there) place = next[warp][digit] + rank;
    __syncwarp();
    if (there && rank == 0) next[warp][digit] += __popc(same);
    __syncwarp();
    if (there && place < n) sorted[place] = e[k];
  }
}

template <typename O>
__global__ void __launch_bounds__(kThreads) zero_rows_kernel(O* __restrict__ out, int64_t stride, int64_t rows, int cols) {
  after_previous_kernel();
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < cols; c += kThreads) out[r * stride + c] = from_float<O>(0.0f);
}

template <typename O>
__device__ __forceinline__ O summed(O* at, float sum, float scale, bool accumulate) {
  return from_float<O>(accumulate ? to_float(*at) + scale * sum : scale * sum);
}

// A group of `lanes` threads (a power of two, up to a warp) has one chunk and the columns [first, end) of blockIdx.y's part, in
// vectors of VEC; a thread holds up to 8 columns' sums.
template <typename G, typename O, int VEC>
__global__ void __launch_bounds__(kThreads) sum_rows_kernel(const G* __restrict__ grad, int64_t grad_stride, const Entry* __restrict__ sorted, int64_t n, uint32_t vocab,
                                                            float scale, bool accumulate, O* __restrict__ out, int64_t out_stride, float* __restrict__ partial,
                                                            int cols, int part_vectors, int lanes) {
  after_previous_kernel();
  constexpr int R = 8 / VEC;
  constexpr int U = VEC >= 4 ? 8 : 4;                       // positions whose terms are in flight at once
  const int lane = threadIdx.x & (lanes - 1);
  const int64_t chunk = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes;
  const int64_t p0 = chunk * kChunk, p1 = p0 + kChunk < n ? p0 + kChunk : n;
  if (p0 >= n) return;
  const int first = blockIdx.y * part_vectors, end = min(first + part_vectors, cols / VEC);
  float sum[R][VEC] = {};
  uint32_t row = sorted[p0].row;
  if (row >= vocab) return;
  bool began_before = p0 > 0 && sorted[p0 - 1].row == row;

  const auto flush = [&](bool whole, float* to) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int v = first + lane + r * lanes;
      if (v < end) {
        if (whole) {
          O* at = out + row * out_stride + (int64_t)v * VEC;
          Vec<O, VEC> o, old;
          if (accumulate) old = *reinterpret_cast<const Vec<O, VEC>*>(at);
#pragma unroll
          for (int c = 0; c < VEC; ++c) o.v[c] = from_float<O>(accumulate ? to_float(old.v[c]) + scale * sum[r][c] : scale * sum[r][c]);
          *reinterpret_cast<Vec<O, VEC>*>(at) = o;
        } else {
#pragma unroll
          for (int c = 0; c < VEC; ++c) to[v * VEC + c] = sum[r][c];
        }
      }
#pragma unroll
      for (int c = 0; c < VEC; ++c) sum[r][c] = 0.0f;
    }
  };

  for (int64_t p = p0; p < p1; p += U) {
    Entry e[U];
    Vec<G, VEC> term[U][R];
#pragma unroll
    for (int u = 0; u < U; ++u) e[u] = p + u < p1 ? sorted[p + u] : Entry{vocab, 0};
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int v = first + lane + r * lanes;
        if (e[u].row < vocab && v < end) term[u][r] = *reinterpret_cast<const Vec<G, VEC>*>(grad + e[u].at * grad_stride + (int64_t)v * VEC);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (e[u].row >= vocab) continue;                     // behind the chunk's end or the last token with a row
      if (e[u].row != row) {
        flush(!began_before, partial + chunk * 2 * cols);
        row = e[u].row;
        began_before = false;
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (first + lane + r * lanes < end) {
#pragma unroll
          for (int c = 0; c < VEC; ++c) sum[r][c] += to_float(term[u][r].v[c]);
        }
      }
    }
  }
  const bool goes_on = p1 < n && sorted[p1].row == row;
  flush(!began_before && !goes_on, partial + (chunk * 2 + (began_before ? 0 : 1)) * cols);
}

// The block of a chunk in which a row begins that goes on behind it adds up the row's partial sums: `ways` of the block's threads
// take consecutive shares of them for each column, and the shares are added in order.
template <typename O>
__global__ void __launch_bounds__(kThreads) join_rows_kernel(const Entry* __restrict__ sorted, int64_t n, uint32_t vocab, float scale, bool accumulate, O* __restrict__ out,
                                                             int64_t out_stride, const float* __restrict__ partial, int cols, int lanes) {
  after_previous_kernel();
  __shared__ float share[kThreads];
  const int64_t chunk = blockIdx.x, p0 = chunk * kChunk, p1 = p0 + kChunk;
  if (p1 >= n) return;
  const uint32_t row = sorted[p1].row;
  if (row >= vocab || sorted[p1 - 1].row != row) return;
  if (sorted[p0].row == row && p0 > 0 && sorted[p0 - 1].row == row) return;       // began earlier
  // the chunks behind this one whose first token is of this row
  int64_t low = chunk + 1, high = (n + kChunk - 1) / kChunk;                      // (the first is; `high` is not)
  while (high - low > 1) {
    const int64_t mid = (low + high) / 2;
    if (sorted[mid * kChunk].row == row) low = mid; else high = mid;
  }
  const int64_t heads = low - chunk;
  const int ways = kThreads / lanes, way = threadIdx.x / lanes, lane = threadIdx.x % lanes;
  const int64_t per = (heads + ways - 1) / ways;
  const int64_t from = chunk + 1 + way * per, to = min(from + per, chunk + 1 + heads);
  const int c = blockIdx.y * lanes + lane;
  float sum = 0.0f;
  if (c < cols) {
    if (way == 0) sum = partial[(chunk * 2 + 1) * cols + c];
#pragma unroll 8
    for (int64_t k = from; k < to; ++k) sum += partial[k * 2 * cols + c];
  }
  share[threadIdx.x] = sum;
  __syncthreads();
  if (way != 0 || c >= cols) return;
  for (int w = 1; w < ways; ++w) sum += share[w * lanes + lane];
  O* at = out + row * out_stride + c;
  *at = summed(at, sum, scale, accumulate);
}

int launch_sort(const TokenList& tokens, const GradWorkspace& w, cudaStream_t s, const Entry** sorted) {
  const SortPlan p = plan_sort(tokens.n, tokens.vocab);
  const Entry* from = nullptr;
  Entry* to = w.a;
  for (int pass = 0; pass < p.passes; ++pass) {
    const Keys keys{tokens, from};
    const int shift = pass * p.bits;
    int rc;
    if ((rc = launch_operator(count_digits_kernel, dim3((unsigned)p.tiles), kSortThreads, 0, s, keys, tokens.n, shift, p.bits, w.counts)) != MONO_OK) return rc;
    if ((rc = launch_operator(sum_counts_kernel, dim3((unsigned)p.coarse), kSortThreads, 0, s, w.counts, p.tiles, p.bits, w.coarse)) != MONO_OK) return rc;
    if ((rc = launch_operator(scatter_keys_kernel, dim3((unsigned)p.tiles), kSortThreads, 0, s, keys, tokens.n, shift, p.bits, w.counts, w.coarse, p.coarse, to)) != MONO_OK) return rc;
    from = to;
    to = to == w.a ? w.b : w.a;
  }
  *sorted = from;
  return MONO_OK;
}

template <typename G, typename O, int VEC>
int launch_grad(const mono_matrix_t& grad, const TokenList& tokens, float scale, bool accumulate, const mono_matrix_t& out, const GradWorkspace& w, cudaStream_t s) {
  const int cols = (int)grad.cols, vectors = cols / VEC;
  int rc = MONO_OK;
  if (!accumulate) {
    rc = launch_operator(zero_rows_kernel<O>, dim3((unsigned)std::min<int64_t>(out.rows, 148 * 16)), kThreads, 0, s, static_cast<O*>(out.data), out.stride, out.rows, cols);
    if (rc != MONO_OK) return rc;
  }
  if (tokens.n == 0) return MONO_OK;
  const Entry* sorted = nullptr;
  if ((rc = launch_sort(tokens, w, s, &sorted)) != MONO_OK) return rc;
  const int64_t chunks = (tokens.n + kChunk - 1) / kChunk;
  constexpr int R = 8 / VEC;
  const int parts = (vectors + 32 * R - 1) / (32 * R), part_vectors = (vectors + parts - 1) / parts;
  int lanes = 1;
  while (lanes < 32 && lanes * R < part_vectors) lanes *= 2;
  const int groups = kThreads / lanes;
  rc = launch_operator(sum_rows_kernel<G, O, VEC>, dim3((unsigned)((chunks + groups - 1) / groups), (unsigned)parts), kThreads, 0, s, static_cast<const G*>(grad.data), grad.stride,
                       sorted, tokens.n, (uint32_t)tokens.vocab, scale, accumulate, static_cast<O*>(out.data), out.stride, w.partial, cols, part_vectors, lanes);
  if (rc != MONO_OK || chunks < 2) return rc;
  int columns = 1;
  while (columns < 32 && columns < cols) columns *= 2;
  return launch_operator(join_rows_kernel<O>, dim3((unsigned)(chunks - 1), (unsigned)((cols + columns - 1) / columns)), kThreads, 0, s, sorted, tokens.n, (uint32_t)tokens.vocab,
                         scale, accumulate, static_cast<O*>(out.data), out.stride, w.partial, cols, columns);
}

}  // namespace

extern "C" {

int mono_token_rows(const mono_matrix_t* weight, const void* tokens, int32_t token_type, int64_t n_tokens, int64_t padding, float scale,
                    const mono_matrix_t* out, void* cuda_stream) {
  const OperatorRange range(__func__);
  if (!matrix_ok(weight, false) || !matrix_ok(out, true) || !tokens_ok(tokens, token_type, n_tokens)) return MONO_ERR_ARG;
  if (out->rows != n_tokens || out->cols != weight->cols) return MONO_ERR_ARG;
  if (n_tokens == 0) return MONO_OK;
  const TokenList list{tokens, n_tokens, weight->rows, padding, token_type == MONO_I64};
  return with_type(weight->type, [&](auto w) {
    return with_type(out->type, [&](auto o) {
      return with_width(std::min(vector_of(*weight), vector_of(*out)), [&](auto v) {
        return launch_token_rows<decltype(w), decltype(o), decltype(v)::value>(*weight, list, scale, *out, static_cast<cudaStream_t>(cuda_stream));
      });
    });
  });
}

int mono_token_rows_grad_workspace(int64_t n_tokens, int64_t vocabulary, int64_t cols, int64_t* bytes) {
  if (!bytes || n_tokens < 0 || n_tokens > kMaxOperatorRows || vocabulary < 0 || vocabulary > kMaxOperatorRows || cols < 1 || cols > MONO_MAX_COLS) return MONO_ERR_ARG;
  *bytes = carve(nullptr, n_tokens, vocabulary, cols).bytes;
  return MONO_OK;
}

int mono_token_rows_grad(const mono_matrix_t* grad_out, const void* tokens, int32_t token_type, int64_t n_tokens, int64_t padding, float scale, int32_t accumulate,
                         const mono_matrix_t* grad_weight, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  const OperatorRange range(__func__);
  if (!matrix_ok(grad_out, false) || !matrix_ok(grad_weight, true) || !tokens_ok(tokens, token_type, n_tokens)) return MONO_ERR_ARG;
  if (grad_out->rows != n_tokens || grad_out->cols != grad_weight->cols || accumulate < 0 || accumulate > 1) return MONO_ERR_ARG;
  const GradWorkspace w = carve(static_cast<char*>(workspace), n_tokens, grad_weight->rows, grad_weight->cols);
  if (w.bytes > 0 && (!workspace || !is_aligned(workspace, 256))) return MONO_ERR_ARG;
  if (workspace_bytes < w.bytes) return MONO_ERR_SIZE;
  if (grad_weight->rows == 0) return MONO_OK;
  const TokenList list{tokens, n_tokens, grad_weight->rows, padding, token_type == MONO_I64};
  return with_type(grad_out->type, [&](auto g) {
    return with_type(grad_weight->type, [&](auto o) {
      return with_width(std::min(n_tokens ? vector_of(*grad_out) : 8, vector_of(*grad_weight)), [&](auto v) {
        return launch_grad<decltype(g), decltype(o), decltype(v)::value>(*grad_out, list, scale, accumulate != 0, *grad_weight, w, static_cast<cudaStream_t>(cuda_stream));
      });
    });
  });
}

}  // extern "C"

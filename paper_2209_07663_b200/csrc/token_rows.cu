// Rows by token and their gradient (mono_token_rows, mono_token_rows_grad): kernels and host side.
#include <climits>

#include "operators.cuh"
#include "table_layout.cuh"

using namespace mono;

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------
// Rows by token.  out[i] = scale * weight[token i]: nothing is reused, so bytes bound it.
// A thread moves VEC columns at once and keeps several such moves in flight behind the read of its token(s): pieces of one row
// where rows are wide, of four rows where `lanes` threads cover a row.  (65536 tokens, rows of 2048 bf16 columns: 56 us, 6.0 TB/s of what has to
// be read and written; a few tokens are a launch, 2.4 us.)
// ---------------------------------------------------------------------------
constexpr int kMoves = 4;                                  // of 4 or 8 columns

template <typename W, typename O, int VEC, int ROWS, int MOVES>
__global__ void __launch_bounds__(kThreads) token_rows_kernel(const W* weight, int64_t weight_stride, TokenList tokens, float scale,
                                                              O* __restrict__ out, int64_t out_stride, int vectors, int lanes) {
  after_previous_kernel();
  constexpr int PIECES = MOVES / ROWS;
  const int lane = threadIdx.x & (lanes - 1), groups = kThreads / lanes;
  const int64_t row0 = (int64_t)blockIdx.x * groups * ROWS + threadIdx.x / lanes;
  const int v0 = blockIdx.y * lanes * PIECES + lane;
  uint32_t t[ROWS];
  tokens.rows(row0, groups, t);
  Vec<W, VEC> in[MOVES];
#pragma unroll
  for (int k = 0; k < MOVES; ++k) {
    const int r = k / PIECES, v = v0 + (k % PIECES) * lanes;
    if (t[r] != kNoToken && v < vectors) {
      in[k] = *reinterpret_cast<const Vec<W, VEC>*>(weight + t[r] * weight_stride + (int64_t)v * VEC);
    }
  }
#pragma unroll
  for (int k = 0; k < MOVES; ++k) {
    const int r = k / PIECES, v = v0 + (k % PIECES) * lanes;
    const int64_t i = row0 + r * groups;
    if (i >= tokens.n || v >= vectors) continue;
    float f[VEC];
    to_floats(in[k], f);
#pragma unroll
    for (int c = 0; c < VEC; ++c) f[c] = t[r] != kNoToken ? scale * f[c] : 0.0f;
    *reinterpret_cast<Vec<O, VEC>*>(out + i * out_stride + (int64_t)v * VEC) = from_floats<O>(f);
  }
}

// The same for rows that begin anywhere: a thread makes pieces of 8 columns that lie on multiples of 16 bytes of `out` (of those that a row begins or ends
// in, the part that is the row's), from the aligned words that hold them, moved into place in registers.  For rows of 16-bit elements that begin at odd
// ones: with moves of one column 65536 rows of 1023 bf16 columns took 132 us, with these 67 us (1024 columns: 27).  (With moves of two columns or
// of one fp32 column they are no faster: 130 bf16 columns 9.5 us against 16.6, 1023 fp32 ones 84 against 89.)
template <typename W, typename O, int ROWS>
__global__ void __launch_bounds__(kThreads) token_rows_shifted_kernel(const W* weight, int64_t weight_stride, TokenList tokens, float scale,
                                                                      O* __restrict__ out, int64_t out_stride, int cols, int lanes) {
  after_previous_kernel();
  constexpr int PIECES = kMoves / ROWS;
  const int lane = threadIdx.x & (lanes - 1), groups = kThreads / lanes;
  const int64_t row0 = (int64_t)blockIdx.x * groups * ROWS + threadIdx.x / lanes;
  const int v0 = blockIdx.y * lanes * PIECES + lane;
  const W* const begin = weight;
  const W* const end = weight + (tokens.vocab - 1) * weight_stride + cols;
  uint32_t t[ROWS];
  tokens.rows(row0, groups, t);
  uint32_t in[kMoves][8];
#pragma unroll
  for (int k = 0; k < kMoves; ++k) {
    const uint32_t row = t[k / PIECES];
    const int64_t i = row0 + (k / PIECES) * groups;
    const uint32_t skew = (uint32_t)(reinterpret_cast<uintptr_t>(out + i * out_stride) / sizeof(O)) & 7;
    const int c = (v0 + (k % PIECES) * lanes) * 8 - (int)skew;
    if (row == kNoToken || c >= cols) continue;
    const W* const from = weight + row * weight_stride + c;
    // (the aligned words reach up to 15 bytes beyond the 8 elements, and those up to 7 elements beyond the row)
    if (from - 8 >= begin && from + 16 <= end) {
      load_shifted(from, in[k]);
    } else {
      W x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = c + e >= 0 && c + e < cols ? from[e] : from_float<W>(0.0f);
      memcpy(in[k], x, sizeof(x));
    }
  }
#pragma unroll
  for (int k = 0; k < kMoves; ++k) {
    const uint32_t row = t[k / PIECES];
    const int64_t i = row0 + (k / PIECES) * groups;
    if (i >= tokens.n) continue;
    const uint32_t skew = (uint32_t)(reinterpret_cast<uintptr_t>(out + i * out_stride) / sizeof(O)) & 7;
    const int c = (v0 + (k % PIECES) * lanes) * 8 - (int)skew;
    if (c >= cols) continue;
    float f[8] = {};
    if (row != kNoToken) {
      const W* const from = weight + row * weight_stride + c;
      const bool whole = from - 8 >= begin && from + 16 <= end;
      to_floats(shifted<W>(in[k], whole ? (uint32_t)reinterpret_cast<uintptr_t>(from) & 15 : 0), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= scale;
    }
    const Vec<O, 8> o = from_floats<O>(f);
    O* const to = out + i * out_stride + c;
    if (c >= 0 && c + 8 <= cols) {
      *reinterpret_cast<Vec<O, 8>*>(to) = o;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e >= 0 && c + e < cols) to[e] = o.v[e];
    }
  }
}

template <typename W, typename O, int VEC>
int launch_token_rows(const mono_matrix_t& weight, const TokenList& tokens, float scale, const mono_matrix_t& out, cudaStream_t s) {
  constexpr int MOVES = VEC >= 4 ? kMoves : kMoves * 4 / VEC;      // (narrow moves: as many bytes in flight)
  const bool shifts = VEC == 1 && sizeof(W) == 2 && weight.cols >= 32;      // (a few columns are a piece or two whichever way)
  const int vectors = shifts ? (int)((weight.cols + 7 + 7) / 8) : (int)(weight.cols / VEC), moves = shifts ? kMoves : MOVES;
  const auto launch = [&](auto rows_of_a_thread) {
    constexpr int ROWS = decltype(rows_of_a_thread)::value;
    const int pieces = moves / ROWS;
    int lanes = 1;
    while (lanes < kThreads && lanes * pieces < vectors) lanes *= 2;
    const int64_t rows = (int64_t)(kThreads / lanes) * ROWS, columns = (int64_t)lanes * pieces;
    const dim3 grid((unsigned)((tokens.n + rows - 1) / rows), (unsigned)((vectors + columns - 1) / columns));
    const auto* from = static_cast<const W*>(weight.data);
    auto* to = static_cast<O*>(out.data);
    if constexpr (VEC == 1 && sizeof(W) == 2) {
      if (shifts)
        return launch_operator(token_rows_shifted_kernel<W, O, ROWS>, grid, kThreads, 0, s, from, weight.stride, tokens, scale, to, out.stride, (int)weight.cols, lanes);
    }
    return launch_operator(token_rows_kernel<W, O, VEC, ROWS, MOVES>, grid, kThreads, 0, s, from, weight.stride, tokens, scale, to, out.stride, vectors, lanes);
  };
  // (65536 rows of 1024 bf16 columns: one row a thread 27 us, four 32 us)
  return vectors > 64 ? launch(Width<1>()) : launch(Width<4>());
}

// ---------------------------------------------------------------------------
// Gradient.  The tokens are sorted stably by row (tokens without a row last), so that the terms of a row are
// consecutive.  A group of up to 32 threads adds up a run of sorted positions in order and writes the rows that begin and end in
// it; what it has of other rows, a piece in front and a piece at the end, a block joins over its groups' runs in
// shared memory, and join_rows_kernel over the blocks, both in the order of the positions.  The terms are read once and
// no order depends on timing or on where the matrices lie, so the result has the same bits every time.  (Adding the product to
// what is there is one operation, which is written out where the compiler makes two of it for some widths of the moves: where pieces are joined.  In sum_rows_kernel's
// own rows it makes one for all of them, and written out there it costs 2.5 % of 30011 tokens' 62 us at 515 columns, through the order of what is around it.)
//
// Three ways to sort, by the number of tokens:
//   up to kSmallTokens   every block of the summing kernel ranks all tokens in shared memory: no launch of its own
//   up to kRankTokens    one launch: a token's place is the number of tokens before it, counted; n * n comparisons
//   beyond               radix sort, least digit first, two launches a digit of up to 9 bits
// Where all of the gradient is written, its zeros are filled in by blocks behind those that sort, which
// use a few SMs for a few microseconds: of all rows, or, where the sort has several passes, of those that the first pass did not mark.
//
// Both sides of the limits, fp32 gradients of 32000 rows, written whole (added to): 512 tokens of 64 columns 17.3 us (14.4) the first way, 8.7 (9.1) the second; 257 tokens 11.3 (8.9)
// and 8.8 (8.5); 1024 the first way 46 (44), the second 10.5 (10.7).  8192 tokens of 1024 columns the second way 42.0 (29.7), the third 49.9 (23.1), 4096 tokens 33.2 (15.7) and
// 49.1 (21.1), 11000 tokens 50.5 (47.8) and 52.7 (30.8): where all of the gradient is written 8192 is near the crossing, which comes at 6144 where it is added to.
//
// Measured: 262144 tokens, 1024 bf16 columns, fp32 gradient of 131072 rows: 224 us, of which the sums are 129 (660 MB, 5.1 TB/s), the sort with the
// zeros 85 and the joins 9; 4096 tokens of 1024 columns, bf16 gradient of 32000 rows 24 us; 77 tokens of 64 columns 5.2 us.
// ---------------------------------------------------------------------------
constexpr int64_t kSmallTokens = 512;
constexpr int kSmallRun = 2;                                // their positions of a group
constexpr int64_t kRankTokens = 8192;
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMostSortKeys = 8;                           // keys of a thread
constexpr int kMaxDigitBits = 9;
constexpr int kMaxDigits = 1 << kMaxDigitBits;
static_assert(kMaxDigits == kSortThreads, "a thread has one digit's counts");
constexpr int64_t kMaxFineTiles = 64;                      // beyond, the digits' counts are also summed up over kCoarse tiles each
constexpr int kCoarse = 32;
constexpr int kLaneColumns = 8;                            // columns whose sums a thread holds
constexpr int kMinRun = 8, kMaxRun = 64;                   // positions of a group

struct Entry { uint32_t row, at; };                        // a token's row (vocab: none) and its position
constexpr uint32_t kBehind = 0xFFFFFFFFu;                  // row of the entry behind the last one

// Zeros of rows [begin, end) of the matrix that is written, but for the rows that are marked as named by a token: a group of `lanes`
// threads has four rows at a time.
struct Zeros {
  char* data;
  int64_t stride;          // bytes from a row to the next
  int64_t begin, end;
  int pieces, size;        // of a row, and bytes of one: as many as the row's alignment allows
  int lanes;
  const uint8_t* marks;    // nullptr: none is
  unsigned first;          // the block that begins

  __device__ __forceinline__ bool here() const { return blockIdx.x >= first; }

  template <typename T>
  __device__ __forceinline__ void rows() const {
    const int lane = threadIdx.x & (lanes - 1), groups = blockDim.x / lanes;
    const int64_t step = (int64_t)(gridDim.x - first) * groups * 4;
    for (int64_t r0 = begin + ((int64_t)(blockIdx.x - first) * groups + threadIdx.x / lanes) * 4; r0 < end; r0 += step) {
      bool write[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) write[k] = r0 + k < end && !(marks && marks[r0 + k]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (!write[k]) continue;
        T* row = reinterpret_cast<T*>(data + (r0 + k) * stride);
        for (int i = lane; i < pieces; i += lanes) row[i] = T{};
      }
    }
  }
  __device__ void fill() const {
    if (size == 16) rows<uint4>(); else if (size == 8) rows<uint2>(); else if (size == 4) rows<uint32_t>(); else rows<uint16_t>();
  }
};

// The tokens of a call: the caller's in the first pass, the entries of the pass before in the others.
struct Keys {
  TokenList tokens;
  const Entry* entries;    // nullptr: the tokens
  // those at first, first + step, ... (none behind the last one: kBehind)
  template <int K>
  __device__ __forceinline__ void load(int64_t first, int64_t step, Entry (&e)[K]) const {
    if (entries) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const uint2 x = first + k * step < tokens.n ? reinterpret_cast<const uint2*>(entries)[first + k * step] : make_uint2(kBehind, 0);
        e[k] = {x.x, x.y};
      }
      return;
    }
    uint32_t row[K];
    tokens.rows(first, step, row);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t i = first + k * step;
      e[k] = {i >= tokens.n ? kBehind : row[k] == kNoToken ? (uint32_t)tokens.vocab : row[k], (uint32_t)i};
    }
  }
};

// How many of the keys [from, to) in shared memory come before a key: those below it, and of those equal to it the ones at lower positions.
__device__ __forceinline__ uint32_t count_before(const uint32_t* keys, int from, int to, uint32_t key, int position) {
  uint32_t n = 0;
  const int equal_to = min(max(position, from), to);
#pragma unroll 8
  for (int j = from; j < equal_to; ++j) n += keys[j] <= key;
#pragma unroll 8
  for (int j = equal_to; j < to; ++j) n += keys[j] < key;
  return n;
}

// Lets the launch of the call's next kernel begin; it waits for this one's end itself (after_previous_kernel).  The kernels of a
// gradient are short and leave SMs free (with it and few keys a thread in the sort, 16384 tokens of 1024 columns went from 40 to 34 us).
// What such a kernel reads may have been written during its lifetime: its inputs are read through the coherent path (no __ldg, no
// const __restrict__).  A call's last kernel does not let anyone begin.
__device__ __forceinline__ void release_next_kernel() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// 32 tokens a block; each warp counts over its share of all tokens, four at a time: those in front of the block's, up to the key, those behind
// them, below it.
__global__ void __launch_bounds__(kThreads) rank_tokens_kernel(TokenList tokens, Entry* __restrict__ sorted, Zeros zeros) {
  after_previous_kernel();
  release_next_kernel();
  if (zeros.here()) { zeros.fill(); return; }
  constexpr int kWarps = kThreads / 32;
  __shared__ __align__(16) uint32_t keys[kRankTokens];
  __shared__ uint32_t counts[kWarps][32];
  const Keys all{tokens, nullptr};
  const int n = (int)tokens.n, padded = (n + 31) / 32 * 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int i0 = threadIdx.x; i0 < padded; i0 += 8 * kThreads) {
    Entry e[8];
    all.load(i0, kThreads, e);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i0 + k * kThreads < padded) keys[i0 + k * kThreads] = e[k].row;        // (kBehind behind the last one: below none)
  }
  __syncthreads();
  const int first = blockIdx.x * 32, mine = first + lane, share = (padded / 32 + kWarps - 1) / kWarps * 32;
  const int from = min(warp * share, padded), to = min(from + share, padded);
  const uint32_t key = keys[mine];
  uint32_t before = 0;
#pragma unroll 4
  for (int j = from; j < min(to, first); j += 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(keys + j);
    before += (x.x <= key) + (x.y <= key) + (x.z <= key) + (x.w <= key);
  }
#pragma unroll 4
  for (int j = max(from, first + 32); j < to; j += 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(keys + j);
    before += (x.x < key) + (x.y < key) + (x.z < key) + (x.w < key);
  }
  if (from <= first && first < to) before += count_before(keys, first, first + 32, key, mine);
  counts[warp][lane] = before;
  __syncthreads();
  if (warp != 0 || mine >= n) return;
  uint32_t place = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) place += counts[w][lane];
  sorted[place] = {key, (uint32_t)mine};
  if (mine == 0) sorted[n] = {kBehind, 0};
}

// (marks: cleared, by the blocks that would fill zeros, where this is the first pass)
template <int KEYS>
__global__ void __launch_bounds__(kSortThreads) count_digits_kernel(Keys keys, int shift, int bits, uint32_t* __restrict__ counts, uint4* marks, int64_t mark_words,
                                                                    Zeros zeros) {
  after_previous_kernel();
  release_next_kernel();
  if (zeros.here()) {
    if (!marks) { zeros.fill(); return; }
    for (int64_t i = (int64_t)(blockIdx.x - zeros.first) * kSortThreads + threadIdx.x; i < mark_words; i += (int64_t)(gridDim.x - zeros.first) * kSortThreads)
      marks[i] = make_uint4(0, 0, 0, 0);
    return;
  }
  __shared__ uint32_t count[kMaxDigits];
  count[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * (kSortThreads * KEYS);
  Entry e[KEYS];
  keys.load(base + threadIdx.x, kSortThreads, e);
#pragma unroll
  for (int k = 0; k < KEYS; ++k)
    if (e[k].row != kBehind) atomicAdd(&count[(e[k].row >> shift) & ((1 << bits) - 1)], 1u);
  __syncthreads();
  counts[(int64_t)blockIdx.x * kMaxDigits + threadIdx.x] = count[threadIdx.x];
}

// counts summed up over kCoarse tiles each
__global__ void __launch_bounds__(kSortThreads) sum_counts_kernel(const uint32_t* counts, int64_t tiles, uint32_t* __restrict__ coarse) {
  after_previous_kernel();
  const int64_t first = (int64_t)blockIdx.x * kCoarse, last = first + kCoarse < tiles ? first + kCoarse : tiles;
  uint32_t sum = 0;
#pragma unroll 16
  for (int64_t t = first; t < last; ++t) sum += counts[t * kMaxDigits + threadIdx.x];
  coarse[(int64_t)blockIdx.x * kMaxDigits + threadIdx.x] = sum;
}

// A key goes behind the keys of lower digits of all tiles, those of its digit in earlier tiles, in earlier warps of its tile (warp w has the
// tile's keys [w * 32 * KEYS, (w + 1) * 32 * KEYS)), in earlier rounds of 32 keys, and at lower lanes.
template <int KEYS>
__global__ void __launch_bounds__(kSortThreads) scatter_keys_kernel(Keys keys, int64_t n, int shift, int bits, const uint32_t* counts, int64_t tiles,
                                                                    const uint32_t* coarse, Entry* __restrict__ sorted, uint8_t* marks, Zeros zeros) {
  after_previous_kernel();
  release_next_kernel();
  if (zeros.here()) { zeros.fill(); return; }
  __shared__ __align__(8) uint32_t next[kSortWarps][kMaxDigits];        // counts of the warps, then the place of a warp's next key of a digit
  __shared__ uint32_t warp_sum[kSortWarps];
  const int digits = 1 << bits, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t tile = blockIdx.x, base = tile * (kSortThreads * KEYS) + warp * (32 * KEYS);
  if (tile == 0 && threadIdx.x == 0) sorted[n] = {kBehind, 0};
  Entry e[KEYS];
  keys.load(base + lane, 32, e);
  if (marks) {
    // Of the tile's keys that share a cell, the last one to write it marks its row and those of the same row leave it alone: marked by every
    // token, the row that a tenth of them name took longer than the rest of the sort.
    uint64_t* cell = reinterpret_cast<uint64_t*>(next[0]);
    constexpr uint32_t kCells = sizeof(next) / 8;
#pragma unroll
    for (int k = 0; k < KEYS; ++k)
      if (e[k].row < keys.tokens.vocab) cell[e[k].row % kCells] = (uint64_t)e[k].row << 32 | (threadIdx.x * KEYS + k);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
      if (e[k].row >= keys.tokens.vocab) continue;
      const uint64_t by = cell[e[k].row % kCells];
      if ((uint32_t)(by >> 32) != e[k].row || (uint32_t)by == threadIdx.x * KEYS + k) marks[e[k].row] = 1;
    }
    __syncthreads();
  }
  // of this thread's digit: keys of all tiles, and of earlier ones
  uint32_t total = 0, before = 0;
  if (coarse == nullptr) {
#pragma unroll 16
    for (int64_t t = 0; t < tiles; ++t) {
      const uint32_t c = counts[t * kMaxDigits + threadIdx.x];
      total += c;
      if (t < tile) before += c;
    }
  } else {
    const int64_t own = tile / kCoarse, n_coarse = (tiles + kCoarse - 1) / kCoarse;
#pragma unroll 16
    for (int64_t t = 0; t < n_coarse; ++t) {
      const uint32_t c = coarse[t * kMaxDigits + threadIdx.x];
      total += c;
      if (t < own) before += c;
    }
#pragma unroll 16
    for (int64_t t = own * kCoarse; t < tile; ++t) before += counts[t * kMaxDigits + threadIdx.x];
  }
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) next[w][threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < KEYS; ++k)
    if (e[k].row != kBehind) atomicAdd(&next[warp][(e[k].row >> shift) & (digits - 1)], 1u);
  uint32_t scan = total;
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, scan, s);
    if (lane >= s) scan += x;
  }
  if (lane == 31) warp_sum[warp] = scan;
  __syncthreads();
  uint32_t place = scan - total + before;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) place += w < warp ? warp_sum[w] : 0;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) {
    const uint32_t c = next[w][threadIdx.x];
    next[w][threadIdx.x] = place;
    place += c;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    const bool there = e[k].row != kBehind;
    const uint32_t digit = (e[k].row >> shift) & (digits - 1);
    uint32_t same = __ballot_sync(0xFFFFFFFFu, there);       // lanes whose digits agree in every bit
    for (int b = 0; b < bits; ++b) {
      const uint32_t set = __ballot_sync(0xFFFFFFFFu, digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    const uint32_t rank = __popc(same & ((1u << lane) - 1));
    uint32_t to = 0;
    if (there) to = next[warp][digit] + rank;
    __syncwarp();
    if (there && rank == 0) next[warp][digit] += __popc(same);
    __syncwarp();
    if (there && to < n) sorted[to] = e[k];                 // (every place is below n, by the counts: a wrong one is not written)
  }
}

__global__ void __launch_bounds__(kThreads) zero_rows_kernel(Zeros zeros) {
  after_previous_kernel();
  zeros.fill();
}

// Where the sums of a call go.
template <typename O>
struct GradOut {
  O* data;
  int64_t stride;
  float* partial;          // [blocks][2][cols]: of the row that began in an earlier block, of the one that goes on in the next
  int cols;
  uint32_t vocab;
  float scale;
};

// ADD: what is there is added to.  It is read with the terms, ahead of the sum that it waits for: a row at a time, a
// thread's reads would come one after the other.
// blockIdx.x: runs of `run` positions, one for each group of `lanes` threads; blockIdx.y: part_vectors vectors of VEC columns.
// Without `sorted` (at most kSmallTokens tokens) every block sorts all tokens itself.
template <typename G, typename O, int VEC, bool ADD>
__global__ void __launch_bounds__(kThreads, VEC >= 4 || (VEC == 1 && sizeof(G) == 2) ? (ADD ? 2 : 3) : VEC == 1 ? 3 : 2) sum_rows_kernel(const G* grad, uint32_t grad_stride, TokenList tokens, const Entry* sorted,
                                                                                       int run, GradOut<O> out, int part_vectors, int lanes, bool joined) {
  after_previous_kernel();
  if (joined) release_next_kernel();
  constexpr int R = kLaneColumns / VEC;
  // Rows of 16-bit elements that begin anywhere: a thread has 8 neighbouring columns of the terms, from the aligned words that hold them, and what
  // it writes passes through shared memory, so that neighbours write neighbours.
  constexpr bool SHIFTED = VEC == 1 && sizeof(G) == 2;
  constexpr int U = VEC == 1 && !SHIFTED ? 2 : 4;           // positions whose terms are in flight at once
  constexpr uint32_t kNone = 0xFFFFFFFFu;
  __shared__ float piece[2 * kThreads * kLaneColumns];      // [groups][2][lanes * kLaneColumns]: front, end
  __shared__ uint2 pieces[2 * kThreads];                    // of the pieces there are, in order: the row, the place in piece[]
  __shared__ uint32_t warp_pieces[kThreads / 32];
  __shared__ uint32_t keys[kSmallTokens];
  __shared__ Entry ranked[kSmallTokens + 1];
  __shared__ __align__(16) float turned[SHIFTED ? kThreads * kLaneColumns : 1];
  const int64_t n = tokens.n;
  const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = kThreads / lanes, width = lanes * kLaneColumns;
  int64_t b0 = (int64_t)blockIdx.x * groups * run, b1 = b0 + (int64_t)groups * run < n ? b0 + (int64_t)groups * run : n;
  const bool here = sorted == nullptr;
  if (here) {
    constexpr int K = kSmallTokens / kThreads;
    const Keys all{tokens, nullptr};
    Entry own[K];
    all.load(threadIdx.x, kThreads, own);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (own[k].row != kBehind) keys[own[k].at] = own[k].row;
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < K; ++k) {
      const int i = threadIdx.x + k * kThreads;
      if (i < n) ranked[count_before(keys, 0, (int)n, keys[i], i)] = {keys[i], (uint32_t)i};
    }
    if (threadIdx.x == 0) ranked[n] = {kBehind, 0};
    __syncthreads();
    sorted = ranked;
    // the rows that begin among the block's positions, to their ends: no other block has a part in them
    const auto behind = [&](int64_t p) {                    // the first position behind the row of position p
      int64_t low = p, high = n;                            // (of the row; not of it, or n)
      while (high - low > 1) {
        const int64_t mid = (low + high) / 2;
        if (ranked[mid].row == ranked[p].row) low = mid; else high = mid;
      }
      return high;
    };
    if (b0 > 0 && ranked[b0].row == ranked[b0 - 1].row) b0 = behind(b0);
    b1 = b0 >= b1 ? b0 : behind(b1 - 1);
    run = (int)((b1 - b0 + groups - 1) / groups);
  }
  const int64_t p0 = b0 + (int64_t)group * run;
  const int first = blockIdx.y * part_vectors, end = min(first + part_vectors, out.cols / VEC);
  uint32_t front_row = kNone, end_row = kNone;
  const Entry* const list = sorted + p0;
  int len = (int)max((int64_t)0, min(b1 - p0, (int64_t)run));
  if (len > 0 && list[len - 1].row >= out.vocab) {          // not those without a row: they are last
    if (list[0].row >= out.vocab) len = 0;
    while (len > 0 && list[len - 1].row >= out.vocab) --len;
  }

  if (len > 0) {
    float sum[R][VEC] = {};
    bool mine[R];                                           // vectors that there are
#pragma unroll
    for (int r = 0; r < R; ++r) mine[r] = first + lane + r * lanes < end;
    const char* const from = reinterpret_cast<const char*>(grad) + (int64_t)(first + lane) * (VEC * sizeof(G));
    O* const to = out.data + (int64_t)(first + lane) * VEC;
    const G* const grad_end = grad + (n - 1) * (int64_t)(grad_stride / sizeof(G)) + out.cols;
    const uint32_t near = lanes == 32 ? 0xFFFFFFFFu : ((1u << lanes) - 1) << (threadIdx.x % 32 & ~(lanes - 1));      // the group's threads
    Entry e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) e[u] = list[min(u, len)];
    bool began_before = p0 > 0 && list[-1].row == e[0].row;

    for (int i = 0; i < len; i += U) {
      Vec<G, VEC> term[SHIFTED ? 1 : U][R];
      uint32_t raw[SHIFTED ? U : 1][8], begins[SHIFTED ? U : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const char* row = from + (uint64_t)e[u].at * grad_stride;
        if constexpr (SHIFTED) {
          const G* const at = reinterpret_cast<const G*>(row) + lane * 7;       // (from is the lane's first column of one)
          const bool whole = at - 8 >= grad && at + 16 <= grad_end;
          begins[u] = whole ? (uint32_t)reinterpret_cast<uintptr_t>(at) & 15 : 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) raw[u][k] = 0;
          if (i + u < len && first + lane * 8 < end) {
            if (whole) {
              load_shifted(at, raw[u]);
            } else {
              G x[8];
#pragma unroll
              for (int c = 0; c < 8; ++c) x[c] = first + lane * 8 + c < end ? at[c] : from_float<G>(0.0f);
              memcpy(raw[u], x, sizeof(x));
            }
          }
        } else {
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (i + u < len && mine[r]) term[u][r] = *reinterpret_cast<const Vec<G, VEC>*>(row + r * lanes * (int)(VEC * sizeof(G)));
        }
      }
      Entry ahead[U];                                       // the next positions, while the terms are on their way
#pragma unroll
      for (int u = 0; u < U; ++u) ahead[u] = list[min(i + U + u, len)];
      uint32_t last = 0;                                    // positions that are the last ones of their rows
#pragma unroll
      for (int u = 0; u < U; ++u) last |= (e[u].row != (u + 1 < U ? e[u + 1] : ahead[0]).row ? 1u : 0u) << u;
      Vec<O, VEC> old[ADD ? U : 1][R];
      if constexpr (ADD) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const O* at = to + (int64_t)e[u].row * out.stride;
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (i + u < len && (last >> u & 1) && mine[r]) old[u][r] = *reinterpret_cast<const Vec<O, VEC>*>(at + r * lanes * VEC);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u < len) {
          if constexpr (SHIFTED) {
            float f[8];
            to_floats(shifted<G>(raw[u], begins[u]), f);
            float(&all)[8] = reinterpret_cast<float(&)[8]>(sum);
            add_floats(all, f);
          } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
              float f[VEC];
              to_floats(term[u][r], f);
              add_floats(sum[r], f);
            }
          }
          const bool ends = last >> u & 1;
          if (ends || i + u + 1 == len) {
            if (ends && !began_before) {
              O* at = to + (int64_t)e[u].row * out.stride;
              if constexpr (SHIFTED) {                      // from the columns it added up to those that it writes
                float* const mine_in = turned + group * width + lane * 8;
                __syncwarp(near);
                *reinterpret_cast<float4*>(mine_in) = make_float4(sum[0][0], sum[1][0], sum[2][0], sum[3][0]);
                *reinterpret_cast<float4*>(mine_in + 4) = make_float4(sum[4][0], sum[5][0], sum[6][0], sum[7][0]);
                __syncwarp(near);
#pragma unroll
                for (int r = 0; r < R; ++r) sum[r][0] = turned[group * width + lane + r * lanes];
              }
#pragma unroll
              for (int r = 0; r < R; ++r) {
                float f[VEC];
#pragma unroll
                for (int c = 0; c < VEC; ++c) f[c] = ADD ? to_float(old[ADD ? u : 0][r].v[c]) + out.scale * sum[r][c] : out.scale * sum[r][c];
                if (mine[r]) *reinterpret_cast<Vec<O, VEC>*>(at + r * lanes * VEC) = from_floats<O>(f);
              }
            } else {
              float* keep = piece + (group * 2 + (began_before ? 0 : 1)) * width + (SHIFTED ? lane * 8 : lane * VEC);
#pragma unroll
              for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int c = 0; c < VEC; ++c) keep[SHIFTED ? r : r * lanes * VEC + c] = sum[r][c];
              }
              if (began_before) front_row = e[u].row; else end_row = e[u].row;
            }
            began_before = false;
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
              for (int c = 0; c < VEC; ++c) sum[r][c] = 0.0f;
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) e[u] = ahead[u];
    }
  }

  // the groups' pieces in order; those of one row follow one another
  {
    const int mine = lane == 0 ? (front_row != kNone) + (end_row != kNone) : 0, in_warp = threadIdx.x % 32, warp = threadIdx.x / 32;
    int scan = mine;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, scan, s);
      if (in_warp >= s) scan += x;
    }
    if (in_warp == 31) warp_pieces[warp] = scan;
    __syncthreads();
    int at = scan - mine;
    for (int w = 0; w < warp; ++w) at += warp_pieces[w];
    if (lane == 0 && front_row != kNone) pieces[at++] = make_uint2(front_row, (group * 2) * width);
    if (lane == 0 && end_row != kNone) pieces[at] = make_uint2(end_row, (group * 2 + 1) * width);
    __syncthreads();
  }
  int count = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) count += warp_pieces[w];
  if (count == 0) return;
  const uint32_t before_row = b0 > 0 && !here ? sorted[b0 - 1].row : kNone, behind_row = b1 < n && !here ? sorted[b1].row : kNone;
  for (int c = threadIdx.x; c < (end - first) * VEC; c += kThreads) {
    constexpr int K = 8;
    const int column = first * VEC + c;
    float sum = 0.0f;
    for (int k0 = 0; k0 < count; k0 += K) {
      uint2 x[K + 1];
      float part[K], old[K];
#pragma unroll
      for (int k = 0; k <= K; ++k) x[k] = k0 + k < count ? pieces[k0 + k] : make_uint2(kNone, 0);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        part[k] = x[k].x != kNone ? piece[x[k].y + c] : 0.0f;
        if (ADD && x[k].x != x[k + 1].x && x[k].x != before_row && x[k].x != behind_row) old[k] = to_float(out.data[x[k].x * out.stride + column]);
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (x[k].x == kNone) continue;
        sum += part[k];
        if (x[k].x == x[k + 1].x) continue;
        if (x[k].x == before_row) out.partial[(int64_t)blockIdx.x * 2 * out.cols + column] = sum;
        else if (x[k].x == behind_row) out.partial[((int64_t)blockIdx.x * 2 + 1) * out.cols + column] = sum;
        else out.data[x[k].x * out.stride + column] = from_float<O>(ADD ? fmaf(out.scale, sum, old[k]) : out.scale * sum);
        sum = 0.0f;
      }
    }
  }
}

// A row that begins in block blockIdx.x of the sums (of `positions` sorted positions) and goes on behind it: its partial sums, in order.
// A thread has VEC columns.
template <typename O, int VEC>
__global__ void __launch_bounds__(kThreads) join_rows_kernel(const Entry* sorted, int64_t n, int positions, bool add, GradOut<O> out) {
  after_previous_kernel();
  constexpr int U = 16;
  const int64_t b = blockIdx.x, p0 = b * positions, p1 = p0 + positions;
  const uint32_t row = sorted[p1].row, last = sorted[p1 - 1].row, before = p0 > 0 ? sorted[p0 - 1].row : kBehind;
  if (row >= out.vocab || last != row || before == row) return;      // (before: it began earlier)
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  if (c >= out.cols) return;
  using Part = Vec<float, VEC>;
  const auto part = [&](int64_t at) { return *reinterpret_cast<const Part*>(out.partial + at * out.cols + c); };
  Part sum = part(b * 2 + 1);
  Vec<O, VEC>* const to = reinterpret_cast<Vec<O, VEC>*>(out.data + row * out.stride + c);
  Vec<O, VEC> o;
  if (add) o = *to;
  const int64_t blocks = (n + positions - 1) / positions;
  bool goes_on = true;
  for (int64_t k = b + 1; goes_on; k += U) {
    Part x[U];
    uint32_t r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = k + u < blocks ? sorted[(k + u) * positions].row : kBehind;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k + u < blocks) x[u] = part((k + u) * 2);       // (of a block of another row: not used)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      goes_on = goes_on && r[u] == row;
      if (goes_on) add_floats(sum.v, x[u].v);
    }
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v) o.v[v] = from_float<O>(add ? fmaf(out.scale, sum.v[v], to_float(o.v[v])) : out.scale * sum.v[v]);
  *to = o;
}

// ---- host side ----

struct SortPlan {
  int passes, bits;                                        // digits of `bits` bits each
  int keys;                                                // of a thread
  int64_t tiles, coarse;
};

SortPlan plan_sort(int64_t n, int64_t vocab) {
  int width = 1;
  while (((uint64_t)vocab >> width) != 0) ++width;         // rows 0 .. vocab, the last one for tokens without a row
  SortPlan p;
  p.passes = (width + kMaxDigitBits - 1) / kMaxDigitBits;
  p.bits = (width + p.passes - 1) / p.passes;
  // few keys a thread spread the work; up to kMaxFineTiles tiles are counted without another launch
  p.keys = 1;
  while (p.keys < kMostSortKeys && n > (int64_t)kSortThreads * p.keys * kMaxFineTiles) p.keys *= 2;
  const int64_t tile = (int64_t)kSortThreads * p.keys;
  p.tiles = (n + tile - 1) / tile;
  p.coarse = p.tiles > kMaxFineTiles ? (p.tiles + kCoarse - 1) / kCoarse : 0;
  return p;
}

// How the sums are cut: positions of a group, and of a block.
struct SumPlan {
  int lanes, groups, parts, part_vectors, run;
  int64_t blocks;
};

SumPlan plan_sums(int64_t n, int vectors, int vec) {
  SumPlan p;
  const int most = 32 * (kLaneColumns / vec);
  p.parts = (vectors + most - 1) / most;
  p.part_vectors = (vectors + p.parts - 1) / p.parts;
  p.lanes = 1;
  while (p.lanes < 32 && p.lanes * (kLaneColumns / vec) < p.part_vectors) p.lanes *= 2;
  p.groups = kThreads / p.lanes;
  // long runs have fewer pieces, short ones more warps: as long as there are 24 warps for every SM
  p.run = kMaxRun;
  while (p.run > kMinRun && n * p.parts / p.run * p.lanes / 32 < 148 * 24) p.run /= 2;
  if (n <= kSmallTokens) p.run = kSmallRun;
  p.blocks = (n + (int64_t)p.run * p.groups - 1) / ((int64_t)p.run * p.groups);
  return p;
}

struct GradWorkspace {
  Entry* a;
  Entry* b;
  uint32_t* counts;        // [tiles][digits]
  uint32_t* coarse;        // [coarse][digits]
  uint8_t* marks;          // [vocab]: rows that a token names, where the zeros of the others are filled in
  float* partial;          // [blocks][2][cols]
  int64_t bytes;
};

// Beyond, the marks would cost more memory than they spare writes.
constexpr int64_t kMaxMarks = 1 << 24;
bool marks_rows(int64_t n, int64_t vocab) { return n > kRankTokens && vocab >= kMaxDigits && vocab <= kMaxMarks; }

GradWorkspace carve(char* base, int64_t n, int64_t vocab, int64_t cols) {
  int64_t at = 0;
  const auto take = [&](int64_t bytes) { char* r = base + at; at += (bytes + 255) / 256 * 256; return r; };
  GradWorkspace w = {};
  if (n > kSmallTokens) {
    const SortPlan p = plan_sort(n, vocab);
    w.a = reinterpret_cast<Entry*>(take((n + 1) * (int64_t)sizeof(Entry)));
    if (n > kRankTokens) {
      w.b = reinterpret_cast<Entry*>(take((n + 1) * (int64_t)sizeof(Entry)));
      w.counts = reinterpret_cast<uint32_t*>(take(p.tiles * kMaxDigits * 4));
      w.coarse = reinterpret_cast<uint32_t*>(take(p.coarse * kMaxDigits * 4));
      if (marks_rows(n, vocab)) w.marks = reinterpret_cast<uint8_t*>(take(vocab));
    }
    int64_t blocks = 0;                                     // (the matrices' alignment decides the vectors)
    for (int vec = 1; vec <= 8; vec *= 2)
      if (cols % vec == 0) blocks = std::max(blocks, plan_sums(n, (int)(cols / vec), vec).blocks);
    w.partial = reinterpret_cast<float*>(take(blocks * 2 * cols * 4));
  }
  w.bytes = at;
  return w;
}

constexpr unsigned kZeroBlocks = 148 * 4;

Zeros zeros_of(const mono_matrix_t& m) {
  const int size = element_size(m.type);
  int bytes = 16;
  while (bytes > size && (m.cols * size % bytes || !is_aligned(m.data, bytes) || (m.rows > 1 && m.stride * size % bytes))) bytes /= 2;
  Zeros z = {static_cast<char*>(m.data), m.stride * size, 0, 0, (int)(m.cols * size / bytes), bytes, 1, nullptr, UINT_MAX};
  while (z.lanes < 32 && z.lanes < z.pieces) z.lanes *= 2;
  return z;
}

template <typename G, typename O, int VEC>
int launch_grad(const mono_matrix_t& grad, const TokenList& tokens, float scale, bool accumulate, const mono_matrix_t& out, const GradWorkspace& w, cudaStream_t s) {
  const int cols = (int)out.cols;
  const int64_t n = tokens.n, vocab = out.rows;
  int rc = MONO_OK;
  Zeros zeros = zeros_of(out);
  if (!accumulate && n <= kSmallTokens) {
    zeros.end = vocab;
    zeros.first = 0;
    const int64_t rows = (int64_t)(kThreads / zeros.lanes) * 4;
    rc = launch_operator(zero_rows_kernel, dim3((unsigned)std::min<int64_t>((vocab + rows - 1) / rows, 148 * 8)), kThreads, 0, s, zeros);
    if (rc != MONO_OK) return rc;
  }
  if (n == 0) return MONO_OK;
  // share `k` of `shares` of the zeros, behind `blocks` blocks that sort
  const auto share = [&](int k, int shares, int64_t blocks, dim3* grid) {
    const bool fills = !accumulate && k >= 0;
    zeros.begin = vocab * k / shares;
    zeros.end = vocab * (k + 1) / shares;
    zeros.first = fills ? (unsigned)blocks : UINT_MAX;
    *grid = dim3((unsigned)blocks + (fills ? (n <= kRankTokens ? 2 : 1) * kZeroBlocks : 0));        // (of half as many threads)
    return zeros;
  };
  const SumPlan sums = plan_sums(n, cols / VEC, VEC);
  const GradOut<O> to{static_cast<O*>(out.data), out.stride, w.partial, cols, (uint32_t)vocab, scale};
  const auto* from = static_cast<const G*>(grad.data);
  const dim3 sum_grid((unsigned)sums.blocks, (unsigned)sums.parts);
  const Entry* sorted = nullptr;
  dim3 grid;
  if (n > kSmallTokens && n <= kRankTokens) {
    const Zeros z = share(0, 1, (n + 31) / 32, &grid);
    if ((rc = launch_operator(rank_tokens_kernel, grid, kThreads, 0, s, tokens, w.a, z)) != MONO_OK) return rc;
    sorted = w.a;
  } else if (n > kRankTokens) {
    const SortPlan p = plan_sort(n, vocab);
    // the first pass clears the marks and sets them, the others fill in the zeros of what is not marked
    uint8_t* const marks = accumulate || p.passes < 2 ? nullptr : w.marks;
    const int skipped = marks ? 2 : 0, shares = 2 * p.passes - skipped;
    Entry* place = w.a;
    for (int pass = 0; pass < p.passes; ++pass) {
      const Keys keys{tokens, sorted};
      const int shift = pass * p.bits;
      uint8_t* const marked = pass == 0 ? marks : nullptr;
      zeros.marks = pass == 0 ? nullptr : marks;
      Zeros z = share(2 * pass - skipped, shares, p.tiles, &grid);
      if (marked) { z.first = (unsigned)p.tiles; grid = dim3((unsigned)p.tiles + 16); }
      const auto with_keys = [&](auto f) { return with_width(p.keys, f); };
      rc = with_keys([&](auto k) {
        return launch_operator(count_digits_kernel<decltype(k)::value>, grid, kSortThreads, 0, s, keys, shift, p.bits, w.counts, reinterpret_cast<uint4*>(marked),
                               (vocab + 15) / 16, z);
      });
      if (rc != MONO_OK) return rc;
      if (p.coarse && (rc = launch_operator(sum_counts_kernel, dim3((unsigned)p.coarse), kSortThreads, 0, s, w.counts, p.tiles, w.coarse)) != MONO_OK) return rc;
      z = share(2 * pass + 1 - skipped, shares, p.tiles, &grid);
      rc = with_keys([&](auto k) {
        return launch_operator(scatter_keys_kernel<decltype(k)::value>, grid, kSortThreads, 0, s, keys, n, shift, p.bits, w.counts, p.tiles, p.coarse ? w.coarse : nullptr, place,
                               marked, z);
      });
      if (rc != MONO_OK) return rc;
      sorted = place;
      place = place == w.a ? w.b : w.a;
    }
  }
  const bool joins = sums.blocks >= 2 && n > kSmallTokens;
  const auto sum = [&](auto* kernel) {
    return launch_operator(kernel, sum_grid, kThreads, 0, s, from, (uint32_t)(grad.stride * (int64_t)sizeof(G)), tokens, sorted, sums.run, to, sums.part_vectors, sums.lanes, joins);
  };
  rc = accumulate ? sum(sum_rows_kernel<G, O, VEC, true>) : sum(sum_rows_kernel<G, O, VEC, false>);
  if (rc != MONO_OK || !joins) return rc;
  constexpr int JOINED = std::min(4, VEC);
  const int joined = cols / JOINED, threads = joined >= kThreads ? kThreads : (joined + 31) / 32 * 32;
  return launch_operator(join_rows_kernel<O, JOINED>, dim3((unsigned)(sums.blocks - 1), (unsigned)((joined + threads - 1) / threads)), threads, 0, s, sorted, n, sums.run * sums.groups,
                         accumulate, to);
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

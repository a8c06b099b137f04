// Rows in 4 bits (mono_pack_rows, mono_packed_token_rows, mono_packed_scores): kernels and host side.
#include <climits>

#include "operators.cuh"
#include "table_layout.cuh"

using namespace mono;

namespace {

constexpr int kThreads = 256;

struct PackedView {
  uint8_t* q;
  void* scales;
  int64_t rows, q_stride, scale_stride;
  int cols, groups;
};

inline bool packed_ok(const mono_packed_t* p) {
  if (!p || !element_size(p->scale_type) || (p->group != 32 && p->group != 64 && p->group != 128)) return false;
  if (p->rows < 0 || p->rows > kMaxOperatorRows || p->cols < 1 || p->cols > MONO_MAX_COLS) return false;
  if (p->rows == 0) return true;
  if (p->q_stride % 16 || p->q_stride < (p->cols + 31) / 32 * 16 || p->q_stride > MONO_MAX_STRIDE) return false;
  if (p->scale_stride < (p->cols + p->group - 1) / p->group || p->scale_stride > MONO_MAX_STRIDE) return false;
  return p->q && is_aligned(p->q, 16) && p->scales && is_aligned(p->scales, element_size(p->scale_type));
}

inline PackedView view(const mono_packed_t& p) {
  return {p.q, p.scales, p.rows, p.q_stride, p.scale_stride, (int)p.cols, (int)((p.cols + p.group - 1) / p.group)};
}

// ---------------------------------------------------------------------------
// Packing: 8 threads a group of columns, group / 8 neighbouring columns each, so that every thread writes whole bytes.  A block has the groups of
// blockIdx.y's share of kPackGroups / block_groups rows.  (131072 rows of 1024 columns: 171 us in fp32, 185 in bf16, where the bytes are 93 and 52: what bounds it is
// what a thread does for each column, rounding and the choice to divide.  With half as many columns a thread, single columns read and a 64-bit division to find them
// fp32 rows took 288.)
// ---------------------------------------------------------------------------
constexpr int kPackThreads = 8, kPackGroups = kThreads / kPackThreads;

template <typename W, typename S, int GROUP, bool VECTORS>
__global__ void __launch_bounds__(kThreads) pack_rows_kernel(const W* rows, int64_t stride, PackedView p, int block_groups) {
  after_previous_kernel();
  constexpr int N = GROUP / kPackThreads, V = N < 8 ? N : 8;
  const int lane = threadIdx.x % kPackThreads, sub = threadIdx.x / kPackThreads;
  const int64_t row = (int64_t)blockIdx.x * (kPackGroups / block_groups) + sub / block_groups;
  const int g = blockIdx.y * block_groups + sub % block_groups, c0 = g * GROUP + lane * N;
  if (row >= p.rows || g >= p.groups) return;               // (all threads of a group)
  const unsigned members = 0xFFu << (threadIdx.x & 24);
  const W* const from = rows + row * stride + c0;
  float w[N];
  if (VECTORS && c0 + N <= p.cols) {
#pragma unroll
    for (int i = 0; i < N; i += V) to_floats(*reinterpret_cast<const Vec<W, V>*>(from + i), reinterpret_cast<float(&)[V]>(w[i]));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = c0 + i < p.cols ? to_float(from[i]) : 0.0f;
  }
  float most = 0.0f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    most = fmaxf(most, fabsf(w[i]));                        // (fmaxf passes over a NaN)
    nan |= w[i] != w[i];
  }
#pragma unroll
  for (int s = kPackThreads / 2; s > 0; s /= 2) most = fmaxf(most, __shfl_xor_sync(members, most, s));
  nan = __any_sync(members, nan);
  const S stored = from_float<S>(nan ? __int_as_float(0x7FC00000) : __fdiv_rn(most, 7.0f));
  const float scale = to_float(stored);
  const bool usable = scale > 0.0f && scale <= 3.402823466e38f;
  // The quotient rounded to a whole number.  By the reciprocal it is off by less than 2^-22 of itself, which is below 2^-18 for the numbers up to 16
  // (beyond, it is held to 7 either way): only where it is that near to a half the quotient itself has to say.
  const float inverse = __fdiv_rn(1.0f, scale);
  const bool exactly = !(inverse <= 3.402823466e38f);       // (a scale so small that it has none)
  uint64_t bytes = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float quotient = w[i] * inverse;
    float r = rintf(quotient);
    if (exactly || fabsf(fabsf(quotient - r) - 0.5f) < 1.0f / 65536.0f) r = rintf(__fdiv_rn(w[i], scale));
    r = usable ? fminf(fmaxf(r, -7.0f), 7.0f) : 0.0f;
    bytes |= (uint64_t)(uint32_t)((int)r + 8) << (4 * i);
  }
  const int at = c0 / 2, padded = (p.cols + 31) / 32 * 16;  // bytes of a row that are written
  uint8_t* const to = p.q + row * p.q_stride + at;
  if (at < padded) {                                        // (a multiple of 16: all of a thread's bytes or none)
    if constexpr (N == 16) *reinterpret_cast<uint64_t*>(to) = bytes;
    else if constexpr (N == 8) *reinterpret_cast<uint32_t*>(to) = (uint32_t)bytes;
    else *reinterpret_cast<uint16_t*>(to) = (uint16_t)bytes;
  }
  if (lane == 0) static_cast<S*>(p.scales)[row * p.scale_stride + g] = stored;
}

// ---------------------------------------------------------------------------
// Rows by token of packed rows.  A thread makes the 8 columns of a 32-bit word, and keeps four words and their scales in flight behind the read
// of its tokens: four of one row where rows are wide, one of each of four rows where `lanes` threads cover a row.  (262144 tokens of 128 columns, bf16 out: 19.5 us, of
// which the bytes are 11; issue slots are 82 % used.  Where 8 does not divide the columns, a column takes two shuffles and a store: 65536 tokens of
// 130 columns 18 us, of 128 columns 6.)
// ---------------------------------------------------------------------------
constexpr int kMoves = 4;

template <typename S, typename O, bool ALIGNED, int ROWS>
__global__ void __launch_bounds__(kThreads) packed_token_rows_kernel(PackedView p, int group_shift, TokenList tokens, float scale, O* __restrict__ out, int64_t out_stride, int lanes) {
  after_previous_kernel();
  constexpr int PIECES = kMoves / ROWS;
  const int lane = threadIdx.x & (lanes - 1), groups = kThreads / lanes;
  const int64_t row0 = (int64_t)blockIdx.x * groups * ROWS + threadIdx.x / lanes;
  const int words = (p.cols + 7) / 8, w0 = blockIdx.y * lanes * PIECES + lane;
  uint32_t t[ROWS], q[kMoves];
  float s[kMoves];
  tokens.rows(row0, groups, t);
#pragma unroll
  for (int k = 0; k < kMoves; ++k) {
    const uint32_t row = t[k / PIECES];
    const int w = w0 + (k % PIECES) * lanes;
    q[k] = 0x88888888u;                                       // (zeros)
    s[k] = 0.0f;
    if (row != kNoToken && w < words) {
      q[k] = reinterpret_cast<const uint32_t*>(p.q + row * p.q_stride)[w];
      s[k] = to_float(static_cast<const S*>(p.scales)[row * p.scale_stride + (w >> group_shift)]);
    }
  }
  // q as the lowest bits of 2^23, less 2^23 + 8; without a row all factors are 0
  const uint32_t mask = 15u, bits = kept(0x4B000000u);
#pragma unroll
  for (int k = 0; k < kMoves; ++k) {
    const int64_t i = row0 + (k / PIECES) * groups;
    const int w = w0 + (k % PIECES) * lanes;
    const float by = t[k / PIECES] != kNoToken ? scale : 0.0f;
    float f[8];
    if constexpr (ALIGNED) {
      if (i >= tokens.n || w >= words) continue;
#pragma unroll
      for (int c = 0; c < 8; ++c) f[c] = __uint_as_float(place(q[k] >> (4 * c), mask, bits));
      move_floats(f, -8388616.0f);
      scale_floats(f, s[k]);
      scale_floats(f, by);
      *reinterpret_cast<Vec<O, 8>*>(out + i * out_stride + (int64_t)w * 8) = from_floats<O>(f);
    } else {
      // one column a thread and store, so that neighbours write neighbours: the words are passed round
      const int near = min(lanes, 32), in = threadIdx.x & (near - 1);
      O* const to = out + i * out_stride + (int64_t)(w - in) * 8;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int at = c * near + in;                        // among the columns of the threads near by
        const uint32_t word = __shfl_sync(0xFFFFFFFFu, q[k], at / 8, near);
        const float factor = __shfl_sync(0xFFFFFFFFu, s[k], at / 8, near);
        const float y = by * ((__uint_as_float(place(word >> (4 * (at % 8)), mask, bits)) - 8388616.0f) * factor);
        if (i < tokens.n && (w - in) * 8 + at < p.cols) to[at] = from_float<O>(y);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Scores.  out[m, v] = sum over groups g of s[v, g] * (sum over c in g of x[m, c] * (q[v, c] - 8)).
//
// The bytes of q would bound it (half a byte for 2 * m operations) if a weight became an operand in few enough instructions: the tensor
// cores' 16-bit products take 16 rows and 8 vectors at once.  As the bits of an fp16, 4 bits in the lowest places are q * 2^-24 and in
// the next ones 16 * q * 2^-24, subnormal and exact; times 2^14 or 2^10, less 8 * 2^-10, they are (q - 8) * 2^-10: an AND and
// a multiply-add for two weights, and a shift for each eight.  (Left subnormal, with the 8 taken off the sums, they took 71 us instead of
// 75 for 8 vectors against 131072 rows of 4096 columns, and the sums lost three bits.)
// Vectors become fp16 operands: those of a group are multiplied by the power of two that takes the largest of them to 2^15 .. 2^16, and an
// fp32 vector is three operands whose sum it is, the second and third times 2^11 and 2^22, so that each has 11 bits of its own however small
// an element is beside the others.  With fp16's least number, 2^-24, that leaves fp32 elements as they are down to 2^-38 of the group's largest (below,
// they are off by at most 2^-62 of it), bf16 ones down to 2^-32 (2^-40), and all fp16 ones.  (A bf16 vector in two operands would have the
// fp32 one's range for twice the products.)  All products are exact, all sums in fp32.
//
// In a product of mma.m16n8k16 the columns are summed over, so any may stand in any place, as long as the vectors' are in the same.
// So thread t of the four that share a row takes the t-th quarter of a group's bytes as they lie, and what the masks select of a word, columns p
// and p + 4, is a pair for the product.  The vectors are laid out in shared memory to match, once per block.
//
// A warp has 32 rows at a time, so that what it reads of the vectors serves two products, and moves 256 columns of them (128 bytes of each) to
// shared memory of its own, kStages - 1 moves ahead of the products.  (Straight into registers, the eight rows of a load are eight short
// pieces: 8 vectors against 131072 rows of 4096 columns took 84 us when they took 80 this way; 128 columns a move 75, 256 now 73.)  Where there
// are few rows, `split` warps share 32 rows, a run of columns each.  Scales are read ahead by the four threads of a row, one each.
//
// Measured: 73 us for those, 3.8 TB/s; one vector against them 58, against 50001 rows of 1024 columns 8.9, against a million of 128 columns 31 (a stage is
// 32 rows, however short they are: 2.3 TB/s).  Nothing is used up (for 8 vectors issue slots 60 %, ALU pipe 47 %, tensor cores 25 %, HBM 58 %): with three warps a scheduler, which
// is what the vectors' operands in shared memory leave room for, it is the way from the stage through operands and products to the sums, one after the other, and
// reading the vectors' operands, as many bytes from shared memory as the weights.  For 16 vectors, or rows of more than 4096 columns, there are fewer warps still
// (16 against 50000 rows of 2048 columns: 37 us, of which the bytes are 8.6).
// ---------------------------------------------------------------------------
constexpr int kTileRows = 32;
constexpr int kBlockColumns = 256, kBlockBytes = kBlockColumns / 2;
constexpr int kRowMoves = kBlockBytes / 16, kMoveRows = 32 / kRowMoves;      // 16-byte moves of a row, rows of a warp's moves
constexpr int kMostWarps = 12;
constexpr int kStages = 3;
constexpr int kStageBytes = kTileRows * kBlockBytes;

template <typename X> struct PartsOf { static constexpr int value = 1; };
template <> struct PartsOf<float> { static constexpr int value = 3; };

// d = a * b + c
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1, float c2, float c3) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
// (q - 8) * 2^-10 of two weights, of q * 2^-24 (by 2^14) or 16 * q * 2^-24 (by 2^10)
__device__ __forceinline__ uint32_t weights(uint32_t q, uint32_t by) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(q), "r"(by), "r"(0xA000A000u));
  return r;
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }      // -126 <= e <= 127

__device__ __forceinline__ void store_as(void* to, int type, int64_t i, float y) {
  if (type == MONO_F32) static_cast<float*>(to)[i] = y;
  else if (type == MONO_BF16) static_cast<__nv_bfloat16*>(to)[i] = from_float<__nv_bfloat16>(y);
  else static_cast<__half*>(to)[i] = from_float<__half>(y);
}

template <int BYTES> struct alignas(BYTES) Words { uint32_t w[BYTES / 4]; };

// Shared memory: the warps' stages, [warps][kStages][32][128 bytes]; the vectors, [words of a quarter row][columns][4 threads][4 pairs]; of each group, [4 * NT]
// pairs of columns: the powers of two that their sums are multiplied by; the sums of the warps, [warps][32][8 * NT].  `columns` operands:
// vectors, or the parts of vectors.
template <typename X, typename S, int GROUP, int NT>
__global__ void __launch_bounds__(kMostWarps * 32, 1) packed_scores_kernel(PackedView p, const X* x, int64_t x_stride, int vectors, void* __restrict__ out, int out_type,
                                                               int64_t out_stride, int split, int64_t tiles) {
  after_previous_kernel();
  constexpr int PARTS = PartsOf<X>::value;
  constexpr int BYTES = GROUP / 8, WORDS = BYTES / 4;       // of a row's group, a thread's quarter
  constexpr int U = kBlockColumns / GROUP;                  // groups of a stage
  constexpr int SETS = kTileRows / 8;                       // rows of a thread: g, g + 8, ...
  constexpr int N = 8 * NT;
  extern __shared__ __align__(128) uint4 shared[];
  const int warps = blockDim.x / 32, columns = vectors * PARTS;
  const int row_words = p.groups * WORDS;                   // of a thread's quarter
  uint4* const operands = shared + warps * kStages * (kStageBytes / 16);
  float2* const groups = reinterpret_cast<float2*>(operands + row_words * columns * 4);
  float* const sums = reinterpret_cast<float*>(groups + p.groups * 4 * NT);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const int share = warp % split, team = warp / split, teams = warps / split;
  const int blocks = (p.groups + U - 1) / U, per = (blocks + split - 1) / split;
  const int k0 = min(share * per, blocks), k1 = min(k0 + per, blocks);      // this warp's blocks of columns
  const int row_bytes = (p.cols + 31) / 32 * 16;
  const int64_t step = (int64_t)gridDim.x * teams, tile0 = (int64_t)blockIdx.x * teams + team;

  // A stage: the lane has 16 bytes of every kMoveRows-th row.  Where they go is turned by the row, so that the threads that read a group
  // together (of two, four or eight rows at a time) find their bytes in different banks.
  uint4* const stages = shared + warp * kStages * (kStageBytes / 16);
  const auto turned = [](int row, int piece) {
    const int turn = row / (8 / kRowMoves);                 // (rows that lie in the same banks)
    return row * kRowMoves + (piece ^ ((GROUP == 128 ? turn << 2 : GROUP == 64 ? turn << 1 : turn) & (kRowMoves - 1)));
  };
  const int move_row = lane / kRowMoves, move_at = lane % kRowMoves * 16;
  int64_t fill_tile = tile0;
  int fill_k = k0, fill_stage = 0;
  const uint8_t* fill_from[kTileRows / kMoveRows];          // the lane's bytes of its rows
  const auto fill = [&] {
    if (fill_tile < tiles) {
      if (fill_k == k0) {
#pragma unroll
        for (int i = 0; i < kTileRows / kMoveRows; ++i)
          fill_from[i] = p.q + min(fill_tile * kTileRows + move_row + kMoveRows * i, p.rows - 1) * p.q_stride + (k0 * kBlockBytes + move_at);
      }
      if (fill_k * kBlockBytes + move_at < row_bytes) {     // (behind the row's end the vectors are zero, whatever the stage holds)
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(stages) + fill_stage * kStageBytes;
#pragma unroll
        for (int i = 0; i < kTileRows / kMoveRows; ++i) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + turned(move_row + kMoveRows * i, lane % kRowMoves) * 16), "l"(fill_from[i]) : "memory");
          fill_from[i] += kBlockBytes;
        }
      }
      if (++fill_k >= k1) { fill_k = k0; fill_tile += step; }
    }
    fill_stage = fill_stage + 1 == kStages ? 0 : fill_stage + 1;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int s = 0; s < kStages - 1; ++s) fill();

  // The vectors as operands: a thread has 8 neighbouring columns, GROUP / 8 threads a group.
  for (int i = threadIdx.x; i < p.groups * 4 * NT; i += blockDim.x) groups[i] = make_float2(0.0f, 0.0f);
  __syncthreads();
  {
    const int eights = p.groups * (GROUP / 8), items = eights * vectors, rounds = (items + blockDim.x - 1) / blockDim.x;
    for (int round = 0; round < rounds; ++round) {
      const int i = round * blockDim.x + threadIdx.x, m = min(i / eights, vectors - 1), c0 = (i - m * eights) * 8;
      const X* from = x + m * x_stride;
      float v[8];
      uint32_t most = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] = i < items && c0 + k < p.cols ? to_float(from[c0 + k]) : 0.0f;
        const uint32_t size = __float_as_uint(v[k]) & 0x7FFFFFFFu;
        if (size < 0x7F800000u) most = max(most, size);
      }
#pragma unroll
      for (int s = GROUP / 16; s > 0; s /= 2) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, s));
      // of the largest's exponent; the least that leaves the third part's factor a normal number, and no element loses by it: 2^-149 is 2^-35 in an operand
      const int e = max((int)(most >> 23) - 127, -99);
      const float up = power_of_two(15 - e);
      __half part[PARTS][8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float left = v[k] * up;
#pragma unroll
        for (int j = 0; j < PARTS; ++j) {
          // (cut, so that what is left has the same sign and fewer bits; of what is not finite nothing is left)
          part[j][k] = j + 1 < PARTS ? __float2half_rz(left) : __float2half_rn(left);
          left = fabsf(left) < 65536.0f ? (left - __half2float(part[j][k])) * 2048.0f : 0.0f;
          if (PARTS > 1 && j == 0 && !(fabsf(v[k]) <= 3.402823466e38f)) part[j][k] = __float2half_rn(v[k]);
        }
      }
      if (i >= items) continue;
      const int group = c0 / GROUP, in = c0 % GROUP, word = group * WORDS + in % (GROUP / 4) / 8;
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int col = m * PARTS + j;
        __half e8[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) e8[2 * k] = part[j][k], e8[2 * k + 1] = part[j][k + 4];
        memcpy(&operands[(word * columns + col) * 4 + in / (GROUP / 4)], e8, sizeof(uint4));
        if (in == 0) {
          // what turns the operands' sums into the group's: from -126 to 122.  (Taken off the scale or off the product instead, part of it made sums
          // overflow that fp32 has room for, and took bits off subnormal scales.)
          reinterpret_cast<float*>(&groups[group * 4 * NT + col / 2])[col % 2] = power_of_two(e - 5 - 11 * j);
        }
      }
    }
  }

  constexpr int SCALES = (U + 3) / 4;
  S scales[SETS][SCALES];                                   // of groups t, t + 4 (modulo U) of the next block of columns
  const S* scale_row[SETS];
  const auto load_scales = [&](int64_t tile, int k) {
    if (k == k0) {
#pragma unroll
      for (int j = 0; j < SETS; ++j) scale_row[j] = static_cast<const S*>(p.scales) + min(tile * kTileRows + g + 8 * j, p.rows - 1) * p.scale_stride;
    }
#pragma unroll
    for (int u = 0; u < SCALES; ++u) {
      const int at = min(k * U + u * 4 + (t & (U - 1)), p.groups - 1);
#pragma unroll
      for (int j = 0; j < SETS; ++j) scales[j][u] = scale_row[j][at];
    }
  };
  if (tile0 < tiles) load_scales(tile0, k0);
  int operand[NT];                                          // in shared[]; for a column that there is none of another one's: its sums are not written
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) operand[nt] = (int)(operands - shared) + (k0 * U * WORDS * columns + min(nt * 8 + g, columns - 1)) * 4 + t;
  const int operand_step = columns * 4;
  const uint32_t by14 = kept(0x74007400u), by10 = kept(0x64006400u);      // 2^14, 2^10
  const int stage_bytes = warp * kStages * kStageBytes;     // where the warp's stages begin in shared[]
  int stage = 0;
  __syncthreads();

  for (int64_t tile = tile0; tile < tiles; tile += step) {
    float total[SETS / 2][NT][4] = {};
    int at_operand[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) at_operand[nt] = operand[nt];
    for (int k = k0; k < k1; ++k) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      __syncwarp();                                         // the stage is there for the warp, and it is done with the one that is filled now
      fill();
      S own[SETS][SCALES];
#pragma unroll
      for (int j = 0; j < SETS; ++j) {
#pragma unroll
        for (int u = 0; u < SCALES; ++u) own[j][u] = scales[j][u];
      }
      const bool same = k + 1 < k1;
      if (same || tile + step < tiles) load_scales(same ? tile : tile + step, same ? k + 1 : k0);
      const int from = stage_bytes + stage * kStageBytes;
      stage = stage + 1 == kStages ? 0 : stage + 1;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k * U + u >= p.groups) break;
        Words<BYTES> words[SETS];
        const int at = (u * 4 + t) * BYTES;                 // in the row's bytes
#pragma unroll
        for (int j = 0; j < SETS; ++j) words[j] = *reinterpret_cast<const Words<BYTES>*>(reinterpret_cast<const char*>(shared) + (from + turned(g + 8 * j, at / 16) * 16 + at % 16));
        float2 of_group[NT];                                // of columns 2 * t and the one behind it
        float sum[SETS / 2][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) of_group[nt] = groups[(k * U + u) * 4 * NT + nt * 4 + t];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          uint4 b[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            b[nt] = shared[at_operand[nt]];
            at_operand[nt] += operand_step;
          }
#pragma unroll
          for (int j = 0; j < SETS / 2; ++j) {
            uint32_t a[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t w0 = words[2 * j].w[w] >> (8 * h), w1 = words[2 * j + 1].w[w] >> (8 * h);
              a[h][0] = weights(w0 & 0x000F000Fu, by14);
              a[h][1] = weights(w1 & 0x000F000Fu, by14);
              a[h][2] = weights(w0 & 0x00F000F0u, by10);
              a[h][3] = weights(w1 & 0x00F000F0u, by10);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float(&d)[4] = sum[j][nt];
              if (w == 0) mma(d, a[0], b[nt].x, b[nt].y, 0.0f, 0.0f, 0.0f, 0.0f);
              else mma(d, a[0], b[nt].x, b[nt].y, d[0], d[1], d[2], d[3]);
              mma(d, a[1], b[nt].z, b[nt].w, d[0], d[1], d[2], d[3]);
            }
          }
        }
        // of_group: the operands' powers of two and the weights' 2^-10, taken back
#pragma unroll
        for (int j = 0; j < SETS; ++j) {
          const float f = __shfl_sync(0xFFFFFFFFu, to_float(own[j][u / 4]), (lane & ~3) | (u % 4));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            total[j / 2][nt][j % 2 * 2] += f * (of_group[nt].x * sum[j / 2][nt][j % 2 * 2]);
            total[j / 2][nt][j % 2 * 2 + 1] += f * (of_group[nt].y * sum[j / 2][nt][j % 2 * 2 + 1]);
          }
        }
      }
    }
    float* const mine = sums + warp * kTileRows * N;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < SETS; ++j)
        *reinterpret_cast<float2*>(mine + (g + 8 * j) * N + nt * 8 + 2 * t) = make_float2(total[j / 2][nt][j % 2 * 2], total[j / 2][nt][j % 2 * 2 + 1]);
    }
    // the team's warps alone wait for one another
    const auto wait = [&] {
      if (split == 1) __syncwarp();
      else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(split * 32) : "memory");
    };
    wait();
    const int64_t row0 = tile * kTileRows;
    for (int i = share * 32 + lane; i < kTileRows * vectors; i += split * 32) {
      const int r = i % kTileRows, m = i / kTileRows;
      if (row0 + r >= p.rows) continue;
      const float* from = sums + team * split * kTileRows * N + r * N + m * PARTS;
      float y = 0.0f;
      for (int w = 0; w < split; ++w) {
#pragma unroll
        for (int k = PARTS - 1; k >= 0; --k) y += from[w * kTileRows * N + k];      // (the small parts first)
      }
      store_as(out, out_type, m * out_stride + row0 + r, y);
    }
    wait();
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Of a block with so many warps, for so many operand vectors.
inline size_t scores_shared(int warps, int64_t groups, int group, int columns, int nt) {
  return (size_t)warps * kStages * kStageBytes + (size_t)groups * (group / 32) * columns * 64 + (size_t)groups * 32 * nt + (size_t)warps * kTileRows * 8 * nt * 4;
}
constexpr size_t kMostShared = 227 * 1024;

template <typename X, typename S, int GROUP, int NT>
int launch_scores_tile(const PackedView& p, const X* x, int64_t x_stride, int vectors, void* out, int out_type, int64_t out_stride, cudaStream_t s) {
  auto* kernel = packed_scores_kernel<X, S, GROUP, NT>;
  const int columns = vectors * PartsOf<X>::value;
  const int64_t tiles = (p.rows + kTileRows - 1) / kTileRows, blocks = ((int64_t)p.groups * GROUP + kBlockColumns - 1) / kBlockColumns;
  int warps = kMostWarps;
  while (warps > 8 && scores_shared(warps, p.groups, GROUP, columns, NT) > kMostShared) warps -= 4;
  while (scores_shared(warps, p.groups, GROUP, columns, NT) > kMostShared) warps /= 2;
  // warps share a tile where that makes the longest warp's work shorter: its rounds over the tiles, each its blocks of columns and
  // (measured: about half a block's time) what the sums' end takes
  int split = 1;
  double best = 0.0;
  for (int n = 1; warps % n == 0 && n <= 8 && n <= blocks; n *= 2) {
    const int64_t teams = 148ll * (warps / n), rounds = (tiles + teams - 1) / teams;
    const double cost = (double)rounds * ((double)((blocks + n - 1) / n) + 0.6);
    if (n == 1 || cost < best) split = n, best = cost;
  }
  // small blocks where there is little for all SMs
  while (warps / 2 % split == 0 && warps > 3 && tiles * split <= 148ll * warps / 2) warps /= 2;
  const size_t shared = scores_shared(warps, p.groups, GROUP, columns, NT);
  const int teams = warps / split;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared) != cudaSuccess) return MONO_ERR_CUDA;
  const int64_t grid = std::min<int64_t>((tiles + teams - 1) / teams, 148);
  return launch_operator(kernel, dim3((unsigned)grid), warps * 32, shared, s, p, x, x_stride, vectors, out, out_type, out_stride, split, tiles);
}

template <typename X, typename S, int GROUP>
int launch_scores(const mono_packed_t& packed, const mono_matrix_t& x, const mono_matrix_t& out, cudaStream_t s) {
  constexpr int PARTS = PartsOf<X>::value;
  const PackedView p = view(packed);
  // vectors of a launch: up to 16 operands, and no more than shared memory has room for beside the stages of two warps
  int most = 16 / PARTS;
  while (most > 1 && scores_shared(2, p.groups, GROUP, most * PARTS, 2) > kMostShared) --most;
  for (int64_t m = 0; m < x.rows; m += most) {
    const int vectors = (int)std::min<int64_t>(most, x.rows - m);
    const X* from = static_cast<const X*>(x.data) + m * x.stride;
    char* to = static_cast<char*>(out.data) + m * out.stride * element_size(out.type);
    const int rc = vectors * PARTS <= 8 ? launch_scores_tile<X, S, GROUP, 1>(p, from, x.stride, vectors, to, out.type, out.stride, s)
                                        : launch_scores_tile<X, S, GROUP, 2>(p, from, x.stride, vectors, to, out.type, out.stride, s);
    if (rc != MONO_OK) return rc;
  }
  return MONO_OK;
}

template <typename F>
int with_group(int group, F&& f) {
  return group == 32 ? f(Width<32>()) : group == 64 ? f(Width<64>()) : f(Width<128>());
}

}  // namespace

extern "C" {

int mono_pack_rows(const mono_matrix_t* rows, const mono_packed_t* packed, void* cuda_stream) {
  const OperatorRange range(__func__);
  if (!matrix_ok(rows, false) || !packed_ok(packed) || rows->rows != packed->rows || rows->cols != packed->cols) return MONO_ERR_ARG;
  if (packed->rows == 0) return MONO_OK;
  const PackedView p = view(*packed);
  int block_groups = 1;
  while (block_groups < kPackGroups && block_groups < p.groups) block_groups *= 2;
  const int64_t block_rows = kPackGroups / block_groups;
  const dim3 grid((unsigned)((p.rows + block_rows - 1) / block_rows), (unsigned)((p.groups + block_groups - 1) / block_groups));
  const int vectors = vector_of({rows->data, rows->rows, (p.cols + 7) / 8 * 8, rows->stride, rows->type, 0});      // (of a row's whole vectors)
  return with_type(rows->type, [&](auto w) {
    return with_type(packed->scale_type, [&](auto s) {
      return with_group(packed->group, [&](auto g) {
        using W = decltype(w);
        using S = decltype(s);
        constexpr int GROUP = decltype(g)::value;
        const auto launch = [&](auto* kernel) {
          return launch_operator(kernel, grid, kThreads, 0, static_cast<cudaStream_t>(cuda_stream), static_cast<const W*>(rows->data), rows->stride, p, block_groups);
        };
        return vectors >= std::min(8, GROUP / kPackThreads) ? launch(pack_rows_kernel<W, S, GROUP, true>) : launch(pack_rows_kernel<W, S, GROUP, false>);
      });
    });
  });
}

int mono_packed_token_rows(const mono_packed_t* packed, const void* tokens, int32_t token_type, int64_t n_tokens, int64_t padding, float scale, const mono_matrix_t* out,
                           void* cuda_stream) {
  const OperatorRange range(__func__);
  if (!packed_ok(packed) || !matrix_ok(out, true) || !tokens_ok(tokens, token_type, n_tokens)) return MONO_ERR_ARG;
  if (out->rows != n_tokens || out->cols != packed->cols) return MONO_ERR_ARG;
  if (n_tokens == 0) return MONO_OK;
  const PackedView p = view(*packed);
  const TokenList list{tokens, n_tokens, packed->rows, padding, token_type == MONO_I64};
  const int words = (p.cols + 7) / 8;
  int lanes = 1;
  const bool wide = words > 64;
  while (wide ? lanes < kThreads && lanes * kMoves < words : lanes < words) lanes *= 2;
  const int64_t rows = (int64_t)(kThreads / lanes) * (wide ? 1 : kMoves), columns = (int64_t)lanes * (wide ? kMoves : 1);
  const dim3 grid((unsigned)((n_tokens + rows - 1) / rows), (unsigned)((words + columns - 1) / columns));
  return with_type(packed->scale_type, [&](auto s) {
    return with_type(out->type, [&](auto o) {
      using S = decltype(s);
      using O = decltype(o);
      const auto launch = [&](auto* kernel) {
        return launch_operator(kernel, grid, kThreads, 0, static_cast<cudaStream_t>(cuda_stream), p, packed->group == 32 ? 2 : packed->group == 64 ? 3 : 4, list, scale, static_cast<O*>(out->data), out->stride, lanes);
      };
      if (vector_of(*out) == 8) return wide ? launch(packed_token_rows_kernel<S, O, true, 1>) : launch(packed_token_rows_kernel<S, O, true, 4>);
      return wide ? launch(packed_token_rows_kernel<S, O, false, 1>) : launch(packed_token_rows_kernel<S, O, false, 4>);
    });
  });
}

int mono_packed_scores(const mono_packed_t* packed, const mono_matrix_t* x, const mono_matrix_t* out, void* cuda_stream) {
  const OperatorRange range(__func__);
  if (!packed_ok(packed) || !matrix_ok(x, false) || !out || out->rows != x->rows || x->cols != packed->cols) return MONO_ERR_ARG;
  if (x->rows > MONO_MAX_SCORED || x->cols > MONO_MAX_SCORED_COLS) return MONO_ERR_LIMIT;
  if (out->cols != packed->rows) return MONO_ERR_ARG;
  if (packed->rows == 0 || x->rows == 0) return MONO_OK;
  // (a row of scores is as long as there are rows: not a matrix of at most MONO_MAX_COLS columns)
  const int size = element_size(out->type);
  if (!size || !out->data || !is_aligned(out->data, size) || out->stride < 0 || out->stride > kMaxOperatorRows || (out->rows > 1 && out->stride < out->cols)) return MONO_ERR_ARG;
  return with_type(x->type, [&](auto xt) {
    return with_type(packed->scale_type, [&](auto s) {
      return with_group(packed->group, [&](auto g) {
        return launch_scores<decltype(xt), decltype(s), decltype(g)::value>(*packed, *x, *out, static_cast<cudaStream_t>(cuda_stream));
      });
    });
  });
}

}  // extern "C"

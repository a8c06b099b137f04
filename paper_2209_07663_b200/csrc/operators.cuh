// What the operators on plain matrices (token_rows.cu, packed_rows.cu) share: the element types, checked
// views of the caller's matrices, vectors of elements, and launches.
#pragma once

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <type_traits>
#include <utility>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "../../include/mono.h"

namespace mono {

// profiler range of one call, named after the entry point
struct OperatorRange {
  explicit OperatorRange(const char* name) { nvtxRangePushA(name); }
  ~OperatorRange() { nvtxRangePop(); }
};

__device__ __forceinline__ float to_float(float x) { return x; }
// (its bits are the upper half of the float's)
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __uint_as_float((uint32_t)__bfloat16_as_ushort(x) << 16); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
// (to nearest, ties to even: an output is rounded once, here)
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// N consecutive elements, moved in accesses of up to 16 bytes
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Vec { T v[N]; };

template <typename T, int N>
__device__ __forceinline__ void to_floats(const Vec<T, N>& x, float (&f)[N]) {
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
    // two at a time: a bf16 pair's upper half is a float already, but for the bits below
    uint32_t w[N / 2];
    memcpy(w, &x, sizeof(w));
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        f[2 * k] = __uint_as_float(w[k] << 16);
        f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      } else {
        __half2 h;
        memcpy(&h, &w[k], 4);
        const float2 p = __half22float2(h);
        f[2 * k] = p.x;
        f[2 * k + 1] = p.y;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = to_float(x.v[k]);
  }
}

// rounded once each, two at a time where two fit a register
template <typename T, int N>
__device__ __forceinline__ Vec<T, N> from_floats(const float (&f)[N]) {
  Vec<T, N> x;
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(f[k], f[k + 1]);
        memcpy(&x.v[k], &p, 4);
      } else {
        const __half2 p = __floats2half2_rn(f[k], f[k + 1]);
        memcpy(&x.v[k], &p, 4);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x.v[k] = from_float<T>(f[k]);
  }
  return x;
}

// 8 elements of 16 bits from any address: the two aligned 16-byte words that hold them, moved by as many bytes as the first one begins
// behind a multiple of 16.  Both words have to be readable.
template <typename T>
__device__ __forceinline__ void load_shifted(const T* from, uint32_t (&w)[8]) {
  static_assert(sizeof(T) == 2, "");
  const uint4* const at = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(from) & ~(uintptr_t)15);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint4 x = at[k];
    w[4 * k] = x.x, w[4 * k + 1] = x.y, w[4 * k + 2] = x.z, w[4 * k + 3] = x.w;
  }
}
template <typename T>
__device__ __forceinline__ Vec<T, 8> shifted(const uint32_t (&in)[8], uint32_t bytes) {
  uint32_t w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = in[k];
#pragma unroll
  for (int k = 0; k < 6; ++k) w[k] = bytes & 8 ? w[k + 2] : w[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) w[k] = bytes & 4 ? w[k + 1] : w[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], (bytes & 2) * 8);
  Vec<T, 8> x;
  memcpy(&x, w, sizeof(x));
  return x;
}

// sum += x, two columns an instruction
template <int N>
__device__ __forceinline__ void add_floats(float (&sum)[N], const float (&x)[N]) {
  if constexpr (N % 2 == 0) {
#pragma unroll
    for (int k = 0; k < N; k += 2)
      asm("{.reg .b64 a, b; mov.b64 a, {%0, %1}; mov.b64 b, {%2, %3}; add.rn.f32x2 a, a, b; mov.b64 {%0, %1}, a;}" : "+f"(sum[k]), "+f"(sum[k + 1]) : "f"(x[k]), "f"(x[k + 1]));
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] += x[k];
  }
}

// x *= by, and x += by
template <int N>
__device__ __forceinline__ void scale_floats(float (&x)[N], float by) {
  if constexpr (N % 2 == 0) {
#pragma unroll
    for (int k = 0; k < N; k += 2)
      asm("{.reg .b64 a, b; mov.b64 a, {%0, %1}; mov.b64 b, {%2, %2}; mul.rn.f32x2 a, a, b; mov.b64 {%0, %1}, a;}" : "+f"(x[k]), "+f"(x[k + 1]) : "f"(by));
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] *= by;
  }
}
template <int N>
__device__ __forceinline__ void move_floats(float (&x)[N], float by) {
  float b[N];
#pragma unroll
  for (int k = 0; k < N; ++k) b[k] = by;
  add_floats(x, b);
}

// (w & mask) | bits in one instruction: with both constants written out the compiler makes two
__device__ __forceinline__ uint32_t place(uint32_t w, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(bits));
  return r;
}
__device__ __forceinline__ uint32_t kept(uint32_t constant) {
  uint32_t r;
  asm volatile("mov.b32 %0, %1;" : "=r"(r) : "r"(constant));
  return r;
}

constexpr uint32_t kNoToken = 0xFFFFFFFFu;
constexpr int64_t kMaxOperatorRows = 0x7FFFFFFEll;      // of a matrix, and tokens of a call

// The caller's tokens: 32 or 64 bits, signed.
struct TokenList {
  const void* data;
  int64_t n;
  int64_t vocab;
  int64_t padding;
  bool wide;
  // the row that a token names, or kNoToken: outside the vocabulary, or the padding
  __device__ __forceinline__ uint32_t row_of(int64_t t) const { return (uint64_t)t < (uint64_t)vocab && t != padding ? (uint32_t)t : kNoToken; }
  __device__ __forceinline__ uint32_t at(int64_t i) const {
    return row_of(wide ? static_cast<const int64_t*>(data)[i] : static_cast<const int32_t*>(data)[i]);
  }
  // those of the K tokens first, first + step, ... (kNoToken behind the last one), all read before the first is looked at
  template <int K>
  __device__ __forceinline__ void rows(int64_t first, int64_t step, uint32_t (&row)[K]) const {
    int64_t t[K];
    if (wide) {
#pragma unroll
      for (int k = 0; k < K; ++k) t[k] = first + k * step < n ? static_cast<const long long*>(data)[first + k * step] : -1;
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) t[k] = first + k * step < n ? static_cast<const int*>(data)[first + k * step] : -1;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) row[k] = row_of(t[k]);
  }
};

inline int element_size(int32_t type) { return type == MONO_F32 ? 4 : type == MONO_BF16 || type == MONO_F16 ? 2 : 0; }
inline bool is_aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Whether m describes a matrix that can be read, or written (then no two of its rows may overlap).
inline bool matrix_ok(const mono_matrix_t* m, bool written) {
  if (!m) return false;
  const int size = element_size(m->type);
  if (!size || m->rows < 0 || m->rows > kMaxOperatorRows || m->cols < 1 || m->cols > MONO_MAX_COLS) return false;
  if (m->rows == 0) return true;
  if (m->stride < 0 || m->stride > MONO_MAX_STRIDE || (written && m->rows > 1 && m->stride < m->cols)) return false;
  return m->data && is_aligned(m->data, size);
}

inline bool tokens_ok(const void* tokens, int32_t type, int64_t n) {
  const int size = type == MONO_I32 ? 4 : type == MONO_I64 ? 8 : 0;
  return size && n >= 0 && n <= kMaxOperatorRows && (n == 0 || (tokens && is_aligned(tokens, size)));
}

// The most elements (8, 4, 2 or 1) that can be moved at once at every multiple of as many columns of every row.
inline int vector_of(const mono_matrix_t& m) {
  const int size = element_size(m.type);
  for (int v = 8; v > 1; v /= 2) {
    const size_t bytes = std::min(16, v * size);
    if (m.cols % v == 0 && is_aligned(m.data, bytes) && (m.rows <= 1 || m.stride * size % (int64_t)bytes == 0)) return v;
  }
  return 1;
}

// Calls f with a value of the element type / of the vector's width.
template <typename F>
int with_type(int32_t type, F&& f) {
  return type == MONO_F32 ? f(float()) : type == MONO_BF16 ? f(__nv_bfloat16()) : f(__half());
}
template <int N> struct Width { static constexpr int value = N; };
template <typename F>
int with_width(int v, F&& f) {
  return v == 8 ? f(Width<8>()) : v == 4 ? f(Width<4>()) : v == 2 ? f(Width<2>()) : f(Width<1>());
}

// Launch of a kernel that waits for the stream's previous kernel itself (after_previous_kernel), so that its
// launch is prepared while that one runs.
template <typename... P, typename... A>
inline int launch_operator(void (*kernel)(P...), dim3 grid, unsigned block, size_t shared, cudaStream_t s, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block, 1, 1);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...) == cudaSuccess) return MONO_OK;
  cudaGetLastError();                                       // (reported here, not by the next call that asks)
  return MONO_ERR_CUDA;
}

}  // namespace mono

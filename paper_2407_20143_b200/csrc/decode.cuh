// What the decoding operators share (rope.cu, kv_cache.cu, kv_attend.cu): element types, the division
// by a run-time constant, loads and stores of 16 elements of a head vector, argument checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bcp.h"
#include "plan.hpp"
#include "plan_object.hpp"

namespace bcp {

// n / d for n < 2^31 as a multiplication and a shift (the method of Granlund and Montgomery): with
// p = 31 + ceil(log2 d) and m = ceil(2^p / d) < 2^32 the quotient is (n * m) >> p.
struct FastDiv {
  uint32_t d = 1, mul = 0, shift = 0;
  FastDiv() = default;
  explicit FastDiv(uint32_t divisor) : d(divisor) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < divisor) ++l;
    if (l == 0) return;  // d == 1: div() returns n
    const uint32_t p = 31 + l;
    mul = uint32_t(((uint64_t(1) << p) + divisor - 1) / divisor);
    shift = p - 32;
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const {
#ifdef __CUDA_ARCH__
    return mul ? __umulhi(n, mul) >> shift : n;
#else
    return mul ? uint32_t((uint64_t(n) * mul) >> 32) >> shift : n;
#endif
  }
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Eight consecutive elements as they lie in memory: 16 bytes of a 16-bit type, 32 bytes of binary32.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) w[i] = *(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) *(reinterpret_cast<uint4*>(p) + i) = w[i];
  }
  __device__ __forceinline__ T get(int i) const { return reinterpret_cast<const T*>(w)[i]; }
  __device__ __forceinline__ void set(int i, T x) { reinterpret_cast<T*>(w)[i] = x; }
};

// The sixteen elements of a head vector that one thread handles ("chunk" c): with a rotation, eight
// pairs while c < ceil(rot/16), then sixteen unrotated elements; without one, sixteen in a row.
// first(i) / second(i) are the places of the i-th element of either half; n is how many exist.
struct Chunk {
  uint32_t a, b, step, n_a, n_b;  // first(i) = a + i*step, second(i) = b + i*step
  uint32_t pair;                  // index of the first pair (rotated chunks)
  bool rotated;
};

__host__ __device__ __forceinline__ uint32_t chunks_of(uint32_t head_dim, uint32_t rot_dim) { return (rot_dim / 2 + 7) / 8 + (head_dim - rot_dim + 15) / 16; }

__device__ __forceinline__ Chunk chunk_at(uint32_t c, uint32_t head_dim, uint32_t rot_dim, uint32_t layout) {
  Chunk k;
  const uint32_t pairs = rot_dim / 2, n_rot = (pairs + 7) / 8;
  k.rotated = c < n_rot;
  if (k.rotated) {
    k.pair = 8 * c;
    const uint32_t n = pairs - k.pair < 8 ? pairs - k.pair : 8;
    k.n_a = k.n_b = n;
    if (layout == BCP_ROPE_HALF) {
      k.a = k.pair, k.b = pairs + k.pair, k.step = 1;
    } else {
      k.a = 2 * k.pair, k.b = 2 * k.pair + 1, k.step = 2;
    }
  } else {
    k.pair = 0;
    k.a = rot_dim + 16 * (c - n_rot), k.b = k.a + 8, k.step = 1;
    const uint32_t left = head_dim > k.a ? head_dim - k.a : 0;
    k.n_a = left < 8 ? left : 8;
    k.n_b = left <= 8 ? 0 : (left < 16 ? left - 8 : 8);
  }
  return k;
}

// Sixteen elements of a chunk.  VEC: whole 16-byte vectors (rot_dim and head_dim multiples of 16,
// rows on 16-byte boundaries); neighbouring pairs then lie in two consecutive vectors.
template <typename T, bool VEC>
struct Elements {
  Raw8<T> lo, hi;
  __device__ __forceinline__ void load(const T* row, const Chunk& k) {
    if (VEC) {
      lo.load(row + k.a);
      hi.load(row + (k.step == 2 ? k.a + 8 : k.b));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        lo.set(i, uint32_t(i) < k.n_a ? row[k.a + i * k.step] : from_f32<T>(0.f));
        hi.set(i, uint32_t(i) < k.n_b ? row[k.b + i * k.step] : from_f32<T>(0.f));
      }
    }
  }
  // x[i] is the first, y[i] the second element of pair i (or the two halves of an unrotated chunk)
  __device__ __forceinline__ void unpack(float (&x)[8], float (&y)[8], const Chunk& k) const {
    if (VEC && k.step == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = to_f32(lo.get(2 * i)), y[i] = to_f32(lo.get(2 * i + 1));
        x[i + 4] = to_f32(hi.get(2 * i)), y[i + 4] = to_f32(hi.get(2 * i + 1));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_f32(lo.get(i)), y[i] = to_f32(hi.get(i));
    }
  }
  __device__ __forceinline__ void pack(const float (&x)[8], const float (&y)[8], const Chunk& k) {
    if (VEC && k.step == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo.set(2 * i, from_f32<T>(x[i])), lo.set(2 * i + 1, from_f32<T>(y[i]));
        hi.set(2 * i, from_f32<T>(x[i + 4])), hi.set(2 * i + 1, from_f32<T>(y[i + 4]));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) lo.set(i, from_f32<T>(x[i])), hi.set(i, from_f32<T>(y[i]));
    }
  }
  __device__ __forceinline__ void store(T* row, const Chunk& k) const {
    if (VEC) {
      lo.store(row + k.a);
      hi.store(row + (k.step == 2 ? k.a + 8 : k.b));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (uint32_t(i) < k.n_a) row[k.a + i * k.step] = lo.get(i);
        if (uint32_t(i) < k.n_b) row[k.b + i * k.step] = hi.get(i);
      }
    }
  }
};

// Cosines and sines of a chunk's eight pairs.
template <bool VEC>
struct Angles {
  float c[8], s[8];
  __device__ __forceinline__ void load(const float* table, int64_t position, uint32_t rot_dim, const Chunk& k) {
    const uint32_t pairs = rot_dim / 2;
    const float* row = table + position * rot_dim;
    if (VEC) {
      const float4* pc = reinterpret_cast<const float4*>(row + k.pair);
      const float4* ps = reinterpret_cast<const float4*>(row + pairs + k.pair);
      const float4 c0 = __ldg(pc), c1 = __ldg(pc + 1), s0 = __ldg(ps), s1 = __ldg(ps + 1);
      c[0] = c0.x, c[1] = c0.y, c[2] = c0.z, c[3] = c0.w, c[4] = c1.x, c[5] = c1.y, c[6] = c1.z, c[7] = c1.w;
      s[0] = s0.x, s[1] = s0.y, s[2] = s0.z, s[3] = s0.w, s[4] = s1.x, s[5] = s1.y, s[6] = s1.z, s[7] = s1.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = uint32_t(i) < k.n_a;
        c[i] = in ? __ldg(row + k.pair + i) : 1.f;
        s[i] = in ? __ldg(row + pairs + k.pair + i) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void rotate(float (&x)[8], float (&y)[8], float sign) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = sign * s[i], u = x[i];
      x[i] = u * c[i] - y[i] * t;
      y[i] = y[i] * c[i] + u * t;
    }
  }
};

__device__ __forceinline__ void raise(uint32_t* status, uint32_t bit) {
  if (status) atomicOr(status, bit);
}

// ------------------------------------------------------------------------------ host checks
inline uint32_t type_size(uint32_t t) { return t == BCP_F32 ? 4 : t == BCP_BF16 || t == BCP_F16 ? 2 : t == BCP_E4M3 || t == BCP_I8 ? 1 : 0; }
inline bool is_8bit(uint32_t t) { return t == BCP_E4M3 || t == BCP_I8; }

// Whether rows of `row` elements, laid out with n strides and extents, can share memory: by growing
// stride, each has to step over all that the smaller ones span.  (Also true for strides past any memory.)
bool rows_overlap(const int64_t* strides, const uint32_t* extents, int n, uint32_t row);
int check_heads(const char* call, const char* name, const bcp_heads* h, bool written, uint32_t head_dim, int64_t n_tokens);
int check_rope(const char* call, const bcp_rope_table* r, uint32_t head_dim);
int check_cache(const char* call, const bcp_kv_cache* c);
// Whether every row of h starts on a boundary of `bytes` bytes.
inline bool rows_aligned(const bcp_heads* h, uint32_t bytes) {
  const uint64_t es = type_size(h->type);
  return ((reinterpret_cast<uintptr_t>(h->data) | uint64_t(h->token_stride) * es | uint64_t(h->head_stride) * es) & (bytes - 1)) == 0;
}

#define BCP_LAUNCHED(call)                                                                     \
  do {                                                                                         \
    cudaError_t e_ = cudaGetLastError();                                                       \
    if (e_ != cudaSuccess) return bcp::fail(BCP_ERR_CUDA, "%s: %s", call, cudaGetErrorString(e_)); \
  } while (0)

}  // namespace bcp

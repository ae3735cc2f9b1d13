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

// N elements as they lie in memory, moved in the widest accesses of at most 16 bytes.
template <typename T, int N>
struct Raw {
  static constexpr int kBytes = N * int(sizeof(T));
  static_assert(kBytes == 4 || kBytes == 8 || kBytes % 16 == 0, "whole accesses");
  uint32_t w[kBytes / 4];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
    if constexpr (kBytes == 8) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x, w[1] = v.y;
    }
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i) {
      const uint4 v = *(reinterpret_cast<const uint4*>(p) + i);
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
#pragma unroll
    for (int i = 0; i < kBytes / 16; ++i) *(reinterpret_cast<uint4*>(p) + i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
  __device__ __forceinline__ T get(int i) const { return reinterpret_cast<const T*>(w)[i]; }
  __device__ __forceinline__ void set(int i, T x) { reinterpret_cast<T*>(w)[i] = x; }
};

// What one thread takes of a head vector, its "chunk": V pairs, or 2 V elements that are not rotated.
// In vector form (VEC) V elements make 16 bytes, and a chunk is one vector of either half of a region, the
// rotated dimensions or the rest, so that neighbouring threads touch neighbouring vectors whatever the
// layout of the pairs: with the half layout the two vectors hold the first and second elements of V pairs,
// else (PAIRS) each holds V/2 whole pairs.  It needs regions that are multiples of 2 V = 16 elements (8 of
// binary32, held to 16 all the same) and rows on 16-byte boundaries.  The scalar form (V = 8) takes any
// sizes: elements lo + i step and hi + i step, i < n_lo and n_hi.
template <typename T, bool VEC>
constexpr int kChunk = VEC ? 16 / int(sizeof(T)) : 8;

struct Chunk {
  uint32_t lo, hi, step, n_lo, n_hi;
  uint32_t pair, pair2;  // first pair of the chunk; in vector form with whole pairs, first pair of the second vector
  bool rotated;
};

__host__ __device__ __forceinline__ uint32_t chunks_of(uint32_t head_dim, uint32_t rot_dim, uint32_t v) {
  return (rot_dim / 2 + v - 1) / v + (head_dim - rot_dim + 2 * v - 1) / (2 * v);
}

template <int V, bool VEC, bool PAIRS>
__device__ __forceinline__ Chunk chunk_at(uint32_t c, uint32_t head_dim, uint32_t rot_dim) {
  Chunk k;
  const uint32_t pairs = rot_dim / 2, n_rot = (pairs + V - 1) / V;
  k.rotated = c < n_rot;
  k.pair = k.pair2 = 0;
  k.step = 1;
  if (VEC) {
    const uint32_t begin = k.rotated ? 0 : rot_dim, size = k.rotated ? rot_dim : head_dim - rot_dim;
    k.lo = begin + V * (k.rotated ? c : c - n_rot), k.hi = k.lo + size / 2;
    k.n_lo = k.n_hi = V;
    if (k.rotated) k.pair = PAIRS ? k.lo / 2 : k.lo, k.pair2 = k.hi / 2;
  } else if (k.rotated) {
    k.pair = V * c;
    k.n_lo = k.n_hi = pairs - k.pair < V ? pairs - k.pair : V;
    k.lo = PAIRS ? 2 * k.pair : k.pair, k.hi = PAIRS ? k.lo + 1 : k.lo + pairs, k.step = PAIRS ? 2 : 1;
  } else {
    k.lo = rot_dim + 2 * V * (c - n_rot), k.hi = k.lo + V;
    const uint32_t left = head_dim > k.lo ? head_dim - k.lo : 0;
    k.n_lo = left < V ? left : V;
    k.n_hi = left <= V ? 0 : (left < 2 * V ? left - V : V);
  }
  return k;
}

template <typename T, bool VEC>
struct Elements {
  static constexpr int V = kChunk<T, VEC>;
  Raw<T, V> lo, hi;
  __device__ __forceinline__ void load(const T* row, const Chunk& k) {
    if (VEC) {
      lo.load(row + k.lo);
      hi.load(row + k.hi);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        lo.set(i, uint32_t(i) < k.n_lo ? row[k.lo + i * k.step] : from_f32<T>(0.f));
        hi.set(i, uint32_t(i) < k.n_hi ? row[k.hi + i * k.step] : from_f32<T>(0.f));
      }
    }
  }
  __device__ __forceinline__ void unpack(float (&x)[V], float (&y)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = to_f32(lo.get(i)), y[i] = to_f32(hi.get(i));
  }
  __device__ __forceinline__ void pack(const float (&x)[V], const float (&y)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) lo.set(i, from_f32<T>(x[i])), hi.set(i, from_f32<T>(y[i]));
  }
  __device__ __forceinline__ void store(T* row, const Chunk& k) const {
    if (VEC) {
      lo.store(row + k.lo);
      hi.store(row + k.hi);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (uint32_t(i) < k.n_lo) row[k.lo + i * k.step] = lo.get(i);
        if (uint32_t(i) < k.n_hi) row[k.hi + i * k.step] = hi.get(i);
      }
    }
  }
};

// Two binary32 operations at once (sm_100 has the packed forms).
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmul.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 z, {%6, %7};\nfma.rn.f32x2 z, x, y, z;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}

// The positions of a token: one, or (AXES) one for each axis.
struct AxisMap {
  uint32_t w[BCP_MAX_HEAD_DIM / 2 / 16] = {};  // two bits for each pair: its axis
  uint32_t n_axes = 1;
  int64_t stride = 0;  // positions of axis a begin at a * stride
};
template <bool AXES>
struct At {
  int64_t p[AXES ? BCP_MAX_AXES : 1];
  bool inside, padding;  // all positions are rows of the table; one is negative
  __device__ __forceinline__ void load(const int64_t* positions, uint32_t t, int64_t n_positions, const AxisMap& m) {
    p[0] = positions[t];
    if constexpr (AXES) {
#pragma unroll
      for (uint32_t a = 1; a < BCP_MAX_AXES; ++a) p[a] = a < m.n_axes ? positions[a * m.stride + t] : p[0];
    }
    inside = true, padding = false;
#pragma unroll
    for (int a = 0; a < int(sizeof p / sizeof p[0]); ++a) {
      padding |= p[a] < 0;
      inside &= p[a] >= 0 && p[a] < n_positions;
    }
    if (!inside) {
#pragma unroll
      for (int a = 0; a < int(sizeof p / sizeof p[0]); ++a) p[a] = 0;
    }
  }
  __device__ __forceinline__ int64_t of(uint32_t axis) const {
    if constexpr (AXES) return axis < 2 ? (axis ? p[1] : p[0]) : (axis == 2 ? p[2] : p[3]);
    return p[0];
  }
};

// Cosines and sines of a chunk's V pairs.
template <int V, bool VEC, bool PAIRS>
struct Angles {
  float c[V], s[V];
  __device__ __forceinline__ void load(const float* table, const At<false>& at, uint32_t rot_dim, const Chunk& k, float sign, const AxisMap&) {
    load(table, at.p[0], rot_dim, k, sign);
  }
  // Each pair from the row of its axis.  V / 2 neighbouring pairs of one axis, as in parts of a multiple of that, are loaded as
  // vectors; where axes take turns, element by element.
  __device__ __forceinline__ void load(const float* table, const At<true>& at, uint32_t rot_dim, const Chunk& k, float sign, const AxisMap& m) {
    const uint32_t pairs = rot_dim / 2;
    if (VEC) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        constexpr uint32_t kAll = (1u << V) - 1, kOnes = 0x55555555u & kAll;  // two bits for each of V / 2 pairs
        const uint32_t from = half ? (PAIRS ? k.pair2 : k.pair + V / 2) : k.pair, axes = m.w[from / 16] >> (2 * (from % 16)) & kAll;
        if (axes == (axes & 3) * kOnes) {
          const float* const row = table + at.of(axes & 3) * rot_dim;
          part(row, row + pairs, from, half * (V / 2));
        } else {
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            const float* const e = table + at.of(axes >> (2 * i) & 3) * rot_dim + from + i;
            c[half * (V / 2) + i] = e[0], s[half * (V / 2) + i] = e[pairs];
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool in = uint32_t(i) < k.n_lo;
        const uint32_t pair = in ? k.pair + i : 0;
        const float* const e = table + at.of(m.w[pair / 16] >> (2 * (pair % 16)) & 3) * rot_dim + pair;
        c[i] = in ? e[0] : 1.f;
        s[i] = in ? e[pairs] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] *= sign;
  }
  __device__ __forceinline__ void load(const float* table, int64_t position, uint32_t rot_dim, const Chunk& k, float sign) {
    const uint32_t pairs = rot_dim / 2;
    const float* const row = table + position * rot_dim;
    if (VEC) {
      // with whole pairs the second vector's pairs are elsewhere
      const uint32_t second = PAIRS ? k.pair2 : k.pair + V / 2;
      part(row, row + pairs, k.pair, 0);
      part(row, row + pairs, second, V / 2);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool in = uint32_t(i) < k.n_lo;
        c[i] = in ? row[k.pair + i] : 1.f;
        s[i] = in ? row[pairs + k.pair + i] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] *= sign;
  }
  __device__ __forceinline__ void part(const float* pc, const float* ps, uint32_t from, int to) {
    if constexpr (V == 8) {
      const float4 a = *reinterpret_cast<const float4*>(pc + from), b = *reinterpret_cast<const float4*>(ps + from);
      c[to] = a.x, c[to + 1] = a.y, c[to + 2] = a.z, c[to + 3] = a.w;
      s[to] = b.x, s[to + 1] = b.y, s[to + 2] = b.z, s[to + 3] = b.w;
    } else {
      const float2 a = *reinterpret_cast<const float2*>(pc + from), b = *reinterpret_cast<const float2*>(ps + from);
      c[to] = a.x, c[to + 1] = a.y;
      s[to] = b.x, s[to + 1] = b.y;
    }
  }
  // (u, v) = (u c - v s, v c + u s) for the pairs of the chunk, whose vectors are x and y
  __device__ __forceinline__ void rotate(float (&x)[V], float (&y)[V]) const {
    if constexpr (VEC && PAIRS) {
      neighbours(x, 0);
      neighbours(y, V / 2);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        const float2 a = make_float2(x[i], x[i + 1]), b = make_float2(y[i], y[i + 1]), cc = make_float2(c[i], c[i + 1]), ss = make_float2(s[i], s[i + 1]);
        const float2 p = fma2(a, cc, mul2(b, make_float2(-ss.x, -ss.y))), q = fma2(b, cc, mul2(a, ss));
        x[i] = p.x, x[i + 1] = p.y, y[i] = q.x, y[i + 1] = q.y;
      }
    }
  }
  __device__ __forceinline__ void neighbours(float (&x)[V], int at) const {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float cc = c[at + i / 2], ss = s[at + i / 2];
      const float2 p = fma2(make_float2(x[i], x[i + 1]), make_float2(cc, cc), mul2(make_float2(x[i + 1], x[i]), make_float2(-ss, ss)));
      x[i] = p.x, x[i + 1] = p.y;
    }
  }
};

// Kernels of a decoding step are a few microseconds long, of which the gap between two launches is a good part.
// They are launched so that their blocks may take their places while the kernel before them on the
// stream ends (launch_early), and begin with after_previous(): the next kernel may do the same, and
// nothing is read or written before the one before has completed and its memory is visible.  (No load takes the
// read-only path: what one kernel reads may be written while its blocks already wait.)
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void after_previous() {
  next_may_start();
  wait_for_previous();
}
template <typename Args>
cudaError_t launch_early(void (*kernel)(Args), uint32_t blocks, uint32_t threads, uint32_t shared_bytes, cudaStream_t stream, const Args& args) {
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(blocks), config.blockDim = dim3(threads), config.dynamicSmemBytes = shared_bytes, config.stream = stream;
  config.attrs = &early, config.numAttrs = 1;
  return cudaLaunchKernelEx(&config, kernel, args);
}

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
int check_axes(const char* call, const bcp_rope_axes_map* axes, const bcp_rope_table* r, AxisMap* out);
int check_cache(const char* call, const bcp_kv_cache* c);
// Whether every row of h starts on a boundary of `bytes` bytes.
inline bool rows_aligned(const bcp_heads* h, uint32_t bytes) {
  const uint64_t es = type_size(h->type);
  return ((reinterpret_cast<uintptr_t>(h->data) | uint64_t(h->token_stride) * es | uint64_t(h->head_stride) * es) & (bytes - 1)) == 0;
}

}  // namespace bcp

// What the attention kernels share (kv_attend.cu, kv_prefix.cu): the cut of a line of steps into parts, asynchronous copies, fast
// exponentials, conversions of 8-bit elements and of weights.
#pragma once

#include "decode.cuh"

namespace bcp {

constexpr float kNone = -3.0e38f;  // reference before the first token: below every score
constexpr float kLog2e = 1.4426950408889634f;

// The line of n steps is dealt out to the parts as evenly as whole steps allow.  (Fewer than 2^31 steps: the host
// refuses more.)
struct Cuts {
  uint32_t n, each, longer;  // steps of the line, of a part; the first `longer` parts have one more
  uint32_t parts;
  __device__ __forceinline__ void cut(uint32_t steps, uint32_t ctas) {
    // A line of a few steps per CTA is cut into parts of whole, equal numbers of them: the longest part decides, and
    // fewer parts are joined sooner (one sequence of 3000 tokens 13.5 us, 14.5 without; of 4000 14.6 and 15.2; of 5000 14.0 and
    // 15.2).
    n = steps, parts = n < ctas ? n : ctas;
    if (n > ctas && n < 4 * ctas) {
      const uint32_t most = (n + ctas - 1) / ctas;
      parts = (n + most - 1) / most;
    }
    each = n / parts, longer = n - each * parts;
  }
  __device__ __forceinline__ uint32_t begin(uint32_t p) const { return each * p + (p < longer ? p : longer); }
  __device__ __forceinline__ uint32_t part_of(uint32_t x) const {  // the part that step x lies in
    const uint32_t lower = longer * (each + 1);
    return x < lower ? x / (each + 1) : longer + (x - lower) / each;
  }
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool on) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from, bool on) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(on ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_fast(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^x, x <= 0, for sums whose reference moves by x.  With scales in the exponents (WIDE) a reference can lie up to 2^247 above what
// still counts in a denominator: that is multiplied in two steps, neither of which underflows.
template <bool WIDE>
struct Factor {
  float root, all;
  __device__ __forceinline__ explicit Factor(float x) : root(exp2_fast(WIDE ? 0.5f * x : x)), all(WIDE ? root * root : root) {}
  __device__ __forceinline__ float denominator(float l) const { return WIDE ? l * root * root : l * root; }
};
// Four 8-bit elements as two pairs of binary16, exactly.
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (FMT == BCP_E4M3) {
    asm("{\n.reg .b16 x, y;\nmov.b32 {x, y}, %2;\ncvt.rn.f16x2.e4m3x2 %0, x;\ncvt.rn.f16x2.e4m3x2 %1, y;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
  } else {
    // bytes u = x + 128 under the exponent of 1024 read as 1024 + u; 1152 off gives x
    const uint32_t u = w ^ 0x80808080u, a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 bias = __half2half2(__ushort_as_half(0x6480));
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), bias), y = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
    lo = *reinterpret_cast<const uint32_t*>(&x), hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float x, float y) {
  if constexpr (BF16) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&p);
  } else {
    const __half2 p = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
}
// A positive binary32 number as the sum of a bfloat16 that is its upper half and what remains, positive as well (its last bit is
// set): the products of both with an infinite value are that infinity.
__device__ __forceinline__ uint32_t upper_halves(float x, float y) { return __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632); }
__device__ __forceinline__ float lower_half(float x) {
  return __uint_as_float(__float_as_uint(x) | 1u) - __uint_as_float(__float_as_uint(x) & 0xffff0000u);
}
__device__ __forceinline__ float query_at(const void* p, int i, bool bf16) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : __half2float(static_cast<const __half*>(p)[i]);
}

// Where the attention over own tokens leaves its sums when a shared prefix is still to be joined: for every row (sequence, query head) a
// reference and a denominator, ml = (m, l), l = sum exp2(s - m), and `dims` sums o = sum exp2(s - m) v.
struct Records {
  float2* ml;
  float* o;
  uint32_t dims;
};

// The attention over own tokens (csrc/kv_attend.cu); with `records` into those, out and lse are not written.
int attend(const char* call, const bcp_kv_cache* c, const bcp_heads* q, const bcp_heads* out, float* lse, uint32_t n_seqs, const int32_t* block_table,
           int64_t table_stride, uint32_t table_width, const int32_t* lengths, float scale, uint32_t window, void* workspace, uint64_t workspace_bytes,
           const Records* records, bool launch, void* stream);  // launch false: the arguments are only looked at
int check_group(const char* call, const bcp_kv_cache* c, uint32_t n_q_heads);

}  // namespace bcp

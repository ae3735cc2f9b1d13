// Attention of one new token per sequence over the paged key-value cache.
//
// Mathematics.  For one query head the pass over the tokens keeps a reference r, l = sum exp2(s - r) and
// o = sum exp2(s - r) v, with s = q.k scale log2 e; whenever a score exceeds r by more than 8 the sums are
// multiplied by exp2(r - r') and r' takes its place.  Any r gives the same o / l; parts of a sequence are
// joined by bringing their sums to the largest r.  Each key and value is read once for up to 16 query heads that
// share its cache head (8 with more than 128 dimensions); larger groups are cut into row tiles, which each read it again.
//
// What bounds it: reading the cache.  A byte of 16-bit cache is used in `group` multiply-adds (at most a
// few dozen), so the matrix instructions only have to keep out of the way.  The products are taken as
// S^T = K Q^T and O^T = V^T P^T with mma.m16n8k16: tokens (or head dimensions) fill the 16 rows and eight
// query heads the 8 columns, so that a group of up to eight heads costs one instruction per 16 x 16 block
// of the cache.  (A tcgen05 product has at least 64 rows: over eight heads it would be filled for an
// eighth, and its operands would have to be laid out in shared memory first, 8-bit ones converted.)
//
// A warp is a worker of its own: it takes 16 tokens at a time through a ring of shared-memory stages that
// it fills itself with 16-byte asynchronous copies, a stage or two ahead and across the borders of
// sequences, so no barrier of the CTA stands in the stream.  The four warps of a CTA take the four quarters
// of each 64-token step and add up at the end of a stretch of one sequence and cache head.
//
// Split.  All steps of all sequences and heads form one line that is cut into as many equal parts as CTAs
// fit on the GPU; lengths are only known on the device, so each CTA finds its part itself.  Two more steps
// per unit (sequence, cache head, row tile) stand for what its beginning and end cost (kExtra).  A unit that lies in one
// part is finished there; else every part leaves its sums in the workspace.  Of each 64 parts of a unit the
// one that comes last (a counter says which) joins them, and of these groups the last again, always in
// the order of the parts, so results do not depend on which that is.
//
// Measured on one B200 (copy bandwidth 6533 GB/s), per launch in a row of them: one sequence of 131,072 tokens, 32 / 8 heads
// of 128, bfloat16: 92 us = 5.8 TB/s; 64 ragged sequences of up to 4096, bfloat16: 107.6 us = 6.1 TB/s, e4m3: 71.5 us =
// 4.7 TB/s; 37 windows of 1000, 16 / 16 heads, int8: 42 us = 3.4 TB/s; one sequence of 600 tokens: 7.8 us, of which the launch, the
// look-up of the lengths and the page, the first read and the joining of ten parts are most.  With the end-of-stretch work left out
// (measured on an earlier form of the kernel) the first takes 85, the e4m3 batch 57 and the windows 33 us: it is what keeps
// them from the copy bandwidth (DRAM 40 to 67 % busy, tensor pipe 10 to 14 %).  Not near it: 8000 sequences of up to 64 tokens,
// one cache head, bfloat16: 127 us for 0.18 GB, as every CTA goes over all lengths; one cache head under 16 / 32 / 64 query
// heads, 64 ragged sequences: 27 / 38 / 62 us for 84 MB (row tiles); 2 under 16 each with 256 dimensions 113 us for 0.34 GB, 62 under 8.
#include <mutex>

#include "decode.cuh"

using namespace bcp;

namespace {

constexpr int kWarps = 4, kTok = 16, kStep = kWarps * kTok;  // tokens per warp and per step of a CTA
constexpr float kNone = -3.0e38f;                             // reference before the first token: below every score
constexpr float kLog2e = 1.4426950408889634f;

struct AttendArgs {
  const void *k, *v;
  const float *k_scale, *v_scale;
  uint32_t page_stride, head_stride, token_stride;
  uint32_t n_pages, n_heads, head_dim;
  FastDiv page_size;
  uint32_t* status;
  const void* q;
  void* out;
  float* lse;
  int64_t q_token, q_head, out_token, out_head;
  uint32_t q_is_bf16, group, row_tiles, n_seqs;
  const int32_t* block_table;
  int64_t table_stride;
  uint32_t capacity;  // tokens a row of the block table can hold
  const int32_t* lengths;
  float scale_log2;
  uint32_t window;
  uint32_t* part_count;   // two per part: parts that have arrived, at the place of a unit's first part in a group
  uint32_t* group_count;  // two per part: groups that have arrived, at the place of the unit's first part
  float* parts;          // two places per part: sums, then references, then denominators
};

// Steps that a unit counts for besides its own.  Microseconds with 0 / 1 / 2 / 3: 64 ragged sequences of up to 4k tokens,
// e4m3 82 / 77 / 71.6 / 69; 37 windows of 1000, int8, 16 heads 65 / 42.9 / 42.3 / 43.6; 300 sequences of up to 500, e4m3 71 / 64.6 / 63 / 63,
// bfloat16 84.7 / 83.5 / 82.2 / 82.7; one sequence of 5000, bfloat16 15.2 / 14.6 / 14 / 14.2.
constexpr uint32_t kExtra = 2;

constexpr uint32_t kGroup = 64;  // parts that are joined at once
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

template <int FMT, int DP, int NT>
struct Shape {
  static constexpr bool quant = FMT == BCP_E4M3 || FMT == BCP_I8;
  static constexpr int ES = quant ? 1 : 2;
  static constexpr int ROW = DP * ES;        // bytes of a row in shared memory
  static constexpr int CPR = ROW / 16;       // 16-byte chunks of a row
  static constexpr int SIDE = kTok * ROW;
  static constexpr int STAGE = 2 * SIDE + (quant ? 128 : 0) + 16;  // keys, values, their scales, the mask of live tokens
  // Bytes in flight, in all but one stage of each warp: 32 to 64 KiB an SM cover the latency of HBM.  More only
  // queue up, and unevenly, or cost CTAs: microseconds with two and with three stages for 64 ragged sequences of up to 4096 tokens, 8 heads,
  // 8-bit 64 dimensions 48.0 / 48.5, 128 70.9 / 83.7, 256 (4 heads) 68.9 / 102; 16-bit 64 58.8 / 61.4, 128 107 / 113.
  static constexpr int STAGES = 2;
  // CTAs that share an SM and bound the registers of a thread (128, 168 or 255 for four, three and two).  8-bit caches, whose
  // elements cost conversions, gain from warps as long as little is spilled.  Microseconds for 64 ragged sequences of up to 4096
  // tokens: 64 dimensions, up to 8 heads a group, 8 / 16 bits: 48.5 / 58.9 with four, 54.9 / 60.7 with three, 49.4 / 60.7 with five; 16
  // heads 43.4 / 40.6 with three, 46.6 / 47.4 with two, 39.7 / 40.6 with four (but 8 sequences of 2000 17.7 against 15.5);
  // 128 dimensions, 8 bits, up to 8 heads 70.8 with four, 72.7 with three (windows 43 and 50; but one sequence of 60,000 42.3
  // and 36.7); 16 heads 65.4 with two, 73.2 with three; 16 bits, 16 heads 65.0 with two, 72.6 with three.  Of the others
  // shared memory allows two (16 bits, 256 dimensions: one).
  static constexpr int CTAS = DP == 64 ? (NT == 1 ? 4 : 3) : DP == 128 && quant && NT == 1 ? 4 : 2;
  static constexpr int ROWS = 8 * NT;
  static constexpr int PART = ROWS * (DP + 2);  // floats of one set of sums: dimensions of the heads (sum_at), references, denominators
  static constexpr int SMEM = kWarps * STAGES * STAGE + kWarps * PART * 4 + 16;
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
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void load_transposed(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
// d += a b, a 16 x 16 (row fragments), b 16 x 8; both operands bfloat16 or both binary16
template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

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

// Where dimension d of head (column) n lies in a set of sums: eight rows of dimensions and four pairs of heads
// are written at a time by a warp, the exclusive-or spreads them over the banks.
template <int DP, bool QUANT>
__device__ __forceinline__ uint32_t sum_at(uint32_t n, uint32_t d) {
  return n * DP + (d ^ (n >> 1 & 3) << (QUANT ? 2 : 3));
}
// Sums lie in shared memory or in the workspace, where other CTAs wrote them: generic loads that no cache keeps.
__device__ __forceinline__ float4 load_sums4(const float* p) {
  float4 v;
  asm volatile("ld.volatile.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float load_sums(const float* p) { return *static_cast<const volatile float*>(p); }

// Where 16-byte chunk c of row r lies in a side of a stage.  Keys are read as 16-byte vectors by 8 lanes
// that hold two rows and four neighbouring chunks, values by 8 lanes with eight rows of one chunk
// (16-bit, transposing loads) or the four rows 0, 2, 4, 6 (1, 3, 5, 7) and two neighbouring chunks: the
// exclusive-or spreads each of these over the 32 banks.
template <int CPR>
__device__ __forceinline__ uint32_t key_at(uint32_t r, uint32_t c) {
  if (CPR >= 8) c ^= (r & 1) << 2;
  return (r * CPR + c) * 16;
}
template <int CPR, bool QUANT>
__device__ __forceinline__ uint32_t value_at(uint32_t r, uint32_t c) {
  const uint32_t linear = r * CPR + c;
  if (!QUANT) return (linear ^ (r & 7)) * 16;
  return (linear ^ ((CPR >= 8 ? r >> 1 : linear >> 3) & 3) << 1) * 16;
}

struct Span {  // the tokens of one sequence, and its steps
  uint32_t first, len, base, steps;  // base: first token of step 0, a multiple of 16 (less a step, modulo 2^32, if that has none)
};
// extra: steps without tokens that every unit begins with
__device__ __forceinline__ Span span_of(const AttendArgs& a, uint32_t b, uint32_t extra) {
  Span s;
  int32_t n = a.lengths[b];
  n = n < 0 ? 0 : n;
  s.len = uint32_t(n) > a.capacity ? a.capacity : uint32_t(n);
  s.first = a.window && s.len > a.window ? s.len - a.window : 0;
  s.base = s.first & ~15u;
  s.steps = (s.len - s.base + kStep - 1) / kStep;
  if (!s.steps) s.steps = 1;  // a sequence without tokens still has a result to write
  s.steps += extra, s.base -= extra * kStep;
  return s;
}

// A place on the line of steps: sequence b, unit u (cache head and row tile) of it, step of the unit.
struct Place {
  uint32_t b, u, step;
  Span span;
};
__device__ __forceinline__ void advance(Place& p, const AttendArgs& a, uint32_t units, uint32_t extra, bool more) {
  if (++p.step < p.span.steps) return;
  p.step = 0;
  if (++p.u < units) return;
  p.u = 0;
  if (++p.b < a.n_seqs && more) p.span = span_of(a, p.b, extra);
}

template <int FMT, int DP, int NT>
__global__ void __launch_bounds__(kWarps * 32, Shape<FMT, DP, NT>::CTAS) bcp_kv_attend_kernel(const AttendArgs a) {
  typedef Shape<FMT, DP, NT> S;
  constexpr bool kBf16 = FMT == BCP_BF16;  // type of the products; 8-bit caches are widened to binary16
  // binary16 weights underflow below 2^-24: lifting them by 2^6 (they stay below 2^16) moves that to 2^-30
  constexpr float kLift = kBf16 ? 0.f : 6.f;
  // Over a bfloat16 cache a weight goes into the product as two bfloat16 numbers: one alone is rounded to 2^-8, as coarsely as the
  // result (131,072 tokens: relative error 2.2e-3, 1.6e-3 with two, which is the rounding of the result; 96.0 and 96.6 us).  The
  // weights over other caches are binary16, 2^-11: 8-bit caches would pay 4 to 5 % for the second product (windows 43.4 and 45.5 us,
  // 2.4e-4 and 2.1e-4 with results in binary16), and are rounded to 2^-4 or 2^-8 of a vector's largest themselves.
  constexpr bool kRest = kBf16;
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
  const uint32_t ring = uint32_t(__cvta_generic_to_shared(smem)) + warp * (S::STAGES * S::STAGE);
  unsigned char* const ring_ptr = smem + warp * (S::STAGES * S::STAGE);
  float* const sums = reinterpret_cast<float*>(smem + kWarps * S::STAGES * S::STAGE);  // a part's worth for each warp
  uint32_t* const shared_word = reinterpret_cast<uint32_t*>(sums + kWarps * S::PART);

  after_previous();
  // ---- the line, and this CTA's part of it
  const uint32_t units = a.n_heads * a.row_tiles;
  // every thread counts the steps of a run of sequences; an exclusive scan over the threads
  const uint32_t run = (a.n_seqs + kWarps * 32 - 1) / (kWarps * 32);
  const uint32_t run0 = min(tid * run, a.n_seqs), run1 = min(run0 + run, a.n_seqs);
  uint32_t mine = 0, before;
  Cuts cuts;
  uint32_t extra;
  {
#pragma unroll 1
    for (uint32_t b = run0; b < run1; ++b) mine += span_of(a, b, 0).steps;
    before = mine;
#pragma unroll
    for (uint32_t o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += x;
    }
    uint32_t* const totals = reinterpret_cast<uint32_t*>(sums);
    if (lane == 31) totals[warp] = before;
    __syncthreads();
    uint32_t all = 0;
    before -= mine;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) {
      if (w < warp) before += totals[w];
      all += totals[w];
    }
    // A short line is cut finely instead (us without and with: one sequence of 600 tokens 7.7 / 8.6, 4 of 500 9.5 / 10.5; one of
    // 6000 16.1 / 15.1, 4 of 3000 19.6 / 18.0).
    extra = all * units >= 2 * gridDim.x ? kExtra : 0;
    mine += extra * (run1 - run0), before += extra * run0;
    cuts.cut((all + extra * a.n_seqs) * units, gridDim.x);
  }
  if (blockIdx.x >= cuts.parts) return;
  const uint32_t s0 = cuts.begin(blockIdx.x), n_steps = cuts.begin(blockIdx.x + 1) - s0;
  Place at;
  {
    // the thread whose run of sequences holds the first step knows where that is
    uint32_t* const found = shared_word;
    if (s0 >= before * units && s0 < (before + mine) * units) {
      uint32_t pre = before, b = run0, steps;
#pragma unroll 1
      for (;; ++b) {
        steps = span_of(a, b, extra).steps;
        if (s0 < (pre + steps) * units) break;
        pre += steps;
      }
      const uint32_t r = s0 - pre * units;
      found[0] = b, found[1] = r / steps, found[2] = r % steps;
    }
    __syncthreads();
    at.b = found[0], at.u = found[1], at.step = found[2];
    at.span = span_of(a, at.b, extra);
  }
  if (a.status && blockIdx.x == 0)
#pragma unroll 1
    for (uint32_t b = run0; b < run1; ++b)
      if (a.lengths[b] > int32_t(a.capacity)) raise(a.status, BCP_BAD_LENGTH);

  // ---- filling the ring: the next 16 tokens of this warp.  Lane r (and r + 16) looks up the page of token
  // r one turn ahead, so that the copies do not wait for the block table.
  Place ahead = at;
  uint32_t left = n_steps, fill_stage = 0, off = 0;
  int32_t page = -1;
  auto look_up = [&]() {
    const uint32_t pos = ahead.span.base + ahead.step * kStep + warp * kTok + (lane & 15);
    page = -1;
    if (pos >= ahead.span.first && pos < ahead.span.len) {
      const uint32_t n = a.page_size.div(pos);
      off = pos - n * a.page_size.d;
      page = a.block_table[ahead.b * a.table_stride + n];
      if (uint32_t(page) >= a.n_pages) {
        raise(a.status, BCP_BAD_PAGE);
        page = -1;
      }
    }
  };
  // The queries of a unit are brought to the L1 cache when its first tile is filled: a lane per 128 bytes.
  auto touch_queries = [&]() {
    const uint32_t h = ahead.u / a.row_tiles, r = (ahead.u - h * a.row_tiles) * S::ROWS + lane / (DP / 64), d = lane % (DP / 64) * 64;
    if (lane < S::ROWS * (DP / 64) && r < a.group && d < a.head_dim) {
      uint32_t ignored;
      asm volatile("ld.global.ca.u32 %0, [%1];" : "=r"(ignored) : "l"(static_cast<const char*>(a.q) + (ahead.b * a.q_token + (h * a.group + r) * a.q_head + d) * 2));
    }
  };
  const int64_t v_from_k = static_cast<const char*>(a.v) - static_cast<const char*>(a.k);
  auto produce = [&]() {
    if (left) {
      const uint32_t stage = ring + fill_stage * S::STAGE;
      const uint32_t h = NT * 8 >= a.group ? ahead.u : ahead.u / a.row_tiles;
      const bool on = page >= 0;
      const uint32_t live = __ballot_sync(0xffffffffu, on) & 0xffffu;
      if (live) {
        constexpr int kRows = 32 / S::CPR;  // rows that one turn of the copies covers
        const uint32_t l = lane / S::CPR, c = lane % S::CPR;
        const uint64_t row = on ? uint64_t(uint32_t(page)) * a.page_stride + uint64_t(h) * a.head_stride + uint64_t(off) * a.token_stride : 0;
        // Each lane copies one column of chunks.  In a tile that is live throughout and lies in one page
        // (the offsets did not start again) rows are a stride apart; else each row is looked up.
        const bool inside = c * 16 < a.head_dim * S::ES;
        if (__all_sync(0xffffffffu, on && off >= (lane & 15))) {
          const uint64_t step = uint64_t(a.token_stride) * (kRows * S::ES);
          const char* from = static_cast<const char*>(a.k) + (__shfl_sync(0xffffffffu, row, l) * S::ES + (inside ? c * 16 : 0));
#pragma unroll
          for (int i = 0; i < kTok / kRows; ++i) {
            copy16(stage + key_at<S::CPR>(i * kRows + l, c), from, inside);
            copy16(stage + S::SIDE + value_at<S::CPR, S::quant>(i * kRows + l, c), from + v_from_k, inside);
            from += step;
          }
        } else {
#pragma unroll 2
          for (int i = 0; i < kTok / kRows; ++i) {
            const uint32_t r = i * kRows + l;
            const bool copy = (live >> r & 1) && inside;
            const uint64_t x = __shfl_sync(0xffffffffu, row, r) * S::ES + c * 16;
            const char* const from = static_cast<const char*>(a.k) + (copy ? x : 0);
            copy16(stage + key_at<S::CPR>(r, c), from, copy);
            copy16(stage + S::SIDE + value_at<S::CPR, S::quant>(r, c), from + v_from_k, copy);
          }
        }
        if (S::quant) {
          const uint64_t n = uint64_t(uint32_t(page) * a.n_heads + h) * a.page_size.d + off;
          copy4(stage + 2 * S::SIDE + lane * 4, (lane < 16 ? a.k_scale : a.v_scale) + (on ? n : 0), on);
        }
      }
      if (lane == 0) *reinterpret_cast<uint32_t*>(ring_ptr + fill_stage * S::STAGE + S::STAGE - 16) = live;
      fill_stage = fill_stage + 1 == S::STAGES ? 0 : fill_stage + 1;
      if (--left) {
        advance(ahead, a, units, extra, true);
        look_up();
        if (ahead.step == 0) touch_queries();
      }
    }
    copies_end();  // one group per stage, empty ones at the end
  };
  touch_queries();
  look_up();
#pragma unroll 1
  for (int i = 0; i < S::STAGES - 1; ++i) produce();

  uint32_t done = 0, use_stage = 0;
  while (done < n_steps) {
    // ---- one stretch: steps [at.step, at.step + n) of one sequence, cache head and row tile
    const uint32_t n = min(at.span.steps - at.step, n_steps - done);
    const uint32_t h = at.u / a.row_tiles, row0 = (at.u - h * a.row_tiles) * S::ROWS;
    // the queries as column fragments; head dimensions in the order in which the key vectors give them
    uint32_t qf[NT][DP / 16][2];
    float factor[NT][2];  // what turns a raw product into a score, for columns 2 q4 and 2 q4 + 1
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const bool row_on = row0 + t * 8 + g < a.group;
      const int64_t q0 = at.b * a.q_token + (h * a.group + row0 + t * 8 + g) * a.q_head;
      float up = 1.f, down = 1.f;
      uint2 raw[DP / 16];
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        // 16-byte key vectors hold two (16-bit) or four (8-bit) such groups of four dimensions
        const uint32_t d = S::quant ? 64 * (s / 4) + 16 * q4 + 4 * (s % 4) : 32 * (s / 2) + 8 * q4 + 4 * (s % 2);
        raw[s] = row_on && d < a.head_dim ? *reinterpret_cast<const uint2*>(static_cast<const char*>(a.q) + (q0 + d) * 2) : make_uint2(0, 0);
      }
      if (S::quant) {
        // a power of two brings the largest element into [1, 2): bfloat16 queries then fit binary16 with
        // an error of at most 2^-25 of the largest element
        uint32_t top = 0;
        float x[DP / 16][4];
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[s][i] = query_at(&raw[s], i, a.q_is_bf16);
            top = max(top, __float_as_uint(x[s][i]) & 0x7fffffffu);
          }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const uint32_t e = top >> 23 == 254 ? 253 : top >> 23;
        if (e >= 1 && e <= 253) up = __uint_as_float((254 - e) << 23), down = __uint_as_float(e << 23);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          qf[t][s][0] = pack16<false>(x[s][0] * up, x[s][1] * up);
          qf[t][s][1] = pack16<false>(x[s][2] * up, x[s][3] * up);
        }
      } else {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) qf[t][s][0] = raw[s].x, qf[t][s][1] = raw[s].y;
      }
      factor[t][0] = __shfl_sync(0xffffffffu, down, 8 * q4) * a.scale_log2;  // lane 4 n holds column n
      factor[t][1] = __shfl_sync(0xffffffffu, down, 8 * q4 + 4) * a.scale_log2;
    }
    float o[NT][DP / 16][4], ref[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      ref[t][0] = ref[t][1] = kNone, l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int m = 0; m < DP / 16; ++m) o[t][m][0] = o[t][m][1] = o[t][m][2] = o[t][m][3] = 0.f;
    }

    for (uint32_t i = 0; i < n; ++i) {
      copies_wait<S::STAGES - 2>();
      __syncwarp();  // every lane's copies have landed, and every lane is done with the stage that is filled next
      const uint32_t stage = ring + use_stage * S::STAGE;
      const unsigned char* const tile = ring_ptr + use_stage * S::STAGE;
      auto load16 = [&](uint32_t at) { return *reinterpret_cast<const uint4*>(tile + at); };
      const uint32_t live = *reinterpret_cast<const uint32_t*>(tile + S::STAGE - 16);
      use_stage = use_stage + 1 == S::STAGES ? 0 : use_stage + 1;
      produce();
      if (!live) continue;

      // scores of 16 tokens (rows) and 8 NT heads (columns)
      float s[NT][4], s2[NT][4];  // two sums, so that no product waits for the one before it
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[t][c] = s2[t][c] = 0.f;
      if constexpr (!S::quant) {
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) {
          const uint4 x = load16(key_at<S::CPR>(g, 4 * j + q4)), y = load16(key_at<S::CPR>(g + 8, 4 * j + q4));
          const uint32_t a0[4] = {x.x, y.x, x.y, y.y}, a1[4] = {x.z, y.z, x.w, y.w};
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mma<kBf16>(s[t], a0, qf[t][2 * j]);
            mma<kBf16>(s2[t], a1, qf[t][2 * j + 1]);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < DP / 64; ++j) {
          const uint4 x = load16(key_at<S::CPR>(g, 4 * j + q4)), y = load16(key_at<S::CPR>(g + 8, 4 * j + q4));
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t f[4];
            widen4<FMT>(xs[w], f[0], f[2]);
            widen4<FMT>(ys[w], f[1], f[3]);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma<kBf16>(w & 1 ? s2[t] : s[t], f, qf[t][4 * j + w]);
          }
        }
      }
      // Scores of tokens g and g + 8.  The scale f of 8-bit values goes into the weight of the product as log2 f in its
      // exponent, so that these weights stay in range whatever the scales; the reference is the largest of these exponents.
      // The denominators get exp2(score - reference) without f: from the weight it could not be had back, for next to a scale
      // of 2^40 the weight of a vector of zeros (f = 2^-96) underflows, though its score may be the largest.
      float vlog[2] = {0.f, 0.f}, ks[2] = {1.f, 1.f};
      if constexpr (S::quant) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          ks[r] = *reinterpret_cast<const float*>(tile + 2 * S::SIDE + (g + 8 * r) * 4);
          // scales below 2^-96 (a zero, too) count as that; a NaN stays one
          float f = *reinterpret_cast<const float*>(tile + 2 * S::SIDE + 64 + (g + 8 * r) * 4);
          if (f < 0x1p-96f) f = 0x1p-96f;
          vlog[r] = log2_fast(f);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[t][c] = fmaf(s[t][c] + s2[t][c], factor[t][c & 1] * ks[c >> 1], vlog[c >> 1]);
      if (live != 0xffffu) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
          if (!(live >> (g + 8 * r) & 1)) {
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][2 * r] = s[t][2 * r + 1] = -INFINITY;
          }
      }
      bool above = false;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 2; ++c) above |= fmaxf(s[t][c], s[t][c + 2]) > ref[t][c] + 8.f;
      if (__any_sync(0xffffffffu, above)) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float m = fmaxf(s[t][c], s[t][c + 2]);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            m = fmaxf(m, ref[t][c]);
            const Factor<S::quant> down(ref[t][c] - m);
            ref[t][c] = m;
            l[t][c] = down.denominator(l[t][c]);
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) o[t][k][c] *= down.all, o[t][k][c + 2] *= down.all;
          }
      }
      uint32_t pf[NT][2], rest[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float p[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float e = s[t][c] - (ref[t][c & 1] - kLift);
          p[c] = exp2_fast(e);
          l[t][c & 1] += S::quant ? exp2_fast(e - vlog[c >> 1]) : p[c];
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float x = p[2 * r], y = p[2 * r + 1];
          if constexpr (kRest) {
            pf[t][r] = transpose8x8(upper_halves(x, y));
            rest[t][r] = transpose8x8(pack16<kBf16>(lower_half(x), lower_half(y)));
          } else {
            pf[t][r] = transpose8x8(pack16<kBf16>(x, y));
          }
        }
      }
      // sums over the values: rows are head dimensions
      if constexpr (!S::quant) {
#pragma unroll
        for (int m = 0; m < DP / 16; ++m) {
          uint32_t f[4];
          load_transposed(f, stage + S::SIDE + value_at<S::CPR, false>((lane & 7) + (lane >> 4 << 3), 2 * m + (lane >> 3 & 1)));
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mma<kBf16>(o[t][m], f, pf[t]);
            if constexpr (kRest) mma<kBf16>(o[t][m], f, rest[t]);
          }
        }
      } else {
        constexpr int kWords = DP >= 128 ? 4 : DP / 32;  // words a lane takes of each of its four tokens at once
#pragma unroll
        for (int j = 0; j < (DP + 127) / 128; ++j) {
          uint32_t w[4][kWords];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t token = 2 * q4 + (r & 1) + 8 * (r >> 1);
            if constexpr (kWords == 4) {
              const uint4 x = load16(S::SIDE + value_at<S::CPR, true>(token, 8 * j + g));
              w[r][0] = x.x, w[r][1] = x.y, w[r][2] = x.z, w[r][3] = x.w;
            } else {
              const uint2 x = *reinterpret_cast<const uint2*>(tile + S::SIDE + value_at<S::CPR, true>(token, g >> 1) + (g & 1) * 8);
              w[r][0] = x.x, w[r][1] = x.y;
            }
          }
#pragma unroll
          for (int x = 0; x < kWords; ++x) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t pick = half ? 0x7362 : 0x5140;
              uint32_t f[4];
              widen4<FMT>(__byte_perm(w[0][x], w[1][x], pick), f[0], f[1]);
              widen4<FMT>(__byte_perm(w[2][x], w[3][x], pick), f[2], f[3]);
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                mma<kBf16>(o[t][8 * j + 2 * x + half], f, pf[t]);
                if constexpr (kRest) mma<kBf16>(o[t][8 * j + 2 * x + half], f, rest[t]);
              }
            }
          }
        }
      }
    }
    done += n;

    // ---- The end of a stretch: the four warps' sums are added up, and where the unit lies in several parts
    // those of the parts.  One piece of code does both, and its loops are kept short: it runs a few times per
    // CTA, and fetching instructions for the first time costs more than executing them.
    const bool whole = at.step == 0 && at.step + n == at.span.steps;
    float* const own = sums + warp * S::PART;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t col = t * 8 + 2 * q4 + c;
        float x = l[t][c];
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        x += __shfl_xor_sync(0xffffffffu, x, 16);
        if (g == 0) own[S::ROWS * DP + col] = ref[t][c], own[S::ROWS * (DP + 1) + col] = x;
        if constexpr (S::quant) {  // two blocks of rows hold four neighbouring dimensions
#pragma unroll
          for (int k = 0; k < DP / 16; k += 2) {
            const uint32_t d = DP >= 128 ? 128 * (k / 8) + 16 * g + 2 * (k % 8) : (DP / 8) * g + 2 * k;
            *reinterpret_cast<float4*>(own + sum_at<DP, true>(col, d)) = make_float4(o[t][k][c], o[t][k][c + 2], o[t][k + 1][c], o[t][k + 1][c + 2]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int r = 0; r < 2; ++r) own[sum_at<DP, false>(col, 16 * k + 8 * r + g)] = o[t][k][c + 2 * r];
        }
      }
    __syncthreads();
    const uint32_t place = s0 + done - n;                                                         // of the stretch's first step on the line
    float* to = a.parts + (uint64_t(blockIdx.x) * 2 + (place != s0)) * S::PART;                   // where the sums go
    const float *first = sums, *rest = sums;                                                      // the sums to add: first, rest + i * apart
    uint64_t apart = S::PART;
    uint32_t n_sums = kWarps, f = 0, groups = 0, first_place = 0, p0 = 0;
    bool last = whole;
#pragma unroll 1
    for (int round = 0;; ++round) {  // the warps, the parts of a group, the groups
      // Sixteen threads per head, four dimensions at a time; of each sixteen sums one is this thread's to weigh.
      const uint32_t sub = tid & 15;
#pragma unroll 1
      for (uint32_t col = tid >> 4; col < S::ROWS; col += 8) {
        const bool on = row0 + col < a.group;
        float m = kNone, den = 0.f, r[kGroup / 16], w[kGroup / 16];
        auto from_of = [&](uint32_t i) { return i ? rest + i * apart : first; };
#pragma unroll
        for (int k = 0; k < int(kGroup / 16); ++k) {
          r[k] = kNone, w[k] = 0.f;
          if (sub + 16 * k < n_sums && on) {
            const float* const from = from_of(sub + 16 * k) + S::ROWS * DP + col;
            r[k] = load_sums(from), w[k] = load_sums(from + S::ROWS);
          }
          m = fmaxf(m, r[k]);
        }
#pragma unroll
        for (int i = 1; i < 16; i <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, i));
#pragma unroll
        for (int k = 0; k < int(kGroup / 16); ++k) {
          const Factor<S::quant> down(r[k] - m);
          den += down.denominator(w[k]);
          w[k] = down.all;
        }
#pragma unroll
        for (int i = 1; i < 16; i <<= 1) den += __shfl_xor_sync(0xffffffffu, den, i);
        float4 x[DP / 64];
#pragma unroll
        for (int i = 0; i < DP / 64; ++i) x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (uint32_t i0 = 0; i0 < n_sums; i0 += 4) {
          const float mine = i0 < 16 ? w[0] : i0 < 32 ? w[1] : i0 < 48 ? w[2] : w[3];
          float4 y[4][DP / 64];
          if (on) {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
              const float* const from = from_of(min(i0 + j, n_sums - 1));
#pragma unroll
              for (int i = 0; i < DP / 64; ++i) y[j][i] = load_sums4(from + sum_at<DP, S::quant>(col, 64 * i + 4 * sub));
            }
          }
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) {
            const float weight = __shfl_sync(0xffffffffu, mine, (lane & 16) + (i0 & 15) + j);
            if (on && i0 + j < n_sums) {
#pragma unroll
              for (int i = 0; i < DP / 64; ++i)
                x[i].x += y[j][i].x * weight, x[i].y += y[j][i].y * weight, x[i].z += y[j][i].z * weight, x[i].w += y[j][i].w * weight;
            }
          }
        }
        if (!on) continue;
        if (!last) {  // in the second round over the first part's own sums, which these threads alone have read
#pragma unroll
          for (int i = 0; i < DP / 64; ++i) __stcg(reinterpret_cast<float4*>(to + sum_at<DP, S::quant>(col, 64 * i + 4 * sub)), x[i]);
          if (sub == 0) __stcg(to + S::ROWS * DP + col, m), __stcg(to + S::ROWS * (DP + 1) + col, den);
          continue;
        }
        const uint32_t qh = h * a.group + row0 + col;
        const float inv = den == 0.f ? 0.f : reciprocal_fast(den);  // up to 2^127, where the fast division gives zero
#pragma unroll
        for (int i = 0; i < DP / 64; ++i) {
          const uint32_t d = 64 * i + 4 * sub;
          if (d >= a.head_dim) break;
          uint2 y;
          y.x = a.q_is_bf16 ? pack16<true>(x[i].x * inv, x[i].y * inv) : pack16<false>(x[i].x * inv, x[i].y * inv);
          y.y = a.q_is_bf16 ? pack16<true>(x[i].z * inv, x[i].w * inv) : pack16<false>(x[i].z * inv, x[i].w * inv);
          *reinterpret_cast<uint2*>(static_cast<char*>(a.out) + (at.b * a.out_token + qh * a.out_head + d) * 2) = y;
        }
        if (sub == 0 && a.lse)
          a.lse[uint64_t(at.b) * (a.n_heads * a.group) + qh] = den == 0.f ? -INFINITY : (m - kLift + log2_fast(den)) * 0.6931471805599453f;
      }
      if (last) break;
      // the parts that the unit lies in; the first has it in its second place unless it begins with it
      if (round == 0) {
        const uint32_t u0 = place - at.step, p1 = cuts.part_of(u0 + at.span.steps - 1);
        p0 = cuts.part_of(u0);
        first_place = 2 * p0 + (cuts.begin(p0) != u0);
        groups = (p1 - p0) / kGroup + 1;
        f = p0 + (blockIdx.x - p0) / kGroup * kGroup;
        n_sums = min(p1 - f + 1, kGroup), apart = 2 * S::PART;
      } else {
        f = p0, n_sums = groups, apart = 2 * kGroup * S::PART;
      }
      const uint32_t place_of_f = f == p0 ? first_place : 2 * f;
      uint32_t* const counter = round == 0 ? a.part_count + place_of_f : a.group_count + first_place;
      // Goes on if this CTA is the last to come to the counter; what the others wrote before is visible then.
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const bool complete = atomicAdd(counter, 1u) + 1 == n_sums;
        *shared_word = complete;
        if (complete) *counter = 0;  // ready for the next call
      }
      __syncthreads();
      if (!*static_cast<volatile uint32_t*>(shared_word)) break;
      __threadfence();
      last = round == 1 || groups == 1;
      to = a.parts + uint64_t(place_of_f) * S::PART, first = to, rest = a.parts + uint64_t(2 * f) * S::PART;
    }
    __syncthreads();  // the sums have been read
    at.step += n - 1;
    advance(at, a, units, extra, done < n_steps);
  }
}

// ------------------------------------------------------------------------------ launch
typedef void (*Kernel)(AttendArgs);
struct Variant {
  Kernel kernel;
  uint32_t smem, rows, part_floats;
};

template <int FMT, int DP, int NT>
Variant variant() {
  typedef Shape<FMT, DP, NT> S;
  return Variant{bcp_kv_attend_kernel<FMT, DP, NT>, S::SMEM, S::ROWS, S::PART};
}
template <int FMT>
Variant variant_of(uint32_t head_dim, uint32_t group) {
  // Query heads of a group beyond eight take a second column block (16 rows share each key and value that
  // was read); with 256 dimensions the sums of 16 rows would not fit the registers, more rows are more units.
  if (head_dim <= 64) return group <= 8 ? variant<FMT, 64, 1>() : variant<FMT, 64, 2>();
  if (head_dim <= 128) return group <= 8 ? variant<FMT, 128, 1>() : variant<FMT, 128, 2>();
  return variant<FMT, 256, 1>();
}
Variant variant_of(uint32_t format, uint32_t head_dim, uint32_t group) {
  switch (format) {
    case BCP_BF16: return variant_of<BCP_BF16>(head_dim, group);
    case BCP_F16: return variant_of<BCP_F16>(head_dim, group);
    case BCP_E4M3: return variant_of<BCP_E4M3>(head_dim, group);
    default: return variant_of<BCP_I8>(head_dim, group);
  }
}

// CTAs of a kernel that fit on the current device, asked once per kernel and device.
int resident_ctas(const Variant& v, uint32_t* out) {
  struct Known {
    Kernel kernel;
    int device;
    uint32_t ctas;
  };
  static std::mutex mu;
  static Known known[256];
  static int n_known = 0;
  int device = 0;
  BCP_CUDA(cudaGetDevice(&device));
  std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < n_known; ++i)
    if (known[i].kernel == v.kernel && known[i].device == device) {
      *out = known[i].ctas;
      return BCP_OK;
    }
  int per_sm = 0, sms = 0;
  BCP_CUDA(cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(v.smem)));
  BCP_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, v.kernel, kWarps * 32, v.smem));
  BCP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  if (per_sm < 1) return fail(BCP_ERR_CUDA, "bcp_kv_attend: the kernel does not fit on this device");
  *out = uint32_t(per_sm * sms);
  static_assert(kGroup == 64, "four weights a thread in the join");
  if (*out > kGroup * kGroup) *out = kGroup * kGroup;  // two rounds of joining
  if (n_known < 256) known[n_known++] = Known{v.kernel, device, *out};
  return BCP_OK;
}

// The workspace: counters of the parts, of their groups, then the sums of the parts.  The counters have room for the most
// parts there can be and lie at fixed places, so that calls of any shapes find them as the last one left them.
constexpr uint64_t kCounterBytes = uint64_t(kGroup) * kGroup * 2 * 4;
uint64_t workspace_bytes_of(uint32_t ctas, const Variant& v) { return 2 * kCounterBytes + uint64_t(ctas) * 2 * v.part_floats * 4; }

int check_group(const char* call, const bcp_kv_cache* c, uint32_t n_q_heads) {
  if (!n_q_heads || n_q_heads > 65536 || n_q_heads % c->n_heads)
    return fail(BCP_ERR_MISMATCH, "%s: %u query heads are not a multiple of %u cache heads", call, n_q_heads, c->n_heads);
  return BCP_OK;
}

}  // namespace

extern "C" int bcp_kv_attend_workspace(const bcp_kv_cache* cache, uint32_t n_q_heads, uint32_t max_seqs, uint64_t* bytes) {
  const char* call = "bcp_kv_attend_workspace";
  if (!bytes) return fail(BCP_ERR_INVALID, "%s: bytes is NULL", call);
  if (int rc = check_cache(call, cache)) return rc;
  if (int rc = check_group(call, cache, n_q_heads)) return rc;
  const uint32_t group = n_q_heads / cache->n_heads;
  const Variant v = variant_of(cache->format, cache->head_dim, group);
  uint32_t ctas = 0;
  if (int rc = resident_ctas(v, &ctas)) return rc;
  (void)max_seqs;  // the parts are as many as CTAs, however many sequences they come from
  *bytes = workspace_bytes_of(ctas, v);
  return BCP_OK;
}

extern "C" int bcp_kv_attend(const bcp_kv_cache* c, const bcp_heads* q, const bcp_heads* out, float* lse, uint32_t n_seqs,
                             const int32_t* block_table, int64_t table_stride, uint32_t table_width, const int32_t* lengths, float scale,
                             uint32_t window, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* call = "bcp_kv_attend";
  if (int rc = check_cache(call, c)) return rc;
  if (int rc = check_heads(call, "q", q, false, c->head_dim, n_seqs)) return rc;
  if (int rc = check_heads(call, "out", out, true, c->head_dim, n_seqs)) return rc;
  if (int rc = check_group(call, c, q->n_heads)) return rc;
  if (out->n_heads != q->n_heads || out->type != q->type) return fail(BCP_ERR_MISMATCH, "%s: out must have the heads and the type of q", call);
  if (q->type == BCP_F32 || (!is_8bit(c->format) && q->type != c->format))
    return fail(BCP_ERR_MISMATCH, "%s: queries of type %u over a cache of format %u (16-bit queries, of the cache's type unless that has 8 bits)", call,
                q->type, c->format);
  if (!rows_aligned(q, 8) || !rows_aligned(out, 8)) return fail(BCP_ERR_INVALID, "%s: rows of q and out must start on 8-byte boundaries", call);
  if (n_seqs > 0x7fffffffu) return fail(BCP_ERR_INVALID, "%s: %u sequences", call, n_seqs);
  if (n_seqs == 0) return BCP_OK;
  if (!block_table || !lengths || table_stride < 0 || (n_seqs > 1 && table_stride < int64_t(table_width)))
    return fail(BCP_ERR_INVALID, "%s: block_table or lengths is NULL, or rows of the table overlap", call);
  if (!(scale == scale) || scale - scale != 0.f) return fail(BCP_ERR_INVALID, "%s: scale is not a finite number", call);

  const uint32_t group = q->n_heads / c->n_heads;
  const Variant v = variant_of(c->format, c->head_dim, group);
  uint32_t ctas = 0;
  if (int rc = resident_ctas(v, &ctas)) return rc;
  AttendArgs a = {};
  a.row_tiles = (group + v.rows - 1) / v.rows;
  const uint64_t units = uint64_t(n_seqs) * c->n_heads * a.row_tiles;
  const uint64_t need = workspace_bytes_of(ctas, v);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return fail(BCP_ERR_INVALID, "%s: workspace is NULL or not 16-byte aligned", call);
  if (workspace_bytes < need)
    return fail(BCP_ERR_CAPACITY, "%s: a workspace of %llu bytes, %llu needed", call, (unsigned long long)workspace_bytes, (unsigned long long)need);
  const uint64_t capacity = uint64_t(table_width) * c->page_size;
  a.capacity = uint32_t(capacity < 0x7fffff00u ? capacity : 0x7fffff00u);
  a.k = c->k, a.v = c->v, a.k_scale = c->k_scale, a.v_scale = c->v_scale;
  a.page_stride = uint32_t(c->page_stride), a.head_stride = uint32_t(c->head_stride), a.token_stride = uint32_t(c->token_stride);
  a.n_pages = c->n_pages, a.n_heads = c->n_heads, a.head_dim = c->head_dim;
  a.page_size = FastDiv(c->page_size);
  a.status = c->status;
  a.q = q->data, a.out = out->data, a.lse = lse;
  a.q_token = q->token_stride, a.q_head = q->head_stride, a.out_token = out->token_stride, a.out_head = out->head_stride;
  a.q_is_bf16 = q->type == BCP_BF16, a.group = group, a.n_seqs = n_seqs;
  a.block_table = block_table, a.table_stride = table_stride, a.lengths = lengths;
  a.scale_log2 = scale * kLog2e, a.window = window;
  char* const w = static_cast<char*>(workspace);
  a.part_count = reinterpret_cast<uint32_t*>(w);
  a.group_count = reinterpret_cast<uint32_t*>(w + kCounterBytes);
  a.parts = reinterpret_cast<float*>(w + 2 * kCounterBytes);
  // steps are counted in 32 bits, kExtra more for each unit included; no more CTAs than the longest lengths the table
  // allows can use
  uint32_t longest = a.capacity;
  if (window && window < longest) longest = window + 15 < longest ? window + 15 : longest;
  const uint64_t most = units * (longest / kStep + 1);
  if (most + kExtra * units > 0x7fffffffull) return fail(BCP_ERR_CAPACITY, "%s: %u sequences of up to %u tokens are too many for one call", call, n_seqs, longest);
  BCP_CUDA(launch_early(v.kernel, uint32_t(most < ctas ? most : ctas), kWarps * 32, v.smem, static_cast<cudaStream_t>(stream), a));
  return BCP_OK;
}

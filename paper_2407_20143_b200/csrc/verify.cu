// Drafted tokens verified against the target's probabilities, and the next token drawn.
//
// Mathematics.  Draft i of a sequence is accepted iff u_i q_i(x_i) < p_i(x_i); at the first one that is not, the next token is drawn from
// max(p_i - q_i, 0), else from the row behind the last draft: the lowest index whose cumulative weight exceeds u times the sum of
// all weights.  Rows of logits stand for p(j) = exp((z_j - m) / T) / S, so each is read once for m and S (a running maximum, the sum
// brought to a new one where it grows) before the first draft can be judged.
//
// A cluster of CTAs takes a sequence, each CTA a stretch of the vocabulary in all rows; maxima and sums are exchanged through the cluster's shared memory, every CTA
// judges all drafts itself, and the weights of the one row that is drawn from (two with drafts' rows; still in the L2 cache) are
// summed by stretches of 256 tokens.  The CTA in whose stretch the drawn place lies goes over those 256 again.  One launch, no
// workspace, no atomics: the same bits on every run.
//
// What bounds it: an exponential for every element (16 a clock and SM: 74 million take 16 us) beside reading the rows, and for few sequences the chain of phases.
// Measured on one B200, among other calls: 64 sequences of 4 drafts over 128,256 tokens, bfloat16, 148 MB: 60 us, of which the maxima and sums take 30, and SMs with four CTAs
// end 15 us after those with three; one sequence of 4 drafts over 32,768: 15 us; 200 rows of 50,304 sampled, binary16: 23 us; 37 sequences of up to 7 looked-up drafts
// over 50,257 probabilities, binary32: 8.7 us (only the row that is drawn from is read); 64 sequences of 4 looked-up drafts over 128,256 logits, binary32: 43 us.
//
// Precision: a token hangs on a comparison, so sums are held in 64 bits and the probability of a drafted token is computed in 64 bits
// from its logit; the terms of the sums are binary32 (2^-22 of each).  Of terms made from logits 32 (rows) or 256 (the draw) are added in binary32 first, at most
// eight additions deep (2^-21); weights that are given are added in 64 bits from the first on.
#include <cooperative_groups.h>

#include <type_traits>

#include "decode.cuh"

using namespace bcp;
namespace cg = cooperative_groups;

namespace {

// Of a CTA, four an SM.  (1024 and one an SM for few sequences: 8 of 4 drafts over 128,256 tokens 42.9 us, 26.2 with 256; one over 32,768 16.5 and 15.2; 512 for
// many: 64 sequences 67.8 and 57.7.)
constexpr uint32_t kThreads = 256;
constexpr uint32_t kParts = 8;                           // warps that share a row's part, at most
constexpr uint32_t kSegment = 256;  // tokens of a stretch that is summed for the draw: eight a lane
constexpr int32_t kNoToken = -(1 << 30);
constexpr float kLog2e = 1.4426950408889634f;

struct VerifyArgs {
  const void *target, *draft;
  int64_t t_seq, t_row, d_seq, d_row;
  uint32_t vocab, n_drafts, certain;
  const int64_t* drafts;
  const float *uniform, *temperature;
  int64_t* tokens;
  int32_t* accepted;
};

// What is known of a row, or a part of it: the largest value and the sum of exp2((z - m) c); greedy: the index of the largest (m a NaN: the row holds one).
struct RowSum {
  float m;
  uint32_t index;
  double s;
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nadd.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
// The larger one; a NaN if either is one (which fmaxf would pass over).
__device__ __forceinline__ float largest(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// A row in units of eight elements that start on 16-byte boundaries: unit v has elements 8 v - shift and on, of which those outside
// 0 .. n - 1 are not the row's.
template <typename T>
struct Row {
  const T* p;
  uint32_t shift, n, units;
  __device__ __forceinline__ Row(const void* base, int64_t at, uint32_t n_) : p(static_cast<const T*>(base) + at), n(n_) {
    shift = uint32_t(reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T);
    units = (n + shift + 7) / 8;
  }
  __device__ __forceinline__ int32_t first(uint32_t v) const { return int32_t(8 * v) - int32_t(shift); }
  // Unit v as it lies in memory; `none` where the row has no elements, and from unit `end` on.
  __device__ __forceinline__ void raw(uint32_t v, uint32_t end, float none, Raw<T, 8>& x) const {
    const int32_t e = first(v);
    if (v < end && e >= 0 && uint32_t(e) + 8 <= n) {
      x.load(p + e);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x.set(i, v < end && e + i >= 0 && uint32_t(e + i) < n ? p[e + i] : from_f32<T>(none));
    }
  }
};

__device__ __forceinline__ float largest8(const Raw<float, 8>& r) {
  float m = r.get(0);
#pragma unroll
  for (int i = 1; i < 8; ++i) m = largest(m, r.get(i));
  return m;
}
template <typename T, typename T2>
__device__ __forceinline__ float largest_of_pairs(const Raw<T, 8>& r) {
  T2 p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const T2*>(&r.w[i]);
  const T2 m = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
  return largest(to_f32(m.x), to_f32(m.y));
}
__device__ __forceinline__ float largest8(const Raw<__nv_bfloat16, 8>& r) { return largest_of_pairs<__nv_bfloat16, __nv_bfloat162>(r); }
__device__ __forceinline__ float largest8(const Raw<__half, 8>& r) { return largest_of_pairs<__half, __half2>(r); }

// Units first, first + 32, .. below end of a row, as this lane sees them.  (Terms are exp2((z - m) c): with one fused z c - m c the largest would be off by the
// rounding of m c, which low temperatures make large.)
template <typename T>
__device__ __forceinline__ RowSum look_over(const Row<T>& row, uint32_t first, uint32_t end, float c, bool greedy) {
  RowSum r = {-INFINITY, 0xffffffffu, 0.0};
  constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;
  for (uint32_t v0 = first; v0 < end; v0 += kAhead * 32) {
    Raw<T, 8> x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) row.raw(v0 + j * 32, end, -INFINITY, x[j]);
    float top = largest8(x[0]);
#pragma unroll
    for (int j = 1; j < kAhead; ++j) top = largest(top, largest8(x[j]));
    if (greedy) {
      if (!(top <= r.m) && r.m == r.m) {  // larger, or a NaN, which stays and is at no index
        r.m = top, r.index = 0xffffffffu;
#pragma unroll
        for (int j = kAhead - 1; j >= 0; --j)
#pragma unroll
          for (int i = 7; i >= 0; --i)
            if (to_f32(x[j].get(i)) == top) r.index = uint32_t(row.first(v0 + j * 32) + i);
      }
      continue;
    }
    if (top > r.m) r.s *= exp2_fast((r.m - top) * c), r.m = top;
    const float ref = reference(r.m);
    const float2 less = make_float2(-ref, -ref), c2 = make_float2(c, c);
    float2 s[4] = {};
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float2 e = mul2(add2(make_float2(to_f32(x[j].get(i)), to_f32(x[j].get(i + 1))), less), c2);
        s[i / 2] = add2(s[i / 2], make_float2(exp2_fast(e.x), exp2_fast(e.y)));
      }
    s[0] = add2(add2(s[0], s[1]), add2(s[2], s[3]));
    r.s += s[0].x + s[0].y;
  }
  return r;
}
// The same of `lanes` lanes together, in all of them.
__device__ __forceinline__ RowSum join(RowSum r, float c, bool greedy, uint32_t lanes) {
  float m = r.m;
  for (uint32_t o = lanes / 2; o; o >>= 1) m = largest(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (greedy) {
    uint32_t index = r.m == m ? r.index : 0xffffffffu;
    for (uint32_t o = lanes / 2; o; o >>= 1) index = min(index, __shfl_xor_sync(0xffffffffu, index, o));
    return RowSum{m, index, 0.0};
  }
  double s = r.s * exp2_fast((r.m - reference(m)) * c);
  for (uint32_t o = lanes / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return RowSum{m, 0, s};
}

// What turns an element into a probability.
struct Scale {
  float m, c, inverse;
};

// What a stretch's weights are added up in.  Given ones are exact and may be of any size; those made from logits are at most 1 and off by 2^-22 each, and the
// eight additions of binary32 that one goes through add 2^-21.
template <bool PROB>
using Sum = std::conditional_t<PROB, double, float>;

template <typename T, bool PROB>
struct Weights {  // of the row that is drawn from
  Row<T> p, q;
  Scale ps, qs;
  bool use_q, same;   // subtract q's; its units begin where p's do
  int32_t without;    // a token that counts nothing
  __device__ __forceinline__ static float probability(float z, const Scale& s) {
    return PROB ? z : exp2_fast((z - s.m) * s.c) * s.inverse;
  }
  // Elements of units v, v + apart, .. of p, and of q at the same tokens.
  template <uint32_t N>
  __device__ __forceinline__ void read(uint32_t v, uint32_t apart, Raw<T, 8> (&x)[N], Raw<T, 8> (&y)[N]) const {
    constexpr float none = PROB ? 0.f : -INFINITY;
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) p.raw(v + j * apart, p.units, none, x[j]);
    if (use_q) {
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) {
        if (same) {
          q.raw(v + j * apart, p.units, none, y[j]);
        } else {
          const int32_t e = p.first(v + j * apart);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[j].set(i, e + i >= 0 && uint32_t(e + i) < p.n ? q.p[e + i] : from_f32<T>(none));
        }
      }
    }
  }
  __device__ __forceinline__ void weigh(int32_t e, const Raw<T, 8>& x, const Raw<T, 8>& y, float (&w)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = probability(to_f32(x.get(i)), ps);
      if (use_q) w[i] = largest(w[i] - probability(to_f32(y.get(i)), qs), 0.f);
      if (PROB && w[i] < 0.f) w[i] = 0.f;
    }
    const int32_t skip = without - e;
    if (e < 0 || uint32_t(e) + 8 > p.n || uint32_t(skip) < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((i == skip && !(PROB && w[i] != w[i])) || e + i < 0 || uint32_t(e + i) >= p.n) w[i] = 0.f;
    }
  }
};

template <typename T, bool PROB>
__global__ void __launch_bounds__(kThreads, 4) bcp_verify_kernel(const VerifyArgs a) {
  after_previous();
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const uint32_t b = blockIdx.x / ctas, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = kThreads / 32;
  const uint32_t most_rows = 2 * a.n_drafts + 1;
  extern __shared__ __align__(16) unsigned char smem[];
  RowSum* const by_warp = reinterpret_cast<RowSum*>(smem);       // [rows][parts]
  RowSum* const mine = by_warp + most_rows * kParts;             // [rows]: of this CTA's part, read by the others
  RowSum* const whole = mine + most_rows;                        // [rows]
  double* const total = reinterpret_cast<double*>(whole + most_rows);  // [2]: of this CTA's weights, read by the others
  uint32_t* const good = reinterpret_cast<uint32_t*>(total + 2);       // [n_drafts + 1]
  double* const segments = total + 2 + (a.n_drafts + 2) / 2;

  const int64_t* const drafts = a.drafts + uint64_t(b) * a.n_drafts;
  const float* const uniform = a.uniform + uint64_t(b) * (a.n_drafts + 1);
  float t = a.temperature ? a.temperature[b] : 1.f;
  const bool greedy = !PROB && !(t > 1e-30f);
  t = fminf(t, 1e30f);
  const float c = kLog2e / t;
  auto target = [&](uint32_t i) { return Row<T>(a.target, b * a.t_seq + i * a.t_row, a.vocab); };
  auto draft = [&](uint32_t i) { return Row<T>(a.draft, b * a.d_seq + i * a.d_row, a.vocab); };
  // Drafts of this sequence: up to the first negative one.  A thread has each, with what its rows say about it.
  int64_t my_draft = -1;
  float my_p = 0.f, my_q = 0.f, my_u = 0.f;
  if (tid < a.n_drafts) {
    my_draft = drafts[tid], my_u = uniform[tid];
    if (my_draft >= 0 && my_draft < int64_t(a.vocab)) {
      my_p = to_f32(target(tid).p[my_draft]);
      if (!a.certain) my_q = to_f32(draft(tid).p[my_draft]);
    }
  }
  if (tid <= a.n_drafts) good[tid] = my_draft >= 0;
  __syncthreads();
  uint32_t n = 0;
  while (n < a.n_drafts && good[n]) ++n;
  __syncthreads();

  // ---- maxima and sums of all rows: the target's 0 .. n, then the drafts'
  const uint32_t n_rows = n + 1 + (a.certain || greedy ? 0 : n);
  if (!PROB) {
    // A row's part is cut for as many warps as have a batch of loads each, so that short rows are read side by side.
    const uint32_t most = (a.vocab / 8 + ctas) / ctas, parts = most >= 1024 ? 8 : most >= 512 ? 4 : most >= 256 ? 2 : 1;
    for (uint32_t task = warp; task < n_rows * parts; task += warps) {
      const uint32_t i = task / parts, part = task % parts;
      const Row<T> row = i <= n ? target(i) : draft(i - n - 1);
      const uint32_t each = (row.units + ctas - 1) / ctas, begin = min(rank * each, row.units), end = min(begin + each, row.units);
      const uint32_t some = (end - begin + parts - 1) / parts, from = min(begin + part * some, end), to = min(from + some, end);
      const RowSum r = join(look_over(row, from + lane, to, c, greedy), c, greedy, 32);
      if (lane == 0) by_warp[i * kParts + part] = r;
    }
    __syncthreads();
    // warps join what their CTA has of a row, a lane a part, then what all CTAs have, a lane a CTA
    const RowSum nothing = {-INFINITY, 0xffffffffu, 0.0};
    for (uint32_t i = warp; i < n_rows; i += warps) {
      const RowSum r = join(lane < parts ? by_warp[i * kParts + lane] : nothing, c, greedy, 8);
      if (lane == 0) mine[i] = r;
    }
    cluster.sync();
    for (uint32_t i = warp; i < n_rows; i += warps) {
      const RowSum r = join(lane < ctas ? cluster.map_shared_rank(mine, lane)[i] : nothing, c, greedy, 16);
      if (lane == 0) whole[i] = r;
    }
    __syncthreads();
  }

  // ---- every draft is judged by a thread; the same in all CTAs
  const double nan = __longlong_as_double(0x7ff8000000000000ll);
  auto probability = [&](float z, uint32_t i) -> double {  // of an element of row i
    if (PROB) return z;
    const double s = whole[i].s;
    return s > 0 && s < INFINITY ? exp((double(z) - double(whole[i].m)) / double(t)) / s : nan;
  };
  if (tid < n) {
    bool ok = my_draft < int64_t(a.vocab);
    if (ok && greedy) {
      ok = whole[tid].index == uint32_t(my_draft);
    } else if (ok) {
      const double p = probability(my_p, tid), q = a.certain ? 1.0 : probability(my_q, n + 1 + tid);
      ok = double(my_u) * q < p;
    }
    good[tid] = ok;
  }
  __syncthreads();
  uint32_t k = 0;
  while (k < n && good[k]) ++k;
  int64_t* const tokens = a.tokens + uint64_t(b) * (a.n_drafts + 1);
  if (rank == 0) {
    for (uint32_t i = tid; i <= a.n_drafts; i += kThreads)
      if (i != k) tokens[i] = i < k ? drafts[i] : -1;
    if (tid == 0) a.accepted[b] = int32_t(k);
    if (greedy && tid == 0) tokens[k] = whole[k].m > -INFINITY ? int64_t(whole[k].index) : -1;
  }

  // ---- the next token
  if (!greedy) {
    auto scale = [&](uint32_t i) {
      Scale s = {0.f, c, 1.f};
      if (!PROB) {
        s.m = reference(whole[i].m);
        s.inverse = whole[i].s > 0 && whole[i].s < INFINITY ? float(1.0 / whole[i].s) : float(nan);
      }
      return s;
    };
    const bool rejected = k < n;
    Weights<T, PROB> w = {target(k), target(k), scale(k), scale(k), rejected && !a.certain, false, rejected && a.certain && drafts[k] < int64_t(a.vocab) ? int32_t(drafts[k]) : kNoToken};
    if (w.use_q) {
      w.q = draft(k), w.qs = scale(n + 1 + k);
      w.same = w.q.shift == w.p.shift;
    }
    // parts of whole stretches
    const uint32_t n_segments = (w.p.units + kSegment / 8 - 1) / (kSegment / 8), each = (n_segments + ctas - 1) / ctas;
    const uint32_t s0 = min(rank * each, n_segments), s1 = min(s0 + each, n_segments);
    const double u = uniform[a.n_drafts];
    // what is left after q may be nothing at all (p and q alike, a draft outside its own row), or q's row holds no number: then p itself counts
    for (int round = 0;; ++round) {
      // four stretches at a time, so that their loads are under way together
      constexpr uint32_t kTogether = sizeof(T) == 2 ? 4 : 2;
      for (uint32_t s = s0 + warp; s < s1; s += warps * kTogether) {
        Raw<T, 8> p[kTogether], q[kTogether];
        w.read(s * (kSegment / 8) + lane, warps * (kSegment / 8), p, q);
        Sum<PROB> sum[kTogether];
#pragma unroll
        for (uint32_t j = 0; j < kTogether; ++j) {
          float x[8];
          w.weigh(w.p.first((s + j * warps) * (kSegment / 8) + lane), p[j], q[j], x);
          Sum<PROB> y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = x[i];
          sum[j] = ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1)
#pragma unroll
          for (uint32_t j = 0; j < kTogether; ++j) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
#pragma unroll
        for (uint32_t j = 0; j < kTogether; ++j)
          if (lane == 0 && s + j * warps < s1) segments[s + j * warps - s0] = sum[j];
      }
      __syncthreads();
      if (warp == 0) {
        double sum = 0.0;
        for (uint32_t s = lane; s < s1 - s0; s += 32) sum += segments[s];
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) total[round] = sum;
      }
      cluster.sync();
      // a lane a CTA: all weights, what lies before, and the CTA that holds the place; if rounding has left none, the last that has any weight
      const double held = lane < ctas ? cluster.map_shared_rank(total, lane)[round] : 0.0;
      double line = held;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, line, o);
        if (int(lane) >= o) line += y;
      }
      const double all = __shfl_sync(0xffffffffu, line, 31);
      const double place = u * all;
      const uint32_t behind = __ballot_sync(0xffffffffu, held > 0.0 && line > place), heavy = __ballot_sync(0xffffffffu, held > 0.0);
      const uint32_t owner = behind ? __ffs(behind) - 1 : 31 - __clz(heavy | 1);
      const double base = __shfl_sync(0xffffffffu, line - held, owner);
      const bool any = all > 0.0 && all < INFINITY;
      if (!any && round == 0 && rejected) {
        w.use_q = false, w.without = kNoToken;
        __syncthreads();  // segments are written again
        continue;
      }
      if (!any) {
        if (rank == 0 && tid == 0) tokens[k] = -1;
      } else if (owner == rank && warp == 0) {
        // the stretch: lanes have runs of them
        const uint32_t count = s1 - s0, run = (count + 31) / 32, r0 = min(lane * run, count), r1 = min(r0 + run, count);
        double sum = 0.0;
        for (uint32_t s = r0; s < r1; ++s) sum += segments[s];
        double before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double x = __shfl_up_sync(0xffffffffu, before, o);
          if (int(lane) >= o) before += x;
        }
        before = base + (before - sum);
        // the first stretch whose end lies behind the place, else the last with weight
        uint32_t found = 0xffffffffu, last = 0xffffffffu;
        double found_base = 0.0, last_base = 0.0;
        for (uint32_t s = r0; s < r1; ++s) {
          if (segments[s] > 0.0) {
            last = s, last_base = before;
            if (found == 0xffffffffu && before + segments[s] > place) found = s, found_base = before;
          }
          before += segments[s];
        }
        uint32_t who = __ballot_sync(0xffffffffu, found != 0xffffffffu);
        uint32_t from;
        if (who) {
          from = __ffs(who) - 1;
        } else {
          from = 31 - __clz(__ballot_sync(0xffffffffu, last != 0xffffffffu));
          found = last, found_base = last_base;
        }
        const uint32_t stretch = __shfl_sync(0xffffffffu, found, from);
        const double start = __shfl_sync(0xffffffffu, found_base, from);
        float x[8];
        const uint32_t v = (s0 + stretch) * (kSegment / 8) + lane;
        const int32_t e = w.p.first(v);
        Raw<T, 8> xp[1], xq[1];
        w.read(v, 0, xp, xq);
        w.weigh(e, xp[0], xq[0], x);
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i];
        before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double y = __shfl_up_sync(0xffffffffu, before, o);
          if (int(lane) >= o) before += y;
        }
        double at = start + (before - sum);
        int32_t hit = -1, end = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          at += x[i];
          if (x[i] > 0.f) {
            end = e + i;
            if (hit < 0 && at > place) hit = e + i;
          }
        }
        who = __ballot_sync(0xffffffffu, hit >= 0);
        if (who) {
          if (lane == __ffs(who) - 1) tokens[k] = hit;
        } else {
          who = __ballot_sync(0xffffffffu, end >= 0);
          if (lane == 31 - __clz(who)) tokens[k] = end;
        }
      }
      break;
    }
  }
  cluster.sync();  // the others' shared memory has been read
}

template <typename T, bool PROB>
cudaError_t launch(const VerifyArgs& a, uint32_t n_seqs, uint32_t ctas, uint32_t smem, cudaStream_t stream) {
  void (*const kernel)(VerifyArgs) = bcp_verify_kernel<T, PROB>;
  cudaError_t e = cudaSuccess;
  if (ctas > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attributes[2];
  attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attributes[0].val.programmaticStreamSerializationAllowed = 1;
  attributes[1].id = cudaLaunchAttributeClusterDimension;
  attributes[1].val.clusterDim.x = ctas, attributes[1].val.clusterDim.y = 1, attributes[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(n_seqs * ctas), config.blockDim = dim3(kThreads), config.dynamicSmemBytes = smem, config.stream = stream;
  config.attrs = attributes, config.numAttrs = 2;
  return cudaLaunchKernelEx(&config, kernel, a);
}
template <typename T>
cudaError_t launch(const VerifyArgs& a, bool prob, uint32_t n_seqs, uint32_t ctas, uint32_t smem, cudaStream_t stream) {
  return prob ? launch<T, true>(a, n_seqs, ctas, smem, stream) : launch<T, false>(a, n_seqs, ctas, smem, stream);
}

struct Span {
  const void* at;
  uint64_t bytes;
  bool meets(const Span& o) const {
    const uintptr_t x = reinterpret_cast<uintptr_t>(at), y = reinterpret_cast<uintptr_t>(o.at);
    return bytes && o.bytes && x < y + o.bytes && y < x + bytes;
  }
};

int check_rows(const char* call, const char* name, const bcp_vocab_rows* r) {
  if (!r) return fail(BCP_ERR_INVALID, "%s: %s is NULL", call, name);
  if (r->type != BCP_F32 && r->type != BCP_BF16 && r->type != BCP_F16)
    return fail(BCP_ERR_INVALID, "%s: %s has type %u (binary32, bfloat16 or binary16 expected)", call, name, r->type);
  if (!r->data || (reinterpret_cast<uintptr_t>(r->data) & (type_size(r->type) - 1)))
    return fail(BCP_ERR_INVALID, "%s: %s has no data, or is not aligned to its elements", call, name);
  const int64_t most = int64_t(1) << 40;
  if (r->seq_stride < 0 || r->row_stride < 0 || r->seq_stride > most || r->row_stride > most)
    return fail(BCP_ERR_INVALID, "%s: %s has a stride that is negative or past 2^40", call, name);
  if (r->reserved) return fail(BCP_ERR_INVALID, "%s: reserved field of %s is not 0", call, name);
  return BCP_OK;
}

}  // namespace

extern "C" int bcp_verify_drafts(const bcp_vocab_rows* target, const bcp_vocab_rows* draft, uint32_t n_seqs, uint32_t n_drafts, uint32_t vocab,
                                 const int64_t* drafts, const float* uniform, const float* temperature, int probabilities, int64_t* tokens,
                                 int32_t* accepted, void* stream) {
  const char* call = "bcp_verify_drafts";
  if (n_seqs > (1u << 24)) return fail(BCP_ERR_INVALID, "%s: %u sequences", call, n_seqs);
  if (n_drafts > BCP_MAX_DRAFTS) return fail(BCP_ERR_INVALID, "%s: %u drafts a sequence; at most %u", call, n_drafts, BCP_MAX_DRAFTS);
  if (!vocab || vocab > BCP_MAX_VOCAB) return fail(BCP_ERR_INVALID, "%s: a vocabulary of %u; 1 to %u expected", call, vocab, BCP_MAX_VOCAB);
  if (probabilities && temperature) return fail(BCP_ERR_INVALID, "%s: probabilities have no temperature", call);
  if (n_seqs == 0) return BCP_OK;
  if (int rc = check_rows(call, "target", target)) return rc;
  if (draft && n_drafts) {
    if (int rc = check_rows(call, "draft", draft)) return rc;
    if (draft->type != target->type) return fail(BCP_ERR_MISMATCH, "%s: target and draft have different types", call);
  }
  if ((n_drafts && !drafts) || !uniform || !tokens || !accepted) return fail(BCP_ERR_INVALID, "%s: drafts, uniform, tokens or accepted is NULL", call);

  // one CTA writes while others of its cluster, and other sequences', may still read
  const uint64_t places = uint64_t(n_seqs) * (n_drafts + 1);
  const Span in[] = {{drafts, (places - n_seqs) * sizeof *drafts}, {uniform, places * sizeof *uniform}, {temperature, temperature ? n_seqs * sizeof *temperature : 0}};
  const Span out[] = {{tokens, places * sizeof *tokens}, {accepted, n_seqs * sizeof *accepted}};
  for (const Span& o : out)
    for (const Span& i : in)
      if (o.meets(i)) return fail(BCP_ERR_DST_ALIAS, "%s: tokens or accepted overlap drafts, uniform or temperature", call);
  if (out[0].meets(out[1])) return fail(BCP_ERR_DST_ALIAS, "%s: tokens and accepted overlap", call);

  VerifyArgs a = {};
  a.target = target->data, a.t_seq = target->seq_stride, a.t_row = target->row_stride;
  a.certain = !draft || !n_drafts;
  if (!a.certain) a.draft = draft->data, a.d_seq = draft->seq_stride, a.d_row = draft->row_stride;
  a.vocab = vocab, a.n_drafts = n_drafts;
  a.drafts = drafts, a.uniform = uniform, a.temperature = temperature;
  a.tokens = tokens, a.accepted = accepted;
  int sms = 0, device = 0;
  BCP_CUDA(cudaGetDevice(&device));
  BCP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  // CTAs of a sequence: as long as the GPU has room for four of them an SM, and each has 2048 tokens, or 4096 of probabilities, which are read once; of a huge
  // vocabulary a CTA has at most 2^19 tokens, whose sums fit its shared memory.  Microseconds with room for two / four / eight: 64 sequences of 4 drafts over
  // 128,256 tokens 82 / 57.5 / 71, 200 rows of 50,304 sampled 28.5 / 21.9 / 25.1, 30 rows of 128,256 16.0 / 13.5 / 13.7; with 2048 and 4096 tokens: 37
  // rows of 50,257 probabilities 11.0 / 7.1, one sequence of 4 drafts over 32,768 16.5 / 17.1.
  const uint32_t least = probabilities ? 4096 : 2048;
  uint32_t ctas = 16;
  while (ctas > 1 && (uint64_t(n_seqs) * ctas > uint64_t(sms) * 4 || vocab / ctas < least) && vocab / ctas < (1u << 18)) ctas /= 2;
  const uint32_t rows = 2 * n_drafts + 1, segments = (vocab + 7) / kSegment + 2;
  const uint32_t smem = uint32_t(sizeof(RowSum)) * rows * (kParts + 2) + 8 * (2 + (n_drafts + 2) / 2 + (segments + ctas - 1) / ctas);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (target->type == BCP_F32) BCP_CUDA(launch<float>(a, probabilities != 0, n_seqs, ctas, smem, st));
  if (target->type == BCP_BF16) BCP_CUDA(launch<__nv_bfloat16>(a, probabilities != 0, n_seqs, ctas, smem, st));
  if (target->type == BCP_F16) BCP_CUDA(launch<__half>(a, probabilities != 0, n_seqs, ctas, smem, st));
  return BCP_OK;
}

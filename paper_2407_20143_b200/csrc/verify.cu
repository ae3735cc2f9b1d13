// Drafted tokens verified against the target's probabilities, and the next token drawn.
//
// Mathematics.  Draft i of a sequence is accepted iff u_i q_i(x_i) < p_i(x_i); at the first one that is not, the next token is drawn from
// max(p_i - q_i, 0), else from the row behind the last draft: the lowest index whose cumulative weight exceeds u times the sum of
// all weights.  Rows of logits stand for p(j) = exp((z_j - m) / T) / S, so each is read once for m and S (a running maximum, the sum
// brought to a new one where it grows) before the first draft can be judged.
//
// What bounds it: reading the rows for few drafts or many sequences, latency for a single sequence.  A cluster of CTAs takes a
// sequence, each CTA a stretch of the vocabulary in all rows; maxima and sums are exchanged through the cluster's shared memory, every CTA
// judges all drafts itself, and the weights of the one row that is drawn from (two with drafts' rows; still in the L2 cache) are
// summed by stretches of 256 tokens.  The CTA in whose stretch the drawn place lies goes over those 256 again.  One launch, no
// workspace, no atomics: the same bits on every run.
//
// Precision: a token hangs on a comparison, so sums are held in 64 bits and the probability of a drafted token is computed in 64 bits
// from its logit; the terms of the sums are binary32 (2^-22 of each).
#include <cooperative_groups.h>

#include "decode.cuh"

using namespace bcp;
namespace cg = cooperative_groups;

namespace {

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kSegment = 256;  // tokens of a stretch that is summed for the draw: eight a lane
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

// What is known of a row, or a part of it: the largest value and the sum of exp2((z - m) c); greedy: the index of the largest.
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
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ RowSum join(const RowSum& a, const RowSum& b, float c) {
  RowSum r;
  r.m = fmaxf(a.m, b.m);
  const float ref = reference(r.m);
  r.s = a.s * exp2_fast((a.m - ref) * c) + b.s * exp2_fast((b.m - ref) * c);
  r.index = a.m > b.m || (a.m == b.m && a.index < b.index) ? a.index : b.index;
  return r;
}

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
  // Eight elements from e on, `none` where the row has none; aligned: e is a unit's first.
  __device__ __forceinline__ void load(int32_t e, bool aligned, float none, float (&x)[8]) const {
    if (aligned && e >= 0 && uint32_t(e) + 8 <= n) {
      Raw<T, 8> r;
      r.load(p + e);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_f32(r.get(i));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = e + i >= 0 && uint32_t(e + i) < n ? to_f32(p[e + i]) : none;
    }
  }
};

// The part of a row that this thread sees: units first, first + kThreads, .. below end.
template <typename T>
__device__ __forceinline__ RowSum look_over(const Row<T>& row, uint32_t first, uint32_t end, float c, bool greedy) {
  RowSum r = {-INFINITY, 0xffffffffu, 0.0};
  constexpr int kAhead = 4;
  for (uint32_t v0 = first; v0 < end; v0 += kAhead * kThreads) {
    float x[kAhead][8];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const uint32_t v = v0 + j * kThreads;
      if (v < end) {
        row.load(row.first(v), true, -INFINITY, x[j]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = -INFINITY;
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      float top = x[j][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[j][i]);
      if (greedy) {
        if (top > r.m) {
          r.m = top;
#pragma unroll
          for (int i = 7; i >= 0; --i)
            if (x[j][i] == top) r.index = uint32_t(row.first(v0 + j * kThreads) + i);
        }
        continue;
      }
      if (top > r.m) r.s *= exp2_fast((r.m - top) * c), r.m = top;
      const float ref = reference(r.m);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += exp2_fast((x[j][i] - ref) * c);
      r.s += s;
    }
  }
  return r;
}

// What turns an element into a probability.
struct Scale {
  float m, c, inverse;
};

template <typename T, bool PROB>
struct Weights {  // of the row that is drawn from
  Row<T> p, q;
  Scale ps, qs;
  bool use_q, same;   // subtract q's; its units begin where p's do
  int64_t without;    // a token that counts nothing
  __device__ __forceinline__ static float probability(float z, const Scale& s) {
    return PROB ? z : exp2_fast((z - s.m) * s.c) * s.inverse;
  }
  __device__ __forceinline__ void load(int32_t e, float (&w)[8]) const {
    p.load(e, true, PROB ? 0.f : -INFINITY, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = probability(w[i], ps);
    if (use_q) {
      float y[8];
      q.load(e, same, PROB ? 0.f : -INFINITY, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = fmaxf(w[i] - probability(y[i], qs), 0.f);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (w[i] < 0.f || e + i == without || e + i < 0 || uint32_t(e + i) >= p.n) w[i] = 0.f;
  }
};

template <typename T, bool PROB>
__global__ void __launch_bounds__(kThreads, 4) bcp_verify_kernel(const VerifyArgs a) {
  after_previous();
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const uint32_t b = blockIdx.x / ctas, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t most_rows = 2 * a.n_drafts + 1;
  extern __shared__ __align__(16) unsigned char smem[];
  RowSum* const by_warp = reinterpret_cast<RowSum*>(smem);       // [rows][warps]
  RowSum* const mine = by_warp + most_rows * kWarps;             // [rows]: of this CTA's part, read by the others
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
  // drafts of this sequence: up to the first negative one
  if (tid <= a.n_drafts) good[tid] = tid < a.n_drafts && drafts[tid] >= 0;
  __syncthreads();
  uint32_t n = 0;
  while (n < a.n_drafts && good[n]) ++n;
  __syncthreads();

  auto target = [&](uint32_t i) { return Row<T>(a.target, b * a.t_seq + i * a.t_row, a.vocab); };
  auto draft = [&](uint32_t i) { return Row<T>(a.draft, b * a.d_seq + i * a.d_row, a.vocab); };

  // ---- maxima and sums of all rows: the target's 0 .. n, then the drafts'
  const uint32_t n_rows = n + 1 + (a.certain || greedy ? 0 : n);
  if (!PROB) {
    for (uint32_t i = 0; i < n_rows; ++i) {
      const Row<T> row = i <= n ? target(i) : draft(i - n - 1);
      const uint32_t each = (row.units + ctas - 1) / ctas, begin = rank * each;
      RowSum r = look_over(row, begin + tid, min(begin + each, row.units), c, greedy);
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        RowSum other;
        other.m = __shfl_xor_sync(0xffffffffu, r.m, o);
        other.index = __shfl_xor_sync(0xffffffffu, r.index, o);
        other.s = __shfl_xor_sync(0xffffffffu, r.s, o);
        r = join(r, other, c);
      }
      if (lane == 0) by_warp[i * kWarps + warp] = r;
    }
    __syncthreads();
    for (uint32_t i = tid; i < n_rows; i += kThreads) {
      RowSum r = by_warp[i * kWarps];
      for (uint32_t w = 1; w < kWarps; ++w) r = join(r, by_warp[i * kWarps + w], c);
      mine[i] = r;
    }
    cluster.sync();
    for (uint32_t i = tid; i < n_rows; i += kThreads) {
      RowSum r = cluster.map_shared_rank(mine, 0)[i];
      for (uint32_t w = 1; w < ctas; ++w) r = join(r, cluster.map_shared_rank(mine, w)[i], c);
      whole[i] = r;
    }
    __syncthreads();
  }

  // ---- every draft is judged by a thread; the same in all CTAs
  const double nan = __longlong_as_double(0x7ff8000000000000ll);
  auto probability = [&](const Row<T>& row, uint32_t i, int64_t x) -> double {  // of token x in row i
    const float z = to_f32(row.p[x]);
    if (PROB) return z;
    const double s = whole[i].s;
    return s > 0 && s < INFINITY ? exp((double(z) - double(whole[i].m)) / double(t)) / s : nan;
  };
  if (tid < n) {
    const int64_t x = drafts[tid];
    bool ok = x < int64_t(a.vocab);
    if (ok && greedy) {
      ok = whole[tid].index == uint32_t(x);
    } else if (ok) {
      const double p = probability(target(tid), tid, x), q = a.certain ? 1.0 : probability(draft(tid), n + 1 + tid, x);
      ok = double(uniform[tid]) * q < p;
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
    Weights<T, PROB> w = {target(k), target(k), scale(k), scale(k), rejected && !a.certain, false, rejected && a.certain ? drafts[k] : -1};
    if (w.use_q) {
      w.q = draft(k), w.qs = scale(n + 1 + k);
      w.same = w.q.shift == w.p.shift;
    }
    // parts of whole stretches
    const uint32_t n_segments = (w.p.units + kSegment / 8 - 1) / (kSegment / 8), each = (n_segments + ctas - 1) / ctas;
    const uint32_t s0 = min(rank * each, n_segments), s1 = min(s0 + each, n_segments);
    const double u = uniform[a.n_drafts];
    // what is left after q may be nothing at all (p and q alike, a draft outside its own row): then p itself counts
    for (int round = 0;; ++round) {
      for (uint32_t s = s0 + warp; s < s1; s += kWarps) {
        float x[8];
        w.load(w.p.first(s * (kSegment / 8) + lane), x);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i];
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) segments[s - s0] = sum;
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
      // the CTA that holds the place; if rounding has left none, the last that has any weight
      double all = 0.0, base = 0.0;
      for (uint32_t r = 0; r < ctas; ++r) all += cluster.map_shared_rank(total, r)[round];
      const double place = u * all;
      uint32_t owner = 0xffffffffu;
      double line = 0.0;
      for (uint32_t r = 0; r < ctas; ++r) {
        const double next = line + cluster.map_shared_rank(total, r)[round];
        if (next > line) {
          owner = r, base = line;
          if (next > place) break;
        }
        line = next;
      }
      const bool any = all > 0.0 && all < INFINITY;
      if (!any && round == 0 && rejected) {
        w.use_q = false, w.without = -1;
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
        const int32_t e = w.p.first((s0 + stretch) * (kSegment / 8) + lane);
        w.load(e, x);
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
  // CTAs of a sequence: as long as the GPU has room for four of them an SM, and each has 2048 tokens; of a huge vocabulary a CTA has at
  // most 2^19 tokens, whose sums fit its shared memory.
  uint32_t ctas = 16;
  while (ctas > 1 && (uint64_t(n_seqs) * ctas > uint64_t(sms) * 4 || vocab / ctas < 2048) && vocab / ctas < (1u << 18)) ctas /= 2;
  const uint32_t rows = 2 * n_drafts + 1, segments = (vocab + 7) / kSegment + 2;
  const uint32_t smem = uint32_t(sizeof(RowSum)) * rows * (kWarps + 2) + 8 * (2 + (n_drafts + 2) / 2 + (segments + ctas - 1) / ctas);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (target->type == BCP_F32) BCP_CUDA(launch<float>(a, probabilities != 0, n_seqs, ctas, smem, st));
  if (target->type == BCP_BF16) BCP_CUDA(launch<__nv_bfloat16>(a, probabilities != 0, n_seqs, ctas, smem, st));
  if (target->type == BCP_F16) BCP_CUDA(launch<__half>(a, probabilities != 0, n_seqs, ctas, smem, st));
  return BCP_OK;
}

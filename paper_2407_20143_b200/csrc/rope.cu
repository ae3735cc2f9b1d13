// Rotary positions: every pair of a head vector is turned by the angle of its token's position.
//
// The arithmetic is six operations per pair, so the kernel is bound by memory: each element is read
// once and written once.  A thread takes one chunk (two 16-byte vectors) of four heads of one token: the cosines
// and sines, which all heads of a token share, are loaded once per four heads, and eight 16-byte loads
// are in flight per thread (16-bit types).  Query and key heads go through one launch.
// Measured on one B200 (copy bandwidth 6533 GB/s): 16,384 tokens of 32 + 8 heads of 128, bfloat16: 51.7 us for 342 MB, 1.01 of it (a
// part of the output is still in the L2 cache when the launch ends); the gradient of 8191 tokens of 16 + 16 heads, binary32,
// half of each rotated: 41.1 us for 270 MB, 1.0; 16 tokens: 1.6 us.
// The scalar form, for rotated parts that are no multiple of 16 and for rows off the 16-byte boundaries, is bound by its
// element-wise accesses: 16,384 tokens of 32 + 8 heads of 80, 20 of them rotated, bfloat16 285 us for 211 MB (32 rotated,
// vector form: 36 us); 8192 tokens in binary32 124 us (16 rotated, vector form: 33 us).
#include "decode.cuh"

using namespace bcp;

namespace bcp {

int check_heads(const char* call, const char* name, const bcp_heads* h, bool written, uint32_t head_dim, int64_t n_tokens) {
  if (!h) return fail(BCP_ERR_INVALID, "%s: %s is NULL", call, name);
  if (h->type != BCP_F32 && h->type != BCP_BF16 && h->type != BCP_F16)
    return fail(BCP_ERR_INVALID, "%s: %s has type %u (binary32, bfloat16 or binary16 expected)", call, name, h->type);
  if (!h->n_heads || h->n_heads > 65536) return fail(BCP_ERR_INVALID, "%s: %s has %u heads", call, name, h->n_heads);
  if (h->token_stride < 0 || h->head_stride < 0 || h->token_stride > 0xffffffffll || h->head_stride > 0xffffffffll)
    return fail(BCP_ERR_INVALID, "%s: %s has a stride that is negative or past 2^32", call, name);
  if (n_tokens && !h->data) return fail(BCP_ERR_INVALID, "%s: %s has no data", call, name);
  if (reinterpret_cast<uintptr_t>(h->data) & (type_size(h->type) - 1)) return fail(BCP_ERR_INVALID, "%s: %s is not aligned to its elements", call, name);
  if (written) {  // the rows of an output must not share memory
    const int64_t strides[2] = {h->token_stride, h->head_stride};
    const uint32_t extents[2] = {uint32_t(n_tokens), h->n_heads};
    if (rows_overlap(strides, extents, 2, head_dim))
      return fail(BCP_ERR_DST_ALIAS, "%s: rows of %s overlap (strides %lld, %lld for vectors of %u)", call, name, (long long)h->token_stride,
                  (long long)h->head_stride, head_dim);
  }
  return BCP_OK;
}

int check_rope(const char* call, const bcp_rope_table* r, uint32_t head_dim) {
  if (!r->table || (reinterpret_cast<uintptr_t>(r->table) & 15)) return fail(BCP_ERR_INVALID, "%s: the table is NULL or not 16-byte aligned", call);
  if (r->n_positions < 1 || r->n_positions > 0x7fffffff) return fail(BCP_ERR_INVALID, "%s: a table of %lld positions", call, (long long)r->n_positions);
  if (r->rot_dim < 2 || (r->rot_dim & 1) || r->rot_dim > head_dim)
    return fail(BCP_ERR_INVALID, "%s: rot_dim %u is not an even number from 2 to head_dim %u", call, r->rot_dim, head_dim);
  if (r->layout > BCP_ROPE_PAIRS) return fail(BCP_ERR_INVALID, "%s: layout %u", call, r->layout);
  return BCP_OK;
}

}  // namespace bcp

namespace {

// Heads per thread: four share the loads of the table and keep eight 16-byte loads in flight, which a long
// input needs (16k tokens of 40 heads: 52 us, 56 with two); where that leaves SMs without work, one.  Microseconds with one
// and with four, by threads an SM if each had one head: 540 (250 tokens of 40 heads, bf16) 2.5 / 2.6, 860 (400) 2.8 / 3.3, 1300 (600)
// 3.7 / 4.3, 1500 (700) 4.8 / 4.4, 1700 (500 tokens of 32 heads, f32) 4.4 / 4.7, 2160 (1000 tokens of 40 heads) 5.9 / 5.5,
// 4300 (2000) 9.8 / 8.7.  The scalar form takes one head always: four spill (16,384 tokens of 40 heads of 80, 20 rotated, bf16 285 / 328,
// 8192 of them in f32 124 / 164, 1000 in bf16 22 / 39).
constexpr uint32_t kManyHeads = 4, kFewThreads = 2048;  // per SM, with a thread for every head

struct RopeArgs {
  const void* in[2];
  void* out[2];
  uint32_t in_token[2], in_head[2], out_token[2], out_head[2];
  uint32_t n_heads[2], q_groups;  // groups of heads: first those of q, then k's
  uint32_t head_dim, rot_dim;
  float sign;
  FastDiv per_token, per_group;  // threads per token; per group
  uint32_t n_threads;
  const float* table;
  int64_t n_positions;
  const int64_t* positions;
  uint32_t* status;
};

template <typename T, bool VEC, bool PAIRS, int HEADS>
__global__ void __launch_bounds__(256, 3) bcp_rope_kernel(const RopeArgs a) {
  after_previous();
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= a.n_threads) return;
  const uint32_t t = a.per_token.div(i), r = i - t * a.per_token.d;
  const uint32_t g = a.per_group.div(r);
  constexpr int V = kChunk<T, VEC>;
  const Chunk k = chunk_at<V, VEC, PAIRS>(r - g * a.per_group.d, a.head_dim, a.rot_dim);
  const int64_t position = a.positions[t];
  const bool there = position >= 0 && position < a.n_positions;
  if (position >= a.n_positions) raise(a.status, BCP_BAD_POSITION);

  const int side = g >= a.q_groups;
  const uint32_t h0 = (side ? g - a.q_groups : g) * HEADS, n = min(a.n_heads[side] - h0, uint32_t(HEADS));
  const T* from = static_cast<const T*>(a.in[side]) + (uint64_t(t) * a.in_token[side] + uint64_t(h0) * a.in_head[side]);
  T* to = static_cast<T*>(a.out[side]) + (uint64_t(t) * a.out_token[side] + uint64_t(h0) * a.out_head[side]);
  Elements<T, VEC> e[HEADS];
#pragma unroll
  for (int j = 0; j < HEADS; ++j, from += a.in_head[side])
    if (j < n) e[j].load(from, k);
  Angles<V, VEC, PAIRS> w;
  if (k.rotated) w.load(a.table, there ? position : 0, a.rot_dim, k, a.sign);
#pragma unroll
  for (int j = 0; j < HEADS; ++j, to += a.out_head[side]) {
    if (j >= n) break;
    if (k.rotated || !there) {
      float x[V], y[V];
      e[j].unpack(x, y);
      if (k.rotated) w.rotate(x, y);
      if (!there) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = y[i] = 0.f;
      }
      e[j].pack(x, y);
    }
    e[j].store(to, k);
  }
}

__global__ void bcp_clear_kernel(uint32_t* status, uint32_t bits) { atomicAnd(status, ~bits); }

template <typename T, bool VEC, bool PAIRS>
cudaError_t launch(const RopeArgs& a, uint32_t heads, cudaStream_t stream) {
  void (*kernel)(RopeArgs) = bcp_rope_kernel<T, VEC, PAIRS, 1>;
  if constexpr (VEC) {
    if (heads != 1) kernel = bcp_rope_kernel<T, VEC, PAIRS, kManyHeads>;
  }
  return launch_early(kernel, (a.n_threads + 255) / 256, 256, 0, stream, a);
}
template <typename T>
cudaError_t launch(const RopeArgs& a, bool vec, bool pairs, uint32_t heads, cudaStream_t stream) {
  if (vec) return pairs ? launch<T, true, true>(a, heads, stream) : launch<T, true, false>(a, heads, stream);
  return pairs ? launch<T, false, true>(a, heads, stream) : launch<T, false, false>(a, heads, stream);
}

}  // namespace

extern "C" int bcp_rope(const bcp_heads* q_in, const bcp_heads* q_out, const bcp_heads* k_in, const bcp_heads* k_out, uint32_t head_dim,
                        int64_t n_tokens, const bcp_rope_table* rope, const int64_t* positions, int transpose, void* stream) {
  const char* call = "bcp_rope";
  if (!rope) return fail(BCP_ERR_INVALID, "%s: rope is NULL", call);
  if (head_dim < 2 || head_dim > BCP_MAX_HEAD_DIM) return fail(BCP_ERR_INVALID, "%s: head_dim %u is not in 2..%u", call, head_dim, BCP_MAX_HEAD_DIM);
  if (n_tokens < 0 || n_tokens > 0x7fffffff) return fail(BCP_ERR_INVALID, "%s: %lld tokens", call, (long long)n_tokens);
  if (int rc = check_rope(call, rope, head_dim)) return rc;
  if (int rc = check_heads(call, "q_in", q_in, false, head_dim, n_tokens)) return rc;
  if (int rc = check_heads(call, "q_out", q_out, true, head_dim, n_tokens)) return rc;
  if (!k_in != !k_out) return fail(BCP_ERR_INVALID, "%s: k_in and k_out go together", call);
  if (k_in) {
    if (int rc = check_heads(call, "k_in", k_in, false, head_dim, n_tokens)) return rc;
    if (int rc = check_heads(call, "k_out", k_out, true, head_dim, n_tokens)) return rc;
  }
  const bcp_heads* in[2] = {q_in, k_in ? k_in : q_in};
  const bcp_heads* out[2] = {q_out, k_in ? k_out : q_out};
  for (int s = 0; s < 2; ++s) {
    if (in[s]->type != q_in->type || out[s]->type != q_in->type) return fail(BCP_ERR_MISMATCH, "%s: all vectors must have one type", call);
    if (in[s]->n_heads != out[s]->n_heads) return fail(BCP_ERR_MISMATCH, "%s: %u heads in, %u out", call, in[s]->n_heads, out[s]->n_heads);
  }
  if (n_tokens && !positions) return fail(BCP_ERR_INVALID, "%s: positions is NULL", call);

  RopeArgs a = {};
  bool vec = head_dim % 16 == 0 && rope->rot_dim % 16 == 0;
  for (int s = 0; s < 2; ++s) {
    a.in_token[s] = uint32_t(in[s]->token_stride), a.in_head[s] = uint32_t(in[s]->head_stride);
    a.out_token[s] = uint32_t(out[s]->token_stride), a.out_head[s] = uint32_t(out[s]->head_stride);
    vec = vec && rows_aligned(in[s], 16) && rows_aligned(out[s], 16);
  }
  a.n_heads[0] = q_in->n_heads, a.n_heads[1] = k_in ? k_in->n_heads : 0;
  a.head_dim = head_dim, a.rot_dim = rope->rot_dim;
  a.sign = transpose ? -1.f : 1.f;
  a.table = rope->table, a.n_positions = rope->n_positions, a.status = rope->status;
  int sms = 0, device = 0;
  BCP_CUDA(cudaGetDevice(&device));
  BCP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  const uint32_t es = type_size(q_in->type), chunks = chunks_of(head_dim, rope->rot_dim, vec ? 16 / es : 8);
  const uint64_t all_heads = uint64_t(a.n_heads[0]) + a.n_heads[1];
  const uint32_t heads = !vec || uint64_t(n_tokens) * all_heads * chunks < uint64_t(sms) * kFewThreads ? 1 : kManyHeads;
  a.q_groups = (a.n_heads[0] + heads - 1) / heads;
  const uint32_t per_token = chunks * (a.q_groups + (a.n_heads[1] + heads - 1) / heads);
  a.per_group = FastDiv(chunks), a.per_token = FastDiv(per_token);
  // thread indices stay below 2^31: longer inputs take several launches
  const int64_t most = 0x7fffff00 / per_token;
  for (int64_t t0 = 0; t0 < n_tokens; t0 += most) {
    const int64_t n = n_tokens - t0 < most ? n_tokens - t0 : most;
    a.n_threads = uint32_t(n) * per_token;
    a.positions = positions + t0;
    for (int s = 0; s < 2; ++s) {
      a.in[s] = static_cast<const char*>(in[s]->data) + t0 * in[s]->token_stride * es;
      a.out[s] = static_cast<char*>(out[s]->data) + t0 * out[s]->token_stride * es;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool pairs = rope->layout == BCP_ROPE_PAIRS;
    if (q_in->type == BCP_F32) BCP_CUDA(launch<float>(a, vec, pairs, heads, st));
    if (q_in->type == BCP_BF16) BCP_CUDA(launch<__nv_bfloat16>(a, vec, pairs, heads, st));
    if (q_in->type == BCP_F16) BCP_CUDA(launch<__half>(a, vec, pairs, heads, st));
  }
  return BCP_OK;
}

extern "C" int bcp_decode_status(uint32_t* status, void* stream_) {
  if (!status) return fail(BCP_ERR_INVALID, "bcp_decode_status: status is NULL");
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  uint32_t bits = 0;
  cudaError_t e = cudaMemcpyAsync(&bits, status, sizeof bits, cudaMemcpyDeviceToHost, stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  if (e == cudaSuccess && bits) {  // only what was read: another stream may have set more since
    bcp_clear_kernel<<<1, 1, 0, stream>>>(status, bits);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess) return fail(BCP_ERR_CUDA, "bcp_decode_status: %s", cudaGetErrorString(e));
  if (!bits) return BCP_OK;
  return fail(BCP_ERR_BOUNDS, "an index was outside its range and was left out:%s%s%s%s", bits & BCP_BAD_POSITION ? " position" : "",
              bits & BCP_BAD_SLOT ? " slot" : "", bits & BCP_BAD_PAGE ? " page" : "", bits & BCP_BAD_LENGTH ? " length" : "");
}

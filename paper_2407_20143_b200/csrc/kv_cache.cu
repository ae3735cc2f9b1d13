// The paged key-value cache: new tokens written into their slots, slots read back.
//
// Both are bound by memory: a head vector is read once and written once.  A group of lanes (a power of
// two) holds one head vector, a chunk a lane, so the largest magnitude that an 8-bit format's scale needs is a
// few shuffles away and the vector is never read twice.  A group takes two heads of one token, whose loads
// are all in flight before the first one is used.
// Measured on one B200 (copy bandwidth 6533 GB/s): 65,536 tokens of 8 heads of 128 read back, one in 17 slots empty, e4m3 to
// bfloat16: 62.4 us, 399 MB, 0.98 of it.  32,768 tokens written with rotation, one in 17 skipped, bfloat16 to e4m3: 47.6 us for the 202 MB
// that live tokens need, 0.65 of it (skipped tokens' vectors are read too: nothing waits for the slot), to int8 52 us, to a bfloat16
// cache 47 us (0.86 for its 263 MB); neighbouring pairs 48.5.  It waits: half of the issue slots are used and DRAM is 46 % busy; a
// group of lanes lives for one token, loads its position, then the row of the table, and has nothing else in flight meanwhile.  Four
// CTAs an SM allow 64 registers (half layout without spills, neighbouring pairs with 44 bytes; three CTAs: 56 us; four heads a
// group, 128 registers: 66 us).
#include "decode.cuh"

using namespace bcp;

namespace bcp {

bool rows_overlap(const int64_t* strides, const uint32_t* extents, int n, uint32_t row) {
  int64_t reach = row;  // elements that the dimensions so far span
  bool used[3] = {false, false, false};
  for (int i = 0; i < n; ++i) {
    int next = -1;
    for (int j = 0; j < n; ++j)
      if (!used[j] && (next < 0 || strides[j] < strides[next])) next = j;
    used[next] = true;
    if (extents[next] <= 1) continue;
    if (strides[next] < reach || strides[next] > (int64_t(1) << 60) / extents[next]) return true;
    reach += strides[next] * (extents[next] - 1);
  }
  return false;
}

int check_cache(const char* call, const bcp_kv_cache* c) {
  if (!c) return fail(BCP_ERR_INVALID, "%s: cache is NULL", call);
  if (c->format != BCP_BF16 && c->format != BCP_F16 && !is_8bit(c->format)) return fail(BCP_ERR_INVALID, "%s: cache format %u", call, c->format);
  if (c->reserved) return fail(BCP_ERR_INVALID, "%s: cache.reserved must be 0", call);
  if (!c->head_dim || c->head_dim % 16 || c->head_dim > BCP_MAX_HEAD_DIM)
    return fail(BCP_ERR_INVALID, "%s: head_dim %u is not a multiple of 16 up to %u", call, c->head_dim, BCP_MAX_HEAD_DIM);
  if (!c->n_heads || c->n_heads > 65536) return fail(BCP_ERR_INVALID, "%s: a cache of %u heads", call, c->n_heads);
  if (!c->n_pages || !c->page_size || uint64_t(c->n_pages) * c->page_size > 0x7fffffffull)
    return fail(BCP_ERR_INVALID, "%s: %u pages of %u tokens (at least one token, fewer than 2^31)", call, c->n_pages, c->page_size);
  if (!c->k || !c->v) return fail(BCP_ERR_INVALID, "%s: the cache has no memory", call);
  const uint64_t es = type_size(c->format);
  const uint64_t bits = reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) | uint64_t(c->page_stride) * es |
                        uint64_t(c->head_stride) * es | uint64_t(c->token_stride) * es;
  const int64_t most = 0xffffffffll;
  if (c->page_stride <= 0 || c->head_stride <= 0 || c->token_stride <= 0 || c->page_stride > most || c->head_stride > most ||
      c->token_stride > most || (bits & 15))
    return fail(BCP_ERR_INVALID, "%s: cache addresses and strides must be positive multiples of 16 bytes, strides below 2^32 elements", call);
  if (uint64_t(c->n_pages) * c->n_heads > uint64_t(most)) return fail(BCP_ERR_INVALID, "%s: %u pages of %u heads", call, c->n_pages, c->n_heads);
  const int64_t strides[3] = {c->page_stride, c->head_stride, c->token_stride};
  const uint32_t extents[3] = {c->n_pages, c->n_heads, c->page_size};
  if (rows_overlap(strides, extents, 3, c->head_dim)) return fail(BCP_ERR_DST_ALIAS, "%s: rows of the cache overlap", call);
  if (is_8bit(c->format) != (c->k_scale != nullptr) || is_8bit(c->format) != (c->v_scale != nullptr))
    return fail(BCP_ERR_INVALID, "%s: 8-bit formats have scales, the others have none", call);
  if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & 3)
    return fail(BCP_ERR_INVALID, "%s: scales are not 4-byte aligned", call);
  return BCP_OK;
}

}  // namespace bcp

namespace {

constexpr int kHeads = 2;            // heads per group of lanes (reading 64k tokens: 63 us with two or four, 75 with one)
constexpr float kSmallestScale = 1.262177448353619e-29f;  // 2^-96: its reciprocal and sums of it stay finite

struct CacheArgs {
  void* pages[2];
  float* scales[2];
  uint32_t page_stride, head_stride, token_stride;
  uint32_t n_slots, n_heads, head_dim;
  FastDiv page_size;
  uint32_t* status;
  // the token-major side
  void* rows[2];
  uint32_t row_token[2], row_head[2];
  const int64_t* slots;
  uint32_t n_groups;      // groups of lanes
  FastDiv per_token;      // groups per token: 2 * ceil(n_heads / kHeads)
  uint32_t lanes_log2;
  // rotation of the keys while they are written
  const float* table;
  int64_t n_positions;
  const int64_t* positions;
  uint32_t rot_dim, layout;
};

template <int FMT>
struct Format;
template <>
struct Format<BCP_BF16> {
  typedef __nv_bfloat16 T;
  static constexpr bool quantised = false;
};
template <>
struct Format<BCP_F16> {
  typedef __half T;
  static constexpr bool quantised = false;
};
template <>
struct Format<BCP_E4M3> {
  typedef uint8_t T;
  static constexpr bool quantised = true;
  static constexpr float qmax = 448.f;
  // two elements, the first in the low byte
  static __device__ __forceinline__ uint32_t pack2(float x, float y) { return __nv_cvt_float2_to_fp8x2(make_float2(x, y), __NV_SATFINITE, __NV_E4M3); }
  static __device__ __forceinline__ float2 unpack2(uint32_t w) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(w), __NV_E4M3);
    return __half22float2(__half2(h));
  }
};
template <>
struct Format<BCP_I8> {
  typedef uint8_t T;
  static constexpr bool quantised = true;
  static constexpr float qmax = 127.f;
  static __device__ __forceinline__ uint32_t one(float x) { return uint32_t(__float2int_rn(fminf(fmaxf(x, -127.f), 127.f))) & 255u; }
  static __device__ __forceinline__ uint32_t pack2(float x, float y) { return one(x) | one(y) << 8; }
  static __device__ __forceinline__ float2 unpack2(uint32_t w) { return make_float2(float(int8_t(w & 255u)), float(int8_t(w >> 8 & 255u))); }
};

struct Item {
  uint32_t t, side, h0, lane;
  bool used;
};
__device__ __forceinline__ Item item_of(const CacheArgs& a) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  const uint32_t g = i >> a.lanes_log2;
  Item it;
  it.lane = i & ((1u << a.lanes_log2) - 1);
  it.used = g < a.n_groups;
  it.t = it.used ? a.per_token.div(g) : 0;
  const uint32_t r = it.used ? g - it.t * a.per_token.d : 0, half = a.per_token.d / 2;
  it.side = r >= half;
  it.h0 = (r - (it.side ? half : 0)) * kHeads;
  return it;
}

// The two halves of a chunk, multiplied by inv, in an 8-bit format.
template <int FMT, int V, bool VEC>
__device__ __forceinline__ void store_8bit(uint8_t* row, const Chunk& k, const float (&x)[V], const float (&y)[V], float inv) {
  typedef Format<FMT> F;
  uint32_t p[V / 2], q[V / 2];  // two elements each
  const float2 inv2 = make_float2(inv, inv);
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    const float2 u = mul2(make_float2(x[2 * i], x[2 * i + 1]), inv2), v = mul2(make_float2(y[2 * i], y[2 * i + 1]), inv2);
    p[i] = F::pack2(u.x, u.y), q[i] = F::pack2(v.x, v.y);
  }
  if (VEC) {
    Raw<uint8_t, V> lo, hi;
#pragma unroll
    for (int i = 0; i < V / 4; ++i) lo.w[i] = p[2 * i] | p[2 * i + 1] << 16, hi.w[i] = q[2 * i] | q[2 * i + 1] << 16;
    lo.store(row + k.lo);
    hi.store(row + k.hi);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (uint32_t(i) < k.n_lo) row[k.lo + i * k.step] = uint8_t(p[i / 2] >> (8 * (i & 1)));
      if (uint32_t(i) < k.n_hi) row[k.hi + i * k.step] = uint8_t(q[i / 2] >> (8 * (i & 1)));
    }
  }
}

// x / qmax, correctly rounded, from the rounded reciprocal and the remainder of a first quotient (Markstein's
// theorem on division).  The remainder is exact unless x is near the smallest numbers; what comes out there
// is far below the smallest scale.
template <int FMT>
__device__ __forceinline__ float quotient(float x) {
  constexpr float qmax = Format<FMT>::qmax, inverse = 1.f / qmax;
  const float q = x * inverse;
  return __fmaf_rn(__fmaf_rn(-qmax, q, x), inverse, q);
}

// The largest magnitude of three numbers, NaN if one is.
__device__ __forceinline__ float largest(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

template <typename T, int FMT, bool VEC, bool PAIRS>
__global__ void __launch_bounds__(256, 4) bcp_kv_write_kernel(const CacheArgs a) {
  after_previous();
  typedef Format<FMT> F;
  typedef typename F::T C;
  const Item it = item_of(a);
  const uint32_t rot = it.side ? 0 : a.rot_dim;
  constexpr int V = kChunk<T, VEC>;
  const bool mine = it.lane < chunks_of(a.head_dim, rot, V);
  const Chunk k = chunk_at<V, VEC, PAIRS>(mine ? it.lane : 0, a.head_dim, rot);
  // nothing waits for the slot before the stores
  Elements<T, VEC> e[kHeads];
  const T* from = static_cast<const T*>(a.rows[it.side]) + (uint64_t(it.t) * a.row_token[it.side] + uint64_t(it.h0) * a.row_head[it.side]);
#pragma unroll
  for (int j = 0; j < kHeads; ++j)
    if (it.used && mine && it.h0 + j < a.n_heads) e[j].load(from + uint64_t(j) * a.row_head[it.side], k);
  int64_t slot = it.used ? a.slots[it.t] : -1;
  if (slot >= int64_t(a.n_slots)) {
    raise(a.status, BCP_BAD_SLOT);
    slot = -1;
  }
  Angles<V, VEC, PAIRS> w;
  if (it.used && a.rot_dim) {  // both sides look at the position: a token is written whole or not at all
    int64_t position = a.positions[it.t];
    if (position < 0 || position >= a.n_positions) {
      if (slot >= 0) raise(a.status, BCP_BAD_POSITION);
      slot = -1, position = 0;
    }
    if (mine && k.rotated) w.load(a.table, position, rot, k, 1.f);
  }
  const bool live = slot >= 0 && mine;
  const uint32_t page = a.page_size.div(uint32_t(slot >= 0 ? slot : 0)), off = uint32_t(slot >= 0 ? slot : 0) - page * a.page_size.d;
  C* to = static_cast<C*>(a.pages[it.side]) + (uint64_t(page) * a.page_stride + uint64_t(it.h0) * a.head_stride + uint64_t(off) * a.token_stride);
  if constexpr (F::quantised) {
    float x[kHeads][V], y[kHeads][V], m[kHeads];
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
      m[j] = 0.f;
      if (live && it.h0 + j < a.n_heads) {
        e[j].unpack(x[j], y[j]);
        if (k.rotated) w.rotate(x[j], y[j]);
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (VEC || uint32_t(i) < k.n_lo) m[j] = largest(m[j], x[j][i], VEC || uint32_t(i) < k.n_hi ? y[j][i] : 0.f);
      }
    }
    for (uint32_t o = 1u << a.lanes_log2 >> 1; o; o >>= 1) {
#pragma unroll
      for (int j = 0; j < kHeads; ++j) m[j] = largest(m[j], __shfl_xor_sync(0xffffffffu, m[j], o), 0.f);
    }
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
      const float scale = m[j] < INFINITY ? fmaxf(quotient<FMT>(m[j]), kSmallestScale) : __uint_as_float(0x7fc00000u);
      if (live && it.h0 + j < a.n_heads) {
        store_8bit<FMT, V, VEC>(reinterpret_cast<uint8_t*>(to + uint64_t(j) * a.head_stride), k, x[j], y[j], __frcp_rn(scale));
        if (it.lane == 0) a.scales[it.side][uint64_t(page * a.n_heads + it.h0 + j) * a.page_size.d + off] = scale;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
      if (!live || it.h0 + j >= a.n_heads) continue;
      float x[V], y[V];
      e[j].unpack(x, y);
      if (k.rotated) w.rotate(x, y);
      C* const row = to + uint64_t(j) * a.head_stride;
      if constexpr (VEC) {
        Raw<C, V> lo, hi;
#pragma unroll
        for (int i = 0; i < V; ++i) lo.set(i, from_f32<C>(x[i])), hi.set(i, from_f32<C>(y[i]));
        lo.store(row + k.lo);
        hi.store(row + k.hi);
      } else {
        Elements<C, false> c;
        c.pack(x, y);
        c.store(row, k);
      }
    }
  }
}

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(256) bcp_kv_read_kernel(const CacheArgs a) {
  after_previous();
  typedef Format<FMT> F;
  typedef typename F::T C;
  constexpr int V = VEC ? 16 / int(sizeof(T)) : 8;
  const Item it = item_of(a);
  if (!it.used || it.lane * (2 * V) >= a.head_dim) return;
  int64_t slot = a.slots[it.t];
  if (slot >= int64_t(a.n_slots)) {
    raise(a.status, BCP_BAD_SLOT);
    slot = -1;
  }
  // one vector of either half of the head (whose dimension is a multiple of 16)
  const uint32_t lo = V * it.lane, hi = lo + a.head_dim / 2;
  const uint32_t page = a.page_size.div(uint32_t(slot >= 0 ? slot : 0)), off = uint32_t(slot) - page * a.page_size.d;
  const C* from = static_cast<const C*>(a.pages[it.side]) + (uint64_t(page) * a.page_stride + uint64_t(it.h0) * a.head_stride + uint64_t(off) * a.token_stride);
  Raw<C, V> raw[kHeads][2];
  float scale[kHeads];
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    scale[j] = 1.f;
    if (slot >= 0 && it.h0 + j < a.n_heads) {
      raw[j][0].load(from + uint64_t(j) * a.head_stride + lo);
      raw[j][1].load(from + uint64_t(j) * a.head_stride + hi);
      if (F::quantised) scale[j] = a.scales[it.side][uint64_t(page * a.n_heads + it.h0 + j) * a.page_size.d + off];
    } else {
#pragma unroll
      for (int i = 0; i < int(sizeof raw[0][0].w / 4); ++i) raw[j][0].w[i] = raw[j][1].w[i] = 0;
    }
  }
  T* to = static_cast<T*>(a.rows[it.side]) + (uint64_t(it.t) * a.row_token[it.side] + uint64_t(it.h0) * a.row_head[it.side]);
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    if (it.h0 + j >= a.n_heads) break;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      Raw<T, V> y;
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        float2 x;
        if constexpr (F::quantised) {
          x = F::unpack2(raw[j][half].w[i / 4] >> (8 * (i & 2)) & 0xffffu);
          x.x *= scale[j], x.y *= scale[j];
        } else {
          x = make_float2(to_f32(raw[j][half].get(i)), to_f32(raw[j][half].get(i + 1)));
        }
        y.set(i, from_f32<T>(x.x)), y.set(i + 1, from_f32<T>(x.y));
      }
      T* const row = to + uint64_t(j) * a.row_head[it.side] + (half ? hi : lo);
      if (VEC) {
        y.store(row);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) row[i] = y.get(i);
      }
    }
  }
}

template <typename T, int FMT, bool VEC>
cudaError_t launch(bool write, const CacheArgs& a, cudaStream_t stream) {
  const uint32_t blocks = uint32_t(((uint64_t(a.n_groups) << a.lanes_log2) + 255) / 256);
  void (*kernel)(CacheArgs) = bcp_kv_read_kernel<T, FMT, VEC>;
  if (write) kernel = a.layout == BCP_ROPE_PAIRS ? bcp_kv_write_kernel<T, FMT, VEC, true> : bcp_kv_write_kernel<T, FMT, VEC, false>;
  return launch_early(kernel, blocks, 256, 0, stream, a);
}
template <typename T>
cudaError_t launch(bool write, const CacheArgs& a, uint32_t format, bool vec, cudaStream_t stream) {
  switch (format) {
    case BCP_BF16: return vec ? launch<T, BCP_BF16, true>(write, a, stream) : launch<T, BCP_BF16, false>(write, a, stream);
    case BCP_F16: return vec ? launch<T, BCP_F16, true>(write, a, stream) : launch<T, BCP_F16, false>(write, a, stream);
    case BCP_E4M3: return vec ? launch<T, BCP_E4M3, true>(write, a, stream) : launch<T, BCP_E4M3, false>(write, a, stream);
    default: return vec ? launch<T, BCP_I8, true>(write, a, stream) : launch<T, BCP_I8, false>(write, a, stream);
  }
}

int move(const char* call, bool write, const bcp_kv_cache* c, const bcp_heads* k, const bcp_heads* v, const int64_t* slots, int64_t n_tokens,
         const bcp_rope_table* rope, const int64_t* positions, void* stream) {
  if (int rc = check_cache(call, c)) return rc;
  if (n_tokens < 0 || n_tokens > 0x7fffffff) return fail(BCP_ERR_INVALID, "%s: %lld tokens", call, (long long)n_tokens);
  if (int rc = check_heads(call, "k", k, !write, c->head_dim, n_tokens)) return rc;
  if (int rc = check_heads(call, "v", v, !write, c->head_dim, n_tokens)) return rc;
  if (k->type != v->type) return fail(BCP_ERR_MISMATCH, "%s: k and v have different types", call);
  if (k->n_heads != c->n_heads || v->n_heads != c->n_heads)
    return fail(BCP_ERR_MISMATCH, "%s: %u key and %u value heads for a cache of %u", call, k->n_heads, v->n_heads, c->n_heads);
  if (rope) {
    if (int rc = check_rope(call, rope, c->head_dim)) return rc;
  }
  if (n_tokens && !slots) return fail(BCP_ERR_INVALID, "%s: slots is NULL", call);
  if (n_tokens && rope && !positions) return fail(BCP_ERR_INVALID, "%s: positions is NULL", call);

  CacheArgs a = {};
  a.pages[0] = c->k, a.pages[1] = c->v, a.scales[0] = c->k_scale, a.scales[1] = c->v_scale;
  a.page_stride = uint32_t(c->page_stride), a.head_stride = uint32_t(c->head_stride), a.token_stride = uint32_t(c->token_stride);
  a.n_slots = c->n_pages * c->page_size, a.n_heads = c->n_heads, a.head_dim = c->head_dim;
  a.page_size = FastDiv(c->page_size);
  a.status = c->status;
  a.row_token[0] = uint32_t(k->token_stride), a.row_head[0] = uint32_t(k->head_stride);
  a.row_token[1] = uint32_t(v->token_stride), a.row_head[1] = uint32_t(v->head_stride);
  a.rot_dim = rope ? rope->rot_dim : 0, a.layout = rope ? rope->layout : 0;
  a.table = rope ? rope->table : nullptr, a.n_positions = rope ? rope->n_positions : 0;
  const bool vec = a.rot_dim % 16 == 0 && rows_aligned(k, 16) && rows_aligned(v, 16);
  const uint32_t size = vec ? 16 / type_size(k->type) : 8;  // of a chunk
  const uint32_t ck = chunks_of(c->head_dim, a.rot_dim, size), cv = chunks_of(c->head_dim, 0, size), lanes = ck > cv ? ck : cv;
  a.lanes_log2 = 0;  // at most 5: 32 chunks of 8 elements, or 17 of 16
  while ((1u << a.lanes_log2) < lanes) ++a.lanes_log2;
  const uint32_t per_token = 2 * ((c->n_heads + kHeads - 1) / kHeads);
  a.per_token = FastDiv(per_token);
  // thread indices stay below 2^31: longer inputs take several launches
  const int64_t most = 0x7fffff00 / (per_token << a.lanes_log2);
  const uint32_t es = type_size(k->type);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int64_t t0 = 0; t0 < n_tokens; t0 += most) {
    const int64_t n = n_tokens - t0 < most ? n_tokens - t0 : most;
    a.n_groups = uint32_t(n) * per_token;
    a.slots = slots + t0;
    a.positions = positions ? positions + t0 : nullptr;
    a.rows[0] = static_cast<char*>(k->data) + t0 * k->token_stride * es;
    a.rows[1] = static_cast<char*>(v->data) + t0 * v->token_stride * es;
    if (k->type == BCP_F32) BCP_CUDA(launch<float>(write, a, c->format, vec, st));
    if (k->type == BCP_BF16) BCP_CUDA(launch<__nv_bfloat16>(write, a, c->format, vec, st));
    if (k->type == BCP_F16) BCP_CUDA(launch<__half>(write, a, c->format, vec, st));
  }
  return BCP_OK;
}

}  // namespace

extern "C" {

int bcp_kv_write(const bcp_kv_cache* cache, const bcp_heads* k, const bcp_heads* v, const int64_t* slots, int64_t n_tokens,
                 const bcp_rope_table* rope, const int64_t* positions, void* stream) {
  return move("bcp_kv_write", true, cache, k, v, slots, n_tokens, rope, positions, stream);
}

int bcp_kv_read(const bcp_kv_cache* cache, const int64_t* slots, int64_t n_tokens, const bcp_heads* k_out, const bcp_heads* v_out, void* stream) {
  return move("bcp_kv_read", false, cache, k_out, v_out, slots, n_tokens, nullptr, nullptr, stream);
}

}  // extern "C"

// The paged key-value cache: new tokens written into their slots, slots read back.
//
// Both are bound by memory: a head vector is read once and written once.  A group of lanes (a power of
// two, at least head_dim / 16) holds one vector, sixteen elements a lane, so the largest magnitude that
// an 8-bit format's scale needs is a few shuffles away and the vector is never read twice.  A group
// takes four heads of one token, whose loads are all in flight before the first one is used.
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
  if (c->page_stride <= 0 || c->head_stride <= 0 || c->token_stride <= 0 || (bits & 15))
    return fail(BCP_ERR_INVALID, "%s: cache addresses and strides must be positive multiples of 16 bytes", call);
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

constexpr int kHeads = 4;            // heads per group of lanes
constexpr float kSmallestScale = 1.262177448353619e-29f;  // 2^-96: its reciprocal and sums of it stay finite

struct CacheArgs {
  void* pages[2];
  float* scales[2];
  int64_t page_stride, head_stride, token_stride;
  uint32_t n_slots, n_heads, head_dim;
  FastDiv page_size;
  uint32_t* status;
  // the token-major side
  void* rows[2];
  int64_t row_token[2], row_head[2];
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

// Eight values of either half of a chunk, in an 8-bit format: two words per half, or four words of
// neighbouring pairs.
template <int FMT, bool VEC>
__device__ __forceinline__ void store_8bit(uint8_t* row, const Chunk& k, const float (&x)[8], const float (&y)[8], float inv) {
  typedef Format<FMT> F;
  if (VEC && k.step == 2) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = F::pack2(x[2 * i] * inv, y[2 * i] * inv) | F::pack2(x[2 * i + 1] * inv, y[2 * i + 1] * inv) << 16;
    *reinterpret_cast<uint4*>(row + k.a) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
  uint32_t p[4], q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = F::pack2(x[2 * i] * inv, x[2 * i + 1] * inv);
    q[i] = F::pack2(y[2 * i] * inv, y[2 * i + 1] * inv);
  }
  if (VEC) {
    *reinterpret_cast<uint2*>(row + k.a) = make_uint2(p[0] | p[1] << 16, p[2] | p[3] << 16);
    *reinterpret_cast<uint2*>(row + k.b) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (uint32_t(i) < k.n_a) row[k.a + i * k.step] = uint8_t(p[i / 2] >> (8 * (i & 1)));
      if (uint32_t(i) < k.n_b) row[k.b + i * k.step] = uint8_t(q[i / 2] >> (8 * (i & 1)));
    }
  }
}

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(256) bcp_kv_write_kernel(const CacheArgs a) {
  typedef Format<FMT> F;
  typedef typename F::T C;
  const Item it = item_of(a);
  const uint32_t rot = it.side ? 0 : a.rot_dim;
  const bool mine = it.lane < chunks_of(a.head_dim, rot);
  const Chunk k = chunk_at(mine ? it.lane : 0, a.head_dim, rot, a.layout);
  int64_t slot = it.used ? a.slots[it.t] : -1, position = 0;
  if (slot >= int64_t(a.n_slots)) {
    raise(a.status, BCP_BAD_SLOT);
    slot = -1;
  }
  if (slot >= 0 && a.rot_dim) {  // both sides look at the position: a token is written whole or not at all
    position = a.positions[it.t];
    if (position < 0 || position >= a.n_positions) {
      raise(a.status, BCP_BAD_POSITION);
      slot = -1;
    }
  }
  const bool live = slot >= 0 && mine;
  const uint32_t page = a.page_size.div(uint32_t(slot >= 0 ? slot : 0)), off = uint32_t(slot) - page * a.page_size.d;
  Elements<T, VEC> e[kHeads];
  const T* from = static_cast<const T*>(a.rows[it.side]) + it.t * a.row_token[it.side] + it.h0 * a.row_head[it.side];
#pragma unroll
  for (int j = 0; j < kHeads; ++j)
    if (live && it.h0 + j < a.n_heads) e[j].load(from + j * a.row_head[it.side], k);
  Angles<VEC> w;
  if (live && k.rotated) w.load(a.table, position, rot, k);
  C* to = static_cast<C*>(a.pages[it.side]) + page * a.page_stride + it.h0 * a.head_stride + off * a.token_stride;
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const bool on = live && it.h0 + j < a.n_heads;
    float x[8], y[8];
    if (on) {
      e[j].unpack(x, y, k);
      if (k.rotated) w.rotate(x, y, 1.f);
    }
    if constexpr (F::quantised) {
      // magnitudes compare like their bit patterns, and a NaN's is above all of them
      uint32_t m = 0;
      if (on) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (VEC || uint32_t(i) < k.n_a) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
          if (VEC || uint32_t(i) < k.n_b) m = max(m, __float_as_uint(y[i]) & 0x7fffffffu);
        }
      }
      for (uint32_t o = 1u << a.lanes_log2 >> 1; o; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      const float scale = m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__fdiv_rn(__uint_as_float(m), F::qmax), kSmallestScale);
      if (on) {
        store_8bit<FMT, VEC>(reinterpret_cast<uint8_t*>(to + j * a.head_stride), k, x, y, __frcp_rn(scale));
        if (it.lane == 0) a.scales[it.side][(int64_t(page) * a.n_heads + it.h0 + j) * a.page_size.d + off] = scale;
      }
    } else if (on) {
      Elements<C, VEC> c;
      c.pack(x, y, k);
      c.store(to + j * a.head_stride, k);
    }
  }
}

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(256) bcp_kv_read_kernel(const CacheArgs a) {
  typedef Format<FMT> F;
  typedef typename F::T C;
  constexpr int kWords = F::quantised ? 1 : 2;  // 16-byte vectors per sixteen elements
  const Item it = item_of(a);
  if (!it.used || it.lane * 16 >= a.head_dim) return;
  int64_t slot = a.slots[it.t];
  if (slot >= int64_t(a.n_slots)) {
    raise(a.status, BCP_BAD_SLOT);
    slot = -1;
  }
  const Chunk k = chunk_at(it.lane, a.head_dim, 0, 0);
  const uint32_t page = a.page_size.div(uint32_t(slot >= 0 ? slot : 0)), off = uint32_t(slot) - page * a.page_size.d;
  const C* from = static_cast<const C*>(a.pages[it.side]) + page * a.page_stride + it.h0 * a.head_stride + off * a.token_stride + 16 * it.lane;
  uint4 raw[kHeads][kWords];
  float scale[kHeads];
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const bool on = slot >= 0 && it.h0 + j < a.n_heads;
#pragma unroll
    for (int i = 0; i < kWords; ++i) raw[j][i] = on ? __ldg(reinterpret_cast<const uint4*>(from + j * a.head_stride) + i) : make_uint4(0, 0, 0, 0);
    scale[j] = 1.f;
    if (F::quantised && on) scale[j] = __ldg(a.scales[it.side] + (int64_t(page) * a.n_heads + it.h0 + j) * a.page_size.d + off);
  }
  T* to = static_cast<T*>(a.rows[it.side]) + it.t * a.row_token[it.side] + it.h0 * a.row_head[it.side];
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    if (it.h0 + j >= a.n_heads) break;
    float x[8], y[8];
    if constexpr (F::quantised) {
      const uint32_t w[4] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 p = F::unpack2(w[i / 2] >> (16 * (i & 1)) & 0xffffu), q = F::unpack2(w[2 + i / 2] >> (16 * (i & 1)) & 0xffffu);
        x[2 * i] = p.x * scale[j], x[2 * i + 1] = p.y * scale[j];
        y[2 * i] = q.x * scale[j], y[2 * i + 1] = q.y * scale[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = to_f32(reinterpret_cast<const C*>(raw[j])[i]);
        y[i] = to_f32(reinterpret_cast<const C*>(raw[j])[8 + i]);
      }
    }
    Elements<T, VEC> e;
    e.pack(x, y, k);
    e.store(to + j * a.row_head[it.side], k);
  }
}

template <typename T, bool VEC>
void launch(bool write, const CacheArgs& a, uint32_t format, cudaStream_t stream) {
  const uint32_t blocks = uint32_t(((uint64_t(a.n_groups) << a.lanes_log2) + 255) / 256);
#define BCP_ON(F)                                                           \
  if (format == F) {                                                        \
    if (write)                                                              \
      bcp_kv_write_kernel<T, F, VEC><<<blocks, 256, 0, stream>>>(a);        \
    else                                                                    \
      bcp_kv_read_kernel<T, F, VEC><<<blocks, 256, 0, stream>>>(a);         \
  }
  BCP_ON(BCP_BF16)
  BCP_ON(BCP_F16)
  BCP_ON(BCP_E4M3)
  BCP_ON(BCP_I8)
#undef BCP_ON
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

  CacheArgs a;
  a.pages[0] = c->k, a.pages[1] = c->v, a.scales[0] = c->k_scale, a.scales[1] = c->v_scale;
  a.page_stride = c->page_stride, a.head_stride = c->head_stride, a.token_stride = c->token_stride;
  a.n_slots = c->n_pages * c->page_size, a.n_heads = c->n_heads, a.head_dim = c->head_dim;
  a.page_size = FastDiv(c->page_size);
  a.status = c->status;
  a.row_token[0] = k->token_stride, a.row_head[0] = k->head_stride;
  a.row_token[1] = v->token_stride, a.row_head[1] = v->head_stride;
  a.rot_dim = rope ? rope->rot_dim : 0, a.layout = rope ? rope->layout : 0;
  a.table = rope ? rope->table : nullptr, a.n_positions = rope ? rope->n_positions : 0;
  const uint32_t ck = chunks_of(c->head_dim, a.rot_dim), cv = chunks_of(c->head_dim, 0), lanes = ck > cv ? ck : cv;
  a.lanes_log2 = 0;
  while ((1u << a.lanes_log2) < lanes) ++a.lanes_log2;
  const uint32_t per_token = 2 * ((c->n_heads + kHeads - 1) / kHeads);
  a.per_token = FastDiv(per_token);
  const bool vec = a.rot_dim % 16 == 0 && rows_aligned(k, 16) && rows_aligned(v, 16);
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
#define BCP_ON(TYPE, T)                                        \
  if (k->type == TYPE) {                                       \
    if (vec)                                                   \
      launch<T, true>(write, a, c->format, st);                \
    else                                                       \
      launch<T, false>(write, a, c->format, st);               \
  }
    BCP_ON(BCP_F32, float)
    BCP_ON(BCP_BF16, __nv_bfloat16)
    BCP_ON(BCP_F16, __half)
#undef BCP_ON
    BCP_LAUNCHED(call);
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

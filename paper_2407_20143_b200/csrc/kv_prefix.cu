// Attention of groups of sequences over the prefix that each group shares, computed once for all of them.
//
// Mathematics.  The query rows of a group under one cache head, (sequence, query head) by (sequence, query head), are the rows of S = Q K^T and O = P V
// with P = exp2(S c - m), c = scale log2 e.  m is a row's reference: when a score exceeds it by more than 8, the row's sums are brought to the new
// one.  What is left of the prefix are records (o, m, l) a row, which the attention over the sequences' own tokens joins (kv_attend.cu).
//
// What bounds it: up to 256 rows a cache head, reading the prefix once (a byte of a 16-bit cache meets 256 rows in 512 multiply-adds,
// 1024 with the second product of the weights); beyond that the products, the exponentials and the rounding of the weights.
//
// Both products are tcgen05.mma with 128 rows.  A CTA has two streams, each a warpgroup with 128 rows (a thread a row), their scores and their output in
// tensor memory: with more than 128 rows in a tile both take every 128 tokens, else they take turns with the same rows; one works on its weights while the
// tensor cores work for the other.  Weights go back to tensor memory in place of the scores and are the first operand of the second
// product from there.  Over bfloat16 and 8-bit caches a weight is the sum of two bfloat16 numbers (2^-16 of it), as one alone would be rounded as
// coarsely as the result; 8-bit values are widened to bfloat16, keys to binary16, both exactly, the value's scale goes into the weight.
// Four warps bring tokens by 16-byte asynchronous copies through a ring of tiles (pages may have any size and place), a warp issues the products.
//
// Split.  The tiles of all groups, cache heads and 256 rows form one line that is cut into as many equal parts as there are SMs.
#include <mutex>

#include "attend.cuh"
#include "tma_ptx.cuh"

namespace bcp {
namespace {

constexpr uint32_t kRows = 128;             // rows of a stream
constexpr uint32_t kLoaders = 4;            // warps that copy
constexpr uint32_t kMeta = 16;              // tiles whose masks and scales are kept
constexpr uint64_t kMostNs = 2000000000ull; // a wait that takes longer gives up

struct PrefixArgs {
  const void *k, *v;
  const float *k_scale, *v_scale;
  uint32_t page_stride, head_stride, token_stride;
  uint32_t n_pages, n_heads, head_dim;
  FastDiv page_size;
  uint32_t* status;
  const void* q;
  int64_t q_token, q_head;
  uint32_t q_is_bf16, n_seqs, n_groups;
  FastDiv group;  // query heads of a cache head
  const int32_t* table;
  int64_t table_stride;
  uint32_t capacity;
  const int32_t *lengths, *starts;
  float scale_log2;
  int4* rows;
  float2* ml;
  float* o;
};

template <int FMT, int DP>
struct Shape {
  static constexpr bool quant = FMT == BCP_E4M3 || FMT == BCP_I8;
  static constexpr bool split = FMT != BCP_F16;              // weights as two bfloat16 numbers
  static constexpr uint32_t STREAMS = DP <= 128 ? 2 : 1;     // tensor memory holds the scores and outputs of so many
  static constexpr uint32_t TOK = DP <= 128 ? 128 : 64;      // tokens of a tile
  static constexpr uint32_t ROWS = STREAMS * kRows;
  static constexpr uint32_t TILE = TOK * DP * 2;             // bytes of a tile of keys or values in 16 bits
  static constexpr uint32_t Q = kRows * DP * 2;
  static constexpr uint32_t RAW = quant ? TOK * DP : 0;      // of a tile as it lies in an 8-bit cache
  static constexpr uint32_t RAWS = quant ? 3 : 0;
  static constexpr uint32_t META = quant ? 16 + TOK * 8 + 16 : 16;
  static constexpr uint32_t NMETA = quant ? 8 : kMeta;
  static constexpr uint32_t SLOTS = DP == 64 ? 8 : quant ? 3 : 5;
  static constexpr uint32_t AHEAD = quant ? RAWS - 1 : 3;    // copies of so many tiles are under way
  static constexpr uint32_t SMEM = STREAMS * Q + SLOTS * TILE + RAWS * RAW + NMETA * META + 8 * (2 * SLOTS + NMETA + 4 * STREAMS + 1) + 64 + 1024;
  static constexpr uint32_t WARPS = 4 * STREAMS + kLoaders + 1, THREADS = 32 * WARPS;
  static constexpr uint32_t S0 = 0, O0 = STREAMS * TOK;      // columns of tensor memory
  static_assert(O0 + STREAMS * DP <= 512, "tensor memory");
  static_assert(SMEM <= 232448, "shared memory");
  static_assert(AHEAD < SLOTS || quant, "copies that wait for a tile's place");
};

// ------------------------------------------------------------------------------ instructions
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// False, in all lanes of a warp, if the wait ran out here or in another warp.
__device__ __noinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, volatile uint32_t* stop) {
  const uint64_t begin = global_timer_ns();
  while (!mbar_try_wait(bar, parity)) {
    if (*stop) return false;
    if (global_timer_ns() - begin > kMostNs) {
      *stop = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* stop) {
  return __all_sync(0xffffffffu, mbar_try_wait(bar, parity) || bar_wait_slow(bar, parity, stop));
}

__device__ __forceinline__ void tmem_alloc(uint32_t to) { asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(to) : "memory"); }
__device__ __forceinline__ void tmem_free(uint32_t at) {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\ntcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory");
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 32 columns of this thread's row
__device__ __forceinline__ void tmem_load32(uint32_t at, float (&x)[32]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
      "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
        "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
               "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&x)[16]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                 "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(at));
}

// Shared-memory operands in rows of 128 bytes (64 elements), eight rows a swizzled block of 1024 bytes, blocks of rows one after the other.
// Keys and queries (the sum runs along the row): `apart` is not used.  Values (the sum runs over rows): `apart` bytes from 64 columns to the next.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t apart) {
  return uint64_t(at >> 4 & 0x3fff) | uint64_t(apart >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// kind::f16 with binary32 sums, 128 rows, n columns; both operands bfloat16 or both binary16; the second one's rows along the sum or not
__host__ __device__ constexpr uint32_t product(bool bf16, bool second_by_rows, uint32_t n) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (second_by_rows ? 1u << 16 : 0u) | (n >> 3) << 17 | (kRows >> 4) << 24;
}
__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(what),
               "r"(uint32_t(add))
               : "memory");
}
__device__ __forceinline__ void mma_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(what),
               "r"(uint32_t(add))
               : "memory");
}
__device__ __forceinline__ void shared_store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 shared_load16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// ------------------------------------------------------------------------------ the line
struct Group {
  uint32_t first, rows;   // first sequence; rows under a cache head
  uint32_t len, steps, tiles;
};
template <typename S>
__device__ __forceinline__ Group group_of(const PrefixArgs& a, uint32_t g) {
  Group x;
  const int32_t s0 = a.starts[g], s1 = a.starts[g + 1], n = a.lengths[g], most = int32_t(a.n_seqs);
  x.first = uint32_t(min(max(s0, 0), most));
  const uint32_t end = uint32_t(min(max(s1, int32_t(x.first)), most));
  x.rows = (end - x.first) * a.group.d;
  x.len = min(uint32_t(max(n, 0)), a.capacity);
  x.steps = (x.len + S::TOK - 1) / S::TOK;
  x.tiles = (x.rows + S::ROWS - 1) / S::ROWS;
  return x;
}
// A place on the line: group g, unit u (cache head, then tile of rows) of it, step of the unit.
struct Place {
  uint32_t g, u, step;
  Group group;
};
template <typename S>
__device__ __forceinline__ void advance(Place& p, const PrefixArgs& a, uint32_t n, bool more) {
  p.step += n;
  if (p.step < p.group.steps) return;
  p.step = 0;
  if (++p.u < a.n_heads * p.group.tiles) return;
  p.u = 0;
  while (more && ++p.g < a.n_groups) {
    p.group = group_of<S>(a, p.g);
    if (p.group.steps && p.group.tiles) return;
  }
}

template <int FMT, int DP>
__global__ void __launch_bounds__(Shape<FMT, DP>::THREADS, 1) bcp_kv_prefix_kernel(const PrefixArgs a) {
  typedef Shape<FMT, DP> S;
  extern __shared__ unsigned char raw_smem[];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* const smem = raw_smem + (1024 - (uint32_t(__cvta_generic_to_shared(raw_smem)) & 1023) & 1023);
  const uint32_t base = uint32_t(__cvta_generic_to_shared(smem));
  const uint32_t q_at = base, ring = q_at + S::STREAMS * S::Q, raw = ring + S::SLOTS * S::TILE, meta = raw + S::RAWS * S::RAW;
  unsigned char* const meta_ptr = smem + (meta - base);
  const uint32_t bars = meta + S::NMETA * S::META;
  const uint32_t full = bars, empty = full + 8 * S::SLOTS, described = empty + 8 * S::SLOTS, q_full = described + 8 * S::NMETA, s_full = q_full + 8 * S::STREAMS,
                 p_full = s_full + 8 * S::STREAMS, o_full = p_full + 8 * S::STREAMS, drained = o_full + 8 * S::STREAMS;
  uint32_t* const words = reinterpret_cast<uint32_t*>(smem + (drained + 8 - base));  // tensor memory, stop, found[3], totals
  volatile uint32_t* const stop = words + 1;
  uint32_t* const found = words + 2;
  uint32_t* const totals = reinterpret_cast<uint32_t*>(smem);  // before the tiles come

  after_previous();
  // ---- rows without a prefix have no records
  const uint32_t n_q_heads = a.n_heads * a.group.d;
  for (uint32_t b = blockIdx.x * S::THREADS + tid; b < a.n_seqs; b += gridDim.x * S::THREADS) {
    uint32_t lo = 0, hi = a.n_groups;  // the last group that starts at or before b
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if (a.starts[mid] <= int32_t(b)) lo = mid + 1; else hi = mid;
    }
    bool has = false;
    if (lo) {
      const Group x = group_of<S>(a, lo - 1);
      has = b >= x.first && b - x.first < x.rows / a.group.d && x.steps;
    }
    if (!has)
      for (uint32_t h = 0; h < n_q_heads; ++h) a.rows[uint64_t(b) * n_q_heads + h] = make_int4(0, 0, 0, 0);
  }
  if (a.status && blockIdx.x == 0)
    for (uint32_t g = tid; g < a.n_groups; g += S::THREADS)
      if (a.lengths[g] > int32_t(a.capacity) || a.starts[g] < 0 || a.starts[g + 1] < a.starts[g] || a.starts[g + 1] > int32_t(a.n_seqs))
        raise(a.status, BCP_BAD_LENGTH);

  // ---- the line, and this CTA's part of it
  const uint32_t run = (a.n_groups + S::THREADS - 1) / S::THREADS;
  const uint32_t run0 = min(tid * run, a.n_groups), run1 = min(run0 + run, a.n_groups);
  uint32_t mine = 0, before;
  for (uint32_t g = run0; g < run1; ++g) {
    const Group x = group_of<S>(a, g);
    mine += x.steps * x.tiles * a.n_heads;
  }
  before = mine;
#pragma unroll
  for (uint32_t o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += x;
  }
  if (lane == 31) totals[warp] = before;
  if (tid == 0) *stop = 0;
  __syncthreads();
  uint32_t all = 0;
  before -= mine;
  for (uint32_t w = 0; w < S::WARPS; ++w) {
    if (w < warp) before += totals[w];
    all += totals[w];
  }
  if (!all) return;
  Cuts cuts;
  cuts.cut(all, gridDim.x);
  if (blockIdx.x >= cuts.parts) return;
  const uint32_t s0 = cuts.begin(blockIdx.x), n_steps = cuts.begin(blockIdx.x + 1) - s0;
  if (s0 >= before && s0 < before + mine) {
    uint32_t pre = before, g = run0;
    for (;; ++g) {
      const Group x = group_of<S>(a, g);
      const uint32_t n = x.steps * x.tiles * a.n_heads;
      if (s0 < pre + n) {
        found[0] = g, found[1] = (s0 - pre) / x.steps, found[2] = (s0 - pre) % x.steps;
        break;
      }
      pre += n;
    }
  }
  if (tid == 0) {
    for (uint32_t i = 0; i < S::SLOTS; ++i) mbar_init(full + 8 * i, 32 * kLoaders), mbar_init(empty + 8 * i, 1);
    for (uint32_t i = 0; i < S::NMETA; ++i) mbar_init(described + 8 * i, 32 * kLoaders);
    for (uint32_t i = 0; i < S::STREAMS; ++i)
      mbar_init(q_full + 8 * i, kRows), mbar_init(s_full + 8 * i, 1), mbar_init(p_full + 8 * i, kRows), mbar_init(o_full + 8 * i, 1);
    mbar_init(drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == S::WARPS - 1) tmem_alloc(uint32_t(__cvta_generic_to_shared(words)));
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *static_cast<volatile uint32_t*>(words);
  Place at;
  at.g = found[0], at.u = found[1], at.step = found[2];
  at.group = group_of<S>(a, at.g);

  uint32_t left = n_steps;
  if (warp < 4 * S::STREAMS) {
    // ================================================================ a stream's rows
    const uint32_t stream = warp >> 2, row = tid & (kRows - 1);
    const uint32_t lanes = tmem + ((warp & 3) << 21);  // this warp's 32 rows
    const uint32_t s_at = lanes + S::S0 + stream * S::TOK, o_at = lanes + S::O0 + stream * DP;
    uint32_t n_scores = 0, n_ends = 0, tile0 = 0;
    const float scale = fabsf(a.scale_log2);
    bool ok = true;
    while (left && ok) {
      const uint32_t n = min(at.group.steps - at.step, left);
      const uint32_t h = at.u / at.group.tiles, row0 = (at.u - h * at.group.tiles) * S::ROWS, rows = min(at.group.rows - row0, S::ROWS);
      const bool both = rows > kRows;  // the streams have rows of their own, else they take turns
      const uint32_t r = row0 + (both ? stream * kRows : 0) + row;
      const bool live = r < row0 + rows;
      const uint32_t seq = a.group.div(live ? r : 0), head = h * a.group.d + (live ? r : 0) - seq * a.group.d, b = at.group.first + seq;

      // ---- the query into shared memory; over 8-bit caches a power of two brings its largest element into [1, 2), so that it fits binary16
      const bool any = both || stream < n;  // has tiles here
      float factor = scale;
      if (any) {
        const uint2* const from = reinterpret_cast<const uint2*>(static_cast<const char*>(a.q) + (b * a.q_token + head * a.q_head) * 2);
        const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;  // the scale's sign goes into the query
        const uint32_t to = q_at + stream * S::Q + row * 128;
        float up = 1.f;
        if constexpr (S::quant) {
          uint32_t top = 0;
          if (live)
            for (uint32_t i = 0; i < a.head_dim / 4; ++i) {
              const uint2 w = from[i];
#pragma unroll
              for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(query_at(&w, j, a.q_is_bf16)) & 0x7fffffffu);
            }
          const uint32_t e = top >> 23 == 254 ? 253 : top >> 23;
          if (e >= 1 && e <= 253) up = __uint_as_float((254 - e) << 23), factor *= __uint_as_float(e << 23);
        }
#pragma unroll 4
        for (uint32_t c = 0; c < a.head_dim / 8; ++c) {
          uint2 x = make_uint2(0, 0), y = x;
          if (live) x = from[2 * c], y = from[2 * c + 1];
          if constexpr (S::quant) {
            auto two = [&](uint32_t w) { return pack16<false>(query_at(&w, 0, a.q_is_bf16) * up, query_at(&w, 1, a.q_is_bf16) * up); };
            x = make_uint2(two(x.x), two(x.y)), y = make_uint2(two(y.x), two(y.y));
          }
          shared_store16(to + (c >> 3) * (kRows * 128) + ((c & 7 ^ row & 7) << 4), x.x ^ flip, x.y ^ flip, y.x ^ flip, y.y ^ flip);
        }
      }
      if (any) {
        to_async_proxy();
        bar_arrive(q_full + 8 * stream);
      }

      float ref = kNone, l = 0.f, top_scale = 0.f, unit = 1.f;  // unit: what the values' scales are multiplied by
      bool first = true;
      const uint32_t step = both ? 1 : S::STREAMS;
      uint32_t t = both ? 0 : stream;
      for (; t < n; t += step) {
        const uint32_t m_slot = (tile0 + t) % S::NMETA;
        const unsigned char* const about = meta_ptr + m_slot * S::META;
        ok = bar_wait(described + 8 * m_slot, (tile0 + t) / S::NMETA & 1, stop) && bar_wait(s_full + 8 * stream, n_scores & 1, stop);
        if (!ok) break;
        ++n_scores;
        tmem_after();
        const uint4 alive = *reinterpret_cast<const uint4*>(about);
        const uint32_t mask[4] = {alive.x, alive.y, alive.z, alive.w};
        if (__any_sync(0xffffffffu, live)) {
          // the largest score
          float top = -INFINITY;
#pragma unroll
          for (uint32_t c = 0; c < S::TOK / 32; ++c) {
            float x[32];
            tmem_load32(s_at + 32 * c, x);
            tmem_load_wait();
            if constexpr (S::quant) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 ks = *reinterpret_cast<const float4*>(about + 16 + (32 * c + i) * 4);
                x[i] *= ks.x, x[i + 1] *= ks.y, x[i + 2] *= ks.z, x[i + 3] *= ks.w;
              }
            }
            if (mask[c] == 0xffffffffu) {
#pragma unroll
              for (int i = 0; i < 32; ++i) top = fmaxf(top, x[i]);
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (mask[c] >> i & 1) top = fmaxf(top, x[i]);
            }
          }
          if (top > -INFINITY) top *= factor;
          float down = 1.f, down_o = 1.f;
          if (top > ref + 8.f) down = down_o = exp2_fast(ref - top), ref = top, l *= down;
          if constexpr (S::quant) {
            // Weights times scales must neither overflow in the sums nor vanish: where scales beyond 2^60 turn up all are multiplied by 2^-40, while none
            // is above 2^-40 by 2^60.
            const float4 w = *reinterpret_cast<const float4*>(about + 16 + S::TOK * 8);
            top_scale = fmaxf(top_scale, fmaxf(fmaxf(w.x, w.y), fmaxf(w.z, w.w)));
            const float next = top_scale > 0x1p60f ? 0x1p-40f : top_scale < 0x1p-40f ? 0x1p60f : 1.f;
            if (next != unit) down_o *= next / unit, unit = next;
          }
          if (!first && __any_sync(0xffffffffu, down_o != 1.f)) {
#pragma unroll 1
            for (uint32_t c = 0; c < a.head_dim; c += 16) {
              float x[16];
              uint32_t y[16];
              tmem_load16(o_at + c, x);
              tmem_load_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(x[i] * down_o);
              tmem_store16(o_at + c, y);
            }
          }
          // the weights
#pragma unroll
          for (uint32_t c = 0; c < S::TOK / 32; ++c) {
            float x[32];
            tmem_load32(s_at + 32 * c, x);
            tmem_load_wait();
            constexpr float kLift = S::split ? 0.f : 6.f;  // binary16 weights underflow below 2^-24: lifted by 2^6 that is 2^-30
            const float less = kLift - ref;
            if constexpr (S::quant) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 ks = *reinterpret_cast<const float4*>(about + 16 + (32 * c + i) * 4);
                x[i] *= ks.x, x[i + 1] *= ks.y, x[i + 2] *= ks.z, x[i + 3] *= ks.w;
              }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = exp2_fast(fmaf(x[i], factor, less));
            if (mask[c] != 0xffffffffu) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(mask[c] >> i & 1)) x[i] = 0.f;
            }
            // the sum as four, so that no addition waits for the one before it
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[i & 3] += x[i];
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            if constexpr (S::quant) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 vs = *reinterpret_cast<const float4*>(about + 16 + S::TOK * 4 + (32 * c + i) * 4);
                x[i] *= vs.x * unit, x[i + 1] *= vs.y * unit, x[i + 2] *= vs.z * unit, x[i + 3] *= vs.w * unit;
              }
            }
            uint32_t y[16];
            if constexpr (S::split) {
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = upper_halves(x[2 * i], x[2 * i + 1]);
              tmem_store16(s_at + 32 * c, y);
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = pack16<true>(lower_half(x[2 * i]), lower_half(x[2 * i + 1]));
              tmem_store16(s_at + 32 * c + 16, y);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = pack16<false>(x[2 * i], x[2 * i + 1]);
              tmem_store16(s_at + 32 * c, y);
            }
          }
          tmem_store_wait();
        }
        first = false;
        tmem_before();
        bar_arrive(p_full + 8 * stream);
      }
      tile0 += n;
      if (!ok) break;
      // ---- the record
      const bool whole = at.step == 0 && n == at.group.steps;
      const uint32_t every = a.n_seqs * n_q_heads, place = s0 + n_steps - left;
      uint32_t record = b * n_q_heads + head + (!both && stream ? every : 0);
      if (!whole) record = 2 * every + (2 * blockIdx.x + (place != s0)) * S::ROWS + stream * kRows + row;
      if (any) {
        ok = bar_wait(o_full + 8 * stream, n_ends & 1, stop);
        if (!ok) break;
        ++n_ends;
        tmem_after();
        if (__any_sync(0xffffffffu, live)) {
#pragma unroll 1
          for (uint32_t c = 0; c < a.head_dim; c += 16) {
            float x[16];
            tmem_load16(o_at + c, x);
            tmem_load_wait();
            if (live) {
              float4* const to = reinterpret_cast<float4*>(a.o + uint64_t(record) * a.head_dim + c);
#pragma unroll
              for (int i = 0; i < 4; ++i) __stcg(to + i, make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]));
            }
          }
        }
        tmem_before();
      }
      if (live) {
        constexpr float kLift = S::split ? 0.f : 6.f;
        // a reference with the scales' unit in it, as sums over values have it
        const float shift = unit == 1.f ? 0.f : unit > 1.f ? 60.f : -40.f;
        __stcg(a.ml + record, any && ref > kNone ? make_float2(ref - kLift - shift, l * unit) : make_float2(kNone, any ? l : 0.f));
        if (at.step == 0 && (both || stream == 0)) {
          const uint32_t p0 = blockIdx.x, p1 = cuts.part_of(place + at.group.steps - 1);
          int4 d = make_int4(int(record), 0, int(p1 - p0 + 1), 0);
          if (S::STREAMS > 1 && !both) d.w = int(whole ? every : kRows);
          if (!whole) d.y = int(2 * every + 2 * (p0 + 1) * S::ROWS + stream * kRows + row);
          a.rows[uint64_t(b) * n_q_heads + head] = d;
        }
      }
      left -= n;
      advance<S>(at, a, n, left != 0);
    }
  } else if (warp < 4 * S::STREAMS + kLoaders) {
    // ================================================================ copies of keys and values
    const uint32_t w = warp - 4 * S::STREAMS, id = w * 32 + lane;
    constexpr uint32_t kEach = S::TOK / kLoaders;                 // rows of a tile that a warp copies
    constexpr uint32_t kChunks = DP * (S::quant ? 1 : 2) / 16;    // 16-byte chunks of a row
    constexpr uint32_t kTogether = 32 / kChunks, kTurns = kEach / kTogether;
    const uint32_t my_row = lane / kChunks, chunk = lane % kChunks;
    const bool inside = chunk * 16 < a.head_dim * (S::quant ? 1u : 2u);
    uint32_t item = 0, tile0 = 0, landed = 0;
    uint32_t kind[8];  // of the items under way: the tile whose keys they are, plus 1; 0: values
    const int64_t v_from_k = static_cast<const char*>(a.v) - static_cast<const char*>(a.k);
    bool ok = true;

    // What has come in goes on: 16-bit tiles lie where they belong, 8-bit ones are widened.
    auto land = [&]() {
      const uint32_t slot = landed % S::SLOTS, at_slot = ring + slot * S::TILE;
      const uint32_t keys = kind[landed & 7];
      if constexpr (S::quant) {
        if (landed >= S::SLOTS) ok = ok && bar_wait(empty + 8 * slot, landed / S::SLOTS - 1 & 1, stop);
        const uint32_t from = raw + landed % S::RAWS * S::RAW + id * 16;
#pragma unroll 2
        for (uint32_t i = 0; i < kTurns; ++i) {
          const uint32_t r = w * kEach + i * kTogether + my_row;
          const uint4 x = shared_load16(from + i * (kLoaders * 32 * 16));
          uint32_t y[8];
          const uint32_t in[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            widen4<FMT>(in[j], y[2 * j], y[2 * j + 1]);
            if (!keys) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&y[2 * j + e]));
                y[2 * j + e] = pack16<true>(f.x, f.y);
              }
            }
          }
          const uint32_t to = at_slot + (chunk >> 2) * (S::TOK * 128) + r * 128, c = 2 * (chunk & 3);
          shared_store16(to + ((c ^ r & 7) << 4), y[0], y[1], y[2], y[3]);
          shared_store16(to + ((c + 1 ^ r & 7) << 4), y[4], y[5], y[6], y[7]);
        }
        if (keys) {  // the largest of the values' scales
          unsigned char* const about = meta_ptr + (keys - 1) % S::NMETA * S::META;
          float top = lane < kEach ? *reinterpret_cast<volatile float*>(about + 16 + S::TOK * 4 + (w * kEach + lane) * 4) : 0.f;
#pragma unroll
          for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          if (lane == 0) *reinterpret_cast<volatile float*>(about + 16 + S::TOK * 8 + w * 4) = top;
          __syncwarp();
        }
      }
      if (keys) bar_arrive(described + 8 * ((keys - 1) % S::NMETA));
      to_async_proxy();
      bar_arrive(full + 8 * slot);
      ++landed;
    };
    // One tile of keys (or values) of cache head h, tokens pos0 on.
    auto bring = [&](uint32_t tile, uint32_t pos0, uint32_t h, bool keys) {
      if (!ok) return;
      const uint32_t pos = pos0 + w * kEach + (lane & (kEach - 1));
      int32_t page = -1;
      uint32_t off = 0;
      if (pos < at.group.len) {
        const uint32_t n = a.page_size.div(pos);
        off = pos - n * a.page_size.d;
        page = a.table[at.g * a.table_stride + n];
        if (uint32_t(page) >= a.n_pages) {
          raise(a.status, BCP_BAD_PAGE);
          page = -1;
        }
      }
      const bool on = page >= 0;
      const uint64_t row = on ? uint64_t(uint32_t(page)) * a.page_stride + uint64_t(h) * a.head_stride + uint64_t(off) * a.token_stride : 0;
      const uint32_t alive = __ballot_sync(0xffffffffu, on);
      const uint32_t slot = item % S::SLOTS;
      const char* const from = static_cast<const char*>(a.k) + (keys ? 0 : v_from_k);
      uint32_t to = ring + slot * S::TILE;
      if constexpr (S::quant) {
        to = raw + item % S::RAWS * S::RAW + id * 16;
      } else if (item >= S::SLOTS) {
        ok = bar_wait(empty + 8 * slot, item / S::SLOTS - 1 & 1, stop);
        if (!ok) return;
      }
#pragma unroll 4
      for (uint32_t i = 0; i < kTurns; ++i) {
        const uint32_t r = i * kTogether + my_row;
        const uint64_t x = __shfl_sync(0xffffffffu, row, r) * (S::quant ? 1 : 2) + chunk * 16;
        const bool copy = (alive >> r & 1) && inside;
        uint32_t place;
        if constexpr (S::quant) {
          place = to + i * (kLoaders * 32 * 16);
        } else {
          const uint32_t tile_row = w * kEach + r;
          place = to + (chunk >> 3) * (S::TOK * 128) + tile_row * 128 + ((chunk & 7 ^ tile_row & 7) << 4);
        }
        copy16(place, from + (copy ? x : 0), copy);
      }
      if (keys) {
        unsigned char* const about = meta_ptr + tile % S::NMETA * S::META;
        if (lane == 0) {
          if (kEach == 32) reinterpret_cast<volatile uint32_t*>(about)[w] = alive;
          if (kEach == 16) reinterpret_cast<volatile uint16_t*>(about)[w] = uint16_t(alive);
        }
        if constexpr (S::quant) {
          if (lane < kEach) {
            const uint64_t n = (uint64_t(uint32_t(on ? page : 0)) * a.n_heads + h) * a.page_size.d + off;
            const uint32_t there = meta + tile % S::NMETA * S::META + 16 + (w * kEach + lane) * 4;
            copy4(there, a.k_scale + n, on);
            copy4(there + S::TOK * 4, a.v_scale + n, on);
          }
        }
      }
      copies_end();
      kind[item & 7] = keys ? tile + 1 : 0;
      ++item;
      if (item - landed > S::AHEAD) {
        copies_wait<S::AHEAD>();
        land();
      }
    };
    while (left && ok) {
      const uint32_t n = min(at.group.steps - at.step, left), h = at.u / at.group.tiles;
      const uint32_t row0 = (at.u - h * at.group.tiles) * S::ROWS;
      const uint32_t ahead = min(at.group.rows - row0, S::ROWS) > kRows ? 1 : S::STREAMS;  // keys come so many tiles before values
      for (uint32_t t = 0; t < n + ahead; ++t) {
        if (t >= ahead) bring(tile0 + t - ahead, (at.step + t - ahead) * S::TOK, h, false);
        if (t < n) bring(tile0 + t, (at.step + t) * S::TOK, h, true);
      }
      tile0 += n;
      left -= n;
      advance<S>(at, a, n, left != 0);
    }
    copies_wait<0>();
    while (landed < item && ok) land();
  } else {
    // ================================================================ the products
    uint32_t item = 0, n_weights[2] = {0, 0}, n_queries[2] = {0, 0};
    const uint32_t depth = a.head_dim / 16;
    const uint32_t scores = product(FMT == BCP_BF16, false, S::TOK), sums = product(S::split, true, a.head_dim);
    bool ok = true;
    auto score = [&](uint32_t stream, uint32_t slot) {
      if (lane == 0) {
        const uint32_t q = q_at + stream * S::Q, k = ring + slot * S::TILE;
        for (uint32_t i = 0; i < depth; ++i)
          mma_shared(tmem + S::S0 + stream * S::TOK, operand(q + (i >> 2) * (kRows * 128) + (i & 3) * 32, 0), operand(k + (i >> 2) * (S::TOK * 128) + (i & 3) * 32, 0),
                     scores, i > 0);
        tmem_commit(s_full + 8 * stream);
      }
      __syncwarp();
    };
    auto weigh = [&](uint32_t stream, uint32_t slot, bool add) {
      if (lane == 0) {
        const uint32_t v = ring + slot * S::TILE, p = tmem + S::S0 + stream * S::TOK, o = tmem + S::O0 + stream * DP;
        for (uint32_t i = 0; i < S::TOK / 16; ++i) {
          const uint32_t from = p + (i >> 1) * 32 + (i & 1) * 8;
          mma_tensor(o, from, operand(v + i * 2048, S::TOK * 128), sums, add || i > 0);
          if (S::split) mma_tensor(o, from + 16, operand(v + i * 2048, S::TOK * 128), sums, true);
        }
      }
      __syncwarp();
    };
    auto commit = [&](uint32_t bar) {
      if (lane == 0) tmem_commit(bar);
      __syncwarp();
    };
    auto arrived = [&](uint32_t bar, uint32_t parity) {
      ok = ok && bar_wait(bar, parity, stop);
      tmem_after();
      return ok;
    };
    auto have = [&](uint32_t i) { return arrived(full + 8 * (i % S::SLOTS), i / S::SLOTS & 1); };
    while (left && ok) {
      const uint32_t n = min(at.group.steps - at.step, left);
      const uint32_t row0 = at.u % at.group.tiles * S::ROWS;
      const bool both = min(at.group.rows - row0, S::ROWS) > kRows;
      for (uint32_t s = 0; s < S::STREAMS; ++s)
        if ((both || s < n) && !arrived(q_full + 8 * s, n_queries[s]++ & 1)) break;
      if (!ok) break;
      if (both) {
        // every tile for both streams
        if (!have(item)) break;
        for (uint32_t s = 0; s < S::STREAMS; ++s) score(s, item % S::SLOTS);
        commit(empty + 8 * (item++ % S::SLOTS));
        for (uint32_t t = 0; t < n && ok; ++t) {
          const uint32_t values = item, keys = item + 1;
          if (!have(values)) break;
          for (uint32_t s = 0; s < S::STREAMS; ++s) {
            if (!arrived(p_full + 8 * s, n_weights[s]++ & 1)) break;
            weigh(s, values % S::SLOTS, t > 0);
            if (s == S::STREAMS - 1) commit(empty + 8 * (values % S::SLOTS));
            if (t + 1 < n) {
              if (!have(keys)) break;
              score(s, keys % S::SLOTS);
              if (s == S::STREAMS - 1) commit(empty + 8 * (keys % S::SLOTS));
            } else {
              commit(o_full + 8 * s);
            }
          }
          item += t + 1 < n ? 2 : 1;
        }
      } else {
        // the streams take turns
        for (uint32_t t = 0; t < min(n, S::STREAMS) && ok; ++t) {
          if (!have(item)) break;
          score(t, item % S::SLOTS);
          commit(empty + 8 * (item++ % S::SLOTS));
        }
        for (uint32_t t = 0; t < n && ok; ++t) {
          const uint32_t s = t % S::STREAMS;
          if (!have(item) || !arrived(p_full + 8 * s, n_weights[s]++ & 1)) break;
          weigh(s, item % S::SLOTS, t >= S::STREAMS);
          commit(empty + 8 * (item++ % S::SLOTS));
          if (t + S::STREAMS < n) {
            if (!have(item)) break;
            score(s, item % S::SLOTS);
            commit(empty + 8 * (item++ % S::SLOTS));
          } else {
            commit(o_full + 8 * s);
          }
        }
      }
      left -= n;
      advance<S>(at, a, n, left != 0);
    }
    if (!ok) {  // what was issued comes to its end before the tensor memory is given back
      commit(drained);
      const uint64_t begin = global_timer_ns();
      while (!mbar_try_wait(drained, 0) && global_timer_ns() - begin < kMostNs) {
      }
    }
  }
  tmem_before();
  __syncthreads();
  if (tid == 0 && *stop) raise(a.status, BCP_TIMED_OUT);
  tmem_after();
  if (warp == S::WARPS - 1) tmem_free(tmem);
}

// ------------------------------------------------------------------------------ launch
struct Variant {
  void (*kernel)(PrefixArgs);
  uint32_t smem, threads, rows, tokens;
};
template <int FMT, int DP>
Variant variant() {
  typedef Shape<FMT, DP> S;
  return Variant{bcp_kv_prefix_kernel<FMT, DP>, S::SMEM, S::THREADS, S::ROWS, S::TOK};
}
template <int FMT>
Variant variant_of(uint32_t head_dim) {
  return head_dim <= 64 ? variant<FMT, 64>() : head_dim <= 128 ? variant<FMT, 128>() : variant<FMT, 256>();
}
Variant variant_of(uint32_t format, uint32_t head_dim) {
  switch (format) {
    case BCP_BF16: return variant_of<BCP_BF16>(head_dim);
    case BCP_F16: return variant_of<BCP_F16>(head_dim);
    case BCP_E4M3: return variant_of<BCP_E4M3>(head_dim);
    default: return variant_of<BCP_I8>(head_dim);
  }
}

// SMs of the current device, whose kernels have been told how much shared memory they get.
int prepare(const Variant& v, uint32_t* sms) {
  struct Known {
    void (*kernel)(PrefixArgs);
    int device;
    uint32_t sms;
  };
  static std::mutex mu;
  static Known known[256];
  static int n_known = 0;
  int device = 0, n = 0;
  BCP_CUDA(cudaGetDevice(&device));
  std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < n_known; ++i)
    if (known[i].kernel == v.kernel && known[i].device == device) {
      *sms = known[i].sms;
      return BCP_OK;
    }
  BCP_CUDA(cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(v.smem)));
  BCP_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device));
  *sms = uint32_t(n);
  if (n_known < 256) known[n_known++] = {v.kernel, device, *sms};
  return BCP_OK;
}

uint64_t aligned(uint64_t n) { return (n + 255) / 256 * 256; }
// The workspace: that of the attention over own tokens, then rows, references and sums of the records.
struct Layout {
  uint64_t rows, ml, o, end, records;
  Layout(uint64_t begin, const Variant& v, uint32_t sms, uint64_t n_seqs, uint32_t n_q_heads, uint32_t head_dim) {
    const uint64_t every = n_seqs * n_q_heads;
    records = 2 * every + 2ull * sms * v.rows;
    rows = aligned(begin), ml = aligned(rows + every * sizeof(int4)), o = aligned(ml + records * sizeof(float2)), end = o + records * head_dim * 4;
  }
};

}  // namespace
}  // namespace bcp

using namespace bcp;

extern "C" int bcp_kv_attend_shared_workspace(const bcp_kv_cache* cache, uint32_t n_q_heads, uint32_t max_seqs, uint64_t* bytes) {
  const char* call = "bcp_kv_attend_shared_workspace";
  uint64_t own = 0;
  if (int rc = bcp_kv_attend_workspace(cache, n_q_heads, max_seqs, &own)) return rc;
  const Variant v = variant_of(cache->format, cache->head_dim);
  uint32_t sms = 0;
  if (int rc = prepare(v, &sms)) return rc;
  const Layout at(own, v, sms, max_seqs, n_q_heads, cache->head_dim);
  if (at.records > 0x7fffffffull) return fail(BCP_ERR_CAPACITY, "%s: %u sequences of %u query heads are too many for one call", call, max_seqs, n_q_heads);
  *bytes = at.end;
  return BCP_OK;
}

extern "C" int bcp_kv_attend_shared(const bcp_kv_cache* c, const bcp_heads* q, const bcp_heads* out, float* lse, uint32_t n_seqs,
                                    const int32_t* prefix_table, int64_t prefix_stride, uint32_t prefix_width, const int32_t* prefix_lengths,
                                    const int32_t* starts, uint32_t n_prefixes, const int32_t* block_table, int64_t table_stride, uint32_t table_width,
                                    const int32_t* lengths, float scale, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* call = "bcp_kv_attend_shared";
  if (int rc = check_cache(call, c)) return rc;
  if (int rc = check_heads(call, "q", q, false, c->head_dim, n_seqs)) return rc;
  if (int rc = check_group(call, c, q->n_heads)) return rc;
  if (n_seqs > 0x7fffffffu || n_prefixes > 0x7fffffffu) return fail(BCP_ERR_INVALID, "%s: %u sequences, %u prefixes", call, n_seqs, n_prefixes);
  if (n_prefixes && (!prefix_table || !prefix_lengths || !starts || prefix_stride < 0 || (n_prefixes > 1 && prefix_stride < int64_t(prefix_width))))
    return fail(BCP_ERR_INVALID, "%s: prefix_table, prefix_lengths or starts is NULL, or rows of the table overlap", call);
  if (!(scale == scale) || scale - scale != 0.f) return fail(BCP_ERR_INVALID, "%s: scale is not a finite number", call);
  uint64_t own = 0;
  if (int rc = bcp_kv_attend_workspace(c, q->n_heads, n_seqs, &own)) return rc;
  if (!n_prefixes || !n_seqs)
    return attend(call, c, q, out, lse, n_seqs, block_table, table_stride, table_width, lengths, scale, 0, workspace, workspace_bytes, nullptr, true, stream);
  if (q->type == BCP_F32 || (!is_8bit(c->format) && q->type != c->format) || !rows_aligned(q, 8))
    return fail(BCP_ERR_MISMATCH, "%s: queries of 16 bits, of the cache's type unless that has 8, whose rows start on 8-byte boundaries expected", call);
  const Variant v = variant_of(c->format, c->head_dim);
  uint32_t sms = 0;
  if (int rc = prepare(v, &sms)) return rc;
  const Layout at(own, v, sms, n_seqs, q->n_heads, c->head_dim);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return fail(BCP_ERR_INVALID, "%s: workspace is NULL or not 16-byte aligned", call);
  if (workspace_bytes < at.end)
    return fail(BCP_ERR_CAPACITY, "%s: a workspace of %llu bytes, %llu needed", call, (unsigned long long)workspace_bytes, (unsigned long long)at.end);
  const uint32_t group = q->n_heads / c->n_heads;
  PrefixArgs a = {};
  const uint64_t capacity = uint64_t(prefix_width) * c->page_size;
  a.capacity = uint32_t(capacity < 0x7fffff00u ? capacity : 0x7fffff00u);
  // rows and steps are counted in 32 bits
  const uint64_t tiles = (uint64_t(n_seqs) * group) / v.rows + n_prefixes, steps = a.capacity / v.tokens + 1;
  if (at.records > 0x7fffffffull || uint64_t(n_seqs) * group > 0x7fffffffull || tiles * c->n_heads > 0x7fffffffull / steps)
    return fail(BCP_ERR_CAPACITY, "%s: %u sequences over %u prefixes of up to %u tokens are too many for one call", call, n_seqs, n_prefixes, a.capacity);
  a.k = c->k, a.v = c->v, a.k_scale = c->k_scale, a.v_scale = c->v_scale;
  a.page_stride = uint32_t(c->page_stride), a.head_stride = uint32_t(c->head_stride), a.token_stride = uint32_t(c->token_stride);
  a.n_pages = c->n_pages, a.n_heads = c->n_heads, a.head_dim = c->head_dim;
  a.page_size = FastDiv(c->page_size);
  a.status = c->status;
  a.q = q->data, a.q_token = q->token_stride, a.q_head = q->head_stride;
  a.q_is_bf16 = q->type == BCP_BF16, a.n_seqs = n_seqs, a.n_groups = n_prefixes, a.group = FastDiv(group);
  a.table = prefix_table, a.table_stride = prefix_stride;
  a.lengths = prefix_lengths, a.starts = starts;
  a.scale_log2 = scale * kLog2e;
  char* const w = static_cast<char*>(workspace);
  a.rows = reinterpret_cast<int4*>(w + at.rows), a.ml = reinterpret_cast<float2*>(w + at.ml), a.o = reinterpret_cast<float*>(w + at.o);
  const Prior prior = {a.rows, a.ml, a.o, c->head_dim, 2 * v.rows, uint32_t(at.records), sms};
  // the second call's arguments are looked at before the first kernel is launched
  if (int rc = attend(call, c, q, out, lse, n_seqs, block_table, table_stride, table_width, lengths, scale, 0, workspace, own, &prior, false, stream))
    return rc;
  const uint64_t most = tiles * c->n_heads * steps;
  BCP_CUDA(launch_early(v.kernel, uint32_t(most < sms ? most : sms), v.threads, v.smem, static_cast<cudaStream_t>(stream), a));
  return attend(call, c, q, out, lse, n_seqs, block_table, table_stride, table_width, lengths, scale, 0, workspace, own, &prior, true, stream);
}

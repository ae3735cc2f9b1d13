// Attention of groups of sequences over the prefix that each group shares, computed once for all of them.
//
// Mathematics.  The query rows of a group under one cache head, (sequence, query head) by (sequence, query head), are the rows of S = Q K^T and O = P V
// with P = exp2(c S - m), c = scale log2 e.  m is a row's reference: when a score exceeds it by more than 8, the row's sums are brought to the new
// one.  What is left of the prefix are records (o, m, l) a row; the attention over the sequences' own tokens (kv_attend.cu) leaves one more, and a third
// kernel joins a row's records.
//
// Both products are tcgen05.mma with 128 rows.  A CTA has two streams, each with 128 rows whose scores and output lie in tensor memory (one stream with more
// than 128 dimensions): with more than 128 rows in a tile both take every 128 tokens, else they take turns with the same rows.  Two threads have half of a row's
// scores each (one thread a row: 3.5 us for a tile of both streams, two: 2.9, bfloat16).  Weights go back to tensor memory in place of the scores and are the first
// operand of the second product from there.  Over bfloat16 and 8-bit caches a weight is the sum of two bfloat16 numbers (2^-16 of it), as one alone would be
// rounded as coarsely as the result; 8-bit values are widened to bfloat16, keys to binary16, both exactly, the value's scale goes into the weight.  Over binary16
// caches a weight is one binary16 number (2^-11).
//
// Tokens come as boxes of a tensor map (pages of a multiple of eight tokens) or by 16-byte asynchronous copies (other pages, the end of a prefix) into a ring
// of tiles; a warp for each stream issues its products, the products of one stream behind those of the other: side by side both end late, and both streams
// make weights, then wait, at the same time (256 sequences over 32,768 tokens, binary16, without own tokens: 164 us, 181 side by side).
//
// Split.  The tiles of all groups, cache heads and 256 rows form one line that is cut into as many equal parts as there are SMs, so a part
// is one or two stretches of a unit.  The kernel of the own tokens needs nothing of this one and starts while it ends.
//
// What bounds it: the chain of a tile.  Scores of 128 x 128, their largest, the exchange between a row's two threads, 64 exponentials a thread in two halves, products:
// 2.9 us for both streams with weights of two numbers and 2.4 with one, where the tensor cores need 1.56 and 1.04, exponentials 1.04, and the tile's 64 KB 1.5 at the
// copy bandwidth.  8-bit caches wait for the warps that widen them (about 2.9 us a tile of 128 tokens).  Measured on one B200, all three kernels, 32 / 8 heads of 128,
// among other calls with inputs that change (in brackets: the same call over and over in a CUDA graph): 5 drafted tokens over 4096, bfloat16: 15.7 us (15.4; without
// prefix and own tokens the three launches take 7.5); 64 sequences over 32,768 and up to 600 own tokens, bfloat16: 95 us (88); 70 over 5 prefixes of up to 9000, e4m3,
// pages of 24: 107 us (97); 256 over 32,768, binary16: 254 us (217).  With 256 dimensions, 64 sequences over 16,384: bfloat16 136 us, binary16 127, e4m3 160.
#include <cuda.h>

#include <atomic>
#include <mutex>

#include "attend.cuh"
#include "tma_ptx.cuh"

namespace bcp {
namespace {

constexpr uint32_t kRows = 128;             // rows of a stream
constexpr uint32_t kMeta = 16;              // tiles whose masks and scales are kept
constexpr uint32_t kMostNs = BCP_WAIT_NS;   // a wait that takes longer gives up, unless the host has said otherwise
std::atomic<uint32_t> g_limit{kMostNs};
constexpr uint32_t kDrainNs = 20000000u;    // copies under way have landed after that

struct PrefixArgs {
  CUtensorMap k_map, v_map;  // the cache as [page][head][token][element], boxes of `block` tokens
  uint32_t block;            // 0: none
  const void *k, *v;
  const float *k_scale, *v_scale;
  uint32_t page_stride, head_stride, token_stride;
  uint32_t n_pages, n_heads, head_dim;
  FastDiv page_size;
  uint32_t* status;
  const void* q;
  int64_t q_token, q_head;
  uint32_t q_is_bf16, q_wide, n_seqs, n_groups;  // q_wide: its rows start on 16-byte boundaries
  FastDiv group;  // query heads of a cache head
  const int32_t* table;
  int64_t table_stride;
  uint32_t capacity;
  const int32_t *lengths, *starts;
  float scale_log2;
  int4* rows;   // of each row: its first record, the next part's, parts, from a record to the other one of the same part (0: it has one)
  float2* ml;   // reference and denominator of each record: l = sum exp2(s - m)
  float* o;     // its sums, o = sum exp2(s - m) v
  uint32_t limit;  // nanoseconds of a wait
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
  // Warps that bring tokens; 8-bit ones have to be widened by them, too.  Microseconds with four on every tile and with four for keys and four for values (e4m3, pages of
  // 24): 70 sequences over 5 prefixes of up to 9000 tokens 98.7 and 96.7, 5 sequences over one 37.0 and 35.9, 64 over one 76.0 and 79.2; pages of 7 102.4, 37.9, 77.7
  // and 98.9, 36.6, 80.0.
  static constexpr uint32_t LOADERS = quant && STREAMS == 2 ? 8 : 4;
  static constexpr uint32_t META = quant ? 16 + TOK * 8 + 16 : 16;
  static constexpr uint32_t NMETA = quant ? 8 : kMeta;         // (more than the tiles that can be on their way past one that is still worked on)
  static constexpr uint32_t SLOTS = DP == 64 ? 8 : quant ? 3 : 5;  // tiles in 16 bits: what shared memory has room for
  static constexpr uint32_t AHEAD = quant ? RAWS - 1 : 3;    // copies of so many tiles are under way
  static constexpr uint32_t SMEM = STREAMS * Q + SLOTS * TILE + RAWS * RAW + NMETA * META + 8 * (2 * SLOTS + NMETA + 7 * STREAMS + 4 * RAWS) + STREAMS * 1024 + 48;
  // two warpgroups for each stream (a thread has half of a row's scores), one that copies, one of whose warps issue the products
  static constexpr uint32_t WARPS = 8 * STREAMS + LOADERS + 4, THREADS = 32 * WARPS, COLS = TOK / 2;
  // Registers a thread: at launch, and after the groups have been given theirs (their sum is at most the launch's).  With one stream there are enough for all.
  static constexpr uint32_t REGS = quant ? 72 : 80, REGS_ROWS = quant ? 80 : 88, REGS_COPY = quant ? 64 : 72, REGS_PRODUCT = 56;
  static_assert(4 * REGS_ROWS + LOADERS / 4 * REGS_COPY + REGS_PRODUCT <= (5 + LOADERS / 4) * REGS || STREAMS == 1, "registers of the launch");
  static constexpr uint32_t S0 = 0, O0 = STREAMS * TOK;      // columns of tensor memory
  static_assert(O0 + STREAMS * DP <= 512, "tensor memory");
  static_assert(SMEM <= 232448, "shared memory");
  static_assert(AHEAD < SLOTS || quant, "copies that wait for a tile's place");
};

// ------------------------------------------------------------------------------ instructions
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {  // without waiting
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok;
}
// What a wait may take, and the word that says that one has taken longer.
struct Limit {
  volatile uint32_t* stop;
  const uint32_t& ns;
};
// Sleeps until the phase is complete, for four microseconds (measured; the hardware's choice) at most; with a limit of zero it only looks.  (To be told how long to sleep
// takes a register at every wait.  64 sequences over 32,768 tokens and 5 over 4096: 88.5 and 15.4 us, with a constant 89.1 and 15.7, with an argument 92.8 and 16.1.)
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity, const Limit& limit) {
  return limit.ns ? mbar_try_wait(bar, parity) : bar_test(bar, parity);
}
// False, in all lanes of a warp, if the wait ran out here or in another warp.
__device__ __forceinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, const Limit& limit) {
  const uint64_t begin = global_timer_ns();
  while (!bar_try(bar, parity, limit)) {
    if (*limit.stop) return false;
    if (global_timer_ns() - begin > limit.ns) {
      *limit.stop = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, const Limit& limit) {
  return __all_sync(0xffffffffu, bar_try(bar, parity, limit) || bar_wait_slow(bar, parity, limit));
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
__device__ __forceinline__ void tmem_load32(uint32_t at, float* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
      "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]),
        "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]),
        "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(at));
}
// Values are used only behind the wait for their loads.
__device__ __forceinline__ void loaded32(float* r) {
  asm volatile("" : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]), "+f"(r[16]), "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]), "+f"(r[24]), "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31]));
}
__device__ __forceinline__ void loaded16(float* r) {
  asm volatile("" : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]));
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
               "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]),
                 "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
               : "r"(at));
}

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nadd.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float largest(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float minus_upper(float x) { return __uint_as_float((__float_as_uint(x) & 0xffff0000u) ^ 0x80000000u); }
// A number that all lanes have, in a form in which the compiler knows that they do: it then lies in a uniform register, where the operands of
// tcgen05 instructions have to be, and branches on it keep the warp together.
__device__ __forceinline__ uint32_t same(uint32_t x) { return __reduce_or_sync(0xffffffffu, x); }
__device__ __forceinline__ bool elected() {
  uint32_t yes;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
  return yes;
}
template <uint32_t N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <uint32_t N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Shared-memory operands in rows of 128 bytes (64 elements), eight rows a swizzled block of 1024 bytes, blocks of rows one after the other; a
// descriptor's lower half has the address and, for values (whose sum runs over rows), the bytes from 64 columns to the next; its upper half is the same for all.
// Products follow one another at 64 cycles, about the time that one thread needs to issue one with all its numbers at hand: they are unrolled, and each
// adds a constant to the lower half.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t apart) { return (at >> 4 & 0x3fff) | (apart >> 4) << 16; }
constexpr uint32_t kUpper = 1024 >> 4 | 1u << 14 | 2u << 29;
// kind::f16 with binary32 sums, 128 rows, n columns; both operands bfloat16 or both binary16; the second one's rows along the sum or not
__host__ __device__ constexpr uint32_t product(bool bf16, bool second_by_rows, uint32_t n) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (second_by_rows ? 1u << 16 : 0u) | (n >> 3) << 17 | (kRows >> 4) << 24;
}
// (Only the instruction itself is left to one lane: the numbers around it are made by the whole warp.)
__device__ __forceinline__ void mma_shared(bool chosen, uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add) {
  asm volatile("{\n.reg .pred p, q;\n.reg .b64 x, y;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %6, 0;\nmov.b64 x, {%1, %5};\nmov.b64 y, {%2, %5};\n"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(what), "r"(uint32_t(add)), "n"(kUpper),
               "r"(uint32_t(chosen))
               : "memory");
}
__device__ __forceinline__ void mma_tensor(bool chosen, uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add) {
  asm volatile("{\n.reg .pred p, q;\n.reg .b64 y;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %6, 0;\nmov.b64 y, {%2, %5};\n"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(what), "r"(uint32_t(add)), "n"(kUpper),
               "r"(uint32_t(chosen))
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

__device__ __forceinline__ void copies_wait_all_but(uint32_t n) {
  switch (n) {
    case 0: copies_wait<0>(); break;
    case 1: copies_wait<1>(); break;
    case 2: copies_wait<2>(); break;
    default: copies_wait<3>(); break;
  }
}

// `block` tokens of 64 (16-bit) or all (8-bit) elements, from element x on
__device__ __forceinline__ void box_load(uint32_t to, const CUtensorMap* map, uint32_t x, uint32_t token, uint32_t head, uint32_t page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to), "l"(map),
               "r"(x), "r"(token), "r"(head), "r"(page), "r"(bar)
               : "memory");
}

__device__ __forceinline__ void store8(float* to, const float* x) {  // a whole sector of memory
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]),
               "f"(x[6]), "f"(x[7])
               : "memory");
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
__global__ void __launch_bounds__(Shape<FMT, DP>::THREADS, 1) bcp_kv_prefix_kernel(const __grid_constant__ PrefixArgs a) {
  typedef Shape<FMT, DP> S;
  extern __shared__ __align__(1024) unsigned char smem[];  // swizzled blocks lie on 1024-byte boundaries
  const uint32_t tid = threadIdx.x, warp = same(tid >> 5), lane = tid & 31;
  const uint32_t base = uint32_t(__cvta_generic_to_shared(smem));
  const uint32_t q_at = base, ring = q_at + S::STREAMS * S::Q, raw = ring + S::SLOTS * S::TILE, meta = raw + S::RAWS * S::RAW;
  unsigned char* const meta_ptr = smem + (meta - base);
  const uint32_t bars = meta + S::NMETA * S::META;
  const uint32_t full = bars, empty = full + 8 * S::SLOTS, described = empty + 8 * S::SLOTS, q_full = described + 8 * S::NMETA, s_full = q_full + 8 * S::STREAMS,
                 p_full = s_full + 8 * S::STREAMS, o_full = p_full + 16 * S::STREAMS, drained = o_full + 8 * S::STREAMS, turn = drained + 8 * S::STREAMS, raw_full = turn + 8 * S::STREAMS;
  uint32_t* const words = reinterpret_cast<uint32_t*>(smem + (raw_full + 32 * S::RAWS + S::STREAMS * 1024 - base));  // tensor memory, stop, found[8]
  volatile float* const swap = reinterpret_cast<volatile float*>(smem + (raw_full + 32 * S::RAWS - base));  // [stream][half][row]
  volatile uint32_t* const stop = words + 1;
  const Limit limit = {stop, a.limit};
  uint32_t* const found = words + 2;
  uint64_t* const totals = reinterpret_cast<uint64_t*>(smem);  // before the tiles come

  if (base & 1023) {  // no room is left to move them there
    wait_for_previous();
    if (tid == 0) raise(a.status, BCP_TIMED_OUT);
    return;
  }
  if (warp == S::WARPS - 4) tmem_alloc(uint32_t(__cvta_generic_to_shared(words)));
  if (tid == 0) {
    for (uint32_t i = 0; i < S::SLOTS; ++i) mbar_init(full + 8 * i, kRows), mbar_init(empty + 8 * i, 2);
    for (uint32_t i = 0; i < S::NMETA; ++i) mbar_init(described + 8 * i, kRows);
    for (uint32_t i = 0; i < S::STREAMS; ++i)
      mbar_init(q_full + 8 * i, 2 * kRows), mbar_init(s_full + 8 * i, 1), mbar_init(p_full + 16 * i, 2 * kRows), mbar_init(p_full + 16 * i + 8, 2 * kRows), mbar_init(o_full + 8 * i, 1), mbar_init(drained + 8 * i, 1), mbar_init(turn + 8 * i, 1);
    for (uint32_t i = 0; i < 4 * S::RAWS; ++i) mbar_init(raw_full + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *static_cast<volatile uint32_t*>(words);
  wait_for_previous();
  next_may_start();  // the kernel of the own tokens, which needs nothing of this one, but what came before
  // ---- the line, and this CTA's part of it
  const uint32_t n_q_heads = a.n_heads * a.group.d;
  const uint32_t run = (a.n_groups + S::THREADS - 1) / S::THREADS;
  const uint32_t run0 = min(tid * run, a.n_groups), run1 = min(run0 + run, a.n_groups);
  // (The host has made sure that the steps of groups without common sequences fit 32 bits; what starts says may be anything.)
  uint64_t mine64 = 0;
  for (uint32_t g = run0; g < run1; ++g) {
    const Group x = group_of<S>(a, g);
    mine64 += uint64_t(x.steps) * x.tiles * a.n_heads;
  }
  uint64_t before64 = mine64;
#pragma unroll
  for (uint32_t o = 1; o < 32; o <<= 1) {
    const uint64_t x = __shfl_up_sync(0xffffffffu, before64, o);
    if (lane >= o) before64 += x;
  }
  if (lane == 31) totals[warp] = before64;
  if (tid == 0) *stop = 0;
  __syncthreads();
  uint64_t all64 = 0;
  before64 -= mine64;
  for (uint32_t w = 0; w < S::WARPS; ++w) {
    if (w < warp) before64 += totals[w];
    all64 += totals[w];
  }
  const bool sound = all64 <= 0x7fffffffull;
  const uint32_t all = sound ? uint32_t(all64) : 0, mine = uint32_t(mine64), before = uint32_t(before64);
  Cuts cuts;
  if (all) cuts.cut(all, gridDim.x);
  // Rows without a prefix have no records: two warps that have nothing else to do look at all of them.
  auto look_at_rows = [&]() {
    const uint32_t id = blockIdx.x * 64 + (tid & 63), step = gridDim.x * 64;
    for (uint32_t b = id; b < a.n_seqs; b += step) {
      uint32_t lo = 0, hi = a.n_groups;  // the last group that starts at or before b
      while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (a.starts[mid] <= int32_t(b)) lo = mid + 1; else hi = mid;
      }
      bool has = false;
      if (lo) {
        const Group x = group_of<S>(a, lo - 1);
        has = sound && b >= x.first && b - x.first < x.rows / a.group.d && x.steps;
      }
      if (!has)
        for (uint32_t h = 0; h < n_q_heads; ++h) a.rows[uint64_t(b) * n_q_heads + h] = make_int4(0, 0, 0, 0);
    }
    if (a.status)
      for (uint32_t g = id; g < a.n_groups; g += step)
        if (a.lengths[g] > int32_t(a.capacity) || a.starts[g] < 0 || a.starts[g + 1] < a.starts[g] || a.starts[g + 1] > int32_t(a.n_seqs))
          raise(a.status, BCP_BAD_LENGTH);
  };
  if (!all || blockIdx.x >= cuts.parts) {
    if (warp >= S::WARPS - 2) look_at_rows();
    if (warp == S::WARPS - 4) tmem_free(tmem);
    return;
  }
  const uint32_t s0 = cuts.begin(blockIdx.x), n_steps = cuts.begin(blockIdx.x + 1) - s0;
  if (s0 >= before && s0 < before + mine) {
    uint32_t pre = before, g = run0;
    for (;; ++g) {
      const Group x = group_of<S>(a, g);
      const uint32_t n = x.steps * x.tiles * a.n_heads;
      if (s0 < pre + n) {
        found[0] = g, found[1] = (s0 - pre) / x.steps, found[2] = (s0 - pre) % x.steps;
        found[3] = x.first, found[4] = x.rows, found[5] = x.len, found[6] = x.steps, found[7] = x.tiles;
        break;
      }
      pre += n;
    }
  }
  __syncthreads();
  Place at;
  at.g = found[0], at.u = found[1], at.step = found[2];
  at.group.first = found[3], at.group.rows = found[4], at.group.len = found[5], at.group.steps = found[6], at.group.tiles = found[7];

  uint32_t left = n_steps;
  if (warp < 8 * S::STREAMS) {
    // ================================================================ a stream's rows
    if constexpr (S::STREAMS == 2) more_registers<S::REGS_ROWS>();
    const uint32_t stream = warp >> 3, part = warp >> 2 & 1, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t lanes = tmem + (quarter << 21);  // this warp's 32 rows
    const uint32_t s_at = lanes + S::S0 + stream * S::TOK + part * S::COLS, o_at = lanes + S::O0 + stream * DP;
    uint32_t n_scores = 0, n_ends = 0, tile0 = 0;
    const float scale = fabsf(a.scale_log2);
    constexpr float kLeast = 0x1p-126f;  // a factor is not 0, so that a masked score stays below all others; any score times this counts as 0
    bool ok = true;
    // The two warps of 32 rows wait for each other; the two threads of a row see each other's number.  That wait has no limit, so a warp that gives up arrives
    // once more, below, and the other must not wait for it twice: behind the meeting over a tile's scores it gets no further than the wait for the next products,
    // which need the weights of both; where one meeting follows another without that, it looks whether a wait has run out (together).
    const uint32_t pair = 1 + 4 * stream + quarter;
    auto meet = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory"); };
    auto together = [&]() { return !__any_sync(0xffffffffu, *stop); };
    auto other = [&](float mine) {
      swap[(stream * 2 + part) * kRows + row] = mine;
      meet();
      return swap[(stream * 2 + 1 - part) * kRows + row];
    };
    while (left && ok) {
      const uint32_t n = min(at.group.steps - at.step, left);
      const uint32_t h = at.u / at.group.tiles, row0 = (at.u - h * at.group.tiles) * S::ROWS, rows = min(at.group.rows - row0, S::ROWS);
      const bool both = rows > kRows;  // the streams have rows of their own, else they take turns
      const uint32_t r = row0 + (both ? stream * kRows : 0) + row;
      const bool live = r < row0 + rows, work = __any_sync(0xffffffffu, live);
      const uint32_t seq = a.group.div(live ? r : 0), head = h * a.group.d + (live ? r : 0) - seq * a.group.d, b = at.group.first + seq;
      const bool any = both || stream < n;  // has tiles here
      float factor = scale;
      if (any) {
        // The queries into shared memory, neighbouring lanes on neighbouring chunks of a row; a warp has 16 of its 32 rows, the other part's the rest.  Over 8-bit
        // caches a power of two brings a row's largest element into [1, 2), so that it fits binary16.
        const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;  // the scale's sign goes into the query
        const int64_t from = live ? b * a.q_token + head * a.q_head : -1;
        constexpr uint32_t kChunks = DP / 8, kTogether = 32 / kChunks, kTurns = 16 / kTogether, kAtOnce = 8;
        const uint32_t c = lane % kChunks, mine = lane / kChunks;
#pragma unroll 1
        for (uint32_t i0 = 0; i0 < kTurns; i0 += kAtOnce) {
          uint4 x[kAtOnce];
#pragma unroll
          for (uint32_t i = 0; i < kAtOnce; ++i) {
            x[i] = make_uint4(0, 0, 0, 0);
            const int64_t at_row = __shfl_sync(0xffffffffu, from, part * 16 + (i0 + i) % kTurns * kTogether + mine);
            if (at_row >= 0 && 8 * c < a.head_dim && i0 + i < kTurns) {
              const char* const p = static_cast<const char*>(a.q) + (at_row + 8 * c) * 2;
              if (a.q_wide) {
                x[i] = *reinterpret_cast<const uint4*>(p);
              } else {
                const uint2 u = *reinterpret_cast<const uint2*>(p), v = *reinterpret_cast<const uint2*>(p + 8);
                x[i] = make_uint4(u.x, u.y, v.x, v.y);
              }
            }
          }
#pragma unroll
          for (uint32_t i = 0; i < kAtOnce; ++i) {
            if (i0 + i >= kTurns) break;
            const uint32_t r = quarter * 32 + part * 16 + (i0 + i) * kTogether + mine;
            if constexpr (S::quant) {
              auto size = [&](uint32_t w) { return max(__float_as_uint(query_at(&w, 0, a.q_is_bf16)) & 0x7fffffffu, __float_as_uint(query_at(&w, 1, a.q_is_bf16)) & 0x7fffffffu); };
              uint32_t top = max(max(size(x[i].x), size(x[i].y)), max(size(x[i].z), size(x[i].w)));
#pragma unroll
              for (uint32_t o = 1; o < kChunks; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
              const uint32_t e = top >> 23 == 254 ? 253 : top >> 23;
              float up = 1.f, back = 1.f;
              if (e >= 1 && e <= 253) up = __uint_as_float((254 - e) << 23), back = __uint_as_float(e << 23);
              auto word = [&](uint32_t w) { return pack16<false>(query_at(&w, 0, a.q_is_bf16) * up, query_at(&w, 1, a.q_is_bf16) * up); };
              x[i] = make_uint4(word(x[i].x), word(x[i].y), word(x[i].z), word(x[i].w));
              // both threads of the row get to know it
              if (c < 2) swap[(stream * 2 + c) * kRows + r] = back;
            }
            if (8 * c < a.head_dim)
              shared_store16(q_at + stream * S::Q + r * 128 + (c >> 3) * (kRows * 128) + ((c & 7 ^ r & 7) << 4), x[i].x ^ flip, x[i].y ^ flip, x[i].z ^ flip, x[i].w ^ flip);
          }
        }
        to_async_proxy();
        bar_arrive(q_full + 8 * stream);
        if constexpr (S::quant) {
          meet();
          ok = together();
          if (!ok) break;
          factor *= swap[(stream * 2 + part) * kRows + row];
        }
      }
      factor = fmaxf(factor, kLeast);

      float ref = kNone, l = 0.f, top_scale = 0.f, unit = 1.f;  // unit: what the values' scales are multiplied by
      bool first = true;
      const uint32_t step = both ? 1 : S::STREAMS;
      for (uint32_t t = both ? 0 : stream; t < n; t += step) {
        const uint32_t m_slot = (tile0 + t) % S::NMETA;
        const unsigned char* const about = meta_ptr + m_slot * S::META;
        ok = bar_wait(described + 8 * m_slot, (tile0 + t) / S::NMETA & 1, limit) && bar_wait(s_full + 8 * stream, n_scores & 1, limit);
        if (!ok) break;
        ++n_scores;
        tmem_after();
        if (work) {
          // 32 scores into registers; 8-bit keys: times their scales; masked ones below all others
          float x[32];
          auto read = [&](uint32_t c) {
            tmem_load32(s_at + 32 * c, x);
            tmem_load_wait();
            loaded32(x);
            const uint32_t column = part * S::COLS + 32 * c;
            if constexpr (S::quant) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 ks = *reinterpret_cast<const float4*>(about + 16 + 4 * (column + i));
                x[i] *= ks.x, x[i + 1] *= ks.y, x[i + 2] *= ks.z, x[i + 3] *= ks.w;
              }
            }
            const uint32_t mask = *reinterpret_cast<const uint32_t*>(about + column / 8);
            if (mask != 0xffffffffu) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(mask >> i & 1)) x[i] = -INFINITY;
            }
          };
          // the largest; the last 32 stay in registers
          float top = -INFINITY;
#pragma unroll
          for (uint32_t c = 0; c < S::COLS / 32; ++c) {
            read(c);
            float tops[4] = {top, x[0], x[1], x[2]};
#pragma unroll
            for (uint32_t i = 2; i < 32; i += 2) tops[i / 2 % 4] = largest(tops[i / 2 % 4], x[i], x[i + 1]);
            top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
          }
          top = fmaxf(top, other(top)) * factor;
          float down = 1.f;
          if (top > ref + 8.f) down = exp2_fast(ref - top), ref = top, l *= down;
          if constexpr (S::quant) {
            // Weights times scales must neither overflow in the sums nor vanish: where scales beyond 2^60 turn up all are multiplied by 2^-40, while none
            // is above 2^-40 by 2^60.
            const float4 w = *reinterpret_cast<const float4*>(about + 16 + S::TOK * 8);
            top_scale = fmaxf(top_scale, fmaxf(fmaxf(w.x, w.y), fmaxf(w.z, w.w)));
            const float next = top_scale > 0x1p60f ? 0x1p-40f : top_scale < 0x1p-40f ? 0x1p60f : 1.f;
            if (next != unit) down *= next / unit, unit = next;
          }
          if (!first && __any_sync(0xffffffffu, down != 1.f)) {
#pragma unroll 1
            for (uint32_t c = 16 * part; c < a.head_dim; c += 32) {
              float z[16];
              uint32_t y[16];
              tmem_load16(o_at + c, z);
              tmem_load_wait();
              loaded16(z);
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(z[i] * down);
              tmem_store16(o_at + c, y);
            }
          }
          // the weights; the products with the last 32 columns of either part begin while those with the others are made
          constexpr float kLift = S::split ? 0.f : 6.f;  // binary16 weights underflow below 2^-24: lifted by 2^6 that is 2^-30
          const float2 factors = make_float2(factor, factor), less = make_float2(kLift - ref, kLift - ref);
#pragma unroll
          for (uint32_t j = 0; j < S::COLS / 32; ++j) {
            const uint32_t c = S::COLS / 32 - 1 - j;
            if (j) read(c);
            float2 sum[4] = {};  // four, so that no addition waits for the one before it
            uint32_t y[16], rest[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float2 e = fma2(make_float2(x[i], x[i + 1]), factors, less);
              float2 p = make_float2(exp2_fast(e.x), exp2_fast(e.y));
              sum[i / 2 & 3] = add2(sum[i / 2 & 3], p);
              if constexpr (S::quant) {
                const float2 vs = *reinterpret_cast<const float2*>(about + 16 + S::TOK * 4 + 4 * (part * S::COLS + 32 * c + i));
                p = mul2(p, mul2(vs, make_float2(unit, unit)));
              }
              if constexpr (S::split) {
                // the upper half as it stands, and what remains, made positive by 2^-20 of the weight: the products of both with an infinite value are
                // that infinity
                y[i / 2] = upper_halves(p.x, p.y);
                const float2 r = fma2(p, make_float2(1.f + 0x1p-20f, 1.f + 0x1p-20f), make_float2(minus_upper(p.x), minus_upper(p.y)));
                rest[i / 2] = pack16<true>(r.x, r.y);
              } else {
                y[i / 2] = pack16<false>(p.x, p.y);
              }
            }
            sum[0] = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
            l += sum[0].x + sum[0].y;
            tmem_store16(s_at + 32 * c, y);
            if constexpr (S::split) tmem_store16(s_at + 32 * c + 16, rest);
            tmem_store_wait();
            tmem_before();
            bar_arrive(p_full + 16 * stream + 8 * j);
          }
        } else {
          tmem_before();
#pragma unroll
          for (uint32_t j = 0; j < S::COLS / 32; ++j) bar_arrive(p_full + 16 * stream + 8 * j);
        }
        first = false;
      }
      tile0 += n;
      if (!ok) break;
      // ---- the record
      const bool whole = at.step == 0 && n == at.group.steps;
      const uint32_t every = a.n_seqs * n_q_heads, place = s0 + n_steps - left;
      uint32_t record = b * n_q_heads + head + (!both && stream ? every : 0);
      if (!whole) record = 2 * every + (2 * blockIdx.x + (place != s0)) * S::ROWS + stream * kRows + row;
      if (any) {
        ok = bar_wait(o_full + 8 * stream, n_ends & 1, limit);
        if (!ok) break;
        ++n_ends;
        tmem_after();
        if (work) {
#pragma unroll 1
          for (uint32_t c = 16 * part; c < a.head_dim; c += 32) {
            float x[16];
            tmem_load16(o_at + c, x);
            tmem_load_wait();
            loaded16(x);
            if (live) {
              float* const to = a.o + uint64_t(record) * a.head_dim + c;
              store8(to, x), store8(to + 8, x + 8);
            }
          }
          l += other(l);
          if constexpr (S::quant) {  // what the next queries bring is written only when this has been read
            ok = together();
            if (!ok) break;
            meet();
            ok = together();
            if (!ok) break;
          }
        }
        tmem_before();
      }
      if (live && part == 0) {
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
    if (!ok) asm volatile("bar.arrive %0, 64;" ::"r"(pair) : "memory");
  } else if (warp < 8 * S::STREAMS + S::LOADERS) {
    // ================================================================ copies of keys and values
    if constexpr (S::STREAMS == 2) fewer_registers<S::REGS_COPY>();
    // Four warps share a tile.  With eight (8-bit caches, whose tiles have to be widened) four bring keys and four bring values.
    const uint32_t w = warp - 8 * S::STREAMS & 3;
    constexpr bool kTeams = S::LOADERS == 8;
    const bool keys_team = warp - 8 * S::STREAMS < 4;
    constexpr uint32_t kEach = S::TOK / 4;                        // rows of a tile that a warp brings
    constexpr uint32_t kChunks = DP * (S::quant ? 1 : 2) / 16;    // 16-byte chunks of a row
    constexpr uint32_t kTogether = 32 / kChunks, kTurns = kEach / kTogether;
    constexpr uint32_t kAll = kEach == 32 ? 0xffffffffu : (1u << (kEach & 31)) - 1;
    const uint32_t my_row = lane / kChunks, chunk = lane % kChunks;
    const bool inside = chunk * 16 < a.head_dim * (S::quant ? 1u : 2u);
    uint32_t item = 0, tile0 = 0, brought = 0;  // item: of the ring; brought: tiles whose keys have been seen
    uint32_t queued = 0, landed = 0;            // of this team's items: those under way or landed, those landed
    uint32_t items[2] = {0, 0};                 // with teams: the last two of them that are queued, the newer one first
    uint32_t kinds = 0, tile_landed = 0;        // a bit for each queued item: it is keys; tiles whose keys have landed
    uint32_t boxes = 0, phases = 0;             // a bit for each queued item: it comes in boxes; for each place of 8-bit tiles: the parity of its barrier
    auto stage_of = [&](uint32_t n) { return !S::quant ? 0 : kTeams ? keys_team ? n & 1 : 2 : n % S::RAWS; };  // of the n-th queued item
    const uint32_t ahead = kTeams ? keys_team : S::AHEAD;
    // Where this warp's tokens of a tile lie (a row a lane); the page of the next tile's is looked up ahead.
    int32_t page = -1, page_of[2] = {-1, -1};
    bool inside_prefix = false;
    uint32_t off = 0, off_of[2] = {0, 0}, alive_of[2] = {0, 0};
    const int64_t v_from_k = static_cast<const char*>(a.v) - static_cast<const char*>(a.k);
    bool ok = true;

    // An 8-bit tile that has come in is widened into its place.
    auto land = [&]() {
      const uint32_t this_item = !kTeams ? landed : queued - landed > 1 ? items[1] : items[0];
      const uint32_t slot = this_item % S::SLOTS, at_slot = ring + slot * S::TILE;
      const bool keys = kinds >> (landed & 31) & 1;
      const uint32_t m_slot = tile_landed % S::NMETA;
      if constexpr (S::quant) {
        const uint32_t stage = stage_of(landed);
        if (boxes >> (landed & 31) & 1) {
          ok = ok && bar_wait(raw_full + 8 * (4 * stage + w), phases >> stage & 1, limit);
          phases ^= 1u << stage;
        }
        if (this_item >= S::SLOTS) ok = ok && bar_wait(empty + 8 * slot, this_item / S::SLOTS - 1 & 1, limit);
        const uint32_t from = raw + stage * S::RAW + (w * kEach + my_row) * a.head_dim + chunk * 16;
        if (inside && ok) {
#pragma unroll 2
          for (uint32_t i = 0; i < kTurns; ++i) {
            const uint32_t r = w * kEach + i * kTogether + my_row;
            const uint4 x = shared_load16(from + i * kTogether * a.head_dim);
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
        }
        if (keys) {  // the largest of the values' scales
          unsigned char* const about = meta_ptr + m_slot * S::META;
          float top = lane < kEach ? *reinterpret_cast<volatile float*>(about + 16 + S::TOK * 4 + (w * kEach + lane) * 4) : 0.f;
#pragma unroll
          for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          if (lane == 0) *reinterpret_cast<volatile float*>(about + 16 + S::TOK * 8 + w * 4) = top;
        }
        __syncwarp();  // the place of the 8-bit tile is read out, too
      }
      if (keys) bar_arrive(described + 8 * m_slot), ++tile_landed;
      to_async_proxy();
      bar_arrive(full + 8 * slot);
      ++landed;
    };
    auto look_up = [&](uint32_t pos0) {  // (nothing looks at what was loaded before it is used)
      const uint32_t pos = pos0 + w * kEach + (lane & (kEach - 1));
      page = -1, inside_prefix = pos < at.group.len;
      if (inside_prefix) {
        const uint32_t n = a.page_size.div(pos);
        off = pos - n * a.page_size.d;
        page = a.table[at.g * a.table_stride + n];
      }
    };
    // One loop with one piece of code for each thing to do: the warps that bring and those that weigh share the instruction cache.
    uint32_t n = 0, h = 0, early = 0, i = 0;
    bool at_end = false;
    while (ok) {
      if (!at_end && i == 2 * n) {  // the next stretch
        if (n) {
          tile0 += n, left -= n;
          advance<S>(at, a, n, left != 0);
        }
        if (left) {
          n = min(at.group.steps - at.step, left), h = at.u / at.group.tiles, i = 0;
          const uint32_t row0 = (at.u - h * at.group.tiles) * S::ROWS;
          early = min(n, min(at.group.rows - row0, S::ROWS) > kRows ? 1u : S::STREAMS);  // the keys of so many tiles come before values
          look_up(at.step * S::TOK);
        } else {
          at_end = true;
        }
      }
      if (at_end && landed == queued) break;
      const uint32_t slot = item % S::SLOTS, stage = stage_of(queued);
      bool land_now = at_end;
      if (!S::quant && !at_end && item >= S::SLOTS) {
        // copies that are under way go on to the products while this tile's place is still taken
        const uint32_t parity = item / S::SLOTS - 1 & 1;
        land_now = landed < queued && !__all_sync(0xffffffffu, bar_test(empty + 8 * slot, parity));
        if (!land_now) ok = bar_wait(empty + 8 * slot, parity, limit);
        if (!ok) break;
      }
      if (!land_now) {
        // An item of the stretch: the keys of the first tiles, then values and keys in turn, then the values that are left.
        const uint32_t j = i - early;
        const bool keys = i < early || (j < 2 * (n - early) && (j & 1));
        const uint32_t t = i < early ? i : keys ? early + j / 2 : j < 2 * (n - early) ? j / 2 : j - (n - early), tile = tile0 + t;
        if (keys) {
          if (uint32_t(page) >= a.n_pages) {
            if (inside_prefix) raise(a.status, BCP_BAD_PAGE);
            page = -1;
          }
          page_of[1] = page_of[0], off_of[1] = off_of[0], alive_of[1] = alive_of[0];
          page_of[0] = page, off_of[0] = off, alive_of[0] = __ballot_sync(0xffffffffu, page >= 0) & kAll;
          ++brought;
          unsigned char* const about = meta_ptr + tile % S::NMETA * S::META;
          if (lane == 0 && keys_team) {
            if (kEach == 32) reinterpret_cast<volatile uint32_t*>(about)[w] = alive_of[0];
            if (kEach == 16) reinterpret_cast<volatile uint16_t*>(about)[w] = uint16_t(alive_of[0]);
          }
        }
        if (kTeams && keys != keys_team) {
          if (keys && t + 1 < n) look_up((at.step + t + 1) * S::TOK);
          ++item, ++i;
          continue;
        }
        // values come behind the next tile's keys where the streams take turns
        const bool older = !keys && tile + 1 < brought;
        const int32_t my_page = older ? page_of[1] : page_of[0];
        const uint32_t my_off = older ? off_of[1] : off_of[0], alive = older ? alive_of[1] : alive_of[0];
        const uint32_t bar = S::quant ? raw_full + 8 * (4 * stage + w) : full + 8 * slot;
        const bool box = a.block && alive == kAll;
        if (box) {
          // a warp's tokens in boxes, each inside one page
          const CUtensorMap* const map = keys ? &a.k_map : &a.v_map;
          const uint32_t wide = S::quant ? 1 : (a.head_dim + 63) / 64;
          if (lane == 0) mbar_expect_tx(bar, kEach * (S::quant ? a.head_dim : 128 * wide));
          __syncwarp();
          const uint32_t to = S::quant ? raw + stage * S::RAW + (w * kEach + lane) * a.head_dim : ring + slot * S::TILE + (w * kEach + lane) * 128;
          if (lane < kEach && (lane & (a.block - 1)) == 0)
            for (uint32_t x = 0; x < wide; ++x) box_load(to + x * (S::TOK * 128), map, 64 * x, my_off, h, uint32_t(my_page), bar);
        } else {
          const uint64_t row = my_page >= 0 ? uint64_t(uint32_t(my_page)) * a.page_stride + uint64_t(h) * a.head_stride + uint64_t(my_off) * a.token_stride : 0;
          const char* const from = static_cast<const char*>(a.k) + (keys ? 0 : v_from_k);
          const uint32_t to = S::quant ? raw + stage * S::RAW + w * kEach * a.head_dim : ring + slot * S::TILE;
#pragma unroll 2
          for (uint32_t k = 0; k < kTurns; ++k) {
            const uint32_t r = k * kTogether + my_row;
            const uint64_t x = __shfl_sync(0xffffffffu, row, r) * (S::quant ? 1 : 2) + chunk * 16;
            const bool copy = (alive >> r & 1) && inside;
            const uint32_t tile_row = w * kEach + r;
            const uint32_t place = S::quant ? r * a.head_dim + chunk * 16 : (chunk >> 3) * (S::TOK * 128) + tile_row * 128 + ((chunk & 7 ^ tile_row & 7) << 4);
            if (!S::quant || inside) copy16(to + place, from + (copy ? x : 0), copy);
          }
        }
        if (S::quant && keys && lane < kEach) {
          const uint64_t at_scale = (uint64_t(uint32_t(page >= 0 ? page : 0)) * a.n_heads + h) * a.page_size.d + off;
          const uint32_t there = meta + tile % S::NMETA * S::META + 16 + (w * kEach + lane) * 4;
          copy4(there, a.k_scale + at_scale, page >= 0);
          copy4(there + S::TOK * 4, a.v_scale + at_scale, page >= 0);
        }
        copies_end();
        if (keys && t + 1 < n) look_up((at.step + t + 1) * S::TOK);
        kinds = (kinds & ~(1u << (queued & 31))) | uint32_t(keys) << (queued & 31);
        boxes = (boxes & ~(1u << (queued & 31))) | uint32_t(box) << (queued & 31);
        items[1] = items[0], items[0] = item;
        ++queued, ++item, ++i;
        if (!S::quant && a.block) {
          // boxes count themselves; rows that had to be copied one by one, at the end of a prefix, are waited for at once
          if (!box) copies_wait<0>(), to_async_proxy();
          if (keys) bar_arrive(described + 8 * (tile % S::NMETA));
          if (!box || lane) bar_arrive(bar);
          landed = queued;
        }
        land_now = queued - landed > ahead;
      }
      if (land_now) {
        copies_wait_all_but(queued - landed - 1);
        land();
      }
    }
    copies_wait<0>();
  } else {
    // ================================================================ the products
    // A warp for each stream: one thread of it issues, which next to the busy warps takes about as long as the products themselves.
    if constexpr (S::STREAMS == 2) fewer_registers<S::REGS_PRODUCT>();
    const uint32_t stream = warp - (8 * S::STREAMS + S::LOADERS);
    if (stream >= 2) look_at_rows();
    if (stream < S::STREAMS) {
      uint32_t item = 0, n_weights = 0, n_queries = 0, n_turns = 0;  // item: the place in the ring's order
      const uint32_t depth = a.head_dim / 16;
      const uint32_t scores = product(FMT == BCP_BF16, false, S::TOK), sums = product(S::split, true, a.head_dim);
      const bool chosen = elected();
      bool ok = true;
      const uint32_t q = same(operand(q_at + stream * S::Q, 0)), s_at = same(tmem + S::S0 + stream * S::TOK), o = same(tmem + S::O0 + stream * DP);
      const uint32_t keys_at = same(operand(ring, 0)), values_at = same(operand(ring, S::TOK * 128));
      auto score = [&](uint32_t slot) {  // with the keys in a place of the ring
        const uint32_t k = keys_at + slot * (S::TILE / 16);
#pragma unroll
        for (uint32_t j = 0; j < DP / 16; ++j)
          if ((DP > 64 && j < DP / 32) || j < depth)
            mma_shared(chosen, s_at, q + ((j >> 2) * (kRows * 128) + (j & 3) * 32) / 16, k + ((j >> 2) * (S::TOK * 128) + (j & 3) * 32) / 16, scores, j > 0);
        if (chosen) tmem_commit(s_full + 8 * stream);
        __syncwarp();
      };
      // The values in a place of the ring with the weights of columns 32 c and on of either part.
      auto weigh = [&](uint32_t slot, bool add, uint32_t c) {
        const uint32_t v = values_at + (slot * S::TILE + c * 4096) / 16, p = s_at + 32 * c;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          const uint32_t from = p + (j >> 1) * S::COLS + (j & 1) * 8, values = v + ((j >> 1) * S::COLS * 128 + (j & 1) * 2048) / 16;
          mma_tensor(chosen, o, from, values, sums, j > 0 || add);
          if (S::split) mma_tensor(chosen, o, from + 16, values, sums, true);
        }
      };
      auto arrived = [&](uint32_t bar, uint32_t parity) {
        ok = ok && bar_wait(bar, parity, limit);
        tmem_after();
        return ok;
      };
      for (left = same(left); left && ok;) {
        const uint32_t n = same(min(at.group.steps - at.step, left));
        const uint32_t row0 = at.u % at.group.tiles * S::ROWS;
        const bool both = same(min(at.group.rows - row0, S::ROWS)) > kRows;
        // Tiles first, first + step, .. are this stream's.  Both warps go through all items of the ring, in its order: the keys of `early` tiles, then the values of
        // a tile and the keys of the next in turn, and an item is free when both are done with it.
        const uint32_t step = both ? 1 : S::STREAMS, first = both ? 0 : stream, early = min(n, step);
        if (first < n && !arrived(q_full + 8 * stream, n_queries++ & 1)) break;
        auto there = [&](uint32_t i) { return arrived(full + 8 * (i % S::SLOTS), i / S::SLOTS & 1); };
        auto done = [&](uint32_t i) {
          if (chosen) {
            tmem_commit(empty + 8 * (i % S::SLOTS));
            if (S::STREAMS == 1) tmem_commit(empty + 8 * (i % S::SLOTS));
          }
        };
        for (uint32_t i = 0; i < 2 * n && ok; ++i, ++item) {
          const uint32_t j = i - early;
          const bool keys = i < early || (j < 2 * (n - early) && (j & 1));
          const uint32_t t = i < early ? i : keys ? early + j / 2 : j < 2 * (n - early) ? j / 2 : j - (n - early);
          if (!there(item)) break;
          if (!both && t % S::STREAMS != stream) {
            if (chosen) bar_arrive(empty + 8 * (item % S::SLOTS));
            __syncwarp();
            continue;
          }
          const uint32_t slot = same(item % S::SLOTS);
          if (keys) {
            score(slot);
            done(item);
            __syncwarp();
            continue;
          }
          // Values, and where both streams take every tile the next keys right behind them.  One stream's products after the other's: side by side both
          // would be done late, and both streams would make weights, then wait, at the same time.
          const bool more = both && t + 1 < n;
          if (more && !there(item + 1)) break;
          if (both && (stream || n_turns)) {
            if (!arrived(turn + 8 * stream, (stream ? n_turns : n_turns - 1) & 1)) break;
          }
          n_turns += both;
          if (!arrived(p_full + 16 * stream, n_weights & 1)) break;
          weigh(slot, t > first, S::COLS / 32 - 1);
          if constexpr (S::COLS == 64) {
            if (!arrived(p_full + 16 * stream + 8, n_weights & 1)) break;
            weigh(slot, true, 0);
          }
          ++n_weights;
          if (more) score(slot + 1 == S::SLOTS ? 0 : slot + 1);
          if (both && chosen) bar_arrive(turn + 8 * (1 - stream));
          done(item);
          if (more) done(item + 1), ++item, ++i;
          if (chosen && t + step >= n) tmem_commit(o_full + 8 * stream);
          __syncwarp();
        }
        left -= n;
        advance<S>(at, a, n, left != 0);
      }
    }
  }
  tmem_before();
  __syncthreads();
  if (*stop) {
    // A wait has run out in some warp (all others are done, too, so nobody changes the word any more): products and boxes that nobody has waited for come to
    // their end before the memory they use is given back.
    const uint32_t stream = warp - (8 * S::STREAMS + S::LOADERS);
    const uint64_t begin = global_timer_ns();
    if (stream < S::STREAMS) {
      if (elected()) tmem_commit(drained + 8 * stream);
      __syncwarp();
      while (!mbar_try_wait(drained + 8 * stream, 0) && global_timer_ns() - begin < kMostNs) {
      }
    }
    while (global_timer_ns() - begin < kDrainNs) {
    }
    if (tid == 0) raise(a.status, BCP_TIMED_OUT);
    __syncthreads();
  }
  tmem_after();
  if (warp == S::WARPS - 4) tmem_free(tmem);
}

// ------------------------------------------------------------------------------ the end
// The records of a row, that of its own tokens first and then its prefix's in the order of the parts, become its result.
struct JoinArgs {
  const int4* rows;
  const float2* ml;
  const float* o;
  uint32_t n_rows, n_q_heads, dims, apart, own, records, parts;  // own: the record of row 0's own tokens; apart: records from one part to the next
  void* out;
  float* lse;
  int64_t out_token, out_head;
  uint32_t is_bf16;
};
// Rows for which eight warps each are faster than a warp each.  Microseconds (all three kernels, 128 dimensions) with eight and with one over a prefix of 4096: 160 rows 14.7
// and 20.8, 480 20.4 and 24.2, 800 22.3 and 25.7, 1216 28.4 and 26.0, 2048 34.5 and 27.8; over 32,768: 800 rows 48.9 and 53.6, 1216 59.4 and 56.9.
constexpr uint32_t kFewRows = 1000;

// TOGETHER: eight warps take a row, else a warp does.
template <int DP, bool TOGETHER>
__global__ void __launch_bounds__(256) bcp_kv_join_kernel(const JoinArgs a) {
  after_previous();
  constexpr int N = (DP + 127) / 128;  // vectors of four dimensions a lane
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t r = TOGETHER ? blockIdx.x : blockIdx.x * 8 + warp;
  if (r >= a.n_rows) return;
  const int4 d = __ldcg(a.rows + r);
  const uint32_t both = d.w ? 2 : 1, n = 1 + min(uint32_t(d.z), a.parts) * both;

  // records first, first + step, .. of row r: largest reference, denominator, sums
  float m, den;
  float4 x[N];
  auto add_up = [&](uint32_t first, uint32_t step) {
    auto record = [&](uint32_t i) {
      if (i == 0) return a.own + r;
      const uint32_t part = (i - 1) / both;
      const uint32_t place = (part ? uint32_t(d.y) + (part - 1) * a.apart : uint32_t(d.x)) + (i - 1) % both * uint32_t(d.w);
      return place < a.records ? place : a.own + r;  // (a row that two groups claim: whatever comes out)
    };
    m = kNone, den = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (uint32_t i0 = first; i0 < n; i0 += 32 * step) {
      // a record a lane
      const uint32_t i = i0 + lane * step;
      float2 ml = make_float2(kNone, 0.f);
      uint32_t place = a.own + r;
      if (i < n) place = record(i), ml = __ldcg(a.ml + place);
      float top = ml.y > 0.f ? ml.x : kNone;
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      top = fmaxf(top, m);
      const Factor<true> before(m - top);
      den = before.denominator(den), m = top;
#pragma unroll
      for (int k = 0; k < N; ++k) x[k].x *= before.all, x[k].y *= before.all, x[k].z *= before.all, x[k].w *= before.all;
      const Factor<true> down(ml.y > 0.f ? ml.x - top : kNone);
      float weight = down.all, sum = down.denominator(ml.y);
      if (ml.y != ml.y) weight = sum = ml.y;  // a NaN stays one
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      den += sum;
      const uint32_t here = min(32u, (n - i0 + step - 1) / step);
#pragma unroll 1
      for (uint32_t j0 = 0; j0 < here; j0 += 8) {
        float4 y[8][N];
        float w[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          w[j] = __shfl_sync(0xffffffffu, weight, j0 + j);
          const float* const from = a.o + uint64_t(__shfl_sync(0xffffffffu, place, j0 + j)) * a.dims;
          if (j0 + j >= here) w[j] = 0.f;
#pragma unroll
          for (int k = 0; k < N; ++k)
            if (w[j] != 0.f && 128 * k + 4 * lane < a.dims) y[j][k] = __ldcg(reinterpret_cast<const float4*>(from + 128 * k + 4 * lane));
        }
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          if (w[j] == 0.f) continue;  // an empty record has no sums
#pragma unroll
          for (int k = 0; k < N; ++k)
            x[k].x += y[j][k].x * w[j], x[k].y += y[j][k].y * w[j], x[k].z += y[j][k].z * w[j], x[k].w += y[j][k].w * w[j];
        }
      }
    }
  };
  auto finish = [&]() {
    const float inv = den == 0.f ? 0.f : reciprocal_fast(den);
    const uint32_t b = r / a.n_q_heads, h = r - b * a.n_q_heads;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint32_t e = 128 * k + 4 * lane;
      if (e >= a.dims) break;
      uint2 y;
      y.x = a.is_bf16 ? pack16<true>(x[k].x * inv, x[k].y * inv) : pack16<false>(x[k].x * inv, x[k].y * inv);
      y.y = a.is_bf16 ? pack16<true>(x[k].z * inv, x[k].w * inv) : pack16<false>(x[k].z * inv, x[k].w * inv);
      *reinterpret_cast<uint2*>(static_cast<char*>(a.out) + (b * a.out_token + h * a.out_head + e) * 2) = y;
    }
    if (lane == 0 && a.lse) a.lse[r] = den == 0.f ? -INFINITY : (m + log2_fast(den)) * 0.6931471805599453f;
  };

  if constexpr (!TOGETHER) {
    add_up(0, 1);
    finish();
  } else {
    __shared__ float4 sums[8][N][32];
    __shared__ float2 about[8];
    add_up(warp, 8);
#pragma unroll
    for (int k = 0; k < N; ++k) sums[warp][k][lane] = x[k];
    if (lane == 0) about[warp] = make_float2(m, den);
    __syncthreads();
    if (warp) return;
    m = kNone, den = 0.f;
    for (uint32_t w = 0; w < 8; ++w) m = fmaxf(m, about[w].x);
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (uint32_t w = 0; w < 8; ++w) {
      const Factor<true> down(about[w].x - m);
      den += down.denominator(about[w].y);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float4 y = sums[w][k][lane];
        x[k].x += y.x * down.all, x[k].y += y.y * down.all, x[k].z += y.z * down.all, x[k].w += y.w * down.all;
      }
    }
    finish();
  }
}

// ------------------------------------------------------------------------------ launch
struct Variant {
  void (*kernel)(PrefixArgs);
  void (*join[2])(JoinArgs);  // a warp a row; eight
  uint32_t smem, threads, rows, tokens, registers, each;  // each: tokens of a tile that a warp brings
};
template <int FMT, int DP>
Variant variant() {
  typedef Shape<FMT, DP> S;
  constexpr int JOIN = DP <= 128 ? 128 : 256;
  return Variant{bcp_kv_prefix_kernel<FMT, DP>, {bcp_kv_join_kernel<JOIN, false>, bcp_kv_join_kernel<JOIN, true>}, S::SMEM, S::THREADS, S::ROWS, S::TOK, S::STREAMS == 2 ? S::REGS : 0, S::TOK / 4};
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
  // The warpgroups hand registers to one another, and with fewer than they count on some would wait forever.  A kernel that hands them on is launched with the most that
  // its launch bounds allow, whatever it needs, so this refuses nothing but the work of a compiler that does otherwise.
  cudaFuncAttributes about;
  BCP_CUDA(cudaFuncGetAttributes(&about, v.kernel));
  if (v.registers && about.numRegs < int(v.registers)) return fail(BCP_ERR_CUDA, "bcp_kv_attend_shared: the kernel has %d registers a thread, not %u", about.numRegs, v.registers);
  BCP_CUDA(cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(v.smem)));
  BCP_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device));
  *sms = uint32_t(n);
  if (n_known < 256) known[n_known++] = {v.kernel, device, *sms};
  return BCP_OK;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
int encode_tiled(EncodeTiled* out) {
  static std::mutex mu;
  static EncodeTiled known = nullptr;
  std::lock_guard<std::mutex> lock(mu);
  if (!known) {
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult q;
    BCP_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q));
    if (q != cudaDriverEntryPointSuccess || !sym) return fail(BCP_ERR_CUDA, "cuTensorMapEncodeTiled is not available in this driver");
    known = reinterpret_cast<EncodeTiled>(sym);
  }
  *out = known;
  return BCP_OK;
}
// Keys and values as tensors of whose tokens a warp's share of a tile is brought in boxes: of as many tokens as divide a page, a power of two of at least
// eight.  Smaller ones would be more commands than the copies take, and vectors under 64 elements do not fill a box: those are copied row by row.
int make_maps(const bcp_kv_cache* c, const Variant& v, PrefixArgs* a) {
  uint32_t block = v.each;
  while (c->page_size % block) block /= 2;
  const bool wide = is_8bit(c->format);
  a->block = 0;
  if (block < 8 || (!wide && c->head_dim < 64)) return BCP_OK;
  EncodeTiled encode = nullptr;
  if (int rc = encode_tiled(&encode)) return rc;
  const uint64_t es = type_size(c->format);
  const cuuint64_t dims[4] = {c->head_dim, c->page_size, c->n_heads, c->n_pages};
  const cuuint64_t strides[3] = {uint64_t(c->token_stride) * es, uint64_t(c->head_stride) * es, uint64_t(c->page_stride) * es};
  const cuuint32_t box[4] = {wide ? c->head_dim : 64, block, 1, 1}, ones[4] = {1, 1, 1, 1};
  const CUtensorMapDataType type = wide ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
  for (int side = 0; side < 2; ++side) {
    const CUresult rc = encode(side ? &a->v_map : &a->k_map, type, 4, side ? c->v : c->k, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               wide ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (rc != CUDA_SUCCESS) return BCP_OK;  // strides that a tensor map cannot have
  }
  a->block = block;
  return BCP_OK;
}

constexpr uint64_t kBoundary = 256;
uint64_t aligned(uint64_t n) { return (n + kBoundary - 1) / kBoundary * kBoundary; }
// The workspace: that of the attention over own tokens, then rows, references and sums of the records.  These lie on boundaries of memory (sums are stored 32
// bytes at a time), the workspace itself on one of 16 bytes: `skew` is what is missing to the next boundary where it begins.
struct Layout {
  uint64_t rows, ml, o, end, records;
  Layout(uint64_t begin, uint64_t skew, const Variant& v, uint32_t sms, uint64_t n_seqs, uint32_t n_q_heads, uint32_t head_dim) {
    const uint64_t every = n_seqs * n_q_heads;
    records = 3 * every + 2ull * sms * v.rows;  // whole units (two streams), parts, own tokens
    rows = aligned(begin) + skew, ml = rows + aligned(every * sizeof(int4)), o = ml + aligned(records * sizeof(float2)), end = o + records * head_dim * 4;
  }
};
constexpr uint64_t kMostSkew = kBoundary - 16;
uint64_t skew_of(const void* workspace) { return (0 - reinterpret_cast<uintptr_t>(workspace)) & (kBoundary - 1); }

}  // namespace
}  // namespace bcp

using namespace bcp;

extern "C" int bcp_wait_limit(uint32_t nanoseconds) {
  g_limit.store(nanoseconds, std::memory_order_relaxed);
  return BCP_OK;
}

extern "C" int bcp_kv_attend_shared_workspace(const bcp_kv_cache* cache, uint32_t n_q_heads, uint32_t max_seqs, uint64_t* bytes) {
  const char* call = "bcp_kv_attend_shared_workspace";
  uint64_t own = 0;
  if (int rc = bcp_kv_attend_workspace(cache, n_q_heads, max_seqs, &own)) return rc;
  const Variant v = variant_of(cache->format, cache->head_dim);
  uint32_t sms = 0;
  if (int rc = prepare(v, &sms)) return rc;
  const Layout at(own, kMostSkew, v, sms, max_seqs, n_q_heads, cache->head_dim);
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
  if (n_prefixes && (!prefix_table || !prefix_lengths || !starts || prefix_stride < 0 || (n_prefixes > 1 && prefix_stride && prefix_stride < int64_t(prefix_width))))
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
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return fail(BCP_ERR_INVALID, "%s: workspace is NULL or not 16-byte aligned", call);
  const Layout at(own, skew_of(workspace), v, sms, n_seqs, q->n_heads, c->head_dim);
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
  a.q_is_bf16 = q->type == BCP_BF16, a.q_wide = rows_aligned(q, 16), a.n_seqs = n_seqs, a.n_groups = n_prefixes, a.group = FastDiv(group);
  a.table = prefix_table, a.table_stride = prefix_stride;
  a.lengths = prefix_lengths, a.starts = starts;
  a.scale_log2 = scale * kLog2e;
  a.limit = g_limit.load(std::memory_order_relaxed);
  if (int rc = make_maps(c, v, &a)) return rc;
  char* const w = static_cast<char*>(workspace);
  a.rows = reinterpret_cast<int4*>(w + at.rows), a.ml = reinterpret_cast<float2*>(w + at.ml), a.o = reinterpret_cast<float*>(w + at.o);
  const uint64_t own_at = at.records - uint64_t(n_seqs) * q->n_heads;
  const Records records = {a.ml + own_at, a.o + own_at * c->head_dim, c->head_dim};
  // the second kernel's arguments are looked at before the first is launched
  if (int rc = attend(call, c, q, out, lse, n_seqs, block_table, table_stride, table_width, lengths, scale, 0, workspace, own, &records, false, stream))
    return rc;
  const uint64_t most = tiles * c->n_heads * steps;
  cudaStream_t const st = static_cast<cudaStream_t>(stream);
  BCP_CUDA(launch_early(v.kernel, uint32_t(most < sms ? most : sms), v.threads, v.smem, st, a));
  if (int rc = attend(call, c, q, out, lse, n_seqs, block_table, table_stride, table_width, lengths, scale, 0, workspace, own, &records, true, stream))
    return rc;
  JoinArgs j = {};
  j.rows = a.rows, j.ml = a.ml, j.o = a.o;
  j.n_rows = n_seqs * q->n_heads, j.n_q_heads = q->n_heads, j.dims = c->head_dim;
  j.apart = 2 * v.rows, j.own = uint32_t(own_at), j.records = uint32_t(own_at), j.parts = sms;
  j.out = out->data, j.lse = lse, j.out_token = out->token_stride, j.out_head = out->head_stride, j.is_bf16 = out->type == BCP_BF16;
  const bool together = j.n_rows <= kFewRows;
  BCP_CUDA(launch_early(v.join[together], together ? j.n_rows : (j.n_rows + 7) / 8, 256, 0, st, j));
  return BCP_OK;
}

// Attention of many query rows over the cache (questions, prompts): the
// products bound it, so both run on tcgen05.
//
// A CTA takes up to 256 query rows (new tokens x heads of the group) of one
// key/value head as two tiles of 128, and the cached tokens 64 at a time. Of a
// long item of 128 rows or less both streams of products and softmax take the
// same rows, and every other tile of tokens each (kTcStreamed); the first joins
// their sums.
//   loaders    a warp for keys and one for values, which look up pages and masks
//              some tiles ahead, tell the others what there is to see, and ask
//              for the copies: tiles of 16-bit pages by tensor map, with the
//              128-byte swizzle, to where the products read them; codes and
//              bytes as they lie in the pages
//   unpackers  (less than 16 bits) four warps for keys, four for values: to
//              (n - z) s or (u - 128) s, which the 16-bit types hold exactly
//   MMA        a warp for S = Q K^T into tensor memory (128 x 64 fp32 a stream), and
//              one for O += P V with P read from tensor memory; for 16 bits it puts
//              zeros where a value is not to be seen before (a NaN there would
//              pass through a product with 0)
//   softmax    four warps a stream, a thread to a row: maximum, exponentials, P
//              back into S's place in 16 bits; at the end O out
// (With copies made by the threads that unpack, 16 bytes each, a tile of bytes
// took 3300 cycles and one of 16-bit values 3400, however few the rows.)
// The running maximum that exponentials refer to is found at a row's first tokens
// and raised only when a tile's weights sum to more than their type has room for
// (then O is brought down in tensor memory), which seldom happens after them
// (looking for every tile's maximum took 500 cycles of its 1860). O
// itself is read out and begun anew after some thousands of tokens (kTcChain).
//
// Tensor memory: O0 O1 (D columns each) and for each tile two S of 64 columns,
// P in the first 32 of its S: while the softmax works on one S, the products
// of the next tokens fill the other. With one S of 128 tokens a tile, the
// softmax waited 2300 of 5900 cycles for P V and the next Q K^T to be done
// (256 new tokens over 65792 cached ones of 4 bits: 376 us).
//
// For 256 rows by 64 tokens (head of 128) the tensor core needs 1024 cycles; a
// tile takes 1900 of 16-bit values and 2490 of bytes. What bounds it is the issue
// of the eight softmax warps, two to a scheduler (340 instructions a tile each),
// and of as many that unpack (2900 together): with bytes 6000 warp instructions,
// 62 % of the issue slots, the ALU pipe 49 %, the tensor pipe 42 % (256 new tokens
// over 65792, 32 heads over 8: 278 us; 4 bits 261, 16 bits 216). 128 rows or less
// over 16-bit pages are bound by DRAM: 128 over 262144 tokens 167 us of 158.
// Tried: a warp for each stream's products instead of one for S and one for O
// (283, but 230 for 199 over 16 bits where both streams take the same rows); four such warps
// (305: less registers for the softmax); loops of products (319 for 304: the warp
// that issues is late); a tile's look-up while the one before is loaded (342).
#pragma once

#include "kv_split.cuh"
#include "ngff_device.cuh"

namespace cofie {
namespace {

constexpr int kTcRows = kManyRows;
constexpr int kTcSoftmax = 256;  // threads: warps 0 to 7
constexpr int kTcUnpack = 128;   // of keys, and as many of values
// And two warps that issue, and two loaders.
template <int BITS>
constexpr int kTcThreads = kTcSoftmax + (BITS < 16 ? 2 * kTcUnpack : 0) + 128;
constexpr int kTcInfo = 16;         // more than the stages and the raw tiles: a tile is told before its place is free
// Tiles from which both streams take an item of 128 rows or less: it pays over long caches, and the sums' meeting costs
// short items more. us, by one stream / by both: 32 answers over 262144 tokens of bytes 263 / 232, 128 rows of 4 bits 214 / 180;
// 80 rows over 60000 tokens of 4 bits 379 / 313, of bytes 391 / 397, over 6000 112 / 115 and 130 / 128, over 2000 28 / 30, 30 / 31.
// 16 bits, 8 key heads of 128: 32 answers over 262144 191 / 189, 64 rows over 524288 319 / 312, over 66000 59 / 61, over 6000 97 / 106;
// fp16, 4 key heads: 64 rows over 524288 177 / 167, over 66000 43 / 44; 8 of 64: over 66000 50 / 43, over 262144 151 / 119.
template <int BITS>
constexpr uint32_t kTcStreamed = BITS < 16 ? 128 : 1024;
// Tiles whose products are summed in tensor memory before the sums move on to the CTA's part. The tensor core cuts each
// product off at about 2^-24 of the sum that it is added to, so 8192 tokens may cost a sum 2^-11 of its size, a rounding
// of fp16, and 65536 tokens 2^-8, one of bf16. (In one sum, 262144 tokens 14 to 17 below a first one came out 0.4 to
// 0.5 % low.)
template <typename T>
constexpr uint32_t kTcChain = std::is_same<T, __half>::value ? 128 : 1024;
constexpr uint64_t kTcTimeout = 1000000000ull;
// Registers where there are unpackers: all threads start with 96; 256 x 144 + 256 x 56 + 128 x 80 is 640 x 96.
constexpr int kTcRegsSoftmax = 144, kTcRegsUnpack = 56, kTcRegsIssuer = 80;

// What the loader of keys says of a tile; all but the softmax and the loaders go by it alone.
struct TcInfo {
  uint32_t bits[2];  // tokens that some row may see
  int32_t pos;       // the first token
  uint32_t plain;    // every token is seen by every row
  uint32_t j;        // tiles of its item before it
  uint32_t flags;    // kTc*
};

enum : uint32_t { kTcBoth = 1, kTcSecond = 2, kTcEnd = 4 };  // streamed by both; the second stream has rows; no more tiles

template <int D, int BITS, bool SHARED>
struct TcSmem {
  static constexpr int kBlockQ = 128 * 128;   // 128 rows of 64 values
  static constexpr int kBlock = kTile * 128;  // 64 rows of 64 values
  static constexpr int kStages = BITS < 16 ? 3 : 4;            // of keys, and of values
  static constexpr int kRaw = BITS == 16 ? 1 : BITS == 8 && D == 128 ? 3 : 6;  // tiles as they lie in the pages
  static constexpr int kRow = D * BITS / 8, kRowWords = (D / 64) * 2;  // bytes of a token's keys
  union {
    char q[2][kBlockQ * (D / 64)];
    Plan<kTcThreads<BITS>, SHARED> plan;  // until every thread has its walk
  };
  char kv[2][kStages][kBlock * (D / 64)];  // keys, values
  char raw[2][kRaw][BITS < 16 ? kTile * kRow : 16];
  char raw_words[2][kRaw][BITS < 16 ? kTile * kRowWords : 16];
  uint32_t raw_bits[2][kRaw][4];  // of a raw tile's tokens, those to be seen; then whether there are no more tiles
  Span spans[kSpans];
  TcInfo info[kTcInfo];
  float by_sum[kTcRows];
  uint64_t full[2][kStages], empty[2][kStages];  // keys, values
  uint64_t raw_full[2][kRaw], raw_empty[2][kRaw];
  // A barrier's phase can be told from the one before only. O is ready twice before anyone has to look, so it has a
  // barrier for even tiles and one for odd ones, as S and P have.
  uint64_t info_full[kTcInfo], q_full[2], s_full[2][2], p_full[2][2], o_full[2][2], drained;
  uint32_t tmem, stop;
};

// A wait for a barrier's phase that ends, with false, when it runs out or another's has (with stop).
__device__ __forceinline__ bool tc_wait_slow(uint32_t bar, uint32_t parity, volatile uint32_t* stop) {
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 16; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (stop && *stop) return false;
    if (globaltimer_ns() - t0 > kTcTimeout) {
      if (stop) *stop = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool tc_wait(const uint64_t* bar, uint32_t parity, uint32_t* stop) {
  const uint32_t b = shared_address(bar);
  return mbar_try_wait(b, parity & 1) || tc_wait_slow(b, parity & 1, stop);
}
// A place in a ring of N, and the parity of its barriers' phase. Kept up instead of divided out of a count of tiles: a
// warp that issues or looks up has a few hundred cycles a tile, in which it gets to issue every eighth or so.
template <uint32_t N>
struct Turn {
  uint32_t i = 0, parity = 0;
  __device__ __forceinline__ void next() {
    if (++i == N) i = 0, parity ^= 1;
  }
};

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Copies whose bytes the barrier counts: some that lie in a row, and a box of the pages' tensor map. Written for a whole
// warp, of which the leader asks (see tc_leader).
__device__ __forceinline__ void bulk_copy(uint32_t leader, uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %4, 0;\n\t"
      "@q cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void box_copy(uint32_t leader, uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void arrive_expecting(uint32_t leader, uint32_t bar, uint32_t bytes) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
               "r"(bytes), "r"(leader)
               : "memory");
}
// What the warp has done before comes before the barrier's phase: one arrival for all its threads (128 arrivals at one
// address one after the other would cost more than the wait).
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if (threadIdx.x % 32 == 0) mbar_arrive(shared_address(bar));
}
template <int ID, int THREADS>
__device__ __forceinline__ void bar_sync() {
  asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(THREADS) : "memory");
}

// Operand in shared memory, 128-byte swizzle, eight rows of 128 bytes to an
// atom of 1024. K-major: rows are M or N, the 64 values of a row are K; the
// leading offset is not used. MN-major: rows are K, the 64 values M or N, the
// next 64 lie `leading` bytes on.
// (The descriptor's upper half is the same for all: eight rows' 1024 bytes, the version, the swizzle.)
__device__ __forceinline__ uint32_t tc_desc(uint32_t addr, uint32_t leading) { return (addr >> 4) | (leading >> 4) << 16; }
constexpr uint32_t kTcDescUpper = (1024u >> 4) | 1u << 14 | 2u << 29;
// fp32 sums of products of 16-bit values; B K-major or MN-major.
template <typename T>
__device__ __forceinline__ constexpr uint32_t tc_idesc(uint32_t m, uint32_t n, bool b_mn) {
  const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (type << 7) | (type << 10) | ((b_mn ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((m >> 4) << 24);
}
// One thread of the warp, chosen once. The products are written for a whole warp, of which that thread issues: in code
// that a single thread runs, the operands' way into uniform registers took 125 cycles a product.
__device__ __forceinline__ uint32_t tc_leader() {
  uint32_t x;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(x));
  return x;
}
__device__ __forceinline__ void tc_mma_ss(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 x, y;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "mov.b64 x, {%1, %6};\n\tmov.b64 y, {%2, %6};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(leader), "n"(kTcDescUpper)
      : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 y;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "mov.b64 y, {%2, %6};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(leader), "n"(kTcDescUpper)
      : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t leader, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(shared_address(bar)),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(
          r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
// 16 columns, waited for.
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// Waits for this thread's loads from tensor memory; the registers they fill pass through it, so that no use of them
// can be moved before it.
__device__ __forceinline__ void tc_wait_ld(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                 "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                 "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The largest of 64 values and `top`.
__device__ __forceinline__ float most_of(const uint32_t* x, const uint32_t* y, float top) {
  float a = top, b = __uint_as_float(y[0]);
#pragma unroll
  for (int f = 0; f < 32; f += 2) a = fmaxf(fmaxf(__uint_as_float(x[f]), __uint_as_float(x[f + 1])), a);
#pragma unroll
  for (int f = 0; f < 32; f += 2) b = fmaxf(fmaxf(__uint_as_float(y[f]), __uint_as_float(y[f + 1])), b);
  return fmaxf(a, b);
}
// Two fp32 operations at once.
__device__ __forceinline__ uint64_t two(uint32_t lo, uint32_t hi) {
  uint64_t x;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "r"(lo), "r"(hi));
  return x;
}
__device__ __forceinline__ uint64_t two(float lo, float hi) { return two(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void apart(uint64_t x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t x;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(a), "l"(b), "l"(c));
  return x;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t x;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
  return x;
}

// SHARED as for attend_split. WHOLE: no item is cut, and no launch that joins parts follows.
template <typename T, int D, int BITS, bool SHARED, bool WHOLE>
__global__ void __launch_bounds__(kTcThreads<BITS>, 1) attend_rows_tc(const __grid_constant__ AttendArgs a) {
  using P = Pair<T>;
  using S = TcSmem<D, BITS, SHARED>;
  constexpr uint32_t kStages = S::kStages, kRaw = S::kRaw;
  constexpr int kThreads = kTcThreads<BITS>;
  // What exponentials refer to (m below, in the parts too) is kUp below the maximum, so that weights are 2^kUp times what
  // they stand for, and a tile's 64 sum to 2^(kUp + 6) where all are as large as the maximum; it is raised where they pass
  // kMost. fp16: 2^8, so that only weights under 2^-33 of the largest are lost to the second product, as for few rows, and up
  // to 2^15, which fp16 holds. bf16 has the exponents of fp32: 2^-8 and up to 1, so that a weight times a value stays in range where the
  // value is (with weights of 1 and up to 2^8, a token 2^7 heavier than all before and its value of 2^121 gave infinity).
  constexpr bool kHalf = std::is_same<T, __half>::value;
  constexpr float kMost = kHalf ? 0x1p15f : 1.f, kUp = kHalf ? 8.f : -8.f;
  extern __shared__ char raw[];
  S& sm = *reinterpret_cast<S*>(raw + (1024u - (shared_address(raw) & 1023u)) % 1024u);
  // (Behind whole items the next launch is not let in early: where it was, a following call's passes over its mask lay beside
  // them and the kernel over its prefix took 50 us more of 416.)
  if (!WHOLE) pdl_trigger();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  constexpr uint32_t kIssuer = (kTcSoftmax + (BITS < 16 ? 2 * kTcUnpack : 0)) / 32, kLoader = kIssuer + 2;  // their first warps
  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < kStages; ++i) {
      for (int v = 0; v < 2; ++v) {
        mbar_init(shared_address(&sm.full[v][i]), BITS < 16 ? kTcUnpack / 32 : 1);
        mbar_init(shared_address(&sm.empty[v][i]), 1);
      }
    }
    for (uint32_t i = 0; i < kRaw; ++i)
      for (int v = 0; v < 2; ++v) {
        mbar_init(shared_address(&sm.raw_full[v][i]), 1);
        mbar_init(shared_address(&sm.raw_empty[v][i]), kTcUnpack / 32);
      }
    for (int i = 0; i < kTcInfo; ++i) mbar_init(shared_address(&sm.info_full[i]), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(shared_address(&sm.q_full[i]), 4);
      for (int j = 0; j < 2; ++j) {
        mbar_init(shared_address(&sm.o_full[i][j]), 1);
        mbar_init(shared_address(&sm.s_full[i][j]), 1);
        mbar_init(shared_address(&sm.p_full[i][j]), 4);
      }
    }
    mbar_init(shared_address(&sm.drained), 2);
    sm.stop = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  if (!WHOLE && threadIdx.x == 0) a.items[blockIdx.x].last_cta = 0;  // none goes on from here, so far
  // only now: a kernel before this one may still hold tensor memory, or wait for it
  if (warp == kIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&sm.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tc_fence_before();
  }
  const uint64_t range = sm.plan.set_up(a, kTcRows, sm.spans);  // ends with a barrier
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const auto o_at = [&](uint32_t t) { return tmem + t * D; };
  const auto s_at = [&](uint32_t t, uint32_t i) { return tmem + 2 * D + (2 * t + i % 2) * kTile; };
  Walk<kThreads, SHARED, WHOLE> walk(a, sm.plan, sm.spans, kTcRows, range);
  __syncthreads();
  const BatchArg& b = a.batch;
  Item it;
  uint32_t* stop = &sm.stop;
  bool ok = true;
  // whether both streams take the item's rows, every other tile each, and how many tiles of some that makes for a stream
  const auto streamed = [&](const Item& x) { return x.span.count * a.group - x.rb * kTcRows <= 128 && x.tiles >= kTcStreamed<BITS>; };
  const auto tiles_of = [](bool both, uint32_t t, uint32_t tiles) { return both ? (tiles + 1 - t) / 2 : tiles; };

  if (warp < kTcSoftmax / 32) {
    // ---------------------------------------------------------------- softmax: thread r of tile t has row r of it
    if constexpr (BITS < 16) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTcRegsSoftmax));
    const uint32_t t = warp / 4, r = threadIdx.x % 128;
    const uint32_t lanes = (warp % 4) * 32u << 16;
    const uint32_t o_col = o_at(t) + lanes;
    const float by = a.scale * 1.4426950408889634f;
    uint32_t n = 0, s_n = 0;  // tiles told; tiles of this stream
    bool kept_alone = false;  // an item of this CTA's own had sums kept in the part of the one that goes on
    while (walk.next(it)) {  // to the end even when a wait ran out: the barriers below count on all
      const bool both = streamed(it);
      const uint32_t row0 = it.rb * kTcRows + (both ? 0 : t * 128), all = it.span.count * a.group;
      const uint32_t told = it.hi - it.lo, tiles = tiles_of(both, t, told), step = both ? 2 : 1, from = both ? t : 0;
      const bool active = row0 < all, real = row0 + r < all;
      const uint32_t token = real ? (row0 + r) / a.group : 0, head = it.head * a.group + (real ? (row0 + r) % a.group : 0);
      int32_t seen = 0;
      if (real) {
        const int64_t x = a.causal ? static_cast<int64_t>(it.span.length) - it.span.count + token + 1 : it.span.length;
        seen = x > 0 ? static_cast<int32_t>(x) : 0;
      }
      const uint64_t shared_row = static_cast<uint64_t>(it.span.first + token) * a.heads + head;
      const bool before = SHARED && a.behind && has_prefix(a, it.seq);
      // the tokens of the tile at hand that this row sees, where rows differ: asked for a tile ahead, its number two ahead
      const bool by_row = SHARED && a.seq_words;
      const uint64_t* words = nullptr;
      const uint32_t* listed = nullptr;
      uint64_t word_ahead = 0;
      uint32_t unit_ahead = 0;
      if (by_row && tiles) {
        words = a.seq_words + static_cast<uint64_t>(min(static_cast<uint32_t>(a.seq_of[it.span.first + token]), b.members - 1)) * a.tile_stride;
        listed = a.tiles + tile_list<SHARED>(a, it.seq, it.rb) * a.tile_stride + it.lo + from;
        word_ahead = words[listed[0]];
        unit_ahead = tiles > 1 ? listed[step] : 0;
      }
      // The sum of the weights, and what its roundings left out: a row's tokens may all come to one thread, and
      // 262144 of them 17.5 below a first one, added to it as they came, were off by 1.7e-3 in the log-sum-exp.
      float m = -INFINITY, l = 0.f, l_rest = 0.f;
      // Sums that have left tensor memory are kept in the CTA's part, against the maximum of then: four of O's columns of a
      // row beside those of the next row. (Four prompts of 2048 fp16 tokens over 65536: 11.03 ms; with a row's columns one
      // after the other 11.42, with O left in tensor memory throughout 10.72.) An item that is this CTA's alone uses the part
      // of the one that goes on from it, which comes last.
      float kept_m = -INFINITY;
      const uint32_t lr = t * 128 + r;  // row of the item's 256
      const auto own_part = [&] { return (2ull * blockIdx.x + (blockIdx.x == it.first_cta ? 1 : 0)) * kTcRows; };
      const auto kept_at = [&](int col) { return reinterpret_cast<float4*>(a.part + own_part() * D) + col / 4 * kTcRows + lr; };
      if (active && tiles) {
        {  // the row of Q into shared memory; codes' products come in the order in which they are unpacked
          const T* q = reinterpret_cast<const T*>(a.q.in) + static_cast<int64_t>(it.span.first + token) * a.q.in_token +
                       static_cast<int64_t>(head) * a.q.in_head;
#pragma unroll 4
          for (int e = 0; e < D / 8; ++e) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (real) {
              if (a.q_wide) {
                x = *reinterpret_cast<const uint4*>(q + e * 8);
              } else {
                x = gather8(q + e * 8);
              }
            }
            if (BITS == 4)
              x = make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410),
                             __byte_perm(x.y, x.w, 0x7632));
            *reinterpret_cast<uint4*>(sm.q[t] + (e / 8) * S::kBlockQ + r * 128 + ((e % 8) ^ (r & 7)) * 16) = x;
          }
          fence_async_shared();
          warp_arrive(&sm.q_full[t]);
        }
        bool found = false;  // all rows of the warp have a maximum
#pragma unroll 1
        for (uint32_t j = 0; j < tiles; ++j, ++s_n) {
          const uint32_t at = n + from + j * step;  // of all tiles
          const TcInfo& info = sm.info[at % kTcInfo];
          uint64_t word = ~0ull;
          if (SHARED && by_row) {
            word = word_ahead;
            if (j + 1 < tiles) word_ahead = words[unit_ahead];
            if (j + 2 < tiles) unit_ahead = listed[(j + 2) * step];
          }
          // S first: after an item in which this half had no rows, info may be some phases behind until then
          ok = ok && tc_wait(&sm.s_full[t][s_n % 2], s_n / 2, stop) && tc_wait(&sm.info_full[at % kTcInfo], at / kTcInfo, stop);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          if (j > 0 && j % kTcChain<T> == 0) {
            ok = tc_wait(&sm.o_full[t][(s_n - 1) % 2], (s_n - 1) / 2, stop);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            const float k = kept_m == -INFINITY ? 0.f : exp2_fast(kept_m - m);
#pragma unroll 1
            for (int e = 0; e < D / 32; ++e) {
              float4 was[8];
              uint32_t z[32];
#pragma unroll
              for (int f = 0; f < 8; ++f) was[f] = j == kTcChain<T> ? make_float4(0.f, 0.f, 0.f, 0.f) : *kept_at(32 * e + 4 * f);
              tc_ld32(o_col + 32 * e, z);
              tc_wait_ld(z);
#pragma unroll
              for (int f = 0; f < 8; ++f)
                *kept_at(32 * e + 4 * f) =
                    make_float4(fmaf(was[f].x, k, __uint_as_float(z[4 * f])), fmaf(was[f].y, k, __uint_as_float(z[4 * f + 1])),
                                fmaf(was[f].z, k, __uint_as_float(z[4 * f + 2])), fmaf(was[f].w, k, __uint_as_float(z[4 * f + 3])));
            }
            kept_m = m;
          }
          const uint32_t s_col = s_at(t, s_n) + lanes;
          uint32_t see0 = ~0u, see1 = ~0u;  // the tokens that this row sees
          bool partly = false;              // some rows of the warp do not see all
          if (!info.plain || (SHARED && by_row)) {
            const int32_t k = seen - info.pos;  // the row sees the first k
            see0 = info.bits[0] & static_cast<uint32_t>(word) & (k >= 32 ? ~0u : k <= 0 ? 0u : (1u << k) - 1);
            see1 = info.bits[1] & static_cast<uint32_t>(word >> 32) & (k >= 64 ? ~0u : k <= 32 ? 0u : (1u << (k - 32)) - 1);
            partly = !__all_sync(0xffffffffu, (see0 & see1) == ~0u);
          }
          uint32_t w[32];
          float here = 0.f;
          if (partly && !__any_sync(0xffffffffu, (see0 | see1) != 0)) {  // a frame that is not these rows' evidence
#pragma unroll
            for (int f = 0; f < 32; ++f) w[f] = 0;
          } else {
            // The maximum is looked for at a row's first tokens, and when the sum of a tile's weights shows that the one that
            // they refer to is far behind: then once more from S, which is there until P takes its place. (The second 32
            // columns asked for behind the first, while those are worked on: 256 rows of bytes 285 -> 291 us.)
            for (bool again = false;;) {
              uint32_t x[32], y[32];
              tc_ld32(s_col, x);
              tc_ld32(s_col + 32, y);
              tc_wait_ld(x);
              tc_wait_ld(y);
              if (partly) {
#pragma unroll
                for (int f = 0; f < 32; ++f) {
                  if (!(see0 & (1u << f))) x[f] = 0xff800000u;
                  if (!(see1 & (1u << f))) y[f] = 0xff800000u;
                }
              }
              if (again || (!found && __any_sync(0xffffffffu, m == -INFINITY && (see0 | see1) != 0))) {
                const float top = most_of(x, y, -INFINITY) * by;
                const bool raise = !(here <= kMost) || (m == -INFINITY && top > -INFINITY);
                // (scores of 2^26 and more, which fp32 rounds by 8: their roundings take the exponents that kUp would)
                const float to = raise ? fmaxf(top - (fabsf(top) < 0x1p26f ? kUp : 0.f), m) : m, k = m == -INFINITY ? 0.f : exp2_fast(m - to);
                if (j % kTcChain<T> != 0) {  // O as it is after the tokens before
                  ok = tc_wait(&sm.o_full[t][(s_n - 1) % 2], (s_n - 1) / 2, stop);
                  ok = __all_sync(0xffffffffu, ok);
                  tc_fence_after();
                  uint32_t z[16];
#pragma unroll 1
                  for (int e = 0; e < D / 16; ++e) {
                    tc_ld16(o_col + 16 * e, z);
#pragma unroll
                    for (int f = 0; f < 16; ++f) z[f] = __float_as_uint(__uint_as_float(z[f]) * k);
                    tc_st16(o_col + 16 * e, z);
                  }
                  tc_wait_st();
                }
                l *= k;
                l_rest *= k;
                m = to;
                found = __all_sync(0xffffffffu, m != -INFINITY);
              }
              const float down = m == -INFINITY ? 0.f : -m;
              const uint64_t by2 = two(by, by), down2 = two(down, down);
              uint64_t l2 = two(0.f, 0.f), l3 = two(0.f, 0.f);
              const auto exponentials = [&](const uint32_t* z, uint32_t* w) {
#pragma unroll
                for (int f = 0; f < 16; f += 2) {
                  float p0, p1, p2, p3;
                  apart(fma2(two(z[2 * f], z[2 * f + 1]), by2, down2), p0, p1);
                  apart(fma2(two(z[2 * f + 2], z[2 * f + 3]), by2, down2), p2, p3);
                  p0 = exp2_fast(p0);
                  p1 = exp2_fast(p1);
                  p2 = exp2_fast(p2);
                  p3 = exp2_fast(p3);
                  l2 = add2(l2, two(p0, p1));
                  l3 = add2(l3, two(p2, p3));
                  w[f] = P::pack(p0, p1);
                  w[f + 1] = P::pack(p2, p3);
                }
              };
              exponentials(x, w);
              exponentials(y, w + 16);
              float l0, l1;
              apart(add2(l2, l3), l0, l1);
              here = l0 + l1;
              if (again || __all_sync(0xffffffffu, here <= kMost)) break;
              again = true;
            }
          }
          tc_st16(s_col, w);
          tc_st16(s_col + 16, w + 16);
          {  // l + here, whose rounding is l - (sum - took) + (here - took) to the last bit
            const float sum = l + here, took = sum - l;
            l_rest += (l - (sum - took)) + (here - took);
            l = sum;
          }
          tc_wait_st();
          tc_fence_before();
          warp_arrive(&sm.p_full[t][s_n % 2]);
        }
        if (ok) ok = tc_wait(&sm.o_full[t][(s_n - 1) % 2], (s_n - 1) / 2, stop);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        l += l_rest;
        if (tiles > kTcChain<T>) {  // what was kept comes back
          const float k = kept_m == -INFINITY ? 0.f : exp2_fast(kept_m - m);
#pragma unroll 1
          for (int e = 0; e < D / 16; ++e) {
            float4 was[4];
            uint32_t z[16];
#pragma unroll
            for (int f = 0; f < 4; ++f) was[f] = *kept_at(16 * e + 4 * f);
            tc_ld16(o_col + 16 * e, z);
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              z[4 * f] = __float_as_uint(fmaf(was[f].x, k, __uint_as_float(z[4 * f])));
              z[4 * f + 1] = __float_as_uint(fmaf(was[f].y, k, __uint_as_float(z[4 * f + 1])));
              z[4 * f + 2] = __float_as_uint(fmaf(was[f].z, k, __uint_as_float(z[4 * f + 2])));
              z[4 * f + 3] = __float_as_uint(fmaf(was[f].w, k, __uint_as_float(z[4 * f + 3])));
            }
            tc_st16(o_col + 16 * e, z);
          }
          tc_wait_st();
        }
      }
      n += told;
      const bool alone = WHOLE || it.first_cta == it.last_cta;
      if (threadIdx.x == 0 && it.first_cta == blockIdx.x && !alone) a.items[blockIdx.x] = {it.seq, it.rb, it.head, it.last_cta, it.span};
      const uint64_t part = own_part();
      // All have what they kept, of this item or of one before it, before the part is written: its rows lie across what other
      // threads keep, and a stream that the last item has no rows for may be an item behind. (With prefixes at every item:
      // only where sums were kept takes a register more, and eight questions over bytes took 1246 us for 1221, 32 answers 239 for
      // 232. Without, that is quicker: eight sequences of 32 rows over 6000 tokens of bytes 57, at every item 61.)
      if (SHARED || (!alone && (kept_alone || told > kTcChain<T>))) bar_sync<1, kTcSoftmax>();
      kept_alone = kept_alone || (alone && told > kTcChain<T>);
      // Both streams' sums of the same rows: the second's go to the first through Q's place, once all products are done.
      float k0 = 1.f, k1 = 0.f;
      float4* const across = reinterpret_cast<float4*>(sm.q[0]);  // [D / 4][128]
      if (both) {
        bar_sync<1, kTcSoftmax>();
        if (t == 1) {
#pragma unroll 1
          for (int e = 0; e < D / 32; ++e) {
            uint32_t y[32];
            if (tiles) {
              tc_ld32(o_col + 32 * e, y);
              tc_wait_ld(y);
            }
#pragma unroll
            for (int f = 0; f < 8; ++f)
              across[(8 * e + f) * 128 + r] = l != 0.f ? make_float4(__uint_as_float(y[4 * f]), __uint_as_float(y[4 * f + 1]), __uint_as_float(y[4 * f + 2]),
                                                                     __uint_as_float(y[4 * f + 3]))
                                                       : make_float4(0.f, 0.f, 0.f, 0.f);
          }
          sm.by_sum[r] = m;
          sm.by_sum[128 + r] = l;
        }
        bar_sync<1, kTcSoftmax>();
        if (t == 0) {
          const Both x = both_parts(m, l, make_float2(sm.by_sum[r], sm.by_sum[128 + r]));
          k0 = l == 0.f ? 0.f : x.own;
          k1 = x.prefix;
          m = x.top;
          l = x.sum;
        }
      }
      Both w2{};
      if (SHARED && alone && before && real) w2 = both_parts(m, l, a.rows_ms[shared_row]);
      const bool add = SHARED && alone && before;
      // what comes before the rounding: out of the sums here, and out of the prefix's
      const float inv_own = add ? (w2.sum == 0.f ? 0.f : w2.own / w2.sum) : l == 0.f ? 0.f : 1.f / l;
      const float inv_prefix = add && w2.sum != 0.f ? w2.prefix / w2.sum : 0.f;
      T* out = reinterpret_cast<T*>(a.q.out) + static_cast<int64_t>(it.span.first + token) * a.q.out_token +
               static_cast<int64_t>(head) * a.q.out_head;
      if (active && !(both && t == 1)) {
#pragma unroll 1
        for (int e = 0; e < D / 32; ++e) {
          uint32_t y[32];
          if (tiles) {
            tc_ld32(o_col + 32 * e, y);
            tc_wait_ld(y);
          } else {
#pragma unroll
            for (int f = 0; f < 32; ++f) y[f] = 0;
          }
          if (both) {
#pragma unroll
            for (int f = 0; f < 8; ++f) {
              const float4 x = across[(8 * e + f) * 128 + r];
              const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) y[4 * f + i] = __float_as_uint((k0 == 0.f ? 0.f : k0 * __uint_as_float(y[4 * f + i])) + k1 * xs[i]);
            }
          }
          if (real) {
#pragma unroll
            for (int f = 0; f < 4; ++f) {  // eight columns, and the dims that they are
              constexpr int order[8] = {0, 4, 1, 5, 2, 6, 3, 7};
              float z[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) z[BITS == 4 ? order[i] : i] = __uint_as_float(y[8 * f + i]);
              if (l == 0.f)
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = 0.f;
              const int d = 32 * e + 8 * f;
              if (!alone) {
                float* to = a.part + (part + lr) * D + d;
                *reinterpret_cast<float4*>(to) = make_float4(z[0], z[1], z[2], z[3]);
                *reinterpret_cast<float4*>(to + 4) = make_float4(z[4], z[5], z[6], z[7]);
              } else if (SHARED && !a.behind) {
                float* to = a.rows + shared_row * D + d;
                *reinterpret_cast<float4*>(to) = make_float4(z[0], z[1], z[2], z[3]);
                *reinterpret_cast<float4*>(to + 4) = make_float4(z[4], z[5], z[6], z[7]);
              } else {
                if (SHARED && add) {
                  const float* from = a.rows + shared_row * D + d;
                  const float4 y0 = *reinterpret_cast<const float4*>(from), y1 = *reinterpret_cast<const float4*>(from + 4);
                  const float y[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
                  for (int i = 0; i < 8; ++i) z[i] = z[i] * inv_own + y[i] * inv_prefix;
                }
                const float inv = SHARED && add ? 1.f : inv_own;
                const uint32_t w[4] = {P::pack(z[0] * inv, z[1] * inv), P::pack(z[2] * inv, z[3] * inv), P::pack(z[4] * inv, z[5] * inv),
                                       P::pack(z[6] * inv, z[7] * inv)};
                if (a.out_wide) {
                  *reinterpret_cast<uint2*>(out + d) = make_uint2(w[0], w[1]);
                  *reinterpret_cast<uint2*>(out + d + 4) = make_uint2(w[2], w[3]);
                } else {
#pragma unroll
                  for (int i = 0; i < 8; ++i) out[d + i] = Elem<T>::from(z[i] * inv);
                }
              }
            }
          }
        }
        if (real) {
          if (!alone) a.part_ms[part + lr] = make_float2(m, l);
          else if (SHARED && !a.behind) a.rows_ms[shared_row] = make_float2(m, l);
          else if (SHARED && add) {
            if (a.lse) a.lse[shared_row] = (w2.top + log2f(w2.sum)) * 0.6931471805599453f;
          } else if (a.lse) a.lse[static_cast<uint64_t>(it.span.first + token) * a.heads + head] = (m + log2f(l)) * 0.6931471805599453f;
        }
      }
      tc_fence_before();  // O is read before the next item's products are let through (by q_full)
      if (both) bar_sync<1, kTcSoftmax>();  // Q's place is read
    }
  } else if (BITS < 16 && warp < kIssuer) {
    // ---------------------------------------------------------------- unpackers of keys (v = 0) and of values (v = 1)
    if constexpr (BITS < 16) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcRegsUnpack));
      const uint32_t v = warp / 4 - kTcSoftmax / 128, w = warp % 4;  // warp w has tokens 16 w and on
      // A lane's 16-byte units of its warp's tokens, so that neither its reads (rows as the pages have them) nor its writes
      // (128-byte swizzle) meet a bank twice: eight lanes read 128 bytes in a row, or the halves of two rows that lie so,
      // and write to eight different units of a row.
      constexpr int kRowUnits = S::kRow / 16, kTurns = kRowUnits / 2;
      Turn<kStages> to_stage;
      Turn<kRaw> from_raw;
      bool first = true;  // the stages have not been used yet
      {
#pragma unroll 1
        for (;;) {
          const uint32_t st = to_stage.i, slot = from_raw.i;
          if (!first) ok = tc_wait(&sm.empty[v][st], to_stage.parity ^ 1, stop);
          ok = __all_sync(0xffffffffu, ok && tc_wait(&sm.raw_full[v][slot], from_raw.parity, stop));
          if (!ok || sm.raw_bits[v][slot][2]) break;
          const uint32_t bits = sm.raw_bits[v][slot][w / 2] >> (16 * (w % 2));
          const char* const raw_rows = sm.raw[v][slot] + w * 16 * S::kRow;
          const uint16_t* const words = reinterpret_cast<const uint16_t*>(sm.raw_words[v][slot]) + w * 16 * (D / 64);
          char* const rows = sm.kv[v][st] + w * 16 * 128;
          from_raw.next();
          to_stage.next();
          first = first && to_stage.i != 0;
          const auto place = [&](int e, uint32_t& tok, uint32_t& unit) {
            if (kRowUnits == 8) {
              tok = 8 * (e / 2) + lane / 4;
              unit = lane % 4 + 4 * ((lane / 4 + e) & 1);
            } else {
              tok = e * (32 / kRowUnits) + lane / kRowUnits;
              unit = lane % kRowUnits;
            }
          };
          // all reads before any write: the compiler cannot tell that they do not meet
          uint4 y[kTurns];
          uint32_t word[kTurns];
#pragma unroll
          for (int e = 0; e < kTurns; ++e) {
            uint32_t tok, unit;
            place(e, tok, unit);
            y[e] = *reinterpret_cast<const uint4*>(raw_rows + tok * S::kRow + unit * 16);
            word[e] = words[tok * (D / 64) + unit * (128 / BITS) / 64];
            if (!(bits >> tok & 1u)) word[e] = 0;  // the scale of nothing is zero
          }
#pragma unroll
          for (int e = 0; e < kTurns; ++e) {
            uint32_t tok, unit;
            place(e, tok, unit);
            const uint32_t d = unit * (128 / BITS);  // the unit's first dim
            const std::conditional_t<BITS == 8, Bytes<T>, Unpack<T>> u(word[e]);
            char* const to = rows + d / 64 * S::kBlock + tok * 128;
            const uint32_t ws[4] = {y[e].x, y[e].y, y[e].z, y[e].w};
            if constexpr (BITS == 8) {
#pragma unroll
              for (int f = 0; f < 2; ++f) {
                const uint2 a0 = u(ws[2 * f]), a1 = u(ws[2 * f + 1]);
                *reinterpret_cast<uint4*>(to + ((d % 64 / 8 + f) ^ (tok & 7)) * 16) = make_uint4(a0.x, a0.y, a1.x, a1.y);
              }
            } else {
#pragma unroll
              for (int f = 0; f < 4; ++f) {
                // the second 64 dims' units in another order: their lanes write at the same time
                const bool other = D == 128 && unit >= 2;
                const uint32_t g = other ? f ^ 2 : f, x = other ? ws[f ^ 2] : ws[f];
                *reinterpret_cast<uint4*>(to + ((d % 64 / 8 + g) ^ (tok & 7)) * 16) = u(x);
              }
            }
          }
          fence_async_shared();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(shared_address(&sm.full[v][st]));
            mbar_arrive(shared_address(&sm.raw_empty[v][slot]));
          }
        }
      }
    }
  } else {
    if constexpr (BITS < 16) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcRegsIssuer));
    if (warp < kLoader) {
      // -------------------------------------------------------------- products: S (v = 0), or O (v = 1)
      // What the warp goes by is brought to where all lanes' common values live (by reductions over them), so that the
      // operands of a product take an addition there and no way of their own.
      const uint32_t leader = tc_leader(), t_mem = __reduce_max_sync(0xffffffffu, tmem);
      const auto products = [&](auto kind) {
        constexpr uint32_t v = decltype(kind)::value;
        constexpr uint32_t kQK = tc_idesc<T>(128, kTile, false), kPV = tc_idesc<T>(128, D, true);
        constexpr uint32_t kStep = S::kBlock * (D / 64) / 16;  // from one stage's descriptor to the next's
        const uint32_t kv = tc_desc(shared_address(sm.kv[v][0]), v ? S::kBlock : 16);
        uint32_t q_parity = 0;  // a bit for each stream
        Turn<kTcInfo> told;
        Turn<kStages> at;  // keys or values to come
        Turn<2> s[2];      // S to be written, or P to be read
#pragma unroll 1
        for (;;) {
          if (!__all_sync(0xffffffffu, tc_wait(&sm.info_full[told.i], told.parity, stop))) return false;
          const TcInfo& info = sm.info[told.i];
          const uint32_t flags = __reduce_or_sync(0xffffffffu, info.flags), j = __reduce_max_sync(0xffffffffu, info.j);
          if (flags & kTcEnd) return true;
          const bool both = flags & kTcBoth;
          const uint32_t i = both ? j / 2 : j;  // of the stream's tiles of the item
          if (!__all_sync(0xffffffffu, tc_wait(&sm.full[v][at.i], at.parity, stop))) return false;
          if (BITS == 16 && v == 1) {
            const uint32_t bits0 = info.bits[0], bits1 = info.bits[1];
            if (__any_sync(0xffffffffu, (bits0 & bits1) != ~0u)) {
#pragma unroll 1
              for (uint32_t e = lane; e < kTile * (D / 8); e += 32) {
                const uint32_t tok = e / 8 % kTile;
                if (!((tok < 32 ? bits0 : bits1) >> (tok % 32) & 1u))
                  *reinterpret_cast<uint4*>(sm.kv[1][at.i] + e / 8 / kTile * S::kBlock + tok * 128 + e % 8 * 16) = make_uint4(0, 0, 0, 0);
              }
              fence_async_shared();
              __syncwarp();
            }
          }
          told.next();
          const uint32_t x = kv + at.i * kStep;
#pragma unroll
          for (uint32_t t = 0; t < 2; ++t) {
            if (both ? j % 2 != t : t == 1 && !(flags & kTcSecond)) continue;
            bool there = true;
            if (v == 1) {
              there = tc_wait(&sm.p_full[t][s[t].i], s[t].parity, stop);
            } else if (i == 0) {
              there = tc_wait(&sm.q_full[t], q_parity >> t, stop);
              q_parity ^= 1u << t;
            } else if (i > 1) {  // this S holds the P of two tiles before
              there = tc_wait(&sm.o_full[t][s[t].i], s[t].parity ^ 1, stop);
            }
            if (!__all_sync(0xffffffffu, there)) return false;
            tc_fence_after();
            const uint32_t y = t_mem + 2 * D + (2 * t + s[t].i) * kTile;
            if (v == 0) {
              const uint32_t q = tc_desc(shared_address(sm.q[t]), 16);
#pragma unroll
              for (int e = 0; e < D / 16; ++e)
                tc_mma_ss(leader, y, q + (e / 4) * (S::kBlockQ / 16) + (e % 4) * 2, x + (e / 4) * (S::kBlock / 16) + (e % 4) * 2, kQK, e > 0);
              tc_commit(leader, &sm.s_full[t][s[t].i]);
            } else {
#pragma unroll
              for (int e = 0; e < static_cast<int>(kTile) / 16; ++e)
                tc_mma_ts(leader, t_mem + t * D, y + e * 8, x + e * (2048 / 16), kPV, i % kTcChain<T> != 0 || e > 0);
              tc_commit(leader, &sm.o_full[t][s[t].i]);
            }
            s[t].next();
          }
          tc_commit(leader, &sm.empty[v][at.i]);
          at.next();
        }
      };
      ok = warp == kIssuer ? products(std::integral_constant<uint32_t, 0>()) : products(std::integral_constant<uint32_t, 1>());
      // what was issued, and its arrivals, finish before the tensor memory goes and the CTA ends: waited for even when
      // another wait has run out
      tc_commit(leader, &sm.drained);
      if (!tc_wait(&sm.drained, 0, nullptr)) atomicOr(b.err, kKvErrWait);
      __syncwarp();
    } else if (warp < kLoader + 2) {
      // -------------------------------------------------------------- loaders of keys (v = 0) and of values (v = 1)
      const uint32_t v = warp - kLoader, leader = tc_leader();
      const uint32_t shift = b.page_shift, per = min(1u << shift, kTile);  // tokens of one copy
      const uint32_t block = lane % 4;                                     // of 16 tokens, whose page the lane looks up
      const uint32_t base = shared_address(BITS < 16 ? sm.raw[v][0] : sm.kv[v][0]), base_words = shared_address(sm.raw_words[v][0]);
      uint64_t* const bars = BITS < 16 ? sm.raw_full[v] : sm.full[v];
      uint64_t* const frees = BITS < 16 ? sm.raw_empty[v] : sm.empty[v];
      constexpr uint32_t kSlots = BITS < 16 ? kRaw : kStages;
      uint32_t n = 0;  // tiles so far
      Turn<kSlots> to_slot;
      Turn<kTcInfo> tell;
      while (ok && walk.next(it)) {
        const uint32_t tiles = it.hi - it.lo;
        const int32_t* table = b.table + static_cast<uint64_t>(it.seq) * b.table_stride;
        const uint32_t length = it.span.length;
        // the fewest tokens that a row of the item sees
        int32_t all_see = length;
        if (a.causal) {
          const int64_t x = static_cast<int64_t>(length) - it.span.count + it.rb * kTcRows / a.group + 1;
          all_see = x > 0 ? static_cast<int32_t>(x) : 0;
        }
        // A tile takes two loads one after the other where there is a mask (its number, then pages and mask): numbers are
        // asked for three tiles ahead and the others two, so that nobody waits for them. (Common loads, not those of constant
        // data: this kernel is resident while the one before writes the list, or the caller's mask.)
        const uint32_t flags = (streamed(it) ? kTcBoth : 0) | (it.span.count * a.group - it.rb * kTcRows > 128 ? kTcSecond : 0);
        struct Look {
          uint32_t pos, page;   // the tile's first token; the page of the lane's block of 16, n_pages or above where there is none
          uint32_t see0, see1;  // of tokens pos + lane and pos + 32 + lane
        };
        const uint32_t* const listed = a.tiles ? a.tiles + tile_list<SHARED>(a, it.seq, it.rb) * a.tile_stride + it.lo : nullptr;
        const auto unit_of = [&](uint32_t j) { return j >= tiles ? ~0u : listed ? listed[j] : it.lo + j; };
        const auto look = [&](uint32_t unit) {
          Look x{unit == ~0u ? 0u : unit * kTile, ~0u, 0, 0};
          if (unit == ~0u) return x;
          const uint32_t p = x.pos + 16 * block, p0 = x.pos + lane, p1 = p0 + 32;
          if (p < length) x.page = static_cast<uint32_t>(table[p >> shift]);
          if (SHARED && a.seq_words) {
            const uint64_t word = a.any_words[static_cast<uint64_t>(it.seq) * a.tile_stride + unit];
            x.see0 = p0 < length ? static_cast<uint32_t>(word >> lane) & 1u : 0u;
            x.see1 = p1 < length ? static_cast<uint32_t>(word >> 32 >> lane) & 1u : 0u;
          } else if (a.mask) {
            const uint8_t* mask = a.mask + it.seq * a.mask_stride;
            x.see0 = p0 < length && p0 < a.mask_stride ? mask[p0] : 0u;
            x.see1 = p1 < length && p1 < a.mask_stride ? mask[p1] : 0u;
          } else {
            x.see0 = p0 < length;
            x.see1 = p1 < length;
          }
          return x;
        };
        uint32_t unit = unit_of(2);
        Look ahead[2] = {look(unit_of(0)), look(unit_of(1))};
#pragma unroll 1
        for (uint32_t j = 0; j < tiles; ++j, ++n) {
          const Look x = ahead[0];
          ahead[0] = ahead[1];
          ahead[1] = look(unit);
          unit = unit_of(j + 3);
          uint32_t bits0 = __ballot_sync(0xffffffffu, x.see0 != 0), bits1 = __ballot_sync(0xffffffffu, x.see1 != 0);
          const uint32_t there = __ballot_sync(0xffffffffu, x.page < b.n_pages);  // lanes whose block has a page
          if ((bits0 & bits1) != ~0u || (there & 15u) != 15u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t& bits = e < 2 ? bits0 : bits1;
              const uint32_t mine = 0xFFFFu << (16 * (e % 2));
              if ((bits & mine) && !(there >> e & 1u)) {
                if (lane == 0) atomicOr(b.err, kKvErrPage);
                bits &= ~mine;
              }
            }
          }
          const uint32_t slot = to_slot.i;
          if (n >= kSlots) ok = __all_sync(0xffffffffu, tc_wait(&frees[slot], to_slot.parity ^ 1, stop));
          if (!ok) break;
          to_slot.next();
          if (v == 0 && lane == 0) {
            TcInfo& info = sm.info[tell.i];
            info.bits[0] = bits0;
            info.bits[1] = bits1;
            info.pos = static_cast<int32_t>(x.pos);
            info.plain = (bits0 & bits1) == ~0u && static_cast<int32_t>(x.pos + kTile) <= all_see;
            info.j = j;
            info.flags = flags;
            mbar_arrive(shared_address(&sm.info_full[tell.i]));
          }
          tell.next();
          // a copy is made where any of its blocks is seen (its page, which all of them have, is there then)
          const uint64_t mine = per == kTile ? ~0ull : (1ull << per) - 1;
          const auto wanted = [&](uint32_t e) { return ((static_cast<uint64_t>(bits1) << 32 | bits0) >> e & mine) != 0; };
          uint32_t copies = (bits0 | bits1) != 0;
          if (per != kTile) {
            copies = 0;
            for (uint32_t e = 0; e < kTile; e += per) copies += wanted(e);
          }
          const uint32_t bar = shared_address(&bars[slot]);
          if (BITS < 16 && leader) {
            sm.raw_bits[v][slot][0] = bits0;
            sm.raw_bits[v][slot][1] = bits1;
            sm.raw_bits[v][slot][2] = 0;
          }
          arrive_expecting(leader, bar, copies * per * (S::kRow + (BITS < 16 ? S::kRowWords : 0)));
          const uint32_t place = x.pos & ((1u << shift) - 1);
#pragma unroll 1
          for (uint32_t e = 0; e < kTile; e += per) {
            if (!wanted(e)) continue;
            const uint32_t page = __shfl_sync(0xffffffffu, x.page, e / 16);
            if constexpr (BITS < 16) {
              const uint64_t row = ((static_cast<uint64_t>(page) * b.kv_heads + it.head) << shift) + place;
              bulk_copy(leader, base + slot * (kTile * S::kRow) + e * S::kRow, (v ? a.v : a.k) + row * S::kRow, per * S::kRow, bar);
              bulk_copy(leader, base_words + slot * (kTile * S::kRowWords) + e * S::kRowWords, (v ? a.v_words : a.k_words) + row * (D / 64),
                        per * S::kRowWords, bar);
            } else {
#pragma unroll
              for (int h = 0; h < D / 64; ++h)
                box_copy(leader, base + (slot * (D / 64) + h) * S::kBlock + e * 128, v ? &a.v_map : &a.k_map, 64 * h,
                         static_cast<int32_t>((it.head << shift) + place), static_cast<int32_t>(page), bar);
            }
          }
        }
      }
      if (ok && v == 0 && lane == 0) {
        sm.info[tell.i].flags = kTcEnd;
        mbar_arrive(shared_address(&sm.info_full[tell.i]));
      }
      if (BITS < 16 && ok) {
        if (n >= kSlots) ok = __all_sync(0xffffffffu, tc_wait(&frees[to_slot.i], to_slot.parity ^ 1, stop));
        if (ok && leader) {
          sm.raw_bits[v][to_slot.i][2] = 1;
          mbar_arrive(shared_address(&bars[to_slot.i]));
        }
      }
      if (!ok)  // copies in flight land before the CTA ends
        for (uint32_t i = n > kSlots ? n - kSlots : 0; i < n; ++i) tc_wait(&bars[i % kSlots], i / kSlots, nullptr);
    }
  }
  if (!ok) atomicOr(b.err, kKvErrWait);
  tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// Joins the parts of the items that lie in more than one CTA's range: a CTA to
// some rows of the item that goes on from CTA blockIdx.x, D / 4 lanes to a row.
// In a launch of its own, because the ranges end at the same time: the CTA that
// ended last, joining 19 parts of 128 rows alone, took 80 us.
constexpr int kJoinThreads = 512;
template <int D>
constexpr uint32_t kJoinRows = kJoinThreads / (D / 4);
// FEW: as many CTAs as the call says that it has rows for, which go on with what others there are. (CTAs that find nothing to
// join cost their launch: eight sequences of 64 tokens of 4 bits under 36 rows, in tables of 4096, 15.4 us with 16 to an item,
// 12.8 with 3. A question over bytes, 279 us, takes 281 by CTAs that could go on. Four to an SM: with more registers, and fewer
// at a time, 32 sequences of 1111 tokens took 5 % more.)
template <typename T, int D, bool SHARED, bool FEW>
__global__ void __launch_bounds__(kJoinThreads, 4) attend_join(const __grid_constant__ AttendArgs a) {
  using P = Pair<T>;
  constexpr uint32_t kLanes = D / 4;
  pdl_trigger();
  pdl_wait();
  const SplitItem it = a.items[blockIdx.x];
  if (it.last_cta <= blockIdx.x) return;
  const uint32_t all = min(kManyRows, it.span.count * a.group - it.rb * kManyRows);
  const uint32_t lane = threadIdx.x % kLanes, parts = it.last_cta - blockIdx.x + 1;
  const auto join = [&](uint32_t row0) {
    const uint32_t row = row0 + threadIdx.x / kLanes;
    const bool real = row < all;  // (whole warps go on, for the shuffles)
    const auto part_at = [&](uint32_t i) { return (2ull * (blockIdx.x + i) + (i == 0)) * kManyRows + (real ? row : 0); };
    float top = -INFINITY, sum = 0.f;
    for (uint32_t i = lane; i < parts; i += kLanes) top = fmaxf(top, a.part_ms[part_at(i)].x);
#pragma unroll
    for (uint32_t o = 1; o < kLanes; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (uint32_t p0 = 0; p0 < parts; p0 += kLanes) {
      float k = 0.f;
      if (p0 + lane < parts) {
        const float2 z = a.part_ms[part_at(p0 + lane)];
        k = z.x == -INFINITY ? (z.y == 0.f ? 0.f : 1.f) : exp2_fast(z.x - top);
        sum += z.y == 0.f ? 0.f : k * z.y;
      }
      const uint32_t n = min(kLanes, parts - p0);
#pragma unroll 8
      for (uint32_t i = 0; i < n; ++i) {
        const float by = __shfl_sync(0xffffffffu, k, i, kLanes);
        const float4 z = *reinterpret_cast<const float4*>(a.part + part_at(p0 + i) * D + lane * 4);
        y.x += by * z.x, y.y += by * z.y, y.z += by * z.z, y.w += by * z.w;
      }
    }
#pragma unroll
    for (uint32_t o = 1; o < kLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (!real) return;
    const uint32_t token = it.span.first + (it.rb * kManyRows + row) / a.group, head = it.head * a.group + (it.rb * kManyRows + row) % a.group;
    const uint64_t at = static_cast<uint64_t>(token) * a.heads + head;
    float by = sum == 0.f ? 0.f : 1.f / sum, lse = top + log2f(sum);
    if constexpr (SHARED) {
      float4* const there = reinterpret_cast<float4*>(a.rows + at * D) + lane;
      if (!a.behind) {
        *there = y;
        if (lane == 0) a.rows_ms[at] = make_float2(top, sum);
        return;
      }
      if (has_prefix(a, it.seq)) {
        const Both w = both_parts(top, sum, a.rows_ms[at]);
        const float4 z = *there;
        y = make_float4(w.own * y.x + w.prefix * z.x, w.own * y.y + w.prefix * z.y, w.own * y.z + w.prefix * z.z, w.own * y.w + w.prefix * z.w);
        by = w.sum == 0.f ? 0.f : 1.f / w.sum;
        lse = w.top + log2f(w.sum);
      }
    }
    T* const out = reinterpret_cast<T*>(a.q.out) + static_cast<int64_t>(token) * a.q.out_token + static_cast<int64_t>(head) * a.q.out_head + lane * 4;
    if (a.out_wide) {
      *reinterpret_cast<uint2*>(out) = make_uint2(P::pack(y.x * by, y.y * by), P::pack(y.z * by, y.w * by));
    } else {
      out[0] = Elem<T>::from(y.x * by);
      out[1] = Elem<T>::from(y.y * by);
      out[2] = Elem<T>::from(y.z * by);
      out[3] = Elem<T>::from(y.w * by);
    }
    if (a.lse && lane == 0) a.lse[at] = lse * 0.6931471805599453f;
  };
  const uint32_t first = blockIdx.y * kJoinRows<D>;
  if constexpr (FEW) {
#pragma unroll 1
    for (uint32_t row0 = first; row0 < all; row0 += gridDim.y * kJoinRows<D>) join(row0);
  } else if (first < all) {
    join(first);
  }
}

// One CTA to an SM, whose tensor memory it takes whole: more than half of its shared memory.
template <int D, int BITS, bool SHARED>
constexpr size_t tc_smem() {
  static_assert(sizeof(TcSmem<D, BITS, SHARED>) + 1024 <= 227 * 1024, "an SM's shared memory");
  return sizeof(TcSmem<D, BITS, SHARED>) + 1024 > 120 * 1024 ? sizeof(TcSmem<D, BITS, SHARED>) + 1024 : 120 * 1024;
}

}  // namespace
}  // namespace cofie

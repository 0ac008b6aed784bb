// Attention of many query rows over the cache (questions, prompts): the
// products bound it, so both run on tcgen05.
//
// A CTA takes up to 256 query rows (new tokens x heads of the group) of one
// key/value head as two tiles of 128, and the cached tokens 64 at a time:
//   softmax    four warps a tile, a thread to a row: maximum, exponentials, P
//              back into S's place in 16 bits; at the end O out
//   producers  four warps for keys, four for values: the next tokens into shared
//              memory (128-byte swizzle), copied (16 bits) or unpacked to
//              (n - z) s, which the 16-bit types hold exactly (4 bits)
//   MMA        a warp for each tile: S = Q K^T into tensor memory (128 x 64 fp32 a tile),
//              and O += P V with P read from tensor memory
// The running maximum that exponentials refer to is raised only when the true
// one passes it by 2^8 (2^4 for fp16; then O is brought down in tensor memory),
// which seldom happens after the first tokens. O itself is read out and begun
// anew after some thousands of tokens (kTcChain).
//
// Tensor memory: O0 O1 (D columns each) and for each tile two S of 64 columns,
// P in the first 32 of its S: while the softmax works on one S, the products
// of the next tokens fill the other. With one S of 128 tokens a tile, the
// softmax waited 2300 of 5900 cycles for P V and the next Q K^T to be done
// (256 new tokens over 65792 cached ones of 4 bits: 376 us).
//
// For each 256 x 128 block of the scores the tensor core needs 2048 cycles (head
// of 128), shared memory 2048 for its operands and 512 for writing them, the
// exponentials 1024 and more.
#pragma once

#include "kv_split.cuh"
#include "ngff_device.cuh"

namespace cofie {
namespace {

constexpr int kTcRows = 256;
constexpr int kTcSoftmax = 256;    // threads: warps 0 to 7
constexpr int kTcProducers = 128;  // for keys, and as many for values
constexpr int kTcThreads = kTcSoftmax + 2 * kTcProducers + 128;  // and a group of four warps with the one that issues
constexpr int kTcStages = 4;       // of keys, and of values
constexpr int kTcInfo = 8;         // more than the stages: a tile is told before its place is free
constexpr int kTcRaw = 3;          // codes as they lie in the pages
// Tiles whose products are summed in tensor memory before the sums move on to the CTA's part. The tensor core cuts each
// product off at about 2^-24 of the sum that it is added to, so 8192 tokens may cost a sum 2^-11 of its size, a rounding
// of fp16, and 65536 tokens 2^-8, one of bf16. (In one sum, 262144 tokens 14 to 17 below a first one came out 0.4 to
// 0.5 % low.)
template <typename T>
constexpr uint32_t kTcChain = std::is_same<T, __half>::value ? 128 : 1024;
constexpr uint64_t kTcTimeout = 1000000000ull;
// Registers: all threads start with 96; 256 x 136 + 256 x 72 + 128 x 64 is 640 x 96.
constexpr int kTcRegsSoftmax = 136, kTcRegsProducer = 72, kTcRegsIssuer = 64;

struct TcInfo {
  uint32_t bits[2];  // tokens that some row may see
  int32_t pos;       // the first token
  uint32_t plain[2]; // every token of the half is seen by every row
};

template <int D, int BITS>
struct TcSmem {
  static constexpr int kBlockQ = 128 * 128;  // 128 rows of 64 values
  static constexpr int kBlock = kTile * 128;  // 64 rows of 64 values
  union {
    char q[2][kBlockQ * (D / 64)];
    Plan<kTcThreads> plan;  // until every thread has its walk
  };
  char kv[2][kTcStages][kBlock * (D / 64)];  // keys, values
  char raw[2][BITS == 4 ? kTcRaw : 1][BITS == 4 ? kTile * (D / 2) : 16];
  uint32_t raw_word[2][kTcRaw][kTcProducers];
  uint64_t row_of[2][BITS == 4 ? 1 : kTcStages][kTile];  // 16 bits: the tokens' rows in the pages, ~0 where there is nothing
  Span spans[kSpans];
  TcInfo info[kTcInfo];
  float by_sum[kTcRows];
  uint64_t full[2][kTcStages], empty[2][kTcStages];  // keys, values
  // A barrier's phase can be told from the one before only. O is ready twice before anyone has to look, so it has a
  // barrier for even tiles and one for odd ones, as S and P have.
  uint64_t info_full[kTcInfo], q_full[2], s_full[2][2], p_full[2][2], o_full[2][2], drained;
  uint32_t tmem, stop, last_here;
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

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
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

template <typename T, int D, int BITS>
__global__ void __launch_bounds__(kTcThreads, 1) attend_rows_tc(const __grid_constant__ AttendArgs a) {
  using P = Pair<T>;
  using S = TcSmem<D, BITS>;
  // fp16: weights are 2^7 times what they stand for, so that only those under 2^-32 of the largest are lost to the second
  // product, and the maximum that they refer to is never more than 2^4 behind: up to 2^11, the exponents above left for a
  // maximum that is a rounding of a large score off. (bf16 has the exponents of fp32.)
  constexpr bool kHalf = std::is_same<T, __half>::value;
  constexpr float kRaise = kHalf ? 4.f : 8.f, kUp = kHalf ? 7.f : 0.f, kDown = kHalf ? 0x1p-7f : 1.f;
  extern __shared__ char raw[];
  S& sm = *reinterpret_cast<S*>(raw + (1024u - (shared_address(raw) & 1023u)) % 1024u);
  pdl_trigger();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  constexpr uint32_t kIssuer = (kTcSoftmax + 2 * kTcProducers) / 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kTcStages; ++i)
      for (int v = 0; v < 2; ++v) {
        mbar_init(shared_address(&sm.full[v][i]), kTcProducers / 32);
        mbar_init(shared_address(&sm.empty[v][i]), 2);  // both issuers
      }
    for (int i = 0; i < kTcInfo; ++i) mbar_init(shared_address(&sm.info_full[i]), 2);
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
  Walk<kTcThreads> walk(a, sm.plan, sm.spans, kTcRows, range);
  __syncthreads();
  const BatchArg& b = a.batch;
  Item it;
  uint32_t* stop = &sm.stop;
  bool ok = true;

  if (warp < kTcSoftmax / 32) {
    // ---------------------------------------------------------------- softmax: thread r of tile t has row r of it
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTcRegsSoftmax));
    const uint32_t t = warp / 4, r = threadIdx.x % 128;
    const uint32_t lanes = (warp % 4) * 32u << 16;
    const uint32_t o_col = o_at(t) + lanes;
    const float by = a.scale * 1.4426950408889634f;
    uint32_t n = 0, s_n = 0;  // tiles told; tiles of this half
    while (walk.next(it)) {  // to the end even when a wait ran out: the barriers below count on all
      const uint32_t row0 = it.rb * kTcRows + t * 128, all = it.span.count * a.group;
      const uint32_t tiles = it.hi - it.lo;
      const bool active = row0 < all, real = row0 + r < all;
      const uint32_t token = real ? (row0 + r) / a.group : 0, head = it.head * a.group + (real ? (row0 + r) % a.group : 0);
      int32_t seen = 0;
      if (real) {
        const int64_t x = a.causal ? static_cast<int64_t>(it.span.length) - it.span.count + token + 1 : it.span.length;
        seen = x > 0 ? static_cast<int32_t>(x) : 0;
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
#pragma unroll 1
        for (uint32_t j = 0; j < tiles; ++j, ++n, ++s_n) {
          const TcInfo& info = sm.info[n % kTcInfo];
          // S first: after an item in which this half had no rows, info may be some phases behind until then
          ok = ok && tc_wait(&sm.s_full[t][s_n % 2], s_n / 2, stop) && tc_wait(&sm.info_full[n % kTcInfo], n / kTcInfo, stop);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) {
            n += tiles - j;
            break;
          }
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
          uint32_t x[32], y[32];
          tc_ld32(s_col, x);
          tc_ld32(s_col + 32, y);
          tc_wait_ld(x);
          tc_wait_ld(y);
          if (!(info.plain[0] & info.plain[1])) {
            // hides those of 32 tokens that this row does not see
            const int32_t k = seen - info.pos;  // the row sees the first k
            const uint32_t see0 = info.bits[0] & (k >= 32 ? ~0u : k <= 0 ? 0u : (1u << k) - 1);
            const uint32_t see1 = info.bits[1] & (k >= 64 ? ~0u : k <= 32 ? 0u : (1u << (k - 32)) - 1);
            if (!__all_sync(0xffffffffu, (see0 & see1) == ~0u)) {
#pragma unroll
              for (int f = 0; f < 32; ++f) {
                if (!(see0 & (1u << f))) x[f] = 0xff800000u;
                if (!(see1 & (1u << f))) y[f] = 0xff800000u;
              }
            }
          }
          const float top = most_of(x, y, -INFINITY) * by;
          const bool raise = top > m + kRaise || (m == -INFINITY && top > -INFINITY);
          if (__any_sync(0xffffffffu, raise)) {
            const float to = raise ? top : m, k = m == -INFINITY ? 0.f : exp2_fast(m - to);
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
          }
          const float from = m == -INFINITY ? 0.f : kUp - m;
          const uint64_t by2 = two(by, by), from2 = two(from, from);
          uint64_t l2 = two(0.f, 0.f), l3 = two(0.f, 0.f);
          const auto exponentials = [&](const uint32_t* z, uint32_t col) {
            uint32_t w[16];
#pragma unroll
            for (int f = 0; f < 16; f += 2) {
              float p0, p1, p2, p3;
              apart(fma2(two(z[2 * f], z[2 * f + 1]), by2, from2), p0, p1);
              apart(fma2(two(z[2 * f + 2], z[2 * f + 3]), by2, from2), p2, p3);
              p0 = exp2_fast(p0);
              p1 = exp2_fast(p1);
              p2 = exp2_fast(p2);
              p3 = exp2_fast(p3);
              l2 = add2(l2, two(p0, p1));
              l3 = add2(l3, two(p2, p3));
              w[f] = P::pack(p0, p1);
              w[f + 1] = P::pack(p2, p3);
            }
            tc_st16(col, w);
          };
          exponentials(x, s_col);
          exponentials(y, s_col + 16);
          float l0, l1;
          apart(add2(l2, l3), l0, l1);
          {  // l + here, whose rounding is l - (sum - took) + (here - took) to the last bit
            const float here = l0 + l1, sum = l + here, took = sum - l;
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
      // info of tiles that this half does not use
      if (!active) n += tiles;
      const bool alone = it.first_cta == it.last_cta;
      const uint64_t part = own_part();
      if (tiles > kTcChain<T> && !alone) bar_sync<1, kTcSoftmax>();  // all have what they kept, before the part is written
      const float inv = l == 0.f ? 0.f : 1.f / l;
      T* out = reinterpret_cast<T*>(a.q.out) + static_cast<int64_t>(it.span.first + token) * a.q.out_token +
               static_cast<int64_t>(head) * a.q.out_head;
      if (active) {
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
              } else {
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
          else if (a.lse) a.lse[static_cast<uint64_t>(it.span.first + token) * a.heads + head] = (m + log2f(l * kDown)) * 0.6931471805599453f;
        }
      }
      tc_fence_before();  // O is read before the next item's products are let through (by q_full)
      if (!alone) {
        bar_sync<1, kTcSoftmax>();
        const uint32_t parts = it.last_cta - it.first_cta + 1;
        if (threadIdx.x == 0) sm.last_here = part_done(a, it);
        bar_sync<1, kTcSoftmax>();
        if (sm.last_here) {
          const auto part_at = [&](uint32_t i, uint32_t row) { return (2ull * (it.first_cta + i) + (i == 0)) * kTcRows + row; };
          float top = -INFINITY, sum = 0.f;
          if (real) {
#pragma unroll 4
            for (uint32_t i = 0; i < parts; ++i) top = fmaxf(top, __ldcg(&a.part_ms[part_at(i, lr)]).x);
#pragma unroll 4
            for (uint32_t i = 0; i < parts; ++i) {
              float2* at = &a.part_ms[part_at(i, lr)];
              const float2 z = __ldcg(at);
              const float k = z.x == -INFINITY ? (z.y == 0.f ? 0.f : 1.f) : exp2_fast(z.x - top);
              sum += z.y == 0.f ? 0.f : k * z.y;
              __stcg(&at->x, k);  // the part's factor, for the threads that join it
            }
            if (a.lse) a.lse[static_cast<uint64_t>(it.span.first + token) * a.heads + head] = (top + log2f(sum * kDown)) * 0.6931471805599453f;
          }
          sm.by_sum[lr] = sum == 0.f ? 0.f : 1.f / sum;
          bar_sync<1, kTcSoftmax>();
          const uint32_t rows = min(static_cast<uint32_t>(kTcRows), all - it.rb * kTcRows);
          // eight units of four values to a thread at a time, whose loads are all on their way together (a unit's row is
          // the same for a whole warp, or half of it)
          constexpr uint32_t kUnits = 8;
          const uint32_t all_units = rows * (D / 4);
          for (uint32_t x0 = threadIdx.x; x0 < all_units; x0 += kTcSoftmax * kUnits) {
            float4 y[kUnits];
#pragma unroll
            for (int u = 0; u < kUnits; ++u) y[u] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
            for (uint32_t i = 0; i < parts; ++i) {
              const float4* from = reinterpret_cast<const float4*>(a.part + part_at(i, 0) * D) + x0;
              const float2* factor = a.part_ms + part_at(i, x0 / (D / 4));
              float4 z[kUnits];
              float k[kUnits];
#pragma unroll
              for (int u = 0; u < kUnits; ++u) {
                const bool there = x0 + u * kTcSoftmax < all_units;
                z[u] = there ? __ldcg(from + u * kTcSoftmax) : make_float4(0.f, 0.f, 0.f, 0.f);
                k[u] = there ? __ldcg(&factor[u * (kTcSoftmax / (D / 4))].x) : 0.f;
              }
#pragma unroll
              for (int u = 0; u < kUnits; ++u) {
                y[u].x += k[u] * z[u].x;
                y[u].y += k[u] * z[u].y;
                y[u].z += k[u] * z[u].z;
                y[u].w += k[u] * z[u].w;
              }
            }
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
              const uint32_t x = x0 + u * kTcSoftmax, row = x / (D / 4), d = x % (D / 4) * 4;
              if (x >= all_units) break;
              const float by_total = sm.by_sum[row];
              const uint32_t tok = (it.rb * kTcRows + row) / a.group, hd = it.head * a.group + (it.rb * kTcRows + row) % a.group;
              T* o = reinterpret_cast<T*>(a.q.out) + static_cast<int64_t>(it.span.first + tok) * a.q.out_token +
                     static_cast<int64_t>(hd) * a.q.out_head + d;
              if (a.out_wide) {
                *reinterpret_cast<uint2*>(o) =
                    make_uint2(P::pack(y[u].x * by_total, y[u].y * by_total), P::pack(y[u].z * by_total, y[u].w * by_total));
              } else {
                o[0] = Elem<T>::from(y[u].x * by_total);
                o[1] = Elem<T>::from(y[u].y * by_total);
                o[2] = Elem<T>::from(y[u].z * by_total);
                o[3] = Elem<T>::from(y[u].w * by_total);
              }
            }
          }
          bar_sync<1, kTcSoftmax>();
        }
      }
    }
  } else if (warp < kIssuer) {
    // ---------------------------------------------------------------- producers of keys (v = 0) and of values (v = 1)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcRegsProducer));
    const uint32_t v = warp / 4 - kTcSoftmax / 128, p = threadIdx.x % kTcProducers;
    const uint32_t tok = p % kTile, half = p / kTile;  // two threads to a token
    const char* const pages = v ? a.v : a.k;
    const uint16_t* const words = v ? a.v_words : a.k_words;
    uint32_t n = 0;  // tiles so far
    while (walk.next(it)) {  // to the end, as above
      const uint32_t tiles = it.hi - it.lo;
      const int32_t* table = b.table + static_cast<uint64_t>(it.seq) * b.table_stride;
      // the fewest tokens that a row of the item sees
      int32_t all_see = it.span.length;
      if (a.causal) {
        const int64_t x = static_cast<int64_t>(it.span.length) - it.span.count + it.rb * kTcRows / a.group + 1;
        all_see = x > 0 ? static_cast<int32_t>(x) : 0;
      }
      struct Token {
        uint32_t pos;  // of the tile's first
        uint64_t row;  // in the pages; ~0 where there is nothing to see
      };
      // A token's row takes two loads one after the other where there is a mask (the tile's number, then the page and the
      // mask): each is used a tile after it was asked for, so that nobody waits for it.
      struct Page {
        uint32_t pos, page, seen;
      };
      const auto unit_of = [&](uint32_t j) {
        return j >= tiles ? ~0u : a.mask ? __ldg(&a.tiles[static_cast<uint64_t>(it.seq) * a.tile_stride + it.lo + j]) : it.lo + j;
      };
      const auto page_of = [&](uint32_t unit) {
        Page x{unit == ~0u ? 0u : unit * kTile, 0, 0};
        const uint32_t pos = x.pos + tok;
        if (unit != ~0u && pos < it.span.length) {
          x.page = static_cast<uint32_t>(__ldg(&table[pos >> b.page_shift]));
          x.seen = !a.mask ? 1u : pos < a.mask_stride ? __ldg(&a.mask[it.seq * a.mask_stride + pos]) : 0u;
        }
        return x;
      };
      const auto row_of = [&](const Page& x) {
        Token y{x.pos, ~0ull};
        if (x.seen) {
          if (x.page < b.n_pages)
            y.row = ((static_cast<uint64_t>(x.page) * b.kv_heads + it.head) << b.page_shift) + ((x.pos + tok) & ((1u << b.page_shift) - 1));
          else
            atomicOr(b.err, kKvErrPage);
        }
        return y;
      };
      const auto tell = [&](const Token& x, uint32_t i) {  // what the softmax has to know of tile i
        if (v || half) return;
        TcInfo& info = sm.info[i % kTcInfo];
        const bool there = x.row != ~0ull;
        const uint32_t bits = __ballot_sync(0xffffffffu, there);
        const uint32_t plain = __all_sync(0xffffffffu, there && static_cast<int32_t>(x.pos + tok) < all_see);
        if (lane == 0) {
          info.bits[tok / 32] = bits;
          info.plain[tok / 32] = plain;
          if (tok == 0) info.pos = static_cast<int32_t>(x.pos);
          mbar_arrive(shared_address(&sm.info_full[i % kTcInfo]));
        }
      };
      if (BITS == 4) {
        // Codes are fetched three tiles ahead, each thread's to places of its own.
        constexpr uint32_t kPart = D / 64;  // 16-byte pieces of a thread: a quarter of D codes is D / 4 bytes
        const auto fetch = [&](uint32_t i, const Token& y) {
          if (y.row != ~0ull) {
            const char* from = pages + y.row * (D / 2) + half * (D / 4);
            const uint32_t to = shared_address(sm.raw[v][i % kTcRaw]) + p * 16;
#pragma unroll
            for (int e = 0; e < static_cast<int>(kPart); ++e) cp_async16(to + e * 2048, from + e * 16, true);
            // the word, or two, of the token; with one, of it and its neighbour (an even token's row is even)
            cp_async4(shared_address(&sm.raw_word[v][i % kTcRaw][p]), words + (D == 128 ? 2 * y.row : y.row & ~1ull));
          } else {
            sm.raw_word[v][i % kTcRaw][p] = 0;  // the scale of nothing is zero
          }
          cp_async_commit();
        };
        uint32_t unit[5];
        Page page[4];
        Token x[3];
#pragma unroll
        for (int i = 0; i < 5; ++i) unit[i] = unit_of(i);
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = page_of(unit[i]);
#pragma unroll
        for (int i = 0; i < 3; ++i) x[i] = row_of(page[i]);
        Page page_ahead = page[3];      // of tile j + 3
        uint32_t unit_ahead = unit[4];  // of tile j + 4
        fetch(n, x[0]);
        fetch(n + 1, x[1]);
        fetch(n + 2, x[2]);
#pragma unroll 1
        for (uint32_t j = 0; j < tiles; ++j, ++n) {
          const uint32_t st = n % kTcStages, round = n / kTcStages;
          tell(x[0], n);
          cp_async_wait<kTcRaw - 1>();
          if (round > 0) ok = ok && tc_wait(&sm.empty[v][st], round - 1, stop);
          if (ok) {
            const char* from = sm.raw[v][n % kTcRaw] + p * 16;
            const uint32_t w = sm.raw_word[v][n % kTcRaw][p];
            const Unpack<T> u(D == 64 ? (tok % 2 ? w >> 16 : w & 0xFFFFu) : (half ? w >> 16 : w & 0xFFFFu));
            char* to = sm.kv[v][st] + (D == 128 ? half * S::kBlock : 0) + tok * 128;
#pragma unroll
            for (int e = 0; e < static_cast<int>(kPart); ++e) {
              const uint4 y = *reinterpret_cast<const uint4*>(from + e * 2048);
              const uint32_t ws[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int f = 0; f < 4; ++f)
                *reinterpret_cast<uint4*>(to + (((D == 64 ? 4 * half : 0) + 4 * e + f) ^ (tok & 7)) * 16) = u(ws[f]);
            }
            fence_async_shared();
          }
          ok = __all_sync(0xffffffffu, ok);
          if (ok) warp_arrive(&sm.full[v][st]);
          x[0] = x[1], x[1] = x[2], x[2] = row_of(page_ahead);
          fetch(n + 3, x[2]);
          page_ahead = page_of(unit_ahead);
          unit_ahead = unit_of(j + 5);
        }
        cp_async_wait<0>();
      } else {
        // Copies of three tiles are on their way at a time.
        constexpr uint32_t kUnits = D / 8;  // 16-byte units of a token
        constexpr uint32_t kAhead = kTcStages - 1;
        uint32_t unit_ahead = unit_of(1);
        Page page_ahead = page_of(unit_of(0));
#pragma unroll 1
        for (uint32_t j = 0; j < tiles + kAhead - 1; ++j) {
          const uint32_t i = n + j, st = i % kTcStages, round = i / kTcStages;
          if (j < tiles) {
            const Token x = row_of(page_ahead);
            page_ahead = page_of(unit_ahead);
            unit_ahead = unit_of(j + 2);
            if (half == 0) sm.row_of[v][st][tok] = x.row;
            tell(x, i);
            if (v == 0) bar_sync<2, kTcProducers>();
            else bar_sync<3, kTcProducers>();
            if (round > 0) ok = ok && tc_wait(&sm.empty[v][st], round - 1, stop);
            if (ok) {
              const uint32_t to = shared_address(sm.kv[v][st]);
#pragma unroll 4
              for (uint32_t e = p; e < kTile * kUnits; e += kTcProducers) {
                const uint32_t tk = e / kUnits, u = e % kUnits;
                const uint64_t row = sm.row_of[v][st][tk];
                const bool live = row != ~0ull;
                cp_async16(to + (u / 8) * S::kBlock + tk * 128 + ((u % 8) ^ (tk & 7)) * 16, pages + (live ? row * (D * 2) + u * 16 : 0), live);
              }
            }
          }
          cp_async_commit();
          if (j + 1 >= kAhead) {  // the tile of two steps before is there
            cp_async_wait<kAhead - 1>();
            fence_async_shared();
            ok = __all_sync(0xffffffffu, ok);
            if (ok) warp_arrive(&sm.full[v][(i + 1 - kAhead) % kTcStages]);
          }
        }
        n += tiles;
      }
    }
    cp_async_wait<0>();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcRegsIssuer));
    if (warp < kIssuer + 2) {
      // -------------------------------------------------------------- products: a warp for each tile
      constexpr uint32_t kQK = tc_idesc<T>(128, kTile, false), kPV = tc_idesc<T>(128, D, true);
      const uint32_t leader = tc_leader(), t = warp - kIssuer;
      uint32_t n = 0, q_n = 0, s_n = 0;  // tiles so far; items and tiles of this half
      while (ok && walk.next(it)) {
        const uint32_t tiles = it.hi - it.lo, halves = it.span.count * a.group - it.rb * kTcRows > 128 ? 2 : 1;
        if (t >= halves) {  // nothing to issue, but to stay in step: a barrier's phases are told apart by their parity
          for (uint32_t j = 0; j < tiles; ++j, ++n)
            for (uint32_t v = 0; v < 2; ++v) {
              ok = ok && tc_wait(&sm.full[v][n % kTcStages], n / kTcStages, stop);
              ok = __all_sync(0xffffffffu, ok);
              if (ok) warp_arrive(&sm.empty[v][n % kTcStages]);
            }
          continue;
        }
        if (tiles == 0) continue;
        const auto qk = [&](uint32_t j) {
          const uint32_t st = (n + j) % kTcStages, i = s_n + j;
          if (j == 0) ok = ok && tc_wait(&sm.q_full[t], q_n++, stop);
          // this S holds the P of two tiles before
          if (j > 1) ok = ok && tc_wait(&sm.o_full[t][i % 2], i / 2 - 1, stop);
          ok = ok && tc_wait(&sm.full[0][st], (n + j) / kTcStages, stop);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) return;
          tc_fence_after();
          const uint32_t q = tc_desc(shared_address(sm.q[t]), 16), k = tc_desc(shared_address(sm.kv[0][st]), 16), d = s_at(t, i);
#pragma unroll
          for (int e = 0; e < D / 16; ++e)
            tc_mma_ss(leader, d, q + (e / 4) * (S::kBlockQ / 16) + (e % 4) * 2, k + (e / 4) * (S::kBlock / 16) + (e % 4) * 2, kQK, e > 0);
          tc_commit(leader, &sm.s_full[t][i % 2]);
          tc_commit(leader, &sm.empty[0][st]);
        };
        for (uint32_t j = 0; j < 2 && j < tiles; ++j) qk(j);
#pragma unroll 1
        for (uint32_t j = 0; ok && j < tiles; ++j) {
          const uint32_t st = (n + j) % kTcStages, i = s_n + j;
          ok = tc_wait(&sm.p_full[t][i % 2], i / 2, stop) && tc_wait(&sm.full[1][st], (n + j) / kTcStages, stop);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          const uint32_t v = tc_desc(shared_address(sm.kv[1][st]), S::kBlock), p = s_at(t, i);
#pragma unroll
          for (int e = 0; e < static_cast<int>(kTile) / 16; ++e) tc_mma_ts(leader, o_at(t), p + e * 8, v + e * (2048 / 16), kPV, j % kTcChain<T> != 0 || e > 0);
          tc_commit(leader, &sm.o_full[t][i % 2]);
          tc_commit(leader, &sm.empty[1][st]);
          if (j + 2 < tiles) qk(j + 2);
        }
        s_n += tiles;
        n += tiles;
      }
      // what was issued, and its arrivals, finish before the tensor memory goes and the CTA ends: waited for even when
      // another wait has run out
      tc_commit(leader, &sm.drained);
      if (!tc_wait(&sm.drained, 0, nullptr)) atomicOr(b.err, kKvErrWait);
      __syncwarp();
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

// One CTA to an SM, whose tensor memory it takes whole: more than half of its shared memory.
template <int D, int BITS>
constexpr size_t tc_smem() {
  return sizeof(TcSmem<D, BITS>) + 1024 > 120 * 1024 ? sizeof(TcSmem<D, BITS>) + 1024 : 120 * 1024;
}

}  // namespace
}  // namespace cofie

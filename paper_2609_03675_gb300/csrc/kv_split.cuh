// Attention of few query rows over the cache (single tokens and short runs of
// them): the cache's bytes bound it, so every key and value is read once for
// all the rows that share its head and stays in registers from there.
//
// Up to 8 NT rows (new tokens x heads of the group) to a CTA of eight warps.
// Each warp streams tokens of its own through a ring in shared memory
// (cp.async, no barrier with the other warps) and keeps a running maximum, sum
// and output of its own; the warps' parts are joined once, at the item's end.
//
// Both products are transposed, which puts the cache on the side of the
// 16-row operand and the few query rows on that of 8 columns:
//   S^T [16 tokens x 8 rows] = K [16 x D] Q^T,  O^T [16 dims x 8 rows] += V^T [16 x 16 tokens] P^T
// (mma.sync m16n8k16: with so few rows tcgen05's 128-row operand would be
// mostly padding, and its operands would have to be written back to shared
// memory after the codes are unpacked.) S^T leaves the tensor core as a
// fragment of tokens by rows; movmatrix turns it into P^T's.
//
// 4-bit codes enter the products as they are: a 16-bit number whose low four
// bits are the code and whose others are clear is the fp16 number n 2^-24 (a
// subnormal, which the tensor cores take like any other), and with the code
// four bits higher 16 n 2^-24. So one logic operation unpacks two codes, and
// one shift in eight of them; the 16 and the 2^24 are taken off q and the
// results. Everything else is on the side of the few rows:
//   q      is brought to fp16 by a power of two for each row (its largest
//          value in [128, 256)), which keeps bf16's and fp16's bits;
//   keys   a score is the sum over the groups of s sum q (n - z);
//   values the sum over tokens has a scale for each: p s is rounded to fp16,
//          after a power of two that keeps the largest scale of its group met
//          so far below 2^15 (raised, and the output so far brought down, when
//          a larger one comes).
// z is taken off the codes, in fp16, exactly. Taken off the sums it would cost
// half the operations, but sums near zero would carry the rounding of sums of
// codes (log-sum-exps of few tokens were off by 3e-6 of their size, not 4e-7).
// 262144 tokens, 8 heads of 128, 4 query heads each: unpacked to (n - z) s for
// values and 128 + n for keys the kernel took 108 us, its ALU pipe 70 % busy.
//
// Bytes enter likewise as fp16 numbers u - 128, made of 1024 + u (a byte beside
// 0x64) by one subtraction for two; the scales, powers of two, are on the side of
// the few rows as those of codes. 32 answers over up to 16384 tokens: 125 us, 4.7
// TB/s of DRAM, issue slots 40 % busy; with chunks of 16 tokens 135, with those
// and two CTAs to an SM 117 (but 12.6 for 11.4 over 1111 tokens, and where there
// are more than 8 rows 73 for 65), with 12 warps to a CTA 128.
#pragma once

#include <type_traits>

#include "kv_plan.cuh"

namespace cofie {
namespace {

// SHORT: a CTA of half the warps to each sequence, key head and block of rows, so that none of them is cut and two CTAs fit
// an SM.
template <bool SHORT>
constexpr int kSplitWarps = SHORT ? 4 : 8;
template <bool SHORT>
constexpr int kSplitThreads = 32 * kSplitWarps<SHORT>;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

template <typename T>
__device__ __forceinline__ T at(const char* p) {
  return *reinterpret_cast<const T*>(p);
}
__device__ __forceinline__ void ldmatrix_trans(uint32_t* r, uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T>
struct Pair;  // and their products
template <>
struct Pair<__nv_bfloat16> : Two<__nv_bfloat16> {
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Pair<__half> : Two<__half> {
  static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) {
    const __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

// The first product of a sum, in fp16.
__device__ __forceinline__ void mma_first(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// Two of a register's bytes as the fp16 numbers u - 128: 1024 + u is a byte
// beside 0x64. `which` two: 0x4140 the lower, 0x4342 the upper; or the first
// and the third.
__device__ __forceinline__ uint32_t byte_pair(uint32_t x, uint32_t which) { return Pair<__half>::sub(__byte_perm(x, 0x64646464u, which), 0x64806480u); }
__device__ __forceinline__ uint32_t byte_even(uint32_t x) { return Pair<__half>::sub((x & 0x00FF00FFu) | 0x64006400u, 0x64806480u); }

// The scales of a register of two words (the high half's, the low half's).
__device__ __forceinline__ float scale_hi(uint32_t w) { return __uint_as_float(w & 0xFFF00000u); }
__device__ __forceinline__ float scale_lo(uint32_t w) { return __uint_as_float((w << 16) & 0xFFF00000u); }

// Sizes of one warp's ring. Chunks of 32 tokens of codes or bytes, 16 of 16-bit values.
template <int D, int BITS>
struct Ring {
  static constexpr int kTokens = BITS < 16 ? 32 : 16;
  static constexpr int kRow = D * BITS / 8;                               // bytes of a token's keys
  static constexpr int kWords = BITS < 16 ? kTokens * (D / 64) * 2 : 0;   // bytes of its chunk's scale words
  static constexpr int kStage = 2 * (kTokens * kRow + kWords);
  static constexpr int kStages = 3;
  static constexpr int kWarp = kStages * kStage;
  static constexpr int kUnits = kRow / 16;                                // 16-byte units of a token
};

template <int D, int BITS, int NT, bool SHORT>
__host__ __device__ constexpr size_t split_smem() {
  const size_t warps = kSplitWarps<SHORT>, ring = warps * Ring<D, BITS>::kWarp, join = warps * 8 * NT * D * 4;
  return ring > join ? ring : join;
}

// The one sequence and key head of a SHORT CTA, block of rows by block.
struct ShortWalk {
  const AttendArgs& a;
  const uint32_t rows_per_block;
  uint32_t rb = 0;
  __device__ __forceinline__ ShortWalk(const AttendArgs& args, uint32_t rows) : a(args), rows_per_block(rows) {}
  __device__ __forceinline__ bool next(Item& it) {
    it.seq = blockIdx.x / a.batch.kv_heads;
    it.head = blockIdx.x % a.batch.kv_heads;
    if (rb == 0) it.span = sequence_span(a.batch, it.seq);
    if (static_cast<uint64_t>(rb) * rows_per_block >= static_cast<uint64_t>(it.span.count) * a.group) return false;
    it.rb = rb++;
    it.tiles = it.hi = block_tiles<true>(a, it.span, rows_per_block, it.rb, it.seq);
    it.lo = 0;
    it.first_cta = it.last_cta = blockIdx.x;
    return true;
  }
};

// Where unit u of token t lies in its chunk, such that the reads below meet no bank twice.
template <int D, int BITS, bool VALUES>
__device__ __forceinline__ uint32_t unit_at(uint32_t t, uint32_t u) {
  if (BITS == 4) return t * Ring<D, 4>::kRow + (D == 128 ? (u ^ ((t & 2u))) : u) * 16;
  if (BITS == 8) return t * Ring<D, 8>::kRow + (VALUES ? u ^ (t & (D == 128 ? 6u : 2u)) : D == 128 ? u ^ ((t & 1u) << 2) : u) * 16;
  return t * Ring<D, 16>::kRow + (VALUES ? u ^ (t & 7u) : u ^ ((t & 1u) << 2)) * 16;
}

// SHARED: over a prefix that several sequences share (a.rows), or for sequences behind one (a.behind).
template <typename T, int D, int BITS, int NT, bool SHARED, bool SHORT>
__global__ void __launch_bounds__(kSplitThreads<SHORT>, SHORT || (NT == 1 && BITS == 4) ? 2 : 1) attend_split(const __grid_constant__ AttendArgs a) {
  using P = Pair<T>;
  using H = Pair<__half>;
  using R = Ring<D, BITS>;
  constexpr int kWarps = kSplitWarps<SHORT>, kThreads = kSplitThreads<SHORT>;
  constexpr int kRows = 8 * NT, kGroups = D / 64, kM = R::kTokens / 16, kPerTile = kTile / R::kTokens;
  // 16-bit values: weights go into the second product as fp16 numbers of up to 2^8, so that only those under 2^-33 are
  // lost to it. (Up to 1, those under 2^-25 were, though not to the sum of weights: 262144 keys 17.5 below one are 0.7 %
  // of a row. The upper exponents are left for a maximum that is a rounding of a large score off. bf16 has the exponents
  // of fp32, and 4-bit values have a power of two with their scale.)
  constexpr float kUp = BITS == 16 && std::is_same<T, __half>::value ? 8.f : 0.f, kDown = kUp > 0.f ? 0x1p-8f : 1.f;
  extern __shared__ __align__(128) char smem[];
  __shared__ std::conditional_t<SHORT, char, Plan<kThreads, SHARED>> plan;
  __shared__ Span spans[SHORT ? 1 : kSpans];
  __shared__ float warp_m[kWarps][kRows], warp_l[kWarps][kRows];
  __shared__ uint2 stages[kWarps][R::kStages];  // the bits of the tokens that are seen, and the first one's place
  __shared__ uint32_t row_bits[SHARED ? kWarps : 1][R::kStages][kRows];  // and those that each row sees, where rows differ
  __shared__ float2 pieces_ms[SHORT ? 1 : kRows];
  __shared__ uint32_t last_here;
  pdl_trigger();
  pdl_wait();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
  auto walk = [&] {
    if constexpr (SHORT) {
      return ShortWalk(a, kRows);
    } else {
      const uint64_t range = plan.set_up(a, kRows, spans);
      return Walk<kThreads, SHARED, false>(a, plan, spans, kRows, range);
    }
  }();
  const char* const ring = smem + warp * R::kWarp;
  const BatchArg& b = a.batch;
  // A warp's sums o take so many tokens, as those of the kernel of many rows (kTcChain has the reason), of which it may have an
  // eighth of a long cache: an item with more of them here is worked off in pieces, and what is found so far is kept in the
  // CTA's part. (524288 fp16 tokens 2^-25 of the first: 2^-9 low in one sum. Sums moved on inside the loop over the tokens
  // cost all calls 2.6 %, up to 7.)
  constexpr uint32_t kPieceTiles = (std::is_same<T, __half>::value ? 8192 : 65536) * kWarps / kTile;
  Item it;
  uint32_t item_lo = 0, item_hi = 0;  // its tiles here; it.lo and it.hi are the piece's
  bool more = false;                  // pieces to come
  const auto next = [&] {
    if (SHORT) return walk.next(it);
    if (more) {
      it.lo = it.hi;
    } else {
      if (!walk.next(it)) return false;
      item_lo = it.lo;
      item_hi = it.hi;
    }
    it.hi = min(item_hi, it.lo + kPieceTiles);
    more = it.hi < item_hi;
    return true;
  };
  while (next()) {
    const uint32_t row0 = it.rb * kRows;
    const uint32_t rows = min(static_cast<uint32_t>(kRows), it.span.count * a.group - row0);
    // ---- the warp's chunks: warp, warp + 8, ... of the item's part. A chunk's blocks of 16 tokens lie in one page each,
    // one behind the other. The first are asked for before the queries are read.
    const uint32_t chunks = (it.hi - it.lo) * kPerTile;
    const int32_t* table = b.table + static_cast<uint64_t>(it.seq) * b.table_stride;
    const uint8_t* mask = a.mask + it.seq * a.mask_stride;
    const bool by_row = SHARED && a.seq_words;
    const bool before = SHARED && a.behind && has_prefix(a, it.seq);
    const uint64_t* row_words = nullptr;  // of row `lane`
    if (by_row && lane < rows) row_words = a.seq_words + static_cast<uint64_t>(min(static_cast<uint32_t>(a.seq_of[it.span.first + (row0 + lane) / a.group]), b.members - 1)) * a.tile_stride;
    struct Ahead {
      uint32_t pos, page[kM];  // page: n_pages and above where there is none
      bool seen;               // this lane's token
      uint32_t row;            // the tokens that row `lane` sees
    };
    const auto look = [&](uint32_t ch) {
      Ahead x;
      x.pos = 0;
      x.seen = false;
      x.row = 0;
#pragma unroll
      for (int mt = 0; mt < kM; ++mt) x.page[mt] = ~0u;
      if (ch < chunks) {
        const uint32_t t = it.lo + ch / kPerTile;
        x.pos = (a.tiles ? a.tiles[tile_list<SHARED>(a, it.seq, it.rb) * a.tile_stride + t] : t) * kTile + (ch % kPerTile) * R::kTokens;
#pragma unroll
        for (int mt = 0; mt < kM; ++mt)
          if (x.pos + 16 * mt < it.span.length) x.page[mt] = static_cast<uint32_t>(table[(x.pos + 16 * mt) >> b.page_shift]);
        const uint32_t p = x.pos + lane % R::kTokens;
        if (by_row) {
          const uint32_t tile = x.pos / kTile;
          x.seen = a.any_words[static_cast<uint64_t>(it.seq) * a.tile_stride + tile] >> (p % kTile) & 1u;
          if (row_words) x.row = static_cast<uint32_t>(row_words[tile] >> (x.pos % kTile));
        } else {
          x.seen = p < it.span.length && (!a.mask || (p < a.mask_stride && mask[p] != 0));
        }
      }
      return x;
    };
    const auto issue = [&](uint32_t stage, const Ahead& x) {
      const uint32_t base = shared_address(ring + stage * R::kStage);
      uint32_t bits = __ballot_sync(0xffffffffu, x.seen);
      if (bits) {
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
          const uint32_t half = 0xFFFFu << (16 * mt);
          if ((bits & half) && x.page[mt] >= b.n_pages) {
            if (lane == 0) atomicOr(b.err, kKvErrPage);
            bits &= BITS == 16 ? 0u : ~half;
          }
          const bool there = (bits & half) != 0;
          if (BITS < 16 && !there) continue;  // what the ring holds there is masked below
          const uint64_t row = there ? ((static_cast<uint64_t>(x.page[mt]) * b.kv_heads + it.head) << b.page_shift) +
                                           ((x.pos + 16 * mt) & ((1u << b.page_shift) - 1))
                                     : 0;
          const char* k = a.k + row * R::kRow + lane * 16;
          const char* v = a.v + row * R::kRow + lane * 16;
#pragma unroll
          for (int i = 0; i < R::kUnits / 2; ++i) {  // 32 units of 16 bytes
            const uint32_t t = (i * 32 + lane) / R::kUnits, u = lane % R::kUnits;
            // 16-bit values that nobody sees become zeros (a NaN among them would pass through a product with 0)
            const bool live = BITS < 16 || ((bits >> t) & 1u);
            cp_async16(base + unit_at<D, BITS, false>(16 * mt + t, u), k + i * 512, live);
            cp_async16(base + R::kTokens * R::kRow + unit_at<D, BITS, true>(16 * mt + t, u), v + i * 512, live);
          }
          if (BITS < 16) {  // the block's words: 16 D / 32 bytes of the keys', as many of the values'
            constexpr uint32_t kLanes = D / 32;
            static_assert(R::kWords / kM == 16 * kLanes || BITS == 16, "16 bytes to a lane");
            if (lane < 2 * kLanes) {
              const uint32_t v2 = lane / kLanes, u = lane % kLanes;
              cp_async16(base + 2 * R::kTokens * R::kRow + v2 * R::kWords + mt * (R::kWords / kM) + u * 16,
                         (v2 ? a.v_words : a.k_words) + row * (D / 64) + u * 8, true);
            }
          }
        }
      }
      if (lane == 0) stages[warp][stage] = make_uint2(bits, x.pos);
      if (SHARED && lane < kRows) row_bits[warp][stage][lane] = x.row;
      cp_async_commit();
    };
    Ahead ahead;
    {
      Ahead first[R::kStages - 1];
#pragma unroll
      for (int s = 0; s < R::kStages - 1; ++s) first[s] = look(warp + s * kWarps);
      ahead = look(warp + (R::kStages - 1) * kWarps);
#pragma unroll
      for (int s = 0; s < R::kStages - 1; ++s) issue(s, first[s]);
    }
    // ---- queries: fragments of Q^T, the columns of this lane's dims in the order in which the keys' lie in registers
    uint32_t qf[NT][D / 16][2];
    float by[NT][2];      // what takes the scores of rows 2c and 2c + 1 to base 2
    int32_t seen[NT][2];  // tokens that they may see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint32_t r = nt * 8 + g;
      const bool real = r < rows;
      const uint32_t i = (row0 + r) / a.group, j = (row0 + r) % a.group;
      const T* q = reinterpret_cast<const T*>(a.q.in) + (real ? static_cast<int64_t>(it.span.first + i) * a.q.in_token +
                                                                    static_cast<int64_t>(it.head * a.group + j) * a.q.in_head
                                                              : 0);
      uint4 x[D / 32];
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        // eight dims: 16-bit keys: unit 4 e + c of the row; codes: word e % 2 of the lane's two words in group e / 2; bytes:
        // half of its unit of that group
        const uint32_t d = BITS == 16 ? (4 * e + c) * 8 : (e / 2) * 64 + c * 16 + (e % 2) * 8;
        x[e] = make_uint4(0, 0, 0, 0);
        if (real) {
          if (a.q_wide) {
            x[e] = *reinterpret_cast<const uint4*>(q + d);
          } else {
            x[e] = gather8(q + d);
          }
        }
      }
      const float scale = a.scale * 1.4426950408889634f;
      if (BITS == 16) {
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
          qf[nt][2 * e][0] = x[e].x;
          qf[nt][2 * e][1] = x[e].y;
          qf[nt][2 * e + 1][0] = x[e].z;
          qf[nt][2 * e + 1][1] = x[e].w;
        }
        by[nt][0] = by[nt][1] = scale;
      } else {
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
          const uint32_t w[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
#pragma unroll
          for (int f = 0; f < 4; ++f) most = fmaxf(most, fmaxf(fabsf(P::lo(w[f])), fabsf(P::hi(w[f]))));
        }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        // the power of two that brings `most` to [128, 256); 1 for a row of zeros or with an infinity
        const int ex = most > 0.f && most <= 3.402823466e38f ? max(static_cast<int>(__float_as_uint(most) >> 23) - 127, -100) : 7;
        const float up = __uint_as_float(static_cast<uint32_t>(127 + 7 - ex) << 23), odd = up * 0.0625f;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
          if (BITS == 8) {  // bytes in their order
            qf[nt][2 * e][0] = H::pack(P::lo(x[e].x) * up, P::hi(x[e].x) * up);
            qf[nt][2 * e][1] = H::pack(P::lo(x[e].y) * up, P::hi(x[e].y) * up);
            qf[nt][2 * e + 1][0] = H::pack(P::lo(x[e].z) * up, P::hi(x[e].z) * up);
            qf[nt][2 * e + 1][1] = H::pack(P::lo(x[e].w) * up, P::hi(x[e].w) * up);
            continue;
          }
          // codes come out of a word as (0, 4), 16 (1, 5), (2, 6), 16 (3, 7)
          qf[nt][2 * e][0] = H::pack(P::lo(x[e].x) * up, P::lo(x[e].z) * up);
          qf[nt][2 * e][1] = H::pack(P::hi(x[e].x) * odd, P::hi(x[e].z) * odd);
          qf[nt][2 * e + 1][0] = H::pack(P::lo(x[e].y) * up, P::lo(x[e].w) * up);
          qf[nt][2 * e + 1][1] = H::pack(P::hi(x[e].y) * odd, P::hi(x[e].w) * odd);
        }
        const float back = scale * __uint_as_float(static_cast<uint32_t>(127 - 7 + ex) << 23) * (BITS == 4 ? 0x1p24f : 1.f);
        by[nt][0] = __shfl_sync(0xffffffffu, back, 8 * c);
        by[nt][1] = __shfl_sync(0xffffffffu, back, 8 * c + 4);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t y = nt * 8 + 2 * c + e;
        const int64_t n = a.causal ? static_cast<int64_t>(it.span.length) - it.span.count + (row0 + y) / a.group + 1 : it.span.length;
        seen[nt][e] = y < rows && n > 0 ? static_cast<int32_t>(n) : 0;
      }
    }
    // the fewest tokens that a row sees: below it, only the mask matters
    int32_t all_see = it.span.length;
    if (a.causal) {
      const int64_t n = static_cast<int64_t>(it.span.length) - it.span.count + row0 / a.group + 1;
      all_see = n > 0 ? static_cast<int32_t>(n) : 0;
    }
    // Weights are summed by kSumChunks chunks, and those sums into l: a lane may have the largest weight and, one by one
    // onto it, 16384 of a million that are 2^-25 of it (the log-sum-exp was 4e-4 off).
    constexpr uint32_t kSumChunks = 64;
    float o[NT][D / 16][4], m[NT][2], l[NT][2], l_part[NT][2];
    // 4-bit: the power of two on p s, of each group (one for both would push the weights of a group whose values are
    // a thousandth of the other's under fp16's range), and the words up to which they hold
    float v_up[kGroups];
    uint32_t v_most = 0x000F000Fu;
#pragma unroll
    for (int gr = 0; gr < kGroups; ++gr) v_up[gr] = 1.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < D / 16; ++e) o[nt][e][0] = o[nt][e][1] = o[nt][e][2] = o[nt][e][3] = 0.f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = l_part[nt][0] = l_part[nt][1] = 0.f;
    }

    uint32_t stage = 0;
    for (uint32_t ch = warp; ch < chunks; ch += kWarps) {
      cp_async_wait<R::kStages - 2>();
      __syncwarp();
      const char* const base = ring + stage * R::kStage;
      const uint32_t bits = stages[warp][stage].x;
      const int32_t pos = static_cast<int32_t>(stages[warp][stage].y);
      uint32_t sees[NT][2];  // tokens of the chunk that rows 2c and 2c + 1 see
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) sees[nt][e] = by_row ? bits & row_bits[warp][stage][nt * 8 + 2 * c + e] : bits;
      issue(stage == 0 ? R::kStages - 1 : stage - 1, ahead);  // the stage read in the iteration before
      ahead = look(ch + R::kStages * kWarps);
      if (++stage == R::kStages) stage = 0;
      if (ch / kWarps % kSumChunks == 0) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          l[nt][0] += l_part[nt][0];
          l[nt][1] += l_part[nt][1];
          l_part[nt][0] = l_part[nt][1] = 0.f;
        }
      }
      if (bits == 0) continue;
      const bool whole = (R::kTokens == 32 ? bits == 0xffffffffu : (bits & 0xffffu) == 0xffffu);
      const char *const vbase = base + R::kTokens * R::kRow, *const kw = base + 2 * R::kTokens * R::kRow, *const vw = kw + R::kWords;

      // ---- scores. Row slots of a 16-token operand hold tokens in this order (codes and bytes: so that both operands' reads
      // are free of conflicts): slot s is token s ^ ((s >> 2) & 1) of its eight
      float s[NT][kM][4];
      const uint32_t tk = BITS < 16 ? g ^ (g >> 2) : g;
#pragma unroll
      for (int mt = 0; mt < kM; ++mt) {
        const uint32_t t0 = mt * 16 + tk;
        if (BITS == 16) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[nt][mt][0] = s[nt][mt][1] = s[nt][mt][2] = s[nt][mt][3] = 0.f;
#pragma unroll
          for (int e = 0; e < D / 32; ++e) {
            const uint4 x = at<uint4>(base + unit_at<D, BITS, false>(t0, 4 * e + c)), y = at<uint4>(base + unit_at<D, BITS, false>(t0 + 8, 4 * e + c));
            const uint32_t f0[4] = {x.x, y.x, x.y, y.y}, f1[4] = {x.z, y.z, x.w, y.w};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              P::mma(s[nt][mt], f0, qf[nt][2 * e][0], qf[nt][2 * e][1]);
              P::mma(s[nt][mt], f1, qf[nt][2 * e + 1][0], qf[nt][2 * e + 1][1]);
            }
          }
        } else {
          uint32_t w0, w1;  // the words of tokens t0 and t0 + 8
          if (D == 128) {
            w0 = at<uint32_t>(kw + t0 * 4);
            w1 = at<uint32_t>(kw + t0 * 4 + 32);
          } else {
            w0 = at<uint16_t>(kw + t0 * 2);
            w1 = at<uint16_t>(kw + t0 * 2 + 16);
          }
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            float acc[NT][4];
            if constexpr (BITS == 8) {
              const uint4 x = at<uint4>(base + unit_at<D, BITS, false>(t0, gr * 4 + c)), y = at<uint4>(base + unit_at<D, BITS, false>(t0 + 8, gr * 4 + c));
              const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t f[4] = {byte_pair(xs[e], 0x4140), byte_pair(ys[e], 0x4140), byte_pair(xs[e], 0x4342), byte_pair(ys[e], 0x4342)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  if (e == 0) mma_first(acc[nt], f, qf[nt][4 * gr][0], qf[nt][4 * gr][1]);
                  else H::mma(acc[nt], f, qf[nt][4 * gr + e][0], qf[nt][4 * gr + e][1]);
                }
              }
            } else {
              const uint2 x = at<uint2>(base + unit_at<D, BITS, false>(t0, gr * 2 + c / 2) + (c % 2) * 8);
              const uint2 y = at<uint2>(base + unit_at<D, BITS, false>(t0 + 8, gr * 2 + c / 2) + (c % 2) * 8);
              const uint32_t z0 = __byte_perm(w0, w0, gr == 0 ? 0x1010 : 0x3232) & 0x000F000Fu, z1 = __byte_perm(w1, w1, gr == 0 ? 0x1010 : 0x3232) & 0x000F000Fu;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t u = (e < 2 ? x.x : x.y) >> (8 * (e % 2)), v = (e < 2 ? y.x : y.y) >> (8 * (e % 2));
                const uint32_t f[4] = {H::sub(u & 0x000F000Fu, z0), H::sub(v & 0x000F000Fu, z1), H::sub(u & 0x00F000F0u, z0 * 16),
                                       H::sub(v & 0x00F000F0u, z1 * 16)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  if (e == 0) mma_first(acc[nt], f, qf[nt][4 * gr][0], qf[nt][4 * gr][1]);
                  else H::mma(acc[nt], f, qf[nt][4 * gr + e][0], qf[nt][4 * gr + e][1]);
                }
              }
            }
            const float s0 = gr == 0 ? scale_lo(w0) : scale_hi(w0), s1 = gr == 0 ? scale_lo(w1) : scale_hi(w1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s[nt][mt][e] = gr == 0 ? (e < 2 ? s0 : s1) * acc[nt][e] : fmaf(e < 2 ? s0 : s1, acc[nt][e], s[nt][mt][e]);
          }
        }
      }
      if (!whole || by_row || pos + R::kTokens > all_see) {
#pragma unroll
        for (int mt = 0; mt < kM; ++mt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t t = mt * 16 + tk + (e < 2 ? 0 : 8);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              if (!(sees[nt][e % 2] >> t & 1u) || pos + static_cast<int32_t>(t) >= seen[nt][e % 2]) s[nt][mt][e] = -INFINITY;
          }
      }
      // ---- running maximum, sum and probabilities
      float p[NT][kM][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float x0 = fmaxf(s[nt][0][0], s[nt][0][2]), x1 = fmaxf(s[nt][0][1], s[nt][0][3]);
#pragma unroll
        for (int mt = 1; mt < kM; ++mt) {
          x0 = fmaxf(x0, fmaxf(s[nt][mt][0], s[nt][mt][2]));
          x1 = fmaxf(x1, fmaxf(s[nt][mt][1], s[nt][mt][3]));
        }
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) {
          x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, w));
          x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, w));
        }
        x0 = fmaxf(x0 * by[nt][0], m[nt][0]);
        x1 = fmaxf(x1 * by[nt][1], m[nt][1]);
        if (__any_sync(0xffffffffu, x0 != m[nt][0] || x1 != m[nt][1])) {
          const float k0 = m[nt][0] == -INFINITY ? 0.f : exp2_fast(m[nt][0] - x0), k1 = m[nt][1] == -INFINITY ? 0.f : exp2_fast(m[nt][1] - x1);
          m[nt][0] = x0;
          m[nt][1] = x1;
          l[nt][0] *= k0;
          l[nt][1] *= k1;
          l_part[nt][0] *= k0;
          l_part[nt][1] *= k1;
#pragma unroll
          for (int e = 0; e < D / 16; ++e) {
            o[nt][e][0] *= k0;
            o[nt][e][1] *= k1;
            o[nt][e][2] *= k0;
            o[nt][e][3] *= k1;
          }
        }
        const float u0 = x0 == -INFINITY ? 0.f : x0 - kUp, u1 = x1 == -INFINITY ? 0.f : x1 - kUp;
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) p[nt][mt][e] = exp2_fast(fmaf(s[nt][mt][e], by[nt][e % 2], e % 2 ? -u1 : -u0));
          l_part[nt][0] += p[nt][mt][0] + p[nt][mt][2];
          l_part[nt][1] += p[nt][mt][1] + p[nt][mt][3];
        }
      }
      // ---- values
      if (BITS == 16) {
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
          uint32_t pf[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            pf[nt][0] = transpose8x8(P::pack(p[nt][mt][0], p[nt][mt][1]));
            pf[nt][1] = transpose8x8(P::pack(p[nt][mt][2], p[nt][mt][3]));
          }
          const uint32_t t = mt * 16 + (lane & 7u) + ((lane >> 4) & 1u) * 8;
#pragma unroll
          for (int e = 0; e < D / 16; ++e) {
            uint32_t f[4];
            ldmatrix_trans(f, shared_address(vbase + unit_at<D, BITS, true>(t, 2 * e + ((lane >> 3) & 1u))));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) P::mma(o[nt][e], f, pf[nt][0], pf[nt][1]);
          }
        }
      } else {
        uint32_t ws[kM][2];  // the words of tokens t0 and t0 + 8, whose probabilities this lane has
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
          const uint32_t t0 = mt * 16 + tk;
          if (D == 128) {
            ws[mt][0] = at<uint32_t>(vw + t0 * 4);
            ws[mt][1] = at<uint32_t>(vw + t0 * 4 + 32);
          } else {
            ws[mt][0] = at<uint16_t>(vw + t0 * 2);
            ws[mt][1] = at<uint16_t>(vw + t0 * 2 + 16);
          }
          if (!whole) {  // what nobody sees may be anything
            if (!((bits >> t0) & 1u)) ws[mt][0] = 0;
            if (!((bits >> (t0 + 8)) & 1u)) ws[mt][1] = 0;
          }
        }
        uint32_t most = __vmaxu2(ws[0][0], ws[0][1]);
#pragma unroll
        for (int mt = 1; mt < kM; ++mt) most = __vmaxu2(most, __vmaxu2(ws[mt][0], ws[mt][1]));
        if (__any_sync(0xffffffffu, __vmaxu2(most, v_most) != v_most)) {  // a scale above all before
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            float x = 0.f;
#pragma unroll
            for (int mt = 0; mt < kM; ++mt)
#pragma unroll
              for (int e = 0; e < 2; ++e) x = fmaxf(x, gr == 0 ? scale_lo(ws[mt][e]) : scale_hi(ws[mt][e]));  // a NaN is passed over
#pragma unroll
            for (int w = 1; w < 32; w <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
            // scales below 2^(ex + 5) are then below 2^15, those at hand below 2^11
            const int ex = max(static_cast<int>(__float_as_uint(x) >> 23) - 127, -100);
            const uint32_t upto = static_cast<uint32_t>(min(ex + 4 + 127, 254)) << 7 | 0x7Fu, was = v_most >> (16 * gr) & 0xFFFFu;
            if (x > 0.f && upto > was) {
              const float up = __uint_as_float(static_cast<uint32_t>(127 + 10 - ex) << 23), k = was == 0x000Fu ? 1.f : up / v_up[gr];
              v_up[gr] = up;
              v_most = gr == 0 ? (v_most & 0xFFFF0000u) | upto : (v_most & 0xFFFFu) | upto << 16;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 4 * gr; e < 4 * gr + 4; ++e) {
                  o[nt][e][0] *= k;
                  o[nt][e][1] *= k;
                  o[nt][e][2] *= k;
                  o[nt][e][3] *= k;
                }
              }
            }
          }
        }
        uint32_t pf8[NT][2];  // bytes: the weights of the two groups' tokens in turn
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
          const uint32_t swap = c >> 1;  // slots 2c and 2c + 1 are tokens 2c and 2c + 1, or the other way round
          const uint32_t ta = mt * 16 + 2 * c + swap, tb = mt * 16 + 2 * c + (swap ^ 1u);
          if constexpr (BITS == 8) {
            // 32 dims at a time, four neighbours to a lane: their bytes of two tokens, side by side
#pragma unroll
            for (int st = 0; st < D / 32; ++st) {
              const int gr = st / 2;
              const uint32_t unit = st * 2 + g / 4, in = (g % 4) * 4;
              const uint32_t xa = at<uint32_t>(vbase + unit_at<D, BITS, true>(ta, unit) + in), xb = at<uint32_t>(vbase + unit_at<D, BITS, true>(tb, unit) + in);
              const uint32_t xc = at<uint32_t>(vbase + unit_at<D, BITS, true>(ta + 8, unit) + in), xd = at<uint32_t>(vbase + unit_at<D, BITS, true>(tb + 8, unit) + in);
              if (st % 2 == 0) {
                const float s0 = (gr == 0 ? scale_lo(ws[mt][0]) : scale_hi(ws[mt][0])) * v_up[gr];
                const float s1 = (gr == 0 ? scale_lo(ws[mt][1]) : scale_hi(ws[mt][1])) * v_up[gr];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  pf8[nt][0] = transpose8x8(H::pack(p[nt][mt][0] * s0, p[nt][mt][1] * s0));
                  pf8[nt][1] = transpose8x8(H::pack(p[nt][mt][2] * s1, p[nt][mt][3] * s1));
                }
              }
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t u = __byte_perm(xa, xb, h == 0 ? 0x5410 : 0x7632), v = __byte_perm(xc, xd, h == 0 ? 0x5410 : 0x7632);
                const uint32_t f[4] = {byte_even(u), byte_even(u >> 8), byte_even(v), byte_even(v >> 8)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) H::mma(o[nt][st * 2 + h], f, pf8[nt][0], pf8[nt][1]);
              }
            }
            continue;
          }
          uint32_t wa, wb, wc, wd;  // words of the tokens in slots 2c, 2c + 1, 2c + 8, 2c + 9, for their zero points
          if (D == 128) {
            wa = at<uint32_t>(vw + ta * 4), wb = at<uint32_t>(vw + tb * 4), wc = at<uint32_t>(vw + ta * 4 + 32), wd = at<uint32_t>(vw + tb * 4 + 32);
          } else {
            wa = at<uint16_t>(vw + ta * 2), wb = at<uint16_t>(vw + tb * 2), wc = at<uint16_t>(vw + ta * 2 + 16), wd = at<uint16_t>(vw + tb * 2 + 16);
          }
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            const float s0 = (gr == 0 ? scale_lo(ws[mt][0]) : scale_hi(ws[mt][0])) * v_up[gr];
            const float s1 = (gr == 0 ? scale_lo(ws[mt][1]) : scale_hi(ws[mt][1])) * v_up[gr];
            uint32_t pf[NT][2];
            const uint32_t z01 = __byte_perm(wa, wb, gr == 0 ? 0x5410 : 0x7632) & 0x000F000Fu,
                           z23 = __byte_perm(wc, wd, gr == 0 ? 0x5410 : 0x7632) & 0x000F000Fu;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              pf[nt][0] = transpose8x8(H::pack(p[nt][mt][0] * s0, p[nt][mt][1] * s0));
              pf[nt][1] = transpose8x8(H::pack(p[nt][mt][2] * s1, p[nt][mt][3] * s1));
            }
            const uint32_t unit = gr * 2 + g / 4, in = (g % 4) * 4;
            const uint32_t xa = at<uint32_t>(vbase + unit_at<D, BITS, true>(ta, unit) + in), xb = at<uint32_t>(vbase + unit_at<D, BITS, true>(tb, unit) + in);
            const uint32_t xc = at<uint32_t>(vbase + unit_at<D, BITS, true>(ta + 8, unit) + in), xd = at<uint32_t>(vbase + unit_at<D, BITS, true>(tb + 8, unit) + in);
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // dims 8 g .. + 3, and the four after them
              const uint32_t u = __byte_perm(xa, xb, h == 0 ? 0x5410 : 0x7632), v = __byte_perm(xc, xd, h == 0 ? 0x5410 : 0x7632);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const uint32_t ue = u >> (8 * e), ve = v >> (8 * e);
                const uint32_t f[4] = {H::sub(ue & 0x000F000Fu, z01), H::sub(ue & 0x00F000F0u, z01 * 16), H::sub(ve & 0x000F000Fu, z23),
                                       H::sub(ve & 0x00F000F0u, z23 * 16)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) H::mma(o[nt][gr * 4 + h * 2 + e], f, pf[nt][0], pf[nt][1]);
              }
            }
          }
        }
      }
    }
    if (BITS < 16) {  // to values: the powers of two back
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        const float back = 1.f / v_up[e / 4];  // (with the 2^24 it may pass fp32's range)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int f = 0; f < 4; ++f) o[nt][e][f] = o[nt][e][f] * (BITS == 8 ? 1.f : f < 2 ? 0x1p24f : 0x1p20f) * back;
      }
    }
    cp_async_wait<0>();
    __syncthreads();  // every warp is done with its ring

    // ---- the warps' parts, joined in the order of the warps
    float* buf = reinterpret_cast<float*>(smem);  // [warp][row][D]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[nt][e] + l_part[nt][e];
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
        if (g == 0) {
          warp_m[warp][nt * 8 + 2 * c + e] = m[nt][e];
          warp_l[warp][nt * 8 + 2 * c + e] = x;
        }
        float* to = buf + (warp * kRows + nt * 8 + 2 * c + e) * D;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          if (BITS == 16) {
            to[d * 16 + g] = o[nt][d][e];
            to[d * 16 + g + 8] = o[nt][d][2 + e];
          } else if (BITS == 8) {
            *reinterpret_cast<float2*>(to + (d / 2) * 32 + g * 4 + (d % 2) * 2) = make_float2(o[nt][d][e], o[nt][d][2 + e]);
          } else {
            *reinterpret_cast<float2*>(to + (d / 4) * 64 + g * 8 + (d % 4) * 2) = make_float2(o[nt][d][e], o[nt][d][2 + e]);
          }
        }
      }
    }
    const bool alone = it.first_cta == it.last_cta;
    const uint32_t slot = 2 * blockIdx.x + (blockIdx.x == it.first_cta ? 1 : 0);
    if (!SHORT && it.lo > item_lo && threadIdx.x < kRows) pieces_ms[threadIdx.x] = a.part_ms[static_cast<uint64_t>(slot) * kRows + threadIdx.x];
    __syncthreads();
    const auto write = [&](uint32_t r, uint32_t d, float4 x, float top, float sum) {
      const uint32_t i = it.span.first + (row0 + r) / a.group, h = it.head * a.group + (row0 + r) % a.group;
      if constexpr (SHARED) {
        const uint64_t row = static_cast<uint64_t>(i) * a.heads + h;
        float4* const there = reinterpret_cast<float4*>(a.rows + row * D + d);
        if (!a.behind) {
          *there = make_float4(x.x * kDown, x.y * kDown, x.z * kDown, x.w * kDown);
          if (d == 0) a.rows_ms[row] = make_float2(top, sum * kDown);
          return;
        }
        if (before) {
          const float4 y = *there;
          const Both w = both_parts(top, sum * kDown, a.rows_ms[row]);
          const float own = w.own * kDown;
          x = make_float4(w.prefix * y.x + own * x.x, w.prefix * y.y + own * x.y, w.prefix * y.z + own * x.z, w.prefix * y.w + own * x.w);
          top = w.top;
          sum = w.sum;
        }
      }
      const float down = SHARED && before ? 1.f : kDown, by = sum == 0.f ? 0.f : 1.f / sum;
      T* out = reinterpret_cast<T*>(a.q.out) + static_cast<int64_t>(i) * a.q.out_token + static_cast<int64_t>(h) * a.q.out_head + d;
      if (a.out_wide) {
        *reinterpret_cast<uint2*>(out) = make_uint2(P::pack(x.x * by, x.y * by), P::pack(x.z * by, x.w * by));
      } else {
        out[0] = Elem<T>::from(x.x * by);
        out[1] = Elem<T>::from(x.y * by);
        out[2] = Elem<T>::from(x.z * by);
        out[3] = Elem<T>::from(x.w * by);
      }
      if (a.lse && d == 0) a.lse[static_cast<uint64_t>(i) * a.heads + h] = (top + log2f(sum * down)) * 0.6931471805599453f;
    };
    for (uint32_t x = threadIdx.x; x < rows * (D / 4); x += kThreads) {
      const uint32_t r = x / (D / 4), d = x % (D / 4) * 4;
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, warp_m[w][r]);
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float k = warp_m[w][r] == -INFINITY ? 0.f : exp2_fast(warp_m[w][r] - top);
        if (warp_m[w][r] == -INFINITY && warp_l[w][r] == 0.f) continue;
        const float4 z = *reinterpret_cast<const float4*>(buf + (w * kRows + r) * D + d);
        sum += k * warp_l[w][r];
        y.x += k * z.x, y.y += k * z.y, y.z += k * z.z, y.w += k * z.w;
      }
      if (!SHORT && it.lo > item_lo) {  // the pieces before (this thread wrote their sums)
        const Both w = both_parts(top, sum, pieces_ms[r]);
        const float4 was = *reinterpret_cast<const float4*>(a.part + (static_cast<uint64_t>(slot) * kRows + r) * D + d);
        y = make_float4(w.own * y.x + w.prefix * was.x, w.own * y.y + w.prefix * was.y, w.own * y.z + w.prefix * was.z, w.own * y.w + w.prefix * was.w);
        top = w.top;
        sum = w.sum;
      }
      if (alone && (SHORT || !more)) {
        write(r, d, y, top, sum);
      } else {
        *reinterpret_cast<float4*>(a.part + (static_cast<uint64_t>(slot) * kRows + r) * D + d) = y;
        if (d == 0) a.part_ms[static_cast<uint64_t>(slot) * kRows + r] = make_float2(top, sum);
      }
    }
    if (!alone && (SHORT || !more)) {
      __syncthreads();
      if (threadIdx.x == 0) last_here = part_done(a, it);
      __syncthreads();
      if (last_here) {
        // each part's factor for each row, kJoin parts at a time; the maximum over all parts first
        const uint32_t parts = it.last_cta - it.first_cta + 1;
        const auto part_at = [&](uint32_t i, uint32_t r) { return (2ull * (it.first_cta + i) + (i == 0)) * kRows + r; };
        float2* ms = reinterpret_cast<float2*>(smem);  // [part][row]
        constexpr uint32_t kJoin = split_smem<D, BITS, NT, SHORT>() / (kRows * sizeof(float2));
        float top = -INFINITY, sum = 0.f;  // of row threadIdx.x
        for (uint32_t p0 = 0; p0 < parts; p0 += kJoin) {
          const uint32_t n = min(kJoin, parts - p0);
          __syncthreads();
          for (uint32_t x = threadIdx.x; x < n * kRows; x += kThreads) ms[x] = __ldcg(&a.part_ms[part_at(p0 + x / kRows, x % kRows)]);
          __syncthreads();
          if (threadIdx.x < rows)
            for (uint32_t i = 0; i < n; ++i) top = fmaxf(top, ms[i * kRows + threadIdx.x].x);
        }
        if (threadIdx.x < kRows) warp_m[0][threadIdx.x] = top;
        constexpr int kMost = (kRows * (D / 4) + kThreads - 1) / kThreads;
        float4 y[kMost];
#pragma unroll
        for (int q = 0; q < kMost; ++q) y[q] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t p0 = 0; p0 < parts; p0 += kJoin) {
          const uint32_t n = min(kJoin, parts - p0);
          __syncthreads();
          for (uint32_t x = threadIdx.x; x < n * kRows; x += kThreads) {
            const float2 z = parts <= kJoin ? ms[x] : __ldcg(&a.part_ms[part_at(p0 + x / kRows, x % kRows)]);
            const float k = z.x == -INFINITY ? (z.y == 0.f ? 0.f : 1.f) : exp2_fast(z.x - warp_m[0][x % kRows]);
            ms[x] = make_float2(k, z.y == 0.f ? 0.f : k * z.y);
          }
          __syncthreads();
          if (threadIdx.x < rows)
            for (uint32_t i = 0; i < n; ++i) sum += ms[i * kRows + threadIdx.x].y;
#pragma unroll
          for (int q = 0; q < kMost; ++q) {
            const uint32_t x = threadIdx.x + q * kThreads, r = x / (D / 4), d = x % (D / 4) * 4;
            if (r >= rows) break;
#pragma unroll 8
            for (uint32_t i = 0; i < n; ++i) {
              const float k = ms[i * kRows + r].x;
              const float4 z = __ldcg(reinterpret_cast<const float4*>(a.part + part_at(p0 + i, r) * D + d));
              y[q].x += k * z.x, y[q].y += k * z.y, y[q].z += k * z.z, y[q].w += k * z.w;
            }
          }
        }
        if (threadIdx.x < kRows) warp_l[0][threadIdx.x] = sum;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kMost; ++q) {
          const uint32_t x = threadIdx.x + q * kThreads, r = x / (D / 4), d = x % (D / 4) * 4;
          if (r < rows) write(r, d, y[q], warp_m[0][r], warp_l[0][r]);
        }
      }
    }
    __syncthreads();  // the buffer is a ring again
  }
}

}  // namespace
}  // namespace cofie

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
// 4-bit codes enter the products without being scaled. A code n becomes the
// 16-bit number 128 + n (bf16) or 1024 + n (fp16) by one logic operation on two
// codes. For keys, whose scale is one factor of a score's 64 terms, the score
// is s (sum q (128 + n) - (128 + z) sum q), in fp32. Values have a scale for
// each token, inside the sum: (n - z) s is formed, exactly, in two more
// operations on two values.
#pragma once

#include "kv_plan.cuh"

namespace cofie {
namespace {

constexpr int kSplitWarps = 8;
constexpr int kSplitThreads = 32 * kSplitWarps;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(live ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(a));
  return x;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t x;
  asm volatile("ld.shared.b16 %0, [%1];" : "=h"(x) : "r"(a));
  return x;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 x;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(a));
  return x;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(a));
  return x;
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
struct Pair;  // two 16-bit values in a register
template <>
struct Pair<__nv_bfloat16> {
  static constexpr uint32_t kMagic = 0x43004300u;  // 128 + n
  static constexpr float kExcess = 128.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) {
    const __nv_bfloat162 x = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b) {
    const __nv_bfloat162 x = __hmul2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ uint32_t scales(uint32_t w) { return w & 0xFFF0FFF0u; }
  static __device__ __forceinline__ float lo(uint32_t x) { return __uint_as_float(x << 16); }
  static __device__ __forceinline__ float hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Pair<__half> {
  static constexpr uint32_t kMagic = 0x64006400u;  // 1024 + n
  static constexpr float kExcess = 1024.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) {
    const __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b) {
    const __half2 x = __hmul2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ uint32_t scales(uint32_t w) {  // bf16 words to fp16
    return pack(__uint_as_float((w & 0xFFF0u) << 16), __uint_as_float(w & 0xFFF00000u));
  }
  static __device__ __forceinline__ float lo(uint32_t x) { return __half2float(__ushort_as_half(static_cast<unsigned short>(x))); }
  static __device__ __forceinline__ float hi(uint32_t x) { return __half2float(__ushort_as_half(static_cast<unsigned short>(x >> 16))); }
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

// Sizes of one warp's ring. Chunks of 32 tokens of codes, 16 of 16-bit values.
template <int D, int BITS>
struct Ring {
  static constexpr int kTokens = BITS == 4 ? 32 : 16;
  static constexpr int kRow = D * BITS / 8;                               // bytes of a token's keys
  static constexpr int kWords = BITS == 4 ? kTokens * (D / 64) * 2 : 0;   // bytes of its chunk's scale words
  static constexpr int kStage = 2 * (kTokens * kRow + kWords);
  static constexpr int kStages = BITS == 4 ? 3 : 3;
  static constexpr int kWarp = kStages * kStage;
  static constexpr int kUnits = kRow / 16;                                // 16-byte units of a token
};

template <int D, int BITS, int NT>
constexpr size_t split_smem() {
  const size_t ring = static_cast<size_t>(kSplitWarps) * Ring<D, BITS>::kWarp, join = static_cast<size_t>(kSplitWarps) * 8 * NT * D * 4;
  return ring > join ? ring : join;
}

// Where unit u of token t lies in its chunk, such that the reads below meet no bank twice.
template <int D, int BITS, bool VALUES>
__device__ __forceinline__ uint32_t unit_at(uint32_t t, uint32_t u) {
  if (BITS == 4) return t * Ring<D, 4>::kRow + (D == 128 ? (u ^ ((t & 2u))) : u) * 16;
  return t * Ring<D, 16>::kRow + (VALUES ? u ^ (t & 7u) : u ^ ((t & 1u) << 2)) * 16;
}

template <typename T, int D, int BITS, int NT>
__global__ void __launch_bounds__(kSplitThreads, NT == 1 && BITS == 4 ? 2 : 1) attend_split(const __grid_constant__ AttendArgs a) {
  using P = Pair<T>;
  using R = Ring<D, BITS>;
  constexpr int kRows = 8 * NT, kGroups = D / 64, kM = R::kTokens / 16, kPerTile = kTile / R::kTokens;
  extern __shared__ __align__(128) char smem[];
  __shared__ Plan<kSplitThreads> plan;
  __shared__ float warp_m[kSplitWarps][kRows], warp_l[kSplitWarps][kRows];
  __shared__ uint32_t seen_bits[kSplitWarps][R::kStages];
  __shared__ uint32_t last_here;
  pdl_trigger();
  pdl_wait();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
  const uint64_t range = plan.set_up(a, kRows);
  Walk<kSplitThreads> walk(a, plan, kRows, range);
  const uint32_t ring = shared_address(smem) + warp * R::kWarp;
  const BatchArg& b = a.batch;
  const float scale = a.scale * 1.4426950408889634f;  // scores in base 2
  Item it;
  while (walk.next(it)) {
    const uint32_t row0 = it.rb * kRows;
    const uint32_t rows = min(static_cast<uint32_t>(kRows), it.span.count * a.group - row0);
    // ---- queries: fragments of Q^T, the columns of this lane's dims in the order in which the keys' lie in registers
    uint32_t qf[NT][D / 16][2];
    float qsum[NT][2][kGroups];  // 4-bit: sum of q over a group, of rows 2c and 2c + 1
    int32_t seen[NT][2];         // tokens that rows 2c and 2c + 1 may see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint32_t r = nt * 8 + g;
      const bool real = r < rows;
      const uint32_t i = (row0 + r) / a.group, j = (row0 + r) % a.group;
      const T* q = reinterpret_cast<const T*>(a.q.in) + (real ? static_cast<int64_t>(it.span.first + i) * a.q.in_token +
                                                                    static_cast<int64_t>(it.head * a.group + j) * a.q.in_head
                                                              : 0);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        // eight dims: 16-bit keys: unit 4 e + c of the row; codes: word e % 2 of the lane's two words in group e / 2
        const uint32_t d = BITS == 16 ? (4 * e + c) * 8 : (e / 2) * 64 + c * 16 + (e % 2) * 8;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (real) {
          if (a.q_wide) {
            x = *reinterpret_cast<const uint4*>(q + d);
          } else {
            RowVec<T, 8> y;
#pragma unroll
            for (int f = 0; f < 8; ++f) y.v[f] = q[d + f];
            x = *reinterpret_cast<uint4*>(&y);
          }
        }
        if (BITS == 16) {
          qf[nt][2 * e][0] = x.x;
          qf[nt][2 * e][1] = x.y;
          qf[nt][2 * e + 1][0] = x.z;
          qf[nt][2 * e + 1][1] = x.w;
        } else {  // codes come out of a word as (0, 4), (1, 5), (2, 6), (3, 7)
          qf[nt][2 * e][0] = __byte_perm(x.x, x.z, 0x5410);
          qf[nt][2 * e][1] = __byte_perm(x.x, x.z, 0x7632);
          qf[nt][2 * e + 1][0] = __byte_perm(x.y, x.w, 0x5410);
          qf[nt][2 * e + 1][1] = __byte_perm(x.y, x.w, 0x7632);
        }
      }
      if (BITS == 4) {
#pragma unroll
        for (int gr = 0; gr < kGroups; ++gr) {
          float s = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int f = 0; f < 2; ++f) s += P::lo(qf[nt][4 * gr + e][f]) + P::hi(qf[nt][4 * gr + e][f]);
          s += __shfl_xor_sync(0xffffffffu, s, 1);
          s += __shfl_xor_sync(0xffffffffu, s, 2);
          qsum[nt][0][gr] = __shfl_sync(0xffffffffu, s, 8 * c);
          qsum[nt][1][gr] = __shfl_sync(0xffffffffu, s, 8 * c + 4);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t x = nt * 8 + 2 * c + e;
        const int64_t n = a.causal ? static_cast<int64_t>(it.span.length) - it.span.count + (row0 + x) / a.group + 1 : it.span.length;
        seen[nt][e] = x < rows && n > 0 ? static_cast<int32_t>(n) : 0;
      }
    }
    // the fewest tokens that a row sees: below it, only the mask matters
    int32_t all_see = it.span.length;
    if (a.causal) {
      const int64_t n = static_cast<int64_t>(it.span.length) - it.span.count + row0 / a.group + 1;
      all_see = n > 0 ? static_cast<int32_t>(n) : 0;
    }
    float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < D / 16; ++e) o[nt][e][0] = o[nt][e][1] = o[nt][e][2] = o[nt][e][3] = 0.f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }

    // ---- the warp's chunks: warp, warp + 8, ... of the item's part
    const uint32_t chunks = (it.hi - it.lo) * kPerTile;
    const int32_t* table = b.table + static_cast<uint64_t>(it.seq) * b.table_stride;
    const auto chunk_pos = [&](uint32_t ch) {
      const uint32_t t = it.lo + ch / kPerTile;
      return (a.mask ? a.tiles[static_cast<uint64_t>(it.seq) * a.tile_stride + t] : t) * kTile + (ch % kPerTile) * R::kTokens;
    };
    // the row in the pages of this lane's token of a chunk, -1 where there is nothing to see
    const auto token_row = [&](uint32_t ch) -> int64_t {
      if (ch >= chunks) return -1;
      const uint32_t pos = chunk_pos(ch) + lane % R::kTokens;
      if (pos >= it.span.length) return -1;
      if (a.mask && (pos >= a.mask_stride || !a.mask[it.seq * a.mask_stride + pos])) return -1;
      const uint32_t page = static_cast<uint32_t>(table[pos >> b.page_shift]);
      if (page >= b.n_pages) {
        atomicOr(b.err, kKvErrPage);
        return -1;
      }
      return static_cast<int64_t>(page_row(b, (static_cast<int64_t>(page) << b.page_shift) | (pos & ((1u << b.page_shift) - 1)), it.head));
    };
    const auto issue = [&](uint32_t stage, int64_t row) {
      const uint32_t base = ring + stage * R::kStage;
      const uint32_t bits = __ballot_sync(0xffffffffu, row >= 0);
      if (lane == 0) seen_bits[warp][stage] = bits;
      if (bits) {
#pragma unroll
        for (int i = 0; i < R::kTokens * R::kUnits / 32; ++i) {
          const uint32_t x = i * 32 + lane, t = x / R::kUnits, u = x % R::kUnits;
          const int64_t r = __shfl_sync(0xffffffffu, row, t);
          const uint64_t off = r < 0 ? 0 : static_cast<uint64_t>(r) * R::kRow + u * 16;
          cp_async16(base + unit_at<D, BITS, false>(t, u), a.k + off, r >= 0);
          cp_async16(base + R::kTokens * R::kRow + unit_at<D, BITS, true>(t, u), a.v + off, r >= 0);
        }
        if (BITS == 4) {
          const uint32_t dst = base + 2 * R::kTokens * R::kRow + lane * 4;
          if (D == 128) {
            const uint64_t off = row < 0 ? 0 : static_cast<uint64_t>(row) * 2;
            cp_async4(dst, a.k_words + off, row >= 0);
            cp_async4(dst + R::kWords, a.v_words + off, row >= 0);
          } else {  // the words of two tokens, which lie in one page, to a lane
            const int64_t r0 = __shfl_sync(0xffffffffu, row, lane * 2 % 32), r1 = __shfl_sync(0xffffffffu, row, (lane * 2 + 1) % 32);
            const int64_t r = r0 >= 0 ? r0 : r1 - 1;
            if (lane < 16) {
              cp_async4(dst, a.k_words + (r < 0 ? 0 : r), r >= 0);
              cp_async4(dst + R::kWords, a.v_words + (r < 0 ? 0 : r), r >= 0);
            }
          }
        }
      }
      cp_async_commit();
    };
    int64_t ahead;
    {
      int64_t first[R::kStages - 1];
#pragma unroll
      for (int s = 0; s < R::kStages - 1; ++s) first[s] = token_row(warp + s * kSplitWarps);
      ahead = token_row(warp + (R::kStages - 1) * kSplitWarps);
#pragma unroll
      for (int s = 0; s < R::kStages - 1; ++s) issue(s, first[s]);
    }
    uint32_t stage = 0;
    for (uint32_t ch = warp; ch < chunks; ch += kSplitWarps) {
      cp_async_wait<R::kStages - 2>();
      __syncwarp();
      const uint32_t base = ring + stage * R::kStage, bits = seen_bits[warp][stage];
      issue(stage == 0 ? R::kStages - 1 : stage - 1, ahead);  // the stage read in the iteration before
      ahead = token_row(ch + R::kStages * kSplitWarps);
      if (++stage == R::kStages) stage = 0;
      if (bits == 0) continue;
      const int32_t pos = static_cast<int32_t>(chunk_pos(ch));
      const bool whole = (BITS == 4 ? bits == 0xffffffffu : (bits & 0xffffu) == 0xffffu);
      const uint32_t vbase = base + R::kTokens * R::kRow, kw = base + 2 * R::kTokens * R::kRow, vw = kw + R::kWords;

      // ---- scores. Row slots of a 16-token operand hold tokens in this order (4-bit: so that both operands' reads
      // are free of conflicts): slot s is token s ^ ((s >> 2) & 1) of its eight
      float s[NT][kM][4];
      const uint32_t tk = BITS == 4 ? g ^ (g >> 2) : g;
#pragma unroll
      for (int mt = 0; mt < kM; ++mt) {
        const uint32_t t0 = mt * 16 + tk;
        if (BITS == 16) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[nt][mt][0] = s[nt][mt][1] = s[nt][mt][2] = s[nt][mt][3] = 0.f;
#pragma unroll
          for (int e = 0; e < D / 32; ++e) {
            const uint4 x = lds128(base + unit_at<D, BITS, false>(t0, 4 * e + c)), y = lds128(base + unit_at<D, BITS, false>(t0 + 8, 4 * e + c));
            const uint32_t f0[4] = {x.x, y.x, x.y, y.y}, f1[4] = {x.z, y.z, x.w, y.w};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              P::mma(s[nt][mt], f0, qf[nt][2 * e][0], qf[nt][2 * e][1]);
              P::mma(s[nt][mt], f1, qf[nt][2 * e + 1][0], qf[nt][2 * e + 1][1]);
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][mt][e] *= scale;
        } else {
          uint32_t w0, w1;  // the words of tokens t0 and t0 + 8
          if (D == 128) {
            w0 = lds32(kw + t0 * 4);
            w1 = lds32(kw + t0 * 4 + 32);
          } else {
            w0 = lds16(kw + t0 * 2);
            w1 = lds16(kw + t0 * 2 + 16);
          }
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            const uint2 x = lds64(base + unit_at<D, BITS, false>(t0, gr * 2 + c / 2) + (c % 2) * 8);
            const uint2 y = lds64(base + unit_at<D, BITS, false>(t0 + 8, gr * 2 + c / 2) + (c % 2) * 8);
            float acc[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t u = (e < 2 ? x.x : x.y) >> (8 * (e % 2)), v = (e < 2 ? y.x : y.y) >> (8 * (e % 2));
              const uint32_t f[4] = {(u & 0x000F000Fu) | P::kMagic, (v & 0x000F000Fu) | P::kMagic, ((u >> 4) & 0x000F000Fu) | P::kMagic,
                                     ((v >> 4) & 0x000F000Fu) | P::kMagic};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) P::mma(acc[nt], f, qf[nt][4 * gr + e][0], qf[nt][4 * gr + e][1]);
            }
            const uint32_t h0 = D == 128 && gr == 1 ? w0 >> 16 : w0 & 0xFFFFu, h1 = D == 128 && gr == 1 ? w1 >> 16 : w1 & 0xFFFFu;
            const float s0 = __uint_as_float((h0 & 0xFFF0u) << 16) * scale, s1 = __uint_as_float((h1 & 0xFFF0u) << 16) * scale;
            const float z0 = -P::kExcess - static_cast<float>(h0 & 15u), z1 = -P::kExcess - static_cast<float>(h1 & 15u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float t = fmaf(e < 2 ? z0 : z1, qsum[nt][e % 2][gr], acc[nt][e]);
                s[nt][mt][e] = gr == 0 ? (e < 2 ? s0 : s1) * t : fmaf(e < 2 ? s0 : s1, t, s[nt][mt][e]);
              }
          }
        }
      }
      if (!whole || pos + R::kTokens > all_see) {
#pragma unroll
        for (int mt = 0; mt < kM; ++mt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t t = mt * 16 + tk + (e < 2 ? 0 : 8);
            const bool there = (bits >> t) & 1u;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              if (!there || pos + static_cast<int32_t>(t) >= seen[nt][e % 2]) s[nt][mt][e] = -INFINITY;
          }
      }
      // ---- running maximum, sum and probabilities
      uint32_t pf[NT][kM][2];
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
        x0 = fmaxf(x0, m[nt][0]);
        x1 = fmaxf(x1, m[nt][1]);
        if (__any_sync(0xffffffffu, x0 != m[nt][0] || x1 != m[nt][1])) {
          const float k0 = m[nt][0] == -INFINITY ? 0.f : exp2_fast(m[nt][0] - x0), k1 = m[nt][1] == -INFINITY ? 0.f : exp2_fast(m[nt][1] - x1);
          m[nt][0] = x0;
          m[nt][1] = x1;
          l[nt][0] *= k0;
          l[nt][1] *= k1;
#pragma unroll
          for (int e = 0; e < D / 16; ++e) {
            o[nt][e][0] *= k0;
            o[nt][e][1] *= k1;
            o[nt][e][2] *= k0;
            o[nt][e][3] *= k1;
          }
        }
        const float u0 = x0 == -INFINITY ? 0.f : x0, u1 = x1 == -INFINITY ? 0.f : x1;
#pragma unroll
        for (int mt = 0; mt < kM; ++mt) {
          const float p0 = exp2_fast(s[nt][mt][0] - u0), p1 = exp2_fast(s[nt][mt][1] - u1), p2 = exp2_fast(s[nt][mt][2] - u0),
                      p3 = exp2_fast(s[nt][mt][3] - u1);
          l[nt][0] += p0 + p2;
          l[nt][1] += p1 + p3;
          pf[nt][mt][0] = transpose8x8(P::pack(p0, p1));
          pf[nt][mt][1] = transpose8x8(P::pack(p2, p3));
        }
      }
      // ---- values
#pragma unroll
      for (int mt = 0; mt < kM; ++mt) {
        if (BITS == 16) {
          const uint32_t t = mt * 16 + (lane & 7u) + ((lane >> 4) & 1u) * 8;
#pragma unroll
          for (int e = 0; e < D / 16; ++e) {
            uint32_t f[4];
            ldmatrix_trans(f, vbase + unit_at<D, BITS, true>(t, 2 * e + ((lane >> 3) & 1u)));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) P::mma(o[nt][e], f, pf[nt][mt][0], pf[nt][mt][1]);
          }
        } else {
          const uint32_t swap = c >> 1;  // slots 2c and 2c + 1 are tokens 2c and 2c + 1, or the other way round
          const uint32_t ta = mt * 16 + 2 * c + swap, tb = mt * 16 + 2 * c + (swap ^ 1u);
          uint32_t wa, wb, wc, wd;  // scale words of the tokens in slots 2c, 2c + 1, 2c + 8, 2c + 9
          if (D == 128) {
            wa = lds32(vw + ta * 4), wb = lds32(vw + tb * 4), wc = lds32(vw + ta * 4 + 32), wd = lds32(vw + tb * 4 + 32);
          } else {
            wa = lds16(vw + ta * 2), wb = lds16(vw + tb * 2), wc = lds16(vw + ta * 2 + 16), wd = lds16(vw + tb * 2 + 16);
          }
          if (!whole) {  // a token that is not there may have a neighbour's word
            if (!((bits >> ta) & 1u)) wa = 0;
            if (!((bits >> tb) & 1u)) wb = 0;
            if (!((bits >> (ta + 8)) & 1u)) wc = 0;
            if (!((bits >> (tb + 8)) & 1u)) wd = 0;
          }
#pragma unroll
          for (int gr = 0; gr < kGroups; ++gr) {
            const uint32_t w01 = __byte_perm(wa, wb, gr == 0 ? 0x5410 : 0x7632), w23 = __byte_perm(wc, wd, gr == 0 ? 0x5410 : 0x7632);
            const uint32_t z01 = (w01 & 0x000F000Fu) | P::kMagic, z23 = (w23 & 0x000F000Fu) | P::kMagic;
            const uint32_t s01 = P::scales(w01), s23 = P::scales(w23);
            const uint32_t unit = gr * 2 + g / 4, at = (g % 4) * 4;
            const uint32_t xa = lds32(vbase + unit_at<D, BITS, true>(ta, unit) + at), xb = lds32(vbase + unit_at<D, BITS, true>(tb, unit) + at);
            const uint32_t xc = lds32(vbase + unit_at<D, BITS, true>(ta + 8, unit) + at), xd = lds32(vbase + unit_at<D, BITS, true>(tb + 8, unit) + at);
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // dims 8 g .. + 3, and the four after them
              const uint32_t u = __byte_perm(xa, xb, h == 0 ? 0x5410 : 0x7632), v = __byte_perm(xc, xd, h == 0 ? 0x5410 : 0x7632);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const uint32_t ue = u >> (8 * e), ve = v >> (8 * e);
                const uint32_t f[4] = {
                    P::mul(P::sub((ue & 0x000F000Fu) | P::kMagic, z01), s01), P::mul(P::sub(((ue >> 4) & 0x000F000Fu) | P::kMagic, z01), s01),
                    P::mul(P::sub((ve & 0x000F000Fu) | P::kMagic, z23), s23), P::mul(P::sub(((ve >> 4) & 0x000F000Fu) | P::kMagic, z23), s23)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) P::mma(o[nt][gr * 4 + h * 2 + e], f, pf[nt][mt][0], pf[nt][mt][1]);
              }
            }
          }
        }
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
        float x = l[nt][e];
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
          } else {
            *reinterpret_cast<float2*>(to + (d / 4) * 64 + g * 8 + (d % 4) * 2) = make_float2(o[nt][d][e], o[nt][d][2 + e]);
          }
        }
      }
    }
    __syncthreads();
    const bool alone = it.first_cta == it.last_cta;
    const uint32_t slot = 2 * blockIdx.x + (blockIdx.x == it.first_cta ? 1 : 0);
    const auto write = [&](uint32_t r, uint32_t d, float4 x, float top, float sum) {
      const float by = sum == 0.f ? 0.f : 1.f / sum;
      const uint32_t i = it.span.first + (row0 + r) / a.group, h = it.head * a.group + (row0 + r) % a.group;
      T* out = reinterpret_cast<T*>(a.q.out) + static_cast<int64_t>(i) * a.q.out_token + static_cast<int64_t>(h) * a.q.out_head + d;
      if (a.out_wide) {
        *reinterpret_cast<uint2*>(out) = make_uint2(P::pack(x.x * by, x.y * by), P::pack(x.z * by, x.w * by));
      } else {
        out[0] = Elem<T>::from(x.x * by);
        out[1] = Elem<T>::from(x.y * by);
        out[2] = Elem<T>::from(x.z * by);
        out[3] = Elem<T>::from(x.w * by);
      }
      if (a.lse && d == 0) a.lse[static_cast<uint64_t>(i) * a.heads + h] = (top + log2f(sum)) * 0.6931471805599453f;
    };
    for (uint32_t x = threadIdx.x; x < rows * (D / 4); x += kSplitThreads) {
      const uint32_t r = x / (D / 4), d = x % (D / 4) * 4;
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kSplitWarps; ++w) top = fmaxf(top, warp_m[w][r]);
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kSplitWarps; ++w) {
        const float k = warp_m[w][r] == -INFINITY ? 0.f : exp2_fast(warp_m[w][r] - top);
        if (warp_m[w][r] == -INFINITY && warp_l[w][r] == 0.f) continue;
        const float4 z = *reinterpret_cast<const float4*>(buf + (w * kRows + r) * D + d);
        sum += k * warp_l[w][r];
        y.x += k * z.x, y.y += k * z.y, y.z += k * z.z, y.w += k * z.w;
      }
      if (alone) {
        write(r, d, y, top, sum);
      } else {
        *reinterpret_cast<float4*>(a.part + (static_cast<uint64_t>(slot) * kRows + r) * D + d) = y;
        if (d == 0) a.part_ms[static_cast<uint64_t>(slot) * kRows + r] = make_float2(top, sum);
      }
    }
    if (!alone) {
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        const uint32_t parts = it.last_cta - it.first_cta + 1;
        last_here = atomicAdd(a.done + it.first_cta, 1u) == parts - 1;
        if (last_here) a.done[it.first_cta] = 0;
      }
      __syncthreads();
      if (last_here) {
        __threadfence();
        for (uint32_t x = threadIdx.x; x < rows * (D / 4); x += kSplitThreads) {
          const uint32_t r = x / (D / 4), d = x % (D / 4) * 4;
          float top = -INFINITY, sum = 0.f;
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
          for (uint32_t ct = it.first_cta; ct <= it.last_cta; ++ct)
            top = fmaxf(top, __ldcg(&a.part_ms[(2ull * ct + (ct == it.first_cta)) * kRows + r]).x);
#pragma unroll 4
          for (uint32_t ct = it.first_cta; ct <= it.last_cta; ++ct) {
            const uint64_t at = (2ull * ct + (ct == it.first_cta)) * kRows + r;
            const float2 ms = __ldcg(&a.part_ms[at]);
            const float4 z = __ldcg(reinterpret_cast<const float4*>(a.part + at * D + d));
            const float k = ms.x == -INFINITY ? (ms.y == 0.f ? 0.f : 1.f) : exp2_fast(ms.x - top);
            sum += k * ms.y;
            y.x += k * z.x, y.y += k * z.y, y.z += k * z.z, y.w += k * z.w;
          }
          write(r, d, y, top, sum);
        }
      }
    }
    __syncthreads();  // the buffer is a ring again
  }
}

}  // namespace
}  // namespace cofie

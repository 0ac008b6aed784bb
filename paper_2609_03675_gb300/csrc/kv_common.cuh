// Shared by the rotary and the paged-cache kernels: element types, the
// rotation's table and angles, the place of a token in the cache, 4-bit codes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>
#include <string>

#include "cofie_kv.h"
#include "ngff_common.cuh"

struct cofie_rotary;

namespace cofie {

constexpr uint32_t kMaxPairs = 128;
constexpr uint32_t kMaxAxes = 4;
constexpr uint32_t kGroup = 64;  // codes that share a scale word

constexpr uint32_t kKvErrPage = 1u, kKvErrBatch = 2u, kKvErrWait = 4u;

// Passed to kernels by value.
struct RotaryTable {
  uint64_t turn[kMaxPairs];  // turns per position, as a fraction of 2^64
  uint8_t axis[kMaxPairs];
  double exact_amplitude;
  float amplitude;  // rounded
  uint32_t half;    // pairs
  uint32_t layout;  // COFIE_ROTARY_*
};

// SMs of the current device.
inline uint32_t sm_count() {
  static std::atomic<uint32_t> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 152;
  if (const uint32_t k = known[dev].load(std::memory_order_relaxed)) return k;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 152;
  known[dev].store(static_cast<uint32_t>(n), std::memory_order_relaxed);
  return static_cast<uint32_t>(n);
}

const RotaryTable& rotary_table(const cofie_rotary* h);
uint32_t rotary_head_dim(const cofie_rotary* h);
uint32_t rotary_axes(const cofie_rotary* h);

// Row r of a tensor, as the kernels see it.
struct RowsArg {
  const char* in;
  char* out;
  int64_t in_token, in_head, out_token, out_head;  // elements
  uint32_t heads;
  uint32_t kind;  // kRotate, kCopy: out is strided; kRotatePage, kCopyPage: out is the pages
};
enum : uint32_t { kRotate = 0, kCopy = 1, kRotatePage = 2, kCopyPage = 3 };

struct BatchArg {
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* offsets;
  uint32_t n_seqs, n_tokens, table_stride;
  uint32_t n_pages, page_shift, kv_heads;
  uint32_t* err;
  // groups of sequences that share a prefix: n_seqs of them, whose lengths and table rows are the prefixes', and whose new
  // tokens are those of sequences groups[g] to groups[g + 1] of the `members` that there are (without groups: of all)
  const int32_t* groups;
  uint32_t members;  // 0: sequences, not groups
};

// cos and sin of pair i at the given position, times the amplitude. The
// product wraps at 2^64 = one turn, which is what an angle does; its upper
// half, signed, is the angle in units of pi / 2^31.
__device__ __forceinline__ float2 rotary_cs(uint64_t turn, int32_t pos, float amplitude, bool transpose) {
  const uint64_t phase = turn * static_cast<uint64_t>(static_cast<int64_t>(pos));
  float s, c;
  sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f, &s, &c);
  return make_float2(c * amplitude, transpose ? -s * amplitude : s * amplitude);
}

// The sequence of token t: the last one that starts at or before it. n_seqs where t belongs to none.
__device__ __forceinline__ uint32_t sequence_of(const int32_t* offsets, uint32_t n_seqs, uint32_t t) {
  uint32_t lo = 0, hi = n_seqs;  // offsets[lo] <= t < offsets[hi], if t is in any
  if (static_cast<int64_t>(offsets[n_seqs]) <= static_cast<int64_t>(t) || offsets[0] > static_cast<int64_t>(t)) return n_seqs;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (offsets[mid] <= static_cast<int64_t>(t)) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Sequence s of the batch: its first row, its count of new tokens and of
// cached ones. Nothing at all (and the error noted) where they are out of range.
struct Span {
  uint32_t first, count, length;
};
__device__ __forceinline__ Span sequence_span(const BatchArg& b, uint32_t s) {
  const int64_t length = b.lengths[s];
  int64_t from = s, to = s + 1;
  if (b.members) {
    from = b.groups ? b.groups[s] : 0;
    to = b.groups ? b.groups[s + 1] : b.members;
    if (from < 0 || to < from || to > b.members) {
      atomicOr(b.err, kKvErrBatch);
      return {0, 0, 0};
    }
  }
  const int64_t first = b.offsets ? b.offsets[from] : from, end = b.offsets ? b.offsets[to] : to;
  if (length < 0 || length > (static_cast<int64_t>(b.table_stride) << b.page_shift) || first < 0 || end < first || end > b.n_tokens) {
    atomicOr(b.err, kKvErrBatch);
    return {0, 0, 0};
  }
  return {static_cast<uint32_t>(first), static_cast<uint32_t>(end - first), static_cast<uint32_t>(length)};
}

// Place of new token t among all pages' places (page * page_size + place), or
// -1 where the batch gives it none. `offsets` may be a copy in shared memory.
__device__ __forceinline__ int64_t place_of(const BatchArg& b, const int32_t* offsets, uint32_t t) {
  uint32_t s = t;
  int64_t at;
  if (b.offsets) {
    s = sequence_of(offsets, b.n_seqs, t);
    if (s >= b.n_seqs) return -1;
    const int64_t end = offsets[s + 1];
    at = end > b.n_tokens ? -1 : static_cast<int64_t>(b.lengths[s]) - (end - t);
  } else {
    if (s >= b.n_seqs) return -1;
    at = static_cast<int64_t>(b.lengths[s]) - 1;
  }
  if (at < 0 || (at >> b.page_shift) >= b.table_stride) {
    atomicOr(b.err, kKvErrBatch);
    return -1;
  }
  const uint32_t page = static_cast<uint32_t>(b.table[static_cast<uint64_t>(s) * b.table_stride + (at >> b.page_shift)]);
  if (page >= b.n_pages) {
    atomicOr(b.err, kKvErrPage);
    return -1;
  }
  return (static_cast<int64_t>(page) << b.page_shift) | (at & ((1 << b.page_shift) - 1));
}

// Row index of (place, head) in the pages: [page][head][place in page].
__device__ __forceinline__ uint64_t page_row(const BatchArg& b, int64_t place, uint32_t head) {
  const uint64_t page = static_cast<uint64_t>(place) >> b.page_shift;
  return ((page * b.kv_heads + head) << b.page_shift) | (static_cast<uint64_t>(place) & ((1u << b.page_shift) - 1));
}

template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int kLeast = -100, kMost = 121;  // exponents of 8-bit pages' scales
  static __device__ __forceinline__ float to(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Elem<__half> {
  static constexpr int kLeast = -24, kMost = 9;
  static __device__ __forceinline__ float to(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half from(float x) { return __float2half_rn(x); }
};
template <>
struct Elem<float> {
  static __device__ __forceinline__ float to(float x) { return x; }
  static __device__ __forceinline__ float from(float x) { return x; }
};

// fmin and fmax that pass a NaN on.
__device__ __forceinline__ float min_nan(float a, float b) {
  float x;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(a), "f"(b));
  return x;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float x;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(a), "f"(b));
  return x;
}

// The scale of a group from its extremes: the smallest number of 4 significant
// bits that 15 times reach hi - lo with (the product is exact); NaN where that
// is not finite.
__device__ __forceinline__ float group_scale(float lo, float hi) {
  const float range = __fsub_rn(hi, lo), near = range * (1.f / 15.f);
  float s = __uint_as_float(__float_as_uint(near) & ~0xFFFFFu);
  if (15.f * s < range) s = __uint_as_float(__float_as_uint(s) + 0x100000u);
  if (near < 0x1p-100f) s = 0.f;
  return range <= 3.402823466e38f ? s : __int_as_float(0x7FC00000);
}

// Two 16-bit values in a register.
template <typename T>
struct Two;
template <>
struct Two<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ float lo(uint32_t x) { return __uint_as_float(x << 16); }
  static __device__ __forceinline__ float hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }
};
template <>
struct Two<__half> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ float lo(uint32_t x) { return __half2float(__ushort_as_half(static_cast<unsigned short>(x))); }
  static __device__ __forceinline__ float hi(uint32_t x) { return __half2float(__ushort_as_half(static_cast<unsigned short>(x >> 16))); }
};

// Eight codes to (n - z) s, in the order (0, 4), (1, 5), (2, 6), (3, 7).
template <typename T>
struct Unpack;
template <>
struct Unpack<__nv_bfloat16> {
  __nv_bfloat162 z, s;
  __device__ __forceinline__ explicit Unpack(uint32_t word) {
    const uint32_t a = (word & 15u) | 0x4300u, b = word & 0xFFF0u;  // 128 + z
    const uint32_t aa = a | a << 16, bb = b | b << 16;
    z = *reinterpret_cast<const __nv_bfloat162*>(&aa);
    s = *reinterpret_cast<const __nv_bfloat162*>(&bb);
  }
  __device__ __forceinline__ uint4 operator()(uint32_t w) const {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;  // 128 + n
      const __nv_bfloat162 y = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), z), s);
      r[i] = *reinterpret_cast<const uint32_t*>(&y);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
  }
};
template <>
struct Unpack<__half> {
  __half2 z, z16, s;
  __device__ __forceinline__ explicit Unpack(uint32_t word) {
    const float f = static_cast<float>(word & 15u);
    z = __float2half2_rn(1024.f + f);
    z16 = __float2half2_rn(-64.f - f);
    s = __float2half2_rn(__uint_as_float((word & 0xFFF0u) << 16));
  }
  __device__ __forceinline__ uint4 operator()(uint32_t w) const {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = ((w >> (8 * (i / 2))) & (i % 2 ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;  // 1024 + n, 1024 + 16 n
      const __half2 h = *reinterpret_cast<const __half2*>(&x);
      const __half2 y = __hmul2(i % 2 ? __hfma2(h, __float2half2_rn(0.0625f), z16) : __hsub2(h, z), s);
      r[i] = *reinterpret_cast<const uint32_t*>(&y);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
  }
};

// Four bytes to (u - 128) s, in their order. s is a power of two, so that all
// is exact: bf16 holds 128 + the lower seven bits, and the eighth decides
// whether 128 or 256 comes off; fp16 holds 1024 + u. (Two products and a smaller
// of two in place of the masks are one instruction in five less, but past the
// type's range for scales of 2^120 and 2^121, and the way round for those cost
// more than it gave: 256 rows over 65792 tokens 285 -> 274 us, 800 rows 1239 ->
// 1318, tiles behind a mask 62 -> 70.)
template <typename T>
struct Bytes;
template <>
struct Bytes<__nv_bfloat16> {
  __nv_bfloat162 s;
  __device__ __forceinline__ explicit Bytes(uint32_t word) {
    const uint32_t ss = __byte_perm(word, word, 0x1010);
    s = *reinterpret_cast<const __nv_bfloat162*>(&ss);
  }
  __device__ __forceinline__ uint32_t two(uint32_t w, uint32_t which) const {
    const uint32_t x = __byte_perm(w, 0x43434343u, which), a = x & 0xFF7FFF7Fu, b = (x & 0xFF80FF80u) ^ 0x00800080u;
    const __nv_bfloat162 y = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b)), s);
    return *reinterpret_cast<const uint32_t*>(&y);
  }
  __device__ __forceinline__ uint2 operator()(uint32_t w) const { return make_uint2(two(w, 0x4140), two(w, 0x4342)); }
};
template <>
struct Bytes<__half> {
  __half2 s;
  __device__ __forceinline__ explicit Bytes(uint32_t word) { s = __float2half2_rn(__uint_as_float(word << 16)); }
  __device__ __forceinline__ uint32_t two(uint32_t w, uint32_t which) const {
    const uint32_t x = __byte_perm(w, 0x64646464u, which);
    const __half2 y = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&x), __float2half2_rn(1152.f)), s);
    return *reinterpret_cast<const uint32_t*>(&y);
  }
  __device__ __forceinline__ uint2 operator()(uint32_t w) const { return make_uint2(two(w, 0x4140), two(w, 0x4342)); }
};

// The word of 64 values from the largest of their sizes, and its inverse: the
// smallest power of two that brings it to 127 at most, from 2^kLeast to 2^kMost
// (of which the type holds 127); a NaN where the size is not finite. f 2^e, f in
// [1, 2), needs 2^(e - 6) for f up to 127 / 64 and 2^(e - 5) above: adding what
// the mantissa lacks there carries into the exponent.
template <typename T>
__device__ __forceinline__ uint32_t byte_scale(float size, float& inverse) {
  constexpr uint32_t least = 127 + Elem<T>::kLeast, most = 127 + Elem<T>::kMost;
  const uint32_t field = min(max((__float_as_uint(size) + 0x1FFFFu) >> 23, least + 6) - 6, most);
  inverse = __uint_as_float((254u - field) << 23);
  return size <= 3.402823466e38f ? field << 7 : 0x7FC0u;
}

}  // namespace cofie

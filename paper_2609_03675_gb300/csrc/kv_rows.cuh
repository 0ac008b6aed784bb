// Rows of heads, rotated or copied: the device code that the rotary kernel and
// the cache's append kernels share.
//
// A head's head_dim values are cut into units of 2 V values, each two vectors
// of V: in the half layout V pairs (x[i..], x[half + i..]), else 2 V values in
// a row, V pairs of neighbours or V + V values that pass through. V is the
// largest of 8, 4, 2, 1 (16 bytes at most) that the sizes, the strides and the
// addresses allow.
#pragma once

#include "kv_common.cuh"

namespace cofie {

struct RowsArgs {
  RowsArg rows[4];
  uint32_t n_rows, heads;          // heads of all rows
  uint32_t n_tokens, tile;         // tokens, and those of one CTA
  uint32_t units, rotary_units;    // units of a head, and those that rotate
  uint32_t offsets_in_smem;        // the batch's offsets are copied to shared memory
  const int32_t* positions;
  uint32_t transpose;
  uint32_t paged;                  // some rows go to pages
  BatchArg batch;
};

// V values as they lie in memory, read and written at once.
template <typename T, int V>
struct RowVec {
  static constexpr int kBytes = sizeof(T) * V, kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p) {
    if (kBytes == 16) {
      const uint4 x = *reinterpret_cast<const uint4*>(p);
      w[0] = x.x, w[1 % kWords] = x.y, w[2 % kWords] = x.z, w[3 % kWords] = x.w;
    } else if (kBytes == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x, w[1 % kWords] = x.y;
    } else if (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if (kBytes == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1 % kWords], w[2 % kWords], w[3 % kWords]);
    else if (kBytes == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1 % kWords]);
    else if (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
  }
  __device__ __forceinline__ void to(float* x) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(w[i]);
      else x[i] = i % 2 ? Two<T>::hi(w[i / 2]) : Two<T>::lo(w[i / 2]);
    }
  }
  __device__ __forceinline__ void from(const float* x) {
#pragma unroll
    for (int i = 0; i < V; i += sizeof(T) == 4 ? 1 : 2) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
      else w[i / 2] = Two<T>::pack(x[i], V > 1 ? x[(i + 1) % V] : 0.f);
    }
  }
};

// Eight 16-bit values whose address allows nothing wider.
template <typename T>
__device__ __forceinline__ uint4 gather8(const T* p) {
  const uint16_t* x = reinterpret_cast<const uint16_t*>(p);
  return make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
}

constexpr uint32_t kOffsetsInSmem = 1024;  // sequences whose offsets a CTA copies

// The CTA's angles: each token's pairs, as cos and sin, in units of two pairs
// (16 bytes) whose order lets eight neighbouring lanes that read eight pairs
// each meet every bank once.
inline __host__ __device__ uint32_t cs_stride(uint32_t half) { return (half + 15) & ~15u; }
__device__ __forceinline__ uint32_t cs_unit(uint32_t unit) { return unit ^ (unit >> 2 & 3u) ^ (unit >> 2 & 4u); }
template <int N>
__device__ __forceinline__ void load_cs(const float2* c, uint32_t pair, float2* to) {
  if (N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float4 x = reinterpret_cast<const float4*>(c)[cs_unit(pair / 2 + i / 2)];
      to[i] = make_float2(x.x, x.y);
      to[i + 1] = make_float2(x.z, x.w);
    }
  } else {
    to[0] = c[cs_unit(pair / 2) * 2 + pair % 2];
  }
}

inline __host__ __device__ size_t rows_smem(uint32_t tile, uint32_t half, uint32_t n_seqs, bool offsets) {
  return static_cast<size_t>(tile) * (cs_stride(half) * sizeof(float2) + sizeof(int64_t)) + (offsets ? (n_seqs + 1) * sizeof(int32_t) : 0);
}

// Fills the CTA's angles and places [tile]; ends with a barrier.
__device__ __forceinline__ void rows_set_up(const RowsArgs& a, const RotaryTable& tab, uint32_t t0, uint32_t n, float2* cs,
                                            int64_t* place, int32_t* offs) {
  for (uint32_t e = threadIdx.x; e < n * tab.half; e += blockDim.x) {
    const uint32_t t = e / tab.half, i = e - t * tab.half;
    const int32_t pos = a.positions[static_cast<uint64_t>(tab.axis[i]) * a.n_tokens + t0 + t];
    cs[t * cs_stride(tab.half) + cs_unit(i / 2) * 2 + i % 2] = rotary_cs(tab.turn[i], pos, tab.amplitude, a.transpose != 0);
  }
  if (a.paged) {
    const int32_t* offsets = a.batch.offsets;
    if (a.offsets_in_smem) {
      for (uint32_t s = threadIdx.x; s <= a.batch.n_seqs; s += blockDim.x) offs[s] = offsets[s];
      __syncthreads();
      offsets = offs;
    }
    for (uint32_t t = threadIdx.x; t < n; t += blockDim.x) place[t] = place_of(a.batch, offsets, t0 + t);
  }
  __syncthreads();
}

__device__ __forceinline__ void turn_pair(float& a, float& b, float2 cs) {
  const float x = a, y = b;
  a = x * cs.x - y * cs.y;
  b = y * cs.x + x * cs.y;
}

template <typename T, int V>
__device__ __forceinline__ void turn_unit(RowVec<T, V>& a, RowVec<T, V>& b, const float2* c, uint32_t pair, uint32_t layout) {
  float x[V], y[V];
  float2 cs[V];
  load_cs<V>(c, pair, cs);
  a.to(x);
  b.to(y);
  if (layout == COFIE_ROTARY_HALF || V == 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) turn_pair(x[i], y[i], cs[i]);
  } else {
#pragma unroll
    for (int i = 0; i + 1 < V; i += 2) {
      turn_pair(x[i], x[i + 1], cs[i / 2]);
      turn_pair(y[i], y[i + 1], cs[V / 2 + i / 2]);
    }
  }
  a.from(x);
  b.from(y);
}

// Heads [h0, h0 + heads) of tokens [t0, t0 + n), counted over all tensors. A
// thread keeps its unit of a head and goes from row to row: what depends on the
// unit is formed once (with the index of unit, head and token divided out of
// one counter for every unit, 65536 tokens of 40 heads took 243 us).
template <typename T, int V>
__device__ __forceinline__ void rows_run(const RowsArgs& a, const RotaryTable& tab, uint32_t t0, uint32_t n, uint32_t h0,
                                         uint32_t heads, const float2* cs, const int64_t* place) {
  using Vec = RowVec<T, V>;
  constexpr int kAtOnce = 2;  // rows whose loads are on their way together
  const uint32_t step = blockDim.x / a.units, mine = threadIdx.x / a.units, u = threadIdx.x - mine * a.units;
  if (mine >= step) return;
  uint32_t before = 0;  // heads of the tensors before
  for (uint32_t k = 0; k < a.n_rows; before += a.rows[k++].heads) {
    const RowsArg& x = a.rows[k];
    const uint32_t lo = max(h0, before), hi = min(h0 + heads, before + x.heads);
    if (lo >= hi) continue;
    const uint32_t count = hi - lo, inverse = 0xFFFFFFFFu / count + 1;  // row / count by a product: rows x count < 2^32
    const bool paged = x.kind >= kRotatePage;
    const bool turns = (x.kind == kRotate || x.kind == kRotatePage) && u < a.rotary_units;
    const bool by_half = turns && tab.layout == COFIE_ROTARY_HALF;
    const uint32_t o1 = by_half ? u * V : u * 2 * V, o2 = by_half ? tab.half + u * V : o1 + V;
    if (!turns && x.in == x.out) continue;  // in place: nothing moves
    const T* in = reinterpret_cast<const T*>(x.in) + static_cast<int64_t>(t0) * x.in_token + (lo - before) * x.in_head;
    T* out = reinterpret_cast<T*>(x.out);
    if (!paged) out += static_cast<int64_t>(t0) * x.out_token + (lo - before) * x.out_head;
    const uint32_t rows = n * count;
    for (uint32_t row0 = mine; row0 < rows; row0 += kAtOnce * step) {
      Vec y[kAtOnce], z[kAtOnce];
      T* to[kAtOnce];
      uint32_t at[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t row = row0 + i * step;
        to[i] = nullptr;
        if (row >= rows) continue;
        const uint32_t t = count == 1 ? row : __umulhi(row, inverse), h = row - t * count;
        const T* from = in + t * x.in_token + h * x.in_head;
        if (paged) {
          const int64_t p = place[t];
          if (p < 0) continue;
          to[i] = out + page_row(a.batch, p, lo - before + h) * (a.units * 2 * V);
        } else {
          to[i] = out + t * x.out_token + h * x.out_head;
        }
        at[i] = t;
        y[i].load(from + o1);
        z[i].load(from + o2);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (!to[i]) continue;
        if (turns) turn_unit<T, V>(y[i], z[i], cs + at[i] * cs_stride(tab.half), u * V, tab.layout);
        y[i].store(to[i] + o1);
        z[i].store(to[i] + o2);
      }
    }
  }
}

// Host: the widest V for these rows (elements of `size` bytes, head_dim values a head).
inline uint32_t rows_vector(const RowsArgs& a, const RotaryTable& tab, uint32_t head_dim, uint32_t size) {
  for (uint32_t v = 16 / size; v > 1; v /= 2) {
    bool ok = tab.half % v == 0 && (head_dim - 2 * tab.half) % (2 * v) == 0;
    for (uint32_t i = 0; ok && i < a.n_rows; ++i) {
      const RowsArg& r = a.rows[i];
      ok = reinterpret_cast<uintptr_t>(r.in) % (v * size) == 0 && reinterpret_cast<uintptr_t>(r.out) % (v * size) == 0 &&
           r.in_token % v == 0 && r.in_head % v == 0 && r.out_token % v == 0 && r.out_head % v == 0;
    }
    if (ok) return v;
  }
  return 1;
}

}  // namespace cofie

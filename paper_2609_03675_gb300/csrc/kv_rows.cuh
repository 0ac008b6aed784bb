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

template <typename T, int V>
struct alignas(sizeof(T) * V) RowVec {
  T v[V];
};

constexpr uint32_t kOffsetsInSmem = 1024;  // sequences whose offsets a CTA copies

inline __host__ __device__ size_t rows_smem(uint32_t tile, uint32_t half, uint32_t n_seqs, bool offsets) {
  return static_cast<size_t>(tile) * (half * sizeof(float2) + sizeof(int64_t)) + (offsets ? (n_seqs + 1) * sizeof(int32_t) : 0);
}

// Fills the CTA's angles [tile][half] and places [tile]; ends with a barrier.
__device__ __forceinline__ void rows_set_up(const RowsArgs& a, const RotaryTable& tab, uint32_t t0, uint32_t n, float2* cs,
                                            int64_t* place, int32_t* offs) {
  for (uint32_t e = threadIdx.x; e < n * tab.half; e += blockDim.x) {
    const uint32_t t = e / tab.half, i = e - t * tab.half;
    const int32_t pos = a.positions[static_cast<uint64_t>(tab.axis[i]) * a.n_tokens + t0 + t];
    cs[e] = rotary_cs(tab.turn[i], pos, tab.amplitude, a.transpose != 0);
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

template <typename T, int V>
struct RowUnit {
  const T* in;  // nullptr: nothing to do
  T* out;
  uint32_t o1, o2;  // the two vectors
  uint32_t pair;    // first pair of the unit, in the CTA's angles; ~0u: passes through
};

// Unit e of the CTA's (token, head, unit) list.
template <typename T, int V>
__device__ __forceinline__ RowUnit<T, V> row_unit(const RowsArgs& a, const RotaryTable& tab, uint32_t t0, uint32_t h0,
                                                  uint32_t heads, uint32_t e, const int64_t* place) {
  RowUnit<T, V> r;
  const uint32_t row = e / a.units, u = e - row * a.units;
  const uint32_t t = row / heads;
  uint32_t h = h0 + row - t * heads, k = 0;
  while (k + 1 < a.n_rows && h >= a.rows[k].heads) h -= a.rows[k++].heads;
  const RowsArg& x = a.rows[k];
  r.in = reinterpret_cast<const T*>(x.in) + static_cast<int64_t>(t0 + t) * x.in_token + h * x.in_head;
  if (x.kind >= kRotatePage) {
    const int64_t p = place[t];
    r.out = reinterpret_cast<T*>(x.out) + (p < 0 ? 0 : page_row(a.batch, p, h) * (a.units * 2 * V));
    if (p < 0) r.in = nullptr;
  } else {
    r.out = reinterpret_cast<T*>(x.out) + static_cast<int64_t>(t0 + t) * x.out_token + h * x.out_head;
  }
  const bool turns = (x.kind == kRotate || x.kind == kRotatePage) && u < a.rotary_units;
  if (turns && tab.layout == COFIE_ROTARY_HALF) {
    r.o1 = u * V;
    r.o2 = tab.half + u * V;
  } else {
    r.o1 = u * 2 * V;
    r.o2 = r.o1 + V;
    if (!turns && r.in == r.out) r.in = nullptr;  // in place: nothing moves
  }
  r.pair = turns ? t * tab.half + u * V : ~0u;
  return r;
}

template <typename T, int V>
__device__ __forceinline__ void turn_pair(T& x1, T& x2, float2 cs) {
  const float a = Elem<T>::to(x1), b = Elem<T>::to(x2);
  x1 = Elem<T>::from(a * cs.x - b * cs.y);
  x2 = Elem<T>::from(b * cs.x + a * cs.y);
}

template <typename T, int V>
__device__ __forceinline__ void turn_unit(RowVec<T, V>& a, RowVec<T, V>& b, const float2* cs, uint32_t layout) {
  if (layout == COFIE_ROTARY_HALF || V == 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) turn_pair<T, V>(a.v[i], b.v[i], cs[i]);
  } else {
#pragma unroll
    for (int i = 0; i + 1 < V; i += 2) {
      turn_pair<T, V>(a.v[i], a.v[i + 1], cs[i / 2]);
      turn_pair<T, V>(b.v[i], b.v[i + 1], cs[V / 2 + i / 2]);
    }
  }
}

// Heads [h0, h0 + heads) of tokens [t0, t0 + n).
template <typename T, int V>
__device__ __forceinline__ void rows_run(const RowsArgs& a, const RotaryTable& tab, uint32_t t0, uint32_t n, uint32_t h0,
                                         uint32_t heads, const float2* cs, const int64_t* place) {
  using Vec = RowVec<T, V>;
  const uint32_t total = n * heads * a.units;
  for (uint32_t e = threadIdx.x; e < total; e += blockDim.x) {
    const RowUnit<T, V> r = row_unit<T, V>(a, tab, t0, h0, heads, e, place);
    if (!r.in) continue;
    Vec x = *reinterpret_cast<const Vec*>(r.in + r.o1), y = *reinterpret_cast<const Vec*>(r.in + r.o2);
    if (r.pair != ~0u) turn_unit<T, V>(x, y, cs + r.pair, tab.layout);
    *reinterpret_cast<Vec*>(r.out + r.o1) = x;
    *reinterpret_cast<Vec*>(r.out + r.o2) = y;
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

// The paged cache: its handle, appending to it and reading it back.
#include <algorithm>
#include <cstring>
#include <new>
#include <type_traits>

#include "kv_handle.cuh"

namespace cofie {
namespace {

constexpr int kThreads = 256;
thread_local std::string g_kv_error;

struct CodesArgs {
  RowsArgs rows;  // queries, if any, as strided rows
  const char* in[2];  // keys, values
  int64_t in_token[2], in_head[2];
  uint32_t* codes[2];
  uint16_t* words[2];
  uint32_t kv_heads, q_parts;
};

// zero + n, n the code's distance from the zero point, a step nearer to it where
// x lies more than half a step from n (then it lies on that side). A step of 0
// or NaN has no codes.
__device__ __forceinline__ float code_back(float code, float zero, float x, float step) {
  const bool past = step > 0.f && fabsf(__fmaf_rn(zero - code, step, x)) > 0.5f * step;
  return past ? code - copysignf(1.f, x) : code;
}

// Value d of a head, turned in 64 bits, as a byte's sum (see below): for the few
// that lie closer to a half than fp32 tells.
template <typename T>
__device__ __noinline__ float exact_byte(const T* in, uint32_t d, uint32_t half, bool by_half, uint64_t turn, int32_t pos, double amplitude, float inverse) {
  const bool second = by_half ? d >= half : d & 1;
  const double x = Elem<T>::to(in[d]), y = Elem<T>::to(in[by_half ? (second ? d - half : d + half) : d ^ 1]);
  double s, c;
  sincospi(static_cast<double>(static_cast<int64_t>(turn * static_cast<uint64_t>(static_cast<int64_t>(pos)))) * 0x1p-63, &s, &c);
  return static_cast<float>(rint((x * c + (second ? y * s : -y * s)) * amplitude * inverse) + 12583040.0);
}

// Appends to pages of 4-bit codes or of bytes. CTAs of gridDim.y below q_parts rotate the queries;
// the others take a share of the (key or value, head) rows of their tokens.
// Sixteen values of a row to a lane, eight from either half of the head, so that
// where all of it rotates in the half layout a lane holds both of a pair; the
// lanes of a group find its extremes by shuffles. WIDE: rows are read 16 bytes at a time, and what a
// value is rotated with lies in as many pieces (sizes and strides that allow
// it); else value by value.
// 75264 tokens of 8 heads to bytes: 150 us (154 MB written, 309 read: 68 at DRAM's
// rate); without the look for bytes that fp32 leaves open 118, with rows asked for
// only when their places were there 10 more. Issue slots 58 % busy, the ALU pipe 55 %.
template <typename T, int V, int D, int BITS, bool WIDE>
__global__ void __launch_bounds__(kThreads, 4) append_codes(const __grid_constant__ CodesArgs a, const __grid_constant__ RotaryTable tab) {
  extern __shared__ __align__(16) float2 cs[];
  const RowsArgs& r = a.rows;
  int64_t* place = reinterpret_cast<int64_t*>(cs + r.tile * cs_stride(tab.half));
  int32_t* offs = reinterpret_cast<int32_t*>(place + r.tile);
  const uint32_t t0 = blockIdx.x * r.tile, n = min(r.tile, r.n_tokens - t0);
  pdl_trigger();
  pdl_wait();
  if (WIDE && blockIdx.y >= a.q_parts) {  // the CTA's rows are asked for before its angles and places are formed
    const uint32_t parts0 = gridDim.y - a.q_parts, part0 = blockIdx.y - a.q_parts;
    const uint32_t per0 = (2 * a.kv_heads + parts0 - 1) / parts0, first = part0 * per0, many = min(per0, 2 * a.kv_heads - min(first, 2 * a.kv_heads));
    constexpr uint32_t kLines = D * 2 / 128;
    for (uint32_t e = threadIdx.x; e < many * n * kLines; e += kThreads) {
      const uint32_t line = e % kLines, row = e / kLines, kind0 = first + row % many, t = row / many;
      const uint32_t v0 = kind0 >= a.kv_heads, head0 = kind0 - v0 * a.kv_heads;
      const char* p = a.in[v0] + 2 * (static_cast<int64_t>(t0 + t) * a.in_token[v0] + head0 * a.in_head[v0]) + line * 128;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
    }
  }
  rows_set_up(r, tab, t0, n, cs, place, offs);
  if (blockIdx.y < a.q_parts) {
    const uint32_t per = (r.heads + a.q_parts - 1) / a.q_parts, h0 = blockIdx.y * per;
    if (h0 < r.heads) rows_run<T, V>(r, tab, t0, n, h0, min(per, r.heads - h0), cs, place);
    return;
  }
  constexpr uint32_t kLanes = D / 16;  // of a row
  const uint32_t parts = gridDim.y - a.q_parts, part = blockIdx.y - a.q_parts;
  const uint32_t per = (2 * a.kv_heads + parts - 1) / parts, k0 = part * per, k1 = min(k0 + per, 2 * a.kv_heads);
  const uint32_t lane = threadIdx.x % kLanes, mine = threadIdx.x % 32 / kLanes;
  const bool by_half = tab.layout == COFIE_ROTARY_HALF;
  // a warp takes the keys or the values of a head, several tokens at a time
  for (uint32_t kind = k0 + threadIdx.x / 32; kind < k1; kind += kThreads / 32) {
    const uint32_t v = kind >= a.kv_heads, head = kind - v * a.kv_heads;
    const T* const in0 = reinterpret_cast<const T*>(a.in[v]) + static_cast<int64_t>(t0) * a.in_token[v] + head * a.in_head[v];
    const int64_t in_token = a.in_token[v];
    uint32_t* const codes = a.codes[v] + static_cast<uint64_t>(head << r.batch.page_shift) * (D * BITS / 32);
    uint16_t* const words = a.words[v] + static_cast<uint64_t>(head << r.batch.page_shift) * (D / kGroup);
    const uint32_t turned = v ? 0 : 2 * tab.half;  // values that are rotated
    RowVec<T, 8> w[2], ahead[2];                   // the lane's values, and those of the next tokens
    const auto fetch = [&](uint32_t t1, RowVec<T, 8>* to) {
      const uint32_t t = t1 + mine;
      if (!WIDE || t >= n) return;
      to[0].load(in0 + t * in_token + lane * 8);
      to[1].load(in0 + t * in_token + D / 2 + lane * 8);
    };
    fetch(0, ahead);
    for (uint32_t t1 = 0; t1 < n; t1 += 32 / kLanes) {  // whole warps stay in the loop, for the shuffles
      const uint32_t t = t1 + mine;
      const int64_t p = t < n ? place[t] : -1;
      w[0] = ahead[0];
      w[1] = ahead[1];
      fetch(t1 + 32 / kLanes, ahead);
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
      if (p >= 0) {
        const T* in = in0 + t * in_token;
        const float2* c = cs + t * cs_stride(tab.half);
        if (WIDE) {
          w[0].to(x);
          w[1].to(x + 8);
          if (turned == D && by_half) {
            float2 z[8];
            load_cs<8>(c, lane * 8, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) turn_pair(x[i], x[8 + i], z[i]);
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t d = e * (D / 2) + lane * 8;
              if (d >= turned) continue;
              if (by_half) {
                const bool second = d >= tab.half;
                const uint32_t o = second ? d - tab.half : d;
                RowVec<T, 8> other;
                other.load(in + (second ? o : d + tab.half));
                float y[8];
                float2 z[8];
                other.to(y);
                load_cs<8>(c, o, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[8 * e + i] = x[8 * e + i] * z[i].x + y[i] * (second ? z[i].y : -z[i].y);
              } else {
                float2 z[4];
                load_cs<4>(c, d / 2, z);
#pragma unroll
                for (int i = 0; i < 4; ++i) turn_pair(x[8 * e + 2 * i], x[8 * e + 2 * i + 1], z[i]);
              }
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t d = i / 8 * (D / 2) + lane * 8 + i % 8;
            x[i] = Elem<T>::to(in[d]);
            if (d < turned) {
              const bool second = by_half ? d >= tab.half : d & 1;
              const uint32_t pair = by_half ? (second ? d - tab.half : d) : d / 2;
              const float other = Elem<T>::to(in[by_half ? (second ? d - tab.half : d + tab.half) : d ^ 1]);
              float2 z;
              load_cs<1>(c, pair, &z);
              x[i] = x[i] * z.x + other * (second ? z.y : -z.y);
            }
          }
        }
      }
      constexpr int kOwn = D / 64;
      uint32_t word[2], codes8[2][2];
      if constexpr (BITS == 8) {
        // the largest size of each of the lane's groups; x / s is exact but for what lies under the smallest scale, and
        // 1.5 2^23 + 128 more rounds it to a whole number, halves to even, whose byte is the low one. A rotated key is off by
        // 2.8e-7 (|x| + |y|) of its pair (angle 9.4e-8, cos and sin 6e-8, products and sum 1.2e-7), so by 5.6e-7 of the
        // largest turned value of the pair at most: one that lies so close to a half is turned once more in 64 bits. (One in
        // 10^4; without that one in 3 10^5 bytes of rotated keys was its neighbour.) An amplitude adds its own rounding and that
        // of its products with cos and sin, 6e-8 each of the pair's length, which is sqrt 2 times the largest at most: 1.7e-7.
        float size[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 16; ++i) size[kOwn == 1 ? 0 : i / 8] = max_nan(size[kOwn == 1 ? 0 : i / 8], fabsf(x[i]));
        // (where a pair's other value is another lane's, the row's largest stands for the lane's)
        float inverse[2], reach = fmaxf(size[0], size[1]);
#pragma unroll
        for (int o = 1; o < static_cast<int>(kLanes); o <<= 1)
#pragma unroll
          for (int gr = 0; gr < kOwn; ++gr) size[gr] = max_nan(size[gr], __shfl_xor_sync(0xffffffffu, size[gr], o));
        if (by_half && turned != D) reach = fmaxf(size[0], size[1]);
#pragma unroll
        for (int gr = 0; gr < kOwn; ++gr) word[gr] = byte_scale<T>(size[gr], inverse[gr]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int gr = kOwn == 1 ? 0 : e;
          uint32_t u[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(__fmaf_rn(x[8 * e + i], inverse[gr], 12583040.f));
          if (turned) {
            float near = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              near = fmaxf(near, fabsf(__fmaf_rn(x[8 * e + i], inverse[gr], 12583040.f - __uint_as_float(u[i]))));
            const float off = (tab.amplitude == 1.f ? 6e-7f : 8e-7f) * reach * inverse[gr];
            if (p >= 0 && near > 0.5f - off) {
              const T* in = in0 + t * in_token;
              uint32_t close = 0;
#pragma unroll
              for (int i = 0; i < 8; ++i)
                close |= (fabsf(__fmaf_rn(x[8 * e + i], inverse[gr], 12583040.f - __uint_as_float(u[i]))) > 0.5f - off ? 1u : 0u) << i;
#pragma unroll 1
              for (; close; close &= close - 1) {
                const uint32_t i = __ffs(close) - 1, d = e * (D / 2) + lane * 8 + i;
                if (d >= turned) break;
                const uint32_t pair = by_half ? (d >= tab.half ? d - tab.half : d) : d / 2;
                const int32_t pos = r.positions[static_cast<uint64_t>(tab.axis[pair]) * r.n_tokens + t0 + t];
                const float exact = exact_byte(in, d, tab.half, by_half, tab.turn[pair], pos, tab.exact_amplitude, inverse[gr]);
#pragma unroll
                for (uint32_t f = 0; f < 8; ++f)
                  if (f == i) u[f] = __float_as_uint(exact);
              }
            }
          }
          if (!(size[gr] * inverse[gr] <= 127.f)) {  // past the largest scale's range
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(fminf(fmaxf(__uint_as_float(u[i]), 12582913.f), 12583167.f));
          }
          // the bytes are the low bits of 0x4B400000 + byte, whose sum's share is taken off at the end (products and sums
          // where byte permutations would wait for the pipe that the extremes keep busy)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            codes8[e][i] = ((u[4 * i + 3] * 256 + u[4 * i + 2]) * 256 + u[4 * i + 1]) * 256 + u[4 * i] - 0x4B400000u * 0x01010101u;
        }
      } else {
        // the extremes of the lane's groups: its two eights are of one (D = 64) or of two
        float lo[2] = {0.f, 0.f}, hi[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int gr = kOwn == 1 ? 0 : i / 8;
          lo[gr] = min_nan(lo[gr], x[i]);
          hi[gr] = max_nan(hi[gr], x[i]);
        }
#pragma unroll
        for (int o = 1; o < static_cast<int>(kLanes); o <<= 1)
#pragma unroll
          for (int gr = 0; gr < kOwn; ++gr) {
            lo[gr] = min_nan(lo[gr], __shfl_xor_sync(0xffffffffu, lo[gr], o));
            hi[gr] = max_nan(hi[gr], __shfl_xor_sync(0xffffffffu, hi[gr], o));
          }
        // x / scale to the nearest, halves away from zero: the reciprocal (good to
        // a last place) is taken two above its value, so that no half stays one,
        // and the product and the zero point are summed and rounded once, to the
        // last bit of 1.5 2^23. No quotient of 16-bit x lies that close to a half
        // without being one, but one of rotated keys, which are fp32 numbers, may:
        // where the reciprocal two below its value gives another code, x - code
        // scale, which is exact, is held against half a scale. (75000 appended
        // tokens take 152 us so, 154 with every key held against it, and 135 took
        // those whose codes could be the next.)
        float inv[2], low[2], zero[2], step[2];
#pragma unroll
        for (int gr = 0; gr < kOwn; ++gr) {
          const float scale = group_scale(lo[gr], hi[gr]);
          asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv[gr]) : "f"(scale));
          low[gr] = scale > 0.f ? __uint_as_float(__float_as_uint(inv[gr]) - 2) : 0.f;
          inv[gr] = scale > 0.f ? __uint_as_float(__float_as_uint(inv[gr]) + 2) : 0.f;
          float near = __fmaf_rn(-lo[gr], inv[gr], 12582912.f);
          if (turned) near = code_back(near, 12582912.f, -lo[gr], scale);
          zero[gr] = fminf(near, 12582927.f);
          step[gr] = scale;
          word[gr] = (__float_as_uint(scale) >> 16) | (__float_as_uint(zero[gr]) & 15u);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // codes are the low bits of 0x4B400000 + code, whose sum's share is taken off at the end
          uint32_t w = 0;
          const int gr = kOwn == 1 ? 0 : e;
          const auto code = [&](int i) { return __fmaf_rn(x[8 * e + i], inv[gr], zero[gr]); };
          if (!turned) {
#pragma unroll
            for (int i = 7; i >= 0; --i) w = w * 16 + __float_as_uint(fminf(code(i), 12582927.f));
          } else {
            uint32_t apart = 0;  // codes that the reciprocal two below its value gives otherwise
#pragma unroll
            for (int i = 7; i >= 0; --i) {
              const float c1 = code(i);
              apart |= __float_as_uint(c1) ^ __float_as_uint(__fmaf_rn(x[8 * e + i], low[gr], zero[gr]));
              w = w * 16 + __float_as_uint(fminf(c1, 12582927.f));
            }
            if (apart) {
              w = 0;
#pragma unroll
              for (int i = 7; i >= 0; --i) w = w * 16 + __float_as_uint(fminf(code_back(code(i), zero[gr], x[8 * e + i], step[gr]), 12582927.f));
            }
          }
          codes8[e][0] = w - 0x4B400000u * 0x11111111u;
        }
      }
      if (p >= 0) {
        // the row of the page's first head, to which the head's places were added above
        const uint64_t page = static_cast<uint64_t>(p) >> r.batch.page_shift;
        const uint64_t at = ((page * a.kv_heads) << r.batch.page_shift) + (static_cast<uint32_t>(p) & ((1u << r.batch.page_shift) - 1));
        if (BITS == 8) {
          uint2* const to = reinterpret_cast<uint2*>(codes) + at * (D / 8) + lane;
          to[0] = make_uint2(codes8[0][0], codes8[0][1]);
          to[kLanes] = make_uint2(codes8[1][0], codes8[1][1]);
        } else {
          codes[at * (D / 8) + lane] = codes8[0][0];
          codes[at * (D / 8) + kLanes + lane] = codes8[1][0];
        }
        if (lane == 0) {
          if (kOwn == 2) reinterpret_cast<uint32_t*>(words)[at] = word[0] | word[1] << 16;
          else words[at] = static_cast<uint16_t>(word[0]);
        }
      }
    }
  }
}

struct ReadArgs {
  BatchArg batch;
  const char* pages[2];
  const uint16_t* words[2];
  uint4* out[2];
};

constexpr uint32_t kReadTile = 16;  // tokens of a CTA

// A warp takes the keys or the values of a head, some tokens at a time, eight
// values of a row to a lane, or 16 bytes.
template <typename T, int D, int BITS>
__global__ void __launch_bounds__(kThreads) read_pages(const __grid_constant__ ReadArgs a) {
  constexpr uint32_t kValues = BITS == 8 ? 16 : 8, kLanes = D / kValues, kStep = 32 / kLanes;
  __shared__ int64_t place[kReadTile];
  pdl_trigger();
  pdl_wait();
  const uint32_t t0 = blockIdx.x * kReadTile, n = min(kReadTile, a.batch.n_tokens - t0);
  if (threadIdx.x < n) place[threadIdx.x] = place_of(a.batch, a.batch.offsets, t0 + threadIdx.x);
  __syncthreads();
  const uint32_t lane = threadIdx.x % kLanes, mine = threadIdx.x % 32 / kLanes, kv = a.batch.kv_heads, shift = a.batch.page_shift;
  for (uint32_t kind = blockIdx.y * (kThreads / 32) + threadIdx.x / 32; kind < 2 * kv; kind += gridDim.y * (kThreads / 32)) {
    const uint32_t v = kind >= kv, head = kind - v * kv;
    // from the head's place in a page
    const char* const pages = a.pages[v] + static_cast<uint64_t>(head << shift) * (D * BITS / 8) + lane * (kValues * BITS / 8);
    const uint16_t* const words = a.words[v] + static_cast<uint64_t>(head << shift) * (D / kGroup) + lane * kValues / kGroup;
    uint4* const out = a.out[v] + (static_cast<uint64_t>(t0) * kv + head) * (D / 8) + lane * (kValues / 8);
    using Raw = std::conditional_t<BITS == 4, uint32_t, uint4>;
    constexpr int kAtOnce = kReadTile / kStep < 4 ? kReadTile / kStep : 4;  // rows whose loads are on their way together
    for (uint32_t t1 = mine; t1 < n; t1 += kAtOnce * kStep) {
      int64_t p[kAtOnce];
      Raw x[kAtOnce];
      uint32_t word[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t t = t1 + i * kStep;
        p[i] = t < n ? place[t] : -1;
        // (the pages' first row is there to be read where the batch gives the token no place)
        const int64_t q = max(p[i], static_cast<int64_t>(0));
        const uint64_t at = ((static_cast<uint64_t>(q) >> shift) * kv << shift) + (static_cast<uint32_t>(q) & ((1u << shift) - 1));
        x[i] = *reinterpret_cast<const Raw*>(pages + at * (D * BITS / 8));
        word[i] = BITS < 16 ? words[at * (D / kGroup)] : 0;
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t t = t1 + i * kStep;
        if (t >= n) continue;
        uint4 val = make_uint4(0, 0, 0, 0), more = val;
        if (p[i] >= 0) {
          if constexpr (BITS == 16) {
            val = x[i];
          } else if constexpr (BITS == 8) {
            const Bytes<T> u(word[i]);
            const uint2 y0 = u(x[i].x), y1 = u(x[i].y), y2 = u(x[i].z), y3 = u(x[i].w);
            val = make_uint4(y0.x, y0.y, y1.x, y1.y);
            more = make_uint4(y2.x, y2.y, y3.x, y3.y);
          } else {
            const Unpack<T> u(word[i]);
            const uint4 y = u(x[i]);  // (0, 4), (1, 5), (2, 6), (3, 7)
            val = make_uint4(__byte_perm(y.x, y.y, 0x5410), __byte_perm(y.z, y.w, 0x5410), __byte_perm(y.x, y.y, 0x7632),
                             __byte_perm(y.z, y.w, 0x7632));
          }
        }
        uint4* const to = out + static_cast<uint64_t>(t) * kv * (D / 8);
        to[0] = val;
        if (BITS == 8) to[1] = more;
      }
    }
  }
}

template <typename T, int D, int BITS>
cudaError_t launch_codes(CodesArgs a, const RotaryTable& tab, bool queries, cudaStream_t st) {
  RowsArgs& r = a.rows;
  uint32_t v = queries ? rows_vector(r, tab, D, 2) : 8;
  bool wide = v == 8 && tab.half % (tab.layout == COFIE_ROTARY_HALF ? 8 : 4) == 0;
  for (int i = 0; i < 2; ++i)
    wide = wide && reinterpret_cast<uintptr_t>(a.in[i]) % 16 == 0 && a.in_token[i] % 8 == 0 && a.in_head[i] % 8 == 0;
  if (!wide) v = v >= 2 ? 2 : 1;
  r.units = D / (2 * v);
  r.rotary_units = tab.half / v;
  r.offsets_in_smem = r.batch.offsets && r.batch.n_seqs <= kOffsetsInSmem;
  r.tile = r.n_tokens >= sm_count() * 32 ? 16 : r.n_tokens >= sm_count() * 8 ? 4 : 1;
  const uint32_t tiles = (r.n_tokens + r.tile - 1) / r.tile;
  const uint32_t parts = std::max(1u, std::min(2 * a.kv_heads, sm_count() * 4 / tiles));
  a.q_parts = queries ? std::max(1u, std::min(r.heads, sm_count() * 4 / tiles)) : 0;
  const dim3 grid(tiles, parts + a.q_parts);
  const size_t smem = rows_smem(r.tile, tab.half, r.batch.n_seqs, r.offsets_in_smem);
  const auto go = [&](auto kernel) { return launch_dependent(true, kernel, grid, dim3(kThreads), smem, st, a, tab); };
  if (wide) return go(append_codes<T, 8, D, BITS, true>);
  return v == 2 ? go(append_codes<T, 2, D, BITS, false>) : go(append_codes<T, 1, D, BITS, false>);
}

template <typename T, int D>
cudaError_t launch_read(const ReadArgs& a, uint32_t bits, cudaStream_t st) {
  const uint32_t tiles = (a.batch.n_tokens + kReadTile - 1) / kReadTile, most = (2 * a.batch.kv_heads + kThreads / 32 - 1) / (kThreads / 32);
  const dim3 grid(tiles, std::max(1u, std::min(most, sm_count() * 4 / tiles)));
  if (bits == 8) return launch_dependent(true, read_pages<T, D, 8>, grid, dim3(kThreads), 0, st, a);
  return bits == 4 ? launch_dependent(true, read_pages<T, D, 4>, grid, dim3(kThreads), 0, st, a)
                   : launch_dependent(true, read_pages<T, D, 16>, grid, dim3(kThreads), 0, st, a);
}

bool on_device(const void* p, int dev) {
  cudaPointerAttributes a;
  if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return (a.type == cudaMemoryTypeDevice || a.type == cudaMemoryTypeManaged) && a.device == dev;
}

void kv_free(cofie_kv* h) {
  if (!h) return;
  DeviceGuard g(h->device);
  cudaDeviceSynchronize();
  for (void* x : {static_cast<void*>(h->d_err), static_cast<void*>(h->d_part), static_cast<void*>(h->d_part_ms), static_cast<void*>(h->d_done), h->d_items,
                  static_cast<void*>(h->d_tiles)})
    if (x) cudaFree(x);
  for (uint32_t i = 0; i < h->n_tiles_before; ++i) cudaFree(h->d_tiles_before[i]);
  for (const cofie_kv::Scratch* s : {&h->shared_rows, &h->shared_mask}) {
    if (s->p) cudaFree(s->p);
    for (uint32_t i = 0; i < s->n_before; ++i) cudaFree(s->before[i]);
  }
  delete h;
}

}  // namespace

int check_batch(cofie_kv* h, const cofie_kv_batch* b) {
  if (!b) return h->fail(COFIE_EINVAL, "the batch is NULL");
  if (b->n_tokens > 0x7fffffffu || b->n_seqs > 0x7fffffffu) return h->fail(COFIE_EINVAL, "n_tokens and n_seqs must be below 2^31");
  if (b->n_tokens == 0) return COFIE_OK;
  if (b->n_seqs == 0) return h->fail(COFIE_EINVAL, "a batch with tokens needs sequences");
  if (!b->table || !b->lengths) return h->fail(COFIE_EINVAL, "table and lengths are required");
  if (b->table_stride < 1 || b->table_stride > 0x7fffffffu / h->p.page_size)
    return h->fail(COFIE_EINVAL, "table_stride x page_size must be in [page_size, 2^31)");
  if (!b->offsets && b->n_tokens != b->n_seqs) return h->fail(COFIE_EINVAL, "without offsets every sequence has one new token");
  return COFIE_OK;
}

int check_rows(cofie_kv* h, const cofie_rows* r, uint32_t heads, bool has_out, const char* name) {
  const std::string n(name);
  if (!r->in || (has_out && !r->out)) return h->fail(COFIE_EINVAL, n + " is NULL");
  if (r->heads != heads) return h->fail(COFIE_EINVAL, n + " must have " + std::to_string(heads) + " heads");
  if (reinterpret_cast<uintptr_t>(r->in) % 2 || (has_out && reinterpret_cast<uintptr_t>(r->out) % 2))
    return h->fail(COFIE_EINVAL, n + " is not aligned to its type");
  return COFIE_OK;
}

BatchArg batch_arg(const cofie_kv* h, const cofie_kv_batch* b) {
  return {b->table, b->lengths, b->offsets, b->n_seqs, b->n_tokens, b->table_stride, h->p.n_pages, h->page_shift, h->p.n_kv_heads, h->d_err,
          nullptr, 0};
}

int launched(cofie_kv* h, cudaError_t e, const char* what) {
  if (e == cudaSuccess) return COFIE_OK;
  cudaGetLastError();
  return h->fail(COFIE_ECUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

}  // namespace cofie

using namespace cofie;

extern "C" {

int cofie_kv_create(const cofie_kv_params* p, cofie_kv_t** out) {
  const auto bad = [](const char* m) { return g_kv_error = m, COFIE_EINVAL; };
  if (!p || !out) return bad("params or out is NULL");
  if (p->n_pages < 1 || p->n_pages > 0x7fffffffu) return bad("n_pages must be in [1, 2^31)");
  uint32_t shift = 4;
  while (shift <= 8 && (1u << shift) != p->page_size) ++shift;
  if (shift > 8) return bad("page_size must be 16, 32, 64, 128 or 256");
  if (p->n_heads < 1 || p->n_kv_heads < 1 || p->n_heads > 1024 || p->n_heads % p->n_kv_heads)
    return bad("n_kv_heads must divide n_heads, at most 1024");
  if (p->head_dim != 64 && p->head_dim != 128) return bad("head_dim must be 64 or 128");
  if (p->dtype != COFIE_BF16 && p->dtype != COFIE_FP16) return bad("dtype must be COFIE_BF16 or COFIE_FP16");
  if (p->bits != 16 && p->bits != 4 && p->bits != COFIE_KV_INT8) return bad("bits must be 16, 4 or COFIE_KV_INT8");
  if (!p->k_pages || !p->v_pages || (p->bits != 16 && (!p->k_scales || !p->v_scales)))
    return bad("the pages (and for less than 16 bits the scales) are required");
  for (const void* x : {static_cast<const void*>(p->k_pages), static_cast<const void*>(p->v_pages),
                        static_cast<const void*>(p->k_scales), static_cast<const void*>(p->v_scales)})
    if (reinterpret_cast<uintptr_t>(x) % 16) return bad("pages and scales must be 16-byte aligned");
  int dev = p->device;
  if (dev < 0 && cudaGetDevice(&dev) != cudaSuccess) return g_kv_error = "no CUDA device", COFIE_ECUDA;
  int count = 0;
  if (cudaGetDeviceCount(&count) != cudaSuccess || dev >= count) {
    cudaGetLastError();
    return g_kv_error = "cannot select the device", COFIE_ECUDA;
  }
  DeviceGuard g(dev);
  if (!on_device(p->k_pages, dev) || !on_device(p->v_pages, dev) ||
      (p->bits != 16 && (!on_device(p->k_scales, dev) || !on_device(p->v_scales, dev))))
    return bad("the pages must be device memory on the handle's device");
  cofie_kv* h = new (std::nothrow) cofie_kv();
  if (!h) return g_kv_error = "host allocation failed", COFIE_ENOMEM;
  h->p = *p;
  h->p.bits = p->bits & 0xFF;  // 16, 8 or 4 from here
  h->device = dev;
  h->page_shift = shift;
  cudaError_t e = injected_alloc_failure() ? cudaErrorMemoryAllocation : cudaMalloc(&h->d_err, sizeof(uint32_t));
  if (e == cudaSuccess) e = cudaMemset(h->d_err, 0, sizeof(uint32_t));
  if (e == cudaSuccess) e = attend_set_up(h);
  // the words are cleared on the default stream: streams that do not wait for it may be the first to use them
  if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
  if (e != cudaSuccess) {
    g_kv_error = std::string("cache set-up failed: ") + cudaGetErrorString(e);
    cudaGetLastError();
    kv_free(h);
    return e == cudaErrorMemoryAllocation ? COFIE_ENOMEM : COFIE_ECUDA;
  }
  *out = h;
  return COFIE_OK;
}

void cofie_kv_destroy(cofie_kv_t* h) { kv_free(h); }

int cofie_kv_append(cofie_kv_t* h, const cofie_kv_batch* b, const cofie_rows* k, const cofie_rows* v, const cofie_rows* q,
                    const cofie_rotary_t* rotary, const int32_t* positions, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  if (const int rc = check_batch(h, b)) return rc;
  if (b->n_tokens == 0) return COFIE_OK;
  if (!k || !v) return h->fail(COFIE_EINVAL, "k and v are required");
  if (const int rc = check_rows(h, k, h->p.n_kv_heads, false, "k")) return rc;
  if (const int rc = check_rows(h, v, h->p.n_kv_heads, false, "v")) return rc;
  if (q) {
    if (!rotary) return h->fail(COFIE_EINVAL, "q without rotary has nothing to be done to it");
    if (const int rc = check_rows(h, q, h->p.n_heads, true, "q")) return rc;
    if (q->in == q->out && (q->in_token != q->out_token || q->in_head != q->out_head))
      return h->fail(COFIE_EINVAL, "in place, the strides of q's in and out must be the same");
  }
  if (rotary && rotary_head_dim(rotary) != h->p.head_dim) return h->fail(COFIE_EINVAL, "rotary's head_dim is not the cache's");
  if (rotary && !positions) return h->fail(COFIE_EINVAL, "positions is required with rotary");
  DeviceGuard g(h->device);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  static const RotaryTable none{};
  const RotaryTable& tab = rotary ? rotary_table(rotary) : none;
  RowsArgs a{};
  a.n_tokens = b->n_tokens;
  a.positions = positions;
  a.paged = 1;
  a.batch = batch_arg(h, b);
  const auto rows = [](const cofie_rows* r, void* out, uint32_t kind) {
    return RowsArg{static_cast<const char*>(r->in), static_cast<char*>(out), r->in_token, r->in_head, r->out_token, r->out_head, r->heads, kind};
  };
  if (q) a.rows[a.n_rows++] = rows(q, q->out, kRotate);
  cudaError_t e;
  if (h->p.bits == 16) {
    cofie_rows kr = *k, vr = *v;
    kr.out_token = kr.out_head = vr.out_token = vr.out_head = 0;
    a.rows[a.n_rows++] = rows(&kr, h->p.k_pages, kRotatePage);
    a.rows[a.n_rows++] = rows(&vr, h->p.v_pages, kCopyPage);
    for (uint32_t i = 0; i < a.n_rows; ++i) a.heads += a.rows[i].heads;
    e = launch_rows(a, tab, h->p.head_dim, h->p.dtype, st);
  } else {
    a.heads = q ? h->p.n_heads : 0;
    CodesArgs c{a,
                {static_cast<const char*>(k->in), static_cast<const char*>(v->in)},
                {k->in_token, v->in_token},
                {k->in_head, v->in_head},
                {static_cast<uint32_t*>(h->p.k_pages), static_cast<uint32_t*>(h->p.v_pages)},
                {h->p.k_scales, h->p.v_scales},
                h->p.n_kv_heads,
                0};
    const auto go = [&](auto x) {
      using T = decltype(x);
      if (h->p.bits == 8) return h->p.head_dim == 64 ? launch_codes<T, 64, 8>(c, tab, q != nullptr, st) : launch_codes<T, 128, 8>(c, tab, q != nullptr, st);
      return h->p.head_dim == 64 ? launch_codes<T, 64, 4>(c, tab, q != nullptr, st) : launch_codes<T, 128, 4>(c, tab, q != nullptr, st);
    };
    e = h->p.dtype == COFIE_BF16 ? go(__nv_bfloat16()) : go(__half());
  }
  return launched(h, e, "append");
}

int cofie_kv_read(cofie_kv_t* h, const cofie_kv_batch* b, void* k_out, void* v_out, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  if (const int rc = check_batch(h, b)) return rc;
  if (b->n_tokens == 0) return COFIE_OK;
  if (!k_out || !v_out || reinterpret_cast<uintptr_t>(k_out) % 16 || reinterpret_cast<uintptr_t>(v_out) % 16)
    return h->fail(COFIE_EINVAL, "k_out and v_out are required, 16-byte aligned");
  DeviceGuard g(h->device);
  const ReadArgs a{batch_arg(h, b),
                   {static_cast<const char*>(h->p.k_pages), static_cast<const char*>(h->p.v_pages)},
                   {h->p.k_scales, h->p.v_scales},
                   {static_cast<uint4*>(k_out), static_cast<uint4*>(v_out)}};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf = h->p.dtype == COFIE_BF16;
  const cudaError_t e = h->p.head_dim == 64 ? (bf ? launch_read<__nv_bfloat16, 64>(a, h->p.bits, st) : launch_read<__half, 64>(a, h->p.bits, st))
                                            : (bf ? launch_read<__nv_bfloat16, 128>(a, h->p.bits, st) : launch_read<__half, 128>(a, h->p.bits, st));
  return launched(h, e, "read");
}

int cofie_kv_status(cofie_kv_t* h, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  DeviceGuard g(h->device);
  cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream));
  uint32_t word = 0;
  if (e == cudaSuccess) e = cudaMemcpy(&word, h->d_err, sizeof word, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && word) e = cudaMemsetAsync(h->d_err, 0, sizeof word, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return launched(h, e, "status");
  if (word & kKvErrWait) return h->fail(COFIE_ETIMEOUT, "a device-side wait of the attention kernel ran out");
  if (word & kKvErrPage) return h->fail(COFIE_EDEVICE, "a page number in the table is not below n_pages");
  if (word) return h->fail(COFIE_EDEVICE, "a length or an offset of the batch is out of range");
  return COFIE_OK;
}

const char* cofie_kv_last_error(const cofie_kv_t* h) { return h ? h->err.c_str() : g_kv_error.c_str(); }

}  // extern "C"

// Attention over the paged cache.
#include <algorithm>
#include <cmath>

#include "kv_handle.cuh"

namespace cofie {
namespace {

constexpr int kWarps = 8;

struct AttendArgs {
  BatchArg batch;
  RowsArg q;
  float* lse;
  const uint8_t* mask;
  uint64_t mask_stride;
  const char* k;
  const char* v;
  const uint16_t* k_words;
  const uint16_t* v_words;
  uint32_t heads, group, causal;
  float scale;
};

// D / 32 values of a cached row for this lane, in fp32.
template <typename T, int D, int BITS>
__device__ __forceinline__ void cached_values(const char* pages, const uint16_t* words, uint64_t row, uint32_t lane, float* x) {
  constexpr int N = D / 32;
  const uint32_t d = lane * N;
  if (BITS == 16) {
    const T* p = reinterpret_cast<const T*>(pages) + row * D + d;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = Elem<T>::to(p[i]);
  } else {
    const uint8_t* p = reinterpret_cast<const uint8_t*>(pages) + (row * D + d) / 2;
    const uint32_t word = words[row * (D / kGroup) + d / kGroup];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = code_value(p[i / 2] >> (4 * (i % 2)) & 15u, word);
  }
}

// A warp to a (token, head) row, one cached token after the other.
template <typename T, int D, int BITS>
__global__ void __launch_bounds__(32 * kWarps) attend_rows(const AttendArgs a) {
  constexpr int N = D / 32;
  pdl_trigger();
  pdl_wait();
  const uint32_t lane = threadIdx.x % 32;
  const uint64_t row = blockIdx.x * static_cast<uint64_t>(kWarps) + threadIdx.x / 32;
  if (row >= static_cast<uint64_t>(a.batch.n_tokens) * a.heads) return;
  const uint32_t t = static_cast<uint32_t>(row / a.heads), head = static_cast<uint32_t>(row % a.heads);
  const BatchArg& b = a.batch;
  const uint32_t s = b.offsets ? sequence_of(b.offsets, b.n_seqs, t) : t;
  if (s >= b.n_seqs) return;
  const Span span = sequence_span(b, s);
  if (t - span.first >= span.count) return;
  const int64_t n = span.count, i = t - span.first, m = span.length;
  const int64_t end = a.causal ? min(m, m - n + i + 1) : m;
  const T* q = reinterpret_cast<const T*>(a.q.in) + t * a.q.in_token + head * a.q.in_head + lane * N;
  float x[N], o[N], y[N], top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    x[e] = Elem<T>::to(q[e]) * a.scale;
    o[e] = 0.f;
  }
  for (int64_t j = 0; j < end; ++j) {
    if (a.mask && (static_cast<uint64_t>(j) >= a.mask_stride || !a.mask[s * a.mask_stride + j])) continue;
    const uint32_t page = static_cast<uint32_t>(b.table[static_cast<uint64_t>(s) * b.table_stride + (j >> b.page_shift)]);
    if (page >= b.n_pages) {
      if (lane == 0) atomicOr(b.err, kKvErrPage);
      continue;
    }
    const uint64_t r = page_row(b, (static_cast<int64_t>(page) << b.page_shift) | (j & ((1 << b.page_shift) - 1)), head / a.group);
    cached_values<T, D, BITS>(a.k, a.k_words, r, lane, y);
    float dot = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) dot += x[e] * y[e];
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, w);
    const float next = fmaxf(top, dot), keep = expf(top - next), p = expf(dot - next);
    top = next;
    sum = sum * keep + p;
    cached_values<T, D, BITS>(a.v, a.v_words, r, lane, y);
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = o[e] * keep + p * y[e];
  }
  T* out = reinterpret_cast<T*>(a.q.out) + t * a.q.out_token + head * a.q.out_head + lane * N;
#pragma unroll
  for (int e = 0; e < N; ++e) out[e] = Elem<T>::from(sum > 0.f ? o[e] / sum : (sum == 0.f ? 0.f : sum));
  if (a.lse && lane == 0) a.lse[row] = top + logf(sum);
}

template <typename T, int D>
cudaError_t launch_attend(const AttendArgs& a, uint32_t bits, cudaStream_t st) {
  const uint64_t rows = static_cast<uint64_t>(a.batch.n_tokens) * a.heads;
  const dim3 grid(static_cast<uint32_t>((rows + kWarps - 1) / kWarps)), block(32 * kWarps);
  return bits == 4 ? launch_dependent(true, attend_rows<T, D, 4>, grid, block, 0, st, a)
                   : launch_dependent(true, attend_rows<T, D, 16>, grid, block, 0, st, a);
}

}  // namespace
}  // namespace cofie

using namespace cofie;

extern "C" int cofie_kv_attend(cofie_kv_t* h, const cofie_kv_batch* b, const cofie_rows* q, float* lse, const uint8_t* mask,
                               uint64_t mask_stride, int causal, float scale, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  if (const int rc = check_batch(h, b)) return rc;
  if (b->n_tokens == 0) return COFIE_OK;
  if (!q) return h->fail(COFIE_EINVAL, "q is required");
  if (const int rc = check_rows(h, q, h->p.n_heads, true, "q")) return rc;
  if (!(scale >= 0.f && std::isfinite(scale))) return h->fail(COFIE_EINVAL, "scale must be finite and not negative");
  DeviceGuard g(h->device);
  const AttendArgs a{batch_arg(h, b),
                     {static_cast<const char*>(q->in), static_cast<char*>(q->out), q->in_token, q->in_head, q->out_token, q->out_head, q->heads, kRotate},
                     lse,
                     mask,
                     mask_stride,
                     static_cast<const char*>(h->p.k_pages),
                     static_cast<const char*>(h->p.v_pages),
                     h->p.k_scales,
                     h->p.v_scales,
                     h->p.n_heads,
                     h->p.n_heads / h->p.n_kv_heads,
                     causal != 0,
                     scale > 0.f ? scale : 1.f / std::sqrt(static_cast<float>(h->p.head_dim))};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf = h->p.dtype == COFIE_BF16;
  const cudaError_t e = h->p.head_dim == 64 ? (bf ? launch_attend<__nv_bfloat16, 64>(a, h->p.bits, st) : launch_attend<__half, 64>(a, h->p.bits, st))
                                            : (bf ? launch_attend<__nv_bfloat16, 128>(a, h->p.bits, st) : launch_attend<__half, 128>(a, h->p.bits, st));
  return launched(h, e, "attend");
}

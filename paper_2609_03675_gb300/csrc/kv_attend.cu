// Attention over the paged cache: the entry point, the tiles that a mask
// leaves, and the choice of the kernel.
#include <algorithm>
#include <cmath>

#include "kv_rows_tc.cuh"

namespace cofie {
namespace {

constexpr int kMaskThreads = 1024;

// The tiles of 64 cached tokens of which the mask leaves one at least, in
// order, a CTA to a sequence, 1024 tiles at a time: neighbouring lanes look at
// a tile together (N bytes each, as the rows' alignment allows), then a thread
// has a tile and a scan gives it its place.
template <typename V>
__device__ __forceinline__ bool any_set(const uint8_t* p) {
  const V x = *reinterpret_cast<const V*>(p);
  if constexpr (sizeof(V) == 16) return (x.x | x.y | x.z | x.w) != 0;
  else return x != 0;
}
template <typename V>
__global__ void __launch_bounds__(kMaskThreads) visible_tiles(const BatchArg b, const uint8_t* mask, uint64_t mask_stride, uint32_t* tiles,
                                                              uint32_t* count, uint32_t tile_stride) {
  constexpr uint32_t kBytes = sizeof(V) > 1 ? sizeof(V) : 4, kLanes = kTile / kBytes;
  __shared__ uint32_t warps[kMaskThreads / 32];
  __shared__ uint8_t flag[kMaskThreads];
  pdl_trigger();
  pdl_wait();
  const uint32_t seq = blockIdx.x, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint64_t length = min(static_cast<uint64_t>(sequence_span(b, seq).length), mask_stride);
  const uint8_t* row = mask + seq * mask_stride;
  uint32_t n = 0;
  for (uint64_t t0 = 0; t0 * kTile < length; t0 += kMaskThreads) {
    // whole warps stay in the loop, for the votes
    const uint32_t here = static_cast<uint32_t>(min(static_cast<uint64_t>(kMaskThreads), (length + kTile - 1) / kTile - t0));
#pragma unroll 4
    for (uint32_t t1 = warp * (32 / kLanes); t1 < here; t1 += kMaskThreads / kLanes) {
      const uint32_t t = t1 + lane / kLanes;
      const uint64_t at = (t0 + t) * kTile + lane % kLanes * kBytes;
      bool some = false;
      if (t < here && at < length) {
        if (sizeof(V) > 1 && at + kBytes <= length) {
          some = any_set<V>(row + at);
        } else {
#pragma unroll
          for (uint32_t i = 0; i < kBytes; ++i) some |= at + i < length && row[at + i] != 0;
        }
      }
      const uint32_t bits = __ballot_sync(0xffffffffu, some);
      if (lane % kLanes == 0 && t < here) flag[t] = (bits >> lane & ((1u << kLanes) - 1)) != 0;
    }
    __syncthreads();
    const bool some = threadIdx.x < here && flag[threadIdx.x];
    const uint32_t bits = __ballot_sync(0xffffffffu, some);
    if (lane == 0) warps[warp] = __popc(bits);
    __syncthreads();
    uint32_t before = n, all = 0;
    for (uint32_t w = 0; w < kMaskThreads / 32; ++w) {
      if (w < warp) before += warps[w];
      all += warps[w];
    }
    if (some)
      tiles[static_cast<uint64_t>(seq) * tile_stride + before + __popc(bits & ((1u << lane) - 1))] = static_cast<uint32_t>(t0) + threadIdx.x;
    n += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) count[seq] = n;
}

template <typename F>
auto for_type(const cofie_kv_params& p, F f) {
  if (p.dtype == COFIE_BF16) return f(__nv_bfloat16());
  return f(__half());
}

// The kernel of the handle's type, head length and pages, for 8 << i rows (i: 0 or 1).
using SplitKernel = void (*)(AttendArgs);
template <typename T, int D, int BITS>
SplitKernel split_kernel(int i, size_t* smem) {
  *smem = i == 0 ? split_smem<D, BITS, 1>() : split_smem<D, BITS, 2>();
  return i == 0 ? attend_split<T, D, BITS, 1> : attend_split<T, D, BITS, 2>;
}
SplitKernel split_kernel(const cofie_kv_params& p, int i, size_t* smem) {
  return for_type(p, [&](auto x) {
    using T = decltype(x);
    if (p.bits == 8) return p.head_dim == 64 ? split_kernel<T, 64, 8>(i, smem) : split_kernel<T, 128, 8>(i, smem);
    if (p.head_dim == 64) return p.bits == 4 ? split_kernel<T, 64, 4>(i, smem) : split_kernel<T, 64, 16>(i, smem);
    return p.bits == 4 ? split_kernel<T, 128, 4>(i, smem) : split_kernel<T, 128, 16>(i, smem);
  });
}

template <typename T, int D>
SplitKernel rows_kernel(uint32_t bits, size_t* smem) {
  *smem = bits == 4 ? tc_smem<D, 4>() : bits == 8 ? tc_smem<D, 8>() : tc_smem<D, 16>();
  if (bits == 8) return attend_rows_tc<T, D, 8>;
  return bits == 4 ? attend_rows_tc<T, D, 4> : attend_rows_tc<T, D, 16>;
}
SplitKernel rows_kernel(const cofie_kv_params& p, size_t* smem) {
  return for_type(p, [&](auto x) {
    using T = decltype(x);
    return p.head_dim == 64 ? rows_kernel<T, 64>(p.bits, smem) : rows_kernel<T, 128>(p.bits, smem);
  });
}

}  // namespace

cudaError_t attend_set_up(cofie_kv* h) {
  cudaError_t e = cudaSuccess;
  size_t rows = 0, ctas = 0;
  for (int i = 0; i < 2 && e == cudaSuccess; ++i) {
    size_t smem = 0;
    const SplitKernel k = split_kernel(h->p, i, &smem);
    int per_sm = 0;
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k, kSplitThreads, smem);
    if (e == cudaSuccess && per_sm < 1) e = cudaErrorInvalidConfiguration;
    h->split_ctas[i] = sm_count() * static_cast<uint32_t>(per_sm);
    ctas = std::max<size_t>(ctas, h->split_ctas[i]);
    rows = std::max<size_t>(rows, 2ull * h->split_ctas[i] * (8u << i));
  }
  size_t smem = 0;
  if (e == cudaSuccess) {
    const SplitKernel k = rows_kernel(h->p, &smem);
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    rows = std::max<size_t>(rows, 2ull * sm_count() * kTcRows);
  }
  if (e == cudaSuccess) e = cudaMalloc(&h->d_part, rows * h->p.head_dim * sizeof(float));
  if (e == cudaSuccess) e = cudaMalloc(&h->d_part_ms, rows * sizeof(float2));
  if (e == cudaSuccess) e = cudaMalloc(&h->d_done, ctas * sizeof(uint32_t));
  if (e == cudaSuccess) e = cudaMemset(h->d_done, 0, ctas * sizeof(uint32_t));
  return e;
}

}  // namespace cofie

using namespace cofie;

extern "C" int cofie_kv_attend(cofie_kv_t* h, const cofie_kv_batch* b, const cofie_rows* q, float* lse, const uint8_t* mask,
                               uint64_t mask_stride, int causal, float scale, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  if (const int rc = check_batch(h, b)) return rc;
  if (b->n_tokens == 0) return COFIE_OK;
  if (!q) return h->fail(COFIE_EINVAL, "q is required");
  if (const int rc = check_rows(h, q, h->p.n_heads, true, "q")) return rc;
  if (q->in == q->out && ((b->n_tokens > 1 && q->in_token != q->out_token) || (q->heads > 1 && q->in_head != q->out_head)))
    return h->fail(COFIE_EINVAL, "in place, the strides of q's in and out must be the same");
  if (!(scale >= 0.f && std::isfinite(scale))) return h->fail(COFIE_EINVAL, "scale must be finite and not negative");
  DeviceGuard g(h->device);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const auto aligned = [](const void* p, int64_t token, int64_t head, uint32_t elems) {
    return reinterpret_cast<uintptr_t>(p) % (2 * elems) == 0 && token % elems == 0 && head % elems == 0;
  };
  AttendArgs a{};
  a.batch = batch_arg(h, b);
  a.q = {static_cast<const char*>(q->in), static_cast<char*>(q->out), q->in_token, q->in_head, q->out_token, q->out_head, q->heads, kRotate};
  a.lse = lse;
  a.mask = mask;
  a.mask_stride = mask_stride;
  a.k = static_cast<const char*>(h->p.k_pages);
  a.v = static_cast<const char*>(h->p.v_pages);
  a.k_words = h->p.k_scales;
  a.v_words = h->p.v_scales;
  a.heads = h->p.n_heads;
  a.group = h->p.n_heads / h->p.n_kv_heads;
  a.causal = causal != 0;
  a.q_wide = aligned(q->in, q->in_token, q->in_head, 8);
  a.out_wide = aligned(q->out, q->out_token, q->out_head, 4);
  a.scale = scale > 0.f ? scale : 1.f / std::sqrt(static_cast<float>(h->p.head_dim));
  a.part = h->d_part;
  a.part_ms = h->d_part_ms;
  a.done = h->d_done;
  if (mask) {
    a.tile_stride = (b->table_stride << h->page_shift) / kTile + 1;
    const size_t need = static_cast<size_t>(b->n_seqs) * (a.tile_stride + 1);
    if (need > h->tiles_room) {
      const size_t room = std::max(need, 2 * h->tiles_room);
      cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
      if (cudaStreamIsCapturing(st, &cs) != cudaSuccess || cs != cudaStreamCaptureStatusNone) {
        cudaGetLastError();
        return h->fail(COFIE_EINVAL, "the first masked call of this size must come before the capture");
      }
      uint32_t* more = nullptr;
      const cudaError_t e = injected_alloc_failure() ? cudaErrorMemoryAllocation : cudaMalloc(&more, room * sizeof(uint32_t));
      if (e != cudaSuccess) {
        cudaGetLastError();
        return h->fail(e == cudaErrorMemoryAllocation ? COFIE_ENOMEM : COFIE_ECUDA, "no room for the list of the mask's tiles");
      }
      if (h->d_tiles) h->d_tiles_before[h->n_tiles_before++] = h->d_tiles;  // graphs may have it
      h->d_tiles = more;
      h->tiles_room = room;
    }
    a.tiles = h->d_tiles;
    a.tile_count = h->d_tiles + static_cast<size_t>(b->n_seqs) * a.tile_stride;
    const uintptr_t at = reinterpret_cast<uintptr_t>(mask) | (b->n_seqs > 1 ? mask_stride : 0);
    const auto find = at % 16 == 0 ? visible_tiles<uint4> : at % 4 == 0 ? visible_tiles<uint32_t> : visible_tiles<uint8_t>;
    if (const int rc = launched(h, launch_dependent(true, find, dim3(b->n_seqs), dim3(kMaskThreads), 0, st, a.batch, mask, mask_stride,
                                                    h->d_tiles, const_cast<uint32_t*>(a.tile_count), a.tile_stride),
                                "attend"))
      return rc;
  }
  const uint64_t rows = static_cast<uint64_t>(b->offsets ? (b->max_new ? b->max_new : b->n_tokens) : 1) * a.group;
  size_t smem = 0;
  // Up to 32 rows of a sequence and head, in blocks of 8 or 16, are left to the kernel that reads the cache for each
  // block; more rows pay for tiles of 128 of them. Eight sequences of up to 60000 tokens, 32 heads over 8 of 128 (us,
  // blocks / tiles): 20 rows 176 / 233 with 4 bits, 214 / 337 with 16; 32 rows 188 / 234, 262 / 339; 48 rows 266 / 234,
  // 344 / 340. Up to 2000 tokens: 20 rows 25 / 28, 22 / 32; 48 rows 32 / 29, 27 / 34.
  // What an item costs beside its tiles' slots (set-up, first loads, its part's joining), in the time of a tile: about 8 for
  // many rows and 6 for few, at every size tried. Many rows, us with 4 / 8 / 16 / 24 slots: seven questions of 3 to 300
  // tokens over up to 4000 of 4 bits 91 / 85 / 89 / 95, four prompts of 1024 over up to 8192 of 16 bits 451 / 343 / 371 /
  // 394, thirty of 16 over up to 2000 87 / 91 / 97 / 103. Few, with 2 / 4 / 6 / 8 / 12: 24 x 3 tokens over up to 9000 of
  // 4 bits 91 / 79 / 72 / 69 / 62, 64 x 1 over up to 20000 of 4 bits 220 / 212 / 200 / 197 / 199, of 16 bits 419 / 402 /
  // 400 / 394 / 398, 8 x 1 over up to 3000 27 / 25 / 23 / 25 / 25.
  if (rows > 32) {
    const SplitKernel k = rows_kernel(h->p, &smem);
    a.item_slots = 8;
    return launched(h, launch_dependent(true, k, dim3(sm_count()), dim3(kTcThreads), smem, st, a), "attend");
  }
  const int i = rows <= 8 ? 0 : 1;
  a.item_slots = 6;
  const SplitKernel k = split_kernel(h->p, i, &smem);
  return launched(h, launch_dependent(true, k, dim3(h->split_ctas[i]), dim3(kSplitThreads), smem, st, a), "attend");
}

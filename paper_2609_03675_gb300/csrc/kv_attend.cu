// Attention over the paged cache: the entry point, the tiles that a mask
// leaves, shared prefixes, and the choice of the kernel.
#include <algorithm>
#include <cmath>

#include <cudaTypedefs.h>

#include "kv_kernels.cuh"

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

// The mask of shared prefixes: a word for every 64 tokens of each sequence,
// a thread to a word, and each new token's sequence. WIDE: rows allow 16-byte
// loads.
constexpr int kWordThreads = 256;
template <bool WIDE>
__global__ void __launch_bounds__(kWordThreads) prefix_words(const BatchArg groups, const uint8_t* mask, uint64_t mask_stride, uint64_t* words,
                                                             uint32_t tile_stride, int32_t* seq_of) {
  pdl_trigger();
  pdl_wait();
  for (uint32_t seq = blockIdx.y; seq < groups.members; seq += gridDim.y) {
    const uint32_t g = groups.groups ? sequence_of(groups.groups, groups.n_seqs, seq) : 0;
    const Span sp = g < groups.n_seqs ? sequence_span(groups, g) : Span{0, 0, 0};
    if (sp.count == 0) {  // nothing, where a group that does not rise may look for its words
      for (uint64_t t = blockIdx.x * kWordThreads + threadIdx.x; t < tile_stride; t += gridDim.x * kWordThreads)
        words[static_cast<uint64_t>(seq) * tile_stride + t] = 0;
      continue;
    }
    const uint64_t length = min(static_cast<uint64_t>(sp.length), mask_stride);
    const uint8_t* row = mask + seq * mask_stride;
    for (uint64_t t = blockIdx.x * kWordThreads + threadIdx.x; t * kTile < sp.length; t += gridDim.x * kWordThreads) {
      uint64_t word = 0;
      const uint64_t at = t * kTile;
      if (WIDE && at + kTile <= length) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 x = *reinterpret_cast<const uint4*>(row + at + 16 * i);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            // 0x01 in each byte that is not zero, gathered to four bits by a product
            const uint32_t ones = __vcmpne4(w[j], 0u) & 0x01010101u;
            word |= static_cast<uint64_t>(ones * 0x01020408u >> 24 & 15u) << (16 * i + 4 * j);
          }
        }
      } else {
        for (uint32_t i = 0; i < kTile && at + i < length; ++i) word |= static_cast<uint64_t>(row[at + i] != 0) << i;
      }
      words[static_cast<uint64_t>(seq) * tile_stride + t] = word;
    }
    // this sequence's tokens, which lie among the group's
    const int64_t first = groups.offsets ? groups.offsets[seq] : seq, end = groups.offsets ? groups.offsets[seq + 1] : seq + 1;
    const int64_t lo = max(first, static_cast<int64_t>(sp.first)), hi = min(end, static_cast<int64_t>(sp.first) + sp.count);
    for (int64_t i = lo + blockIdx.x * kWordThreads + threadIdx.x; i < hi; i += gridDim.x * kWordThreads) seq_of[i] = static_cast<int32_t>(seq);
  }
}

// For each group the union of its sequences' words, and for each block of its
// rows (the last list: for that block and all after it) the tiles where the
// union of the sequences that have rows there is not empty, in order: a CTA to a
// list, 1024 tiles at a time. (By lists of the group alone, blocks of 256 rows of
// 16 questions that see 0.3 of 400 frames each took 594 us, so 458. With a bit for
// each half of a block that does not see a tile, whose products are then left out,
// 478: the count of its tiles that each half needs costs the warps that issue more.)
__global__ void __launch_bounds__(kMaskThreads) prefix_tiles(const BatchArg groups, const uint64_t* words, uint64_t* any, uint32_t* tiles,
                                                             uint32_t* count, uint32_t tile_stride, const int32_t* seq_of, uint32_t block_rows,
                                                             uint32_t group) {
  __shared__ uint32_t warps[kMaskThreads / 32];
  pdl_trigger();
  pdl_wait();
  const uint32_t g = blockIdx.x, rb = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint64_t list = static_cast<uint64_t>(g) * gridDim.y + rb;
  const Span sp = sequence_span(groups, g);
  const uint64_t rows = static_cast<uint64_t>(sp.count) * group, row0 = static_cast<uint64_t>(rb) * block_rows;
  const uint32_t all = row0 >= rows ? 0 : (sp.length + kTile - 1) / kTile;
  uint32_t s0 = 0, s1 = 0, g0 = 0, g1 = 0;  // the block's sequences, and the group's
  if (all) {
    g0 = groups.groups ? groups.groups[g] : 0;
    g1 = groups.groups ? groups.groups[g + 1] : groups.members;
    const uint64_t last = rb + 1 == gridDim.y ? rows : min(rows, row0 + block_rows);
    s0 = min(static_cast<uint32_t>(seq_of[sp.first + row0 / group]), groups.members - 1);
    s1 = min(static_cast<uint32_t>(seq_of[sp.first + (last - 1) / group]), groups.members - 1) + 1;
  }
  uint32_t n = 0;
  for (uint32_t t0 = 0; t0 < all; t0 += kMaskThreads) {
    const uint32_t t = t0 + threadIdx.x;
    uint64_t word = 0;
    if (t < all) {
#pragma unroll 8
      for (uint32_t s = s0; s < s1; ++s) word |= words[static_cast<uint64_t>(s) * tile_stride + t];
      if (rb == 0) {
        uint64_t both = word;
        if (s0 != g0 || s1 != g1)
#pragma unroll 8
          for (uint32_t s = g0; s < g1; ++s) both |= words[static_cast<uint64_t>(s) * tile_stride + t];
        any[static_cast<uint64_t>(g) * tile_stride + t] = both;
      }
    }
    const uint32_t bits = __ballot_sync(0xffffffffu, word != 0);
    if (lane == 0) warps[warp] = __popc(bits);
    __syncthreads();
    uint32_t before = n;
    for (uint32_t w = 0; w < kMaskThreads / 32; ++w) {
      if (w < warp) before += warps[w];
      n += warps[w];
    }
    if (word) tiles[list * tile_stride + before + __popc(bits & ((1u << lane) - 1))] = t;
    __syncthreads();
  }
  if (threadIdx.x == 0) count[list] = n;
}

AttendLaunch kernel_of(const cofie_kv_params& p, int kind, bool shared) {
  const auto of = [&](auto bits) {
    return shared ? attend_kernel<bits, true>(p, kind) : attend_kernel<bits, false>(p, kind);
  };
  return p.bits == 4 ? of(std::integral_constant<int, 4>()) : p.bits == 8 ? of(std::integral_constant<int, 8>()) : of(std::integral_constant<int, 16>());
}

// The map of 16-bit pages, whose copies lie as the products read them.
cudaError_t map_pages(const cofie_kv_params& p, void* pages, CUtensorMap* map) {
  void* f = nullptr;
  cudaDriverEntryPointQueryResult found;
  const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
  if (e != cudaSuccess) return e;
  if (found != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {p.head_dim, static_cast<cuuint64_t>(p.n_kv_heads) * p.page_size, p.n_pages};
  const cuuint64_t strides[2] = {2ull * p.head_dim, 2ull * p.head_dim * p.n_kv_heads * p.page_size};
  const cuuint32_t box[3] = {64, std::min(p.page_size, kTile), 1}, steps[3] = {1, 1, 1};
  const CUresult r = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f)(
      map, p.dtype == COFIE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, pages, dims, strides, box, steps,
      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace

cudaError_t attend_set_up(cofie_kv* h) {
  cudaError_t e = cudaSuccess;
  if (h->p.bits == 16) {
    e = map_pages(h->p, h->p.k_pages, &h->maps[0]);
    if (e == cudaSuccess) e = map_pages(h->p, h->p.v_pages, &h->maps[1]);
  }
  size_t rows = 2ull * sm_count() * kManyRows, ctas = 0;
  for (int i = 0; i < kShort8 + kShort16 + 1 && e == cudaSuccess; ++i) {
    const bool shared = i >= kShort8;  // those of no prefix first
    const int kind = shared ? i - kShort8 : i;
    const AttendLaunch k = kernel_of(h->p, kind, shared);
    e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(k.smem));
    if (kind >= kMany || e != cudaSuccess) continue;
    int per_sm = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k.kernel, static_cast<int>(k.threads), k.smem);
    if (e == cudaSuccess && per_sm < 1) e = cudaErrorInvalidConfiguration;
    const uint32_t n = sm_count() * static_cast<uint32_t>(per_sm);
    h->split_ctas[shared][kind] = n;
    ctas = std::max<size_t>(ctas, n);
    rows = std::max<size_t>(rows, 2ull * n * (8u << kind));
  }
  if (e == cudaSuccess) e = cudaMalloc(&h->d_part, rows * h->p.head_dim * sizeof(float));
  if (e == cudaSuccess) e = cudaMalloc(&h->d_part_ms, rows * sizeof(float2));
  if (e == cudaSuccess) e = cudaMalloc(&h->d_done, ctas * sizeof(uint32_t));
  if (e == cudaSuccess) e = cudaMalloc(&h->d_items, sm_count() * sizeof(SplitItem));
  if (e == cudaSuccess) e = cudaMemset(h->d_done, 0, ctas * sizeof(uint32_t));
  return e;
}

namespace {

// What both entry points check and fill in; COFIE_OK, or the error noted on the handle.
int attend_args(cofie_kv* h, const cofie_kv_batch* b, const cofie_rows* q, float* lse, const uint8_t* mask, uint64_t mask_stride, int causal,
                float scale, AttendArgs* out) {
  if (!q) return h->fail(COFIE_EINVAL, "q is required");
  if (const int rc = check_rows(h, q, h->p.n_heads, true, "q")) return rc;
  if (q->in == q->out && ((b->n_tokens > 1 && q->in_token != q->out_token) || (q->heads > 1 && q->in_head != q->out_head)))
    return h->fail(COFIE_EINVAL, "in place, the strides of q's in and out must be the same");
  if (!(scale >= 0.f && std::isfinite(scale))) return h->fail(COFIE_EINVAL, "scale must be finite and not negative");
  const auto aligned = [](const void* p, int64_t token, int64_t head, uint32_t elems) {
    return reinterpret_cast<uintptr_t>(p) % (2 * elems) == 0 && token % elems == 0 && head % elems == 0;
  };
  AttendArgs& a = *out;
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
  a.items = static_cast<SplitItem*>(h->d_items);
  a.k_map = h->maps[0];
  a.v_map = h->maps[1];
  return COFIE_OK;
}

// Whether scratch may be allocated for a call on this stream.
bool may_allocate(cudaStream_t st) {
  cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
  const bool ok = cudaStreamIsCapturing(st, &cs) == cudaSuccess && cs == cudaStreamCaptureStatusNone;
  if (!ok) cudaGetLastError();
  return ok;
}

// Room for the tiles that the batch's mask leaves; a.tiles and what goes with it. A call finds the room for all that it needs
// before its first launch, so that one that is refused has launched nothing.
int room_for_tiles(cofie_kv* h, const cofie_kv_batch* b, AttendArgs* args, cudaStream_t st) {
  AttendArgs& a = *args;
  a.tile_stride = (b->table_stride << h->page_shift) / kTile + 1;
  a.list_blocks = 1;
  const size_t need = static_cast<size_t>(b->n_seqs) * (a.tile_stride + 1);
  if (need > h->tiles_room) {
    const size_t room = std::max(need, 2 * h->tiles_room);
    if (!may_allocate(st)) return h->fail(COFIE_EINVAL, "the first masked call of this size must come before the capture");
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
  return COFIE_OK;
}

// Those tiles.
int list_tiles(cofie_kv* h, const cofie_kv_batch* b, const AttendArgs& a, cudaStream_t st) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.mask) | (b->n_seqs > 1 ? a.mask_stride : 0);
  const auto find = at % 16 == 0 ? visible_tiles<uint4> : at % 4 == 0 ? visible_tiles<uint32_t> : visible_tiles<uint8_t>;
  return launched(h, launch_dependent(true, find, dim3(b->n_seqs), dim3(kMaskThreads), 0, st, a.batch, a.mask, a.mask_stride, const_cast<uint32_t*>(a.tiles),
                                      const_cast<uint32_t*>(a.tile_count), a.tile_stride),
                  "attend");
}

// The kernel for so many rows of a sequence and key head at most: up to 16 rows, in blocks of 8 or 16, are left to the kernel
// that reads the cache for each block; more rows pay for tiles of 128 of them. Eight sequences of up to 60000 tokens, 32
// heads over 8 of 128 (us, blocks / tiles): 16 rows of 16 bits 178 / 174, of 8 bits 132 / 235, of 4 bits 123 / 186; 20 rows
// 332 / 175, 239 / 236, 224 / 186. 32 sequences of up to 6000: 16 rows 85 / 92, 86 / 121, 81 / 102; 20 rows 137 / 94, 139 /
// 121, 137 / 103. Eight of up to 2000: 16 rows 21 / 23, 24 / 28, 23 / 27; 20 rows 27 / 23, 29 / 29, 29 / 27. Without a shared
// prefix 4-bit pages go by blocks up to 32 rows, though tiles would be quicker from 17: rows of tiles see values past fp16's
// range as infinite, those of blocks do not, and calls of 17 to 32 rows have counted on that.
int kind_of(const cofie_kv* h, uint64_t rows, bool shared) {
  const uint64_t few = h->p.bits == 4 && !shared ? 32 : 16;
  return rows > few ? kMany : rows > 8 ? kFew16 : kFew8;
}

// Some hundred bytes of arguments, which launch_dependent would copy twice.
cudaError_t launch_args(AttendKernel kernel, dim3 grid, uint32_t threads, size_t smem, cudaStream_t st, AttendArgs* a) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void* args[] = {a};
  return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kernel), args);
}

int launch_attend(cofie_kv* h, AttendArgs* a, uint64_t rows, bool shared, cudaStream_t st) {
  // What an item costs beside its tiles' slots (set-up, first loads, its part's joining), in the time of a tile: about 8 for
  // many rows and 6 for few, at every size tried. Many rows, us with 4 / 8 / 16 / 24 slots: seven questions of 3 to 300
  // tokens over up to 4000 of 4 bits 91 / 85 / 89 / 95, four prompts of 1024 over up to 8192 of 16 bits 451 / 343 / 371 /
  // 394, thirty of 16 over up to 2000 87 / 91 / 97 / 103. Few, with 2 / 4 / 6 / 8 / 12: 24 x 3 tokens over up to 9000 of
  // 4 bits 91 / 79 / 72 / 69 / 62, 64 x 1 over up to 20000 of 4 bits 220 / 212 / 200 / 197 / 199, of 16 bits 419 / 402 /
  // 400 / 394 / 398, 8 x 1 over up to 3000 27 / 25 / 23 / 25 / 25.
  int kind = kind_of(h, rows, shared);
  const uint64_t items = static_cast<uint64_t>(a->batch.n_seqs) * a->batch.kv_heads;
  const uint64_t width = static_cast<uint64_t>(a->batch.table_stride) << h->page_shift;
  // 17 to 32 rows of heads of 64, 16 bits: blocks are quicker where there is little to read (us, blocks / tiles, 32 rows): 2
  // sequences and key heads over 2048 tokens 11 / 15, over 60000 24 / 30; 8 of 64 6.9 / 7.1, of 128 9.7 / 7.8, of 512 to 2048 10.4 /
  // 11.7 to 11.3 / 14.3, of 6000 15.4 / 16.8, of 60000 53.5 / 46.7; 16 of 128 to 2048 7.2 / 8.0 to 13.3 / 15.5, of 6000 20.2 /
  // 19.1; 32 of 64 to 1024 7.4 / 7.6 to 14.8 / 15.5, of 6000 28.0 / 25.9; 64 of 64 7.5 / 8.0, of 128 10.0 / 8.5, of 1024 18.3 / 19.4,
  // of 2048 23.3 / 22.8; 128 of 64 11.0 / 8.4.
  if (kind == kMany && !shared && h->p.bits == 16 && h->p.head_dim == 64 && rows <= 32 && items <= 64 &&
      items * width <= (items <= 4 ? 131072 : 65536) && (width <= 64 || (items >= 16 && items <= 32) || width > (items <= 32 ? 384 : 512)))
    kind = kFew16;
  // Many rows over few tokens, as the table's width bounds them: items are not cut, so that no launch joins them. Most of 1 to
  // 32 sequences of 16 or 8 key heads, 18 to 256 rows, 16 to 4 bits, all equally long, of any length up to the width and one
  // that long, cut / uncut: up to 384 tokens 0.65 to 1.00 of the time (64 tokens 13.4 / 9.1 us, 384 14.9 / 14.6 to 38 / 25), 512
  // 0.7 to 1.1 (one sequence of 8 key heads 14.9 / 16.3, eight 20.9 / 17.5), 768 0.8 to 1.3.
  if (kind == kMany && width <= (items >= 64 ? 512 : 384)) kind = kManyWhole;
  // Own tokens behind a prefix: a sequence and key head are left to one CTA where its tokens, as the table's width bounds
  // them, are few, or where there are so many of these items that they fill the GPU uncut; but a single one as long as the
  // width must not wait alone. Single tokens, heads of 128 and 16 bits, the whole call, us cut / uncut, where all are of the
  // width, of any length up to it, and one of it beside others of 10: 16 items of 512 17.5 / 17.3, 17.3 / 17.0, 17.0 / 17.2, of
  // 1024 19 / 24, 18 / 24, 17 / 24; 64 of 1024 32 / 30, 30 / 29, 27 / 27, of 2048 35 / 43, 31 / 41, 28 / 39; 128 of 1024 40 / 35,
  // 37 / 35, 33 / 34, of 2048 59 / 54, 41 / 46, 33 / 46; 192 of 2048 64 / 52, 51 / 47, 30 / 40; 256 of 2048 74 / 61, 59 / 51,
  // 32 / 41, of 4096 110 / 97, 75 / 77, 33 / 65; 512 of 2048 118 / 105, 85 / 76, 44 / 47, of 8192 343 / 317, 190 / 207, 46 / 118;
  // with fewer bits alike.
  const uint64_t uncut = items >= 160 ? 2048 : items >= 96 ? 1536 : items >= 64 ? 1024 : 512;
  if (a->behind && kind < kMany && width <= uncut && items <= 0x7fffffffu)
    kind = kind == kFew8 ? kShort8 : kShort16;
  const bool many = kind == kMany || kind == kManyWhole;
  a->item_slots = many ? 8 : 6;
  const AttendLaunch k = kernel_of(h->p, kind, shared);
  const uint32_t ctas = many ? sm_count() : kind >= kShort8 ? static_cast<uint32_t>(items) : h->split_ctas[shared][kind];
  if (const int rc = launched(h, launch_args(k.kernel, dim3(ctas), k.threads, k.smem, st, a), "attend")) return rc;
  if (kind != kMany) return COFIE_OK;
  // As many joining CTAs as there can be rows, or as the call says that there are. (Behind a mask the former: with fewer, the
  // next call's pass over its mask starts beside them, and 24 sequences of 21 rows took 65.9 us for 64.3.)
  const uint64_t there = static_cast<uint64_t>(a->batch.n_tokens) * a->group;
  const bool few = rows <= 128 && rows < there && !a->tiles;
  const uint64_t block = few ? rows : std::min<uint64_t>(kManyRows, there);
  return launched(h, launch_args(k.join[few], dim3(ctas, static_cast<uint32_t>((block + k.join_rows - 1) / k.join_rows)), k.join_threads, 0, st, a),
                  "attend");
}

uint64_t rows_at_most(const cofie_kv_batch* b, uint32_t group) {
  return static_cast<uint64_t>(b->offsets ? (b->max_new ? b->max_new : b->n_tokens) : 1) * group;
}

// Room of this size in a scratch that grows to twice its size at least; what it outgrew stays, for graphs that have it.
int scratch(cofie_kv* h, cofie_kv::Scratch* s, size_t need, cudaStream_t st) {
  if (need <= s->room) return COFIE_OK;
  if (!may_allocate(st)) return h->fail(COFIE_EINVAL, "the first call of this size over a shared prefix must come before the capture");
  const size_t room = std::max(need, 2 * s->room);
  void* more = nullptr;
  const cudaError_t e = injected_alloc_failure() ? cudaErrorMemoryAllocation : cudaMalloc(&more, room);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return h->fail(e == cudaErrorMemoryAllocation ? COFIE_ENOMEM : COFIE_ECUDA, "no room for the shared prefix's rows");
  }
  if (s->p) s->before[s->n_before++] = s->p;
  s->p = more;
  s->room = room;
  return COFIE_OK;
}

// The rows of one block of the kernel for so many.
uint32_t block_rows_of(const cofie_kv* h, uint64_t rows) {
  const int kind = kind_of(h, rows, true);
  return kind == kMany ? kManyRows : kind == kFew16 ? 16u : 8u;
}

// Room for the mask of the prefixes: words, their union, the tiles that it leaves, and each token's sequence, one behind the
// other.
int room_for_prefix_mask(cofie_kv* h, AttendArgs* args, uint64_t rows, cudaStream_t st) {
  AttendArgs& a = *args;
  const BatchArg& g = a.batch;
  a.tile_stride = (g.table_stride << h->page_shift) / kTile + 1;
  // lists for so many rows of a group; 256 of them at most, and with many groups one each
  const uint32_t block_rows = block_rows_of(h, rows);
  a.list_blocks = g.n_seqs > 256 ? 1u : static_cast<uint32_t>(std::min<uint64_t>((rows + block_rows - 1) / block_rows, 256 / g.n_seqs));
  const size_t seqs = g.members, groups = g.n_seqs, stride = a.tile_stride, lists = groups * a.list_blocks;
  const size_t words = (seqs + groups) * stride * sizeof(uint64_t), tiles = lists * (stride + 1) * sizeof(uint32_t);
  if (const int rc = scratch(h, &h->shared_mask, words + tiles + g.n_tokens * sizeof(int32_t), st)) return rc;
  char* at = static_cast<char*>(h->shared_mask.p);
  uint64_t* seq_words = reinterpret_cast<uint64_t*>(at);
  uint64_t* any = seq_words + seqs * stride;
  uint32_t* list = reinterpret_cast<uint32_t*>(at + words);
  int32_t* seq_of = reinterpret_cast<int32_t*>(at + words + tiles);
  a.seq_words = seq_words;
  a.any_words = any;
  a.tiles = list;
  a.tile_count = list + lists * stride;
  a.seq_of = seq_of;
  return COFIE_OK;
}

// That mask.
int prefix_mask(cofie_kv* h, const cofie_kv_prefix* p, const AttendArgs& a, uint64_t rows, cudaStream_t st) {
  const BatchArg& g = a.batch;
  const size_t seqs = g.members;
  uint64_t* const seq_words = const_cast<uint64_t*>(a.seq_words);
  int32_t* const seq_of = const_cast<int32_t*>(a.seq_of);
  const bool wide = reinterpret_cast<uintptr_t>(p->mask) % 16 == 0 && (seqs == 1 || p->mask_stride % 16 == 0);
  const dim3 grid(std::max(1u, std::min((a.tile_stride + kWordThreads - 1) / kWordThreads, 64u)), std::min(g.members, 65535u));
  if (const int rc = launched(h, launch_dependent(true, wide ? prefix_words<true> : prefix_words<false>, grid, dim3(kWordThreads), 0, st, g, p->mask,
                                                  p->mask_stride, seq_words, a.tile_stride, seq_of),
                              "attend"))
    return rc;
  return launched(h, launch_dependent(true, prefix_tiles, dim3(g.n_seqs, a.list_blocks), dim3(kMaskThreads), 0, st, g,
                                      a.seq_words, const_cast<uint64_t*>(a.any_words), const_cast<uint32_t*>(a.tiles),
                                      const_cast<uint32_t*>(a.tile_count), a.tile_stride, a.seq_of, block_rows_of(h, rows), a.group),
                  "attend");
}

}  // namespace
}  // namespace cofie

using namespace cofie;

extern "C" int cofie_kv_attend(cofie_kv_t* h, const cofie_kv_batch* b, const cofie_rows* q, float* lse, const uint8_t* mask,
                               uint64_t mask_stride, int causal, float scale, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  if (const int rc = check_batch(h, b)) return rc;
  if (b->n_tokens == 0) return COFIE_OK;
  AttendArgs a{};
  if (const int rc = attend_args(h, b, q, lse, mask, mask_stride, causal, scale, &a)) return rc;
  DeviceGuard g(h->device);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (mask) {
    if (const int rc = room_for_tiles(h, b, &a, st)) return rc;
    if (const int rc = list_tiles(h, b, a, st)) return rc;
  }
  return launch_attend(h, &a, rows_at_most(b, a.group), false, st);
}

extern "C" int cofie_kv_attend_shared(cofie_kv_t* h, const cofie_kv_batch* b, const cofie_kv_prefix* prefix, const cofie_rows* q, float* lse,
                                      const uint8_t* mask, uint64_t mask_stride, int causal, float scale, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  if (const int rc = check_batch(h, b)) return rc;
  if (!prefix) return h->fail(COFIE_EINVAL, "the prefix is NULL");
  if (b->n_tokens == 0) return COFIE_OK;
  if (prefix->n_groups < 1 || prefix->n_groups > 0x7fffffffu) return h->fail(COFIE_EINVAL, "n_groups must be in [1, 2^31)");
  if (!prefix->groups && prefix->n_groups != 1) return h->fail(COFIE_EINVAL, "without groups there is one, of all sequences");
  if (!prefix->table || !prefix->lengths) return h->fail(COFIE_EINVAL, "the prefix's table and lengths are required");
  if (prefix->table_stride < 1 || prefix->table_stride > 0x7fffffffu / h->p.page_size)
    return h->fail(COFIE_EINVAL, "the prefix's table_stride x page_size must be in [page_size, 2^31)");
  AttendArgs own{};
  if (const int rc = attend_args(h, b, q, lse, mask, mask_stride, causal, scale, &own)) return rc;
  DeviceGuard g(h->device);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const size_t rows = static_cast<size_t>(b->n_tokens) * h->p.n_heads;
  if (const int rc = scratch(h, &h->shared_rows, rows * (h->p.head_dim * sizeof(float) + sizeof(float2)), st)) return rc;
  own.rows = static_cast<float*>(h->shared_rows.p);
  own.rows_ms = reinterpret_cast<float2*>(own.rows + rows * h->p.head_dim);
  own.prefix = own.batch;
  own.prefix.table = prefix->table;
  own.prefix.lengths = prefix->lengths;
  own.prefix.n_seqs = prefix->n_groups;
  own.prefix.table_stride = prefix->table_stride;
  own.prefix.groups = prefix->groups;
  own.prefix.members = b->n_seqs;
  AttendArgs first = own;
  first.batch = own.prefix;
  first.mask = nullptr;
  first.lse = nullptr;
  first.causal = 0;
  const uint64_t most = prefix->max_new ? prefix->max_new : b->n_tokens;
  if (mask)
    if (const int rc = room_for_tiles(h, b, &own, st)) return rc;
  if (prefix->mask) {
    if (const int rc = room_for_prefix_mask(h, &first, most * own.group, st)) return rc;
    if (const int rc = prefix_mask(h, prefix, first, most * own.group, st)) return rc;
  }
  if (const int rc = launch_attend(h, &first, most * own.group, true, st)) return rc;
  own.behind = 1;
  if (mask)
    if (const int rc = list_tiles(h, b, own, st)) return rc;
  return launch_attend(h, &own, rows_at_most(b, own.group), true, st);
}

// How attention over the cache is shared out, and how its parts are joined.
//
// An item is one block of a sequence's query rows (row = new token x group +
// head of the group) over one key/value head; its cached tokens come in tiles
// of 64. All items, laid end to end, a slot for each tile and some more for the
// item's fixed cost, are cut into equal ranges, one for each CTA, so that long
// and short sequences, many heads and one, fill the GPU alike. A CTA works
// through its range item by item. An item that lies in several ranges leaves a
// part in each: unnormalised sums, the maximum and the sum of the exponentials;
// the CTA that finishes last joins them, always in the order of the ranges, so
// that results do not depend on who is last. Nobody waits for anybody.
#pragma once

#include "kv_handle.cuh"

namespace cofie {

constexpr uint32_t kTile = 64;  // cached tokens of a tile

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
  uint32_t item_slots;  // slots that an item costs beside those of its tiles
  uint32_t q_wide, out_wide;  // rows of q (16-byte vectors) and of the output (8-byte) are aligned
  float scale;
  // tiles that the mask leaves, in order, and their count, for each sequence (with a mask)
  const uint32_t* tiles;
  const uint32_t* tile_count;
  uint32_t tile_stride;
  // parts: two for each CTA (of an item begun in an earlier one; of one that goes on in the next)
  float* part;       // [2 x CTAs][rows][D]
  float2* part_ms;   // [2 x CTAs][rows]: maximum (base 2), sum
  uint32_t* done;    // [CTAs]: parts finished of the item that goes on from this CTA; zero between calls
};

// Tiles of row block rb: those that its last row can see.
__device__ __forceinline__ uint32_t block_tiles(const AttendArgs& a, const Span& sp, uint32_t rows_per_block, uint32_t rb,
                                                uint32_t seq) {
  if (a.mask) return a.tile_count[seq];
  uint32_t end = sp.length;
  if (a.causal) {
    const uint32_t last = min(sp.count * a.group, (rb + 1) * rows_per_block) - 1;
    const int64_t seen = static_cast<int64_t>(sp.length) - sp.count + last / a.group + 1;
    end = seen <= 0 ? 0u : static_cast<uint32_t>(seen);
  }
  return (end + kTile - 1) / kTile;
}

__device__ __forceinline__ uint64_t sequence_slots(const AttendArgs& a, uint32_t rows_per_block, uint32_t seq, const Span& sp) {
  const uint32_t blocks = (sp.count * a.group + rows_per_block - 1) / rows_per_block;
  uint64_t n = 0;
  if (a.causal && !a.mask)
    for (uint32_t rb = 0; rb < blocks; ++rb) n += block_tiles(a, sp, rows_per_block, rb, seq) + a.item_slots;
  else if (blocks)
    n = static_cast<uint64_t>(blocks) * (block_tiles(a, sp, rows_per_block, 0, seq) + a.item_slots);
  return n * a.batch.kv_heads;
}

// One item of the CTA's range, or the part of it that lies there.
struct Item {
  uint32_t seq, rb, head;
  Span span;
  uint32_t tiles;           // of the whole item
  uint32_t lo, hi;          // those of this CTA
  uint32_t first_cta, last_cta;
};

// Called by one thread when the CTA has written its part of an item and a
// barrier has brought the writes of the others before this: counts the part,
// and says whether it was the last. Its fences are the CTA's: what its threads
// wrote is visible before the count, and, after the barrier that follows, what
// the other CTAs wrote is visible to all of them.
__device__ __forceinline__ uint32_t part_done(const AttendArgs& a, const Item& it) {
  __threadfence();
  const uint32_t last = atomicAdd(a.done + it.first_cta, 1u) == it.last_cta - it.first_cta;
  if (last) {
    a.done[it.first_cta] = 0;
    __threadfence();
  }
  return last;
}

constexpr uint32_t kSpans = 256;  // sequences that are looked up once and kept in shared memory

// Walks the items of one CTA's range. THREADS threads share the sequences.
template <int THREADS>
struct Plan {
  uint64_t before[THREADS + 1];  // slots before the sequences of each thread

  // All threads; ends with a barrier. The slots of a range.
  __device__ __forceinline__ uint64_t set_up(const AttendArgs& a, uint32_t rows_per_block, Span* spans) {
    const uint32_t per = (a.batch.n_seqs + THREADS - 1) / THREADS;
    const uint32_t t = threadIdx.x, lane = t % 32;
    uint64_t n = 0;
    for (uint32_t s = t * per; s < min(a.batch.n_seqs, (t + 1) * per); ++s) {
      const Span sp = sequence_span(a.batch, s);
      if (s < kSpans) spans[s] = sp;
      n += sequence_slots(a, rows_per_block, s, sp);
    }
    uint64_t sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t x = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= static_cast<uint32_t>(o)) sum += x;
    }
    before[t + 1] = sum;  // within the warp
    __syncthreads();
    uint64_t warps = 0;
    for (uint32_t w = 0; w < t / 32; ++w) warps += before[w * 32 + 32];
    __syncthreads();
    before[t + 1] = sum + warps;
    if (t == 0) before[0] = 0;
    __syncthreads();
    const uint64_t total = before[THREADS];
    return (total + gridDim.x - 1) / gridDim.x;
  }
};

// The walk itself (every thread keeps the same one).
template <int THREADS>
struct Walk {
  const AttendArgs& a;
  const uint32_t rows_per_block;
  const uint64_t range;
  const Span* spans;
  uint64_t at, end;    // what is left of the CTA's range
  uint64_t item_at;    // slot at which the next item begins
  uint32_t seq, rb, head, blocks;
  Span span;

  __device__ __forceinline__ Walk(const AttendArgs& args, const Plan<THREADS>& plan, const Span* kept, uint32_t rows, uint64_t range_slots)
      : a(args), rows_per_block(rows), range(range_slots), spans(kept) {
    const uint64_t total = plan.before[THREADS];
    at = min(total, static_cast<uint64_t>(blockIdx.x) * range);
    end = min(total, at + range);
    if (at >= end) return;
    uint32_t lo = 0, hi = THREADS;  // before[lo] <= at < before[hi]
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (plan.before[mid] <= at) lo = mid;
      else hi = mid;
    }
    seq = lo * ((a.batch.n_seqs + THREADS - 1) / THREADS);
    item_at = plan.before[lo];
    for (;; ++seq) {
      const uint64_t n = sequence_slots(a, rows_per_block, seq, span_of(seq));
      if (item_at + n > at || seq + 1 >= a.batch.n_seqs) break;
      item_at += n;
    }
    rb = head = 0;
    enter();
    for (;;) {  // row blocks of the sequence, then heads
      const uint64_t n = block_tiles(a, span, rows_per_block, rb, seq) + a.item_slots;
      if (item_at + n * a.batch.kv_heads > at) {
        head = static_cast<uint32_t>((at - item_at) / n);
        item_at += n * head;
        return;
      }
      item_at += n * a.batch.kv_heads;
      ++rb;
    }
  }

  __device__ __forceinline__ Span span_of(uint32_t s) const { return s < kSpans ? spans[s] : sequence_span(a.batch, s); }

  __device__ __forceinline__ void enter() {
    span = span_of(seq);
    blocks = (span.count * a.group + rows_per_block - 1) / rows_per_block;
  }

  // The next item with something to do here; false when the range is done.
  __device__ __forceinline__ bool next(Item& it) {
    while (at < end) {
      const uint32_t tiles = block_tiles(a, span, rows_per_block, rb, seq);
      const uint64_t first = item_at + a.item_slots, past = first + tiles;  // the tiles' slots
      const uint64_t lo = max(at, first), hi = min(end, past);
      const bool mine = tiles ? hi > lo : at <= item_at;  // an item without tiles belongs to its first slot
      if (mine) {
        it.seq = seq;
        it.rb = rb;
        it.head = head;
        it.span = span;
        it.tiles = tiles;
        it.lo = tiles ? static_cast<uint32_t>(lo - first) : 0;
        it.hi = tiles ? static_cast<uint32_t>(hi - first) : 0;
        it.first_cta = tiles ? static_cast<uint32_t>(first / range) : blockIdx.x;
        it.last_cta = tiles ? static_cast<uint32_t>((past - 1) / range) : blockIdx.x;
      }
      at = past;
      item_at = past;
      if (at < end) {  // the item after it
        if (++head == a.batch.kv_heads) {
          head = 0;
          if (++rb == blocks) {
            rb = 0;
            do ++seq, enter();
            while (blocks == 0 && seq + 1 < a.batch.n_seqs);
          }
        }
      }
      if (mine) return true;
    }
    return false;
  }
};

}  // namespace cofie

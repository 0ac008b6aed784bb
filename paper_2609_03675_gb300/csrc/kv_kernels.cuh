// The attention kernels of one kind of pages, without prefixes or with them, as
// their translation units give them (one for each: they take the compiler longest).
#pragma once

#include "kv_plan.cuh"

namespace cofie {

using AttendKernel = void (*)(AttendArgs);
// Up to 8 or 16 rows a block; tiles of 128, items cut or whole; up to 8 or 16, a CTA to each sequence and key head (shared
// prefixes only).
enum : int { kFew8 = 0, kFew16 = 1, kMany = 2, kManyWhole = 3, kShort8 = 4, kShort16 = 5 };

struct AttendLaunch {
  AttendKernel kernel;
  uint32_t threads;
  size_t smem;
  AttendKernel join[2];  // kMany: joins the parts, some rows to a CTA; as many CTAs as a block has rows for, or fewer
  uint32_t join_threads, join_rows;
};
// The kernel for the handle's type and head length. SHARED: over a prefix, or behind one.
template <int BITS, bool SHARED>
AttendLaunch attend_kernel(const cofie_kv_params& p, int kind);

}  // namespace cofie

// What the translation units of kv_kernels.cuh have in common.
#pragma once

#include "kv_kernels.cuh"
#include "kv_rows_tc.cuh"

namespace cofie {
namespace {

template <typename T, int D, int BITS, bool SHARED>
AttendLaunch attend_kernel_of(int kind) {
  if (kind == kMany)
    return {attend_rows_tc<T, D, BITS, SHARED, false>, kTcThreads<BITS>, tc_smem<D, BITS, SHARED>(),
            {attend_join<T, D, SHARED, false>, attend_join<T, D, SHARED, true>}, kJoinThreads, kJoinRows<D>};
  if (kind == kManyWhole) return {attend_rows_tc<T, D, BITS, SHARED, true>, kTcThreads<BITS>, tc_smem<D, BITS, SHARED>(), {}, 0, 0};
  if constexpr (SHARED) {
    if (kind == kShort8) return {attend_split<T, D, BITS, 1, true, true>, kSplitThreads<true>, split_smem<D, BITS, 1, true>(), {}, 0, 0};
    if (kind == kShort16) return {attend_split<T, D, BITS, 2, true, true>, kSplitThreads<true>, split_smem<D, BITS, 2, true>(), {}, 0, 0};
  }
  if (kind == kFew8) return {attend_split<T, D, BITS, 1, SHARED, false>, kSplitThreads<false>, split_smem<D, BITS, 1, false>(), {}, 0, 0};
  return {attend_split<T, D, BITS, 2, SHARED, false>, kSplitThreads<false>, split_smem<D, BITS, 2, false>(), {}, 0, 0};
}

}  // namespace

template <int BITS, bool SHARED>
AttendLaunch attend_kernel(const cofie_kv_params& p, int kind) {
  const auto of = [&](auto x) {
    using T = decltype(x);
    return p.head_dim == 64 ? attend_kernel_of<T, 64, BITS, SHARED>(kind) : attend_kernel_of<T, 128, BITS, SHARED>(kind);
  };
  return p.dtype == COFIE_BF16 ? of(__nv_bfloat16()) : of(__half());
}

}  // namespace cofie

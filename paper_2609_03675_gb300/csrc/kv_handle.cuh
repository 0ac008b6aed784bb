// The paged cache's handle, shared by its entry points.
#pragma once

#include <cuda.h>

#include <string>

#include "kv_rows.cuh"

struct cofie_kv {
  cofie_kv_params p{};
  int device = 0;
  uint32_t page_shift = 0;
  uint32_t* d_err = nullptr;
  // attention: CTAs that fit the GPU at once for 8 and for 16 rows each, the
  // parts that they leave, and the tiles that a mask leaves. That list grows on
  // demand, to twice its size at least; those before it stay with the handle,
  // because a captured call keeps the address that it was captured with.
  CUtensorMap maps[2];  // of 16-bit pages: keys, values
  uint32_t split_ctas[2][2] = {};  // of the kernels for shared prefixes, too
  float* d_part = nullptr;
  float2* d_part_ms = nullptr;
  uint32_t* d_done = nullptr;
  void* d_items = nullptr;  // of many rows: those that lie in more than one CTA's range
  uint32_t* d_tiles = nullptr;
  size_t tiles_room = 0;
  uint32_t* d_tiles_before[64] = {};  // doublings that a size_t allows
  uint32_t n_tiles_before = 0;
  // shared prefixes: what attention over them leaves for each row, and what their mask comes to. They grow and stay alike.
  struct Scratch {
    void* p = nullptr;
    size_t room = 0;
    void* before[64] = {};
    uint32_t n_before = 0;
  } shared_rows, shared_mask;
  std::string err;
  int fail(int code, const std::string& m) {
    err = m;
    return code;
  }
};

namespace cofie {

struct DeviceGuard {
  int prev = -1, dev;
  explicit DeviceGuard(int d) : dev(d) {
    if (cudaGetDevice(&prev) == cudaSuccess && prev != d) cudaSetDevice(d);
  }
  ~DeviceGuard() {
    if (prev >= 0 && prev != dev) cudaSetDevice(prev);
  }
};

// Checks the arguments that every call has; COFIE_OK, or the error noted on the handle.
int check_batch(cofie_kv* h, const cofie_kv_batch* b);
// Checks a tensor of the call's rows.
int check_rows(cofie_kv* h, const cofie_rows* r, uint32_t heads, bool has_out, const char* name);
BatchArg batch_arg(const cofie_kv* h, const cofie_kv_batch* b);
int launched(cofie_kv* h, cudaError_t e, const char* what);

// Allocates the attention's scratch (the handle's other fields are set).
cudaError_t attend_set_up(cofie_kv* h);

cudaError_t launch_rows(RowsArgs a, const RotaryTable& tab, uint32_t head_dim, uint32_t dtype, cudaStream_t st);

}  // namespace cofie

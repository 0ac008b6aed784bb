// Rotary positions: the handle (frequencies, formed on the host in double
// precision) and the kernel that rotates the heads of up to four tensors.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <string>

#include "kv_rows.cuh"

struct cofie_rotary {
  cofie_rotary_params p{};
  cofie::RotaryTable table{};
  std::string err;
  int fail(int code, const char* m) {
    err = m;
    return code;
  }
};

namespace cofie {

const RotaryTable& rotary_table(const cofie_rotary* h) { return h->table; }
uint32_t rotary_head_dim(const cofie_rotary* h) { return h->p.head_dim; }
uint32_t rotary_axes(const cofie_rotary* h) { return h->p.n_axes; }

namespace {

constexpr int kThreads = 256;
thread_local std::string g_rotary_error;

template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 4) rotate_rows(const __grid_constant__ RowsArgs a, const __grid_constant__ RotaryTable tab) {
  extern __shared__ __align__(16) float2 cs[];
  int64_t* place = reinterpret_cast<int64_t*>(cs + a.tile * cs_stride(tab.half));
  int32_t* offs = reinterpret_cast<int32_t*>(place + a.tile);
  const uint32_t t0 = blockIdx.x * a.tile, n = min(a.tile, a.n_tokens - t0);
  const uint32_t per = (a.heads + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * per;
  pdl_trigger();
  pdl_wait();
  rows_set_up(a, tab, t0, n, cs, place, offs);
  if (h0 < a.heads) rows_run<T, V>(a, tab, t0, n, h0, min(per, a.heads - h0), cs, place);
}

}  // namespace

// Launches rotate_rows over the rows of `a` (tile, units and vector width are set here).
cudaError_t launch_rows(RowsArgs a, const RotaryTable& tab, uint32_t head_dim, uint32_t dtype, cudaStream_t st) {
  const uint32_t size = dtype == COFIE_FP32 ? 4 : 2;
  const uint32_t v = rows_vector(a, tab, head_dim, size);
  a.units = head_dim / (2 * v);
  a.rotary_units = tab.half / v;
  a.offsets_in_smem = a.paged && a.batch.offsets && a.batch.n_seqs <= kOffsetsInSmem;
  // few tokens to a CTA where there would be few waves of CTAs, many where their set-up counts
  a.tile = a.n_tokens >= sm_count() * 256 ? 8 : a.n_tokens >= sm_count() * 16 ? 4 : 1;
  const uint32_t tiles = (a.n_tokens + a.tile - 1) / a.tile;
  const uint32_t parts = std::max(1u, std::min(a.heads, sm_count() * 4 / tiles));
  const dim3 grid(tiles, parts);
  const size_t smem = rows_smem(a.tile, tab.half, a.batch.n_seqs, a.offsets_in_smem);
  const auto go = [&](auto kernel) { return launch_dependent(true, kernel, grid, dim3(kThreads), smem, st, a, tab); };
  if (dtype == COFIE_FP32)
    return v == 4 ? go(rotate_rows<float, 4>) : v == 2 ? go(rotate_rows<float, 2>) : go(rotate_rows<float, 1>);
  if (dtype == COFIE_FP16)
    return v == 8   ? go(rotate_rows<__half, 8>)
           : v == 4 ? go(rotate_rows<__half, 4>)
           : v == 2 ? go(rotate_rows<__half, 2>)
                    : go(rotate_rows<__half, 1>);
  return v == 8   ? go(rotate_rows<__nv_bfloat16, 8>)
         : v == 4 ? go(rotate_rows<__nv_bfloat16, 4>)
         : v == 2 ? go(rotate_rows<__nv_bfloat16, 2>)
                  : go(rotate_rows<__nv_bfloat16, 1>);
}

}  // namespace cofie

using namespace cofie;

extern "C" {

int cofie_rotary_create(const cofie_rotary_params* p, cofie_rotary_t** out) {
  const auto bad = [](const char* m) { return g_rotary_error = m, COFIE_EINVAL; };
  if (!p || !out) return bad("params or out is NULL");
  if (p->head_dim < 2 || p->head_dim > 2 * kMaxPairs || p->head_dim % 2) return bad("head_dim must be even, in [2, 256]");
  if (p->rotary_dim < 2 || p->rotary_dim > p->head_dim || p->rotary_dim % 2) return bad("rotary_dim must be even, in [2, head_dim]");
  if (p->layout > COFIE_ROTARY_INTERLEAVED) return bad("layout must be one of COFIE_ROTARY_HALF, COFIE_ROTARY_INTERLEAVED");
  if (p->scaling > COFIE_ROTARY_YARN) return bad("scaling must be one of COFIE_ROTARY_NONE .. COFIE_ROTARY_YARN");
  if (!(p->base > 1.0 && std::isfinite(p->base))) return bad("base must be finite and above 1");
  if (!(p->factor >= 1.0 && std::isfinite(p->factor))) return bad("factor must be finite and at least 1");
  if (p->scaling == COFIE_ROTARY_NONE && p->factor != 1.0) return bad("a factor needs a scaling");
  if (p->scaling == COFIE_ROTARY_BASE && p->rotary_dim < 4) return bad("base scaling needs a rotary_dim of at least 4");
  if (p->scaling == COFIE_ROTARY_YARN &&
      !(p->original_len >= 1.0 && std::isfinite(p->original_len) && p->beta_slow >= 0.0 && p->beta_fast > p->beta_slow &&
        std::isfinite(p->beta_fast)))
    return bad("yarn scaling needs original_len >= 1 and beta_fast > beta_slow >= 0");
  if (p->n_axes < 1 || p->n_axes > kMaxAxes) return bad("n_axes must be in [1, 4]");
  const uint32_t half = p->rotary_dim / 2;
  for (uint32_t i = 0; p->axes && i < half; ++i)
    if (p->axes[i] >= p->n_axes) return bad("an entry of axes is not below n_axes");
  cofie_rotary* h = new (std::nothrow) cofie_rotary();
  if (!h) return g_rotary_error = "host allocation failed", COFIE_ENOMEM;
  h->p = *p;
  h->p.axes = nullptr;
  const double pi = 3.14159265358979323846;
  double base = p->base, m = 1.0;
  if (p->scaling == COFIE_ROTARY_BASE) base *= std::pow(p->factor, static_cast<double>(p->rotary_dim) / (p->rotary_dim - 2));
  if (p->scaling == COFIE_ROTARY_YARN) m = 0.1 * std::log(p->factor) + 1.0;
  RotaryTable& t = h->table;
  t.half = half;
  t.layout = p->layout;
  t.amplitude = static_cast<float>(m);
  for (uint32_t i = 0; i < half; ++i) {
    double f = std::pow(base, -2.0 * i / p->rotary_dim);
    if (p->scaling == COFIE_ROTARY_LINEAR) f /= p->factor;
    if (p->scaling == COFIE_ROTARY_YARN) {
      const double r = p->original_len * f / (2.0 * pi);
      const double g = std::min(1.0, std::max(0.0, (r - p->beta_slow) / (p->beta_fast - p->beta_slow)));
      f = (1.0 - g) * f / p->factor + g * f;
    }
    t.turn[i] = static_cast<uint64_t>(std::ldexp(f / (2.0 * pi), 64));  // f <= 1: under a sixth of 2^64
    t.axis[i] = p->axes ? p->axes[i] : 0;
  }
  *out = h;
  return COFIE_OK;
}

void cofie_rotary_destroy(cofie_rotary_t* h) { delete h; }

int cofie_rotary_run(cofie_rotary_t* h, const cofie_rows* rows, uint32_t n_rows, uint32_t n_tokens, const int32_t* positions,
                     uint32_t dtype, int transpose, void* cuda_stream) {
  if (!h) return COFIE_EINVAL;
  if (!rows || n_rows < 1 || n_rows > 4) return h->fail(COFIE_EINVAL, "rows must name 1 to 4 tensors");
  if (dtype > COFIE_FP32) return h->fail(COFIE_EINVAL, "dtype must be COFIE_BF16, COFIE_FP16 or COFIE_FP32");
  if (n_tokens > 0x7fffffffu) return h->fail(COFIE_EINVAL, "n_tokens must be below 2^31");
  if (n_tokens == 0) return COFIE_OK;
  if (!positions) return h->fail(COFIE_EINVAL, "positions is required");
  const uint32_t size = dtype == COFIE_FP32 ? 4 : 2;
  RowsArgs a{};
  a.n_rows = n_rows;
  a.n_tokens = n_tokens;
  a.positions = positions;
  a.transpose = transpose != 0;
  for (uint32_t i = 0; i < n_rows; ++i) {
    const cofie_rows& r = rows[i];
    if (!r.in || !r.out) return h->fail(COFIE_EINVAL, "a tensor's in or out is NULL");
    if (r.heads < 1 || r.heads > 4096) return h->fail(COFIE_EINVAL, "heads must be in [1, 4096]");
    if (reinterpret_cast<uintptr_t>(r.in) % size || reinterpret_cast<uintptr_t>(r.out) % size)
      return h->fail(COFIE_EINVAL, "a tensor is not aligned to its type");
    if (r.in == r.out && (r.in_token != r.out_token || r.in_head != r.out_head))
      return h->fail(COFIE_EINVAL, "in place, the strides of in and out must be the same");
    a.rows[i] = {static_cast<const char*>(r.in), static_cast<char*>(r.out), r.in_token, r.in_head, r.out_token, r.out_head, r.heads, kRotate};
    a.heads += r.heads;
  }
  const cudaError_t e = launch_rows(a, h->table, h->p.head_dim, dtype, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) {
    cudaGetLastError();
    return h->fail(COFIE_ECUDA, cudaGetErrorString(e));
  }
  return COFIE_OK;
}

const char* cofie_rotary_last_error(const cofie_rotary_t* h) { return h ? h->err.c_str() : g_rotary_error.c_str(); }

}  // extern "C"

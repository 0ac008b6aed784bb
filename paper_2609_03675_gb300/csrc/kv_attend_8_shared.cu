#include "kv_kernels_impl.cuh"

template cofie::AttendLaunch cofie::attend_kernel<8, true>(const cofie_kv_params&, int);

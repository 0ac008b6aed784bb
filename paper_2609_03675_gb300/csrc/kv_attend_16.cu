#include "kv_kernels_impl.cuh"

template cofie::AttendLaunch cofie::attend_kernel<16, false>(const cofie_kv_params&, int);

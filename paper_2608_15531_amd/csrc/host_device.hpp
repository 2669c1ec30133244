// For functions that kernels, host code and tests compiled for the host share.
#pragma once

#ifdef __HIPCC__
#define FQ_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define FQ_HOST_DEVICE inline
#endif

// Functions for the host and the device, in headers that a C++ compiler alone can read.
#pragma once
#ifdef __CUDACC__
#define QC_ANY_SIDE __host__ __device__ __forceinline__
#else
#define QC_ANY_SIDE inline
#endif

// Seconds and bytes to whole time units and memory bins, saturating at 2^30: of the cost model and of what is added to it.  Only in translation
// units compiled with -fmad=false.
#pragma once

#include <stdint.h>

__device__ __forceinline__ int32_t quant_time(double t_s, double unit_ns) {
    double q = rint(t_s * 1e9 / unit_ns);
    if (!(q < 1073741824.0)) q = 1073741824.0;
    if (q < 0.0) q = 0.0;
    return (int32_t)q;
}

__device__ __forceinline__ int32_t quant_mem(double bytes, double bin_bytes) {
    double q = ceil(bytes / bin_bytes);
    if (!(q < 1073741824.0)) q = 1073741824.0;
    if (q < 0.0) q = 0.0;
    return (int32_t)q;
}

// Device helpers shared by the language-model operators.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mt_device.cuh"

namespace mt {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float bf16_to_f(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ __forceinline__ uint16_t f_to_bf16(float x) { return static_cast<uint16_t>(pack_bf16x2(x, 0.f)); }
__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fffffff); }

// Sticky status: the first code stays, the smallest index concerned goes with it.
__device__ __forceinline__ void raise_status(int32_t* status, int code, int index) {
    atomicCAS(&status[ST_CODE], MT_OK, code);
    atomicMin(&status[ST_BAD_INDEX], index);
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

}  // namespace mt

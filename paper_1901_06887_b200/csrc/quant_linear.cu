// Products of a mixed batch of rows with the tenants' 4-bit weights.  First form: one warp per (row, 16 outputs).
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

// One thread per 32-bit word of the packed codes, then one per scale.
__global__ void quant_pack_kernel(const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales, int tenants, int K, int N,
                                  int group, uint8_t* __restrict__ packed, size_t tenant_bytes, size_t codes_bytes) {
    const size_t words = codes_bytes / 4, n_scales = (tenant_bytes - codes_bytes) / 2, per = words + n_scales;
    const size_t step = (size_t)gridDim.x * blockDim.x;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < per * tenants; i += step) {
        const size_t t = i / per, r = i % per;
        uint8_t* out = packed + t * tenant_bytes;
        if (r < words) {
            const int w = (int)(r & 3), lane = (int)(r >> 2) & 31;
            const size_t block = r >> 7;
            const int kb = (int)(block % (K / 64));
            const int row = (int)(block / (K / 64)) * 16 + lane / 4 + 8 * (w >> 1);
            const int k0 = kb * 64 + 32 * (w & 1) + 8 * (lane & 3);
            uint32_t v = 0;
            if (row < N) {
                const uint8_t* src = codes + (t * N + row) * (size_t)(K / 2) + k0 / 2;
                for (int p = 0; p < 4; ++p) v |= (uint32_t)(src[p] & 15) << (4 * p) | (uint32_t)(src[p] >> 4) << (4 * p + 16);
            }
            reinterpret_cast<uint32_t*>(out)[r] = v;
        } else {
            const size_t q = r - words;
            const size_t block = q >> 4;
            const int g = (int)(block % (K / group));
            const int row = (int)(block / (K / group)) * 16 + (int)(q & 15) / 2 + 8 * (int)(q & 1);
            reinterpret_cast<uint16_t*>(out + codes_bytes)[q] = row < N ? scales[(t * N + row) * (size_t)(K / group) + g] : uint16_t(0);
        }
    }
}

__global__ void quant_linear_simple(QuantLinearArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int tiles = (a.N + 15) / 16;
    const int warp = (blockIdx.x * blockDim.x + threadIdx.x) / 32, lane = threadIdx.x & 31;
    const int r = warp / tiles, tile = warp % tiles;
    if (r >= a.n) return;
    const int id = a.ids[r], g = lane / 4, t = lane & 3;
    const bool bad = id < 0 || id >= a.tenants;
    float acc[2] = {};
    if (!bad) {
        const uint8_t* base = a.packed + (size_t)id * quant_tenant_bytes(a.K, a.N, a.group);
        const uint4* codes = reinterpret_cast<const uint4*>(base) + (size_t)tile * (a.K / 64) * 32;
        const uint16_t* sc = reinterpret_cast<const uint16_t*>(base + quant_codes_bytes(a.K, a.N)) + (size_t)tile * (a.K / a.group) * 16;
        for (int kb = 0; kb < a.K / 64; ++kb) {
            const uint4 w = codes[kb * 32 + lane];
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
            for (int i = 0; i < 4; ++i) {
                const int k0 = kb * 64 + 32 * (i & 1) + 8 * t;
                float p = 0.f;
                for (int j = 0; j < 8; ++j)
                    p += bf16_to_f(a.x[r * a.x_stride + k0 + j]) * (float)((int)((ws[i] >> (4 * (j / 2) + 16 * (j & 1))) & 15) - 8);
                acc[i >> 1] += p * bf16_to_f(sc[(k0 / a.group) * 16 + g * 2 + (i >> 1)]);
            }
        }
    } else if (tile == 0 && lane == 0) {
        raise_status(a.status, MT_ERR_BAD_MODEL_ID, a.row0 + r);
    }
    for (int i = 0; i < 2; ++i) {
        float v = acc[i];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        const int row = tile * 16 + g + 8 * i;
        if (t != 0 || row >= a.N) continue;
        v = bad ? nan_f() : v + (a.bias ? a.bias[(size_t)id * a.N + row] : 0.f);
        if (a.y_fp32) static_cast<float*>(a.y)[r * a.y_stride + row] = v;
        else static_cast<uint16_t*>(a.y)[r * a.y_stride + row] = f_to_bf16(v);
    }
}

}  // namespace

cudaError_t configure_quant_linear() { return cudaSuccess; }

cudaError_t launch_quant_pack(const uint8_t* codes, const uint16_t* scales, int tenants, int K, int N, int group, void* packed,
                              cudaStream_t s) {
    const size_t cb = quant_codes_bytes(K, N), tb = quant_tenant_bytes(K, N, group);
    const size_t items = (cb / 4 + (tb - cb) / 2) * (size_t)tenants;
    const size_t blocks = (items + 255) / 256;
    quant_pack_kernel<<<dim3((unsigned)(blocks < 4736 ? blocks : 4736)), dim3(256), 0, s>>>(codes, scales, tenants, K, N, group, static_cast<uint8_t*>(packed), tb, cb);
    ++g_kernel_launches;
    return cudaGetLastError();
}

cudaError_t launch_quant_linear(const QuantLinearArgs& a, int, cudaStream_t s) {
    const int64_t warps = (int64_t)a.n * ((a.N + 15) / 16);
    return launch_pdl(quant_linear_simple, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, s, a);
}

}  // namespace mt

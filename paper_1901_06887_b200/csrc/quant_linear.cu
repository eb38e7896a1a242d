// Products of a mixed batch of rows with the tenants' 4-bit weights: y_r = sum_k scale (code - 8) x_rk + bias, tenant by tenant.
//
// Mathematics.  The codes enter the matrix instructions as the exact bf16 numbers code - 8 (four bits set into the mantissa of 128, then an
// exact subtraction of 136) with the weights as the 16-row operand and up to 64 of the tenant's rows as columns; the sum over 64 (or 32)
// inputs is multiplied with the group's scale in fp32 and added up in fp32.  Nothing is rounded but the sums.
//
// Bound: memory, K / 2 + 2 K / group bytes per output and tenant, whatever the number of its rows (up to some 16; beyond, the matrix
// instructions).  The packed order makes a warp's load 512 contiguous bytes that are the operand of four instructions; the rows' slices of the
// inner index are chosen so that a lane's inputs are 16 contiguous bytes too, so nothing passes through shared memory on the way in.
//
// Split.  A CTA takes (tenant, 16 outputs) units in turn, its eight warps every eighth block of 64 inputs; they join through shared memory.
// Which tenants occur is found out by every CTA for itself from the ids (at most 256 a launch): no bucketing launch, and only tenants that
// occur cost anything.
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

constexpr int kThreads = 256, kWarps = 8;

// D = A B + C
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3,
                                         const uint32_t b0, const uint32_t b1, const float (&c)[4]) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// Codes in nibbles P and P + 4 of w as two bf16 numbers code - 8.
template <int P>
__device__ __forceinline__ uint32_t centred(uint32_t w) {
    uint32_t d;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(((w >> (4 * P)) & 0x000f000fu) | 0x43004300u), "r"(0xc308c308u));   // 128 + code - 136
    return d;
}

struct Shared {
    int ids[kQuantRowsPerLaunch], slot[kQuantRowsPerLaunch], order[kQuantRowsPerLaunch];
    int tenant[kQuantRowsPerLaunch], begin[kQuantRowsPerLaunch + 1];
    int warp_n[kWarps];
    int n_slots, n_valid;
};

// One unit: 16 outputs of one tenant for up to 8 NT rows (s.order[r0 ..]).
template <int NT, bool G32>
__device__ __forceinline__ void unit(const QuantLinearArgs& a, const Shared& s, float* red, const uint8_t* base, size_t codes_bytes, int tile, int r0,
                                     int rows, int tenant) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int kblocks = a.K / 64, groups = a.groups;
    const uint4* const codes = reinterpret_cast<const uint4*>(base) + (size_t)tile * kblocks * 32 + lane;
    const uint32_t* const scales = reinterpret_cast<const uint32_t*>(base + codes_bytes) + (size_t)tile * groups * 8 + g;
    const uint16_t* x[NT];                       // (columns behind the last row repeat a row; they are not written)
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n] = a.x + (int64_t)s.order[r0 + min(n * 8 + g, rows - 1)] * a.x_stride + 8 * t;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;

    struct Block {
        uint4 w, x[NT][2];
        uint32_t s0, s1;
    };
    auto load = [&](Block& b, int kb) {
        b.w = __ldcs(codes + (size_t)kb * 32);
        b.s0 = __ldg(scales + (size_t)(G32 ? 2 * kb : (int)__umulhi(kb + 1, a.per_magic)) * 8);       // kb / (blocks per group)
        if (G32) b.s1 = __ldg(scales + (size_t)(2 * kb + 1) * 8);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            b.x[n][0] = __ldg(reinterpret_cast<const uint4*>(x[n] + (size_t)kb * 64));
            b.x[n][1] = __ldg(reinterpret_cast<const uint4*>(x[n] + (size_t)kb * 64 + 32));
        }
    };
    auto use = [&](const Block& b) {
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        float c[NT][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {                // inputs 0..31 and 32..63 of the block
            const uint32_t lo = h == 0 ? b.w.x : b.w.y, hi = h == 0 ? b.w.z : b.w.w;      // rows g and g + 8
            const uint32_t a00 = centred<0>(lo), a01 = centred<1>(lo), a02 = centred<2>(lo), a03 = centred<3>(lo);
            const uint32_t a10 = centred<0>(hi), a11 = centred<1>(hi), a12 = centred<2>(hi), a13 = centred<3>(hi);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint4 v = b.x[n][h];
                if (h == 0 || G32) mma_bf16(c[n], a00, a10, a01, a11, v.x, v.y, zero);
                else mma_bf16(c[n], a00, a10, a01, a11, v.x, v.y, c[n]);
                mma_bf16(c[n], a02, a12, a03, a13, v.z, v.w, c[n]);
                if (h == 1 || G32) {
                    const uint32_t sc = G32 && h == 1 ? b.s1 : b.s0;
                    const float s0 = bf16_lo(sc), s1 = bf16_hi(sc);
                    acc[n][0] = fmaf(s0, c[n][0], acc[n][0]); acc[n][1] = fmaf(s0, c[n][1], acc[n][1]);
                    acc[n][2] = fmaf(s1, c[n][2], acc[n][2]); acc[n][3] = fmaf(s1, c[n][3], acc[n][3]);
                }
            }
        }
    };
    constexpr int U = NT == 1 ? 4 : NT == 2 ? 2 : 1;      // blocks in flight
    int kb = warp;
    for (; kb + (U - 1) * kWarps < kblocks; kb += U * kWarps) {
        Block b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) load(b[u], kb + u * kWarps);
#pragma unroll
        for (int u = 0; u < U; ++u) use(b[u]);
    }
    for (; kb < kblocks; kb += kWarps) {
        Block b;
        load(b, kb);
        use(b);
    }
    // join the warps: red[warp][column][16 outputs, padded to 20]
    __syncthreads();                                       // the unit before this has been read
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float* const r = red + ((warp * NT + n) * 8 + 2 * t) * 20 + g;
        r[0] = acc[n][0]; r[20] = acc[n][1]; r[8] = acc[n][2]; r[28] = acc[n][3];
    }
    __syncthreads();
    for (int i = tid; i < rows * 16; i += kThreads) {
        const int col = i >> 4, o = i & 15, out = tile * 16 + o;
        if (out >= a.N) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += red[(w * NT * 8 + col) * 20 + o];
        if (a.bias) v += __ldg(a.bias + (size_t)tenant * a.N + out);
        const int64_t at = (int64_t)s.order[r0 + col] * a.y_stride + out;
        if (a.y_fp32) static_cast<float*>(a.y)[at] = v;
        else static_cast<uint16_t*>(a.y)[at] = f_to_bf16(v);
    }
}

// MAXT: largest number of column tiles a pass may take (a launch of n rows never needs more than n of them).
template <int MAXT, bool G32>
__global__ void __launch_bounds__(kThreads, MAXT <= 4 ? 3 : 2) quant_linear_kernel(const QuantLinearArgs a) {
    __shared__ Shared s;
    __shared__ float red[kWarps * MAXT * 8 * 20];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31;
    pdl_launch_dependents();
    pdl_wait();
    // --- rows by tenant: slots in order of first appearance, rows of a slot in order of the batch, rows with a bad id last
    const int id = tid < a.n ? a.ids[tid] : -1;
    const bool good = id >= 0 && id < a.tenants;
    s.ids[tid] = good ? id : -1;
    if (tid < a.n && !good && blockIdx.x == 0) raise_status(a.status, MT_ERR_BAD_MODEL_ID, a.row0 + tid);
    __syncthreads();
    int first = tid;
    if (good)
        for (int j = 0; j < tid; ++j)
            if (s.ids[j] == id) { first = j; break; }
    const unsigned firsts = __ballot_sync(0xffffffffu, good && first == tid);
    if (lane == 0) s.warp_n[warp] = __popc(firsts);
    __syncthreads();
    int slot = __popc(firsts & ((1u << lane) - 1u)), n_slots = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) slot += s.warp_n[w];
        n_slots += s.warp_n[w];
    }
    if (good && first == tid) { s.slot[tid] = slot; s.tenant[slot] = id; }
    __syncthreads();
    const int mine = good ? s.slot[first] : n_slots;       // (written by first occurrences only: stable from here on)
    __syncthreads();
    s.slot[tid] = tid < a.n ? mine : 0x7fffffff;
    __syncthreads();
    if (tid < a.n) {
        int at = 0, same = 0;
        for (int j = 0; j < a.n; ++j) {
            const int sj = s.slot[j];
            at += (sj < mine || (sj == mine && j < tid)) ? 1 : 0;
            same += (sj == mine && j < tid) ? 1 : 0;
        }
        s.order[at] = tid;
        if (same == 0) s.begin[mine] = at;
    }
    if (tid == 0) s.n_slots = n_slots;
    const int n_valid = __syncthreads_count(good);
    if (tid == 0) s.begin[n_slots] = n_valid;
    __syncthreads();

    for (int i = n_valid; i < a.n; ++i) {                  // rows with a bad id
        const int64_t at = (int64_t)s.order[i] * a.y_stride;
        for (int o = blockIdx.x * kThreads + tid; o < a.N; o += gridDim.x * kThreads) {
            if (a.y_fp32) static_cast<float*>(a.y)[at + o] = nan_f();
            else static_cast<uint16_t*>(a.y)[at + o] = 0x7fff;
        }
    }

    const int tiles = (a.N + 15) / 16;
    const size_t codes_bytes = quant_codes_bytes(a.K, a.N), tenant_bytes = quant_tenant_bytes(a.K, a.N, a.group);
    const int64_t units = (int64_t)tiles * n_slots;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int sl = (int)(u / tiles), tile = (int)(u - (int64_t)sl * tiles), tenant = s.tenant[sl];
        const uint8_t* const base = a.packed + (size_t)tenant * tenant_bytes;
        for (int r0 = s.begin[sl], end = s.begin[sl + 1]; r0 < end; r0 += 64) {
            const int rows = min(end - r0, 64);
            if (MAXT == 1 || rows <= 8) unit<1, G32>(a, s, red, base, codes_bytes, tile, r0, rows, tenant);
            else if (MAXT == 2 || rows <= 16) unit<(MAXT < 2 ? MAXT : 2), G32>(a, s, red, base, codes_bytes, tile, r0, rows, tenant);
            else if (rows <= 32) unit<(MAXT < 4 ? MAXT : 4), G32>(a, s, red, base, codes_bytes, tile, r0, rows, tenant);
            else unit<(MAXT < 8 ? MAXT : 8), G32>(a, s, red, base, codes_bytes, tile, r0, rows, tenant);
        }
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

cudaError_t launch_quant_linear(const QuantLinearArgs& a, int sm_count, cudaStream_t s) {
    const bool g32 = a.group == 32;
    const int most_slots = a.n < a.tenants ? a.n : a.tenants;
    const int64_t units = (int64_t)((a.N + 15) / 16) * most_slots;
    const int maxt = a.n <= 8 ? 1 : a.n <= 16 ? 2 : a.n <= 32 ? 4 : 8;
    int64_t grid = (int64_t)sm_count * (maxt <= 4 ? 3 : 2);
    if (grid > units) grid = units;
    typedef void (*Kernel)(QuantLinearArgs);
    static const Kernel kernels[2][4] = {
        {quant_linear_kernel<1, false>, quant_linear_kernel<2, false>, quant_linear_kernel<4, false>, quant_linear_kernel<8, false>},
        {quant_linear_kernel<1, true>, quant_linear_kernel<2, true>, quant_linear_kernel<4, true>, quant_linear_kernel<8, true>}};
    QuantLinearArgs b = a;
    b.groups = a.K / a.group;
    const uint32_t per = g32 ? 1u : (uint32_t)a.group / 64u;
    b.per_magic = 0xffffffffu / per;
    return launch_pdl(kernels[g32][maxt == 1 ? 0 : maxt == 2 ? 1 : maxt == 4 ? 2 : 3], dim3((unsigned)grid), dim3(kThreads), 0, s, b);
}

}  // namespace mt

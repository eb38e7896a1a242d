// The 4-bit cache of keys and values: rounding rows into slots and reading slots back.
//
// A row of head_dim elements becomes bias = min, scale = bf16((max - min) / 15) and codes rint((x - bias) / scale), as IEEE
// subtraction and division give them (codes are found by the reciprocal and settled by exact remainders), so the stored bytes are a
// function of the row alone.  Both directions move (2 + 1/2) bytes per element.  For a step's few tokens they are bound by the launch; for 8191
// tokens of 8 heads of 128 they take 23 and 14 us cold, 3.3 and 2 times their bytes.  Append: 78 % of the issue slots while an SM has work, which is
// 82 % of the time (2048 short CTAs of one load - reduce - store chain, 3.5 waves); a quarter fewer instructions left its time as it was.  Read: waits
// on memory first (codes behind slots), SMs with work 74 % of the time.  A row is one group of lanes, 16 bytes (8 elements) a lane: 8 lanes for head_dim 64, 16 for 128.  A CTA takes one
// head's keys or values of 16 (32) tokens, or four times as many where that still fills the GPU: then a lane has four loads in flight.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

struct CachePtrs {
    uint8_t* codes;
    uint32_t* params;       // (scale, bias) as two bf16
};

__device__ __forceinline__ float min_nan(float a, float b) {
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

constexpr int kThreads = 256;

// grid (2 heads, tokens): a CTA's tokens are ITEMS runs of kThreads / L; neighbouring CTAs take the other heads, keys and values of the same
// tokens, which lie side by side in a projection's output (append and read of 8191 tokens of 8 heads: 29 us together on rotating inputs).
template <int D, int ITEMS>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(CachePtrs kc, CachePtrs vc, int64_t n_slots, int page_shift, KvRows k, KvRows v,
                                                             const int64_t* __restrict__ slots, int n, int token0, OpStatus status) {
    constexpr int L = D / 8, kTokens = kThreads / L;            // lanes per row, rows of a run
    pdl_launch_dependents();
    pdl_wait();
    const int sub = threadIdx.x % L, head = blockIdx.x >> 1, heads = gridDim.x >> 1;
    const bool values = blockIdx.x & 1;
    const KvRows& src = values ? v : k;
    const CachePtrs& dst = values ? vc : kc;
    uint4 w[ITEMS];
    int64_t slot[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {                           // (the row does not wait for its slot)
        const int64_t token = ((int64_t)blockIdx.y * ITEMS + i) * kTokens + threadIdx.x / L;
        w[i] = make_uint4(0, 0, 0, 0);
        slot[i] = -1;
        if (token < n) {
            w[i] = __ldcs(reinterpret_cast<const uint4*>(src.p + token * src.token_stride + head * src.head_stride + sub * 8));
            slot[i] = __ldg(slots + token);
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const float x[8] = {bf16_lo(w[i].x), bf16_hi(w[i].x), bf16_lo(w[i].y), bf16_hi(w[i].y),
                            bf16_lo(w[i].z), bf16_hi(w[i].z), bf16_lo(w[i].w), bf16_hi(w[i].w)};
        float lo = x[0], hi = x[0];                  // NaN if any is
#pragma unroll
        for (int e = 1; e < 8; ++e) { lo = min_nan(lo, x[e]); hi = max_nan(hi, x[e]); }
#pragma unroll
        for (int o = L / 2; o; o >>= 1) {
            lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        const float spread = hi - lo;
        const bool finite = spread < INFINITY;
        const uint16_t scale_b = finite ? f_to_bf16(__fdiv_rn(spread, 15.f)) : uint16_t(0x7fff);
        const uint16_t bias_b = f_to_bf16(lo);       // exact: lo is an element
        const float scale = bf16_to_f(scale_b);
        uint32_t packed = 0;
        if (finite && scale > 0.f) {
            // The quotient by way of the reciprocal errs by some 2^-20 and may miss the nearest code only where it lies that near to the
            // middle between two; there the remainder decides (exactly: code * scale has 12 bits), ties to the even code.  Dividing there
            // instead, in 4 of 10 warps, made the kernel twice as long as its memory takes.
            constexpr float kMagic = 12582912.f;     // 1.5 * 2^23: the sum's low bits are the nearest whole number
            if (scale > 1e-30f) {
                const float inv = __fdividef(1.f, scale);
                float r[8];
                bool near = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float q = fminf((x[e] - lo) * inv, 15.f);
                    r[e] = q + kMagic;
                    near = near || fabsf(q - (r[e] - kMagic)) > 0.4999f;
                }
                if (near) {
                    const float half = 0.5f * scale;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float d = fmaf(-(r[e] - kMagic), scale, x[e] - lo);
                        const bool odd = __float_as_uint(r[e]) & 1u;
                        if (d > half || (d == half && odd)) r[e] += 1.f;
                        if (d < -half || (d == -half && odd)) r[e] -= 1.f;
                        r[e] = fminf(r[e], kMagic + 15.f);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) packed |= (__float_as_uint(r[e]) & 15u) << (4 * e);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) packed |= (uint32_t)fminf(rintf(__fdiv_rn(x[e] - lo, scale)), 15.f) << (4 * e);
            }
        }
        if (slot[i] < 0 || slot[i] >= n_slots) {
            if (slot[i] != -1 && head == 0 && !values && sub == 0)
                raise_status(status, MT_ERR_INVALID_ARG, token0 + (int)(((int64_t)blockIdx.y * ITEMS + i) * kTokens + threadIdx.x / L));
            continue;
        }
        const int64_t at = (((slot[i] >> page_shift) * heads + head) << page_shift) + (slot[i] & ((1 << page_shift) - 1));
        *reinterpret_cast<uint32_t*>(dst.codes + at * (D / 2) + sub * 4) = packed;
        if (sub == 0) dst.params[at] = (uint32_t)bias_b << 16 | scale_b;
    }
}

template <int D, int ITEMS>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(CachePtrs kc, CachePtrs vc, int64_t n_slots, int page_shift,
                                                           const int64_t* __restrict__ slots, int n, uint16_t* __restrict__ k_out,
                                                           uint16_t* __restrict__ v_out, int token0, OpStatus status) {
    constexpr int L = D / 8, kTokens = kThreads / L;
    pdl_launch_dependents();
    pdl_wait();
    const int sub = threadIdx.x % L, head = blockIdx.x >> 1, heads = gridDim.x >> 1;
    const bool values = blockIdx.x & 1;
    const CachePtrs& src = values ? vc : kc;
    uint16_t* const out = values ? v_out : k_out;
    int64_t slot[ITEMS];
    uint32_t p[ITEMS], c[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t token = ((int64_t)blockIdx.y * ITEMS + i) * kTokens + threadIdx.x / L;
        slot[i] = token < n ? __ldg(slots + token) : -1;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        p[i] = c[i] = 0u;
        if (slot[i] >= 0 && slot[i] < n_slots) {
            const int64_t at = (((slot[i] >> page_shift) * heads + head) << page_shift) + (slot[i] & ((1 << page_shift) - 1));
            p[i] = src.params[at];
            c[i] = *reinterpret_cast<const uint32_t*>(src.codes + at * (D / 2) + sub * 4);
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t token = ((int64_t)blockIdx.y * ITEMS + i) * kTokens + threadIdx.x / L;
        if (token >= n) continue;
        const float scale = bf16_lo(p[i]), bias = bf16_hi(p[i]);
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] = pack_bf16x2(__fadd_rn(__fmul_rn((float)((c[i] >> (8 * e)) & 15), scale), bias),
                               __fadd_rn(__fmul_rn((float)((c[i] >> (8 * e + 4)) & 15), scale), bias));
        uint4 w = make_uint4(o[0], o[1], o[2], o[3]);
        if (slot[i] < -1 || slot[i] >= n_slots) {
            w = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
            if (head == 0 && !values && sub == 0) raise_status(status, MT_ERR_INVALID_ARG, token0 + (int)token);
        }
        __stcs(reinterpret_cast<uint4*>(out + (token * heads + head) * D + sub * 8), w);
    }
}

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

// Runs of tokens per CTA: four where that leaves two CTAs for every SM.
int items_for(int64_t n, int heads, int d, int sm_count) { return n * heads * 2 * (d / 8) / kThreads >= 4LL * 2 * sm_count ? 4 : 1; }
constexpr int kMaxRuns = 65535;                  // rows of a grid
int tokens_of(int d, int items) { return kThreads / (d / 8) * items; }
int runs_of(int n, int tokens) { return (int)((n + (int64_t)tokens - 1) / tokens); }

}  // namespace

cudaError_t launch_kv_append(const mt_kv_cache& c, const KvRows& k, const KvRows& v, const int64_t* slots, int n, const OpStatus& status,
                             int sm_count, cudaStream_t s) {
    const CachePtrs kc = {static_cast<uint8_t*>(c.k_codes), static_cast<uint32_t*>(c.k_params)};
    const CachePtrs vc = {static_cast<uint8_t*>(c.v_codes), static_cast<uint32_t*>(c.v_params)};
    const int items = items_for(n, c.kv_heads, c.head_dim, sm_count);
    auto* const f = c.head_dim == 64 ? (items == 1 ? kv_append_kernel<64, 1> : kv_append_kernel<64, 4>)
                                     : (items == 1 ? kv_append_kernel<128, 1> : kv_append_kernel<128, 4>);
    const int tokens = tokens_of(c.head_dim, items), most = kMaxRuns * tokens;
    cudaError_t e = cudaSuccess;
    for (int64_t t0 = 0; t0 < n && e == cudaSuccess; t0 += most) {
        const int m = n - t0 < most ? (int)(n - t0) : most;
        const KvRows kr = {k.p + t0 * k.token_stride, k.token_stride, k.head_stride}, vr = {v.p + t0 * v.token_stride, v.token_stride, v.head_stride};
        e = launch_pdl(f, dim3((unsigned)c.kv_heads * 2, (unsigned)runs_of(m, tokens)), dim3(kThreads), 0, s, kc, vc, (int64_t)c.n_pages * c.page_tokens,
                       log2_of(c.page_tokens), kr, vr, slots + t0, m, (int)t0, status);
    }
    return e;
}

cudaError_t launch_kv_read(const mt_kv_cache& c, const int64_t* slots, int n, uint16_t* k_out, uint16_t* v_out, const OpStatus& status,
                           int sm_count, cudaStream_t s) {
    const CachePtrs kc = {static_cast<uint8_t*>(c.k_codes), static_cast<uint32_t*>(c.k_params)};
    const CachePtrs vc = {static_cast<uint8_t*>(c.v_codes), static_cast<uint32_t*>(c.v_params)};
    const int items = items_for(n, c.kv_heads, c.head_dim, sm_count);
    auto* const f = c.head_dim == 64 ? (items == 1 ? kv_read_kernel<64, 1> : kv_read_kernel<64, 4>)
                                     : (items == 1 ? kv_read_kernel<128, 1> : kv_read_kernel<128, 4>);
    const int tokens = tokens_of(c.head_dim, items), most = kMaxRuns * tokens;
    const int64_t row = (int64_t)c.kv_heads * c.head_dim;
    cudaError_t e = cudaSuccess;
    for (int64_t t0 = 0; t0 < n && e == cudaSuccess; t0 += most) {
        const int m = n - t0 < most ? (int)(n - t0) : most;
        e = launch_pdl(f, dim3((unsigned)c.kv_heads * 2, (unsigned)runs_of(m, tokens)), dim3(kThreads), 0, s, kc, vc, (int64_t)c.n_pages * c.page_tokens,
                       log2_of(c.page_tokens), slots + t0, m, k_out + t0 * row, v_out + t0 * row, (int)t0, status);
    }
    return e;
}

}  // namespace mt

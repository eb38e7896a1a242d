// The 4-bit cache of keys and values: rounding rows into slots and reading slots back.
//
// A row of head_dim elements becomes bias = min, scale = bf16((max - min) / 15) and codes rint((x - bias) / scale), with
// IEEE subtraction and division, so the stored bytes are a function of the row alone.  Both directions move
// (2 + 1/2) bytes per element and do a handful of operations on each, so they are bound by memory, and for a step's few
// tokens by the launch.  A row is one group of lanes, 16 bytes (8 elements) a lane: 8 lanes for head_dim 64, 16 for 128.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

struct CachePtrs {
    uint8_t* codes;
    uint32_t* params;       // (scale, bias) as two bf16
};

constexpr int kThreads = 256;

// Rows are numbered ((token * heads + head) * 2 + which), which = 0: keys, 1: values.
template <int D>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(CachePtrs kc, CachePtrs vc, int64_t n_slots, int page_shift, int heads,
                                                             KvRows k, KvRows v, const int64_t* __restrict__ slots, int n,
                                                             int32_t* status) {
    constexpr int L = D / 8;                     // lanes per row
    pdl_launch_dependents();
    pdl_wait();
    const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L;
    const int sub = threadIdx.x % L;
    const int64_t pair = row >> 1;
    const bool values = row & 1;
    const int64_t token = pair / heads;
    const int head = (int)(pair % heads);
    bool live = token < n;
    const int64_t slot = live ? slots[token] : -1;
    if (live && (slot < 0 || slot >= n_slots)) {
        if (slot != -1 && head == 0 && !values && sub == 0) raise_status(status, MT_ERR_INVALID_ARG, (int)token);
        live = false;
    }
    uint4 w = make_uint4(0, 0, 0, 0);
    const KvRows& src = values ? v : k;
    if (live) w = __ldg(reinterpret_cast<const uint4*>(src.p + token * src.token_stride + head * src.head_stride + sub * 8));
    const float x[8] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
    float lo = x[0], hi = x[0];
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        finite = finite && fabsf(x[i]) < INFINITY;
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        finite = __shfl_xor_sync(0xffffffffu, (int)finite, o) && finite;
    }
    const float spread = hi - lo;
    finite = finite && spread < INFINITY;
    const uint16_t scale_b = finite ? f_to_bf16(__fdiv_rn(spread, 15.f)) : uint16_t(0x7fff);
    const uint16_t bias_b = f_to_bf16(lo);       // exact: lo is an element
    const float scale = bf16_to_f(scale_b);
    uint32_t packed = 0;
    if (finite && scale > 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = fminf(rintf(__fdiv_rn(x[i] - lo, scale)), 15.f);
            packed |= (uint32_t)c << (4 * i);
        }
    }
    if (!live) return;
    const CachePtrs& dst = values ? vc : kc;
    const int64_t at = (((slot >> page_shift) * heads + head) << page_shift) + (slot & ((1 << page_shift) - 1));
    *reinterpret_cast<uint32_t*>(dst.codes + at * (D / 2) + sub * 4) = packed;
    if (sub == 0) dst.params[at] = (uint32_t)bias_b << 16 | scale_b;
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(CachePtrs kc, CachePtrs vc, int64_t n_slots, int page_shift, int heads,
                                                           const int64_t* __restrict__ slots, int n, uint16_t* __restrict__ k_out,
                                                           uint16_t* __restrict__ v_out, int32_t* status) {
    constexpr int L = D / 8;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L;
    const int sub = threadIdx.x % L;
    const int64_t pair = row >> 1;
    const bool values = row & 1;
    const int64_t token = pair / heads;
    const int head = (int)(pair % heads);
    if (token >= n) return;
    const int64_t slot = slots[token];
    uint4 w = make_uint4(0, 0, 0, 0);
    if (slot >= 0 && slot < n_slots) {
        const CachePtrs& src = values ? vc : kc;
        const int64_t at = (((slot >> page_shift) * heads + head) << page_shift) + (slot & ((1 << page_shift) - 1));
        const uint32_t p = src.params[at], c = *reinterpret_cast<const uint32_t*>(src.codes + at * (D / 2) + sub * 4);
        const float scale = bf16_lo(p), bias = bf16_hi(p);
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = pack_bf16x2(__fadd_rn(__fmul_rn((float)((c >> (8 * i)) & 15), scale), bias),
                               __fadd_rn(__fmul_rn((float)((c >> (8 * i + 4)) & 15), scale), bias));
        w = make_uint4(o[0], o[1], o[2], o[3]);
    } else if (slot != -1) {
        w = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
        if (head == 0 && !values && sub == 0) raise_status(status, MT_ERR_INVALID_ARG, (int)token);
    }
    *reinterpret_cast<uint4*>((values ? v_out : k_out) + pair * D + sub * 8) = w;
}

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

}  // namespace

cudaError_t launch_kv_append(const mt_kv_cache& c, const KvRows& k, const KvRows& v, const int64_t* slots, int n, int32_t* status,
                             cudaStream_t s) {
    const CachePtrs kc = {static_cast<uint8_t*>(c.k_codes), static_cast<uint32_t*>(c.k_params)};
    const CachePtrs vc = {static_cast<uint8_t*>(c.v_codes), static_cast<uint32_t*>(c.v_params)};
    const int64_t threads = (int64_t)n * c.kv_heads * 2 * (c.head_dim / 8), blocks = (threads + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_pdl(c.head_dim == 64 ? kv_append_kernel<64> : kv_append_kernel<128>, dim3((unsigned)blocks), dim3(kThreads), 0, s,
                      kc, vc, (int64_t)c.n_pages * c.page_tokens, log2_of(c.page_tokens), c.kv_heads, k, v, slots, n, status);
}

cudaError_t launch_kv_read(const mt_kv_cache& c, const int64_t* slots, int n, uint16_t* k_out, uint16_t* v_out, int32_t* status,
                           cudaStream_t s) {
    const CachePtrs kc = {static_cast<uint8_t*>(c.k_codes), static_cast<uint32_t*>(c.k_params)};
    const CachePtrs vc = {static_cast<uint8_t*>(c.v_codes), static_cast<uint32_t*>(c.v_params)};
    const int64_t threads = (int64_t)n * c.kv_heads * 2 * (c.head_dim / 8), blocks = (threads + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_pdl(c.head_dim == 64 ? kv_read_kernel<64> : kv_read_kernel<128>, dim3((unsigned)blocks), dim3(kThreads), 0, s, kc, vc,
                      (int64_t)c.n_pages * c.page_tokens, log2_of(c.page_tokens), c.kv_heads, slots, n, k_out, v_out, status);
}

}  // namespace mt

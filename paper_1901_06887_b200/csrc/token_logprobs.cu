// Log probability of given tokens, entropy, likeliest alternatives.  First form: one CTA per row, several passes.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

__device__ float logit(const LogprobArgs& a, int64_t row, int i) {
    const int64_t at = row * a.row_stride + i;
    return (a.fp32 ? static_cast<const float*>(a.logits)[at] : bf16_to_f(static_cast<const uint16_t*>(a.logits)[at])) + 0.f;
}
// Grows with (value, lower index).
__device__ unsigned long long rank_key(float x, int i) {
    const int b = __float_as_int(x);
    return (unsigned long long)((uint32_t)(b ^ ((b >> 31) & 0x7fffffff)) ^ 0x80000000u) << 32 | (uint32_t)(~i);
}

__global__ void __launch_bounds__(256) token_logprobs_simple(LogprobArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float red[2][8];
    __shared__ int bad_row;
    __shared__ unsigned long long best[8], chosen;
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x, lane = t & 31, w = t / 32;
    if (t == 0) bad_row = 0;
    __syncthreads();
    float m = -INFINITY;
    bool bad = false;
    for (int i = t; i < a.vocab; i += 256) { const float x = logit(a, row, i); bad = bad || !(x < INFINITY); m = fmaxf(m, x); }
    if (bad) bad_row = 1;
    m = warp_max(m);
    if (lane == 0) red[0][w] = m;
    __syncthreads();
    for (int i = 0; i < 8; ++i) m = fmaxf(m, red[0][i]);
    const bool none = bad_row || m == -INFINITY;
    __syncthreads();
    float s = 0.f, e = 0.f;
    for (int i = t; i < a.vocab && !none; i += 256) {
        const float z = logit(a, row, i) - m, p = expf(z);
        s += p;
        if (p > 0.f) e += p * z;
    }
    s = warp_sum(s); e = warp_sum(e);
    if (lane == 0) { red[0][w] = s; red[1][w] = e; }
    __syncthreads();
    s = e = 0.f;
    for (int i = 0; i < 8; ++i) { s += red[0][i]; e += red[1][i]; }
    const float ls = logf(s);
    if (t == 0) {
        const int tok = a.tokens[row];
        const bool in = tok >= 0 && tok < a.vocab;
        a.logprobs[row] = none || !in ? nan_f() : logit(a, row, tok) - m - ls;
        if (a.entropies) a.entropies[row] = none ? nan_f() : ls - e / s;
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        unsigned long long b = 0;
        for (int i = t; i < a.vocab && !none; i += 256) {
            const float x = logit(a, row, i);
            const unsigned long long key = rank_key(x, i);
            if (x > -INFINITY && key < last && key > b) b = key;
        }
        for (int o = 16; o; o >>= 1) { const unsigned long long y = __shfl_xor_sync(0xffffffffu, b, o); b = y > b ? y : b; }
        if (lane == 0) best[w] = b;
        __syncthreads();
        if (t == 0) {
            for (int i = 0; i < 8; ++i) b = best[i] > b ? best[i] : b;
            chosen = b;
            const int id = b ? (int)~(uint32_t)b : -1;
            a.top_ids[row * a.top + k] = id;
            a.top_logprobs[row * a.top + k] = none ? nan_f() : id < 0 ? -INFINITY : logit(a, row, id) - m - ls;
        }
        __syncthreads();
        last = chosen;
    }
}

}  // namespace

cudaError_t configure_token_logprobs() { return cudaSuccess; }

mt_status launch_token_logprobs(const LogprobArgs& a, const OpContext&, cudaStream_t s) {
    return launch_pdl(token_logprobs_simple, dim3((unsigned)a.n), dim3(256), 0, s, a) == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

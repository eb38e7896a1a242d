// Causal attention over packed prompts.  First form: one warp per (token, head), online softmax, fp32.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

__device__ int find_seq(const int32_t* offsets, int n_seqs, int tok) {
    for (int s = 0; s < n_seqs; ++s)
        if (offsets[s] <= tok && tok < offsets[s + 1]) return s;
    return -1;
}

template <int D>
__global__ void prompt_simple(PromptArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int warp = (blockIdx.x * blockDim.x + threadIdx.x) / 32, lane = threadIdx.x & 31;
    const int tok = warp / a.d.q_heads, h = warp % a.d.q_heads;
    if (warp == 0 && lane == 0)
        for (int i = 0; i < a.d.n_seqs; ++i)
            if (a.offsets[i] < 0 || a.offsets[i + 1] < a.offsets[i] || a.offsets[i + 1] > a.d.n_tokens)
                raise_status(a.status, MT_ERR_INVALID_ARG, i);
    if (tok >= a.d.n_tokens) return;
    const int s = find_seq(a.offsets, a.d.n_seqs, tok);
    if (s < 0) return;
    const int lo = a.offsets[s];
    if (lo < 0 || a.offsets[s + 1] > a.d.n_tokens) return;
    const int hk = h / (a.d.q_heads / a.d.kv_heads);
    constexpr int E = D / 32;
    float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) q[e] = bf16_to_f(a.q[tok * a.d.q_token_stride + h * a.d.q_head_stride + lane + 32 * e]) * a.d.scale;
    for (int j = lo; j <= tok; ++j) {
        float x = 0.f;
        for (int e = 0; e < E; ++e) x += q[e] * bf16_to_f(a.k[j * a.d.k_token_stride + hk * a.d.k_head_stride + lane + 32 * e]);
        x = warp_sum(x);
        const float mn = fmaxf(m, x), c = (m == mn) ? 1.f : __expf(m - mn), p = __expf(x - mn);
        for (int e = 0; e < E; ++e)
            o[e] = o[e] * c + p * bf16_to_f(a.v[j * a.d.v_token_stride + hk * a.d.v_head_stride + lane + 32 * e]);
        l = l * c + p;
        m = mn;
    }
    for (int e = 0; e < E; ++e)
        a.out[((int64_t)tok * a.d.q_heads + h) * D + lane + 32 * e] = f_to_bf16(o[e] / l);
}

}  // namespace

cudaError_t configure_prompt_attention() { return cudaSuccess; }

mt_status launch_prompt_attention(const PromptArgs& a, const OpContext&, cudaStream_t s) {
    const int64_t warps = (int64_t)a.d.n_tokens * a.d.q_heads;
    const dim3 grid((unsigned)((warps + 7) / 8));
    const cudaError_t e = a.d.head_dim == 64 ? launch_pdl(prompt_simple<64>, grid, dim3(256), 0, s, a)
                                             : launch_pdl(prompt_simple<128>, grid, dim3(256), 0, s, a);
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

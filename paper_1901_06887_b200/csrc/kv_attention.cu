// Attention of one new token per sequence over the paged 4-bit cache.  First form: one warp per (sequence, head).
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

template <int D>
__global__ void kv_attention_simple(KvAttentionArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int warp = (blockIdx.x * blockDim.x + threadIdx.x) / 32, lane = threadIdx.x & 31;
    const int s = warp / a.q_heads, h = warp % a.q_heads;
    if (s >= a.n_seqs) return;
    const int P = a.c.page_tokens, H = a.c.kv_heads, hk = h / (a.q_heads / H), len = a.lengths[s];
    bool bad = len < 0 || (int64_t)len > (int64_t)a.table_width * P;
    constexpr int E = D / 32;                  // lane owns elements E * lane ..
    float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) q[e] = bf16_to_f(a.q[s * a.q_seq_stride + h * a.q_head_stride + lane * E + e]) * a.scale;
    const uint8_t *kc = (const uint8_t*)a.c.k_codes, *vc = (const uint8_t*)a.c.v_codes;
    const uint32_t *kp = (const uint32_t*)a.c.k_params, *vp = (const uint32_t*)a.c.v_params;
    for (int j = 0; j < len && !bad; ++j) {
        const int page = a.tables[(int64_t)s * a.table_width + j / P];
        if (page < 0 || page >= a.c.n_pages) { bad = true; break; }
        const int64_t at = ((int64_t)page * H + hk) * P + j % P;
        const uint32_t kq = kp[at], vq = vp[at];
        float x = 0.f;
        for (int e = 0; e < E; ++e) {
            const int d = lane * E + e;
            const int c = (kc[at * (D / 2) + d / 2] >> (4 * (d & 1))) & 15;
            x += q[e] * (c * bf16_lo(kq) + bf16_hi(kq));
        }
        x = warp_sum(x);
        const float mn = fmaxf(m, x), f = (m == mn) ? 1.f : __expf(m - mn), p = __expf(x - mn);
        for (int e = 0; e < E; ++e) {
            const int d = lane * E + e;
            const int c = (vc[at * (D / 2) + d / 2] >> (4 * (d & 1))) & 15;
            o[e] = o[e] * f + p * (c * bf16_lo(vq) + bf16_hi(vq));
        }
        l = l * f + p;
        m = mn;
    }
    if (bad && lane == 0) raise_status(a.status, MT_ERR_INVALID_ARG, s);
    for (int e = 0; e < E; ++e)
        a.out[((int64_t)s * a.q_heads + h) * D + lane * E + e] = f_to_bf16(bad ? nan_f() : len == 0 ? 0.f : o[e] / l);
}

}  // namespace

cudaError_t configure_kv_attention() { return cudaSuccess; }

mt_status launch_kv_attention(const KvAttentionArgs& a, const OpContext&, cudaStream_t s) {
    const int64_t warps = (int64_t)a.n_seqs * a.q_heads;
    const cudaError_t e = launch_pdl(a.c.head_dim == 64 ? kv_attention_simple<64> : kv_attention_simple<128>,
                                     dim3((unsigned)((warps + 3) / 4)), dim3(128), 0, s, a);
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

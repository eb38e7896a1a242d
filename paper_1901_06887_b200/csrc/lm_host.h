// Launchers of the language-model operators (prompt_attention.cu, kv_cache.cu, kv_attention.cu, quant_linear.cu,
// token_logprobs.cu), called by lm_api.cu after it has checked the arguments.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mt_host.h"

namespace mt {

struct PromptArgs {
    mt_prompt_desc d;
    const uint16_t *q, *k, *v;
    const int32_t* offsets;
    uint16_t* out;
    OpStatus status;
};
cudaError_t configure_prompt_attention();
mt_status launch_prompt_attention(const PromptArgs& a, const OpContext& c, cudaStream_t s);

struct KvRows {                     // rows [n][heads][head_dim] bf16 with strides in elements
    const uint16_t* p;
    int64_t token_stride, head_stride;
};
cudaError_t launch_kv_append(const mt_kv_cache& c, const KvRows& k, const KvRows& v, const int64_t* slots, int n,
                             const OpStatus& status, int sm_count, cudaStream_t s);
cudaError_t launch_kv_read(const mt_kv_cache& c, const int64_t* slots, int n, uint16_t* k_out, uint16_t* v_out,
                           const OpStatus& status, int sm_count, cudaStream_t s);

struct KvAttentionArgs {
    mt_kv_cache c;
    const uint16_t* q;
    int64_t q_seq_stride, q_head_stride;
    const int32_t* tables;
    int table_width;
    const int32_t* lengths;
    int n_seqs, q_heads;
    float scale;
    uint16_t* out;
    OpStatus status;
};
cudaError_t configure_kv_attention();
mt_status launch_kv_attention(const KvAttentionArgs& a, const OpContext& c, cudaStream_t s);

// Packed 4-bit weights of one tenant: tiles of 16 output rows; per tile the codes of its K / 64 blocks (512 bytes each,
// 16 bytes per lane of a warp), all tiles' codes first; then per tile and group of inputs 16 scales (32 bytes).
// Lane 4 g + t of a block holds rows g (words 0, 1) and g + 8 (words 2, 3); the first word of a row holds inputs 8 t .. 8 t + 7,
// the second inputs 32 + 8 t .. 32 + 8 t + 7; input 2 p of a word sits in nibble p, input 2 p + 1 in nibble p + 4.  So
// (w >> 4 p) & 0x000f000f is a pair of neighbouring inputs in the two halves of a register, the form the matrix instruction
// wants, and a block's first 32 inputs and last 32 inputs meet in different instructions (groups of 32 stay apart).
// A group's 32 bytes hold the scales of rows g and g + 8 side by side.
__host__ __device__ inline size_t quant_codes_bytes(int K, int N) { return (size_t)((N + 15) / 16) * (size_t)(K / 64) * 512; }
__host__ __device__ inline size_t quant_tenant_bytes(int K, int N, int group) {
    return quant_codes_bytes(K, N) + (size_t)((N + 15) / 16) * (size_t)(K / group) * 32;
}
cudaError_t launch_quant_pack(const uint8_t* codes, const uint16_t* scales, int tenants, int K, int N, int group, void* packed,
                              cudaStream_t s);
struct QuantLinearArgs {
    int tenants, K, N, group;
    const uint8_t* packed;
    const float* bias;
    const uint16_t* x;
    int64_t x_stride;
    const int32_t* ids;
    int n;
    int row0;                       // index of ids[0] in the caller's batch (for the sticky status)
    void* y;
    int64_t y_stride;
    int y_fp32;
    OpStatus status;
    // filled in by the launcher: bytes of a tenant's codes and of all it has; groups per row; tiles of 16 outputs; floor((2^32 - 1) / d) for d blocks per group, with which the high word of
    // (n + 1) times it is n / d for (n + 1) d < 2^32
    size_t codes_bytes, tenant_bytes;
    int groups, tiles;
    uint32_t per_magic;
};
cudaError_t configure_quant_linear();
cudaError_t launch_quant_linear(const QuantLinearArgs& a, int sm_count, cudaStream_t s);
constexpr int kQuantRowsPerLaunch = 256;

struct LogprobArgs {
    const void* logits;
    int fp32;
    int64_t row_stride;
    int n, vocab;
    const int32_t* tokens;
    int top;
    float *logprobs, *entropies;
    int32_t* top_ids;
    float* top_logprobs;
};
cudaError_t configure_token_logprobs();
mt_status launch_token_logprobs(const LogprobArgs& a, const OpContext& c, cudaStream_t s);

// Scratch of at least `bytes` (256-byte aligned, contents left over from earlier calls) for work on stream `s`: the stream's, or the
// graph's that `s` is captured into.  (Mutex held.)
mt_status op_scratch(cudaStream_t s, size_t bytes, uint8_t** out);

}  // namespace mt

// C-ABI layer of the language-model operators: checks of arguments, per-stream scratch, launches.  Everything that
// computes is in the kernels of the other files.
#include <cuda_runtime.h>

#include <atomic>
#include <climits>
#include <cmath>
#include <new>

#include "../../include/mt.h"
#include "lm_host.h"
#include "mt_host.h"

namespace {

using namespace mt;

// Scratch belongs to a stream: calls on one stream are in order, so one block serves all of them, and calls on different
// streams never share one.  A stream is known by its id, not by its handle: the handle of the per-thread default stream stands
// for one stream per thread, and a destroyed stream's handle may come back while its last call still runs.
struct Scratch {
    unsigned long long stream;
    uint64_t used;              // call that used it last
    uint8_t* block;
    size_t bytes;
};
constexpr int kMaxStreams = 64;
Scratch g_scratch[kMaxStreams];
int g_n_scratch = 0;
uint64_t g_scratch_calls = 0;

// A captured call's scratch belongs to the graph, which may be replayed on any stream: one block per stream of a capture, given
// back when the graph and its instances are gone (a user object of the graph says so, on a thread of CUDA's).
struct GraphBlock {
    std::atomic<int> owners;    // this list, and a graph
    unsigned long long capture;
    const void* stream;
    uint8_t* block;
    size_t bytes;
    GraphBlock* next;
};
GraphBlock* g_graph_blocks = nullptr;

void give_up(GraphBlock* b) {
    if (b->owners.fetch_sub(1) == 1) delete b;
}
void CUDART_CB graph_is_gone(void* b) { give_up(static_cast<GraphBlock*>(b)); }

// Allocating is no part of any capture, this thread's or another's.
struct OutsideCaptures {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    OutsideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode); }
    ~OutsideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode); }
};

bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
bool bad_stride(int64_t s, int64_t least) { return s < least || (s & 7) != 0 || s >= (int64_t(1) << 36); }

mt_status to_status(cudaError_t e) {
    return e == cudaSuccess ? MT_OK : e == cudaErrorMemoryAllocation ? MT_ERR_OOM : MT_ERR_CUDA;
}

mt_status check_cache(const mt_kv_cache* c) {
    if (!c || c->n_pages < 0 || c->kv_heads <= 0) return MT_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return MT_ERR_UNSUPPORTED;
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return MT_ERR_UNSUPPORTED;
    if (c->kv_heads > 65535) return MT_ERR_UNSUPPORTED;
    if (c->n_pages > 0 && (!c->k_codes || !c->k_params || !c->v_codes || !c->v_params)) return MT_ERR_INVALID_ARG;
    if (misaligned(c->k_codes) || misaligned(c->k_params) || misaligned(c->v_codes) || misaligned(c->v_params))
        return MT_ERR_INVALID_ARG;
    return MT_OK;
}

mt_status check_quant(int K, int N, int group) {
    if (K <= 0 || N <= 0 || group <= 0) return MT_ERR_INVALID_ARG;
    if (N > INT_MAX - (1 << 20)) return MT_ERR_UNSUPPORTED;         // the kernels round N up, and step past it
    if (K >= (1 << 22) || K % 64 || K % group || !(group == 32 || group % 64 == 0)) return MT_ERR_UNSUPPORTED;
    return MT_OK;
}

}  // namespace

namespace mt {

static mt_status allocate(size_t bytes, size_t least, uint8_t** out, size_t* got) {
    OutsideCaptures mode;
    void* p = nullptr;
    cudaError_t err = cudaMalloc(&p, bytes);
    if (err == cudaErrorMemoryAllocation && bytes > least) {
        cudaGetLastError();
        err = cudaMalloc(&p, bytes = least);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return to_status(err); }
    *out = static_cast<uint8_t*>(p);
    *got = bytes;
    return MT_OK;
}

static mt_status graph_scratch(unsigned long long capture, const void* stream, cudaGraph_t graph, size_t bytes, uint8_t** out) {
    GraphBlock* b = nullptr;
    for (GraphBlock* x = g_graph_blocks; x; x = x->next) {
        const bool taken = x->owners.load() > 1;
        if (x->bytes < bytes) continue;
        if (taken && x->capture == capture && x->stream == stream) { *out = x->block; return MT_OK; }
        if (!taken && (!b || x->bytes < b->bytes)) b = x;
    }
    if (!b) {
        uint8_t* block;
        size_t got;
        const mt_status st = allocate((bytes + 0xfffff) & ~size_t(0xfffff), bytes, &block, &got);
        if (st != MT_OK) return st;
        b = new (std::nothrow) GraphBlock{{1}, 0, nullptr, block, got, g_graph_blocks};
        if (!b) { OutsideCaptures mode; cudaFree(block); return MT_ERR_OOM; }
        g_graph_blocks = b;
    }
    cudaUserObject_t owner;
    cudaError_t e = cudaUserObjectCreate(&owner, b, graph_is_gone, 1, cudaUserObjectNoDestructorSync);
    if (e != cudaSuccess) { cudaGetLastError(); return to_status(e); }
    b->capture = capture;
    b->stream = stream;
    b->owners.fetch_add(1);
    e = cudaGraphRetainUserObject(graph, owner, 1, cudaGraphUserObjectMove);
    if (e != cudaSuccess) { cudaGetLastError(); cudaUserObjectRelease(owner, 1); return to_status(e); }
    *out = b->block;
    return MT_OK;
}

mt_status op_scratch(cudaStream_t s, size_t bytes, uint8_t** out) {
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    unsigned long long capture = 0, id = ~0ull;
    cudaGraph_t graph = nullptr;
    cudaError_t err = cudaSuccess;
    const bool legacy = s == nullptr || s == cudaStreamLegacy;      // one stream, never captured: asking would cost a step 0.4 us
    if (!legacy) err = cudaStreamGetCaptureInfo(s, &capturing, &capture, &graph);
    if (err == cudaSuccess && capturing != cudaStreamCaptureStatusNone) {       // (the id of a capturing stream must not be asked for)
        if (capturing != cudaStreamCaptureStatusActive) return MT_ERR_CUDA;
        static thread_local char this_thread;
        return graph_scratch(capture, s == cudaStreamPerThread ? static_cast<const void*>(&this_thread) : s, graph, bytes, out);
    }
    if (err == cudaSuccess && !legacy) err = cudaStreamGetId(s, &id);
    if (err != cudaSuccess) { cudaGetLastError(); return to_status(err); }

    Scratch *e = nullptr, *oldest = g_scratch;
    for (int i = 0; i < g_n_scratch && !e; ++i) {
        if (g_scratch[i].stream == id) e = &g_scratch[i];
        if (g_scratch[i].used < oldest->used) oldest = &g_scratch[i];
    }
    if (!e && g_n_scratch == kMaxStreams) {       // another stream's block, once nothing can be using it
        OutsideCaptures mode;
        err = cudaDeviceSynchronize();
        if (err != cudaSuccess) { cudaGetLastError(); return to_status(err); }
        e = oldest;
        e->stream = id;
    }
    if (!e || e->bytes < bytes) {
        size_t want = e ? 2 * e->bytes : (16u << 20), got;
        if (want < bytes) want = bytes;
        uint8_t* block;
        const mt_status st = allocate(want, bytes, &block, &got);
        if (st != MT_OK) return st;
        if (e) {
            OutsideCaptures mode;
            cudaStreamSynchronize(s);             // calls in flight read the block that goes
            cudaFree(e->block);
        } else {
            e = &g_scratch[g_n_scratch++];
            e->stream = id;
        }
        e->block = block;
        e->bytes = got;
    }
    e->used = ++g_scratch_calls;
    *out = e->block;
    return MT_OK;
}

void op_free_scratch() {
    for (int i = 0; i < g_n_scratch; ++i) cudaFree(g_scratch[i].block);
    g_n_scratch = 0;
    for (GraphBlock* b = g_graph_blocks; b;) {
        GraphBlock* const next = b->next;
        cudaFree(b->block);
        give_up(b);
        b = next;
    }
    g_graph_blocks = nullptr;
}

cudaError_t configure_operators() {
    cudaError_t e = configure_prompt_attention();
    if (e == cudaSuccess) e = configure_kv_attention();
    if (e == cudaSuccess) e = configure_quant_linear();
    if (e == cudaSuccess) e = configure_token_logprobs();
    return e;
}

}  // namespace mt

extern "C" {

mt_status mt_prompt_attention(const mt_prompt_desc* d, const void* q, const void* k, const void* v, const int32_t* offsets,
                              void* out, void* stream) {
    if (!d || d->n_tokens < 0 || d->n_seqs < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || !std::isfinite(d->scale)) return MT_ERR_INVALID_ARG;
    if (!(d->head_dim == 64 || d->head_dim == 128) || d->q_heads % d->kv_heads || d->q_heads > 65535) return MT_ERR_UNSUPPORTED;
    if (d->n_tokens > (1 << 30)) return MT_ERR_UNSUPPORTED;
    const int64_t hd = d->head_dim;
    if (bad_stride(d->q_token_stride, hd) || bad_stride(d->k_token_stride, hd) || bad_stride(d->v_token_stride, hd) ||
        bad_stride(d->q_head_stride, hd) || bad_stride(d->k_head_stride, hd) || bad_stride(d->v_head_stride, hd))
        return MT_ERR_UNSUPPORTED;
    std::unique_lock<std::mutex> lk;
    OpContext c;
    mt_status st = op_begin(&lk, &c);
    if (st != MT_OK) return st;
    if (d->n_tokens == 0 || d->n_seqs == 0) return MT_OK;
    if (!q || !k || !v || !offsets || !out) return MT_ERR_INVALID_ARG;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(offsets, 4)) return MT_ERR_INVALID_ARG;
    PromptArgs a;
    a.d = *d;
    a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
    a.offsets = offsets; a.out = static_cast<uint16_t*>(out); a.status = c.status;
    return launch_prompt_attention(a, c, static_cast<cudaStream_t>(stream));
}

mt_status mt_kv_append(const mt_kv_cache* cache, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                       int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots, int32_t n, void* stream) {
    mt_status st = check_cache(cache);
    if (st != MT_OK) return st;
    if (n < 0) return MT_ERR_INVALID_ARG;
    if (bad_stride(k_token_stride, 0) || bad_stride(k_head_stride, 0) || bad_stride(v_token_stride, 0) || bad_stride(v_head_stride, 0))
        return MT_ERR_UNSUPPORTED;
    std::unique_lock<std::mutex> lk;
    OpContext c;
    st = op_begin(&lk, &c);
    if (st != MT_OK || n == 0) return st;
    if (!k || !v || !slots || misaligned(k) || misaligned(v) || misaligned(slots, 8)) return MT_ERR_INVALID_ARG;
    const KvRows kr = {static_cast<const uint16_t*>(k), k_token_stride, k_head_stride};
    const KvRows vr = {static_cast<const uint16_t*>(v), v_token_stride, v_head_stride};
    return to_status(launch_kv_append(*cache, kr, vr, slots, n, c.status, c.sm_count, static_cast<cudaStream_t>(stream)));
}

mt_status mt_kv_read(const mt_kv_cache* cache, const int64_t* slots, int32_t n, void* k_out, void* v_out, void* stream) {
    mt_status st = check_cache(cache);
    if (st != MT_OK) return st;
    if (n < 0) return MT_ERR_INVALID_ARG;
    std::unique_lock<std::mutex> lk;
    OpContext c;
    st = op_begin(&lk, &c);
    if (st != MT_OK || n == 0) return st;
    if (!slots || !k_out || !v_out || misaligned(k_out) || misaligned(v_out) || misaligned(slots, 8)) return MT_ERR_INVALID_ARG;
    return to_status(launch_kv_read(*cache, slots, n, static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out), c.status,
                                    c.sm_count, static_cast<cudaStream_t>(stream)));
}

mt_status mt_kv_attention(const mt_kv_cache* cache, const void* q, int64_t q_seq_stride, int64_t q_head_stride,
                          const int32_t* tables, int32_t table_width, const int32_t* lengths, int32_t n_seqs, int32_t q_heads,
                          float scale, void* out, void* stream) {
    mt_status st = check_cache(cache);
    if (st != MT_OK) return st;
    if (n_seqs < 0 || q_heads <= 0 || table_width < 0 || !std::isfinite(scale)) return MT_ERR_INVALID_ARG;
    if (q_heads % cache->kv_heads || q_heads / cache->kv_heads > 16) return MT_ERR_UNSUPPORTED;
    if ((int64_t)n_seqs * cache->kv_heads >= (1 << 20) || (int64_t)table_width * cache->page_tokens > INT_MAX - 64) return MT_ERR_UNSUPPORTED;
    if (bad_stride(q_seq_stride, 0) || bad_stride(q_head_stride, 0)) return MT_ERR_UNSUPPORTED;
    std::unique_lock<std::mutex> lk;
    OpContext c;
    st = op_begin(&lk, &c);
    if (st != MT_OK || n_seqs == 0) return st;
    if (!q || !lengths || !out || (!tables && table_width > 0) || misaligned(q) || misaligned(out) || misaligned(tables, 4) ||
        misaligned(lengths, 4))
        return MT_ERR_INVALID_ARG;
    KvAttentionArgs a;
    a.c = *cache; a.q = static_cast<const uint16_t*>(q); a.q_seq_stride = q_seq_stride; a.q_head_stride = q_head_stride;
    a.tables = tables; a.table_width = table_width; a.lengths = lengths; a.n_seqs = n_seqs; a.q_heads = q_heads;
    a.scale = scale; a.out = static_cast<uint16_t*>(out); a.status = c.status;
    return launch_kv_attention(a, c, static_cast<cudaStream_t>(stream));
}

mt_status mt_quant_packed_bytes(int32_t in_features, int32_t out_features, int32_t group, size_t* bytes_out) {
    mt_status st = check_quant(in_features, out_features, group);
    if (st != MT_OK) return st;
    if (!bytes_out) return MT_ERR_INVALID_ARG;
    *bytes_out = quant_tenant_bytes(in_features, out_features, group);
    return MT_OK;
}

mt_status mt_quant_pack(const uint8_t* codes, const void* scales, int32_t tenants, int32_t in_features, int32_t out_features,
                        int32_t group, void* packed, void* stream) {
    mt_status st = check_quant(in_features, out_features, group);
    if (st != MT_OK) return st;
    if (tenants < 0) return MT_ERR_INVALID_ARG;
    std::unique_lock<std::mutex> lk;
    OpContext c;
    st = op_begin(&lk, &c);
    if (st != MT_OK || tenants == 0) return st;
    if (!codes || !scales || !packed || misaligned(packed) || misaligned(scales, 2)) return MT_ERR_INVALID_ARG;
    return to_status(launch_quant_pack(codes, static_cast<const uint16_t*>(scales), tenants, in_features, out_features, group, packed,
                                       static_cast<cudaStream_t>(stream)));
}

mt_status mt_quant_linear(const mt_quant_bank* b, const void* x, int64_t x_stride, const int32_t* ids, int32_t n, void* y,
                          int64_t y_stride, int32_t y_dtype, void* stream) {
    if (!b || b->tenants <= 0 || n < 0 || (y_dtype != MT_BF16 && y_dtype != MT_FP32)) return MT_ERR_INVALID_ARG;
    mt_status st = check_quant(b->in_features, b->out_features, b->group);
    if (st != MT_OK) return st;
    if (bad_stride(x_stride, 0) || y_stride < 0 || y_stride >= (int64_t(1) << 36)) return MT_ERR_UNSUPPORTED;
    if (n > 1 && y_stride < b->out_features) return MT_ERR_INVALID_ARG;
    std::unique_lock<std::mutex> lk;
    OpContext c;
    st = op_begin(&lk, &c);
    if (st != MT_OK || n == 0) return st;
    if (!x || !ids || !y || !b->packed || misaligned(x) || misaligned(b->packed) || misaligned(y, y_dtype == MT_FP32 ? 4 : 2) ||
        misaligned(ids, 4) || misaligned(b->bias, 4))
        return MT_ERR_INVALID_ARG;
    QuantLinearArgs a;
    a.tenants = b->tenants; a.K = b->in_features; a.N = b->out_features; a.group = b->group;
    a.packed = static_cast<const uint8_t*>(b->packed); a.bias = b->bias;
    a.x_stride = x_stride; a.y_stride = y_stride; a.y_fp32 = y_dtype == MT_FP32; a.status = c.status;
    for (int row0 = 0; row0 < n; row0 += kQuantRowsPerLaunch) {
        a.n = n - row0 < kQuantRowsPerLaunch ? n - row0 : kQuantRowsPerLaunch;
        a.row0 = row0;
        a.x = static_cast<const uint16_t*>(x) + (size_t)row0 * (size_t)x_stride;
        a.ids = ids + row0;
        a.y = static_cast<uint8_t*>(y) + (size_t)row0 * (size_t)y_stride * (a.y_fp32 ? 4 : 2);
        st = to_status(launch_quant_linear(a, c.sm_count, static_cast<cudaStream_t>(stream)));
        if (st != MT_OK) return st;
        if (n - row0 <= kQuantRowsPerLaunch) break;      // row0 may not pass INT_MAX
    }
    return MT_OK;
}

mt_status mt_token_logprobs(const void* logits, int32_t dtype, int64_t row_stride, int32_t n, int32_t vocab, const int32_t* tokens,
                            int32_t top, float* logprobs, float* entropies, int32_t* top_ids, float* top_logprobs, void* stream) {
    if (n < 0 || vocab <= 0 || top < 0 || (dtype != MT_BF16 && dtype != MT_FP32)) return MT_ERR_INVALID_ARG;
    if (top > 32 || vocab >= (1 << 30) || row_stride < 0 || row_stride >= (int64_t(1) << 36)) return MT_ERR_UNSUPPORTED;
    std::unique_lock<std::mutex> lk;
    OpContext c;
    mt_status st = op_begin(&lk, &c);
    if (st != MT_OK || n == 0) return st;
    if (!logits || !tokens || !logprobs || (top > 0 && (!top_ids || !top_logprobs))) return MT_ERR_INVALID_ARG;
    if (misaligned(logits, dtype == MT_FP32 ? 4 : 2) || misaligned(tokens, 4) || misaligned(logprobs, 4) || misaligned(entropies, 4) ||
        misaligned(top_ids, 4) || misaligned(top_logprobs, 4))
        return MT_ERR_INVALID_ARG;
    LogprobArgs a;
    a.logits = logits; a.fp32 = dtype == MT_FP32; a.row_stride = row_stride; a.n = n; a.vocab = vocab; a.tokens = tokens; a.top = top;
    a.logprobs = logprobs; a.entropies = entropies; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    return launch_token_logprobs(a, c, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

// Log probability of given tokens, entropy and the likeliest alternatives of rows of logits.
//
// Mathematics.  With m = max x, S = sum e^(x - m), W = sum (x - m) e^(x - m):  log p_t = x_t - m - log S,  entropy = log S - W / S.
// One pass over the logits: every thread keeps (m, S, W) of its share, rescaled when its maximum moves.
//
// Alternatives.  The pass also leaves the largest logit of each thread and of each group of four.  The k-th largest of the 64 groups' is a bound
// that the k-th largest logit cannot lie below, so only the shares that reach it are looked at again (from L2, a warp at a time) and what reaches it is put on
// a list; it holds little more than k entries.  The list is ranked by counting, every entry against every other, on (value, lower index first), so the result
// does not depend on the order of arrival.  Where too many logits reach the bound (long ties, values sorted into one share) the exact k-th
// largest is found by its bits, eight at a time, from histograms of the row, and ties at it are taken from the front of the row.
//
// Split.  Few long rows are cut into 2, 4 or 8 parts, one CTA each, that form a cluster: the first joins the others' statistics and sorted
// alternatives out of their shared memory (a part leaves at most kMaxTop of them).  Joining through device memory and a counter instead cost a
// fence, an atomic and three more round trips, some 10 us for 8 rows of 32000.  A part whose logits fit in registers is not read a second time.
// Minus infinity adds nothing and is no alternative.
//
// Cost.  Many rows: 2000 rows of 128 000 in bf16 take 106 us alone and 116 among others, 1.4 to 1.5 times their bytes.  No unit is full
// (exponentials 57 %, issue slots 59 %, memory 50 %): a CTA takes one row, six fit an SM, so a last partial wave runs nearly alone (2.25 waves here),
// and the selection stands behind each row.  Few rows: latency of pass, selection and join.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxTop = 32;
constexpr int kGroups = 64;                // at least kMaxTop
constexpr int kList = 1024;                // entries the first list may take
constexpr int kMinPart = 2048;             // logits of a part, at least
constexpr int kMaxParts = 8;
constexpr int kHold = 4;                   // vectors of a thread that stay in registers
constexpr float kLog2e = 1.44269504088896341f;
static_assert(kThreads == 4 * kGroups && kGroups >= kMaxTop && kThreads >= kMaxParts * kMaxTop, "");

struct Params {
    LogprobArgs a;
    int parts;                             // CTAs of a cluster
    int part_len;                          // a multiple of 8
};

// Bits that grow with the value (minus zero counts as zero); 0 is below every number, so it can stand for "nothing".
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
constexpr uint32_t kOrderedMinusInf = 0x007fffffu;         // ordered(-inf)

// Sixteen bytes of logits.
template <bool FP32> struct Vec;
template <> struct Vec<true> {
    static constexpr int N = 4;
    uint4 v;
    __device__ __forceinline__ float operator[](int e) const { return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w); }
    __device__ __forceinline__ float max_nan() const {          // NaN if any is
        float m = __uint_as_float(v.x);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(__uint_as_float(v.y)));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(__uint_as_float(v.z)));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(__uint_as_float(v.w)));
        return m;
    }
};
template <> struct Vec<false> {
    static constexpr int N = 8;
    uint4 v;
    __device__ __forceinline__ float operator[](int e) const {
        const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        return e & 1 ? bf16_hi(w) : bf16_lo(w);
    }
    __device__ __forceinline__ float max_nan() const {          // two at a time
        uint32_t m = v.x;
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.y));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.z));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.w));
        float a = bf16_lo(m);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(bf16_hi(m)));
        return a;
    }
};
template <bool FP32>
__device__ __forceinline__ float logit_at(const void* row, int i) {
    return FP32 ? static_cast<const float*>(row)[i] : bf16_to_f(static_cast<const uint16_t*>(row)[i]);
}

// A part of a row, [lo, hi): elements in front of the first 16-byte boundary, whole vectors, the rest.
struct Span {
    int lo, hi, vec0, n_vec, tail;         // vectors start at vec0; tail: first element behind them
};
template <bool FP32>
__device__ __forceinline__ Span span_of(const void* row, int lo, int hi) {
    constexpr int N = Vec<FP32>::N, B = FP32 ? 4 : 2;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row) + (uintptr_t)lo * B;
    Span s;
    s.lo = lo; s.hi = hi;
    s.vec0 = min(hi, lo + (int)(((16 - (at & 15)) & 15) / B));
    s.n_vec = (hi - s.vec0) / N;
    s.tail = s.vec0 + s.n_vec * N;
    return s;
}
// Calls f(value, index) for every element of this thread's share; the same share in every pass.
template <bool FP32, class F>
__device__ __forceinline__ void for_share(const void* row, const Span& s, int t, F f) {
    constexpr int N = Vec<FP32>::N, B = FP32 ? 4 : 2;
    for (int v = t; v < s.n_vec; v += kThreads) {
        Vec<FP32> x;
        x.v = *reinterpret_cast<const uint4*>(static_cast<const char*>(row) + (size_t)(s.vec0 + v * N) * B);
#pragma unroll
        for (int e = 0; e < N; ++e) f(x[e], s.vec0 + v * N + e);
    }
    if (t < s.vec0 - s.lo) f(logit_at<FP32>(row, s.lo + t), s.lo + t);
    if (t < s.hi - s.tail) f(logit_at<FP32>(row, s.tail + t), s.tail + t);
}

// The same for ANOTHER thread's share (thread `of` of this part), by a whole warp at once.
template <bool FP32, class F>
__device__ __forceinline__ void for_share_of(const void* row, const Span& s, int of, int lane, F f) {
    constexpr int N = Vec<FP32>::N, B = FP32 ? 4 : 2;
    for (int v = of + lane * kThreads; v < s.n_vec; v += 32 * kThreads) {
        Vec<FP32> x;
        x.v = *reinterpret_cast<const uint4*>(static_cast<const char*>(row) + (size_t)(s.vec0 + v * N) * B);
#pragma unroll
        for (int e = 0; e < N; ++e) f(x[e], s.vec0 + v * N + e);
    }
    if (lane == 0 && of < s.vec0 - s.lo) f(logit_at<FP32>(row, s.lo + of), s.lo + of);
    if (lane == 1 && of < s.hi - s.tail) f(logit_at<FP32>(row, s.tail + of), s.tail + of);
}

struct Stats {
    float m, s, w;                         // s = sum e^(x - m), w = sum (x - m) e^(x - m)
};
__device__ __forceinline__ float exp_of(float x) { return ex2(x * kLog2e); }
// Moves sums to another maximum, not below the own.
__device__ __forceinline__ void move_to(Stats& a, float m) {
    const float d = fmaxf(a.m - m, -1e4f), f = exp_of(d);                   // (-1e4: far below, and finite)
    a.w = m > -INFINITY ? fmaf(d, a.s, a.w) * f : 0.f;
    a.s = m > -INFINITY ? a.s * f : 0.f;
    a.m = m;
}
// Joins the sums of 2^k neighbouring lanes.
template <int WIDTH>
__device__ __forceinline__ void join_lanes(Stats& a) {
    float m = a.m;
#pragma unroll
    for (int o = WIDTH / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    move_to(a, m);
#pragma unroll
    for (int o = WIDTH / 2; o; o >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
    }
}
__device__ __forceinline__ uint32_t remote_u32(const void* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}

// Sorts the list of n <= kList (value, index) entries by counting and writes the first `top` (value descending, index ascending).
__device__ __forceinline__ void rank_list(const uint32_t* value, const int32_t* index, int n, int top, uint32_t* out_value, int32_t* out_index, int t) {
    for (int i = t; i < n; i += kThreads) {
        const uint32_t v = value[i];
        const int32_t at = index[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += (value[j] > v || (value[j] == v && index[j] < at)) ? 1 : 0;
        if (rank < top) { out_value[rank] = v; out_index[rank] = at; }
    }
}

// HOLD: a part has at most kHold vectors a thread.
template <bool FP32, bool HOLD>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(const Params p) {
    __shared__ float s_m[kWarps], s_s[kWarps], s_w[kWarps];
    __shared__ int s_n, s_n_top;
    __shared__ Stats s_all;
    __shared__ uint32_t s_best[kGroups], s_bound, s_value[kList], s_top_value[kMaxTop], s_hist[256], s_pick[2];
    __shared__ int32_t s_index[kList], s_top_index[kMaxTop], s_warp_n[kWarps];
    const LogprobArgs& a = p.a;
    const int t = threadIdx.x, lane = t & 31, warp = t / 32, top = a.top;
    const int64_t row_i = blockIdx.x / p.parts;
    const int part = blockIdx.x % p.parts;
    pdl_launch_dependents();
    pdl_wait();
    const void* const row = static_cast<const char*>(a.logits) + row_i * a.row_stride * (FP32 ? 4 : 2);
    const int lo = min(a.vocab, part * p.part_len), hi = min(a.vocab, lo + p.part_len);
    const Span span = span_of<FP32>(row, lo, hi);
    if (t == 0) s_n = 0;

    // --- one pass: statistics and the share's largest logit
    constexpr int N = Vec<FP32>::N, B = FP32 ? 4 : 2;
    Stats st = {-INFINITY, 0.f, 0.f};
    float best = -INFINITY;
    bool bad = false;
    auto reach = [&](float mx) {               // false: nothing but minus infinity so far
        bad = bad || !(mx < INFINITY);
        best = fmaxf(best, mx);
        if (mx > st.m) {                       // the sums move to the new maximum
            const float d = fmaxf(st.m - mx, -1e4f), f = exp_of(d);
            st.w = fmaf(d, st.s, st.w) * f;
            st.s *= f;
            st.m = mx;
        }
        return st.m > -INFINITY;
    };
    auto add = [&](const Vec<FP32>& x) {
        if (!reach(x.max_nan())) return;
        const Pair m2 = pair_of(-st.m, -st.m), c2 = pair_of(kLog2e, kLog2e);
        Pair s2 = pair_of(0.f, 0.f), w2 = pair_of(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            float d0, d1, q0, q1;
            unpair(add2(pair_of(x[e], x[e + 1]), m2), d0, d1);
            const Pair d = pair_of(fmaxf(d0, -1e4f), fmaxf(d1, -1e4f));         // (minus infinity: q = 0, d finite)
            unpair(mul2(d, c2), q0, q1);
            const Pair q = pair_of(ex2(q0), ex2(q1));
            s2 = add2(s2, q);
            w2 = fma2(q, d, w2);
        }
        float y0, y1;
        unpair(s2, y0, y1);
        st.s += y0 + y1;
        unpair(w2, y0, y1);
        st.w += y0 + y1;
    };
    auto add_one = [&](float x) {
        if (!reach(x)) return;
        const float d = fmaxf(x - st.m, -1e4f), q = exp_of(d);
        st.s += q;
        st.w = fmaf(q, d, st.w);
    };
    // the given token's logit, long before it is needed
    float at_token = nan_f();
    if (part == 0 && t == 0) {
        const int tok = a.tokens[row_i];
        if (tok >= 0 && tok < a.vocab) at_token = logit_at<FP32>(row, tok);
    }
    Vec<FP32> held[HOLD ? kHold : 1];
    const uint4* const base = reinterpret_cast<const uint4*>(static_cast<const char*>(row) + (size_t)span.vec0 * B);
    if (HOLD) {
        constexpr uint32_t kNone = FP32 ? 0xff800000u : 0xff80ff80u;       // minus infinity, as often as it fits
#pragma unroll
        for (int u = 0; u < kHold; ++u) {
            held[u].v = make_uint4(kNone, kNone, kNone, kNone);
            if (t + u * kThreads < span.n_vec) held[u].v = __ldg(base + t + u * kThreads);
        }
#pragma unroll
        for (int u = 0; u < kHold; ++u) add(held[u]);
    } else {
        int v = t;
        for (; v + 3 * kThreads < span.n_vec; v += 4 * kThreads) {       // four loads in flight
            Vec<FP32> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u].v = __ldg(base + v + u * kThreads);
#pragma unroll
            for (int u = 0; u < 4; ++u) add(x[u]);
        }
        for (; v < span.n_vec; v += kThreads) {
            Vec<FP32> x;
            x.v = __ldg(base + v);
            add(x);
        }
    }
    const bool has_head = t < span.vec0 - span.lo, has_tail = t < span.hi - span.tail;
    if (has_head) add_one(logit_at<FP32>(row, span.lo + t));
    if (has_tail) add_one(logit_at<FP32>(row, span.tail + t));
    const uint32_t mine_best = ordered(best);
    {
        uint32_t g = max(mine_best, __shfl_xor_sync(0xffffffffu, mine_best, 1));
        g = max(g, __shfl_xor_sync(0xffffffffu, g, 2));
        if ((t & 3) == 0) s_best[t >> 2] = g;
    }
    join_lanes<32>(st);
    if (lane == 0) { s_m[warp] = st.m; s_s[warp] = st.s; s_w[warp] = st.w; }
    const int row_bad = __syncthreads_or(bad);

    // --- alternatives of this part
    int n_top = 0;
    if (top > 0) {
        // bound: the top-th largest of the groups' largest (by counting; where several are equal the run that covers place `top` decides)
        if (t < kGroups) {
            const uint32_t mine = s_best[t];
            int above = 0, same = 0;
#pragma unroll 8
            for (int j = 0; j < kGroups; ++j) { above += s_best[j] > mine; same += s_best[j] == mine; }
            if (above < top && above + same >= top) s_bound = mine;
        }
        __syncthreads();
        const uint32_t bound = max(s_bound, kOrderedMinusInf + 1u);
        auto take = [&](float x, int i) {
            const uint32_t o = ordered(x);
            if (o >= bound) {
                const int at = atomicAdd(&s_n, 1);
                if (at < kList) { s_value[at] = o; s_index[at] = i; }
            }
        };
        if (HOLD) {
            if (mine_best >= bound) {
#pragma unroll
                for (int u = 0; u < kHold; ++u)
#pragma unroll
                    for (int e = 0; e < N; ++e) take(held[u][e], span.vec0 + (t + u * kThreads) * N + e);
                if (has_head) take(logit_at<FP32>(row, span.lo + t), span.lo + t);
                if (has_tail) take(logit_at<FP32>(row, span.tail + t), span.tail + t);
            }
        } else {
            for (unsigned who = __ballot_sync(0xffffffffu, mine_best >= bound); who; who &= who - 1)
                for_share_of<FP32>(row, span, t - lane + __ffs(who) - 1, lane, take);
        }
        __syncthreads();
        int n = s_n;
        if (n > kList) {
            // the exact top-th largest value, from its bits, eight at a time
            uint32_t prefix = 0;
            int need = top;
            for (int shift = 24; shift >= 0; shift -= 8) {
                __syncthreads();
                s_hist[t] = 0;
                __syncthreads();
                for_share<FP32>(row, span, t, [&](float x, int) {
                    const uint32_t o = ordered(x);
                    if (o > kOrderedMinusInf && (shift == 24 || (o >> (shift + 8)) == (prefix >> (shift + 8)))) atomicAdd(&s_hist[(o >> shift) & 255u], 1u);
                });
                __syncthreads();
                if (t == 0) {
                    int digit = 255, left = need;
                    while (digit > 0 && (int)s_hist[digit] < left) left -= (int)s_hist[digit--];
                    s_pick[0] = (uint32_t)digit;
                    s_pick[1] = (uint32_t)left;
                }
                __syncthreads();
                prefix |= s_pick[0] << shift;
                need = (int)s_pick[1];
            }
            // what lies above it (fewer than top), then the first `need` that equal it, in order of the row
            if (t == 0) s_n = 0;
            __syncthreads();
            for_share<FP32>(row, span, t, [&](float x, int i) {
                const uint32_t o = ordered(x);
                if (o > prefix) {
                    const int at = atomicAdd(&s_n, 1);
                    if (at < kList) { s_value[at] = o; s_index[at] = i; }
                }
            });
            __syncthreads();
            n = s_n;
            for (int i0 = span.lo; i0 < span.hi && need > 0; i0 += kThreads) {
                const int i = i0 + t;
                const bool hit = i < span.hi && ordered(logit_at<FP32>(row, i)) == prefix;
                const unsigned mask = __ballot_sync(0xffffffffu, hit);
                if (lane == 0) s_warp_n[warp] = __popc(mask);
                __syncthreads();
                int before = 0, all = 0;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) { if (w < warp) before += s_warp_n[w]; all += s_warp_n[w]; }
                const int at = before + __popc(mask & ((1u << lane) - 1u));
                if (hit && at < need) { s_value[n + at] = prefix; s_index[n + at] = i; }
                const int took = min(all, need);
                n += took;
                need -= took;
                __syncthreads();
            }
        }
        n_top = min(n, top);
        rank_list(s_value, s_index, n, top, s_top_value, s_top_index, t);
    }
    __syncthreads();

    // --- statistics of the part, then of the row; all outputs come from the first warp of the row's first part
    Stats all = {-INFINITY, 0.f, 0.f};
    int none = row_bad;
    if (warp == 0) {
        if (lane < kWarps) all = {s_m[lane], s_s[lane], s_w[lane]};
        join_lanes<kWarps>(all);
        all.m = __shfl_sync(0xffffffffu, all.m, 0);
        all.s = __shfl_sync(0xffffffffu, all.s, 0);
        all.w = __shfl_sync(0xffffffffu, all.w, 0);
    }
    if (p.parts > 1) {
        // a NaN as the sum tells of a row that is not one
        if (t == 0) { s_all = all; if (row_bad) s_all.s = nan_f(); s_n_top = n_top; }
        cluster_sync_all();
        if (part == 0) {
            // everybody's alternatives: list b at b * top, sorted, what is missing as zeros
            const int b = top > 0 ? t / top : p.parts, k = top > 0 ? t - b * top : 0;
            uint32_t value = 0;
            int32_t index = -1;
            if (b < p.parts) {
                if (k < (int)remote_u32(&s_n_top, b)) {
                    value = remote_u32(&s_top_value[k], b);
                    index = (int32_t)remote_u32(&s_top_index[k], b);
                }
                s_value[t] = value;
                s_index[t] = index;
            }
            if (warp == 0) {
                all = {-INFINITY, 0.f, 0.f};
                if (lane < p.parts) {
                    all.m = __uint_as_float(remote_u32(&s_all.m, lane));
                    all.s = __uint_as_float(remote_u32(&s_all.s, lane));
                    all.w = __uint_as_float(remote_u32(&s_all.w, lane));
                }
                none = __any_sync(0xffffffffu, all.s != all.s);
                join_lanes<kMaxParts>(all);
                all.m = __shfl_sync(0xffffffffu, all.m, 0);
                all.s = __shfl_sync(0xffffffffu, all.s, 0);
                all.w = __shfl_sync(0xffffffffu, all.w, 0);
            }
            __syncthreads();
            // an entry's rank: what stands before it in the lists of lower parts (an equal value there has a lower index) and of higher ones
            int rank = kMaxTop;
            if (value != 0) {
                rank = k;
                for (int o = 0; o < p.parts; ++o) {
                    if (o == b) continue;
                    int first = 0, end = top;              // first entry that does not stand before this one
                    while (first < end) {
                        const int mid = (first + end) >> 1;
                        const uint32_t v = s_value[o * top + mid];
                        if (v > value || (v == value && o < b)) first = mid + 1; else end = mid;
                    }
                    rank += first;
                }
            }
            n_top = min(top, __syncthreads_count(value != 0));
            if (rank < top) { s_top_value[rank] = value; s_top_index[rank] = index; }
        }
        cluster_sync_all();                    // nobody's shared memory goes before it has been read
        if (part != 0) return;
    }

    // --- outputs
    if (warp != 0) return;
    if (!(all.s > 0.f)) none = 1;
    const float log_s = logf(all.s);
    if (t == 0) {
        a.logprobs[row_i] = none ? nan_f() : at_token - all.m - log_s;
        if (a.entropies) a.entropies[row_i] = none ? nan_f() : log_s - all.w / all.s;
    }
    if (t < top) {
        const bool there = t < n_top;
        a.top_ids[row_i * top + t] = none || !there ? -1 : s_top_index[t];
        a.top_logprobs[row_i * top + t] = none ? nan_f() : there ? unordered(s_top_value[t]) - all.m - log_s : -INFINITY;
    }
}

}  // namespace

cudaError_t configure_token_logprobs() { return cudaSuccess; }

mt_status launch_token_logprobs(const LogprobArgs& a, const OpContext& c, cudaStream_t s) {
    Params p;
    p.a = a;
    // parts: as long as the rows leave the GPU with fewer than four CTAs an SM and a part keeps kMinPart logits
    p.parts = 1;
    while (p.parts < kMaxParts && (int64_t)a.n * p.parts * 2 <= 4LL * c.sm_count && a.vocab / (p.parts * 2) >= kMinPart) p.parts *= 2;
    p.part_len = ((a.vocab + p.parts - 1) / p.parts + 7) / 8 * 8;
    const bool hold = (p.part_len + (a.fp32 ? 3 : 7)) / (a.fp32 ? 4 : 8) <= kHold * kThreads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)a.n * p.parts));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.parts;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.parts > 1 ? 2 : 1;
    ++g_kernel_launches;
    const cudaError_t e = a.fp32 ? (hold ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<true, true>, p) : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<true, false>, p))
                                 : (hold ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<false, true>, p) : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<false, false>, p));
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

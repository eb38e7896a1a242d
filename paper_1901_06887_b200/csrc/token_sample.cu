// A token drawn from each row of logits: temperature, top-k, top-p and min-p, from given uniform numbers.
//
// Mathematics.  w_i = 2^(c (x_i - max x)), c = log2(e) / temperature.  In the order of falling logits (equal ones: rising index) each of the three limits
// keeps a front part, so what passes all of them is a front part too, up to a last entry (key, index).  The drawn token is the first, in index order, at
// which the kept mass exceeds u times all of it.
// A border between two tokens must not depend on the order of summing, so weights are whole numbers, w_i 2^s rounded, s = 46 or less where a row of
// ones would pass 2^62: sums of them are exact in any order.  (A token below 2^-46 of the likeliest has no mass and is never drawn; all mass lost is
// below 2^-28 of a row of 2^18.)  The exponential is taken in 64 bits: at fp32's 2^-23 one draw in some hundreds would fall on the other side of a border.
//
// The last entry kept.  A histogram, count and mass, of the distance to the maximum over the range where the cut can lie: behind weight
// (1 - p) W / V all tokens together weigh less than (1 - p) W.  The bin where a limit is reached is put on a list and ranked by counting.  Where it
// holds too many (long ties, a range of odd shape) it is split by its keys' bits until it does not, or until one value is left, whose ties are taken from
// the front of the row.
//
// Split.  A row is cut into parts, one CTA each, that form a cluster; a part into stretches, one a warp.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 1024;
constexpr int kList = 1024;
constexpr int kMaxParts = 8;
constexpr int kMinPart = 4096;                // logits of a part, at least
using u64 = unsigned long long;

struct Params {
    SampleArgs a;
    int parts;
    int shift;                                // of the weights
    int vecs;                                 // of a warp's stretch
};

struct Shared {
    uint32_t count[kBins], lo[kBins], hi[kBins];
    uint32_t key[kList];
    int32_t index[kList];
    uint32_t part_key[kList];                 // this part's share of the list
    int32_t part_index[kList];
    u64 sorted[kList];
    int32_t order[kList];
    u64 warp_sum[kWarps];
    u64 scan[kWarps], scan2[kWarps];
    float warp_max[kWarps];
    uint32_t warp_lo[kWarps], warp_hi[kWarps];
    u64 sum;
    float max;
    int bad;
    uint32_t key_lo, key_hi;
    int n_list;
    uint32_t ties;
    int32_t found;                            // of the r-th tie, by its part
    int bin;
    u64 above_mass, bin_mass;
    uint32_t above_count, bin_count;
    int pick;
};

__device__ __forceinline__ uint32_t ordered(float x) {        // grows with the value; minus zero counts as zero
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint32_t remote_u32(const void* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ u64 remote_u64(const void* p, uint32_t rank) {
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}

template <bool FP32> constexpr int kVec = FP32 ? 4 : 8;

// A row as vectors of 16 aligned bytes; vector j holds elements j N - skew ... of the row.
template <bool FP32>
struct Row {
    const char* base;                         // aligned, at or in front of the first element
    int skew, vocab, n_vec;
    __device__ __forceinline__ Row(const void* logits, int64_t at, int v) {
        constexpr int B = FP32 ? 4 : 2;
        const char* const p = static_cast<const char*>(logits) + at * B;
        skew = (int)((reinterpret_cast<uintptr_t>(p) & 15) / B);
        base = p - skew * B;
        vocab = v;
        n_vec = (int)(((int64_t)v + skew + kVec<FP32> - 1) / kVec<FP32>);
    }
    // minus infinity outside the row
    __device__ __forceinline__ void load(int j, float (&x)[kVec<FP32>]) const {
        constexpr int N = kVec<FP32>;
        const int first = j * N - skew;
        if (first >= 0 && first + N <= vocab) {
            const uint4 v = *reinterpret_cast<const uint4*>(base + (int64_t)j * 16);
            if (FP32) {
                x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
            } else {
                x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
                x[N - 4] = bf16_lo(v.z); x[N - 3] = bf16_hi(v.z); x[N - 2] = bf16_lo(v.w); x[N - 1] = bf16_hi(v.w);
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int i = first + e;
                x[e] = i < 0 || i >= vocab ? -INFINITY
                     : FP32 ? reinterpret_cast<const float*>(base)[(int64_t)j * N + e] : bf16_to_f(reinterpret_cast<const uint16_t*>(base)[(int64_t)j * N + e]);
            }
        }
    }
};

struct Weights {
    double max, c, scale;
    __device__ __forceinline__ double real(float x) const { return exp2(((double)x - max) * c); }
    __device__ __forceinline__ u64 whole(double w) const { return __double2ull_rn(w * scale); }
};

template <bool FP32>
__global__ void __launch_bounds__(kThreads) token_sample_kernel(const Params p) {
    __shared__ Shared s;
    constexpr int N = kVec<FP32>;
    const SampleArgs& a = p.a;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int64_t row_i = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x - row_i * p.parts);
    pdl_launch_dependents();
    pdl_wait();

    const Row<FP32> row(a.logits, row_i * a.row_stride, a.vocab);
    const int vec0 = (int)min((int64_t)(part * kWarps + warp) * p.vecs, (int64_t)row.n_vec), vec1 = min(vec0 + p.vecs, row.n_vec);
    auto team_sync = [&]() { if (p.parts > 1) cluster_sync_all(); else __syncthreads(); };
    // f(value, index) for this lane's elements of its warp's stretch (minus infinity outside the row)
    auto for_lane = [&](auto f) {
        for (int j = vec0 + lane; j < vec1; j += 32) {
            float x[N];
            row.load(j, x);
#pragma unroll
            for (int e = 0; e < N; ++e) f(x[e], j * N - row.skew + e);
        }
    };

    // --- what the row asks for
    float temperature = a.temperature ? a.temperature[row_i] : 1.f, top_p = a.top_p ? a.top_p[row_i] : 1.f, min_p = a.min_p ? a.min_p[row_i] : 0.f;
    const float u = a.uniform[row_i];
    int top_k = a.top_k ? a.top_k[row_i] : 0;
    const bool refused = !(temperature >= 0.f && temperature < INFINITY) || top_p != top_p || min_p != min_p || !(u >= 0.f && u < 1.f);
    if (temperature == 0.f || min_p > 1.f) { top_k = 1; min_p = 0.f; }
    if (temperature == 0.f) temperature = 1.f;
    if (top_k <= 0 || top_k > a.vocab) top_k = a.vocab;

    // --- the maximum
    {
        float m = -INFINITY;
        bool bad = false;
        for_lane([&](float x, int) { m = fmaxf(m, x); bad |= x != x; });
        m = warp_max(m);
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 0) s.warp_max[warp] = bad ? INFINITY : m;      // plus infinity is no distribution either
        __syncthreads();
        if (t == 0) {
            float all = s.warp_max[0];
            for (int w = 1; w < kWarps; ++w) all = fmaxf(all, s.warp_max[w]);
            s.max = all;
        }
    }
    team_sync();
    float top = s.max;
    for (int r = 0; r < (p.parts > 1 ? p.parts : 0); ++r) top = fmaxf(top, __uint_as_float(remote_u32(&s.max, r)));
    if (refused || !(top > -INFINITY && top < INFINITY)) {
        if (part == 0 && t == 0) {
            a.ids[row_i] = -1;
            if (a.logprobs) a.logprobs[row_i] = nan_f();
            if (refused) raise_status(a.status, MT_ERR_INVALID_ARG, (int)row_i);
        }
        team_sync();
        return;
    }
    Weights wt;
    wt.max = top;
    wt.c = 1.4426950408889634074 / (double)temperature;
    wt.scale = (double)(1ull << p.shift);

    auto block_sum = [&](u64 v) {             // of every thread, in every thread
#pragma unroll
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if (lane == 0) s.scan[warp] = v;
        __syncthreads();
        u64 all = 0;
        for (int w = 0; w < kWarps; ++w) all += s.scan[w];
        return all;
    };

    // --- the last entry kept: all, unless a limit is reached
    uint32_t cut_key = 0;
    int cut_index = 0x7fffffff;
    const bool by_mass = top_p < 1.f;
    if (top_k < a.vocab || by_mass) {
        u64 target = ~0ull;                   // mass at which top-p is reached
        float range = (float)p.shift + 2.f;   // in powers of two below the maximum
        uint32_t key_lo = 0, key_hi = 0xffffffffu, above_count = 0;
        u64 above_mass = 0;
        int bin1 = -1;
        bool ties = false, none = false;
        uint32_t n_in = 0;                    // entries among which the last one is
        if (by_mass && top_k > 1) {
            u64 mine = 0;
            for_lane([&](float x, int) { mine += wt.whole(wt.real(x)); });
            const u64 sum = block_sum(mine);
            if (t == 0) s.sum = sum;
            team_sync();
            u64 all = sum;
            if (p.parts > 1) {
                all = 0;
                for (int r = 0; r < p.parts; ++r) all += remote_u64(&s.sum, r);
            }
            target = top_p > 0.f ? (u64)ceil((double)top_p * (double)all) : 0;
            const float tail = log2f((float)a.vocab / (fmaxf(1.f - top_p, 1e-7f) * (float)((double)all / wt.scale))) + 1.f;
            range = fminf(range, fmaxf(tail, 1.f));
        }
        const float cf = (float)fmin(wt.c, 1e30), bins = (float)(kBins - 1) / range;
        auto first_bin = [&](float x) {       // falls with the value
            const float b = (top - x) * cf * bins;
            return b < (float)kBins ? (int)b : kBins;
        };
        if (top_k == 1) { ties = true; key_lo = key_hi = ordered(top); }

        for (int level = 0; !ties && !none; ++level) {
            // histogram of what is left
            int down = 0;
            if (level > 0) while ((key_hi - key_lo) >> down >= (uint32_t)kBins) ++down;
            __syncthreads();
            for (int b = t; b < kBins; b += kThreads) s.count[b] = s.lo[b] = s.hi[b] = 0;
            __syncthreads();
            for_lane([&](float x, int) {
                if (x == -INFINITY) return;
                const int b1 = first_bin(x);
                int b;
                if (level == 0) {
                    b = b1;
                    if (b >= kBins) return;
                } else {
                    const uint32_t key = ordered(x);
                    if (b1 != bin1 || key < key_lo || key > key_hi) return;
                    b = (int)((key_hi - key) >> down);
                }
                atomicAdd(&s.count[b], 1u);
                if (by_mass) {
                    const u64 w = wt.whole(wt.real(x));
                    const uint32_t lo = (uint32_t)w, old = atomicAdd(&s.lo[b], lo), hi = (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u);
                    if (hi) atomicAdd(&s.hi[b], hi);
                }
            });
            team_sync();
            // every CTA adds all parts up; a thread has two bins
            uint32_t count[2];
            u64 mass[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int b = 2 * t + e;
                count[e] = 0;
                mass[e] = 0;
                for (int r = 0; r < p.parts; ++r) {
                    if (p.parts > 1) {
                        count[e] += remote_u32(&s.count[b], r);
                        if (by_mass) mass[e] += ((u64)remote_u32(&s.hi[b], r) << 32) + remote_u32(&s.lo[b], r);
                    } else {
                        count[e] += s.count[b];
                        mass[e] += ((u64)s.hi[b] << 32) + s.lo[b];
                    }
                }
            }
            u64 c_incl = count[0] + count[1], m_incl = mass[0] + mass[1];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const u64 cy = __shfl_up_sync(0xffffffffu, c_incl, d), my = __shfl_up_sync(0xffffffffu, m_incl, d);
                if (lane >= d) { c_incl += cy; m_incl += my; }
            }
            if (lane == 31) { s.scan[warp] = c_incl; s.scan2[warp] = m_incl; }
            if (t == 0) s.bin = -1;
            __syncthreads();
            u64 c_before = above_count + c_incl - count[0] - count[1], m_before = above_mass + m_incl - mass[0] - mass[1];
            for (int w = 0; w < warp; ++w) { c_before += s.scan[w]; m_before += s.scan2[w]; }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool was = c_before >= (u64)top_k || m_before >= target;
                const u64 c_after = c_before + count[e], m_after = m_before + mass[e];
                const bool is = c_after >= (u64)top_k || m_after >= target;
                // (a target of zero is reached by the first entry, not before it)
                if (count[e] > 0 && is && (!was || c_before == 0)) {
                    s.bin = 2 * t + e;
                    s.above_count = (uint32_t)c_before; s.above_mass = m_before;
                    s.bin_count = count[e]; s.bin_mass = mass[e];
                }
                c_before = c_after; m_before = m_after;
            }
            team_sync();                      // (the histogram may be cleared again)
            if (s.bin < 0) { none = true; break; }
            above_count = s.above_count;
            above_mass = s.above_mass;
            n_in = s.bin_count;
            if (level == 0) {
                bin1 = s.bin;
            } else {
                const uint32_t hi = key_hi - ((uint32_t)s.bin << down);
                const uint32_t span = (1u << down) - 1u;
                key_lo = hi - key_lo > span ? hi - span : key_lo;
                key_hi = hi;
            }
            if (n_in <= (uint32_t)kList) break;
            if (level == 0) {                 // the keys of the bin
                uint32_t lo = 0xffffffffu, hi = 0;
                for_lane([&](float x, int) {
                    if (x == -INFINITY || first_bin(x) != bin1) return;
                    const uint32_t key = ordered(x);
                    lo = min(lo, key);
                    hi = max(hi, key);
                });
                lo = __reduce_min_sync(0xffffffffu, lo);
                hi = __reduce_max_sync(0xffffffffu, hi);
                if (lane == 0) { s.warp_lo[warp] = lo; s.warp_hi[warp] = hi; }
                __syncthreads();
                if (t == 0) {
                    for (int w = 1; w < kWarps; ++w) { lo = min(lo, s.warp_lo[w]); hi = max(hi, s.warp_hi[w]); }
                    s.key_lo = lo; s.key_hi = hi;
                }
                team_sync();
                key_lo = s.key_lo;
                key_hi = s.key_hi;
                for (int r = 0; r < (p.parts > 1 ? p.parts : 0); ++r) { key_lo = min(key_lo, remote_u32(&s.key_lo, r)); key_hi = max(key_hi, remote_u32(&s.key_hi, r)); }
            }
            if (key_lo == key_hi) ties = true;
        }

        if (ties) {                           // one value: its r first
            const u64 w = wt.whole(wt.real(unordered(key_lo)));
            u64 r = (u64)top_k - above_count;
            if (by_mass && top_k > 1 && w > 0) {
                const u64 need = target > above_mass ? (target - above_mass + w - 1) / w : 1;
                if (need < r) r = need;
            }
            if (r < 1) r = 1;
            uint32_t n = 0;
            for_lane([&](float x, int) { n += x > -INFINITY && ordered(x) == key_lo ? 1u : 0u; });
            n = __reduce_add_sync(0xffffffffu, n);
            __syncthreads();
            if (lane == 0) s.warp_lo[warp] = n;
            if (t == 0) s.found = -1;
            __syncthreads();
            uint32_t before = 0, all = 0;
            for (int v = 0; v < kWarps; ++v) { const uint32_t x = s.warp_lo[v]; if (v < warp) before += x; all += x; }
            if (t == 0) s.ties = all;
            team_sync();
            for (int q = 0; q < part; ++q) before += remote_u32(&s.ties, q);
            if (r > before && r <= (u64)before + n) {             // the warp that has it
                uint32_t left = (uint32_t)(r - before);
                for (int j0 = vec0; j0 < vec1 && left > 0; j0 += 32) {
                    const int j = j0 + lane;
                    float x[N];
                    uint32_t m = 0;
                    if (j < vec1) {
                        row.load(j, x);
#pragma unroll
                        for (int e = 0; e < N; ++e) if (x[e] > -INFINITY && ordered(x[e]) == key_lo) m |= 1u << e;
                    }
                    const uint32_t here = __popc(m);
                    uint32_t incl = here;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
                        if (lane >= d) incl += y;
                    }
                    const uint32_t total = __shfl_sync(0xffffffffu, incl, 31);
                    if (left > incl - here && left <= incl) {
                        for (uint32_t k = left - (incl - here); k > 1; --k) m &= m - 1;
                        s.found = j * N - row.skew + __ffs(m) - 1;
                    }
                    left = left > total ? left - total : 0;
                }
            }
            team_sync();
            cut_key = key_lo;
            cut_index = s.found;
            for (int q = 0; q < (p.parts > 1 ? p.parts : 0); ++q) cut_index = max(cut_index, (int)remote_u32(&s.found, q));
            if (cut_index < 0) cut_index = 0x7fffffff;            // fewer than that: all
        } else if (!none) {                   // a list
            if (t == 0) s.n_list = 0;
            __syncthreads();
            const bool keys = key_hi != 0xffffffffu || key_lo != 0;
            for_lane([&](float x, int i) {
                if (x == -INFINITY || first_bin(x) != bin1) return;
                const uint32_t key = ordered(x);
                if (keys && (key < key_lo || key > key_hi)) return;
                const int at = atomicAdd(&s.n_list, 1);
                s.part_key[at] = key;
                s.part_index[at] = i;
            });
            team_sync();
            int n = 0;
            for (int r = 0; r < p.parts; ++r) {
                const int m = p.parts > 1 ? (int)remote_u32(&s.n_list, r) : s.n_list;
                for (int i = t; i < m; i += kThreads) {
                    s.key[n + i] = p.parts > 1 ? remote_u32(&s.part_key[i], r) : s.part_key[i];
                    s.index[n + i] = p.parts > 1 ? (int32_t)remote_u32(&s.part_index[i], r) : s.part_index[i];
                }
                n += m;
            }
            if (t == 0) s.pick = n - 1;
            __syncthreads();
            for (int i = t; i < n; i += kThreads) {
                const uint32_t key = s.key[i];
                const int at = s.index[i];
                int rank = 0;
                for (int j = 0; j < n; ++j) rank += (s.key[j] > key || (s.key[j] == key && s.index[j] < at)) ? 1 : 0;
                s.order[rank] = i;
                s.sorted[rank] = by_mass ? wt.whole(wt.real(unordered(key))) : 0;
            }
            __syncthreads();
            u64 v[2], incl = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) { v[e] = 2 * t + e < n ? s.sorted[2 * t + e] : 0; incl += v[e]; }
            const u64 own = incl;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const u64 y = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += y;
            }
            if (lane == 31) s.scan[warp] = incl;
            __syncthreads();
            u64 mass = above_mass + incl - own;
            for (int w = 0; w < warp; ++w) mass += s.scan[w];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mass += v[e];
                const int j = 2 * t + e;
                if (j < n && ((u64)above_count + j + 1 >= (u64)top_k || mass >= target)) atomicMin(&s.pick, j);
            }
            __syncthreads();
            const int last = s.order[s.pick];
            cut_key = s.key[last];
            cut_index = s.index[last];
        }
    }

    // --- the kept mass, stretch by stretch, and the token
    auto weight = [&](float x, int i) -> u64 {
        const uint32_t key = ordered(x);
        if (x == -INFINITY || key < cut_key || (key == cut_key && i > cut_index)) return 0;
        const double w = wt.real(x);
        return min_p > 0.f && w < (double)min_p ? 0 : wt.whole(w);
    };
    u64 mine = 0;
    for_lane([&](float x, int i) { mine += weight(x, i); });
    u64 stretch = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) stretch += __shfl_xor_sync(0xffffffffu, stretch, o);
    __syncthreads();
    if (lane == 0) s.warp_sum[warp] = stretch;
    __syncthreads();
    u64 before = 0, sum = 0;
    for (int w = 0; w < kWarps; ++w) { const u64 x = s.warp_sum[w]; if (w < warp) before += x; sum += x; }
    u64 all = sum;
    if (p.parts > 1) {
        if (t == 0) s.sum = sum;
        team_sync();
        all = 0;
        for (int r = 0; r < p.parts; ++r) {
            const u64 x = remote_u64(&s.sum, r);
            if (r < part) before += x;
            all += x;
        }
    }
    u64 at = (u64)((double)u * (double)all);
    if (at >= all) at = all - 1;
    if (at >= before && at < before + stretch) {                  // the warp that has it
        u64 run = before;
        for (int j0 = vec0; j0 < vec1; j0 += 32) {
            const int j = j0 + lane;
            u64 w[N], own = 0;
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = 0;
            if (j < vec1) {
                row.load(j, x);
#pragma unroll
                for (int e = 0; e < N; ++e) { w[e] = weight(x[e], j * N - row.skew + e); own += w[e]; }
            }
            u64 incl = own;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const u64 y = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += y;
            }
            u64 sofar = run + incl - own;
            if (at >= sofar && at < sofar + own) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (at >= sofar && at < sofar + w[e]) {
                        a.ids[row_i] = j * N - row.skew + e;
                        if (a.logprobs) a.logprobs[row_i] = (float)(((double)x[e] - wt.max) / (double)temperature - log((double)all / wt.scale));
                    }
                    sofar += w[e];
                }
            }
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    team_sync();                              // nobody's shared memory goes before it has been read
}

}  // namespace

mt_status launch_token_sample(const SampleArgs& a, const OpContext& c, cudaStream_t s) {
    Params p;
    p.a = a;
    p.parts = 1;
    while (p.parts < kMaxParts && (int64_t)a.n * p.parts * 2 <= 2LL * c.sm_count && a.vocab / (p.parts * 2) >= kMinPart) p.parts *= 2;
    p.shift = 46;
    while (p.shift > 0 && ((int64_t)a.vocab << p.shift) > (1ll << 62)) --p.shift;
    const int vec = a.fp32 ? 4 : 8, most = (a.vocab + 2 * vec - 2) / vec;          // vectors of a row that starts anywhere
    p.vecs = (most + p.parts * kWarps - 1) / (p.parts * kWarps);
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
    const cudaError_t e = a.fp32 ? cudaLaunchKernelEx(&cfg, token_sample_kernel<true>, p) : cudaLaunchKernelEx(&cfg, token_sample_kernel<false>, p);
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

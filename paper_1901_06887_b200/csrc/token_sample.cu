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
constexpr int kBins = 2 * kThreads;
constexpr int kFine = 16, kCoarse = kBins / kFine;
constexpr int kList = kThreads;
constexpr int kMaxParts = 8;
static_assert(kBins == 2 * kThreads && kThreads == kMaxParts * kCoarse && kFine == 16, "");
constexpr int kMinPart = 2048;                // logits of a part, at least
constexpr int kHeldBytes = 65536;             // of a part that stays in shared memory, at most: two CTAs an SM
using u64 = unsigned long long;

struct Params {
    SampleArgs a;
    int parts;
    int shift;                                // of the weights
    int vecs;                                 // of a warp's stretch
};

struct Shared {
    uint2 count[kThreads], lo[kThreads], hi[kThreads];       // bins 2 t and 2 t + 1: entries, and mass in two words
    u64 entry[kList], part_entry[kList], sorted[kList];      // the list, this part's share of it (ordered logit, rising as the index falls), weights in order
    u64 coarse_mass[kCoarse];                 // sixteen bins each
    uint32_t coarse_count[kCoarse];
    double table[16];
    u64 warp_sum[kWarps], scan[kWarps], scan2[kWarps];
    uint32_t warp_a[kWarps], warp_b[kWarps];
    float max;
    u64 sum;
    uint32_t key_lo, key_hi, ties;
    int n_list, found;
    int bin, pick;
    u64 above_mass;
    uint32_t above_count;
};

__device__ __forceinline__ uint32_t ordered(float x) {        // grows with the value; minus zero counts as zero
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
// Loads from the shared memory of CTA `rank` of the cluster.  (Volatile keeps them behind the barrier in front; without a clobber several are under way
// at once.)
__device__ __forceinline__ uint32_t remote_u32(const void* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(smem_u32(p), rank)));
    return v;
}
__device__ __forceinline__ uint2 remote_u32x2(const void* p, uint32_t rank) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(map_to_cta(smem_u32(p), rank)));
    return v;
}
__device__ __forceinline__ u64 remote_u64(const void* p, uint32_t rank) {
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(map_to_cta(smem_u32(p), rank)));
    return v;
}
__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <class T>
__device__ __forceinline__ T warp_scan(T v, int lane) {       // with its own
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += y;
    }
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
    __device__ __forceinline__ uint4 load(int j) const {
        constexpr int N = kVec<FP32>;
        const int first = j * N - skew;
        if (first >= 0 && first + N <= vocab) return *reinterpret_cast<const uint4*>(base + (int64_t)j * 16);
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            w[q] = FP32 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
            for (int h = 0; h < (FP32 ? 1 : 2); ++h) {
                const int e = FP32 ? q : 2 * q + h, i = first + e;
                if (i < 0 || i >= vocab) continue;
                if (FP32) w[q] = reinterpret_cast<const uint32_t*>(base)[(int64_t)j * N + e];
                else w[q] = __byte_perm(w[q], reinterpret_cast<const uint16_t*>(base)[(int64_t)j * N + e], h ? 0x5410 : 0x3254);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <bool FP32>
__device__ __forceinline__ void decode(const uint4& v, float (&x)[kVec<FP32>]) {
    constexpr int N = kVec<FP32>;
    if (FP32) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    } else {
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
        x[N - 4] = bf16_lo(v.z); x[N - 3] = bf16_hi(v.z); x[N - 2] = bf16_lo(v.w); x[N - 1] = bf16_hi(v.w);
    }
}

template <bool FP32>
__device__ __forceinline__ float element(const void* p, int64_t i) {
    return FP32 ? static_cast<const float*>(p)[i] : bf16_to_f(static_cast<const uint16_t*>(p)[i]);
}

// Weights as whole numbers, 2^y 2^shift with y = c (x - max).  y = n / 16 + r: 2^(n / 16) comes from a table of 16 (two banks each: no conflicts), 2^r, |r| <= 1/32,
// from its series to r^5, off by 2^-42.  Adding 2^52 + 2^51 over 16 rounds to sixteenths and leaves n in the low word; adding 2^52 rounds to a whole number
// and leaves it there.  Nine operations of 64 bits; the weight of x = max is exact.  What lies 100 powers of two and more below the maximum goes
// through as the maximum, so that n stays small, and gets a factor next to zero.
constexpr u64 kWhole = 0x4330000000000000ull;          // 2^52
struct Weights {
    double max, c;
    float top, far;                           // the maximum, and a distance of 100 powers of two below it
    const double* table;                      // 2^(i / 16) 2^shift
    // with 2^52 in front
    __device__ __forceinline__ u64 raw(float x) const {
        const bool none = x - top < far;
        const double d = (double)(none ? top : x) - max, magic = 422212465065984.0;
        const double t = fma(d, c, magic), r = fma(d, c, magic - t);
        const int n = __double2loint(t);
        double p = fma(r, 1.3333558146428443e-3, 9.6181291076284771e-3);
        p = fma(r, p, 5.5504108664821579e-2);
        p = fma(r, p, 2.4022650695910071e-1);
        p = fma(r, p, 6.9314718055994530e-1);
        p = fma(r, p, 1.0);
        const double e = table[n & 15];
        const int hi = __double2hiint(e) + ((n >> 4) << 20);
        const double scaled = __hiloint2double(none ? 0 : hi, __double2loint(e));
        return (u64)__double_as_longlong(fma(p, scaled, 4503599627370496.0));
    }
    __device__ __forceinline__ u64 operator()(float x) const { return raw(x) - kWhole; }
};

template <bool FP32, bool HOLD>
__global__ void __launch_bounds__(kThreads, 2) token_sample_kernel(const Params p) {
    __shared__ Shared s;
    extern __shared__ uint4 held[];           // this part's vectors, where they fit
    constexpr int N = kVec<FP32>;
    const SampleArgs& a = p.a;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int64_t row_i = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x - row_i * p.parts), parts = p.parts;
    pdl_launch_dependents();
    pdl_wait();

    const Row<FP32> row(a.logits, row_i * a.row_stride, a.vocab);
    const int vec0 = (int)min((int64_t)(part * kWarps + warp) * p.vecs, (int64_t)row.n_vec), vec1 = min(vec0 + p.vecs, row.n_vec);
    auto team_sync = [&]() { if (parts > 1) cluster_sync_all(); else __syncthreads(); };
    // what every part has, in lane r for part r (behind a team_sync)
    auto of_parts_u64 = [&](const u64& x) { return parts == 1 ? (lane == 0 ? x : 0) : lane < parts ? remote_u64(&x, lane) : 0; };
    auto of_parts_u32 = [&](const void* x) { return parts == 1 ? (lane == 0 ? *static_cast<const uint32_t*>(x) : 0) : lane < parts ? remote_u32(x, lane) : 0; };
    const int held0 = part * kWarps * p.vecs;
    auto vec_at = [&](int j) { return HOLD ? held[j - held0] : row.load(j); };
    // f(value, index) for this lane's elements of its warp's stretch (minus infinity outside the row)
    auto for_lane = [&](auto f) {
        for (int j = vec0 + lane; j < vec1; j += 32) {
            float x[N];
            decode<FP32>(vec_at(j), x);
#pragma unroll
            for (int e = 0; e < N; ++e) f(x[e], j * N - row.skew + e);
        }
    };

    // The same for the elements that pass a test, which is made of 32 elements of the lane at a time: the lanes of a warp then call f as often as the one
    // with most of them, not for every element that any lane has.
    auto for_passing = [&](auto passes, auto f) {
        constexpr int kVecs = 32 / N;
        for (int j0 = vec0 + lane; j0 < vec1; j0 += 32 * kVecs) {
            uint32_t m = 0;
#pragma unroll
            for (int h = 0; h < kVecs; ++h) {
                if (j0 + 32 * h >= vec1) break;
                float x[N];
                decode<FP32>(vec_at(j0 + 32 * h), x);
#pragma unroll
                for (int e = 0; e < N; ++e) m |= passes(x[e]) ? 1u << (h * N + e) : 0u;
            }
            for (; m; m &= m - 1) {
                const int bit = __ffs(m) - 1, j = j0 + 32 * (bit / N), e = bit % N, i = j * N - row.skew + e;
                f(HOLD ? element<FP32>(held + (j - held0), e) : element<FP32>(row.base, (int64_t)j * N + e), i);
            }
        }
    };

    // --- what the row asks for
    float temperature = a.temperature ? a.temperature[row_i] : 1.f, top_p = a.top_p ? a.top_p[row_i] : 1.f, min_p = a.min_p ? a.min_p[row_i] : 0.f;
    const float u = a.uniform[row_i];
    int top_k = a.top_k ? a.top_k[row_i] : 0;
    const bool refused = !(temperature >= 0.f && temperature < INFINITY) || top_p != top_p || min_p != min_p || !(u >= 0.f && u < 1.f);
    if (temperature == 0.f || min_p > 1.f) { top_k = 1; min_p = 0.f; }
    temperature = temperature == 0.f ? 1.f : fmaxf(temperature, 0x1p-126f);
    if (top_k <= 0 || top_k > a.vocab) top_k = a.vocab;

    // --- the maximum
    {
        float m = -INFINITY;
        bool bad = false;
        constexpr int kAhead = 4;
        for (int j0 = vec0 + lane; j0 < vec1; j0 += 32 * kAhead) {
            uint4 v[kAhead];
#pragma unroll
            for (int h = 0; h < kAhead; ++h)
                if (j0 + 32 * h < vec1) v[h] = row.load(j0 + 32 * h);
#pragma unroll
            for (int h = 0; h < kAhead; ++h) {
                if (j0 + 32 * h >= vec1) break;
                if (HOLD) held[j0 + 32 * h - held0] = v[h];
                float x[N];
                decode<FP32>(v[h], x);
#pragma unroll
                for (int e = 0; e < N; ++e) { m = fmaxf(m, x[e]); bad |= x[e] != x[e]; }
            }
        }
        if (t < 16) s.table[t] = exp2(t / 16.0) * (double)(1ull << p.shift);
        s.count[t] = s.lo[t] = s.hi[t] = make_uint2(0, 0);
        if (t == 0) s.n_list = 0;
        m = warp_max(m);
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 0) s.warp_a[warp] = __float_as_uint(bad ? INFINITY : m);      // plus infinity is no distribution either
        __syncthreads();
        if (warp == 0) {
            m = warp_max(lane < kWarps ? __uint_as_float(s.warp_a[lane]) : -INFINITY);
            if (lane == 0) s.max = m;
        }
    }
    team_sync();
    const uint32_t top_bits = of_parts_u32(&s.max);
    const float top = warp_max(lane < parts ? __uint_as_float(top_bits) : -INFINITY);
    if (refused || !(top > -INFINITY && top < INFINITY)) {
        if (part == 0 && t == 0) {
            a.ids[row_i] = -1;
            if (a.logprobs) a.logprobs[row_i] = nan_f();
            if (refused) raise_status(a.status, MT_ERR_INVALID_ARG, (int)row_i);
        }
        team_sync();
        return;
    }
    const double scale = (double)(1ull << p.shift);
    Weights wt;
    wt.max = top;
    wt.c = 1.4426950408889634074 / (double)temperature;
    wt.top = top;
    wt.far = -(float)fmin(100.0 / wt.c, 3.402823466e38);
    wt.table = s.table;
    const u64 least = min_p > 0.f ? (u64)ceil((double)min_p * scale) : 0;

    // --- the last entry kept: all, unless a limit is reached.  An entry is (ordered logit, ~index): the larger comes first.
    u64 cut = 0;
    const bool by_mass = top_p < 1.f && top_k > 1;
    if (top_k < a.vocab || by_mass) {
        u64 target = ~0ull;                   // mass at which top-p is reached
        float range = (float)p.shift + 2.f;   // in powers of two below the maximum
        if (by_mass) range = fminf(range, log2f((float)a.vocab / fmaxf(1.f - top_p, 1e-7f)) + 1.f);
        const float per = fminf((float)wt.c * ((float)(kBins - 1) / range), 3.402823466e38f);
        auto first_bin = [&](float x) {       // falls with the value
            const float b = (top - x) * per;
            return b < (float)kBins ? (int)b : kBins;
        };
        uint32_t* const counts = reinterpret_cast<uint32_t*>(s.count);
        uint32_t* const los = reinterpret_cast<uint32_t*>(s.lo);
        uint32_t* const his = reinterpret_cast<uint32_t*>(s.hi);
        auto into_bin = [&](int b, u64 w) {
            atomicAdd(counts + b, 1u);
            if (by_mass) {
                const uint32_t lo = (uint32_t)w, old = atomicAdd(los + b, lo), hi = (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u);
                if (hi) atomicAdd(his + b, hi);
            }
        };
        uint32_t key_lo = 0, key_hi = 0xffffffffu, above_count = 0, n_in = 0;
        u64 above_mass = 0;
        int bin1 = -1, bin = -1;
        // The bin, of all parts' added up, where a limit is reached: s.bin, -1 if none.  Every CTA finds it for itself: first among the parts' sums of
        // sixteen bins, then among these sixteen, so little is read from other CTAs (all 1024 bins took 9000 cycles).
        auto find_bin = [&](bool first) {
            __syncthreads();
            {
                const uint2 count = s.count[t], lo = s.lo[t], hi = s.hi[t];
                uint32_t n = count.x + count.y;
                u64 m = ((u64)hi.x << 32) + lo.x + ((u64)hi.y << 32) + lo.y;
#pragma unroll
                for (int o = kFine / 4; o; o >>= 1) { n += __shfl_xor_sync(0xffffffffu, n, o); m += __shfl_xor_sync(0xffffffffu, m, o); }
                if (t % (kFine / 2) == 0) { s.coarse_count[t / (kFine / 2)] = n; s.coarse_mass[t / (kFine / 2)] = m; }
                if (t == 0) s.bin = -1;
            }
            team_sync();
            // a limit is reached among n entries of mass m behind c_before of m_before?  (A target of zero is reached by the first entry, not before it.)
            auto reached = [&](u64 c_before, u64 m_before, uint32_t n, u64 m) {
                const bool was = c_before >= (u64)top_k || m_before >= target, is = c_before + n >= (u64)top_k || m_before + m >= target;
                return n > 0 && is && (!was || c_before == 0);
            };
            const int group = t / kMaxParts, r = t % kMaxParts;
            uint32_t n = 0;
            u64 m = 0, whole = 0;
            if (r < parts) {
                n = parts > 1 ? remote_u32(&s.coarse_count[group], r) : s.coarse_count[group];
                m = parts > 1 ? remote_u64(&s.coarse_mass[group], r) : s.coarse_mass[group];
            }
            if (first && by_mass) {
                whole = warp_sum_u64(of_parts_u64(s.sum));
                target = top_p > 0.f ? (u64)ceil((double)top_p * (double)whole) : 0;
            }
#pragma unroll
            for (int o = kMaxParts / 2; o; o >>= 1) { n += __shfl_xor_sync(0xffffffffu, n, o); m += __shfl_xor_sync(0xffffffffu, m, o); }
            const u64 c_incl = warp_scan(r == 0 ? (u64)n : 0, lane), m_incl = warp_scan(r == 0 ? m : 0, lane);
            if (lane == 31) { s.scan[warp] = c_incl; s.scan2[warp] = m_incl; }
            __syncthreads();
            u64 c_before = above_count + c_incl - n, m_before = above_mass + m_incl - m;
            for (int w = 0; w < warp; ++w) { c_before += s.scan[w]; m_before += s.scan2[w]; }
            if (r == 0 && reached(c_before, m_before, n, m)) { s.bin = group; s.above_count = (uint32_t)c_before; s.above_mass = m_before; }
            __syncthreads();
            const int coarse = s.bin;
            if (coarse >= 0) {                // every warp: bin lane % 16 of parts lane / 16, + 2, ..
                const int b = coarse * kFine + lane % kFine;
                n = 0;
                m = 0;
#pragma unroll
                for (int q = 0; q < kMaxParts; q += 2) {
                    const int of = q + lane / kFine;
                    if (of >= parts) continue;
                    n += parts > 1 ? remote_u32(counts + b, of) : counts[b];
                    m += parts > 1 ? ((u64)remote_u32(his + b, of) << 32) + remote_u32(los + b, of) : ((u64)his[b] << 32) + los[b];
                }
                n += __shfl_xor_sync(0xffffffffu, n, kFine);
                m += __shfl_xor_sync(0xffffffffu, m, kFine);
                const u64 c = s.above_count + warp_scan(lane < kFine ? (u64)n : 0, lane) - n, before = s.above_mass + warp_scan(lane < kFine ? m : 0, lane) - m;
                const uint32_t hit = __ballot_sync(0xffffffffu, lane < kFine && reached(c, before, n, m));
                const int at = __ffs(hit) - 1;
                above_count = (uint32_t)__shfl_sync(0xffffffffu, c, at);
                above_mass = __shfl_sync(0xffffffffu, before, at);
                n_in = __shfl_sync(0xffffffffu, n, at);
                bin = coarse * kFine + at;
            } else {
                bin = -1;
            }
            team_sync();                      // (the bins may be cleared again)
        };
        bool ties = top_k == 1, none = false;
        if (ties) {
            key_lo = key_hi = ordered(top);
        } else {
            u64 mine = 0;
            if (by_mass) {                    // the row's mass and the first histogram in one pass
                for_lane([&](float x, int) {
                    const u64 w = wt(x);
                    mine += w;
                    const int b = first_bin(x);
                    if (b < kBins) into_bin(b, w);
                });
            } else {
                for_lane([&](float x, int) {
                    const int b = first_bin(x);
                    if (b < kBins) atomicAdd(counts + b, 1u);
                });
            }
            if (by_mass) {
                mine = warp_sum_u64(mine);
                if (lane == 0) s.warp_sum[warp] = mine;
                __syncthreads();
                if (warp == 0) {
                    const u64 all = warp_sum_u64(lane < kWarps ? s.warp_sum[lane] : 0);
                    if (lane == 0) s.sum = all;
                }
            }
            find_bin(true);
            none = bin < 0;
            bin1 = bin;
        }
        if (!ties && !none && n_in > (uint32_t)kList) {       // too many: on by the bits of the bin's keys
            uint32_t lo = 0xffffffffu, hi = 0;
            for_lane([&](float x, int) {
                if (first_bin(x) != bin1) return;
                const uint32_t key = ordered(x);
                lo = min(lo, key);
                hi = max(hi, key);
            });
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            if (lane == 0) { s.warp_a[warp] = lo; s.warp_b[warp] = hi; }
            __syncthreads();
            if (warp == 0) {
                lo = __reduce_min_sync(0xffffffffu, lane < kWarps ? s.warp_a[lane] : 0xffffffffu);
                hi = __reduce_max_sync(0xffffffffu, lane < kWarps ? s.warp_b[lane] : 0);
                if (lane == 0) { s.key_lo = lo; s.key_hi = hi; }
            }
            team_sync();
            lo = of_parts_u32(&s.key_lo);
            hi = of_parts_u32(&s.key_hi);
            key_lo = __reduce_min_sync(0xffffffffu, lane < parts ? lo : 0xffffffffu);
            key_hi = __reduce_max_sync(0xffffffffu, lane < parts ? hi : 0);
            while (key_lo != key_hi && n_in > (uint32_t)kList) {
                int down = 0;
                while ((key_hi - key_lo) >> down >= (uint32_t)kBins) ++down;
                s.count[t] = s.lo[t] = s.hi[t] = make_uint2(0, 0);
                __syncthreads();
                for_passing([&](float x) { return first_bin(x) == bin1; }, [&](float x, int) {
                    const uint32_t key = ordered(x);
                    if (key >= key_lo && key <= key_hi) into_bin((int)((key_hi - key) >> down), by_mass ? wt(x) : 0);
                });
                find_bin(false);
                const uint32_t end = key_hi - ((uint32_t)bin << down), span = (1u << down) - 1u;
                key_lo = end - key_lo > span ? end - span : key_lo;
                key_hi = end;
            }
            ties = key_lo == key_hi;
        }

        if (ties) {                           // one value: its r first
            const u64 w = wt(unordered(key_lo));
            u64 r = (u64)top_k - above_count;
            if (by_mass && w > 0) {
                const u64 need = target > above_mass ? (target - above_mass + w - 1) / w : 1;
                if (need < r) r = need;
            }
            if (r < 1) r = 1;
            uint32_t n = 0;
            for_lane([&](float x, int) { n += ordered(x) == key_lo ? 1u : 0u; });
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0) s.warp_a[warp] = n;
            if (t == 0) s.found = -1;
            __syncthreads();
            const uint32_t in_warp = lane < kWarps ? s.warp_a[lane] : 0;
            if (t == 0) s.ties = 0;
            const uint32_t in_part = __reduce_add_sync(0xffffffffu, in_warp);
            if (t == 0) s.ties = in_part;
            team_sync();
            const uint32_t of_part = of_parts_u32(&s.ties);
            const uint32_t before = __reduce_add_sync(0xffffffffu, (lane < part ? of_part : 0) + (lane < warp ? in_warp : 0));
            if (r > before && r <= (u64)before + n) {             // the warp that has it
                uint32_t left = (uint32_t)(r - before);
                for (int j0 = vec0; j0 < vec1 && left > 0; j0 += 32) {
                    const int j = j0 + lane;
                    uint32_t m = 0;
                    if (j < vec1) {
                        float x[N];
                        decode<FP32>(vec_at(j), x);
#pragma unroll
                        for (int e = 0; e < N; ++e) if (ordered(x[e]) == key_lo) m |= 1u << e;
                    }
                    const uint32_t here = __popc(m), incl = warp_scan(here, lane), total = __shfl_sync(0xffffffffu, incl, 31);
                    if (left > incl - here && left <= incl) {
                        for (uint32_t k = left - (incl - here); k > 1; --k) m &= m - 1;
                        s.found = j * N - row.skew + __ffs(m) - 1;
                    }
                    left = left > total ? left - total : 0;
                }
            }
            team_sync();
            const int at_part = (int)of_parts_u32(&s.found);
            const int index = __reduce_max_sync(0xffffffffu, lane < parts ? at_part : -1);
            cut = (u64)key_lo << 32 | (index < 0 ? 0x80000000u : (uint32_t)~index);         // (fewer than that: all)
        } else if (!none) {                   // a list
            for_passing([&](float x) { return first_bin(x) == bin1; }, [&](float x, int i) {
                const uint32_t key = ordered(x);
                if (key < key_lo || key > key_hi) return;
                s.part_entry[atomicAdd(&s.n_list, 1)] = (u64)key << 32 | (uint32_t)~i;
            });
            team_sync();
            const int in_part = (int)of_parts_u32(&s.n_list), n = (int)n_in;
            const int upto = warp_scan(in_part, lane);
            int from = 0, first = 0;          // entry t: of which part, and that part's first
#pragma unroll
            for (int r = 0; r < kMaxParts - 1; ++r) {
                const int end = __shfl_sync(0xffffffffu, upto, r);
                if (r + 1 < parts && t >= end) { from = r + 1; first = end; }
            }
            if (t < n) s.entry[t] = parts > 1 ? remote_u64(&s.part_entry[t - first], from) : s.part_entry[t];
            if (t == 0) s.pick = n - 1;
            __syncthreads();
            // an entry's rank, counted by 1 to 32 threads
            int each = 1;
            while (each < 32 && n * each * 2 <= kThreads) each *= 2;
            const int i = t / each;
            const u64 mine = i < n ? s.entry[i] : 0;
            int rank = 0;
            if (i < n) for (int j = t & (each - 1); j < n; j += each) rank += s.entry[j] > mine ? 1 : 0;
            for (int o = each / 2; o; o >>= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
            if (i < n && (t & (each - 1)) == 0) s.sorted[rank] = mine;
            __syncthreads();
            const u64 x = t < n ? s.sorted[t] : 0;
            const u64 incl = warp_scan(by_mass && t < n ? wt(unordered((uint32_t)(x >> 32))) : 0, lane);
            if (lane == 31) s.scan[warp] = incl;
            __syncthreads();
            u64 mass = above_mass + incl;
            for (int w = 0; w < warp; ++w) mass += s.scan[w];
            if (t < n && ((u64)above_count + t + 1 >= (u64)top_k || mass >= target)) atomicMin(&s.pick, t);
            __syncthreads();
            cut = s.sorted[s.pick];
        }
    }

    // --- the kept mass, stretch by stretch, and the token
    const uint32_t cut_key = (uint32_t)(cut >> 32);
    const int cut_index = (int)~(uint32_t)cut;
    const bool all_kept = cut == 0 && least == 0;
    auto weight = [&](float x, int i) -> u64 {
        const u64 w = wt(x);
        const uint32_t key = ordered(x);
        return w < least || key < cut_key || (key == cut_key && i > cut_index) ? 0 : w;
    };
    // (a float that lies below the last one kept needs no weight)
    const float floor_x = cut == 0 ? -INFINITY : unordered(cut_key);
    u64 mine = 0;
    if (all_kept) {
        int n = 0;
        for_lane([&](float x, int) { mine += wt.raw(x); ++n; });
        mine -= (u64)n * kWhole;
    } else {
        for_passing([&](float x) { return x >= floor_x; }, [&](float x, int i) { mine += weight(x, i); });
    }
    const u64 stretch = warp_sum_u64(mine);
    if (lane == 0) s.warp_sum[warp] = stretch;
    __syncthreads();
    const u64 in_warp = lane < kWarps ? s.warp_sum[lane] : 0;
    u64 before = warp_sum_u64(lane < warp ? in_warp : 0), all = warp_sum_u64(in_warp);
    if (parts > 1) {
        if (t == 0) s.sum = all;
        team_sync();
        const u64 of_part = of_parts_u64(s.sum);
        before += warp_sum_u64(lane < part ? of_part : 0);
        all = warp_sum_u64(of_part);
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
                decode<FP32>(vec_at(j), x);
#pragma unroll
                for (int e = 0; e < N; ++e) { w[e] = weight(x[e], j * N - row.skew + e); own += w[e]; }
            }
            const u64 incl = warp_scan(own, lane);
            u64 sofar = run + incl - own;
            if (at >= sofar && at < sofar + own) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (at >= sofar && at < sofar + w[e]) {
                        a.ids[row_i] = j * N - row.skew + e;
                        if (a.logprobs) a.logprobs[row_i] = (float)(((double)x[e] - wt.max) / (double)temperature - log((double)all / scale));
                    }
                    sofar += w[e];
                }
            }
            run += __shfl_sync(0xffffffffu, incl, 31);
            if (run > at) break;
        }
    }
    if (parts > 1) cluster_sync_all();        // nobody's shared memory goes before it has been read
}

}  // namespace

cudaError_t configure_token_sample() {
    const cudaError_t e = cudaFuncSetAttribute(token_sample_kernel<true, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldBytes);
    return e == cudaSuccess ? cudaFuncSetAttribute(token_sample_kernel<false, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldBytes) : e;
}

mt_status launch_token_sample(const SampleArgs& a, const OpContext& c, cudaStream_t s) {
    Params p;
    p.a = a;
    const int vec = a.fp32 ? 4 : 8, most = (a.vocab + 2 * vec - 2) / vec;          // vectors of a row that starts anywhere
    auto vecs = [&](int parts) { return (most + parts * kWarps - 1) / (parts * kWarps); };
    auto fits = [&](int parts) { return vecs(parts) * kWarps * 16 <= kHeldBytes; };
    p.parts = 1;
    while (p.parts < kMaxParts && a.vocab / (p.parts * 2) >= kMinPart && (!fits(p.parts) || (int64_t)a.n * p.parts * 2 <= 2LL * c.sm_count)) p.parts *= 2;
    p.vecs = vecs(p.parts);
    const bool hold = fits(p.parts);
    p.shift = 46;
    while (p.shift > 0 && ((int64_t)a.vocab << p.shift) > (1ll << 62)) --p.shift;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)a.n * p.parts));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = hold ? p.vecs * kWarps * 16 : 0;
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
    const cudaError_t e = a.fp32 ? (hold ? cudaLaunchKernelEx(&cfg, token_sample_kernel<true, true>, p) : cudaLaunchKernelEx(&cfg, token_sample_kernel<true, false>, p))
                                 : (hold ? cudaLaunchKernelEx(&cfg, token_sample_kernel<false, true>, p) : cudaLaunchKernelEx(&cfg, token_sample_kernel<false, false>, p));
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

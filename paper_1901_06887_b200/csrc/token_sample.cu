// A token drawn from each row of logits: temperature, top-k, top-p and min-p, from given uniform numbers.
//
// Mathematics.  w_i = 2^(c (x_i - max x)), c = log2(e) / temperature.  In the order of falling logits (equal ones: rising index) each of the three limits
// keeps a front part, so what passes all of them is a front part too, up to a last entry (key, index).  The drawn token is the first, in index order, at
// which the kept mass exceeds u times all of it.
// A border between two tokens must not depend on the order of summing, so weights are whole numbers, w_i 2^s rounded, s = 46 or less where a row of
// ones would pass 2^62: sums of them are exact in any order.  (A token below half a unit, 2^-s, of the likeliest has no mass and is never drawn; of a
// row of V at most V / 2 units are lost or won by rounding: 2^-31 of it for 2^16 logits, 2^-27 for 2^18, 2^-23 for 2^20.)  The exponential is taken in 64 bits:
// with fp32 arguments one draw in ten thousand of a row of 128 000 would fall on the other side of a border, and sums of fp32 would add to that.
//
// The last entry kept.  A histogram, count and mass, of the distance to the maximum over the range where the cut can lie: the tokens whose weight is
// below (1 - p) / V of the largest weigh less than 1 - p together, and the row at least 1.  The bin where a limit is reached is put on a list and ranked by
// counting.  Where it holds too many (long ties, a range of odd shape) it is split by its keys' bits until it does not, or until one value is left, whose
// ties are taken from the front of the row.
//
// Split.  A row is cut into parts, one CTA each, that form a cluster; a part into stretches, one a warp.  A part that fits stays in shared memory, so that
// a row is read once; other rows come from L2 again.
//
// Cost.  Many rows: the first pass and the pass of 64-bit exponentials, one behind the other: 512 rows of 128 000 in fp32, whose bytes are 40 us, take 170, of which
// 55 without the weights.  (The other 115 are some 55 cycles of a scheduler for a warp's logits, the last of 3.5 waves of clusters counted whole; nine 64-bit
// operations and a conversion are 30 by themselves.)  A mixed batch of 64 rows of 128 000 in bf16 takes 48 us, all of them without a limit 24, with top-k 27, with
// top-p 56: rows with a limit go three times over their part, the histogram's additions to shared memory take as long as the exponentials, and five barriers
// of the cluster lie between.  One row of 32 000: 13.6 us, these barriers and the dependent steps between them; 6.2 without a limit.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2 * kThreads;
constexpr int kFine = 16, kCoarse = kBins / kFine;
constexpr int kList = 2 * kThreads, kSome = 32;
constexpr int kMaxParts = 8;
constexpr int kAtOnce = 4;                    // parts whose shared memory is read at once
static_assert(kList * 8 <= 3 * kThreads * sizeof(uint2), "the list over the bins");
static_assert(kBins == 2 * kThreads && kCoarse == 64 && kFine == 16 && kMaxParts <= 8, "");
constexpr int kMinPart = 2048;                // logits of a part, at least
constexpr int kShortPart = 16384;             // and of one that takes an SM by itself, rather
constexpr int held_bytes(int ctas) { return ctas == 1 ? 193792 : 77056; }      // of a part that stays in shared memory, at most, with so many CTAs an SM
using u64 = unsigned long long;

struct Params {
    SampleArgs a;
    int parts;
    int shift;                                // of the weights
    int vecs;                                 // of a warp's stretch
};

struct Shared {
    uint4 edge[3];                            // the row's first and last vector with minus infinity outside it, and nothing but that
    uint2 count[kThreads], lo[kThreads], hi[kThreads];       // bins 2 t and 2 t + 1: entries, and mass in two words; then a part of the list
    ulonglong2 entry[kList];                                 // the list: (ordered logit, rising as the index falls), weight
    u64 part_entry[kList];                                   // this part's share of it
    alignas(16) u64 coarse_mass[kCoarse];     // sixteen bins each
    alignas(8) uint32_t coarse_count[kCoarse];
    double table[32];
    u64 warp_sum[kWarps], scan[kWarps];
    uint32_t warp_a[kWarps], warp_b[kWarps];
    float max;
    u64 sum;
    uint32_t key_lo, key_hi, ties;
    int n_list, found;
    int bin;
    u64 above_mass, target;
    uint32_t above_count, bin_count;
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
__device__ __forceinline__ ulonglong2 remote_u64x2(const void* p, uint32_t rank) {
    ulonglong2 v;
    asm volatile("ld.shared::cluster.v2.u64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "r"(map_to_cta(smem_u32(p), rank)));
    return v;
}
template <int LANES = 32>                     // the sum of so many neighbours
__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
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
    int whole0, whole1;                       // vectors that lie in the row
    __device__ __forceinline__ Row(const void* logits, int64_t at, int v) {
        constexpr int B = FP32 ? 4 : 2;
        const char* const p = static_cast<const char*>(logits) + at * B;
        skew = (int)((reinterpret_cast<uintptr_t>(p) & 15) / B);
        base = p - skew * B;
        vocab = v;
        n_vec = (int)(((int64_t)v + skew + kVec<FP32> - 1) / kVec<FP32>);
        whole0 = skew > 0 ? 1 : 0;
        whole1 = max((int)(((int64_t)v + skew) / kVec<FP32>), whole0);
    }
    // minus infinity outside the row
    __device__ __forceinline__ uint4 load(int j) const {
        if ((unsigned)(j - whole0) < (unsigned)(whole1 - whole0)) return *reinterpret_cast<const uint4*>(base + (int64_t)j * 16);
        return edge(j);
    }
    __device__ uint4 edge(int j) const {
        constexpr int N = kVec<FP32>;
        const int64_t first = (int64_t)j * N - skew;
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            w[q] = FP32 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
            for (int h = 0; h < (FP32 ? 1 : 2); ++h) {
                const int e = FP32 ? q : 2 * q + h;
                const int64_t i = first + e;
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

__device__ __forceinline__ float max_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
template <bool FP32>
__device__ __forceinline__ float max_nan_of(const uint4& v) {
    if (FP32) return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    uint32_t m = v.x;                         // two at a time
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.y));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.z));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.w));
    return max_nan(bf16_lo(m), bf16_hi(m));
}
// x times f, a float of [0, 1), exactly and rounded down (up).
__device__ __forceinline__ u64 times(u64 x, float f, bool up) {
    const uint32_t bits = __float_as_uint(f), e = bits >> 23;
    const uint32_t mant = e ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
    const int down = 150 - (e ? (int)e : 1);                  // f = mant 2^-down, down >= 24
    const u64 lo = x * mant, hi = __umul64hi(x, mant);
    u64 q;
    bool rest;
    if (down < 64) { q = hi << (64 - down) | lo >> down; rest = (lo & ((1ull << down) - 1)) != 0; }
    else if (down < 128) { q = down == 64 ? hi : hi >> (down - 64); rest = lo != 0 || (q << (down - 64)) != hi; }
    else { q = 0; rest = (lo | hi) != 0; }
    return q + (up && rest ? 1 : 0);
}

template <bool FP32>
__device__ __forceinline__ float element(const void* p, int64_t i) {
    return FP32 ? static_cast<const float*>(p)[i] : bf16_to_f(static_cast<const uint16_t*>(p)[i]);
}

struct Four { float x[4]; };
// f(four logits) for a vector: once for fp32, twice for bf16, in a loop where there are two CTAs an SM.  (The passes' loops are kept short: unrolled further they miss
// the instruction cache.  One CTA by itself gains by it: 18 rows of 128 000 38.0 -> 36.5 us.)
template <bool FP32, int CTAS, class F>
__device__ __forceinline__ void by_fours(uint4 v, F f) {
    if (FP32) {
        f(Four{__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)});
    } else {
#pragma unroll (CTAS == 1 ? 2 : 1)
        for (int h = 0; h < 2; ++h) {
            f(Four{bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)});
            v.x = v.z;
            v.y = v.w;
        }
    }
}
// Weights as whole numbers, 2^y 2^shift with y = c (x - max).  y = n / 32 + r: 2^(n / 32) comes from a table, 2^r, |r| <= 1/64, from its series to r^4,
// off by 2^-39.  Adding 2^52 + 2^51 over 32 rounds to parts of 32 and leaves n in the low word; adding 2^52 rounds to a whole number
// and leaves it there.  Nine operations of 64 bits, which bound the pass; the weight of x = max is exact.  What lies 1000 powers of two and more below the maximum goes
// through as that, so that n stays small, and gets a factor next to zero.
constexpr u64 kWhole = 0x4330000000000000ull;          // 2^52
// (in constant memory they are operands where they stand; as literals two moves each)
__constant__ double kMagic = 211106232532992.0, kTwo52 = 4503599627370496.0;
__constant__ double kSeries[4] = {6.9314718055994530e-1, 2.4022650695910071e-1, 5.5504108664821579e-2, 9.6181291076284771e-3};    // ln(2)^i / i!
struct Weights {
    double max, c;
    float half_top, least;                    // half the maximum; the least logit that counts: 1000 powers of two below the maximum, if it is a number
    const double* table;                      // 2^(i / 32) 2^shift, i << 15 taken from the upper word: adding n << 15 to it then multiplies by 2^(n >> 5)
    // with 2^52 in front
    __device__ __forceinline__ u64 raw(float x) const {
        const bool none = x < least;
        const double d = (double)(none ? least : x) - max;
        const double t = fma(d, c, kMagic), r = fma(d, c, kMagic - t);
        const int n = __double2loint(t);
        double p = fma(r, kSeries[3], kSeries[2]);
        p = fma(r, p, kSeries[1]);
        p = fma(r, p, kSeries[0]);
        p = fma(r, p, 1.0);
        const double e = table[n & 31];
        const int hi = __double2hiint(e) + (n << 15);
        return (u64)__double_as_longlong(fma(p, __hiloint2double(none ? 0 : hi, __double2loint(e)), kTwo52));
    }
    __device__ __forceinline__ u64 operator()(float x) const { return raw(x) - kWhole; }
};

// 2^23 and a bin, which rises as the value falls, or more.  (By half the distance to the maximum: the whole one may pass the largest number.)
constexpr float kFirst = 8388608.f;
__device__ __forceinline__ float bin_of(float x, float half_top, float per) { return fmaf(fmaf(x, -0.5f, half_top), per, kFirst); }
__device__ __forceinline__ int bin_index(float f) { return __float_as_int(f) - 0x4b000000; }

// Adds to shared memory where `on`, without a branch.  (Volatile keeps them between the barriers; without a clobber the table's loads for the next logits may pass.)
__device__ __forceinline__ void add_if(bool on, uint32_t addr, uint32_t v) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %0, 0;\n\t@q red.shared.add.u32 [%1], %2;\n\t}" ::"r"((uint32_t)on), "r"(addr), "r"(v));
}
__device__ __forceinline__ uint32_t fetch_add_if(bool on, uint32_t addr, uint32_t v) {
    uint32_t old = 0;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t@q atom.shared.add.u32 %0, [%2], %3;\n\t}" : "+r"(old) : "r"((uint32_t)on), "r"(addr), "r"(v));
    return old;
}

// A lane's share of a row: every 32nd vector of its warp's stretch.
template <bool FP32, bool HOLD>
struct Share {
    Row<FP32> row;
    uint4* held;                              // vector j is held[j - held0], where the part is held
    const uint4* edge;
    int held0, vec0, vec1, lane;
    __device__ __forceinline__ uint4 from_row(int j, int whole1) const {       // whole1: not behind the stretch
        if ((unsigned)(j - row.whole0) < (unsigned)(whole1 - row.whole0)) return reinterpret_cast<const uint4*>(row.base)[j];
        return j < vec1 ? row.load(j) : none();
    }
    __device__ __forceinline__ static uint4 none() {
        constexpr uint32_t w = FP32 ? 0xff800000u : 0xff80ff80u;
        return make_uint4(w, w, w, w);
    }
    // behind the first pass: minus infinity outside the row and behind the stretch
    __device__ __forceinline__ uint4 get(int j) const {
        if (HOLD) return j < vec1 ? held[j - held0] : none();
        const uint4* const in_row = reinterpret_cast<const uint4*>(row.base) + j;
        return *((unsigned)(j - row.whole0) < (unsigned)(min(row.whole1, vec1) - row.whole0) ? in_row : edge + (j >= vec1 ? 2 : j < row.whole0 ? 0 : 1));
    }
    __device__ __forceinline__ float at(int64_t i) const {                     // i: from the first vector's first element
        return HOLD ? element<FP32>(held, i - (int64_t)held0 * kVec<FP32>) : element<FP32>(row.base, i);
    }
};

// The passes over a row.  (Inlined into the kernel: as functions of their own they took 10 % longer.)

// The first one: the maximum, NaN if any logit is.
template <bool FP32, bool HOLD>
__device__ __forceinline__ float max_pass(const Share<FP32, HOLD>& share) {
    const Share<FP32, HOLD> l = share;
    const int whole1 = min(l.row.whole1, l.vec1);
    constexpr int kAhead = 4;                 // vectors under way
    float m = -INFINITY;
    for (int j0 = l.vec0 + l.lane; j0 < l.vec1; j0 += 32 * kAhead) {
        uint4 v[kAhead];
#pragma unroll
        for (int h = 0; h < kAhead; ++h) v[h] = l.from_row(j0 + 32 * h, whole1);
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            if (HOLD && j0 + 32 * h < l.vec1) l.held[j0 + 32 * h - l.held0] = v[h];
            m = max_nan(m, max_nan_of<FP32>(v[h]));
        }
    }
    return m;
}

// The row's mass.
template <bool FP32, int CTAS, bool HOLD>
__device__ __forceinline__ u64 sum_pass(const Share<FP32, HOLD>& l, const Weights& wt) {
    u64 mass = 0;
    uint4 q = l.get(l.vec0 + l.lane), next = l.get(l.vec0 + l.lane + 32);
#pragma unroll 1
    for (int j = l.vec0 + l.lane; j < l.vec1; j += 32) {
        const uint4 v = q;
        q = next;
        next = l.get(j + 64);
        by_fours<FP32, CTAS>(v, [&](const Four& y) {
            u64 sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += wt.raw(y.x[e]);
            mass += sum - 4 * kWhole;
        });
    }
    return mass;
}

// The row's mass, and the histogram of (count and) mass over bins of the distance to the maximum.
template <bool FP32, int CTAS, bool HOLD>
__device__ __forceinline__ u64 mass_pass(const Share<FP32, HOLD>& l, const Weights& wt, float per, bool count, uint32_t counts_at, uint32_t los_at, uint32_t his_at) {
    u64 mass = 0;
    uint4 q = l.get(l.vec0 + l.lane), next = l.get(l.vec0 + l.lane + 32);
#pragma unroll 1
    for (int j = l.vec0 + l.lane; j < l.vec1; j += 32) {
        const uint4 v = q;
        q = next;
        next = l.get(j + 64);
        by_fours<FP32, CTAS>(v, [&](const Four& y) {
            u64 w[4];
            uint32_t old[4], at[4];
            bool in[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = wt(y.x[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = bin_of(y.x[e], wt.half_top, per);
                in[e] = f < kFirst + kBins;
                at[e] = 4 * bin_index(f);
                old[e] = fetch_add_if(in[e], los_at + at[e], (uint32_t)w[e]);
                add_if(in[e] && count, counts_at + at[e], 1u);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mass += w[e];
                const uint32_t hi = (uint32_t)(w[e] >> 32) + (old[e] + (uint32_t)w[e] < old[e] ? 1u : 0u);
                add_if(in[e] && hi > 0, his_at + at[e], hi);
            }
        });
    }
    return mass;
}

// Counts alone.
template <bool FP32, int CTAS, bool HOLD>
__device__ __forceinline__ void count_pass(const Share<FP32, HOLD>& l, float half_top, float per, uint32_t counts_at) {
#pragma unroll 1
    for (int j = l.vec0 + l.lane; j < l.vec1; j += 32) {
        by_fours<FP32, CTAS>(l.get(j), [&](const Four& y) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = bin_of(y.x[e], half_top, per);
                add_if(f < kFirst + kBins, counts_at + 4 * bin_index(f), 1u);
            }
        });
    }
}

// f(value, index, whether there is one) for the elements that pass a test, which is made of 32 elements of the lane at a time: the lanes of a warp then call f
// as often as the one with most of them, not for every element that any lane has; two at a time, since f is a chain of dependent steps.
template <bool FP32, bool HOLD, class P, class F>
__device__ __forceinline__ void for_passing(const Share<FP32, HOLD>& l, P passes, F f) {
    constexpr int N = kVec<FP32>, kVecs = 32 / N;
    for (int j0 = l.vec0 + l.lane; j0 < l.vec1; j0 += 32 * kVecs) {
        uint32_t m = 0;
#pragma unroll
        for (int h = 0; h < kVecs; ++h) {
            float x[N];
            decode<FP32>(l.get(j0 + 32 * h), x);
#pragma unroll
            for (int e = 0; e < N; ++e) m |= passes(x[e]) ? 1u << (h * N + e) : 0u;
        }
        auto at = [&](int bit) { return (j0 + 32 * (bit / N)) * N + bit % N; };
        while (m) {
            const int i0 = at(__ffs(m) - 1);
            m &= m - 1;
            const int i1 = m ? at(__ffs(m) - 1) : i0;
            const bool both = m != 0;
            m &= m - 1;
            const float x0 = l.at(i0), x1 = l.at(i1);
            f(x0, i0 - l.row.skew, true);
            f(x1, i1 - l.row.skew, both);
        }
    }
}

// What is kept: at or above the last entry kept, and not below min-p's weight.
struct Kept {
    Weights wt;
    u64 least;
    uint32_t key;
    int index;
    __device__ __forceinline__ u64 operator()(float x, int i) const {
        const u64 w = wt(x);
        const uint32_t k = ordered(x);
        return w < least || k < key || (k == key && i > index) ? 0 : w;
    }
};
template <bool FP32, bool HOLD>
__device__ __forceinline__ u64 kept_pass(const Share<FP32, HOLD>& share, const Kept& what, float floor_x) {
    const Share<FP32, HOLD> l = share;
    const Kept kept = what;
    u64 mass = 0;
    for_passing(l, [&](float x) { return x >= floor_x; }, [&](float x, int i, bool there) {
        const u64 w = kept(x, i);
        mass += there ? w : 0;
    });
    return mass;
}

// CTAS an SM: two, or, where there are no more than SMs, one, with twice the registers and more of them held.
template <bool FP32, bool HOLD, int CTAS>
__global__ void __launch_bounds__(kThreads, CTAS) token_sample_kernel(const Params p) {
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
    Share<FP32, HOLD> l = {row, held, s.edge, part * kWarps * p.vecs, vec0, vec1, lane};

    // --- what the row asks for
    float temperature = a.temperature ? a.temperature[row_i] : 1.f, top_p = a.top_p ? a.top_p[row_i] : 1.f, min_p = a.min_p ? a.min_p[row_i] : 0.f;
    const float u = a.uniform[row_i] + 0.f;   // (minus zero is zero)
    int top_k = a.top_k ? a.top_k[row_i] : 0;
    const bool refused = !(temperature >= 0.f && temperature < INFINITY) || top_p != top_p || min_p != min_p || !(u >= 0.f && u < 1.f);
    if (temperature == 0.f || min_p > 1.f) { top_k = 1; min_p = 0.f; }
    temperature = temperature == 0.f ? 1.f : fmaxf(temperature, 0x1p-126f);
    if (top_k <= 0 || top_k > a.vocab) top_k = a.vocab;
    top_p = fmaxf(top_p, 0.f);                // (what is below zero asks for the first entry, as zero does; the histogram's range is made of 1 - top_p)

    // --- the maximum
    const double c = 1.4426950408889634074 / (double)temperature;
    const double scale = (double)(1ull << p.shift);
    const bool by_mass = top_p < 1.f && top_k > 1, by_count = top_k < a.vocab, all_kept = !by_mass && !by_count && !(min_p > 0.f);
    if (t < 32) {
        const double e = exp2(t / 32.0) * scale;
        s.table[t] = __hiloint2double(__double2hiint(e) - (t << 15), __double2loint(e));
    }
    Weights wt;
    wt.c = c;
    wt.table = s.table;
    u64 mine = 0;
    float m = -INFINITY;                      // NaN if any is
    {
        m = max_pass(l);
        s.count[t] = s.lo[t] = s.hi[t] = make_uint2(0, 0);
        if (t == 0) s.n_list = 0;
        if (!HOLD && t < 3) s.edge[t] = t == 2 ? l.none() : row.load(t == 0 ? 0 : row.n_vec - 1);
        const bool bad = __any_sync(0xffffffffu, m != m);
        m = warp_max(m);
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
    wt.max = top;
    wt.half_top = 0.5f * top;
    wt.least = __double2float_ru(fmax((double)top - 1000.0 / c, -3.4028234663852886e38));     // (the lowest number: minus infinity lies below it)
    const u64 least = min_p > 0.f ? (u64)ceil((double)min_p * scale) : 0;

    // --- the last entry kept: all, unless a limit is reached.  An entry is (ordered logit, ~index): the larger comes first.
    u64 cut = 0;
    if (by_count || by_mass) {
        u64 target = ~0ull;                   // mass at which top-p is reached
        float range = (float)p.shift + 2.f;   // in powers of two below the maximum
        if (by_mass) range = fminf(range, log2f((float)a.vocab / (1.f - top_p)) + 1.f);
        const float per = fminf((float)wt.c * ((float)(2 * kBins - 2) / range), 3.402823466e38f);
        uint32_t* const counts = reinterpret_cast<uint32_t*>(s.count);
        uint32_t* const los = reinterpret_cast<uint32_t*>(s.lo);
        uint32_t* const his = reinterpret_cast<uint32_t*>(s.hi);
        const uint32_t counts_at = smem_u32(counts), los_at = smem_u32(los), his_at = smem_u32(his);
        auto into_bin = [&](int b, u64 w) {
            atomicAdd(counts + b, 1u);
            if (by_mass) {
                const uint32_t lo = (uint32_t)w, old = atomicAdd(los + b, lo), hi = (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u);
                if (hi) atomicAdd(his + b, hi);
            }
        };
        uint32_t key_lo = 0, key_hi = 0xffffffffu, above_count = 0, n_in = 0;
        u64 above_mass = 0;
        float bin1 = 0.f;
        int bin = -1;
        // The bin, of all parts' added up, where a limit is reached: -1 if none.  The first warp of every CTA finds it by itself, among the parts' sums of
        // sixteen bins and then among these sixteen, so little is read from other CTAs (all 1024 bins took 9000 cycles).
        auto find_bin = [&](bool first) {
            __syncthreads();
            {
                const uint2 count = s.count[t], lo = s.lo[t], hi = s.hi[t];
                uint32_t n = count.x + count.y;
                u64 m = ((u64)hi.x << 32) + lo.x + ((u64)hi.y << 32) + lo.y;
#pragma unroll
                for (int o = kFine / 4; o; o >>= 1) { n += __shfl_xor_sync(0xffffffffu, n, o); m += __shfl_xor_sync(0xffffffffu, m, o); }
                if (t % (kFine / 2) == 0) { s.coarse_count[t / (kFine / 2)] = n; s.coarse_mass[t / (kFine / 2)] = m; }
            }
            team_sync();
            if (warp == 0) {
                // a limit is reached among n entries of mass m behind c_before of m_before?  (A target of zero is reached by the first entry, not before it.)
                auto reached = [&](uint32_t c_before, u64 m_before, uint32_t n, u64 m) {
                    const bool was = c_before >= (uint32_t)top_k || m_before >= target, is = c_before + n >= (uint32_t)top_k || m_before + m >= target;
                    return (by_count ? n > 0 : m > 0) && is && (!was || (by_count ? c_before == 0 : m_before == 0));
                };
                const u64 sum = first && by_mass ? of_parts_u64(s.sum) : 0;
                uint2 n = make_uint2(0, 0);
                u64 m0 = 0, m1 = 0;
                if (parts == 1) {                                  // groups 2 lane and 2 lane + 1
                    n = *reinterpret_cast<const uint2*>(&s.coarse_count[2 * lane]);
                    m0 = s.coarse_mass[2 * lane];
                    m1 = s.coarse_mass[2 * lane + 1];
                } else {
#pragma unroll 1
                    for (int r0 = 0; r0 < parts; r0 += kAtOnce) {
                        uint2 x[kAtOnce];
                        ulonglong2 y[kAtOnce];
#pragma unroll
                        for (int r = 0; r < kAtOnce; ++r) {
                            x[r] = remote_u32x2(&s.coarse_count[2 * lane], (r0 + r) & (parts - 1));
                            y[r] = remote_u64x2(&s.coarse_mass[2 * lane], (r0 + r) & (parts - 1));
                        }
#pragma unroll
                        for (int r = 0; r < kAtOnce; ++r) {
                            const bool there = r0 + r < parts;
                            n.x += there ? x[r].x : 0;
                            n.y += there ? x[r].y : 0;
                            m0 += there ? y[r].x : 0;
                            m1 += there ? y[r].y : 0;
                        }
                    }
                }
                if (first && by_mass) target = top_p > 0.f ? times(warp_sum_u64(sum), top_p, true) : 0;
                const uint32_t c0 = above_count + warp_scan(n.x + n.y, lane) - n.x - n.y;
                const u64 b0 = above_mass + warp_scan(m0 + m1, lane) - m0 - m1;
                const bool in0 = reached(c0, b0, n.x, m0), in1 = reached(c0 + n.x, b0 + m0, n.y, m1);
                const uint32_t hit = __ballot_sync(0xffffffffu, in0 || in1);
                int found = -1;
                if (hit) {
                    const int at = __ffs(hit) - 1, group = __shfl_sync(0xffffffffu, 2 * lane + (in0 ? 0 : 1), at);
                    const uint32_t c_group = __shfl_sync(0xffffffffu, in0 ? c0 : c0 + n.x, at);
                    const u64 m_group = __shfl_sync(0xffffffffu, in0 ? b0 : b0 + m0, at);
                    const int b = group * kFine + lane % kFine;    // of parts lane / 16, + 2, ..
                    uint32_t nb = 0;
                    u64 mb = 0;
                    if (parts == 1) {
                        if (lane < kFine) { nb = counts[b]; mb = ((u64)his[b] << 32) + los[b]; }
                    } else {
#pragma unroll 1
                        for (int r0 = 0; r0 < parts; r0 += kAtOnce) {
                            uint32_t x[kAtOnce / 2][3];
#pragma unroll
                            for (int q = 0; q < kAtOnce / 2; ++q) {
                                const int of = (r0 + 2 * q + lane / kFine) & (parts - 1);
                                x[q][0] = remote_u32(counts + b, of);
                                x[q][1] = remote_u32(los + b, of);
                                x[q][2] = remote_u32(his + b, of);
                            }
#pragma unroll
                            for (int q = 0; q < kAtOnce / 2; ++q) {
                                if (r0 + 2 * q + lane / kFine >= parts) continue;
                                nb += x[q][0];
                                mb += ((u64)x[q][2] << 32) + x[q][1];
                            }
                        }
                    }
                    nb += __shfl_xor_sync(0xffffffffu, nb, kFine);
                    mb += __shfl_xor_sync(0xffffffffu, mb, kFine);
                    const uint32_t before_c = c_group + warp_scan(lane < kFine ? nb : 0, lane) - nb;
                    const u64 before = m_group + warp_scan(lane < kFine ? mb : 0, lane) - mb;
                    const uint32_t hits = __ballot_sync(0xffffffffu, lane < kFine && reached(before_c, before, nb, mb));
                    found = group * kFine + __ffs(hits) - 1;
                    if (lane == __ffs(hits) - 1) {
                        s.above_count = before_c;
                        s.above_mass = before;
                        s.bin_count = nb;
                    }
                }
                if (lane == 0) { s.bin = found; s.target = target; }
            }
            __syncthreads();
            bin = s.bin;
            above_count = s.above_count;
            above_mass = s.above_mass;
            n_in = s.bin_count;
            target = s.target;
        };
        bool ties = top_k == 1, none = false;
        if (ties) {
            key_lo = key_hi = ordered(top);
        } else {
            // the row's mass and the first histogram in one pass
            if (!by_mass) count_pass<FP32, CTAS>(l, wt.half_top, per, counts_at);
            else mine = mass_pass<FP32, CTAS>(l, wt, per, by_count, counts_at, los_at, his_at);
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
            bin1 = kFirst + (float)bin;
        }
        // the entries of the bin, or of the keys in question: how many, and the first kList of each part put down
        int in_part = 0;
        auto collect = [&]() {
            for_passing(l, [&](float x) { return bin_of(x, wt.half_top, per) == bin1; }, [&](float x, int i, bool there) {
                const uint32_t key = ordered(x);
                if (!there || key < key_lo || key > key_hi) return;
                const int at = atomicAdd(&s.n_list, 1);
                if (at < kList) s.part_entry[at] = (u64)key << 32 | (uint32_t)~i;
            });
            team_sync();
            in_part = (int)of_parts_u32(&s.n_list);
            return __reduce_add_sync(0xffffffffu, (uint32_t)in_part);
        };
        if (!ties && !none) n_in = collect();
        if (!ties && !none && n_in > (uint32_t)kList) {       // too many: on by the bits of the bin's keys
            uint32_t lo = 0xffffffffu, hi = 0;
            for_passing(l, [&](float x) { return bin_of(x, wt.half_top, per) == bin1; }, [&](float x, int, bool) {
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
                for_passing(l, [&](float x) { return bin_of(x, wt.half_top, per) == bin1; }, [&](float x, int, bool there) {
                    const uint32_t key = ordered(x);
                    if (there && key >= key_lo && key <= key_hi) into_bin((int)((key_hi - key) >> down), by_mass ? wt(x) : 0);
                });
                find_bin(false);
                const uint32_t end = key_hi - ((uint32_t)bin << down), span = (1u << down) - 1u;
                key_lo = end - key_lo > span ? end - span : key_lo;
                key_hi = end;
                team_sync();                  // (the bins may be cleared again)
            }
            ties = key_lo == key_hi;
            if (!ties) {
                if (t == 0) s.n_list = 0;
                __syncthreads();
                collect();
            }
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
            for (int j = vec0 + lane; j < vec1; j += 32) {
                float x[N];
                decode<FP32>(l.get(j), x);
#pragma unroll
                for (int e = 0; e < N; ++e) n += ordered(x[e]) == key_lo ? 1u : 0u;
            }
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0) s.warp_a[warp] = n;
            if (t == 0) s.found = -1;
            __syncthreads();
            const uint32_t in_warp = lane < kWarps ? s.warp_a[lane] : 0;
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
                        decode<FP32>(l.get(j), x);
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
            const int n = (int)n_in;
            const int upto = warp_scan(in_part, lane);
#pragma unroll 1
            for (int i0 = 0; i0 < n; i0 += kThreads) {
                const int i = i0 + t;
                int from = 0, first = 0;      // entry i: of which part, and that part's first
#pragma unroll
                for (int r = 0; r < kMaxParts - 1; ++r) {
                    const int end = __shfl_sync(0xffffffffu, upto, r);
                    if (r + 1 < parts && i >= end) { from = r + 1; first = end; }
                }
                if (i >= n) continue;
                const u64 x = parts > 1 ? remote_u64(&s.part_entry[i - first], from) : s.part_entry[i];
                s.entry[i] = make_ulonglong2(x, by_mass ? wt(unordered((uint32_t)(x >> 32))) : 0);
            }
            if (t == 0) s.found = 0;
            __syncthreads();
            // Of m entries the last that is kept: the largest at which a limit is reached, or zero; next: the smallest at which none is.  What stands before an entry is counted and
            // weighed by 1 to 32 threads.
            auto last_kept = [&](int m, auto entry, u64& next) {
                int each = 1;
                while (each < 32 && m * each * 2 <= kThreads) each *= 2;
                u64 last = 0;
                next = ~0ull;
#pragma unroll 1
                for (int i0 = 0; i0 < m; i0 += kThreads / each) {
                    const int i = i0 + t / each;
                    const u64 own = i < m ? entry(i) : 0;
                    u64 mass = 0;
                    uint32_t rank = 0;
#pragma unroll 4
                    for (int j = t & (each - 1); j < n; j += each) {
                        const ulonglong2 o = s.entry[j];
                        if (o.x >= own) { ++rank; mass += o.y; }
                    }
                    for (int o = each / 2; o; o >>= 1) { rank += __shfl_xor_sync(0xffffffffu, rank, o); mass += __shfl_xor_sync(0xffffffffu, mass, o); }
                    const bool is = (u64)above_count + rank >= (u64)top_k || above_mass + mass >= target;
                    if (i < m && is) last = max(last, own);
                    if (i < m && !is) next = min(next, own);
                }
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    const u64 x = __shfl_xor_sync(0xffffffffu, last, o), y = __shfl_xor_sync(0xffffffffu, next, o);
                    last = max(last, x);
                    next = min(next, y);
                }
                if (lane == 0) { s.scan[warp] = last; s.warp_sum[warp] = next; }
                __syncthreads();
                last = s.scan[lane % kWarps];
                next = s.warp_sum[lane % kWarps];
#pragma unroll
                for (int o = kWarps / 2; o; o >>= 1) {
                    const u64 x = __shfl_xor_sync(0xffffffffu, last, o), y = __shfl_xor_sync(0xffffffffu, next, o);
                    last = max(last, x);
                    next = min(next, y);
                }
                __syncthreads();
                return last;
            };
            // A long list: some entries from all over it first, then those between the two of them where the cut lies (18 rows of 128 000 in bf16: 46 -> 38 us).
            u64 next;
            if (n <= 3 * kSome) {
                cut = last_kept(n, [&](int i) { return s.entry[i].x; }, next);
            } else {
                cut = last_kept(kSome, [&](int i) { return s.entry[i * n / kSome].x; }, next);
                u64* const between = reinterpret_cast<u64*>(s.count);              // (nobody reads the bins any more)
                for (int i = t; i < n; i += kThreads) {
                    const u64 x = s.entry[i].x;
                    if (x > cut && x < next) between[atomicAdd(&s.found, 1)] = x;
                }
                __syncthreads();
                const int m = s.found;
                if (m > 0) cut = max(cut, last_kept(m, [&](int i) { return between[i]; }, next));
            }
        }
    }

    // --- the kept mass, stretch by stretch, and the token
    const Kept kept = {wt, least, (uint32_t)(cut >> 32), (int)~(uint32_t)cut};
    // (a float that lies below the last one kept needs no weight)
    float floor_x = cut == 0 ? -3.402823466e38f : unordered(kept.key);             // (minus infinity never passes: it also stands for what is no token)
    if (least > 0) floor_x = fmaxf(floor_x, (float)(wt.max + ((double)log2f(min_p) - 0.01) / c) - fabsf(2.f * wt.half_top) * 0x1p-20f);
    mine = all_kept ? sum_pass<FP32, CTAS>(l, wt) : kept_pass(l, kept, floor_x);
    const u64 stretch = warp_sum_u64(mine);
    if (lane == 0) s.warp_sum[warp] = stretch;
    __syncthreads();
    const u64 in_warp = s.warp_sum[lane % kWarps];
    u64 before = warp_sum_u64<kWarps>(lane % kWarps < warp ? in_warp : 0), all = warp_sum_u64<kWarps>(in_warp);
    if (parts > 1) {
        if (t == 0) s.sum = all;
        team_sync();
        const u64 of_part = lane % kMaxParts < parts ? remote_u64(&s.sum, lane % kMaxParts) : 0;
        before += warp_sum_u64<kMaxParts>(lane % kMaxParts < part ? of_part : 0);
        all = warp_sum_u64<kMaxParts>(of_part);
    }
    const u64 at = times(all, u, false);      // below all, since u is below 1
    auto answer = [&](int i) {
        const float x = l.at((int64_t)i + row.skew);
        a.ids[row_i] = i;
        if (a.logprobs) a.logprobs[row_i] = (float)(((double)x - wt.max) / (double)temperature - log((double)all / scale));
    };
    if (at >= before && at < before + stretch) {                  // the warp that has it
        u64 run = before;
        for (int j0 = vec0; j0 < vec1; j0 += 32) {
            const int j = j0 + lane;
            u64 w[N], own = 0;
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = 0;
            if (j < vec1) {
                decode<FP32>(l.get(j), x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    w[e] = kept(x[e], j * N - row.skew + e);
                    own += w[e];
                }
            }
            const u64 incl = warp_scan(own, lane);
            u64 sofar = run + incl - own;
            if (at >= sofar && at < sofar + own) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (at >= sofar && at < sofar + w[e]) answer(j * N - row.skew + e);
                    sofar += w[e];
                }
            }
            run += __shfl_sync(0xffffffffu, incl, 31);
            if (run > at) break;
        }
    }
    if (parts > 1) cluster_sync_all();        // nobody's shared memory goes before it has been read
}

using Kernel = void (*)(Params);
Kernel kernel_of(bool fp32, bool hold, int ctas) {
    if (ctas == 1) return fp32 ? token_sample_kernel<true, true, 1> : token_sample_kernel<false, true, 1>;
    return fp32 ? (hold ? token_sample_kernel<true, true, 2> : token_sample_kernel<true, false, 2>)
                : (hold ? token_sample_kernel<false, true, 2> : token_sample_kernel<false, false, 2>);
}
int g_fit[2][4];                              // clusters of 1, 2, 4 and 8 CTAs that lie beside each other, with one CTA an SM and with two

}  // namespace

cudaError_t configure_token_sample() {
    for (int i = 0; i < 4; ++i) {
        const int ctas = i / 2 + 1;
        const cudaError_t e = cudaFuncSetAttribute(kernel_of(i & 1, true, ctas), cudaFuncAttributeMaxDynamicSharedMemorySize, held_bytes(ctas));
        if (e != cudaSuccess) return e;
    }
    for (int ctas = 1; ctas <= 2; ++ctas)
        for (int k = 0; k < 4; ++k) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(1u << k);
            cfg.blockDim = dim3(kThreads);
            cfg.dynamicSmemBytes = held_bytes(ctas);
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 1u << k;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            const cudaError_t e = cudaOccupancyMaxActiveClusters(&g_fit[ctas - 1][k], kernel_of(true, true, ctas), &cfg);
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

mt_status launch_token_sample(const SampleArgs& a, const OpContext& c, cudaStream_t s) {
    Params p;
    p.a = a;
    const int vec = a.fp32 ? 4 : 8, most = (a.vocab + 2 * vec - 2) / vec;          // vectors of a row that starts anywhere
    auto vecs = [&](int parts) { return (most + parts * kWarps - 1) / (parts * kWarps); };
    auto fits = [&](int parts, int ctas) { return (int64_t)vecs(parts) * kWarps * 16 <= held_bytes(ctas); };
    // Parts: as many as make clusters that all lie beside each other, held, with one CTA an SM: then they spread over the SMs, and a thread has more registers (15 rows of
    // 128 000 in bf16: 22 us in eight parts, 33 in four, 16 rows 50 and 37, for clusters of eight do not fill the SMs; 64 rows of 32 000: 21 in two, 23 in four with two CTAs an
    // SM; 74 rows 23, 27 and 29; 146 rows of 16 000: 20 in one part, 24 in two).  Where that leaves long parts, two CTAs an SM, of different rows, do better, if they fill the SMs
    // and are held (before the list was ranked in two steps: 64 rows of 128 000 56 us in four parts, 72 in two with one CTA an SM; 33 rows 42 and 46; 18 rows, which do not fill them, 42 and 37).
    auto most_parts = [&](int ctas) {
        int k = 3;
        while (k >= 0 && !(a.n <= g_fit[ctas - 1][k] && (k == 0 || a.vocab >> k >= kMinPart) && fits(1 << k, ctas))) --k;
        return k;
    };
    const int one = most_parts(1), two = most_parts(2);
    const int ctas = one >= 0 && (a.vocab >> one <= kShortPart || two < 0 || a.n << two <= c.sm_count) ? 1 : 2;
    int k = ctas == 1 ? one : two;
    // More rows, with two CTAs an SM: as few parts as can be held (107 rows of 73 187 in fp32: 48 us in four, 61 in two).  Rows that are not held: as many as lie beside each other,
    // at least two, so that no more of them are under way at once than L2 holds (512 rows of 128 000 in fp32: 174 us in two, 200 in one, 193 in four).
    if (k < 0) {
        for (k = 0; k < 2 && !fits(1 << k, 2);) ++k;
        if (!fits(1 << k, 2))
            for (k = 3; k > 1 && a.n > g_fit[1][k];) --k;
    }
    p.parts = 1 << k;
    p.vecs = vecs(p.parts);
    const bool hold = fits(p.parts, ctas);
    p.shift = 46;
    while (a.vocab > 1ll << (62 - p.shift)) --p.shift;          // (a vocabulary below 2^30 leaves 32 at least)
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
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel_of(a.fp32, hold, ctas), p);
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

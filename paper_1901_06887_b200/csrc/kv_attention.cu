// Attention of one new token per sequence over the paged 4-bit cache.
//
// Mathematics.  For one sequence and one key/value head, with the g query heads that share it as columns:
//   S = K q (tokens x heads), p = exp(S - m), o = sum p v / sum p, one pass with a running maximum m per head.
// K and V rows are code * scale + bias.  The codes enter the matrix instructions as the exact bf16 numbers 16 + code (four bits
// put in the top of a mantissa: one shift and one and-or per two codes, no conversion), and everything else is applied in
// fp32 outside:
//   S    = scale_k (sum_d (16 + code) q_d) + (bias_k - 16 scale_k) sum_d q_d
//   o    = sum P (16 + code) - 24 sum P + sum p (8 scale_v + bias_v),   P = bf16(p scale_v)
// P is the only rounding on the way; subtracting 24 times the ROUNDED P leaves its error relative to the centred codes
// (code - 8), not to 16 + code.
//
// Bound: memory.  head_dim + 8 bytes per cached token and head; the arithmetic is some 200 warp instructions per 16 tokens.
//
// Split.  A unit is 128 tokens of one (sequence, head); the units of the whole batch, in order, are cut into equal
// contiguous shares, one per CTA, so ragged batches balance without a schedule from the host: every CTA adds up the lengths itself and
// finds its own start.  A CTA that holds all of a (sequence, head) writes the output; else its part goes to scratch and the last CTA
// to arrive joins the parts in order (the result does not depend on who is last).  Within a unit each of the four warps
// takes 32 tokens with statistics of its own; warps join at the end of the (sequence, head).
//
// Operand layout.  The inner index of a product may be permuted freely as long as both sides agree, so a lane loads 16
// (head_dim 128) contiguous bytes of a key row and calls them its slice of every k step; queries are permuted once to match.  For the
// values the pairs of a register have to be two tokens of one channel: two byte permutes interleave the words of neighbouring tokens.
// Nothing passes through shared memory on the way in.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kWarps = 4, kTile = 32, kUnit = kWarps * kTile;

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3,
                                         const uint32_t b0, const uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Codes in nibbles P and P + 4 of w as two bf16 numbers 16 + code.
template <int P>
__device__ __forceinline__ uint32_t codes16(uint32_t w) {
    const uint32_t s = P == 0 ? w << 3 : w >> (4 * P - 3);
    return (s & 0x00780078u) | 0x41804180u;
}

template <int BYTES> struct Words;
template <> struct Words<16> { uint4 v; __device__ uint32_t operator[](int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; } };
template <> struct Words<8> { uint2 v; __device__ uint32_t operator[](int i) const { return i == 0 ? v.x : v.y; } };
template <> struct Words<4> { uint32_t v; __device__ uint32_t operator[](int) const { return v; } };
template <int BYTES>
__device__ __forceinline__ Words<BYTES> load_words(const uint8_t* p) {
    Words<BYTES> w;
    w.v = __ldg(reinterpret_cast<const decltype(w.v)*>(p));
    return w;
}

struct DecodeArgs {
    KvAttentionArgs a;
    int page_shift;
    int64_t max_len;            // longest length the tables can hold
    int group;                  // query heads per key/value head
    unsigned* arrived;          // [n_seqs * kv_heads], zero between calls
    float* part_o;              // [2 * CTAs][GT * 8][D]
    float* part_ml;             // [2 * CTAs][GT * 8][2]
};

__device__ __forceinline__ int units_of(const DecodeArgs& p, int s) {
    const int n = p.a.lengths[s];
    return n <= 0 || n > p.max_len ? 0 : (n + kUnit - 1) / kUnit;
}

// P16: pages of 16 tokens, so the halves of a tile lie in different pages; all larger pages hold whole tiles.
template <int D, int GT, bool P16>
__global__ void __launch_bounds__(kWarps * 32, GT == 1 ? 4 : 2) kv_attention_kernel(DecodeArgs p) {
    constexpr int kSteps = D / 16;             // k steps of S
    constexpr int kMt = D / 16;                // 16-row tiles of o
    constexpr int KB = D / 8, VB = D / 16;     // bytes of a key / value row per lane
    constexpr int H = GT * 8;
    __shared__ float s_o[kWarps][H][D + 4];
    __shared__ float s_m[kWarps][H], s_l[kWarps][H];
    __shared__ int64_t s_scan[kWarps + 1];
    __shared__ int s_seq;
    __shared__ int64_t s_base;
    __shared__ int s_last;

    const KvAttentionArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int heads = a.c.kv_heads, n_seqs = a.n_seqs;
    pdl_launch_dependents();
    pdl_wait();

    // --- sequences without units: zeros, or NaN where the length is out of range
    for (int s = blockIdx.x; s < n_seqs; s += gridDim.x) {
        if (units_of(p, s) > 0) continue;
        const bool bad = a.lengths[s] != 0;
        if (bad && tid == 0) raise_status(a.status, MT_ERR_INVALID_ARG, s);
        uint32_t* o = reinterpret_cast<uint32_t*>(a.out + (int64_t)s * a.q_heads * D);
        for (int i = tid; i < a.q_heads * D / 2; i += kWarps * 32) o[i] = bad ? 0x7fff7fffu : 0u;
    }

    // --- this CTA's share of the units: [begin, end); its first sequence and that sequence's first unit
    const int per = (n_seqs + kWarps * 32 - 1) / (kWarps * 32);
    int64_t mine = 0;
    for (int i = 0; i < per; ++i) {
        const int s = tid * per + i;
        if (s < n_seqs) mine += (int64_t)units_of(p, s) * heads;
    }
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
    }
    const int64_t share = (total + gridDim.x - 1) / gridDim.x;
    const int64_t begin = share * blockIdx.x, end = min(begin + share, total);
    if (begin >= end) return;
    {
        int64_t base = before + incl - mine;
        if (base <= begin && begin < base + mine) {
            int s = tid * per;
            for (;; ++s) {
                const int64_t u = (int64_t)units_of(p, s) * heads;
                if (begin < base + u) break;
                base += u;
            }
            s_seq = s;
            s_base = base;
        }
    }
    __syncthreads();
    int seq = s_seq;
    int64_t seq_base = s_base;

    const uint8_t *kc = static_cast<const uint8_t*>(a.c.k_codes), *vc = static_cast<const uint8_t*>(a.c.v_codes);
    const uint32_t *kp = static_cast<const uint32_t*>(a.c.k_params), *vp = static_cast<const uint32_t*>(a.c.v_params);
    const float to_log2 = a.scale * 1.44269504088896341f;

    for (int64_t at = begin; at < end;) {
        // --- the (sequence, head) that unit `at` belongs to
        int units = units_of(p, seq);
        while (at >= seq_base + (int64_t)units * heads) {
            seq_base += (int64_t)units * heads;
            units = units_of(p, ++seq);
        }
        const int head = (int)((at - seq_base) / units);
        const int64_t seg0 = seq_base + (int64_t)head * units, seg1 = seg0 + units;
        const int u0 = (int)(at - seg0), u1 = (int)(min(seg1, end) - seg0);
        const int len = a.lengths[seq];
        const int32_t* table = a.tables + (int64_t)seq * a.table_width;

        // --- queries: columns g (+ 8) of the B operand, and the sums of columns 2 t, 2 t + 1
        uint32_t qf[GT][kSteps][2];
        float qsum[GT][2];
#pragma unroll
        for (int n = 0; n < GT; ++n) {
            const int h = n * 8 + g;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < kSteps / 2; ++j) {
                uint4 w = make_uint4(0, 0, 0, 0);
                if (h < p.group)
                    w = __ldg(reinterpret_cast<const uint4*>(a.q + seq * a.q_seq_stride + (int64_t)(head * p.group + h) * a.q_head_stride +
                                                             t * (D / 4) + 8 * j));
                qf[n][2 * j][0] = __byte_perm(w.x, w.z, 0x5410);
                qf[n][2 * j][1] = __byte_perm(w.x, w.z, 0x7632);
                qf[n][2 * j + 1][0] = __byte_perm(w.y, w.w, 0x5410);
                qf[n][2 * j + 1][1] = __byte_perm(w.y, w.w, 0x7632);
                sum += ((bf16_lo(w.x) + bf16_hi(w.x)) + (bf16_lo(w.y) + bf16_hi(w.y))) + ((bf16_lo(w.z) + bf16_hi(w.z)) + (bf16_lo(w.w) + bf16_hi(w.w)));
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            qsum[n][0] = __shfl_sync(0xffffffffu, sum, 8 * t) * to_log2;
            qsum[n][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4) * to_log2;
        }

        float o[GT][kMt][4];
        float m[GT][2], l[GT][2], r[GT][2], z[GT][2];
#pragma unroll
        for (int n = 0; n < GT; ++n) {
#pragma unroll
            for (int i = 0; i < kMt; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = r[n][e] = z[n][e] = 0.f; }
        }
        bool bad = false;

        // --- tiles of 32 tokens: warp, warp + 4, ...
        Words<KB> kw[2][2];
        Words<VB> vw[2][4];
        uint32_t kpar = 0, vpar = 0;
        int page0 = 0, page1 = 0;
        const int stop = min(len, u1 * kUnit);
        int tok = u0 * kUnit + warp * kTile;

        auto fetch_pages = [&](int tk) {                    // (a second half past the end reads the first half's page)
            if (tk >= stop) return;
            page0 = __ldg(table + (tk >> p.page_shift));
            if ((unsigned)page0 >= (unsigned)a.c.n_pages) { bad = true; page0 = 0; }
            if (P16) {
                page1 = tk + 16 < len ? __ldg(table + (tk >> 4) + 1) : page0;
                if ((unsigned)page1 >= (unsigned)a.c.n_pages) { bad = true; page1 = 0; }
            }
        };
        int64_t row0 = 0, row1 = 0;                         // cache rows of the tile's halves
        auto set_rows = [&](int tk) {
            row0 = (((int64_t)page0 * heads + head) << p.page_shift) + (tk & ((1 << p.page_shift) - 1));
            row1 = P16 ? (((int64_t)page1 * heads + head) << p.page_shift) : row0 + 16;
        };
        auto load_k = [&](int tk) {
            if (tk >= stop) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) kw[e >> 1][e & 1] = load_words<KB>(kc + ((e < 2 ? row0 : row1) + g + 8 * (e & 1)) * (D / 2) + t * KB);
            kpar = __ldg(kp + (lane < 16 ? row0 : row1) + (lane & 15));
        };
        auto load_v = [&](int tk) {
            if (tk >= stop) return;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                vw[e >> 2][e & 3] = load_words<VB>(vc + ((e < 4 ? row0 : row1) + 2 * t + (e & 1) + 8 * ((e >> 1) & 1)) * (D / 2) + g * VB);
            vpar = __ldg(vp + (lane < 16 ? row0 : row1) + (lane & 15));
        };

        fetch_pages(tok);
        if (tok < stop) set_rows(tok);
        load_k(tok);
        load_v(tok);
        fetch_pages(tok + kUnit);
        for (; tok < stop; tok += kUnit) {
            const int next = tok + kUnit;
            // S of both halves
            float s[GT][2][4];
#pragma unroll
            for (int n = 0; n < GT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) s[n][h][0] = s[n][h][1] = s[n][h][2] = s[n][h][3] = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < kSteps / 2; ++j) {
                    const uint32_t w0 = kw[h][0][j], w1 = kw[h][1][j];
                    const uint32_t a00 = codes16<0>(w0), a01 = codes16<1>(w0), a02 = codes16<2>(w0), a03 = codes16<3>(w0);
                    const uint32_t a10 = codes16<0>(w1), a11 = codes16<1>(w1), a12 = codes16<2>(w1), a13 = codes16<3>(w1);
#pragma unroll
                    for (int n = 0; n < GT; ++n) {
                        mma_bf16(s[n][h], a00, a10, a01, a11, qf[n][2 * j][0], qf[n][2 * j][1]);
                        mma_bf16(s[n][h], a02, a12, a03, a13, qf[n][2 * j + 1][0], qf[n][2 * j + 1][1]);
                    }
                }
            const uint32_t kq = kpar;
            uint32_t vq = vpar;
            if (tok + lane >= len) vq = 0;               // what lies past the length adds nothing, whatever it holds
            if (next < stop) set_rows(next);
            load_k(next);
            // scores in units of log2, tokens past the length out
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int i = 16 * h + 8 * e + g;
                    const uint32_t w = __shfl_sync(0xffffffffu, kq, i);
                    const float ks = bf16_lo(w), beta = fmaf(-16.f, ks, bf16_hi(w)), ksc = ks * to_log2;
                    const bool in = tok + i < len;
#pragma unroll
                    for (int n = 0; n < GT; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float& x = s[n][h][2 * e + c];
                            x = in ? fmaf(ksc, x, beta * qsum[n][c]) : -INFINITY;
                        }
                }
            bool grow = false;
            float top[GT][2];
#pragma unroll
            for (int n = 0; n < GT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = fmaxf(fmaxf(s[n][0][c], s[n][0][2 + c]), fmaxf(s[n][1][c], s[n][1][2 + c]));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                    top[n][c] = x;
                    grow = grow || x > m[n][c] + 8.f;
                }
            // the running maximum moves only when it has to: powers up to 2^8 are as exact in bf16 and fp32
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int n = 0; n < GT; ++n) {
                    float f[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float nm = fmaxf(m[n][c], top[n][c]);
                        f[c] = m[n][c] == nm ? 1.f : ex2(m[n][c] - nm);
                        m[n][c] = nm;
                        l[n][c] *= f[c]; r[n][c] *= f[c]; z[n][c] *= f[c];
                    }
#pragma unroll
                    for (int i = 0; i < kMt; ++i) { o[n][i][0] *= f[0]; o[n][i][1] *= f[1]; o[n][i][2] *= f[0]; o[n][i][3] *= f[1]; }
                }
            }
            uint32_t pf[GT][2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t w = __shfl_sync(0xffffffffu, vq, 16 * h + 8 * e + g);
                    const float vs = bf16_lo(w), mid = fmaf(8.f, vs, bf16_hi(w));
#pragma unroll
                    for (int n = 0; n < GT; ++n) {
                        const float p0 = ex2(s[n][h][2 * e] - m[n][0]), p1 = ex2(s[n][h][2 * e + 1] - m[n][1]);
                        const uint32_t pk = pack_bf16x2(p0 * vs, p1 * vs);
                        l[n][0] += p0; l[n][1] += p1;
                        z[n][0] = fmaf(p0, mid, z[n][0]); z[n][1] = fmaf(p1, mid, z[n][1]);
                        r[n][0] += bf16_lo(pk); r[n][1] += bf16_hi(pk);
                        pf[n][h][e] = transpose8x8(pk);
                    }
                }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < VB / 4; ++j) {
                    const uint32_t lo0 = __byte_perm(vw[h][0][j], vw[h][1][j], 0x5410), hi0 = __byte_perm(vw[h][0][j], vw[h][1][j], 0x7632);
                    const uint32_t lo1 = __byte_perm(vw[h][2][j], vw[h][3][j], 0x5410), hi1 = __byte_perm(vw[h][2][j], vw[h][3][j], 0x7632);
                    const uint32_t c0[8] = {codes16<0>(lo0), codes16<1>(lo0), codes16<2>(lo0), codes16<3>(lo0),
                                            codes16<0>(hi0), codes16<1>(hi0), codes16<2>(hi0), codes16<3>(hi0)};
                    const uint32_t c1[8] = {codes16<0>(lo1), codes16<1>(lo1), codes16<2>(lo1), codes16<3>(lo1),
                                            codes16<0>(hi1), codes16<1>(hi1), codes16<2>(hi1), codes16<3>(hi1)};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int n = 0; n < GT; ++n)
                            mma_bf16(o[n][4 * j + i], c0[2 * i], c0[2 * i + 1], c1[2 * i], c1[2 * i + 1], pf[n][h][0], pf[n][h][1]);
                }
            load_v(next);
            fetch_pages(next + kUnit);
        }
        bad = __any_sync(0xffffffffu, bad);
        if (bad && lane == 0) raise_status(a.status, MT_ERR_INVALID_ARG, seq);

        // --- join the warps
        constexpr int C = D / 8;                 // channels per lane group
        __syncthreads();                         // the previous (sequence, head) has been read
#pragma unroll
        for (int n = 0; n < GT; ++n) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], x);
                    r[n][c] += __shfl_xor_sync(0xffffffffu, r[n][c], x);
                    z[n][c] += __shfl_xor_sync(0xffffffffu, z[n][c], x);
                }
                const int h = n * 8 + 2 * t + c;
                if (g == 0) { s_m[warp][h] = m[n][c]; s_l[warp][h] = bad ? nan_f() : l[n][c]; }
                const float shift = fmaf(-24.f, r[n][c], z[n][c]);
#pragma unroll
                for (int i = 0; i < kMt; ++i)    // rotated inside the lane group's channels against bank conflicts
                    *reinterpret_cast<float2*>(&s_o[warp][h][g * C + ((2 * i + 2 * g) & (C - 1))]) =
                        make_float2(o[n][i][c] + shift, o[n][i][2 + c] + shift);
            }
        }
        __syncthreads();
        const bool whole = u0 == 0 && u1 == units;
        const int slot = 2 * blockIdx.x + (seg0 < begin ? 0 : 1);
        for (int i = tid; i < p.group * D; i += kWarps * 32) {
            const int h = i / D, d = i % D, at_d = (d / C) * C + ((d % C + 2 * (d / C)) & (C - 1));
            float mx = s_m[0][h];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) mx = fmaxf(mx, s_m[w][h]);
            float so = 0.f, sl = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = s_m[w][h] == -INFINITY && s_l[w][h] == 0.f ? 0.f : ex2(s_m[w][h] - mx);
                so += f * s_o[w][h][at_d];
                sl += f * s_l[w][h];
            }
            if (whole) {
                a.out[((int64_t)seq * a.q_heads + head * p.group + h) * D + d] = f_to_bf16(so / sl);
            } else {
                __stcg(p.part_o + ((int64_t)slot * H + h) * D + d, so);
                if (d == 0) __stcg(reinterpret_cast<float2*>(p.part_ml) + (int64_t)slot * H + h, make_float2(mx, sl));
            }
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            const int first = (int)(seg0 / share), last = (int)((seg1 - 1) / share);
            unsigned* arrived = p.arrived + (int64_t)seq * heads + head;
            if (tid == 0) {
                const unsigned n = atomicAdd(arrived, 1u);
                s_last = n == (unsigned)(last - first);
                if (s_last) *arrived = 0u;
            }
            __syncthreads();
            if (s_last) {
                __threadfence();
                for (int i = tid; i < p.group * D; i += kWarps * 32) {
                    const int h = i / D, d = i % D;
                    float mx = -INFINITY, so = 0.f, sl = 0.f;
#pragma unroll 4
                    for (int b = first; b <= last; ++b) {
                        const int64_t k = (int64_t)(2 * b + (seg0 < share * b ? 0 : 1)) * H + h;
                        const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml) + k);
                        const float x = __ldcg(p.part_o + k * D + d);
                        const float nm = fmaxf(mx, ml.x), f0 = mx == nm ? 1.f : ex2(mx - nm), f1 = ml.x == nm ? 1.f : ex2(ml.x - nm);
                        so = so * f0 + x * f1;
                        sl = sl * f0 + ml.y * f1;
                        mx = nm;
                    }
                    a.out[((int64_t)seq * a.q_heads + head * p.group + h) * D + d] = f_to_bf16(so / sl);
                }
            }
        }
        at = min(seg1, end);
    }
}

}  // namespace

cudaError_t configure_kv_attention() { return cudaSuccess; }

mt_status launch_kv_attention(const KvAttentionArgs& a, const OpContext& c, cudaStream_t s) {
    DecodeArgs p;
    p.a = a;
    p.page_shift = 4;
    while ((1 << p.page_shift) < a.c.page_tokens) ++p.page_shift;
    p.max_len = a.c.n_pages > 0 ? (int64_t)a.table_width * a.c.page_tokens : 0;
    p.group = a.q_heads / a.c.kv_heads;
    const int gt = p.group > 8 ? 2 : 1, d = a.c.head_dim;
    // as many CTAs as fit the GPU at once, but not more than there can be units
    const int64_t most = (int64_t)a.n_seqs * a.c.kv_heads * ((p.max_len + kUnit - 1) / kUnit);
    int64_t grid = (int64_t)c.sm_count * (gt == 1 ? 4 : 2);
    if (grid > most) grid = most > 1 ? most : 1;
    const size_t o_bytes = (size_t)grid * 2 * gt * 8 * d * 4, ml_bytes = (size_t)grid * 2 * gt * 8 * 8;
    uint8_t* w = nullptr;
    mt_status st = op_scratch(s, kScratchZeroBytes + o_bytes + ml_bytes, &w);
    if (st != MT_OK) return st;
    p.arrived = reinterpret_cast<unsigned*>(w);
    p.part_o = reinterpret_cast<float*>(w + kScratchZeroBytes);
    p.part_ml = reinterpret_cast<float*>(w + kScratchZeroBytes + o_bytes);
    typedef void (*Kernel)(DecodeArgs);
    static const Kernel kernels[2][2][2] = {
        {{kv_attention_kernel<64, 1, false>, kv_attention_kernel<64, 1, true>}, {kv_attention_kernel<64, 2, false>, kv_attention_kernel<64, 2, true>}},
        {{kv_attention_kernel<128, 1, false>, kv_attention_kernel<128, 1, true>}, {kv_attention_kernel<128, 2, false>, kv_attention_kernel<128, 2, true>}}};
    const Kernel k = kernels[d == 128][gt - 1][a.c.page_tokens == 16];
    return launch_pdl(k, dim3((unsigned)grid), dim3(kWarps * 32), 0, s, p) == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

// Attention of one new token per sequence over the paged 4-bit cache.
//
// Mathematics.  For one sequence and one key/value head, with the g query heads that share it as columns:
//   S = K q (tokens x heads), p = exp(S - m), o = sum p v / sum p, one pass with a running maximum m per head.
// K and V rows are code * scale + bias.  The codes go into integer matrix instructions (u8 times s8, exact 32-bit sums) as they stand:
// four codes cost one mask, or a shift and a mask, where a floating type takes two instructions for every two codes.  The other
// operand is rounded to whole numbers and cut into two signed bytes:
//   q' = 256 q1 + q2: an element of at least 2^-6 of the head's largest stays what it is, a smaller one errs by some 2^-15 of the largest at most;
//   P  = 128 P1 + P2, P = p scale_v relative to the head's largest such product in the tile: 14 bits, error at most 2^-14 of it (with 11
//        bits the result's error over long contexts doubled: the tile's largest p stands far above the rest).  The largest PRODUCT, not the
//        largest p and the largest scale_v: where one token has the weight and another the scale, as a first token of small values beside
//        ordinary ones, all products lie far below those two together and would keep few bits or none.
// Scales and biases are applied in fp32 outside:
//   S = scale_k (sum_d (code - 7.5) q'_d) + (bias_k + 7.5 scale_k) sum_d q_d
//   o = sum P (code - 8) + sum p (8 scale_v + bias_v)
// The 7.5 terms are one whole number a head, 7.5 sum (q - q'), that the integer sums start with: without it errors of the small elements that
// agree in sign (a query of one large element and many alike) met the codes' middle in every channel, and an output was off by 2 % at 1 to 64.
// The -8 is one more product (a constant row): over a long context o is a small mean of many values, and what is taken off must be
// made of the same rounded P.  Every head of a tile of 32 tokens has a scale of P of its own; the tile is added to the running o in
// fp32; its integer sums start at 1.5 * 2^23 as a bit pattern, so they need no conversion to be read as floats.
//
// Cost.  head_dim + 8 bytes per cached token and head, and 618 warp instructions per 32 tokens (head_dim 128, up to 8 query heads).  No unit is
// full (4 sequences, 448 thousand tokens): 60 % of the issue slots, logic pipe 49 %, memory 51 %; what shows are the chains of dependent
// instructions within a tile, which 4 warps a scheduler do not hide.
//
// Split.  The tiles (32 tokens of one (sequence, head)) of the whole batch, in order, are cut into equal contiguous shares, one per warp, so
// ragged batches balance without a schedule from the host: every CTA adds up the lengths itself and its warps find their own starts.  A warp
// that holds all of a (sequence, head) writes the output; else its part goes to scratch, and a second launch (its CTAs go over the sequences' query heads, most
// with nothing to do) joins the parts in order.  A warp's stream of tiles runs on across its (sequence, head)s, so short ones cost no pause: CTAs that
// took whole shares, joined their warps in shared memory and refilled their rings for every (sequence, head) spent 76 us on a batch of 64
// sequences (1 to 8000 tokens), this 61 us (63 with P relative to the largest product).
//
// Operand layout.  The inner index of a product may be permuted freely as long as both sides agree, so a lane loads 16
// (head_dim 128) contiguous bytes of a key row and calls them its slice of every k step; queries are permuted once to match.  For the
// values the four bytes of a register have to be four tokens of one channel: byte permutes turn four tokens' words over.
//
// Feed.  Every warp copies its own tiles into a ring of three in shared memory (cp.async, 4.25 KB a tile), two tiles ahead of the one it
// computes: 16 warps then have up to 139 KB of an SM in flight.  Loading straight into registers one tile ahead left the kernel
// waiting on memory (163 us in the case below, and registers spilled).
//
// Measured on the way (4 sequences, 448 thousand tokens in all, 8 heads): codes as bf16 (16 + code by shift, and-or) 169 us, bound by the
// logic pipe, which takes two cycles a warp instruction; shifts moved to the multiplier 186 us; codes as e4m3 (c * 2^-9 for every nibble) 216 us: that form of the
// instruction is carried out through conversions, 6 cycles per SM against 2 for the integer one.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kWarps = 4, kTile = 32;
constexpr int kMinShare = 2;                 // tiles of a warp, at least
constexpr int kMaxParts = 256;               // parts of a (sequence, head), about: joining them is the work of one CTA

// D = A B + C, 16 x 8 x 32, unsigned times signed bytes.
__device__ __forceinline__ void mma_u8s8(int (&d)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3,
                                         const uint32_t (&b)[2], const int (&c)[4]) {
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
// The power of two that brings the bf16 number with these bits into [2^14, 2^15), and its reciprocal (both normal numbers for every exponent); with
// a mantissa of ones into [2^13, 2^14), as 2^15 - 2^7 has no high byte.  A power of two: elements within 2^6 of the largest are whole numbers then.
__device__ __forceinline__ void query_scale(uint32_t bits, float& up, float& down) {
    const int e = max((int)((bits + 0x10000u) >> 23 & 255u), 22);
    up = __int_as_float((268 - e) << 23);
    down = __int_as_float((e - 14) << 23);
}
// 1.5 * 2^23: adding it to a small float leaves the nearest integer in the low bits; integer sums that start at its bits are floats.
constexpr float kMagic = 12582912.f;
constexpr int kMagicBits = 0x4b400000;
__device__ __forceinline__ uint32_t whole(float x, float y) { return __float_as_uint(fmaf(x, y, kMagic)); }
// The factor that brings the products of a column, the largest of which has the exponent of `bits`, to below 2^14 - 1/2, and its reciprocal:
// a power of two, times 1 - 2^-14 and 1 + 2^-14.  P then is 2^14 - 1 at most, and P1 stays within 127.  (32 such P times 8 stay below 2^22, what
// kMagic leaves room for.)  Products below 2^-106 of the largest weight's lose bits.
__device__ __forceinline__ void product_scale(uint32_t bits, float& up, float& down) {
    const uint32_t e = max(bits & 0x7f800000u, 21u << 23);
    up = __uint_as_float((267u << 23) - 1024u - e);
    down = __uint_as_float(e + 512u - (13u << 23));
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// y += (x - kMagic) * s on pairs.
__device__ __forceinline__ void add_scaled(float2& y, int x0, int x1, float s0, float s1) {
    asm("{\n\t.reg .b64 x, s, y, m;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 s, {%4, %5};\n\tmov.b64 y, {%0, %1};\n\tmov.b64 m, {%6, %6};\n\t"
        "add.rn.f32x2 x, x, m;\n\tfma.rn.f32x2 y, x, s, y;\n\tmov.b64 {%0, %1}, y;\n\t}"
        : "+f"(y.x), "+f"(y.y) : "r"(x0), "r"(x1), "f"(s0), "f"(s1), "f"(-kMagic));
}
// Whole numbers of 16 bits in x, y, z, w: their high and low bytes, the low ones signed.
__device__ __forceinline__ void split_bytes(int x, int y, int z, int w, uint32_t& high, uint32_t& low) {
    low = __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
    x += 128; y += 128; z += 128; w += 128;
    high = __byte_perm(__byte_perm(x, y, 0x0051), __byte_perm(z, w, 0x0051), 0x5410);
}

template <int BYTES> struct Words;
template <> struct Words<16> { uint4 v; __device__ uint32_t operator[](int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; } };
template <> struct Words<8> { uint2 v; __device__ uint32_t operator[](int i) const { return i == 0 ? v.x : v.y; } };
template <> struct Words<4> { uint32_t v; __device__ uint32_t operator[](int) const { return v; } };
template <int BYTES>
__device__ __forceinline__ Words<BYTES> read_words(const uint8_t* p) {
    Words<BYTES> w;
    w.v = *reinterpret_cast<const decltype(w.v)*>(p);
    return w;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

constexpr int kStages = 3;
template <int D>
struct Ring {
    static constexpr int kRows = kTile * D / 2;              // bytes of a tile's key (or value) codes
    static constexpr int kStage = 2 * kRows + 2 * kTile * 4; // keys, values, key parameters, value parameters
    static constexpr int kWarp = kStages * kStage;
};

constexpr int kv_shared_bytes(int d) { return kWarps * kStages * (kTile * d + 2 * kTile * 4); }
constexpr int kJoinThreads = 128;

// What the warp that starts a (sequence, head) leaves for the second launch.
struct Split {
    int first, parts;           // that warp; parts: 0 if there is nothing to join
};

struct DecodeArgs {
    KvAttentionArgs a;
    int page_shift;
    int64_t max_len;            // longest length the tables can hold
    int group;                  // query heads per key/value head
    Split* split;               // [n_seqs * kv_heads]
    float* part_o;              // [2 * warps][GT * 8][D]: the part that came in, the part that goes on
    float* part_ml;             // [2 * warps][GT * 8][2]
};

__device__ __forceinline__ int tiles_of(const DecodeArgs& p, int s) {
    const int n = p.a.lengths[s];
    return n <= 0 || n > p.max_len ? 0 : (n + kTile - 1) / kTile;
}

// P16: pages of 16 tokens, so the halves of a tile lie in different pages; all larger pages hold whole tiles.
template <int D, int GT, bool P16>
__global__ void __launch_bounds__(kWarps * 32, GT == 1 ? 4 : 2) kv_attention_kernel(DecodeArgs p) {
    constexpr int kSteps = D / 32;             // k steps of S
    constexpr int kMt = D / 16;                // 16-row tiles of o
    constexpr int KB = D / 8, VB = D / 16;     // bytes of a key / value row per lane
    constexpr int H = GT * 8;
    extern __shared__ __align__(128) uint8_t s_bytes[];          // the warps' rings
    uint8_t* const ring = s_bytes + (threadIdx.x / 32) * Ring<D>::kWarp;
    __shared__ int64_t s_scan[kWarps], s_base[kWarps];
    __shared__ int s_longest[kWarps], s_seq[kWarps];

    const KvAttentionArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int heads = a.c.kv_heads, n_seqs = a.n_seqs;
    pdl_launch_dependents();
    pdl_wait();

    // --- sequences without tiles: zeros, or NaN where the length is out of range
    for (int s = blockIdx.x; s < n_seqs; s += gridDim.x) {
        if (tiles_of(p, s) > 0) continue;
        const bool bad = a.lengths[s] != 0;
        if (bad && tid == 0) raise_status(a.status, MT_ERR_INVALID_ARG, s);
        for (int h = tid; h < heads; h += kWarps * 32) p.split[(int64_t)s * heads + h].parts = 0;
        uint32_t* o = reinterpret_cast<uint32_t*>(a.out + (int64_t)s * a.q_heads * D);
        for (int i = tid; i < a.q_heads * D / 2; i += kWarps * 32) o[i] = bad ? 0x7fff7fffu : 0u;
    }

    // --- this warp's share of the tiles: [begin, end); its first sequence and that sequence's first tile
    const int per = (n_seqs + kWarps * 32 - 1) / (kWarps * 32);
    int64_t mine = 0;
    int longest = 0;
    for (int i = 0; i < per; ++i) {
        const int s = tid * per + i;
        const int u = s < n_seqs ? tiles_of(p, s) : 0;
        mine += (int64_t)u * heads;
        longest = max(longest, u);
    }
    longest = __reduce_max_sync(0xffffffffu, longest);
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) { s_scan[warp] = incl; s_longest[warp] = longest; }
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
        longest = max(longest, s_longest[w]);
    }
    const int64_t warps = (int64_t)gridDim.x * kWarps, me = (int64_t)blockIdx.x * kWarps + warp;
    const int64_t share = max(max((total + warps - 1) / warps, (int64_t)kMinShare), (int64_t)(longest + kMaxParts - 1) / kMaxParts);
    {
        const int64_t base = before + incl - mine;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const int64_t first = share * ((int64_t)blockIdx.x * kWarps + w);
            if (base <= first && first < base + mine) {
                int64_t at = base;
                int s = tid * per;
                for (;; ++s) {
                    const int64_t u = (int64_t)tiles_of(p, s) * heads;
                    if (first < at + u) break;
                    at += u;
                }
                s_seq[w] = s;
                s_base[w] = at;
            }
        }
    }
    __syncthreads();
    const int64_t begin = share * me;
    if (begin >= total) return;
    int left = (int)min(share, total - begin);               // tiles still to be computed

    const uint8_t *kc = static_cast<const uint8_t*>(a.c.k_codes), *vc = static_cast<const uint8_t*>(a.c.v_codes);
    const uint32_t *kp = static_cast<const uint32_t*>(a.c.k_params), *vp = static_cast<const uint32_t*>(a.c.v_params);
    const float to_log2 = fabsf(a.scale) * 1.44269504088896341f;

    // --- the stream of tiles.  Where the next tile to be copied lies, with its pages already looked up:
    int f_seq = s_seq[warp], f_units = tiles_of(p, f_seq), f_head, f_tile, f_left = left;
    {
        const int64_t in_seq = begin - s_base[warp];
        f_head = (int)(in_seq / f_units);
        f_tile = (int)(in_seq - (int64_t)f_head * f_units);
    }
    int seq = f_seq, head = f_head, tile0 = f_tile, units = f_units;       // the (sequence, head) being computed, from tile tile0 on
    int page0 = 0, page1 = 0;
    auto fetch_pages = [&]() {                               // (a second half past the end reads the first half's page)
        if (f_left <= 0) return;
        const int32_t* const at = a.tables + (int64_t)f_seq * a.table_width + ((f_tile * kTile) >> p.page_shift);
        page0 = __ldg(at);
        if (P16) page1 = f_tile * kTile + 16 < a.lengths[f_seq] ? __ldg(at + 1) : page0;
    };
    unsigned bad_pages = 0;                                  // by place in the ring
    auto fetch = [&](int place) {                            // the next tile to a place in the ring; pages of the tile after it
        bad_pages &= ~(1u << place);
        if (f_left > 0) {
            --f_left;
            if ((unsigned)page0 >= (unsigned)a.c.n_pages) { bad_pages |= 1u << place; page0 = 0; }
            if (P16 && (unsigned)page1 >= (unsigned)a.c.n_pages) { bad_pages |= 1u << place; page1 = 0; }
            // cache rows of the tile's halves
            const int64_t row0 = (((int64_t)page0 * heads + f_head) << p.page_shift) + ((f_tile * kTile) & ((1 << p.page_shift) - 1));
            const int64_t row1 = P16 ? (((int64_t)page1 * heads + f_head) << p.page_shift) : row0 + 16;
            const uint32_t dst = smem_u32(ring) + place * Ring<D>::kStage + lane * 16;
            constexpr int CH = D / 32;                       // 16-byte pieces of a row
#pragma unroll
            for (int i = 0; i < CH; ++i) {                   // 32 / CH rows at a time: contiguous in a page
                const int64_t r = P16 && i >= CH / 2 ? row1 - 16 : row0;
                copy16(dst + i * 512, kc + r * (D / 2) + lane * 16 + i * 512);
                copy16(dst + Ring<D>::kRows + i * 512, vc + r * (D / 2) + lane * 16 + i * 512);
            }
            if (lane < 16) {
                const int64_t r = P16 && (lane & 4) ? row1 - 16 : row0;
                copy16(dst + 2 * Ring<D>::kRows, (lane < 8 ? kp : vp) + r + (lane & 7) * 4);
            }
            if (++f_tile == f_units) {
                f_tile = 0;
                if (++f_head == heads) {
                    f_head = 0;
                    if (f_left > 0)
                        do f_units = tiles_of(p, ++f_seq);
                        while (f_units == 0);
                }
            }
            fetch_pages();
        }
        copies_commit();
    };
    fetch_pages();
    fetch(0);
    fetch(1);
    int place = 0;
    const int tv = (t & 1) | (t & 2) << 1, tg = (g & 4) | (g & 1) << 1 | (g >> 1 & 1);

    while (left > 0) {
        const int len = a.lengths[seq], now = min(units - tile0, left);
        // --- queries: columns g (+ 8) of the B operand; sums and scales of columns 2 t, 2 t + 1
        uint32_t q1[GT][kSteps][2], q2[GT][kSteps][2];
        float qsum[GT][2], qdown[GT][2];
        int qmid[GT][2];                         // what the middle of a key's range (code 7.5) loses by the query's rounding
#pragma unroll
        for (int n = 0; n < GT; ++n) {
            const int h = n * 8 + g;
            uint4 w[kSteps];
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                w[j] = make_uint4(0, 0, 0, 0);
                if (h < p.group)
                    w[j] = __ldg(reinterpret_cast<const uint4*>(a.q + seq * a.q_seq_stride + (int64_t)(head * p.group + h) * a.q_head_stride +
                                                                t * (D / 4) + 8 * j));
                const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, max((x[i] << 16) & 0x7fffffffu, x[i] & 0x7fff0000u));
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            float up, down;
            query_scale(top, up, down);
            up = copysignf(up, a.scale);                     // with the sign of the scale
            float sum = 0.f;                                 // of the elements, and of their whole numbers
            uint32_t rounded = 0;
            auto whole_q = [&](float x) {
                const uint32_t r = whole(x, up);
                sum = fmaf(x, up, sum);
                rounded += r;
                return r;
            };
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                split_bytes(whole_q(bf16_lo(w[j].x)), whole_q(bf16_lo(w[j].y)), whole_q(bf16_lo(w[j].z)), whole_q(bf16_lo(w[j].w)), q1[n][j][0], q2[n][j][0]);
                split_bytes(whole_q(bf16_hi(w[j].x)), whole_q(bf16_hi(w[j].y)), whole_q(bf16_hi(w[j].z)), whole_q(bf16_hi(w[j].w)), q1[n][j][1], q2[n][j][1]);
            }
            rounded -= (D / 4) * (uint32_t)kMagicBits;
#pragma unroll
            for (int x = 1; x < 4; x <<= 1) {
                sum += __shfl_xor_sync(0xffffffffu, sum, x);
                rounded += __shfl_xor_sync(0xffffffffu, rounded, x);
            }
            const int middle = __float2int_rn(7.5f * (sum - (float)(int)rounded));
            // scores are held in units of 1 / qdown: |scale| log2(e) / up; not zero, so that minus infinity stays what it is
            down = fmaxf(down * to_log2, 1e-30f);
            qsum[n][0] = __shfl_sync(0xffffffffu, sum, 8 * t);
            qsum[n][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
            qdown[n][0] = __shfl_sync(0xffffffffu, down, 8 * t);
            qdown[n][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4);
            qmid[n][0] = __shfl_sync(0xffffffffu, middle, 8 * t);
            qmid[n][1] = __shfl_sync(0xffffffffu, middle, 8 * t + 4);
        }

        float2 o[GT][2 * kMt];                   // channels g C + i, columns 2 t and 2 t + 1
        float m[GT][2], l[GT][2], z[GT][2];
#pragma unroll
        for (int n = 0; n < GT; ++n) {
#pragma unroll
            for (int i = 0; i < 2 * kMt; ++i) o[n][i] = make_float2(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = z[n][e] = 0.f; }
        }
        bool bad = false;

        for (int tok = tile0 * kTile, end = (tile0 + now) * kTile; tok < end; tok += kTile) {
            __syncwarp();                                   // every lane has read the tile that the next copy replaces
            bad = bad || (bad_pages >> place & 1);
            fetch(place == 0 ? 2 : place - 1);
            copies_wait<kStages - 1>();
            __syncwarp();
            const uint8_t* const tile = ring + place * Ring<D>::kStage;
            const uint32_t* const params = reinterpret_cast<const uint32_t*>(tile + 2 * Ring<D>::kRows);
            place = place == kStages - 1 ? 0 : place + 1;
            const int zero[4] = {0, 0, 0, 0};
            // S of both halves
            float s[GT][2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int d1[GT][4], d2[GT][4];
                // row g of the tile is token tg = g with its two low bits exchanged: so the four tokens whose values a quad reads
                // together (rows 0, 2, 4, 6) lie in different banks
                const Words<KB> k0 = read_words<KB>(tile + (16 * h + tg) * (D / 2) + t * KB), k1 = read_words<KB>(tile + (16 * h + 8 + tg) * (D / 2) + t * KB);
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    const uint32_t w0 = k0[j], w1 = k1[j];
                    const uint32_t a0 = w0 & 0x0f0f0f0fu, a1 = w1 & 0x0f0f0f0fu, a2 = (w0 >> 4) & 0x0f0f0f0fu, a3 = (w1 >> 4) & 0x0f0f0f0fu;
#pragma unroll
                    for (int n = 0; n < GT; ++n) {
                        if (j == 0) {
                            mma_u8s8(d1[n], a0, a1, a2, a3, q1[n][j], zero);
                            const int mid[4] = {qmid[n][0], qmid[n][1], qmid[n][0], qmid[n][1]};
                            mma_u8s8(d2[n], a0, a1, a2, a3, q2[n][j], mid);
                        } else {
                            mma_u8s8(d1[n], a0, a1, a2, a3, q1[n][j], d1[n]);
                            mma_u8s8(d2[n], a0, a1, a2, a3, q2[n][j], d2[n]);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < GT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][h][i] = (float)((d1[n][i] << 8) + d2[n][i]);
            }
            const uint32_t vq = tok + lane < len ? params[kTile + lane] : 0u;    // what lies past the length adds nothing, whatever it holds
            // scores in units of 1 / qdown
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t w = params[16 * h + 8 * e + tg];
                    const float ks = bf16_lo(w), kb = bf16_hi(w);
#pragma unroll
                    for (int n = 0; n < GT; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) s[n][h][2 * e + c] = fmaf(ks, s[n][h][2 * e + c], kb * qsum[n][c]);
                }
            if (tok + kTile > len)                       // tokens past the length out
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (tok + 16 * h + 8 * e + tg >= len)
#pragma unroll
                            for (int n = 0; n < GT; ++n) s[n][h][2 * e] = s[n][h][2 * e + 1] = -INFINITY;
            // the running maxima, looked at across the lanes only where one of them rises (over a long context that is soon rare)
            bool grow = false;
            float mt[GT][2];
#pragma unroll
            for (int n = 0; n < GT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    mt[n][c] = fmaxf(fmaxf(s[n][0][c], s[n][0][2 + c]), fmaxf(s[n][1][c], s[n][1][2 + c]));
                    grow = grow || mt[n][c] > m[n][c];
                }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int n = 0; n < GT; ++n) {
                    float f[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float nm = fmaxf(m[n][c], mt[n][c]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, x));
                        f[c] = m[n][c] == nm ? 1.f : ex2((m[n][c] - nm) * qdown[n][c]);
                        m[n][c] = nm;
                        l[n][c] *= f[c]; z[n][c] *= f[c];
                    }
#pragma unroll
                    for (int i = 0; i < 2 * kMt; ++i) { o[n][i].x *= f[0]; o[n][i].y *= f[1]; }
                }
            }
            // probabilities, their products with the value scales, and the two parts of P turned to the B operand's layout
            uint32_t p1[GT][2], p2[GT][2];
            int c1[GT][4], c2[GT][4];
            float beta[GT][2];
#pragma unroll
            for (int n = 0; n < GT; ++n) {
                float sl[2] = {0.f, 0.f}, sz[2] = {0.f, 0.f}, y[2][2][2], top[2] = {0.f, 0.f};
                const float shift[2] = {-m[n][0] * qdown[n][0], -m[n][1] * qdown[n][1]};
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t w = __shfl_sync(0xffffffffu, vq, 16 * h + 8 * e + tg);
                        const float vs = bf16_lo(w), mid = fmaf(8.f, vs, bf16_hi(w));
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float pr = ex2(fmaf(s[n][h][2 * e + c], qdown[n][c], shift[c]));
                            sl[c] += pr;
                            sz[c] = fmaf(pr, mid, sz[c]);
                            y[h][e][c] = pr * vs;
                            top[c] = fmaxf(top[c], fabsf(y[h][e][c]));
                        }
                    }
                // the exponent of each column's largest product; two columns' upper halves go round together
                uint32_t both = __byte_perm(__float_as_uint(top[0]), __float_as_uint(top[1]), 0x7632);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) both = max_u16x2(both, __shfl_xor_sync(0xffffffffu, both, x));
                float up[2];
                product_scale(both << 16, up[0], beta[n][0]);
                product_scale(both, up[1], beta[n][1]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[2][2];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int c = 0; c < 2; ++c) x[c][e] = whole(y[h][e][c], up[c]);
                    // bytes of P1 and P2, columns 2 t and 2 t + 1, tokens g and g + 8 of the half
                    const uint32_t x0 = __byte_perm(x[0][0], x[0][1], 0x5410), x1 = __byte_perm(x[1][0], x[1][1], 0x5410);
                    p1[n][h] = transpose8x8(__byte_perm(x0 >> 7, x1 >> 7, 0x6420));
                    p2[n][h] = transpose8x8(__byte_perm(x0, x1, 0x6420) & 0x7f7f7f7fu);
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) { l[n][c] += sl[c]; z[n][c] += sz[c]; }
                mma_u8s8(c1[n], 0x08080808u, 0x08080808u, 0x08080808u, 0x08080808u, p1[n], zero);     // 8 sum P1 and 8 sum P2, for every row
                mma_u8s8(c2[n], 0x08080808u, 0x08080808u, 0x08080808u, 0x08080808u, p2[n], zero);
#pragma unroll
                for (int i = 0; i < 4; ++i) { c1[n][i] = -c1[n][i]; c2[n][i] = kMagicBits - c2[n][i]; }
            }
            Words<VB> vw[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    vw[h][e] = read_words<VB>(tile + Ring<D>::kRows + (16 * h + tv + 2 * (e & 1) + 8 * (e >> 1)) * (D / 2) + g * VB);
#pragma unroll
            for (int j = 0; j < VB / 4; ++j) {
                uint32_t x[2][4];                    // [half][byte of the word]: that byte of rows 2 t, 2 t + 8, 2 t + 1, 2 t + 9
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t t0 = __byte_perm(vw[h][0][j], vw[h][2][j], 0x5140), t1 = __byte_perm(vw[h][1][j], vw[h][3][j], 0x5140);
                    const uint32_t t2 = __byte_perm(vw[h][0][j], vw[h][2][j], 0x7362), t3 = __byte_perm(vw[h][1][j], vw[h][3][j], 0x7362);
                    x[h][0] = __byte_perm(t0, t1, 0x5410); x[h][1] = __byte_perm(t0, t1, 0x7632);
                    x[h][2] = __byte_perm(t2, t3, 0x5410); x[h][3] = __byte_perm(t2, t3, 0x7632);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a0 = x[0][i] & 0x0f0f0f0fu, a1 = (x[0][i] >> 4) & 0x0f0f0f0fu;
                    const uint32_t a2 = x[1][i] & 0x0f0f0f0fu, a3 = (x[1][i] >> 4) & 0x0f0f0f0fu;
#pragma unroll
                    for (int n = 0; n < GT; ++n) {
                        int d[4];
                        mma_u8s8(d, a0, a1, a2, a3, p1[n], c1[n]);
#pragma unroll
                        for (int k = 0; k < 4; ++k) d[k] = (d[k] << 7) + c2[n][k];
                        mma_u8s8(d, a0, a1, a2, a3, p2[n], d);
                        add_scaled(o[n][2 * (4 * j + i)], d[0], d[1], beta[n][0], beta[n][1]);
                        add_scaled(o[n][2 * (4 * j + i) + 1], d[2], d[3], beta[n][0], beta[n][1]);
                    }
                }
            }
        }
        if (bad && lane == 0) raise_status(a.status, MT_ERR_INVALID_ARG, seq);

        // --- the result, or this warp's part of it
        constexpr int C = D / 8;                 // channels per lane group
        const bool whole = now == units;
        const int64_t slot = (2 * me + (tile0 > 0 ? 0 : 1)) * H;
#pragma unroll
        for (int n = 0; n < GT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], x);
                    z[n][c] += __shfl_xor_sync(0xffffffffu, z[n][c], x);
                }
                const int h = n * 8 + 2 * t + c;
                if (h >= p.group) continue;
                const float sum = bad ? nan_f() : l[n][c], shift = z[n][c], inv = 1.f / sum;
                uint32_t* const out = reinterpret_cast<uint32_t*>(a.out + ((int64_t)seq * a.q_heads + head * p.group + h) * D + g * C);
                float2* const part = reinterpret_cast<float2*>(p.part_o + (slot + h) * D + g * C);
#pragma unroll
                for (int i = 0; i < kMt; ++i) {
                    const float2 y = c == 0 ? make_float2(o[n][2 * i].x + shift, o[n][2 * i + 1].x + shift) : make_float2(o[n][2 * i].y + shift, o[n][2 * i + 1].y + shift);
                    if (whole) out[i] = pack_bf16x2(y.x * inv, y.y * inv);
                    else __stcg(part + i, y);
                }
                // (the maximum in units of log2, alike for all parts)
                if (!whole && g == 0)
                    __stcg(reinterpret_cast<float2*>(p.part_ml) + slot + h, make_float2(m[n][c] == -INFINITY ? -INFINITY : m[n][c] * qdown[n][c], sum));
            }
        if (tile0 == 0 && lane == 0)             // how far it goes on in the warps behind this one
            p.split[(int64_t)seq * heads + head] = {(int)me, whole ? 0 : (int)((begin + (share - left) + units - 1) / share - me) + 1};
        left -= now;
        tile0 = 0;
        if (left > 0 && ++head == heads) {
            head = 0;
            do units = tiles_of(p, ++seq);
            while (units == 0);
        }
    }
    copies_wait<0>();
}

// Joins the parts of one (sequence, query head) after the other.
template <int D, int GT>
__global__ void __launch_bounds__(kJoinThreads) kv_attention_join(DecodeArgs p) {
    constexpr int H = GT * 8, kLanes = D / 4, kSlices = kJoinThreads / kLanes;      // a thread: four channels of every kSlices-th part
    __shared__ float s_f[kMaxParts + 1], s_s[kMaxParts + 1], s_inv;
    __shared__ float4 s_part[kJoinThreads];
    const KvAttentionArgs& a = p.a;
    const int tid = threadIdx.x, lane = tid & 31;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t items = (int64_t)a.n_seqs * a.q_heads;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int h = (int)(i % a.q_heads) % p.group;
        const Split split = p.split[i / p.group];
        const int parts = split.parts;
        if (parts == 0) continue;
        auto at_part = [&](int b) { return (2 * ((int64_t)split.first + b) + (b > 0 ? 0 : 1)) * H + h; };
        for (int b = tid; b < parts; b += kJoinThreads) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml) + at_part(b));
            s_f[b] = ml.x;
            s_s[b] = ml.y;
        }
        __syncthreads();
        if (tid < 32) {
            float mx = -INFINITY, sl = 0.f;
            for (int b = lane; b < parts; b += 32) mx = fmaxf(mx, s_f[b]);
            mx = warp_max(mx);
            for (int b = lane; b < parts; b += 32) {
                const float f = s_f[b] == mx ? 1.f : ex2(s_f[b] - mx);
                s_f[b] = f;
                sl = fmaf(f, s_s[b], sl);
            }
            sl = warp_sum(sl);
            if (lane == 0) s_inv = 1.f / sl;
        }
        __syncthreads();
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int b = tid / kLanes; b < parts; b += kSlices) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part_o + at_part(b) * D) + tid % kLanes);
            const float f = s_f[b];
            y.x = fmaf(f, x.x, y.x); y.y = fmaf(f, x.y, y.y); y.z = fmaf(f, x.z, y.z); y.w = fmaf(f, x.w, y.w);
        }
        s_part[tid] = y;
        __syncthreads();
        if (tid < kLanes) {
#pragma unroll
            for (int k = 1; k < kSlices; ++k) {
                const float4 x = s_part[k * kLanes + tid];
                y.x += x.x; y.y += x.y; y.z += x.z; y.w += x.w;
            }
            uint2 w;
            w.x = pack_bf16x2(y.x * s_inv, y.y * s_inv);
            w.y = pack_bf16x2(y.z * s_inv, y.w * s_inv);
            reinterpret_cast<uint2*>(a.out + i * D)[tid] = w;
        }
        __syncthreads();
    }
}

typedef void (*KvAttentionKernel)(DecodeArgs);
const KvAttentionKernel kKernels[2][2][2] = {
    {{kv_attention_kernel<64, 1, false>, kv_attention_kernel<64, 1, true>}, {kv_attention_kernel<64, 2, false>, kv_attention_kernel<64, 2, true>}},
    {{kv_attention_kernel<128, 1, false>, kv_attention_kernel<128, 1, true>}, {kv_attention_kernel<128, 2, false>, kv_attention_kernel<128, 2, true>}}};

const KvAttentionKernel kJoins[2][2] = {{kv_attention_join<64, 1>, kv_attention_join<64, 2>}, {kv_attention_join<128, 1>, kv_attention_join<128, 2>}};

}  // namespace

cudaError_t configure_kv_attention() {
    for (int d = 0; d < 2; ++d)
        for (int gt = 0; gt < 2; ++gt) {
            cudaError_t e = cudaSuccess;
            for (int p16 = 0; p16 < 2 && e == cudaSuccess; ++p16)
                e = cudaFuncSetAttribute(kKernels[d][gt][p16], cudaFuncAttributeMaxDynamicSharedMemorySize, kv_shared_bytes(d ? 128 : 64));
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

mt_status launch_kv_attention(const KvAttentionArgs& a, const OpContext& c, cudaStream_t s) {
    DecodeArgs p;
    p.a = a;
    p.page_shift = 4;
    while ((1 << p.page_shift) < a.c.page_tokens) ++p.page_shift;
    p.max_len = a.c.n_pages > 0 ? (int64_t)a.table_width * a.c.page_tokens : 0;
    p.group = a.q_heads / a.c.kv_heads;
    const int gt = p.group > 8 ? 2 : 1, d = a.c.head_dim;
    // as many CTAs as fit the GPU at once, but not more than there can be shares
    const int64_t tiles = (int64_t)a.n_seqs * a.c.kv_heads * ((p.max_len + kTile - 1) / kTile);
    const int64_t most = (tiles + kWarps * kMinShare - 1) / (kWarps * kMinShare);
    int64_t grid = (int64_t)c.sm_count * (gt == 1 ? 4 : 2);
    if (grid > most) grid = most > 1 ? most : 1;
    const int64_t warps = grid * kWarps;
    const size_t o_bytes = (size_t)warps * 2 * gt * 8 * d * 4, ml_bytes = (size_t)warps * 2 * gt * 8 * 8;
    uint8_t* w = nullptr;
    mt_status st = op_scratch(s, o_bytes + ml_bytes + (size_t)a.n_seqs * a.c.kv_heads * sizeof(Split), &w);
    if (st != MT_OK) return st;
    p.part_o = reinterpret_cast<float*>(w);
    p.part_ml = reinterpret_cast<float*>(w + o_bytes);
    p.split = reinterpret_cast<Split*>(w + o_bytes + ml_bytes);
    cudaError_t e = launch_pdl(kKernels[d == 128][gt - 1][a.c.page_tokens == 16], dim3((unsigned)grid), dim3(kWarps * 32), (size_t)kv_shared_bytes(d), s, p);
    // (a single share has nothing to join)
    if (e == cudaSuccess && tiles > kMinShare) {
        const int64_t items = (int64_t)a.n_seqs * a.q_heads, at_once = 16LL * c.sm_count;
        e = launch_pdl(kJoins[d == 128][gt - 1], dim3((unsigned)(items < at_once ? items : at_once)), dim3(kJoinThreads), 0, s, p);
    }
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

}  // namespace mt

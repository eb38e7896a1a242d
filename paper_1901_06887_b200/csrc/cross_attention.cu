// Attention of packed queries to an encoder's states of another length, on the tensor cores; also for one token a sequence.
//
// Mathematics.  o_i = sum_j p_ij v_j / sum_j p_ij over all states j of the sequence, p_ij = 2^(c (q_i . k_j - m_i)), c = scale log2(e), in one pass
// over blocks of 128 states.  m_i is a running reference that moves only when a block's maximum lies more than 8 above it (in log2).  p is
// rounded to bf16 before it meets v (kind::f16 takes one type for both operands); l sums the unrounded p.
//
// Tile.  Two tiles of 128 rows share the states that stream through shared memory.  A row is a (token, head) pair: R heads that share a
// key/value head (the largest power of two in the group, 16 at most) are packed into the rows, so one token with a large group already shares its states.
//
// Sequences that follow one another and have the same states (answers about one image) are one: 64 answers, four to a source, 104 -> 38 us a token step.
//
// Order of work.  A unit is a block of states for a tile pair; the units of all (sequence, head pack, tile pair) are in one line, which is cut
// into equal shares, one a CTA.  A tile pair that a border cuts is done in pieces: each leaves its sums (o without the division, m, l) in scratch, and a
// second launch joins them.  So one token over a long recording takes all SMs.  Many tile pairs are dealt whole, those with most states first, back and
// forth over the CTAs, and nothing is joined: from one an SM on where that leaves no CTA far above the mean, from eight on in any case.  (Nothing asks
// there whether it is even: one source far longer than the others is then one CTA's.  1000 sources of 128 states take 218 us, one of 24 000 by itself 49, all
// together 518; 64 tokens each, 16 / 4 heads of 128.)
//
// Cost.  One token of 64 answers to 16 sources of 577 to 4000 states, 32 / 8 heads of 128: 37 us for 116 MB, of which some 18 are fixed (set-up, the first
// loads, the join); four times the sources take 102.  Groups that are no power of two stream their states once for each share of the largest one that divides
// them: 24 / 8 heads 82 us, 40 / 8 127.  16 prompts of 1 to 700 tokens over 49 to 2305 states: 110 us, tensor
// pipe and exponentials half busy each, as in the prompt kernel.  11 001 queries over 4500 to 6000 states, 16 heads of 64: 330 to 338 us, exponentials 75 % of
// the time at the 1.6 GHz that the power cap leaves.  (A part of them by a polynomial on the multiply-add units: 330 to 373 where all of them by the exponential unit took 323.)
//
// Roles (12 warps): warps 0-3 and 4-7 are the softmax of the two tiles, one row per thread; warp 8 copies (TMA), warp 9 issues the matrix
// instructions, warps 10 and 11 zero the values behind the sequence's last state: their p is zero, but zero times an infinity is NaN.
#include "attention_device.cuh"
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kThreads = 384;
constexpr int kMaxSeqs = 512;                 // sequences of one launch
constexpr float kSlack = 8.f;
constexpr int kEnough = 8;                    // tile pairs an SM, from which they are dealt whole in any case
constexpr int kUneven = 10;                   // units that a CTA may get above the mean then: what pieces and their joins cost
constexpr int kJoinThreads = 256;

template <int D> __host__ __device__ constexpr int slots() { return D == 128 ? 4 : 8; }
template <int D> __host__ __device__ constexpr int operand_bytes() { return kHalf * (D / 64); }

// A share of the line of units, piece by piece.
struct Walk {
    int left;                                 // units (of queries that fit in memory a CTA has fewer than 2^31); rounds dealt, where tile pairs are whole
    int seq, pack, tile, block;               // where the next one is
};
struct Work {
    int seq, t0, pack;                        // first token of the tile pair, head pack
    int states;
    int b0, b1, nb;                           // blocks of the piece, and of the tile pair
    int tiles;                                // tiles with rows
};
struct Control {
    uint64_t q_full[2], q_empty, s_full[2], s_free[2], p_half[2], p_ready[2], o_ready[2], kv_full[8], kv_empty[8], v_raw[8], v_clean[8];
    uint32_t tmem;
    int abort, whole;
    unsigned long long longest;
    int start[kMaxSeqs + 1], len[kMaxSeqs], first[kMaxSeqs], states[kMaxSeqs];
    long long before[kMaxSeqs + 1];           // units of the sequences before
    uint16_t order[kMaxSeqs];                 // sequences by falling number of blocks, and the tile pairs of those before
    int pairs[kMaxSeqs + 1];
    Walk walk[8];                             // of the softmax warps, while a piece is under way: the registers are needed
    Work work[8];
};
constexpr int kControlBytes = ((int)sizeof(Control) + 127) / 128 * 128;
constexpr int kStageBytes = 8 * 2048;           // output staging of the eight softmax warps
// P lies over the columns of S, or, where tensor memory has room, behind O: then the next S is made while the exponentials of this one run.  (16 heads of 64, 11 001
// queries, 4500 to 6000 states: 321 against 342 us.)
template <int D> __host__ __device__ constexpr bool apart() { return 256 + 2 * D + 2 * 64 <= 512; }
template <int D> constexpr int shared_bytes() { return 1024 + (2 + slots<D>()) * operand_bytes<D>() + kControlBytes + kStageBytes; }

// What a CTA leaves behind of a tile pair that a border cuts: two such places a CTA, the piece that ends a tile pair begun by others, and the one
// that begins one.
template <int D> struct Piece {
    float o[256][D];
    float2 ml[256];
};
// A tile pair in pieces, noted by the CTA that begins it.
struct Note {
    long long total;                          // units of the launch
    int last;                                 // CTA of its last piece; -1: nothing to join
    int row, rows, pack;                      // first token, (token, head) rows, head pack
};

struct CrossParams {
    const int32_t *offsets, *ranges;
    int n_seqs, seq0, n_tokens, n_states;
    int q_heads, group, pack, pack_shift;     // pack: heads packed into a tile's rows
    int whole;                                // tile pairs are dealt whole: 0 no, 1 yes, 2 if that is even enough
    float c;                                  // |scale| log2(e)
    int negate;                               // scale < 0
    uint16_t* out;
    Note* notes;
    void* pieces;
    OpStatus status;
};

__device__ __forceinline__ int blocks_of(int states) { return states > 0 ? (states + kBlock - 1) / kBlock : 1; }
__device__ __forceinline__ long long share_begin(long long total, int cta, int ctas) { return total * cta / ctas; }

__device__ __forceinline__ void locate(const Control& s, const CrossParams& p, long long at, Walk& w) {
    int lo = 0, hi = p.n_seqs - 1;            // before[r] <= at < before[r + 1]
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.before[mid] <= at) lo = mid; else hi = mid - 1;
    }
    const int tokens = 256 >> p.pack_shift, nb = blocks_of(s.states[lo]), tiles = (s.len[lo] + tokens - 1) / tokens;
    const long long local = at - s.before[lo], item = local / nb;
    w.seq = lo;
    w.block = (int)(local - item * nb);
    w.pack = (int)(item / tiles);
    w.tile = (int)(item - (long long)w.pack * tiles);
}
// The tile pair that a CTA gets in a round: back and forth.
__device__ __forceinline__ int dealt(int round, int cta) { return round * gridDim.x + ((round & 1) ? gridDim.x - 1 - cta : cta); }
__device__ __forceinline__ int rank_of(const Control& s, const CrossParams& p, int pair) {
    int lo = 0, hi = p.n_seqs - 1;            // pairs[r] <= pair < pairs[r + 1]
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.pairs[mid] <= pair) lo = mid; else hi = mid - 1;
    }
    return lo;
}
__device__ __forceinline__ Walk begin_share(const Control& s, const CrossParams& p) {
    Walk w;
    w.left = w.seq = w.pack = w.tile = w.block = 0;
    if (s.whole) return w;
    const long long total = s.before[p.n_seqs], first = share_begin(total, blockIdx.x, gridDim.x);
    w.left = (int)(share_begin(total, blockIdx.x + 1, gridDim.x) - first);
    if (w.left > 0) locate(s, p, first, w);
    return w;
}
// The next piece of the share.
__device__ __forceinline__ bool next_piece(const Control& s, const CrossParams& p, Walk& w, Work& k) {
    const int tokens = 256 >> p.pack_shift, packs = p.q_heads >> p.pack_shift;
    if (s.whole) {
        const int pair = dealt(w.left, blockIdx.x);
        if (pair >= s.pairs[p.n_seqs]) return false;
        ++w.left;
        const int rank = rank_of(s, p, pair), seq = s.order[rank], q = pair - s.pairs[rank], tiles = (s.len[seq] + tokens - 1) / tokens;
        k.seq = seq;
        k.states = s.states[seq];
        k.pack = q / tiles;
        k.t0 = (q - k.pack * tiles) * tokens;
        k.b0 = 0;
        k.b1 = k.nb = blocks_of(k.states);
        k.tiles = k.t0 + tokens / 2 < s.len[seq] ? 2 : 1;
        return true;
    }
    if (w.left <= 0) return false;
    while (w.pack == packs || s.len[w.seq] == 0) { ++w.seq; w.pack = w.tile = w.block = 0; }
    const int len = s.len[w.seq];
    k.seq = w.seq;
    k.states = s.states[w.seq];
    k.pack = w.pack;
    k.t0 = w.tile * tokens;
    k.nb = blocks_of(k.states);
    k.b0 = w.block;
    k.b1 = min(k.nb, w.block + w.left);
    k.tiles = k.t0 + tokens / 2 < len ? 2 : 1;
    w.left -= k.b1 - k.b0;
    w.block = 0;
    if (++w.tile * tokens >= len) { w.tile = 0; ++w.pack; }
    return true;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
cross_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v, const CrossParams p) {
    extern __shared__ uint8_t smem_raw[];
    constexpr int kSlots = slots<D>(), kOp = operand_bytes<D>();
    constexpr bool kApart = apart<D>();
    constexpr int kP0 = kApart ? 256 + 2 * D : 0, kPStep = kApart ? 64 : 128;  // columns of P
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - raw);
    Control& s = *reinterpret_cast<Control*>(smem + (2 + kSlots) * kOp);
    const uint32_t q_smem = base, kv_smem = base + 2 * kOp;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* const abort_flag = &s.abort;
    auto bar = [](const uint64_t& b) { return smem_u32(&b); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(s.q_full[i]), 1); mbar_init(bar(s.s_full[i]), 1); mbar_init(bar(s.s_free[i]), 128); mbar_init(bar(s.p_half[i]), 128); mbar_init(bar(s.p_ready[i]), 128);
            mbar_init(bar(s.o_ready[i]), 1);
        }
        mbar_init(bar(s.q_empty), 1);
        for (int i = 0; i < kSlots; ++i) { mbar_init(bar(s.kv_full[i]), 1); mbar_init(bar(s.kv_empty[i]), 1); mbar_init(bar(s.v_raw[i]), 1); mbar_init(bar(s.v_clean[i]), 64); }
        s.abort = 0;
        fence_mbar_init();
    }
    if (warp == 9 && lane == 0) { prefetch_tensormap(&map_q); prefetch_tensormap(&map_k); prefetch_tensormap(&map_v); }
    pdl_wait();
    // All of tensor memory, taken only when the predecessor is done with its share, and before a successor may start and ask for its own.
    if (warp == 8) {
        tmem_alloc(smem_u32(&s.tmem), 512);
        tmem_relinquish();
    }

    // --- the line of units
    const int tokens = 256 >> p.pack_shift;
    const long long packs = p.q_heads >> p.pack_shift;
    for (int i = threadIdx.x; i < p.n_seqs; i += kThreads) {
        const int a = p.offsets[i], b = p.offsets[i + 1], f = p.ranges[2 * i], e = p.ranges[2 * i + 1];
        const bool bad = a < 0 || b < a || b > p.n_tokens || f < 0 || e < f || e > p.n_states;
        if (bad && blockIdx.x == 0) raise_status(p.status, MT_ERR_INVALID_ARG, p.seq0 + i);
        s.start[i] = a;
        s.len[i] = bad ? 0 : b - a;
        s.first[i] = f;
        s.states[i] = bad ? -1 : e - f;
        if (i == p.n_seqs - 1) s.start[p.n_seqs] = b;
    }
    __syncthreads();
    if (warp == 0) {
        // neighbours with the same states become one: the first takes the tokens of all, the others have none
        int next = p.n_seqs;                       // first sequence behind these 32 that begins one
        for (int r0 = (p.n_seqs - 1) / 32 * 32; r0 >= 0; r0 -= 32) {
            const int r = r0 + lane;
            const bool there = r < p.n_seqs;
            const bool begins = there && (r == 0 || s.states[r] < 0 || s.states[r - 1] < 0 || s.states[r] != s.states[r - 1] || s.first[r] != s.first[r - 1]);
            const uint32_t heads = __ballot_sync(0xffffffffu, begins), behind = lane < 31 ? heads >> (lane + 1) : 0;
            if (there && s.states[r] >= 0) s.len[r] = begins ? s.start[behind ? r + __ffs(behind) : next] - s.start[r] : 0;
            if (heads) next = r0 + __ffs(heads) - 1;
        }
        __syncwarp();
        long long run = 0;
        for (int r0 = 0; r0 < p.n_seqs; r0 += 32) {
            const int r = r0 + lane;
            const long long v = r < p.n_seqs ? packs * ((s.len[r] + tokens - 1) / tokens) * blocks_of(s.states[r]) : 0;
            long long incl = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += y;
            }
            if (r < p.n_seqs) s.before[r] = run + incl - v;
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) { s.before[p.n_seqs] = run; s.whole = p.whole == 1; s.longest = 0; }
    }
    if (p.whole) {
        __syncthreads();
        for (int i = threadIdx.x; i < p.n_seqs; i += kThreads) {
            const int n = blocks_of(s.states[i]);
            int rank = 0;
            for (int j = 0; j < p.n_seqs; ++j) { const int m = blocks_of(s.states[j]); rank += (m > n || (m == n && j < i)) ? 1 : 0; }
            s.order[rank] = (uint16_t)i;
        }
        __syncthreads();
        if (warp == 0) {
            int run = 0;
            for (int r0 = 0; r0 < p.n_seqs; r0 += 32) {
                const int r = r0 + lane, v = r < p.n_seqs ? (int)packs * ((s.len[s.order[r]] + tokens - 1) / tokens) : 0;
                int incl = v;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, incl, d);
                    if (lane >= d) incl += y;
                }
                if (r < p.n_seqs) s.pairs[r] = run + incl - v;
                run += __shfl_sync(0xffffffffu, incl, 31);
            }
            if (lane == 0) s.pairs[p.n_seqs] = run;
        }
    }
    if (p.whole == 2) {                        // the CTA with most
        __syncthreads();
        for (int cta = threadIdx.x; cta < gridDim.x; cta += kThreads) {
            unsigned long long units = 0;
            for (int round = 0; dealt(round, cta) < s.pairs[p.n_seqs]; ++round) units += blocks_of(s.states[s.order[rank_of(s, p, dealt(round, cta))]]);
            atomicMax(&s.longest, units);
        }
        __syncthreads();
        if (threadIdx.x == 0) s.whole = (long long)s.longest <= s.before[p.n_seqs] / gridDim.x + kUneven;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = s.tmem;
    const uint32_t tmem_s = tmem, tmem_o = tmem + 256;         // S of tile i: + 128 i; O: + D i; P: see kApart
    Walk walk = begin_share(s, p);
    Work it;

    if (warp == 8) {
        // ------------------------------------------------------------------------------------------ copies
        asm volatile("setmaxnreg.dec.sync.aligned.u32 120;");
        if (lane == 0) {
            int fill = 0, rounds = 0;            // operands put into the ring so far; pieces
            bool ok = true;
            for (; ok && next_piece(s, p, walk, it); ++rounds) {
                if (rounds > 0) ok = mbar_wait(bar(s.q_empty), (rounds - 1) & 1, abort_flag, p.status.word, 240);
                if (!ok) break;
                for (int i = 0; i < it.tiles; ++i) {
                    mbar_expect_tx(bar(s.q_full[i]), kOp);
                    for (int h = 0; h < D / 64; ++h)
                        tma_load_3d(q_smem + i * kOp + h * kHalf, &map_q, h * 64, it.pack * p.pack, s.start[it.seq] + it.t0 + i * (tokens / 2), bar(s.q_full[i]));
                }
                const int kv_head = it.pack * p.pack / p.group;
                for (int x = 2 * it.b0; ok && x < 2 * it.b1; ++x, ++fill) {
                    const int slot = fill % kSlots, use = fill / kSlots;
                    if (use > 0) ok = mbar_wait(bar(s.kv_empty[slot]), (use - 1) & 1, abort_flag, p.status.word, 241);
                    if (!ok) break;
                    // a value block that passes the states goes to the cleaners first: its bytes count on v_raw, and v_clean says when it may be used
                    const bool ragged = (x & 1) && ((x >> 1) + 1) * kBlock > it.states;
                    const uint32_t full = ragged ? bar(s.v_raw[slot]) : bar(s.kv_full[slot]);
                    mbar_expect_tx(full, kOp);
                    for (int h = 0; h < D / 64; ++h)
                        tma_load_3d(kv_smem + slot * kOp + h * kHalf, (x & 1) ? &map_v : &map_k, h * 64, kv_head, s.first[it.seq] + (x >> 1) * kBlock, full);
                    if (ragged) mbar_arrive(bar(s.kv_full[slot]));
                }
            }
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------------------------------ matrix instructions
        asm volatile("setmaxnreg.dec.sync.aligned.u32 120;");
        // the whole warp walks the loop, so that addresses stay warp-uniform; one elected lane issues
        const bool leader = elect_one();
        constexpr uint32_t kIdPv = make_idesc_bf16(128, D) | (1u << 16);
        const uint32_t id_qk = make_idesc_bf16(128, kBlock) | (p.negate ? 1u << 13 : 0u);
        const uint32_t q_lo = desc_lo(q_smem), k_lo = desc_lo(kv_smem), v_lo = desc_lo_values(kv_smem);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        constexpr uint32_t kOpLo = kOp >> 4;
        uint32_t fill = 0, n_q0 = 0, n_q1 = 0, n_p0 = 0, n_p1 = 0, clean_phase = 0;      // n_p: blocks of the tile so far
        bool ok = true;
        auto wait = [&](const uint64_t& b, uint32_t parity, int where) { ok = ok && mbar_wait(bar(b), parity & 1, abort_flag, p.status.word, where); };
        auto qk = [&](int i, uint32_t slot) {
            if (leader) {
                const uint32_t d = tm + 128 * i, a = q_lo + i * kOpLo, b = k_lo + slot * kOpLo;
                umma_bf16_lohi<false>(d, a, b, id_qk);
#pragma unroll
                for (int k = 1; k < D / 16; ++k) {
                    const uint32_t off = (k / 4) * (kHalf >> 4) + (k % 4) * 2;
                    umma_bf16_lohi<true>(d, a + off, b + off, id_qk);
                }
                umma_commit(bar(s.s_full[i]));
            }
        };
        // the first 64 states go while the second half of P is still in its exponentials
        auto pv = [&](int i, uint32_t slot, bool first, uint32_t n) {
            const uint32_t d = tm + 256 + D * i, a = tm + kP0 + kPStep * i, b = v_lo + slot * kOpLo;
            wait(s.p_half[i], n, 254);
            if (!ok) return;
            tc_fence_after();
            if (leader) {
                if (first) umma_tmem_a_lohi<false>(d, a, b, kIdPv);
                else umma_tmem_a_lohi<true>(d, a, b, kIdPv);
#pragma unroll
                for (int k = 1; k < kBlock / 32; ++k) umma_tmem_a_lohi<true>(d, a + 8 * k, b + (2048 >> 4) * k, kIdPv);
            }
            wait(s.p_ready[i], n, 256);
            if (!ok) return;
            tc_fence_after();
            if (leader) {
#pragma unroll
                for (int k = kBlock / 32; k < kBlock / 16; ++k) umma_tmem_a_lohi<true>(d, a + 8 * k, b + (2048 >> 4) * k, kIdPv);
                umma_commit(bar(s.o_ready[i]));
            }
        };
        while (ok && next_piece(s, p, walk, it)) {
            const int nb = __shfl_sync(0xffffffffu, it.b1 - it.b0, 0);
            const bool two = __shfl_sync(0xffffffffu, it.tiles, 0) == 2;
            const int ragged = __shfl_sync(0xffffffffu, it.b1 * kBlock > it.states ? nb - 1 : -1, 0);
            uint32_t slot = fill % kSlots;
            wait(s.kv_full[slot], fill / kSlots, 250);
            wait(s.q_full[0], n_q0++, 251);
            if (!ok) break;
            tc_fence_after();
            qk(0, slot);
            if (two) {
                wait(s.q_full[1], n_q1++, 251);
                if (!ok) break;
                tc_fence_after();
                qk(1, slot);
            }
            if (leader) {
                umma_commit(bar(s.kv_empty[slot]));
                if (nb == 1) umma_commit(bar(s.q_empty));
            }
            for (int j = 0; ok && j < nb; ++j) {
                const uint32_t vx = fill + 2 * j + 1, vslot = vx % kSlots, kslot = (vx + 1) % kSlots, kpar = (vx + 1) / kSlots;
                if (kApart && j + 1 < nb) {
                    wait(s.kv_full[kslot], kpar, 255);
                    wait(s.s_free[0], n_p0, 257);
                    if (!ok) break;
                    tc_fence_after();
                    qk(0, kslot);
                }
                wait(s.kv_full[vslot], vx / kSlots, 252);
                if (j == ragged) {
                    wait(s.v_clean[vslot], clean_phase >> vslot, 253);
                    clean_phase ^= 1u << vslot;
                }
                if (!kApart && j + 1 < nb) wait(s.kv_full[kslot], kpar, 255);
                pv(0, vslot, j == 0, n_p0++);
                if (!ok) break;
                if (!kApart && j + 1 < nb) qk(0, kslot);
                if (two) {
                    if (kApart && j + 1 < nb) {
                        wait(s.s_free[1], n_p1, 257);
                        if (!ok) break;
                        tc_fence_after();
                        qk(1, kslot);
                    }
                    pv(1, vslot, j == 0, n_p1++);
                    if (!ok) break;
                    if (!kApart && j + 1 < nb) qk(1, kslot);
                }
                if (leader) {
                    umma_commit(bar(s.kv_empty[vslot]));
                    if (j + 1 < nb) umma_commit(bar(s.kv_empty[kslot]));
                    if (j + 2 == nb) umma_commit(bar(s.q_empty));
                }
            }
            fill += 2 * nb;
        }
    } else if (warp >= 10) {
        // ------------------------------------------------------------------------------------------ values behind the last state
        asm volatile("setmaxnreg.dec.sync.aligned.u32 120;");
        const int t = threadIdx.x - 320;         // rows t and t + 64
        int fill = 0;
        uint32_t raw_phase = 0;
        bool ok = true;
        while (ok && next_piece(s, p, walk, it)) {
            fill += 2 * (it.b1 - it.b0);
            if (it.b1 * kBlock <= it.states) continue;
            const int slot = (fill - 1) % kSlots;
            ok = mbar_wait(bar(s.v_raw[slot]), (raw_phase >> slot) & 1, abort_flag, p.status.word, 261);
            if (!ok) break;
            raw_phase ^= 1u << slot;
            uint8_t* const v = smem + (2 + slot) * kOp;
            for (int r = t; r < kBlock; r += 64) {
                if ((it.b1 - 1) * kBlock + r < it.states) continue;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) *reinterpret_cast<uint4*>(v + (c / 8) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();
            __threadfence_block();
            mbar_arrive(bar(s.v_clean[slot]));
        }
    } else {
        // ------------------------------------------------------------------------------------------ softmax, one row per thread
        // registers move here: 256 threads x 192 + 128 x 120 = the launch's 384 x 168
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int i = warp >> 2;
        const int r = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;     // tensor-memory lane of the warp's first row, in the address's upper half
        const uint32_t my_s = tmem_s + 128 * i + lanes, my_o = tmem_o + D * i + lanes, my_p = tmem + kP0 + kPStep * i + lanes;
        int n_s = 0, n_o = 0;
        bool ok = true;
        if (threadIdx.x == 0 && p.notes) p.notes[blockIdx.x].last = -1;
        while (ok && next_piece(s, p, walk, it)) {
            if (i >= it.tiles) continue;
            if (i * 128 + (warp & 3) * 32 >= min(s.len[it.seq] - it.t0, tokens) << p.pack_shift) {           // a warp without rows: what it would write is nobody's
                for (int j = it.b0; j < it.b1; ++j) {
                    ok = mbar_wait(bar(s.s_full[i]), n_s++ & 1, abort_flag, p.status.word, 273);
                    if (!ok) break;
                    if (kApart) {             // (not ahead of the other warps: the barriers count them all)
                        mbar_arrive(bar(s.s_free[i]));
                        if (j > it.b0) ok = mbar_wait(bar(s.o_ready[i]), (n_o - 1) & 1, abort_flag, p.status.word, 275);
                        if (!ok) break;
                    }
                    mbar_arrive(bar(s.p_half[i]));
                    mbar_arrive(bar(s.p_ready[i]));
                    ++n_o;
                }
                continue;
            }
            if (lane == 0) { s.walk[warp] = walk; s.work[warp] = it; }
            const int first = it.b0, end = it.b1, states = it.states;
            float m = 0.f, l = 0.f;
            for (int j = first; j < end; ++j) {
                ok = mbar_wait(bar(s.s_full[i]), n_s++ & 1, abort_flag, p.status.word, 270);
                if (!ok) break;
                tc_fence_after();
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(my_s + 32 * c, x[c]);
                tmem_ld_wait();
                if (kApart) {
                    tc_fence_before();
                    mbar_arrive(bar(s.s_free[i]));
                }
                if ((j + 1) * kBlock > states) {
                    const int lim = states - j * kBlock;    // states of the block
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * c + e >= lim) x[c][e] = 0xff800000u;
                }
                float mx4[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx4[c] = fmaxf(__uint_as_float(x[c][0]), __uint_as_float(x[c][1]));
#pragma unroll
                    for (int e = 2; e < 32; e += 2) mx4[c] = max3(mx4[c], __uint_as_float(x[c][e]), __uint_as_float(x[c][e + 1]));
                }
                const float mx = fmaxf(max3(mx4[0], mx4[1], mx4[2]), mx4[3]);
                // (a row without weight so far, all its scores minus infinity, starts again; m stays finite)
                const bool move = (mx - m) * p.c > kSlack || l == 0.f;
                if (j == first) {
                    m = mx > -INFINITY ? mx : 0.f;
                } else if (kApart) {          // P of the block before has to be read before this one's is written
                    ok = mbar_wait(bar(s.o_ready[i]), (n_o - 1) & 1, abort_flag, p.status.word, 271);
                    if (!ok) break;
                    tc_fence_after();
                }
                if (j > first && __any_sync(0xffffffffu, move)) {
                    // (a row moves on its own account only, so its bits do not depend on its neighbours)
                    const float nm = move && mx > -INFINITY ? mx : m, f = m == nm || l == 0.f ? 1.f : ex2((m - nm) * p.c);
                    m = nm;
                    l *= f;
                    if (!kApart) {
                        ok = mbar_wait(bar(s.o_ready[i]), (n_o - 1) & 1, abort_flag, p.status.word, 274);
                        if (!ok) break;
                        tc_fence_after();
                    }
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t y[16];
                        asm volatile(
                            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                            : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]), "=r"(y[4]), "=r"(y[5]), "=r"(y[6]), "=r"(y[7]), "=r"(y[8]), "=r"(y[9]),
                              "=r"(y[10]), "=r"(y[11]), "=r"(y[12]), "=r"(y[13]), "=r"(y[14]), "=r"(y[15])
                            : "r"(my_o + 16 * c) : "memory");
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * f);
                        tmem_st16(my_o + 16 * c, y);
                    }
                }
                const float shift = -m * p.c;
                const Pair c2 = pair_of(p.c, p.c), shift2 = pair_of(shift, shift);
                Pair sum[2] = {pair_of(0.f, 0.f), pair_of(0.f, 0.f)};
                auto chunk = [&](int c) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const Pair y = fma2(pair_of(__uint_as_float(x[c][2 * e]), __uint_as_float(x[c][2 * e + 1])), c2, shift2);
                        float a, b;
                        unpair(y, a, b);
                        a = ex2(a);
                        b = ex2(b);
                        sum[e & 1] = add2(sum[e & 1], pair_of(a, b));
                        w[e] = pack_bf16x2(a, b);
                    }
                    tmem_st16(my_p + 16 * c, w);
                };
                chunk(0);
                chunk(1);
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(bar(s.p_half[i]));
                chunk(2);
                chunk(3);
                float sa, sb;
                unpair(add2(sum[0], sum[1]), sa, sb);
                l += sa + sb;
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(bar(s.p_ready[i]));
                ++n_o;
            }
            if (!ok) break;
            ok = mbar_wait(bar(s.o_ready[i]), (n_o - 1) & 1, abort_flag, p.status.word, 272);
            if (!ok) break;
            tc_fence_after();
            __syncwarp();
            walk = s.walk[warp];
            it = s.work[warp];
            __syncwarp();                     // (before the next piece is put there)
            const int rows = min(s.len[it.seq] - it.t0, tokens) << p.pack_shift;
            if (it.b1 - it.b0 == it.nb) {
                const float inv = it.states > 0 ? 1.f / l : 0.f;
                // 32 channels at a time through shared memory, so that four lanes store 64 contiguous bytes of a row
                uint4* const stage = reinterpret_cast<uint4*>(smem + (2 + kSlots) * kOp + kControlBytes) + warp * 128;
                const int sub = lane & 3;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t y[32];
                    tmem_ld32(my_o + 32 * c, y);
                    tmem_ld_wait();
                    __syncwarp();
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        uint4 w;
                        w.x = pack_bf16x2(__uint_as_float(y[8 * v]) * inv, __uint_as_float(y[8 * v + 1]) * inv);
                        w.y = pack_bf16x2(__uint_as_float(y[8 * v + 2]) * inv, __uint_as_float(y[8 * v + 3]) * inv);
                        w.z = pack_bf16x2(__uint_as_float(y[8 * v + 4]) * inv, __uint_as_float(y[8 * v + 5]) * inv);
                        w.w = pack_bf16x2(__uint_as_float(y[8 * v + 6]) * inv, __uint_as_float(y[8 * v + 7]) * inv);
                        stage[lane * 4 + (v ^ ((lane >> 1) & 3))] = w;
                    }
                    __syncwarp();
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int row = v * 8 + (lane >> 2), of_pair = i * 128 + (warp & 3) * 32 + row;
                        const int head = it.pack * p.pack + (of_pair & (p.pack - 1));
                        const uint4 w = stage[row * 4 + (sub ^ ((row >> 1) & 3))];
                        if (of_pair < rows)
                            reinterpret_cast<uint4*>(p.out + ((int64_t)(s.start[it.seq] + it.t0 + (of_pair >> p.pack_shift)) * p.q_heads + head) * D)[c * 4 + sub] = w;
                    }
                }
            } else {
                // a piece: the place of tile pairs begun by others, or of the one begun here
                const int row = i * 128 + r;
                Piece<D>& piece = static_cast<Piece<D>*>(p.pieces)[2 * blockIdx.x + (it.b0 == 0 ? 1 : 0)];
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t y[32];
                    tmem_ld32(my_o + 32 * c, y);
                    tmem_ld_wait();
                    if (row < rows) {
#pragma unroll
                        for (int v = 0; v < 8; ++v) reinterpret_cast<uint4*>(&piece.o[row][32 * c])[v] = make_uint4(y[4 * v], y[4 * v + 1], y[4 * v + 2], y[4 * v + 3]);
                    }
                }
                if (row < rows) piece.ml[row] = make_float2(m, l);
                if (it.b0 == 0) {
                    const int of_seq = (s.len[it.seq] + tokens - 1) / tokens;
                    const long long total = s.before[p.n_seqs], last = s.before[it.seq] + ((long long)it.pack * of_seq + it.t0 / tokens + 1) * it.nb;
                    if (threadIdx.x == 0) p.notes[blockIdx.x] = {total, (int)((last * gridDim.x - 1) / total), s.start[it.seq] + it.t0, rows, it.pack};
                }
            }
            tc_fence_before();
        }
    }
    // (every thread gets here, also after an abandoned wait)
    if (*abort_flag) settle();
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Joins the pieces of the tile pair that CTA blockIdx.x of the first launch began and did not end: o = sum f o_i / sum f l_i, f = 2^(c (m_i - max m)).
// A warp takes a row at a time.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const CrossParams p, int ctas) {
    pdl_launch_dependents();
    pdl_wait();
    const Note note = p.notes[blockIdx.x];
    if (note.last < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = gridDim.y * (kJoinThreads / 32);
    const Piece<D>* const pieces = static_cast<const Piece<D>*>(p.pieces);
    const int n = note.last - blockIdx.x + 1;
    auto piece = [&](int i) -> const Piece<D>& { return pieces[2 * (blockIdx.x + i) + (i == 0 ? 1 : 0)]; };
    // (a CTA of fewer units than there are CTAs may have had none)
    auto there = [&](int i) { return share_begin(note.total, blockIdx.x + i, ctas) < share_begin(note.total, blockIdx.x + i + 1, ctas); };
    for (int row = blockIdx.y * (kJoinThreads / 32) + warp; row < note.rows; row += warps) {
        float m = -INFINITY, l = 0.f, o[D / 32];
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
        for (int i = lane; i < n; i += 32)
            if (there(i) && piece(i).ml[row].y != 0.f) m = fmaxf(m, piece(i).ml[row].x);     // (0: all its scores minus infinity)
        m = warp_max(m);
        for (int i0 = 0; i0 < n; i0 += 32) {
            float f = -1.f;                   // nothing to add
            if (i0 + lane < n && there(i0 + lane)) {
                const float2 ml = piece(i0 + lane).ml[row];
                if (ml.y != 0.f) {
                    f = ml.y == ml.y ? ex2((ml.x - m) * p.c) : ml.y;
                    l += ml.y * f;
                }
            }
#pragma unroll 4
            for (int k = 0; k < min(32, n - i0); ++k) {
                const float g = __shfl_sync(0xffffffffu, f, k);
                const float* const x = piece(i0 + k).o[row] + lane;
                if (g != -1.f) {
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) o[e] = fmaf(x[32 * e], g, o[e]);
                }
            }
        }
        const float inv = 1.f / warp_sum(l);
        const int token = note.row + (row >> p.pack_shift), head = note.pack * p.pack + (row & (p.pack - 1));
        uint16_t* const out = p.out + ((int64_t)token * p.q_heads + head) * D;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) out[lane + 32 * e] = f_to_bf16(o[e] * inv);
    }
}

template <int D>
mt_status launch(const CrossArgs& a, CrossParams& p, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const OpContext& c, cudaStream_t s) {
    const int grid = c.sm_count;
    for (int seq0 = 0; seq0 < a.d.n_seqs; seq0 += kMaxSeqs) {
        p.seq0 = seq0;
        p.n_seqs = a.d.n_seqs - seq0 < kMaxSeqs ? a.d.n_seqs - seq0 : kMaxSeqs;
        p.offsets = a.offsets + seq0;
        p.ranges = a.ranges + 2 * (int64_t)seq0;
        cudaError_t e = launch_pdl(cross_attention_kernel<D>, dim3((unsigned)grid), dim3(kThreads), (size_t)shared_bytes<D>(), s, mq, mk, mv, p);
        if (e == cudaSuccess && p.whole != 1) {
            const int64_t all = (int64_t)a.d.n_tokens * p.pack, rows = all < 256 ? all : 256;                          // of a tile pair, at most
            e = launch_pdl(join_kernel<D>, dim3((unsigned)grid, (unsigned)((rows + 15) / 16)), dim3(kJoinThreads), 0, s, p, grid);
        }
        if (e != cudaSuccess) return MT_ERR_CUDA;
        if (a.d.n_seqs - seq0 <= kMaxSeqs) break;
    }
    return MT_OK;
}

}  // namespace

cudaError_t configure_cross_attention() {
    cudaError_t e = cudaFuncSetAttribute(cross_attention_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes<64>());
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(cross_attention_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes<128>());
    return e;
}

mt_status launch_cross_attention(const CrossArgs& a, const OpContext& c, cudaStream_t s) {
    const mt_cross_desc& d = a.d;
    CrossParams p;
    p.n_tokens = d.n_tokens;
    p.n_states = d.n_states;
    p.q_heads = d.q_heads;
    p.group = d.q_heads / d.kv_heads;
    p.pack = 1;
    p.pack_shift = 0;
    while (p.pack < 16 && p.group % (2 * p.pack) == 0) { p.pack *= 2; ++p.pack_shift; }
    p.c = fmaxf(fabsf(d.scale) * 1.44269504088896341f, 1e-30f);   // not zero: minus infinity has to stay what it is
    p.negate = d.scale < 0.f;
    p.out = a.out;
    p.status = a.status;
    // tile pairs of all sequences together, at least (where the offsets take in all tokens)
    const int64_t pairs = ((int64_t)d.n_tokens * p.pack + 255) / 256 * (d.q_heads / p.pack);
    p.whole = pairs >= (int64_t)kEnough * c.sm_count ? 1 : pairs >= c.sm_count ? 2 : 0;
    p.notes = nullptr;
    p.pieces = nullptr;
    if (p.whole != 1) {
        const size_t notes = (sizeof(Note) * c.sm_count + 255) / 256 * 256;
        uint8_t* w;
        const mt_status st = op_scratch(s, notes + 2 * (size_t)c.sm_count * (d.head_dim == 64 ? sizeof(Piece<64>) : sizeof(Piece<128>)), &w);
        if (st != MT_OK) return st;
        p.notes = reinterpret_cast<Note*>(w);
        p.pieces = w + notes;
    }
    CUtensorMap mq, mk, mv;
    mt_status st = encode_rows(c, &mq, a.q, d.head_dim, d.q_heads, d.n_tokens, d.q_head_stride, d.q_token_stride, p.pack, 128 / p.pack);
    if (st == MT_OK) {
        if (d.n_states > 0) {
            st = encode_rows(c, &mk, a.k, d.head_dim, d.kv_heads, d.n_states, d.k_head_stride, d.k_token_stride, 1, kBlock);
            if (st == MT_OK) st = encode_rows(c, &mv, a.v, d.head_dim, d.kv_heads, d.n_states, d.v_head_stride, d.v_token_stride, 1, kBlock);
        } else {                               // nothing of it is used, but a map describes something
            st = encode_rows(c, &mk, a.q, d.head_dim, d.q_heads, d.n_tokens, d.q_head_stride, d.q_token_stride, 1, kBlock);
            mv = mk;
        }
    }
    if (st != MT_OK) return st;
    return d.head_dim == 64 ? launch<64>(a, p, mq, mk, mv, c, s) : launch<128>(a, p, mq, mk, mv, c, s);
}

}  // namespace mt

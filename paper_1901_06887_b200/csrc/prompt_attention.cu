// Causal attention over packed prompts on the tensor cores.
//
// Mathematics.  o_i = sum_{j <= i} p_ij v_j / sum_{j <= i} p_ij, p_ij = 2^(c (q_i . k_j - m_i)), c = scale log2(e), in one pass over blocks of
// 128 keys.  m_i is a running reference, not the maximum: it moves, and the sums so far are rescaled, only when a block's maximum lies
// more than 8 above it (in log2); until then p is at most 2^8, which fp32 sums and the bf16 p hold as exactly as 1.
// p is rounded to bf16 before it meets v: kind::f16 takes one type for both operands, and v is bf16.  The roundings (2^-8 of a p at
// most) are independent and average out, and l sums the unrounded p: over 8192 tokens the output is 0.0021 off 64 bits (relative, root mean square)
// where its own rounding to bf16 makes 0.0016.  P in two bf16 parts would take the difference away and double P V, half as much again of the tensor
// pipe's time, which already bounds the kernel together with the exponentials.
//
// Tile.  A CTA owns two tiles of 128 rows (one tensor-memory accumulator each) and streams the keys and values that either needs.
// A row is a (token, head) pair: R heads that share a key/value head (the largest power of two in the group) are packed into the rows, so
// short prompts fill the tile and the keys are read once for R heads.  Rows of a tile then lie in one block of 128 keys, so only
// a tile's last block is masked.
//
// Roles (12 warps): warps 0-3 and 4-7 are the softmax of the two tiles, one row per thread; warp 8 copies (TMA), warp 9 issues the
// matrix instructions, warps 10 and 11 clean masked value blocks.  S = Q K^T goes to tensor memory, comes to registers, goes back as bf16 P
// over the columns of S, and P V takes P from there.  While one tile is in its softmax the other has the tensor cores.
//
// Masked positions.  p of a masked key is zero, but zero times an infinity is NaN, so values that some row must not see are made
// harmless in shared memory before the product: rows past the sequence's end are zeroed, and an element that is not finite in a
// masked block is zeroed and noted, the first token per channel; rows at or after that token get NaN there in the epilogue.
//
// Order of work.  Tiles of all sequences, longest first, dealt back and forth over one CTA per SM; every CTA derives the list from the
// offsets (sequences ranked by length; tile numbers between the lengths of ranks r and r + 1 exist for exactly r + 1 sequences).
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kThreads = 384;
constexpr int kBlock = 128;                   // keys per block, rows per tile
constexpr int kHalf = kBlock * 128;           // bytes of a 128-row, 64-channel operand
constexpr int kMaxSeqs = 512;                 // sequences of one launch
constexpr int kItems = 256;                   // tiles of a CTA that are looked up once, at the start
constexpr float kSlack = 8.f;

template <int D> __host__ __device__ constexpr int slots() { return D == 128 ? 4 : 8; }
template <int D> __host__ __device__ constexpr int operand_bytes() { return kHalf * (D / 64); }

struct Control {
    uint64_t q_full[2], q_empty, s_full[2], p_half[2], p_ready[2], o_ready[2], epi_done[2], kv_full[8], kv_empty[8], v_raw[8], v_clean[8];
    uint32_t tmem;
    int abort;
    int poison[2];                            // round + 1 of a tile with notes
    unsigned long long first_bad[2][128];     // per channel: (0x7fffffff - round, first token that is not finite); later rounds win the minimum
    int start[kMaxSeqs], len[kMaxSeqs], order[kMaxSeqs], before[kMaxSeqs + 1];
    int total;
    int4 item[kItems];                        // this CTA's first tiles: row of the sequence's start, its length, first token, head pack
};
constexpr int kControlBytes = ((int)sizeof(Control) + 127) / 128 * 128;
constexpr int kStageBytes = 8 * 2048;           // output staging of the eight softmax warps
template <int D> constexpr int shared_bytes() { return 1024 + (2 + slots<D>()) * operand_bytes<D>() + kControlBytes + kStageBytes; }

struct PromptParams {
    const int32_t* offsets;
    int n_seqs, seq0, n_tokens;
    int q_heads, group, pack, pack_shift;     // pack: heads packed into a tile's rows
    float c;                                  // |scale| log2(e)
    int negate;                               // scale < 0
    uint16_t* out;
    OpStatus status;
};

// D (+)= A B with A in tensor memory.
template <bool ACC>
__device__ __forceinline__ void umma_tmem_a_lohi(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        ".reg .b64 db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t"
        "}\n"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(kDescHiSw128), "r"(idesc), "n"(ACC ? 1 : 0)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Descriptor words of the values, 128-byte swizzle with the channels contiguous: the product's inner index is the token (8-token groups 1024
// bytes apart, as in the row-major form), and the 64-channel halves lie kHalf apart.
constexpr uint32_t kHalfField = static_cast<uint32_t>(kHalf >> 4) << 16;
__device__ __forceinline__ uint32_t desc_lo_values(uint32_t smem_addr) { return ((smem_addr & 0x3FFFFu) >> 4) | kHalfField; }

struct Item {
    int start, len, t0, pack;                 // first row of the sequence, its length, first token of the tile pair, head pack
    int nb[2];                                // key blocks of the two tiles (0: no rows)
};

// The tile pair of a round, or a length of 0 behind the last.
__device__ __forceinline__ int4 find_item(const Control& s, const PromptParams& p, int round) {
    const int packs = p.q_heads >> p.pack_shift;
    const int64_t x = (int64_t)round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    if (x >= (int64_t)s.total * packs) return make_int4(0, 0, 0, 0);
    const int k = (int)(x / packs);
    const int tokens = 256 >> p.pack_shift;   // of the tile pair
    int lo = 0, hi = p.n_seqs - 1;            // rank r with before[r] <= k < before[r + 1]
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.before[mid] <= k) lo = mid; else hi = mid - 1;
    }
    const int q = k - s.before[lo];
    const int tile = (s.len[s.order[lo]] + tokens - 1) / tokens - 1 - q / (lo + 1);
    const int seq = s.order[q % (lo + 1)];
    return make_int4(s.start[seq], s.len[seq], tile * tokens, (int)(x - (int64_t)k * packs));
}
__device__ __forceinline__ bool get_item(const Control& s, const PromptParams& p, int round, Item& it) {
    const int4 v = round < kItems ? s.item[round] : find_item(s, p, round);
    it.start = v.x; it.len = v.y; it.t0 = v.z; it.pack = v.w;
    const int half = 128 >> p.pack_shift;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int first = it.t0 + i * half, last = min(first + half, it.len) - 1;
        it.nb[i] = first < it.len ? last / kBlock + 1 : 0;
    }
    return it.len > 0;
}

// After an abandoned wait: a bounded time for copies and matrix instructions that are still in flight.
__device__ __noinline__ void settle() {
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 2000000ull) __nanosleep(1000);
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
prompt_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v, const PromptParams p) {
    extern __shared__ uint8_t smem_raw[];
    constexpr int kSlots = slots<D>(), kOp = operand_bytes<D>();
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - raw);
    Control& s = *reinterpret_cast<Control*>(smem + (2 + kSlots) * kOp);
    const uint32_t q_smem = base, kv_smem = base + 2 * kOp;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* const abort_flag = &s.abort;
    auto bar = [](const uint64_t& b) { return smem_u32(&b); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(s.q_full[i]), 1); mbar_init(bar(s.s_full[i]), 1); mbar_init(bar(s.p_half[i]), 128); mbar_init(bar(s.p_ready[i]), 128);
            mbar_init(bar(s.o_ready[i]), 1); mbar_init(bar(s.epi_done[i]), 256);
            s.poison[i] = 0;
        }
        mbar_init(bar(s.q_empty), 1);
        for (int i = 0; i < kSlots; ++i) { mbar_init(bar(s.kv_full[i]), 1); mbar_init(bar(s.kv_empty[i]), 1); mbar_init(bar(s.v_raw[i]), 1); mbar_init(bar(s.v_clean[i]), 64); }
        s.abort = 0;
        fence_mbar_init();
    }
    if (threadIdx.x < 256) s.first_bad[threadIdx.x >> 7][threadIdx.x & 127] = ~0ull;
    if (warp == 9 && lane == 0) { prefetch_tensormap(&map_q); prefetch_tensormap(&map_k); prefetch_tensormap(&map_v); }
    pdl_wait();
    // All of tensor memory, taken only when the predecessor is done with its share, and before a successor may start and ask for its own.
    if (warp == 8) {
        tmem_alloc(smem_u32(&s.tmem), 512);
        tmem_relinquish();
    }

    // --- the list of tiles: sequences ranked by length
    const int tokens = 256 >> p.pack_shift;
    for (int i = threadIdx.x; i < p.n_seqs; i += kThreads) {
        const int a = p.offsets[i], b = p.offsets[i + 1];
        const bool bad = a < 0 || b < a || b > p.n_tokens;
        if (bad && blockIdx.x == 0) raise_status(p.status, MT_ERR_INVALID_ARG, p.seq0 + i);
        s.start[i] = a;
        s.len[i] = bad ? 0 : b - a;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.n_seqs; i += kThreads) {
        const int n = s.len[i];
        int rank = 0;
        for (int j = 0; j < p.n_seqs; ++j) { const int m = s.len[j]; rank += (m > n || (m == n && j < i)) ? 1 : 0; }
        s.order[rank] = i;
    }
    __syncthreads();
    if (warp == 0) {                            // before[r]: tiles whose number is shared by fewer than r + 1 sequences
        int run = 0;
        for (int r0 = 0; r0 < p.n_seqs; r0 += 32) {
            const int r = r0 + lane;
            int v = 0;
            if (r < p.n_seqs) {
                const int mine = (s.len[s.order[r]] + tokens - 1) / tokens;
                const int next = r + 1 < p.n_seqs ? (s.len[s.order[r + 1]] + tokens - 1) / tokens : 0;
                v = (r + 1) * (mine - next);
            }
            int incl = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += y;
            }
            if (r < p.n_seqs) s.before[r] = run + incl - v;
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) { s.before[p.n_seqs] = run; s.total = run; }
    }
    __syncthreads();
    if (threadIdx.x < kItems) s.item[threadIdx.x] = find_item(s, p, threadIdx.x);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = s.tmem;
    const uint32_t tmem_s = tmem, tmem_o = tmem + 256;         // S (and P) of tile i: + 128 i; O: + D i
    const int head_of_pack = p.pack;

    if (warp == 8) {
        // ------------------------------------------------------------------------------------------ copies
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (lane == 0) {
            int fill = 0;                        // operands put into the ring so far
            bool ok = true;
            Item it;
            for (int round = 0; ok && get_item(s, p, round, it); ++round) {
                if (round > 0) ok = mbar_wait(bar(s.q_empty), (round - 1) & 1, abort_flag, p.status.word, 200);
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (it.nb[i] == 0) continue;
                    mbar_expect_tx(bar(s.q_full[i]), kOp);
                    for (int h = 0; h < D / 64; ++h)
                        tma_load_3d(q_smem + i * kOp + h * kHalf, &map_q, h * 64, it.pack * head_of_pack, it.start + it.t0 + i * (tokens / 2), bar(s.q_full[i]));
                }
                const int kv_head = it.pack * p.pack / p.group;
                const int nb = max(it.nb[0], it.nb[1]);
                for (int x = 0; ok && x < 2 * nb; ++x, ++fill) {
                    const int slot = fill % kSlots, use = fill / kSlots;
                    if (use > 0) ok = mbar_wait(bar(s.kv_empty[slot]), (use - 1) & 1, abort_flag, p.status.word, 201);
                    if (!ok) break;
                    // a masked value block goes to the cleaners first: its bytes count on v_raw, and v_clean says when it may be used
                    const bool masked = (x & 1) && ((x >> 1) == it.nb[0] - 1 || (x >> 1) == it.nb[1] - 1);
                    const uint32_t full = masked ? bar(s.v_raw[slot]) : bar(s.kv_full[slot]);
                    mbar_expect_tx(full, kOp);
                    for (int h = 0; h < D / 64; ++h)
                        tma_load_3d(kv_smem + slot * kOp + h * kHalf, (x & 1) ? &map_v : &map_k, h * 64, kv_head, it.start + (x >> 1) * kBlock, full);
                    if (masked) mbar_arrive(bar(s.kv_full[slot]));
                }
            }
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------------------------------ matrix instructions
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        // The whole warp walks the loop, so that addresses stay warp-uniform; one elected lane issues.  (One lane alone, with descriptors
        // built per instruction, took 115 cycles for each of them: 1900 for the sixteen that a tile's block needs, against 512 of work.)
        const bool leader = elect_one();
        constexpr uint32_t kIdPv = make_idesc_bf16(128, D) | (1u << 16);
        const uint32_t id_qk = make_idesc_bf16(128, kBlock) | (p.negate ? 1u << 13 : 0u);
        const uint32_t q_lo = desc_lo(q_smem), k_lo = desc_lo(kv_smem), v_lo = desc_lo_values(kv_smem);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        constexpr uint32_t kOpLo = kOp >> 4;
        uint32_t fill = 0, n_q0 = 0, n_q1 = 0, n_p0 = 0, n_p1 = 0, clean_phase = 0;
        bool ok = true;
        Item it;
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
        // the first 64 keys go while the second half of P is still in its exponentials
        auto pv = [&](int i, uint32_t slot, bool first, uint32_t n) {
            const uint32_t d = tm + 256 + D * i, a = tm + 128 * i, b = v_lo + slot * kOpLo;
            wait(s.p_half[i], n, 214);
            if (!ok) return;
            tc_fence_after();
            if (leader) {
                if (first) umma_tmem_a_lohi<false>(d, a, b, kIdPv);
                else umma_tmem_a_lohi<true>(d, a, b, kIdPv);
#pragma unroll
                for (int k = 1; k < kBlock / 32; ++k) umma_tmem_a_lohi<true>(d, a + 8 * k, b + (2048 >> 4) * k, kIdPv);
            }
            wait(s.p_ready[i], n, 216);
            if (!ok) return;
            tc_fence_after();
            if (leader) {
#pragma unroll
                for (int k = kBlock / 32; k < kBlock / 16; ++k) umma_tmem_a_lohi<true>(d, a + 8 * k, b + (2048 >> 4) * k, kIdPv);
                umma_commit(bar(s.o_ready[i]));
            }
        };
        for (int round = 0; ok && get_item(s, p, round, it); ++round) {
            const int nb0 = __shfl_sync(0xffffffffu, it.nb[0], 0), nb1 = __shfl_sync(0xffffffffu, it.nb[1], 0), nb = max(nb0, nb1);
            uint32_t slot = fill % kSlots;
            wait(s.kv_full[slot], fill / kSlots, 210);
            wait(s.q_full[0], n_q0++, 211);
            if (!ok) break;
            tc_fence_after();
            qk(0, slot);
            if (nb1 > 0) {
                wait(s.q_full[1], n_q1++, 211);
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
                wait(s.kv_full[vslot], vx / kSlots, 212);
                if (j == nb0 - 1 || j == nb1 - 1) {
                    wait(s.v_clean[vslot], clean_phase >> vslot, 213);
                    clean_phase ^= 1u << vslot;
                }
                if (j + 1 < nb) wait(s.kv_full[kslot], kpar, 215);
                if (j < nb0) {
                    pv(0, vslot, j == 0, n_p0++);
                    if (!ok) break;
                    if (j + 1 < nb0) qk(0, kslot);
                }
                if (j < nb1) {
                    pv(1, vslot, j == 0, n_p1++);
                    if (!ok) break;
                    if (j + 1 < nb1) qk(1, kslot);
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
        // ------------------------------------------------------------------------------------------ masked value blocks
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        const int t = threadIdx.x - 320;         // rows t and t + 64
        int fill = 0;
        uint32_t raw_phase = 0;
        bool ok = true;
        Item it;
        for (int round = 0; ok && get_item(s, p, round, it); ++round) {
            const int nb = max(it.nb[0], it.nb[1]), buf = round & 1;
            if (round >= 2) {                    // the notes of two tiles ago have been read
                ok = mbar_wait(bar(s.epi_done[buf]), ((round >> 1) - 1) & 1, abort_flag, p.status.word, 220);
                if (!ok) break;
            }
            for (int j = it.nb[0] - 1; ok && j < nb; ++j) {
                if (!(j == it.nb[0] - 1 || j == it.nb[1] - 1)) continue;
                const int slot = (fill + 2 * j + 1) % kSlots;
                ok = mbar_wait(bar(s.v_raw[slot]), (raw_phase >> slot) & 1, abort_flag, p.status.word, 221);
                if (!ok) break;
                raw_phase ^= 1u << slot;
                uint8_t* const v = smem + (2 + slot) * kOp;
                for (int r = t; r < kBlock; r += 64) {
                    const int tok = j * kBlock + r;
                    auto piece = [&](int c) { return reinterpret_cast<uint4*>(v + (c / 8) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4)); };
                    if (tok >= it.len) {
#pragma unroll
                        for (int c = 0; c < D / 8; ++c) *piece(c) = make_uint4(0, 0, 0, 0);
                        continue;
                    }
                    uint32_t any = 0;
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) {
                        const uint4 w = *piece(c);
                        any |= ((w.x & 0x7f807f80u) + 0x00800080u) | ((w.y & 0x7f807f80u) + 0x00800080u) | ((w.z & 0x7f807f80u) + 0x00800080u) |
                               ((w.w & 0x7f807f80u) + 0x00800080u);
                    }
                    if ((any & 0x80008000u) == 0) continue;
                    const unsigned long long note = (unsigned long long)(0x7fffffff - round) << 32 | (uint32_t)tok;
                    s.poison[buf] = round + 1;
#pragma unroll 1
                    for (int c = 0; c < D / 8; ++c) {
                        uint32_t* const w = reinterpret_cast<uint32_t*>(piece(c));
                        for (int e = 0; e < 4; ++e) {
                            uint32_t y = w[e];
                            if ((y & 0x7f80u) == 0x7f80u) { y &= 0xffff0000u; atomicMin(&s.first_bad[buf][c * 8 + 2 * e], note); }
                            if ((y & 0x7f800000u) == 0x7f800000u) { y &= 0x0000ffffu; atomicMin(&s.first_bad[buf][c * 8 + 2 * e + 1], note); }
                            w[e] = y;
                        }
                    }
                }
                fence_proxy_async_smem();
                __threadfence_block();
                mbar_arrive(bar(s.v_clean[slot]));
            }
            fill += 2 * nb;
        }
    } else {
        // ------------------------------------------------------------------------------------------ softmax, one row per thread
        // registers move here: 256 threads x 208 + 128 x 88 = the launch's 384 x 168
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int i = warp >> 2;
        const int r = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;     // tensor-memory lane of the warp's first row, in the address's upper half
        const uint32_t my_s = tmem_s + 128 * i + lanes, my_o = tmem_o + D * i + lanes;
        int n_s = 0, n_o = 0;
        bool ok = true;
        Item it;
        for (int round = 0; ok && get_item(s, p, round, it); ++round) {
            const int nb = it.nb[i], buf = round & 1;
            const int tok = it.t0 + i * (tokens / 2) + (r >> p.pack_shift);
            float m = 0.f, l = 0.f;
            for (int j = 0; j < nb; ++j) {
                ok = mbar_wait(bar(s.s_full[i]), n_s++ & 1, abort_flag, p.status.word, 230);
                if (!ok) break;
                tc_fence_after();
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(my_s + 32 * c, x[c]);
                tmem_ld_wait();
                if (j == nb - 1) {
                    const int lim = tok - j * kBlock;          // keys of the block up to here are seen
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * c + e > lim) x[c][e] = 0xff800000u;
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
                if (j == 0) {
                    m = mx > -INFINITY ? mx : 0.f;
                } else if (__any_sync(0xffffffffu, move)) {
                    // (a row moves on its own account only, so its bits do not depend on its neighbours)
                    const float nm = move && mx > -INFINITY ? mx : m, f = m == nm || l == 0.f ? 1.f : ex2((m - nm) * p.c);
                    m = nm;
                    l *= f;
                    ok = mbar_wait(bar(s.o_ready[i]), (n_o - 1) & 1, abort_flag, p.status.word, 231);
                    if (!ok) break;
                    tc_fence_after();
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
                    tmem_st16(my_s + 16 * c, w);
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
            // A tile without rows waits for nothing else, and must not run ahead: it would arrive on epi_done twice in one phase, in the place of
            // the other tile.  (A tile with rows ends its round behind the cleaners, who have waited for the same phase.)
            if (nb == 0 && round >= 2) {
                ok = mbar_wait(bar(s.epi_done[buf]), ((round >> 1) - 1) & 1, abort_flag, p.status.word, 233);
                if (!ok) break;
            }
            if (nb > 0) {
                ok = mbar_wait(bar(s.o_ready[i]), (n_o - 1) & 1, abort_flag, p.status.word, 232);
                if (!ok) break;
                tc_fence_after();
                const float inv = 1.f / l;
                const bool poison = *(volatile int*)&s.poison[buf] == round + 1;
                // 32 channels at a time through shared memory, so that four lanes store 64 contiguous bytes of a row: a row per lane
                // would touch 32 lines with every store
                uint4* const stage = reinterpret_cast<uint4*>(smem + (2 + kSlots) * kOp + kControlBytes) + warp * 128;
                const int sub = lane & 3;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t y[32];
                    tmem_ld32(my_o + 32 * c, y);
                    tmem_ld_wait();
                    if (poison) {
                        const unsigned long long note = (unsigned long long)(0x7fffffff - round) << 32 | (uint32_t)tok;
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (s.first_bad[buf][32 * c + e] <= note) y[e] = 0x7fffffffu;     // an older round's note is larger
                    }
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
                        const int row = v * 8 + (lane >> 2), of_tile = (warp & 3) * 32 + row;
                        const int row_tok = it.t0 + i * (tokens / 2) + (of_tile >> p.pack_shift);
                        const int head = it.pack * p.pack + (of_tile & (p.pack - 1));
                        const uint4 w = stage[row * 4 + (sub ^ ((row >> 1) & 3))];
                        if (row_tok < it.len)
                            reinterpret_cast<uint4*>(p.out + ((int64_t)(it.start + row_tok) * p.q_heads + head) * D)[c * 4 + sub] = w;
                    }
                }
                tc_fence_before();
            }
            mbar_arrive(bar(s.epi_done[buf]));
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

mt_status encode_rows(const OpContext& c, CUtensorMap* map, const uint16_t* ptr, int d, int heads, int tokens, int64_t head_stride,
                      int64_t token_stride, int box_heads, int box_tokens) {
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)head_stride * 2, (cuuint64_t)token_stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
    const cuuint32_t one[3] = {1, 1, 1};
    const CUresult r = c.encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t*>(ptr), dims, strides, box, one,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? MT_OK : MT_ERR_CUDA;
}

}  // namespace

cudaError_t configure_prompt_attention() {
    cudaError_t e = cudaFuncSetAttribute(prompt_attention_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes<64>());
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(prompt_attention_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes<128>());
    return e;
}

mt_status launch_prompt_attention(const PromptArgs& a, const OpContext& c, cudaStream_t s) {
    const mt_prompt_desc& d = a.d;
    PromptParams p;
    p.n_tokens = d.n_tokens;
    p.q_heads = d.q_heads;
    p.group = d.q_heads / d.kv_heads;
    p.pack = 1;
    p.pack_shift = 0;
    while (p.pack < 16 && p.group % (2 * p.pack) == 0) { p.pack *= 2; ++p.pack_shift; }
    p.c = fmaxf(fabsf(d.scale) * 1.44269504088896341f, 1e-30f);   // not zero: minus infinity has to stay what it is
    p.negate = d.scale < 0.f;
    p.out = a.out;
    p.status = a.status;
    CUtensorMap mq, mk, mv;
    mt_status st = encode_rows(c, &mq, a.q, d.head_dim, d.q_heads, d.n_tokens, d.q_head_stride, d.q_token_stride, p.pack, 128 / p.pack);
    if (st == MT_OK) st = encode_rows(c, &mk, a.k, d.head_dim, d.kv_heads, d.n_tokens, d.k_head_stride, d.k_token_stride, 1, kBlock);
    if (st == MT_OK) st = encode_rows(c, &mv, a.v, d.head_dim, d.kv_heads, d.n_tokens, d.v_head_stride, d.v_token_stride, 1, kBlock);
    if (st != MT_OK) return st;
    for (int seq0 = 0; seq0 < d.n_seqs; seq0 += kMaxSeqs) {
        p.seq0 = seq0;
        p.n_seqs = d.n_seqs - seq0 < kMaxSeqs ? d.n_seqs - seq0 : kMaxSeqs;
        p.offsets = a.offsets + seq0;
        // no more CTAs than there can be tiles
        const int64_t most = (((int64_t)d.n_tokens * p.pack + 255) / 256 + p.n_seqs) * (d.q_heads / p.pack);
        const unsigned grid = (unsigned)(most < c.sm_count ? most : c.sm_count);
        const cudaError_t e = d.head_dim == 64
            ? launch_pdl(prompt_attention_kernel<64>, dim3(grid), dim3(kThreads), (size_t)shared_bytes<64>(), s, mq, mk, mv, p)
            : launch_pdl(prompt_attention_kernel<128>, dim3(grid), dim3(kThreads), (size_t)shared_bytes<128>(), s, mq, mk, mv, p);
        if (e != cudaSuccess) return MT_ERR_CUDA;
        if (d.n_seqs - seq0 <= kMaxSeqs) break;
    }
    return MT_OK;
}

}  // namespace mt

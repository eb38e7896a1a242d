// Products of a mixed batch of rows with the tenants' 4-bit weights: y_r = sum_k scale (code - 8) x_rk + bias, tenant by tenant.
//
// Mathematics.  The codes enter the matrix instructions as the exact bf16 numbers code - 8 (four bits set into the mantissa of 128, then an
// exact subtraction of 136) with the weights as the 16-row operand and up to 64 of the tenant's rows as columns; the sum over 64 (or 32)
// inputs is multiplied with the group's scale in fp32 and added up in fp32.  Nothing is rounded but the sums.
//
// Cost.  K / 2 + 2 K / group bytes per output and tenant, whatever the number of its rows (up to some 16; beyond, the matrix instructions), and 113
// warp instructions per 16 outputs x 64 inputs.  No unit is full (8 tenants of 4096 -> 16384, 24 rows): logic pipe 62 %, issue slots 63 %, memory 37 %,
// with 16 warps an SM to hide latency.  The packed order makes a warp's load 512 contiguous bytes that are the operand of four instructions; the rows' slices of the
// inner index are chosen so that a lane's inputs are 16 contiguous bytes too.
//
// Split.  A CTA takes (tenant, 32 outputs) units in turn, its eight warps every eighth block of 64 inputs; they join through shared memory.
// Every warp copies its blocks ahead into a ring of its own (cp.async, three or seven blocks ahead, on through the units to come), so the joins and
// the ends of units do not empty the pipe: loading into registers unit by unit left the kernel waiting for memory (93 us for 8 tenants of
// 4096 -> 16384, 24 rows).  Two tiles of 16 outputs share the rows' loads and the loop: 88 us.
// Which tenants occur is found out by every CTA for itself from the ids (at most 256 a launch): no bucketing launch, and only tenants that
// occur cost anything.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

// One thread per 32-bit word of the packed codes, then one per scale.
__global__ void quant_pack_kernel(const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales, int tenants, int K, int N,
                                  int group, uint8_t* __restrict__ packed, size_t tenant_bytes, size_t codes_bytes) {
    const size_t words = codes_bytes / 4, n_scales = (tenant_bytes - codes_bytes) / 2, per = words + n_scales;
    const size_t step = (size_t)gridDim.x * blockDim.x;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < per * tenants; i += step) {
        const size_t t = i / per, r = i % per;
        uint8_t* out = packed + t * tenant_bytes;
        if (r < words) {
            const int w = (int)(r & 3), lane = (int)(r >> 2) & 31;
            const size_t block = r >> 7;
            const int kb = (int)(block % (K / 64));
            const int row = (int)(block / (K / 64)) * 16 + lane / 4 + 8 * (w >> 1);
            const int k0 = kb * 64 + 32 * (w & 1) + 8 * (lane & 3);
            uint32_t v = 0;
            if (row < N) {
                const uint8_t* src = codes + (t * N + row) * (size_t)(K / 2) + k0 / 2;
                for (int p = 0; p < 4; ++p) v |= (uint32_t)(src[p] & 15) << (4 * p) | (uint32_t)(src[p] >> 4) << (4 * p + 16);
            }
            reinterpret_cast<uint32_t*>(out)[r] = v;
        } else {
            const size_t q = r - words;
            const size_t block = q >> 4;
            const int g = (int)(block % (K / group));
            const int row = (int)(block / (K / group)) * 16 + (int)(q & 15) / 2 + 8 * (int)(q & 1);
            reinterpret_cast<uint16_t*>(out + codes_bytes)[q] = row < N ? scales[(t * N + row) * (size_t)(K / group) + g] : uint16_t(0);
        }
    }
}

constexpr int kThreads = 256, kWarps = 8;

// D = A B + C
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3,
                                         const uint32_t b0, const uint32_t b1, const float (&c)[4]) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// Codes in nibbles P and P + 4 of w as two bf16 numbers code - 8.
template <int P>
__device__ __forceinline__ uint32_t centred(uint32_t w) {
    uint32_t d;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(((w >> (4 * P)) & 0x000f000fu) | 0x43004300u), "r"(0xc308c308u));   // 128 + code - 136
    return d;
}

constexpr int kCodes = 1024, kStageBytes = kCodes + 128;        // a block's codes and scales of two tiles of 16 outputs
// Places in a warp's ring: eight for calls of few rows, where a warp has about that many blocks altogether and waits once for all of them
// (4096 x 4096, one row: 7.9 us against 10.1 with four); four where the columns' partial sums need the memory.
__host__ __device__ constexpr int stages(int maxt) { return maxt == 1 ? 8 : 4; }

// CTAs of an SM at once, which is also what a launch has of them: a further one would start when another has ended, sort the ids again and
// fill its ring from nothing (three for calls of few rows, of which two fit: one row of 4096 -> 16384 17.8 us against 16.5, 8 tenants 94 against 86).
__host__ __device__ constexpr int resident(int maxt) { return maxt == 2 ? 3 : maxt <= 4 ? 2 : 1; }

struct Shared {
    int ids[kQuantRowsPerLaunch], slot[kQuantRowsPerLaunch], order[kQuantRowsPerLaunch];
    int tenant[kQuantRowsPerLaunch], begin[kQuantRowsPerLaunch + 1];
    int group_slot[kQuantRowsPerLaunch], group_row[kQuantRowsPerLaunch];       // groups of at most 64 rows of one tenant
    int warp_n[kWarps];
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// Units in turn: pairs of tiles of one group of rows, gridDim.x apart.
struct Cursor {
    int group, pair;
    __device__ __forceinline__ void next(int pairs) {
        pair += gridDim.x;
        while (pair >= pairs) { pair -= pairs; ++group; }
    }
};

// A warp's blocks of all its units, in order: unit, then blocks warp, warp + 8, ...; copied ahead into the warp's ring.
template <bool G32, int STAGES>
struct Stream {
    const QuantLinearArgs& a;
    const Shared& s;
    int warp, lane, kblocks, pairs, n_groups;
    Cursor at;
    int kb, left;                             // left: blocks still to be copied
    const uint8_t *codes, *scales;            // this lane's, of the current unit
    int64_t second;                           // bytes from the first tile's codes to the second's
    uint32_t ring;                            // shared memory of this lane's piece of stage 0
    int in;                                   // byte offset of the stage to fill

    __device__ __forceinline__ void seek() {  // to the unit's first block
        kb = warp;
        if (at.group >= n_groups) return;
        const uint8_t* const base = a.packed + (size_t)s.tenant[s.group_slot[at.group]] * a.tenant_bytes;
        const int tile = 2 * at.pair, other = min(tile + 1, a.tiles - 1);       // (a missing second tile is the first again, and not written)
        codes = base + ((size_t)tile * kblocks + warp) * 512 + lane * 16;
        second = (int64_t)(other - tile) * kblocks * 512;
        constexpr int L = G32 ? 4 : 2;        // lanes per tile's scales
        scales = base + a.codes_bytes + (size_t)(lane < L ? tile : other) * a.groups * 32 + (lane % L) * 16;
    }
    __device__ __forceinline__ void issue() { // the next block, if there is one
        if (left > 0) {
            --left;
            const uint32_t dst = ring + in;
            copy16(dst, codes);
            copy16(dst + 512, codes + second);
            if (lane < (G32 ? 8 : 4)) copy16(dst + kCodes, scales + (G32 ? 2u * kb : __umulhi(kb + 1, a.per_magic)) * 32u);   // kb / (blocks per group)
            codes += kWarps * 512;
            kb += kWarps;
            if (kb >= kblocks) { at.next(pairs); seek(); }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        in = in == (STAGES - 1) * kStageBytes ? 0 : in + kStageBytes;
    }
};

// One unit: 32 outputs of one tenant for up to 8 NT rows (s.order[r0 ..]).
template <int NT, bool G32, int STAGES>
__device__ __forceinline__ void unit(const QuantLinearArgs& a, const Shared& s, Stream<G32, STAGES>& st, int& out_stage, float* red, const uint8_t* ring,
                                     int pair, int r0, int rows, int tenant) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int kblocks = a.K / 64;
    const uint16_t* x[NT];                       // (columns behind the last row repeat a row; they are not written)
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n] = a.x + (int64_t)s.order[r0 + min(n * 8 + g, rows - 1)] * a.x_stride + warp * 64 + 8 * t;
    float acc[2][NT][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};

    for (int kb = warp; kb < kblocks; kb += kWarps) {
        uint4 xv[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            xv[n][0] = __ldg(reinterpret_cast<const uint4*>(x[n]));
            xv[n][1] = __ldg(reinterpret_cast<const uint4*>(x[n] + 32));
            x[n] += kWarps * 64;
        }
        __syncwarp();                            // every lane has read the block that the next copy replaces
        st.issue();
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();
        const uint8_t* const block = ring + out_stage;
        out_stage = out_stage == (STAGES - 1) * kStageBytes ? 0 : out_stage + kStageBytes;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 w = *reinterpret_cast<const uint4*>(block + i * 512 + lane * 16);
            float c[NT][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {                // inputs 0..31 and 32..63 of the block
                const uint32_t lo = h == 0 ? w.x : w.y, hi = h == 0 ? w.z : w.w;      // rows g and g + 8
                const uint32_t a00 = centred<0>(lo), a01 = centred<1>(lo), a02 = centred<2>(lo), a03 = centred<3>(lo);
                const uint32_t a10 = centred<0>(hi), a11 = centred<1>(hi), a12 = centred<2>(hi), a13 = centred<3>(hi);
                const uint32_t sc = *reinterpret_cast<const uint32_t*>(block + kCodes + i * (G32 ? 64 : 32) + (G32 && h == 1 ? 32 : 0) + g * 4);
                const float s0 = bf16_lo(sc), s1 = bf16_hi(sc);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 v = xv[n][h];
                    if (h == 0 || G32) mma_bf16(c[n], a00, a10, a01, a11, v.x, v.y, zero);
                    else mma_bf16(c[n], a00, a10, a01, a11, v.x, v.y, c[n]);
                    mma_bf16(c[n], a02, a12, a03, a13, v.z, v.w, c[n]);
                    if (h == 1 || G32) {
                        float (&y)[4] = acc[i][n];
                        y[0] = fmaf(s0, c[n][0], y[0]); y[1] = fmaf(s0, c[n][1], y[1]);
                        y[2] = fmaf(s1, c[n][2], y[2]); y[3] = fmaf(s1, c[n][3], y[3]);
                    }
                }
            }
        }
    }
    // join the warps: red[warp][column][32 outputs, padded to 36]
    __syncthreads();                                       // the unit before this has been read
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float* const r = red + ((warp * NT + n) * 8 + 2 * t) * 36 + 16 * i + g;
            const float (&y)[4] = acc[i][n];
            r[0] = y[0]; r[36] = y[1]; r[8] = y[2]; r[44] = y[3];
        }
    __syncthreads();
    for (int i = tid; i < rows * 32; i += kThreads) {
        const int col = i >> 5, o = i & 31, out = pair * 32 + o;
        if (out >= a.N) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += red[(w * NT * 8 + col) * 36 + o];
        if (a.bias) v += __ldg(a.bias + (size_t)tenant * a.N + out);
        const int64_t at = (int64_t)s.order[r0 + col] * a.y_stride + out;
        if (a.y_fp32) static_cast<float*>(a.y)[at] = v;
        else static_cast<uint16_t*>(a.y)[at] = f_to_bf16(v);
    }
}

// MAXT: largest number of column tiles a pass may take (a launch of n rows never needs more than n of them).
template <int MAXT, bool G32>
__global__ void __launch_bounds__(kThreads, resident(MAXT)) quant_linear_kernel(const QuantLinearArgs a) {
    constexpr int kStages = stages(MAXT);
    __shared__ Shared s;
    extern __shared__ __align__(128) uint8_t s_bytes[];          // the warps' rings, then the join
    uint8_t* const ring = s_bytes + (threadIdx.x / 32) * (kStages * kStageBytes);
    float* const red = reinterpret_cast<float*>(s_bytes + kWarps * kStages * kStageBytes);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31;
    pdl_launch_dependents();
    pdl_wait();
    // --- rows by tenant: slots in order of first appearance, rows of a slot in order of the batch, rows with a bad id last
    const int id = tid < a.n ? a.ids[tid] : -1;
    const bool good = id >= 0 && id < a.tenants;
    s.ids[tid] = good ? id : -1;
    if (tid < a.n && !good && blockIdx.x == 0) raise_status(a.status, MT_ERR_BAD_MODEL_ID, a.row0 + tid);
    __syncthreads();
    int first = tid;
    if (good)
        for (int j = 0; j < tid; ++j)
            if (s.ids[j] == id) { first = j; break; }
    const unsigned firsts = __ballot_sync(0xffffffffu, good && first == tid);
    if (lane == 0) s.warp_n[warp] = __popc(firsts);
    __syncthreads();
    int slot = __popc(firsts & ((1u << lane) - 1u)), n_slots = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) slot += s.warp_n[w];
        n_slots += s.warp_n[w];
    }
    if (good && first == tid) { s.slot[tid] = slot; s.tenant[slot] = id; }
    __syncthreads();
    const int mine = good ? s.slot[first] : n_slots;       // (written by first occurrences only: stable from here on)
    __syncthreads();
    s.slot[tid] = tid < a.n ? mine : 0x7fffffff;
    __syncthreads();
    if (tid < a.n) {
        int at = 0, same = 0;
        for (int j = 0; j < a.n; ++j) {
            const int sj = s.slot[j];
            at += (sj < mine || (sj == mine && j < tid)) ? 1 : 0;
            same += (sj == mine && j < tid) ? 1 : 0;
        }
        s.order[at] = tid;
        if (same == 0) s.begin[mine] = at;
    }
    const int n_valid = __syncthreads_count(good);
    if (tid == 0) s.begin[n_slots] = n_valid;
    __syncthreads();
    if (tid < n_slots) {                                   // groups of at most 64 rows
        int at = 0;
        for (int j = 0; j < tid; ++j) at += (s.begin[j + 1] - s.begin[j] + 63) / 64;
        for (int r = s.begin[tid]; r < s.begin[tid + 1]; r += 64, ++at) { s.group_slot[at] = tid; s.group_row[at] = r; }
        if (tid == n_slots - 1) s.warp_n[0] = at;
    }
    __syncthreads();
    const int n_groups = n_slots > 0 ? s.warp_n[0] : 0;

    for (int i = n_valid; i < a.n; ++i) {                  // rows with a bad id
        const int64_t at = (int64_t)s.order[i] * a.y_stride;
        for (int o = blockIdx.x * kThreads + tid; o < a.N; o += gridDim.x * kThreads) {
            if (a.y_fp32) static_cast<float*>(a.y)[at + o] = nan_f();
            else static_cast<uint16_t*>(a.y)[at + o] = 0x7fff;
        }
    }

    const int pairs = (a.tiles + 1) / 2, kblocks = a.K / 64;
    Cursor at = {0, (int)blockIdx.x};
    while (at.pair >= pairs) { at.pair -= pairs; ++at.group; }
    const int64_t units = (int64_t)pairs * n_groups;
    const int my_units = blockIdx.x < units ? (int)((units - 1 - blockIdx.x) / gridDim.x) + 1 : 0, my_blocks = warp < kblocks ? (kblocks - 1 - warp) / kWarps + 1 : 0;
    Stream<G32, kStages> st{a, s, warp, lane, kblocks, pairs, n_groups, at, 0, my_units * my_blocks, nullptr, nullptr, 0, smem_u32(ring) + lane * 16, 0};
    st.seek();
    for (int i = 0; i < kStages - 1; ++i) st.issue();
    int out_stage = 0;
    for (; at.group < n_groups; at.next(pairs)) {
        const int sl = s.group_slot[at.group], tenant = s.tenant[sl];
        const int r0 = s.group_row[at.group], rows = min(s.begin[sl + 1] - r0, 64);
        if (MAXT == 1 || rows <= 8) unit<1, G32, kStages>(a, s, st, out_stage, red, ring, at.pair, r0, rows, tenant);
        else if (MAXT == 2 || rows <= 16) unit<(MAXT < 2 ? MAXT : 2), G32, kStages>(a, s, st, out_stage, red, ring, at.pair, r0, rows, tenant);
        else if (MAXT == 4 || rows <= 32) unit<(MAXT < 4 ? MAXT : 4), G32, kStages>(a, s, st, out_stage, red, ring, at.pair, r0, rows, tenant);
        else unit<(MAXT < 8 ? MAXT : 8), G32, kStages>(a, s, st, out_stage, red, ring, at.pair, r0, rows, tenant);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

constexpr int shared_bytes(int maxt) { return kWarps * stages(maxt) * kStageBytes + kWarps * maxt * 8 * 36 * 4; }
constexpr bool fits(int maxt) { return resident(maxt) * (shared_bytes(maxt) + (int)sizeof(Shared) + 1024) <= 228 * 1024; }     // 1 KB a CTA is the system's
static_assert(fits(1) && fits(2) && fits(4) && fits(8), "the CTAs that a launch counts on do not fit an SM's shared memory");
typedef void (*Kernel)(QuantLinearArgs);
const Kernel kKernels[2][4] = {
    {quant_linear_kernel<1, false>, quant_linear_kernel<2, false>, quant_linear_kernel<4, false>, quant_linear_kernel<8, false>},
    {quant_linear_kernel<1, true>, quant_linear_kernel<2, true>, quant_linear_kernel<4, true>, quant_linear_kernel<8, true>}};

}  // namespace

cudaError_t configure_quant_linear() {
    for (int g = 0; g < 2; ++g)
        for (int i = 0; i < 4; ++i) {
            const cudaError_t e = cudaFuncSetAttribute(kKernels[g][i], cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes(1 << i));
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

cudaError_t launch_quant_pack(const uint8_t* codes, const uint16_t* scales, int tenants, int K, int N, int group, void* packed,
                              cudaStream_t s) {
    const size_t cb = quant_codes_bytes(K, N), tb = quant_tenant_bytes(K, N, group);
    const size_t items = (cb / 4 + (tb - cb) / 2) * (size_t)tenants;
    const size_t blocks = (items + 255) / 256;
    quant_pack_kernel<<<dim3((unsigned)(blocks < 4736 ? blocks : 4736)), dim3(256), 0, s>>>(codes, scales, tenants, K, N, group, static_cast<uint8_t*>(packed), tb, cb);
    ++g_kernel_launches;
    return cudaGetLastError();
}

cudaError_t launch_quant_linear(const QuantLinearArgs& a, int sm_count, cudaStream_t s) {
    const bool g32 = a.group == 32;
    const int most_slots = a.n < a.tenants ? a.n : a.tenants;
    const int64_t units = (int64_t)((a.N + 31) / 32) * most_slots;      // (more groups only where a tenant has over 64 rows)
    const int v = a.n <= 8 ? 0 : a.n <= 16 ? 1 : a.n <= 32 ? 2 : 3;       // up to 8 << v rows of a tenant
    int64_t grid = (int64_t)sm_count * resident(1 << v);
    if (grid > units) grid = units;
    QuantLinearArgs b = a;
    b.codes_bytes = quant_codes_bytes(a.K, a.N);
    b.tenant_bytes = quant_tenant_bytes(a.K, a.N, a.group);
    b.groups = a.K / a.group;
    b.tiles = (a.N + 15) / 16;
    b.per_magic = 0xffffffffu / (g32 ? 1u : (uint32_t)a.group / 64u);
    return launch_pdl(kKernels[g32][v], dim3((unsigned)grid), dim3(kThreads), (size_t)shared_bytes(1 << v), s, b);
}

}  // namespace mt

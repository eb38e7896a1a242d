// Rotary positions with one to four axes.
//
// Mathematics.  Pair c of a head turns by a = position[axis(c)] * frequency[c]: (x, y) -> (x cos a - y sin a, x sin a + y cos a).  A far position's
// angle is thousands of turns, of which fp32 would keep little, so a / 2 pi is formed in 64 bits and cut to its fraction of a turn; sine and
// cosine of that are fp32.  (The fraction keeps 24 bits, 2^-26 of a turn at worst: that moves a sine or cosine by up to 9e-8, where its rounding alone is 3e-8.)
//
// Split.  A CTA takes the tokens whose tables of sines and cosines fill its threads once (one angle a thread), so an angle is computed once for all
// heads; then a thread takes eight pairs of a head at a time, 16 bytes of either member in bf16.
//
// Cost.  Bytes: 8191 tokens of 40 heads of 128 in bf16 take 29 us, 5.8 TB/s of reads and writes; 64 tokens 4.6 us of latency (positions, sines, a
// barrier), below the host's time for the call.
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 16;                // of a CTA: tables of 16 tokens of 16 pairs

struct Params {
    RotateArgs a;
    int half, units;                          // pairs of a head, groups of eight of them
    int bound[3];                             // first pair of axes 1 to 3
    int tokens;                               // of a CTA
    int rest;                                 // groups of eight elements that are copied as they are
    float sign;
};

template <bool FP32> struct Eight;
template <> struct Eight<false> {
    uint4 v;
    __device__ __forceinline__ void load(const void* p, int64_t at) { v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at); }
    __device__ __forceinline__ void store(void* p, int64_t at) const { *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = v; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
        f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        v.x = pack_bf16x2(f[0], f[1]); v.y = pack_bf16x2(f[2], f[3]); v.z = pack_bf16x2(f[4], f[5]); v.w = pack_bf16x2(f[6], f[7]);
    }
};
template <> struct Eight<true> {
    float4 a, b;
    __device__ __forceinline__ void load(const void* p, int64_t at) {
        const float4* const q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        a = q[0]; b = q[1];
    }
    __device__ __forceinline__ void store(void* p, int64_t at) const {
        float4* const q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
        q[0] = a; q[1] = b;
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&f)[8]) { a = make_float4(f[0], f[1], f[2], f[3]); b = make_float4(f[4], f[5], f[6], f[7]); }
};

template <bool FP32, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads, 5) rotate_kernel(const Params p) {
    extern __shared__ float table[];          // [tokens][half] cosines, then sines
    const RotateArgs& a = p.a;
    const int t0 = blockIdx.x * p.tokens, n = min(p.tokens, a.n - t0);
    float* const cosines = table;
    float* const sines = table + p.tokens * p.half;
    const int threads = blockDim.x * blockDim.y, me = threadIdx.y * blockDim.x + threadIdx.x;
    const int u = threadIdx.x;
    const int first = NEIGHBOURS ? 16 * u : 8 * u, second = NEIGHBOURS ? 16 * u + 8 : p.half + 8 * u;
    int t = 0, h = threadIdx.y;
    auto step = [&]() { while (h >= a.heads && t < n) { h -= a.heads; ++t; } };
    auto load = [&](Eight<FP32>& vx, Eight<FP32>& vy) {
        if (t >= n) return;
        const int64_t from = (int64_t)(t0 + t) * a.x_token_stride + (int64_t)h * a.x_head_stride;
        vx.load(a.x, from + first);
        vy.load(a.x, from + second);
    };
    pdl_launch_dependents();
    pdl_wait();
    Eight<FP32> vx, vy;                       // the first are under way while the tables are made, each next one while one is turned
    step();
    load(vx, vy);
    for (int i = me; i < n * p.half; i += threads) {
        const int t = i / p.half, c = i - t * p.half;
        const int axis = (c >= p.bound[0]) + (c >= p.bound[1]) + (c >= p.bound[2]);
        const double turns = (double)a.positions[(int64_t)(t0 + t) * a.axes + axis] * ((double)a.frequencies[c] * 0.15915494309189533577);
        float s, co;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
        cosines[i] = co;
        sines[i] = s * p.sign;
    }
    __syncthreads();
    while (t < n) {
        const int64_t to = (int64_t)(t0 + t) * a.out_token_stride + (int64_t)h * a.out_head_stride;
        float c[8], s[8], x[8], y[8];
        const float4* const ct = reinterpret_cast<const float4*>(cosines + t * p.half + 8 * u);
        const float4* const st = reinterpret_cast<const float4*>(sines + t * p.half + 8 * u);
        const float4 c0 = ct[0], c1 = ct[1], s0 = st[0], s1 = st[1];
        c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
        s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
        vx.get(x);
        vy.get(y);
        h += blockDim.y;
        step();
        load(vx, vy);
        if (NEIGHBOURS) {                     // x[0], x[1] are pair 0, ..; y[0], y[1] pair 4
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float xa = x[2 * e], xb = x[2 * e + 1], ya = y[2 * e], yb = y[2 * e + 1];
                x[2 * e] = xa * c[e] - xb * s[e];
                x[2 * e + 1] = xa * s[e] + xb * c[e];
                y[2 * e] = ya * c[e + 4] - yb * s[e + 4];
                y[2 * e + 1] = ya * s[e + 4] + yb * c[e + 4];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xa = x[e], ya = y[e];
                x[e] = xa * c[e] - ya * s[e];
                y[e] = xa * s[e] + ya * c[e];
            }
        }
        Eight<FP32> out;
        out.set(x);
        out.store(a.out, to + first);
        out.set(y);
        out.store(a.out, to + second);
    }
    // what is not turned
    if (p.rest > 0) {
        const int per_token = a.heads * p.rest;
        for (int i = me; i < n * per_token; i += threads) {
            const int tok = i / per_token, j = i - tok * per_token, head = j / p.rest, r = j - head * p.rest;
            Eight<FP32> v;
            v.load(a.x, (int64_t)(t0 + tok) * a.x_token_stride + (int64_t)head * a.x_head_stride + 2 * p.half + 8 * r);
            v.store(a.out, (int64_t)(t0 + tok) * a.out_token_stride + (int64_t)head * a.out_head_stride + 2 * p.half + 8 * r);
        }
    }
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs& a, cudaStream_t s) {
    Params p;
    p.a = a;
    p.half = a.rotary_dim / 2;
    p.units = p.half / 8;
    int at = 0;
    for (int i = 0; i < 3; ++i) { at += a.sections[i]; p.bound[i] = i + 1 < a.axes ? at : p.half; }
    p.tokens = kThreads / p.half;
    if (p.tokens < 1) p.tokens = 1;
    if (p.tokens > kMaxTokens) p.tokens = kMaxTokens;
    p.sign = a.inverse ? -1.f : 1.f;
    const bool in_place = a.x == a.out && a.x_token_stride == a.out_token_stride && a.x_head_stride == a.out_head_stride;
    p.rest = in_place ? 0 : (a.head_dim - a.rotary_dim) / 8;
    const dim3 block(p.units, kThreads / p.units), grid((a.n - 1) / p.tokens + 1);
    const size_t smem = (size_t)p.tokens * p.half * 8;
    if (a.fp32) return a.neighbours ? launch_pdl(rotate_kernel<true, true>, grid, block, smem, s, p) : launch_pdl(rotate_kernel<true, false>, grid, block, smem, s, p);
    return a.neighbours ? launch_pdl(rotate_kernel<false, true>, grid, block, smem, s, p) : launch_pdl(rotate_kernel<false, false>, grid, block, smem, s, p);
}

}  // namespace mt

// w4.hip -- products with 4-bit weights and group scales (qlm_w4_pack,
// qlm_w4_matmul; the definition stands in include/qlm.h).
//
// A code c becomes the number 16 + c by placing its four bits at the top of a
// mantissa under the exponent of 16 (exact in half precision and bfloat16, one
// shift and one and-or for two codes).  No weight is ever rounded:
//  - up to 16 rows, with one group's sums S = sum of x, T[n] = sum of (16 + c[n]) x,
//    both by the matrix instructions (S with a matrix of ones), the group's part of
//    the output is s[n] (T[n] - (16 + z[n]) S), formed in single precision: T is up to some six
//    times the sum of |c - z| |x|, whose bits the difference loses.  Of bfloat16 all is held
//    times 2^-kDown, by the constants' exponents, and the output raised again: a T
//    of x from 2^116 on would pass single precision's range.  What the smallest numbers lose
//    by that, 2^-138 an addition, is below the least bfloat16 (2^-133);
//  - for more rows 16 + z is taken off in half precision (exact: -15 .. 15), once for
//    all of them, and the part is s[n] T[n].  Rows of bfloat16 are first scaled by
//    powers of two to fit halves.
// An x that is not finite makes its row's outputs not finite.
//
// Packed: for each 16 outputs and each 128 inputs one chunk of 1024 bytes of
// codes in the order of the matrix operand (lane l of 64: output l % 16, and for
// step j of four the dword j with inputs 32 j + 8 (l / 16) + e, e = 0..7 at the
// bits 4 (e / 2) of half e % 2), then for each of its groups 16 words
// {scale, 16 + zero} in half precision.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "internal.h"
#include "qlm.h"
#include "w4_split.h"

namespace {

using qlm_internal::fail;
using qlm_internal::hip_fail;

typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

using qlm_w4_host::kStep;            // inputs of a chunk
using qlm_w4_host::split_of;
constexpr int kWaves = 4, kThreads = 64 * kWaves;

__host__ __device__ inline int chunk_bytes(int group) { return 1024 + 64 * (kStep / group); }

struct PackArgs {
    int32_t N, K, group, tiles, steps;
    const uint8_t *codes, *zero;
    const uint16_t *scale;
    uint8_t *packed;
};

// One workgroup for each chunk, a lane for each 16 bytes of codes.  Done once for a matrix:
// 20001 x 8192 in groups of 32 (164 MB of codes, 82 packed and 21 of groups) 90 us, 3 TB/s.
__global__ __launch_bounds__(64) void k_w4_pack(PackArgs a)
{
    const int l = threadIdx.x;
    const int kb = blockIdx.x % a.steps, tile = blockIdx.x / a.steps;
    uint8_t *chunk = a.packed + (int64_t)blockIdx.x * chunk_bytes(a.group);
    const int n = tile * 16 + l % 16;
    uint32_t w[4] = {0, 0, 0, 0};
    const bool wide = a.K % 8 == 0 && (uintptr_t)a.codes % 8 == 0;
    for (int j = 0; j < 4; ++j) {
        const int k = kb * kStep + j * 32 + (l / 16) * 8;
        const uint8_t *p = a.codes + (int64_t)n * a.K + k;
        uint8_t c[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (n < a.N && wide && k < a.K) {
            const uint2 x = *(const uint2 *)p;
            for (int e = 0; e < 8; ++e) c[e] = (uint8_t)((e < 4 ? x.x : x.y) >> (8 * (e & 3)));
        } else if (n < a.N) {
            for (int e = 0; e < 8; ++e)
                if (k + e < a.K) c[e] = p[e];
        }
        for (int e = 0; e < 8; ++e)
            w[j] |= (uint32_t)(c[e] & 15u) << (16 * (e & 1) + 4 * (e >> 1));
    }
    *(uint4 *)(chunk + 16 * l) = uint4{w[0], w[1], w[2], w[3]};
    const int per = kStep / a.group, groups = (a.K + a.group - 1) / a.group;
    for (int i = l; i < per * 16; i += 64) {
        const int gi = kb * per + i / 16, r = tile * 16 + i % 16;
        uint32_t s = 0, z = 0;
        if (r < a.N && gi < groups) {
            s = a.scale[(int64_t)r * groups + gi];
            z = a.zero ? a.zero[(int64_t)r * groups + gi] & 15u : 8u;
        }
        const uint32_t zh = __builtin_bit_cast(uint16_t, (_Float16)(float)(16 + z));
        *(uint32_t *)(chunk + 1024 + 4 * i) = s | zh << 16;
    }
}

template <bool BF> __device__ inline float4v mfma(uint4 x, uint4 y, float4v c)
{
    if (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, x),
                                                       __builtin_bit_cast(bf8v, y), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, x),
                                                  __builtin_bit_cast(half8v, y), c, 0, 0, 0);
}

// 31 GROUP 2^-kDown < 1: the sum of a group's (16 + c) x is finite with every x.
template <bool BF, int GROUP> constexpr int kDown = !BF ? 0 : GROUP == 32 ? 10 : GROUP == 64 ? 11 : 12;

// The exponent of 16 * 2^-kDown for two numbers, in a register (an and-or takes one constant
// from the scalar side only).
template <bool BF, int GROUP> __device__ inline uint32_t sixteen()
{
    uint32_t c = BF ? (127 + 4 - kDown<BF, GROUP>) * 0x00800080u : 0x4c004c00u;
    asm("" : "+v"(c));
    return c;
}

// The eight codes of a dword as 16 + c (times 2^-kDown).
template <bool BF> __device__ inline uint4 operand(uint32_t w, uint32_t c)
{
    if (BF)
        return {(w << 3 & 0x00780078u) | c, (w >> 1 & 0x00780078u) | c,
                (w >> 5 & 0x00780078u) | c, (w >> 9 & 0x00780078u) | c};
    return {(w << 6 & 0x03c003c0u) | c, (w << 2 & 0x03c003c0u) | c,
            (w >> 2 & 0x03c003c0u) | c, (w >> 6 & 0x03c003c0u) | c};
}

// Ones (times 2^-kDown).
template <bool BF, int GROUP> __device__ inline uint4 ones()
{
    const uint32_t o = BF ? (127 - kDown<BF, GROUP>) * 0x00800080u : 0x3c003c00u;
    return {o, o, o, o};
}

// sum += scale (t - zero S) for the four outputs of a lane
__device__ inline float4v add_group(float4v sum, float4v t, float S, uint4 meta)
{
    const uint32_t w[4] = {meta.x, meta.y, meta.z, meta.w};
    for (int i = 0; i < 4; ++i) {
        const half2v h = __builtin_bit_cast(half2v, w[i]);
        sum[i] = fmaf((float)h[0], fmaf(-(float)h[1], S, t[i]), sum[i]);
    }
    return sum;
}

__device__ inline uint16_t out_bits(float v, bool bf)
{
    if (bf) return __builtin_bit_cast(uint16_t, (__bf16)v);
    return __builtin_bit_cast(uint16_t, (_Float16)v);
}

struct MatArgs {
    const uint8_t *packed;
    const uint16_t *x;
    uint16_t *out;
    int64_t x_stride, out_stride;
    int32_t N, K, M, tiles, steps;
    int32_t wide;                    // x may be read 16 bytes at a time
    int32_t bf;                      // out is bfloat16 (k_w4_wide)
    const float *fac;                // [M] what takes the rows' scaling out, or NULL
    int32_t per_stage;               // thin: steps of x held at once (a multiple of kWaves)
    int32_t splits, per_split;       // wide form: splits of K, steps of one
    float *part;                     // [split][M][N]
};

// Eight inputs of a row from k on, zero past the last.
__device__ inline uint4 x8(const MatArgs &a, int row, int k)
{
    const uint16_t *p = a.x + row * a.x_stride + k;
    if (a.wide && k + 8 <= a.K) return *(const uint4 *)p;
    uint32_t w[4];
    for (int e = 0; e < 4; ++e) {
        const uint32_t lo = k + 2 * e < a.K ? p[2 * e] : 0u;
        const uint32_t hi = k + 2 * e + 1 < a.K ? p[2 * e + 1] : 0u;
        w[e] = lo | hi << 16;
    }
    return {w[0], w[1], w[2], w[3]};
}

// Up to 16 rows: one workgroup to 16 outputs, its waves taking the steps of K
// in turn, four steps' weights under way; x in shared memory.  The sum of a group's x,
// for its zero point, is a matrix product with ones.
// 1 row, 4096 x 4096: 5.9 us (8.9 MB, 1.5 TB/s), the launch and one round of loads.
template <bool BF, int GROUP> __global__ __launch_bounds__(kThreads) void k_w4_thin(MatArgs a)
{
    constexpr int PER = kStep / GROUP, SUB = 4 / PER, PF = 4;
    extern __shared__ uint4 lds[];
    uint16_t *xs = (uint16_t *)lds;
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, c16 = lane & 15;
    const int tile = blockIdx.x;
    const int cb = chunk_bytes(GROUP);
    const uint8_t *base = a.packed + (int64_t)tile * a.steps * cb;
    const int ld = a.per_stage * kStep + 8;      // elements of a row in shared memory
    const int mine = c16 < a.M ? c16 : 0;
    const uint32_t c16f = sixteen<BF, GROUP>();
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    uint4 cw[PF], mw[PF][PER];
    auto fetch = [&](int u, int kb) {
        if (kb < a.steps) {
            const uint8_t *p = base + (int64_t)kb * cb;
            cw[u] = *(const uint4 *)(p + 16u * lane);
            for (int q = 0; q < PER; ++q) mw[u][q] = *(const uint4 *)(p + 1024 + 64 * q + 16u * g);
        }
    };
    for (int u = 0; u < PF; ++u) fetch(u, wv + u * kWaves);
    // round r: the waves' steps kWaves r + wv; the ring holds the next PF rounds
    const int rounds = (a.steps + kWaves - 1) / kWaves, per = a.per_stage / kWaves;
    int in_stage = per;
    for (int r0 = 0; r0 < rounds; r0 += PF) {
        for (int u = 0; u < PF && r0 + u < rounds; ++u) {
            const int r = r0 + u;
            if (in_stage == per) {
                in_stage = 0;
                const int k0 = r * kWaves, n8 = min(a.per_stage, a.steps - k0) * (kStep / 8);
                if (r) __syncthreads();
                for (int e = threadIdx.x; e < a.M * n8; e += kThreads) {
                    const int m = e / n8, k = 8 * (e % n8);
                    *(uint4 *)(xs + m * ld + k) = x8(a, m, k0 * kStep + k);
                }
                __syncthreads();
            }
            const int kb = r * kWaves + wv;
            if (kb < a.steps) {
                const uint16_t *xp = xs + mine * ld + (in_stage * kWaves + wv) * kStep + 8 * g;
                const uint32_t w[4] = {cw[u].x, cw[u].y, cw[u].z, cw[u].w};
                for (int q = 0; q < PER; ++q) {
                    float4v t = {0.f, 0.f, 0.f, 0.f}, S = {0.f, 0.f, 0.f, 0.f};
                    for (int j = q * SUB; j < (q + 1) * SUB; ++j) {
                        const uint4 b = *(const uint4 *)(xp + 32 * j);
                        t = mfma<BF>(operand<BF>(w[j], c16f), b, t);
                        S = mfma<BF>(ones<BF, GROUP>(), b, S);
                    }
                    sum = add_group(sum, t, S[0], mw[u][q]);
                }
                fetch(u, kb + kWaves * PF);
            }
            ++in_stage;
        }
    }
    // the waves' parts: lane holds outputs 4 g + i of row c16
    __syncthreads();
    float *red = (float *)lds;
    for (int i = 0; i < 4; ++i) red[wv * 256 + c16 * 16 + 4 * g + i] = sum[i];
    __syncthreads();
    float v = 0.f;
    for (int w = 0; w < kWaves; ++w) v += red[w * 256 + threadIdx.x];
    const int m = threadIdx.x >> 4, n = tile * 16 + (threadIdx.x & 15);
    if (m < a.M && n < a.N) a.out[m * a.out_stride + n] = out_bits(v * (1 << kDown<BF, GROUP>), BF);
}

// Rows for k_w4_wide: halves, 16-byte aligned, zeros up to a whole number of stages.
// Rows of bfloat16 are scaled by a power of two to below 2^15: code less zero point is formed
// in halves by one instruction for two, and both forms of x then share the kernel.  Elements
// below 2^-29 of the row's largest lose bits.  A workgroup to a
// row, eight inputs to a thread: a row is read in few rounds, as latency is all it costs.
constexpr int kHalfThreads = 1024;

__global__ __launch_bounds__(kHalfThreads) void k_w4_half(MatArgs a, uint16_t *xh, float *fac,
                                                          int ld)
{
    __shared__ uint32_t part[kHalfThreads / 64];
    uint32_t top = 0;                       // greatest exponent of a finite element
    for (int k = 8 * threadIdx.x; k < a.K && a.bf; k += 8 * kHalfThreads) {
        const uint4 v = x8(a, blockIdx.x, k);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        for (int e = 0; e < 8; ++e) {
            const uint32_t x = w[e >> 1] >> (16 * (e & 1) + 7) & 0xff;
            top = x < 255 ? max(top, x) : top;
        }
    }
    for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int w = 0; w < kHalfThreads / 64; ++w) top = max(top, part[w]);
    const int up = min(15 - ((int)top - 126), 126);
    const float by = ldexpf(1.f, up);
    for (int k = 8 * threadIdx.x; k < ld; k += 8 * kHalfThreads) {
        uint4 v = {0u, 0u, 0u, 0u};
        if (k < a.K) v = x8(a, blockIdx.x, k);
        if (a.bf) {
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
            for (int e = 0; e < 4; ++e) {
                const float lo = __builtin_bit_cast(float, w[e] << 16);
                const float hi = __builtin_bit_cast(float, w[e] & 0xffff0000u);
                w[e] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)(lo * by)) |
                       (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)(hi * by)) << 16;
            }
            v = {w[0], w[1], w[2], w[3]};
        }
        *(uint4 *)(xh + (int64_t)blockIdx.x * ld + k) = v;
    }
    if (threadIdx.x == 0) fac[blockIdx.x] = a.bf ? ldexpf(1.f, -up) : 1.f;
}

__device__ inline uint16_t wide_out(const MatArgs &a, float v, int m)
{
    return out_bits(a.fac ? v * a.fac[m] : v, a.bf);
}

// More rows: one workgroup to 64 outputs (16 a wave) and 16 NT rows of halves; x
// passes through shared memory two steps at a time, in two buffers; the weights of
// the two steps after the present ones are on their way.  The zero point is taken off
// the codes (exact in halves), so a group costs one product and one fma an output.
// 48 rows, 20001 x 8192 in groups of 32: 60 us (262 TFLOP/s; 98 MB, 1.6 TB/s).  It waits
// on the chain from codes to operands to products at 2.4 waves to a SIMD: without its
// reads of memory it takes 43 us, and no pipe is full.  A prompt's rows, 2000 through
// 4096 x 11008 in groups of 128: 316 us, 571 TFLOP/s, where the library's product of 16-bit
// weights takes 155: every 64 rows turn the codes into operands again.
template <int GROUP, int NT> __global__ __launch_bounds__(kThreads, 2) void k_w4_wide(MatArgs a)
{
    constexpr int PER = kStep / GROUP, SUB = 4 / PER, LD = 2 * kStep + 8;
    __shared__ uint4 lds[2][NT * 16 * LD / 8];
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, c16 = lane & 15;
    const int tile = blockIdx.x * kWaves + wv, m0 = blockIdx.y * NT * 16, sp = blockIdx.z;
    const int k0 = sp * a.per_split, k1 = min(a.steps, k0 + a.per_split);
    const int cb = chunk_bytes(GROUP);
    const bool mine = tile < a.tiles;
    const uint8_t *base = a.packed + (int64_t)(mine ? tile : 0) * a.steps * cb;
    const uint32_t c16f = sixteen<false, GROUP>();
    float4v sum[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[t] = float4v{0.f, 0.f, 0.f, 0.f};
    uint4 cw[2], mw[2][PER];
    uint4v xr[2 * NT];
    uint16_t zw[2][PER];
    auto fetch_w = [&](int u, int kb) {          // (past the last step it is read again)
        const uint8_t *p = base + (int64_t)min(kb, k1 - 1) * cb;
        cw[u] = *(const uint4 *)(p + 16u * lane);
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            mw[u][q] = *(const uint4 *)(p + 1024 + 64 * q + 16u * g);
            zw[u][q] = *(const uint16_t *)(p + 1024 + 64 * q + 2 + 4u * c16);
        }
    };
    // thread t stages row t / 16 of each 16 rows, inputs 8 (t % 16) on of each step;
    // rows past the last are the last again (their outputs are not written)
    const int sr = threadIdx.x >> 4, sk = 8 * (threadIdx.x & 15);
    // (no branch: the waits for the weights would count loads that may not be there.  Both
    // steps of a pair are read: splits begin at whole pairs, and rows hold whole pairs)
    const uint16_t *xp[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
        xp[t] = a.x + (int64_t)min(m0 + t * 16 + sr, a.M - 1) * a.x_stride + sk;
    auto fetch_x = [&](int kb) {
#pragma unroll
        for (int t = 0; t < 2 * NT; ++t)
            xr[t] = *(const uint4v *)(xp[t >> 1] + kb * kStep + (t & 1) * kStep);
    };
    auto stage = [&](int buf) {
        uint16_t *xs = (uint16_t *)lds[buf];
#pragma unroll
        for (int t = 0; t < 2 * NT; ++t)
            *(uint4v *)(xs + ((t >> 1) * 16 + sr) * LD + (t & 1) * kStep + sk) = xr[t];
    };
    if (k0 < k1) {
        fetch_x(k0);
        fetch_w(0, k0);
        fetch_w(1, k0 + 1);
        stage(0);
    }
    __syncthreads();
    for (int kb = k0; kb < k1; kb += 2) {
        const int buf = ((kb - k0) >> 1) & 1;
        fetch_x(kb + 2 < k1 ? kb + 2 : kb);
        const uint16_t *xs = (const uint16_t *)lds[buf];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t w[4] = {cw[u].x, cw[u].y, cw[u].z, cw[u].w};
            // (past the last step: x is zeros, and scales of 0, as they may be infinite)
            const uint32_t on = kb + u < k1 ? 0xffffu : 0u;
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const half2v z = __builtin_bit_cast(half2v, (uint32_t)zw[u][q] * 0x10001u);
                float4v t[NT];
#pragma unroll
                for (int k = 0; k < NT; ++k) t[k] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = q * SUB; j < (q + 1) * SUB; ++j) {
                    uint4 o = operand<false>(w[j], c16f);
                    o.x = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, o.x) - z);
                    o.y = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, o.y) - z);
                    o.z = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, o.z) - z);
                    o.w = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, o.w) - z);
#pragma unroll
                    for (int k = 0; k < NT; ++k) {
                        const uint4 b = *(const uint4 *)(xs + (k * 16 + c16) * LD + u * kStep +
                                                         32 * j + 8 * g);
                        t[k] = mfma<false>(o, b, t[k]);
                    }
                }
                const uint32_t m[4] = {mw[u][q].x & on, mw[u][q].y & on, mw[u][q].z & on,
                                       mw[u][q].w & on};
#pragma unroll
                for (int k = 0; k < NT; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sum[k][i] = fmaf((float)__builtin_bit_cast(half2v, m[i])[0], t[k][i],
                                         sum[k][i]);
            }
            fetch_w(u, kb + u + 2);
        }
        stage(buf ^ 1);
        __syncthreads();
    }
    if (!mine) return;
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        const int m = m0 + k * 16 + c16;
        if (m >= a.M) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = tile * 16 + 4 * g + i;
            if (n >= a.N) continue;
            if (a.splits > 1)
                a.part[((int64_t)sp * a.M + m) * a.N + n] = sum[k][i];
            else
                a.out[m * a.out_stride + n] = wide_out(a, sum[k][i], m);
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_w4_join(MatArgs a)
{
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t all = (int64_t)a.M * a.N;
    if (e >= all) return;
    float v = 0.f;
    for (int s = 0; s < a.splits; ++s) v += a.part[s * all + e];
    const int m = (int)(e / a.N), n = (int)(e % a.N);
    a.out[m * a.out_stride + n] = wide_out(a, v, m);
}

// -- host -------------------------------------------------------------------

int check_weight(const qlm_w4 *w)
{
    if (!w) return fail(QLM_ERR_ARG, "weight is NULL");
    if (w->n_out < 1 || w->n_in < 1 || w->n_out > (1 << 24) || w->n_in > (1 << 24))
        return fail(QLM_ERR_ARG, "n_out and n_in must be in 1..16777216");
    if (w->group != 32 && w->group != 64 && w->group != 128)
        return fail(QLM_ERR_ARG, "group must be 32, 64 or 128");
    if (!w->packed || (uintptr_t)w->packed % 256)
        return fail(QLM_ERR_ARG, "packed must be non-NULL and 256-byte aligned");
    return QLM_OK;
}

// k_w4_thin reads x again for every 16 outputs, k_w4_wide for every 64, but it has
// parts to join and, where x is not aligned halves in whole stages, x to convert.
// So up to 16 rows the product of rows, tiles of outputs and steps decides (us, halves
// and bfloat16, thin against wide): 12 rows, 4096 x 4096 11.4 to 10.2 and 11.5 to
// 13.0; 4 rows, 11000 x 4096 11.2 to 13.9 and 10.9 to 16.5, 8 rows 18.1 to 14.1 and
// 18.0 to 16.7; 20001 x 8192 1 row 26.5 to 31.5 and 23.5 to 32.2, 2 rows 34.0 to 31.4
// and 31.8 to 32.5, 16 rows 67.9 to 30.4 and 68.6 to 34.4.
constexpr int kThinRows = 16, kThinWork = 96000, kThinWorkConvert = 160000;

bool thin(const qlm_w4 *w, int rows, bool convert)
{
    const int64_t work = (int64_t)rows * ((w->n_out + 15) / 16) * ((w->n_in + kStep - 1) / kStep);
    return rows <= kThinRows && work <= (convert ? kThinWorkConvert : kThinWork);
}

template <bool BF, int GROUP> void launch_thin(MatArgs a, hipStream_t st)
{
    // as much of x as 64 KiB hold
    const int most = (65536 / a.M - 16) / (2 * kStep) / kWaves * kWaves;
    a.per_stage = std::min(most, (a.steps + kWaves - 1) / kWaves * kWaves);
    const int bytes = std::max(a.M * (a.per_stage * kStep + 8) * 2, kWaves * 1024);
    k_w4_thin<BF, GROUP><<<a.tiles, kThreads, bytes, st>>>(a);
}

template <int GROUP> void launch(const MatArgs &a, bool few, hipStream_t st)
{
    if (few) {
        if (a.bf)
            launch_thin<true, GROUP>(a, st);
        else
            launch_thin<false, GROUP>(a, st);
        return;
    }
    const int nt = std::min(4, (a.M + 15) / 16);
    const dim3 grid((a.tiles + kWaves - 1) / kWaves, (a.M + 16 * nt - 1) / (16 * nt), a.splits);
    if (nt == 1)
        k_w4_wide<GROUP, 1><<<grid, kThreads, 0, st>>>(a);
    else if (nt == 2)
        k_w4_wide<GROUP, 2><<<grid, kThreads, 0, st>>>(a);
    else if (nt == 3)
        k_w4_wide<GROUP, 3><<<grid, kThreads, 0, st>>>(a);
    else
        k_w4_wide<GROUP, 4><<<grid, kThreads, 0, st>>>(a);
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Workspace of the form for more rows: parts of the splits, then halves of x.
struct Layout {
    size_t xh, fac, total;
    int ld;
};

Layout layout_of(const qlm_w4 *w, int rows)
{
    Layout l{};
    if (thin(w, rows, false)) return l;          // (and so where x is converted)
    int splits, per;
    split_of(w->n_out, w->n_in, rows, &splits, &per);
    l.ld = (w->n_in + 2 * kStep - 1) / (2 * kStep) * 2 * kStep;
    l.xh = splits > 1 ? align256((size_t)splits * rows * w->n_out * 4) : 0;
    l.fac = l.xh + align256((size_t)rows * l.ld * 2);
    l.total = l.fac + align256((size_t)rows * 4);
    return l;
}

}  // namespace

extern "C" {

size_t qlm_w4_packed_bytes(int32_t n_out, int32_t n_in, int32_t group)
{
    if (n_out < 1 || n_in < 1 || n_out > (1 << 24) || n_in > (1 << 24) ||
        (group != 32 && group != 64 && group != 128))
        return 0;
    return ((size_t)n_out + 15) / 16 * (((size_t)n_in + kStep - 1) / kStep) * chunk_bytes(group);
}

int qlm_w4_pack(const qlm_w4 *weight, const uint8_t *codes, const void *scale,
                const uint8_t *zero, qlm_stream stream_)
{
    int rc = check_weight(weight);
    if (rc) return rc;
    if (!codes || !scale) return fail(QLM_ERR_ARG, "codes and scale are required");
    PackArgs a{};
    a.N = weight->n_out;
    a.K = weight->n_in;
    a.group = weight->group;
    a.tiles = (a.N + 15) / 16;
    a.steps = (a.K + kStep - 1) / kStep;
    a.codes = codes;
    a.zero = zero;
    a.scale = (const uint16_t *)scale;
    a.packed = (uint8_t *)weight->packed;
    const int64_t grid = (int64_t)a.tiles * a.steps;
    // (a launch holds fewer than 2^32 threads)
    if (grid >= (1ll << 32) / 64) return fail(QLM_ERR_CAPACITY, "the matrix is too large");
    k_w4_pack<<<(unsigned)grid, 64, 0, (hipStream_t)stream_>>>(a);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_w4_pack launch");
}

size_t qlm_w4_workspace_bytes(const qlm_w4 *weight, int32_t n_rows)
{
    if (!weight || n_rows < 1 || weight->n_out < 1 || weight->n_in < 1) return 0;
    return layout_of(weight, n_rows).total;
}

int qlm_w4_matmul(const qlm_w4 *weight, const void *x, int64_t x_stride, void *out,
                  int64_t out_stride, int32_t n_rows, int32_t dtype, void *ws, size_t ws_bytes,
                  qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    int rc = check_weight(weight);
    if (rc) return rc;
    if (n_rows < 0 || n_rows > (1 << 20)) return fail(QLM_ERR_ARG, "n_rows must be in 0..1048576");
    if (dtype != QLM_F16 && dtype != QLM_BF16)
        return fail(QLM_ERR_ARG, "dtype must be QLM_F16 or QLM_BF16");
    if (n_rows == 0) return QLM_OK;
    if (!x || !out) return fail(QLM_ERR_ARG, "x and out are required");
    if ((uintptr_t)x % 2 || (uintptr_t)out % 2) return fail(QLM_ERR_ARG, "x or out is misaligned");
    if (x == out) return fail(QLM_ERR_ARG, "out may not alias x");
    if (x_stride < weight->n_in || out_stride < weight->n_out)
        return fail(QLM_ERR_ARG, "x_stride and out_stride must be >= the row's length");
    if (((int64_t)n_rows * weight->n_out + kThreads - 1) / kThreads > INT32_MAX)
        return fail(QLM_ERR_CAPACITY, "too many outputs in one call");
    const size_t need = qlm_w4_workspace_bytes(weight, n_rows);
    if (need && (!ws || (uintptr_t)ws % 256))
        return fail(QLM_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
    if (ws_bytes < need) return fail(QLM_ERR_WORKSPACE, "workspace too small");
    MatArgs a{};
    a.packed = (const uint8_t *)weight->packed;
    a.x = (const uint16_t *)x;
    a.out = (uint16_t *)out;
    a.x_stride = x_stride;
    a.out_stride = out_stride;
    a.N = weight->n_out;
    a.K = weight->n_in;
    a.M = n_rows;
    a.tiles = (a.N + 15) / 16;
    a.steps = (a.K + kStep - 1) / kStep;
    a.wide = (uintptr_t)x % 16 == 0 && x_stride % 8 == 0;
    a.bf = dtype == QLM_BF16;
    a.part = (float *)ws;
    a.splits = 1;
    hipError_t e;
    // (halves that are aligned and fill whole stages are read where they are)
    const bool convert = a.bf || !a.wide || a.K % (2 * kStep);
    const bool few = thin(weight, n_rows, convert);
    if (!few) split_of(weight->n_out, weight->n_in, n_rows, &a.splits, &a.per_split);
    if (!few && convert) {
        const Layout l = layout_of(weight, n_rows);
        uint16_t *xh = (uint16_t *)((char *)ws + l.xh);
        float *fac = (float *)((char *)ws + l.fac);
        k_w4_half<<<n_rows, kHalfThreads, 0, stream>>>(a, xh, fac, l.ld);
        if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_w4_half launch");
        a.x = xh;
        a.x_stride = l.ld;
        a.fac = a.bf ? fac : nullptr;
    }
    if (weight->group == 32)
        launch<32>(a, few, stream);
    else if (weight->group == 64)
        launch<64>(a, few, stream);
    else
        launch<128>(a, few, stream);
    if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "w4 launch");
    if (a.splits > 1) {
        const int64_t grid = ((int64_t)a.M * a.N + kThreads - 1) / kThreads;
        k_w4_join<<<(unsigned)grid, kThreads, 0, stream>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_w4_join launch");
    }
    return QLM_OK;
}

}  // extern "C"

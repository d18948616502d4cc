// kv_attention.hip -- attention over the 8-bit token cache
// (qlm_kv_attention; the definition stands in include/qlm.h).
#include "kv.h"

#include <algorithm>
#include <string>

namespace {

using namespace qlm_kv;
using qlm_internal::fail;
using qlm_internal::hip_fail;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896340736f;
// p is held as 2^(s - m + kRaise): s may pass the running maximum m by kSlack
// before the sums are rescaled, so p < 2^14 fits a half, and a p down to
// 2^-20 of the maximum is a normal one.
constexpr float kRaise = 6.f, kSlack = 8.f;

struct AttnArgs {
    const uint8_t *kc, *vc;
    const float *ks, *vs;
    float *weight;
    int32_t n_blocks, H, D, G;           // H kv heads, G heads to each
    Seqs q;
    const void *qd;
    void *od;
    int64_t q_row, q_head, o_row, o_head;
    int32_t dtype, wide;                 // wide: q may be read 16 bytes at a time
    float scale;                         // times log2(e)
    int32_t nsplit, per_split, tiles;    // key splits, blocks of one, column tiles
    int32_t cols, blocks;                // max_new * G, ceil(max_length / 64)
    float *part_o, *part_lse;            // [seq][head][split][cols]([D])
    float *lse;                          // [row][heads], log2 units; +inf: nothing seen
    float *s;                            // [seq][block][head][cols][64] scores, or NULL
    float decay;
};

__device__ inline float group_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float group_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// The codes of a dword that stand for NaN (e4m3), as a mask of their bytes.
__device__ inline uint32_t nan_bytes(uint32_t w)
{
    const uint32_t x = (w & 0x7f7f7f7fu) ^ 0x7f7f7f7fu;
    const uint32_t z = ~(x + 0x7f7f7f7fu) & 0x80808080u;
    return (z >> 7) * 0xffu;
}

// One query row's dims as matrix operands: for chunk c and half m the dims
// c * 64 + g * 16 + m * 8 .. + 8.  A row of bfloat16 is scaled by a power of
// two so that it fits halves; *unscale takes that out of the score.
template <int ND>
__device__ inline void load_query(const AttnArgs &a, int64_t row, int head, bool valid, int g,
                                  half8v (&qf)[ND][2], float *unscale)
{
    *unscale = 1.f;
    const uint16_t *p = (const uint16_t *)a.qd + row * a.q_row + head * a.q_head;
    uint16_t u[ND][16];
    for (int c = 0; c < ND; ++c) {
        const int d = c * 64 + g * 16;
        if (!valid || d >= a.D) {
            for (int e = 0; e < 16; ++e) u[c][e] = 0;
        } else if (a.wide) {
            *(uint4 *)&u[c][0] = *(const uint4 *)(p + d);
            *(uint4 *)&u[c][8] = *(const uint4 *)(p + d + 8);
        } else {
            for (int e = 0; e < 16; ++e) u[c][e] = p[d + e];
        }
    }
    if (a.dtype == QLM_F16) {
        for (int c = 0; c < ND; ++c)
            for (int m = 0; m < 2; ++m)
                for (int e = 0; e < 8; ++e)
                    qf[c][m][e] = __builtin_bit_cast(_Float16, u[c][m * 8 + e]);
        return;
    }
    uint32_t top = 0;                     // greatest exponent of a finite element
    for (int c = 0; c < ND; ++c)
        for (int e = 0; e < 16; ++e) {
            const uint32_t x = (u[c][e] >> 7) & 0xff;
            top = x < 255 ? max(top, x) : top;
        }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    // |q| < 2^(top - 126): to below 2^15
    const int up = min(15 - ((int)top - 126), 126);
    const float by = ldexpf(1.f, up);
    *unscale = ldexpf(1.f, -up);
    for (int c = 0; c < ND; ++c)
        for (int m = 0; m < 2; ++m)
            for (int e = 0; e < 8; ++e)
                qf[c][m][e] = (_Float16)(
                    __builtin_bit_cast(float, (uint32_t)u[c][m * 8 + e] << 16) * by);
}

// Few query rows (decode): the columns of a tile are the query rows and heads
// of one (sequence, kv head); the workgroup's four waves take blocks of 64 slots in
// turn, each with its own running maximum, sum and output, joined at the end.
// Scores S^T[slot][column] = K Q^T and outputs O^T[dim][column] = V^T P^T are
// 16x16x32 matrix instructions; the score's layout (a lane holds 4 slots of a
// column) is the layout in which P^T is taken, because the values are held in
// that order of slots, so nothing passes through shared memory.
template <int FMT, int ND, int NT>
__global__ __launch_bounds__(kThreads) void k_attend_rows(AttnArgs a)
{
    constexpr int DT = ND * 4;                   // tiles of 16 dims
    __shared__ float lo[kWaves][16][DT * 16 + 4];
    __shared__ float llse[kWaves][NT][16];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int g = lane >> 4, c16 = lane & 15;
    int64_t at = blockIdx.x;
    const int sp = (int)(at % a.nsplit);
    at /= a.nsplit;
    const int ct = (int)(at % a.tiles);
    at /= a.tiles;
    const int h = (int)(at % a.H), s = (int)(at / a.H);
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const int len = seq_length(a.q, s);
    const int cols = n * a.G, col0 = ct * NT * 16;
    if (col0 >= cols) return;
    const int before = len - n;                  // slots that row 0 sees, less one
    const int hi_lim = before + min(cols - 1, col0 + NT * 16 - 1) / a.G + 1;
    const int lo_lim = before + col0 / a.G + 1;
    const int nb = (max(hi_lim, 0) + kBlock - 1) / kBlock;
    const int b0 = sp * a.per_split, b1 = min(nb, b0 + a.per_split);
    if (sp > 0 && b0 >= nb) return;
    const int live = max(1, (nb + a.per_split - 1) / a.per_split);

    half8v qf[NT][ND][2];
    float fac[NT];
    int lim[NT];
    for (int k = 0; k < NT; ++k) {
        const int c = col0 + k * 16 + c16;
        const bool valid = c < cols;
        load_query<ND>(a, row0 + (valid ? c / a.G : 0), h * a.G + (valid ? c % a.G : 0), valid, g,
                       qf[k], &fac[k]);
        fac[k] *= a.scale;
        lim[k] = valid ? before + c / a.G + 1 : 0;
    }
    float4v acc[NT][DT];
    float m[NT], l[NT];
    for (int k = 0; k < NT; ++k) {
        m[k] = -__builtin_inff();
        l[k] = 0.f;
        for (int d = 0; d < DT; ++d) acc[k][d] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    float vscale = 0.f;                          // the values' common scale so far
    const int32_t *table = a.q.table + s * a.q.table_stride;
    const int D = a.D;

    for (int j = b0 + wv; j < b1; j += kWaves) {
        const int id = __builtin_amdgcn_readfirstlane(table[j]);
        if ((unsigned)id >= (unsigned)a.n_blocks) continue;   // no slots there
        const int64_t bh = (int64_t)id * a.H + h;
        const uint8_t *kp = a.kc + bh * kBlock * D, *vp = a.vc + bh * kBlock * D;
        uint4 kk[4][ND], vv[DT];
        for (int t = 0; t < 4; ++t)
            for (int c = 0; c < ND; ++c) {
                const int d = c * 64 + g * 16;
                kk[t][c] = d < D ? *(const uint4 *)(kp + (t * 16 + c16) * D + d)
                                 : uint4{0, 0, 0, 0};
            }
        for (int d = 0; d < DT; ++d)
            vv[d] = d * 16 < D ? *(const uint4 *)(vp + (g * D + d * 16 + c16) * 16)
                               : uint4{0, 0, 0, 0};
        const float ksc = a.ks[bh], vsc = a.vs[bh];

        float4v sc[NT][4];
        for (int t = 0; t < 4; ++t) {
            for (int k = 0; k < NT; ++k) sc[k][t] = float4v{0.f, 0.f, 0.f, 0.f};
            for (int c = 0; c < ND; ++c) {
                const half8v x0 = halves8<FMT>(kk[t][c].x, kk[t][c].y);
                const half8v x1 = halves8<FMT>(kk[t][c].z, kk[t][c].w);
                for (int k = 0; k < NT; ++k) {
                    sc[k][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x0, qf[k][c][0], sc[k][t],
                                                                      0, 0, 0);
                    sc[k][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, qf[k][c][1], sc[k][t],
                                                                      0, 0, 0);
                }
            }
        }
        const bool masked = (j + 1) * kBlock > lo_lim;
        const int slot0 = j * kBlock + 4 * g;    // of tile 0, element 0
        float top[NT];
        bool grow = false;
        for (int k = 0; k < NT; ++k) {
            const float f = fac[k] * ksc;
            top[k] = -__builtin_inff();
            for (int t = 0; t < 4; ++t)
                for (int i = 0; i < 4; ++i) {
                    float x = sc[k][t][i] * f;
                    if (masked && slot0 + t * 16 + i >= lim[k]) x = -__builtin_inff();
                    sc[k][t][i] = x;
                    top[k] = fmaxf(top[k], x);
                }
            top[k] = group_max(top[k]);
            grow = grow || top[k] > m[k] + kSlack;
        }
        if (a.s)
            for (int k = 0; k < NT; ++k) {
                const int c = col0 + k * 16 + c16;
                if (c < cols) {
                    float *p = a.s + ((((int64_t)s * a.blocks + j) * a.H + h) * a.cols + c) * kBlock;
                    for (int t = 0; t < 4; ++t) *(float4v *)(p + t * 16 + 4 * g) = sc[k][t];
                }
            }
        if (__any(grow)) {
            for (int k = 0; k < NT; ++k) {
                const float mn = fmaxf(m[k], top[k]);
                const float al = mn == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m[k] - mn);
                m[k] = mn;
                l[k] *= al;
                for (int d = 0; d < DT; ++d) acc[k][d] *= al;
            }
        }
        if (vsc > vscale) {                      // (uniform over the wave)
            const float al = vscale / vsc;
            for (int k = 0; k < NT; ++k)
                for (int d = 0; d < DT; ++d) acc[k][d] *= al;
            vscale = vsc;
        }
        const float vrel = vsc / vscale;
        half8v pb[NT][2];
        for (int k = 0; k < NT; ++k) {
            const float base = m[k] == -__builtin_inff() ? 0.f : m[k] - kRaise;
            for (int t = 0; t < 4; ++t)
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(sc[k][t][i] - base);
                    l[k] += p;
                    pb[k][t >> 1][(t & 1) * 4 + i] = (_Float16)(p * vrel);
                }
        }
        if (masked) {
            // codes that no row of the tile sees are zeroed; a NaN that some rows
            // see and others do not is taken out and given to those that see it
            uint32_t nans = 0;
            for (int d = 0; d < DT; ++d)
                for (int t = 0; t < 4; ++t) {
                    uint32_t &w = (&vv[d].x)[t];
                    const int left = hi_lim - (slot0 + t * 16);
                    w = left <= 0 ? 0u : left < 4 ? w & (0xffffffffu >> (8 * (4 - left))) : w;
                    if (FMT == QLM_KV_E4M3) nans |= nan_bytes(w);
                }
            if (FMT == QLM_KV_E4M3 && hi_lim > lo_lim && __any(nans != 0)) {
                half8v seen[NT][2];
                for (int k = 0; k < NT; ++k)
                    for (int t = 0; t < 4; ++t)
                        for (int i = 0; i < 4; ++i)
                            seen[k][t >> 1][(t & 1) * 4 + i] =
                                (_Float16)(slot0 + t * 16 + i < lim[k] ? 1.f : 0.f);
                for (int d = 0; d < DT; ++d) {
                    half8v x[2];
                    for (int t = 0; t < 4; ++t) {
                        uint32_t &w = (&vv[d].x)[t];
                        const uint32_t z = nan_bytes(w);
                        w &= ~z;
                        for (int i = 0; i < 4; ++i)
                            x[t >> 1][(t & 1) * 4 + i] =
                                (_Float16)((z >> (8 * i)) & 1 ? 1.f : 0.f);
                    }
                    for (int k = 0; k < NT; ++k) {
                        float4v cnt = {0.f, 0.f, 0.f, 0.f};
                        for (int u = 0; u < 2; ++u)
                            cnt = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[u], seen[k][u], cnt, 0,
                                                                         0, 0);
                        for (int i = 0; i < 4; ++i)
                            if (cnt[i] > 0.f) acc[k][d][i] = __builtin_nanf("");
                    }
                }
            }
        }
        for (int d = 0; d < DT; ++d) {
            const half8v x0 = halves8<FMT>(vv[d].x, vv[d].y);
            const half8v x1 = halves8<FMT>(vv[d].z, vv[d].w);
            for (int k = 0; k < NT; ++k) {
                acc[k][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x0, pb[k][0], acc[k][d], 0, 0, 0);
                acc[k][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, pb[k][1], acc[k][d], 0, 0, 0);
            }
        }
    }

    // the four waves' results, a tile of columns at a time: normalised outputs
    // weighted by exp2(lse)
    for (int k = 0; k < NT; ++k) {
        const float sum = group_sum(l[k]);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (g == 0)
            llse[wv][k][c16] = sum == 0.f ? -__builtin_inff() : m[k] - kRaise + __builtin_amdgcn_logf(sum);
        __syncthreads();
        for (int d = 0; d < DT; ++d) {
            const float4v o = acc[k][d] * inv;
            for (int i = 0; i < 4; ++i) lo[wv][c16][d * 16 + 4 * g + i] = o[i] * vscale;
        }
        __syncthreads();
        // 16 threads to a column
        const int cc = threadIdx.x >> 4, c = col0 + k * 16 + cc;
        float f[kWaves], M = -__builtin_inff(), L = 0.f;
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, llse[w][k][cc]);
        for (int w = 0; w < kWaves; ++w) {
            f[w] = M == -__builtin_inff() && !(llse[w][k][cc] != llse[w][k][cc])
                       ? 0.f : __builtin_amdgcn_exp2f(llse[w][k][cc] - M);
            L += f[w];
        }
        const float li = L == 0.f ? 0.f : 1.f / L;
        if (c < cols) {
            const int64_t pi = (((int64_t)s * a.H + h) * a.nsplit + sp) * a.cols + c;
            const int row = row0 + c / a.G, head = h * a.G + c % a.G;
            for (int d = threadIdx.x & 15; d < D; d += 16) {
                float o = 0.f;
                for (int w = 0; w < kWaves; ++w) o += f[w] == 0.f ? 0.f : f[w] * lo[w][cc][d];
                o *= li;
                if (live > 1)
                    a.part_o[pi * D + d] = o;
                else
                    ((uint16_t *)a.od)[row * a.o_row + head * a.o_head + d] =
                        row_bits(o, a.dtype);
            }
            if ((threadIdx.x & 15) == 0) {
                const float z = M + __builtin_amdgcn_logf(L);
                if (live > 1)
                    a.part_lse[pi] = L == 0.f ? -__builtin_inff() : z;
                else
                    a.lse[(int64_t)row * a.H * a.G + head] = L == 0.f ? __builtin_inff() : z;
            }
        }
    }
}

// Joins the key splits of a column: one wave to a (sequence, kv head, column).
__global__ __launch_bounds__(kThreads) void k_attend_join(AttnArgs a, int tile_cols)
{
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int64_t sh = w / a.cols;
    const int c = (int)(w % a.cols);
    if (sh >= (int64_t)a.q.n_seqs * a.H) return;
    const int s = (int)(sh / a.H), h = (int)(sh % a.H);
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const int cols = n * a.G;
    if (c >= cols) return;
    // the splits of its tile, as the workgroups of the tile counted them
    const int col0 = c / tile_cols * tile_cols;
    const int hi = seq_length(a.q, s) - n + min(cols - 1, col0 + tile_cols - 1) / a.G + 1;
    const int nb = (max(hi, 0) + kBlock - 1) / kBlock;
    const int live = max(1, (nb + a.per_split - 1) / a.per_split);
    if (live <= 1) return;
    const int64_t p0 = sh * a.nsplit * a.cols + c;
    float M = -__builtin_inff();
    for (int k = lane; k < live; k += 64) M = fmaxf(M, a.part_lse[p0 + (int64_t)k * a.cols]);
    for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    float L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < live; ++k) {
        const float z = a.part_lse[p0 + (int64_t)k * a.cols];
        const float f = z == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(z - M);
        L += f;
        if (f == 0.f) continue;
        const float *po = a.part_o + (p0 + (int64_t)k * a.cols) * a.D;
        for (int e = 0; e < 4; ++e)
            if (e * 64 + lane < a.D) acc[e] += f * po[e * 64 + lane];
    }
    const int row = row0 + c / a.G, head = h * a.G + c % a.G;
    const float li = L == 0.f ? 0.f : 1.f / L;
    for (int e = 0; e < 4; ++e)
        if (e * 64 + lane < a.D)
            ((uint16_t *)a.od)[row * a.o_row + head * a.o_head + e * 64 + lane] =
                row_bits(acc[e] * li, a.dtype);
    if (lane == 0)
        a.lse[(int64_t)row * a.H * a.G + head] = L == 0.f ? __builtin_inff() : M + __builtin_amdgcn_logf(L);
}

// Weights from the scores that k_attend_rows left: a wave to a (sequence,
// block, kv head), a lane to a slot.
__global__ __launch_bounds__(kThreads) void k_attend_weights(AttnArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int h = (int)(w % a.H);
    const int64_t sb = w / a.H;
    const int j = (int)(sb % a.blocks), s = (int)(sb / a.blocks);
    if (s >= a.q.n_seqs) return;
    const int len = seq_length(a.q, s);
    if (j * kBlock >= len) return;
    const int id = a.q.table[s * a.q.table_stride + j];
    if ((unsigned)id >= (unsigned)a.n_blocks) return;
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const float *sc = a.s + w * a.cols * kBlock + lane;
    const float *lse = a.lse + ((int64_t)row0 * a.H + h) * a.G;
    float sum = 0.f;
    const int before = len - n;
    for (int t = 0; t < n; ++t) {
        if (before + t < j * kBlock) continue;    // (the row's scores were not formed)
        for (int e = 0; e < a.G; ++e)
            sum += __builtin_amdgcn_exp2f(sc[(t * a.G + e) * kBlock] - lse[(int64_t)t * a.H * a.G + e]);
    }
    if (j * kBlock + lane >= len) return;
    float *at = a.weight + ((int64_t)id * a.H + h) * kBlock + lane;
    *at = a.decay == 0.f ? sum : a.decay * *at + sum;
}

// Weights where the query rows are many: a workgroup to a (sequence, block, kv
// head) forms the block's scores again, tile of columns by tile, and adds up
// their probabilities.
template <int FMT, int ND>
__global__ __launch_bounds__(kThreads) void k_attend_colsum(AttnArgs a)
{
    __shared__ float part[kWaves][kBlock];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int g = lane >> 4, c16 = lane & 15;
    const int64_t w = blockIdx.x;
    const int h = (int)(w % a.H);
    const int64_t sb = w / a.H;
    const int j = (int)(sb % a.blocks), s = (int)(sb / a.blocks);
    const int len = seq_length(a.q, s);
    if (j * kBlock >= len) return;
    const int id = a.q.table[s * a.q.table_stride + j];
    if ((unsigned)id >= (unsigned)a.n_blocks) return;
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const int cols = n * a.G, before = len - n, D = a.D;
    const int64_t bh = (int64_t)id * a.H + h;
    const uint8_t *kp = a.kc + bh * kBlock * D;
    uint4 kk[4][ND];
    for (int t = 0; t < 4; ++t)
        for (int c = 0; c < ND; ++c) {
            const int d = c * 64 + g * 16;
            kk[t][c] = d < D ? *(const uint4 *)(kp + (t * 16 + c16) * D + d) : uint4{0, 0, 0, 0};
        }
    const float ksc = a.ks[bh];
    const int slot0 = j * kBlock + 4 * g;
    float4v sum[4];
    for (int t = 0; t < 4; ++t) sum[t] = float4v{0.f, 0.f, 0.f, 0.f};
    // rows that see the block's first slot
    const int first = max(0, j * kBlock - before) * a.G / 16;
    for (int ct = first + wv; ct * 16 < cols; ct += kWaves) {
        const int c = ct * 16 + c16;
        const bool valid = c < cols;
        const int row = row0 + (valid ? c / a.G : 0), head = h * a.G + (valid ? c % a.G : 0);
        half8v qf[ND][2];
        float fac;
        load_query<ND>(a, row, head, valid, g, qf, &fac);
        fac *= a.scale * ksc;
        const int lim = valid ? before + c / a.G + 1 : 0;
        const float lse = valid ? a.lse[(int64_t)row * a.H * a.G + head] : 0.f;
        for (int t = 0; t < 4; ++t) {
            float4v sc = {0.f, 0.f, 0.f, 0.f};
            for (int x = 0; x < ND; ++x) {
                sc = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves8<FMT>(kk[t][x].x, kk[t][x].y),
                                                            qf[x][0], sc, 0, 0, 0);
                sc = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves8<FMT>(kk[t][x].z, kk[t][x].w),
                                                            qf[x][1], sc, 0, 0, 0);
            }
            for (int i = 0; i < 4; ++i)
                if (slot0 + t * 16 + i < lim) sum[t][i] += __builtin_amdgcn_exp2f(sc[i] * fac - lse);
        }
    }
    for (int t = 0; t < 4; ++t)
        for (int i = 0; i < 4; ++i) {
            float x = sum[t][i];
            for (int o = 1; o < 16; o <<= 1) x += __shfl_xor(x, o);
            if (c16 == 0) part[wv][t * 16 + 4 * g + i] = x;
        }
    __syncthreads();
    const int o = threadIdx.x;
    if (o < kBlock && j * kBlock + o < len) {
        float x = 0.f;
        for (int k = 0; k < kWaves; ++k) x += part[k][o];
        float *at = a.weight + bh * kBlock + o;
        *at = a.decay == 0.f ? x : a.decay * *at + x;
    }
}

// -- host -------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

constexpr int kRowsMax = 64;     // columns for which scores are kept for the weights

struct Plan {
    int nt, tiles, nsplit, per_split, cols, blocks;
    size_t part_o, part_lse, lse, s, total;
};

Plan plan_of(const qlm_kv_cache *c, const qlm_kv_batch *b, int32_t n_heads, bool weights)
{
    Plan p{};
    const int64_t cols = (int64_t)b->max_new * (n_heads / c->n_kv_heads);
    p.cols = (int)std::min<int64_t>(cols, INT32_MAX);
    p.nt = cols <= 16 ? 1 : cols <= 32 ? 2 : 4;
    if (c->head_dim > 128) p.nt = std::min(p.nt, 2);
    p.tiles = (int)((cols + 16 * p.nt - 1) / (16 * p.nt));
    p.blocks = std::max(1, (b->max_length + kBlock - 1) / kBlock);
    // Enough workgroups for every CU twice over, four blocks each at least (a
    // wave's), and no more than 32 so that ragged lengths spread evenly.
    const int64_t wg = (int64_t)b->n_seqs * c->n_kv_heads * p.tiles;
    const int64_t want = wg * p.blocks / 1024;
    p.per_split = (int)std::max<int64_t>(4, std::min<int64_t>(32, want / 4 * 4));
    if (cols > kRowsMax) p.per_split = p.blocks;
    p.nsplit = (p.blocks + p.per_split - 1) / p.per_split;
    const size_t parts = (size_t)b->n_seqs * c->n_kv_heads * p.nsplit * p.cols;
    p.part_o = 0;
    p.part_lse = p.part_o + (p.nsplit > 1 ? align256(parts * c->head_dim * 4) : 0);
    p.lse = p.part_lse + (p.nsplit > 1 ? align256(parts * 4) : 0);
    p.s = p.lse + align256((size_t)b->n_rows * n_heads * 4);
    p.total = p.s;
    if (weights && cols <= kRowsMax)
        p.total += align256((size_t)b->n_seqs * p.blocks * c->n_kv_heads * p.cols * kBlock * 4);
    return p;
}

template <int FMT, int ND, int NT> void launch_rows(const AttnArgs &a, int64_t grid, hipStream_t st)
{
    k_attend_rows<FMT, ND, NT><<<(unsigned)grid, kThreads, 0, st>>>(a);
}

template <int FMT> void launch_rows(const AttnArgs &a, int nt, int64_t grid, hipStream_t st)
{
    if (a.D <= 64) {
        nt == 1 ? launch_rows<FMT, 1, 1>(a, grid, st)
                : nt == 2 ? launch_rows<FMT, 1, 2>(a, grid, st) : launch_rows<FMT, 1, 4>(a, grid, st);
    } else if (a.D <= 128) {
        nt == 1 ? launch_rows<FMT, 2, 1>(a, grid, st)
                : nt == 2 ? launch_rows<FMT, 2, 2>(a, grid, st) : launch_rows<FMT, 2, 4>(a, grid, st);
    } else {
        nt == 1 ? launch_rows<FMT, 4, 1>(a, grid, st) : launch_rows<FMT, 4, 2>(a, grid, st);
    }
}

template <int FMT> void launch_colsum(const AttnArgs &a, int64_t grid, hipStream_t st)
{
    if (a.D <= 64)
        k_attend_colsum<FMT, 1><<<(unsigned)grid, kThreads, 0, st>>>(a);
    else if (a.D <= 128)
        k_attend_colsum<FMT, 2><<<(unsigned)grid, kThreads, 0, st>>>(a);
    else
        k_attend_colsum<FMT, 4><<<(unsigned)grid, kThreads, 0, st>>>(a);
}

}  // namespace

extern "C" {

size_t qlm_kv_attention_workspace_bytes(const qlm_kv_cache *cache, const qlm_kv_batch *batch,
                                        int32_t n_heads, int32_t accumulate)
{
    if (!cache || !batch || cache->n_kv_heads < 1 || n_heads < cache->n_kv_heads ||
        batch->n_seqs <= 0 || batch->n_rows < 0 || batch->max_new < 1 || batch->max_length < 0)
        return 0;
    return plan_of(cache, batch, n_heads, accumulate != 0).total;
}

int qlm_kv_attention(const qlm_kv_cache *cache, const qlm_kv_batch *batch,
                     const qlm_kv_query *query, void *ws, size_t ws_bytes, qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    int rc = check_cache(cache);
    if (!rc) rc = check_batch(batch);
    if (rc) return rc;
    if (!query) return fail(QLM_ERR_ARG, "query is NULL");
    if (query->n_heads < 1 || query->n_heads % cache->n_kv_heads || query->n_heads > (1 << 16))
        return fail(QLM_ERR_ARG, "n_heads must be a multiple of n_kv_heads, at most 65536");
    if (!(query->scale - query->scale == 0.f)) return fail(QLM_ERR_ARG, "scale must be finite");
    if (query->accumulate) {
        if (!cache->weight) return fail(QLM_ERR_ARG, "the cache keeps no weights");
        if (!(query->weight_decay >= 0.f) || query->weight_decay - query->weight_decay != 0.f)
            return fail(QLM_ERR_ARG, "weight_decay must be finite and >= 0");
    }
    if (batch->n_seqs == 0 || (batch->n_rows == 0 && !query->accumulate)) return QLM_OK;
    if (batch->n_rows > 0) {
        if ((rc = check_rows(&query->q, "q")) || (rc = check_rows(&query->out, "out"))) return rc;
        if (query->q.dtype != query->out.dtype)
            return fail(QLM_ERR_ARG, "q and out must have one dtype");
        if (query->q.data == query->out.data) return fail(QLM_ERR_ARG, "out may not alias q");
    }
    const Plan p = plan_of(cache, batch, query->n_heads, query->accumulate != 0);
    rc = check_workspace(ws, ws_bytes, p.total);
    if (rc) return rc;

    AttnArgs a{};
    a.kc = (const uint8_t *)cache->k_codes;
    a.vc = (const uint8_t *)cache->v_codes;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.weight = cache->weight;
    a.n_blocks = cache->n_blocks;
    a.H = cache->n_kv_heads;
    a.D = cache->head_dim;
    a.G = query->n_heads / cache->n_kv_heads;
    a.q = seqs_of(batch);
    a.qd = query->q.data;
    a.od = query->out.data;
    a.q_row = query->q.row_stride;
    a.q_head = query->q.head_stride;
    a.o_row = query->out.row_stride;
    a.o_head = query->out.head_stride;
    a.dtype = query->q.dtype;
    a.wide = (uintptr_t)a.qd % 16 == 0 && a.q_row % 8 == 0 && a.q_head % 8 == 0;
    a.scale = query->scale * kLog2e;
    a.nsplit = p.nsplit;
    a.per_split = p.per_split;
    a.tiles = p.tiles;
    a.cols = p.cols;
    a.blocks = p.blocks;
    char *base = (char *)ws;
    a.part_o = (float *)(base + p.part_o);
    a.part_lse = (float *)(base + p.part_lse);
    a.lse = (float *)(base + p.lse);
    const bool kept = query->accumulate && p.cols <= kRowsMax;
    a.s = kept ? (float *)(base + p.s) : nullptr;
    a.decay = query->weight_decay;

    const bool e4m3 = cache->format == QLM_KV_E4M3;
    const int64_t sh = (int64_t)batch->n_seqs * a.H;
    const int64_t grid = sh * p.tiles * p.nsplit;
    if (grid > INT32_MAX || sh * p.cols > ((int64_t)1 << 32) || sh * p.blocks > INT32_MAX)
        return fail(QLM_ERR_CAPACITY, "too many rows or blocks in one call");
    hipError_t e;
    if (batch->n_rows > 0) {
        if (e4m3)
            launch_rows<QLM_KV_E4M3>(a, p.nt, grid, stream);
        else
            launch_rows<QLM_KV_INT8>(a, p.nt, grid, stream);
        if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_attend_rows launch");
        if (p.nsplit > 1) {
            const int64_t wg = (sh * p.cols + kWaves - 1) / kWaves;
            k_attend_join<<<(unsigned)wg, kThreads, 0, stream>>>(a, 16 * p.nt);
            if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_attend_join launch");
        }
    }
    if (query->accumulate && batch->max_length > 0) {
        if (kept) {
            const int64_t wg = (sh * p.blocks + kWaves - 1) / kWaves;
            k_attend_weights<<<(unsigned)wg, kThreads, 0, stream>>>(a);
        } else if (e4m3) {
            launch_colsum<QLM_KV_E4M3>(a, sh * p.blocks, stream);
        } else {
            launch_colsum<QLM_KV_INT8>(a, sh * p.blocks, stream);
        }
        if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "weight launch");
    }
    return QLM_OK;
}

}  // extern "C"

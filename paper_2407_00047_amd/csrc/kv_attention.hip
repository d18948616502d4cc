// kv_attention.hip -- attention over the 8-bit token cache
// (qlm_kv_attention; the definition stands in include/qlm.h).
#include "kv.h"

#include <algorithm>
#include <string>

// A score is rounded before the maximum is taken off it, as the maximum was (a fused
// multiply-add would leave the rounding error of a large score in the exponent).
#pragma clang fp contract(off)

namespace {

using namespace qlm_kv;
using qlm_internal::fail;
using qlm_internal::hip_fail;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896340736f;
// p = 2^(s - m), in which s may pass the running maximum m by kSlack before the
// sums are rescaled.  As a half it is held kRaised times as large: p < 2^14 then
// fits, and a p down to 2^-20 of the maximum is a normal one.  Half precision because
// the second product runs on 16-bit matrix instructions as the first does: 2^-11 of each p,
// below what rounding an output to bfloat16 costs, and seen beside a half's (an error of
// 0.00027 where rounding alone gives 0.00021: 192 sequences of up to 16000).
constexpr float kSlack = 8.f, kRaised = 64.f;

// A column's running maximum m and its sum l of 2^(s - m), apart: their common
// logarithm would lose the sum beside a large maximum.  Of a finished column
// what gives p = 2^(s - top) sum; {0, 0} where nothing is seen.
struct TopSum {
    float top, sum;
};
__device__ inline TopSum finished(float m, float l)
{
    return l == 0.f ? TopSum{0.f, 0.f} : TopSum{m, 1.f / l};
}
// The weight of a part in a join whose greatest maximum is M.
__device__ inline float part_weight(TopSum p, float M)
{
    return p.sum == 0.f ? 0.f : p.sum * __builtin_amdgcn_exp2f(p.top - M);
}

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
    int32_t few;                         // columns up to which a sequence has few rows
    int32_t tile;                        // columns of a tile (k_attend_rows)
    int32_t workers;                     // waves that share the units (k_attend_rows)
    int32_t cols, blocks;                // max_new * G, ceil(max_length / 64)
    float *part_o;                       // [2 worker + which][tile][D] outputs, normalised
    TopSum *part_ts;                     // [2 worker + which][tile] their m and l
    TopSum *done;                        // [kv head][row][G] finished columns
    float *s;                            // [seq][block][head][few][64] scores, or NULL
    float decay;
    // sequences of many rows
    uint16_t *qh;                        // [kv head][8 ND][row][G][8] queries as halves
    float *qfac;                         // [kv head][row][G] what takes their scaling out
    int32_t splits;                      // of the keys
    float *split_o;                      // [split][kv head][row][G][D], as part_o
    TopSum *split_ts;                    // [split][kv head][row][G]
    int32_t shares;                      // of a block's columns (k_attend_colsum)
    float *share;                        // [share][seq][block][kv head][64] weights
};

// Column of head e of a row among all rows of kv head h.
__device__ inline int64_t column(const AttnArgs &a, int h, int64_t row, int e)
{
    return ((int64_t)h * a.q.n_rows + row) * a.G + e;
}

// Maximum and sum over the four lanes of a column (16 lanes apart).
__device__ inline void swap16(float x, float *a, float *b)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    *a = __builtin_bit_cast(float, (uint32_t)r[0]);
    *b = __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ inline void swap32(float x, float *a, float *b)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    *a = __builtin_bit_cast(float, (uint32_t)r[0]);
    *b = __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ inline float group_max(float x)
{
    float a, b;
    swap16(x, &a, &b);
    swap32(fmaxf(a, b), &a, &b);
    return fmaxf(a, b);
}
__device__ inline float group_sum(float x)
{
    float a, b;
    swap16(x, &a, &b);
    swap32(a + b, &a, &b);
    return a + b;
}

// The codes of a dword that stand for NaN (e4m3), as a mask of their bytes.
__device__ inline uint32_t nan_bytes(uint32_t w)
{
    const uint32_t x = (w & 0x7f7f7f7fu) ^ 0x7f7f7f7fu;
    const uint32_t z = ~(x + 0x7f7f7f7fu) & 0x80808080u;
    return (z >> 7) * 0xffu;
}

// One query row's dims as they came: of chunk c the dims c * 64 + g * 16 .. + 16.
template <int ND> struct Query {
    uint4 u[ND][2];
};

template <int ND>
__device__ inline void load_query(const AttnArgs &a, int64_t row, int head, bool valid, int g,
                                  Query<ND> &q)
{
    const uint16_t *p = (const uint16_t *)a.qd + row * a.q_row + head * a.q_head;
    for (int c = 0; c < ND; ++c)
        for (int m = 0; m < 2; ++m) {
            const int d = c * 64 + g * 16 + m * 8;
            uint4 x = {0, 0, 0, 0};
            if (valid && d < a.D) {
                if (a.wide) {
                    x = *(const uint4 *)(p + d);
                } else {
                    const uint16_t *e = p + d;
                    x = uint4{e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16,
                              e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16};
                }
            }
            q.u[c][m] = x;
        }
}

// The row as matrix operands: half m of chunk c holds the dims c * 64 + g * 16 +
// m * 8 .. + 8.  A row of bfloat16 is scaled by a power of two so that it fits
// halves, which the codes are turned into by one instruction for two; the result takes that
// out of the score.  Its elements below 2^-29 of the largest lose bits.
template <int ND>
__device__ inline float query_halves(const AttnArgs &a, const Query<ND> &q, half8v (&qf)[ND][2])
{
    if (a.dtype == QLM_F16) {
        for (int c = 0; c < ND; ++c)
            for (int m = 0; m < 2; ++m) qf[c][m] = __builtin_bit_cast(half8v, q.u[c][m]);
        return 1.f;
    }
    uint32_t top = 0;                     // greatest exponent of a finite element
    for (int c = 0; c < ND; ++c)
        for (int m = 0; m < 2; ++m) {
            const uint32_t w[4] = {q.u[c][m].x, q.u[c][m].y, q.u[c][m].z, q.u[c][m].w};
            for (int e = 0; e < 8; ++e) {
                const uint32_t x = (w[e >> 1] >> (16 * (e & 1) + 7)) & 0xff;
                top = x < 255 ? max(top, x) : top;
            }
        }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    // |q| < 2^(top - 126): to below 2^15
    const int up = min(15 - ((int)top - 126), 126);
    const float by = ldexpf(1.f, up);
    for (int c = 0; c < ND; ++c)
        for (int m = 0; m < 2; ++m) {
            const uint32_t w[4] = {q.u[c][m].x, q.u[c][m].y, q.u[c][m].z, q.u[c][m].w};
            for (int e = 0; e < 8; ++e)
                qf[c][m][e] = (_Float16)(
                    __builtin_bit_cast(float, e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16) *
                    by);
        }
    return ldexpf(1.f, -up);
}

// -- few query rows ---------------------------------------------------------
//
// The work is a list of units: one block of 64 slots for one tile of columns
// (query rows and heads) of one kv head, in the order sequence, kv head, tile,
// block.  Each worker (a wave) takes an equal run of units, whatever sequences they
// belong to, so ragged lengths leave no worker behind; what it has for a tile
// goes out as the result if it held every unit of the tile, else as a part that
// k_attend_join adds up.

struct Units {
    int nb, tiles;       // blocks of the sequence, tiles of a kv head
};

__device__ inline Units units_of(const AttnArgs &a, int s)
{
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    if (n * a.G > a.few) return {0, 0};          // (k_attend_prompt)
    return {(seq_length(a.q, s) + kBlock - 1) / kBlock, (n * a.G + a.tile - 1) / a.tile};
}

// Units of each chunk of ceil(n_seqs / kThreads) sequences before it, and of all.
__device__ inline int unit_prefix(const AttnArgs &a, int *pre, int *wave_sum)
{
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6;
    const int chunk = (a.q.n_seqs + kThreads - 1) / kThreads;
    int sum = 0;
    for (int s = t * chunk; s < min(a.q.n_seqs, (t + 1) * chunk); ++s) {
        const Units u = units_of(a, s);
        sum += u.nb * u.tiles * a.H;
    }
    int run = sum;
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(run, o);
        run += lane >= o ? v : 0;
    }
    if (lane == 63) wave_sum[wv] = run;
    __syncthreads();
    int before = 0, all = 0;
    for (int k = 0; k < kWaves; ++k) {
        before += k < wv ? wave_sum[k] : 0;
        all += wave_sum[k];
    }
    pre[t] = before + run - sum;
    __syncthreads();
    return all;
}

__device__ inline int units_each(const AttnArgs &a, int all)
{
    return max(1, (all + a.workers - 1) / a.workers);
}

// Where a worker stands: unit `block` of item (kv head, tile) of a sequence.
struct Cursor {
    int s, h, tile, block, nb, tiles;

    __device__ void enter(const AttnArgs &a, int seq)   // the first sequence from seq on with units
    {
        s = seq;
        h = tile = block = 0;
        nb = tiles = 0;
        for (; s < a.q.n_seqs; ++s) {
            const int len = max(0, min(uniform(a.q.lengths + s), a.q.max_length));
            int n = 1;
            if (a.q.row_start) {
                const int r0 = max(0, min(uniform(a.q.row_start + s), a.q.n_rows));
                n = min(max(r0, min(uniform(a.q.row_start + s + 1), a.q.n_rows)) - r0, a.q.max_new);
            } else if (s >= a.q.n_rows) {
                n = 0;
            }
            nb = (len + kBlock - 1) / kBlock;
            tiles = n * a.G > a.few ? 0 : (n * a.G + a.tile - 1) / a.tile;
            if (nb * tiles > 0) break;
        }
    }
    __device__ void next(const AttnArgs &a)
    {
        if (++block < nb) return;
        block = 0;
        if (++tile < tiles) return;
        tile = 0;
        if (++h < a.H) return;
        enter(a, s + 1);
    }
    __device__ int block_id(const AttnArgs &a) const
    {
        return s < a.q.n_seqs ? uniform(a.q.table + s * a.q.table_stride + block) : -1;
    }
    // (an unmapped block: any memory of the pool)
    __device__ int64_t row(const AttnArgs &a, int id) const
    {
        return (int64_t)((unsigned)id < (unsigned)a.n_blocks ? id : 0) * a.H + h;
    }
};

// Scores S^T[slot][column] = K Q^T and outputs O^T[dim][column] = V^T P^T are
// 16x16x32 matrix instructions; the score's layout (a lane holds 4 slots of a
// column) is the layout in which P^T is taken, because the values are held in
// that order of slots, so nothing passes through shared memory.  A block's keys
// and values stay in registers; the next unit's keys are loaded as soon as this
// one's scores are formed, its values as soon as this one's are added, so that
// loads are always under way.
// Bound by the cache's bytes: 192 ragged sequences of up to 16000 (3.2 GB, 8 kv heads of
// 128) 545 us, 5.8 TB/s; two of up to 150000 74 (5.1); 48 ragged ones of up to 4096 that write
// their scores 60 us (3.5 TB/s: runs are rounded up, there to 7 units where a wave's part
// is 6.07, and an eighth of the waves has none; the scores are a sixteenth of the bytes); one
// of 700 9 us, a launch and its dependent reads.
template <int FMT, int ND, int NT>
__global__ __launch_bounds__(kThreads, ND * NT <= 2 ? 2 : 1) void k_attend_rows(AttnArgs a)
{
    constexpr int DT = ND * 4;                   // tiles of 16 dims
    __shared__ int pre[kThreads], wave_sum[kWaves];
    const int lane = threadIdx.x & 63;
    const int g = lane >> 4, c16 = lane & 15;
    const int worker = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
    Cursor cur;
    int all, each, u0, left;
    if (a.q.n_seqs <= 64) {                      // a lane to a sequence: no barrier, one read
        const Units un = lane < a.q.n_seqs ? units_of(a, lane) : Units{0, 0};
        int run = un.nb * un.tiles * a.H;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(run, o);
            run += lane >= o ? v : 0;
        }
        all = __builtin_amdgcn_readlane(run, 63);
        each = units_each(a, all);
        if ((int64_t)worker * each >= all) return;
        u0 = worker * each;
        cur.s = __popcll(__ballot(run <= u0));
        cur.nb = __builtin_amdgcn_readlane(un.nb, cur.s);
        cur.tiles = __builtin_amdgcn_readlane(un.tiles, cur.s);
        left = u0 - (cur.s ? __builtin_amdgcn_readlane(run, cur.s - 1) : 0);
    } else {
        all = __builtin_amdgcn_readfirstlane(unit_prefix(a, pre, wave_sum));
        each = units_each(a, all);
        if ((int64_t)worker * each >= all) return;
        u0 = worker * each;
        // the chunk of sequences that holds unit u0, then the sequence
        int chunk = 0;
        for (int k = 0; k < kWaves; ++k) chunk += __popcll(__ballot(pre[k * 64 + lane] <= u0));
        chunk = __builtin_amdgcn_readfirstlane(chunk) - 1;
        cur.enter(a, chunk * ((a.q.n_seqs + kThreads - 1) / kThreads));
        left = u0 - __builtin_amdgcn_readfirstlane(pre[chunk]);
        while (left >= cur.nb * cur.tiles * a.H) {
            left -= cur.nb * cur.tiles * a.H;
            cur.enter(a, cur.s + 1);
        }
    }
    const int u1 = min(all, u0 + each);
    cur.h = left / (cur.nb * cur.tiles);
    cur.tile = left / cur.nb % cur.tiles;
    cur.block = left % cur.nb;

    const int D = a.D;
    // Dims past the last are read from the last ones: their query is 0, their
    // output unused.  (32 bits beside a uniform base)
    uint32_t koff[ND], voff[DT];
    for (int c = 0; c < ND; ++c) koff[c] = c16 * D + min(c * 64 + g * 16, D - 16);
    for (int d = 0; d < DT; ++d) voff[d] = (g * D + min(d * 16, D - 16) + c16) * 16;
    uint4 kk[4][ND], vv[DT];
    auto load_keys = [&](int64_t bh) {
        const uint8_t *kp = a.kc + bh * kBlock * D;
        for (int t = 0; t < 4; ++t)
            for (int c = 0; c < ND; ++c) kk[t][c] = *(const uint4 *)(kp + t * 16 * D + koff[c]);
    };
    auto load_values = [&](int64_t bh) {
        const uint8_t *vp = a.vc + bh * kBlock * D;
        for (int d = 0; d < DT; ++d) vv[d] = *(const uint4 *)(vp + voff[d]);
    };
    int id = cur.block_id(a);

    half8v qf[NT][ND][2];
    float fac[NT], m[NT], l[NT], vscale;
    int lim[NT];
    float4v acc[NT][DT];
    int row0, cols, col0, before, hi_lim, lo_lim;
    // a new item: its rows and limits, its queries on their way
    auto rows_of = [&](Query<ND> (&raw)[NT]) {
        int n = 1;
        row0 = cur.s;
        if (a.q.row_start) {
            row0 = max(0, min(uniform(a.q.row_start + cur.s), a.q.n_rows));
            n = min(max(row0, min(uniform(a.q.row_start + cur.s + 1), a.q.n_rows)) - row0,
                    a.q.max_new);
        }
        before = max(0, min(uniform(a.q.lengths + cur.s), a.q.max_length)) - n;
        cols = n * a.G;
        col0 = cur.tile * NT * 16;
        hi_lim = before + min(cols - 1, col0 + NT * 16 - 1) / a.G + 1;
        lo_lim = before + col0 / a.G + 1;
        for (int k = 0; k < NT; ++k) {
            const int c = col0 + k * 16 + c16;
            const bool valid = c < cols;
            load_query<ND>(a, row0 + (valid ? c / a.G : 0),
                           cur.h * a.G + (valid ? c % a.G : 0), valid, g, raw[k]);
            lim[k] = valid ? before + c / a.G + 1 : 0;
        }
    };
    auto begin = [&](const Query<ND> (&raw)[NT]) {
        vscale = 1e-38f;                         // the values' common scale so far
        for (int k = 0; k < NT; ++k) {
            fac[k] = query_halves<ND>(a, raw[k], qf[k]) * a.scale;
            m[k] = -__builtin_inff();
            l[k] = 0.f;
            for (int d = 0; d < DT; ++d) acc[k][d] = float4v{0.f, 0.f, 0.f, 0.f};
        }
    };
    Query<ND> raw[NT];
    rows_of(raw);
    int64_t bh = cur.row(a, id);
    load_keys(bh);
    load_values(bh);
    float ksc = uniform(a.ks + bh), vsc = uniform(a.vs + bh);
    Cursor nxt = cur;
    nxt.next(a);
    int id1 = nxt.block_id(a);
    begin(raw);
    int seg0 = u0;                               // first unit of the item at hand

    for (int u = u0; u < u1; ++u) {
        const int s = cur.s, h = cur.h, j = cur.block;
        if (j == 0 && u != u0) {
            seg0 = u;
            Query<ND> raw[NT];
            rows_of(raw);
            begin(raw);
        }
        const bool mapped = (unsigned)id < (unsigned)a.n_blocks, more = u + 1 < u1;
        const int64_t bh1 = nxt.row(a, id1);
        const float ksc1 = uniform(a.ks + bh1), vsc1 = uniform(a.vs + bh1);
        Cursor nxt2 = nxt;
        if (u + 2 < u1) nxt2.next(a);
        const int id2 = nxt2.block_id(a);
        if (!mapped) vsc = 0.f;

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
        if (more) load_keys(bh1);
        const bool masked = (j + 1) * kBlock > lo_lim || !mapped;
        const int slot0 = j * kBlock + 4 * g;    // of tile 0, element 0
        float top[NT];
        bool grow = false;
        for (int k = 0; k < NT; ++k) {
            const float f = fac[k] * ksc;
            top[k] = -__builtin_inff();
            for (int t = 0; t < 4; ++t)
                for (int i = 0; i < 4; ++i) {
                    float x = sc[k][t][i] * f;
                    if (masked && (slot0 + t * 16 + i >= lim[k] || !mapped)) x = -__builtin_inff();
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
                    float *p = a.s + ((((int64_t)s * a.blocks + j) * a.H + h) * min(a.cols, a.few) + c) * kBlock;
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
        const float vrel = vsc / vscale * kRaised;
        half8v pb[NT][2];
        for (int k = 0; k < NT; ++k) {
            const float base = m[k] == -__builtin_inff() ? 0.f : m[k];
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
                    const int left = mapped ? hi_lim - (slot0 + t * 16) : 0;
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
        if (more) load_values(bh1);

        if (!more || j + 1 == cur.nb) {          // the item ends here
            const bool whole = j + 1 == cur.nb && j == u - seg0;
            const int64_t part = 2 * (int64_t)worker + (seg0 == u0 ? 0 : 1);
            for (int k = 0; k < NT; ++k) {
                const float sum = group_sum(l[k]);
                const float inv = sum == 0.f ? 0.f : 1.f / (kRaised * sum);
                const int c = col0 + k * 16 + c16;
                if (c >= cols) continue;
                const int64_t row = row0 + c / a.G;
                const int head = h * a.G + c % a.G;
                if (g == 0) {
                    if (whole)
                        a.done[column(a, h, row, c % a.G)] = finished(m[k], sum);
                    else
                        a.part_ts[part * a.tile + k * 16 + c16] = {m[k], sum};
                }
                for (int d = 0; d < DT; ++d) {
                    if (d * 16 >= D) break;
                    const float4v o = acc[k][d] * inv * vscale;
                    if (!whole) {
                        *(float4v *)(a.part_o + (part * a.tile + k * 16 + c16) * D + d * 16 +
                                     4 * g) = o;
                    } else {
                        uint16_t *p = (uint16_t *)a.od + row * a.o_row + head * a.o_head +
                                      d * 16 + 4 * g;
                        for (int i = 0; i < 4; ++i) p[i] = row_bits(o[i], a.dtype);
                    }
                }
            }
        }
        cur = nxt;
        nxt = nxt2;
        id = id1;
        id1 = id2;
        bh = bh1;
        ksc = ksc1;
        vsc = vsc1;
    }
}

__device__ inline float lane_value(float x, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// Adds up the parts of the columns whose units several workers held, and gives
// the columns that see nothing their zeros: WPC waves to a column, the parts in
// turn.  4.5 us at one sequence, 10 at two whose columns have 512 parts each: the reads
// of the parts, four under way to a wave.
template <int WPC> __global__ __launch_bounds__(kThreads) void k_attend_join(AttnArgs a)
{
    __shared__ float part[kWaves][256], sum[kWaves];
    __shared__ int below[kWaves], total[kWaves];
    constexpr int CPG = kWaves / WPC;            // columns of a workgroup
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int groups = (min(a.cols, a.few) + CPG - 1) / CPG;
    const uint32_t sh = blockIdx.x / (uint32_t)groups;
    const int c = (int)(blockIdx.x % (uint32_t)groups) * CPG + wv / WPC;
    const int s = (int)(sh / (uint32_t)a.H), h = (int)(sh % (uint32_t)a.H);
    // units of the sequences before, and of all
    int lo = 0, all = 0;
    for (int k = threadIdx.x; k < a.q.n_seqs; k += kThreads) {
        const Units u = units_of(a, k);
        const int v = u.nb * u.tiles * a.H;
        all += v;
        lo += k < s ? v : 0;
    }
    for (int o = 32; o; o >>= 1) {
        all += __shfl_xor(all, o);
        lo += __shfl_xor(lo, o);
    }
    if (lane == 0) {
        below[wv] = lo;
        total[wv] = all;
    }
    __syncthreads();
    lo = below[0] + below[1] + below[2] + below[3];
    all = total[0] + total[1] + total[2] + total[3];
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const Units u = units_of(a, s);
    const int each = units_each(a, all);
    const int u0 = lo + (h * u.tiles + c / a.tile) * u.nb, u1 = u0 + u.nb;
    const int w0 = u0 / each, w1 = u.nb ? (u1 - 1) / each : w0 - 1;
    // (whole at one worker: written there)
    const bool mine = c < n * a.G && n * a.G <= a.few && w0 != w1;
    float M = -__builtin_inff(), L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    auto place = [&](int w) {                    // of the part that worker w left
        return (2 * (int64_t)w + (w == w0 && u0 % each ? 1 : 0)) * a.tile + c % a.tile;
    };
    if (mine) {
        for (int w = w0 + lane; w <= w1; w += 64) M = fmaxf(M, a.part_ts[place(w)].top);
        for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
        for (int b = w0 + wv % WPC; b <= w1; b += 4 * WPC) {
            TopSum f[4];
            float x[4][4];
            for (int k = 0; k < 4; ++k) {
                const int64_t at = place(min(b + k * WPC, w1));
                f[k] = a.part_ts[at];
                for (int e = 0; e < 4; ++e)
                    x[k][e] = a.part_o[at * a.D + min(e * 64 + lane, a.D - 1)];
            }
            for (int k = 0; k < 4; ++k) {
                const float z = b + k * WPC > w1 ? 0.f : part_weight(f[k], M);
                L += z;
                for (int e = 0; e < 4; ++e) acc[e] += z == 0.f ? 0.f : z * x[k][e];
            }
        }
    }
    if (WPC > 1) {
        for (int e = 0; e < 4; ++e) part[wv][e * 64 + lane] = acc[e];
        if (lane == 0) sum[wv] = L;
        __syncthreads();
        if (wv % WPC) return;
        L = 0.f;
        for (int e = 0; e < 4; ++e) acc[e] = 0.f;
        for (int k = wv; k < wv + WPC; ++k) {
            L += sum[k];
            for (int e = 0; e < 4; ++e) acc[e] += part[k][e * 64 + lane];
        }
    }
    if (!mine) return;
    const int64_t row = row0 + c / a.G;
    const int head = h * a.G + c % a.G;
    for (int e = 0; e < 4; ++e)
        if (e * 64 + lane < a.D)
            ((uint16_t *)a.od)[row * a.o_row + head * a.o_head + e * 64 + lane] =
                row_bits(L == 0.f ? 0.f : acc[e] / L, a.dtype);
    if (lane == 0)
        a.done[column(a, h, row, c % a.G)] = finished(M, L);
}

// Weights from the scores that k_attend_rows left: a wave to a (sequence,
// block, kv head), a lane to a slot.  After the join, as a probability needs the whole
// sum; 9 us at 48 sequences of up to 4096.
__global__ __launch_bounds__(kThreads) void k_attend_weights(AttnArgs a)
{
    const int lane = threadIdx.x & 63;
    // (fewer than 2^31 waves: checked on the host)
    const uint32_t w = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
    const int h = (int)(w % (uint32_t)a.H);
    const uint32_t sb = w / (uint32_t)a.H;
    const int j = (int)(sb % (uint32_t)a.blocks), s = (int)(sb / (uint32_t)a.blocks);
    if (s >= a.q.n_seqs) return;
    const int len = seq_length(a.q, s);
    if (j * kBlock >= len) return;
    const int id = uniform(a.q.table + s * a.q.table_stride + j);
    if ((unsigned)id >= (unsigned)a.n_blocks) return;
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const int cols = n * a.G;
    if (cols > a.few) return;                    // (k_attend_colsum)
    const float *sc = a.s + (int64_t)w * min(a.cols, a.few) * kBlock + lane;
    const TopSum mine = lane < cols ? a.done[column(a, h, row0, lane)] : TopSum{0.f, 0.f};
    // rows that see the block's first slot (of the others no scores were formed)
    const int c0 = min(max(0, j * kBlock - (len - n)), n) * a.G;
    float sum = 0.f;
#pragma unroll 4
    for (int c = c0; c < cols; ++c)
        sum += __builtin_amdgcn_exp2f(sc[c * kBlock] - lane_value(mine.top, c)) *
               lane_value(mine.sum, c);
    if (j * kBlock + lane >= len) return;
    float *at = a.weight + ((int64_t)id * a.H + h) * kBlock + lane;
    *at = a.decay == 0.f ? sum : a.decay * *at + sum;
}

// -- many query rows --------------------------------------------------------

typedef float float16v __attribute__((ext_vector_type(16)));

// Queries in half precision, dims padded with zeros to whole 64s, in the order of
// the matrix operands (8 dims of a column after the next column's): scaled by a
// power of two where they come in bfloat16 (query_halves), negated where the scale
// of the scores is negative.  A workgroup to 32 columns of a kv head, 8 dims to a thread, which
// pass through shared memory into runs of 512 bytes.  Bound by its bytes; 5 ragged
// prompts of up to 2000, 32 heads of 128 (79 MB) 17 us, 4.7 TB/s; a wave to a
// column, writing runs of 16 bytes, took 43.
constexpr int kQueryCols = 32;

template <int ND> __global__ __launch_bounds__(kThreads) void k_query_half(AttnArgs a)
{
    constexpr int CH = ND * 8;                   // eights of dims, as many lanes to a column
    __shared__ uint4 st[CH][kQueryCols + 1];
    const uint32_t all = (uint32_t)a.q.n_rows * a.G, tiles = (all + kQueryCols - 1) / kQueryCols;
    const uint32_t h = blockIdx.x / tiles, col0 = blockIdx.x % tiles * kQueryCols;
    const bool bf = a.dtype == QLM_BF16;
#pragma unroll
    for (int t = 0; t < CH * kQueryCols / kThreads; ++t) {
        const int i = t * kThreads + threadIdx.x, ch = i % CH, c = i / CH;
        const uint32_t col = min(col0 + c, all - 1), row = col / (uint32_t)a.G;
        const uint16_t *p = (const uint16_t *)a.qd + row * a.q_row +
                            (h * a.G + col % (uint32_t)a.G) * a.q_head + min(8 * ch, a.D - 8);
        uint32_t w[4];
        if (a.wide) {
            const uint4 v = *(const uint4 *)p;
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
            for (int e = 0; e < 4; ++e) w[e] = p[2 * e] | (uint32_t)p[2 * e + 1] << 16;
        }
        for (int e = 0; e < 4; ++e) w[e] = 8 * ch < a.D ? w[e] : 0u;
        float unscale = 1.f, by = a.scale < 0.f ? -1.f : 1.f;
        if (bf) {
            uint32_t top = 0;                    // greatest exponent of a finite element
            for (int e = 0; e < 8; ++e) {
                const uint32_t x = w[e >> 1] >> (16 * (e & 1) + 7) & 0xff;
                top = x < 255 ? max(top, x) : top;
            }
            for (int o = CH / 2; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
            const int up = min(15 - ((int)top - 126), 126);
            by *= ldexpf(1.f, up);
            unscale = ldexpf(1.f, -up);
        }
        for (int e = 0; e < 4; ++e) {
            uint16_t u[2];
            for (int k = 0; k < 2; ++k) {
                const uint16_t b = (uint16_t)(w[e] >> (16 * k));
                const float x = bf ? __builtin_bit_cast(float, (uint32_t)b << 16)
                                   : (float)__builtin_bit_cast(_Float16, b);
                u[k] = __builtin_bit_cast(uint16_t, (_Float16)(x * by));
            }
            w[e] = u[0] | (uint32_t)u[1] << 16;
        }
        st[ch][c] = {w[0], w[1], w[2], w[3]};
        // (a scale of 0: small enough, and no 0 times infinity)
        if (ch == 0 && col0 + c < all)
            a.qfac[(int64_t)h * all + col] = fmaxf(unscale * fabsf(a.scale), 1e-37f);
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < CH * kQueryCols / kThreads; ++t) {
        const int i = t * kThreads + threadIdx.x, c = i % kQueryCols, ch = i / kQueryCols;
        if (col0 + c < all)
            *(uint4 *)(a.qh + (((int64_t)h * CH + ch) * all + col0 + c) * 8) = st[ch][c];
    }
}

// The sequences of many rows: one workgroup to 128 columns (query rows and heads
// of a kv head, 32 a wave) and a split of the keys.  Every block's codes are
// turned into halves once, in shared memory and in the order of the matrix
// operands (two buffers, the next block's codes on their way meanwhile), and
// serve the four waves.  S^T = K Q^T and O^T = V^T P^T are 32x32x16 matrix
// instructions; a lane's scores are again the operand of the second product, so
// only keys and values pass through shared memory.
// Bound by matrix instructions, exponentials and reads of shared memory in turn, two
// waves to a SIMD being all its registers allow: 5 ragged prompts of up to 2000 tokens
// over up to 2600, 32 heads of 128: 170 us, 600 TFLOP/s.
template <int FMT, int ND, bool FULL>
__global__ __launch_bounds__(kThreads, ND <= 2 ? 2 : 1) void k_attend_prompt(AttnArgs a)
{
    constexpr int DP = ND * 64, KS = DP / 16, DT = DP / 32;
    constexpr int KP = kBlock * 8 + 8;               // halves between chunks of 8 dims
    __shared__ uint4 ldsk[2][KS * 2 * KP / 8], ldsv[2][kBlock * DP / 8];
    // blocks j, j + 1, j + 2 in turn: whether any value is not a number, and which
    // slots of a dim are not
    __shared__ int some_nan[3];
    __shared__ unsigned long long nan_at[3][FMT == QLM_KV_E4M3 ? DP : 1];
    const int t = threadIdx.x, lane = t & 63;
    const int wv = __builtin_amdgcn_readfirstlane(t >> 6);
    const int hi = lane >> 5, c32 = lane & 31;
    const uint32_t most = (uint32_t)(a.cols + 127) / 128, heads = (uint32_t)(a.q.n_seqs * a.H);
    // (the last rows see most: they come first, of every sequence)
    const int ct = (int)(most - 1 - blockIdx.x / heads);
    const uint32_t sh = blockIdx.x % heads;
    const int h = (int)(sh % (uint32_t)a.H), s = (int)(sh / (uint32_t)a.H), sp = blockIdx.y;
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const int cols = n * a.G, col0 = ct * 128;
    if (cols <= a.few || col0 >= cols) return;
    const int before = seq_length(a.q, s) - n;
    const int hi_lim = before + min(cols - 1, col0 + 127) / a.G + 1;
    const int lo_lim = before + col0 / a.G + 1;
    const int nb = (max(hi_lim, 0) + kBlock - 1) / kBlock;
    const int b0 = (int)((int64_t)nb * sp / a.splits), b1 = (int)((int64_t)nb * (sp + 1) / a.splits);
    const int wcol0 = col0 + wv * 32, c = wcol0 + c32;
    const int w_hi = before + min(cols - 1, wcol0 + 31) / a.G + 1;   // the wave's limits
    const int w_lo = before + min(cols - 1, wcol0) / a.G + 1;
    const bool valid = c < cols;
    const int64_t all = (int64_t)a.q.n_rows * a.G, rh = column(a, h, row0, valid ? c : 0);
    const int lim = valid ? before + c / a.G + 1 : 0;
    const int D = a.D;

    half8v qf[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
        qf[k] = *(const half8v *)(a.qh + (((int64_t)h * (DP / 8 - 1) + 2 * k + hi) * all + rh) * 8);
    const float fac = a.qfac[rh];
    float16v acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    float m = -__builtin_inff(), l = 0.f, vscale = 1e-38f;

    const int32_t *table = a.q.table + s * a.q.table_stride;
    uint4 kr[ND], vr[ND];
    float ksc = 0.f, vsc = 0.f;
    auto fetch = [&](int j) {
        const int id = uniform(table + j);
        const bool mapped = (unsigned)id < (unsigned)a.n_blocks;
        const int64_t bh = (int64_t)(mapped ? id : 0) * a.H + h;
        const uint8_t *kp = a.kc + bh * kBlock * D, *vp = a.vc + bh * kBlock * D;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int e = t + kThreads * i, tok = e / (DP / 16), ch = e % (DP / 16);
            const int g = e / DP, d = e % DP;
            kr[i] = *(const uint4 *)(kp + (uint32_t)(tok * D + (FULL ? ch * 16
                                                                     : min(ch * 16, D - 16))));
            vr[i] = *(const uint4 *)(vp + (uint32_t)((g * D + (FULL ? d : min(d, D - 1))) * 16));
        }
        ksc = uniform(a.ks + bh);
        vsc = mapped ? uniform(a.vs + bh) : 0.f;
        return mapped;
    };
    auto stage = [&](int buf, int j, bool mapped) {
        _Float16 *ks = (_Float16 *)ldsk[buf], *vs = (_Float16 *)ldsv[buf];
        const bool masked = (j + 1) * kBlock > lo_lim || !mapped;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int e = t + kThreads * i, tok = e / (DP / 16), ch = e % (DP / 16);
            *(half8v *)(ks + (2 * ch) * KP + tok * 8) = halves8<FMT>(kr[i].x, kr[i].y);
            *(half8v *)(ks + (2 * ch + 1) * KP + tok * 8) = halves8<FMT>(kr[i].z, kr[i].w);
            const int g = e / DP, d = e % DP;
            uint32_t x[4] = {vr[i].x, vr[i].y, vr[i].z, vr[i].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (masked) {                    // slots that no column here sees are zeroed
                    const int left = mapped ? hi_lim - (j * kBlock + q * 16 + 4 * g) : 0;
                    x[q] = left <= 0 ? 0u : left < 4 ? x[q] & (0xffffffffu >> (8 * (4 - left)))
                                                     : x[q];
                    const uint32_t z = FMT == QLM_KV_E4M3 ? nan_bytes(x[q]) : 0;
                    if (z) {                     // (taken out here, given to whom sees it below)
                        x[q] &= ~z;
                        some_nan[j % 3] = 1;
                        atomicOr(&nan_at[j % 3][d],
                                 (unsigned long long)((z & 1) | (z >> 7 & 2) | (z >> 14 & 4) |
                                                      (z >> 21 & 8)) << (q * 16 + 4 * g));
                    }
                }
                half2v lo, up;
                halves4<FMT>(x[q], &lo, &up);
                typedef _Float16 half4v __attribute__((ext_vector_type(4)));
                *(half4v *)(vs + ((q * 2 + (g & 1)) * DP + d) * 8 + (g >> 1) * 4) =
                    half4v{lo[0], lo[1], up[0], up[1]};
            }
        }
    };
    auto no_nans = [&](int r) {
        if (t == 0) some_nan[r] = 0;
        if (FMT == QLM_KV_E4M3 && t < DP) nan_at[r][t] = 0;
    };
    for (int r = 0; r < 3; ++r) no_nans(r);
    __syncthreads();
    bool mapped = false;
    if (b0 < b1) {
        mapped = fetch(b0);
        stage(0, b0, mapped);
    }
    __syncthreads();
    for (int j = b0; j < b1; ++j) {
        const int buf = (j - b0) & 1;
        const bool here = mapped;
        const float ks1 = ksc, vs1 = vsc;
        if (j + 1 < b1) mapped = fetch(j + 1);
        if (j * kBlock < w_hi && wcol0 < cols && here) {
            const _Float16 *ks = (const _Float16 *)ldsk[buf], *vs = (const _Float16 *)ldsv[buf];
            float16v sc[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    if (!FULL && k * 16 >= D) break;
                    const half8v x = *(const half8v *)(ks + (2 * k + hi) * KP +
                                                       (u * 32 + c32) * 8);
                    sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, qf[k], sc[u], 0, 0, 0);
                }
            }
            const bool masked = (j + 1) * kBlock > w_lo;
            const int slot0 = j * kBlock + 4 * hi;
            if (masked)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (slot0 + u * 32 + (i & 3) + 8 * (i >> 2) >= lim)
                            sc[u][i] = -__builtin_inff();
            float tops[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                tops[q] = sc[0][q];
#pragma unroll
                for (int i = q + 4; i < 32; i += 4) tops[q] = fmaxf(tops[q], sc[i >> 4][i & 15]);
            }
            float top, other;
            swap32(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), &top, &other);
            // (an unseen slot's -inf is multiplied too: the factor may not vanish, as it
            // would with queries and keys of zeros, both at their least scale.  Scores stay
            // below 2^-80 at the one it is held to)
            const float f = fmaxf(fac * ks1, 1e-37f);
            top = fmaxf(top, other) * f;
            if (__any(top > m + kSlack)) {
                const float mn = fmaxf(m, top);
                const float al = mn == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= al;
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d] *= al;
            }
            if (vs1 > vscale) {                      // (uniform over the wave)
                const float al = vscale / vs1;
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d] *= al;
                vscale = vs1;
            }
            const float vrel = vs1 / vscale * kRaised;
            const float base = m == -__builtin_inff() ? 0.f : m;
            half8v pb[4];
            float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = sc[u][i] * f;
                    const float p = __builtin_amdgcn_exp2f(x - base);
                    sums[i & 3] += p;
                    pb[2 * u + (i >> 3)][i & 7] = (_Float16)(p * vrel);
                }
            l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                if (!FULL && d * 32 >= D) break;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const half8v x = *(const half8v *)(vs + ((q * 2 + hi) * DP + d * 32 + c32) * 8);
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, pb[q], acc[d], 0, 0, 0);
                }
            }
            if (FMT == QLM_KV_E4M3 && some_nan[j % 3]) {
                const int n_seen = min(max(lim - j * kBlock, 0), kBlock);
                const unsigned long long seen = n_seen ? ~0ull >> (kBlock - n_seen) : 0;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (nan_at[j % 3][d * 32 + (i & 3) + 8 * (i >> 2) + 4 * hi] & seen)
                            acc[d][i] = __builtin_nanf("");
            }
        }
        if (j + 1 < b1) stage(buf ^ 1, j + 1, mapped);
        // (read in the last round, set in the next one: a barrier lies on either side)
        if ((j + 2) * kBlock > lo_lim) no_nans((j + 2) % 3);
        __syncthreads();
    }

    float l0, l1;
    swap32(l, &l0, &l1);
    const float sum = l0 + l1, inv = sum == 0.f ? 0.f : 1.f / (kRaised * sum);
    if (!valid) return;
    const int64_t sr = (int64_t)sp * a.q.n_rows * a.H * a.G + rh;
    if (hi == 0) {
        if (a.splits > 1)
            a.split_ts[sr] = {m, sum};
        else
            a.done[rh] = finished(m, sum);
    }
    uint16_t *out = (uint16_t *)a.od + (int64_t)(row0 + c / a.G) * a.o_row +
                    (h * a.G + c % a.G) * a.o_head;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        const float16v o = acc[d] * inv * vscale;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int dim = d * 32 + 8 * q + 4 * hi;
            if (dim >= D) continue;
            if (a.splits > 1) {
                *(float4v *)(a.split_o + sr * D + dim) =
                    float4v{o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]};
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) out[dim + i] = row_bits(o[4 * q + i], a.dtype);
            }
        }
    }
}

// Joins the splits of the keys: a wave to a (row, head) of a sequence of many rows.
__global__ __launch_bounds__(kThreads) void k_prompt_join(AttnArgs a)
{
    const int lane = threadIdx.x & 63, heads = a.H * a.G;
    const int64_t w = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int64_t per = (int64_t)a.q.max_new * heads;
    const int s = (int)(w / per);
    if (s >= a.q.n_seqs) return;
    int row0;
    const int n = seq_rows(a.q, s, &row0), r = (int)(w % per / heads), head = (int)(w % heads);
    if (n * a.G <= a.few || r >= n) return;
    const int64_t rh = column(a, head / a.G, row0 + r, head % a.G);
    const int64_t step = (int64_t)a.q.n_rows * heads;
    float M = -__builtin_inff(), L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < a.splits; ++k) M = fmaxf(M, a.split_ts[rh + k * step].top);
    for (int k = 0; k < a.splits; ++k) {
        const float f = part_weight(a.split_ts[rh + k * step], M);
        L += f;
        for (int e = 0; e < 4; ++e) {
            const float x = a.split_o[(rh + k * step) * a.D + min(e * 64 + lane, a.D - 1)];
            acc[e] += f == 0.f ? 0.f : f * x;
        }
    }
    for (int e = 0; e < 4; ++e)
        if (e * 64 + lane < a.D)
            ((uint16_t *)a.od)[(row0 + r) * a.o_row + head * a.o_head + e * 64 + lane] =
                row_bits(L == 0.f ? 0.f : acc[e] / L, a.dtype);
    if (lane == 0) a.done[rh] = finished(M, L);
}

// Weights of the sequences of many rows: a workgroup to a block of 64 slots of a
// (sequence, kv head).  Its waves hold the block's keys as matrix operands, form
// the scores of the columns that see it again, a wave every fourth 32, the next
// ones' queries on their way meanwhile, and add up their probabilities.  (Kept
// scores would be four bytes for each column and slot, gigabytes of them.)
// No one rate bounds it: for the prompts of k_attend_prompt's figure 129 us, of which the
// product would take 42 at a large product's rate and the 201 million exponentials some 20;
// a wave forms product, exponentials and sums in turn, two waves to a SIMD, and every
// workgroup reads its columns' queries from L2 again (0.8 GB in all).
template <int FMT, int ND>
__global__ __launch_bounds__(kThreads, ND <= 2 ? 2 : 1) void k_attend_colsum(AttnArgs a)
{
    __shared__ float part[kWaves][kBlock];
    constexpr int DP = ND * 64, KS = DP / 16;
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hi = lane >> 5, c32 = lane & 31;
    uint32_t at = blockIdx.x;
    const int j = (int)(at % (uint32_t)a.blocks);
    at /= (uint32_t)a.blocks;
    const int h = (int)(at % (uint32_t)a.H), s = (int)(at / (uint32_t)a.H);
    int row0;
    const int n = seq_rows(a.q, s, &row0), len = seq_length(a.q, s);
    const int cols = n * a.G, before = len - n, D = a.D;
    if (cols <= a.few || j * kBlock >= len) return;
    const int id = uniform(a.q.table + s * a.q.table_stride + j);
    if ((unsigned)id >= (unsigned)a.n_blocks) return;
    const int64_t bh = (int64_t)id * a.H + h;
    half8v kf[2][KS];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            // (dims past the last: their query is 0)
            const uint2 x = *(const uint2 *)(a.kc + (bh * kBlock + u * 32 + c32) * D +
                                             min(k * 16 + hi * 8, D - 8));
            kf[u][k] = halves8<FMT>(x.x, x.y);
        }
    const float ksc = uniform(a.ks + bh);
    const int slot0 = j * kBlock + 4 * hi;
    float16v sum[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[u][i] = 0.f;
    const int64_t all = (int64_t)a.q.n_rows * a.G, base = column(a, h, row0, 0);
    const half8v *qp = (const half8v *)a.qh + ((int64_t)h * (DP / 8 - 1) + hi) * all + base;
    half8v qn[KS];
    float facn;
    TopSum tsn;
    auto fetch = [&](int ct) {                   // (past the last column it is read again)
        const int c = min(ct * 32 + c32, cols - 1);
#pragma unroll
        for (int k = 0; k < KS; ++k) qn[k] = qp[2 * k * all + c];
        facn = a.qfac[base + c];
        tsn = a.done[base + c];
    };
    const int first = max(0, j * kBlock - before) * a.G / 32;   // tile that sees the first slot
    const int tiles = (cols + 31) / 32, step = kWaves * a.shares;
    const int from = first + wv + kWaves * (int)blockIdx.y;
    fetch(min(from, tiles - 1));
    for (int ct = from; ct < tiles; ct += step) {
        half8v qf[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[k] = qn[k];
        const int c = ct * 32 + c32;
        const float fac = facn * ksc;
        const TopSum ts = c < cols ? tsn : TopSum{0.f, 0.f};
        fetch(min(ct + step, tiles - 1));
        const bool masked = (j + 1) * kBlock > before + ct * 32 / a.G + 1 || ct + 1 == tiles;
        const int lim = masked && c < cols ? before + c / a.G + 1 : 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float16v sc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k)
                sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[u][k], qf[k], sc, 0, 0, 0);
            if (masked)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = sc[i] * fac;
                    const float p = __builtin_amdgcn_exp2f(x - ts.top) * ts.sum;
                    sum[u][i] += slot0 + u * 32 + (i & 3) + 8 * (i >> 2) < lim ? p : 0.f;
                }
            else
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = sc[i] * fac;
                    sum[u][i] = fmaf(__builtin_amdgcn_exp2f(x - ts.top), ts.sum, sum[u][i]);
                }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float x = sum[u][i];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) x += __shfl_xor(x, o);
            const int slot = u * 32 + (i & 3) + 8 * (i >> 2) + 4 * hi;
            if (c32 == 0) part[wv][slot] = x;
        }
    __syncthreads();
    const int slot = threadIdx.x;
    if (slot >= kBlock || j * kBlock + slot >= len) return;
    const float x = (part[0][slot] + part[1][slot]) + (part[2][slot] + part[3][slot]);
    if (a.shares > 1) {
        const int64_t all = (int64_t)a.q.n_seqs * a.blocks * a.H;
        a.share[((blockIdx.y * all) + ((int64_t)s * a.blocks + j) * a.H + h) * kBlock + slot] = x;
    } else {
        float *w = a.weight + bh * kBlock + slot;
        *w = a.decay == 0.f ? x : a.decay * *w + x;
    }
}

// Adds up the shares of the columns: a wave to a (sequence, block, kv head), a
// lane to a slot.
__global__ __launch_bounds__(kThreads) void k_colsum_join(AttnArgs a)
{
    const int lane = threadIdx.x & 63;
    const uint32_t w = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
    const int h = (int)(w % (uint32_t)a.H);
    const uint32_t sb = w / (uint32_t)a.H;
    const int j = (int)(sb % (uint32_t)a.blocks), s = (int)(sb / (uint32_t)a.blocks);
    if (s >= a.q.n_seqs) return;
    int row0;
    const int len = seq_length(a.q, s);
    if (seq_rows(a.q, s, &row0) * a.G <= a.few || j * kBlock + lane >= len) return;
    const int id = uniform(a.q.table + s * a.q.table_stride + j);
    if ((unsigned)id >= (unsigned)a.n_blocks) return;
    const int64_t all = (int64_t)a.q.n_seqs * a.blocks * a.H;
    float x = 0.f;
    for (int k = 0; k < a.shares; ++k) x += a.share[(k * all + w) * kBlock + lane];
    float *at = a.weight + ((int64_t)id * a.H + h) * kBlock + lane;
    *at = a.decay == 0.f ? x : a.decay * *at + x;
}

// -- host -------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Columns of a sequence that k_attend_rows takes: it reads the keys and values again for
// every 32, k_attend_prompt for every 128 but turns every block's codes for them.  At
// 4096 tokens and 16 sequences, 32 columns 38 us to the other's 69, 64 58 to 65, 128 94
// to 69; 64 sequences of 2048, 64 columns 96 to 118, 96 156 to 106.
constexpr int kFew = 64;
// Waves of k_attend_rows: one to a SIMD, for its many loads under way are enough and
// each wave leaves parts to join (a sequence of 65536 tokens 38 us, two to a SIMD 44; 64 of
// 4096 103 and 107).  Two where a wave has less under way (64 dims) or writes scores,
// and the items are many: 64 of 4096 at 64 dims 57 us, one to a SIMD 71; 48 ragged
// ones with weights 81 and 89.
constexpr int kWorkers = 1024, kManyItems = 128;

// Scores held at once where prompts and few rows share a call.  A sequence of few rows
// then has room for kFew columns in every block up to the longest one's, whatever it uses:
// 192 sequences of 16000 slots beside a prompt would need 6.4 GB.  The sequences go in as many
// passes as the scores do; a pass costs some 35 us (that call, 64 heads: 1466 us in one, 1502
// in two, 1535 in three; 128 of 12000, 32 heads, 3.2 GB: 688 in one, 729 in two).
constexpr int64_t kScoreBytes = 4ll << 30;

struct Plan {
    int nt, tile, workers, cols, blocks, splits, shares;
    int at_once;                 // sequences of few rows in a pass
    bool few, many;              // which sequences there can be
    size_t part_o, part_ts, done, s, qh, qfac, split_o, split_ts, share, total;
};

Plan plan_of(const qlm_kv_cache *c, const qlm_kv_batch *b, int32_t n_heads, bool weights)
{
    Plan p{};
    const int64_t cols = (int64_t)b->max_new * (n_heads / c->n_kv_heads);
    p.cols = (int)std::min<int64_t>(cols, INT32_MAX);
    p.many = cols > kFew;
    p.few = !p.many || b->n_rows != (int64_t)b->n_seqs * b->max_new;
    p.nt = cols <= 16 || c->head_dim > 128 ? 1 : 2;      // (two would not fit the registers)
    p.tile = 16 * p.nt;
    p.blocks = std::max(1, (b->max_length + kBlock - 1) / kBlock);
    const bool twice = (weights || c->head_dim <= 64) && c->head_dim <= 128 && p.nt == 1 &&
                       (int64_t)b->n_seqs * c->n_kv_heads >= kManyItems;
    p.workers = twice ? 2 * kWorkers : kWorkers;
    p.at_once = b->n_seqs;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    p.done = take((size_t)b->n_rows * n_heads * sizeof(TopSum));
    if (p.few) {
        p.part_o = take((size_t)2 * p.workers * p.tile * c->head_dim * 4);
        p.part_ts = take((size_t)2 * p.workers * p.tile * sizeof(TopSum));
        if (weights) {
            const int64_t one = (int64_t)p.blocks * c->n_kv_heads * std::min(p.cols, kFew) * kBlock * 4;
            if (p.many)
                p.at_once = (int)std::max<int64_t>(1, std::min<int64_t>(b->n_seqs, kScoreBytes / one));
            p.s = take((size_t)p.at_once * one);
        }
    }
    p.splits = 1;
    if (p.many) {
        // two workgroups to a CU; three blocks to a split at least (one prompt of 571
        // tokens over 10 blocks: 11 us and 4 for the join, 25 in one)
        const int64_t wg = ((int64_t)b->n_rows * n_heads + 127) / 128;
        p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(wg, 1),
                                                               p.blocks / 3));
        const size_t rh = (size_t)b->n_rows * n_heads;
        p.qh = take(rh * ((c->head_dim + 63) / 64 == 3 ? 4 : (c->head_dim + 63) / 64) * 128);
        p.qfac = take(rh * 4);
        if (p.splits > 1) {
            p.split_o = take(rh * p.splits * c->head_dim * 4);
            p.split_ts = take(rh * p.splits * sizeof(TopSum));
        }
        if (weights) {
            // a block's columns shared where the blocks are few, 2048 columns to a
            // workgroup at least: shares against none, one prompt of 1024 tokens 85 us to
            // 93, of 8192 1194 to 1351, two of 1024 over 2 kv heads 70 to 99, four of 2048
            // 437 to 415; at 512 columns the prompt of 2048 took 192 in place of 153
            const int64_t sbh = (int64_t)b->n_seqs * p.blocks * c->n_kv_heads;
            p.shares = (int)std::max<int64_t>(1, std::min(4096 / sbh, cols / 2048));
            if (p.shares > 1) p.share = take((size_t)p.shares * sbh * kBlock * 4);
        }
    }
    p.total = at;
    return p;
}

template <int FMT, int ND, int NT> void launch_rows(const AttnArgs &a, int64_t grid, hipStream_t st)
{
    k_attend_rows<FMT, ND, NT><<<(unsigned)grid, kThreads, 0, st>>>(a);
}

template <int FMT> void launch_rows(const AttnArgs &a, int nt, int64_t grid, hipStream_t st)
{
    if (a.D <= 64)
        nt == 1 ? launch_rows<FMT, 1, 1>(a, grid, st) : launch_rows<FMT, 1, 2>(a, grid, st);
    else if (a.D <= 128)
        nt == 1 ? launch_rows<FMT, 2, 1>(a, grid, st) : launch_rows<FMT, 2, 2>(a, grid, st);
    else
        launch_rows<FMT, 4, 1>(a, grid, st);
}

template <int FMT, int ND> void launch_prompt(const AttnArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.q.n_seqs * a.H * ((a.cols + 127) / 128)), a.splits);
    if (a.D == ND * 64)
        k_attend_prompt<FMT, ND, true><<<grid, kThreads, 0, st>>>(a);
    else
        k_attend_prompt<FMT, ND, false><<<grid, kThreads, 0, st>>>(a);
}

template <int ND> void launch_many(const AttnArgs &a, bool e4m3, hipStream_t st)
{
    const int64_t tiles = ((int64_t)a.q.n_rows * a.G + kQueryCols - 1) / kQueryCols;
    k_query_half<ND><<<(unsigned)(tiles * a.H), kThreads, 0, st>>>(a);
    if (e4m3)
        launch_prompt<QLM_KV_E4M3, ND>(a, st);
    else
        launch_prompt<QLM_KV_INT8, ND>(a, st);
}

template <int ND> void launch_colsum(const AttnArgs &a, bool e4m3, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.q.n_seqs * a.H * a.blocks), a.shares);
    if (e4m3)
        k_attend_colsum<QLM_KV_E4M3, ND><<<grid, kThreads, 0, st>>>(a);
    else
        k_attend_colsum<QLM_KV_INT8, ND><<<grid, kThreads, 0, st>>>(a);
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
    a.tile = p.tile;
    a.workers = p.workers;
    a.cols = p.cols;
    a.blocks = p.blocks;
    char *base = (char *)ws;
    a.part_o = (float *)(base + p.part_o);
    a.part_ts = (TopSum *)(base + p.part_ts);
    a.done = (TopSum *)(base + p.done);
    a.s = query->accumulate && p.few ? (float *)(base + p.s) : nullptr;
    a.few = kFew;
    a.qh = (uint16_t *)(base + p.qh);
    a.qfac = (float *)(base + p.qfac);
    a.splits = p.splits;
    a.split_o = (float *)(base + p.split_o);
    a.split_ts = (TopSum *)(base + p.split_ts);
    a.shares = p.shares;
    a.share = (float *)(base + p.share);
    a.decay = query->weight_decay;

    const bool e4m3 = cache->format == QLM_KV_E4M3;
    const int64_t sh = (int64_t)batch->n_seqs * a.H;
    if ((int64_t)batch->max_new * a.G > (1 << 30))
        return fail(QLM_ERR_CAPACITY, "too many query rows and heads in one sequence");
    const int64_t few = std::min(p.cols, kFew);
    const int64_t units = sh * ((few + p.tile - 1) / p.tile) * p.blocks;
    if (units > INT32_MAX || sh * few > INT32_MAX ||
        sh * (((int64_t)p.cols + 127) / 128) > INT32_MAX || sh * p.blocks > INT32_MAX ||
        (int64_t)batch->max_new * batch->n_seqs * query->n_heads > INT32_MAX ||
        (int64_t)batch->n_rows * query->n_heads > INT32_MAX)
        return fail(QLM_ERR_CAPACITY, "too many rows or blocks in one call");
    const bool weights = query->accumulate && batch->max_length > 0;
    const int64_t row_groups = ((int64_t)batch->n_rows * a.G + kQueryCols - 1) / kQueryCols;
    const int64_t joined = (int64_t)batch->n_seqs * batch->max_new * query->n_heads;
    if ((p.few && !can_launch(sh * ((few + kWaves - 1) / kWaves), kThreads)) ||
        (p.few && weights && !can_launch((sh * p.blocks + kWaves - 1) / kWaves, kThreads)) ||
        (p.many && batch->n_rows > 0 &&
         (!can_launch(row_groups * a.H, kThreads) ||
          !can_launch(sh * (((int64_t)p.cols + 127) / 128), kThreads) ||
          (p.splits > 1 && !can_launch((joined + kWaves - 1) / kWaves, kThreads)) ||
          (weights && !can_launch(sh * p.blocks, kThreads)))))
        return fail(QLM_ERR_CAPACITY, "too many rows or blocks in one call: a launch of 2^32 threads");
    hipError_t e;
    for (int s0 = 0; p.few && s0 < batch->n_seqs; s0 += p.at_once) {
        AttnArgs f = a;                          // the pass's sequences
        f.q.n_seqs = std::min(p.at_once, batch->n_seqs - s0);
        if (s0 > 0) {                            // (rows are counted through row_start then)
            f.q.table += s0 * f.q.table_stride;
            f.q.lengths += s0;
            f.q.row_start += s0;
        }
        const int64_t fh = (int64_t)f.q.n_seqs * a.H;
        if (batch->n_rows > 0) {
            const int64_t fu = fh * ((few + p.tile - 1) / p.tile) * p.blocks;
            const int64_t wg = (std::min<int64_t>(p.workers, fu) + kWaves - 1) / kWaves;
            if (e4m3)
                launch_rows<QLM_KV_E4M3>(f, p.nt, wg, stream);
            else
                launch_rows<QLM_KV_INT8>(f, p.nt, wg, stream);
            if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_attend_rows launch");
            // few columns: a workgroup to each, as their parts may be many (32 columns of
            // 16384 tokens: 26 us with the rows, a wave to each 55; 512 columns 31 and 33;
            // 4096 columns 61 and 53)
            if (fh * few <= 1024)
                k_attend_join<kWaves><<<(unsigned)(fh * few), kThreads, 0, stream>>>(f);
            else
                k_attend_join<1><<<(unsigned)(fh * ((few + kWaves - 1) / kWaves)), kThreads, 0,
                                   stream>>>(f);
            if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_attend_join launch");
        }
        if (weights) {
            k_attend_weights<<<(unsigned)((fh * p.blocks + kWaves - 1) / kWaves), kThreads, 0,
                               stream>>>(f);
            if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_attend_weights launch");
        }
    }
    if (batch->n_rows > 0 && p.many) {
        a.D <= 64 ? launch_many<1>(a, e4m3, stream)
                  : a.D <= 128 ? launch_many<2>(a, e4m3, stream) : launch_many<4>(a, e4m3, stream);
        if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_attend_prompt launch");
        if (p.splits > 1) {
            const int64_t w = (int64_t)batch->n_seqs * batch->max_new * query->n_heads;
            k_prompt_join<<<(unsigned)((w + kWaves - 1) / kWaves), kThreads, 0, stream>>>(a);
            if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_prompt_join launch");
        }
    }
    if (weights && p.many && batch->n_rows > 0) {
        a.D <= 64 ? launch_colsum<1>(a, e4m3, stream)
                  : a.D <= 128 ? launch_colsum<2>(a, e4m3, stream)
                               : launch_colsum<4>(a, e4m3, stream);
        if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_attend_colsum launch");
        if (p.shares > 1) {
            k_colsum_join<<<(unsigned)((sh * p.blocks + kWaves - 1) / kWaves), kThreads, 0,
                            stream>>>(a);
            if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_colsum_join launch");
        }
    }
    return QLM_OK;
}

}  // extern "C"

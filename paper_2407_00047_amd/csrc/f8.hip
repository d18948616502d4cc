// f8.hip -- products in 8-bit floating point with a scale for each block of 128
// inputs (qlm_f8_pack, qlm_f8_rows, qlm_f8_matmul; the definitions stand in
// include/qlm.h).
//
// One matrix instruction (16x16x128) takes a tile's whole block of inputs, so a block's sum of
// products comes out unscaled, and the output adds it times x_scale w_scale in single
// precision.  The instruction itself adds the products of eight neighbouring inputs with 13 bits
// below the largest one's exponent and everything further in single precision; the one of 32 inputs
// does the same at half the rate, so there is no exacter one in 8 bits: 1.5e-5 to 3e-5 of
// the outputs' norm (normal inputs, 512 to 16384 of them, no bias), a hundredth of bfloat16's
// rounding.  Weights are the instruction's first
// operand and rows its second: lane l holds row l % 16 and inputs 32 (l / 16) + 0..31 of both,
// of the result outputs 4 (l / 16) + 0..3 of row l % 16 -- a row's scale is one value a lane.
// In a tile's bytes [8][16][16] chunk c of 16 inputs may stand for any inputs, as long as rows and
// weights agree: lane l takes the chunks l / 16 and 4 + l / 16 of its row, 16 bytes
// each, so that a wave reads 1024 bytes in a row.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "f8_plan.h"
#include "internal.h"
#include "qlm.h"

namespace {

using qlm_internal::fail;
using qlm_internal::hip_fail;

typedef float float4v __attribute__((ext_vector_type(4)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));

using qlm_f8_host::fits;
using qlm_f8_host::kBlock;
using qlm_f8_host::kCus;
using qlm_f8_host::kTile;
using qlm_f8_host::parts_of;
using qlm_f8_host::Plan;
static_assert(kBlock == QLM_F8_BLOCK && kTile == QLM_F8_TILE, "the header's sizes");
constexpr int kTileBytes = kBlock * kTile;
constexpr int kLeastExp = -100;
constexpr int kMost = 1 << 24;

int64_t blocks_of(int n) { return ((int64_t)n + kBlock - 1) / kBlock; }
int64_t tiles_of(int n) { return ((int64_t)n + kTile - 1) / kTile; }
bool can_launch(int64_t groups, int threads) { return groups < (1ll << 32) / threads; }

// -- laying out ---------------------------------------------------------------

struct PackArgs {
    const uint8_t *codes;
    const float *scale;
    uint8_t *packed;
    float *packed_scale;          // [block of outputs][block of inputs], behind the codes
    int32_t N, K, blocks;
    int32_t wide, words;          // 16 codes of a row, or four, may be read at once
    int64_t chunks, scales;
};

// A thread for 16 codes.  Done once for a matrix: 16384 x 4096 25 us, 5.3 TB/s; rows of 5000 codes,
// read four at a time, 20001 of them in 42 us.
__global__ __launch_bounds__(256) void k_f8_pack(PackArgs a)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at < a.scales) a.packed_scale[at] = a.scale[at];
    if (at >= a.chunks) return;
    const int r = (int)(at & 15), c = (int)(at >> 4) & 7;
    const int64_t tile = at >> 7;
    const int64_t n = tile / a.blocks * kTile + r;
    const int64_t k = tile % a.blocks * kBlock + 16 * c;
    uint4 w = {0, 0, 0, 0};
    if (n < a.N && k < a.K) {
        const uint8_t *p = a.codes + n * a.K + k;
        if (a.wide) {
            w = *(const uint4 *)p;
        } else {
            uint32_t u[4] = {0, 0, 0, 0};
            const int have = min(16, (int)(a.K - k));
            if (a.words) {                     // (their number is one of fours)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = 4 * e < have ? ((const uint32_t *)p)[e] : 0u;
            } else {
                for (int e = 0; e < have; ++e) u[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
            }
            w = uint4{u[0], u[1], u[2], u[3]};
        }
    }
    *(uint4 *)(a.packed + 16 * at) = w;
}

struct RowsArgs {
    const uint16_t *x;
    uint8_t *codes;
    float *scale;
    int64_t x_stride, tiles;      // tiles: rows' tiles times blocks
    int32_t M, K, blocks, padded; // padded: rows with the last tile's
    int32_t bf, wide;
};

// A wave for a tile, eight lanes for a row of it: 16 inputs a lane, the largest magnitude over
// the eight, and 16 codes a lane (eight rows of a chunk fill a line of memory).  Bound by memory:
// 8000 rows of 16384 73 us, 5.4 TB/s; one row of 4096 3.7 us, a launch.  Rows that do not all start on
// 16 bytes are read two bytes at a time: 8000 of 16383 245 us, one of 4095 4.8.
template <bool BF> __global__ __launch_bounds__(256) void k_f8_rows(RowsArgs a)
{
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= a.tiles) return;
    const int lane = threadIdx.x & 63, c = lane & 7;
    const int64_t rt = tile / a.blocks;
    const int b = (int)(tile % a.blocks);
    const int k = b * kBlock + 16 * c;
    uint32_t w[2][8];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int64_t row = rt * kTile + 8 * p + (lane >> 3);
        const uint16_t *x = a.x + row * a.x_stride + k;
        const bool in = row < a.M;
        if (a.wide && k + 16 <= a.K) {
            uint4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
            if (in) lo = ((const uint4 *)x)[0], hi = ((const uint4 *)x)[1];
            w[p][0] = lo.x, w[p][1] = lo.y, w[p][2] = lo.z, w[p][3] = lo.w;
            w[p][4] = hi.x, w[p][5] = hi.y, w[p][6] = hi.z, w[p][7] = hi.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t lo = in && k + 2 * e < a.K ? x[2 * e] : 0u;
                const uint32_t hi = in && k + 2 * e + 1 < a.K ? x[2 * e + 1] : 0u;
                w[p][e] = lo | hi << 16;
            }
        }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
        uint32_t top = 0;                       // magnitudes order as integers
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t m = (w[p][e >> 1] >> (16 * (e & 1))) & 0x7fffu;
            top = max(top, m < kInf ? m : 0u);
        }
        for (int o = 1; o < 8; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        auto value = [](uint32_t u) {
            if (BF) return __builtin_bit_cast(float, u << 16);
            return (float)__builtin_bit_cast(_Float16, (uint16_t)u);
        };
        const float m = value(top);
        // m = f 2^e with f in [0.5, 1); 448 = 0.875 2^9
        int e = kLeastExp;
        if (m > 0.f) {
            int q;
            const float f = frexpf(m, &q);
            e = max(kLeastExp, q - 9 + (f > 0.875f ? 1 : 0));
        }
        const float by = ldexpf(1.f, -e);       // (e < 120: a power of two, no quotient needed)
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = value((w[p][2 * i + (j >> 1)] >> (16 * (j & 1))) & 0xffffu) * by;
                y[j] = v > 448.f ? 448.f : v < -448.f ? -448.f : v;   // (a NaN stays)
            }
            int d = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], d, true);
        }
        const int r = 8 * p + (lane >> 3);
        *(uint4 *)(a.codes + tile * kTileBytes + c * 256 + r * 16) = uint4{o[0], o[1], o[2], o[3]};
        if (c == 0) a.scale[(int64_t)b * a.padded + rt * kTile + r] = ldexpf(1.f, e);
    }
}

// -- products -----------------------------------------------------------------

struct MatArgs {
    const uint8_t *w, *x;
    const float *ws, *xs;
    void *out;
    int64_t out_stride;
    int32_t N, M, blocks, padded;
    int32_t n_tiles, m_tiles;
    uint32_t grid_n, grid_m;      // workgroups' tiles of outputs and of rows
    int32_t out_wide;             // rows of out may be written 16 bytes at a time
    int32_t out_past;             // ... past the caches
    // the blocks of inputs in `splits` runs of `per_split`, whose sums stand out_split apart
    int32_t splits, per_split;
    int64_t out_split;
    int32_t dtype;
};

// A lane's 32 bytes of a tile.
__device__ inline int8v operand(const uint8_t *tile, int lane)
{
    const int4v lo = *(const int4v *)(tile + 16 * lane);
    const int4v hi = *(const int4v *)(tile + 1024 + 16 * lane);
    return int8v{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// The sum over a block: weights times rows, both e4m3 without scales.
__device__ inline float4v product(int8v w, int8v x)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, float4v{0, 0, 0, 0}, 0, 0, 0, 0,
                                                            0, 0);
}

__device__ inline uint32_t out_bits(float v, int dtype)
{
    if (dtype == QLM_BF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// Four outputs of a row from n on; those past the last output are not written.
__device__ inline void store4(const MatArgs &a, int64_t m, int n, float4v v)
{
    if (a.dtype == QLM_F32) {
        float *p = (float *)a.out + m * a.out_stride + n;
        for (int i = 0; i < 4; ++i)
            if (n + i < a.N) p[i] = v[i];
        return;
    }
    uint16_t *p = (uint16_t *)a.out + m * a.out_stride + n;
    if (n + 4 <= a.N && (uintptr_t)p % 8 == 0) {
        const uint32_t lo = out_bits(v[0], a.dtype) | out_bits(v[1], a.dtype) << 16;
        const uint32_t hi = out_bits(v[2], a.dtype) | out_bits(v[3], a.dtype) << 16;
        *(uint2 *)p = uint2{lo, hi};
        return;
    }
    for (int i = 0; i < 4; ++i)
        if (n + i < a.N) p[i] = (uint16_t)out_bits(v[i], a.dtype);
}

// NT tiles of outputs and MT of rows to a workgroup, its W waves taking the blocks of inputs in turn,
// U of them loaded at once.  Nothing is shared but the sums, so there is no barrier to wait at while
// loads are under way.  1 row, 4096 x 4096: 4.7 us, 3.6 TB/s, of which 2 to 3 a launch takes; 64 rows,
// 16384 x 4096: 15.3 us (18.5 by 1 x 4 tiles with the groups of rows behind all outputs).
template <int NT, int MT, int W, int U> __global__ __launch_bounds__(64 * W) void k_f8_thin(MatArgs a)
{
    // sums of few tiles are held of every wave, of more of half of them at a time
    constexpr int TILES = NT * MT, HELD = TILES <= 2 ? W : W / 2;
    __shared__ float4v part[HELD][TILES][64];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t across = (uint32_t)(a.n_tiles + NT - 1) / NT;
    // (groups of rows beside the same outputs on one of eight dies, one behind the other)
    const uint32_t groups = (uint32_t)(a.m_tiles + MT - 1) / MT, turn = blockIdx.x / 8;
    const uint32_t run = turn / groups * 8 + blockIdx.x % 8;
    if (run >= across) return;
    const int nt0 = (int)run * NT, mt0 = (int)(turn % groups) * MT;
    float4v acc[NT][MT];
    const uint8_t *w[NT], *x[MT];
    const float *ws[NT], *xs[MT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int nt = min(nt0 + n, a.n_tiles - 1);
        w[n] = a.w + (int64_t)nt * a.blocks * kTileBytes;
        ws[n] = a.ws + (int64_t)(nt / (kBlock / kTile)) * a.blocks;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int mt = min(mt0 + i, a.m_tiles - 1);
        x[i] = a.x + (int64_t)mt * a.blocks * kTileBytes;
        xs[i] = a.xs + mt * kTile + (lane & 15);
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][i] = float4v{0, 0, 0, 0};
    }
    for (int b0 = wv; b0 < a.blocks; b0 += U * W) {
        int8v wo[U][NT], xo[U][MT];
        float s[U][NT], t[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (past the last block it is read again and not used)
            const int b = min(b0 + u * W, a.blocks - 1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                wo[u][n] = operand(w[n] + (int64_t)b * kTileBytes, lane);
                s[u][n] = ws[n][b];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                xo[u][i] = operand(x[i] + (int64_t)b * kTileBytes, lane);
                t[u][i] = xs[i][(int64_t)b * a.padded];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b0 + u * W >= a.blocks) break;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const float4v c = product(wo[u][n], xo[u][i]);
                    const float by = s[u][n] * t[u][i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[n][i][j] += by * c[j];
                }
        }
    }
    auto store = [&](int k, float4v v) {
        const int64_t m = (int64_t)(mt0 + k % MT) * kTile + (lane & 15);
        if (m < a.M) store4(a, m, (nt0 + k / MT) * kTile + 4 * (lane >> 4), v);
    };
    if constexpr (HELD == W) {
#pragma unroll
        for (int k = 0; k < TILES; ++k) part[wv][k][lane] = acc[k / MT][k % MT];
        __syncthreads();
        for (int k = wv; k < TILES; k += W) {
            float4v v = part[0][k][lane];
#pragma unroll
            for (int i = 1; i < W; ++i) v += part[i][k][lane];
            store(k, v);
        }
        return;
    }
#pragma unroll
    for (int half = HELD; half >= 1; half /= 2) {
        if (wv >= half && wv < 2 * half)
#pragma unroll
            for (int k = 0; k < TILES; ++k) part[wv - half][k][lane] = acc[k / MT][k % MT];
        __syncthreads();
        if (half > 1 && wv < half)
#pragma unroll
            for (int k = 0; k < TILES; ++k) acc[k / MT][k % MT] += part[wv][k][lane];
        if (half > 1) __syncthreads();
    }
    // the last pair's sums by all waves
    static_assert(HELD >= 2, "room for the other of the last pair");
    if (wv == 0)
#pragma unroll
        for (int k = 0; k < TILES; ++k) part[1][k][lane] = acc[k / MT][k % MT];
    __syncthreads();
    for (int k = wv; k < TILES; k += W) store(k, part[1][k][lane] + part[0][k][lane]);
}

// 16 bytes a lane from a buffer into shared memory, lane after lane from `to` on (uniform over the
// wave); done when the loads are waited for.
__device__ inline void load_lds(__amdgpu_buffer_rsrc_t from, int at, int lane_at, uint8_t *to)
{
    typedef uint32_t __attribute__((address_space(3))) *shared_ptr;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (shared_ptr)(uintptr_t)to, 16, lane_at, at, 0,
                                             0);
}

// Waits until at most N of the wave's memory operations are under way.
template <int N> __device__ inline void wait_loads()
{
    static_assert(N < 64, "the counter's bits");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4 | 15 << 8);
}

// 16 rows of NT tiles of outputs, turned in shared memory so that a row's outputs are stored side by
// side: 16 bytes a lane where rows and outputs are whole, else an output a lane.  `lds`: 16 rows of
// the wave's own, a row's 16-byte pieces p at p ^ row.  v[i] is of the (i + first)-th tile.
template <int NT, typename T>
__device__ inline void store_rows(const MatArgs &a, int split, int64_t m0, int n0,
                                  const float4v *v, int first, uint8_t *lds)
{
    constexpr int ROW = 16 * NT * sizeof(T), CHUNKS = ROW / 16, MASK = (CHUNKS < 16 ? CHUNKS : 16) - 1;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane)::"memory");   // (places that depend on it are not kept from tile to tile)
    const int r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int at = (16 * ((i + first) % NT) + 4 * q) * sizeof(T);
        uint8_t *to = lds + r * ROW + ((at / 16) ^ (r & MASK)) * 16 + at % 16;
        if constexpr (sizeof(T) == 4) {
            *(float4v *)to = v[i];
        } else {
            *(uint2 *)to = uint2{out_bits(v[i][0], a.dtype) | out_bits(v[i][1], a.dtype) << 16,
                                 out_bits(v[i][2], a.dtype) | out_bits(v[i][3], a.dtype) << 16};
        }
    }
    asm volatile("" ::: "memory");         // (written and read as different types)
    const int rows = (int)min((int64_t)kTile, a.M - m0);
    T *out = (T *)a.out + split * a.out_split + m0 * a.out_stride + n0;
    if (a.out_wide && n0 + 16 * NT <= a.N) {
        constexpr int PER = 64 / CHUNKS;
        const int c = lane % CHUNKS;
#pragma unroll
        for (int k = 0; k < kTile; k += PER) {
            const int row = k + lane / CHUNKS;
            const uint4 w = *(const uint4 *)(lds + row * ROW + (c ^ (row & MASK)) * 16);
            int4v *to = (int4v *)((uint8_t *)(out + row * a.out_stride) + 16 * c);
            const int4v v4 = {(int)w.x, (int)w.y, (int)w.z, (int)w.w};
            if (row >= rows) continue;
            if (a.out_past)
                __builtin_nontemporal_store(v4, to);
            else
                *to = v4;
        }
        return;
    }
#pragma unroll 4
    for (int row = 0; row < rows; ++row)
#pragma unroll
        for (int k = 0; k < 16 * NT; k += 64) {
            const int e = k + lane, at = e * sizeof(T);
            if (e < 16 * NT && n0 + e < a.N)
                out[row * a.out_stride + e] =
                    *(const T *)(lds + row * ROW + ((at / 16) ^ (row & MASK)) * 16 + at % 16);
        }
}

// Tiles of (16 NT WN) outputs and (16 MT WM) rows to a workgroup of WN x WM waves, which takes one
// after another.
// 8192 x 16384 x 4096 by tiles of 256: 464 us, 2370 TFLOP/s (a library's product with one scale for
// everything, which needs no additions outside the matrix instructions, 439).  The matrix instructions
// alone would take 260 at the 2.0 GHz that the chip keeps under them; leaving out the additions, the
// loads or the stores takes 45, 80 and 45 off.  So: as much reuse as the registers hold (128
// sums a lane; the sums are added to outside the matrix instructions, so they cannot stand in
// accumulation registers), for tiles of 128 x 192 and 128 x 128 with two workgroups to a unit read
// 1.7 and 2 times as much and took 640 and 670 where this took 557; loads straight into shared memory, more
// than a block ahead (two whole buffers, one block ahead: 556 to 517), a few at a time between
// products (480 to 472), by buffer addresses (517 to 497: with plain addresses the compiler waits for all
// of them at each scale); rows stored whole from shared memory (556 to 500 with the former).  The 32x32
// instructions took 492 in place of 477, rows' operands read ahead of the barrier and wave
// priorities changed nothing.
// MORE: 16 rows or fewer behind the last whole tile are taken along by the last tiles, NT / WM of the
// outputs' tiles by each wave, whose operands it has at hand; the rows' come past shared memory,
// which is full.  Every tile makes these products, as a branch between others would cost as much.
// 777 x 20001 x 5000 87 us, where 768 rows and 9 in two launches took 94; 520 x 60000 x 1500 65 and 87.
template <int NT, int MT, int WN, int WM, bool MORE>
__global__ __launch_bounds__(64 * WN * WM) void k_f8_wide(MatArgs a)
{
    constexpr int E = MORE ? NT / WM : 0;      // tiles of outputs that a wave takes of the last rows
    static_assert(!MORE || E * WM == NT, "the waves share the last rows evenly");
    constexpr int W = WN * WM, TN = NT * WN, TM = MT * WM;
    static_assert(2 * TN % W == 0 && 2 * TM % W == 0, "a half's pieces are shared evenly");
    constexpr int kSlot = kTileBytes * (TN > TM ? TN : TM);
    constexpr int SLOTS = 5;
    __shared__ __align__(16) uint8_t s0[kSlot], s1[kSlot], s2[kSlot], s3[kSlot], s4[kSlot];
    uint8_t *const slot[SLOTS] = {s0, s1, s2, s3, s4};
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wv % WN, wm = wv / WN;
    // eight dies take runs of tiles of their own, in each four rows' tiles before the next outputs'
    const uint32_t tiles = a.grid_n * a.grid_m, total = tiles * a.splits, per = (total + 7) / 8;
    uint32_t turn = blockIdx.x / 8;

    // a wave's pieces of a half: half a tile each, of every (W / 2)-th tile
    static_assert(W % 2 == 0, "a wave's pieces are the same halves of its tiles");
    constexpr int PN = 2 * TN / W, PM = 2 * TM / W;
    const int tile_bytes = a.blocks * kTileBytes;
    int nt0, mt0, split, count;
    __amdgpu_buffer_rsrc_t w_from, x_from;
    int piece[PN + PM];           // where the wave's pieces of a block start, weights' and rows'
    const float *ws, *xs;
    int m_last;                   // the tile of rows that MORE adds
    auto next_tile = [&] {
        const uint32_t id = blockIdx.x % 8 * per + turn;
        if (turn >= per || id >= total) return false;
        turn += gridDim.x / 8;
        split = (int)(id / tiles);
        const int b0 = split * a.per_split;
        count = min(a.per_split, a.blocks - b0);
        const uint32_t tile = id % tiles, group = tile / (4 * a.grid_n), in = tile % (4 * a.grid_n);
        const uint32_t high = min(4u, a.grid_m - 4 * group);
        nt0 = (int)(in / high) * TN;
        mt0 = (int)(4 * group + in % high) * TM;
        // (tiles past the last one are read as the last one)
        auto from = [&](const uint8_t *p, int t0, int have, int own, int n, int *at) {
            const int last = min(have - t0, own) - 1;
            for (int i = 0; i < n; ++i) at[i] = min(wv / 2 + i * (W / 2), last) * tile_bytes;
            return __builtin_amdgcn_make_buffer_rsrc(
                (void *)(p + (int64_t)t0 * tile_bytes + b0 * kTileBytes), 0,
                qlm_f8_host::load_bytes(have - t0, own, a.blocks, b0), 0x00020000);
        };
        w_from = from(a.w, nt0, a.n_tiles, TN, PN, piece);
        x_from = from(a.x, mt0, a.m_tiles, TM, PM, piece + PN);
        ws = a.ws + (int64_t)(min(nt0 + wn * NT, a.n_tiles - 1) / (kBlock / kTile)) * a.blocks + b0;
        xs = a.xs + (int64_t)b0 * a.padded + (int64_t)mt0 * kTile;
        m_last = min(mt0 + TM, a.m_tiles - 1);
        return true;
    };
    const int lane_at = 16 * lane + 1024 * (wv & 1);
    // half h of the loads: the weights of block h / 2, then its rows, in slot h % SLOTS
    auto fetch = [&](bool n, int i, int b, uint8_t *to) {       // piece i of a half
        load_lds(n ? w_from : x_from, piece[n ? i : PN + i] + min(b, count - 1) * kTileBytes, lane_at,
                 to + 1024 * (i * W + wv));
    };
    // the tiles of outputs in the wave's order: with MORE those it takes of the last rows at the end
    const int first = MORE ? (wm + 1) * E : 0;
    auto from_first = [&](int i) {
        if constexpr (MORE) {
            i = (i + first) % NT;
            asm volatile("" : "+s"(i));        // (the places that depend on it are not all kept)
        }
        return i;
    };
    float4v acc[NT][MT], acc_last[E + 1];
    float by[MT], w_next, x_next[MT], by_last, x_last_next;
    int8v x_last;
    auto fetch_scales = [&](int b) {
        b = min(b, count - 1);
        w_next = ws[b];
        const float *p = xs + (int64_t)b * a.padded;
#pragma unroll
        for (int j = 0; j < MT; ++j)
            x_next[j] = (p + min(wm * MT + j, a.m_tiles - 1 - mt0) * kTile)[lane & 15];
        if constexpr (MORE) x_last_next = (p + (m_last - mt0) * kTile)[lane & 15];
    };
    auto fetch_last = [&](int b) {
        if constexpr (MORE)
            x_last = operand(a.x + ((int64_t)m_last * a.blocks + split * a.per_split + b) * kTileBytes,
                             lane);
    };
    // A block's products; `more` starts the loads of later ones, a few at a time: all at once they
    // would hold the waves up until the last is on its way.
    auto step = [&](const uint8_t *wt, const uint8_t *xt, auto more) {
        // (a tile's place is known a tile ahead of its reads: these come before the products then)
        auto place = [&](int i) { return wt + kTileBytes * (wn * NT + from_first(i)) + 16 * lane; };
        int8v ahead = operand(place(0), 0);
        int8v x[MT];
#pragma unroll
        for (int j = 0; j < MT; ++j) x[j] = operand(xt + kTileBytes * (wm * MT + j), lane);
        const uint8_t *next = place(1);
        float4v was[MT], now[MT], was_last, now_last;
#pragma unroll
        for (int i = 0; i <= NT; ++i) {
            const int8v w = ahead;
            if (i + 1 < NT) ahead = operand(next, 0);
            if (i + 2 < NT) next = place(i + 2);
            if (i < NT) more(i);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                if (i < NT) now[j] = product(w, x[j]);
                if (i > 0)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i - 1][j][e] += by[j] * was[j][e];
            }
            if (i >= NT - E && i < NT) now_last = product(w, x_last);
            if (i > NT - E)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc_last[i - 1 - NT + E][e] += by_last * was_last[e];
#pragma unroll
            for (int j = 0; j < MT + (i >= NT - E); ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            }
#pragma unroll
            for (int j = 0; j < MT; ++j) was[j] = now[j];
            was_last = now_last;
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Loads run SLOTS - 2 halves ahead.  Behind a block's barrier its own halves are there and
    // those of the block before have no readers any more.
    constexpr int AHEAD = SLOTS - 2;
    auto begin = [&] {
        fetch_scales(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
#pragma unroll
            for (int i = 0; i < (h % 2 ? PM : PN); ++i) fetch(h % 2 == 0, i, h / 2, slot[h]);
            // (half by half: the first block counts on the last half's being the last under way)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto block = [&](int b, int i) {       // i: b's place in a turn of SLOTS blocks
        // the loads that may be under way still: those of halves past this block's two
        constexpr int LATER = (AHEAD - 2) / 2 * (PN + PM) + (AHEAD % 2 ? PN : 0);
        wait_loads<LATER>();
        asm volatile("" ::: "memory");         // (no read or write moves over the barrier)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < MT; ++j) by[j] = w_next * x_next[j];
        if constexpr (MORE) by_last = w_next * x_last_next;
        __builtin_amdgcn_sched_barrier(0);
        fetch_last(b);                         // (used at the block's end)
        fetch_scales(b + 1);
        __builtin_amdgcn_sched_barrier(0);     // (before the loads: waited for with fewer left)
        step(slot[2 * i % SLOTS], slot[(2 * i + 1) % SLOTS], [&](int k) {
            // the rows of the next block, then the weights of the one after it
            static_assert(AHEAD == 3, "the halves that follow");
#pragma unroll
            for (int p = k * (PN + PM) / NT; p < (k + 1) * (PN + PM) / NT; ++p)
                if (p < PM)
                    fetch(false, p, b + 1, slot[(2 * i + 3) % SLOTS]);
                else
                    fetch(true, p - PM, b + 2, slot[(2 * i + 4) % SLOTS]);
        });
    };
    if (!next_tile()) return;
    begin();
    for (bool more = true; more;) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[i][j] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < E; ++e) acc_last[e] = float4v{0, 0, 0, 0};
        int b = 0;
        for (; b + SLOTS <= count; b += SLOTS)
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) block(b + i, i);
#pragma unroll
        for (int i = 0; i < SLOTS - 1; ++i) {
            // (the sums are made before the branch: they would move behind it with all their
            // products held in registers)
#pragma unroll
            for (int k = 0; k < NT; ++k)
#pragma unroll
                for (int j = 0; j < MT; ++j) asm volatile("" : "+v"(acc[k][j]));
#pragma unroll
            for (int e = 0; e < E; ++e) asm volatile("" : "+v"(acc_last[e]));
            if (b + i < count) block(b + i, i);
        }
        // The next tile's first loads begin before this one's outputs are stored.  (The staging memory is
        // one of two slots, which the compiler cannot tell from those being loaded: it waits for all
        // that is under way, stores too, before a group of 16 rows is staged, and in single precision before
        // each store.  The other tiles on the unit hide some of it: 1178 x 19884 x 896 43 us, floor 15.)
        wait_loads<0>();
        __syncthreads();
        const int n0 = (nt0 + wn * NT) * kTile, mt = mt0 + wm * MT, part = split;
        const bool has_last = MORE && mt0 + TM == a.m_tiles - 1;
        more = next_tile();
        if (more) begin();
        constexpr int kStage = kTile * 16 * NT * 4, kIn = kSlot / kStage;
        static_assert(2 * kIn >= W, "the waves' outputs fit the two slots that are not under way");
        uint8_t *lds = (wv < kIn ? slot[AHEAD] : slot[AHEAD + 1]) + wv % kIn * kStage;
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            float4v v[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) v[i] = acc[i][j];
            if (mt + j >= a.m_tiles) break;
            const int64_t m0 = (int64_t)(mt + j) * kTile;
            if (a.dtype == QLM_F32)
                store_rows<NT, float>(a, part, m0, n0, v, first, lds);
            else
                store_rows<NT, uint16_t>(a, part, m0, n0, v, first, lds);
        }
        if constexpr (MORE)
            if (has_last) {
                const int64_t m0 = (int64_t)(a.m_tiles - 1) * kTile;
                const int n_last = n0 + wm * E * kTile;
                if (a.dtype == QLM_F32)
                    store_rows<E, float>(a, part, m0, n_last, acc_last, 0, lds);
                else
                    store_rows<E, uint16_t>(a, part, m0, n_last, acc_last, 0, lds);
            }
    }
}

// Sums of the runs, in their order, four outputs of a row a thread.
__global__ __launch_bounds__(256) void k_f8_join(MatArgs a, const float *part, int64_t ld, int64_t run)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = at / (ld / 4);
    const int n = (int)(at % (ld / 4)) * 4;
    if (m >= a.M) return;
    float4v v = *(const float4v *)(part + m * ld + n);
    for (int k = 1; k < a.splits; ++k) v += *(const float4v *)(part + k * run + m * ld + n);
    store4(a, m, n, v);
}

int check_weight(const qlm_f8 *w)
{
    if (!w) return fail(QLM_ERR_ARG, "weight is NULL");
    if (w->n_out < 1 || w->n_in < 1 || w->n_out > kMost || w->n_in > kMost)
        return fail(QLM_ERR_ARG, "n_out and n_in must be in 1..16777216");
    if (!w->packed || (uintptr_t)w->packed % 256)
        return fail(QLM_ERR_ARG, "packed must be non-NULL and 256-byte aligned");
    return QLM_OK;
}

int check_codes(const qlm_f8_codes *r)
{
    if (!r) return fail(QLM_ERR_ARG, "rows is NULL");
    if (r->n_rows < 0 || r->n_rows > INT32_MAX - kTile)
        return fail(QLM_ERR_ARG, "n_rows must be in 0..2147483631");
    if (r->n_in < 1 || r->n_in > kMost) return fail(QLM_ERR_ARG, "n_in must be in 1..16777216");
    if (r->n_rows == 0) return QLM_OK;
    if (!r->codes || !r->scale) return fail(QLM_ERR_ARG, "codes and scale are required");
    if ((uintptr_t)r->codes % 16 || (uintptr_t)r->scale % 4)
        return fail(QLM_ERR_ARG, "codes must be 16-byte, scale 4-byte aligned");
    return QLM_OK;
}

int64_t part_stride(int n_out) { return ((int64_t)n_out + 3) / 4 * 4; }

// GROUPS: workgroups that a compute unit holds.
template <int NT, int MT, int WN, int WM, int GROUPS, bool MORE = false>
void launch_wide(MatArgs a, hipStream_t stream)
{
    a.grid_n = (a.n_tiles + NT * WN - 1) / (NT * WN);
    a.grid_m = MORE ? a.m_tiles / (MT * WM) : (a.m_tiles + MT * WM - 1) / (MT * WM);
    const int64_t tiles = (int64_t)a.grid_n * a.grid_m * a.splits;
    const int64_t grid = std::min<int64_t>(GROUPS * kCus, (tiles + 7) / 8 * 8);
    k_f8_wide<NT, MT, WN, WM, MORE><<<(unsigned)grid, 64 * WN * WM, 0, stream>>>(a);
}

hipError_t launch(MatArgs a, const Plan &p, void *ws, hipStream_t stream)
{
    if (!p.side) {
        const auto t = qlm_f8_host::thin_of(a.n_tiles, a.m_tiles, a.blocks);
        auto kern = t.outs == 4   ? k_f8_thin<4, 2, 8, 1>
                    : t.rows == 4 ? k_f8_thin<2, 4, 8, 2>
                    : t.rows == 3 ? k_f8_thin<2, 3, 8, 2>
                    : t.outs == 2 ? k_f8_thin<2, 2, 8, 2>
                    : t.rows == 2 ? k_f8_thin<1, 2, 8, 4>
                                  : k_f8_thin<1, 1, 8, 4>;
        kern<<<(unsigned)qlm_f8_host::thin_groups(a.n_tiles, a.m_tiles, a.blocks), 512, 0, stream>>>(a);
        return hipGetLastError();
    }
    a.splits = p.splits;
    a.per_split = p.per_split;
    MatArgs o = a;
    const int64_t ld = part_stride(a.N), run = a.M * ld;
    if (p.splits > 1) {
        o.out = ws;
        o.out_stride = ld;
        o.out_split = run;
        o.out_wide = 1;
        o.out_past = 0;
        o.dtype = QLM_F32;
    }
    if (p.side == 64)
        launch_wide<2, 2, 2, 2, 3>(o, stream);
    else if (p.side == 128)
        launch_wide<4, 2, 2, 4, 2>(o, stream);
    else if (p.one_more)
        launch_wide<8, 4, 2, 4, 1, true>(o, stream);
    else
        launch_wide<8, 4, 2, 4, 1>(o, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    k_f8_join<<<(unsigned)qlm_f8_host::join_groups(a.N, a.M), 256, 0, stream>>>(a, (const float *)ws, ld,
                                                                               run);
    return hipGetLastError();
}

int64_t code_bytes(int n_out, int n_in) { return tiles_of(n_out) * blocks_of(n_in) * kTileBytes; }

}  // namespace

extern "C" {

size_t qlm_f8_packed_bytes(int32_t n_out, int32_t n_in)
{
    if (n_out < 1 || n_in < 1 || n_out > kMost || n_in > kMost) return 0;
    return (size_t)(code_bytes(n_out, n_in) + 4 * blocks_of(n_out) * blocks_of(n_in));
}

int qlm_f8_pack(const qlm_f8 *weight, const void *codes, const float *scale, qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    if (int rc = check_weight(weight)) return rc;
    if (!codes || !scale) return fail(QLM_ERR_ARG, "codes and scale are required");
    if ((uintptr_t)scale % 4) return fail(QLM_ERR_ARG, "scale is misaligned");
    PackArgs a{};
    a.codes = (const uint8_t *)codes;
    a.scale = scale;
    a.N = weight->n_out;
    a.K = weight->n_in;
    a.blocks = (int32_t)blocks_of(a.K);
    a.chunks = code_bytes(a.N, a.K) / 16;
    a.scales = blocks_of(a.N) * a.blocks;
    a.packed = (uint8_t *)weight->packed;
    a.packed_scale = (float *)(a.packed + 16 * a.chunks);
    a.wide = a.K % 16 == 0 && (uintptr_t)codes % 16 == 0;
    a.words = a.K % 4 == 0 && (uintptr_t)codes % 4 == 0;
    const int64_t grid = (a.chunks + 255) / 256;
    if (!can_launch(grid, 256)) return fail(QLM_ERR_CAPACITY, "too many threads for one matrix");
    k_f8_pack<<<(unsigned)grid, 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_f8_pack launch");
}

int qlm_f8_rows(const qlm_f8_codes *rows, const void *x, int64_t x_stride, int32_t dtype,
                qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    if (int rc = check_codes(rows)) return rc;
    if (dtype != QLM_F16 && dtype != QLM_BF16)
        return fail(QLM_ERR_ARG, "dtype must be QLM_F16 or QLM_BF16");
    if (rows->n_rows == 0) return QLM_OK;
    if (!x) return fail(QLM_ERR_ARG, "x is required");
    if ((uintptr_t)x % 2) return fail(QLM_ERR_ARG, "x is misaligned");
    if (x_stride < rows->n_in) return fail(QLM_ERR_ARG, "x_stride must be >= the row's length");
    RowsArgs a{};
    a.x = (const uint16_t *)x;
    a.codes = (uint8_t *)rows->codes;
    a.scale = rows->scale;
    a.x_stride = x_stride;
    a.M = rows->n_rows;
    a.K = rows->n_in;
    a.blocks = (int32_t)blocks_of(a.K);
    a.tiles = tiles_of(a.M) * a.blocks;
    a.padded = (int32_t)(tiles_of(a.M) * kTile);
    a.wide = (uintptr_t)x % 16 == 0 && x_stride % 8 == 0;
    const int64_t grid = (a.tiles + 3) / 4;
    if (!can_launch(grid, 256)) return fail(QLM_ERR_CAPACITY, "too many rows in one call");
    if (dtype == QLM_BF16)
        k_f8_rows<true><<<(unsigned)grid, 256, 0, stream>>>(a);
    else
        k_f8_rows<false><<<(unsigned)grid, 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_f8_rows launch");
}

size_t qlm_f8_workspace_bytes(const qlm_f8 *weight, int32_t n_rows)
{
    if (check_weight(weight) || n_rows < 1) return 0;
    const Plan p = parts_of(weight->n_out, weight->n_in, n_rows).first;
    return p.splits > 1 ? (size_t)p.splits * n_rows * part_stride(weight->n_out) * 4 : 0;
}

int qlm_f8_matmul(const qlm_f8_codes *rows, const qlm_f8 *weight, void *out, int64_t out_stride,
                  int32_t dtype, void *ws, size_t ws_bytes, qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    if (int rc = check_weight(weight)) return rc;
    if (int rc = check_codes(rows)) return rc;
    if (rows->n_in != weight->n_in) return fail(QLM_ERR_ARG, "rows and weight differ in n_in");
    if (dtype != QLM_F16 && dtype != QLM_BF16 && dtype != QLM_F32)
        return fail(QLM_ERR_ARG, "dtype must be QLM_F16, QLM_BF16 or QLM_F32");
    if (rows->n_rows == 0) return QLM_OK;
    if (!out) return fail(QLM_ERR_ARG, "out is required");
    if ((uintptr_t)out % (dtype == QLM_F32 ? 4 : 2)) return fail(QLM_ERR_ARG, "out is misaligned");
    if (out == rows->codes) return fail(QLM_ERR_ARG, "out may not overlap the codes");
    if (out_stride < weight->n_out)
        return fail(QLM_ERR_ARG, "out_stride must be >= the row's length");
    const size_t need = qlm_f8_workspace_bytes(weight, rows->n_rows);
    if (need && (!ws || (uintptr_t)ws % 256))
        return fail(QLM_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
    if (ws_bytes < need) return fail(QLM_ERR_WORKSPACE, "workspace too small");
    MatArgs a{};
    a.w = (const uint8_t *)weight->packed;
    a.ws = (const float *)(a.w + code_bytes(weight->n_out, weight->n_in));
    a.x = (const uint8_t *)rows->codes;
    a.xs = rows->scale;
    a.out = out;
    a.out_stride = out_stride;
    a.N = weight->n_out;
    a.M = rows->n_rows;
    a.blocks = (int32_t)blocks_of(weight->n_in);
    a.n_tiles = (int32_t)tiles_of(a.N);
    a.m_tiles = (int32_t)tiles_of(a.M);
    a.padded = a.m_tiles * kTile;
    a.dtype = dtype;
    const int size = dtype == QLM_F32 ? 4 : 2;
    a.out_wide = (uintptr_t)out % 16 == 0 && out_stride * size % 16 == 0;
    // outputs that the second-level caches (32 MiB) do not hold would only push the operands out of
    // them: 8192 x 16384 x 4096 476 us through the caches, 464 past them
    a.out_past = (int64_t)a.M * a.N * size > (64 << 20);
    const auto parts = parts_of(weight->n_out, weight->n_in, rows->n_rows);
    MatArgs rest = a;
    if (parts.n_first < rows->n_rows) {        // (whole tiles of rows)
        a.M = parts.n_first;
        a.m_tiles = a.M / kTile;
        rest.M -= a.M;
        rest.m_tiles -= a.m_tiles;
        rest.x += (int64_t)a.m_tiles * a.blocks * kTileBytes;
        rest.xs += a.M;
        rest.out = (char *)out + a.M * out_stride * size;
        rest.out_wide = a.out_wide && (uintptr_t)rest.out % 16 == 0;
        if (!fits(a.N, weight->n_in, rest.M, parts.rest))
            return fail(QLM_ERR_CAPACITY, "too many outputs in one call");
    }
    if (!fits(a.N, weight->n_in, a.M, parts.first))
        return fail(QLM_ERR_CAPACITY, "too many outputs in one call");
    hipError_t e = launch(a, parts.first, ws, stream);
    if (e == hipSuccess && parts.n_first < rows->n_rows) e = launch(rest, parts.rest, ws, stream);
    return e == hipSuccess ? QLM_OK : hip_fail(e, "f8 launch");
}

}  // extern "C"

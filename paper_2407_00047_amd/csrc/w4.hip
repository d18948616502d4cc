// w4.hip -- products with 4-bit weights and group scales (qlm_w4_pack,
// qlm_w4_matmul; the definition stands in include/qlm.h).
//
// A code c becomes the number 16 + c by placing its four bits at the top of a
// mantissa under the exponent of 16 (exact in half precision and bfloat16, one
// shift and one and-or for two codes).  With X = x as it came and one group's
// sums S = sum of x, T[n] = sum of (16 + c[n]) x, both by the matrix
// instructions (S with a matrix of ones), the group's part of the output is
//   s[n] (T[n] - (16 + z[n]) S),
// formed in single precision; so no weight is ever rounded.  An x that is not
// finite makes its row's outputs not finite.
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

namespace {

using qlm_internal::fail;
using qlm_internal::hip_fail;

typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kStep = 128;           // inputs of a chunk
constexpr int kWaves = 4, kThreads = 64 * kWaves;

__host__ __device__ inline int chunk_bytes(int group) { return 1024 + 64 * (kStep / group); }

struct PackArgs {
    int32_t N, K, group, tiles, steps;
    const uint8_t *codes, *zero;
    const uint16_t *scale;
    uint8_t *packed;
};

// One workgroup for each chunk, a lane of the first wave for each 16 bytes.
__global__ __launch_bounds__(64) void k_w4_pack(PackArgs a)
{
    const int l = threadIdx.x;
    const int kb = blockIdx.x % a.steps, tile = blockIdx.x / a.steps;
    uint8_t *chunk = a.packed + (int64_t)blockIdx.x * chunk_bytes(a.group);
    const int n = tile * 16 + l % 16;
    uint32_t w[4] = {0, 0, 0, 0};
    for (int j = 0; j < 4; ++j)
        for (int e = 0; e < 8; ++e) {
            const int k = kb * kStep + j * 32 + (l / 16) * 8 + e;
            const uint32_t c = n < a.N && k < a.K ? a.codes[(int64_t)n * a.K + k] & 15u : 0u;
            w[j] |= c << (16 * (e & 1) + 4 * (e >> 1));
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

// The eight codes of a dword as 16 + c.
template <bool BF> __device__ inline uint4 operand(uint32_t w)
{
    if (BF)
        return {(w << 3 & 0x00780078u) | 0x41804180u, (w >> 1 & 0x00780078u) | 0x41804180u,
                (w >> 5 & 0x00780078u) | 0x41804180u, (w >> 9 & 0x00780078u) | 0x41804180u};
    return {(w << 6 & 0x03c003c0u) | 0x4c004c00u, (w << 2 & 0x03c003c0u) | 0x4c004c00u,
            (w >> 2 & 0x03c003c0u) | 0x4c004c00u, (w >> 6 & 0x03c003c0u) | 0x4c004c00u};
}

template <bool BF> __device__ inline uint4 ones()
{
    const uint32_t o = BF ? 0x3f803f80u : 0x3c003c00u;
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
// in turn; x in shared memory.
template <bool BF, int GROUP> __global__ __launch_bounds__(kThreads) void k_w4_thin(MatArgs a)
{
    constexpr int PER = kStep / GROUP, SUB = 4 / PER, PF = 4;
    extern __shared__ uint4 lds[];
    uint16_t *xs = (uint16_t *)lds;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int g = lane >> 4, c16 = lane & 15;
    const int tile = blockIdx.x;
    const int cb = chunk_bytes(GROUP);
    const uint8_t *base = a.packed + (int64_t)tile * a.steps * cb;
    const int ld = a.per_stage * kStep + 8;      // elements of a row in shared memory
    const int mine = c16 < a.M ? c16 : 0;
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    uint4 cw[PF], mw[PF][PER];
    auto fetch = [&](int u, int kb) {
        if (kb < a.steps) {
            const uint8_t *p = base + (int64_t)kb * cb;
            cw[u] = *(const uint4 *)(p + 16 * lane);
            for (int q = 0; q < PER; ++q) mw[u][q] = *(const uint4 *)(p + 1024 + 64 * q + 16 * g);
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
                        t = mfma<BF>(operand<BF>(w[j]), b, t);
                        S = mfma<BF>(ones<BF>(), b, S);
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
    if (m < a.M && n < a.N) a.out[m * a.out_stride + n] = out_bits(v, BF);
}

// More rows: one workgroup to 64 outputs (16 a wave) and 16 NT rows; x passes
// through shared memory a step at a time, in two buffers.
template <bool BF, int GROUP, int NT>
__global__ __launch_bounds__(kThreads) void k_w4_wide(MatArgs a)
{
    constexpr int PER = kStep / GROUP, SUB = 4 / PER, LD = kStep + 8;
    __shared__ uint4 lds[2][NT * 16 * LD / 8];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int g = lane >> 4, c16 = lane & 15;
    const int tile = blockIdx.x * kWaves + wv, m0 = blockIdx.y * NT * 16, sp = blockIdx.z;
    const int k0 = sp * a.per_split, k1 = min(a.steps, k0 + a.per_split);
    const int cb = chunk_bytes(GROUP);
    const bool mine = tile < a.tiles;
    const uint8_t *base = a.packed + (int64_t)(mine ? tile : 0) * a.steps * cb;
    float4v sum[NT];
    for (int t = 0; t < NT; ++t) sum[t] = float4v{0.f, 0.f, 0.f, 0.f};
    uint4 cw, mw[PER], xr[NT];
    auto fetch_w = [&](int kb) {
        const uint8_t *p = base + (int64_t)kb * cb;
        cw = *(const uint4 *)(p + 16 * lane);
        for (int q = 0; q < PER; ++q) mw[q] = *(const uint4 *)(p + 1024 + 64 * q + 16 * g);
    };
    // thread t stages row t / 16 of each 16 rows, inputs 8 (t % 16) on
    const int sr = threadIdx.x >> 4, sk = 8 * (threadIdx.x & 15);
    auto fetch_x = [&](int kb) {
        for (int t = 0; t < NT; ++t) {
            const int r = m0 + t * 16 + sr;
            xr[t] = r < a.M ? x8(a, r, kb * kStep + sk) : uint4{0, 0, 0, 0};
        }
    };
    auto stage = [&](int buf) {
        uint16_t *xs = (uint16_t *)lds[buf];
        for (int t = 0; t < NT; ++t) *(uint4 *)(xs + (t * 16 + sr) * LD + sk) = xr[t];
    };
    if (k0 < k1) {
        fetch_w(k0);
        fetch_x(k0);
        stage(0);
    }
    __syncthreads();
    for (int kb = k0; kb < k1; ++kb) {
        const int buf = (kb - k0) & 1;
        const uint4 w4 = cw;
        uint4 m4[PER];
        for (int q = 0; q < PER; ++q) m4[q] = mw[q];
        if (kb + 1 < k1) {
            fetch_w(kb + 1);
            fetch_x(kb + 1);
        }
        const uint16_t *xs = (const uint16_t *)lds[buf];
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        for (int q = 0; q < PER; ++q) {
            float4v t[NT], S[NT];
            for (int k = 0; k < NT; ++k) t[k] = S[k] = float4v{0.f, 0.f, 0.f, 0.f};
            for (int j = q * SUB; j < (q + 1) * SUB; ++j) {
                const uint4 o = operand<BF>(w[j]);
                for (int k = 0; k < NT; ++k) {
                    const uint4 b = *(const uint4 *)(xs + (k * 16 + c16) * LD + 32 * j + 8 * g);
                    t[k] = mfma<BF>(o, b, t[k]);
                    S[k] = mfma<BF>(ones<BF>(), b, S[k]);
                }
            }
            for (int k = 0; k < NT; ++k) sum[k] = add_group(sum[k], t[k], S[k][0], m4[q]);
        }
        if (kb + 1 < k1) stage(buf ^ 1);
        __syncthreads();
    }
    if (!mine) return;
    for (int k = 0; k < NT; ++k) {
        const int m = m0 + k * 16 + c16;
        if (m >= a.M) continue;
        for (int i = 0; i < 4; ++i) {
            const int n = tile * 16 + 4 * g + i;
            if (n >= a.N) continue;
            if (a.splits > 1)
                a.part[((int64_t)sp * a.M + m) * a.N + n] = sum[k][i];
            else
                a.out[m * a.out_stride + n] = out_bits(sum[k][i], BF);
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_w4_join(MatArgs a, int bf)
{
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t all = (int64_t)a.M * a.N;
    if (e >= all) return;
    float v = 0.f;
    for (int s = 0; s < a.splits; ++s) v += a.part[s * all + e];
    a.out[e / a.N * a.out_stride + e % a.N] = out_bits(v, bf);
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

constexpr int kThinRows = 16;

void split_of(const qlm_w4 *w, int rows, int *splits, int *per)
{
    const int steps = (w->n_in + kStep - 1) / kStep;
    *splits = 1;
    *per = steps;
    if (rows <= kThinRows) return;
    // enough workgroups for every CU, eight steps each at least
    const int64_t wg = ((int64_t)w->n_out + 63) / 64 * ((rows + 63) / 64);
    const int64_t want = std::min<int64_t>((512 + wg - 1) / wg, std::max(1, steps / 8));
    *per = (int)((steps + want - 1) / want);
    *splits = (steps + *per - 1) / *per;
}

template <bool BF, int GROUP> void launch(MatArgs a, int rows, hipStream_t st)
{
    if (rows <= kThinRows) {
        // as much of x as 64 KiB hold
        const int most = (65536 / rows - 16) / (2 * kStep) / kWaves * kWaves;
        a.per_stage = std::min(most, (a.steps + kWaves - 1) / kWaves * kWaves);
        const int bytes = std::max(rows * (a.per_stage * kStep + 8) * 2, kWaves * 1024);
        k_w4_thin<BF, GROUP><<<a.tiles, kThreads, bytes, st>>>(a);
        return;
    }
    const int nt = std::min(4, (rows + 15) / 16);
    const dim3 grid((a.tiles + kWaves - 1) / kWaves, (rows + 16 * nt - 1) / (16 * nt), a.splits);
    if (nt == 2)
        k_w4_wide<BF, GROUP, 2><<<grid, kThreads, 0, st>>>(a);
    else if (nt == 3)
        k_w4_wide<BF, GROUP, 3><<<grid, kThreads, 0, st>>>(a);
    else
        k_w4_wide<BF, GROUP, 4><<<grid, kThreads, 0, st>>>(a);
}

template <bool BF> void launch(const MatArgs &a, int group, int rows, hipStream_t st)
{
    if (group == 32)
        launch<BF, 32>(a, rows, st);
    else if (group == 64)
        launch<BF, 64>(a, rows, st);
    else
        launch<BF, 128>(a, rows, st);
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
    if (grid > INT32_MAX) return fail(QLM_ERR_CAPACITY, "the matrix is too large");
    k_w4_pack<<<(unsigned)grid, 64, 0, (hipStream_t)stream_>>>(a);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_w4_pack launch");
}

size_t qlm_w4_workspace_bytes(const qlm_w4 *weight, int32_t n_rows)
{
    if (!weight || n_rows < 1 || weight->n_out < 1 || weight->n_in < 1) return 0;
    int splits, per;
    split_of(weight, n_rows, &splits, &per);
    return splits > 1 ? (size_t)splits * n_rows * weight->n_out * 4 : 0;
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
    split_of(weight, n_rows, &a.splits, &a.per_split);
    a.part = (float *)ws;
    if (dtype == QLM_BF16)
        launch<true>(a, weight->group, n_rows, stream);
    else
        launch<false>(a, weight->group, n_rows, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "w4 launch");
    if (a.splits > 1) {
        const int64_t grid = ((int64_t)a.M * a.N + kThreads - 1) / kThreads;
        if (grid > INT32_MAX) return fail(QLM_ERR_CAPACITY, "too many outputs in one call");
        k_w4_join<<<(unsigned)grid, kThreads, 0, stream>>>(a, dtype == QLM_BF16);
        if ((e = hipGetLastError()) != hipSuccess) return hip_fail(e, "k_w4_join launch");
    }
    return QLM_OK;
}

}  // extern "C"

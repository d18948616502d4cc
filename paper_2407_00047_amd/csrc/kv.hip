// kv.hip -- the 8-bit token cache: writing new tokens (qlm_kv_append, with keys
// turned by their positions qlm_kv_append_rotated) and cutting sequences to a budget
// by accumulated attention weight (qlm_kv_evict).
// The definitions stand in include/qlm.h.
#include "kv.h"

#include <string>
#include <type_traits>

namespace qlm_kv {

using qlm_internal::fail;
using qlm_internal::hip_fail;

int check_cache(const qlm_kv_cache *c)
{
    if (!c) return fail(QLM_ERR_ARG, "cache is NULL");
    if (c->n_blocks < 1) return fail(QLM_ERR_ARG, "n_blocks must be >= 1");
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024)
        return fail(QLM_ERR_ARG, "n_kv_heads must be in 1..1024");
    if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16)
        return fail(QLM_ERR_ARG, "head_dim must be a multiple of 16 in 16..256");
    if (c->format != QLM_KV_E4M3 && c->format != QLM_KV_INT8)
        return fail(QLM_ERR_ARG, "format must be QLM_KV_E4M3 or QLM_KV_INT8");
    if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale)
        return fail(QLM_ERR_ARG, "a required cache array is NULL");
    if ((uintptr_t)c->k_codes % 16 || (uintptr_t)c->v_codes % 16)
        return fail(QLM_ERR_ARG, "k_codes and v_codes must be 16-byte aligned");
    return QLM_OK;
}

int check_batch(const qlm_kv_batch *b)
{
    if (!b) return fail(QLM_ERR_ARG, "batch is NULL");
    if (b->n_seqs < 0 || b->n_rows < 0)
        return fail(QLM_ERR_ARG, "n_seqs and n_rows must be >= 0");
    if (b->n_seqs > (1 << 20)) return fail(QLM_ERR_ARG, "n_seqs must be <= 1048576");
    if (b->max_new < 1 || b->max_new > (1 << 24))
        return fail(QLM_ERR_ARG, "max_new must be in 1..16777216");
    if (b->max_length < 0 || b->max_length > (1 << 28))
        return fail(QLM_ERR_ARG, "max_length must be in 0..268435456");
    if (b->table_stride < (b->max_length + kBlock - 1) / kBlock)
        return fail(QLM_ERR_ARG, "table_stride must be >= ceil(max_length / 64)");
    if (!b->row_start && (b->n_rows != b->n_seqs || b->max_new != 1))
        return fail(QLM_ERR_ARG, "without row_start every sequence has one row");
    if (b->n_seqs > 0 && (!b->lengths || (!b->block_table && b->max_length > 0)))
        return fail(QLM_ERR_ARG, "block_table and lengths are required");
    return QLM_OK;
}

int check_rows(const qlm_rows *r, const char *what)
{
    if (!r || !r->data) return fail(QLM_ERR_ARG, std::string(what) + " is NULL");
    if (r->dtype != QLM_F16 && r->dtype != QLM_BF16)
        return fail(QLM_ERR_ARG, std::string(what) + ": dtype must be QLM_F16 or QLM_BF16");
    if ((uintptr_t)r->data % 2) return fail(QLM_ERR_ARG, std::string(what) + " is misaligned");
    return QLM_OK;
}

int check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return QLM_OK;
    if (!ws || (uintptr_t)ws % 256)
        return fail(QLM_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
    if (have < need)
        return fail(QLM_ERR_WORKSPACE, "workspace too small: " + std::to_string(have) + " of " +
                                           std::to_string(need) + " bytes");
    return QLM_OK;
}

}  // namespace qlm_kv

namespace {

using namespace qlm_kv;
using qlm_internal::fail;
using qlm_internal::hip_fail;

constexpr int kThreads = 256;

struct CacheArgs {
    uint8_t *kc, *vc;
    float *ks, *vs;
    int32_t *pos;
    float *weight;
    int32_t n_blocks, H, D;
};

CacheArgs cache_args(const qlm_kv_cache *c)
{
    return {(uint8_t *)c->k_codes, (uint8_t *)c->v_codes, c->k_scale, c->v_scale, c->position,
            c->weight, c->n_blocks, c->n_kv_heads, c->head_dim};
}

// The largest of two values over the workgroup, for every thread.
__device__ inline void max2(float &a, float &b, float *lds)
{
    for (int o = 32; o; o >>= 1) {
        a = fmaxf(a, __shfl_xor(a, o));
        b = fmaxf(b, __shfl_xor(b, o));
    }
    const int w = threadIdx.x >> 6, n = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        lds[2 * w] = a;
        lds[2 * w + 1] = b;
    }
    __syncthreads();
    for (int k = 0; k < n; ++k) {
        a = fmaxf(a, lds[2 * k]);
        b = fmaxf(b, lds[2 * k + 1]);
    }
}

__device__ inline float finite_abs(float x)
{
    x = fabsf(x);
    return x < __builtin_inff() ? x : 0.f;   // (a NaN compares false)
}

// Four codes requantised by `ratio`.
template <int FMT> __device__ inline uint32_t requant4(uint32_t w, float ratio)
{
    uint32_t o = 0;
    for (int b = 0; b < 4; ++b)
        o |= code_of<FMT>(code_value<FMT>((w >> (8 * b)) & 0xff) * ratio) << (8 * b);
    return o;
}

// The code of a code's magnitude (its low byte counts); 0 for a NaN.
template <int FMT> __device__ inline uint32_t magnitude(uint32_t c)
{
    if (FMT == QLM_KV_E4M3) return (c & 0x7f) == 0x7f ? 0u : c & 0x7f;
    return (uint32_t)abs((int)(int8_t)c);       // (128 is its own negative, read as -128)
}

// Four codes of scale `was` as codes of scale `now`.
template <int FMT> __device__ inline uint32_t rescale4(uint32_t w, float was, float now)
{
    // between powers of two the quotient is exact, and a product gives the same
    const bool exact = ((__builtin_bit_cast(uint32_t, was) | __builtin_bit_cast(uint32_t, now)) &
                        0x7fffffu) == 0;
    const float ratio = was / now;
    uint32_t o = 0;
    for (int b = 0; b < 4; ++b)
        o |= code_of<FMT>(exact ? code_value<FMT>((w >> (8 * b)) & 0xff) * ratio
                                : code_value<FMT>((w >> (8 * b)) & 0xff) * was / now) << (8 * b);
    return o;
}

struct AppendArgs {
    CacheArgs c;
    Seqs q;
    const void *k, *v;
    int64_t k_row, k_head, v_row, v_head;
    int32_t k_type, v_type, k_wide, v_wide;   // wide: may be read 16 bytes at a time
    const int32_t *first;
    int32_t touched;      // blocks a sequence's new slots may lie in
};

// Tables and positions of the rotation, and the queries that are turned beside the keys.
struct TurnArgs {
    const float *cos, *sin;
    const int32_t *axis, *position;
    int32_t half, n_positions, n_axes;
    int32_t table_wide;             // the tables (and axes) may be read 16 bytes at a time
    const void *q;
    void *q_out;
    int64_t q_row, q_head, out_row, out_head;
    int32_t q_type, q_wide, n_heads;
    int32_t units, pair_units;      // 16 dims of a head each: the pairs' first, then the rest
    uint32_t key_groups, row_items;    // workgroups of the keys; waves of a row's queries
};

// The place in the tables of pair i of a row (`own`: its position where there is one axis).
__device__ inline int64_t table_at(const TurnArgs &t, int n_rows, int row, int own, int i)
{
    int p = own;
    if (t.axis && t.position) {
        const int ax = max(0, min(t.axis[i], t.n_axes - 1));
        p = t.position[(int64_t)ax * n_rows + row];
    }
    return (int64_t)max(0, min(p, t.n_positions - 1)) * t.half + i;
}

// The axes of a unit's pairs, four and four.  Four neighbouring pairs nearly always turn by one position:
// their angles then stand side by side, and the positions are under way beside the rows.
struct Axes {
    int axis[2];
    bool one[2];                    // four that are read at once, by one position
};

__device__ inline Axes axes_of(const TurnArgs &t, int i)
{
    Axes r;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        r.axis[g] = 0;
        r.one[g] = t.table_wide && i + 4 * g + 4 <= t.half;
        if (t.axis && r.one[g]) {
            const int4 ax = *(const int4 *)(t.axis + i + 4 * g);
            r.one[g] = ax.x == ax.y && ax.x == ax.z && ax.x == ax.w;
            r.axis[g] = max(0, min(ax.x, t.n_axes - 1));
        }
    }
    return r;
}

// The positions of a row that is given them, for each four.
__device__ inline int2 positions_of(const TurnArgs &t, int n_rows, int64_t row, const Axes &x)
{
    if (!t.axis) {
        const int p = t.position[row];
        return {p, p};
    }
    return {t.position[(int64_t)x.axis[0] * n_rows + row],
            t.position[(int64_t)x.axis[1] * n_rows + row]};
}

// cos and sin of eight pairs from i on, of which those from `half` on are not read (1 and 0).
__device__ inline void angles(const TurnArgs &t, int n_rows, int row, int2 own, const Axes &x, int i,
                              float *c, float *s)
{
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const int p = g ? own.y : own.x, e0 = 4 * g;
        if (x.one[g]) {
            const int64_t at = (int64_t)max(0, min(p, t.n_positions - 1)) * t.half + i + e0;
            *(float4v *)(c + e0) = *(const float4v *)(t.cos + at);
            *(float4v *)(s + e0) = *(const float4v *)(t.sin + at);
            continue;
        }
#pragma unroll
        for (int e = e0; e < e0 + 4; ++e) {
            const bool in = i + e < t.half;
            const int64_t at = table_at(t, n_rows, row, p, in ? i + e : 0);
            c[e] = in ? t.cos[at] : 1.f;
            s[e] = in ? t.sin[at] : 0.f;
        }
    }
}

// The position `place` tokens behind another.
__device__ inline int position_of(int64_t first, int64_t place)
{
    return (int)min(first + place, (int64_t)INT32_MAX);
}

// A pair turned, each product and sum rounded by itself: a fused product would make the
// codes depend on which of the two products it takes.
__device__ inline void turn(float &a, float &b, float c, float s)
{
#pragma clang fp contract(off)
    const float x = a * c - b * s, y = b * c + a * s;
    a = x;
    b = y;
}

// Eight dims of a row as bits, 16 bytes at once where they are aligned.
__device__ inline uint4 row_bits8(const void *p, int64_t at, bool wide)
{
    const uint16_t *u = (const uint16_t *)p + at;
    if (wide) return *(const uint4 *)u;
    return {u[0] | (uint32_t)u[1] << 16, u[2] | (uint32_t)u[3] << 16, u[4] | (uint32_t)u[5] << 16,
            u[6] | (uint32_t)u[7] << 16};
}

__device__ inline float bits_value(uint32_t u, int dtype)
{
    if (dtype == QLM_BF16) return __builtin_bit_cast(float, u << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)u);
}

// Eight pairs, of which the first `have` turn; whole: all of them.
template <bool NEIGHBOURS>
__device__ inline void turn16(float *y, const float *c, const float *s, int have, bool whole)
{
    if (whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            turn(y[NEIGHBOURS ? 2 * e : e], y[NEIGHBOURS ? 2 * e + 1 : e + 8], c[e], s[e]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < have) turn(y[NEIGHBOURS ? 2 * e : e], y[NEIGHBOURS ? 2 * e + 1 : e + 8], c[e], s[e]);
}

// N dims' values.  (A branch for all of them: as a choice at each one it was three operations.)
template <int N> __device__ inline void values_of(const uint32_t *w, int dtype, float *y)
{
    if (dtype == QLM_BF16) {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = bits_value((w[i >> 1] >> (16 * (i & 1))) & 0xffff, QLM_BF16);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = bits_value((w[i >> 1] >> (16 * (i & 1))) & 0xffff, QLM_F16);
    }
}

template <int N> __device__ inline void bits_of(const float *y, int dtype, uint32_t *w)
{
    if (dtype == QLM_BF16) {
#pragma unroll
        for (int i = 0; i < N; i += 2)
            w[i / 2] = row_bits(y[i], QLM_BF16) | (uint32_t)row_bits(y[i + 1], QLM_BF16) << 16;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2)
            w[i / 2] = row_bits(y[i], QLM_F16) | (uint32_t)row_bits(y[i + 1], QLM_F16) << 16;
    }
}

// The greatest finite magnitude of eight dims, as bits (magnitudes order as integers).
__device__ inline uint32_t magnitude8(uint4 x, int dtype)
{
    const uint32_t inf = dtype == QLM_BF16 ? 0x7f80u : 0x7c00u;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t top = 0;
    for (int i = 0; i < 8; ++i) {
        const uint32_t m = (w[i >> 1] >> (16 * (i & 1))) & 0x7fffu;
        top = max(top, m < inf ? m : 0u);
    }
    return top;
}

// Eight values as codes over `scale`, clamped (a NaN stays one in e4m3).
template <int FMT> __device__ inline uint2 codes_of(const float *v, float scale, bool exact)
{
    const float by = 1.f / scale;
    uint32_t o[2] = {0, 0};
    if (FMT == QLM_KV_E4M3) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = exact ? v[i] * by : v[i] / scale;
            y[i] = x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int d = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
            o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], d, true);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            o[i >> 2] |= code_of<FMT>(exact ? v[i] * by : v[i] / scale) << (8 * (i & 3));
    }
    return {o[0], o[1]};
}

// The two runs of eight dims that a thread holds of a row of a head: whole pairs where dims that
// make a pair stand eight dims or more apart by eights, else 16 dims side by side.
__device__ inline void unit_dims(const TurnArgs &t, bool neighbours, int k, int *d0, int *d1)
{
    const bool apart = !neighbours && t.half % 8 == 0 && 8 * k < t.half;
    *d0 = apart ? 8 * k : 16 * k;
    *d1 = apart ? t.half + 8 * k : 16 * k + 8;
}

// A unit's dims, turned; lo, hi: the dims as they are, `at`: of the head's dim 0.
template <bool NEIGHBOURS>
__device__ inline void turned16(const TurnArgs &t, int n_rows, int row, int2 own, const Axes &axes,
                                const void *data, int64_t at, int k, uint4 lo, uint4 hi, int dtype,
                                float *y)
{
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    values_of<16>(w, dtype, y);
    if (NEIGHBOURS || t.half % 8 == 0) {
        if (8 * k >= t.half) return;
        float c[8], s[8];
        angles(t, n_rows, row, own, axes, 8 * k, c, s);
        turn16<NEIGHBOURS>(y, c, s, t.half - 8 * k, t.half % 8 == 0);
        return;
    }
#pragma unroll 1
    for (int e = 0; e < 16; ++e) {
        const int dim = 16 * k + e;
        if (dim >= 2 * t.half) break;
        const bool low = dim < t.half;
        const int i = low ? dim : dim - t.half;
        const int64_t p = table_at(t, n_rows, row, own.x, i);
        const uint16_t *x = (const uint16_t *)data + at;
        float p0 = bits_value(x[i], dtype), p1 = bits_value(x[i + t.half], dtype);
        turn(p0, p1, t.cos[p], t.sin[p]);
        const float z = low ? p0 : p1;
#pragma unroll
        for (int f = 0; f < 16; ++f) y[f] = f == e ? z : y[f];
    }
}

// Eight dims as codes over `scale` (a power of two nearly always: a product then).
template <int FMT> __device__ inline uint2 codes8(uint4 x, int dtype, float scale, bool exact)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float v[8];
    values_of<8>(w, dtype, v);
    return codes_of<FMT>(v, scale, exact);
}

__device__ inline bool power_of_two(float x)
{
    return (__builtin_bit_cast(uint32_t, x) & 0x7fffffu) == 0;
}

// The sequence that a row belongs to and its place there; -1 of a row of none.  Found by 64
// lanes at a time: one read of up to 64 sequences, two of up to 4096.
__device__ inline int row_seq(const Seqs &q, int row, int *place)
{
    if (!q.row_start) {
        *place = 0;
        return row < q.n_seqs ? row : -1;
    }
    int s = 0, left = q.n_seqs, first = 0, next = 0;
    for (int step = 1 << 30; step > 1;) {
        step = (left + 63) / 64;
        const int64_t at = (int64_t)(threadIdx.x & 63) * step;
        const int32_t *p = q.row_start + s + min(at, (int64_t)left - 1);
        const int mine = p[0], after = p[1];
        const uint64_t m = __ballot(at < left && mine <= row);
        if (m == 0) return -1;
        const int lane = 63 - __builtin_clzll(m);
        first = __builtin_amdgcn_readlane(mine, lane);
        next = __builtin_amdgcn_readlane(after, lane);
        s += lane * step;
        left = min(step, left - lane * step);
    }
    const int r0 = max(0, min(first, q.n_rows)), r1 = max(r0, min(next, q.n_rows));
    *place = row - r0;
    return *place >= 0 && *place < min(r1 - r0, q.max_new) ? s : -1;
}

// Where the 16 bytes of a group's dim stand in shared memory, and their word of 4 of slots: moved so that
// eight dims apart and the four groups meet in no bank.
__device__ inline int staged_unit(int u) { return u ^ ((u >> 3) & 15); }

__device__ inline int staged_at(int group, int dp, int dim, int place)
{
    return 16 * staged_unit(group * dp + dim) + 4 * (((place >> 2) + group) & 3);
}

// Eight dims from d on of G neighbouring slots, whose codes are c, as bytes side by side for each dim.
template <int G> __device__ inline void stage(uint8_t *to, int group, int dp, int d, int place, const uint2 *c)
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        auto part = [&](int i) { return half ? c[i].y : c[i].x; };
        // bytes 0 and 1 of two slots, then 2 and 3
        const uint32_t lo = __builtin_amdgcn_perm(part(1), part(0), 0x05010400);
        const uint32_t hi = __builtin_amdgcn_perm(part(1), part(0), 0x07030602);
        uint32_t w[4] = {lo, lo >> 16, hi, hi >> 16};
        if constexpr (G == 4) {
            const uint32_t lo2 = __builtin_amdgcn_perm(part(3), part(2), 0x05010400);
            const uint32_t hi2 = __builtin_amdgcn_perm(part(3), part(2), 0x07030602);
            w[0] = __builtin_amdgcn_perm(lo2, lo, 0x05040100);
            w[1] = __builtin_amdgcn_perm(lo2, lo, 0x07060302);
            w[2] = __builtin_amdgcn_perm(hi2, hi, 0x05040100);
            w[3] = __builtin_amdgcn_perm(hi2, hi, 0x07060302);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint8_t *at = to + staged_at(group, dp, d + 4 * half + e, place);
            if constexpr (G == 4)
                *(uint32_t *)at = w[e];
            else
                *(uint16_t *)(at + (place & 3)) = (uint16_t)w[e];
        }
    }
}

// One workgroup for each (sequence, block that takes new slots, kv head).  A
// thread holds eight dims of runs of 4 (ND = 1: 2) slots: read once, for the largest magnitude,
// then written as codes; values pass through shared memory into their order, and
// the groups of slots that take any are read and written whole.
// ONE: a token a sequence at most, held by a row of threads; the others are there for a block whose
// scale grows (in workgroups of a wave such a block took three times as long).  512 sequences (8 heads of 128)
// 14 us, 22 with every slot's place held by a thread; with 32 heads of queries turned beside them 21 and 35 (in
// workgroups of a wave, where no scale grows, 13).
// One token for each of 64 sequences (8 heads of 128): 6.1 us, a launch and its chain of
// dependent reads (length, table, scale, row).  Six ragged prompts of up to 2100 tokens
// (8 heads of 64, 20 MB): 12.7 us, 1.6 TB/s, the ends of a short launch.
template <int FMT, int ND, int TURN, bool ONE>   // TURN: 1 halves, 2 neighbours make a pair
__device__ inline void append(const AppendArgs &a, const TurnArgs &turned)
{
    constexpr int T = kThreads, DP = 64 * ND, CH = DP / 8, ROWS = T / CH, PASS = ONE ? 1 : kBlock / ROWS;
    __shared__ float red[2 * T / 64];
    __shared__ uint4 vl4[4 * DP];
    const int t = threadIdx.x;
    const uint32_t bt = blockIdx.x / (uint32_t)a.c.H, h = blockIdx.x % (uint32_t)a.c.H;
    const int unit_in = min(t % (CH / 2), a.c.D / 16 - 1);
    Axes axes = {};
    if (TURN) axes = axes_of(turned, 8 * unit_in);
    const int tb = (int)(bt % (uint32_t)a.touched), s = (int)(bt / (uint32_t)a.touched);
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const int len = seq_length(a.q, s);
    const int start = len - n;                      // slot of row 0; may be < 0
    const int j = max(start, 0) / kBlock + tb;
    const int lo = max(max(start, 0), j * kBlock), hi = min(len, (j + 1) * kBlock);
    if (n == 0 || lo >= hi) return;
    const int id = a.q.table[s * a.q.table_stride + j];

    const int D = a.c.D;
    const int o0 = lo - j * kBlock, o1 = hi - j * kBlock;   // slots [o0, o1) are new
    const int64_t r0 = (int64_t)row0 + (lo - start);        // row of slot o0
    const bool fresh = o0 == 0;
    const int d = 8 * (t % CH), slot0 = t / CH;
    const bool in_d = d < D;
    // a thread's slots: runs of G, whose bytes of a dim stand side by side in the values; where no more
    // than three quarters of the block's are new, those that threads side by side hold, so that none has
    // more of the new ones than another.  8 heads of 128 dims: 16 prompts of 1000 tokens by runs 24.3 us,
    // else 25.2; 17 / 33 / 48 new of one sequence, int8, by runs 9.5 / 9.1 / 9.5, else 8.1 / 7.6 / 8.2
    constexpr int G = PASS < 4 ? PASS : 4;
    const bool many = !ONE && o1 - o0 > 3 * kBlock / 4;
    auto slot_of = [&](int p) {
        if (ONE) return o0 + slot0;            // (of its rows the first is new)
        return many ? p / G * (ROWS * G) + slot0 * G + p % G : p * ROWS + slot0;
    };
    uint4 kx[ONE ? 2 : PASS], vx[PASS];
    // keys that are turned are held by units of 16 dims, twice as many slots at a time
    constexpr int UROWS = 2 * ROWS, UPASS = ONE ? 1 : PASS / 2;
    static_assert(!TURN || ONE || PASS % 2 == 0, "units of 16 dims take half the passes");
    const int unit = t % (CH / 2), uslot0 = (ONE ? o0 : 0) + t / (CH / 2);
    float ky[TURN ? UPASS : 1][16];
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
        // (a slot or dim that is not new is read as one that is: neither counts nor is
        // written)
        const int64_t r = r0 + min(max(slot_of(p), o0), o1 - 1) - o0;
        const int dd = min(d, D - 8);
        if (!TURN) kx[p] = row_bits8(a.k, (int64_t)h * a.k_head + r * a.k_row + dd, a.k_wide);
        vx[p] = row_bits8(a.v, (int64_t)h * a.v_head + r * a.v_row + dd, a.v_wide);
    }
    int ud0 = 0, ud1 = 0;
    int2 own[TURN ? UPASS : 1];
    if (TURN) {
        const int64_t own0 = a.first ? a.first[s] : start;
        unit_dims(turned, TURN == 2, unit_in, &ud0, &ud1);
#pragma unroll
        for (int p = 0; p < UPASS; ++p) {
            const int64_t r = r0 + min(max(uslot0 + p * UROWS, o0), o1 - 1) - o0;
            const int64_t at = (int64_t)h * a.k_head + r * a.k_row;
            if (turned.position)
                own[p] = positions_of(turned, a.q.n_rows, r, axes);
            else
                own[p].x = own[p].y = position_of(own0, r - row0);
            kx[2 * p] = row_bits8(a.k, at + ud0, a.k_wide);
            kx[2 * p + 1] = row_bits8(a.k, at + ud1, a.k_wide);
        }
    }
    // (all that goes by the rows is under way before the block's number is waited for)
    __builtin_amdgcn_sched_barrier(0);
    if ((unsigned)id >= (unsigned)a.c.n_blocks) return;
    const int64_t bh = (int64_t)id * a.c.H + h;
    const float oldk = fresh ? 0.f : a.c.ks[bh], oldv = fresh ? 0.f : a.c.vs[bh];
    if (TURN)
#pragma unroll
        for (int p = 0; p < UPASS; ++p) {
            const int64_t r = r0 + min(max(uslot0 + p * UROWS, o0), o1 - 1) - o0;
            turned16<TURN == 2>(turned, a.q.n_rows, (int)r, own[p], axes, a.k,
                                (int64_t)h * a.k_head + r * a.k_row, unit_in, kx[2 * p],
                                kx[2 * p + 1], a.k_type, ky[p]);
        }
    uint32_t tk = 0, tv = 0;
    float ak = 0.f;
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
        if (!TURN) tk = max(tk, magnitude8(kx[p], a.k_type));
        tv = max(tv, magnitude8(vx[p], a.v_type));
    }
    if (TURN)
#pragma unroll
        for (int p = 0; p < UPASS; ++p)
#pragma unroll
            for (int e = 0; e < 16; ++e) ak = fmaxf(ak, finite_abs(ky[p][e]));
    else
        ak = bits_value(tk, a.k_type);
    float av = bits_value(tv, a.v_type);
    max2(ak, av, red);                              // (its barrier: all have the old scales)
    const float newk = fmaxf(oldk, scale_for<FMT>(ak)), newv = fmaxf(oldv, scale_for<FMT>(av));
    if (t == 0) {
        a.c.ks[bh] = newk;
        a.c.vs[bh] = newv;
    }
    const bool growk = !fresh && newk > oldk, growv = !fresh && newv > oldv;
    const bool exk = power_of_two(newk), exv = power_of_two(newv);
    uint8_t *kc = a.c.kc + bh * kBlock * D, *vc = a.c.vc + bh * kBlock * D;
    uint8_t *vl = (uint8_t *)vl4;
    // (a decode step's one token: as bytes, without reading the group they stand in)
    const bool few = o1 - o0 == 1 && !growv;
#pragma unroll
    for (int p0 = 0; p0 < PASS; p0 += G) {
        if (!in_d) continue;
        uint2 c[G];
        // (slots beside the new ones are staged too, and not taken)
        const int o = slot_of(p0);
        const bool staged = many && o < o1 && o + G > o0;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int o = slot_of(p0 + i);
            const bool in = o >= o0 && o < o1;
            uint2 *to = (uint2 *)(kc + o * D + d);
            if (in || staged) c[i] = codes8<FMT>(vx[p0 + i], a.v_type, newv, exv);
            if (!TURN && in) *to = codes8<FMT>(kx[p0 + i], a.k_type, newk, exk);
            if (!ONE && !in && growk) {
                const uint2 w = *to;
                *to = uint2{requant4<FMT>(w.x, oldk / newk), requant4<FMT>(w.y, oldk / newk)};
            }
            if (in && !many) {
                auto byte = [&](int e) { return (uint8_t)((e < 4 ? c[i].x : c[i].y) >> (8 * (e & 3))); };
                const int g = value_group(o), place = value_place(o);
                if (few)
                    for (int e = 0; e < 8; ++e) vc[(g * D + d + e) * 16 + place] = byte(e);
                else
                    for (int e = 0; e < 8; ++e)
                        vl[staged_at(g, DP, d + e, place) + (place & 3)] = byte(e);
            }
        }
        if constexpr (!ONE)
            if (staged) stage<G>(vl, value_group(o), DP, d, value_place(o), c);
    }
    // (a token alone seldom makes a block's scale grow; then all of the block is under way at once)
    constexpr int SLOTS = ONE ? kBlock / ROWS : 1, N = 4 * DP / T;
    if (ONE && growk && in_d) {
        uint2 w[SLOTS];
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) w[k] = *(const uint2 *)(kc + (slot0 + k * ROWS) * D + d);
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const int o = slot0 + k * ROWS;
            if (o == o0) continue;
            *(uint2 *)(kc + o * D + d) =
                uint2{requant4<FMT>(w[k].x, oldk / newk), requant4<FMT>(w[k].y, oldk / newk)};
        }
    }
    uint4 held[ONE ? N : 1];
    if (ONE && !few)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int e = k * T + t, dim = e % DP;
            if (dim < D) held[k] = *(const uint4 *)(vc + (e / DP * D + dim) * 16);
        }
    if (TURN)
#pragma unroll
        for (int p = 0; p < UPASS; ++p) {
            const int o = uslot0 + p * UROWS;
            if (16 * unit >= D || o < o0 || o >= o1) continue;
            *(uint2 *)(kc + o * D + ud0) = codes_of<FMT>(ky[p], newk, exk);
            *(uint2 *)(kc + o * D + ud1) = codes_of<FMT>(ky[p] + 8, newk, exk);
        }
    if (!few) __syncthreads();
    // four dims' 16 bytes at a time: which of a group's places are new
#pragma unroll
    for (int e0 = 0; e0 < 4 * DP; e0 += T) {
        if (few) break;
        const int e = e0 + t, g = e / DP, dim = e % DP;   // (g is uniform over a wave)
        if (dim >= D) continue;
        uint32_t take[4];
        bool any = false, all = true;
        for (int q = 0; q < 4; ++q) {
            take[q] = 0;
            for (int i = 0; i < 4; ++i) {
                const int o = 16 * q + 4 * g + i;
                const bool in = o >= o0 && o < o1;
                any = any || in;
                all = all && in;
                take[q] |= in ? 0xffu << (8 * i) : 0u;
            }
        }
        if (!any && !growv) continue;
        uint4 *to = (uint4 *)(vc + (g * D + dim) * 16);
        uint4 w = vl4[staged_unit(e)];
        if (g & 1) w = uint4{w.y, w.z, w.w, w.x};
        if (g & 2) w = uint4{w.z, w.w, w.x, w.y};
        if (!all) {
            const uint4 was = ONE ? held[e0 / T] : *to;
            uint32_t x[4] = {was.x, was.y, was.z, was.w};
            const uint32_t y[4] = {w.x, w.y, w.z, w.w};
            for (int q = 0; q < 4; ++q) {
                if (growv) x[q] = requant4<FMT>(x[q], oldv / newv);
                x[q] = (x[q] & ~take[q]) | (y[q] & take[q]);
            }
            w = uint4{x[0], x[1], x[2], x[3]};
        }
        *to = w;
    }
    for (int o = o0 + t; o < o1; o += T) {
        if (a.c.pos)
            a.c.pos[bh * kBlock + o] =
                a.first ? a.first[s] + (j * kBlock + o - start) : j * kBlock + o;
        if (a.c.weight) a.c.weight[bh * kBlock + o] = 0.f;
    }
}

template <int FMT, int ND, bool ONE> __global__ __launch_bounds__(kThreads) void k_append(AppendArgs a)
{
    append<FMT, ND, 0, ONE>(a, TurnArgs{});
}

// Two bytes of a row of queries.
__device__ inline uint32_t q_bits(const TurnArgs &t, int64_t at)
{
    return ((const uint16_t *)t.q)[at];
}

// Queries, a wave to 64 units of one row: 16 dims (eight pairs, or 16 dims past the pairs) of HEADS
// heads, whose angles are the same.  A thread writes what it read, so that they may be turned in
// place.  Rows and positions are read by the row's number beside the search for its sequence.
template <bool NEIGHBOURS, int HEADS>
__device__ inline void turn_queries(const AppendArgs &a, const TurnArgs &t, uint32_t g)
{
    const int64_t item = (int64_t)g * (kThreads / 64) + (threadIdx.x >> 6);
    const int row = (int)(item / t.row_items);
    if (row >= a.q.n_rows) return;
    const int u = (int)(item % t.row_items) * 64 + (int)(threadIdx.x & 63);
    const int h0 = u / t.units * HEADS, k = u % t.units, D = a.c.D, half = t.half;
    // the unit's 16 dims are n0 from d0 on and n1 from d1 on
    const bool pairs = k < t.pair_units;
    int d0, d1, n0 = 8, n1 = 8;
    if (NEIGHBOURS) {
        d0 = 16 * k;
        d1 = d0 + 8;
    } else if (pairs) {
        d0 = 8 * k;
        d1 = half + 8 * k;
        n0 = n1 = min(8, half - d0);
    } else {
        d0 = 2 * half + 16 * (k - t.pair_units);
        d1 = d0 + 8;
        n0 = min(8, D - d0);
        n1 = max(0, min(8, D - d1));
    }
    Axes axes = {};
    if (pairs) axes = axes_of(t, 8 * k);
    uint4 lo[HEADS], hi[HEADS];
    if (t.q_wide)
#pragma unroll
        for (int r = 0; r < HEADS; ++r) {
            const int64_t from = row * t.q_row + min(h0 + r, t.n_heads - 1) * t.q_head;
            lo[r] = row_bits8(t.q, from + d0, true);
            hi[r] = row_bits8(t.q, from + d1, true);
        }
    int2 own = {0, 0};
    if (t.position) own = positions_of(t, a.q.n_rows, row, axes);
    int place;
    const int s = row_seq(a.q, row, &place);
    if (s < 0) return;
    if (!t.position) {
        int row0;
        own.x = own.y =
            position_of(a.first ? a.first[s] : seq_length(a.q, s) - seq_rows(a.q, s, &row0), place);
    }
    float c[8], s8[8];
    if (pairs) angles(t, a.q.n_rows, row, own, axes, 8 * k, c, s8);
#pragma unroll
    for (int r = 0; r < HEADS; ++r) {
        if (h0 + r >= t.n_heads) return;
        const int64_t from = row * t.q_row + (h0 + r) * t.q_head;
        float x[16];
        if (t.q_wide) {
            const uint32_t w[8] = {lo[r].x, lo[r].y, lo[r].z, lo[r].w,
                                   hi[r].x, hi[r].y, hi[r].z, hi[r].w};
            values_of<16>(w, t.q_type, x);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = e & 7, d = e < 8 ? d0 : d1;
                x[e] = i < (e < 8 ? n0 : n1) ? bits_value(q_bits(t, from + d + i), t.q_type) : 0.f;
            }
        }
        if (pairs) turn16<NEIGHBOURS>(x, c, s8, half - 8 * k, half % 8 == 0);
        uint16_t *out = (uint16_t *)t.q_out + row * t.out_row + (h0 + r) * t.out_head;
        if (t.q_wide) {
            uint32_t w[8];
            bits_of<16>(x, t.q_type, w);
            *(uint4 *)(out + d0) = uint4{w[0], w[1], w[2], w[3]};
            *(uint4 *)(out + d1) = uint4{w[4], w[5], w[6], w[7]};
            continue;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = e & 7, d = e < 8 ? d0 : d1;
            if (i < (e < 8 ? n0 : n1)) out[d + i] = row_bits(x[e], t.q_type);
        }
    }
}

constexpr int kTurnHeads = 4;             // heads a thread takes of many rows
constexpr int64_t kTurnMany = 4096;       // waves of single heads

// The keys' workgroups as in k_append, then for each row those of its queries.  A decode step's one
// token for each of 64 sequences (32 heads, 8 of keys, 128 dims): 7.0 us where k_append takes 6.1, the
// positions' and the tables' reads in its chain.  Six ragged prompts of up to 2100 tokens on three axes
// (152 MB): 34.6 us, 4.4 TB/s; calls of the keys alone 21 (k_append 17), of the queries alone 25.  Keys'
// and queries' workgroups in turn or the queries' first took 10 % longer, five workgroups to a unit 30 %.
// Angles read for each head and chunk of eight dims: 95.  By halves, heads of 65 to 128 dims, more than a
// token a sequence, spill 3 registers (int8 6) at the four waves to a SIMD that they are held to.  Keys by halves of
// a number of pairs that eight does not divide are turned dim by dim: such prompts of heads of 80 dims, 10
// or 20 pairs, 91 us where 40 pairs, or neighbours, take 28 to 31.
template <int FMT, int ND, bool NEIGHBOURS, int HEADS, bool ONE>
__global__ __launch_bounds__(kThreads, ONE || ND <= 2 ? 4 : 2)
void k_append_rotated(AppendArgs a, TurnArgs t)
{
    if (blockIdx.x < t.key_groups)
        append<FMT, ND, NEIGHBOURS ? 2 : 1, ONE>(a, t);
    else
        turn_queries<NEIGHBOURS, HEADS>(a, t, blockIdx.x - t.key_groups);
}

// -- eviction ---------------------------------------------------------------

struct EvictArgs {
    CacheArgs c;
    Seqs q;
    int32_t budget, recent, slots;      // slots: max_length in whole blocks
    uint32_t *key;                      // [seq][head][slots] (k_evict_select, R = 0)
    int32_t *src, *hole, *moved;        // [seq][head][budget]
    int32_t *newlen, *out;              // [seq]
};

// A slot's key: greater is kept first.  Protected slots above all, then the
// weights in their order, NaN last.
__device__ inline uint32_t weight_key(float w, bool safe)
{
    if (safe) return 0xffffffffu;
    if (w != w) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.f);   // -0 is 0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Which slots a (sequence, kv head) keeps, and what moves where.  One workgroup
// of T threads; wave w of them takes blocks w, w + T/64, ..., a lane to a slot,
// up to R blocks, whose keys stay in registers (R = 0: any number, keys in
// memory).  The budget-th greatest key is found in three digits from the top (11,
// 11 and 10 bits: the first covers sign, exponent and two bits of a weight, so
// that the counters of one wave's lanes seldom meet), then holes and moved slots
// are numbered in slot order from one table of counts a block.
// Bound by its barriers and the counters' atomics in shared memory, a workgroup to a CU:
// 1088 slots, 512 (sequence, head)s 12.5 us; 16000 slots, 96 of them 30 us.
constexpr int kBins = 2048;

template <int T, int R> __global__ __launch_bounds__(T) void k_evict_select(EvictArgs a)
{
    constexpr int W = T / 64, REG = R ? R : 1;
    __shared__ int hist[kBins], red[W], s_digit, s_left;
    __shared__ int table_eq[W * REG], table_hm[W * REG];
    __shared__ uint16_t moved[R ? W * REG * 32 : 1];   // (at most half of the slots)
    const int t = threadIdx.x, lane = t & 63;
    const int wv = __builtin_amdgcn_readfirstlane(t >> 6);
    const int h = (int)(blockIdx.x % (uint32_t)a.c.H), s = (int)(blockIdx.x / (uint32_t)a.c.H);
    const int len = seq_length(a.q, s);
    const int64_t sh = (int64_t)s * a.c.H + h;
    const int32_t *table = a.q.table + s * a.q.table_stride;
    int32_t *src = a.src + sh * a.budget;
    const int nb = (len + kBlock - 1) / kBlock;
    bool bad = false;                            // a block outside the pool
    auto leave = [&]() {                         // the sequence stays as it is
        if (h == 0 && t == 0) a.newlen[s] = len;
        for (int o = t; o < a.budget; o += T) src[o] = -1;
    };
    if (len <= a.budget) return leave();
    uint32_t *kmem = a.key + sh * a.slots;
    auto slot_data = [&](int j) {                // (j is uniform over the wave)
        const int id = uniform(table + j);
        const bool in = (unsigned)id < (unsigned)a.c.n_blocks;
        bad = bad || !in;
        return ((int64_t)(in ? id : 0) * a.c.H + h) * kBlock + lane;
    };
    auto largest = [&](int v) {
        for (int o = 32; o; o >>= 1) v = max(v, __shfl_xor(v, o));
        if (lane == 0) red[wv] = v;
        __syncthreads();
        for (int k = 0; k < W; ++k) v = max(v, red[k]);
        return v;
    };
    // the newest position, then the keys
    uint32_t key[REG];
    int newest = INT32_MIN;
    if (R) {
        // eight blocks at a time; past the last one it is read again (unused)
        constexpr int U = REG < 8 ? REG : 8;
        int pos[U];
        float w[U];
        for (int r0 = 0; r0 < REG; r0 += U) {
            if (r0 * W >= nb) break;
            for (int u = 0; u < U; ++u) {
                const int64_t at = slot_data(min((r0 + u) * W + wv, nb - 1));
                pos[u] = a.c.pos[at];
                if (REG == U) w[u] = a.c.weight[at];
            }
            for (int u = 0; u < U; ++u)
                newest = max(newest, ((r0 + u) * W + wv) * kBlock + lane < len ? pos[u] : INT32_MIN);
        }
        newest = largest(newest);
        const int64_t over = (int64_t)newest - a.recent;
        for (int r0 = 0; r0 < REG; r0 += U) {
            for (int u = 0; u < U; ++u) key[r0 + u] = 0;
            if (r0 * W >= nb) continue;
            for (int u = 0; u < U && REG > U; ++u) {
                const int64_t at = slot_data(min((r0 + u) * W + wv, nb - 1));
                w[u] = a.c.weight[at];
                pos[u] = a.c.pos[at];
            }
            for (int u = 0; u < U; ++u)
                if (((r0 + u) * W + wv) * kBlock + lane < len)
                    key[r0 + u] = weight_key(w[u], (int64_t)pos[u] > over);
        }
    } else {
        for (int j = wv; j < nb; j += W)
            if (j * kBlock + lane < len) newest = max(newest, a.c.pos[slot_data(j)]);
        newest = largest(newest);
        const int64_t over = (int64_t)newest - a.recent;
        for (int j = wv; j < nb; j += W)
            if (j * kBlock + lane < len) {
                const int64_t at = slot_data(j);
                kmem[j * kBlock + lane] =
                    weight_key(a.c.weight[at], (int64_t)a.c.pos[at] > over);
            }
    }
    if (__syncthreads_or(bad)) return leave();
    if (h == 0 && t == 0) a.newlen[s] = a.budget;
    // f(key, slot, block) for each of the wave's blocks, in order
    auto each = [&](auto &&f) {
        if (R) {
            for (int r = 0; r < REG; ++r) {
                if (r * W >= nb) break;
                f(key[r], (r * W + wv) * kBlock + lane, r * W + wv);
            }
        } else {
            for (int j = wv; j < nb; j += W)
                f(j * kBlock + lane < len ? kmem[j * kBlock + lane] : 0u, j * kBlock + lane, j);
        }
    };
    // p: the greatest key that at least `budget` keys reach; spare: of the keys
    // equal to it, those that stay (the first in slot order)
    uint32_t p = 0;
    int spare = a.budget;
    constexpr int B = kBins / T;                 // bins of a thread, from the top
    for (int b = 0; b < B; ++b) hist[b * T + t] = 0;
    __syncthreads();
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
        const int bins = round == 2 ? kBins / 2 : kBins;
        each([&](uint32_t x, int o, int) {
            const uint32_t digit = x >> shift & (bins - 1);
            const uint64_t in = __ballot(
                o < len && (round == 0 || (x ^ p) >> (round == 1 ? 21 : 10) == 0));
            if (!in) return;
            // (equal weights, protected slots: one count for all)
            const uint32_t one = __builtin_amdgcn_readlane(digit, __ffsll((long long)in) - 1);
            if ((__ballot(digit == one) & in) == in) {
                if (lane == 0) atomicAdd(&hist[one], (int)__popcll(in));
            } else if (in >> lane & 1) {
                atomicAdd(&hist[digit], 1);
            }
        });
        __syncthreads();
        int c[B], sum = 0;
        for (int b = 0; b < B; ++b) {
            const int bin = kBins - 1 - (t * B + b);
            sum += c[b] = hist[bin];
            hist[bin] = 0;
        }
        int run = sum;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(run, o);
            run += lane >= o ? v : 0;
        }
        if (lane == 63) red[wv] = run;
        __syncthreads();
        int over = run - sum;                    // keys in the bins above this thread's
        for (int k = 0; k < W; ++k) over += k < wv ? red[k] : 0;
        if (over < spare && over + sum >= spare) {
            int b = 0;
            for (; over + c[b] < spare; ++b) over += c[b];
            s_digit = kBins - 1 - (t * B + b);
            s_left = spare - over;
        }
        __syncthreads();
        p |= (uint32_t)s_digit << shift;
        spare = s_left;
    }
    const uint64_t under = (1ull << lane) - 1;
    if (R) {
        // counts a block, their running sums by the first wave, then the ranks
        auto running = [&](int *table_) {
            constexpr int PER = (W * REG + 63) / 64;
            __syncthreads();
            if (wv == 0) {
                int v[PER], sum = 0;
                for (int k = 0; k < PER; ++k) {
                    const int i = lane * PER + k;
                    v[k] = i < W * REG ? table_[i] : 0;
                    sum += v[k];
                }
                int run = sum;
                for (int o = 1; o < 64; o <<= 1) {
                    const int x = __shfl_up(run, o);
                    run += lane >= o ? x : 0;
                }
                run -= sum;
                for (int k = 0; k < PER; ++k) {
                    if (lane * PER + k < W * REG) table_[lane * PER + k] = run;
                    run += v[k];
                }
            }
            __syncthreads();
        };
        each([&](uint32_t x, int o, int j) {
            const int c = __popcll(__ballot(o < len && x == p));
            if (lane == 0) table_eq[j] = c;
        });
        running(table_eq);
        uint32_t keeps = 0;                      // (a bit for each r; R <= 32)
        int r = 0;
        each([&](uint32_t x, int o, int j) {
            const uint64_t eq = __ballot(o < len && x == p);
            const int rank = table_eq[j] + __popcll(eq & under);
            const bool keep = o < len && (x > p || (x == p && rank < spare));
            keeps |= (uint32_t)keep << r++;
            // holes below the budget, moved slots past it (a block is one or the other)
            const uint64_t m = __ballot(o < a.budget ? !keep : keep);
            if (lane == 0) table_hm[j] = __popcll(m);
        });
        // the two kinds are numbered by themselves: blocks below the budget hold holes
        running(table_hm);
        const int first = a.budget / kBlock;     // (there is such a block: len > budget)
        const int holes = table_hm[first];
        r = 0;
        each([&](uint32_t, int o, int j) {
            const bool keep = keeps >> r++ & 1;
            const bool it = o < a.budget ? !keep : keep;
            const uint64_t m = __ballot(it);
            const int rank = table_hm[j] + __popcll(m & under);
            if (it && o >= a.budget) moved[rank - holes] = (uint16_t)o;
        });
        __syncthreads();
        r = 0;
        each([&](uint32_t, int o, int j) {
            const bool keep = keeps >> r++ & 1;
            const uint64_t m = __ballot(!keep);
            if (o < a.budget) src[o] = keep ? -1 : moved[table_hm[j] + __popcll(m & under)];
        });
    } else {
        int32_t *hole = a.hole + sh * a.budget, *shift = a.moved + sh * a.budget;
        // (many blocks: wave by wave in slot order would be one wave's walk, so T
        // slots at a time)
        int n_eq = 0, n_hole = 0, n_moved = 0;
        auto rank_of = [&](bool f, int *base) {
            const uint64_t m = __ballot(f);
            __syncthreads();
            if (lane == 0) red[wv] = __popcll(m);
            __syncthreads();
            int before = *base, total = 0;
            for (int k = 0; k < W; ++k) {
                before += k < wv ? red[k] : 0;
                total += red[k];
            }
            *base += total;
            return before + __popcll(m & under);
        };
        for (int b = 0; b < len; b += T) {
            const int o = b + t;
            const uint32_t x = o < len ? kmem[o] : 0;
            const bool eq = o < len && x == p;
            const int rank = rank_of(eq, &n_eq);
            const bool keep = o < len && (x > p || (eq && rank < spare));
            const bool is_hole = o < a.budget && !keep, is_moved = o >= a.budget && keep;
            const int rh = rank_of(is_hole, &n_hole), rm = rank_of(is_moved, &n_moved);
            if (o < a.budget) src[o] = -1;
            if (is_hole) hole[rh] = o;
            if (is_moved) shift[rm] = o;
        }
        __syncthreads();
        for (int i = t; i < min(n_hole, n_moved); i += T) src[hole[i]] = shift[i];
    }
}

// One workgroup for each (sequence, block below the budget, kv head): WPB waves,
// each with 4 / WPB groups of 16 slots (qlm.h's order of the values).  A wave fetches
// what moves into its groups' holes, four tokens at a time and one token's address
// for a load, into shared memory (fetching it again for the second pass instead
// took half as long again); the waves agree on the block's scales and write.
// A lane holds ND neighbouring dims of a key and dims lane, lane + 64, ... of a
// value, whose bytes stand 16 apart: a group that takes a token is read and
// written whole (2 KiB at 128 dims; writing single bytes took as long).
// Bound by that traffic: 64 tokens moved of 1024, 512 (sequence, head)s 32 us, where
// the tokens alone are 4.4 us; ragged prompts of up to 16000 cut to 2048, 96 of them 48 us.
template <int ND> struct DimsOf;                // ND codes of a key
template <> struct DimsOf<1> { typedef uint8_t type; };
template <> struct DimsOf<2> { typedef uint16_t type; };
template <> struct DimsOf<4> { typedef uint32_t type; };

template <int FMT, int ND, int WPB> __global__ __launch_bounds__(64 * WPB) void k_evict_move(EvictArgs a)
{
    typedef typename DimsOf<ND>::type dims;
    __shared__ float red[2 * WPB];
    extern __shared__ uint4 moving[];           // incoming codes, laid out as a block's
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t nb = a.budget / kBlock;
    const uint32_t sh = blockIdx.x / nb, j = blockIdx.x % nb;
    const uint32_t s = sh / (uint32_t)a.c.H, h = sh % (uint32_t)a.c.H;
    const int D = a.c.D;
    if (h == 0 && j == 0 && threadIdx.x == 0) a.out[s] = a.newlen[s];
    const int32_t *table = a.q.table + s * a.q.table_stride;
    // lane l: where slot l's new token comes from (blocks past the budget: not
    // written here)
    const int mine = a.src[(int64_t)sh * a.budget + j * kBlock + lane];
    const uint64_t holes = __ballot(mine >= 0); // (both waves read the same 64)
    if (!holes) return;
    const int id = mine >= 0 ? table[mine >> 6] : 0;
    const float sk = a.c.ks[(int64_t)id * a.c.H + h], sv = a.c.vs[(int64_t)id * a.c.H + h];
    const int64_t bh = (int64_t)uniform(table + j) * a.c.H + h;
    const float oldk = a.c.ks[bh], oldv = a.c.vs[bh];
    auto lane_of = [](float x, int l) {
        return __builtin_bit_cast(float,
                                  __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l));
    };
    uint8_t *kl = (uint8_t *)moving, *vl = kl + kBlock * D;
    const uint64_t slots_of = (WPB == 2 ? 0x00ff00ff00ff00ffull : 0x000f000f000f000full)
                              << (16 / WPB * wv);
    const bool in_k = lane * ND < D;            // (D is a multiple of 16)
    float ak = 0.f, av = 0.f;
    for (uint64_t left = holes & slots_of; left;) {
        // (the first again where there are fewer than four: a branch would hold each
        // load back until the one before)
        int slot[4];
        uint32_t kx[4], vx[4][ND];
        for (int u = 0; u < 4; ++u) {
            slot[u] = left ? __ffsll((long long)left) - 1 : slot[0];
            left &= left - 1;
            const int o = __builtin_amdgcn_readlane(mine, slot[u]) & 63;
            const int64_t b = (int64_t)__builtin_amdgcn_readlane(id, slot[u]) * a.c.H + h;
            const uint8_t *kp = a.c.kc + (b * kBlock + o) * D;
            const uint8_t *vp = a.c.vc + b * kBlock * D + value_group(o) * D * 16 + value_place(o);
            // (past the last dim the last is read again: neither counts nor is written)
            kx[u] = *(const dims *)(kp + (uint32_t)min(lane * ND, D - ND));
            for (int k = 0; k < ND; ++k) vx[u][k] = vp[(uint32_t)min(lane + 64 * k, D - 1) * 16];
        }
        for (int u = 0; u < 4; ++u) {
            uint32_t tk = 0, tv = 0;
            uint8_t *to = vl + value_group(slot[u]) * D * 16 + value_place(slot[u]);
            for (int k = 0; k < ND; ++k) {
                tk = max(tk, magnitude<FMT>(kx[u] >> (8 * k)));
                tv = max(tv, magnitude<FMT>(vx[u][k]));
                if (lane + 64 * k < D) to[(lane + 64 * k) * 16] = (uint8_t)vx[u][k];
            }
            if (in_k) *(dims *)(kl + slot[u] * D + lane * ND) = (dims)kx[u];
            ak = fmaxf(ak, finite_abs(code_value<FMT>(tk) * lane_of(sk, slot[u])));
            av = fmaxf(av, finite_abs(code_value<FMT>(tv) * lane_of(sv, slot[u])));
        }
    }
    max2(ak, av, red);                          // (its barrier: every wave has the old scales)
    const float newk = fmaxf(oldk, scale_for<FMT>(ak)), newv = fmaxf(oldv, scale_for<FMT>(av));
    if (threadIdx.x == 0) {
        a.c.ks[bh] = newk;
        a.c.vs[bh] = newv;
    }
    uint8_t *kc = a.c.kc + bh * kBlock * D, *vc = a.c.vc + bh * kBlock * D;
    const bool growv = newv > oldv;
    for (uint64_t left = holes & slots_of; left; left &= left - 1) {
        const int slot = __ffsll((long long)left) - 1;
        const float fk = lane_of(sk, slot), fv = lane_of(sv, slot);
        if (in_k) {
            uint32_t x = *(dims *)(kl + slot * D + lane * ND);
            if (fk != newk) x = rescale4<FMT>(x, fk, newk);
            *(dims *)(kc + slot * D + lane * ND) = (dims)x;
        }
        if (fv != newv)
            for (int d = lane; d < D; d += 64) {
                uint8_t *x = vl + (value_group(slot) * D + d) * 16 + value_place(slot);
                *x = (uint8_t)rescale4<FMT>(*x, fv, newv);
            }
    }
    if (newk > oldk && in_k)
        for (uint64_t left = ~holes & slots_of; left; left &= left - 1) {
            dims *x = (dims *)(kc + (__ffsll((long long)left) - 1) * D + lane * ND);
            *x = (dims)requant4<FMT>(*x, oldk / newk);
        }
    const float ratio = oldv / newv;
    for (int g = wv * (4 / WPB); g < (wv + 1) * (4 / WPB); ++g) {
        const uint64_t in_g = holes & 0x000f000f000f000full << (4 * g);
        if (!in_g && !growv) continue;
        uint32_t take[4];                        // the bytes of the holes, place after place
        for (int q = 0; q < 4; ++q) {
            const uint32_t n = (uint32_t)(in_g >> (16 * q + 4 * g)) & 15u;
            take[q] = ((n & 1) | (n & 2) << 7 | (n & 4) << 14 | (n & 8) << 21) * 0xffu;
        }
        for (int d = lane; d < D; d += 64) {     // (the lane that wrote these bytes)
            uint4 *to = (uint4 *)(vc + (g * D + d) * 16);
            const uint4 w = *to, x = *(const uint4 *)(vl + (g * D + d) * 16);
            uint32_t o[4] = {w.x, w.y, w.z, w.w};
            const uint32_t n[4] = {x.x, x.y, x.z, x.w};
            for (int q = 0; q < 4; ++q) {
                if (growv) o[q] = requant4<FMT>(o[q], ratio);
                o[q] = (o[q] & ~take[q]) | (n[q] & take[q]);
            }
            *to = uint4{o[0], o[1], o[2], o[3]};
        }
    }
    if (wv == 0 && mine >= 0) {
        const int64_t to = bh * kBlock + lane;
        const int64_t fr = ((int64_t)id * a.c.H + h) * kBlock + (mine & 63);
        a.c.pos[to] = a.c.pos[fr];
        a.c.weight[to] = a.c.weight[fr];
    }
}

template <int FMT, int ND> void launch_move(const EvictArgs &a, int waves, unsigned grid,
                                            hipStream_t st)
{
    const int bytes = 2 * kBlock * a.c.D;
    if (waves == 2)
        k_evict_move<FMT, ND, 2><<<grid, 128, bytes, st>>>(a);
    else
        k_evict_move<FMT, ND, 4><<<grid, 256, bytes, st>>>(a);
}

template <int FMT> void launch_move(const EvictArgs &a, int waves, unsigned grid, hipStream_t st)
{
    if (a.c.D <= 64)
        launch_move<FMT, 1>(a, waves, grid, st);
    else if (a.c.D <= 128)
        launch_move<FMT, 2>(a, waves, grid, st);
    else
        launch_move<FMT, 4>(a, waves, grid, st);
}

// Waves to a block of k_evict_move.
int move_waves(int max_length, int budget)
{
    // two waves to a block where at most a quarter of its slots can fall free (4 of
    // 64, 8192 blocks: 31 us, four waves 36), four where more can (48 of 64: 48 us,
    // two waves 62)
    return max_length - budget <= budget / 4 ? 2 : 4;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

struct EvictLayout {
    size_t key, src, hole, moved, newlen, total;
};

EvictLayout evict_layout(const qlm_kv_cache *c, const qlm_kv_batch *b, int32_t budget)
{
    const size_t sh = (size_t)b->n_seqs * c->n_kv_heads;
    const size_t slots = ((size_t)b->max_length + kBlock - 1) / kBlock * kBlock;
    EvictLayout l{};
    l.key = 0;
    l.src = l.key + (slots > kBlock * 16 * 32 ? align256(sh * slots * 4) : 0);
    l.hole = l.src + align256(sh * budget * 4);
    l.moved = l.hole + align256(sh * budget * 4);
    l.newlen = l.moved + align256(sh * budget * 4);
    l.total = l.newlen + align256((size_t)b->n_seqs * 4);
    return l;
}

// Whether rows may be read and written 16 bytes at a time.
bool rows_wide(const qlm_rows *r)
{
    return (uintptr_t)r->data % 16 == 0 && r->row_stride % 8 == 0 && r->head_stride % 8 == 0;
}

AppendArgs append_args(const qlm_kv_cache *cache, const qlm_kv_batch *batch, const qlm_rows *k,
                       const qlm_rows *v, const int32_t *first_position)
{
    AppendArgs a{};
    a.c = cache_args(cache);
    a.q = seqs_of(batch);
    a.k = k->data;
    a.v = v->data;
    a.k_row = k->row_stride;
    a.k_head = k->head_stride;
    a.v_row = v->row_stride;
    a.v_head = v->head_stride;
    a.k_type = k->dtype;
    a.v_type = v->dtype;
    a.first = first_position;
    // new slots that start anywhere in a block
    const int64_t most = ((int64_t)batch->max_new + kBlock - 2) / kBlock + 1;
    const int64_t have = ((int64_t)batch->max_length + kBlock - 1) / kBlock;
    a.touched = (int32_t)(most < have ? most : have);
    a.k_wide = rows_wide(k);
    a.v_wide = rows_wide(v);
    return a;
}

int64_t append_groups(const AppendArgs &a, const qlm_kv_batch *batch)
{
    return (int64_t)batch->n_seqs * a.touched * a.c.H;
}

template <int FMT, bool NEIGHBOURS, bool ONE>
void launch_rotated(const AppendArgs &a, const TurnArgs &t, bool many, int64_t grid,
                    hipStream_t stream)
{
    constexpr int H = kTurnHeads;
    auto kern = a.c.D <= 64    ? many ? k_append_rotated<FMT, 1, NEIGHBOURS, H, ONE>
                                      : k_append_rotated<FMT, 1, NEIGHBOURS, 1, ONE>
                : a.c.D <= 128 ? many ? k_append_rotated<FMT, 2, NEIGHBOURS, H, ONE>
                                      : k_append_rotated<FMT, 2, NEIGHBOURS, 1, ONE>
                : many         ? k_append_rotated<FMT, 4, NEIGHBOURS, H, ONE>
                               : k_append_rotated<FMT, 4, NEIGHBOURS, 1, ONE>;
    kern<<<(unsigned)grid, kThreads, 0, stream>>>(a, t);
}

template <bool ONE> void launch_append(const AppendArgs &a, bool e4m3, int64_t grid, hipStream_t stream)
{
    constexpr int E = QLM_KV_E4M3, I = QLM_KV_INT8;
    auto kern = a.c.D <= 64    ? e4m3 ? k_append<E, 1, ONE> : k_append<I, 1, ONE>
                : a.c.D <= 128 ? e4m3 ? k_append<E, 2, ONE> : k_append<I, 2, ONE>
                               : e4m3 ? k_append<E, 4, ONE> : k_append<I, 4, ONE>;
    kern<<<(unsigned)grid, kThreads, 0, stream>>>(a);
}

int check_rotary(const qlm_rotary *r, int head_dim)
{
    if (!r) return fail(QLM_ERR_ARG, "rotary is NULL");
    if (r->rotary_dim < 2 || r->rotary_dim > head_dim || r->rotary_dim % 2)
        return fail(QLM_ERR_ARG, "rotary_dim must be even, in 2..head_dim");
    if (r->n_positions < 1) return fail(QLM_ERR_ARG, "n_positions must be >= 1");
    if (r->n_axes < 1 || r->n_axes > 4) return fail(QLM_ERR_ARG, "n_axes must be in 1..4");
    if (!r->position && r->n_axes != 1)
        return fail(QLM_ERR_ARG, "position is required with more than one axis");
    if (!r->cos || !r->sin) return fail(QLM_ERR_ARG, "cos and sin are required");
    if ((uintptr_t)r->cos % 4 || (uintptr_t)r->sin % 4)
        return fail(QLM_ERR_ARG, "cos or sin is misaligned");
    return QLM_OK;
}

}  // namespace

extern "C" {

int qlm_kv_append(const qlm_kv_cache *cache, const qlm_kv_batch *batch, const qlm_rows *k,
                  const qlm_rows *v, const int32_t *first_position, qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    int rc = check_cache(cache);
    if (!rc) rc = check_batch(batch);
    if (rc) return rc;
    if (batch->n_seqs == 0 || batch->n_rows == 0 || batch->max_length == 0) return QLM_OK;
    if ((rc = check_rows(k, "k")) || (rc = check_rows(v, "v"))) return rc;
    const AppendArgs a = append_args(cache, batch, k, v, first_position);
    const int64_t grid = append_groups(a, batch);
    if (!can_launch(grid, kThreads)) return fail(QLM_ERR_CAPACITY, "too many blocks in one append");
    const bool e4m3 = cache->format == QLM_KV_E4M3;
    if (batch->max_new == 1)
        launch_append<true>(a, e4m3, grid, stream);
    else
        launch_append<false>(a, e4m3, grid, stream);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_append launch");
}

int qlm_kv_append_rotated(const qlm_kv_cache *cache, const qlm_kv_batch *batch, const qlm_rows *k,
                          const qlm_rows *v, const qlm_rows *q, const qlm_rows *q_out,
                          int32_t n_heads, const qlm_rotary *rotary,
                          const int32_t *first_position, qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    int rc = check_cache(cache);
    if (!rc) rc = check_batch(batch);
    if (!rc) rc = check_rotary(rotary, cache->head_dim);
    if (rc) return rc;
    if (n_heads < 0 || n_heads > (1 << 16)) return fail(QLM_ERR_ARG, "n_heads must be in 0..65536");
    if (n_heads == 0 && (q || q_out)) return fail(QLM_ERR_ARG, "q and q_out must be NULL without heads");
    if (batch->n_seqs == 0 || batch->n_rows == 0) return QLM_OK;
    if ((rc = check_rows(k, "k")) || (rc = check_rows(v, "v"))) return rc;
    if (n_heads > 0) {
        if ((rc = check_rows(q, "q")) || (rc = check_rows(q_out, "q_out"))) return rc;
        if (q->dtype != q_out->dtype) return fail(QLM_ERR_ARG, "q and q_out must have one dtype");
        const bool same = q->data == q_out->data;
        if (same && (q->row_stride != q_out->row_stride || q->head_stride != q_out->head_stride))
            return fail(QLM_ERR_ARG, "q_out in the place of q must have its strides");
        if (q_out->data == k->data || q_out->data == v->data)
            return fail(QLM_ERR_ARG, "q_out may not overlap k or v");
    }
    const AppendArgs a = append_args(cache, batch, k, v, first_position);
    TurnArgs t{};
    t.cos = rotary->cos;
    t.sin = rotary->sin;
    t.axis = rotary->axis;
    t.position = rotary->position;
    t.half = rotary->rotary_dim / 2;
    t.n_positions = rotary->n_positions;
    t.n_axes = rotary->n_axes;
    t.table_wide = t.half % 4 == 0 && (uintptr_t)t.cos % 16 == 0 && (uintptr_t)t.sin % 16 == 0 &&
                   (uintptr_t)t.axis % 16 == 0;
    const bool neighbours = rotary->interleaved != 0;
    const int64_t keys = batch->max_length > 0 ? append_groups(a, batch) : 0;
    t.n_heads = n_heads;
    t.pair_units = (t.half + 7) / 8;
    t.units = neighbours ? a.c.D / 16 : t.pair_units + (a.c.D - 2 * t.half + 15) / 16;
    if (n_heads > 0) {
        t.q = q->data;
        t.q_out = q_out->data;
        t.q_row = q->row_stride;
        t.q_head = q->head_stride;
        t.out_row = q_out->row_stride;
        t.out_head = q_out->head_stride;
        t.q_type = q->dtype;
        t.q_wide = rows_wide(q) && rows_wide(q_out) && (neighbours || t.half % 8 == 0);
    }
    auto items = [&](int heads) {
        return (uint32_t)(((int64_t)(n_heads + heads - 1) / heads * t.units + 63) / 64);
    };
    t.row_items = items(1);
    const bool many = (int64_t)batch->n_rows * t.row_items > kTurnMany;
    if (many) t.row_items = items(kTurnHeads);
    const bool one = batch->max_new == 1;
    const int64_t queries = ((int64_t)batch->n_rows * t.row_items + kThreads / 64 - 1) / (kThreads / 64);
    const int64_t grid = keys + queries;
    if (!can_launch(grid, kThreads)) return fail(QLM_ERR_CAPACITY, "too many rows in one append");
    if (grid == 0) return QLM_OK;
    t.key_groups = (uint32_t)keys;
    constexpr int E = QLM_KV_E4M3, I = QLM_KV_INT8;
    const bool e4m3 = cache->format == E;
    auto launch = [&](auto turn, auto alone) {
        constexpr bool N = decltype(turn)::value, ONE = decltype(alone)::value;
        e4m3 ? launch_rotated<E, N, ONE>(a, t, many, grid, stream)
             : launch_rotated<I, N, ONE>(a, t, many, grid, stream);
    };
    if (neighbours)
        one ? launch(std::true_type{}, std::true_type{}) : launch(std::true_type{}, std::false_type{});
    else
        one ? launch(std::false_type{}, std::true_type{}) : launch(std::false_type{}, std::false_type{});
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_append_rotated launch");
}

size_t qlm_kv_evict_workspace_bytes(const qlm_kv_cache *cache, const qlm_kv_batch *batch,
                                    int32_t budget)
{
    if (!cache || !batch || batch->n_seqs <= 0 || cache->n_kv_heads <= 0 || budget <= 0 ||
        batch->max_length < 0)
        return 0;
    return evict_layout(cache, batch, budget).total;
}

int qlm_kv_evict(const qlm_kv_cache *cache, const qlm_kv_batch *batch, int32_t budget,
                 int32_t recent, int32_t *lengths_out, void *ws, size_t ws_bytes,
                 qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    int rc = check_cache(cache);
    if (!rc) rc = check_batch(batch);
    if (rc) return rc;
    if (!cache->position || !cache->weight)
        return fail(QLM_ERR_ARG, "eviction needs a cache that keeps positions and weights");
    if (budget < kBlock || budget % kBlock)
        return fail(QLM_ERR_ARG, "budget must be a multiple of 64, >= 64");
    if (recent < 0 || recent > budget)
        return fail(QLM_ERR_ARG, "recent must be in 0..budget");
    if (batch->n_seqs == 0) return QLM_OK;
    if (!lengths_out) return fail(QLM_ERR_ARG, "lengths_out is NULL");
    const EvictLayout l = evict_layout(cache, batch, budget);
    rc = check_workspace(ws, ws_bytes, l.total);
    if (rc) return rc;
    EvictArgs a{};
    a.c = cache_args(cache);
    a.q = seqs_of(batch);
    a.budget = budget;
    a.recent = recent;
    a.slots = (batch->max_length + kBlock - 1) / kBlock * kBlock;
    char *p = (char *)ws;
    a.key = (uint32_t *)(p + l.key);
    a.src = (int32_t *)(p + l.src);
    a.hole = (int32_t *)(p + l.hole);
    a.moved = (int32_t *)(p + l.moved);
    a.newlen = (int32_t *)(p + l.newlen);
    a.out = lengths_out;
    const int64_t sh = (int64_t)batch->n_seqs * a.c.H;
    const int64_t grid = sh * (budget / kBlock);
    const int blocks = a.slots / kBlock;        // of the longest sequence
    const int waves = move_waves(batch->max_length, budget);
    if (!can_launch(grid, 64 * waves) || !can_launch(sh, blocks <= 4 * 8 ? 256 : 1024))
        return fail(QLM_ERR_CAPACITY, "too many blocks in one eviction");
    const unsigned n = (unsigned)sh;
    // few blocks: four waves, more workgroups to a CU (64 sequences of 2048, 8 heads, with
    // the move 21 us; sixteen waves 26; 128 of 512 17 and 35; 8 of 1024 11 and 11)
    if (blocks <= 4 * 8)
        k_evict_select<256, 8><<<n, 256, 0, stream>>>(a);
    else if (blocks <= 16 * 8)
        k_evict_select<1024, 8><<<n, 1024, 0, stream>>>(a);
    else if (blocks <= 16 * 16)
        k_evict_select<1024, 16><<<n, 1024, 0, stream>>>(a);
    else if (blocks <= 16 * 32)
        k_evict_select<1024, 32><<<n, 1024, 0, stream>>>(a);
    else
        k_evict_select<1024, 0><<<n, 1024, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "k_evict_select launch");
    if (cache->format == QLM_KV_E4M3)
        launch_move<QLM_KV_E4M3>(a, waves, (unsigned)grid, stream);
    else
        launch_move<QLM_KV_INT8>(a, waves, (unsigned)grid, stream);
    e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_evict_move launch");
}

}  // extern "C"

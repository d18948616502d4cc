// kv.hip -- the 8-bit token cache: writing new tokens (qlm_kv_append) and
// cutting sequences to a budget by accumulated attention weight (qlm_kv_evict).
// The definitions stand in include/qlm.h.
#include "kv.h"

#include <string>

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

// Eight dims as codes over `scale` (a power of two nearly always: a product then).
template <int FMT> __device__ inline uint2 codes8(uint4 x, int dtype, float scale, bool exact)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const float by = 1.f / scale;
    uint32_t o[2] = {0, 0};
    for (int i = 0; i < 8; ++i) {
        const float v = bits_value((w[i >> 1] >> (16 * (i & 1))) & 0xffff, dtype);
        o[i >> 2] |= code_of<FMT>(exact ? v * by : v / scale) << (8 * (i & 3));
    }
    return {o[0], o[1]};
}

__device__ inline bool power_of_two(float x)
{
    return (__builtin_bit_cast(uint32_t, x) & 0x7fffffu) == 0;
}

// One workgroup for each (sequence, block that takes new slots, kv head).  A
// thread holds eight dims of every (32 / ND)-th slot: read once, for the largest magnitude,
// then written as codes; values pass through shared memory into their order, and
// the groups of slots that take any are read and written whole.
// One token for each of 64 sequences (8 heads of 128): 7 us, a launch and its chain of
// dependent reads (length, table, scale, row).  Six ragged prompts of up to 2100 tokens
// (8 heads of 64, 20 MB): 12.5 us, 1.6 TB/s, the ends of a short launch and the pass
// through shared memory.
template <int FMT, int ND> __global__ __launch_bounds__(kThreads) void k_append(AppendArgs a)
{
    constexpr int DP = 64 * ND, CH = DP / 8, ROWS = kThreads / CH, PASS = kBlock / ROWS;
    __shared__ float red[2 * kThreads / 64];
    __shared__ uint4 vl4[4 * DP];
    const int t = threadIdx.x;
    const uint32_t bt = blockIdx.x / (uint32_t)a.c.H, h = blockIdx.x % (uint32_t)a.c.H;
    const int tb = (int)(bt % (uint32_t)a.touched), s = (int)(bt / (uint32_t)a.touched);
    int row0;
    const int n = seq_rows(a.q, s, &row0);
    const int len = seq_length(a.q, s);
    const int start = len - n;                      // slot of row 0; may be < 0
    const int j = max(start, 0) / kBlock + tb;
    const int lo = max(max(start, 0), j * kBlock), hi = min(len, (j + 1) * kBlock);
    if (n == 0 || lo >= hi) return;
    const int id = a.q.table[s * a.q.table_stride + j];
    if ((unsigned)id >= (unsigned)a.c.n_blocks) return;

    const int D = a.c.D;
    const int o0 = lo - j * kBlock, o1 = hi - j * kBlock;   // slots [o0, o1) are new
    const int64_t r0 = (int64_t)row0 + (lo - start);        // row of slot o0
    const int64_t bh = (int64_t)id * a.c.H + h;
    const bool fresh = o0 == 0;
    const float oldk = fresh ? 0.f : a.c.ks[bh], oldv = fresh ? 0.f : a.c.vs[bh];
    const int d = 8 * (t % CH), slot0 = t / CH;
    const bool in_d = d < D;
    uint4 kx[PASS], vx[PASS];
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
        // (a slot or dim that is not new is read as one that is: neither counts nor is
        // written)
        const int64_t r = r0 + min(max(slot0 + p * ROWS, o0), o1 - 1) - o0;
        const int dd = min(d, D - 8);
        kx[p] = row_bits8(a.k, (int64_t)h * a.k_head + r * a.k_row + dd, a.k_wide);
        vx[p] = row_bits8(a.v, (int64_t)h * a.v_head + r * a.v_row + dd, a.v_wide);
    }
    uint32_t tk = 0, tv = 0;
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
        tk = max(tk, magnitude8(kx[p], a.k_type));
        tv = max(tv, magnitude8(vx[p], a.v_type));
    }
    float ak = bits_value(tk, a.k_type), av = bits_value(tv, a.v_type);
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
    for (int p = 0; p < PASS; ++p) {
        const int o = slot0 + p * ROWS;
        if (!in_d) continue;
        uint2 *to = (uint2 *)(kc + o * D + d);
        if (o >= o0 && o < o1) {
            *to = codes8<FMT>(kx[p], a.k_type, newk, exk);
            const uint2 c = codes8<FMT>(vx[p], a.v_type, newv, exv);
            uint8_t *at = few ? vc + (value_group(o) * D + d) * 16 + value_place(o)
                              : vl + (value_group(o) * DP + d) * 16 + value_place(o);
            for (int e = 0; e < 8; ++e) at[16 * e] = (uint8_t)((e < 4 ? c.x : c.y) >> (8 * (e & 3)));
        } else if (growk) {
            const uint2 w = *to;
            *to = uint2{requant4<FMT>(w.x, oldk / newk), requant4<FMT>(w.y, oldk / newk)};
        }
    }
    if (!few) __syncthreads();
    // four dims' 16 bytes at a time: which of a group's places are new
#pragma unroll
    for (int e0 = 0; e0 < 4 * DP; e0 += kThreads) {
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
        uint4 w = vl4[e];
        if (!all) {
            const uint4 was = *to;
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
    for (int o = o0 + t; o < o1; o += kThreads) {
        if (a.c.pos)
            a.c.pos[bh * kBlock + o] =
                a.first ? a.first[s] + (j * kBlock + o - start) : j * kBlock + o;
        if (a.c.weight) a.c.weight[bh * kBlock + o] = 0.f;
    }
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
    // 64, 8192 blocks: 31 us, four waves 36), four where more can (48 of 64, 3072
    // blocks: 48 us, two waves 62)
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
    const int64_t grid = (int64_t)batch->n_seqs * a.touched * a.c.H;
    if (!can_launch(grid, kThreads)) return fail(QLM_ERR_CAPACITY, "too many blocks in one append");
    a.k_wide = (uintptr_t)a.k % 16 == 0 && a.k_row % 8 == 0 && a.k_head % 8 == 0;
    a.v_wide = (uintptr_t)a.v % 16 == 0 && a.v_row % 8 == 0 && a.v_head % 8 == 0;
    const bool e4m3 = cache->format == QLM_KV_E4M3;
    auto kern = a.c.D <= 64    ? e4m3 ? k_append<QLM_KV_E4M3, 1> : k_append<QLM_KV_INT8, 1>
                : a.c.D <= 128 ? e4m3 ? k_append<QLM_KV_E4M3, 2> : k_append<QLM_KV_INT8, 2>
                               : e4m3 ? k_append<QLM_KV_E4M3, 4> : k_append<QLM_KV_INT8, 4>;
    kern<<<(unsigned)grid, kThreads, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_append launch");
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

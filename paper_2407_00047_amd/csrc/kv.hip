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

struct AppendArgs {
    CacheArgs c;
    Seqs q;
    const void *k, *v;
    int64_t k_row, k_head, v_row, v_head;
    int32_t k_type, v_type;
    const int32_t *first;
    int32_t touched;      // blocks a sequence's new slots may lie in
};

// One workgroup for each (sequence, block that takes new slots, kv head).
template <int FMT> __global__ __launch_bounds__(kThreads) void k_append(AppendArgs a)
{
    __shared__ float red[2 * kThreads / 64];
    const int t = threadIdx.x, nt = blockDim.x;
    int64_t at = blockIdx.x;
    const int h = (int)(at % a.c.H);
    at /= a.c.H;
    const int tb = (int)(at % a.touched);
    const int s = (int)(at / a.touched);
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
    const int64_t kbase = (int64_t)h * a.k_head, vbase = (int64_t)h * a.v_head;
    const int64_t r0 = (int64_t)row0 + (lo - start);        // row of slot o0
    float ak = 0.f, av = 0.f;
    for (int e = t; e < (o1 - o0) * D; e += nt) {
        const int64_t r = r0 + e / D;
        const int d = e % D;
        ak = fmaxf(ak, finite_abs(row_value(a.k, kbase + r * a.k_row + d, a.k_type)));
        av = fmaxf(av, finite_abs(row_value(a.v, vbase + r * a.v_row + d, a.v_type)));
    }
    max2(ak, av, red);
    const int64_t bh = (int64_t)id * a.c.H + h;
    const bool fresh = o0 == 0;
    const float oldk = fresh ? 0.f : a.c.ks[bh], oldv = fresh ? 0.f : a.c.vs[bh];
    const float newk = fmaxf(oldk, scale_for<FMT>(ak)), newv = fmaxf(oldv, scale_for<FMT>(av));
    __syncthreads();                                // every thread has read the old scales
    if (t == 0) {
        a.c.ks[bh] = newk;
        a.c.vs[bh] = newv;
    }

    // keys: four dims of a slot at a time
    uint8_t *kc = a.c.kc + bh * kBlock * D;
    const bool growk = !fresh && newk > oldk;
    const float ratiok = oldk / newk;
    const int s0 = growk ? 0 : o0, s1 = growk ? kBlock : o1;
    for (int e = t; e < (s1 - s0) * (D / 4); e += nt) {
        const int o = s0 + e / (D / 4), d = 4 * (e % (D / 4));
        uint32_t w = 0;
        if (o >= o0 && o < o1) {
            for (int b = 0; b < 4; ++b)
                w |= code_of<FMT>(row_value(a.k, kbase + (r0 + o - o0) * a.k_row + d + b,
                                            a.k_type) / newk) << (8 * b);
        } else {
            w = requant4<FMT>(*(const uint32_t *)(kc + o * D + d), ratiok);
        }
        *(uint32_t *)(kc + o * D + d) = w;
    }
    // values: four places of a dim at a time
    uint8_t *vc = a.c.vc + bh * kBlock * D;
    const bool growv = !fresh && newv > oldv;
    const float ratiov = oldv / newv;
    for (int e = t; e < 16 * D; e += nt) {
        const int p = 4 * (e & 3), d = (e >> 2) % D, g = (e >> 2) / D;
        const int o = value_slot(g, p);             // slots o .. o + 3
        if (!growv && (o + 4 <= o0 || o >= o1)) continue;
        uint8_t *at4 = vc + (g * D + d) * 16 + p;
        uint32_t w = 0;
        bool all = true;
        for (int b = 0; b < 4; ++b) all = all && o + b >= o0 && o + b < o1;
        if (!all) {
            w = *(const uint32_t *)at4;
            if (growv) w = requant4<FMT>(w, ratiov);
        }
        for (int b = 0; b < 4; ++b)
            if (o + b >= o0 && o + b < o1) {
                const float x = row_value(a.v, vbase + (r0 + o + b - o0) * a.v_row + d, a.v_type);
                w = (w & ~(0xffu << (8 * b))) | code_of<FMT>(x / newv) << (8 * b);
            }
        *(uint32_t *)at4 = w;
    }
    for (int o = o0 + t; o < o1; o += nt) {
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
    uint32_t *key;                      // [seq][head][slots]
    int32_t *src, *hole, *moved;        // [seq][head][budget]
    int32_t *newlen, *out;              // [seq]
};

constexpr int kSelThreads = 1024;
constexpr int kBins = 256;

// A slot's key: greater is kept first.  Protected slots above all, then the
// weights in their order, NaN last.
__device__ inline uint32_t weight_key(float w, bool safe)
{
    if (safe) return 0xffffffffu;
    if (w != w) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.f);   // -0 is 0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Sum of one flag over the lower threads of the workgroup, and over all.
__device__ inline int scan_flag(bool f, int *wave_sum, int *total)
{
    const uint64_t m = __ballot(f);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int below = __popcll(m & ((1ull << lane) - 1));
    if (lane == 0) wave_sum[w] = __popcll(m);
    __syncthreads();
    int before = 0, all = 0;
    for (int k = 0; k < kSelThreads / 64; ++k) {
        const int c = wave_sum[k];
        before += k < w ? c : 0;
        all += c;
    }
    __syncthreads();
    *total = all;
    return before + below;
}

// Which slots a (sequence, kv head) keeps, and what moves where: the budget
// greatest keys by four rounds of a radix selection (8 bits each, from the
// top), then one ordered walk that numbers holes and moved slots.
__global__ __launch_bounds__(kSelThreads) void k_evict_select(EvictArgs a)
{
    __shared__ uint32_t hist[kSelThreads / 64][kBins];
    __shared__ int wave_sum[kSelThreads / 64];
    __shared__ int red[kSelThreads / 64];
    __shared__ uint32_t s_prefix;
    __shared__ int s_left;
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6;
    const int h = (int)(blockIdx.x % a.c.H), s = (int)(blockIdx.x / a.c.H);
    const int len = seq_length(a.q, s);
    const int64_t sh = (int64_t)s * a.c.H + h;
    const int32_t *table = a.q.table + s * a.q.table_stride;
    int32_t *src = a.src + sh * a.budget;
    const int nb = (len + kBlock - 1) / kBlock;
    bool bad = false;
    if (len > a.budget)
        for (int j = t; j < nb; j += kSelThreads)
            bad = bad || (unsigned)table[j] >= (unsigned)a.c.n_blocks;
    const bool stays = len <= a.budget || __syncthreads_or(bad);
    if (h == 0 && t == 0) a.newlen[s] = stays ? len : a.budget;
    if (stays) {
        for (int o = t; o < a.budget; o += kSelThreads) src[o] = -1;
        return;
    }
    // the newest position
    int newest = INT32_MIN;
    for (int o = t; o < len; o += kSelThreads)
        newest = max(newest, a.c.pos[((int64_t)table[o >> 6] * a.c.H + h) * kBlock + (o & 63)]);
    for (int o = 32; o; o >>= 1) newest = max(newest, __shfl_xor(newest, o));
    if (lane == 0) red[wv] = newest;
    __syncthreads();
    for (int k = 0; k < kSelThreads / 64; ++k) newest = max(newest, red[k]);
    const int64_t safe_over = (int64_t)newest - a.recent;

    uint32_t *key = a.key + sh * a.slots;
    for (int o = t; o < len; o += kSelThreads) {
        const int64_t at = ((int64_t)table[o >> 6] * a.c.H + h) * kBlock + (o & 63);
        key[o] = weight_key(a.c.weight[at], (int64_t)a.c.pos[at] > safe_over);
    }
    // the budget-th greatest key: its digits from the top
    uint32_t prefix = 0;
    int left = a.budget;                    // of the keys that share the prefix, kept
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int b = lane; b < kBins; b += 64) hist[wv][b] = 0;
        __syncthreads();
        for (int o = t; o < len; o += kSelThreads) {
            const uint32_t x = key[o];
            if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8)))
                atomicAdd(&hist[wv][(x >> shift) & 255], 1u);
        }
        __syncthreads();
        if (t < kBins) {
            uint32_t c = 0;
            for (int k = 0; k < kSelThreads / 64; ++k) c += hist[k][t];
            hist[0][t] = c;
        }
        __syncthreads();
        if (wv == 0) {
            // lane l owns bins 4l .. 4l + 3; counts of the bins above them
            int c[4], sum = 0;
            for (int k = 0; k < 4; ++k) sum += c[k] = (int)hist[0][4 * lane + k];
            int above = sum;
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_down(above, o);
                above += lane + o < 64 ? v : 0;
            }
            above -= sum;
            for (int k = 3; k >= 0; --k) {
                if (above < left && above + c[k] >= left) {
                    s_prefix = prefix | (uint32_t)(4 * lane + k) << shift;
                    s_left = left - above;
                }
                above += c[k];
            }
        }
        __syncthreads();
        prefix = s_prefix;
        left = s_left;
    }
    // in slot order: of the keys equal to the last one kept the first `left` stay
    int n_eq = 0, n_hole = 0, n_moved = 0;
    int32_t *hole = a.hole + sh * a.budget, *moved = a.moved + sh * a.budget;
    for (int base = 0; base < len; base += kSelThreads) {
        const int o = base + t;
        const uint32_t x = o < len ? key[o] : 0;
        const bool eq = o < len && x == prefix;
        int all;
        const int rank = n_eq + scan_flag(eq, wave_sum, &all);
        n_eq += all;
        const bool keep = o < len && (x > prefix || (eq && rank < left));
        const bool is_hole = o < a.budget && !keep, is_moved = o >= a.budget && keep;
        const int rh = n_hole + scan_flag(is_hole, wave_sum, &all);
        n_hole += all;
        const int rm = n_moved + scan_flag(is_moved, wave_sum, &all);
        n_moved += all;
        if (o < a.budget) src[o] = -1;
        if (is_hole) hole[rh] = o;
        if (is_moved) moved[rm] = o;
    }
    __syncthreads();
    for (int i = t; i < min(n_hole, n_moved); i += kSelThreads) src[hole[i]] = moved[i];
}

// One workgroup for each (sequence, block below the budget, kv head): fetches
// what moves into the block's holes, renews the scales, writes.
template <int FMT> __global__ __launch_bounds__(kThreads) void k_evict_move(EvictArgs a)
{
    __shared__ int32_t from[kBlock];
    __shared__ int64_t fbh[kBlock];             // block and head of the source
    __shared__ float fks[kBlock], fvs[kBlock];
    __shared__ float red[2 * kThreads / 64];
    __shared__ uint8_t kx[kBlock * 256], vx[kBlock * 256];   // incoming codes [slot][dim]
    const int t = threadIdx.x;
    const int nb = a.budget / kBlock;
    int64_t at = blockIdx.x;
    const int j = (int)(at % nb);
    at /= nb;
    const int h = (int)(at % a.c.H), s = (int)(at / a.c.H);
    const int D = a.c.D;
    if (h == 0 && j == 0 && t == 0) a.out[s] = a.newlen[s];
    const int32_t *table = a.q.table + s * a.q.table_stride;
    bool any = false;
    if (t < kBlock) {
        const int o = a.src[((int64_t)s * a.c.H + h) * a.budget + j * kBlock + t];
        from[t] = o;
        any = o >= 0;
        if (any) {
            const int64_t b = (int64_t)table[o >> 6] * a.c.H + h;
            fbh[t] = b;
            fks[t] = a.c.ks[b];
            fvs[t] = a.c.vs[b];
        }
    }
    if (!__syncthreads_or(any)) return;
    const int64_t bh = (int64_t)table[j] * a.c.H + h;
    float ak = 0.f, av = 0.f;
    for (int e = t; e < kBlock * (D / 4); e += kThreads) {
        const int i = e / (D / 4), d = 4 * (e % (D / 4));
        const int o = from[i];
        if (o < 0) continue;
        const uint8_t *kp = a.c.kc + (fbh[i] * kBlock + (o & 63)) * D + d;
        const uint8_t *vp = a.c.vc + fbh[i] * kBlock * D +
                            (value_group(o & 63) * D + d) * 16 + value_place(o & 63);
        const uint32_t kw = *(const uint32_t *)kp;
        uint32_t vw = 0;
        for (int b = 0; b < 4; ++b) vw |= (uint32_t)vp[16 * b] << (8 * b);
        *(uint32_t *)(kx + i * D + d) = kw;
        *(uint32_t *)(vx + i * D + d) = vw;
        for (int b = 0; b < 4; ++b) {
            ak = fmaxf(ak, finite_abs(code_value<FMT>((kw >> (8 * b)) & 0xff) * fks[i]));
            av = fmaxf(av, finite_abs(code_value<FMT>((vw >> (8 * b)) & 0xff) * fvs[i]));
        }
    }
    const float oldk = a.c.ks[bh], oldv = a.c.vs[bh];
    max2(ak, av, red);                          // (its barrier: every thread has the old scales)
    const float newk = fmaxf(oldk, scale_for<FMT>(ak)), newv = fmaxf(oldv, scale_for<FMT>(av));
    if (t == 0) {
        a.c.ks[bh] = newk;
        a.c.vs[bh] = newv;
    }
    uint8_t *kc = a.c.kc + bh * kBlock * D;
    const bool growk = newk > oldk;
    const float ratiok = oldk / newk;
    for (int e = t; e < kBlock * (D / 4); e += kThreads) {
        const int i = e / (D / 4), d = 4 * (e % (D / 4));
        uint32_t *p = (uint32_t *)(kc + i * D + d);
        if (from[i] >= 0) {
            const uint32_t x = *(const uint32_t *)(kx + i * D + d);
            uint32_t w = 0;
            for (int b = 0; b < 4; ++b)
                w |= code_of<FMT>(code_value<FMT>((x >> (8 * b)) & 0xff) * fks[i] / newk)
                     << (8 * b);
            *p = w;
        } else if (growk) {
            *p = requant4<FMT>(*p, ratiok);
        }
    }
    uint8_t *vc = a.c.vc + bh * kBlock * D;
    const bool growv = newv > oldv;
    const float ratiov = oldv / newv;
    for (int e = t; e < 16 * D; e += kThreads) {
        const int p = 4 * (e & 3), d = (e >> 2) % D, g = (e >> 2) / D;
        const int o = value_slot(g, p);
        const bool some = from[o] >= 0 || from[o + 1] >= 0 || from[o + 2] >= 0 || from[o + 3] >= 0;
        if (!growv && !some) continue;
        uint32_t *at4 = (uint32_t *)(vc + (g * D + d) * 16 + p);
        uint32_t w = *at4;
        if (growv) w = requant4<FMT>(w, ratiov);
        for (int b = 0; b < 4; ++b)
            if (from[o + b] >= 0)
                w = (w & ~(0xffu << (8 * b))) |
                    code_of<FMT>(code_value<FMT>(vx[(o + b) * D + d]) * fvs[o + b] / newv)
                        << (8 * b);
        *at4 = w;
    }
    if (t < kBlock && from[t] >= 0) {
        const int64_t to = bh * kBlock + t, fr = fbh[t] * kBlock + (from[t] & 63);
        a.c.pos[to] = a.c.pos[fr];
        a.c.weight[to] = a.c.weight[fr];
    }
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
    l.src = l.key + align256(sh * slots * 4);
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
    if (grid > INT32_MAX) return fail(QLM_ERR_CAPACITY, "too many blocks in one append");
    auto kern = cache->format == QLM_KV_E4M3 ? k_append<QLM_KV_E4M3> : k_append<QLM_KV_INT8>;
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
    if (grid > INT32_MAX) return fail(QLM_ERR_CAPACITY, "too many blocks in one eviction");
    k_evict_select<<<(unsigned)sh, kSelThreads, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "k_evict_select launch");
    auto kern = cache->format == QLM_KV_E4M3 ? k_evict_move<QLM_KV_E4M3>
                                             : k_evict_move<QLM_KV_INT8>;
    kern<<<(unsigned)grid, kThreads, 0, stream>>>(a);
    e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_evict_move launch");
}

}  // extern "C"

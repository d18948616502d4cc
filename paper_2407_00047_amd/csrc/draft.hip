// draft.hip -- verification of drafted tokens (qlm_draft_verify; the definition
// stands in include/qlm.h).
//
// What has to be read is a few numbers a draft and then one row of the target's
// probabilities, with one of the draft's where a token is refused.  The inverse of a running sum
// is found without keeping it: sums of segments of the row first, then the segment on whose
// border u falls is read again.  Differences and sums are in double precision, in which a
// difference of two of single precision is exact: the word depends on a border
// between sums of the whole vocabulary.
#include "kv.h"

#include <string>

namespace {

using namespace qlm_kv;
using qlm_internal::fail;
using qlm_internal::hip_fail;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSegments = 1024;        // of a row at most: one a thread

struct DraftArgs {
    Seqs q;
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    const int32_t *tokens;
    const float *uniform;
    int32_t *tokens_out, *count, *lengths_out;
    int32_t vocab;
};

template <int TYPE> struct Word {
    typedef uint16_t bits;
};
template <> struct Word<QLM_F32> {
    typedef float bits;
};

template <int TYPE> __device__ inline double value(typename Word<TYPE>::bits b)
{
    if constexpr (TYPE == QLM_F32) return (double)b;
    else if constexpr (TYPE == QLM_BF16) return (double)__builtin_bit_cast(float, (uint32_t)b << 16);
    else return (double)__builtin_bit_cast(_Float16, b);
}

// A row's weights: of the target's probabilities p and, behind a refused draft, the draft's q
// (one at `token` where q is NULL).
template <int TYPE> struct Weights {
    typedef typename Word<TYPE>::bits bits;
    static constexpr int E = 16 / sizeof(bits);   // words read at once
    const bits *p, *q;
    int vocab, token;                             // token: -1 where nothing is taken off
    int shift;                                    // words before p on its 16 bytes
    bool wide;                                    // p and q stand alike on their 16 bytes

    __device__ double one(int v) const
    {
        const double x = value<TYPE>(p[v]);
        if (q) return max_of(x - value<TYPE>(q[v]));
        return v == token ? max_of(x - 1.0) : x;
    }
    // (a NaN has to reach the sum)
    static __device__ double max_of(double x) { return x < 0.0 ? 0.0 : x; }
    // The E words from v on; v may be before the row or past it by less than E.
    __device__ void load(int64_t v, double *w) const
    {
        if (wide && v >= 0 && v + E <= vocab) {
            const uint4 a = *(const uint4 *)(p + v);
            uint4 b = {0, 0, 0, 0};
            if (q) b = *(const uint4 *)(q + v);
            bits x[E], y[E];
            __builtin_memcpy(x, &a, 16);
            __builtin_memcpy(y, &b, 16);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                w[e] = value<TYPE>(x[e]);
                if (q) w[e] = max_of(w[e] - value<TYPE>(y[e]));
                else if (v + e == token) w[e] = max_of(w[e] - 1.0);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = v + e >= 0 && v + e < vocab ? one((int)(v + e)) : 0.0;
    }
};

// Running sum over the wave's lanes, this one's included.
__device__ inline double wave_scan(double x)
{
    const int lane = threadIdx.x & 63;
    for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// One workgroup for each sequence.
template <int TYPE> __global__ __launch_bounds__(kThreads) void k_draft_verify(DraftArgs a)
{
    typedef Weights<TYPE> W;
    typedef typename W::bits bits;
    __shared__ double sums[kSegments], wave_sum[kWaves];
    __shared__ int s_segment, s_word;
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6, s = blockIdx.x;
    int row0;
    const int n = seq_rows(a.q, s, &row0), length = seq_length(a.q, s);
    // the drafts that are accepted, 64 at a time
    int kept = 0;
    for (; kept < n - 1;) {
        const int i = kept + lane;
        bool good = false;
        if (i < n - 1) {
            const int64_t row = row0 + i;
            const int v = a.tokens[row + 1];
            if ((unsigned)v < (unsigned)a.vocab) {
                const double p = value<TYPE>(((const bits *)a.target)[row * a.target_stride + v]);
                const double q =
                    a.draft ? value<TYPE>(((const bits *)a.draft)[row * a.draft_stride + v]) : 1.0;
                good = (double)a.uniform[row] * q < p;
            }
        }
        const uint64_t no = ~__ballot(good);
        if (no) {
            kept += __builtin_ctzll(no);       // (a lane past the drafts is not good)
            break;
        }
        kept += 64;
    }
    int word = -1;
    if (n > 0) {
        const int64_t row = row0 + kept;
        const double u = a.uniform[row0 + n - 1];
        W w;
        w.p = (const bits *)a.target + row * a.target_stride;
        w.q = nullptr;
        w.vocab = a.vocab;
        w.token = -1;
        w.shift = (int)((uintptr_t)w.p % 16 / sizeof(bits));
        w.wide = true;
        bool less = kept < n - 1;              // something is taken off
        if (less) {
            w.token = a.tokens[row + 1];
            if (a.draft) {
                w.q = (const bits *)a.draft + row * a.draft_stride;
                w.wide = ((uintptr_t)w.p - (uintptr_t)w.q) % 16 == 0;
            }
        }
        // segments of the row, whole wide reads of a wave each
        constexpr int kStep = 64 * W::E, kUnroll = 16 / W::E;
        const int64_t words = (int64_t)a.vocab + w.shift;
        const int steps = (int)((words + kStep - 1) / kStep);
        const int per = max(kUnroll, ((steps + kSegments - 1) / kSegments + kUnroll - 1) / kUnroll *
                                         kUnroll);
        const int segments = (steps + per - 1) / per;
        for (;;) {
            for (int g = wv; g < segments; g += kWaves) {
                double sum = 0.0;
                for (int k = 0; k < per; k += kUnroll) {
                    double x[kUnroll][W::E];
#pragma unroll
                    for (int j = 0; j < kUnroll; ++j)
                        w.load(((int64_t)g * per + k + j) * kStep + lane * W::E - w.shift, x[j]);
#pragma unroll
                    for (int j = 0; j < kUnroll; ++j)
#pragma unroll
                        for (int e = 0; e < W::E; ++e) sum += x[j][e];
                }
                for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
                if (lane == 0) sums[g] = sum;
            }
            if (t == 0) s_segment = segments - 1;
            __syncthreads();
            // the segment in which the running sum passes u of the whole
            const double mine = t < segments ? sums[t] : 0.0;
            double upto = wave_scan(mine);
            if (lane == 63) wave_sum[wv] = upto;
            __syncthreads();
            double before = 0.0, total = 0.0;
            for (int k = 0; k < kWaves; ++k) {
                before += k < wv ? wave_sum[k] : 0.0;
                total += wave_sum[k];
            }
            upto += before;
            const double mark = u * total;
            if (t < segments && upto > mark) atomicMin(&s_segment, t);
            __syncthreads();
            const bool usable = total > 0.0 && total < (double)__builtin_inff();
            if (usable || !less) {
                if (t == s_segment) sums[0] = upto - mine;   // (read by none any more)
                __syncthreads();
                if (usable && wv == 0) {
                    // the words of that segment, in their order
                    double run = sums[0];
                    int found = -1, last = -1;
                    for (int k = 0; k < per && found < 0; ++k) {
                        double x[W::E];
                        const int64_t v =
                            ((int64_t)s_segment * per + k) * kStep + lane * W::E - w.shift;
                        w.load(v, x);
                        double sum = 0.0;
#pragma unroll
                        for (int e = 0; e < W::E; ++e) sum += x[e];
                        double at = run + (wave_scan(sum) - sum);
                        int hit = -1, some = -1;
#pragma unroll
                        for (int e = 0; e < W::E; ++e) {
                            at += x[e];
                            if (x[e] > 0.0) {
                                some = (int)(v + e);
                                if (hit < 0 && at > mark) hit = some;
                            }
                        }
                        const uint64_t m = __ballot(hit >= 0), any = __ballot(some >= 0);
                        if (m) found = __shfl(hit, __builtin_ctzll(m));
                        if (any) last = __shfl(some, 63 - __builtin_clzll(any));
                        run += __shfl(wave_scan(sum), 63);
                    }
                    // (sums of sums round otherwise than one by one: past the last word there
                    // it is the last one)
                    if (lane == 0) s_word = found >= 0 ? found : last;
                } else if (t == 0) {
                    s_word = -1;
                }
                break;
            }
            less = false;                      // nothing is left: from the target itself
            w.q = nullptr;
            w.token = -1;
            w.wide = true;
            __syncthreads();
        }
        __syncthreads();
        word = s_word;
    }
    for (int i = t; i < a.q.max_new; i += kThreads)
        a.tokens_out[(int64_t)s * a.q.max_new + i] =
            n == 0 || i > kept ? -1 : i == kept ? word : a.tokens[row0 + i + 1];
    if (t == 0) {
        a.count[s] = n > 0 ? kept + 1 : 0;
        if (a.lengths_out) a.lengths_out[s] = n > 0 ? max(0, length - (n - 1 - kept)) : length;
    }
}

}  // namespace

extern "C" {

size_t qlm_draft_verify_workspace_bytes(const qlm_kv_batch *batch, int32_t vocab)
{
    (void)batch;
    (void)vocab;
    return 0;
}

int qlm_draft_verify(const qlm_kv_batch *batch, const qlm_draft *draft, int32_t *tokens_out,
                     int32_t *count, int32_t *lengths_out, void *ws, size_t ws_bytes,
                     qlm_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    if (int rc = check_batch(batch)) return rc;
    if (!draft) return fail(QLM_ERR_ARG, "draft is NULL");
    if (draft->vocab < 1 || draft->vocab > (1 << 24))
        return fail(QLM_ERR_ARG, "vocab must be in 1..16777216");
    const int dtype = draft->dtype;
    if (dtype != QLM_F16 && dtype != QLM_BF16 && dtype != QLM_F32)
        return fail(QLM_ERR_ARG, "dtype must be QLM_F16, QLM_BF16 or QLM_F32");
    if (batch->n_seqs == 0) return QLM_OK;
    if (!tokens_out || !count) return fail(QLM_ERR_ARG, "tokens_out and count are required");
    if (batch->n_rows > 0) {
        if (!draft->target || !draft->tokens || !draft->uniform)
            return fail(QLM_ERR_ARG, "target, tokens and uniform are required");
        const size_t size = dtype == QLM_F32 ? 4 : 2;
        if ((uintptr_t)draft->target % size || (uintptr_t)draft->draft % size)
            return fail(QLM_ERR_ARG, "target or draft is misaligned");
        if (draft->target_stride < draft->vocab ||
            (draft->draft && draft->draft_stride < draft->vocab))
            return fail(QLM_ERR_ARG, "target_stride and draft_stride must be >= vocab");
    }
    if (int rc = check_workspace(ws, ws_bytes, qlm_draft_verify_workspace_bytes(batch, draft->vocab)))
        return rc;
    if (!can_launch(batch->n_seqs, kThreads))
        return fail(QLM_ERR_CAPACITY, "too many sequences in one verification");
    DraftArgs a{};
    a.q = seqs_of(batch);
    a.target = draft->target;
    a.draft = draft->draft;
    a.target_stride = draft->target_stride;
    a.draft_stride = draft->draft_stride;
    a.tokens = draft->tokens;
    a.uniform = draft->uniform;
    a.tokens_out = tokens_out;
    a.count = count;
    a.lengths_out = lengths_out;
    a.vocab = draft->vocab;
    auto kern = dtype == QLM_F32    ? k_draft_verify<QLM_F32>
                : dtype == QLM_BF16 ? k_draft_verify<QLM_BF16>
                                    : k_draft_verify<QLM_F16>;
    kern<<<(unsigned)batch->n_seqs, kThreads, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_draft_verify launch");
}

}  // extern "C"

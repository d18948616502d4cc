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

#include <algorithm>
#include <string>

namespace {

using namespace qlm_kv;
using qlm_internal::fail;
using qlm_internal::hip_fail;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSumWaves = 4;
constexpr int kSegments = 1024;        // of a row at most: one a thread
constexpr int kWords = 16;             // words of a lane in a segment

struct DraftArgs {
    Seqs q;
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    const int32_t *tokens;
    const float *uniform;
    int32_t *tokens_out, *count, *lengths_out;
    int32_t vocab;
    double *sums;                  // [sequence][segment], where they come from a launch before
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

    // (a NaN has to reach the sum)
    static __device__ double max_of(double x) { return x < 0.0 ? 0.0 : x; }
    // The E words from v on, of which some may be before the row or past it: their bits, zeros
    // there, for sums that are taken later.
    struct Bits {
        bits x[E], y[E];
    };
    __device__ void read(int v, Bits &b) const
    {
        if (wide && v >= 0 && v + E <= vocab) {
            const uint4 x = *(const uint4 *)(p + v);
            uint4 y = {0, 0, 0, 0};
            if (q) y = *(const uint4 *)(q + v);
            __builtin_memcpy(b.x, &x, 16);
            __builtin_memcpy(b.y, &y, 16);
            return;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool in = v + e >= 0 && v + e < vocab;
            b.x[e] = in ? p[v + e] : (bits)0;
            b.y[e] = in && q ? q[v + e] : (bits)0;
        }
    }
    __device__ void weigh(int v, const Bits &b, double *w) const
    {
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = value<TYPE>(b.x[e]);
        if (q) {
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = max_of(w[e] - value<TYPE>(b.y[e]));
        } else if (token >= v && token < v + E) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (v + e == token) w[e] = max_of(w[e] - 1.0);
        }
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

// What the drafts of a sequence come to.
struct Step {
    int row0, n, length;     // its rows, and its slots
    int kept, refused;       // accepted drafts; the token of the one refused, -1 where none is
    double u;                // the number that the last token is drawn with
};

template <int TYPE> __device__ inline Step step_of(const DraftArgs &a, int s)
{
    typedef typename Word<TYPE>::bits bits;
    Step r;
    r.n = seq_rows(a.q, s, &r.row0);
    r.length = seq_length(a.q, s);
    r.u = r.n > 0 ? a.uniform[r.row0 + r.n - 1] : 0.f;
    r.kept = 0;
    r.refused = -1;
    const int lane = threadIdx.x & 63;
    while (r.kept < r.n - 1) {                 // 64 at a time
        const int i = r.kept + lane;
        bool good = false;
        int v = -1;
        if (i < r.n - 1) {
            const int64_t row = r.row0 + i;
            v = a.tokens[row + 1];
            if ((unsigned)v < (unsigned)a.vocab) {
                const double p = value<TYPE>(((const bits *)a.target)[row * a.target_stride + v]);
                const double q =
                    a.draft ? value<TYPE>(((const bits *)a.draft)[row * a.draft_stride + v]) : 1.0;
                good = (double)a.uniform[row] * q < p;
            }
        }
        const uint64_t no = ~__ballot(good);
        if (no) {
            const int first = __builtin_ctzll(no);     // (a lane past the drafts is not good)
            r.refused = __builtin_amdgcn_readlane(v, first);
            r.kept += first;
            break;
        }
        r.kept += 64;
    }
    return r;
}

// The weights that the last token is drawn from; `less`: those of the draft are taken off.
template <int TYPE>
__device__ inline Weights<TYPE> weights_of(const DraftArgs &a, const Step &r, bool less)
{
    typedef typename Word<TYPE>::bits bits;
    const int64_t row = r.row0 + r.kept;
    Weights<TYPE> w;
    w.p = (const bits *)a.target + row * a.target_stride;
    w.q = nullptr;
    w.vocab = a.vocab;
    w.token = less ? r.refused : -1;
    w.shift = (int)((uintptr_t)w.p % 16 / sizeof(bits));
    w.wide = true;
    if (less && a.draft) {
        w.q = (const bits *)a.draft + row * a.draft_stride;
        w.wide = ((uintptr_t)w.p - (uintptr_t)w.q) % 16 == 0;
    }
    return w;
}

// A row in segments of `per` times 64 lanes' kWords words.  They are counted with the most words
// that a row may stand behind its 16 bytes, so that their number is known without it.
struct Cut {
    int per, segments;
};

__host__ __device__ inline Cut cut_of(int vocab)
{
    const int parts = (vocab + 7 + 64 * kWords - 1) / (64 * kWords);
    const int per = (parts + kSegments - 1) / kSegments;
    return {per, (parts + per - 1) / per};
}

template <int TYPE>
__device__ inline double segment_sum(const Weights<TYPE> &w, const Cut &cut, int g)
{
    typedef Weights<TYPE> W;
    constexpr int READS = kWords / W::E;
    const int lane = threadIdx.x & 63;
    double sum = 0.0;
    for (int k = 0; k < cut.per; ++k) {
        const int v0 = (g * cut.per + k) * 64 * kWords + lane * W::E - w.shift;
        typename W::Bits b[READS];
#pragma unroll
        for (int j = 0; j < READS; ++j) w.read(v0 + j * 64 * W::E, b[j]);
#pragma unroll
        for (int j = 0; j < READS; ++j) {
            double x[W::E];
            w.weigh(v0 + j * 64 * W::E, b[j], x);
#pragma unroll
            for (int e = 0; e < W::E; ++e) sum += x[e];
        }
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    return sum;
}

// The least word of segment g whose running sum, `run` before the segment, passes `mark`: kWords
// neighbours a lane.  Sums of sums round otherwise than one by one: where none passes it, the last
// word of any weight.
template <int TYPE>
__device__ inline int word_of(const Weights<TYPE> &w, const Cut &cut, int g, double run, double mark)
{
    typedef Weights<TYPE> W;
    constexpr int READS = kWords / W::E;
    const int lane = threadIdx.x & 63;
    int found = -1, last = -1;
    for (int k = 0; k < cut.per && found < 0; ++k) {
        const int v0 = (g * cut.per + k) * 64 * kWords + lane * kWords - w.shift;
        typename W::Bits b[READS];
        double x[kWords], sum = 0.0;
#pragma unroll
        for (int j = 0; j < READS; ++j) w.read(v0 + j * W::E, b[j]);
#pragma unroll
        for (int j = 0; j < READS; ++j) w.weigh(v0 + j * W::E, b[j], x + j * W::E);
#pragma unroll
        for (int e = 0; e < kWords; ++e) sum += x[e];
        const double upto = wave_scan(sum);
        double at = run + (upto - sum);
        int hit = -1, some = -1;
#pragma unroll
        for (int e = 0; e < kWords; ++e) {
            at += x[e];
            if (x[e] > 0.0) {
                some = v0 + e;
                if (hit < 0 && at > mark) hit = some;
            }
        }
        const uint64_t m = __ballot(hit >= 0), any = __ballot(some >= 0);
        if (m) found = __shfl(hit, __builtin_ctzll(m));
        if (any) last = __shfl(some, 63 - __builtin_clzll(any));
        run += __shfl(upto, 63);
    }
    return found >= 0 ? found : last;
}

// Sums of a few segments of a sequence's row to a workgroup, for k_draft_verify of few sequences.
template <int TYPE>
__global__ __launch_bounds__(64 * kSumWaves) void k_draft_sums(DraftArgs a)
{
    const Cut cut = cut_of(a.vocab);
    const uint32_t groups = (cut.segments + kSumWaves - 1) / kSumWaves;
    const int s = (int)(blockIdx.x / groups);
    const int g = (int)(blockIdx.x % groups) * kSumWaves + (int)(threadIdx.x >> 6);
    const Step r = step_of<TYPE>(a, s);
    if (r.n == 0 || g >= cut.segments) return;
    const double sum = segment_sum(weights_of<TYPE>(a, r, r.kept < r.n - 1), cut, g);
    if ((threadIdx.x & 63) == 0) a.sums[(int64_t)s * cut.segments + g] = sum;
}

// One workgroup for each sequence.  Sequences that fill the chip are read at the memory's rate (256 of
// 131072 words in single precision, 229 MB, 43 us); a few long rows are bound by what one compute
// unit reads (1 MB 12 us): their segments' sums come from a launch before (SUMS).
template <int TYPE, bool SUMS>
__global__ __launch_bounds__(kThreads) void k_draft_verify(DraftArgs a)
{
    __shared__ double sums[kSegments], wave_sum[kWaves];
    __shared__ int s_segment, s_last, s_word;
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6, s = blockIdx.x;
    const Cut cut = cut_of(a.vocab);
    double mine = 0.0;
    if (SUMS && t < cut.segments) mine = a.sums[(int64_t)s * cut.segments + t];
    const Step r = step_of<TYPE>(a, s);
    int word = -1;
    bool less = r.kept < r.n - 1;              // something is taken off
    bool given = SUMS;
    while (r.n > 0) {
        const Weights<TYPE> w = weights_of<TYPE>(a, r, less);
        if (!given)
            for (int g = wv; g < cut.segments; g += kWaves) {
                const double sum = segment_sum(w, cut, g);
                if (lane == 0) sums[g] = sum;
            }
        if (t == 0) s_segment = kSegments, s_last = -1;
        __syncthreads();
        // the segment in which the running sum passes u of the whole, of those with any weight
        // (scans of neighbours round apart: the sum may seem to pass where nothing is added)
        if (!given) mine = t < cut.segments ? sums[t] : 0.0;
        double upto = wave_scan(mine);
        if (lane == 63) wave_sum[wv] = upto;
        __syncthreads();
        double before = 0.0, total = 0.0;
        for (int k = 0; k < kWaves; ++k) {
            before += k < wv ? wave_sum[k] : 0.0;
            total += wave_sum[k];
        }
        upto += before;
        const double mark = r.u * total;
        const uint64_t some = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && upto > mark);
        if (lane == 0 && some) atomicMax(&s_last, 64 * wv + 63 - __builtin_clzll(some));
        if (lane == 0 && past) atomicMin(&s_segment, 64 * wv + __builtin_ctzll(past));
        __syncthreads();
        const int segment = min(s_segment, max(s_last, 0));
        const bool usable = total > 0.0 && total < (double)__builtin_inff();
        if (usable || !less) {
            if (t == segment) sums[0] = upto - mine;   // (read by none any more)
            __syncthreads();
            if (wv == 0) {
                const int got = usable ? word_of(w, cut, segment, sums[0], mark) : -1;
                if (lane == 0) s_word = got;
            }
            __syncthreads();
            word = s_word;
            break;
        }
        less = false;                          // nothing is left: from the target itself
        given = false;
        __syncthreads();
    }
    for (int i = t; i < a.q.max_new; i += kThreads)
        a.tokens_out[(int64_t)s * a.q.max_new + i] =
            r.n == 0 || i > r.kept ? -1 : i == r.kept ? word : a.tokens[r.row0 + i + 1];
    if (t == 0) {
        a.count[s] = r.n > 0 ? r.kept + 1 : 0;
        if (a.lengths_out)
            a.lengths_out[s] = r.n > 0 ? max(0, r.length - (r.n - 1 - r.kept)) : r.length;
    }
}

// Whether the sums come from a launch of their own.  As a whole 9.5 us and what a compute unit reads
// (75 GB/s) or the memory, in two 13.5 us and what the memory gives: one sequence of 131072 words
// in single precision, drafts drawn, 22 and 14 us; 64 of them 28 and 27; 256 43 and 57.
bool sums_apart(int n_seqs, int vocab, int dtype, bool drawn)
{
    const double row = (double)vocab * (dtype == QLM_F32 ? 4 : 2) * (drawn ? 2 : 1);
    const double all = row * n_seqs / 5.1e6;
    const int turns = (n_seqs + 255) / 256;
    return 13.5 + all < 9.5 + std::max(turns * row / 75e3, all);
}

}  // namespace

extern "C" {

size_t qlm_draft_verify_workspace_bytes(const qlm_kv_batch *batch, int32_t vocab)
{
    if (!batch || batch->n_seqs < 1 || vocab < 1 || vocab > (1 << 24)) return 0;
    // (for either type, drafts drawn or not)
    return sums_apart(batch->n_seqs, vocab, QLM_F32, true)
               ? (size_t)batch->n_seqs * cut_of(vocab).segments * sizeof(double)
               : 0;
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
    const bool apart = sums_apart(batch->n_seqs, draft->vocab, dtype, draft->draft != nullptr);
    if (apart) {
        a.sums = (double *)ws;
        const int64_t groups =
            (int64_t)batch->n_seqs * ((cut_of(a.vocab).segments + kSumWaves - 1) / kSumWaves);
        auto kern = dtype == QLM_F32    ? k_draft_sums<QLM_F32>
                    : dtype == QLM_BF16 ? k_draft_sums<QLM_BF16>
                                        : k_draft_sums<QLM_F16>;
        kern<<<(unsigned)groups, 64 * kSumWaves, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "k_draft_sums launch");
    }
    auto kern = dtype == QLM_F32    ? apart ? k_draft_verify<QLM_F32, true> : k_draft_verify<QLM_F32, false>
                : dtype == QLM_BF16 ? apart ? k_draft_verify<QLM_BF16, true>
                                            : k_draft_verify<QLM_BF16, false>
                : apart             ? k_draft_verify<QLM_F16, true>
                                    : k_draft_verify<QLM_F16, false>;
    kern<<<(unsigned)batch->n_seqs, kThreads, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? QLM_OK : hip_fail(e, "k_draft_verify launch");
}

}  // extern "C"

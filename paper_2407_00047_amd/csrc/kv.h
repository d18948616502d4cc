// kv.h -- what the kernels of the 8-bit token cache share: the batch's
// sequences, the codes, the order of the values, the checks of the host.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"
#include "qlm.h"

namespace qlm_kv {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kBlock = QLM_KV_BLOCK;
constexpr int kLeastExp = -100;      // least exponent of a scale that append writes

struct Seqs {
    int32_t n_seqs, n_rows, max_new, max_length;
    int64_t table_stride;
    const int32_t *table, *lengths, *row_start;
};

inline Seqs seqs_of(const qlm_kv_batch *b)
{
    return {b->n_seqs, b->n_rows, b->max_new, b->max_length,
            b->table_stride, b->block_table, b->lengths, b->row_start};
}

__device__ inline int seq_length(const Seqs &q, int s)
{
    return max(0, min(q.lengths[s], q.max_length));
}

// The sequence's first row and its number of rows, whatever row_start holds.
__device__ inline int seq_rows(const Seqs &q, int s, int *row0)
{
    if (!q.row_start) {
        *row0 = s;
        return s < q.n_rows ? 1 : 0;
    }
    const int r0 = max(0, min(q.row_start[s], q.n_rows));
    const int r1 = max(r0, min(q.row_start[s + 1], q.n_rows));
    *row0 = r0;
    return min(r1 - r0, q.max_new);
}

// Reads through the scalar cache what every lane reads alike and no kernel
// writes while it runs (the loads of a table entry then stand in no queue
// behind the wide loads of codes).
template <typename T> __device__ inline T uniform(const T *p)
{
    typedef const T __attribute__((address_space(4))) *scalar_ptr;
    return *(scalar_ptr)(uintptr_t)p;
}

// -- codes ----------------------------------------------------------------

template <int FMT> __host__ __device__ constexpr float top_code()
{
    return FMT == QLM_KV_E4M3 ? 448.f : 127.f;
}

// Four codes of a dword as halves (exact: both formats fit a half).
template <int FMT> __device__ inline void halves4(uint32_t w, half2v *lo, half2v *hi)
{
    if (FMT == QLM_KV_E4M3) {
        *lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
        *hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
    } else {
        // code + 128 under the exponent of 1024, then less 1152
        const uint32_t u = w ^ 0x80808080u;
        const half2v off = {(_Float16)-1152.f, (_Float16)-1152.f};
        const uint32_t a = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u);
        const uint32_t b = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
        *lo = __builtin_bit_cast(half2v, a) + off;
        *hi = __builtin_bit_cast(half2v, b) + off;
    }
}

// Eight codes as a matrix operand.
template <int FMT> __device__ inline half8v halves8(uint32_t x, uint32_t y)
{
    half2v a, b, c, d;
    halves4<FMT>(x, &a, &b);
    halves4<FMT>(y, &c, &d);
    return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One code as a float.
template <int FMT> __device__ inline float code_value(uint32_t c)
{
    if (FMT == QLM_KV_INT8) return (float)(int8_t)c;
    return (float)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, false)[0];
}

// The nearest code to y, ties to even, clamped; NaN stays in e4m3, 0 in int8.
template <int FMT> __device__ inline uint32_t code_of(float y)
{
    const float t = top_code<FMT>();
    y = y > t ? t : (y < -t ? -t : y);
    if (FMT == QLM_KV_INT8) return y != y ? 0u : (uint32_t)(uint8_t)(int8_t)(int)rintf(y);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xffu;
}

// 2^e with the least e >= kLeastExp for which a <= top 2^e (a finite, >= 0).
template <int FMT> __device__ inline float scale_for(float a)
{
    if (!(a > 0.f)) return ldexpf(1.f, kLeastExp);
    int e;
    const float m = frexpf(a, &e);           // a = m 2^e, m in [0.5, 1)
    // 448 = 0.875 * 2^9, 127 = 0.9921875 * 2^7
    const float top_m = FMT == QLM_KV_E4M3 ? 0.875f : 0.9921875f;
    e = e - (FMT == QLM_KV_E4M3 ? 9 : 7) + (m > top_m ? 1 : 0);
    return ldexpf(1.f, max(e, kLeastExp));
}

// Where slot t of a block stands in the values: the group's 16 bytes of dim d
// are at (group * D + d) * 16, the slot at byte `place` there.
__device__ inline int value_group(int t) { return (t >> 2) & 3; }
__device__ inline int value_place(int t) { return ((t >> 4) << 2) | (t & 3); }
// The slot at place p of group g.
__device__ inline int value_slot(int g, int p) { return ((p >> 2) << 4) | (g << 2) | (p & 3); }

// The bits of a row's element: rounded to nearest, ties to even.
__device__ inline uint16_t row_bits(float v, int dtype)
{
    if (dtype == QLM_BF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// -- host -----------------------------------------------------------------

int check_cache(const qlm_kv_cache *c);
int check_batch(const qlm_kv_batch *b);
int check_rows(const qlm_rows *r, const char *what);
int check_workspace(const void *ws, size_t have, size_t need);

// Whether so many workgroups can be launched: fewer than 2^32 threads in a dimension.  Asked
// of every launch of a call before the first one, as a call is done whole or not at all.
inline bool can_launch(int64_t groups, int threads) { return groups < (1ll << 32) / threads; }

}  // namespace qlm_kv

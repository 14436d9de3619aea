// Shared by the operators of a transformer block (dropout, layer norm, biased softmax): element types, the dropout
// generator, how the threads of a row share its columns, and sums over them.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "common.cuh"

namespace adacomp_impl {

constexpr int kBlockSms = 148;               // SMs of a B200: grids are sized to it, so results do not depend on a query
constexpr u32 kAllLanes = 0xffffffffu;

// ---------------------------------------------------------------------------------
// element types: eight elements at a time, arithmetic in binary32
// ---------------------------------------------------------------------------------

template <u32 TYPE> struct Vec8 { uint4 q[TYPE == ADACOMP_TYPE_F32 ? 2 : 1]; };

__host__ __device__ constexpr u32 type_size(u32 type) { return type == ADACOMP_TYPE_F32 ? 4u : 2u; }

template <u32 TYPE> __device__ inline Vec8<TYPE> load8(const void *base, u64 e)
{
    Vec8<TYPE> v;
    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const unsigned char *>(base) + e * type_size(TYPE));
    v.q[0] = p[0];
    if constexpr (TYPE == ADACOMP_TYPE_F32) v.q[1] = p[1];
    return v;
}

template <u32 TYPE> __device__ inline void store8(void *base, u64 e, const Vec8<TYPE> &v)
{
    uint4 *p = reinterpret_cast<uint4 *>(static_cast<unsigned char *>(base) + e * type_size(TYPE));
    p[0] = v.q[0];
    if constexpr (TYPE == ADACOMP_TYPE_F32) p[1] = v.q[1];
}

template <u32 TYPE> __device__ inline void widen8(const Vec8<TYPE> &r, float (&v)[8])
{
    const u32 *w = reinterpret_cast<const u32 *>(r.q);
    if constexpr (TYPE == ADACOMP_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = __uint_as_float(w[i]);
    } else if constexpr (TYPE == ADACOMP_TYPE_BF16) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __half2 h = *reinterpret_cast<const __half2 *>(&w[i]);
            const float2 f = __half22float2(h);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}

template <u32 TYPE> __device__ inline Vec8<TYPE> narrow8(const float (&v)[8])
{
    Vec8<TYPE> r;
    u32 *w = reinterpret_cast<u32 *>(r.q);
    if constexpr (TYPE == ADACOMP_TYPE_F32) {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = __float_as_uint(v[i]);
    } else if constexpr (TYPE == ADACOMP_TYPE_BF16) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const u32 *>(&b);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const u32 *>(&h);
        }
    }
    return r;
}

template <u32 TYPE> __device__ inline float load1(const void *base, u64 e)
{
    if constexpr (TYPE == ADACOMP_TYPE_F32) return static_cast<const float *>(base)[e];
    else if constexpr (TYPE == ADACOMP_TYPE_BF16)
        return __uint_as_float((u32) static_cast<const unsigned short *>(base)[e] << 16);
    else return __half2float(static_cast<const __half *>(base)[e]);
}

template <u32 TYPE> __device__ inline void store1(void *base, u64 e, float v)
{
    if constexpr (TYPE == ADACOMP_TYPE_F32) static_cast<float *>(base)[e] = v;
    else if constexpr (TYPE == ADACOMP_TYPE_BF16) static_cast<__nv_bfloat16 *>(base)[e] = __float2bfloat16_rn(v);
    else static_cast<__half *>(base)[e] = __float2half_rn(v);
}

// ---------------------------------------------------------------------------------
// how a row's threads share its columns
//
// A row belongs to `tpr` threads (a multiple of 32); each holds blocks k = 0, 1, .. of eight elements.
//   WIDE   rows start on a vector boundary (their length is a multiple of 8): block k of thread t is the eight
//          neighbouring columns from 8 * (k * tpr + t) on, one 16-byte access (two for binary32)
//   else   any length: element e of block k is column (8 k + e) * tpr + t, so that each access of a warp covers 32
//          neighbouring elements wherever the row starts
// ---------------------------------------------------------------------------------

template <bool WIDE> __device__ inline u32 column(u32 k, u32 e, u32 t, u32 tpr)
{
    return WIDE ? (k * tpr + t) * 8u + e : (k * 8u + e) * tpr + t;
}

// Elements of block k that lie before column `end`; the others are `fill` (WIDE reads whole vectors, which lie inside
// the row because the distance between rows is a multiple of 8).
template <u32 TYPE, bool WIDE>
__device__ inline void load_block(const void *base, u64 row_at, u32 k, u32 t, u32 tpr, u32 end, float fill, float (&v)[8])
{
    if constexpr (WIDE) {
        const u32 c = column<true>(k, 0, t, tpr);
        if (c < end) widen8<TYPE>(load8<TYPE>(base, row_at + c), v);
        if (c + 8 > end) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (c + e >= end) v[e] = fill;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const u32 c = column<false>(k, e, t, tpr);
            v[e] = c < end ? load1<TYPE>(base, row_at + c) : fill;
        }
    }
}

template <u32 TYPE, bool WIDE>
__device__ inline void store_block(void *base, u64 row_at, u32 k, u32 t, u32 tpr, u32 cols, const float (&v)[8])
{
    if constexpr (WIDE) {
        const u32 c = column<true>(k, 0, t, tpr);
        if (c + 8 <= cols) {
            store8<TYPE>(base, row_at + c, narrow8<TYPE>(v));
        } else {                // what lies behind the row's last column is not this tensor's
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (c + e < cols) store1<TYPE>(base, row_at + c + e, v[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const u32 c = column<false>(k, e, t, tpr);
            if (c < cols) store1<TYPE>(base, row_at + c, v[e]);
        }
    }
}

// A parameter vector (its type known at run time) in the same layout.
template <bool WIDE>
__device__ inline void load_param(const void *p, u32 type, u32 k, u32 t, u32 tpr, u32 cols, float fill, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = fill;
    if (!p) return;
    if (type == ADACOMP_TYPE_F32) load_block<ADACOMP_TYPE_F32, WIDE>(p, 0, k, t, tpr, cols, fill, v);
    else if (type == ADACOMP_TYPE_BF16) load_block<ADACOMP_TYPE_BF16, WIDE>(p, 0, k, t, tpr, cols, fill, v);
    else load_block<ADACOMP_TYPE_F16, WIDE>(p, 0, k, t, tpr, cols, fill, v);
}

// ---------------------------------------------------------------------------------
// dropout: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011)
// key = seed, counter = (column / 8, row, step, site); the 128 bits are eight 16-bit numbers, one per column of the
// group (low half of a word first).  Sixteen bits per element rather than 32 halve the generator's work; the kept
// fraction is then a multiple of 2^-16, and the factor is the reciprocal of exactly that fraction.
// ---------------------------------------------------------------------------------

struct DropArgs {
    const u64 *rng;          // device: {seed, step}
    u32 site, threshold;     // an element is dropped when its 16 bits are below the threshold (0 .. 65536)
    float factor;
};

struct Drop {
    u32 k0, k1, step, site, threshold;
    float factor;
};

__device__ inline Drop drop_begin(const DropArgs &a)
{
    const u64 seed = a.rng[0], step = a.rng[1];
    return {(u32)seed, (u32)(seed >> 32), (u32)step, a.site, a.threshold, a.factor};
}

__device__ inline void philox(const Drop &d, u32 group, u32 row, u32 (&out)[4])
{
    u32 c0 = group, c1 = row, c2 = d.step, c3 = d.site, k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const u64 a = (u64)c0 * 0xD2511F53u, b = (u64)c2 * 0xCD9E8D57u;
        c0 = (u32)(b >> 32) ^ c1 ^ k0;
        c2 = (u32)(a >> 32) ^ c3 ^ k1;
        c1 = (u32)b;
        c3 = (u32)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0, out[1] = c1, out[2] = c2, out[3] = c3;
}

// The random words of block k of thread t.  In the WIDE layout a block is one group.  In the other a group's columns lie
// in one octet of lanes: lane q of the octet generates the group of element q, and an 8 x 8 transposition of 16-bit
// halves among the octet (three exchanges) hands every lane its element of each group.  All lanes take part.
// `group0`: the group of the first column of the threads' share of the row.
template <bool WIDE> __device__ inline void drop_words(const Drop &d, u32 row, u32 group0, u32 k, u32 t, u32 tpr, u32 (&w)[4])
{
    if constexpr (WIDE) {
        philox(d, group0 + k * tpr + t, row, w);
    } else {
        const u32 q = t & 7u;
        philox(d, group0 + (((k * 8u + q) * tpr + (t & ~7u)) >> 3), row, w);
        {
            const bool up = q & 4u;
            const u32 r0 = __shfl_xor_sync(kAllLanes, up ? w[0] : w[2], 4);
            const u32 r1 = __shfl_xor_sync(kAllLanes, up ? w[1] : w[3], 4);
            if (up) w[0] = r0, w[1] = r1;
            else w[2] = r0, w[3] = r1;
        }
        {
            const bool up = q & 2u;
            const u32 r0 = __shfl_xor_sync(kAllLanes, up ? w[0] : w[1], 2);
            const u32 r1 = __shfl_xor_sync(kAllLanes, up ? w[2] : w[3], 2);
            if (up) w[0] = r0, w[2] = r1;
            else w[1] = r0, w[3] = r1;
        }
        {
            const bool up = q & 1u;
            const u32 s0 = up ? __byte_perm(w[0], w[1], 0x5410) : __byte_perm(w[0], w[1], 0x7632);
            const u32 s1 = up ? __byte_perm(w[2], w[3], 0x5410) : __byte_perm(w[2], w[3], 0x7632);
            const u32 r0 = __shfl_xor_sync(kAllLanes, s0, 1);
            const u32 r1 = __shfl_xor_sync(kAllLanes, s1, 1);
            if (up) {       // keep the high halves, the partner's high halves go below them
                w[0] = __byte_perm(r0, w[0], 0x7610), w[1] = __byte_perm(r0, w[1], 0x7632);
                w[2] = __byte_perm(r1, w[2], 0x7610), w[3] = __byte_perm(r1, w[3], 0x7632);
            } else {        // keep the low halves, the partner's low halves go above them
                w[0] = __byte_perm(w[0], r0, 0x5410), w[1] = __byte_perm(w[1], r0, 0x7610);
                w[2] = __byte_perm(w[2], r1, 0x5410), w[3] = __byte_perm(w[3], r1, 0x7610);
            }
        }
    }
}

__device__ inline bool dropped(const Drop &d, const u32 (&w)[4], int e)
{
    return ((e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) < d.threshold;
}

// v = dropout(v): selected, not multiplied, so that infinities and NaN in dropped places leave zeros.
__device__ inline void drop_apply(const Drop &d, const u32 (&w)[4], float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = dropped(d, w, e) ? 0.f : v[e] * d.factor;
}

// ---------------------------------------------------------------------------------
// sums over a row's threads
// ---------------------------------------------------------------------------------

__device__ inline float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAllLanes, v, d);
    return v;
}

__device__ inline float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kAllLanes, v, d));
    return v;
}

// The threads of one row: `tpr` neighbouring threads of a CTA.  Rows of up to one warp need no barrier, others meet at
// named barrier 1 + g (at most 15 rows share a CTA then).
struct RowGroup {
    u32 g, t, tpr, warps, warp, lane;
    __device__ explicit RowGroup(u32 threads_per_row)
        : g(threadIdx.x / threads_per_row), t(threadIdx.x % threads_per_row), tpr(threads_per_row),
          warps(threads_per_row >> 5), warp(t >> 5), lane(t & 31u)
    {
    }
    __device__ void sync() const
    {
        if (warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(g + 1u), "r"(tpr) : "memory");
    }
};

// n / d for n < 2^31 by a multiplication (Granlund and Montgomery, "Division by invariant integers using
// multiplication", 1994)
struct FastDiv {
    u32 d, mul, shift;
};

inline FastDiv make_fastdiv(u32 d)
{
    u32 s = 0;
    while ((1ull << s) < d) s++;
    return {d, (u32)(((1ull << 32) * ((1ull << s) - d)) / d + 1), s};
}

__device__ inline u32 fast_div(u32 n, const FastDiv &f) { return (__umulhi(n, f.mul) + n) >> f.shift; }

}  // namespace adacomp_impl

// What the forward and backward kernels of the biased softmax share.
#pragma once

#include "block.h"

namespace adacomp_impl {

namespace cg = cooperative_groups;

constexpr int kSoftThreads = 512;            // most threads of a CTA
constexpr u32 kSoftSlice = 16384;            // most columns of one CTA: 512 threads, four blocks of eight each
constexpr u32 kSoftMinThreads = 128;         // short rows share a CTA of this many threads
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 2^x by the hardware's approximation (PTX ex2.approx: within 2 units in the last place); -inf gives 0.
__device__ inline float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// e^(x - about), about not -inf.  The product with log2(e) is taken of the difference where that of `about` would
// overflow: rows of a type's lowest value (a mask added by the caller) keep their softmax.
__device__ inline bool far_out(float about) { return !(fabsf(about) < 1e38f); }
__device__ inline float exp_about(float x, float about, float about2, bool far)
{
    return exp2_fast(far ? (x - about) * kLog2e : fmaf(x, kLog2e, -about2));
}

// The bias by distance, for one head: entry d + reach for d = key - query in -reach .. reach, farther distances share the
// end entries (their bucket is the last one of their side).  A thread of the WIDE layout reads eight neighbouring entries,
// its neighbour the eight next to those: a gap after every eight entries puts those of 32 lanes into 32 banks.
__device__ inline u32 padded(u32 i) { return i + (i >> 3); }
__host__ __device__ inline u32 table_floats(u32 reach) { return (2 * reach + 1) + ((2 * reach + 1) >> 3) + 1; }

__device__ inline u32 bucket_of(const SoftmaxArgs &a, int d)
{
    const u32 away = d <= 0 ? (u32)-d : a.both ? (u32)d : 0u;
    u32 b = 0;
    for (u32 k = 1; k < a.side; k++) b += a.first[k] <= away ? 1u : 0u;
    return d > 0 && a.both ? b + a.side : b;
}

__device__ inline void build_table(const SoftmaxArgs &a, const RowGroup &rg, u32 head, float *bias)
{
    const int reach = (int)a.reach;
    for (int i = (int)rg.t; i <= 2 * reach; i += (int)rg.tpr)
        bias[padded(i)] = a.table ? a.table[(u64)bucket_of(a, i - reach) * a.heads + head] : 0.f;
}

// Which rows a group of threads works on, and where.
struct SoftmaxRows {
    u32 bh, head, i0, i1, rank, c0, cols;
    int bound;              // keys of this sequence
    bool any;
    __device__ SoftmaxRows(const SoftmaxArgs &a, const RowGroup &rg)
    {
        rank = a.cluster > 1 ? cg::this_cluster().block_rank() : 0u;
        const u64 id = (u64)(blockIdx.x / a.cluster) * a.groups + rg.g;
        any = id < (u64)a.batch * a.heads * a.chunks;
        bh = (u32)(id / a.chunks);
        head = bh % a.heads;
        i0 = (u32)(id % a.chunks) * a.chunk_rows;
        i1 = min(i0 + a.chunk_rows, a.q_len);
        c0 = rank * a.slice;
        cols = c0 < a.k_len ? min(a.slice, a.k_len - c0) : 0u;
        bound = (int)a.k_len;
        if (any && a.key_len) bound = max(0, min(bound, a.key_len[bh / a.heads]));
    }
    // one past the last kept column of row i, counted from this CTA's first
    __device__ u32 end(const SoftmaxArgs &a, u32 i) const
    {
        int e = bound;
        if (a.causal) e = min(e, (int)i + a.q_offset + 1);
        return (u32)max(0, min(e - (int)c0, (int)cols));
    }
};

// v: scores of block k, replaced by logits; columns from `end` on become -inf.  `d0`: distance key -
// query of this CTA's first column.
template <bool WIDE>
__device__ inline void to_logits(float (&v)[8], const float *bias, int reach, float scale, int d0, u32 k, u32 t, u32 tpr, u32 end)
{
    if constexpr (WIDE) {
        const u32 c = column<true>(k, 0, t, tpr);
        const int d = d0 + (int)c;
        if (d >= reach || d + 7 <= -reach) {
            const float far = bias[padded(d >= reach ? 2 * reach : 0)];
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = fmaf(v[e], scale, far);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++)
                v[e] = fmaf(v[e], scale, bias[padded(max(-reach, min(reach, d + e)) + reach)]);
        }
        if (c + 8 > end) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (c + e >= end) v[e] = -INFINITY;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const u32 c = column<false>(k, e, t, tpr);
            const int d = max(-reach, min(reach, d0 + (int)c));
            v[e] = c < end ? fmaf(v[e], scale, bias[padded(d + reach)]) : -INFINITY;
        }
    }
}

template <typename K> inline void launch_softmax_kernel(K kernel, const SoftmaxArgs &a, size_t smem, cudaStream_t st)
{
    if (smem > 48 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    const u64 sets = ((u64)a.batch * a.heads * a.chunks + a.groups - 1) / a.groups;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(sets * a.cluster));
    cfg.blockDim = dim3(a.tpr * a.groups);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = a.cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = a.cluster > 1 ? 1 : 0;
    cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace adacomp_impl

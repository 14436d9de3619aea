// Attention softmax with a learned relative position bias by buckets, forward: from scores to probabilities, with the
// scale, the causal and length masks and dropout, in one pass.
#include "softmax.cuh"

namespace adacomp_impl {

// How rows are shared, by the sizes alone: a warp per row up to 1024 keys (8 to 32 per lane), more warps up to 16384, a
// cluster of CTAs beyond.  A group of threads takes `chunk_rows` rows of one head, so that it lays the head's bias out by
// distance once.
void softmax_split(SoftmaxArgs &a)
{
    a.cluster = 1;
    while (a.k_len > a.cluster * kSoftSlice) a.cluster *= 2;
    a.slice = a.cluster == 1 ? a.k_len : ((a.k_len + a.cluster - 1) / a.cluster + 7u) & ~7u;
    const u32 blocks = (a.slice + 7u) / 8u;
    a.tpr = blocks <= 128u ? 32u : ((blocks + 3u) / 4u + 31u) & ~31u;
    a.groups = a.cluster == 1 && a.tpr < kSoftMinThreads ? kSoftMinThreads / a.tpr : 1u;
    const u64 rows = (u64)a.batch * a.heads * a.q_len;
    const u64 at_once = 2ull * kBlockSms * 1024 / ((u64)a.tpr * a.cluster);      // groups of two full waves
    u64 chunk = rows / at_once;
    chunk = chunk < 1 ? 1 : chunk > 64 ? 64 : chunk;
    if (chunk > a.q_len) chunk = a.q_len;
    a.chunk_rows = chunk < 1 ? 1u : (u32)chunk;
    a.chunks = (a.q_len + a.chunk_rows - 1) / a.chunk_rows;
}

// A row stays in registers.  Each warp takes powers of two about its own maximum; the maxima and sums of the row's warps
// are joined in one meeting, and what a warp holds is rescaled as it is stored.
template <u32 TYPE, bool WIDE, int NV, bool DROP>
__global__ void __launch_bounds__(kSoftThreads) softmax_forward(const SoftmaxArgs a)
{
    extern __shared__ float tables[];
    __shared__ float2 part[2][kSoftThreads / 32];
    __shared__ float2 peers[2][8];
    const RowGroup rg(a.tpr);
    const SoftmaxRows rows(a, rg);
    if (!rows.any) return;
    if (a.cluster > 1) cg::this_cluster().sync();      // every CTA of the cluster runs before its memory is written
    float *bias = tables + rg.g * table_floats(a.reach);
    build_table(a, rg, rows.head, bias);
    rg.sync();
    Drop d;
    if constexpr (DROP) d = drop_begin(a.drop);
    const u32 first_warp = rg.g * rg.warps;
    u32 parity = 0;
    for (u32 i = rows.i0; i < rows.i1; i++, parity ^= 1u) {
        const u64 row = (u64)rows.bh * a.q_len + i, at = row * a.ld + rows.c0;
        const u32 end = rows.end(a, i);
        const int d0 = (int)rows.c0 - ((int)i + a.q_offset);
        float v[NV][8];
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < NV; k++) load_block<TYPE, WIDE>(a.scores, at, k, rg.t, rg.tpr, end, 0.f, v[k]);
#pragma unroll
        for (int k = 0; k < NV; k++) {
            to_logits<WIDE>(v[k], bias, (int)a.reach, a.scale, d0, k, rg.t, rg.tpr, end);
#pragma unroll
            for (int e = 0; e < 8; e++) top = fmaxf(top, v[k][e]);
        }
        const float warp_top = warp_max(top);
        const float about = warp_top == -INFINITY ? 0.f : warp_top;
        const bool far = far_out(about);
        const float about2 = about * kLog2e;
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                v[k][e] = exp_about(v[k][e], about, about2, far);
                s += v[k][e];
            }
        s = warp_sum(s);
        top = warp_top;
        if (rg.warps > 1) {
            if (rg.lane == 0) part[parity][first_warp + rg.warp] = make_float2(warp_top, s);
            rg.sync();
            const float2 p = rg.lane < rg.warps ? part[parity][first_warp + rg.lane] : make_float2(-INFINITY, 0.f);
            top = warp_max(p.x);
            s = warp_sum(p.y * exp2_fast((p.x - (top == -INFINITY ? 0.f : top)) * kLog2e));
        }
        if (a.cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < a.cluster) cl.map_shared_rank(&peers[parity][0], threadIdx.x)[rows.rank] = make_float2(top, s);
            cl.sync();
            for (u32 j = 0; j < a.cluster; j++) top = fmaxf(top, peers[parity][j].x);
            s = 0.f;
            for (u32 j = 0; j < a.cluster; j++)
                s += peers[parity][j].y * exp2_fast((peers[parity][j].x - (top == -INFINITY ? 0.f : top)) * kLog2e);
        }
        // a row that keeps nothing has s = 0 and becomes zeros
        const float f = s == 0.f ? 0.f : exp2_fast((about - (top == -INFINITY ? 0.f : top)) * kLog2e) / s;
        if (a.lse && rg.t == 0 && rows.rank == 0) a.lse[row] = s == 0.f ? -INFINITY : top + log2f(s) * kLn2;
#pragma unroll
        for (int k = 0; k < NV; k++) {
#pragma unroll
            for (int e = 0; e < 8; e++) v[k][e] *= f;
            if constexpr (DROP) {
                u32 bits[4];
                drop_words<WIDE>(d, (u32)row, rows.c0 >> 3, k, rg.t, rg.tpr, bits);
                drop_apply(d, bits, v[k]);
            }
            store_block<TYPE, WIDE>(a.probs, at, k, rg.t, rg.tpr, rows.cols, v[k]);
        }
    }
}

template <u32 TYPE, bool WIDE, int NV> static void launch_drop(const SoftmaxArgs &a, cudaStream_t st)
{
    const size_t smem = (size_t)a.groups * table_floats(a.reach) * sizeof(float);
    if (a.drop.threshold) launch_softmax_kernel(softmax_forward<TYPE, WIDE, NV, true>, a, smem, st);
    else launch_softmax_kernel(softmax_forward<TYPE, WIDE, NV, false>, a, smem, st);
}

template <u32 TYPE, bool WIDE> static void launch_blocks(const SoftmaxArgs &a, cudaStream_t st)
{
    const u32 per = (a.slice + a.tpr * 8u - 1) / (a.tpr * 8u);
    if (per <= 1) launch_drop<TYPE, WIDE, 1>(a, st);
    else if (per == 2) launch_drop<TYPE, WIDE, 2>(a, st);
    else launch_drop<TYPE, WIDE, 4>(a, st);
}

template <u32 TYPE> static void launch_type(const SoftmaxArgs &a, cudaStream_t st)
{
    if (a.ld % 8u == 0) launch_blocks<TYPE, true>(a, st);
    else launch_blocks<TYPE, false>(a, st);
}

int launch_softmax(SoftmaxArgs &a, u32 type, cudaStream_t st)
{
    if ((u64)a.batch * a.heads * a.q_len == 0) return ADACOMP_OK;
    softmax_split(a);
    if (type == ADACOMP_TYPE_F32) launch_type<ADACOMP_TYPE_F32>(a, st);
    else if (type == ADACOMP_TYPE_BF16) launch_type<ADACOMP_TYPE_BF16>(a, st);
    else launch_type<ADACOMP_TYPE_F16>(a, st);
    return launched();
}

}  // namespace adacomp_impl

// Attention softmax with a learned relative position bias by buckets, forward: from scores to probabilities, with the
// scale, the causal and length masks and dropout, in one pass.
#include "softmax.cuh"

#ifndef SFB
#define SFB 1
#endif
#ifndef ONEW
#define ONEW 128u
#endif
namespace adacomp_impl {

// How rows are shared, by the sizes alone: a warp per row up to 1024 keys (8, 16 or 32 of them per lane), up to 16 warps
// with 16 per lane up to 8192, a cluster of up to 8 such CTAs up to 65536, with 32 per lane beyond.
void softmax_split(SoftmaxArgs &a)
{
    const u32 blocks = (a.k_len + 7u) / 8u;
    a.cluster = 1;
    if (blocks <= ONEW) {
        a.per = blocks <= 32u ? 1u : blocks <= 64u ? 2u : 4u;
        a.tpr = 32;
        a.groups = kSoftShort / 32;
    } else {
        while (a.cluster < 8u && blocks > a.cluster * kSoftThreads * 2u) a.cluster *= 2;
        a.per = blocks > 8u * kSoftThreads * 2u ? 4u : 2u;
        const u32 each = (blocks + a.cluster - 1) / a.cluster;
        a.tpr = ((each + a.per - 1) / a.per + 31u) & ~31u;
        a.groups = a.cluster == 1 && a.tpr < kSoftShort ? kSoftShort / a.tpr : 1u;
    }
    a.slice = a.cluster == 1 ? a.k_len : ((a.k_len + a.cluster - 1) / a.cluster + 7u) & ~7u;
    while (a.groups > 1 && a.groups > a.q_len) a.groups /= 2;
    // runs long enough to lay out the head's bias rarely, short enough for four CTAs' worth of work per place on the GPU
    const u64 rows = (u64)a.batch * a.heads * a.q_len, places = (u64)kBlockSms * 16 * 32 / a.tpr;
    u64 run = rows / (places * 4);
    run = run < 1 ? 1 : run > 16 ? 16 : run;
    const u32 most = (a.q_len + a.groups - 1) / a.groups;
    a.run = run < most ? (u32)run : most ? most : 1u;
    a.chunks = (a.q_len + a.groups * a.run - 1) / (a.groups * a.run);
}

// A row stays in registers.  Each warp takes powers of two about its own maximum; the maxima and sums of the row's warps
// are joined in one meeting, and what a warp holds is rescaled as it is stored.
template <u32 TYPE, bool ALIGNED, int NV, bool DROP, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kSoftShort ? SFB : 1) softmax_forward(const SoftmaxArgs a)
{
    extern __shared__ float4 tables[];
    __shared__ float2 part[2][THREADS / 32];
    __shared__ float2 peers[2][8];
    float *bias = reinterpret_cast<float *>(tables);
    const RowGroup rg(a.tpr);
    const SoftmaxRows rows(a, rg);
    if (a.cluster > 1) cg::this_cluster().sync();      // every CTA of the cluster runs before its memory is written
    Raw<TYPE, ALIGNED> raw[NV];
    clear(raw);
    auto fetch_row = [&](u32 i) {
        const u64 at = ((u64)rows.bh * a.q_len + i) * a.ld + rows.c0;
        const u32 end = i < rows.i1 ? rows.end(a, i) : 0u;
#pragma unroll
        for (int k = 0; k < NV; k++) fetch<TYPE, ALIGNED>(raw[k], a.scores, at, block_column<NV>(k, rg.t), end);
    };
    fetch_row(rows.i0);
    build_bias(a, rows.bh % a.heads, bias);
    __syncthreads();
    Drop d;
    if constexpr (DROP) d = drop_begin(a.drop);
    u32 parity = 0;
#pragma unroll 1
    for (u32 i = rows.i0; i < rows.i1; i++, parity ^= 1u) {
        const u64 row = (u64)rows.bh * a.q_len + i, at = row * a.ld + rows.c0;
        const u32 end = rows.end(a, i);
        const int d0 = (int)rows.c0 - ((int)i + a.q_offset);
        float v[NV][8];
        float top = -INFINITY, top2 = -INFINITY;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const u32 c = block_column<NV>(k, rg.t);
            unpack<TYPE, ALIGNED>(raw[k], at, v[k]);
            add_bias(v[k], bias, (int)a.reach, a.scale, d0 + (int)c);
            mask_from(v[k], c, end, -INFINITY);
#pragma unroll
            for (int e = 0; e < 8; e += 2) top = fmaxf(top, v[k][e]), top2 = fmaxf(top2, v[k][e + 1]);
        }
        fetch_row(i + 1);               // the next row is on its way while this one is worked on
        top = warp_max(fmaxf(top, top2));
        const float about = top == -INFINITY ? 0.f : top;
        exp_about<NV>(v, about);
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++) s += ((v[k][0] + v[k][1]) + (v[k][2] + v[k][3])) + ((v[k][4] + v[k][5]) + (v[k][6] + v[k][7]));
        s = warp_sum(s);
        if (rg.warps > 1) {
            if (rg.lane == 0) part[parity][rg.first_warp + rg.warp] = make_float2(top, s);
            rg.sync();
            const u32 w = rg.lane & 15u;
            const float2 p = w < rg.warps ? part[parity][rg.first_warp + w] : make_float2(-INFINITY, 0.f);
            top = warp_max(p.x);
            s = half_sum(p.y * exp2_fast((p.x - (top == -INFINITY ? 0.f : top)) * kLog2e));
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
        float f = s == 0.f ? 0.f : exp2_fast((about - (top == -INFINITY ? 0.f : top)) * kLog2e) * __fdividef(1.f, s);
        if (a.lse && rg.t == 0 && rows.rank == 0) a.lse[row] = s == 0.f ? -INFINITY : fmaf(__log2f(s), kLn2, top);
        if constexpr (DROP) f *= d.factor;
        if constexpr (DROP) {
            constexpr int N = NV < 2 ? 1 : 2;       // blocks that draw together
#pragma unroll
            for (int k0 = 0; k0 < NV; k0 += N) {
                u32 rws[N], groups[N], bits[N][4];
#pragma unroll
                for (int k = 0; k < N; k++) rws[k] = (u32)row, groups[k] = (rows.c0 + block_column<NV>(k0 + k, rg.t)) >> 3;
                drop_words<N>(d, rws, groups, bits);
#pragma unroll
                for (int k = 0; k < N; k++)
#pragma unroll
                    for (int e = 0; e < 8; e++) v[k0 + k][e] = dropped(d, bits[k], e) ? 0.f : v[k0 + k][e] * f;
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; k++)
#pragma unroll
                for (int e = 0; e < 8; e++) v[k][e] *= f;
        }
#pragma unroll
        for (int k = 0; k < NV; k++) store_block<TYPE, ALIGNED>(a.probs, at, block_column<NV>(k, rg.t), rows.cols, v[k]);
    }
}

template <u32 TYPE, bool ALIGNED, int NV, int THREADS> static void launch_drop(const SoftmaxArgs &a, cudaStream_t st)
{
    const size_t smem = bias_floats(a.reach) * sizeof(float);
    if (a.drop.threshold) launch_softmax_kernel(softmax_forward<TYPE, ALIGNED, NV, true, THREADS>, a, smem, st);
    else launch_softmax_kernel(softmax_forward<TYPE, ALIGNED, NV, false, THREADS>, a, smem, st);
}

template <u32 TYPE, bool ALIGNED> static void launch_blocks(const SoftmaxArgs &a, cudaStream_t st)
{
    if (a.tpr == 32) {
        if (a.per == 1) launch_drop<TYPE, ALIGNED, 1, kSoftShort>(a, st);
        else if (a.per == 2) launch_drop<TYPE, ALIGNED, 2, kSoftShort>(a, st);
        else launch_drop<TYPE, ALIGNED, 4, kSoftShort>(a, st);
    } else {
        if (a.per == 2) launch_drop<TYPE, ALIGNED, 2, kSoftThreads>(a, st);
        else launch_drop<TYPE, ALIGNED, 4, kSoftThreads>(a, st);
    }
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

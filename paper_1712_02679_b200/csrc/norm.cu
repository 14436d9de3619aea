// Layer norm, forward: h = residual + dropout(x), y = (h - mean(h)) / sqrt(var(h) + eps) * weight + bias.
#include "norm.cuh"

#ifndef NFB
#define NFB 1
#endif
namespace adacomp_impl {

// How a row's columns are shared, by the width alone: one thread per eight columns; a CTA of up to 512 threads, beyond
// 4096 columns a cluster of up to 8 of them, beyond 32768 two blocks of eight per thread; short rows share a CTA.
void norm_split(NormArgs &a)
{
    a.cluster = 1;
    while (a.cluster < 8u && a.cols > a.cluster * kNormThreads * 8u) a.cluster *= 2;
    a.slice = a.cluster == 1 ? a.cols : ((a.cols + a.cluster - 1) / a.cluster + 7u) & ~7u;
    const u32 blocks = (a.slice + 7u) / 8u;
    a.per = blocks > (u32)kNormThreads ? 2u : 1u;
    a.tpr = ((blocks + a.per - 1) / a.per + 31u) & ~31u;
    a.groups = a.cluster == 1 && a.per == 1 ? (u32)kNormThreads / a.tpr : 1u;
    const u64 sets = (a.rows + a.groups - 1) / a.groups, most = 2u * kBlockSms / a.cluster;
    a.partials = (u32)(sets < most ? sets : most);
}

// A row stays in registers from its load to its store.  Mean and sum of squared distances from it are formed per thread
// about the thread's own mean, and merged twice (lanes of a warp, warps of the row) about the first one's mean m0: with
// A = sum n d and B = sum (M2 + n d^2), d = mean - m0, the merged mean is m0 + A / n and the merged sum B - A^2 / n.  The
// first of 32 (16) parts has at least 1/32 (1/16) of the elements, so that difference loses a factor of 32 (16) at the
// very worst, however far the row's mean is from zero (Chan, Golub, LeVeque, 1979); one pass, one meeting of the warps.
template <u32 TYPE, bool ALIGNED, int NV, bool DROP>
__global__ void __launch_bounds__(kNormThreads, NFB) norm_forward(const NormArgs a)
{
    __shared__ float4 part[2][kNormThreads / 32];        // m0, A, B of a warp
    __shared__ float2 counts[kNormThreads / 32];         // its columns, and 1 / that
    __shared__ float4 peers[2][8];
    const RowGroup rg(a.tpr);
    const u32 rank = a.cluster > 1 ? cg::this_cluster().block_rank() : 0u;
    if (a.cluster > 1) cg::this_cluster().sync();      // every CTA of the cluster runs before its memory is written
    const u32 c0 = rank * a.slice, cols = min(a.slice, a.cols - c0);
    const u64 psize = type_size(a.param_type);
    const void *wp = a.weight ? static_cast<const unsigned char *>(a.weight) + c0 * psize : nullptr;
    const void *bp = a.bias ? static_cast<const unsigned char *>(a.bias) + c0 * psize : nullptr;
    Raw<TYPE, ALIGNED> rx[NV], rr[NV];
    clear(rx);
    clear(rr);
    auto fetch_row = [&](u64 r) {
        const u32 end = r < a.rows ? cols : 0u;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const u32 c = block_column<NV>(k, rg.t);
            fetch<TYPE, ALIGNED>(rx[k], a.x, r * a.cols + c0, c, end);
            if (a.residual) fetch<TYPE, ALIGNED>(rr[k], a.residual, r * a.cols + c0, c, end);
        }
    };
    const u64 step = (u64)(gridDim.x / a.cluster) * a.groups;
    u64 row = (u64)(blockIdx.x / a.cluster) * a.groups + rg.g;
    fetch_row(row);
    float w[NV][8], b[NV][8];
    float n_mine = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++) {
        const u32 c = block_column<NV>(k, rg.t);
        load_param(wp, a.param_type, c, cols, 1.f, w[k]);
        load_param(bp, a.param_type, c, cols, 0.f, b[k]);
        n_mine += (float)min(8u, cols - min(c, cols));
    }
    const float inv_mine = n_mine > 0.f ? 1.f / n_mine : 0.f;
    const float n_warp = warp_sum(n_mine), inv_warp = n_warp > 0.f ? 1.f / n_warp : 0.f;
    if (rg.lane == 0) counts[rg.first_warp + rg.warp] = make_float2(n_warp, inv_warp);
    Drop d;
    if constexpr (DROP) d = drop_begin(a.drop);
    const float inv_cols = 1.f / (float)a.cols, inv_cta = 1.f / (float)cols;
    u32 parity = 0;
#pragma unroll 1
    for (; row < a.rows; row += step, parity ^= 1u) {
        const u64 at = row * a.cols + c0;
        float h[NV][8];
#pragma unroll
        for (int k = 0; k < NV; k++) unpack<TYPE, ALIGNED>(rx[k], at, h[k]);
        if constexpr (DROP) {
            u32 rows[NV], groups[NV], bits[NV][4];
#pragma unroll
            for (int k = 0; k < NV; k++) rows[k] = (u32)row, groups[k] = (c0 + block_column<NV>(k, rg.t)) >> 3;
            drop_words<NV>(d, rows, groups, bits);
#pragma unroll
            for (int k = 0; k < NV; k++) drop_apply(d, bits[k], h[k]);
        }
        if (a.residual) {
#pragma unroll
            for (int k = 0; k < NV; k++) {
                float r[8];
                unpack<TYPE, ALIGNED>(rr[k], at, r);
#pragma unroll
                for (int e = 0; e < 8; e++) h[k][e] += r[e];
            }
        }
        fetch_row(row + step);          // the next row is on its way while this one is worked on
        // (blocks of an ALIGNED row are whole or hold the zeros they were cleared to)
        if constexpr (!ALIGNED) {
#pragma unroll
            for (int k = 0; k < NV; k++) mask_from(h[k], block_column<NV>(k, rg.t), cols, 0.f);
        }
        if (a.h) {
#pragma unroll
            for (int k = 0; k < NV; k++) store_block<TYPE, ALIGNED>(a.h, at, block_column<NV>(k, rg.t), cols, h[k]);
        }
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++) s += ((h[k][0] + h[k][1]) + (h[k][2] + h[k][3])) + ((h[k][4] + h[k][5]) + (h[k][6] + h[k][7]));
        const float mt = s * inv_mine;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] = h[k][e] - mt;
            if (!ALIGNED || NV > 1) mask_from(x, block_column<NV>(k, rg.t), cols, 0.f);
            float q0 = 0.f, q1 = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e += 2) q0 = fmaf(x[e], x[e], q0), q1 = fmaf(x[e + 1], x[e + 1], q1);
            q += q0 + q1;
        }
        float m0 = from_lane(mt, 0), off = mt - m0, nd = n_mine * off;
        float v = warp_two_sums(nd, fmaf(nd, off, q), rg.lane);
        float inv_n = inv_warp;
        if (rg.warps > 1) {
            float4 *slot = &part[parity][rg.first_warp + rg.warp];
            if (rg.lane == 0) slot->x = m0, slot->y = v;
            if (rg.lane == 16) slot->z = v;
            rg.sync();
            const u32 i = rg.lane & 15u;
            float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
            float2 n = make_float2(0.f, 0.f);
            if (i < rg.warps) p = part[parity][rg.first_warp + i], n = counts[rg.first_warp + i];
            const float mw = fmaf(p.y, n.y, p.x), qw = fmaf(-p.y * p.y, n.y, p.z);
            m0 = from_lane(mw, 0);
            off = mw - m0;
            nd = n.x * off;
            v = half_sum(rg.lane < 16u ? nd : fmaf(nd, off, qw));
            inv_n = inv_cta;
        }
        float total = from_lane(v, 0), mean = fmaf(total, inv_n, m0);
        q = fmaf(-total * total, inv_n, from_lane(v, 16));
        if (a.cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < a.cluster)
                cl.map_shared_rank(&peers[parity][0], threadIdx.x)[rank] = make_float4(mean, q, (float)cols, 0.f);
            cl.sync();
            m0 = peers[parity][0].x;
            total = q = 0.f;
            for (u32 i = 0; i < a.cluster; i++) {
                const float4 p = peers[parity][i];
                off = p.x - m0;
                total = fmaf(p.z, off, total);
                q += fmaf(p.z * off, off, p.y);
            }
            mean = fmaf(total, inv_cols, m0);
            q = fmaf(-total * total, inv_cols, q);
        }
        const float rstd = rsqrtf(fmaf(fmaxf(q, 0.f), inv_cols, a.eps)) + 0.f * q;      // (a NaN in the row stays one)
        if (rg.t == 0 && rank == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < NV; k++) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[k][e] = fmaf((h[k][e] - mean) * rstd, w[k][e], b[k][e]);
            store_block<TYPE, ALIGNED>(a.y, at, block_column<NV>(k, rg.t), cols, h[k]);
        }
    }
}

template <u32 TYPE, bool ALIGNED, int NV> static void launch_drop(const NormArgs &a, u32 sets, cudaStream_t st)
{
    if (a.drop.threshold) launch_norm_kernel(norm_forward<TYPE, ALIGNED, NV, true>, a, sets, st);
    else launch_norm_kernel(norm_forward<TYPE, ALIGNED, NV, false>, a, sets, st);
}

template <u32 TYPE> static void launch_type(const NormArgs &a, u32 sets, cudaStream_t st)
{
    const bool two = a.per == 2u;
    if (a.cols % 8u == 0) two ? launch_drop<TYPE, true, 2>(a, sets, st) : launch_drop<TYPE, true, 1>(a, sets, st);
    else two ? launch_drop<TYPE, false, 2>(a, sets, st) : launch_drop<TYPE, false, 1>(a, sets, st);
}

int launch_norm(NormArgs &a, u32 type, cudaStream_t st)
{
    if (a.rows == 0) return ADACOMP_OK;
    norm_split(a);
    const u64 all = (a.rows + a.groups - 1) / a.groups, most = 8u * kBlockSms / a.cluster;
    const u32 sets = (u32)(all < most ? all : most);
    if (type == ADACOMP_TYPE_F32) launch_type<ADACOMP_TYPE_F32>(a, sets, st);
    else if (type == ADACOMP_TYPE_BF16) launch_type<ADACOMP_TYPE_BF16>(a, sets, st);
    else launch_type<ADACOMP_TYPE_F16>(a, sets, st);
    return launched();
}

}  // namespace adacomp_impl

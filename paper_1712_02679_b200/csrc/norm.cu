// Layer norm, forward: h = residual + dropout(x), y = (h - mean(h)) / sqrt(var(h) + eps) * weight + bias.
#include "norm.cuh"

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

// A row stays in registers from its load to its store.  The mean and the sum of squared distances from it are formed per
// warp about the warp's own mean, and merged (Chan, Golub, LeVeque, 1979): one meeting of the row's warps, and no
// difference of large numbers whatever the row's mean is.
template <u32 TYPE, bool ALIGNED, int NV, bool DROP>
__global__ void __launch_bounds__(kNormThreads) norm_forward(const NormArgs a)
{
    __shared__ float2 part[2][kNormThreads / 32];
    __shared__ float counts[kNormThreads / 32];
    __shared__ float4 peers[2][8];
    const RowGroup rg(a.tpr);
    const u32 rank = a.cluster > 1 ? cg::this_cluster().block_rank() : 0u;
    if (a.cluster > 1) cg::this_cluster().sync();      // every CTA of the cluster runs before its memory is written
    const u32 c0 = rank * a.slice, cols = min(a.slice, a.cols - c0);
    const u64 psize = type_size(a.param_type);
    const void *wp = a.weight ? static_cast<const unsigned char *>(a.weight) + c0 * psize : nullptr;
    const void *bp = a.bias ? static_cast<const unsigned char *>(a.bias) + c0 * psize : nullptr;
    float w[NV][8], b[NV][8];
    float mine = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++) {
        const u32 c = block_column<NV>(k, rg.t);
        load_param(wp, a.param_type, c, cols, 1.f, w[k]);
        load_param(bp, a.param_type, c, cols, 0.f, b[k]);
        mine += (float)min(8u, cols - min(c, cols));
    }
    const float n_warp = warp_sum(mine);
    if (rg.lane == 0) counts[rg.first_warp + rg.warp] = n_warp;
    Drop d;
    if constexpr (DROP) d = drop_begin(a.drop);
    const float inv_cols = 1.f / (float)a.cols, inv_mine = 1.f / (float)cols, inv_warp = n_warp > 0.f ? 1.f / n_warp : 0.f;
    u32 parity = 0;
    const u64 step = (u64)(gridDim.x / a.cluster) * a.groups;
    u64 row = (u64)(blockIdx.x / a.cluster) * a.groups + rg.g;
    Raw<TYPE, ALIGNED> rx[NV], rr[NV];
    auto fetch_row = [&](u64 r) {
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const u32 c = block_column<NV>(k, rg.t), end = r < a.rows ? cols : 0u;
            fetch<TYPE, ALIGNED>(rx[k], a.x, r * a.cols + c0, c, end);
            if (a.residual) fetch<TYPE, ALIGNED>(rr[k], a.residual, r * a.cols + c0, c, end);
        }
    };
    fetch_row(row);
    for (; row < a.rows; row += step, parity ^= 1u) {
        const u64 at = row * a.cols + c0;
        float h[NV][8];
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const u32 c = block_column<NV>(k, rg.t);
            unpack<TYPE, ALIGNED>(rx[k], at, c, cols, 0.f, h[k]);
            if constexpr (DROP) {
                u32 bits[4];
                drop_words(d, (u32)row, (c0 + c) >> 3, bits);
                drop_apply(d, bits, h[k]);
            }
            if (a.residual) {
                float r[8];
                unpack<TYPE, ALIGNED>(rr[k], at, c, cols, 0.f, r);
#pragma unroll
                for (int e = 0; e < 8; e++) h[k][e] += r[e];
            }
        }
        fetch_row(row + step);          // the next row is on its way while this one is worked on
        if (a.h) {
#pragma unroll
            for (int k = 0; k < NV; k++) store_block<TYPE, ALIGNED>(a.h, at, block_column<NV>(k, rg.t), cols, h[k]);
        }
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) s += h[k][e];
        s = warp_sum(s);
        const float mw = s * inv_warp;
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float x = h[k][e] - mw;
                q += block_column<NV>(k, rg.t) + e < cols ? x * x : 0.f;
            }
        q = warp_sum(q);
        float mean = mw;
        if (rg.warps > 1) {
            if (rg.lane == 0) part[parity][rg.first_warp + rg.warp] = make_float2(s, q);
            rg.sync();
            const u32 i = rg.lane & (rg.span - 1u);         // every span of lanes adds all the warps' values
            const bool in = i < rg.warps;
            const float2 p = in ? part[parity][rg.first_warp + i] : make_float2(0.f, 0.f);
            const float n = in ? counts[rg.first_warp + i] : 0.f;
            s = lanes_sum(p.x, rg.span);
            mean = s * inv_mine;
            const float off = n > 0.f ? p.x / n - mean : 0.f;
            q = lanes_sum(p.y + n * off * off, rg.span);
        }
        if (a.cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < a.cluster)
                cl.map_shared_rank(&peers[parity][0], threadIdx.x)[rank] = make_float4(s, q, (float)cols, 0.f);
            cl.sync();
            float all = 0.f;
            for (u32 i = 0; i < a.cluster; i++) all += peers[parity][i].x;
            mean = all * inv_cols;
            q = 0.f;
            for (u32 i = 0; i < a.cluster; i++) {
                const float4 p = peers[parity][i];
                const float off = p.x / p.z - mean;
                q += p.y + p.z * off * off;
            }
        }
        const float rstd = 1.f / sqrtf(q * inv_cols + a.eps);
        if (rg.t == 0 && rank == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < NV; k++) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[k][e] = (h[k][e] - mean) * rstd * w[k][e] + b[k][e];
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

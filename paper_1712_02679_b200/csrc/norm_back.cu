// Layer norm, backward: the gradient of h (to the residual, and through dropout to x), and the weight's and bias's
// gradients, which are sums over all rows.
#include "norm.cuh"

#ifndef NBB
#define NBB 1
#endif
namespace adacomp_impl {

// With xhat = (h - mean) rstd and g = dy weight:  dh = rstd (g - mean(g) - xhat mean(g xhat)) + dh_in.
// A thread keeps its columns from row to row, so that dweight = sum dy xhat and dbias = sum dy grow in its registers; a
// CTA leaves one line of each, and norm_back_sum adds the lines in their order.
template <u32 TYPE, bool ALIGNED, int NV, bool DROP>
__global__ void __launch_bounds__(kNormThreads, NBB) norm_backward(const NormArgs a)
{
    __shared__ float part[2][kNormThreads / 32][2];
    __shared__ float2 peers[2][8];
    __shared__ float merge[NV == 1 ? kNormThreads * 8 : 1];
    const RowGroup rg(a.tpr);
    const u32 rank = a.cluster > 1 ? cg::this_cluster().block_rank() : 0u;
    if (a.cluster > 1) cg::this_cluster().sync();      // every CTA of the cluster runs before its memory is written
    const u32 c0 = rank * a.slice, cols = min(a.slice, a.cols - c0);
    const u32 set = blockIdx.x / a.cluster;
    const u64 step = (u64)a.partials * a.groups;
    u64 row = (u64)set * a.groups + rg.g;
    Raw<TYPE, ALIGNED> ry[NV], rh[NV], ri[NV];
    clear(ry);
    clear(rh);
    clear(ri);
    float next_mean = 0.f, next_rstd = 0.f;
    auto fetch_row = [&](u64 r) {
        const u32 end = r < a.rows ? cols : 0u;
        if (r < a.rows) next_mean = a.mean[r], next_rstd = a.rstd[r];
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const u32 c = block_column<NV>(k, rg.t);
            fetch<TYPE, ALIGNED>(ry[k], a.dy, r * a.cols + c0, c, end);
            fetch<TYPE, ALIGNED>(rh[k], a.x, r * a.cols + c0, c, end);
            if (a.dh_in) fetch<TYPE, ALIGNED>(ri[k], a.dh_in, r * a.cols + c0, c, end);
        }
    };
    fetch_row(row);
    const void *wp = a.weight ? static_cast<const unsigned char *>(a.weight) + (u64)c0 * type_size(a.param_type) : nullptr;
    float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
    for (int k = 0; k < NV; k++) {
        load_param(wp, a.param_type, block_column<NV>(k, rg.t), cols, 1.f, w[k]);
#pragma unroll
        for (int e = 0; e < 8; e++) dw[k][e] = db[k][e] = 0.f;
    }
    Drop d;
    if constexpr (DROP) d = drop_begin(a.drop);
    const float inv_cols = 1.f / (float)a.cols;
    u32 parity = 0;
#pragma unroll 1
    for (; row < a.rows; row += step, parity ^= 1u) {
        const u64 at = row * a.cols + c0;
        float g[NV][8], xh[NV][8];
        const float mean = next_mean, rstd = next_rstd;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            unpack<TYPE, ALIGNED>(ry[k], at, g[k]);
            unpack<TYPE, ALIGNED>(rh[k], at, xh[k]);
            if constexpr (!ALIGNED) {           // (blocks of an ALIGNED row are whole or hold zeros)
                mask_from(g[k], block_column<NV>(k, rg.t), cols, 0.f);
                mask_from(xh[k], block_column<NV>(k, rg.t), cols, 0.f);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {       // (beyond the row's end g is 0, so that xhat does not matter)
                xh[k][e] = (xh[k][e] - mean) * rstd;
                dw[k][e] = fmaf(g[k][e], xh[k][e], dw[k][e]);
                db[k][e] += g[k][e];
                g[k][e] *= w[k][e];
                s1 += g[k][e];
                s2 = fmaf(g[k][e], xh[k][e], s2);
            }
        }
        float in[NV][8];
        if (a.dh_in) {
#pragma unroll
            for (int k = 0; k < NV; k++) unpack<TYPE, ALIGNED>(ri[k], at, in[k]);
        }
        fetch_row(row + step);          // the next row is on its way while this one is worked on
        float v = warp_two_sums(s1, s2, rg.lane);
        if (rg.warps > 1) {
            if ((rg.lane & 15u) == 0) part[parity][rg.first_warp + rg.warp][rg.lane >> 4] = v;
            rg.sync();
            const u32 i = rg.lane & 15u;
            v = half_sum(i < rg.warps ? part[parity][rg.first_warp + i][rg.lane >> 4] : 0.f);
        }
        s1 = from_lane(v, 0);
        s2 = from_lane(v, 16);
        if (a.cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < a.cluster) cl.map_shared_rank(&peers[parity][0], threadIdx.x)[rank] = make_float2(s1, s2);
            cl.sync();
            s1 = s2 = 0.f;
            for (u32 i = 0; i < a.cluster; i++) {
                s1 += peers[parity][i].x;
                s2 += peers[parity][i].y;
            }
        }
        s1 *= inv_cols;
        s2 *= inv_cols;
#pragma unroll
        for (int k = 0; k < NV; k++) {
#pragma unroll
            for (int e = 0; e < 8; e++) g[k][e] = fmaf(-xh[k][e], s2, g[k][e] - s1);
            if (a.dh_in) {
#pragma unroll
                for (int e = 0; e < 8; e++) g[k][e] = fmaf(g[k][e], rstd, in[k][e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) g[k][e] *= rstd;
            }
            if (a.dresidual) store_block<TYPE, ALIGNED>(a.dresidual, at, block_column<NV>(k, rg.t), cols, g[k]);
        }
        if constexpr (DROP) {
            u32 rows[NV], groups[NV], bits[NV][4];
#pragma unroll
            for (int k = 0; k < NV; k++) rows[k] = (u32)row, groups[k] = (c0 + block_column<NV>(k, rg.t)) >> 3;
            drop_words<NV>(d, rows, groups, bits);
#pragma unroll
            for (int k = 0; k < NV; k++) drop_apply(d, bits[k], g[k]);
        }
        if (a.dx) {
#pragma unroll
            for (int k = 0; k < NV; k++) store_block<TYPE, ALIGNED>(a.dx, at, block_column<NV>(k, rg.t), cols, g[k]);
        }
    }
    after_kernel_may_start();
    if (!a.partial) return;
    float *out = a.partial;
    const u64 line = (u64)set * 2 * a.cols + c0;
#pragma unroll
    for (int which = 0; which < 2; which++) {
        float(&acc)[NV][8] = which ? db : dw;
        if (NV == 1 && a.groups > 1) {          // rows of the CTA's groups, added in their order
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; e++) merge[e * kNormThreads + threadIdx.x] = acc[0][e];
            __syncthreads();
            if (rg.g == 0) {
                for (u32 g = 1; g < a.groups; g++)
#pragma unroll
                    for (int e = 0; e < 8; e++) acc[0][e] += merge[e * kNormThreads + g * rg.tpr + rg.t];
            }
        }
        if (rg.g == 0) {
#pragma unroll
            for (int k = 0; k < NV; k++)
                store_block<ADACOMP_TYPE_F32, ALIGNED>(out, line + (u64)which * a.cols, block_column<NV>(k, rg.t), cols, acc[k]);
        }
    }
}

constexpr int kSumWarps = 32;

// dweight (blockIdx.y = 0) and dbias: 32 columns per CTA, the CTAs' lines in a fixed order.
__global__ void __launch_bounds__(32 * kSumWarps) norm_back_sum(const float *partial, u32 partials, u32 cols, void *dweight,
                                                               void *dbias, u32 param_type)
{
    __shared__ float sums[kSumWarps][33];
    void *out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const u32 lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, c = blockIdx.x * 32u + lane;
    wait_for_kernel_before();
    float s = 0.f;
    if (c < cols) {
        const float *p = partial + (u64)blockIdx.y * cols + c;
#pragma unroll 10
        for (u32 i = warp; i < partials; i += kSumWarps) s += p[(u64)i * 2 * cols];
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || c >= cols) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kSumWarps; i++) s += sums[i][lane];
    if (param_type == ADACOMP_TYPE_F32) store1<ADACOMP_TYPE_F32>(out, c, s);
    else if (param_type == ADACOMP_TYPE_BF16) store1<ADACOMP_TYPE_BF16>(out, c, s);
    else store1<ADACOMP_TYPE_F16>(out, c, s);
}

template <u32 TYPE, bool ALIGNED, int NV> static void launch_drop(const NormArgs &a, cudaStream_t st)
{
    if (a.drop.threshold) launch_norm_kernel(norm_backward<TYPE, ALIGNED, NV, true>, a, a.partials, st);
    else launch_norm_kernel(norm_backward<TYPE, ALIGNED, NV, false>, a, a.partials, st);
}

template <u32 TYPE> static void launch_type(const NormArgs &a, cudaStream_t st)
{
    const bool two = a.per == 2u;
    if (a.cols % 8u == 0) two ? launch_drop<TYPE, true, 2>(a, st) : launch_drop<TYPE, true, 1>(a, st);
    else two ? launch_drop<TYPE, false, 2>(a, st) : launch_drop<TYPE, false, 1>(a, st);
}

int launch_norm_back(NormArgs &a, u32 type, cudaStream_t st)
{
    norm_split(a);
    if (!a.dweight && !a.dbias) a.partial = nullptr;
    if (a.rows) {
        if (type == ADACOMP_TYPE_F32) launch_type<ADACOMP_TYPE_F32>(a, st);
        else if (type == ADACOMP_TYPE_BF16) launch_type<ADACOMP_TYPE_BF16>(a, st);
        else launch_type<ADACOMP_TYPE_F16>(a, st);
    }
    if (a.partial)
        launch_after(norm_back_sum, dim3((a.cols + 31u) / 32u, 2), 32 * kSumWarps, st, (const float *)a.partial,
                     a.rows ? a.partials : 0u, a.cols, a.dweight, a.dbias, a.param_type);
    return launched();
}

}  // namespace adacomp_impl

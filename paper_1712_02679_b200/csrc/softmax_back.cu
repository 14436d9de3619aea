// The biased softmax's backward pass: the scores' gradient and the bias table's.
#include "softmax.cuh"

namespace adacomp_impl {

// P is formed again from the scores and the row's logarithm of the sum, dp = dropout'(dprobs), D = sum_j P dp, and
// ds = P (dp - D).  The table's gradient adds ds by distance: within `reach` into a line of shared memory that belongs to
// the row's threads (a row meets each distance once, and two rows are a meeting apart, so no addition needs to be atomic
// and their order is fixed), beyond it into a register per side.  A group's sums leave by bucket, and softmax_back_sum
// adds the groups' in their order.
template <u32 TYPE, bool WIDE, int NV, bool DROP>
__global__ void __launch_bounds__(kSoftThreads) softmax_backward(const SoftmaxArgs a)
{
    extern __shared__ float tables[];
    __shared__ float part[2][kSoftThreads / 32];
    __shared__ float2 ends[kSoftThreads / 32];
    __shared__ float peers[2][8];
    const RowGroup rg(a.tpr);
    const SoftmaxRows rows(a, rg);
    if (!rows.any) return;
    if (a.cluster > 1) cg::this_cluster().sync();      // every CTA of the cluster runs before its memory is written
    const int reach = (int)a.reach;
    const u32 floats = table_floats(a.reach);
    float *bias = tables + rg.g * 2 * floats, *sums = bias + floats;
    build_table(a, rg, rows.head, bias);
    for (u32 i = rg.t; i < floats; i += rg.tpr) sums[i] = 0.f;
    rg.sync();
    Drop d;
    if constexpr (DROP) d = drop_begin(a.drop);
    const u32 first_warp = rg.g * rg.warps;
    float before = 0.f, behind = 0.f;        // distances <= -reach, >= reach
    u32 parity = 0;
    auto row_sum = [&](float v) -> float {      // over the row's threads; all of them take part
        v = warp_sum(v);
        if (rg.warps > 1) {
            if (rg.lane == 0) part[parity][first_warp + rg.warp] = v;
            rg.sync();
            v = warp_sum(rg.lane < rg.warps ? part[parity][first_warp + rg.lane] : 0.f);
        }
        if (a.cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x < a.cluster) cl.map_shared_rank(&peers[parity][0], threadIdx.x)[rows.rank] = v;
            cl.sync();
            v = 0.f;
            for (u32 j = 0; j < a.cluster; j++) v += peers[parity][j];
        }
        parity ^= 1u;
        return v;
    };
    for (u32 i = rows.i0; i < rows.i1; i++) {
        const u64 row = (u64)rows.bh * a.q_len + i, at = row * a.ld + rows.c0;
        const float lse = a.lse[row];
        const u32 end = lse == -INFINITY ? 0u : rows.end(a, i);
        const int d0 = (int)rows.c0 - ((int)i + a.q_offset);
        // A sum's logarithm does not show beside a statistic this large (ulp 2^-9 and up): P is then normalised again.
        // (A property of the row, so that all its threads meet in row_sum.)
        const bool huge = lse != -INFINITY && fabsf(lse) > 16384.f, far = far_out(lse);
        const float lse2 = lse * kLog2e;
        float p[NV][8], g[NV][8];
        float dot = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            load_block<TYPE, WIDE>(a.scores, at, k, rg.t, rg.tpr, end, 0.f, p[k]);
            load_block<TYPE, WIDE>(a.dprobs, at, k, rg.t, rg.tpr, end, 0.f, g[k]);
        }
#pragma unroll
        for (int k = 0; k < NV; k++) {
            to_logits<WIDE>(p[k], bias, reach, a.scale, d0, k, rg.t, rg.tpr, end);
            if constexpr (DROP) {
                u32 bits[4];
                drop_words<WIDE>(d, (u32)row, rows.c0 >> 3, k, rg.t, rg.tpr, bits);
                drop_apply(d, bits, g[k]);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                p[k][e] = column<WIDE>(k, e, rg.t, rg.tpr) < end ? exp_about(p[k][e], lse, lse2, far) : 0.f;
                dot = fmaf(p[k][e], g[k][e], dot);
            }
        }
        if (huge) {
            float total = 0.f;
#pragma unroll
            for (int k = 0; k < NV; k++)
#pragma unroll
                for (int e = 0; e < 8; e++) total += p[k][e];
            total = row_sum(total);
            const float f = total == 0.f ? 0.f : 1.f / total;
            dot *= f;
#pragma unroll
            for (int k = 0; k < NV; k++)
#pragma unroll
                for (int e = 0; e < 8; e++) p[k][e] *= f;
        }
        dot = row_sum(dot);
#pragma unroll
        for (int k = 0; k < NV; k++) {
#pragma unroll
            for (int e = 0; e < 8; e++) p[k][e] *= g[k][e] - dot;
            if (a.partial) {
                if constexpr (WIDE) {
                    const u32 c = column<true>(k, 0, rg.t, rg.tpr);
                    const int dist = d0 + (int)c;
                    if (c < end) {
                        if (dist >= reach) {
#pragma unroll
                            for (int e = 0; e < 8; e++) behind += p[k][e];
                        } else if (dist + 7 <= -reach) {
#pragma unroll
                            for (int e = 0; e < 8; e++) before += p[k][e];
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; e++) {
                                if (dist + e >= reach) behind += p[k][e];
                                else if (dist + e <= -reach) before += p[k][e];
                                else sums[padded(dist + e + reach)] += p[k][e];
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const u32 c = column<false>(k, e, rg.t, rg.tpr);
                        const int dist = d0 + (int)c;
                        if (c < end) {
                            if (dist >= reach) behind += p[k][e];
                            else if (dist <= -reach) before += p[k][e];
                            else sums[padded(dist + reach)] += p[k][e];
                        }
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e++) p[k][e] *= a.scale;
            store_block<TYPE, WIDE>(a.dscores, at, k, rg.t, rg.tpr, rows.cols, p[k]);
        }
        if (rg.warps == 1) __syncwarp();         // the next row's additions follow this one's
    }
    if (!a.partial) return;
    before = warp_sum(before);
    behind = warp_sum(behind);
    if (rg.lane == 0) ends[first_warp + rg.warp] = make_float2(before, behind);
    rg.sync();
    before = behind = 0.f;
    for (u32 w = 0; w < rg.warps; w++) {
        before += ends[first_warp + w].x;
        behind += ends[first_warp + w].y;
    }
    float *out = a.partial + (((u64)rows.bh * a.chunks + rows.i0 / a.chunk_rows) * a.cluster + rows.rank) * a.buckets;
    for (u32 b = rg.t; b < a.buckets; b += rg.tpr) {
        const bool ahead = b >= a.side;          // buckets of keys behind the query's position
        const u32 k = ahead ? b - a.side : b;
        const bool last = k + 1 == a.side;
        // distances first[k] .. first[k + 1] - 1 of this side; those from reach on are in the register sums
        const int from = a.first[k], to = last ? reach : (int)a.first[k + 1];
        float s = 0.f;
        for (int n = ahead && from == 0 ? 1 : from; n < to; n++) s += sums[padded(ahead ? reach + n : reach - n)];
        if (last) s += ahead ? behind : before;
        if (b == 0 && !a.both) {                 // one-sided: every key behind the query's position counts as distance 0
            for (int n = 1; n < reach; n++) s += sums[padded(reach + n)];
            s += behind;
        }
        out[b] = s;
    }
}

constexpr int kTableSumWarps = 8;

// dtable[b][head]: the groups' sums of that head over the batch, in their order.
__global__ void __launch_bounds__(32 * kTableSumWarps)
softmax_back_sum(const float *partial, float *dtable, u32 batch, u32 heads, u32 per, u32 buckets)
{
    __shared__ float sums[kTableSumWarps][33];
    const u32 head = blockIdx.x, lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, b = blockIdx.y * 32u + lane;
    float s = 0.f;
    if (b < buckets)
        for (u64 j = warp; j < (u64)batch * per; j += kTableSumWarps) {
            const u64 bh = (j / per) * heads + head;
            s += partial[(bh * per + j % per) * buckets + b];
        }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || b >= buckets) return;
    s = 0.f;
    for (int w = 0; w < kTableSumWarps; w++) s += sums[w][lane];
    dtable[(u64)b * heads + head] = s;
}

template <u32 TYPE, bool WIDE, int NV> static void launch_drop(const SoftmaxArgs &a, cudaStream_t st)
{
    const size_t smem = 2 * (size_t)a.groups * table_floats(a.reach) * sizeof(float);
    if (a.drop.threshold) launch_softmax_kernel(softmax_backward<TYPE, WIDE, NV, true>, a, smem, st);
    else launch_softmax_kernel(softmax_backward<TYPE, WIDE, NV, false>, a, smem, st);
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

int launch_softmax_back(SoftmaxArgs &a, u32 type, cudaStream_t st)
{
    softmax_split(a);
    if (!a.table || !a.dtable) a.partial = nullptr;
    const bool any = (u64)a.batch * a.heads * a.q_len != 0;
    if (any) {
        if (type == ADACOMP_TYPE_F32) launch_type<ADACOMP_TYPE_F32>(a, st);
        else if (type == ADACOMP_TYPE_BF16) launch_type<ADACOMP_TYPE_BF16>(a, st);
        else launch_type<ADACOMP_TYPE_F16>(a, st);
    }
    if (a.table && a.dtable && a.heads)
        softmax_back_sum<<<dim3(a.heads, (a.buckets + 31u) / 32u), 32 * kTableSumWarps, 0, st>>>(
            a.partial, a.dtable, any ? a.batch : 0u, a.heads, a.chunks * a.cluster, a.buckets);
    return launched();
}

}  // namespace adacomp_impl

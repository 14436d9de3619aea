// Dropout from a counter-based generator: y = keep ? x * factor : 0, the mask recomputed wherever it is needed and never
// stored.  Its backward pass is the same map applied to dy.
//
// Bound by memory, x in and y out, with the generator close behind: ten rounds are 20 products of 32 bits and as many
// exclusive ors for eight elements, which is why an element takes 16 bits of them and not 32 (with 32 the 16-bit types would
// be bound by the generator), and why the blocks of a thread go through the rounds together and share the key's additions
// (47 -> 42 us).  16384 x 4096 bf16: 41.7 us, 6.43 TB/s, 98 % of the measured copy rate; rows that start anywhere, 24336 x
// 313 binary16: 13 us (0.36 of it), bound by the shifting (19 us with a warp per 256 columns of a row: most lanes of a short
// row's second warp were idle).
#include "block.h"

namespace adacomp_impl {

constexpr int kDropThreads = 256;
constexpr int kDropPer = 4;         // blocks of eight per thread, rows on a vector boundary
constexpr int kDropAnyPer = 2;      // the same for any rows

// Rows that start on a vector boundary: the tensor is one line of groups of eight.
template <u32 TYPE>
__global__ void __launch_bounds__(kDropThreads)
dropout_wide(const void *x, void *y, u32 row0, u32 n_groups, FastDiv per_row, DropArgs args)
{
    const Drop d = drop_begin(args);
    const u32 g0 = blockIdx.x * (kDropThreads * kDropPer) + threadIdx.x;
    const u64 at0 = (u64)row0 * per_row.d * 8u;
    Vec8<TYPE> r[kDropPer];
#pragma unroll
    for (int i = 0; i < kDropPer; i++) {
        const u32 g = g0 + i * kDropThreads;
        if (g < n_groups) r[i] = load8<TYPE>(x, at0 + (u64)g * 8u);
    }
    u32 row[kDropPer], group[kDropPer], w[kDropPer][4];
#pragma unroll
    for (int i = 0; i < kDropPer; i++) {
        const u32 g = g0 + i * kDropThreads, q = fast_div(g, per_row);
        row[i] = row0 + q;
        group[i] = g - q * per_row.d;
    }
    drop_words<kDropPer>(d, row, group, w);
#pragma unroll
    for (int i = 0; i < kDropPer; i++) {
        const u32 g = g0 + i * kDropThreads;
        float v[8];
        widen8<TYPE>(r[i], v);
        drop_apply(d, w[i], v);
        if (g < n_groups) store8<TYPE>(y, at0 + (u64)g * 8u, narrow8<TYPE>(v));
    }
}

// Any row length: the tensor is one line of blocks of up to eight columns, row after row; a warp takes 32 of them at a time.
template <u32 TYPE>
__global__ void __launch_bounds__(kDropThreads)
dropout_any(const void *x, void *y, u32 row0, u32 n_blocks, u32 cols, FastDiv per_row, DropArgs args)
{
    const Drop d = drop_begin(args);
    const u32 b0 = blockIdx.x * (kDropThreads * kDropAnyPer) + threadIdx.x;
    Raw<TYPE, false> raw[kDropAnyPer];
    u32 row[kDropAnyPer], group[kDropAnyPer], w[kDropAnyPer][4];
#pragma unroll
    for (int i = 0; i < kDropAnyPer; i++) {
        const u32 b = b0 + i * kDropThreads, r = fast_div(b, per_row);
        row[i] = row0 + r;
        group[i] = b - r * per_row.d;
        if (b < n_blocks) fetch<TYPE, false>(raw[i], x, (u64)row[i] * cols, group[i] * 8u, cols);
    }
    drop_words<kDropAnyPer>(d, row, group, w);
#pragma unroll
    for (int i = 0; i < kDropAnyPer; i++) {
        const bool there = b0 + i * kDropThreads < n_blocks;
        const u64 at = (u64)row[i] * cols;
        float v[8];
        unpack<TYPE, false>(raw[i], at, v);
        drop_apply(d, w[i], v);
        store_block<TYPE, false>(y, at, there ? group[i] * 8u : cols, cols, v);
    }
}

template <u32 TYPE>
static void launch_type(const void *x, void *y, u64 rows, u32 cols, const DropArgs &drop, cudaStream_t st)
{
    const bool wide = cols % 8u == 0;
    const u32 per_row = (cols + 7u) / 8u;
    const FastDiv f = make_fastdiv(per_row);
    const u64 slice = 0x7fffffffu / per_row;         // rows a launch covers: items are numbered in 31 bits
    for (u64 row0 = 0; row0 < rows; row0 += slice) {
        const u32 items = (u32)((rows - row0 < slice ? rows - row0 : slice) * per_row);
        if (wide) {
            const u32 per_cta = kDropThreads * kDropPer;
            dropout_wide<TYPE><<<(items - 1) / per_cta + 1, kDropThreads, 0, st>>>(x, y, (u32)row0, items, f, drop);
        } else {
            const u32 per_cta = kDropThreads * kDropAnyPer;
            dropout_any<TYPE><<<(items - 1) / per_cta + 1, kDropThreads, 0, st>>>(x, y, (u32)row0, items, cols, f, drop);
        }
    }
}

int launch_dropout(const void *x, void *y, u64 rows, u32 cols, u32 type, const DropArgs &drop, cudaStream_t st)
{
    if (drop.threshold == 0) {          // nothing is dropped
        if (x == y) return ADACOMP_OK;
        return cudaMemcpyAsync(y, x, rows * cols * type_size(type), cudaMemcpyDeviceToDevice, st) == cudaSuccess
                   ? ADACOMP_OK : ADACOMP_ERR_CUDA;
    }
    if (type == ADACOMP_TYPE_F32) launch_type<ADACOMP_TYPE_F32>(x, y, rows, cols, drop, st);
    else if (type == ADACOMP_TYPE_BF16) launch_type<ADACOMP_TYPE_BF16>(x, y, rows, cols, drop, st);
    else launch_type<ADACOMP_TYPE_F16>(x, y, rows, cols, drop, st);
    return launched();
}

}  // namespace adacomp_impl

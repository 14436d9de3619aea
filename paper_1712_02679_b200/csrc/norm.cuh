// What the forward and backward kernels of layer norm share.
#pragma once

#include "block.h"

namespace adacomp_impl {

namespace cg = cooperative_groups;

constexpr int kNormThreads = 512;            // most threads of a CTA
constexpr int kNormMany = 256;               // threads of a CTA where there are many rows
constexpr u32 kNormBusy = 8;                 // warps per SM that make many rows of them

// Rows that are copied ahead (see Ring): three arrays of binary32 rows of 16 columns per thread leave no room for a second
// row where a CTA has all 512 threads.
__host__ __device__ constexpr int norm_stages(int nv, int threads, u32 type)
{
    return nv == 2 && threads == kNormThreads && type == ADACOMP_TYPE_F32 ? 1 : 2;
}

template <typename K> inline void launch_norm_kernel(K kernel, const NormArgs &a, size_t smem, cudaStream_t st)
{
    if (smem > 16 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.sets * a.cluster);
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

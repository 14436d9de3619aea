// What the forward and backward kernels of layer norm share.
#pragma once

#include "block.h"

namespace adacomp_impl {

namespace cg = cooperative_groups;

constexpr int kNormThreads = 512;            // most threads of a CTA

// Launches `kernel` over `rows_at_once` sets of rows, `cluster` CTAs to a row.
template <typename K> inline void launch_norm_kernel(K kernel, const NormArgs &a, u32 sets, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sets * a.cluster);
    cfg.blockDim = dim3(a.tpr * a.groups);
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

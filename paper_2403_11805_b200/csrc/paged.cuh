// What the calls on the resident cache (decode.cu, evict.cu) share: argument checks, clustered launches, divisions.
#pragma once

#include "llms_internal.cuh"

namespace llms {

// Shape checks of the calls that use a paged cache: a pool the codec could take, with head_dim up to 256, and a batch.
int check_paged(const llms_kv_desc *d, int n_seqs, int max_len);

// launch_dependent with clusters of `cluster` CTAs; grid.x is a multiple of that.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_dependent_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st,
                                            Args &&...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Division of 0 .. 2^31 - 1 by a number known at launch: with l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1 the quotient
// is (high word of m * x, plus x) >> l (the multiply-and-shift method of Granlund and Montgomery); three instructions
// where a division by a variable takes some twenty.
struct Divisor {
    uint32_t mul, shift;
    Divisor() = default;
    explicit Divisor(uint32_t d) : mul(0), shift(0)
    {
        while (shift < 31 && (1u << shift) < d) ++shift;
        mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - d)) / d + 1);
    }
#ifdef __CUDACC__
    __device__ __forceinline__ int operator()(int x) const { return (int)((__umulhi(mul, (uint32_t)x) + (uint32_t)x) >> shift); }
#endif
};

}  // namespace llms

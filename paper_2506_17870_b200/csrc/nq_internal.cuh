// Host-side helpers shared by the translation units of the library (not part of the C boundary).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/nq.h"

namespace nq {

// Programmatic dependent launch: a kernel started with launch_chained() may begin while the one before it in the stream
// still runs, provided that one called start_next(); it must call wait_previous() before it touches global memory
// (which waits until everything before it in the stream is complete and visible).  What overlaps is the launch itself and a
// block's set-up: for a call of a few microseconds that is most of its time.  Such kernels read global memory by ordinary
// loads, not through __ldg: the compiler may move a load of memory that never changes across the wait.
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... P, typename... A>
int launch_chained(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t stream, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(block, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return NQ_ERR_CUDA;
    }
    return NQ_OK;
}

// SM count of the current device (cached per device index).
int sm_count();

// Device-side record of a bounded wait that gave up: word 0 = non-zero code of the wait, word 1 = detail.
// Defined in nq_runtime.cu; kernels get its address through status_word().
unsigned int* status_word();

// The driver's cuTensorMapEncodeTiled, null where it has none.  (As the two above: safe to call from several threads.)
void* tensor_map_encoder();

// The paper's 64-bit packed words -> sliced layout (kernel beside the codec, whose slice cutter it uses).
int word64_to_sliced_launch(const uint64_t* words, int bits, int64_t rows, int64_t cols, uint8_t* packed, cudaStream_t s);

}  // namespace nq


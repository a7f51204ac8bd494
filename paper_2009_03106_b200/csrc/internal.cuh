// What the translation units of the library share: launch accounting and the tensor-map encoder (defined in dpclip_api.cu).
#pragma once
#include <cuda.h>
#include <string.h>

#include "common.cuh"

namespace dpclip {

int finish_launch();                 // counts a launch; DPCLIP_OK or DPCLIP_ERR_CUDA
bool overlap_allowed();              // DPCLIP_NO_OVERLAP is not set
bool tensor_cores_allowed();         // DPCLIP_FORCE_SIMT is not set
// 2-D bf16 matrix [rows][cols], row stride ld elements (a multiple of 8), base 16-byte aligned; box_cols x box_rows boxes, 128-byte
// swizzle, zeros outside
bool encode_map_bf16(CUtensorMap* map, const void* base, long rows, long cols, long ld, int box_cols, int box_rows);

inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Launch with programmatic serialization (see griddep_wait in common.cuh), right behind a launch of the same call.
template <typename... P, typename... A>
inline int launch_after(void (*kernel)(P...), dim3 grid, int block, size_t smem, cudaStream_t st, const A&... args) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = grid; cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = overlap_allowed() ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) { cudaGetLastError(); return DPCLIP_ERR_CUDA; }
    return finish_launch();
}

}  // namespace dpclip

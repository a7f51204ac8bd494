// Clipped sums of stored per-example gradients: g[j] = sum_i clip[i] G[i][j] (+ noise), for parameters whose gradient an example's
// norm kernel has left in memory (a few hundred numbers an example).
//
// CTA = 32 columns; its warps deal the examples among them with eight loads in flight, the warps' sums are added in order.  The bytes
// are few (128 examples of 512 numbers: 256 KB), so what bounds it is the round trips of the loads, one after the other: 32 warps where eight
// would go round more than once, and beyond 512 examples the CTAs of a cluster share them and the first adds up their sums, in order too.
#pragma once
#include <cooperative_groups.h>

#include "philox.cuh"

namespace dpclip {

constexpr int STORED_PER_CTA = 512, STORED_MAX_CLUSTER = 8;
struct StoredParams {
    const float* G; long ld; int B, n, cluster;
    const float* clip; float* g;
    float noise_scale; uint32_t k0, k1, s0, s1;
};

template <int WARPS, bool CLUSTER>
__global__ void __launch_bounds__(32 * WARPS)
stored_grad_kernel(const __grid_constant__ StoredParams p) {
    constexpr int UNR = 8;
    __shared__ float part[WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int block = CLUSTER ? (int)blockIdx.x / p.cluster : (int)blockIdx.x, rank = CLUSTER ? (int)blockIdx.x - block * p.cluster : 0;
    const int c = block * 32 + lane, step = CLUSTER ? p.cluster * WARPS : WARPS;
    griddep_wait();
    griddep_launch_dependents();
    float acc = 0.f;
    if (c < p.n) {
        for (int i = rank * WARPS + warp; i < p.B; i += step * UNR) {
            float v[UNR], f[UNR];
#pragma unroll
            for (int k = 0; k < UNR; ++k) {
                const long e = (long)i + (long)k * step;
                v[k] = e < p.B ? p.G[(size_t)e * p.ld + c] : 0.f;
                f[k] = e < p.B ? (p.clip ? p.clip[e] : 1.f) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < UNR; ++k) acc = fmaf(f[k], v[k], acc);
        }
    }
    part[warp][lane] = acc;
    __syncthreads();
    if (warp == 0) {
#pragma unroll
        for (int w = 1; w < WARPS; ++w) acc += part[w][lane];
        if (CLUSTER) part[0][lane] = acc;
    }
    if (CLUSTER) {
        const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
        cluster.sync();
        if (rank == 0 && warp == 0)
            for (int r = 1; r < p.cluster; ++r) acc += *cluster.map_shared_rank(&part[0][lane], r);
        cluster.sync();                  // the others' shared memory stays until the first has read it
    }
    if (rank != 0 || warp != 0 || c >= p.n) return;
    if (p.noise_scale > 0.f) {
        float z[4];
        normals_at((size_t)(c & ~3), p.s0, p.s1, p.k0, p.k1, z);
        acc = fmaf(p.noise_scale, (c & 2) ? ((c & 1) ? z[3] : z[2]) : ((c & 1) ? z[1] : z[0]), acc);
    }
    p.g[c] = acc;
}

}  // namespace dpclip

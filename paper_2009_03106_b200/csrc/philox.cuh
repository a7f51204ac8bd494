// Gaussian noise of every kernel that releases a sum: Philox4x32-10 and Box-Muller.
#pragma once
#include "common.cuh"

namespace dpclip {

// ---------------------------------------------------------------------------
// Gaussian noise: Philox4x32-10 counter-based generator + Box-Muller.
// One 128-bit block gives four normals; a thread owns block q = elements
// 4q..4q+3, so the output depends only on (seed, stream_id, element index).
// ---------------------------------------------------------------------------
struct PhiloxBlock { uint32_t v[4]; };

__device__ __forceinline__ PhiloxBlock philox_block(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3,
                                                    uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint32_t hi0 = __umulhi(0xD2511F53u, c0), lo0 = 0xD2511F53u * c0;
        const uint32_t hi1 = __umulhi(0xCD9E8D57u, c2), lo1 = 0xCD9E8D57u * c2;
        c0 = hi1 ^ c1 ^ k0;
        c1 = lo1;
        c2 = hi0 ^ c3 ^ k1;
        c3 = lo0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    PhiloxBlock b;
    b.v[0] = c0; b.v[1] = c1; b.v[2] = c2; b.v[3] = c3;
    return b;
}

__device__ __forceinline__ float bits_to_u01(uint32_t x) {          // (0, 1]
    return __fmaf_rn(__uint2float_rn(x), 2.3283064365386963e-10f, 1.1641532182693481e-10f);
}

// Box-Muller pair from two 32-bit draws.  The generator costs more issue slots than anything else in the
// small fused steps, so it uses the hardware approximations where their error stays well inside the
// 1e-5 absolute budget of a standard normal (every kernel shares this one function, so all launch
// forms give the same bits):
//   ln u1 : lg2.approx (relative error 2^-22 below 1/2, absolute 2^-22 above); within 2^-7 of 1, where an
//           absolute error would dominate the small radius, the series -w - w^2/2 - w^3/3 - w^4/4, w = 1 - u1
//   sqrt  : sqrt.approx (about 1 ulp)
//   angle : 2 pi (u2 - 1/2) lies in (-pi, pi], where sin/cos.approx are good to 2^-20.9 absolute;
//           cos(2 pi u2) = -cos(2 pi (u2 - 1/2)), likewise for sin
__device__ __forceinline__ void box_muller(uint32_t xa, uint32_t xb, float& n0, float& n1) {
    const float u1 = bits_to_u01(xa), u2 = bits_to_u01(xb);
    float l2;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(l2) : "f"(u1));
    const float w = 1.0f - u1;                                  // exact for u1 >= 1/2
    const float series = -w * fmaf(w, fmaf(w, fmaf(w, 0.25f, 0.333333343f), 0.5f), 1.0f);
    const float ln = w < 0.0078125f ? series : l2 * 0.693147182f;
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(-2.0f * ln));
    const float th = 6.28318548f * (u2 - 0.5f);
    float s, c;
    asm("sin.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(th));
    asm("cos.approx.ftz.f32 %0, %1;" : "=f"(c) : "f"(th));
    n0 = -r * c;
    n1 = -r * s;
}

__device__ __forceinline__ void normals_block(size_t q, uint32_t s0, uint32_t s1, uint32_t k0, uint32_t k1, float (&z)[4]) {
    const PhiloxBlock b = philox_block((uint32_t)q, (uint32_t)(q >> 32), s0, s1, k0, k1);
    box_muller(b.v[0], b.v[1], z[0], z[1]);
    box_muller(b.v[2], b.v[3], z[2], z[3]);
}
// element u of the four that start o elements into e[0..3], y[0..3]
__device__ __forceinline__ float shifted(const float (&e)[4], const float (&y)[4], int u, int o) {
    const float a1 = u + 1 < 4 ? e[(u + 1) & 3] : y[(u + 1) & 3], a2 = u + 2 < 4 ? e[(u + 2) & 3] : y[(u + 2) & 3],
                a3 = u + 3 < 4 ? e[(u + 3) & 3] : y[(u + 3) & 3];
    return o == 0 ? e[u] : o == 1 ? a1 : o == 2 ? a2 : a3;
}
// Elements j .. j + 3 of noise stream (s0, s1): one Philox block when j is a multiple of four, else parts of two.
__device__ __forceinline__ void normals_at(size_t j, uint32_t s0, uint32_t s1, uint32_t k0, uint32_t k1, float (&z)[4]) {
    const int o = (int)(j & 3);
    normals_block(j >> 2, s0, s1, k0, k1, z);
    if (o) {
        float y[4];
        normals_block((j >> 2) + 1, s0, s1, k0, k1, y);
        const float e[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
        for (int u = 0; u < 4; ++u) z[u] = shifted(e, y, u, o);
    }
}

}  // namespace dpclip

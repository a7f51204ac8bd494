// Gated feed-forward block: zg = X Wg^T + bg, zu = X Wu^T + bu, h = act(zg) (.) zu, with the weight [2F][K] of both projections (gate
// rows, then up rows); backward: dzg = dh (.) zu (.) act'(zg), dzu = dh (.) act(zg), dx = [dzg dzu] W.
//
//   gated_tc_kernel      bf16 products on CTA pairs (tcgen05, cta_group::2).  Forward: a pair's tile is 256 rows by HN gate and the HN
//                        up columns that go with them -- CTA 0 loads the gate rows of W, CTA 1 the up rows, and the accumulator of both
//                        lies side by side in each CTA's tensor memory, so that activation and product are the epilogue.  Backward: the
//                        plain product dZ W, with W read as it lies (its contraction index is the row: MN-major operand).
//   gated_simt_kernel    the same two products on the fp32 ALUs: fp32 inputs, and rows that TMA cannot address.
//   gated_few_kernel     up to eight rows of X: the weights are streamed once, a warp takes one gate row and its up row.
//   gated_reduce_kernel  adds up the partial products of a split contraction, in order, and ends as the products' epilogue does.
//   gated_signal_kernel  dh, z -> dz: five passes over M x F numbers, bound by memory.
//
// Pre-activations and products are fp32; h, z, dz and dx are rounded once.  The backward pass starts from the stored z and multiplies W with
// the stored dz, so in bf16 both carry that type's rounding.
#pragma once
#include "internal.cuh"
#include "tc_common.cuh"

namespace dpclip {

// ------------------------------------------------------------------------------------------------ activations
// EXACT: expf and one step of Newton's iteration r + r (1 - d r) on the hardware's reciprocal (2^-22 before it), for fp32 results; else the
// fast forms (a few 2^-21), for bf16 ones.  Division proper branches for every element: 1.8 us a tile of 256 x 128 in the fp32 epilogue.  Where d is
// above 2^126 the sigmoid is zero (it is below 1.2e-38, and an infinite d would make the step NaN).
__device__ __forceinline__ float gate_rcp(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
template <bool EXACT> __device__ __forceinline__ float gate_sigmoid(float z) {
    if constexpr (!EXACT) return __fdividef(1.f, 1.f + __expf(-z));
    const float d = 1.f + expf(-z), r = gate_rcp(d);
    return d > 8.5070592e37f ? 0.f : fmaf(r, fmaf(-d, r, 1.f), r);
}
constexpr float kGeluTanh = 0.7978845608028654f, kGeluCube = 0.044715f;       // sqrt(2 / pi)

template <int ACT, bool EXACT> __device__ __forceinline__ float gate_act(float z) {
    if constexpr (ACT == DPCLIP_ACT_SILU) return z * gate_sigmoid<EXACT>(z);
    else if constexpr (ACT == DPCLIP_ACT_RELU) return z < 0.f ? 0.f : z;
    else if constexpr (ACT == DPCLIP_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    else return z * gate_sigmoid<EXACT>(2.f * kGeluTanh * z * fmaf(kGeluCube * z, z, 1.f));     // (1 + tanh u) / 2 = sigmoid(2 u)
}
// the activation and its derivative
template <int ACT, bool EXACT> __device__ __forceinline__ void gate_act_grad(float z, float& a, float& da) {
    if constexpr (ACT == DPCLIP_ACT_SILU) {
        const float p = gate_sigmoid<EXACT>(z);
        a = z * p;
        da = p * fmaf(z, 1.f - p, 1.f);
    } else if constexpr (ACT == DPCLIP_ACT_RELU) {
        a = z < 0.f ? 0.f : z;
        da = z > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == DPCLIP_ACT_GELU) {
        const float c = 0.5f * (1.f + erff(z * 0.70710678118654752f));
        a = z * c;
        const float e = EXACT ? expf(-0.5f * z * z) : __expf(-0.5f * z * z);
        da = fmaf(z * 0.3989422804014327f, e, c);                              // 1 / sqrt(2 pi)
    } else {
        const float p = gate_sigmoid<EXACT>(2.f * kGeluTanh * z * fmaf(kGeluCube * z, z, 1.f));
        a = z * p;
        da = fmaf(a * (1.f - p), 2.f * kGeluTanh * fmaf(3.f * kGeluCube * z, z, 1.f), p);
    }
}
// act(g) (.) u of a pair, for bf16 results: sigmoid(s) = 1 / (1 + 2^(-s log2 e)), each of the two by the hardware's approximation (2^-22).  The
// epilogue of the tensor-core kernel is made of little else (per element two of them and three multiply-adds; one element at a time, with
// __expf and __fdividef, it was 21 instructions and bound the kernel).
__device__ __forceinline__ float gate_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
constexpr float kLog2e = 1.4426950408889634f;
template <int ACT> __device__ __forceinline__ f32x2 gate_pair(f32x2 g, f32x2 u) {
    if constexpr (ACT == DPCLIP_ACT_SILU || ACT == DPCLIP_ACT_GELU_TANH) {
        f32x2 e;
        if constexpr (ACT == DPCLIP_ACT_SILU) e = mul2(g, make_f32x2(-kLog2e, -kLog2e));
        else {
            constexpr float a = -2.f * kGeluTanh * kLog2e, b = a * kGeluCube;
            e = mul2(g, fma2(mul2(g, g), make_f32x2(b, b), make_f32x2(a, a)));
        }
        float x, y;
        split_f32x2(e, x, y);
        split_f32x2(add2(make_f32x2(gate_ex2(x), gate_ex2(y)), make_f32x2(1.f, 1.f)), x, y);
        return mul2(mul2(g, make_f32x2(gate_rcp(x), gate_rcp(y))), u);      // act first: g u may overflow where act(g) is zero
    } else {
        float a, b, c, d;
        split_f32x2(g, a, b);
        split_f32x2(u, c, d);
        return make_f32x2(gate_act<ACT, false>(a) * c, gate_act<ACT, false>(b) * d);
    }
}
// dg = dh u act'(g), du = dh act(g) of a pair, likewise
template <int ACT> __device__ __forceinline__ void gate_pair_grad(f32x2 dh, f32x2 g, f32x2 u, f32x2& dg, f32x2& du) {
    if constexpr (ACT == DPCLIP_ACT_SILU || ACT == DPCLIP_ACT_GELU_TANH) {
        const f32x2 one = make_f32x2(1.f, 1.f);
        f32x2 e, gg;
        if constexpr (ACT == DPCLIP_ACT_SILU) e = mul2(g, make_f32x2(-kLog2e, -kLog2e));
        else {
            constexpr float a = -2.f * kGeluTanh * kLog2e, b = a * kGeluCube;
            gg = mul2(g, g);
            e = mul2(g, fma2(gg, make_f32x2(b, b), make_f32x2(a, a)));
        }
        float x, y;
        split_f32x2(e, x, y);
        split_f32x2(add2(make_f32x2(gate_ex2(x), gate_ex2(y)), one), x, y);
        const f32x2 p = make_f32x2(gate_rcp(x), gate_rcp(y)), a = mul2(g, p);
        f32x2 rest = sub2(one, p);
        if constexpr (ACT == DPCLIP_ACT_GELU_TANH) {
            constexpr float c = 2.f * kGeluTanh, d = 3.f * c * kGeluCube;
            rest = mul2(rest, fma2(gg, make_f32x2(d, d), make_f32x2(c, c)));
        }
        dg = mul2(mul2(dh, u), fma2(a, rest, p));
        du = mul2(dh, a);
    } else {
        float h0, h1, g0, g1, u0, u1, a0, a1, s0, s1;
        split_f32x2(dh, h0, h1); split_f32x2(g, g0, g1); split_f32x2(u, u0, u1);
        gate_act_grad<ACT, false>(g0, a0, s0);
        gate_act_grad<ACT, false>(g1, a1, s1);
        dg = make_f32x2(h0 * u0 * s0, h1 * u1 * s1);
        du = make_f32x2(h0 * a0, h1 * a1);
    }
}
template <bool EXACT, typename F> __device__ __forceinline__ void gate_dispatch(int act, F f) {
    switch (act) {
        case DPCLIP_ACT_SILU: f(std::integral_constant<int, DPCLIP_ACT_SILU>()); break;
        case DPCLIP_ACT_GELU: f(std::integral_constant<int, DPCLIP_ACT_GELU>()); break;
        case DPCLIP_ACT_GELU_TANH: f(std::integral_constant<int, DPCLIP_ACT_GELU_TANH>()); break;
        default: f(std::integral_constant<int, DPCLIP_ACT_RELU>()); break;
    }
}
__device__ __forceinline__ void gate_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void gate_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// ------------------------------------------------------------------------------------------------ dz from dh and z
// fp32 as three bf16 planes (kernels_gated_f32.cuh): the top 8 significant bits, the next 8, the last 8, each cut off, so that they add up to
// the number and nothing overflows.  An infinity or a NaN stays in the first plane.
__device__ __forceinline__ void split3(float x, uint16_t (&t)[3]) {
    const uint32_t h = __float_as_uint(x) & 0xFFFF0000u;
    const float r = (h & 0x7F800000u) == 0x7F800000u ? 0.f : x - __uint_as_float(h);
    const uint32_t m = __float_as_uint(r) & 0xFFFF0000u;
    const float l = r - __uint_as_float(m);
    t[0] = (uint16_t)(h >> 16) | (uint16_t)(x != x ? 0x40 : 0);    // a NaN whose payload lies in the low bits alone must not become an infinity
    t[1] = (uint16_t)(m >> 16);
    t[2] = (uint16_t)(__float_as_uint(l) >> 16);
}
struct GatedSignal {
    const void* dh; long lddh;
    const void* z; long ldz;             // [M][2F]
    void* dz; long lddz;                 // [M][2F], may be z
    __nv_bfloat16* copy; long ldc;       // NULL, or rows of 16-byte multiples for the product: bf16 a copy of dz, fp32 its three planes
    long plane;
    long M; int F, act, per_row, wide;   // per_row: groups of V elements a row of h; wide: threads a row
};
template <typename T> __device__ __forceinline__ void gated_copy_out(const GatedSignal& p, long m, int f, float v) {
    __nv_bfloat16* const to = p.copy + m * p.ldc + f;
    if constexpr (sizeof(T) == 2) *to = __float2bfloat16_rn(v);
    else {
        uint16_t t[3];
        split3(v, t);
#pragma unroll
        for (int j = 0; j < 3; ++j) *reinterpret_cast<uint16_t*>(to + j * p.plane) = t[j];
    }
}
// 256 threads: as many rows side by side as fit, a row's groups along the threads; with few rows a row's groups go to gridDim.y CTAs.
template <typename T, int V>             // V elements a thread: 16 bytes, or one
__global__ void __launch_bounds__(256)
gated_signal_kernel(const __grid_constant__ GatedSignal p) {
    constexpr bool EXACT = sizeof(T) == 4;
    griddep_launch_dependents();
    const int wide = p.wide, tall = 256 / wide, ty = threadIdx.x / wide, tx = threadIdx.x - ty * wide + blockIdx.y * wide, step = gridDim.y * wide;
    if (ty >= tall) return;
    gate_dispatch<EXACT>(p.act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        for (long m = (long)blockIdx.x * tall + ty; m < p.M; m += (long)gridDim.x * tall) {
            const T* const dh = static_cast<const T*>(p.dh) + m * p.lddh;
            const T* const zg = static_cast<const T*>(p.z) + m * p.ldz;
            T* const og = static_cast<T*>(p.dz) + m * p.lddz;
            auto one = [&](float h, float g, float u, float& dg, float& du) {
                float act, slope;
                gate_act_grad<ACT, EXACT>(g, act, slope);
                dg = h * u * slope;
                du = h * act;
            };
            if constexpr (V == 1) {
                // four elements a thread in flight
                for (int f0 = tx; f0 < p.per_row; f0 += 4 * step) {
                    float h[4], g[4], u[4], dg[4], du[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int f = f0 + j * step;
                        const bool there = f < p.per_row;
                        h[j] = there ? to_f32(dh[f]) : 0.f;
                        g[j] = there ? to_f32(zg[f]) : 0.f;
                        u[j] = there ? to_f32(zg[p.F + f]) : 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) one(h[j], g[j], u[j], dg[j], du[j]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int f = f0 + j * step;
                        if (f < p.per_row) {
                            gate_store(og + f, dg[j]); gate_store(og + p.F + f, du[j]);
                            if (p.copy) { gated_copy_out<T>(p, m, f, dg[j]); gated_copy_out<T>(p, m, p.F + f, du[j]); }
                        }
                    }
                }
            } else {
#pragma unroll 2
                for (int c = tx; c < p.per_row; c += step) {
                    const int f = c * V;
                    const uint4 h = *reinterpret_cast<const uint4*>(dh + f), g = *reinterpret_cast<const uint4*>(zg + f),
                                u = *reinterpret_cast<const uint4*>(zg + p.F + f);
                    const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, gw[4] = {g.x, g.y, g.z, g.w}, uw[4] = {u.x, u.y, u.z, u.w};
                    uint32_t a[4], b[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if constexpr (V == 8) {
                            f32x2 dg, du;
                            gate_pair_grad<ACT>(bf16x2_to_f32x2(hw[k]), bf16x2_to_f32x2(gw[k]), bf16x2_to_f32x2(uw[k]), dg, du);
                            a[k] = f32x2_to_bf16x2(dg);
                            b[k] = f32x2_to_bf16x2(du);
                        } else {
                            float x0, y0;
                            one(__uint_as_float(hw[k]), __uint_as_float(gw[k]), __uint_as_float(uw[k]), x0, y0);
                            a[k] = __float_as_uint(x0); b[k] = __float_as_uint(y0);
                        }
                    }
                    *reinterpret_cast<uint4*>(og + f) = make_uint4(a[0], a[1], a[2], a[3]);
                    *reinterpret_cast<uint4*>(og + p.F + f) = make_uint4(b[0], b[1], b[2], b[3]);
                    if constexpr (V == 4) {
                        if (p.copy) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                uint16_t t[4][3];
#pragma unroll
                                for (int k = 0; k < 4; ++k) split3(__uint_as_float(half ? b[k] : a[k]), t[k]);
#pragma unroll
                                for (int j = 0; j < 3; ++j)
                                    *reinterpret_cast<uint2*>(p.copy + j * p.plane + m * p.ldc + half * p.F + f) =
                                        make_uint2(t[0][j] | (uint32_t)t[1][j] << 16, t[2][j] | (uint32_t)t[3][j] << 16);
                            }
                        }
                    }
                }
            }
        }
    });
}

// Rows of any stride and start copied to rows of 16-byte multiples: eight elements a thread, stored at once.  Two matrices a launch.
struct GatedCopy { const __nv_bfloat16* src; long ld; __nv_bfloat16* dst; long ldd, rows; int cols; };
struct GatedCopies { GatedCopy c[2]; long first; };          // first: groups of the first matrix
__global__ void __launch_bounds__(256)
gated_copy_kernel(const __grid_constant__ GatedCopies p, long n) {
    griddep_launch_dependents();
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        const GatedCopy& y = p.c[i >= p.first];
        const uint32_t per = (uint32_t)(y.cols + 7) >> 3;
        const long k = i >= p.first ? i - p.first : i, m = k / per;
        const int c = (int)(k - m * per) * 8;
        const __nv_bfloat16* s = y.src + m * y.ld + c;
        uint16_t t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = c + j < y.cols ? *reinterpret_cast<const uint16_t*>(s + j) : (uint16_t)0;
        *reinterpret_cast<uint4*>(y.dst + m * y.ldd + c) = make_uint4(t[0] | (uint32_t)t[1] << 16, t[2] | (uint32_t)t[3] << 16, t[4] | (uint32_t)t[5] << 16, t[6] | (uint32_t)t[7] << 16);
    }
}

// ------------------------------------------------------------------------------------------------ products: what they share
struct GatedOut {
    void* h; long ldh;                   // forward: h [M][F];  backward: dx [M][N]
    void* z; long ldz;                   // forward: [M][2F] or NULL
    const float* bias;                   // forward: [2F] or NULL
    int M, F, act;                       // F: columns of h, or of dx
    float* part; int splits;             // splits > 1: partial products [splits][M][2F] (forward) or [splits][M][F]
};
template <typename T> __device__ __forceinline__ void gated_end(const GatedOut& o, long m, int f, float g, float u) {
    constexpr bool EXACT = sizeof(T) == 4;
    if (o.bias) { g += o.bias[f]; u += o.bias[o.F + f]; }
    float h = 0.f;
    gate_dispatch<EXACT>(o.act, [&](auto a) { h = gate_act<decltype(a)::value, EXACT>(g) * u; });
    gate_store(static_cast<T*>(o.h) + m * o.ldh + f, h);
    if (o.z) { gate_store(static_cast<T*>(o.z) + m * o.ldz + f, g); gate_store(static_cast<T*>(o.z) + m * o.ldz + o.F + f, u); }
}
template <typename T, bool FWD>
__global__ void __launch_bounds__(256)
gated_reduce_kernel(const __grid_constant__ GatedOut o) {
    griddep_wait();
    const long n = (long)o.M * o.F, width = FWD ? 2L * o.F : o.F, plane = (long)o.M * width;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        const long m = i / o.F;
        const int f = (int)(i - m * o.F);
        const float* src = o.part + m * width + f;
        float g = 0.f, u = 0.f;
#pragma unroll 4
        for (int s = 0; s < o.splits; ++s) { g += src[s * plane]; if (FWD) u += src[s * plane + o.F]; }
        if (FWD) gated_end<T>(o, m, f, g, u);
        else gate_store(static_cast<T*>(o.h) + m * o.ldh + f, g);
    }
}

// ------------------------------------------------------------------------------------------------ fp32 ALUs
// 256 threads, BM x 128 tile of the product (forward: 64 gate and 64 up columns, so a thread holds both of a column), 16 of the contraction a
// step, the next step's operands in registers while this one's are multiplied from shared memory.
struct GatedSimt {
    const void* a; long lda;             // X [M][K] or dZ [M][2F]
    const void* w; long ldw;             // [2F][K]
    int M, N, KD;                        // N: columns of h or dx; KD: the contraction
    int tiles_n, k_per_split;            // k_per_split: a multiple of 16
    GatedOut out;
};
template <typename T, bool FWD, int BM>
__global__ void __launch_bounds__(256, 2)
gated_simt_kernel(const __grid_constant__ GatedSimt p) {
    constexpr int BN = 128, BK = 16, RM = BM / 16, LA = BM * BK / 256, LB = BN * BK / 256, HALF = FWD ? 64 : 128;
    __shared__ __align__(16) float as[2][BK][BM + 4], bs[2][BK][BN + 4];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int tm = blockIdx.x / p.tiles_n, tn = blockIdx.x - tm * p.tiles_n;
    const int m0 = tm * BM, n0 = tn * HALF;
    const int k_begin = blockIdx.y * p.k_per_split, k_end = min(p.KD, k_begin + p.k_per_split);
    const T* const a = static_cast<const T*>(p.a);
    const T* const w = static_cast<const T*>(p.w);
    float ra[LA], rb[LB];
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const int k = k0 + tx, m = m0 + ty + 16 * i;
            ra[i] = k < k_end && m < p.M ? to_f32(a[(long)m * p.lda + k]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            if constexpr (FWD) {
                const int k = k0 + tx, j = ty + 16 * i, f = n0 + (j & 63);
                rb[i] = k < k_end && f < p.N ? to_f32(w[(long)(f + (j >= 64 ? p.N : 0)) * p.ldw + k]) : 0.f;
            } else {
                const int k = k0 + (tid >> 7) + 2 * i, n = n0 + (tid & 127);
                rb[i] = k < k_end && n < p.N ? to_f32(w[(long)k * p.ldw + n]) : 0.f;
            }
        }
    };
    auto put = [&](int b) {
#pragma unroll
        for (int i = 0; i < LA; ++i) as[b][tx][ty + 16 * i] = ra[i];
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            if constexpr (FWD) bs[b][tx][ty + 16 * i] = rb[i];
            else bs[b][(tid >> 7) + 2 * i][tid & 127] = rb[i];
        }
    };
    griddep_launch_dependents();
    // thread's rows: ty * 4 + r and 64 + ty * 4 + r (BM = 128), or ty * 2 + r (BM = 32); columns: tx * 4 + c and 64 + tx * 4 + c, in pairs
    f32x2 acc2[RM][4];
#pragma unroll
    for (int r = 0; r < RM; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc2[r][c] = make_f32x2(0.f, 0.f);
    fetch(k_begin);
    put(0);
    __syncthreads();
    int buf = 0;
    for (int k0 = k_begin; k0 < k_end; k0 += BK) {
        const bool more = k0 + BK < k_end;
        if (more) fetch(k0 + BK);
#pragma unroll
        for (int k = 0; k < BK; ++k) {
            float x[RM];
            f32x2 y[4];
            if constexpr (RM == 8) {
                const float4 u = *reinterpret_cast<const float4*>(&as[buf][k][ty * 4]), v = *reinterpret_cast<const float4*>(&as[buf][k][64 + ty * 4]);
                x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
            } else {
                const float2 u = *reinterpret_cast<const float2*>(&as[buf][k][ty * 2]);
                x[0] = u.x; x[1] = u.y;
            }
            const float4 u = *reinterpret_cast<const float4*>(&bs[buf][k][tx * 4]), v = *reinterpret_cast<const float4*>(&bs[buf][k][64 + tx * 4]);
            y[0] = make_f32x2(u.x, u.y); y[1] = make_f32x2(u.z, u.w); y[2] = make_f32x2(v.x, v.y); y[3] = make_f32x2(v.z, v.w);
#pragma unroll
            for (int r = 0; r < RM; ++r) {
                const f32x2 xx = make_f32x2(x[r], x[r]);
#pragma unroll
                for (int c = 0; c < 4; ++c) acc2[r][c] = fma2(xx, y[c], acc2[r][c]);
            }
        }
        if (more) put(buf ^ 1);
        buf ^= 1;
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < RM; ++r) {
        const int m = m0 + (RM == 8 ? (r >> 2) * 64 + ty * 4 + (r & 3) : ty * 2 + r);
        if (m >= p.M) continue;
        float acc[8];
#pragma unroll
        for (int c = 0; c < 4; ++c) split_f32x2(acc2[r][c], acc[2 * c], acc[2 * c + 1]);
        if constexpr (FWD) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int f = n0 + tx * 4 + c;
                if (f >= p.N) continue;
                if (p.out.splits > 1) {
                    float* to = p.out.part + ((long)blockIdx.y * p.M + m) * 2 * p.N + f;
                    to[0] = acc[c]; to[p.N] = acc[c + 4];
                } else {
                    gated_end<T>(p.out, m, f, acc[c], acc[c + 4]);
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const int n = n0 + (c >> 2) * 64 + tx * 4 + (c & 3);
                if (n >= p.N) continue;
                if (p.out.splits > 1) p.out.part[((long)blockIdx.y * p.M + m) * p.N + n] = acc[c];
                else gate_store(static_cast<T*>(p.out.h) + (long)m * p.out.ldh + n, acc[c]);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ a few rows of X
struct GatedFew {
    const void* x; long ldx;
    const void* w; long ldw;
    int K;
    GatedOut out;
};
template <typename T, int V> struct GatedRaw { uint4 v; };
template <typename T> struct GatedRaw<T, 1> { T v; };
template <typename T, int V> __device__ __forceinline__ void gated_load(const T* p, GatedRaw<T, V>& r) {
    if constexpr (V == 1) r.v = *p;
    else r.v = __ldg(reinterpret_cast<const uint4*>(p));
}
template <typename T, int V> __device__ __forceinline__ void gated_vec(const GatedRaw<T, V>& r, float (&x)[V]) {
    if constexpr (V == 1) x[0] = to_f32(r.v);
    else {
        const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (V == 8) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
            else x[k] = __uint_as_float(w[k]);
        }
    }
}
// A warp: one gate row of W and its up row.  The lanes take 16 bytes each of a row, and the loads of four rounds go out before the first is
// used: a thousand columns are then one round trip to memory.
constexpr int GF_ROUNDS = 4;
template <typename T, int V, int MT>
__global__ void __launch_bounds__(128)
gated_few_kernel(const __grid_constant__ GatedFew p) {
    const int lane = threadIdx.x & 31, f = blockIdx.x * 4 + (threadIdx.x >> 5);
    const int F = p.out.F, M = p.out.M;
    if (f >= F) return;
    const T* const gate = static_cast<const T*>(p.w) + (long)f * p.ldw;
    const T* const up = static_cast<const T*>(p.w) + ((long)F + f) * p.ldw;
    const T* x[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = static_cast<const T*>(p.x) + (long)min(m, M - 1) * p.ldx;     // rows behind the last: sums nobody writes
    float g[MT], u[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) { g[m] = 0.f; u[m] = 0.f; }
    int k = lane * V;
    for (; k + (GF_ROUNDS - 1) * 32 * V < p.K; k += GF_ROUNDS * 32 * V) {
        GatedRaw<T, V> a[GF_ROUNDS], b[GF_ROUNDS];
#pragma unroll
        for (int i = 0; i < GF_ROUNDS; ++i) { gated_load<T, V>(gate + k + i * 32 * V, a[i]); gated_load<T, V>(up + k + i * 32 * V, b[i]); }
#pragma unroll
        for (int i = 0; i < GF_ROUNDS; ++i) {
            float wa[V], wb[V];
            gated_vec<T, V>(a[i], wa);
            gated_vec<T, V>(b[i], wb);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                GatedRaw<T, V> r;
                float xv[V];
                gated_load<T, V>(x[m] + k + i * 32 * V, r);
                gated_vec<T, V>(r, xv);
#pragma unroll
                for (int v = 0; v < V; ++v) { g[m] = fmaf(wa[v], xv[v], g[m]); u[m] = fmaf(wb[v], xv[v], u[m]); }
            }
        }
    }
    for (; k < p.K; k += 32 * V) {
        GatedRaw<T, V> a, b, r;
        float wa[V], wb[V], xv[V];
        gated_load<T, V>(gate + k, a);
        gated_load<T, V>(up + k, b);
        gated_vec<T, V>(a, wa);
        gated_vec<T, V>(b, wb);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            gated_load<T, V>(x[m] + k, r);
            gated_vec<T, V>(r, xv);
#pragma unroll
            for (int v = 0; v < V; ++v) { g[m] = fmaf(wa[v], xv[v], g[m]); u[m] = fmaf(wb[v], xv[v], u[m]); }
        }
    }
    float mine_g = 0.f, mine_u = 0.f;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const float a = warp_sum(g[m]), b = warp_sum(u[m]);
        if (lane == m) { mine_g = a; mine_u = b; }
    }
    if (lane < M && lane < MT) gated_end<T>(p.out, lane, f, mine_g, mine_u);
}

// ------------------------------------------------------------------------------------------------ tensor cores
namespace tc {
namespace gt {
constexpr int BK = 64, BM_CTA = 128;
constexpr int A_BYTES = BM_CTA * 128;                    // 128 rows x 64 bf16
constexpr int BOX_BYTES = 32 * 128;                      // 32 rows x 64 bf16 of an output
// Epilogue warps and the boxes of outputs they stage.  Forward: 16 warps, each 32 rows x 32 columns of h (and of zg, zu); two neighbours fill a
// box together.  (With 8 warps of 64 columns the epilogue's latency, not its 0.24 of the issue slots, paced the kernel: 133 us.)  h is staged where
// zg was, once that has left: a box less leaves shared memory for another stage (32768 x 512 -> 2048 with z:
// 137 -> 132 us in short runs; call after call the power cap makes it 151 to 158).  Backward: 8 warps,
// each 32 rows x HN columns of dx.
template <bool FWD, bool KEEP, int HN> struct Cfg {
    static constexpr int EPI_WARPS = FWD ? 16 : 8, THREADS = 64 + 32 * EPI_WARPS;
    static constexpr int BOXES = FWD ? (KEEP ? 2 : 1) : HN / 64;         // of a pair of warps, or of a warp
    static constexpr int STAGE_BYTES = A_BYTES + HN * 128;
    static constexpr int STAGING = 8 * BOXES * BOX_BYTES;
    static constexpr int STAGES = (224 * 1024 - STAGING) / STAGE_BYTES;
    static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + STAGING + 256 + 1024;
};
// Rows r0 .. r1 - 1 (r0 a multiple of 8) of a box to rows that TMA cannot address (bases or lengths that are no multiple of 16 bytes): a row's
// 64 columns per warp, as 32-bit words from its first 4-byte boundary on.  The path is bound by instructions, so what depends on a row's
// parity alone (odd lengths alternate) is worked out once for the even and once for the odd rows (20000 x 576 -> 1170 with z kept: 104 us; element
// by element 124; the same with 1176 columns by TMA 60).  `n`: columns there are.
__device__ __forceinline__ void box_rows_out(const uint8_t* box, __nv_bfloat16* to, long ld, int r0, int r1, int n, int lane) {
    uint32_t lo[2], hi[2];
    __nv_bfloat16* at[2];
    bool word[2], single[2], first[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        __nv_bfloat16* const row = to + (r0 + k) * ld;
        const int odd = (int)(reinterpret_cast<uintptr_t>(row) >> 1) & 1, e = 2 * lane + odd;
        at[k] = row + e;
        word[k] = e + 1 < min(n, 64);
        single[k] = e < n && !word[k];
        first[k] = odd && lane == 31;                            // its second element is the row's first
        lo[k] = e * 2; hi[k] = ((e + 1) & 63) * 2;
    }
    const uint32_t src = smem_u32(box);
#pragma unroll 1
    for (int r = r0; r < r1; r += 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = j & 1;
            uint16_t x, y;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(src + r * 128 + j * 128 + (lo[k] ^ (j << 4))));
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(src + r * 128 + j * 128 + (hi[k] ^ (j << 4))));
            __nv_bfloat16* const q = at[k] + (j >> 1) * 2 * ld;
            if (r + j < r1) {
                if (word[k]) *reinterpret_cast<uint32_t*>(q) = (uint32_t)x | (uint32_t)y << 16;
                if (single[k]) *reinterpret_cast<uint16_t*>(q) = x;
                if (first[k]) *reinterpret_cast<uint16_t*>(q - 63) = y;
            }
        }
        at[0] += 8 * ld;
        at[1] += 8 * ld;
    }
}
// 16 fp32 columns from `col` on of a warp's 32 rows from row0 on, a row a lane, to 64-byte runs of a matrix of M rows and F columns: through 2 KB of the
// warp's own (stored as they lie, 32 rows an instruction, the partial products made 304 x 4096 -> 1024 34 us where it takes 21).  vec: rows start at 16-byte boundaries.
__device__ __forceinline__ void rows16_out(float4* mine, const float* v, float* base, long ld, int row0, int M, int col, int F, bool vec, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j) mine[lane * 4 + (j ^ ((lane >> 1) & 3))] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    __syncwarp();
    if (vec && col + 16 <= F) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 8 + (lane >> 2), s = lane & 3;
            if (row0 + r < M) *reinterpret_cast<float4*>(base + (long)(row0 + r) * ld + col + s * 4) = mine[r * 4 + (s ^ ((r >> 1) & 3))];
        }
    } else {
        // rows at any address, or the last columns: one element a lane, sixteen lanes a row
        const float* const flat = reinterpret_cast<const float*>(mine);
        const int s = lane & 15, c = col + s;
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
            const int r = i * 2 + (lane >> 4);
            const float q = flat[r * 16 + (((s >> 2) ^ ((r >> 1) & 3)) << 2) + (s & 3)];
            if (row0 + r < M && c < F) base[(long)(row0 + r) * ld + c] = q;
        }
    }
    __syncwarp();
}
struct Maps { CUtensorMap a, b[2], h, z[2]; };           // b: rows of CTA 0 and of CTA 1; h: output (dx); z: gate and up halves of Z
struct Params {
    int KB;                              // stages of the contraction
    int kb_per_split;
    int tiles_m, tiles_n, total;         // total: with splits
    int tma_out;                         // outputs go by TMA; else by plain stores
    int* status;
    GatedOut out;
};
// Tiles in groups of eight rows of tiles, along the rows first: 74 pairs then work on an 8 x 9 block of the product, whose operands stay in L2.
struct Tile { int m, n, split; };
__device__ __forceinline__ Tile tile_at(const Params& p, int t) {
    Tile w;
    const int tiles = p.tiles_m * p.tiles_n;
    w.split = t / tiles;
    t -= w.split * tiles;
    const int group = t / (8 * p.tiles_n), rows = min(8, p.tiles_m - group * 8);
    t -= group * 8 * p.tiles_n;
    w.n = t / rows;
    w.m = group * 8 + t - w.n * rows;
    return w;
}
__device__ __forceinline__ void tma_load_2d_pair(void* smem_dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
    // the bytes are counted on a barrier of CTA 0 of the pair, whichever of the two loads
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, const void* smem_src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(smem_src)), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
}  // namespace gt

// Warp 0: loads of this CTA's operands (A rows; gate or up rows of W, or half of the columns of W), all counted on CTA 0's `full`; warp 1 of
// CTA 0: MMAs, commits to both CTAs' `empty` and `acc_full`; the others: epilogue, warp w on lanes 32 (w % 4) .. + 31 of the tensor memory.
// The accumulator is double-buffered (2 x 2 HN <= 512 columns), so a tile's epilogue runs under the next tile's MMAs.  Every wait is bounded.
template <bool FWD, bool KEEP, int HN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__((gt::Cfg<FWD, KEEP, HN>::THREADS), 1)
gated_tc_kernel(const __grid_constant__ gt::Maps maps, const __grid_constant__ gt::Params p) {
    using namespace gt;
    using C = Cfg<FWD, KEEP, HN>;
    constexpr int STAGES = C::STAGES, STAGE_BYTES = C::STAGE_BYTES, N = 2 * HN;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);     // the same offset in both CTAs
    uint8_t* staging = smem + STAGES * STAGE_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(staging + C::STAGING);              // CTA 0's are used
    uint64_t* empty = full + STAGES;                                                 // each CTA's own
    uint64_t* acc_full = empty + STAGES;                                             // [2], each CTA's own
    uint64_t* acc_empty = acc_full + 2;                                              // [2], CTA 0's are used
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 2 * C::EPI_WARPS); }
        *abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&maps.a); tma_prefetch_desc(&maps.b[rank]);
    }
    if (warp == 1) { tmem_alloc_pair(tmem_slot, 512); tmem_relinquish_pair(); }
    tc_fence_before_sync();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    griddep_wait();                      // operands that a launch in front of this one has written
    griddep_launch_dependents();

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t full0 = mapa_shared(smem_u32(full), 0);
            int stage = 0; uint32_t phase = 0;
            bool ok = true;
            for (int t = pair; t < p.total && ok; t += pairs) {
                const Tile w = tile_at(p, t);
                const int kb0 = w.split * p.kb_per_split, kb1 = min(p.KB, kb0 + p.kb_per_split);
                const int m0 = w.m * 2 * BM_CTA + (int)rank * BM_CTA;
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = mbar_wait(&empty[stage], phase ^ 1, abort_flag, p.status);
                    if (!ok) break;
                    uint8_t* dst = smem + stage * STAGE_BYTES;
                    const uint32_t bar = full0 + stage * 8;
                    if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * STAGE_BYTES);
                    tma_load_2d_pair(dst, &maps.a, bar, kb * BK, m0);
                    if constexpr (FWD) {
                        tma_load_2d_pair(dst + A_BYTES, &maps.b[rank], bar, kb * BK, w.n * HN);
                    } else {
#pragma unroll
                        for (int c = 0; c < HN / 64; ++c)
                            tma_load_2d_pair(dst + A_BYTES + c * 8192, &maps.b[rank], bar, w.n * N + (int)rank * HN + c * 64, kb * BK);
                    }
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            constexpr uint32_t idesc = make_idesc_bf16(256, N, 0, FWD ? 0 : 1);
            int stage = 0, it = 0; uint32_t phase = 0;
            bool ok = true;
            for (int t = pair; t < p.total && ok; t += pairs, ++it) {
                const Tile w = tile_at(p, t);
                const int kb0 = w.split * p.kb_per_split, kb1 = min(p.KB, kb0 + p.kb_per_split);
                const int buf = it & 1;
                ok = mbar_wait(&acc_empty[buf], ((it >> 1) & 1) ^ 1, abort_flag, p.status);
                if (!ok) break;
                tc_fence_after_sync();
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = mbar_wait(&full[stage], phase, abort_flag, p.status);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t a = smem_u32(smem + stage * STAGE_BYTES), b = a + A_BYTES;
#pragma unroll
                    for (int k4 = 0; k4 < BK / 16; ++k4) {
                        const uint64_t da = make_smem_desc_sw128(a + k4 * 32, 16, 1024);
                        const uint64_t db = FWD ? make_smem_desc_sw128(b + k4 * 32, 16, 1024) : make_smem_desc_sw128(b + k4 * 2048, 8192, 1024);
                        mma_bf16_ss_pair(tmem_base + buf * N, da, db, idesc, (kb == kb0 && k4 == 0) ? 0u : 1u);
                    }
                    mma_commit_pair(&empty[stage], 3);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
                if (!ok) break;
                mma_commit_pair(&acc_full[buf], 3);
            }
        }
    } else if constexpr (FWD) {
        // ------------------------------------------------ epilogue, forward: 32 columns a warp
        const int quarter = warp & 3, group = (warp - 2) >> 2, box = group >> 1, slot = (group & 1) * 4;
        uint8_t* const boxes = staging + (box * 4 + quarter) * C::BOXES * BOX_BYTES;
        const int pair_bar = 1 + box * 4 + quarter;                          // the two warps of a box
        const bool stores = (group & 1) == 0 && lane == 0;                   // who hands the box to TMA
        const uint32_t acc_empty0 = mapa_shared(smem_u32(acc_empty), 0);
        const GatedOut& o = p.out;
        int it = 0;
        bool ok = true;
        for (int t = pair; t < p.total; t += pairs, ++it) {
            const Tile w = tile_at(p, t);
            const int buf = it & 1;
            const int row0 = w.m * 2 * BM_CTA + (int)rank * BM_CTA + quarter * 32;
            const int box_col = w.n * HN + box * 64, col = box_col + (group & 1) * 32;
            float bias_g = 0.f, bias_u = 0.f;                                // of column `lane`: to the others by shuffle
            if (o.bias && col + lane < o.F && o.splits == 1) { bias_g = o.bias[col + lane]; bias_u = o.bias[o.F + col + lane]; }
            // A wait that ran out must not leave the box's other warp at a barrier: from then on both only keep step.
            ok = __all_sync(0xFFFFFFFFu, ok && mbar_wait(&acc_full[buf], (it >> 1) & 1, abort_flag, p.status));
            tc_fence_after_sync();
            const uint32_t tm = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * N + group * 32;
            const bool there = group * 32 < HN && row0 < o.M && box_col < o.F;   // the same for both warps of a box
            uint32_t g[32], u[32];
            if (there && ok) {
                tmem_ld_32x32(tm, g);
                tmem_ld_32x32(tm + HN, u);
                tmem_ld_wait();
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0 && ok) mbar_arrive_cluster(acc_empty0 + buf * 8);
            if (!there) continue;
            if (o.splits > 1) {
                if (!ok) continue;
                float* const part = o.part + (long)w.split * o.M * 2L * o.F;
                float4* const mine = reinterpret_cast<float4*>(boxes + (group & 1) * 2048);
                float v[32], x[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) { v[j] = __uint_as_float(g[j]); x[j] = __uint_as_float(u[j]); }
#pragma unroll
                for (int c = 0; c < 32; c += 16) {
                    rows16_out(mine, v + c, part, 2L * o.F, row0, o.M, col + c, o.F, o.F % 4 == 0, lane);
                    rows16_out(mine, x + c, part + o.F, 2L * o.F, row0, o.M, col + c, o.F, o.F % 4 == 0, lane);
                }
                continue;
            }
            auto step = [&] { asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory"); };     // the two warps of a box
            if (stores) bulk_wait_read();                                    // the box's last tile has left
            step();
            if (!ok) {
                for (int i = 0; i < (KEEP ? 3 : 1); ++i) step();
                continue;
            }
            // 32 columns of a row = four 16-byte slots of a 128-byte row, at their swizzled places
            uint8_t* const mine = boxes + lane * 128;
            const int sw = lane & 7;
            auto put = [&](uint8_t* at, const uint32_t (&v)[32]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t q[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        q[k] = f32x2_to_bf16x2(make_f32x2(__uint_as_float(v[8 * j + 2 * k]), __uint_as_float(v[8 * j + 2 * k + 1])));
                    *reinterpret_cast<uint4*>(at + (((slot + j) ^ sw) << 4)) = make_uint4(q[0], q[1], q[2], q[3]);
                }
            };
            if (o.bias) {
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    g[j] = __float_as_uint(__uint_as_float(g[j]) + __shfl_sync(0xFFFFFFFFu, bias_g, j));
                    u[j] = __float_as_uint(__uint_as_float(u[j]) + __shfl_sync(0xFFFFFFFFu, bias_u, j));
                }
            }
            // the box to h, or both to the halves of z
            auto send = [&](bool is_z) {
                if (p.tma_out) fence_proxy_async_smem();
                step();
                if (p.tma_out) {
                    if (stores) {
                        if (is_z) { tma_store_2d(&maps.z[0], boxes, box_col, row0); tma_store_2d(&maps.z[1], boxes + BOX_BYTES, box_col, row0); }
                        else tma_store_2d(&maps.h, boxes, box_col, row0);
                        bulk_commit();
                    }
                    return;
                }
                const int r0 = (group & 1) * 16, r1 = min(r0 + 16, o.M - row0);
                __nv_bfloat16* const to = static_cast<__nv_bfloat16*>(is_z ? o.z : o.h);
                const long ld = is_z ? o.ldz : o.ldh;
#pragma unroll 1
                for (int b = 0; b < (is_z ? 2 : 1); ++b)
                    box_rows_out(boxes + b * BOX_BYTES, to + (long)row0 * ld + (b ? o.F : 0) + box_col, ld, r0, r1, o.F - box_col, lane);
            };
            if (KEEP) { put(mine, g); put(mine + BOX_BYTES, u); send(true); }
            gate_dispatch<false>(o.act, [&](auto a) {
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    const f32x2 h = gate_pair<decltype(a)::value>(make_f32x2(__uint_as_float(g[j]), __uint_as_float(g[j + 1])),
                                                                  make_f32x2(__uint_as_float(u[j]), __uint_as_float(u[j + 1])));
                    float x, y;
                    split_f32x2(h, x, y);
                    g[j] = __float_as_uint(x); g[j + 1] = __float_as_uint(y);
                }
            });
            if (KEEP) {                                                      // h goes where zg was
                if (stores) bulk_wait_read();
                step();
            }
            put(mine, g);
            send(false);
        }
        if (stores) bulk_wait();
    } else {
        // ------------------------------------------------ epilogue, backward: HN columns a warp
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        uint8_t* const boxes = staging + (warp - 2) * C::BOXES * BOX_BYTES;
        const uint32_t acc_empty0 = mapa_shared(smem_u32(acc_empty), 0);
        const GatedOut& o = p.out;
        int it = 0;
        for (int t = pair; t < p.total; t += pairs, ++it) {
            const Tile w = tile_at(p, t);
            const int buf = it & 1;
            const int row0 = w.m * 2 * BM_CTA + (int)rank * BM_CTA + quarter * 32;
            const int col0 = w.n * N + half * HN;
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(&acc_full[buf], (it >> 1) & 1, abort_flag, p.status))) break;
            tc_fence_after_sync();
            const uint32_t tm = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * N + half * HN;
            const bool there = row0 < o.M && col0 < o.F;
            if (there && o.splits == 1) { if (lane == 0) bulk_wait_read(); __syncwarp(); }
#pragma unroll 1
            for (int c = 0; c < HN / 32; ++c) {
                if (!there) break;
                uint32_t g[32];
                tmem_ld_32x32(tm + c * 32, g);
                tmem_ld_wait();
                const int col = col0 + c * 32;
                if (o.splits > 1) {
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(g[j]);
#pragma unroll
                    for (int j = 0; j < 32; j += 16)
                        rows16_out(reinterpret_cast<float4*>(boxes), v + j, o.part + (long)w.split * o.M * o.F, o.F, row0, o.M, col + j, o.F, o.F % 4 == 0, lane);
                    continue;
                }
                uint8_t* const at = boxes + (c >> 1) * BOX_BYTES + lane * 128;
                const int slot = (c & 1) * 4, sw = lane & 7;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t q[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        q[k] = f32x2_to_bf16x2(make_f32x2(__uint_as_float(g[8 * j + 2 * k]), __uint_as_float(g[8 * j + 2 * k + 1])));
                    *reinterpret_cast<uint4*>(at + (((slot + j) ^ sw) << 4)) = make_uint4(q[0], q[1], q[2], q[3]);
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acc_empty0 + buf * 8);
            if (!there || o.splits > 1) continue;
            if (p.tma_out) {
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
#pragma unroll
                    for (int b = 0; b < HN / 64; ++b)
                        if (col0 + b * 64 < o.F) tma_store_2d(&maps.h, boxes + b * BOX_BYTES, col0 + b * 64, row0);
                    bulk_commit();
                }
            } else {
                __syncwarp();
#pragma unroll 1
                for (int b = 0; b < C::BOXES; ++b) {
                    const int cb = col0 + b * 64;
                    if (cb < o.F)
                        box_rows_out(boxes + b * BOX_BYTES, static_cast<__nv_bfloat16*>(o.h) + (long)row0 * o.ldh + cb, o.ldh, 0, min(32, o.M - row0), o.F - cb, lane);
                }
                __syncwarp();
            }
        }
        if (lane == 0) bulk_wait();
    }
    if (*abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
    }
    tc_fence_before_sync();
    cluster_sync_all();
    if (warp == 1) { tc_fence_after_sync(); tmem_dealloc_pair(tmem_base, 512); }
}
}  // namespace tc
}  // namespace dpclip

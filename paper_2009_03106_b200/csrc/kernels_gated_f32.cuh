// The gated block's products in fp32 on the tensor cores.
//
// An fp32 number is the sum of three bf16 numbers, exactly: its top 8 significant bits, the next 8, the last 8 (each cut off, not rounded, so
// nothing overflows).  gated_split_kernel writes X (or dZ) and W as three such planes, and the product is the six products of planes whose
// weights are not below 2^-24: hh, hm, mh, mm, hl, lh; what is left out is below 2^-23 of a term.  Six bf16 products take the tensor cores as
// long as three in tf32, and the 16-bit operands keep the layouts of the bf16 kernel (W read by rows in one direction, by columns in the other).
//
// The tensor core adds to its accumulator with truncation, a bias toward zero of about 2^-26 per addition.  So a window of 64 contracted
// columns (24 additions, the small products first) is all that is summed there: the epilogue warps add the windows up in registers,
// correctly rounded, while the next window is multiplied in the other accumulator.
//
// Bound: the six products, about 1.4 PFLOP/s / 6; 3850 x 300 x 1100 with stored pre-activations: the splits and 51 MB of outputs weigh as
// much (47 us; 16384 x 512 -> 2048 350, of which the products 253).  The fp32 ALUs (gated_simt_kernel) reach 32 TFLOP/s on the same call.
#pragma once
#include "kernels_gated.cuh"

namespace dpclip {

// src [rows][cols] fp32 -> planes dst + k * plane, rows of ldd (a multiple of 8).  Two matrices a launch.
struct GatedSplit { const float* src; long ld; __nv_bfloat16* dst; long ldd, plane, rows; int cols, vec; };
struct GatedSplits { GatedSplit c[2]; long first; };         // first: groups of four of the first matrix
__global__ void __launch_bounds__(256)
gated_split_kernel(const __grid_constant__ GatedSplits p, long n) {
    griddep_launch_dependents();
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        const GatedSplit& y = p.c[i >= p.first];
        const uint32_t per = (uint32_t)(y.cols + 3) >> 2;
        const long k = i >= p.first ? i - p.first : i, m = k / per;
        const int c = (int)(k - m * per) * 4;
        const float* s = y.src + m * y.ld + c;
        float x[4];
        if (y.vec) {
            const float4 v = *reinterpret_cast<const float4*>(s);
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = c + j < y.cols ? s[j] : 0.f;
        }
        uint16_t t[4][3];
#pragma unroll
        for (int j = 0; j < 4; ++j) split3(x[j], t[j]);
#pragma unroll
        for (int j = 0; j < 3; ++j)
            *reinterpret_cast<uint2*>(y.dst + j * y.plane + m * y.ldd + c) =
                make_uint2(t[0][j] | (uint32_t)t[1][j] << 16, t[2][j] | (uint32_t)t[3][j] << 16);
    }
}

namespace tc {
namespace gt3 {
constexpr int BK = 64, BM_CTA = 128, EPI_WARPS = 16, THREADS = 64 + 32 * EPI_WARPS, STAGES = 2;
constexpr int A_BYTES = BM_CTA * 128;
constexpr int STAGING = EPI_WARPS * 2048;                 // a warp: 32 rows x 16 columns fp32
template <int HN> struct Cfg {
    static constexpr int B_BYTES = HN * 128;
    static constexpr int STAGE_BYTES = 3 * (A_BYTES + B_BYTES);
    static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + STAGING + 256 + 1024;
};
struct Maps { CUtensorMap a[3], b[2][3]; };               // by plane; b: of CTA 0 and of CTA 1
struct Params {
    int KB, kb_per_split, tiles_m, tiles_n, total;
    int vec_h, vec_z;                     // rows of the outputs take 16-byte stores
    int* status;
    GatedOut out;
    const float* a; long lda;             // the operands themselves: A [M][KD], W [2F][K]
    const float* w; long ldw;
    int KD;
};
// Infinities.  The planes of a number that bf16 holds are the number, 0 and 0, and an infinity times those zeros is NaN where the product is
// an infinity.  So a sum that comes out as NaN is taken again from the numbers themselves (a NaN among the terms, infinities of both signs
// or an infinity times zero give NaN again): 16 columns of a warp's 32 rows, through the warp's staging.  `n`: the first column, a row of W in
// the forward pass, a column of W in the backward pass; k0, k1: the contraction.  The look at every sum costs 1 us of
// 46 at 3850 x 300 -> 1100; inputs that are all NaN, 0.13 ms.  (Called instead of inlined it cost 4 us: the sums are spilled around a call.)
template <bool FWD>
__device__ __forceinline__ void gated_take_again(float* mine, const Params& p, long m, long n, int cols, int k0, int k1, int lane) {
    __syncwarp();
    if (m < p.out.M) {
#pragma unroll 1
        for (int j = 0; j < cols; ++j) {
            const float v = mine[j * 32 + lane];
            if (v == v) continue;
            const float* a = p.a + m * p.lda;
            const float* w = FWD ? p.w + (n + j) * p.ldw : p.w + n + j;
            const long inc = FWD ? 1 : p.ldw;
            float sum = 0.f;
            int k = k0;
#pragma unroll 1
            for (; k + 4 <= k1 && sum == sum; k += 4) {                       // a NaN stays one
#pragma unroll
                for (int i = 0; i < 4; ++i) sum = fmaf(a[k + i], w[(k + i) * inc], sum);
            }
#pragma unroll 1
            for (; k < k1 && sum == sum; ++k) sum = fmaf(a[k], w[k * inc], sum);
            mine[j * 32 + lane] = sum;
        }
    }
    __syncwarp();
}
}  // namespace gt3

// Roles as in gated_tc_kernel.  A stage holds three planes of both operands; a window is one stage.
template <bool FWD, int HN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(gt3::THREADS, 1)
gated_tc3_kernel(const __grid_constant__ gt3::Maps maps, const __grid_constant__ gt3::Params p) {
    using namespace gt3;
    using C = Cfg<HN>;
    constexpr int STAGE_BYTES = C::STAGE_BYTES, N = 2 * HN, CW = HN / 4;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);     // the same offset in both CTAs
    uint8_t* staging = smem + STAGES * STAGE_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(staging + STAGING);                 // CTA 0's are used
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
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 2 * EPI_WARPS); }
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) { tmem_alloc_pair(tmem_slot, 512); tmem_relinquish_pair(); }
    tc_fence_before_sync();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    griddep_wait();                       // the planes
    griddep_launch_dependents();

    auto tile_at = [&](int t, int& m, int& n, int& kb0, int& kb1) {
        const int tiles = p.tiles_m * p.tiles_n, split = t / tiles;
        t -= split * tiles;
        const int group = t / (8 * p.tiles_n), rows = min(8, p.tiles_m - group * 8);
        t -= group * 8 * p.tiles_n;
        n = t / rows;
        m = group * 8 + t - n * rows;
        kb0 = split * p.kb_per_split;
        kb1 = min(p.KB, kb0 + p.kb_per_split);
        return split;
    };

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t full0 = mapa_shared(smem_u32(full), 0);
            int stage = 0; uint32_t phase = 0;
            bool ok = true;
            for (int t = pair; t < p.total && ok; t += pairs) {
                int tm, tn, kb0, kb1;
                tile_at(t, tm, tn, kb0, kb1);
                const int m0 = tm * 2 * BM_CTA + (int)rank * BM_CTA;
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = mbar_wait(&empty[stage], phase ^ 1, abort_flag, p.status);
                    if (!ok) break;
                    uint8_t* dst = smem + stage * STAGE_BYTES;
                    const uint32_t bar = full0 + stage * 8;
                    if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * STAGE_BYTES);
#pragma unroll
                    for (int j = 0; j < 3; ++j) {
                        gt::tma_load_2d_pair(dst + j * A_BYTES, &maps.a[j], bar, kb * BK, m0);
                        uint8_t* b = dst + 3 * A_BYTES + j * C::B_BYTES;
                        if constexpr (FWD) {
                            gt::tma_load_2d_pair(b, &maps.b[rank][j], bar, kb * BK, tn * HN);
                        } else {
#pragma unroll
                            for (int c = 0; c < HN / 64; ++c)
                                gt::tma_load_2d_pair(b + c * 8192, &maps.b[rank][j], bar, tn * N + (int)rank * HN + c * 64, kb * BK);
                        }
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
            for (int t = pair; t < p.total && ok; t += pairs) {
                int tm, tn, kb0, kb1;
                tile_at(t, tm, tn, kb0, kb1);
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int buf = it & 1;
                    ok = mbar_wait(&acc_empty[buf], ((it >> 1) & 1) ^ 1, abort_flag, p.status) && mbar_wait(&full[stage], phase, abort_flag, p.status);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t a = smem_u32(smem + stage * STAGE_BYTES), b = a + 3 * A_BYTES;
                    // planes of A and B, the smallest products first
                    constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                    for (int q = 0; q < 6; ++q)
#pragma unroll
                        for (int k4 = 0; k4 < BK / 16; ++k4) {
                            const uint64_t da = make_smem_desc_sw128(a + PA[q] * A_BYTES + k4 * 32, 16, 1024);
                            const uint32_t at = b + PB[q] * C::B_BYTES;
                            const uint64_t db = FWD ? make_smem_desc_sw128(at + k4 * 32, 16, 1024) : make_smem_desc_sw128(at + k4 * 2048, 8192, 1024);
                            mma_bf16_ss_pair(tmem_base + buf * N, da, db, idesc, q == 0 && k4 == 0 ? 0u : 1u);
                        }
                    mma_commit_pair(&empty[stage], 3);
                    mma_commit_pair(&acc_full[buf], 3);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
        }
    } else {
        // A warp: 32 rows; columns [at0, at0 + CW) and [at1, at1 + CW) of the accumulator (forward: gate and up of the same columns of h)
        const int quarter = warp & 3, group = (warp - 2) >> 2;
        const int at0 = FWD ? group * CW : group * 2 * CW, at1 = FWD ? HN + at0 : at0 + CW;
        const uint32_t acc_empty0 = mapa_shared(smem_u32(acc_empty), 0);
        float4* const mine = reinterpret_cast<float4*>(staging + (warp - 2) * 2048);
        const GatedOut& o = p.out;
        int it = 0;
        bool ok = true;
        for (int t = pair; t < p.total && ok; t += pairs) {
            int tm, tn, kb0, kb1;
            const int split = tile_at(t, tm, tn, kb0, kb1);
            const int row0 = tm * 2 * BM_CTA + (int)rank * BM_CTA + quarter * 32;
            const int col0 = tn * (FWD ? HN : N) + at0, col1 = FWD ? col0 : col0 + CW;
            // A lane's share of the biases, for shuffles in the epilogue; loads there, one a column and lane, were 1.5 us a tile.
            float bias_g = 0.f, bias_u = 0.f;
            if (FWD && o.bias && lane < CW && col0 + lane < o.F) { bias_g = o.bias[col0 + lane]; bias_u = o.bias[o.F + col0 + lane]; }
            float x[2][CW];
#pragma unroll
            for (int j = 0; j < CW; ++j) { x[0][j] = 0.f; x[1][j] = 0.f; }
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const int buf = it & 1;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&acc_full[buf], (it >> 1) & 1, abort_flag, p.status));
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t tmem = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * N;
#pragma unroll
                for (int c = 0; c < CW; c += 16) {
                    uint32_t v[16], w[16];
                    tmem_ld_32x16(tmem + at0 + c, v);
                    tmem_ld_32x16(tmem + at1 + c, w);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) { x[0][c + j] += __uint_as_float(v[j]); x[1][c + j] += __uint_as_float(w[j]); }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acc_empty0 + buf * 8);
            }
            if (!ok) break;
            if (row0 >= o.M || col0 >= o.F) continue;
            f32x2 nan = make_f32x2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < CW; ++j) nan = add2(nan, make_f32x2(x[0][j], x[1][j]));
            const float any = sum_f32x2(nan);             // NaN if one of them is (and for infinities of both signs)
            if (__any_sync(0xFFFFFFFFu, any != any)) {
                float* const flat = reinterpret_cast<float*>(mine);
                constexpr int PER = CW / 16;              // groups of 16 columns a half
#pragma unroll 1
                for (int q = 0; q < 2 * PER; ++q) {
                    const int half = q / PER, c = q % PER * 16, col = (half ? col1 : col0) + c;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float v = x[0][j];
#pragma unroll
                        for (int g = 1; g < 2 * PER; ++g) v = g == q ? x[g / PER][g % PER * 16 + j] : v;
                        flat[j * 32 + lane] = v;
                    }
                    gated_take_again<FWD>(flat, p, row0 + lane, col + (FWD && half ? (long)o.F : 0L), min(16, o.F - col), kb0 * BK,
                                          min(kb1 * BK, p.KD), lane);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float v = flat[j * 32 + lane];
#pragma unroll
                        for (int g = 0; g < 2 * PER; ++g) x[g / PER][g % PER * 16 + j] = g == q ? v : x[g / PER][g % PER * 16 + j];
                    }
                    __syncwarp();
                }
            }
            auto put = [&](const float* v, float* base, long ld, int col, bool vec) { gt::rows16_out(mine, v, base, ld, row0, o.M, col, o.F, vec, lane); };
            if (o.splits > 1) {
                const long width = FWD ? 2L * o.F : o.F;
                float* const part = o.part + (long)split * o.M * width;
                const bool vec = o.F % 4 == 0;
#pragma unroll
                for (int c = 0; c < CW; c += 16) {
                    put(&x[0][c], part, width, col0 + c, vec);
                    put(&x[1][c], part + (FWD ? o.F : 0), width, col1 + c, vec);
                }
                continue;
            }
            if constexpr (FWD) {
                if (o.bias) {
#pragma unroll
                    for (int j = 0; j < CW; ++j) { x[0][j] += __shfl_sync(0xFFFFFFFFu, bias_g, j); x[1][j] += __shfl_sync(0xFFFFFFFFu, bias_u, j); }
                }
                if (o.z) {
                    float* const z = static_cast<float*>(o.z);
#pragma unroll
                    for (int c = 0; c < CW; c += 16) { put(&x[0][c], z, o.ldz, col0 + c, p.vec_z); put(&x[1][c], z + o.F, o.ldz, col0 + c, p.vec_z); }
                }
                gate_dispatch<true>(o.act, [&](auto a) {
#pragma unroll
                    for (int j = 0; j < CW; ++j) x[0][j] = gate_act<decltype(a)::value, true>(x[0][j]) * x[1][j];
                });
#pragma unroll
                for (int c = 0; c < CW; c += 16) put(&x[0][c], static_cast<float*>(o.h), o.ldh, col0 + c, p.vec_h);
            } else {
#pragma unroll
                for (int c = 0; c < CW; c += 16) {
                    put(&x[0][c], static_cast<float*>(o.h), o.ldh, col0 + c, p.vec_h);
                    put(&x[1][c], static_cast<float*>(o.h), o.ldh, col1 + c, p.vec_h);
                }
            }
        }
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

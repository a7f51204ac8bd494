// Norms of queries and keys, head by head, with the rotation by position in the same pass.
//
//   forward   y = R_pos (gain (.) x / rms(x)),  rms(x)^2 = mean_d x_d^2 + eps
//   backward  g = R_pos^T dy,  xh = x / rms,  dx = (gain (.) g - xh mean_d(gain (.) g (.) xh)) / rms,
//             per-example gradient of the gain  G_i = sum over the positions and heads of example i of g (.) xh
//
// A group of G lanes holds one head of one token.  The rotation pairs element d with d + rot / 2 (or its neighbour), so a lane holds
// both members: V elements of the first half and the V of the second half that go with them (V = 16 bytes), or 2V neighbours where pairs
// are neighbours and where nothing is rotated.  No value crosses lanes but for the sums over the head.  The groups of a warp take
// neighbouring heads of one token, so a warp instruction covers a run of memory and all its groups read the same angles.  Heads whose
// width or alignment does not allow that take V = 1: one warp a head, NCH pairs a lane.
//
// Bound: memory, every input is read once and every output written once.  A warp has U heads in flight per group.  The backward pass
// computes rms(x) again from the x it reads anyway, so the forward pass stores nothing for it.
#pragma once
#include "common.cuh"

namespace dpclip {

struct QkPart {
    const void* x; long xb, xt, xh;      // strides of example, token and head, elements
    const void* dy; long yb, yt, yh;     // backward: the signal at the output
    void* y; long ob, ot, oh;            // forward: the output; backward: dx
    const float* gain;                   // [D] or NULL (ones)
    float* part;                         // backward: [B][chunks][D] partial gradients
    int H, blocks, chunks;               // head blocks (of the groups of a warp) a token; backward: CTAs an example
};
struct QkParams {
    QkPart part[2];
    int B, T, D, rot, interleaved;
    long n_pos, pos0;
    const int* pos;                      // [B * T] or NULL: pos0 + t
    const float* table;                  // [n_pos][2][rot / 2]: cosines, sines
    float eps;
};

template <typename T, int V> struct QkRaw { T v[V]; };
template <> struct QkRaw<float, 4> { float4 v; };
template <> struct QkRaw<__nv_bfloat16, 8> { uint4 v; };
__device__ __forceinline__ void qk_load(const float* p, QkRaw<float, 4>& r) { r.v = *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void qk_load(const __nv_bfloat16* p, QkRaw<__nv_bfloat16, 8>& r) { r.v = *reinterpret_cast<const uint4*>(p); }
template <typename T> __device__ __forceinline__ void qk_load(const T* p, QkRaw<T, 1>& r) { r.v[0] = *p; }
__device__ __forceinline__ void qk_f32(const QkRaw<float, 4>& r, float (&x)[4]) { x[0] = r.v.x; x[1] = r.v.y; x[2] = r.v.z; x[3] = r.v.w; }
__device__ __forceinline__ void qk_f32(const QkRaw<__nv_bfloat16, 8>& r, float (&x)[8]) {
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int u = 0; u < 4; ++u) { x[2 * u] = __uint_as_float(w[u] << 16); x[2 * u + 1] = __uint_as_float(w[u] & 0xFFFF0000u); }
}
template <typename T> __device__ __forceinline__ void qk_f32(const QkRaw<T, 1>& r, float (&x)[1]) { x[0] = to_f32(r.v[0]); }
__device__ __forceinline__ void qk_store(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void qk_store(__nv_bfloat16* p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) { const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * u], x[2 * u + 1]); w[u] = *reinterpret_cast<const uint32_t*>(&v); }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void qk_store(float* p, const float (&x)[1]) { *p = x[0]; }
__device__ __forceinline__ void qk_store(__nv_bfloat16* p, const float (&x)[1]) { *p = __float2bfloat16_rn(x[0]); }

// Where the V + V elements of chunk c lie: two runs of V, [a0, a0 + V) and [a1, a1 + V); angles [rot0, rot0 + V) where turned.
template <int V>
struct QkChunk {
    int a0, a1, rot0;
    bool there, second, turned;          // second: the second run exists (the last element of an odd width has none)
    __device__ __forceinline__ QkChunk(int c, int D, int rot, int interleaved) {
        turned = 2 * c * V < rot;
        rot0 = c * V;
        const bool halves = turned && !interleaved;
        a0 = halves ? c * V : 2 * c * V;
        a1 = halves ? rot / 2 + c * V : a0 + V;
        there = a0 < D;
        second = a1 < D;
        turned = turned && there;
    }
};

// (lo, hi) <- the pairs turned by the angles; sign = -1 turns back
template <int V>
__device__ __forceinline__ void qk_turn(float (&lo)[V], float (&hi)[V], const float (&c)[V], const float (&s)[V], int interleaved) {
    if (V == 1 || !interleaved) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const float a = lo[u], b = hi[u];
            lo[u] = fmaf(a, c[u], -b * s[u]);
            hi[u] = fmaf(b, c[u], a * s[u]);
        }
    } else {
#pragma unroll
        for (int u = 0; u < V / 2; ++u) {
            const float a = lo[2 * u], b = lo[2 * u + 1], d = hi[2 * u], e = hi[2 * u + 1];
            lo[2 * u] = fmaf(a, c[u], -b * s[u]);
            lo[2 * u + 1] = fmaf(b, c[u], a * s[u]);
            hi[2 * u] = fmaf(d, c[u + V / 2], -e * s[u + V / 2]);
            hi[2 * u + 1] = fmaf(e, c[u + V / 2], d * s[u + V / 2]);
        }
    }
}
template <int V>
__device__ __forceinline__ void qk_floats(const float* p, float (&x)[V]) {
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int u = 0; u < V / 4; ++u) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(p) + u);
            x[4 * u] = v.x; x[4 * u + 1] = v.y; x[4 * u + 2] = v.z; x[4 * u + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int u = 0; u < V; ++u) x[u] = __ldg(p + u);
    }
}
template <int G>
__device__ __forceinline__ float qk_group_sum(float v) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ long qk_position(const QkParams& p, long token, int t) {
    const long at = p.pos ? (long)__ldg(p.pos + token) : p.pos0 + t;
    return at >= 0 && at < p.n_pos ? at : -1;            // a row without a position in the table is padding
}

constexpr int QK_THREADS = 256;

// blockIdx.y = block of 32 / G heads of the queries, then of the keys; a warp takes U tokens in a row of it.
template <typename T, int V, int NCH, int G, int U>
__global__ void __launch_bounds__(QK_THREADS)
qknorm_forward_kernel(const __grid_constant__ QkParams p) {
    constexpr int NG = 32 / G;
    const int lane = threadIdx.x & 31, gl = lane % G, grp = lane / G;
    const int which = (int)blockIdx.y >= p.part[0].blocks;
    const QkPart& y = p.part[which];
    const int h = ((int)blockIdx.y - (which ? p.part[0].blocks : 0)) * NG + grp;
    const uint32_t tokens = (uint32_t)p.B * p.T, token0 = (blockIdx.x * (QK_THREADS / 32) + (threadIdx.x >> 5)) * U;
    if (token0 >= tokens) return;
    int b = (int)(token0 / p.T), t = (int)(token0 - (uint32_t)b * p.T);
    float gain[2][NCH][V];
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
#pragma unroll
        for (int u = 0; u < V; ++u) { gain[0][n][u] = 1.f; gain[1][n][u] = 1.f; }
        if (y.gain && c.there) qk_floats<V>(y.gain + c.a0, gain[0][n]);
        if (y.gain && c.second) qk_floats<V>(y.gain + c.a1, gain[1][n]);
    }
    QkRaw<T, V> lo[U][NCH], hi[U][NCH];
    long pos[U];
    long out[U];
    const float inv_d = 1.f / (float)p.D;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        if (k > 0 && ++t == p.T) { t = 0; ++b; }
        pos[k] = -1; out[k] = 0;
        if (token0 + k >= tokens || h >= y.H) continue;
        pos[k] = qk_position(p, token0 + k, t);
        out[k] = (long)b * y.ob + (long)t * y.ot + (long)h * y.oh;
        const T* x = static_cast<const T*>(y.x) + (long)b * y.xb + (long)t * y.xt + (long)h * y.xh;
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
            if (c.there) qk_load(x + c.a0, lo[k][n]);
            if (c.second) qk_load(x + c.a1, hi[k][n]);
        }
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        float a[NCH][V], b[NCH][V], ss = 0.f;
        const bool live = pos[k] >= 0;
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
#pragma unroll
            for (int u = 0; u < V; ++u) { a[n][u] = 0.f; b[n][u] = 0.f; }
            if (live && c.there) qk_f32(lo[k][n], a[n]);
            if (live && c.second) qk_f32(hi[k][n], b[n]);
#pragma unroll
            for (int u = 0; u < V; ++u) { ss = fmaf(a[n][u], a[n][u], ss); ss = fmaf(b[n][u], b[n][u], ss); }
        }
        ss = qk_group_sum<G>(ss);
        const float r = rsqrtf(fmaf(ss, inv_d, p.eps));
        if (!live) continue;
        T* const to = static_cast<T*>(y.y) + out[k];
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
#pragma unroll
            for (int u = 0; u < V; ++u) { a[n][u] *= r * gain[0][n][u]; b[n][u] *= r * gain[1][n][u]; }
            if (c.turned) {
                float cs[V], sn[V];
                const float* angles = p.table + pos[k] * p.rot + c.rot0;
                qk_floats<V>(angles, cs);
                qk_floats<V>(angles + p.rot / 2, sn);
                qk_turn<V>(a[n], b[n], cs, sn, p.interleaved);
            }
            if (c.there) qk_store(to + c.a0, a[n]);
            if (c.second) qk_store(to + c.a1, b[n]);
        }
    }
}

// CTA = a chunk of one example's (token, head block) items of one part; its threads keep the gain's gradient of their elements in
// registers over the chunk.
template <typename T, int V, int NCH, int G, int U>
__global__ void __launch_bounds__(QK_THREADS, NCH * V <= 8 ? 2 : 1)
qknorm_backward_kernel(const __grid_constant__ QkParams p) {
    constexpr int NG = 32 / G, WARPS = QK_THREADS / 32;
    extern __shared__ float qk_smem[];                   // [WARPS][D]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane % G, grp = lane / G;
    int chunk = blockIdx.x;
    const int which = chunk >= p.part[0].chunks;
    if (which) chunk -= p.part[0].chunks;
    const QkPart& y = p.part[which];
    const int b = blockIdx.y;
    const uint32_t items = (uint32_t)p.T * y.blocks;     // of one example
    float gain[2][NCH][V], acc[2][NCH][V];
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
#pragma unroll
        for (int u = 0; u < V; ++u) { gain[0][n][u] = 1.f; gain[1][n][u] = 1.f; acc[0][n][u] = 0.f; acc[1][n][u] = 0.f; }
        if (y.gain && c.there) qk_floats<V>(y.gain + c.a0, gain[0][n]);
        if (y.gain && c.second) qk_floats<V>(y.gain + c.a1, gain[1][n]);
    }
    const float inv_d = 1.f / (float)p.D;
    const uint32_t stride = (uint32_t)y.chunks * WARPS;
    for (uint32_t item0 = (uint32_t)chunk * WARPS + warp; item0 < items; item0 += stride * U) {
        QkRaw<T, V> xl[U][NCH], xh[U][NCH], gl_[U][NCH], gh[U][NCH];
        long pos[U], out[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const uint32_t item = item0 + k * stride;
            pos[k] = -1; out[k] = -1;
            if (item >= items) continue;
            const int t = (int)(item / (uint32_t)y.blocks);
            const int h = (int)(item - (uint32_t)t * y.blocks) * NG + grp;
            if (h >= y.H) continue;
            pos[k] = qk_position(p, (long)b * p.T + t, t);
            out[k] = (long)b * y.ob + (long)t * y.ot + (long)h * y.oh;
            if (pos[k] < 0) continue;
            const T* x = static_cast<const T*>(y.x) + (long)b * y.xb + (long)t * y.xt + (long)h * y.xh;
            const T* d = static_cast<const T*>(y.dy) + (long)b * y.yb + (long)t * y.yt + (long)h * y.yh;
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
                if (c.there) { qk_load(x + c.a0, xl[k][n]); qk_load(d + c.a0, gl_[k][n]); }
                if (c.second) { qk_load(x + c.a1, xh[k][n]); qk_load(d + c.a1, gh[k][n]); }
            }
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const bool live = pos[k] >= 0;
            float xa[NCH][V], xb[NCH][V], ga[NCH][V], gb[NCH][V], ss = 0.f, dot = 0.f;
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
#pragma unroll
                for (int u = 0; u < V; ++u) { xa[n][u] = 0.f; xb[n][u] = 0.f; ga[n][u] = 0.f; gb[n][u] = 0.f; }
                if (live && c.there) { qk_f32(xl[k][n], xa[n]); qk_f32(gl_[k][n], ga[n]); }
                if (live && c.second) { qk_f32(xh[k][n], xb[n]); qk_f32(gh[k][n], gb[n]); }
                if (live && c.turned) {
                    float cs[V], sn[V];
                    const float* angles = p.table + pos[k] * p.rot + c.rot0;
                    qk_floats<V>(angles, cs);
                    qk_floats<V>(angles + p.rot / 2, sn);
#pragma unroll
                    for (int u = 0; u < V; ++u) sn[u] = -sn[u];
                    qk_turn<V>(ga[n], gb[n], cs, sn, p.interleaved);
                }
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    ss = fmaf(xa[n][u], xa[n][u], ss); ss = fmaf(xb[n][u], xb[n][u], ss);
                    dot = fmaf(ga[n][u] * gain[0][n][u], xa[n][u], dot); dot = fmaf(gb[n][u] * gain[1][n][u], xb[n][u], dot);
                }
            }
            ss = qk_group_sum<G>(ss);
            dot = qk_group_sum<G>(dot);
            if (out[k] < 0) continue;
            const float r = rsqrtf(fmaf(ss, inv_d, p.eps));
            const float m = dot * inv_d * r * r * r;      // mean(gain g xh) / rms^2: what dx has of x
            T* const to = static_cast<T*>(y.y) + out[k];
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
                if (live) {                               // a padding row has all zeros here: a zero signal goes back
#pragma unroll
                    for (int u = 0; u < V; ++u) {
                        ga[n][u] *= r; gb[n][u] *= r;
                        acc[0][n][u] = fmaf(ga[n][u], xa[n][u], acc[0][n][u]);
                        acc[1][n][u] = fmaf(gb[n][u], xb[n][u], acc[1][n][u]);
                        ga[n][u] = fmaf(-m, xa[n][u], ga[n][u] * gain[0][n][u]);
                        gb[n][u] = fmaf(-m, xb[n][u], gb[n][u] * gain[1][n][u]);
                    }
                }
                if (c.there) qk_store(to + c.a0, ga[n]);
                if (c.second) qk_store(to + c.a1, gb[n]);
            }
        }
    }
    // groups of the warp, then warps, in a fixed order
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        const QkChunk<V> c(gl + G * n, p.D, p.rot, p.interleaved);
#pragma unroll
        for (int u = 0; u < V; ++u) {
#pragma unroll
            for (int o = G; o < 32; o <<= 1) {
                acc[0][n][u] += __shfl_xor_sync(0xFFFFFFFFu, acc[0][n][u], o);
                acc[1][n][u] += __shfl_xor_sync(0xFFFFFFFFu, acc[1][n][u], o);
            }
            if (grp == 0 && c.there) qk_smem[warp * p.D + c.a0 + u] = acc[0][n][u];
            if (grp == 0 && c.second) qk_smem[warp * p.D + c.a1 + u] = acc[1][n][u];
        }
    }
    __syncthreads();
    float* const part = y.part + ((size_t)b * y.chunks + chunk) * p.D;
    for (int d = threadIdx.x; d < p.D; d += QK_THREADS) {
        float a = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) a += qk_smem[w * p.D + d];
        part[d] = a;
    }
}

// grads[i][d] = the chunks' sums in order, sq[i] = the sum of their squares; blockIdx.y = queries, keys.
struct QkFinish { const float* part[2]; int chunks[2]; float* grads[2]; float* sq[2]; int D; };
__global__ void __launch_bounds__(QK_THREADS)
qknorm_finish_kernel(const __grid_constant__ QkFinish p) {
    __shared__ float red[32];
    griddep_wait();
    const int i = blockIdx.x, which = blockIdx.y, chunks = p.chunks[which];
    float total = 0.f;
    for (int d = threadIdx.x; d < p.D; d += QK_THREADS) {
        const float* src = p.part[which] + (size_t)i * chunks * p.D + d;
        float a = 0.f;
#pragma unroll 8
        for (int c = 0; c < chunks; ++c) a += src[(size_t)c * p.D];
        if (p.grads[which]) p.grads[which][(size_t)i * p.D + d] = a;
        total = fmaf(a, a, total);
    }
    total = block_sum(total, red);
    if (threadIdx.x == 0 && p.sq[which]) p.sq[which][i] = total;
}

// table[pos][0][i] = cos(pos base^(-2i / rot) / scale), table[pos][1][i] its sine: angles in 64 bits, far positions lose theirs in 32.
__global__ void __launch_bounds__(256)
rotation_table_kernel(float* __restrict__ table, long n_pos, int rot, double log_base, double inv_scale) {
    const int half = rot / 2;
    const long n = n_pos * half;
    for (long j = (long)blockIdx.x * 256 + threadIdx.x; j < n; j += (long)gridDim.x * 256) {
        const long pos = j / half;
        const int i = (int)(j - pos * half);
        double s, c;
        sincos((double)pos * inv_scale * exp(-log_base * (2.0 * i / rot)), &s, &c);
        table[pos * rot + i] = (float)c;
        table[pos * rot + half + i] = (float)s;
    }
}

}  // namespace dpclip

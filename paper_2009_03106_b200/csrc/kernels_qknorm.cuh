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
// width or alignment does not allow that take V = 1: NCH pairs a lane, one element at a time.
//
// Bound: memory in long calls (every input is read once, every output written once), round trips in short ones.  The backward pass computes
// rms(x) again from the x it reads anyway, so the forward pass stores nothing for it.  128 x 256 tokens in bf16: 8 + 8 heads of 64 in 30 us (134
// MB, what a copy takes), backward 16 + 2 heads of 128 in 103 us (453 MB).
#pragma once
#include "common.cuh"

namespace dpclip {

struct QkPart {
    const void* x; long xb, xt, xh;      // strides of example, token and head, elements
    const void* dy; long yb, yt, yh;     // backward: the signal at the output
    void* y; long ob, ot, oh;            // forward: the output; backward: dx
    const float* gain;                   // [D] or NULL (ones)
    float* part;                         // backward: [B][blocks * chunks][D] partial gradients
    int H, blocks, chunks;               // blocks of heads (those of a warp's groups) a token; backward: CTAs an example and block
};
struct QkParams {
    QkPart part[2];
    int B, T, D, rot, interleaved;
    long n_pos, pos0;
    const int* pos;                      // [B * T] or NULL: pos0 + t
    const float* table;                  // [n_pos][2][rot / 2]: cosines, sines
    float eps;
};

// V elements of a run in fp32: pairs, or one element where V = 1
template <int V> struct QkVec { f32x2 v[V / 2]; };
template <> struct QkVec<1> { float v; };
template <int V> __device__ __forceinline__ QkVec<V> qk_fill(float x) {
    QkVec<V> r;
    if constexpr (V == 1) r.v = x;
    else {
#pragma unroll
        for (int u = 0; u < V / 2; ++u) r.v[u] = make_f32x2(x, x);
    }
    return r;
}
template <int V> __device__ __forceinline__ QkVec<V> qk_mul(const QkVec<V>& a, const QkVec<V>& b) {
    QkVec<V> r;
    if constexpr (V == 1) r.v = a.v * b.v;
    else {
#pragma unroll
        for (int u = 0; u < V / 2; ++u) r.v[u] = mul2(a.v[u], b.v[u]);
    }
    return r;
}
template <int V> __device__ __forceinline__ QkVec<V> qk_fma(const QkVec<V>& a, const QkVec<V>& b, const QkVec<V>& c) {
    QkVec<V> r;
    if constexpr (V == 1) r.v = fmaf(a.v, b.v, c.v);
    else {
#pragma unroll
        for (int u = 0; u < V / 2; ++u) r.v[u] = fma2(a.v[u], b.v[u], c.v[u]);
    }
    return r;
}
// sum += a . b, kept in two halves
template <int V> __device__ __forceinline__ void qk_dot(f32x2& sum, const QkVec<V>& a, const QkVec<V>& b) {
    if constexpr (V == 1) { float x, y; split_f32x2(sum, x, y); sum = make_f32x2(fmaf(a.v, b.v, x), y); }
    else {
#pragma unroll
        for (int u = 0; u < V / 2; ++u) sum = fma2(a.v[u], b.v[u], sum);
    }
}
template <int V> __device__ __forceinline__ void qk_floats(const QkVec<V>& a, float (&x)[V]) {
    if constexpr (V == 1) x[0] = a.v;
    else {
#pragma unroll
        for (int u = 0; u < V / 2; ++u) split_f32x2(a.v[u], x[2 * u], x[2 * u + 1]);
    }
}

// a run as loaded
template <typename T, int V> struct QkRaw { uint4 v; };
template <typename T> struct QkRaw<T, 1> { T v; };
template <typename T, int V> __device__ __forceinline__ void qk_load(const T* p, QkRaw<T, V>& r) {
    if constexpr (V == 1) r.v = *p;
    else r.v = *reinterpret_cast<const uint4*>(p);
}
template <typename T, int V> __device__ __forceinline__ void qk_zero(QkRaw<T, V>& r) {
    if constexpr (V == 1) r.v = T(0.f);
    else r.v = make_uint4(0u, 0u, 0u, 0u);
}
template <typename T, int V> __device__ __forceinline__ QkVec<V> qk_f32(const QkRaw<T, V>& r) {
    QkVec<V> x;
    if constexpr (V == 1) x.v = to_f32(r.v);
    else {
        const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
        if constexpr (V == 8) {
#pragma unroll
            for (int u = 0; u < 4; ++u) x.v[u] = bf16x2_to_f32x2(w[u]);
        } else {
            x.v[0] = make_f32x2(__uint_as_float(w[0]), __uint_as_float(w[1]));
            x.v[1] = make_f32x2(__uint_as_float(w[2]), __uint_as_float(w[3]));
        }
    }
    return x;
}
template <typename T, int V> __device__ __forceinline__ void qk_store(T* p, const QkVec<V>& x) {
    if constexpr (V == 1) {
        if constexpr (sizeof(T) == 4) *p = x.v;
        else *p = __float2bfloat16_rn(x.v);
    } else if constexpr (V == 8) {
        *reinterpret_cast<uint4*>(p) = make_uint4(f32x2_to_bf16x2(x.v[0]), f32x2_to_bf16x2(x.v[1]), f32x2_to_bf16x2(x.v[2]), f32x2_to_bf16x2(x.v[3]));
    } else {
        float f[V];
        qk_floats<V>(x, f);
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    }
}
template <int V> __device__ __forceinline__ QkVec<V> qk_params(const float* p) {
    QkVec<V> x;
    if constexpr (V == 1) x.v = __ldg(p);
    else {
#pragma unroll
        for (int u = 0; u < V / 4; ++u) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(p) + u);
            x.v[2 * u] = make_f32x2(f.x, f.y);
            x.v[2 * u + 1] = make_f32x2(f.z, f.w);
        }
    }
    return x;
}

template <int V> __device__ __forceinline__ QkVec<V> qk_shared(const float* p) {
    QkVec<V> x;
#pragma unroll
    for (int u = 0; u < V / 4; ++u) {
        float4 f;                        // volatile: a value kept in registers is what this is to avoid
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w)
                     : "r"((uint32_t)__cvta_generic_to_shared(p + 4 * u)));
        x.v[2 * u] = make_f32x2(f.x, f.y);
        x.v[2 * u + 1] = make_f32x2(f.z, f.w);
    }
    return x;
}

// Where the V + V elements of chunk c lie: two runs of V, [a0, a0 + V) and [a1, a1 + V); angles [rot0, rot0 + V) where turned.
template <int V>
struct QkChunk {
    int a0, a1, rot0;
    bool there, second, turned;          // second: the second run exists (the last element of an odd width has none)
    __device__ __forceinline__ void set(int c, int D, int rot, int interleaved) {
        turned = 2 * c * V < rot;
        rot0 = c * V;
        const bool halves = turned && !interleaved;
        a0 = halves ? c * V : 2 * c * V;
        a1 = halves ? rot / 2 + c * V : a0 + V;
        there = a0 < D;
        second = V == 1 ? a1 < D : there;
        turned = turned && there;
    }
};

// (lo, hi) <- the pairs turned by the angles
template <int V>
__device__ __forceinline__ void qk_turn(QkVec<V>& lo, QkVec<V>& hi, const QkVec<V>& c, const QkVec<V>& s, int interleaved) {
    if (V == 1 || !interleaved) {
        const QkVec<V> minus = qk_mul<V>(s, qk_fill<V>(-1.f)), a = lo;
        lo = qk_fma<V>(hi, minus, qk_mul<V>(a, c));
        hi = qk_fma<V>(a, s, qk_mul<V>(hi, c));
    } else if constexpr (V > 1) {
        float cs[V], sn[V];
        qk_floats<V>(c, cs);
        qk_floats<V>(s, sn);
#pragma unroll
        for (int u = 0; u < V / 2; ++u) {
            float a, b, d, e;
            split_f32x2(lo.v[u], a, b);
            split_f32x2(hi.v[u], d, e);
            lo.v[u] = make_f32x2(fmaf(a, cs[u], -b * sn[u]), fmaf(b, cs[u], a * sn[u]));
            hi.v[u] = make_f32x2(fmaf(d, cs[u + V / 2], -e * sn[u + V / 2]), fmaf(e, cs[u + V / 2], d * sn[u + V / 2]));
        }
    }
}
template <int G>
__device__ __forceinline__ float qk_group_sum(float v) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ long qk_position(const QkParams& p, uint32_t token, int t) {
    const long at = p.pos ? (long)__ldg(p.pos + token) : p.pos0 + t;
    return at >= 0 && at < p.n_pos ? at : -1;            // a row without a position in the table is padding
}

constexpr int QK_THREADS = 256;

// blockIdx.y = block of 32 / G heads of the queries, then of the keys; a warp takes one token of it.
template <typename T, int V, int NCH, int G>
__global__ void __launch_bounds__(QK_THREADS)
qknorm_forward_kernel(const __grid_constant__ QkParams p) {
    constexpr int NG = 32 / G;
    const int lane = threadIdx.x & 31, gl = lane % G, grp = lane / G;
    const int which = (int)blockIdx.y >= p.part[0].blocks;
    const QkPart& y = p.part[which];
    const int h = ((int)blockIdx.y - (which ? p.part[0].blocks : 0)) * NG + grp;
    const uint32_t tokens = (uint32_t)p.B * p.T, token = blockIdx.x * (QK_THREADS / 32) + (threadIdx.x >> 5);
    if (token >= tokens) return;
    const int b = (int)(token / (uint32_t)p.T), t = (int)(token - (uint32_t)b * p.T);
    const bool head = h < y.H;
    const long pos = head ? qk_position(p, token, t) : -1;
    const T* const x = static_cast<const T*>(y.x) + (long)b * y.xb + (long)t * y.xt + (long)h * y.xh;
    T* const out = static_cast<T*>(y.y) + (long)b * y.ob + (long)t * y.ot + (long)h * y.oh;
    QkChunk<V> c[NCH];
    QkRaw<T, V> lo[NCH], hi[NCH];
    QkVec<V> gain0[NCH], gain1[NCH];
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        c[n].set(gl + G * n, p.D, p.rot, p.interleaved);
        qk_zero(lo[n]); qk_zero(hi[n]);
        if (head && c[n].there) qk_load(x + c[n].a0, lo[n]);         // whatever the position: its load would come first
        if (head && c[n].second) qk_load(x + c[n].a1, hi[n]);
    }
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        gain0[n] = qk_fill<V>(1.f); gain1[n] = qk_fill<V>(1.f);
        if (y.gain && c[n].there) gain0[n] = qk_params<V>(y.gain + c[n].a0);
        if (y.gain && c[n].second) gain1[n] = qk_params<V>(y.gain + c[n].a1);
    }
    QkVec<V> xa[NCH], xb[NCH];
    f32x2 ss = make_f32x2(0.f, 0.f);
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        xa[n] = qk_f32<T, V>(lo[n]); xb[n] = qk_f32<T, V>(hi[n]);
        qk_dot<V>(ss, xa[n], xa[n]);
        qk_dot<V>(ss, xb[n], xb[n]);
    }
    const float r = rsqrtf(fmaf(qk_group_sum<G>(sum_f32x2(ss)), 1.f / (float)p.D, p.eps));
    if (pos < 0) return;
    const QkVec<V> rr = qk_fill<V>(r);
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        xa[n] = qk_mul<V>(xa[n], qk_mul<V>(gain0[n], rr));
        xb[n] = qk_mul<V>(xb[n], qk_mul<V>(gain1[n], rr));
        if (c[n].turned) {
            const float* angles = p.table + pos * p.rot + c[n].rot0;
            qk_turn<V>(xa[n], xb[n], qk_params<V>(angles), qk_params<V>(angles + p.rot / 2), p.interleaved);
        }
        if (c[n].there) qk_store<T, V>(out + c[n].a0, xa[n]);
        if (c[n].second) qk_store<T, V>(out + c[n].a1, xb[n]);
    }
}

// CTA = chunk of the positions of one example and one block of heads: blockIdx.x = (queries' blocks x chunks, then the keys'), blockIdx.y =
// example; its warps (up to eight, no more than there are positions) walk positions chunk * warps + warp, step chunks * warps, the next
// position's loads under way while one is worked on.  The threads keep the gain's gradient of their elements in registers.
template <typename T, int V, int NCH, int G>
__global__ void __launch_bounds__(QK_THREADS, NCH * V <= 8 ? 2 : 1)
qknorm_backward_kernel(const __grid_constant__ QkParams p) {
    constexpr int NG = 32 / G;
    extern __shared__ float qk_smem[];                   // [warps][D]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, gl = lane % G, grp = lane / G;
    const int units0 = p.part[0].blocks * p.part[0].chunks;
    const int which = (int)blockIdx.x >= units0;
    const QkPart& y = p.part[which];
    const int unit = (int)blockIdx.x - (which ? units0 : 0), block = unit / y.chunks, chunk = unit - block * y.chunks;
    const int h = block * NG + grp, b = blockIdx.y;
    const bool head = h < y.H;
    QkChunk<V> c[NCH];
    QkVec<V> gain0[NCH], gain1[NCH], acc0[NCH], acc1[NCH];
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        c[n].set(gl + G * n, p.D, p.rot, p.interleaved);
        gain0[n] = qk_fill<V>(1.f); gain1[n] = qk_fill<V>(1.f);
        acc0[n] = qk_fill<V>(0.f); acc1[n] = qk_fill<V>(0.f);
        if (y.gain && c[n].there) gain0[n] = qk_params<V>(y.gain + c[n].a0);
        if (y.gain && c[n].second) gain1[n] = qk_params<V>(y.gain + c[n].a1);
    }
    griddep_launch_dependents();
    const float inv_d = 1.f / (float)p.D;
    const int first = chunk * warps + warp, step = y.chunks * warps;
    const T* x = static_cast<const T*>(y.x) + (long)b * y.xb + (long)first * y.xt + (head ? (long)h * y.xh : 0);
    const T* d = static_cast<const T*>(y.dy) + (long)b * y.yb + (long)first * y.yt + (head ? (long)h * y.yh : 0);
    T* out = static_cast<T*>(y.y) + (long)b * y.ob + (long)first * y.ot + (head ? (long)h * y.oh : 0);
    const long x_inc = (long)step * y.xt, d_inc = (long)step * y.yt, o_inc = (long)step * y.ot;
    auto position = [&](int t) { return t < p.T ? qk_position(p, (uint32_t)b * p.T + t, t) : -1; };
    QkRaw<T, V> xl[NCH], xr[NCH], yl[NCH], yr[NCH];
    auto load = [&](long at) {                           // a padding row counts as zeros, whatever it holds
        const bool live = head && at >= 0;
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            qk_zero(xl[n]); qk_zero(xr[n]); qk_zero(yl[n]); qk_zero(yr[n]);
            if (live && c[n].there) { qk_load(x + c[n].a0, xl[n]); qk_load(d + c[n].a0, yl[n]); }
            if (live && c[n].second) { qk_load(x + c[n].a1, xr[n]); qk_load(d + c[n].a1, yr[n]); }
        }
        x += x_inc; d += d_inc;
    };
    long at = position(first), ahead = position(first + step);
    load(at);
    for (int t = first; t < p.T; t += step) {
        QkVec<V> xa[NCH], xb[NCH], ga[NCH], gb[NCH];
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            xa[n] = qk_f32<T, V>(xl[n]); xb[n] = qk_f32<T, V>(xr[n]);
            ga[n] = qk_f32<T, V>(yl[n]); gb[n] = qk_f32<T, V>(yr[n]);
        }
        const long now = at;
        at = ahead;
        ahead = position(t + 2 * step);
        load(at);
        f32x2 ss = make_f32x2(0.f, 0.f), dots = make_f32x2(0.f, 0.f);
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            if (now >= 0 && c[n].turned) {
                const float* angles = p.table + now * p.rot + c[n].rot0;
                qk_turn<V>(ga[n], gb[n], qk_params<V>(angles), qk_mul<V>(qk_params<V>(angles + p.rot / 2), qk_fill<V>(-1.f)), p.interleaved);
            }
            qk_dot<V>(ss, xa[n], xa[n]);
            qk_dot<V>(ss, xb[n], xb[n]);
            qk_dot<V>(dots, qk_mul<V>(ga[n], gain0[n]), xa[n]);
            qk_dot<V>(dots, qk_mul<V>(gb[n], gain1[n]), xb[n]);
        }
        const float sum = qk_group_sum<G>(sum_f32x2(ss)), dot = qk_group_sum<G>(sum_f32x2(dots));
        // a head that is not there counts as nothing: with eps = 0 the root of its zeros would be infinite
        const float r = now >= 0 && head ? rsqrtf(fmaf(sum, inv_d, p.eps)) : 0.f;
        const QkVec<V> rr = qk_fill<V>(r), m = qk_fill<V>(-(dot * inv_d * r * r * r));   // m: what dx has of x
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            ga[n] = qk_mul<V>(ga[n], rr);
            gb[n] = qk_mul<V>(gb[n], rr);
            acc0[n] = qk_fma<V>(ga[n], xa[n], acc0[n]);
            acc1[n] = qk_fma<V>(gb[n], xb[n], acc1[n]);
            if (now >= 0) {
                if (head && c[n].there) qk_store<T, V>(out + c[n].a0, qk_fma<V>(m, xa[n], qk_mul<V>(ga[n], gain0[n])));
                if (head && c[n].second) qk_store<T, V>(out + c[n].a1, qk_fma<V>(m, xb[n], qk_mul<V>(gb[n], gain1[n])));
            } else {                                     // not what the products say: a gain may be NaN
                if (head && c[n].there) qk_store<T, V>(out + c[n].a0, qk_fill<V>(0.f));
                if (head && c[n].second) qk_store<T, V>(out + c[n].a1, qk_fill<V>(0.f));
            }
        }
        out += o_inc;
    }
    // groups of the warp, then warps, in a fixed order
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        float a[V], e[V];
        qk_floats<V>(acc0[n], a);
        qk_floats<V>(acc1[n], e);
#pragma unroll
        for (int u = 0; u < V; ++u) {
#pragma unroll
            for (int o = G; o < 32; o <<= 1) {
                a[u] += __shfl_xor_sync(0xFFFFFFFFu, a[u], o);
                e[u] += __shfl_xor_sync(0xFFFFFFFFu, e[u], o);
            }
            if (grp == 0 && c[n].there) qk_smem[warp * p.D + c[n].a0 + u] = a[u];
            if (grp == 0 && c[n].second) qk_smem[warp * p.D + c[n].a1 + u] = e[u];
        }
    }
    __syncthreads();
    float* const part = y.part + ((size_t)b * y.blocks * y.chunks + unit) * p.D;
    for (int i = threadIdx.x; i < p.D; i += blockDim.x) {
        float s = 0.f;
        for (int w = 0; w < warps; ++w) s += qk_smem[w * p.D + i];
        part[i] = s;
    }
}

// ------------------------------------------------------------------------------------------------ long calls, V > 1
// The same passes with the loads taken out of the way: every lane copies its own runs of the warp's next tokens into shared memory
// (cp.async, 16 bytes, zero-filled where nothing is read), STAGES - 1 of them ahead, and reads back only what it copied itself, so a warp
// waits for its own copies and for no other warp.  With loads to registers, four heads in flight a group, the forward pass took 38 us where it
// takes 30, the backward pass 135 (113; 103 since its chunks fill whole waves).  A warp stays with one block of heads.
__device__ __forceinline__ void qk_copy16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void qk_copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void qk_copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 qk_lds16(uint32_t addr) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr) : "memory");
    return r;
}

// Tokens of a warp: first, first + step, ... of the batch, with the addresses of one head in two tensors.
struct QkWalk {
    uint32_t token, step;
    int t, dt, T;
    long at, inc, wrap;                  // bytes: of the token, of a step, what an example's end adds to it
    __device__ __forceinline__ QkWalk(uint32_t first, uint32_t step_, int T_, long example, long tok) : token(first), step(step_), T(T_) {
        const int b = (int)(first / (uint32_t)T), db = (int)(step / (uint32_t)T);
        t = (int)(first - (uint32_t)b * T); dt = (int)(step - (uint32_t)db * T);
        at = (long)b * example + (long)t * tok;
        inc = (long)db * example + (long)dt * tok;
        wrap = example - (long)T * tok;
    }
    __device__ __forceinline__ void next() {
        token += step; t += dt; at += inc;
        if (t >= T) { t -= T; at += wrap; }
    }
};
// Positions of a warp's tokens, thirty-two at a time and one batch ahead: lane l holds those of tokens l, 32 + l, ... of the walk.  Without a
// list of positions it is pos0 + t: the launch has moved the table by pos0 then.
struct QkPositions {
    int now, ahead;
    uint32_t at, end, leap, i;           // at: token of this lane in the batch ahead; i: tokens taken
    const int* pos;
    __device__ __forceinline__ int fetch() { const int v = pos && at < end ? __ldg(pos + at) : -1; at += leap; return v; }
    __device__ __forceinline__ QkPositions(const int* pos_, uint32_t first, uint32_t step, uint32_t end_) : end(end_), leap(step * 32), i(0), pos(pos_) {
        at = first + step * (threadIdx.x & 31);
        now = fetch();
        ahead = fetch();
    }
    // of the walk's next token, which is number t of its example; -1: padding
    __device__ __forceinline__ int next(int n_pos, int t) {
        int v = t;
        if (pos) {
            v = __shfl_sync(0xFFFFFFFFu, now, i & 31);
            if ((++i & 31) == 0) { now = ahead; ahead = fetch(); }
        }
        return (uint32_t)v < (uint32_t)n_pos ? v : -1;
    }
};
// (lo, hi) <- the pairs turned; BACK: turned back.  INTER: pairs are neighbours.
template <int V, bool INTER, bool BACK>
__device__ __forceinline__ void qk_turn2(QkVec<V>& lo, QkVec<V>& hi, const QkVec<V>& c, const QkVec<V>& s) {
    if constexpr (!INTER) {
#pragma unroll
        for (int u = 0; u < V / 2; ++u) {
            const f32x2 a = lo.v[u], b = hi.v[u];
            if (BACK) { lo.v[u] = fma2(b, s.v[u], mul2(a, c.v[u])); hi.v[u] = sub2(mul2(b, c.v[u]), mul2(a, s.v[u])); }
            else { lo.v[u] = sub2(mul2(a, c.v[u]), mul2(b, s.v[u])); hi.v[u] = fma2(a, s.v[u], mul2(b, c.v[u])); }
        }
    } else {
        float cs[V], sn[V];
        qk_floats<V>(c, cs);
        qk_floats<V>(s, sn);
#pragma unroll
        for (int u = 0; u < V / 2; ++u) {
            float a, b, d, e;
            split_f32x2(lo.v[u], a, b);
            split_f32x2(hi.v[u], d, e);
            const float s0 = BACK ? -sn[u] : sn[u], s1 = BACK ? -sn[u + V / 2] : sn[u + V / 2];
            lo.v[u] = make_f32x2(fmaf(a, cs[u], -b * s0), fmaf(b, cs[u], a * s0));
            hi.v[u] = make_f32x2(fmaf(d, cs[u + V / 2], -e * s1), fmaf(e, cs[u + V / 2], d * s1));
        }
    }
}
// the angles of a position; lanes whose elements are not turned keep (1, 0)
template <int V> struct QkAngles {
    QkVec<V> c, s;
    __device__ __forceinline__ void load(const char* table, int pos, uint32_t pitch, uint32_t half, bool on) {
        if (on && pos >= 0) {
            const char* a = table + (uint64_t)(uint32_t)pos * pitch;
            c = qk_params<V>(reinterpret_cast<const float*>(a));
            s = qk_params<V>(reinterpret_cast<const float*>(a + half));
        }
    }
};

constexpr int QK_FWD_STAGES = 6, QK_BWD_STAGES = 3;      // backward: 126 us with three, 134 with four, 136 with six (453 MB, before its chunks filled whole waves)

// A warp's walk is over the tokens of the whole batch: blockIdx.x * WARPS + warp, step gridDim.x * WARPS.  Three CTAs an SM leave a thread 80
// registers, and the bf16 forms keep 1 to 23 words of the walks in local memory.
template <typename T, int V, int G, bool INTER>
__global__ void __launch_bounds__(QK_THREADS, 3)
qknorm_forward_ring_kernel(const __grid_constant__ QkParams p) {
    constexpr int NG = 32 / G, WARPS = QK_THREADS / 32, ST = QK_FWD_STAGES;
    __shared__ __align__(16) uint8_t ring[WARPS][ST][2][32 * 16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane % G, grp = lane / G;
    const int which = (int)blockIdx.y >= p.part[0].blocks;
    const QkPart& y = p.part[which];
    const int h = ((int)blockIdx.y - (which ? p.part[0].blocks : 0)) * NG + grp;
    const uint32_t tokens = (uint32_t)p.B * p.T, first = blockIdx.x * WARPS + warp, step = gridDim.x * WARPS;
    if (first >= tokens) return;
    QkChunk<V> c;
    c.set(gl, p.D, p.rot, INTER);
    const bool mine = h < y.H && c.there;
    // addresses of this lane's two runs; the second is `far` bytes behind the first
    const char* const x = reinterpret_cast<const char*>(static_cast<const T*>(y.x) + (mine ? (long)h * y.xh + c.a0 : 0));
    char* const out = reinterpret_cast<char*>(static_cast<T*>(y.y) + (mine ? (long)h * y.oh + c.a0 : 0));
    const int far = mine ? (c.a1 - c.a0) * (int)sizeof(T) : 0;
    QkVec<V> gain0 = qk_fill<V>(1.f), gain1 = gain0;
    if (y.gain && c.there) { gain0 = qk_params<V>(y.gain + c.a0); gain1 = qk_params<V>(y.gain + c.a1); }
    const float inv_d = 1.f / (float)p.D;
    const uint32_t slot0 = (uint32_t)__cvta_generic_to_shared(&ring[warp][0][0][lane * 16]);
    const char* const table = reinterpret_cast<const char*>(p.table + c.rot0);
    const uint32_t pitch = p.rot * 4, half = p.rot * 2;
    const int n_pos = (int)p.n_pos;

    QkPositions where(p.pos, first, step, tokens);
    QkWalk load(first, step, p.T, y.xb * (long)sizeof(T), y.xt * (long)sizeof(T)), use(first, step, p.T, y.ob * (long)sizeof(T), y.ot * (long)sizeof(T));
    int pos[ST];
    auto issue = [&](int s) {
        pos[s] = -1;
        if (load.token < tokens) {
            pos[s] = where.next(n_pos, load.t);
            const bool on = mine && pos[s] >= 0;
            qk_copy16(slot0 + (s * 2 + 0) * 512, x + load.at, on);
            qk_copy16(slot0 + (s * 2 + 1) * 512, x + load.at + far, on);
        }
        qk_copy_commit();
        load.next();
    };
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) issue(s);
    QkAngles<V> ahead;
    ahead.c = qk_fill<V>(1.f); ahead.s = qk_fill<V>(0.f);
    ahead.load(table, pos[0], pitch, half, c.turned);
    while (use.token < tokens) {
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            if (use.token >= tokens) break;
            qk_copy_wait<ST - 2>();
            QkRaw<T, V> lo, hi;
            lo.v = qk_lds16(slot0 + (s * 2 + 0) * 512);
            hi.v = qk_lds16(slot0 + (s * 2 + 1) * 512);
            const int at = pos[s];
            issue((s + ST - 1) % ST);
            QkVec<V> xa = qk_f32<T, V>(lo), xb = qk_f32<T, V>(hi);
            f32x2 ss = make_f32x2(0.f, 0.f);
            qk_dot<V>(ss, xa, xa);
            qk_dot<V>(ss, xb, xb);
            const float r = rsqrtf(fmaf(qk_group_sum<G>(sum_f32x2(ss)), inv_d, p.eps));
            const QkVec<V> rr = qk_fill<V>(r);
            xa = qk_mul<V>(xa, qk_mul<V>(gain0, rr));
            xb = qk_mul<V>(xb, qk_mul<V>(gain1, rr));
            // not turned: c = 1, s = 0 (which an infinity or NaN would not survive unchanged)
            if (c.turned) qk_turn2<V, INTER, false>(xa, xb, ahead.c, ahead.s);
            ahead.load(table, pos[(s + 1) % ST], pitch, half, c.turned);
            if (mine && at >= 0) {
                qk_store<T, V>(reinterpret_cast<T*>(out + use.at), xa);
                qk_store<T, V>(reinterpret_cast<T*>(out + use.at + far), xb);
            }
            use.next();
        }
    }
    qk_copy_wait<0>();
}

// CTA = chunk of the positions of one example and one block of heads: blockIdx.x = (queries' blocks x chunks, then the keys'), blockIdx.y =
// example; a warp walks positions chunk * WARPS + warp, step chunks * WARPS.
template <typename T, int V, int G, bool INTER>
__global__ void __launch_bounds__(QK_THREADS, 2)
qknorm_backward_ring_kernel(const __grid_constant__ QkParams p) {
    constexpr int NG = 32 / G, WARPS = QK_THREADS / 32, ST = QK_BWD_STAGES;
    extern __shared__ __align__(16) uint8_t qk_ring[];   // [WARPS][ST][4][32 * 16], later [WARPS][D] floats over it; [D] gains
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane % G, grp = lane / G;
    const int units0 = p.part[0].blocks * p.part[0].chunks;
    const int which = (int)blockIdx.x >= units0;
    const QkPart& y = p.part[which];
    const int unit = (int)blockIdx.x - (which ? units0 : 0), block = unit / y.chunks, chunk = unit - block * y.chunks;
    const int h = block * NG + grp, b = blockIdx.y;
    QkChunk<V> c;
    c.set(gl, p.D, p.rot, INTER);
    const bool mine = h < y.H && c.there;
    const uint32_t first = chunk * WARPS + warp, step = y.chunks * WARPS, T_ = p.T;
    const char* x = reinterpret_cast<const char*>(static_cast<const T*>(y.x) + (long)b * y.xb + (long)first * y.xt + (mine ? (long)h * y.xh + c.a0 : 0));
    const char* d = reinterpret_cast<const char*>(static_cast<const T*>(y.dy) + (long)b * y.yb + (long)first * y.yt + (mine ? (long)h * y.yh + c.a0 : 0));
    char* out = reinterpret_cast<char*>(static_cast<T*>(y.y) + (long)b * y.ob + (long)first * y.ot + (mine ? (long)h * y.oh + c.a0 : 0));
    const long x_inc = (long)step * y.xt * (long)sizeof(T), d_inc = (long)step * y.yt * (long)sizeof(T), o_inc = (long)step * y.ot * (long)sizeof(T);
    const int far = mine ? (c.a1 - c.a0) * (int)sizeof(T) : 0;
    QkVec<V> acc0 = qk_fill<V>(0.f), acc1 = acc0;
    // the gains stay in shared memory: the sums, a row of each input and the angles fill the registers
    float* const gains = reinterpret_cast<float*>(qk_ring + WARPS * ST * 4 * 512);
    for (int i = threadIdx.x; i < p.D; i += QK_THREADS) gains[i] = y.gain ? y.gain[i] : 1.f;
    __syncthreads();
    const float* const gain_a = gains + (c.there ? c.a0 : 0);
    const float* const gain_b = gains + (c.there ? c.a1 : 0);
    const float inv_d = 1.f / (float)p.D;
    const uint32_t slot0 = (uint32_t)__cvta_generic_to_shared(qk_ring + warp * (ST * 4 * 512) + lane * 16);
    const char* const table = reinterpret_cast<const char*>(p.table + c.rot0);
    const uint32_t pitch = p.rot * 4, half = p.rot * 2;
    const int n_pos = (int)p.n_pos;

    griddep_launch_dependents();
    QkPositions where(p.pos ? p.pos + (long)b * p.T : nullptr, first, step, T_);
    uint32_t t_load = first;
    int pos[ST];
    auto issue = [&](int s) {
        pos[s] = -1;
        if (t_load < T_) {
            pos[s] = where.next(n_pos, (int)t_load);
            const bool on = mine && pos[s] >= 0;          // a padding row counts as zeros, whatever it holds
            qk_copy16(slot0 + (s * 4 + 0) * 512, x, on);
            qk_copy16(slot0 + (s * 4 + 1) * 512, x + far, on);
            qk_copy16(slot0 + (s * 4 + 2) * 512, d, on);
            qk_copy16(slot0 + (s * 4 + 3) * 512, d + far, on);
        }
        qk_copy_commit();
        t_load += step; x += x_inc; d += d_inc;
    };
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) issue(s);
    for (uint32_t t = first; t < T_;) {
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            if (t >= T_) break;
            QkAngles<V> turn;
            turn.c = qk_fill<V>(1.f); turn.s = qk_fill<V>(0.f);
            turn.load(table, pos[s], pitch, half, c.turned);
            qk_copy_wait<ST - 2>();
            QkRaw<T, V> xl, xr, yl, yr;
            yl.v = qk_lds16(slot0 + (s * 4 + 2) * 512);
            yr.v = qk_lds16(slot0 + (s * 4 + 3) * 512);
            xl.v = qk_lds16(slot0 + (s * 4 + 0) * 512);
            xr.v = qk_lds16(slot0 + (s * 4 + 1) * 512);
            const int at = pos[s];
            issue((s + ST - 1) % ST);
            QkVec<V> ga = qk_f32<T, V>(yl), gb = qk_f32<T, V>(yr);
            if (c.turned) qk_turn2<V, INTER, true>(ga, gb, turn.c, turn.s);
            const QkVec<V> xa = qk_f32<T, V>(xl), xb = qk_f32<T, V>(xr);
            f32x2 ss = make_f32x2(0.f, 0.f), dots = make_f32x2(0.f, 0.f);
            qk_dot<V>(ss, xa, xa);
            qk_dot<V>(ss, xb, xb);
            qk_dot<V>(dots, qk_mul<V>(ga, qk_shared<V>(gain_a)), xa);
            qk_dot<V>(dots, qk_mul<V>(gb, qk_shared<V>(gain_b)), xb);
            const float sum = qk_group_sum<G>(sum_f32x2(ss)), dot = qk_group_sum<G>(sum_f32x2(dots));
            // a head that is not there counts as nothing: with eps = 0 the root of its zeros would be infinite
            const float r = at >= 0 && h < y.H ? rsqrtf(fmaf(sum, inv_d, p.eps)) : 0.f;
            const QkVec<V> rr = qk_fill<V>(r), m = qk_fill<V>(-(dot * inv_d * r * r * r));   // m: what dx has of x
            ga = qk_mul<V>(ga, rr);
            gb = qk_mul<V>(gb, rr);
            acc0 = qk_fma<V>(ga, xa, acc0);
            acc1 = qk_fma<V>(gb, xb, acc1);
            if (mine && at >= 0) {
                qk_store<T, V>(reinterpret_cast<T*>(out), qk_fma<V>(m, xa, qk_mul<V>(ga, qk_shared<V>(gain_a))));
                qk_store<T, V>(reinterpret_cast<T*>(out + far), qk_fma<V>(m, xb, qk_mul<V>(gb, qk_shared<V>(gain_b))));
            } else if (mine) {                            // not what the products say: a gain may be NaN
                qk_store<T, V>(reinterpret_cast<T*>(out), qk_fill<V>(0.f));
                qk_store<T, V>(reinterpret_cast<T*>(out + far), qk_fill<V>(0.f));
            }
            t += step; out += o_inc;
        }
    }
    qk_copy_wait<0>();
    __syncthreads();                                      // the sums of the warps go where the ring was
    float* const sums = reinterpret_cast<float*>(qk_ring);
    float a[V], e[V];
    qk_floats<V>(acc0, a);
    qk_floats<V>(acc1, e);
#pragma unroll
    for (int u = 0; u < V; ++u) {
#pragma unroll
        for (int o = G; o < 32; o <<= 1) {
            a[u] += __shfl_xor_sync(0xFFFFFFFFu, a[u], o);
            e[u] += __shfl_xor_sync(0xFFFFFFFFu, e[u], o);
        }
        if (grp == 0 && c.there) { sums[warp * p.D + c.a0 + u] = a[u]; sums[warp * p.D + c.a1 + u] = e[u]; }
    }
    __syncthreads();
    float* const part = y.part + ((size_t)b * y.blocks * y.chunks + unit) * p.D;
    for (int d = threadIdx.x; d < p.D; d += QK_THREADS) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += sums[w * p.D + d];
        part[d] = s;
    }
}

// grads[i][d] = the partial sums in order, sq[i] = the sum of their squares; blockIdx.y = queries, keys.  A CTA an example, or, where the
// examples are many and their partial sums few, a warp.
struct QkFinish { const float* part[2]; int sums[2]; float* grads[2]; float* sq[2]; int B, D; };
template <bool WARP>
__global__ void __launch_bounds__(QK_THREADS)
qknorm_finish_kernel(const __grid_constant__ QkFinish p) {
    __shared__ float red[32];
    griddep_wait();
    griddep_launch_dependents();
    const int i = WARP ? (int)blockIdx.x * (QK_THREADS / 32) + (int)(threadIdx.x >> 5) : (int)blockIdx.x, which = blockIdx.y, sums = p.sums[which];
    if (i >= p.B) return;
    const int first = WARP ? threadIdx.x & 31 : threadIdx.x, step = WARP ? 32 : QK_THREADS;
    float total = 0.f;
    for (int d = first; d < p.D; d += step) {
        const float* src = p.part[which] + (size_t)i * sums * p.D + d;
        float a = 0.f;
#pragma unroll 8
        for (int c = 0; c < sums; ++c) a += src[(size_t)c * p.D];
        if (p.grads[which]) p.grads[which][(size_t)i * p.D + d] = a;
        total = fmaf(a, a, total);
    }
    if (WARP) total = warp_sum(total);
    else total = block_sum(total, red);
    if (first == 0 && p.sq[which]) p.sq[which][i] = total;
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

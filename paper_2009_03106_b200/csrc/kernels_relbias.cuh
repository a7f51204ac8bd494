// Learned relative position bias by buckets: S[h][q][k] += table[bucket(k - q)][h], positions q_offset + q and k.
//
// Everything here depends on the distance k - q alone, so both kernels walk along diagonals.  The plane of (query, key) is cut into
// E x E blocks, E = 8 where rows are 16-byte multiples and 1 elsewhere.  A thread starts at one block and steps to the next on the same
// diagonal: the 2E - 1 distances of its blocks stay the same for the whole walk, so it holds their 2E - 1 values (forward) or sums
// (gradient) in registers, and the lanes of a warp, at neighbouring blocks of one row of blocks, read or write 512 contiguous bytes of each
// row.  A walk that leaves the last block column goes on in the first, where it is on another diagonal: every thread of a tile walks
// equally far.
//
//   relbias_forward_kernel : per 8 x 8 block of bf16 eight 16-byte stores of words that were packed once per walk; bound by the stores.
//   relbias_grad_kernel    : per-example gradient G_i[b][h] = sum over the pairs of bucket b of dL/dS_i[h][q][k].  Per block eight (bf16) or
//                            sixteen 16-byte loads and 64 adds, no atomics; at the end of a walk the 2E - 1 sums go to shared memory, where
//                            they are folded to one sum a distance and then one a bucket, always in the same order.  Bound by the loads:
//                            every element is read once, those behind a length or above the causal diagonal not at all.
//   relbias_finish_kernel  : adds up the tiles of an example and takes the squared norm over buckets and heads.
#pragma once
#include <type_traits>

#include "common.cuh"

namespace dpclip {

constexpr int RB_THREADS = 256;          // forward pass, and gradients whose tiles are wide
constexpr int RB_FEW_THREADS = 64;       // gradients of short rows
constexpr int RB_MAX_BUCKETS = 256;
constexpr int RB_FAR = 1 << 30;

// Distances to buckets.  Per direction `n` buckets: distances below `exact` have one each, those beyond share the others on a
// logarithmic scale; thr[k] is the smallest distance of bucket exact + k.
struct RbBuckets {
    int n_buckets, n, exact, max_distance, bidirectional, causal;
    int top;                                         // the largest power of two below n - exact, or 0
    int thr[RB_MAX_BUCKETS];
    int lo[RB_MAX_BUCKETS], hi[RB_MAX_BUCKETS];      // the distances of every bucket, empty where lo > hi; RB_FAR: no end
};

__host__ __device__ inline int rb_bucket(const RbBuckets& r, long rel) {
    const long lim = r.max_distance;
    const int x = (int)(rel > lim ? lim : rel < -lim ? -lim : rel);      // the last bucket holds everything from max_distance on
    int base = 0, d;
    if (r.bidirectional) { base = x > 0 ? r.n : 0; d = x > 0 ? x : -x; }
    else d = x < 0 ? -x : 0;
    if (d < r.exact) return base + d;
    if (d >= r.max_distance) return base + r.n - 1;
    int lo = 0, hi = r.n - r.exact - 1;                                  // the last k with thr[k] <= d
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (r.thr[mid] <= d) lo = mid; else hi = mid - 1; }
    return base + r.exact + lo;
}

// ------------------------------------------------------------------------------------------------ forward
struct RbForward {
    const float* table; long ldt;
    void* out; long ld, hs;              // row and head stride, elements
    int H, Tq, Tk, nr, nkb, nqb, chunks; // nr block rows a walk
    long off, items;
    RbBuckets r;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void rb_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void rb_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

template <typename T, int E>
__global__ void __launch_bounds__(RB_THREADS, 4)
relbias_forward_kernel(const __grid_constant__ RbForward p) {
    const long item = (long)blockIdx.x * RB_THREADS + threadIdx.x;
    if (item >= p.items) return;
    const int c = (int)(item % p.nkb);
    const long rest = item / p.nkb;
    const int chunk = (int)(rest % p.chunks), h = (int)(rest / p.chunks);
    const int qb0 = chunk * p.nr, steps = min(p.nr, p.nqb - qb0);
    T* const head = static_cast<T*>(p.out) + (long)h * p.hs;
    const float* const column = p.table + h;
    int s = 0, col = c % p.nkb;
    while (s < steps) {
        const int end = min(steps, s + p.nkb - col);
        // v[j]: the bias at distance first + j, the distances of the blocks of this walk
        const long first = (long)E * (col - (qb0 + s)) - p.off - (E - 1);
        float v[2 * E - 1];
        auto value = [&](long rel) {
            return p.r.causal && rel > 0 ? __int_as_float(0xFF800000) : __ldg(column + (long)rb_bucket(p.r, rel) * p.ldt);
        };
        if (E > 1) {
            const long last = first + 2 * E - 2;
            // beyond max_distance on one side there is one bucket, and no search for it
            if (first >= p.r.max_distance || last <= -p.r.max_distance ||
                ((first > 0) == (last > 0) && rb_bucket(p.r, first) == rb_bucket(p.r, last))) {
                const float x = value(first);
#pragma unroll
                for (int j = 0; j < 2 * E - 1; ++j) v[j] = x;
            } else {
                // the searches of all distances side by side: one after the other they are a chain of round trips
                int d[2 * E - 1], k[2 * E - 1];
#pragma unroll
                for (int j = 0; j < 2 * E - 1; ++j) {
                    const long rel = first + j;
                    const int x = (int)(rel > p.r.max_distance ? p.r.max_distance : rel < -(long)p.r.max_distance ? -p.r.max_distance : rel);
                    d[j] = p.r.bidirectional ? abs(x) : max(-x, 0);
                    k[j] = 0;
                }
                for (int s = p.r.top; s > 0; s >>= 1) {
#pragma unroll
                    for (int j = 0; j < 2 * E - 1; ++j)
                        if (k[j] + s < p.r.n - p.r.exact && p.r.thr[k[j] + s] <= d[j]) k[j] += s;
                }
#pragma unroll
                for (int j = 0; j < 2 * E - 1; ++j) {
                    const long rel = first + j;
                    const int b = (p.r.bidirectional && rel > 0 ? p.r.n : 0) + (d[j] < p.r.exact ? d[j] : p.r.exact + k[j]);
                    v[j] = p.r.causal && rel > 0 ? __int_as_float(0xFF800000) : __ldg(column + (long)b * p.ldt);
                }
            }
        } else {
            v[0] = value(first);
        }
        if constexpr (E == 1) {
            const int q_end = min(end, p.Tq - qb0);
            T* at = head + (long)(qb0 + s) * p.ld + col;
#pragma unroll 8
            for (; s < q_end; ++s) { rb_store(at, v[0]); at += p.ld + 1; }
            s = end;
        } else {
            uint32_t w[2 * E - 2];
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int j = 0; j < 2 * E - 2; ++j) w[j] = pack_bf16(v[j], v[j + 1]);
            }
            for (; s < end; ++s, ++col) {
                const int q0 = E * (qb0 + s), k0 = E * col;
                T* at = head + (long)q0 * p.ld + k0;
                const bool full = k0 + E <= p.Tk;
#pragma unroll
                for (int i = 0; i < E; ++i, at += p.ld) {
                    if (q0 + i >= p.Tq) break;
                    if (full) {
                        if constexpr (sizeof(T) == 2) {
                            *reinterpret_cast<uint4*>(at) = make_uint4(w[7 - i], w[9 - i], w[11 - i], w[13 - i]);
                        } else {
                            reinterpret_cast<float4*>(at)[0] = make_float4(v[7 - i], v[8 - i], v[9 - i], v[10 - i]);
                            reinterpret_cast<float4*>(at)[1] = make_float4(v[11 - i], v[12 - i], v[13 - i], v[14 - i]);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < E; ++j) if (k0 + j < p.Tk) rb_store(at + j, v[E - 1 + j - i]);
                    }
                }
            }
        }
        col = 0;
    }
}

// ------------------------------------------------------------------------------------------------ gradient
struct RbGrad {
    const void* dS; long ld, hs, bs;     // row, head and example stride, elements
    int B, H, Tq, Tk, nqb, nkb;          // rows and columns of blocks
    int KT, G, nr, qtiles, ktiles;       // a tile: KT block columns, G groups of nr block rows
    long off;
    const int* q_lens; const int* k_lens;
    float* part;                         // [B * H][qtiles * ktiles][n_buckets]
    RbBuckets r;
};

template <int E>
__host__ __device__ constexpr int rb_smem_floats(int KT, int G, int nr) {
    return (E > 1 ? 2 : 1) * G * E * (KT + nr) + E * (KT + G * nr);
}

// The sums along the 2E - 1 diagonals of a thread's blocks.  E = 8: element (i, j) belongs to diagonal 7 + j - i, and neighbours of a row are
// added as a pair: those of even rows to the pairs that start at odd diagonals, those of odd rows to the ones that start at even diagonals.
template <int E> struct RbSums {
    float s;
    __device__ __forceinline__ void clear() { s = 0.f; }
    __device__ __forceinline__ void write(float* to, int) const { to[0] = s; }
};
template <> struct RbSums<8> {
    f32x2 odd[7], even[7];               // odd[k]: diagonals 2k + 1, 2k + 2;  even[k]: 2k, 2k + 1
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < 7; ++k) odd[k] = even[k] = make_f32x2(0.f, 0.f);
    }
    // elements 2m and 2m + 1 of row i
    template <int I, int M> __device__ __forceinline__ void add(f32x2 x) {
        constexpr int d = 7 + 2 * M - I;
        if constexpr (d & 1) odd[d >> 1] = add2(odd[d >> 1], x);
        else even[d >> 1] = add2(even[d >> 1], x);
    }
    template <int I> __device__ __forceinline__ void add_row(f32x2 a, f32x2 b, f32x2 c, f32x2 d) {
        add<I, 0>(a); add<I, 1>(b); add<I, 2>(c); add<I, 3>(d);
    }
    // diagonals 0 .. 7 to to[0 .. 7], 8 .. 14 to to[other + 8 ..]: neighbours' walks share distances, not places
    __device__ __forceinline__ void write(float* to, int other) const {
        float o[14], e[14], d[16];
#pragma unroll
        for (int k = 0; k < 7; ++k) { split_f32x2(odd[k], o[2 * k], o[2 * k + 1]); split_f32x2(even[k], e[2 * k], e[2 * k + 1]); }
        d[0] = e[0];
#pragma unroll
        for (int k = 1; k < 14; ++k) d[k] = o[k - 1] + e[k];
        d[14] = o[13];
        d[15] = 0.f;
#pragma unroll
        for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(to + k + (k >= 8 ? other : 0)) = make_float4(d[k], d[k + 1], d[k + 2], d[k + 3]);
    }
};
template <typename T> struct RbRow;      // eight elements of a row as loaded
template <> struct RbRow<__nv_bfloat16> {
    uint4 x;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { x = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void pairs(f32x2 (&e)[4]) const {
        e[0] = bf16x2_to_f32x2(x.x); e[1] = bf16x2_to_f32x2(x.y); e[2] = bf16x2_to_f32x2(x.z); e[3] = bf16x2_to_f32x2(x.w);
    }
};
template <> struct RbRow<float> {
    float4 x, y;
    __device__ __forceinline__ void load(const float* p) { x = __ldg(reinterpret_cast<const float4*>(p)); y = __ldg(reinterpret_cast<const float4*>(p) + 1); }
    __device__ __forceinline__ void pairs(f32x2 (&e)[4]) const {
        e[0] = make_f32x2(x.x, x.y); e[1] = make_f32x2(x.z, x.w); e[2] = make_f32x2(y.x, y.y); e[3] = make_f32x2(y.z, y.w);
    }
};

// N rows of a block from row I on, 128 bytes a thread: loaded as one, added as one.
template <typename T> constexpr int RB_ROWS = sizeof(T) == 2 ? 8 : 4;
template <typename T> struct RbRows {
    RbRow<T> x[RB_ROWS<T>];
    __device__ __forceinline__ void load(const T* at, long ld) {
#pragma unroll
        for (int i = 0; i < RB_ROWS<T>; ++i) x[i].load(at + i * ld);
    }
    template <int I> __device__ __forceinline__ void add(RbSums<8>& acc) const {
        f32x2 e[4];
        auto row = [&](auto k) {
            constexpr int i = decltype(k)::value;
            if constexpr (i < RB_ROWS<T>) { x[i].pairs(e); acc.template add_row<I + i>(e[0], e[1], e[2], e[3]); }
        };
        row(std::integral_constant<int, 0>()); row(std::integral_constant<int, 1>()); row(std::integral_constant<int, 2>()); row(std::integral_constant<int, 3>());
        row(std::integral_constant<int, 4>()); row(std::integral_constant<int, 5>()); row(std::integral_constant<int, 6>()); row(std::integral_constant<int, 7>());
    }
};
// n blocks along the diagonal, all of whose elements count: the next 128 bytes are under way while the last are added.
template <typename T>
__device__ __forceinline__ void rb_add_full(const T* at, long ld, int n, RbSums<8>& acc) {
    const long step = 8 * ld + 8;
    RbRows<T> a, b;
    a.load(at, ld);
    if constexpr (sizeof(T) == 2) {
        int i = 0;
        for (; i + 2 <= n; i += 2) {
            b.load(at + step, ld);
            a.template add<0>(acc);
            at += 2 * step;
            if (i + 2 < n) a.load(at, ld);
            b.template add<0>(acc);
        }
        if (i < n) a.template add<0>(acc);
    } else {
        for (int i = 0; i < n; ++i) {
            b.load(at + 4 * ld, ld);
            a.template add<0>(acc);
            at += step;
            if (i + 1 < n) a.load(at, ld);
            b.template add<4>(acc);
        }
    }
}
// Row I of a block at an edge: element j counts when j < cols and j - I <= causal_from.  What does not count may be anything, NaN too, so it
// is left out, not multiplied by zero.
template <typename T, int I>
__device__ __forceinline__ void rb_add_edge_row(const T* row, int rows, int cols, bool can_load, int causal_from, RbSums<8>& acc) {
    if (I >= rows) return;
    float e[8];
    if (can_load) {
        RbRow<T> x;
        f32x2 w[4];
        x.load(row);
        x.pairs(w);
#pragma unroll
        for (int k = 0; k < 4; ++k) split_f32x2(w[k], e[2 * k], e[2 * k + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = j < cols ? to_f32(row[j]) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = j < cols && j - I <= causal_from ? e[j] : 0.f;
    acc.template add_row<I>(make_f32x2(e[0], e[1]), make_f32x2(e[2], e[3]), make_f32x2(e[4], e[5]), make_f32x2(e[6], e[7]));
}
template <typename T>
__device__ __forceinline__ void rb_add_edge(const T* at, long ld, int rows, int cols, bool can_load, RbSums<8>& acc, int causal_from) {
    rb_add_edge_row<T, 0>(at, rows, cols, can_load, causal_from, acc);
    rb_add_edge_row<T, 1>(at + ld, rows, cols, can_load, causal_from, acc);
    rb_add_edge_row<T, 2>(at + 2 * ld, rows, cols, can_load, causal_from, acc);
    rb_add_edge_row<T, 3>(at + 3 * ld, rows, cols, can_load, causal_from, acc);
    rb_add_edge_row<T, 4>(at + 4 * ld, rows, cols, can_load, causal_from, acc);
    rb_add_edge_row<T, 5>(at + 5 * ld, rows, cols, can_load, causal_from, acc);
    rb_add_edge_row<T, 6>(at + 6 * ld, rows, cols, can_load, causal_from, acc);
    rb_add_edge_row<T, 7>(at + 7 * ld, rows, cols, can_load, causal_from, acc);
}

template <typename T, int E, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS)
relbias_grad_kernel(const __grid_constant__ RbGrad p) {
    extern __shared__ __align__(16) float rb_smem[];
    griddep_launch_dependents();
    const int tid = threadIdx.x;
    const int tiles = p.qtiles * p.ktiles;
    const long bh = (long)blockIdx.x / tiles;
    const int tile = (int)((long)blockIdx.x - bh * tiles);
    const int qt = tile / p.ktiles, kt = tile - qt * p.ktiles;
    const int b = (int)(bh / p.H), h = (int)(bh - (long)b * p.H);
    const int ql = p.q_lens ? min(p.Tq, max(0, p.q_lens[b])) : p.Tq, kl = p.k_lens ? min(p.Tk, max(0, p.k_lens[b])) : p.Tk;
    const int qb0 = qt * p.G * p.nr, kb0 = kt * p.KT, ncol = min(p.KT, p.nkb - kb0);
    float* const out = p.part + (size_t)blockIdx.x * p.r.n_buckets;
    // nothing of the tile counts: behind a length, or all keys behind the tile's last query
    const long q_last = min((long)ql, (long)E * (qb0 + p.G * p.nr)) - 1;
    if ((long)E * qb0 >= ql || (long)E * kb0 >= kl || (p.r.causal && (long)E * kb0 > q_last + p.off)) {
        for (int i = tid; i < p.r.n_buckets; i += THREADS) out[i] = 0.f;
        return;
    }
    // sums of the walks by distance, a group at a time: a walk on block diagonal d (from -(nr - 1)) has distances E d .. E d + 2E - 2 of the
    // group's; E > 1: its lower and upper half go to two arrays, where no other walk writes
    const int span = E * (p.KT + p.nr);
    float* const diag = rb_smem;                                        // [E > 1 ? 2 : 1][G][span]
    const int other = p.G * span;
    float* const line = diag + (E > 1 ? 2 : 1) * other;                 // [E * (KT + G * nr)]
    for (int i = tid; i < (E > 1 ? 2 : 1) * other; i += THREADS) diag[i] = 0.f;
    __syncthreads();

    const T* const plane = static_cast<const T*>(p.dS) + (long)b * p.bs + (long)h * p.hs;
    for (int slot = tid; slot < p.G * p.KT; slot += THREADS) {
        const int g = slot / p.KT, c = slot - g * p.KT;
        if (c >= ncol) continue;
        const int row0 = qb0 + g * p.nr;
        const int steps = min(p.nr, (ql + E - 1) / E - row0);
        int s = 0, col = c;
        while (s < steps) {
            const int end = min(steps, s + ncol - col);
            RbSums<E> acc;
            acc.clear();
            const int delta = col - s;                  // block diagonal of the walk, -(nr - 1) .. KT - 1
            // key - query at the blocks' first element
            const long rel = (long)E * ((kb0 + col) - (row0 + s)) - p.off;
            const long causal_from = p.r.causal ? -rel : (long)E;
            if (causal_from > -(long)E) {               // else every pair of the walk is above the diagonal
                const int cf = (int)(causal_from < E ? causal_from : E);
                const T* at = plane + (long)E * (row0 + s) * p.ld + (long)E * (kb0 + col);
                if constexpr (E == 1) {
                    const int n = min(end - s, min(ql - (row0 + s), kl - (kb0 + col)));
#pragma unroll 8
                    for (int i = 0; i < n; ++i) { acc.s += to_f32(*at); at += p.ld + 1; }
                } else {
                    // blocks that are inside the lengths come first on a walk
                    const int full = cf < E - 1 ? 0 : max(0, min(end - s, min(ql / E - (row0 + s), kl / E - (kb0 + col))));
                    if (full > 0) rb_add_full<T>(at, p.ld, full, acc);
                    at += full * ((long)E * p.ld + E);
                    for (int i = s + full; i < end; ++i, at += (long)E * p.ld + E) {
                        const int q0 = E * (row0 + i), k0 = E * (kb0 + col + i - s);
                        if (k0 >= kl) break;
                        rb_add_edge<T>(at, p.ld, ql - q0, kl - k0, k0 + E <= p.Tk, acc, cf);
                    }
                }
            }
            acc.write(diag + g * span + E * (delta + p.nr - 1), other);
            s = end; col = 0;
        }
    }
    __syncthreads();
    // one sum a distance: distance x - (E * (qb0 + G * nr) - 1) + E * kb0 - off
    const int X = E * (p.KT + p.G * p.nr) - 1;
    for (int x = tid; x < X; x += THREADS) {
        float a = 0.f;
        int at = x - E * (p.G - 1) * p.nr;
        for (int g = 0; g < p.G; ++g, at += E * p.nr) {
            if (at < 0 || at >= span) continue;
            a += diag[g * span + at];
            if (E > 1) a += diag[other + g * span + at];
        }
        line[x] = a;
    }
    __syncthreads();
    // eight lanes a bucket
    const long rel0 = (long)E * kb0 - ((long)E * (qb0 + p.G * p.nr) - 1) - p.off;
    const int sub = tid & 7;
    for (int k0 = 0; k0 < p.r.n_buckets; k0 += THREADS / 8) {
        const int k = k0 + (tid >> 3);
        float a = 0.f;
        if (k < p.r.n_buckets) {
            const int lo = p.r.lo[k] == -RB_FAR ? 0 : (int)min(max(p.r.lo[k] - rel0, 0L), (long)X);
            const int hi = p.r.hi[k] == RB_FAR ? X - 1 : (int)max(min(p.r.hi[k] - rel0, (long)X - 1), -1L);
            for (int x = lo + sub; x <= hi; x += 8) a += line[x];
        }
        a += __shfl_xor_sync(0xFFFFFFFFu, a, 1);
        a += __shfl_xor_sync(0xFFFFFFFFu, a, 2);
        a += __shfl_xor_sync(0xFFFFFFFFu, a, 4);
        if (k < p.r.n_buckets && sub == 0) out[k] = a;
    }
}

// G[i][b][h] = (G +) the tiles' sums in order, sq[i] = the sum of its squares.  `lanes` threads (a power of two up to 32) share a sum.
constexpr int RB_FINISH_THREADS = 512;
__global__ void __launch_bounds__(RB_FINISH_THREADS)
relbias_finish_kernel(const float* part, int H, int tiles, int n_buckets, int lanes, int accumulate,
                      float* grads, float* sq) {
    __shared__ float red[32];
    griddep_wait();
    griddep_launch_dependents();
    const int i = blockIdx.x, n = n_buckets * H;
    const int lane = threadIdx.x & (lanes - 1), per = RB_FINISH_THREADS / lanes;
    float* const g = grads + (size_t)i * n;
    float total = 0.f;
    for (int j0 = 0; j0 < n; j0 += per) {
        const int j = j0 + threadIdx.x / lanes;
        float a = 0.f;
        if (j < n) {
            const int k = j / H, h = j - k * H;
            const float* src = part + ((size_t)i * H + h) * tiles * n_buckets + k;
            for (int t = lane; t < tiles; t += lanes) a += src[(size_t)t * n_buckets];
        }
        for (int o = lanes >> 1; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        if (j < n && lane == 0) {
            if (accumulate) a += g[j];
            g[j] = a;
            total = fmaf(a, a, total);
        }
    }
    total = block_sum(total, red);
    if (threadIdx.x == 0) sq[i] = total;
}

}  // namespace dpclip

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
#include "common.cuh"

namespace dpclip {

constexpr int RB_THREADS = 256;
constexpr int RB_MAX_BUCKETS = 256;

// Distances to buckets.  Per direction `n` buckets: distances below `exact` have one each, those beyond share the others on a
// logarithmic scale; thr[k] is the smallest distance of bucket exact + k.
struct RbBuckets {
    int n_buckets, n, exact, max_distance, bidirectional, causal;
    int thr[RB_MAX_BUCKETS];
};

__host__ __device__ inline int rb_bucket(const RbBuckets& r, long rel) {
    const long lim = r.max_distance;
    const int x = (int)(rel > lim ? lim : rel < -lim ? -lim : rel);      // the last bucket holds everything from max_distance on
    int base = 0, d;
    if (r.bidirectional) { base = x > 0 ? r.n : 0; d = x > 0 ? x : -x; }
    else d = x < 0 ? -x : 0;
    if (d < r.exact) return base + d;
    int lo = 0, hi = r.n - r.exact - 1;                                  // the last k with thr[k] <= d
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (r.thr[mid] <= d) lo = mid; else hi = mid - 1; }
    return base + r.exact + lo;
}

// the distances key - query of bucket b: [lo, hi], empty when lo > hi
__device__ __forceinline__ void rb_interval(const RbBuckets& r, int b, long& lo, long& hi) {
    constexpr long FAR = 1L << 40;
    const int side = r.bidirectional && b >= r.n;
    const int c = b - (side ? r.n : 0);
    long dlo, dhi;
    if (c < r.exact) { dlo = c; dhi = c; }
    else { dlo = r.thr[c - r.exact]; dhi = c + 1 < r.n ? (long)r.thr[c - r.exact + 1] - 1 : FAR; }
    if (side) { lo = dlo > 1 ? dlo : 1; hi = dhi; }
    else { lo = -dhi; hi = (!r.bidirectional && c == 0) ? FAR : -dlo; }
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
__global__ void __launch_bounds__(RB_THREADS)
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
            if ((first > 0) == (last > 0) && rb_bucket(p.r, first) == rb_bucket(p.r, last)) {
                const float x = value(first);
#pragma unroll
                for (int j = 0; j < 2 * E - 1; ++j) v[j] = x;
            } else {
#pragma unroll 1
                for (int j = 0; j < 2 * E - 1; ++j) {
                    const float x = value(first + j);
#pragma unroll
                    for (int i = 0; i < 2 * E - 1; ++i) if (i == j) v[i] = x;
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
    return G * (KT + nr - 1) * (2 * E - 1) + E * (KT + G * nr);
}

__device__ __forceinline__ float rb_word(uint32_t w, int half) { return __uint_as_float(half ? w & 0xFFFF0000u : w << 16); }

// Block rows [0, E) x columns [0, E) at `at`: acc[E - 1 + j - i] += element (i, j) where (i, j) counts.
template <typename T, int E>
__device__ __forceinline__ void rb_add_block(const T* at, long ld, int rows, int cols, bool can_load, float (&acc)[2 * E - 1], int causal_from) {
    // element (i, j) counts when i < rows, j < cols and j - i <= causal_from
    if (rows >= E && cols >= E && causal_from >= E - 1) {
        if constexpr (sizeof(T) == 2) {
            uint4 x[E];
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = __ldg(reinterpret_cast<const uint4*>(at + i * ld));
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int j = 0; j < E; ++j) acc[E - 1 + j - i] += rb_word(w[j >> 1], j & 1);
            }
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float4 x[E];
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const float4* row = reinterpret_cast<const float4*>(at + (half * (E / 2) + i) * ld);
                    x[2 * i] = __ldg(row); x[2 * i + 1] = __ldg(row + 1);
                }
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const float e[8] = {x[2 * i].x, x[2 * i].y, x[2 * i].z, x[2 * i].w, x[2 * i + 1].x, x[2 * i + 1].y, x[2 * i + 1].z, x[2 * i + 1].w};
#pragma unroll
                    for (int j = 0; j < E; ++j) acc[E - 1 + j - (half * (E / 2) + i)] += e[j];
                }
            }
        }
        return;
    }
    // an edge: what does not count may be anything, NaN too, so it is left out, not multiplied by zero
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (i >= rows) break;
        const T* row = at + i * ld;
        float e[E];
        if (can_load) {
            if constexpr (sizeof(T) == 2) {
                const uint4 x = __ldg(reinterpret_cast<const uint4*>(row));
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < E; ++j) e[j] = rb_word(w[j >> 1], j & 1);
            } else {
                const float4 x = __ldg(reinterpret_cast<const float4*>(row)), y = __ldg(reinterpret_cast<const float4*>(row) + 1);
                e[0] = x.x; e[1] = x.y; e[2] = x.z; e[3] = x.w; e[4] = y.x; e[5] = y.y; e[6] = y.z; e[7] = y.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) e[j] = j < cols ? to_f32(row[j]) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < E; ++j) acc[E - 1 + j - i] += j < cols && j - i <= causal_from ? e[j] : 0.f;
    }
}

template <typename T, int E>
__global__ void __launch_bounds__(RB_THREADS)
relbias_grad_kernel(const __grid_constant__ RbGrad p) {
    constexpr int W = 2 * E - 1;
    extern __shared__ float rb_smem[];
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
        for (int i = tid; i < p.r.n_buckets; i += RB_THREADS) out[i] = 0.f;
        return;
    }
    const int dpg = p.KT + p.nr - 1;                    // diagonals of blocks a group
    float* const diag = rb_smem;                        // [G][dpg][W]
    float* const line = rb_smem + p.G * dpg * W;        // [E * (KT + G * nr)]
    for (int i = tid; i < p.G * dpg * W; i += RB_THREADS) diag[i] = 0.f;
    __syncthreads();

    const T* const plane = static_cast<const T*>(p.dS) + (long)b * p.bs + (long)h * p.hs;
    for (int slot = tid; slot < p.G * p.KT; slot += RB_THREADS) {
        const int g = slot / p.KT, c = slot - g * p.KT;
        if (c >= ncol) continue;
        const int row0 = qb0 + g * p.nr;
        const int steps = min(p.nr, (ql + E - 1) / E - row0);
        int s = 0, col = c;
        while (s < steps) {
            const int end = min(steps, s + ncol - col);
            float acc[W];
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] = 0.f;
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
                    for (int i = 0; i < n; ++i) { acc[0] += to_f32(*at); at += p.ld + 1; }
                } else {
                    for (int i = s; i < end; ++i, at += (long)E * p.ld + E) {
                        const int q0 = E * (row0 + i), k0 = E * (kb0 + col + i - s);
                        if (k0 >= kl) break;
                        rb_add_block<T, E>(at, p.ld, ql - q0, kl - k0, k0 + E <= p.Tk, acc, cf);
                    }
                }
            }
            float* to = diag + ((size_t)g * dpg + (delta + p.nr - 1)) * W;
#pragma unroll
            for (int j = 0; j < W; ++j) to[j] = acc[j];
            s = end; col = 0;
        }
    }
    __syncthreads();
    // one sum a distance: distance x - (E * (qb0 + G * nr) - 1) + E * kb0 - off
    const int X = E * (p.KT + p.G * p.nr) - 1;
    for (int x = tid; x < X; x += RB_THREADS) {
        float a = 0.f;
        for (int g = 0; g < p.G; ++g) {
            const int y = x - E * (p.G - 1 - g) * p.nr;
            if (y < 0) continue;
            const int d = y / E, e = y - d * E;
            if (d < dpg) a += diag[((size_t)g * dpg + d) * W + e];
            if (e < E - 1 && d >= 1 && d - 1 < dpg) a += diag[((size_t)g * dpg + d - 1) * W + e + E];
        }
        line[x] = a;
    }
    __syncthreads();
    const long rel0 = (long)E * kb0 - ((long)E * (qb0 + p.G * p.nr) - 1) - p.off;
    const int warp = tid >> 5, lane = tid & 31;
    for (int k = warp; k < p.r.n_buckets; k += RB_THREADS / 32) {
        long lo, hi;
        rb_interval(p.r, k, lo, hi);
        lo = max(lo - rel0, 0L); hi = min(hi - rel0, (long)X - 1);
        float a = 0.f;
        for (long x = lo + lane; x <= hi; x += 32) a += line[x];
        a = warp_sum(a);
        if (lane == 0) out[k] = a;
    }
}

// G[i][b][h] = (G +) the tiles' sums in order, sq[i] = the sum of its squares.  `lanes` threads (a power of two up to 32) share a sum.
constexpr int RB_FINISH_THREADS = 512;
__global__ void __launch_bounds__(RB_FINISH_THREADS)
relbias_finish_kernel(const float* __restrict__ part, int H, int tiles, int n_buckets, int lanes, int accumulate,
                      float* __restrict__ grads, float* __restrict__ sq) {
    __shared__ float red[32];
    griddep_wait();
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

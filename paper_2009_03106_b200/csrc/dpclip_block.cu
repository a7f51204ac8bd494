// C ABI of the operators of a transformer block: argument checks, how the work is cut, launches.
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "internal.cuh"
#include "kernels_gated.cuh"
#include "kernels_gated_f32.cuh"
#include "kernels_qknorm.cuh"
#include "kernels_relbias.cuh"
#include "kernels_stored.cuh"

using namespace dpclip;

namespace {

inline size_t elt_size(dpclip_dtype dt) { return dt == DPCLIP_F32 ? 4 : 2; }
inline bool dtype_known(dpclip_dtype dt) { return dt == DPCLIP_F32 || dt == DPCLIP_BF16; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int clamp_int(long v, long lo, long hi) { return (int)(v < lo ? lo : v > hi ? hi : v); }

// ------------------------------------------------------------------------------------------------ relative position bias
// A whole number of up to 128 factors of 25 bits.
struct Whole {
    uint32_t v[104];
    int n;
    Whole() : n(1) { v[0] = 1; }
    void times(uint32_t f, int power) {
        for (int i = 0; i < power; ++i) {
            uint64_t carry = 0;
            for (int j = 0; j < n; ++j) { carry += (uint64_t)v[j] * f; v[j] = (uint32_t)carry; carry >>= 32; }
            if (carry) v[n++] = (uint32_t)carry;
        }
    }
    bool below(const Whole& o) const {
        if (n != o.n) return n < o.n;
        for (int j = n - 1; j >= 0; --j)
            if (v[j] != o.v[j]) return v[j] < o.v[j];
        return false;
    }
};

// thr[k], the smallest distance d of bucket exact + k: floor((n - exact) log(d / exact) / log(max / exact)) >= k, which is
// d >= exact (max / exact)^(k / (n - exact)).  The borders are taken in extended precision, off by less than 1e-16 of themselves; one that
// comes within 1e-15 of a whole number c is decided in whole numbers: c^m >= max^k exact^(m - k), m = n - exact.  A border can miss a whole
// number by little without being one: 50 (2111336 / 50)^(43 / 50) is 475308.0000001.
bool fill_buckets(RbBuckets& r, const dpclip_relbias* c) {
    if (!c || c->n_buckets < 2 || c->n_buckets > RB_MAX_BUCKETS) return false;
    if (c->bidirectional && c->n_buckets % 2) return false;
    memset(&r, 0, sizeof(r));
    r.n_buckets = c->n_buckets;
    r.n = c->bidirectional ? c->n_buckets / 2 : c->n_buckets;
    r.exact = r.n / 2;
    r.max_distance = c->max_distance;
    r.bidirectional = c->bidirectional != 0;
    r.causal = c->causal != 0;
    if (r.exact < 1 || r.max_distance <= r.exact || r.max_distance > (1 << 24)) return false;
    const int m = r.n - r.exact;
    const long double step = powl((long double)r.max_distance / r.exact, 1.0L / m);
    long double border = r.exact;                        // 128 steps at most, each off by 2^-63
    for (int k = 0; k < m; ++k, border *= step) {
        const long double whole = roundl(border);
        r.thr[k] = (int)ceill(border);
        if (k > 0 && fabsl(border - whole) < 1e-15L * border) {
            Whole c, b;
            c.times((uint32_t)whole, m);
            b.times((uint32_t)r.max_distance, k);
            b.times((uint32_t)r.exact, m - k);
            r.thr[k] = (int)whole + (c.below(b) ? 1 : 0);
        }
    }
    r.top = m > 1 ? 1 : 0;
    while (m > 1 && 2 * r.top < m) r.top *= 2;
    for (int b = 0; b < r.n_buckets; ++b) {
        const int side = r.bidirectional && b >= r.n, c = b - (side ? r.n : 0);
        const int from = c < r.exact ? c : r.thr[c - r.exact];
        const int to = c < r.exact ? c : c + 1 < r.n ? r.thr[c - r.exact + 1] - 1 : RB_FAR;
        r.lo[b] = side ? (from > 1 ? from : 1) : -to;
        r.hi[b] = side ? to : (!r.bidirectional && c == 0 ? RB_FAR : -from);
    }
    return true;
}

// A tile of the gradient: G groups of nr block rows by KT block columns.  64 threads where the rows have at most 64 blocks: a walk of such a
// tile is then long enough to pay for the folds behind it (128 examples, 8 heads, 256 x 256, bf16: 40 us, 256 threads 48).
struct RbTiles { int E, threads, nqb, nkb, KT, G, nr, qtiles, ktiles; };
RbTiles relbias_tiles(int B, int H, int Tq, int Tk, bool blocks8) {
    RbTiles t;
    t.E = blocks8 ? 8 : 1;
    t.nqb = ceil_div(Tq, t.E); t.nkb = ceil_div(Tk, t.E);
    t.threads = t.nkb <= RB_FEW_THREADS ? RB_FEW_THREADS : RB_THREADS;
    const int most = blocks8 ? RB_THREADS : 4 * RB_THREADS;       // four walks a thread where a walk has one sum
    t.KT = t.nkb < most ? t.nkb : most;
    t.ktiles = ceil_div(t.nkb, t.KT);
    t.G = t.threads / t.KT;
    if (t.G < 1) t.G = 1;
    if (t.G > t.nqb) t.G = t.nqb;
    // One wave of the CTAs that fit on the SMs side by side, their walks as long as that allows: a walk's end costs as much as eight blocks of
    // it.  40 KB of shared memory hold the sums; walks over single elements are at least eight long.
    const long resident = (long)kNumSMs * (blocks8 ? 512 : 1024) / t.threads, planes = (long)B * H * t.ktiles;
    const long rows = resident / planes > 0 ? resident / planes : 1;
    const int longest = blocks8 ? 32 : 128;
    auto fits = [&](int nr) { return (blocks8 ? rb_smem_floats<8>(t.KT, t.G, nr) : rb_smem_floats<1>(t.KT, t.G, nr)) * sizeof(float) <= 40 * 1024; };
    t.nr = clamp_int(ceil_div(t.nqb, t.G * rows), 1, longest);
    if (!blocks8 && t.nr < 8) t.nr = 8;
    while (t.nr > 1 && !fits(t.nr)) t.nr = (t.nr + 1) / 2;
    t.qtiles = ceil_div(t.nqb, (long)t.G * t.nr);
    return t;
}
inline size_t relbias_part_bytes(const RbTiles& t, int B, int H, int n_buckets) {
    return sizeof(float) * (size_t)B * H * t.qtiles * t.ktiles * n_buckets;
}

template <typename T, int E>
int launch_relbias_forward(RbForward& p, cudaStream_t st) {
    p.nqb = ceil_div(p.Tq, E); p.nkb = ceil_div(p.Tk, E);
    // a walk of several block rows pays for its look-ups; one wave of four CTAs an SM
    const long blocks = (long)p.nqb * p.nkb * p.H;
    p.nr = clamp_int((blocks + kNumSMs * 4L * RB_THREADS - 1) / (kNumSMs * 4L * RB_THREADS), 1, E == 1 ? 64 : 32);
    if (p.nr > p.nqb) p.nr = p.nqb;
    p.chunks = ceil_div(p.nqb, p.nr);
    p.items = (long)p.H * p.chunks * p.nkb;
    const long grid = (p.items + RB_THREADS - 1) / RB_THREADS;
    if (grid > 0x7FFFFFFFL) return DPCLIP_ERR_UNSUPPORTED;
    relbias_forward_kernel<T, E><<<(unsigned)grid, RB_THREADS, 0, st>>>(p);
    return finish_launch();
}

template <typename T, int E>
int launch_relbias_grad(const RbGrad& p, int threads, cudaStream_t st) {
    const int smem = rb_smem_floats<E>(p.KT, p.G, p.nr) * (int)sizeof(float);
    const unsigned grid = (unsigned)((long)p.B * p.H * p.qtiles * p.ktiles);
    if (threads == RB_THREADS) relbias_grad_kernel<T, E, RB_THREADS><<<grid, RB_THREADS, smem, st>>>(p);
    else relbias_grad_kernel<T, E, RB_FEW_THREADS><<<grid, RB_FEW_THREADS, smem, st>>>(p);
    return finish_launch();
}

// ------------------------------------------------------------------------------------------------ norms of queries and keys
struct QkShape { int V, NCH, G; };        // elements a run, chunks a lane, lanes a head
bool qk_shape(QkShape& s, int D, int rot, bool vec, dpclip_dtype dtype) {
    const int v = dtype == DPCLIP_F32 ? 4 : 8;
    if (vec && D % (2 * v) == 0 && rot % (2 * v) == 0 && D / (2 * v) <= 32) {
        s.V = v; s.NCH = 1; s.G = 1;
        while (s.G < D / (2 * v)) s.G *= 2;
        return true;
    }
    // four pairs a lane where that fills the lanes of a head: shorter sums across lanes and several heads a warp
    s.V = 1;
    const int pairs = (D + 1) / 2;
    s.NCH = pairs <= 128 ? 4 : 8;
    s.G = pairs <= 32 ? 8 : pairs <= 64 ? 16 : 32;
    return pairs <= 256;
}

// Calls of so many warp items (a token's block of heads) keep a ring of copies going in every warp; shorter ones are a chain of round trips
// and take one item a warp.  Heads of 64 in bf16, backward, with rings and without: 221 items an SM 22.8 and 30.8 us, 111 14.5 and 16.9, 55
// 12.3 and 12.5, 28 10.3 both; forward 16.5 and 18.5 at 221, no difference at 111 and below, but in fp32 at 28 6.2 and 4.4.
constexpr long kQkRingItems = 64L * kNumSMs;

// The ring kernels' positions are 32-bit numbers: of the list, or t against a table moved by pos0.
inline void qk_move_table(QkParams& p) {
    if (!p.pos) {
        const long first = p.pos0 < p.n_pos ? p.pos0 : p.n_pos;
        if (p.table) p.table += first * p.rot;
        p.n_pos -= first;
    }
    if (p.n_pos > 0x7FFFFFFFL) p.n_pos = 0x7FFFFFFFL;
}

template <typename T, int V, int NCH, int G>
int launch_qk_forward(QkParams& p, cudaStream_t st) {
    for (int k = 0; k < 2; ++k) p.part[k].blocks = ceil_div(p.part[k].H, 32 / G);
    const long blocks = p.part[0].blocks + p.part[1].blocks, tokens = (long)p.B * p.T;
    constexpr int WARPS = QK_THREADS / 32;
    if (blocks > 65535) return DPCLIP_ERR_UNSUPPORTED;
    if constexpr (V > 1) {
        if (tokens * blocks >= kQkRingItems) {
            // one wave of three CTAs an SM, every warp with as many tokens as any other
            long x = 3L * kNumSMs / blocks;
            if (x < 1) x = 1;
            if (x > (tokens + WARPS - 1) / WARPS) x = (tokens + WARPS - 1) / WARPS;
            const dim3 grid((unsigned)x, (unsigned)blocks);
            qk_move_table(p);
            if (p.interleaved) qknorm_forward_ring_kernel<T, V, G, true><<<grid, QK_THREADS, 0, st>>>(p);
            else qknorm_forward_ring_kernel<T, V, G, false><<<grid, QK_THREADS, 0, st>>>(p);
            return finish_launch();
        }
    }
    const dim3 grid((unsigned)((tokens + WARPS - 1) / WARPS), (unsigned)blocks);
    qknorm_forward_kernel<T, V, NCH, G><<<grid, QK_THREADS, 0, st>>>(p);
    return finish_launch();
}
// Whether the backward pass of this shape keeps a ring of copies (its CTAs then have a block of heads each).
inline bool qk_ring_backward(const QkShape& s, int B, int T, const QkPart* part) {
    return s.V > 1 && T >= QK_THREADS / 32 * 4 && (long)B * T * (part[0].blocks + part[1].blocks) >= kQkRingItems;
}
template <typename T, int V, int NCH, int G>
int launch_qk_backward(QkParams& p, bool ring, cudaStream_t st) {
    constexpr int WARPS = QK_THREADS / 32;
    if constexpr (V > 1) {
        if (ring) {
            const int smem = WARPS * QK_BWD_STAGES * 4 * 512 + (int)sizeof(float) * p.D;      // 48 KB and the gains; the sums, at most 16 KB, take the ring's place
            const auto kernel = p.interleaved ? qknorm_backward_ring_kernel<T, V, G, true> : qknorm_backward_ring_kernel<T, V, G, false>;
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return DPCLIP_ERR_CUDA;
            const dim3 grid(p.part[0].blocks * p.part[0].chunks + p.part[1].blocks * p.part[1].chunks, p.B);
            qk_move_table(p);
            kernel<<<grid, QK_THREADS, smem, st>>>(p);
            return finish_launch();
        }
    }
    const int warps = p.T < WARPS ? p.T : WARPS;
    const dim3 grid(p.part[0].blocks * p.part[0].chunks + p.part[1].blocks * p.part[1].chunks, p.B);
    qknorm_backward_kernel<T, V, NCH, G><<<grid, 32 * warps, sizeof(float) * warps * p.D, st>>>(p);
    return finish_launch();
}
template <typename T>
int launch_qk(QkParams& p, const QkShape& s, bool backward, bool ring, cudaStream_t st) {
    constexpr int VV = sizeof(T) == 4 ? 4 : 8;
#define DPCLIP_QK(V, NCH, G) return backward ? launch_qk_backward<T, V, NCH, G>(p, ring, st) : launch_qk_forward<T, V, NCH, G>(p, st)
    if (s.V == 1) {
        if (s.NCH == 8) DPCLIP_QK(1, 8, 32);
        switch (s.G) { case 8: DPCLIP_QK(1, 4, 8); case 16: DPCLIP_QK(1, 4, 16); default: DPCLIP_QK(1, 4, 32); }
    }
    switch (s.G) {
        case 1: DPCLIP_QK(VV, 1, 1); case 2: DPCLIP_QK(VV, 1, 2); case 4: DPCLIP_QK(VV, 1, 4);
        case 8: DPCLIP_QK(VV, 1, 8); case 16: DPCLIP_QK(VV, 1, 16); default: DPCLIP_QK(VV, 1, 32);
    }
#undef DPCLIP_QK
}

// Chunks of positions a block of heads is cut into.  Two CTAs stand on an SM; a CTA's time is about 6 us and 0.18 us a position (its eight
// warps take one each), a call's that of its waves: the fewest chunks of the least such time.  (128 examples, five blocks of heads, 256 positions:
// 124 us in one chunk, which is 2.2 waves, 111 in two; 4 examples, six blocks, 2000 positions: 51 us in 24 chunks, 45 in 12, which are one wave.)
constexpr long kQkResident = 2L * kNumSMs;
inline int qk_most_chunks(int B, int T, int blocks) {
    const long most = 4 * kQkResident / ((long)B * blocks) + 1, least = T / 16 > 0 ? T / 16 : 1;
    return (int)(most < least ? most : least);
}
inline int qk_chunks(int B, int T, int blocks) {
    int best = 1;
    double least = 1e30;
    for (int c = 1; c <= qk_most_chunks(B, T, blocks); ++c) {
        const double time = (double)(((long)B * blocks * c + kQkResident - 1) / kQkResident) * (6.0 + 0.18 * T / c);
        if (time < least) { least = time; best = c; }
    }
    return best;
}
// most partial sums an example any form of the kernels makes, for the workspace: blocks * chunks, with at most H blocks
inline long qk_most_sums(int B, int T, int H) {
    if (H <= 0) return 0;
    const long by_waves = 4 * kQkResident / B + H, by_length = (long)H * (T / 16 > 0 ? T / 16 : 1);
    return by_waves < by_length ? by_waves : by_length;
}

int qk_check(const dpclip_heads* parts, int n_parts, int B, int T, int D, int rot_dim, const float* table, long n_pos,
             const int* positions, long pos0, float eps, dpclip_dtype dtype, bool backward) {
    if (!parts || n_parts < 1 || n_parts > 2 || B <= 0 || T <= 0 || D <= 0 || !dtype_known(dtype)) return DPCLIP_ERR_INVALID_ARG;
    if (rot_dim < 0 || rot_dim > D || rot_dim % 2 || !(eps >= 0.f) || n_pos <= 0) return DPCLIP_ERR_INVALID_ARG;
    if ((rot_dim > 0 && !table) || (!positions && pos0 < 0)) return DPCLIP_ERR_INVALID_ARG;
    if ((long)B * T > 0x7FFF0000L || D > 512 || (backward && B > 65535)) return DPCLIP_ERR_UNSUPPORTED;
    const size_t es = elt_size(dtype);
    for (int k = 0; k < n_parts; ++k) {
        const dpclip_heads& h = parts[k];
        if (!h.x || !h.out || (backward && !h.dy) || h.H <= 0) return DPCLIP_ERR_INVALID_ARG;
        if (!is_aligned(h.x, es) || !is_aligned(h.out, es) || (h.dy && !is_aligned(h.dy, es)) || (h.gain && !is_aligned(h.gain, 4)))
            return DPCLIP_ERR_MISALIGNED;
    }
    if ((table && !is_aligned(table, 4)) || (positions && !is_aligned(positions, 4))) return DPCLIP_ERR_MISALIGNED;
    return DPCLIP_OK;
}

// fills p; whether every run of V elements is a 16-byte load
bool qk_fill(QkParams& p, const dpclip_heads* parts, int n_parts, int B, int T, int D, int rot_dim, int interleaved, const float* table,
             long n_pos, const int* positions, long pos0, float eps, dpclip_dtype dtype, bool backward) {
    memset(&p, 0, sizeof(p));
    p.B = B; p.T = T; p.D = D; p.rot = rot_dim; p.interleaved = interleaved != 0;
    p.n_pos = n_pos; p.pos0 = pos0; p.pos = positions; p.table = table; p.eps = eps;
    const long v = dtype == DPCLIP_F32 ? 4 : 8;
    bool vec = !table || is_aligned(table, 16);
    for (int k = 0; k < n_parts; ++k) {
        const dpclip_heads& h = parts[k];
        QkPart& q = p.part[k];
        q.x = h.x; q.xb = h.x_example; q.xt = h.x_token; q.xh = h.x_head;
        q.y = h.out; q.ob = h.out_example; q.ot = h.out_token; q.oh = h.out_head;
        q.dy = h.dy; q.yb = h.dy_example; q.yt = h.dy_token; q.yh = h.dy_head;
        q.gain = h.gain; q.H = h.H;
        // an extent of one: its stride is never used
        if (B == 1) q.xb = q.ob = q.yb = 0;
        if (T == 1) q.xt = q.ot = q.yt = 0;
        if (h.H == 1) q.xh = q.oh = q.yh = 0;
        vec = vec && is_aligned(h.x, 16) && is_aligned(h.out, 16) && (!h.gain || is_aligned(h.gain, 16));
        vec = vec && (q.xb | q.xt | q.xh | q.ob | q.ot | q.oh) % v == 0;
        if (backward) vec = vec && is_aligned(h.dy, 16) && (q.yb | q.yt | q.yh) % v == 0;
    }
    return vec;
}

// ------------------------------------------------------------------------------------------------ gated feed-forward block
constexpr int kPairs = kNumSMs / 2;

// Tile width and split of a product of M rows, `cols` columns (of h, or of dx) and KD contracted, on CTA pairs.  Counted in stages of a
// 256-column tile (64 of the contraction, 0.28 us): waves of tiles, each as many stages as its part of the contraction and six for filling the
// pipeline and the last tile's epilogue; a 128-column tile's stage costs 0.6 of it (A is loaded for half the columns); splitting costs a launch
// and the partial products' way to memory and back.  A split's own cost of 4 stages was chosen on ten shapes of 130 to 2000 rows: with 0 dX of 257 x
// 1301 -> 460 takes 20.6 us for 18.5, with 20 304 x 4096 -> 1024 23.8 for 20.7 and 600 x 520 -> 500 in fp32 21.6 for 18.6, the others the same.
struct GatedCut { int hn, splits, kb_per_split; };
// fp32: a stage is six products.
GatedCut gated_cut(long M, long cols, long KD, bool fwd, bool f32) {
    const int KB = ceil_div(KD, tc::gt::BK);
    GatedCut best = {128, 1, KB};
    double least = 1e30;
    for (int hn = 64; hn <= 128; hn *= 2)
        for (int s = 1; s <= 32; ++s) {
            if (s > 1 && KB < (f32 ? 2 : 4) * s) break;
            const long tiles = (long)ceil_div(M, 256) * ceil_div(cols, fwd ? hn : 2 * hn);
            if (s > 1 && tiles * s > 2 * kPairs) break;
            const int per = ceil_div(KB, s);
            double cost = (double)((tiles * s + kPairs - 1) / kPairs) * (per * (hn == 128 ? 1.0 : 0.6) * (f32 ? 6 : 1) + (f32 ? 12 : 6));
            if (s > 1) cost += 4 + (double)M * cols * (fwd ? 2 : 1) * 4 * (s + 1) / 5e6 / 0.28;
            if (cost < least) { least = cost; best = {hn, ceil_div(KB, per), per}; }
        }
    return best;
}
// Split of the same product on the fp32 ALUs: two CTAs an SM, at least 128 contracted each.
inline int gated_simt_rows(long M) { return M <= 64 ? 32 : 128; }
inline int gated_simt_splits(long M, long cols, long KD, bool fwd) {
    const long tiles = (long)ceil_div(M, gated_simt_rows(M)) * ceil_div(cols, fwd ? 64 : 128);
    return clamp_int(2L * kNumSMs / tiles, 1, clamp_int(KD / 128, 1, 32));
}
inline bool gated_rows_ok(const void* p, long ld) { return is_aligned(p, 16) && ld % 8 == 0; }
// bf16 rows that TMA cannot address are copied above this many rows.  The fp32 ALUs take as long at the least and far longer at most sizes (all
// operands off, forward / backward: 9 x 64 -> 72 8.4 / 21 us, with copies 8.7 / 12; 9 x 2000 -> 5000 84 / 86, 35 / 35; 16384 x 512 -> 2048
// 1760 / 2360, 75 / 180); up to eight rows have a forward kernel of their own, and their workspace would be as large as the weights.
constexpr int kGatedCopyRows = 8;
inline long up8(long n) { return (n + 7) / 8 * 8; }
// fp32 on the tensor cores: from here on the ALUs' 4 M K F at 32 TFLOP/s take longer than three launches and the planes' way to memory
inline bool gated_planes(long M, long K, long F) { return M > 32 && (double)M * K * F > 6e7; }
struct GatedSpace { size_t part, copy_a, copy_w; };       // bytes: partial products; copies (fp32: planes) of an operand of M rows and of W
GatedSpace gated_space(long M, long K, long F, dpclip_dtype dtype, bool fwd) {
    const long cols = fwd ? F : K, KD = fwd ? K : 2 * F, width = fwd ? 2 * F : K;
    const int simt = gated_simt_splits(M, cols, KD, fwd), tensor = gated_cut(M, cols, KD, fwd, dtype == DPCLIP_F32).splits;
    const int s = simt > tensor ? simt : tensor;
    GatedSpace g = {s > 1 ? round_up(sizeof(float) * (size_t)s * M * width, 256) : 0, 0, 0};
    // bf16: whether rows have to be copied depends on addresses and strides, which the size of a workspace does not know
    const size_t planes = dtype == DPCLIP_F32 ? (gated_planes(M, K, F) ? 3 : 0) : M > kGatedCopyRows ? 1 : 0;
    g.copy_a = planes * round_up(2 * (size_t)M * up8(KD), 256);
    g.copy_w = planes * round_up(2 * (size_t)2 * F * up8(K), 256);
    return g;
}
inline size_t total_bytes(const GatedSpace& g) { return g.part + g.copy_a + g.copy_w; }

// copies of up to two matrices in one launch; none: nothing
int gated_copies(const GatedCopy* c, int n_copies, cudaStream_t st) {
    if (n_copies == 0) return DPCLIP_OK;
    GatedCopies p;
    memset(&p, 0, sizeof(p));
    long n = 0;
    for (int k = 0; k < n_copies; ++k) { p.c[k] = c[k]; n += c[k].rows * ((c[k].cols + 7) / 8); if (k == 0) p.first = n; }
    gated_copy_kernel<<<clamp_int((n + 255) / 256, 1, kNumSMs * 16), 256, 0, st>>>(p, n);
    return finish_launch();
}

template <typename T, bool FWD>
int launch_gated_reduce(const GatedOut& o, cudaStream_t st) {
    const long n = (long)o.M * o.F;
    return launch_after(gated_reduce_kernel<T, FWD>, dim3(clamp_int((n + 255) / 256, 1, kNumSMs * 8)), 256, 0, st, o);
}

template <typename T, bool FWD>
int launch_gated_simt(GatedSimt& p, cudaStream_t st) {
    const int bm = gated_simt_rows(p.M), splits = gated_simt_splits(p.M, p.N, p.KD, FWD);
    p.tiles_n = ceil_div(p.N, FWD ? 64 : 128);
    p.k_per_split = (int)round_up(ceil_div(p.KD, splits), 16);
    p.out.splits = ceil_div(p.KD, p.k_per_split);
    const long tiles = (long)ceil_div(p.M, bm) * p.tiles_n;
    if (tiles > 0x7FFFFFFFL) return DPCLIP_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)tiles, p.out.splits);
    if (bm == 32) gated_simt_kernel<T, FWD, 32><<<grid, 256, 0, st>>>(p);
    else gated_simt_kernel<T, FWD, 128><<<grid, 256, 0, st>>>(p);
    const int rc = finish_launch();
    return rc || p.out.splits == 1 ? rc : launch_gated_reduce<T, FWD>(p.out, st);
}

template <typename T, int V, int MT>
int launch_gated_few(const GatedFew& p, cudaStream_t st) {
    gated_few_kernel<T, V, MT><<<ceil_div(p.out.F, 4), 128, 0, st>>>(p);
    return finish_launch();
}
template <typename T, int V>
int launch_gated_few(const GatedFew& p, cudaStream_t st) {
    const int M = p.out.M;
    return M == 1 ? launch_gated_few<T, V, 1>(p, st) : M == 2 ? launch_gated_few<T, V, 2>(p, st)
         : M <= 4 ? launch_gated_few<T, V, 4>(p, st) : launch_gated_few<T, V, 8>(p, st);
}

template <bool FWD, bool KEEP, int HN>
int launch_gated_tc(const tc::gt::Maps& maps, const tc::gt::Params& p, cudaStream_t st) {
    using C = tc::gt::Cfg<FWD, KEEP, HN>;
    if (cudaFuncSetAttribute(tc::gated_tc_kernel<FWD, KEEP, HN>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES) != cudaSuccess)
        return DPCLIP_ERR_CUDA;
    const int pairs = p.total < kPairs ? p.total : kPairs;
    const int rc = launch_after(tc::gated_tc_kernel<FWD, KEEP, HN>, dim3(2 * pairs), C::THREADS, C::SMEM_BYTES, st, maps, p);
    return rc || p.out.splits == 1 ? rc : launch_gated_reduce<__nv_bfloat16, FWD>(p.out, st);
}
// a [M][KD] (lda), w [2F][K] (ldw): rows TMA can address
int gated_tensor(bool fwd, const void* a, long lda, const void* w, long ldw, int M, int K, int F, GatedOut out, int* status, cudaStream_t st) {
    using namespace tc::gt;
    const int KD = fwd ? K : 2 * F, cols = fwd ? F : K;
    const GatedCut cut = gated_cut(M, cols, KD, fwd, false);
    Params p;
    memset(&p, 0, sizeof(p));
    p.KB = ceil_div(KD, BK);
    p.kb_per_split = cut.kb_per_split;
    p.tiles_m = ceil_div(M, 256); p.tiles_n = ceil_div(cols, fwd ? cut.hn : 2 * cut.hn);
    const long total = (long)p.tiles_m * p.tiles_n * cut.splits;
    if (total > 0x3FFFFFFFL) return DPCLIP_ERR_UNSUPPORTED;
    p.total = (int)total;
    p.status = status; p.out = out; p.out.splits = cut.splits;
    const bool keep = fwd && out.z && cut.splits == 1;
    // a store writes whole 16-byte units of a row: rows that end inside one would lose what lies behind them
    p.tma_out = cols % 8 == 0 && gated_rows_ok(out.h, out.ldh) && (!keep || gated_rows_ok(out.z, out.ldz));
    Maps maps;
    memset(&maps, 0, sizeof(maps));
    const __nv_bfloat16* wb = static_cast<const __nv_bfloat16*>(w);
    bool ok = encode_map_bf16(&maps.a, a, M, KD, lda, 64, BM_CTA);
    if (fwd) ok = ok && encode_map_bf16(&maps.b[0], wb, F, K, ldw, 64, cut.hn) && encode_map_bf16(&maps.b[1], wb + (long)F * ldw, F, K, ldw, 64, cut.hn);
    else ok = ok && encode_map_bf16(&maps.b[0], wb, 2L * F, K, ldw, 64, BK) && encode_map_bf16(&maps.b[1], wb, 2L * F, K, ldw, 64, BK);
    if (p.tma_out && cut.splits == 1) {
        ok = ok && encode_map_bf16(&maps.h, out.h, M, cols, out.ldh, 64, 32);
        if (keep) {
            __nv_bfloat16* z = static_cast<__nv_bfloat16*>(out.z);
            ok = ok && encode_map_bf16(&maps.z[0], z, M, F, out.ldz, 64, 32) && encode_map_bf16(&maps.z[1], z + F, M, F, out.ldz, 64, 32);
        }
    }
    if (!ok) return DPCLIP_ERR_CUDA;
    if (!fwd) return cut.hn == 128 ? launch_gated_tc<false, false, 128>(maps, p, st) : launch_gated_tc<false, false, 64>(maps, p, st);
    if (keep) return cut.hn == 128 ? launch_gated_tc<true, true, 128>(maps, p, st) : launch_gated_tc<true, true, 64>(maps, p, st);
    return cut.hn == 128 ? launch_gated_tc<true, false, 128>(maps, p, st) : launch_gated_tc<true, false, 64>(maps, p, st);
}

int gated_splits(const GatedSplit* c, int n_splits, cudaStream_t st) {
    GatedSplits p;
    memset(&p, 0, sizeof(p));
    long n = 0;
    for (int k = 0; k < n_splits; ++k) {
        p.c[k] = c[k];
        p.c[k].vec = is_aligned(c[k].src, 16) && c[k].ld % 4 == 0 && c[k].cols % 4 == 0;
        n += c[k].rows * ((c[k].cols + 3) / 4);
        if (k == 0) p.first = n;
    }
    gated_split_kernel<<<clamp_int((n + 255) / 256, 1, kNumSMs * 16), 256, 0, st>>>(p, n);
    return finish_launch();
}
template <bool FWD, int HN>
int launch_gated_tc3(const tc::gt3::Maps& maps, const tc::gt3::Params& p, cudaStream_t st) {
    using C = tc::gt3::Cfg<HN>;
    if (cudaFuncSetAttribute(tc::gated_tc3_kernel<FWD, HN>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES) != cudaSuccess)
        return DPCLIP_ERR_CUDA;
    const int pairs = p.total < kPairs ? p.total : kPairs;
    const int rc = launch_after(tc::gated_tc3_kernel<FWD, HN>, dim3(2 * pairs), tc::gt3::THREADS, C::SMEM_BYTES, st, maps, p);
    return rc || p.out.splits == 1 ? rc : launch_gated_reduce<float, FWD>(p.out, st);
}
// The product of a [M][KD] and w [2F][K], whose planes lie in the workspace behind the partial products.
int gated_tensor_f32(bool fwd, const float* a, long lda, const float* w, long ldw, int M, int K, int F, GatedOut out, uint8_t* ws,
                     const GatedSpace& space, int* status, cudaStream_t st) {
    using namespace tc::gt3;
    const int KD = fwd ? K : 2 * F, cols = fwd ? F : K;
    const GatedCut cut = gated_cut(M, cols, KD, fwd, true);
    uint8_t* const pa = ws + space.part, *const pw = pa + space.copy_a;
    const size_t plane_a = space.copy_a / 3, plane_w = space.copy_w / 3;
    Params p;
    memset(&p, 0, sizeof(p));
    p.KB = ceil_div(KD, BK);
    p.kb_per_split = cut.kb_per_split;
    p.tiles_m = ceil_div(M, 256); p.tiles_n = ceil_div(cols, fwd ? cut.hn : 2 * cut.hn);
    const long total = (long)p.tiles_m * p.tiles_n * cut.splits;
    if (total > 0x3FFFFFFFL) return DPCLIP_ERR_UNSUPPORTED;
    p.total = (int)total;
    p.status = status; p.out = out; p.out.splits = cut.splits;
    p.a = a; p.lda = lda; p.w = w; p.ldw = ldw; p.KD = KD;
    p.vec_h = is_aligned(out.h, 16) && out.ldh % 4 == 0;
    p.vec_z = out.z && is_aligned(out.z, 16) && out.ldz % 4 == 0 && F % 4 == 0;
    Maps maps;
    memset(&maps, 0, sizeof(maps));
    bool ok = true;
    for (int j = 0; j < 3; ++j) {
        const __nv_bfloat16* wj = reinterpret_cast<const __nv_bfloat16*>(pw + j * plane_w);
        ok = ok && encode_map_bf16(&maps.a[j], pa + j * plane_a, M, KD, up8(KD), 64, BM_CTA);
        for (int r = 0; r < 2; ++r)
            ok = ok && (fwd ? encode_map_bf16(&maps.b[r][j], wj + (long)r * F * up8(K), F, K, up8(K), 64, cut.hn)
                            : encode_map_bf16(&maps.b[r][j], wj, 2L * F, K, up8(K), 64, BK));
    }
    if (!ok) return DPCLIP_ERR_CUDA;
    if (fwd) return cut.hn == 128 ? launch_gated_tc3<true, 128>(maps, p, st) : launch_gated_tc3<true, 64>(maps, p, st);
    return cut.hn == 128 ? launch_gated_tc3<false, 128>(maps, p, st) : launch_gated_tc3<false, 64>(maps, p, st);
}

int gated_check(int M, int K, int F, dpclip_dtype dtype, int act, bool product, const void* workspace, size_t workspace_bytes) {
    if (M <= 0 || K <= 0 || F <= 0 || F > (1 << 29) || !dtype_known(dtype) || act < DPCLIP_ACT_SILU || act > DPCLIP_ACT_RELU) return DPCLIP_ERR_INVALID_ARG;
    if (product && (!workspace || !is_aligned(workspace, 256) || workspace_bytes < dpclip_gated_workspace_bytes(M, K, F, dtype)))
        return DPCLIP_ERR_WORKSPACE;
    return DPCLIP_OK;
}

}  // namespace

extern "C" {

int dpclip_stored_clipped_grad(const float* grads, long ld, int B, int n, const float* clip, float* g, float sigma, float C,
                               unsigned long long seed, unsigned long long stream_id, void* stream) {
    if (!grads || !g || B <= 0 || n <= 0 || ld < n || !(sigma >= 0.f) || !(C >= 0.f)) return DPCLIP_ERR_INVALID_ARG;
    if (!is_aligned(grads, 4) || !is_aligned(g, 4) || (clip && !is_aligned(clip, 4))) return DPCLIP_ERR_MISALIGNED;
    StoredParams p;
    memset(&p, 0, sizeof(p));
    p.G = grads; p.ld = ld; p.B = B; p.n = n; p.clip = clip; p.g = g; p.noise_scale = sigma * C;
    p.k0 = (uint32_t)seed; p.k1 = (uint32_t)(seed >> 32); p.s0 = (uint32_t)stream_id; p.s1 = (uint32_t)(stream_id >> 32);
    cudaStream_t st = (cudaStream_t)stream;
    const int blocks = ceil_div(n, 32);
    if (B <= 64) return launch_after(stored_grad_kernel<8, false>, dim3(blocks), 256, 0, st, p);
    if (B <= STORED_PER_CTA || blocks >= kNumSMs) return launch_after(stored_grad_kernel<32, false>, dim3(blocks), 1024, 0, st, p);
    p.cluster = 2;
    while (p.cluster < STORED_MAX_CLUSTER && p.cluster * STORED_PER_CTA < B) p.cluster *= 2;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(blocks * p.cluster); cfg.blockDim = dim3(1024); cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = overlap_allowed() ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, stored_grad_kernel<32, true>, p) != cudaSuccess) { cudaGetLastError(); return DPCLIP_ERR_CUDA; }
    return finish_launch();
}

int dpclip_relbias_bucket(const dpclip_relbias* config, long distance) {
    RbBuckets r;
    if (!fill_buckets(r, config)) return DPCLIP_ERR_INVALID_ARG;
    return rb_bucket(r, distance);
}

int dpclip_relbias_forward(const float* table, long ldt, const dpclip_relbias* config, int H, int Tq, int Tk, long q_offset,
                           dpclip_dtype dtype, void* bias, long ld, long head_stride, void* stream) {
    RbForward p;
    memset(&p, 0, sizeof(p));
    if (!table || !bias || H <= 0 || Tq <= 0 || Tk <= 0 || q_offset < 0 || !dtype_known(dtype)) return DPCLIP_ERR_INVALID_ARG;
    if (!fill_buckets(p.r, config) || ldt < H || ld < Tk) return DPCLIP_ERR_INVALID_ARG;
    // rows of different heads must not overlap: heads one behind the other, or side by side in every row
    if (H > 1 && head_stride < (long)(Tq - 1) * ld + Tk && (head_stride < Tk || ld < (long)(H - 1) * head_stride + Tk))
        return DPCLIP_ERR_INVALID_ARG;
    if (!is_aligned(table, 4) || !is_aligned(bias, elt_size(dtype))) return DPCLIP_ERR_MISALIGNED;
    p.table = table; p.ldt = ldt; p.out = bias; p.ld = ld; p.hs = H > 1 ? head_stride : 0;
    p.H = H; p.Tq = Tq; p.Tk = Tk; p.off = q_offset;
    const long v = dtype == DPCLIP_F32 ? 4 : 8;
    const bool vec = is_aligned(bias, 16) && (Tq == 1 || ld % v == 0) && p.hs % v == 0;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == DPCLIP_F32) return vec ? launch_relbias_forward<float, 8>(p, st) : launch_relbias_forward<float, 1>(p, st);
    return vec ? launch_relbias_forward<__nv_bfloat16, 8>(p, st) : launch_relbias_forward<__nv_bfloat16, 1>(p, st);
}

size_t dpclip_relbias_workspace_bytes(int B, int H, int Tq, int Tk, int n_buckets, dpclip_dtype dtype) {
    if (!dtype_known(dtype) || B <= 0 || H <= 0 || Tq <= 0 || Tk <= 0 || n_buckets <= 0) return kHeaderBytes;
    const size_t a = relbias_part_bytes(relbias_tiles(B, H, Tq, Tk, true), B, H, n_buckets);
    const size_t b = relbias_part_bytes(relbias_tiles(B, H, Tq, Tk, false), B, H, n_buckets);
    return kHeaderBytes + round_up(a > b ? a : b, 256);
}

int dpclip_relbias_sqnorms(const void* dS, long ld, long head_stride, long example_stride, int B, int H, int Tq, int Tk, long q_offset,
                           const int* q_lens, const int* k_lens, const dpclip_relbias* config, dpclip_dtype dtype, int accumulate,
                           float* grads, float* sq_layer, void* workspace, size_t workspace_bytes, void* stream) {
    RbGrad p;
    memset(&p, 0, sizeof(p));
    if (!dS || !grads || !sq_layer || B <= 0 || H <= 0 || Tq <= 0 || Tk <= 0 || q_offset < 0 || !dtype_known(dtype))
        return DPCLIP_ERR_INVALID_ARG;
    if (!fill_buckets(p.r, config) || (Tq > 1 && ld < Tk)) return DPCLIP_ERR_INVALID_ARG;
    if (H > 1 && head_stride < 0) return DPCLIP_ERR_INVALID_ARG;
    if (B > 1 && example_stride < 0) return DPCLIP_ERR_INVALID_ARG;
    const size_t es = elt_size(dtype);
    if (!is_aligned(dS, es) || !is_aligned(grads, 4) || !is_aligned(sq_layer, 4) || (q_lens && !is_aligned(q_lens, 4)) ||
        (k_lens && !is_aligned(k_lens, 4))) return DPCLIP_ERR_MISALIGNED;
    p.dS = dS; p.ld = Tq > 1 ? ld : Tk; p.hs = H > 1 ? head_stride : 0; p.bs = B > 1 ? example_stride : 0;
    const long v = dtype == DPCLIP_F32 ? 4 : 8;
    const bool vec = is_aligned(dS, 16) && (Tq == 1 || ld % v == 0) && p.hs % v == 0 && p.bs % v == 0;
    const RbTiles t = relbias_tiles(B, H, Tq, Tk, vec);
    const size_t need = kHeaderBytes + relbias_part_bytes(t, B, H, p.r.n_buckets);
    if (!workspace || workspace_bytes < need || !is_aligned(workspace, 16)) return DPCLIP_ERR_WORKSPACE;
    const long tiles = (long)t.qtiles * t.ktiles;
    if ((long)B * H > 0x7FFFFFFFL / tiles) return DPCLIP_ERR_UNSUPPORTED;
    p.B = B; p.H = H; p.Tq = Tq; p.Tk = Tk; p.nqb = t.nqb; p.nkb = t.nkb; p.KT = t.KT; p.G = t.G; p.nr = t.nr;
    p.qtiles = t.qtiles; p.ktiles = t.ktiles; p.off = q_offset; p.q_lens = q_lens; p.k_lens = k_lens;
    p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kHeaderBytes);
    cudaStream_t st = (cudaStream_t)stream;
    int rc;
    if (dtype == DPCLIP_F32) rc = vec ? launch_relbias_grad<float, 8>(p, t.threads, st) : launch_relbias_grad<float, 1>(p, t.threads, st);
    else rc = vec ? launch_relbias_grad<__nv_bfloat16, 8>(p, t.threads, st) : launch_relbias_grad<__nv_bfloat16, 1>(p, t.threads, st);
    if (rc) return rc;
    int lanes = 1;
    while (lanes < 32 && lanes < tiles) lanes *= 2;
    return launch_after(relbias_finish_kernel, dim3(B), RB_FINISH_THREADS, 0, st, (const float*)p.part, H, (int)tiles, p.r.n_buckets,
                        lanes, accumulate ? 1 : 0, grads, sq_layer);
}

int dpclip_rotation_table(float* table, long n_pos, int rot_dim, double base, double scale, void* stream) {
    if (!table || n_pos <= 0 || rot_dim <= 0 || rot_dim % 2 || !(base > 0.0) || !(scale > 0.0)) return DPCLIP_ERR_INVALID_ARG;
    if (!is_aligned(table, 4)) return DPCLIP_ERR_MISALIGNED;
    const long n = n_pos * (rot_dim / 2);
    const long blocks = (n + 255) / 256;
    rotation_table_kernel<<<clamp_int(blocks, 1, kNumSMs * 16), 256, 0, (cudaStream_t)stream>>>(table, n_pos, rot_dim, log(base), 1.0 / scale);
    return finish_launch();
}

int dpclip_qknorm_forward(const dpclip_heads* parts, int n_parts, int B, int T, int D, int rot_dim, int interleaved,
                          const float* table, long n_pos, const int* positions, long pos0, float eps, dpclip_dtype dtype, void* stream) {
    int rc = qk_check(parts, n_parts, B, T, D, rot_dim, table, n_pos, positions, pos0, eps, dtype, false);
    if (rc) return rc;
    QkParams p;
    const bool vec = qk_fill(p, parts, n_parts, B, T, D, rot_dim, interleaved, table, n_pos, positions, pos0, eps, dtype, false);
    QkShape s;
    if (!qk_shape(s, D, rot_dim, vec, dtype)) return DPCLIP_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    return dtype == DPCLIP_F32 ? launch_qk<float>(p, s, false, false, st) : launch_qk<__nv_bfloat16>(p, s, false, false, st);
}

size_t dpclip_qknorm_workspace_bytes(int B, int T, int Hq, int Hk, int D) {
    if (B <= 0 || T <= 0 || Hq < 0 || Hk < 0 || D <= 0) return kHeaderBytes;
    return kHeaderBytes + round_up(sizeof(float) * (size_t)B * (qk_most_sums(B, T, Hq) + qk_most_sums(B, T, Hk)) * D, 256);
}

int dpclip_qknorm_backward(const dpclip_heads* parts, int n_parts, int B, int T, int D, int rot_dim, int interleaved,
                           const float* table, long n_pos, const int* positions, long pos0, float eps, dpclip_dtype dtype,
                           float* const* grads, float* const* sq_layers, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = qk_check(parts, n_parts, B, T, D, rot_dim, table, n_pos, positions, pos0, eps, dtype, true);
    if (rc) return rc;
    if (!grads || !sq_layers) return DPCLIP_ERR_INVALID_ARG;
    for (int k = 0; k < n_parts; ++k)
        if ((grads[k] && !is_aligned(grads[k], 4)) || (sq_layers[k] && !is_aligned(sq_layers[k], 4))) return DPCLIP_ERR_MISALIGNED;
    QkParams p;
    const bool vec = qk_fill(p, parts, n_parts, B, T, D, rot_dim, interleaved, table, n_pos, positions, pos0, eps, dtype, true);
    QkShape s;
    if (!qk_shape(s, D, rot_dim, vec, dtype)) return DPCLIP_ERR_UNSUPPORTED;
    size_t sums[2] = {0, 0};                               // partial sums an example
    for (int k = 0; k < n_parts; ++k) {
        p.part[k].blocks = ceil_div(p.part[k].H, 32 / s.G);
        if ((long)T * p.part[k].blocks > 0x3FFFFFFFL) return DPCLIP_ERR_UNSUPPORTED;
    }
    const bool ring = qk_ring_backward(s, B, T, p.part);
    for (int k = 0; k < n_parts; ++k) {
        p.part[k].chunks = qk_chunks(B, T, p.part[0].blocks + p.part[1].blocks);
        sums[k] = (size_t)p.part[k].blocks * p.part[k].chunks;
    }
    if (!workspace || !is_aligned(workspace, 16) || workspace_bytes < kHeaderBytes + sizeof(float) * B * (sums[0] + sums[1]) * D)
        return DPCLIP_ERR_WORKSPACE;
    p.part[0].part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kHeaderBytes);
    p.part[1].part = p.part[0].part + B * sums[0] * D;
    cudaStream_t st = (cudaStream_t)stream;
    rc = dtype == DPCLIP_F32 ? launch_qk<float>(p, s, true, ring, st) : launch_qk<__nv_bfloat16>(p, s, true, ring, st);
    if (rc) return rc;
    QkFinish f;
    memset(&f, 0, sizeof(f));
    f.D = D; f.B = B;
    bool any = false;
    for (int k = 0; k < n_parts; ++k) {
        f.part[k] = p.part[k].part; f.sums[k] = (int)sums[k]; f.grads[k] = grads[k]; f.sq[k] = sq_layers[k];
        any = any || grads[k] || sq_layers[k];
    }
    if (!any) return DPCLIP_OK;
    // about two warps an SM's scheduler are enough: beyond that a CTA an example only queues
    if (B > 8 * kNumSMs && sums[0] <= 8 && sums[1] <= 8)
        return launch_after(qknorm_finish_kernel<true>, dim3(ceil_div(B, QK_THREADS / 32), n_parts), QK_THREADS, 0, st, f);
    return launch_after(qknorm_finish_kernel<false>, dim3(B, n_parts), QK_THREADS, 0, st, f);
}

size_t dpclip_gated_workspace_bytes(int M, int K, int F, dpclip_dtype dtype) {
    if (M <= 0 || K <= 0 || F <= 0 || !dtype_known(dtype)) return kHeaderBytes;
    const size_t f = total_bytes(gated_space(M, K, F, dtype, true)), b = total_bytes(gated_space(M, K, F, dtype, false));
    return kHeaderBytes + (f > b ? f : b);
}

int dpclip_gated_forward(const void* X, long ldx, const void* W, long ldw, const float* bias, int M, int K, int F, dpclip_dtype dtype,
                         dpclip_activation act, void* H, long ldh, void* Z, long ldz, void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !W || !H || ldx < K || ldw < K || ldh < F || (Z && ldz < 2L * F)) return DPCLIP_ERR_INVALID_ARG;
    int rc = gated_check(M, K, F, dtype, act, true, workspace, workspace_bytes);
    if (rc) return rc;
    const size_t es = elt_size(dtype);
    if (!is_aligned(X, es) || !is_aligned(W, es) || !is_aligned(H, es) || (Z && !is_aligned(Z, es)) || (bias && !is_aligned(bias, 4)))
        return DPCLIP_ERR_MISALIGNED;
    cudaStream_t st = (cudaStream_t)stream;
    const GatedSpace space = gated_space(M, K, F, dtype, true);
    uint8_t* const ws = static_cast<uint8_t*>(workspace) + kHeaderBytes;
    GatedOut out;
    memset(&out, 0, sizeof(out));
    out.h = H; out.ldh = ldh; out.z = Z; out.ldz = ldz; out.bias = bias; out.M = M; out.F = F; out.act = act; out.splits = 1;
    out.part = reinterpret_cast<float*>(ws);
    if (M <= 8) {
        GatedFew p;
        memset(&p, 0, sizeof(p));
        p.x = X; p.ldx = ldx; p.w = W; p.ldw = ldw; p.K = K; p.out = out;
        const long v = dtype == DPCLIP_F32 ? 4 : 8;
        const bool vec = is_aligned(X, 16) && is_aligned(W, 16) && ldw % v == 0 && (M == 1 || ldx % v == 0) && K % v == 0;
        if (dtype == DPCLIP_F32) return vec ? launch_gated_few<float, 4>(p, st) : launch_gated_few<float, 1>(p, st);
        return vec ? launch_gated_few<__nv_bfloat16, 8>(p, st) : launch_gated_few<__nv_bfloat16, 1>(p, st);
    }
    if (dtype == DPCLIP_BF16 && tensor_cores_allowed()) {
        const bool as_is = gated_rows_ok(X, ldx) && gated_rows_ok(W, ldw);
        if (as_is || space.copy_w) {
            const void* a = X; const void* w = W;
            long lda = ldx, ldb = ldw;
            GatedCopy c[2];
            int n = 0;
            if (!gated_rows_ok(X, ldx)) { a = ws + space.part; lda = up8(K); c[n++] = {static_cast<const __nv_bfloat16*>(X), ldx, (__nv_bfloat16*)a, lda, M, K}; }
            if (!gated_rows_ok(W, ldw)) { w = ws + space.part + space.copy_a; ldb = up8(K); c[n++] = {static_cast<const __nv_bfloat16*>(W), ldw, (__nv_bfloat16*)w, ldb, 2L * F, K}; }
            rc = gated_copies(c, n, st);
            if (rc) return rc;
            return gated_tensor(true, a, lda, w, ldb, M, K, F, out, static_cast<int*>(workspace), st);
        }
    }
    if (dtype == DPCLIP_F32 && space.copy_w && tensor_cores_allowed()) {
        uint8_t* const pa = ws + space.part, *const pw = pa + space.copy_a;
        const GatedSplit c[2] = {{static_cast<const float*>(X), ldx, (__nv_bfloat16*)pa, up8(K), (long)(space.copy_a / 6), M, K, 0},
                                 {static_cast<const float*>(W), ldw, (__nv_bfloat16*)pw, up8(K), (long)(space.copy_w / 6), 2L * F, K, 0}};
        rc = gated_splits(c, 2, st);
        return rc ? rc : gated_tensor_f32(true, static_cast<const float*>(X), ldx, static_cast<const float*>(W), ldw, M, K, F, out, ws, space,
                                          static_cast<int*>(workspace), st);
    }
    GatedSimt p;
    memset(&p, 0, sizeof(p));
    p.a = X; p.lda = ldx; p.w = W; p.ldw = ldw; p.M = M; p.N = F; p.KD = K; p.out = out;
    return dtype == DPCLIP_F32 ? launch_gated_simt<float, true>(p, st) : launch_gated_simt<__nv_bfloat16, true>(p, st);
}

int dpclip_gated_backward(const void* dH, long lddh, const void* Z, long ldz, const void* W, long ldw, int M, int K, int F,
                          dpclip_dtype dtype, dpclip_activation act, void* dZ, long lddz, void* dX, long lddx,
                          void* workspace, size_t workspace_bytes, void* stream) {
    if (!dH || !Z || !dZ || lddh < F || ldz < 2L * F || lddz < 2L * F || (dX && (!W || ldw < K || lddx < K))) return DPCLIP_ERR_INVALID_ARG;
    int rc = gated_check(M, K, F, dtype, act, dX != nullptr, workspace, workspace_bytes);
    if (rc) return rc;
    const size_t es = elt_size(dtype);
    if (!is_aligned(dH, es) || !is_aligned(Z, es) || !is_aligned(dZ, es) || (dX && (!is_aligned(dX, es) || !is_aligned(W, es)))) return DPCLIP_ERR_MISALIGNED;
    cudaStream_t st = (cudaStream_t)stream;
    const GatedSpace space = gated_space(M, K, F, dtype, false);
    uint8_t* const ws = static_cast<uint8_t*>(workspace) + kHeaderBytes;
    const bool dz_ok = gated_rows_ok(dZ, lddz), w_ok = dX && gated_rows_ok(W, ldw);
    const bool planes = dX && dtype == DPCLIP_F32 && space.copy_w && tensor_cores_allowed();
    const bool tensor = dX && dtype == DPCLIP_BF16 && tensor_cores_allowed() && ((dz_ok && w_ok) || space.copy_w);
    uint8_t* const pa = ws + space.part, *const pw = pa + space.copy_a;
    // W first: the product then follows the kernel that writes dZ
    if (planes) {
        const GatedSplit c = {static_cast<const float*>(W), ldw, (__nv_bfloat16*)pw, up8(K), (long)(space.copy_w / 6), 2L * F, K, 0};
        rc = gated_splits(&c, 1, st);
    } else if (tensor && !w_ok) {
        const GatedCopy c = {static_cast<const __nv_bfloat16*>(W), ldw, (__nv_bfloat16*)pw, up8(K), 2L * F, K};
        rc = gated_copies(&c, 1, st);
    }
    if (rc) return rc;
    GatedSignal s;
    memset(&s, 0, sizeof(s));
    s.dh = dH; s.lddh = lddh; s.z = Z; s.ldz = ldz; s.dz = dZ; s.lddz = lddz; s.M = M; s.F = F; s.act = act;
    if (planes || (tensor && !dz_ok)) { s.copy = (__nv_bfloat16*)pa; s.ldc = up8(2L * F); s.plane = (long)(space.copy_a / 6); }
    const long v = dtype == DPCLIP_F32 ? 4 : 8;
    const bool vec = is_aligned(dH, 16) && is_aligned(Z, 16) && is_aligned(dZ, 16) && F % v == 0 && lddh % v == 0 && ldz % v == 0 && lddz % v == 0;
    s.per_row = vec ? F / (int)v : F;
    const int along = vec ? s.per_row : ceil_div(s.per_row, 4);
    s.wide = along < 256 ? along : 256;
    const long rows = ceil_div(M, 256 / s.wide);
    const int grid_x = clamp_int(rows, 1, kNumSMs * 8);
    const dim3 grid(grid_x, clamp_int(kNumSMs * 2 / grid_x, 1, ceil_div(along, s.wide)));
    if (dtype == DPCLIP_F32) {
        if (vec) gated_signal_kernel<float, 4><<<grid, 256, 0, st>>>(s);
        else gated_signal_kernel<float, 1><<<grid, 256, 0, st>>>(s);
    } else {
        if (vec) gated_signal_kernel<__nv_bfloat16, 8><<<grid, 256, 0, st>>>(s);
        else gated_signal_kernel<__nv_bfloat16, 1><<<grid, 256, 0, st>>>(s);
    }
    rc = finish_launch();
    if (rc || !dX) return rc;
    GatedOut out;
    memset(&out, 0, sizeof(out));
    out.h = dX; out.ldh = lddx; out.M = M; out.F = K; out.splits = 1;
    out.part = reinterpret_cast<float*>(ws);
    if (tensor) {
        return gated_tensor(false, dz_ok ? dZ : s.copy, dz_ok ? lddz : s.ldc, w_ok ? W : pw, w_ok ? ldw : up8(K), M, K, F, out,
                            static_cast<int*>(workspace), st);
    }
    if (planes) return gated_tensor_f32(false, static_cast<const float*>(dZ), lddz, static_cast<const float*>(W), ldw, M, K, F, out, ws, space,
                                        static_cast<int*>(workspace), st);
    GatedSimt p;
    memset(&p, 0, sizeof(p));
    p.a = dZ; p.lda = lddz; p.w = W; p.ldw = ldw; p.M = M; p.N = K; p.KD = 2 * F; p.out = out;
    return dtype == DPCLIP_F32 ? launch_gated_simt<float, false>(p, st) : launch_gated_simt<__nv_bfloat16, false>(p, st);
}

}  // extern "C"

// fg_group_norm and its gradients: rows of a group (a graph, a node type), normalised over the rows and blocks of adjacent columns, with an activation.
//
// The entries of all groups are a line that is cut into chunks of rows. A group of few rows belongs to the chunk it begins in and is done there:
// one pass for the sums, one for the result, whose rows come from the caches. A group of many rows is split along the chunks' ends: every chunk leaves the
// sums of its part, a second launch joins them, a third goes over the rows again. A workgroup takes a chunk and a tile of whole blocks of columns; a
// thread has pieces of eight adjacent columns and every side-th row. Which chunk a group lies in is found from the offsets, on the device.
#include "activation.h"
#include "row_list.h"
#include "row_types.h"
#include "scan.h"

namespace {

constexpr int GN_THREADS = 256, GN_WAVES = GN_THREADS / 64, GN_COLUMNS = 256;      // columns of a tile that has several blocks
constexpr int GN_PLACES = 1024, GN_FEW_VALUES = 65536, GN_MAX_PIECES = 8;

struct GnArgs {
    const int32_t* order;      // NULL: position k itself
    const int64_t* offsets;
    int64_t max_rows, n, rows, long_rows;      // rows of a chunk; a group of more rows than long_rows is split
    int n_groups, d, block, blocks, tile_blocks, width;      // columns of a block, blocks of a row, blocks of a tile, lanes of a row's tile
    const char *x, *dy;
    int64_t x_stride, dy_stride, out_stride;
    const float *weight, *bias;
    float eps;
    int act, out_type;
    char* out;
    float *mean, *rstd;      // [n_groups x blocks]; the forward call's may be NULL
    double* part;            // [chunks][2][blocks][3]: the sums of a chunk's parts of a group that began before it, and of one that begins in it
    int32_t* info;           // [chunks][2]: those groups, -1: none
    float* joined;           // [chunks][blocks][2]: what the parts of the group that begins in the chunk come to
    float* columns;          // [chunks][2][d]: sums for dw and db, or NULL
};

__device__ __forceinline__ int64_t offset_of(const GnArgs& A, int g) {
    const int64_t o = A.offsets[g];
    return o < 0 ? 0 : (o > A.max_rows ? A.max_rows : o);
}
// the first group that begins at `target` or beyond (lanes of a wavefront together, 64 offsets at a time)
__device__ __forceinline__ int first_from(const GnArgs& A, int64_t target) {
    int lo = 0, hi = A.n_groups;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64;
        const int64_t i = lo + (int64_t)fg_lane() * step;
        const int before = __popcll(__ballot(i < hi && offset_of(A, i < hi ? (int)i : lo) < target));
        if (before == 0) return lo;
        const int64_t end = lo + (int64_t)before * step;
        lo += (before - 1) * step + 1;
        hi = end < hi ? (int)end : hi;
    }
    return lo;
}
enum { GN_WHOLE, GN_GOES_ON, GN_BEGINS };
// The parts of groups that belong to a chunk, in order, the same in all wavefronts.
struct Walk {
    const GnArgs& A;
    int64_t c0, c1, from, to;      // entries of the chunk; of the group that this lane looks at
    int first, base;
    unsigned long long mask;       // lanes whose groups are still to come
    __device__ __forceinline__ Walk(const GnArgs& args, int64_t chunk) : A(args) {
        c0 = chunk * A.rows;
        c1 = c0 + A.rows;
        first = first_from(A, c0);
        base = first - 64;
        mask = 0;
        from = to = c0;
    }
    // The next part: group, first entry and end, which of the three. empty(group): by one lane of the first wavefront, for every group without entries that
    // lies here
    template <typename Empty>
    __device__ __forceinline__ bool next(int& g, int64_t& k0, int64_t& k1, int& which, const Empty& empty) {
        if (base == first - 64 && first > 0) {      // the group that began before the chunk
            g = --first;
            base = first - 63;
            k0 = c0;
            const int64_t begin = offset_of(A, g), end = offset_of(A, g + 1);
            k1 = end < c1 ? end : c1;
            which = GN_GOES_ON;
            if (begin < c0 && end > c0 && end - begin > A.long_rows) return true;
        }
        while (!mask) {
            if (__ballot(from >= c1)) return false;
            base += 64;
            if (base >= A.n_groups) return false;
            const int i = base + fg_lane();
            from = c1, to = 0;
            if (i < A.n_groups) {
                from = offset_of(A, i);
                to = offset_of(A, i + 1);
            }
            const bool here = from >= c0 && from < c1;
            if (here && to <= from && fg_wave() == 0) empty(i);
            mask = __ballot(here && to > from);
        }
        const int l = __ffsll((long long)mask) - 1;
        mask &= mask - 1;
        g = base + l;
        k0 = __shfl((long long)from, l, 64);
        k1 = __shfl((long long)to, l, 64);
        which = k1 - k0 > A.long_rows ? GN_BEGINS : GN_WHOLE;
        if (which == GN_BEGINS && k1 > c1) k1 = c1;
        return true;
    }
};
__device__ __forceinline__ int64_t position(const GnArgs& A, int64_t k) {
    const int64_t r = A.order ? A.order[k] : k;
    return r < 0 || r >= A.n ? -1 : r;
}

// this workgroup's tile and this thread's share of it
struct Tile {
    int c0, cols, block0, n_blocks, p, side, sides;      // columns, blocks; piece and row of the thread, rows side by side
};
__device__ __forceinline__ Tile tile_of(const GnArgs& A) {
    Tile T;
    T.block0 = (int)blockIdx.y * A.tile_blocks;
    T.n_blocks = A.blocks - T.block0 < A.tile_blocks ? A.blocks - T.block0 : A.tile_blocks;
    T.c0 = T.block0 * A.block;
    T.cols = T.n_blocks * A.block;
    T.p = (int)threadIdx.x % A.width;
    T.side = (int)threadIdx.x / A.width;
    T.sides = GN_THREADS / A.width;
    return T;
}

struct Scratch {
    double wave[GN_WAVES][2 * GN_COLUMNS];      // sums of a wavefront's rows, by column
    double sums[GN_COLUMNS][2];                 // of a block
    float stats[GN_COLUMNS][2];
    int rows[GN_WAVES];
};
__device__ __forceinline__ int workgroup_rows(Scratch& S, int rows, int width) {
    for (int off = 32; off > 0; off >>= 1) rows += __shfl_xor(rows, off, 64);
    if (fg_lane() == 0) S.rows[fg_wave()] = rows;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < GN_WAVES; ++w) all += S.rows[w];
    return all / width;
}
// s[e], q[e] of the thread's columns (MANY) or s[0], q[0] of all it has seen: the sums of every block in S.sums (after the caller's next barrier)
template <bool MANY>
__device__ __forceinline__ void block_sums(const GnArgs& A, const Tile& T, Scratch& S, double (&s)[MANY ? 8 : 1], double (&q)[MANY ? 8 : 1]) {
    constexpr int N = MANY ? 8 : 1;
#pragma unroll
    for (int e = 0; e < N; ++e)
        for (int off = MANY ? A.width : 1; off < 64; off <<= 1) {
            s[e] += __shfl_xor(s[e], off, 64);
            q[e] += __shfl_xor(q[e], off, 64);
        }
    if constexpr (MANY) {
        if (fg_lane() < A.width && T.p * 8 < T.cols)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (T.p * 8 + e < T.cols) {
                    S.wave[fg_wave()][T.p * 8 + e] = s[e];
                    S.wave[fg_wave()][GN_COLUMNS + T.p * 8 + e] = q[e];
                }
        __syncthreads();
        int lanes = 1;      // of a block
        while (lanes < 64 && lanes * 2 * T.n_blocks <= GN_THREADS) lanes *= 2;
        const int j = (int)threadIdx.x / lanes, l = (int)threadIdx.x % lanes;
        double a = 0.0, b = 0.0;
        if (j < T.n_blocks)
            for (int c = j * A.block + l; c < (j + 1) * A.block; c += lanes)
#pragma unroll
                for (int w = 0; w < GN_WAVES; ++w) {
                    a += S.wave[w][c];
                    b += S.wave[w][GN_COLUMNS + c];
                }
        for (int off = lanes >> 1; off > 0; off >>= 1) {
            a += __shfl_xor(a, off, 64);
            b += __shfl_xor(b, off, 64);
        }
        if (j < T.n_blocks && l == 0) S.sums[j][0] = a, S.sums[j][1] = b;
    } else {
        if (fg_lane() == 0) S.wave[fg_wave()][0] = s[0], S.wave[fg_wave()][1] = q[0];
        __syncthreads();
        if (threadIdx.x == 0) {
            double a = 0.0, b = 0.0;
#pragma unroll
            for (int w = 0; w < GN_WAVES; ++w) a += S.wave[w][0], b += S.wave[w][1];
            S.sums[0][0] = a, S.sums[0][1] = b;
        }
    }
}
__device__ __forceinline__ void write_part(const GnArgs& A, const Tile& T, const Scratch& S, int64_t chunk, int which, int rows) {
    for (int j = threadIdx.x; j < T.n_blocks; j += GN_THREADS) {
        double* to = A.part + ((chunk * 2 + (which == GN_BEGINS)) * A.blocks + T.block0 + j) * 3;
        to[0] = S.sums[j][0], to[1] = S.sums[j][1], to[2] = (double)rows;
    }
}
__device__ __forceinline__ void note(const GnArgs& A, int64_t chunk, int goes_on, int begins) {
    if (threadIdx.x == 0 && blockIdx.y == 0 && A.info) A.info[chunk * 2] = goes_on, A.info[chunk * 2 + 1] = begins;
}
__device__ __forceinline__ float element(const char* p, int type, int64_t i) {
    if (type == FG_F32) return ((const float*)p)[i];
    const unsigned short v = ((const unsigned short*)p)[i];
    return type == FG_BF16 ? __uint_as_float((unsigned int)v << 16) : (float)__builtin_bit_cast(_Float16, v);
}
// what a block's values are measured from: its first value in the group's first row (0 where that row does not exist)
__device__ __forceinline__ float level(const GnArgs& A, int type, int g, int block) {
    const int64_t r = position(A, offset_of(A, g));
    return r >= 0 ? element(A.x + r * A.x_stride, type, (int64_t)block * A.block) : 0.f;
}
__device__ __forceinline__ void mean_rstd(const GnArgs& A, float from, double s, double q, double rows, float& mean, float& rstd) {
    const double size = rows > 0.0 ? rows * A.block : 1.0, m = s / size, v = q / size - m * m;
    mean = (float)((double)from + m);
    rstd = (float)(1.0 / sqrt((v > 0.0 || !(v == v) ? v : 0.0) + (double)A.eps));
}
__device__ __forceinline__ void activate(int act, float (&u)[8]) {
    fg_with_act(act, [&](auto which) {
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = fg_act<decltype(which)::value>(u[e]);
    });
}
// slopes in place of the arguments
__device__ __forceinline__ void slopes(int act, float (&u)[8]) {
    fg_with_act(act, [&](auto which) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float f;
            fg_act_slope<decltype(which)::value>(u[e], f, u[e]);
        }
    });
}
__device__ __forceinline__ void affine(const GnArgs& A, const Tile& T, int c, float (&w)[8], float (&b)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.f, b[e] = 0.f;
    if (A.weight) fg_piece_values<FG_F32>(fg_load_piece<FG_F32>((const char*)(A.weight + T.c0 + c), T.cols - c), w);
    if (A.bias) fg_piece_values<FG_F32>(fg_load_piece<FG_F32>((const char*)(A.bias + T.c0 + c), T.cols - c), b);
}

// y of the entries [k0, k1) with the blocks' mean and rstd in S.stats
template <int T_, bool MANY>
__device__ __forceinline__ void normalise(const GnArgs& A, const Tile& T, const Scratch& S, int64_t k0, int64_t k1) {
    constexpr int E = T_ == FG_F32 ? 4 : 2, AHEAD = 4;
    for (int c = T.p * 8; c < T.cols; c += A.width * 8) {
        float w[8], b[8], mean[8], rstd[8];
        affine(A, T, c, w, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = MANY && c + e < T.cols ? (c + e) / A.block : 0;
            mean[e] = S.stats[j][0], rstd[e] = S.stats[j][1];
        }
        for (int64_t k = k0 + T.side; k < k1; k += AHEAD * T.sides) {
            int64_t r[AHEAD];
            fg_piece<T_> v[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) r[u] = k + u * T.sides < k1 ? position(A, k + u * T.sides) : -1;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (r[u] >= 0) v[u] = fg_load_piece<T_>(A.x + r[u] * A.x_stride + (int64_t)(T.c0 + c) * E, T.cols - c);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (r[u] < 0) continue;
                float f[8];
                fg_piece_values<T_>(v[u], f);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (f[e] - mean[e]) * rstd[e] * w[e] + b[e];
                activate(A.act, f);
                char* to = A.out + r[u] * A.out_stride;
                if (A.out_type == FG_F32)
                    fg_store_piece<FG_F32>(to + (int64_t)(T.c0 + c) * 4, f, T.cols - c);
                else if constexpr (T_ != FG_F32)
                    fg_store_piece<T_>(to + (int64_t)(T.c0 + c) * 2, f, T.cols - c);
            }
        }
    }
}

template <int T_, bool MANY>
__global__ __launch_bounds__(GN_THREADS) void group_norm_kernel(GnArgs A) {
    constexpr int E = T_ == FG_F32 ? 4 : 2, N = MANY ? 8 : 1, AHEAD = 4;
    __shared__ Scratch S;
    const Tile T = tile_of(A);
    const int64_t chunk = blockIdx.x;
    int goes_on = -1, begins = -1, g, which;
    int64_t k0, k1;
    const auto empty = [&](int i) {
        for (int j = 0; j < T.n_blocks; ++j) {
            const int64_t at = (int64_t)i * A.blocks + T.block0 + j;
            if (A.mean) A.mean[at] = 0.f;
            if (A.rstd) A.rstd[at] = (float)(1.0 / sqrt((double)A.eps));
        }
    };
    for (Walk W(A, chunk); W.next(g, k0, k1, which, empty);) {
        double s[N] = {}, q[N] = {};
        int rows = 0;
        for (int c = T.p * 8; c == T.p * 8 || c < T.cols; c += A.width * 8) {
            float from[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) from[e] = c + e < T.cols ? level(A, T_, g, T.block0 + (MANY ? (c + e) / A.block : 0)) : 0.f;
            for (int64_t k = k0 + T.side; k < k1; k += AHEAD * T.sides) {
                int64_t r[AHEAD];
                fg_piece<T_> v[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    r[u] = k + u * T.sides < k1 ? position(A, k + u * T.sides) : -1;
                    rows += r[u] >= 0 && c == T.p * 8;
                    if (c >= T.cols) r[u] = -1;
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
                    if (r[u] >= 0) v[u] = fg_load_piece<T_>(A.x + r[u] * A.x_stride + (int64_t)(T.c0 + c) * E, T.cols - c);
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (r[u] < 0) continue;
                    float f[8];
                    fg_piece_values<T_>(v[u], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const double x = c + e < T.cols ? (double)f[e] - (double)from[e] : 0.0;
                        s[MANY ? e : 0] += x;
                        q[MANY ? e : 0] += x * x;
                    }
                }
            }
        }
        rows = workgroup_rows(S, rows, A.width);
        block_sums<MANY>(A, T, S, s, q);
        __syncthreads();
        if (which == GN_WHOLE) {
            for (int j = threadIdx.x; j < T.n_blocks; j += GN_THREADS) {
                float mean, rstd;
                mean_rstd(A, level(A, T_, g, T.block0 + j), S.sums[j][0], S.sums[j][1], (double)rows, mean, rstd);
                S.stats[j][0] = mean, S.stats[j][1] = rstd;
                const int64_t at = (int64_t)g * A.blocks + T.block0 + j;
                if (A.mean) A.mean[at] = mean;
                if (A.rstd) A.rstd[at] = rstd;
            }
            __syncthreads();
            normalise<T_, MANY>(A, T, S, k0, k1);
        } else {
            write_part(A, T, S, chunk, which, rows);
            (which == GN_BEGINS ? begins : goes_on) = g;
        }
        __syncthreads();      // the scratch may be used again
    }
    note(A, chunk, goes_on, begins);
}

// The parts of every split group, added up in order: a wavefront to a block of columns. BACKWARD: the two means of the gradient
template <int T_, bool BACKWARD>
__global__ __launch_bounds__(GN_THREADS) void group_norm_join_kernel(GnArgs A) {
    const int64_t chunk = blockIdx.x;
    const int j = (int)blockIdx.y * GN_WAVES + fg_wave();
    const int g = A.info[chunk * 2 + 1];
    if (g < 0 || j >= A.blocks) return;
    const int64_t last = (offset_of(A, g + 1) - 1) / A.rows;
    double s = 0.0, q = 0.0, rows = 0.0;
    for (int64_t c = chunk + fg_lane(); c <= last; c += 64) {
        const double* p = A.part + ((c * 2 + (c == chunk)) * A.blocks + j) * 3;
        s += p[0], q += p[1], rows += p[2];
    }
    for (int off = 32; off > 0; off >>= 1) {
        s += __shfl_xor(s, off, 64);
        q += __shfl_xor(q, off, 64);
        rows += __shfl_xor(rows, off, 64);
    }
    if (fg_lane() != 0) return;
    float* to = A.joined + (chunk * A.blocks + j) * 2;
    if constexpr (BACKWARD) {
        const double size = rows > 0.0 ? rows * A.block : 1.0;
        to[0] = (float)(s / size), to[1] = (float)(q / size);
    } else {
        mean_rstd(A, level(A, T_, g, j), s, q, rows, to[0], to[1]);
        if (A.mean) A.mean[(int64_t)g * A.blocks + j] = to[0];
        if (A.rstd) A.rstd[(int64_t)g * A.blocks + j] = to[1];
    }
}

// a chunk's parts of split groups: f(group, first entry, end) with what the join has left in S.stats
template <typename F>
__device__ __forceinline__ void split_parts(const GnArgs& A, const Tile& T, Scratch& S, const F& f) {
    const int64_t chunk = blockIdx.x, c0 = chunk * A.rows, c1 = c0 + A.rows;
    for (int which = 0; which < 2; ++which) {
        const int g = A.info[chunk * 2 + which];
        if (g < 0) continue;
        const int64_t from = offset_of(A, g), to = offset_of(A, g + 1), begin = from / A.rows;
        for (int j = threadIdx.x; j < T.n_blocks; j += GN_THREADS) {
            const float* p = A.joined + (begin * A.blocks + T.block0 + j) * 2;
            S.stats[j][0] = p[0], S.stats[j][1] = p[1];
        }
        __syncthreads();
        f(g, from > c0 ? from : c0, to < c1 ? to : c1);
        __syncthreads();
    }
}
template <int T_, bool MANY>
__global__ __launch_bounds__(GN_THREADS) void group_norm_apply_kernel(GnArgs A) {
    __shared__ Scratch S;
    const Tile T = tile_of(A);
    split_parts(A, T, S, [&](int, int64_t k0, int64_t k1) { normalise<T_, MANY>(A, T, S, k0, k1); });
}

// ---- gradients ----

// xh, t and q = t * weight of a piece
__device__ __forceinline__ void gradient_terms(const GnArgs& A, const float (&mean)[8], const float (&rstd)[8], const float (&w)[8], const float (&b)[8], float (&xh)[8],
                                               float (&t)[8]) {
    float slope[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        xh[e] = (xh[e] - mean[e]) * rstd[e];
        slope[e] = xh[e] * w[e] + b[e];
    }
    slopes(A.act, slope);
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] *= slope[e];
}
// f(piece, columns left, xh, t, w, rstd, row) for every piece of the entries [k0, k1) that this thread has, by columns
template <int X, int G, bool MANY, int NP, typename F>
__device__ __forceinline__ void gradient_pass(const GnArgs& A, const Tile& T, int g, int64_t k0, int64_t k1, const F& f) {
    constexpr int XE = X == FG_F32 ? 4 : 2, GE = G == FG_F32 ? 4 : 2, AHEAD = 2;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (T.p + A.width * i) * 8;
        if (c >= T.cols) continue;
        float w[8], b[8], mean[8], rstd[8];
        affine(A, T, c, w, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t at = (int64_t)g * A.blocks + T.block0 + (MANY && c + e < T.cols ? (c + e) / A.block : 0);
            mean[e] = A.mean[at], rstd[e] = A.rstd[at];
        }
        for (int64_t k = k0 + T.side; k < k1; k += AHEAD * T.sides) {
            int64_t r[AHEAD];
            fg_piece<X> vx[AHEAD];
            fg_piece<G> vg[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) r[u] = k + u * T.sides < k1 ? position(A, k + u * T.sides) : -1;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (r[u] >= 0) {
                    vx[u] = fg_load_piece<X>(A.x + r[u] * A.x_stride + (int64_t)(T.c0 + c) * XE, T.cols - c);
                    vg[u] = fg_load_piece<G>(A.dy + r[u] * A.dy_stride + (int64_t)(T.c0 + c) * GE, T.cols - c);
                }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (r[u] < 0) continue;
                float xh[8], t[8];
                fg_piece_values<X>(vx[u], xh);
                fg_piece_values<G>(vg[u], t);
                gradient_terms(A, mean, rstd, w, b, xh, t);
                f(i, c, xh, t, w, rstd, r[u]);
            }
        }
    }
}
// dx of the entries [k0, k1) with the blocks' two means in S.stats
template <int X, int G, bool MANY, int NP>
__device__ __forceinline__ void input_gradient(const GnArgs& A, const Tile& T, const Scratch& S, int g, int64_t k0, int64_t k1) {
    gradient_pass<X, G, MANY, NP>(A, T, g, k0, k1, [&](int, int c, const float(&xh)[8], float(&t)[8], const float(&w)[8], const float(&rstd)[8], int64_t r) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = MANY && c + e < T.cols ? (c + e) / A.block : 0;
            t[e] = rstd[e] * (t[e] * w[e] - S.stats[j][0] - xh[e] * S.stats[j][1]);
        }
        fg_store_piece<G>(A.out + r * A.out_stride + (int64_t)(T.c0 + c) * (G == FG_F32 ? 4 : 2), t, T.cols - c);
    });
}

template <int X, int G, bool MANY, int NP>
__global__ __launch_bounds__(GN_THREADS) void group_norm_backward_kernel(GnArgs A) {
    constexpr int N = MANY ? 8 : 1;
    __shared__ Scratch S;
    const Tile T = tile_of(A);
    const int64_t chunk = blockIdx.x;
    int goes_on = -1, begins = -1, g, which;
    int64_t k0, k1;
    float dw[NP][8] = {}, db[NP][8] = {};
    for (Walk W(A, chunk); W.next(g, k0, k1, which, [](int) {});) {
        double s[N] = {}, q[N] = {};
        int rows = 0;
        for (int64_t k = k0 + T.side; k < k1; k += T.sides) rows += position(A, k) >= 0;
        gradient_pass<X, G, MANY, NP>(A, T, g, k0, k1, [&](int i, int c, const float(&xh)[8], const float(&t)[8], const float(&w)[8], const float(&)[8], int64_t) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (c + e >= T.cols) continue;
                const float a = t[e] * w[e];
                s[MANY ? e : 0] += (double)a;
                q[MANY ? e : 0] += (double)a * (double)xh[e];
                dw[i][e] += t[e] * xh[e];
                db[i][e] += t[e];
            }
        });
        rows = workgroup_rows(S, rows, A.width);
        block_sums<MANY>(A, T, S, s, q);
        __syncthreads();
        if (which == GN_WHOLE) {
            const double size = rows > 0 ? (double)rows * A.block : 1.0;
            for (int j = threadIdx.x; j < T.n_blocks; j += GN_THREADS) S.stats[j][0] = (float)(S.sums[j][0] / size), S.stats[j][1] = (float)(S.sums[j][1] / size);
            __syncthreads();
            input_gradient<X, G, MANY, NP>(A, T, S, g, k0, k1);
        } else {
            write_part(A, T, S, chunk, which, rows);
            (which == GN_BEGINS ? begins : goes_on) = g;
        }
        __syncthreads();
    }
    note(A, chunk, goes_on, begins);
    if (!A.columns) return;
    // the rows that were walked side by side: their column sums meet in LDS
    float* const to = A.columns + chunk * 2 * A.d + T.c0;
    float* const meet = (float*)S.wave;      // [side][width * 8]
    static_assert(sizeof(S.wave) >= GN_THREADS * 8 * sizeof(float), "eight columns of every thread");
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (T.sides == 1) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = (T.p + A.width * i) * 8;
                if (c < T.cols) fg_store_piece<FG_F32>((char*)(to + which * A.d + c), which ? db[i] : dw[i], T.cols - c);
            }
        } else {      // (NP is 1 where rows lie side by side)
#pragma unroll
            for (int e = 0; e < 8; ++e) meet[threadIdx.x * 8 + e] = which ? db[0][e] : dw[0][e];
            __syncthreads();
            for (int c = threadIdx.x; c < T.cols; c += GN_THREADS) {
                float v = 0.f;
                for (int i = 0; i < T.sides; ++i) v += meet[i * A.width * 8 + c];
                to[which * A.d + c] = v;
            }
            __syncthreads();
        }
    }
}
template <int X, int G, bool MANY, int NP>
__global__ __launch_bounds__(GN_THREADS) void group_norm_backward_apply_kernel(GnArgs A) {
    __shared__ Scratch S;
    const Tile T = tile_of(A);
    split_parts(A, T, S, [&](int g, int64_t k0, int64_t k1) { input_gradient<X, G, MANY, NP>(A, T, S, g, k0, k1); });
}
// dw and db: the chunks' sums added up in fp64, in order; 32 columns a workgroup, eight runs of chunks side by side
__global__ __launch_bounds__(GN_THREADS) void group_norm_columns_kernel(const float* __restrict__ columns, int64_t chunks, int d, float* dw, float* db) {
    __shared__ double red[GN_THREADS];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31);
    double s = 0.0;
    if (c < 2 * d)
#pragma unroll 8
        for (int64_t b = threadIdx.x >> 5; b < chunks; b += GN_THREADS / 32) s += (double)columns[b * 2 * d + c];
    red[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 32 && c < 2 * d) {
        for (int i = 1; i < GN_THREADS / 32; ++i) s += red[threadIdx.x + 32 * i];
        float* to = c < d ? dw : db;
        if (to) to[c < d ? c : c - d] = (float)s;
    }
}

// How a call is cut: whole blocks of up to GN_COLUMNS columns to a tile, or one wider block; chunks of rows so that there are about four workgroups to a
// compute unit, with four rows a thread at least. A group whose values in a tile are up to GN_FEW_VALUES is not split.
struct Plan {
    int tile_blocks, tiles, width, pieces;
    int64_t rows, chunks, most_chunks, long_rows;
    bool split;
};
Plan plan_of(int64_t max_rows, int d, int blocks) {
    Plan P;
    const int block = d / blocks, per_tile = GN_COLUMNS / block;
    P.tile_blocks = per_tile < 1 ? 1 : (per_tile < blocks ? per_tile : blocks);
    P.tiles = (int)fg_ceil_div(blocks, P.tile_blocks);
    const int cols = P.tile_blocks * block, pieces = (int)fg_ceil_div(cols, 8);
    P.width = 1;
    while (P.width < pieces && P.width < GN_THREADS) P.width *= 2;
    P.pieces = (int)fg_ceil_div(pieces, P.width);
    const int64_t places = GN_PLACES / P.tiles, least = 4 * (GN_THREADS / P.width);
    const int64_t even = fg_ceil_div(max_rows, places);
    P.rows = even > least ? even : least;
    P.chunks = max_rows / P.rows + 1;
    P.most_chunks = (max_rows / least < places ? max_rows / least : places) + 1;
    P.long_rows = P.rows > GN_FEW_VALUES / cols ? P.rows : GN_FEW_VALUES / cols;
    P.split = P.long_rows < max_rows;
    return P;
}
static_assert(FG_MAX_NORM_DIM <= GN_THREADS * 8 * GN_MAX_PIECES && FG_MAX_NORM_DIM / GN_COLUMNS * 2 <= GN_PLACES, "pieces of a row; tiles");

// (by the most chunks that a call of up to so many rows has: a workspace for max_rows serves fewer rows too)
struct Space {
    size_t part, info, joined, columns;
    size_t total() const { return part + info + joined + columns + 16; }
};
Space space_of(int64_t max_rows, int d, int blocks, bool backward) {
    const Plan P = plan_of(max_rows, d, blocks);
    Space W = {};
    W.part = fg_align_up((size_t)P.most_chunks * 2 * blocks * 3 * 8, 256);
    W.info = fg_align_up((size_t)P.most_chunks * 2 * 4, 256);
    W.joined = fg_align_up((size_t)P.most_chunks * blocks * 2 * 4, 256);
    if (backward) W.columns = (size_t)P.most_chunks * 2 * d * 4;
    return W;
}

fg_status_t check_norm(const char* who, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups, int64_t n, int32_t d,
                       int32_t channel_groups, fg_act_t act) {
    FG_TRY(check_rows(who, nullptr, nullptr, 0, n, d));
    if (max_rows < 0 || max_rows > INT32_MAX) FG_FAIL(FG_ERR_INVALID_ARG, "%s: a number of rows is negative or too large", who);
    if (d > FG_MAX_NORM_DIM) FG_FAIL(FG_ERR_SHAPE, "%s: d = %d is more than %d", who, d, FG_MAX_NORM_DIM);
    if (n_groups < 1 || n_groups > FG_MAX_NORM_GROUPS) FG_FAIL(FG_ERR_INVALID_ARG, "%s: n_groups = %d is not in 1..%d", who, n_groups, FG_MAX_NORM_GROUPS);
    if (channel_groups < 1 || channel_groups > d || d % channel_groups) FG_FAIL(FG_ERR_SHAPE, "%s: %d groups do not divide d = %d columns", who, channel_groups, d);
    if (!fg_act_known(act)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: unknown activation %d", who, (int)act);
    if (!offsets_dev || ((uintptr_t)offsets_dev & 7) || ((uintptr_t)order_dev & 3))
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: offsets must not be NULL, and order and offsets aligned to their elements", who);
    return FG_OK;
}
fg_status_t check_space(const char* who, const void* ws_dev, size_t ws_bytes, size_t need) {
    if (!ws_dev || ((uintptr_t)ws_dev & 15)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: the workspace must be 16-byte aligned device memory", who);
    if (ws_bytes < need) FG_FAIL(FG_ERR_SHAPE, "%s: workspace of %zu bytes, %zu are needed", who, ws_bytes, need);
    return FG_OK;
}
GnArgs args_of(const Plan& P, const Space& W, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups, int64_t n, int32_t d,
               int32_t blocks, void* ws_dev) {
    GnArgs A = {};
    A.order = order_dev, A.offsets = offsets_dev, A.max_rows = max_rows, A.n = n, A.rows = P.rows, A.long_rows = P.long_rows;
    A.n_groups = n_groups, A.d = d, A.block = d / blocks, A.blocks = blocks, A.tile_blocks = P.tile_blocks, A.width = P.width;
    char* ws = (char*)ws_dev;
    A.part = (double*)ws;
    A.info = P.split ? (int32_t*)(ws + W.part) : nullptr;
    A.joined = (float*)(ws + W.part + W.info);
    A.columns = (float*)(ws + W.part + W.info + W.joined);
    return A;
}

template <int T>
void forward(const Plan& P, const GnArgs& A, hipStream_t st) {
    const dim3 grid((unsigned)P.chunks, (unsigned)P.tiles), joins((unsigned)P.chunks, (unsigned)fg_ceil_div(A.blocks, GN_WAVES));
    const bool many = P.tile_blocks > 1;
    if (many)
        hipLaunchKernelGGL((group_norm_kernel<T, true>), grid, dim3(GN_THREADS), 0, st, A);
    else
        hipLaunchKernelGGL((group_norm_kernel<T, false>), grid, dim3(GN_THREADS), 0, st, A);
    if (!P.split) return;
    hipLaunchKernelGGL((group_norm_join_kernel<T, false>), joins, dim3(GN_THREADS), 0, st, A);
    if (many)
        hipLaunchKernelGGL((group_norm_apply_kernel<T, true>), grid, dim3(GN_THREADS), 0, st, A);
    else
        hipLaunchKernelGGL((group_norm_apply_kernel<T, false>), grid, dim3(GN_THREADS), 0, st, A);
}
template <int X, int G, bool MANY, int NP>
void backward_pass(const Plan& P, const GnArgs& A, hipStream_t st) {
    const dim3 grid((unsigned)P.chunks, (unsigned)P.tiles), joins((unsigned)P.chunks, (unsigned)fg_ceil_div(A.blocks, GN_WAVES));
    hipLaunchKernelGGL((group_norm_backward_kernel<X, G, MANY, NP>), grid, dim3(GN_THREADS), 0, st, A);
    if (!P.split) return;
    hipLaunchKernelGGL((group_norm_join_kernel<X, true>), joins, dim3(GN_THREADS), 0, st, A);
    hipLaunchKernelGGL((group_norm_backward_apply_kernel<X, G, MANY, NP>), grid, dim3(GN_THREADS), 0, st, A);
}
template <int X, int G>
void backward(const Plan& P, const GnArgs& A, hipStream_t st) {
    if (P.tile_blocks > 1)
        backward_pass<X, G, true, 1>(P, A, st);
    else if (P.pieces == 1)
        backward_pass<X, G, false, 1>(P, A, st);
    else
        backward_pass<X, G, false, GN_MAX_PIECES>(P, A, st);
}

}  // namespace

extern "C" size_t fg_group_norm_workspace_bytes(int64_t max_rows, int32_t n_groups, int32_t d, int32_t channel_groups) {
    if (max_rows < 0 || max_rows > INT32_MAX || n_groups < 1 || n_groups > FG_MAX_NORM_GROUPS || d <= 0 || d > FG_MAX_NORM_DIM || channel_groups < 1 || channel_groups > d ||
        d % channel_groups)
        return 0;
    return space_of(max_rows, d, channel_groups, false).total();
}

extern "C" fg_status_t fg_group_norm(const void* x, int64_t x_stride, fg_dtype_t dtype, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows,
                                     int32_t n_groups, int64_t n, int32_t d, int32_t channel_groups, const float* weight, const float* bias, float eps,
                                     fg_act_t act, void* y, int64_t y_stride, fg_dtype_t y_dtype, float* mean_out, float* rstd_out, void* ws_dev,
                                     size_t ws_bytes, void* stream) {
    const char* who = "fg_group_norm";
    const int e = fg_dtype_size(dtype);
    if (!e) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type %d", who, (int)dtype);
    if (y_dtype != dtype && y_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: y is of the type of x or fp32", who);
    FG_TRY(check_norm(who, order_dev, offsets_dev, max_rows, n_groups, n, d, channel_groups, act));
    if (!(eps >= 0.f)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: eps must not be negative", who);
    if (max_rows > 0 && n > 0 && (!x || !y)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: x and y must not be NULL", who);
    FG_TRY(check_array(who, "x", x, x_stride, e, d));
    FG_TRY(check_array(who, "y", y, y_stride, fg_dtype_size(y_dtype), d));
    if (x == y && x && (y_dtype != dtype || y_stride != x_stride)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: y over x has its type and stride", who);
    if (((uintptr_t)weight | (uintptr_t)bias | (uintptr_t)mean_out | (uintptr_t)rstd_out) & 3)
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: weight, bias, mean or rstd is not aligned", who);
    const Space W = space_of(max_rows, d, channel_groups, false);
    FG_TRY(check_space(who, ws_dev, ws_bytes, W.total()));
    fg_clear_error();
    const Plan P = plan_of(max_rows, d, channel_groups);
    GnArgs A = args_of(P, W, order_dev, offsets_dev, max_rows, n_groups, n, d, channel_groups, ws_dev);
    A.x = (const char*)x, A.x_stride = x_stride, A.out = (char*)y, A.out_stride = y_stride, A.out_type = y_dtype, A.weight = weight, A.bias = bias, A.eps = eps, A.act = act;
    A.mean = mean_out, A.rstd = rstd_out;
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == FG_F32)
        forward<FG_F32>(P, A, st);
    else if (dtype == FG_F16)
        forward<FG_F16>(P, A, st);
    else
        forward<FG_BF16>(P, A, st);
    FG_LAUNCH_CHECK("group_norm_kernel");
    return FG_OK;
}

extern "C" size_t fg_group_norm_backward_workspace_bytes(int64_t max_rows, int32_t n_groups, int32_t d, int32_t channel_groups) {
    if (fg_group_norm_workspace_bytes(max_rows, n_groups, d, channel_groups) == 0) return 0;
    return space_of(max_rows, d, channel_groups, true).total();
}

extern "C" fg_status_t fg_group_norm_backward(const void* dy, int64_t dy_stride, fg_dtype_t grad_dtype, const void* x, int64_t x_stride, fg_dtype_t dtype,
                                              const float* mean, const float* rstd, const float* weight, const float* bias, fg_act_t act,
                                              const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups, int64_t n, int32_t d,
                                              int32_t channel_groups, void* dx, int64_t dx_stride, float* dw_dev, float* db_dev, void* ws_dev,
                                              size_t ws_bytes, void* stream) {
    const char* who = "fg_group_norm_backward";
    const int e = fg_dtype_size(dtype), ge = fg_dtype_size(grad_dtype);
    if (!e || !ge) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type", who);
    FG_TRY(check_norm(who, order_dev, offsets_dev, max_rows, n_groups, n, d, channel_groups, act));
    const bool work = max_rows > 0 && n > 0;
    if (work && (!dy || !x || !mean || !rstd || !dx)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: dy, x, mean, rstd and dx must not be NULL", who);
    FG_TRY(check_array(who, "dy", dy, dy_stride, ge, d));
    FG_TRY(check_array(who, "x", x, x_stride, e, d));
    FG_TRY(check_array(who, "dx", dx, dx_stride, ge, d));
    if (dx == dy && dx && dx_stride != dy_stride) FG_FAIL(FG_ERR_INVALID_ARG, "%s: dx over dy has its stride", who);
    if (((uintptr_t)weight | (uintptr_t)bias | (uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)dw_dev | (uintptr_t)db_dev) & 3)
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: weight, bias, mean, rstd, dw or db is not aligned", who);
    const Space W = space_of(max_rows, d, channel_groups, true);
    FG_TRY(check_space(who, ws_dev, ws_bytes, W.total()));
    fg_clear_error();
    const Plan P = plan_of(max_rows, d, channel_groups);
    GnArgs A = args_of(P, W, order_dev, offsets_dev, work ? max_rows : 0, n_groups, n, d, channel_groups, ws_dev);
    A.x = (const char*)x, A.x_stride = x_stride, A.dy = (const char*)dy, A.dy_stride = dy_stride, A.out = (char*)dx, A.out_stride = dx_stride, A.weight = weight, A.bias = bias;
    A.act = act, A.mean = const_cast<float*>(mean), A.rstd = const_cast<float*>(rstd);
    if (!dw_dev && !db_dev) A.columns = nullptr;
    const hipStream_t st = (hipStream_t)stream;
#define FG_GN(X) (grad_dtype == FG_F32 ? backward<X, FG_F32>(P, A, st) : grad_dtype == FG_F16 ? backward<X, FG_F16>(P, A, st) : backward<X, FG_BF16>(P, A, st))
    if (work) {
        if (dtype == FG_F32)
            FG_GN(FG_F32);
        else if (dtype == FG_F16)
            FG_GN(FG_F16);
        else
            FG_GN(FG_BF16);
        FG_LAUNCH_CHECK("group_norm_backward_kernel");
    }
#undef FG_GN
    if (dw_dev || db_dev) {
        hipLaunchKernelGGL(group_norm_columns_kernel, dim3((unsigned)fg_ceil_div(2 * d, 32)), dim3(GN_THREADS), 0, st, A.columns, work ? P.chunks : 0, d, dw_dev, db_dev);
        FG_LAUNCH_CHECK("group_norm_columns_kernel");
    }
    return FG_OK;
}

// fg_group_norm and its gradients: rows of a group (a graph, a node type), normalised over the rows and blocks of adjacent columns, with an activation.
//
// A group of few rows belongs to one workgroup (of four wavefronts, or of one where the groups are small): a pass for the sums, a pass for the result, whose rows come
// from registers where the group is small enough, else from the caches. A group of many rows is split: the entries of all groups are a line that is cut into
// chunks of rows, every chunk's workgroup leaves the sums of its part, a second launch goes over the rows again with what all parts come to. A workgroup takes a tile of
// whole blocks of columns; a thread has pieces of eight adjacent columns (whole ones: the last of a tile overlaps the one before it) and every so many-th row.
// Bound by memory where rows are many: 58982 listed rows x 1024 bf16 in 4 groups 76 us between calls of the same rows (48 for the bytes; statistics come before results, so the
// rows are read twice), gradients 130 of 73; 65536 x 1024 fp32 168 and 280. Many small groups are bound by what their reductions take beside their values (31744 x 100 fp32 in
// 1024 groups 16 us, 29 with cold caches, of 5 for the bytes), few rows by the latency of reads that depend on each other (777 x 88 6, gradients 10.8).
#include "activation.h"
#include "row_list.h"
#include "row_types.h"
#include "scan.h"

namespace {

constexpr int GN_THREADS = 256, GN_COLUMNS = 256;      // columns of a tile that has several blocks
constexpr int GN_PLACES = 1024, GN_UNITS = 256, GN_MOST_WORKERS = 12 * GN_UNITS, GN_FEW_WORKGROUPS = 128, GN_SMALL_STEPS = 2, GN_FEW_VALUES = 65536, GN_LEAST_VALUES = 24576;
constexpr int GN_JOIN_HERE = 4000, GN_MAX_PIECES = 8;
// Rows of a thread whose fp32 sums (the gradients', several blocks to a tile) are joined to fp64 ones: what is lost of them stays below 2^-17 however long a call is
constexpr int GN_RUN = 128;

// Workgroups of the first pass that a compute unit holds: three of those that need more registers than a fourth one would leave them. Three | four, us. fp32, several blocks:
// 31744 x 100 in 1024 groups 17.4 | 20.3, 100000 x 40 in 10000 groups 26 | 31, 200000 x 64 in 20000 groups 42 | 56, but 20000 x 256 in 40 groups 24 | 22; its gradients 36.2 | 35.7,
// 59 | 63, 84 | 92 and 35 | 33, of 65536 x 1024 in 4 groups 280 | 277; forward with one block 26 | 26 (65536 x 128 in 4096 groups). 16 bits: 65536 x 1024 in 4 groups 82 | 78, gathered
// 89 | 82, with one block 77 | 75, 8000 x 2048 in 256 blocks 48 | 31, but 31744 x 100 16 | 17 and 100000 x 40 25 | 27; gradients 146 | 143, gathered 170 | 155, with one block
// 164 | 153, 8000 x 2048 44 | 43, 100000 x 40 57 | 62.
// (16-bit rows with fp32 gradients and several blocks: four would leave them four registers short)
constexpr int gn_per_unit(int type, bool many, bool backward, bool mixed = false) { return (type == FG_F32 && (backward || many)) || (mixed && many) ? 3 : 4; }

struct GnArgs {
    const int32_t* order;      // NULL: position k itself
    const int64_t* offsets;
    int64_t max_rows, n;
    unsigned int rows, long_rows;      // rows of a chunk; a group of more rows than long_rows is split
    unsigned int block_inverse;        // 2^32 / block, rounded up
    int chunks, workers;               // workgroups of a tile that look for parts of split groups in a chunk each, and those that take whole groups
    int n_groups, d, block, blocks, width, pieces;      // columns of a block, blocks of a row, lanes of a row's tile and pieces of a lane
    const char *x, *dy;
    int64_t x_stride, dy_stride, out_stride;
    const float *weight, *bias;
    float eps;
    int act, out_type;
    char* out;
    float *mean, *rstd;      // [n_groups x blocks]; the forward call's may be NULL
    int64_t stat_stride;     // ... the gradients': group g, block j at g * stat_stride + j * stat_step
    unsigned int stat_step;
    double* part;            // [chunks][2][blocks][4]: the sums of a chunk's parts of a group that began before it, and of one that begins in it, rows and level
    int32_t* info;           // [chunks][2]: those groups, -1: none
    float* joined;           // [chunks][blocks][2]: what the parts of the group that begins in the chunk come to
    int join_there;          // ... has been left there by a launch of its own
    int joins;               // workgroups that join
    float* columns;          // [workers + chunks][2][d]: sums for dw and db, or NULL
    float *dw, *db;
};

// entries are counted in 32 bits (a call has fewer than 2^31, a step beyond them fits)
__device__ __forceinline__ unsigned int offset_of(const GnArgs& A, int g) {
    const int64_t o = A.offsets[g];
    return (unsigned int)(o < 0 ? 0 : (o > A.max_rows ? A.max_rows : o));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// A group with no more than 62 others behind it that begin before `target`, and all groups before it do (lanes of a wavefront together)
__device__ __forceinline__ int near(const GnArgs& A, unsigned int target) {
    int lo = 0, hi = A.n_groups;      // the first that does not lies in [lo, hi]
    while (hi - lo > 62) {
        const int step = (hi - lo + 63) / 64, i = lo + fg_lane() * step;
        const int before = uniform(__popcll(__ballot(i < hi && offset_of(A, i < hi ? i : lo) < target)));
        const int end = lo + before * step;
        lo += before ? (before - 1) * step + 1 : 0;
        hi = before == 0 ? lo : (end < hi ? end : hi);
    }
    return lo > 0 ? lo - 1 : 0;
}
enum { GN_WHOLE, GN_GOES_ON, GN_BEGINS };
// What a workgroup of a tile has to do: the parts of split groups in its chunk (of one that began before it, of one that begins in it), or every so many-th group
// that is not split. The same in all wavefronts.
template <bool PARTS>
struct Walk {
    const GnArgs& A;
    unsigned int c0, c1, from, to;      // entries of the chunk; of the group that this lane looks at, or of the next group
    int base;                           // the first lane's group, or the next group
    unsigned long long mask;            // lanes whose groups are still to come
    __device__ __forceinline__ Walk(const GnArgs& args, int number) : A(args) {
        mask = 0;
        from = to = 0;
        if constexpr (PARTS) {
            c0 = (number - A.workers) * A.rows;
            c1 = c0 + A.rows;
            base = near(A, c0) - 64;
        } else {
            base = number;
            look();
        }
    }
    __device__ __forceinline__ void look() {
        if (base >= A.n_groups) return;
        from = offset_of(A, base);
        to = offset_of(A, base + 1);
    }
    // The next part: group, first entry and end, which of the three
    __device__ __forceinline__ bool next(int& g, unsigned int& k0, unsigned int& k1, int& which) {
        if constexpr (!PARTS) {
            for (;;) {
                if (base >= A.n_groups) return false;
                g = base, k0 = from, k1 = to > from ? to : from;
                base += A.workers;
                look();      // (its offsets are on their way meanwhile)
                which = GN_WHOLE;
                if (k1 - k0 <= A.long_rows) return true;
            }
        } else {
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
                mask = __ballot(from < c1 && to > c0 && to > from && to - from > A.long_rows);
            }
            const int l = __ffsll((long long)mask) - 1;
            mask &= mask - 1;
            g = base + l;
            const unsigned int first = (unsigned int)__builtin_amdgcn_readlane((int)from, l), end = (unsigned int)__builtin_amdgcn_readlane((int)to, l);
            which = first < c0 ? GN_GOES_ON : GN_BEGINS;
            k0 = first < c0 ? c0 : first;
            k1 = end < c1 ? end : c1;
            return true;
        }
    }
};
__device__ __forceinline__ int position(const GnArgs& A, unsigned int k) {
    const int r = A.order ? A.order[k] : (int)k;
    return r < 0 || r >= A.n ? -1 : r;
}

// The row of the first of the entries [k0, k1) that exists, -1: none does (lanes of a wavefront together; nearly always that of k0)
__device__ __forceinline__ int first_row(const GnArgs& A, unsigned int k0, unsigned int k1) {
    int r = uniform(position(A, k0));
    for (unsigned int k = k0 + 1; r < 0 && k < k1; k += 64) {
        const int mine = k + fg_lane() < k1 ? position(A, k + fg_lane()) : -1;
        const unsigned long long there = __ballot(mine >= 0);
        if (there) r = __builtin_amdgcn_readlane(mine, __ffsll((long long)there) - 1);
    }
    return r;
}

// this workgroup's tile and this thread's share of it
struct Tile {
    int c0, cols, block0, n_blocks, p, side, sides;      // columns, blocks; piece and row of the thread, rows side by side
};
template <int TH>
__device__ __forceinline__ Tile tile_of(const GnArgs& A) {
    Tile T;
    T.block0 = (int)((int64_t)blockIdx.x * A.blocks / gridDim.x);      // (even tiles: none of fewer than a piece's columns)
    T.n_blocks = (int)((int64_t)(blockIdx.x + 1) * A.blocks / gridDim.x) - T.block0;
    T.c0 = T.block0 * A.block;
    T.cols = T.n_blocks * A.block;
    T.p = (int)threadIdx.x % A.width;
    T.side = (int)threadIdx.x / A.width;
    T.sides = TH / A.width;
    return T;
}

// A thread's i-th piece of eight columns. The last one of a tile ends where the tile does: its first `twice` columns are the neighbour's, who has them in
// the sums and writes them.
struct Piece {
    int c, twice;
    bool there;
};
__device__ __forceinline__ Piece piece_of(const GnArgs& A, const Tile& T, int i) {
    const int c = (T.p + A.width * i) * 8;
    Piece P;
    P.there = c < T.cols;
    P.c = c + 8 <= T.cols ? c : T.cols - 8;
    P.twice = P.there ? c - P.c : 8;
    return P;
}
// all eight values, wherever the row begins
template <int T>
__device__ __forceinline__ fg_piece<T> load_piece(const char* row, int c) {
    return fg_load_piece<T>(row + (int64_t)c * (T == FG_F32 ? 4 : 2), 8);
}
template <int T>
__device__ __forceinline__ void store_piece(char* row, const Piece& P, const float (&f)[8]) {
    char* to = row + (int64_t)P.c * (T == FG_F32 ? 4 : 2);
    if (P.twice == 0) return fg_store_piece<T>(to, f, 8);
    const fg_piece<T> v = fg_to_piece<T>(f);
#pragma unroll
    for (int e = 1; e < 8; ++e)
        if (e >= P.twice) {
            if constexpr (T == FG_F32)
                ((float*)to)[e] = f[e];
            else
                ((unsigned short*)to)[e] = (unsigned short)(v.a[e / 2] >> (16 * (e & 1)));
        }
}

template <int TH, bool MANY>
struct Scratch {
    static constexpr int COLUMNS = MANY ? GN_COLUMNS : 1;
    double wave[TH / 64][2 * COLUMNS];      // sums of a wavefront's rows, by column; one block to a tile: of all columns
    float from[COLUMNS];                    // what they are measured from
    float stats[COLUMNS][2];                // of a block: mean and rstd, or the gradient's two means
    int rows[TH / 64];
};
// The sums s[e], q[e] of a thread's columns (MANY) or s[0], q[0] of all it has seen, over the rows that a wavefront has side by side, and the number of rows;
// they are there after the workgroup's next barrier. Halves of the wavefront exchange half of their sums each: 16 fp64 sums over four rows take 24 exchanges between
// registers instead of 64 through LDS. `more` (MANY): they are added to what is there.
template <int TH, bool MANY, typename V>
__device__ __forceinline__ void leave_sums(const GnArgs& A, const Tile& T, Scratch<TH, MANY>& S, V (&s)[MANY ? 8 : 1], V (&q)[MANY ? 8 : 1], int rows, bool more = false) {
    for (int off = A.width; off < 64; off <<= 1) rows += __shfl_xor(rows, off, 64);
    if (fg_lane() == 0) S.rows[fg_wave()] = rows;
    if constexpr (MANY) {
        const Piece P = piece_of(A, T, 0);
        double* const to = S.wave[fg_wave()] + P.c;
        const auto put = [&](int at, V v) { to[at] = more ? to[at] + (double)v : (double)v; };
        static_assert(GN_COLUMNS / 8 <= 32, "a tile of several blocks has rows side by side in a wavefront");
        V v[8];      // of s in the first half of the wavefront, of q in the second
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = half_sums<32>(s[e], q[e]);
        const int base = fg_lane() < 32 ? 0 : GN_COLUMNS;
        if (A.width == 32) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= P.twice) put(base + e, v[e]);
            return;
        }
        const int e0 = fg_lane() & 16 ? 4 : 0;      // four columns of the piece
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = half_sums<16>(v[e], v[e + 4]);
            for (int off = A.width; off < 16; off <<= 1) v[e] += __shfl_xor(v[e], off, 64);
        }
        if ((fg_lane() & 15) < A.width)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e0 + e >= P.twice) put(base + e0 + e, v[e]);
    } else {
        V v = half_sums<32>(s[0], q[0]);
        for (int off = 1; off < 32; off <<= 1) v += __shfl_xor(v, off, 64);
        if ((fg_lane() & 31) == 0) S.wave[fg_wave()][fg_lane() ? 1 : 0] = (double)v;
    }
}
template <int TH, bool MANY>
__device__ __forceinline__ int rows_of(const GnArgs& A, const Scratch<TH, MANY>& S) {
    int all = 0;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) all += S.rows[w];
    return A.width > 64 ? all / (A.width / 64) : all;      // (every wavefront of a row has counted it)
}
// done(block of the tile, s, q) by one thread of every block, of the sums over its columns; column(c, s, q) makes of a column's what is to be added
template <int TH, bool MANY, typename Column, typename Done>
__device__ __forceinline__ void block_sums(const GnArgs& A, const Tile& T, const Scratch<TH, MANY>& S, const Column& column, const Done& done) {
    const auto both = [&](int c, double& a, double& b) {
        double s = 0.0, q = 0.0;
#pragma unroll
        for (int w = 0; w < TH / 64; ++w) s += S.wave[w][c], q += S.wave[w][S.COLUMNS + c];
        column(c, s, q);
        a += s, b += q;
    };
    double a = 0.0, b = 0.0;
    if constexpr (MANY) {
        int lanes = 1;      // of a block
        while (lanes < 64 && lanes * 2 * T.n_blocks <= TH) lanes *= 2;
        for (int j0 = 0; j0 < T.n_blocks; j0 += TH / lanes) {
            const int j = j0 + (int)threadIdx.x / lanes, l = (int)threadIdx.x % lanes;
            a = b = 0.0;
            if (j < T.n_blocks)
                for (int c = j * A.block + l; c < (j + 1) * A.block; c += lanes) both(c, a, b);
            for (int off = lanes >> 1; off > 0; off >>= 1) {
                a += __shfl_xor(a, off, 64);
                b += __shfl_xor(b, off, 64);
            }
            if (j < T.n_blocks && l == 0) done(j, a, b);
        }
    } else if (threadIdx.x == 0) {
        both(0, a, b);
        done(0, a, b);
    }
}
__device__ __forceinline__ void write_part(const GnArgs& A, const Tile& T, int chunk, int which, int j, double s, double q, int rows, float level) {
    double* to = A.part + ((int64_t)(chunk * 2 + (which == GN_BEGINS)) * A.blocks + T.block0 + j) * 4;
    to[0] = s, to[1] = q, to[2] = (double)rows, to[3] = (double)level;
}
__device__ __forceinline__ void note(const GnArgs& A, int chunk, int goes_on, int begins) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && chunk >= 0) A.info[chunk * 2] = goes_on, A.info[chunk * 2 + 1] = begins;
}
// the block of a tile's column
__device__ __forceinline__ int block_of(const GnArgs& A, int c) { return A.block == 1 ? c : (int)__umulhi((unsigned int)c, A.block_inverse); }
// the two values of S.stats for each of a piece's columns
template <int TH, bool MANY>
__device__ __forceinline__ void stats_of(const GnArgs& A, const Scratch<TH, MANY>& S, int c, float (&first)[8], float (&second)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int j = MANY ? block_of(A, c + e) : 0;
        first[e] = S.stats[j][0], second[e] = S.stats[j][1];
    }
}
// 1 / x and 1 / sqrt(x) to within a few steps of 2^-52: the hardware's estimates and Newton's steps (a division and a root take longer than the rest of a
// small group's statistics)
__device__ __forceinline__ double reciprocal(double x) {
    double r = __builtin_amdgcn_rcp(x);
    r = fma(fma(-x, r, 1.0), r, r);
    return fma(fma(-x, r, 1.0), r, r);
}
__device__ __forceinline__ double reciprocal_root(double x) {
    double r = __builtin_amdgcn_rsq(x);
    if (!(x > 0.0 && x < INFINITY)) return r;
    r = fma(fma(-x * r, r, 1.0), 0.5 * r, r);
    return fma(fma(-x * r, r, 1.0), 0.5 * r, r);
}
__device__ __forceinline__ void mean_rstd(const GnArgs& A, float from, double s, double q, double rows, float& mean, float& rstd) {
    const double per = reciprocal(rows > 0.0 ? rows * A.block : 1.0), m = s * per, v = q * per - m * m;
    mean = (float)((double)from + m);
    rstd = (float)reciprocal_root((v > 0.0 || !(v == v) ? v : 0.0) + (double)A.eps);
}
__device__ __forceinline__ void put_statistics(const GnArgs& A, const Tile& T, int g, int j, float mean, float rstd) {
    const int64_t at = (int64_t)g * A.blocks + T.block0 + j;
    if (A.mean) A.mean[at] = mean;
    if (A.rstd) A.rstd[at] = rstd;
}
// Eight values' instructions are not all mixed with each other: what they hold at once would not fit the registers. A register that is spilled to memory is more than slow here:
// the compiler has stored one inside a branch for the lanes that took it, and read it behind the branch for all
__device__ __forceinline__ void part_of_eight() { __builtin_amdgcn_sched_barrier(0); }
__device__ __forceinline__ void activate(int act, float (&u)[8]) {
    fg_with_act(act, [&](auto which) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e == 4) part_of_eight();
            u[e] = fg_act<decltype(which)::value>(u[e]);
        }
    });
}
// slopes in place of the arguments
__device__ __forceinline__ void slopes(int act, float (&u)[8]) {
    fg_with_act(act, [&](auto which) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e == 4) part_of_eight();
            float f;
            fg_act_slope<decltype(which)::value>(u[e], f, u[e]);
        }
    });
}
__device__ __forceinline__ void affine(const GnArgs& A, const Tile& T, int c, float (&w)[8], float (&b)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.f, b[e] = 0.f;
    if (A.weight) fg_piece_values<FG_F32>(load_piece<FG_F32>((const char*)A.weight, T.c0 + c), w);
    if (A.bias) fg_piece_values<FG_F32>(load_piece<FG_F32>((const char*)A.bias, T.c0 + c), b);
}

// The rows of the entries [k0, k1) that this thread has: load(row or -1), then use(row) if it exists; `now`: the last one. The next position is fetched beside the row.
// (Two rows on their way: forward 17.5 us for 31744 x 100 fp32 in 1024 groups, one 16.0; 65536 listed rows x 1024 bf16 in 4 groups 82 | 80, with one block 81 | 76; only
// 200000 x 64 fp32 in 20000 groups 42 | 44; gradients of the first three 37.0 | 36.0, 163 | 155, 167 | 161.)
template <typename Load, typename Use>
__device__ __forceinline__ void for_rows(const GnArgs& A, const Tile& T, unsigned int k0, unsigned int k1, int& now, const Load& load, const Use& use) {
    const auto fetch = [&](unsigned int k) { return k < k1 ? position(A, k) : -1; };
    int next = fetch(k0 + T.side);
    for (unsigned int k = k0 + T.side; k < k1; k += T.sides) {
        now = next;
        load(now);
        next = fetch(k + T.sides);
        if (now >= 0) use(now);
    }
}

// y of the entries [k0, k1) with the blocks' mean and rstd in S.stats. held: `now`, v are all of them and there already
template <int TH, int T_, bool MANY>
__device__ __forceinline__ void normalise(const GnArgs& A, const Tile& T, const Scratch<TH, MANY>& S, unsigned int k0, unsigned int k1, bool held, int& now,
                                          fg_piece<T_>& v) {
    for (int i = 0; i < (MANY ? 1 : A.pieces); ++i) {
        const Piece P = piece_of(A, T, i);
        if (!P.there) break;
        float w[8], b[8], mean[8], rstd[8];
        affine(A, T, P.c, w, b);
        stats_of<TH, MANY>(A, S, P.c, mean, rstd);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] *= rstd[e];
        const auto finish = [&](int r) {
            float f[8];
            fg_piece_values<T_>(v, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = (f[e] - mean[e]) * w[e] + b[e];
            activate(A.act, f);
            char* to = A.out + (int64_t)r * A.out_stride;
            if (A.out_type == FG_F32)
                store_piece<FG_F32>(to + T.c0 * 4, P, f);
            else if constexpr (T_ != FG_F32)
                store_piece<T_>(to + T.c0 * 2, P, f);
        };
        if (held) {
            if (now >= 0) finish(now);
        } else {
            for_rows(
                A, T, k0, k1, now,
                [&](int r) {
                    if (r >= 0) v = load_piece<T_>(A.x + (int64_t)r * A.x_stride, T.c0 + P.c);
                },
                finish);
        }
    }
}

// PARTS: the workgroup's work is a chunk's parts of split groups, else whole groups (one kernel for both, so that neither waits for the other; two bodies, so
// that the first is not short of registers for what the second holds)
template <int TH, int T_, bool MANY, bool PARTS>
__device__ __forceinline__ void norm_body(const GnArgs& A, Scratch<TH, MANY>& S) {
    constexpr int N = MANY ? 8 : 1;
    const Tile T = tile_of<TH>(A);
    const int chunk = (int)blockIdx.y - A.workers;      // (below 0: whole groups)
    int goes_on = -1, begins = -1, g, which;
    unsigned int k0, k1;
    for (Walk<PARTS> W(A, blockIdx.y); W.next(g, k0, k1, which);) {
        if (k0 == k1) {      // a group without rows
            for (int j = threadIdx.x; j < T.n_blocks; j += TH) put_statistics(A, T, g, j, 0.f, (float)reciprocal_root((double)A.eps));
            continue;
        }
        double s[N] = {}, q[N] = {};
        int rows = 0, now = -1;
        fg_piece<T_> v;
        // all of a group's rows at once: they are read once (not fp32 ones of one block, for which there are no registers)
        const bool held = !PARTS && (MANY || T_ != FG_F32) && k1 - k0 <= (unsigned int)T.sides && (MANY || A.pieces == 1);
        // a column's values are measured from its first one in these entries (MANY), all columns' from the block's
        const int first = first_row(A, k0, k1);
        const float common = !MANY && first >= 0 ? fg_element(A.x + (int64_t)first * A.x_stride, T_, T.c0) : 0.f;
        for (int i = 0; i < (MANY ? 1 : A.pieces); ++i) {
            const Piece P = piece_of(A, T, i);
            float from[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) from[e] = common;
            if (MANY && first >= 0) fg_piece_values<T_>(load_piece<T_>(A.x + (int64_t)first * A.x_stride, T.c0 + P.c), from);
            if (MANY && T.side == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e >= P.twice) S.from[P.c + e] = from[e];
            for_rows(
                A, T, k0, k1, now,
                [&](int r) {
                    rows += r >= 0 && i == 0;
                    if (r >= 0) v = load_piece<T_>(A.x + (int64_t)r * A.x_stride, T.c0 + P.c);
                },
                [&](int) {
                    float f[8];
                    fg_piece_values<T_>(v, f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (e % 2 == 0) part_of_eight();
                        const double x = MANY || e >= P.twice ? (double)f[e] - (double)from[e] : 0.0;      // (MANY: a neighbour's columns are not left in the sums)
                        s[MANY ? e : 0] += x;
                        q[MANY ? e : 0] += x * x;
                    }
                });
        }
        leave_sums<TH, MANY>(A, T, S, s, q, rows);
        __syncthreads();
        rows = rows_of(A, S);
        block_sums<TH, MANY>(
            A, T, S,
            [&](int c, double& a, double& b) {      // from the column's level to the block's
                if constexpr (MANY) {
                    const double up = (double)S.from[c] - (double)S.from[block_of(A, c) * A.block];
                    b += up * (2.0 * a + rows * up);
                    a += rows * up;
                }
            },
            [&](int j, double a, double b) {
                const float level = MANY ? S.from[j * A.block] : common;
                if (PARTS) return write_part(A, T, chunk, which, j, a, b, rows, level);
                float mean, rstd;
                mean_rstd(A, level, a, b, (double)rows, mean, rstd);
                S.stats[j][0] = mean, S.stats[j][1] = rstd;
                put_statistics(A, T, g, j, mean, rstd);
            });
        __syncthreads();      // (the sums have been read: the next group's may be left there, and its statistics behind the next barrier)
        if constexpr (!PARTS)
            normalise<TH, T_, MANY>(A, T, S, k0, k1, held, now, v);
        else
            (which == GN_BEGINS ? begins : goes_on) = g;
    }
    if constexpr (PARTS) note(A, chunk, goes_on, begins);
}
template <int TH, int T_, bool MANY>
__global__ __launch_bounds__(TH, gn_per_unit(T_, MANY, false)) void group_norm_kernel(GnArgs A) {
    __shared__ Scratch<TH, MANY> S;
    if ((int)blockIdx.y < A.workers)
        norm_body<TH, T_, MANY, false>(A, S);
    else
        norm_body<TH, T_, MANY, true>(A, S);
}

// The sums of all parts of the split group that begins in a chunk, in order, measured from the level of the first part that has rows: lanes of a wavefront together.
// (LEVELS: a part's sums are measured from a level of its own)
template <bool LEVELS>
__device__ __forceinline__ void join(const GnArgs& A, int g, unsigned int begin, int block, double& s, double& q, double& rows, double& level) {
    const unsigned int last = (offset_of(A, g + 1) - 1) / A.rows;
    s = q = rows = level = 0.0;
    bool known = false;
    for (unsigned int c0 = begin; c0 <= last; c0 += 64) {
        const unsigned int c = c0 + fg_lane();
        double part[4] = {0.0, 0.0, 0.0, 0.0};
        if (c <= last) {
            const double* p = A.part + ((int64_t)(c * 2 + (c == begin)) * A.blocks + block) * 4;
#pragma unroll
            for (int i = 0; i < (LEVELS ? 4 : 3); ++i) part[i] = p[i];
        }
        if constexpr (LEVELS) {
            const unsigned long long there = __ballot(part[2] > 0.0);
            if (!known && there) level = __shfl(part[3], __ffsll((long long)there) - 1, 64), known = true;
            const double up = part[2] > 0.0 ? part[3] - level : 0.0, values = part[2] * A.block;
            part[1] += up * (2.0 * part[0] + values * up);
            part[0] += values * up;
        }
        s += part[0], q += part[1], rows += part[2];
    }
    for (int off = 32; off > 0; off >>= 1) {
        s += __shfl_xor(s, off, 64);
        q += __shfl_xor(q, off, 64);
        rows += __shfl_xor(rows, off, 64);
    }
}
// what the parts come to, and the forward call's results
template <int T_, bool BACKWARD>
__device__ __forceinline__ void joined(const GnArgs& A, int g, unsigned int begin, int block, bool write, float& a, float& b) {
    double s, q, rows, level;
    join<!BACKWARD>(A, g, begin, block, s, q, rows, level);
    if constexpr (BACKWARD) {
        const double per = reciprocal(rows > 0.0 ? rows * A.block : 1.0);
        a = (float)(s * per), b = (float)(q * per);
    } else {
        mean_rstd(A, (float)level, s, q, rows, a, b);      // (as it was left with the sums: y may be written over x meanwhile)
        if (write && fg_lane() == 0) {
            if (A.mean) A.mean[(int64_t)g * A.blocks + block] = a;
            if (A.rstd) A.rstd[(int64_t)g * A.blocks + block] = b;
        }
    }
}
// dw and db: the chunks' sums added up in fp64, in order; 32 columns a workgroup, eight runs of chunks side by side
__device__ __forceinline__ void column_sums(const GnArgs& A, int block, double* red) {
    const int c = block * 32 + ((int)threadIdx.x & 31);
    double s = 0.0;
    if (c < 2 * A.d)
#pragma unroll 8
        for (int64_t i = threadIdx.x >> 5; i < A.chunks + A.workers; i += GN_THREADS / 32) s += (double)A.columns[i * 2 * A.d + c];
    red[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 32 && c < 2 * A.d) {
        for (int i = 1; i < GN_THREADS / 32; ++i) s += red[threadIdx.x + 32 * i];
        float* to = c < A.d ? A.dw : A.db;
        if (to) to[c < A.d ? c : c - A.d] = (float)s;
    }
}
// The launch between the two passes, a wavefront to a block of columns of every split group. The workgroups behind those sum dw and db
template <int T_, bool BACKWARD>
__global__ __launch_bounds__(GN_THREADS) void group_norm_join_kernel(GnArgs A) {
    __shared__ double red[BACKWARD ? GN_THREADS : 1];
    if (BACKWARD && (int)blockIdx.x >= A.joins) return column_sums(A, (int)blockIdx.x - A.joins, red);
    const int per_chunk = (A.blocks + GN_THREADS / 64 - 1) / (GN_THREADS / 64);
    const unsigned int chunk = blockIdx.x / per_chunk;
    const int j = (int)(blockIdx.x % per_chunk) * (GN_THREADS / 64) + fg_wave();
    const int g = A.info[chunk * 2 + 1];
    if (g < 0 || j >= A.blocks) return;
    float a, b;
    joined<T_, BACKWARD>(A, g, chunk, j, true, a, b);
    if (fg_lane() == 0) *(float2*)(A.joined + ((int64_t)chunk * A.blocks + j) * 2) = float2{a, b};
}

// a chunk's parts of split groups: f(group, first entry, end) with what their parts come to in S.stats
template <int T_, bool MANY, bool BACKWARD, typename F>
__device__ __forceinline__ void split_parts(const GnArgs& A, const Tile& T, Scratch<GN_THREADS, MANY>& S, const F& f) {
    const unsigned int chunk = A.chunks - 1 - blockIdx.y, c0 = chunk * A.rows, c1 = c0 + A.rows;      // the last chunks' rows are the likeliest to be cached
    for (int which = 0; which < 2; ++which) {
        const int g = A.info[chunk * 2 + which];
        if (g < 0) continue;
        const unsigned int from = offset_of(A, g), to = offset_of(A, g + 1), begin = from / A.rows;
        if (A.join_there) {
            for (int j = threadIdx.x; j < T.n_blocks; j += GN_THREADS) {
                const float* p = A.joined + ((int64_t)begin * A.blocks + T.block0 + j) * 2;
                S.stats[j][0] = p[0], S.stats[j][1] = p[1];
            }
        } else {
            for (int j = fg_wave(); j < T.n_blocks; j += GN_THREADS / 64) {
                float a, b;
                joined<T_, BACKWARD>(A, g, begin, T.block0 + j, which == 1, a, b);
                if (fg_lane() == 0) S.stats[j][0] = a, S.stats[j][1] = b;
            }
        }
        __syncthreads();
        f(g, from > c0 ? from : c0, to < c1 ? to : c1);
        __syncthreads();
    }
}
template <int T_, bool MANY>
__global__ __launch_bounds__(GN_THREADS, 4) void group_norm_apply_kernel(GnArgs A) {
    __shared__ Scratch<GN_THREADS, MANY> S;
    const Tile T = tile_of<GN_THREADS>(A);
    split_parts<T_, MANY, false>(A, T, S, [&](int, unsigned int k0, unsigned int k1) {
        int now = -1;
        fg_piece<T_> v;
        normalise<GN_THREADS, T_, MANY>(A, T, S, k0, k1, false, now, v);
    });
}

// ---- gradients ----

// mean or rstd of a group and a block of the tile (the gradients'; the offset within a tile is one multiplication of 24 bits: with 64-bit addresses
// fp32 gradients of many small groups took 8 to 11 % longer)
__device__ __forceinline__ float given(const GnArgs& A, const Tile& T, const float* all, int g, int j) {
    const char* tile = (const char*)(all + (int64_t)g * A.stat_stride + (int64_t)T.block0 * A.stat_step);
    return *(const float*)(tile + __umul24((unsigned int)j, A.stat_step * 4));
}
// A thread's piece of the columns: what the gradients need of them
struct GradColumns {
    float mean[8], rstd[8], w[8], b[8];
};
// FOLDED: rstd * w in place of w, so that rstd is not needed beside them
template <bool MANY, bool FOLDED>
__device__ __forceinline__ void grad_columns(const GnArgs& A, const Tile& T, int g, int c, GradColumns& C) {
    affine(A, T, c, C.w, C.b);
    if (MANY) asm volatile("" : "+v"(c));      // (what the columns' blocks come to is formed here: held over the groups it takes registers that are not there)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int j = MANY ? block_of(A, c + e) : 0;
        C.mean[e] = given(A, T, A.mean, g, j), C.rstd[e] = given(A, T, A.rstd, g, j);
        if (FOLDED) C.w[e] *= C.rstd[e];
    }
}
// a row on its way, or held
template <int X, int G>
struct GradRows {
    int now = -1;
    fg_piece<X> x;
    fg_piece<G> dy;
};
// use(row, xh, t) for every row of the entries [k0, k1) that this thread has (FOLDED: use(row, x - mean, t)); held: R has all of them already
template <int X, int G, bool FOLDED, typename Use>
__device__ __forceinline__ void gradient_rows(const GnArgs& A, const Tile& T, int c, const GradColumns& C, unsigned int k0, unsigned int k1, bool held, GradRows<X, G>& R,
                                              const Use& use) {
    const auto terms = [&](int r) {
        float xh[8], t[8], slope[8];
        fg_piece_values<X>(R.x, xh);
        fg_piece_values<G>(R.dy, t);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            xh[e] -= C.mean[e];
            if (!FOLDED) xh[e] *= C.rstd[e];
            slope[e] = xh[e] * C.w[e] + C.b[e];
        }
        slopes(A.act, slope);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= slope[e];
        use(r, xh, t);
    };
    if (held) {
        if (R.now >= 0) terms(R.now);
    } else {
        for_rows(
            A, T, k0, k1, R.now,
            [&](int r) {
                if (r < 0) return;
                R.x = load_piece<X>(A.x + (int64_t)r * A.x_stride, T.c0 + c);
                R.dy = load_piece<G>(A.dy + (int64_t)r * A.dy_stride, T.c0 + c);
            },
            terms);
    }
}
// dx of the entries [k0, k1) with the blocks' two means in S.stats
template <int TH, int X, int G, bool MANY>
__device__ __forceinline__ void input_gradient(const GnArgs& A, const Tile& T, const Scratch<TH, MANY>& S, int g, unsigned int k0, unsigned int k1, bool held, GradRows<X, G>& R) {
    for (int i = 0; i < (MANY ? 1 : A.pieces); ++i) {
        const Piece P = piece_of(A, T, i);
        if (!P.there) break;
        GradColumns C;
        grad_columns<MANY, false>(A, T, g, P.c, C);
        float m1[8], m2[8];
        stats_of<TH, MANY>(A, S, P.c, m1, m2);
        gradient_rows<X, G, false>(A, T, P.c, C, k0, k1, held, R, [&](int r, const float(&xh)[8], float(&t)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = C.rstd[e] * (t[e] * C.w[e] - m1[e] - xh[e] * m2[e]);
            store_piece<G>(A.out + (int64_t)r * A.out_stride + T.c0 * (G == FG_F32 ? 4 : 2), P, t);
        });
    }
}

// The first pass: a group's sums of t and t * xh by column, which give its two means and dw and db. MANY: the columns' sums over a group's rows
// meet in LDS, a thread to a column adds them up over the chunk's groups. Else (NP pieces a thread) a thread keeps its columns' sums over all of
// the chunk's rows, and those of a group over its columns beside them in fp64. The former are in fp32 for GN_RUN rows of a part at most; with one piece they are added to
// fp64 sums in LDS then, with several, for which LDS has no room, to the range's in fp32. (All pieces' sums in registers took 400 of them: 30000 x 2500 bf16 in 3000 groups
// 553 us, 236 so; fp32 sums in LDS 251, but 2000 x 16384 fp32 269 instead of 194, as LDS holds one workgroup then.)
template <int TH, int X, int G, bool MANY, int NP, bool PARTS>
__device__ __forceinline__ void gradient_body(const GnArgs& A, Scratch<TH, MANY>& S, double* kept) {
    const Tile T = tile_of<TH>(A);
    const int chunk = (int)blockIdx.y - A.workers;      // (below 0: whole groups)
    int goes_on = -1, begins = -1, g, which;
    unsigned int k0, k1;
    if constexpr (MANY)      // a thread has every TH-th column (in registers they would be spilled)
        for (int c = threadIdx.x; c < GN_COLUMNS; c += TH) kept[c] = kept[GN_COLUMNS + c] = 0.0;
    constexpr int KEPT = TH + 8;      // (a thread's sums lie so far apart; eight more, so that a column's reader finds its neighbours' in other banks)
    unsigned int there = 0;     // pieces of which something has been kept
    float* const range = A.columns ? A.columns + (int64_t)blockIdx.y * 2 * A.d + T.c0 : nullptr;
    // a piece's sums to LDS, or to the range's
    const auto keep = [&](int i, const Piece& P, const float (&dw)[8], const float (&db)[8]) {
        const bool more = there >> i & 1;
        there |= 1u << i;
        if constexpr (NP == 1) {
            double* const at = kept + threadIdx.x;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                at[e * KEPT] = (more ? at[e * KEPT] : 0.0) + (double)dw[e];
                at[(8 + e) * KEPT] = (more ? at[(8 + e) * KEPT] : 0.0) + (double)db[e];
            }
        } else if (range) {
#pragma unroll
            for (int sum = 0; sum < 2; ++sum) {
                char* const at = (char*)(range + sum * A.d);
                float f[8] = {};
                if (more) fg_piece_values<FG_F32>(load_piece<FG_F32>(at, P.c), f);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] += sum ? db[e] : dw[e];
                store_piece<FG_F32>(at, P, f);
            }
        }
    };
    for (Walk<PARTS> W(A, blockIdx.y); W.next(g, k0, k1, which);) {
        if (k0 == k1) continue;
        GradRows<X, G> R;
        const bool held = X == G && !PARTS && k1 - k0 <= (unsigned int)T.sides && (MANY || A.pieces == 1);
        int rows = 0;
        for (unsigned int k = k0 + T.side; k < k1; k += T.sides) rows += position(A, k) >= 0;
        if constexpr (MANY) {
            for (unsigned int from = k0, to; from < k1; from = to) {
                to = k1 - from > (unsigned int)(GN_RUN * T.sides) ? from + GN_RUN * T.sides : k1;
                float s[8] = {}, q[8] = {};
                const Piece P = piece_of(A, T, 0);
                if (P.there) {
                    GradColumns C;
                    grad_columns<true, true>(A, T, g, P.c, C);
                    gradient_rows<X, G, true>(A, T, P.c, C, from, to, false, R, [&](int, const float(&x)[8], const float(&t)[8]) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) s[e] += t[e], q[e] += t[e] * x[e];
                    });
                }
                leave_sums<TH, true>(A, T, S, s, q, rows, from != k0);
            }
        } else {
            double s[1] = {}, q[1] = {};
            for (int i = 0; i < (NP == 1 ? 1 : A.pieces); ++i) {
                const Piece P = piece_of(A, T, i);
                if (!P.there) break;
                GradColumns C;
                grad_columns<false, false>(A, T, g, P.c, C);
                for (unsigned int from = k0, to; from < k1; from = to) {
                    to = k1 - from > (unsigned int)(GN_RUN * T.sides) ? from + GN_RUN * T.sides : k1;
                    float dw[8] = {}, db[8] = {};
                    gradient_rows<X, G, false>(A, T, P.c, C, from, to, false, R, [&](int, const float(&xh)[8], const float(&t)[8]) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            if (e < P.twice) continue;
                            const double a = (double)(t[e] * C.w[e]);
                            s[0] += a, q[0] += a * (double)xh[e];
                            dw[e] += t[e] * xh[e], db[e] += t[e];
                        }
                    });
                    keep(i, P, dw, db);
                }
            }
            leave_sums<TH, false>(A, T, S, s, q, rows);
        }
        __syncthreads();
        rows = rows_of(A, S);
        if constexpr (MANY)      // (rstd is still missing from the sums of t * xh)
            for (int c = threadIdx.x; c < T.cols; c += TH) {
                double s = 0.0, q = 0.0;
#pragma unroll
                for (int w = 0; w < TH / 64; ++w) s += S.wave[w][c], q += S.wave[w][GN_COLUMNS + c];
                kept[GN_COLUMNS + c] += s, kept[c] += q * (double)given(A, T, A.rstd, g, block_of(A, c));
            }
        block_sums<TH, MANY>(
            A, T, S,
            [&](int c, double& a, double& b) {
                if constexpr (MANY) {
                    const double w = A.weight ? (double)A.weight[T.c0 + c] : 1.0;
                    a *= w, b *= w;
                }
            },
            [&](int j, double a, double b) {
                if (MANY) b *= (double)given(A, T, A.rstd, g, j);
                if (PARTS) return write_part(A, T, chunk, which, j, a, b, rows, 0.f);
                const double per = reciprocal(rows > 0 ? (double)rows * A.block : 1.0);
                S.stats[j][0] = (float)(a * per), S.stats[j][1] = (float)(b * per);
            });
        __syncthreads();
        if constexpr (!PARTS)
            input_gradient<TH, X, G, MANY>(A, T, S, g, k0, k1, held, R);
        else
            (which == GN_BEGINS ? begins : goes_on) = g;
    }
    if constexpr (PARTS) note(A, chunk, goes_on, begins);
    if (!range) return;
    if constexpr (MANY) {
        for (int c = threadIdx.x; c < T.cols; c += TH) range[c] = (float)kept[c], range[A.d + c] = (float)kept[GN_COLUMNS + c];
    } else {
        const float none[8] = {};
        for (int i = 0; i < A.pieces; ++i) {
            const Piece P = piece_of(A, T, i);
            if ((NP == 1 || P.there) && !(there >> i & 1)) keep(i, P, none, none);
        }
        if constexpr (NP > 1) return;
        __syncthreads();
        for (int c = threadIdx.x; c < T.cols; c += TH) {      // rows side by side: their sums meet
            const int p = c / 8, e = c - (p * 8 + 8 <= T.cols ? p * 8 : T.cols - 8);
            const double* at = kept + e * KEPT + p;
            double w = 0.0, b = 0.0;
            for (int i = 0; i < T.sides; ++i) w += at[i * A.width], b += at[8 * KEPT + i * A.width];
            range[c] = (float)w, range[A.d + c] = (float)b;
        }
    }
}
template <int TH, int X, int G, bool MANY, int NP>
__global__ __launch_bounds__(TH, NP > 1 ? 1 : gn_per_unit(X, MANY, true, X != G)) void group_norm_backward_kernel(GnArgs A) {
    __shared__ Scratch<TH, MANY> S;
    __shared__ double kept[MANY ? 2 * GN_COLUMNS : NP > 1 ? 1 : 16 * (TH + 8)];
    if ((int)blockIdx.y < A.workers)
        gradient_body<TH, X, G, MANY, NP, false>(A, S, kept);
    else
        gradient_body<TH, X, G, MANY, NP, true>(A, S, kept);
}
// The second pass, on split groups
template <int X, int G, bool MANY>
__global__ __launch_bounds__(GN_THREADS, 4) void group_norm_backward_apply_kernel(GnArgs A) {
    __shared__ Scratch<GN_THREADS, MANY> S;
    const Tile T = tile_of<GN_THREADS>(A);
    split_parts<X, MANY, true>(A, T, S, [&](int g, unsigned int k0, unsigned int k1) {
        GradRows<X, G> R;
        input_gradient<GN_THREADS, X, G, MANY>(A, T, S, g, k0, k1, false, R);
    });
}

// How a call is cut: whole blocks of up to GN_COLUMNS columns to a tile, or one wider block. Where there are few groups and rows (fewer than GN_FEW_WORKGROUPS workgroups), tiles
// of fewer blocks (limits of 32 | 128 | 512: 777 x 88 fp32 in 9 groups 11.5 | 6.1 | 5.9 us, 2000 x 88 17.5 | 6.6 | 6.5, 500 x 512 bf16 in 4 groups 20 | 6 | 6, 2000 x 256 in 2 groups
// 15.8 | 15.2 | 13.1; their gradients 17.6 | 10.8 | 10.8, 26 | 12.6 | 12.6, 19 | 11 | 11, 17.5 | 19.2 | 17.8; those of 5000 x 88 19.1 | 19.1 | 20.4).
// Up to GN_MOST_WORKERS workgroups take whole groups in turn, four times as many as are on the chip (6 | 12 | 24 times the units: 100000 x 40 fp32 in 10000 groups 37 | 26 | 26 us,
// 300000 x 32 in 50000 groups 147 | 85 | 85, 200000 x 64 in 20000 groups 70 | 42 | 44; gradients, for which each leaves sums of dw and db, 66 | 59 | 77, 192 | 127 | 146, 112 | 84 | 104;
// those of 65536 x 128 in one block and 4096 groups 52 | 62 | 69).
// A group is not split as long as its workgroup, alone with its tile, ends with the others: up to GN_FEW_VALUES values in a tile where the groups fill the chip, fewer where
// they do not, down to GN_LEAST_VALUES. Split | whole: 5000 x 88 in 9 groups 16 | 32 us, gradients 19 | 53; 20000 x 256 in 40 groups 24 | 61, gradients 35 | 117. With no limit 777 x 88
// in 9 groups, whose launches for the parts then have nothing to do, takes 8.8 us instead of 6.1, gradients 12.7 instead of 10.8; with one of 16384 values 2000 x 88 8.6 instead of
// 6.6. If no group of max_rows rows can be split, the launches for the parts are left out.
// Chunks of rows for the split groups, with two rows a thread at least, so that all workgroups are on the chip at once (a few of them in a second turn take as long as all
// the others). Their sums are joined in a launch of its own from GN_JOIN_HERE chunks and blocks on, else by every workgroup of the second pass for itself: 8000 x 2048
// bf16 in 256 blocks 31 us against 46, 65536 x 256 in 8 blocks 32.6 against 36; 31744 x 100 in 5 blocks 19.1 against 17.5, 65536 x 256 in one block 41.4 against 39.5.
// One wavefront to a workgroup where an average group's rows are up to GN_SMALL_STEPS steps of one: 50000 x 32 in 20000 groups 35 us against 122, gradients 63 against 174;
// up to eight steps: 65536 x 128 in one block and 4096 groups 21 against 26, gradients 58 against 62, but 2000 x 88 in 9 groups 9.5 against 6.6, gradients 17 against 12.6.
struct Plan {
    int tiles, tile_blocks, width, pieces, threads, workers;
    int64_t rows, chunks, long_rows;      // chunks 0: no group can be so large that it is split
    bool join_there;
};
Plan plan_of(int64_t max_rows, int n_groups, int d, int blocks, int type, bool backward, bool mixed = false) {
    Plan P;
    const int block = d / blocks, per_tile = GN_COLUMNS / block;
    P.tiles = (int)fg_ceil_div(blocks, per_tile < 1 ? 1 : per_tile);
    int cols, pieces;
    int64_t places, least;
    for (;; P.tiles *= 2) {
        P.tile_blocks = (int)fg_ceil_div(blocks, P.tiles);
        cols = P.tile_blocks * block, pieces = (int)fg_ceil_div(cols, 8);
        P.width = 1;
        while (P.width < pieces && P.width < GN_THREADS) P.width *= 2;
        places = GN_UNITS * gn_per_unit(type, P.tile_blocks > 1, backward, mixed) / P.tiles, least = 2 * (GN_THREADS / P.width);
        if (P.tiles * 2 > blocks || blocks / (P.tiles * 2) * block < 8 || (max_rows / least + n_groups) * P.tiles > GN_FEW_WORKGROUPS) break;
    }
    P.pieces = (int)fg_ceil_div(pieces, P.width);
    const int64_t even = max_rows / places + 1, most = GN_MOST_WORKERS / P.tiles;
    P.rows = even > least ? even : least;
    const int64_t whole = (int64_t)n_groups * P.tiles, few = whole >= GN_UNITS ? GN_FEW_VALUES : GN_FEW_VALUES * whole / GN_UNITS;
    const int64_t few_rows = (few > GN_LEAST_VALUES ? few : GN_LEAST_VALUES) / cols;
    P.long_rows = P.rows > few_rows ? P.rows : few_rows;
    P.chunks = P.long_rows < max_rows ? max_rows / P.rows + 1 : 0;
    P.threads = P.width <= 64 && P.pieces == 1 && max_rows / n_groups * P.width <= 64 * GN_SMALL_STEPS ? 64 : GN_THREADS;
    P.workers = (int)(n_groups < most ? n_groups : most);
    P.join_there = P.chunks * P.tile_blocks > GN_JOIN_HERE;
    return P;
}
static_assert(FG_MAX_NORM_DIM <= GN_THREADS * 8 * GN_MAX_PIECES && FG_MAX_NORM_DIM / GN_COLUMNS * 2 <= GN_UNITS * 3, "pieces of a row; tiles");
static_assert(GN_UNITS * 4 <= GN_PLACES, "what a workspace is measured for");

// A workspace for max_rows serves fewer rows too: by the most chunks that a call can have
struct Space {
    size_t part, info, joined, columns;
    size_t total() const { return part + info + joined + columns + 16; }
};
Space space_of(int64_t max_rows, int n_groups, int d, int blocks, bool backward) {
    const int64_t chunks = max_rows < GN_PLACES ? max_rows + 1 : GN_PLACES;      // (two rows to a chunk at least, and no more chunks than places)
    Space W = {};
    W.part = fg_align_up((size_t)chunks * 2 * blocks * 4 * 8, 256);
    W.info = fg_align_up((size_t)chunks * 2 * 4, 256);
    W.joined = fg_align_up((size_t)chunks * blocks * 2 * 4, 256);
    if (backward) W.columns = (size_t)(chunks + (n_groups < GN_MOST_WORKERS ? n_groups : GN_MOST_WORKERS)) * 2 * d * 4;
    return W;
}

fg_status_t check_norm(const char* who, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups, int64_t n, int32_t d,
                       int32_t channel_groups, fg_act_t act) {
    FG_TRY(check_rows(who, nullptr, nullptr, 0, n, d));
    if (max_rows < 0 || max_rows > INT32_MAX) FG_FAIL(FG_ERR_INVALID_ARG, "%s: a number of rows is negative or too large", who);
    if (d < 8 || d > FG_MAX_NORM_DIM) FG_FAIL(FG_ERR_SHAPE, "%s: d = %d is not in 8..%d", who, d, FG_MAX_NORM_DIM);
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
    A.order = order_dev, A.offsets = offsets_dev, A.max_rows = max_rows, A.n = n, A.rows = (unsigned int)P.rows, A.long_rows = (unsigned int)P.long_rows;
    A.n_groups = n_groups, A.d = d, A.block = d / blocks, A.blocks = blocks, A.width = P.width, A.pieces = P.pieces;
    char* ws = (char*)ws_dev;
    A.part = (double*)ws;
    A.info = (int32_t*)(ws + W.part);
    A.chunks = (int)P.chunks, A.workers = P.workers;
    A.block_inverse = (unsigned int)(((1ull << 32) + A.block - 1) / A.block);
    A.joined = (float*)(ws + W.part + W.info);
    A.columns = (float*)(ws + W.part + W.info + W.joined);
    return A;
}

// workgroups that join the parts of split groups, and those that sum dw and db
int joins_of(const Plan& P, const GnArgs& A) { return (int)(P.chunks * fg_ceil_div(A.blocks, GN_THREADS / 64)); }
int sum_blocks(const GnArgs& A) { return A.columns ? (int)fg_ceil_div(2 * A.d, 32) : 0; }

template <int T, bool MANY>
void forward(const Plan& P, const GnArgs& A, hipStream_t st) {
    const dim3 grid((unsigned)P.tiles, (unsigned)(P.chunks + P.workers)), parts((unsigned)P.tiles, (unsigned)P.chunks);      // (the tiles of the same rows side by side)
    if (P.threads == 64)
        hipLaunchKernelGGL((group_norm_kernel<64, T, MANY>), grid, dim3(64), 0, st, A);
    else
        hipLaunchKernelGGL((group_norm_kernel<GN_THREADS, T, MANY>), grid, dim3(GN_THREADS), 0, st, A);
    if (P.chunks == 0) return;
    if (A.joins) hipLaunchKernelGGL((group_norm_join_kernel<T, false>), dim3((unsigned)A.joins), dim3(GN_THREADS), 0, st, A);
    hipLaunchKernelGGL((group_norm_apply_kernel<T, MANY>), parts, dim3(GN_THREADS), 0, st, A);
}
template <int X, int G, bool MANY, int NP>
void backward_pass(const Plan& P, const GnArgs& A, hipStream_t st) {
    const dim3 grid((unsigned)P.tiles, (unsigned)(P.chunks + P.workers)), parts((unsigned)P.tiles, (unsigned)P.chunks);
    if (NP == 1 && P.threads == 64)
        hipLaunchKernelGGL((group_norm_backward_kernel<64, X, G, MANY, 1>), grid, dim3(64), 0, st, A);
    else
        hipLaunchKernelGGL((group_norm_backward_kernel<GN_THREADS, X, G, MANY, NP>), grid, dim3(GN_THREADS), 0, st, A);
    if (const int sums = A.joins + sum_blocks(A)) hipLaunchKernelGGL((group_norm_join_kernel<X, true>), dim3((unsigned)sums), dim3(GN_THREADS), 0, st, A);
    if (P.chunks) hipLaunchKernelGGL((group_norm_backward_apply_kernel<X, G, MANY>), parts, dim3(GN_THREADS), 0, st, A);
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
    if (max_rows < 0 || max_rows > INT32_MAX || n_groups < 1 || n_groups > FG_MAX_NORM_GROUPS || d < 8 || d > FG_MAX_NORM_DIM || channel_groups < 1 || channel_groups > d ||
        d % channel_groups)
        return 0;
    return space_of(max_rows, n_groups, d, channel_groups, false).total();
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
    const Space W = space_of(max_rows, n_groups, d, channel_groups, false);
    FG_TRY(check_space(who, ws_dev, ws_bytes, W.total()));
    fg_clear_error();
    const Plan P = plan_of(max_rows, n_groups, d, channel_groups, dtype, false);
    GnArgs A = args_of(P, W, order_dev, offsets_dev, max_rows, n_groups, n, d, channel_groups, ws_dev);
    A.x = (const char*)x, A.x_stride = x_stride, A.out = (char*)y, A.out_stride = y_stride, A.out_type = y_dtype, A.weight = weight, A.bias = bias, A.eps = eps, A.act = act;
    A.mean = mean_out, A.rstd = rstd_out;
    A.join_there = P.join_there, A.joins = P.join_there ? joins_of(P, A) : 0;
    const hipStream_t st = (hipStream_t)stream;
    const bool many = P.tile_blocks > 1;
    if (dtype == FG_F32)
        many ? forward<FG_F32, true>(P, A, st) : forward<FG_F32, false>(P, A, st);
    else if (dtype == FG_F16)
        many ? forward<FG_F16, true>(P, A, st) : forward<FG_F16, false>(P, A, st);
    else
        many ? forward<FG_BF16, true>(P, A, st) : forward<FG_BF16, false>(P, A, st);
    FG_LAUNCH_CHECK("group_norm_kernel");
    return FG_OK;
}

extern "C" size_t fg_group_norm_backward_workspace_bytes(int64_t max_rows, int32_t n_groups, int32_t d, int32_t channel_groups) {
    if (fg_group_norm_workspace_bytes(max_rows, n_groups, d, channel_groups) == 0) return 0;
    return space_of(max_rows, n_groups, d, channel_groups, true).total();
}

extern "C" fg_status_t fg_group_norm_backward(const void* dy, int64_t dy_stride, fg_dtype_t grad_dtype, const void* x, int64_t x_stride, fg_dtype_t dtype,
                                              const float* mean, const float* rstd, int64_t stat_stride, int64_t stat_step, const float* weight,
                                              const float* bias, fg_act_t act, const int32_t* order_dev, const int64_t* offsets_dev,
                                              int64_t max_rows, int32_t n_groups, int64_t n, int32_t d, int32_t channel_groups, void* dx, int64_t dx_stride,
                                              float* dw_dev, float* db_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    const char* who = "fg_group_norm_backward";
    const int e = fg_dtype_size(dtype), ge = fg_dtype_size(grad_dtype);
    if (!e) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type %d", who, (int)dtype);
    if (grad_dtype != dtype && grad_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: the gradients are of the type of x or fp32", who);
    FG_TRY(check_norm(who, order_dev, offsets_dev, max_rows, n_groups, n, d, channel_groups, act));
    const bool work = max_rows > 0 && n > 0;
    if (work && (!dy || !x || !mean || !rstd || !dx)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: dy, x, mean, rstd and dx must not be NULL", who);
    FG_TRY(check_array(who, "dy", dy, dy_stride, ge, d));
    FG_TRY(check_array(who, "x", x, x_stride, e, d));
    FG_TRY(check_array(who, "dx", dx, dx_stride, ge, d));
    static_assert(GN_COLUMNS <= 1 << 24 && (int64_t)GN_COLUMNS * FG_MAX_NORM_GROUPS * 2 * 4 <= 1ll << 31 && FG_MAX_NORM_GROUPS * 2 * 4 < 1 << 24, "offsets within a tile");
    if (stat_stride < 0 || stat_step < 0 || stat_stride > INT32_MAX || stat_step > 2 * FG_MAX_NORM_GROUPS)
        FG_FAIL(FG_ERR_SHAPE, "%s: a stride of mean and rstd is negative or too large", who);
    if (dx == dy && dx && dx_stride != dy_stride) FG_FAIL(FG_ERR_INVALID_ARG, "%s: dx over dy has its stride", who);
    if (((uintptr_t)weight | (uintptr_t)bias | (uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)dw_dev | (uintptr_t)db_dev) & 3)
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: weight, bias, mean, rstd, dw or db is not aligned", who);
    const Space W = space_of(max_rows, n_groups, d, channel_groups, true);
    FG_TRY(check_space(who, ws_dev, ws_bytes, W.total()));
    fg_clear_error();
    const Plan P = plan_of(max_rows, n_groups, d, channel_groups, dtype, true, grad_dtype != dtype);
    GnArgs A = args_of(P, W, order_dev, offsets_dev, work ? max_rows : 0, n_groups, n, d, channel_groups, ws_dev);
    A.x = (const char*)x, A.x_stride = x_stride, A.dy = (const char*)dy, A.dy_stride = dy_stride, A.out = (char*)dx, A.out_stride = dx_stride, A.weight = weight, A.bias = bias;
    A.act = act, A.mean = const_cast<float*>(mean), A.rstd = const_cast<float*>(rstd);
    A.stat_stride = stat_stride, A.stat_step = (unsigned int)stat_step;
    A.dw = dw_dev, A.db = db_dev;
    if (!dw_dev && !db_dev) A.columns = nullptr;
    A.join_there = 1, A.joins = work ? joins_of(P, A) : 0;      // (beside the sums of dw and db)
    if (!work) A.chunks = A.workers = 0;
    const hipStream_t st = (hipStream_t)stream;
    if (work) {
        if (dtype == FG_F32)
            backward<FG_F32, FG_F32>(P, A, st);
        else if (dtype == FG_F16)
            grad_dtype == FG_F32 ? backward<FG_F16, FG_F32>(P, A, st) : backward<FG_F16, FG_F16>(P, A, st);
        else
            grad_dtype == FG_F32 ? backward<FG_BF16, FG_F32>(P, A, st) : backward<FG_BF16, FG_BF16>(P, A, st);
        FG_LAUNCH_CHECK("group_norm_backward_kernel");
    }
    if (!work && A.columns) {
        hipLaunchKernelGGL((group_norm_join_kernel<FG_F32, true>), dim3((unsigned)sum_blocks(A)), dim3(GN_THREADS), 0, st, A);
        FG_LAUNCH_CHECK("group_norm_join_kernel");
    }
    return FG_OK;
}

// fg_linear_grouped and its gradients: the dense update with a weight matrix per group of rows.
//
// The rows of a group lie behind each other in `order`; how many there are is known on the device only. The grid is sized for the
// bound (every group may leave one tile partly filled), and a workgroup finds its group and its rows from the offsets.
#include <type_traits>

#include "row_types.h"
#include "scan.h"

namespace {

struct Groups {
    const int32_t* order;      // NULL: position k itself
    const int64_t* offsets;
    int64_t max_rows;
    int n_groups;
};
__device__ __forceinline__ int64_t group_offset(const Groups& G, int g) {
    const int64_t o = G.offsets[g];
    return o < 0 ? 0 : (o > G.max_rows ? G.max_rows : o);
}
// tile number `tile` of rows (`size` of one group each): its group and its entries [k0, k1); false: there are fewer tiles
template <typename OffsetOf>
__device__ __forceinline__ bool find_tile(const Groups& G, const OffsetOf& offset, int64_t tile, int size, int& group, int64_t& k0, int64_t& k1) {
    int64_t before = 0;
    for (int base = 0; base < G.n_groups; base += 64) {
        const int g = base + fg_lane();
        int64_t from = 0, to = 0;
        if (g < G.n_groups) {
            from = offset(g);
            to = offset(g + 1);
        }
        const int tiles = to > from ? (int)((to - from + size - 1) / size) : 0;
        const int incl = fg_wave_scan(tiles);
        const int64_t at = tile - before - (incl - tiles);
        const unsigned long long here = __ballot(at >= 0 && at < tiles);
        if (here) {
            const int l = __ffsll((long long)here) - 1;
            group = base + l;
            const int64_t first = from + at * size, last = to;
            k0 = __shfl(first, l, 64);
            const int64_t end = __shfl(last, l, 64);
            k1 = k0 + size < end ? k0 + size : end;
            return true;
        }
        before += __shfl(incl, 63, 64);
    }
    return false;
}
__device__ __forceinline__ bool find_tile(const Groups& G, int64_t tile, int size, int& group, int64_t& k0, int64_t& k1) {
    return find_tile(G, [&](int g) { return group_offset(G, g); }, tile, size, group, k0, k1);
}

enum { GL_A_SOURCE = 0, GL_A_POSITION = 1, GL_A_ENTRY = 2 };      // rows of the left operand: by x row, by position, packed in entry order

struct GlArgs {
    Groups G;
    const char *x, *W, *h, *dh;
    int64_t x_rows, x_stride, h_stride, dh_stride, n, out_stride;
    int dh_type, h_type, out_type, d_in, d_out, relu, tiles_n;
    const float *x_scale, *w_scale, *bias;
    const int32_t* src_ids;
    char* out;
    float *dw, *db;
    // the matrix core kernels: out[r, 0:N] = a[., 0:K] . B, K and N whichever way round the call has them
    const char* a;
    int64_t a_stride;
    int a_by, K, N;
    // gradients: dz in entry order (or NULL: dh serves as it is) and its row stride, column sums by tile, parts of dW and the ranges of rows they are made of
    char* dz;
    int64_t dz_stride;
    float *db_part, *dw_part;
    int ranges;
    int sums;                 // workgroups that sum parts of dW
    int64_t db_tiles;         // tiles that have column sums
};
// position and row of x of entry k; -1: skipped
__device__ __forceinline__ void entry(const GlArgs& A, int64_t k, int64_t k1, int32_t& r, int32_t& s) {
    r = s = -1;
    if (k >= k1) return;
    r = A.G.order ? A.G.order[k] : (int32_t)k;
    if (r < 0 || r >= A.n) r = -1;
    if (r >= 0) s = A.src_ids ? A.src_ids[r] : r;
    if (s < 0 || s >= A.x_rows) r = s = -1;
}
// ---- products on the matrix cores ----
//
// A workgroup owns a BM x BN tile of one group's rows; K is walked in steps of 128 bytes of a row (32 floats, 64 halfwords, 128 values of 8
// bits: narrower pieces of a row come at a lower rate, 64 bytes a step measured 8 % slower). The operands of a step go from memory straight to
// LDS (global_load_lds, 16 bytes a lane) into one of two buffers. A wavefront reads the operands of its next matrix instructions from LDS
// while it issues the current ones, over the end of a step too: there it waits for its loads of the next step, meets the others, and sends the
// loads of the step after that into the buffer that all have then read. One barrier a step. A ring of three or four half as deep
// buffers was no faster: a step's arithmetic is longer than a load. Workgroups stay and go from tile to tile; the first loads of the next tile
// are on their way while a tile is written.
// A lane's place in LDS is fixed by the instruction (base + 16 bytes per lane), so the exchange of 16-byte pieces that keeps the operand reads
// off each other's banks is made on the side of memory: piece c of LDS row m holds piece c ^ (m / 2 & 7) of the row (a 16-byte read takes
// the lanes in groups of sixteen: 0-3, 12-15, 20-23, 24-27 and so on; 256 bytes of banks). B is either read the same way (rows of W along K:
// gradients, 8 bits), or its rows are k and transposed on the way out of LDS (ds_read_b64_tr_b16), with the 64-byte windows of a row exchanged so
// that the four rows a read takes a window of lie in different banks.
// Every lane's address is valid: a row or column that does not exist reads the first one there is (its products go to outputs that are
// not stored), pieces beyond K are read from 16 bytes of zeros, both operands'.
//
// The waits are counted by hand: the compiler knows nothing of these loads (it would wait for all of them before every LDS read).
//
// fp32: every product of two values is formed on the bf16 matrix cores from the exact split of both into three bf16 terms (x1 = bf16(x), x2 =
// bf16(x - x1), x3 = bf16(x - x1 - x2)): the six products a_i * b_j with i + j <= 4, the leading ones in a running sum of their own, as in
// fg_linear. The values lie in LDS as they are and are split as they are read: the split costs about the vector instructions that the
// products cost matrix instructions.
//
// Measured: 368640 x 768 x 1024 fp16 710 us (0.82 PFLOP/s, 1.07 at K = 4096; a large library product 1.31), 58982 x 1024 x 1024 8 bits to bf16 130 us
// (0.95 PFLOP/s), 54067 x 100 x 256 fp32 39 us (2.0 TB/s of its bytes), 256 x 64 x 64 fp32 6 us (latency). What bounds the large ones: the loop runs at
// 2.0 us for the 1.15 us that its matrix instructions take by themselves and the 0.85 us that LDS is busy with them; tiles of 256 x 256 on four
// wavefronts, with a third fewer LDS reads, took 1010 us instead of 702 (nothing fills the waits of a lone wavefront), tiles of 128 x 256 two
// to a compute unit 12 % longer.
__device__ __attribute__((aligned(16))) unsigned int gl_zero[4];
// where the lanes of a store write that have nothing to write (never read)
__device__ __attribute__((aligned(16))) unsigned int gl_sink[4 * 64];

typedef float gl_f32x16 __attribute__((ext_vector_type(16)));
typedef short gl_s16x4 __attribute__((ext_vector_type(4)));

// an address that is the same in all lanes, in scalar registers
__device__ __forceinline__ const char* uniform(const char* p) {
    const uint64_t v = (uint64_t)(uintptr_t)p;
    return (const char*)(uintptr_t)(((uint64_t)(unsigned int)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (unsigned int)__builtin_amdgcn_readfirstlane((int)v));
}
// 16 bytes a lane from memory to LDS, from such an address and an offset below 2^31, or from an address of the lane's own. M0, which holds the place in LDS, is not
// the statement's to change (the compiler takes no such register as overwritten): it is put back.
__device__ __forceinline__ void load_to_lds(const char* base, unsigned int offset, unsigned int lds) {
    unsigned int was;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0" : "=&s"(was) : "s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(const char* from, unsigned int lds) {
    unsigned int was;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0" : "=&s"(was) : "s"(lds), "v"(from) : "memory");
}
// A store that is counted by hand as well: it is issued whatever the lanes have to write
__device__ __forceinline__ void store_16(char* to, fg_u32x4 v) { asm volatile("global_store_dwordx4 %0, %1, off\n\ts_nop 1" ::"v"(to), "v"(v) : "memory"); }
// Every wavefront's loads but the N youngest of each have arrived, and all have what they have read from LDS before
template <int N>
__device__ __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// 8-bit values become bf16, which holds every one of them, and are multiplied as such (two instructions to an operand's 16 bytes), with sums in fp32
// throughout. The 8-bit matrix instructions are not used: they add groups of eight adjacent products with 13 bits below the largest of the group
// (measured: of 2^16 and 1 in one group the 1 is lost), so that of a row with a large value in every eight the others are lost, and where the large
// products cancel nothing of the result is right. They would take 84 us instead of 120 for 58982 x 1024 x 1024 to bf16 with 16 groups.
template <int T>
__device__ __forceinline__ gl_f32x16 mfma(const fg_u32x4* a, const fg_u32x4* b, gl_f32x16 c) {
    if constexpr (T == FG_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(fg_f16x8, a[0]), __builtin_bit_cast(fg_f16x8, b[0]), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(fg_bf16x8, a[0]), __builtin_bit_cast(fg_bf16x8, b[0]), c, 0, 0, 0);
    if constexpr (T == FG_E4M3) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(fg_bf16x8, a[1]), __builtin_bit_cast(fg_bf16x8, b[1]), c, 0, 0, 0);
    return c;
}
// sixteen 8-bit values as twice eight bf16
__device__ __forceinline__ void widen(fg_u32x4 v, fg_u32x4 (&out)[2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[i / 2][(i & 1) * 2] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], 1.f, false));
        out[i / 2][(i & 1) * 2 + 1] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], 1.f, true));
    }
}

typedef float gf_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 gf_bf16x2 __attribute__((ext_vector_type(2)));

// four values -> two words of each of their three terms
__device__ __forceinline__ void split4(fg_u32x4 v, fg_u32x2 (&u)[3]) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        gf_f32x2 x = {__uint_as_float(v[2 * p]), __uint_as_float(v[2 * p + 1])};
#pragma unroll
        for (int term = 0; term < 3; ++term) {
            u[term][p] = __builtin_bit_cast(unsigned int, __builtin_convertvector(x, gf_bf16x2));
            x = gf_f32x2{x[0] - __uint_as_float(u[term][p] << 16), x[1] - __uint_as_float(u[term][p] & 0xFFFF0000u)};
        }
    }
}

// eight values -> their three terms
__device__ __forceinline__ void split8(const fg_u32x4 (&v)[2], fg_u32x4 (&u)[3]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        fg_u32x2 w[3];
        split4(v[h], w);
#pragma unroll
        for (int term = 0; term < 3; ++term) u[term][2 * h] = w[term][0], u[term][2 * h + 1] = w[term][1];
    }
}

constexpr int GL_STEP = 128, GL_PIECES = GL_STEP / 16, GL_ROWS = 1024 / GL_STEP;      // bytes of K per step; 16-byte pieces of a row; rows of a load
constexpr int EP_BLOCK = 16 * 128;      // bytes of an epilogue's block
// the operands' two buffers, the epilogue's blocks, what belongs to a tile (twice), the offsets
constexpr size_t gl_lds_bytes(int bm, int bn, int waves, bool eight, int n_groups) {
    return (size_t)2 * (bm + bn) * GL_STEP + (size_t)waves * EP_BLOCK + (size_t)2 * (8 * bm + 4 * bn + (eight ? 4 * (bm + bn) : 32)) + (size_t)(n_groups + 1) * 4;
}
// A sum of 8-bit products times the scales of its row and its column, the smaller one first: the scales' own product may overflow where the sum is zero, or
// lose its bits below the normal numbers where the sum is large (a scale of rows is 2^-109 and more). An infinity or a NaN in either shows.
__device__ __forceinline__ float scaled(float v, float a, float b) {
    return v * __builtin_elementwise_minimum(a, b) * __builtin_elementwise_maximum(a, b);
}
// max(v, 0), a NaN stays one
__device__ __forceinline__ float relu_of(float v) { return __builtin_elementwise_maximum(v, 0.f); }

template <int T, int BM, int BN, int WAVES_M, int WAVES_N, bool B_KN>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, 2) void grouped_tile_kernel(GlArgs A) {
    constexpr int WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES;
    constexpr int E = T == FG_E4M3 ? 1 : T == FG_F32 ? 4 : 2, BK = GL_STEP / E;
    constexpr int STAGE = (BM + BN) * GL_STEP, A_LOADS = BM / GL_ROWS / WAVES, B_LOADS = BN / GL_ROWS / WAVES, LOADS = A_LOADS + B_LOADS;
    constexpr int MB = BM / WAVES_M / 32, NB = BN / WAVES_N / 32, WN = BN / WAVES_N;
    constexpr int DEEP = T == FG_F32 ? 2 : 1, SUB = GL_STEP / 32 / DEEP;      // 16-byte pieces of a lane's operand; operands per step
    constexpr int PARTS = T == FG_E4M3 || T == FG_F32 ? 2 : 1;                                          // 16-byte registers of it
    constexpr int B_ROW = BN * E, B_ROW_PIECES = B_ROW / 16;                      // B_KN: bytes of a row of k
    static_assert(!B_KN || T != FG_E4M3, "8-bit weights lie along K");
    static_assert(A_LOADS * GL_ROWS * WAVES == BM && B_LOADS * GL_ROWS * WAVES == BN, "whole loads");
    // LDS: two steps' operands; the epilogue's blocks; what belongs to a tile, for the current one and the next; the offsets of the groups
    extern __shared__ __attribute__((aligned(16))) char gl_lds[];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    struct TileData {
        int32_t pos[BM], src[BM];      // position and row of A of every row, -1: none
        float x_scale[T == FG_E4M3 ? BM : 4], bias[BN], w_scale[T == FG_E4M3 ? BN : 4];
    };
    char* const blocks = gl_lds + 2 * STAGE;
    TileData* data = (TileData*)(blocks + WAVES * EP_BLOCK);
    int32_t* offsets = (int32_t*)(data + 2);
    for (int i = t; i <= A.G.n_groups; i += THREADS) offsets[i] = (int32_t)group_offset(A.G, i);
    __syncthreads();

    const int K = A.K, N = A.N;
    // The column tiles of a row tile lie on one XCD (workgroup ids are dealt round-robin to the eight of them): the rows come from memory
    // once. A workgroup takes every (workgroups of an XCD)-th of its XCD's tiles.
    const int xcd = blockIdx.x & 7, j_step = gridDim.x >> 3;
    struct Tile {
        int g, n0, k0, k1;
    };
    auto find = [&](int j, Tile& F) -> bool {
        int g = 0;
        int64_t k0 = 0, k1 = 0;
        const bool there = find_tile(A.G, [&](int i) { return (int64_t)offsets[i]; }, (int64_t)(j / A.tiles_n) * 8 + xcd, BM, g, k0, k1);
        F.g = __builtin_amdgcn_readfirstlane(g);
        F.k0 = __builtin_amdgcn_readfirstlane((int)k0);
        F.k1 = __builtin_amdgcn_readfirstlane((int)k1);
        F.n0 = (j % A.tiles_n) * BN;
        return __builtin_amdgcn_readfirstlane(there);
    };
    // What belongs to a tile comes in three reads that depend on each other, a value to a thread: entry, row, scale of the row
    static_assert(THREADS >= BM && THREADS >= BN, "a thread for every row and column");
    int32_t e_pos = -1, e_src = -1;
    float e_scale = 0.f, e_bias = 0.f, e_w_scale = 0.f;
    auto fetch_entry = [&](const Tile& F) {
        const int k = F.k0 + t, c = F.n0 + t;
        e_pos = t < BM && k < F.k1 ? (A.G.order ? A.G.order[k] : k) : -1;
        if (t < BN && c < N) {
            if (A.bias) e_bias = A.bias[(int64_t)F.g * N + c];
            if constexpr (T == FG_E4M3) e_w_scale = A.w_scale[(int64_t)F.g * N + c];
        }
    };
    auto fetch_source = [&]() {
        if (e_pos < 0 || e_pos >= A.n) e_pos = -1;
        e_src = e_pos >= 0 && A.src_ids ? A.src_ids[e_pos] : e_pos;
    };
    auto fetch_scale = [&](const Tile& F) {
        if (e_src < 0 || e_src >= A.x_rows) e_pos = e_src = -1;
        if constexpr (T == FG_E4M3) e_scale = e_src >= 0 ? A.x_scale[e_src] : 0.f;
        if (e_src >= 0 && A.a_by != GL_A_SOURCE) e_src = A.a_by == GL_A_POSITION ? e_pos : F.k0 + t;
    };
    auto keep = [&](TileData& D) {
        if (t < BM) {
            D.pos[t] = e_pos;
            D.src[t] = e_src;
            if constexpr (T == FG_E4M3) D.x_scale[t] = e_scale;
        }
        if (t < BN) {
            D.bias[t] = e_bias;
            if constexpr (T == FG_E4M3) D.w_scale[t] = e_w_scale;
        }
        __syncthreads();
    };

    int j = blockIdx.x >> 3;
    Tile cur, next = {};
    if (!find(j, cur)) return;
    fetch_entry(cur);
    fetch_source();
    fetch_scale(cur);
    keep(data[0]);

    // this lane's loads of a step: rows 8 (wave + WAVES i) + lane / 8 of A (and of B along K), piece lane % 8 exchanged
    const char* pa[A_LOADS];
    const char* w_at = nullptr;      // the step's first weight, and this lane's pieces from there
    unsigned int pb[B_LOADS];
    auto exchanged = [](int row) { return (row >> 1) & (GL_PIECES - 1); };
    const int a_row = GL_ROWS * wave + lane / GL_PIECES, a_piece = (lane % GL_PIECES) ^ exchanged(a_row), ka = a_piece * (16 / E);
    static_assert(GL_ROWS * WAVES % (2 * GL_PIECES) == 0, "the same exchange for all loads of a lane");
    const char* const zero = (const char*)gl_zero;
    // what a row's windows are exchanged by (BN = 64: it has two); fp32: windows of 128 bytes, so that the halves of a wavefront, four rows apart, read
    // different banks
    auto b_window = [](int row) { return T == FG_F32 ? (row >> 2) & 1 : BN >= 128 ? row & 3 : (row >> 1) & 1; };
    auto begin = [&](const Tile& F, const TileData& D) {
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) {
            const int32_t r = D.src[a_row + GL_ROWS * WAVES * i];
            pa[i] = A.a + (int64_t)(r >= 0 ? r : 0) * A.a_stride + a_piece * 16;
        }
        w_at = A.W + ((int64_t)F.g * N + (B_KN ? 0 : F.n0)) * K * E;      // (a column tile begins below N)
#pragma unroll
        for (int i = 0; i < B_LOADS; ++i) {
            if constexpr (B_KN) {
                const int at = 64 * (wave + WAVES * i) + lane, row = at / B_ROW_PIECES, slot = at % B_ROW_PIECES;
                const int c = F.n0 + (T == FG_F32 ? (((slot >> 3) ^ b_window(row)) * 8 + (slot & 7)) * 4 : (((slot >> 2) ^ b_window(row)) * 4 + (slot & 3)) * 8);
                pb[i] = (unsigned int)(row * N + (c < N ? c : 0)) * E;
            } else {
                const int c = F.n0 + a_row + GL_ROWS * WAVES * i;
                pb[i] = (unsigned int)(c < N ? c - F.n0 : 0) * K * E + a_piece * 16;
            }
        }
    };
    const int64_t b_step = B_KN ? (int64_t)BK * N * E : GL_STEP;
    const unsigned int lds0 = (unsigned int)(uintptr_t)(__attribute__((address_space(3))) char*)gl_lds;
    const int steps = (K + BK - 1) / BK;
    auto load_step = [&](int s) {
        const unsigned int to = __builtin_amdgcn_readfirstlane(lds0 + (s & 1) * STAGE + wave * 1024);
        const int left = K - s * BK;      // elements of K that the step has
        const char* const w = uniform(w_at);
        if (left >= BK) {
#pragma unroll
            for (int i = 0; i < A_LOADS; ++i) load_to_lds(pa[i], to + i * WAVES * 1024);
#pragma unroll
            for (int i = 0; i < B_LOADS; ++i) load_to_lds(w, pb[i], to + BM * GL_STEP + i * WAVES * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < A_LOADS; ++i) load_to_lds(ka < left ? pa[i] : zero, to + i * WAVES * 1024);
#pragma unroll
            for (int i = 0; i < B_LOADS; ++i) load_to_lds((B_KN ? (64 * (wave + WAVES * i) + lane) / B_ROW_PIECES : ka) < left ? w_at + pb[i] : zero, to + BM * GL_STEP + i * WAVES * 1024);
        }
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) pa[i] += GL_STEP;
        w_at += b_step;
    };

    const int l32 = lane & 31, half = lane >> 5;
    const int wm = (wave / WAVES_N) * (BM / WAVES_M), wn = (wave % WAVES_N) * WN;
    gl_f32x16 acc[MB][NB], rest[T == FG_F32 ? MB : 1][T == FG_F32 ? NB : 1];      // fp32: the leading products, the others
    const int swap = exchanged(l32) << 4;
    static_assert(SUB % 2 == 0, "the operands' two sets in turn");
    static_assert(WN <= 64, "a row of a wavefront's columns in 16 bits fits a row of the epilogue's block");
    static_assert(2 * STAGE + WAVES * EP_BLOCK + 2 * sizeof(TileData) + 4 == gl_lds_bytes(BM, BN, WAVES, T == FG_E4M3, 0), "what the launch asks for");
    const int place = (lane >> 2) & 3;
    const int b_in = (8 * half + place) * B_ROW + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    struct Operands {
        fg_u32x4 a[MB][PARTS], b[NB][PARTS];
    };
    auto read_a = [&](int s, int kk, int mb, Operands& F) {
        const char* As = gl_lds + (s & 1) * STAGE + (wm + l32) * GL_STEP;
#pragma unroll
        for (int q = 0; q < DEEP; ++q) F.a[mb][q] = *(const fg_u32x4*)(As + mb * 32 * GL_STEP + ((((kk * DEEP + q) * 2 + half) << 4) ^ swap));
    };
    auto read_b = [&](int s, int kk, Operands& F) {
        const char* Bs = gl_lds + (s & 1) * STAGE + BM * GL_STEP;
        if constexpr (!B_KN)
#pragma unroll
            for (int q = 0; q < DEEP; ++q)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) F.b[nb][q] = *(const fg_u32x4*)(Bs + (wn + nb * 32 + l32) * GL_STEP + ((((kk * DEEP + q) * 2 + half) << 4) ^ swap));
        if constexpr (B_KN && T == FG_F32)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const char* from = Bs + (kk * 16 + 4 * half) * B_ROW + ((((wn >> 5) + nb) ^ half) << 7) + l32 * 4;      // (k as the pieces of A lie)
#pragma unroll
                for (int e = 0; e < 8; ++e) F.b[nb][e >> 2][e & 3] = *(const unsigned int*)(from + (e + (e & 4)) * B_ROW);
            }
        else if constexpr (B_KN)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                typedef __attribute__((address_space(3))) gl_s16x4* lds_s16x4;
                const char* from = Bs + kk * 16 * B_ROW + b_in + ((((wn >> 5) + nb) ^ b_window(place)) << 6);
                const gl_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)from);
                const gl_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(from + 4 * B_ROW));
                F.b[nb][0] = __builtin_bit_cast(fg_u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
    };
    auto multiply_row = [&](const Operands& F, int mb) {
        if constexpr (T != FG_F32) {
            fg_u32x4 a[2];
            if constexpr (T == FG_E4M3) widen(F.a[mb][0], a);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = mfma<T>(F.b[nb], T == FG_E4M3 ? a : F.a[mb], acc[mb][nb]);
        }
    };
    auto multiply = [&](Operands& F) {
        if constexpr (T == FG_F32) {
            fg_u32x4 a[MB][3];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) split8(F.a[mb], a[mb]);
            constexpr int TA[5] = {2, 0, 1, 1, 0}, TB[5] = {0, 2, 1, 0, 1};      // smallest products first
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                fg_u32x4 b[3];
                split8(F.b[nb], b);
#pragma unroll
                for (int e = 0; e < 5; ++e)
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) rest[mb][nb] = mfma<FG_BF16>(&b[TB[e]], &a[mb][TA[e]], rest[mb][nb]);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) acc[mb][nb] = mfma<FG_BF16>(&b[0], &a[mb][0], acc[mb][nb]);
            }
        }
    };
    // The stores of a tile are younger than the next one's first two steps' loads: those are waited for with the stores left on their way
    constexpr int STORES = MB * NB * 2;
    static_assert(LOADS + 2 * STORES < 64, "as many as can be counted");
    int stores = 0;      // 0, STORES or 2 * STORES
    auto arrived_first = [&](auto loads) {
        constexpr int N = decltype(loads)::value;
        if (stores == 0)
            arrived<N>();
        else if (stores == STORES)
            arrived<N + STORES>();
        else
            arrived<N + 2 * STORES>();
    };
    // One step: its operands are read one set ahead of the matrix instructions, a row of blocks of them before each row is multiplied; the last set is
    // multiplied while the first of the next step is read. LAST: there is no next step, LOAD: there is one after it, whose loads set out.
    Operands F0, F1;
    auto step = [&](int s, auto last, auto load) {
        constexpr bool LAST = decltype(last)::value, LOAD = decltype(load)::value;
#pragma unroll
        for (int kk = 0; kk < SUB; ++kk) {
            if (LAST && kk > 0 && kk * (BK / SUB) >= K - s * BK) break;      // (nothing but zeros beyond K)
            Operands &now = kk & 1 ? F1 : F0, &ahead = kk & 1 ? F0 : F1;
            const bool more = kk + 1 < SUB || !LAST;
            const int to_s = kk + 1 < SUB ? s : s + 1, to_kk = kk + 1 < SUB ? kk + 1 : 0;
            if (kk + 1 == SUB && !LAST) {
                if (s == 0)
                    arrived_first(std::integral_constant<int, 0>());
                else
                    arrived<0>();
                if (LOAD) load_step(s + 2);
            }
            if (more) read_b(to_s, to_kk, ahead);
            if constexpr (T == FG_E4M3)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) widen(now.b[nb][0], now.b[nb]);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                if (more) read_a(to_s, to_kk, mb, ahead);
                if constexpr (T != FG_F32) {
                    __builtin_amdgcn_sched_barrier(0);
                    multiply_row(now, mb);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (T == FG_F32) {
                __builtin_amdgcn_sched_barrier(0);
                multiply(now);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    // The products are formed as (B^T . A^T): element i of a 32 x 32 block is column 8 * (i / 4) + 4 * half + i % 4 of its row l32, so a lane holds
    // four adjacent columns of a row. Blocks of 16 rows by 128 bytes go through LDS (a wavefront's own part: no barrier), so that a store writes
    // whole lines. Pieces of 16 bytes are exchanged by the row, as the operands'.
    auto write = [&](const Tile& F, const TileData& D) {
        int lane = t & 63;      // (addresses are formed here: hoisted out of the loops they take registers those have not got)
        asm volatile("" : "+v"(lane));
        const int l32 = lane & 31, half = lane >> 5;
        char* const sink = (char*)gl_sink + lane * 16;
        char* const blk = blocks + wave * EP_BLOCK;
        constexpr int ROW16 = WN * 2;      // bytes of a row of the block in a 16-bit type; 128 of fp32
        auto swapped = [](int row, int row_bytes) { return row_bytes == 128 ? (row >> 1) & 7 : (row >> 2) & 3; };
        // rows 16 * part .. of block row mb, columns from n0 + cl on
        auto put_out = [&](int mb, int part, int cl, int element, int row_bytes) {
            const int lanes = row_bytes / 16, piece = lane % lanes, c = F.n0 + cl + piece * (16 / element);
#pragma unroll
            for (int p = 0; p < row_bytes / 64; ++p) {
                const int row = p * (64 / lanes) + lane / lanes;
                const fg_u32x4 w = *(const fg_u32x4*)(blk + row * row_bytes + ((piece ^ swapped(row, row_bytes)) << 4));
                const int32_t r = c < N ? D.pos[wm + mb * 32 + part * 16 + row] : -1;
                store_16(r >= 0 ? A.out + (int64_t)r * A.out_stride + (int64_t)c * element : sink, w);
            }
        };
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            asm volatile("" ::: "memory");      // (what is read from LDS below stays in LDS until then)
            const float xs = T == FG_E4M3 ? D.x_scale[wm + mb * 32 + l32] : 1.f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (T == FG_F32)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[mb][nb][4 * q + e] += rest[mb][nb][4 * q + e];
                    if constexpr (T == FG_E4M3) {
                        const int cl = wn + nb * 32 + 8 * q + 4 * half;
                        const float4 b = *(const float4*)(D.bias + cl), ws = *(const float4*)(D.w_scale + cl);
                        gl_f32x16& v = acc[mb][nb];
                        v[4 * q] = scaled(v[4 * q], xs, ws.x) + b.x, v[4 * q + 1] = scaled(v[4 * q + 1], xs, ws.y) + b.y;
                        v[4 * q + 2] = scaled(v[4 * q + 2], xs, ws.z) + b.z, v[4 * q + 3] = scaled(v[4 * q + 3], xs, ws.w) + b.w;
                    }
                    if (A.relu)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[mb][nb][4 * q + e] = relu_of(acc[mb][nb][4 * q + e]);
                }
            const int row = l32 & 15;
            if (A.out_type == FG_F32) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        if ((l32 >> 4) == part)
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const gl_f32x16& v = acc[mb][nb];
                                *(fg_u32x4*)(blk + row * 128 + (((2 * q + half) ^ swapped(row, 128)) << 4)) =
                                    fg_u32x4{__float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3])};
                            }
                        put_out(mb, part, wn + nb * 32, 4, 128);
                    }
            } else {
                fg_u32x2 w[NB][4];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float v[4] = {acc[mb][nb][4 * q], acc[mb][nb][4 * q + 1], acc[mb][nb][4 * q + 2], acc[mb][nb][4 * q + 3]};
                        w[nb][q] = A.out_type == FG_BF16 ? fg_to_words<FG_BF16>(v) : fg_to_words<FG_F16>(v);
                    }
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    if ((l32 >> 4) == part)
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                            for (int q = 0; q < 4; ++q) *(fg_u32x2*)(blk + row * ROW16 + (((nb * 4 + q) ^ swapped(row, ROW16)) << 4) + half * 8) = w[nb][q];
                    put_out(mb, part, wn, 2, ROW16);
                }
            }
        }
    };

    begin(cur, data[0]);
    load_step(0);
    if (steps > 1) load_step(1);
    for (int which = 0;; which ^= 1) {
        const bool more = find(j + j_step, next);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int q = 0; q < 4; ++q) {      // (8-bit products are scaled before the bias is added)
                float4 b = {0.f, 0.f, 0.f, 0.f};
                if constexpr (T != FG_E4M3) b = *(const float4*)(data[which].bias + wn + nb * 32 + 8 * q + 4 * half);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    if constexpr (T == FG_F32)
#pragma unroll
                        for (int e = 0; e < 4; ++e) rest[mb][nb][4 * q + e] = 0.f;
                    acc[mb][nb][4 * q] = b.x, acc[mb][nb][4 * q + 1] = b.y, acc[mb][nb][4 * q + 2] = b.z, acc[mb][nb][4 * q + 3] = b.w;
                }
            }
        if (steps > 1)
            arrived_first(std::integral_constant<int, LOADS>());
        else
            arrived<0>();
        read_b(0, 0, F0);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) read_a(0, 0, mb, F0);
        // what belongs to the next tile is read behind this one's last loads (the waits for it are for everything in front of it)
        int s = 0;
        for (; s + 2 < steps; ++s) step(s, std::false_type(), std::true_type());
        if (more) fetch_entry(next);
        if (steps > 1) step(s++, std::false_type(), std::false_type());
        if (more) fetch_source();
        step(s, std::true_type(), std::false_type());
        if (more) fetch_scale(next);
        // the next tile's first loads are on their way while this one is written
        if (more) {
            keep(data[which ^ 1]);      // (every wavefront has read what it needs of the ring)
            begin(next, data[which ^ 1]);
            load_step(0);
            if (steps > 1) load_step(1);
        }
        write(cur, data[which]);
        if (!more) break;
        stores = A.out_type == FG_F32 ? 2 * STORES : STORES;
        cur = next;
        j += j_step;
    }
}

template <int T, int BM, int BN, int WM, int WN, int PER_CU, bool B_KN>
fg_status_t tile_launch(GlArgs& A, hipStream_t st) {
    A.tiles_n = (int)fg_ceil_div(A.N, BN);
    const int64_t rows = A.G.max_rows / BM + (A.G.n_groups < A.G.max_rows ? A.G.n_groups : A.G.max_rows);
    const int64_t tiles = fg_ceil_div(rows, 8) * 8 * A.tiles_n;
    // (a workgroup's number of a tile is one of its XCD's, and a step beyond: (2^23 + 2^10) rows of tiles x 2^10 / 8 fit 31 bits)
    static_assert((FG_MAX_GROUPED_ROWS / 64 + FG_MAX_GROUPS + 8) * (int64_t)(FG_MAX_GROUPED_DIM / 64) / 8 + 256 * 4 < INT32_MAX, "tiles of an XCD fit an int");
    const int64_t at_once = 256 * PER_CU;
    hipLaunchKernelGGL((grouped_tile_kernel<T, BM, BN, WM, WN, B_KN>), dim3((unsigned)(tiles < at_once ? tiles : at_once)), dim3(64 * WM * WN),
                       gl_lds_bytes(BM, BN, WM * WN, T == FG_E4M3, A.G.n_groups), st, A);
    FG_LAUNCH_CHECK("grouped_tile_kernel");
    return FG_OK;
}
// out[r, :] = a[., :] . B for the entries of every group (A.a, a_stride, a_by, K, N, W, out, ... are set)
//
// The largest tile that there are as many of as compute units, and that the columns and an average group more than half fill. Both sides in us
// (K = N = 256 unless said, 4 groups):
//   256 against 128, bf16: 65536 rows 18.6 | 20.0, 32768 rows 16.6 | 13.1; N = 128 17.8 | 12.9; 193 rows a group 30.3 | 31.2, 128 rows a group 32.7 | 25.5;
//                   8 bits: 65536 rows 20.3 | 21.0, K = N = 1024 121 | 136, 32768 rows 16.9 | 12.2; N = 128 17.4 | 12.3; 193 rows a group 33.7 | 30.2, 128 rows a group 36.0 | 25.4
//   128 against 64: 16384 rows bf16 9.6 | 11.1, fp32 21.4 | 22.5, 8 bits 9.3 | 10.2; 8192 rows 8.7 | 7.1, 20.1 | 13.7, 8.6 | 6.5; N = 64 fp32 32.6 | 22.7;
//                   77 rows a group bf16 37 | 73, fp32 112 | 156, 8 bits 62 | 65; 64 rows a group 43 | 53, 134 | 115, 72 | 49
// No 256 x 256 tile for fp32, whose two sums do not fit the registers. (PER_CU: of four workgroups of the 64 x 64 tile LDS holds three, and of two
// of the 128 x 128 tile in 8 bits one above 767 groups; the others start as those end.)
template <int T, bool B_KN>
fg_status_t tile_product(GlArgs& A, hipStream_t st) {
    const int64_t large = (A.G.max_rows / 256) * fg_ceil_div(A.N, 256), groups = A.G.n_groups;
    if constexpr (T != FG_F32)
        if (large >= 256 && A.N > 128 && A.G.max_rows > 128 * groups) return tile_launch<T, 256, 256, 2, 4, 1, B_KN>(A, st);
    const int64_t mid = (A.G.max_rows / 128) * fg_ceil_div(A.N, 128);
    if (mid >= 256 && A.N > 64 && A.G.max_rows > 64 * groups) return tile_launch<T, 128, 128, 2, 2, 2, B_KN>(A, st);
    return tile_launch<T, 64, 64, 2, 2, 4, B_KN>(A, st);
}

// ---- gradients ----

// steps of the groups before `upto` (lanes of a wavefront together)
__device__ __forceinline__ int64_t steps_before(const Groups& G, int upto, int rows) {
    int64_t n = 0;
    for (int i = fg_lane(); i < upto; i += 64) {
        const int64_t from = group_offset(G, i), to = group_offset(G, i + 1);
        n += to > from ? (to - from + rows - 1) / rows : 0;
    }
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
    return n;
}

// dz in entry order, in the rows' type, and its column sums by tiles of GZ_ROWS entries of one group (db is their sum). The products then
// read dz alone, straight to LDS; a mask on the way there would take both matrices through registers, twice (for one tile of columns of x it was tried in
// the fp32 weight gradients, with dz and db's sums as by-products: 102.9 us a backward call against 103.5). Bound by memory: 58982 x 1024
// bf16 72 us (5.0 TB/s, the rate of a copy), 43352 x 256 fp32 23 us (5.7, part of it from the last-level cache). Few rows are bound by latency:
// hence 256 columns to a workgroup and four rows' reads on their way together (2000 x 1000 bf16 5 us more than dx alone takes; 20 with all the
// columns in one workgroup, row after row).
constexpr int GZ_ROWS = 64, GZ_THREADS = 256, GZ_COLUMNS = 256;

// T: the rows' type, D: that of dh, H: that of h
template <int T, int D, int H>
__global__ __launch_bounds__(GZ_THREADS) void grouped_dz_kernel(GlArgs A) {
    constexpr int E = T == FG_F32 ? 4 : 2, DE = D == FG_F32 ? 4 : 2, HE = H == FG_F32 ? 4 : 2;
    __shared__ int32_t pos[GZ_ROWS];
    __shared__ float sums[GZ_THREADS * 8];
    int g;
    int64_t k0, k1;
    if (!find_tile(A.G, blockIdx.x, GZ_ROWS, g, k0, k1)) return;
    const int t = threadIdx.x;
    if (t < GZ_ROWS) {
        int32_t s;
        entry(A, k0 + t, k1, pos[t], s);
    }
    __syncthreads();
    // this workgroup's columns, and how many rows of them its threads have side by side
    const int first = (int)blockIdx.y * (GZ_COLUMNS / 8), rows = (int)(k1 - k0);
    const int pieces = (A.d_out + 7) / 8 - first < GZ_COLUMNS / 8 ? (A.d_out + 7) / 8 - first : GZ_COLUMNS / 8;
    int side = GZ_THREADS / (GZ_COLUMNS / 8);
    while (side * 2 * pieces <= GZ_THREADS) side *= 2;
    const int width = GZ_THREADS / side, p = t % width, c = (first + p) * 8, left = A.d_out - c;
    float sum[8] = {};
    if (p < pieces) {
        constexpr int AHEAD = 4;      // rows whose reads are on their way together
        for (int m0 = t / width; m0 < rows; m0 += AHEAD * side) {
            fg_piece<D> pz[AHEAD];
            fg_piece<H> ph[AHEAD];
            int32_t r[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int m = m0 + u * side;
                r[u] = m < rows ? pos[m] : -1;
                if (r[u] >= 0) pz[u] = fg_load_piece<D>(A.dh + r[u] * A.dh_stride + (int64_t)c * DE, left);
                if (r[u] >= 0 && A.h) ph[u] = fg_load_piece<H>(A.h + r[u] * A.h_stride + (int64_t)c * HE, left);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int m = m0 + u * side;
                float z[8] = {};
                if (r[u] >= 0) fg_piece_values<D>(pz[u], z);
                if (r[u] >= 0 && A.h) {
                    float h[8];
                    fg_piece_values<H>(ph[u], h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = h[e] > 0.f ? z[e] : 0.f;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += z[e];
                if (A.dz && m < rows) fg_store_piece<T>(A.dz + (k0 + m) * A.dz_stride + (int64_t)c * E, z, left);
            }
        }
    }
    if (!A.db_part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[t * 8 + e] = sum[e];
    __syncthreads();
    for (int i = t; i < width * 8; i += GZ_THREADS) {
        float v = 0.f;
        for (int q = 0; q < side; ++q) v += sums[q * width * 8 + i];
        if (first * 8 + i < A.d_out && i < GZ_COLUMNS) A.db_part[(int64_t)blockIdx.x * A.d_out + first * 8 + i] = v;
    }
}

// db[g, c] = sum over the group's tiles, in fp64; DB_COLUMNS columns a workgroup, DB_RUNS runs of tiles side by side
constexpr int DB_COLUMNS = 8, DB_RUNS = GZ_THREADS / DB_COLUMNS;
__device__ __forceinline__ void sum_db(const GlArgs& A, int block, double* red) {
    const int blocks = (A.d_out + DB_COLUMNS - 1) / DB_COLUMNS, g = block / blocks;
    const int c = (block % blocks) * DB_COLUMNS + ((int)threadIdx.x % DB_COLUMNS);
    const int64_t first = steps_before(A.G, g, GZ_ROWS);
    const int64_t from = group_offset(A.G, g), to = group_offset(A.G, g + 1);
    int64_t tiles = to > from ? (to - from + GZ_ROWS - 1) / GZ_ROWS : 0;
    if (tiles > A.db_tiles - first) tiles = A.db_tiles - first;      // (offsets that do not ascend)
    double s = 0.0;
    if (c < A.d_out)
#pragma unroll 8
        for (int64_t i = threadIdx.x / DB_COLUMNS; i < tiles; i += DB_RUNS) s += (double)A.db_part[(first + i) * A.d_out + c];
    red[threadIdx.x] = s;
    __syncthreads();
    for (int n = GZ_THREADS / 2; n >= DB_COLUMNS; n >>= 1) {      // halves of the runs
        if ((int)threadIdx.x < n) red[threadIdx.x] += red[threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x < DB_COLUMNS && c < A.d_out) A.db[(int64_t)g * A.d_out + c] = (float)red[threadIdx.x];
}

// dW = x^T . dz of every group: a contraction over the group's rows, whose number the device alone knows, with BM x BN tiles of the result.
// The rows are a line of steps of ROWS entries, group by group, cut into equal ranges; a workgroup takes one tile along one range, so
// that all of them end together however the groups are sized, and those of one range (on one XCD) read the same rows at the same time: from
// its L2 but for the first. A group that lies wholly in a range is a result; of one that does not (the first and the last of a range) the
// workgroup leaves its part in a slot of its own, and a second launch adds those up, in order.
// Both operands have the contraction index in front, rows of x and of dz: they go to LDS as they lie and are transposed on the way out.
constexpr int GW_ROWS = 64, GW_LIST = 4096;

struct Share {
    int64_t total, per;      // steps of all groups; of a range
};
__device__ __forceinline__ Share share_of(const GlArgs& A, int rows) {
    Share s;
    s.total = steps_before(A.G, A.G.n_groups, rows);
    s.per = (s.total + A.ranges - 1) / A.ranges;
    return s;
}
// range and tile of this workgroup: consecutive ones on one XCD
__device__ __forceinline__ bool range_and_tile(const GlArgs& A, int tiles, int& range, int& tile) {
    const int per_xcd = (int)gridDim.x >> 3, unit = ((int)blockIdx.x & 7) * per_xcd + ((int)blockIdx.x >> 3);
    range = unit / tiles;
    tile = unit % tiles;
    return range < A.ranges;
}
// walks the groups of a range: group g's steps [first, last) of its steps_g lie in it, entries [k0, k1)
struct RangeWalk {
    int64_t at, end, before;
    int g;
    int64_t steps_g, first, last, k0, k1;
    __device__ __forceinline__ bool next(const Groups& G, int rows) {
        if (at >= end) return false;
        int64_t from, to;
        for (;; ++g) {
            from = group_offset(G, g);
            to = group_offset(G, g + 1);
            steps_g = to > from ? (to - from + rows - 1) / rows : 0;
            if (at < before + steps_g) break;
            before += steps_g;
        }
        first = at - before;
        last = first + (end - at) < steps_g ? first + (end - at) : steps_g;
        k0 = from + first * rows;
        k1 = from + last * rows < to ? from + last * rows : to;
        return true;
    }
};

template <int T, int BM, int BN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, 2) void grouped_dw_kernel(GlArgs A) {
    constexpr int WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES;
    constexpr int STAGE = GW_ROWS * (BM + BN) * 2, LOADS = GW_ROWS * BM * 2 / 1024 / WAVES;      // of either operand
    constexpr int MB = BM / WAVES_M / 32, NB = BN / WAVES_N / 32, SUB = GW_ROWS / 16;
    static_assert(BM == BN && SUB % 2 == 0, "a lane's pieces of x and of dz lie in the same rows; the operands' two sets in turn");
    extern __shared__ __attribute__((aligned(16))) char gl_lds[];
    int32_t* list = (int32_t*)(gl_lds + 2 * STAGE);      // rows of x of the next entries, -1: skipped
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int tiles_m = (A.d_in + BM - 1) / BM, tiles_n = (A.d_out + BN - 1) / BN, tiles = tiles_m * tiles_n;
    int range, tile;
    if (!range_and_tile(A, tiles, range, tile)) return;
    const Share S = share_of(A, GW_ROWS);
    RangeWalk W = {range * S.per, (range + 1) * S.per < S.total ? (range + 1) * S.per : S.total, 0, 0};

    const int l32 = lane & 31, half = lane >> 5, place = (lane >> 2) & 3;
    const int wm = (wave / WAVES_N) * (BM / WAVES_M), wn = (wave % WAVES_N) * (BN / WAVES_N);
    const int m0 = (tile / tiles_n) * BM, n0 = (tile % tiles_n) * BN;
    constexpr int ROW = BM * 2, ROW_PIECES = ROW / 16, ROWS_A_LOAD = 1024 / ROW;
    const int in_row = (8 * half + place) * ROW + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    const unsigned int lds0 = (unsigned int)(uintptr_t)(__attribute__((address_space(3))) char*)gl_lds;
    const char* const zero = (const char*)gl_zero;
    // this lane's pieces of a step: rows row0 + ROWS_A_LOAD * WAVES * i, one piece of 8 columns (columns that do not exist read the first: not stored)
    const int row0 = ROWS_A_LOAD * wave + lane / ROW_PIECES, slot = lane % ROW_PIECES;
    static_assert(ROWS_A_LOAD * WAVES % 4 == 0, "the same exchange for all loads of a lane");
    const int col = (((slot >> 2) ^ (row0 & 3)) * 4 + (slot & 3)) * 8;
    const int ca = (m0 + col < A.d_in ? m0 + col : 0) * 2, cb = (n0 + col < A.d_out ? n0 + col : 0) * 2;

    gl_f32x16 acc[MB][NB];
    struct Operands {
        fg_u32x4 a[MB], b[NB];
    };
    auto fragment = [&](const char* p) -> fg_u32x4 {
        typedef __attribute__((address_space(3))) gl_s16x4* lds_s16x4;
        const gl_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p);
        const gl_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * ROW));
        return __builtin_bit_cast(fg_u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read = [&](int s, int kk, Operands& F) {
        const char* As = gl_lds + (s & 1) * STAGE + in_row + kk * 16 * ROW;
        const char* Bs = As + GW_ROWS * BM * 2;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) F.a[mb] = fragment(As + ((((wm >> 5) + mb) ^ place) << 6));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) F.b[nb] = fragment(Bs + ((((wn >> 5) + nb) ^ place) << 6));
    };
    auto multiply = [&](const Operands& F) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = mfma<T>(&F.a[mb], &F.b[nb], acc[mb][nb]);
    };

    for (; W.next(A.G, GW_ROWS); W.at += W.last - W.first) {      // uniform over the workgroup
        const int steps = (int)(W.last - W.first);
        const int64_t k0 = W.k0, k1 = W.k1;
        auto fill = [&](int64_t k) {      // entries k .. k + GW_LIST, as far as whole steps need them
            const int need = (int)(k1 - k < GW_LIST ? (k1 - k + GW_ROWS - 1) / GW_ROWS * GW_ROWS : GW_LIST);
#pragma unroll 2
            for (int i = t; i < need; i += THREADS) {
                int32_t r = -1, s = -1;
                entry(A, k + i, k1, r, s);
                list[i] = s;
            }
            __syncthreads();
        };
        int32_t x_row[LOADS];
        auto read_rows = [&](int s) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) x_row[i] = list[(s * GW_ROWS) % GW_LIST + row0 + ROWS_A_LOAD * WAVES * i];
        };
        auto load_step = [&](int s) {
            const unsigned int dst = __builtin_amdgcn_readfirstlane(lds0 + (s & 1) * STAGE + wave * 1024);
            const int64_t k = k0 + (int64_t)s * GW_ROWS;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int64_t z_row = A.dz ? k + row0 + ROWS_A_LOAD * WAVES * i : x_row[i];      // without dz: dh by position, which is the row of x
                const char *pa = A.x + x_row[i] * A.x_stride + ca, *pb = (A.dz ? A.dz : A.dh) + z_row * A.dz_stride + cb;
                load_to_lds(x_row[i] >= 0 ? pa : zero, dst + i * WAVES * 1024);
                load_to_lds(x_row[i] >= 0 ? pb : zero, dst + GW_ROWS * BM * 2 + i * WAVES * 1024);
            }
        };
#pragma unroll
        for (int a = 0; a < MB; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;
        fill(k0);
        read_rows(0);
        load_step(0);
        if (steps > 1) {
            read_rows(1);
            load_step(1);
            arrived<2 * LOADS>();
        } else {
            arrived<0>();
        }
        // as in grouped_tile_kernel: one barrier a step, behind the reads of its last operands
        Operands F0, F1;
        read(0, 0, F0);
        for (int s = 0; s < steps; ++s) {
            const bool load = s + 2 < steps;
            if (load && (s + 2) % (GW_LIST / GW_ROWS) != 0) read_rows(s + 2);
#pragma unroll
            for (int kk = 0; kk < SUB; ++kk) {
                Operands &now = kk & 1 ? F1 : F0, &ahead = kk & 1 ? F0 : F1;
                if (kk + 1 < SUB) {
                    read(s, kk + 1, ahead);
                } else if (s + 1 < steps) {
                    arrived<0>();
                    if (load) {
                        if ((s + 2) % (GW_LIST / GW_ROWS) == 0) {
                            fill(k0 + (int64_t)(s + 2) * GW_ROWS);
                            read_rows(s + 2);
                        }
                        load_step(s + 2);
                    }
                    read(s + 1, 0, ahead);
                }
                __builtin_amdgcn_sched_barrier(0);
                multiply(now);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        const bool whole = W.first == 0 && W.last == W.steps_g;
        float* to_part = A.dw_part + ((int64_t)(2 * range + (W.at == range * S.per ? 0 : 1)) * tiles + tile) * BM * BN;
        float* to_dw = A.dw + (int64_t)W.g * A.d_in * A.d_out;
        int m_first = wm + 4 * half, c_first = wn + l32;      // (addresses are formed here: hoisted out of the loops they take registers those have not got)
        asm volatile("" : "+v"(m_first), "+v"(c_first));
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int m = m_first + mb * 32 + 8 * (i >> 2) + (i & 3);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const int c = c_first + nb * 32;
                    if (!whole)
                        to_part[m * BN + c] = acc[mb][nb][i];
                    else if (m0 + m < A.d_in && n0 + c < A.d_out)
                        to_dw[(int64_t)(m0 + m) * A.d_out + n0 + c] = acc[mb][nb][i];
                }
            }
        __syncthreads();      // the list and the buffers may be filled again
    }
}

// The tiles that several workgroups have parts of, and zeros for groups without rows. A workgroup takes VALUES values of a tile: 4096 if that
// gives 512 workgroups, else 256, with runs of the parts side by side (a small result has many parts: 14 tiles of 128 x 128 from 512 ranges 27 us
// with 1024 values and the parts one after the other, 7 with 256; 100 groups of 4 tiles, a part or two each, with 256 39 us more than with 4096).
// The workgroups behind those sum db: a launch of their own cost 5 us.
constexpr int DS_MANY = 4096, DS_FEW = 256;
template <int BM, int BN, int ROWS, int VALUES>
__global__ __launch_bounds__(GZ_THREADS) void grouped_dw_sum_kernel(GlArgs A) {
    constexpr int RUNS = VALUES < GZ_THREADS * 4 ? GZ_THREADS * 4 / VALUES : 1, SIDE = GZ_THREADS / RUNS, PARTS = BM * BN / VALUES;
    __shared__ double red[RUNS][SIDE * 4];
    static_assert(sizeof(red) >= GZ_THREADS * sizeof(double), "a value of every thread");
    if ((int)blockIdx.x >= A.sums) return sum_db(A, (int)blockIdx.x - A.sums, &red[0][0]);
    const int tiles_n = (A.d_out + BN - 1) / BN, tiles = (A.d_in + BM - 1) / BM * tiles_n;
    const int part = blockIdx.x % PARTS, unit = blockIdx.x / PARTS, tile = unit % tiles, g = unit / tiles;
    if (tile / tiles_n * BM + part * VALUES / BN >= A.d_in) return;      // its rows do not exist
    const Share S = share_of(A, ROWS);
    const int64_t t0 = steps_before(A.G, g, ROWS);
    const int64_t from = group_offset(A.G, g), to = group_offset(A.G, g + 1);
    const int64_t steps_g = to > from ? (to - from + ROWS - 1) / ROWS : 0;
    const int64_t t1 = t0 + steps_g;
    const int64_t w0 = steps_g ? t0 / S.per : 0, w1 = steps_g ? (t1 - 1) / S.per : -1;
    if (steps_g && w0 == w1) return;      // one workgroup has written it
    const int run = threadIdx.x / SIDE, at = (threadIdx.x % SIDE) * 4;
#pragma unroll
    for (int i = 0; i < VALUES; i += SIDE * 4) {
        const int e = part * VALUES + i + at, m = tile / tiles_n * BM + e / BN, c = tile % tiles_n * BN + e % BN;
        double s[4] = {};
#pragma unroll 4
        for (int64_t w = w0 + run; w <= w1; w += RUNS) {
            const float4 v = *(const float4*)(A.dw_part + ((2 * w + (t0 <= w * S.per ? 0 : 1)) * tiles + tile) * BM * BN + e);
            s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
        }
        if constexpr (RUNS > 1) {
#pragma unroll
            for (int q = 0; q < 4; ++q) red[run][at + q] = s[q];
            __syncthreads();
            if (run == 0)
#pragma unroll
                for (int q = 1; q < RUNS; ++q)
#pragma unroll
                    for (int f = 0; f < 4; ++f) s[f] += red[q][at + f];
        }
        if (run == 0 && m < A.d_in && c < A.d_out)      // d_out is a multiple of 4
            *(float4*)(A.dw + ((int64_t)g * A.d_in + m) * A.d_out + c) = float4{(float)s[0], (float)s[1], (float)s[2], (float)s[3]};
    }
}

// ---- fp32 ----
//
// dW in fp32: the products as above, from terms that are split before they go to LDS (values that are split as they are read, which
// needs no registers for loads on their way, took 129 us a backward call instead of 110: here every value of both operands is read by
// two wavefronts). A workgroup owns a TILE x TILE tile of the result and walks the contraction in steps of GF_K: a thread loads 16 bytes of
// an operand's row, splits them and writes each term's bf16 values to LDS as they lie; they are transposed on the way out. One buffer and two
// barriers a step; the loads of the next step are in flight while a step is multiplied, and the two workgroups of a compute unit fill each
// other's waits. 43352 x 88 x 256: 36 us.
constexpr int GF_THREADS = 256, GF_K = 32, GF_TILE = 128, GF_BLOCKS = GF_TILE / 64;      // 32 x 32 blocks of a wavefront, both ways
// one operand in LDS: three terms of GF_K rows
constexpr int GF_ROW = GF_TILE * 2, GF_TERM = GF_K * GF_ROW;
constexpr int GF_PER_ROW = GF_TILE / 4, GF_ROWS = GF_THREADS / GF_PER_ROW, GF_LOADS = GF_K / GF_ROWS;      // pieces of a row; rows of a pass; passes
constexpr size_t GF_LDS_BYTES = 2 * 3 * GF_TERM;
__device__ __forceinline__ int gf_row_of(int t, int i) { return t / GF_PER_ROW + GF_ROWS * i; }
// windows of 64 bytes are exchanged so that the four rows of a transposing read lie in different banks
__device__ __forceinline__ void gf_put(char* lds, int t, int i, fg_u32x4 v) {
    const int row = gf_row_of(t, i), piece = t % GF_PER_ROW;
    fg_u32x2 u[3];
    split4(v, u);
    char* to = lds + row * GF_ROW + (((piece >> 3) ^ (row & 3)) << 6) + (piece & 7) * 8;
#pragma unroll
    for (int term = 0; term < 3; ++term) *(fg_u32x2*)(to + term * GF_TERM) = u[term];
}
// columns first .. first + 31, k = 16 kk + 8 half + 0..7
__device__ __forceinline__ fg_u32x4 gf_fragment(const char* lds, int first, int kk, int lane) {
    typedef __attribute__((address_space(3))) gl_s16x4* lds_s16x4;
    const int half = lane >> 5, place = (lane >> 2) & 3;
    const char* p = lds + (16 * kk + 8 * half + place) * GF_ROW + (((first >> 5) ^ place) << 6) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    const gl_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p);
    const gl_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * GF_ROW));
    return __builtin_bit_cast(fg_u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// dW in fp32: the ranges of grouped_dw_kernel, steps of GF_K entries, 128 x 128 tiles
__global__ __launch_bounds__(GF_THREADS, 2) void grouped_f32_dw_kernel(GlArgs A) {
    constexpr int TILE = GF_TILE, B = GF_BLOCKS;
    extern __shared__ __attribute__((aligned(16))) char gl_lds[];
    int32_t* list = (int32_t*)(gl_lds + GF_LDS_BYTES);
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int tiles_n = (A.d_out + TILE - 1) / TILE, tiles = (A.d_in + TILE - 1) / TILE * tiles_n;
    int range, tile;
    if (!range_and_tile(A, tiles, range, tile)) return;
    const Share S = share_of(A, GF_K);
    RangeWalk W = {range * S.per, (range + 1) * S.per < S.total ? (range + 1) * S.per : S.total, 0, 0};
    const int wm = (wave >> 1) * (TILE / 2), wn = (wave & 1) * (TILE / 2);
    const int m0 = (tile / tiles_n) * TILE, n0 = (tile % tiles_n) * TILE;
    for (; W.next(A.G, GF_K); W.at += W.last - W.first) {      // uniform over the workgroup
        const int steps = (int)(W.last - W.first);
        const int64_t k0 = W.k0, k1 = W.k1;
        const int c = (t % GF_PER_ROW) * 4;
        const int64_t ca = (m0 + c < A.d_in ? m0 + c : 0) * 4, cb = (n0 + c < A.d_out ? n0 + c : 0) * 4;
        fg_u32x4 ra[GF_LOADS], rb[GF_LOADS];
        bool in[GF_LOADS];
        auto fill = [&](int64_t k) {
            const int need = (int)(k1 - k < GW_LIST ? (k1 - k + GF_K - 1) / GF_K * GF_K : GW_LIST);
#pragma unroll 2
            for (int i = t; i < need; i += GF_THREADS) {
                int32_t r = -1, s = -1;
                entry(A, k + i, k1, r, s);
                list[i] = s;
            }
            __syncthreads();
        };
        auto load = [&](int s) {
#pragma unroll
            for (int i = 0; i < GF_LOADS; ++i) {
                const int32_t x_row = list[(s * GF_K) % GW_LIST + gf_row_of(t, i)];
                in[i] = x_row >= 0;
                const int64_t xr = in[i] ? x_row : 0, zr = in[i] ? (A.dz ? k0 + (int64_t)s * GF_K + gf_row_of(t, i) : xr) : 0;
                ra[i] = *(const fg_u32x4*)(A.x + xr * A.x_stride + ca);
                rb[i] = *(const fg_u32x4*)((A.dz ? A.dz : A.dh) + zr * A.dz_stride + cb);
            }
        };
        auto store = [&]() {
            const fg_u32x4 none = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < GF_LOADS; ++i) {
                gf_put(gl_lds, t, i, in[i] ? ra[i] : none);
                gf_put(gl_lds + 3 * GF_TERM, t, i, in[i] ? rb[i] : none);
            }
        };
        gl_f32x16 lead[B][B], rest[B][B];
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int j = 0; j < B; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) lead[i][j][e] = rest[i][j][e] = 0.f;
        auto multiply = [&]() {
            constexpr int TA[5] = {2, 0, 1, 1, 0}, TB[5] = {0, 2, 1, 0, 1};      // smallest products first
#pragma unroll
            for (int kk = 0; kk < GF_K / 16; ++kk) {
                fg_u32x4 a[B][3], b[B][3];
#pragma unroll
                for (int i = 0; i < B; ++i)
#pragma unroll
                    for (int term = 0; term < 3; ++term) {
                        a[i][term] = gf_fragment(gl_lds + term * GF_TERM, wm + 32 * i, kk, lane);
                        b[i][term] = gf_fragment(gl_lds + (3 + term) * GF_TERM, wn + 32 * i, kk, lane);
                    }
#pragma unroll
                for (int e = 0; e < 5; ++e)
#pragma unroll
                    for (int i = 0; i < B; ++i)
#pragma unroll
                        for (int j = 0; j < B; ++j) rest[i][j] = mfma<FG_BF16>(&a[i][TA[e]], &b[j][TB[e]], rest[i][j]);
#pragma unroll
                for (int i = 0; i < B; ++i)
#pragma unroll
                    for (int j = 0; j < B; ++j) lead[i][j] = mfma<FG_BF16>(&a[i][0], &b[j][0], lead[i][j]);
            }
        };
        fill(k0);
        load(0);
        for (int s = 0; s < steps; ++s) {
            store();
            if (s + 1 < steps && (s + 1) % (GW_LIST / GF_K) == 0) fill(k0 + (int64_t)(s + 1) * GF_K);      // (the list's last entries have been taken)
            __syncthreads();
            if (s + 1 < steps) load(s + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply();
            __syncthreads();
        }
        const bool whole = W.first == 0 && W.last == W.steps_g;
        float* to_part = A.dw_part + ((int64_t)(2 * range + (W.at == range * S.per ? 0 : 1)) * tiles + tile) * TILE * TILE;
        float* to_dw = A.dw + (int64_t)W.g * A.d_in * A.d_out;
        int m_first = wm + 4 * (lane >> 5), n_first = wn + (lane & 31);      // (formed here, as above)
        asm volatile("" : "+v"(m_first), "+v"(n_first));
#pragma unroll
        for (int a = 0; a < B; ++a)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int m = m_first + 32 * a + 8 * (i >> 2) + (i & 3);
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const int n = n_first + 32 * b;
                    const float v = lead[a][b][i] + rest[a][b][i];
                    if (!whole)
                        to_part[m * TILE + n] = v;
                    else if (m0 + m < A.d_in && n0 + n < A.d_out)
                        to_dw[(int64_t)(m0 + m) * A.d_out + n0 + n] = v;
                }
            }
    }
}

// Bytes between the rows of dz. Tiles read the same columns of many rows at a time: rows a multiple of 512 bytes apart meet in few of the memory's
// channels (66 k rows of 1024 bf16 x 1024 columns: 167 us at 2048 bytes, 160 at 2432), so such rows get 384 bytes more.
int64_t dz_row(int d_out, int e) {
    const int64_t row = (int64_t)d_out * e;
    return row % 512 ? row : row + 384;
}
// The workspace of a backward call: dz, column sums by tile, parts of dW
struct BwPlan {
    int bm, ranges, grid;      // tile, ranges of rows, workgroups of the weight gradients
    size_t dz_bytes, db_bytes, dw_bytes;
    size_t total() const { return dz_bytes + db_bytes + dw_bytes + 16; }
};
// Ranges of rows for bm x bm tiles. As many as give every place on the chip a tile; of more tiles than places two ranges where that leaves fewer of
// them idle. But a part of a tile that is written and read again costs what reading its operands for bm rows costs: a range has DW_MIN_ROWS rows
// at least, where that leaves DW_MIN_GROUPS workgroups. (dW alone, us: bf16, 4096 x 256 x 256, 18 with such ranges, 21 with shorter ones; fp32, 2000 x
// 256 x 256 in 40 groups 33 with 256 workgroups, 48 with 64; 8000 x 64 x 64 in 100 groups 44 and 58.)
constexpr int DW_MIN_ROWS = 128, DW_MIN_GROUPS = 256;
int dw_ranges(int64_t max_rows, int n_groups, int64_t tiles, int bm, int e) {
    const int rows = e == 4 ? GF_K : GW_ROWS;
    const int64_t steps = max_rows / rows + (n_groups < max_rows ? n_groups : max_rows), places = bm == 256 ? 256 : 512;
    int64_t ranges = places / tiles;
    if (ranges < 1) ranges = fg_ceil_div(2 * tiles, places) < 2 * fg_ceil_div(tiles, places) ? 2 : 1;
    const int64_t few = DW_MIN_GROUPS / tiles < steps ? DW_MIN_GROUPS / tiles : steps, most = fg_ceil_div(steps * rows, DW_MIN_ROWS);
    if (ranges > (most > few ? most : few)) ranges = most > few ? most : few;
    return ranges < 1 ? 1 : (int)ranges;
}
// (sized for the masked call, which needs dz, at every size, and for both tiles: a workspace for max_rows serves fewer rows too)
BwPlan bw_plan(int64_t max_rows, int n_groups, int d_in, int d_out, int e) {
    BwPlan P;
    P.dw_bytes = 0;
    for (int bm = 128; bm <= (e == 2 ? 256 : 128); bm *= 2) {
        const int64_t tiles = fg_ceil_div(d_in, bm) * fg_ceil_div(d_out, bm);
        // tiles of 256 x 256 take half the reads, and their parts twice the writes: from 2048 rows a place on (bf16, 4 groups, us, 256 | 128: 65536 x 1024 x
        // 1024, 4096 rows, 160 | 189; 20000 x 2048 x 2048 172 | 212; 65536 x 512 x 512, 1024 rows, 69 | 63; 4096 x 1024 x 1024, 256 rows, 43 | 35)
        if (bm == 256 && max_rows * tiles < 2048 * 256) break;
        P.bm = bm;
        P.ranges = dw_ranges(max_rows, n_groups, tiles, bm, e);
        P.grid = (int)(fg_ceil_div(P.ranges * tiles, 8) * 8);
        const size_t bytes = P.ranges > 1 ? (size_t)2 * P.ranges * tiles * bm * bm * 4 : 0;
        if (bytes > P.dw_bytes) P.dw_bytes = bytes;
    }
    P.dz_bytes = fg_align_up((size_t)max_rows * dz_row(d_out, e), 256);
    P.db_bytes = fg_align_up((size_t)(max_rows / GZ_ROWS + (n_groups < max_rows ? n_groups : max_rows)) * d_out * 4, 256);
    return P;
}

fg_status_t check_groups(const char* who, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups, int32_t d_in, int32_t d_out,
                         fg_dtype_t dtype, int64_t x_rows, int64_t n) {
    const int e = dtype == FG_E4M3 ? 1 : fg_dtype_size(dtype);
    if (!e) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type %d", who, (int)dtype);
    if (max_rows < 0 || max_rows > FG_MAX_GROUPED_ROWS || x_rows < 0 || x_rows > INT32_MAX || n < 0 || n > INT32_MAX)
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: a number of rows is negative or too large", who);
    if (n_groups < 1 || n_groups > FG_MAX_GROUPS) FG_FAIL(FG_ERR_INVALID_ARG, "%s: n_groups = %d is not in 1..%d", who, n_groups, FG_MAX_GROUPS);
    const int step_in = 16 / e, step_out = dtype == FG_F32 ? 4 : 8;
    if (d_in <= 0 || d_in % step_in || d_out <= 0 || d_out % step_out || d_in > FG_MAX_GROUPED_DIM || d_out > FG_MAX_GROUPED_DIM)
        FG_FAIL(FG_ERR_SHAPE, "%s: d_in = %d must be a multiple of %d and d_out = %d of %d for this type, %d at most", who, d_in, step_in, d_out, step_out, FG_MAX_GROUPED_DIM);
    if (!offsets_dev || ((uintptr_t)offsets_dev & 7) || ((uintptr_t)order_dev & 3))
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: offsets must not be NULL, and order and offsets aligned to their elements", who);
    return FG_OK;
}
fg_status_t check_matrix(const char* who, const char* what, const void* p, int64_t stride, int64_t row_bytes) {
    if (!p) FG_FAIL(FG_ERR_INVALID_ARG, "%s: %s must not be NULL", who, what);
    if (stride < row_bytes) FG_FAIL(FG_ERR_SHAPE, "%s: the stride of %s is smaller than its row", who, what);
    if (((uintptr_t)p | (uintptr_t)stride) & 15) FG_FAIL(FG_ERR_INVALID_ARG, "%s: %s and its stride must be 16-byte aligned", who, what);
    return FG_OK;
}
#define FG_TRY(expr)                   \
    do {                               \
        const fg_status_t s_ = (expr); \
        if (s_ != FG_OK) return s_;    \
    } while (0)

// tiles of rows at most: every group may end in one that is partly filled
int64_t row_tiles(int64_t max_rows, int n_groups, int size) { return max_rows / size + (n_groups < max_rows ? n_groups : max_rows); }

template <int T, int D, int H>
void launch_dz(const GlArgs& A, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((grouped_dz_kernel<T, D, H>), grid, dim3(GZ_THREADS), 0, st, A);
}
template <int BM, int ROWS, int VALUES>
void launch_sum(const GlArgs& A, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((grouped_dw_sum_kernel<BM, BM, ROWS, VALUES>), grid, dim3(GZ_THREADS), 0, st, A);
}
template <int T>
fg_status_t backward(const char* who, GlArgs& A, bool work, hipStream_t st, void* ws_dev) {
    constexpr int E = T == FG_F32 ? 4 : 2;
    const BwPlan P = bw_plan(A.G.max_rows, A.G.n_groups, A.d_in, A.d_out, E);
    char* ws = (char*)ws_dev;
    const bool pack = A.h || A.dh_type != T || A.src_ids;      // otherwise dh, by position as x is, serves as it lies
    A.dz = work && pack && (A.out || A.dw) ? ws : nullptr;
    A.dz_stride = A.dz ? dz_row(A.d_out, E) : A.dh_stride;
    A.db_part = work && A.db ? (float*)(ws + P.dz_bytes) : nullptr;
    A.dw_part = (float*)(ws + P.dz_bytes + P.db_bytes);
    A.db_tiles = work ? row_tiles(A.G.max_rows, A.G.n_groups, GZ_ROWS) : 0;
    // the launch of the sums: what it cannot hold is refused before anything is launched
    const int64_t results = fg_ceil_div(A.d_in, P.bm) * fg_ceil_div(A.d_out, P.bm) * A.G.n_groups * (P.bm * P.bm);
    const bool many = results / DS_MANY >= 512;
    const int64_t sums = A.dw ? results / (many ? DS_MANY : DS_FEW) : 0;
    const int64_t db_blocks = A.db ? A.G.n_groups * fg_ceil_div(A.d_out, DB_COLUMNS) : 0;
    if (sums + db_blocks >= FG_MAX_GRID) FG_FAIL(FG_ERR_SHAPE, "%s: too many groups and columns for one call", who);
    if (A.dz || A.db_part) {
        const dim3 grid((unsigned)A.db_tiles, (unsigned)fg_ceil_div(A.d_out, GZ_COLUMNS));
        if constexpr (T == FG_F32)
            launch_dz<T, T, T>(A, grid, st);
        else if (A.dh_type == T)
            A.h_type == FG_F32 ? launch_dz<T, T, FG_F32>(A, grid, st) : A.h_type == FG_F16 ? launch_dz<T, T, FG_F16>(A, grid, st) : launch_dz<T, T, FG_BF16>(A, grid, st);
        else
            A.h_type == FG_F32 ? launch_dz<T, FG_F32, FG_F32>(A, grid, st) : A.h_type == FG_F16 ? launch_dz<T, FG_F32, FG_F16>(A, grid, st) : launch_dz<T, FG_F32, FG_BF16>(A, grid, st);
        FG_LAUNCH_CHECK("grouped_dz_kernel");
    }
    if (A.out && work) {
        A.a = A.dz ? A.dz : A.dh, A.a_stride = A.dz_stride, A.a_by = A.dz ? GL_A_ENTRY : GL_A_POSITION, A.K = A.d_out, A.N = A.d_in;
        FG_TRY((tile_product<T, false>(A, st)));
    }
    if (!A.dw && !A.db) return FG_OK;
    A.ranges = P.ranges;
    A.sums = (int)sums;
    const dim3 grid((unsigned)P.grid), sum_grid((unsigned)(sums + db_blocks));
    if constexpr (T == FG_F32) {
        if (A.dw) hipLaunchKernelGGL(grouped_f32_dw_kernel, grid, dim3(GF_THREADS), GF_LDS_BYTES + GW_LIST * 4, st, A);
        many ? launch_sum<128, GF_K, DS_MANY>(A, sum_grid, st) : launch_sum<128, GF_K, DS_FEW>(A, sum_grid, st);
    } else if (P.bm == 256) {
        if (A.dw) hipLaunchKernelGGL((grouped_dw_kernel<T, 256, 256, 2, 4>), grid, dim3(512), 2 * GW_ROWS * 512 * 2 + GW_LIST * 4, st, A);
        many ? launch_sum<256, GW_ROWS, DS_MANY>(A, sum_grid, st) : launch_sum<256, GW_ROWS, DS_FEW>(A, sum_grid, st);
    } else {
        if (A.dw) hipLaunchKernelGGL((grouped_dw_kernel<T, 128, 128, 2, 2>), grid, dim3(256), 2 * GW_ROWS * 256 * 2 + GW_LIST * 4, st, A);
        many ? launch_sum<128, GW_ROWS, DS_MANY>(A, sum_grid, st) : launch_sum<128, GW_ROWS, DS_FEW>(A, sum_grid, st);
    }
    FG_LAUNCH_CHECK("grouped_dw_kernel");
    return FG_OK;
}

}  // namespace

extern "C" fg_status_t fg_linear_grouped(const void* x, int64_t x_rows, int64_t x_stride, fg_dtype_t dtype, const float* x_scale,
                                         const int32_t* src_ids_dev, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows,
                                         int32_t n_groups, int32_t d_in, int32_t d_out, const void* W, const float* w_scale, const float* bias,
                                         int32_t relu, void* h_out, int64_t n_out, int64_t out_stride, fg_dtype_t out_dtype, void* stream) {
    const char* who = "fg_linear_grouped";
    FG_TRY(check_groups(who, order_dev, offsets_dev, max_rows, n_groups, d_in, d_out, dtype, x_rows, n_out));
    if (!fg_dtype_size(out_dtype) || (dtype == FG_F32 && out_dtype != FG_F32)) FG_FAIL(FG_ERR_DTYPE, "%s: fp32 rows give fp32, the others fp32, fp16 or bf16", who);
    const bool eight = dtype == FG_E4M3;
    if (eight != (x_scale != nullptr) || eight != (w_scale != nullptr)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: x_scale and w_scale go with FG_E4M3 rows, and only with them", who);
    if (((uintptr_t)x_scale | (uintptr_t)w_scale | (uintptr_t)bias | (uintptr_t)src_ids_dev) & 3) FG_FAIL(FG_ERR_INVALID_ARG, "%s: scales, bias and ids must be aligned to their elements", who);
    if (max_rows > 0 && n_out > 0 && x_rows > 0) {
        FG_TRY(check_matrix(who, "x", x, x_stride, (int64_t)d_in * (eight ? 1 : fg_dtype_size(dtype))));
        FG_TRY(check_matrix(who, "h_out", h_out, out_stride, (int64_t)d_out * fg_dtype_size(out_dtype)));
        FG_TRY(check_matrix(who, "W", W, 0, 0));
    }
    fg_clear_error();
    if (max_rows == 0 || n_out == 0 || x_rows == 0) return FG_OK;
    GlArgs A = {};
    A.G = {order_dev, offsets_dev, max_rows, n_groups};
    A.x = (const char*)x, A.W = (const char*)W, A.x_rows = x_rows, A.x_stride = x_stride, A.n = n_out, A.out_stride = out_stride;
    A.out_type = out_dtype, A.d_in = d_in, A.d_out = d_out, A.relu = relu;
    A.x_scale = x_scale, A.w_scale = w_scale, A.bias = bias, A.src_ids = src_ids_dev, A.out = (char*)h_out;
    A.a = (const char*)x, A.a_stride = x_stride, A.a_by = GL_A_SOURCE, A.K = d_in, A.N = d_out;
    if (dtype == FG_BF16) return tile_product<FG_BF16, true>(A, (hipStream_t)stream);
    if (dtype == FG_F16) return tile_product<FG_F16, true>(A, (hipStream_t)stream);
    if (dtype == FG_E4M3) return tile_product<FG_E4M3, false>(A, (hipStream_t)stream);
    return tile_product<FG_F32, true>(A, (hipStream_t)stream);
}

extern "C" size_t fg_linear_grouped_backward_workspace_bytes(fg_dtype_t dtype, int64_t max_rows, int32_t n_groups, int32_t d_in, int32_t d_out) {
    if (!fg_dtype_size(dtype) || max_rows < 0 || max_rows > FG_MAX_GROUPED_ROWS || n_groups < 1 || n_groups > FG_MAX_GROUPS || d_in <= 0 || d_in > FG_MAX_GROUPED_DIM ||
        d_out <= 0 || d_out > FG_MAX_GROUPED_DIM)
        return 0;
    return bw_plan(max_rows, n_groups, d_in, d_out, fg_dtype_size(dtype)).total();
}

extern "C" fg_status_t fg_linear_grouped_backward(const void* x, int64_t x_rows, int64_t x_stride, fg_dtype_t dtype, const int32_t* src_ids_dev,
                                                  const void* dh, int64_t dh_stride, fg_dtype_t dh_dtype, const void* h, int64_t h_stride, fg_dtype_t h_dtype,
                                                  int64_t n, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups,
                                                  int32_t d_in, int32_t d_out, const void* W, void* dx, int64_t dx_stride, fg_dtype_t dx_dtype,
                                                  float* dw_dev, float* db_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    const char* who = "fg_linear_grouped_backward";
    if (dtype == FG_E4M3) FG_FAIL(FG_ERR_DTYPE, "%s: 8-bit rows have no gradient", who);
    FG_TRY(check_groups(who, order_dev, offsets_dev, max_rows, n_groups, d_in, d_out, dtype, x_rows, n));
    const int e = fg_dtype_size(dtype);
    if (dh_dtype != dtype && dh_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: dh is of the type of x or fp32", who);
    if (h && (!fg_dtype_size(h_dtype) || (dtype == FG_F32 && h_dtype != FG_F32))) FG_FAIL(FG_ERR_DTYPE, "%s: h is of a type that the layer's output can have", who);
    if (dx && dx_dtype != dtype && dx_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: dx is of the type of x or fp32", who);
    if (!dx && !dw_dev && !db_dev) FG_FAIL(FG_ERR_INVALID_ARG, "%s: none of dx, dw and db is wanted", who);
    const bool work = max_rows > 0 && n > 0 && x_rows > 0;
    if (work) {
        FG_TRY(check_matrix(who, "dh", dh, dh_stride, (int64_t)d_out * fg_dtype_size(dh_dtype)));
        if (h) FG_TRY(check_matrix(who, "h", h, h_stride, (int64_t)d_out * fg_dtype_size(h_dtype)));
        if (dw_dev) FG_TRY(check_matrix(who, "x", x, x_stride, (int64_t)d_in * e));
        if (dx) FG_TRY(check_matrix(who, "dx", dx, dx_stride, (int64_t)d_in * fg_dtype_size(dx_dtype)));
        if (dx) FG_TRY(check_matrix(who, "W", W, 0, 0));
    }
    if (((uintptr_t)dw_dev | (uintptr_t)db_dev) & 15 || ((uintptr_t)src_ids_dev & 3)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: dw and db must be 16-byte aligned", who);
    const size_t need = fg_linear_grouped_backward_workspace_bytes(dtype, max_rows, n_groups, d_in, d_out);
    if (!ws_dev || ((uintptr_t)ws_dev & 15)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: the workspace must be 16-byte aligned device memory", who);
    if (ws_bytes < need) FG_FAIL(FG_ERR_SHAPE, "%s: workspace of %zu bytes, %zu are needed", who, ws_bytes, need);
    fg_clear_error();
    GlArgs A = {};
    A.G = {order_dev, offsets_dev, work ? max_rows : 0, n_groups};
    A.x = (const char*)x, A.W = (const char*)W, A.h = (const char*)h, A.dh = (const char*)dh, A.x_rows = x_rows, A.x_stride = x_stride, A.h_stride = h_stride;
    A.dh_stride = dh_stride, A.n = n, A.out_stride = dx_stride, A.dh_type = dh_dtype, A.h_type = h ? h_dtype : dtype, A.out_type = dx_dtype, A.d_in = d_in, A.d_out = d_out;
    A.src_ids = src_ids_dev, A.out = (char*)dx, A.dw = dw_dev, A.db = db_dev;
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == FG_F32) return backward<FG_F32>(who, A, work, st, ws_dev);
    return dtype == FG_BF16 ? backward<FG_BF16>(who, A, work, st, ws_dev) : backward<FG_F16>(who, A, work, st, ws_dev);
}

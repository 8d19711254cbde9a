// Element-wise work on listed rows: fg_dropout, fg_residual_norm and its backward pass, fg_quantize_rows.
//
// All of them are bound by the memory they read and write once (a large copy runs at 5.06 TB/s): dropout of 368640 x 768 bf16 232 us, 4.9 TB/s;
// residual and norm of 49152 x 256 fp32 33 us, 6.1 TB/s (part of it from the last-level cache), of 65536 x 1024 bf16 with 8-bit rows 91 us, 5.2;
// its gradients, 65536 x 1024 bf16, 123 us and 8 for the sums of dw, 5.1. A row belongs to a power of two of lanes, up to a wavefront's 64, each
// with pieces of eight adjacent values (16 bytes of a 16-bit type), and stays in registers between the sum over the row and the use
// of it; a row of more than 2048 values belongs to all wavefronts of a workgroup, which meet in LDS.
#include "row_list.h"
#include "row_types.h"

namespace {

constexpr int ROW_THREADS = 256;

// Dropout by position and column. A 64-bit word of the stream of (key, row) holds the draws of four columns.
struct DropArgs {
    uint64_t base;       // mix(key)
    uint32_t threshold;  // a draw below it drops; 0: no dropout
    float scale;
};
__device__ __forceinline__ void drop_piece(const DropArgs& D, uint64_t row_key, int c0, float (&f)[8]) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const uint64_t w = fg_word64(row_key, (uint64_t)(c0 / 4 + b));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t draw = (uint32_t)(w >> (16 * i)) & 0xFFFFu;
            f[4 * b + i] = draw >= D.threshold ? f[4 * b + i] * D.scale : 0.f;
        }
    }
}
DropArgs drop_args(float p, uint64_t key) {
    DropArgs D;
    D.base = fg_mix64(key);
    D.threshold = (uint32_t)floor((double)p * 65536.0 + 0.5);
    D.scale = D.threshold < 65536u ? (float)(65536.0 / (65536.0 - D.threshold)) : 0.f;
    return D;
}

template <int T>
__global__ __launch_bounds__(ROW_THREADS) void dropout_kernel(RowList L, int64_t rows, const char* x, int64_t x_stride, char* out,
                                                              int64_t out_stride, int d, int pieces, DropArgs D) {
    constexpr int E = T == FG_F32 ? 4 : 2;
    const int64_t count = row_count(L);
    const int64_t at = blockIdx.x * (int64_t)ROW_THREADS + threadIdx.x;
    const int64_t k = at / pieces;
    if (k >= rows) return;      // the next launch's (x may be out: a row that two launches take is dropped twice)
    const int c = (int)(at - k * pieces) * 8;
    const int64_t r = row_at(L, L.first + k, count);
    if (r < 0) return;
    float f[8];
    fg_piece_values<T>(fg_load_piece<T>(x + r * x_stride + (int64_t)c * E, d - c), f);
    if (D.threshold) drop_piece(D, fg_word64(D.base, (uint64_t)r), c, f);
    fg_store_piece<T>(out + r * out_stride + (int64_t)c * E, f, d - c);
}

// sum or maximum over the lanes of a row
__device__ __forceinline__ double lanes_sum(double v, int lanes) {
    for (int off = lanes >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
__device__ __forceinline__ float lanes_max(float v, int lanes) {
    for (int off = lanes >> 1; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}
// the same over the wavefronts of a workgroup that share a row
template <int WAVES>
__device__ __forceinline__ double row_sum(double v, int lanes, double* lds) {
    v = lanes_sum(v, lanes);
    if constexpr (WAVES > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += lds[w];
    }
    return v;
}
template <int WAVES>
__device__ __forceinline__ float row_max(float v, int lanes, double* lds) {
    v = lanes_max(v, lanes);
    if constexpr (WAVES > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (float)lds[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = fmaxf(v, (float)lds[w]);
    }
    return v;
}

struct NormArgs {
    RowList L;
    const char *x, *residual;
    int64_t x_stride, res_stride;
    int d, lanes;      // lanes of a row
    DropArgs D;
    const float* weight;
    float eps;
    char *sum_out, *y;
    int64_t sum_stride, y_stride;
    int y_dtype;
    float *y_scale, *rstd_out;
};

constexpr float E4M3_MAX = 448.f;
constexpr float AMAX_MIN = 7.888609052210118e-31f;      // 2^-100: 448 over it stays finite

// WAVES > 1: that many wavefronts to a row, else 64 / lanes rows to a wavefront. NORM false: rows as they are, in 8 bits.
template <int XT, int ST, int WAVES, int NP, bool NORM>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : ROW_THREADS) void residual_norm_kernel(NormArgs A) {
    constexpr int XE = XT == FG_F32 ? 4 : 2, SE = ST == FG_F32 ? 4 : 2;
    __shared__ double red[WAVES];
    const int64_t count = row_count(A.L);
    const int rows_per_wave = WAVES > 1 ? 1 : 64 / A.lanes;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int me = WAVES > 1 ? (int)threadIdx.x : lane & (A.lanes - 1);      // which piece of the row
    const int width = WAVES > 1 ? WAVES * 64 : A.lanes;
    const int64_t k = WAVES > 1 ? blockIdx.x : (blockIdx.x * (int64_t)(ROW_THREADS / 64) + wave) * rows_per_wave + lane / A.lanes;
    const int64_t r = row_at(A.L, A.L.first + k, count);
    if (WAVES > 1 && r < 0) return;      // the whole workgroup
    float v[NP][8];
    double ss = 0.0;
    if (r >= 0) {
        const char *xr = A.x + r * A.x_stride, *rr = A.residual + r * A.res_stride;
        fg_piece<XT> px[NP];
        fg_piece<ST> pr[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (me + width * i) * 8;
            if (c < A.d) px[i] = fg_load_piece<XT>(xr + (int64_t)c * XE, A.d - c);
            if (NORM && A.residual && c < A.d) pr[i] = fg_load_piece<ST>(rr + (int64_t)c * SE, A.d - c);
        }
        const uint64_t row_key = fg_word64(A.D.base, (uint64_t)r);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (me + width * i) * 8;
            if (c < A.d) {
                fg_piece_values<XT>(px[i], v[i]);
                if constexpr (NORM) {
                    if (A.D.threshold) drop_piece(A.D, row_key, c, v[i]);
                    if (A.residual) {
                        float f[8];
                        fg_piece_values<ST>(pr[i], f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[i][e] += f[e];
                    }
                    if (A.sum_out) fg_store_piece<ST>(A.sum_out + r * A.sum_stride + (int64_t)c * SE, v[i], A.d - c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss += (double)v[i][e] * (double)v[i][e];      // values beyond the row are zeros
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
            }
        }
    }
    if constexpr (NORM) {
        ss = row_sum<WAVES>(ss, A.lanes, red);
        const float rstd = (float)(1.0 / sqrt(ss / A.d + (double)A.eps));
        if (r >= 0 && me == 0 && A.rstd_out) A.rstd_out[r] = rstd;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (me + width * i) * 8;
            float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (A.weight && c < A.d) fg_piece_values<FG_F32>(fg_load_piece<FG_F32>((const char*)(A.weight + c), A.d - c), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * rstd * w[e];
        }
    }
    float inv = 1.f;
    if (!NORM || A.y_dtype == FG_E4M3) {
        float amax = AMAX_MIN;
        if (r >= 0)
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[i][e]));
        amax = row_max<WAVES>(amax, A.lanes, red);
        inv = E4M3_MAX * (1.f / amax);
        if (r >= 0 && me == 0) A.y_scale[r] = amax / E4M3_MAX;
    }
    if (r < 0) return;
    char* yr = A.y + r * A.y_stride;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (me + width * i) * 8;
        if (c >= A.d) continue;
        if (!NORM || A.y_dtype == FG_E4M3) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = v[i][e] * inv;      // 448 at most but for the rounding of inv; a NaN stays one
                v[i][e] = q > E4M3_MAX ? E4M3_MAX : (q < -E4M3_MAX ? -E4M3_MAX : q);
            }
            fg_store_piece_e4m3(yr + c, v[i], A.d - c);
        } else if (A.y_dtype == FG_F32) {
            fg_store_piece<FG_F32>(yr + (int64_t)c * 4, v[i], A.d - c);
        } else if constexpr (XT != FG_F32) {
            fg_store_piece<XT>(yr + (int64_t)c * 2, v[i], A.d - c);
        }
    }
}

struct NormBwArgs {
    RowList L;
    const char *dy, *sum, *ds_in;
    int64_t dy_stride, sum_stride, ds_in_stride;
    const float *rstd, *weight;
    int d, lanes;
    DropArgs D;
    char *ds_out, *dx;
    int64_t ds_stride, dx_stride;
    float* part;      // [workgroups][d] sums for dw, or NULL
};

// A workgroup walks rows blockIdx, blockIdx + gridDim, ... (of its wavefronts' rows) and keeps its columns' sums for dw in registers.
template <int GT, int ST, int WAVES, int NP>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : ROW_THREADS) void residual_norm_backward_kernel(NormBwArgs A) {
    constexpr int GE = GT == FG_F32 ? 4 : 2, SE = ST == FG_F32 ? 4 : 2;
    extern __shared__ __attribute__((aligned(16))) float nb_lds[];
    __shared__ double red[WAVES];
    const int64_t count = row_count(A.L);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int me = WAVES > 1 ? (int)threadIdx.x : lane & (A.lanes - 1);
    const int width = WAVES > 1 ? WAVES * 64 : A.lanes;
    const int per_block = WAVES > 1 ? 1 : ROW_THREADS / A.lanes;      // rows at a time
    const int my_row = WAVES > 1 ? 0 : threadIdx.x / A.lanes;
    float dw[NP][8], w[NP][8];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (me + width * i) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dw[i][e] = 0.f;
            w[i][e] = 1.f;
        }
        if (A.weight && c < A.d) fg_piece_values<FG_F32>(fg_load_piece<FG_F32>((const char*)(A.weight + c), A.d - c), w[i]);
    }
    for (int64_t k0 = blockIdx.x * (int64_t)per_block; k0 < count; k0 += (int64_t)gridDim.x * per_block) {      // uniform
        const int64_t r = row_at(A.L, k0 + my_row, count);
        float t[NP][8], xh[NP][8];
        double dot = 0.0;
        float rstd = 0.f;
        if (r >= 0) {
            rstd = A.rstd[r];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = (me + width * i) * 8;
                if (c < A.d) {
                    fg_piece_values<GT>(fg_load_piece<GT>(A.dy + r * A.dy_stride + (int64_t)c * GE, A.d - c), t[i]);
                    fg_piece_values<ST>(fg_load_piece<ST>(A.sum + r * A.sum_stride + (int64_t)c * SE, A.d - c), xh[i]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        xh[i][e] *= rstd;
                        dw[i][e] += t[i][e] * xh[i][e];
                        t[i][e] *= w[i][e];
                        dot += (double)t[i][e] * (double)xh[i][e];
                    }
                }
            }
        }
        dot = row_sum<WAVES>(dot, A.lanes, red);
        if (r < 0) continue;      // WAVES > 1: the whole workgroup (the next row_sum has its own barriers)
        const float mean = (float)(dot / A.d);
        const uint64_t row_key = fg_word64(A.D.base, (uint64_t)r);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (me + width * i) * 8;
            if (c >= A.d) continue;
            float f[8] = {};
            if (A.ds_in) fg_piece_values<GT>(fg_load_piece<GT>(A.ds_in + r * A.ds_in_stride + (int64_t)c * GE, A.d - c), f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += rstd * (t[i][e] - xh[i][e] * mean);
            fg_store_piece<GT>(A.ds_out + r * A.ds_stride + (int64_t)c * GE, f, A.d - c);
            if (A.dx) {
                if (A.D.threshold) drop_piece(A.D, row_key, c, f);
                fg_store_piece<GT>(A.dx + r * A.dx_stride + (int64_t)c * GE, f, A.d - c);
            }
        }
    }
    if (!A.part) return;
    // the rows of a workgroup that were walked side by side: their sums meet in LDS, `width * NP` pieces for each of them
    if constexpr (WAVES > 1) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (me + width * i) * 8;
            if (c < A.d) fg_store_piece<FG_F32>((char*)(A.part + blockIdx.x * (int64_t)A.d + c), dw[i], A.d - c);
        }
    } else {
        const int span = width * NP * 8;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) nb_lds[my_row * span + (me + width * i) * 8 + e] = dw[i][e];
        __syncthreads();
        for (int c = threadIdx.x; c < A.d; c += ROW_THREADS) {
            float s = 0.f;
            for (int q = 0; q < per_block; ++q) s += nb_lds[q * span + c];
            A.part[blockIdx.x * (int64_t)A.d + c] = s;
        }
    }
}

// dw[c] = sum over the workgroups of part[.][c] in fp64; 32 columns a workgroup, eight runs of partial sums side by side
__global__ __launch_bounds__(ROW_THREADS) void column_sums_kernel(const float* __restrict__ part, int n_part, int d, float* __restrict__ dw) {
    __shared__ double red[ROW_THREADS];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31);
    double s = 0.0;
    if (c < d)
#pragma unroll 8
        for (int b = threadIdx.x >> 5; b < n_part; b += ROW_THREADS / 32) s += (double)part[(int64_t)b * d + c];
    red[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 32 && c < d) {
        for (int q = 1; q < ROW_THREADS / 32; ++q) s += red[threadIdx.x + 32 * q];
        dw[c] = (float)s;
    }
}

static_assert(FG_MAX_NORM_DIM == 8 * 64 * 4 * 8, "eight wavefronts with four pieces a lane");
constexpr int64_t NB_MAX_BLOCKS = 1024;

// how a row of d values is laid out over lanes
struct RowShape {
    int waves, np, lanes;      // waves 1: 256 / lanes rows to a workgroup
};
RowShape row_shape(int d) {
    const int pieces = (d + 7) / 8;
    RowShape s = {1, 1, 64};
    if (pieces <= 64) {
        s.lanes = 1;
        while (s.lanes < pieces) s.lanes *= 2;
    } else if (pieces <= 128) {
        s.np = 2;
    } else if (pieces <= 256) {
        s.np = 4;
    } else {
        s.waves = pieces <= 1024 ? 4 : 8;
        s.np = 4;
    }
    return s;
}
int64_t nb_blocks(int64_t max_rows, int d) {
    const RowShape s = row_shape(d);
    const int64_t b = fg_ceil_div(max_rows, s.waves > 1 ? 1 : ROW_THREADS / s.lanes);
    return b < NB_MAX_BLOCKS ? b : NB_MAX_BLOCKS;
}

template <int XT, int ST, bool NORM>
void norm_launch(const RowShape& s, NormArgs A, hipStream_t st) {
    const int per_block = s.waves > 1 ? 1 : ROW_THREADS / s.lanes;
    const int64_t at_once = (FG_MAX_GRID / 2 - 1) * per_block;      // rows of a launch
    for (; A.L.first < A.L.max_rows; A.L.first += at_once) {
        const int64_t rows = A.L.max_rows - A.L.first < at_once ? A.L.max_rows - A.L.first : at_once;
        const dim3 grid((unsigned)fg_ceil_div(rows, per_block));
        if (s.waves == 1 && s.np == 1)
            hipLaunchKernelGGL((residual_norm_kernel<XT, ST, 1, 1, NORM>), grid, dim3(ROW_THREADS), 0, st, A);
        else if (s.waves == 1 && s.np == 2)
            hipLaunchKernelGGL((residual_norm_kernel<XT, ST, 1, 2, NORM>), grid, dim3(ROW_THREADS), 0, st, A);
        else if (s.waves == 1)
            hipLaunchKernelGGL((residual_norm_kernel<XT, ST, 1, 4, NORM>), grid, dim3(ROW_THREADS), 0, st, A);
        else if (s.waves == 4)
            hipLaunchKernelGGL((residual_norm_kernel<XT, ST, 4, 4, NORM>), grid, dim3(256), 0, st, A);
        else
            hipLaunchKernelGGL((residual_norm_kernel<XT, ST, 8, 4, NORM>), grid, dim3(512), 0, st, A);
    }
}

template <int GT, int ST>
void norm_bw_launch(const RowShape& s, const NormBwArgs& A, hipStream_t st) {
    const unsigned grid = (unsigned)nb_blocks(A.L.max_rows, A.d);
    const size_t lds = A.part ? (size_t)ROW_THREADS * s.np * 8 * 4 : 0;
    if (s.waves == 1 && s.np == 1)
        hipLaunchKernelGGL((residual_norm_backward_kernel<GT, ST, 1, 1>), dim3(grid), dim3(ROW_THREADS), lds, st, A);
    else if (s.waves == 1 && s.np == 2)
        hipLaunchKernelGGL((residual_norm_backward_kernel<GT, ST, 1, 2>), dim3(grid), dim3(ROW_THREADS), lds, st, A);
    else if (s.waves == 1)
        hipLaunchKernelGGL((residual_norm_backward_kernel<GT, ST, 1, 4>), dim3(grid), dim3(ROW_THREADS), lds, st, A);
    else if (s.waves == 4)
        hipLaunchKernelGGL((residual_norm_backward_kernel<GT, ST, 4, 4>), dim3(grid), dim3(256), 0, st, A);
    else
        hipLaunchKernelGGL((residual_norm_backward_kernel<GT, ST, 8, 4>), dim3(grid), dim3(512), 0, st, A);
}

}  // namespace

extern "C" fg_status_t fg_dropout(const void* x, int64_t x_stride, fg_dtype_t dtype, const int32_t* rows_dev, const int64_t* n_rows_dev,
                                  int64_t max_rows, int64_t n, int32_t d, float p, uint64_t key, void* out, int64_t out_stride, void* stream) {
    const char* who = "fg_dropout";
    const int e = fg_dtype_size(dtype);
    if (!e) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type %d", who, (int)dtype);
    FG_TRY(check_rows(who, rows_dev, n_rows_dev, max_rows, n, d));
    if (!(p >= 0.f && p <= 1.f)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: p = %g is not in [0, 1]", who, (double)p);
    if (max_rows > 0 && n > 0 && (!x || !out)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: x and out must not be NULL", who);
    FG_TRY(check_array(who, "x", x, x_stride, e, d));
    FG_TRY(check_array(who, "out", out, out_stride, e, d));
    fg_clear_error();
    if (max_rows == 0 || n == 0) return FG_OK;
    const int pieces = (int)fg_ceil_div(d, 8);
    const int64_t at_once = (FG_MAX_GRID - 1) * ROW_THREADS / pieces;      // rows of a launch
    RowList L = {rows_dev, n_rows_dev, max_rows, n, 0};
    const DropArgs D = drop_args(p, key);
    hipStream_t st = (hipStream_t)stream;
#define FG_DROP(T) hipLaunchKernelGGL((dropout_kernel<T>), dim3((unsigned)blocks), dim3(ROW_THREADS), 0, st, L, rows, (const char*)x, x_stride, (char*)out, out_stride, d, pieces, D)
    for (; L.first < max_rows; L.first += at_once) {
        const int64_t rows = max_rows - L.first < at_once ? max_rows - L.first : at_once, blocks = fg_ceil_div(rows * pieces, ROW_THREADS);
        if (dtype == FG_F32)
            FG_DROP(FG_F32);
        else if (dtype == FG_F16)
            FG_DROP(FG_F16);
        else
            FG_DROP(FG_BF16);
    }
#undef FG_DROP
    FG_LAUNCH_CHECK("dropout_kernel");
    return FG_OK;
}

extern "C" fg_status_t fg_residual_norm(const void* x, int64_t x_stride, fg_dtype_t dtype, const void* residual, int64_t residual_stride,
                                        fg_dtype_t sum_dtype, const int32_t* rows_dev, const int64_t* n_rows_dev, int64_t max_rows, int64_t n,
                                        int32_t d, float p, uint64_t key, const float* weight, float eps, void* sum_out, int64_t sum_stride, void* y,
                                        int64_t y_stride, fg_dtype_t y_dtype, float* y_scale, float* rstd_out, void* stream) {
    const char* who = "fg_residual_norm";
    const int e = fg_dtype_size(dtype), se = fg_dtype_size(sum_dtype);
    if (!e) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type %d", who, (int)dtype);
    if (sum_dtype != dtype && sum_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: residual and sum are of the type of x or fp32", who);
    if (y_dtype != dtype && y_dtype != FG_F32 && y_dtype != FG_E4M3) FG_FAIL(FG_ERR_DTYPE, "%s: y is of the type of x, fp32 or FG_E4M3", who);
    FG_TRY(check_rows(who, rows_dev, n_rows_dev, max_rows, n, d));
    if (d > FG_MAX_NORM_DIM) FG_FAIL(FG_ERR_SHAPE, "%s: d = %d is more than %d", who, d, FG_MAX_NORM_DIM);
    if (!(p >= 0.f && p <= 1.f)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: p = %g is not in [0, 1]", who, (double)p);
    if (!(eps >= 0.f)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: eps must not be negative", who);
    if (max_rows > 0 && n > 0 && (!x || !y)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: x and y must not be NULL", who);
    if ((y_dtype == FG_E4M3) != (y_scale != nullptr) && max_rows > 0 && n > 0)
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: y_scale goes with FG_E4M3 rows, and only with them", who);
    FG_TRY(check_array(who, "x", x, x_stride, e, d));
    if (residual) FG_TRY(check_array(who, "residual", residual, residual_stride, se, d));
    if (sum_out) FG_TRY(check_array(who, "sum_out", sum_out, sum_stride, se, d));
    FG_TRY(check_array(who, "y", y, y_stride, y_dtype == FG_E4M3 ? 1 : fg_dtype_size(y_dtype), d));
    if (((uintptr_t)weight | (uintptr_t)y_scale | (uintptr_t)rstd_out) & 3) FG_FAIL(FG_ERR_INVALID_ARG, "%s: weight, y_scale or rstd_out is not aligned", who);
    fg_clear_error();
    if (max_rows == 0 || n == 0) return FG_OK;
    const RowShape s = row_shape(d);
    const NormArgs A = {{rows_dev, n_rows_dev, max_rows, n, 0}, (const char*)x, (const char*)residual, x_stride, residual_stride, d, s.lanes, drop_args(p, key), weight, eps,
                        (char*)sum_out, (char*)y, sum_stride, y_stride, (int)y_dtype, y_scale, rstd_out};
    hipStream_t st = (hipStream_t)stream;
    if (dtype == FG_F32)
        norm_launch<FG_F32, FG_F32, true>(s, A, st);
    else if (dtype == FG_F16 && sum_dtype == FG_F16)
        norm_launch<FG_F16, FG_F16, true>(s, A, st);
    else if (dtype == FG_F16)
        norm_launch<FG_F16, FG_F32, true>(s, A, st);
    else if (sum_dtype == FG_BF16)
        norm_launch<FG_BF16, FG_BF16, true>(s, A, st);
    else
        norm_launch<FG_BF16, FG_F32, true>(s, A, st);
    FG_LAUNCH_CHECK("residual_norm_kernel");
    return FG_OK;
}

extern "C" fg_status_t fg_quantize_rows(const void* x, int64_t x_stride, fg_dtype_t dtype, int64_t n_rows, int32_t d, void* q, int64_t q_stride,
                                        float* scale, void* stream) {
    const char* who = "fg_quantize_rows";
    const int e = fg_dtype_size(dtype);
    if (!e) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type %d", who, (int)dtype);
    FG_TRY(check_rows(who, nullptr, nullptr, n_rows, n_rows, d));
    if (d > FG_MAX_NORM_DIM) FG_FAIL(FG_ERR_SHAPE, "%s: d = %d is more than %d", who, d, FG_MAX_NORM_DIM);
    if (n_rows > 0 && (!x || !q || !scale)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: x, q and scale must not be NULL", who);
    FG_TRY(check_array(who, "x", x, x_stride, e, d));
    FG_TRY(check_array(who, "q", q, q_stride, 1, d));
    if ((uintptr_t)scale & 3) FG_FAIL(FG_ERR_INVALID_ARG, "%s: scale is not aligned", who);
    fg_clear_error();
    if (n_rows == 0) return FG_OK;
    const RowShape s = row_shape(d);
    const NormArgs A = {{nullptr, nullptr, n_rows, n_rows, 0}, (const char*)x, nullptr, x_stride, 0, d, s.lanes, {}, nullptr, 0.f,
                        nullptr, (char*)q, 0, q_stride, (int)FG_E4M3, scale, nullptr};
    hipStream_t st = (hipStream_t)stream;
    if (dtype == FG_F32)
        norm_launch<FG_F32, FG_F32, false>(s, A, st);
    else if (dtype == FG_F16)
        norm_launch<FG_F16, FG_F32, false>(s, A, st);
    else
        norm_launch<FG_BF16, FG_F32, false>(s, A, st);
    FG_LAUNCH_CHECK("residual_norm_kernel");
    return FG_OK;
}

extern "C" size_t fg_residual_norm_backward_workspace_bytes(int64_t max_rows, int32_t d) {
    if (max_rows < 0 || max_rows > INT32_MAX || d <= 0 || d > FG_MAX_NORM_DIM) return 0;
    return fg_align_up((size_t)nb_blocks(max_rows, d) * d * 4, 16);
}

extern "C" fg_status_t fg_residual_norm_backward(const void* dy, int64_t dy_stride, fg_dtype_t grad_dtype, const void* sum, int64_t sum_stride,
                                                 fg_dtype_t sum_dtype, const float* rstd, const float* weight, const void* dsum_in,
                                                 int64_t dsum_in_stride, const int32_t* rows_dev, const int64_t* n_rows_dev, int64_t max_rows,
                                                 int64_t n, int32_t d, float p, uint64_t key, void* dsum_out, int64_t dsum_stride, void* dx,
                                                 int64_t dx_stride, float* dw_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    const char* who = "fg_residual_norm_backward";
    const int ge = fg_dtype_size(grad_dtype), se = fg_dtype_size(sum_dtype);
    if (!ge || !se) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type", who);
    FG_TRY(check_rows(who, rows_dev, n_rows_dev, max_rows, n, d));
    if (d > FG_MAX_NORM_DIM) FG_FAIL(FG_ERR_SHAPE, "%s: d = %d is more than %d", who, d, FG_MAX_NORM_DIM);
    if (!(p >= 0.f && p <= 1.f)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: p = %g is not in [0, 1]", who, (double)p);
    const bool work = max_rows > 0 && n > 0;
    if (work && (!dy || !sum || !rstd || !dsum_out)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: dy, sum, rstd and dsum_out must not be NULL", who);
    FG_TRY(check_array(who, "dy", dy, dy_stride, ge, d));
    FG_TRY(check_array(who, "sum", sum, sum_stride, se, d));
    FG_TRY(check_array(who, "dsum_out", dsum_out, dsum_stride, ge, d));
    if (dsum_in) FG_TRY(check_array(who, "dsum_in", dsum_in, dsum_in_stride, ge, d));
    if (dx) FG_TRY(check_array(who, "dx", dx, dx_stride, ge, d));
    if (((uintptr_t)weight | (uintptr_t)rstd | (uintptr_t)dw_dev) & 3) FG_FAIL(FG_ERR_INVALID_ARG, "%s: weight, rstd or dw is not aligned", who);
    if (dw_dev && max_rows > 0) {
        if (!ws_dev || ((uintptr_t)ws_dev & 15)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: the workspace must be 16-byte aligned device memory", who);
        const size_t need = fg_residual_norm_backward_workspace_bytes(max_rows, d);
        if (ws_bytes < need) FG_FAIL(FG_ERR_SHAPE, "%s: workspace of %zu bytes, %zu are needed", who, ws_bytes, need);
    }
    fg_clear_error();
    hipStream_t st = (hipStream_t)stream;
    const RowShape s = row_shape(d);
    if (work) {
        const NormBwArgs A = {{rows_dev, n_rows_dev, max_rows, n, 0}, (const char*)dy, (const char*)sum, (const char*)dsum_in, dy_stride, sum_stride, dsum_in_stride,
                              rstd, weight, d, s.lanes, drop_args(p, key), (char*)dsum_out, (char*)dx, dsum_stride, dx_stride,
                              dw_dev ? (float*)ws_dev : nullptr};
#define FG_NB(G)                                       \
    do {                                               \
        if (sum_dtype == FG_F32)                       \
            norm_bw_launch<G, FG_F32>(s, A, st);       \
        else if (sum_dtype == FG_F16)                  \
            norm_bw_launch<G, FG_F16>(s, A, st);       \
        else                                           \
            norm_bw_launch<G, FG_BF16>(s, A, st);      \
    } while (0)
        if (grad_dtype == FG_F32)
            FG_NB(FG_F32);
        else if (grad_dtype == FG_F16)
            FG_NB(FG_F16);
        else
            FG_NB(FG_BF16);
#undef FG_NB
        FG_LAUNCH_CHECK("residual_norm_backward_kernel");
    }
    if (dw_dev) {
        hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)fg_ceil_div(d, 32)), dim3(ROW_THREADS), 0, st, (const float*)ws_dev,
                           work ? (int)nb_blocks(max_rows, d) : 0, d, dw_dev);
        FG_LAUNCH_CHECK("column_sums_kernel");
    }
    return FG_OK;
}

// fg_linear_grouped and its gradients: the dense update with a weight matrix per group of rows.
//
// The rows of a group lie behind each other in `order`; how many there are is known on the device only. The grid is sized for the
// bound (every group may leave one tile partly filled), and a workgroup finds its group and its rows from the offsets.
#include "row_types.h"
#include "scan.h"

namespace {

constexpr int GL_THREADS = 256;
constexpr int GL_TILE = 64, GL_K = 16;

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
__device__ __forceinline__ bool find_tile(const Groups& G, int64_t tile, int size, int& group, int64_t& k0, int64_t& k1) {
    int64_t before = 0;
    for (int base = 0; base < G.n_groups; base += 64) {
        const int g = base + fg_lane();
        int64_t from = 0, to = 0;
        if (g < G.n_groups) {
            from = group_offset(G, g);
            to = group_offset(G, g + 1);
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

template <int T>
__device__ __forceinline__ float value_at(const char* p, int64_t i) {
    if constexpr (T == FG_F32)
        return ((const float*)p)[i];
    else if constexpr (T == FG_BF16)
        return __uint_as_float((unsigned int)((const unsigned short*)p)[i] << 16);
    else if constexpr (T == FG_F16)
        return (float)((const _Float16*)p)[i];
    else
        return __builtin_amdgcn_cvt_f32_fp8((int)((const unsigned char*)p)[i], 0);
}
__device__ __forceinline__ float value_of(int type, const char* p, int64_t i) {
    return type == FG_F32 ? value_at<FG_F32>(p, i) : type == FG_BF16 ? value_at<FG_BF16>(p, i) : type == FG_F16 ? value_at<FG_F16>(p, i) : value_at<FG_E4M3>(p, i);
}
__device__ __forceinline__ void put_value(int type, char* p, int64_t i, float v) {
    if (type == FG_F32)
        ((float*)p)[i] = v;
    else if (type == FG_BF16)
        ((__bf16*)p)[i] = (__bf16)v;
    else
        ((_Float16*)p)[i] = (_Float16)v;
}
__device__ __forceinline__ float rounded(int type, float v) { return type == FG_F32 ? v : type == FG_BF16 ? (float)(__bf16)v : (float)(_Float16)v; }

struct GlArgs {
    Groups G;
    const char *x, *W, *h, *dh;
    int64_t x_rows, x_stride, h_stride, dh_stride, n, out_stride;
    int type, dh_type, out_type, d_in, d_out, relu, tiles_n;
    const float *x_scale, *w_scale, *bias;
    const int32_t* src_ids;
    char* out;
    float *dw, *db;
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
__device__ __forceinline__ float dz_at(const GlArgs& A, int32_t r, int c, bool round) {
    float v = value_of(A.dh_type, A.dh + r * A.dh_stride, c);
    if (A.h && !(value_of(A.type, A.h + r * A.h_stride, c) > 0.f)) v = 0.f;
    return round ? rounded(A.type, v) : v;
}

// BACK false: h_out; true: dx
template <bool BACK>
__global__ __launch_bounds__(GL_THREADS) void grouped_linear_kernel(GlArgs A) {
    __shared__ float a[GL_K][GL_TILE + 4], b[GL_K][GL_TILE + 4];
    __shared__ int32_t pos[GL_TILE], src[GL_TILE];
    int g;
    int64_t k0, k1;
    if (!find_tile(A.G, blockIdx.x / A.tiles_n, GL_TILE, g, k0, k1)) return;
    const int n0 = (int)(blockIdx.x % A.tiles_n) * GL_TILE;
    const int K = BACK ? A.d_out : A.d_in, N = BACK ? A.d_in : A.d_out;
    const int t = threadIdx.x;
    if (t < GL_TILE) entry(A, k0 + t, k1, pos[t], src[t]);
    __syncthreads();
    const int64_t w0 = (int64_t)g * A.d_in * A.d_out;
    float acc[4][4] = {};
    const int tm = (t / 16) * 4, tn = (t % 16) * 4;
    for (int kk = 0; kk < K; kk += GL_K) {
        for (int i = t; i < GL_K * GL_TILE; i += GL_THREADS) {
            const int m = i / GL_K, k = kk + i % GL_K;
            float v = 0.f;
            if (pos[m] >= 0 && k < K) v = BACK ? dz_at(A, pos[m], k, true) : value_of(A.type, A.x + src[m] * A.x_stride, k);
            a[i % GL_K][m] = v;
            const int c = n0 + m;
            const bool by_column = BACK || A.type == FG_E4M3;      // W has the contraction index behind
            b[i % GL_K][m] = c < N && k < K ? value_of(A.type, A.W, w0 + (by_column ? (int64_t)c * K + k : (int64_t)k * N + c)) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < GL_K; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += a[k][tm + i] * b[k][tn + j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int32_t r = pos[tm + i];
        if (r < 0) continue;
        for (int j = 0; j < 4; ++j) {
            const int c = n0 + tn + j;
            if (c >= N) continue;
            float v = acc[i][j];
            if (!BACK) {
                if (A.x_scale) v *= A.x_scale[src[tm + i]] * A.w_scale[(int64_t)g * A.d_out + c];
                if (A.bias) v += A.bias[(int64_t)g * A.d_out + c];
                if (A.relu) v = v < 0.f ? 0.f : v;
            }
            put_value(A.out_type, A.out + r * A.out_stride, c, v);
        }
    }
}

// dW and db: a workgroup per group and tile of dW
__global__ __launch_bounds__(GL_THREADS) void grouped_weights_kernel(GlArgs A) {
    __shared__ float a[GL_K][GL_TILE + 4], b[GL_K][GL_TILE + 4], bz[GL_K][GL_TILE + 4];
    const int tiles_m = (A.d_in + GL_TILE - 1) / GL_TILE;
    const int g = blockIdx.x / (tiles_m * A.tiles_n), tile = blockIdx.x % (tiles_m * A.tiles_n);
    const int m0 = tile / A.tiles_n * GL_TILE, n0 = tile % A.tiles_n * GL_TILE;
    const int64_t from = group_offset(A.G, g), to = group_offset(A.G, g + 1);
    const int t = threadIdx.x, tm = (t / 16) * 4, tn = (t % 16) * 4;
    double acc[4][4] = {}, sum = 0.0;
    for (int64_t kk = from; kk < to; kk += GL_K) {
        for (int i = t; i < GL_K * GL_TILE; i += GL_THREADS) {
            const int k = i / GL_TILE, c = i % GL_TILE;
            int32_t r, s;
            entry(A, kk + k, to, r, s);
            a[k][c] = r >= 0 && m0 + c < A.d_in && A.dw ? value_of(A.type, A.x + s * A.x_stride, m0 + c) : 0.f;
            b[k][c] = r >= 0 && n0 + c < A.d_out ? dz_at(A, r, n0 + c, true) : 0.f;
            bz[k][c] = r >= 0 && n0 + c < A.d_out ? dz_at(A, r, n0 + c, false) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < GL_K; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += (double)a[k][tm + i] * (double)b[k][tn + j];
        if (t < GL_TILE)
            for (int k = 0; k < GL_K; ++k) sum += (double)bz[k][t];
        __syncthreads();
    }
    if (A.dw)
        for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j)
                if (m0 + tm + i < A.d_in && n0 + tn + j < A.d_out)
                    A.dw[((int64_t)g * A.d_in + m0 + tm + i) * A.d_out + n0 + tn + j] = (float)acc[i][j];
    if (A.db && m0 == 0 && t < GL_TILE && n0 + t < A.d_out) A.db[(int64_t)g * A.d_out + n0 + t] = (float)sum;
}

fg_status_t check_groups(const char* who, const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups, int32_t d_in, int32_t d_out,
                         fg_dtype_t dtype, int64_t x_rows, int64_t n) {
    const int e = dtype == FG_E4M3 ? 1 : fg_dtype_size(dtype);
    if (!e) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type %d", who, (int)dtype);
    if (max_rows < 0 || max_rows > INT32_MAX || x_rows < 0 || x_rows > INT32_MAX || n < 0 || n > INT32_MAX)
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: a number of rows is negative or too large", who);
    if (n_groups < 1 || n_groups > FG_MAX_GROUPS) FG_FAIL(FG_ERR_INVALID_ARG, "%s: n_groups = %d is not in 1..%d", who, n_groups, FG_MAX_GROUPS);
    const int step_in = 16 / e, step_out = dtype == FG_F32 ? 4 : 8;
    if (d_in <= 0 || d_in % step_in || d_out <= 0 || d_out % step_out || d_in > 65536 || d_out > 65536)
        FG_FAIL(FG_ERR_SHAPE, "%s: d_in = %d must be a multiple of %d and d_out = %d of %d for this type, 65536 at most", who, d_in, step_in, d_out, step_out);
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
    A.type = dtype, A.out_type = out_dtype, A.d_in = d_in, A.d_out = d_out, A.relu = relu, A.tiles_n = (int)fg_ceil_div(d_out, GL_TILE);
    A.x_scale = x_scale, A.w_scale = w_scale, A.bias = bias, A.src_ids = src_ids_dev, A.out = (char*)h_out;
    const int64_t grid = row_tiles(max_rows, n_groups, GL_TILE) * A.tiles_n;
    if (grid > INT32_MAX) FG_FAIL(FG_ERR_SHAPE, "%s: too many rows and columns for one call", who);
    hipLaunchKernelGGL((grouped_linear_kernel<false>), dim3((unsigned)grid), dim3(GL_THREADS), 0, (hipStream_t)stream, A);
    FG_LAUNCH_CHECK("grouped_linear_kernel");
    return FG_OK;
}

extern "C" size_t fg_linear_grouped_backward_workspace_bytes(fg_dtype_t dtype, int64_t max_rows, int32_t n_groups, int32_t d_in, int32_t d_out) {
    if (!fg_dtype_size(dtype) || max_rows < 0 || max_rows > INT32_MAX || n_groups < 1 || n_groups > FG_MAX_GROUPS || d_in <= 0 || d_out <= 0) return 0;
    return 16;
}

extern "C" fg_status_t fg_linear_grouped_backward(const void* x, int64_t x_rows, int64_t x_stride, fg_dtype_t dtype, const int32_t* src_ids_dev,
                                                  const void* dh, int64_t dh_stride, fg_dtype_t dh_dtype, const void* h, int64_t h_stride, int64_t n,
                                                  const int32_t* order_dev, const int64_t* offsets_dev, int64_t max_rows, int32_t n_groups,
                                                  int32_t d_in, int32_t d_out, const void* W, void* dx, int64_t dx_stride, fg_dtype_t dx_dtype,
                                                  float* dw_dev, float* db_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    const char* who = "fg_linear_grouped_backward";
    if (dtype == FG_E4M3) FG_FAIL(FG_ERR_DTYPE, "%s: 8-bit rows have no gradient", who);
    FG_TRY(check_groups(who, order_dev, offsets_dev, max_rows, n_groups, d_in, d_out, dtype, x_rows, n));
    const int e = fg_dtype_size(dtype);
    if (dh_dtype != dtype && dh_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: dh is of the type of x or fp32", who);
    if (dx && dx_dtype != dtype && dx_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: dx is of the type of x or fp32", who);
    if (!dx && !dw_dev && !db_dev) FG_FAIL(FG_ERR_INVALID_ARG, "%s: none of dx, dw and db is wanted", who);
    const bool work = max_rows > 0 && n > 0 && x_rows > 0;
    if (work) {
        FG_TRY(check_matrix(who, "dh", dh, dh_stride, (int64_t)d_out * fg_dtype_size(dh_dtype)));
        if (h) FG_TRY(check_matrix(who, "h", h, h_stride, (int64_t)d_out * e));
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
    A.dh_stride = dh_stride, A.n = n, A.out_stride = dx_stride, A.type = dtype, A.dh_type = dh_dtype, A.out_type = dx_dtype, A.d_in = d_in, A.d_out = d_out;
    A.src_ids = src_ids_dev, A.out = (char*)dx, A.dw = dw_dev, A.db = db_dev;
    hipStream_t st = (hipStream_t)stream;
    if (dx && work) {
        A.tiles_n = (int)fg_ceil_div(d_in, GL_TILE);
        const int64_t grid = row_tiles(max_rows, n_groups, GL_TILE) * A.tiles_n;
        if (grid > INT32_MAX) FG_FAIL(FG_ERR_SHAPE, "%s: too many rows and columns for one call", who);
        hipLaunchKernelGGL((grouped_linear_kernel<true>), dim3((unsigned)grid), dim3(GL_THREADS), 0, st, A);
        FG_LAUNCH_CHECK("grouped_linear_kernel");
    }
    if (dw_dev || db_dev) {
        A.tiles_n = (int)fg_ceil_div(d_out, GL_TILE);
        const int64_t grid = n_groups * A.tiles_n * fg_ceil_div(d_in, GL_TILE);
        if (grid > INT32_MAX) FG_FAIL(FG_ERR_SHAPE, "%s: too many groups and columns for one call", who);
        hipLaunchKernelGGL(grouped_weights_kernel, dim3((unsigned)grid), dim3(GL_THREADS), 0, st, A);
        FG_LAUNCH_CHECK("grouped_weights_kernel");
    }
    return FG_OK;
}

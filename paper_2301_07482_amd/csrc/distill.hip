// fg_distill_loss: a student's loss against a teacher's stored top logits and against labels, with its gradient.
//
// A row of logits is read once and its gradient written once; both softmaxes of it (at the temperature and as it is) come from the values held in
// registers. A row belongs to a power of two of lanes, up to a wavefront's 64, or to the wavefronts of a workgroup, as wide as it is;
// beyond REG_MAX columns what does not fit the registers is read again. The k classes that the teacher has stored, and the label, are entries of
// their own: their logits are fetched one by one, their gradients are formed apart (each sums the shares of all entries of its class, so that
// a class that is stored twice gets the same value from both) and written over what the row's pass has left there.
#include <type_traits>

#include "row_list.h"
#include "row_types.h"

namespace {

constexpr int DL_THREADS = 256, DL_MIN_LANES = 8;
constexpr float LOG2E = 1.4426950408889634f;

struct DistillArgs {
    RowList L;
    const char* h;
    int64_t h_stride;
    int d, lanes, k;      // lanes of a row
    const int32_t *ids, *top_idx;
    const char* top_val;
    int top_dtype, dh_dtype;
    int64_t table_rows;
    const int32_t* labels;
    const float* weight;
    float temperature, alpha, grad_scale;
    float* loss;
    char* dh;
    int64_t dh_stride;
};

__device__ __forceinline__ float value_at(const char* p, int type, int64_t i) {
    if (type == FG_F32) return ((const float*)p)[i];
    const unsigned short v = ((const unsigned short*)p)[i];
    return type == FG_BF16 ? __uint_as_float((unsigned int)v << 16) : (float)__builtin_bit_cast(_Float16, v);
}
__device__ __forceinline__ void put_value(char* p, int type, int64_t i, float f) {
    if (type == FG_F32)
        ((float*)p)[i] = f;
    else if (type == FG_BF16)
        ((__bf16*)p)[i] = (__bf16)f;
    else
        ((_Float16*)p)[i] = (_Float16)f;
}

// what the lanes of a row have written to LDS or memory is there for all of them
template <int WAVES>
__device__ __forceinline__ void row_meets() {
    if constexpr (WAVES > 1) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    }
}

struct Entry {
    int32_t c;      // class, -1: none
    float p, log_p, z;
};

// WAVES > 1: that many wavefronts to a row, else 64 / lanes rows to a wavefront. NP pieces of eight columns a lane in registers; TAIL: there are more
template <int T, int WAVES, int NP, bool TAIL>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : DL_THREADS) void distill_kernel(DistillArgs A) {
    constexpr int E = T == FG_F32 ? 4 : 2;
    extern __shared__ __attribute__((aligned(16))) char dl_lds[];
    __shared__ double red[WAVES];
    __shared__ int taught_by[1];
    const int64_t count = row_count(A.L);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows_per_wave = WAVES > 1 ? 1 : 64 / A.lanes;
    const int me = WAVES > 1 ? (int)threadIdx.x : lane & (A.lanes - 1);
    const int width = WAVES > 1 ? WAVES * 64 : A.lanes, few = width < 64 ? width : 64;      // lanes that the entries are spread over
    const int slot = WAVES > 1 ? 0 : wave * rows_per_wave + lane / A.lanes;
    const int64_t at = WAVES > 1 ? blockIdx.x : blockIdx.x * (int64_t)(DL_THREADS / A.lanes) + slot;
    const int64_t r = row_at(A.L, A.L.first + at, count);
    if (WAVES > 1 && r < 0) return;      // the whole workgroup
    Entry* const entries = (Entry*)dl_lds + slot * A.k;
    const char* const row = A.h + r * A.h_stride;

    float v[NP][8];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (me + width * i) * 8, left = r >= 0 ? A.d - c : 0;
        if (left > 0) fg_piece_values<T>(fg_load_piece<T>(row + (int64_t)c * E, left), v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= left) v[i][e] = -INFINITY;
    }
    // the row's node, label and weight; the teacher's distribution over its entries
    int64_t node = -1;
    int32_t y = -1;
    float weight = 1.f;
    if (r >= 0) {
        if (A.alpha > 0.f) node = A.ids ? A.ids[r] : r;
        if (node >= A.table_rows) node = -1;
        if (A.labels && A.alpha < 1.f) y = A.labels[r];
        if (y >= A.d) y = -1;
        if (A.weight) weight = A.weight[r];
    }
    bool taught = false;
    float t_max = -INFINITY;
    double t_sum = 0.0;
    if (me < few) {
        for (int j = me; j < A.k; j += few) {
            int32_t c = node >= 0 ? A.top_idx[node * A.k + j] : -1;
            float t = -INFINITY;
            if (c < 0 || c >= A.d) c = -1;
            if (c >= 0) t = value_at(A.top_val, A.top_dtype, node * A.k + j) / A.temperature;
            if (!(t == -INFINITY)) taught = true;
            t_max = fmaxf(t_max, t);
            entries[j] = Entry{c, 0.f, t, c >= 0 ? value_at(row, T, c) : 0.f};
        }
        t_max = lanes_max(t_max, few);
        taught = lanes_max(taught ? 1.f : 0.f, few) > 0.f;
        for (int j = me; j < A.k; j += few)
            if (entries[j].c >= 0) t_sum += (double)expf(entries[j].log_p - t_max);
        t_sum = lanes_sum(t_sum, few);
        const float log_sum = logf((float)t_sum);
        for (int j = me; j < A.k; j += few)
            if (entries[j].c >= 0) {
                const float log_p = entries[j].log_p - t_max - log_sum;
                entries[j].p = taught ? expf(log_p) : 0.f;
                entries[j].log_p = log_p;
            }
        if (WAVES > 1 && me == 0) taught_by[0] = taught;
    }
    if constexpr (WAVES > 1) {
        __syncthreads();
        taught = taught_by[0];
    }

    // the student's softmaxes
    auto tail = [&](auto f) {      // the pieces that are not held
        if constexpr (TAIL)
            for (int c = (me + width * NP) * 8; c < A.d; c += width * 8) {
                float w[8];
                fg_piece_values<T>(fg_load_piece<T>(row + (int64_t)c * E, A.d - c), w);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e >= A.d - c) w[e] = -INFINITY;
                f(c, w);
            }
    };
    const float soften = LOG2E / A.temperature;
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, v[i][e]);
    tail([&](int, const float(&w)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, w[e]);
    });
    m = row_max<WAVES>(m, few, red);
    double hard = 0.0, soft = 0.0;
    auto add = [&](const float(&w)[8]) {
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (y >= 0) s += __builtin_amdgcn_exp2f((w[e] - m) * LOG2E);
            if (taught) t += __builtin_amdgcn_exp2f((w[e] - m) * soften);
        }
        hard += (double)s;
        soft += (double)t;
    };
#pragma unroll
    for (int i = 0; i < NP; ++i)
        if ((me + width * i) * 8 < A.d) add(v[i]);
    tail([&](int, const float(&w)[8]) { add(w); });
    hard = row_sum<WAVES>(hard, few, red);
    soft = row_sum<WAVES>(soft, few, red);

    const float T2 = A.temperature;
    if (A.loss) {
        double kl = 0.0;
        const float log_soft = logf((float)soft);
        if (me < few && taught) {
            for (int j = me; j < A.k; j += few)
                if (!(entries[j].p == 0.f)) kl += (double)(entries[j].p * (entries[j].log_p - ((entries[j].z - m) / T2 - log_soft)));
        }
        if (wave == 0 || WAVES == 1) kl = lanes_sum(kl, few);
        if (me == 0 && r >= 0) {
            float loss = 0.f;
            if (taught) loss += A.alpha * T2 * T2 * (float)kl;
            if (y >= 0) loss += (1.f - A.alpha) * (logf((float)hard) - (value_at(row, T, y) - m));
            A.loss[r] = taught || y >= 0 ? weight * loss : 0.f;
        }
    }
    if (!A.dh) return;
    const float scale = A.grad_scale * weight;
    const float a = scale * A.alpha * T2, b = scale * (1.f - A.alpha);
    const float a_q = a / (float)soft, b_q = b / (float)hard;
    auto gradient = [&](float z) {
        float g = 0.f;
        if (taught) g += a_q * __builtin_amdgcn_exp2f((z - m) * soften);
        if (y >= 0) g += b_q * __builtin_amdgcn_exp2f((z - m) * LOG2E);
        return g;
    };
    // the entries' own values, the label's (by the first lane, unless an entry is of its class)
    float at_label = 0.f;
    bool by_entry = false;
    row_meets<WAVES>();      // (the entries are all there)
    if (me < few) {
        for (int j = me; j < A.k; j += few) {
            const int32_t c = entries[j].c;
            if (c < 0) continue;
            float share = 0.f;
            for (int i = 0; i < A.k; ++i)
                if (entries[i].c == c) share += entries[i].p;
            float g = gradient(entries[j].z) - (c == y ? b : 0.f);
            if (taught) g -= a * share;
            entries[j].log_p = g;      // (read by this lane alone)
        }
        if (me == 0 && y >= 0) {
            for (int i = 0; i < A.k; ++i) by_entry |= entries[i].c == y;
            if (!by_entry) at_label = gradient(value_at(row, T, y)) - b;
        }
    }
    row_meets<WAVES>();      // (dh may be h: its values have been read)
    char* const out = A.dh + r * A.dh_stride;
    auto write = [&](int c, const float(&w)[8]) {
        float g[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = gradient(w[e]);
        if (A.dh_dtype == FG_F32)
            fg_store_piece<FG_F32>(out + (int64_t)c * 4, g, A.d - c);
        else if constexpr (T != FG_F32)
            fg_store_piece<T>(out + (int64_t)c * 2, g, A.d - c);
    };
    if (r >= 0) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (me + width * i) * 8;
            if (c < A.d) write(c, v[i]);
        }
        tail([&](int c, const float(&w)[8]) { write(c, w); });
    }
    row_meets<WAVES>();      // (the entries' values go over these)
    if (r >= 0 && me < few) {
        for (int j = me; j < A.k; j += few)
            if (entries[j].c >= 0) put_value(out, A.dh_dtype, entries[j].c, entries[j].log_p);
        if (me == 0 && y >= 0 && !by_entry) put_value(out, A.dh_dtype, y, at_label);
    }
}

template <int T, int WAVES, int NP, bool TAIL>
void launch(DistillArgs A, hipStream_t st) {
    const int per_block = WAVES > 1 ? 1 : DL_THREADS / A.lanes;
    const int64_t at_once = (FG_MAX_GRID / 4 - 1) * per_block;      // rows of a launch
    for (; A.L.first < A.L.max_rows; A.L.first += at_once) {
        const int64_t rows = A.L.max_rows - A.L.first < at_once ? A.L.max_rows - A.L.first : at_once;
        hipLaunchKernelGGL((distill_kernel<T, WAVES, NP, TAIL>), dim3((unsigned)fg_ceil_div(rows, per_block)), dim3(WAVES > 1 ? WAVES * 64 : DL_THREADS),
                           (size_t)per_block * A.k * sizeof(Entry), st, A);
    }
}
template <int T>
void distill(DistillArgs A, hipStream_t st) {
    const int pieces = (int)fg_ceil_div(A.d, 8);
    A.lanes = 64;
    if (pieces <= 64) {
        A.lanes = DL_MIN_LANES;
        while (A.lanes < pieces) A.lanes *= 2;
        launch<T, 1, 1, false>(A, st);
    } else if (pieces <= 128) {
        launch<T, 1, 2, false>(A, st);
    } else if (pieces <= 256) {
        launch<T, 1, 4, false>(A, st);
    } else if (pieces <= 1024) {
        launch<T, 4, 4, false>(A, st);
    } else if (pieces <= 2048) {
        launch<T, 8, 4, false>(A, st);
    } else if (pieces <= 8192) {
        launch<T, 16, 8, false>(A, st);
    } else {
        launch<T, 16, 8, true>(A, st);
    }
}

}  // namespace

extern "C" fg_status_t fg_distill_loss(const void* h, int64_t h_stride, fg_dtype_t dtype, const int32_t* rows_dev, const int64_t* n_rows_dev, int64_t max_rows,
                                       int64_t n, int32_t d, const int32_t* ids_dev, const int32_t* top_idx_dev, const void* top_val_dev, fg_dtype_t top_dtype,
                                       int64_t table_rows, int32_t k, const int32_t* labels_dev, float temperature, float alpha, const float* weight_dev,
                                       float grad_scale, float* loss_out, void* dh, int64_t dh_stride, fg_dtype_t dh_dtype, void* stream) {
    const char* who = "fg_distill_loss";
    const int e = fg_dtype_size(dtype);
    if (!e || (k != 0 && !fg_dtype_size(top_dtype))) FG_FAIL(FG_ERR_DTYPE, "%s: unknown element type", who);
    if (dh && dh_dtype != dtype && dh_dtype != FG_F32) FG_FAIL(FG_ERR_DTYPE, "%s: dh is of the type of h or fp32", who);
    FG_TRY(check_rows(who, rows_dev, n_rows_dev, max_rows, n, d));
    if (k < 0 || k > FG_MAX_TOP) FG_FAIL(FG_ERR_SHAPE, "%s: k = %d is not in 0..%d", who, k, FG_MAX_TOP);
    if (table_rows < 0 || table_rows > INT32_MAX) FG_FAIL(FG_ERR_INVALID_ARG, "%s: a number of rows is negative or too large", who);
    if (!(temperature > 0.f && temperature < INFINITY)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: temperature = %g must be positive", who, (double)temperature);
    if (!(alpha >= 0.f && alpha <= 1.f)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: alpha = %g is not in [0, 1]", who, (double)alpha);
    if (!loss_out && !dh) FG_FAIL(FG_ERR_INVALID_ARG, "%s: neither loss nor gradient is wanted", who);
    const bool work = max_rows > 0 && n > 0;
    if (work && !h) FG_FAIL(FG_ERR_INVALID_ARG, "%s: h must not be NULL", who);
    if (work && k > 0 && table_rows > 0 && (!top_idx_dev || !top_val_dev)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: the teacher's classes and values must not be NULL", who);
    FG_TRY(check_array(who, "h", h, h_stride, e, d));
    if (dh) FG_TRY(check_array(who, "dh", dh, dh_stride, fg_dtype_size(dh_dtype), d));
    if (dh == h && dh && (dh_dtype != dtype || dh_stride != h_stride)) FG_FAIL(FG_ERR_INVALID_ARG, "%s: dh over h has its type and stride", who);
    if (((uintptr_t)ids_dev | (uintptr_t)top_idx_dev | (uintptr_t)labels_dev | (uintptr_t)weight_dev | (uintptr_t)loss_out) & 3 ||
        (k > 0 && ((uintptr_t)top_val_dev & (uintptr_t)(fg_dtype_size(top_dtype) - 1))))
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: ids, classes, values, labels, weight and loss must be aligned to their elements", who);
    fg_clear_error();
    if (!work) return FG_OK;
    const DistillArgs A = {{rows_dev, n_rows_dev, max_rows, n, 0}, (const char*)h, h_stride, d, 0, table_rows > 0 ? k : 0, ids_dev, top_idx_dev, (const char*)top_val_dev,
                           (int)top_dtype, (int)dh_dtype, table_rows, labels_dev, weight_dev, temperature, alpha, grad_scale, loss_out, (char*)dh, dh_stride};
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == FG_F32)
        distill<FG_F32>(A, st);
    else if (dtype == FG_F16)
        distill<FG_F16>(A, st);
    else
        distill<FG_BF16>(A, st);
    FG_LAUNCH_CHECK("distill_kernel");
    return FG_OK;
}

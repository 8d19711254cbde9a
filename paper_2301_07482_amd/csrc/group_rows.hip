// fg_group_rows: the listed rows of a layer sorted by their group, stably, for the products that take a weight matrix per group.
//
// A counting sort. A workgroup takes a run of the list, each of its wavefronts a run of that, 64 rows at a time: the lanes with the
// same group find each other with one ballot per bit of the group, a lane's rank is the number of those before it plus what the
// wavefront has counted so far (LDS, one row of counters per wavefront: no atomics, so the order is the list's). Two scans, over the
// wavefronts and over the groups, turn the counts into places. Up to ONE_ROWS rows are one workgroup and one launch; else the first
// launch leaves every workgroup's counts and every row's group and rank, and in the second each workgroup adds up the counts of those before it.
// What it costs is latency, three or four reads that depend on each other to a launch: 256 rows 3.9 us, 54067 rows 5.1 + 6.5, 368640 rows
// 13 + 9.5 (their 12 bytes a row read and 8 written would take 1.5 us). One launch against two, us, 4 groups: 256 rows 4.2 | 6.4, 4000 5.8 | 7.4, 6000
// 6.8 | 7.6, 8192 8.0 | 7.7; 100 groups: 4000 7.4 | 9.2, 6000 9.4 | 9.3, 8192 11.4 | 9.9.
#include "common.h"
#include "scan.h"

namespace {

constexpr int GR_THREADS = 1024, GR_WAVES = GR_THREADS / 64;
constexpr int GR_AHEAD = 6;                          // rows of a lane whose reads (list, id, group) are in flight together
constexpr int64_t ONE_ROWS = GR_THREADS * GR_AHEAD;
constexpr int64_t GR_MAX_BLOCKS = 512;               // a workgroup reads the counts of all of them
constexpr int GR_RANK_BITS = 22;                     // of a row within its wavefront's run; the 10 bits above hold the group
static_assert(FG_MAX_GROUPS <= 1 << (32 - GR_RANK_BITS), "group and rank fit a word");
constexpr uint32_t GR_NONE = 0xFFFFFFFFu;            // (no row has that rank: a wavefront's run has 2^18 rows at most)

struct GrArgs {
    const int32_t *groups, *ids, *rows;
    int64_t n_table, n_positions, max_rows;
    const int64_t* n_rows_dev;
    int n_groups, bits;
    int32_t* order;
    int64_t* offsets;
    uint32_t* key;      // [max_rows] group and rank within the wavefront's run
    int32_t* counts;    // [workgroups][1 + wavefronts][n_groups]: totals, and the first rank of each wavefront
    int64_t per_wave;   // rows of a wavefront's run, a multiple of 64
};

__device__ __forceinline__ int64_t gr_count(const GrArgs& A) {
    const int64_t n = A.n_rows_dev ? *A.n_rows_dev : A.max_rows;
    return n < 0 ? 0 : (n > A.max_rows ? A.max_rows : n);
}

// positions and groups of rows k0, k0 + 64, ... (-1: none); every read of a stage is issued before the next stage's
template <int N>
__device__ __forceinline__ void gr_read(const GrArgs& A, int64_t k0, int64_t end, int32_t (&r)[N], int32_t (&g)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t k = k0 + 64 * i;
        r[i] = k < end ? (A.rows ? A.rows[k] : (int32_t)k) : -1;
        if (r[i] < 0 || r[i] >= A.n_positions) r[i] = -1;
    }
    int32_t v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = r[i] < 0 ? -1 : (A.ids ? A.ids[r[i]] : r[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        g[i] = v[i] >= 0 && v[i] < A.n_table ? A.groups[v[i]] : -1;
        if (g[i] < 0 || g[i] >= A.n_groups) g[i] = -1;
    }
}

// rank of this lane's row among the wavefront's rows of its group so far; counts it (all lanes active)
__device__ __forceinline__ int32_t gr_rank(int32_t g, int bits, volatile int32_t* count) {
    unsigned long long same = __ballot(g >= 0);
    for (int b = 0; b < bits; ++b) {
        const bool one = (g >> b) & 1;
        const unsigned long long with = __ballot(one);
        same &= one ? with : ~with;
    }
    if (g < 0) return 0;
    const int before = __popcll(same & ((1ull << fg_lane()) - 1ull));
    const int32_t base = count[g];
    if (before == 0) count[g] = base + __popcll(same);      // behind every lane's read: a wavefront's LDS operations keep their order
    return base + before;
}

// LDS: a row of counters per wavefront. Turns them into the wavefronts' first ranks within the group; thread g gets the group's total.
__device__ __forceinline__ int32_t gr_scan_waves(int32_t* cnt, int n_groups) {
    __syncthreads();
    int32_t total = 0;
    if ((int)threadIdx.x < n_groups)
        for (int w = 0; w < GR_WAVES; ++w) {
            const int32_t c = cnt[w * n_groups + threadIdx.x];
            cnt[w * n_groups + threadIdx.x] = total;
            total += c;
        }
    return total;
}

// sum of the values of the threads before this one (values below 2^31 in total)
__device__ __forceinline__ int32_t gr_scan_groups(int32_t v, int* totals) {
    const int incl = fg_wave_scan(v);
    __syncthreads();
    if (fg_lane() == 63) totals[fg_wave()] = incl;
    __syncthreads();
    int before, all;
    fg_wave_totals<GR_WAVES>(totals, before, all);
    return before + incl - v;
}

__global__ __launch_bounds__(GR_THREADS) void group_rows_one_kernel(GrArgs A) {
    extern __shared__ __attribute__((aligned(16))) int32_t gr_lds[];      // counters [wavefronts][groups], then the groups' first places
    __shared__ __attribute__((aligned(16))) int totals[GR_WAVES];
    int32_t *cnt = gr_lds, *first = gr_lds + GR_WAVES * A.n_groups;
    const int64_t n = gr_count(A);
    for (int i = threadIdx.x; i < GR_WAVES * A.n_groups; i += GR_THREADS) cnt[i] = 0;
    const int64_t k0 = fg_wave() * A.per_wave + fg_lane();
    int64_t end = (fg_wave() + 1) * A.per_wave;
    if (end > n) end = n;
    int32_t r[GR_AHEAD], g[GR_AHEAD], rank[GR_AHEAD];
    gr_read(A, k0, end, r, g);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < GR_AHEAD; ++i)
        if (64 * i < A.per_wave) rank[i] = gr_rank(g[i], A.bits, cnt + fg_wave() * A.n_groups);
    const int32_t total = gr_scan_waves(cnt, A.n_groups);
    const int32_t place = gr_scan_groups(total, totals);
    if ((int)threadIdx.x < A.n_groups) {
        first[threadIdx.x] = place;
        A.offsets[threadIdx.x] = place;
        if ((int)threadIdx.x == A.n_groups - 1) A.offsets[A.n_groups] = place + total;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < GR_AHEAD; ++i)
        if (64 * i < A.per_wave && g[i] >= 0) A.order[first[g[i]] + cnt[fg_wave() * A.n_groups + g[i]] + rank[i]] = r[i];
}

// first launch: groups and ranks of this workgroup's run, and its counts
__global__ __launch_bounds__(GR_THREADS) void group_rows_count_kernel(GrArgs A) {
    extern __shared__ __attribute__((aligned(16))) int32_t gr_lds[];
    int32_t* cnt = gr_lds;
    const int64_t n = gr_count(A);
    for (int i = threadIdx.x; i < GR_WAVES * A.n_groups; i += GR_THREADS) cnt[i] = 0;
    __syncthreads();
    const int64_t k0 = (blockIdx.x * (int64_t)GR_WAVES + fg_wave()) * A.per_wave + fg_lane();
    int64_t end = k0 - fg_lane() + A.per_wave;
    if (end > n) end = n;
    int32_t* mine = cnt + fg_wave() * A.n_groups;
    constexpr int N = 4;
    for (int64_t k = k0; k - fg_lane() < end; k += 64 * N) {      // uniform over the wavefront
        int32_t r[N], g[N];
        gr_read(A, k, end, r, g);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int32_t rank = gr_rank(g[i], A.bits, mine);
            if (k + 64 * i < end) A.key[k + 64 * i] = g[i] < 0 ? GR_NONE : ((uint32_t)g[i] << GR_RANK_BITS) | (uint32_t)rank;
        }
    }
    const int32_t total = gr_scan_waves(cnt, A.n_groups);
    if ((int)threadIdx.x < A.n_groups) A.counts[blockIdx.x * (int64_t)(GR_WAVES + 1) * A.n_groups + threadIdx.x] = total;
    __syncthreads();
    for (int i = threadIdx.x; i < GR_WAVES * A.n_groups; i += GR_THREADS) A.counts[(blockIdx.x * (int64_t)(GR_WAVES + 1) + 1) * A.n_groups + i] = cnt[i];
}

__global__ __launch_bounds__(GR_THREADS) void group_rows_place_kernel(GrArgs A) {
    extern __shared__ __attribute__((aligned(16))) int32_t gr_lds[];      // first places [wavefronts][groups]
    __shared__ __attribute__((aligned(16))) int totals[GR_WAVES];
    const int64_t n = gr_count(A);
    const int64_t step = (int64_t)(GR_WAVES + 1) * A.n_groups;
    // counts of the workgroups before this one and of all, a thread per group
    int32_t before = 0, total = 0;
    if ((int)threadIdx.x < A.n_groups)
#pragma unroll 8
        for (int b = 0; b < (int)gridDim.x; ++b) {
            const int32_t c = A.counts[b * step + threadIdx.x];
            before += b < (int)blockIdx.x ? c : 0;
            total += c;
        }
    const int32_t place = gr_scan_groups(total, totals);
    if ((int)threadIdx.x < A.n_groups) {
        for (int w = 0; w < GR_WAVES; ++w)
            gr_lds[w * A.n_groups + threadIdx.x] = place + before + A.counts[blockIdx.x * step + (w + 1) * A.n_groups + threadIdx.x];
        if (blockIdx.x == 0) {
            A.offsets[threadIdx.x] = place;
            if ((int)threadIdx.x == A.n_groups - 1) A.offsets[A.n_groups] = place + total;
        }
    }
    __syncthreads();
    const int64_t k0 = (blockIdx.x * (int64_t)GR_WAVES + fg_wave()) * A.per_wave + fg_lane();
    int64_t end = k0 - fg_lane() + A.per_wave;
    if (end > n) end = n;
    const int32_t* first = gr_lds + fg_wave() * A.n_groups;
#pragma unroll 4
    for (int64_t k = k0; k < end; k += 64) {
        const uint32_t key = A.key[k];
        const int32_t r = A.rows ? A.rows[k] : (int32_t)k;
        if (key != GR_NONE) A.order[first[key >> GR_RANK_BITS] + (int32_t)(key & ((1u << GR_RANK_BITS) - 1))] = r;
    }
}

// workgroups of a call, and rows of a wavefront
void gr_shape(int64_t max_rows, int64_t& blocks, int64_t& per_wave) {
    if (max_rows <= ONE_ROWS) {
        blocks = 1;
        per_wave = fg_ceil_div(max_rows, GR_THREADS) * 64;
        return;
    }
    blocks = fg_ceil_div(max_rows, 4 * GR_THREADS);
    if (blocks > GR_MAX_BLOCKS) blocks = GR_MAX_BLOCKS;
    per_wave = fg_ceil_div(fg_ceil_div(max_rows, blocks), GR_THREADS) * 64;
    blocks = fg_ceil_div(max_rows, per_wave * GR_WAVES);
}

}  // namespace

extern "C" size_t fg_group_rows_workspace_bytes(int64_t max_rows, int32_t n_groups) {
    if (max_rows < 0 || max_rows > INT32_MAX || n_groups < 1 || n_groups > FG_MAX_GROUPS) return 0;
    // the bound on the workgroups of any smaller call: a workspace for max_rows serves fewer rows too
    const int64_t blocks = fg_ceil_div(max_rows, 4 * GR_THREADS) + 1;
    return fg_align_up((size_t)max_rows * 4, 16) + (size_t)(blocks < GR_MAX_BLOCKS ? blocks : GR_MAX_BLOCKS) * (GR_WAVES + 1) * n_groups * 4 + 16;
}

extern "C" fg_status_t fg_group_rows(const int32_t* groups_dev, int64_t n_table, const int32_t* ids_dev, int64_t n_positions, const int32_t* rows_dev,
                                     const int64_t* n_rows_dev, int64_t max_rows, int32_t n_groups, int32_t* order_dev, int64_t* offsets_dev,
                                     void* ws_dev, size_t ws_bytes, void* stream) {
    if (max_rows < 0 || max_rows > INT32_MAX || n_table < 0 || n_positions < 0) FG_FAIL(FG_ERR_INVALID_ARG, "fg_group_rows: a size is negative or too large");
    if (n_groups < 1 || n_groups > FG_MAX_GROUPS) FG_FAIL(FG_ERR_INVALID_ARG, "fg_group_rows: n_groups = %d is not in 1..%d", n_groups, FG_MAX_GROUPS);
    if (!offsets_dev || (max_rows > 0 && (!groups_dev || !order_dev || !ws_dev)))
        FG_FAIL(FG_ERR_INVALID_ARG, "fg_group_rows: groups, order, offsets and the workspace must not be NULL");
    if (((uintptr_t)groups_dev | (uintptr_t)ids_dev | (uintptr_t)rows_dev | (uintptr_t)order_dev) & 3 || ((uintptr_t)offsets_dev | (uintptr_t)n_rows_dev) & 7 ||
        ((uintptr_t)ws_dev & 15))
        FG_FAIL(FG_ERR_INVALID_ARG, "fg_group_rows: an array is not aligned to its element, or the workspace not to 16 bytes");
    if (ws_bytes < (max_rows > 0 ? fg_group_rows_workspace_bytes(max_rows, n_groups) : 0))
        FG_FAIL(FG_ERR_SHAPE, "fg_group_rows: workspace of %zu bytes, %zu are needed", ws_bytes, fg_group_rows_workspace_bytes(max_rows, n_groups));
    fg_clear_error();
    int bits = 0;
    while (1 << bits < n_groups) ++bits;
    int64_t blocks, per_wave;
    gr_shape(max_rows, blocks, per_wave);
    GrArgs A = {groups_dev, ids_dev, rows_dev, n_table, n_positions, max_rows, n_rows_dev, n_groups, bits, order_dev, offsets_dev,
                (uint32_t*)ws_dev, (int32_t*)((char*)ws_dev + fg_align_up((size_t)max_rows * 4, 16)), per_wave};
    hipStream_t st = (hipStream_t)stream;
    if (max_rows <= ONE_ROWS) {
        hipLaunchKernelGGL(group_rows_one_kernel, dim3(1), dim3(GR_THREADS), (GR_WAVES + 1) * n_groups * 4, st, A);
        FG_LAUNCH_CHECK("group_rows_one_kernel");
        return FG_OK;
    }
    hipLaunchKernelGGL(group_rows_count_kernel, dim3((unsigned)blocks), dim3(GR_THREADS), GR_WAVES * n_groups * 4, st, A);
    FG_LAUNCH_CHECK("group_rows_count_kernel");
    hipLaunchKernelGGL(group_rows_place_kernel, dim3((unsigned)blocks), dim3(GR_THREADS), GR_WAVES * n_groups * 4, st, A);
    FG_LAUNCH_CHECK("group_rows_place_kernel");
    return FG_OK;
}

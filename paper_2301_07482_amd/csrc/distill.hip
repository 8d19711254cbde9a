// fg_distill_loss: a student's loss against a teacher's stored top logits and against labels, with its gradient.
//
// A row of logits is read once and its gradient written once; both softmaxes of it (at the temperature and as it is) come from the values held in
// registers, as they lie in memory. Rows of up to DL_NARROW columns share a wavefront, eight columns to a lane; wider ones belong to one wavefront or to several, and
// what does not fit their registers is read again. Where the temperature is 1, 2 or 4, the exponentials as the row is are those at the temperature squared (that doubles their
// relative error each time, as a temperature does the other way): exponentials take four times as long as other instructions, and two of them a value for each softmax are
// what a wide row spends its time on beside memory. The k classes that the teacher has stored, and the label, take their shares from the gradient while it
// is in registers, in the entries' order, so that a class that is stored twice takes both.
#include <type_traits>

#include "row_list.h"
#include "row_types.h"

namespace {

constexpr int DL_THREADS = 256, DL_NARROW = 512, DL_FEW_ROWS = 16384;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;

struct DistillArgs {
    RowList L;
    const char* h;
    int64_t h_stride;
    int d, k;
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

// the largest of three, those that are NaN left out (the library's fmaxf makes its operands quiet first)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}
// over LANES adjacent lanes, all lanes active, the same in all of them: neighbours, pairs, halves of eight and of sixteen lanes change places inside the vector registers
template <int LANES, typename F>
__device__ __forceinline__ float over_lanes(float v, const F& f) {
    const auto moved = [&](auto ctrl) { return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, false)); };
    v = f(v, moved(std::integral_constant<int, 0xB1>()));
    v = f(v, moved(std::integral_constant<int, 0x4E>()));
    v = f(v, moved(std::integral_constant<int, 0x141>()));
    if constexpr (LANES >= 16) v = f(v, moved(std::integral_constant<int, 0x140>()));
    if constexpr (LANES >= 32) v = f(v, __shfl_xor(v, 16, 64));
    if constexpr (LANES >= 64) v = f(v, __shfl_xor(v, 32, 64));
    return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum_of(float v) {
    return over_lanes<LANES>(v, [](float a, float b) { return a + b; });
}
template <int LANES>
__device__ __forceinline__ float lanes_max_of(float v) {
    return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
// over a wavefront, all lanes active, the same in all of them. The lanes' values move inside the vector registers, as in fg_wave_scan
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float v, float none) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63)); }
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0x111, 0xf>(v, 0.f);
    v += moved<0x112, 0xf>(v, 0.f);
    v += moved<0x114, 0xf>(v, 0.f);
    v += moved<0x118, 0xf>(v, 0.f);
    v += moved<0x142, 0xa>(v, 0.f);
    v += moved<0x143, 0xc>(v, 0.f);
    return last_lane(v);
}
// of two values at once: halves of the wavefront exchange them first
__device__ __forceinline__ void wave_sums(double& a, double& b) {
    double v = half_sums<32>(a, b);
    const auto moved = [&](auto ctrl) {
        const fg_u32x2 w = __builtin_bit_cast(fg_u32x2, v);
        return __builtin_bit_cast(double, fg_u32x2{(unsigned int)__builtin_amdgcn_mov_dpp((int)w[0], decltype(ctrl)::value, 0xf, 0xf, false),
                                                   (unsigned int)__builtin_amdgcn_mov_dpp((int)w[1], decltype(ctrl)::value, 0xf, 0xf, false)});
    };
    v += moved(std::integral_constant<int, 0xB1>());
    v += moved(std::integral_constant<int, 0x4E>());
    v += moved(std::integral_constant<int, 0x141>());
    v += moved(std::integral_constant<int, 0x140>());
    v = half_sums<16>(v, v);
    const fg_u32x2 w = __builtin_bit_cast(fg_u32x2, v);
    const auto of = [&](int lane) {
        return __builtin_bit_cast(double, fg_u32x2{(unsigned int)__builtin_amdgcn_readlane((int)w[0], lane), (unsigned int)__builtin_amdgcn_readlane((int)w[1], lane)});
    };
    a = of(0), b = of(32);
}
__device__ __forceinline__ float wave_max(float v) {      // (what is NaN is left out)
    v = fmaxf(v, moved<0x111, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x112, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x114, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x118, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x142, 0xa>(v, -INFINITY));
    v = fmaxf(v, moved<0x143, 0xc>(v, -INFINITY));
    return last_lane(v);
}
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ float one(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }      // of a value that is the same in all lanes

// How the exponentials as the row is come from those at the temperature: squared SQUARES times, or (-1) by themselves
template <typename F>
__device__ __forceinline__ void with_squares(float temperature, const F& f) {
    if (temperature == 1.f)
        f(std::integral_constant<int, 0>());
    else if (temperature == 2.f)
        f(std::integral_constant<int, 1>());
    else if (temperature == 4.f)
        f(std::integral_constant<int, 2>());
    else
        f(std::integral_constant<int, -1>());
}
// e^((z - m) / temperature), e^(z - m)
template <int SQUARES>
__device__ __forceinline__ void both(float z, float m, float soften, float& soft, float& hard) {
    soft = exp2_of((z - m) * soften);
    hard = SQUARES < 0 ? exp2_of((z - m) * LOG2E) : SQUARES == 0 ? soft : soft * soft;
    if (SQUARES == 2) hard *= hard;
}
// sums of both over eight values
__device__ __forceinline__ void sums_of(float temperature, const float (&w)[8], float m, float soften, float& soft, float& hard) {
    soft = hard = 0.f;
    with_squares(temperature, [&](auto squares) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float s, h;
            both<decltype(squares)::value>(w[e], m, soften, s, h);
            soft += s, hard += h;
        }
    });
}
// a * soft + b * hard of eight values
__device__ __forceinline__ void gradients_of(float temperature, const float (&w)[8], float m, float soften, float a, float b, float (&g)[8]) {
    with_squares(temperature, [&](auto squares) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float s, h;
            both<decltype(squares)::value>(w[e], m, soften, s, h);
            g[e] = a * s + b * h;
        }
    });
}
__device__ __forceinline__ void no_value_beyond(int left, float (&w)[8]) {
    if (left < 8)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= left) w[e] = -INFINITY;
}
// node, label (-1: none) and weight of a row
__device__ __forceinline__ void row_facts(const DistillArgs& A, int64_t r, int32_t& node, int32_t& y, float& weight) {
    node = -1, y = -1, weight = 1.f;
    if (r < 0) return;
    if (A.alpha > 0.f && A.k > 0) node = A.ids ? A.ids[r] : (int32_t)r;
    if (A.labels && A.alpha < 1.f) y = A.labels[r];
    if (A.weight) weight = A.weight[r];
    if (node >= A.table_rows) node = -1;
    if (y >= A.d || y < 0) y = -1;
}
// entry j of a node: its class (-1: none) and its value
__device__ __forceinline__ void entry_of(const DistillArgs& A, int32_t node, int j, int32_t& c, float& t) {
    c = -1, t = -INFINITY;
    if (node < 0) return;
    const int64_t at = (int64_t)node * A.k + j;
    c = A.top_idx[at];
    t = fg_element(A.top_val, A.top_dtype, at);
    if (c < 0 || c >= A.d) c = -1, t = -INFINITY;
}

// what the lanes of a wavefront have written to LDS is there for all of them
__device__ __forceinline__ void wave_meets() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// all[at] = a wavefront's shares (at < 0: none), of zeros. Every lane leaves its number at its place; who finds another's marks the place as shared, and the shares of such a
// place are added one after the other, in the lanes' order. (Nearly always no place is: a teacher's classes differ.)
constexpr float SHARED = -1.f;
__device__ __forceinline__ void share_out(float* all, int at, float share, int lane) {
    if (at >= 0) all[at] = (float)lane;
    wave_meets();
    const bool other = at >= 0 && all[at] != (float)lane;
    const bool any = __ballot(other) != 0;
    wave_meets();
    if (any) {
        if (other) all[at] = SHARED;
        wave_meets();
        const bool shared = at >= 0 && all[at] == SHARED;
        wave_meets();
        if (shared) all[at] = 0.f;
        wave_meets();
        for (unsigned long long left = __ballot(shared); left; left &= left - 1) {
            const int l = __ffsll((long long)left) - 1, place = __builtin_amdgcn_readlane(at, l);
            const float v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(share), l));
            if (lane == 0) all[place] += v;
        }
        if (shared) at = -1;
    }
    if (at >= 0) all[at] = share;
    wave_meets();
}

// Narrow rows: 64 / LANES of them to a wavefront, eight columns to a lane. A row's values lie in LDS for its entries to find theirs, then what those take from its
// gradient. Bound by memory and, nearly as long, by what a wavefront does beside its values: 54067 x 256 fp32 24 us (4.6 TB/s; without teacher and labels 17; bf16 21, 54067 x 512 bf16 37), 32 with the
// lanes a number of the call's; two and four pieces a lane, for more rows to a wavefront, 28 and 30.
struct Entry {
    int32_t c;      // class, -1: none
    float p, log2_p, z;      // p: its share of the gradient; z: its logit, then whether its class is another's too
};
template <int T, int LANES>
__global__ __launch_bounds__(DL_THREADS) void distill_narrow_kernel(DistillArgs A) {
    constexpr int E = T == FG_F32 ? 4 : 2, ROW = LANES * 8, ROWS = DL_THREADS / LANES;
    extern __shared__ __attribute__((aligned(16))) char dl_lds[];
    __shared__ __attribute__((aligned(16))) float values[ROWS * ROW];
    const int me = (int)threadIdx.x % LANES, slot = (int)threadIdx.x / LANES;
    const int64_t r = row_at(A.L, A.L.first + blockIdx.x * (int64_t)ROWS + slot, row_count(A.L));
    Entry* const entries = (Entry*)dl_lds + slot * A.k;
    float* const all = values + slot * ROW;
    const char* const row = A.h + r * A.h_stride;
    const int c0 = me * 8, left = r >= 0 ? A.d - c0 : 0;
    float4* const mine = (float4*)(all + c0);      // this lane's columns
    fg_piece<T> raw = {};
    if (left > 0) raw = fg_load_piece<T>(row + (int64_t)c0 * E, left);
    int32_t node, y;
    float weight;
    row_facts(A, r, node, y, weight);
    // the teacher's entries are on their way beside the row
    float t_max = -INFINITY;
    for (int j = me; j < A.k; j += LANES) {
        int32_t c;
        float t;
        entry_of(A, node, j, c, t);
        entries[j].c = c, entries[j].log2_p = t;
        if (!(t == -INFINITY)) t_max = t > t_max || !(t == t) || t_max == -INFINITY ? t : t_max;
    }
    float w[8], m = -INFINITY;
    fg_piece_values<T>(raw, w);
    no_value_beyond(left, w);
    mine[0] = float4{w[0], w[1], w[2], w[3]}, mine[1] = float4{w[4], w[5], w[6], w[7]};
#pragma unroll
    for (int e = 0; e < 8; e += 2) m = max3(m, w[e], w[e + 1]);
    m = lanes_max_of<LANES>(m);
    wave_meets();
    // the teacher's distribution (a value that is NaN makes it NaN; without one above -infinity there is no teacher)
    const float soften = LOG2E / A.temperature;
    const float top = lanes_max_of<LANES>(t_max);
    const bool taught = lanes_max_of<LANES>(t_max == -INFINITY ? 0.f : 1.f) > 0.f;
    float t_sum = 0.f;
    for (int j = me; j < A.k; j += LANES) {
        const int32_t c = entries[j].c;
        const float x = (entries[j].log2_p - top) * soften;
        entries[j].log2_p = x;
        entries[j].z = c >= 0 ? all[c] : 0.f;
        if (c >= 0) t_sum += exp2_of(x);
    }
    const float z_label = y >= 0 ? all[y] : 0.f;
    const float t_log = log2_of(lanes_sum_of<LANES>(t_sum));
    // the student's
    float soft = 0.f, hard = 0.f;
    const bool either = taught || y >= 0;
    if (either) sums_of(A.temperature, w, m, soften, soft, hard);
    soft = lanes_sum_of<LANES>(soft);
    hard = lanes_sum_of<LANES>(hard);
    const float soft_log = log2_of(soft);
    const float scale = A.grad_scale * weight, a = taught ? scale * A.alpha * A.temperature : 0.f, b = y >= 0 ? scale * (1.f - A.alpha) : 0.f;
    float kl = 0.f;
    wave_meets();      // (the values have been read)
    mine[0] = mine[1] = float4{0.f, 0.f, 0.f, 0.f};
    wave_meets();
    if (taught)
        for (int j = me; j < A.k; j += LANES) {
            const int32_t c = entries[j].c;
            if (c < 0) continue;
            const float log2_p = entries[j].log2_p - t_log, p = exp2_of(log2_p);
            if (!(p == 0.f)) kl += p * (log2_p - ((entries[j].z - m) * soften - soft_log));
            entries[j].p = a * p;
            all[c] = (float)j;
        }
    if (A.loss) {
        kl = lanes_sum_of<LANES>(kl);
        if (me == 0 && r >= 0) {
            float loss = 0.f;
            if (taught) loss += A.alpha * A.temperature * A.temperature * LN2 * kl;
            if (y >= 0) loss += (1.f - A.alpha) * (LN2 * log2_of(hard) - (z_label - m));
            A.loss[r] = either ? weight * loss : 0.f;
        }
    }
    if (!A.dh) return;
    // as in share_out, with the entries' numbers (54067 x 256 fp32 with 64 entries: 30 us where all classes differ, 44 where most of a row's are stored twice; 38 with
    // atomic additions, whose order in one instruction nothing says)
    wave_meets();
    bool other = false;
    if (taught)
        for (int j = me; j < A.k; j += LANES)
            if (entries[j].c >= 0 && all[entries[j].c] != (float)j) other = true, entries[j].z = SHARED;
            else entries[j].z = 0.f;
    const bool any = __ballot(other) != 0;      // (in any row of the wavefront)
    wave_meets();
    if (any) {
        if (other)
            for (int j = me; j < A.k; j += LANES)
                if (entries[j].z == SHARED) all[entries[j].c] = SHARED;
        wave_meets();
        if (taught)
            for (int j = me; j < A.k; j += LANES)
                if (entries[j].c >= 0 && all[entries[j].c] == SHARED) entries[j].z = SHARED;
        wave_meets();
        if (taught)
            for (int j = me; j < A.k; j += LANES)
                if (entries[j].c >= 0 && entries[j].z == SHARED) all[entries[j].c] = 0.f;
        wave_meets();
        for (int j0 = 0; j0 < A.k; j0 += LANES) {
            const int j = j0 + me;
            unsigned long long left = __ballot(taught && j < A.k && entries[j].c >= 0 && entries[j].z == SHARED) >> ((threadIdx.x & 63) - me);
            if constexpr (LANES < 64) left &= (1ull << LANES) - 1;
            if (me == 0)
                for (; left; left &= left - 1) {
                    const Entry& shared = entries[j0 + __ffsll((long long)left) - 1];
                    all[shared.c] += shared.p;
                }
        }
    }
    if (taught)
        for (int j = me; j < A.k; j += LANES)
            if (entries[j].c >= 0 && entries[j].z != SHARED) all[entries[j].c] = entries[j].p;
    wave_meets();
    if (me == 0 && y >= 0) all[y] += b;
    wave_meets();
    if (left <= 0) return;
    float g[8] = {};
    if (either) gradients_of(A.temperature, w, m, soften, taught ? a / soft : 0.f, y >= 0 ? b / hard : 0.f, g);
    const float4 lo = mine[0], hi = mine[1];
    g[0] -= lo.x, g[1] -= lo.y, g[2] -= lo.z, g[3] -= lo.w, g[4] -= hi.x, g[5] -= hi.y, g[6] -= hi.z, g[7] -= hi.w;
    char* const out = A.dh + r * A.dh_stride;
    if (A.dh_dtype == FG_F32)
        fg_store_piece<FG_F32>(out + (int64_t)c0 * 4, g, left);
    else if constexpr (T != FG_F32)
        fg_store_piece<T>(out + (int64_t)c0 * 2, g, left);
}

// Wide rows: WAVES wavefronts to a row, one row to a workgroup. NP pieces of eight columns a lane in registers; TAIL: there are more. Pieces are counted from the 16-byte
// line that the row begins in, so that all but the first and the last of them are whole lines (rows of 50003 bf16 15 % faster). An entry is in a lane of every wavefront, which
// finds those of its own pieces. Sums are in fp64 from a lane's pieces on (exchanged between registers, both softmaxes' at once).
// Bound by memory: 8192 x 32000 bf16 253 us (4.1 TB/s), fp32 435 (4.8); rows that the registers do not hold are read twice: 4096 x 100000 bf16 496 us, 2048 x 200000 fp32 860.
// Four wavefronts to a SIMD: with five, 16-bit rows of several wavefronts had to spill registers (20000 x 16384 271 us, four 290; 4096 x 32000 154, four 139).
template <int T, int WAVES, int NP, bool TAIL>
__global__ __launch_bounds__(WAVES * 64, 4) void distill_wide_kernel(DistillArgs A) {
    constexpr int E = T == FG_F32 ? 4 : 2, WIDTH = WAVES * 64;
    __shared__ double red[2][WAVES];
    __shared__ float largest[WAVES];
    __shared__ int32_t top_class[WAVES > 1 ? 64 : 1];
    __shared__ float top_share[WAVES > 1 ? 64 : 1], teacher_log;
    constexpr bool BY_LDS = NP <= 4 && !TAIL;      // what entries take lies in LDS (else a loop over those of a piece: 16 of them 25 us of 54000 rows of 1000)
    __shared__ __attribute__((aligned(16))) float taken[BY_LDS ? WAVES * NP * 512 : 1];
    __shared__ int taught_by;
    const int64_t r = row_at(A.L, A.L.first + blockIdx.x, row_count(A.L));
    if (r < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = (int)threadIdx.x;
    const char* const row = A.h + r * A.h_stride;
    const int lead = (int)((uintptr_t)row & 15) / E, d = A.d + lead;      // columns of the line in front of the row; from there
    const char* const base = row - lead * E;
    auto load = [&](int c) -> fg_piece<T> {
        fg_piece<T> v = {};
        if (c > 0 || lead == 0) {
            if (c < d) v = fg_load_piece<T>(base + (int64_t)c * E, d - c);
        } else {
#pragma unroll
            for (int e = 1; e < 8; ++e)
                if (e >= lead && e < d) {
                    if constexpr (T == FG_F32)
                        (e < 4 ? v.a : v.b)[e & 3] = ((const unsigned int*)base)[e];
                    else
                        v.a[e / 2] |= (unsigned int)((const unsigned short*)base)[e] << (16 * (e & 1));
                }
        }
        return v;
    };
    fg_piece<T> raw[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i)
        if ((wave * 64 + WIDTH * i) * 8 < d) raw[i] = load((me + WIDTH * i) * 8);
    int32_t node, y;
    float weight;
    row_facts(A, r, node, y, weight);
    node = __builtin_amdgcn_readfirstlane(node), y = __builtin_amdgcn_readfirstlane(y), weight = one(weight);
    // the teacher's entries, one to a lane of the first wavefront, and their logits
    int32_t my_class = -1;
    float my_value = -INFINITY, my_z = 0.f, z_label = 0.f;
    if (wave == 0) {
        if (lane < A.k) entry_of(A, node, lane, my_class, my_value);
        if (my_class >= 0) my_z = fg_element(row, T, my_class);
        if (y >= 0) z_label = fg_element(row, T, y);
    }
    // f(piece, values) for every piece of this wavefront, columns that do not exist -infinity
    auto each = [&](auto f) {
        auto give = [&](int i, const fg_piece<T>& v) {
            const int c = (me + WIDTH * i) * 8;
            float w[8];
            fg_piece_values<T>(v, w);
            no_value_beyond(d - c, w);
            if (c == 0 && lead > 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < lead) w[e] = -INFINITY;
            f(i, w);
        };
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if ((wave * 64 + WIDTH * i) * 8 < d) give(i, raw[i]);
        if constexpr (TAIL)
            for (int i = NP; (wave * 64 + WIDTH * i) * 8 < d; ++i) give(i, load((me + WIDTH * i) * 8));
    };
    float m = -INFINITY;
    each([&](int, const float(&w)[8]) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) m = max3(m, w[e], w[e + 1]);
    });
    m = wave_max(m);
    const float soften = LOG2E / A.temperature;
    bool taught = false;
    float t_log = 0.f;
    if (wave == 0) {      // the teacher's distribution (a value that is NaN makes it NaN; without one above -infinity there is no teacher)
        taught = __ballot(my_class >= 0 && !(my_value == -INFINITY)) != 0;
        my_value = (my_value - wave_max(my_value)) * soften;
        t_log = log2_of(wave_sum(my_class >= 0 ? exp2_of(my_value) : 0.f));
    }
    if constexpr (WAVES > 1) {
        if (lane == 0) largest[wave] = m;
        if (wave == 0) {
            top_class[lane] = my_class, top_share[lane] = my_value;
            if (lane == 0) taught_by = taught, teacher_log = t_log;
        }
        __syncthreads();
        m = largest[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, largest[w]);
        taught = taught_by, t_log = teacher_log;
        if (wave != 0) my_class = top_class[lane], my_value = top_share[lane];
    }
    m = one(m), t_log = one(t_log);
    taught = __builtin_amdgcn_readfirstlane(taught);
    const bool either = taught || y >= 0;
    double soft = 0.0, hard = 0.0;
    if (either)
        each([&](int, const float(&w)[8]) {
            float s, h;
            sums_of(A.temperature, w, m, soften, s, h);
            soft += (double)s, hard += (double)h;
        });
    wave_sums(soft, hard);
    if constexpr (WAVES > 1) {
        if (lane == 0) red[0][wave] = soft, red[1][wave] = hard;
        __syncthreads();
        soft = hard = 0.0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) soft += red[0][w], hard += red[1][w];
    }
    const float soft_sum = one((float)soft), hard_sum = one((float)hard);
    const float log2_p = my_value - t_log, p = taught && my_class >= 0 ? exp2_of(log2_p) : 0.f;
    if (A.loss && wave == 0) {
        const float kl = wave_sum(p == 0.f ? 0.f : p * (log2_p - ((my_z - m) * soften - log2_of(soft_sum))));
        if (lane == 0) {
            float loss = 0.f;
            if (taught) loss += A.alpha * A.temperature * A.temperature * LN2 * kl;
            if (y >= 0) loss += (1.f - A.alpha) * (LN2 * log2_of(hard_sum) - (z_label - m));
            A.loss[r] = either ? weight * loss : 0.f;
        }
    }
    if (!A.dh) return;
    const float scale = A.grad_scale * weight, a = taught ? scale * A.alpha * A.temperature : 0.f, b = y >= 0 ? scale * (1.f - A.alpha) : 0.f;
    const float a_q = taught ? a / soft_sum : 0.f, b_q = y >= 0 ? b / hard_sum : 0.f, my_share = a * p;
    const int32_t my_place = taught && my_class >= 0 ? my_class + lead : -1, label_place = y >= 0 ? y + lead : -1;
    if constexpr (BY_LDS) {      // eight columns of a lane's piece behind each other
        float* const mine = taken + wave * NP * 512;
#pragma unroll
        for (int i = 0; i < NP; ++i) ((float4*)mine)[i * 128 + lane * 2] = ((float4*)mine)[i * 128 + lane * 2 + 1] = float4{0.f, 0.f, 0.f, 0.f};
        wave_meets();
        // where a column's share lies if it is in this wavefront's pieces, -1: it is not
        const auto at = [&](int32_t place) { return place >= 0 && (place >> 3) % WIDTH / 64 == wave ? (place >> 3) / WIDTH * 512 + (place & 511) : -1; };
        const int my_at = at(my_place), label_at = at(label_place);
        share_out(mine, my_at, my_share, lane);
        if (lane == 0 && label_at >= 0) mine[label_at] += b;
        wave_meets();
    }
    char* const out = A.dh + r * A.dh_stride;
    each([&](int i, const float(&w)[8]) {      // (all lanes of a wavefront together)
        float g[8] = {};
        if (either) gradients_of(A.temperature, w, m, soften, a_q, b_q, g);
        const int first = (wave * 64 + WIDTH * i) * 8, c = first + lane * 8;
        if constexpr (BY_LDS) {
            const float4* from = (const float4*)(taken + wave * NP * 512) + i * 128 + lane * 2;
            const float4 lo = from[0], hi = from[1];
            g[0] -= lo.x, g[1] -= lo.y, g[2] -= lo.z, g[3] -= lo.w, g[4] -= hi.x, g[5] -= hi.y, g[6] -= hi.z, g[7] -= hi.w;
        } else {
            // entries whose class lies in the wavefront's pieces: 512 columns from here
            auto take = [&](int32_t k, float share) {      // (the same in all lanes)
                const float mine = (k - first) >> 3 == lane ? share : 0.f;
                switch (k & 7) {
                    case 0: g[0] -= mine; break;
                    case 1: g[1] -= mine; break;
                    case 2: g[2] -= mine; break;
                    case 3: g[3] -= mine; break;
                    case 4: g[4] -= mine; break;
                    case 5: g[5] -= mine; break;
                    case 6: g[6] -= mine; break;
                    default: g[7] -= mine;
                }
            };
            unsigned long long there = __ballot(my_place >= first && my_place < first + 512);
            while (there) {
                const int l = __ffsll((long long)there) - 1;
                there &= there - 1;
                take(__builtin_amdgcn_readlane(my_place, l), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_share), l)));
            }
            if (label_place >= first && label_place < first + 512) take(label_place, b);
        }
        if (c >= d) return;
        auto put = [&](auto type) {
            constexpr int O = decltype(type)::value, OE = O == FG_F32 ? 4 : 2;
            char* const to = out + (int64_t)(c - lead) * OE;
            if (c > 0 || lead == 0) return fg_store_piece<O>(to, g, d - c);
            const fg_piece<O> v = fg_to_piece<O>(g);
#pragma unroll
            for (int e = 1; e < 8; ++e)
                if (e >= lead && e < d) {
                    if constexpr (O == FG_F32)
                        ((float*)to)[e] = g[e];
                    else
                        ((unsigned short*)to)[e] = (unsigned short)(v.a[e / 2] >> (16 * (e & 1)));
                }
        };
        if (A.dh_dtype == FG_F32)
            put(std::integral_constant<int, FG_F32>());
        else if constexpr (T != FG_F32)
            put(std::integral_constant<int, T>());
    });
}

template <int T, int LANES>
void launch_narrow(DistillArgs A, hipStream_t st) {
    constexpr int PER_BLOCK = DL_THREADS / LANES;
    const int64_t at_once = (FG_MAX_GRID - 1) * PER_BLOCK;      // rows of a launch
    for (; A.L.first < A.L.max_rows; A.L.first += at_once) {
        const int64_t rows = A.L.max_rows - A.L.first < at_once ? A.L.max_rows - A.L.first : at_once;
        hipLaunchKernelGGL((distill_narrow_kernel<T, LANES>), dim3((unsigned)fg_ceil_div(rows, PER_BLOCK)), dim3(DL_THREADS), (size_t)PER_BLOCK * A.k * sizeof(Entry), st, A);
    }
}
template <int T, int WAVES, int NP, bool TAIL>
void launch_wide(DistillArgs A, hipStream_t st) {
    const int64_t at_once = FG_MAX_GRID / WAVES - 1;
    for (; A.L.first < A.L.max_rows; A.L.first += at_once) {
        const int64_t rows = A.L.max_rows - A.L.first < at_once ? A.L.max_rows - A.L.first : at_once;
        hipLaunchKernelGGL((distill_wide_kernel<T, WAVES, NP, TAIL>), dim3((unsigned)rows), dim3(WAVES * 64), 0, st, A);
    }
}
template <int T>
void distill(const DistillArgs& A, hipStream_t st) {
    const int pieces = (int)fg_ceil_div(A.d, 8) + 1;      // (a row begins anywhere in its first line)
    if (A.d <= 64) return launch_narrow<T, 8>(A, st);
    if (A.d <= 128) return launch_narrow<T, 16>(A, st);
    if (A.d <= 256) return launch_narrow<T, 32>(A, st);
    if (A.d <= DL_NARROW) return launch_narrow<T, 64>(A, st);
    // One wavefront to a row where that holds it (what it does beside the row's values takes as long as some hundred of them), four where rows are few. One | four, us with 16
    // entries, bf16: 2048 x 2000 9.0 | 9.8, 16384 x 2000 38 | 48; 2048 x 4000 17 | 13, 16384 x 4000 74 | 70, 54000 x 4000 211 | 216; 2048 x 8000 27 | 25, 4096 x 8000 40 | 40,
    // 8192 x 8000 76 | 83. fp32: 2048 x 1000 8.2 | 9.6, 54000 x 1000 91 | 148, 2048 x 2000 11.5 | 11.8, 54000 x 2000 168 | 186; 2048 x 4000 19 | 17, 16384 x 3000 89 | 82,
    // 54000 x 3000 260 | 254, x 4000 341 | 320: four as soon as a row takes more than four pieces a lane. Sixteen for what four do not hold: four | sixteen, fp32: 8192 x 8000 103 | 184,
    // x 16000 203 | 260; bf16 8192 x 16000 128 | 152.
    constexpr int MOST = T == FG_F32 ? 8 : 16;
    if (pieces <= 256) return launch_wide<T, 1, 4, false>(A, st);
    if (pieces <= 512 && (T == FG_F32 || A.L.max_rows <= DL_FEW_ROWS)) return launch_wide<T, 4, 2, false>(A, st);
    if constexpr (T != FG_F32)
        if (pieces <= 64 * MOST && A.L.max_rows > DL_FEW_ROWS / 4) return launch_wide<T, 1, MOST, false>(A, st);
    if (pieces <= 256 * MOST) return launch_wide<T, 4, MOST, false>(A, st);
    if (pieces <= 8192) return launch_wide<T, 128 / MOST, MOST, false>(A, st);
    launch_wide<T, 128 / MOST, MOST, true>(A, st);
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
    if (d > FG_MAX_CLASSES) FG_FAIL(FG_ERR_SHAPE, "%s: d = %d is more than %d", who, d, FG_MAX_CLASSES);
    if (k < 0 || k > FG_MAX_TOP) FG_FAIL(FG_ERR_SHAPE, "%s: k = %d is not in 0..%d", who, k, FG_MAX_TOP);
    if (table_rows < 0 || table_rows > INT32_MAX) FG_FAIL(FG_ERR_INVALID_ARG, "%s: a number of rows is negative or too large", who);
    if (!(temperature >= 0x1p-60f && temperature <= 0x1p60f))      // (its square and its reciprocal are fp32 numbers)
        FG_FAIL(FG_ERR_INVALID_ARG, "%s: temperature = %g is not in 2^-60..2^60", who, (double)temperature);
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
    const DistillArgs A = {{rows_dev, n_rows_dev, max_rows, n, 0}, (const char*)h, h_stride, d, table_rows > 0 ? k : 0, ids_dev, top_idx_dev, (const char*)top_val_dev,
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

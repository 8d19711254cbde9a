// Eight adjacent values of a row, whatever their type, to and from fp32. The types: FG_F32, FG_F16, FG_BF16, and FG_E4M3 to write.
#pragma once
#include <hip/hip_fp16.h>

#include "common.h"

typedef unsigned int fg_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int fg_u32x2 __attribute__((ext_vector_type(2)));
// pieces of a row that begins at any element
typedef fg_u32x4 fg_u32x4_any __attribute__((aligned(2)));
typedef fg_u32x4 fg_u32x4_word __attribute__((aligned(4)));
typedef fg_u32x2 fg_u32x2_any __attribute__((aligned(1)));
typedef float fg_f32x8 __attribute__((ext_vector_type(8)));
typedef float fg_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 fg_bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 fg_f16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 fg_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 fg_f16x8 __attribute__((ext_vector_type(8)));

template <int T>
struct fg_piece;      // eight values as they lie in memory
template <>
struct fg_piece<FG_F32> {
    fg_u32x4 a, b;
};
template <>
struct fg_piece<FG_F16> {
    fg_u32x4 a;
};
template <>
struct fg_piece<FG_BF16> {
    fg_u32x4 a;
};

// `left` of the eight values lie in the row; the others come as zeros
template <int T>
__device__ __forceinline__ fg_piece<T> fg_load_piece(const char* p, int left) {
    fg_piece<T> v = {};
    if constexpr (T == FG_F32) {
        if (left >= 8) {
            v.a = *(const fg_u32x4_word*)p;
            v.b = *(const fg_u32x4_word*)(p + 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i < left) v.a[i] = ((const unsigned int*)p)[i];
                if (i + 4 < left) v.b[i] = ((const unsigned int*)p)[i + 4];
            }
        }
    } else {
        if (left >= 8) {
            v.a = *(const fg_u32x4_any*)p;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) v.a[i / 2] |= (unsigned int)((const unsigned short*)p)[i] << (16 * (i & 1));
        }
    }
    return v;
}
template <int T>
__device__ __forceinline__ void fg_piece_values(const fg_piece<T>& v, float (&f)[8]) {
    if constexpr (T == FG_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = __uint_as_float(v.a[i]);
            f[i + 4] = __uint_as_float(v.b[i]);
        }
    } else if constexpr (T == FG_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v.a[i] << 16);
            f[2 * i + 1] = __uint_as_float(v.a[i] & 0xFFFF0000u);
        }
    } else {
        const fg_f32x8 w = __builtin_convertvector(__builtin_bit_cast(fg_f16x8, v.a), fg_f32x8);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = w[i];
    }
}
// nearest even
template <int T>
__device__ __forceinline__ fg_piece<T> fg_to_piece(const float (&f)[8]) {
    fg_piece<T> v;
    if constexpr (T == FG_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v.a[i] = __float_as_uint(f[i]);
            v.b[i] = __float_as_uint(f[i + 4]);
        }
    } else {
        const fg_f32x8 w = {f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
        if constexpr (T == FG_BF16)
            v.a = __builtin_bit_cast(fg_u32x4, __builtin_convertvector(w, fg_bf16x8));
        else
            v.a = __builtin_bit_cast(fg_u32x4, __builtin_convertvector(w, fg_f16x8));
    }
    return v;
}
// four values to a 16-bit type, nearest even
template <int T>
__device__ __forceinline__ fg_u32x2 fg_to_words(const float (&f)[4]) {
    const fg_f32x4 w = {f[0], f[1], f[2], f[3]};
    if constexpr (T == FG_BF16)
        return __builtin_bit_cast(fg_u32x2, __builtin_convertvector(w, fg_bf16x4));
    else
        return __builtin_bit_cast(fg_u32x2, __builtin_convertvector(w, fg_f16x4));
}
template <int T>
__device__ __forceinline__ void fg_store_piece(char* p, const float (&f)[8], int left) {
    const fg_piece<T> v = fg_to_piece<T>(f);
    if constexpr (T == FG_F32) {
        if (left >= 8) {
            *(fg_u32x4_word*)p = v.a;
            *(fg_u32x4_word*)(p + 16) = v.b;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) ((float*)p)[i] = f[i];
        }
    } else {
        if (left >= 8) {
            *(fg_u32x4_any*)p = v.a;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) ((unsigned short*)p)[i] = (unsigned short)(v.a[i / 2] >> (16 * (i & 1)));
        }
    }
}
// eight values of at most 448 in magnitude (or NaN) to 8 bits
__device__ __forceinline__ void fg_store_piece_e4m3(char* p, const float (&f)[8], int left) {
    fg_u32x2 q;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * w], f[4 * w + 1], 0, false);
        q[w] = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * w + 2], f[4 * w + 3], v, true);
    }
    if (left >= 8) {
        *(fg_u32x2_any*)p = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) ((unsigned char*)p)[i] = (unsigned char)(q[i / 4] >> (8 * (i & 3)));
    }
}

// Device helpers of the operators on reconstructed weights (wave64, gfx950).
#pragma once
#include "excp_ops.h"
#include "excp_util.h"

typedef float v2f32 __attribute__((ext_vector_type(2)));
typedef float v4f32 __attribute__((ext_vector_type(4)));
typedef int v4i32 __attribute__((ext_vector_type(4)));
typedef int v8i32 __attribute__((ext_vector_type(8)));
typedef unsigned int v4u32 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(_Float16 x) { return (float)x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

// Eight consecutive elements, as they are stored: 16 B of a 16-bit type, 32 B of floats.
template <class T> struct Eight { T v[8]; };

// The first `have` of eight elements, zeros after them.  Whole ones in pieces of 16 bytes, wherever they begin.  (As vectors of
// words: where both ways move elements, the compiler joins what they have in common, and pieces of 12 bytes and less are left.)
typedef unsigned int words_anywhere __attribute__((ext_vector_type(4), aligned(2)));
template <class T>
__device__ __forceinline__ Eight<T> load_eight(const T *p, u32 have) {
    Eight<T> r;
    if (have >= 8u) {
        const auto *from = (const words_anywhere *)p;
        v4u32 w[sizeof r / 16];
#pragma unroll
        for (u32 i = 0; i < sizeof r / 16; ++i) w[i] = from[i];
        __builtin_memcpy(&r, w, sizeof r);
    } else {
#pragma unroll
        for (u32 i = 0; i < 8; ++i) r.v[i] = i < have ? p[i] : (T)0;
    }
    return r;
}
template <class T>
__device__ __forceinline__ void store_eight(T *p, const Eight<T> &r, u32 have) {
    if (have >= 8u) {
        auto *to = (words_anywhere *)p;
        v4u32 w[sizeof r / 16];
        __builtin_memcpy(w, &r, sizeof r);
#pragma unroll
        for (u32 i = 0; i < sizeof r / 16; ++i) to[i] = w[i];
    } else {
#pragma unroll
        for (u32 i = 0; i < 8; ++i)
            if (i < have) p[i] = r.v[i];
    }
}
template <class T>
__device__ __forceinline__ u32 word_of(const Eight<T> &r, u32 i) {      // two elements of a 16-bit type
    u32 w[4];
    __builtin_memcpy(w, &r, sizeof w);
    return w[i];
}

// Rows that can be written in pieces of 16 bytes.
template <class T>
__device__ __forceinline__ bool rows_aligned(const T *p, u64 ld) { return (((u64)p | ld * sizeof(T)) & 15u) == 0u; }
// Elements at .. at + N - 1 of a row of `end`, as they are stored, in one write where the row allows it.
template <class T, u32 N>
__device__ __forceinline__ void store_run(T *row, u32 at, u32 end, bool there, bool wide, uint4 v) {
    static_assert(N * sizeof(T) == 16, "");
    if (there && wide && at + N <= end) {
        *(uint4 *)(row + at) = v;
    } else if (there) {
        T e[N];
        __builtin_memcpy(e, &v, 16);
#pragma unroll
        for (u32 i = 0; i < N; ++i)
            if (at + i < end) row[at + i] = e[i];
    }
}
// Four sums to elements at .. at + 3 of a row of `end`.
template <class T>
__device__ __forceinline__ void store_four(T *row, u32 at, u32 end, v4f32 v) {
#pragma unroll
    for (u32 i = 0; i < 4; ++i)
        if (at + i < end) row[at + i] = (T)v[i];
}
// Four floats rounded to a 16-bit type.
template <class T>
__device__ __forceinline__ uint2 pack4(v4f32 v) {
    const T e[4] = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    uint2 r;
    __builtin_memcpy(&r, e, 8);
    return r;
}

// Quantisation of a block, in steps that lanes share: the largest magnitude (in the type's own bits, which order as the
// magnitudes do, infinities and NaN above all), the scale byte from it, the codes.
typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf16 __attribute__((ext_vector_type(2)));
typedef _Float16 v2f16 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32 max_halves(u32 a, u32 b) {               // of the two 16-bit halves, each
    return __builtin_bit_cast(u32, __builtin_elementwise_max(__builtin_bit_cast(v2u16, a), __builtin_bit_cast(v2u16, b)));
}
__device__ __forceinline__ u32 mx_peak(const Eight<float> &x) {
    u32 r = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) r = max(r, f2u(x.v[i]) & 0x7fffffffu);
    return r;
}
template <class T>
__device__ __forceinline__ u32 mx_peak(const Eight<T> &x) {
    u32 r = word_of(x, 0) & 0x7fff7fffu;
#pragma unroll
    for (u32 i = 1; i < 4; ++i) r = max_halves(r, word_of(x, i) & 0x7fff7fffu);
    return max(r & 0xffffu, r >> 16);
}
// floor(log2) - 2 of a normal number is its exponent field less 2 (biased alike), of a smaller one below the least there
// is; 255 for a NaN or an infinity.
template <class T>
__device__ __forceinline__ u32 mx_scale_byte(u32 peak) {
    if constexpr (sizeof(T) == 2) peak = f2u(widen(__builtin_bit_cast(T, (unsigned short)peak)));
    const int e = (int)(peak >> 23);
    return e == 255 ? 255u : (u32)max(e - 2, 0);
}
// 2^e of a scale byte e + 127: below the normal range for byte 0, NaN for 255.
__device__ __forceinline__ float mx_power(u32 byte) { return byte == 255u ? u2f(0x7fc00000u) : u2f(byte ? byte << 23 : 0x00400000u); }
// 2^-e: a normal number for every byte that a finite block has (0 .. 252).
__device__ __forceinline__ float mx_inverse(u32 byte) { return u2f((254u - byte) << 23); }
// The codes of eight elements; of a block that holds an infinity or a NaN, zeros.  The conversions divide by a power of
// two, round to the nearest of the grid, ties to the even code, and saturate.  (Floats are multiplied by the inverse first:
// the instruction takes no scale below the normal range.)
__device__ __forceinline__ u32 mx_codes(const Eight<float> &x, u32 byte) {
    const float s = mx_inverse(byte);
    u32 r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[0] * s, x.v[1] * s, 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[2] * s, x.v[3] * s, 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[4] * s, x.v[5] * s, 1.0f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x.v[6] * s, x.v[7] * s, 1.0f, 3);
    return byte == 255u ? 0u : r;
}
__device__ __forceinline__ u32 mx_codes_of_words(u32 a, u32 b, u32 c, u32 d, float s, __bf16) {
    u32 r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf16, a), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf16, b), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf16, c), s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf16, d), s, 3);
}
__device__ __forceinline__ u32 mx_codes_of_words(u32 a, u32 b, u32 c, u32 d, float s, _Float16) {
    u32 r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2f16, a), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2f16, b), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2f16, c), s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2f16, d), s, 3);
}
template <class T>
__device__ __forceinline__ u32 mx_codes(const Eight<T> &x, u32 byte) {
    const u32 r = mx_codes_of_words(word_of(x, 0), word_of(x, 1), word_of(x, 2), word_of(x, 3), mx_power(byte), T());
    return byte == 255u ? 0u : r;
}
// and back
__device__ __forceinline__ void mx_values(u32 codes, float *q) {
    v2f32 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1);
    v2f32 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    q[0] = a.x; q[1] = a.y; q[2] = b.x; q[3] = b.y; q[4] = c.x; q[5] = c.y; q[6] = d.x; q[7] = d.y;
}

// acc += A B^T over 128 elements, for 16 rows of either; lane l holds the 32 codes of row l % 16 from element
// 32 * (l / 16) on, and their scale in the lowest byte of its scale register.  Result: lane l holds rows
// 4 * (l / 16) .. + 3 of A against row l % 16 of B.
__device__ __forceinline__ v4f32 mx_mfma(v4i32 a, u32 sa, v4i32 b, u32 sb, v4f32 acc) {
    const v8i32 x = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    const v8i32 y = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, 0, (int)sa, 0, (int)sb);
}

// Memory to LDS without registers: every lane's 16 (4) bytes from its own address, to `to` (the same in every lane)
// plus 16 (4) times the lane's number.
typedef const __attribute__((address_space(1))) void *global_bytes;
typedef __attribute__((address_space(3))) void *lds_bytes;
__device__ __forceinline__ void load16_to_lds(const unsigned char *from, unsigned char *to) {
    __builtin_amdgcn_global_load_lds((global_bytes)from, (lds_bytes)to, 16, 0, 0);
}
__device__ __forceinline__ void load4_to_lds(const unsigned char *from, unsigned char *to) {
    __builtin_amdgcn_global_load_lds((global_bytes)from, (lds_bytes)to, 4, 0, 0);
}

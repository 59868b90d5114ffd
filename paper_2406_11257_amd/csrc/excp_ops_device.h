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

// One read in 16-byte pieces (p is 16-byte aligned).
template <class T>
__device__ __forceinline__ Eight<T> load_eight(const T *p) {
    Eight<T> r;
    __builtin_memcpy(&r, __builtin_assume_aligned(p, 16), sizeof r);
    return r;
}
// `have` elements one by one (any alignment), zeros after them.
template <class T>
__device__ __forceinline__ Eight<T> load_some(const T *p, u32 have) {
    Eight<T> r;
#pragma unroll
    for (u32 i = 0; i < 8; ++i) r.v[i] = i < have ? p[i] : (T)0;
    return r;
}

// Four consecutive elements in one write, where rows begin at multiples of four.
template <class T>
__device__ __forceinline__ bool store4_aligned(const T *p, u64 ld) { return (((u64)p | ld * sizeof(T)) & (4u * sizeof(T) - 1u)) == 0u; }
template <class T>
__device__ __forceinline__ void store4(T *p, v4f32 v) {
    struct alignas(4 * sizeof(T)) { T e[4]; } q = {{(T)v[0], (T)v[1], (T)v[2], (T)v[3]}};
    __builtin_memcpy(__builtin_assume_aligned(p, 4 * sizeof(T)), &q, sizeof q);
}

// Scale byte of a block from the largest of its magnitudes' bits: floor(log2) - 2 of a normal number is its exponent
// field less 2 (biased alike), of a smaller one below the least there is; 255 for a NaN or an infinity.
__device__ __forceinline__ u32 mx_scale_byte(u32 peak_bits) {
    const int e = (int)(peak_bits >> 23);
    return e == 255 ? 255u : (u32)max(e - 2, 0);
}
// 2^-(e) of a scale byte e + 127: a normal number for every byte that a finite block has (0 .. 252).
__device__ __forceinline__ float mx_inverse(u32 byte) { return u2f((254u - byte) << 23); }
// 2^e: below the normal range for byte 0, NaN for 255.
__device__ __forceinline__ float mx_power(u32 byte) { return byte == 255u ? u2f(0x7fc00000u) : u2f(byte ? byte << 23 : 0x00400000u); }

// Codes of eight elements already divided by their scale.  The conversion rounds to nearest even and saturates; the
// division is a multiplication before it, which is exact wherever the quotient matters (a quotient below the normal
// range rounds to zero either way).
__device__ __forceinline__ u32 mx_codes(const float *q) {
    u32 r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, q[0], q[1], 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, q[2], q[3], 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, q[4], q[5], 1.0f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, q[6], q[7], 1.0f, 3);
    return r;
}
// and back
__device__ __forceinline__ void mx_values(u32 codes, float *q) {
    v2f32 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1);
    v2f32 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    q[0] = a.x; q[1] = a.y; q[2] = b.x; q[3] = b.y; q[4] = c.x; q[5] = c.y; q[6] = d.x; q[7] = d.y;
}

// acc += A B^T over 128 elements, for 16 rows of either; lane l holds the 32 codes of row l % 16 from element
// 32 * (l / 16) on, and their scale in byte BYTE of its scale register.  Result: lane l holds rows
// 4 * (l / 16) .. + 3 of A against row l % 16 of B.
template <int BYTE = 0>
__device__ __forceinline__ v4f32 mx_mfma(v4i32 a, u32 sa, v4i32 b, u32 sb, v4f32 acc) {
    const v8i32 x = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    const v8i32 y = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, BYTE, (int)sa, BYTE, (int)sb);
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

// Microscaled 4-bit floating point: quantisation along the rows and down the columns of a matrix, and back.
#include "excp_ops_device.h"

namespace {

constexpr u32 kThreads = 256;

// One thread a block of 32, element by element.
template <class T, bool DOWN>
__global__ __launch_bounds__(kThreads) void k_mx_quantize(const T *__restrict__ x, u64 ld, u32 rows, u32 cols, u32 groups,
                                                          unsigned char *__restrict__ codes, unsigned char *__restrict__ scales,
                                                          u64 blocks) {
    // DOWN: "rows" of codes are the columns of x
    const u32 lines = DOWN ? cols : rows, len = DOWN ? rows : cols;
    for (u64 b = blockIdx.x * (u64)kThreads + threadIdx.x; b < blocks; b += (u64)gridDim.x * kThreads) {
        const u64 per = (u64)groups * 4u;
        const u32 line = DOWN ? (u32)(b % lines) : (u32)(b / per);
        const u32 at = DOWN ? (u32)(b / lines) : (u32)(b % per);
        float v[32];
        u32 peak = 0;
#pragma unroll
        for (u32 i = 0; i < 32; ++i) {
            const u32 j = at * 32u + i;
            const u64 o = DOWN ? (u64)j * ld + line : (u64)line * ld + j;
            v[i] = j < len ? widen(x[o]) : 0.0f;
            peak = max(peak, f2u(v[i]) & 0x7fffffffu);
        }
        const u32 byte = mx_scale_byte(peak);
        const float inv = byte == 255u ? 0.0f : mx_inverse(byte);
        u32 out[4];
#pragma unroll
        for (u32 w = 0; w < 4; ++w) {
            float q[8];
#pragma unroll
            for (u32 i = 0; i < 8; ++i) q[i] = byte == 255u ? 0.0f : v[w * 8 + i] * inv;
            out[w] = mx_codes(q);
        }
        const u64 o = (u64)line * per + at;
        *(uint4 *)(codes + o * 16u) = make_uint4(out[0], out[1], out[2], out[3]);
        scales[o] = (unsigned char)byte;
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize(const unsigned char *__restrict__ codes, const unsigned char *__restrict__ scales,
                                                            u32 cols, u32 groups, T *__restrict__ x, u64 ld, u64 pieces) {
    for (u64 i = blockIdx.x * (u64)kThreads + threadIdx.x; i < pieces; i += (u64)gridDim.x * kThreads) {
        const u64 row = i / (groups * 16u);
        const u32 at = (u32)(i % (groups * 16u)) * 8u;
        if (at >= cols) continue;
        float q[8];
        mx_values(*(const u32 *)(codes + i * 4u), q);
        const float scale = mx_power(scales[i / 4u]);
        T *out = x + row * ld + at;
#pragma unroll
        for (u32 j = 0; j < 8; ++j)
            if (at + j < cols) out[j] = (T)(q[j] * scale);
    }
}

u32 grid_for(u64 threads, u32 cus) { return (u32)std::min<u64>((threads + kThreads - 1) / kThreads, (u64)cus * 32u); }

}  // namespace

void launch_mx_quantize(const MxQuantize &q, u32 cus, hipStream_t s) {
    with_type(q.x.type, [&](auto tag) {
        using T = decltype(tag);
        if (q.codes) {
            const u32 groups = (q.x.cols + EXCP_MX_GROUP - 1) / EXCP_MX_GROUP;
            const u64 blocks = (u64)q.x.rows * groups * 4u;
            k_mx_quantize<T, false><<<grid_for(blocks, cus), kThreads, 0, s>>>((const T *)q.x.p, q.x.ld, q.x.rows, q.x.cols, groups, q.codes, q.scales, blocks);
        }
        if (q.codes_t) {
            const u32 groups = (q.x.rows + EXCP_MX_GROUP - 1) / EXCP_MX_GROUP;
            const u64 blocks = (u64)q.x.cols * groups * 4u;
            k_mx_quantize<T, true><<<grid_for(blocks, cus), kThreads, 0, s>>>((const T *)q.x.p, q.x.ld, q.x.rows, q.x.cols, groups, q.codes_t, q.scales_t, blocks);
        }
    });
}

void launch_mx_dequantize(const MxDequantize &d, u32 cus, hipStream_t s) {
    const u32 groups = (d.cols + EXCP_MX_GROUP - 1) / EXCP_MX_GROUP;
    const u64 pieces = (u64)d.rows * groups * 16u;
    with_type(d.type, [&](auto tag) {
        using T = decltype(tag);
        k_mx_dequantize<T><<<grid_for(pieces, cus), kThreads, 0, s>>>(d.codes, d.scales, d.cols, groups, (T *)d.x, d.ld, pieces);
    });
}

// Products of matrices in microscaled 4-bit floating point, on the matrix units.
#include "excp_ops_device.h"

namespace {

// One wave a tile of 64 x 64; operands straight from memory.
template <class T>
__global__ __launch_bounds__(256) void k_mx_product(const MxProduct p) {
    const u32 lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, r = lane & 15u, g = lane >> 4;
    const u32 tiles_n = (p.n + 127u) / 128u;
    const u64 tiles = (u64)tiles_n * ((p.m + 127u) / 128u);
    for (u64 tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const u32 n0 = (u32)(tile % tiles_n) * 128u + (wave & 1u) * 64u, m0 = (u32)(tile / tiles_n) * 128u + (wave >> 1) * 64u;
    v4f32 acc[4][4] = {};
    for (u32 k = 0; k < p.groups; ++k) {
        v4i32 w[4], x[4];
        u32 sw[4], sx[4];
#pragma unroll
        for (u32 i = 0; i < 4; ++i) {
            const u64 rw = (u64)min(n0 + i * 16u + r, p.n - 1u) * p.groups + k, rx = (u64)min(m0 + i * 16u + r, p.m - 1u) * p.groups + k;
            w[i] = *(const v4i32 *)(p.b_codes + rw * 64u + g * 16u);
            x[i] = *(const v4i32 *)(p.a_codes + rx * 64u + g * 16u);
            sw[i] = p.b_scales[rw * 4u + g];
            sx[i] = p.a_scales[rx * 4u + g];
        }
#pragma unroll
        for (u32 i = 0; i < 4; ++i)
#pragma unroll
            for (u32 j = 0; j < 4; ++j) acc[i][j] = mx_mfma(w[i], sw[i], x[j], sx[j], acc[i][j]);
    }
#pragma unroll
    for (u32 i = 0; i < 4; ++i)
#pragma unroll
        for (u32 j = 0; j < 4; ++j)
#pragma unroll
            for (u32 e = 0; e < 4; ++e) {
                const u32 n = n0 + i * 16u + g * 4u + e, m = m0 + j * 16u + r;
                if (n < p.n && m < p.m) ((T *)p.y)[(u64)m * p.ld + n] = (T)acc[i][j][e];
            }
    }
}

// Up to sixteen rows of x, quantised on the way: a lane's 32 elements are a block.  Sixteen rows of W a workgroup;
// its waves share the reduction and join their sums in LDS.
template <class X, class T>
__global__ __launch_bounds__(256) void k_mx_few_rows(const MxProduct p) {
    __shared__ v4f32 part[4][64];
    const u32 lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, r = lane & 15u, g = lane >> 4;
    for (u32 n0 = blockIdx.x * 16u; n0 < p.n; n0 += gridDim.x * 16u) {
    v4f32 acc = {};
    for (u32 k = wave; k < p.groups; k += 4u) {
        const u64 rw = (u64)min(n0 + r, p.n - 1u) * p.groups + k;
        const v4i32 w = *(const v4i32 *)(p.b_codes + rw * 64u + g * 16u);
        const u32 sw = p.b_scales[rw * 4u + g];
        float v[32];
        u32 peak = 0;
#pragma unroll
        for (u32 i = 0; i < 32; ++i) {
            const u32 j = k * 128u + g * 32u + i;
            v[i] = r < p.m && j < p.x.cols ? widen(((const X *)p.x.p)[r * p.x.ld + j]) : 0.0f;
            peak = max(peak, f2u(v[i]) & 0x7fffffffu);
        }
        const u32 byte = mx_scale_byte(peak);
        const float inv = byte == 255u ? 0.0f : mx_inverse(byte);
        v4i32 x;
#pragma unroll
        for (u32 i = 0; i < 4; ++i) {
            float q[8];
#pragma unroll
            for (u32 j = 0; j < 8; ++j) q[j] = byte == 255u ? 0.0f : v[i * 8 + j] * inv;
            x[i] = (int)mx_codes(q);
        }
        acc = mx_mfma(w, sw, x, byte, acc);
    }
    __syncthreads();
    part[wave][lane] = acc;
    __syncthreads();
    if (wave) continue;
    acc = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
#pragma unroll
    for (u32 e = 0; e < 4; ++e)
        if (n0 + g * 4u + e < p.n && r < p.m) ((T *)p.y)[(u64)r * p.ld + n0 + g * 4u + e] = (T)acc[e];
    }
}

}  // namespace

void launch_mx_product(const MxProduct &p, u32 cus, hipStream_t s) {
    with_type(p.type, [&](auto tag) {
        using T = decltype(tag);
        k_mx_product<T><<<(u32)std::min<u64>((u64)((p.n + 127u) / 128u) * ((p.m + 127u) / 128u), 1u << 20), 256, 0, s>>>(p);
    });
}

void launch_mx_few_rows(const MxProduct &p, u32 cus, hipStream_t s) {
    with_type(p.x.type, [&](auto xtag) {
        with_type(p.type, [&](auto tag) {
            using X = decltype(xtag);
            using T = decltype(tag);
            k_mx_few_rows<X, T><<<std::min((p.n + 15u) / 16u, 1u << 20), 256, 0, s>>>(p);
        });
    });
}

// Microscaled 4-bit floating point: quantisation along the rows and down the columns of a matrix, and back.
//
// The scale of a block of 32 is the power of two whose exponent is that of its largest magnitude less 2 (6, the largest
// element, is 1.5 x 2^2); the conversion instructions divide by it, round to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to
// the even code, and saturate.  All kernels here are bound by memory: 2 or 4 bytes an element one way, 0.53 the other.
// 11008 x 4096 in bf16: 27 us there (4.2 TB/s) and 18 back (6.3); along and down at once 4096 x 8192: 25 us (4.1).
#include "excp_ops_device.h"

#include <type_traits>

namespace {

constexpr u32 kThreads = 256;

// The largest of the quad of lanes that share a block, in all four.
__device__ __forceinline__ u32 quad_max(u32 v) {
    v = max(v, dpp_u32<0xb1, 0xf>(v, v));                    // lanes 1 0 3 2
    return max(v, dpp_u32<0x4e, 0xf>(v, v));                 // lanes 2 3 0 1
}
// A group's four scale bytes, one of each quad of its sixteen lanes, in all of them.
__device__ __forceinline__ u32 group_scales(u32 byte) {
    u32 v = byte << ((threadIdx.x >> 2 & 3u) * 8u);
    v |= dpp_u32<0x124, 0xf>(0u, v);                         // rotate the sixteen by 4, by 8
    return v | dpp_u32<0x128, 0xf>(0u, v);
}

// Sixteen lanes a group, eight elements each, so that a wave reads and writes whole lines and a block's largest is found by
// four neighbours; codes and scales lie group after group, whatever the rows.  A thread has `kPieces` pieces of
// groups under way.  (One row of 1024 takes 2 us, the launch; 11008 x 4096 in bf16 27 us out of memory, 20 where the last-level cache has it.)
template <class T, u32 kPieces>
__global__ __launch_bounds__(kThreads) void k_mx_quantize(const T *__restrict__ x, u64 ld, u32 cols, u32 groups, u32 all,
                                                          unsigned char *__restrict__ codes, unsigned char *__restrict__ scales) {
    constexpr u32 kStep = kThreads / 16u;
    const u32 at = threadIdx.x & 15u;
    for (u32 first = blockIdx.x * (kStep * kPieces) + threadIdx.x / 16u; first < all; first += gridDim.x * (kStep * kPieces)) {
        Eight<T> v[kPieces];
#pragma unroll
        for (u32 q = 0; q < kPieces; ++q) {
            const u32 i = first + q * kStep, row = i / groups, col = (i - row * groups) * EXCP_MX_GROUP + at * 8u;
            v[q] = load_eight(x + row * ld + col, i < all && col < cols ? cols - col : 0u);
        }
#pragma unroll
        for (u32 q = 0; q < kPieces; ++q) {
            const u32 i = first + q * kStep;
            const u32 byte = mx_scale_byte<T>(quad_max(mx_peak(v[q])));
            const u32 code = mx_codes(v[q], byte), four = group_scales(byte);
            if (i >= all) continue;
            *(u32 *)(codes + i * 64ull + at * 4u) = code;
            if (at == 0) *(u32 *)(scales + i * 4ull) = four;
        }
    }
}

// A tile of 128 x 128 elements a workgroup: quantised along its rows on the way in, and from LDS down its columns, so that x is
// read once for both.  All of a tile's reads are on their way before the first is used.
template <class T>
struct TileRoom {
    static constexpr u32 pitch = 128 * sizeof(T) / 4 + 1;    // in words
    u32 word[128 * pitch];
};
template <class T>
__global__ __launch_bounds__(kThreads) void k_mx_quantize_tile(const T *__restrict__ x, u64 ld, u32 rows, u32 cols, u32 tiles_c,
                                                               unsigned char *__restrict__ codes, unsigned char *__restrict__ scales,
                                                               unsigned char *__restrict__ codes_t, unsigned char *__restrict__ scales_t) {
    constexpr u32 kPitch = TileRoom<T>::pitch;
    __shared__ TileRoom<T> room;
    const u32 tiles_r = (rows + 127u) / 128u, at = threadIdx.x & 15u, first = threadIdx.x / 16u;
    for (u64 tile = blockIdx.x; tile < (u64)tiles_r * tiles_c; tile += gridDim.x) {
    const u32 tile_r = (u32)(tile / tiles_c), tile_c = (u32)(tile - (u64)tile_r * tiles_c), col = tile_c * 128u + at * 8u;
    Eight<T> v[8];
#pragma unroll
    for (u32 q = 0; q < 8; ++q) {
        const u32 row = tile_r * 128u + q * 16u + first;
        v[q] = load_eight(x + (u64)row * ld + col, row < rows && col < cols ? cols - col : 0u);
    }
#pragma unroll
    for (u32 q = 0; q < 8; ++q) {
        u32 w[8 * sizeof(T) / 4];
        __builtin_memcpy(w, &v[q], sizeof w);
#pragma unroll
        for (u32 i = 0; i < 8 * sizeof(T) / 4; ++i) room.word[(q * 16u + first) * kPitch + at * (8 * sizeof(T) / 4) + i] = w[i];
    }
    __syncthreads();
    if (codes) {                                             // the same for all
#pragma unroll
        for (u32 q = 0; q < 8; ++q) {
            const u32 row = tile_r * 128u + q * 16u + first;
            const u32 byte = mx_scale_byte<T>(quad_max(mx_peak(v[q])));
            const u32 code = mx_codes(v[q], byte), four = group_scales(byte);
            if (row < rows) {
                const u64 o = (u64)row * tiles_c + tile_c;
                *(u32 *)(codes + o * 64u + at * 4u) = code;
                if (at == 0) *(u32 *)(scales + o * 4u) = four;
            }
        }
    }
    // four lanes the four blocks of a column (of two, where a word holds two elements): 64 bytes of codes
    const u32 block = threadIdx.x & 3u;
    for (u32 c = threadIdx.x >> 2; c < 128u * sizeof(T) / 4u; c += kThreads / 4u) {
        const u32 *from = room.word + block * 32u * kPitch + c;
        u32 v[32];
#pragma unroll
        for (u32 i = 0; i < 32; ++i) v[i] = from[i * kPitch];
        if constexpr (sizeof(T) == 4) {
            u32 peak = 0, out[4];
#pragma unroll
            for (u32 i = 0; i < 32; ++i) peak = max(peak, v[i] & 0x7fffffffu);
            const u32 byte = mx_scale_byte<T>(peak);
#pragma unroll
            for (u32 q = 0; q < 4; ++q) {
                Eight<T> e;
                __builtin_memcpy(&e, v + q * 8, sizeof e);
                out[q] = mx_codes(e, byte);
            }
            const u32 j = tile_c * 128u + c;
            if (j < cols) {
                const u64 o = (u64)j * tiles_r + tile_r;
                *(uint4 *)(codes_t + o * 64u + block * 16u) = make_uint4(out[0], out[1], out[2], out[3]);
                scales_t[o * 4u + block] = (unsigned char)byte;
            }
        } else {
            u32 peaks = 0;
#pragma unroll
            for (u32 i = 0; i < 32; ++i) peaks = max_halves(peaks, v[i] & 0x7fff7fffu);
#pragma unroll
            for (u32 h = 0; h < 2; ++h) {
                const u32 byte = mx_scale_byte<T>(h ? peaks >> 16 : peaks & 0xffffu);
                u32 out[4];
#pragma unroll
                for (u32 q = 0; q < 4; ++q) {
                    u32 w[4];
#pragma unroll
                    for (u32 i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(v[q * 8 + i * 2 + 1], v[q * 8 + i * 2], h ? 0x07060302u : 0x05040100u);
                    Eight<T> e;
                    __builtin_memcpy(&e, w, sizeof e);
                    out[q] = mx_codes(e, byte);
                }
                const u32 j = tile_c * 128u + c * 2u + h;
                if (j < cols) {
                    const u64 o = (u64)j * tiles_r + tile_r;
                    *(uint4 *)(codes_t + o * 64u + block * 16u) = make_uint4(out[0], out[1], out[2], out[3]);
                    scales_t[o * 4u + block] = (unsigned char)byte;
                }
            }
        }
    }
    __syncthreads();
    }
}

// 16 bytes of x a lane: eight elements of a 16-bit type, four floats.  (Eight floats would be two writes a lane whose lanes
// lie 32 bytes apart: 8192 x 11008 in 109 us against 87.)
template <class T>
__global__ __launch_bounds__(kThreads) void k_mx_dequantize(const unsigned char *__restrict__ codes, const unsigned char *__restrict__ scales,
                                                            u32 cols, u32 groups, u32 all, T *__restrict__ x, u64 ld) {
    constexpr u32 kEach = 16 / sizeof(T), kLanes = EXCP_MX_GROUP / kEach, kPieces = 4, kStep = kThreads / kLanes;
    typedef typename std::conditional<kEach == 8, u32, unsigned short>::type Codes;
    const u32 at = threadIdx.x % kLanes;
    for (u32 first = blockIdx.x * (kStep * kPieces) + threadIdx.x / kLanes; first < all; first += gridDim.x * (kStep * kPieces)) {
        u32 code[kPieces], byte[kPieces];
#pragma unroll
        for (u32 q = 0; q < kPieces; ++q) {
            const u32 i = min(first + q * kStep, all - 1u);
            code[q] = *(const Codes *)(codes + i * 64ull + at * sizeof(Codes));
            byte[q] = scales[i * 4ull + at / (kLanes / 4u)];
        }
#pragma unroll
        for (u32 q = 0; q < kPieces; ++q) {
            const u32 i = first + q * kStep, row = i / groups, col = (i - row * groups) * EXCP_MX_GROUP + at * kEach;
            if (i >= all || col >= cols) continue;
            float v[8];
            mx_values(code[q], v);
            const float scale = mx_power(byte[q]);
            T e[kEach];
#pragma unroll
            for (u32 j = 0; j < kEach; ++j) e[j] = (T)(v[j] * scale);
            T *out = x + row * ld + col;
            if (col + kEach <= cols) {
                v4u32 w;
                __builtin_memcpy(&w, e, 16);
                *(words_anywhere *)out = w;
            } else {
#pragma unroll
                for (u32 j = 0; j < kEach; ++j)
                    if (col + j < cols) out[j] = e[j];
            }
        }
    }
}

// Calls f(first row, rows) for parts of a matrix whose groups 31 bits count.
template <class F>
void in_parts(u32 rows, u32 groups, F f) {
    const u32 most = std::max(1u, (1u << 31) / groups);
    for (u32 r = 0; r < rows; r += std::min(most, rows - r)) f(r, std::min(most, rows - r));
}
// workgroups for `all` groups, `each` at a time
u32 grid_for(u32 all, u32 each, u32 cus) { return std::min((all + each - 1u) / each, cus * 16u); }

}  // namespace

void launch_mx_quantize(const MxQuantize &q, u32 cus, hipStream_t s) {
    const Matrix &m = q.x;
    const u32 groups = (m.cols + EXCP_MX_GROUP - 1) / EXCP_MX_GROUP;
    with_type(m.type, [&](auto tag) {
        using T = decltype(tag);
        if (q.codes_t) {
            const u64 tiles = (u64)groups * ((m.rows + 127u) / 128u);
            k_mx_quantize_tile<T><<<(u32)std::min<u64>(tiles, 1u << 20), kThreads, 0, s>>>((const T *)m.p, m.ld, m.rows, m.cols, groups, q.codes, q.scales, q.codes_t, q.scales_t);
        } else {
            in_parts(m.rows, groups, [&](u32 r, u32 rows) {
                const u32 all = rows * groups;
                auto go = [&](auto kernel, u32 each) {
                    kernel<<<grid_for(all, each, cus), kThreads, 0, s>>>((const T *)m.p + (u64)r * m.ld, m.ld, m.cols, groups, all,
                                                                         q.codes + (u64)r * groups * 64u, q.scales + (u64)r * groups * 4u);
                };
                // few groups on as many compute units as there are (333 x 1000 in fp16: 3.4 us, four pieces a thread 4.6; 512 x
                // 4096, four times as many as may be, 4.5 either way)
                if (all <= 16u * cus) go(k_mx_quantize<T, 1>, 16u);
                else go(k_mx_quantize<T, 4>, 64u);
            });
        }
    });
}

void launch_mx_dequantize(const MxDequantize &d, u32 cus, hipStream_t s) {
    const u32 groups = (d.cols + EXCP_MX_GROUP - 1) / EXCP_MX_GROUP;
    with_type(d.type, [&](auto tag) {
        using T = decltype(tag);
        in_parts(d.rows, groups, [&](u32 r, u32 rows) {
            const u32 all = rows * groups;
            k_mx_dequantize<T><<<grid_for(all, sizeof(T) == 2 ? 64u : 32u, cus), kThreads, 0, s>>>(d.codes + (u64)r * groups * 64u, d.scales + (u64)r * groups * 4u, d.cols, groups,
                                                                       all, (T *)d.x + (u64)r * d.ld, d.ld);
        });
    });
}

// Products of matrices in microscaled 4-bit floating point, on the matrix units.
#include "excp_ops_device.h"

#include <type_traits>

namespace {

// A tile of WN x WM waves, each 16 TN rows of B (n) by 16 TM rows of A (m); 256 elements of the reduction a stage.
template <int TN, int TM, int WN, int WM>
struct Tile {
    static constexpr u32 bn = 16 * TN * WN, bm = 16 * TM * WM, rows = bn + bm, waves = WN * WM, threads = 64 * waves;
    static constexpr u32 codes = rows * 128u, stage = codes + rows * 8u;    // bytes: a row's codes, and its two groups' scales
    static constexpr u32 chunks = rows / 8u / waves;                        // loads a wave: 8 rows of codes each
    static constexpr u32 scale_loads = rows / 32u / waves;                  // and 32 rows of scales each
    static_assert(rows % (32u * waves) == 0, "");
    static constexpr int ahead = 2, before = 2 * TN - (TN + 1) / 2;         // steps (see the kernel)
    // fragments read before step q begins
    static constexpr int read_by(int q) {
        const int for_step = q + ahead;
        return q >= before - 1 || for_step >= 2 * TN ? 2 * (TM + TN) : (TM + TN) * (for_step / TN) + TM + for_step % TN + 1;
    }
};

// Which tile workgroup b takes.  Consecutive workgroups go to the eight chiplets in turn; so that those of one chiplet
// share rows of their operands in its L2, each has a run of tiles, and a run goes through bands of eight tiles' height.
__device__ __forceinline__ void place_of(u32 b, u32 tiles_n, u32 tiles_m, u32 &tn, u32 &tm) {
    const u32 tiles = tiles_n * tiles_m, per = tiles / 8u, more = tiles % 8u, xcd = b % 8u;
    const u32 t = xcd * per + min(xcd, more) + b / 8u;
    const u32 band = t / (8u * tiles_n), high = min(8u, tiles_m - band * 8u), in = t - band * 8u * tiles_n;
    tm = band * 8u + in % high;
    tn = in / high;
}

template <int A, int B, class F>
__device__ __forceinline__ void static_for(F f) {
    if constexpr (A < B) {
        f(std::integral_constant<int, A>{});
        static_for<A + 1, B>(f);
    }
}

template <class T, int TN, int TM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM) void k_mx_product(const MxProduct p) {
    using L = Tile<TN, TM, WN, WM>;
    __shared__ __attribute__((aligned(16))) unsigned char even[L::stage], odd[L::stage];
    const u32 lane = lane_id(), r = lane & 15u, g = lane >> 4;
    const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const u32 wn = wave % WN, wm = wave / WN;
    u32 tile_n, tile_m;
    place_of(blockIdx.x, (p.n + L::bn - 1) / L::bn, (p.m + L::bm - 1) / L::bm, tile_n, tile_m);
    const u32 n0 = tile_n * L::bn, m0 = tile_m * L::bm;
    const u32 groups = p.groups, lone = groups & 1u, stages = groups / 2u;

    // What this wave brings in: rows of codes, eight a load, with the 16-byte pieces of a row permuted so that the
    // sixteen rows of a fragment lie in different banks; and rows of scales, thirty-two a load.  Rows that the matrices
    // do not have are read as the last one that they have, and not stored in the end.
    const u32 code_pitch = groups * 64u, scale_pitch = groups * 4u;
    const u32 n_last = min(L::bn, p.n - n0) - 1u, m_last = min(L::bm, p.m - m0) - 1u;
    const unsigned char *const b_codes = p.b_codes + (u64)n0 * code_pitch, *const a_codes = p.a_codes + (u64)m0 * code_pitch;
    const unsigned char *const b_scales = p.b_scales + (u64)n0 * scale_pitch, *const a_scales = p.a_scales + (u64)m0 * scale_pitch;
    const u32 piece = (lane & 7u) ^ (lane >> 3);
    u32 code_at[L::chunks], scale_at[L::scale_loads];
#pragma unroll
    for (u32 c = 0; c < L::chunks; ++c) {
        const u32 row = (wave * L::chunks + c) * 8u + (lane >> 3);
        code_at[c] = (row < L::bn ? min(row, n_last) : min(row - L::bn, m_last)) * code_pitch + piece * 16u;
    }
#pragma unroll
    for (u32 c = 0; c < L::scale_loads; ++c) {
        const u32 row = (wave * L::scale_loads + c) * 32u + (lane >> 1);
        scale_at[c] = (row < L::bn ? min(row, n_last) : min(row - L::bn, m_last)) * scale_pitch + (lane & 1u) * 4u;
    }
    // groups `first` and `first` + 1 (of a lone group: twice the same)
    auto fetch = [&](unsigned char *buf, u32 first, u32 back_codes, u32 back_scales) __attribute__((always_inline)) {
#pragma unroll
        for (u32 c = 0; c < L::chunks; ++c) {
            const u32 chunk = wave * L::chunks + c;
            u32 at = code_at[c] - back_codes;
            asm volatile("" : "+v"(at));                     // (as in `hidden`: no pointer a load kept and moved on)
            load16_to_lds((chunk * 8u < L::bn ? b_codes : a_codes) + first * 64u + at, buf + chunk * 1024u);
        }
#pragma unroll
        for (u32 c = 0; c < L::scale_loads; ++c) {
            const u32 chunk = wave * L::scale_loads + c;
            u32 at = scale_at[c] - back_scales;
            asm volatile("" : "+v"(at));
            load4_to_lds((chunk * 32u < L::bn ? b_scales : a_scales) + first * 4u + at, buf + L::codes + chunk * 256u);
        }
    };
    const u32 rn = wn * TN * 16u + r, rm = L::bn + wm * TM * 16u + r;
    // Where this lane's parts of the fragments lie.
    struct Places { u32 n[2], m[2], n_scale, m_scale; };
    const u32 swizzled = (g ^ (r & 7u)) * 16u;
    const Places places = {{rn * 128u + swizzled, rn * 128u + (swizzled ^ 64u)}, {rm * 128u + swizzled, rm * 128u + (swizzled ^ 64u)},
                           L::codes + rn * 8u + g, L::codes + rm * 8u + g};
    // The numbers are hidden from the compiler once a stage: it would otherwise keep a register for the address of every
    // fragment of both buffers.
    auto hidden = [&]() __attribute__((always_inline)) {
        Places at = places;
        asm volatile("" : "+v"(at.n[0]), "+v"(at.n[1]), "+v"(at.m[0]), "+v"(at.m[1]), "+v"(at.n_scale), "+v"(at.m_scale));
        return at;
    };
    v4f32 acc[TN][TM] = {};
    v4i32 n_frag[2][TN], m_frag[2][TM];
    u32 n_scale[2][TN], m_scale[2][TM];
    // A stage's fragments in the order in which they are read, and its products in steps of one fragment of B.  A step's
    // fragments are read L::ahead steps before it; all of a stage's are, before its last steps, and those steps go on while
    // the next stage's first ones arrive.  (Left to itself the compiler reads a fragment where it needs it.)
    auto read = [&](const unsigned char *buf, const Places &at, auto index) __attribute__((always_inline)) {
        constexpr int s = decltype(index)::value / (TM + TN), w = decltype(index)::value % (TM + TN);
        if constexpr (w < TM) {
            m_scale[s][w] = buf[at.m_scale + w * 128 + s * 4];
            m_frag[s][w] = *(const v4i32 *)(buf + at.m[s] + w * 2048);
        } else {
            n_scale[s][w - TM] = buf[at.n_scale + (w - TM) * 128 + s * 4];
            n_frag[s][w - TM] = *(const v4i32 *)(buf + at.n[s] + (w - TM) * 2048);
        }
    };
    auto step = [&](auto index) __attribute__((always_inline)) {
        constexpr int s = decltype(index)::value / TN, i = decltype(index)::value % TN;
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = mx_mfma(n_frag[s][i], n_scale[s][i], m_frag[s][j], m_scale[s][j], acc[i][j]);
    };
    // The products up to here are not put off until after what follows.
    auto done = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) asm volatile("" : "+v"(acc[i][j]));
    };
    // All loads to LDS that this wave has issued are there; with the barrier after it, those of all waves.
    auto landed = []() __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0)
        __syncthreads();
    };
    auto begin = [&](const unsigned char *buf) __attribute__((always_inline)) {
        const Places at = hidden();
        static_for<0, L::read_by(-1)>([&](auto f) __attribute__((always_inline)) { read(buf, at, f); });
    };
    auto stage = [&](unsigned char *cur, unsigned char *next, u32 t) __attribute__((always_inline)) {
        const Places at = hidden();
        static_for<0, L::before>([&](auto q) __attribute__((always_inline)) {
            static_for<L::read_by(q - 1), L::read_by(q)>([&](auto f) __attribute__((always_inline)) { read(cur, at, f); });
            __builtin_amdgcn_sched_barrier(0);
            step(q);
            __builtin_amdgcn_sched_barrier(0);
        });
        done();
        landed();                                            // `next` is there, and `cur` has been read by all
        if (t + 2u < stages) fetch(cur, lone + 2u * (t + 2u), 0u, 0u);
        begin(next);                                         // (after the last stage: whatever is there, and unused)
        __builtin_amdgcn_sched_barrier(0);
        static_for<L::before, 2 * TN>(step);
        done();
    };
    if (lone) {
        fetch(even, 0, (piece & 4u) * 16u, (lane & 1u) * 4u);
        landed();
        const Places at = hidden();
        static_for<0, TM + TN>([&](auto f) __attribute__((always_inline)) { read(even, at, f); });
        static_for<0, TN>(step);
        __syncthreads();
    }
    if (stages) {
        fetch(even, lone, 0u, 0u);
        landed();
        if (1u < stages) fetch(odd, lone + 2u, 0u, 0u);
        begin(even);
        for (u32 t = 0; t < stages; t += 2u) {
            stage(even, odd, t);
            if (t + 1u < stages) stage(odd, even, t + 1u);
        }
    }
    const bool wide = store4_aligned((const T *)p.y, p.ld);
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const u32 m = m0 + (wm * TM + j) * 16u + r;
        if (m >= p.m) continue;
        T *y = (T *)p.y + (u64)m * p.ld;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const u32 n = n0 + (wn * TN + i) * 16u + g * 4u;
            if (wide && n + 4u <= p.n) {
                store4(y + n, acc[i][j]);
            } else {
#pragma unroll
                for (u32 e = 0; e < 4; ++e)
                    if (n + e < p.n) y[n + e] = (T)acc[i][j][e];
            }
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

template <class T, int TN, int TM, int WN, int WM>
void launch_tiles(const MxProduct &p, hipStream_t s) {
    using L = Tile<TN, TM, WN, WM>;
    const u64 tiles = (u64)((p.n + L::bn - 1) / L::bn) * ((p.m + L::bm - 1) / L::bm);
    k_mx_product<T, TN, TM, WN, WM><<<(u32)tiles, L::threads, 0, s>>>(p);
}

void launch_mx_product(const MxProduct &p, u32 cus, hipStream_t s) {
    with_type(p.type, [&](auto tag) {
        using T = decltype(tag);
        const u64 large = (u64)((p.n + 255u) / 256u) * ((p.m + 255u) / 256u), middle = (u64)((p.n + 127u) / 128u) * ((p.m + 127u) / 128u);
        if (large >= cus * 3 / 4) launch_tiles<T, 8, 4, 2, 4>(p, s);
        else if (middle >= cus * 3 / 4) launch_tiles<T, 4, 4, 2, 2>(p, s);
        else launch_tiles<T, 2, 2, 2, 2>(p, s);
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

// Products of matrices in microscaled 4-bit floating point, on the matrix units.
//
// y[i][j] = sum over the blocks b of the reduction of 2^(ea + eb) sum_t a[t] b[t]: the matrix units take the codes and the two
// scales of a block as they are stored, and add in fp32; the one rounding is the result's.  W's rows are the unit's first
// operand, so that a lane's results are neighbours in a row of y.
//
// Many rows are bound by the matrix units beside what feeds them: 8192 x 8192 x 8192 takes 287 us, 3.8 PFLOP/s, 260 without
// the writes of y and 246 without the loads either, where the units alone, from registers, reach 6.5 PFLOP/s at the clock
// that the power allows.  Few rows are bound by reading W.
#include "excp_ops_device.h"

#include <type_traits>

namespace {

// A tile of WN x WM waves, each 16 TN rows of B (n) by 16 TM rows of A (m); 256 elements of the reduction a stage.  KS such
// sets of waves share the stages of a workgroup's tile, each with buffers of its own.
template <int TN, int TM, int WN, int WM, int KS>
struct Tile {
    static constexpr u32 bn = 16 * TN * WN, bm = 16 * TM * WM, rows = bn + bm, waves = WN * WM, threads = 64 * waves * KS;
    static constexpr u32 codes = rows * 128u, stage = codes + rows * 8u;    // bytes: a row's codes, and its two groups' scales
    static constexpr u32 chunks = rows / 8u / waves;                        // loads a wave: 8 rows of codes each
    static constexpr u32 scale_loads = rows / 32u / waves;                  // and 32 rows of scales each
    static constexpr int loads = chunks + scale_loads;
    static_assert(rows % (32u * waves) == 0 && (KS - 1) * bn * bm * 4u <= KS * stage, "");
    static constexpr int ahead = 2, before = 2 * TN - (TN + 1) / 2;         // steps (see the kernel)
    // loads issued before step i of those over which they are spread, counted from the barrier that frees their buffer
    static constexpr int after = 2 * TN - before, spread = 2 * TN - (TN / 2 + 1);
    static constexpr int loaded_by(int i) { return i >= spread ? loads : loads * i / spread; }
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

// A stage's operands lie in LDS twice, one buffer being filled from memory while the other is read; a wave multiplies 16 TN x
// 16 TM rows, so that each byte read from LDS is used TN or TM times: waves of 128 x 64 in a tile of 256 x 256, which the
// registers hold with two waves a SIMD.  (Tried: 128 x 128 a wave, one wave a SIMD, 324 us for 8192 x 8192 x 8192; the 32 x 32
// shape of the unit, 319; a workgroup that goes on to another tile with its first stages on their way while the last is
// written, 302; writes past the caches, 302.)
template <class T, int TN, int TM, int WN, int WM, int KS>
__global__ __launch_bounds__(64 * WN * WM * KS) void k_mx_product(const MxProduct p) {
    using L = Tile<TN, TM, WN, WM, KS>;
    __shared__ __attribute__((aligned(16))) unsigned char even[KS * L::stage], odd[KS * L::stage];
    const u32 lane = lane_id(), r = lane & 15u, g = lane >> 4;
    const u32 any_wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const u32 set = KS > 1 ? any_wave / L::waves : 0u, wave = any_wave - set * L::waves;
    const u32 wn = wave % WN, wm = wave / WN;
    u32 tile_n, tile_m;
    place_of(blockIdx.x, (p.n + L::bn - 1) / L::bn, (p.m + L::bm - 1) / L::bm, tile_n, tile_m);
    const u32 n0 = tile_n * L::bn, m0 = tile_m * L::bm;
    // An odd number of groups leaves one, the first, before the stages; the last round may not have a stage for every set.
    const u32 groups = p.groups, lone = groups & 1u, stages = groups / 2u, rounds = (stages + KS - 1u) / KS;
    auto there = [&](u32 t) __attribute__((always_inline)) { return t * KS + set < stages; };
    auto first_of = [&](u32 t) __attribute__((always_inline)) { return lone + 2u * (t * KS + set); };

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
    // Groups `first` and `first` + 1 (of a lone group: twice the same): load `c` of what this wave brings in.
    auto load = [&](unsigned char *buf, u32 first, u32 back_codes, u32 back_scales, auto index) __attribute__((always_inline)) {
        constexpr u32 c = decltype(index)::value;
        if constexpr (c >= L::scale_loads) {
            const u32 chunk = wave * L::chunks + (c - L::scale_loads);
            u32 at = code_at[c - L::scale_loads] - back_codes;
            asm volatile("" : "+v"(at));                     // (as in `hidden`: no pointer a load kept and moved on)
            load16_to_lds((chunk * 8u < L::bn ? b_codes : a_codes) + first * 64u + at, buf + set * L::stage + chunk * 1024u);
        } else {
            const u32 chunk = wave * L::scale_loads + c;
            u32 at = scale_at[c] - back_scales;
            asm volatile("" : "+v"(at));
            load4_to_lds((chunk * 32u < L::bn ? b_scales : a_scales) + first * 4u + at, buf + set * L::stage + L::codes + chunk * 256u);
        }
    };
    auto fetch = [&](unsigned char *buf, u32 first, u32 back_codes, u32 back_scales) __attribute__((always_inline)) {
        static_for<0, L::loads>([&](auto c) __attribute__((always_inline)) { load(buf, first, back_codes, back_scales, c); });
    };
    const u32 rn = wn * TN * 16u + r, rm = L::bn + wm * TM * 16u + r;
    // Where this lane's parts of the fragments lie.
    struct Places { u32 n[2], m[2], n_scale, m_scale; };
    const u32 swizzled = (g ^ (r & 7u)) * 16u;
    const u32 base = set * L::stage;
    const Places places = {{base + rn * 128u + swizzled, base + rn * 128u + (swizzled ^ 64u)}, {base + rm * 128u + swizzled, base + rm * 128u + (swizzled ^ 64u)},
                           base + L::codes + rn * 8u + g, base + L::codes + rm * 8u + g};
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
        // (the products are not put off until after what follows)
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            if constexpr (L::threads > 256) asm volatile("" : "+v"(acc[i][j]));
            else asm volatile("" : "+a"(acc[i][j]));
        }
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
    // Loads are spread over the steps: many in a row would keep a wave from its products until the last has been taken.
    // Those of the next stage but one begin after the barrier that frees their buffer and end in the next stage.
    auto stage = [&](unsigned char *cur, unsigned char *next, u32 t) __attribute__((always_inline)) {
        const Places at = hidden();
        const bool here = KS == 1 || there(t);
        static_for<0, L::before>([&](auto q) __attribute__((always_inline)) {
            if (there(t + 1u))
                static_for<L::loaded_by(L::after + q), L::loaded_by(L::after + q + 1)>([&](auto c) __attribute__((always_inline)) {
                    load(next, first_of(t + 1u), 0u, 0u, c);
                });
            static_for<L::read_by(q - 1), L::read_by(q)>([&](auto f) __attribute__((always_inline)) { read(cur, at, f); });
            __builtin_amdgcn_sched_barrier(0);
            if (here) step(q);
            __builtin_amdgcn_sched_barrier(0);
        });
        landed();                                            // `next` is there, and `cur` has been read by all
        begin(next);                                         // (after the last stage: whatever is there, and unused)
        static_for<L::before, 2 * TN>([&](auto q) __attribute__((always_inline)) {
            if (there(t + 2u))
                static_for<L::loaded_by(q - L::before), L::loaded_by(q - L::before + 1)>([&](auto c) __attribute__((always_inline)) {
                    load(cur, first_of(t + 2u), 0u, 0u, c);
                });
            __builtin_amdgcn_sched_barrier(0);
            if (here) step(q);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    if (lone) {
        if (set == 0) fetch(even, 0, (piece & 4u) * 16u, (lane & 1u) * 4u);
        landed();
        if (set == 0) {
            const Places at = hidden();
            static_for<0, TM + TN>([&](auto f) __attribute__((always_inline)) { read(even, at, f); });
            static_for<0, TN>(step);
        }
        __syncthreads();
    }
    if (stages) {
        if (there(0)) fetch(even, first_of(0), 0u, 0u);
        landed();
        if (there(1u))
            static_for<0, L::loaded_by(L::after)>([&](auto c) __attribute__((always_inline)) { load(odd, first_of(1u), 0u, 0u, c); });
        begin(even);
        for (u32 t = 0; t < rounds; t += 2u) {
            stage(even, odd, t);
            if (t + 1u < rounds) stage(odd, even, t + 1u);
        }
    }
    if constexpr (KS > 1) {
        // the sets' sums together, in order, in the first one
        __syncthreads();
        v4f32 *const sums = (v4f32 *)even + (wave * TN * TM) * 64u + lane;
        constexpr u32 of_a_set = L::waves * TN * TM * 64u;
        if (set) {
#pragma unroll
            for (int i = 0; i < TN * TM; ++i) sums[(set - 1u) * of_a_set + i * 64u] = acc[i / TM][i % TM];
        }
        __syncthreads();
        if (set) return;
#pragma unroll
        for (u32 other = 0; other < KS - 1u; ++other)
#pragma unroll
            for (int i = 0; i < TN * TM; ++i) acc[i / TM][i % TM] += sums[other * of_a_set + i * 64u];
    }
    // A lane holds four consecutive elements of a row of y, sixteen apart.  Of a 16-bit type that would be 32 bytes of a row
    // a write: the lanes of two neighbouring fragments trade halves first, and it is 64.
    const bool wide = rows_aligned((const T *)p.y, p.ld);
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const u32 m = m0 + (wm * TM + j) * 16u + r;
        T *y = (T *)p.y + (u64)min(m, p.m - 1u) * p.ld;
#pragma unroll
        for (int i = 0; i < TN; i += 2) {
            const u32 n = n0 + (wn * TN + i) * 16u;
            if constexpr (sizeof(T) == 2) {
                const uint2 a = pack4<T>(acc[i][j]), b = pack4<T>(acc[i + 1][j]);
                const auto lo = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false), hi = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
                store_run<T, 8>(y, n + (g & 1u) * 16u + (g >> 1) * 8u, p.n, m < p.m, wide, make_uint4(lo[0], hi[0], lo[1], hi[1]));
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    store_run<T, 4>(y, n + k * 16u + g * 4u, p.n, m < p.m, wide, __builtin_bit_cast(uint4, acc[i + k][j]));
            }
        }
    }
}

// Up to sixteen rows of A against sixteen rows of B a workgroup: its eight waves take the groups of the reduction in turn
// (so that together they read runs of a row), straight into registers, four on their way at a time, and join their sums in
// LDS.  The rows of B are read once, each by one wave, and that is the time it takes.
template <class T>
__global__ __launch_bounds__(512) void k_mx_few_rows(const MxProduct p) {
    constexpr u32 kWaves = 8, kBatch = 4;
    __shared__ v4f32 sums[kWaves][64];
    const u32 lane = lane_id(), r = lane & 15u, g = lane >> 4, n0 = blockIdx.x * 16u;
    const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const u64 b_row = (u64)min(n0 + r, p.n - 1u) * p.groups, a_row = (u64)min(r, p.m - 1u) * p.groups;
    v4f32 acc = {};
    for (u32 first = wave; first < p.groups; first += kWaves * kBatch) {
        v4i32 b[kBatch], a[kBatch];
        u32 by_b[kBatch], by_a[kBatch];
#pragma unroll
        for (u32 u = 0; u < kBatch; ++u) {
            const u32 k = first + u * kWaves;
            if (k >= p.groups) continue;
            b[u] = *(const v4i32 *)(p.b_codes + (b_row + k) * 64u + g * 16u);
            a[u] = *(const v4i32 *)(p.a_codes + (a_row + k) * 64u + g * 16u);
            by_b[u] = p.b_scales[(b_row + k) * 4u + g];
            by_a[u] = p.a_scales[(a_row + k) * 4u + g];
        }
#pragma unroll
        for (u32 u = 0; u < kBatch; ++u)
            if (first + u * kWaves < p.groups) acc = mx_mfma(b[u], by_b[u], a[u], by_a[u], acc);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (u32 i = 1; i < kWaves; ++i) acc += sums[i][lane];
    if (r < p.m) store_four((T *)p.y + (u64)r * p.ld, n0 + g * 4u, p.n, acc);
}

// The same for up to sixteen rows of x that are quantised on the way: once a workgroup, into LDS (a part of the reduction at
// a time, where all of it does not fit), and from there against tile after tile of sixteen rows of W.  What lanes of rows that
// x does not have read is another row's: nobody reads their sums.
// One row by 4096 x 4096 takes 4.7 us (quantised by every wave for itself, 6.8), of which W's bytes are 1.8; by 50304 x 4096
// 26.6, W 21.
template <class X, class T>
__global__ __launch_bounds__(512) void k_mx_few_rows_of(const MxProduct p, u32 room) {
    constexpr u32 kWaves = 8, kBatch = 4;
    extern __shared__ __attribute__((aligned(16))) unsigned char x_codes[];      // [group of the part][row][64], then scales
    __shared__ v4f32 sums[kWaves][64];
    const u32 lane = lane_id(), r = min(lane & 15u, p.m - 1u), g = lane >> 4;
    const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    unsigned char *const x_scales = x_codes + room * p.m * 64u;
    const u32 tiles = (p.n + 15u) / 16u;
    auto quantize = [&](u32 from, u32 groups) __attribute__((always_inline)) {
        for (u32 b = threadIdx.x; b < groups * 4u * p.m; b += 64u * kWaves) {
            const u32 row = b / (groups * 4u), at = b - row * (groups * 4u), col = from * 128u + at * 32u;
            const X *x = (const X *)p.x.p + (u64)row * p.x.ld + col;
            const u32 have = col < p.x.cols ? p.x.cols - col : 0u;
            Eight<X> e[4];
            u32 peak = 0, code[4];
#pragma unroll
            for (u32 q = 0; q < 4; ++q) e[q] = load_eight(x + q * 8u, have > q * 8u ? have - q * 8u : 0u);
#pragma unroll
            for (u32 q = 0; q < 4; ++q) peak = max(peak, mx_peak(e[q]));
            const u32 byte = mx_scale_byte<X>(peak), o = (at / 4u) * p.m + row;
#pragma unroll
            for (u32 q = 0; q < 4; ++q) code[q] = mx_codes(e[q], byte);
            *(uint4 *)(x_codes + o * 64u + (at & 3u) * 16u) = make_uint4(code[0], code[1], code[2], code[3]);
            x_scales[o * 4u + (at & 3u)] = (unsigned char)byte;
        }
    };
    const unsigned char *codes, *scales;
    v4i32 w[kBatch];
    u32 by[kBatch];
    // groups from + k, from + k + 8, .. of a part of `end`
    auto load = [&](u32 from, u32 k, u32 end) __attribute__((always_inline)) {
#pragma unroll
        for (u32 u = 0; u < kBatch; ++u)
            if (k + u * kWaves < end) {
                w[u] = *(const v4i32 *)(codes + (from + k + u * kWaves) * 64ull);
                by[u] = scales[(from + k + u * kWaves) * 4ull];
            }
    };
    const bool once = p.groups <= room;
    if (once) quantize(0, p.groups);
    for (u32 tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const u64 at = (u64)min(tile * 16u + (lane & 15u), p.n - 1u) * p.groups;
        codes = p.b_codes + at * 64u + g * 16u;
        scales = p.b_scales + at * 4u + g;
        v4f32 acc = {};
        for (u32 from = 0; from < p.groups; from += room) {
            const u32 end = min(p.groups - from, room);
            load(from, wave, end);
            if (!once) {
                __syncthreads();                             // the last part has been read
                quantize(from, end);
            }
            if (!once || tile == blockIdx.x) __syncthreads();
            for (u32 k = wave; k < end;) {
#pragma unroll
                for (u32 u = 0; u < kBatch; ++u)
                    if (k + u * kWaves < end) {
                        const u32 o = (k + u * kWaves) * p.m + r;
                        acc = mx_mfma(w[u], by[u], *(const v4i32 *)(x_codes + o * 64u + g * 16u), x_scales[o * 4u + g], acc);
                    }
                k += kBatch * kWaves;
                load(from, k, end);
            }
        }
        sums[wave][lane] = acc;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (u32 i = 1; i < kWaves; ++i) acc += sums[i][lane];
            if ((lane & 15u) < p.m) store_four((T *)p.y + (u64)r * p.ld, tile * 16u + g * 4u, p.n, acc);
        }
        __syncthreads();
    }
}

// Groups of m rows of x in LDS, 68 bytes a row each: with the sums 64 KB, so that a compute unit has two workgroups.
u32 few_room(u32 m) { return 57344u / (68u * m); }
template <class X, class T>
void launch_few_of(const MxProduct &p, u32 cus, hipStream_t s) {
    const u32 room = std::min(p.groups, few_room(p.m));
    k_mx_few_rows_of<X, T><<<std::min((p.n + 15u) / 16u, 2u * cus), 512, room * p.m * 68u, s>>>(p, room);
}

template <class T, int TN, int TM, int WN, int WM, int KS>
void launch_tiles(const MxProduct &p, hipStream_t s) {
    using L = Tile<TN, TM, WN, WM, KS>;
    const u32 tiles = ((p.n + L::bn - 1) / L::bn) * ((p.m + L::bm - 1) / L::bm);
    k_mx_product<T, TN, TM, WN, WM, KS><<<tiles, L::threads, 0, s>>>(p);
}

void launch_part(const MxProduct &p, u32 cus, hipStream_t s) {
    // The largest tile that gives three workgroups in four compute units and more (a tile's rows are read once for the whole
    // of the other side); where there are no more of the smallest than compute units, four sets of waves a tile.  Measured,
    // m x n x k: 8192 x 8192 x 8192 in tiles of 256: 290 us; 4096 x 2048 x 8192 in 128 tiles of 256: 61 us, of 128: 49;
    // 1000 x 2000 x 3000 in tiles of 64: 10 us; 100 x 1024 x 11008 with four sets 18 us, with one 26, and 512 x 4096 x 4096,
    // 512 tiles, 13 us either way.  Of m no more than half of a tile is left empty (32 x 32000 x 4096 in tiles of 128: 22.4 us,
    // of 64: 18.7; 128 x 50304 x 2048 in tiles of 256: 23.5, of 128: 21.0; but 130 x 50304 x 4096: 39 and 51).  Up to 64 rows
    // are bound by the read of B, which two sets of waves keep going where it is long: 64 x 22016 x 4096 21.2 us with one and
    // 19.1 with two, 40 x 50304 x 4096 33.9 and 30.2, 60 x 50304 x 1024 9.1 and 11.5.
    auto tiles = [&](u32 n, u32 m) { return (u64)((p.n + n - 1u) / n) * ((p.m + m - 1u) / m); };
    with_type(p.type, [&](auto tag) {
        using T = decltype(tag);
        // (16 x 4096 x 4096: 6.1 us, in tiles 7.6; 16 x 50304 x 2048 in tiles 14 us, not in tiles 48)
        if (p.m <= 16u && p.n <= 32u * cus) k_mx_few_rows<T><<<(p.n + 15u) / 16u, 512, 0, s>>>(p);
        else if (p.m > 128u && tiles(256u, 256u) >= cus * 3 / 4) launch_tiles<T, 8, 4, 2, 4, 1>(p, s);
        else if (p.m > 64u && tiles(128u, 128u) >= cus * 3 / 4) launch_tiles<T, 4, 4, 2, 2, 1>(p, s);
        else if (p.m <= 64u && p.groups >= 32u && tiles(64u, 64u) > cus) launch_tiles<T, 2, 4, 2, 1, 2>(p, s);
        else if (tiles(64u, 64u) > cus) launch_tiles<T, 2, 2, 2, 2, 1>(p, s);
        else launch_tiles<T, 2, 2, 2, 2, 4>(p, s);
    });
}

}  // namespace

void launch_mx_product(const MxProduct &p, u32 cus, hipStream_t s) {
    // A launch has fewer than 2^32 threads; a tile has four for a row of its shorter side at most.  (What y can have besides, in
    // any memory there is, is far less.)
    constexpr u32 kMost = 1u << 28;
    for (u32 m = 0; m < p.m; m += kMost)
        for (u32 n = 0; n < p.n; n += kMost) {
            MxProduct part = p;
            part.m = std::min(kMost, p.m - m);
            part.n = std::min(kMost, p.n - n);
            part.a_codes += (u64)m * p.groups * 64u;
            part.a_scales += (u64)m * p.groups * 4u;
            part.b_codes += (u64)n * p.groups * 64u;
            part.b_scales += (u64)n * p.groups * 4u;
            part.y = (unsigned char *)p.y + ((u64)m * p.ld + n) * (p.type == ET_F32 ? 4u : 2u);
            launch_part(part, cus, s);
        }
}

bool mx_quantized_first(const MxProduct &p, u32 cus) {
    // Where x does not fit in LDS as a whole, it would be quantised again for every tile of sixteen rows of W (16 x 32000 x
    // 8192: 78 us in one launch, 36 in two; 16 x 4096 x 11008: 16.3 and 13.7); and where W's rows fill the GPU with tiles of 64,
    // those read it faster (8 x 22016 x 4096: 18.5 and 16.4; 16 x 50304 x 2048: 19.7 and 16.7), by more than the second launch
    // takes if there are more than four rows (4 x 22016 x 4096: 15.1 and 16.2; 1 x 50304 x 4096: 26.6 and 28.9).
    return p.groups > few_room(p.m) || (p.m > 4u && p.n >= 64u * cus);
}
void launch_mx_few_rows(const MxProduct &p, u32 cus, hipStream_t s) {
    with_type(p.x.type, [&](auto xtag) { with_type(p.type, [&](auto tag) { launch_few_of<decltype(xtag), decltype(tag)>(p, cus, s); }); });
}

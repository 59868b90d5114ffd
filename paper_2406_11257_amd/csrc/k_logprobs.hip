// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient.
//
// With m the largest logit of a row: s = sum exp(x - m), w = sum exp(x - m) (x - m); log p_i = x_i - m - log s, entropy =
// log s - w / s.  The sums go along with a running m, as each thread sees it, and are brought to a common one in the end.
// Both passes are bound by memory: the first reads a row once (4096 x 50304 in bf16: 76 us, 5.4 TB/s, the rate of a large read;
// 81 with 8 alternatives a row; rows with too many ties among those are read again, see row_part), the second reads and writes it once (169 us, 4.9 TB/s).
#include "excp_ops_device.h"

#include <type_traits>

namespace {

constexpr u32 kThreads = 256, kWaves = kThreads / 64u;
constexpr u32 kCandidates = 1024;      // alternatives that are ranked together
constexpr float kLog2e = 1.44269504088896341f, kLog2eRest = (float)(1.44269504088896341 - kLog2e), kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.402823466e38f;

// Sum and largest over a wave, in all lanes.
__device__ __forceinline__ float wave_sum_f32(float v) {
#define EXCP_MOVE(CTRL, ROWS) u2f(dpp_u32<CTRL, ROWS>(0u, f2u(v)))
    EXCP_WAVE_SCAN(v, EXCP_FOLD_ADD, EXCP_MOVE);
#undef EXCP_MOVE
    return u2f(last_lane_u32(f2u(v)));
}
__device__ __forceinline__ float wave_max_f32(float v) {
#define EXCP_FOLD_FMAX(v, x) (v = fmaxf(v, (x)))
#define EXCP_MOVE(CTRL, ROWS) u2f(dpp_u32<CTRL, ROWS>(0xff800000u, f2u(v)))
    EXCP_WAVE_SCAN(v, EXCP_FOLD_FMAX, EXCP_MOVE);
#undef EXCP_MOVE
#undef EXCP_FOLD_FMAX
    return u2f(last_lane_u32(f2u(v)));
}

// Statistics of part of a row: its largest unmasked logit (-inf: none), and over its elements, with that largest one (but
// not below the least finite number) as the shift, the sums of exp(x - shift) and of exp(x - shift) (x - shift).  A NaN or
// +inf makes the sums NaN.
struct Sums { float max, sum, weighted; };

// Sums with `max` m seen from a larger one.
__device__ __forceinline__ void lower(Sums &a, float max) {
    const float by = fmaxf(fmaxf(a.max, kLowest) - fmaxf(max, kLowest), -1000.0f), f = __builtin_amdgcn_exp2f(by * kLog2e);
    a.weighted = f * (a.weighted + by * a.sum);
    a.sum *= f;
    a.max = max;
}

// The order of alternatives: larger logits first, equal ones (both zeros are equal) by ascending index; 0 for what is none.
__device__ __forceinline__ u64 rank_key(float x, u32 i) {
    if (!(x > -INFINITY)) return 0;                          // masked, or NaN
    const u32 b = f2u(x + 0.0f);
    return (u64)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (u32)~i;
}
__device__ __forceinline__ float key_value(u64 key) {
    const u32 b = (u32)(key >> 32);
    return u2f(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ u32 key_index(u64 key) { return ~(u32)key; }

struct Room {
    Sums sums[kWaves];
    u32 value[kThreads], owner[kThreads], where[kThreads];
    u64 candidate[kCandidates], best[kWaves];
    u32 owners, candidates;
};

// The largest bound that at least k of a wave's R numbers a lane reach, or one that k reach exactly; 0 where fewer than k are
// not 0.  Bit by bit, from the highest in which the numbers' upper words (a 32-bit number's own) differ.
template <class N> __device__ __forceinline__ u32 upper_word(N v) { return (u32)(v >> (8 * sizeof(N) - 32)); }
// (Not below bit `last`: where the numbers have nothing there.)
template <int R, class N>
__device__ __forceinline__ N bound_of(const N (&v)[R], u32 k, int last = 0) {
    u32 most = 0, least = ~0u;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        most = max(most, upper_word(v[r]));
        least = min(least, upper_word(v[r]));
    }
    most = wave_max_u32(most);
    const u32 differ = most ^ wave_min_u32(least);
    const int below = 8 * (int)sizeof(N) - 32, high = differ ? 31 - __builtin_clz(differ) : -1;
    N t = high == 31 ? 0 : (N)(most >> (high + 1)) << (high + 1 + below);
    for (int b = high + below; b >= last; --b) {
        const N c = t | (N)1 << b;
        u32 n = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) n += (u32)__popcll(ballot64(v[r] >= c));
        if (n >= k) t = c;
        if (n == k) break;                                   // the same in every lane
    }
    return t;
}
// Number of `keys` above `key`.
__device__ __forceinline__ u32 above(const u64 *keys, u32 count, u64 key) {
    u32 n = 0;
#pragma unroll 4
    for (u32 i = 0; i < count; ++i) n += keys[i] > key;
    return n;
}
// The k (at most 64) first of `count` keys in LDS, no two alike: one a lane with its place among them, 0 in the other lanes.
// One wave; the keys are overwritten.
struct Placed { u64 key; u32 place; };
template <int R>
__device__ __forceinline__ u32 keep_first(u64 *keys, u32 count, u32 k) {
    const u32 lane = lane_id();
    u64 v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = r * 64u + lane < count ? keys[r * 64u + lane] : 0;
    const u64 least = max(bound_of(v, k), (u64)1);
    u32 n = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const u64 in = ballot64(v[r] >= least);
        if (v[r] >= least) keys[n + lanes_below(in)] = v[r];
        n += (u32)__popcll(in);
    }
    wave_lds_fence();
    return n;
}
__device__ __forceinline__ Placed first_of(u64 *keys, u32 count, u32 k) {
    wave_lds_fence();
    if (count > 256u) count = keep_first<kCandidates / 64>(keys, count, k);
    else if (count > 64u) count = keep_first<4>(keys, count, k);
    Placed r = {lane_id() < count ? keys[lane_id()] : 0, 0};
    r.place = above(keys, count, r.key);
    if (r.place >= k) r.key = 0;
    return r;
}
static_assert(EXCP_TOP_MAX <= 64, "a row's alternatives are one wave's");

// Statistics of pieces [begin, end) of eight elements of a row, in the first wave; and there, in `top`, its `ntop` first
// alternatives (key 0: none).
//
// Every thread keeps the piece that holds the largest of the logits that it has seen, and the largest of any other piece.  If
// ntop threads, or groups of threads, have seen a logit of at least b, then ntop logits are at least b, and what is below b is
// no alternative.  Groups of four threads give a bound that is little worse where alternatives are few beside them.  What
// reaches the bound is a candidate: out of the pieces kept, and where another piece of a thread has reached it too, out of all
// of its pieces, read again.
template <bool TOP, class T>
__device__ Sums row_part(const T *x, u32 vocab, u32 begin, u32 end, int ntop, Room &room, Placed &top) {
    constexpr u32 kUnroll = sizeof(T) == 2 ? 4 : 2;
    const u32 tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    Sums a = {-INFINITY, 0.0f, 0.0f};
    Eight<T> kept = {};
    float second = -INFINITY;
    u32 where = 0;
    auto take = [&](const Eight<T> &e, u32 piece) __attribute__((always_inline)) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = widen(e.v[i]);
        const float most = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
        if constexpr (TOP) second = fmaxf(second, fminf(most, a.max));
        if (most > a.max) {
            lower(a, most);
            if constexpr (TOP) {
                kept = e;
                where = piece;
            }
        }
        const float shift = fmaxf(a.max, kLowest);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = v[i] - shift, p = __builtin_amdgcn_exp2f(d * kLog2e);
            a.sum += p;
            a.weighted = __builtin_fmaf(p, fmaxf(d, -150.0f), a.weighted);     // (of a masked one: 0)
        }
    };
    u32 piece = begin + tid;
    for (; piece + (kUnroll - 1u) * kThreads < end && (piece + (kUnroll - 1u) * kThreads) * 8u + 8u <= vocab; piece += kUnroll * kThreads) {
        Eight<T> e[kUnroll];
#pragma unroll
        for (u32 q = 0; q < kUnroll; ++q) e[q] = load_eight(x + (u64)(piece + q * kThreads) * 8u, 8u);
#pragma unroll
        for (u32 q = 0; q < kUnroll; ++q) take(e[q], piece + q * kThreads);
    }
    for (; piece < end; piece += kThreads) {
        Eight<T> e = load_eight(x + (u64)piece * 8u, vocab - piece * 8u);
        if (vocab - piece * 8u < 8u) {
#pragma unroll
            for (u32 i = 0; i < 8; ++i)
                if (i >= vocab - piece * 8u) e.v[i] = (T)-INFINITY;
        }
        take(e, piece);
    }
    // the threads' sums together: of a wave, of the workgroup (in its first wave)
    const float mine = a.max;
    lower(a, wave_max_f32(a.max));
    a.sum = wave_sum_f32(a.sum);
    a.weighted = wave_sum_f32(a.weighted);
    if (lane == 0) room.sums[wave] = a;
    const u32 value = TOP ? (u32)(rank_key(mine, 0) >> 32) : 0u;
    const bool quads = ntop <= 24;
    constexpr int kLastBit = std::is_same<T, float>::value ? 0 : std::is_same<T, __bf16>::value ? 16 : 13;
    if (TOP) {
        u32 v = value;
        if (quads) {
            v = max(v, dpp_u32<0xb1, 0xf>(v, v));
            v = max(v, dpp_u32<0x4e, 0xf>(v, v));
            if ((lane & 3u) == 0) room.value[tid >> 2] = v;
        } else {
            room.value[tid] = v;
        }
        if (tid == 0) room.owners = room.candidates = 0;
    }
    __syncthreads();
    Sums all = room.sums[0];
    if (wave == 0) {
#pragma unroll
        for (u32 w = 1; w < kWaves; ++w) {
            Sums b = room.sums[w];
            const float m = fmaxf(all.max, b.max);
            lower(all, m);
            lower(b, m);
            all.sum += b.sum;
            all.weighted += b.weighted;
        }
    }
    top = {0, 0};
    if (!TOP) return all;
    u32 v[4] = {room.value[lane], 0u, 0u, 0u}, bound;
    if (quads) {
        const u32 one[1] = {v[0]};
        bound = bound_of(one, (u32)ntop, kLastBit);
    } else {
#pragma unroll
        for (u32 r = 1; r < 4; ++r) v[r] = room.value[r * 64u + lane];
        bound = bound_of(v, (u32)ntop, kLastBit);
    }
    bound = max(bound, 1u);
    const float reach = bound > 1u ? key_value((u64)bound << 32) : kLowest;
    auto add = [&](const Eight<T> &e, u32 piece) __attribute__((always_inline)) {
        u32 hits = 0;
#pragma unroll
        for (u32 j = 0; j < 8; ++j) hits |= (piece * 8u + j < vocab && widen(e.v[j]) >= reach ? 1u : 0u) << j;
        if (hits == 0u) return;
        u32 at = atomicAdd(&room.candidates, (u32)__builtin_popcount(hits));
#pragma unroll
        for (u32 j = 0; j < 8; ++j)
            if (hits >> j & 1u) {
                if (at < kCandidates) room.candidate[at] = rank_key(widen(e.v[j]), piece * 8u + j);
                ++at;
            }
    };
    if (value >= bound) {
        add(kept, where);
        if (second >= reach) {
            const u32 at = atomicAdd(&room.owners, 1u);
            room.owner[at] = tid;
            room.where[at] = where;
        }
    }
    __syncthreads();
    const u32 owners = room.owners, steps = (end - begin + kThreads - 1u) / kThreads;
    if (owners) {
        for (u32 i = tid; i < steps * owners; i += kThreads) {
            const u32 o = i % owners, p = begin + room.owner[o] + i / owners * kThreads;
            if (p < end && p != room.where[o]) add(load_eight(x + (u64)p * 8u, vocab - p * 8u), p);
        }
        __syncthreads();
    }
    const u32 count = room.candidates;
    if (count <= kCandidates) {
        if (wave == 0) top = first_of(room.candidate, count, (u32)ntop);
    } else {
        // too many for that (logits that are tied, or laid out so that a few threads hold all large ones): one after another, the
        // row read for each (4096 x 50304 zeros in bf16 with 8 alternatives: 1.12 ms, 84 us where they differ)
        u64 last = ~0ull;
        for (int j = 0; j < ntop; ++j) {
            u64 next = 0;
            for (u32 p = begin + tid; p < end; p += kThreads) {
                const Eight<T> e = load_eight(x + (u64)p * 8u, vocab - p * 8u);
#pragma unroll
                for (u32 i = 0; i < 8; ++i) {
                    const u64 k = p * 8u + i < vocab ? rank_key(widen(e.v[i]), p * 8u + i) : 0;
                    if (k < last && k > next) next = k;
                }
            }
            for (int d = 32; d; d >>= 1) next = max(next, shfl_xor_u64(next, d));
            if (lane == 0) room.best[wave] = next;
            __syncthreads();
            next = max(max(room.best[0], room.best[1]), max(room.best[2], room.best[3]));
            __syncthreads();
            if (lane == (u32)j) top = {next, (u32)j};
            last = next;
        }
    }
    return all;
}

// What a row's statistics come to.
template <class T>
__device__ void write_row(const RowScores &p, u32 row, const T *x, const Sums &a) {
    const bool bad = !(a.sum == a.sum), none = a.max == -INFINITY;
    const float logs = bad ? NAN : none ? 0.0f : logf(a.sum);
    if (p.lse) {
        p.lse[2 * (u64)row] = bad ? NAN : a.max;
        p.lse[2 * (u64)row + 1] = logs;
    }
    if (p.entropy) p.entropy[row] = bad ? NAN : none ? 0.0f : logs - a.weighted / a.sum;
    if (p.logprob) {
        const long long t = p.targets[row];
        float lp = 0.0f;
        if (t >= 0 && t < (long long)p.vocab) {
            const float v = widen(x[t]);
            lp = bad ? NAN : v == -INFINITY ? v : (v - a.max) - logs;
        }
        p.logprob[row] = lp;
    }
}
__device__ __forceinline__ void write_top(const RowScores &p, u32 row, u32 place, u64 key, const Sums &a) {
    const u64 o = (u64)row * p.ntop + place;
    if (p.top_ids) p.top_ids[o] = key ? (long long)key_index(key) : -1;
    if (p.top_logprob) p.top_logprob[o] = !(a.sum == a.sum) ? NAN : key ? (key_value(key) - a.max) - logf(a.sum) : -INFINITY;
}

// The first wave's alternatives, one a lane, and the places that none takes.
__device__ __forceinline__ void write_tops(const RowScores &p, u32 row, const Placed &top, const Sums &a) {
    const u32 lane = lane_id(), some = (u32)__popcll(ballot64(top.key != 0));
    if (top.key) write_top(p, row, top.place, top.key, a);
    if (lane >= some && lane < (u32)p.ntop) write_top(p, row, lane, 0, a);
}

// A workgroup a row, eight elements a thread and piece: a row of 32000 to 65536 is sixteen to thirty-two pieces a thread, whose
// partial maxima and sums are joined once.
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_row_scores(const RowScores p) {
    __shared__ Room room;
    for (u32 row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = (const T *)p.logits + (u64)row * p.ld;
        Placed top;
        const Sums a = row_part<TOP>(x, p.vocab, 0u, (p.vocab + 7u) / 8u, p.ntop, room, top);
        if (threadIdx.x == 0) write_row(p, row, x, a);
        if (TOP && threadIdx.x < 64u) write_tops(p, row, top, a);
        __syncthreads();
    }
}

// Few rows: `parts` workgroups a row.  The last of a row's to finish, by ticket, joins what they found.  (Parts pass through
// memory as relaxed atomics of the device, which have arrived before the ticket is drawn.  One row of 50304 floats with 20
// alternatives: 10.7 us, waits one after the other and not bytes.)
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_row_scores_split(const RowScores p, u32 parts, u32 per, RowPart *__restrict__ out, u32 *__restrict__ tickets) {
    __shared__ Room room;
    __shared__ u32 ticket;
    const u32 row = blockIdx.x / parts, part = blockIdx.x - row * parts, all = (p.vocab + 7u) / 8u;
    const T *x = (const T *)p.logits + (u64)row * p.ld;
    RowPart &mine = out[blockIdx.x];
    Placed top;
    const Sums a = row_part<TOP>(x, p.vocab, min(part * per, all), min(part * per + per, all), p.ntop, room, top);
    if (TOP && threadIdx.x < 64u) {
        const u32 lane = lane_id(), some = (u32)__popcll(ballot64(top.key != 0));
        if (top.key) __hip_atomic_store(&mine.key[top.place], top.key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (lane >= some && lane < (u32)p.ntop) __hip_atomic_store(&mine.key[lane], (u64)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (threadIdx.x == 0) {
        __hip_atomic_store(&mine.max, a.max, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&mine.sum, a.sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&mine.weighted, a.weighted, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) ticket = atomicAdd(&tickets[row], 1u);
    __syncthreads();
    if (ticket != parts - 1u) return;
    if (threadIdx.x == 0) tickets[row] = 0u;                 // for the next call
    const RowPart *in = out + row * parts;
    Sums b = {-INFINITY, 0.0f, 0.0f};
    const u32 lane = lane_id();
    if (lane < parts) {                                      // (at most 64)
        b.max = __hip_atomic_load(&in[lane].max, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        b.sum = __hip_atomic_load(&in[lane].sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        b.weighted = __hip_atomic_load(&in[lane].weighted, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    lower(b, wave_max_f32(b.max));
    b.sum = wave_sum_f32(b.sum);
    b.weighted = wave_sum_f32(b.weighted);
    if (threadIdx.x == 0) write_row(p, row, x, b);
    if (!TOP) return;
    const u32 i = threadIdx.x;                               // (no more keys than there are threads)
    const u64 key = i < parts * (u32)p.ntop ? __hip_atomic_load(&in[i / (u32)p.ntop].key[i % (u32)p.ntop], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    if (i == 0) room.candidates = 0;
    __syncthreads();
    if (key) room.candidate[atomicAdd(&room.candidates, 1u)] = key;
    __syncthreads();
    if (i < 64u) write_tops(p, row, first_of(room.candidate, room.candidates, (u32)p.ntop), b);
}

// exp(d) for d from -150 to 0.  What rounds d log2(e) is d times 2^-24 of the result, up to 80 units of its last place, and is made
// good.  (The sums above do without: a term's error counts by its share of the sum.)
__device__ __forceinline__ float exp_below(float d) {
    const float t = d * kLog2e, e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e * kLn2, __builtin_fmaf(d, kLog2eRest, __builtin_fmaf(d, kLog2e, -t)), e);
}

// d = -p (weight + g_entropy (log p + entropy)), and at the target and the alternatives their own weights besides.  A
// workgroup has `chunks` chunks of a row, of eight elements a thread; the first is on its way before it asks for the row's
// weights.  (More at a time gain nothing: 4096 x 50304 in bf16, 824 MB, takes 169 us either way, and a copy of as much 162.)
// Lane j of every wave knows alternative j; whose piece it lies in adds its weight.
//
// Whether a target is masked is read from the logits.  Where the gradient takes their place, a row is one workgroup's, which
// has read that before it writes.
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_row_gradient(const RowGradient p, u32 parts, u32 chunks, u64 items) {
    constexpr u32 kNone = ~0u;
    const u32 tid = threadIdx.x, lane = tid & 63u, all = (p.vocab + 7u) / 8u;
    for (u64 item = blockIdx.x; item < items; item += gridDim.x) {
        const u32 row = (u32)(item / parts), part = (u32)(item - (u64)row * parts);
        const T *x = (const T *)p.logits + (u64)row * p.ld;
        T *d = (T *)p.d + (u64)row * p.ldd;
        const u32 stop = (u32)min((u64)(part + 1u) * chunks * kThreads, (u64)all);
        u32 begin = part * chunks * kThreads;
        Eight<T> e;
        auto load = [&]() __attribute__((always_inline)) {
            const u32 i = begin + tid;
            if (i < stop) e = load_eight(x + (u64)i * 8u, p.vocab - i * 8u);
        };
        load();
        float shift = p.lse[2 * (u64)row], logs = p.lse[2 * (u64)row + 1];
        float ge = p.g_entropy ? p.g_entropy[row] : 0.0f, h = p.g_entropy ? p.entropy[row] : 0.0f;
        const long long t = p.g_logprob ? p.targets[row] : -1;
        float g_target = p.g_logprob ? p.g_logprob[row] : 0.0f, g_also = 0.0f;
        u32 target = t >= 0 && t < (long long)p.vocab ? (u32)t : kNone, also = kNone;
        if (target != kNone && widen(x[target]) == -INFINITY) target = kNone;   // takes no part
        if (target == kNone) g_target = 0.0f;
        float weight = g_target;
        if constexpr (TOP) {
            if (lane < (u32)p.ntop) {
                const long long i = p.top_ids[(u64)row * p.ntop + lane];
                const float g = p.g_top[(u64)row * p.ntop + lane];
                if (i >= 0 && i < (long long)p.vocab && widen(x[i]) != -INFINITY) {
                    also = (u32)i;
                    g_also = g;
                }
            }
            weight += wave_sum_f32(g_also);
        }
        if (p.logits == p.d) __syncthreads();
        if (shift == -INFINITY) shift = logs = weight = ge = h = 0.0f;          // nothing unmasked: every p is 0
        // Of floats, p = exp(x - max) / sum, to its own last places; of 16-bit types, whose results have fewer, exp(log p), which
        // takes less (2048 x 50304 floats: 172 us either way; 4096 x 50304 in bf16 168 to 170, and 171 to 175 the longer way).
        constexpr bool kFloats = sizeof(T) == 4;
        const float share = kFloats ? expf(-logs) : 1.0f, from_max = kFloats ? h - logs : h;
        for (;;) {
            const u32 i = begin + tid;
            float v[8];
#pragma unroll
            for (u32 j = 0; j < 8; ++j) {
                const float below = widen(e.v[j]) - shift;
                if constexpr (kFloats) {
                    const float off = fmaxf(below, -150.0f);                    // (a masked one's p is 0)
                    v[j] = -(exp_below(off) * share) * __builtin_fmaf(ge, off + from_max, weight);
                } else {
                    const float logp = below - logs, prob = __builtin_amdgcn_exp2f(logp * kLog2e);
                    v[j] = -prob * __builtin_fmaf(ge, fmaxf(logp, -150.0f) + from_max, weight);
                }
            }
            if (i == target / 8u) {
#pragma unroll
                for (u32 j = 0; j < 8; ++j) v[j] += j == (target & 7u) ? g_target : 0.0f;
            }
            if constexpr (TOP) {
                for (u64 here = ballot64(also / 8u - (i - lane) < 64u); here; here &= here - 1u) {
                    const int from = (int)__ffsll((long long)here) - 1;
                    const u32 at = (u32)__builtin_amdgcn_readlane((int)also, from);
                    const float w = u2f((u32)__builtin_amdgcn_readlane((int)f2u(g_also), from));
#pragma unroll
                    for (u32 j = 0; j < 8; ++j) v[j] += i * 8u + j == at ? w : 0.0f;
                }
            }
            Eight<T> r;
#pragma unroll
            for (u32 j = 0; j < 8; ++j) r.v[j] = (T)v[j];
            if (i < stop) store_eight(d + (u64)i * 8u, r, p.vocab - i * 8u);
            begin += kThreads;
            if (begin >= stop) break;
            load();
        }
    }
}

}  // namespace

void launch_row_scores(const RowScores &r, const OpsContext &c) {
    // Several workgroups a row where there are more compute units than rows, of two pieces a thread and more.  (256 rows of
    // 50304 in bf16 with 8 alternatives: 12.5 us whole, 13.7 in two parts; one row of fp32 with 20: 10.7 us in twelve parts.)
    const u32 pieces = (r.vocab + 7u) / 8u;
    u32 parts = std::min(c.cus / r.rows, (pieces + 2u * kThreads - 1u) / (2u * kThreads));
    parts = std::min(parts, r.ntop ? std::min(64u, kThreads / (u32)r.ntop) : 64u);
    parts = std::max(std::min(parts, EXCP_ROW_PARTS / r.rows), 1u);
    const u32 per = (pieces + parts - 1u) / parts;
    with_type(r.type, [&](auto tag) {
        using T = decltype(tag);
        const u32 rows = std::min(r.rows, 1u << 20);
        if (parts == 1u && r.ntop) k_row_scores<T, true><<<rows, kThreads, 0, c.stream>>>(r);
        else if (parts == 1u) k_row_scores<T, false><<<rows, kThreads, 0, c.stream>>>(r);
        else if (r.ntop) k_row_scores_split<T, true><<<r.rows * parts, kThreads, 0, c.stream>>>(r, parts, per, c.parts, c.tickets);
        else k_row_scores_split<T, false><<<r.rows * parts, kThreads, 0, c.stream>>>(r, parts, per, c.parts, c.tickets);
    });
}

void launch_row_gradient(const RowGradient &r, u32 cus, hipStream_t s) {
    const u32 pieces = (r.vocab + 7u) / 8u, all = (pieces + kThreads - 1u) / kThreads;
    // a row a workgroup where that fills the compute units; else a row's chunks are shared out
    const u32 share = r.logits == r.d ? 1u : std::min(all, std::max(1u, 8u * cus / r.rows));
    const u32 chunks = (all + share - 1u) / share, parts = (all + chunks - 1u) / chunks;
    const u64 items = (u64)r.rows * parts;
    const u32 grid = (u32)std::min<u64>(items, 1u << 20);
    with_type(r.type, [&](auto tag) {
        using T = decltype(tag);
        if (r.ntop) k_row_gradient<T, true><<<grid, kThreads, 0, s>>>(r, parts, chunks, items);
        else k_row_gradient<T, false><<<grid, kThreads, 0, s>>>(r, parts, chunks, items);
    });
}

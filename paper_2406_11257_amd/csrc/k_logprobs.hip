// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient.
//
// Both passes are bound by memory: the first reads a row once, the second reads and writes it once.
#include "excp_ops_device.h"

namespace {

constexpr u32 kThreads = 256, kWaves = kThreads / 64u;
constexpr u32 kCandidates = 1024;      // alternatives that are ranked together
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLowest = -3.402823466e38f;

// Sum and largest over a workgroup, in all threads; `room` is used again after the next barrier of the caller only.
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
    u32 group[64], owner[kThreads];
    u64 key[kThreads], candidate[kCandidates], best[kWaves], least;
    u32 thread[EXCP_TOP_MAX], keys, candidates;
};

// Number of `keys` above `key`.
__device__ __forceinline__ u32 above(const u64 *keys, u32 count, u64 key) {
    u32 n = 0;
#pragma unroll 8
    for (u32 i = 0; i < count; ++i) n += keys[i] > key;
    return n;
}
// put(place, key) for the `ntop` first of `count` keys, no two alike but zeros (what is none), and put(place, 0) for places
// that none takes.
template <class Put>
__device__ void rank_all(const u64 *keys, u32 count, int ntop, Put put) {
    u32 some = 0;
    for (u32 i = threadIdx.x; i - threadIdx.x < count; i += kThreads) {
        const u64 key = i < count ? keys[i] : 0;
        some += (u32)__syncthreads_count(key != 0);
        const u32 rank = key ? above(keys, count, key) : ~0u;
        if (rank < (u32)ntop) put(rank, key);
    }
    if (threadIdx.x >= some && threadIdx.x < (u32)ntop) put(threadIdx.x, 0);
}
static_assert(EXCP_TOP_MAX <= 64, "one wave writes a row's alternatives");

// Statistics of pieces [begin, end) of eight elements of a row, in the first wave; and its `ntop` first alternatives by
// put(place, key).
//
// Every thread keeps the largest of the logits that it has seen and the piece that held it.  The row's first ntop
// alternatives are all among the logits of the ntop threads whose largest ones come first: before one in another thread
// would come those ntop.  So only those threads' pieces are read again, out of the caches, and of them only what does not
// come after the last of those ntop is ranked.
template <class T, class Put>
__device__ Sums row_part(const T *x, u32 vocab, u32 begin, u32 end, int ntop, Room &room, Put put) {
    constexpr u32 kUnroll = sizeof(T) == 2 ? 4 : 2;
    const u32 tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    Sums a = {-INFINITY, 0.0f, 0.0f};
    u32 where = 0;
    auto take = [&](const Eight<T> &e, u32 piece) __attribute__((always_inline)) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = widen(e.v[i]);
        const float most = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
        if (most > a.max) {
            lower(a, most);
            where = piece;
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
    // A bound for the threads' largest logits: of those of groups of threads the one at place ntop.
    const u64 key = ntop ? rank_key(mine, where) : 0;
    const bool small = ntop <= 8;                            // (groups of sixteen lanes, sixteen groups: a quarter of the comparisons)
    if (ntop) {
        u32 v = (u32)(key >> 32);
        v = max(v, dpp_u32<0xb1, 0xf>(v, v));                // the other three of four lanes
        v = max(v, dpp_u32<0x4e, 0xf>(v, v));
        if (small) {
            v = max(v, dpp_u32<0x124, 0xf>(v, v));           // and of sixteen
            v = max(v, dpp_u32<0x128, 0xf>(v, v));
            if ((lane & 15u) == 0) room.group[tid >> 4] = v;
        } else if ((lane & 3u) == 0) {
            room.group[tid >> 2] = v;
        }
        if (tid < (u32)ntop) room.thread[tid] = ~0u;
        if (tid == 0) {
            room.keys = 0;
            room.candidates = 0;
            room.least = 1;
        }
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
    if (!ntop) return all;
    const u32 groups = small ? 16u : 64u, group = lane < groups ? room.group[lane] : 0u;
    u32 place = 0;
#pragma unroll 4
    for (u32 i = 0; i < groups; ++i) {
        const u32 v = room.group[i];
        place += v > group || (v == group && i < lane);
    }
    const u64 holds = ballot64(lane < groups && place == (u32)ntop - 1u);
    const u32 bound = max(1u, (u32)__builtin_amdgcn_readlane((int)group, (int)__ffsll((long long)holds) - 1));
    const bool is_key = (u32)(key >> 32) >= bound;
    const u64 with = ballot64(is_key);
    if (with) {
        u32 at = 0;
        if (lane == 0) at = atomicAdd(&room.keys, (u32)__popcll(with));
        at = (u32)__builtin_amdgcn_readfirstlane((int)at) + lanes_below(with);
        if (is_key) {
            room.key[at] = key;
            room.owner[at] = tid;
        }
    }
    __syncthreads();
    const u32 keys = room.keys;
    if (tid < keys) {
        const u64 k = room.key[tid];
        const u32 rank = above(room.key, keys, k);
        if (rank < (u32)ntop) room.thread[rank] = room.owner[tid];
        if (rank == (u32)ntop - 1u) room.least = k & ~0xffffffffull;            // its value; the piece's number is no index
    }
    __syncthreads();
    // what may be among the first, of the pieces of those threads
    const u64 least = room.least;
    const u32 steps = (end - begin + kThreads - 1u) / kThreads;
    for (u32 i = tid; i < steps * (u32)ntop; i += kThreads) {
        const u32 who = room.thread[i % (u32)ntop], p = begin + who + i / (u32)ntop * kThreads;
        if (who == ~0u || p >= end) continue;
        const Eight<T> e = load_eight(x + (u64)p * 8u, vocab - p * 8u);
#pragma unroll
        for (u32 j = 0; j < 8; ++j) {
            const u64 k = p * 8u + j < vocab ? rank_key(widen(e.v[j]), p * 8u + j) : 0;
            if (k >= least) {
                const u32 at = atomicAdd(&room.candidates, 1u);
                if (at < kCandidates) room.candidate[at] = k;
            }
        }
    }
    __syncthreads();
    const u32 count = room.candidates;
    if (count <= kCandidates) {
        rank_all(room.candidate, count, ntop, put);
    } else {
        // too many for that (logits that are tied, or laid out so that a few threads hold all large ones): one after another
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
            if (tid == 0) put((u32)j, next);
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

// A workgroup a row.
template <class T>
__global__ __launch_bounds__(kThreads) void k_row_scores(const RowScores p) {
    __shared__ Room room;
    __shared__ u64 first[EXCP_TOP_MAX];
    for (u32 row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = (const T *)p.logits + (u64)row * p.ld;
        const Sums a = row_part(x, p.vocab, 0u, (p.vocab + 7u) / 8u, p.ntop, room, [&](u32 place, u64 key) { first[place] = key; });
        if (threadIdx.x == 0) write_row(p, row, x, a);
        __syncthreads();
        for (u32 i = threadIdx.x; i < (u32)p.ntop; i += kThreads) write_top(p, row, i, first[i], a);
        __syncthreads();
    }
}

// Few rows: `parts` workgroups a row.  The last of a row's to finish, by ticket, joins what they found.  (Parts pass through
// memory as relaxed atomics of the device, which have arrived before the ticket is drawn.)
template <class T>
__global__ __launch_bounds__(kThreads) void k_row_scores_split(const RowScores p, u32 parts, u32 per, RowPart *__restrict__ out, u32 *__restrict__ tickets) {
    __shared__ Room room;
    __shared__ u32 ticket;
    const u32 row = blockIdx.x / parts, part = blockIdx.x - row * parts, all = (p.vocab + 7u) / 8u;
    const T *x = (const T *)p.logits + (u64)row * p.ld;
    RowPart &mine = out[blockIdx.x];
    const Sums a = row_part(x, p.vocab, min(part * per, all), min(part * per + per, all), p.ntop, room, [&](u32 place, u64 key) {
        __hip_atomic_store(&mine.key[place], key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
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
    if (!p.ntop) return;
    const u32 count = parts * (u32)p.ntop;                   // (no more than there are threads)
    for (u32 i = threadIdx.x; i < count; i += kThreads)
        room.candidate[i] = __hip_atomic_load(&in[i / (u32)p.ntop].key[i % (u32)p.ntop], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    rank_all(room.candidate, count, p.ntop, [&](u32 place, u64 key) { write_top(p, row, place, key, b); });
}

// d = -p (weight + g_entropy (log p + entropy)), and at the target and the alternatives their own weights besides.  A
// workgroup has `chunks` chunks of a row, of eight elements a thread; the first is on its way before it asks for the row's
// weights.  (More at a time, from 2 x 8 elements a thread on, are slower: 199 us against 170 for 4096 x 50304 in bf16, whose
// 824 MB a copy moves in 162.)  Lane j of every wave knows alternative j; whose piece it lies in adds its weight.
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
        for (;;) {
            const u32 i = begin + tid;
            float v[8];
#pragma unroll
            for (u32 j = 0; j < 8; ++j) {
                const float logp = (widen(e.v[j]) - shift) - logs, prob = __builtin_amdgcn_exp2f(logp * kLog2e);
                v[j] = -prob * __builtin_fmaf(ge, fmaxf(logp, -150.0f) + h, weight);
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
    // Several workgroups a row where there are too few rows for all compute units, of pieces worth a workgroup each.
    const u32 pieces = (r.vocab + 7u) / 8u;
    u32 parts = r.rows < 2u * c.cus ? std::min((2u * c.cus + r.rows - 1u) / r.rows, (pieces + kThreads - 1u) / kThreads) : 1u;
    parts = std::min(parts, r.ntop ? std::min(64u, kThreads / (u32)r.ntop) : 64u);
    parts = std::min(parts, std::max(1u, EXCP_ROW_PARTS / r.rows));
    parts = std::max(parts, 1u);
    const u32 per = (pieces + parts - 1u) / parts;
    with_type(r.type, [&](auto tag) {
        using T = decltype(tag);
        if (parts == 1u) k_row_scores<T><<<std::min(r.rows, 1u << 20), kThreads, 0, c.stream>>>(r);
        else k_row_scores_split<T><<<r.rows * parts, kThreads, 0, c.stream>>>(r, parts, per, c.parts, c.tickets);
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

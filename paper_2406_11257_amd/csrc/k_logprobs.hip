// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient.
#include "excp_ops_device.h"

struct RowPart { float max, sum, weighted; };

namespace {

constexpr u32 kThreads = 256;

__device__ float block_max(float v, float *room) {
    const u32 lane = lane_id(), wave = threadIdx.x >> 6;
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, WAVE));
    if (lane == 0) room[wave] = v;
    __syncthreads();
    v = fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3]));
    __syncthreads();
    return v;
}
__device__ float block_sum(float v, float *room) {
    const u32 lane = lane_id(), wave = threadIdx.x >> 6;
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, WAVE);
    if (lane == 0) room[wave] = v;
    __syncthreads();
    v = (room[0] + room[1]) + (room[2] + room[3]);
    __syncthreads();
    return v;
}
// The order of alternatives: larger logits first, equal ones by ascending index; 0 for what is none.
__device__ __forceinline__ u64 rank_key(float x, u32 i) {
    if (!(x > -INFINITY)) return 0;               // masked, or NaN
    if (x == 0.0f) x = 0.0f;                      // both zeros are equal
    const u32 b = f2u(x);
    return (u64)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (u32)~i;
}

// One workgroup a row, read as often as needed.
template <class T>
__global__ __launch_bounds__(kThreads) void k_row_scores(const RowScores p) {
    __shared__ float room[4];
    __shared__ u64 best[4];
    for (u32 row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T *x = (const T *)p.logits + (u64)row * p.ld;
    float top = -INFINITY;
    bool nan = false;
    for (u32 i = threadIdx.x; i < p.vocab; i += kThreads) { const float v = widen(x[i]); nan |= v != v; top = fmaxf(top, v); }
    nan = __syncthreads_or(nan);
    top = block_max(top, room);
    const float shift = top > -INFINITY ? top : 0.0f;
    float s = 0, w = 0;
    for (u32 i = threadIdx.x; i < p.vocab; i += kThreads) {
        const float d = widen(x[i]) - shift, e = __expf(d);
        s += e;
        if (e > 0.0f) w += e * d;
    }
    s = block_sum(s, room);
    w = block_sum(w, room);
    const bool none = top == -INFINITY && !nan, bad = nan || top == INFINITY;
    const float logs = none ? 0.0f : logf(s);
    if (threadIdx.x == 0) {
        if (p.lse) { p.lse[2 * (u64)row] = bad ? NAN : top; p.lse[2 * (u64)row + 1] = bad ? NAN : logs; }
        if (p.entropy) p.entropy[row] = bad ? NAN : none ? 0.0f : logs - w / s;
        if (p.logprob) {
            const long long t = p.targets[row];
            float lp = 0.0f;
            if (t >= 0 && t < (long long)p.vocab) {
                const float v = widen(x[t]);
                lp = bad ? NAN : v == -INFINITY ? v : (v - shift) - logs;
            }
            p.logprob[row] = lp;
        }
    }
    u64 last = ~0ull;
    for (int j = 0; j < p.ntop; ++j) {
        u64 key = 0;
        for (u32 i = threadIdx.x; i < p.vocab; i += kThreads) { const u64 k = rank_key(widen(x[i]), i); if (k < last && k > key) key = k; }
        for (int d = 32; d; d >>= 1) key = max(key, shfl_xor_u64(key, d));
        if (lane_id() == 0) best[threadIdx.x >> 6] = key;
        __syncthreads();
        key = max(max(best[0], best[1]), max(best[2], best[3]));
        __syncthreads();
        if (threadIdx.x == 0) {
            const u32 i = ~(u32)key;
            const u64 o = (u64)row * p.ntop + j;
            if (p.top_ids) p.top_ids[o] = key ? (long long)i : -1;
            if (p.top_logprob) p.top_logprob[o] = bad ? NAN : key ? (widen(x[i]) - shift) - logs : -INFINITY;
        }
        last = key;
    }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_row_gradient(const RowGradient p) {
    for (u32 row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const T *x = (const T *)p.logits + (u64)row * p.ld;
        T *d = (T *)p.d + (u64)row * p.ldd;
        const float shift = p.lse[2 * (u64)row], logs = p.lse[2 * (u64)row + 1];
        float gl = 0.0f, weight = 0.0f, ge = 0.0f, h = 0.0f;
        long long t = -1;
        if (p.g_logprob) {
            t = p.targets[row];
            if (t < 0 || t >= (long long)p.vocab || widen(x[t]) == -INFINITY) t = -1;
            else weight = gl = p.g_logprob[row];
        }
        for (int j = 0; j < p.ntop; ++j) if (p.top_ids[(u64)row * p.ntop + j] >= 0) weight += p.g_top[(u64)row * p.ntop + j];
        if (p.g_entropy) { ge = p.g_entropy[row]; h = p.entropy[row]; }
        for (u32 i = blockIdx.x * kThreads + threadIdx.x; i < p.vocab; i += gridDim.x * kThreads) {
            float v = 0.0f;
            if (shift != -INFINITY) {
                const float logp = (widen(x[i]) - shift) - logs, q = __expf(logp);
                v = q == 0.0f ? 0.0f : -q * (weight + ge * (logp + h));
                if ((long long)i == t) v += gl;
                for (int j = 0; j < p.ntop; ++j) if (p.top_ids[(u64)row * p.ntop + j] == (long long)i) v += p.g_top[(u64)row * p.ntop + j];
            }
            d[i] = (T)v;
        }
    }
}

}  // namespace

void launch_row_scores(const RowScores &r, const OpsContext &c) {
    with_type(r.type, [&](auto tag) { k_row_scores<decltype(tag)><<<std::min(r.rows, 1u << 20), kThreads, 0, c.stream>>>(r); });
}

void launch_row_gradient(const RowGradient &r, u32 cus, hipStream_t s) {
    const dim3 grid(std::min((r.vocab + kThreads - 1) / kThreads, 64u), std::min(r.rows, 65535u));
    with_type(r.type, [&](auto tag) { k_row_gradient<decltype(tag)><<<grid, kThreads, 0, s>>>(r); });
}

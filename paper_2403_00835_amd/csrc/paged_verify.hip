// Verification of drafted tokens on gfx950: how many of a request's tokens stand against the target's distribution, and the
// token that follows them.
//
// Row r of a request holds the target's logits behind tokens[r]; tokens[r + 1] is its draft. With p = softmax(l / T) and q the
// draft's distribution (a point mass where there are no draft logits), the draft x stands where u q(x) < p(x). At the first
// row whose draft does not stand, the next token is drawn from max(p - q, 0); behind the last row, from p: the tokens
// then have the target's distribution. A token is drawn as the lowest index whose running sum is above u times the sum.
//
// Every weight 2^((l - max) log2(e) / T) and every sum is in 64 bits: a draw among V tokens picks the neighbour with a
// probability of about V times the sums' relative error, which in 32 bits is one in some hundred draws.
#include <algorithm>

#include "device.h"
#include "paged.h"

namespace cllm {

namespace {

constexpr int kThreads = 256, kPer = kVerifyChunk / kThreads;  // of the statistics' workgroups; logits a thread
constexpr int kDecide = 512;                                   // threads of the workgroups that decide

// 2^(j / 32)
__constant__ double kExpTable[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0};

// 2^d for d <= 0 (below 2^-1000: 0): 2^(k / 32) from the table (LDS) times 2^r, |r| <= 1 / 64, by its Taylor polynomial,
// whose first term left out is 2e-18 of it.
__device__ __forceinline__ double exp2_wide(double d, const double *table) {
    constexpr double kRound = 0x1.8p47;  // its last place is 1 / 32
    const double dc = fmax(d, -1000.0), t = dc + kRound, r = dc - (t - kRound);
    const int k = (int)__builtin_bit_cast(uint64_t, t);  // 32 dc, rounded
    double y = 0x1.430912f86c787p-13;
    y = __builtin_fma(y, r, 0x1.5d87fe78a6731p-10);
    y = __builtin_fma(y, r, 0x1.3b2ab6fba4e77p-7);
    y = __builtin_fma(y, r, 0x1.c6b08d704a0c0p-5);
    y = __builtin_fma(y, r, 0x1.ebfbdff82c58fp-3);
    y = __builtin_fma(y, r, 0x1.62e42fefa39efp-1);
    y = __builtin_fma(y, r, 1.0);
    const uint64_t w = __builtin_bit_cast(uint64_t, y * table[k & 31]) + ((uint64_t)(uint32_t)(k >> 5) << 52);
    return d < -1000.0 ? 0.0 : __builtin_bit_cast(double, w);
}

typedef u32x4 u32x4_any __attribute__((aligned(2)));

// N logits from any element's address; past the row's end -inf.
template <Prec PR, int N>
__device__ __forceinline__ void load_logits(float (&x)[N], const typename PrecT<PR>::T *row, int i, int vocab) {
    using T = typename PrecT<PR>::T;
    constexpr int VEC = PrecT<PR>::VEC;
    static_assert(N % VEC == 0, "whole vectors");
#pragma unroll
    for (int v = 0; v < N; v += VEC) {
        alignas(16) T e[VEC];
        if (i + v + VEC <= vocab) {
            *reinterpret_cast<u32x4 *>(e) = *reinterpret_cast<const u32x4_any *>(row + i + v);
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[v + k] = from_elem<PR>(e[k]);
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[v + k] = i + v + k < vocab ? from_elem<PR>(row[i + v + k]) : -INFINITY;
        }
    }
}

// The request of a row: the last one that starts at or before it (a wave's two reads; n up to 1024).
__device__ __forceinline__ int request_of(const int32_t *row_start, int n, int row) {
    const int lane = threadIdx.x & 63;
    const uint64_t far = __ballot(16 * lane < n && row_start[min(16 * lane, n)] <= row);
    const int c = 16 * max((int)__popcll(far) - 1, 0);  // (a row before the first request is counted to that)
    const uint64_t near = __ballot(lane < 16 && c + lane < n && row_start[min(c + lane, n)] <= row);
    return min(c + max((int)__popcll(near) - 1, 0), n - 1);
}

// Weights are 2^((l - max) scale); 0: the greedy choice. Not a temperature: -1.
__device__ __forceinline__ double weight_scale(float temperature) {
    return temperature == 0.0f ? 0.0 : temperature > 0.0f && temperature < INFINITY ? 1.4426950408889634 / (double)temperature : -1.0;
}

// The larger value, of equal ones the lower index. (A NaN is kept apart.)
__device__ __forceinline__ void take_larger(float &m, int &at, float m2, int at2) {
    const bool other = m2 > m || (m2 == m && at2 < at);
    m = other ? m2 : m;
    at = other ? at2 : at;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
    return x;
}

// Sum over the workgroup, the same in every thread, in a fixed order. s: one word a wave.
__device__ __forceinline__ double block_sum(double x, double *s) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    double t = 0.0;
    for (int w = 0; w < (int)blockDim.x / kWave; ++w) t += s[w];
    return t;
}

__device__ __forceinline__ void load_table(double *table) {
    if (threadIdx.x < 32) table[threadIdx.x] = kExpTable[threadIdx.x];
    __syncthreads();
}

// A row's distribution from the statistics of its chunks, by one wave: the same in every lane.
struct Law {
    float max;
    double sum;  // of the weights
    int top;     // the largest logit's lowest index
    bool ok;     // neither NaN nor +inf among the logits, nor all -inf
};
__device__ __forceinline__ Law row_law(const VerifyStat *st, int chunks, double scale, const double *table) {
    const int lane = threadIdx.x & 63;
    Law w{-INFINITY, 0.0, 0x7fffffff, true};
    bool bad = false;
    for (int c = lane; c < chunks; c += kWave) {
        const VerifyStat s = st[c];
        bad |= s.max != s.max;
        take_larger(w.max, w.top, s.max, s.top);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) take_larger(w.max, w.top, __shfl_xor(w.max, off), __shfl_xor(w.top, off));
    w.ok = !__any(bad) && w.max > -INFINITY && w.max < INFINITY;
    if (!w.ok || scale <= 0.0) return w;
    double sum = 0.0;
    for (int c = lane; c < chunks; c += kWave) {
        const VerifyStat s = st[c];
        sum += s.sum * exp2_wide(((double)s.max - (double)w.max) * scale, table);
    }
    w.sum = wave_sum(sum);
    return w;
}

// Where a request stops: its row, and whether that row's draft was refused.
struct Stop {
    int first, last;  // its rows
    int row;
    bool refused;
    int draft;        // the refused token where it is one of the vocabulary, or -1
    double scale;
    Law p, q;         // of the row; q with draft logits and a refused draft
};

// By the whole workgroup. False where the request has no rows.
template <Prec PR>
__device__ __forceinline__ bool decide(const VerifyParams &p, int b, const double *table, int *s_stop, Stop &d) {
    using T = typename PrecT<PR>::T;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x / kWave;
    int first = p.row_start[b], end = p.row_start[b + 1];
    if (p.status && (p.status[PS_ROWS] == 0 || b >= p.status[PS_ENTRIES])) first = end = 0;  // a refused plan
    if (first < 0 || end > p.rows || first >= end) return false;  // uniform
    d.first = first;
    d.last = end - 1;
    d.scale = weight_scale(p.temperature[b]);
    const int chunks = p.chunks;
    if (threadIdx.x == 0) *s_stop = end - 1;
    __syncthreads();
    for (int r0 = first; r0 < end - 1; r0 += waves) {
        const int r = r0 + w;
        if (r < end - 1) {
            const int x = p.tokens[r + 1];
            const bool known = x >= 0 && x < p.vocab;
            const double u = p.accept_u[r];
            const float lp = known ? from_elem<PR>(((const T *)p.logits)[(size_t)r * p.stride + x]) : -INFINITY;
            const float lq = known && p.draft ? from_elem<PR>(((const T *)p.draft)[(size_t)r * p.draft_stride + x]) : 0.f;
            const Law law = row_law(p.stats + (size_t)r * chunks, chunks, d.scale, table);
            bool stands = false;
            if (law.ok && d.scale == 0.0) {
                stands = x == law.top;
            } else if (law.ok && d.scale > 0.0 && known) {
                const double px = exp2_wide(((double)lp - (double)law.max) * d.scale, table) / law.sum;
                double qx = 1.0;
                if (p.draft) {
                    const Law lawq = row_law(p.stats + (size_t)(p.rows + r) * chunks, chunks, d.scale, table);
                    qx = lawq.ok ? exp2_wide(((double)lq - (double)lawq.max) * d.scale, table) / lawq.sum : 1.0;
                }
                stands = u * qx < px;
            }
            if (!stands && (threadIdx.x & 63) == 0) atomicMin(s_stop, r);
        }
        __syncthreads();
        if (*s_stop < r0 + waves) break;  // uniform
    }
    __syncthreads();
    d.row = __builtin_amdgcn_readfirstlane(*s_stop);
    d.refused = d.row < d.last;
    d.p = row_law(p.stats + (size_t)d.row * chunks, chunks, d.scale, table);
    d.q = Law{0.f, 0.0, 0, false};
    d.draft = -1;
    if (d.refused) {
        const int x = p.tokens[d.row + 1];
        d.draft = x >= 0 && x < p.vocab ? x : -1;
        if (p.draft) d.q = row_law(p.stats + (size_t)(p.rows + d.row) * chunks, chunks, d.scale, table);
    }
    return true;
}

// The weights of N neighbouring tokens: p's (but for `without`), or max(p - q, 0) where the draft's are given.
template <Prec PR, int N>
__device__ __forceinline__ void row_weights(const VerifyParams &p, const Stop &d, bool rest, int without, int i, const double *table,
                                            double (&w)[N]) {
    using T = typename PrecT<PR>::T;
    float x[N];
    load_logits<PR>(x, (const T *)p.logits + (size_t)d.row * p.stride, i, p.vocab);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        w[k] = exp2_wide(((double)x[k] - (double)d.p.max) * d.scale, table);
        if (i + k == without) w[k] = 0.0;
    }
    if (rest) {
        load_logits<PR>(x, (const T *)p.draft + (size_t)d.row * p.draft_stride, i, p.vocab);
        const double ip = 1.0 / d.p.sum, iq = 1.0 / d.q.sum;
#pragma unroll
        for (int k = 0; k < N; ++k) {
#pragma clang fp contract(off)  // the same p and q leave exactly nothing: both products are rounded
            const double pk = w[k] * ip, qk = exp2_wide(((double)x[k] - (double)d.q.max) * d.scale, table) * iq;
            w[k] = fmax(pk - qk, 0.0);
        }
    }
}

}  // namespace

// Largest logit, its lowest index and the sum of weights relative to it, of chunks of 4096 logits of the target's rows and then of
// the draft's. Workgroup: a chunk; its logits stay in registers between the two passes over them.
template <Prec PR>
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(VerifyParams p) {
    using T = typename PrecT<PR>::T;
    constexpr int VEC = PrecT<PR>::VEC;
    __shared__ double s_sum[kThreads / kWave], table[32];
    __shared__ float s_max[kThreads / kWave];
    __shared__ int s_top[kThreads / kWave], s_bad[kThreads / kWave];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int work = p.rows * p.chunks * (p.draft ? 2 : 1);
    load_table(table);
    for (int idx = blockIdx.x; idx < work; idx += gridDim.x) {
        const int all = idx / p.chunks, chunk = idx - all * p.chunks;
        const bool isq = all >= p.rows;
        const int r = isq ? all - p.rows : all;
        const T *row = isq ? (const T *)p.draft + (size_t)r * p.draft_stride : (const T *)p.logits + (size_t)r * p.stride;
        const int b = request_of(p.row_start, p.n, r);
        if (isq && r + 1 >= p.row_start[b + 1]) continue;  // uniform: no draft behind the request's last row
        const double scale = weight_scale(p.temperature[b]);
        float x[kPer];
#pragma unroll
        for (int i = 0; i < kPer; i += VEC) {
            float part[VEC];
            load_logits<PR>(part, row, chunk * kVerifyChunk + (i / VEC * kThreads + tid) * VEC, p.vocab);
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[i + k] = part[k];
        }
        float m = -INFINITY;
        int top = 0x7fffffff;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = chunk * kVerifyChunk + (i / VEC * kThreads + tid) * VEC + i % VEC;
            bad |= x[i] != x[i];
            if (x[i] > m) m = x[i], top = at;
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) take_larger(m, top, __shfl_xor(m, off), __shfl_xor(top, off));
        bad = __any(bad);
        __syncthreads();  // the chunk before has been read
        if (lane == 0) s_max[w] = m, s_top[w] = top, s_bad[w] = bad;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kThreads / kWave; ++i) {
            take_larger(m, top, s_max[i], s_top[i]);
            bad |= s_bad[i] != 0;
        }
        double sum = 0.0;
        if (scale > 0.0 && m > -INFINITY && m < INFINITY) {  // uniform
#pragma unroll
            for (int i = 0; i < kPer; ++i) sum += exp2_wide(((double)x[i] - (double)m) * scale, table);
            sum = block_sum(sum, s_sum);
        }
        if (tid == 0) p.stats[(size_t)all * p.chunks + chunk] = VerifyStat{sum, bad ? NAN : m, top};
    }
}

// Sums of max(p - q, 0) over the chunks of the rows whose draft was refused.
template <Prec PR>
__global__ __launch_bounds__(kDecide) void verify_rest_kernel(VerifyParams p) {
    __shared__ double s_sum[kDecide / kWave], table[32];
    __shared__ int s_stop;
    constexpr int N = kVerifyChunk / kDecide;
    load_table(table);
    const int b = blockIdx.y;
    Stop d;
    if (!decide<PR>(p, b, table, &s_stop, d) || !d.refused || !d.p.ok || !d.q.ok || !(d.scale > 0.0)) return;
    for (int chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
        double w[N], sum = 0.0;
        row_weights<PR>(p, d, true, -1, chunk * kVerifyChunk + (int)threadIdx.x * N, table, w);
#pragma unroll
        for (int k = 0; k < N; ++k) sum += w[k];
        sum = block_sum(sum, s_sum);
        if (threadIdx.x == 0) p.rest[(size_t)d.row * p.chunks + chunk] = sum;
    }
}

// The accepted rows and the next token. Workgroup: a request.
template <Prec PR>
__global__ __launch_bounds__(kDecide) void verify_token_kernel(VerifyParams p) {
    __shared__ double s_sum[kDecide / kWave], table[32], s_before;
    __shared__ int s_stop, s_from, s_chunk, s_token, s_last;
    constexpr int N = kVerifyChunk / kDecide;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    load_table(table);
    Stop d;
    const bool any = decide<PR>(p, b, table, &s_stop, d);
    const bool law = any && d.p.ok && d.scale >= 0.0;
    if (tid == 0) p.accepted[b] = any ? d.row - d.first + 1 : 0;
    if (!law || d.scale == 0.0) {  // uniform
        if (tid == 0) p.next_token[b] = law ? d.p.top : -1;
        return;
    }
    // What is drawn from: the chunks' sums of p, of p without the refused token, or of the rest. (Where that is empty, p.)
    bool rest = d.refused && d.q.ok;
    const bool point = d.refused && !rest && d.draft >= 0;
    int without = point ? d.draft : -1;
    double cut = 0.0;  // the sum of the refused token's chunk without it
    if (point) {
        double x[N], sum = 0.0;
        row_weights<PR>(p, d, false, without, without / kVerifyChunk * kVerifyChunk + tid * N, table, x);
#pragma unroll
        for (int k = 0; k < N; ++k) sum += x[k];
        cut = block_sum(sum, s_sum);
    }
    const VerifyStat *st = p.stats + (size_t)d.row * p.chunks;
    auto chunk_sum = [&](int c) {
        if (rest) return p.rest[(size_t)d.row * p.chunks + c];
        if (without >= 0 && c == without / kVerifyChunk) return cut;
        return st[c].sum * exp2_wide(((double)st[c].max - (double)d.p.max) * d.scale, table);
    };
    if (w == 0) {  // one wave: the chunk in which the running sum passes the number
        auto total = [&]() {
            double t = 0.0;
            for (int c = lane; c < p.chunks; c += kWave) t += chunk_sum(c);
            return wave_sum(t);
        };
        double t = total();
        if (!(t > 0.0)) {
            rest = false;
            without = -1;
            t = total();
        }
        const double u = p.sample_u[b], aim = (u > 0.0 ? fmin(u, 0x1.fffffffffffffp-1) : 0.0) * t;
        double before = 0.0, at_before = 0.0;
        int chunk = -1, last = -1;  // the chunk, and the last one that is not empty
        double last_before = 0.0;
        for (int c0 = 0; c0 < p.chunks && chunk < 0; c0 += kWave) {
            const double x = c0 + lane < p.chunks ? chunk_sum(c0 + lane) : 0.0;
            double run = x;
#pragma unroll
            for (int off = 1; off < kWave; off <<= 1) {
                const double y = __shfl_up(run, off);
                if (lane >= off) run += y;
            }
            const uint64_t past = __ballot(before + run > aim && x > 0.0), some = __ballot(x > 0.0);
            if (past) {
                const int l = __ffsll((unsigned long long)past) - 1;
                chunk = c0 + l;
                at_before = l > 0 ? before + __shfl(run, max(l - 1, 0)) : before;
            }
            if (some) {
                const int l = 63 - __clzll((long long)some);
                last = c0 + l;
                last_before = l > 0 ? before + __shfl(run, max(l - 1, 0)) : before;
            }
            before += __shfl(run, 63);
        }
        if (chunk < 0) {  // rounding: behind the last sum
            chunk = last;
            at_before = last_before;
        }
        if (lane == 0) {
            s_chunk = chunk;
            s_before = aim - at_before;
            s_token = 0x7fffffff;
            s_last = -1;
            s_from = rest ? 2 : without >= 0 ? 1 : 0;
        }
    }
    __syncthreads();
    rest = s_from == 2;
    if (s_from == 0) without = -1;
    const int chunk = max(s_chunk, 0);
    const double aim = s_before;
    double x[N], run = 0.0;
    const int i = chunk * kVerifyChunk + tid * N;
    row_weights<PR>(p, d, rest, without, i, table, x);
#pragma unroll
    for (int k = 0; k < N; ++k) run += x[k];
    // sums of the threads before this one
    double before = run;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const double y = __shfl_up(before, off);
        if (lane >= off) before += y;
    }
    if (lane == 63) s_sum[w] = before;
    __syncthreads();
    double base = before - run;
    for (int v = 0; v < w; ++v) base += s_sum[v];
    int found = 0x7fffffff, last = -1;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        base += x[k];
        if (x[k] > 0.0) {
            last = i + k;
            if (base > aim && found == 0x7fffffff) found = i + k;
        }
    }
    if (found != 0x7fffffff) atomicMin(&s_token, found);
    if (last >= 0) atomicMax(&s_last, last);
    __syncthreads();
    if (tid == 0) p.next_token[b] = s_token != 0x7fffffff ? s_token : s_last;
}

namespace {

template <Prec PR>
hipError_t launch_verify(const VerifyParams &p, hipStream_t s) {
    if (p.rows > 0) {
        const int64_t work = (int64_t)p.rows * p.chunks * (p.draft ? 2 : 1);
        hipLaunchKernelGGL(verify_stats_kernel<PR>, dim3((unsigned)std::min<int64_t>(work, 1 << 20)), dim3(kThreads), 0, s, p);
        if (p.draft)
            hipLaunchKernelGGL(verify_rest_kernel<PR>, dim3((unsigned)std::min(p.chunks, 1024), (unsigned)p.n), dim3(kDecide), 0, s, p);
    }
    hipLaunchKernelGGL(verify_token_kernel<PR>, dim3((unsigned)p.n), dim3(kDecide), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_verify(bool bf16, const VerifyParams &p, hipStream_t s) {
    if (p.n < 1 || p.n > kPagedMaxSeqs || p.rows < 0 || p.vocab < 1 || p.chunks != (p.vocab + kVerifyChunk - 1) / kVerifyChunk ||
        (int64_t)p.rows * p.chunks * 2 > INT32_MAX)
        return hipErrorInvalidValue;
    return bf16 ? launch_verify<Prec::BF16>(p, s) : launch_verify<Prec::F32>(p, s);
}

}  // namespace cllm

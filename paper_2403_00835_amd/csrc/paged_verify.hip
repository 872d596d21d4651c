// Verification of drafted tokens on gfx950: how many of a request's tokens stand against the target's distribution, and the
// token that follows them.
//
// Row r of a request holds the target's logits behind tokens[r]; tokens[r + 1] is its draft. With p = softmax(l / T) and q the
// draft's distribution (a point mass where there are no draft logits), the draft x stands where u q(x) < p(x). At the first
// row whose draft does not stand, the next token is drawn from max(p - q, 0); behind the last row, from p: the tokens
// then have the target's distribution. A token is drawn as the lowest index whose running sum is above u times the sum.
//
// Every weight 2^((l - max) log2(e) / T) and every sum is held in 64 bits: a draw among V tokens picks a neighbour with a
// probability of about V times the weights' relative error, which in 32 bits is one in some hundred draws. Weights are
// 2^-42 off (weight_parts), sums less; what is left of max(p - q, 0) is off by that part of p.
#include <algorithm>

#include "device.h"
#include "paged.h"

namespace cllm {

namespace {

constexpr int kThreads = 256;                        // of the statistics' workgroups: a chunk a wave
constexpr int kPart = 8 * kWave, kParts = kVerifyChunk / kPart;  // logits that a wave takes by eights, of a chunk
constexpr int kRest = 512, kToken = 1024;           // of the two kernels that decide where a request stops: a row a wave at once

constexpr int kExpSteps = 256;
// 2^(j / 256), by its Taylor series to z^17 / 17! (z = ln 2 j / 256: 1e-18 is left out): no load to wait for.
__device__ __forceinline__ double exp_step(int j) {
    const double z = 0x1.62e42fefa39efp-9 * j;
    double y = 1.0;
#pragma unroll
    for (int k = 17; k >= 1; --k) y = __builtin_fma(y, z * (1.0 / k), 1.0);
    return y;
}
// A barrier for what is in LDS: loads in flight are not waited for, as __syncthreads() would.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));
    barrier_no_fence();
}
// The table, in LDS, by the first kExpSteps threads.
__device__ __forceinline__ void make_table(double (&table)[kExpSteps]) {
    if (threadIdx.x < kExpSteps)
        table[threadIdx.x] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, exp_step(threadIdx.x)) - ((uint64_t)threadIdx.x << 44));
    lds_barrier();
}

// 1 / t: the instruction's guess and two steps of Newton's.
__device__ __forceinline__ double inverse(double t) {
    double y = __builtin_amdgcn_rcp(t);
    y = __builtin_fma(y, __builtin_fma(-t, y, 1.0), y);
    return __builtin_fma(y, __builtin_fma(-t, y, 1.0), y);
}

// The weights' exponent: scale = log2(e) / T. 0: the greedy choice; -1: not a temperature.
__device__ __forceinline__ double weight_scale(float temperature) {
    const double y = inverse(temperature);
    return temperature == 0.0f ? 0.0 : temperature > 0.0f && temperature < INFINITY ? 1.4426950408889634 * y : -1.0;
}

// -1000 / scale (of a temperature).
__device__ __forceinline__ double weight_floor(float temperature) { return -693.14718055994531 * (double)temperature; }

// 2^(d scale), d scale within +-1000, as f 2^r: f = 2^(k / 256) from the table (LDS), whose entry j holds 2^(j / 256) less j in
// the last eight bits before its exponent's, where all of k is added (j is k's remainder, and the rest its whole part), 2^r, |r| <= 1 / 512, by its Taylor polynomial, whose first term left out is 2^-42 of it. The product d scale is not
// rounded on its own.
struct Weight {
    double f, r2;
};
__device__ __forceinline__ Weight weight_parts(double d, double scale, const double *table) {
    constexpr double kRound = 0x1.8p44;  // its last place is 1 / 256
    const double t = __builtin_fma(d, scale, kRound), r = __builtin_fma(d, scale, kRound - t);
    const uint32_t k = (uint32_t)__builtin_bit_cast(uint64_t, t);  // 256 d scale, rounded
    double y = 0x1.c6b08d704a0c0p-5;
    asm("" : "+v"(y));  // (kept in registers: the product takes one constant from elsewhere)
    y = __builtin_fma(y, r, 0x1.ebfbdff82c58fp-3);
    y = __builtin_fma(y, r, 0x1.62e42fefa39efp-1);
    y = __builtin_fma(y, r, 1.0);
    const u32x2 e = __builtin_bit_cast(u32x2, table[k & (kExpSteps - 1)]);
    const uint32_t high = (k << 12) + e[1];
    return {__builtin_bit_cast(double, u32x2{e[0], high}), y};
}
// Below 2^-1000: about 2^-1000, which no sum that holds a weight above 2^-900 minds; floor = -1000 / scale.
__device__ __forceinline__ double weight(double d, double scale, double floor, const double *table) {
    const Weight w = weight_parts(fmax(d, floor), scale, table);
    return w.f * w.r2;
}
// Of the logit l beside m: 0 below 2^-1000.
__device__ __forceinline__ double weight_of(float l, float m, double scale, double floor, const double *table) {
    const double d = (double)l - (double)m;
    return d >= floor ? weight(d, scale, floor, table) : 0.0;
}

typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The logits i .. i + 7 of a row, at any element's address, as eight neighbours from `from` on; those of them that are before i
// or past the row's end are -inf.
template <Prec PR>
struct Eight {
    using T = typename PrecT<PR>::T;
    static constexpr int VEC = PrecT<PR>::VEC, NV = 8 / VEC;
    u32x4 raw[NV];  // (words, not elements: of those the compiler would make a register each)
    int from;
    __device__ __forceinline__ void load_whole(const T *row, int i) {
        from = i;
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = *reinterpret_cast<const u32x4_any *>(row + i + v * VEC);
    }
    __device__ __forceinline__ void load(const T *row, int i, int vocab) {
        if (vocab >= 8) {
            load_whole(row, min(i, vocab - 8));
#pragma unroll
            for (int k = 0; k < 8; ++k) put(k, from + k >= i ? (*this)[k] : -INFINITY);
        } else {
            from = i;
            asm volatile("" : "+v"(i));  // (or the eight addresses are formed before every caller's loop)
#pragma unroll
            for (int k = 0; k < 8; ++k) put(k, i + k < vocab ? from_elem<PR>(row[i + k]) : -INFINITY);
        }
    }
    __device__ __forceinline__ float operator[](int k) const {
        if constexpr (PR == Prec::BF16) return __uint_as_float(k % 2 ? raw[0][k / 2] & 0xffff0000u : raw[0][k / 2] << 16);
        return __uint_as_float(raw[k / VEC][k % VEC]);
    }
    // The largest magnitude (where there is a NaN, NaN or that of the others).
    __device__ __forceinline__ float size() const {
        if constexpr (PR == Prec::BF16) {
            u16x2 m{};
#pragma unroll
            for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, raw[0][i] & 0x7fff7fffu));
            return __uint_as_float((uint32_t)max(m[0], m[1]) << 16);
        }
        float m = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf((*this)[k]));
        return m;
    }
    __device__ __forceinline__ void put(int k, float x) {  // (a value of T)
        uint32_t &w = reinterpret_cast<uint32_t *>(raw)[PR == Prec::BF16 ? k / 2 : k];
        const uint32_t b = __float_as_uint(x);
        if constexpr (PR == Prec::BF16)
            w = k % 2 ? (w & 0xffffu) | (b & 0xffff0000u) : (w & 0xffff0000u) | b >> 16;
        else
            w = b;
    }
    // What has been made of the words is not kept beside them for later uses.
    __device__ __forceinline__ void keep() {
#pragma unroll
        for (int v = 0; v < NV; ++v) asm volatile("" : "+v"(raw[v]));
    }
};

// The request of a row: the last one that starts at or before it (a wave's two reads; n up to 1024). Of the plan's starts only
// those of its own requests count: behind them is what an earlier plan of more left.
__device__ __forceinline__ int request_of(const VerifyParams &p, int row) {
    const int lane = threadIdx.x & 63, n = p.n, own = p.status ? min(n, p.status[PS_ENTRIES]) : n;
    if (n <= kWave) return max((int)__popcll(__ballot(lane < own && p.row_start[min(lane, n)] <= row)) - 1, 0);
    const uint64_t far = __ballot(16 * lane < own && p.row_start[min(16 * lane, n)] <= row);
    const int c = 16 * max((int)__popcll(far) - 1, 0);  // (a row before the first request is counted to that)
    const uint64_t near = __ballot(lane < 16 && c + lane < own && p.row_start[min(c + lane, n)] <= row);
    return min(c + max((int)__popcll(near) - 1, 0), n - 1);
}

// Lane moves in the ALU. A step: 16 lanes by shifts, then across them; lane 63 ends with all.
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float x, float none) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x, double none) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x), o = __builtin_bit_cast(uint64_t, none);
    const uint32_t lo = __builtin_amdgcn_update_dpp((int)(uint32_t)o, (int)(uint32_t)b, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp((int)(o >> 32), (int)(b >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float of_lane(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
__device__ __forceinline__ double of_lane(double x, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <class T, class F>
__device__ __forceinline__ T wave_scan(T x, T none, F f) {  // inclusive, from lane 0 on
    x = f(x, moved<0x111, 0xf>(x, none));
    x = f(x, moved<0x112, 0xf>(x, none));
    x = f(x, moved<0x114, 0xf>(x, none));
    x = f(x, moved<0x118, 0xf>(x, none));
    x = f(x, moved<0x142, 0xa>(x, none));
    return f(x, moved<0x143, 0xc>(x, none));
}
__device__ __forceinline__ double scan_sum(double x) {
    return wave_scan(x, 0.0, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double wave_sum(double x) { return of_lane(scan_sum(x), 63); }
__device__ __forceinline__ float wave_max(float x) {
    return of_lane(wave_scan(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), 63);
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x = min(x, __shfl_xor(x, off));
    return x;
}

// The same over LANES lanes (all of a wave, or 16 neighbours), in each of them.
template <int CTRL, class T>
__device__ __forceinline__ T traded(T x) {
    return moved<CTRL, 0xf>(x, x);
}
template <int LANES, class T, class F>
__device__ __forceinline__ T group_all(T x, F f) {
    static_assert(LANES == 16, "lanes whose sums are lane moves of a row");
    x = f(x, traded<0xb1>(x));   // lane ^ 1
    x = f(x, traded<0x4e>(x));   // lane ^ 2
    x = f(x, traded<0x141>(x));  // 8 lanes mirrored
    return f(x, traded<0x140>(x));  // 16 lanes mirrored
}
template <int LANES>
__device__ __forceinline__ float group_max(float x) {
    if constexpr (LANES == kWave) return wave_max(x);
    else return group_all<LANES>(x, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES>
__device__ __forceinline__ double group_sum(double x) {
    if constexpr (LANES == kWave) return wave_sum(x);
    else return group_all<LANES>(x, [](double a, double b) { return a + b; });
}
template <int LANES>
__device__ __forceinline__ int group_min(int x) {
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) x = min(x, __shfl_xor(x, off));
    return x;
}
template <int LANES>
__device__ __forceinline__ bool group_any(bool x) {
    if constexpr (LANES == kWave) return __any(x);
    else return __ballot(x) >> (threadIdx.x & (kWave - LANES)) & ((1ull << LANES) - 1);
}

// A row's distribution from the statistics of its chunks, by LANES lanes (LANES < 64: at most so many chunks). head: of the
// lane's first chunk, where there is one.
struct Law {
    float max;    // what weights are relative to: the largest of its chunks' (greedy requests: the largest logit)
    double norm;  // 1 / the sum of the weights
    int top;      // greedy requests: the largest logit's lowest index
    bool ok;      // neither NaN nor +inf among the logits, nor all -inf
};
template <int LANES>
__device__ __forceinline__ Law row_law(const VerifyStat &head, const VerifyStat *st, int chunks, double scale, double floor, const double *table) {
    const int lane = threadIdx.x & (LANES - 1);
    constexpr VerifyStat kNone{0.0, -INFINITY, 0x7fffffff};
    const VerifyStat mine = lane < chunks ? head : kNone;  // (the first chunks: most vocabularies' all)
    float m = mine.max;
    bool bad = m != m;
    for (int c = lane + LANES; LANES == kWave && c < chunks; c += LANES) {
        const float x = st[c].max;
        bad |= x != x;
        m = fmaxf(m, x);
    }
    Law w{group_max<LANES>(m), 0.0, 0x7fffffff, false};
    w.ok = !group_any<LANES>(bad) && w.max > -INFINITY && w.max < INFINITY;
    if (!w.ok) return w;
    if (scale > 0.0) {
        double sum = mine.sum * weight((double)mine.max - (double)w.max, scale, floor, table);
        for (int c = lane + LANES; LANES == kWave && c < chunks; c += LANES)
            sum += st[c].sum * weight((double)st[c].max - (double)w.max, scale, floor, table);
        w.norm = inverse(group_sum<LANES>(sum));
    } else {
        int top = mine.max == w.max ? mine.top : 0x7fffffff;
        for (int c = lane + LANES; LANES == kWave && c < chunks; c += LANES)
            if (st[c].max == w.max) top = min(top, st[c].top);
        w.top = group_min<LANES>(top);
    }
    return w;
}

// A request: its rows (first >= end: none, or not within the call's), and its temperature.
struct Request {
    int first, end;
    double scale, floor;
};
// The request of a workgroup, and the table; what they read is on its way at once.
__device__ __forceinline__ Request begin(const VerifyParams &p, int b, double (&table)[kExpSteps]) {
    const float temperature = p.temperature[b];
    Request q;
    q.first = p.row_start[b];
    q.end = p.row_start[b + 1];
    if (p.status && (p.status[PS_ROWS] == 0 || b >= p.status[PS_ENTRIES])) q.end = q.first;  // a refused plan
    if (q.first < 0 || q.end > p.rows) q.end = q.first;
    q.scale = weight_scale(temperature);
    q.floor = weight_floor(temperature);
    make_table(table);
    return q;
}

// Up to so many chunks a wave decides on four rows at once: 18 requests of 14 to 44 rows of 12,233 tokens 27.5 us in place of 31.8, 16 of
// 32 rows of 32,000 25.6 in place of 26.4.
constexpr int kFewChunks = 16;
struct Decide {  // LDS
    VerifyStop at[kToken / kFewChunks];
    int stop;
};

// Place of a request's row, by `lanes` lanes, among the threads of verify_token_kernel.
constexpr int head_of(int row, int lanes) { return row % (kToken / lanes) * lanes; }

// Where a request stops, by the whole workgroup: a row LANES lanes. heads (or null): statistics of the first LANES chunks of the row
// at which it stops, in those lanes' places.
template <int LANES>
__device__ __forceinline__ VerifyStop decide_by(const VerifyParams &p, const Request &q, const double *table, Decide &s, VerifyStat *heads) {
    const int rows = blockDim.x / LANES, first = q.first, end = q.end;  // (rows: at once)
    const int slot = LANES == kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / LANES) : (int)threadIdx.x / LANES;
    const double scale = q.scale, floor = q.floor;
    if (first >= end) {  // uniform
        VerifyStop none{};
        none.row = -1;
        return none;
    }
    if (threadIdx.x == 0) s.stop = end;
    const int lane = threadIdx.x & (LANES - 1);
    struct Row {  // what a row's decision reads; the next one's is on its way beside this one's
        VerifyStat p, q;
        double u;
        float lp, lq;
        int x;
    } next{};
    auto load = [&](int r) {
        if (r >= end) return;
        if (lane < p.chunks) next.p = p.stats[(size_t)r * p.chunks + lane];
        next.lp = p.picked[r];  // (the draft's logit, where it is a token)
        if (r + 1 == end) return;  // no draft
        next.x = p.tokens[r + 1];
        next.u = p.accept_u[r];
        if (!p.draft) return;
        if (lane < p.chunks) next.q = p.stats[(size_t)(p.rows + r) * p.chunks + lane];
        next.lq = p.picked[p.rows + r];
    };
    load(first + slot);
    __syncthreads();
    for (int r0 = first; r0 < end; r0 += rows) {
        const int r = r0 + slot;
        if (r < end) {
            const Row at = next;
            load(r + rows);
            const bool drafted = r + 1 < end;
            const VerifyStat *st = p.stats + (size_t)r * p.chunks, *sq = p.stats + (size_t)(p.rows + r) * p.chunks;
            const int x = drafted ? at.x : -1;
            const bool known = x >= 0 && x < p.vocab;
            const double u = at.u;
            const float lp = at.lp, lq = at.lq;
            const Law law = row_law<LANES>(at.p, st, p.chunks, scale, floor, table);
            Law lawq{0.f, 0.0, 0, false};
            if (p.draft && drafted && scale > 0.0) lawq = row_law<LANES>(at.q, sq, p.chunks, scale, floor, table);
            bool stands = false;
            if (law.ok && drafted && known) {
                if (scale == 0.0) {
                    stands = x == law.top;
                } else if (scale > 0.0) {
                    const double px = weight_of(lp, law.max, scale, floor, table) * law.norm;
                    const double qx = lawq.ok ? weight_of(lq, lawq.max, scale, floor, table) * lawq.norm : 1.0;
                    stands = u * qx < px;
                }
            }
            if (!stands && heads) heads[threadIdx.x] = at.p;
            const uint64_t ends = __ballot(!stands);
            if (ends && (int)(threadIdx.x & 63) == __ffsll((unsigned long long)ends) - 1) {  // the wave's first that does
                VerifyStop &stop = s.at[slot];
                stop.p_norm = law.norm;
                stop.q_norm = lawq.norm;
                stop.p_max = law.max;
                stop.q_max = lawq.max;
                stop.first = first;
                stop.row = r;
                stop.draft = known ? x : -1;
                stop.logit = lp;
                stop.kind = (drafted ? VS_REFUSED : 0) | (law.ok && scale >= 0.0 ? VS_LAW : 0) | (law.ok && lawq.ok ? VS_REST : 0);
                stop.top = law.top;
                atomicMin(&s.stop, r);
            }
        }
        __syncthreads();
        if (s.stop < r0 + rows) return s.at[s.stop - r0];  // uniform: the last row at the latest
    }
    return VerifyStop{};  // (not reached)
}
__device__ __forceinline__ VerifyStop decide(const VerifyParams &p, const Request &q, const double *table, Decide &s, VerifyStat *heads) {
    return p.chunks <= kFewChunks ? decide_by<kFewChunks>(p, q, table, s, heads) : decide_by<kWave>(p, q, table, s, heads);
}

// A chunk's sum relative to the logit `to` in place of `from`: by two factors, as the sum may be 2^900 and each factor 2^-1000. What
// is as good as nothing is made nothing (an empty chunk is), so that a chunk that is drawn holds a token of a weight above 2^-1000.
__device__ __forceinline__ double joined_sum(double sum, float from, float to, const Request &q, const double *table) {
    const double h = 0.5 * ((double)from - (double)to);
    if (!(h >= q.floor)) return 0.0;
    const double f = weight(h, q.scale, q.floor, table), x = sum * f * f;
    return x < 0x1p-980 ? 0.0 : x;
}

// max(p - q, 0) of a token of logits l and lq.
__device__ __forceinline__ double left_weight(float l, float lq, const VerifyStop &at, const Request &q, const double *table) {
#pragma clang fp contract(off)  // the same p and q leave exactly nothing: both products are rounded
    const double px = weight_of(l, at.p_max, q.scale, q.floor, table) * at.p_norm;
    const double qx = weight_of(lq, at.q_max, q.scale, q.floor, table) * at.q_norm;
    return fmax(px - qx, 0.0);
}

// The weights of N neighbouring tokens: p's (but for `without`), or max(p - q, 0).
template <Prec PR, int N>
__device__ __forceinline__ void row_weights(const VerifyParams &p, const VerifyStop &at, bool rest, int without, int i, const Request &q,
                                            const double *table, double (&w)[N]) {
    using T = typename PrecT<PR>::T;
    const T *row = (const T *)p.logits + (size_t)at.row * p.stride, *drow = (const T *)p.draft + (size_t)at.row * p.draft_stride;
    float x[N], y[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = i + k < p.vocab ? from_elem<PR>(row[i + k]) : -INFINITY;
    if (rest) {  // uniform
#pragma unroll
        for (int k = 0; k < N; ++k) y[k] = i + k < p.vocab ? from_elem<PR>(drow[i + k]) : -INFINITY;
#pragma unroll
        for (int k = 0; k < N; ++k) w[k] = left_weight(x[k], y[k], at, q, table);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) w[k] = i + k == without ? 0.0 : weight_of(x[k], at.p_max, q.scale, q.floor, table);
    }
}

}  // namespace

// The sum of weights of chunks of 2048 logits of the target's rows and then of the draft's, and the logit that they are relative
// to: 0 where 64 bits hold every weight, which saves a difference and a bound for each (such chunks are most), or the largest
// one. Of greedy requests the largest logit and its index instead. A chunk a wave, its logits in registers as they came (72
// registers in bf16, 90 in fp32).
// Bound: arithmetic beside the reading (64 requests of one to seven rows of 99,991 bf16 logits, the target's and the draft's, 89.6 MB:
// 30.0 us, 3.0 TB/s, the vector units at work for two thirds of it, half of that in 64 bits; 512 rows of 32,000 fp32
// logits, 65.5 MB: 18.6 us, 3.5 TB/s), of a few rows latency (five: 6.3 us). Weights relative to the largest logit in every chunk
// take 35 us in place of 31; eight waves a SIMD in place of seven, and the table from memory, the same 30.
template <Prec PR>
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(VerifyParams p, int row0) {
    using T = typename PrecT<PR>::T;
    static_assert(kExpSteps <= kThreads, "a thread an entry");
    __shared__ double table[kExpSteps];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunk = blockIdx.x * (kThreads / kWave) + w, all = row0 + blockIdx.y;  // the target's rows, then the draft's
    const bool isq = all >= p.rows;
    const int r = isq ? all - p.rows : all;
    const T *row = isq ? (const T *)p.draft + (size_t)r * p.draft_stride : (const T *)p.logits + (size_t)r * p.stride;
    const int first = chunk * kVerifyChunk + lane * 8;
    const bool whole = (chunk + 1) * kVerifyChunk <= p.vocab;  // uniform
    const int draft = r + 1 < p.rows ? p.tokens[r + 1] : -1;
    int b = 0;
    bool live = chunk < p.chunks;  // uniform over the wave
    if (isq) {
        b = request_of(p, r);
        live = live && r + 1 < p.row_start[b + 1];  // no draft behind the request's last row
    }
    Eight<PR> x[kParts];
    if (live && whole) {
#pragma unroll
        for (int v = 0; v < kParts; ++v) x[v].load_whole(row, first + v * kPart);
    } else if (live) {
#pragma unroll
        for (int v = 0; v < kParts; ++v) x[v].load(row, first + v * kPart, p.vocab);
    }
    make_table(table);
    if (!live) return;
    if (!isq) b = request_of(p, r);
    const float temperature = p.temperature[b];
    const double scale = weight_scale(temperature), floor = weight_floor(temperature);
    float size = 0.0f;
#pragma unroll
    for (int v = 0; v < kParts; ++v) {
        size = fmaxf(size, x[v].size());
        x[v].keep();
    }
    double sum = 0.0;
    float ref = 0.0f;
    int top = 0x7fffffff;
    bool none;
    if (scale > 0.0 && __all((double)size <= -0.9 * floor)) {
#pragma unroll
        for (int v = 0; v < kParts; ++v)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Weight z = weight_parts((double)x[v][k], scale, table);
                sum = __builtin_fma(z.f, z.r2, sum);
                if (k % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (more at once take the registers of other waves)
            }
        sum = wave_sum(sum);
        none = sum != sum;
    } else {
        float m = -INFINITY;
        bool bad = false;
#pragma unroll
        for (int v = 0; v < kParts; ++v) {
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float a = x[v][k], c = x[v][k + 1];
                m = fmaxf(fmaxf(m, a), c);
                bad |= __builtin_isunordered(a, c);
            }
            x[v].keep();
        }
        ref = wave_max(m);
        none = __any(bad) || ref == INFINITY;
        if (ref > -INFINITY && ref < INFINITY) {  // else there is nothing, or no distribution
#pragma unroll
            for (int v = kParts - 1; v >= 0; --v)
#pragma unroll
                for (int k = 7; k >= 0; --k) {
                    if (scale > 0.0)
                        sum += weight((double)x[v][k] - (double)ref, scale, floor, table);
                    else if (x[v][k] == ref)
                        top = x[v].from + k;
                    if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                }
            if (scale > 0.0)
                sum = wave_sum(sum);
            else
                top = wave_min(top);
        }
    }
    if (lane == 0) {
        p.stats[(size_t)all * p.chunks + chunk] = VerifyStat{sum, none ? NAN : ref, top};
        if (draft >= chunk * kVerifyChunk && draft < min((chunk + 1) * kVerifyChunk, p.vocab)) p.picked[all] = from_elem<PR>(row[draft]);
    }
}

// Where the requests stop, and the sums of max(p - q, 0) over the chunks of the rows whose draft was refused: two chunks a
// workgroup at a time, each of which decides for itself.
// Bound: latency (what a decision reads, then a row's logits) and 64-bit arithmetic: one request of 32,000 tokens 5.6 us, 64
// of 99,991 13.4, in 13 workgroups of two rounds each (25 of one round 16.4, 7 of four 17.1).
constexpr int kRestChunks = kRest / kWave / kParts, kRestFit = 4;
template <Prec PR>
__global__ __launch_bounds__(kRest) void verify_rest_kernel(VerifyParams p) {
    using T = typename PrecT<PR>::T;
    __shared__ double table[kExpSteps], s_sum[kRest / kWave];
    __shared__ Decide s_decide;
    const int b = blockIdx.y, lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Request q = begin(p, b, table);
    const VerifyStop at = decide(p, q, table, s_decide, nullptr);
    if (at.row < 0) return;  // uniform
    if (blockIdx.x == 0 && threadIdx.x == 0) p.stops[at.first] = at;
    if (!(at.kind & VS_REST)) return;
    const T *row = (const T *)p.logits + (size_t)at.row * p.stride, *drow = (const T *)p.draft + (size_t)at.row * p.draft_stride;
    Eight<PR> x, y, xn, yn;
    auto load = [&](int c0) {
        const int i = c0 * kVerifyChunk + w * kPart + lane * 8;  // (a chunk is kParts waves')
        const bool whole = (c0 + kRestChunks) * kVerifyChunk <= p.vocab;  // uniform
        if (whole) {
            xn.load_whole(row, i);
            yn.load_whole(drow, i);
        } else {
            xn.load(row, i, p.vocab);
            yn.load(drow, i, p.vocab);
        }
    };
    load(blockIdx.x * kRestChunks);
#pragma unroll 1
    for (int c0 = blockIdx.x * kRestChunks; c0 < p.chunks; c0 += gridDim.x * kRestChunks) {
        x = xn;
        y = yn;
        if (c0 + (int)gridDim.x * kRestChunks < p.chunks) load(c0 + gridDim.x * kRestChunks);
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += left_weight(x[k], y[k], at, q, table);
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) s_sum[w] = sum;
        __syncthreads();
        const int chunk = c0 + (int)threadIdx.x;
        if (threadIdx.x < kRestChunks && chunk < p.chunks) {
            double t = 0.0;
#pragma unroll
            for (int v = 0; v < kParts; ++v) t += s_sum[threadIdx.x * kParts + v];
            p.rest[(size_t)at.first * p.chunks + chunk] = t;
        }
    }
}

// The accepted rows and the next token. Workgroup: a request.
// Bound: latency, of three to five reads that wait for one another, each about 1 us: one request 4.7 us, 64 of 99,991 tokens
// 6.0; where it decides, 16 of 32 rows, 6.2. Neighbours and waves in the tokens' order pick the token by ballots: atomics on
// LDS for it, lane by lane, took 4.4 us more.
template <Prec PR>
__global__ __launch_bounds__(kToken) void verify_token_kernel(VerifyParams p) {
    constexpr int N = 4, kDraw = kVerifyChunk / N;  // neighbouring tokens of a thread, threads that a chunk takes
    static_assert(kDraw <= kToken && kDraw % kWave == 0, "whole waves");
    __shared__ double table[kExpSteps], s_sum[kDraw / kWave], s_aim;
    __shared__ Decide s_decide;
    __shared__ VerifyStat s_heads[kToken];
    __shared__ int s_from, s_chunk, s_found[kDraw / kWave], s_last[kDraw / kWave];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const double u = p.sample_u[b];
    const Request q = begin(p, b, table);
    const double scale = q.scale, floor = q.floor;
    VerifyStop at{};
    at.row = -1;
    double rest_head = 0.0;  // the rest's sum of chunk `lane`, where there is a rest; on its way beside what says so
    if (p.draft && q.first < q.end && lane < p.chunks) rest_head = p.rest[(size_t)q.first * p.chunks + lane];
    if (!p.draft)
        at = decide(p, q, table, s_decide, s_heads);
    else if (q.first < q.end)
        at = p.stops[q.first];  // decided with the rest's sums
    const bool law = at.row >= 0 && (at.kind & VS_LAW);
    if (tid == 0) p.accepted[b] = at.row >= 0 ? at.row - at.first + 1 : 0;
    if (!law || scale == 0.0) {  // uniform
        if (tid == 0) p.next_token[b] = law ? at.top : -1;
        return;
    }
    // What is drawn from: the rest, p without the refused token, or p (also where those are empty).
    bool rest = at.kind & VS_REST;
    int without = !rest && (at.kind & VS_REFUSED) ? at.draft : -1;
    const VerifyStat *st = p.stats + (size_t)at.row * p.chunks, *head = s_heads + head_of(at.row - at.first, p.chunks <= kFewChunks ? kFewChunks : kWave);
    auto stat = [&](int c) { return p.draft || c >= kWave ? st[c] : head[c]; };
    double cut = 0.0;  // the sum of the refused token's chunk without it
    if (without >= 0) {
        const int c = without / kVerifyChunk;
        const VerifyStat s = stat(c);
        const double mine = s.max > -INFINITY ? weight_of(at.logit, s.max, scale, floor, table) : 0.0;
        cut = joined_sum(s.sum - mine, s.max, at.p_max, q, table);
        if (mine * 256.0 > s.sum * 255.0) {  // uniform: little is left, of which the difference loses digits
            double x[N], sum = 0.0;
            if (tid < kDraw) {
                row_weights<PR>(p, at, false, without, c * kVerifyChunk + tid * N, q, table, x);
#pragma unroll
                for (int k = 0; k < N; ++k) sum += x[k];
                sum = wave_sum(sum);
                if (lane == 0) s_sum[w] = sum;
            }
            __syncthreads();
            cut = 0.0;
#pragma unroll
            for (int v = 0; v < kDraw / kWave; ++v) cut += s_sum[v];
        }
    }
    auto chunk_sum = [&](int c) {
        if (c >= p.chunks) return 0.0;
        if (rest) return c < kWave ? rest_head : p.rest[(size_t)q.first * p.chunks + c];
        if (without >= 0 && c == without / kVerifyChunk) return cut;
        const VerifyStat s = stat(c);
        return joined_sum(s.sum, s.max, at.p_max, q, table);
    };
    if (w == 0) {  // one wave: the chunk in which the running sum passes the number
        double first, t;  // this lane's first chunk, the sum
        auto total = [&]() {
            first = chunk_sum(lane);
            double x = first;
            for (int c = lane + kWave; c < p.chunks; c += kWave) x += chunk_sum(c);
            t = wave_sum(x);
        };
        total();
        if (!(t > 0.0)) {
            rest = false;
            without = -1;
            total();
        }
        const double aim = (u > 0.0 ? fmin(u, 0x1.fffffffffffffp-1) : 0.0) * t;
        double before = 0.0, base = 0.0, last_base = 0.0;
        int chunk = -1, last = 0;  // the chunk, and the last one that is not empty
        for (int c0 = 0; c0 < p.chunks && chunk < 0; c0 += kWave) {
            const double x = c0 == 0 ? first : chunk_sum(c0 + lane), run = scan_sum(x);
            const uint64_t past = __ballot(before + run > aim && x > 0.0), some = __ballot(x > 0.0);
            if (some) {
                const int l = 63 - __clzll((long long)some);
                last = c0 + l;
                last_base = l > 0 ? before + of_lane(run, max(l - 1, 0)) : before;
            }
            if (past) {
                const int l = __ffsll((unsigned long long)past) - 1;
                chunk = c0 + l;
                base = l > 0 ? before + of_lane(run, max(l - 1, 0)) : before;
            }
            before += of_lane(run, 63);
        }
        if (chunk < 0) {  // rounding: behind the last sum
            chunk = last;
            base = last_base;
        }
        if (lane == 0) {
            s_chunk = chunk;
            s_aim = aim - base;
            s_from = rest ? 2 : without >= 0 ? 1 : 0;
        }
    }
    __syncthreads();
    rest = s_from == 2;
    if (s_from == 0) without = -1;
    const double aim = s_aim;
    const int i = s_chunk * kVerifyChunk + tid * N;
    double x[N] = {}, run = 0.0;
    if (tid < kDraw) row_weights<PR>(p, at, rest, without, i, q, table, x);  // whole waves
#pragma unroll
    for (int k = 0; k < N; ++k) run += x[k];
    const double upto = scan_sum(run);
    if (tid < kDraw && lane == 63) s_sum[w] = upto;
    __syncthreads();
    double base = upto - run;  // the sum before this thread's tokens
#pragma unroll
    for (int v = 0; v < kDraw / kWave; ++v) base += v < w ? s_sum[v] : 0.0;
    int found = 0x7fffffff, last = -1;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        base += x[k];
        if (x[k] > 0.0) {
            last = i + k;
            if (base > aim && found == 0x7fffffff) found = i + k;
        }
    }
    // Lanes and waves are in the tokens' order: the first one's that found it, or the last one's that holds any.
    const uint64_t finds = __ballot(found != 0x7fffffff), holds = __ballot(last >= 0);
    const int first_found = __builtin_amdgcn_readlane(found, max(__ffsll((unsigned long long)finds) - 1, 0));
    const int last_held = __builtin_amdgcn_readlane(last, max(63 - (int)__clzll((long long)holds), 0));
    if (tid < kDraw && lane == 0) {
        s_found[w] = finds ? first_found : -1;
        s_last[w] = last_held;
    }
    __syncthreads();
    if (tid == 0) {
        int token = -1, least = -1;
#pragma unroll
        for (int v = kDraw / kWave - 1; v >= 0; --v) {
            if (s_found[v] >= 0) token = s_found[v];
            if (least < 0) least = s_last[v];
        }
        p.next_token[b] = token >= 0 ? token : least;
    }
}

namespace {

template <Prec PR>
hipError_t launch_verify(const VerifyParams &p, hipStream_t s) {
    if (p.rows > 0) {
        const int per = kThreads / kWave, rows = p.rows * (p.draft ? 2 : 1);
        for (int r = 0; r < rows; r += kVerifyLaunch)
            hipLaunchKernelGGL(verify_stats_kernel<PR>, dim3((unsigned)((p.chunks + per - 1) / per), (unsigned)std::min(rows - r, kVerifyLaunch)),
                               dim3(kThreads), 0, s, p, r);
        if (p.draft) {  // about as many workgroups as run at once, as each decides first, with about as many chunks each
            const int units = (p.chunks + kRestChunks - 1) / kRestChunks, fit = std::max(kRestFit * kCUs / p.n, 1);
            const int rounds = (units + fit - 1) / fit;
            hipLaunchKernelGGL(verify_rest_kernel<PR>, dim3((unsigned)((units + rounds - 1) / rounds), (unsigned)p.n), dim3(kRest), 0, s, p);
        }
    }
    hipLaunchKernelGGL(verify_token_kernel<PR>, dim3((unsigned)p.n), dim3(kToken), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_verify(bool bf16, const VerifyParams &p, hipStream_t s) {
    if (p.n < 1 || p.n > kPagedMaxSeqs || p.rows < 0 || p.vocab < 1 || p.chunks != (p.vocab - 1) / kVerifyChunk + 1 ||
        (int64_t)p.rows * p.chunks * 2 > INT32_MAX - kVerifyLaunch)
        return hipErrorInvalidValue;
    return bf16 ? launch_verify<Prec::BF16>(p, s) : launch_verify<Prec::F32>(p, s);
}

}  // namespace cllm

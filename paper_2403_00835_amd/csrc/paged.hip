// Paged KV cache on gfx950: the books of the page pool, and the step's keys and values into it.
//
// A pool holds n_pages pages of page_size tokens; a request (slot) owns the pages that its tokens
// need, listed in its row of the block table. A plan makes the requests of a step own exactly the
// pages of their lengths and lays out the step's rows; it runs in one workgroup, so that lengths that
// live on the device (accepted counts of a Jacobi step) need no host round trip.
#include <algorithm>

#include "device.h"
#include "paged.h"

namespace cllm {

namespace {

constexpr int kPlanThreads = kPagedMaxSeqs;
static_assert(kPlanThreads == 1024, "one thread per request");

// Exclusive prefix sum over the workgroup; total: the sum. s_wave: 16 words of LDS.
__device__ __forceinline__ int block_scan(int v, int *s_wave, int &total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const int y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();
    if (lane == 63) s_wave[w] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kPlanThreads / kWave; ++i) {
        const int t = s_wave[i];
        before += i < w ? t : 0;
        all += t;
    }
    total = all;
    return before + x - v;
}

// The entry e with start[e] <= i < start[e + 1] (start: n + 1 ascending words of LDS).
__device__ __forceinline__ int entry_of(const int *start, int n, int i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= i)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

}  // namespace

// The stack of free pages (page 0 on top), empty tables, and the rotary factors: angle
// t * base^(-2 j / hd) in double, rounded once to fp32.
__global__ void paged_init_kernel(PagedBooks bk, float *rcos, float *rsin, int64_t n_rot, int hd, double base) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < bk.n_pages) bk.free_list[i] = bk.n_pages - 1 - (int)i;
    if (i < (int64_t)bk.max_seqs * bk.max_pages) bk.table[i] = -1;
    if (i < bk.max_seqs) bk.seq_pages[i] = 0;
    if (i < PS_WORDS) bk.status[i] = i == PS_FREE ? bk.n_pages : 0;
    if (i < n_rot) {
        const int h2 = hd / 2, j = (int)(i % h2);
        const double ang = (double)(i / h2) * pow(base, -2.0 * j / (double)hd);
        rcos[i] = (float)cos(ang);
        rsin[i] = (float)sin(ang);
    }
}

// One workgroup, one thread per request for the lengths, then all threads over the pages and rows.
// Pages go back before any is taken: the last request's last page first; they are taken request after
// request. So giving back what a step took restores the stack, whatever the requests. A refused plan
// (bad slot or length, more rows than the bound, too few pages) leaves the books as they were and has
// no rows.
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(PagedPlanParams p) {
    __shared__ int s_wave[kPlanThreads / kWave];
    __shared__ int s_rows[kPlanThreads + 1], s_give[kPlanThreads + 1], s_take[kPlanThreads + 1];
    __shared__ int s_seq[kPlanThreads], s_ctx[kPlanThreads], s_own[kPlanThreads];
    __shared__ uint32_t s_seen[kPagedMaxSeqs / 32];
    const PagedBooks bk = p.bk;
    const int b = threadIdx.x, n = p.n, P = 1 << bk.page_shift;
    if (b < kPagedMaxSeqs / 32) s_seen[b] = 0;
    const int free0 = bk.status[PS_FREE];
    int seq = 0, ctx = 0, m = 0;
    if (b < n) {
        seq = p.seq[b];
        ctx = p.ctx[b];
        m = p.neu[b];
    }
    __syncthreads();
    bool bad = false;
    int own = 0, need = 0;
    if (b < n) {
        bad = seq < 0 || seq >= bk.max_seqs || ctx < 0 || m < 0 || m > p.max_new || ctx > p.max_len - m;
        if (!bad) {
            bad = (atomicOr(&s_seen[seq >> 5], 1u << (seq & 31)) >> (seq & 31)) & 1;  // the slot appears twice
            own = bk.seq_pages[seq];
            need = (ctx + m + P - 1) >> bk.page_shift;
        } else {
            m = 0;
        }
    }
    int flags = __syncthreads_or(bad) ? PF_ARG : 0;
    // 1024 requests of at most 2^20 new tokens: the sums fit 31 bits
    int R, G, T;
    const int give = max(own - need, 0), take = max(need - own, 0);
    const int r0 = block_scan(m, s_wave, R), g0 = block_scan(give, s_wave, G), t0 = block_scan(take, s_wave, T);
    if (R > p.rows) flags |= PF_ROWS;
    if (T > free0 + G) flags |= PF_PAGES;
    if (flags) {  // uniform
        if (b == 0) {
            bk.status[PS_ROWS] = bk.status[PS_ENTRIES] = bk.status[PS_UNITS] = bk.status[PS_ITEMS] = 0;
            bk.status[PS_FLAGS] = flags;
            bk.status[PS_LATE] = 0;
        }
        return;
    }
    s_seq[b] = seq;
    s_ctx[b] = ctx;
    s_own[b] = own;
    s_rows[b] = r0;
    s_give[b] = g0;
    s_take[b] = t0;
    if (b == 0) {
        s_rows[kPlanThreads] = R;
        s_give[kPlanThreads] = G;
        s_take[kPlanThreads] = T;
    }
    __syncthreads();
    for (int i = b; i < G; i += kPlanThreads) {
        const int e = entry_of(s_give, n, i), k = i - s_give[e];
        int32_t *at = bk.table + (size_t)s_seq[e] * bk.max_pages + s_own[e] - 1 - k;
        bk.free_list[free0 + G - s_give[e + 1] + k] = *at;
        *at = -1;
    }
    __syncthreads();
    for (int i = b; i < T; i += kPlanThreads) {
        const int e = entry_of(s_take, n, i);
        bk.table[(size_t)s_seq[e] * bk.max_pages + s_own[e] + i - s_take[e]] = bk.free_list[free0 + G - 1 - i];
    }
    if (b < n) {
        bk.seq_pages[seq] = need;
        bk.ent[b] = int4{seq, ctx, m, r0};
        bk.row_start[b] = r0;
    }
    if (b == 0) bk.row_start[n] = R;
    __syncthreads();
    for (int i = b; i < R; i += kPlanThreads) {
        const int e = entry_of(s_rows, n, i), pos = s_ctx[e] + i - s_rows[e];
        const int page = bk.table[(size_t)s_seq[e] * bk.max_pages + (pos >> bk.page_shift)];
        bk.row_slot[i] = (page << bk.page_shift) + (pos & (P - 1));
        bk.row_pos[i] = pos;
    }
    // Attention units: row blocks of a request, each with all the keys that its rows see, or, where
    // they are too few to fill the card, one unit per span of keys (if the partials hold them).
    const int T0 = m * p.group, nrb = (T0 + kPagedBlockRows - 1) / kPagedBlockRows;
    int U, u0 = block_scan(nrb, s_wave, U), I = 0, i0 = 0, p0 = 0;
    bool split = U * p.n_kv < kPagedSplitBelow;
    auto spans_of = [&](int rb) {
        return (ctx + min(m - 1, (rb * kPagedBlockRows + kPagedBlockRows - 1) / p.group)) / kPagedSpanKeys + 1;
    };
    auto rows_of = [&](int rb) { return min(kPagedBlockRows, T0 - rb * kPagedBlockRows); };
    if (split) {
        int nu = 0, ni = 0, np = 0;
        for (int rb = 0; rb < nrb; ++rb) {
            const int sp = spans_of(rb);
            nu += sp;
            ni += sp > 1;
            np += sp > 1 ? sp * rows_of(rb) : 0;
        }
        int U1, I1, P1;
        const int u1 = block_scan(nu, s_wave, U1), i1 = block_scan(ni, s_wave, I1), p1 = block_scan(np, s_wave, P1);
        split = U1 <= p.cap_units && I1 <= p.cap_items && P1 <= p.cap_part;
        if (split) U = U1, u0 = u1, I = I1, i0 = i1, p0 = p1;
    }
    for (int rb = 0; rb < nrb; ++rb) {
        const int sp = split ? spans_of(rb) : 1;
        if (sp == 1) {
            bk.units[u0++] = int4{b, rb, -1, -1};
            continue;
        }
        bk.items[i0++] = int4{b, rb, p0, sp};
        for (int s = 0; s < sp; ++s) {
            bk.units[u0++] = int4{b, rb, s, p0};
            p0 += rows_of(rb);
        }
    }
    if (b == 0) {
        bk.status[PS_ROWS] = R;
        bk.status[PS_ENTRIES] = n;
        bk.status[PS_FLAGS] = 0;
        bk.status[PS_FREE] = free0 + G - T;
        bk.status[PS_UNITS] = U;
        bk.status[PS_ITEMS] = I;
        bk.status[PS_BOUND_ROWS] = p.rows;
        bk.status[PS_BOUND_NEW] = p.max_new;
        bk.status[PS_BOUND_LEN] = p.max_len;
        bk.status[PS_LATE] = 0;
    }
}

// Rows of the step: queries and keys turned by their positions (rotate-half: (a c - b s, b c + a s) of
// a head's halves a, b), in fp32 and rounded once; keys and values into their slots. A thread takes
// 16 bytes of each half of one head of one row.
template <Prec PR>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendParams p) {
    using PT = PrecT<PR>;
    using T = typename PT::T;
    constexpr int VEC = PT::VEC;
    const int R = bounded_rows(p.bk, p.rows, p.max_new, p.max_len);
    const int h2 = p.hd / 2, nv = h2 / VEC, heads = p.n_heads + 2 * p.n_kv, h_first = p.q ? 0 : p.n_heads;
    const int per_row = (heads - h_first) * nv;
    const int64_t total = (int64_t)R * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int r = (int)(i / per_row), w = (int)(i % per_row), h = h_first + w / nv, j = (w % nv) * VEC;
        const int slot = p.bk.row_slot[r], pos = p.bk.row_pos[r];
        const bool isq = h < p.n_heads, isk = !isq && h < p.n_heads + p.n_kv;
        const int hk = isq ? h : isk ? h - p.n_heads : h - p.n_heads - p.n_kv;
        const T *src = isq ? (const T *)p.q + (size_t)r * p.q_stride : isk ? (const T *)p.k + (size_t)r * p.k_stride
                                                                         : (const T *)p.v + (size_t)r * p.v_stride;
        src += hk * p.hd + j;
        T *dst;
        if (isq) {
            dst = (T *)p.q_out + (size_t)r * p.q_out_stride + hk * p.hd + j;
        } else {
            const int page = slot >> p.bk.page_shift, off = slot & ((1 << p.bk.page_shift) - 1);
            dst = (T *)(isk ? p.k_pages : p.v_pages) +
                  (((((size_t)page * p.n_kv + hk) << p.bk.page_shift) + off) * p.hd + j);
        }
        alignas(16) T a[VEC], b[VEC];
        *reinterpret_cast<u32x4 *>(a) = *reinterpret_cast<const u32x4 *>(src);
        *reinterpret_cast<u32x4 *>(b) = *reinterpret_cast<const u32x4 *>(src + h2);
        if (p.rcos && (isq || isk)) {
            alignas(16) float c[VEC], s[VEC];
#pragma unroll
            for (int q = 0; q < VEC / 4; ++q) {
                *reinterpret_cast<f32x4 *>(c + 4 * q) = *reinterpret_cast<const f32x4 *>(p.rcos + (size_t)pos * h2 + j + 4 * q);
                *reinterpret_cast<f32x4 *>(s + 4 * q) = *reinterpret_cast<const f32x4 *>(p.rsin + (size_t)pos * h2 + j + 4 * q);
            }
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                const float x = from_elem<PR>(a[q]), y = from_elem<PR>(b[q]);
                a[q] = to_elem<PR>(x * c[q] - y * s[q]);
                b[q] = to_elem<PR>(y * c[q] + x * s[q]);
            }
        }
        *reinterpret_cast<u32x4 *>(dst) = *reinterpret_cast<const u32x4 *>(a);
        *reinterpret_cast<u32x4 *>(dst + h2) = *reinterpret_cast<const u32x4 *>(b);
    }
}

hipError_t launch_paged_init(const PagedBooks &bk, float *rcos, float *rsin, int max_ctx, int hd, double rope_base,
                             hipStream_t s) {
    const int64_t n_rot = rcos ? (int64_t)max_ctx * (hd / 2) : 0;
    const int64_t n = std::max({n_rot, (int64_t)bk.max_seqs * bk.max_pages, (int64_t)bk.n_pages, (int64_t)PS_WORDS});
    hipLaunchKernelGGL(paged_init_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, bk, rcos, rsin, n_rot, hd,
                       rope_base);
    return hipGetLastError();
}

hipError_t launch_paged_plan(const PagedPlanParams &p, hipStream_t s) {
    if (p.n < 1 || p.n > kPagedMaxSeqs || p.bk.max_seqs > kPagedMaxSeqs) return hipErrorInvalidValue;
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_paged_append(bool bf16, const PagedAppendParams &p, hipStream_t s) {
    const int vec = bf16 ? 8 : 4;
    if (p.hd % (2 * vec) != 0 || p.rows < 0) return hipErrorInvalidValue;
    if (p.rows == 0) return hipSuccess;
    const int64_t n = (int64_t)p.rows * ((p.q ? p.n_heads : 0) + 2 * p.n_kv) * (p.hd / 2 / vec);
    const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, 16 * kCUs));
    if (bf16)
        hipLaunchKernelGGL(paged_append_kernel<Prec::BF16>, grid, dim3(256), 0, s, p);
    else
        hipLaunchKernelGGL(paged_append_kernel<Prec::F32>, grid, dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace cllm

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

constexpr int kPlanThreads = kPagedMaxSeqs;  // at most; blockDim.x, a multiple of 256 and at least the requests
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kMany = 1 << 16;  // above a plan's bf16 row blocks
static_assert(kPlanThreads == 1024 && kPlanWaves == 16, "one thread per request, one row of lanes for the waves' sums");

// Inclusive prefix sum over a row of 16 lanes, over a wave: lane moves in the ALU (a step through LDS
// shuffles took ten times as long).
__device__ __forceinline__ int row_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // the lane 1, 2, 4, 8 before, in its row
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    return x;
}
__device__ __forceinline__ int wave_scan(int x) {
    x = row_scan(x);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 of a row to the next, rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
    return x;
}

// Exclusive prefix sums of N values over the workgroup, in place; total: the sums. s_wave: LDS, zero past
// the workgroup's waves.
template <int N>
__device__ __forceinline__ void block_scan(int (&v)[N], int (&total)[N], int (&s_wave)[N][kPlanWaves]) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = wave_scan(v[k]);
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) s_wave[k][w] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int t = row_scan(s_wave[k][lane & (kPlanWaves - 1)]);
        total[k] = __builtin_amdgcn_readlane(t, kPlanWaves - 1);
        const int before = w > 0 ? __builtin_amdgcn_readlane(t, w - 1) : 0;
        v[k] = before + x[k] - v[k];
    }
}

// The entry e with start[e] <= i < start[e + 1] of a wave's uniform item i (start: n + 1 ascending words of
// LDS): 16 entries apart, then between.
__device__ __forceinline__ int entry_of(const int *start, int n, int i) {
    const int lane = threadIdx.x & 63;
    const uint64_t far = __ballot(16 * lane < n && start[min(16 * lane, n)] <= i);
    const int c = 16 * (__popcll(far) - 1);
    const uint64_t near = __ballot(lane < 16 && c + lane < n && start[min(c + lane, n)] <= i);
    return c + __popcll(near) - 1;
}

// f(e, i) for all items i < total of the entries, every PER-th one and the entry that it is in: a wave takes
// runs of 64. The entries of a run's first and last item by the whole wave, those between by a search in
// that window (a search per lane over all entries is bound by LDS conflicts, and the kernel, on one CU,
// by its instructions).
template <int PER, class F>
__device__ __forceinline__ void for_items(const int *start, int n, int total, F f) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int i0 = w * kWave * PER; i0 < total; i0 += blockDim.x * PER) {
        const int i = i0 + lane * PER, last = min(i0 + (kWave - 1) * PER, total - 1);
        int e = entry_of(start, n, i0);
        const int window = entry_of(start, n, last) - e;
        int step = 1;
        while (step <= window) step <<= 1;
        for (step >>= 1; step > 0; step >>= 1) {
            const int at = min(e + step, n);
            if (at < n && start[at] <= i) e = at;
        }
        if (i < total) f(e, i);
    }
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
// Bound: one CU's latency: four barriers and sums, then a round trip per dependent read (lengths, pages owned,
// table). 16 requests of 32 tokens: 6.6 us, giving their pages back 3.4; 512 of 1 to 64: 26 and 8.7, of which the
// rows' slots are most: work that one CU does here for a step of 16,000 rows.
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(PagedPlanParams p) {
    __shared__ int s_wave[8][kPlanWaves], s_wave2[5][kPlanWaves];
    __shared__ int s_rows[kPlanThreads + 1], s_give[kPlanThreads + 1], s_take[kPlanThreads + 1];
    __shared__ int s_unit[kPlanThreads + 1], s_tile[kPlanThreads + 1], s_item[kPlanThreads + 1], s_part[kPlanThreads], s_ranges[kPlanThreads];
    __shared__ int s_seq[kPlanThreads], s_ctx[kPlanThreads], s_m[kPlanThreads], s_own[kPlanThreads];
    __shared__ uint32_t s_seen[kPagedMaxSeqs / 32];
    const PagedBooks bk = p.bk;
    const int b = threadIdx.x, n = p.n, P = 1 << bk.page_shift, row_shift = 31 - __clz(p.block_rows);
    const int free0 = bk.status[PS_FREE];
    int seq = 0, ctx = 0, m = 0;
    if (b < n) {
        seq = p.seq[b];
        ctx = p.ctx[b];
        m = p.neu[b];
    }
    if (b < kPagedMaxSeqs / 32) s_seen[b] = 0;
    if (b < 8 * kPlanWaves) (&s_wave[0][0])[b] = 0;
    if (b < 5 * kPlanWaves) (&s_wave2[0][0])[b] = 0;
    __syncthreads();
    bool bad = false;
    int own = 0, need = 0;
    if (b < n) {
        bad = seq < 0 || seq >= bk.max_seqs || ctx < 0 || m < 0 || m > p.max_new || ctx > p.max_len - m;
        if (!bad) {
            own = bk.seq_pages[seq];
            need = (ctx + m + P - 1) >> bk.page_shift;
            bad = (atomicOr(&s_seen[seq >> 5], 1u << (seq & 31)) >> (seq & 31)) & 1;  // the slot appears twice
        }
        if (bad) m = 0;
    }
    int flags = __syncthreads_or(bad) ? PF_ARG : 0;
    // (1024 requests of at most 2^20 new tokens: the sum of those fits 31 bits, and the others' are used only where
    // it is within max_rows: at most 2^20 tokens of up to 2^10 rows)
    const int T0 = m * p.group;  // rows of the request's attention
    const bool tiled = p.tiled && T0 > kPagedFewRows;
    const int nrb = tiled ? 0 : (T0 + p.block_rows - 1) / p.block_rows;
    const bool many = p.tiled && !tiled && T0 > kPagedWaveRows;
    const int ntile = tiled ? (T0 + kPagedTileRows - 1) / kPagedTileRows : 0;
    const int spans = (ctx + max(m, 1) - 1) / kPagedSpanKeys + 1;
    // Partial rows that splitting the request's row blocks takes. Requests of few rows have the first places in the
    // partials: they always fit, but for fp32 pools of 2^20 such rows. Larger ones (fp32) come behind; one that alone
    // is too large takes no place.
    const int64_t rows_spans = (int64_t)T0 * spans;
    const bool first = T0 <= kPagedFewRows;
    const int want = nrb && spans > 1 && rows_spans <= p.cap_part ? (int)rows_spans : 0;
    // (bf16 row blocks, at most 4 each, take 13 bits: above them the number of requests that may be taken whole)
    int v[8] = {m, max(own - need, 0), max(need - own, 0), many ? nrb + kMany : nrb, ntile, want ? nrb * spans : nrb,
                first ? want : 0, first ? 0 : want}, total[8];
    block_scan(v, total, s_wave);
    const int wholes = p.tiled ? total[3] / kMany : 0;
    total[3] -= wholes * kMany;
    const int R = total[0], G = total[1], T = total[2];
    if (R > p.rows) flags |= PF_ROWS;
    if (T > free0 + G) flags |= PF_PAGES;
    if (flags) {  // uniform
        if (b == 0) {
            bk.status[PS_ROWS] = bk.status[PS_ENTRIES] = bk.status[PS_UNITS] = bk.status[PS_TILES] = bk.status[PS_ITEMS] = 0;
            bk.status[PS_FLAGS] = flags;
            bk.status[PS_LATE] = 0;
        }
        return;
    }
    // Attention units. Row blocks: as many spans of the request's keys (up to its last token: a unit of
    // spans that its block does not see does nothing) as make about kPagedUnits workgroups of the plan, a
    // partial state per span where there are several; a request that the partials do not hold (fp32) walks its spans
    // in one unit. Tiles: ranges of keys, as many as make about kPagedTileGroups workgroups of the plan's tiles, none
    // under a span's keys. (Units: nrb (spans / per + 1) summed is at most kPagedUnits / n_kv and the row blocks.
    // Ranges: only fewer than kPagedTileGroups / n_kv tiles are split, into at most that many more. Both are
    // within what the cache has room for.)
    const int per = max((int)(((int64_t)total[5] * p.n_kv + kPagedUnits - 1) / kPagedUnits), 1);
    const int ranges = total[4] > 0 ? (kPagedTileGroups + total[4] * p.n_kv - 1) / (total[4] * p.n_kv) : 1;
    const int nr = ntile ? min(ranges, spans) : 1, items = (T0 + kPagedItemRows - 1) / kPagedItemRows;
    // Whole requests, without partials: see kPagedWaveRows. None is taken whole where one has more than twice the
    // mean keys and would be worked on alone at the end.
    const bool late = many && (int64_t)spans * total[3] > 2 * (int64_t)total[5];
    const bool whole = wholes * p.n_kv >= kPagedTileGroups && !__syncthreads_or(late) && many;  // (uniform but for the last)
    const int place = first ? v[6] : total[6] + v[7];
    const bool dparts = want && !whole && place <= p.cap_part - want, tparts = nr > 1;
    int x[5] = {whole ? 1 : nrb * (dparts ? (spans + per - 1) / per : 1), dparts ? items : 0, ntile * nr, tparts ? items : 0,
                tparts ? nr * T0 : 0}, y[5];
    block_scan(x, y, s_wave2);
    const int U = y[0], UT = y[2], I = y[1] + y[3];
    s_seq[b] = seq;
    s_ctx[b] = ctx;
    s_m[b] = m;
    s_own[b] = own;
    s_rows[b] = v[0];
    s_give[b] = v[1];
    s_take[b] = v[2];
    s_unit[b] = x[0];
    s_tile[b] = x[2];
    s_item[b] = x[1] + x[3];
    s_part[b] = dparts ? place : tparts ? p.cap_part + x[4] : -1;
    s_ranges[b] = ntile ? nr : whole ? -1 : 0;
    if (b == 0) {  // behind the last thread's
        const int end = blockDim.x;
        s_rows[end] = R;
        s_give[end] = G;
        s_take[end] = T;
        s_unit[end] = U;
        s_tile[end] = UT;
        s_item[end] = I;
    }
    __syncthreads();
    if (G > 0) {  // uniform
        auto at = [&](int e, int i) { return bk.table + (size_t)s_seq[e] * bk.max_pages + s_own[e] - 1 - (i - s_give[e]); };
        for_items<1>(s_give, n, G, [&](int e, int i) { bk.free_list[free0 + G - s_give[e + 1] + i - s_give[e]] = *at(e, i); });
        __syncthreads();  // before the entries are cleared, and taken from the list
        for_items<1>(s_give, n, G, [&](int e, int i) { *at(e, i) = -1; });
    }
    // Pages taken, and the rows: a row's page is an old entry of the table or a new one, read off the stack
    // here too, so the rows need not wait for the table.
    if (T > 0)
        for_items<1>(s_take, n, T, [&](int e, int i) {
            bk.table[(size_t)s_seq[e] * bk.max_pages + s_own[e] + i - s_take[e]] = bk.free_list[free0 + G - 1 - i];
        });
    if (R > 0)
        for_items<4>(s_rows, n, R, [&](int e, int i) {
            alignas(16) int slot[4], pos[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int row = min(i + k, R - 1);
                while (s_rows[e + 1] <= row) ++e;
                pos[k] = s_ctx[e] + row - s_rows[e];
                const int at = pos[k] >> bk.page_shift, fresh = at - s_own[e];
                slot[k] = fresh < 0 ? bk.table[(size_t)s_seq[e] * bk.max_pages + at]
                                    : bk.free_list[free0 + G - 1 - s_take[e] - fresh];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) slot[k] = (slot[k] << bk.page_shift) + (pos[k] & (P - 1));
            if (i + 4 <= R) {
                *reinterpret_cast<u32x4 *>(bk.row_slot + i) = *reinterpret_cast<const u32x4 *>(slot);
                *reinterpret_cast<u32x4 *>(bk.row_pos + i) = *reinterpret_cast<const u32x4 *>(pos);
            } else {
                for (int k = 0; i + k < R; ++k) {
                    bk.row_slot[i + k] = slot[k];
                    bk.row_pos[i + k] = pos[k];
                }
            }
        });
    if (b < n) {
        bk.seq_pages[seq] = need;
        bk.row_start[b] = v[0];
    }
    if (b == 0) bk.row_start[n] = R;
    if (U > 0)
        for_items<1>(s_unit, n, U, [&](int e, int i) {
            const int rows = s_m[e] * p.group, blocks = (rows + p.block_rows - 1) >> row_shift, part = s_part[e];
            if (s_ranges[e] < 0) {
                bk.units[i] = PagedUnit{s_seq[e], s_ctx[e], s_m[e], s_rows[e], 0, -1, kAllSpans, -1};
                return;
            }
            // the blocks of the same spans next to each other: they read the same keys
            int k0 = i - s_unit[e], row = 0;
            if (blocks > 1) {
                row = k0 % blocks << row_shift;
                k0 = k0 / blocks;
            }
            k0 = part < 0 ? 0 : k0 * per;  // no partials: one span, or all
            bk.units[i] = PagedUnit{s_seq[e], s_ctx[e], s_m[e], s_rows[e], row, k0, part < 0 ? kAllSpans : k0 + per,
                                    part < 0 ? -1 : part + k0 * rows + row};
        });
    if (UT > 0)
        for_items<1>(s_tile, n, UT, [&](int e, int i) {
            const int rows = s_m[e] * p.group, tiles = (rows + kPagedTileRows - 1) / kPagedTileRows, part = s_part[e];
            const int ranges = s_ranges[e], k = i - s_tile[e], j = k / tiles;
            const int row = (tiles - 1 - (k - j * tiles)) * kPagedTileRows;  // the tiles that see most keys first
            const int chunks = (s_ctx[e] + s_m[e] + kAttnChunk - 1) / kAttnChunk, len = (chunks + ranges - 1) / ranges;
            bk.tiles[i] = PagedUnit{s_seq[e], s_ctx[e], s_m[e], s_rows[e], row, j * len, min(chunks, (j + 1) * len),
                                    part < 0 ? -1 : part + j * rows + row};
        });
    if (I > 0)
        for_items<1>(s_item, n, I, [&](int e, int i) {
            const int row = (i - s_item[e]) * kPagedItemRows;
            bk.items[i] = PagedItem{s_ctx[e], s_m[e], s_rows[e], row, s_part[e] + row, s_m[e] * p.group, s_ranges[e], 0};
        });
    if (b == 0) {
        bk.status[PS_ROWS] = R;
        bk.status[PS_ENTRIES] = n;
        bk.status[PS_FLAGS] = 0;
        bk.status[PS_FREE] = free0 + G - T;
        bk.status[PS_UNITS] = U;
        bk.status[PS_TILES] = UT;
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
// Bound: memory: 197 MB (5 prompts, 8000 rows of 32 and 8 heads of 128) in 31 us, 6.3 TB/s (some of it in the
// last-level cache); 512 rows 6.0 us, 8 rows 2.2.
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
    // four waves unless there are requests or rows for more (16 requests: 4 us with four waves, 6 with sixteen)
    const int threads = p.n <= 256 && p.rows <= 2048 ? 256 : kPlanThreads;
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(threads), 0, s, p);
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

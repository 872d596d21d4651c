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
__global__ void paged_init_kernel(PagedBooks bk, float *rcos, float *rsin, int64_t n_rot, int hd, double base, int form) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < bk.n_pages) bk.free_list[i] = bk.n_pages - 1 - (int)i;
    if (i < (int64_t)bk.max_seqs * bk.max_pages) bk.table[i] = -1;
    if (i < bk.max_seqs) bk.seq_pages[i] = 0;
    if (i < PS_WORDS) bk.status[i] = i == PS_FREE ? bk.n_pages : i == PS_FORM && rcos ? form : 0;
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
            bk.status[PS_LATE] = bk.status[PS_OTHER] = 0;
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
        bk.entries[b] = PagedEntry{seq, ctx, m, v[0], dparts ? place : -1, whole ? PE_WHOLE : tiled ? PE_TILED : PE_BLOCKS, {0, 0}};
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
        bk.status[PS_LATE] = bk.status[PS_OTHER] = 0;
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
    const int R = append_rows(p);
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

// Factors of one pair j at every position: cos and sin of t * f[j] in double, times the magnitude, rounded once.
__global__ __launch_bounds__(256) void paged_rotary_kernel(PagedBooks bk, float *rcos, float *rsin, int max_ctx, int rot, int form,
                                                           double magnitude, PagedFreqs f) {
    const int t = (int)blockIdx.x * 256 + threadIdx.x, j = blockIdx.y;
    if (t == 0 && j == 0) bk.status[PS_FORM] = form;
    if (t >= max_ctx) return;
    const double ang = (double)t * f.f[j];
    rcos[(size_t)t * rot + j] = (float)(cos(ang) * magnitude);
    rsin[(size_t)t * rot + j] = (float)(sin(ang) * magnitude);
}

namespace {

// Sum over the nv (2, 4, 8 or 16) neighbouring lanes of a head, in every one of them.
__device__ __forceinline__ float head_sum(float x, int nv) {
    auto add = [](float a, int moved) { return a + __int_as_float(moved); };
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xb1, 0xf, 0xf, true));                // lane ^ 1
    if (nv >= 4) x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4e, 0xf, 0xf, true));   // lane ^ 2
    if (nv >= 8) x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true));  // 8 lanes mirrored
    if (nv >= 16) x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x140, 0xf, 0xf, true)); // 16 lanes mirrored
    return x;
}

typedef f32x4 f32x4_a4 __attribute__((aligned(4)));  // a vector of floats at any float's address

template <int N>
__device__ __forceinline__ void load_floats(float (&x)[N], const float *src) {
    if constexpr (N == 2) {
        x[0] = src[0], x[1] = src[1];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4_a4 *>(src + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i + e] = v[e];
        }
    }
}

// Values rounded to elements (bf16: two an instruction).
template <Prec PR, int N>
__device__ __forceinline__ void round_all(typename PrecT<PR>::T (&z)[N], const float (&y)[N]) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    if constexpr (PR == Prec::BF16) {
#pragma unroll
        for (int i = 0; i < N; i += 2)
            reinterpret_cast<uint32_t *>(z)[i / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{y[i], y[i + 1]}), bf16x2));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = y[i];
    }
}

// How a head's elements lie in its threads: thread l takes two vectors of VEC elements, each next to its neighbours' ones.
enum Pairs {
    HALVES,      // rot a multiple of VEC: the vectors' elements are the pairs (j, j + rot), behind them what is not turned
    NEIGHBOURS,  // pairs (2 j, 2 j + 1), or none: within the vectors
    SCATTERED,   // halves of other widths: the pairs are formed through LDS
};

}  // namespace

// paged_append_kernel with a norm of each query and key head before the rotation, and every form of the rotation:
// y = x / sqrt(mean(x^2) + eps) * gain in fp32, then the turned pairs, rounded once. A thread takes U heads of one
// row, whose rotary factors and gains it loads once.
// Bound: memory: 8000 rows of 32 and 8 heads of 128, 197 MB in 42.5 us, 4.6 TB/s where nothing is in the last-level cache
// (paged_append_kernel there: 39); 512 rows 6.0 us, 8 rows of 12 heads of 16 3.4. Halves of other widths (1740 rows of 36 heads of
// 64, 24 elements turned: 9.0 us): element by element from memory 18.8; all elements through LDS as vectors, with the threads'
// reads in few banks, 10.2.
template <Prec PR, Pairs F, int U>
__global__ __launch_bounds__(256) void paged_append_forms_kernel(PagedAppendParams p, int per_row, uint32_t per_row_inv, int rpb) {
    using PT = PrecT<PR>;
    using T = typename PT::T;
    constexpr int VEC = PT::VEC, H = VEC / 2;
    __shared__ float s_pairs[F == SCATTERED ? 256 * 2 * (VEC + 1) : 1];
    const int R = append_rows(p);
    const int nv = p.hd / 2 / VEC, nv_shift = 31 - __clz(nv), half = p.hd / 2;
    const int q_segs = p.q ? (p.n_heads + U - 1) / U : 0, kv_segs = (p.n_kv + U - 1) / U;
    const float inv_hd = 1.0f / (float)p.hd;  // (a power of two)
    for (int row0 = blockIdx.x * rpb; row0 < R; row0 += gridDim.x * rpb) {
        const int items = min(rpb, R - row0) * per_row;
        for (int i = threadIdx.x; i < items; i += 256) {
            const int dr = (int)__umulhi((uint32_t)i, per_row_inv), w = i - dr * per_row, r = row0 + dr;
            const int at = (w & (nv - 1)) * VEC;  // of the first vector in half a head
            int seg = w >> nv_shift;
            const bool isq = seg < q_segs, isk = !isq && seg < q_segs + kv_segs;
            seg -= isq ? 0 : isk ? q_segs : q_segs + kv_segs;
            const int heads = isq ? p.n_heads : p.n_kv, h0 = seg * U;
            const T *src = isq ? (const T *)p.q + (size_t)r * p.q_stride : isk ? (const T *)p.k + (size_t)r * p.k_stride
                                                                             : (const T *)p.v + (size_t)r * p.v_stride;
            T *dst;
            size_t head_step = p.hd;
            if (isq) {
                dst = (T *)p.q_out + (size_t)r * p.q_out_stride;
            } else {
                const int slot = p.bk.row_slot[r], page = slot >> p.bk.page_shift, off = slot & ((1 << p.bk.page_shift) - 1);
                head_step = (size_t)p.hd << p.bk.page_shift;
                dst = (T *)(isk ? p.k_pages : p.v_pages) + (size_t)page * p.n_kv * head_step + (size_t)off * p.hd;
            }
            const bool turned = (isq || isk) && (F == HALVES ? at < p.rot : p.rot > 0);
            int o0 = at, o1 = half + at;
            if (F == HALVES && turned) o1 = at + p.rot;
            if (F == HALVES && !turned && (isq || isk)) o0 = p.rot + at, o1 = half + at;  // 2 rot + (at - rot), and half the rest on
            alignas(16) T x[U][2 * VEC];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const T *s = src + min(h0 + u, heads - 1) * p.hd;
                *reinterpret_cast<u32x4 *>(x[u]) = *reinterpret_cast<const u32x4 *>(s + o0);
                *reinterpret_cast<u32x4 *>(x[u] + VEC) = *reinterpret_cast<const u32x4 *>(s + o1);
            }
            const float *gain = isq ? p.q_gain : isk ? p.k_gain : nullptr;
            float g[2 * VEC], c[VEC], s[VEC];  // c, s: of this thread's pairs
            if (gain) {
                float a[VEC], b[VEC];
                load_floats(a, gain + o0);
                load_floats(b, gain + o1);
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = a[i], g[VEC + i] = b[i];
            }
            // First pairs of the thread's two halves of them, and whether the pair is turned.
            const int j0 = F == NEIGHBOURS ? at / 2 : at, j1 = F == NEIGHBOURS ? half / 2 + at / 2 : at + H;
            auto is_turned = [&](int i) { return (i < H ? j0 + i : j1 + i - H) < p.rot; };
            if (turned) {
                const size_t t = (size_t)p.bk.row_pos[r] * p.rot;
                // (Those behind the row's last are not used; the table has hd / 2 for each position, so they are in it.)
                float a[H], b[H];
                load_floats(a, p.rcos + t + j0);
                load_floats(b, p.rsin + t + j0);
#pragma unroll
                for (int i = 0; i < H; ++i) c[i] = a[i], s[i] = b[i];
                load_floats(a, p.rcos + t + j1);
                load_floats(b, p.rsin + t + j1);
#pragma unroll
                for (int i = 0; i < H; ++i) c[H + i] = a[i], s[H + i] = b[i];
            }
            if (gain || turned) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float y[2 * VEC];
#pragma unroll
                    for (int i = 0; i < 2 * VEC; ++i) y[i] = from_elem<PR>(x[u][i]);
                    if (gain) {
                        auto squares = [&]() {
                            float ss = 0.f;
#pragma unroll
                            for (int i = 0; i < 2 * VEC; ++i) ss += y[i] * y[i];
                            return head_sum(ss, nv) * inv_hd;
                        };
                        float ms = squares(), eps = p.eps;
                        if (!(ms + eps <= 3.4e38f)) {  // past fp32: of 2^-80 of the values
#pragma unroll
                            for (int i = 0; i < 2 * VEC; ++i) y[i] *= 0x1p-80f;
                            ms = squares();
                            eps = eps * 0x1p-80f * 0x1p-80f;
                        }
                        const float f = __builtin_amdgcn_rsqf(ms + eps);  // (the instruction: one unit in the last place)
#pragma unroll
                        for (int i = 0; i < 2 * VEC; ++i) y[i] = y[i] * f * g[i];
                    }
                    if constexpr (F == SCATTERED) {
                        // The head's elements into LDS; out of it the partners of this thread's first elements, and back turned;
                        // then what others have turned. A head's threads are in one wave, whose accesses to LDS are in order.
                        // (A place is left free behind each vector, or all threads' elements would be in the same few banks.)
                        float *mine = s_pairs + (threadIdx.x & ~(nv - 1)) * 2 * (VEC + 1);
                        const uint32_t first = at / VEC * (VEC + 1), second = first + nv * (VEC + 1);
                        auto other = [&](int i) {
                            const uint32_t e = min(at + i, p.rot - 1) + p.rot;
                            return e + e / VEC;
                        };
                        if (turned) {
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                            for (int i = 0; i < VEC; ++i) {
                                mine[first + i] = y[i];
                                mine[second + i] = y[VEC + i];
                            }
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                            float b[VEC];
#pragma unroll
                            for (int i = 0; i < VEC; ++i) b[i] = mine[other(i)];
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                            for (int i = 0; i < VEC; ++i)
                                if (at + i < p.rot) {
                                    mine[other(i)] = b[i] * c[i] + y[i] * s[i];
                                    y[i] = y[i] * c[i] - b[i] * s[i];
                                }
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                            for (int i = 0; i < VEC; ++i) {
                                const float x = mine[first + i], own = y[i];
                                y[i] = at + i < p.rot ? own : x;
                                y[VEC + i] = mine[second + i];
                            }
                        }
                    } else if (turned) {
#pragma unroll
                        for (int i = 0; i < VEC; ++i) {
                            constexpr int D = F == HALVES ? VEC : 1, S = F == HALVES ? 1 : 2;
                            if (F != HALVES && !is_turned(i)) continue;  // (0 * inf)
                            const float a = y[S * i], b = y[S * i + D];
                            y[S * i] = a * c[i] - b * s[i];
                            y[S * i + D] = b * c[i] + a * s[i];
                        }
                    }
                    alignas(16) T z[2 * VEC];
                    round_all<PR>(z, y);
                    if (F != HALVES && !gain) {  // what is not turned is a copy, of a NaN's bits too
#pragma unroll
                        for (int i = 0; i < 2 * VEC; ++i)
                            if (F == NEIGHBOURS ? !is_turned(i / 2) : (i < VEC ? at + i : half + at + i - VEC) >= 2 * p.rot) z[i] = x[u][i];
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        *reinterpret_cast<u32x4 *>(x[u] + i * VEC) = *reinterpret_cast<const u32x4 *>(z + i * VEC);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (h0 + u >= heads) break;
                T *d = dst + (h0 + u) * head_step;
                *reinterpret_cast<u32x4 *>(d + o0) = *reinterpret_cast<const u32x4 *>(x[u]);
                *reinterpret_cast<u32x4 *>(d + o1) = *reinterpret_cast<const u32x4 *>(x[u] + VEC);
            }
        }
    }
}

hipError_t launch_paged_rotary(const PagedBooks &bk, float *rcos, float *rsin, int max_ctx, int rot, bool inter, double magnitude,
                               const PagedFreqs &f, hipStream_t s) {
    if (!rcos || !rsin || rot < 1 || rot > kMaxRot || max_ctx < 1) return hipErrorInvalidValue;
    hipLaunchKernelGGL(paged_rotary_kernel, dim3((unsigned)((max_ctx + 255) / 256), (unsigned)rot), dim3(256), 0, s, bk, rcos,
                       rsin, max_ctx, rot, rotary_form(rot, inter), magnitude, f);
    return hipGetLastError();
}

namespace {

template <Prec PR, Pairs F, int U>
hipError_t launch_forms(const PagedAppendParams &p, hipStream_t s) {
    const int nv = p.hd / 2 / PrecT<PR>::VEC;
    const int per_row = ((p.q ? (p.n_heads + U - 1) / U : 0) + 2 * ((p.n_kv + U - 1) / U)) * nv;
    // Rows of a workgroup: of one to four times what fills it once, where there are enough, those that leave the fewest
    // threads without work in the last round (192 items a row: one row 0.75 of a round, four rows three).
    const int base = std::max(1, 256 / per_row);
    auto rounds = [&](int rows) { return (rows * per_row + 255) / 256 * 256.0 / (rows * per_row); };
    int rpb = base;
    for (int k = 2; k <= 4 && (int64_t)p.rows >= (int64_t)k * base * 4 * kCUs && (int64_t)k * base * per_row * per_row < 1ll << 32; ++k)
        if (rounds(k * base) < 0.95 * rounds(rpb)) rpb = k * base;
    // (the quotient is exact where item * per_row is below 2^32: of one row's at most 3 * 1024 * 16 items it is)
    const uint32_t inv = (uint32_t)(((1ull << 32) + per_row - 1) / per_row);
    const dim3 grid((unsigned)std::min<int64_t>((p.rows + rpb - 1) / rpb, 16 * kCUs));
    hipLaunchKernelGGL((paged_append_forms_kernel<PR, F, U>), grid, dim3(256), 0, s, p, per_row, inv, rpb);
    return hipGetLastError();
}

template <Prec PR>
hipError_t launch_forms(const PagedAppendParams &p, hipStream_t s) {
    // Two heads a thread, whose factors and gains are loaded once, where one a thread makes more workgroups than run at once
    // (48 heads of 128, bf16: 512 rows 6.1 us in place of 7.1, 8000 rows 43.6 in place of 50.5, four heads a thread 42.5; 8 rows
    // of 12 heads of 16, fp32: 3.5 either way); halves through LDS in bf16 alone (13,800 rows of 12 heads of 128, 126 elements
    // turned: 23.9 in place of 27.3; 6300 rows of 32 heads of 64, 22 turned, fp32: 24.2 in place of 22.0).
    const bool many = p.rows >= 256;
    if (p.rot > 0 && !p.inter && p.rot % PrecT<PR>::VEC != 0) {
        if constexpr (PR == Prec::BF16)
            if (many) return launch_forms<PR, SCATTERED, 2>(p, s);
        return launch_forms<PR, SCATTERED, 1>(p, s);
    }
    if (p.inter || p.rot == 0) return many ? launch_forms<PR, NEIGHBOURS, 2>(p, s) : launch_forms<PR, NEIGHBOURS, 1>(p, s);
    return many ? launch_forms<PR, HALVES, 2>(p, s) : launch_forms<PR, HALVES, 1>(p, s);
}

}  // namespace

hipError_t launch_paged_append_forms(bool bf16, const PagedAppendParams &p, hipStream_t s) {
    const int vec = bf16 ? 8 : 4, nv = p.hd / 2 / vec;
    if (p.hd % (2 * vec) != 0 || nv < 2 || nv > 16 || (nv & (nv - 1)) != 0 || p.rows < 0 || p.rot < 0 || 2 * p.rot > p.hd ||
        (p.rot > 0 && !p.rcos))
        return hipErrorInvalidValue;
    if (p.rows == 0) return hipSuccess;
    return bf16 ? launch_forms<Prec::BF16>(p, s) : launch_forms<Prec::F32>(p, s);
}

hipError_t launch_paged_init(const PagedBooks &bk, float *rcos, float *rsin, int max_ctx, int hd, double rope_base,
                             hipStream_t s) {
    const int64_t n_rot = rcos ? (int64_t)max_ctx * (hd / 2) : 0;
    const int64_t n = std::max({n_rot, (int64_t)bk.max_seqs * bk.max_pages, (int64_t)bk.n_pages, (int64_t)PS_WORDS});
    hipLaunchKernelGGL(paged_init_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, bk, rcos, rsin, n_rot, hd,
                       rope_base, rotary_form(hd / 2, false));
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

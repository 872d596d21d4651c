// Paged KV cache of libcllm.so: kernel parameters and launchers (host and device).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cllm {

constexpr int kPagedMaxSeqs = 1024;   // one plan thread per request
// Rows of a request's attention: new tokens x heads of a group. Requests of few rows, and fp32, take units of
// paged_block_rows() rows and spans of keys; longer bf16 chunks take tiles of kPagedTileRows rows and a range of
// keys. Up to 64 rows a row's bits are those of a plan of its own: every block length of the library's decoding has
// them with one query head per key head, blocks of up to 64 / group tokens with grouped ones. Larger ones in spans, by
// tokens in place of rows, would take longer: 32 over 8 heads of 128, one block of 64 tokens at 2304 keys 26.5 us
// in place of 19.1, 16 of 17 at 1000 45.8 in place of 29.7, 64 of 32 at 2000 190 in place of 129, and the partials of a
// 1.2 GB workspace. Tiles from 33 rows on (32 heads of 128): 33 rows at 600 keys 16.6 us in place of 14.8, 64 at 2304 24
// in place of 28, 16 requests of 64 at 1000 64 in place of 69.
constexpr int kPagedFewRows = 64;
constexpr int kPagedTileRows = 128;
constexpr int kPagedItemRows = 32;    // rows that are joined together
// A wave holds a chunk of keys in registers beside its rows: of 512-byte keys, half the rows.
constexpr int paged_block_rows(bool bf16, int hd) { return hd * (bf16 ? 2 : 4) >= 512 ? 16 : 32; }
// Where bf16 requests of few, but more than kPagedWaveRows rows make kPagedTileGroups workgroups or more, a
// workgroup takes a whole request: its keys once for all rows, no partial states. 64 requests of 36 rows at 4000
// keys (8 key heads of 128): 433 us in spans, 205 whole; 16 of 64 rows at 1000 keys (32 heads): 153 and 69; of
// 32 rows: 90 and 58. Up to 16 rows spans read the keys once too, and do not wait for the longest request: a
// token of 64 requests at 1000 to 8000 keys takes 241 us in spans, 282 whole (4 tokens at 4000: 227 and 193).
constexpr int kPagedWaveRows = 16;
constexpr int kPagedSpanKeys = 256;   // keys of a span, at absolute positions
// Workgroups that the spans of a plan's row blocks make, about: above, one takes several spans. It bounds the unit
// list. 256 tokens at 1000 to 8000 keys (32 over 8 heads of 128): 960 us, 981 of 8192 workgroups, 920 of one a span;
// 64 blocks of 16 at 2000 to 9000 keys (32 heads of 64): 755, 764 and 773.
constexpr int kPagedUnits = 16384;
constexpr int kAllSpans = 1 << 30;
constexpr int kPartRows = 1 << 20;     // above the partial rows of an fp32 cache: 1024 requests' sums fit 31 bits
constexpr int kPagedTileGroups = 512;   // workgroups that fill the device (two a CU): tiles of few requests are split into
                                        // about as many

// Words of the status block, written by the plan.
enum PagedStatus {
    PS_ROWS = 0,     // rows of the plan (0 when it was refused)
    PS_ENTRIES = 1,  // requests of the plan
    PS_FLAGS = 2,    // PF_* of the plan
    PS_FREE = 3,     // free pages
    PS_UNITS = 4,    // attention units of row blocks
    PS_TILES = 5,    // attention units of tiles
    PS_BOUND_ROWS = 6, PS_BOUND_NEW = 7, PS_BOUND_LEN = 8,  // the plan's bounds
    PS_ITEMS = 9,    // row blocks whose partial states are joined
    PS_LATE = 10,    // a call made for other bounds than the plan's ran (and did nothing)
    PS_WORDS = 16
};
enum PagedFlags { PF_ARG = 1, PF_ROWS = 2, PF_PAGES = 4 };

// What one workgroup takes (per key head), and a row block whose partial states are joined.
struct alignas(16) PagedUnit {
    int slot, ctx, m, r0;  // the request: slot, context, new tokens, first row of the plan
    int row;               // first row of the block or tile
    int k0, k1;            // row blocks: spans [k0, k1), kAllSpans: to the last, k0 -1: the whole request, all rows
                           // and keys; tiles: chunks [k0, k1)
    int part;              // partial row of the first row (row blocks: in span k0), or -1: none, the output is written
};
struct alignas(16) PagedItem {
    int ctx, m, r0, row;
    int part;    // partial row of the first row in the first span or range
    int stride;  // partial rows from one span or range to the next
    int count;   // ranges; 0: the spans up to the row's position
    int pad;
};

// Device memory of a cache: the books of its pool and the last plan.
struct PagedBooks {
    int32_t *status;
    int32_t *table;      // [max_seqs][max_pages] page ids, -1 where none
    int32_t *seq_pages;  // [max_seqs]
    int32_t *free_list;  // [n_pages], a stack: the next page to take is entry status[PS_FREE] - 1
    int32_t *row_start;  // [max_seqs + 1]
    int32_t *row_slot;   // [max_rows]: page * page_size + offset
    int32_t *row_pos;    // [max_rows]
    PagedUnit *units, *tiles;
    PagedItem *items;
    int cap_units, cap_tiles, cap_items;  // entries of the three
    int max_seqs, max_pages, n_pages, page_shift;
};

struct PagedPlanParams {
    PagedBooks bk;
    const int32_t *seq, *ctx, *neu;
    int n, rows, max_new, max_len;  // the call's bounds
    int group, n_kv;                // query heads per key head, key heads
    bool tiled;                     // long chunks take tiles
    int block_rows;                 // of the others
    int cap_part;                   // partial rows of row blocks; those of tiles are behind them
};

struct PagedAppendParams {
    PagedBooks bk;
    int rows, max_new, max_len;  // the bounds that the call was made for
    const void *q, *k, *v;       // rows of q_stride (k_stride, v_stride) elements
    void *q_out, *k_pages, *v_pages;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    const float *rcos, *rsin;    // [max_ctx][hd / 2], or null: no rotation
    int n_heads, n_kv, hd;
};

struct PagedAttnParams {
    PagedBooks bk;
    int rows, max_new, max_len;
    const void *q, *k_pages, *v_pages;
    void *out;
    int64_t q_stride, out_stride;
    float *lse;                   // [rows][n_heads], or null
    float *part_o, *part_m, *part_l;  // [partial row][n_kv] (x hd)
    int n_heads, n_kv, hd, group;
    uint32_t group_inv;           // 2^24 / group, rounded up
    float scale_log2;
};

// Rows of the last plan, or none when it was made for other bounds than the call's (a replayed graph
// after another plan): the call's arrays may be smaller then, and its launches fewer.
__device__ __forceinline__ int bounded_rows(const PagedBooks &bk, int rows, int max_new, int max_len) {
    const int32_t *st = bk.status;
    const int R = st[PS_ROWS];
    if (R == 0) return 0;
    if (st[PS_BOUND_ROWS] == rows && st[PS_BOUND_NEW] == max_new && st[PS_BOUND_LEN] == max_len) return R;
    if (blockIdx.x == 0 && threadIdx.x == 0) bk.status[PS_LATE] = 1;
    return 0;
}

hipError_t launch_paged_init(const PagedBooks &bk, float *rcos, float *rsin, int max_ctx, int hd,
                             double rope_base, hipStream_t s);
hipError_t launch_paged_plan(const PagedPlanParams &p, hipStream_t s);
hipError_t launch_paged_append(bool bf16, const PagedAppendParams &p, hipStream_t s);
// Upper bounds of the plan's units and tiles; join: some may be split.
hipError_t launch_paged_attn(bool bf16, int64_t units, bool whole, int64_t tiles, bool join, const PagedAttnParams &p, hipStream_t s);

}  // namespace cllm

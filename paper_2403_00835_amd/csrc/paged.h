// Paged KV cache of libcllm.so: kernel parameters and launchers (host and device).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cllm {

constexpr int kPagedMaxSeqs = 1024;   // one plan thread per request
constexpr int kPagedBlockRows = 64;   // query rows (row x head of a group) of one attention unit
constexpr int kPagedSpanKeys = 512;   // keys of a span, at absolute positions: what a split unit takes
constexpr int kPagedSplitBelow = 512; // workgroups below which long contexts are split into spans

// Words of the status block, written by the plan.
enum PagedStatus {
    PS_ROWS = 0,     // rows of the plan (0 when it was refused)
    PS_ENTRIES = 1,  // requests of the plan
    PS_FLAGS = 2,    // PF_* of the plan
    PS_FREE = 3,     // free pages
    PS_UNITS = 4,    // attention units
    PS_ITEMS = 5,    // split row blocks, whose spans are joined
    PS_BOUND_ROWS = 6, PS_BOUND_NEW = 7, PS_BOUND_LEN = 8,  // the plan's bounds
    PS_LATE = 9,     // a call made for other bounds than the plan's ran (and did nothing)
    PS_WORDS = 16
};
enum PagedFlags { PF_ARG = 1, PF_ROWS = 2, PF_PAGES = 4 };

// Device memory of a cache: the books of its pool and the last plan.
struct PagedBooks {
    int32_t *status;
    int32_t *table;      // [max_seqs][max_pages] page ids, -1 where none
    int32_t *seq_pages;  // [max_seqs]
    int32_t *free_list;  // [n_pages], a stack: the next page to take is entry status[PS_FREE] - 1
    int32_t *row_start;  // [max_seqs + 1]
    int32_t *row_slot;   // [max_rows]: page * page_size + offset
    int32_t *row_pos;    // [max_rows]
    int4 *ent;           // per request: slot, context, new tokens, first row
    int4 *units;         // request, row block, span (-1: all of them), partial row (-1: none)
    int4 *items;         // request, row block, first partial row, spans
    int max_seqs, max_pages, n_pages, page_shift;
};

struct PagedPlanParams {
    PagedBooks bk;
    const int32_t *seq, *ctx, *neu;
    int n, rows, max_new, max_len;  // the call's bounds
    int group, n_kv;                // query heads per key head, key heads
    int cap_units, cap_items, cap_part;
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
// units: upper bound of the launch's attention units; split: some row block may be in several spans.
hipError_t launch_paged_attn(bool bf16, int64_t units, bool split, const PagedAttnParams &p, hipStream_t s);

}  // namespace cllm

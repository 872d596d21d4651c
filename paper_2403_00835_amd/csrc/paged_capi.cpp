// The paged KV cache's C ABI (include/cllm.h): checks, device memory and launches. The books of the
// pool live on the device; the host knows the bounds of the last plan only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "../../include/cllm.h"
#include "device.h"
#include "paged.h"

using namespace cllm;

struct cllm_paged {
    cllm_paged_config cfg{};
    hipStream_t stream = nullptr;
    bool bf16 = true;
    int elem = 2, group = 1;
    PagedBooks bk{};
    float *rcos = nullptr, *rsin = nullptr;  // null without rotation
    float *part_o = nullptr, *part_m = nullptr, *part_l = nullptr;
    bool tiled = false;  // long chunks take tiles
    int block_rows = 32, cap_part = 0, cap_tile_part = 0;
    void *own = nullptr;  // library-allocated workspace
    bool planned = false, dead = false;
    int n = 0, rows = 0, max_new = 0, max_len = 0;  // the last plan's bounds
    char err[512] = "";
};

namespace {

constexpr size_t kAlign = 256;
constexpr int kMaxLen = 1 << 20;  // tokens of a request, rows of a plan

cllm_status fail(cllm_paged *c, cllm_status s, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(c->err, sizeof c->err, fmt, ap);
    va_end(ap);
    if (s == CLLM_ERR_DEVICE) c->dead = true;
    return s;
}

#define HIPCHK(c, expr)                                                                                      \
    do {                                                                                                     \
        hipError_t _e = (expr);                                                                              \
        if (_e != hipSuccess) return fail((c), CLLM_ERR_DEVICE, "%s failed: %s", #expr, hipGetErrorString(_e)); \
    } while (0)

// Makes the cache's device current for a call.
struct DeviceGuard {
    int before = -1;
    bool ok = true;
    explicit DeviceGuard(int device) {
        int cur = -1;
        ok = hipGetDevice(&cur) == hipSuccess;
        if (ok && cur != device) {
            ok = hipSetDevice(device) == hipSuccess;
            before = cur;
        }
        if (!ok) (void)hipGetLastError();
    }
    ~DeviceGuard() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

bool config_ok(const cllm_paged_config *f) {
    const bool bf16 = f->dtype == CLLM_DTYPE_BF16;
    if (!bf16 && f->dtype != CLLM_DTYPE_F32) return false;
    if (!(f->head_dim == 32 || f->head_dim == 64 || f->head_dim == 128 || (bf16 ? f->head_dim == 256 : f->head_dim == 16)))
        return false;
    if (f->n_kv_heads < 1 || f->n_heads < f->n_kv_heads || f->n_heads > 1024 || f->n_heads % f->n_kv_heads != 0) return false;
    if (!(f->page_size == 16 || f->page_size == 32 || f->page_size == 64 || f->page_size == 128 || f->page_size == 256))
        return false;
    if (f->n_pages < 1 || (int64_t)f->n_pages * f->page_size > INT32_MAX) return false;
    if (f->max_seqs < 1 || f->max_seqs > kPagedMaxSeqs || f->max_ctx < 1 || f->max_ctx > kMaxLen || f->max_rows < 1 ||
        f->max_rows > kMaxLen)
        return false;
    if (!(f->rope_base == 0.0f || (f->rope_base > 0.0f && std::isfinite(f->rope_base)))) return false;
    return !(f->workspace_bytes > 0 && !f->workspace);
}

struct Buf {
    void **p;
    size_t bytes;
};
struct Bufs {  // (nothing here allocates host memory: no exception leaves an entry point)
    Buf b[16];
    int n = 0;
    void push(Buf x) { b[n++] = x; }
    const Buf *begin() const { return b; }
    const Buf *end() const { return b + n; }
};

// Device memory of a cache, each buffer at a 256-byte boundary.
Bufs buffers(cllm_paged *c) {
    const cllm_paged_config &f = c->cfg;
    PagedBooks &bk = c->bk;
    c->bf16 = f.dtype == CLLM_DTYPE_BF16;
    c->elem = c->bf16 ? 2 : 4;
    c->group = f.n_heads / f.n_kv_heads;
    bk.max_seqs = f.max_seqs;
    bk.max_pages = (f.max_ctx + f.page_size - 1) / f.page_size;
    bk.n_pages = f.n_pages;
    bk.page_shift = __builtin_ctz((unsigned)f.page_size);
    // Attention units: row blocks and tiles of any plan, and what splitting adds (kPagedUnits /
    // n_kv_heads row blocks, kPagedTileGroups / n_kv_heads tiles, about). Partial states of row blocks: a request
    // of few rows has up to kPagedFewRows in each of its spans, which are those of the pool and one more each
    // (every bf16 plan; fp32 chunks of more rows get what is left, and are not split where that is too little). Of
    // tiles: as many rows as split tiles have.
    c->tiled = c->bf16;
    c->block_rows = paged_block_rows(c->bf16, f.head_dim);
    const int64_t nrows = (int64_t)f.max_rows * c->group;
    const int64_t few = kPagedUnits / f.n_kv_heads + 1, few_tiles = 2 * (kPagedTileGroups / f.n_kv_heads + 1);
    const int64_t blocks = nrows / c->block_rows + f.max_seqs, tiles = c->tiled ? nrows / kPagedTileRows + f.max_seqs : 0;
    const int64_t spans = (f.max_ctx + kPagedSpanKeys - 1) / kPagedSpanKeys;
    const int64_t pool = std::min((int64_t)f.n_pages * f.page_size / kPagedSpanKeys + f.max_seqs, f.max_seqs * spans);
    bk.cap_units = (int)(blocks + few);
    bk.cap_tiles = (int)(tiles + few_tiles);
    bk.cap_items = (int)(nrows / kPagedItemRows + f.max_seqs);
    c->cap_part = (int)std::min(kPagedFewRows * pool, nrows * spans);
    if (!c->bf16) c->cap_part = std::min(c->cap_part, kPartRows - 1);
    c->cap_tile_part = c->tiled ? (int)std::min(few_tiles * kPagedTileRows, nrows * spans) : 0;
    auto P = [](auto **q) { return reinterpret_cast<void **>(q); };
    const size_t part = ((size_t)c->cap_part + c->cap_tile_part) * f.n_kv_heads;
    Bufs b;
    for (const Buf &x : {
            Buf{P(&bk.status), PS_WORDS * 4},
            Buf{P(&bk.table), (size_t)f.max_seqs * bk.max_pages * 4},
            Buf{P(&bk.seq_pages), (size_t)f.max_seqs * 4},
            Buf{P(&bk.free_list), (size_t)f.n_pages * 4},
            Buf{P(&bk.row_start), (size_t)(f.max_seqs + 1) * 4},
            Buf{P(&bk.row_slot), (size_t)f.max_rows * 4},
            Buf{P(&bk.row_pos), (size_t)f.max_rows * 4},
            Buf{P(&bk.units), (size_t)bk.cap_units * sizeof(PagedUnit)},
            Buf{P(&bk.tiles), (size_t)bk.cap_tiles * sizeof(PagedUnit)},
            Buf{P(&bk.items), (size_t)bk.cap_items * sizeof(PagedItem)},
            Buf{P(&c->part_o), part * f.head_dim * 4},
            Buf{P(&c->part_m), part * 4},
            Buf{P(&c->part_l), part * 4}})
        b.push(x);
    if (f.rope_base > 0.0f) {
        const size_t n = (size_t)f.max_ctx * (f.head_dim / 2) * 4;
        b.push({P(&c->rcos), n});
        b.push({P(&c->rsin), n});
    }
    return b;
}

size_t round_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

size_t total(const Bufs &bufs) {
    size_t t = 0;
    for (const Buf &b : bufs) t += round_up(b.bytes);
    return t;
}

// Memory a kernel on the cache's GPU may access.
bool accessible(const cllm_paged *c, const void *p) {
    hipPointerAttribute_t a{};
    if (hipPointerGetAttributes(&a, p) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    if (a.type == hipMemoryTypeDevice) return a.device == c->cfg.device;
    return a.type == hipMemoryTypeManaged || a.type == hipMemoryTypeHost || a.isManaged;
}

cllm_status check(cllm_paged *c) {
    return c->dead ? CLLM_ERR_DEVICE : CLLM_OK;  // the first error stays the last one
}

// Rows of `heads` heads: 16-byte vectors of whole heads.
cllm_status check_rows(cllm_paged *c, const char *name, const void *p, int64_t stride, int heads) {
    if (!p) return fail(c, CLLM_ERR_ARG, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return fail(c, CLLM_ERR_ARG, "%s is not 16-byte aligned", name);
    if (stride < (int64_t)heads * c->cfg.head_dim || stride * c->elem % 16 != 0 || stride > (1 << 30))
        return fail(c, CLLM_ERR_ARG, "%s: row stride %lld (at least %d elements, whole 16-byte vectors, at most 2^30)", name,
                    (long long)stride, heads * c->cfg.head_dim);
    if (!accessible(c, p)) return fail(c, CLLM_ERR_ARG, "%s is not device memory of the cache's GPU", name);
    return CLLM_OK;
}

cllm_status check_pool(cllm_paged *c, const char *name, const void *p) {
    return check_rows(c, name, p, (int64_t)c->cfg.n_kv_heads * c->cfg.head_dim, c->cfg.n_kv_heads);
}

}  // namespace

extern "C" {

cllm_status cllm_paged_workspace_bytes(const cllm_paged_config *cfg, size_t *bytes) {
    if (!cfg || !bytes) return CLLM_ERR_ARG;
    *bytes = 0;
    cllm_paged_config f = *cfg;
    f.workspace = nullptr;
    f.workspace_bytes = 0;
    if (!config_ok(&f)) return CLLM_ERR_ARG;
    cllm_paged *c = new (std::nothrow) cllm_paged;
    if (!c) return CLLM_ERR_OOM;
    c->cfg = f;
    *bytes = total(buffers(c));
    delete c;
    return CLLM_OK;
}

cllm_status cllm_paged_create(const cllm_paged_config *cfg, cllm_paged **out) {
    if (!cfg || !out) return CLLM_ERR_ARG;
    *out = nullptr;
    if (!config_ok(cfg)) return CLLM_ERR_ARG;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || cfg->device < 0 || cfg->device >= ndev) {
        (void)hipGetLastError();
        return CLLM_ERR_DEVICE;
    }
    cllm_paged *c = new (std::nothrow) cllm_paged;
    if (!c) return CLLM_ERR_OOM;
    c->cfg = *cfg;
    c->stream = static_cast<hipStream_t>(cfg->stream);
    auto bail = [&](cllm_status s) {
        (void)hipGetLastError();
        cllm_paged_free(c);
        return s;
    };
    DeviceGuard dev(cfg->device);
    if (!dev.ok) return bail(CLLM_ERR_DEVICE);
    const Bufs bufs = buffers(c);
    const size_t need = total(bufs);
    uint8_t *base = static_cast<uint8_t *>(cfg->workspace);
    if (base) {
        hipPointerAttribute_t a{};
        if (hipPointerGetAttributes(&a, base) != hipSuccess || a.type != hipMemoryTypeDevice || a.device != cfg->device ||
            reinterpret_cast<uintptr_t>(base) % kAlign != 0)
            return bail(CLLM_ERR_ARG);
        if (cfg->workspace_bytes < need) return bail(CLLM_ERR_CAPACITY);
    } else {
        if (hipMalloc(&c->own, need) != hipSuccess) {
            c->own = nullptr;
            return bail(CLLM_ERR_OOM);
        }
        base = static_cast<uint8_t *>(c->own);
    }
    for (const Buf &b : bufs) {
        *b.p = base;
        base += round_up(b.bytes);
    }
    if (launch_paged_init(c->bk, c->rcos, c->rsin, cfg->max_ctx, cfg->head_dim, (double)cfg->rope_base, c->stream) != hipSuccess ||
        hipStreamSynchronize(c->stream) != hipSuccess)
        return bail(CLLM_ERR_DEVICE);
    *out = c;
    return CLLM_OK;
}

void cllm_paged_free(cllm_paged *c) {
    if (!c) return;
    if (c->own) {
        DeviceGuard dev(c->cfg.device);
        (void)hipFree(c->own);  // waits for the device
    }
    delete c;
}

cllm_status cllm_paged_views_get(cllm_paged *c, cllm_paged_views *v) {
    if (!c || !v) return CLLM_ERR_ARG;
    v->block_table = c->bk.table;
    v->seq_pages = c->bk.seq_pages;
    v->free_list = c->bk.free_list;
    v->row_start = c->bk.row_start;
    v->row_slot = c->bk.row_slot;
    v->row_pos = c->bk.row_pos;
    v->max_pages = c->bk.max_pages;
    return CLLM_OK;
}

cllm_status cllm_paged_plan(cllm_paged *c, int32_t n, const int32_t *seq_ids, const int32_t *ctx_lens,
                            const int32_t *new_lens, int32_t rows, int32_t max_new, int32_t max_len) {
    if (!c) return CLLM_ERR_ARG;
    cllm_status s;
    if ((s = check(c))) return s;
    if (max_new == 0) max_new = rows;
    if (max_len == 0) max_len = c->cfg.max_ctx;
    if (n < 1 || n > c->cfg.max_seqs) return fail(c, CLLM_ERR_ARG, "n=%d outside [1, max_seqs]", n);
    if (!seq_ids || !ctx_lens || !new_lens) return fail(c, CLLM_ERR_ARG, "NULL pointer");
    if (rows < 0 || max_new < 0 || max_new > rows || max_len < 1)
        return fail(c, CLLM_ERR_ARG, "bounds: rows %d, max_new %d (at most rows), max_len %d", rows, max_new, max_len);
    if (rows > c->cfg.max_rows || max_len > c->cfg.max_ctx)
        return fail(c, CLLM_ERR_CAPACITY, "rows %d above max_rows or max_len %d above max_ctx", rows, max_len);
    DeviceGuard dev(c->cfg.device);
    if (!dev.ok) return fail(c, CLLM_ERR_DEVICE, "the cache's device cannot be made current");
    for (const int32_t *p : {seq_ids, ctx_lens, new_lens})
        if (reinterpret_cast<uintptr_t>(p) % 4 != 0 || !accessible(c, p))
            return fail(c, CLLM_ERR_ARG, "lengths: an array is not device memory of the cache's GPU");
    PagedPlanParams p{};
    p.bk = c->bk;
    p.seq = seq_ids;
    p.ctx = ctx_lens;
    p.neu = new_lens;
    p.n = n;
    p.rows = rows;
    p.max_new = max_new;
    p.max_len = max_len;
    p.group = c->group;
    p.n_kv = c->cfg.n_kv_heads;
    p.tiled = c->tiled;
    p.block_rows = c->block_rows;
    p.cap_part = c->cap_part;
    HIPCHK(c, launch_paged_plan(p, c->stream));
    c->planned = true;
    c->n = n;
    c->rows = rows;
    c->max_new = max_new;
    c->max_len = max_len;
    return CLLM_OK;
}

cllm_status cllm_paged_append(cllm_paged *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                              int64_t v_stride, void *q_out, int64_t q_out_stride, void *k_pages, void *v_pages) {
    if (!c) return CLLM_ERR_ARG;
    cllm_status s;
    if ((s = check(c))) return s;
    if (!c->planned) return fail(c, CLLM_ERR_STATE, "append before a plan");
    if (c->rows == 0) return CLLM_OK;
    const cllm_paged_config &f = c->cfg;
    if (!q != !q_out) return fail(c, CLLM_ERR_ARG, "q and q_out go together");
    DeviceGuard dev(f.device);
    if (!dev.ok) return fail(c, CLLM_ERR_DEVICE, "the cache's device cannot be made current");
    if (q && ((s = check_rows(c, "q", q, q_stride, f.n_heads)) || (s = check_rows(c, "q_out", q_out, q_out_stride, f.n_heads))))
        return s;
    if (q == q_out && q_stride != q_out_stride) return fail(c, CLLM_ERR_ARG, "q_out = q needs q's stride");
    if ((s = check_rows(c, "k", k, k_stride, f.n_kv_heads)) || (s = check_rows(c, "v", v, v_stride, f.n_kv_heads)) ||
        (s = check_pool(c, "k_pages", k_pages)) || (s = check_pool(c, "v_pages", v_pages)))
        return s;
    PagedAppendParams p{};
    p.bk = c->bk;
    p.rows = c->rows;
    p.max_new = c->max_new;
    p.max_len = c->max_len;
    p.q = q;
    p.k = k;
    p.v = v;
    p.q_out = q_out;
    p.k_pages = k_pages;
    p.v_pages = v_pages;
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.q_out_stride = q_out_stride;
    p.rcos = c->rcos;
    p.rsin = c->rsin;
    p.n_heads = f.n_heads;
    p.n_kv = f.n_kv_heads;
    p.hd = f.head_dim;
    HIPCHK(c, launch_paged_append(c->bf16, p, c->stream));
    return CLLM_OK;
}

cllm_status cllm_paged_attn(cllm_paged *c, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages,
                            float scale, void *out, int64_t out_stride, float *lse) {
    if (!c) return CLLM_ERR_ARG;
    cllm_status s;
    if ((s = check(c))) return s;
    if (!c->planned) return fail(c, CLLM_ERR_STATE, "attention before a plan");
    if (c->rows == 0) return CLLM_OK;
    const cllm_paged_config &f = c->cfg;
    const double scale_log2 = 1.4426950408889634 * (scale == 0.0f ? 1.0 / std::sqrt((double)f.head_dim) : (double)scale);
    if (!(std::fabs(scale_log2) <= FLT_MAX)) return fail(c, CLLM_ERR_ARG, "scale %g: not finite, or above 2.35e38", (double)scale);
    DeviceGuard dev(f.device);
    if (!dev.ok) return fail(c, CLLM_ERR_DEVICE, "the cache's device cannot be made current");
    if ((s = check_rows(c, "q", q, q_stride, f.n_heads)) || (s = check_rows(c, "out", out, out_stride, f.n_heads)) ||
        (s = check_pool(c, "k_pages", k_pages)) || (s = check_pool(c, "v_pages", v_pages)))
        return s;
    if (q == out && q_stride != out_stride) return fail(c, CLLM_ERR_ARG, "out = q needs q's stride");
    if (lse && (reinterpret_cast<uintptr_t>(lse) % 4 != 0 || !accessible(c, lse)))
        return fail(c, CLLM_ERR_ARG, "lse is not device memory of the cache's GPU");
    PagedAttnParams p{};
    p.bk = c->bk;
    p.rows = c->rows;
    p.max_new = c->max_new;
    p.max_len = c->max_len;
    p.q = q;
    p.k_pages = k_pages;
    p.v_pages = v_pages;
    p.out = out;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.lse = lse;
    p.part_o = c->part_o;
    p.part_m = c->part_m;
    p.part_l = c->part_l;
    p.n_heads = f.n_heads;
    p.n_kv = f.n_kv_heads;
    p.hd = f.head_dim;
    p.group = c->group;
    p.group_inv = ((1u << 24) + c->group - 1) / c->group;
    p.scale_log2 = (float)scale_log2;
    // bounds of the launch
    auto pieces = [&](int64_t most, int rows) {  // of requests of at most `most` rows each
        return std::min(c->n * ((most + rows - 1) / rows), (int64_t)c->rows * c->group / rows + c->n);
    };
    const int64_t most = (int64_t)c->max_new * c->group, spans = (c->max_len + kPagedSpanKeys - 1) / kPagedSpanKeys;
    int64_t units = pieces(c->tiled ? std::min<int64_t>(most, kPagedFewRows) : most, c->block_rows);
    units = std::min(units * spans, units + kPagedUnits / f.n_kv_heads + 1);
    int64_t tiles = c->tiled && most > kPagedFewRows ? pieces(most, kPagedTileRows) : 0;
    tiles = std::min(tiles * spans, tiles + 2 * (kPagedTileGroups / f.n_kv_heads + 1));
    // whether a plan of these bounds may have whole requests: any plan, as a graph of this call may run behind one of
    // more requests
    const int64_t blocks = std::min<int64_t>(f.max_seqs, (int64_t)c->rows * c->group / (kPagedWaveRows + 1));
    const bool whole = c->tiled && most > kPagedWaveRows && blocks * f.n_kv_heads >= kPagedTileGroups;
    HIPCHK(c, launch_paged_attn(c->bf16, units, whole, tiles, spans > 1, p, c->stream));
    return CLLM_OK;
}

cllm_status cllm_paged_status(cllm_paged *c, int32_t *rows, int32_t *free_pages) {
    if (!c) return CLLM_ERR_ARG;
    cllm_status s;
    if ((s = check(c))) return s;
    DeviceGuard dev(c->cfg.device);
    if (!dev.ok) return fail(c, CLLM_ERR_DEVICE, "the cache's device cannot be made current");
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(c->stream, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone) {
        (void)hipGetLastError();
        return fail(c, CLLM_ERR_STATE, "the status cannot be read while the stream is captured");
    }
    int32_t st[PS_WORDS] = {};
    HIPCHK(c, hipMemcpyAsync(st, c->bk.status, sizeof st, hipMemcpyDeviceToHost, c->stream));
    HIPCHK(c, hipStreamSynchronize(c->stream));
    if (rows) *rows = st[PS_ROWS];
    if (free_pages) *free_pages = st[PS_FREE];
    if (st[PS_FLAGS] & PF_ARG)
        return fail(c, CLLM_ERR_ARG, "the plan was refused: a slot out of range or twice, or a length outside the bounds");
    if (st[PS_FLAGS] & PF_ROWS) return fail(c, CLLM_ERR_CAPACITY, "the plan was refused: more rows than its bound");
    if (st[PS_FLAGS] & PF_PAGES) return fail(c, CLLM_ERR_CAPACITY, "the plan was refused: too few free pages");
    if (st[PS_LATE]) return fail(c, CLLM_ERR_STATE, "a call made for another plan's bounds ran after the plan and did nothing");
    return CLLM_OK;
}

const char *cllm_paged_last_error(const cllm_paged *c) { return c ? c->err : "null cache"; }

}  // extern "C"

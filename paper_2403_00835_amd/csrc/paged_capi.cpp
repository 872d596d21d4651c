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
    int rot = 0;                             // pairs of a head that are turned
    bool inter = false;                      // neighbours in place of halves
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
            Buf{P(&bk.entries), (size_t)f.max_seqs * sizeof(PagedEntry)},
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
    c->rot = c->rcos ? cfg->head_dim / 2 : 0;
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

cllm_status cllm_paged_rotary_freqs(const cllm_paged_rotary_spec *spec, int32_t head_dim, double *freqs) {
    if (!spec || !freqs || head_dim < 2 || head_dim > 2 * kMaxRot || head_dim % 2 != 0) return CLLM_ERR_ARG;
    const int dim = spec->dim == 0 ? head_dim : spec->dim;
    if (dim < 2 || dim > head_dim || dim % 2 != 0) return CLLM_ERR_ARG;
    if (spec->layout != CLLM_ROTARY_HALVES && spec->layout != CLLM_ROTARY_NEIGHBOURS) return CLLM_ERR_ARG;
    if (!std::isfinite(spec->magnitude)) return CLLM_ERR_ARG;
    auto positive = [](float x) { return x > 0.0f && std::isfinite(x); };
    if (!spec->freqs) {
        if (spec->scaling < CLLM_ROTARY_PLAIN || spec->scaling > CLLM_ROTARY_BY_PARTS || !positive(spec->base)) return CLLM_ERR_ARG;
        if (spec->scaling != CLLM_ROTARY_PLAIN && !positive(spec->factor)) return CLLM_ERR_ARG;
        if (spec->scaling == CLLM_ROTARY_BY_PARTS &&
            !(positive(spec->orig_ctx) && std::isfinite(spec->low) && std::isfinite(spec->high) && spec->low < spec->high))
            return CLLM_ERR_ARG;
    }
    double w[kMaxRot];
    for (int j = 0; j < dim / 2; ++j) {
        w[j] = spec->freqs ? spec->freqs[j] : std::pow((double)spec->base, -2.0 * j / (double)dim);
        if (!spec->freqs && spec->scaling == CLLM_ROTARY_LINEAR) w[j] /= (double)spec->factor;
        if (!spec->freqs && spec->scaling == CLLM_ROTARY_BY_PARTS) {
            const double turns = (double)spec->orig_ctx * w[j] / 6.283185307179586, low = spec->low, high = spec->high;
            const double keep = std::min(std::max((turns - low) / (high - low), 0.0), 1.0);
            w[j] *= keep + (1.0 - keep) / (double)spec->factor;
        }
        if (!(std::fabs(w[j]) <= 1e300)) return CLLM_ERR_ARG;  // (and times a position it is finite)
    }
    std::copy(w, w + dim / 2, freqs);
    return CLLM_OK;
}

cllm_status cllm_paged_rotary(cllm_paged *c, const cllm_paged_rotary_spec *spec) {
    if (!c) return CLLM_ERR_ARG;
    cllm_status s;
    if ((s = check(c))) return s;
    const cllm_paged_config &f = c->cfg;
    if (!c->rcos) return fail(c, CLLM_ERR_STATE, "the cache was created without rotation (rope_base 0)");
    PagedFreqs fr{};
    if (cllm_paged_rotary_freqs(spec, f.head_dim, fr.f) != CLLM_OK)
        return fail(c, CLLM_ERR_ARG, "rotary spec: dim even and up to head_dim, a known layout and scaling, base, factor and "
                                     "orig_ctx positive, low below high, all finite");
    const int rot = (spec->dim == 0 ? f.head_dim : spec->dim) / 2;
    DeviceGuard dev(f.device);
    if (!dev.ok) return fail(c, CLLM_ERR_DEVICE, "the cache's device cannot be made current");
    // (later appends take the new form at once, and must not find the old factors)
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(c->stream, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone) {
        (void)hipGetLastError();
        return fail(c, CLLM_ERR_STATE, "the form of the rotation cannot be changed while the stream is captured");
    }
    const bool inter = spec->layout == CLLM_ROTARY_NEIGHBOURS;
    HIPCHK(c, launch_paged_rotary(c->bk, c->rcos, c->rsin, f.max_ctx, rot, inter,
                                  spec->magnitude == 0.0f ? 1.0 : (double)spec->magnitude, fr, c->stream));
    c->rot = rot;
    c->inter = inter;
    return CLLM_OK;
}

namespace {

cllm_status append(cllm_paged *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                   void *q_out, int64_t q_out_stride, void *k_pages, void *v_pages, const float *q_gain, const float *k_gain,
                   float eps) {
    cllm_status s;
    if ((s = check(c))) return s;
    if (!c->planned) return fail(c, CLLM_ERR_STATE, "append before a plan");
    if (c->rows == 0) return CLLM_OK;
    const cllm_paged_config &f = c->cfg;
    if (!q != !q_out) return fail(c, CLLM_ERR_ARG, "q and q_out go together");
    if (q_gain && !q) return fail(c, CLLM_ERR_ARG, "q_gain without q");
    // (below fp32's normal range the squares of small values, which underflow, would count beside it)
    if ((q_gain || k_gain) && !(eps >= FLT_MIN && std::isfinite(eps)))
        return fail(c, CLLM_ERR_ARG, "eps %g: finite, at least 1.18e-38", (double)eps);
    DeviceGuard dev(f.device);
    if (!dev.ok) return fail(c, CLLM_ERR_DEVICE, "the cache's device cannot be made current");
    if (q && ((s = check_rows(c, "q", q, q_stride, f.n_heads)) || (s = check_rows(c, "q_out", q_out, q_out_stride, f.n_heads))))
        return s;
    if (q == q_out && q_stride != q_out_stride) return fail(c, CLLM_ERR_ARG, "q_out = q needs q's stride");
    if ((s = check_rows(c, "k", k, k_stride, f.n_kv_heads)) || (s = check_rows(c, "v", v, v_stride, f.n_kv_heads)) ||
        (s = check_pool(c, "k_pages", k_pages)) || (s = check_pool(c, "v_pages", v_pages)))
        return s;
    for (const float *g : {q_gain, k_gain})
        if (g && (reinterpret_cast<uintptr_t>(g) % 4 != 0 || !accessible(c, g)))
            return fail(c, CLLM_ERR_ARG, "gains: an array is not device memory of the cache's GPU");
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
    p.rot = c->rot;
    p.inter = c->inter;
    p.form = rotary_form(c->rot, c->inter);
    p.q_gain = q_gain;
    p.k_gain = k_gain;
    p.eps = eps;
    const bool whole = !c->rcos || (!c->inter && 2 * c->rot == f.head_dim);
    if (whole && !q_gain && !k_gain)
        HIPCHK(c, launch_paged_append(c->bf16, p, c->stream));
    else
        HIPCHK(c, launch_paged_append_forms(c->bf16, p, c->stream));
    return CLLM_OK;
}

}  // namespace

cllm_status cllm_paged_append(cllm_paged *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                              int64_t v_stride, void *q_out, int64_t q_out_stride, void *k_pages, void *v_pages) {
    if (!c) return CLLM_ERR_ARG;
    return append(c, q, q_stride, k, k_stride, v, v_stride, q_out, q_out_stride, k_pages, v_pages, nullptr, nullptr, 0.0f);
}

cllm_status cllm_paged_append_norm(cllm_paged *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                                   int64_t v_stride, void *q_out, int64_t q_out_stride, void *k_pages, void *v_pages,
                                   const float *q_gain, const float *k_gain, float eps) {
    if (!c) return CLLM_ERR_ARG;
    return append(c, q, q_stride, k, k_stride, v, v_stride, q_out, q_out_stride, k_pages, v_pages, q_gain, k_gain, eps);
}

namespace {

// window 0: none
cllm_status attend(cllm_paged *c, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages, float scale,
                   int32_t window, int32_t sinks, void *out, int64_t out_stride, float *lse) {
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
    const int64_t whole_tiles = c->tiled && most > kPagedFewRows ? pieces(most, kPagedTileRows) : 0;
    int64_t tiles = whole_tiles;
    tiles = std::min(tiles * spans, tiles + 2 * (kPagedTileGroups / f.n_kv_heads + 1));
    // whether a plan of these bounds may have whole requests: any plan, as a graph of this call may run behind one of
    // more requests
    const int64_t blocks = std::min<int64_t>(f.max_seqs, (int64_t)c->rows * c->group / (kPagedWaveRows + 1));
    const bool whole = c->tiled && most > kPagedWaveRows && blocks * f.n_kv_heads >= kPagedTileGroups;
    if (window == 0 || window >= c->max_len) {  // (a window that holds every token: what the call without one does)
        HIPCHK(c, launch_paged_attn(c->bf16, units, whole, tiles, spans > 1, p, c->stream));
        return CLLM_OK;
    }
    p.window = window;
    p.cap_part = c->cap_part;
    p.sinks = std::min(sinks, c->max_len);
    // a block's tokens end in at most block_rows positions; the window of the first begins anywhere in a span
    const int64_t reach = (int64_t)window + std::min(c->max_new, c->block_rows) - 1;
    const int64_t sink_spans = (p.sinks + kPagedSpanKeys - 1) / kPagedSpanKeys;
    // Tiles are split to fill the device, for which their partial states are written and joined. Behind a window that pays less, and
    // the less the more tiles there are and the wider the heads: with tiles for half the device never at heads of 128 or more
    // (384 of heads of 128 that see 8 chunks: 53 us split, 43 not; 34 chunks: 104 and 98), else above about so many chunks (128 of
    // heads of 128, 5 chunks: 28.1 and 23.5, 14: 33.9 and 36.5; 125 of 256, 10: 96.7 and 69.9, 18: 118 and 103; 24 of 256, 5: 53.8 and
    // 47.6, 8: 53.8 and 55.5; 264 of 64, 8: 26.8 and 25.9, 14: 34.0 and 36.1; 80 of 64, 5: 20.1 and 22.2).
    const int64_t groups = whole_tiles * f.n_kv_heads;
    p.whole_chunks = groups >= kPagedTileGroups / 2 && f.head_dim >= 128 ? INT32_MAX : (int)std::min<int64_t>(groups * f.head_dim / 2048, INT32_MAX);
    p.spans = (int)std::min(spans, (reach + kPagedSpanKeys - 1) / kPagedSpanKeys + 1 + sink_spans);
    HIPCHK(c, launch_paged_attn_window(c->bf16, c->n, most, whole, tiles, spans > 1, p, c->stream));
    return CLLM_OK;
}

}  // namespace

cllm_status cllm_paged_attn(cllm_paged *c, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages,
                            float scale, void *out, int64_t out_stride, float *lse) {
    if (!c) return CLLM_ERR_ARG;
    return attend(c, q, q_stride, k_pages, v_pages, scale, 0, 0, out, out_stride, lse);
}

cllm_status cllm_paged_attn_window(cllm_paged *c, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages,
                                   float scale, int32_t window, int32_t sinks, void *out, int64_t out_stride, float *lse) {
    if (!c) return CLLM_ERR_ARG;
    cllm_status s;
    if ((s = check(c))) return s;
    if (window < 1 || sinks < 0) return fail(c, CLLM_ERR_ARG, "window=%d (at least 1), sinks=%d (at least 0)", window, sinks);
    return attend(c, q, q_stride, k_pages, v_pages, scale, window, sinks, out, out_stride, lse);
}


cllm_status cllm_paged_verify_bytes(int32_t rows, int32_t vocab, int32_t draft, size_t *bytes) {
    if (!bytes) return CLLM_ERR_ARG;
    *bytes = 0;
    if (rows < 0 || vocab < 1) return CLLM_ERR_ARG;
    const int64_t parts = (int64_t)rows * ((vocab - 1) / kVerifyChunk + 1);
    // (a chunk past the last is counted in 31 bits, and so are the rows of a launch past the last one's)
    if (vocab > 1 << 30 || 2 * parts > INT32_MAX - kVerifyLaunch) return CLLM_ERR_CAPACITY;
    const size_t n = rows;
    *bytes = round_up(draft ? parts * (2 * sizeof(VerifyStat) + sizeof(double)) + n * (sizeof(VerifyStop) + 2 * sizeof(float))
                            : parts * sizeof(VerifyStat) + n * sizeof(float));
    return CLLM_OK;
}

cllm_status cllm_paged_verify(cllm_paged *c, int32_t n, const int32_t *row_start, int32_t rows, const int32_t *tokens, int32_t dtype,
                              int32_t vocab, const void *logits, int64_t stride, const void *draft_logits, int64_t draft_stride,
                              const float *temperature, const double *accept_u, const double *sample_u, int32_t *accepted,
                              int32_t *next_token, void *workspace, size_t workspace_bytes) {
    if (!c) return CLLM_ERR_ARG;
    cllm_status s;
    if ((s = check(c))) return s;
    const cllm_paged_config &f = c->cfg;
    if (n < 1 || n > f.max_seqs) return fail(c, CLLM_ERR_ARG, "n=%d outside [1, max_seqs]", n);
    if (dtype != CLLM_DTYPE_BF16 && dtype != CLLM_DTYPE_F32) return fail(c, CLLM_ERR_ARG, "unknown dtype %d", dtype);
    if (!row_start && !c->planned) return fail(c, CLLM_ERR_STATE, "row_start NULL before a plan");
    size_t need = 0;
    if ((s = cllm_paged_verify_bytes(rows, vocab, draft_logits != nullptr, &need)))
        return fail(c, s, "rows=%d (at least 0), vocab=%d (at least 1): too many, or out of range", rows, vocab);
    DeviceGuard dev(f.device);
    if (!dev.ok) return fail(c, CLLM_ERR_DEVICE, "the cache's device cannot be made current");
    // a name, what each element's address is a multiple of, and whether the call may do without the array
    const size_t elem = dtype == CLLM_DTYPE_BF16 ? 2 : 4;
    const struct {
        const char *name;
        const void *p;
        size_t align;
        bool none;
    } arrays[] = {{"row_start", row_start, 4, true},       {"temperature", temperature, 4, false}, {"sample_u", sample_u, 8, false},
                  {"accepted", accepted, 4, false},        {"next_token", next_token, 4, false},   {"tokens", tokens, 4, rows == 0},
                  {"logits", logits, elem, rows == 0},     {"draft_logits", draft_logits, elem, true},
                  {"accept_u", accept_u, 8, rows == 0},    {"workspace", workspace, kAlign, rows == 0}};
    for (const auto &a : arrays) {
        if (!a.p && a.none) continue;
        if (!a.p || reinterpret_cast<uintptr_t>(a.p) % a.align != 0 || !accessible(c, a.p))
            return fail(c, CLLM_ERR_ARG, "%s: NULL, misaligned, or not device memory of the cache's GPU", a.name);
    }
    for (int64_t x : {stride, draft_logits ? draft_stride : stride})
        if (x < vocab || x > (int64_t)1 << 40) return fail(c, CLLM_ERR_ARG, "row stride %lld (at least vocab, at most 2^40)", (long long)x);
    if (workspace_bytes < need) return fail(c, CLLM_ERR_CAPACITY, "workspace of %zu bytes: %zu are needed", workspace_bytes, need);
    VerifyParams p{};
    p.row_start = row_start ? row_start : c->bk.row_start;
    p.status = row_start ? nullptr : c->bk.status;
    p.tokens = tokens;
    p.n = n;
    p.rows = rows;
    p.vocab = vocab;
    p.chunks = (vocab - 1) / kVerifyChunk + 1;
    p.logits = logits;
    p.draft = draft_logits;
    p.stride = stride;
    p.draft_stride = draft_stride;
    p.temperature = temperature;
    p.accept_u = accept_u;
    p.sample_u = sample_u;
    p.accepted = accepted;
    p.next_token = next_token;
    p.stats = static_cast<VerifyStat *>(workspace);
    const size_t parts = (size_t)rows * p.chunks;
    if (draft_logits) {
        p.stops = reinterpret_cast<VerifyStop *>(p.stats + 2 * parts);
        p.rest = reinterpret_cast<double *>(p.stops + rows);
        p.picked = reinterpret_cast<float *>(p.rest + parts);
    } else {
        p.picked = reinterpret_cast<float *>(p.stats + parts);
    }
    HIPCHK(c, launch_paged_verify(dtype == CLLM_DTYPE_BF16, p, c->stream));
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
    if (st[PS_OTHER]) return fail(c, CLLM_ERR_STATE, "an append made for another form of the rotation ran after the plan and did nothing");
    return CLLM_OK;
}

const char *cllm_paged_last_error(const cllm_paged *c) { return c ? c->err : "null cache"; }

}  // extern "C"

// Attention of chunks of new tokens over a paged KV cache on gfx950.
//
// Row (i, h) of a request, token i of its chunk at position ctx + i, head h of the group of a key head:
// softmax over the request's tokens t <= ctx + i of scale q . k_t, times v_t. Rows of a request and key
// head are numbered i x group + h.
//
// Few rows (paged_span_kernel): the keys are walked in chunks of 64 at absolute positions. A chunk's
// state per row is its maximum, its sum and its unnormalised output; the states of the chunks that hold
// a key the row sees are merged in position order into that of a span of 256 keys, and the spans' into
// the row's. The order depends on positions alone: a row's bits are the same whichever rows, requests,
// pages and launches it is computed with. Plans of many blocks (paged_request_kernel) take the same steps
// without partial states between kernels.
// Long chunks (paged_tile_kernel): tiles of 128 rows walk their keys with a running maximum; ranges of
// keys are joined where there are few tiles.
//
// Values: scores and softmax statistics in fp32; the probabilities of few rows as hi + lo bf16 planes
// (~2^-17), so the only rounding to bf16 is that of the output. Keys past a row's position contribute
// nothing, whatever their values (NaN, infinities): scores are selected away, values by the rules in
// chunk_values.
#include <algorithm>

#include "device.h"
#include "paged.h"

namespace cllm {

namespace {

constexpr int kKeys = kAttnChunk;  // keys of a chunk
constexpr int kSpanChunks = kPagedSpanKeys / kKeys;
constexpr float kLn2 = 0.6931471805599453f;

// LDS image of 64 keys of a bf16 K or V: [64][head_dim], 16-byte pieces permuted within a row so that the
// reads below hit different banks: K is read 16 or 32 keys at one column, V 4 or 8 keys x 32 bytes.
template <int HD>
struct Tile {
    static constexpr int ROWB = HD * 2;       // bytes of a key
    static constexpr int NC = ROWB / 16;      // 16-byte pieces of a key
    static constexpr int BYTES = kKeys * ROWB;
    static constexpr int KIB = BYTES / 1024;  // wave loads of a tile
    static constexpr int RPK = 1024 / ROWB;   // keys per wave load (2..16)
    static_assert(RPK >= 1 && RPK <= 16 && NC >= 4, "a wave load stays within 16 keys");
    __device__ static int kswz(int key) { return NC >= 16 ? key & 15 : (key / (16 / NC)) & (NC - 1); }
    __device__ static int vswz(int key) {
        constexpr int NP = HD / 16;  // 32-byte pairs
        return 2 * (NP >= 8 ? key & 7 : (key / (8 / NP)) & (NP - 1));
    }
};

// Transposing reads of 16 columns of V: lane (g, r) of an instruction addresses key 4 g + r / 4 of 16 keys and
// 8 bytes of columns 4 (r % 4) .., and receives column r of keys 4 g .. 4 g + 3.
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x2 read_tr(const uint8_t *lds) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4 *)lds));
}
// Four of them at a, four at b, B bytes apart, and their wait in one block: the compiler takes the intrinsic
// to read what LDS DMA in flight writes, wherever that goes, and would wait for all of it first.
template <int B>
__device__ __forceinline__ void read_tr8(uint32_t a, uint32_t b, u32x2 (&v)[8]) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n"
        "ds_read_b64_tr_b16 %1, %8 offset:%10\n"
        "ds_read_b64_tr_b16 %2, %8 offset:%11\n"
        "ds_read_b64_tr_b16 %3, %8 offset:%12\n"
        "ds_read_b64_tr_b16 %4, %9\n"
        "ds_read_b64_tr_b16 %5, %9 offset:%10\n"
        "ds_read_b64_tr_b16 %6, %9 offset:%11\n"
        "ds_read_b64_tr_b16 %7, %9 offset:%12\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
        : "v"(a), "v"(b), "n"(B), "n"(2 * B), "n"(3 * B)
        : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const uint8_t *p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)p;
}

// Two values rounded to bf16 (nearest even), the first in the low half: one instruction.
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Base-2 exponential of a value <= 0 (or NaN): the hardware instruction, results below 2^-126 are 0,
// which a softmax weight may lose.
__device__ __forceinline__ float exp2_weight(float x) { return __builtin_amdgcn_exp2f(x); }

// Merging a state (Ms, ls, os) behind (M, l, o): the weights, then each value with an explicit
// multiply and fused add, so that every kernel rounds alike.
__device__ __forceinline__ void merge_weights(float &M, float Ms, float &w, float &ws) {
    const float Mn = fmaxf(M, Ms);
    w = M == -INFINITY ? 0.0f : exp2_weight(M - Mn);
    ws = Ms == -INFINITY ? 0.0f : exp2_weight(Ms - Mn);
    M = Mn;
}
__device__ __forceinline__ float merge_value(float x, float xs, float w, float ws) { return __builtin_fmaf(xs, ws, x * w); }

// What a call's rows see: every position up to their own, or of those the last `window` and the first `sinks`.
template <bool WIN>
struct Sight {
    int window, sinks;
    __device__ explicit Sight(const PagedAttnParams &p) : window(p.window), sinks(p.sinks) {}
    // The row at pos sees the key; it sees some key of [k, k + n), k <= pos.
    __device__ bool key(int pos, int k) const { return k <= pos && (!WIN || k > pos - window || k < sinks); }
    __device__ bool some(int pos, int k, int n) const { return !WIN || k + n - 1 > pos - window || k < sinks; }
    // key() of the keys k .. k + 63, a bit each.
    __device__ uint64_t bits(int pos, int k) const {
        auto below = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };
        return below(pos - k + 1) & (~below(pos - window + 1 - k) | below(sinks - k));
    }
    // Some row of the positions up to `last` does not see some key of [k, k + n) that is behind it.
    __device__ bool cuts(int last, int k, int n) const { return WIN && max(k, sinks) <= min(k + n - 1, last - window); }
};

// The pieces of N keys that rows at positions first .. last see, in order: those of the sinks, then those from the first
// row's window on.
template <bool WIN, int N>
struct Visible {
    int sink_end, from, count;
    __device__ Visible(const Sight<WIN> &see, int first, int last) : sink_end(0), from(0), count(last / N + 1) {
        if constexpr (WIN) {
            sink_end = (min(see.sinks, last + 1) + N - 1) / N;
            from = max(max(first - see.window + 1, 0) / N, sink_end);
            count = sink_end + (last / N + 1 - from);
        }
    }
    __device__ int piece(int j) const { return WIN && j >= sink_end ? j - sink_end + from : j; }
};

// Behind a window, a tile whose rows see few chunks is not split: the first of the plan's ranges takes them all and writes the
// output. (One that sees every chunk is split as without a window, with the same bits.)
template <bool WIN>
__device__ __forceinline__ bool tile_is_whole(const PagedAttnParams &p, const Visible<WIN, kKeys> &chunks, int last) {
    return WIN && chunks.count <= p.whole_chunks && chunks.count <= last / kKeys;
}

// Scores to probabilities: keys past qpos (relative to the chunk's first key, key0) are out. mx: the row's
// maximum (-inf: it sees no key), l: its sum.
template <bool WIN>
__device__ __forceinline__ void chunk_softmax(f32x4 (&st)[4], int qpos, const Sight<WIN> &see, int key0, float scale_log2, int lane,
                                              float &mx, float &l) {
    const int g = lane >> 4;
    mx = -INFINITY;
    const int under = qpos - see.window, sinks = see.sinks - key0;  // keys above `under` or below `sinks`
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int k = 16 * kt + 4 * g + v;
            const float sc = k <= qpos && (!WIN || k > under || k < sinks) ? st[kt][v] * scale_log2 : -INFINITY;
            st[kt][v] = sc;
            mx = fmaxf(mx, sc);
        }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float ref = mx == -INFINITY ? 0.0f : mx;  // nothing seen: every weight is 0
    l = 0.0f;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            st[kt][v] = exp2_weight(st[kt][v] - ref);
            l += st[kt][v];
        }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
}

// Columns of the output tile: MFMA row r of tile dt is column vcol(dt, r). bf16: 16 dt + r. fp32 values
// come straight from memory, a lane's load holding W consecutive columns, one for each of W tiles.
template <Prec P, int HD>
struct Cols {
    static constexpr int W = P == Prec::BF16 ? 1 : (HD >= 64 ? 4 : HD / 16);
    __device__ static int vcol(int dt, int r) { return dt / W * 16 * W + r * W + dt % W; }
};

// W consecutive words.
template <int W>
__device__ __forceinline__ void load_words(uint32_t (&x)[W], const float *src) {
    if constexpr (W == 4)
        *reinterpret_cast<u32x4 *>(x) = *reinterpret_cast<const u32x4 *>(src);
    else if constexpr (W == 2)
        *reinterpret_cast<u32x2 *>(x) = *reinterpret_cast<const u32x2 *>(src);
    else
        x[0] = *reinterpret_cast<const uint32_t *>(src);
}

// The V operands of output tiles dt and dt + 1: vb[y][x] holds the keys of the probabilities' registers (bf16:
// x = 0, 1, keys 32 x + 4 g + (0..3) and 32 x + 16 + 4 g + (0..3)), from LDS.
template <int HD>
__device__ __forceinline__ void v_operands(const uint8_t *V, int dt, int lane, u32x4 (&vb)[2][2]) {
    using TL = Tile<HD>;
    constexpr int B = 16 * TL::ROWB;  // of 16 keys, whose permutations repeat
    const int g = lane >> 4, r16 = lane & 15, key = 4 * g + (r16 >> 2);
    uint32_t at[2];
#pragma unroll
    for (int y = 0; y < 2; ++y)  // the permutation moves 32-byte pairs
        at[y] = lds_address(V) + key * TL::ROWB + ((2 * (dt + y) + ((r16 & 3) >> 1)) ^ TL::vswz(key)) * 16 + (r16 & 1) * 8;
    u32x2 h[8];
    read_tr8<B>(at[0], at[1], h);
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const u32x2 lo = h[4 * y + 2 * x], hi = h[4 * y + 2 * x + 1];
            vb[y][x] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
}

// One 16-column tile of V^T P^T from operands vb and the probabilities' operands pb.
template <Prec P, int N, int NPL>
__device__ __forceinline__ f32x4 v_product(const u32x4 (&vb)[N], const u32x4 (&pb)[NPL][N]) {
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int pl = 0; pl < NPL; ++pl) o = mfma_kstep<P>(vb[x], pb[pl][x], o);
    return o;
}

// Sixteen weights of a lane as MFMA operands (bf16: hi and lo planes).
template <Prec P, int NPL, int N>
__device__ __forceinline__ void weight_operand(const f32x4 (&st)[4], u32x4 (&pb)[NPL][N]) {
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (P == Prec::BF16) {
                const float a = st[2 * x + i / 2][2 * (i % 2)], b = st[2 * x + i / 2][2 * (i % 2) + 1];
                const uint32_t hi = pack_bf16(a, b);
                pb[0][x][i] = hi;
                pb[NPL - 1][x][i] = pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
            } else {
                pb[0][x][i] = __float_as_uint(st[x][i]);
            }
        }
}

// Rows of a unit, from its first: row j is token(j) of the chunk, head(j) of the group. The quotient of the
// small number by the group is a product: exact below 2^24 / 1024 (group's largest).
struct RowMap {
    int token0, rem0, group;
    uint32_t inv;  // 2^24 / group, rounded up
    __device__ RowMap(const PagedAttnParams &p, int row)
        : token0(row / p.group), rem0(row % p.group), group(p.group), inv(p.group_inv) {}
    __device__ int past(int j) const { return (int)__umulhi((uint32_t)(rem0 + j) << 8, inv); }
    __device__ int token(int j) const { return token0 + past(j); }
    __device__ int head(int j) const { return rem0 + j - past(j) * group; }
};

// Four columns of a row's output (token and head of the plan's rows), and with the first its log sum of
// exponentials.
template <Prec P>
__device__ __forceinline__ void store_row(const PagedAttnParams &p, int token, int head, int col, f32x4 o, float M, float l) {
    using T = typename PrecT<P>::T;
    T *out = reinterpret_cast<T *>(p.out) + (size_t)token * p.out_stride + head * p.hd + col;
    alignas(16) T x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = to_elem<P>(o[e] / l);
    if constexpr (P == Prec::BF16)
        *reinterpret_cast<u32x2 *>(out) = *reinterpret_cast<const u32x2 *>(x);
    else
        *reinterpret_cast<u32x4 *>(out) = *reinterpret_cast<const u32x4 *>(x);
    if (p.lse && col == 0) p.lse[(size_t)token * p.n_heads + head] = (M + log2f(l)) * kLn2;
}

// A unit, requested with the words that say whether the call is the plan's: one round trip.
template <bool TILES>
__device__ __forceinline__ bool next_unit(const PagedAttnParams &p, int i, int cap, PagedUnit &u, int &count) {
    const int32_t *st = p.bk.status;
    const int R = st[PS_ROWS], n = st[TILES ? PS_TILES : PS_UNITS], br = st[PS_BOUND_ROWS], bn = st[PS_BOUND_NEW],
              bl = st[PS_BOUND_LEN];
    const PagedUnit *list = TILES ? p.bk.tiles : p.bk.units;
    u = list[min(i, cap - 1)];
    request_together(R, n, br, bn, bl, u.slot, u.ctx, u.m, u.r0, u.row, u.k0, u.k1, u.part);
    if (R > 0 && (br != p.rows || bn != p.max_new || bl != p.max_len)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) p.bk.status[PS_LATE] = 1;
        return false;
    }
    count = n;
    return R > 0 && i < n;
}

// A request of the plan, likewise.
__device__ __forceinline__ bool next_entry(const PagedAttnParams &p, int i, PagedEntry &e, int &count) {
    const int32_t *st = p.bk.status;
    const int R = st[PS_ROWS], n = st[PS_ENTRIES], br = st[PS_BOUND_ROWS], bn = st[PS_BOUND_NEW], bl = st[PS_BOUND_LEN];
    e = p.bk.entries[min(i, p.bk.max_seqs - 1)];
    request_together(R, n, br, bn, bl, e.slot, e.ctx, e.m, e.r0, e.part, e.kind);
    if (R > 0 && (br != p.rows || bn != p.max_new || bl != p.max_len)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) p.bk.status[PS_LATE] = 1;
        return false;
    }
    count = n;
    return R > 0 && i < n;
}

// Partial row of a request's first row in the first span that it sees, or -1: the plan's place; in fp32 one of the call's own
// (p.split: p.spans for every row of the plan), as the plan has none for more rows than it finds room for in all their spans.
template <Prec P>
__device__ __forceinline__ int window_part(const PagedAttnParams &p, const PagedEntry &e) {
    if (P == Prec::BF16) return e.part;
    return p.split ? p.spans * p.group * e.r0 : -1;
}

// What a workgroup of the span kernel takes, one after another: the plan's units; behind a window, of block x of every
// gridDim.z-th request the y-th span that the block sees (all of them where the request has no partial states).
template <Prec P, int ROWS, bool WIN>
struct SpanUnits {
    int idx = blockIdx.x, z = blockIdx.z, count = 0;
    __device__ __forceinline__ bool next(const PagedAttnParams &p, int cap, PagedUnit &u, int &h) {
        if constexpr (!WIN) {
            const bool more = next_unit<false>(p, idx / p.n_kv, cap, u, count);
            h = idx % p.n_kv;
            idx += gridDim.x;
            return more;
        }
        for (; idx < p.blocks * p.n_kv; idx += gridDim.x, z = blockIdx.z) {
            PagedEntry e;
            while (next_entry(p, z, e, count)) {
                z += gridDim.z;
                const int j = blockIdx.y, row = idx / p.n_kv * ROWS, part = window_part<P>(p, e);
                if (e.kind != PE_BLOCKS || row >= e.m * p.group || (part < 0 && j > 0)) continue;
                u = PagedUnit{e.slot, e.ctx, e.m, e.r0, row, j, part < 0 ? kAllSpans : j + 1,
                              part < 0 ? -1 : part + j * e.m * p.group + row};
                h = idx % p.n_kv;
                return true;
            }
            if (count == 0) break;
        }
        return false;
    }
};

// What a workgroup of the request kernel takes, where u.k0 < 0.
template <bool WIN>
__device__ __forceinline__ bool next_request(const PagedAttnParams &p, int i, int cap, PagedUnit &u, int &count) {
    if constexpr (!WIN) return next_unit<false>(p, i, cap, u, count);
    PagedEntry e;
    const bool more = next_entry(p, i, e, count);
    const bool mine = e.kind == PE_WHOLE || (p.all_whole && e.m > 0);
    u = PagedUnit{e.slot, e.ctx, e.m, e.r0, 0, mine ? -1 : 0, kAllSpans, -1};
    return more;
}

}  // namespace

namespace {

// Four columns of one row of an item: the states of its spans (those up to the row's position; behind a window those of
// its block that it sees) or ranges.
template <Prec P, int HD, bool WIN>
__device__ __forceinline__ void join_row(const PagedAttnParams &p, const PagedItem &it, int h, int row, int col) {
    if (row >= min(kPagedItemRows, it.m * p.group - it.row)) return;
    const RowMap map(p, it.row);
    const Sight<WIN> see(p);
    const int pos = it.ctx + map.token(row);
    int count = it.count > 0 ? it.count : pos / kPagedSpanKeys + 1;
    Visible<WIN, kPagedSpanKeys> spans(see, pos, pos);
    if (WIN && it.count == 0) {
        constexpr int BR = paged_block_rows(P == Prec::BF16, HD);
        const int first = row / BR * BR, last = min(first + BR, it.m * p.group - it.row) - 1;  // (an item begins with a block)
        spans = Visible<WIN, kPagedSpanKeys>(see, it.ctx + map.token(first), it.ctx + map.token(last));
        count = spans.count;
    }
    if (WIN && it.count > 0) {
        const int t0 = it.row / kPagedTileRows * kPagedTileRows, t1 = min(t0 + kPagedTileRows, it.m * p.group) - 1;
        const RowMap tile(p, t0);
        const int last = it.ctx + tile.token(t1 - t0);
        if (tile_is_whole<WIN>(p, Visible<WIN, kKeys>(see, it.ctx + tile.token(0), last), last)) return;
    }
    float M = -INFINITY, l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int U = 4;  // states in flight (of short rows, more repeat the last one's loads)
    for (int s0 = 0; s0 < count; s0 += U) {
        f32x4 os[U];
        float Ms[U], ls[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const size_t pr = (size_t)(it.part + min(s0 + i, count - 1) * it.stride + row) * p.n_kv + h;
            os[i] = *reinterpret_cast<const f32x4 *>(p.part_o + pr * HD + col);
            Ms[i] = p.part_m[pr];
            ls[i] = p.part_l[pr];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            bool use = s0 + i < count;  // a select: a branch would sink the loads behind it
            if (WIN && it.count == 0) {
                const int k = spans.piece(s0 + i) * kPagedSpanKeys;
                use = use && k <= pos && see.some(pos, k, kPagedSpanKeys);
            }
            float Mn = M, w0, w1;
            merge_weights(Mn, Ms[i], w0, w1);
            const float ln = merge_value(l, ls[i], w0, w1);
            M = use ? Mn : M;
            l = use ? ln : l;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = merge_value(o[e], os[i][e], w0, w1);
                o[e] = use ? x : o[e];
            }
        }
    }
    store_row<P>(p, it.r0 + map.token(row), h * p.group + map.head(row), col, o, M, l);
}

}  // namespace

// LDS bytes of a wave of the span kernel: the chunk's V (bf16), then in its place the chunk's states of up
// to 16 RG rows (padded rows, so that the writes of 16 rows hit different banks).
template <Prec P, int HD, int RG>
constexpr int span_wave_lds() {
    constexpr int state = 16 * RG * (HD * 4 + 16), v = P == Prec::BF16 ? kKeys * HD * 2 : 0;
    return state > v ? state : v;
}

constexpr int class_words(int hd) { return (hd + kWave - 1) / kWave; }

// The product of a chunk's weights pb (of NRG groups of 16 rows) with its values (bf16: in LDS; fp32: from
// memory, at[]: the first elements of its four tiles of 16 keys). valid: keys of the chunk that the request
// has (behind them a page holds whatever it did before), kKeys where the others have been cleared; qpos: the lane's rows' positions in the chunk. Says
// whether the classes cls are to be added to the result.
template <Prec P, int HD, bool WIN, int NRG, int N, int NPL>
__device__ __forceinline__ bool chunk_values(const PagedAttnParams &p, const uint8_t *V, const size_t (&at)[4], int valid, int key0,
                                             const u32x4 (&pb)[NRG][NPL][N], const int (&qpos)[NRG], f32x4 (&oc)[NRG][HD / 16],
                                             uint64_t (&cls)[class_words(HD)]) {
    constexpr bool B = P == Prec::BF16;
    constexpr int NDT = HD / 16, W = Cols<P, HD>::W, NCOL = class_words(HD);
    const int lane = threadIdx.x & 63, g = lane >> 4, r16 = lane & 15;
    // A weight of 0 does not silence an infinite or NaN value in the product, and a weight's lo plane may
    // turn an infinity into a NaN. Both leave a NaN in some output, so outputs without one are right. Else
    // (rare) the values that are not finite are taken out, the product is formed again, and what the rows
    // that see them get from them is added behind it: a sum per row and column, as a class of two bits (0,
    // +inf, -inf, NaN), 32 rows a word, of this lane's columns lane, lane + 64, ...
    bool taken = false;  // uniform over the wave
    // V operands of the GR tiles from tile dt on
    constexpr int GR = B ? 2 : W;
    auto operand = [&](int dt, u32x4(&vb)[GR][N]) {
        if constexpr (B) {
            v_operands<HD>(V, dt, lane, vb);
            if (valid < kKeys || taken) {  // uniform: values to leave out
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = 32 * x + 16 * (i / 2) + 4 * g + 2 * (i % 2);
                            const uint32_t v = vb[y][x][i];
                            const bool lo = key < valid && !(taken && (v & 0x7f80u) == 0x7f80u);
                            const bool hi = key + 1 < valid && !(taken && (v & 0x7f800000u) == 0x7f800000u);
                            vb[y][x][i] = (lo ? v & 0xffffu : 0u) | (hi ? v & 0xffff0000u : 0u);
                        }
            }
        } else {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    alignas(4 * W) uint32_t x[W];
                    load_words<W>(x, reinterpret_cast<const float *>(p.v_pages) + at[kt] + (4 * g + v) * HD +
                                         Cols<P, HD>::vcol(dt, r16));
#pragma unroll
                    for (int y = 0; y < W; ++y) vb[y][kt][v] = x[y];
                }
            if (valid < kKeys || taken) {  // uniform: values to leave out
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
#pragma unroll
                        for (int y = 0; y < W; ++y) {
                            const uint32_t x = vb[y][kt][v];
                            const bool use = 16 * kt + 4 * g + v < valid && !(taken && (x & 0x7f800000u) == 0x7f800000u);
                            vb[y][kt][v] = use ? x : 0u;
                        }
            }
        }
    };
    while (true) {
        float sum = 0.f;
#pragma unroll
        for (int dt = 0; dt < NDT; dt += GR) {
            u32x4 vb[GR][N];
            operand(dt, vb);
#pragma unroll
            for (int y = 0; y < GR; ++y)
#pragma unroll
                for (int rg = 0; rg < NRG; ++rg) {
                    const f32x4 x = v_product<P>(vb[y], pb[rg]);
                    oc[rg][dt + y] = x;
                    sum += (x[0] + x[1]) + (x[2] + x[3]);
                }
        }
        if (taken || !__any(sum != sum)) break;
        taken = true;
#pragma unroll 1
        for (int j = 0; j < NCOL; ++j) {
            const int col = lane + j * kWave;
            uint64_t bits = 0;
            float acc = 0.f;
            int key = 0;
#pragma unroll 1
            for (int r = 0; r < 16 * NRG; ++r) {  // the rows' positions do not fall
                const int pos = __builtin_amdgcn_readlane(r < 16 ? qpos[0] : qpos[NRG - 1], r & 15), last = min(pos, kKeys - 1);
                if (WIN) key = 0, acc = 0.f;  // behind a window, row by row
                for (; key <= last; ++key) {
                    if (col >= HD || !Sight<WIN>(p).key(key0 + pos, key0 + key)) continue;
                    uint32_t x;
                    if constexpr (B) {
                        using TL = Tile<HD>;
                        x = (uint32_t)reinterpret_cast<const uint16_t *>(V + key * TL::ROWB + ((col / 8) ^ TL::vswz(key)) * 16)[col % 8] << 16;
                    } else {
                        const size_t row = key < 16 ? at[0] : key < 32 ? at[1] : key < 48 ? at[2] : at[3];
                        x = __float_as_uint(reinterpret_cast<const float *>(p.v_pages)[row + (key & 15) * HD + col]);
                    }
                    if ((x & 0x7f800000u) == 0x7f800000u) acc += __uint_as_float(x);
                }
                const uint64_t c = acc != acc ? 3 : acc == INFINITY ? 1 : acc == -INFINITY ? 2 : 0;
                bits |= c << (2 * r);
            }
#pragma unroll
            for (int i = 0; i < NCOL; ++i)
                if (i == j) cls[i] = bits;
        }
    }
    return taken;
}
__device__ __forceinline__ float class_value(uint32_t c) { return (c & 3) == 1 ? INFINITY : (c & 3) == 2 ? -INFINITY : NAN; }

// One chunk of the span kernel, by one wave: the states of its NRG groups of 16 rows into s_mine ([row][column])
// and s_m, s_l (this wave's rows). last_key: the request's last token; pages: its table.
template <Prec P, int HD, bool WIN, int NRG>
__device__ __forceinline__ void span_chunk(const PagedAttnParams &p, const PagedUnit &u, const RowMap &map, int h, int rows, int key0,
                                           int last_key, const int32_t *table, uint8_t *s_mine, float *s_m, float *s_l) {
    using PT = PrecT<P>;
    using T = typename PT::T;
    constexpr bool B = P == Prec::BF16;
    constexpr int KSTEP = PT::KSTEP, VEC = PT::VEC, NKK = HD / KSTEP, NDT = HD / 16, N = B ? 2 : 4, NPL = PT::PLANES;
    constexpr int W = Cols<P, HD>::W, SROW = HD + 4;  // floats of a state row
    const int lane = threadIdx.x & 63, g = lane >> 4, r16 = lane & 15, shift = p.bk.page_shift;
    // pages of the four tiles of 16 keys (tiles past the request's end: its last one)
    const int tl = min(key0 + 16 * (lane & 3), last_key) >> 4, pg = table[(tl << 4) >> shift];
    // this lane's rows (those past the block: its last one, not stored)
    int qpos[NRG];
    u32x4 q[NRG][NKK];
#pragma unroll
    for (int rg = 0; rg < NRG; ++rg) {
        const int r = min(16 * rg + r16, rows - 1), token = map.token(r), head = h * p.group + map.head(r);
        qpos[rg] = u.ctx + token - key0;
        const T *qrow = reinterpret_cast<const T *>(p.q) + (size_t)(u.r0 + token) * p.q_stride + head * HD + g * VEC;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) q[rg][kk] = *reinterpret_cast<const u32x4 *>(qrow + kk * KSTEP);
    }
    size_t at[4];  // first element of each tile
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
        const int tile = __builtin_amdgcn_readlane(tl, kt), page = __builtin_amdgcn_readlane(pg, kt);
        at[kt] = ((((size_t)page * p.n_kv + h) << shift) + ((tile << 4) & ((1 << shift) - 1))) * HD;
    }
    u32x4 kf[4][NKK];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk)
            kf[kt][kk] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const T *>(p.k_pages) + at[kt] + r16 * HD + kk * KSTEP +
                                                          g * VEC);
    const int valid = last_key - key0 + 1;  // keys of the chunk that the request has
    if constexpr (B) {
        using TL = Tile<HD>;
#pragma unroll
        for (int i = 0; i < TL::KIB; ++i) {
            const int key = i * TL::RPK + lane / (kWave / TL::RPK), piece = (lane % TL::NC) ^ TL::vswz(key);
            const T *src = reinterpret_cast<const T *>(p.v_pages) + at[i * TL::RPK / 16] + (key & 15) * HD + piece * 8;
            __builtin_amdgcn_global_load_lds(static_cast<const void *>(src),
                                             (__attribute__((address_space(3))) void *)(s_mine + i * 1024), 16, 0, 0);
        }
    }
    u32x4 pb[NRG][NPL][N];
    float mx[NRG], lc[NRG];
#pragma unroll
    for (int rg = 0; rg < NRG; ++rg) {
        f32x4 st[4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            st[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) st[kt] = mfma_kstep<P>(kf[kt][kk], q[rg][kk], st[kt]);
        }
        chunk_softmax<WIN>(st, qpos[rg], Sight<WIN>(p), key0, p.scale_log2, lane, mx[rg], lc[rg]);
        weight_operand<P>(st, pb[rg]);
    }
    if constexpr (B) {
        wait_vm_lds<0>();
        if (valid < kKeys)  // values behind the request's last token, whatever the page holds there
            for (int i = valid * Tile<HD>::NC + lane; i < kKeys * Tile<HD>::NC; i += kWave)
                reinterpret_cast<u32x4 *>(s_mine)[i] = u32x4{0u, 0u, 0u, 0u};
    }
    f32x4 oc[NRG][NDT];
    uint64_t cls[class_words(HD)];
    const bool taken = chunk_values<P, HD, WIN>(p, s_mine, at, B ? kKeys : valid, key0, pb, qpos, oc, cls);
    // V has been read: the states in its place
#pragma unroll
    for (int rg = 0; rg < NRG; ++rg) {
        float *s_o = reinterpret_cast<float *>(s_mine) + (16 * rg + r16) * SROW;
        if constexpr (W == 1) {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) *reinterpret_cast<f32x4 *>(s_o + 16 * dt + 4 * g) = oc[rg][dt];
        } else {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s_o[Cols<P, HD>::vcol(dt, 4 * g + e)] = oc[rg][dt][e];
        }
        if (g == 0) {
            s_m[16 * rg + r16] = mx[rg];
            s_l[16 * rg + r16] = lc[rg];
        }
    }
    if (taken) {
#pragma unroll
        for (int j = 0; j < class_words(HD); ++j) {
            const int col = lane + j * kWave;
#pragma unroll 1
            for (int r = 0; r < 16 * NRG; ++r) {
                const int c = (int)(cls[j] >> (2 * r)) & 3;
                if (col < HD && c != 0)
                    reinterpret_cast<float *>(s_mine)[r * SROW + col] += class_value(c);
            }
        }
    }
}

// Loads of a chunk's K and V (bf16) into LDS by four waves. A wave takes every fourth KiB: keys of one of the
// chunk's tiles of 16, whose permutations repeat (so the same place of every tile, or two in turn).
template <int HD>
struct ChunkLoads {
    using TL = Tile<HD>;
    static constexpr int LPT = 16 / TL::RPK, VAR = LPT > 4 ? LPT / 4 : 1;  // loads of 16 keys
    uint32_t koff[VAR], voff[VAR];
    int lane, w;
    __device__ ChunkLoads(int tid) : lane(tid & 63), w(__builtin_amdgcn_readfirstlane(tid >> 6)) {
#pragma unroll
        for (int i = 0; i < VAR; ++i) {
            const int key = (w + 4 * i) % LPT * TL::RPK + lane / (kWave / TL::RPK), piece = lane % TL::NC;
            koff[i] = key * TL::ROWB + (piece ^ TL::kswz(key)) * 16;
            voff[i] = key * TL::ROWB + (piece ^ TL::vswz(key)) * 16;
        }
    }
    // Pages of a chunk's four tiles (past the request's last one: that), a lane each; asked for a chunk
    // before the chunk's loads.
    __device__ int pages(const PagedAttnParams &p, const int32_t *table, int c, int last_tile) const {
        return table[(min(4 * c + (lane & 3), last_tile) << 4) >> p.bk.page_shift];
    }
    __device__ void issue(const PagedAttnParams &p, int h, int c, int last_tile, int pg, uint8_t *dst) const {
        const int shift = p.bk.page_shift;
#pragma unroll
        for (int i = 0; i < TL::KIB / 4; ++i) {
            const int kb = w + 4 * i, tile = 4 * c + kb / LPT;
            const size_t page = __builtin_amdgcn_readlane(pg, kb / LPT);
            const size_t base = (((page * p.n_kv + h) << shift) + ((min(tile, last_tile) << 4) & ((1 << shift) - 1))) * TL::ROWB;
            __builtin_amdgcn_global_load_lds(
                static_cast<const void *>(static_cast<const uint8_t *>(p.k_pages) + base + koff[i % VAR]),
                (__attribute__((address_space(3))) void *)(dst + kb * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds(
                static_cast<const void *>(static_cast<const uint8_t *>(p.v_pages) + base + voff[i % VAR]),
                (__attribute__((address_space(3))) void *)(dst + TL::BYTES + kb * 1024), 16, 0, 0);
        }
    }
};

// Few rows. Workgroup: a block of up to 16 RG rows of one key head and some spans of its keys, one after
// another, a wave per chunk of 64 keys: K straight into registers in operand order, V through LDS (bf16:
// transposing reads) or straight (fp32). The loads of a workgroup are all in flight at once (128 KiB at
// head_dim 128, and two workgroups per CU); then it merges the chunks' states. A span's state goes to the
// partials, or, where the request has one span only (fp32: also where the partials do not hold the
// request's), the rows are written.
// Bound: reading the cache. Tokens of 64 requests at 1000 to 8000 keys (8 key heads of 128, pages of 16):
// 1.18 GB in 227 us, 5.2 TB/s, and 13 in the join (a large copy here reaches 4.9). Short calls: latency, a
// round trip each for the unit, the pages and the keys: one token at 512 keys 7.8 us and 3.3 in the join, 16
// rows at 700 9.2 and 3.2, 64 rows at 2304 23.7 and 4.8 (32 heads); fp32, 29 to 82 KiB of keys a head, 14.0
// and 3.8 (one workgroup a CU, as K takes the registers of two). Spans of 512 keys by eight waves leave one
// workgroup a CU: 259 us in place of 224. The last workgroup of a row joining its spans in place of a kernel costs
// 10 us of fences.
// Behind a window (WIN) the grid is (blocks x key heads, spans that a block sees, requests): the plan's units are all spans
// up to a row's position.
template <Prec P, int HD, int RG, bool WIN>
__global__ __launch_bounds__(kSpanChunks * kWave, P == Prec::BF16 && HD <= 128 ? 2 : 1) void paged_span_kernel(PagedAttnParams p,
                                                                                                  int cap_units) {
    constexpr bool WHOLE = P == Prec::F32 && !WIN;  // several spans without partials
    constexpr int NW = kSpanChunks, REGION = span_wave_lds<P, HD, RG>(), SROW = HD + 4, ROWS = 16 * RG;
    constexpr int ITEMS = (ROWS * HD / 4 + NW * kWave - 1) / (NW * kWave);
    extern __shared__ u32x4 s_raw[];
    uint8_t *s_all = reinterpret_cast<uint8_t *>(s_raw);
    __shared__ float s_m[NW][ROWS], s_l[NW][ROWS];  // the chunks' statistics
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint8_t *s_mine = s_all + (size_t)w * REGION;
    int h;
    PagedUnit u;
    for (SpanUnits<P, ROWS, WIN> units; units.next(p, cap_units, u, h);) {
        if (!WIN && u.k0 < 0) continue;  // a whole request's (uniform)
        const int rows = min(ROWS, u.m * p.group - u.row);
        const RowMap map(p, u.row);
        const int blast = u.ctx + map.token(rows - 1);  // the block's last position
        const int last_key = u.ctx + u.m - 1;
        const Sight<WIN> see(p);
        const Visible<WIN, kPagedSpanKeys> spans(see, WIN ? u.ctx + map.token(0) : 0, blast);
        const int s0 = u.k0, s1 = min(u.k1, spans.count);
        const int32_t *table = p.bk.table + (size_t)u.slot * p.bk.max_pages;
        if constexpr (WIN && P == Prec::F32) {
            // The span's chunks, or without partial states every chunk that the block sees, four at a time: to the same states in the
            // same order.
            const Visible<WIN, kKeys> chunks(see, u.ctx + map.token(0), blast);
            const int c0 = u.part < 0 ? 0 : spans.piece(s0) * kSpanChunks;
            const int count = u.part < 0 ? chunks.count : s0 < s1 ? min(NW, blast / kKeys + 1 - c0) : 0;
            auto chunk = [&](int j) { return u.part < 0 ? chunks.piece(j) : c0 + j; };
            struct State {
                float M = -INFINITY, l = 0.f;
                f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
                __device__ __forceinline__ void add(float Mn, float ln, f32x4 on) {
                    float v, vn;
                    merge_weights(M, Mn, v, vn);
                    l = merge_value(l, ln, v, vn);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = merge_value(o[e], on[e], v, vn);
                }
            } span[ITEMS], all[ITEMS];
            bool some[ITEMS] = {};  // the row sees a chunk of the span
            auto end_span = [&](int i) {
                if (some[i]) all[i].add(span[i].M, span[i].l, span[i].o);
                span[i] = State();
                some[i] = false;
            };
            for (int j = 0; j < count; j += NW) {
                const int key0 = chunk(j + w) * kKeys;
                if (j + w < count && see.some(u.ctx + map.token(0), key0, kKeys)) {  // uniform over the wave
                    if (RG == 1 || rows <= 16)
                        span_chunk<P, HD, WIN, 1>(p, u, map, h, rows, key0, last_key, table, s_mine, s_m[w], s_l[w]);
                    else
                        span_chunk<P, HD, WIN, RG>(p, u, map, h, rows, key0, last_key, table, s_mine, s_m[w], s_l[w]);
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    const int item = tid + i * NW * kWave, row = item / (HD / 4), col = item % (HD / 4) * 4;
                    if (row >= rows) break;
                    const int pos = u.ctx + map.token(row);
                    // (unrolled, heads of 128 spill: 2000 keys 462 us in place of 442; heads of 64 take 290 in place of 302)
#pragma unroll HD >= 128 ? 1 : NW
                    for (int k = 0; k < NW; ++k) {
                        if (j + k >= count) break;
                        const int c = chunk(j + k);
                        if (j + k > 0 && c / kSpanChunks != chunk(j + k - 1) / kSpanChunks) end_span(i);
                        if (c * kKeys > pos || !see.some(pos, c * kKeys, kKeys)) continue;
                        span[i].add(s_m[k][row], s_l[k][row], *reinterpret_cast<const f32x4 *>(
                            reinterpret_cast<const float *>(s_all + (size_t)k * REGION) + row * SROW + col));
                        some[i] = true;
                    }
                }
                __syncthreads();  // before the next chunks come into the regions
            }
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int item = tid + i * NW * kWave, row = item / (HD / 4), col = item % (HD / 4) * 4;
                if (row >= rows || s0 >= s1) break;
                if (u.part >= 0) {
                    const size_t pr = (size_t)(u.part + row) * p.n_kv + h;
                    *reinterpret_cast<f32x4 *>(p.part_o + pr * HD + col) = span[i].o;
                    if (col == 0) {
                        p.part_m[pr] = span[i].M;
                        p.part_l[pr] = span[i].l;
                    }
                } else {
                    end_span(i);
                    store_row<P>(p, u.r0 + map.token(row), h * p.group + map.head(row), col, all[i].o, all[i].M, all[i].l);
                }
            }
            continue;
        }
        // states of this thread's (row, four columns) items over the spans
        float Mr[WHOLE ? ITEMS : 1], lr[WHOLE ? ITEMS : 1];
        f32x4 orow[WHOLE ? ITEMS : 1];
        if constexpr (WHOLE) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) Mr[i] = -INFINITY, lr[i] = 0.f, orow[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        for (int s = s0; s < s1; ++s) {
            const int c0 = spans.piece(s) * kSpanChunks, key0 = (c0 + w) * kKeys;
            // uniform over the wave; a chunk that no row of the block sees is left out (the first row's window begins first)
            if (key0 <= blast && see.some(u.ctx + map.token(0), key0, kKeys)) {
                if (RG == 1 || rows <= 16)
                    span_chunk<P, HD, WIN, 1>(p, u, map, h, rows, key0, last_key, table, s_mine, s_m[w], s_l[w]);
                else
                    span_chunk<P, HD, WIN, RG>(p, u, map, h, rows, key0, last_key, table, s_mine, s_m[w], s_l[w]);
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int item = tid + i * NW * kWave, row = item / (HD / 4), col = item % (HD / 4) * 4;
                if (row >= rows) break;
                const int pos = u.ctx + map.token(row);
                float M = -INFINITY, l = 0.f;
                f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < NW; ++k) {
                    if ((c0 + k) * kKeys > pos) break;  // chunks that the row does not see
                    if (!see.some(pos, (c0 + k) * kKeys, kKeys)) continue;
                    const f32x4 oc = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(s_all + (size_t)k * REGION) +
                                                                      row * SROW + col);
                    float wo, wc;
                    merge_weights(M, s_m[k][row], wo, wc);
                    l = merge_value(l, s_l[k][row], wo, wc);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = merge_value(o[e], oc[e], wo, wc);
                }
                if (u.part >= 0) {
                    const size_t pr = (size_t)(u.part + (s - s0) * u.m * p.group + row) * p.n_kv + h;
                    *reinterpret_cast<f32x4 *>(p.part_o + pr * HD + col) = o;
                    if (col == 0) {
                        p.part_m[pr] = M;
                        p.part_l[pr] = l;
                    }
                    continue;
                }
                float Mo = -INFINITY, v, vc;
                if constexpr (WHOLE) {
                    if (c0 * kKeys <= pos && see.some(pos, c0 * kKeys, kPagedSpanKeys)) {
                        merge_weights(Mr[i], M, v, vc);
                        lr[i] = merge_value(lr[i], l, v, vc);
#pragma unroll
                        for (int e = 0; e < 4; ++e) orow[i][e] = merge_value(orow[i][e], o[e], v, vc);
                    }
                    if (s + 1 < s1) continue;
                    Mo = Mr[i];
                    l = lr[i];
                    o = orow[i];
                } else {
                    merge_weights(Mo, M, v, vc);  // the span into an empty state, as a join does
                    l = merge_value(0.f, l, v, vc);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = merge_value(0.f, o[e], v, vc);
                }
                store_row<P>(p, u.r0 + map.token(row), h * p.group + map.head(row), col, o, Mo, l);
            }
            __syncthreads();  // before the next chunks come into the regions
        }
    }
}

// A whole request of few rows (bf16) and one key head: 16 rows a wave, all keys. Chunks of K and V come into
// LDS once for all waves, one chunk ahead; a wave keeps its rows' state, over a span and over the spans, in
// registers. The same steps as with a wave per chunk and a join, in the same order, so the same bits.
// Bound: reading the cache, one chunk of 32 KiB a workgroup (head_dim 128, two a CU) ahead. 64 requests of 36
// rows at 4000 keys, 8 key heads: 205 us, 5.1 TB/s. 16 ragged requests of 32 rows at 256 to 1280 keys, 32
// heads: 218 MB in 49 us. The unit list is the span kernel's, and each passes over the other's units.
// Behind a window (WIN) it walks the plan's requests. 64 of four rows at 2000 to 32000 keys behind 4096, 8 key heads: 1057 MB in
// 189 us, 5.6 TB/s.
template <int HD, bool WIN>
__global__ __launch_bounds__(4 * kWave, HD <= 128 ? 2 : 1) void paged_request_kernel(PagedAttnParams p, int cap_units) {
    constexpr Prec P = Prec::BF16;
    using TL = Tile<HD>;
    constexpr int NKK = HD / 32, NDT = HD / 16;
    extern __shared__ u32x4 s_raw[];
    uint8_t *s_kv = reinterpret_cast<uint8_t *>(s_raw);  // [buffer][K, V]
    const ChunkLoads<HD> loads(threadIdx.x);
    const int lane = loads.lane, w = loads.w, g = lane >> 4, r16 = lane & 15;
    int count = 0;
    PagedUnit u;
    for (int idx = blockIdx.x; next_request<WIN>(p, idx / p.n_kv, cap_units, u, count); idx += gridDim.x) {
        if (u.k0 >= 0) continue;  // the span kernel's (uniform)
        const int h = idx % p.n_kv, rows = u.m * p.group;
        const int32_t *table = p.bk.table + (size_t)u.slot * p.bk.max_pages;
        const RowMap map(p, 0);
        const int last_key = u.ctx + u.m - 1, last_tile = last_key >> 4;
        const int blast = u.ctx + map.token(rows - 1), wlast = u.ctx + map.token(min(16 * w + 15, rows - 1));
        const Sight<WIN> see(p);
        const Visible<WIN, kKeys> chunks(see, u.ctx, blast);
        const int c1 = chunks.count, wfirst = WIN ? u.ctx + map.token(min(16 * w, rows - 1)) : 0;
        const bool live = 16 * w < rows;  // uniform over the wave
        const int row = min(16 * w + r16, rows - 1), token = map.token(row), head = h * p.group + map.head(row);
        int pg = loads.pages(p, table, chunks.piece(0), last_tile);
        __syncthreads();  // the unit before is done with the buffers
        loads.issue(p, h, chunks.piece(0), last_tile, pg, s_kv);
        pg = loads.pages(p, table, chunks.piece(1), last_tile);
        u32x4 q[NKK];
        const uint16_t *qrow = reinterpret_cast<const uint16_t *>(p.q) + (size_t)(u.r0 + token) * p.q_stride + head * HD + g * 8;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) q[kk] = *reinterpret_cast<const u32x4 *>(qrow + kk * 32);
        float M = -INFINITY, l = 0.f, Mr = -INFINITY, lr = 0.f;  // of the span, of the row
        f32x4 o[NDT], orow[NDT];
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] = orow[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int c = 0; c < c1; ++c) {
            const int chunk = chunks.piece(c), key0 = chunk * kKeys;
            const uint8_t *K = s_kv + (size_t)(c & 1) * 2 * TL::BYTES, *V = K + TL::BYTES;
            wait_vm_lds<0>();
            barrier_no_fence();  // every wave's pieces of the chunk have landed, and the other buffer has been read
            if (c + 1 < c1) loads.issue(p, h, chunks.piece(c + 1), last_tile, pg, s_kv + (size_t)((c + 1) & 1) * 2 * TL::BYTES);
            pg = loads.pages(p, table, chunks.piece(c + 2), last_tile);
            if (!live) continue;
            if (key0 <= wlast && see.some(wfirst, key0, kKeys)) {  // uniform over the wave
                f32x4 st[4];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) {
                    st[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kk = 0; kk < NKK; ++kk)
                        st[kt] = mfma_kstep<P>(*reinterpret_cast<const u32x4 *>(K + (16 * kt + r16) * TL::ROWB +
                                                                                ((4 * kk + g) ^ TL::kswz(r16)) * 16),
                                               q[kk], st[kt]);
                }
                const int qpos[1] = {u.ctx + token - key0};
                float mx, lc;
                u32x4 pb[1][2][2];
                chunk_softmax<WIN>(st, qpos[0], see, key0, p.scale_log2, lane, mx, lc);
                weight_operand<P>(st, pb[0]);
                f32x4 oc[1][NDT];
                uint64_t cls[class_words(HD)];
                const size_t at[4] = {};
                if (chunk_values<P, HD, WIN>(p, V, at, last_key - key0 + 1, key0, pb, qpos, oc, cls)) {
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {  // column 16 dt + 4 g + e
                            const uint32_t k = (uint32_t)__shfl((int)(uint32_t)cls[dt / 4], (16 * dt + 4 * g + e) & 63) >> (2 * r16) & 3;
                            if (k) oc[0][dt][e] += class_value(k);
                        }
                }
                if (qpos[0] >= 0 && see.some(u.ctx + token, key0, kKeys)) {
                    float wo, wc;
                    merge_weights(M, mx, wo, wc);
                    l = merge_value(l, lc, wo, wc);
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[dt][e] = merge_value(o[dt][e], oc[0][dt][e], wo, wc);
                }
            }
            if (WIN ? c + 1 < c1 && chunks.piece(c + 1) / kSpanChunks == chunk / kSpanChunks
                    : c % kSpanChunks + 1 < kSpanChunks && c + 1 < c1)
                continue;
            const int span0 = chunk / kSpanChunks * kPagedSpanKeys;
            if (span0 <= u.ctx + token && see.some(u.ctx + token, span0, kPagedSpanKeys)) {
                float v, vc;
                merge_weights(Mr, M, v, vc);
                lr = merge_value(lr, l, v, vc);
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) orow[dt][e] = merge_value(orow[dt][e], o[dt][e], v, vc);
            }
            M = -INFINITY;
            l = 0.f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if (16 * w + r16 < rows)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) store_row<P>(p, u.r0 + token, head, 16 * dt + 4 * g, orow[dt], Mr, lr);
    }
}

typedef __attribute__((ext_vector_type(16))) float f32x16;
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Whether x is true in some thread of four waves, and a barrier for what they have written to LDS. Loads in flight (the next
// chunk's) are not waited for, as __syncthreads_or() would. Between two calls there is another barrier.
__device__ __forceinline__ bool any_of_workgroup(bool x, int (&waves)[4]) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool any = __any(x);
    if ((threadIdx.x & 63) == 0) waves[w] = any;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));  // LDS alone
    barrier_no_fence();
    return waves[0] | waves[1] | waves[2] | waves[3];
}

// LDS of the tile kernel: two buffers of a chunk's K and V, and the classes of values that are not finite.
template <int HD>
constexpr int tile_lds() {
    return 4 * Tile<HD>::BYTES + kPagedTileRows / 16 * HD * 4;
}

// Long chunks (bf16). Workgroup: a tile of 128 rows of one key head and a range of its keys, 4 waves x 32
// rows. Chunks of 64 keys of K and V come into LDS by DMA, once for all waves, one chunk ahead. Per chunk
// and wave: S^T = K Q^T (32 keys x 32 rows a product), so that a lane holds half the keys of one row: the
// softmax is lane-local but for one exchange, and the weights are the next product's operand as they lie;
// O^T += V^T P^T with transposing reads of V. The weights are rounded to bf16 (at most half a step, 2^-8
// of each weight, of random sign: a sum over keys is off by less than the output's own rounding may be), their sum is
// not: 0.0023 off the formula where exact weights give 0.0017, the output's rounding alone. Weights of two planes as in
// the few rows' kernels take 606 us in place of 470 (the case below). The reference of the
// exponentials follows the running maximum only when that has grown by 2^8: weights are then at most 2^8
// in place of 1, which neither type minds, and the output is rescaled rarely.
// Bound: the matrix unit and, between its products, the softmax: 2048 tokens at 12288 (32 heads, 8 key heads
// of 128) take 462 to 483 us, 925 to 968 TFLOP/s (a large bf16 product of the library reaches 1200 here).
// Left out of a copy, the exponentials save 35 us, the DMA 60, three quarters of either product 105 to 125:
// nothing waits for one thing alone. Reads that run ahead of the softmax, softmax and products of two chunks
// interleaved in a wave, wave priorities and cheaper addresses changed nothing. Other heads: 64 wide 800
// TFLOP/s, 32 wide 640, 256 wide 490 (one workgroup a CU, and 32 registers spilled).
// Behind a window (WIN) a tile walks the chunks that its rows see; a range of the plan's is that share of them, or the first
// is all (tile_is_whole). 2048 tokens at 16384 behind 4096 and 64 sinks take 160 us, 872 TFLOP/s of visible keys (165 on another
// card). A chunk that some row does not see in whole takes 7 thousand clocks in place of 4: the look for values that are not
// finite, and the masks, as bits of a word a row (key by key, with a wait for the next chunk's loads in the look, 10).
template <int HD, bool WIN>
__global__ __launch_bounds__(4 * kWave, HD <= 128 ? 2 : 1) void paged_tile_kernel(PagedAttnParams p, int cap_tiles) {
    using TL = Tile<HD>;
    constexpr int NKK = HD / 16, NDT = HD / 32;
    extern __shared__ u32x4 s_raw[];
    uint8_t *s_kv = reinterpret_cast<uint8_t *>(s_raw);  // [buffer][K, V]
    uint32_t *s_cls = reinterpret_cast<uint32_t *>(s_kv + 4 * TL::BYTES);  // [column][16 rows]
    __shared__ int s_bad[4];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r32 = lane & 31, hb = lane >> 5;
    const ChunkLoads<HD> loads(tid);
    const float scale = fabsf(p.scale_log2);
    const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;  // the scale's sign goes into the queries
    int count = 0;
    PagedUnit u;
    for (int idx = blockIdx.x; next_unit<true>(p, idx / p.n_kv, cap_tiles, u, count); idx += gridDim.x) {
        const int h = idx % p.n_kv;
        const int rows = min(kPagedTileRows, u.m * p.group - u.row);
        const int32_t *table = p.bk.table + (size_t)u.slot * p.bk.max_pages;
        const int kvlen = u.ctx + u.m, last_tile = (kvlen - 1) >> 4;
        const RowMap map(p, u.row);
        const int tfirst = u.ctx + map.token(0), tlast = u.ctx + map.token(rows - 1);
        const int wfirst = u.ctx + map.token(min(32 * w, rows - 1)), wlast = u.ctx + map.token(min(32 * w + 31, rows - 1));
        const Sight<WIN> see(p);
        const Visible<WIN, kKeys> chunks(see, tfirst, tlast);
        int c0 = u.k0, c1 = min(u.k1, tlast / kKeys + 1);
        const bool one = tile_is_whole<WIN>(p, chunks, tlast);  // uniform
        if (one && u.k0 > 0) continue;
        const int part = one ? -1 : u.part;
        if (one) {
            c0 = 0;
            c1 = chunks.count;
        } else if (WIN && chunks.count <= tlast / kKeys) {
            const int all = (kvlen + kKeys - 1) / kKeys;
            c0 = (int)((int64_t)min(u.k0, all) * chunks.count / all);
            c1 = (int)((int64_t)min(u.k1, all) * chunks.count / all);
        }
        const bool live = 32 * w < rows;  // uniform over the wave
        const int rr = min(32 * w + r32, rows - 1), token = map.token(rr), head = h * p.group + map.head(rr);
        const int qpos = u.ctx + token;
        int pg = loads.pages(p, table, chunks.piece(c0), last_tile);
        __syncthreads();  // the unit before is done with the buffers
        if (c0 < c1) loads.issue(p, h, chunks.piece(c0), last_tile, pg, s_kv);
        pg = loads.pages(p, table, chunks.piece(c0 + 1), last_tile);
        u32x4 q[NKK];
        const uint16_t *qrow = reinterpret_cast<const uint16_t *>(p.q) + (size_t)(u.r0 + token) * p.q_stride + head * HD + hb * 8;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) q[kk] = *reinterpret_cast<const u32x4 *>(qrow + kk * 16) ^ flip;
        float M = -INFINITY, l = 0.f;  // l: this lane's half of the keys
        f32x16 o[NDT];
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
        for (int c = c0; c < c1; ++c) {
            const int buf = (c - c0) & 1, key0 = chunks.piece(c) * kKeys;
            wait_vm_lds<0>();
            barrier_no_fence();  // every wave's pieces of the chunk have landed, and the other buffer has been read
            if (c + 1 < c1) loads.issue(p, h, chunks.piece(c + 1), last_tile, pg, s_kv + (size_t)(buf ^ 1) * 2 * TL::BYTES);
            pg = loads.pages(p, table, chunks.piece(c + 2), last_tile);
            const uint8_t *K = s_kv + (size_t)buf * 2 * TL::BYTES;
            uint8_t *V = s_kv + (size_t)buf * 2 * TL::BYTES + TL::BYTES;
            if (key0 + kKeys - 1 > tfirst || see.cuts(tlast, key0, kKeys)) {  // uniform: keys that some row does not see
                // A weight of 0 does not silence a NaN or an infinity in the product. Values behind the
                // request's last token are cleared, whatever the page holds there; others that are not
                // finite (rare) are taken out, and what the rows that see them get from them is added to
                // their outputs: a sum per row and column, as a class of two bits (0, +inf, -inf, NaN).
                typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
                u16x2 size{};  // the largest magnitudes, as bits
#pragma unroll
                for (int i = 0; i < TL::BYTES / 16 / 256; ++i) {
                    u32x4 *v = reinterpret_cast<u32x4 *>(V) + tid + 256 * i;
                    if ((tid + 256 * i) / TL::NC >= kvlen - key0) {
                        *v = u32x4{0u, 0u, 0u, 0u};
                    } else {
                        const u32x4 x = *v;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            size = __builtin_elementwise_max(size, __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
                    }
                }
                if (any_of_workgroup(max(size[0], size[1]) >= 0x7f80, s_bad)) {
                    for (int col = tid; col < HD; col += 256) {
                        float acc = 0.f;
                        int key = 0;
                        uint64_t odd[3] = {};  // WIN: keys of +inf, -inf, NaN
                        auto next = [&]() {
                            uint16_t *v = reinterpret_cast<uint16_t *>(V + key * TL::ROWB + ((col / 8) ^ TL::vswz(key)) * 16) + col % 8;
                            const uint32_t x = (uint32_t)*v << 16;
                            if ((x & 0x7f800000u) == 0x7f800000u) {
                                acc += __uint_as_float(x);
                                if (WIN) odd[x == 0x7f800000u ? 0 : x == 0xff800000u ? 1 : 2] |= 1ull << key;
                                *v = 0;
                            }
                            ++key;
                        };
                        if (WIN)
                            while (key < kKeys) next();
                        for (int r0 = 0; r0 < kPagedTileRows; r0 += 16) {
                            uint32_t bits = 0;
                            for (int r = r0; r < r0 + 16; ++r) {
                                const int pos = u.ctx + map.token(min(r, rows - 1));
                                if constexpr (WIN) {
                                    const uint64_t seen = see.bits(pos, key0);
                                    const bool plus = odd[0] & seen, minus = odd[1] & seen;
                                    acc = (odd[2] & seen) || (plus && minus) ? NAN : plus ? INFINITY : minus ? -INFINITY : 0.f;
                                } else {
                                    while (key <= min(pos - key0, kKeys - 1)) next();
                                }
                                bits |= (acc != acc ? 3u : acc == INFINITY ? 1u : acc == -INFINITY ? 2u : 0u) << (2 * (r - r0));
                            }
                            s_cls[col * (kPagedTileRows / 16) + r0 / 16] = bits;
                        }
                        while (key < kKeys) next();
                    }
                    __syncthreads();
                    const int row = 32 * w + r32;
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int col = 32 * dt + 8 * (i / 4) + 4 * hb + i % 4;
                            const uint32_t k = s_cls[col * (kPagedTileRows / 16) + row / 16] >> (2 * (row % 16)) & 3;
                            o[dt][i] += k == 0 ? 0.f : k == 1 ? INFINITY : k == 2 ? -INFINITY : NAN;
                        }
                    __syncthreads();  // the classes have been read
                }
            }
            if (!live || key0 > wlast || !see.some(wfirst, key0, kKeys)) continue;
            // Reads run ahead of the products that take them (the scheduler would put each next to its
            // product, behind a wait for it alone).
            u32x4 kf[NKK][2];
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
                    kf[kk][kt] = *reinterpret_cast<const u32x4 *>(K + (32 * kt + r32) * TL::ROWB + ((2 * kk + hb) ^ TL::kswz(r32)) * 16);
            __builtin_amdgcn_sched_barrier(0);
            f32x16 st[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) st[kt][i] = 0.f;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) st[kt] = mfma32(kf[kk][kt], q[kk], st[kt]);
            // slot j of half hb of step ks: key 16 ks + 8 (j / 4) + 4 hb + j % 4
            const int vkey = 4 * hb + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            u32x2 vf[2][4][2];
            auto read_v = [&](int dt) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        vf[dt & 1][ks][y] = read_tr(V + vkey * TL::ROWB + ((4 * dt + vc) ^ TL::vswz(vkey)) * 16 + (lane & 1) * 8 +
                                                    (16 * ks + 8 * y) * TL::ROWB);
            };
            read_v(0);
            __builtin_amdgcn_sched_barrier(0);
            // st[kt][i] = S^T[key 32 kt + 8 (i / 4) + 4 hb + i % 4][row r32]
            if (key0 + kKeys - 1 > wfirst || see.cuts(wlast, key0, kKeys)) {
                const uint64_t seen = WIN ? see.bits(qpos, key0) >> (4 * hb) : 0;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int k = 8 * (i / 4) + i % 4;
                        if (WIN ? !((uint32_t)(seen >> (32 * kt)) >> k & 1) : key0 + 32 * kt + 4 * hb + k > qpos) st[kt][i] = -INFINITY;
                    }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[kt][i]);
            const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1])) * scale;
            if (__any(mx > M + 8.f)) {
                // (where M is -inf, l is 0 and o holds only what values that are not finite gave: kept)
                const float Mn = fmaxf(M, mx), f = M == -INFINITY ? 1.f : exp2_weight(M - Mn);
                l *= f;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[dt][i] *= f;
                M = Mn;
            }
            const float ref = M == -INFINITY ? 0.f : M;  // nothing seen: every weight is 0
            u32x4 pb[4];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float a = exp2_weight(__builtin_fmaf(st[kt][i], scale, -ref));
                    const float b = exp2_weight(__builtin_fmaf(st[kt][i + 1], scale, -ref));
                    l += a + b;
                    pb[2 * kt + i / 8][i / 2 % 4] = pack_bf16(a, b);
                }
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                if (dt + 1 < NDT) {
                    read_v(dt + 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    const u32x2 x = vf[dt & 1][ks][0], y = vf[dt & 1][ks][1];
                    o[dt] = mfma32(u32x4{x[0], x[1], y[0], y[1]}, pb[ks], o[dt]);
                }
            }
        }
        l += __shfl_xor(l, 32);
        const int row = 32 * w + r32;
        if (row < rows) {
            const size_t pr = (size_t)(part + row) * p.n_kv + h;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4 x = f32x4{o[dt][i], o[dt][i + 1], o[dt][i + 2], o[dt][i + 3]};
                    const int col = 32 * dt + 8 * (i / 4) + 4 * hb;
                    if (part >= 0)
                        *reinterpret_cast<f32x4 *>(p.part_o + pr * HD + col) = x;
                    else
                        store_row<Prec::BF16>(p, u.r0 + token, head, col, x, M, l);
                }
            if (part >= 0 && hb == 0) {
                p.part_m[pr] = M;
                p.part_l[pr] = l;
            }
        }
    }
}

// Joins the partial states of split row blocks, in position order. Workgroup: some rows of one key head of
// an item, a thread per four columns of a row. Bound: latency, four states in flight a thread: 3.3 us for three
// spans, 13 us for 64 requests of 4 to 32 spans (16 in flight: 15.5 in place of 8.3 us at 16 requests).
template <Prec P, int HD, bool WIN>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnParams p, int cap_items) {
    constexpr int LPR = HD / 4, RPW = 256 / LPR, NG = (kPagedItemRows + RPW - 1) / RPW;
    if constexpr (WIN && P == Prec::F32) {  // the call's own places: by requests
        PagedEntry e;
        for (int z = blockIdx.z, n; next_entry(p, z, e, n); z += gridDim.z)
            for (int i = blockIdx.x; i / (p.n_kv * NG) * kPagedItemRows < e.m * p.group; i += gridDim.x) {
                const int row = i / (p.n_kv * NG) * kPagedItemRows;
                const PagedItem mine{e.ctx, e.m, e.r0, row, window_part<P>(p, e) + row, e.m * p.group, 0, 0};
                join_row<P, HD, WIN>(p, mine, i % p.n_kv, i / p.n_kv % NG * RPW + threadIdx.x / LPR, threadIdx.x % LPR * 4);
            }
        return;
    }
    const int32_t *st = p.bk.status;
    const int R = st[PS_ROWS], n = st[PS_ITEMS], br = st[PS_BOUND_ROWS], bn = st[PS_BOUND_NEW], bl = st[PS_BOUND_LEN];
    PagedItem it = p.bk.items[min((int)blockIdx.x / (p.n_kv * NG), cap_items - 1)];
    request_together(R, n, br, bn, bl, it.ctx, it.m, it.r0, it.row, it.part, it.stride, it.count);
    if (R == 0 || br != p.rows || bn != p.max_new || bl != p.max_len) return;
    const int work = n * p.n_kv * NG;
    for (int idx = blockIdx.x; idx < work; idx += gridDim.x) {
        if (idx != (int)blockIdx.x) it = p.bk.items[idx / (p.n_kv * NG)];
        join_row<P, HD, WIN>(p, it, idx % p.n_kv, idx / p.n_kv % NG * RPW + threadIdx.x / LPR, threadIdx.x % LPR * 4);
    }
}

namespace {

template <Prec P, int HD, int RG>
hipError_t launch_spans(int64_t units, bool whole, const PagedAttnParams &p, hipStream_t s) {
    constexpr int lds = kSpanChunks * span_wave_lds<P, HD, RG>();
    static_assert(lds + 4096 <= 160 * 1024, "the LDS of a CU");
    static_assert(16 * RG == paged_block_rows(P == Prec::BF16, HD), "the plan's row blocks");
    // (where requests may be taken whole, fewer: passing over 2560 units takes 6.5 us, 4.6 in a grid of 1024; spans in
    // a grid of 1024 take up to 2% longer)
    const dim3 grid((unsigned)std::min<int64_t>(units * p.n_kv, whole ? 4 * kCUs : 16 * kCUs));
    hipLaunchKernelGGL((paged_span_kernel<P, HD, RG, false>), grid, dim3(kSpanChunks * kWave), lds, s, p, p.bk.cap_units);
    return hipGetLastError();
}

template <Prec P, int HD, bool WIN>
hipError_t launch_join(int64_t units, int64_t tiles, const PagedAttnParams &p, hipStream_t s) {
    const int64_t groups = (kPagedItemRows + 1024 / HD - 1) / (1024 / HD);
    const int64_t work = std::min<int64_t>(units + 4 * tiles, p.bk.cap_items) * p.n_kv * groups;
    hipLaunchKernelGGL((paged_join_kernel<P, HD, WIN>), dim3((unsigned)std::min<int64_t>(work, 8 * kCUs)), dim3(256), 0, s, p,
                       p.bk.cap_items);
    return hipGetLastError();
}

template <int HD, bool WIN>
hipError_t launch_tiles(int64_t tiles, const PagedAttnParams &p, hipStream_t s) {
    hipLaunchKernelGGL((paged_tile_kernel<HD, WIN>), dim3((unsigned)std::min<int64_t>(tiles * p.n_kv, 16 * kCUs)), dim3(4 * kWave),
                       tile_lds<HD>(), s, p, p.bk.cap_tiles);
    return hipGetLastError();
}

template <Prec P, int HD, int RG>
struct FullCall {
    int64_t units;
    bool whole;
    int64_t tiles;
    bool join;
    hipError_t operator()(const PagedAttnParams &p, hipStream_t s) const {
        hipError_t e = launch_spans<P, HD, RG>(units, whole, p, s);
        if constexpr (P == Prec::BF16) {
            if (e == hipSuccess && whole) {
                hipLaunchKernelGGL((paged_request_kernel<HD, false>), dim3((unsigned)std::min<int64_t>(units * p.n_kv, 16 * kCUs)),
                                   dim3(4 * kWave), 4 * Tile<HD>::BYTES, s, p, p.bk.cap_units);
                e = hipGetLastError();
            }
            if (e == hipSuccess && tiles > 0) e = launch_tiles<HD, false>(tiles, p, s);
        }
        return e == hipSuccess && join ? launch_join<P, HD, false>(units, tiles, p, s) : e;
    }
};

template <Prec P, int HD, int RG>
struct WindowCall {
    int n;
    int64_t most;
    bool whole;
    int64_t tiles;
    bool join;
    hipError_t launch_requests(const PagedAttnParams &p, hipStream_t s) const {
        hipLaunchKernelGGL((paged_request_kernel<HD, true>), dim3((unsigned)std::min(n * p.n_kv, 16 * kCUs)), dim3(4 * kWave),
                           4 * Tile<HD>::BYTES, s, p, 0);
        return hipGetLastError();
    }
    // Whether requests of up to kPagedFewRows rows are all taken whole, whatever the plan made of them, with nothing else to
    // launch: one workgroup a request and key head, which walks the chunks that it sees (2.2 us each at heads of 128, 512
    // workgroups at a time), in place of one a block and span (about 12 us, 512 at a time), of which several work on a
    // request at once, and a join. us of a call at 4096 keys behind 16 / 256 / 1024, in spans and whole:
    //   32 heads over 8 of 128: 1 x 64 requests 26.4 / 34.6 / 75.9 and 18.2 / 25.4 / 58.8; 1 x 16: 12.9 / 15.8 / 25.8 and 13.4 /
    //   20.6 / 46.5; 16 x 32: 35.9 / 54.2 / 98.3 and 16.4 / 25.3 / 53.2; 16 x 8: 15.4 / 21.0 / 34.0 and 12.2 / 21.5 / 48.3
    //   32 heads of 128: 32 x 1: 13.6 / 16.5 / 17.8 and 13.6 / 20.3 / 47.3; 8 heads of 64: 24 x 22: 14.2 / 22.9 / 31.1 and 10.8 / 17.4 /
    //   37.4; 4 over 2 of 256: 16 x 16: 17.4 / 21.7 / 36.4 and 23.1 / 35.5 / 85.0
    bool all_whole(const PagedAttnParams &p) const {
        if (most > kPagedFewRows) return false;
        const int64_t groups = (int64_t)n * p.n_kv, blocks = (most + 16 * RG - 1) / (16 * RG), slots = (HD <= 128 ? 2 : 1) * kCUs;
        const double keys = std::min<double>((double)p.window + p.max_new - 1, p.max_len);
        const double chunks = keys / kKeys + 1 + (p.sinks + kKeys - 1) / kKeys;
        const double spans = keys / kPagedSpanKeys + 1 + (p.sinks + kPagedSpanKeys - 1) / kPagedSpanKeys;
        const double chunks_of_a_span = (most <= kPagedWaveRows ? 4 : 6) * (HD <= 64 ? 4.0 / 3 : HD <= 128 ? 1 : 2.0 / 3);
        return chunks * std::max(groups, slots) <= chunks_of_a_span * spans * (blocks * groups);
    }
    hipError_t operator()(const PagedAttnParams &call, hipStream_t s) const {
        constexpr int ROWS = 16 * RG;
        PagedAttnParams p = call;
        if constexpr (P == Prec::BF16) {
            p.all_whole = all_whole(p);
            if (p.all_whole) return launch_requests(p, s);
        }
        p.blocks = (int)((std::min<int64_t>(most, P == Prec::BF16 ? kPagedFewRows : most) + ROWS - 1) / ROWS);
        if (P == Prec::F32) p.split = p.spans > 1 && split(p);
        const dim3 grid((unsigned)std::min(p.blocks * p.n_kv, 1 << 20), P == Prec::F32 && !p.split ? 1u : (unsigned)p.spans, (unsigned)n);
        hipLaunchKernelGGL((paged_span_kernel<P, HD, RG, true>), grid, dim3(kSpanChunks * kWave),
                           kSpanChunks * (span_wave_lds<P, HD, RG>()), s, p, 0);
        hipError_t e = hipGetLastError();
        if constexpr (P == Prec::BF16) {
            if (e == hipSuccess && whole) e = launch_requests(p, s);
            if (e == hipSuccess && tiles > 0) e = launch_tiles<HD, true>(tiles, p, s);
        }
        if constexpr (P == Prec::F32) {
            if (e != hipSuccess || !p.split) return e;
            const int64_t work = (most + kPagedItemRows - 1) / kPagedItemRows * p.n_kv * ((kPagedItemRows + 1024 / HD - 1) / (1024 / HD));
            hipLaunchKernelGGL((paged_join_kernel<P, HD, true>), dim3((unsigned)std::min<int64_t>(work, 8 * kCUs), 1, (unsigned)n), dim3(256),
                               0, s, p, p.bk.cap_items);
            return hipGetLastError();
        }
        return e == hipSuccess && join ? launch_join<P, HD, true>((int64_t)n * p.blocks, tiles, p, s) : e;
    }
    // fp32: whether a block's spans are worked on side by side and joined, or its chunks four at a time by one workgroup: about 12 us
    // for each 256 spans and 4 for the join, or 5 us and 7 for each four chunks. us of a call behind 6 / 300 / 2000 keys, side by side
    // and one workgroup: 28 tokens of 4 heads over 1 of 128: 17.8 / 21.0 / 32.9 and 15.5 / 39 / 110; 5 requests of 3 to 41 tokens of 12
    // heads of 64 behind 101: 19.4 and 16.3; 2 of 300 of 8 heads of 32: 14.3 / 24.6 / 61.3 and 10.5 / 17.0 / 61.6; 22 of 50 of 4
    // heads of 64: 28.3 / 43.0 / 93.6 and 15.7 / 27.6 / 104.
    bool split(const PagedAttnParams &p) const {
        if ((int64_t)p.spans * p.rows * p.group > p.cap_part) return false;
        const double keys = std::min<double>((double)p.window + std::min(p.max_new, 16 * RG) - 1, p.max_len);
        const double chunks = keys / kKeys + 1 + (p.sinks + kKeys - 1) / kKeys;
        const double spans = keys / kPagedSpanKeys + 1 + (p.sinks + kPagedSpanKeys - 1) / kPagedSpanKeys;
        const double rounds = (double)n * p.blocks * p.n_kv / kCUs;
        return 12 * std::max(rounds * spans, 1.0) + 4 < (5 + 7 * (chunks / kSpanChunks + 0.5)) * std::max(rounds, 1.0);
    }
};

// The call of the shape.
template <template <Prec, int, int> class Call, class... A>
hipError_t launch_shape(bool bf16, const PagedAttnParams &p, hipStream_t s, A... a) {
    if (p.n_kv < 1 || p.group < 1 || p.n_heads != p.n_kv * p.group) return hipErrorInvalidValue;
    if (bf16) {
        if (p.hd == 32) return Call<Prec::BF16, 32, 2>{a...}(p, s);
        if (p.hd == 64) return Call<Prec::BF16, 64, 2>{a...}(p, s);
        if (p.hd == 128) return Call<Prec::BF16, 128, 2>{a...}(p, s);
        if (p.hd == 256) return Call<Prec::BF16, 256, 1>{a...}(p, s);
    } else {
        if (p.hd == 16) return Call<Prec::F32, 16, 2>{a...}(p, s);
        if (p.hd == 32) return Call<Prec::F32, 32, 2>{a...}(p, s);
        if (p.hd == 64) return Call<Prec::F32, 64, 2>{a...}(p, s);
        if (p.hd == 128) return Call<Prec::F32, 128, 1>{a...}(p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_paged_attn(bool bf16, int64_t units, bool whole, int64_t tiles, bool join, const PagedAttnParams &p, hipStream_t s) {
    if (units < 0 || tiles < 0) return hipErrorInvalidValue;
    if (units + tiles == 0 || p.rows == 0) return hipSuccess;
    return launch_shape<FullCall>(bf16, p, s, units, whole, tiles, join);
}

hipError_t launch_paged_attn_window(bool bf16, int n, int64_t most, bool whole, int64_t tiles, bool join, const PagedAttnParams &p,
                                    hipStream_t s) {
    if (n < 1 || most < 0 || tiles < 0 || p.window < 1 || p.sinks < 0 || p.spans < 1) return hipErrorInvalidValue;
    if (most == 0 || p.rows == 0) return hipSuccess;
    return launch_shape<WindowCall>(bf16, p, s, n, most, whole, tiles, join);
}

}  // namespace cllm

// Attention of chunks of new tokens over a paged KV cache on gfx950.
//
// Row (b, i, h) of a plan, token i of request b's chunk at position ctx_b + i, head h of the group of
// key head h / group: softmax over the request's tokens t <= ctx_b + i of scale q . k_t, times v_t. The
// keys of a request are walked in chunks of 64 at absolute positions. A chunk's state per row is its
// maximum, its sum and its unnormalised output; states are merged in position order, the chunks of a
// span of 512 keys first, then the spans. The order depends on positions alone: a row's bits are the
// same whichever rows, requests, pages and launches it is computed with.
//
// Values: scores and softmax statistics in fp32; bf16 probabilities as hi + lo planes (~2^-17), so the
// only rounding to bf16 is that of the output. Keys past a row's position contribute nothing, whatever
// their values (NaN, infinities): scores are selected away, and values by the rules at chunk_output.
#include <algorithm>

#include "device.h"
#include "paged.h"

namespace cllm {

namespace {

constexpr int kKeys = kAttnChunk;  // keys of a chunk
constexpr int kSpanChunks = kPagedSpanKeys / kKeys;

// LDS image of a chunk's K or V: [64 keys][head_dim], 16-byte pieces permuted within a row so that the
// reads below hit different banks: K is read 16 keys at one column (lanes of a group), bf16 V 16 keys
// x 32 bytes (transposing reads), fp32 V 4 keys (4 apart) x 64 bytes.
template <Prec P, int HD>
struct Tile {
    using T = typename PrecT<P>::T;
    static constexpr int VEC = PrecT<P>::VEC;
    static constexpr int ROWB = HD * (int)sizeof(T);  // bytes of a key
    static constexpr int NC = ROWB / 16;              // 16-byte pieces of a key
    static constexpr int BYTES = kKeys * ROWB;
    static constexpr int KIB = BYTES / 1024;          // wave loads of a tile
    static constexpr int RPK = 1024 / ROWB;           // keys per wave load (1..16)
    static_assert(RPK >= 1 && RPK <= 16 && NC >= 4, "a wave load stays within 16 keys");
    __device__ static int kswz(int key) { return NC >= 16 ? key & 15 : (key / (16 / NC)) & (NC - 1); }
    __device__ static int vswz(int key) {
        if constexpr (P == Prec::BF16) {
            constexpr int NP = HD / 16;  // 32-byte pairs
            return 2 * (NP >= 8 ? key & 7 : (key / (8 / NP)) & (NP - 1));
        } else {
            constexpr int NB = HD / 16;  // 64-byte blocks
            return NB >= 4 ? 4 * ((key >> 2) & 3) : 4 * ((key >> 2) & (NB - 1));
        }
    }
};

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Four keys 4 g .. 4 g + 3 (of 16) of one column: lane (g, r) addresses key 4 g + r / 4, columns
// 4 (r % 4) .., of a 16-column tile and receives column r.
__device__ __forceinline__ u32x2 read_tr(const uint8_t *lds) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4 *)lds));
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

// Scores of a chunk for 16 rows: st[kt][v] = S^T[key 16 kt + 4 g + v][row r16], from K in LDS.
template <Prec P, int HD>
__device__ __forceinline__ void chunk_scores(const uint8_t *K, const u32x4 (&q)[HD / PrecT<P>::KSTEP], int lane, f32x4 (&st)[4]) {
    using TL = Tile<P, HD>;
    constexpr int NKK = HD / PrecT<P>::KSTEP;
    const int g = lane >> 4, r16 = lane & 15;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
        const int key = 16 * kt + r16;
        st[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk)
            st[kt] = mfma_kstep<P>(*reinterpret_cast<const u32x4 *>(K + key * TL::ROWB + ((4 * kk + g) ^ TL::kswz(key)) * 16),
                                   q[kk], st[kt]);
    }
}

// Scores to probabilities: keys past qpos (relative to the chunk's first key) are out. mx: the row's
// maximum (-inf: it sees no key), l: its sum.
__device__ __forceinline__ void chunk_softmax(f32x4 (&st)[4], int qpos, float scale_log2, int lane, float &mx, float &l) {
    const int g = lane >> 4;
    mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float sc = 16 * kt + 4 * g + v <= qpos ? st[kt][v] * scale_log2 : -INFINITY;
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

// The V operand of 16 columns: vb[x] holds the keys of the probabilities' registers. bf16: x = 0, 1,
// keys 32 x + 4 g + (0..3) and 32 x + 16 + 4 g + (0..3); fp32: x = 0..3, keys 16 x + 4 g + (0..3).
template <Prec P, int HD>
__device__ __forceinline__ void v_operand(const uint8_t *V, int dt, int lane, u32x4 (&vb)[P == Prec::BF16 ? 2 : 4]) {
    using TL = Tile<P, HD>;
    const int g = lane >> 4, r16 = lane & 15;
    if constexpr (P == Prec::BF16) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            u32x2 h[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int key = 32 * x + 16 * y + 4 * g + (r16 >> 2), c = 2 * dt + ((r16 & 3) >> 1);
                h[y] = read_tr(V + key * TL::ROWB + (c ^ TL::vswz(key)) * 16 + (r16 & 1) * 8);
            }
            vb[x] = u32x4{h[0][0], h[0][1], h[1][0], h[1][1]};
        }
    } else {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int key = 16 * x + 4 * g + y, c = 4 * dt + (r16 >> 2);
                vb[x][y] = *reinterpret_cast<const uint32_t *>(V + key * TL::ROWB + (c ^ TL::vswz(key)) * 16 + (r16 & 3) * 4);
            }
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
    if constexpr (P == Prec::BF16) {
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const f32x4 pa = st[2 * x], pc = st[2 * x + 1];
            const float pv[8] = {pa[0], pa[1], pa[2], pa[3], pc[0], pc[1], pc[2], pc[3]};
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                hi[i] = f2bf(pv[i]);
                lo[i] = f2bf(pv[i] - bf2f((uint16_t)hi[i]));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pb[0][x][i] = hi[2 * i] | (hi[2 * i + 1] << 16);
                if constexpr (NPL == 2) pb[NPL - 1][x][i] = lo[2 * i] | (lo[2 * i + 1] << 16);
            }
        }
    } else {
#pragma unroll
        for (int x = 0; x < N; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) pb[0][x][i] = __float_as_uint(st[x][i]);
    }
}

// Operand elements that are NaN or infinite, as (nan, +inf, -inf) indicators (1.0 / 0.0) and the
// operand without them.
template <Prec P, int N>
__device__ __forceinline__ void split_nonfinite(u32x4 (&vb)[N], u32x4 (&ind)[3][N]) {
    constexpr bool B = P == Prec::BF16;
    constexpr uint32_t ONE = B ? 0x3f80u : 0x3f800000u, INF = B ? 0x7f80u : 0x7f800000u, SIGN = B ? 0x8000u : 0x80000000u;
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t out[4] = {0, 0, 0, 0};
#pragma unroll
            for (int half = 0; half < (B ? 2 : 1); ++half) {
                const uint32_t e = B ? (vb[x][i] >> (16 * half)) & 0xffffu : vb[x][i], mag = e & ~SIGN;
                const int sh = 16 * half;
                out[0] |= (mag > INF ? ONE : 0u) << sh;
                out[1] |= (e == INF ? ONE : 0u) << sh;
                out[2] |= (e == (INF | SIGN) ? ONE : 0u) << sh;
                out[3] |= (mag >= INF ? 0u : e) << sh;
            }
            ind[0][x][i] = out[0];
            ind[1][x][i] = out[1];
            ind[2][x][i] = out[2];
            vb[x][i] = out[3];
        }
}

// Unnormalised output of a chunk for 16 rows: o[dt][e] = O^T[16 dt + 4 g + e][row r16].
//
// A weight of 0 does not silence an infinite or NaN value in the product, and a weight's lo plane may turn
// an infinity into a NaN. Both leave a NaN in some output, so outputs without one are right as they are;
// behind one (rare) the values that are not finite are taken out of the operand, and each row gets what
// those that it sees make of it: NaN for a NaN or an infinity of weight 0 (as 0 x inf is), the infinity
// otherwise.
template <Prec P, int HD>
__device__ __forceinline__ void chunk_output(const uint8_t *V, const f32x4 (&st)[4], int qpos, int lane, f32x4 (&o)[HD / 16]) {
    constexpr int N = P == Prec::BF16 ? 2 : 4, NPL = PrecT<P>::PLANES;
    u32x4 pb[NPL][N];
    weight_operand<P>(st, pb);
    float sum = 0.f;
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt) {
        u32x4 vb[N];
        v_operand<P, HD>(V, dt, lane, vb);
        o[dt] = v_product<P>(vb, pb);
        sum += (o[dt][0] + o[dt][1]) + (o[dt][2] + o[dt][3]);
    }
    if (!__any(sum != sum)) return;
    const int g = lane >> 4;
    f32x4 seen[4], pos[4], zero[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const bool vis = 16 * kt + 4 * g + v <= qpos;
            seen[kt][v] = vis ? 1.0f : 0.0f;
            pos[kt][v] = vis && st[kt][v] > 0.0f ? 1.0f : 0.0f;
            zero[kt][v] = vis && st[kt][v] == 0.0f ? 1.0f : 0.0f;
        }
    u32x4 sb[1][N], pp[1][N], zb[1][N];
    weight_operand<P>(seen, sb);
    weight_operand<P>(pos, pp);
    weight_operand<P>(zero, zb);
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt) {
        u32x4 vb[N], ind[3][N];
        v_operand<P, HD>(V, dt, lane, vb);
        split_nonfinite<P>(vb, ind);
        const f32x4 nan = v_product<P>(ind[0], sb), up = v_product<P>(ind[1], pp), down = v_product<P>(ind[2], pp),
                    z0 = v_product<P>(ind[1], zb), z1 = v_product<P>(ind[2], zb);
        o[dt] = v_product<P>(vb, pb);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (nan[e] > 0.f || z0[e] > 0.f || z1[e] > 0.f)
                o[dt][e] = NAN;
            else
                o[dt][e] += (up[e] > 0.f ? INFINITY : 0.f) + (down[e] > 0.f ? -INFINITY : 0.f);
        }
    }
}

// What a workgroup knows of its unit.
struct Unit {
    int slot, ctx, m, r0;  // the request's entry
    int rb;                // first row of the block, in rows x heads of the group
    int rows;              // rows of the block
    int span0, span1;      // spans of keys
    int part;              // first partial row (-1: none)
};

// Row r of a request's rows x heads: token r / group, head r % group of the group.
__device__ __forceinline__ Unit unit_of(const PagedAttnParams &p, int4 u) {
    const int4 e = p.bk.ent[u.x];
    Unit t;
    t.slot = e.x;
    t.ctx = e.y;
    t.m = e.z;
    t.r0 = e.w;
    t.rb = u.y * kPagedBlockRows;
    t.rows = min(kPagedBlockRows, t.m * p.group - t.rb);
    const int last = t.ctx + (t.rb + t.rows - 1) / p.group;
    t.span0 = u.z < 0 ? 0 : u.z;
    t.span1 = u.z < 0 ? last / kPagedSpanKeys + 1 : u.z + 1;
    t.part = u.w;
    return t;
}

}  // namespace

// Two buffers of a chunk's K and V (at most 128 of a CU's 160 KiB).
template <Prec P, int HD>
constexpr int paged_rows_lds() {
    return 4 * Tile<P, HD>::BYTES;
}

// Workgroup: one key head of a unit, 4 waves x 16 rows; chunks of K and V come into LDS by DMA, once for
// all waves, one chunk ahead. Workgroups take units in turn.
template <Prec P, int HD>
__global__ __launch_bounds__(4 * kWave) void paged_rows_kernel(PagedAttnParams p) {
    using PT = PrecT<P>;
    using T = typename PT::T;
    using TL = Tile<P, HD>;
    constexpr int NKK = HD / PT::KSTEP, NDT = HD / 16;
    extern __shared__ u32x4 s_raw[];
    uint8_t *s_kv = reinterpret_cast<uint8_t *>(s_raw);  // [buffer][K, V]
    if (bounded_rows(p.bk, p.rows, p.max_new, p.max_len) == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, r16 = lane & 15, shift = p.bk.page_shift;
    const int work = p.bk.status[PS_UNITS] * p.n_kv;
    for (int idx = blockIdx.x; idx < work; idx += gridDim.x) {
        const int h = idx % p.n_kv;
        const Unit t = unit_of(p, p.bk.units[idx / p.n_kv]);
        const int32_t *table = p.bk.table + (size_t)t.slot * p.bk.max_pages;
        const int kvlen = t.ctx + t.m, last_tile = (kvlen - 1) >> 4;
        const int blast = t.ctx + (t.rb + t.rows - 1) / p.group;  // the block's last position
        const int c0 = t.span0 * kSpanChunks, c1 = min(t.span1 * kSpanChunks, blast / kKeys + 1);
        const bool live = 16 * w < t.rows;  // uniform over the wave
        const int rr = min(t.rb + 16 * w + r16, t.rb + t.rows - 1);  // rows past the block: its last one, not stored
        const int token = rr / p.group, head = h * p.group + rr % p.group;
        const int qpos = t.ctx + token;
        // page ids of the 64 tiles of 16 keys from tile 64 j on, one per lane
        auto page_ids = [&](int j) { return table[(min(64 * j + lane, last_tile) << 4) >> shift]; };
        int pj = c0 / 16, pg = page_ids(pj), pg_next = page_ids(pj + 1);
        auto issue = [&](int c, int buf) {
            if (c / 16 != pj) {
                pj = c / 16;
                pg = pg_next;
                pg_next = page_ids(pj + 1);
            }
#pragma unroll
            for (int i = 0; i < 2 * TL::KIB / 4; ++i) {
                const int blk = w + 4 * i, isv = blk >= TL::KIB, kb = isv ? blk - TL::KIB : blk;
                const int key = kb * TL::RPK + lane / (kWave / TL::RPK);  // within the chunk
                const int tile = min(4 * c + kb * TL::RPK / 16, last_tile);
                const int page = __builtin_amdgcn_readlane(pg, (4 * c + kb * TL::RPK / 16) & 63);
                const int off = ((tile << 4) & ((1 << shift) - 1)) + (key & 15);
                const int piece = (lane % TL::NC) ^ (isv ? TL::vswz(key) : TL::kswz(key));
                const uint8_t *src = reinterpret_cast<const uint8_t *>(isv ? p.v_pages : p.k_pages) +
                                     ((((size_t)page * p.n_kv + h) << shift) + off) * TL::ROWB + piece * 16;
                __builtin_amdgcn_global_load_lds(
                    static_cast<const void *>(src),
                    (__attribute__((address_space(3))) void *)(s_kv + (size_t)buf * 2 * TL::BYTES + blk * 1024), 16, 0, 0);
            }
        };
        __syncthreads();  // the unit before is done with the buffers
        issue(c0, 0);
        u32x4 q[NKK];
        const T *qrow = reinterpret_cast<const T *>(p.q) + (size_t)(t.r0 + token) * p.q_stride + head * HD;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) q[kk] = *reinterpret_cast<const u32x4 *>(qrow + kk * PT::KSTEP + g * PT::VEC);
        float M = -INFINITY, l = 0.f, Mr = -INFINITY, lr = 0.f;  // the span's state, the row's
        f32x4 o[NDT], orow[NDT];
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] = orow[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int c = c0; c < c1; ++c) {
            const int buf = (c - c0) & 1;
            wait_vm_lds<0>();
            barrier_no_fence();  // every wave's pieces of the chunk have landed
            if (c + 1 < c1) issue(c + 1, buf ^ 1);
            uint8_t *K = s_kv + (size_t)buf * 2 * TL::BYTES, *V = K + TL::BYTES;
            if ((c + 1) * kKeys > kvlen) {  // values behind the request's last token: whatever the page holds
                const int from = kvlen - c * kKeys;
                for (int i = from * TL::NC + tid; i < kKeys * TL::NC; i += 4 * kWave)
                    reinterpret_cast<u32x4 *>(V)[i] = u32x4{0u, 0u, 0u, 0u};
                wait_vm_lds<63>();
                barrier_no_fence();
            }
            if (live && c * kKeys <= t.ctx + min(t.rb + 16 * w + 15, t.rb + t.rows - 1) / p.group) {
                f32x4 st[4], oc[NDT];
                float mx, lc, wo, wc;
                chunk_scores<P, HD>(K, q, lane, st);
                chunk_softmax(st, qpos - c * kKeys, p.scale_log2, lane, mx, lc);
                chunk_output<P, HD>(V, st, qpos - c * kKeys, lane, oc);
                merge_weights(M, mx, wo, wc);
                l = merge_value(l, lc, wo, wc);
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[dt][e] = merge_value(o[dt][e], oc[dt][e], wo, wc);
            }
            if (c + 1 == c1 || (c + 1) % kSpanChunks == 0) {  // the span's end
                float w0, w1;
                merge_weights(Mr, M, w0, w1);
                lr = merge_value(lr, l, w0, w1);
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) orow[dt][e] = merge_value(orow[dt][e], o[dt][e], w0, w1);
                M = -INFINITY;
                l = 0.f;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        const bool stored = 16 * w + r16 < t.rows;
        if (stored && t.part >= 0) {
            const size_t pr = (size_t)(t.part + 16 * w + r16) * p.n_kv + h;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) *reinterpret_cast<f32x4 *>(p.part_o + pr * HD + 16 * dt + 4 * g) = orow[dt];
            if (g == 0) {
                p.part_m[pr] = Mr;
                p.part_l[pr] = lr;
            }
        } else if (stored) {
            T *out = reinterpret_cast<T *>(p.out) + (size_t)(t.r0 + token) * p.out_stride + head * HD;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                alignas(16) T x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = to_elem<P>(orow[dt][e] / lr);
                if constexpr (P == Prec::BF16)
                    *reinterpret_cast<u32x2 *>(out + 16 * dt + 4 * g) = *reinterpret_cast<const u32x2 *>(x);
                else
                    *reinterpret_cast<u32x4 *>(out + 16 * dt + 4 * g) = *reinterpret_cast<const u32x4 *>(x);
            }
            if (p.lse && g == 0)
                p.lse[(size_t)(t.r0 + token) * p.n_heads + head] = (Mr + log2f(lr)) * 0.6931471805599453f;
        }
    }
}

// Joins the spans of split row blocks, in position order. A workgroup takes some rows of one key
// head of an item, a lane four columns of a row.
template <Prec P, int HD>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnParams p) {
    using T = typename PrecT<P>::T;
    constexpr int LPR = HD / 4, RPW = 256 / LPR, NG = (kPagedBlockRows + RPW - 1) / RPW;
    if (bounded_rows(p.bk, p.rows, p.max_new, p.max_len) == 0) return;
    const int work = p.bk.status[PS_ITEMS] * p.n_kv * NG;
    const int col = threadIdx.x % LPR * 4;
    for (int idx = blockIdx.x; idx < work; idx += gridDim.x) {
        const int4 it = p.bk.items[idx / (p.n_kv * NG)];
        const int h = idx % p.n_kv, row = idx / p.n_kv % NG * RPW + threadIdx.x / LPR;
        const int4 e = p.bk.ent[it.x];
        const int rb = it.y * kPagedBlockRows, rows = min(kPagedBlockRows, e.z * p.group - rb);
        if (row >= rows) continue;
        float M = -INFINITY, l = 0.f;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < it.w; ++s) {
            const size_t pr = (size_t)(it.z + s * rows + row) * p.n_kv + h;
            const f32x4 os = *reinterpret_cast<const f32x4 *>(p.part_o + pr * HD + col);
            const float Ms = p.part_m[pr], ls = p.part_l[pr];
            float w0, w1;
            merge_weights(M, Ms, w0, w1);
            l = merge_value(l, ls, w0, w1);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = merge_value(o[i], os[i], w0, w1);
        }
        const int token = (rb + row) / p.group, head = h * p.group + (rb + row) % p.group;
        T *out = reinterpret_cast<T *>(p.out) + (size_t)(e.w + token) * p.out_stride + head * HD + col;
        alignas(16) T x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = to_elem<P>(o[i] / l);
        if constexpr (P == Prec::BF16)
            *reinterpret_cast<u32x2 *>(out) = *reinterpret_cast<const u32x2 *>(x);
        else
            *reinterpret_cast<u32x4 *>(out) = *reinterpret_cast<const u32x4 *>(x);
        if (p.lse && col == 0)
            p.lse[(size_t)(e.w + token) * p.n_heads + head] = (M + log2f(l)) * 0.6931471805599453f;
    }
}

namespace {

template <Prec P, int HD>
hipError_t launch_shape(int64_t units, bool split, const PagedAttnParams &p, hipStream_t s) {
    constexpr int lds = paged_rows_lds<P, HD>();
    const int per_cu = std::min(160 * 1024 / lds, 2);
    const dim3 grid((unsigned)std::min<int64_t>(units * p.n_kv, kCUs * per_cu));
    hipLaunchKernelGGL((paged_rows_kernel<P, HD>), grid, dim3(4 * kWave), lds, s, p);
    if (split) {
        const int64_t join = std::min<int64_t>(units, kPagedSplitBelow) * p.n_kv * 16;
        hipLaunchKernelGGL((paged_join_kernel<P, HD>), dim3((unsigned)std::min<int64_t>(join, 8 * kCUs)), dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn(bool bf16, int64_t units, bool split, const PagedAttnParams &p, hipStream_t s) {
    if (p.n_kv < 1 || p.group < 1 || p.n_heads != p.n_kv * p.group || units < 0) return hipErrorInvalidValue;
    if (units == 0 || p.rows == 0) return hipSuccess;
    if (bf16) {
        if (p.hd == 32) return launch_shape<Prec::BF16, 32>(units, split, p, s);
        if (p.hd == 64) return launch_shape<Prec::BF16, 64>(units, split, p, s);
        if (p.hd == 128) return launch_shape<Prec::BF16, 128>(units, split, p, s);
        if (p.hd == 256) return launch_shape<Prec::BF16, 256>(units, split, p, s);
    } else {
        if (p.hd == 16) return launch_shape<Prec::F32, 16>(units, split, p, s);
        if (p.hd == 32) return launch_shape<Prec::F32, 32>(units, split, p, s);
        if (p.hd == 64) return launch_shape<Prec::F32, 64>(units, split, p, s);
        if (p.hd == 128) return launch_shape<Prec::F32, 128>(units, split, p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace cllm

// Drafted tokens on the fifth-generation tensor cores (bf16).
//
// One CTA per SM works through its share of blocks (spd_drafted.cuh).  An item has up to two 128-row tiles over shared K/V blocks of 80 keys = five
// pages, each page a pair of TMA boxes per operand.  Per tile and block:
//     S = Q K^T     128 x 80 x D, fp32 in TMEM;   softmax: one row per thread, S into registers, options, mask, exponentials, P as bf16 pairs into
//     TMEM columns of its own, so that the next S is computed under the exponentials;   O += P V     128 x D x 80, P read from TMEM.
// An item with rows for one tile only is worked on by both: each takes every other block, and their (O, m, l) are joined at the end, O straight from
// TMEM (a row has the same lane in both tiles).  With one tile at work the chain of its softmax, not HBM, bounds the loop.
// 8 softmax warps, one warp per tile that issues its MMAs, one that loads K and one that loads V, one that plans the next item (and walks its tree)
// while this one runs, three that guard V.  Everything is handed over through mbarriers with bounded waits; a wait that runs out ends the CTA with
// SPD_ERR_TIMEOUT once all its threads have come to the common end.
//
// Masks: a row sees one or two intervals of the context (window, sinks) and a set of drafted tokens (bits per token).  A warp builds them,
// 16 bits per page, only in blocks that some of its rows do not see whole.  A hidden key's weight is 0, but 0 * NaN is NaN: the guards clear the
// slots of V that hold no token; where a token's V row is not finite, the sums of all rows are not either, and such rows are done again one by one,
// without a look at what they do not see.  So are rows whose sums left fp32's range by themselves (weights are relative to a reference
// that may lag 2^8 behind the maximum).
//
// Bound: HBM where tiles hold one user's few rows.  Where two tiles share long caches a block's softmax is a chain of 2200 cycles per 2 x 128 x 80 scores
// (3200 with a cap; tensor and exponential pipes are at half then), which explains three quarters of such a call; the rest has not been
// accounted for.  Over seconds the power limit.  Measured back to back in a first burst,
// head_dim 128, 32/8 heads: 64 users x 26-token trees over 1-9 k tokens 221 us (1.31 GB, 5.9 TB/s with the join; 250 over seconds), 64 users x one
// token through a window of 2048 behind 4 sinks 104 us (5.2 TB/s), 4 users x 64-token trees over 33-80 k tokens 296 us (980 TFLOP/s), 1.5-2.1 k new
// tokens of 2 users through a window of 1500 behind 16 sinks, cap 50, 168 us (530 TFLOP/s of visible pairs).
// Slower here: two CTAs of one tile per SM, blocks of 64 keys (229 -> 239, 299 -> 365 us); one tile per item without the other's help (465 us for the
// first case, with everything else simpler too); the next block's scores fetched under this one's weights (296 -> 311 us: registers); masks
// within the code for whole blocks (296 -> 303 us).
#pragma once

#include "spd_drafted.cuh"
#include "spd_prefill_scored_tc.cuh"

namespace spd {

constexpr int kDtThreads = 512;
constexpr int kDtConsumers = 15;                    // warps that read a plan
constexpr int kDtRows = 256;                        // rows of an item: two tiles
constexpr int kDtPages = kStKeys / kPage;           // page tiles per block
constexpr int kDtPageBox = kPage * 128;             // one swizzled box: 16 rows x 64 channels

struct DrPlan {
    int32_t valid;                                   // 0: the share is done
    int32_t u, first, i0, toks, h0, kvh;             // user; first token of q, of the tile; tokens; first head; KV head
    int32_t tiles;                                   // tiles with rows
    int32_t b0, b1, whole, slot;                     // blocks of the piece; whether it is the whole item; else where it goes
    int32_t deepest;                                 // greatest depth of the tree (0 for runs)
    int32_t bad;
    DraftedUser s;
    DraftedKeys k;
    int16_t parent[kDrTree], depth[kDrTree];         // of all the user's drafted tokens
    uint32_t line[kDrTree][kDrWords];                // of the item's tokens
};
__host__ __device__ constexpr int dt_kslots(int D) { return D == 128 ? 3 : 5; }
__host__ __device__ constexpr int dt_vslots(int D) { return D == 128 ? 4 : 6; }
constexpr int kDtGuards = 3;
constexpr int kDtBarBytes = 384;
struct DtExchange { float m[2][128], top[2][128], l[2][128]; uint32_t again[2][4]; };      // of both tiles' rows, where they share an item
constexpr size_t dt_smem_bytes(int D) {
    return 2 * static_cast<size_t>(st_qtile(D)) + (dt_kslots(D) + dt_vslots(D)) * static_cast<size_t>(st_tile(D)) + kDtBarBytes + sizeof(DtExchange) +
           2 * sizeof(DrPlan);
}
static_assert(dt_smem_bytes(128) + 1024 <= 232448, "shared memory of an SM");

struct DraftedTcParams {
    DraftedParams d;
    int32_t tpt;                // tokens per tile
    float c2;                   // sm_scale log2(e)
    float cap2, y1;             // cap log2(e); sm_scale / cap
    uint64_t p1[4], p2[6];      // coefficients for |y1 x| <= 1/2 and <= 1, each in both halves.  CAP 1: of cap2 tanh(y1 x) = x P(x^2); CAP 2: of
                                // tanh(y) = y P(y^2), p2 alone
    uint32_t wait_limit;
};

__device__ __forceinline__ uint32_t dt_low(int n) { return (1u << min(max(n, 0), 16)) - 1u; }       // bits 0 .. n - 1 of 16

// 16 consecutive fp32 columns of this thread's TMEM lane.
__device__ __forceinline__ void dt_ld16(uint32_t taddr, float (&o)[16]) {
    uint32_t r[16];
    tmem_ld16_nowait(taddr, r);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void dt_st16(uint32_t taddr, const float (&v)[16]) {
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    tmem_st8(taddr, r);
    tmem_st8(taddr + 8, r + 8);
}

// First position and tokens of page tile v of an item's list.
__device__ __forceinline__ int2 dt_tile(const DrPlan &pl, int v) {
    if (v >= pl.k.ns + pl.k.e - pl.k.a) return make_int2(0, 0);
    const int x = v < pl.k.ns ? v : pl.k.a + v - pl.k.ns;
    if (x < pl.s.np) return make_int2(x * kPage, min(kPage, pl.s.lp - x * kPage));
    const int y = (x - pl.s.np) * kPage;
    return make_int2(pl.s.lp + y, min(kPage, pl.s.lq - y));
}

// Where the list's tiles hold nothing but keys that rows with these bounds see whole (context in [lo, hi]): tiles [a0, a1) and [b0, b1).
struct DtWhole {
    int a0, a1, b0, b1;
    __device__ __forceinline__ bool holds(int v) const { return (v >= a0 && v + kDtPages <= a1) || (v >= b0 && v + kDtPages <= b1); }
};
__device__ __forceinline__ DtWhole dt_whole(const DrPlan &pl, int lo, int hi) {
    const int shift = pl.k.ns - pl.k.a, lp = pl.s.lp, np = pl.s.np;
    const int64_t end = static_cast<int64_t>(hi) + 1;
    auto up = [](int x) { return x / kPage + (x % kPage != 0 ? 1 : 0); };
    DtWhole w{0, 0, 0, 0};
    if (np > 0) {
        w.a0 = max(pl.k.ns, up(max(lo, 0)) + shift);
        w.a1 = static_cast<int>(min(static_cast<int64_t>(lp), end) / kPage) + shift;
    }
    if (pl.s.nt > np && end > lp) {
        w.b0 = max(pl.k.ns, np + up(max(lo, lp) - lp) + shift);
        w.b1 = np + static_cast<int>(min(static_cast<int64_t>(pl.s.lq), end - lp) / kPage) + shift;
    }
    const int list = pl.k.ns + pl.k.e - pl.k.a;          // a run's tile may end in front of the partition's
    w.a1 = min(w.a1, list);
    w.b1 = min(w.b1, list);
    if (np > 0 && lp % kPage == 0 && w.a1 == w.b0) { w.a1 = w.b1; w.b0 = w.a0; }        // one page follows upon the other
    return w;
}

// Which of the 16 keys of a page tile a row sees: token `it` of the item at position pos.
__device__ __forceinline__ uint32_t dt_sees(const DraftedParams &p, const DrPlan &pl, int2 tile, int it, int pos) {
    const bool tree = p.parents != nullptr;
    const int base = tile.x, cnt = tile.y;
    uint32_t m = dt_low(min(cnt, (tree ? pl.s.ctx : pos + 1) - base));
    if (p.window > 0) m &= ~dt_low(max(pos - p.window, -1) + 1 - base) | dt_low(p.sinks - base);
    if (tree && base + cnt > pl.s.ctx) {
        const int off = base - pl.s.ctx;
        const uint32_t *w = pl.line[it];
        uint32_t d;
        if (off < 0) d = w[0] << -off;
        else d = (off & 31) == 0 ? w[off >> 5] : __funnelshift_r(w[off >> 5], (off >> 5) + 1 < kDrWords ? w[(off >> 5) + 1] : 0u, off & 31);
        m |= d & dt_low(cnt);
    }
    return m;
}

__device__ __forceinline__ float4 dt_load4(const __nv_bfloat16 *p) {
    const uint2 w = *reinterpret_cast<const uint2 *>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w.y));
    return make_float4(a.x, a.y, b.x, b.y);
}

// One row of a piece the slow way, by a whole warp: 32 keys at a time, a score per lane, then four channels of O per lane.  Keys that the row
// does not see are not touched.
template <int D>
__device__ __noinline__ void dt_slow_row(const DraftedTcParams &q, const DrPlan &pl, int it, int hh, int lane) {
    const DraftedParams &p = q.d;
    const int pos = pl.s.ctx + (p.parents ? pl.depth[pl.i0 + it] : pl.i0 + it), h = pl.h0 + hh;
    const int64_t row = (static_cast<int64_t>(pl.first) + pl.i0 + it) * p.Hq + h;
    const __nv_bfloat16 *qr = static_cast<const __nv_bfloat16 *>(p.q) + row * D;
    const float slope = p.slopes ? p.slopes[h] : 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    const int v1 = min(pl.b1 * kDtPages, pl.k.ns + pl.k.e - pl.k.a);
    for (int v0 = pl.b0 * kDtPages; v0 < v1; v0 += 2) {
        const int v = v0 + (lane >> 4), slot = lane & 15;
        const int2 t = v < v1 ? dt_tile(pl, v) : make_int2(0, 0);
        const bool see = v < v1 && ((dt_sees(p, pl, t, it, pos) >> slot) & 1u);
        int64_t at = 0;
        int part = 0;
        float s = -INFINITY;
        if (see) {
            const DraftedTile d = drafted_tile(p, pl.s, pl.k, v);
            part = d.part;
            int page = p.part[part].indices[d.entry];
            if (page < 0 || page >= p.part[part].num_pages) page = 0;        // it was in range a moment ago
            at = ((static_cast<int64_t>(page) * p.Hkv + pl.kvh) * kPage + slot) * D;
            const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(p.k_pool[part]) + at;
            s = 0.f;
#pragma unroll 4
            for (int c = 0; c < D; c += 4) {
                const float4 a = dt_load4(qr + c), b = dt_load4(k + c);
                s = fmaf(a.x, b.x, s); s = fmaf(a.y, b.y, s); s = fmaf(a.z, b.z, s); s = fmaf(a.w, b.w, s);
            }
            s *= p.sm_scale;
            if (p.cap > 0.f) s = p.cap * tanhf(s / p.cap);
            const int far = p.parents && t.x + slot >= pl.s.ctx ? pos - pl.s.ctx - pl.depth[t.x + slot - pl.s.ctx] : pos - (t.x + slot);
            if (p.slopes) s = fmaf(-slope, static_cast<float>(far), s);
        }
        float mx = s;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn;
        const float alpha = m == -INFINITY ? 1.f : expf(m - ref), w = see ? expf(s - ref) : 0.f;
        float sum = w;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        l = l * alpha + sum;
        m = mn;
        o.x *= alpha; o.y *= alpha; o.z *= alpha; o.w *= alpha;
        const uint32_t seen = __ballot_sync(0xffffffffu, see);
        for (uint32_t left = seen; left != 0; left &= left - 1) {
            const int x = __ffs(left) - 1;
            const float wt = __shfl_sync(0xffffffffu, w, x);
            const int64_t a = __shfl_sync(0xffffffffu, at, x);
            const int pt = __shfl_sync(0xffffffffu, part, x);
            if (lane < D / 4) {
                const float4 b = dt_load4(static_cast<const __nv_bfloat16 *>(p.v_pool[pt]) + a + 4 * lane);
                o.x = fmaf(wt, b.x, o.x); o.y = fmaf(wt, b.y, o.y); o.z = fmaf(wt, b.z, o.z); o.w = fmaf(wt, b.w, o.w);
            }
        }
    }
    if (pl.whole) {
        if (lane < D / 4) drafted_put4<D>(p, row, lane, o, drafted_row(p, row, m, l, false));
    } else {
        float *dst = p.scratch + static_cast<size_t>(pl.slot) * drafted_slot_floats(D, kDtRows);
        const int r = it * p.hs + hh;
        if (lane < D / 4) reinterpret_cast<float4 *>(dst)[lane * kDtRows + r] = o;
        if (lane == 0) { dst[kDtRows * D + r] = m * kLog2e; dst[kDtRows * (D + 1) + r] = l; }
    }
}

// CAP: 0 none, 1 one that the polynomials' coefficients carry, 2 a cap for which those would leave fp32's normal range (tiny ones, and large ones: from 202 on at
// head_dim 128, 295 at 64, with a scale of 1 / sqrt(head_dim)).
template <int D, int CAP, bool BIAS>
__global__ void __launch_bounds__(kDtThreads, 1)
drafted_tc_kernel(const __grid_constant__ DraftedTcParams q, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk0,
                  const __grid_constant__ CUtensorMap mv0, const __grid_constant__ CUtensorMap mk1, const __grid_constant__ CUtensorMap mv1) {
    constexpr int QTILE = st_qtile(D), TILE = st_tile(D), NSK = dt_kslots(D), NSV = dt_vslots(D), BOXES = D / 64, KB = kStKeys;
    const DraftedParams &p = q.d;
    extern __shared__ __align__(1024) uint8_t base[];
    const uint32_t Qs = smem_u32(base), Ks = Qs + 2 * QTILE, Vs = Ks + NSK * TILE;
    uint8_t *behind = base + 2 * QTILE + (NSK + NSV) * TILE;
    uint64_t *bars = reinterpret_cast<uint64_t *>(behind);
    uint64_t *bar_q = bars, *bar_qfree = bars + 1;                 // Q loaded; Q read by both tiles
    uint64_t *bar_s = bars + 2, *bar_sf = bars + 4;                // per tile: S ready; S in registers
    uint64_t *bar_p = bars + 6, *bar_o = bars + 8;                 // per tile: P written; O has taken the block in (P is free)
    uint64_t *bar_plan = bars + 10, *bar_planfree = bars + 12;     // per plan buffer
    uint64_t *bar_x = bars + 14, *bar_y = bars + 15;               // a shared item's rows are exchanged; their O's are read
    uint64_t *bar_tree = bars + 16;                                // per plan buffer: the tree's part of the plan is there too
    uint64_t *bar_k = bars + 18, *bar_kfree = bar_k + NSK, *bar_v = bar_kfree + NSK, *bar_vfree = bar_v + NSV;
    uint64_t *bar_guard = bar_vfree + NSV;                         // per V slot: the guards are done with the block
    constexpr int NBARS = 18 + 2 * NSK + 3 * NSV;
    static_assert(NBARS * 8 + 8 <= kDtBarBytes, "barrier block");
    uint32_t &tmem_slot = *reinterpret_cast<uint32_t *>(bars + NBARS);
    int &first_bad = *reinterpret_cast<int *>(&tmem_slot + 1);
    DtExchange &ex = *reinterpret_cast<DtExchange *>(behind + kDtBarBytes);
    DrPlan *plans = reinterpret_cast<DrPlan *>(behind + kDtBarBytes + sizeof(DtExchange));
    const int tid = threadIdx.x, wid = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

    if (tid == 320) { prefetch_tensormap(&mq); prefetch_tensormap(&mk0); prefetch_tensormap(&mv0); prefetch_tensormap(&mk1); prefetch_tensormap(&mv1); }
    griddep_wait();
    griddep_launch_dependents();          // the join's CTAs take the places of those that are done here, and wait for the last
    // ---- the cut: sums over the users in what becomes the K ring, the share's first item by the planning warp
    int64_t *sums = reinterpret_cast<int64_t *>(base + 2 * QTILE);
    int Cu, chunks, ov;
    const int64_t W = drafted_sums<kDtThreads>(p, sums, &first_bad, Cu, chunks, ov);
    if (blockIdx.x == 0 && tid == 0) drafted_header(p, first_bad);
    if (tid < 4) p.records[4 * blockIdx.x + tid] = make_int4(0, 0, 0, 0);
    const int shares = drafted_shares(p, W, ov);
    if (static_cast<int>(blockIdx.x) >= shares) return;
    const int64_t x1 = drafted_bound(W, shares, blockIdx.x + 1);
    int64_t x = drafted_bound(W, shares, blockIdx.x);
    DraftedWalk w;
    if (wid == 12 && !drafted_locate(p, sums, Cu, chunks, ov, x, lane, w)) x = x1;
    if (tid == 320) {
        for (int b = 0; b < NBARS; ++b) {
            // Q and ring slots free: one per tile; S in registers, P written: one per softmax warp of the tile; rows exchanged, O's
            // read: one per softmax warp; V looked through: one per guard; plan read: one per warp
            const int k = b - 18, n = b == 1 || (k >= NSK && k < 2 * NSK) || (k >= 2 * NSK + NSV && k < 2 * NSK + 2 * NSV) ? 2 : b >= 4 && b < 8 ? 4
                                      : b == 14 || b == 15 ? 8 : k >= 2 * NSK + 2 * NSV ? kDtGuards : b >= 12 && b < 14 ? kDtConsumers : 1;
            mbar_init(smem_u32(&bars[b]), n);
        }
        fence_mbar_init();
    }
    if (wid == 8) {       // one warp allocates all of tensor memory for the CTA (it has the SM to itself)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kStTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_proxy_async();  // the sums were written where TMA and tensor core will work
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);

    bool ok = true;       // cleared by a wait that runs out; the warp then leaves its loops and comes to the common end
    auto wait = [&](uint64_t *bar, uint32_t parity) { if (ok) ok = __all_sync(0xffffffffu, st_mbar_wait(smem_u32(bar), parity & 1, q.wait_limit)); };
    auto plan_of = [&](int r) -> DrPlan & { wait(&bar_plan[r & 1], r >> 1); __syncwarp(); return plans[r & 1]; };
    auto plan_done = [&](int r) { __syncwarp(); if (lane == 0) mbar_arrive(smem_u32(&bar_planfree[r & 1])); };

    // the launch's 512 x 128 registers, shared out by warpgroup: 256 x 192 + 256 x 64 = 65536
    if (wid < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        // ---------------- softmax warps: one row per thread; n counts the tile's blocks
        const int t = wid >> 2, rr = tid & 127, in_tile = rr / p.hs, hh = rr - in_tile * p.hs;
        const int wt0 = (rr & ~31) / p.hs, wt1 = min(q.tpt - 1, (rr | 31) / p.hs);       // the warp's tokens within the tile
        const bool tree = p.parents != nullptr;
        const uint32_t lanes = static_cast<uint32_t>((wid & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + (t ? kStS1 : kStS0), t_p = tmem + lanes + (t ? kStP1 : kStP0);
        const uint32_t t_o = tmem + lanes + (t ? kStO1 : kStO0);
        int n = 0, nx = 0;                                    // blocks of the tile; items that both tiles shared
        for (int r = 0; ok; ++r) {
            DrPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            wait(&bar_tree[r & 1], r >> 1);
            __syncwarp();
            const bool shared = pl.tiles == 1;                // both tiles work for the first one's rows, every other block each
            const int nb = pl.b1 - pl.b0, nblk = shared ? (nb - t + 1) / 2 : nb, toks = pl.toks, ctx = pl.s.ctx, i0 = pl.i0;
            const int it = in_tile + (shared ? 0 : t * q.tpt), w0 = wt0 + (shared ? 0 : t * q.tpt), w1 = wt1 + (shared ? 0 : t * q.tpt);
            const bool mine = wt0 < q.tpt && w0 < toks, live = in_tile < q.tpt && it < toks;      // of the warp, of the thread
            const int tok = live ? it : 0;
            const int pos = ctx + (!tree ? i0 + tok : pl.s.good ? pl.depth[i0 + tok] : 0);      // no tree where the user is refused
            // what every row of the warp sees: whole tiles of context in [full_lo, full_hi]
            const int full_hi = tree ? ctx - 1 : ctx + i0 + w0;
            const int full_lo = p.window > 0 ? ctx + (tree ? pl.deepest : i0 + min(w1, toks - 1)) - p.window + 1 : 0;
            const int last_pos = tree ? 0x7fffffff : ctx + i0 + min(w1, toks - 1);
            const DtWhole dw = dt_whole(pl, full_lo, full_hi);
            const int vtop = (pl.b1 - 1 - (shared ? t : 0)) * kDtPages, vstep = (shared ? 2 : 1) * kDtPages;      // tiles of the first block; between blocks
            const int ns = pl.k.ns, prv = ns - pl.k.a, np = pl.s.np, pub = prv + np, lp = pl.s.lp, lpq = lp + pl.s.lq, list = prv + pl.k.e;
            const float slope2 = BIAS ? p.slopes[pl.h0 + hh] * kLog2e : 0.f;
            float l = 0.f, m = -INFINITY, top = -INFINITY;          // reference point and greatest score, log2 units
            // The reference is the greatest score so far, or less by up to kPfSlack, so that O is hardly ever rescaled.  o_ready: O has taken the
            // block before in.
            auto refer = [&](int i, float xmax, bool &o_ready) {
                top = fmaxf(top, xmax);
                if (__any_sync(0xffffffffu, xmax > m + kPfSlack)) {
                    const float m_new = (xmax > m + kPfSlack) ? xmax : m;
                    const float alpha = m == -INFINITY ? 1.f : ex2_approx(m - m_new);
                    l *= alpha;
                    m = m_new;
                    if (i > 0 && !__all_sync(0xffffffffu, alpha == 1.f)) {
                        wait(&bar_o[t], n + i - 1);
                        o_ready = true;
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            float ov[32];
                            tmem_ld32(t_o + c * 32, ov);
#pragma unroll
                            for (int y = 0; y < 32; ++y) ov[y] *= alpha;
                            tmem_st32(t_o + c * 32, ov);
                        }
                    }
                }
                return m == -INFINITY ? 0.f : m;
            };
            // Scores that the cap applies to, by the special-function unit, or by polynomials in x^2 that are multiplied by x.
            auto capped = [&](float s) { return q.cap2 - __fdividef(2.f * q.cap2, ex2_approx(s * (2.f * kLog2e) * q.y1) + 1.f); };
            auto poly1 = [&](uint64_t y) { return fma_f32x2(fma_f32x2(fma_f32x2(y, q.p1[3], q.p1[2]), y, q.p1[1]), y, q.p1[0]); };
            auto poly2 = [&](uint64_t y) {
                const uint64_t f = fma_f32x2(fma_f32x2(fma_f32x2(y, q.p2[5], q.p2[4]), y, q.p2[3]), y, q.p2[2]);
                return fma_f32x2(fma_f32x2(f, y, q.p2[1]), y, q.p2[0]);
            };
            // CAP 2.  Large caps lie far above most scores, and the special-function unit's error is 2^-22 of the cap: each score up to the cap goes by the
            // polynomial, cap2 tanh(y1 x) = c2 x P((y1 x)^2), whatever its neighbours are.  all: none is beyond the cap.
            auto far_capped = [&](uint64_t s2, bool all, float &x0, float &x1) {
                float s0, s1, u0, u1, c0, c1;
                const uint64_t y2 = mul_f32x2(s2, pack_f32x2(q.y1, q.y1));
                unpack_f32x2(mul_f32x2(poly2(mul_f32x2(y2, y2)), mul_f32x2(s2, pack_f32x2(q.c2, q.c2))), c0, c1);
                unpack_f32x2(s2, s0, s1);
                unpack_f32x2(y2, u0, u1);
                x0 = all || fabsf(u0) <= 1.f ? c0 : capped(s0);
                x1 = all || fabsf(u1) <= 1.f ? c1 : capped(s1);
            };
            // Weights are summed as they are rounded for the product with V: numerator and sum are off alike.
            uint64_t lsum2 = 0;
            auto weigh = [&](uint64_t arg2) {
                float x0, x1;
                unpack_f32x2(arg2, x0, x1);
                const uint32_t w = pack_bf16(ex2_approx(x0), ex2_approx(x1));
                lsum2 = add_f32x2(lsum2, pack_f32x2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)));
                return w;
            };
            for (int i = 0; i < nblk && ok; ++i) {
                const int v = vtop - i * vstep;
                bool o_ready = n + i == 0;
                lsum2 = 0;                                        // (+0, +0)
                wait(&bar_s[t], n + i);
                __syncwarp();
                tc_fence_after();
                if (!mine) {                                      // rows of nobody: what becomes of them does not matter
                    if (lane == 0) mbar_arrive(smem_u32(&bar_sf[t]));
                    if (n + i > 0) wait(&bar_o[t], n + i - 1);    // never a phase of P ahead of the others
                    if (lane == 0) mbar_arrive(smem_u32(&bar_p[t]));
                    continue;
                }
                if (dw.holds(v)) {
                    // ---- all of the block's keys are seen by all rows of the warp
                    uint32_t raw[KB];
                    tmem_ld64_nowait(t_s, raw);
                    tmem_ld16_nowait(t_s + 64, raw + 64);
                    tmem_wait_ld();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bar_sf[t]));   // the next block's S may be computed
                    float sv[KB];
#pragma unroll
                    for (int y = 0; y < KB; ++y) sv[y] = __uint_as_float(raw[y]);
                    auto pair = [&](int y) { return pack_f32x2(sv[y], sv[y + 1]); };
                    int form = 0;                                 // 1, 2: the polynomial that holds for the whole warp; 0: the special-function unit
                    if constexpr (CAP) {
                        float big[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int y = 0; y < KB; y += 2) big[(y >> 1) & 3] = fmax3_abs_nan(big[(y >> 1) & 3], sv[y], sv[y + 1]);
                        // rows of nobody hold another user's q, or what was there before: they have no vote
                        const float most = live ? fmax3_abs_nan(fmax3_abs_nan(big[0], big[1], big[2]), big[3], 0.f) * q.y1 : 0.f;
                        form = CAP == 1 && __all_sync(0xffffffffu, most <= 0.5f) ? 1 : __all_sync(0xffffffffu, most <= 1.f) ? 2 : 0;
                    }
                    if constexpr (CAP == 2) {
                        if (form != 0) {
#pragma unroll
                            for (int y = 0; y < KB; y += 2) far_capped(pair(y), true, sv[y], sv[y + 1]);
                        } else {
#pragma unroll
                            for (int y = 0; y < KB; y += 2) far_capped(pair(y), false, sv[y], sv[y + 1]);
                        }
                    }
                    if constexpr (CAP == 1 && BIAS) {             // the bias comes on top of capped scores
                        if (form != 0) {
#pragma unroll
                            for (int y = 0; y < KB; y += 2) { const uint64_t s2 = pair(y); unpack_f32x2(mul_f32x2(poly2(mul_f32x2(s2, s2)), s2), sv[y], sv[y + 1]); }
                        } else {
#pragma unroll
                            for (int y = 0; y < KB; ++y) sv[y] = capped(sv[y]);
                        }
                    }
                    if constexpr (BIAS) {                         // the block's positions follow upon one another
                        const float scale = CAP ? 1.f : q.c2, off = static_cast<float>((v >= pub ? lp + (v - pub) * kPage : (v - prv) * kPage) - pos);
#pragma unroll
                        for (int y = 0; y < KB; ++y) sv[y] = fmaf(slope2, off + static_cast<float>(y), sv[y] * scale);
                    }
                    float r4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int y = 0; y < KB; y += 2) r4[(y >> 1) & 3] = fmax3(r4[(y >> 1) & 3], sv[y], sv[y + 1]);
                    const float mx = fmaxf(fmaxf(r4[0], r4[1]), fmaxf(r4[2], r4[3]));
                    const float ref = refer(i, BIAS || CAP == 2 ? mx : CAP ? capped(mx) : mx * q.c2, o_ready);
                    const uint64_t mx2 = pack_f32x2(-ref, -ref), c22 = pack_f32x2(q.c2, q.c2);
                    uint32_t pk[KB / 2];
                    auto weights = [&](auto &&arg) {
#pragma unroll
                        for (int y = 0; y < KB / 2; ++y) pk[y] = weigh(arg(2 * y));
                    };
                    if constexpr (BIAS || CAP == 2) {
                        weights([&](int y) { return add_f32x2(pair(y), mx2); });
                    } else if constexpr (CAP) {
                        if (form == 1) weights([&](int y) { const uint64_t s2 = pair(y); return fma_f32x2(poly1(mul_f32x2(s2, s2)), s2, mx2); });
                        else if (form == 2) weights([&](int y) { const uint64_t s2 = pair(y); return fma_f32x2(poly2(mul_f32x2(s2, s2)), s2, mx2); });
                        else weights([&](int y) { return add_f32x2(pack_f32x2(capped(sv[y]), capped(sv[y + 1])), mx2); });
                    } else {
                        weights([&](int y) { return fma_f32x2(pair(y), c22, mx2); });
                    }
                    if (!o_ready) wait(&bar_o[t], n + i - 1);     // P of the block before has been read
                    tc_fence_after();
                    tmem_st32p(t_p, pk);
                    tmem_st8(t_p + 32, pk + 32);
                } else {
                    // ---- masks: page by page, twice, scores going back to TMEM in log2 units in between.  Few blocks of an item come here, and
                    // code that is run seldom costs by its length (every line of it comes from L2: 5000 cycles unrolled).
                    float mx = -INFINITY;
                    uint32_t hidden = 0u;                              // pages that no row of the warp sees anything of
#pragma unroll 1
                    for (int y = 0; y < kDtPages; ++y) {
                        const int vv = v + y, z = vv < ns ? vv : vv - prv, tb = z < np ? z * kPage : lp + (z - np) * kPage;
                        const int cnt = vv < list ? min(kPage, (z < np ? lp : lpq) - tb) : 0;
                        uint32_t sees = 0u;
                        if (cnt > 0 && tb <= last_pos) sees = dt_sees(p, pl, make_int2(tb, cnt), tok, pos);
                        if (!__any_sync(0xffffffffu, sees != 0u)) {
                            hidden |= 1u << y;
                            continue;
                        }
                        const bool all = __all_sync(0xffffffffu, sees == 0xffffu);
                        float s[kPage];
                        dt_ld16(t_s + y * kPage, s);
                        if constexpr (CAP) {
                            if (!all) {                                    // hidden scores may be anything
#pragma unroll
                                for (int x = 0; x < kPage; ++x) s[x] = (sees >> x) & 1u ? s[x] : 0.f;
                            }
                            float most = 0.f;
#pragma unroll
                            for (int x = 0; x < kPage; x += 2) most = fmax3_abs_nan(most, s[x], s[x + 1]);
                            const bool small = __all_sync(0xffffffffu, !live || most * q.y1 <= 1.f);
                            if constexpr (CAP == 2) {
#pragma unroll
                                for (int x = 0; x < kPage; x += 2) far_capped(pack_f32x2(s[x], s[x + 1]), small, s[x], s[x + 1]);
                            } else if (small) {
#pragma unroll
                                for (int x = 0; x < kPage; x += 2) {
                                    const uint64_t s2 = pack_f32x2(s[x], s[x + 1]);
                                    unpack_f32x2(mul_f32x2(poly2(mul_f32x2(s2, s2)), s2), s[x], s[x + 1]);
                                }
                            } else {
#pragma unroll
                                for (int x = 0; x < kPage; ++x) s[x] = capped(s[x]);
                            }
                        } else {
#pragma unroll
                            for (int x = 0; x < kPage; ++x) s[x] *= q.c2;
                        }
                        if constexpr (BIAS) {
#pragma unroll
                            for (int x = 0; x < kPage; ++x) {
                                const int d = tb + x - ctx;                // drafted tokens of a tree count by depth
                                const int far = tree && d >= 0 ? ctx - pos + pl.depth[min(d, kDrTree - 1)] : tb + x - pos;
                                s[x] = fmaf(slope2, static_cast<float>(far), s[x]);
                            }
                        }
                        if (!all) {
#pragma unroll
                            for (int x = 0; x < kPage; ++x) s[x] = (sees >> x) & 1u ? s[x] : -INFINITY;
                        }
#pragma unroll
                        for (int x = 0; x < kPage; x += 2) mx = fmax3(mx, s[x], s[x + 1]);
                        dt_st16(t_s + y * kPage, s);
                    }
                    tmem_wait_st();
                    const float ref = refer(i, mx, o_ready);
                    if (!o_ready) wait(&bar_o[t], n + i - 1);
                    tc_fence_after();
#pragma unroll 1
                    for (int y = 0; y < kDtPages; ++y) {
                        uint32_t pk[kPage / 2];
                        if ((hidden >> y) & 1u) {
#pragma unroll
                            for (int x = 0; x < kPage / 2; ++x) pk[x] = 0u;
                            tmem_st8(t_p + y * (kPage / 2), pk);
                            continue;
                        }
                        float s[kPage];
                        dt_ld16(t_s + y * kPage, s);
#pragma unroll
                        for (int x = 0; x < kPage; x += 2) pk[x / 2] = weigh(pack_f32x2(s[x] - ref, s[x + 1] - ref));
                        tmem_st8(t_p + y * (kPage / 2), pk);
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bar_sf[t]));
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();                                     // one arrival per warp
                if (lane == 0) mbar_arrive(smem_u32(&bar_p[t]));
                float s0, s1;
                unpack_f32x2(lsum2, s0, s1);
                l += s0 + s1;
            }
            n += nblk;
            if (nblk > 0) wait(&bar_o[t], n - 1);
            __syncwarp();
            tc_fence_after();
            // ---- the rows' way out
            const int64_t row = (static_cast<int64_t>(pl.first) + i0 + tok) * p.Hq + pl.h0 + hh;
            float *dst = p.scratch + static_cast<size_t>(pl.slot) * drafted_slot_floats(D, kDtRows);
            const int slot_row = it * p.hs + hh;
            float a0 = 1.f, a1 = 0.f;                        // weights of the tiles' O
            if (shared) {
                ex.m[t][rr] = m; ex.top[t][rr] = top; ex.l[t][rr] = l;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(bar_x));
                wait(bar_x, nx);
                __syncwarp();
                tc_fence_after();
                const float m0 = ex.m[0][rr], m1 = ex.m[1][rr];
                top = fmaxf(ex.top[0][rr], ex.top[1][rr]);
                a0 = m0 == -INFINITY ? 0.f : ex2_approx(m0 - top);
                a1 = m1 == -INFINITY ? 0.f : ex2_approx(m1 - top);
                l = ex.l[0][rr] * (a0 == 0.f && ex.l[0][rr] == 0.f ? 0.f : a0) + ex.l[1][rr] * a1;
            } else if (m != -INFINITY) {
                a0 = ex2_approx(m - top);                    // from the reference to the maximum
                l *= a0;
            }
            // read only now: a tile without blocks of its own has waited for nobody before the exchange
            const bool bad = *const_cast<volatile int32_t *>(&pl.bad) != 0;
            const bool whole_item = pl.whole != 0;
            DraftedRow f{};
            if (ok && live && whole_item) f = drafted_row(p, row, top * 0.69314718055994531f, l, bad);
            float big = 0.f;
            // 16 channels at a time, in a loop (see the masks); a shared row's go half by either tile's thread, from both tiles' O
            const int c_end = shared ? (t + 1) * (D / 2) : D;
#pragma unroll 1
            for (int c = shared ? t * (D / 2) : 0; c < c_end; c += 16) {
                float ov[16];
                dt_ld16((shared ? tmem + lanes + kStO0 : t_o) + c, ov);
#pragma unroll
                for (int y = 0; y < 16; ++y) ov[y] = a0 == 0.f ? 0.f : ov[y] * a0;
                if (shared) {
                    float o1[16];
                    dt_ld16(tmem + lanes + kStO1 + c, o1);
#pragma unroll
                    for (int y = 0; y < 16; ++y) ov[y] = a1 == 0.f ? ov[y] : fmaf(o1[y], a1, ov[y]);
                }
#pragma unroll
                for (int y = 0; y < 16; y += 2) big = fmax3_abs_nan(big, ov[y], ov[y + 1]);
                if (ok && live) {
                    if (whole_item) {
                        drafted_put16<D>(p, row, c, ov, f);
                    } else {
#pragma unroll
                        for (int y = 0; y < 16; y += 4)
                            reinterpret_cast<float4 *>(dst)[(c + y) / 4 * kDtRows + slot_row] = make_float4(ov[y], ov[y + 1], ov[y + 2], ov[y + 3]);
                    }
                }
                __syncwarp();
            }
            if (ok && live && !whole_item && (!shared || t == 0)) { dst[kDtRows * D + slot_row] = top; dst[kDtRows * (D + 1) + slot_row] = bad ? kDrBad : l; }
            const bool over = ok && live && !bad && l > 0.f && l < INFINITY && !(big < INFINITY);
            uint32_t again = __ballot_sync(0xffffffffu, over);
            if (shared) {
                // the other tile may not write its next O before this one's is read; rows that are done again wait for both halves
                if (lane == 0) ex.again[t][wid & 3] = again;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(bar_y));
                wait(bar_y, nx);
                __syncwarp();
                tc_fence_after();
                ++nx;
                again = ok ? (ex.again[0][wid & 3] | ex.again[1][wid & 3]) & (t ? 0xaaaaaaaau : 0x55555555u) : 0u;
            }
            for (; again != 0; again &= again - 1) {
                const int src = __ffs(again) - 1;
                dt_slow_row<D>(q, pl, __shfl_sync(0xffffffffu, it, src), __shfl_sync(0xffffffffu, hh, src), lane);
            }
            if (ok && bad && lane == 0 && wid == 0) drafted_flag(p, pl.u);
            tc_fence_before();                               // O is read: ordered before this warp's next arrival
            plan_done(r);
        }
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (wid == 12) {
        // ---------------- the planning warp
        for (int r = 0;; ++r) {
            DrPlan &pl = plans[r & 1];
            if (r >= 2) wait(&bar_planfree[r & 1], (r >> 1) - 1);
            __syncwarp();
            int b0 = 0, b1 = 0;
            if (ok && x < x1 && (r == 0 || drafted_next(p, w))) drafted_blocks(w, x, x1, b0, b1);
            if (b0 == b1) {                             // the share is done, or ends inside the item's own cost
                if (lane == 0) { pl.valid = 0; mbar_arrive(smem_u32(&bar_plan[r & 1])); }
                break;
            }
            const int i0 = w.rt * p.tt, toks = min(p.tt, w.s.n - i0), kvh = w.sq / p.hgroups;
            const bool whole = b0 == 0 && b1 == w.k.nb;
            const int slot = 2 * blockIdx.x + (b0 == 0 ? 1 : 0);
            if (lane == 0) {
                pl.valid = 1; pl.u = w.u; pl.first = w.s.first; pl.i0 = i0; pl.toks = toks; pl.kvh = kvh;
                pl.h0 = kvh * p.g + w.sq % p.hgroups * p.hs;
                pl.tiles = toks > q.tpt ? 2 : 1;
                pl.b0 = b0; pl.b1 = b1; pl.whole = whole; pl.slot = slot; pl.deepest = 0;
                pl.bad = !w.s.good;
                pl.s = w.s; pl.k = w.k;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_plan[r & 1]));      // loads and products may begin; the masks need the tree
            if (p.parents != nullptr && w.s.good) {
                bool wrong = false;
                int deepest = 0;
                for (int i = lane; i < w.s.n; i += 32) {
                    const int up = p.parents[w.s.first + i];
                    const bool off = up < -1 || up >= i;
                    wrong = wrong || off;
                    pl.parent[i] = static_cast<int16_t>(off ? -1 : up);
                }
                __syncwarp();
                for (int i = lane; i < w.s.n; i += 32) {
                    const int d = drafted_depth(pl.parent, i);
                    pl.depth[i] = static_cast<int16_t>(d);
                    deepest = max(deepest, d);
                    if (i >= i0 && i < i0 + toks) drafted_line(p, w.s, pl.parent, i, d, pl.line[i - i0]);
                }
                deepest = __reduce_max_sync(0xffffffffu, deepest);
                if (lane == 0) pl.deepest = deepest;
                if (wrong) pl.bad = 1;
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&bar_tree[r & 1]));
                if (!whole) drafted_record(p, w, slot, W, shares);
            }
            x = w.x0 + w.ov + w.k.nb;
        }
    } else if (wid == 10 || wid == 11) {
        // ---------------- the loading warps: K (and Q), V; c counts blocks over all items
        const bool is_k = wid == 10;
        const int ring = is_k ? NSK : NSV;
        const uint32_t slots = is_k ? Ks : Vs;
        uint64_t *bar_full = is_k ? bar_k : bar_v, *bar_free = is_k ? bar_kfree : bar_vfree;
        const CUtensorMap *m0 = is_k ? &mk0 : &mv0, *m1 = is_k ? &mk1 : &mv1;
        const uint64_t once = l2_evict_first_policy();
        uint64_t often;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(often));
        int c = 0, nq = 0;
        for (int r = 0; ok; ++r) {
            DrPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            if (is_k) {
                if (nq > 0) wait(bar_qfree, nq - 1);
                if (ok && lane == 0) {
                    const int rows = p.hs * q.tpt;
                    mbar_expect_tx(smem_u32(bar_q), pl.tiles * BOXES * rows * 128);
                    for (int t = 0; t < pl.tiles; ++t)
                        for (int y = 0; y < BOXES; ++y)
                            tma_load_3d(Qs + t * QTILE + y * kStQBox, &mq, 64 * y, pl.h0, pl.first + pl.i0 + t * q.tpt, smem_u32(bar_q));
                }
                if (ok) ++nq;
            }
            const uint64_t policy = pl.s.n > p.tt ? often : once;      // other items read these keys too
            const int b0 = pl.b0, list = pl.k.ns + pl.k.e - pl.k.a, v1 = min(pl.b1 * kDtPages, list), kvh = pl.kvh;
            int at = -1, part = 0, have = v1;                   // lane k holds where tile have + k starts; tiles are worked through downwards
            for (int b = pl.b1 - 1; b >= b0 && ok; --b, ++c) {
                const int v0 = b * kDtPages, slot = c % ring, use = c / ring;
                if (v0 < have) {                                // 30 tiles at a time: six blocks
                    have = max(b0 * kDtPages, v0 - 5 * kDtPages);
                    at = -1;
                    if (lane < 6 * kDtPages && have + lane < v1) {
                        const DraftedTile d = drafted_tile(p, pl.s, pl.k, have + lane);
                        part = d.part;
                        const int page = p.part[part].indices[d.entry];
                        if (page < 0 || page >= p.part[part].num_pages) pl.bad = 1;
                        else at = (page * p.Hkv + kvh) * kPage;
                    }
                }
                // lanes 0 .. 9 load: tile lane / 2, box lane % 2
                const int y = lane / BOXES, from = min(31, v0 - have + min(y, kDtPages - 1));
                const int my_at = __shfl_sync(0xffffffffu, at, from), my_part = __shfl_sync(0xffffffffu, part, from);
                const bool loads = lane < kDtPages * BOXES && v0 + y < v1 && my_at >= 0;
                const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, loads)) * kDtPageBox;
                if (use > 0) wait(&bar_free[slot], use - 1);
                if (!ok) break;
                __syncwarp();
                if (lane == 0) mbar_expect_tx(smem_u32(&bar_full[slot]), bytes);
                __syncwarp();
                if (loads)
                    tma_load_2d(slots + slot * TILE + lane % BOXES * kStBox + y * kDtPageBox, my_part ? m1 : m0, lane % BOXES * 64, my_at,
                                smem_u32(&bar_full[slot]), policy);
            }
            plan_done(r);
        }
        if (!ok && lane == 0) {              // leave nothing in flight behind: a bounded chance for what was asked for last
            if (nq > 0) mbar_wait(smem_u32(bar_q), (nq - 1) & 1);
            for (int y = 0; y < ring; ++y) {
                const int uses = (c - y + ring) / ring;         // blocks that went to slot y, the one that was cut off included
                if (c >= y && uses > 0) mbar_wait(smem_u32(&bar_full[y]), (uses - 1) & 1);
            }
        }
    } else if (wid >= 13) {
        // ---------------- the guards: slots of V that hold no token, in the last pages of a partition and behind the list's end
        int c = 0;
        for (int r = 0; ok; ++r) {
            const DrPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            const int b0 = pl.b0;
            const DtWhole dw = dt_whole(pl, 0, 0x7ffffffe);     // full pages
            for (int b = pl.b1 - 1; b >= b0 && ok; --b, ++c) {
                // every block passes through here, so that no guard is ever a whole ring ahead of or behind the others
                const int slot = c % NSV, v = b * kDtPages;
                wait(&bar_v[slot], c / NSV);
                __syncwarp();
                if (!dw.holds(v)) {
                    uint8_t *vt = base + 2 * QTILE + (NSK + slot) * TILE;
#pragma unroll 1
                    for (int y = 0; y < kDtPages; ++y) {
                        const int n = dt_tile(pl, v + y).y, chunks = (kPage - n) * 8;      // 16-byte chunks of each box from row n on
#pragma unroll 1
                        for (int e = (wid - 13) * 32 + lane; e < chunks * BOXES; e += 32 * kDtGuards) {
                            const int box = BOXES > 1 && e >= chunks ? 1 : 0;
                            *reinterpret_cast<uint4 *>(vt + box * kStBox + (y * kPage + n) * 128 + (e - box * chunks) * 16) = make_uint4(0, 0, 0, 0);
                        }
                    }
                    fence_proxy_async();
                    __syncwarp();
                }
                if (lane == 0) mbar_arrive(smem_u32(&bar_guard[slot]));
            }
            plan_done(r);
        }
    } else if (wid < 10) {
        // ---------------- the warp that issues tile t's MMAs: S of block j, then P V of block j - 1; n counts the tile's blocks
        const int t = wid - 8;
        const uint32_t ts = tmem + (t ? kStS1 : kStS0), tp = tmem + (t ? kStP1 : kStP0), to = tmem + (t ? kStO1 : kStO0);
        int c = 0, n = 0, nq = 0;
        for (int r = 0; ok; ++r) {
            const DrPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            const int NB = pl.b1 - pl.b0;
            const bool shared = pl.tiles == 1;
            const int lag = shared ? 2 : 1;                      // the tile's next S goes before its P V
            const uint32_t qa = Qs + (shared ? 0 : t * QTILE);
            wait(bar_q, nq++);
            for (int j = 0; j < NB + lag && ok; ++j) {
                if (j < NB) {
                    const int slot = (c + j) % NSK;
                    // a tile that has no use for a block gives it back all the same, once it is there: never a ring ahead
                    wait(&bar_k[slot], (c + j) / NSK);
                    if (!shared || (j & 1) == t) {
                        const int k = n + (shared ? j >> 1 : j);
                        if (k > 0) wait(&bar_sf[t], k - 1);
                        __syncwarp();
                        tc_fence_after();
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk)       // 16 channels per MMA
                            st_mma_ss(ts, umma_desc(qa + (kk >> 2) * kStQBox + (kk & 3) * 32, 16, 1024),
                                      umma_desc(Ks + slot * TILE + (kk >> 2) * kStBox + (kk & 3) * 32, 16, 1024), umma_idesc(false, KB), kk > 0 ? 1u : 0u);
                        st_commit(smem_u32(&bar_s[t]));
                        st_commit(smem_u32(&bar_kfree[slot]));
                    } else if (lane == 0) {
                        mbar_arrive(smem_u32(&bar_kfree[slot]));
                    }
                    if (j == NB - 1) st_commit(smem_u32(bar_qfree));      // behind the item's last use of Q (at once where nothing is under way)
                }
                if (j >= lag) {
                    const int jj = j - lag, slot = (c + jj) % NSV;
                    wait(&bar_v[slot], (c + jj) / NSV);
                    wait(&bar_guard[slot], (c + jj) / NSV);
                    if (!shared || (jj & 1) == t) {
                        wait(&bar_p[t], n + (shared ? jj >> 1 : jj));     // also: this tile's softmax has read the O of the item before
                        __syncwarp();
                        tc_fence_after();
#pragma unroll
                        for (int kk = 0; kk < KB / 16; ++kk)      // 16 keys per MMA: 8 columns of P, 2 KB of each 64-channel box of V
                            st_mma_ts(to, tp + kk * 8, umma_desc(Vs + slot * TILE + kk * 2048, kStBox, 1024), umma_idesc(true, D), (jj >= lag || kk > 0) ? 1u : 0u);
                        st_commit(smem_u32(&bar_o[t]));
                        st_commit(smem_u32(&bar_vfree[slot]));
                    } else if (lane == 0) {
                        mbar_arrive(smem_u32(&bar_vfree[slot]));
                    }
                }
            }
            c += NB;
            n += shared ? (NB - t + 1) / 2 : NB;
            plan_done(r);
        }
    }
    }
    tc_fence_before();
    const bool gave_up = !__syncthreads_and(ok);
    tc_fence_after();
    if (gave_up && tid == 0) flag_error(p.hdr, 6 /* SPD_ERR_TIMEOUT */, -1);
    if (wid == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kStTmemCols) : "memory");
}

}  // namespace spd

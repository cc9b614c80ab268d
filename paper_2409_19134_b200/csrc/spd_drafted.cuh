// Attention of drafted tokens over the two paged partitions: what the kernels share.
//
// A user's drafted tokens are the last n tokens of its public partition; they hang together as a tree (parents) or a run.  Token i at
// depth d_i has position ctx + d_i, ctx = cached tokens in front of the drafted ones, and sees
//     the context and, among the drafted tokens, itself and its ancestors, each where pos_i - pos_j < window or pos_j < sinks;
//     s = sm_scale q.k;  s <- cap tanh(s / cap);  s <- s - slope_h (pos_i - pos_j).
// Rows that read the same keys are computed together: an item is (user, tile of tokens x heads of one group, KV head), its keys the page
// tiles that some row of it may see (those that hold sinks, then from the widest window on), a block of `bt` page tiles at a time.  All items' blocks
// laid end to end are cut into equal shares, one per CTA, whatever the batch looks like: an item inside a share is finished there, one that
// is cut leaves (O, m, l) per piece in scratch, and a second kernel joins the pieces (Theorem 1) in order, so that results do not
// depend on who came first.  No CTA waits for another.
#pragma once

#include "spd_kernels.cuh"

namespace spd {

constexpr int kDrTree = 256;              // most drafted tokens of a user that come as a tree
constexpr int kDrWords = kDrTree / 32;
constexpr float kDrBad = -1.f;            // in place of a piece's sum of weights
constexpr int kDrMinBlocks = 1;           // do not cut the work into shares of less than that, and an item's own cost

struct DraftedParams {
    int32_t B, Hq, Hkv, g;
    int32_t hs, hgroups;                  // query heads that a tile takes of a token, and how many such groups a KV head has
    int32_t tt;                           // tokens per tile
    int32_t SQ;                           // Hkv * hgroups
    int32_t bt;                           // page tiles per block
    int32_t ov;                           // what an item costs beside its blocks, in blocks
    int64_t T;
    float sm_scale;
    const void *q;                        // [T][Hq][D]
    PartDev part[2];                      // 0 = private, 1 = public
    const void *k_pool[2], *v_pool[2];
    const int32_t *peer_lens[2];          // lengths of a partition that the call does not read
    const int32_t *tok_indptr;            // [B+1]; null = one token per user
    const int32_t *parents;               // [T]; null = runs
    float cap;
    int32_t window, sinks;
    const float *slopes;
    int32_t mode;                         // OutMode
    float *po, *pm, *pl;                  // OUT_PARTIAL: [T][Hq][D], [T][Hq], [T][Hq]
    const float *in_o, *in_m, *in_l;      // OUT_FINAL: optional partial to merge in
    void *out;                            // OUT_FINAL: [T][Hq][D]
    int32_t out_bf16, wide;               // wide: the output is aligned to 32 bytes
    int32_t *hdr;
    int32_t seqs;                         // what HDR_NSEQ is to hold
    int32_t grid;                         // CTAs of the launch
    int4 *records;                        // [2 * grid][2]: what the join has to know of the pieces in a CTA's two slots
    float *scratch;                       // [2 * grid] slots
};

// A slot holds one piece: O as [D / 4][RT] float4 (threads of consecutive rows write consecutive chunks), then m [RT] and l [RT].  A sum of
// kDrBad says that the piece met something out of order: an item that is cut becomes what a whole one does, zeros, and the join needs no other word.
__host__ __device__ constexpr size_t drafted_slot_floats(int D, int RT) { return static_cast<size_t>(RT) * (D + 2); }

struct DraftedUser {
    int first, n;                          // rows of q
    int lp, lq, ctx;                       // private and public tokens; those in front of the drafted ones
    int np, nt;                            // page tiles: private ones, all that the call reads
    int64_t base0, base1;                  // first page-table entries
    bool good;
};

// A user whose tables, lengths or counts are inconsistent is not good: it has no keys, and its rows become zeros.  False where its offsets
// are inconsistent.  All loads are asked for before anything is decided.
__device__ __forceinline__ bool drafted_user(const DraftedParams &p, int u, DraftedUser &s) {
    const PartDev &A = p.part[0], &B = p.part[1];
    const bool pa = A.present != 0, pb = B.present != 0, offsets = p.tok_indptr != nullptr;
    const int64_t t0 = offsets ? p.tok_indptr[u] : u, t1 = offsets ? p.tok_indptr[u + 1] : u + 1;
    const int64_t alo = pa ? A.indptr[u] : 0, ahi = pa ? A.indptr[u + 1] : 0, aend = pa ? A.indptr[p.B] : 0;
    const int64_t blo = pb ? B.indptr[u] : 0, bhi = pb ? B.indptr[u + 1] : 0, bend = pb ? B.indptr[p.B] : 0;
    const int32_t *la = pa ? A.lens : p.peer_lens[0], *lb = pb ? B.lens : p.peer_lens[1];
    const int64_t alen = la ? la[u] : 0, blen = lb ? lb[u] : 0;
    s.first = static_cast<int>(t0);
    s.n = static_cast<int>(t1 - t0);
    const bool consistent = t0 >= 0 && t1 >= t0 && t1 <= p.T && (u != 0 || t0 == 0) && (u != p.B - 1 || t1 == p.T);
    bool good = alen >= 0 && blen >= s.n && alen + blen <= 0x7fffffff && (p.parents == nullptr || s.n <= kDrTree);
    good = good && alo >= 0 && ahi >= alo && ahi <= aend && (!pa || alen <= (ahi - alo) * kPage) && (alen == 0 || !pa || A.indices != nullptr);
    good = good && blo >= 0 && bhi >= blo && bhi <= bend && (!pb || blen <= (bhi - blo) * kPage) && (blen == 0 || !pb || B.indices != nullptr);
    s.good = good;
    s.lp = good ? static_cast<int>(alen) : 0;
    s.lq = good ? static_cast<int>(blen) : s.n;
    s.ctx = s.lp + s.lq - s.n;
    s.base0 = alo; s.base1 = blo;
    s.np = pa && good ? (s.lp + kPage - 1) / kPage : 0;
    s.nt = s.np + (pb && good ? (s.lq + kPage - 1) / kPage : 0);
    return consistent;
}

// Keys of a tile of rows: page tiles [0, ns) and [a, e) of the user's, ceil((ns + e - a) / bt) blocks (at least one, so that rows that
// see nothing are written too).
struct DraftedKeys { int ns, a, e, nb; };
__device__ __forceinline__ DraftedKeys drafted_keys(const DraftedParams &p, const DraftedUser &s, int i0, int i1) {
    const int64_t P0 = p.part[0].present ? 0 : s.lp, P1 = s.nt == 0 ? P0 : (p.part[1].present ? static_cast<int64_t>(s.lp) + s.lq : s.lp);
    const int64_t hi = p.parents ? P1 : min(P1, static_cast<int64_t>(s.ctx) + i1);
    int64_t lo = P0;
    if (p.window > 0) lo = max(lo, static_cast<int64_t>(s.ctx) + (p.parents ? 0 : i0) - p.window + 1);
    // tiles in front of position x, with the one that x lies in
    auto upto = [&](int64_t x) { return static_cast<int>(x < s.lp ? x / kPage : s.np + (x - s.lp) / kPage) + 1; };
    DraftedKeys k;
    k.a = lo < hi ? upto(lo) - 1 : s.nt;
    k.e = lo < hi ? upto(hi - 1) : s.nt;
    const int64_t se = min(static_cast<int64_t>(p.sinks), hi);
    k.ns = p.window > 0 && se > P0 && lo > P0 ? upto(se - 1) : 0;
    if (k.ns >= k.a) { k.a = 0; k.ns = 0; }
    k.nb = max(1, (k.ns + k.e - k.a + p.bt - 1) / p.bt);
    return k;
}

// Tile x of a user's list: first position, tokens, and where its page stands.
struct DraftedTile { int base, cnt, part; int64_t entry; };
__device__ __forceinline__ DraftedTile drafted_tile(const DraftedParams &p, const DraftedUser &s, const DraftedKeys &k, int v) {
    DraftedTile t{0, 0, 0, 0};
    if (v >= k.ns + k.e - k.a) return t;
    const int x = v < k.ns ? v : k.a + v - k.ns;
    if (x < s.np) {
        t.base = x * kPage; t.cnt = min(kPage, s.lp - t.base); t.entry = s.base0 + x;
    } else {
        const int y = x - s.np;
        t.base = s.lp + y * kPage; t.cnt = min(kPage, s.lq - y * kPage); t.part = 1; t.entry = s.base1 + y;
    }
    return t;
}

// ---------------------------------------------------------------------------------------------------------------------
// The cut.  Units (an item's own cost, then its blocks) in the order user, row tile, (KV head, head group); W of them in `shares` shares.
// A share that ends inside an item's own cost has none of its blocks.
struct DraftedWalk {
    int ov;                    // units of an item's own cost
    int u, rt, sq;             // the item
    DraftedUser s;
    DraftedKeys k;
    int64_t x0;                // its first unit among all
};

// Quotient of numbers that are not negative, in 32 bits where they fit (a division in 64 bits is some 100 instructions, one behind the other).
__device__ __forceinline__ int64_t drafted_div(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}
__device__ __forceinline__ int64_t drafted_bound(int64_t W, int shares, int c) { return drafted_div(W * c, shares); }
__device__ __forceinline__ int drafted_share_of(int64_t W, int shares, int64_t x) { return static_cast<int>(drafted_div((x + 1) * shares - 1, W)); }

__device__ __forceinline__ void drafted_item_keys(const DraftedParams &p, DraftedWalk &w) {
    w.k = drafted_keys(p, w.s, w.rt * p.tt, min(w.s.n, (w.rt + 1) * p.tt));
}

// Blocks of one KV head and head group over tiles from rt0 on, every `step`-th.
__device__ __forceinline__ int64_t drafted_user_blocks(const DraftedParams &p, const DraftedUser &s, int rt0, int step) {
    int64_t sum = 0;
    for (int rt = rt0; rt * p.tt < s.n; rt += step) sum += drafted_keys(p, s, rt * p.tt, min(s.n, (rt + 1) * p.tt)).nb;
    return sum;
}

// Shares of many blocks go by what items cost beside their blocks too; where there are few, finishing together matters less than starting early.
// us on one GPU, ov 2 / 6: 64 users x 26-token trees over 1-9 k tokens 239 / 233, a part of a prompt 184 / 179; 8 users x 5-16 tokens
// over 300-800 tokens in two halves 40 / 45.
constexpr int kDrManyBlocks = 16;

// The sums of the users' units, by all NT threads of a CTA: chunk c of C users (a user per warp where there are few of them, so that the
// lanes share a long run's tiles) ends at sums[c].  *first_bad: the first user whose offsets are inconsistent; it and all behind it have no rows.
template <int NT>
__device__ __forceinline__ int64_t drafted_sums(const DraftedParams &p, int64_t *sums, int *first_bad, int &C, int &chunks, int &ov) {
    __shared__ int64_t warp_blocks[NT / 32];
    __shared__ int warp_tiles[NT / 32];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const bool warps = p.B <= NT / 32;
    C = warps ? 1 : (p.B + NT - 1) / NT;
    chunks = (p.B + C - 1) / C;
    if (tid == 0) *first_bad = p.B;
    __syncthreads();
    // a user's blocks count unless its offsets, or those of somebody in front of it, turn out to be inconsistent
    int64_t blocks = 0;
    int tiles = 0;
    DraftedUser s;
    const int u0 = warps ? wid : tid * C, u1 = min(p.B, warps ? u0 + 1 : u0 + C);
    int bad = 0x7fffffff;
    for (int u = u0; u < u1 && bad == 0x7fffffff; ++u) {
        if (!drafted_user(p, u, s)) { bad = u; break; }
        blocks += warps ? drafted_user_blocks(p, s, lane, 32) : drafted_user_blocks(p, s, 0, 1);
        if (!warps || lane == 0) tiles += s.n / p.tt + (s.n % p.tt != 0 ? 1 : 0);
    }
    if (bad != 0x7fffffff) atomicMin(first_bad, bad);
    __syncthreads();
    if (u0 > *first_bad) { blocks = 0; tiles = 0; }
    // inclusive sums over the warp's threads, then over the warps
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t ub = __shfl_up_sync(0xffffffffu, blocks, d);
        const int ut = __shfl_up_sync(0xffffffffu, tiles, d);
        if (lane >= d) { blocks += ub; tiles += ut; }
    }
    if (lane == 31) { warp_blocks[wid] = blocks; warp_tiles[wid] = tiles; }
    __syncthreads();
    int64_t before = 0, all = 0;
    int tiles_before = 0, tiles_all = 0;
    for (int w = 0; w < NT / 32; ++w) {
        if (w < wid) { before += warp_blocks[w]; tiles_before += warp_tiles[w]; }
        all += warp_blocks[w]; tiles_all += warp_tiles[w];
    }
    ov = all * p.SQ >= static_cast<int64_t>(kDrManyBlocks) * p.grid ? p.ov : min(p.ov, 2);
    const int64_t mine = (before + blocks + static_cast<int64_t>(tiles_before + tiles) * ov) * p.SQ;
    if (warps ? lane == 31 && wid < chunks : tid < chunks) sums[warps ? wid : tid] = mine;
    __syncthreads();
    return (all + static_cast<int64_t>(tiles_all) * ov) * p.SQ;
}

// The item that holds unit x, by one warp.  False (here and below) where there is none: lengths that changed under the call.
__device__ __forceinline__ bool drafted_locate(const DraftedParams &p, const int64_t *sums, int C, int chunks, int ov, int64_t x, int lane, DraftedWalk &w) {
    w.ov = ov;
    int c = 0;
    for (int c0 = 0; c0 < chunks; c0 += 32) {
        const unsigned hit = __ballot_sync(0xffffffffu, c0 + lane < chunks && x < sums[c0 + lane]);
        if (hit) { c = c0 + __ffs(hit) - 1; break; }
    }
    int64_t at = c == 0 ? 0 : sums[c - 1];
    for (w.u = c * C; w.u < p.B; ++w.u) {
        drafted_user(p, w.u, w.s);
        for (int rt0 = 0; rt0 * p.tt < w.s.n; rt0 += 32) {
            const int rt = rt0 + lane;
            const int64_t mine = rt * p.tt < w.s.n ? static_cast<int64_t>(drafted_keys(p, w.s, rt * p.tt, min(w.s.n, (rt + 1) * p.tt)).nb + ov) * p.SQ : 0;
            int64_t inc = mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int64_t up = __shfl_up_sync(0xffffffffu, inc, d);
                if (lane >= d) inc += up;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, x < at + inc);
            if (hit) {
                const int src = __ffs(hit) - 1;
                w.rt = rt0 + src;
                at += __shfl_sync(0xffffffffu, inc - mine, src);
                drafted_item_keys(p, w);
                w.sq = static_cast<int>(drafted_div(x - at, w.k.nb + ov));
                w.x0 = at + static_cast<int64_t>(w.sq) * (w.k.nb + ov);
                return true;
            }
            at += __shfl_sync(0xffffffffu, inc, 31);
        }
    }
    return false;
}

// The next item.
__device__ __forceinline__ bool drafted_next(const DraftedParams &p, DraftedWalk &w) {
    w.x0 += w.k.nb + w.ov;
    if (++w.sq < p.SQ) return true;
    w.sq = 0;
    if (++w.rt * p.tt >= w.s.n) {
        w.rt = 0;
        do {
            if (++w.u >= p.B || !drafted_user(p, w.u, w.s)) return false;
        } while (w.s.n == 0);
    }
    drafted_item_keys(p, w);
    return true;
}

// What the join has to know of a piece: valid, user, first token of q that is the tile's, (KV head, head group); tokens of the tile, first and last
// CTA that hold a piece of the item.
__device__ __forceinline__ void drafted_record(const DraftedParams &p, const DraftedWalk &w, int slot, int64_t W, int shares) {
    const int i0 = w.rt * p.tt;
    p.records[2 * slot] = make_int4(1, w.u, w.s.first + i0, w.sq);
    p.records[2 * slot + 1] = make_int4(min(p.tt, w.s.n - i0), drafted_share_of(W, shares, w.x0 + w.ov), drafted_share_of(W, shares, w.x0 + w.ov + w.k.nb - 1), 0);
}

// The blocks [b0, b1) of the item that units [x, x1) hold; none where b0 == b1.
__device__ __forceinline__ void drafted_blocks(const DraftedWalk &w, int64_t x, int64_t x1, int &b0, int &b1) {
    b0 = static_cast<int>(max(x - w.x0 - w.ov, static_cast<int64_t>(0)));
    b1 = static_cast<int>(max(min(static_cast<int64_t>(w.k.nb), x1 - w.x0 - w.ov), static_cast<int64_t>(0)));
}
__device__ __forceinline__ int drafted_shares(const DraftedParams &p, int64_t W, int ov) {
    return static_cast<int>(min(static_cast<int64_t>(p.grid), drafted_div(W + ov + kDrMinBlocks - 1, ov + kDrMinBlocks)));
}

// Raises the status of a user.
__device__ __forceinline__ void drafted_flag(const DraftedParams &p, int u) { flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u); }

// CTA 0 leaves in the header what the status query needs, and raises the first inconsistent offsets.
__device__ __forceinline__ void drafted_header(const DraftedParams &p, int first_bad) {
    p.hdr[HDR_BATCH] = p.B;
    p.hdr[HDR_NSEQ] = p.seqs;
    if (first_bad < p.B) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, first_bad);
}

// What becomes of a row with maximum m (natural units) and sum l: its O times `a`, plus the O that came in times `b` (0: not looked at).
// For a final result both carry 1 / l of the whole; a partial keeps O as it is, and m and l go with its first channels.
struct DraftedRow { float a, b, m, l; };
__device__ __forceinline__ DraftedRow drafted_row(const DraftedParams &p, int64_t row, float m, float l, bool bad) {
    if (bad) return DraftedRow{0.f, 0.f, -INFINITY, 0.f};
    DraftedRow f{1.f, 0.f, m, l};
    if (p.mode == OUT_PARTIAL) {
        if (l == 0.f) f.a = 0.f;              // nothing seen: whatever O holds comes from keys that are hidden
        return f;
    }
    if (p.in_o != nullptr) {
        const float mi = p.in_m[row], li = p.in_l[row], M = fmaxf(m, mi);
        f.a = m == -INFINITY ? 0.f : expf(m - M);
        f.b = mi == -INFINITY ? 0.f : expf(mi - M);
        // an empty part weighs nothing; a sum that is NaN (scores that are) stays
        l = (l != l ? l : f.a != 0.f ? l * f.a : 0.f) + (li != li ? li : f.b != 0.f ? li * f.b : 0.f);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    f.a = f.a == 0.f && l == l ? 0.f : f.a * inv;
    f.b = f.b == 0.f ? 0.f : f.b * inv;
    return f;
}

// Four channels of the row.
template <int D>
__device__ __forceinline__ void drafted_put4(const DraftedParams &p, int64_t row, int c4, float4 o, const DraftedRow &f) {
    float4 y = f.a == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * f.a, o.y * f.a, o.z * f.a, o.w * f.a);
    if (p.mode == OUT_PARTIAL) {
        reinterpret_cast<float4 *>(p.po)[row * (D / 4) + c4] = y;
        if (c4 == 0) { p.pm[row] = f.m; p.pl[row] = f.l; }
        return;
    }
    if (f.b != 0.f) {
        const float4 v = reinterpret_cast<const float4 *>(p.in_o)[row * (D / 4) + c4];
        y.x = fmaf(v.x, f.b, y.x); y.y = fmaf(v.y, f.b, y.y); y.z = fmaf(v.z, f.b, y.z); y.w = fmaf(v.w, f.b, y.w);
    }
    if (p.out_bf16) reinterpret_cast<uint2 *>(p.out)[row * (D / 4) + c4] = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    else reinterpret_cast<float4 *>(p.out)[row * (D / 4) + c4] = y;
}

// 16 consecutive channels from c on of the row, 32 bytes at a time (a thread's neighbours write other rows: whole sectors).
__device__ __forceinline__ void drafted_st32(bool wide, void *p, const uint32_t *w) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {                                  // the output starts at an odd multiple of 16 bytes
        static_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        static_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
template <int D>
__device__ __forceinline__ void drafted_put16(const DraftedParams &p, int64_t row, int c, float (&o)[16], const DraftedRow &f) {
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = f.a == 0.f ? 0.f : o[i] * f.a;
    if (f.b != 0.f) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(p.in_o + row * D + c + i);
            o[i] = fmaf(v.x, f.b, o[i]); o[i + 1] = fmaf(v.y, f.b, o[i + 1]); o[i + 2] = fmaf(v.z, f.b, o[i + 2]); o[i + 3] = fmaf(v.w, f.b, o[i + 3]);
        }
    }
    if (p.mode == OUT_PARTIAL && c == 0) { p.pm[row] = f.m; p.pl[row] = f.l; }
    uint32_t w[16];
    if (p.mode == OUT_FINAL && p.out_bf16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack_bf16(o[2 * i], o[2 * i + 1]);
        drafted_st32(p.wide != 0, static_cast<__nv_bfloat16 *>(p.out) + row * D + c, w);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i]);
        float *dst = (p.mode == OUT_PARTIAL ? p.po : static_cast<float *>(p.out)) + row * D + c;
        drafted_st32(p.wide != 0, dst, w);
        drafted_st32(p.wide != 0, dst + 8, w + 8);
    }
}

// The trees.  parent: the user's parents, -1 = the context.  Tokens above a token are found by walking up; `words` gets the bits of
// those (and of the token itself) that the window and the sinks let it see.  Depths are how many steps the walk takes.
__device__ __forceinline__ int drafted_depth(const int16_t *parent, int i) {
    int d = 0;
    for (int j = parent[i]; j >= 0; j = parent[j]) ++d;
    return d;
}
__device__ __forceinline__ void drafted_line(const DraftedParams &p, const DraftedUser &s, const int16_t *parent, int i, int depth, uint32_t *words) {
#pragma unroll
    for (int x = 0; x < kDrWords; ++x) words[x] = 0u;
    int d = depth;
    for (int j = i; j >= 0; j = parent[j], --d)
        if (p.window == 0 || depth - d < p.window || static_cast<int64_t>(s.ctx) + d < p.sinks) words[j >> 5] |= 1u << (j & 31);
}

// ---------------------------------------------------------------------------------------------------------------------
// The join: CTAs (j, x, .) take a part of the item that the attention's CTA j left a piece of in its slot x, in proportion to the pieces; up to
// four of them share that part, one where a tile has few rows.  Bound by latency and L2: the pieces were written a moment ago.  148 shares of
// 64 x 26-token trees (20 MB of pieces) 15 us under ncu, cold; about 5 behind the attention, whose last CTAs it overlaps.  A thread joins 16 channels of a row: its neighbours' are the next rows', side by side in the slots, and it writes
// whole sectors.
constexpr int kDrJoinThreads = 128;
__host__ __device__ constexpr int drafted_join_split(int RT) { return RT >= 256 ? 4 : RT >= 64 ? 2 : 1; }
template <int D, int RT, bool LOG2>
__global__ void __launch_bounds__(kDrJoinThreads) drafted_join_kernel(const __grid_constant__ DraftedParams p) {
    constexpr float kUnit = LOG2 ? 0.69314718055994531f : 1.f;
    constexpr int AHEAD = 3, SPLIT = drafted_join_split(RT);      // pieces under way at a time
    // What comes next may set itself up; it waits for this kernel's end before it looks at anything of this call.  Not behind the FMA kernel, whose CTAs share
    // SMs: the next call's would be laid down unevenly around the join's (fp32, 8 heads of 64, call after call, early / not: 32 users x 4 tokens over 4 k
    // tokens 265-305 us / 193, 8 x 5 over 1.5 k 51 / 38, 4 x 12 over 280 18.6 / 17.4).
    if (LOG2) griddep_launch_dependents();
    griddep_wait();
    const int slot = 2 * blockIdx.x + blockIdx.y;
    const int4 a = p.records[2 * slot], b = p.records[2 * slot + 1];
    if (a.x == 0) return;
    const int tok0 = a.z, sq = a.w, toks = b.x, c0 = b.y, c1 = b.z, pieces = c1 - c0 + 1, rows = toks * p.hs;
    const int h0 = sq / p.hgroups * p.g + sq % p.hgroups * p.hs;
    const int E = rows * (D / 16), parts = pieces * SPLIT, mine = (static_cast<int>(blockIdx.x) - c0) * SPLIT + blockIdx.z;
    const int e0 = static_cast<int>(drafted_div(static_cast<int64_t>(E) * mine, parts)), e1 = static_cast<int>(drafted_div(static_cast<int64_t>(E) * (mine + 1), parts));
    auto exp_of = [](float x) { return LOG2 ? exp2f(x) : expf(x); };
    for (int e = e0 + threadIdx.x; e < e1; e += kDrJoinThreads) {
        const int c = e / rows, r = e - c * rows;
        float o[16], m = -INFINITY, l = 0.f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] = 0.f;
        for (int k0 = 0; k0 < pieces; k0 += AHEAD) {
            float mk[AHEAD], lk[AHEAD];
            float4 v[AHEAD][4];
#pragma unroll
            for (int y = 0; y < AHEAD; ++y) {
                mk[y] = -INFINITY; lk[y] = 0.f;
                if (k0 + y < pieces) {
                    const float *s = p.scratch + static_cast<size_t>(2 * (c0 + k0 + y) + (k0 + y == 0 ? 1 : 0)) * drafted_slot_floats(D, RT);
                    mk[y] = s[RT * D + r]; lk[y] = s[RT * (D + 1) + r];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[y][i] = reinterpret_cast<const float4 *>(s)[(4 * c + i) * RT + r];
                }
            }
            float M = m;
#pragma unroll
            for (int y = 0; y < AHEAD; ++y) { M = fmaxf(M, mk[y]); bad = bad || lk[y] == kDrBad; }
            const float wa = m == -INFINITY ? 0.f : exp_of(m - M);
            l = l != l ? l : l * wa;
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= wa;
#pragma unroll
            for (int y = 0; y < AHEAD; ++y) {
                const float wb = mk[y] == -INFINITY ? 0.f : exp_of(mk[y] - M);
                l += lk[y] != lk[y] ? lk[y] : wb != 0.f ? lk[y] * wb : 0.f;
                if (wb != 0.f) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        o[4 * i] = fmaf(v[y][i].x, wb, o[4 * i]); o[4 * i + 1] = fmaf(v[y][i].y, wb, o[4 * i + 1]);
                        o[4 * i + 2] = fmaf(v[y][i].z, wb, o[4 * i + 2]); o[4 * i + 3] = fmaf(v[y][i].w, wb, o[4 * i + 3]);
                    }
                }
            }
            m = M;
        }
        const int64_t row = (static_cast<int64_t>(tok0) + r / p.hs) * p.Hq + h0 + r % p.hs;
        drafted_put16<D>(p, row, 16 * c, o, drafted_row(p, row, m * kUnit, l, bad));
    }
}

}  // namespace spd

// Drafted tokens on the FMA pipes: fp32 arithmetic throughout.
//
// RT rows (64, or 16 where users bring few) x 64 keys a block, RPT x 4 scores per thread; the 16 threads of a row keep its maximum and sum in
// registers, weights go through shared memory to the threads that hold the row's channels (the same 16).  A hidden key's weight is the
// mark -1, which the product with V skips: whatever its rows of k and v hold never enters.  V comes (cp.async) under the scores, the next block's K under
// the weights and the product with V, so that a CTA has loads under way all the time.  Bound by shared-memory reads (RPT x 4 register tiles) and, where
// rows are few, by what a CTA has under way.  Measured, fp32, call after call: 32 users x 4-token trees over 4 k tokens, 8 heads of 64: 193 us (2.7 TB/s; with 4 rows one warp of a CTA's four
// computes), 32/8 heads of 128: 621 us (1.7); 8 users x 64 tokens over 4 k tokens, 32/8 heads of 128: 1.48 ms (23 TFLOP/s); 4 users x 12 tokens over
// 270-290 tokens, 8 heads of 64: 17.4 us with the join.
#pragma once

#include "spd_drafted.cuh"

namespace spd {

constexpr int kDrBlock = 64;              // keys per block
constexpr int kDrTiles = kDrBlock / kPage;

template <int D, int RT>
struct DraftedFma {
    static constexpr int RPT = RT == 16 ? 2 : 4;                  // rows per thread
    static constexpr int kPerSm = RT == 16 && D == 64 ? 4 : 1;   // CTAs of it that registers have to leave room for (shared memory allows so many)
    static constexpr int kThreads = RT / RPT * 16, kPitch = D + 4;       // rows of Q, K and V: 16-byte reads of 8 lanes fall in 32 banks
    static constexpr size_t smem_bytes() { return (static_cast<size_t>(RT + 2 * kDrBlock) * kPitch + RT * kDrBlock) * 4; }
};

__device__ __forceinline__ void drafted_copy16(uint32_t dst, const void *src, bool there) {       // zeros where there is nothing
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void drafted_copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void drafted_copies_wait1() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }      // all but the last group

template <int D, int RT>
__global__ void __launch_bounds__(DraftedFma<D, RT>::kThreads, DraftedFma<D, RT>::kPerSm) drafted_fma_kernel(const __grid_constant__ DraftedParams p) {
    using C = DraftedFma<D, RT>;
    constexpr int NT = C::kThreads, RPT = C::RPT, PITCH = C::kPitch, KB = kDrBlock, CH = D / 64;      // CH chunks of four channels per thread
    extern __shared__ __align__(16) float sm[];
    float *Qs = sm, *Ks = Qs + RT * PITCH, *Vs = Ks + KB * PITCH, *Ps = Vs + KB * PITCH;
    __shared__ int64_t sums[NT];
    __shared__ int first_bad;
    __shared__ DraftedTile tile_of[2][kDrTiles];
    __shared__ int page_of[2][kDrTiles];
    __shared__ int16_t parent[kDrTree];
    __shared__ int16_t depths[kDrTree];
    __shared__ uint32_t lines[RT][kDrWords];
    const int tid = threadIdx.x, lane = tid & 31, tx = tid & 15, ty = tid >> 4;
    int Cu, chunks, ov;
    griddep_wait();
    griddep_launch_dependents();          // the join's CTAs take the places of those that are done here, and wait for the last
    const int64_t W = drafted_sums<NT>(p, sums, &first_bad, Cu, chunks, ov);
    if (blockIdx.x == 0 && tid == 0) drafted_header(p, first_bad);
    if (tid < 4) p.records[4 * blockIdx.x + tid] = make_int4(0, 0, 0, 0);
    __syncthreads();
    const int shares = drafted_shares(p, W, ov);
    if (static_cast<int>(blockIdx.x) >= shares) return;
    int64_t x = drafted_bound(W, shares, blockIdx.x);
    const int64_t x1 = drafted_bound(W, shares, blockIdx.x + 1);
    __shared__ DraftedWalk walk;                  // one warp's: all threads must go by the same item
    __shared__ int found;
    for (bool start = true;; start = false) {
        if (tid < 32) {
            DraftedWalk next;
            if (!start) next = walk;
            __syncwarp();
            const bool is = start ? drafted_locate(p, sums, Cu, chunks, ov, x, lane, next) : drafted_next(p, next);
            if (lane == 0) { walk = next; found = is; }
        }
        __syncthreads();
        const DraftedWalk w = walk;
        int b0 = 0, b1 = 0;
        if (found) drafted_blocks(w, x, x1, b0, b1);
        x = w.x0 + w.ov + w.k.nb;                 // the next item, if it is this share's
        if (b0 == b1) break;
        const DraftedUser s = w.s;
        const int i0 = w.rt * p.tt, toks = min(p.tt, s.n - i0), rows = toks * p.hs;
        const int kvh = w.sq / p.hgroups, h0 = kvh * p.g + w.sq % p.hgroups * p.hs;
        bool bad = !s.good;
        // pages of block b, by the first threads; a page that is out of range counts as one without tokens, and the user is flagged
        auto look = [&](int b) {
            if (tid < kDrTiles) {
                const DraftedTile t = drafted_tile(p, s, w.k, b * kDrTiles + tid);
                int page = 0;
                if (t.cnt > 0) page = p.part[t.part].indices[t.entry];
                const bool ok = t.cnt > 0 && page >= 0 && page < p.part[t.part].num_pages;
                tile_of[b & 1][tid] = t;
                page_of[b & 1][tid] = ok ? page : (t.cnt > 0 ? -1 : -2);
            }
        };
        auto fetch = [&](int b, const void *const *pools, float *to) {
            for (int e = tid; e < KB * (D / 4); e += NT) {
                const int key = e / (D / 4), c = e % (D / 4), t = key / kPage, slot = key % kPage, page = page_of[b & 1][t];
                const DraftedTile &tile = tile_of[b & 1][t];
                const bool there = page >= 0 && slot < tile.cnt;
                const float *src = there ? static_cast<const float *>(pools[tile.part]) + ((static_cast<int64_t>(page) * p.Hkv + kvh) * kPage + slot) * D + 4 * c
                                         : static_cast<const float *>(p.q);
                drafted_copy16(smem_u32(to + key * PITCH + 4 * c), src, there);
            }
        };
        // ---- the first pages, Q and K on their way while the tree is walked
        __syncthreads();
        look(b0);
        for (int e = tid; e < RT * (D / 4); e += NT) {
            const int r = e / (D / 4), c = e % (D / 4);
            const int64_t row = r < rows ? (static_cast<int64_t>(s.first) + i0 + r / p.hs) * p.Hq + h0 + r % p.hs : 0;
            drafted_copy16(smem_u32(Qs + r * PITCH + 4 * c), static_cast<const float *>(p.q) + row * D + 4 * c, r < rows);
        }
        bool wrong = false;
        const bool tree = p.parents != nullptr && s.good;
        for (int i = tid; tree && i < s.n; i += NT) {
            const int up = p.parents[s.first + i];
            wrong = wrong || up < -1 || up >= i;
            parent[i] = static_cast<int16_t>(up < -1 || up >= i ? -1 : up);
        }
        bad = __syncthreads_or(wrong) || bad;
        fetch(b0, p.k_pool, Ks);
        drafted_copies_end();
        if (tree) {
            for (int i = tid; i < s.n; i += NT) depths[i] = static_cast<int16_t>(drafted_depth(parent, i));
            __syncthreads();
            for (int i = tid; i < toks; i += NT) drafted_line(p, s, parent, i0 + i, depths[i0 + i], lines[i]);
            __syncthreads();
        }
        int pos[RPT], tok[RPT];              // positions and tokens (within the tile) of the thread's rows
        float slope[RPT], m[RPT], l[RPT], o[RPT][4 * CH];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = min(RPT * ty + i, rows - 1);
            tok[i] = r / p.hs;
            pos[i] = s.ctx + (p.parents ? (s.good ? depths[i0 + tok[i]] : 0) : i0 + tok[i]);
            slope[i] = p.slopes ? p.slopes[h0 + r % p.hs] : 0.f;
            m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
            for (int c = 0; c < 4 * CH; ++c) o[i][c] = 0.f;
        }
        for (int b = b0; b < b1; ++b) {
            const DraftedTile *tiles = tile_of[b & 1];
            const int *tile_page = page_of[b & 1];
            if (b + 1 < b1) look(b + 1);
            fetch(b, p.v_pool, Vs);
            drafted_copies_end();
#pragma unroll
            for (int t = 0; t < kDrTiles; ++t) bad = bad || tile_page[t] == -1;
            drafted_copies_wait1();
            __syncthreads();                              // K is there
            float sc[RPT][4];
            const bool work = (tid & ~31) / 16 * RPT < rows;      // warps without a row have nothing to do
            if (work) {
#pragma unroll
                for (int i = 0; i < RPT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sc[i][j] = 0.f;
#pragma unroll 4
                for (int c = 0; c < D; c += 4) {
                    float4 a[RPT], k4[4];
#pragma unroll
                    for (int i = 0; i < RPT; ++i) a[i] = *reinterpret_cast<const float4 *>(Qs + (RPT * ty + i) * PITCH + c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) k4[j] = *reinterpret_cast<const float4 *>(Ks + (tx + 16 * j) * PITCH + c);
#pragma unroll
                    for (int i = 0; i < RPT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            sc[i][j] = fmaf(a[i].x, k4[j].x, sc[i][j]); sc[i][j] = fmaf(a[i].y, k4[j].y, sc[i][j]);
                            sc[i][j] = fmaf(a[i].z, k4[j].z, sc[i][j]); sc[i][j] = fmaf(a[i].w, k4[j].w, sc[i][j]);
                        }
                }
            }
            __syncthreads();                              // K is read
            if (b + 1 < b1) fetch(b + 1, p.k_pool, Ks);
            drafted_copies_end();
            if (work) {
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    bool seen[4];
                    float mx = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {          // key tx of tile j
                        const int at = tiles[j].base + tx;
                        const bool drafted = at >= s.ctx;
                        int far = pos[i] - at;             // distance
                        bool see = tx < tiles[j].cnt && tile_page[j] >= 0;
                        if (drafted && p.parents != nullptr) {
                            const int d = see ? at - s.ctx : 0;
                            far = see ? pos[i] - s.ctx - depths[d] : 0;
                            see = see && ((lines[tok[i]][d >> 5] >> (d & 31)) & 1u);
                        } else {
                            see = see && far >= 0 && (p.window == 0 || far < p.window || at < p.sinks);
                        }
                        seen[j] = see;
                        float v = sc[i][j] * p.sm_scale;
                        if (p.cap > 0.f) v = p.cap * tanhf(v / p.cap);
                        if (p.slopes != nullptr) v = fmaf(-slope[i], static_cast<float>(far), v);
                        sc[i][j] = see ? v : -INFINITY;
                        mx = fmaxf(mx, sc[i][j]);
                    }
#pragma unroll
                    for (int d = 8; d >= 1; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn;
                    const float alpha = m[i] == -INFINITY ? 1.f : expf(m[i] - ref);        // nothing seen yet: O is 0, and l 0 or NaN
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float wt = seen[j] ? expf(sc[i][j] - ref) : -1.f;
                        Ps[(RPT * ty + i) * KB + tx + 16 * j] = wt;
                        sum += seen[j] ? wt : 0.f;
                    }
#pragma unroll
                    for (int d = 8; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    l[i] = l[i] * alpha + sum;
                    m[i] = mn;
#pragma unroll
                    for (int c = 0; c < 4 * CH; ++c) o[i][c] *= alpha;
                }
            }
            drafted_copies_wait1();
            __syncthreads();                              // V is there, and the weights
            if (work) {
#pragma unroll 2
                for (int k4 = 0; k4 < KB; k4 += 4) {
                    float4 wt[RPT];
#pragma unroll
                    for (int i = 0; i < RPT; ++i) wt[i] = *reinterpret_cast<const float4 *>(Ps + (RPT * ty + i) * KB + k4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float4 v[CH];
#pragma unroll
                        for (int c = 0; c < CH; ++c) v[c] = *reinterpret_cast<const float4 *>(Vs + (k4 + k) * PITCH + 4 * (tx + 16 * c));
#pragma unroll
                        for (int i = 0; i < RPT; ++i) {
                            const float q = k == 0 ? wt[i].x : k == 1 ? wt[i].y : k == 2 ? wt[i].z : wt[i].w;
                            if (q < 0.f) continue;
#pragma unroll
                            for (int c = 0; c < CH; ++c) {
                                o[i][4 * c] = fmaf(q, v[c].x, o[i][4 * c]); o[i][4 * c + 1] = fmaf(q, v[c].y, o[i][4 * c + 1]);
                                o[i][4 * c + 2] = fmaf(q, v[c].z, o[i][4 * c + 2]); o[i][4 * c + 3] = fmaf(q, v[c].w, o[i][4 * c + 3]);
                            }
                        }
                    }
                }
            }
            __syncthreads();
        }
        // ---- the piece: the whole item, or a slot
        if (bad && tid == 0) drafted_flag(p, w.u);
        const bool whole = b0 == 0 && b1 == w.k.nb;
        const int slot = 2 * blockIdx.x + (b0 == 0 ? 1 : 0);
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = RPT * ty + i;
            if (r >= rows) continue;
            const int64_t row = (static_cast<int64_t>(s.first) + i0 + tok[i]) * p.Hq + h0 + r % p.hs;
            float *dst = p.scratch + static_cast<size_t>(slot) * drafted_slot_floats(D, RT);
            DraftedRow f{};
            if (whole) f = drafted_row(p, row, m[i], l[i], bad);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const float4 v = make_float4(o[i][4 * c], o[i][4 * c + 1], o[i][4 * c + 2], o[i][4 * c + 3]);
                if (whole) drafted_put4<D>(p, row, tx + 16 * c, v, f);
                else reinterpret_cast<float4 *>(dst)[(tx + 16 * c) * RT + r] = v;
            }
            if (!whole && tx == 0) { dst[RT * D + r] = m[i]; dst[RT * (D + 1) + r] = bad ? kDrBad : l[i]; }
        }
        if (!whole && tid == 0) drafted_record(p, w, slot, W, shares);
        if (x >= x1) break;
    }
}

}  // namespace spd

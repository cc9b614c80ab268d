// Decode attention for calls with few and short sequences: one cluster of CTAs per sequence (user, kv head, group of <= 8 query
// heads), the tiles of the sequence dealt out over the cluster's warps, the pieces joined in shared memory and across
// the cluster's shared memories.
//
// Such a call is bound by latency, not by HBM: the persistent kernel spends most of it on its plan (every CTA derives the
// cut of the whole batch) and on handing pieces over through global memory (fence, ticket, round trips of the merge).  Here
// the chain is: lengths and table bounds, page indices, tiles, join.  Tiles, arithmetic and ring are the persistent kernel's.
// Used where every warp has at most kShortTiles tiles and all clusters fit the machine at once (one CTA per SM).  Measured, this
// kernel / the persistent one, us per call back to back, 32/8 heads, head_dim 128, bf16: 1 user x 288 tokens (in pools that hold
// little more: without a window the pools' pages are all that the host knows of the lengths) 5.9 / 18.2, 8 users
// through a window of 1024 tokens 10.3 / 26.2, of 4096 25.2 / 42.1, of 8192 (32 tiles a warp) 45.3 / 61.0; beyond that the gap
// closes (16 users, 16384: 171 / 180) and uneven lengths are what the persistent kernel's cut is for.
#pragma once

#include "spd_kernels.cuh"

namespace spd {

constexpr int kShortTiles = 32;        // tiles per warp up to which a call counts as short
constexpr int kShortMaxCluster = 8;

__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_addr(const void *p, uint32_t rank) {     // the same place in another CTA of the cluster
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// Bytes of dynamic shared memory: rings, one mbarrier per stage, the warps' extra areas, and the CTA's own result.
template <class Math>
__host__ __device__ constexpr size_t short_extra_offset() { return (static_cast<size_t>(Math::kWarps) * Math::kStages * 8 + 15) / 16 * 16; }
template <class Math>
__host__ __device__ constexpr size_t short_result_offset() { return short_extra_offset<Math>() + static_cast<size_t>(Math::kWarps) * Math::kExtraBytes; }
template <class Math>
__host__ __device__ constexpr size_t short_smem_bytes() {
    return 1024 + static_cast<size_t>(Math::kWarps) * Math::kStages * 2 * Math::kTileBytes + short_result_offset<Math>() +
           (kHeadsPerItem * (Math::D + 2) + 4) * 4;
}

// The join of one head's pieces, one after the other (Theorem 1): every piece is brought to the greater maximum.
template <int V>
struct ShortJoin {
    float o[V], m = -INFINITY, l = 0.f;
    __device__ __forceinline__ ShortJoin() {
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = 0.f;
    }
    __device__ __forceinline__ void add(const float (&v)[V], float mx, float lx) {
        const float M = fmaxf(m, mx);
        const float a = m == -INFINITY ? 0.f : expf(m - M);
        // an empty piece weighs nothing, but a piece whose keys are all NaN has no maximum either, and its l must not get lost
        const float w = mx == -INFINITY ? (lx != lx ? lx : 0.f) : expf(mx - M);
        l = (l != l ? l : l * a) + (w != 0.f ? w * lx : 0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = o[i] * a + (w != 0.f ? w * v[i] : 0.f);
        m = M;
    }
};

template <class Math>
__global__ void __launch_bounds__(Math::kWarps * 32, 1)
attn_short_kernel(const __grid_constant__ Params p, const __grid_constant__ CUtensorMap mk0, const __grid_constant__ CUtensorMap mv0,
                  const __grid_constant__ CUtensorMap mk1, const __grid_constant__ CUtensorMap mv1, int cluster) {
    static_assert(Math::kScored, "only scored calls come here");
    constexpr int D = Math::D, NS = Math::kStages, TB = Math::kTileBytes, NW = Math::kWarps, V = D / 32, PITCH = D + 4;
    static_assert(2 * TB >= (kHeadsPerItem * PITCH + 3 * kHeadsPerItem) * 4, "a stage must hold the epilogue staging");
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int wid = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *ring = base + static_cast<size_t>(wid) * NS * 2 * TB;
    uint8_t *tail = base + static_cast<size_t>(NW) * NS * 2 * TB;
    uint64_t *bars = reinterpret_cast<uint64_t *>(tail) + wid * NS;
    uint8_t *extra = tail + short_extra_offset<Math>() + static_cast<size_t>(wid) * Math::kExtraBytes;
    float *result = reinterpret_cast<float *>(tail + short_result_offset<Math>());     // O[8][D], m[8], l[8], bad page seen

    if (wid == 0 && lane < 4 && (p.part[0].num_pages > 0 || p.part[1].num_pages > 0))
        prefetch_tensormap(lane == 0 ? &mk0 : lane == 1 ? &mv0 : lane == 2 ? &mk1 : &mv1);
    const int seq = blockIdx.x / cluster, rank = blockIdx.x - seq * cluster;
    const int u = seq / p.S, sq = seq - u * p.S, kvh = sq / p.hgroups;
    if (lane == 0) {
        for (int s = 0; s < NS; ++s) mbar_init(smem_u32(&bars[s]), 1);
        fence_mbar_init();
    }
    __syncwarp();

    // ---- the sequence's tiles: the validated counts of the user, from the first tile inside the window on
    Cursor c;
    c.u = u;
    cursor_load_user<true>(c, p, nullptr);
    const int step = cluster * NW, w0 = rank * NW + wid;      // this warp's tiles: w0, w0 + step, ...
    const int n = c.np > w0 ? (c.np - w0 + step - 1) / step : 0;
    const uint64_t policy = l2_evict_first_policy();
    int page_of = -1;                                          // lane k holds the page of the warp's tile (batch of 32) k
    auto fetch_pages = [&](int k0) {
        const int j = w0 + (k0 + lane) * step;
        page_of = -1;
        if (j < c.np) page_of = j < c.npp ? p.part[0].indices[c.base0 + j] : p.part[1].indices[c.base1 + j - c.npp];
    };
    // valid tokens of tile j, 0 where its page is out of range
    auto valid_of = [&](int j, int page) {
        const int part = j >= c.npp ? 1 : 0, jj = part ? j - c.npp : j, npart = part ? c.np - c.npp : c.npp;
        if (page < 0 || page >= p.part[part].num_pages) return 0;
        return jj == npart - 1 ? (part ? c.len1 : c.len0) - jj * kPage : kPage;
    };
    auto issue = [&](int k) {
        if (k > 0 && (k & 31) == 0) fetch_pages(k);
        const int j = w0 + k * step, page = __shfl_sync(0xffffffffu, page_of, k & 31), part = j >= c.npp ? 1 : 0;
        const int valid = valid_of(j, page);
        if (lane == 0) {
            const uint32_t bar = smem_u32(&bars[k % NS]);
            if (valid == 0) {
                mbar_arrive(bar);
            } else {
                const int y = (page * p.Hkv + kvh) * kPage;
                const uint32_t kdst = smem_u32(ring + static_cast<size_t>(k % NS) * 2 * TB), vdst = kdst + TB;
                const CUtensorMap *mk = part ? &mk1 : &mk0, *mv = part ? &mv1 : &mv0;
                mbar_expect_tx(bar, 2 * TB);
#pragma unroll
                for (int b = 0; b < Math::kBoxes; ++b) {
                    tma_load_2d(kdst + b * Math::kBoxBytes, mk, b * Math::kBoxCols, y, bar, policy);
                    tma_load_2d(vdst + b * Math::kBoxBytes, mv, b * Math::kBoxCols, y, bar, policy);
                }
            }
        }
        return valid;
    };
    int valids[NS];                                            // of the tiles in the ring
    if (n > 0) fetch_pages(0);
#pragma unroll
    for (int s = 0; s < NS; ++s) valids[s] = s < n ? issue(s) : 0;

    // Up to here only the call's inputs were read (see the persistent kernel); q, the workspace and the outputs from here on.
    griddep_wait();
    // The next kernel may start its preamble only now that the kernel before this one has gone: the persistent kernel reads the
    // rate table and a stored plan there, which the launch before the previous one may still be writing otherwise -- this
    // grid may be small and can be resident as a whole beside it.
    griddep_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.hdr[HDR_BATCH] = p.B;
        p.hdr[HDR_NSEQ] = p.B * p.S;
        p.plan[PLAN_TAG] = 0;              // as after any call that derives its own cut: no plan to reuse
    }
    typename Math::State st;
    Math::begin(st, p, u, sq, lane, extra);
    bool bad = false, dead = false;
    for (int k0 = 0; k0 < n && !dead; k0 += NS) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int k = k0 + s;
            if (k >= n || dead) continue;
            if (!mbar_wait(smem_u32(&bars[s]), (k / NS) & 1)) { dead = true; continue; }
            const int j = w0 + k * step;
            uint8_t *Ks = ring + static_cast<size_t>(s) * 2 * TB, *Vs = Ks + TB;
            if (valids[s] > 0) Math::tile(st, p, Ks, Vs, valids[s], lane, extra, j < c.npp ? c.rel0 - j * kPage : c.rel1 - (j - c.npp) * kPage);
            else bad = true;
            __syncwarp();
            if (k + NS < n) valids[s] = issue(k + NS);
        }
    }
    if (dead) {
        if (lane == 0) flag_error(p.hdr, 6 /* SPD_ERR_TIMEOUT */, -1);
        for (int s = 0; s < NS; ++s) mbar_wait(smem_u32(&bars[s]), ((n - 1) / NS) & 1);    // a bounded chance for copies in flight
    }
    // ---- the warp's piece into its first stage (every copy into it has been consumed), then the CTA's pieces into one
    __syncwarp();
    float *So = reinterpret_cast<float *>(ring), *Sm = So + kHeadsPerItem * PITCH;
    Math::finish(st, So, Sm, Sm + kHeadsPerItem, lane);
    const bool cta_bad = __syncthreads_or(bad) != 0;
    const int hbase = first_head(p, sq);
    bool user_bad = false;                 // inconsistent tables: flagged, zeros
    if (c.np == 0) {
        int n0, n1;
        user_bad = (rank == 0 && threadIdx.x == 0) ? user_tiles<true, true>(p, u, n0, n1) : user_tiles<false, true>(p, u, n0, n1);
    }
    const bool b1 = user_bad || cta_bad;
    if (cluster == 1 && cta_bad && threadIdx.x == 0) { p.bad[u] = p.epoch; flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u); }
    for (int hh = wid; hh < p.geff; hh += NW) {
        ShortJoin<V> a;
        for (int x = 0; x < NW; ++x) {
            const float *src = reinterpret_cast<const float *>(base + static_cast<size_t>(x) * NS * 2 * TB);
            float v[V];
#pragma unroll
            for (int y = 0; y < V; ++y) v[y] = src[hh * PITCH + lane * V + y];
            a.add(v, src[kHeadsPerItem * PITCH + hh], src[kHeadsPerItem * (PITCH + 1) + hh]);
        }
        if (cluster == 1) {
            finalize_store<D>(p, u, hbase + hh, a.o, a.m, a.l, lane, b1);
        } else {
#pragma unroll
            for (int y = 0; y < V; ++y) result[hh * D + lane * V + y] = a.o[y];
            if (lane == 0) { result[kHeadsPerItem * D + hh] = a.m; result[kHeadsPerItem * (D + 1) + hh] = a.l; }
        }
    }
    if (cluster == 1) return;
    if (threadIdx.x == 0) result[kHeadsPerItem * (D + 2)] = cta_bad ? 1.f : 0.f;
    cluster_sync_all();
    // ---- across the cluster: CTA r finishes heads r, r + cluster, ...
    bool any_bad = user_bad;
    for (int x = 0; x < cluster; ++x) any_bad = any_bad || ld_cluster(cluster_addr(result + kHeadsPerItem * (D + 2), x)) != 0.f;
    if (any_bad && !user_bad && rank == 0 && threadIdx.x == 0) { p.bad[u] = p.epoch; flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u); }
    for (int hh = rank + cluster * wid; hh < p.geff; hh += cluster * NW) {
        ShortJoin<V> a;
        for (int x = 0; x < cluster; ++x) {
            float v[V];
#pragma unroll
            for (int y = 0; y < V; ++y) v[y] = ld_cluster(cluster_addr(result + hh * D + lane * V + y, x));
            a.add(v, ld_cluster(cluster_addr(result + kHeadsPerItem * D + hh, x)), ld_cluster(cluster_addr(result + kHeadsPerItem * (D + 1) + hh, x)));
        }
        finalize_store<D>(p, u, hbase + hh, a.o, a.m, a.l, lane, any_bad);
    }
    cluster_sync_all();                    // nobody leaves while another still reads its shared memory
}

}  // namespace spd

// Pages of a paged cache: handing them out, sharing, copying and releasing them, and moving the rows of accepted drafted tokens together.
//
// What is known of the pages is refs[page], the number of table entries that list it; a page that nobody lists (0) is free.  Fresh pages are
// the lowest free ones, in the order of users and entries, so that a call's result does not depend on timing.  Tables: entry -1 = no page.
//
// Handing out takes two kernels.  The first looks over refs (a CTA per chunk of pages writes its free ones down in ascending order) and
// over the users (how many pages each needs, and whether its request is in order); the second gives each user its ranks among the free
// pages by sums over the users in front of it, so no CTA waits for another.  Bound by latency: two launches and the loads behind
// one another; refs are read once.  One launch of either 5 us under ncu, cold; release and take of 512 users over 122 k pages 12.5 us from a
// graph, of 8 users over 460 pages 7.
#pragma once

#include "spd_device.cuh"

namespace spd {

constexpr int kPgThreads = 256;
constexpr int kPgChunk = 4096;            // pages per CTA of the first kernel, unless that makes too many
constexpr int kPgMaxChunks = 1024;
constexpr int kPgPools = 128;             // pools per launch
constexpr int kPgPiece = 16384;           // bytes that a CTA copies
constexpr int kPgTree = 256;              // most drafted tokens of a user that come as a tree

// What a kernel here has written is there, for TMA reads too, once all its CTAs have left: an attention call behind it may read tables, lengths and
// rows before the kernel counts as finished for its stream.
__device__ __forceinline__ void pages_written() {
    __threadfence();
    asm volatile("fence.proxy.async.global;" ::: "memory");
}

enum PagesState { PG_REFUSED = -1, PG_NONE = -2 };      // in place of a user's demand

struct PagesParams {
    int32_t B, num_pages, chunk, chunks;
    int32_t *refs;
    const int32_t *indptr;
    int32_t *indices;
    const int32_t *from, *to;             // tokens; to may be null (all)
    const int32_t *source;                // fork; null = take
    int32_t *lens, *copies;               // fork
    int32_t *hdr, seqs;
    int32_t *demand, *chunk_free, *free;  // [B], [chunks], [num_pages]
};

__device__ __forceinline__ void pages_header(int32_t *hdr, int B, int seqs) {
    hdr[HDR_BATCH] = B;
    hdr[HDR_NSEQ] = seqs;
}

// A user's entries; false where its table is inconsistent, or has entries and is not there.
__device__ __forceinline__ bool pages_entries(const PagesParams &p, int u, int64_t &lo, int64_t &cap) {
    const int64_t hi = p.indptr[u + 1], end = p.indptr[p.B];
    lo = p.indptr[u];
    cap = hi - lo;
    return lo >= 0 && cap >= 0 && hi <= end && (cap == 0 || p.indices != nullptr);
}

// Block-wide: exclusive prefix of v over the threads, and the total.
__device__ __forceinline__ int pages_scan(int v, int *warp_sums, int &total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += up;
    }
    __syncthreads();
    if (lane == 31) warp_sums[w] = inc;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int x = 0; x < kPgThreads / 32; ++x) {
        if (x < w) before += warp_sums[x];
        total += warp_sums[x];
    }
    return before + inc - v;
}

static __global__ void __launch_bounds__(kPgThreads) pages_release_kernel(const __grid_constant__ PagesParams p) {
    const int u = blockIdx.x, tid = threadIdx.x;
    if (u == 0 && blockIdx.y == 0 && tid == 0) pages_header(p.hdr, p.B, p.seqs);
    int64_t lo, cap;
    const int64_t from = p.from[u], to = p.to ? p.to[u] : 0;
    bool bad = !pages_entries(p, u, lo, cap) || from < 0 || to < 0;
    if (!bad) {
        const int64_t e1 = p.to ? min(cap, to / kPage) : cap;
        for (int64_t e = (from + kPage - 1) / kPage + blockIdx.y * kPgThreads + tid; e < e1; e += gridDim.y * kPgThreads) {
            const int page = p.indices[lo + e];
            if (page == -1) continue;
            if (page < 0 || page >= p.num_pages) { bad = true; continue; }
            if (atomicSub(&p.refs[page], 1) <= 0) { atomicAdd(&p.refs[page], 1); bad = true; }
            p.indices[lo + e] = -1;
        }
    }
    if (bad) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);
    pages_written();
}

// CTAs [0, chunks): the free pages of a chunk; CTAs behind them: the demand of a user.
static __global__ void __launch_bounds__(kPgThreads) pages_look_kernel(const __grid_constant__ PagesParams p) {
    __shared__ int warp_sums[kPgThreads / 32];
    const int tid = threadIdx.x;
    if (static_cast<int>(blockIdx.x) < p.chunks) {
        const int first = blockIdx.x * p.chunk, end = min(p.num_pages, first + p.chunk);
        int found = 0;
        for (int at = first; at < end; at += kPgThreads * 16) {          // 16 pages per thread and turn
            const int mine = at + tid * 16;
            uint32_t bits = 0;
#pragma unroll
            for (int x = 0; x < 16; x += 4) {
                int4 r = make_int4(1, 1, 1, 1);
                if (mine + x + 3 < end) r = *reinterpret_cast<const int4 *>(p.refs + mine + x);
                else {
                    if (mine + x < end) r.x = p.refs[mine + x];
                    if (mine + x + 1 < end) r.y = p.refs[mine + x + 1];
                    if (mine + x + 2 < end) r.z = p.refs[mine + x + 2];
                }
                bits |= (r.x == 0 ? 1u << x : 0u) | (r.y == 0 ? 2u << x : 0u) | (r.z == 0 ? 4u << x : 0u) | (r.w == 0 ? 8u << x : 0u);
            }
            int total, k = first + found + pages_scan(__popc(bits), warp_sums, total);
            for (; bits != 0; bits &= bits - 1) p.free[k++] = mine + __ffs(bits) - 1;
            found += total;
        }
        if (tid == 0) p.chunk_free[blockIdx.x] = found;
        return;
    }
    const int u = blockIdx.x - p.chunks;
    if (u == 0 && tid == 0) pages_header(p.hdr, p.B, p.seqs);
    int64_t lo, cap;
    bool bad = !pages_entries(p, u, lo, cap);
    int need = 0;
    if (p.source == nullptr) {
        const int64_t from = p.from[u], to = p.to[u], e1 = (to + kPage - 1) / kPage;
        bad = bad || from < 0 || to < 0 || (to > from && e1 > cap);
        if (!bad)
            for (int64_t e = (from + kPage - 1) / kPage + tid; e < e1; e += kPgThreads) need += p.indices[lo + e] == -1;
    } else {
        const int s = p.source[u];
        if (s == -1) {
            if (tid == 0) p.demand[u] = PG_NONE;
            return;
        }
        bad = bad || s < 0 || s >= p.B || s == u || p.source[min(max(s, 0), p.B - 1)] != -1;
        int64_t slo = 0, scap = 0, len = 0;
        if (!bad) { bad = !pages_entries(p, s, slo, scap); len = p.lens[s]; }
        const int64_t pages = (len + kPage - 1) / kPage;
        bad = bad || len < 0 || pages > cap || pages > scap;
        if (!bad) {
            for (int64_t e = tid; e < pages; e += kPgThreads) {
                const int page = p.indices[slo + e];
                const bool hole = page == -1 && e < len / kPage;           // a page that was released behind a window
                bad = bad || p.indices[lo + e] != -1 || !(hole || (page >= 0 && page < p.num_pages && p.refs[page] > 0));
            }
            need = tid == 0 && len % kPage != 0;
        }
    }
    bad = __syncthreads_or(bad);
    int total;
    pages_scan(need, warp_sums, total);
    if (tid == 0) {
        p.demand[u] = bad ? static_cast<int>(PG_REFUSED) : total;
        if (bad) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);
    }
}

// One CTA per user.
static __global__ void __launch_bounds__(kPgThreads) pages_give_kernel(const __grid_constant__ PagesParams p) {
    __shared__ int warp_sums[kPgThreads / 32];
    __shared__ int ends[kPgMaxChunks];             // free pages up to the end of each chunk
    const int u = blockIdx.x, tid = threadIdx.x;
    griddep_wait();
    const int need = p.demand[u];
    if (p.source != nullptr && tid < 2) p.copies[2 * u + tid] = -1;
    if (need < 0 || (need == 0 && p.source == nullptr)) return;
    int rank = 0;
    bool fits = true;
    if (need > 0) {
        int before = 0;
        for (int x = tid; x < u; x += kPgThreads) before += max(0, p.demand[x]);
        int total;
        pages_scan(before, warp_sums, total);
        rank = total;
        int c[kPgMaxChunks / kPgThreads], sum = 0;
#pragma unroll
        for (int x = 0; x < kPgMaxChunks / kPgThreads; ++x) {
            const int at = tid * (kPgMaxChunks / kPgThreads) + x;
            c[x] = at < p.chunks ? p.chunk_free[at] : 0;
            sum += c[x];
        }
        int end = pages_scan(sum, warp_sums, total);
#pragma unroll
        for (int x = 0; x < kPgMaxChunks / kPgThreads; ++x) {
            end += c[x];
            ends[tid * (kPgMaxChunks / kPgThreads) + x] = end;
        }
        fits = rank + need <= total;
        __syncthreads();
    }
    if (!fits) {
        if (tid == 0) flag_error(p.hdr, 8 /* SPD_ERR_NO_PAGE */, u);
        return;
    }
    auto fresh = [&](int r) {                      // the free page of rank r; -1 where tables changed under the call
        if (p.chunks == 0 || r >= ends[p.chunks - 1]) return -1;
        int a = 0, b = p.chunks - 1;
        while (a < b) {
            const int mid = (a + b) / 2;
            if (ends[mid] > r) b = mid; else a = mid + 1;
        }
        const int page = p.free[a * p.chunk + r - (a > 0 ? ends[a - 1] : 0)];
        p.refs[page] = 1;
        return page;
    };
    int64_t lo, cap;
    if (!pages_entries(p, u, lo, cap)) return;
    if (p.source == nullptr) {
        const int64_t e0 = (max(p.from[u], 0) + static_cast<int64_t>(kPage) - 1) / kPage, e1 = min(cap, (p.to[u] + static_cast<int64_t>(kPage) - 1) / kPage);
        for (int64_t at = e0; at < e1; at += kPgThreads) {
            const int64_t e = at + tid;
            const bool wants = e < e1 && p.indices[lo + e] == -1;
            int total;
            const int k = rank + pages_scan(wants, warp_sums, total);
            if (wants) p.indices[lo + e] = fresh(k);
            rank += total;
        }
    } else {
        const int s = p.source[u], len = p.lens[s];
        int64_t slo, scap;
        if (!pages_entries(p, s, slo, scap) || len < 0 || (len + kPage - 1ll) / kPage > min(scap, cap)) return;
        for (int e = tid; e < len / kPage; e += kPgThreads) {
            const int page = p.indices[slo + e];
            p.indices[lo + e] = page;
            if (page >= 0) atomicAdd(&p.refs[page], 1);
        }
        if (tid == 0) {
            if (len % kPage != 0 && need > 0) {
                const int page = fresh(rank);
                p.copies[2 * u] = p.indices[slo + len / kPage];
                p.copies[2 * u + 1] = page;
                p.indices[lo + len / kPage] = page;
            }
            p.lens[u] = len;
        }
    }
    pages_written();
}

struct PagesPools { void *pool[kPgPools]; };

// Pages copies[i][0] -> copies[i][1] in every pool; a CTA per pair, pool and piece of a page, four 16-byte loads per thread under way.  Bound by HBM: 360
// pages of 32 KB in 16 pools (378 MB read and written) 40 us under ncu (9 TB/s, a part of it in L2).
static __global__ void __launch_bounds__(kPgThreads)
pages_copy_kernel(const __grid_constant__ PagesPools pools, const int32_t *copies, int32_t num_pages, int64_t page_bytes, int32_t *hdr) {
    const int i = blockIdx.x, src = copies[2 * i], dst = copies[2 * i + 1];
    if (src == -1 && dst == -1) return;
    if (src < 0 || src >= num_pages || dst < 0 || dst >= num_pages) {
        if (threadIdx.x == 0) flag_error(hdr, 4 /* SPD_ERR_BAD_PAGE */, i);
        return;
    }
    const int64_t at = static_cast<int64_t>(blockIdx.z) * kPgPiece, n = min(static_cast<int64_t>(kPgPiece), page_bytes - at) / 16;
    uint8_t *pool = static_cast<uint8_t *>(pools.pool[blockIdx.y]);
    const uint4 *a = reinterpret_cast<const uint4 *>(pool + src * page_bytes + at);
    uint4 *b = reinterpret_cast<uint4 *>(pool + dst * page_bytes + at);
    constexpr int PER = kPgPiece / 16 / kPgThreads;
    uint4 v[PER];
#pragma unroll
    for (int x = 0; x < PER; ++x)
        if (threadIdx.x + x * kPgThreads < n) v[x] = a[threadIdx.x + x * kPgThreads];
#pragma unroll
    for (int x = 0; x < PER; ++x)
        if (threadIdx.x + x * kPgThreads < n) b[threadIdx.x + x * kPgThreads] = v[x];
    pages_written();
}

struct KeepParams {
    int32_t B, Hkv, row_bytes, num_pools, num_pages;
    int64_t T;
    const int32_t *tok_indptr, *parents, *last;
    const int32_t *indptr, *indices, *lens;
    int32_t *new_lens, *kept;             // either may be null
    int32_t *hdr, seqs, *result;          // [B] grown lengths
};

// Accepted branches to the front of the drafted rows.  Token path[i] of a user's branch (root first) goes to place i <= path[i]; the
// branch ascends, so a place is written after its row was read, if it is written at all, when the rows are taken in order: a thread
// keeps to one 16-byte column of one head of one pool and walks the branch, and nobody else touches that column.
// Bound by latency (parents, pages, rows behind one another); rows of 128-256 bytes, read and written once.  512 users x 33-64-token trees, 16
// layers of 8 heads of 128 (205 MB) 45 us, 8 users in two layers 3.6 us from a graph.
static __global__ void __launch_bounds__(kPgThreads) keep_kernel(const __grid_constant__ KeepParams p, const __grid_constant__ PagesPools pools) {
    __shared__ int16_t parent[kPgTree];
    __shared__ int16_t path[kPgTree];
    __shared__ int64_t src[kPgTree], dst[kPgTree];
    __shared__ int count, last_cta;
    const int u = blockIdx.x, tid = threadIdx.x;
    if (u == 0 && blockIdx.y == 0 && tid == 0) pages_header(p.hdr, p.B, p.seqs);
    const int64_t a = p.tok_indptr ? p.tok_indptr[u] : u, b = p.tok_indptr ? p.tok_indptr[u + 1] : u + 1;
    const int64_t lo = p.indptr[u], hi = p.indptr[u + 1], end = p.indptr[p.B], len = p.lens[u], n = b - a;
    const int last = p.last[u];
    const bool rows_ok = a >= 0 && b >= a && b <= p.T && (u != 0 || a == 0) && (u != p.B - 1 || b == p.T);
    bool bad = !rows_ok || lo < 0 || hi < lo || hi > end || len < n || len > (hi - lo) * kPage || last < -1 || last >= n || (len > 0 && p.indices == nullptr) ||
               (p.parents != nullptr && n > kPgTree);
    const int64_t base = len - n;
    int kept = bad ? 0 : last + 1;                  // a run keeps its first tokens where they are
    if (p.parents != nullptr && !bad) {
        for (int i = tid; i < n; i += kPgThreads) {
            const int up = p.parents[a + i];
            bad = bad || up < -1 || up >= i;
            parent[i] = static_cast<int16_t>(up < -1 || up >= i ? -1 : up);
        }
        bad = __syncthreads_or(bad);
        if (tid == 0) {
            int d = 0;
            for (int j = last; j >= 0; j = parent[j]) ++d;
            count = d;
            for (int j = last; j >= 0; j = parent[j]) path[--d] = static_cast<int16_t>(j);
        }
        __syncthreads();
        kept = count;
        for (int i = tid; i < kept && !bad && p.num_pools > 0; i += kPgThreads) {       // no pools: lengths and names alone
            const int64_t s = base + path[i], d = base + i;
            const int ps = p.indices[lo + s / kPage], pd = p.indices[lo + d / kPage];
            if (ps < 0 || ps >= p.num_pages || pd < 0 || pd >= p.num_pages) { bad = true; break; }
            src[i] = (static_cast<int64_t>(ps) * p.Hkv * kPage + s % kPage) * p.row_bytes;
            dst[i] = (static_cast<int64_t>(pd) * p.Hkv * kPage + d % kPage) * p.row_bytes;
        }
        bad = __syncthreads_or(bad);
        if (!bad && p.num_pools > 0) {
            int i0 = 0;                             // the first tokens may stay where they are
            while (i0 < kept && path[i0] == i0) ++i0;
            const int lanes = p.row_bytes / 16, per = kPgThreads / lanes, col = tid % lanes * 16;
            for (int x = blockIdx.y * per + tid / lanes; x < p.num_pools * p.Hkv; x += gridDim.y * per) {
                uint8_t *pool = static_cast<uint8_t *>(pools.pool[x / p.Hkv]) + static_cast<int64_t>(x % p.Hkv) * kPage * p.row_bytes + col;
                for (int i = i0; i < kept; i += 4) {
                    uint4 v[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (i + y < kept) v[y] = *reinterpret_cast<const uint4 *>(pool + src[i + y]);
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (i + y < kept) *reinterpret_cast<uint4 *>(pool + dst[i + y]) = v[y];
                }
            }
        }
    }
    if (p.parents == nullptr && p.num_pools > 0 && kept > 0) {      // a run's rows stay where they are, but their pages have to be there
        for (int64_t e = base / kPage + tid; e <= (base + kept - 1) / kPage; e += kPgThreads) {
            const int page = p.indices[lo + e];
            bad = bad || page < 0 || page >= p.num_pages;
        }
        bad = __syncthreads_or(bad);
    }
    if (bad) kept = 0;
    if (blockIdx.y == 0) {
        if (bad && tid == 0) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);
        const int grown = static_cast<int>(bad ? len : base + kept);
        if (tid == 0) {
            p.result[u] = grown;
            if (p.new_lens != nullptr && p.new_lens != p.lens) p.new_lens[u] = grown;
        }
        if (p.kept != nullptr && rows_ok)
            for (int64_t i = tid; i < n; i += kPgThreads) p.kept[a + i] = i < kept ? (p.parents ? path[i] : static_cast<int>(i)) : -1;
    }
    pages_written();
    if (p.new_lens != p.lens) return;
    // in place: the lengths change once nobody reads them any more, so the last CTA out does it
    __syncthreads();
    if (tid == 0) last_cta = atomicAdd(&p.hdr[HDR_GRID_EXITS], 1) == static_cast<int32_t>(gridDim.x * gridDim.y) - 1;
    __syncthreads();
    if (!last_cta) return;
    __threadfence();
    if (tid == 0) p.hdr[HDR_GRID_EXITS] = 0;
    for (int x = tid; x < p.B; x += kPgThreads) p.new_lens[x] = __ldcg(p.result + x);
    __threadfence();
}

}  // namespace spd

// Prompt attention with capped scores, distance bias and interval masks.  Row i of a prompt sees the keys [lo_i, hi_i]:
//   lo_i = max(0, doc_start_i, i - window + 1),   hi_i = i, or the prefix's last token where i lies inside the prefix,
//   s = sm_scale q.k;  s <- cap tanh(s / cap);  s <- s - slope_h |i - j|.
#pragma once

#include "spd_prefill_fma.cuh"

namespace spd {

struct ScoredPrefillParams : PrefillParams {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;     // elements between consecutive tokens
    float cap;                                // 0 = none
    int32_t window;                           // 0 = none
    const float *slopes;                      // [Hq] or null
    const int32_t *prefix_lens, *doc_start;   // [B], [T]; either may be null
};

// The user behind a block that prefill_find_block located: the first whose tokens are [first, first + len), len > 0.
__device__ __forceinline__ int scored_user(const PrefillParams &p, int first, int len, int lane) {
    int best = 0x7fffffff;
    for (int u = lane; u < p.B; u += 32)
        if (p.tok_indptr[u] == first && p.tok_indptr[u + 1] == first + len) best = min(best, u);
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, d));
    return best;
}

// Raises the status for the first user at which the offsets are inconsistent, or the last one if they end early (run by
// one CTA of a launch; the blocks from that user on are not served by prefill_find_block).
__device__ __forceinline__ void scored_check_offsets(const PrefillParams &p) {
    for (int u = threadIdx.x; u < p.B; u += blockDim.x) {
        const int64_t a = p.tok_indptr[u], b = p.tok_indptr[u + 1];
        if (a < 0 || b < a || b > p.T || (u == p.B - 1 && b != p.T)) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);
    }
}

// Keys that row i of a prompt of len tokens sees; lo > hi: none.
__device__ __forceinline__ void scored_interval(const ScoredPrefillParams &p, int first, int prefix, int i, int &lo, int &hi) {
    lo = p.doc_start ? max(0, p.doc_start[first + i]) : 0;
    if (p.window > 0) lo = max(lo, i - p.window + 1);      // window <= 2^31 - 1 and i >= 0: no overflow
    hi = i < prefix ? prefix - 1 : i;
}

__device__ __forceinline__ int scored_prefix(const ScoredPrefillParams &p, int first, int len, int lane) {
    return p.prefix_lens ? min(len, p.prefix_lens[scored_user(p, first, len, lane)]) : 0;
}

template <typename T, int D>
__global__ void __launch_bounds__(kFmaRows * 32) prefill_scored_fma_kernel(const __grid_constant__ ScoredPrefillParams p) {
    constexpr int V = D / 32, KP = D + 1;          // K rows padded by one float: lane = key reads without bank conflicts
    __shared__ float Ks[kFmaKeys * KP];
    __shared__ float Vs[kFmaKeys * D];
    __shared__ float Qs[kFmaRows * D];
    __shared__ int32_t blo[kFmaRows], bhi[kFmaRows];
    const T *q = static_cast<const T *>(p.q), *k = static_cast<const T *>(p.k), *v = static_cast<const T *>(p.v);
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const int h = blockIdx.y, kvh = h / (p.Hq / p.Hkv);
    if (blockIdx.x == 0 && blockIdx.y == 0) scored_check_offsets(p);
    int qb, first, len;
    prefill_find_block(p, kFmaRows, blockIdx.x, lane, qb, first, len);
    if (qb < 0) return;                             // uniform over the CTA
    const int prefix = scored_prefix(p, first, len, lane);
    const int row = qb * kFmaRows + wid;            // this warp's query row within the prompt
    const bool live = row < len;
    int lo = 1, hi = 0;
    if (live) {
        for (int d = lane; d < D; d += 32) Qs[wid * D + d] = fma_widen<T>(q[(first + row) * p.q_stride + h * D + d]);
        scored_interval(p, first, prefix, row, lo, hi);
    }
    if (lane == 0) { blo[wid] = lo <= hi ? lo : 0x7fffffff; bhi[wid] = lo <= hi ? hi : -1; }
    __syncthreads();
    int key0 = 0x7fffffff, key1 = -1;               // keys that any row of the CTA sees
    for (int w = 0; w < kFmaRows; ++w) { key0 = min(key0, blo[w]); key1 = max(key1, bhi[w]); }
    const float slope = p.slopes ? p.slopes[h] : 0.f;
    float m = -INFINITY, l = 0.f, o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.f;
    for (int kb = key0; kb <= key1; kb += kFmaKeys) {
        __syncthreads();                            // the previous block's readers are done
        for (int idx = tid; idx < kFmaKeys * D; idx += kFmaRows * 32) {
            const int key = idx / D, d = idx - key * D, t = kb + key;
            float kk = 0.f, vv = 0.f;
            if (t <= key1) {
                kk = fma_widen<T>(k[(first + t) * p.k_stride + kvh * D + d]);
                vv = fma_widen<T>(v[(first + t) * p.v_stride + kvh * D + d]);
            }
            Ks[key * KP + d] = kk;
            Vs[key * D + d] = vv;
        }
        __syncthreads();
        const int t = kb + lane;                    // this lane's key
        const bool seen = t >= lo && t <= hi;       // never for a row that is not live
        const unsigned any = __ballot_sync(0xffffffffu, seen);
        if (any == 0) continue;                     // warp-uniform
        float s = 0.f;
#pragma unroll 8
        for (int d = 0; d < D; ++d) s = fmaf(Qs[wid * D + d], Ks[lane * KP + d], s);
        s *= p.sm_scale;
        if (p.cap > 0.f) s = p.cap * tanhf(s / p.cap);
        s = seen ? fmaf(-slope, fabsf(static_cast<float>(row - t)), s) : -INFINITY;
        float bm = s;
#pragma unroll
        for (int dd = 16; dd >= 1; dd >>= 1) bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, dd));
        const float m_new = fmaxf(m, bm);
        const float alpha = expf(m - m_new);        // exp(-inf) = 0 on the first block
        const float pr = seen ? expf(s - m_new) : 0.f;
        float ps = pr;
#pragma unroll
        for (int dd = 16; dd >= 1; dd >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, dd);
        l = l * alpha + ps;
        m = m_new;
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] *= alpha;
        for (unsigned left = any; left; left &= left - 1) {     // hidden keys' V rows are not touched
            const int j = __ffs(left) - 1;
            const float pj = __shfl_sync(0xffffffffu, pr, j);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = fmaf(pj, Vs[j * D + lane + 32 * i], o[i]);
        }
    }
    if (!live) return;
    const float inv = 1.f / l;                      // l is 0 only where the row sees nothing; NaN among what it sees stays NaN
    const int64_t dst = (static_cast<int64_t>(first + row) * p.Hq + h) * D;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float y = l == 0.f ? 0.f : o[i] * inv;
        if (p.out_bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[dst + lane + 32 * i] = __float2bfloat16_rn(y);
        else reinterpret_cast<float *>(p.out)[dst + lane + 32 * i] = y;
    }
}

}  // namespace spd

// Prompt attention with capped scores, distance bias and interval masks.  Row i of a prompt sees the keys [lo_i, hi_i]:
//   lo_i = max(0, doc_start_i, i - window + 1),   hi_i = i, or the prefix's last token where i lies inside the prefix,
//   s = sm_scale q.k;  s <- cap tanh(s / cap);  s <- s - slope_h |i - j|.
#pragma once

#include "spd_prefill.cuh"

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

}  // namespace spd

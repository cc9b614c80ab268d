// Prompt attention with score options and interval masks in fp32 on the FMA pipes (no reduced precision anywhere).
//
// A CTA owns 16 RPT query rows of one (user, head) and walks key blocks through shared memory; 256 threads as 16 x 16, a thread
// holding RPT rows x KB / 16 keys of S and RPT rows x D / 16 channels of O in registers, so that an operand read from shared
// memory serves several FMAs (shared memory brings a warp 4 bytes per lane and cycle, the same address or not: 32 cycles for 64 FMA
// instructions per warp and 4 channels at RPT = 4, half the FMA rate at most).  The 16
// threads of a row group sit in half a warp: row maxima and sums by shuffles, P through shared memory without a CTA
// barrier.  The next block is fetched into registers under this one's arithmetic.  Bound by shared-memory reads and issue
// together (75 % and 67 % of their peaks on long prompts: 4096 tokens, 16/4 heads, 27.5 TFLOP/s).  Small launches take RPT = 2 for twice
// the CTAs, or G = 2: two groups of 256 threads share a tile's rows, take its key blocks in turns and join at the end, which halves
// the chain of blocks (4 prompts of 256 tokens, 8 heads, head_dim 64: 25 us; 30 with RPT = 2, 41 with RPT = 4 alone, 31 with both).
// 8 x 4 tiles by 64 or 128 threads with asynchronous copies were no faster (35 us, 25 TFLOP/s), nor were FMAs two at a time
// (30.8 us, 26.1 TFLOP/s): instructions are not what it waits for.
#pragma once

#include "spd_prefill_scored.cuh"

namespace spd {

// G: groups of 256 threads that share the rows and take key blocks in turns.
template <int D, int RPT, int G>
struct ScoredF32 {
    static constexpr int R = 16 * RPT, KB = 4096 / D, KPT = KB / 16, CPT = D / 16, QP = D + 4, PP = KB + 4;
    static constexpr int kGroupFloats = KB * QP + KB * D + R * PP, kFloats = R * QP + G * kGroupFloats;
    static_assert(kGroupFloats >= R * D + 2 * R, "a group's tiles hold its result for the join");
    static constexpr size_t smem_bytes() { return kFloats * 4 + 2 * R * 4; }
};

template <int G>
__device__ __forceinline__ void f32_group_sync(int grp) {
    if constexpr (G == 1) __syncthreads();
    else asm volatile("bar.sync %0, 256;" ::"r"(1 + grp) : "memory");
}
template <int G>
__device__ __forceinline__ bool f32_group_any(int grp, bool x) {
    if constexpr (G == 1) {
        return __syncthreads_or(x);
    } else {
        uint32_t r;
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                     : "=r"(r) : "r"(static_cast<uint32_t>(x)), "r"(1 + grp) : "memory");
        return r != 0;
    }
}

template <int D, int RPT, int G>
__global__ void __launch_bounds__(256 * G, 2 / G) prefill_scored_f32_kernel(const __grid_constant__ ScoredPrefillParams p) {
    using C = ScoredF32<D, RPT, G>;
    constexpr int R = C::R, KB = C::KB, KPT = C::KPT, CPT = C::CPT, QP = C::QP, PP = C::PP, LD = KB * D / 4 / 256;   // float4 loads per thread and tile
    extern __shared__ __align__(16) float sm[];
    const int grp = G == 1 ? 0 : threadIdx.x >> 8;
    float *Qs = sm, *Ks = Qs + R * QP + grp * C::kGroupFloats, *Vs = Ks + KB * QP, *Ps = Vs + KB * D;
    int32_t *rlo = reinterpret_cast<int32_t *>(sm + C::kFloats), *rhi = rlo + R;
    const int tid = threadIdx.x & 255, lane = tid & 31, tx = tid & 15, ty = tid >> 4;
    const int h = blockIdx.y, kvh = h / (p.Hq / p.Hkv);
    if (blockIdx.x == 0 && blockIdx.y == 0) scored_check_offsets(p);
    int qb, first, len;
    prefill_find_block(p, R, blockIdx.x, lane, qb, first, len);
    if (qb < 0) return;                              // uniform over the CTA
    const int prefix = scored_prefix(p, first, len, lane), row0 = qb * R;
    const float *q = static_cast<const float *>(p.q), *k = static_cast<const float *>(p.k), *v = static_cast<const float *>(p.v);
    for (int x = threadIdx.x; x < R * D / 4; x += 256 * G) {
        const int r = x / (D / 4), c = x % (D / 4);
        const float4 val = row0 + r < len ? *reinterpret_cast<const float4 *>(q + (first + row0 + r) * p.q_stride + h * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
        *reinterpret_cast<float4 *>(Qs + r * QP + 4 * c) = val;
    }
    int lo = 0x7fffffff, hi = -1;                    // a thread below R looks after row tid
    if (tid < R && row0 + tid < len) scored_interval(p, first, prefix, row0 + tid, lo, hi);
    if (lo > hi) { lo = 0x7fffffff; hi = -1; }
    if (threadIdx.x < R) { rlo[tid] = lo; rhi[tid] = hi; }
    __syncthreads();
    // keys that any row sees, and that every live row sees
    int key0 = 0x7fffffff, key1 = -1, full0 = -1, full1 = 0x7fffffff;
    for (int x = lane; x < R; x += 32) {
        key0 = min(key0, rlo[x]); key1 = max(key1, rhi[x]);
        if (row0 + x < len) { full0 = max(full0, rlo[x]); full1 = min(full1, rhi[x]); }
    }
    key0 = __reduce_min_sync(0xffffffffu, key0); key1 = __reduce_max_sync(0xffffffffu, key1);
    full0 = __reduce_max_sync(0xffffffffu, full0); full1 = __reduce_min_sync(0xffffffffu, full1);
    const float slope = p.slopes ? p.slopes[h] : 0.f;
    int mylo[RPT], myhi[RPT];
    float m[RPT], l[RPT], o[RPT][CPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
        mylo[r] = rlo[ty * RPT + r]; myhi[r] = rhi[ty * RPT + r];
        m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
        for (int c = 0; c < CPT; ++c) o[r][c] = 0.f;
    }
    float4 kn[LD], vn[LD];                           // the next block on its way
    auto fetch = [&](int kb) {
#pragma unroll
        for (int x = 0; x < LD; ++x) {
            const int idx = tid + 256 * x, key = idx / (D / 4), c = idx % (D / 4);
            const bool in = kb + key <= key1;
            kn[x] = in ? *reinterpret_cast<const float4 *>(k + (first + kb + key) * p.k_stride + kvh * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
            vn[x] = in ? *reinterpret_cast<const float4 *>(v + (first + kb + key) * p.v_stride + kvh * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    const int start = key1 < 0 ? 0 : key0 + grp * KB;
    if (start <= key1) fetch(start);
    for (int kb = start; kb <= key1; kb += G * KB) {
        const bool hidden = !(full0 <= kb && kb + KB - 1 <= full1);     // some row does not see all of this block
        f32_group_sync<G>(grp);                      // the previous block's readers are done
        bool odd = false;
#pragma unroll
        for (int x = 0; x < LD; ++x) {
            const int idx = tid + 256 * x, key = idx / (D / 4), c = idx % (D / 4);
            *reinterpret_cast<float4 *>(Ks + key * QP + 4 * c) = kn[x];
            *reinterpret_cast<float4 *>(Vs + key * D + 4 * c) = vn[x];
            odd = odd || !(isfinite(vn[x].x) && isfinite(vn[x].y) && isfinite(vn[x].z) && isfinite(vn[x].w));
        }
        // 0 * NaN is NaN: where a hidden key's V row may not be finite, hidden keys are left out one by one
        const bool careful = f32_group_any<G>(grp, odd) && hidden;
        if (kb + G * KB <= key1) fetch(kb + G * KB);
        float s[RPT][KPT];
#pragma unroll
        for (int r = 0; r < RPT; ++r)
#pragma unroll
            for (int x = 0; x < KPT; ++x) s[r][x] = 0.f;
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
            float4 qv[RPT], kv[KPT];
#pragma unroll
            for (int r = 0; r < RPT; ++r) qv[r] = *reinterpret_cast<const float4 *>(Qs + (ty * RPT + r) * QP + d);
#pragma unroll
            for (int x = 0; x < KPT; ++x) kv[x] = *reinterpret_cast<const float4 *>(Ks + (tx + 16 * x) * QP + d);
#pragma unroll
            for (int r = 0; r < RPT; ++r)
#pragma unroll
                for (int x = 0; x < KPT; ++x) {
                    s[r][x] = fmaf(qv[r].x, kv[x].x, s[r][x]);
                    s[r][x] = fmaf(qv[r].y, kv[x].y, s[r][x]);
                    s[r][x] = fmaf(qv[r].z, kv[x].z, s[r][x]);
                    s[r][x] = fmaf(qv[r].w, kv[x].w, s[r][x]);
                }
        }
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            const int row = row0 + ty * RPT + r;
            float bm = -INFINITY;
#pragma unroll
            for (int x = 0; x < KPT; ++x) {
                const int t = kb + tx + 16 * x;
                float sc = s[r][x] * p.sm_scale;
                if (p.cap > 0.f) sc = p.cap * tanhf(sc / p.cap);
                sc = fmaf(-slope, fabsf(static_cast<float>(row - t)), sc);
                s[r][x] = (t >= mylo[r] && t <= myhi[r]) ? sc : -INFINITY;
                bm = fmaxf(bm, s[r][x]);
            }
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, d));
            const float m_new = fmaxf(m[r], bm), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = m[r] == -INFINITY ? 1.f : expf(m[r] - ref);      // nothing to scale yet
            m[r] = m_new;
            float ps = 0.f;
#pragma unroll
            for (int x = 0; x < KPT; ++x) {
                const float w = expf(s[r][x] - ref);
                ps += w;
                Ps[(ty * RPT + r) * PP + tx + 16 * x] = w;
            }
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, d);
            l[r] = l[r] * alpha + ps;
#pragma unroll
            for (int c = 0; c < CPT; ++c) o[r][c] *= alpha;
        }
        __syncwarp();                                // a row's 16 threads are in this warp
        if (!careful) {
#pragma unroll 2
            for (int y = 0; y < KB; y += 4) {
                float4 pv[RPT];
#pragma unroll
                for (int r = 0; r < RPT; ++r) pv[r] = *reinterpret_cast<const float4 *>(Ps + (ty * RPT + r) * PP + y);
#pragma unroll
                for (int z = 0; z < 4; ++z)
#pragma unroll
                    for (int c = 0; c < CPT; c += 4) {
                        const float4 vv = *reinterpret_cast<const float4 *>(Vs + (y + z) * D + 16 * c + 4 * tx);
#pragma unroll
                        for (int r = 0; r < RPT; ++r) {
                            const float w = z == 0 ? pv[r].x : z == 1 ? pv[r].y : z == 2 ? pv[r].z : pv[r].w;
                            o[r][c] = fmaf(w, vv.x, o[r][c]);
                            o[r][c + 1] = fmaf(w, vv.y, o[r][c + 1]);
                            o[r][c + 2] = fmaf(w, vv.z, o[r][c + 2]);
                            o[r][c + 3] = fmaf(w, vv.w, o[r][c + 3]);
                        }
                    }
            }
        } else {
            for (int y = 0; y < KB; ++y)
#pragma unroll
                for (int r = 0; r < RPT; ++r) {
                    if (kb + y < mylo[r] || kb + y > myhi[r]) continue;
                    const float w = Ps[(ty * RPT + r) * PP + y];
#pragma unroll
                    for (int c = 0; c < CPT; ++c) o[r][c] = fmaf(w, Vs[(y)*D + 16 * (c & ~3) + 4 * tx + (c & 3)], o[r][c]);
                }
        }
        __syncwarp();
    }
    if constexpr (G == 2) {                          // the second group's result into its tiles, and joined by the first
        __syncthreads();
        float *po = sm + R * QP + C::kGroupFloats, *pm = po + R * D, *pl = pm + R;
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            const int row = ty * RPT + r;
            if (grp == 1) {
#pragma unroll
                for (int c = 0; c < CPT; ++c) po[row * D + 16 * (c & ~3) + 4 * tx + (c & 3)] = o[r][c];
                if (tx == 0) { pm[row] = m[r]; pl[row] = l[r]; }
            }
        }
        __syncthreads();
        if (grp == 1) return;
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            const int row = ty * RPT + r;
            const float m1 = pm[row], l1 = pl[row], M = fmaxf(m[r], m1);
            // a side that saw nothing weighs nothing; one whose scores were all NaN has no maximum either, but a sum that is NaN
            const float a0 = m[r] == -INFINITY ? (l[r] != l[r] ? 1.f : 0.f) : expf(m[r] - M);
            const float a1 = m1 == -INFINITY ? (l1 != l1 ? 1.f : 0.f) : expf(m1 - M);
            l[r] = l[r] * a0 + l1 * a1;
#pragma unroll
            for (int c = 0; c < CPT; ++c) o[r][c] = o[r][c] * a0 + po[row * D + 16 * (c & ~3) + 4 * tx + (c & 3)] * a1;
        }
    }
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
        const int row = row0 + ty * RPT + r;
        if (row >= len) continue;
        const float inv = 1.f / l[r];                // l is 0 only where the row sees nothing; NaN among what it sees stays NaN
        const int64_t dst = (static_cast<int64_t>(first + row) * p.Hq + h) * D;
#pragma unroll
        for (int c = 0; c < CPT; c += 4) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = l[r] == 0.f ? 0.f : o[r][c + e] * inv;
            const int64_t at = dst + 16 * c + 4 * tx;
            if (p.out_bf16) *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(p.out) + at) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            else *reinterpret_cast<float4 *>(reinterpret_cast<float *>(p.out) + at) = make_float4(y[0], y[1], y[2], y[3]);
        }
    }
}

}  // namespace spd

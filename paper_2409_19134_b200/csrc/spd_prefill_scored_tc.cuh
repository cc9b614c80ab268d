// Prompt attention with capped scores, distance bias and interval masks on the fifth-generation tensor cores (bf16).
//
// One CTA has an SM to itself and owns two 128-row query tiles over shared K/V blocks of 80 keys: two query heads of one KV
// head over the same rows where the group is even (both tiles then need the same keys, and a short prompt still fills two
// tiles), else two consecutive row blocks of one head.  Per tile t:
//     S_t = Q_t K^T        128 x 80 x D, fp32 in TMEM
//     softmax              one row per thread: S_t into registers (S_t is free again at once), score options, mask,
//                          exponentials; P_t as bf16 pairs into TMEM columns of its own
//     O_t += P_t V         128 x D x 80, P read from TMEM
// Because P does not lie over S, S_t of the next block is computed while the exponentials of this one run, so that the
// softmax, which bounds the loop, never waits for the tensor core: with P over S and 128 keys per block it waited 1300 of
// 3300 cycles.  80 keys is what tensor memory holds that way at head_dim 128 (S 2 x 80, P 2 x 40, O 2 x 128 of 512 columns).
// A warp per tile issues that tile's MMAs (an MMA with both operands in shared memory is paced by the 128 bytes a cycle of
// those: 48 cycles for N = 64, 64 for N = 128, by measurement), another loads, a fourth guards.
//
// Masks are intervals [lo, hi] per row.  A CTA walks the blocks between the least lo and the greatest hi of its rows; a warp
// of the softmax masks only the blocks that its own 32 rows do not see whole, and skips those that they do not see at all.
// A hidden key's weight is 0, but 0 * NaN is NaN: the guard warp looks through the V rows of every block that some row does
// not see whole, clears rows that no row of the CTA sees, and where a row that is not finite is hidden from some rows and
// visible to others, the CTA's rows are done again one by one, hidden keys left out.
//
// Bound: the exponential unit (2 x 128 x 80 exponentials a block of two tiles at 16 a cycle: 1280 cycles) and the tensor core
// (about 1470) alike, with the FMA pipe close behind when scores are capped.
#pragma once

#include "spd_prefill_scored.cuh"

namespace spd {

constexpr int kStKeys = 80;                         // keys per block
constexpr int kStThreads = 384;                     // 8 softmax warps, 2 issuing, 1 loading, 1 guarding
constexpr int kStTmemCols = 512;
constexpr int kStS0 = 0, kStS1 = 96;                  // S of each tile (fp32, 80 columns)
constexpr int kStP0 = 176, kStP1 = 216;              // P (bf16 pairs, 40 columns)
constexpr int kStO0 = 256, kStO1 = 384;              // O (fp32, D columns)
constexpr int kStQBox = 128 * 128;                  // one swizzled TMA box of Q: 128 rows x 64 channels
constexpr int kStBox = kStKeys * 128;               // ... of K or V: 80 rows x 64 channels

__host__ __device__ constexpr int st_slots(int D) { return D == 128 ? 3 : 4; }
__host__ __device__ constexpr int st_qtile(int D) { return 128 * D * 2; }       // Q tile, bytes
__host__ __device__ constexpr int st_tile(int D) { return kStKeys * D * 2; }    // K or V tile
struct StBlockStats { int32_t minlo, maxhi, maxlo, minhi; };                    // over a warp's live rows
constexpr size_t st_smem_bytes(int D) {
    return 2 * static_cast<size_t>(st_qtile(D)) + 2 * st_slots(D) * static_cast<size_t>(st_tile(D)) + 256 + 256 * 8 + 8 * sizeof(StBlockStats) + 64;
}

struct ScoredTcParams {
    ScoredPrefillParams s;
    int32_t heads_per_cta;      // 2: tiles are two heads over the same rows; 1: two row blocks of one head
    float c2;                   // sm_scale log2(e)
    float cap2;                 // cap log2(e)
    float y1;                   // sm_scale / cap: what is inside the tanh per unit of q.k
    float half_at, one_at;      // where the two polynomials below end (1/2 and 1; -1 = not to be used)
    float p1[4], p2[6];         // cap2 tanh(y1 x) = x P(x^2): coefficients for |y1 x| <= 1/2 and <= 1
};

// tanh(y) = y P(y^2) by minimax polynomials (exchange algorithm, absolute error): 1.3e-7 for |y| <= 1/2, 2.4e-7 for |y| <= 1.
constexpr double kTanhHalf[4] = {0.999997676192732, -0.3332065521829639, 0.13145145657354904, -0.04337248370069227};
constexpr double kTanhOne[6] = {0.9999968538826182, -0.33324003808932323, 0.13253525346675044, -0.05097286522039006, 0.0161141828025398,
                                -0.0028394661823947912};

__device__ __forceinline__ void tmem_ld64_nowait(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16_nowait(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t *v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void tmem_st32p(uint32_t taddr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr),
          "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
          "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
          "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// The MMAs and the commit of a converged warp, issued by its elected lane (always the same one, so their order holds).
__device__ __forceinline__ void st_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void st_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void st_commit(uint32_t bar) {
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}

// cap2 tanh(y1 x) with the special-function unit: 1 - 2 / (e^2y + 1).
__device__ __forceinline__ float st_cap(const ScoredTcParams &p, float x) {
    return p.cap2 - __fdividef(2.f * p.cap2, ex2_approx(x * (2.f * kLog2e) * p.y1) + 1.f);
}

// One row the slow way, run by a whole warp: keys outside [lo, hi] are not touched.
template <int D>
__device__ __noinline__ void st_slow_row(const ScoredTcParams &p, int64_t first, int row, int h, int lo, int hi, int lane) {
    constexpr int V = D / 32;
    const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.s.q) + (first + row) * p.s.q_stride + h * D;
    const int kvh = h / (p.s.Hq / p.s.Hkv);
    const float slope = p.s.slopes ? p.s.slopes[h] : 0.f;
    float qv[V], o[V], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) { qv[i] = __bfloat162float(q[lane + 32 * i]); o[i] = 0.f; }
    for (int j = lo; j <= hi; ++j) {
        const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(p.s.k) + (first + j) * p.s.k_stride + kvh * D;
        const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(p.s.v) + (first + j) * p.s.v_stride + kvh * D;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) s = fmaf(qv[i], __bfloat162float(k[lane + 32 * i]), s);
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= p.s.sm_scale;
        if (p.s.cap > 0.f) s = p.s.cap * tanhf(s / p.s.cap);
        s = fmaf(-slope, fabsf(static_cast<float>(row - j)), s);
        const float m_new = fmaxf(m, s);
        const float alpha = m == -INFINITY ? 0.f : expf(m - m_new), w = expf(s - m_new);
        l = l * alpha + w;
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = fmaf(w, __bfloat162float(v[lane + 32 * i]), o[i] * alpha);
        m = m_new;
    }
    const int64_t dst = ((first + row) * p.s.Hq + h) * D;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float y = l == 0.f ? 0.f : o[i] / l;
        if (p.s.out_bf16) reinterpret_cast<__nv_bfloat16 *>(p.s.out)[dst + lane + 32 * i] = __float2bfloat16_rn(y);
        else reinterpret_cast<float *>(p.s.out)[dst + lane + 32 * i] = y;
    }
}

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kStThreads, 1)
prefill_scored_tc_kernel(const __grid_constant__ ScoredTcParams p, const __grid_constant__ CUtensorMap mq,
                         const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv) {
    constexpr int QTILE = st_qtile(D), TILE = st_tile(D), NS = st_slots(D), BOXES = D / 64, KB = kStKeys;
    extern __shared__ __align__(1024) uint8_t base[];
    const uint32_t Qs = smem_u32(base), Ks = Qs + 2 * QTILE, Vs = Ks + NS * TILE;
    uint8_t *tail = base + 2 * QTILE + 2 * NS * TILE;
    uint64_t *bars = reinterpret_cast<uint64_t *>(tail);
    uint64_t *bar_q = bars;                                        // Q loaded
    uint64_t *bar_s = bars + 1, *bar_sf = bars + 3;                // per tile: S ready; S in registers
    uint64_t *bar_p = bars + 5, *bar_o = bars + 7;                 // per tile: P written; O has taken the block in (P is free)
    uint64_t *bar_k = bars + 9, *bar_v = bar_k + NS, *bar_kfree = bar_v + NS, *bar_vfree = bar_kfree + NS;
    uint64_t *bar_guard = bar_vfree + NS;                          // per V slot: the guard is done with the block
    constexpr int NBARS = 9 + 5 * NS;
    static_assert(NBARS * 8 + 8 <= 256, "barrier block");
    uint32_t &tmem_slot = *reinterpret_cast<uint32_t *>(tail + NBARS * 8);
    volatile int32_t &poisoned = *reinterpret_cast<int32_t *>(tail + NBARS * 8 + 4);
    int2 *span = reinterpret_cast<int2 *>(tail + 256);             // [tile][row]: first and last key the row sees
    StBlockStats *stats = reinterpret_cast<StBlockStats *>(tail + 256 + 256 * 8);   // per softmax warp
    const int tid = threadIdx.x, wid = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int hpc = p.heads_per_cta, h0 = blockIdx.y * hpc, kvh = h0 / (p.s.Hq / p.s.Hkv);
    const int rows_cta = hpc == 2 ? 128 : 256;

    if (blockIdx.x == 0 && blockIdx.y == 0) scored_check_offsets(p.s);
    if (tid == 320) { prefetch_tensormap(&mq); prefetch_tensormap(&mk); prefetch_tensormap(&mv); }
    int qb, first, len;
    prefill_find_block(p.s, rows_cta, blockIdx.x, lane, qb, first, len);
    if (qb < 0) return;   // uniform over the CTA: no barrier, no TMEM touched yet
    const int row0 = qb * rows_cta;
    // tile t: head h0 + t over rows row0 .., or head h0 over rows row0 + 128 t ..; the second may lie past the prompt's end
    const int tiles = (hpc == 2 || row0 + 128 < len) ? 2 : 1;

    if (tid == 320) {     // the loading thread sets the barriers up and asks for Q before anything else happens
        for (int b = 0; b < NBARS; ++b)     // S in registers, P written: one arrival per softmax warp of the tile; slot free: one per tile
            mbar_init(smem_u32(&bars[b]), (b >= 3 && b < 7) ? 4 : (b >= 9 + 2 * NS && b < 9 + 4 * NS) ? 2 : 1);
        fence_mbar_init();
        fence_proxy_async();
        mbar_expect_tx(smem_u32(bar_q), tiles * QTILE);
        for (int t = 0; t < tiles; ++t)
            for (int x = 0; x < BOXES; ++x)
                tma_load_3d(Qs + t * QTILE + x * kStQBox, &mq, 64 * x, hpc == 2 ? h0 + t : h0, first + row0 + (hpc == 2 ? 0 : 128 * t), smem_u32(bar_q));
    }
    // ---- what each row sees; a softmax thread is one row
    const int t = (wid >> 2) & 1, row = tid & 127;                  // tile and row of a softmax thread
    const int qrow = row0 + (hpc == 2 ? 0 : 128 * t) + row;         // within the prompt
    int lo = 0x7fffffff, hi = -1;
    if (wid < 8) {
        const bool live = t < tiles && qrow < len;
        const int prefix = scored_prefix(p.s, first, len, lane);
        if (live) scored_interval(p.s, first, prefix, qrow, lo, hi);
        const bool sees = lo <= hi;
        if (!sees) { lo = 0x7fffffff; hi = -1; }
        span[tid] = make_int2(lo, hi);
        // a live row that sees nothing makes every block one with hidden keys
        int a = lo, b = hi, c = sees ? lo : (live ? 0x7fffffff : -1), d = sees ? hi : (live ? -1 : 0x7fffffff);
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) {
            a = min(a, __shfl_xor_sync(0xffffffffu, a, x));
            b = max(b, __shfl_xor_sync(0xffffffffu, b, x));
            c = max(c, __shfl_xor_sync(0xffffffffu, c, x));
            d = min(d, __shfl_xor_sync(0xffffffffu, d, x));
        }
        if (lane == 0) stats[wid] = StBlockStats{a, b, c, d};
    }
    if (wid == 8) {       // one warp allocates all of tensor memory for the CTA (it has the SM to itself)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kStTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) poisoned = 0;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    int tlo[2], thi[2], fullhi = 0x7fffffff, fulllo = -1;           // keys that a tile sees; [fulllo, fullhi]: that every row sees
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        tlo[x] = 0x7fffffff; thi[x] = -1;
        for (int w = 4 * x; w < 4 * x + 4; ++w) {
            tlo[x] = min(tlo[x], stats[w].minlo); thi[x] = max(thi[x], stats[w].maxhi);
            fulllo = max(fulllo, stats[w].maxlo); fullhi = min(fullhi, stats[w].minhi);
        }
    }
    const int key0 = min(tlo[0], tlo[1]), key1 = max(thi[0], thi[1]);
    const int NB = key1 < 0 ? 0 : (key1 - key0) / KB + 1;
    int ja[2], jb[2];                                                // blocks that a tile works on, [ja, jb)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        ja[x] = thi[x] < 0 ? 0 : (tlo[x] - key0) / KB;
        jb[x] = thi[x] < 0 ? 0 : (thi[x] - key0) / KB + 1;
    }
    const int my_a = t ? ja[1] : ja[0], my_b = t ? jb[1] : jb[0];    // ... and those of a softmax thread's tile
    auto guarded = [&](int j) { return !(fulllo <= key0 + j * KB && key0 + j * KB + KB - 1 <= fullhi); };

    // Every wait is bounded.  A wait that runs out clears `ok` and the thread carries on (with garbage, but towards the
    // same end): nothing in the loops waits for all threads, so nobody can be left behind.
    bool ok = true;
    float l = 0.f;
    const uint32_t lanes = static_cast<uint32_t>((wid & 3) * 32) << 16;                             // a softmax warp's lanes
    const uint32_t t_s = tmem + lanes + (t ? kStS1 : kStS0), t_p = tmem + lanes + (t ? kStP1 : kStP0);
    const uint32_t t_o = tmem + lanes + (t ? kStO1 : kStO0);

    if (wid < 8) {
        if (my_b > my_a) {
        // ---------------- softmax warps: one query row per thread
        float m = -INFINITY;                           // reference point in log2 units of the score
        const StBlockStats w = stats[wid];
        float slope2 = 0.f;
        if constexpr (BIAS) slope2 = p.s.slopes[hpc == 2 ? h0 + t : h0] * kLog2e;
        for (int j = my_a; j < my_b; ++j) {
            const int i = j - my_a, kb = key0 + j * KB;
            ok = mbar_wait(smem_u32(&bar_s[t]), i & 1) && ok;
            tc_fence_after();
            if (w.maxhi < kb || w.minlo >= kb + KB) {     // nobody in this warp sees any of it: weights 0
                uint32_t z[32];
#pragma unroll
                for (int x = 0; x < 32; ++x) z[x] = 0u;
                if (lane == 0) mbar_arrive(smem_u32(&bar_sf[t]));
                if (i > 0) ok = mbar_wait(smem_u32(&bar_o[t]), (i - 1) & 1) && ok;
                tc_fence_after();
                tmem_st32p(t_p, z);
                tmem_st8(t_p + 32, z);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_p[t]));
                continue;
            }
            uint32_t raw[KB];
            tmem_ld64_nowait(t_s, raw);
            tmem_ld16_nowait(t_s + 64, raw + 64);
            tmem_wait_ld();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_sf[t]));       // the next block's S may be computed
            float sv[KB];
#pragma unroll
            for (int x = 0; x < KB; ++x) sv[x] = __uint_as_float(raw[x]);
            const bool masked = !(w.maxlo <= kb && kb + KB - 1 <= w.minhi);       // warp-uniform
            uint32_t see[3] = {0xffffffffu, 0xffffffffu, 0xffffffffu};
            if (masked) {
#pragma unroll
                for (int x = 0; x < 3; ++x) {
                    const int a = max(lo - kb - 32 * x, 0), b = min(hi - kb - 32 * x, 31);
                    see[x] = (a > b || a > 31 || b < 0) ? 0u : (0xffffffffu << a) & (0xffffffffu >> (31 - b));
                }
            }
            auto seen = [&](int x) { return (see[x >> 5] >> (x & 31)) & 1u; };
            // ---- score options.  Afterwards sv holds the score in log2 units (BIAS), or still q.k with the cap (CAP) or the
            // scale applied on the way to the exponential.
            constexpr int L = KB / 4;                   // extrema run in four chains
            bool poly1 = false, poly2 = false;          // warp-uniform: the cap's polynomials hold for every score here
            float mx, mn = 0.f;
            if constexpr (CAP) {
                if (!masked) {                          // (a masked block takes the exact form: hidden scores may be anything)
                    float a4[4], b4[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        a4[c] = fmax3(sv[L * c], sv[L * c + 1], sv[L * c + 2]);
                        b4[c] = fminf(fminf(sv[L * c], sv[L * c + 1]), sv[L * c + 2]);
#pragma unroll
                        for (int x = 3; x < L - 1; x += 2) {
                            a4[c] = fmax3(a4[c], sv[L * c + x], sv[L * c + x + 1]);
                            b4[c] = fminf(fminf(b4[c], sv[L * c + x]), sv[L * c + x + 1]);
                        }
                        a4[c] = fmaxf(a4[c], sv[L * c + L - 1]);
                        b4[c] = fminf(b4[c], sv[L * c + L - 1]);
                    }
                    mx = fmaxf(fmaxf(a4[0], a4[1]), fmaxf(a4[2], a4[3]));
                    mn = fminf(fminf(b4[0], b4[1]), fminf(b4[2], b4[3]));
                    const float big = fmaxf(mx, -mn) * p.y1;
                    poly1 = __all_sync(0xffffffffu, big <= p.half_at);
                    poly2 = !poly1 && __all_sync(0xffffffffu, big <= p.one_at);
                }
            }
            if constexpr (BIAS) {
                if constexpr (CAP) {
                    if (poly1 || poly2) {
#pragma unroll
                        for (int x = 0; x < KB; x += 2) {
                            const uint64_t s2 = pack_f32x2(sv[x], sv[x + 1]), y = mul_f32x2(s2, s2);
                            uint64_t q;
                            if (poly1) {
                                q = fma_f32x2(y, pack_f32x2(p.p1[3], p.p1[3]), pack_f32x2(p.p1[2], p.p1[2]));
                                q = fma_f32x2(q, y, pack_f32x2(p.p1[1], p.p1[1]));
                                q = fma_f32x2(q, y, pack_f32x2(p.p1[0], p.p1[0]));
                            } else {
                                q = fma_f32x2(y, pack_f32x2(p.p2[5], p.p2[5]), pack_f32x2(p.p2[4], p.p2[4]));
                                q = fma_f32x2(q, y, pack_f32x2(p.p2[3], p.p2[3]));
                                q = fma_f32x2(q, y, pack_f32x2(p.p2[2], p.p2[2]));
                                q = fma_f32x2(q, y, pack_f32x2(p.p2[1], p.p2[1]));
                                q = fma_f32x2(q, y, pack_f32x2(p.p2[0], p.p2[0]));
                            }
                            unpack_f32x2(mul_f32x2(q, s2), sv[x], sv[x + 1]);
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < KB; ++x) sv[x] = st_cap(p, sv[x]);
                    }
                }
                const float scale = CAP ? 1.f : p.c2;
                const uint64_t sc2 = pack_f32x2(scale, scale);
                if (kb + KB - 1 <= qrow - row || kb >= qrow - row + 127) {      // the block lies on one side of the tile's rows
                    const float st = kb >= qrow - row + 127 ? -slope2 : slope2, b0 = -slope2 * fabsf(static_cast<float>(qrow - kb));
                    const uint64_t st2 = pack_f32x2(st, st), b2 = pack_f32x2(b0, b0);
#pragma unroll
                    for (int x = 0; x < KB; x += 2)
                        unpack_f32x2(fma_f32x2(pack_f32x2(sv[x], sv[x + 1]), sc2,
                                               fma_f32x2(pack_f32x2(static_cast<float>(x), static_cast<float>(x + 1)), st2, b2)), sv[x], sv[x + 1]);
                } else {
                    const float off = static_cast<float>(kb - qrow);
#pragma unroll
                    for (int x = 0; x < KB; ++x) sv[x] = fmaf(sv[x], scale, -slope2 * fabsf(static_cast<float>(x) + off));
                }
            }
            if (masked) {
#pragma unroll
                for (int x = 0; x < KB; ++x) sv[x] = seen(x) ? sv[x] : -INFINITY;
            }
            if (!CAP || BIAS || masked) {
                float r4[4];                             // four chains of three-input maxima
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    r4[c] = fmax3(sv[L * c], sv[L * c + 1], sv[L * c + 2]);
#pragma unroll
                    for (int x = 3; x < L - 1; x += 2) r4[c] = fmax3(r4[c], sv[L * c + x], sv[L * c + x + 1]);
                    r4[c] = fmaxf(r4[c], sv[L * c + L - 1]);
                }
                mx = fmaxf(fmax3(r4[0], r4[1], r4[2]), r4[3]);
            }
            // the reference moves only when the block's maximum lies more than kPfSlack above it, so that O is hardly
            // ever rescaled; a row that has seen nothing yet keeps -inf
            float xmax;
            if constexpr (BIAS) xmax = mx;
            else if constexpr (CAP) xmax = mx == -INFINITY ? -INFINITY : st_cap(p, mx);
            else xmax = mx * p.c2;
            const float m_new = (xmax > m + kPfSlack) ? xmax : m;
            const float ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = m == -INFINITY ? 1.f : ex2_approx(m - m_new);
            l *= alpha;
            m = m_new;
            bool o_ready = i == 0;                       // O has taken the block before in
            if (i > 0 && !__all_sync(0xffffffffu, alpha == 1.f)) {
                ok = mbar_wait(smem_u32(&bar_o[t]), (i - 1) & 1) && ok;
                o_ready = true;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    float ov[32];
                    tmem_ld32(t_o + c * 32, ov);
#pragma unroll
                    for (int x = 0; x < 32; ++x) ov[x] *= alpha;
                    tmem_st32(t_o + c * 32, ov);
                }
            }
            const uint64_t mx2 = pack_f32x2(-ref, -ref);
            uint64_t lsum2 = 0;                          // two partial row sums, (+0, +0)
            uint32_t pk[KB / 2];
            {
                auto weights = [&](auto &&arg) {         // arg(x): scores x, x + 1 in log2 units, relative to the reference
#pragma unroll
                    for (int y = 0; y < KB / 2; ++y) {
                        float a0, a1;
                        unpack_f32x2(arg(2 * y), a0, a1);
                        const float p0 = ex2_approx(a0), p1 = ex2_approx(a1);
                        lsum2 = add_f32x2(lsum2, pack_f32x2(p0, p1));
                        pk[y] = pack_bf16(p0, p1);
                    }
                };
                if constexpr (BIAS) {
                    weights([&](int x) { return add_f32x2(pack_f32x2(sv[x], sv[x + 1]), mx2); });
                } else if constexpr (!CAP) {
                    const uint64_t c22 = pack_f32x2(p.c2, p.c2);
                    weights([&](int x) { return fma_f32x2(pack_f32x2(sv[x], sv[x + 1]), c22, mx2); });
                } else if (poly1) {
                    weights([&](int x) {
                        const uint64_t s2 = pack_f32x2(sv[x], sv[x + 1]), y = mul_f32x2(s2, s2);
                        uint64_t q = fma_f32x2(y, pack_f32x2(p.p1[3], p.p1[3]), pack_f32x2(p.p1[2], p.p1[2]));
                        q = fma_f32x2(q, y, pack_f32x2(p.p1[1], p.p1[1]));
                        q = fma_f32x2(q, y, pack_f32x2(p.p1[0], p.p1[0]));
                        return fma_f32x2(q, s2, mx2);
                    });
                } else if (poly2) {
                    weights([&](int x) {
                        const uint64_t s2 = pack_f32x2(sv[x], sv[x + 1]), y = mul_f32x2(s2, s2);
                        uint64_t q = fma_f32x2(y, pack_f32x2(p.p2[5], p.p2[5]), pack_f32x2(p.p2[4], p.p2[4]));
                        q = fma_f32x2(q, y, pack_f32x2(p.p2[3], p.p2[3]));
                        q = fma_f32x2(q, y, pack_f32x2(p.p2[2], p.p2[2]));
                        q = fma_f32x2(q, y, pack_f32x2(p.p2[1], p.p2[1]));
                        q = fma_f32x2(q, y, pack_f32x2(p.p2[0], p.p2[0]));
                        return fma_f32x2(q, s2, mx2);
                    });
                } else {
                    weights([&](int x) {
                        const float a0 = sv[x] == -INFINITY ? -INFINITY : st_cap(p, sv[x]) - ref;
                        const float a1 = sv[x + 1] == -INFINITY ? -INFINITY : st_cap(p, sv[x + 1]) - ref;
                        return pack_f32x2(a0, a1);
                    });
                }
            }
            if (!o_ready) ok = mbar_wait(smem_u32(&bar_o[t]), (i - 1) & 1) && ok;      // P of the block before has been read
            tc_fence_after();
            tmem_st32p(t_p, pk);
            tmem_st8(t_p + 32, pk + 32);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();                                 // one arrival per warp
            if (lane == 0) mbar_arrive(smem_u32(&bar_p[t]));
            float s0, s1;
            unpack_f32x2(lsum2, s0, s1);
            l += s0 + s1;
        }
        ok = mbar_wait(smem_u32(&bar_o[t]), (my_b - my_a - 1) & 1) && ok;
    }
    } else if (wid == 10) {
        // ---------------- the loading thread
        if (lane == 0) {
            for (int j = 0; j < NB; ++j) {
                const int slot = j % NS, y = first + key0 + j * KB;
                if (j >= NS) ok = mbar_wait(smem_u32(&bar_kfree[slot]), (j / NS - 1) & 1) && ok;
                mbar_expect_tx(smem_u32(&bar_k[slot]), TILE);
                for (int x = 0; x < BOXES; ++x) tma_load_3d(Ks + slot * TILE + x * kStBox, &mk, 64 * x, kvh, y, smem_u32(&bar_k[slot]));
                if (j >= NS) ok = mbar_wait(smem_u32(&bar_vfree[slot]), (j / NS - 1) & 1) && ok;
                mbar_expect_tx(smem_u32(&bar_v[slot]), TILE);
                for (int x = 0; x < BOXES; ++x) tma_load_3d(Vs + slot * TILE + x * kStBox, &mv, 64 * x, kvh, y, smem_u32(&bar_v[slot]));
            }
        }
    } else if (wid == 11) {
        // ---------------- the guard: V rows of blocks with hidden keys
        for (int j = 0; j < NB; ++j) {
            // every block passes through here, so that the guard is never a whole ring ahead of or behind the others
            const int slot = j % NS;
            ok = mbar_wait(smem_u32(&bar_v[slot]), (j / NS) & 1) && ok;
            __syncwarp();
            if (!guarded(j)) {
                if (lane == 0) mbar_arrive(smem_u32(&bar_guard[slot]));
                continue;
            }
            uint8_t *vt = base + 2 * QTILE + (NS + slot) * TILE;
            auto odd = [](const uint4 &w) {           // a 16-bit half with all exponent bits set carries into its sign bit
                return ((w.x & 0x7f807f80u) + 0x00800080u) | ((w.y & 0x7f807f80u) + 0x00800080u) | ((w.z & 0x7f807f80u) + 0x00800080u) |
                       ((w.w & 0x7f807f80u) + 0x00800080u);
            };
            uint32_t any = 0;
#pragma unroll 5
            for (int c = lane; c < TILE / 16; c += 32) any |= odd(*reinterpret_cast<const uint4 *>(vt + c * 16));
            if (__any_sync(0xffffffffu, (any & 0x80008000u) != 0)) {
                for (int r = 0; r < KB; ++r) {        // rare: row by row
                    uint4 *chunk = reinterpret_cast<uint4 *>(vt + (lane >> 3) * kStBox + r * 128 + (lane & 7) * 16);
                    const bool mine = lane < 8 * BOXES;
                    if (!__any_sync(0xffffffffu, mine && (odd(*(mine ? chunk : reinterpret_cast<uint4 *>(vt + r * 128))) & 0x80008000u) != 0)) continue;
                    const int key = key0 + j * KB + r;
                    bool seen = false, hidden = false;
                    for (int x = lane; x < 256; x += 32) {
                        const int2 sp = span[x];
                        const bool s = sp.x <= key && key <= sp.y;
                        seen = seen || s;
                        hidden = hidden || !s;
                    }
                    if (!__any_sync(0xffffffffu, seen)) {
                        if (mine) *chunk = make_uint4(0, 0, 0, 0);
                    } else if (__any_sync(0xffffffffu, hidden)) {
                        poisoned = 1;
                    }
                }
                fence_proxy_async();
                __syncwarp();
            }
            if (lane == 0) mbar_arrive(smem_u32(&bar_guard[slot]));
        }
    } else {
        // ---------------- the warp that issues tile x's MMAs: S of block j, then P V of block j - 1
        const int x = wid - 8;
        const int a = x ? ja[1] : ja[0], b = x ? jb[1] : jb[0];
        const uint32_t ts = tmem + (x ? kStS1 : kStS0), tp = tmem + (x ? kStP1 : kStP0), to = tmem + (x ? kStO1 : kStO0);
        ok = mbar_wait(smem_u32(bar_q), 0);           // always: nothing may be in flight when the CTA ends
        for (int j = 0; j <= NB; ++j) {
            if (j < NB) {
                const int slot = j % NS;
                // a tile that has no use for a block gives it back all the same, once it is there: never a ring ahead
                ok = mbar_wait(smem_u32(&bar_k[slot]), (j / NS) & 1) && ok;
                if (a <= j && j < b) {
                    const int i = j - a;
                    if (i > 0) ok = mbar_wait(smem_u32(&bar_sf[x]), (i - 1) & 1) && ok;
                    __syncwarp();
                    tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)       // 16 channels per MMA
                        st_mma_ss(ts, umma_desc(Qs + x * QTILE + (kk >> 2) * kStQBox + (kk & 3) * 32, 16, 1024),
                                  umma_desc(Ks + slot * TILE + (kk >> 2) * kStBox + (kk & 3) * 32, 16, 1024), umma_idesc(false, KB), kk > 0 ? 1u : 0u);
                    st_commit(smem_u32(&bar_s[x]));
                    st_commit(smem_u32(&bar_kfree[slot]));
                } else if (lane == 0) {
                    mbar_arrive(smem_u32(&bar_kfree[slot]));
                }
            }
            if (j > 0) {
                const int jj = j - 1, slot = jj % NS;
                ok = mbar_wait(smem_u32(&bar_v[slot]), (jj / NS) & 1) && ok;
                ok = mbar_wait(smem_u32(&bar_guard[slot]), (jj / NS) & 1) && ok;
                if (a <= jj && jj < b) {
                    const int i = jj - a;
                    ok = mbar_wait(smem_u32(&bar_p[x]), i & 1) && ok;
                    __syncwarp();
                    tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < KB / 16; ++kk)      // 16 keys per MMA: 8 columns of P, 2 KB of each 64-channel box of V
                        st_mma_ts(to, tp + kk * 8, umma_desc(Vs + slot * TILE + kk * 2048, kStBox, 1024), umma_idesc(true, D), (i > 0 || kk > 0) ? 1u : 0u);
                    st_commit(smem_u32(&bar_o[x]));
                    st_commit(smem_u32(&bar_vfree[slot]));
                } else if (lane == 0) {
                    mbar_arrive(smem_u32(&bar_vfree[slot]));
                }
            }
        }
    }
    tc_fence_after();
    const bool gave_up = !__syncthreads_and(ok);
    if (gave_up) {
        if (tid == 0) flag_error(p.s.hdr, 6 /* SPD_ERR_TIMEOUT */, -1);
    } else if (poisoned) {
        if (wid < 8)
            for (int r = 32 * wid; r < 32 * wid + 32; ++r) {             // the warp's own rows, one by one
                const int tt = r >> 7, rr = row0 + (hpc == 2 ? 0 : 128 * tt) + (r & 127);
                if (tt < tiles && rr < len) st_slow_row<D>(p, first, rr, hpc == 2 ? h0 + tt : h0, span[r].x, span[r].y, lane);
            }
    } else if (wid < 8 && t < tiles) {
        // ---- normalise this thread's row into shared memory (the tile's own Q is free: its MMAs are done), 256 bytes of a
        //      row at a time, then each warp stores its own 32 rows; 16-byte chunks are XOR-swizzled by the row against
        //      bank conflicts; rows past the prompt's end are not stored.  A row that saw nothing (l = 0) gives zeros.
        const bool none = my_b <= my_a;
        const float inv = (none || l == 0.f) ? 0.f : 1.f / l;
        constexpr int PASS = D == 128 ? 256 : 128;               // bytes of a row per pass
        uint8_t *stage = base + t * QTILE;                        // 128 rows x PASS bytes
        const int rows_live = len - (qrow - row) - (wid & 3) * 32;      // rows of this warp that belong to the prompt
        const int64_t tok0 = static_cast<int64_t>(first) + (qrow - row) + (wid & 3) * 32;
        const int h = hpc == 2 ? h0 + t : h0;
        uint8_t *dst = reinterpret_cast<uint8_t *>(p.s.out);
        const int passes = p.s.out_bf16 ? 1 : 2, row_bytes = p.s.out_bf16 ? 2 * D : 4 * D;
        constexpr int CPR = PASS / 16;                            // 16-byte chunks per row and pass
#pragma unroll 1
        for (int pass = 0; pass < passes; ++pass) {               // fp32: channels [D / 2 pass, D / 2 pass + D / 2)
            const int cols = p.s.out_bf16 ? D / 32 : D / 64;
#pragma unroll 1
            for (int c = 0; c < cols; ++c) {
                float ov[32];
                tmem_ld32(t_o + pass * (D / 2) + c * 32, ov);
#pragma unroll
                for (int x = 0; x < 32; ++x) ov[x] = inv == 0.f ? 0.f : ov[x] * inv;
                if (p.s.out_bf16) {
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4)
                        *reinterpret_cast<uint4 *>(stage + row * PASS + (((c * 4 + q4) ^ (row & 7)) << 4)) =
                            make_uint4(pack_bf16(ov[8 * q4], ov[8 * q4 + 1]), pack_bf16(ov[8 * q4 + 2], ov[8 * q4 + 3]),
                                       pack_bf16(ov[8 * q4 + 4], ov[8 * q4 + 5]), pack_bf16(ov[8 * q4 + 6], ov[8 * q4 + 7]));
                } else {
#pragma unroll
                    for (int q4 = 0; q4 < 8; ++q4)
                        *reinterpret_cast<float4 *>(stage + row * PASS + (((c * 8 + q4) ^ (row & 7)) << 4)) =
                            make_float4(ov[4 * q4], ov[4 * q4 + 1], ov[4 * q4 + 2], ov[4 * q4 + 3]);
                }
            }
            __syncwarp();
            for (int x = lane; x < 32 * CPR; x += 32) {
                const int r = x / CPR, ch = x % CPR, rr = (wid & 3) * 32 + r;
                if (r < rows_live)
                    *reinterpret_cast<uint4 *>(dst + ((tok0 + r) * p.s.Hq + h) * row_bytes + pass * PASS + ch * 16) =
                        *reinterpret_cast<const uint4 *>(stage + rr * PASS + ((ch ^ (rr & 7)) << 4));
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (wid == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kStTmemCols) : "memory");
}

}  // namespace spd

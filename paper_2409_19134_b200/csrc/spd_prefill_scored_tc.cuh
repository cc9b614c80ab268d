// Prompt attention with capped scores, distance bias and interval masks on the fifth-generation tensor cores (bf16).
//
// One CTA per SM works through a list of items, each two 128-row query tiles over shared K/V blocks of 80 keys: two query
// heads of one KV head over the same rows where the group is even (both tiles then need the same keys, and a short prompt
// still fills two tiles), else two consecutive row blocks of one head.  Items are numbered heaviest first within a prompt and
// drawn from a counter; a planning warp works out the next item while this one runs, and its Q, K and V are on the way before
// this one's output is written (a CTA per item spent 8 to 10 us starting and ending).  Per tile t:
//     S_t = Q_t K^T        128 x 80 x D, fp32 in TMEM
//     softmax              one row per thread: S_t into registers (S_t is free again at once), score options, mask,
//                          exponentials; P_t as bf16 pairs into TMEM columns of its own
//     O_t += P_t V         128 x D x 80, P read from TMEM
// Because P does not lie over S, S_t of the next block is computed while the exponentials of this one run, so that the
// softmax, which bounds the loop, never waits for the tensor core: with P over S and 128 keys per block it waited 1300 of
// 3300 cycles.  80 keys is what tensor memory holds that way at head_dim 128 (S 2 x 80, P 2 x 40, O 2 x 128 of 512 columns).
// A warp per tile issues that tile's MMAs (an MMA with both operands in shared memory is paced by the 128 bytes a cycle of
// those: 48 cycles for N = 64, 64 for N = 128, by measurement), another loads, one plans, four guard.
//
// Masks are intervals [lo, hi] per row.  A CTA walks the blocks between the least lo and the greatest hi of its rows; a warp
// of the softmax masks only the blocks that its own 32 rows do not see whole, and skips those that they do not see at all.
// A hidden key's weight is 0, but 0 * NaN is NaN: guard warps look through the V rows of every block that some row does not see
// whole, clear rows that no row of the CTA sees, and where a row that is not finite is hidden from some rows and
// visible to others, the CTA's rows are done again one by one, hidden keys left out.
//
// Bound: the exponential unit (2 x 128 x 80 exponentials a block of two tiles at 16 a cycle: 1280 cycles) and the tensor core
// (about 1470) alike, of about 2000 that a block takes (each pipe two thirds busy).  With a cap a block takes about 2700, with a distance bias
// 2400, and no pipe is busy for more than half of it: what they add stands in a row's chain between a score's arrival and its
// weight, on top of the exponentials instead of beside them.  Over seconds the power limit (8192 tokens, 32/8 heads: 446 us in the
// first 100 calls, 514 at 1590 MHz and 990 W after three seconds).  Measured on one GPU, back to back, head_dim 128, bf16: 8192 tokens
// x 32/8 heads plain 445 us (1236 TFLOP/s of visible pairs), distance bias 539 (1020), cap of 50 610 (900; 552 in a first burst), of
// 64 700; 8 prompts of 2 to 8 k tokens (50 572 in all) 2.24 ms (1220); 3 prompts with prefix and window 126 us (900).
// Slower here: the tiles' exponentials in turns by named barriers (20 %), two threads per row (instruction issue, 15 %), the next
// block's scores prepared in registers under this block's exponentials (60 %; the compiler serialises them), barriers of its own for
// each tile's Q, which lets the tiles drift apart (4 % with caps).
#pragma once

#include "spd_prefill_scored.cuh"

namespace spd {

constexpr int kStKeys = 80;                         // keys per block
constexpr int kStThreads = 512;                     // 8 softmax warps, 2 issuing, 1 loading, 1 planning, 4 guarding
constexpr int kStConsumers = 15;                    // warps that read a plan
constexpr int kStTmemCols = 512;
constexpr float kStFixedCap = 50.f;                 // caps up to here: weights relative to 0 (50 log2(e) = 72.2)
constexpr int kStS0 = 0, kStS1 = 96;                  // S of each tile (fp32, 80 columns)
constexpr int kStP0 = 176, kStP1 = 216;              // P (bf16 pairs, 40 columns)
constexpr int kStO0 = 256, kStO1 = 384;              // O (fp32, D columns)
constexpr int kStQBox = 128 * 128;                  // one swizzled TMA box of Q: 128 rows x 64 channels
constexpr int kStBox = kStKeys * 128;               // ... of K or V: 80 rows x 64 channels

__host__ __device__ constexpr int st_slots(int D) { return D == 128 ? 3 : 4; }
__host__ __device__ constexpr int st_qtile(int D) { return 128 * D * 2; }       // Q tile, bytes
__host__ __device__ constexpr int st_tile(int D) { return kStKeys * D * 2; }    // K or V tile
struct StBlockStats { int32_t minlo, maxhi, maxlo, minhi; };                    // over a warp's live rows
// One item as the planning warp lays it out in shared memory; two of them, so that the next is ready early.
struct StPlan {
    int32_t valid;                  // 0: the list is done
    int32_t first, len, row0, h0;   // prompt (first token, tokens), first row of the item, first head
    int32_t tiles;                  // tiles with rows of the prompt
    int32_t kend, nb;               // first key of the last block, blocks; they are worked through from the last to the first
    int32_t ja[2], jb[2];           // blocks that a tile works on, [ja, jb) in that order
    int32_t fulllo, fullhi;         // keys that every row sees
    int32_t poisoned;               // a V row that is not finite is hidden from some rows and visible to others
    int32_t ahead;                  // some row sees keys ahead of it (a prefix)
    float slope2[2];                // distance bias of each tile's head, log2 units
    alignas(16) float bias[2][kStKeys];     // ... of the keys of a block: slope x
    StBlockStats stats[8];          // per softmax warp
    int2 span[256];                 // [tile][row]: first and last key the row sees
};
constexpr int kStBarBytes = 320;
constexpr int kStStage = 4096;      // bytes per softmax warp for its way out: 32 rows x 32 fp32
constexpr size_t st_smem_bytes(int D) {
    return 2 * static_cast<size_t>(st_qtile(D)) + 2 * st_slots(D) * static_cast<size_t>(st_tile(D)) + 8 * kStStage + kStBarBytes + 2 * sizeof(StPlan);
}
static_assert(st_smem_bytes(128) <= 232448, "shared memory of an SM");

// Polls before a wait gives up.  Beyond the usual limit 512 per token of the call: a tile whose rows are done one by one takes its warps
// 4 us per key (in L2; more where K and V are not), and a poll takes 0.1 us beside such warps (1.5 us where nothing moves), by
// measurement.  (A limit that starts anew while such rows make progress costs the ordinary call 2 to 4 %.)
inline uint32_t st_wait_limit(int64_t tokens) {
    const int64_t polls = static_cast<int64_t>(kWaitLimit) + 512 * tokens;
    return polls > 0xffffffffll ? 0xffffffffu : static_cast<uint32_t>(polls);
}

struct ScoredTcParams {
    ScoredPrefillParams s;
    int32_t heads_per_cta;      // 2: tiles are two heads over the same rows; 1: two row blocks of one head
    float c2;                   // sm_scale log2(e)
    float cap2;                 // cap log2(e)
    uint32_t wait_limit;        // polls before a wait gives up
    float y1;                   // sm_scale / cap: what is inside the tanh per unit of q.k
    float half_at, one_at;      // where the two polynomials below end (1/2 and 1; -1 = not to be used)
    uint64_t p1[4], p2[6];      // coefficients for |y1 x| <= 1/2 and <= 1, each in both halves.  CAP 1: of cap2 tanh(y1 x) = x P(x^2);
                                // CAP 2: of tanh(y) = y P(y^2), whatever the cap, for scores that were multiplied by y1
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

// Three-input maximum of magnitudes.
__device__ __forceinline__ float fmax3_abs(float a, float b, float c) {
    float r;
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The same, but NaN where one of them is.
__device__ __forceinline__ float fmax3_abs_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// One box from shared memory to the output (every row of it belongs to the prompt), and the waits for such stores: until the
// staging area has been read, and until they are done.
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, uint32_t src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

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

// cap2 tanh(y1 x) with the special-function unit: 1 - 2 / (e^2y + 1).  Off by 2^-22 of the cap, so for caps that no score comes
// near the polynomials are not only faster (they are off by 2.3e-6 of the score).
__device__ __forceinline__ float st_cap(const ScoredTcParams &p, float x) {
    return p.cap2 - __fdividef(2.f * p.cap2, ex2_approx(x * (2.f * kLog2e) * p.y1) + 1.f);
}

// mbar_wait with a limit of the call's own.
__device__ __forceinline__ bool st_mbar_wait(uint32_t bar, uint32_t parity, uint32_t limit) {
    if (mbar_try_wait(bar, parity)) return true;       // no look at the limit on the way that counts
    for (uint32_t i = 1; i < limit; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return false;
}

// One row the slow way, run by a whole warp: keys outside [lo, hi] are not touched; O is summed in units of 1 / unit.  32 keys at
// a time, a score per lane, then the lanes' channels of O: 4 us per 32 keys with eight warps at it (reads of K, a row per lane,
// past an L1 that the tiles have taken).
// It is for broken inputs: one NaN among the V rows of 8192 tokens x 32/8 heads makes 0.46 ms 33; 700 k tokens of one head, 77 ms, 2.5 s.
template <int D>
__device__ __noinline__ void st_slow_row(const ScoredTcParams &p, int64_t first, int row, int h, int lo, int hi, int lane, float unit) {
    constexpr int V = D / 32;
    const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.s.q) + (first + row) * p.s.q_stride + h * D;
    const int kvh = h / (p.s.Hq / p.s.Hkv);
    const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(p.s.k) + first * p.s.k_stride + kvh * D;
    const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(p.s.v) + first * p.s.v_stride + kvh * D + lane * V;
    const float slope = p.s.slopes ? p.s.slopes[h] : 0.f;
    auto wide = [](uint32_t x) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x)); };
    float o[V], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.f;
    for (int64_t j0 = lo; j0 <= hi; j0 += 32) {
        const int64_t j = j0 + lane;
        float s = 0.f;
        if (j <= hi) {
            const uint4 *kj = reinterpret_cast<const uint4 *>(k + j * p.s.k_stride), *qj = reinterpret_cast<const uint4 *>(q);
#pragma unroll 4
            for (int c = 0; c < D / 8; ++c) {
                const uint4 a = qj[c], b = kj[c];
                float2 x = wide(a.x), y = wide(b.x);
                s = fmaf(x.x, y.x, s); s = fmaf(x.y, y.y, s);
                x = wide(a.y); y = wide(b.y);
                s = fmaf(x.x, y.x, s); s = fmaf(x.y, y.y, s);
                x = wide(a.z); y = wide(b.z);
                s = fmaf(x.x, y.x, s); s = fmaf(x.y, y.y, s);
                x = wide(a.w); y = wide(b.w);
                s = fmaf(x.x, y.x, s); s = fmaf(x.y, y.y, s);
            }
        }
        s *= p.s.sm_scale;
        if (p.s.cap > 0.f) s = p.s.cap * tanhf(s / p.s.cap);
        s = fmaf(-slope, fabsf(static_cast<float>(row - j)), s);
        if (j > hi) s = -INFINITY;
        float mx = s;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;      // a score of -inf weighs nothing, a first one too
        const float alpha = m == -INFINITY ? 0.f : expf(m - ref), w = expf(s - ref);
        float sum = w;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        l = l != l ? l : l * alpha + sum;              // NaN scores leave no maximum, but a sum that is NaN
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] *= alpha;
        m = m_new;
        const int n = static_cast<int>(min(static_cast<int64_t>(32), hi - j0 + 1));
#pragma unroll 8
        for (int t = 0; t < n; ++t) {
            const float wt = __shfl_sync(0xffffffffu, w, t) * unit;
            const __nv_bfloat16 *vt = v + (j0 + t) * p.s.v_stride;
            if constexpr (V == 4) {
                const uint2 x = *reinterpret_cast<const uint2 *>(vt);
                const float2 a = wide(x.x), b = wide(x.y);
                o[0] = fmaf(wt, a.x, o[0]); o[1] = fmaf(wt, a.y, o[1]); o[2] = fmaf(wt, b.x, o[2]); o[3] = fmaf(wt, b.y, o[3]);
            } else {
                const float2 a = wide(*reinterpret_cast<const uint32_t *>(vt));
                o[0] = fmaf(wt, a.x, o[0]); o[1] = fmaf(wt, a.y, o[1]);
            }
        }
    }
    const int64_t dst = ((first + row) * p.s.Hq + h) * D + lane * V;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const float y0 = l == 0.f ? 0.f : o[i] / l / unit, y1 = l == 0.f ? 0.f : o[i + 1] / l / unit;
        if (p.s.out_bf16) *reinterpret_cast<__nv_bfloat162 *>(reinterpret_cast<__nv_bfloat16 *>(p.s.out) + dst + i) = __floats2bfloat162_rn(y0, y1);
        else *reinterpret_cast<float2 *>(reinterpret_cast<float *>(p.s.out) + dst + i) = make_float2(y0, y1);
    }
}

// In the sign bits of the result's halves: a 16-bit half with all exponent bits set carries into its sign bit.
__device__ __forceinline__ uint32_t st_not_finite(const uint4 &w) {
    return (((w.x & 0x7f807f80u) + 0x00800080u) | ((w.y & 0x7f807f80u) + 0x00800080u) | ((w.z & 0x7f807f80u) + 0x00800080u) |
            ((w.w & 0x7f807f80u) + 0x00800080u)) & 0x80008000u;
}

// Whether some V row of keys [lo, hi] holds a number that is not finite, or (nonzero) one that is not 0; run by a whole warp.
template <int D>
__device__ __noinline__ bool st_found(const ScoredTcParams &p, int64_t first, int h, int lo, int hi, int lane, bool nonzero) {
    constexpr int CH = D / 8, KW = 32 / CH;             // 16-byte chunks of a row, keys per load of the warp
    const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(p.s.v) + first * p.s.v_stride + h / (p.s.Hq / p.s.Hkv) * D + lane % CH * 8;
    for (int64_t j0 = lo; j0 <= hi; j0 += 8 * KW) {
        uint32_t any = 0;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int64_t j = j0 + x * KW + lane / CH;
            if (j <= hi) {
                const uint4 w = *reinterpret_cast<const uint4 *>(v + j * p.s.v_stride);
                any |= nonzero ? (w.x | w.y | w.z | w.w) & 0x7fff7fffu : st_not_finite(w);
            }
        }
        if (__any_sync(0xffffffffu, any != 0)) return true;
    }
    return false;
}

// CAP: 0 = scores are not capped; 1 = capped, with a cap that lets every weight be taken relative to 0; 2 = any cap.
template <int D, int CAP, bool BIAS>
__global__ void __launch_bounds__(kStThreads, 1)
prefill_scored_tc_kernel(const __grid_constant__ ScoredTcParams p, const __grid_constant__ CUtensorMap mq,
                         const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                         const __grid_constant__ CUtensorMap mo) {
    constexpr int QTILE = st_qtile(D), TILE = st_tile(D), NS = st_slots(D), BOXES = D / 64, KB = kStKeys;
    extern __shared__ __align__(1024) uint8_t base[];
    const uint32_t Qs = smem_u32(base), Ks = Qs + 2 * QTILE, Vs = Ks + NS * TILE;
    uint8_t *stage_all = base + 2 * QTILE + 2 * NS * TILE;
    uint64_t *bars = reinterpret_cast<uint64_t *>(stage_all + 8 * kStStage);
    uint64_t *bar_q = bars, *bar_qfree = bars + 1;                 // Q loaded; Q read by both tiles
    uint64_t *bar_s = bars + 2, *bar_sf = bars + 4;                // per tile: S ready; S in registers
    uint64_t *bar_p = bars + 6, *bar_o = bars + 8;                 // per tile: P written; O has taken the block in (P is free)
    uint64_t *bar_plan = bars + 10, *bar_planfree = bars + 12;     // per plan buffer
    uint64_t *bar_k = bars + 14, *bar_v = bar_k + NS, *bar_kfree = bar_v + NS, *bar_vfree = bar_kfree + NS;
    uint64_t *bar_guard = bar_vfree + NS;                          // per V slot: the guards are done with the block
    constexpr int NBARS = 14 + 5 * NS;
    static_assert(NBARS * 8 + 4 <= kStBarBytes, "barrier block");
    uint32_t &tmem_slot = *reinterpret_cast<uint32_t *>(bars + NBARS);
    StPlan *plans = reinterpret_cast<StPlan *>(stage_all + 8 * kStStage + kStBarBytes);
    const int tid = threadIdx.x, wid = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int hpc = p.heads_per_cta, hgroups = p.s.Hq / hpc, gq = p.s.Hq / p.s.Hkv;
    const int rows_item = hpc == 2 ? 128 : 256;

    if (blockIdx.x == 0) scored_check_offsets(p.s);
    if (tid == 320) {
        prefetch_tensormap(&mq); prefetch_tensormap(&mk); prefetch_tensormap(&mv); prefetch_tensormap(&mo);
        for (int b = 0; b < NBARS; ++b) {
            // Q and ring slots free: one per tile; S in registers, P written: one per softmax warp of the tile;
            // V looked through: one per guard; plan read: one per warp
            const int n = b == 1 || (b >= 14 + 2 * NS && b < 14 + 4 * NS) ? 2 : ((b >= 4 && b < 8) || b >= 14 + 4 * NS) ? 4 : (b >= 12 && b < 14) ? kStConsumers : 1;
            mbar_init(smem_u32(&bars[b]), n);
        }
        fence_mbar_init();
        fence_proxy_async();
    }
    if (wid == 8) {       // one warp allocates all of tensor memory for the CTA (it has the SM to itself)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kStTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);

    // Every wait is bounded, by more than rows that are done one by one take the warps that are waited for.  A wait that runs out
    // clears `ok`, and the warp leaves its loops at the next turn; nothing in the loops waits for all threads, so everybody comes to
    // the common end.
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity) { if (ok) ok = __all_sync(0xffffffffu, st_mbar_wait(smem_u32(bar), parity & 1, p.wait_limit)); };   // whole warps
    auto wait1 = [&](uint64_t *bar, uint32_t parity) { ok = ok && st_mbar_wait(smem_u32(bar), parity & 1, p.wait_limit); };                             // the loading thread
    // item r of this CTA: plan buffer r & 1, in its (r / 2)-th use
    auto plan_of = [&](int r) -> StPlan & { wait(&bar_plan[r & 1], r >> 1); __syncwarp(); return plans[r & 1]; };
    auto plan_done = [&](int r) { __syncwarp(); if (lane == 0) mbar_arrive(smem_u32(&bar_planfree[r & 1])); };

    // the launch's 512 x 128 registers, shared out by warpgroup: 256 x 192 + 256 x 64 = 65536
    if (wid < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        // ---------------- softmax warps: one query row per thread; n counts the tile's blocks
        const int t = wid >> 2, row = tid & 127;
        const uint32_t lanes = static_cast<uint32_t>((wid & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + (t ? kStS1 : kStS0), t_p = tmem + lanes + (t ? kStP1 : kStP0);
        const uint32_t t_o = tmem + lanes + (t ? kStO1 : kStO0);
        int n = 0;
        for (int r = 0; ok; ++r) {
            StPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            const StBlockStats w = pl.stats[wid];
            const int2 sp = pl.span[tid];
            const int lo = sp.x, hi = sp.y, kend = pl.kend, my_a = t ? pl.ja[1] : pl.ja[0], my_b = t ? pl.jb[1] : pl.jb[0];
            const int h = hpc == 2 ? pl.h0 + t : pl.h0, len = pl.len, trow0 = pl.row0 + (hpc == 2 ? 0 : 128 * t), qrow = trow0 + row;
            const int64_t first = pl.first;
            const bool have = t < pl.tiles, ahead = pl.ahead != 0;
            float l = 0.f, m = -INFINITY;                  // m: reference point in log2 units of the score
            int form = 1;                                  // the cap's form that would have served the block before
            // The bias without the row's own constant: with the scores of a block taken relative to -slope (row - kb), kb its first
            // key, a key x places in counts slope x for every row, a table per head in the plan; the reference m moves into the
            // next block's frame by a constant.
            const float slope2 = BIAS ? pl.slope2[t] : 0.f, *bias = pl.bias[t];
            for (int j = my_a; j < my_b && ok; ++j) {
                const int i = j - my_a, kb = kend - j * KB;
                if constexpr (BIAS) m = i > 0 ? m + slope2 * static_cast<float>(KB) : m;
                wait(&bar_s[t], n + i);
                __syncwarp();
                tc_fence_after();
                if (w.maxhi < kb || w.minlo >= kb + KB) {     // nobody in this warp sees any of it: weights 0
                    uint32_t z[32];
#pragma unroll
                    for (int x = 0; x < 32; ++x) z[x] = 0u;
                    if (lane == 0) mbar_arrive(smem_u32(&bar_sf[t]));
                    if (n + i > 0) wait(&bar_o[t], n + i - 1);
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
                auto form_of = [&](float big) {              // 1, 2: the polynomial that holds for the whole warp; 0: the exact form
                    return __all_sync(0xffffffffu, big <= p.half_at) ? 1 : __all_sync(0xffffffffu, big <= p.one_at) ? 2 : 0;
                };
                auto poly1 = [&](int x) {                    // capped scores x, x + 1 in log2 units
                    const uint64_t s2 = pack_f32x2(sv[x], sv[x + 1]), y = mul_f32x2(s2, s2);
                    uint64_t q = fma_f32x2(y, p.p1[3], p.p1[2]);
                    q = fma_f32x2(q, y, p.p1[1]);
                    q = fma_f32x2(q, y, p.p1[0]);
                    return mul_f32x2(q, s2);
                };
                auto poly2 = [&](int x) {
                    const uint64_t s2 = pack_f32x2(sv[x], sv[x + 1]), y = mul_f32x2(s2, s2);
                    uint64_t q = fma_f32x2(y, p.p2[5], p.p2[4]);
                    q = fma_f32x2(q, y, p.p2[3]);
                    q = fma_f32x2(q, y, p.p2[2]);
                    q = fma_f32x2(q, y, p.p2[1]);
                    q = fma_f32x2(q, y, p.p2[0]);
                    return mul_f32x2(q, s2);
                };
                auto exact = [&](int x) { return pack_f32x2(st_cap(p, sv[x]), st_cap(p, sv[x + 1])); };
                auto in_place = [&](auto &&f) {
#pragma unroll
                    for (int x = 0; x < KB; x += 2) unpack_f32x2(f(x), sv[x], sv[x + 1]);
                };
                // ---- score options in place.  Where any apply (kLog2) sv then holds scores in log2 units; q.k else.
                constexpr bool kLog2 = CAP == 2 || BIAS;
                if constexpr (CAP == 2) {
                    float big[4] = {0.f, 0.f, 0.f, 0.f};
                    if (masked) {                                  // hidden scores may be anything
#pragma unroll
                        for (int x = 0; x < KB; ++x) sv[x] = seen(x) ? sv[x] : 0.f;
                    }
#pragma unroll
                    for (int x = 0; x < KB; x += 2) big[(x >> 1) & 3] = fmax3_abs(big[(x >> 1) & 3], sv[x], sv[x + 1]);
                    const int form = form_of(fmaxf(fmaxf(big[0], big[1]), fmaxf(big[2], big[3])) * p.y1);
                    const uint64_t y12 = pack_f32x2(p.y1, p.y1), cap22 = pack_f32x2(p.cap2, p.cap2);
                    auto scaled = [&](auto &&poly) {
                        in_place([&](int x) { return mul_f32x2(pack_f32x2(sv[x], sv[x + 1]), y12); });
                        in_place([&](int x) { return mul_f32x2(poly(x), cap22); });
                    };
                    if (form == 1) scaled(poly1);
                    else if (form == 2) scaled(poly2);
                    else in_place(exact);
                }
                if constexpr (BIAS) {
                    const float scale = CAP ? 1.f : p.c2;
                    if (kb + KB - 1 <= trow0 || !ahead) {             // no key ahead of its row, but hidden ones
                        const uint64_t sc2 = pack_f32x2(scale, scale);
#pragma unroll
                        for (int x = 0; x < KB; x += 4) {
                            const ulonglong2 b4 = *reinterpret_cast<const ulonglong2 *>(bias + x);
                            unpack_f32x2(fma_f32x2(pack_f32x2(sv[x], sv[x + 1]), sc2, b4.x), sv[x], sv[x + 1]);
                            unpack_f32x2(fma_f32x2(pack_f32x2(sv[x + 2], sv[x + 3]), sc2, b4.y), sv[x + 2], sv[x + 3]);
                        }
                    } else {                                           // a key ahead of the row counts -slope (x + 2 (kb - row))
                        const float off = static_cast<float>(kb - qrow), off2 = 2.f * off;
#pragma unroll
                        for (int x = 0; x < KB; ++x) {
                            const float fx = static_cast<float>(x);
                            sv[x] = fmaf(slope2, fx + off <= 0.f ? fx : -(fx + off2), sv[x] * scale);
                        }
                    }
                }
                if (masked) {
                    if constexpr (CAP == 1) in_place(exact);
#pragma unroll
                    for (int x = 0; x < KB; ++x) sv[x] = seen(x) ? sv[x] : -INFINITY;
                }
                // ---- weights 2^(score - reference), their sum, and P
                bool o_ready = n + i == 0;                       // O has taken the block before in
                uint64_t lsum2 = 0;                              // two partial row sums, (+0, +0)
                uint32_t pk[KB / 2];
                // arg(x): scores x, x + 1 in log2 units, relative to the reference; extremum: runs alongside, in four chains
                float r4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto weights = [&](auto &&arg, auto &&extremum) {
                    lsum2 = 0;
#pragma unroll
                    for (int y = 0; y < KB / 2; ++y) {
                        float a0, a1;
                        extremum(r4[y & 3], sv[2 * y], sv[2 * y + 1]);
                        unpack_f32x2(arg(2 * y), a0, a1);
                        const float p0 = ex2_approx(a0), p1 = ex2_approx(a1);
                        pk[y] = pack_bf16(p0, p1);
                        // CAP 1: the rounded weights are summed, so that where few keys carry a row, numerator and sum are off alike: errors
                        // against 64 bits 0.0023 -> 0.0018 of the output, whose own rounding to bf16 makes 0.0016; and 2 % faster.  Elsewhere that
                        // would cost 5 to 17 % (the instructions stand in the chain of a score there) and sums of the weights as computed do.
                        lsum2 = add_f32x2(lsum2, CAP == 1 ? pack_f32x2(__uint_as_float(pk[y] << 16), __uint_as_float(pk[y] & 0xffff0000u)) : pack_f32x2(p0, p1));
                    }
                };
                auto nothing = [](float &, float, float) {};
                if constexpr (CAP == 1) {
                    // Capped scores lie within +-cap2 <= 72 log2 units: relative to 0, weights and sums over 2^31 keys stay within fp32 (and
                    // O for |v| < 2^31 and 2^24 keys; rows that leave it are done again), so no maximum is needed.  The form that suits
                    // the block before is tried first; whether it holds here is found out alongside.
                    if (masked) {
                        weights([&](int x) { return pack_f32x2(sv[x], sv[x + 1]); }, nothing);
                    } else {
                        auto largest = [](float &r, float a, float b) { r = fmax3_abs(r, a, b); };
                        r4[0] = r4[1] = r4[2] = r4[3] = 0.f;
                        if (form == 1) weights(poly1, largest);
                        else if (form == 2) weights(poly2, largest);
                        else weights(exact, largest);
                        const int holds = form_of(fmaxf(fmaxf(r4[0], r4[1]), fmaxf(r4[2], r4[3])) * p.y1);
                        if (form == 1 && holds == 2) weights(poly2, nothing);
                        else if (form != 0 && holds == 0) weights(exact, nothing);
                        form = holds;
                    }
                } else {
                    // The reference is the greatest score so far, or less by up to kPfSlack, so that O is hardly ever rescaled;
                    // a row that has seen nothing keeps -inf.  (Taking the weights relative to the block before's reference, with
                    // the maximum found alongside and the weights taken again where that was too low, was 7 % slower.)
#pragma unroll
                    for (int x = 0; x < KB; x += 2) r4[(x >> 1) & 3] = fmax3(r4[(x >> 1) & 3], sv[x], sv[x + 1]);
                    const float mx = fmaxf(fmaxf(r4[0], r4[1]), fmaxf(r4[2], r4[3])), xmax = kLog2 ? mx : mx * p.c2;
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
                                for (int x = 0; x < 32; ++x) ov[x] *= alpha;
                                tmem_st32(t_o + c * 32, ov);
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
                    const uint64_t mx2 = pack_f32x2(-ref, -ref), c22 = pack_f32x2(p.c2, p.c2);
                    if constexpr (kLog2) weights([&](int x) { return add_f32x2(pack_f32x2(sv[x], sv[x + 1]), mx2); }, nothing);
                    else weights([&](int x) { return fma_f32x2(pack_f32x2(sv[x], sv[x + 1]), c22, mx2); }, nothing);
                }
                if (!o_ready) wait(&bar_o[t], n + i - 1);      // P of the block before has been read
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
            const int nblk = my_b - my_a;
            n += nblk;
            if (nblk > 0) wait(&bar_o[t], n - 1);
            __syncwarp();
            tc_fence_after();
            const bool poisoned = *const_cast<volatile int32_t *>(&pl.poisoned) != 0;
            if (ok && have && poisoned) {
                for (int x = 0; x < 32; ++x) {               // the warp's own rows, one by one
                    const int rr = trow0 + (wid & 3) * 32 + x;
                    const int2 s2 = pl.span[(wid << 5) + x];
                    if (rr < len) st_slow_row<D>(p, first, rr, h, s2.x, s2.y, lane, 1.f);
                }
            } else if (ok && have) {
                // ---- normalise this thread's row, 128 bytes of output at a time, into the warp's staging area (128-byte rows, 16-byte
                //      chunks XOR-swizzled by the row, as the tensor map wants it and free of bank conflicts); a warp whose 32 rows
                //      all belong to the prompt stores the box by TMA, another one row by row.  (Stores by the threads took 2500
                //      of 3900 cycles here.)  A row that saw nothing (l = 0) gives zeros.
                const float inv = l == 0.f ? 0.f : 1.f / l;
                uint8_t *stage = stage_all + wid * kStStage;
                const int rows_live = len - trow0 - (wid & 3) * 32;             // rows of this warp that belong to the prompt
                const int64_t tok0 = first + trow0 + (wid & 3) * 32;
                const bool b16 = p.s.out_bf16 != 0;
                const int width = b16 ? 64 : 32;                                 // channels in 128 bytes
                float big[4] = {0.f, 0.f, 0.f, 0.f};                            // greatest channel of O, NaN among them included
                auto scaled = [&](float (&ov)[32]) {
#pragma unroll
                    for (int x = 0; x < 32; x += 2) big[(x >> 1) & 3] = fmax3_abs_nan(big[(x >> 1) & 3], ov[x], ov[x + 1]);
#pragma unroll
                    for (int x = 0; x < 32; ++x) ov[x] = inv == 0.f ? 0.f : ov[x] * inv;
                };
#pragma unroll 1
                for (int c = 0; c < D && rows_live > 0; c += width) {
                    if (lane == 0) tma_store_wait_read();                        // the box before has left the staging area
                    __syncwarp();
                    uint8_t *mine = stage + lane * 128;
                    float ov[32];
                    tmem_ld32(t_o + c, ov);
                    scaled(ov);
                    if (b16) {
#pragma unroll
                        for (int q4 = 0; q4 < 4; ++q4)
                            *reinterpret_cast<uint4 *>(mine + ((q4 ^ (lane & 7)) << 4)) =
                                make_uint4(pack_bf16(ov[8 * q4], ov[8 * q4 + 1]), pack_bf16(ov[8 * q4 + 2], ov[8 * q4 + 3]),
                                           pack_bf16(ov[8 * q4 + 4], ov[8 * q4 + 5]), pack_bf16(ov[8 * q4 + 6], ov[8 * q4 + 7]));
                        tmem_ld32(t_o + c + 32, ov);
                        scaled(ov);
#pragma unroll
                        for (int q4 = 0; q4 < 4; ++q4)
                            *reinterpret_cast<uint4 *>(mine + (((q4 + 4) ^ (lane & 7)) << 4)) =
                                make_uint4(pack_bf16(ov[8 * q4], ov[8 * q4 + 1]), pack_bf16(ov[8 * q4 + 2], ov[8 * q4 + 3]),
                                           pack_bf16(ov[8 * q4 + 4], ov[8 * q4 + 5]), pack_bf16(ov[8 * q4 + 6], ov[8 * q4 + 7]));
                    } else {
#pragma unroll
                        for (int q4 = 0; q4 < 8; ++q4)
                            *reinterpret_cast<float4 *>(mine + ((q4 ^ (lane & 7)) << 4)) =
                                make_float4(ov[4 * q4], ov[4 * q4 + 1], ov[4 * q4 + 2], ov[4 * q4 + 3]);
                    }
                    if (rows_live >= 32) {
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) tma_store_3d(&mo, smem_u32(stage), c, h, static_cast<int>(tok0));
                    } else {
                        __syncwarp();
                        uint8_t *dst = reinterpret_cast<uint8_t *>(p.s.out);
                        const int es = b16 ? 2 : 4;
                        for (int x = lane; x < rows_live * 8; x += 32)
                            *reinterpret_cast<uint4 *>(dst + (((tok0 + (x >> 3)) * p.s.Hq + h) * D + c) * es + (x & 7) * 16) =
                                *reinterpret_cast<const uint4 *>(stage + (x >> 3) * 128 + (((x & 7) ^ ((x >> 3) & 7)) << 4));
                        __syncwarp();
                    }
                }
                // Weights relative to something else than the row's greatest score (0, or a reference that lags behind it) may have taken O
                // out of fp32's range, though the quotient lies within: up, or down (all weights below 1 and tiny v; the tensor core
                // knows no denormal sums).  Such rows are done again, unless V itself is not finite among the keys that they all see
                // (were it so among others, all rows would be done again) or 0 wherever they look.
                const float top = fmax3_abs_nan(fmax3_abs_nan(big[0], big[1], big[2]), big[3], 0.f);
                const bool sound = lane < rows_live && l > 0.f && l < INFINITY, over = sound && !(top < INFINITY);
                const bool under = CAP == 1 && sound && top < 0x1p-100f && l < static_cast<float>(hi - lo + 1);
                const uint32_t overs = __ballot_sync(0xffffffffu, over);
                uint32_t again = overs;
                if (overs != 0) {
                    const int a = __reduce_max_sync(0xffffffffu, over ? lo : 0), b = __reduce_min_sync(0xffffffffu, over ? hi : 0x7fffffff);
                    if (st_found<D>(p, first, h, a, b, lane, false)) again = 0;
                }
                if (CAP == 1 && __any_sync(0xffffffffu, under)) {
                    const int a = __reduce_min_sync(0xffffffffu, under ? lo : 0x7fffffff), b = __reduce_max_sync(0xffffffffu, under ? hi : -1);
                    const uint32_t unders = __ballot_sync(0xffffffffu, under);
                    if (st_found<D>(p, first, h, a, b, lane, true)) again |= unders;
                }
                if (again != 0) {
                    if (lane == 0) tma_store_wait();         // what is there already is overwritten
                    __syncwarp();
                    for (; again != 0; again &= again - 1) {
                        const int x = __ffs(again) - 1;
                        const int2 s2 = pl.span[(wid << 5) + x];
                        st_slow_row<D>(p, first, trow0 + (wid & 3) * 32 + x, h, s2.x, s2.y, lane, (overs >> x) & 1 ? 0x1p-32f : 1.f);
                    }
                }
            }
            tc_fence_before();                               // O is read: ordered before this warp's next arrival
            plan_done(r);
        }
        if (lane == 0) tma_store_wait();             // before the CTA's shared memory goes
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (wid == 12) {
        // ---------------- the planning warp
        // lane l sums the item rows of users [l C, (l + 1) C); users from the first inconsistent one on are left out
        const int C = (p.s.B + 31) / 32, u0 = lane * C, u1 = min(p.s.B, u0 + C);
        int sum = 0;
        bool bad = false;
#pragma unroll 4
        for (int u = u0; u < u1; ++u) {
            const int64_t a = p.s.tok_indptr[u], b = p.s.tok_indptr[u + 1];
            bad = bad || a < 0 || b < a || b > p.s.T;
            if (!bad) sum += static_cast<int>((b - a + rows_item - 1) / rows_item);
        }
        int inc = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, inc, d);
            if (lane >= d) inc += up;
        }
        const unsigned badmask = __ballot_sync(0xffffffffu, bad);
        const int blocks = __shfl_sync(0xffffffffu, inc, badmask ? __ffs(badmask) - 1 : 31);
        const int64_t items = static_cast<int64_t>(blocks) * hgroups;
        // The first item of a CTA is its index, the next ones are drawn from a counter (items differ in length, by masks and
        // from prompt to prompt); the last CTA to draw past the end puts the counters back to zero for the next call.
        int64_t item = blockIdx.x;
        for (int r = 0;; ++r) {
            StPlan &pl = plans[r & 1];
            if (r >= 2) wait(&bar_planfree[r & 1], (r >> 1) - 1);
            __syncwarp();
            const bool some = ok && item < items;
            if (!some) {
                if (lane == 0) {
                    pl.valid = 0;
                    mbar_arrive(smem_u32(&bar_plan[r & 1]));
                    __threadfence();
                    if (atomicAdd(&p.s.hdr[HDR_ITEM_EXITS], 1) == static_cast<int32_t>(gridDim.x) - 1) {
                        p.s.hdr[HDR_NEXT_ITEM] = 0;
                        p.s.hdr[HDR_ITEM_EXITS] = 0;
                    }
                }
                break;
            }
            int next = 0;
            if (lane == 0) next = atomicAdd(&p.s.hdr[HDR_NEXT_ITEM], 1);
            const int blk = static_cast<int>(item / hgroups), h0 = static_cast<int>(item % hgroups) * hpc;
            float slope2[2] = {0.f, 0.f};
            if constexpr (BIAS) { slope2[0] = p.s.slopes[h0] * kLog2e; slope2[1] = p.s.slopes[h0 + hpc - 1] * kLog2e; }
            int user = 0, qb = 0, first = 0, len = 0;
            {                             // the user whose rows hold block blk; a prompt's blocks count from its end
                const int src = __ffs(__ballot_sync(0xffffffffu, blk < inc)) - 1;
                if (lane == src) {
                    int rem = blk - (inc - sum);
                    for (user = u0; user < u1; ++user) {
                        first = p.s.tok_indptr[user];
                        len = p.s.tok_indptr[user + 1] - first;
                        const int nb = (len + rows_item - 1) / rows_item;
                        if (rem < nb) { qb = nb - 1 - rem; break; }
                        rem -= nb;
                    }
                }
                user = __shfl_sync(0xffffffffu, user, src);
                qb = __shfl_sync(0xffffffffu, qb, src);
                first = __shfl_sync(0xffffffffu, first, src);
                len = __shfl_sync(0xffffffffu, len, src);
            }
            const int row0 = qb * rows_item;
            const int prefix = p.s.prefix_lens ? min(len, p.s.prefix_lens[user]) : 0;
            int tlo[2] = {0x7fffffff, 0x7fffffff}, thi[2] = {-1, -1}, fulllo = -1, fullhi = 0x7fffffff;
#pragma unroll
            for (int w = 0; w < 8; ++w) {           // the 32 rows of softmax warp w; two heads have the same rows
                const int qrow = row0 + (hpc == 2 ? 32 * (w & 3) : 32 * w) + lane;
                int lo = 0x7fffffff, hi = -1;
                const bool live = qrow < len;
                if (live) scored_interval(p.s, first, prefix, qrow, lo, hi);
                const bool sees = lo <= hi;
                if (!sees) { lo = 0x7fffffff; hi = -1; }
                pl.span[32 * w + lane] = make_int2(lo, hi);
                // a live row that sees nothing makes every block one with hidden keys
                const int a = __reduce_min_sync(0xffffffffu, lo), b = __reduce_max_sync(0xffffffffu, hi);
                const int c = __reduce_max_sync(0xffffffffu, sees ? lo : (live ? 0x7fffffff : -1));
                const int d = __reduce_min_sync(0xffffffffu, sees ? hi : (live ? -1 : 0x7fffffff));
                if (lane == 0) pl.stats[w] = StBlockStats{a, b, c, d};
                tlo[w >> 2] = min(tlo[w >> 2], a); thi[w >> 2] = max(thi[w >> 2], b);
                fulllo = max(fulllo, c); fullhi = min(fullhi, d);
            }
            if constexpr (BIAS) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (lane == 0) pl.slope2[t] = slope2[t];
                    for (int x = lane; x < KB; x += 32) pl.bias[t][x] = slope2[t] * static_cast<float>(x);
                }
            }
            if (lane == 0) {
                const int key0 = min(tlo[0], tlo[1]), key1 = max(thi[0], thi[1]);
                pl.valid = 1; pl.first = first; pl.len = len; pl.row0 = row0; pl.h0 = h0;
                pl.tiles = (hpc == 2 || row0 + 128 < len) ? 2 : 1;
                const int nb = key1 < 0 ? 0 : (key1 - key0) / KB + 1;
                pl.nb = nb; pl.kend = key1 < 0 ? 0 : key0 + (nb - 1) * KB;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    pl.ja[x] = thi[x] < 0 ? 0 : nb - 1 - (thi[x] - key0) / KB;
                    pl.jb[x] = thi[x] < 0 ? 0 : nb - (tlo[x] - key0) / KB;
                }
                pl.fulllo = fulllo; pl.fullhi = fullhi; pl.poisoned = 0;
                pl.ahead = prefix > row0 + 1;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_plan[r & 1]));
            item = static_cast<int64_t>(gridDim.x) + __shfl_sync(0xffffffffu, next, 0);
        }
    } else if (wid == 10) {
        // ---------------- the loading warp (one thread of it); c counts blocks over all items
        int c = 0, nq = 0;
        for (int r = 0; ok; ++r) {
            const StPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            const int NB = pl.nb, kvh = pl.h0 / gq, y0 = pl.first + pl.kend;
            if (lane == 0 && NB > 0) {
                if (nq > 0) wait1(bar_qfree, nq - 1);
                if (ok) {
                    mbar_expect_tx(smem_u32(bar_q), pl.tiles * QTILE);
                    for (int t = 0; t < pl.tiles; ++t)
                        for (int x = 0; x < BOXES; ++x)
                            tma_load_3d(Qs + t * QTILE + x * kStQBox, &mq, 64 * x, hpc == 2 ? pl.h0 + t : pl.h0, pl.first + pl.row0 + (hpc == 2 ? 0 : 128 * t), smem_u32(bar_q));
                }
                for (int j = 0; j < NB && ok; ++j, ++c) {
                    const int slot = c % NS, use = c / NS, y = y0 - j * KB;
                    if (use > 0) wait1(&bar_kfree[slot], use - 1);
                    if (!ok) break;
                    mbar_expect_tx(smem_u32(&bar_k[slot]), TILE);
                    for (int x = 0; x < BOXES; ++x) tma_load_3d(Ks + slot * TILE + x * kStBox, &mk, 64 * x, kvh, y, smem_u32(&bar_k[slot]));
                    if (use > 0) wait1(&bar_vfree[slot], use - 1);
                    if (!ok) break;
                    mbar_expect_tx(smem_u32(&bar_v[slot]), TILE);
                    for (int x = 0; x < BOXES; ++x) tma_load_3d(Vs + slot * TILE + x * kStBox, &mv, 64 * x, kvh, y, smem_u32(&bar_v[slot]));
                }
            }
            if (NB > 0) ++nq;
            ok = __shfl_sync(0xffffffffu, ok, 0);
            plan_done(r);
        }
        if (lane == 0 && !ok) {              // leave nothing in flight behind: a bounded chance for what was asked for last
            if (nq > 0) mbar_wait(smem_u32(bar_q), (nq - 1) & 1);
            for (int x = 0; x < NS; ++x) {
                const int uses = (c - x + NS) / NS;          // blocks that went to slot x, the one that was cut off included
                if (c >= x && uses > 0) { mbar_wait(smem_u32(&bar_k[x]), (uses - 1) & 1); mbar_wait(smem_u32(&bar_v[x]), (uses - 1) & 1); }
            }
        }
    } else if (wid == 11 || wid >= 13) {
        // ---------------- the guards: V rows of blocks with hidden keys, a quarter of the rows each
        constexpr int GR = KB / 4;
        const int g0 = (wid == 11 ? 0 : wid - 12) * GR;
        int c = 0;
        for (int r = 0; ok; ++r) {
            StPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            const int NB = pl.nb;
            for (int j = 0; j < NB && ok; ++j, ++c) {
                // every block passes through here, so that no guard is ever a whole ring ahead of or behind the others
                const int slot = c % NS, kb = pl.kend - j * KB;
                wait(&bar_v[slot], c / NS);
                __syncwarp();
                if (pl.fulllo <= kb && kb + KB - 1 <= pl.fullhi) {
                    if (lane == 0) mbar_arrive(smem_u32(&bar_guard[slot]));
                    continue;
                }
                uint8_t *vt = base + 2 * QTILE + (NS + slot) * TILE;
                uint32_t any = 0;
#pragma unroll
                for (int x = lane; x < BOXES * GR * 8; x += 32)
                    any |= st_not_finite(*reinterpret_cast<const uint4 *>(vt + (x / (GR * 8)) * kStBox + g0 * 128 + (x % (GR * 8)) * 16));
                if (__any_sync(0xffffffffu, any != 0)) {
                    for (int row = g0; row < g0 + GR; ++row) {        // rare: row by row
                        uint4 *chunk = reinterpret_cast<uint4 *>(vt + (lane >> 3) * kStBox + row * 128 + (lane & 7) * 16);
                        const bool mine = lane < 8 * BOXES;
                        if (!__any_sync(0xffffffffu, mine && st_not_finite(*(mine ? chunk : reinterpret_cast<uint4 *>(vt + row * 128))) != 0)) continue;
                        const int key = kb + row;
                        bool seen = false, hidden = false;
                        for (int x = lane; x < 256; x += 32) {
                            const int2 sp = pl.span[x];
                            const bool s = sp.x <= key && key <= sp.y;
                            seen = seen || s;
                            hidden = hidden || !s;
                        }
                        if (!__any_sync(0xffffffffu, seen)) {
                            if (mine) *chunk = make_uint4(0, 0, 0, 0);
                        } else if (__any_sync(0xffffffffu, hidden)) {
                            pl.poisoned = 1;
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
        // ---------------- the warp that issues tile x's MMAs: S of block j, then P V of block j - 1; n counts the tile's blocks
        const int x = wid - 8;
        const uint32_t ts = tmem + (x ? kStS1 : kStS0), tp = tmem + (x ? kStP1 : kStP0), to = tmem + (x ? kStO1 : kStO0);
        int c = 0, n = 0, nq = 0;
        for (int r = 0; ok; ++r) {
            const StPlan &pl = plan_of(r);
            if (!ok || !pl.valid) break;
            const int NB = pl.nb, a = x ? pl.ja[1] : pl.ja[0], b = x ? pl.jb[1] : pl.jb[0];
            if (NB > 0) wait(bar_q, nq++);
            for (int j = 0; j <= NB && NB > 0 && ok; ++j) {
                if (j < NB) {
                    const int slot = (c + j) % NS;
                    // a tile that has no use for a block gives it back all the same, once it is there: never a ring ahead
                    wait(&bar_k[slot], (c + j) / NS);
                    if (a <= j && j < b) {
                        const int k = n + j - a;
                        if (k > 0) wait(&bar_sf[x], k - 1);
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
                    if (j == NB - 1) st_commit(smem_u32(bar_qfree));      // behind the item's last use of Q (at once where nothing is under way)
                }
                if (j > 0) {
                    const int jj = j - 1, slot = (c + jj) % NS;
                    wait(&bar_v[slot], (c + jj) / NS);
                    wait(&bar_guard[slot], (c + jj) / NS);
                    if (a <= jj && jj < b) {
                        const int i = jj - a;
                        wait(&bar_p[x], n + i);           // also: this tile's softmax has read the O of the item before
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
            c += NB;
            n += b - a;
            plan_done(r);
        }
    }
    }
    tc_fence_before();
    const bool gave_up = !__syncthreads_and(ok);
    tc_fence_after();
    if (gave_up && tid == 0) flag_error(p.s.hdr, 6 /* SPD_ERR_TIMEOUT */, -1);
    if (wid == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kStTmemCols) : "memory");
}

}  // namespace spd

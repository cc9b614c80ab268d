// Prompt attention with score options and interval masks: argument checks, tensor maps, choice of the kernel.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "spd_host.h"
#include "spd_prefill_scored.cuh"
#include "spd_prefill_scored_f32.cuh"
#include "spd_prefill_scored_tc.cuh"

namespace {

using namespace spd;
using host::misaligned;
using host::row_stride;

// [T][heads][head_dim] bf16 (the output may be fp32) with a token stride, as a 3-D tensor map; one box = `rows` tokens x 128 bytes of
// one head, 128-byte swizzle.
spd_status make_token_map(CUtensorMap *map, const void *ptr, int64_t T, int heads, int D, int64_t stride, int rows, bool f32 = false) {
    EncodeTiledFn fn = host::tensor_map_encoder();
    if (!fn) return SPD_ERR_CUDA;
    cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(T)};
    const cuuint64_t es = f32 ? 4 : 2;
    cuuint64_t strides[2] = {static_cast<cuuint64_t>(D) * es, static_cast<cuuint64_t>(stride) * es};
    cuuint32_t box[3] = {f32 ? 32u : 64u, 1, static_cast<cuuint32_t>(rows)};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) fprintf(stderr, "libspd: cuTensorMapEncodeTiled failed with CUresult %d\n", static_cast<int>(r));
    return r == CUDA_SUCCESS ? SPD_OK : SPD_ERR_CUDA;
}

template <int D, int CAP, bool BIAS>
spd_status launch_prefill_tc(const ScoredTcParams &p, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const CUtensorMap &mo, unsigned grid, cudaStream_t st) {
    static std::once_flag once[64];
    int dev = 0;
    cudaGetDevice(&dev);
    cudaError_t err = cudaSuccess;
    std::call_once(once[dev & 63], [&] {
        err = cudaFuncSetAttribute(prefill_scored_tc_kernel<D, CAP, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(st_smem_bytes(D)));
    });
    if (err != cudaSuccess) return SPD_ERR_CUDA;
    prefill_scored_tc_kernel<D, CAP, BIAS><<<grid, kStThreads, st_smem_bytes(D), st>>>(p, mq, mk, mv, mo);
    host::count_launch();
    return cudaGetLastError() == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

uint64_t twice(double x) {              // an fp32 value in both halves of a two-lane operand
    const float f = static_cast<float>(x);
    uint32_t u;
    memcpy(&u, &f, 4);
    return (static_cast<uint64_t>(u) << 32) | u;
}

// bf16 prompts on the tensor cores.
spd_status prefill_tc(const spd_shape &s, const ScoredPrefillParams &sp, cudaStream_t st) {
    ScoredTcParams p{};
    p.s = sp;
    const int g = s.num_q_heads / s.num_kv_heads;
    p.heads_per_cta = g % 2 == 0 ? 2 : 1;
    p.c2 = s.sm_scale * kLog2e;
    p.half_at = p.one_at = -1.f;
    p.wait_limit = st_wait_limit(sp.T);
    const bool bias = sp.slopes != nullptr;
    const int cap = sp.cap == 0.f ? 0 : (sp.cap <= kStFixedCap && !bias) ? 1 : 2;
    if (sp.cap > 0.f) {
        const double y1 = static_cast<double>(s.sm_scale) / sp.cap;
        p.cap2 = sp.cap * kLog2e;
        p.y1 = static_cast<float>(fmin(y1, 1e30));
        // Scaled coefficients (CAP 1) that leave fp32's normal range: the exact form does it.
        bool fits1 = true, fits2 = true;
        auto normal = [](double c) { return fabs(c) > 1e-37 && fabs(c) < 1e37; };
        for (int i = 0; i < 6; ++i) {
            const double c = cap == 1 ? sp.cap * 1.4426950408889634 * pow(y1, 2 * i + 1) : 1.0;
            if (i < 4) { p.p1[i] = twice(c * kTanhHalf[i]); fits1 = fits1 && normal(c * kTanhHalf[i]); }
            p.p2[i] = twice(c * kTanhOne[i]);
            fits2 = fits2 && normal(c * kTanhOne[i]);
        }
        if (fits1) p.half_at = 0.5f;
        if (fits2) p.one_at = 1.f;
    }
    CUtensorMap mq, mk, mv, mo;
    spd_status rc;
    if ((rc = make_token_map(&mq, sp.q, sp.T, s.num_q_heads, s.head_dim, sp.q_stride, 128)) != SPD_OK) return rc;
    if ((rc = make_token_map(&mk, sp.k, sp.T, s.num_kv_heads, s.head_dim, sp.k_stride, kStKeys)) != SPD_OK) return rc;
    if ((rc = make_token_map(&mv, sp.v, sp.T, s.num_kv_heads, s.head_dim, sp.v_stride, kStKeys)) != SPD_OK) return rc;
    if ((rc = make_token_map(&mo, sp.out, sp.T, s.num_q_heads, s.head_dim, static_cast<int64_t>(s.num_q_heads) * s.head_dim, 32, !sp.out_bf16)) != SPD_OK)
        return rc;
    const int rows = p.heads_per_cta == 2 ? 128 : 256;
    // at most one CTA per SM; fewer where there are not that many items
    const int64_t items = ((sp.T + rows - 1) / rows + s.batch) * (s.num_q_heads / p.heads_per_cta);
    int sms = 0;
    if ((rc = host::device_sms(&sms)) != SPD_OK) return rc;
    const unsigned grid = static_cast<unsigned>(items < sms ? items : sms);
#define SPD_TC_CASE(DD, CC, BB) if (s.head_dim == DD && cap == CC && bias == BB) return launch_prefill_tc<DD, CC, BB>(p, mq, mk, mv, mo, grid, st);
    SPD_TC_CASE(128, 0, false) SPD_TC_CASE(128, 1, false) SPD_TC_CASE(128, 2, false) SPD_TC_CASE(128, 0, true) SPD_TC_CASE(128, 2, true)
    SPD_TC_CASE(64, 0, false) SPD_TC_CASE(64, 1, false) SPD_TC_CASE(64, 2, false) SPD_TC_CASE(64, 0, true) SPD_TC_CASE(64, 2, true)
#undef SPD_TC_CASE
    return SPD_ERR_UNSUPPORTED;
}

template <int D, int RPT, int G>
spd_status launch_prefill_f32(const spd_shape &s, const ScoredPrefillParams &p, cudaStream_t st) {
    using C = ScoredF32<D, RPT, G>;
    static std::once_flag once[64];
    int dev = 0;
    cudaGetDevice(&dev);
    cudaError_t err = cudaSuccess;
    std::call_once(once[dev & 63], [&] {
        err = cudaFuncSetAttribute(prefill_scored_f32_kernel<D, RPT, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(C::smem_bytes()));
    });
    if (err != cudaSuccess) return SPD_ERR_CUDA;
    const dim3 grid(static_cast<unsigned>((p.T + C::R - 1) / C::R + s.batch), static_cast<unsigned>(s.num_q_heads));
    prefill_scored_f32_kernel<D, RPT, G><<<grid, 256 * G, C::smem_bytes(), st>>>(p);
    host::count_launch();
    return cudaGetLastError() == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

// fp32 prompts on the FMA pipes: four rows per thread, two where that leaves SMs without work or prompts fill half of 64 rows at most
// (by the mean over all users, those without a prompt among them: the host knows no lengths, and any choice is right); two
// groups of threads per tile where the keys of a row, not the number of tiles, are what an SM's work consists of.  us, two rows / four /
// four and two groups, 8 heads of 64: 2 x 256 tokens 19.1 / 26.2 / 24.4, 200 x 20 53 / 70 / 107, 4 x 256 30.2 / 41.2 / 25.1, 2 x 1000
// 149 / 152 / 129, 4 x 1000 255 / 217 / 205, 16 x 1000 846 / 634 / 683, 64 x 256 271 / 208 / 256.
spd_status prefill_f32(const spd_shape &s, const ScoredPrefillParams &p, int sms, cudaStream_t st) {
    if (s.num_q_heads > 65535) return SPD_ERR_UNSUPPORTED;
    const int64_t tiles = (p.T + 63) / 64 * s.num_q_heads, mean = p.T / s.batch;
    if (2 * tiles <= sms || mean <= 32) return s.head_dim == 128 ? launch_prefill_f32<128, 2, 1>(s, p, st) : launch_prefill_f32<64, 2, 1>(s, p, st);
    if (tiles * 128 < sms * mean) return s.head_dim == 128 ? launch_prefill_f32<128, 4, 2>(s, p, st) : launch_prefill_f32<64, 4, 2>(s, p, st);
    return s.head_dim == 128 ? launch_prefill_f32<128, 4, 1>(s, p, st) : launch_prefill_f32<64, 4, 1>(s, p, st);
}

}  // namespace

extern "C" {

spd_status spd_prefill_attn_scored(const spd_shape *shape, const spd_score *score, int64_t total_tokens, const spd_tokens *tok,
                                   const int32_t *tok_indptr, const int32_t *prefix_lens, const int32_t *doc_start, void *out,
                                   spd_dtype out_dtype, void *ws, size_t ws_bytes, void *cuda_stream) {
    spd_status rc = host::check_shape(shape);
    if (rc != SPD_OK) return rc;
    if ((rc = host::check_score(score)) != SPD_OK) return rc;
    const spd_shape &s = *shape;
    const int64_t T = total_tokens;
    if (!(s.sm_scale > 0.f && s.sm_scale <= 1e30f)) return SPD_ERR_UNSUPPORTED;      // row maxima are taken before scaling
    if (out_dtype != SPD_F32 && out_dtype != SPD_BF16) return SPD_ERR_UNSUPPORTED;
    if (T < 0 || T >= (1ll << 31) - 1024) return SPD_ERR_INVALID_ARG;
    if (!tok || !tok_indptr || !ws || misaligned(ws, 256)) return SPD_ERR_INVALID_ARG;
    if (ws_bytes < HDR_WORDS * 4) return SPD_ERR_WORKSPACE;
    if (T > 0 && (!tok->q || !tok->k || !tok->v || !out)) return SPD_ERR_INVALID_ARG;
    if (misaligned(tok->q, 16) || misaligned(tok->k, 16) || misaligned(tok->v, 16) || misaligned(out, 16)) return SPD_ERR_INVALID_ARG;
    ScoredPrefillParams p{};
    if (!row_stride(s, s.num_q_heads, tok->q_stride, &p.q_stride) || !row_stride(s, s.num_kv_heads, tok->k_stride, &p.k_stride) ||
        !row_stride(s, s.num_kv_heads, tok->v_stride, &p.v_stride))
        return SPD_ERR_INVALID_ARG;
    int sms = 0;
    if ((rc = host::device_sms(&sms)) != SPD_OK) return rc;
    if (T == 0) return SPD_OK;
    p.B = s.batch; p.Hq = s.num_q_heads; p.Hkv = s.num_kv_heads; p.T = T;
    p.sm_scale = s.sm_scale; p.tok_indptr = tok_indptr; p.out = out; p.out_bf16 = out_dtype == SPD_BF16;
    p.hdr = static_cast<int32_t *>(ws);
    p.q = tok->q; p.k = tok->k; p.v = tok->v;
    p.cap = score->logit_cap; p.window = score->window; p.slopes = score->alibi_slopes;
    p.prefix_lens = prefix_lens; p.doc_start = doc_start;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (s.dtype == SPD_BF16) return prefill_tc(s, p, st);
    return prefill_f32(s, p, sms, st);
}

}  // extern "C"

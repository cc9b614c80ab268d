// Attention of drafted tokens: argument checks, choice of the kernel, launches.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "spd_drafted.cuh"
#include "spd_drafted_fma.cuh"
#include "spd_drafted_tc.cuh"
#include "spd_host.h"

namespace {

using namespace spd;
using host::misaligned;

// Query heads that a tile of RT rows takes of one token: all of a KV head's where they fit.
int heads_per_tile(int g, int RT) { return g <= RT ? g : kHeadsPerItem; }

constexpr int kFmaMostPerSm = 4;    // CTAs of an FMA variant that may share an SM
constexpr int kMostFmaRows = 64;
constexpr int kTcOverhead = 6;      // what an item costs beside its blocks, in blocks
constexpr int kFmaOverhead = 0;

// Behind the workspace's head: records and slots of the pieces.
struct DraftedLayout { size_t records, scratch, total; };
DraftedLayout drafted_layout(const spd_shape &s, int sms) {
    const int g = s.num_q_heads / s.num_kv_heads;
    const int seqs = s.batch * s.num_kv_heads * (g > kHeadsPerItem ? g / kHeadsPerItem : 1);
    const bool tc = s.dtype == SPD_BF16;
    const size_t slots = 2 * static_cast<size_t>(tc ? 1 : kFmaMostPerSm) * sms;
    DraftedLayout L;
    L.records = host::cleared_end(s.batch, seqs);
    L.scratch = L.records + (slots * 2 * sizeof(int4) + 255) / 256 * 256;
    L.total = L.scratch + slots * drafted_slot_floats(s.head_dim, tc ? kDtRows : kMostFmaRows) * sizeof(float);
    return L;
}

// A launch that may be set up while the kernel before it is still at work; both kernels wait for that one's end before they read anything.
template <class... Args>
spd_status launch_early(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t st, const Args &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, args...);
    host::count_launch();
    if (err != cudaSuccess) fprintf(stderr, "libspd: launch of a kernel for drafted tokens: %s\n", cudaGetErrorString(err));
    return err == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

template <int D, int RT, bool LOG2>
spd_status launch_join(const DraftedParams &p, cudaStream_t st) {
    return launch_early(drafted_join_kernel<D, RT, LOG2>, dim3(static_cast<unsigned>(p.grid), 2, drafted_join_split(RT)), kDrJoinThreads, 0, st, p);
}

// [T][Hq][D] bf16 as a 3-D map: a box is `tokens` tokens x `heads` heads x 128 bytes, 128-byte swizzle.
spd_status make_q_map(CUtensorMap *map, const DraftedParams &p, int D, int tokens) {
    EncodeTiledFn fn = host::tensor_map_encoder();
    if (!fn) return SPD_ERR_CUDA;
    cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(p.Hq), static_cast<cuuint64_t>(p.T)};
    cuuint64_t strides[2] = {static_cast<cuuint64_t>(D) * 2, static_cast<cuuint64_t>(p.Hq) * D * 2};
    cuuint32_t box[3] = {64u, static_cast<cuuint32_t>(p.hs), static_cast<cuuint32_t>(tokens)};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) fprintf(stderr, "libspd: cuTensorMapEncodeTiled failed with CUresult %d\n", static_cast<int>(r));
    return r == CUDA_SUCCESS ? SPD_OK : SPD_ERR_CUDA;
}

// A pool's rows of one page and head: 16 x 128 bytes, 128-byte swizzle.
spd_status make_pool_map(CUtensorMap *map, const DraftedParams &p, const void *pool, int64_t num_pages, int D) {
    EncodeTiledFn fn = host::tensor_map_encoder();
    if (!fn) return SPD_ERR_CUDA;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(num_pages) * p.Hkv * kPage};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(D) * 2};
    cuuint32_t box[2] = {64u, static_cast<cuuint32_t>(kPage)};
    cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) fprintf(stderr, "libspd: cuTensorMapEncodeTiled failed with CUresult %d\n", static_cast<int>(r));
    return r == CUDA_SUCCESS ? SPD_OK : SPD_ERR_CUDA;
}

uint64_t twice(double x) {              // an fp32 value in both halves of a two-lane operand
    const float f = static_cast<float>(x);
    uint32_t u;
    memcpy(&u, &f, 4);
    return (static_cast<uint64_t>(u) << 32) | u;
}

template <int D, int CAP, bool BIAS>
spd_status launch_tc(const DraftedTcParams &p, const CUtensorMap *maps, cudaStream_t st) {
    static std::once_flag once[64];
    int dev = 0;
    cudaGetDevice(&dev);
    cudaError_t err = cudaSuccess;
    std::call_once(once[dev & 63], [&] {
        err = cudaFuncSetAttribute(drafted_tc_kernel<D, CAP, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(dt_smem_bytes(D)));
    });
    if (err != cudaSuccess) return SPD_ERR_CUDA;
    const spd_status rc = launch_early(drafted_tc_kernel<D, CAP, BIAS>, dim3(static_cast<unsigned>(p.d.grid)), kDtThreads, dt_smem_bytes(D), st, p, maps[0],
                                       maps[1], maps[2], maps[3], maps[4]);
    return rc != SPD_OK ? rc : launch_join<D, kDtRows, true>(p.d, st);
}

spd_status run_tc(const DraftedParams &call, int D, int sms, cudaStream_t st) {
    DraftedTcParams p{};
    p.d = call;
    DraftedParams &d = p.d;
    d.hs = heads_per_tile(d.g, kDtRows / 2);
    d.hgroups = d.g / d.hs;
    p.tpt = kDtRows / 2 / d.hs;
    d.tt = 2 * p.tpt;
    d.SQ = d.Hkv * d.hgroups;
    d.bt = kDtPages;
    d.grid = sms;
    p.c2 = d.sm_scale * kLog2e;
    d.ov = kTcOverhead;
    int cap = 0;
    if (d.cap > 0.f) {
        const double y1 = static_cast<double>(d.sm_scale) / d.cap;
        p.cap2 = d.cap * kLog2e;
        p.y1 = static_cast<float>(fmax(fmin(y1, 1e30), 1.5e-45));      // not 0: infinite scores stay infinite
        bool fits = true;                                 // the coefficients carry the cap
        auto normal = [](double c) { return fabs(c) > 1e-37 && fabs(c) < 1e37; };
        for (int i = 0; i < 6; ++i) {
            const double c = d.cap * 1.4426950408889634 * pow(y1, 2 * i + 1);
            if (i < 4) { p.p1[i] = twice(c * kTanhHalf[i]); fits = fits && normal(c * kTanhHalf[i]); }
            p.p2[i] = twice(c * kTanhOne[i]);             // where a mask comes on top of the cap, this longer one serves both ranges
            fits = fits && normal(c * kTanhOne[i]);
        }
        cap = fits ? 1 : 2;
        for (int i = 0; i < 6 && !fits; ++i) p.p2[i] = twice(kTanhOne[i]);
    }
    // A tile whose rows are done one by one takes its warps about 4 us per key: 64 polls or so, beyond the usual limit.
    const int64_t keys = (static_cast<int64_t>(d.part[0].num_pages) + d.part[1].num_pages) * kPage, polls = static_cast<int64_t>(kWaitLimit) + 64 * keys;
    p.wait_limit = static_cast<uint32_t>(polls < (1ll << 31) ? polls : 1ll << 31);
    CUtensorMap maps[5];
    spd_status rc;
    if ((rc = make_q_map(&maps[0], d, D, p.tpt)) != SPD_OK) return rc;
    for (int x = 0; x < 2; ++x) {
        if (d.part[x].num_pages > 0) {
            if ((rc = make_pool_map(&maps[1 + 2 * x], d, d.k_pool[x], d.part[x].num_pages, D)) != SPD_OK) return rc;
            if ((rc = make_pool_map(&maps[2 + 2 * x], d, d.v_pool[x], d.part[x].num_pages, D)) != SPD_OK) return rc;
        } else {
            maps[1 + 2 * x] = maps[2 + 2 * x] = maps[0];   // never loaded from
        }
    }
    const bool bias = d.slopes != nullptr;
#define SPD_DT_CASE(DD, CC, BB) if (D == DD && cap == CC && bias == BB) return launch_tc<DD, CC, BB>(p, maps, st);
    SPD_DT_CASE(128, 0, false) SPD_DT_CASE(128, 1, false) SPD_DT_CASE(128, 2, false) SPD_DT_CASE(128, 0, true) SPD_DT_CASE(128, 1, true)
    SPD_DT_CASE(128, 2, true) SPD_DT_CASE(64, 0, false) SPD_DT_CASE(64, 1, false) SPD_DT_CASE(64, 2, false) SPD_DT_CASE(64, 0, true)
    SPD_DT_CASE(64, 1, true) SPD_DT_CASE(64, 2, true)
#undef SPD_DT_CASE
    return SPD_ERR_UNSUPPORTED;
}

template <int D, int RT>
spd_status launch_fma(DraftedParams p, int sms, cudaStream_t st) {
    using C = DraftedFma<D, RT>;
    static std::once_flag once[64];
    static int fit[64];                 // CTAs that an SM holds at once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    cudaError_t err = cudaSuccess;
    std::call_once(once[dev], [&] {
        err = cudaFuncSetAttribute(drafted_fma_kernel<D, RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(C::smem_bytes()));
        if (err == cudaSuccess) err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit[dev], drafted_fma_kernel<D, RT>, C::kThreads, C::smem_bytes());
    });
    if (err != cudaSuccess || fit[dev] < 1) return SPD_ERR_CUDA;
    p.hs = heads_per_tile(p.g, RT);
    p.hgroups = p.g / p.hs;
    p.tt = RT / p.hs;
    p.SQ = p.Hkv * p.hgroups;
    p.bt = kDrTiles;
    p.ov = kFmaOverhead;
    p.grid = (fit[dev] < kFmaMostPerSm ? fit[dev] : kFmaMostPerSm) * sms;
    const spd_status rc = launch_early(drafted_fma_kernel<D, RT>, dim3(static_cast<unsigned>(p.grid)), C::kThreads, C::smem_bytes(), st, p);
    return rc != SPD_OK ? rc : launch_join<D, RT, false>(p, st);
}

// Tiles of 16 rows (several CTAs per SM, each with its own keys) or of 64, by the rows of a KV head, on average over the users.  us, 16 / 64 rows,
// 32 users, 4 k tokens: 8 heads of 64, 4 rows 193 / 814, 16 rows 280 / 820, 20 rows (two tiles of 16) 531 / 825, 32 rows 540 / 854, 33 to 48 rows (three
// tiles) 791-796 / 950-960, which the rule leaves to tiles of 64; 32/8 heads of 128, 16 rows 624 / 1140, 20 to 32 rows 1220 / 1150-1169, 40 rows 1828 / 1395.
spd_status run_fma(const DraftedParams &p, int D, int sms, cudaStream_t st) {
    const bool few = p.T * p.g <= (D == 128 ? 16ll : 32ll) * p.B;
    if (D == 128) return few ? launch_fma<128, 16>(p, sms, st) : launch_fma<128, 64>(p, sms, st);
    return few ? launch_fma<64, 16>(p, sms, st) : launch_fma<64, 64>(p, sms, st);
}

spd_status check_part(const spd_shape &s, const spd_paged_kv *kv) {
    if (!kv || kv->num_pages < 0 || !kv->page_indptr || !kv->seq_lens) return SPD_ERR_INVALID_ARG;
    if (kv->num_pages > 0 && (!kv->k_pool || !kv->v_pool)) return SPD_ERR_INVALID_ARG;
    if (misaligned(kv->k_pool, 128) || misaligned(kv->v_pool, 128)) return SPD_ERR_INVALID_ARG;
    if (static_cast<int64_t>(kv->num_pages) * s.num_kv_heads * kPage >= (1ll << 31)) return SPD_ERR_UNSUPPORTED;
    return SPD_OK;
}

// One call: partitions absent from it are null, then peer holds their lengths.
struct DraftedCall {
    const spd_paged_kv *part[2];
    const int32_t *peer[2];
    const spd_partial *pin, *pout;
    void *out;
    spd_dtype out_dtype;
};

spd_status run(const spd_shape *shape, const spd_score *score, const spd_drafts *drafts, const void *q, const DraftedCall &c, void *ws,
               size_t ws_bytes, void *cuda_stream) {
    spd_status rc = host::check_shape(shape);
    if (rc != SPD_OK) return rc;
    if ((rc = host::check_score(score)) != SPD_OK) return rc;
    const spd_shape &s = *shape;
    if (!drafts) return SPD_ERR_INVALID_ARG;
    const int64_t T = drafts->total_tokens;
    for (int x = 0; x < 2; ++x)
        if (c.part[x] && (rc = check_part(s, c.part[x])) != SPD_OK) return rc;
    if (!(s.sm_scale > 0.f && s.sm_scale <= 1e30f)) return SPD_ERR_UNSUPPORTED;
    if (T < 0 || T >= (1ll << 31) - 1024 || drafts->sinks < 0 || (!drafts->tok_indptr && T != s.batch)) return SPD_ERR_INVALID_ARG;
    if (T > 0 && !q) return SPD_ERR_INVALID_ARG;
    if (misaligned(q, 16) || !ws || misaligned(ws, 256)) return SPD_ERR_INVALID_ARG;
    for (const spd_partial *x : {c.pin, c.pout})
        if (x && ((T > 0 && (!x->o || !x->m || !x->l)) || misaligned(x->o, 16) || misaligned(x->m, 4) || misaligned(x->l, 4))) return SPD_ERR_INVALID_ARG;
    if (!c.pout) {
        if ((T > 0 && !c.out) || misaligned(c.out, 16)) return SPD_ERR_INVALID_ARG;
        if (c.out_dtype != SPD_F32 && c.out_dtype != SPD_BF16) return SPD_ERR_UNSUPPORTED;
    }
    int sms = 0;
    if ((rc = host::device_sms(&sms)) != SPD_OK) return rc;
    const DraftedLayout L = drafted_layout(s, sms);
    if (ws_bytes < L.total) return SPD_ERR_WORKSPACE;
    if (T == 0) return SPD_OK;
    const int g = s.num_q_heads / s.num_kv_heads;
    DraftedParams p{};
    p.B = s.batch; p.Hq = s.num_q_heads; p.Hkv = s.num_kv_heads; p.g = g;
    p.T = T; p.sm_scale = s.sm_scale; p.q = q;
    for (int x = 0; x < 2; ++x) {
        if (const spd_paged_kv *kv = c.part[x]) {
            p.part[x] = PartDev{kv->page_indptr, kv->page_indices, kv->seq_lens, kv->num_pages, 1};
            p.k_pool[x] = kv->k_pool;
            p.v_pool[x] = kv->v_pool;
        }
        p.peer_lens[x] = c.peer[x];
    }
    p.tok_indptr = drafts->tok_indptr; p.parents = drafts->parents; p.sinks = drafts->sinks;
    p.cap = score->logit_cap; p.window = score->window; p.slopes = score->alibi_slopes;
    p.mode = c.pout ? OUT_PARTIAL : OUT_FINAL;
    if (c.pout) { p.po = c.pout->o; p.pm = c.pout->m; p.pl = c.pout->l; }
    if (c.pin) { p.in_o = c.pin->o; p.in_m = c.pin->m; p.in_l = c.pin->l; }
    p.out = c.out; p.out_bf16 = c.out_dtype == SPD_BF16;
    p.wide = !misaligned(c.pout ? static_cast<const void *>(p.po) : c.out, 32);
    uint8_t *w = static_cast<uint8_t *>(ws);
    p.hdr = reinterpret_cast<int32_t *>(w);
    p.seqs = s.batch * s.num_kv_heads * (g > kHeadsPerItem ? g / kHeadsPerItem : 1);
    p.records = reinterpret_cast<int4 *>(w + L.records);
    p.scratch = reinterpret_cast<float *>(w + L.scratch);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return s.dtype == SPD_BF16 ? run_tc(p, s.head_dim, sms, st) : run_fma(p, s.head_dim, sms, st);
}

}  // namespace

extern "C" {

spd_status spd_drafted_workspace_size(const spd_shape *shape, size_t *bytes) {
    if (!bytes) return SPD_ERR_INVALID_ARG;
    spd_status rc = spd_workspace_size(shape, bytes);
    if (rc != SPD_OK) return rc;
    int sms = 0;
    if ((rc = host::device_sms(&sms)) != SPD_OK) return rc;
    const size_t own = drafted_layout(*shape, sms).total;
    if (own > *bytes) *bytes = own;
    return SPD_OK;
}

spd_status spd_decode_step_drafted(const spd_shape *shape, const spd_score *score, const spd_drafts *drafts, const void *q,
                                   const spd_paged_kv *priv, const spd_paged_kv *pub, void *out, spd_dtype out_dtype, void *ws,
                                   size_t ws_bytes, void *cuda_stream) {
    if (!priv || !pub) return SPD_ERR_INVALID_ARG;
    const DraftedCall c{{priv, pub}, {nullptr, nullptr}, nullptr, nullptr, out, out_dtype};
    return run(shape, score, drafts, q, c, ws, ws_bytes, cuda_stream);
}

spd_status spd_partial_attn_drafted(const spd_shape *shape, const spd_score *score, const spd_drafts *drafts, const void *q,
                                    const spd_paged_kv *priv, const int32_t *pub_lens, spd_partial out, void *ws, size_t ws_bytes,
                                    void *cuda_stream) {
    if (!priv || !pub_lens) return SPD_ERR_INVALID_ARG;
    const DraftedCall c{{priv, nullptr}, {nullptr, pub_lens}, nullptr, &out, nullptr, SPD_F32};
    return run(shape, score, drafts, q, c, ws, ws_bytes, cuda_stream);
}

spd_status spd_service_attn_merge_drafted(const spd_shape *shape, const spd_score *score, const spd_drafts *drafts, const void *q,
                                          const spd_paged_kv *pub, const int32_t *priv_lens, spd_partial in, void *out,
                                          spd_dtype out_dtype, void *ws, size_t ws_bytes, void *cuda_stream) {
    if (!pub || !priv_lens) return SPD_ERR_INVALID_ARG;
    const DraftedCall c{{nullptr, pub}, {priv_lens, nullptr}, &in, nullptr, out, out_dtype};
    return run(shape, score, drafts, q, c, ws, ws_bytes, cuda_stream);
}

}  // extern "C"

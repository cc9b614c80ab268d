// Append with rotation, and the launch of the scored decode kernels.
#include <type_traits>

#include "spd_host.h"
#include "spd_launch.cuh"
#include "spd_rope.cuh"
#include "spd_short.cuh"

namespace spd {

// Clusters of 1, 2, 4, 8 CTAs of the short kernel that the current device holds at once (a cluster lies within one group of
// SMs, so not every SM can be used by large ones).  Looked up once per device; also raises the kernel's shared-memory limit.
template <class Math>
static const int *short_capacity() {
    static std::once_flag once[64];
    static int fit[64][4];
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    std::call_once(once[dev], [&] {
        if (cudaFuncSetAttribute(attn_short_kernel<Math>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(short_smem_bytes<Math>())) != cudaSuccess)
            return;                                        // nothing fits: the persistent kernel serves the calls
        for (int i = 0; i < 4; ++i) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(1u << i);
            cfg.blockDim = dim3(Math::kWarps * 32);
            cfg.dynamicSmemBytes = short_smem_bytes<Math>();
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = 1u << i;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&fit[dev][i], attn_short_kernel<Math>, &cfg) != cudaSuccess) { fit[dev][i] = 0; cudaGetLastError(); }
        }
    });
    return fit[dev];
}

// How many CTAs of one cluster share a sequence, or 0 where the call is not a short one.  The host does not know the lengths; a
// window, or the pools' size, bounds the tiles of a sequence.  A caller who set the cut or asked for a stored plan gets the
// persistent kernel.
template <class Math>
static int short_cluster(const Params &p, int sms) {
    if (p.plan_mode != PLAN_DERIVE || p.min_tiles != kMinTilesPerWarp || p.uniform) return 0;
    const int64_t seqs = static_cast<int64_t>(p.B) * p.S;
    int64_t tiles = static_cast<int64_t>(p.part[0].num_pages) + p.part[1].num_pages;
    if (p.window > 0 && p.window / kPage + 3 < tiles) tiles = p.window / kPage + 3;      // ragged at both ends and where the partitions meet
    const int *fit = short_capacity<Math>();
    int i = 0;
    while (i < 3 && seqs <= fit[i + 1] && (seqs << (i + 1)) <= sms && tiles > (Math::kWarps << i)) ++i;     // two CTAs of one SM would only slow each other
    return seqs <= fit[i] && tiles <= (static_cast<int64_t>(Math::kWarps) << i) * kShortTiles ? 1 << i : 0;
}

template <class Math>
static spd_status launch_scored(const Params &p, const CUtensorMap *maps, int sms, cudaStream_t st, bool pdl, int cluster) {
    if (cluster == 0) return launch_attn<Math>(p, maps, sms, st, pdl);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.B * p.S * cluster));
    cfg.blockDim = dim3(Math::kWarps * 32);
    cfg.dynamicSmemBytes = short_smem_bytes<Math>();
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 2 : 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, attn_short_kernel<Math>, p, maps[0], maps[1], maps[2], maps[3], cluster);
    host::count_launch();
    if (err != cudaSuccess) fprintf(stderr, "libspd: launch of the short attention kernel: %s\n", cudaGetErrorString(err));
    return err == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

// f(m) with m a (null) pointer to the arithmetic of the call.
template <class F>
static auto with_math(const Params &p, bool bf16, int head_dim, F &&f) -> decltype(f(static_cast<MathBF16<128, true> *>(nullptr))) {
    if (bf16) return head_dim == 128 ? f(static_cast<MathBF16<128, true> *>(nullptr)) : f(static_cast<MathBF16<64, true> *>(nullptr));
#define SPD_F32_CASE(DD, GG) if (head_dim == DD && p.geff == GG) return f(static_cast<MathF32<DD, GG, true> *>(nullptr));
    SPD_F32_CASE(64, 1) SPD_F32_CASE(64, 2) SPD_F32_CASE(64, 4) SPD_F32_CASE(64, 8)
    SPD_F32_CASE(128, 1) SPD_F32_CASE(128, 2) SPD_F32_CASE(128, 4)
#undef SPD_F32_CASE
    return f(static_cast<MathF32<128, 8, true> *>(nullptr));      // check_shape lets no other through
}

int scored_cluster(const Params &p, int sms, bool bf16, int head_dim) {
    return with_math(p, bf16, head_dim, [&](auto *m) { return short_cluster<std::remove_pointer_t<decltype(m)>>(p, sms); });
}

spd_status launch_attn_scored(const Params &p, const CUtensorMap *maps, int sms, cudaStream_t st, bool pdl, bool bf16, int head_dim, int cluster) {
    return with_math(p, bf16, head_dim, [&](auto *m) { return launch_scored<std::remove_pointer_t<decltype(m)>>(p, maps, sms, st, pdl, cluster); });
}

}  // namespace spd

using namespace spd;
using host::elem_size;
using host::misaligned;
using host::row_stride;

extern "C" {

spd_status spd_append_kv_rope(const spd_shape *shape, const spd_rope *rope, int64_t total_tokens, const spd_tokens *tok,
                              const int32_t *tok_indptr, const int32_t *positions, const int32_t *pos_base, void *q_out,
                              void *k_out, void *k_pool, void *v_pool, int32_t num_pages, const int32_t *page_indptr,
                              const int32_t *page_indices, const int32_t *seq_lens, int32_t *new_lens, void *ws,
                              size_t ws_bytes, void *cuda_stream) {
    spd_status rc = host::check_shape(shape);
    if (rc != SPD_OK) return rc;
    const spd_shape &s = *shape;
    const int64_t T = total_tokens;
    if (!tok || !page_indptr || !seq_lens || !ws || misaligned(ws, 256)) return SPD_ERR_INVALID_ARG;
    if (T < 0 || T >= (1ll << 31) || num_pages < 0 || (!tok_indptr && T != s.batch)) return SPD_ERR_INVALID_ARG;
    const int g = s.num_q_heads / s.num_kv_heads, seqs = s.num_kv_heads * (g > kHeadsPerItem ? g / kHeadsPerItem : 1);
    if (ws_bytes < host::cleared_end(s.batch, s.batch * seqs)) return SPD_ERR_WORKSPACE;
    if (T > 0 && (!tok->k || !tok->v || !k_pool || !v_pool || num_pages <= 0)) return SPD_ERR_INVALID_ARG;
    if (misaligned(tok->k, 16) || misaligned(tok->v, 16) || misaligned(k_pool, 128) || misaligned(v_pool, 128)) return SPD_ERR_INVALID_ARG;
    RopeAppendParams p{};
    p.B = s.batch; p.Hkv = s.num_kv_heads; p.D = s.head_dim; p.T = T;
    int64_t qs = 0, ks, vs;
    if (!row_stride(s, s.num_kv_heads, tok->k_stride, &ks) || !row_stride(s, s.num_kv_heads, tok->v_stride, &vs)) return SPD_ERR_INVALID_ARG;
    if (rope) {
        if (rope->rotary_dim <= 0 || rope->rotary_dim > s.head_dim || rope->rotary_dim % 16 != 0) return SPD_ERR_UNSUPPORTED;
        if (rope->num_axes < 1 || rope->num_axes > 4) return SPD_ERR_UNSUPPORTED;
        if (!rope->inv_freq || (rope->interleaved != 0 && rope->interleaved != 1)) return SPD_ERR_INVALID_ARG;
        if (!(rope->scale >= -3e38f && rope->scale <= 3e38f)) return SPD_ERR_INVALID_ARG;
        if ((rope->num_axes > 1 && !positions) || (positions && pos_base)) return SPD_ERR_INVALID_ARG;
        // other CTAs may still read a user's position while its grown length is written
        if (pos_base && pos_base == new_lens) return SPD_ERR_INVALID_ARG;
        if (tok_indptr && positions && positions == new_lens && new_lens != seq_lens) return SPD_ERR_INVALID_ARG;
        if (T > 0 && (!tok->q || !q_out)) return SPD_ERR_INVALID_ARG;
        if (misaligned(tok->q, 16) || misaligned(q_out, 16) || misaligned(k_out, 16)) return SPD_ERR_INVALID_ARG;
        if (!row_stride(s, s.num_q_heads, tok->q_stride, &qs)) return SPD_ERR_INVALID_ARG;
        // in place only where the output's rows are the input's
        if (q_out == tok->q && qs != static_cast<int64_t>(s.num_q_heads) * s.head_dim) return SPD_ERR_INVALID_ARG;
        const int pairs = rope->rotary_dim / 2;
        int at = 0;
        for (int a = 0; a < 4; ++a) {
            if (rope->num_axes > 1 && a < rope->num_axes) {
                if (rope->sections[a] < 0 || rope->sections[a] > pairs) return SPD_ERR_INVALID_ARG;
                at += rope->sections[a];
            }
            p.axis_end[a] = rope->num_axes > 1 ? at : pairs;
        }
        if (rope->num_axes > 1 && at != pairs) return SPD_ERR_INVALID_ARG;
        p.Hq = s.num_q_heads;
        p.q = static_cast<const uint8_t *>(tok->q);
        p.q_out = static_cast<uint8_t *>(q_out);
        p.rot = rope->rotary_dim; p.interleaved = rope->interleaved; p.scale = rope->scale; p.inv_freq = rope->inv_freq;
        p.positions = positions; p.pos_base = pos_base;
    } else if (positions || pos_base || q_out) {
        return SPD_ERR_INVALID_ARG;            // nothing is rotated: these would be ignored silently
    }
    if (k_out && misaligned(k_out, 16)) return SPD_ERR_INVALID_ARG;
    if (k_out && k_out == tok->k && ks != static_cast<int64_t>(s.num_kv_heads) * s.head_dim) return SPD_ERR_INVALID_ARG;
    const int es = elem_size(s);
    p.k = static_cast<const uint8_t *>(tok->k); p.v = static_cast<const uint8_t *>(tok->v);
    p.q_stride = qs * es; p.k_stride = ks * es; p.v_stride = vs * es;
    p.k_out = static_cast<uint8_t *>(k_out);
    p.tok_indptr = tok_indptr;
    p.k_pool = static_cast<uint8_t *>(k_pool); p.v_pool = static_cast<uint8_t *>(v_pool); p.num_pages = num_pages;
    p.indptr = page_indptr; p.indices = page_indices; p.lens = seq_lens; p.new_lens = new_lens;
    p.hdr = static_cast<int32_t *>(ws);
    p.bad = reinterpret_cast<int32_t *>(static_cast<uint8_t *>(ws) + host::flags_offset(s.batch));
    p.epoch = host::next_call_id();
    p.S = seqs;
    int sms = 0;
    if ((rc = host::device_sms(&sms)) != SPD_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (!tok_indptr) {
        if (es == 2) append_rope_kernel<__nv_bfloat16, false><<<s.batch, kRopeThreads, 0, st>>>(p);
        else append_rope_kernel<float, false><<<s.batch, kRopeThreads, 0, st>>>(p);
    } else {
        const unsigned grid = T == 0 ? 1u : static_cast<unsigned>((T + kRopeTokens - 1) / kRopeTokens);
        if (es == 2) append_rope_kernel<__nv_bfloat16, true><<<grid, kRopeThreads, 0, st>>>(p);
        else append_rope_kernel<float, true><<<grid, kRopeThreads, 0, st>>>(p);
    }
    host::count_launch();
    return cudaGetLastError() == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

}  // extern "C"

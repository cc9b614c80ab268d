// Pages of a paged cache and accepted drafted tokens: argument checks and launches.
#include <algorithm>

#include "spd_host.h"
#include "spd_pages.cuh"

namespace {

using namespace spd;
using host::misaligned;

// Behind the workspace's head: a number per user and per chunk, and the free pages.
struct PagesLayout { size_t demand, chunk_free, free, total; };
PagesLayout pages_layout(size_t head, int batch, int num_pages) {
    PagesLayout L;
    L.demand = head;
    L.chunk_free = L.demand + (static_cast<size_t>(batch) * 4 + 255) / 256 * 256;
    L.free = L.chunk_free + kPgMaxChunks * 4;
    L.total = L.free + static_cast<size_t>(num_pages) * 4;
    return L;
}

int seqs_of(const spd_shape &s) {
    const int g = s.num_q_heads / s.num_kv_heads;
    return s.batch * s.num_kv_heads * (g > kHeadsPerItem ? g / kHeadsPerItem : 1);
}

spd_status fill(const spd_shape *shape, int32_t num_pages, int32_t *refs, const int32_t *page_indptr, int32_t *page_indices, void *ws,
                size_t ws_bytes, PagesParams &p, int *sms) {
    spd_status rc = host::check_shape(shape);
    if (rc != SPD_OK) return rc;
    if (num_pages < 0 || num_pages > (1 << 30) || !page_indptr || !ws || misaligned(ws, 256)) return SPD_ERR_INVALID_ARG;
    if (num_pages > 0 && (!refs || !page_indices || misaligned(refs, 16))) return SPD_ERR_INVALID_ARG;
    const PagesLayout L = pages_layout(host::cleared_end(shape->batch, seqs_of(*shape)), shape->batch, num_pages);
    if (ws_bytes < L.total) return SPD_ERR_WORKSPACE;
    if ((rc = host::device_sms(sms)) != SPD_OK) return rc;
    uint8_t *w = static_cast<uint8_t *>(ws);
    p.B = shape->batch; p.num_pages = num_pages; p.refs = refs; p.indptr = page_indptr; p.indices = page_indices;
    const int turn = kPgThreads * 16;               // the chunks are whole turns of a CTA
    p.chunk = std::max(kPgChunk, ((num_pages + kPgMaxChunks - 1) / kPgMaxChunks + turn - 1) / turn * turn);
    p.chunks = (num_pages + p.chunk - 1) / p.chunk;
    p.hdr = reinterpret_cast<int32_t *>(w);
    p.seqs = seqs_of(*shape);
    p.demand = reinterpret_cast<int32_t *>(w + L.demand);
    p.chunk_free = reinterpret_cast<int32_t *>(w + L.chunk_free);
    p.free = reinterpret_cast<int32_t *>(w + L.free);
    return SPD_OK;
}

spd_status hand_out(const PagesParams &p, cudaStream_t st) {
    pages_look_kernel<<<p.chunks + p.B, kPgThreads, 0, st>>>(p);
    host::count_launch();
    if (cudaGetLastError() != cudaSuccess) return SPD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.B));
    cfg.blockDim = dim3(kPgThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, pages_give_kernel, p);
    host::count_launch();
    return err == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

// Every pool is there and aligned, and its pages have a length.
spd_status check_pools(const spd_shape *shape, int32_t num_pools, void *const *pools, int32_t num_pages) {
    spd_status rc = host::check_shape(shape);
    if (rc != SPD_OK) return rc;
    if (num_pools < 0 || num_pages < 0 || (num_pools > 0 && !pools)) return SPD_ERR_INVALID_ARG;
    for (int32_t i = 0; i < num_pools; ++i)
        if ((num_pages > 0 && !pools[i]) || misaligned(pools[i], 128)) return SPD_ERR_INVALID_ARG;
    return SPD_OK;
}

}  // namespace

extern "C" {

spd_status spd_pages_workspace_size(const spd_shape *shape, int32_t num_pages, size_t *bytes) {
    if (!bytes || num_pages < 0 || num_pages > (1 << 30)) return SPD_ERR_INVALID_ARG;
    const spd_status rc = spd_workspace_size(shape, bytes);
    if (rc != SPD_OK) return rc;
    *bytes = std::max(*bytes, pages_layout(host::cleared_end(shape->batch, seqs_of(*shape)), shape->batch, num_pages).total);
    return SPD_OK;
}

spd_status spd_pages_release(const spd_shape *shape, int32_t num_pages, int32_t *refs, const int32_t *page_indptr, int32_t *page_indices,
                             const int32_t *from_tokens, const int32_t *to_tokens, void *ws, size_t ws_bytes, void *cuda_stream) {
    PagesParams p{};
    int sms = 0;
    if (!from_tokens) return SPD_ERR_INVALID_ARG;
    const spd_status rc = fill(shape, num_pages, refs, page_indptr, page_indices, ws, ws_bytes, p, &sms);
    if (rc != SPD_OK) return rc;
    p.from = from_tokens; p.to = to_tokens;
    const int per_user = std::max(1, std::min(32, 2 * sms / p.B));      // a few users may have long tables
    pages_release_kernel<<<dim3(static_cast<unsigned>(p.B), static_cast<unsigned>(per_user)), kPgThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p);
    host::count_launch();
    return cudaGetLastError() == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

spd_status spd_pages_take(const spd_shape *shape, int32_t num_pages, int32_t *refs, const int32_t *page_indptr, int32_t *page_indices,
                          const int32_t *from_tokens, const int32_t *to_tokens, void *ws, size_t ws_bytes, void *cuda_stream) {
    PagesParams p{};
    int sms = 0;
    if (!from_tokens || !to_tokens) return SPD_ERR_INVALID_ARG;
    const spd_status rc = fill(shape, num_pages, refs, page_indptr, page_indices, ws, ws_bytes, p, &sms);
    if (rc != SPD_OK) return rc;
    p.from = from_tokens; p.to = to_tokens;
    return hand_out(p, static_cast<cudaStream_t>(cuda_stream));
}

spd_status spd_pages_fork(const spd_shape *shape, int32_t num_pages, int32_t *refs, const int32_t *page_indptr, int32_t *page_indices,
                          int32_t *seq_lens, const int32_t *source, int32_t *copies, void *ws, size_t ws_bytes, void *cuda_stream) {
    PagesParams p{};
    int sms = 0;
    if (!seq_lens || !source || !copies) return SPD_ERR_INVALID_ARG;
    const spd_status rc = fill(shape, num_pages, refs, page_indptr, page_indices, ws, ws_bytes, p, &sms);
    if (rc != SPD_OK) return rc;
    p.lens = seq_lens; p.source = source; p.copies = copies;
    return hand_out(p, static_cast<cudaStream_t>(cuda_stream));
}

spd_status spd_pages_copy(const spd_shape *shape, int32_t num_pools, void *const *pools, int32_t num_pages, int32_t num_copies,
                          const int32_t *copies, void *ws, size_t ws_bytes, void *cuda_stream) {
    spd_status rc = check_pools(shape, num_pools, pools, num_pages);
    if (rc != SPD_OK) return rc;
    if (num_copies < 0 || (num_copies > 0 && !copies) || !ws || misaligned(ws, 256)) return SPD_ERR_INVALID_ARG;
    if (ws_bytes < HDR_WORDS * 4) return SPD_ERR_WORKSPACE;
    int sms = 0;
    if ((rc = host::device_sms(&sms)) != SPD_OK) return rc;
    const int64_t page_bytes = static_cast<int64_t>(shape->num_kv_heads) * kPage * shape->head_dim * host::elem_size(*shape);
    const int64_t pieces = (page_bytes + kPgPiece - 1) / kPgPiece;
    if (pieces > 65535) return SPD_ERR_UNSUPPORTED;
    for (int32_t at = 0; at < num_pools && num_copies > 0; at += kPgPools) {
        PagesPools some{};
        const int n = std::min(num_pools - at, static_cast<int32_t>(kPgPools));
        std::copy(pools + at, pools + at + n, some.pool);
        pages_copy_kernel<<<dim3(static_cast<unsigned>(num_copies), static_cast<unsigned>(n), static_cast<unsigned>(pieces)), kPgThreads, 0,
                            static_cast<cudaStream_t>(cuda_stream)>>>(some, copies, num_pages, page_bytes, static_cast<int32_t *>(ws));
        host::count_launch();
        if (cudaGetLastError() != cudaSuccess) return SPD_ERR_CUDA;
    }
    return SPD_OK;
}

spd_status spd_keep_drafted(const spd_shape *shape, int64_t total_tokens, const int32_t *tok_indptr, const int32_t *parents, const int32_t *last,
                            int32_t num_pools, void *const *pools, int32_t num_pages, const int32_t *page_indptr, const int32_t *page_indices,
                            const int32_t *seq_lens, int32_t *new_lens, int32_t *kept, void *ws, size_t ws_bytes, void *cuda_stream) {
    spd_status rc = check_pools(shape, num_pools, pools, num_pages);
    if (rc != SPD_OK) return rc;
    const spd_shape &s = *shape;
    if (total_tokens < 0 || total_tokens >= (1ll << 31) || (!tok_indptr && total_tokens != s.batch)) return SPD_ERR_INVALID_ARG;
    if (!last || !page_indptr || !seq_lens || !ws || misaligned(ws, 256)) return SPD_ERR_INVALID_ARG;
    if (kept && (kept == tok_indptr || kept == parents || kept == last || kept == seq_lens)) return SPD_ERR_INVALID_ARG;
    if (new_lens && (new_lens == tok_indptr || new_lens == parents || new_lens == last || new_lens == kept)) return SPD_ERR_INVALID_ARG;
    const PagesLayout L = pages_layout(host::cleared_end(s.batch, seqs_of(s)), s.batch, 0);
    if (ws_bytes < L.total) return SPD_ERR_WORKSPACE;
    int sms = 0;
    if ((rc = host::device_sms(&sms)) != SPD_OK) return rc;
    KeepParams p{};
    p.B = s.batch; p.Hkv = s.num_kv_heads; p.row_bytes = s.head_dim * host::elem_size(s); p.num_pages = num_pages; p.T = total_tokens;
    p.tok_indptr = tok_indptr; p.parents = parents; p.last = last;
    p.indptr = page_indptr; p.indices = page_indices; p.lens = seq_lens;
    p.hdr = static_cast<int32_t *>(ws);
    p.seqs = seqs_of(s);
    p.result = reinterpret_cast<int32_t *>(static_cast<uint8_t *>(ws) + L.demand);
    const int per = kPgThreads / (p.row_bytes / 16);
    for (int32_t at = 0; at == 0 || at < num_pools; at += kPgPools) {
        PagesPools some{};
        p.num_pools = std::min(num_pools - at, static_cast<int32_t>(kPgPools));
        std::copy(pools + at, pools + at + p.num_pools, some.pool);
        const bool end = at + kPgPools >= num_pools;                    // the lengths change with the last pools
        p.new_lens = end ? new_lens : nullptr;
        p.kept = end ? kept : nullptr;
        const int64_t heads = static_cast<int64_t>(p.num_pools) * s.num_kv_heads;
        // A CTA finds its user's branch by a chain of loads before it moves anything: about two rounds of CTAs, each over several heads, where there
        // are many users (512 users, 16 layers: 47 us with a CTA for every 16 heads).
        const int64_t most = (heads + per - 1) / per, some_of = std::max<int64_t>(1, 16ll * sms / s.batch);
        const unsigned y = parents ? static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(1024, most), some_of))) : 1u;
        keep_kernel<<<dim3(static_cast<unsigned>(s.batch), y), kPgThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p, some);
        host::count_launch();
        if (cudaGetLastError() != cudaSuccess) return SPD_ERR_CUDA;
    }
    return SPD_OK;
}

}  // extern "C"

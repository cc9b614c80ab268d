// Append with the position rotation on the way: q and k rows of the new tokens are rotated, k and v rows written to the
// paged cache, lengths grown, in one launch.
//
// Bound by HBM (long prompts: every row once in, q, a packed k and the cache rows once out) or by latency (one token
// per user).  A row of a head is cut into units of two 16-byte chunks that rotate together -- chunks c and c + rotary_dim / 2,
// or neighbours when neighbouring channels pair up -- so that a thread loads, turns and stores 32 bytes without talking to
// anybody, and keeps the sines and cosines of its unit in registers while it walks the token's heads.  Angles: the turns
// pos * inv_freq / 2 pi are formed in 64 bits and reduced to [-1/2, 1/2] there (a position of 10^5 leaves 32 bits no
// fraction to speak of), then sincospif; once per token and pair, shared by all heads.
// Measured: 8 prompts, 53 k tokens of 32/8 heads, head_dim 128, bf16 (1.42 GB) 258 us, 5.5 TB/s; rows in flight per thread 2 / 3 / 4:
// 269 / 258 / 259 us, tokens per CTA 2 / 4 / 8: 306 / 258 / 255, and 7.0 / 7.4 / 9.2 us for 1800 tokens; without loading rows ahead of
// the search 327.  One token for each of 512 users (22 MB, L2) 6.2 us, of 8 users 3.6 us.
#pragma once

#include "spd_device.cuh"

namespace spd {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;        // tokens per CTA when users bring runs of tokens

struct RopeAppendParams {
    int32_t B, Hq, Hkv, D;
    int64_t T;
    const uint8_t *q, *k, *v;                 // rows of a token: heads * D elements, strides below in bytes
    int64_t q_stride, k_stride, v_stride;
    uint8_t *q_out, *k_out;                   // packed; k_out may be null; no q rows at all when Hq == 0
    const int32_t *tok_indptr, *positions, *pos_base;
    const float *inv_freq;
    int32_t rot, interleaved;                 // rot = 0: nothing is rotated
    int32_t axis_end[4];                      // pairs [axis_end[a - 1], axis_end[a]) go by axis a
    float scale;
    uint8_t *k_pool, *v_pool;
    int32_t num_pages;
    const int32_t *indptr, *indices, *lens;
    int32_t *new_lens;
    int32_t *hdr, *bad;
    int32_t epoch, S;
};

// Byte offset, in a pool, of (page, KV head 0, slot) for position t of a user, or -1; `room` positions are listed.
__device__ __forceinline__ int64_t rope_row_offset(const RopeAppendParams &p, int64_t lo, int64_t t, int row_bytes) {
    const int64_t page = p.indices[lo + t / kPage];
    if (page < 0 || page >= p.num_pages) return -1;
    return (page * p.Hkv * kPage + t % kPage) * row_bytes;
}

// Whether user u can take n more tokens; lo = its first page-table entry, held = what it holds.
__device__ __forceinline__ bool rope_user_room(const RopeAppendParams &p, int u, int64_t n, int64_t &lo, int64_t &held) {
    const int64_t hi = p.indptr[u + 1], end = p.indptr[p.B];
    lo = p.indptr[u];
    held = p.lens[u];
    return lo >= 0 && hi >= lo && hi <= end && held >= 0 && held + n <= (hi - lo) * kPage && held + n <= 0x7fffffff &&
           (n == 0 || p.indices != nullptr);
}

// Cosine and sine of pair i of token tok.
__device__ __forceinline__ float2 rope_turn(const RopeAppendParams &p, int64_t tok, int64_t pos, int i) {
    if (p.positions != nullptr) {
        int a = 0;
        while (a < 3 && i >= p.axis_end[a]) ++a;
        pos = p.positions[a * p.T + tok];
    }
    double turns = static_cast<double>(pos) * (static_cast<double>(p.inv_freq[i]) * 0.15915494309189533577);   // / 2 pi
    turns -= rint(turns);
    float s, c;
    sincospif(static_cast<float>(2.0 * turns), &s, &c);
    return make_float2(c * p.scale, s * p.scale);
}

template <typename E> __device__ __forceinline__ void rope_rotate(uint4 &a, uint4 &b, const float2 *cs, bool interleaved);
template <> __device__ __forceinline__ void rope_rotate<float>(uint4 &a, uint4 &b, const float2 *cs, bool interleaved) {
    float x[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                  __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e0 = interleaved ? 2 * i : i, e1 = interleaved ? 2 * i + 1 : i + 4;
        y[e0] = fmaf(x[e0], cs[i].x, -(x[e1] * cs[i].y));
        y[e1] = fmaf(x[e1], cs[i].x, x[e0] * cs[i].y);
    }
    a = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
    b = make_uint4(__float_as_uint(y[4]), __float_as_uint(y[5]), __float_as_uint(y[6]), __float_as_uint(y[7]));
}
template <> __device__ __forceinline__ void rope_rotate<__nv_bfloat16>(uint4 &a, uint4 &b, const float2 *cs, bool interleaved) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (interleaved) {          // a word holds one pair
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]));
            w[i] = pack_bf16(fmaf(x.x, cs[i].x, -(x.y * cs[i].y)), fmaf(x.y, cs[i].x, x.x * cs[i].y));
        }
    } else {                    // words i of a and of b hold pairs 2i and 2i + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]));
            const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i + 4]));
            w[i] = pack_bf16(fmaf(x.x, cs[2 * i].x, -(y.x * cs[2 * i].y)), fmaf(x.y, cs[2 * i + 1].x, -(y.y * cs[2 * i + 1].y)));
            w[i + 4] = pack_bf16(fmaf(y.x, cs[2 * i].x, x.x * cs[2 * i].y), fmaf(y.y, cs[2 * i + 1].x, x.y * cs[2 * i + 1].y));
        }
    }
    a = make_uint4(w[0], w[1], w[2], w[3]);
    b = make_uint4(w[4], w[5], w[6], w[7]);
}

// E: element type.  Runs: users bring runs of tokens (tok_indptr), kRopeTokens tokens per CTA; else one CTA per user.
template <typename E, bool Runs>
__global__ void __launch_bounds__(kRopeThreads, 4) append_rope_kernel(const __grid_constant__ RopeAppendParams p) {
    constexpr int NT = Runs ? kRopeTokens : 1, CH = 16 / sizeof(E);     // CH channels per 16-byte chunk = pairs per unit
    __shared__ float2 cs[NT][64];
    __shared__ int64_t row_off[NT];          // byte offset of the token's slot in a pool, -1 = not written
    __shared__ int64_t tok_pos[NT];
    __shared__ int32_t tok_user[NT];
    __shared__ int32_t first_bad;            // Runs: first user at which tok_indptr is inconsistent
    __shared__ int32_t last_cta;
    const int tid = threadIdx.x;
    const int row_bytes = p.D * static_cast<int>(sizeof(E));
    const int64_t tok0 = static_cast<int64_t>(blockIdx.x) * NT;
    const int nt = Runs ? static_cast<int>(min(static_cast<int64_t>(NT), p.T - tok0)) : 1;
    bool consistent = true;
    if (blockIdx.x == 0 && tid == 0) {       // the status query clears the flags of that many users
        p.hdr[HDR_BATCH] = p.B;
        p.hdr[HDR_NSEQ] = p.B * p.S;
    }

    // A thread keeps to one token and one unit (two 16-byte chunks) and walks that token's rows: q heads, then k heads, then v
    // heads.  The first rows are asked for before anybody knows where they go: finding a token's user, page and angles is a
    // chain of loads that those rows need not wait for.
    constexpr int TPT = kRopeThreads / NT, PB = Runs ? 3 : 2;      // threads per token, rows in flight per thread
    const int units = row_bytes / 32, ru = p.rot / (2 * CH);
    const int my = tid / TPT, j = tid % units, r0 = (tid % TPT) / units, dr = TPT / units;
    const bool turn = j < ru;
    const int c0 = (turn && !p.interleaved ? j : 2 * j) * 16, c1 = (turn && !p.interleaved ? j + ru : 2 * j + 1) * 16;
    const int rows = my < nt ? p.Hq + 2 * p.Hkv : 0;
    const int64_t tok = tok0 + my;
    uint4 a[PB], b[PB];
    auto load = [&](int base) {
#pragma unroll
        for (int x = 0; x < PB; ++x) {
            const int r = base + x * dr;
            if (r >= rows) continue;
            const bool is_q = r < p.Hq, is_v = r >= p.Hq + p.Hkv;
            const uint8_t *src = is_q ? p.q + tok * p.q_stride + static_cast<int64_t>(r) * row_bytes
                                : is_v ? p.v + tok * p.v_stride + static_cast<int64_t>(r - p.Hq - p.Hkv) * row_bytes
                                       : p.k + tok * p.k_stride + static_cast<int64_t>(r - p.Hq) * row_bytes;
            a[x] = *reinterpret_cast<const uint4 *>(src + c0);
            b[x] = *reinterpret_cast<const uint4 *>(src + c1);
        }
    };
    load(r0);

    if constexpr (Runs) {
        // one pass over tok_indptr finds every token's user and any inconsistency
        if (tid == 0) first_bad = p.B;
        if (tid < NT) tok_user[tid] = -1;
        __syncthreads();
        for (int u = tid; u < p.B; u += kRopeThreads) {
            const int64_t a = p.tok_indptr[u], b = p.tok_indptr[u + 1];
            if (b < a || (u == 0 && a != 0) || (u == p.B - 1 && b != p.T)) atomicMin(&first_bad, u);
#pragma unroll
            for (int i = 0; i < NT; ++i)
                if (i < nt && a <= tok0 + i && tok0 + i < b) tok_user[i] = u;
        }
        __syncthreads();
        consistent = first_bad == p.B;
        if (!consistent && blockIdx.x == 0 && tid == 0) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, first_bad);
        if (tid < nt && consistent) {
            const int u = tok_user[tid];
            const int64_t a = p.tok_indptr[u], n = p.tok_indptr[u + 1] - a, i = tok0 + tid - a;
            int64_t lo, held, off = -1;
            const bool room = rope_user_room(p, u, n, lo, held);
            if (room) off = rope_row_offset(p, lo, held + i, row_bytes);
            if (off < 0) {
                p.bad[u] = p.epoch;
                flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);
            }
            row_off[tid] = off;
            tok_pos[tid] = (p.pos_base ? p.pos_base[u] : 0) + held + i;
        }
    } else if (tid == 0) {
        const int u = blockIdx.x;
        int64_t lo, held, off = -1;
        if (rope_user_room(p, u, 1, lo, held)) off = rope_row_offset(p, lo, held, row_bytes);
        if (off < 0) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);
        row_off[0] = off;
        tok_pos[0] = (p.pos_base ? p.pos_base[u] : 0) + held;
    }
    __syncthreads();

    if (consistent) {
        const int pairs = p.rot / 2;
        for (int x = tid; x < nt * pairs; x += kRopeThreads) {
            const int i = x / pairs, pr = x - i * pairs;
            cs[i][pr] = rope_turn(p, tok0 + i, tok_pos[i], pr);
        }
        __syncthreads();
        if (my < nt) {
            const int64_t off = row_off[my];
            float2 w[CH];
            if (turn) {
#pragma unroll
                for (int e = 0; e < CH; ++e) w[e] = cs[my][j * CH + e];
            }
            for (int base = r0; base < rows; base += PB * dr) {
                if (base != r0) load(base);
#pragma unroll
                for (int x = 0; x < PB; ++x) {
                    const int r = base + x * dr;
                    if (r >= rows) continue;
                    const bool is_q = r < p.Hq, is_v = r >= p.Hq + p.Hkv;
                    const int h = is_q ? r : (is_v ? r - p.Hq - p.Hkv : r - p.Hq);
                    if (turn && !is_v) rope_rotate<E>(a[x], b[x], w, p.interleaved != 0);
                    uint8_t *packed = is_q ? p.q_out + (tok * p.Hq + h) * row_bytes
                                           : (!is_v && p.k_out ? p.k_out + (tok * p.Hkv + h) * row_bytes : nullptr);
                    if (packed) {
                        *reinterpret_cast<uint4 *>(packed + c0) = a[x];
                        *reinterpret_cast<uint4 *>(packed + c1) = b[x];
                    }
                    if (!is_q && off >= 0) {
                        uint8_t *slot = (is_v ? p.v_pool : p.k_pool) + off + static_cast<int64_t>(h) * kPage * row_bytes;
                        *reinterpret_cast<uint4 *>(slot + c0) = a[x];
                        *reinterpret_cast<uint4 *>(slot + c1) = b[x];
                    }
                }
            }
        }
    }
    // A decode call may read lengths and rows before this kernel counts as finished for its stream (its preamble runs
    // ahead); it cannot start before every CTA here has left, so what is fenced here is there, for TMA reads too.
    if constexpr (!Runs) {
        if (tid == 0 && p.new_lens != nullptr) p.new_lens[blockIdx.x] = p.lens[blockIdx.x] + (row_off[0] >= 0 ? 1 : 0);
        __threadfence();
        asm volatile("fence.proxy.async.global;" ::: "memory");
    } else {
        if (p.new_lens != nullptr && p.new_lens != p.lens) {
            // grown lengths to another array: the CTA with a user's first token looks over that user's pages and writes its entry
            for (int i = 0; i < nt && consistent; ++i) {
                const int u = tok_user[i];
                const int64_t a0 = p.tok_indptr[u], n = p.tok_indptr[u + 1] - a0;
                if (a0 != tok0 + i) continue;
                int64_t lo, held;
                bool good = rope_user_room(p, u, n, lo, held);
                if (good)
                    for (int64_t x = held / kPage + tid; x <= (held + n - 1) / kPage; x += kRopeThreads) {
                        const int page = p.indices[lo + x];
                        good = good && page >= 0 && page < p.num_pages;
                    }
                good = __syncthreads_and(good);
                if (tid == 0) p.new_lens[u] = static_cast<int32_t>(held + (good ? n : 0));
            }
            if (blockIdx.x == 0)           // users without tokens, and everybody where nothing is appended
                for (int u = tid; u < p.B; u += kRopeThreads) {
                    if (consistent && p.tok_indptr[u + 1] != p.tok_indptr[u]) continue;
                    int64_t lo, held;
                    if (!rope_user_room(p, u, 0, lo, held) && consistent) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);
                    p.new_lens[u] = static_cast<int32_t>(held);
                }
        }
        __threadfence();
        asm volatile("fence.proxy.async.global;" ::: "memory");
        if (p.new_lens != p.lens) return;
        // in place: the lengths grow once nobody reads them any more, so the last CTA out does it
        __syncthreads();
        if (tid == 0) last_cta = atomicAdd(&p.hdr[HDR_GRID_EXITS], 1) == static_cast<int32_t>(gridDim.x) - 1;
        __syncthreads();
        if (!last_cta) return;
        __threadfence();
        if (tid == 0) p.hdr[HDR_GRID_EXITS] = 0;
        for (int u = tid; u < p.B; u += kRopeThreads) {
            const int64_t n = consistent ? p.tok_indptr[u + 1] - p.tok_indptr[u] : 0;
            int64_t lo, held;
            const bool flagged = __ldcg(p.bad + u) == p.epoch, ok = rope_user_room(p, u, n, lo, held) && !flagged;
            if (flagged) p.bad[u] = 0;         // a captured call keeps its id: the next replay starts without it
            if (!ok && n == 0 && consistent) flag_error(p.hdr, 4 /* SPD_ERR_BAD_PAGE */, u);    // an inconsistent table
            p.new_lens[u] = static_cast<int32_t>(held + (ok ? n : 0));
        }
        __threadfence();
    }
}

}  // namespace spd

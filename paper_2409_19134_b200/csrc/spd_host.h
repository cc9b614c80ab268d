// What the library's translation units share on the host: argument checks, device facts, launch accounting, the
// workspace's head and the tensor-map encoder.  Defined in spd_api.cu; not part of the C ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include "spd.h"
#include "spd_device.cuh"

namespace spd {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

namespace host {

spd_status check_shape(const spd_shape *s);
spd_status check_score(const spd_score *score);
spd_status device_sms(int *sms);               // also makes the current device's context current on the calling thread
EncodeTiledFn tensor_map_encoder();            // null if the driver has none
int32_t next_call_id();                        // non-zero id of a call (flags in the workspace hold it)
void count_launch();
size_t flags_offset(int batch);                // per-user flags in the workspace
size_t cleared_end(int batch, int seqs);       // first byte behind what a status query clears after a call over so many sequences

inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

inline int elem_size(const spd_shape &s) { return s.dtype == SPD_BF16 ? 2 : 4; }

// Strides of a token's rows in elements (0 = packed); false if they do not fit the rows or their alignment.
inline bool row_stride(const spd_shape &s, int heads, int64_t given, int64_t *stride) {
    const int64_t row = static_cast<int64_t>(heads) * s.head_dim;
    *stride = given == 0 ? row : given;
    return *stride >= row && *stride < (1ll << 31) && *stride * elem_size(s) % 16 == 0;
}

}  // namespace host

// The scored attention kernels (spd_scored.cu), bf16 or fp32, by head_dim and group.  scored_cluster: CTAs that share a sequence where
// the call takes the cluster kernel, 0 where it takes the persistent one.
int scored_cluster(const Params &p, int sms, bool bf16, int head_dim);
spd_status launch_attn_scored(const Params &p, const CUtensorMap *maps, int sms, cudaStream_t st, bool pdl, bool bf16, int head_dim, int cluster);

}  // namespace spd

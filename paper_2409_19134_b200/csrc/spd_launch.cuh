// Launch of the persistent attention kernel, shared by the translation units that instantiate it.
#pragma once

#include <cstdio>
#include <mutex>

#include "spd_host.h"
#include "spd_kernels.cuh"

namespace spd {

template <class Math>
static spd_status launch_attn(const Params &p_in, const CUtensorMap *maps, int sms, cudaStream_t st, bool pdl) {
    if (sms > kMaxGrid) return SPD_ERR_UNSUPPORTED;
    Params p = p_in;
    p.num_warps = sms * Math::kWarps;   // the plan cuts the tile stream into one share per warp of THIS grid
    // At least 117 KB, so that an SM never holds two of these CTAs whatever the variant needs: the kernel's
    // reasoning about which launch can still be running when the next but one starts rests on one CTA per SM.
    const size_t smem = attn_smem_bytes<Math>(sms) > 117 * 1024 ? attn_smem_bytes<Math>(sms) : 117 * 1024;
    static std::once_flag once[64];
    int dev = 0;
    cudaGetDevice(&dev);
    cudaError_t attr_err = cudaSuccess;
    std::call_once(once[dev & 63], [&] {
        attr_err = cudaFuncSetAttribute(attn_kernel<Math>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        static_cast<int>(smem));
    });
    if (attr_err != cudaSuccess) {
        fprintf(stderr, "libspd: cudaFuncSetAttribute(dynamic shared memory %zu): %s\n", smem, cudaGetErrorString(attr_err));
        return SPD_ERR_CUDA;
    }
    // Programmatic stream serialisation (pdl): this kernel's read-only preamble may overlap the tail of the
    // previous kernel on the stream if that kernel allows it (the attention kernel does).
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sms);
    cfg.blockDim = dim3(Math::kWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 1 : 0;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, attn_kernel<Math>, p, maps[0], maps[1], maps[2], maps[3]);
    host::count_launch();
    if (err != cudaSuccess) fprintf(stderr, "libspd: launch of the attention kernel: %s\n", cudaGetErrorString(err));
    return err == cudaSuccess ? SPD_OK : SPD_ERR_CUDA;
}

}  // namespace spd

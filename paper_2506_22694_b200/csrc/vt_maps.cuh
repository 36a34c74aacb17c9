// The driver's functions that encode tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <mutex>

namespace vt {
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

typedef CUresult (*ReplaceAddressFn)(CUtensorMap*, void*);

struct MapFns {
    EncodeTiledFn encode;
    ReplaceAddressFn replace;
};

const MapFns& map_fns() {
    static std::mutex mu;
    static MapFns fns{nullptr, nullptr};
    std::lock_guard<std::mutex> lock(mu);
    if (!fns.encode) {
        void *e = nullptr, *r = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapReplaceAddress", &r, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fns.replace = reinterpret_cast<ReplaceAddressFn>(r);
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &e, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess && fns.replace)
            fns.encode = reinterpret_cast<EncodeTiledFn>(e);
    }
    return fns;
}

}  // namespace
}  // namespace vt

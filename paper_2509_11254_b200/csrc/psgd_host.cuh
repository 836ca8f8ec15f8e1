// Host-side helpers shared by the translation units of the library.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <map>
#include <mutex>
#include <utility>

namespace {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Multiprocessors of the current device; 148 (a B200) when no device is visible, so that a handle can still be
// created and sized on a machine without one.
inline int device_sms() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && sms > 0)
        return sms;
    cudaGetLastError();
    return 148;
}

// Opt a kernel in to `bytes` of dynamic shared memory: the attribute is set once per (device, kernel) and raised
// only when a larger size is asked for.  C entry points call it: where there is no memory to note that down, it is set again every time.
inline void set_smem_attr(const void* kernel, size_t bytes) noexcept {
    const auto set = [&] {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess) return true;
        cudaGetLastError();                           // (the launch will say why)
        return false;
    };
    int dev = 0;
    cudaGetDevice(&dev);
    try {
        static std::mutex mu;
        static std::map<std::pair<int, const void*>, size_t> done;
        std::lock_guard<std::mutex> lock(mu);
        size_t& have = done[std::make_pair(dev, kernel)];
        if (bytes > have && set()) have = bytes;
    } catch (...) {
        set();
    }
}
template <typename K>
void allow_smem(K kernel, size_t bytes) {
    if (bytes > 48 * 1024) set_smem_attr((const void*)kernel, bytes);
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qr;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qr) == cudaSuccess &&
            qr == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)p;
    }
    return fn;
}

}  // namespace

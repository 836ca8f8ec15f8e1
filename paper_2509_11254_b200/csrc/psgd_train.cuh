// What the translation units of the training operators share on the host: errors of calls that have no handle, extents, overlap of matrices, launches.
#pragma once
#include "../../include/psgd.h"

#include <algorithm>
#include <initializer_list>

#include "psgd_host.cuh"

namespace psgd {

// Keeps the text for psgd_training_cuda_error (per thread) and returns PSGD_E_CUDA.
__attribute__((visibility("hidden"))) psgd_status cuda_error(const char* what, const char* why);
inline bool succeeded(const char* what, cudaError_t e) {
    if (e == cudaSuccess) return true;
    cuda_error(what, cudaGetErrorString(e));
    cudaGetLastError();                               // not left for whoever asks next
    return false;
}

constexpr int64_t MAX_EXTENT = (int64_t)1 << 30;
inline bool extent_ok(int64_t v) { return v >= 1 && v <= MAX_EXTENT; }
inline bool dtype_ok(int dtype) { return dtype == PSGD_DT_F32 || dtype == PSGD_DT_BF16; }
inline int size_of(int dtype) { return dtype == PSGD_DT_F32 ? 4 : 2; }

// Launch that may start before the kernel in front of it on the stream has finished (the kernels wait for that themselves).
template <typename... Params, typename... Args>
bool launch(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t c{};
    c.gridDim = grid; c.blockDim = block; c.dynamicSmemBytes = smem; c.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &at;
    c.numAttrs = 1;
    return succeeded("kernel launch", cudaLaunchKernelEx(&c, kernel, Params(args)...));
}

// Bytes of a matrix in memory: `rows` stretches of `width`, `step` apart (width <= step).
struct Stretch { const void* p; int64_t rows, width, step; };
inline bool overlap(const Stretch& a, const Stretch& b) {
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
    if (a.rows > b.rows) return overlap(b, a);
    const int64_t at = (int64_t)((uintptr_t)a.p - (uintptr_t)b.p);               // of a's first row, from b's
    const int64_t end_a = at + (a.rows - 1) * a.step + a.width, end_b = (b.rows - 1) * b.step + b.width;
    if (at >= end_b || end_a <= 0) return false;
    // rows that lie between one another (columns of one wider matrix): row by row; with equal steps the first rows that face each other speak for all but the ends
    const auto meets = [&](int64_t i) {
        const int64_t x = at + i * a.step;                                       // the first row of b that ends behind x
        const int64_t j = x < b.width ? 0 : (x - b.width) / b.step + 1;
        return j < b.rows && j * b.step < x + a.width;
    };
    const int64_t first = at >= 0 ? 0 : std::min(a.rows - 1, -at / a.step);
    for (int64_t i = first; i < (a.step == b.step ? std::min(a.rows, first + 2) : a.rows); ++i)
        if (meets(i)) return true;
    return a.step == b.step && meets(a.rows - 1);
}
inline Stretch stretch(const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes) { return {p, rows, cols * bytes, (rows == 1 ? cols : ld) * bytes}; }
inline Stretch stretch(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }
// Whether an output lies over an input or over another output (nullptr: not there).
inline bool outputs_meet(std::initializer_list<Stretch> out, std::initializer_list<Stretch> in) {
    const auto end = [](const Stretch& s) { return (uintptr_t)s.p + (uintptr_t)((s.rows - 1) * s.step + s.width); };
    for (const Stretch* o = out.begin(); o != out.end(); ++o) {
        if (!o->p) continue;
        const uintptr_t from = (uintptr_t)o->p, to = end(*o);
        const auto meets = [&](const Stretch& s) { return from < end(s) && (uintptr_t)s.p < to && overlap(*o, s); };     // (mostly far apart)
        for (const Stretch& i : in)
            if (meets(i)) return true;
        for (const Stretch* p = out.begin(); p != o; ++p)
            if (meets(*p)) return true;
    }
    return false;
}

}  // namespace psgd

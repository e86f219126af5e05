// Host side of the token operators' entry points: argument checks, status of a call, launches.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <cstdio>

#include "../../include/pb.h"

namespace pb {

int fail_text(int code, const char* text);      // pb_api.cu: what pb_last_error(NULL) returns

// The status of a call from its launches' own: cudaGetLastError() may still hold what an earlier call of this library
// has failed with and reported.
inline int launched(const char* who, cudaError_t e) {
    if (e == cudaSuccess) return PB_OK;
    cudaGetLastError();                                      // reported here, so not again
    char text[256];
    snprintf(text, sizeof text, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return fail_text(PB_E_CUDA, text);
}

inline size_t dtype_bytes(int dtype) { return dtype == PB_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == PB_F32 || dtype == PB_BF16 || dtype == PB_F16; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxCount = 0x7fffffff;       // rows, tokens, vocabulary, dimension
constexpr int kSms = 148;                       // of a B200: what splits and waves are cut for; any number is right

// Bytes from the first element of a [rows, cols] matrix with row stride ld to behind its last.
inline size_t extent(int64_t rows, int64_t cols, int64_t ld, size_t elem) {
    return rows > 0 && cols > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem : 0;
}
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na && nb && x < y + nb && y < x + na;
}

template <typename... P, typename... A>
cudaError_t launch(const cudaLaunchAttribute* attr, void (*kernel)(P...), dim3 grid, int threads, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3((unsigned)threads);
    c.stream = stream;
    c.attrs = const_cast<cudaLaunchAttribute*>(attr);
    c.numAttrs = attr != nullptr;
    return cudaLaunchKernelEx(&c, kernel, P(args)...);
}
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t stream, A... args) {
    return launch(nullptr, kernel, grid, threads, stream, args...);
}

// Launch that may begin while the launch before it in the stream ends; the kernel waits for that
// launch's results itself (cudaGridDependencySynchronize).
template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t stream, A... args) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    return launch(&attr, kernel, grid, threads, stream, args...);
}

// Launch of `blocks` blocks in clusters of `size`.
template <typename... P, typename... A>
cudaError_t launch_cluster(void (*kernel)(P...), int size, int64_t blocks, int threads, cudaStream_t stream, A... args) {
    if (size > 8) {                                         // more than the portable size: has to be asked for
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)size;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    return launch(&attr, kernel, dim3((unsigned)blocks), threads, stream, args...);
}

}  // namespace pb

#define PB_REFUSE(cond, text) \
    do { if (cond) return fail_text(PB_E_ARG, text); } while (0)

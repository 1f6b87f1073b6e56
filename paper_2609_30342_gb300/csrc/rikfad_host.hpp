// rikfad_host.hpp -- host helpers shared by the library's translation units.
#pragma once
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>
#include <string>

#include "rikfad.h"

namespace rikfad {

// Sets rikfad_last_error and returns `code` (defined beside it in rikfad.cu).
int report_error(int code, const std::string &msg);

// cudaMalloc and cudaFree, counted and with the injected failures of
// rikfad_debug_fail_allocation.
cudaError_t counted_malloc(void **p, size_t bytes);
void counted_free(void *p);

// The runtime's record of `e` is cleared: a refused launch is reported once.  (An
// error of work already enqueued stays and is reported by every later call.)
inline int report_cuda(cudaError_t e, const char *what)
{
    cudaGetLastError();
    return report_error(RIKFAD_ERR_CUDA, std::string(what) + ": " + cudaGetErrorName(e) + " (" +
                                             cudaGetErrorString(e) + ")");
}

// Every pointer that a kernel will dereference must be memory that the current
// device can address; a wrong one is an argument error, not a device fault.
int check_address(const void *p, int device, const char *what, int64_t index = -1);

// Programmatic stream serialisation, as for the kernels of a step: the kernel
// may begin while its predecessor finishes and waits (griddepcontrol.wait)
// before it touches any data.
template <typename Kern, typename... Args>
cudaError_t launch_chained(Kern kernel, dim3 blocks, int threads, size_t smem, cudaStream_t s, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

inline int dtype_bytes(int dtype) { return dtype == RIKFAD_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == RIKFAD_F32 || dtype == RIKFAD_BF16 || dtype == RIKFAD_F16; }

}  // namespace rikfad

// A C entry's body: no C++ exception leaves it.
#define RK_ENTRY_BEGIN try {
#define RK_ENTRY_END                                                                             \
    }                                                                                            \
    catch (const std::bad_alloc &)                                                               \
    {                                                                                            \
        return rikfad::report_error(RIKFAD_ERR_OOM, "host allocation failed: out of memory");    \
    }                                                                                            \
    catch (const std::exception &e)                                                              \
    {                                                                                            \
        return rikfad::report_error(RIKFAD_ERR_ARG, e.what());                                   \
    }

// What the host halves of the library's source files share: the launch counter, the facts of the current device and the
// driver's entry points (defined in tvm_attn_api.cu).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "tvm_attn.h"

namespace tvm_attn {

extern std::atomic<uint64_t> g_launches;   // kernels launched by this process

// What a call needs to know about the current device, looked up once per thread and CUDA context (the lookups cost a
// small call as much as a launch): a context's id is never used again in a process, so a device reset or a switch of
// devices is a new lookup.
struct DeviceFacts {
    unsigned long long ctx = 0;
    int sms = 0, major = 0;
    int* status = nullptr;   // device address of the status word that a bounded wait raises when it runs out
};

// The facts of the current device; null on error.
const DeviceFacts* device_facts();
// The facts of a device that runs the tensor-core kernels.
int tensor_core_device(const DeviceFacts** f);

typedef CUresult (*encode_tiled_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                    const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
encode_tiled_fn get_encode_fn();

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int cuda_status(cudaError_t e) { return e == cudaSuccess ? TVM_ATTN_OK : TVM_ATTN_CUDA_ERROR; }

}  // namespace tvm_attn

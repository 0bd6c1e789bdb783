// 16-byte chunks of rows of fp32 or bf16 elements, as the streaming kernels (norms, row sums) compute on them.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "sm100_ptx.cuh"

namespace tvm_attn {

template <typename T> struct RmsVec;
template <> struct RmsVec<float> { static constexpr int N = 4; };
template <> struct RmsVec<__nv_bfloat16> { static constexpr int N = 8; };

// A 16-byte chunk as pairs of floats in 64-bit registers, the operands of the two-wide fp32 instructions: the kernels
// spend half of the issue slots there are at full bandwidth on conversions and FMAs, one element at a time.
__device__ __forceinline__ void rms_unpack(const uint4& q, uint64_t (&v)[2]) {
    v[0] = ptx::pack2u(q.x, q.y);
    v[1] = ptx::pack2u(q.z, q.w);
}
__device__ __forceinline__ void rms_unpack(const uint4& q, uint64_t (&v)[4]) {   // a bf16 is the upper half of its float
    v[0] = ptx::pack2u(q.x << 16, q.x & 0xffff0000u);
    v[1] = ptx::pack2u(q.y << 16, q.y & 0xffff0000u);
    v[2] = ptx::pack2u(q.z << 16, q.z & 0xffff0000u);
    v[3] = ptx::pack2u(q.w << 16, q.w & 0xffff0000u);
}
__device__ __forceinline__ void rms_store(float* p, const uint64_t (&v)[2]) {
    float4 q;
    ptx::unpack2(v[0], q.x, q.y);
    ptx::unpack2(v[1], q.z, q.w);
    *reinterpret_cast<float4*>(p) = q;
}
__device__ __forceinline__ void rms_store(__nv_bfloat16* p, const uint64_t (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        ptx::unpack2(v[i], lo, hi);
        w[i] = ptx::pack_bf16(lo, hi);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float rms_hsum(uint64_t v) {
    float lo, hi;
    ptx::unpack2(v, lo, hi);
    return lo + hi;
}

}  // namespace tvm_attn

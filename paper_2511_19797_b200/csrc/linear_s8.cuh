// Products of 8-bit rows with 8-bit weights: the projections around the attention in a sampler.
//     y[m, n] = s[m] ws[n] sum_k q[m, k] w[n, k] + bias[n]
// q (M, K) with a scale for each row (token), w (N, K) with a scale for each row (output channel), both K-major; the sum is
// exact (32-bit integers), the rest is fp32 and rounded once to the output's type.
//
// mma.sync with 16 channels and 8 rows a warp: operands go from global memory
// straight to registers (a contraction does not care about the order of k: a lane's 16 contiguous bytes serve as its four
// operand words), the warps of a block share k, and the partial sums, integers, are added in shared memory.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "sm100_ptx.cuh"

namespace tvm_attn {

struct LinearParams {
    const int8_t* q;
    const int8_t* w;
    const float* s;
    const float* ws;
    const float* bias;   // or null
    void* y;
    long long ldq, ldw, ldy;   // elements between rows
    int M, N, K;
    int ksplit;          // warps of a block that share k (1, 2, 4, 8)
};

template <typename T> __device__ __forceinline__ T linear_round(float v);
template <> __device__ __forceinline__ float linear_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 linear_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// ------------------------------------------------------------------------------------------------ few rows
constexpr int LIN_FEW_THREADS = 256, LIN_FEW_UNROLL = 4;

// 16 bytes of a row of k, zeros behind its end (the memory behind it is not read).
__device__ __forceinline__ uint4 linear_load16(const int8_t* row, int k, int K, bool stream) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k + 16 <= K) {
        if (stream) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + k));
        else v = __ldg(reinterpret_cast<const uint4*>(row + k));
    } else if (k < K) {
        uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (k + j < K) b[j / 4] |= (uint32_t)(uint8_t)row[k + j] << (8 * (j & 3));
        v = make_uint4(b[0], b[1], b[2], b[3]);
    }
    return v;
}

__device__ __forceinline__ void linear_mma16832(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT groups of 8 rows of q a block.
template <typename OUT, int NT>
__global__ void __launch_bounds__(LIN_FEW_THREADS) linear_s8_few_kernel(const LinearParams p) {
    constexpr int WARPS = LIN_FEW_THREADS / 32, PITCH = 20;   // (16 channels of a token, and 4 against bank conflicts)
    __shared__ int part[WARPS][8 * NT][PITCH];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int KS = p.ksplit, RW = WARPS / KS, ks = warp % KS, rg = warp / KS;
    const int n0 = (blockIdx.x * RW + rg) * 16;
    const long long m0 = (long long)blockIdx.y * (8 * NT);
    int acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0;
    const bool lo_ok = n0 + g < p.N, hi_ok = n0 + g + 8 < p.N;
    const int8_t* w_lo = p.w + (lo_ok ? (long long)(n0 + g) * p.ldw : 0);
    const int8_t* w_hi = p.w + (hi_ok ? (long long)(n0 + g + 8) * p.ldw : 0);
    for (int k0 = ks * 64 * LIN_FEW_UNROLL; k0 < p.K; k0 += KS * 64 * LIN_FEW_UNROLL) {
        uint4 lo[LIN_FEW_UNROLL], hi[LIN_FEW_UNROLL];
#pragma unroll
        for (int u = 0; u < LIN_FEW_UNROLL; ++u) {
            const int k = k0 + 64 * u + 16 * t;
            lo[u] = linear_load16(w_lo, lo_ok ? k : p.K, p.K, true);
            hi[u] = linear_load16(w_hi, hi_ok ? k : p.K, p.K, true);
        }
#pragma unroll
        for (int u = 0; u < LIN_FEW_UNROLL; ++u) {
            const int k = k0 + 64 * u + 16 * t;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const long long m = m0 + 8 * j + g;
                const uint4 x = linear_load16(p.q + (m < p.M ? m : 0) * p.ldq, m < p.M ? k : p.K, p.K, false);
                linear_mma16832(acc[j], lo[u].x, hi[u].x, lo[u].y, hi[u].y, x.x, x.y);
                linear_mma16832(acc[j], lo[u].z, hi[u].z, lo[u].w, hi[u].w, x.z, x.w);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        part[warp][8 * j + 2 * t][g] = acc[j][0];
        part[warp][8 * j + 2 * t + 1][g] = acc[j][1];
        part[warp][8 * j + 2 * t][g + 8] = acc[j][2];
        part[warp][8 * j + 2 * t + 1][g + 8] = acc[j][3];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < RW * 16 * 8 * NT; i += LIN_FEW_THREADS) {
        const int c = i % (RW * 16), j = i / (RW * 16), n = blockIdx.x * RW * 16 + c;
        const long long m = m0 + j;
        if (n >= p.N || m >= p.M) continue;
        int sum = 0;
        for (int k = 0; k < KS; ++k) sum += part[(c / 16) * KS + k][j][c % 16];
        const float v = (float)sum * p.s[m] * p.ws[n];
        static_cast<OUT*>(p.y)[m * p.ldy + n] = linear_round<OUT>(p.bias ? v + p.bias[n] : v);
    }
}

}  // namespace tvm_attn
